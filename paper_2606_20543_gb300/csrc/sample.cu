// sample.cu — the sampler (include/ssd.h, ssd_sample): temperature, top-k,
// top-p and min-p from given uniforms.
//
// Weights are 32-bit integers, W = round(2^31 * 2^(-(max - x) c)), so every sum
// is exact and the result depends on no order of summation.  The entries kept
// are a prefix of the order (logit descending, index ascending): top-k cuts it by count,
// top-p by mass and min-p by weight.  Both cuts are found by a radix search over
// the logits' bits, eight at a time: a histogram (count and mass) of the entries that share
// the digits found so far, and the digit where the count or the mass is
// reached.  Ties at the cut are resolved by index.  The draw sums the kept weights of
// every 256 entries, finds the chunk and then the entry.
#include <algorithm>

#include "kernels.cuh"

namespace ssd {

namespace {

constexpr int kThreads = 512;
constexpr int kSampleWarps = kThreads / 32;
constexpr int kChunkLog = 8;  // entries of a chunk of the draw: 256
constexpr int kMaxChunks = kSampleMaxV >> kChunkLog;
constexpr float kLog2e = 1.4426950408889634f;
typedef unsigned long long u64;

struct SampleRow {
  float top, c;     // largest logit, log2(e) / T
  float min_p;
  int32_t V;
  const void* x;
  int32_t bf16;
};

// Logit i; NaN counts as -inf, and -0 as +0 (they compare equal).
__device__ __forceinline__ float logit(const SampleRow& r, int32_t i) {
  const float x = r.bf16
                      ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(r.x)[i] << 16)
                      : static_cast<const float*>(r.x)[i];
  return x != x ? -INFINITY : x + 0.f;
}
// Order-preserving bits.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ float weight_f(const SampleRow& r, float x) {
  return x == r.top ? 1.f : exp2f(-__fmul_rn(__fsub_rn(r.top, x), r.c));
}
__device__ __forceinline__ uint32_t weight_i(float w) { return __float2uint_rn(w * 0x1p31f); }

struct SampleShared {
  u64 mass[256];
  uint32_t cnt[256];
  u64 red[kSampleWarps];
  float redf[kSampleWarps];
  int32_t redi[kSampleWarps];
  uint32_t prefix;   // key bits found
  u64 need;          // entries or mass still to be reached below the digits found
  u64 above;         // mass of the entries above them
  int32_t cut_idx;
  int32_t pick;
};

__device__ __forceinline__ u64 warp_sum64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ u64 block_sum64(u64 v, SampleShared& sh) {
  v = warp_sum64(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.red[threadIdx.x >> 5] = v;
  __syncthreads();
  u64 s = 0;
  for (int w = 0; w < kSampleWarps; ++w) s += sh.red[w];
  return s;
}

// The entry of the order at which `need` entries (BY_COUNT) or a mass of `need`
// is reached: its key, how many entries equal to it are within (n_eq), the
// mass of everything up to and including those.  need is at least 1 and at most
// the row's count or mass.
template <bool BY_COUNT>
__device__ void select(const SampleRow& r, u64 need, SampleShared& sh, uint32_t* key, u64* n_eq,
                       u64* mass) {
  if (threadIdx.x == 0) {
    sh.prefix = 0;
    sh.need = need;
    sh.above = 0;
  }
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += kThreads) {
      sh.mass[i] = 0;
      sh.cnt[i] = 0;
    }
    __syncthreads();
    const uint32_t prefix = sh.prefix;
    for (int32_t i = threadIdx.x; i < r.V; i += kThreads) {
      const float x = logit(r, i);
      const uint32_t k = key_of(x);
      if (shift < 24 && (k >> (shift + 8)) != prefix) continue;
      const uint32_t d = (k >> shift) & 255u;
      atomicAdd(&sh.cnt[d], 1u);
      const uint32_t w = weight_i(weight_f(r, x));
      if (w != 0) atomicAdd(&sh.mass[d], (u64)w);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      u64 left = sh.need, above = sh.above;
      int d = 255;
      for (; d > 0; --d) {
        const u64 v = BY_COUNT ? (u64)sh.cnt[d] : sh.mass[d];
        if (v >= left) break;
        left -= v;
        above += sh.mass[d];
      }
      sh.need = left;
      sh.above = above;
      sh.prefix = (prefix << 8) | (uint32_t)d;
    }
    __syncthreads();
  }
  *key = sh.prefix;
  const u64 w = weight_i(weight_f(r, of_key(sh.prefix)));
  *n_eq = BY_COUNT ? sh.need : (w > 0 ? (sh.need + w - 1) / w : 0);
  *mass = sh.above + *n_eq * w;
  __syncthreads();
}

__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  __shared__ u64 chunk[kMaxChunks];
  pdl_wait();
  const int32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    __syncthreads();
    auto none = [&]() {
      if (tid == 0) {
        a.out_tok[row] = -1;
        if (a.prob) a.prob[row] = 0.f;
        if (a.kept) a.kept[row] = 0;
      }
    };
    if (a.s.n_drafts != nullptr) {
      const int32_t b = row / a.s.D_max;
      if (row - b * a.s.D_max >= a.s.n_drafts[b]) {
        none();
        continue;
      }
    }
    const float T = a.s.temperatures ? a.s.temperatures[row] : a.s.temperature;
    int32_t k = a.s.top_ks ? a.s.top_ks[row] : a.s.top_k;
    const float top_p = a.s.top_ps ? a.s.top_ps[row] : a.s.top_p;
    const float min_p = a.s.min_ps ? a.s.min_ps[row] : a.s.min_p;
    if (!(T >= 0.f) || T == INFINITY || k < 0 || !(top_p > 0.f && top_p <= 1.f) ||
        !(min_p >= 0.f && min_p <= 1.f)) {
      if (tid == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      none();
      continue;
    }
    SampleRow r;
    r.V = a.V;
    r.bf16 = a.bf16;
    r.x = a.bf16 ? static_cast<const void*>(static_cast<const uint16_t*>(a.logits) + row * a.ld)
                 : static_cast<const void*>(static_cast<const float*>(a.logits) + row * a.ld);
    r.min_p = min_p;
    r.c = T > 0.f ? kLog2e / T : 1.f;
    // ---- the largest logit and its first index
    float m = -INFINITY;
    int32_t mi = 0x7fffffff;
    for (int32_t i = tid; i < r.V; i += kThreads) {
      const float x = logit(r, i);
      if (x > m) {
        m = x;
        mi = i;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float y = __shfl_xor_sync(0xffffffffu, m, o);
      const int32_t yi = __shfl_xor_sync(0xffffffffu, mi, o);
      if (y > m || (y == m && yi < mi)) {
        m = y;
        mi = yi;
      }
    }
    if (lane == 0) {
      sh.redf[warp] = m;
      sh.redi[warp] = mi;
    }
    __syncthreads();
    for (int w = 0; w < kSampleWarps; ++w)
      if (sh.redf[w] > m || (sh.redf[w] == m && sh.redi[w] < mi)) {
        m = sh.redf[w];
        mi = sh.redi[w];
      }
    r.top = m;
    if (m == -INFINITY) {
      none();
      continue;
    }
    if (T == 0.f || k == 1) {
      if (tid == 0) {
        a.out_tok[row] = mi;
        if (a.prob) a.prob[row] = 1.f;
        if (a.kept) a.kept[row] = 1;
      }
      continue;
    }
    // ---- the cut
    uint32_t cut = 0;
    u64 n_eq = ~0ull, total;
    if (k > 0 && k < r.V) {
      select<true>(r, (u64)k, sh, &cut, &n_eq, &total);
    } else {
      u64 s = 0;
      for (int32_t i = tid; i < r.V; i += kThreads) s += weight_i(weight_f(r, logit(r, i)));
      total = block_sum64(s, sh);
    }
    if (top_p < 1.f) {
      const u64 need = (u64)ceil((double)top_p * (double)total);
      u64 mass;
      select<false>(r, need, sh, &cut, &n_eq, &mass);
    }
    // index behind the last kept entry equal to the cut
    if (tid == 0) sh.cut_idx = 0x7fffffff;
    if (n_eq != ~0ull) {
      u64 seen = 0;
      for (int32_t i0 = 0; i0 < r.V; i0 += kThreads) {
        const int32_t i = i0 + tid;
        const bool eq = i < r.V && key_of(logit(r, i)) == cut;
        const uint32_t ball = __ballot_sync(0xffffffffu, eq);
        __syncthreads();
        if (lane == 0) sh.redi[warp] = __popc(ball);
        __syncthreads();
        u64 before = seen;
        for (int w = 0; w < warp; ++w) before += sh.redi[w];
        if (eq && before + __popc(ball & ((1u << lane) - 1u)) + 1 == n_eq) sh.cut_idx = i + 1;
        for (int w = 0; w < kSampleWarps; ++w) seen += sh.redi[w];
        if (seen >= n_eq) break;
      }
    }
    __syncthreads();
    const int32_t cut_idx = sh.cut_idx;
    auto kept_weight = [&](int32_t i) -> uint32_t {
      if (i >= r.V) return 0;
      const float x = logit(r, i);
      const uint32_t kx = key_of(x);
      if (kx < cut || (kx == cut && i >= cut_idx)) return 0;
      const float w = weight_f(r, x);
      return w >= r.min_p ? weight_i(w) : 0;
    };
    // ---- the draw
    const int32_t chunks = (r.V + (1 << kChunkLog) - 1) >> kChunkLog;
    u64 count = 0;
    for (int32_t ch = warp; ch < chunks; ch += kSampleWarps) {
      u64 s = 0;
      for (int32_t u = 0; u < 8; ++u) {
        const uint32_t w = kept_weight((ch << kChunkLog) + u * 32 + lane);
        s += w;
        count += w != 0;
      }
      s = warp_sum64(s);
      if (lane == 0) chunk[ch] = s;
    }
    count = block_sum64(count, sh);
    if (warp == 0) {
      const int32_t per = (chunks + 31) / 32;
      u64 s = 0;
      for (int32_t i = 0; i < per; ++i) s += lane * per + i < chunks ? chunk[lane * per + i] : 0;
      u64 incl = s;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      const u64 Z = __shfl_sync(0xffffffffu, incl, 31);
      const u64 aim = (u64)((double)row_uniforms(a.rng, row).y * (double)Z);
      // sums are whole: sum > u Z iff sum > floor(u Z)
      const uint32_t over = __ballot_sync(0xffffffffu, incl > aim);
      const int32_t l0 = over ? __ffs(over) - 1 : 31;
      int32_t ch = 0;
      u64 before = incl - s;
      if (lane == l0) {
        for (ch = lane * per; ch < min(chunks, (lane + 1) * per) - 1; ++ch) {
          if (before + chunk[ch] > aim) break;
          before += chunk[ch];
        }
      }
      ch = __shfl_sync(0xffffffffu, ch, l0);
      before = __shfl_sync(0xffffffffu, before, l0);
      int32_t pick = -1;
      uint32_t wp = 0;
      for (int32_t u = 0; u < 8 && pick < 0; ++u) {
        const int32_t i = (ch << kChunkLog) + u * 32 + lane;
        const uint32_t w = kept_weight(i);
        u64 c = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const u64 y = __shfl_up_sync(0xffffffffu, c, o);
          if (lane >= o) c += y;
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, before + c > aim);
        if (hit) {
          pick = __shfl_sync(0xffffffffu, i, __ffs(hit) - 1);
          wp = __shfl_sync(0xffffffffu, w, __ffs(hit) - 1);
        }
        before += __shfl_sync(0xffffffffu, c, 31);
      }
      if (lane == 0) {
        a.out_tok[row] = pick;
        if (a.prob) a.prob[row] = (float)((double)wp / (double)Z);
        if (a.kept) a.kept[row] = (int32_t)count;
      }
    }
  }
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, cudaStream_t stream) {
  const unsigned blocks = (unsigned)std::min<int64_t>(a.rows, 4 * (int64_t)device_sm_count());
  return launch_kernel(sample_kernel, dim3(blocks), dim3(kThreads), 0, stream, true, a);
}

}  // namespace ssd
