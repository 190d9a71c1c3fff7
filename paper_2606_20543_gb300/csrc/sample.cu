// sample.cu — the sampler (include/ssd.h, ssd_sample): temperature, top-k,
// top-p and min-p from given uniforms.
//
// Weights are 32-bit integers, W = round(2^31 * 2^(-(max - x) c)), so every sum
// is exact and the result depends on no order of summation.  The entries kept
// are a prefix of the order (logit descending, index ascending): top-k cuts it by count,
// top-p by mass, min-p by weight.  One block of threads takes a row in three passes, the first
// from HBM and the others from L2 (a row of 65536 logits is 256 KB):
//  A the largest logit;
//  B a histogram of z = (max - x) c in bins of 1/64: the entries of each bin where
//    top-k cuts, its mass where top-p does (one 32-bit atomic for each: the weights
//    of a bin are cut to about 15 bits, so its mass is known from below and above).  They give
//    the bin of the k-th entry and the one or two bins that can hold the top-p cut;
//  C the exact weights: the mass of what is kept for certain, by chunks of 256
//    entries, and a list of the few entries in the bins where a cut falls.
// A radix search over the list (exact counts and masses) finds both cuts, ties are
// resolved by index, the listed entries that are kept join their chunks, and the chunk
// and the entry that hold u Z are found.  Where the bins of a cut hold more entries than
// the list takes (equal logits, high temperatures), the radix search runs over the row.
#include <algorithm>

#include "kernels.cuh"

namespace ssd {

namespace {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kChunk = 256;              // entries of a chunk, eight to a lane
constexpr int kBinsLog = 6;              // log2 of the bins per factor of two
constexpr float kBinsPerLog2 = 1 << kBinsLog;
constexpr int kBins = 32 << kBinsLog;    // weights down to 2^-32: below they are 0
constexpr float kMaxC = 0x1p100f;        // largest log2(e) / T
constexpr int kList = 4096;
constexpr float kLog2e = 1.4426950408889634f;
typedef unsigned long long u64;

struct SampleRow {
  float top, c;  // largest logit; kBinsPerLog2 * log2(e) / T
  float min_p;
  int32_t V;
  bool inf;      // the largest logit is infinite: logits count as 0 (infinite) or -inf
  const void* x;
};

// NaN counts as -inf, -0 as +0 (they compare equal).
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : x + 0.f; }
__device__ __forceinline__ float finite_or_not(float x) { return x == INFINITY ? 0.f : -INFINITY; }
// Order-preserving bits.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// Bins below the largest logit: z times a power of two, each operation of z rounded by
// itself.  NaN for a NaN, which no comparison lets through.
__device__ __forceinline__ float bins_of(const SampleRow& r, float x) {
  return __fmul_rn(__fsub_rn(r.top, x), r.c);
}
// 2^-z, 0 <= z <= 32.
__device__ __forceinline__ float weight_f(float bins) {
  return ex2_approx(bins * (-1.f / kBinsPerLog2));
}
__device__ __forceinline__ uint32_t weight_i(float w) { return __float2uint_rn(w * 0x1p31f); }

// How a row is read: vectors of 16 bytes where it is aligned, else entry by
// entry.  Lane l takes entries index(ch, u, l), u < 8, of chunk ch.
enum Mode { kF32Vec, kBf16Vec, kF32, kBf16 };
template <int MODE>
__device__ __forceinline__ int32_t index_of(int32_t ch, int u, int lane) {
  if (MODE == kF32Vec) return ch * kChunk + (u >> 2) * 128 + lane * 4 + (u & 3);
  if (MODE == kBf16Vec) return ch * kChunk + lane * 8 + u;
  return ch * kChunk + u * 32 + lane;
}
template <int MODE>
__device__ __forceinline__ float load1(const SampleRow& r, int32_t i) {
  const float x = MODE == kF32Vec || MODE == kF32
                      ? static_cast<const float*>(r.x)[i]
                      : __uint_as_float((uint32_t) static_cast<const uint16_t*>(r.x)[i] << 16);
  return r.inf ? finite_or_not(x) : x;
}
// The weight of any logit.
__device__ __forceinline__ uint32_t weight_of(const SampleRow& r, float x) {
  const float b = bins_of(r, x);
  return b < (float)kBins ? weight_i(weight_f(b)) : 0;
}
template <int MODE>
__device__ __forceinline__ void load8(const SampleRow& r, int32_t ch, int lane, float (&x)[8]) {
  if ((MODE == kF32Vec || MODE == kBf16Vec) && (ch + 1) * kChunk <= r.V) {
    if constexpr (MODE == kF32Vec) {
      const float4* p = static_cast<const float4*>(r.x) + ch * (kChunk / 4) + lane;
      const float4 a = p[0], b = p[32];
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
      x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
      const uint4 a = static_cast<const uint4*>(r.x)[ch * (kChunk / 8) + lane];
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
    if (r.inf) {
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = finite_or_not(x[u]);
    }
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int32_t i = index_of<MODE>(ch, u, lane);
      x[u] = i < r.V ? load1<MODE>(r, i) : -INFINITY;
    }
  }
}

struct SampleShared {
  uint32_t mass[kBins];  // of a bin, in units of 2^shift_of(bin)
  uint32_t cnt[kBins];
  uint32_t key[kList];   // the list
  int32_t idx[kList];
  u64 rmass[256];        // radix search
  uint32_t rcnt[256];
  u64 red[kSampleWarps];
  u64 red2[kSampleWarps];
  float redf[kSampleWarps];
  int32_t redi[kSampleWarps];
  uint32_t prefix;
  u64 need, above;
  int32_t n_list, cut_idx;
  int32_t bin_k, bin_lo, bin_hi;
  u64 upto_k_lo, upto_k_hi;
};

__device__ __forceinline__ u64 block_sum64(u64 v, u64* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int w = 0; w < kSampleWarps; ++w) s += red[w];
  return s;
}
// Inclusive scan over the block's threads.
__device__ __forceinline__ u64 block_scan64(u64 v, u64* red) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  __syncthreads();
  if (lane == 31) red[warp] = v;
  __syncthreads();
  for (int w = 0; w < warp; ++w) v += red[w];
  return v;
}
// Sum of at most 35-bit values over a warp.
__device__ __forceinline__ u64 warp_sum35(u64 v) {
  const uint32_t lo = __reduce_add_sync(0xffffffffu, (uint32_t)(v & 0xffffffu));
  const uint32_t hi = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 24));
  return ((u64)hi << 24) + lo;
}

// The entry of the order at which `need` entries (BY_COUNT) or a mass of `need`
// is reached among entries 0 .. n - 1 (at(i, &key): whether entry i takes part): its key,
// how many entries equal to it are within, and the mass of everything up to and including
// those.  need is at least 1 and at most the entries' count or mass.
template <bool BY_COUNT, typename At>
__device__ void select(const SampleRow& r, int32_t n, u64 need, SampleShared& sh, At at,
                       uint32_t* key, u64* n_eq, u64* mass) {
  if (threadIdx.x == 0) {
    sh.prefix = 0;
    sh.need = need;
    sh.above = 0;
  }
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (threadIdx.x < 256) {
      sh.rmass[threadIdx.x] = 0;
      sh.rcnt[threadIdx.x] = 0;
    }
    __syncthreads();
    const uint32_t prefix = sh.prefix;
#pragma unroll 1
    for (int32_t i = threadIdx.x; i < n; i += kSampleThreads) {
      uint32_t k;
      if (!at(i, &k)) continue;
      if (shift < 24 && (k >> (shift + 8)) != prefix) continue;
      const uint32_t d = (k >> shift) & 255u;
      atomicAdd(&sh.rcnt[d], 1u);
      const uint32_t w = weight_of(r, of_key(k));
      if (w != 0) atomicAdd(&sh.rmass[d], (u64)w);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
      // lane l: digits 255 - 8 l .. 248 - 8 l, descending
      const int lane = threadIdx.x;
      u64 v = 0, m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = 255 - 8 * lane - i;
        m += sh.rmass[d];
        v += BY_COUNT ? (u64)sh.rcnt[d] : sh.rmass[d];
      }
      u64 vi = v, mi = m;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 a = __shfl_up_sync(0xffffffffu, vi, o), b = __shfl_up_sync(0xffffffffu, mi, o);
        if (lane >= o) {
          vi += a;
          mi += b;
        }
      }
      const u64 left = sh.need, above = sh.above;
      __syncwarp();
      const uint32_t reach = __ballot_sync(0xffffffffu, vi >= left);
      if (lane == (reach ? __ffs(reach) - 1 : 31)) {
        u64 rest = left - (vi - v), over = above + (mi - m);
        int d = 255 - 8 * lane;
        for (int i = 0; i < 7; ++i, --d) {
          const u64 x = BY_COUNT ? (u64)sh.rcnt[d] : sh.rmass[d];
          if (x >= rest) break;
          rest -= x;
          over += sh.rmass[d];
        }
        sh.need = rest;
        sh.above = over;
        sh.prefix = (prefix << 8) | (uint32_t)d;
      }
    }
  }
  __syncthreads();
  *key = sh.prefix;
  const u64 w = weight_of(r, of_key(sh.prefix));
  *n_eq = BY_COUNT ? sh.need : (w > 0 ? (sh.need + w - 1) / w : 0);
  *mass = sh.above + *n_eq * w;
}

// Bits cut off the weights of bin b so that a row's sum stays in 32 bits; the
// sum of a bin is then short by less than 2^-kept of itself.
__device__ __forceinline__ int shift_of(int32_t b, int wide) {
  return max(0, (wide ? 20 : 16) - (b >> kBinsLog));
}

template <int MODE>
__global__ void __launch_bounds__(kSampleThreads, 2) sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(smem_raw);
  u64* chunk = reinterpret_cast<u64*>(smem_raw + sizeof(SampleShared));
  pdl_wait();
  const int32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t chunks = (a.V + kChunk - 1) / kChunk;
  // this warp's last chunk (negative: none)
  const int32_t last_chunk =
      warp < chunks ? warp + (chunks - 1 - warp) / kSampleWarps * kSampleWarps : -1;
  const int wide = a.V > 65536;
#pragma unroll 1
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
    const int32_t k = a.s.top_ks ? a.s.top_ks[row] : a.s.top_k;
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
    r.x = a.bf16 ? static_cast<const void*>(static_cast<const uint16_t*>(a.logits) + row * a.ld)
                 : static_cast<const void*>(static_cast<const float*>(a.logits) + row * a.ld);
    r.min_p = min_p;
    r.c = T > 0.f ? fminf(kLog2e / T, kMaxC) * kBinsPerLog2 : 1.f;
    r.inf = false;
    const bool greedy = T == 0.f || k == 1;
    const bool cut_k = k > 0 && k < r.V, cut_p = top_p < 1.f;

    // ---- A: the largest logit and its first index
    // (a NaN loses every comparison; the lane's chunk that holds its first largest is kept)
    float m = -INFINITY;
    int32_t mc = 0;
#pragma unroll 2
    for (int32_t ch = warp; ch < chunks; ch += kSampleWarps) {
      float x[8];
      load8<MODE>(r, ch, lane, x);
      const float y = fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], x[4], x[5]), fmaxf(x[6], x[7]));
      if (y > m) {
        m = y;
        mc = ch;
      }
    }
    for (int i = tid; i < kBins; i += kSampleThreads) {
      sh.mass[i] = 0;
      sh.cnt[i] = 0;
    }
    if (tid == 0) {
      sh.n_list = 0;
      sh.cut_idx = 0x7fffffff;
    }
    float wm = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
    if (lane == 0) sh.redf[warp] = wm;
    __syncthreads();
    r.top = sh.redf[0];
#pragma unroll
    for (int w = 1; w < kSampleWarps; ++w) r.top = fmaxf(r.top, sh.redf[w]);
    if (r.top == -INFINITY) {
      none();
      continue;
    }
    if (greedy) {
      int32_t at = 0x7fffffff;
      if (m == r.top) {
        for (int u = 7; u >= 0; --u) {
          const int32_t i = index_of<MODE>(mc, u, lane);
          if (i < r.V && load1<MODE>(r, i) == r.top) at = i;
        }
      }
      at = __reduce_min_sync(0xffffffffu, at);
      if (lane == 0) sh.redi[warp] = at;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < kSampleWarps; ++w) at = min(at, sh.redi[w]);
        a.out_tok[row] = at;
        if (a.prob) a.prob[row] = 1.f;
        if (a.kept) a.kept[row] = 1;
      }
      continue;
    }

    if (r.top == INFINITY) {
      r.inf = true;
      r.top = 0.f;
    }

    // ---- B: the bins of the cuts.  From the row's end, which was read last.
    u64 total = 0;  // mass of the row (with top-p)
    if (cut_k || cut_p) {
#pragma unroll 1
      for (int32_t ch = last_chunk; ch >= 0; ch -= kSampleWarps) {
        float x[8];
        load8<MODE>(r, ch, lane, x);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float z = bins_of(r, x[u]);
          const bool in = z < (float)kBins;
          const int32_t b = (int32_t)fminf(z, (float)kBins);
          if (cut_p) {
            const uint32_t w = weight_i(weight_f(fminf(z, (float)kBins)));  // 0 at kBins
            total += w;
            if (in) atomicAdd(&sh.mass[b], w >> shift_of(b, wide));
          }
          if (cut_k && in) atomicAdd(&sh.cnt[b], 1u);
        }
      }
      if (cut_p) total = block_sum64(total, sh.red);
      __syncthreads();
      // thread t: bins 4 t .. 4 t + 3 and the sums before them.  The mass up to a bin is
      // known from below and above by what was cut off the weights before it, and, with the
      // row's exact mass, by what was cut off behind it.
      constexpr int kPer = kBins / kSampleThreads;
      static_assert(kPer * kSampleThreads == kBins, "bins per thread");
      const float over = wide ? 0x1p-9f : 0x1p-13f;  // a bin's mass is short by less than this
      auto low_of = [&](int b) { return (u64)sh.mass[b] << shift_of(b, wide); };
      auto high_of = [&](int b) {
        const u64 q = low_of(b);
        return shift_of(b, wide) == 0 || q == 0 ? q : q + (u64)((float)q * over) + 1;
      };
      u64 n = 0, lo = 0, hi = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int b = tid * kPer + i;
        n += sh.cnt[b];
        lo += low_of(b);
        hi += high_of(b);
      }
      u64 n0 = 0, lo0 = 0, hi0 = 0, lo_all = 0, hi_all = 0;
      if (cut_k) n0 = block_scan64(n, sh.red) - n;
      if (cut_p) {
        lo0 = block_scan64(lo, sh.red) - lo;
        hi0 = block_scan64(hi, sh.red2) - hi;
        lo_all = block_sum64(lo, sh.red);
        hi_all = block_sum64(hi, sh.red2);
      }
      // mass up to a bin whose sums are l and h
      auto least_upto = [&](u64 l, u64 h) { return max(l, total + h > hi_all ? total + h - hi_all : 0); };
      auto most_upto = [&](u64 l, u64 h) { return min(h, total + l - lo_all); };
      if (tid == 0) {
        sh.bin_k = kBins;  // top-k takes every entry with a weight
        sh.bin_lo = sh.bin_hi = kBins;
        sh.upto_k_lo = sh.upto_k_hi = total;
      }
      __syncthreads();
      if (cut_k && n0 < (u64)k && (u64)k <= n0 + n) {
        u64 s = n0, l = lo0, h = hi0;
        for (int i = 0; i < kPer; ++i) {
          const int b = tid * kPer + i;
          if (s + sh.cnt[b] >= (u64)k) {
            sh.bin_k = b;
            sh.need = k - s;  // entries of the bin within top-k
            sh.upto_k_lo = least_upto(l, h);  // mass of the k entries, from below and above
            sh.upto_k_hi = most_upto(l + low_of(b), h + high_of(b));
            break;
          }
          s += sh.cnt[b];
          l += low_of(b);
          h += high_of(b);
        }
      }
      __syncthreads();
      if (cut_p) {
        const double p = top_p;
        const u64 least = (u64)ceil(p * (double)sh.upto_k_lo), most = (u64)ceil(p * (double)sh.upto_k_hi);
        u64 l = lo0, h = hi0;
        for (int i = 0; i < kPer; ++i) {
          const int b = tid * kPer + i;
          const u64 l1 = l + low_of(b), h1 = h + high_of(b);
          // the first bin by which the least wanted can be reached, and the first by
          // which the most wanted is: the cut is in one of them or between
          if (most_upto(l, h) < least && least <= most_upto(l1, h1)) sh.bin_lo = b;
          if (least_upto(l, h) < most && most <= least_upto(l1, h1)) sh.bin_hi = b;
          l = l1;
          h = h1;
        }
      }
      __syncthreads();
    }
    const int32_t bin_k = cut_k ? sh.bin_k : kBins;
    const u64 need_k = cut_k && bin_k < kBins ? sh.need : 0;
    const int32_t bin_lo = cut_p ? sh.bin_lo : kBins;
    const int32_t bin_hi = cut_p ? min(sh.bin_hi, kBins - 1) : -1;
    // entries kept for certain: z in bins below these
    const float sure = (float)min(bin_lo, bin_k);
    __syncthreads();

    // entries between the top-p bins and the top-k one count for top-p's mass
    const float gap = cut_p && bin_hi < bin_k && bin_k < kBins ? (float)(bin_hi + 1) : (float)kBins;
    const float behind = (float)min(kBins, cut_k && bin_k < kBins ? bin_k + 1 : bin_hi + 1);
    const float limit = cut_k || cut_p ? fmaxf(sure, behind) : (float)kBins;

    // ---- C: exact masses by chunk, and the list
    u64 upto = 0, mid = 0;  // masses before the listed bins, and between them
    uint32_t count = 0;
#pragma unroll 1
    for (int32_t ch = warp; ch < chunks; ch += kSampleWarps) {
      float x[8];
      load8<MODE>(r, ch, lane, x);
      float z[8], least = INFINITY;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        z[u] = bins_of(r, x[u]);
        least = fminf(least, z[u]);
      }
      u64 s = 0;
      if (__any_sync(0xffffffffu, least < limit)) {
        bool other = false;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float w = weight_f(fminf(z[u], (float)kBins));
          const bool in = z[u] < sure;
          const uint32_t wi = in ? weight_i(w) : 0;
          upto += wi;
          const uint32_t wk = w >= r.min_p ? wi : 0;
          s += wk;
          count += wk != 0;
          other |= !in && z[u] < limit;
        }
        if (other) {
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            if (!(z[u] >= sure && z[u] < limit)) continue;
            const int32_t b = (int32_t)z[u];
            if (b == bin_k || (b >= bin_lo && b <= bin_hi)) {
              const int32_t at = atomicAdd(&sh.n_list, 1);
              if (at < kList) {
                sh.key[at] = key_of(clean(x[u]));
                sh.idx[at] = index_of<MODE>(ch, u, lane);
              }
            } else if (z[u] >= gap) {
              mid += weight_i(weight_f(z[u]));
            }
          }
        }
        s = warp_sum35(s);
      }
      if (lane == 0) chunk[ch] = s;
    }
    if (cut_p) {
      upto = block_sum64(upto, sh.red);
      mid = block_sum64(mid, sh.red2);
    }
    __syncthreads();
    const int32_t n_list = sh.n_list;
    uint32_t cut = 0;
    u64 n_eq = ~0ull;
    if (n_list > kList) {
      // too many entries where a cut falls: the radix search over the whole row
      auto of_row = [&](int32_t i, uint32_t* key) {
        *key = key_of(clean(load1<MODE>(r, i)));
        return true;
      };
      u64 mass;
      total = 0;
      if (cut_k) {
        select<true>(r, r.V, (u64)k, sh, of_row, &cut, &n_eq, &total);
      } else {
        for (int32_t i = tid; i < r.V; i += kSampleThreads)
          total += weight_of(r, load1<MODE>(r, i));
        total = block_sum64(total, sh.red);
      }
      if (cut_p) {
        const u64 need = (u64)ceil((double)top_p * (double)total);
        select<false>(r, r.V, need, sh, of_row, &cut, &n_eq, &mass);
      }
      // index behind the last kept entry equal to the cut
      u64 seen = 0;
#pragma unroll 1
      for (int32_t i0 = 0; i0 < r.V && seen < n_eq; i0 += kSampleThreads) {
        const int32_t i = i0 + tid;
        const bool eq = i < r.V && key_of(clean(load1<MODE>(r, i))) == cut;
        const uint32_t ball = __ballot_sync(0xffffffffu, eq);
        __syncthreads();
        if (lane == 0) sh.redi[warp] = __popc(ball);
        __syncthreads();
        u64 before = seen;
        for (int w = 0; w < warp; ++w) before += sh.redi[w];
        if (eq && before + __popc(ball & ((1u << lane) - 1u)) + 1 == n_eq) sh.cut_idx = i + 1;
        for (int w = 0; w < kSampleWarps; ++w) seen += sh.redi[w];
      }
      __syncthreads();
    } else if (n_list > 0) {
      auto bin = [&](uint32_t key) { return (int32_t)bins_of(r, of_key(key)); };
      u64 in_k = 0, mass;  // mass of the entries of the top-k bin within top-k
      if (cut_k && bin_k < kBins) {
        auto of_k = [&](int32_t i, uint32_t* key) {
          *key = sh.key[i];
          return bin(*key) == bin_k;
        };
        select<true>(r, n_list, need_k, sh, of_k, &cut, &n_eq, &in_k);
      }
      if (cut_p) {
        // the k entries' mass: before, between and in the listed bins
        u64 s = 0;
        for (int32_t i = tid; i < n_list; i += kSampleThreads) {
          if (bin(sh.key[i]) != bin_k) s += weight_of(r, of_key(sh.key[i]));
        }
        s = block_sum64(s, sh.red);
        const u64 k_mass = bin_k < kBins ? upto + mid + s + in_k : total;
        const u64 need = (u64)ceil((double)top_p * (double)k_mass);
        auto listed = [&](int32_t i, uint32_t* key) {
          *key = sh.key[i];
          return true;
        };
        // (need > upto: the bins before the listed ones cannot reach it; the k-th
        // entry can, so no entry behind it gets in)
        select<false>(r, n_list, need - upto, sh, listed, &cut, &n_eq, &mass);
      }
      if (n_eq != ~0ull) {
        // the n_eq-th lowest index of the entries equal to the cut
        for (int32_t i = tid; i < n_list; i += kSampleThreads) {
          if (sh.key[i] != cut) continue;
          u64 below = 0;
          for (int32_t j = 0; j < n_list; ++j) below += sh.key[j] == cut && sh.idx[j] < sh.idx[i];
          if (below + 1 == n_eq) sh.cut_idx = sh.idx[i] + 1;
        }
      }
      __syncthreads();
    }
    const bool by_row = n_list > kList;
    const int32_t cut_idx = sh.cut_idx;
    auto kept_weight = [&](float x, int32_t i) -> uint32_t {
      const uint32_t kx = key_of(clean(x));
      const float z = bins_of(r, x);
      if (kx < cut || (kx == cut && i >= cut_idx) || !(z < (float)kBins)) return 0;
      const float w = weight_f(z);
      return w >= r.min_p ? weight_i(w) : 0;
    };
    // the listed entries that are kept, into their chunks (or every entry again)
    if (by_row) {
      count = 0;
#pragma unroll 1
      for (int32_t ch = warp; ch < chunks; ch += kSampleWarps) {
        float x[8];
        load8<MODE>(r, ch, lane, x);
        u64 s = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const uint32_t w = kept_weight(x[u], index_of<MODE>(ch, u, lane));
          s += w;
          count += w != 0;
        }
        s = warp_sum35(s);
        if (lane == 0) chunk[ch] = s;
      }
    } else {
      for (int32_t i = tid; i < n_list; i += kSampleThreads) {
        const uint32_t w = kept_weight(of_key(sh.key[i]), sh.idx[i]);
        if (w == 0) continue;
        ++count;
        atomicAdd(&chunk[sh.idx[i] / kChunk], (u64)w);
      }
    }
    const u64 n_kept = block_sum64(count, sh.red);

    // ---- the draw
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
      const uint32_t reach = __ballot_sync(0xffffffffu, incl > aim);
      const int32_t l0 = reach ? __ffs(reach) - 1 : 31;
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
#pragma unroll 1
      for (int32_t u = 0; u < 8 && pick < 0; ++u) {
        const int32_t i = ch * kChunk + u * 32 + lane;
        const uint32_t w = i < r.V ? kept_weight(load1<MODE>(r, i), i) : 0;
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
        if (a.kept) a.kept[row] = (int32_t)n_kept;
      }
    }
  }
}

template <int MODE>
cudaError_t launch(const SampleArgs& a, cudaStream_t stream) {
  const size_t smem = sizeof(SampleShared) + (size_t)((a.V + kChunk - 1) / kChunk) * sizeof(u64);
  const cudaError_t e = cudaFuncSetAttribute(
      sample_kernel<MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // a row per CTA, dealt by the hardware as CTAs end
  const unsigned blocks = (unsigned)std::min<int64_t>(a.rows, 1 << 20);
  return launch_kernel(sample_kernel<MODE>, dim3(blocks), dim3(kSampleThreads), smem, stream, true,
                       a);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, cudaStream_t stream) {
  const int64_t bytes = a.bf16 ? 2 : 4;
  const bool vec = (reinterpret_cast<uintptr_t>(a.logits) & 15u) == 0 && a.ld * bytes % 16 == 0;
  if (a.bf16) return vec ? launch<kBf16Vec>(a, stream) : launch<kBf16>(a, stream);
  return vec ? launch<kF32Vec>(a, stream) : launch<kF32>(a, stream);
}

}  // namespace ssd
