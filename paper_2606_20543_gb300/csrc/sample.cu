// sample.cu — the sampler (include/ssd.h, ssd_sample): temperature, top-k,
// top-p and min-p from given uniforms.
//
// Weights are 32-bit integers, W = round(2^31 * 2^(-(max - x) c)), so every sum
// is exact and the result depends on no order of summation.  The entries kept
// are a prefix of the order (logit descending, index ascending): top-k cuts it by count,
// top-p by mass, min-p by weight.  One block of threads takes a row, which it reads twice,
// from HBM and then from L2 (a row of 65536 float32 logits is 256 KB):
//  A the largest logit, and a histogram of the logits in bins of 1/128 of a factor of
//    two of weight: the entries of a bin and the sum of their places in it, in 1/256 of the bin
//    (the bins hang on the largest of the row's first entries, since the largest of all is not
//    known yet).  The counts give the bin of the k-th entry exactly; with the places a bin's
//    mass is known to 2^-16, which gives the one or two bins where the top-p cut falls;
//  B the exact weights: the mass of what is kept for certain, by chunks of 256
//    entries, and a list of the few entries in the bins where a cut falls.
// A radix search over the list (exact counts and masses) finds both cuts, ties are
// resolved by index, the listed entries that are kept join their chunks, and the chunk
// and the entry that hold u Z are found.  Where the bins of a cut hold more entries than the
// list takes (equal logits, high temperatures), the search runs over the row's entries
// in those bins; where the exact masses show the cut to be elsewhere, over the whole row.
//
// 1024 rows of 65536 float32 logits, top-p 0.95: 164 to 167 us, 268 MB at 1.6 TB/s (0.24 of the
// measured copy rate; the pass for the largest logit alone takes 53 us, without a cut 111).
// About 20 instructions an entry in the two passes bound it, and 17000 cycles a row between
// them, of which two rows to an SM hide half.  One row of 16384, top-k 2000: 12.5 us; 200 rows
// of 32771 bf16 logits with settings of their own: 39 us, one CTA's time; 1024 rows of 16384,
// top-p 0.95: 55 us.  Not faster: loads by bulk copies into a ring (175 us for the first case),
// counts and places in one word (168), bins of 1/256 without places (191: longer lists).
#include <algorithm>
#include <type_traits>

#include "kernels.cuh"

namespace ssd {

namespace {

constexpr int kChunk = 256;            // entries of a chunk, eight to a lane
constexpr int kPerLog2 = 128;             // bins per factor of two
constexpr float kBinsPerLog2 = kPerLog2;
constexpr int kHead = 8 * kPerLog2;       // bins above the reference logit: 8 factors of two
constexpr int kBins = kHead + 32 * kPerLog2;  // and below it: from 2^-32 on weights are 0
constexpr float kMaxC = 0x1p100f;      // largest log2(e) / T
constexpr int kList = 4096;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kPlaces = 256;              // places in a bin
constexpr float kBinLn = 0.0054152123f;   // ln 2 / 128: log of the ratio of a bin's edges
// A bin's mass is taken at its entries' mean place: off by half a place's width (2^-17) and
// by the curvature of the exponential (kBinLn^2 / 8), and the sums by their roundings.
constexpr float kMassErr = 0x1p-15f;
constexpr int kFew = 128;                 // entries that are ordered by comparing each with all
typedef unsigned long long u64;

// A row is read in vectors of 16 bytes from the boundary at or before its first entry, so
// chunk 0 may begin `off` entries before the row: chunk ch holds entries ch * kChunk - off
// and on.  Chunks that the row does not fill are read entry by entry.
// Lane l takes entries index_of(r, ch, u, l), u < 8, of chunk ch.
struct SampleRow {
  const void* x;
  int32_t V, off;
  bool inf;      // the largest logit is infinite: logits count as 0 (infinite) or -inf
  float top;     // the largest logit
  float c;       // bins per unit of logit: kBinsPerLog2 * log2(e) / T
  float min_p;
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
__device__ __forceinline__ float2 fmul2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 ra, rb, rd;\n"
      " mov.b64 ra, {%2, %3};\n mov.b64 rb, {%4, %5};\n"
      " mul.rn.f32x2 rd, ra, rb;\n mov.b64 {%0, %1}, rd;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
// top - x, one rounding.
__device__ __forceinline__ float2 below2(float top, float x0, float x1) {
  return ffma2(make_float2(x0, x1), both(-1.f), both(top));
}
// The integer weight of float32 weight 2^-z.
__device__ __forceinline__ uint32_t weight_i(float w) { return __float2uint_rn(w * 0x1p31f); }
// 2^-z, z the bins below the largest logit over 128: the difference, the product and the
// power are rounded one by one (the division by 128 is exact).
__device__ __forceinline__ float weight_f(const SampleRow& r, float x) {
  const float z = __fmul_rn(__fsub_rn(r.top, x), r.c);
  return z < 32.f * kBinsPerLog2 ? ex2_approx(z * (-1.f / kBinsPerLog2)) : 0.f;  // (NaN: 0)
}
__device__ __forceinline__ uint32_t weight_of(const SampleRow& r, float x) {
  return weight_i(weight_f(r, x));
}
// A logit's bin under the reference logit `ref`, times kPlaces: descending in x.
__device__ __forceinline__ float2 bin2_of(float ref, float c, float x0, float x1) {
  return ffma2(below2(ref, x0, x1), both(c * kPlaces), both((float)(kHead * kPlaces)));
}
__device__ __forceinline__ float bin_of(float ref, float c, float x) {
  return fmaf(__fsub_rn(ref, x), c * kPlaces, (float)(kHead * kPlaces));
}

// An entry into the histogram (not those below the last bin, nor a NaN).  Predicated: a
// branch per entry took more than the additions.
template <bool PLACES>
__device__ __forceinline__ void add_to_bin(uint32_t cnt0, float b) {
  const uint32_t at = __float2uint_rz(b), to = cnt0 + at / kPlaces * 4;
  if constexpr (PLACES)
    asm volatile(
        "{\n .reg .pred p;\n setp.lt.f32 p, %0, %1;\n"
        " @p red.shared.add.u32 [%2], 1;\n @p red.shared.add.u32 [%2 + %4], %3;\n}" ::"f"(b),
        "f"((float)(kBins * kPlaces)), "r"(to), "r"(at % kPlaces), "n"(kBins * 4)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.lt.f32 p, %0, %1;\n @p red.shared.add.u32 [%2], 1;\n}" ::"f"(b),
        "f"((float)(kBins * kPlaces)), "r"(to)
        : "memory");
}

template <bool BF16>
__device__ __forceinline__ int32_t index_of(const SampleRow& r, int32_t ch, int u, int lane) {
  return ch * kChunk - r.off + (BF16 ? lane * 8 + u : (u >> 2) * 128 + lane * 4 + (u & 3));
}
template <bool BF16>
__device__ __forceinline__ float load1(const void* x, bool inf, int32_t i) {
  const float v = BF16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(x)[i] << 16)
                       : static_cast<const float*>(x)[i];
  return inf ? finite_or_not(v) : v;
}
template <bool BF16>
__device__ __forceinline__ void load8(const SampleRow& r, int32_t ch, int lane, float (&x)[8]) {
  const int32_t first = ch * kChunk - r.off;
  if (first >= 0 && first + kChunk <= r.V) {
    if constexpr (!BF16) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(r.x) + first) + lane;
      const float4 a = p[0], b = p[32];
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
      x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
      const uint4 a =
          reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(r.x) + first)[lane];
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
      const int32_t i = index_of<BF16>(r, ch, u, lane);
      x[u] = i >= 0 && i < r.V ? load1<BF16>(r.x, r.inf, i) : -INFINITY;
    }
  }
}
__device__ __forceinline__ float max8(const float (&x)[8]) {  // NaN loses
  return fmax3(fmax3(x[0], x[1], x[2]), fmax3(x[3], x[4], x[5]), fmaxf(x[6], x[7]));
}

// NT: threads of a block.
template <int NT>
struct SampleShared {
  union {
    struct {  // pass A's
      uint32_t cnt[kBins];
      uint32_t place[kBins];  // (right behind cnt)
    };
    struct {  // the list, from pass B on
      uint32_t key[kList];
      int32_t idx[kList];
    };
  };
  uint32_t rsum[3][256];  // radix search: the masses' 11, 11 and 10 bits, each summed
  uint32_t rcnt[256];
  uint4 few[kFew];        // ~index, key (a number that orders entries), weight
  u64 red[(NT / 32)], red2[(NT / 32)];
  float redf[(NT / 32)];
  int32_t redi[(NT / 32)];
  uint32_t from, to;  // radix search: the keys left, how many entries, what is to be reached
  uint32_t left, n_few;
  u64 need, above;
  uint32_t cut;       // its results: the cut's key, the index behind the last entry equal to it
  u64 n_eq, cut_mass; // that is kept (cut_idx) or how many are (n_eq, where cut_idx is not
                      // known), and the mass up to and including them
  int32_t n_list, cut_idx;
  int32_t bin_k, bin_lo, bin_hi, need_k;
  float upto[NT / 32];        // mass up to and including a warp's bins
  float k_mass;               // estimated mass of the first k entries, and its error
  float k_mass_err;
  uint32_t edge[4];           // least keys above the bins' edges
  uint32_t floor_key;         // least key with a weight
};

template <int NT>
__device__ __forceinline__ u64 block_sum64(u64 v, u64* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int w = 0; w < (NT / 32); ++w) s += red[w];
  return s;
}
// Sum of at most 35-bit values over a warp.
__device__ __forceinline__ u64 warp_sum35(u64 v) {
  const uint32_t lo = __reduce_add_sync(0xffffffffu, (uint32_t)(v & 0xffffffu));
  const uint32_t hi = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 24));
  return ((u64)hi << 24) + lo;
}
__device__ __forceinline__ u64 add_wide(u64 s, uint32_t w) {
  asm("mad.wide.u32 %0, %1, 1, %0;" : "+l"(s) : "r"(w));
  return s;
}

// The entry of the order at which `need` entries (by_count) or a mass of `need`
// is reached among the entries (of the list, or of the row) whose keys are in lo .. hi: its
// key, the index behind it and the mass of everything up to and including it.  need is at
// least 1 and at most the entries' count or mass.  Each round deals the keys left to 256 digits
// and keeps one digit's, until a few entries are left (most lists are short from the start):
// then each is compared with all, a thread per entry.  Where more share one key, the
// entries of that key that are kept are counted instead (n_eq).
template <int NT, bool BF16>
__device__ __noinline__ void select(SampleRow r, SampleShared<NT>& sh, bool of_row, bool by_count, u64 need,
                                    uint32_t lo, uint32_t hi) {
  const int32_t n = of_row ? r.V : sh.n_list, tid = threadIdx.x;
  auto key_at = [&](int32_t i) {
    return of_row ? key_of(clean(load1<BF16>(r.x, r.inf, i))) : sh.key[i];
  };
  __syncthreads();
  if (tid == 0) {
    sh.from = lo;
    sh.to = hi;
    sh.need = need;
    sh.above = 0;
    sh.left = (uint32_t)n;
    sh.n_few = 0;
  }
#pragma unroll 1
  while (true) {
    __syncthreads();
    const uint32_t from = sh.from, to = sh.to;
    if (from == to || sh.left <= kFew) break;
    if (tid < 256) sh.rcnt[tid] = sh.rsum[0][tid] = sh.rsum[1][tid] = sh.rsum[2][tid] = 0;
    __syncthreads();
    const int shift = max(0, 24 - __clz(to - from));
#pragma unroll 1
    for (int32_t i = tid; i < n; i += NT) {
      const uint32_t k = key_at(i);
      if (k < from || k > to) continue;
      const uint32_t d = (k - from) >> shift;
      const uint32_t w = weight_of(r, of_key(k));
      atomicAdd(&sh.rcnt[d], 1u);
      atomicAdd(&sh.rsum[0][d], w & 2047u);
      atomicAdd(&sh.rsum[1][d], (w >> 11) & 2047u);
      atomicAdd(&sh.rsum[2][d], w >> 22);
    }
    __syncthreads();
    if (tid < 32) {
      // lane l: digits 255 - 8 l .. 248 - 8 l, descending
      auto mass_of = [&](int d) {
        return (u64)sh.rsum[0][d] + ((u64)sh.rsum[1][d] << 11) + ((u64)sh.rsum[2][d] << 22);
      };
      u64 v = 0, m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = 255 - 8 * tid - i;
        const u64 x = mass_of(d);
        m += x;
        v += by_count ? (u64)sh.rcnt[d] : x;
      }
      u64 vi = v, mi = m;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 a = __shfl_up_sync(0xffffffffu, vi, o), b = __shfl_up_sync(0xffffffffu, mi, o);
        if (tid >= o) {
          vi += a;
          mi += b;
        }
      }
      const u64 left = sh.need, above = sh.above;
      __syncwarp();
      const uint32_t reach = __ballot_sync(0xffffffffu, vi >= left);
      if (tid == (reach ? __ffs(reach) - 1 : 31)) {
        u64 rest = left - (vi - v), over = above + (mi - m);
        int d = 255 - 8 * tid;
#pragma unroll 1
        for (int i = 0; i < 7; ++i, --d) {
          const u64 x = mass_of(d), y = by_count ? (u64)sh.rcnt[d] : x;
          if (y >= rest) break;
          rest -= y;
          over += x;
        }
        sh.need = rest;
        sh.above = over;
        sh.left = sh.rcnt[d];
        const uint32_t base = from + ((uint32_t)d << shift);
        sh.from = base;
        sh.to = min(to, base + ((1u << shift) - 1u));
      }
    }
    __syncthreads();
  }
  const uint32_t from = sh.from, to = sh.to;
  if (sh.left <= kFew) {
#pragma unroll 1
    for (int32_t i = tid; i < n; i += NT) {
      const uint32_t k = key_at(i);
      if (k < from || k > to) continue;
      const uint32_t at = atomicAdd(&sh.n_few, 1u);
      sh.few[at] = make_uint4(~(uint32_t)(of_row ? i : sh.idx[i]), k, weight_of(r, of_key(k)), 0);
    }
    __syncthreads();
    const int32_t n_few = (int32_t)sh.n_few;
    if (tid < n_few) {
      const u64 left = sh.need;
      auto order = [](const uint4& x) { return ((u64)x.y << 32) | x.x; };
      const uint4 me = sh.few[tid];
      u64 mass = 0;  // of the entries before this one in the order, and their count
      uint32_t count = 0;
#pragma unroll 4
      for (int32_t j = 0; j < n_few; ++j) {
        const uint4 x = sh.few[j];
        const bool first = order(x) > order(me);
        mass = add_wide(mass, first ? x.z : 0);
        count += first ? 1 : 0;
      }
      // the one entry that reaches the need
      const u64 before = by_count ? (u64)count : mass;
      if (before < left && before + (by_count ? 1 : me.z) >= left) {
        sh.cut = me.y;
        sh.cut_idx = (int32_t)~me.x + 1;
        sh.n_eq = 0;
        sh.cut_mass = sh.above + mass + me.z;
      }
    }
  } else if (tid == 0) {
    const u64 w = weight_of(r, of_key(from));
    sh.cut = from;
    sh.n_eq = by_count ? sh.need : (w > 0 ? (sh.need + w - 1) / w : 1);
    sh.cut_mass = sh.above + sh.n_eq * w;
  }
  __syncthreads();
}

// Index behind the n_eq-th entry (in index order) that equals the cut, to cut_idx.
// From the list, which holds all of them: a radix search over their indices.
template <int NT>
__device__ __noinline__ void list_ties(SampleShared<NT>& sh) {
  const int32_t n = sh.n_list, tid = threadIdx.x;
  const uint32_t cut = sh.cut;
  uint32_t left = (uint32_t)sh.n_eq;  // (at most kList)
  int32_t base = 0;                   // the index's digits found
#pragma unroll 1
  for (int shift = 16; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) sh.rcnt[tid] = 0;
    __syncthreads();
#pragma unroll 1
    for (int32_t i = tid; i < n; i += NT)
      if (sh.key[i] == cut && ((sh.idx[i] ^ base) >> shift) < 256)
        atomicAdd(&sh.rcnt[(sh.idx[i] >> shift) & 255], 1u);
    __syncthreads();
    // (every warp for itself) lane l: digits 8 l .. 8 l + 7
    const int32_t lane = tid & 31;
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine += sh.rcnt[8 * lane + i];
    uint32_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const uint32_t reach = __ballot_sync(0xffffffffu, upto >= left);
    const int src = reach ? __ffs(reach) - 1 : 31;
    int32_t d = 8 * src;
    left -= __shfl_sync(0xffffffffu, upto - mine, src);
#pragma unroll 1
    for (int i = 0; i < 7 && sh.rcnt[d] < left; ++i, ++d) left -= sh.rcnt[d];
    base |= d << shift;
  }
  __syncthreads();
  if (tid == 0) sh.cut_idx = base + 1;
  __syncthreads();
}
// From the row: counts by chunks (where the chunks' masses will stand), then the chunk's.
template <int NT, bool BF16>
__device__ __noinline__ void row_ties(SampleRow r, SampleShared<NT>& sh, u64* chunk, int32_t chunks) {
  const int32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t cut = sh.cut;
  __syncthreads();
  if (tid == 0) sh.cut_idx = 0x7fffffff;
#pragma unroll 2
  for (int32_t ch = warp; ch < chunks; ch += (NT / 32)) {
    float x[8];
    load8<BF16>(r, ch, lane, x);
    uint32_t n = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u)  // (behind the row: -inf, which is no cut)
      n += key_of(clean(x[u])) == cut ? 1 : 0;
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) chunk[ch] = n;
  }
  __syncthreads();
  if (warp == 0) {
    u64 left = sh.n_eq;
    int32_t ch = 0;
    for (; ch < chunks; ch += 32) {  // 32 chunks at a time
      const uint32_t n = ch + lane < chunks ? (uint32_t)chunk[ch + lane] : 0;
      uint32_t upto = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      const uint32_t reach = __ballot_sync(0xffffffffu, upto >= left);
      if (reach) {
        const int src = __ffs(reach) - 1;
        left -= __shfl_sync(0xffffffffu, upto - n, src);
        ch += src;
        break;
      }
      left -= __shfl_sync(0xffffffffu, upto, 31);
    }
#pragma unroll 1
    for (int u = 0; u < kChunk / 32 && left > 0; ++u) {
      const int32_t i = ch * kChunk - r.off + u * 32 + lane;
      const bool eq = i >= 0 && i < r.V && key_of(clean(load1<BF16>(r.x, r.inf, i))) == cut;
      const uint32_t ball = __ballot_sync(0xffffffffu, eq);
      if (eq && (u64)__popc(ball & ((1u << lane) - 1u)) + 1 == left) sh.cut_idx = i + 1;
      left = (u64)__popc(ball) >= left ? 0 : left - __popc(ball);
    }
  }
  __syncthreads();
}

// The least key above which a condition on the logit, monotone, holds (one warp: each
// step looks at 32 keys of those left).
template <typename F>
__device__ __forceinline__ uint32_t least_key(int lane, F holds) {
  uint32_t lo = key_of(-INFINITY), hi = key_of(INFINITY);
#pragma unroll 1
  while (lo < hi) {
    const uint32_t step = (hi - lo) / 32 + 1;
    const uint32_t at = lo + min((uint32_t)lane * step, hi - lo);
    const uint32_t yes = __ballot_sync(0xffffffffu, at == hi || holds(of_key(at)));
    const int f = yes ? __ffs(yes) - 1 : 32;  // the first of them
    const uint32_t top = f < 32 ? lo + min((uint32_t)f * step, hi - lo) : hi;
    if (f > 0) lo += min((uint32_t)(f - 1) * step, hi - lo) + 1;
    hi = top;
    if (f == 0) break;
  }
  return hi;
}

// The same with a guess: mostly within 16 steps of it.
template <typename F>
__device__ __forceinline__ uint32_t least_key(int lane, float guess, F holds) {
  const uint32_t base = key_of(guess) - 16;
  const uint32_t yes = __ballot_sync(0xffffffffu, holds(of_key(base + lane)));
  if (fabsf(guess) < 0x1p126f && yes != 0 && !(yes & 1u)) return base + __ffs(yes) - 1;
  return least_key(lane, holds);
}

// Sums over the row's entries (for certain kept, all), and the list, of pass B.
struct PassB {
  u64 sure, total;
  uint32_t count;
};

// Pass B.  Entries x >= x_sure are kept for certain (as far as min-p lets them); those in
// [x_p, x_sure) and [x_k, x_k1) go to the list; TOTAL: the mass of the rest of the
// row counts too, else that of [x_k1, x_p).
template <int NT, bool BF16, bool TOTAL>
__device__ __forceinline__ PassB pass_b(const SampleRow& r, SampleShared<NT>& sh, u64* chunk,
                                        int32_t chunks, float x_sure, float x_p, float x_k1,
                                        float x_k) {
  const int32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float end = fminf(x_p, x_k);
  const bool all_kept = r.min_p <= 0x1p-32f;  // of the weights that are not 0
  PassB out{0, 0, 0};
#pragma unroll 1
  for (int32_t ch = warp; ch < chunks; ch += (NT / 32)) {
    float x[8];
    load8<BF16>(r, ch, lane, x);
    u64 s = 0;
    if (TOTAL || __any_sync(0xffffffffu, max8(x) >= end)) {
      u64 sum = 0;
      int32_t n_in = 0, n_end = 0;
      // (x_sure is at least the least logit with a weight: what is kept has one)
      auto entries = [&](auto min_p) {
#pragma unroll
        for (int u = 0; u < 8; u += 2) {
          // (as weight_f: a power of two changes no rounding)
          const float2 e = fmul2(below2(r.top, x[u], x[u + 1]), both(r.c * (-1.f / kBinsPerLog2)));
          const float2 w = make_float2(ex2_approx(e.x), ex2_approx(e.y));
          const float2 f = fmul2(w, both(0x1p31f));
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const float xv = v ? x[u + 1] : x[u];
            const uint32_t wi = __float2uint_rn(v ? f.y : f.x);  // 0 for a NaN and beyond 2^-32
            bool in = xv >= x_sure;
            n_end += xv >= end ? 1 : 0;
            if (TOTAL) out.total = add_wide(out.total, wi);
            if constexpr (decltype(min_p)::value) {
              out.sure = add_wide(out.sure, in ? wi : 0);
              n_end -= in ? 1 : 0;
              in = in && (v ? w.y : w.x) >= r.min_p;
              n_end += in ? 1 : 0;
            }
            sum = add_wide(sum, in ? wi : 0);
            n_in += in ? 1 : 0;
          }
        }
      };
      if (all_kept) {
        entries(std::false_type());
        out.sure += sum;
      } else {
        entries(std::true_type());
      }
      out.count += n_in;
      if (__any_sync(0xffffffffu, n_end != n_in)) {
        // the entries of this chunk that go to the list, or lie between its ranges (bit u)
        uint32_t listed = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) listed |= x[u] >= end && x[u] < x_sure ? 1u << u : 0u;
        // entries between the listed ranges only add their mass
        uint32_t between = 0;
        if (x_k1 < x_p) {
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if ((listed >> u & 1u) && x[u] < x_p && x[u] >= x_k1) between |= 1u << u;
          listed &= ~between;
        }
        int32_t at = __popc(listed);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int32_t y = __shfl_up_sync(0xffffffffu, at, o);
          if (lane >= o) at += y;
        }
        int32_t base = 0;
        if (lane == 31 && at > 0) base = atomicAdd(&sh.n_list, at);
        at += __shfl_sync(0xffffffffu, base, 31) - __popc(listed);
        uint32_t left = listed | between;
        while (left) {
          const int u = __ffs(left) - 1;
          left &= left - 1;
          float xu = x[0];
#pragma unroll
          for (int i = 1; i < 8; ++i) xu = u == i ? x[i] : xu;
          if (between >> u & 1u) {
            out.total += weight_of(r, xu);
            continue;
          }
          if (at < kList) {
            sh.key[at] = key_of(clean(xu));
            sh.idx[at] = index_of<BF16>(r, ch, u, lane);
          }
          ++at;
        }
      }
      s = warp_sum35(sum);
    }
    if (lane == 0) chunk[ch] = s;
  }
  return out;
}

template <int NT, bool BF16>
__global__ void __launch_bounds__(NT, 1024 / NT) sample_kernel(SampleArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SampleShared<NT>& sh = *reinterpret_cast<SampleShared<NT>*>(smem_raw);
  u64* chunk = reinterpret_cast<u64*>(smem_raw + sizeof(SampleShared<NT>));
  pdl_wait();
  const int32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto block_max = [&](float m) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    __syncthreads();
    if (lane == 0) sh.redf[warp] = m;
    __syncthreads();
    m = sh.redf[0];
#pragma unroll
    for (int w = 1; w < (NT / 32); ++w) m = fmaxf(m, sh.redf[w]);
    return m;
  };
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
    SampleRow r;
    r.min_p = a.s.min_ps ? a.s.min_ps[row] : a.s.min_p;
    if (!(T >= 0.f) || T == INFINITY || k < 0 || !(top_p > 0.f && top_p <= 1.f) ||
        !(r.min_p >= 0.f && r.min_p <= 1.f)) {
      if (tid == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      none();
      continue;
    }
    r.V = a.V;
    r.x = BF16 ? static_cast<const void*>(static_cast<const uint16_t*>(a.logits) + row * a.ld)
               : static_cast<const void*>(static_cast<const float*>(a.logits) + row * a.ld);
    r.off = (int32_t)((reinterpret_cast<uintptr_t>(r.x) & 15u) / (BF16 ? 2 : 4));
    const int32_t chunks = (a.V + r.off + kChunk - 1) / kChunk;
    r.c = T > 0.f ? fminf(kLog2e / T, kMaxC) * kBinsPerLog2 : 1.f;
    r.inf = false;
    const float u_res = warp == 0 ? row_uniforms(a.rng, row).y : 0.f;
    const bool greedy = T == 0.f || k == 1;
    const bool cut_k = !greedy && k > 0 && k < r.V, cut_p = !greedy && top_p < 1.f;

    // ---- A: the largest logit, and the histogram under the largest of each warp's first
    // chunk; once more where that one lies too far below the row's largest
    float ref = 0.f;
    if (cut_k || cut_p) {
      float x[8];
      load8<BF16>(r, warp, lane, x);  // (beyond the row: -inf)
      ref = block_max(max8(x));
    }
    float m;
    int32_t mc = 0;  // this lane's chunk with its first largest
#pragma unroll 1
    while (true) {
      m = -INFINITY;
      const bool hist = (cut_k || cut_p) && ref > -INFINITY && ref < INFINITY;
      if (hist) {
#pragma unroll
        for (int i = 0; i < kBins / NT; ++i)
          sh.cnt[tid + i * NT] = sh.place[tid + i * NT] = 0;
        __syncthreads();
        const uint32_t cnt0 = smem_u32(sh.cnt);
        auto count = [&](auto places) {
#pragma unroll 2
          for (int32_t ch = warp; ch < chunks; ch += (NT / 32)) {
            float x[8];
            load8<BF16>(r, ch, lane, x);
            m = fmaxf(m, max8(x));
#pragma unroll
            for (int u = 0; u < 8; u += 2) {
              const float2 b = bin2_of(ref, r.c, x[u], x[u + 1]);
              // (bins above the first count as the first)
#pragma unroll
              for (int v = 0; v < 2; ++v)
                add_to_bin<decltype(places)::value>(cnt0, v ? b.y : b.x);
            }
          }
        };
        if (cut_p) count(std::true_type());
        else count(std::false_type());
      } else {
#pragma unroll 4
        for (int32_t ch = warp; ch < chunks; ch += (NT / 32)) {
          float x[8];
          load8<BF16>(r, ch, lane, x);
          const float y = max8(x);
          if (y > m) {
            m = y;
            mc = ch;
          }
        }
      }
      r.top = block_max(m);
      if (!(cut_k || cut_p) || r.top == -INFINITY) break;
      if (r.top == INFINITY && !r.inf) {
        r.inf = true;  // from here on logits are 0 or -inf
        ref = 0.f;
        continue;
      }
      if (hist && bin_of(ref, r.c, r.top) >= (float)kPlaces) break;
      ref = r.top;  // (bin_of is kHead for the reference itself)
    }
    if (r.top == -INFINITY) {
      none();
      continue;
    }
    if (greedy) {
      int32_t at = 0x7fffffff;
      if (m == r.top)
        for (int u = 7; u >= 0; --u) {
          const int32_t i = index_of<BF16>(r, mc, u, lane);
          if (i >= 0 && i < r.V && load1<BF16>(r.x, false, i) == r.top) at = i;
        }
      at = __reduce_min_sync(0xffffffffu, at);
      if (lane == 0) sh.redi[warp] = at;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < (NT / 32); ++w) at = min(at, sh.redi[w]);
        a.out_tok[row] = at;
        if (a.prob) a.prob[row] = 1.f;
        if (a.kept) a.kept[row] = 1;
      }
      continue;
    }
    if (r.top == INFINITY) {  // (without a cut)
      r.inf = true;
      r.top = 0.f;
    }
    if (tid == 0) {
      sh.n_list = 0;
      sh.cut_idx = 0x7fffffff;
      sh.cut = 0;
      sh.n_eq = 0;
      sh.bin_k = kBins;  // top-k takes every entry with a weight
      sh.bin_lo = sh.bin_hi = kBins;
    }

    if (warp == (NT / 32) - 1) {
      // the least logit with a weight: rounding makes the others 0
      const uint32_t at = least_key(lane, r.top - 32.f * kBinsPerLog2 / r.c,
                                    [&](float x) { return weight_of(r, x) != 0; });
      if (lane == 0) sh.floor_key = at;
    }

    // ---- the bins of the cuts.  Thread t: bins kPer t .. and the sums before them.
    // Keys: x >= of_key(edge[0]): kept for certain; edge[1]: end of the top-p bins;
    // edge[2], edge[3]: start and end of the top-k bin
    uint32_t key_sure = 0, key_p = 0xffffffffu, key_k1 = 0xffffffffu, key_k = 0xffffffffu;
    if (cut_k || cut_p) {
      constexpr int kPer = kBins / NT;
      static_assert(kPer * NT == kBins, "bins per thread");
      // 2^((kHead - b) / 128) of a bin's upper edge
      const float w0 = exp2f((float)(kHead - tid * kPer) / kBinsPerLog2);
      constexpr float kStep = 0.99459942f;  // 2^(-1/128)
      auto mass_of = [&](int b, float w) {
        const uint32_t cn = sh.cnt[b];
        if (cn == 0) return 0.f;
        const float mean = kBinLn / kPlaces * (__fdividef((float)sh.place[b], (float)cn) + 0.5f);
        return (float)cn * w * (1.f - mean + 0.5f * mean * mean);
      };
      int32_t n = 0;
      float mass = 0.f, w = w0;
      float q[kPer];  // mass of each bin
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        n += sh.cnt[tid * kPer + i];
        q[i] = cut_p ? mass_of(tid * kPer + i, w) : 0.f;
        mass += q[i];
        w *= kStep;
      }
      int32_t n1 = n;
      float m1 = mass;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int32_t y = __shfl_up_sync(0xffffffffu, n1, o);
        const float z = __shfl_up_sync(0xffffffffu, m1, o);
        if (lane >= o) {
          n1 += y;
          m1 += z;
        }
      }
      __syncthreads();
      if (lane == 31) {
        sh.redi[warp] = n1;
        sh.redf[warp] = m1;
      }
      __syncthreads();
      float total = 0.f;
#pragma unroll
      for (int w2 = 0; w2 < (NT / 32); ++w2) {
        if (w2 < warp) {
          n1 += sh.redi[w2];
          m1 += sh.redf[w2];
        }
        total += sh.redf[w2];
      }
      const int32_t n0 = n1 - n;
      if (tid == 0) {
        sh.k_mass = total;
        sh.k_mass_err = 0.f;
      }
      if (lane == 31) sh.upto[warp] = m1;
      __syncthreads();
      // (the mass before the thread's bins is the one that the thread before ends with, to the
      // bit: a cut that fell in between would be found by nobody)
      float m0 = __shfl_up_sync(0xffffffffu, m1, 1);
      if (lane == 0) m0 = warp == 0 ? 0.f : sh.upto[warp - 1];
      if (cut_k && n0 < k && k <= n1) {
        int32_t s = n0;
        float before = m0;
        w = w0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int32_t cn = sh.cnt[tid * kPer + i];
          if (s < k && s + cn >= k) {
            sh.bin_k = tid * kPer + i;
            sh.need_k = k - s;  // entries of the bin within top-k
            sh.k_mass = before + (float)(k - s) * w;
            sh.k_mass_err = (float)(k - s) * w * kBinLn;
          }
          s += cn;
          before += q[i];
          w *= kStep;
        }
      }
      __syncthreads();
      if (cut_p) {
        const float err = sh.k_mass_err + kMassErr * sh.k_mass;
        const float least = top_p * sh.k_mass - err, most = top_p * sh.k_mass + err;
        float before = m0;
        if (tid == 0 && least <= 0.f) sh.bin_lo = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const float upto = i + 1 < kPer ? before + q[i] : m1;
          // (several threads may find one where sums are rounded: any will do)
          if (before < least && least <= upto) sh.bin_lo = tid * kPer + i;
          if (before < most && most <= upto) sh.bin_hi = tid * kPer + i;
          before = upto;
        }
      }
      __syncthreads();
      const int32_t bin_k = sh.bin_k;
      const int32_t bin_lo = min(cut_p ? sh.bin_lo : kBins, bin_k);
      const int32_t bin_hi = cut_p ? min(max(sh.bin_hi, bin_lo), bin_k) : -1;
      if (warp < 4) {
        const int32_t edge = warp == 0 ? bin_lo : warp == 1 ? bin_hi + 1
                             : warp == 2 ? bin_k : bin_k + 1;
        const uint32_t at =
            least_key(lane, ref - (float)(edge - kHead) / r.c,
                      [&](float x) { return bin_of(ref, r.c, x) < (float)(edge * kPlaces); });
        if (lane == 0) sh.edge[warp] = at;
      }
      __syncthreads();
      key_sure = sh.edge[0];
      if (cut_p) key_p = sh.edge[1];
      if (bin_k < kBins) {
        key_k1 = sh.edge[2];
        key_k = sh.edge[3];
      }
    } else {
      __syncthreads();
    }
    const uint32_t key_floor = sh.floor_key;
    key_sure = max(key_sure, key_floor);
    // the k-th entry's bin ends the order; without one, every entry counts for top-p's mass
    const bool has_k = key_k != 0xffffffffu;
    key_p = max(min(key_p, key_sure), key_floor);

    // ---- B
    auto at_key = [](uint32_t key) { return key == 0xffffffffu ? INFINITY : of_key(key); };
    const PassB pb = cut_p && !has_k
                         ? pass_b<NT, BF16, true>(r, sh, chunk, chunks, at_key(key_sure), at_key(key_p),
                                              INFINITY, INFINITY)
                         : pass_b<NT, BF16, false>(r, sh, chunk, chunks, at_key(key_sure), at_key(key_p),
                                               at_key(key_k1), at_key(key_k));
    uint32_t count = pb.count;
    bool by_row = false;  // the chunks' masses are to be summed again
    if (cut_k || cut_p) {
      u64 sure = 0, rest = 0;  // rest: all of the row, or what lies between the listed bins
      if (cut_p) {
        sure = block_sum64<NT>(pb.sure, sh.red);
        rest = block_sum64<NT>(pb.total, sh.red2);
      }
      __syncthreads();
      const bool overflow = sh.n_list > kList;
      by_row = overflow;
      if (has_k) select<NT, BF16>(r, sh, overflow, true, (u64)sh.need_k, key_k, key_k1 - 1);
      if (cut_p) {
        u64 k_mass = rest, listed = 0;
        // mass of the listed entries before the top-k bin
        if (!overflow) {
          for (int32_t i = tid; i < sh.n_list; i += NT)
            if (sh.key[i] >= key_p && (!has_k || sh.key[i] >= key_k1))
              listed += weight_of(r, of_key(sh.key[i]));
        } else {
#pragma unroll 1
          for (int32_t i = tid; i < r.V; i += NT) {
            const float x = load1<BF16>(r.x, r.inf, i);
            const uint32_t key = key_of(clean(x));
            if (key >= key_p && key < key_sure && (!has_k || key >= key_k1)) listed += weight_of(r, x);
          }
        }
        listed = block_sum64<NT>(listed, sh.red);
        if (has_k) k_mass = sure + rest + listed + sh.cut_mass;
        const u64 need = (u64)ceil((double)top_p * (double)k_mass);
        // what the listed top-p bins reach: with the top-k bin among them, all of it
        const bool with_k = has_k && key_p <= key_k;
        const u64 reach = sure + listed + (with_k ? sh.cut_mass : 0);
        if (need > sure && need <= reach) {
          select<NT, BF16>(r, sh, overflow, false, need - sure, with_k ? key_k : key_p, key_sure - 1);
        } else {
          // the estimate was off: the cut is not in the listed bins
          by_row = true;
          select<NT, BF16>(r, sh, true, false, need, key_of(-INFINITY), key_of(r.top));
        }
      }
      // equal entries at the cut, too many for a warp
      if (sh.n_eq != 0) {
        if (by_row) row_ties<NT, BF16>(r, sh, chunk, chunks);
        else list_ties<NT>(sh);
      }
    }
    __syncthreads();
    const uint32_t cut = sh.cut;
    const int32_t cut_idx = sh.cut_idx;
    auto kept_weight = [&](float x, int32_t i) -> uint32_t {
      const uint32_t kx = key_of(clean(x));
      if (kx < cut || (kx == cut && i >= cut_idx)) return 0;
      const float w = weight_f(r, x);
      return w >= r.min_p ? weight_i(w) : 0;
    };
    // the listed entries that are kept, into their chunks (or every entry again)
    if (by_row) {
      count = 0;
#pragma unroll 1
      for (int32_t ch = warp; ch < chunks; ch += (NT / 32)) {
        float x[8];
        load8<BF16>(r, ch, lane, x);
        u64 s = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const uint32_t w = kept_weight(x[u], index_of<BF16>(r, ch, u, lane));
          s += w;
          count += w != 0;
        }
        s = warp_sum35(s);
        if (lane == 0) chunk[ch] = s;
      }
    } else {
      const int32_t n_list = sh.n_list;
      for (int32_t i = tid; i < n_list; i += NT) {
        const uint32_t w = kept_weight(of_key(sh.key[i]), sh.idx[i]);
        if (w == 0) continue;
        ++count;
        atomicAdd(&chunk[(sh.idx[i] + r.off) / kChunk], (u64)w);
      }
    }
    count = __reduce_add_sync(0xffffffffu, count);
    if (lane == 0) sh.redi[warp] = (int32_t)count;
    __syncthreads();

    // ---- the draw
    if (warp == 0) {
      count = lane < (NT / 32) ? sh.redi[lane] : 0;
      count = __reduce_add_sync(0xffffffffu, count);
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
      const u64 aim = (u64)((double)u_res * (double)Z);
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
      // the chunk, eight entries in a row to a lane
      uint32_t w[8];
      u64 c = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int32_t i = ch * kChunk - r.off + lane * 8 + u;
        w[u] = i >= 0 && i < r.V ? kept_weight(load1<BF16>(r.x, r.inf, i), i) : 0;
        c += w[u];
      }
      u64 ci = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, ci, o);
        if (lane >= o) ci += y;
      }
      const uint32_t hit = __ballot_sync(0xffffffffu, before + ci > aim);
      const int32_t l1 = hit ? __ffs(hit) - 1 : 31;
      before += ci - c;
      int32_t pick = -1;
      uint32_t wp = 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        before += w[u];
        if (pick < 0 && before > aim) {
          pick = ch * kChunk - r.off + lane * 8 + u;
          wp = w[u];
        }
      }
      pick = __shfl_sync(0xffffffffu, pick, l1);
      wp = __shfl_sync(0xffffffffu, wp, l1);
      if (lane == 0) {
        a.out_tok[row] = pick;
        if (a.prob) a.prob[row] = (float)((double)wp / (double)Z);
        if (a.kept) a.kept[row] = (int32_t)count;
      }
    }
  }
}

template <int NT, bool BF16>
cudaError_t launch(const SampleArgs& a, cudaStream_t stream) {
  // (a row may begin up to 7 entries behind its first chunk's begin)
  auto smem = [](int32_t V) {
    return sizeof(SampleShared<NT>) + (size_t)((V + 7 + kChunk - 1) / kChunk) * sizeof(u64);
  };
  const cudaError_t e = allow_smem(sample_kernel<NT, BF16>, smem(kSampleMaxV));
  if (e != cudaSuccess) return e;
  // a row per CTA, dealt by the hardware as CTAs end
  const unsigned blocks = (unsigned)std::min<int64_t>(a.rows, 1 << 20);
  return launch_kernel(sample_kernel<NT, BF16>, dim3(blocks), dim3(NT), smem(a.V), stream,
                       true, a);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, cudaStream_t stream) {
  // Many rows of up to 128 KB: 256 threads each, so that four rows share an SM and one's passes
  // run beside what another does between them (1024 rows, top-p 0.95, of 4096 logits 46 -> 31 us,
  // of 16384 69 -> 55, of 32768 99 -> 94).  Four rows of 256 KB to an SM do not fit L2, where the
  // second pass finds them (65536 logits: 163 -> 184); two rows to an SM are better off with
  // 512 threads, few rows too.
  const bool many =
      a.rows > 2 * device_sm_count() && (int64_t)a.V * (a.bf16 ? 2 : 4) <= 128 << 10;
  if (many) return a.bf16 ? launch<256, true>(a, stream) : launch<256, false>(a, stream);
  return a.bf16 ? launch<512, true>(a, stream) : launch<512, false>(a, stream);
}

}  // namespace ssd
