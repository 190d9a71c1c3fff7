// cache.cu — the paged 8-bit cache (include/ssd.h): the plan (block tables,
// slot maps and positions from request lengths), the rotary table and the
// append (rotary positions with three axes, e4m3 blocks with a scale per head).
#include <algorithm>

#include "e4m3.cuh"

namespace ssd {

namespace {

// ------------------------------------------------------------------- plan
// One kernel, no workspace.  A block of 256 threads takes either up to 256
// whole sequences (short rows) or a piece of one sequence's row of slots, about
// kPlanSlots slots each.  Where its first sequence's blocks start in the ring
// is the sum of the demands before it, which every block adds up itself: 12
// bytes per sequence from L2, less than the hand-over between two kernels
// costs.  A launch and a chain of five loads bound it: 2.8 us for 16 sequences of
// one token, 5.4 us (1.1 TB/s) for 256 prompts of up to 1088 tokens, which write 5.7 MB.
constexpr int kPlanThreads = 256;
constexpr int kPlanSlots = 1024;

struct PlanSeq {
  int32_t cache, n, held, demand;  // n < 0: bad lengths
};

__device__ __forceinline__ PlanSeq plan_load(const CachePlanArgs& a, int32_t b) {
  PlanSeq q;
  q.cache = a.cache_len[b];
  q.n = a.n_new[b];
  q.held = a.held[b];
  q.demand = 0;
  const int64_t need =
      ((int64_t)q.cache + q.n + (1 << a.block_log) - 1) >> a.block_log;
  if (q.cache < 0 || q.n < 0 || q.n > a.N_max || q.held < 0 || q.held > a.max_blocks ||
      need > a.max_blocks) {
    q.n = -1;
  } else {
    q.demand = max(0, (int32_t)need - q.held);
  }
  return q;
}

// Sum over the block; every thread gets it.
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();  // red may still be read from the call before
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  int64_t s = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 32; ++w) s += red[w];
  return s;
}

struct PlanRow {
  int64_t base;  // ring index of the first new block
  int32_t cache, n, held, served;
};

// per: sequences of a block; pieces: blocks of a sequence (one of them is 1)
__global__ void __launch_bounds__(kPlanThreads)
cache_plan_kernel(CachePlanArgs a, int32_t per, int32_t pieces) {
  __shared__ int64_t red[kPlanThreads / 32];
  __shared__ PlanRow rows[kPlanThreads];
  pdl_wait();
  const int32_t tid = threadIdx.x;
  const int32_t unit = blockIdx.x;
  const int32_t b0 = pieces > 1 ? unit / pieces : unit * per;
  const int32_t piece = pieces > 1 ? unit - b0 * pieces : 0;
  const int32_t nb = min(per, a.B - b0);
  const int64_t head = *a.head, tail = *a.tail;
  const bool ring_ok = head >= 0 && tail >= head && tail - head <= a.ring_size;

  int64_t before = 0;
  for (int32_t b = tid; b < b0; b += kPlanThreads) before += plan_load(a, b).demand;
  before = block_sum(before, red);

  // the block's sequences, one per thread, and an inclusive scan of their demands
  PlanSeq q{0, 0, 0, 0};
  if (tid < nb) q = plan_load(a, b0 + tid);
  int64_t s = q.demand;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, s, o);
    if ((tid & 31) >= o) s += y;
  }
  __syncthreads();
  if ((tid & 31) == 31) red[tid >> 5] = s;
  __syncthreads();
  for (int w = 0; w < (tid >> 5); ++w) s += red[w];
  const int64_t stop = head + before + s;
  if (tid < nb) {
    const int32_t b = b0 + tid;
    const bool fits = ring_ok && stop <= tail;
    const bool ok = q.n >= 0 && ring_ok;
    const bool served = ok && (fits || q.demand == 0);
    rows[tid] = PlanRow{(stop - q.demand) % a.ring_size, q.cache, q.n, q.held, served ? 1 : 0};
    if (piece == 0) {
      a.n_blocks[b] = served ? q.held + q.demand : q.held;
      if (!ok) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      else if (!served) record_status(a.status, SSD_ERR_WORKSPACE);
      // the end of the last demand that fits: demands fit up to some sequence
      // and no further
      if (!ring_ok) {
        if (b == 0) *a.next_head = head;
      } else {
        const bool last = b == a.B - 1;
        const int64_t next = last ? 0 : stop + plan_load(a, b + 1).demand;
        if (fits && (last || next > tail)) *a.next_head = stop;
        if (!fits && b == 0) *a.next_head = head;
      }
    }
  }
  __syncthreads();

  // block table: the new entries
  if (pieces == 1) {
    for (int32_t r = tid >> 5; r < nb; r += kPlanThreads / 32) {
      const PlanRow w = rows[r];
      if (!w.served) continue;
      const int32_t n = ((w.cache + w.n + (1 << a.block_log) - 1) >> a.block_log) - w.held;
      for (int32_t i = tid & 31; i < n; i += 32) {
        int64_t at = w.base + i;
        if (at >= a.ring_size) at -= a.ring_size;
        a.block_table[(int64_t)(b0 + r) * a.max_blocks + w.held + i] = a.ring[at];
      }
    }
  } else if (rows[0].served) {
    const PlanRow w = rows[0];
    const int32_t n = ((w.cache + w.n + (1 << a.block_log) - 1) >> a.block_log) - w.held;
    for (int32_t i = piece * kPlanThreads + tid; i < n; i += pieces * kPlanThreads) {
      int64_t at = w.base + i;
      if (at >= a.ring_size) at -= a.ring_size;
      a.block_table[(int64_t)b0 * a.max_blocks + w.held + i] = a.ring[at];
    }
  }

  // slots and positions.  A token in a new block takes its id from the ring:
  // the table's entry is another thread's write.
  const int32_t lo = pieces > 1 ? piece * kPlanSlots : 0;
  const int32_t hi = pieces > 1 ? min(a.N_max, lo + kPlanSlots) : a.N_max;
  const int32_t width = hi - lo;
  const int32_t S = 1 << a.block_log, P = a.grid.prefix_len;
  for (int32_t x = tid; x < nb * width; x += kPlanThreads) {
    const int32_t r = nb == 1 ? 0 : x / width;
    const int32_t j = lo + x - r * width;
    const PlanRow w = rows[r];
    const int64_t at = (int64_t)(b0 + r) * a.N_max + j;
    int64_t slot = -1;
    int32_t p0 = 0, p1 = 0, p2 = 0;
    if (w.served && j < w.n) {
      const int32_t p = w.cache + j, i = p >> a.block_log;
      int32_t id;
      if (i < w.held) {
        id = a.block_table[(int64_t)(b0 + r) * a.max_blocks + i];
      } else {
        int64_t k = w.base + (i - w.held);
        if (k >= a.ring_size) k -= a.ring_size;
        id = a.ring[k];
      }
      slot = (int64_t)id * S + (p & (S - 1));
      if (p < P) {
        p0 = p1 = p2 = p;
      } else if (a.pos != nullptr) {
        const int32_t g = p - P, y = g / a.grid.row_stride;
        p0 = P;
        p1 = P + y;
        p2 = P + (g - y * a.grid.row_stride);
      }
    }
    a.slots[at] = slot;
    if (a.pos != nullptr) {
      a.pos[3 * at] = p0;
      a.pos[3 * at + 1] = p1;
      a.pos[3 * at + 2] = p2;
    }
  }
}

// ----------------------------------------------------------- rotary table
// Once per model: angles and functions in 64 bits (which this GPU does slowly), so that a
// position of any size keeps its accuracy.
__global__ void rotary_table_kernel(int32_t n, int32_t pairs, const float* freq, float2* table) {
  pdl_wait();
  for (int32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) {
    const int32_t p = i / pairs;
    double s, c;
    sincos((double)p * (double)freq[i - p * pairs], &s, &c);
    table[i] = make_float2((float)c, (float)s);
  }
}

// ----------------------------------------------------------------- append
// Rotation of 16 values of a head: 8 from column c8 on in a, 8 from column c8 +
// d/2 on in b.  Products and sums are rounded one by one (no fused
// multiply-add), so the result does not depend on how a compiler pairs them.
// kFused (behind a norm, whose results are rounded in any case): one rounding less, and two
// instructions of six.
template <bool kFused>
__device__ __forceinline__ void turn(float& x, float& y, float2 cs) {
  if constexpr (kFused) {
    const float u = fmaf(x, cs.x, -__fmul_rn(y, cs.y));
    y = fmaf(y, cs.x, __fmul_rn(x, cs.y));
    x = u;
    return;
  }
  const float u = __fsub_rn(__fmul_rn(x, cs.x), __fmul_rn(y, cs.y));
  y = __fadd_rn(__fmul_rn(y, cs.x), __fmul_rn(x, cs.y));
  x = u;
}

// The eight pairs' cos and sin that 16 values of a token need (positions out of the table:
// recorded, and position 0).  The eight are two runs of four; `wide`: a run lies in one
// section and its table entries on a 16-byte boundary.
template <int D>
__device__ __forceinline__ void load_turns(const CacheAppendArgs& a, const int32_t (&pos)[3],
                                           int32_t c8, bool wide, float2 (&cs)[8]) {
  int32_t at[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    at[i] = pos[i];
    if (at[i] < 0 || at[i] >= a.rot.n_pos) {
      record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      at[i] = 0;
    }
  }
  const int32_t s0 = a.rot.sec[0], s1 = s0 + a.rot.sec[1];
  auto entry = [&](int32_t pair) {
    const int32_t row = pair < s0 ? at[0] : (pair < s1 ? at[1] : at[2]);
    return reinterpret_cast<const float2*>(a.rot.table) + (int64_t)row * (D / 2) + pair;
  };
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int32_t pair = a.rot.interleaved ? (c8 + u * (D / 2)) / 2 : c8 + 4 * u;
    if (wide) {
      const float4* p = reinterpret_cast<const float4*>(entry(pair));
      const float4 x = __ldg(p), y = __ldg(p + 1);
      cs[4 * u] = make_float2(x.x, x.y);
      cs[4 * u + 1] = make_float2(x.z, x.w);
      cs[4 * u + 2] = make_float2(y.x, y.y);
      cs[4 * u + 3] = make_float2(y.z, y.w);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) cs[4 * u + i] = __ldg(entry(pair + i));
    }
  }
}
template <bool kFused>
__device__ __forceinline__ void rotate16(bool interleaved, const float2 (&cs)[8], float (&xa)[8],
                                         float (&xb)[8]) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      turn<kFused>(xa[2 * i], xa[2 * i + 1], cs[i]);
      turn<kFused>(xb[2 * i], xb[2 * i + 1], cs[4 + i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn<kFused>(xa[i], xb[i], cs[i]);
  }
}

// Eight values times their gains plus their biases (null: 1 and 0).  kOnce: rounded once, for keys,
// which e4m3 rounds again: every rounding before that moves a few keys more to a neighbour.
template <bool kOnce>
__device__ __forceinline__ void apply8(const float* gain, const float* bias, float (&x)[8]) {
  const float4* g = reinterpret_cast<const float4*>(gain);
  const float4* b = reinterpret_cast<const float4*>(bias);
  if (kOnce && gain != nullptr && bias != nullptr) {
    const float4 u = __ldg(g), v = __ldg(g + 1), s = __ldg(b), t = __ldg(b + 1);
    x[0] = fmaf(x[0], u.x, s.x), x[1] = fmaf(x[1], u.y, s.y), x[2] = fmaf(x[2], u.z, s.z);
    x[3] = fmaf(x[3], u.w, s.w), x[4] = fmaf(x[4], v.x, t.x), x[5] = fmaf(x[5], v.y, t.y);
    x[6] = fmaf(x[6], v.z, t.z), x[7] = fmaf(x[7], v.w, t.w);
    return;
  }
  if (gain != nullptr) {
    const float4 u = __ldg(g), v = __ldg(g + 1);
    x[0] *= u.x, x[1] *= u.y, x[2] *= u.z, x[3] *= u.w, x[4] *= v.x, x[5] *= v.y, x[6] *= v.z, x[7] *= v.w;
  }
  if (bias != nullptr) {
    const float4 u = __ldg(b), v = __ldg(b + 1);
    x[0] += u.x, x[1] += u.y, x[2] += u.z, x[3] += u.w, x[4] += v.x, x[5] += v.y, x[6] += v.z, x[7] += v.w;
  }
}
// A head's norm over its D / 16 lanes: kNorm 1, x / sqrt(mean x^2 + eps); 2, the same of x less its
// mean (squares of the differences, so a large mean costs no digits); times gain plus bias.  In
// float32, and not rounded before the rotation.  Called by all lanes of a head together, whatever
// the warp's other lanes do.  `at`: of the thread's first value in the gains.
template <int D, int kNorm, bool kOnce>
__device__ __forceinline__ void normalise16(float eps, const float* gain, const float* bias, int32_t at,
                                            float (&xa)[8], float (&xb)[8]) {
  constexpr int LPR = D / 16;
  const uint32_t lanes = ((1u << LPR) - 1u) << (threadIdx.x & 31 & ~(LPR - 1));
  auto sum = [&](float2 v2) {
    float v = v2.x + v2.y;
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(lanes, v, o);
    return v;
  };
  const float2 zero = make_float2(0.f, 0.f);
  auto each = [&](auto f) {  // pairs of values
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 u = f(make_float2(xa[i], xa[i + 1])), v = f(make_float2(xb[i], xb[i + 1]));
      xa[i] = u.x, xa[i + 1] = u.y, xb[i] = v.x, xb[i + 1] = v.y;
    }
  };
  if constexpr (kNorm == 2) {
    float2 s = zero;
    each([&](float2 x) {
      s = fadd2(s, x);
      return x;
    });
    const float less = -sum(s) * (1.f / D);
    each([&](float2 x) { return fadd2(x, make_float2(less, less)); });
  }
  float2 s = zero;
  each([&](float2 x) {
    s = ffma2(x, x, s);
    return x;
  });
  const float r = __frsqrt_rn(fmaf(sum(s), 1.f / D, eps));
  each([&](float2 x) { return ffma2(x, make_float2(r, r), zero); });
  apply8<kOnce>(gain != nullptr ? gain + at : nullptr, bias != nullptr ? bias + at : nullptr, xa);
  apply8<kOnce>(gain != nullptr ? gain + at + D / 2 : nullptr, bias != nullptr ? bias + at + D / 2 : nullptr, xb);
}

// A thread holds 16 values of a row, a row takes D / 16 lanes, and a block of
// threads covers a cache block of S tokens of one head in kPasses passes (at
// least a warp): the new values stay in registers between the search for their
// largest and the rounding, so they are read once.
// It reads and writes every byte once; what bounds it is the chain of dependent loads
// (lengths and the first slot; rows, slots and positions; the table), so each link is asked for
// by all passes at once, and two passes of 66 registers beat four of 98.  16 ragged prompts of
// up to 1088 tokens (221 MB): 42 us, 5.2 TB/s, 0.77 of the measured copy rate (one link after
// the other, each pass by itself and a table entry per head: 93 us); 8 x 128 drafts (23 MB, on
// blocks that are partly full): 9.8 us; a token each of 8 sequences 3.1 us.
constexpr int kPasses = 2;
constexpr int kHeads = 4;  // heads of q that share a thread's cos and sin
constexpr int append_threads(int d, int block) {
  return block * (d / 16) / kPasses < 32 ? 32 : block * (d / 16) / kPasses;
}

// x: new tokens' rows of one head; kIsK: rotated first.
template <int D, bool kIsK, int kNorm>
__device__ __forceinline__ void append_block(const CacheAppendArgs& a, int32_t b, int32_t i,
                                             int32_t g, bool wide, float* red) {
  constexpr int LPR = D / 16;  // lanes of a row
  const int32_t S = a.cache.block, tid = threadIdx.x;
  const int64_t row0 = (int64_t)b * a.N_max;
  const int32_t n = a.n_new[b];
  const int64_t slot0 = a.slots[row0];
  if (n <= 0 || n > a.N_max) {
    if (n != 0 && tid == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
    return;
  }
  if (slot0 < 0) return;  // a sequence that the plan could not serve
  const int32_t off0 = (int32_t)(slot0 & (S - 1));
  const int32_t j0 = i == 0 ? 0 : i * S - off0;  // the block's first new token
  if (j0 >= n) return;
  const int32_t first = i == 0 ? off0 : 0;       // tokens it holds already
  const int32_t count = min(n - j0, S - first);
  const __nv_bfloat16* x =
      static_cast<const __nv_bfloat16*>(kIsK ? a.k : a.v) + (row0 + j0) * (kIsK ? a.ldk : a.ldv) +
      (int64_t)g * D;
  const int64_t ld = kIsK ? a.ldk : a.ldv;
  const int32_t c8 = (tid % LPR) * 8, r0 = tid / LPR, rows = blockDim.x / LPR;

  uint4 wa[kPasses], wb[kPasses];
  int64_t at[kPasses];
  int32_t pos[kPasses][3];
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int32_t r = r0 + u * rows;  // of the new tokens
    if (r >= count) continue;
    wa[u] = *reinterpret_cast<const uint4*>(x + r * ld + c8);
    wb[u] = *reinterpret_cast<const uint4*>(x + r * ld + c8 + D / 2);
    at[u] = a.slots[row0 + j0 + r];
    if (kIsK)
#pragma unroll
      for (int e = 0; e < 3; ++e) pos[u][e] = a.pos[3 * (row0 + j0 + r) + e];
  }
  const int64_t slot = i == 0 ? slot0 : a.slots[row0 + j0];
  if (slot < 0 || slot >= (int64_t)a.cache.num_blocks * S || (int32_t)(slot & (S - 1)) != first) {
    if (tid == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
    return;
  }
  const int64_t head = slot / S * a.cache.Hkv + g;
  uint8_t* out = static_cast<uint8_t*>(kIsK ? a.cache.k : a.cache.v) + head * S * D;
  float* scale = (kIsK ? a.cache.k_scale : a.cache.v_scale) + head;
  const float old = *scale;

  float xa[kPasses][8], xb[kPasses][8];
  bool have[kPasses];
  float m = 0.f;
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int32_t r = r0 + u * rows;
    have[u] = r < count;
    if (have[u] && at[u] != slot + r) {
      record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      have[u] = false;
    }
    if (!have[u]) continue;
    unpack8(wa[u], xa[u]);
    unpack8(wb[u], xb[u]);
    if (kIsK) {
      if constexpr (kNorm != 0)
        normalise16<D, kNorm, true>(a.norm.eps, a.norm.k_gain, a.norm.k_bias,
                              (a.norm.k_heads != 0 ? g * D : 0) + c8, xa[u], xb[u]);
      float2 cs[8];
      load_turns<D>(a, pos[u], c8, wide, cs);
      rotate16<kNorm != 0>(a.rot.interleaved, cs, xa[u], xb[u]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = fabsf(xa[u][e]), q = fabsf(xb[u][e]);
      if (p < INFINITY) m = fmaxf(m, p);  // false for NaN
      if (q < INFINITY) m = fmaxf(m, q);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (blockDim.x > 32) {
    if ((tid & 31) == 0) red[tid >> 5] = m;
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x / 32; ++w) m = fmaxf(m, red[w]);
  }
  const bool grown = first == 0 || m > kTop8 * old;
  const float s = grown ? fmaxf(m, kLeast) / kTop8 : old;
  const float inv = 1.0f / s;
  __syncthreads();  // every thread has the old scale
  if (grown && tid == 0) *scale = s;
  if (grown && first > 0) {  // what the block holds, to the new scale
    const float f = old * inv;
    for (int32_t r = r0; r < first; r += rows) {
      uint2* at = reinterpret_cast<uint2*>(out + r * D + (tid % LPR) * 16);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint2 w = at[h];
        float y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 p = from_e4m3x2((uint16_t)((e < 2 ? w.x : w.y) >> (16 * (e & 1))));
          y[2 * e] = p.x;
          y[2 * e + 1] = p.y;
        }
        at[h] = to_e4m3x8(y, f);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    if (!have[u]) continue;
    uint8_t* at = out + (first + r0 + u * rows) * D + c8;
    *reinterpret_cast<uint2*>(at) = to_e4m3x8(xa[u], inv);
    *reinterpret_cast<uint2*>(at + D / 2) = to_e4m3x8(xb[u], inv);
  }
}

// Grid: first the (sequence, touched block, head) units of K, then those of V, then
// those of q: a thread takes 16 columns of up to kHeads heads of a token.
// 72 registers: with norms the compiler takes 86 to 92, and what is lost in loads under way costs more
// than the 64 to 92 bytes a thread that it spills (16 ragged prompts, layer norms with gains and biases of
// every head, on the same inputs again and again: 66.9 us, 58.5 with 72, 60.3 with 64; root-mean-square norms
// alone 54.9 and 47.6).  On inputs that change: 64 and 55 us, one row of gains for all heads 61 and 53; without
// norms, which spills nothing, 42.
template <int D, int kNorm>
__global__ void __maxnreg__(72)
cache_append_kernel(CacheAppendArgs a, int32_t touched, int64_t kv_units, bool wide) {
  constexpr int LPR = D / 16;
  __shared__ float red[128 * LPR / kPasses / 32];
  pdl_wait();
  int64_t unit = blockIdx.x;
  if (unit < 2 * kv_units) {
    const bool is_k = unit < kv_units;
    if (!is_k) unit -= kv_units;
    const int32_t g = (int32_t)(unit % a.cache.Hkv);
    const int32_t bi = (int32_t)(unit / a.cache.Hkv);
    const int32_t b = bi / touched, i = bi - b * touched;
    if (is_k) append_block<D, true, kNorm>(a, b, i, g, wide, red);
    else append_block<D, false, kNorm>(a, b, i, g, wide, red);
    return;
  }
  unit -= 2 * kv_units;
  const int32_t rows = blockDim.x / LPR, c8 = (threadIdx.x % LPR) * 8;
  const int32_t groups = (a.Hq + kHeads - 1) / kHeads;
  const int64_t r = unit * rows + threadIdx.x / LPR;
  if (r >= (int64_t)a.B * a.N_max * groups) return;
  const int32_t token = (int32_t)r / groups, h0 = ((int32_t)r - token * groups) * kHeads;
  const int32_t b = token / a.N_max, n = a.n_new[b];
  if (token - b * a.N_max >= n || n > a.N_max) return;
  int32_t pos[3];
#pragma unroll
  for (int e = 0; e < 3; ++e) pos[e] = a.pos[3 * (int64_t)token + e];
  const int64_t slot = a.slots[token];
  const __nv_bfloat16* x =
      static_cast<const __nv_bfloat16*>(a.q) + token * a.ldq + (int64_t)h0 * D + c8;
  uint4 wa[kHeads], wb[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (h0 + u >= a.Hq) continue;
    wa[u] = *reinterpret_cast<const uint4*>(x + u * D);
    wb[u] = *reinterpret_cast<const uint4*>(x + u * D + D / 2);
  }
  if (slot < 0) return;
  float2 cs[8];
  load_turns<D>(a, pos, c8, wide, cs);
  __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.q_out) + ((int64_t)token * a.Hq + h0) * D + c8;
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (h0 + u >= a.Hq) continue;
    float xa[8], xb[8];
    unpack8(wa[u], xa);
    unpack8(wb[u], xb);
    if constexpr (kNorm != 0)
      normalise16<D, kNorm, false>(a.norm.eps, a.norm.q_gain, a.norm.q_bias,
                            (a.norm.q_heads != 0 ? (h0 + u) * D : 0) + c8, xa, xb);
    rotate16<kNorm != 0>(a.rot.interleaved, cs, xa, xb);
    *reinterpret_cast<uint4*>(y + u * D) = pack8(xa);
    *reinterpret_cast<uint4*>(y + u * D + D / 2) = pack8(xb);
  }
}

}  // namespace

cudaError_t launch_cache_plan(const CachePlanArgs& a, cudaStream_t stream) {
  const int32_t per = a.N_max >= kPlanSlots ? 1 : std::min(kPlanThreads, kPlanSlots / a.N_max);
  const int32_t pieces = per > 1 ? 1 : (a.N_max + kPlanSlots - 1) / kPlanSlots;
  const int64_t units = per > 1 ? (a.B + per - 1) / per : (int64_t)a.B * pieces;
  if (units > INT32_MAX) return cudaErrorInvalidValue;
  return launch_kernel(cache_plan_kernel, dim3((unsigned)units), dim3(kPlanThreads), 0, stream, true,
                       a, per, pieces);
}

cudaError_t launch_rotary_table(int32_t n_pos, int32_t pairs, const float* freq, float* table,
                                cudaStream_t stream) {
  const int32_t n = n_pos * pairs;
  const unsigned blocks = (unsigned)std::min<int64_t>(((int64_t)n + 255) / 256, 4096);
  return launch_kernel(rotary_table_kernel, dim3(blocks), dim3(256), 0, stream, true, n, pairs,
                       freq, reinterpret_cast<float2*>(table));
}

cudaError_t launch_cache_append(const CacheAppendArgs& a, cudaStream_t stream) {
  const int32_t S = a.cache.block, d = a.cache.d, threads = append_threads(d, S);
  // blocks that N_max tokens can touch: from the last token of one on
  const int32_t touched = 1 + (a.N_max - 1 + S - 1) / S;
  const int64_t kv_units = (int64_t)a.B * touched * a.cache.Hkv;
  const int64_t q_rows = (int64_t)a.B * a.N_max * ((a.Hq + kHeads - 1) / kHeads);
  const int32_t per = threads / (d / 16);
  const int64_t grid = 2 * kv_units + (q_rows + per - 1) / per;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  const int32_t s0 = a.rot.sec[0], s1 = s0 + a.rot.sec[1];
  const bool wide =
      s0 % 4 == 0 && s1 % 4 == 0 && (reinterpret_cast<uintptr_t>(a.rot.table) & 15) == 0;
  auto launch = [&](auto kernel) {
    return launch_kernel(kernel, dim3((unsigned)grid), dim3(threads), 0, stream, true, a, touched,
                         kv_units, wide);
  };
  if (a.norm.kind == SSD_NORM_RMS)
    return launch(d == 128 ? cache_append_kernel<128, 1> : cache_append_kernel<64, 1>);
  if (a.norm.kind == SSD_NORM_LAYER)
    return launch(d == 128 ? cache_append_kernel<128, 2> : cache_append_kernel<64, 2>);
  return launch(d == 128 ? cache_append_kernel<128, 0> : cache_append_kernel<64, 0>);
}

}  // namespace ssd
