// cache_attention.cu — frontier attention over the paged 8-bit cache
// (include/ssd.h, ssd_cache_attention):
//   O[b][j][h] = softmax_s(scale * Q[b][j][h] . (sk K[s]) + M(s, j)) (sv V[s]),
// K and V e4m3 with a scale per block of tokens and KV head (sk, sv).
//
// Every e4m3 value is a float16, so the products run as mma.sync on float16
// with float32 accumulation and the scales stay outside: sk multiplies the
// scores, sv the probabilities before they are rounded to float16.
//
// The products are turned round, S^T = K Q^T and O^T = V^T P^T: the keys (and then
// the columns of V) fill the 16 rows of an mma, and the query rows its 8 columns, so
// the few rows of a token under grouped heads (drafts x the query heads that share
// the KV head) fill it better.  A warp takes 8 or 16 query rows and walks steps of
// 16 keys.  The order of an mma's inner index and of its rows is free as long as
// both operands agree, so each lane reads what it needs from a step in pieces of 16
// bytes: of K, 16 consecutive values of two keys; of V, 16 consecutive columns of
// four keys.  A step's K and V come by TMA (swizzled, so those reads meet no bank
// conflicts) into a ring of the warp's own, four steps deep; a stage is asked for
// again as soon as it is in registers.  P turns round in registers (movmatrix).
// The warps of a CTA split 16-key steps among them and merge at the end.
//
// A token of 16 sequences of 7000 to 27000 keys, 8 KV heads of 4 query heads: 503 MB in 89 us,
// 5.7 TB/s, 0.83 of the measured copy rate (with query rows in the mma's 16 rows, lane-wise
// copies and as many CTAs for each sequence 132 us, the SMs idle for a quarter of it).  What is
// left: the last tenth to even out, and the combine.  Little work is bound by the steps of a
// warp, 900 cycles each while it has its scheduler to itself: one token over 800 keys 9.4 us,
// of which 6 are the launch, the first copies and the rows' way out.

#include <cuda_fp16.h>

#include <algorithm>

#include "cache_attention.cuh"

namespace ssd {

namespace {

constexpr int kStep = 16;           // keys per step
constexpr int kWarps = 4;           // of a CTA
constexpr int kManyWarps = 8;       // where no SM has more than one CTA: a warp alone on its
                                    // scheduler takes 900 cycles a step, most of it waiting
                                    // (8 heads over 800 keys: 12.6 us with four, 10.4)
constexpr int kCtas = 3;            // per SM
// Steps in flight per warp, and CTAs per SM that the registers are for.  Behind shared keys a CTA's keys
// are few, so its set-up and way out count: more of them at once, also beside a CTA that works on
// the shared ones (371 sequences of 67 to 712 own keys, 12/4 heads of 64: 61 us, 56).
template <int NR, int W, bool kShared>
constexpr int kStagesOf = kShared && NR == 1 && W == kWarps ? 3 : 4;
// (Groups differ in size: 16 sequences in 8 groups of 1 to 7, 8 rows a CTA, 3840 keys 28.6 us with one, 21.6
// with two; in groups of 2, where the second CTAs have no rows, 19.5 and 21.9.)
constexpr int kStackTurns = 2;
constexpr int kMostPartTiles = 264;  // of shared keys
template <int NR, int W, bool kShared>
constexpr int kCtasOf = W != kWarps ? 1 : kShared && NR == 1 ? 4 : kCtas;
constexpr int kMinTiles = 8;        // a part's fewest tiles
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMostP = 256.f;     // a probability beyond it moves its reference
constexpr float kUnseen = -3.402823466e38f;  // reference of a row that has seen no key

// (Of at most 16 rows, or little work.)
CacheMmaPlan make_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max) {
  CacheMmaPlan p;
  const int64_t rows = (int64_t)D_max * (Hq / Hkv);
  const int64_t sms = device_sm_count();
  const bool few = cache_attention_few(B, Hkv, rows, L_max);
  p.rows = rows <= 8 || few ? 8 : 16;
  p.row_groups = (int32_t)((rows + p.rows - 1) / p.rows);
  const int64_t tiles = (L_max + kCacheTile - 1) / kCacheTile;
  // CTAs a sequence and head may take; a part has room for so many block ids
  const int64_t most = std::max<int64_t>(1, tiles / kMinTiles);
  const int64_t least = (tiles + kWorkTiles - 1) / kWorkTiles;
  const int64_t target = kCtas * sms / ((int64_t)Hkv * p.row_groups);
  if (target <= B || most < kCutFrom) {
    p.goal = p.uniform = (int32_t)least;
    p.per_head = (int32_t)(B * least);
  } else {
    p.uniform = 0;
    p.goal = (int32_t)std::min(target, B * most);
    p.per_head = (int32_t)std::max<int64_t>(p.goal, B * least);
  }
  const bool alone = (int64_t)p.per_head * Hkv * p.row_groups <= sms;
  p.warps = alone && p.rows == 8 ? kManyWarps : kWarps;
  return p;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two e4m3 (the low or high half of w) as two float16, exactly.
__device__ __forceinline__ uint32_t f16_lo(uint32_t w) {
  uint32_t h;
  asm("{\n .reg .b16 l, u;\n mov.b32 {l, u}, %1;\n cvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(h) : "r"(w));
  return h;
}
__device__ __forceinline__ uint32_t f16_hi(uint32_t w) {
  uint32_t h;
  asm("{\n .reg .b16 l, u;\n mov.b32 {l, u}, %1;\n cvt.rn.f16x2.e4m3x2 %0, u;\n}" : "=r"(h) : "r"(w));
  return h;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t word(const uint4& x, int i) {
  return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
}
// 8 x 8 values of 16 bits, lane (r, q) holding (r, 2 q) and (r, 2 q + 1), turned round.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// NR: groups of 8 query rows of a warp; W: warps.
// kMode 1: a sequence's keys begin behind those that it shares with its group, and its rows always
// go to the part rows.  kMode 2: a group's shared keys, the rows of all its sequences one behind the
// other; grid: parts, KV heads and groups in x, CTAs that take turns at the rows of a group in z (each
// turn reads the keys again).
template <int D, int NR, int W, int kMode>
__global__ void __launch_bounds__(W * 32, (kCtasOf<NR, W, kMode == 1>))
cache_attn_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  CacheAttnArgs a, CacheAttnLaunch L) {
  constexpr bool kShared = kMode == 1, kStack = kMode == 2;
  constexpr int kStages = kStagesOf<NR, W, kShared>;
  constexpr int RW = 8 * NR;          // rows of a warp
  constexpr int NT = D / 16;          // output tiles of 16 columns
  constexpr int KG = D / 64;          // groups of four mma steps of K Q^T
  constexpr int VB = D / 8;           // bytes of V a lane takes per key
  constexpr int kStageBytes = 2 * kStep * D;
  constexpr int kWarpBytes = kStages * kStageBytes;
  constexpr int kRowFloats = D + 4;   // of the partial rows, which take the ring's place
  static_assert(kWarpBytes >= RW * kRowFloats * 4, "a warp's partial rows fit its ring");
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  int32_t* s_id = reinterpret_cast<int32_t*>(smem + W * kWarpBytes);
  float* s_ks = reinterpret_cast<float*>(s_id + L.max_blocks);
  float* s_vs = s_ks + L.max_blocks;
  __shared__ uint64_t s_full[W][kStages];
  __shared__ float2 s_ml[W][RW];
  if (threadIdx.x < 2) prefetch_tensormap(threadIdx.x == 0 ? &tmK : &tmV);
  // (kShared: beside the kernel before it, on the shared keys, which let it start when all before
  // that was done; the first CTA waits for it at the end)
  if (!kShared) pdl_wait();
  if (kStack) pdl_launch_dependents();

  const int32_t tid = threadIdx.x, lane = tid & 31, warp = (int32_t)warp_uniform(tid >> 5);
  // (kShared: a sequence's heads one after the other, the longest sequences first)
  const int32_t cta = kShared ? blockIdx.x + blockIdx.y * gridDim.x : 0;
  const int32_t x_cta = kShared ? cta / a.cache.Hkv : blockIdx.x;
  const int32_t g = kStack ? blockIdx.x / L.s_splits % a.cache.Hkv : kShared ? cta - x_cta * a.cache.Hkv : blockIdx.y;
  const int32_t S = a.cache.block, S_log = 31 - __clz(S), G = a.Hq / a.cache.Hkv;
  const bool first_of = !kStack && g == 0 && blockIdx.z == 0;
  // kStack: the group's first sequence, the one that names the blocks, rows and shared tokens
  int32_t g_first = 0, g_named = -1, g_rows = 0, g_len = 0, g_row0 = 0;
  CacheWork<kShared> work;
  if constexpr (kStack) {
    const int32_t group = blockIdx.x / L.s_splits / a.cache.Hkv, split = blockIdx.x % L.s_splits;
    const int32_t blocks = a.shared[group];
    g_first = min(max(a.group_start[group], 0), a.B);
    const int32_t end = min(max(a.group_start[group + 1], g_first), a.B);
    // (what is out of range is recorded with the sequences' own keys)
    if (blocks <= 0 || blocks > a.max_shared) return;
    g_len = blocks * S;
    g_rows = (end - g_first) * a.D_max * G;
    for (int32_t b0 = g_first; b0 < end && g_named < 0; b0 += 32) {
      const int32_t c = b0 + lane < end ? a.cache_len[b0 + lane] : 0, n = b0 + lane < end ? a.n_drafts[b0 + lane] : 0;
      const uint32_t here = __ballot_sync(0xffffffffu, n > 0 && cache_lengths_ok(a, c, n) && c >= g_len);
      if (here != 0) g_named = b0 + __ffs(here) - 1;
    }
    const int32_t tiles = (g_len + kCacheTile - 1) / kCacheTile, parts = cache_parts(L.s_splits, L.s_min_tiles, tiles);
    g_row0 = blockIdx.z * RW;
    if (g_named < 0 || split >= parts || g_row0 >= g_rows) return;
    work.t_lo = (int32_t)((int64_t)tiles * split / parts);
    work.t_hi = (int32_t)((int64_t)tiles * (split + 1) / parts);
  }
  if (lane == 0) {
    for (int t = 0; t < kStages; ++t) mbar_init(&s_full[warp][t], 1);
    fence_barrier_init();
  }
  uint32_t stage = 0, phase = 0;  // of the warp's next step
  bool more = true;
  if constexpr (!kStack) more = work.first(a, L, x_cta, first_of && tid < 32);
  auto next = [&]() {
    if constexpr (!kStack) return work.next(a);
    g_row0 += gridDim.z * RW;
    return g_row0 < g_rows;
  };
#pragma unroll 1
  for (; more; more = next()) {
    // (the rows of the part before have left the ring's place, and the copies may know it)
    fence_proxy_async_shared();
    __syncthreads();
    const int32_t b = kStack ? g_named : work.b;
    const int32_t cache = kStack ? g_len : a.cache_len[b], nd = kStack ? 0 : a.n_drafts[b];
    const int32_t Lk = cache + nd, rows_total = kStack ? g_rows : nd * G;
    const int32_t row0 = kStack ? g_row0 : blockIdx.z * RW;
    if (!kStack && L.info != nullptr && first_of && tid == 0) {
      if (work.t_lo == 0) L.info[b].x = work.x;
      if (work.t_hi == work.tiles) L.info[b].y = work.x;
    }
    if (row0 >= rows_total) continue;
    const bool whole = kMode == 0 && work.t_lo == 0 && work.t_hi == work.tiles, begins = work.t_lo == 0;
    const int32_t base = kShared ? cache_base(a, b, cache) : 0;
    const int32_t k_lo = base + work.t_lo * kCacheTile, k_hi = min(Lk, base + work.t_hi * kCacheTile);
    int32_t start = !kStack && a.key_start != nullptr ? min(Lk, max(0, a.key_start[b])) : 0;

    // ---- this warp's rows and its share of the steps, and the copies of the first ones
    const int32_t q = lane & 3, r8 = lane >> 2;
    const int32_t first = max(k_lo, start & ~(kStep - 1));  // multiple of 16
    unsigned char* ring = smem + warp * kWarpBytes;
    const int32_t n_steps =
        first >= k_hi ? 0 : (k_hi - first + kStep - 1) / kStep;
    const int32_t steps = n_steps > warp ? (n_steps - warp + W - 1) / W : 0;
    auto key_of = [&](int32_t t) { return first + (t * W + warp) * kStep; };
    auto issue = [&](int32_t t, uint32_t to, int32_t id) {  // by one lane
      const int32_t k0 = key_of(t), z = max(id, 0) * a.cache.Hkv + g;
      unsigned char* dst = ring + to * kStageBytes;
      uint64_t* bar = &s_full[warp][to];
      const uint64_t once = policy_evict_first();
      mbar_arrive_expect_tx(bar, kStageBytes);
      tma_load_3d(dst, &tmK, 0, k0 & (S - 1), z, bar, once);
      tma_load_3d(dst + kStep * D, &tmV, 0, k0 & (S - 1), z, bar, once);
    };
    const int32_t* table = a.block_table + (int64_t)b * a.max_blocks;
    if (lane == 0) {
      for (int t = 0; t < kStages && t < steps; ++t) {
        const int32_t id = table[key_of(t) >> S_log];
        issue(t, (stage + t) % kStages, id < a.cache.num_blocks ? id : -1);
      }
    }
    __syncwarp();

    // ---- the part's block ids and scales
    const int32_t b_lo = k_lo >> S_log;  // (a part may start inside a block of 128)
    const int32_t nb = ((k_hi - 1) >> S_log) + 1 - b_lo;
    for (int32_t i = tid; i < nb; i += blockDim.x) {
      int32_t id = table[b_lo + i];
      if (id < 0 || id >= a.cache.num_blocks) {
        record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
        id = -1;
      }
      s_id[i] = id;
      const int64_t at = (int64_t)id * a.cache.Hkv + g;
      s_ks[i] = id < 0 ? 0.f : a.cache.k_scale[at];
      s_vs[i] = id < 0 ? 0.f : a.cache.v_scale[at];
    }

    // Q as float16 with its row's power of two taken out; column order of K's reads.  A
    // lane holds row 8 n + r8.
    uint32_t qf[NR][KG][4][2];
    float rowc_of[NR];
    int32_t qpos_of[NR];
    int32_t start_of[NR];  // (kStack) the row's first visible key; of no row: INT32_MAX
    const float c2 = (a.scale != 0.f ? a.scale : rsqrtf((float)D)) * kLog2e;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int32_t r = row0 + r8 + 8 * n;
      const bool live = r < rows_total;
      const int32_t j = live ? r / G : 0, h = g * G + (live ? r - j * G : 0);
      const uint4* src = reinterpret_cast<const uint4*>(
          static_cast<const __nv_bfloat16*>(a.q) +
          (((int64_t)(kStack ? g_first : b) * a.D_max + j) * a.Hq + h) * D);
      qpos_of[n] = start_of[n] = 0x7fffffff;
      if constexpr (kStack) {
        const int32_t rb = g_first + j / a.D_max, jj = j - (rb - g_first) * a.D_max;
        if (live) {
          const int32_t c = a.cache_len[rb], n_of = a.n_drafts[rb];
          if (cache_lengths_ok(a, c, n_of) && jj < n_of && c >= g_len) {
            qpos_of[n] = cache_flat_pos(a, rb, c, jj);
            start_of[n] = a.key_start != nullptr ? min(g_len, max(0, a.key_start[rb])) : 0;
          }
        }
      } else if (live) {
        qpos_of[n] = cache_flat_pos(a, b, cache, j);
        if (qpos_of[n] < 0 && begins && g == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      }
      float x[KG][16];
      float m = 0.f;
#pragma unroll
      for (int kg = 0; kg < KG; ++kg)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint4 w = live ? src[(q * KG + kg) * 2 + u] : make_uint4(0, 0, 0, 0);
          const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[kg][u * 8 + 2 * e] = __uint_as_float(v[e] << 16);
            x[kg][u * 8 + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
            m = fmaxf(m, fmaxf(fabsf(x[kg][u * 8 + 2 * e]), fabsf(x[kg][u * 8 + 2 * e + 1])));
          }
        }
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
      // 2^e with m / 2^e in [1, 2) (or less, for the smallest; 4, for the largest)
      const int32_t e = min(126, max(-126, (int32_t)(__float_as_uint(m) >> 23) - 127));
      // (an infinity: every product of the row is NaN, as its softmax is)
      const float down = m == INFINITY ? NAN : __uint_as_float((uint32_t)(127 - e) << 23);
      rowc_of[n] = c2 * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
      for (int kg = 0; kg < KG; ++kg)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          qf[n][kg][s][0] = pack_f16x2(x[kg][4 * s] * down, x[kg][4 * s + 1] * down);
          qf[n][kg][s][1] = pack_f16x2(x[kg][4 * s + 2] * down, x[kg][4 * s + 3] * down);
        }
    }
    // keys below this one are visible to every row of the warp
    int32_t mask_from;
    {
      int32_t minq = qpos_of[0];
      if (NR == 2) minq = min(minq, qpos_of[NR - 1]);
      mask_from = min(cache, min(0x7ffffffe, __reduce_min_sync(0xffffffffu, minq)) + 1);
    }
    int32_t hide_to = start;  // keys below this one are hidden from some row of the warp
    if constexpr (kStack) {
      int32_t lo = 0x7fffffff, hi = 0;
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        lo = min(lo, start_of[n]);
        if (start_of[n] != 0x7fffffff) hi = max(hi, start_of[n]);
      }
      start = min(g_len, __reduce_min_sync(0xffffffffu, lo));  // (those before it may be anything)
      hide_to = __reduce_max_sync(0xffffffffu, hi);
    }
    // From here on a lane's rows are 8 n + 2 q + u: those of its scores and of O.
    float rowc[NR][2];
    int32_t qpos[NR][2];
    int32_t row_start[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        rowc[n][u] = __shfl_sync(0xffffffffu, rowc_of[n], (2 * q + u) * 4);
        qpos[n][u] = __shfl_sync(0xffffffffu, qpos_of[n], (2 * q + u) * 4);
        if (kStack) row_start[n][u] = __shfl_sync(0xffffffffu, start_of[n], (2 * q + u) * 4);
      }
    __syncthreads();  // ids and scales

    // offsets of the lane's pieces in a stage (the swizzle: of 16-byte pieces, by the row)
    uint32_t k_off[KG], v_off[2];
#pragma unroll
    for (int kg = 0; kg < KG; ++kg) {
      const int32_t sw = D == 128 ? r8 : (r8 >> 1) & 3;
      k_off[kg] = r8 * D + (((q * KG + kg) ^ sw) << 4);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int32_t key = 2 * q + u;
      v_off[u] = kStep * D + key * D +
                 (D == 128 ? (r8 ^ key) << 4 : (((r8 >> 1) ^ q) << 4) + (r8 & 1) * 8);
    }

    float o[NR][NT][4];
    // A row's two references: m_ref (log2) of its scores, for the sum, and 1 / v_inv, a power of
    // two, of its probabilities times their V scales.  Those go into the product as float16,
    // below kMostP and with the largest at least 1, whatever the scales of keys that the row
    // does not see or hardly weighs.
    float m_ref[NR][2], v_inv[NR][2], l[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int t = 0; t < NT; ++t) o[n][t][0] = o[n][t][1] = o[n][t][2] = o[n][t][3] = 0.f;
      m_ref[n][0] = m_ref[n][1] = kUnseen;
      v_inv[n][0] = v_inv[n][1] = 1.f;
      l[n][0] = l[n][1] = 0.f;
    }
    bool ok = true;
    int32_t t = 0;
#pragma unroll 1
    for (; t < steps; ++t) {
      ok = wait_warp(&s_full[warp][stage], phase, a.status);
      if (!ok) break;
      const unsigned char* st = ring + stage * kStageBytes;
      uint4 kw[2][KG];
      uint32_t v[4][VB / 4];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int kg = 0; kg < KG; ++kg)
          kw[h][kg] = *reinterpret_cast<const uint4*>(st + k_off[kg] + h * 8 * D);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned char* at = st + v_off[i & 1] + (i >> 1) * 8 * D;
        if constexpr (VB == 16) {
          const uint4 w = *reinterpret_cast<const uint4*>(at);
          v[i][0] = w.x;
          v[i][1] = w.y;
          v[i][2] = w.z;
          v[i][3] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(at);
          v[i][0] = w.x;
          v[i][1] = w.y;
        }
      }
      const int32_t k0 = key_of(t), bi = (k0 >> S_log) - b_lo;
      // (kStack: a block that nobody sees may have any scale)
      const float ks = s_ks[bi], vs = kStack && k0 + kStep <= start ? 0.f : s_vs[bi];
      __syncwarp();
      if (lane == 0 && t + kStages < steps)
        issue(t + kStages, stage, s_id[(key_of(t + kStages) >> S_log) - b_lo]);
      stage = (stage + 1) % kStages;
      phase ^= stage == 0 ? 1u : 0u;

      // ---- S^T = K Q^T
      float x[NR][4];  // keys r8 and r8 + 8 (by 2) of the lane's rows
      {
        float sc[KG][NR][4];
#pragma unroll
        for (int kg = 0; kg < KG; ++kg) {
#pragma unroll
          for (int n = 0; n < NR; ++n) sc[kg][n][0] = sc[kg][n][1] = sc[kg][n][2] = sc[kg][n][3] = 0.f;
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const uint32_t w0 = word(kw[0][kg], s), w1 = word(kw[1][kg], s);
            const uint32_t kf[4] = {f16_lo(w0), f16_lo(w1), f16_hi(w0), f16_hi(w1)};
#pragma unroll
            for (int n = 0; n < NR; ++n) mma_f16(sc[kg][n], kf, qf[n][kg][s][0], qf[n][kg][s][1]);
          }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[n][e] = (KG == 2 ? sc[0][n][e] + sc[KG - 1][n][e] : sc[0][n][e]) * (rowc[n][e & 1] * ks);
      }
      if (k0 < hide_to || k0 + kStep > min(mask_from, k_hi) || s_id[bi] < 0) {
        const bool in_pool = s_id[bi] >= 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int32_t key = k0 + r8 + 8 * h;
          int32_t kp = 0x7fffffff;
          if (key >= start && key < k_hi && in_pool) {
            kp = key;
            if (key >= cache) {
              kp = cache_flat_pos(a, b, cache, key - cache);
              if (kp < 0) kp = 0x7fffffff;
            }
          }
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (kp > qpos[n][u] || kp == 0x7fffffff || (kStack && key < row_start[n][u]))
                x[n][2 * h + u] = -INFINITY;
        }
        // what lies in no key's place may be anything
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int32_t key = k0 + 2 * q + (i & 1) + 8 * (i >> 1);
          if (!(key >= start && key < k_hi && in_pool)) {
#pragma unroll
            for (int w = 0; w < VB / 4; ++w) v[i][w] = 0;
          }
        }
      }
      // ---- softmax against references that move when they fall behind
      float p[NR][4], ratio[NR][2];
      auto weigh = [&]() {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) p[n][e] = ex2_approx(x[n][e] - m_ref[n][e & 1]);
          ratio[n][0] = vs * v_inv[n][0];
          ratio[n][1] = vs * v_inv[n][1];
        }
      };
      weigh();
      bool behind = false;
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float top = fmaxf(p[n][u], p[n][2 + u]);
          behind |= fmaxf(top, top * ratio[n][u]) > kMostP;
        }
      if (__any_sync(0xffffffffu, behind)) {
        const float lg = fmaxf(log2f(vs), -120.f);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float al[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float m = fmaxf(x[n][u], x[n][2 + u]);
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
            const float old = m_ref[n][u];
            const int32_t dv_old = 127 - (int32_t)(__float_as_uint(v_inv[n][u]) >> 23);
            const float m_v = fmaxf(old + (float)dv_old, m + lg);
            m = fmaxf(old, m);
            const int32_t dv = min(126, max(-126, __float2int_rd(m_v - m)));
            m_ref[n][u] = m;
            v_inv[n][u] = __uint_as_float((uint32_t)(127 - dv) << 23);
            l[n][u] *= exp2f(old - m);
            al[u] = exp2f(old - m + (float)(dv_old - dv));
          }
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            o[n][c][0] *= al[0];
            o[n][c][1] *= al[1];
            o[n][c][2] *= al[0];
            o[n][c][3] *= al[1];
          }
        }
        weigh();
      }
      uint32_t pf[NR][2];
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float p0 = p[n][2 * h], p1 = p[n][2 * h + 1];
          l[n][0] += p0;
          l[n][1] += p1;
          pf[n][h] = transpose8x8(pack_f16x2(p0 * ratio[n][0], p1 * ratio[n][1]));
        }
      // ---- O^T += V^T P^T: output tile c holds columns r8 * VB + 2 c and the next
#pragma unroll
      for (int w = 0; w < VB / 4; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t sel = h == 0 ? 0x5140u : 0x7362u;
          const uint32_t x0 = __byte_perm(v[0][w], v[1][w], sel);
          const uint32_t x1 = __byte_perm(v[2][w], v[3][w], sel);
          const uint32_t vf[4] = {f16_lo(x0), f16_hi(x0), f16_lo(x1), f16_hi(x1)};
#pragma unroll
          for (int n = 0; n < NR; ++n) mma_f16(o[n][2 * w + h], vf, pf[n][0], pf[n][1]);
        }
    }
    if (!ok)  // the copies still in flight land before the CTA is let go
      for (int i = 0; i < kStages && t < steps; ++i, ++t) {
        mbar_drain(&s_full[warp][stage], phase);
        stage = (stage + 1) % kStages;
        phase ^= stage == 0 ? 1u : 0u;
      }
    __syncwarp();

    // ---- every warp's rows to its ring's place, then the rows (or the part's share of
    // them), each by a warp that merges what the warps of its rows hold
    {
      float* mine = reinterpret_cast<float*>(ring);
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int32_t r = 8 * n + 2 * q + u;
#pragma unroll
          for (int s = 4; s < 32; s <<= 1) l[n][u] += __shfl_xor_sync(0xffffffffu, l[n][u], s);
          const float v_ref = 1.f / v_inv[n][u];
#pragma unroll
          for (int c = 0; c < NT; c += 2)
            *reinterpret_cast<float4*>(mine + r * kRowFloats + r8 * VB + 2 * c) =
                make_float4(o[n][c][u] * v_ref, o[n][c][2 + u] * v_ref, o[n][c + 1][u] * v_ref,
                            o[n][c + 1][2 + u] * v_ref);
          if (r8 == 0) s_ml[warp][r] = make_float2(m_ref[n][u], l[n][u]);
        }
    }
    if (__syncthreads_or(!ok)) break;
    constexpr int PER = D / 32;
    for (int32_t r = warp; r < RW && row0 + r < rows_total; r += W) {
      float M = -INFINITY;
      for (int32_t w = 0; w < W; ++w) M = fmaxf(M, s_ml[w][r].x);
      float sum = 0.f, acc[PER];
#pragma unroll
      for (int k = 0; k < PER; ++k) acc[k] = 0.f;
      for (int32_t w = 0; w < W; ++w) {
        const float2 ml = s_ml[w][r];
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
        sum += ml.y * f;
        const float* po =
            reinterpret_cast<const float*>(smem + w * kWarpBytes) + r * kRowFloats + lane * PER;
#pragma unroll
        for (int k = 0; k < PER; ++k) acc[k] += po[k] * f;
      }
      const int32_t row = row0 + r, j = row / G, h = g * G + (row - j * G);
      if (whole) {
        const int64_t at = ((int64_t)b * a.D_max + j) * a.Hq + h;
        if (!dbg_in(at, (int64_t)a.B * a.D_max * a.Hq, a.status)) continue;
        const float inv = 1.f / sum;
        uint32_t* ob =
            reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(a.o) + at * D + lane * PER);
#pragma unroll
        for (int k = 0; k < PER; k += 2)
          ob[k / 2] = pack_bf16x2(row_value(acc[k], inv, sum), row_value(acc[k + 1], inv, sum));
        if (a.lse != nullptr && lane == 0)
          a.lse[((int64_t)b * a.Hq + h) * a.D_max + j] = row_lse(M, sum);
      } else if constexpr (kStack) {
        const int64_t at = (((int64_t)g_first * a.D_max + j) * a.Hq + h) * L.s_splits + blockIdx.x % L.s_splits;
        if (!dbg_in(at, (int64_t)a.B * a.D_max * a.Hq * L.s_splits, a.status)) continue;
        float* po = L.s_part_o + at * D + lane * PER;
#pragma unroll
        for (int k = 0; k < PER; ++k) po[k] = acc[k];
        if (lane == 0) L.s_part_ml[at] = make_float2(M, sum);
      } else {
        // (a CTA leaves a share of several sequences, but of neighbours: slot x + b)
        const int64_t slots = L.per_head + a.B;
        const int64_t at = (((int64_t)g * L.row_groups + blockIdx.z) * slots + work.x + b) * RW + r;
        if (!dbg_in(at, (int64_t)a.cache.Hkv * L.row_groups * slots * RW, a.status)) continue;
        float* po = L.part_o + at * D + lane * PER;
#pragma unroll
        for (int k = 0; k < PER; ++k) po[k] = acc[k];
        if (lane == 0) L.part_ml[at] = make_float2(M, sum);
      }
    }
  }
  if (kShared && pdl_first_block()) pdl_wait();
}

// One warp per (sequence, draft, head): the parts of its row, weighted by their
// reference maxima.  The launch is most of its 4 us.
template <int D>
__global__ void __launch_bounds__(256) cache_attn_combine_kernel(CacheAttnArgs a, CacheAttnLaunch L) {
  pdl_wait();
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int32_t lane = threadIdx.x & 31;
  if (row >= (int64_t)a.B * a.D_max * a.Hq) return;
  const int32_t h = (int32_t)(row % a.Hq);
  const int64_t bj = row / a.Hq;
  const int32_t b = (int32_t)(bj / a.D_max), j = (int32_t)(bj - (int64_t)b * a.D_max);
  const int32_t cache = a.cache_len[b], nd = a.n_drafts[b];
  if (!cache_lengths_ok(a, cache, nd) || j >= nd) return;
  int32_t parts;
  int64_t at, step = 1, room;
  if (L.info != nullptr) {
    const int32_t G = a.Hq / a.cache.Hkv, g = h / G;
    const CacheShares x = cache_shares(L, a.B, b, L.info[b], g, j * G + (h - g * G));
    parts = x.parts;
    step = L.group_rows;
    at = x.at;
    room = (int64_t)a.cache.Hkv * L.row_groups * (L.per_head + a.B) * step;
  } else {
    parts = cache_parts(L.splits, L.min_tiles, (cache + nd + kCacheTile - 1) / kCacheTile);
    at = row * L.splits;
    room = (int64_t)a.B * a.D_max * a.Hq * L.splits;
  }
  if (parts <= 1) return;  // written by the attention kernel (or no part is known)
  if (!dbg_in(at + (parts - 1) * step, room, a.status)) return;
  float M = -INFINITY;
  for (int32_t s = lane; s < parts; s += 32) M = fmaxf(M, L.part_ml[at + s * step].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  constexpr int PER = D / 32;
  float acc[PER], sum = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) acc[k] = 0.f;
  for (int32_t s0 = 0; s0 < parts; s0 += 32) {
    float mine = 0.f;  // the factor of part s0 + lane
    if (s0 + lane < parts) {
      const float2 x = L.part_ml[at + (s0 + lane) * step];
      mine = x.x == -INFINITY ? 0.f : exp2f(x.x - M);
      sum += x.y * mine;
    }
    const int32_t n = min(32, parts - s0);
#pragma unroll 4
    for (int32_t s = 0; s < n; ++s) {
      const float f = __shfl_sync(0xffffffffu, mine, s);
      const float* po = L.part_o + (at + (s0 + s) * step) * D + lane * PER;
#pragma unroll
      for (int k = 0; k < PER; ++k) acc[k] += po[k] * f;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const float inv = 1.f / sum;
  __nv_bfloat16* ob = static_cast<__nv_bfloat16*>(a.o) + row * D + lane * PER;
#pragma unroll
  for (int k = 0; k < PER; k += 2)
    *reinterpret_cast<uint32_t*>(ob + k) =
        pack_bf16x2(row_value(acc[k], inv, sum), row_value(acc[k + 1], inv, sum));
  if (a.lse != nullptr && lane == 0)
    a.lse[((int64_t)b * a.Hq + h) * a.D_max + j] = row_lse(M, sum);
}

// 3D view of a cache: {d bytes, tokens of a block, blocks x heads}, box {d, a step, 1}.
bool step_map(CUtensorMap* map, const void* base, const ssd_block_cache& c) {
  EncodeTiledFn fn = tensor_map_encoder();
  if (fn == nullptr) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)c.d, (cuuint64_t)c.block,
                              (cuuint64_t)c.num_blocks * (cuuint64_t)c.Hkv};
  const cuuint64_t strides[2] = {(cuuint64_t)c.d, (cuuint64_t)c.d * (cuuint64_t)c.block};
  const cuuint32_t box[3] = {(cuuint32_t)c.d, kStep, 1}, estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE,
            c.d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int NR, int W, int kMode>
cudaError_t launch_mma(const CacheAttnArgs& a, dim3 grid, const CacheAttnLaunch& L, cudaStream_t stream) {
  CUtensorMap tk, tv;
  if (!step_map(&tk, a.cache.k, a.cache) || !step_map(&tv, a.cache.v, a.cache))
    return cudaErrorInvalidValue;
  auto smem = [](int32_t blocks) {
    return 1024 + (size_t)W * kStagesOf<NR, W, kMode == 1> * 2 * kStep * D + (size_t)blocks * 12;
  };
  const cudaError_t e =
      allow_smem(cache_attn_kernel<D, NR, W, kMode>, smem(part_blocks(kMode == 2 ? kMostPartTiles : kWorkRoom, kLeastBlock)));
  if (e != cudaSuccess) return e;
  return launch_kernel(cache_attn_kernel<D, NR, W, kMode>, grid, dim3(W * 32), smem(L.max_blocks), stream, true, tk, tv, a, L);
}

size_t part_bytes(int64_t rows, int32_t d) {
  return align256((size_t)rows * d * sizeof(float)) + align256((size_t)rows * sizeof(float2));
}
// Part rows of the tensor-core kernel and of the other one (0: nothing is cut).
int64_t tc_part_rows(int32_t B, int32_t Hq, int32_t D_max, int32_t splits) {
  return splits == 1 ? 0 : (int64_t)B * D_max * Hq * splits;
}
template <int D, int kMode>
cudaError_t launch_mma_of(const CacheAttnArgs& a, const CacheMmaPlan& p, const CacheAttnLaunch& L,
                          cudaStream_t stream) {
  const dim3 grid(p.per_head, a.cache.Hkv, p.row_groups);
  return p.rows > 8          ? launch_mma<D, 2, kWarps, kMode>(a, grid, L, stream)
         : p.warps == kWarps ? launch_mma<D, 1, kWarps, kMode>(a, grid, L, stream)
                             : launch_mma<D, 1, kManyWarps, kMode>(a, grid, L, stream);
}

}  // namespace

CacheMmaPlan cache_attention_mma_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max) {
  return make_plan(B, Hq, Hkv, D_max, L_max);
}
int64_t cache_attention_mma_rows(int32_t B, int32_t Hkv, const CacheMmaPlan& p, bool all) {
  return all || p.cut(B) ? (int64_t)Hkv * p.row_groups * (p.per_head + B) * p.rows : 0;
}
void cache_attention_mma_fill(CacheAttnLaunch& L, const CacheMmaPlan& p, int32_t L_max, int32_t block) {
  L.min_tiles = kMinTiles;
  L.per_head = p.per_head;
  L.goal = p.goal;
  L.uniform = p.uniform;
  L.row_groups = p.row_groups;
  L.group_rows = p.rows;
  L.max_blocks = part_blocks(std::min((L_max + kCacheTile - 1) / kCacheTile, kWorkRoom), block);
}
cudaError_t launch_cache_attention_mma(const CacheAttnArgs& a, const CacheMmaPlan& p,
                                       const CacheAttnLaunch& L, cudaStream_t stream) {
  if (a.groups > 0)
    return a.cache.d == 128 ? launch_mma_of<128, 1>(a, p, L, stream) : launch_mma_of<64, 1>(a, p, L, stream);
  return a.cache.d == 128 ? launch_mma_of<128, 0>(a, p, L, stream) : launch_mma_of<64, 0>(a, p, L, stream);
}
cudaError_t launch_cache_attention_stack(const CacheAttnArgs& a, const CacheAttnLaunch& L, int32_t rows,
                                         cudaStream_t stream) {
  const dim3 grid((unsigned)((int64_t)L.s_splits * a.cache.Hkv * a.groups), 1, kStackTurns);
  if (a.cache.d == 128)
    return rows > 8 ? launch_mma<128, 2, kWarps, 2>(a, grid, L, stream) : launch_mma<128, 1, kWarps, 2>(a, grid, L, stream);
  return rows > 8 ? launch_mma<64, 2, kWarps, 2>(a, grid, L, stream) : launch_mma<64, 1, kWarps, 2>(a, grid, L, stream);
}

size_t cache_attention_workspace(int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t D_max,
                                 int32_t L_max) {
  int64_t rows;
  if (cache_attention_tc_runs(B, Hq, Hkv, D_max, L_max)) {
    int32_t splits, min_tiles;
    cache_attention_tc_plan(B, Hq, Hkv, D_max, L_max, &splits, &min_tiles);
    rows = tc_part_rows(B, Hq, D_max, splits);
  } else {
    rows = cache_attention_mma_rows(B, Hkv, make_plan(B, Hq, Hkv, D_max, L_max), false);
  }
  return rows == 0 ? 0 : part_bytes(rows, d) + align256((size_t)B * sizeof(int2));
}

cudaError_t launch_cache_attention(const CacheAttnArgs& a, void* ws, cudaStream_t stream) {
  const int32_t L_max = a.max_blocks * a.cache.block, d = a.cache.d;
  const int32_t tiles = (L_max + kCacheTile - 1) / kCacheTile;
  const bool tc = cache_attention_tc_runs(a.B, a.Hq, a.cache.Hkv, a.D_max, L_max);
  CacheMmaPlan p{};
  CacheAttnLaunch L{};
  int64_t rows;
  if (tc) {
    cache_attention_tc_plan(a.B, a.Hq, a.cache.Hkv, a.D_max, L_max, &L.splits, &L.min_tiles);
    rows = tc_part_rows(a.B, a.Hq, a.D_max, L.splits);
    L.max_blocks = part_blocks(cache_part_tiles(L.splits, L.min_tiles, tiles), a.cache.block);
  } else {
    p = make_plan(a.B, a.Hq, a.cache.Hkv, a.D_max, L_max);
    cache_attention_mma_fill(L, p, L_max, a.cache.block);
    rows = cache_attention_mma_rows(a.B, a.cache.Hkv, p, false);
  }
  if (rows > 0) {
    unsigned char* at = static_cast<unsigned char*>(ws);
    L.part_o = reinterpret_cast<float*>(at);
    at += align256((size_t)rows * d * sizeof(float));
    L.part_ml = reinterpret_cast<float2*>(at);
    at += align256((size_t)rows * sizeof(float2));
    if (!tc) L.info = reinterpret_cast<int2*>(at);
  }
  const cudaError_t e = tc ? launch_cache_attention_tc(a, L, stream) : launch_cache_attention_mma(a, p, L, stream);
  if (e != cudaSuccess || rows == 0) return e;
  const dim3 grid((unsigned)(((int64_t)a.B * a.D_max * a.Hq + 7) / 8));
  return launch_kernel(d == 128 ? cache_attn_combine_kernel<128> : cache_attn_combine_kernel<64>, grid,
                       dim3(256), 0, stream, true, a, L);
}

}  // namespace ssd
