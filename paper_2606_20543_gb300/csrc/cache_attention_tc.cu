// cache_attention_tc.cu — frontier attention over the paged 8-bit cache on the
// 5th-generation tensor cores (include/ssd.h, ssd_cache_attention):
//   O[b][j][h] = softmax_s(scale * Q[b][j][h] . (sk K[s]) + M(s, j)) (sv V[s]).
//
// K stays e4m3 from the cache to the products (kind::f8f6f4): it is copied by TMA, 128 bytes
// a key, and never widened; Q is split in two e4m3 terms, x = hi + lo with hi the nearest
// e4m3 and lo the nearest to the rest, at the cost of twice the products, which run at twice the
// rate of bf16's, after its rows are scaled by a power of two (largest entry in [128, 256)).  That
// keeps bf16's 8 significant bits of entries down to 2^-10 of the row's largest; below, lo's least
// step is absolute, and the error 2^-18 of that largest.  P, which changes with every tile, is rounded to
// float16 instead (a split takes six instructions a pair, and the softmax is what bounds this
// kernel): two warps widen V to float16, exactly, and the second product is kind::f16.  The K
// scale of a block multiplies the scores, its V scale over the row's reference the probabilities.
//
// One CTA (8 warps, two CTAs per SM) per tile of 128 query rows (drafts x the query
// heads of a KV head) and part of the sequence's keys, longest sequences first:
//  warp 4 streams K and V in tiles of 64 keys through rings of kNK and kNV
//    stages, a copy per cache block (TMA, 64- or 128-byte swizzle);
//  warp 5 issues S = (Qhi + Qlo) K^T of the next tile into one of two TMEM buffers, then O += P V
//    of the tile before with P read from TMEM, where it replaced S;
//  warps 6-7 widen V into one of two buffers (and clear the rows that hold no key); as four
//    warps, with another for each product, they took issue slots from the softmax by waiting
//    (25 x 48 drafts 34.3 us, 29.3 now);
//  warps 0-3 (a thread a row, with the registers that the other warps give up) turn S into
//    P.  A row has two references, of its scores (for the sum) and of its scores times their
//    V scales (for P), so P's float16 holds the row whatever the scales of keys that it does not
//    see or hardly weighs.  A reference moves only when its maximum grows by more than 2^8; O is
//    rescaled in TMEM when the second one does.
//
// 128 drafts of 8 sequences over 2300 to 3800 keys, 32 heads (222 MB, 51 GFLOP): 73 us, 3.0 TB/s,
// 0.45 of the measured copy rate; the tensor pipe is busy for a quarter of it.  A tile takes
// 1200 cycles of an SM with two CTAs, and a CTA of such a pair about 2200: 650 for the
// exponentials, 370 for the maximum, 270 for S out of TMEM, the rest between the warps (when all of it
// took 80 us it was 59 without the softmax, 76 without the exponentials, 75 without widening
// V).  All tiles at the first rate are 48 us; the 60 of the longest sequence at the second are
// 65, and units are not cut here (256 for 304 places, 48 of the 152 SMs with one), so that
// sequence bounds it.  With draft_pos 78 us: a tile that holds drafts reads a position per key
// and row.  25 sequences of 48 drafts over 120 to 700 keys,
// 16 heads (56 MB): 29 us (with draft_pos 33), of which a CTA's set-up takes 3.5 and its seven
// tiles about twice that; 48 rows fill three eighths of a tile, and 400 units take a second
// round in 304 places.  The attention over a bf16 cache takes 67 and 20 us for the two: this one
// saves memory, not time.  Tiles of 128 keys with V in e4m3 as well (P in two terms, 8 softmax warps) were
// slower by a sixth, so the products are not what to save.
#include <cuda_fp16.h>

#include <algorithm>

#include "cache_attention.cuh"

namespace ssd {

namespace {

constexpr int kBM = 128;
constexpr int KT = kCacheTile;
constexpr int kNK = 3, kNV = 2;              // K and V stages
constexpr uint32_t kCols = 256;              // S/P x 2 (64 columns each), O at 128
constexpr int kThreadsTC = 256;
// Registers of a thread: 128 at launch (two CTAs per SM), then 184 for the softmax's warps and
// 72 for the others.
constexpr int kRegsSoftmax = 184, kRegsOther = 72;
constexpr int kCtasPerSm = 2;
constexpr int kMinTiles = 6;                 // a part's fewest tiles
constexpr int kMaxPartTiles = 256;           // at most 1024 block ids and scales in shared memory
constexpr int kMaxDrafts = 4096;             // whose positions are kept in shared memory
constexpr float kLog2e = 1.4426950408889634f;
// log2 growth of a row's maxima that moves their references: P stays below 2^8 in float16
constexpr float kGrowth = 8.f;
constexpr float kLeastVScale = 0x1p-110f;    // lesser ones count as this (an append's is 2^-109)
// Bytes of one term of Q, a K (or V) tile and a V tile in float16.
__host__ __device__ constexpr int q_bytes(int d) { return kBM * d; }
__host__ __device__ constexpr int tile_bytes(int d) { return KT * d; }
__host__ __device__ constexpr int wide_bytes(int d) { return 2 * KT * d; }

// fp32 D; A and B e4m3 (kind::f8f6f4) or float16 (kind::f16), whose codes are both 0.
__host__ __device__ constexpr uint32_t idesc_of(int m, int n, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma8_ss(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                        uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// float16 pairs to e4m3 pairs and back (exactly).
__device__ __forceinline__ uint32_t e4m3_of_f16(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
  return r;
}
__device__ __forceinline__ uint32_t f16_of_e4m3(uint32_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
  return h;
}
// A pair as hi and lo terms (16 bits each).
__device__ __forceinline__ void split2(float2 x, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(x.x, x.y);
  const uint32_t hb = *reinterpret_cast<const uint32_t*>(&h);
  hi = e4m3_of_f16(hb);
  const uint32_t back = f16_of_e4m3(hi);
  const __half2 rest = __hsub2(h, *reinterpret_cast<const __half2*>(&back));
  lo = e4m3_of_f16(*reinterpret_cast<const uint32_t*>(&rest));
}

// 16 consecutive 32-bit columns of this thread's TMEM lane (warp-collective).
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
      "%14,%15,%16};\n"
      "tcgen05.wait::st.sync.aligned;" ::"r"(taddr),
      "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
      "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
      "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])), "r"(__float_as_uint(v[8])),
      "r"(__float_as_uint(v[9])), "r"(__float_as_uint(v[10])), "r"(__float_as_uint(v[11])),
      "r"(__float_as_uint(v[12])), "r"(__float_as_uint(v[13])), "r"(__float_as_uint(v[14])),
      "r"(__float_as_uint(v[15]))
      : "memory");
}

// Store 8 columns, without the wait.
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

__device__ __forceinline__ uint64_t low_bits(int32_t n) {
  return n <= 0 ? 0ull : (n >= 64 ? ~0ull : ((1ull << n) - 1ull));
}

// mbar_drain(), inlined: a call has no place beside setmaxnreg.
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) {
#pragma unroll 1
  for (int i = 0; i < (1 << 14) && !mbar_try_wait(bar, parity); ++i) __nanosleep(256);
}

// Arrival of the warp's lane 0, without a branch.
__device__ __forceinline__ void arrive_lane0(uint64_t* bar, int lane) {
  asm volatile(
      "{\n .reg .pred p;\n setp.eq.u32 p, %1, 0;\n"
      " @p mbarrier.arrive.shared::cta.b64 _, [%0];\n}" ::"r"(smem_u32(bar)),
      "r"(lane)
      : "memory");
}

__device__ __forceinline__ void take_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
}
__device__ __forceinline__ void give_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
}

// Rows of d bytes are swizzled over their own length (TMA and products alike): pieces of 16 bytes
// by the row's place among 8 rows (128 bytes), or by that of its pair among 4 (64 bytes).
template <int D>
__device__ __forceinline__ uint32_t piece_at(int row, int piece) {
  return (uint32_t)(row * D + ((piece ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4));
}
// Descriptor of such rows, K-major: groups of 8 rows.
template <int D>
__device__ __forceinline__ uint64_t rows_desc(uint32_t saddr) {
  const uint64_t d = smem_desc(saddr, 16, 8 * D);
  return D == 128 ? d : (d & ~(7ull << 61)) | 4ull << 61;  // 64-byte swizzle
}

struct alignas(16) Shared {
  uint64_t k_full[kNK], k_empty[kNK], v_full[kNV], v_empty[kNV];
  uint64_t w_full[2];  // V widened
  uint64_t s_full[2], p_ready[2], pv_done[2];
  uint32_t tmem;
  int3 seq;             // the sequence, its cache length and drafts
  float rowc[kBM];      // a row's factor of the scores
  int32_t len[kLptMax]; // sequences' keys
};

template <int D>
__global__ void __launch_bounds__(kThreadsTC, kCtasPerSm)
cache_attn_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     CacheAttnArgs a, CacheAttnLaunch L, int32_t mtiles) {
  constexpr int kQBytes = q_bytes(D), kTileBytes = tile_bytes(D), kWideBytes = wide_bytes(D);
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* sQ = smem;                        // hi, lo
  unsigned char* sK = sQ + 2 * kQBytes;
  unsigned char* sV = sK + kNK * kTileBytes;
  unsigned char* sW = sV + kNV * kTileBytes;       // V in float16 [2][d / 64][KT][128 bytes]
  Shared& sh = *reinterpret_cast<Shared*>(sW + 2 * kWideBytes);
  // the part's blocks: K scale, log2 of the V scale, its inverse, id (-1: outside the pool)
  float4* s_blk = reinterpret_cast<float4*>(&sh + 1);
  int32_t* s_flat = reinterpret_cast<int32_t*>(s_blk + L.max_blocks);  // the drafts' positions
  const bool staged = a.draft_pos != nullptr && a.D_max <= kMaxDrafts;
  pdl_wait();

  const int32_t tid = threadIdx.x, lane = tid & 31, warp = (int32_t)warp_uniform(tid >> 5);
  const int32_t S = a.cache.block, S_log = 31 - __clz(S), Hkv = a.cache.Hkv, G = a.Hq / Hkv;
  int32_t unit = blockIdx.x;
  const int32_t split = unit % L.splits;
  unit /= L.splits;
  const int32_t mtile = unit % mtiles;
  unit /= mtiles;
  const int32_t g = unit % Hkv, rank = unit / Hkv;

  // ---- the sequence: the rank-th longest (batches above 256 keep their order)
  int32_t b = rank, cache, nd;
  if (a.B <= 32) {
    // every warp for itself, a sequence a lane
    const int32_t c = lane < a.B ? a.cache_len[lane] : 0, n = lane < a.B ? a.n_drafts[lane] : 0;
    const int32_t mine = lane < a.B ? (cache_lengths_ok(a, c, n) && n > 0 ? c + n : 0) : -1;
    int32_t r = 0;
#pragma unroll
    for (int32_t j = 0; j < 32; ++j) {
      const int32_t kj = __shfl_sync(0xffffffffu, mine, j);
      r += kj > mine || (kj == mine && j < lane);
    }
    b = __ffs(__ballot_sync(0xffffffffu, r == rank)) - 1;
    cache = __shfl_sync(0xffffffffu, c, b);
    nd = __shfl_sync(0xffffffffu, n, b);
  } else if (a.B <= kLptMax) {
    int32_t mine = 0, c = 0, n = 0;
    if (tid < a.B) {
      c = a.cache_len[tid];
      n = a.n_drafts[tid];
      mine = cache_lengths_ok(a, c, n) && n > 0 ? c + n : 0;
      sh.len[tid] = mine;
    }
    __syncthreads();
    if (tid < a.B) {
      int32_t r = 0;
#pragma unroll 4
      for (int32_t j = 0; j < a.B; ++j) {
        const int32_t kj = sh.len[j];
        r += kj > mine || (kj == mine && j < tid);
      }
      if (r == rank) sh.seq = make_int3(tid, c, n);
    }
    __syncthreads();
    b = sh.seq.x;
    cache = sh.seq.y;
    nd = sh.seq.z;
  } else {
    cache = a.cache_len[b];
    nd = a.n_drafts[b];
  }
  if (!cache_lengths_ok(a, cache, nd)) {
    if (tid == 0 && split == 0 && g == 0 && mtile == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
    return;
  }
  const int32_t Lk = cache + nd, rows_total = nd * G, row0 = mtile * kBM;
  const int32_t tiles = (Lk + KT - 1) / KT;
  const int32_t parts = cache_parts(L.splits, L.min_tiles, tiles);
  if (row0 >= rows_total || split >= parts) return;
  int32_t t_lo = 0, t_hi = tiles;
  if (parts > 1) {
    t_lo = (int32_t)((int64_t)tiles * split / parts);
    t_hi = (int32_t)((int64_t)tiles * (split + 1) / parts);
  }
  const int32_t k_lo = t_lo * KT, k_hi = min(Lk, t_hi * KT), ntiles = t_hi - t_lo;
  const int32_t start = a.key_start != nullptr ? min(Lk, max(0, a.key_start[b])) : 0;
  const int32_t b_lo = k_lo >> S_log, nb = ((k_hi - 1) >> S_log) + 1 - b_lo;

  // ---- set-up
  if (tid == 0) {
    for (int i = 0; i < kNK; ++i) {
      mbar_init(&sh.k_full[i], 1);
      mbar_init(&sh.k_empty[i], 1);
    }
    for (int i = 0; i < kNV; ++i) {
      mbar_init(&sh.v_full[i], 1);
      mbar_init(&sh.v_empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.w_full[i], 2);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_ready[i], 4);
      mbar_init(&sh.pv_done[i], 1);
    }
    fence_barrier_init();
  }
  if (warp == 7) {
    tmem_alloc(&sh.tmem, kCols);
    tmem_relinquish();
  }
  if (warp == 4 && lane < 2) prefetch_tensormap(lane == 0 ? &tmK : &tmV);
  bool bad = false;  // a block outside the pool
  // warps 4-7: the part's blocks and the drafts' positions; the others: Q
  const bool stages = warp >= 4 && warp < 8;
  for (int32_t i = stages ? tid - 128 : nb; i < nb; i += 128) {
    int32_t id = a.block_table[(int64_t)b * a.max_blocks + b_lo + i];
    if (id < 0 || id >= a.cache.num_blocks) {
      record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      id = -1;
      bad = true;
    }
    const int64_t at = (int64_t)max(id, 0) * Hkv + g;
    const float vs = a.cache.v_scale[at], least = fmaxf(vs, kLeastVScale);
    s_blk[i] = make_float4(a.cache.k_scale[at], id >= 0 && vs > 0.f ? log2f(least) : -INFINITY,
                           1.f / least, __int_as_float(id));
  }
  if (a.draft_pos != nullptr) {
    for (int32_t j = stages ? tid - 128 : nd; j < nd; j += 128) {
      const int32_t p = cache_flat_pos(a, b, cache, j);
      if (p < 0 && split == 0 && g == 0 && mtile == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      if (staged) s_flat[j] = p;
    }
  }
  // Q as two terms, two threads a row, the row scaled to [128, 256) (rows behind the last
  // one stay what they were: they reach no other row)
#pragma unroll 1
  for (int32_t q_row = tid >> 1; !stages && q_row < kBM && row0 + (q_row & ~15) < rows_total;
       q_row += 64) {
    const int32_t r = row0 + q_row, half = tid & 1;
    const bool live = r < rows_total;
    const int32_t j = live ? r / G : 0, h = g * G + (live ? r - j * G : 0);
    const uint4* src = reinterpret_cast<const uint4*>(
                           static_cast<const __nv_bfloat16*>(a.q) +
                           (((int64_t)b * a.D_max + j) * a.Hq + h) * D) + half * (D / 16);
    uint4 w[D / 16];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) w[i] = live ? src[i] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        m = fmax3(m, fabsf(__uint_as_float(v[e] << 16)), fabsf(__uint_as_float(v[e] & 0xffff0000u)));
    }
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    // 2^(7 - e), e the exponent of the largest entry
    const int32_t e = (int32_t)(__float_as_uint(m) >> 23) - 127, up = max(-120, min(126, 7 - e));
    // (an infinity, which e4m3 would clamp: every product of the row is NaN, as its softmax is)
    const float f = m == INFINITY ? NAN : __uint_as_float((uint32_t)(up + 127) << 23);
    if (half == 0)
      sh.rowc[q_row] = (a.scale != 0.f ? a.scale : rsqrtf((float)D)) * kLog2e *
                       __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4& x = w[2 * c + (i >> 1)];
        const uint32_t p0 = (i & 1) ? x.z : x.x, p1 = (i & 1) ? x.w : x.y;
        uint32_t h0, l0, h1, l1;
        const float2 x0 = make_float2(__uint_as_float(p0 << 16), __uint_as_float(p0 & 0xffff0000u));
        const float2 x1 = make_float2(__uint_as_float(p1 << 16), __uint_as_float(p1 & 0xffff0000u));
        split2(make_float2(x0.x * f, x0.y * f), h0, l0);
        split2(make_float2(x1.x * f, x1.y * f), h1, l1);
        hi[i] = h0 | (h1 << 16);
        lo[i] = l0 | (l1 << 16);
      }
      const uint32_t off = piece_at<D>(q_row, half * (D / 32) + c);
      *reinterpret_cast<uint4*>(sQ + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(sQ + kQBytes + off) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    fence_proxy_async_shared();
  }
  tc_fence_before();
  const bool any_bad = __syncthreads_or(bad) != 0;
  tc_fence_after();
  const uint32_t tmem = sh.tmem, tO = tmem + 128;

  // Rows of tile t that hold no key of the sequence (behind its end, before its
  // start, of a block outside the pool), as a bit mask of the others
  auto live_keys = [&](int32_t c0) -> uint64_t {
    uint64_t m = low_bits(k_hi - c0) & ~low_bits(start - c0);
    if (m == 0) return 0;
#pragma unroll 1
    for (int32_t k = 0; k < KT; k += min(S, KT))
      if (c0 + k < k_hi && __float_as_int(s_blk[((c0 + k) >> S_log) - b_lo].w) < 0)
        m &= ~(low_bits(min(S, KT)) << k);
    return m;
  };

  if (warp == 4) {
    // ------------------------------------------------------------ producer
    give_registers();
    const bool leader = elect_one();
    const uint64_t pol = policy_evict_first();
    const int32_t rows = min(S, KT);
    bool ok = true;
    int32_t t = 0, nk = 0, nv = 0;  // tiles; K and V copies issued
#pragma unroll 1
    for (; t < ntiles && ok; ++t) {
      const int32_t c0 = k_lo + t * KT;
      // (blocks behind the last key are not copied: their rows stay what they were)
      const int32_t n = min(KT, k_hi - c0);
      const uint32_t bytes = (uint32_t)((n + rows - 1) / rows * rows * D);
      auto copy = [&](unsigned char* dst, const CUtensorMap* map, uint64_t* full) {
        if (leader) {
          mbar_arrive_expect_tx(full, bytes);
#pragma unroll 1
          for (int32_t k = 0; k < n; k += rows) {
            const int32_t id = max(__float_as_int(s_blk[((c0 + k) >> S_log) - b_lo].w), 0);
            const int32_t row = (id * Hkv + g) * S + ((c0 + k) & (S - 1));
            tma_load_2d(dst + k * D, map, 0, row, full, pol);
          }
        }
        __syncwarp();
      };
      if (t >= kNK) ok = wait_warp(&sh.k_empty[t % kNK], ((t / kNK) - 1) & 1, a.status);
      if (!ok) break;
      copy(sK + t % kNK * kTileBytes, &tmK, &sh.k_full[t % kNK]);
      nk = t + 1;
      if (t >= kNV) ok = wait_warp(&sh.v_empty[t % kNV], ((t / kNV) - 1) & 1, a.status);
      if (!ok) break;
      copy(sV + t % kNV * kTileBytes, &tmV, &sh.v_full[t % kNV]);
      nv = t + 1;
    }
    // after a wait that gave up, the copies in flight still land here
    if (!ok) {
      for (int32_t u = max(0, nk - kNK); u < nk; ++u) drain(&sh.k_full[u % kNK], (u / kNK) & 1);
      for (int32_t u = max(0, nv - kNV); u < nv; ++u) drain(&sh.v_full[u % kNV], (u / kNV) & 1);
    }
  } else if (warp == 5) {
    // ------------------------------------------------------------- products
    give_registers();
    const uint32_t tSu = warp_uniform(tmem), tOu = warp_uniform(tO), aQ = warp_uniform(smem_u32(sQ));
    const uint32_t aK = warp_uniform(smem_u32(sK)), aW = warp_uniform(smem_u32(sW));
    const bool leader = elect_one();
    const uint64_t dq = rows_desc<D>(aQ);
    constexpr uint32_t kIdescS = idesc_of(kBM, KT, false), kIdescO = idesc_of(kBM, D, true);
    int32_t ns = 0, np = 0;  // tiles whose products were issued
    bool ok = true;
#pragma unroll 1
    while (ok && np < ntiles) {
      // S of the next tile, then PV of the one before
      if (ns < ntiles) {
        const int s = ns % kNK, sb = ns & 1;
        ok = wait_warp(&sh.k_full[s], (ns / kNK) & 1, a.status);
        // the S/P buffer is free once PV of tile ns - 2 is done
        if (ok && ns >= 2) ok = wait_warp(&sh.pv_done[sb], ((ns >> 1) - 1) & 1, a.status);
        if (!ok) break;
        tc_fence_after();
        const uint64_t dk = rows_desc<D>(aK + s * kTileBytes);
        if (leader) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks)
              mma8_ss(tSu + sb * KT, smem_desc_at(dq, u * kQBytes + ks * 32), smem_desc_at(dk, ks * 32),
                      kIdescS, u + ks > 0 ? 1u : 0u);
          mma_commit(&sh.s_full[sb]);
          mma_commit(&sh.k_empty[s]);
        }
        __syncwarp();
        if (ns++ == 0) continue;
      }
      const int sb = np & 1;
      ok = wait_warp(&sh.w_full[sb], (np >> 1) & 1, a.status) &&
           wait_warp(&sh.p_ready[sb], (np >> 1) & 1, a.status);
      if (!ok) break;
      tc_fence_after();
      // A = P in TMEM (16 keys = 8 columns a step), B = V in float16 (MN-major: blocks of 64
      // columns KT * 128 bytes apart, 8-key groups 1 KB apart; 16 keys = 2 KB)
      const uint64_t dv = smem_desc(aW + sb * kWideBytes, KT * 128, 1024);
      if (leader) {
#pragma unroll
        for (int kk = 0; kk < KT / 16; ++kk)
          mma_ts(tOu, tSu + sb * KT + kk * 8, smem_desc_at(dv, kk * 2048), kIdescO,
                 np + kk > 0 ? 1u : 0u);
        mma_commit(&sh.pv_done[sb]);
      }
      __syncwarp();
      ++np;
    }
    if (!ok && ns > 0) drain(&sh.s_full[(ns - 1) & 1], ((ns - 1) >> 1) & 1);
    if (!ok && np > 0) drain(&sh.pv_done[(np - 1) & 1], ((np - 1) >> 1) & 1);
  } else if (warp >= 6) {
    // ------------------------------------------------- V widened, 32 keys a warp
    give_registers();
    // A lane takes 16 values (a 16-byte chunk) of a key, eight keys by four chunks a step:
    // then a lane's places in the swizzled tiles are fixed, and eight lanes' stores fill all
    // banks (with eight chunks of a key a step and the halves swapped to avoid conflicts the
    // warp took 2600 cycles a tile).  Rows without a key hold whatever the pool holds, and
    // their P of 0 times a NaN would be one: cleared.
    const int c = lane & 3, k8 = lane >> 2;
    const uint32_t src0 = piece_at<D>(k8, c), src1 = D == 128 ? piece_at<D>(k8, c + 4) : 0;
    const uint32_t dst0 = k8 * 128 + (((2 * c) ^ k8) << 4), dst1 = k8 * 128 + (((2 * c + 1) ^ k8) << 4);
#pragma unroll 1
    for (int32_t t = 0; t < ntiles; ++t) {
      const int s = t % kNV, sb = t & 1;
      const int32_t c0 = k_lo + t * KT;
      bool ok = wait_warp(&sh.v_full[s], (t / kNV) & 1, a.status);
      if (ok && t >= 2) ok = wait_warp(&sh.pv_done[sb], ((t >> 1) - 1) & 1, a.status);
      if (!ok) break;
      const unsigned char* from = sV + s * kTileBytes;
      unsigned char* to = sW + sb * kWideBytes;
      const bool whole = c0 >= start && c0 + KT <= k_hi && !any_bad;
      const uint64_t live = whole ? ~0ull : live_keys(c0);
#pragma unroll
      for (int i = 4 * (warp - 6); i < 4 * (warp - 6) + 4; ++i) {
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {  // blocks of 64 columns
          uint4 w = *reinterpret_cast<const uint4*>(from + i * 8 * D + (h ? src1 : src0));
          if (!whole && !(live >> (8 * i + k8) & 1ull)) w = make_uint4(0u, 0u, 0u, 0u);
          unsigned char* at = to + h * (KT * 128) + i * 1024;
          *reinterpret_cast<uint4*>(at + dst0) = make_uint4(
              f16_of_e4m3(w.x), f16_of_e4m3(w.x >> 16), f16_of_e4m3(w.y), f16_of_e4m3(w.y >> 16));
          *reinterpret_cast<uint4*>(at + dst1) = make_uint4(
              f16_of_e4m3(w.z), f16_of_e4m3(w.z >> 16), f16_of_e4m3(w.w), f16_of_e4m3(w.w >> 16));
        }
      }
      fence_proxy_async_shared();
      __syncwarp();
      arrive_lane0(&sh.w_full[sb], lane);
      arrive_lane0(&sh.v_empty[s], lane);
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------- softmax
    take_registers();
    const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
    const int32_t r = row0 + tid;
    const bool warp_live = row0 + warp * 32 < rows_total;
    const float rowc = sh.rowc[tid];
    const int32_t j = r < rows_total ? r / G : 0;
    int32_t qpos = 0x7fffffff;
    auto flat_of = [&](int32_t i) { return staged ? s_flat[i] : cache_flat_pos(a, b, cache, i); };
    if (r < rows_total) qpos = flat_of(j);
    // keys below this one are visible to every row of the warp
    const int32_t mask_from = min(cache, __reduce_min_sync(0xffffffffu, qpos) + 1);
    // references (log2) of the scores, for the sum, and of the scores times their V scales, for
    // P; v_ref = 2^(m_v - m_run)
    float m_run = -INFINITY, m_v = -INFINITY, v_ref = 0.f, l_run = 0.f;
    bool ok = true;
    int32_t t = 0;
#pragma unroll 1
    for (; t < ntiles; ++t) {
      const int sb = t & 1;
      const int32_t c0 = k_lo + t * KT;
      // scales of the tile's groups of 16 keys: K's, V's log2 and inverse
      float f[4], lg[4], iv[4];
      if (S_log >= 6) {  // the tile is of one block
        const int32_t at = (c0 >> S_log) - b_lo;
        const float4 x = s_blk[at];
        f[0] = f[1] = f[2] = f[3] = fmaxf(rowc * x.x, 1e-37f);
        lg[0] = lg[1] = lg[2] = lg[3] = x.y;
        iv[0] = iv[1] = iv[2] = iv[3] = x.z;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int32_t at = (min(c0 + 16 * i, k_hi - 1) >> S_log) - b_lo;
          const float4 x = s_blk[at];
          f[i] = fmaxf(rowc * x.x, 1e-37f);
          lg[i] = x.y;
          iv[i] = x.z;
        }
      }
      ok = ok && wait_warp(&sh.s_full[sb], (t >> 1) & 1, a.status);
      if (!ok) break;
      tc_fence_after();
      if (warp_live) {
        float sv[64];
        tmem_ld32(tmem + lane_off + sb * KT, sv);
        tmem_ld32(tmem + lane_off + sb * KT + 32, sv + 32);
        if (c0 + KT > mask_from || c0 < start || c0 + KT > k_hi || any_bad) {
          uint64_t keep;
          if (a.draft_pos == nullptr) {
            keep = low_bits(qpos < 0x7fffffff ? qpos + 1 - c0 : KT);
          } else {
            keep = low_bits(min(cache, qpos < 0x7fffffff ? qpos + 1 : cache) - c0);
#pragma unroll 1
            for (int32_t k = max(0, cache - c0); k < min(KT, k_hi - c0); ++k) {
              const int32_t p = flat_of(c0 + k - cache);
              if (p >= 0 && p <= qpos) keep |= 1ull << k;
            }
          }
          keep &= live_keys(c0);
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (!(keep >> i & 1ull)) sv[i] = -INFINITY;
        }
        float mx = -INFINITY, mxv = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* x = sv + 16 * i;
          float y = fmax3(x[0], x[1], x[2]), z = fmax3(x[3], x[4], x[5]);
#pragma unroll
          for (int e = 6; e < 14; e += 4) {
            y = fmax3(y, x[e], x[e + 1]);
            z = fmax3(z, x[e + 2], x[e + 3]);
          }
          const float top = fmax3(fmaxf(y, z), x[14], x[15]) * f[i];
          mx = fmaxf(mx, top);
          mxv = fmaxf(mxv, top + lg[i]);
        }
        float alpha = 1.f;
        bool moved = false;
        if (mx > m_run + kGrowth) {  // (of nothing: -inf, and a factor of 0)
          l_run *= ex2_approx(m_run - mx);
          m_run = mx;
        }
        if (mxv > m_v + kGrowth) {
          alpha = ex2_approx(m_v - mxv);
          m_v = mxv;
          moved = true;
        }
        if (t > 0 && __any_sync(0xffffffffu, moved)) {
          // O may be rescaled once PV of the tile before is done
          ok = wait_warp(&sh.pv_done[(t - 1) & 1], ((t - 1) >> 1) & 1, a.status);
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            float ov[16];
            tmem_ld16(tO + lane_off + c * 16, ov);
#pragma unroll
            for (int i = 0; i < 16; ++i) ov[i] *= alpha;
            tmem_st16(tO + lane_off + c * 16, ov);
          }
        }
        const float m = m_run == -INFINITY ? 0.f : m_run, v_lg = m_v - m_run;
        v_ref = m_run == -INFINITY ? 0.f : ex2_approx(v_lg);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t pk[8];
          // P times its V scale over the reference, in the exponent.  A block whose scale is
          // next to nothing beside the reference (or 0, a block outside the pool, a row that has
          // seen no key) adds to the sum alone.
          const bool tiny = !(lg[i] - v_lg > -60.f);
          const float off = tiny ? -m : lg[i] - m_v;
          float2 s2[2];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 x = ffma2(make_float2(sv[16 * i + 2 * e], sv[16 * i + 2 * e + 1]),
                                   make_float2(f[i], f[i]), make_float2(off, off));
            const float2 p = make_float2(ex2_approx(x.x), ex2_approx(x.y));
            s2[e & 1] = e < 2 ? p : fadd2(s2[e & 1], p);
            const __half2 h = __floats2half2_rn(p.x, p.y);
            pk[e] = *reinterpret_cast<const uint32_t*>(&h);
          }
          if (tiny) {
#pragma unroll
            for (int e = 0; e < 8; ++e) pk[e] = 0;
          }
          const float2 ss = fadd2(s2[0], s2[1]);
          l_run += (ss.x + ss.y) * (tiny ? 1.f : v_ref * iv[i]);
          tmem_st8(tmem + lane_off + sb * KT + 8 * i, pk);  // (waited for below)
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      }
      tc_fence_before();
      __syncwarp();
      arrive_lane0(&sh.p_ready[sb], lane);
    }
    // ---- epilogue
    if (ok) ok = wait_warp(&sh.pv_done[(ntiles - 1) & 1], ((ntiles - 1) >> 1) & 1, a.status);
    tc_fence_after();
    if (ok && warp_live) {
      const bool live = r < rows_total;
      const int32_t h = g * G + (r - j * G);
      const int64_t orow = ((int64_t)b * a.D_max + j) * a.Hq + h;
      const bool direct = parts == 1;
      const int64_t prow = orow * L.splits + split;
      const bool store = live && (direct ? dbg_in(orow, (int64_t)a.B * a.D_max * a.Hq, a.status)
                                         : dbg_in(prow, (int64_t)a.B * a.D_max * a.Hq * L.splits, a.status));
      const float inv = v_ref / l_run;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float ov[32];
        tmem_ld32(tO + lane_off + c * 32, ov);
        if (!store) continue;
        if (direct) {
          uint4* ob = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.o) + orow * D + c * 32);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = row_value(ov[8 * i + e], inv, l_run);
            ob[i] = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                               pack_bf16x2(x[6], x[7]));
          }
        } else {
          float4* po = reinterpret_cast<float4*>(L.part_o + prow * D + c * 32);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            po[i] = make_float4(ov[4 * i] * v_ref, ov[4 * i + 1] * v_ref, ov[4 * i + 2] * v_ref,
                                ov[4 * i + 3] * v_ref);
        }
      }
      if (store) {
        if (!direct) L.part_ml[prow] = make_float2(m_run, l_run);
        else if (a.lse != nullptr)
          a.lse[((int64_t)b * a.Hq + h) * a.D_max + j] = row_lse(m_run, l_run);
      }
    }
  }
  // ---- teardown
  tc_fence_before();
  __syncthreads();
  if (warp == 7) {
    tc_fence_after();
    tmem_dealloc(tmem, kCols);
  }
}

// 2D view of a cache: {d bytes, rows}, box {d, rows of a copy}.
bool cache_map(CUtensorMap* map, const void* base, int64_t rows, int32_t box_rows, int32_t d) {
  EncodeTiledFn fn = tensor_map_encoder();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)d};
  const cuuint32_t box[2] = {(cuuint32_t)d, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE,
            d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch(const CacheAttnArgs& a, const CacheAttnLaunch& L, cudaStream_t stream) {
  const int32_t mtiles = (int32_t)(((int64_t)a.D_max * (a.Hq / a.cache.Hkv) + kBM - 1) / kBM);
  const int64_t rows = (int64_t)a.cache.num_blocks * a.cache.Hkv * a.cache.block;
  const int32_t box = std::min(a.cache.block, KT);
  CUtensorMap tk, tv;
  if (!cache_map(&tk, a.cache.k, rows, box, D) || !cache_map(&tv, a.cache.v, rows, box, D))
    return cudaErrorInvalidValue;
  auto smem = [](int32_t blocks, int32_t drafts) {
    return 1024 + 2 * q_bytes(D) + (kNK + kNV) * tile_bytes(D) + 2 * wide_bytes(D) + sizeof(Shared) +
           (size_t)blocks * 16 + (size_t)drafts * 4;
  };
  // (a part has at most a tile more than kMaxPartTiles)
  const cudaError_t e = allow_smem(cache_attn_tc_kernel<D>,
                                   smem(part_blocks(kMaxPartTiles + 1, kLeastBlock), kMaxDrafts));
  if (e != cudaSuccess) return e;
  const int64_t grid = (int64_t)a.B * a.cache.Hkv * mtiles * L.splits;
  if (grid > INT32_MAX) return cudaErrorInvalidValue;
  return launch_kernel(cache_attn_tc_kernel<D>, dim3((unsigned)grid), dim3(kThreadsTC),
                       smem(L.max_blocks, a.draft_pos != nullptr && a.D_max <= kMaxDrafts ? a.D_max : 0),
                       stream, true, tk, tv, a, L, mtiles);
}

}  // namespace

// From 17 query rows on (the mma.sync kernel takes 16 to a CTA, and every CTA reads the keys for
// itself): 16 sequences of 4000 keys, 8 heads: 128-wide, 17 rows 44 us here and 59 there; 64-wide
// 35 and 47 (48 rows and 8 sequences of 32 heads: 66 and 130).
bool cache_attention_tc_runs(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max) {
  const int64_t rows = (int64_t)D_max * (Hq / Hkv);
  return rows > 16 && !cache_attention_few(B, Hkv, rows, L_max);
}

void cache_attention_tc_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max,
                             int32_t* splits, int32_t* min_tiles) {
  const int64_t mtiles = ((int64_t)D_max * (Hq / Hkv) + kBM - 1) / kBM;
  const int64_t base = (int64_t)B * Hkv * mtiles, tiles = (L_max + KT - 1) / KT;
  const int64_t target = (int64_t)kCtasPerSm * device_sm_count();
  const int64_t most = std::max<int64_t>(1, tiles / kMinTiles);
  const int64_t least = (tiles + kMaxPartTiles - 1) / kMaxPartTiles;
  *min_tiles = kMinTiles;
  *splits = (int32_t)std::max<int64_t>(least, std::min<int64_t>(target / base, most));
}

cudaError_t launch_cache_attention_tc(const CacheAttnArgs& a, const CacheAttnLaunch& L,
                                      cudaStream_t stream) {
  return a.cache.d == 128 ? launch<128>(a, L, stream) : launch<64>(a, L, stream);
}

}  // namespace ssd
