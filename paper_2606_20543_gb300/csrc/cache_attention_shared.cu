// cache_attention_shared.cu — attention over the paged 8-bit cache for sequences that share the
// blocks of a long prompt (include/ssd.h, ssd_cache_attention_shared).  With P the tokens of the
// blocks that a group shares, a row's softmax over its keys is that over [0, P) joined with that
// over [P, end): with (m, l, o) the maximum, sum and unnormalised output of each,
//   M = max m_i,   o = sum o_i 2^(m_i - M) / sum l_i 2^(m_i - M).
// The keys in [0, P) are the same for all rows of the group, so those rows are stacked into the
// 128-row tiles of the tensor-core kernel (cache_attention_tc.cu), which reads the keys once a tile
// instead of once a sequence; up to 16 rows a group, about, go to the mma.sync kernel
// (cache_attention.cu), 8 or 16 at a time.  The keys from P on are each sequence's own: on the same kernel, in
// the same launch, or, for few rows, on the mma.sync one (cache_attention.cu).  Both leave part rows,
// which the kernel here joins.
//
// One token of 64 sequences of one group, 4352 shared keys and 100 to 1000 own, 32/8 heads (73 MB):
// 38 us, 1.9 TB/s: the set-up, first tile and way out of three kernels' CTAs (18000 cycles of a
// shared unit's 30000), and own keys at 2.5 TB/s beside the shared ones.  48 drafts of 8 groups of 4
// over 1500 to 8000 shared keys, 16 heads: 118 us, the softmax of the tensor-core kernel.  35 tokens of 7
// groups over 6300 shared keys, 8 heads of 64 (46 MB): 20 us, without sharing 54.
#include <algorithm>
#include <cmath>

#include "cache_attention.cuh"

namespace ssd {

namespace {

constexpr int kSharedTiles = 3;        // fewest tiles of a part of the shared keys,
constexpr int kSharedPartTiles = 256;  // and about the most
constexpr double kSharedFixed = 9.5;   // tiles that a unit's set-up, way out and share of the join are worth,
constexpr double kFewFixed = 6;        // and one of few rows on the mma.sync kernel

// Whether sharing pays, by what both ways take (us, from the largest lengths that the call allows).  A
// tile of the tensor-core kernel takes an SM 4.8e-3 of a GPU's us where all its warps have rows,
// less where some have none; the mma.sync kernel streams keys at 5.6 (64-wide heads: 6.4) TB/s; a CTA
// takes 0.75 us a tile however few there are of them (0.7), and 12 ns more (8, of the own keys); the
// join reads its parts at 3 TB/s.  Sharing starts three kernels instead of one and sets up units of few
// tiles: 16 us (11 with few rows of a group, 14 with the own keys in the same launch) instead of 6 (10; 4
// more where sequences are cut).  Measured, shared and not: 64 sequences of one group, 4352 + 1000 keys,
// 32/8 heads 37 and 102; 50 of 4 drafts over 13000, 33 and 138; 8 groups of 4, 48 drafts over 8000 + 600,
// 16 heads 117 and 152; 7 groups of 5 over 6300, 8 heads of 64 20 and 54; 6 of 14, 6 drafts
// over 2200 + 1400, 6/2 heads 35 and 58; 10 of 3 over 1000, 32 heads 60 and 43; 8 groups of 2 over 4900
// + 1900, 41 and 25; 3 of 42 drafts over 1800 + 1000, 6/2 heads 22 and 17.  Where it is wrong: small work, which
// cache_attention_few() keeps from it (20 sequences of 4 groups over 1408, 8 heads of 64: 13 shared, 16 not,
// as chosen); many heads of short own keys (182 of 14 groups over 256, 32 heads: 132 as chosen, 87); 380 of 10
// over 704, 8 heads of 64: 41, 63 as chosen; and groups of very unequal size, whose sizes are on the device: 19 of
// one and one of 61, over 4096, 32/8 heads 176 as chosen (the large
// group's 244 rows, 16 a turn, read the keys eight times one after the other), 95 not.
bool sharing_pays(int32_t B, int32_t groups, int32_t Hq, int32_t Hkv, int32_t d, int32_t D_max,
                  int32_t L_max, int32_t max_shared, const CacheSharedPlan& p) {
  const double G = Hq / Hkv, per_seq = D_max * G, rows = (double)B * D_max * Hq;
  const double shared = std::ceil(max_shared / 64.0), own = std::ceil((L_max - max_shared) / 64.0);
  const double tiles_r = std::max<double>(groups, B * per_seq / 128 + groups / 2.0);
  const double stacked = tiles_r * Hkv * shared * 4.8e-3;
  const double join = rows * (std::min<double>(p.s_splits, shared / p.s_min_tiles) + 1) * d * 4 / 3e6;
  if (p.own_tc) {
    int32_t splits, min_tiles;
    cache_attention_tc_plan(B, Hq, Hkv, D_max, L_max, &splits, &min_tiles);
    const double full = std::ceil(std::min(per_seq, 128.0) / 32) / 4, units = B * Hkv * std::ceil(per_seq / 128);
    const double tile = 4.8e-3 * (0.4 + 0.6 * full), alone = 10 + 12e-3 * units +
                        std::max(units * (shared + own) * tile, 0.75 * (shared + own) / splits);
    return 14 + stacked + units * (own * tile + 12e-3) + join < 0.9 * alone;
  }
  const CacheMmaPlan plan = cache_attention_mma_plan(B, Hq, Hkv, D_max, L_max);
  const double ctas = plan.uniform > 0 ? (double)B * plan.uniform : plan.goal;
  const double us_of_tile = (double)B * Hkv * 2 * d * 64 / (d == 128 ? 5.6e6 : 6.4e6);
  const double alone = 6 + (plan.cut(B) ? 4 : 0) +
                       std::max(us_of_tile * (shared + own), 0.7 * B * (shared + own) / ctas);
  const double few = std::max(us_of_tile / B * groups * shared, 0.7 * shared / p.s_splits);
  return (p.few > 0 ? 11 + few : 16 + stacked) + us_of_tile * own + 8e-3 * B * Hkv + join < 0.9 * alone;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
size_t part_bytes(int64_t rows, int32_t d) {
  return align256((size_t)rows * d * sizeof(float)) + align256((size_t)rows * sizeof(float2));
}

constexpr int kTogether = 4;
template <int N>
struct alignas(4 * N) Lanes {
  float x[N];
};

// One warp per (sequence, draft, head): the parts of its row over the shared keys and over its own.
// CTA: a draft, eight heads.  What bounds it is the chain from the lengths over the parts' places to
// their rows, and its code, which is fetched cold: no division of 64 bits, four parts at a time (14 KB
// of code instead of 26 KB: 64 sequences over 4352 shared keys 39.5 -> 38.2 us, all of the call).
template <int D>
__global__ void __launch_bounds__(256) cache_attn_join_kernel(CacheAttnArgs a, CacheAttnLaunch L) {
  constexpr int PER = D / 32;
  pdl_wait();
  const int32_t lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && blockIdx.y == 0) {  // (nothing else looks at all of the groups)
    bool bad = false;
    for (int32_t g = threadIdx.x; g < a.groups; g += blockDim.x)
      bad |= a.group_start[g] > a.group_start[g + 1];
    if (threadIdx.x == 0) bad |= a.group_start[0] != 0 || a.group_start[a.groups] != a.B;
    if (bad) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
  }
  const int32_t h0 = (blockIdx.y * 8 + (threadIdx.x >> 5)) * L.join_heads;
  if (h0 >= a.Hq) return;
  const int32_t b = (int32_t)(blockIdx.x / (uint32_t)a.D_max), j = blockIdx.x - b * a.D_max;
  const int32_t cache = a.cache_len[b], nd = a.n_drafts[b];
  const int2 cut = L.info != nullptr ? L.info[b] : make_int2(0, 0);
  const CacheGroup group = cache_group_warp(a, b);
  if (!cache_lengths_ok(a, cache, nd) || j >= nd) return;
  const int32_t base = group.base(a, b, cache);
  if (base < 0) return;
  const int32_t shared_tiles = (base + kCacheTile - 1) / kCacheTile;
  const int32_t n_shared = shared_tiles > 0 ? cache_parts(L.s_splits, L.s_min_tiles, shared_tiles) : 0;
  const int32_t n_tiles =
      L.info != nullptr ? 1 : cache_parts(L.splits, L.min_tiles, (cache + nd - base + kCacheTile - 1) / kCacheTile);
#pragma unroll 1
  for (int32_t h = h0; h < min(a.Hq, h0 + L.join_heads); ++h) {
    const int64_t row = (int64_t)blockIdx.x * a.Hq + h;
    int32_t n_own = n_tiles, step = 1;
    int64_t at = row * L.splits;
    if (L.info != nullptr) {
      const int32_t G = a.Hq / a.cache.Hkv, g = h / G;
      const CacheShares x = cache_shares(L, a.B, b, cut, g, j * G + (h - g * G));
      n_own = x.parts;
      step = L.group_rows;
      at = x.at;
      if (!dbg_in(at + (n_own - 1) * step, (int64_t)a.cache.Hkv * L.row_groups * (L.per_head + a.B) * step,
                  a.status))
        return;
    }
    if (n_own <= 0) return;  // (a wait gave up: no part is known)
    const int32_t parts = n_shared + n_own;
    const int64_t s_at = row * L.s_splits, own_at = at - (int64_t)n_shared * step;
    auto ml_of = [&](int32_t s) {
      return s < n_shared ? L.s_part_ml[s_at + s] : L.part_ml[own_at + (int64_t)s * step];
    };
    // The first parts' rows are asked for together with the factors of all.
    Lanes<PER> v[kTogether], acc;
    auto rows_of = [&](int32_t i0) {
#pragma unroll
      for (int i = 0; i < kTogether; ++i) {
        const int32_t s = min(i0 + i, parts - 1);
        const float* p = s < n_shared ? L.s_part_o + (s_at + s) * D : L.part_o + (own_at + (int64_t)s * step) * D;
        v[i] = *reinterpret_cast<const Lanes<PER>*>(p + lane * PER);
      }
    };
    rows_of(0);
    const float2 first = lane < parts ? ml_of(lane) : make_float2(-INFINITY, 0.f);
    float M = first.x;
#pragma unroll 1
    for (int32_t s = 32 + lane; s < parts; s += 32) M = fmaxf(M, ml_of(s).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
    for (int k = 0; k < PER; ++k) acc.x[k] = 0.f;
    float sum = 0.f, mine = 0.f;  // the factor of part (s0 & ~31) + lane
#pragma unroll 1
    for (int32_t s0 = 0; s0 < parts; s0 += kTogether) {
      if ((s0 & 31) == 0) {
        const float2 x = s0 == 0 ? first : s0 + lane < parts ? ml_of(s0 + lane) : make_float2(-INFINITY, 0.f);
        mine = x.x == -INFINITY ? 0.f : exp2f(x.x - M);
        sum += x.y * mine;
      }
      if (s0 > 0) rows_of(s0);
#pragma unroll
      for (int i = 0; i < kTogether; ++i) {
        const float f = __shfl_sync(0xffffffffu, mine, (s0 + i) & 31);
        if (s0 + i >= parts || f == 0.f) continue;
#pragma unroll
        for (int k = 0; k < PER; ++k) acc.x[k] += v[i].x[k] * f;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = 1.f / sum;
    uint32_t w[PER / 2];
#pragma unroll
    for (int k = 0; k < PER; k += 2)
      w[k / 2] = pack_bf16x2(row_value(acc.x[k], inv, sum), row_value(acc.x[k + 1], inv, sum));
    uint32_t* ob = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(a.o) + row * D + lane * PER);
    if constexpr (PER == 4) *reinterpret_cast<uint2*>(ob) = make_uint2(w[0], w[1]);
    else ob[0] = w[0];
    if (a.lse != nullptr && lane == 0) a.lse[((int64_t)b * a.Hq + h) * a.D_max + j] = row_lse(M, sum);
  }
}

}  // namespace

CacheSharedPlan cache_attention_shared_plan(int32_t how, int32_t B, int32_t groups, int32_t Hq, int32_t Hkv,
                                            int32_t d, int32_t D_max, int32_t L_max, int32_t max_shared) {
  CacheSharedPlan p{};
  const int64_t G = Hq / Hkv, per_seq = D_max * G, rows = (int64_t)B * D_max * Hq;
  p.plain = max_shared <= 0 || how == kShareNever ||
            (how != kShareAlways && (2 * (int64_t)groups > B || cache_attention_few(B, Hkv, per_seq, L_max)));
  if (p.plain) return p;
  // (a group's last tile may be part empty)
  const int64_t tiles_r = (B * per_seq) / 128 + groups, tiles = (max_shared + kCacheTile - 1) / kCacheTile;
  // Parts of the shared keys: n of them make base * n units, which take an SM's share of base * n *
  // kSharedFixed tiles beside the tiles themselves, and the end waits for a unit of tiles / n: least for
  // n = sqrt(tiles * SMs / (base * kSharedFixed)); and no second round for a few units.  Measured (us, by
  // n): 64 sequences of one group over 4352 keys, 32/8 heads 1: 82, 3: 41, 6: 36, 11: 39, 20: 50; 72 of
  // two groups over 11900, 32/8 heads 5: 79, 10: 55, 20: 66, 32: 88; 48 drafts, 8 groups of 4 over 1500
  // to 8000, 16 heads 1: 138, 2: 128, 3: 119, 5: 130, 8: 149.
  p.own_tc = per_seq > 16;
  p.few = !p.own_tc && B * per_seq <= 16 * (int64_t)groups ? (int32_t)((B * per_seq + groups - 1) / groups) : 0;
  const int64_t sms = device_sm_count(), base = tiles_r * Hkv, places = (p.few > 0 && d == 64 ? 3 : 2) * sms;
  int64_t n = (int64_t)std::ceil(std::sqrt(tiles * sms / ((p.few > 0 ? kFewFixed : kSharedFixed) * base)));
  if (base <= places && base * n > places && 4 * base * n <= 7 * places) n = places / base;
  p.s_min_tiles = (int32_t)std::min<int64_t>(kSharedPartTiles / 2, std::max<int64_t>(kSharedTiles, tiles / n));
  p.s_splits = (int32_t)std::max<int64_t>(1, tiles / p.s_min_tiles);
  if (base * p.s_splits > INT32_MAX / 2) {
    p.plain = true;
    return p;
  }
  p.s_units = (int32_t)(base * p.s_splits);
  p.s_rows = rows * p.s_splits;
  if (how != kShareAlways && !sharing_pays(B, groups, Hq, Hkv, d, D_max, L_max, max_shared, p)) {
    p.plain = true;
    return p;
  }
  if (p.own_tc) {
    cache_attention_tc_plan(B, Hq, Hkv, D_max, L_max, &p.splits, &p.min_tiles);
    p.rows = rows * p.splits;
  } else {
    p.mma = cache_attention_mma_plan(B, Hq, Hkv, D_max, L_max);
    p.rows = cache_attention_mma_rows(B, Hkv, p.mma, true);
  }
  return p;
}

size_t cache_attention_shared_bytes(const CacheSharedPlan& p, int32_t B, int32_t Hq, int32_t Hkv, int32_t d,
                                    int32_t D_max, int32_t L_max) {
  if (p.plain) return cache_attention_workspace(B, Hq, Hkv, d, D_max, L_max);
  return part_bytes(p.s_rows, d) + part_bytes(p.rows, d) + align256((size_t)B * sizeof(int2));
}

cudaError_t launch_cache_attention_shared(const CacheAttnArgs& a, const CacheSharedPlan& p, void* ws,
                                          cudaStream_t stream) {
  const int32_t S = a.cache.block, L_max = a.max_blocks * S, d = a.cache.d;
  if (p.plain) {
    CacheAttnArgs one = a;
    one.groups = 0;
    return launch_cache_attention(one, ws, stream);
  }
  CacheAttnLaunch L{};
  const int32_t tiles = (L_max + kCacheTile - 1) / kCacheTile;
  const int32_t shared_tiles = (a.max_shared * S + kCacheTile - 1) / kCacheTile;
  const int32_t s_blocks = part_blocks(cache_part_tiles(p.s_splits, p.s_min_tiles, shared_tiles), S);
  L.s_units = p.s_units;
  L.s_splits = p.s_splits;
  L.s_min_tiles = p.s_min_tiles;
  L.early = !p.own_tc;
  unsigned char* at = static_cast<unsigned char*>(ws);
  L.s_part_o = reinterpret_cast<float*>(at);
  at += align256((size_t)p.s_rows * d * sizeof(float));
  L.s_part_ml = reinterpret_cast<float2*>(at);
  at += align256((size_t)p.s_rows * sizeof(float2));
  L.part_o = reinterpret_cast<float*>(at);
  at += align256((size_t)p.rows * d * sizeof(float));
  L.part_ml = reinterpret_cast<float2*>(at);
  at += align256((size_t)p.rows * sizeof(float2));
  L.splits = p.splits;
  L.min_tiles = p.min_tiles;
  L.max_blocks = s_blocks;
  if (p.own_tc)
    L.max_blocks = std::max(s_blocks, part_blocks(cache_part_tiles(p.splits, p.min_tiles, tiles), S));
  cudaError_t e = p.few > 0 ? launch_cache_attention_stack(a, L, p.few, stream)
                            : launch_cache_attention_tc(a, L, stream, p.own_tc);
  if (e != cudaSuccess) return e;
  if (!p.own_tc) {
    L.info = reinterpret_cast<int2*>(at);
    cache_attention_mma_fill(L, p.mma, L_max, S);
    e = launch_cache_attention_mma(a, p.mma, L, stream);
    if (e != cudaSuccess) return e;
  }
  // (with rows for every place of a warp several times over, what a warp looks up serves several heads)
  const int64_t warps = (int64_t)a.B * a.D_max * a.Hq, places = (int64_t)device_sm_count() * 32;
  L.join_heads = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4, warps / (2 * places)));
  const dim3 grid((unsigned)(a.B * a.D_max), (unsigned)((a.Hq + 8 * L.join_heads - 1) / (8 * L.join_heads)));
  return launch_kernel(d == 128 ? cache_attn_join_kernel<128> : cache_attn_join_kernel<64>, grid, dim3(256),
                       0, stream, true, a, L);
}

}  // namespace ssd
