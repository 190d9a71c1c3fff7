// cache_attention.cuh — what the two kernels of the attention over the paged
// 8-bit cache share: how a sequence's keys are split, the partial rows and the
// positions of drafts.
#pragma once

#include "kernels.cuh"

namespace ssd {

constexpr int kCacheTile = 64;  // keys: parts of a sequence are whole tiles

// A sequence that is cut leaves each part's share of its rows for the combine
// kernel, else the attention writes the rows itself.  The tensor-core kernel cuts
// a sequence of `tiles` tiles into parts of about equal length, at most `splits`,
// none shorter than min_tiles (but the only one); part p holds tiles
// [tiles * p / n, tiles * (p + 1) / n).  The other one deals all sequences' tiles to the
// CTAs of a KV head: CacheWork.
struct CacheAttnLaunch {
  int32_t splits, min_tiles;
  int32_t max_blocks;  // most blocks of a part (room for their ids and scales)
  float* part_o;       // [B][D_max][Hq][splits][d]; or [Hkv][row groups][per_head + B][rows][d]
  float2* part_ml;     // the same without d: reference maximum (log2) and sum
  // CacheWork
  int32_t per_head, goal, uniform, row_groups, group_rows;
  int2* info;          // [B]: first and last CTA of a sequence
};

constexpr int kWorkTiles = 128;  // a CTA's most tiles of one sequence, about (kWorkRoom: at most)
constexpr int kWorkRoom = kWorkTiles + 8;

__host__ __device__ __forceinline__ int32_t cache_parts(int32_t splits, int32_t min_tiles,
                                                        int32_t tiles) {
  const int32_t n = tiles / min_tiles;
  return n < 1 ? 1 : (n < splits ? n : splits);
}
constexpr int kLeastBlock = 16;  // tokens
// Most blocks that so many tiles lie in (a part may start inside a block of 128 tokens).
inline int32_t part_blocks(int32_t tiles, int32_t block) {
  return tiles * (kCacheTile / (block < kCacheTile ? block : kCacheTile)) + 1;
}
// Most tiles of a part of any sequence of at most `tiles` tiles.
inline int32_t cache_part_tiles(int32_t splits, int32_t min_tiles, int32_t tiles) {
  const int32_t even = tiles / splits + 1, few = 2 * min_tiles;  // n < splits: tiles / n < 2 min
  return splits == 1 ? tiles : (even > few ? even : few);
}

// A row's shares that the CTAs of CacheWork left: the first one's place among the part rows (the
// next is group_rows on), and how many.  `row`: of the KV head's rows of sequence b; `cut`:
// L.info[b].  A CTA that gave up on a wait leaves the info of its later sequences unwritten, so
// what is no range of CTAs stands for none.
struct CacheShares {
  int64_t at;
  int32_t parts;
};
__host__ __device__ __forceinline__ CacheShares cache_shares(const CacheAttnLaunch& L, int32_t B,
                                                             int32_t b, int2 cut, int32_t g,
                                                             int32_t row) {
  if (cut.x < 0 || cut.y < cut.x || cut.y >= L.per_head) return CacheShares{0, 0};
  const int32_t z = row / L.group_rows;
  const int64_t slots = L.per_head + B;
  return CacheShares{(((int64_t)g * L.row_groups + z) * slots + cut.x + b) * L.group_rows +
                         (row - z * L.group_rows),
                     cut.y - cut.x + 1};
}

// mbar_wait_warp() with one try ahead of the loop: a wait for what is there already takes a try
// and a vote (through the loop 220 cycles on a busy SM, of the 2200 that a tile of 64 keys takes).
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, int32_t* status) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return mbar_wait_warp(bar, parity, status);
}

// A row's way out.  A row that sees no key has the sum 0, and nothing else has: then it is 0 and
// -inf, whatever its products are (0 times a NaN of the pool).  A NaN in a key that it sees, or in
// its query, makes the sum a NaN, and that goes out.
__device__ __forceinline__ float row_value(float x, float inv, float sum) {
  return sum == 0.f ? 0.f : x * inv;
}
__device__ __forceinline__ float row_lse(float m_log2, float sum) {
  return sum == 0.f ? -INFINITY : (m_log2 + log2f(sum)) * 0.6931471805599453f;
}

// Flat position of draft j of sequence b; -1 outside the grid.
__device__ __forceinline__ int32_t cache_flat_pos(const CacheAttnArgs& a, int32_t b, int32_t cache,
                                                  int32_t j) {
  if (a.draft_pos == nullptr) return cache + j;
  const int32_t i = a.draft_pos[(int64_t)b * a.D_max + j];
  if (i < 0 || i >= a.grid.grid_h * a.grid.grid_w) return -1;
  const int32_t y = i / a.grid.grid_w;
  return a.grid.prefix_len + y * a.grid.row_stride + (i - y * a.grid.grid_w);
}

// Whether sequence b's lengths are in range (with cache and nd read).
__device__ __forceinline__ bool cache_lengths_ok(const CacheAttnArgs& a, int32_t cache, int32_t nd) {
  return cache >= 0 && nd >= 0 && nd <= a.D_max && cache <= a.max_blocks * a.cache.block - nd;
}

// What CTA x of a KV head's per_head works on: parts of sequences, one after the other.
//  - The sequences alone fill the GPU (uniform > 0): as many CTAs for every sequence.
//  - Else a sequence gets a CTA for every `chunk` tiles, with the least chunk for which `goal`
//    CTAs (those that run at once) suffice, so lengths that differ leave no CTA with more than
//    `chunk` tiles.
//  - Where that is more than kEvenTiles tiles above an even share (8 sequences for 14 CTAs),
//    the tiles of all sequences, in one line, are cut evenly, and a CTA may work on the end of
//    one sequence and the beginning of the next.  A cut that would leave a sliver of a sequence
//    moves to the sequence's end.  8 sequences of 8000 keys, 32 heads: 108 -> 95 us; with 16
//    sequences of 2000 keys for 57 CTAs, a tile or two from even, the second part's
//    set-up costs more than it gives (20 -> 22 us).
// Called by converged warps; every lane holds the same.
constexpr int kEvenTiles = 8;
// A sequence shorter than this many of the shortest parts is not cut: the launch that combines
// the parts takes 4 us (8 heads over 1200 keys: 12.4 us whole, 14.6 in two).
constexpr int kCutFrom = 3;
struct CacheWork {
  int32_t b, t_lo, t_hi, tiles;  // the part: tiles t_lo .. t_hi - 1 of the tiles of sequence b
  // the line: the CTA's tiles left, and where sequence b begins
  int64_t at, end, start;

  // Tiles of a sequence; report: bad lengths are recorded.
  static __device__ __forceinline__ int32_t tiles_of(const CacheAttnArgs& a, int32_t b, bool report) {
    const int32_t c = a.cache_len[b], n = a.n_drafts[b];
    if (!cache_lengths_ok(a, c, n)) {
      if (report) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      return 0;
    }
    return n == 0 ? 0 : (c + n + kCacheTile - 1) / kCacheTile;
  }

  // The sequence that holds tile x of the line, from sequence b0 = a multiple of 32 on, which
  // begins at `begin`: false if none.
  __device__ __noinline__ bool find(const CacheAttnArgs& a, int64_t x) {
    const int32_t lane = threadIdx.x & 31;
    int64_t before = 0;
    for (int32_t b0 = 0; b0 < a.B; b0 += 32) {
      const int32_t n = b0 + lane < a.B ? tiles_of(a, b0 + lane, false) : 0;
      int64_t upto = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      upto += before;
      const uint32_t here = __ballot_sync(0xffffffffu, x < upto);
      if (here != 0) {
        const int32_t src = __ffs(here) - 1;
        b = b0 + src;
        tiles = __shfl_sync(0xffffffffu, n, src);
        start = __shfl_sync(0xffffffffu, upto, src) - tiles;
        return true;
      }
      before = __shfl_sync(0xffffffffu, upto, 31);
    }
    return false;
  }
  // The cut at tile x, and with it the sequence it lies in.
  __device__ __forceinline__ int64_t cut(const CacheAttnArgs& a, int64_t x, int32_t sliver) {
    if (!find(a, x)) return x;
    if (x - start <= sliver) return start;
    return start + tiles - x <= sliver ? start + tiles : x;
  }
  // The CTA's first part; false: none.  report: the launch's first CTAs, which record bad
  // lengths.
  __device__ __forceinline__ bool first(const CacheAttnArgs& a, const CacheAttnLaunch& L, int32_t x,
                                        bool report) {
    if (L.uniform > 0) {
      b = x / L.uniform;
      const int32_t split = x - b * L.uniform;
      tiles = tiles_of(a, b, report && split == 0);
      const int32_t parts = (tiles + kWorkTiles - 1) / kWorkTiles;
      if (split >= parts) return false;
      t_lo = 0;
      t_hi = tiles;
      if (parts > 1) {
        t_lo = (int32_t)((int64_t)tiles * split / parts);
        t_hi = (int32_t)((int64_t)tiles * (split + 1) / parts);
      }
      at = end = start = 0;
      return true;
    }
    const int32_t lane = threadIdx.x & 31;
    // (the first 32 lengths stay in a register)
    const int32_t mine = lane < a.B ? tiles_of(a, lane, report && x == 0) : 0;
    int64_t total = mine;
    int32_t most = mine;
    for (int32_t i = lane + 32; i < a.B; i += 32) {
      const int32_t t = tiles_of(a, i, report && x == 0);
      total += t;
      most = max(most, t);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    // the chunk: lo - 1 is too small, hi enough (or as long as a part may be)
    most = __reduce_max_sync(0xffffffffu, most);
    auto parts_of = [&](int32_t t, int32_t chunk) {
      const int32_t at_most = t < kCutFrom * L.min_tiles ? (t > 0 ? 1 : 0) : t / L.min_tiles;
      return min((t + chunk - 1) / chunk, at_most);
    };
    int32_t hi = (int32_t)min((int64_t)min(most, kWorkTiles), total / (L.goal - a.B) + 1);
    int32_t lo = max(1, (int32_t)min((int64_t)hi, (total + L.goal - 1) / L.goal));
    while (lo < hi) {
      const int32_t chunk = (lo + hi) >> 1;
      int32_t n = parts_of(mine, chunk);
      for (int32_t i = lane + 32; i < a.B; i += 32) n += parts_of(tiles_of(a, i, false), chunk);
      if (__reduce_add_sync(0xffffffffu, n) <= L.goal) hi = chunk;
      else lo = chunk + 1;
    }
    if (total == 0) return false;
    if (hi <= total / L.goal + kEvenTiles) {
      int32_t before = 0;
      for (int32_t b0 = 0; b0 < a.B; b0 += 32) {
        const int32_t t = b0 == 0 ? mine : b0 + lane < a.B ? tiles_of(a, b0 + lane, false) : 0;
        const int32_t n = parts_of(t, hi);
        int32_t upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int32_t y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        upto += before;
        const uint32_t here = __ballot_sync(0xffffffffu, x < upto);
        if (here != 0) {
          const int32_t src = __ffs(here) - 1;
          b = b0 + src;
          tiles = __shfl_sync(0xffffffffu, t, src);
          const int32_t parts = __shfl_sync(0xffffffffu, n, src);
          const int32_t split = x - (__shfl_sync(0xffffffffu, upto, src) - parts);
          t_lo = (int32_t)((int64_t)tiles * split / parts);
          t_hi = (int32_t)((int64_t)tiles * (split + 1) / parts);
          at = end = start = 0;
          return true;
        }
        before = __shfl_sync(0xffffffffu, upto, 31);
      }
      return false;
    }
    const int64_t n = max((total + kWorkTiles - 1) / kWorkTiles,
                          min((int64_t)L.goal, max((int64_t)1, total / L.min_tiles)));
    if (x >= n) return false;
    const int32_t sliver = L.min_tiles / 2 - 1;
    end = cut(a, total * (x + 1) / n, sliver);
    at = cut(a, total * x / n, sliver);
    if (at >= start + tiles && !find(a, at)) return false;
    part();
    return true;
  }
  __device__ __forceinline__ void part() {
    t_lo = (int32_t)(at - start);
    t_hi = (int32_t)min((int64_t)tiles, end - start);
  }
  // The CTA's next part.
  __device__ __forceinline__ bool next(const CacheAttnArgs& a) {
    at = start + tiles;
    if (at >= end) return false;
    start = at;
    do tiles = tiles_of(a, ++b, false);
    while (tiles == 0);
    part();
    return true;
  }
};

// Little work: as CTAs of 8 rows whose warps share the keys, all of it is resident at once, and
// what counts is how long one CTA takes.  Every 8 rows read the keys again, from L2, so only up
// to 9 * 2^15 keys in all.  64 rows of 8 heads: over 300 keys 7.8 us, on the tensor-core kernel,
// which takes 6500 cycles to get going, 12.3; over 4000 20.3 and 21.2; 96 rows over 4000 24.9 and
// 23.6.  32 heads, 64 rows: over 1000 keys 16.8 and 19.2, over 2000 30.9 and 24.7.
inline bool cache_attention_few(int64_t B, int64_t Hkv, int64_t rows, int64_t L_max) {
  const int64_t ctas = B * Hkv * ((rows + 7) / 8);
  return ctas <= 3 * device_sm_count() && ctas * L_max <= 9 << 15;
}

// cache_attention_tc.cu: the tcgen05 kernel
bool cache_attention_tc_runs(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max);
void cache_attention_tc_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max,
                             int32_t* splits, int32_t* min_tiles);
cudaError_t launch_cache_attention_tc(const CacheAttnArgs& a, const CacheAttnLaunch& L,
                                      cudaStream_t stream);

}  // namespace ssd
