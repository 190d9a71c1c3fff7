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
// [tiles * p / n, tiles * (p + 1) / n).  The other one gives the CTAs of a KV head
// (per_head of them) to the sequences by their lengths: cache_work().
struct CacheAttnLaunch {
  int32_t splits, min_tiles;
  int32_t max_blocks;  // most blocks of a part (room for their ids and scales)
  float* part_o;       // [B][D_max][Hq][splits][d]; or [Hkv][row groups][per_head][rows][d]
  float2* part_ml;     // the same without d: reference maximum (log2) and sum
  // cache_work()
  int32_t per_head, goal, uniform, row_groups, group_rows;
  int2* info;          // [B]: first CTA and parts of a sequence
};

constexpr int kWorkTiles = 128;  // most tiles of a part of cache_work()

__host__ __device__ __forceinline__ int32_t cache_parts(int32_t splits, int32_t min_tiles,
                                                        int32_t tiles) {
  const int32_t n = tiles / min_tiles;
  return n < 1 ? 1 : (n < splits ? n : splits);
}
// Most tiles of a part of any sequence of at most `tiles` tiles.
inline int32_t cache_part_tiles(int32_t splits, int32_t min_tiles, int32_t tiles) {
  const int32_t even = tiles / splits + 1, few = 2 * min_tiles;  // n < splits: tiles / n < 2 min
  return splits == 1 ? tiles : (even > few ? even : few);
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

// What CTA x of a KV head's per_head works on: part `split` of `parts` of sequence b
// (b < 0: nothing).  Called by converged warps; every lane gets the same answer.
// uniform > 0: as many CTAs for every sequence.  Else a sequence gets one for every
// `chunk` tiles, with the least chunk for which `goal` of them (those that run at
// once) suffice, so lengths that differ leave no CTA with more than `chunk` tiles.
struct CacheWork {
  int32_t b, split, parts;
};
// report: the launch's first CTA of a sequence, which records bad lengths.
__device__ __forceinline__ CacheWork cache_work(const CacheAttnArgs& a, const CacheAttnLaunch& L,
                                                int32_t x, bool report) {
  const int32_t lane = threadIdx.x & 31;
  constexpr uint32_t kAll = 0xffffffffu;
  auto tiles_of = [&](int32_t b) -> int32_t {
    const int32_t c = a.cache_len[b], n = a.n_drafts[b];
    if (!cache_lengths_ok(a, c, n)) {
      if (report) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      return 0;
    }
    return n == 0 ? 0 : (c + n + kCacheTile - 1) / kCacheTile;
  };
  auto parts_of = [&](int32_t tiles, int32_t chunk) {
    return min((tiles + chunk - 1) / chunk, tiles == 0 ? 0 : max(1, tiles / L.min_tiles));
  };
  if (L.uniform > 0) {
    const int32_t b = x / L.uniform, split = x - b * L.uniform;
    report = report && split == 0;
    const int32_t parts = L.uniform == 1 ? 1 : parts_of(tiles_of(b), kWorkTiles);
    if (L.uniform == 1) report = report && tiles_of(b) >= 0;
    if (report && L.info != nullptr && lane == 0) L.info[b] = make_int2(b * L.uniform, parts);
    return CacheWork{split < parts ? b : -1, split, parts};
  }
  report = report && x == 0;
  const int32_t mine = lane < a.B ? tiles_of(lane) : 0;  // (what a batch of up to 32 needs)
  int64_t total = mine;
  int32_t most = mine;
  for (int32_t b = lane + 32; b < a.B; b += 32) {
    const int32_t t = tiles_of(b);
    total += t;
    most = max(most, t);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
  most = __reduce_max_sync(kAll, most);
  report = false;
  // (lo - 1 is too few, hi enough; a part longer than kWorkTiles has no room)
  int32_t hi = (int32_t)min((int64_t)min(most, kWorkTiles), total / (L.goal - a.B) + 1);
  int32_t lo = max(1, (int32_t)min((int64_t)hi, (total + L.goal - 1) / L.goal));
  while (lo < hi) {
    const int32_t chunk = (lo + hi) >> 1;
    int32_t n = parts_of(mine, chunk);
    for (int32_t b = lane + 32; b < a.B; b += 32) n += parts_of(tiles_of(b), chunk);
    if (__reduce_add_sync(kAll, n) <= L.goal) hi = chunk;
    else lo = chunk + 1;
  }
  const int32_t chunk = max(1, hi);
  CacheWork w{-1, 0, 0};
  int32_t before = 0;
  for (int32_t b0 = 0; b0 < a.B; b0 += 32) {
    const int32_t b = b0 + lane;
    const int32_t n = b >= a.B ? 0 : parts_of(b0 == 0 ? mine : tiles_of(b), chunk);
    int32_t end = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t y = __shfl_up_sync(kAll, end, o);
      if (lane >= o) end += y;
    }
    end += before;
    if (L.info != nullptr && x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x < 32 && b < a.B)
      L.info[b] = make_int2(end - n, n);
    const uint32_t here = __ballot_sync(kAll, x >= end - n && x < end);
    if (here != 0) {
      const int32_t src = __ffs(here) - 1;
      w = CacheWork{b0 + src, x - __shfl_sync(kAll, end - n, src), __shfl_sync(kAll, n, src)};
      if (x > 0) break;  // (CTA 0 writes every sequence's info)
    }
    before = __shfl_sync(kAll, end, 31);
    if (x == 0 && L.info == nullptr && w.b >= 0) break;
  }
  return w;
}

// cache_attention_tc.cu: the tcgen05 kernel
bool cache_attention_tc_runs(const CacheAttnArgs& a);
void cache_attention_tc_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max,
                             int32_t* splits, int32_t* min_tiles);
cudaError_t launch_cache_attention_tc(const CacheAttnArgs& a, const CacheAttnLaunch& L,
                                      cudaStream_t stream);

}  // namespace ssd
