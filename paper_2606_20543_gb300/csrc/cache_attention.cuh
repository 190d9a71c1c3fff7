// cache_attention.cuh — what the two kernels of the attention over the paged
// 8-bit cache share: how a sequence's keys are split, the partial rows and the
// positions of drafts.
#pragma once

#include "kernels.cuh"

namespace ssd {

constexpr int kCacheTile = 64;  // keys: parts of a sequence are whole tiles

// A sequence of `tiles` tiles is cut into parts of about equal length, at most
// `splits`, none shorter than min_tiles (but the only one); part p holds tiles
// [tiles * p / n, tiles * (p + 1) / n).  With one part the attention writes the
// rows; else every part leaves its share of them for the combine kernel.
struct CacheAttnLaunch {
  int32_t splits, min_tiles;
  int32_t max_blocks;  // most blocks of a part (room for their ids and scales)
  float* part_o;       // [B][D_max][Hq][splits][d]
  float2* part_ml;     // [B][D_max][Hq][splits]: reference maximum (log2) and sum
};

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

// cache_attention_tc.cu: the tcgen05 kernel
bool cache_attention_tc_runs(const CacheAttnArgs& a);
void cache_attention_tc_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max,
                             int32_t* splits, int32_t* min_tiles);
cudaError_t launch_cache_attention_tc(const CacheAttnArgs& a, const CacheAttnLaunch& L,
                                      cudaStream_t stream);

}  // namespace ssd
