// scaled_matmul.cu — products of e4m3 rows and weights with a float32 scale for every 128 entries
// of the inner length (include/ssd.h, ssd_scaled_matmul):
//   C[m][n] = sum_g sa[g][m] sw[g][n / 128] sum_{k in g} A[m][k] W[n][k]  (+ add[m][n]).
//
// The scales change along the inner length, so no accumulator of the tensor cores can hold the sum
// over g: a block of 128 (four tcgen05.mma of kind::f8f6f4) goes into a TMEM buffer of its own, and
// the epilogue's warps add it, times its scales, to sums in their registers while the tensor
// cores work on the next block in another buffer.
//
// One operand's rows are the 128 lanes of a tile, the other's its TN columns:
//  - more than 64 rows: the rows of A on the lanes (the scales are then one number a thread), over
//    64 or 128 rows of W, or a CTA pair (cta_group::2) with 128 lanes each over 256;
//  - fewer: the rows of W on the lanes and those of A as 16, 32 or 64 columns, so that a decode's
//    few rows do not leave most of each product empty.  What bounds it is W's way in, so a tile's
//    inner length is cut over a cluster of CTAs where the tiles alone would leave SMs idle;
//    they add their sums up through distributed shared memory, in the order of their ranks.
// Warps of a CTA: the epilogue's four (or eight), one that copies the lanes' operand, one that
// issues the products, one that copies the columns' operand.
#include <algorithm>

#include "kernels.cuh"

namespace ssd {

namespace {

constexpr int kGroup = 128;  // entries of a scale, bytes of a stage's rows
constexpr int kLaneRows = 128;
constexpr int kPitch = 36;   // floats of a staged row of 32 (rows start four banks apart)
constexpr int kRaster = 8;   // tiles of lanes that share the columns' tiles in L2

template <bool SWAP, bool PAIR, int TN>
struct Shape {
  static constexpr int EW = TN > 128 ? 8 : 4;             // epilogue warps
  static constexpr int CW = TN / (EW / 4);                // columns of one
  static constexpr int kThreads = (EW + 3) * 32;
  static constexpr int NB = TN >= 128 ? 2 : 4;            // TMEM buffers
  static constexpr int kLBytes = kLaneRows * kGroup;
  static constexpr int kCRows = PAIR ? TN / 2 : TN;       // of a CTA's copy
  static constexpr int kCBytes = kCRows * kGroup;
  static constexpr int kStage = kLBytes + kCBytes;
  static constexpr int kCtas = SWAP || TN == 64 ? 2 : 1;  // per SM
  static constexpr int S = PAIR ? 5 : SWAP ? (TN == 16 ? 6 : TN == 32 ? 5 : 4) : TN == 64 ? 3 : 6;
  static constexpr int P = EW == 8 ? 4 : 8;               // blocks whose scales are under way
  static constexpr int kRingFloats = SWAP ? EW * P * (TN + 4) : 2 * P * EW * 32;
  static constexpr int kStaging = SWAP ? 0 : EW * 32 * kPitch * 4;
  static constexpr int kSmem = 1024 + S * kStage + kStaging + kRingFloats * 4;
  static_assert(!SWAP || S * kStage >= TN * kLaneRows * 4, "a CTA's sums fit where its stages were");
};

struct Launch {
  int32_t tiles_l, tiles_c, splits;
  int32_t vec;  // C (and add) may be written four columns at a time
};

__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(live ? 4 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ float ld_peer(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
// An arrival at a barrier of the cluster.
__device__ __forceinline__ void arrive_peer(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// fp32 sums of e4m3 products, M x N, both operands K-major.
__host__ __device__ constexpr uint32_t idesc_e4m3(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ float from_bf16(const void* p, int64_t at) {
  return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16);
}
__device__ __forceinline__ void store_one(const ScaledMatmulArgs& a, int64_t m, int32_t n, float x) {
  if (!dbg_in(m * a.ldc + n, (a.M - 1) * a.ldc + a.N, a.status)) return;
  if (a.add != nullptr) x += from_bf16(a.add, m * a.ldadd + n);
  if (a.c_bf16) static_cast<__nv_bfloat16*>(a.c)[m * a.ldc + n] = __float2bfloat16_rn(x);
  else static_cast<float*>(a.c)[m * a.ldc + n] = x;
}
__device__ __forceinline__ void store_four(const ScaledMatmulArgs& a, int64_t m, int32_t n, float4 x) {
  if (!dbg_in(m * a.ldc + n + 3, (a.M - 1) * a.ldc + a.N, a.status)) return;
  if (a.add != nullptr) {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.add) + m * a.ldadd + n);
    x.x += __uint_as_float(w.x << 16);
    x.y += __uint_as_float(w.x & 0xffff0000u);
    x.z += __uint_as_float(w.y << 16);
    x.w += __uint_as_float(w.y & 0xffff0000u);
  }
  if (a.c_bf16)
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.c) + m * a.ldc + n) =
        make_uint2(pack_bf16x2(x.x, x.y), pack_bf16x2(x.z, x.w));
  else
    *reinterpret_cast<float4*>(static_cast<float*>(a.c) + m * a.ldc + n) = x;
}

template <bool SWAP, bool PAIR, int TN>
__global__ void __launch_bounds__(Shape<SWAP, PAIR, TN>::kThreads, Shape<SWAP, PAIR, TN>::kCtas)
scaled_matmul_kernel(const __grid_constant__ CUtensorMap tmL, const __grid_constant__ CUtensorMap tmC,
                     ScaledMatmulArgs a, Launch L) {
  using H = Shape<SWAP, PAIR, TN>;
  constexpr int EW = H::EW, CW = H::CW, NB = H::NB, S = H::S, P = H::P;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* staging = reinterpret_cast<float*>(smem + S * H::kStage);
  float* ring = reinterpret_cast<float*>(smem + S * H::kStage + H::kStaging);
  __shared__ uint64_t full[S], empty[S], tfull[NB], tempty[NB];
  __shared__ uint32_t tmem_slot;
  pdl_wait();

  const int32_t tid = threadIdx.x, lane = tid & 31, warp = (int32_t)warp_uniform(tid >> 5);
  const int32_t cluster = PAIR ? 2 : L.splits;
  const int32_t rank = cluster > 1 ? (int32_t)(blockIdx.x % cluster) : 0;
  const int32_t first = blockIdx.x / cluster, step = gridDim.x / cluster;
  const int32_t total = L.tiles_l * L.tiles_c;
  const int32_t blocks = (a.K + kGroup - 1) / kGroup;
  int32_t kb_lo = 0, kb_hi = blocks;
  if (SWAP && cluster > 1) {
    kb_lo = (int32_t)((int64_t)blocks * rank / cluster);
    kb_hi = (int32_t)((int64_t)blocks * (rank + 1) / cluster);
  }
  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 2);  // the two producers
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < NB; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], PAIR ? 2 * EW : EW);
    }
    fence_barrier_init();
  }
  if (warp == EW + 1) {
    if constexpr (PAIR) {
      tmem_alloc_pair(&tmem_slot, NB * TN);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(&tmem_slot, NB * TN);
      tmem_relinquish();
    }
  }
  if (warp == EW && lane < 2) prefetch_tensormap(lane == 0 ? &tmL : &tmC);
  tc_fence_before();
  if constexpr (PAIR) cluster_sync_all();  // (the peer's barriers too are initialised)
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  // Tile i: which rows of the lanes' and of the columns' operand.
  auto tile_of = [&](int32_t i, int32_t& l, int32_t& c) {
    if constexpr (SWAP) {
      c = i / L.tiles_l;
      l = i - c * L.tiles_l;
    } else {
      const int32_t per = kRaster * L.tiles_c, g = i / per, r = i - g * per;
      const int32_t n = min(kRaster, L.tiles_l - g * kRaster);
      c = r / n;
      l = g * kRaster + r - c * n;
    }
  };

  if (warp == EW || warp == EW + 2) {
    // ---------------------------------------------------------- producers
    const bool lanes = warp == EW, leader = elect_one();
    const uint64_t pol = !SWAP ? policy_evict_normal()
                               : lanes ? policy_evict_first() : policy_evict_last();
    const uint32_t bytes = (PAIR ? 2u : 1u) * (lanes ? H::kLBytes : H::kCBytes);
    const uint32_t full0 = PAIR ? peer_addr(smem_u32(full), 0) : 0;
    bool ok = true;
    int32_t n = 0, s = 0;
    uint32_t ph = 1;
#pragma unroll 1
    for (int32_t i = first; i < total && ok; i += step) {
      int32_t l, c;
      tile_of(i, l, c);
      const int32_t row = lanes ? (PAIR ? 2 * l + rank : l) * kLaneRows
                                : c * TN + (PAIR ? rank * H::kCRows : 0);
#pragma unroll 1
      for (int32_t kb = kb_lo; kb < kb_hi; ++kb, ++n) {
        if (n >= S) ok = wait_warp(&empty[s], ph, a.status);
        if (!ok) break;
        if (leader) {
          unsigned char* dst = smem + s * H::kStage + (lanes ? 0 : H::kLBytes);
          if (!PAIR || rank == 0) mbar_arrive_expect_tx(&full[s], bytes);
          if constexpr (PAIR)
            tma_load_2d_pair(dst, lanes ? &tmL : &tmC, kb * kGroup, row, full0 + 8 * s, pol);
          else
            tma_load_2d(dst, lanes ? &tmL : &tmC, kb * kGroup, row, &full[s], pol);
        }
        __syncwarp();
        if (++s == S) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    // after a wait that gave up, the copies in flight still land here (a pair's are counted by
    // its even CTA, which waits for both below)
    if (!ok && rank == 0)
      for (int32_t u = max(0, n - S); u < n; ++u) mbar_drain(&full[u % S], (u / S) & 1);
  } else if (warp == EW + 1) {
    // ----------------------------------------------------------- products
    if (!PAIR || rank == 0) {
      constexpr uint32_t kIdesc = idesc_e4m3(PAIR ? 256 : 128, TN);
      const uint32_t base = warp_uniform(smem_u32(smem)), tm = warp_uniform(tmem);
      const bool leader = elect_one();
      bool ok = true;
      int32_t n = 0, s = 0;
      uint32_t ph = 0;
#pragma unroll 1
      for (int32_t i = first; i < total && ok; i += step) {
#pragma unroll 1
        for (int32_t kb = kb_lo; kb < kb_hi; ++kb, ++n) {
          const int b = n % NB;
          if (n >= NB) ok = wait_warp(&tempty[b], ((n / NB) - 1) & 1, a.status);
          ok = ok && wait_warp(&full[s], ph, a.status);
          if (!ok) break;
          tc_fence_after();
          const uint64_t dl = smem_desc(base + s * H::kStage, 16, 1024);
          const uint64_t dc = smem_desc(base + s * H::kStage + H::kLBytes, 16, 1024);
          if (leader) {
#pragma unroll
            for (int k = 0; k < kGroup / 32; ++k) {
              if constexpr (PAIR)
                mma8_ss_pair(tm + b * TN, smem_desc_at(dl, k * 32), smem_desc_at(dc, k * 32), kIdesc, k > 0);
              else
                mma8_ss(tm + b * TN, smem_desc_at(dl, k * 32), smem_desc_at(dc, k * 32), kIdesc, k > 0);
            }
            if constexpr (PAIR) {
              mma_commit_pair(&empty[s]);
              mma_commit_pair(&tfull[b]);
            } else {
              mma_commit(&empty[s]);
              mma_commit(&tfull[b]);
            }
          }
          __syncwarp();
          if (++s == S) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok && n > 0) mbar_drain(&tfull[(n - 1) % NB], ((n - 1) / NB) & 1);
    }
  } else {
    // ----------------------------------------------------------- epilogue
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const int32_t col = (warp >> 2) * CW;  // the warp's first column of a tile
    const int32_t my_lane = (warp & 3) * 32 + lane;
    const uint32_t tempty0 = PAIR ? peer_addr(smem_u32(tempty), 0) : 0;
    // Scales come by cp.async, P - 1 blocks ahead (over the end of a tile, too), into slots that
    // only this thread reads (lanes are rows of A) or only this warp.
    int32_t ahead_tile = first, ahead_kb = kb_lo, ahead_slot = 0;
    int32_t al = 0, ac = 0;
    tile_of(first, al, ac);
    const uint32_t ring_at = smem_u32(ring);
    auto ask = [&]() {
      if (ahead_tile < total) {
        if constexpr (SWAP) {
          const uint32_t to = ring_at + (uint32_t)((warp * P + ahead_slot) * (TN + 4)) * 4;
#pragma unroll
          for (int u = 0; u < TN; u += 32) {
            const int32_t t = u + lane, m = ac * TN + t;
            if (t < TN) cp_async4(to + t * 4, a.a_scale + ahead_kb * a.ldas + min(m, a.M - 1), m < a.M);
          }
          if (lane == 0) cp_async4(to + TN * 4, a.w_scale + ahead_kb * a.ldws + al, true);
        } else {
          const uint32_t to = ring_at + (uint32_t)(ahead_slot * 2 * EW * 32 + tid) * 4;
          const int32_t m = (PAIR ? 2 * al + rank : al) * kLaneRows + my_lane;
          const int32_t n = ac * TN + col;
          cp_async4(to, a.a_scale + ahead_kb * a.ldas + min(m, a.M - 1), m < a.M);
          cp_async4(to + EW * 32 * 4, a.w_scale + ahead_kb * a.ldws + min(n, a.N - 1) / kGroup, n < a.N);
        }
        if (++ahead_kb == kb_hi) {
          ahead_kb = kb_lo;
          ahead_tile += step;
          if (ahead_tile < total) tile_of(ahead_tile, al, ac);
        }
      }
      cp_async_commit();
      ahead_slot = ahead_slot + 1 == P ? 0 : ahead_slot + 1;
    };
#pragma unroll 1
    for (int u = 0; u < P - 1; ++u) ask();

    bool ok = true;
    int32_t n = 0, slot = 0;
#pragma unroll 1
    for (int32_t i = first; i < total && ok; i += step) {
      int32_t l, c;
      tile_of(i, l, c);
      float2 acc[CW / 2];
#pragma unroll
      for (int e = 0; e < CW / 2; ++e) acc[e] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int32_t kb = kb_lo; kb < kb_hi; ++kb, ++n) {
        if constexpr (SWAP) __syncwarp();  // (the slot asked for was read by every lane)
        ask();
        cp_async_wait<P - 1>();
        if constexpr (SWAP) __syncwarp();
        const int b = n % NB;
        ok = wait_warp(&tfull[b], (n / NB) & 1, a.status);
        if (!ok) break;
        tc_fence_after();
        const uint32_t from = tmem + lane_off + b * TN + col;
        if constexpr (SWAP) {
          const float* sc = ring + (warp * P + slot) * (TN + 4);
          const float2 ws = make_float2(sc[TN], sc[TN]), zero = make_float2(0.f, 0.f);
#pragma unroll
          for (int u = 0; u < TN; u += 16) {
            float v[16];
            tmem_ld16(from + u, v);
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const float4 s4 = *reinterpret_cast<const float4*>(sc + u + e);
              float2& x = acc[(u + e) / 2];
              float2& y = acc[(u + e) / 2 + 1];
              x = ffma2(make_float2(v[e], v[e + 1]), ffma2(make_float2(s4.x, s4.y), ws, zero), x);
              y = ffma2(make_float2(v[e + 2], v[e + 3]), ffma2(make_float2(s4.z, s4.w), ws, zero), y);
            }
          }
          tc_fence_before();
          __syncwarp();
          arrive_lane0(&tempty[b], lane);
        } else {
          const float* sc = ring + slot * 2 * EW * 32 + tid;
          const float f = sc[0] * sc[EW * 32];
          const float2 f2 = make_float2(f, f);
#pragma unroll
          for (int u = 0; u < CW; u += 32) {
            float v[32];
            tmem_ld32(from + u, v);
            if (u + 32 == CW) {
              tc_fence_before();
              __syncwarp();
              if constexpr (PAIR) {
                if (lane == 0) arrive_peer(tempty0 + 8 * b);
                __syncwarp();
              } else {
                arrive_lane0(&tempty[b], lane);
              }
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2)
              acc[(u + e) / 2] = ffma2(make_float2(v[e], v[e + 1]), f2, acc[(u + e) / 2]);
          }
        }
        slot = slot + 1 == P ? 0 : slot + 1;
      }
      if (!ok) break;
      // ---- the tile's way out
      if constexpr (SWAP) {
        if (L.splits > 1) {  // to the cluster's sums, below (one tile a CTA)
          float* mine = reinterpret_cast<float*>(smem) + my_lane;
#pragma unroll
          for (int e = 0; e < TN / 2; ++e) {
            mine[2 * e * kLaneRows] = acc[e].x;
            mine[(2 * e + 1) * kLaneRows] = acc[e].y;
          }
        } else {
          const int32_t nn = l * kLaneRows + my_lane;
          if (nn < a.N) {
#pragma unroll
            for (int e = 0; e < TN; ++e) {
              const int32_t m = c * TN + e;
              if (m < a.M) store_one(a, m, nn, e & 1 ? acc[e / 2].y : acc[e / 2].x);
            }
          }
        }
      } else {
        // a warp's 32 rows turned round in shared memory, 32 columns at a time: each store then
        // covers whole sectors of four rows
        float* st = staging + warp * 32 * kPitch;
        const int64_t row0 = (int64_t)(PAIR ? 2 * l + rank : l) * kLaneRows + (warp & 3) * 32;
        const int32_t r8 = lane >> 3, c4 = (lane & 7) * 4;
#pragma unroll
        for (int u = 0; u < CW; u += 32) {
          const int32_t n0 = c * TN + col + u + c4;
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<float4*>(st + lane * kPitch + e) =
                make_float4(acc[(u + e) / 2].x, acc[(u + e) / 2].y, acc[(u + e) / 2 + 1].x,
                            acc[(u + e) / 2 + 1].y);
          __syncwarp();
#pragma unroll 4
          for (int r = r8; r < 32; r += 4) {
            if (row0 + r >= a.M) break;
            const float4 x = *reinterpret_cast<const float4*>(st + r * kPitch + c4);
            if (L.vec && n0 + 4 <= a.N) {
              store_four(a, row0 + r, n0, x);
            } else {
              if (n0 < a.N) store_one(a, row0 + r, n0, x.x);
              if (n0 + 1 < a.N) store_one(a, row0 + r, n0 + 1, x.y);
              if (n0 + 2 < a.N) store_one(a, row0 + r, n0 + 2, x.z);
              if (n0 + 3 < a.N) store_one(a, row0 + r, n0 + 3, x.w);
            }
          }
        }
      }
    }
    cp_async_wait<0>();
  }

  // ---- teardown
  tc_fence_before();
  if (cluster > 1) cluster_sync_all();
  else __syncthreads();
  if constexpr (SWAP) {
    if (cluster > 1) {
      // every CTA of the cluster adds up the rows of A that are its rank's, in the ranks' order
      int32_t l, c;
      tile_of(first, l, c);
      const int32_t n = l * kLaneRows + tid, live = min(TN, a.M - c * TN);
      if (tid < kLaneRows && n < a.N) {
        const uint32_t at = smem_u32(smem) + tid * 4;
        for (int32_t t = rank; t < live; t += cluster) {
          float x = 0.f;
#pragma unroll 8
          for (int32_t r = 0; r < cluster; ++r) x += ld_peer(peer_addr(at + t * kLaneRows * 4, r));
          store_one(a, c * TN + t, n, x);
        }
      }
      cluster_sync_all();
    }
  }
  if (warp == EW + 1) {
    tc_fence_after();
    if constexpr (PAIR) tmem_dealloc_pair(tmem, NB * TN);
    else tmem_dealloc(tmem, NB * TN);
  }
}

// 2D view of e4m3 rows: {K bytes, rows}, box {128, rows of a copy}.
bool rows_map(CUtensorMap* map, const void* base, int32_t K, int64_t rows, int64_t ld, int32_t box_rows) {
  EncodeTiledFn fn = tensor_map_encoder();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {(cuuint32_t)kGroup, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int32_t ceil_div(int64_t a, int64_t b) { return (int32_t)((a + b - 1) / b); }

template <bool SWAP, bool PAIR, int TN>
cudaError_t launch(const ScaledMatmulArgs& a, cudaStream_t stream) {
  using H = Shape<SWAP, PAIR, TN>;
  CUtensorMap tl, tc;
  const bool maps =
      SWAP ? rows_map(&tl, a.w, a.K, a.N, a.ldw, kLaneRows) && rows_map(&tc, a.a, a.K, a.M, a.lda, H::kCRows)
           : rows_map(&tl, a.a, a.K, a.M, a.lda, kLaneRows) && rows_map(&tc, a.w, a.K, a.N, a.ldw, H::kCRows);
  if (!maps) return cudaErrorInvalidValue;
  auto kernel = scaled_matmul_kernel<SWAP, PAIR, TN>;
  const cudaError_t e = allow_smem(kernel, H::kSmem);
  if (e != cudaSuccess) return e;
  Launch L{};
  L.tiles_l = ceil_div(SWAP ? a.N : a.M, PAIR ? 2 * kLaneRows : kLaneRows);
  L.tiles_c = ceil_div(SWAP ? a.M : a.N, TN);
  L.splits = 1;
  const int64_t tiles = (int64_t)L.tiles_l * L.tiles_c;
  const int64_t places = (int64_t)H::kCtas * device_sm_count();
  if (SWAP) {
    const int64_t blocks = ceil_div(a.K, kGroup);
    L.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({8, places / tiles, blocks / 2}));
  }
  auto even = [](const void* p, int64_t ld, uintptr_t bytes) {
    return ld % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
  };
  L.vec = even(a.c, a.ldc, a.c_bf16 ? 8 : 16) && (a.add == nullptr || even(a.add, a.ldadd, 8));
  if (PAIR) {
    const int64_t pairs = std::min<int64_t>(tiles, places / 2);
    return launch_clusters(kernel, dim3((unsigned)(2 * pairs)), dim3(H::kThreads), H::kSmem, stream, true,
                           2, tl, tc, a, L);
  }
  if (L.splits > 1)
    return launch_clusters(kernel, dim3((unsigned)(tiles * L.splits)), dim3(H::kThreads), H::kSmem, stream,
                           true, L.splits, tl, tc, a, L);
  return launch_kernel(kernel, dim3((unsigned)std::min<int64_t>(tiles, places)), dim3(H::kThreads), H::kSmem,
                       stream, true, tl, tc, a, L);
}

}  // namespace

cudaError_t launch_scaled_matmul(const ScaledMatmulArgs& a, cudaStream_t stream) {
  if (a.M <= 16) return launch<true, false, 16>(a, stream);
  if (a.M <= 32) return launch<true, false, 32>(a, stream);
  if (a.M <= 64) return launch<true, false, 64>(a, stream);
  // cycles of a wave of tiles, about: what a block takes and a tile's way in and out
  const int64_t blocks = ceil_div(a.K, kGroup), sms = device_sm_count();
  auto cost = [&](int32_t rows, int32_t cols, int64_t places, int64_t block, int64_t rest) {
    const int64_t tiles = (int64_t)ceil_div(a.M, rows) * ceil_div(a.N, cols);
    return ceil_div(tiles, places) * (blocks * block + rest);
  };
  const int64_t pair = cost(256, 256, sms / 2, 530, 3000), wide = cost(128, 128, sms, 290, 2000);
  const int64_t narrow = std::min(cost(128, 64, 2 * sms, 300, 2000), cost(128, 64, sms, 170, 1500));
  if (pair <= wide && pair <= narrow) return launch<false, true, 256>(a, stream);
  return wide <= narrow ? launch<false, false, 128>(a, stream) : launch<false, false, 64>(a, stream);
}

}  // namespace ssd
