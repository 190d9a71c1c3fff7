// scaled_matmul.cu — products of e4m3 rows and weights with a float32 scale for every 128 entries
// of the inner length (include/ssd.h, ssd_scaled_matmul):
//   C[m][n] = sum_g sa[g][m] sw[g][n / 128] sum_{k in g} A[m][k] W[n][k]  (+ add[m][n]).
//
// The scales change along the inner length, so no accumulator of the tensor cores can hold the sum
// over g: a block of 128 (four tcgen05.mma of kind::f8f6f4) goes into a TMEM buffer of its own, and
// the epilogue's warps add it, times its scales, to sums in their registers while the tensor
// cores work on the next blocks in other buffers.
//
// More than 64 rows: the rows of A are the 128 lanes of a tile (the scales of a block are then one
// number a thread), 128 rows of W its columns; or a CTA pair (cta_group::2) has 128 lanes each and 128
// or 256 columns.  Up to 64 rows, mostly: the other way round (scaled_matmul_few_kernel).
//
// 17408 x 12288 x 4096 (1752 GFLOP) 800 us in a graph, 2190 TFLOP/s: 560 ns a block of 256 x 256 of
// a pair, of which the products are 340; two TMEM buffers' round trips bound it (without the reads of TMEM
// 563 us).  1024 x 4096 x 4096 with a sum 25.0 us; 16 x 65536 x 4096 (273 MB) 43 us, the copy rate.
//
// Barriers count units of U blocks: a wait that is satisfied already costs a warp about 100
// cycles, a commit of products as much.
#include <algorithm>

#include "kernels.cuh"

namespace ssd {

namespace {

constexpr int kGroup = 128;  // entries of a scale, bytes of a stage's rows
constexpr int kLaneRows = 128;
constexpr int kPiece = 32;   // columns staged at a time
constexpr int kPitch = 36;   // floats of a row of them (rows start four banks apart)
constexpr int kOddPitch = 33;  // the same where C's rows may begin anywhere
constexpr int kRaster = 8;   // tiles of lanes that share the columns' tiles in L2
constexpr int kAhead = 4;    // blocks whose scales are asked for together
constexpr int kMaxSplits = 8;
constexpr int64_t kOftenBytes = 32 << 20;  // most of A to hold in L2, about a quarter

template <bool PAIR, int TN, int U>
struct Shape {
  static constexpr int EW = 8;                            // epilogue warps
  static constexpr int CW = TN / 2;                       // columns of one
  static constexpr int CR = 64;                           // columns read from TMEM at a time
  // (a pair's epilogue takes registers from the others, warpgroup by warpgroup)
  static constexpr int kThreads = (EW + (PAIR ? 4 : 3)) * 32;
  static constexpr int kCols = 2 * U * TN;                // two units in TMEM
  static constexpr int kCRows = PAIR ? TN / 2 : TN;       // of a CTA's copy
  static constexpr int kCBytes = kCRows * kGroup;
  static constexpr int kStaging = EW * 32 * kPitch * 4;
  static constexpr int kScales = 2 * kAhead * 2 * EW * 32 * 4;
  static constexpr int kFixed = 1024 + kStaging + kScales;
  static constexpr int kABytes = kLaneRows * kGroup;
  static constexpr int kStage = U * (kABytes + kCBytes);
  static constexpr int S = (224 * 1024 - kFixed) / kStage;
  static constexpr int kSmem = kFixed + S * kStage;
  static_assert(CW % CR == 0 && kCols <= 512 && kAhead % U == 0 && S >= 2, "");
};

struct Launch {
  int32_t tiles_l, tiles_c;
  int32_t often;  // A stays in L2
  int32_t even;  // (C's rows begin anywhere) add's entries lie on four entries where C's do
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
// The arrival of the warp's lane 0 at a barrier of the cluster.  Relaxed: what it hands over is tensor
// memory, ordered by tcgen05.fence; a release would wait for the lanes' own copies of scales
// (17408 x 12288 x 4096: 1750 us instead of 850).
__device__ __forceinline__ void arrive_peer_lane0(uint32_t bar, int lane) {
  asm volatile(
      "{\n .reg .pred p;\n setp.eq.u32 p, %1, 0;\n"
      " @p mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n}" ::"r"(bar),
      "r"(lane)
      : "memory");
}
__device__ __forceinline__ float ld_peer(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
// fp32 sums of e4m3 products, M x N, both operands K-major.
__host__ __device__ constexpr uint32_t idesc_e4m3(int m, int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// mbar_drain(), inlined: a call has no place beside setmaxnreg.  Called by whole warps, whose lanes may
// leave the loop one by one: together again behind it, as the barriers that follow want them.
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) {
#pragma unroll 1
  for (int i = 0; i < (1 << 14) && !mbar_try_wait(bar, parity); ++i) __nanosleep(256);
  __syncwarp();
}
// The same of what is on its way in any case: without a sleep at first.
__device__ __forceinline__ void land(uint64_t* bar, uint32_t parity) {
  bool here = false;
#pragma unroll 1
  for (int i = 0; i < 1024 && !here; ++i) here = __all_sync(0xffffffffu, mbar_try_wait(bar, parity));
  if (!here) drain(bar, parity);
}

// A warp's kPiece columns from n0 on of `rows` rows of C from m0 on: staged with kPitch floats a row, each
// store whole sectors of a few rows: 16 bytes a lane, all asked for (of add) before the first is used;
// columns up to N that end inside of them an element a lane.
__device__ __forceinline__ void write_rows(const ScaledMatmulArgs& a, const float* st, int lane,
                                           int64_t m0, int32_t rows, int32_t n0) {
  const uint16_t* add = static_cast<const uint16_t*>(a.add);
  const bool vec = n0 + kPiece <= a.N;
  if (vec && a.c_bf16) {
    constexpr int kL = kPiece / 8, kRows = 32 / kL;  // lanes of a row, rows of a pass
    const int32_t r0 = lane / kL, c = lane % kL * 8, n = n0 + c;
    uint4 w[kL];
#pragma unroll
    for (int i = 0; i < kL; ++i) {
      w[i] = make_uint4(0, 0, 0, 0);
      if (add != nullptr && r0 + i * kRows < rows)
        w[i] = *reinterpret_cast<const uint4*>(add + (m0 + r0 + i * kRows) * a.ldadd + n);
    }
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.c) + (m0 + r0) * a.ldc + n;
#pragma unroll
    for (int i = 0; i < kL; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(st + (r0 + i * kRows) * kPitch + c);
      const float4 y = *reinterpret_cast<const float4*>(st + (r0 + i * kRows) * kPitch + c + 4);
      const uint32_t* v = &w[i].x;
      const uint4 z = make_uint4(
          pack_bf16x2(x.x + __uint_as_float(v[0] << 16), x.y + __uint_as_float(v[0] & 0xffff0000u)),
          pack_bf16x2(x.z + __uint_as_float(v[1] << 16), x.w + __uint_as_float(v[1] & 0xffff0000u)),
          pack_bf16x2(y.x + __uint_as_float(v[2] << 16), y.y + __uint_as_float(v[2] & 0xffff0000u)),
          pack_bf16x2(y.z + __uint_as_float(v[3] << 16), y.w + __uint_as_float(v[3] & 0xffff0000u)));
      if (r0 + i * kRows < rows) *reinterpret_cast<uint4*>(out) = z;
      out += kRows * a.ldc;
    }
    return;
  } else if (vec) {
    constexpr int kL = kPiece / 4, kRows = 32 / kL;
    const int32_t r0 = lane / kL, c = lane % kL * 4, n = n0 + c;
    uint2 w[kL];
#pragma unroll
    for (int i = 0; i < kL; ++i) {
      w[i] = make_uint2(0, 0);
      if (add != nullptr && r0 + i * kRows < rows)
        w[i] = *reinterpret_cast<const uint2*>(add + (m0 + r0 + i * kRows) * a.ldadd + n);
    }
    float* out = static_cast<float*>(a.c) + (m0 + r0) * a.ldc + n;
#pragma unroll
    for (int i = 0; i < kL; ++i) {
      float4 x = *reinterpret_cast<const float4*>(st + (r0 + i * kRows) * kPitch + c);
      x.x += __uint_as_float(w[i].x << 16);
      x.y += __uint_as_float(w[i].x & 0xffff0000u);
      x.z += __uint_as_float(w[i].y << 16);
      x.w += __uint_as_float(w[i].y & 0xffff0000u);
      if (r0 + i * kRows < rows) *reinterpret_cast<float4*>(out) = x;
      out += kRows * a.ldc;
    }
    return;
  }
  // an element each, a lane's column of eight rows together
  const int32_t n = n0 + lane;
  if (n >= a.N) return;
  const int64_t at = m0 * a.ldc + n;
  const uint16_t* from = add + m0 * a.ldadd + n;
#pragma unroll 1
  for (int32_t r = 0; r < rows; r += 8) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = st[(r + i) * kPitch + lane];
      if (add != nullptr && r + i < rows) x[i] += __uint_as_float((uint32_t)from[(r + i) * a.ldadd] << 16);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (r + i >= rows || !dbg_in(at + (r + i) * a.ldc, (a.M - 1) * a.ldc + a.N, a.status)) continue;
      if (a.c_bf16) static_cast<__nv_bfloat16*>(a.c)[at + (r + i) * a.ldc] = __float2bfloat16_rn(x[i]);
      else static_cast<float*>(a.c)[at + (r + i) * a.ldc] = x[i];
    }
  }
}

// The same of rows that begin anywhere: eight lanes a row, four entries a lane from where C is aligned
// for them (8 or 16 bytes), and the four entries that those leave out at both ends one by one (5848 x
// 58870 x 172 with a sum, to bf16, rows an odd number of entries apart: an entry a lane 1383 us, this
// 782; aligned 519; to float32 without a sum 891, 551 and 485).
template <typename T>
__device__ __forceinline__ void write_rows_any(const ScaledMatmulArgs& a, const float* st, int lane,
                                               int64_t m0, int32_t rows, int32_t n0, bool even) {
  constexpr int kTogether = 4;  // passes whose additions are asked for together
  const int32_t i = lane & 7, r0 = lane >> 3;
  const uint16_t* add = static_cast<const uint16_t*>(a.add);
  if (add != nullptr) add += (m0 + r0) * a.ldadd + n0;
  T* out = static_cast<T*>(a.c) + (m0 + r0) * a.ldc + n0;
  st += r0 * kOddPitch;
  auto value = [](uint32_t x) { return __uint_as_float(x << 16); };
  auto put = [](T* p, float x) {
    if constexpr (sizeof(T) == 2) *p = __float2bfloat16_rn(x);
    else *p = x;
  };
  if (n0 + kPiece > a.N) {
#pragma unroll 1
    for (int32_t r = r0; r < rows; r += 4, out += 4 * a.ldc, st += 4 * kOddPitch) {
#pragma unroll 1
      for (int32_t e = i; n0 + e < a.N; e += 8) put(out + e, st[e] + (add != nullptr ? value(add[e]) : 0.f));
      if (add != nullptr) add += 4 * a.ldadd;
    }
    return;
  }
#pragma unroll 1
  for (int32_t r = r0; r < r0 + 32; r += 4 * kTogether) {
    uint2 w[kTogether];
    uint32_t we[kTogether];
    int32_t first[kTogether], edge[kTogether];
    bool live[kTogether];
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      live[u] = r + 4 * u < rows && dbg_in((m0 + r + 4 * u) * a.ldc + n0, (a.M - 1) * a.ldc + a.N, a.status);
      const int32_t s = (int32_t)(reinterpret_cast<uintptr_t>(out + 4 * u * a.ldc) / sizeof(T)) & 3;
      first[u] = 4 * i - s;
      edge[u] = s == 0 || i > 3 ? -1 : i < 4 - s ? i : 28 + i;
      w[u] = make_uint2(0, 0);
      we[u] = 0;
      if (add != nullptr && live[u]) {
        const uint16_t* from = add + 4 * u * a.ldadd;
        if (first[u] >= 0) {
          const uint16_t* f = from + first[u];
          if (even) w[u] = *reinterpret_cast<const uint2*>(f);
          else w[u] = make_uint2(f[0] | (uint32_t)f[1] << 16, f[2] | (uint32_t)f[3] << 16);
        }
        if (edge[u] >= 0) we[u] = from[edge[u]];
      }
    }
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      const float* from = st + 4 * u * kOddPitch;
      const float* f = from + max(first[u], 0);
      const float x[4] = {f[0] + value(w[u].x), f[1] + __uint_as_float(w[u].x & 0xffff0000u),
                          f[2] + value(w[u].y), f[3] + __uint_as_float(w[u].y & 0xffff0000u)};
      const float y = from[max(edge[u], 0)] + value(we[u]);
      T* to = out + 4 * u * a.ldc;
      if (!live[u]) continue;
      if (first[u] >= 0) {
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<uint2*>(to + first[u]) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
        else
          *reinterpret_cast<float4*>(to + first[u]) = make_float4(x[0], x[1], x[2], x[3]);
      }
      if (edge[u] >= 0) put(to + edge[u], y);
    }
    out += 4 * kTogether * a.ldc;
    st += 4 * kTogether * kOddPitch;
    if (add != nullptr) add += 4 * kTogether * a.ldadd;
  }
}

// The same of 64 columns staged as bf16 (kOddPitch words a row): eight entries a lane, 16 bytes (without
// a sum 904 us, 345; aligned 207).
__device__ __forceinline__ void write_rows_any16(const ScaledMatmulArgs& a, const uint32_t* st, int lane,
                                                 int64_t m0, int32_t rows, int32_t n0) {
  const int32_t i = lane & 7, r0 = lane >> 3;
  uint16_t* out = static_cast<uint16_t*>(a.c) + (m0 + r0) * a.ldc + n0;
  st += r0 * kOddPitch;
  auto entry = [&](int32_t e) { return (uint16_t)(st[e >> 1] >> (16 * (e & 1))); };
  const bool whole = n0 + 64 <= a.N;
#pragma unroll 2
  for (int32_t r = r0; r < rows; r += 4, out += 4 * a.ldc, st += 4 * kOddPitch) {
    if (!dbg_in((m0 + r) * a.ldc + n0, (a.M - 1) * a.ldc + a.N, a.status)) continue;
    if (!whole) {
#pragma unroll 1
      for (int32_t e = i; n0 + e < a.N; e += 8) out[e] = entry(e);
      continue;
    }
    const int32_t s = (int32_t)(reinterpret_cast<uintptr_t>(out) / 2) & 7, first = 8 * i - s;
    const uint32_t* from = st + (max(first, 0) >> 1);
    uint32_t w[5], v[4];
#pragma unroll
    for (int k = 0; k < 5; ++k) w[k] = from[k];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __funnelshift_r(w[k], w[k + 1], 16 * (s & 1));
    if (first >= 0) *reinterpret_cast<uint4*>(out + first) = make_uint4(v[0], v[1], v[2], v[3]);
    const int32_t edge = i < 8 - s ? i : 56 + i;
    if (s != 0) out[edge] = entry(edge);
  }
}

__device__ __forceinline__ float added(const ScaledMatmulArgs& a, int64_t m, int32_t n) {
  if (a.add == nullptr) return 0.f;
  return __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.add)[m * a.ldadd + n] << 16);
}
__device__ __forceinline__ void store_one(const ScaledMatmulArgs& a, int64_t m, int32_t n, float x) {
  if (!dbg_in(m * a.ldc + n, (a.M - 1) * a.ldc + a.N, a.status)) return;
  if (a.c_bf16) static_cast<__nv_bfloat16*>(a.c)[m * a.ldc + n] = __float2bfloat16_rn(x);
  else static_cast<float*>(a.c)[m * a.ldc + n] = x;
}

// Registers of a pair's CTA: 384 threads of 168 at launch, then 256 of 216 and 128 of 72.
constexpr int kRegsEpilogue = 216, kRegsOther = 72;

// kVec: C may be written, and add read, 16 bytes of C at a time.
template <bool PAIR, int TN, int U, bool kVec>
__global__ void __launch_bounds__(Shape<PAIR, TN, U>::kThreads, 1)
scaled_matmul_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                     ScaledMatmulArgs a, Launch L) {
  using H = Shape<PAIR, TN, U>;
  constexpr int EW = H::EW, CW = H::CW, CR = H::CR;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  // a stage: U blocks of A [128][128], U blocks of W [kCRows][128]
  constexpr int S = H::S, a_bytes = H::kABytes, stage_bytes = H::kStage;
  float* staging = reinterpret_cast<float*>(smem + S * stage_bytes);
  float* scales = staging + H::kStaging / 4;
  __shared__ uint64_t full[S], empty[S], tfull[2], tempty[2];
  __shared__ uint32_t tmem_slot;
  pdl_wait();

  const int32_t tid = threadIdx.x, lane = tid & 31, warp = (int32_t)warp_uniform(tid >> 5);
  const int32_t rank = PAIR ? (int32_t)(blockIdx.x & 1) : 0;
  const int32_t first = PAIR ? blockIdx.x >> 1 : blockIdx.x, step = PAIR ? gridDim.x >> 1 : gridDim.x;
  const int32_t total = L.tiles_l * L.tiles_c;
  const int32_t blocks = (a.K + kGroup - 1) / kGroup;
  if (warp == EW && lane < 2) prefetch_tensormap(lane == 0 ? &tmA : &tmW);
  if (tid == EW * 32) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 2);  // the two producers
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&tfull[i], 1);
      mbar_init(&tempty[i], PAIR ? 2 * EW : EW);
    }
    fence_barrier_init();
  }
  if constexpr (PAIR) {
    __syncwarp();
    cluster_sync_all();  // (the peer's barriers too are initialised)
  } else {
    __syncthreads();
  }
  // (the copies begin without tensor memory)
  uint32_t tmem = 0;
  if (warp <= EW + 1 && warp != EW) {
    if (warp == EW + 1) {
      if constexpr (PAIR) {
        tmem_alloc_pair(&tmem_slot, H::kCols);
        tmem_relinquish_pair();
      } else {
        tmem_alloc(&tmem_slot, H::kCols);
        tmem_relinquish();
      }
      tc_fence_before();
    }
    asm volatile("bar.sync 1, %0;" ::"n"((EW + 1) * 32) : "memory");
    tc_fence_after();
    tmem = tmem_slot;
  }

  // Tile i: which rows of A and of W.
  auto tile_of = [&](int32_t i, int32_t& l, int32_t& c) {
    const int32_t per = kRaster * L.tiles_c, g = i / per, r = i - g * per;
    const int32_t n = min(kRaster, L.tiles_l - g * kRaster);
    c = r / n;
    l = g * kRaster + r - c * n;
  };

  if (warp >= EW) {
    if constexpr (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
  }
  if (warp == EW || warp == EW + 2) {
    // ---------------------------------------------------------- producers
    const bool of_a = warp == EW, leader = elect_one();
    const uint64_t pol = of_a && L.often ? policy_evict_last() : policy_evict_normal();
    const int32_t block_bytes = of_a ? a_bytes : H::kCBytes, at = of_a ? 0 : U * a_bytes;
    const CUtensorMap* map = of_a ? &tmA : &tmW;
    const uint32_t full0 = PAIR ? peer_addr(smem_u32(full), 0) : 0;
    bool ok = true;
    int32_t n = 0, s = 0;
    uint32_t ph = 1;
#pragma unroll 1
    for (int32_t i = first; i < total && ok; i += step) {
      int32_t l, c;
      tile_of(i, l, c);
      const int32_t row = of_a ? (PAIR ? 2 * l + rank : l) * kLaneRows
                               : c * TN + (PAIR ? rank * H::kCRows : 0);
#pragma unroll 1
      for (int32_t kb = 0; kb < blocks; kb += U, ++n) {
        if (n >= S) ok = wait_warp(&empty[s], ph, a.status);
        if (!ok) break;
        if (leader) {
          unsigned char* dst = smem + s * stage_bytes + at;
          const int32_t un = min(U, blocks - kb);
          if (!PAIR || rank == 0) mbar_arrive_expect_tx(&full[s], (PAIR ? 2 : 1) * un * block_bytes);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (u >= un) break;
            if constexpr (PAIR)
              tma_load_2d_pair(dst + u * block_bytes, map, (kb + u) * kGroup, row, full0 + 8 * s, pol);
            else
              tma_load_2d(dst + u * block_bytes, map, (kb + u) * kGroup, row, &full[s], pol);
          }
        }
        __syncwarp();
        if (++s == S) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    // after a wait that gave up, the copies in flight still land here (a pair's are counted by
    // its even CTA, for which the other waits below)
    if (!ok && rank == 0)
      for (int32_t u = max(0, n - S); u < n; ++u) drain(&full[u % S], (u / S) & 1);
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
        for (int32_t kb = 0; kb < blocks; kb += U, ++n) {
          const int b = n & 1;
          ok = wait_warp(&full[s], ph, a.status);
          // (last: what these products mostly wait for)
          if (ok && n >= 2) ok = wait_warp(&tempty[b], ((n >> 1) - 1) & 1, a.status);
          if (!ok) break;
          tc_fence_after();
          const uint64_t da = smem_desc(base + s * stage_bytes, 16, 1024);
          const uint64_t dw = smem_desc(base + s * stage_bytes + U * a_bytes, 16, 1024);
          if (leader) {
            // (blocks in turn: a product that adds to the one before it waits for it, 110 cycles
            // of which 32 columns are work)
#pragma unroll
            for (int k = 0; k < kGroup / 32; ++k) {
#pragma unroll
              for (int u = 0; u < U; ++u) {
                if (U > 1 && kb + u >= blocks) break;
                const uint64_t x = smem_desc_at(da, u * a_bytes + k * 32);
                const uint64_t y = smem_desc_at(dw, u * H::kCBytes + k * 32);
                if constexpr (PAIR) mma8_ss_pair(tm + (b * U + u) * TN, x, y, kIdesc, k > 0);
                else mma8_ss(tm + (b * U + u) * TN, x, y, kIdesc, k > 0);
              }
            }
            if constexpr (PAIR) {
              mma_commit_pair(&tfull[b]);
              mma_commit_pair(&empty[s]);
            } else {
              mma_commit(&tfull[b]);
              mma_commit(&empty[s]);
            }
          }
          __syncwarp();
          if (++s == S) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok && n > 0) drain(&tfull[(n - 1) & 1], ((n - 1) >> 1) & 1);
    }
  } else if (warp < EW) {
    // ----------------------------------------------------------- epilogue
    if constexpr (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpilogue));
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const int32_t col = (warp >> 2) * CW;  // the warp's first column of a tile
    const uint32_t tempty0 = PAIR ? peer_addr(smem_u32(tempty), 0) : 0;
    // Scales come by cp.async, kAhead blocks together and as many ahead (over the end of a tile,
    // too), into slots that only this thread reads: [2][kAhead][A's, W's][thread].
    constexpr int kSlot = 2 * EW * 32;
    const uint32_t scales_at = smem_u32(scales + tid);
    int32_t next_tile = first, next_kb = blocks;
    uint32_t next_half = 0;
    const float* next_a = nullptr;
    const float* next_w = nullptr;
    bool live_a = false, live_w = false;
    auto ask = [&]() {
      if (next_kb >= blocks && next_tile < total) {
        int32_t l, c;
        tile_of(next_tile, l, c);
        next_tile += step;
        next_kb = 0;
        const int32_t m = (PAIR ? 2 * l + rank : l) * kLaneRows + (warp & 3) * 32 + lane, n = c * TN + col;
        live_a = m < a.M;
        live_w = n < a.N;
        next_a = a.a_scale + min(m, a.M - 1);
        next_w = a.w_scale + min(n, a.N - 1) / kGroup;
      }
      const uint32_t to = scales_at + next_half * (kAhead * kSlot * 4);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (next_kb + u >= blocks) break;
        cp_async4(to + u * kSlot * 4, next_a, live_a);
        cp_async4(to + u * kSlot * 4 + EW * 32 * 4, next_w, live_w);
        next_a += a.ldas;
        next_w += a.ldws;
      }
      next_kb += kAhead;
      next_half ^= 1u;
      cp_async_commit();
    };
    ask();

    bool ok = true;
    int32_t n = 0;
    uint32_t half = 0;
#pragma unroll 1
    for (int32_t i = first; i < total && ok; i += step) {
      int32_t l, c;
      tile_of(i, l, c);
      const int64_t row0 = (int64_t)(PAIR ? 2 * l + rank : l) * kLaneRows + (warp & 3) * 32;
      const bool have_rows = row0 < a.M;
      if (a.add != nullptr && row0 + lane < a.M) {
        // what is added, on its way to L2 meanwhile (read at the end, it comes from there in a third of
        // the time)
        const uint16_t* from = static_cast<const uint16_t*>(a.add) + (row0 + lane) * a.ldadd + c * TN + col;
#pragma unroll 1
        for (int x = 0; x < CW && c * TN + col + x < a.N; x += 64)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(from + x));
      }
      float2 acc[CW / 2];
#pragma unroll
      for (int e = 0; e < CW / 2; ++e) acc[e] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int32_t kb = 0; kb < blocks; kb += U, ++n) {
        if (kb % kAhead == 0) {
          cp_async_wait<0>();
          half = next_half ^ 1u;
          ask();
        }
        const float* sc = scales + tid + (half * kAhead + kb % kAhead) * kSlot;
        const int b = n & 1;
        ok = wait_warp(&tfull[b], (n >> 1) & 1, a.status);
        if (!ok) break;
        tc_fence_after();
        const uint32_t from = tmem + lane_off + b * U * TN + col;
        auto done = [&]() {
          tc_fence_before();
          __syncwarp();
          if constexpr (PAIR) arrive_peer_lane0(tempty0 + 8 * b, lane);
          else arrive_lane0(&tempty[b], lane);
        };
        if (!have_rows) {
          done();
          continue;
        }
        // A read of TMEM takes 200 cycles whatever its width (to 64 columns): the widest that the
        // registers hold, and two warps on a scheduler.  (Of blocks behind the last, whatever the
        // buffer holds: not added.)
        constexpr int kPer = CW / CR;
#pragma unroll
        for (int q = 0; q < U * kPer; ++q) {
          const int u = q / kPer, x = q % kPer * CR;
          uint32_t w[CR];
          tmem_ask(from + u * TN + x, w);
          const float f = sc[u * kSlot] * sc[u * kSlot + EW * 32];
          const float2 f2 = make_float2(f, f);
          tmem_have(w);
          if (q + 1 == U * kPer) done();
          if (U > 1 && kb + u >= blocks) continue;
#pragma unroll
          for (int e = 0; e < CR; e += 2)
            acc[(x + e) / 2] =
                ffma2(make_float2(__uint_as_float(w[e]), __uint_as_float(w[e + 1])), f2, acc[(x + e) / 2]);
        }
      }
      if (!ok) break;
      // ---- the tile's way out: a warp's 32 rows turned round in shared memory, kPiece columns at a time
      if (have_rows) {
        float* st = staging + warp * 32 * kPitch;
        const int32_t rows = (int32_t)min((int64_t)32, a.M - row0);
        if (a.c_bf16 && a.add == nullptr) {
          // rounded first: half of what shared memory carries (as float32 a tile took 9300 cycles)
          unsigned char* st8 = reinterpret_cast<unsigned char*>(st);
          constexpr int kBytes = 144;  // of a staged row of 64
          const int32_t r0 = lane >> 3, c8 = (lane & 7) * 8;
#pragma unroll 1
          for (int x = 0; x < CW && c * TN + col + x < a.N; x += 64) {
            __syncwarp();
#pragma unroll
            for (int y = 0; y < CW; y += 64) {
              if (x != y) continue;
              if constexpr (kVec) {
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                  const float2* v = acc + y / 2 + e;
                  *reinterpret_cast<uint4*>(st8 + lane * kBytes + e * 4) =
                      make_uint4(pack_bf16x2(v[0].x, v[0].y), pack_bf16x2(v[1].x, v[1].y),
                                 pack_bf16x2(v[2].x, v[2].y), pack_bf16x2(v[3].x, v[3].y));
                }
              } else {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  reinterpret_cast<uint32_t*>(st8)[lane * kOddPitch + e] =
                      pack_bf16x2(acc[y / 2 + e].x, acc[y / 2 + e].y);
              }
            }
            __syncwarp();
            if constexpr (!kVec) {
              write_rows_any16(a, reinterpret_cast<uint32_t*>(st8), lane, row0, rows, c * TN + col + x);
              continue;
            }
            const int32_t n = c * TN + col + x + c8;
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.c) + (row0 + r0) * a.ldc + n;
            const unsigned char* from = st8 + r0 * kBytes + c8 * 2;
            if (n + 8 <= a.N) {
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const uint4 v = *reinterpret_cast<const uint4*>(from + j * 4 * kBytes);
                if (r0 + j * 4 < rows) *reinterpret_cast<uint4*>(out) = v;
                out += 4 * a.ldc;
              }
            } else {
#pragma unroll 1
              for (int32_t r = r0; r < rows; r += 4, out += 4 * a.ldc, from += 4 * kBytes)
                for (int32_t e = 0; n + e < a.N; ++e)
                  out[e] = reinterpret_cast<const __nv_bfloat16*>(from)[e];
            }
          }
          continue;
        }
        // (one copy of the code for all pieces: cold, it takes longer to fetch than to run)
#pragma unroll 1
        for (int x = 0; x < CW && c * TN + col + x < a.N; x += kPiece) {
          __syncwarp();
#pragma unroll
          for (int y = 0; y < CW; y += kPiece) {
            if (x != y) continue;
            if constexpr (kVec) {
#pragma unroll
              for (int e = 0; e < kPiece; e += 4)
                *reinterpret_cast<float4*>(st + lane * kPitch + e) =
                    make_float4(acc[(y + e) / 2].x, acc[(y + e) / 2].y, acc[(y + e) / 2 + 1].x,
                                acc[(y + e) / 2 + 1].y);
            } else {
#pragma unroll
              for (int e = 0; e < kPiece; e += 2) {
                st[lane * kOddPitch + e] = acc[(y + e) / 2].x;
                st[lane * kOddPitch + e + 1] = acc[(y + e) / 2].y;
              }
            }
          }
          __syncwarp();
          const int32_t n = c * TN + col + x;
          if constexpr (kVec) write_rows(a, st, lane, row0, rows, n);
          else if (a.c_bf16) write_rows_any<__nv_bfloat16>(a, st, lane, row0, rows, n, L.even);
          else write_rows_any<float>(a, st, lane, row0, rows, n, L.even);
        }
      }
    }
    cp_async_wait<0>();
  }

  // ---- teardown
  tc_fence_before();
  __syncwarp();  // (cluster barriers take whole warps)
  if constexpr (PAIR) cluster_sync_all();
  else __syncthreads();
  if (warp == EW + 1) {
    tc_fence_after();
    if constexpr (PAIR) tmem_dealloc_pair(tmem, H::kCols);
    else tmem_dealloc(tmem, H::kCols);
  }
}

// ------------------------------------------------------------------ few rows
// Up to 64 rows of A as the TN columns of tiles whose lanes are 128 rows of W: the products then read
// W from shared memory once (with A on the lanes, a tile of 64 rows of W reads 128 of A with it,
// most of them empty: 16 x 65536 x 4096 56 us, here 43).  W's way in bounds it.  Where the tiles
// alone would leave SMs idle, the blocks of a tile are cut over a cluster of up to eight CTAs, which
// add their sums up through distributed shared memory in the order of their ranks (with each other's word
// that no wait gave up, 0.15 us: 1 x 4096 x 4096 6.55 us without it, 6.70).  Two CTAs an SM hold the 64-column
// kernel to 96 registers, which spills nothing.
template <int TN, int U>
struct Few {
  static constexpr int EW = TN < 64 ? 4 : 8;          // epilogue warps,
  static constexpr int CW = TN / (EW / 4);            // rows of A of one
  static constexpr int kThreads = (EW + 2) * 32;      // and copies, products
  static constexpr int kCols = 2 * U * TN;            // two units in TMEM
  static constexpr int kCBytes = TN * kGroup, kWBytes = kLaneRows * kGroup;
  static constexpr int kStage = U * (kWBytes + kCBytes);
  static constexpr int kSlot = CW + 4;                // scales of a warp's block: A's, W's
  static constexpr int kScales = 2 * kAhead * EW * kSlot * 4;
  static constexpr int kFixed = 1024 + kScales;
  static constexpr int S = (112 * 1024 - kFixed) / kStage;
  static constexpr int kSmem = kFixed + S * kStage;
  static_assert(S >= 2 && S * kStage >= TN * kLaneRows * 4, "a CTA's sums fit where its stages were");
};

struct FewLaunch {
  int32_t tiles_w, total, splits;
  uint32_t max_polls, shortfall;  // (ssd_set_wait_limit, ssd_set_barrier_shortfall)
};

template <int TN, int U>
__global__ void __launch_bounds__(Few<TN, U>::kThreads, 2)
scaled_matmul_few_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                         ScaledMatmulArgs a, FewLaunch L) {
  using H = Few<TN, U>;
  constexpr int S = H::S, B = 2, EW = H::EW, CW = H::CW;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* scales = reinterpret_cast<float*>(smem + S * H::kStage);
  __shared__ uint64_t full[S], empty[S], tfull[B], tempty[B];
  __shared__ uint32_t tmem_slot, gave_up;  // (a warp of the epilogue: its sums are not known)
  pdl_wait();

  const int32_t tiles_w = L.tiles_w, total = L.total, splits = L.splits;
  const int32_t tid = threadIdx.x, lane = tid & 31, warp = (int32_t)warp_uniform(tid >> 5);
  const int32_t rank = splits > 1 ? (int32_t)(blockIdx.x % splits) : 0;
  const int32_t first = blockIdx.x / splits, step = gridDim.x / splits;
  const int32_t blocks = (a.K + kGroup - 1) / kGroup;
  const int32_t kb_lo = (int32_t)((int64_t)blocks * rank / splits);
  const int32_t kb_hi = (int32_t)((int64_t)blocks * (rank + 1) / splits);
  if (warp == EW && lane < 2) prefetch_tensormap(lane == 0 ? &tmA : &tmW);
  if (tid == EW * 32) {
    gave_up = 0;
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < B; ++i) {
      mbar_init(&tfull[i], 1 + L.shortfall);
      mbar_init(&tempty[i], EW);
    }
    fence_barrier_init();
  }
  __syncwarp();
  uint32_t tmem = 0;
  if (warp != EW) {  // (the copies begin without the others)
    if (warp == EW + 1) {
      tmem_alloc(&tmem_slot, H::kCols);
      tmem_relinquish();
      tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    tmem = tmem_slot;
  }
  // Tile i: rows (i % tiles_w) * 128 of W and (i / tiles_w) * TN of A.
  if (warp == EW) {
    // ------------------------------------------------------------- copies
    const bool leader = elect_one();
    const uint64_t once = policy_evict_first(), often = policy_evict_last();
    bool ok = true, begun = false;
    int32_t n = 0, s = 0;
    uint32_t ph = 1;
#pragma unroll 1
    for (int32_t i = first; i < total && ok; i += step) {
      const int32_t c = i / tiles_w, row = (i - c * tiles_w) * kLaneRows;
#pragma unroll 1
      for (int32_t kb = kb_lo; kb < kb_hi; kb += U, ++n) {
        if (n == S) {
          __syncthreads();
          begun = true;
        }
        if (n >= S) ok = wait_warp(&empty[s], ph, a.status, L.max_polls);
        if (!ok) break;
        if (leader) {
          unsigned char* dst = smem + s * H::kStage;
          const int32_t un = min(U, kb_hi - kb);
          mbar_arrive_expect_tx(&full[s], un * (H::kWBytes + H::kCBytes));
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (u >= un) break;
            tma_load_2d(dst + u * H::kWBytes, &tmW, (kb + u) * kGroup, row, &full[s], once);
            tma_load_2d(dst + U * H::kWBytes + u * H::kCBytes, &tmA, (kb + u) * kGroup, c * TN, &full[s],
                        often);
          }
        }
        __syncwarp();
        if (++s == S) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    if (!begun) __syncthreads();
    // the last copies land here, also where nobody waits for them any more
    for (int32_t u = max(0, n - S); u < n; ++u) land(&full[u % S], (u / S) & 1);
  } else if (warp == EW + 1) {
    // ----------------------------------------------------------- products
    constexpr uint32_t kIdesc = idesc_e4m3(128, TN);
    const uint32_t base = warp_uniform(smem_u32(smem)), tm = warp_uniform(tmem);
    const bool leader = elect_one();
    bool ok = true;
    int32_t n = 0, s = 0;
    uint32_t ph = 0;
#pragma unroll 1
    for (int32_t i = first; i < total && ok; i += step) {
#pragma unroll 1
      for (int32_t kb = kb_lo; kb < kb_hi; kb += U, ++n) {
        const int b = n % B;
        if (n >= B) ok = wait_warp(&tempty[b], (n / B - 1) & 1, a.status, L.max_polls);
        // (last: W is what these products wait for)
        ok = ok && wait_warp(&full[s], ph, a.status, L.max_polls);
        if (!ok) break;
        tc_fence_after();
        const uint64_t dw = smem_desc(base + s * H::kStage, 16, 1024);
        const uint64_t da = smem_desc(base + s * H::kStage + U * H::kWBytes, 16, 1024);
        if (leader) {
#pragma unroll
          for (int k = 0; k < kGroup / 32; ++k) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
              if (U > 1 && kb + u >= kb_hi) break;
              mma8_ss(tm + (b * U + u) * TN, smem_desc_at(dw, u * H::kWBytes + k * 32),
                      smem_desc_at(da, u * H::kCBytes + k * 32), kIdesc, k > 0);
            }
          }
          mma_commit(&empty[s]);
          mma_commit(&tfull[b]);
        }
        __syncwarp();
        if (++s == S) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    if (n > 0) land(&tfull[(n - 1) % B], ((n - 1) / B) & 1);  // (nor does an epilogue that gave up)
  } else {
    // ----------------------------------------------------------- epilogue
    // a lane's row of W, the warp's first row of A
    const int32_t wrow = (warp & 3) * 32 + lane, col = (warp >> 2) * CW;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    // Scales come by cp.async, kAhead blocks together and as many ahead, into slots that only this
    // warp reads: [2][kAhead][warp][A's, W's].
    const uint32_t scales_at = smem_u32(scales) + warp * H::kSlot * 4;
    int32_t next_tile = first, next_kb = kb_hi;
    uint32_t next_half = 0;
    const float* next_a = nullptr;
    const float* next_w = nullptr;
    int32_t live = 0;
    auto ask = [&]() {
      if (next_kb >= kb_hi && next_tile < total) {
        const int32_t c = next_tile / tiles_w;
        next_w = a.w_scale + kb_lo * a.ldws + (next_tile - c * tiles_w);
        live = max(0, min(CW, a.M - c * TN - col));
        next_a = a.a_scale + kb_lo * a.ldas + (live > 0 ? c * TN + col : 0);
        next_tile += step;
        next_kb = kb_lo;
      }
      const uint32_t to = scales_at + next_half * (kAhead * EW * H::kSlot * 4);
#pragma unroll 1
      for (int u = 0; u < kAhead && next_kb + u < kb_hi; ++u) {
#pragma unroll
        for (int t = 0; t < CW; t += 32)
          if (t + lane < CW)
            cp_async4(to + u * EW * H::kSlot * 4 + (t + lane) * 4, next_a + max(0, min(t + lane, live - 1)),
                      t + lane < live);
        if (lane == 0) cp_async4(to + u * EW * H::kSlot * 4 + CW * 4, next_w, true);
        next_a += a.ldas;
        next_w += a.ldws;
      }
      next_kb += kAhead;
      next_half ^= 1u;
      cp_async_commit();
    };
    ask();
    bool ok = true;
    int32_t n = 0;
    uint32_t half = 0;
#pragma unroll 1
    for (int32_t i = first; i < total && ok; i += step) {
      if (a.add != nullptr && tid < 2 * TN) {  // what is added, on its way to L2 meanwhile
        const int32_t c = i / tiles_w, m = c * TN + (tid >> 1), n = (i - c * tiles_w) * kLaneRows + (tid & 1) * 64;
        if (m < a.M && n < a.N)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint16_t*>(a.add) + m * a.ldadd + n));
      }
      float2 acc[CW / 2];
#pragma unroll
      for (int e = 0; e < CW / 2; ++e) acc[e] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int32_t kb = kb_lo; kb < kb_hi; kb += U, ++n) {
        if ((kb - kb_lo) % kAhead == 0) {
          cp_async_wait<0>();
          __syncwarp();  // (every lane's, and every lane has read the other half)
          half = next_half ^ 1u;
          ask();
        }
        const float* sc = scales + ((half * kAhead + (kb - kb_lo) % kAhead) * EW + warp) * H::kSlot;
        const int b = n % B;
        ok = wait_warp(&tfull[b], (n / B) & 1, a.status, L.max_polls);
        if (!ok) break;
        tc_fence_after();
        // (a unit's blocks lie side by side: where a warp takes all of their columns, one read)
        constexpr int kReads = CW == TN && TN > 16 ? 1 : U, kOf = U / kReads;
#pragma unroll
        for (int q = 0; q < kReads; ++q) {
          uint32_t w[kOf * CW];
          tmem_ask(tmem + lane_off + (b * U + q) * TN + col, w);
          float ws[kOf];
#pragma unroll
          for (int u = 0; u < kOf; ++u) ws[u] = sc[(q + u) * EW * H::kSlot + CW];
          tmem_have(w);
          if (q + 1 == kReads) {
            tc_fence_before();
            __syncwarp();
            arrive_lane0(&tempty[b], lane);
          }
#pragma unroll
          for (int u = 0; u < kOf; ++u) {
            if (U > 1 && kb + q + u >= kb_hi) continue;
            const float4* s4 = reinterpret_cast<const float4*>(sc + (q + u) * EW * H::kSlot);
            const float2 ws2 = make_float2(ws[u], ws[u]), zero = make_float2(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < CW; e += 4) {
              const float4 x = s4[e / 4];
              const uint32_t* v = w + u * CW + e;
              const float2 lo = make_float2(__uint_as_float(v[0]), __uint_as_float(v[1]));
              const float2 hi = make_float2(__uint_as_float(v[2]), __uint_as_float(v[3]));
              acc[e / 2] = ffma2(lo, ffma2(make_float2(x.x, x.y), ws2, zero), acc[e / 2]);
              acc[e / 2 + 1] = ffma2(hi, ffma2(make_float2(x.z, x.w), ws2, zero), acc[e / 2 + 1]);
            }
          }
        }
      }
      if (!ok) break;
      if (splits > 1) {  // to the cluster's sums, below (one tile a CTA)
        float* mine = reinterpret_cast<float*>(smem) + col * kLaneRows + wrow;
#pragma unroll
        for (int e = 0; e < CW / 2; ++e) {
          mine[2 * e * kLaneRows] = acc[e].x;
          mine[(2 * e + 1) * kLaneRows] = acc[e].y;
        }
      } else {
        const int32_t c = i / tiles_w, nn = (i - c * tiles_w) * kLaneRows + wrow, m0 = c * TN + col;
        if (nn < a.N) {
          // (what is added is asked for 16 rows at a time)
#pragma unroll
          for (int e0 = 0; e0 < CW; e0 += 16) {
            float x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = m0 + e0 + e < a.M ? added(a, m0 + e0 + e, nn) : 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (m0 + e0 + e < a.M)
                store_one(a, m0 + e0 + e, nn, (e & 1 ? acc[(e0 + e) / 2].y : acc[(e0 + e) / 2].x) + x[e]);
          }
        }
      }
    }
    cp_async_wait<0>();
    if (!ok && lane == 0) gave_up = 1;
  }

  // ---- teardown
  tc_fence_before();
  __syncwarp();  // (cluster barriers take whole warps)
  if (splits > 1) {
    cluster_sync_all();
    // every CTA of the cluster adds up the rows of A that are its rank's (none where a CTA gave up)
    const int32_t c = first / tiles_w, n = (first - c * tiles_w) * kLaneRows + (tid & 127);
    const int32_t live = min(TN, a.M - c * TN), step = splits * (EW / 4);
    if (warp < EW) {
      constexpr int kTogether = CW / 16;  // rows whose sums are asked for together
      const uint32_t at = smem_u32(smem) + (tid & 127) * 4;
      // (asked for ahead of the sums; splits is a power of two)
      const float unknown = ld_peer(peer_addr(smem_u32(&gave_up), lane & (splits - 1)));
#pragma unroll 1
      for (int32_t t0 = rank + (tid >> 7) * splits; t0 < live; t0 += kTogether * step) {
        float v[kTogether][kMaxSplits], more[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
          const int32_t t = min(t0 + u * step, live - 1);
          more[u] = n < a.N ? added(a, c * TN + t, n) : 0.f;
#pragma unroll
          for (int32_t r = 0; r < kMaxSplits; ++r)
            v[u][r] = r < splits ? ld_peer(peer_addr(at + t * kLaneRows * 4, r)) : 0.f;
        }
        const bool known = !__any_sync(0xffffffffu, __float_as_uint(unknown) != 0);  // (by all lanes)
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
          float x = 0.f;
#pragma unroll
          for (int32_t r = 0; r < kMaxSplits; ++r) x += v[u][r];
          if (known && t0 + u * step < live && n < a.N) store_one(a, c * TN + t0 + u * step, n, x + more[u]);
        }
      }
    }
    __syncwarp();
    cluster_sync_all();
  } else {
    __syncthreads();
  }
  if (warp == EW + 1) {
    tc_fence_after();
    tmem_dealloc(tmem, H::kCols);
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

template <bool PAIR, int TN, int U, bool kVec>
cudaError_t launch_of(const ScaledMatmulArgs& a, cudaStream_t stream) {
  using H = Shape<PAIR, TN, U>;
  Launch L{};
  L.tiles_l = ceil_div(a.M, PAIR ? 2 * kLaneRows : kLaneRows);
  L.tiles_c = ceil_div(a.N, TN);
  CUtensorMap ta, tw;
  if (!rows_map(&ta, a.a, a.K, a.M, a.lda, kLaneRows) || !rows_map(&tw, a.w, a.K, a.N, a.ldw, H::kCRows))
    return cudaErrorInvalidValue;
  auto kernel = scaled_matmul_kernel<PAIR, TN, U, kVec>;
  const cudaError_t e = allow_smem(kernel, H::kSmem);
  if (e != cudaSuccess) return e;
  // Where all SMs read the same few lines of A at once, L2 serves them much faster under this policy
  // (152 tiles of 64 rows, K 1024: 15.5 us, 6.9; 128 rows, 512: 6.3, 4.9).
  L.often = (int64_t)a.M * a.K <= kOftenBytes;
  L.even = (a.ldc - a.ldadd) % 4 == 0 && (reinterpret_cast<uintptr_t>(a.c) / (a.c_bf16 ? 2 : 4) -
                                          reinterpret_cast<uintptr_t>(a.add) / 2) % 4 == 0;
  const int64_t tiles = (int64_t)L.tiles_l * L.tiles_c, sms = device_sm_count();
  if (PAIR)
    return launch_clusters(kernel, dim3((unsigned)(2 * std::min(tiles, sms / 2))), dim3(H::kThreads), H::kSmem,
                           stream, true, 2, ta, tw, a, L);
  return launch_kernel(kernel, dim3((unsigned)std::min(tiles, sms)), dim3(H::kThreads), H::kSmem, stream, true,
                       ta, tw, a, L);
}

// Whether C may be written, and add read, 16 bytes of C at a time.
bool on_vectors(const ScaledMatmulArgs& a) {
  auto even = [&](const void* p, int64_t ld, uintptr_t bytes) {
    return ld % (a.c_bf16 ? 8 : 4) == 0 && (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
  };
  return even(a.c, a.ldc, 16) && (a.add == nullptr || even(a.add, a.ldadd, a.c_bf16 ? 16 : 8));
}
template <bool PAIR, int TN, int U>
cudaError_t launch(const ScaledMatmulArgs& a, bool vec, cudaStream_t stream) {
  return vec ? launch_of<PAIR, TN, U, true>(a, stream) : launch_of<PAIR, TN, U, false>(a, stream);
}

// CTAs that a tile's blocks are cut over: a power of two (clusters of six leave places of a GPC
// empty: 48 tiles of 32 blocks 11.9 us, four CTAs each 8.2, two 8.7, one 11.4), and all at work at
// once (32 tiles of 96 blocks: eight 12.0, four 12.3, one 27.0; 48 of 32: eight 10.0), of short sums on an
// SM each (30 tiles of 9 blocks: eight 6.2, four 5.2).  The cluster's sums cost about a microsecond:
// not for fewer than six blocks (52 tiles of 5: two 6.0, one 5.1), and in two only for many (88 tiles of
// 13: two 11.0, one 7.9; 95 of 57: 19.5 and 22.6).
int32_t few_splits(int32_t tiles, int32_t blocks, int32_t sms) {
  const int64_t most = blocks >= 24 ? sms * 7 / 4 : sms;
  int32_t n = 1;
  while (n < kMaxSplits && (int64_t)tiles * n * 2 <= most && blocks >= n * 2) n *= 2;
  return blocks < 6 || (n == 2 && blocks < 24) ? 1 : n;
}

template <int TN, int U>
cudaError_t launch_few(const ScaledMatmulArgs& a, int32_t splits, cudaStream_t stream) {
  using H = Few<TN, U>;
  CUtensorMap ta, tw;
  if (!rows_map(&ta, a.a, a.K, a.M, a.lda, TN) || !rows_map(&tw, a.w, a.K, a.N, a.ldw, kLaneRows))
    return cudaErrorInvalidValue;
  auto kernel = scaled_matmul_few_kernel<TN, U>;
  const cudaError_t e = allow_smem(kernel, H::kSmem);
  if (e != cudaSuccess) return e;
  const int32_t tiles_w = ceil_div(a.N, kLaneRows), total = tiles_w * ceil_div(a.M, TN);
  const FewLaunch L{tiles_w, total, splits, wait_poll_limit(), std::min(barrier_shortfall(), 1u)};
  if (splits > 1)
    return launch_clusters(kernel, dim3((unsigned)(total * splits)), dim3(H::kThreads), H::kSmem, stream, true,
                           splits, ta, tw, a, L);
  return launch_kernel(kernel, dim3((unsigned)std::min(total, 2 * device_sm_count())), dim3(H::kThreads),
                       H::kSmem, stream, true, ta, tw, a, L);
}

}  // namespace

cudaError_t launch_scaled_matmul(const ScaledMatmulArgs& a, cudaStream_t stream) {
  const int64_t blocks = ceil_div(a.K, kGroup), sms = device_sm_count();
  if (a.M <= 64) {
    // With W's rows on the lanes the blocks are cut, and W is read once at the most tiles; with A's,
    // a CTA gets going sooner and takes 0.26 us a block instead of 0.24 (16 rows), 0.25 (32), 0.35 (64).
    // Measured (us, 96 tiles of 128 of W): 64 rows, 2 blocks 5.8 and 4.2, 16 10.6 and 7.8, 32 18.5 and
    // 12.0, 64 26.7 and 28.8; 48 tiles of 32 rows, 16 9.0 and 7.8, but 152 9.5 and 11.8 (all of them at the
    // same lines of A); 16 of 64 rows, 64 blocks 11.1 and 21.4; 304 of 32 29.2 and 33.6.
    const int32_t tiles = ceil_div(a.N, kLaneRows), n = few_splits(tiles, (int32_t)blocks, (int32_t)sms);
    const bool wide = tiles <= sms && blocks <= 48 && a.M > 16 &&
                      (a.M > 32 ? n == 1 || blocks < 12 || (n < 4 && blocks <= 32)
                                : n == 1 && (tiles * blocks <= 1024 || blocks >= 24));
    if (a.M <= 16) return launch_few<16, 2>(a, n, stream);
    if (!wide) return a.M <= 32 ? launch_few<32, 2>(a, n, stream) : launch_few<64, 2>(a, n, stream);
  }
  // Nanoseconds, about: of a launch, and for every round of tiles what a block takes and a tile's way out
  // (of 256 and of 128 columns).  Tiles of a pair are better for their size and worse where they leave SMs
  // idle.  Measured (us, 256 x 256 and 256 x 128 of a pair, 128 x 128): 1024 x 4096 x 4096 with a sum 24.5,
  // 28, 27; 200 x 5000 x 2050 14.6, 10.3, 9.6; 264 x 24448 x 9134 124, 144, 138; 5848 x 58870 x 172 207, -,
  // 312; to float32 with rows anywhere 551, -, 520.  Over 350 drawn products 1% above the best of the three.
  const bool vec = on_vectors(a);
  const int64_t out256 = a.add != nullptr ? (vec ? 6900 : 10100) : a.c_bf16 ? (vec ? 2700 : 3900) : vec ? 5900 : 6600;
  const int64_t out128 = a.add != nullptr ? (vec ? 3200 : 4800) : a.c_bf16 ? (vec ? 1800 : 2200) : vec ? 2400 : 3300;
  auto cost = [&](int32_t rows, int32_t cols, int64_t places, int64_t fixed, int64_t block, int64_t out) {
    const int64_t tiles = (int64_t)ceil_div(a.M, rows) * ceil_div(a.N, cols);
    return fixed + ceil_div(tiles, places) * (blocks * block + out);
  };
  const int64_t c256 = cost(256, 256, sms / 2, 4000, 500, out256), p128 = cost(256, 128, sms / 2, 3300, 315, out128),
                c128 = cost(128, 128, sms, 2500, 340, out128);
  if (c256 < p128 && c256 < c128) return launch<true, 256, 1>(a, vec, stream);
  return p128 < c128 ? launch<true, 128, 2>(a, vec, stream) : launch<false, 128, 2>(a, vec, stream);
}

}  // namespace ssd
