// cache_attention.cu — frontier attention over the paged 8-bit cache
// (include/ssd.h, ssd_cache_attention):
//   O[b][j][h] = softmax_s(scale * Q[b][j][h] . (sk K[s]) + M(s, j)) (sv V[s]),
// K and V e4m3 with a scale per block of tokens and KV head (sk, sv).
//
// Every e4m3 value is a float16, so the products run as mma.sync on float16
// with float32 accumulation and the scales stay outside: sk multiplies the
// scores, sv the probabilities before they are rounded to float16.
//
// A warp takes 16 query rows (drafts x the query heads that share the KV head)
// and walks steps of 16 keys.  The order of an mma's inner index and of its
// columns is free as long as both operands agree, so each lane reads the 16
// bytes it needs from global memory in one piece: of K, 16 consecutive values
// of a key for four mma steps; of V, 16 consecutive columns of a key for sixteen
// output tiles.  The copies go through a ring of shared memory that only the
// lane itself reads (cp.async; no barrier), four steps deep.
// The warps of a CTA split 16-key steps among them where the rows are few (and
// merge at the end), else they take four row tiles of the same keys.

#include <cuda_fp16.h>

#include <algorithm>

#include "cache_attention.cuh"

namespace ssd {

namespace {

constexpr int kWarps = 4;
constexpr int kStages = 4;          // steps in flight per warp
constexpr int kStep = 16;           // keys per step
constexpr int kMinTiles = 2;        // a part's fewest tiles (times the warps that share its rows / 4)
constexpr int kMaxPartTiles = 256;  // 16384 keys: at most 1024 block ids and scales in shared memory
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// log2 growth of the running maximum (and growth of the V scale) that moves the
// reference: P stays below 2^8 * 2^4 in float16
constexpr float kGrowth = 8.f, kVGrowth = 16.f;

struct Plan {
  int32_t wr, rowgroups, splits, min_tiles;
};

Plan make_plan(int32_t B, int32_t Hq, int32_t Hkv, int32_t D_max, int32_t L_max) {
  Plan p;
  const int64_t rows = (int64_t)D_max * (Hq / Hkv);
  const int64_t row_tiles = (rows + 15) / 16;
  p.wr = row_tiles >= 3 ? 4 : (int32_t)row_tiles;
  p.rowgroups = (int32_t)((row_tiles + p.wr - 1) / p.wr);
  const int64_t base = (int64_t)B * Hkv * p.rowgroups;
  const int64_t target = 3 * (int64_t)device_sm_count();
  p.min_tiles = kMinTiles * (kWarps / p.wr);
  const int64_t tiles = (L_max + kCacheTile - 1) / kCacheTile;
  const int64_t most = std::max<int64_t>(1, tiles / p.min_tiles);
  // (and no part longer than the room for its block ids)
  const int64_t least = (tiles + kMaxPartTiles - 1) / kMaxPartTiles;
  p.splits = (int32_t)std::max<int64_t>(least, std::min<int64_t>((target + base - 1) / base, most));
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
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, bool valid) {
  const uint32_t n = valid ? BYTES : 0;  // the rest is filled with zeros
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n)
                 : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES),
                 "r"(n)
                 : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32, 3)
cache_attn_kernel(CacheAttnArgs a, CacheAttnLaunch L, int32_t row_warps) {
  constexpr int NT = D / 8;           // output tiles of 8 columns
  constexpr int KG = D / 64;          // groups of four mma steps of QK^T
  constexpr int VB = D / 8;           // bytes of V a lane takes per key
  constexpr int kStageBytes = 2 * kStep * D;
  constexpr int kWarpBytes = kStages * kStageBytes;
  static_assert(kWarpBytes >= 16 * D * 4 + 16 * 8, "a warp's partial rows fit its ring");
  extern __shared__ __align__(16) unsigned char smem[];
  int32_t* s_id = reinterpret_cast<int32_t*>(smem + kWarps * kWarpBytes);
  float* s_ks = reinterpret_cast<float*>(s_id + L.max_blocks);
  float* s_vs = s_ks + L.max_blocks;
  pdl_wait();

  const int32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t split = blockIdx.x, b = blockIdx.y / a.cache.Hkv, g = blockIdx.y % a.cache.Hkv;
  const int32_t S = a.cache.block, S_log = 31 - __clz(S), G = a.Hq / a.cache.Hkv;
  const int32_t cache = a.cache_len[b], nd = a.n_drafts[b];
  if (!cache_lengths_ok(a, cache, nd)) {
    if (tid == 0 && split == 0 && g == 0 && blockIdx.z == 0)
      record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
    return;
  }
  const int32_t Lk = cache + nd, rows_total = nd * G;
  const int32_t tiles = (Lk + kCacheTile - 1) / kCacheTile;
  const int32_t parts = cache_parts(L.splits, L.min_tiles, tiles);
  const int32_t row_g0 = blockIdx.z * row_warps * 16;
  if (row_g0 >= rows_total || split >= parts) return;
  const int32_t t_lo = (int32_t)((int64_t)tiles * split / parts);
  const int32_t t_hi = (int32_t)((int64_t)tiles * (split + 1) / parts);
  const int32_t k_lo = t_lo * kCacheTile, k_hi = min(Lk, t_hi * kCacheTile);
  const int32_t start = a.key_start != nullptr ? min(Lk, max(0, a.key_start[b])) : 0;

  // ---- the part's block ids and scales
  const int32_t b_lo = k_lo >> S_log;  // (a part may start inside a block of 128)
  const int32_t nb = ((k_hi - 1) >> S_log) + 1 - b_lo;
  for (int32_t i = tid; i < nb; i += blockDim.x) {
    int32_t id = a.block_table[(int64_t)b * a.max_blocks + b_lo + i];
    if (id < 0 || id >= a.cache.num_blocks) {
      record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      id = -1;
    }
    s_id[i] = id;
    const int64_t at = (int64_t)id * a.cache.Hkv + g;
    s_ks[i] = id < 0 ? 0.f : a.cache.k_scale[at];
    s_vs[i] = id < 0 ? 0.f : a.cache.v_scale[at];
  }

  // ---- this warp's rows and its share of the steps
  const int32_t wk_n = kWarps / row_warps, wr = warp % row_warps, wk = warp / row_warps;
  const int32_t q = lane & 3, r8 = lane >> 2;
  const int32_t row0 = row_g0 + wr * 16;
  int32_t qpos[2];
  int32_t minq = 0x7fffffff;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int32_t r = row0 + r8 + 8 * i;
    qpos[i] = -1;
    if (r < rows_total) {
      qpos[i] = cache_flat_pos(a, b, cache, r / G);
      if (qpos[i] < 0 && split == 0 && g == 0) record_status(a.status, SSD_ERR_DEVICE_BOUNDS);
      minq = min(minq, qpos[i]);
    }
  }
  minq = __reduce_min_sync(0xffffffffu, minq);
  // keys below this one are visible to every row of the warp
  const int32_t mask_from = min(cache, minq + 1);

  // Q as float16 with its row's power of two taken out; column order of K's reads
  uint32_t qf[KG][4][4];
  float rowc[2];
  const float c2 = (a.scale != 0.f ? a.scale : rsqrtf((float)D)) * kLog2e;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int32_t r = row0 + r8 + 8 * i;
    const bool live = r < rows_total;
    const int32_t j = live ? r / G : 0, h = g * G + (live ? r - j * G : 0);
    const uint4* src = reinterpret_cast<const uint4*>(
        static_cast<const __nv_bfloat16*>(a.q) + (((int64_t)b * a.D_max + j) * a.Hq + h) * D);
    float x[KG][16];
    float m = 0.f;
#pragma unroll
    for (int kg = 0; kg < KG; ++kg)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint4 w = live ? src[kg * 8 + q * 2 + u] : make_uint4(0, 0, 0, 0);
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
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    rowc[i] = c2 * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
    for (int kg = 0; kg < KG; ++kg)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        qf[kg][s][i] = pack_f16x2(x[kg][4 * s] * down, x[kg][4 * s + 1] * down);
        qf[kg][s][2 + i] = pack_f16x2(x[kg][4 * s + 2] * down, x[kg][4 * s + 3] * down);
      }
  }
  __syncthreads();  // ids and scales

  const int32_t first = max(k_lo, start & ~(kStep - 1));  // multiple of 16
  const uint32_t ring = smem_u32(smem) + warp * kWarpBytes;
  const uint8_t* kbase = static_cast<const uint8_t*>(a.cache.k);
  const uint8_t* vbase = static_cast<const uint8_t*>(a.cache.v);
  auto key_of = [&](int32_t t) { return first + (t * wk_n + wk) * kStep; };
  auto issue = [&](int32_t t) {
    const int32_t k0 = key_of(t);
    if (k0 < k_hi && row0 < rows_total) {
      const int32_t i = (k0 >> S_log) - b_lo, id = s_id[i];
      const int64_t at =
          (((int64_t)max(id, 0) * a.cache.Hkv + g) * S + (k0 & (S - 1))) * D;
      const uint32_t dst = ring + (t % kStages) * kStageBytes;
      auto valid = [&](int32_t k) { return id >= 0 && k0 + k >= start && k0 + k < k_hi; };
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int kg = 0; kg < KG; ++kg) {
          const int32_t k = n * 8 + r8;
          cp_async<16>(dst + (n * KG + kg) * 512 + lane * 16, kbase + at + k * D + kg * 64 + q * 16,
                       valid(k));
        }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int32_t k = (n >> 1) * 8 + 2 * q + (n & 1);
        cp_async<VB>(dst + kStep * D + n * 32 * VB + lane * VB, vbase + at + k * D + r8 * VB,
                     valid(k));
      }
    }
    cp_commit();
  };
#pragma unroll
  for (int t = 0; t < kStages - 1; ++t) issue(t);

  float o[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
  float m_ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float v_ref = 0.f, v_inv = 0.f;

  if (row0 < rows_total) {
#pragma unroll 1
    for (int32_t t = 0; key_of(t) < k_hi; ++t) {
      cp_wait<kStages - 2>();
      issue(t + kStages - 1);
      const int32_t k0 = key_of(t), bi = (k0 >> S_log) - b_lo;
      const unsigned char* st = smem + warp * kWarpBytes + (t % kStages) * kStageBytes;
      // ---- S = Q K^T
      float sc[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
        for (int kg = 0; kg < KG; ++kg) {
          const uint4 w = *reinterpret_cast<const uint4*>(st + (n * KG + kg) * 512 + lane * 16);
          mma_f16(sc[n], qf[kg][0], f16_lo(w.x), f16_hi(w.x));
          mma_f16(sc[n], qf[kg][1], f16_lo(w.y), f16_hi(w.y));
          mma_f16(sc[n], qf[kg][2], f16_lo(w.z), f16_hi(w.z));
          mma_f16(sc[n], qf[kg][3], f16_lo(w.w), f16_hi(w.w));
        }
      }
      const float ks = s_ks[bi], vs = s_vs[bi];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] *= rowc[e >> 1] * ks;
      if (k0 < start || k0 + kStep > min(mask_from, k_hi) || s_id[bi] < 0) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int32_t key = k0 + n * 8 + 2 * q + u;
            int32_t kp = 0x7fffffff;
            if (key >= start && key < k_hi && s_id[bi] >= 0) {
              kp = key;
              if (key >= cache) {
                kp = cache_flat_pos(a, b, cache, key - cache);
                if (kp < 0) kp = 0x7fffffff;
              }
            }
            if (kp > qpos[0]) sc[n][u] = -INFINITY;
            if (kp > qpos[1]) sc[n][2 + u] = -INFINITY;
          }
      }
      // ---- softmax against a reference maximum that moves when it falls behind
      float mx[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mx[i] = fmaxf(fmaxf(sc[0][2 * i], sc[0][2 * i + 1]), fmaxf(sc[1][2 * i], sc[1][2 * i + 1]));
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
      }
      const bool behind = mx[0] > m_ref[0] + kGrowth || mx[1] > m_ref[1] + kGrowth;
      const bool v_behind = !(vs <= v_ref * kVGrowth);  // the same in every lane
      if (__any_sync(0xffffffffu, behind) || v_behind) {
        float f = 1.f;
        if (v_behind) {
          const float to = fmaxf(vs, 0x1p-120f);
          f = v_ref / to;
          v_ref = to;
          v_inv = 1.f / to;
        }
        float al[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float m = fmaxf(m_ref[i], mx[i]);
          al[i] = m == -INFINITY ? 1.f : exp2f(m_ref[i] - m);
          m_ref[i] = m;
          l[i] *= al[i];
          al[i] *= f;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          o[n][0] *= al[0];
          o[n][1] *= al[0];
          o[n][2] *= al[1];
          o[n][3] *= al[1];
        }
      }
      const float ratio = vs * v_inv;
      uint32_t pf[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float m = m_ref[i] == -INFINITY ? 0.f : m_ref[i];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float p0 = ex2_approx(sc[n][2 * i] - m), p1 = ex2_approx(sc[n][2 * i + 1] - m);
          l[i] += p0 + p1;
          pf[2 * n + i] = pack_f16x2(p0 * ratio, p1 * ratio);
        }
      }
      // ---- O += P V: output tile nt holds column n * VB + nt as its n-th
      uint32_t v[4][VB / 4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const unsigned char* at = st + kStep * D + n * 32 * VB + lane * VB;
        if constexpr (VB == 16) {
          const uint4 w = *reinterpret_cast<const uint4*>(at);
          v[n][0] = w.x;
          v[n][1] = w.y;
          v[n][2] = w.z;
          v[n][3] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(at);
          v[n][0] = w.x;
          v[n][1] = w.y;
        }
      }
#pragma unroll
      for (int w = 0; w < VB / 4; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t sel = h == 0 ? 0x5140u : 0x7362u;
          const uint32_t x0 = __byte_perm(v[0][w], v[1][w], sel);
          const uint32_t x1 = __byte_perm(v[2][w], v[3][w], sel);
          mma_f16(o[4 * w + 2 * h], pf, f16_lo(x0), f16_lo(x1));
          mma_f16(o[4 * w + 2 * h + 1], pf, f16_hi(x0), f16_hi(x1));
        }
    }
  }
  cp_wait<0>();

#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
  }

  // ---- merge the warps that shared the rows
  // a lane's columns of a row: q * 2 * VB + (0 .. VB - 1), then VB more
  if (wk_n > 1) {
    __syncwarp();
    unsigned char* mine = smem + warp * kWarpBytes;
    float2* ml = reinterpret_cast<float2*>(mine + 16 * D * 4);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float* po = reinterpret_cast<float*>(mine) + (r8 + 8 * i) * D;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NT; ++n) po[q * 2 * VB + u * VB + n] = o[n][2 * i + u] * v_ref;
      if (q == 0) ml[r8 + 8 * i] = make_float2(m_ref[i], l[i]);
    }
    __syncthreads();
    if (wk != 0) return;
    v_ref = 1.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t r = r8 + 8 * i;
      float M = -INFINITY;
      for (int w = 0; w < wk_n; ++w)
        M = fmaxf(M, reinterpret_cast<const float2*>(smem + (wr + w * row_warps) * kWarpBytes +
                                                     16 * D * 4)[r].x);
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n][2 * i] = o[n][2 * i + 1] = 0.f;
      for (int w = 0; w < wk_n; ++w) {
        const unsigned char* at = smem + (wr + w * row_warps) * kWarpBytes;
        const float2 x = reinterpret_cast<const float2*>(at + 16 * D * 4)[r];
        const float f = x.x == -INFINITY ? 0.f : exp2f(x.x - M);
        sum += x.y * f;
        const float* po = reinterpret_cast<const float*>(at) + r * D + q * 2 * VB;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          o[n][2 * i] += po[n] * f;
          o[n][2 * i + 1] += po[VB + n] * f;
        }
      }
      m_ref[i] = M;
      l[i] = sum;
    }
  }

  // ---- the rows, or the part's share of them
  const bool direct = parts == 1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int32_t r = row0 + r8 + 8 * i;
    if (r >= rows_total) continue;
    const int32_t j = r / G, h = g * G + (r - j * G);
    if (direct) {
      const int64_t at = ((int64_t)b * a.D_max + j) * a.Hq + h;
      if (!dbg_in(at, (int64_t)a.B * a.D_max * a.Hq, a.status)) continue;
      const float f = l[i] > 0.f ? v_ref / l[i] : 0.f;
      uint32_t* ob = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(a.o) + at * D + q * 2 * VB);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NT; n += 2)
          ob[(u * VB + n) / 2] = pack_bf16x2(o[n][2 * i + u] * f, o[n + 1][2 * i + u] * f);
      if (a.lse != nullptr && q == 0)
        a.lse[((int64_t)b * a.Hq + h) * a.D_max + j] =
            l[i] > 0.f ? (m_ref[i] + log2f(l[i])) * kLn2 : -INFINITY;
    } else {
      const int64_t at = (((int64_t)b * a.D_max + j) * a.Hq + h) * L.splits + split;
      if (!dbg_in(at, (int64_t)a.B * a.D_max * a.Hq * L.splits, a.status)) continue;
      float2* po = reinterpret_cast<float2*>(L.part_o + at * D + q * 2 * VB);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NT; n += 2)
          po[(u * VB + n) / 2] = make_float2(o[n][2 * i + u] * v_ref, o[n + 1][2 * i + u] * v_ref);
      if (q == 0) L.part_ml[at] = make_float2(m_ref[i], l[i]);
    }
  }
}

// One warp per (sequence, draft, head): the parts of its row, weighted by their
// reference maxima.
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
  const int32_t parts =
      cache_parts(L.splits, L.min_tiles, (cache + nd + kCacheTile - 1) / kCacheTile);
  if (parts == 1) return;  // written by the attention kernel
  const int64_t at = row * L.splits;
  if (!dbg_in(at + parts - 1, (int64_t)a.B * a.D_max * a.Hq * L.splits, a.status)) return;
  float M = -INFINITY;
  for (int32_t s = lane; s < parts; s += 32) M = fmaxf(M, L.part_ml[at + s].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  constexpr int PER = D / 32;
  float acc[PER], sum = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) acc[k] = 0.f;
  for (int32_t s = 0; s < parts; ++s) {
    const float2 x = L.part_ml[at + s];
    const float f = x.x == -INFINITY ? 0.f : exp2f(x.x - M);
    sum += x.y * f;
    const float* po = L.part_o + (at + s) * D + lane * PER;
#pragma unroll
    for (int k = 0; k < PER; ++k) acc[k] += po[k] * f;
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  __nv_bfloat16* ob = static_cast<__nv_bfloat16*>(a.o) + row * D + lane * PER;
#pragma unroll
  for (int k = 0; k < PER; k += 2)
    *reinterpret_cast<uint32_t*>(ob + k) = pack_bf16x2(acc[k] * inv, acc[k + 1] * inv);
  if (a.lse != nullptr && lane == 0)
    a.lse[((int64_t)b * a.Hq + h) * a.D_max + j] = sum > 0.f ? (M + log2f(sum)) * kLn2 : -INFINITY;
}

template <int D>
cudaError_t launch_mma(const CacheAttnArgs& a, const Plan& p, const CacheAttnLaunch& L,
                       cudaStream_t stream) {
  const size_t smem = (size_t)kWarps * kStages * 2 * kStep * D + (size_t)L.max_blocks * 12;
  const cudaError_t e = cudaFuncSetAttribute(
      cache_attn_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(cache_attn_kernel<D>, dim3(p.splits, a.B * a.cache.Hkv, p.rowgroups),
                       dim3(kWarps * 32), smem, stream, true, a, L, p.wr);
}

size_t part_bytes(int64_t rows, int32_t splits, int32_t d) {
  if (splits == 1) return 0;
  return align256((size_t)rows * splits * d * sizeof(float)) +
         align256((size_t)rows * splits * sizeof(float2));
}

}  // namespace

// Enough for either kernel: which one runs depends on arguments that the
// query does not have.
size_t cache_attention_workspace(int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t D_max,
                                 int32_t L_max) {
  int32_t splits, min_tiles;
  cache_attention_tc_plan(B, Hq, Hkv, D_max, L_max, &splits, &min_tiles);
  splits = std::max(splits, make_plan(B, Hq, Hkv, D_max, L_max).splits);
  return part_bytes((int64_t)B * D_max * Hq, splits, d);
}

cudaError_t launch_cache_attention(const CacheAttnArgs& a, void* ws, cudaStream_t stream) {
  const int32_t L_max = a.max_blocks * a.cache.block, d = a.cache.d;
  const bool tc = cache_attention_tc_runs(a);
  const Plan p = make_plan(a.B, a.Hq, a.cache.Hkv, a.D_max, L_max);
  CacheAttnLaunch L{p.splits, p.min_tiles, 0, nullptr, nullptr};
  if (tc)
    cache_attention_tc_plan(a.B, a.Hq, a.cache.Hkv, a.D_max, L_max, &L.splits, &L.min_tiles);
  const int32_t tiles = (L_max + kCacheTile - 1) / kCacheTile;
  L.max_blocks =
      cache_part_tiles(L.splits, L.min_tiles, tiles) * (kCacheTile / std::min(a.cache.block, 64)) + 1;
  const int64_t rows = (int64_t)a.B * a.D_max * a.Hq;
  if (L.splits > 1) {
    L.part_o = static_cast<float*>(ws);
    L.part_ml = reinterpret_cast<float2*>(
        static_cast<unsigned char*>(ws) + align256((size_t)rows * L.splits * d * sizeof(float)));
  }
  cudaError_t e = tc ? launch_cache_attention_tc(a, L, stream)
                     : (d == 128 ? launch_mma<128>(a, p, L, stream) : launch_mma<64>(a, p, L, stream));
  if (e != cudaSuccess || L.splits == 1) return e;
  const dim3 grid((unsigned)((rows + 7) / 8));
  return d == 128 ? launch_kernel(cache_attn_combine_kernel<128>, grid, dim3(256), 0, stream, true, a, L)
                  : launch_kernel(cache_attn_combine_kernel<64>, grid, dim3(256), 0, stream, true, a, L);
}

}  // namespace ssd
