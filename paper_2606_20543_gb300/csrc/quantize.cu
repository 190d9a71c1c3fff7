// quantize.cu — rows (or 128 x 128 blocks of a weight) to e4m3 with a float32 scale per 128
// entries (include/ssd.h, ssd_quantize):
//   s = max(largest finite |x|, 2^-100) / 448,   q = e4m3(clamp(x * (1 / s), -448, 448)).
// Every value is read once and held in registers between the search for the largest and the
// rounding.  Memory bound: an entry is 2 (or 4) bytes in and 1 out.  17408 x 4096 of bf16 (216 MB)
// 36.4 us, 5.9 TB/s, 0.89 of the measured copy rate, of float32 57.0; 8 x 4096 2.0 us, a launch; a weight of
// 12288 x 4096 in blocks of 128 x 128 38.2 us (151 MB).
#include <algorithm>

#include "e4m3.cuh"

namespace ssd {

namespace {

constexpr int kGroup = 128;     // columns of a scale
constexpr int kThreads = 256;
constexpr int kLanes = 8;       // of a row's 128 columns, 16 each
constexpr int kAcross = 4;      // scales that a warp's row spans

// 16 values of a row from column c on (0 from column K on), as they lie in memory.
template <typename T>
struct Piece {
  static constexpr int N = sizeof(T);  // 16-byte pieces
  uint4 w[N];
  __device__ __forceinline__ void load(const T* row, int32_t c, int32_t K) {
    if (c + 16 <= K) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __ldcs(reinterpret_cast<const uint4*>(row + c) + i);
      return;
    }
    uint32_t v[4 * N];
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
      v[i] = 0;
      if constexpr (sizeof(T) == 4) {
        if (c + i < K) v[i] = reinterpret_cast<const uint32_t*>(row)[c + i];
      } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
        if (c + 2 * i < K) v[i] = p[c + 2 * i];
        if (c + 2 * i + 1 < K) v[i] |= (uint32_t)p[c + 2 * i + 1] << 16;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  }
  __device__ __forceinline__ void values(float (&x)[16]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[4 * i] = __uint_as_float(w[i].x), x[4 * i + 1] = __uint_as_float(w[i].y);
        x[4 * i + 2] = __uint_as_float(w[i].z), x[4 * i + 3] = __uint_as_float(w[i].w);
      }
    } else {
      float y[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        unpack8(w[i], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[8 * i + e] = y[e];
      }
    }
  }
  // The largest finite magnitude.
  __device__ __forceinline__ float most() const {
    float x[16], m = 0.f;
    values(x);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (fabsf(x[e]) < INFINITY) m = fmaxf(m, fabsf(x[e]));  // (false for NaN)
    return m;
  }
  __device__ __forceinline__ void store(uint8_t* row, int32_t c, int32_t K, float inv) const {
    float x[16];
    values(x);
    const uint2 a = to_e4m3x8(x, inv), b = to_e4m3x8(x + 8, inv);
    if (c + 16 <= K) {
      *reinterpret_cast<uint4*>(row + c) = make_uint4(a.x, a.y, b.x, b.y);
      return;
    }
    const uint32_t v[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (c + e < K) row[c + e] = (uint8_t)(v[e >> 2] >> (8 * (e & 3)));
  }
};

__device__ __forceinline__ float scale_of(float most) { return fmaxf(most, kLeast) / kTop8; }

// A scale per row: a warp takes R rows of 512 columns, all asked for at once; its lanes with the
// rows' results write them side by side.
template <typename T, int R>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(QuantizeArgs a) {
  pdl_wait();
  const int32_t lane = threadIdx.x & 31, part = lane / kLanes;
  const int32_t kb = blockIdx.y * kAcross + part, c = kb * kGroup + (lane % kLanes) * 16;
  const int64_t row0 = ((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * R;
  if (row0 >= a.rows) return;
  const T* x = static_cast<const T*>(a.x);
  uint8_t* out = static_cast<uint8_t*>(a.out);
  Piece<T> p[R];
#pragma unroll
  for (int r = 0; r < R; ++r) p[r].load(x + min(row0 + r, (int64_t)a.rows - 1) * a.ldx, c, a.K);
  float s[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float m = p[r].most();
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    s[r] = scale_of(m);
    if (row0 + r < a.rows && c < a.K) p[r].store(out + (row0 + r) * a.ldo, c, a.K, 1.0f / s[r]);
  }
  const int32_t mine = lane % kLanes;
  float v = s[0];
#pragma unroll
  for (int r = 1; r < R; ++r) v = mine == r ? s[r] : v;
  if (mine < R && row0 + mine < a.rows && kb * kGroup < a.K) a.scale[kb * a.lds + row0 + mine] = v;
}

// A scale per 128 rows: a CTA a block.
template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_blocks_kernel(QuantizeArgs a) {
  constexpr int kPasses = kGroup * kLanes / kThreads;
  __shared__ float red[kThreads / 32];
  pdl_wait();
  const int32_t c = blockIdx.y * kGroup + (threadIdx.x % kLanes) * 16;
  const int64_t row0 = (int64_t)blockIdx.x * kGroup + threadIdx.x / kLanes;
  const T* x = static_cast<const T*>(a.x);
  uint8_t* out = static_cast<uint8_t*>(a.out);
  Piece<T> p[kPasses];
  float m = 0.f;
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int64_t row = row0 + u * (kThreads / kLanes);
    p[u].load(x + min(row, (int64_t)a.rows - 1) * a.ldx, c, a.K);  // (a row twice: the same largest)
  }
#pragma unroll
  for (int u = 0; u < kPasses; ++u) m = fmaxf(m, p[u].most());
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, red[w]);
  const float s = scale_of(m), inv = 1.0f / s;
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int64_t row = row0 + u * (kThreads / kLanes);
    if (row < a.rows && c < a.K) p[u].store(out + row * a.ldo, c, a.K, inv);
  }
  if (threadIdx.x == 0) a.scale[blockIdx.y * a.lds + blockIdx.x] = s;
}

template <typename T>
cudaError_t launch(const QuantizeArgs& a, cudaStream_t stream) {
  const int32_t kb = (a.K + kGroup - 1) / kGroup;
  if (a.block_rows == kGroup)
    return launch_kernel(quantize_blocks_kernel<T>, dim3((unsigned)((a.rows + (int64_t)kGroup - 1) / kGroup), kb),
                         dim3(kThreads), 0, stream, true, a);
  constexpr int R = sizeof(T) == 2 ? 4 : 2;
  const unsigned rows = (kThreads / 32) * R;
  return launch_kernel(quantize_rows_kernel<T, R>,
                       dim3((unsigned)((a.rows + (int64_t)rows - 1) / rows), (kb + kAcross - 1) / kAcross),
                       dim3(kThreads), 0, stream, true, a);
}

}  // namespace

cudaError_t launch_quantize(const QuantizeArgs& a, cudaStream_t stream) {
  return a.bf16 ? launch<__nv_bfloat16>(a, stream) : launch<float>(a, stream);
}

}  // namespace ssd
