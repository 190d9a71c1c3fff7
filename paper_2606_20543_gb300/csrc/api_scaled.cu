// api_scaled.cu — the extern "C" entry points of the 8-bit products (include/ssd.h): host-side
// argument checks and launches on the caller's stream.  No allocation, no synchronisation.
#include "kernels.cuh"

using namespace ssd;

namespace {

ssd_status from_cuda(cudaError_t e) { return e == cudaSuccess ? SSD_OK : SSD_ERR_CUDA; }

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int32_t kScaleGroup = 128;  // entries of a scale

}  // namespace

extern "C" {

ssd_status ssd_quantize(int32_t rows, int32_t K, int32_t block_rows, const void* x, int32_t x_bf16,
                        int64_t ldx, void* out, int64_t ldo, float* scale, int64_t lds,
                        ssd_stream_t stream) {
  if (rows < 0 || K <= 0 || block_rows <= 0) return SSD_ERR_SHAPE;
  if (block_rows != 1 && block_rows != kScaleGroup) return SSD_ERR_UNSUPPORTED;
  if (x_bf16 != 0 && x_bf16 != 1) return SSD_ERR_INVALID_ARG;
  if (ldx < K || ldo < K || lds < ((int64_t)rows + block_rows - 1) / block_rows) return SSD_ERR_SHAPE;
  if (ldx % 8 != 0 || ldo % 16 != 0) return SSD_ERR_SHAPE;
  if (K > kScaleGroup * 65535) return SSD_ERR_UNSUPPORTED;
  if (rows == 0) return SSD_OK;
  if (x == nullptr || out == nullptr || scale == nullptr) return SSD_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(out, 16) || !aligned(scale, 4)) return SSD_ERR_INVALID_ARG;
  QuantizeArgs a{};
  a.rows = rows;
  a.K = K;
  a.block_rows = block_rows;
  a.x = x;
  a.bf16 = x_bf16;
  a.ldx = ldx;
  a.out = out;
  a.ldo = ldo;
  a.scale = scale;
  a.lds = lds;
  return from_cuda(launch_quantize(a, (cudaStream_t)stream));
}

ssd_status ssd_scaled_matmul(int32_t M, int32_t N, int32_t K, const void* a, int64_t lda,
                             const float* a_scale, int64_t ldas, const void* w, int64_t ldw,
                             const float* w_scale, int64_t ldws, const void* add, int64_t ldadd,
                             void* c, int32_t c_bf16, int64_t ldc, int32_t* status,
                             ssd_stream_t stream) {
  if (M < 0 || N <= 0 || K <= 0) return SSD_ERR_SHAPE;
  if (c_bf16 != 0 && c_bf16 != 1) return SSD_ERR_INVALID_ARG;
  if (lda < K || ldw < K || ldc < N || ldas < M || ldws < ((int64_t)N + kScaleGroup - 1) / kScaleGroup)
    return SSD_ERR_SHAPE;
  if (lda % 16 != 0 || ldw % 16 != 0 || (add != nullptr && ldadd < N)) return SSD_ERR_SHAPE;
  if (M > INT32_MAX / 2 || N > INT32_MAX / 2 || K > INT32_MAX / 2) return SSD_ERR_UNSUPPORTED;
  // what a tensor map can hold, and what 32-bit counts of tiles can
  if (lda >= (int64_t)1 << 40 || ldw >= (int64_t)1 << 40) return SSD_ERR_UNSUPPORTED;
  if (((int64_t)M / 128 + 1) * ((int64_t)N / 64 + 1) > INT32_MAX / 32) return SSD_ERR_UNSUPPORTED;
  if (M == 0) return SSD_OK;
  for (const void* p : {a, w, (const void*)a_scale, (const void*)w_scale, (const void*)c,
                        (const void*)status})
    if (p == nullptr) return SSD_ERR_INVALID_ARG;
  if (!aligned(a, 16) || !aligned(w, 16) || !aligned(a_scale, 4) || !aligned(w_scale, 4) ||
      !aligned(add, 2) || !aligned(c, c_bf16 ? 2 : 4))
    return SSD_ERR_INVALID_ARG;
  ScaledMatmulArgs x{};
  x.M = M;
  x.N = N;
  x.K = K;
  x.a = a;
  x.lda = lda;
  x.a_scale = a_scale;
  x.ldas = ldas;
  x.w = w;
  x.ldw = ldw;
  x.w_scale = w_scale;
  x.ldws = ldws;
  x.add = add;
  x.ldadd = ldadd;
  x.c = c;
  x.c_bf16 = c_bf16;
  x.ldc = ldc;
  x.status = status;
  return from_cuda(launch_scaled_matmul(x, (cudaStream_t)stream));
}

}  // extern "C"
