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

}  // extern "C"
