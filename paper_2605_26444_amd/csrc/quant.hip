// Rows in 8 bits with a scale each, and the choice of the heads that multiply them.
#include "common.h"

namespace nanospec {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A wavefront a row; the row is read twice, the second time from the caches.
__global__ __launch_bounds__(256) void quantize_rows_kernel(const uint16_t* __restrict__ X, int64_t rows, int d, int8_t* __restrict__ q, float* __restrict__ scale) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const uint16_t* x = X + row * d;
  uint32_t top = 0;
  for (int c = lane * 8; c < d; c += 512) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(x + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) top = bf16_top(top, v[i]);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const uint32_t t = __shfl_xor(top, o);
    top = t > top ? t : top;
  }
  const I8Row k = i8_row(top);
  for (int c = lane * 8; c < d; c += 512) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(x + c);
    *reinterpret_cast<u32x2*>(q + row * d + c) = u32x2{i8_round4(k, v[0], v[1]), i8_round4(k, v[2], v[3])};
  }
  if (lane == 0) scale[row] = k.scale;
}

hipError_t launch_quantize_rows(const void* X, int64_t rows, int32_t d, int8_t* q, float* scale, hipStream_t s) {
  const int64_t grid = (rows + 3) / 4;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  quantize_rows_kernel<<<dim3((unsigned)grid), 256, 0, s>>>(static_cast<const uint16_t*>(X), rows, d, q, scale);
  return hipGetLastError();
}

// the hidden rows in 8 bits, and their scales
static int64_t rows_bytes(int32_t rows, int32_t d) { return ((int64_t)rows * d + 255) / 256 * 256; }

int64_t head_i8_workspace_bytes(int32_t rows, int32_t d) { return rows_bytes(rows, d) + ((int64_t)rows * 4 + 255) / 256 * 256; }

hipError_t launch_head_i8(const int8_t* W, const float* W_scale, const void* H, const int32_t* ids, const int32_t* n_dev, int32_t cap_rows, int32_t V, int32_t batch,
                          int32_t M, int32_t d, int64_t ld, float* logits, char* ws, hipStream_t s) {
  int8_t* q = reinterpret_cast<int8_t*>(ws);
  float* scale = reinterpret_cast<float*>(ws + rows_bytes(batch * M, d));
  hipError_t e = launch_quantize_rows(H, (int64_t)batch * M, d, q, scale, s);
  return e == hipSuccess ? launch_head_wide_i8(W, W_scale, q, scale, ids, n_dev, cap_rows, V, batch, M, d, ld, logits, s) : e;
}

}  // namespace nanospec
