// Rows in 8 bits with a scale each, and the choice of the heads that multiply them.
#include "common.h"

namespace nanospec {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// WPR wavefronts (1 or 4) a row, which holds what they can of it -- 32 numbers a lane -- in registers and reads the rest again, from the caches.
template <int WPR>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const uint16_t* __restrict__ X, int64_t rows, int d, int8_t* __restrict__ q, float* __restrict__ scale) {
  static_assert(WPR == 1 || WPR == 4, "a row's wavefronts meet in a barrier, or there is one");
  constexpr int P = 4, STEP = 512 * WPR;
  const int tid = threadIdx.x, at = tid % (64 * WPR);
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, row = WPR == 4 ? block : block * 4 + tid / 64;
  if (row >= rows) return;
  const uint16_t* x = X + row * d;
  u32x4 v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int c = at * 8 + i * STEP;
    v[i] = *reinterpret_cast<const u32x4*>(x + (c < d ? c : 0));          // past the end a copy of the row's first
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = bf16_tops(top, v[i][e]);
  for (int c = at * 8 + P * STEP; c < d; c += STEP) {
    const u32x4 y = *reinterpret_cast<const u32x4*>(x + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = bf16_tops(top, y[e]);
  }
  top = wave_top(top);
  if (WPR > 1) {
    __shared__ uint32_t tops[WPR];
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WPR; ++i) top = tops[i] > top ? tops[i] : top;
  }
  const I8Row k = i8_row(top);
  auto put = [&](auto tiny) {
    auto one = [&](int c, const u32x4 y) {
      constexpr bool T = decltype(tiny)::value;
      *reinterpret_cast<u32x2*>(q + row * d + c) = u32x2{i8_round4<T>(k, y[0], y[1]), i8_round4<T>(k, y[2], y[3])};
    };
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = at * 8 + i * STEP;
      if (c < d) one(c, v[i]);
    }
    for (int c = at * 8 + P * STEP; c < d; c += STEP) one(c, *reinterpret_cast<const u32x4*>(x + c));
  };
  if (k.p == 1.f) put(Flag<false>());
  else put(Flag<true>());
  if (at == 0) scale[row] = k.scale;
}

// One wavefront for rows that it holds, else four (us, 1 / 4 / 16 wavefronts: 8 x 4096 3.6 / 2.5 / 2.7, 1024 x 4096 5.5 / 4.3 / 6.4, 512 x 2048 2.6 / 2.7 / 3.6, 32000 x 512 13 / 27 / 104,
// 128256 x 4096 301 / 259 / 550: 6.1 TB/s read and written, 16 x 8192 6.1 / 2.6 / 2.9).
hipError_t launch_quantize_rows(const void* X, int64_t rows, int32_t d, int8_t* q, float* scale, hipStream_t s) {
  const uint16_t* x = static_cast<const uint16_t*>(X);
  const int64_t blocks = d <= 2048 ? (rows + 3) / 4 : rows, line = blocks < (1 << 20) ? blocks : 1 << 20;      // a launch has less than 2^32 threads along x
  const dim3 grid((unsigned)line, (unsigned)((blocks + line - 1) / line));
  if (d <= 2048) quantize_rows_kernel<1><<<grid, 256, 0, s>>>(x, rows, d, q, scale);
  else quantize_rows_kernel<4><<<grid, 256, 0, s>>>(x, rows, d, q, scale);
  return hipGetLastError();
}

// the hidden rows in 8 bits, and their scales
static int64_t rows_bytes(int32_t rows, int32_t d) { return ((int64_t)rows * d + 255) / 256 * 256; }

int64_t head_i8_workspace_bytes(int32_t rows, int32_t d) { return rows_bytes(rows, d) + ((int64_t)rows * 4 + 255) / 256 * 256; }

hipError_t launch_head_i8(const int8_t* W, const float* W_scale, const void* H, const int32_t* ids, const int32_t* n_dev, int32_t cap_rows, int32_t V, int32_t batch,
                          int32_t M, int32_t d, int64_t ld, float* logits, char* ws, hipStream_t s) {
  const bool few = few_supported(M, d);
  if (few && few_rounds(M, d)) return launch_head_few_i8(W, W_scale, H, nullptr, nullptr, ids, n_dev, cap_rows, V, batch, M, d, ld, logits, s);
  int8_t* q = reinterpret_cast<int8_t*>(ws);
  float* scale = reinterpret_cast<float*>(ws + rows_bytes(batch * M, d));
  hipError_t e = launch_quantize_rows(H, (int64_t)batch * M, d, q, scale, s);
  if (e == hipSuccess && few) return launch_head_few_i8(W, W_scale, nullptr, q, scale, ids, n_dev, cap_rows, V, batch, M, d, ld, logits, s);
  return e == hipSuccess ? launch_head_wide_i8(W, W_scale, q, scale, ids, n_dev, cap_rows, V, batch, M, d, ld, logits, s) : e;
}

}  // namespace nanospec
