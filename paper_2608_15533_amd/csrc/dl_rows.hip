// Sums of partial results, shared by the gradients of parameters.
#include "dl_rows.hpp"

namespace dl {
namespace {

struct SumParams {
  const float* part;
  float* out;
  int64_t P, M, stride;
};

// A workgroup for 64 columns; four waves take every fourth row each and are joined in order.
__global__ __launch_bounds__(256) void column_sum_kernel(SumParams p) {
  __shared__ float lds[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t col = int64_t(blockIdx.x) * 64 + lane;
  float acc = 0.0f;
  if (col < p.M)
    for (int64_t r = wave; r < p.P; r += 4) acc += p.part[r * p.stride + col];
  lds[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && col < p.M)
    p.out[col] = (lds[0][lane] + lds[1][lane]) + (lds[2][lane] + lds[3][lane]);
}

}  // namespace

hipError_t launch_column_sum(const float* part, int64_t P, int64_t M, int64_t stride, float* out,
                             hipStream_t s) {
  if (M <= 0) return hipSuccess;
  const SumParams p{part, out, P, M, stride};
  return start_rows(&column_sum_kernel, (M + 63) / 64, 256, p, s);
}

}  // namespace dl
