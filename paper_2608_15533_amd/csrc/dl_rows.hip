// Sums of partial results, shared by the gradients of parameters.
#include "dl_rows.hpp"

namespace dl {
namespace {

// A workgroup for 64 columns.  Each of its waves takes every NW-th row, eight loads at a time (they
// wait for memory, not for each other), and the waves' sums are joined in their order.  512 rows of 256
// columns: 62 us with four waves and a load at a time.
template <int NW>
__global__ __launch_bounds__(64 * NW) void column_sum_kernel(ColumnSums p) {
  __shared__ float lds[NW][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t col = int64_t(blockIdx.x) * 64 + lane;
  const bool live = col < p.width[0] + p.width[1] + p.width[2];
  float acc = 0.0f;
  if (live) {
    constexpr int U = 8;
    const float* at = p.part + col;
    for (int64_t r = wave; r < p.rows; r += U * NW) {
      float v[U];
#pragma unroll
      for (int i = 0; i < U; ++i) v[i] = r + i * NW < p.rows ? at[(r + i * NW) * p.stride] : 0.0f;
#pragma unroll
      for (int i = 0; i < U; ++i) acc += v[i];
    }
  }
  lds[wave][lane] = acc;
  __syncthreads();
  if (wave || !live) return;
  acc = 0.0f;
#pragma unroll
  for (int i = 0; i < NW; ++i) acc += lds[i][lane];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (col >= 0 && col < p.width[k] && p.out[k]) p.out[k][col] = acc;
    col -= p.width[k];
  }
}

}  // namespace

hipError_t launch_column_sums(const ColumnSums& p, hipStream_t s) {
  const int64_t blocks = (p.width[0] + p.width[1] + p.width[2] + 63) / 64;
  if (blocks == 0) return hipSuccess;
  return p.rows >= 64 ? start_rows(&column_sum_kernel<16>, blocks, 1024, p, s)
                      : start_rows(&column_sum_kernel<4>, blocks, 256, p, s);
}

}  // namespace dl
