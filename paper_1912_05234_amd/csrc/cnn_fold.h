// Sums over the workgroups' rows of partial results.
#pragma once

#include "cnn_types.h"

namespace cnn {

// put(c, sum of partial[.][c]) for c < columns: 32 rows side by side and then those, an order that `rows` alone fixes.  (1024 rows of 2048
// columns, 8 MB that the kernel before left in the last cache, take 5 us.)
constexpr int FOLD_COLUMNS = 32, FOLD_ROWS = 32;
template <class PUT>
__global__ __launch_bounds__(FOLD_COLUMNS* FOLD_ROWS) void fold_kernel(const float* partial, int64_t rows, int64_t columns, PUT put) {
  __shared__ float sums[FOLD_ROWS][FOLD_COLUMNS];
  const int column = threadIdx.x % FOLD_COLUMNS, row = threadIdx.x / FOLD_COLUMNS;
  const int64_t c = workgroup() * FOLD_COLUMNS + column;
  float s = 0.0f;
  if (c < columns)
#pragma unroll 8
    for (int64_t r = row; r < rows; r += FOLD_ROWS) s += partial[r * columns + c];
  sums[row][column] = s;
  __syncthreads();
  if (row == 0 && c < columns) {
#pragma unroll
    for (int r = 1; r < FOLD_ROWS; ++r) s += sums[r][column];
    put(c, s);
  }
}

template <class PUT>
int fold(const float* partial, int64_t rows, int64_t columns, PUT put, hipStream_t st) {
  fold_kernel<<<grid_of((columns + FOLD_COLUMNS - 1) / FOLD_COLUMNS), FOLD_COLUMNS * FOLD_ROWS, 0, st>>>(partial, rows, columns, put);
  return launch_status();
}

}  // namespace cnn
