// The second step of sums over all rows: the partial rows that the workgroups of a first pass left (norm, linear).
#pragma once

#include "dgc_internal.h"

namespace dgc {
namespace {

// Partial rows [parts][n] -> their columns' sums, the first `split` of them to a and the others to b (nullptr: not wanted): 16 columns a
// workgroup, 64 partial rows at a time, in double.  7 us for 1024 rows of 512.
__global__ __launch_bounds__(1024) void k_join_columns(const float* partial, int64_t parts, int32_t n, int32_t split, float* a, float* b) {
  __shared__ double lds[64][16];
  const int c = threadIdx.x & 15, p = threadIdx.x >> 4;
  const int64_t col = (int64_t)blockIdx.x * 16 + c;
  double s = 0.;
  if (col < n) {
    for (int64_t k = p; k < parts; k += 64) s += (double)partial[k * n + col];
  }
  lds[p][c] = s;
  __syncthreads();
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    if (p < m) lds[p][c] += lds[p + m][c];
    __syncthreads();
  }
  if (p == 0 && col < n) {
    float* to = col < split ? a : b;
    if (to) to[col < split ? col : col - split] = (float)lds[0][c];
  }
}
void join_columns(const float* partial, int64_t parts, int32_t n, int32_t split, float* a, float* b, hipStream_t st) {
  hipLaunchKernelGGL(k_join_columns, (unsigned)((n + 15) / 16), 1024, 0, st, partial, parts, n, split, a, b);
}

}  // namespace
}  // namespace dgc
