// Sums over partial rows (column_sum): gradients of weights that every workgroup of a backward pass has a part of.  A
// workgroup takes 16 columns (64 bytes of a row) and 64 rows at a time, so that a handful of columns still has its rows
// asked for in parallel; a sum of 1,024 rows is 16 loads deep.  768 rows of 8,192 columns: 9 us, 2.7 TB/s out of the caches;
// 1,024 rows of 200: 4 us, a launch.
#include "ops_device.h"

namespace tgnn {

__global__ __launch_bounds__(1024) void column_sum_kernel(ColumnSum a) {
  __shared__ double parts[16][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m = (int64_t)group_number() * 16 + (threadIdx.x & 15);
  double sum = 0.0;
  if (m < a.cols) {
#pragma unroll 4
    for (int p = threadIdx.x >> 4; p < a.n_part; p += 64) sum += (double)a.part[(int64_t)p * a.cols + m];
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (lane < 16) parts[wave][lane] = sum;
  __syncthreads();
  if (threadIdx.x >= 16 || m >= a.cols) return;
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += parts[w][threadIdx.x];
  int64_t i = m;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    if (i >= 0 && i < a.c[k] && a.out[k] != nullptr) a.out[k][i] = (float)(a.accumulate ? (double)a.out[k][i] + sum : sum);
    i -= a.c[k];
  }
}

void column_sum(const ColumnSum& a, hipStream_t s) {
  if (a.cols <= 0) return;
  hipLaunchKernelGGL(column_sum_kernel, group_grid((a.cols + 15) / 16, 1024), dim3(1024), 0, s, a);
}

}  // namespace tgnn
