// Order of the tiles of a masked differential-attention call: longest first. Rows (columns) of a block mask keep very different
// numbers of blocks; a tile that starts last and runs ten times the mean leaves the other compute units idle. The order changes when
// tiles run, never what they compute.

#include "diff_launch.h"

namespace {

constexpr int kBins = 1024;

// Kept blocks of a row of the mask, a wavefront a row.
__global__ __launch_bounds__(256) void row_lengths_kernel(const uint8_t* mask, int rows, int nb, int32_t* length) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= rows) return;
  int n = 0;
  for (int j = lane; j < nb; j += 64) n += mask[(int64_t)row * nb + j] != 0;
  for (int x = 32; x > 0; x >>= 1) n += __shfl_xor(n, x);
  if (lane == 0) length[row] = n;
}

// Kept blocks of 64 columns over `rows` rows (the mask rows of the heads of one key head, which lie one after another).
__global__ __launch_bounds__(1024) void column_lengths_kernel(const uint8_t* mask, int64_t rows, int nb, int32_t* length) {
  __shared__ int sums[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, j = blockIdx.x * 64 + lane;
  int n = 0;
  if (j < nb) {
#pragma unroll 8
    for (int64_t i = w; i < rows; i += 16) n += mask[((int64_t)blockIdx.y * rows + i) * nb + j] != 0;
  }
  sums[w][lane] = n;
  __syncthreads();
  if (w == 0 && j < nb) {
    for (int x = 1; x < 16; ++x) n += sums[x][lane];
    length[(int64_t)blockIdx.y * nb + j] = n;
  }
}

// Counting sort by length in kBins steps of the longest, longest first.
__global__ __launch_bounds__(1024) void sort_kernel(const int32_t* length, int n, int32_t* order) {
  __shared__ int start[kBins], wave_sum[16], longest;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if (t == 0) longest = 1;
  start[t] = 0;
  __syncthreads();
  for (int i = t; i < n; i += 1024) atomicMax(&longest, length[i]);
  __syncthreads();
  const float scale = (float)(kBins - 1) / longest;
  auto bin = [&](int i) { return kBins - 1 - min((int)(length[i] * scale), kBins - 1); };
  for (int i = t; i < n; i += 1024) atomicAdd(&start[bin(i)], 1);
  __syncthreads();
  const int own = start[t];
  int sum = own;  // inclusive scan over the bins
  for (int x = 1; x < 64; x <<= 1) {
    const int below = __shfl_up(sum, x);
    if (lane >= x) sum += below;
  }
  if (lane == 63) wave_sum[w] = sum;
  __syncthreads();
  for (int x = 0; x < w; ++x) sum += wave_sum[x];
  __syncthreads();
  start[t] = sum - own;
  __syncthreads();
  for (int i = t; i < n; i += 1024) order[atomicAdd(&start[bin(i)], 1)] = i;
}

}  // namespace

hipError_t wa_launch_diff_order(const WaDiffLaunch& a, bool columns, hipStream_t stream) {
  const int units = a.batch * (columns ? a.kv_heads : a.heads), n = units * (columns ? a.nb : a.mb);
  int32_t* length = a.order + n;
  if (columns)
    hipLaunchKernelGGL(column_lengths_kernel, dim3((a.nb + 63) / 64, units), dim3(1024), 0, stream, a.mask,
                       (int64_t)(a.heads / a.kv_heads) * a.mb, a.nb, length);
  else
    hipLaunchKernelGGL(row_lengths_kernel, dim3((n + 3) / 4), dim3(256), 0, stream, a.mask, n, a.nb, length);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(sort_kernel, dim3(1), dim3(1024), 0, stream, length, n, a.order);
  return hipGetLastError();
}
