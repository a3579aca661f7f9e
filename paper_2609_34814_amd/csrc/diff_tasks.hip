// Tasks of a masked differential-attention call. Rows (columns) of a block mask keep very different numbers of blocks; a tile that
// starts last and runs ten times the mean leaves the other compute units idle, and so does one that is longer than their share of the
// call. So tiles run longest first, and one of more blocks than the share L is computed in chunks, which another kernel joins in
// order. L follows from the call's mask alone: results do not depend on the order, but a head's may differ by the order of float32
// sums from those of a call with other heads. Blocks that kv_lens or causal hide count as kept here, so the tiles of such a call are
// dealt out less evenly than those of a mask that drops them itself; the kernels leave them out all the same.
// 6 heads of 14,040 tokens at 25% (660 tiles, 27 blocks on average, 110 the longest, L 71), d 128, values 256: forward
// 541 us longest first, 461 + 13 with chunks, dQ 687 and 565 + 5; its columns, 39 at the longest, are not cut. L is the exact share:
// at half of it the chunks' own cost (their partial results, first loads) takes back what the better fit gives.

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

// Counting sort of the chunks by length in kBins steps of the longest, longest first.
__global__ __launch_bounds__(1024) void task_kernel(int32_t* tasks, int n, int slots, int least) {
  __shared__ int start[kBins], wave_sum[16], longest, cut, chunks_out;
  __shared__ unsigned long long total;
  const int32_t* length = tasks + 4;
  int4* list = (int4*)(tasks + wa_diff_task_list(n));
  int4* cuts = (int4*)(tasks + wa_diff_cut_list(n, slots));
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  if (t == 0) {
    longest = 1;
    cut = chunks_out = 0;
    total = 0;
  }
  start[t] = 0;
  __syncthreads();
  unsigned long long sum_t = 0;
  for (int i = t; i < n; i += 1024) sum_t += length[i];
  for (int x = 32; x > 0; x >>= 1) sum_t += __shfl_xor(sum_t, x);
  if (lane == 0) atomicAdd(&total, sum_t);
  __syncthreads();
  const int share = max((int)((total + slots - 1) / slots), least);
  auto chunks_of = [&](int i) { return min((length[i] + share - 1) / share, kDiffMaxChunks); };
  auto each = [&](int i) { const int c = max(chunks_of(i), 1); return (length[i] + c - 1) / c; };  // a chunk's blocks
  for (int i = t; i < n; i += 1024) atomicMax(&longest, each(i));
  __syncthreads();
  const float scale = (float)(kBins - 1) / longest;
  auto bin = [&](int i) { return kBins - 1 - min((int)(each(i) * scale), kBins - 1); };
  for (int i = t; i < n; i += 1024) atomicAdd(&start[bin(i)], max(chunks_of(i), 1));
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
  if (t == 1023) tasks[0] = sum;
  __syncthreads();
  start[t] = sum - own;
  __syncthreads();
  for (int i = t; i < n; i += 1024) {
    const int c = max(chunks_of(i), 1), at = atomicAdd(&start[bin(i)], c);
    int first = 0;
    if (c > 1) {
      first = atomicAdd(&chunks_out, c);
      cuts[atomicAdd(&cut, 1)] = make_int4(i, c, first, 0);
    }
    for (int x = 0; x < c; ++x) list[at + x] = make_int4(i, x, c, first);
  }
  __syncthreads();
  if (t == 0) tasks[1] = cut;
}

}  // namespace

hipError_t wa_launch_diff_tasks(const WaDiffLaunch& a, bool columns, int slots, hipStream_t stream) {
  const int units = a.batch * (columns ? a.kv_heads : a.heads), n = units * (columns ? a.nb : a.mb);
  int32_t* length = a.tasks + 4;
  if (columns)
    hipLaunchKernelGGL(column_lengths_kernel, dim3((a.nb + 63) / 64, units), dim3(1024), 0, stream, a.mask,
                       (int64_t)(a.heads / a.kv_heads) * a.mb, a.nb, length);
  else
    hipLaunchKernelGGL(row_lengths_kernel, dim3((n + 3) / 4), dim3(256), 0, stream, a.mask, n, a.nb, length);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // a chunk is 1,024 tokens at least
  hipLaunchKernelGGL(task_kernel, dim3(1), dim3(1024), 0, stream, a.tasks, n, slots, 1024 / a.block);
  return hipGetLastError();
}
