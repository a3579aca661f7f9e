// Rotary positions for gfx950 (MI355X): every pair (x, y) of a head's first 2 P columns is turned by the angle
// p_a f_i of its token's position on the pair's axis, and grown by the factor s,
//   (x, y) -> s (x cos t - y sin t, x sin t + y cos t);
// the gradient is the transposed map, the same kernel with the sine's sign changed. q and k share one launch.
//
// Bound by memory: each element is read and written once. A thread keeps the sines and cosines of VEC pairs of one
// token in registers (16 bytes of either half of the pairs, or 32 consecutive bytes of interleaved ones) and walks over
// heads, so an angle is computed once for up to kMaxHeads heads and no table is read. The reads and writes go through strides,
// so the change from the projections' [B][N][H][d] to the attention's [B][H][N][d] costs no pass of its own. 12 + 12 heads of
// 32,760 tokens, d 128, bf16: 86 us, 4.7 TB/s; 40 + 40 heads of 75,600: 617 us, 5.0 TB/s, the rate of a copy of 1 GiB.
//
// Angles: positions times frequencies reach 2^31 radians, where 32 bits hold no fraction at all. The product is taken in
// turns in float64, its whole part dropped there, and only the rest, at most half a turn, goes to the float32 sine.

#include "rotary_launch.h"
#include "wavealign.h"

#include <algorithm>

namespace {

constexpr int kThreads = 256;
// Heads a thread walks over, at most; fewer while the launch would leave compute units empty.
constexpr int kMaxHeads = 16;
constexpr int64_t kFullThreads = 256 * 1024;  // four wavefronts a SIMD on 256 compute units
constexpr int64_t kMaxGrid = 1 << 22;

template <typename T>
struct Chunk;  // 16 bytes <-> floats
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  __device__ static void load(const float* p, float* f) {
    const float4 v = *(const float4*)p;
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  }
  __device__ static void store(float* p, const float* f) { *(float4*)p = make_float4(f[0], f[1], f[2], f[3]); }
};
template <typename T>
struct Chunk {
  static constexpr int N = 8;
  typedef T V __attribute__((ext_vector_type(8)));
  __device__ static void load(const T* p, float* f) {
    const V v = *(const V*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
  }
  __device__ static void store(T* p, const float* f) {  // one rounding, to nearest even
    V v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (T)f[i];
    *(V*)p = v;
  }
};
// one element at a time: rows that are not made of aligned 16-byte pieces
template <typename T>
struct Single {
  static constexpr int N = 1;
  __device__ static void load(const T* p, float* f) { f[0] = (float)*p; }
  __device__ static void store(T* p, const float* f) { *p = (T)f[0]; }
};

// U heads from h0 of one tensor: all reads before the first write, so the memory sees them together.
template <typename T, typename C, bool ILV, int U>
__device__ __forceinline__ void rotate_heads(const WaRotaryLaunch& a, int t, int h0, int b, int n, int unit, bool tail,
                                             const float* cs, const float* sn) {
  constexpr int V = C::N;
  const T* in = (const T*)a.in[t] + b * a.in_stride[t][0] + (int64_t)h0 * a.in_stride[t][1] + n * a.in_stride[t][2];
  T* out = (T*)a.out[t] + b * a.out_stride[t][0] + (int64_t)h0 * a.out_stride[t][1] + n * a.out_stride[t][2];
  // columns of the unit's two pieces
  const int c0 = tail || ILV ? unit * 2 * V : unit * V;
  const int c1 = tail || ILV ? c0 + V : a.pairs + c0;
  const bool second = !tail || c1 < a.head_dim;
  float x[U][2 * V];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    C::load(in + u * a.in_stride[t][1] + c0, x[u]);
    if (second) C::load(in + u * a.in_stride[t][1] + c1, x[u] + V);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!tail) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int p = ILV ? 2 * i : i, q = ILV ? p + 1 : V + i;
        const float xa = x[u][p], xb = x[u][q];
        x[u][p] = xa * cs[i] - xb * sn[i];
        x[u][q] = xa * sn[i] + xb * cs[i];
      }
    }
    C::store(out + u * a.out_stride[t][1] + c0, x[u]);
    if (second) C::store(out + u * a.out_stride[t][1] + c1, x[u] + V);
  }
}

// Thread (group of heads, b, n, unit): a unit is V pairs, or behind them 2 V columns that are copied. W: integer that
// holds the number of threads.
template <typename T, typename C, bool ILV, typename W>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const WaRotaryLaunch a, int rot_units, int units, int per,
                                                          W threads) {
  constexpr int V = C::N;
  W id = (W)blockIdx.x * kThreads + threadIdx.x;
  if constexpr (sizeof(W) == 8) id += (W)blockIdx.y * gridDim.x * kThreads;
  if (id >= threads) return;
  const int unit = (int)(id % (W)units);
  W rest = id / (W)units;
  const int n = (int)(rest % (W)a.tokens);
  rest /= (W)a.tokens;
  const int b = (int)(rest % (W)a.batch);
  const int g = (int)(rest / (W)a.batch);
  const bool tail = unit >= rot_units;

  float cs[V], sn[V];
  if (!tail) {
    double pos[3] = {(double)n, 0.0, 0.0};
    if (a.pos) {
      const int64_t row = (int64_t)(a.pos_batch == 1 ? 0 : b) * a.tokens + n;
      for (int x = 0; x < a.axes; ++x) pos[x] = (double)a.pos[(int64_t)x * a.pos_batch * a.tokens + row];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int p = unit * V + i;
      const double at = p < a.axis_end[0] ? pos[0] : p < a.axis_end[1] ? pos[1] : pos[2];
      const double turns = at * a.freq[p] * 0.15915494309189535;  // 1 / (2 pi)
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      cs[i] = c * a.cos_scale;
      sn[i] = s * a.sin_scale;
    }
  }
  const int total = a.heads[0] + a.heads[1];
  const int end = min((g + 1) * per, total);
  for (int h = g * per; h < end;) {
    const int t = h >= a.heads[0];
    const int stop = t ? end : min(end, a.heads[0]), local = t ? h - a.heads[0] : h;
    if (tail && !a.copy[t]) {
      h = stop;
    } else if (stop - h >= 4) {
      rotate_heads<T, C, ILV, 4>(a, t, local, b, n, unit, tail, cs, sn);
      h += 4;
    } else {
      rotate_heads<T, C, ILV, 1>(a, t, local, b, n, unit, tail, cs, sn);
      h += 1;
    }
  }
}

template <typename T, typename C, bool ILV>
hipError_t launch_units(const WaRotaryLaunch& a, hipStream_t stream) {
  constexpr int V = C::N;
  const int rot = a.pairs / V;
  const int tail = a.copy[0] || a.copy[1] ? (a.head_dim - 2 * a.pairs + 2 * V - 1) / (2 * V) : 0;
  const int units = rot + tail, heads = a.heads[0] + a.heads[1];
  const int64_t rows = (int64_t)a.batch * a.tokens * units;
  const int per = (int)std::min<int64_t>(kMaxHeads, std::max<int64_t>(1, rows * heads / kFullThreads));
  const int64_t threads = rows * ((heads + per - 1) / per);
  const int64_t grid = (threads + kThreads - 1) / kThreads;
  if (threads < ((int64_t)1 << 31)) {
    hipLaunchKernelGGL((rotary_kernel<T, C, ILV, uint32_t>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a, rot, units,
                       per, (uint32_t)threads);
  } else {
    // a dimension of a launch holds fewer than 2^32 threads, so rows of kMaxGrid workgroups
    const dim3 rows_of((unsigned)kMaxGrid, (unsigned)((grid + kMaxGrid - 1) / kMaxGrid));
    hipLaunchKernelGGL((rotary_kernel<T, C, ILV, uint64_t>), rows_of, dim3(kThreads), 0, stream, a, rot, units, per,
                       (uint64_t)threads);
  }
  return hipGetLastError();
}

// Whether every row of every tensor is made of 16-byte pieces that do not cross the border between rotated halves or
// between rotated and copied columns.
bool in_chunks(const WaRotaryLaunch& a, int v) {
  if (a.pairs % v || a.head_dim % v) return false;
  for (int t = 0; t < 2 && a.heads[t] > 0; ++t) {
    if ((uintptr_t)a.in[t] % 16 || (uintptr_t)a.out[t] % 16) return false;
    const int64_t size[3] = {a.batch, a.heads[t], a.tokens};
    for (int i = 0; i < 3; ++i)
      if (size[i] > 1 && (a.in_stride[t][i] % v || a.out_stride[t][i] % v)) return false;
  }
  return true;
}

template <typename T>
hipError_t launch_type(const WaRotaryLaunch& a, hipStream_t stream) {
  if (in_chunks(a, Chunk<T>::N))
    return a.interleaved ? launch_units<T, Chunk<T>, true>(a, stream) : launch_units<T, Chunk<T>, false>(a, stream);
  return a.interleaved ? launch_units<T, Single<T>, true>(a, stream) : launch_units<T, Single<T>, false>(a, stream);
}

}  // namespace

hipError_t wa_launch_rotary(const WaRotaryLaunch& a, hipStream_t stream) {
  switch (a.dtype) {
    case WA_BF16: return launch_type<__bf16>(a, stream);
    case WA_F16: return launch_type<_Float16>(a, stream);
    case WA_F32: return launch_type<float>(a, stream);
  }
  return hipErrorInvalidValue;
}
