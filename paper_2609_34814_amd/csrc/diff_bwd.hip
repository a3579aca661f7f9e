// Gradient of differential attention for gfx950 (MI355X). With P_m recomputed from the forward's log-sum-exps,
//   dP = dO V^T,   D_m = sum_j P_m dP = dO . O_m,   dS_1 = P_1 (dP - D_1),   dS_2 = -lam P_2 (dP - D_2),
//   dQ_m = scale dS_m K_m,   dK_m = scale dS_m^T Q_m,   dV = (P_1 - lam P_2)^T dO,   dlam_h = -sum D_2.
//
// Two kernels, each owning what it writes, so nothing is added with atomics and equal calls give equal bits:
//   diff_dq_kernel: a tile of queries, over its keys; also writes D_m and the tile's part of dlam.
//   diff_dkv_kernel: a tile of keys, over the queries of all heads that share it.
// Both recompute the scores and dP; dP and the product with dO serve both maps. A wavefront holds 32 queries (keys) of both
// maps with their accumulators in registers (for d 128 one wavefront a SIMD, which may use 512), and the other side's tiles pass
// through LDS, copied one ahead. Scores come out with the wavefront's own index in the lanes and the other in the
// registers, so P and dS, rounded to bf16, are operands of the following products as they are.
// dlam is the sum of D_2 from the stored maps and of the float32 P_2 (dP - D_2), which takes their steps' error back: over a
// lane's keys with the roundings carried along, over queries in float64.
// What bounds it (d 128, values 256, 2 x 8 heads of 4,096 tokens): dQ 437 and dK with dV 583 us where each runs alone at 2.3 GHz
// (matrix cores 40% busy; a wavefront issues 55% of its time, waits 20% for the matrix core and 25% for LDS, copies and barriers),
// 514 and 728 one after another, when the power limit lowers the clock. One map a wavefront, so that two share a SIMD, makes a
// fifth to a third more products (dP twice) and is no faster.

#include "diff_tiles.h"
#include "wavealign.h"

#include <algorithm>

namespace {

using namespace wa;

template <int D, int DV, int W, bool SMALL = false>
struct Bwd {
  // Tokens of a passing tile: 64 with four wavefronts, 32 with two (two workgroups share a compute unit's LDS) or where the
  // own side takes LDS too.
  static constexpr int TB = W == 4 && !SMALL ? 64 : 32;
  static constexpr int KRB = D * 2, VRB = DV * 2;
  static constexpr int KBYTES = TB * KRB, VBYTES = TB * VRB, STAGE = 2 * KBYTES + VBYTES;
  static constexpr int DT = D / 32, VT = DV / 32, KS = D / 16, VS = DV / 16;
};
// Operands read ahead of their products, and a fence that keeps the order of the code where a wavefront has its SIMD to itself: the
// scheduler would sink each read to its product. With two wavefronts a SIMD the one hides the other's waits, and registers
// of operands in flight would spill (dK and dV of 2 x 14 heads of 4,096 tokens, d 64, values 128: 646 us with 2, 723 with 3,
// 996 with 4; 788 with one wavefront a SIMD).
template <int WAVES>
constexpr int kAheadRows = WAVES == 1 ? 6 : 2;
template <int WAVES>
constexpr int kAheadCols = WAVES == 1 ? 4 : 2;
template <int WAVES>
__device__ __forceinline__ void in_order() {
  if constexpr (WAVES == 1) WA_SCHED_FENCE();
}
// Wavefronts a SIMD: two share its 512 registers a lane where both hold their accumulators.
template <int D>
constexpr int kDqWaves = D == 64 ? 2 : 1;
template <int D>
constexpr int kDkvWaves = D == 64 ? 2 : 1;

__device__ __forceinline__ void fill(f32x16& x, float f) {
#pragma unroll
  for (int v = 0; v < 16; ++v) x[v] = f;
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Products whose results the vector unit reads. A kernel of one wavefront a SIMD has its accumulators in the 256 accumulation
// registers, and the compiler puts every product's result there: the scores and dP would be moved out one by one, and where the
// accumulators fill them (d 128, values 256) three of those to and fro as well, 96 moves beside 64 products. Written out, these
// results are in vector registers (dK and dV of 2 x 8 heads of 4,096 tokens, d 128, values 256: 670 -> 619 us; values 128, 16 heads:
// 1,033 -> 1,011; dQ 860 -> 846). The compiler does not see these products' latency: two wait states stand before each, for an
// operand that the vector unit has just written, and settled() has to stand before a result is read (12 states, 8 passes).
template <int WAVES, bool ZERO>
__device__ __forceinline__ void product(bf16x8 a, bf16x8 b, f32x16& c) {
  if constexpr (WAVES > 1) {
    if constexpr (ZERO) fill(c, 0.f);
    c = mfma(a, b, c);
  } else if constexpr (ZERO) {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "v"(b));
  } else {
    asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+&v"(c) : "v"(a), "v"(b));
  }
}
template <int WAVES>
__device__ __forceinline__ void settled(f32x16& c) {
  if constexpr (WAVES == 1) asm volatile("s_nop 11" : "+v"(c));
}
template <int WAVES>
__device__ __forceinline__ void settled(f32x16& c, f32x16& d) {
  if constexpr (WAVES == 1) asm volatile("s_nop 11" : "+v"(c), "+v"(d));
}
// Registers 8 s to 8 s + 7 of a product as an operand over its rows.
__device__ __forceinline__ bf16x8 pack8(const float* p) {
  return as_bf16x8(make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])));
}
__device__ __forceinline__ float dot8(bf16x8 a, uint4 b, float sum) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 n = __builtin_bit_cast(s16x8, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = __builtin_fmaf((float)a[i], (float)n[i], sum);
  return sum;
}
__device__ __forceinline__ bf16x8 load8(const uint16_t* p, bool ok) {
  uint4 u = make_uint4(0, 0, 0, 0);
  if (ok) u = *(const uint4*)p;
  return as_bf16x8(u);
}
// acc (rows: columns of the output) to the lane's output row, times f
template <int T>
__device__ __forceinline__ void store_row(uint16_t* out, const f32x16 (&acc)[T], float f, int hf) {
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      *(uint2*)(out + t * 32 + 2 * v + 4 * hf) =
          make_uint2(pack_bf16x2(acc[t][v] * f, acc[t][v + 1] * f), pack_bf16x2(acc[t][v + 2] * f, acc[t][v + 3] * f));
}

// the same unrounded, as a row of a part's result
template <int T>
__device__ __forceinline__ void store_part(float* out, const f32x16 (&acc)[T], float f, int hf) {
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      *(float4*)(out + t * 32 + 2 * v + 4 * hf) = make_float4(acc[t][v] * f, acc[t][v + 1] * f, acc[t][v + 2] * f, acc[t][v + 3] * f);
}

template <int D, int DV, int W>
__global__ __launch_bounds__(64 * W, kDqWaves<D>) void diff_dq_kernel(const WaDiffLaunch a, const WaDiffSide n) {
  using C = Bwd<D, DV, W>;
  constexpr int KB = C::TB, AHEAD = kAheadRows<kDqWaves<D>>, CAHEAD = kAheadCols<kDqWaves<D>>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * C::STAGE];
  __shared__ double lam_sum[W];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Task task;
  if (!take_task<kDqWaves<D>>(a, n.tiles, a.batch * a.heads, n.parts, a.causal, &task)) return;
  const int bh = task.unit, tile = task.tile, b = bh / a.heads, h = bh % a.heads, hk = h / (a.heads / a.kv_heads);
  const int i0 = tile * 32 * W + w * 32, i = i0 + l32, i_last = a.q_len - 1;
  const bool valid = i <= i_last;
  const int start = start_of(a, b), keys = keys_of(a, b, start);
  const int limit = valid ? key_limit(a, keys, start, i) : 0;
  const int some = i0 > i_last ? 0 : key_limit(a, keys, start, min(i0 + 31, i_last));
  const int all = key_limit(a, keys, start, min(i0, i_last));
  const int most = key_limit(a, keys, start, min(tile * 32 * W + 32 * W - 1, i_last));

  const unsigned char* kg = (const unsigned char*)a.k + (((int64_t)b * 2 * a.kv_heads + 2 * hk) * a.kv_len) * C::KRB;
  const unsigned char* vg = (const unsigned char*)a.v + (((int64_t)b * a.kv_heads + hk) * a.kv_len) * C::VRB;
  MaskWalk walk;
  const int shift = a.block == 128 ? 7 : 6;
  if (a.mask) {
    walk.at = uniform_ptr(a.mask + ((int64_t)bh * a.mb + (tile * 32 * W >> shift)) * a.nb);
  }
  int lo, hi;  // this workgroup's keys
  chunk_keys<KB>(a, task, walk, most, lane, &lo, &hi);
  walk.entries = (hi + a.block - 1) >> shift;
  auto next_tile = [&](int key) {
    if (!a.mask || (key & (a.block - 1))) return key;
    return walk.next(key >> shift, lane) << shift;
  };
  auto copy = [&](int key, int buf) {
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));  // nor those of the copies
    const unsigned char* t = lds + buf * C::STAGE;
    copy_tile<C::KRB, KB, W>(t, kg, key, keys - 1, w, lane_o);
    copy_tile<C::KRB, KB, W>(t + C::KBYTES, kg + (int64_t)a.kv_len * C::KRB, key, keys - 1, w, lane_o);
    copy_tile<C::VRB, KB, W>(t + 2 * C::KBYTES, vg, key, keys - 1, w, lane_o);
  };
  int key = lo < hi ? next_tile(lo) : hi, buf = 0;
  if (key < hi) copy(key, 0);

  // the wavefront's queries, their dO, and D_m
  bf16x8 qf[2][C::KS], dof[C::VS];
  const int64_t row0 = ((int64_t)b * 2 * a.heads + 2 * h) * a.q_len + i, row = ((int64_t)bh * a.q_len + i) * DV;
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
#pragma unroll
    for (int m = 0; m < 2; ++m)
      qf[m][s] = load8((const uint16_t*)a.q + (row0 + (int64_t)m * a.q_len) * D + 16 * s + 8 * hf, valid);
  float d[2] = {0.f, 0.f};
#pragma unroll
  for (int s = 0; s < C::VS; ++s) {
    dof[s] = load8((const uint16_t*)a.dout + row + 16 * s + 8 * hf, valid);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (valid) u = *(const uint4*)(a.maps + (row0 + (int64_t)m * a.q_len) * DV + 16 * s + 8 * hf);
      d[m] = dot8(dof[s], u, d[m]);
    }
  }
  // For the side of the keys: what its products start from, scores from the log-sum-exp, so that P_m = exp2(c2 s), and dP from
  // -D_1; and D_1 - D_2.
  const float c2 = a.scale * kLog2e;
  float ref[2] = {0.f, 0.f}, factor = 1.f;  // ref: log-sum-exp in log2 units
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    d[m] = add_halves(d[m]);
    if (valid) {
      const float* st = a.stats + 3 * (row0 + (int64_t)m * a.q_len);
      ref[m] = st[0] * kLog2e;
      d[m] *= st[1];
      factor = st[2];  // of the second map, in the end
    }
  }
  if (valid && hf == 0 && task.chunk == 0) {
    float* to = a.rows + (int64_t)bh * 4 * a.q_len + i;
    to[0] = -ref[0] / c2;
    to[a.q_len] = -ref[1] / c2;
    to[2 * (int64_t)a.q_len] = -d[0];
    to[3 * (int64_t)a.q_len] = d[0] - d[1];
  }
  const float lam = a.lam[h];

  const uint32_t k_row = row_operand<C::KRB>(lane, 0), v_row = 2 * C::KBYTES + row_operand<C::VRB>(lane, 0);
  const uint32_t k_col0 = col_operand<C::KRB>(lane, 0, 0), k_col1 = col_operand<C::KRB>(lane, 0, 1);

  f32x16 dq[2][C::DT];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int c = 0; c < C::DT; ++c) fill(dq[m][c], 0.f);
  float lam_dot = 0.f, lam_lost = 0.f;

  // 32 keys; masked: this lane's query sees only `rest` of them, counted from its first register's.
  auto work = [&](uint32_t t, uint32_t tv, bool masked, int rest) {
    // The tile's place is added before the steps, one exclusive or each; opaque, so that the offsets of all operands are not held
    // across the loop.
    uint32_t kr = k_row + t, vr = v_row + tv, kc0 = k_col0 + t, kc1 = k_col1 + t;
    asm volatile("" : "+v"(kr), "+v"(vr), "+v"(kc0), "+v"(kc1));
    auto row = [&](int x) {  // operand of product x of the scores, then of dP
      const int y = x - 2 * C::KS;
      return x < 2 * C::KS ? read_row(lds + row_step(kr, x >> 1) + (x & 1) * C::KBYTES) : read_row(lds + row_step(vr, y & 7) + (y >> 3) * 256);
    };
    auto col = [&](int x) {  // operand of product x of dQ: 16 keys, map, 32 columns
      const int at = (x / C::DT & 1) * C::KBYTES + 16 * (x / (2 * C::DT)) * C::KRB;
      return read_cols(lds + col_step(kc0, x % C::DT) + at, lds + col_step(kc1, x % C::DT) + at);
    };
    constexpr int ROWS = 2 * C::KS + C::VS, COLS = 4 * C::DT;
    f32x16 s[2], dp;
    constexpr int WV = kDqWaves<D>;
    float p[2][16];
    bf16x8 ring[AHEAD];
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) ring[x] = row(x);
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      in_order<kDqWaves<D>>();
      if (x < 2)
        product<WV, true>(ring[x % AHEAD], qf[x & 1][x >> 1], s[x & 1]);
      else if (x < 2 * C::KS)
        product<WV, false>(ring[x % AHEAD], qf[x & 1][x >> 1], s[x & 1]);
      else if (x == 2 * C::KS)
        product<WV, true>(ring[x % AHEAD], dof[x - 2 * C::KS], dp);
      else
        product<WV, false>(ring[x % AHEAD], dof[x - 2 * C::KS], dp);
      if (x == 2 * C::KS) settled<WV>(s[0], s[1]);
      if (x + AHEAD < ROWS) ring[x % AHEAD] = row(x + AHEAD);
      if (x >= 2 * C::KS) {  // the exponentials run beside the products of dP
        constexpr int PER = 32 / C::VS;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int v = (x - 2 * C::KS) * PER + e;
          p[v >> 4][v & 15] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v >> 4][v & 15], c2, -ref[v >> 4]));
        }
      }
    }
    bf16x8 cring[CAHEAD];
#pragma unroll
    for (int x = 0; x < CAHEAD; ++x) cring[x] = col(x);
    settled<WV>(dp);
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + (v & 3) >= rest) p[0][v] = p[1][v] = 0.f;
    }
    float dot = 0.f;
    auto dscore = [&](int m, int v) {
      p[m][v] *= dp[v] - d[m];
      if (m) dot += p[m][v];
    };
    bf16x8 ds[2];
#pragma unroll
    for (int v = 0; v < 8; ++v) dscore(0, v);
    ds[0] = pack8(p[0]);
#pragma unroll
    for (int v = 0; v < 8; ++v) dscore(1, v);
    ds[1] = pack8(p[1]);
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      in_order<kDqWaves<D>>();
      const int m = x / C::DT & 1;
      if (x == 2 * C::DT) ds[0] = pack8(p[0] + 8);
      if (x == 3 * C::DT) ds[1] = pack8(p[1] + 8);
      dq[m][x % C::DT] = mfma(cring[x % CAHEAD], ds[m], dq[m][x % C::DT]);
      if (x + CAHEAD < COLS) cring[x % CAHEAD] = col(x + CAHEAD);
      if (x < 2 * C::DT) {  // dS of the second 16 keys beside the products of the first
        constexpr int PER = 16 / (2 * C::DT);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int v = x * PER + e;
          dscore(v >> 3, 8 + (v & 7));
        }
      }
    }
    in_order<kDqWaves<D>>();
    const float add = dot - lam_lost, grown = lam_dot + add;
    lam_lost = (grown - lam_dot) - add;
    lam_dot = grown;
  };
  while (key < hi) {
    const int next = next_tile(key + KB);
    WA_WAIT_VM(0);
    WA_BARRIER();
    if (next < hi) copy(next, buf ^ 1);
    int end = KB;
    asm volatile("" : "+s"(end));
#pragma unroll 1
    for (int half = 0; half < end; half += 32) {
      if (key + half >= some) break;
      work(buf * C::STAGE + half * C::KRB, buf * C::STAGE + half * C::VRB, key + half + 32 > all, limit - key - half - 4 * hf);
    }
    key = next;
    buf ^= 1;
  }
  if (task.chunks > 1) {
    float* to = a.part + (task.part * 32 * W + w * 32 + l32) * 2 * D;
    store_part(to, dq[0], a.scale, hf);
    store_part(to + D, dq[1], -lam * a.scale, hf);
  } else if (valid) {
    store_row(((uint16_t*)a.dq) + row0 * D, dq[0], a.scale, hf);
    store_row(((uint16_t*)a.dq) + (row0 + a.q_len) * D, dq[1], -lam * a.scale, hf);
  }
  // sum_j P_2 (dP - D_2), which the stored maps' steps leave of their D_2 (the sum of P_2 is 1), and that D_2
  double lam_row = (double)lam_dot * factor + (valid && hf == 0 && task.chunk == 0 ? (double)d[1] : 0.0);
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) lam_row += __shfl_xor(lam_row, x);
  if (lane == 0) lam_sum[w] = lam_row;
  __syncthreads();
  if (tid == 0) {
    double sum = 0.0;
    for (int x = 0; x < W; ++x) sum += lam_sum[x];
    // of listed tasks, kDiffMaxChunks a tile, 0 past its chunks
    double* to = a.lam_part + task.item * (a.tasks ? kDiffMaxChunks : n.parts);
    to[task.chunk] = sum;
    if (a.tasks && task.chunk == 0)
      for (int x = task.chunks; x < kDiffMaxChunks; ++x) to[x] = 0.0;
  }
}

// One 4-byte-a-lane copy from global memory into LDS at the uniform address lds (lane i writes lds + 4 i).
__device__ __forceinline__ void dma4(const void* gbase, uint32_t voff, const unsigned char* lds) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)lds);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(m0), "v"(voff), "s"(gbase)
      : "memory");
}

template <int D, int DV, int W>
__global__ __launch_bounds__(64 * W, kDkvWaves<D>) void diff_dkv_kernel(const WaDiffLaunch a, const WaDiffSide n, int lam_parts) {
  // Values lie in LDS where, with the keys and the sums of dK and dV, they do not fit the registers: twice the keys' columns, unless
  // 256 of them leave two wavefronts a workgroup too little LDS.
  constexpr bool kValuesInLds = DV == 2 * D && (DV == 128 || W == 4);
  using C = Bwd<D, DV, W, kValuesInLds>;
  constexpr int AHEAD = kAheadRows<kDkvWaves<D>>, CAHEAD = kAheadCols<kDkvWaves<D>>;
  // Keys that do not fit the registers either (d 64) lie in LDS by the lane, as many as leave a compute unit its two workgroups of four
  // wavefronts (three of two): the compiler's own spills are reloaded in the loop, which waits for the next tile's copies too (5 registers
  // of two wavefronts and one of four are left). 2 x 14 heads of 4,096 tokens, values 128: 669 -> 636 us, causal 16 heads over 4 of 2,048:
  // 120 -> 114.
  constexpr int KEPT = !kValuesInLds || D != 64 ? 0 : W == 4 ? 3 : 2;
  constexpr int QB = C::TB, VALUES = kValuesInLds ? 32 * W * C::VRB : 0;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * C::STAGE + VALUES + KEPT * 1024 * W];
  __shared__ __attribute__((aligned(1024))) float stat[2][4 * QB];  // the rows of a.rows

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // dlam: the parts that diff_dq_kernel left, in float64, in one order
  for (int h = blockIdx.x; h < a.heads; h += gridDim.x) {
    if (tid < 64) {
      double sum = 0.0;
      for (int b = 0; b < a.batch; ++b)
        for (int t = lane; t < lam_parts; t += 64) sum += a.lam_part[((int64_t)b * a.heads + h) * lam_parts + t];
      for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
      if (lane == 0) a.dlam[h] = (float)-sum;
    }
  }

  // the first tiles, which the most queries see, come first where that differs
  Task task;
  if (!take_task<kDkvWaves<D>>(a, n.tiles, a.batch * a.kv_heads, n.parts, false, &task)) return;
  const int bh = task.unit, tile = task.tile, b = bh / a.kv_heads, hk = bh % a.kv_heads, per_key_head = a.heads / a.kv_heads;
  const int start = start_of(a, b), keys = keys_of(a, b, start);
  const int k0 = tile * 32 * W + w * 32, kj = k0 + l32;
  const bool valid = kj < keys;
  // first query that sees this lane's key, the wavefront's first key, its last, the workgroup's first
  auto first_query = [&](int j) { return j >= keys ? a.q_len : a.causal ? min(max(j - start, 0), a.q_len) : 0; };
  const int from = first_query(kj);
  const int some = first_query(k0), all = first_query(min(k0 + 31, max(keys - 1, k0)));
  const bool whole = k0 + 31 < keys;
  // this chunk's tiles of queries, counted through the heads one after another: an equal number, or that of an equal number of the
  // column's kept blocks
  const int from0 = first_query(tile * 32 * W), first = from0 / QB * QB;
  const int q_tiles = from0 < a.q_len ? (a.q_len - first + QB - 1) / QB : 0;
  const int64_t all_tiles = (int64_t)per_key_head * q_tiles;
  const int shift = a.block == 128 ? 7 : 6;
  MaskWalk walk;
  int64_t t0 = all_tiles * task.chunk / task.chunks, t1 = all_tiles * (task.chunk + 1) / task.chunks;
  if (a.tasks && task.chunks > 1) {
    walk.at = uniform_ptr(a.mask + ((int64_t)b * a.heads + hk * per_key_head) * a.mb * a.nb + (tile * 32 * W >> shift));
    walk.step = a.nb;
    walk.entries = per_key_head * a.mb;  // the heads' rows lie one after another
    auto tile_of = [&](int chunk) {
      const int e = walk.nth((int)((int64_t)a.tasks[4 + task.item] * chunk / task.chunks), lane), head = e / a.mb;
      return head * (int64_t)q_tiles + min(max(((e - head * a.mb) << shift) - first, 0) / QB, q_tiles);
    };
    t0 = task.chunk > 0 ? tile_of(task.chunk) : 0;
    t1 = task.chunk + 1 < task.chunks ? tile_of(task.chunk + 1) : all_tiles;
  }

  const int64_t krow0 = ((int64_t)b * 2 * a.kv_heads + 2 * hk) * a.kv_len + kj, vrow = (int64_t)bh * a.kv_len + kj;
  bf16x8 kf[2][C::KS], vf[kValuesInLds ? 1 : C::VS];
  unsigned char* const kept_keys = lds + 2 * C::STAGE + VALUES + tid * 16;  // read by the lane that wrote it
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const bf16x8 x = load8((const uint16_t*)a.k + (krow0 + (int64_t)m * a.kv_len) * D + 16 * s + 8 * hf, valid);
      if (m && s >= C::KS - KEPT)
        *(bf16x8*)(kept_keys + (s - C::KS + KEPT) * 1024 * W) = x;
      else
        kf[m][s] = x;
    }
  unsigned char* const values = lds + 2 * C::STAGE;
  if constexpr (kValuesInLds) {
    if (q_tiles > 0)  // so there are keys; those past the last are the last again
      copy_tile<C::VRB, 32 * W, W>(values, (const unsigned char*)a.v + (int64_t)bh * a.kv_len * C::VRB, tile * 32 * W, keys - 1, w, lane);
  } else {
#pragma unroll
    for (int s = 0; s < C::VS; ++s) vf[s] = load8((const uint16_t*)a.v + vrow * DV + 16 * s + 8 * hf, valid);
  }

  const uint32_t q_row = row_operand<C::KRB>(lane, 0), o_row = 2 * C::KBYTES + row_operand<C::VRB>(lane, 0);
  const uint32_t q_col0 = col_operand<C::KRB>(lane, 0, 0), q_col1 = col_operand<C::KRB>(lane, 0, 1);
  const uint32_t o_col0 = 2 * C::KBYTES + col_operand<C::VRB>(lane, 0, 0), o_col1 = 2 * C::KBYTES + col_operand<C::VRB>(lane, 0, 1);
  const uint32_t v_row = 2 * C::STAGE + w * 32 * C::VRB + row_operand<C::VRB>(lane, 0);

  const float c2 = a.scale * kLog2e;
  f32x16 dk[2][C::DT], dv[C::VT];
#pragma unroll
  for (int c = 0; c < C::DT; ++c) {
    fill(dk[0][c], 0.f);
    fill(dk[1][c], 0.f);
  }
#pragma unroll
  for (int c = 0; c < C::VT; ++c) fill(dv[c], 0.f);

  // One loop over the tiles of all heads: head g's run from lo to hi; i is the next one's first query.
  int g = q_tiles > 0 ? (int)(t0 / q_tiles) - 1 : per_key_head, i = 0, hi = 0;
  auto kept = [&](int x) { return a.mask && !(x & (a.block - 1)) ? walk.next(x >> shift, lane) << shift : x; };
  auto advance = [&](int from) {
    i = kept(from);
    while (i >= hi && (g + 1) * (int64_t)q_tiles < t1) {
      ++g;
      const int lo = first + (int)max(t0 - g * (int64_t)q_tiles, (int64_t)0) * QB;
      hi = min((int64_t)first + (t1 - g * (int64_t)q_tiles) * QB, (int64_t)a.q_len);
      if (a.mask) {
        walk.at = uniform_ptr(a.mask + ((int64_t)b * a.heads + hk * per_key_head + g) * a.mb * a.nb + (tile * 32 * W >> shift));
        walk.step = a.nb;
        walk.entries = a.mb;
        walk.word_i = -1;
      }
      // the first tile may begin inside a mask block that the walk has not looked at
      i = a.mask ? max(kept(lo & ~(a.block - 1)), lo) : lo;
    }
    return i < hi;
  };
  auto copy = [&](int buf) {
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));
    const int64_t bh2 = (int64_t)b * a.heads + hk * per_key_head + g;
    const unsigned char* t = lds + buf * C::STAGE;
    const unsigned char* qg = (const unsigned char*)a.q + 2 * bh2 * a.q_len * C::KRB;
    copy_tile<C::KRB, QB, W>(t, qg, i, a.q_len - 1, w, lane_o);
    copy_tile<C::KRB, QB, W>(t + C::KBYTES, qg + (int64_t)a.q_len * C::KRB, i, a.q_len - 1, w, lane_o);
    copy_tile<C::VRB, QB, W>(t + 2 * C::KBYTES, (const unsigned char*)a.dout + bh2 * a.q_len * C::VRB, i, a.q_len - 1, w, lane_o);
    // 4 QB statistics: QB / 16 copies of 64, wavefront w takes copies w, w + W, ...
#pragma unroll
    for (int c = w; c < QB / 16; c += W) {
      const int at = c * 64 + lane_o;  // row at / QB of query i + at % QB
      dma4(a.rows + bh2 * 4 * a.q_len, (uint32_t)(min(i + at % QB, a.q_len - 1) + at / QB * a.q_len) * 4,
           (const unsigned char*)(stat[buf] + c * 64));
    }
  };
  // 32 queries; q0: the query of this lane's first register
  auto work = [&](uint32_t t, uint32_t to, const float* st, float lam, bool masked, int q0) {
    uint32_t qr = q_row + t, orow = o_row + to, qc0 = q_col0 + t, qc1 = q_col1 + t, oc0 = o_col0 + to, oc1 = o_col1 + to, vr = v_row;
    asm volatile("" : "+v"(qr), "+v"(orow), "+v"(qc0), "+v"(qc1), "+v"(oc0), "+v"(oc1), "+v"(vr));
    auto row = [&](int x) {
      const int y = x - 2 * C::KS;
      return x < 2 * C::KS ? read_row(lds + row_step(qr, x >> 1) + (x & 1) * C::KBYTES) : read_row(lds + row_step(orow, y & 7) + (y >> 3) * 256);
    };
    auto value = [&](int y) { return read_row(lds + row_step(vr, y & 7) + (y >> 3) * 256); };
    auto col = [&](int x) {  // of the products of 16 queries: dV's column tiles, then dK's of both maps
      const int x16 = x / (C::VT + 2 * C::DT), y = x % (C::VT + 2 * C::DT);
      if (y < C::VT) {
        const int at = 16 * x16 * C::VRB + (y >> 2) * 256;
        return read_cols(lds + col_step(oc0, y & 3) + at, lds + col_step(oc1, y & 3) + at);
      }
      const int c = (y - C::VT) % C::DT, at = (y - C::VT) / C::DT * C::KBYTES + 16 * x16 * C::KRB;
      return read_cols(lds + col_step(qc0, c) + at, lds + col_step(qc1, c) + at);
    };
    constexpr int ROWS = 2 * C::KS + C::VS, HALF = C::VT + 2 * C::DT;
    f32x16 s[2], dp;
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[0][4 * q4 + e] = st[8 * q4 + e];
        s[1][4 * q4 + e] = st[QB + 8 * q4 + e];
        dp[4 * q4 + e] = st[2 * QB + 8 * q4 + e];
      }
    constexpr int WV = kDkvWaves<D>;
    float p[2][16], pc[16];
#pragma unroll
    for (int s = C::KS - KEPT; s < C::KS; ++s) kf[1][s] = read_row(kept_keys + (s - C::KS + KEPT) * 1024 * W);
    bf16x8 ring[AHEAD], vring[AHEAD];
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) ring[x] = row(x);
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      in_order<kDkvWaves<D>>();
      if (x < 2 * C::KS)
        product<WV, false>(ring[x % AHEAD], kf[x & 1][x >> 1], s[x & 1]);
      else
        product<WV, false>(ring[x % AHEAD], kValuesInLds ? vring[x % AHEAD] : vf[kValuesInLds ? 0 : x - 2 * C::KS], dp);
      if (x == 2 * C::KS) settled<WV>(s[0], s[1]);
      if (x + AHEAD < ROWS) {
        ring[x % AHEAD] = row(x + AHEAD);
        if (kValuesInLds && x + AHEAD >= 2 * C::KS) vring[x % AHEAD] = value(x + AHEAD - 2 * C::KS);
      }
      if (x >= 2 * C::KS) {
        constexpr int PER = 32 / C::VS;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int v = (x - 2 * C::KS) * PER + e;
          p[v >> 4][v & 15] = __builtin_amdgcn_exp2f(s[v >> 4][v & 15] * c2);
        }
      }
    }
    float step[16];
    auto steps = [&](int v) {
#pragma unroll
      for (int e = v; e < v + 4; ++e) step[e] = st[3 * QB + v + e];
    };
    if constexpr (KEPT == 0) {  // else four at a time, where they are used
#pragma unroll
      for (int v = 0; v < 16; v += 4) steps(v);
    }
    bf16x8 cring[CAHEAD];
#pragma unroll
    for (int x = 0; x < CAHEAD; ++x) cring[x] = col(x);
    settled<WV>(dp);
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int q = q0 + 8 * (v >> 2) + (v & 3);
        if (q < from || q >= a.q_len) p[0][v] = p[1][v] = 0.f;
      }
    }
    auto weigh = [&](int v) {
      if (KEPT && v % 4 == 0) steps(v);
      const float p2 = -lam * p[1][v];
      pc[v] = p[0][v] + p2;
      p[0][v] *= dp[v];
      p[1][v] = p2 * (dp[v] + step[v]);
    };
    bf16x8 w8[3];  // of 16 queries: P_1 - lam P_2, dS_1, dS_2
#pragma unroll
    for (int v = 0; v < 8; ++v) weigh(v);
    w8[0] = pack8(pc);
    w8[1] = pack8(p[0]);
    w8[2] = pack8(p[1]);
#pragma unroll
    for (int x = 0; x < 2 * HALF; ++x) {
      in_order<kDkvWaves<D>>();
      const int y = x % HALF;
      if (x == HALF) w8[0] = pack8(pc + 8);
      if (x == HALF + C::VT) w8[1] = pack8(p[0] + 8);
      if (x == HALF + C::VT + C::DT) w8[2] = pack8(p[1] + 8);
      if (y < C::VT)
        dv[y] = mfma(cring[x % CAHEAD], w8[0], dv[y]);
      else
        dk[(y - C::VT) / C::DT][(y - C::VT) % C::DT] =
            mfma(cring[x % CAHEAD], w8[1 + (y - C::VT) / C::DT], dk[(y - C::VT) / C::DT][(y - C::VT) % C::DT]);
      if (x + CAHEAD < 2 * HALF) cring[x % CAHEAD] = col(x + CAHEAD);
#pragma unroll
      for (int v = 8; v < 16; ++v)  // the second 16 queries' beside the products of the first
        if (x == (v - 8) * HALF / 8) weigh(v);
    }
    in_order<kDkvWaves<D>>();
  };
  bool more = advance(0);
  if (more) copy(0);
  int buf = 0;
  while (more) {
    const int i0 = i;
    const float lam = a.lam[hk * per_key_head + g];
    more = advance(i0 + QB);
    WA_WAIT_VM(0);
    WA_BARRIER();
    if (more) copy(buf ^ 1);
    int end = QB;  // opaque: without a loop of its own, the work shares its registers with the next tile's addresses and spills
    asm volatile("" : "+s"(end));
#pragma unroll 1
    for (int half = 0; half < end; half += 32) {
      const int i1 = i0 + half;
      if (i1 + 32 <= some || i1 >= a.q_len) continue;
      work(buf * C::STAGE + half * C::KRB, buf * C::STAGE + half * C::VRB, stat[buf] + half + 4 * hf, lam, !whole || i1 < all || i1 + 32 > a.q_len, i1 + 4 * hf);
    }
    buf ^= 1;
  }
  if (task.chunks > 1) {
    float* to = a.part + (task.part * 32 * W + w * 32 + l32) * (2 * D + DV);
    store_part(to, dk[0], a.scale, hf);
    store_part(to + D, dk[1], a.scale, hf);
    store_part(to + 2 * D, dv, 1.f, hf);
  } else if (kj < a.kv_len) {  // keys that the sequence does not hold, or no query sees, get 0
    store_row((uint16_t*)a.dk + krow0 * D, dk[0], a.scale, hf);
    store_row((uint16_t*)a.dk + (krow0 + a.kv_len) * D, dk[1], a.scale, hf);
    store_row((uint16_t*)a.dv + vrow * DV, dv, 1.f, hf);
  }
}

// Adds the parts' results in order and rounds: a thread four columns of a row (2 D of both maps, then DV).
__global__ __launch_bounds__(256) void diff_parts_kernel(const float* part, uint16_t* maps, uint16_t* values, int64_t rows, int len,
                                                         int tile_rows, int tiles, int parts, int d, int dv) {
  const int width = 2 * d + dv, quads = width / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / quads;
  if (row >= rows) return;
  const int c = (int)(id % quads) * 4;
  const int64_t unit = row / len;
  const int i = row % len;
  const float* at = part + ((unit * tiles + i / tile_rows) * parts * tile_rows + i % tile_rows) * width + c;
  float4 sum = *(const float4*)at;
#pragma unroll 4
  for (int x = 1; x < parts; ++x) {
    const float4 y = *(const float4*)(at + (int64_t)x * tile_rows * width);
    sum.x += y.x;
    sum.y += y.y;
    sum.z += y.z;
    sum.w += y.w;
  }
  uint16_t* out = c < 2 * d ? maps + ((unit * 2 + c / d) * len + i) * d + c % d : values + row * dv + c - 2 * d;
  *(uint2*)out = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
}

// The same for the cut tiles of a list of tasks.
__global__ __launch_bounds__(256) void diff_parts_cut_kernel(const WaDiffLaunch a, const WaDiffSide n, uint16_t* maps, uint16_t* values,
                                                             int len, int dv) {
  const int d = a.head_dim, width = 2 * d + dv, quads = width / 4, rows = 32 * n.waves;
  const int64_t all = (int64_t)a.tasks[1] * rows * quads;
  const int4* cuts = (const int4*)(a.tasks + wa_diff_cut_list(a.task_items, wa_diff_slots(n.waves)));
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < all; id += (int64_t)gridDim.x * 256) {
    const int r = (int)(id / quads), c = (int)(id % quads) * 4;
    const int4 e = cuts[r / rows];
    const int64_t unit = e.x / n.tiles;
    const int i = e.x % n.tiles * rows + r % rows;
    if (i >= len) continue;
    const float* at = a.part + ((int64_t)e.z * rows + r % rows) * width + c;
    float4 sum = *(const float4*)at;
#pragma unroll 4
    for (int x = 1; x < e.y; ++x) {
      const float4 y = *(const float4*)(at + (int64_t)x * rows * width);
      sum.x += y.x;
      sum.y += y.y;
      sum.z += y.z;
      sum.w += y.w;
    }
    uint16_t* out = c < 2 * d ? maps + ((unit * 2 + c / d) * len + i) * d + c % d : values + (unit * len + i) * dv + c - 2 * d;
    *(uint2*)out = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
  }
}

hipError_t launch_parts(const WaDiffLaunch& a, const WaDiffSide& n, void* maps, void* values, int64_t rows, int len, int dv,
                        hipStream_t stream) {
  if (a.tasks) {
    hipLaunchKernelGGL(diff_parts_cut_kernel, dim3(1024), dim3(256), 0, stream, a, n, (uint16_t*)maps, (uint16_t*)values, len, dv);
  } else if (n.parts > 1) {
    const int64_t threads = rows * ((2 * a.head_dim + dv) / 4);
    hipLaunchKernelGGL(diff_parts_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a.part, (uint16_t*)maps,
                       (uint16_t*)values, rows, len, 32 * n.waves, n.tiles, n.parts, a.head_dim, dv);
  }
  return hipGetLastError();
}

// a.tasks for a side, if it has a list; its workgroups
template <bool COLUMNS>
hipError_t start_side(WaDiffLaunch& a, int32_t* tasks, const WaDiffSide& n, unsigned* grid, hipStream_t stream) {
  a.tasks = a.mask && n.parts == 1 && wa_diff_has_tasks(n.items) ? tasks : nullptr;
  *grid = (unsigned)(n.items * n.parts);
  if (!a.tasks) return hipSuccess;
  const int slots = wa_diff_slots(n.waves);
  a.task_items = (int32_t)n.items;
  *grid += slots;
  return wa_launch_diff_tasks(a, COLUMNS, slots, stream);
}

template <int D, int DV>
hipError_t launch_dims(WaDiffLaunch a, hipStream_t stream) {
  const WaDiffSide q = wa_diff_dq_side(a, a.mask), k = wa_diff_dkv_side(a, a.mask);
  int32_t* const tasks = a.tasks;
  unsigned grid;
  hipError_t e = start_side<false>(a, tasks, q, &grid, stream);
  if (e != hipSuccess) return e;
  const int lam_parts = q.tiles * (a.tasks ? kDiffMaxChunks : q.parts);
  if (q.waves == 2)
    hipLaunchKernelGGL((diff_dq_kernel<D, DV, 2>), dim3(grid), dim3(128), 0, stream, a, q);
  else
    hipLaunchKernelGGL((diff_dq_kernel<D, DV, 4>), dim3(grid), dim3(256), 0, stream, a, q);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if ((e = launch_parts(a, q, a.dq, nullptr, (int64_t)a.batch * a.heads * a.q_len, a.q_len, 0, stream)) != hipSuccess) return e;

  if ((e = start_side<true>(a, tasks, k, &grid, stream)) != hipSuccess) return e;
  if (k.waves == 2)
    hipLaunchKernelGGL((diff_dkv_kernel<D, DV, 2>), dim3(grid), dim3(128), 0, stream, a, k, lam_parts);
  else
    hipLaunchKernelGGL((diff_dkv_kernel<D, DV, 4>), dim3(grid), dim3(256), 0, stream, a, k, lam_parts);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  return launch_parts(a, k, a.dk, a.dv, (int64_t)a.batch * a.kv_heads * a.kv_len, a.kv_len, DV, stream);
}

// Tiles of 128 tokens, or 64 where a mask block or the sequence is no longer. A call of few tiles does each in parts, so many
// as fill the chip's workgroups once (256 of four wavefronts, 512 of two, times per_cu); twice where the tiles are of
// different lengths. A part is 4 tiles of 64 of the other side at least, and its float32 result is written and read once more: with
// per_cu 2 for d 64, where two wavefronts share a SIMD, dK and dV of 2 x 16 causal heads of 2,048 tokens and 4 key heads take
// 117 + 21 us instead of 136 + 12, but dQ 88 + 12 instead of 90.
WaDiffSide side_of(const WaDiffLaunch& a, bool masked, int len, int units, int64_t other, int per_cu) {
  WaDiffSide s;
  s.waves = len <= 64 || (masked && a.block == 64) ? 2 : 4;
  s.tiles = (len + 32 * s.waves - 1) / (32 * s.waves);
  s.items = (int64_t)units * s.tiles;
  const int64_t slots = (s.waves == 2 ? 512 : 256) * per_cu * (a.causal || masked ? 2 : 1);
  s.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(slots / s.items, other / 256));
  return s;
}

}  // namespace

WaDiffSide wa_diff_dq_side(const WaDiffLaunch& a, bool masked) { return side_of(a, masked, a.q_len, a.batch * a.heads, a.kv_len, 1); }
WaDiffSide wa_diff_dkv_side(const WaDiffLaunch& a, bool masked) {
  return side_of(a, masked, a.kv_len, a.batch * a.kv_heads, (int64_t)(a.heads / a.kv_heads) * a.q_len, a.head_dim == 64 ? 2 : 1);
}
int64_t wa_diff_side_tiles(const WaDiffSide& s, bool masked) {
  return s.parts > 1 ? s.items * s.parts : masked && wa_diff_has_tasks(s.items) ? 2 * wa_diff_slots(s.waves) : 0;
}

hipError_t wa_launch_diff_backward(const WaDiffLaunch& a, hipStream_t stream) {
  if (a.head_dim == 64 && a.value_dim == 64) return launch_dims<64, 64>(a, stream);
  if (a.head_dim == 64 && a.value_dim == 128) return launch_dims<64, 128>(a, stream);
  if (a.head_dim == 128 && a.value_dim == 128) return launch_dims<128, 128>(a, stream);
  if (a.head_dim == 128 && a.value_dim == 256) return launch_dims<128, 256>(a, stream);
  return hipErrorInvalidValue;
}
