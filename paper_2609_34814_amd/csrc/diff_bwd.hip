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
// dlam is summed from the float32 P_2 dP, not from the stored maps: over a lane's keys with the roundings carried along, over
// queries in float64.

#include "diff_tiles.h"
#include "wavealign.h"

#include <algorithm>

namespace {

using namespace wa;

template <int D, int DV, int W>
struct Bwd {
  // Tokens of a passing tile: 64 with four wavefronts, 32 with two (two workgroups share a compute unit's LDS).
  static constexpr int TB = W == 4 ? 64 : 32;
  static constexpr int KRB = D * 2, VRB = DV * 2;
  static constexpr int KBYTES = TB * KRB, VBYTES = TB * VRB, STAGE = 2 * KBYTES + VBYTES;
  static constexpr int DT = D / 32, VT = DV / 32, KS = D / 16, VS = DV / 16;
};
// Wavefronts a SIMD: two share its 512 registers a lane where both hold their accumulators without spilling.
template <int D>
constexpr int kDqWaves = D == 64 ? 2 : 1;
template <int DV>
constexpr int kDkvWaves = DV == 64 ? 2 : 1;

__device__ __forceinline__ void clear(f32x16& x) {
#pragma unroll
  for (int v = 0; v < 16; ++v) x[v] = 0.f;
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
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

template <int D, int DV, int W>
__global__ __launch_bounds__(64 * W, kDqWaves<D>) void diff_dq_kernel(const WaDiffLaunch a, int tiles) {
  using C = Bwd<D, DV, W>;
  constexpr int KB = C::TB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * C::STAGE];
  __shared__ double lam_sum[W];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // heads one after another, the longest tiles of each first where later queries see more keys
  const int bh = blockIdx.x / tiles, b = bh / a.heads, h = bh % a.heads, hk = h / (a.heads / a.kv_heads);
  const int tile = a.causal ? tiles - 1 - blockIdx.x % tiles : blockIdx.x % tiles;
  const int i0 = tile * 32 * W + w * 32, i = i0 + l32, i_last = a.q_len - 1;
  const bool valid = i <= i_last;
  const int keys = keys_of(a, b), start = start_of(a, b);
  const int limit = valid ? key_limit(a, keys, start, i) : 0;
  const int some = i0 > i_last ? 0 : key_limit(a, keys, start, min(i0 + 31, i_last));
  const int all = key_limit(a, keys, start, min(i0, i_last));
  const int hi = key_limit(a, keys, start, min(tile * 32 * W + 32 * W - 1, i_last));

  const unsigned char* kg = (const unsigned char*)a.k + (((int64_t)b * 2 * a.kv_heads + 2 * hk) * a.kv_len) * C::KRB;
  const unsigned char* vg = (const unsigned char*)a.v + (((int64_t)b * a.kv_heads + hk) * a.kv_len) * C::VRB;
  MaskWalk walk;
  const int shift = a.block == 128 ? 7 : 6;
  if (a.mask) {
    walk.at = uniform_ptr(a.mask + ((int64_t)bh * a.mb + (tile * 32 * W >> shift)) * a.nb);
    walk.entries = (hi + a.block - 1) >> shift;
  }
  auto next_tile = [&](int key) {
    if (!a.mask || (key & (a.block - 1))) return key;
    return walk.next(key >> shift, lane) << shift;
  };
  auto copy = [&](int key, int buf) {
    const unsigned char* t = lds + buf * C::STAGE;
    copy_tile<C::KRB, KB, W>(t, kg, key, keys - 1, w, lane);
    copy_tile<C::KRB, KB, W>(t + C::KBYTES, kg + (int64_t)a.kv_len * C::KRB, key, keys - 1, w, lane);
    copy_tile<C::VRB, KB, W>(t + 2 * C::KBYTES, vg, key, keys - 1, w, lane);
  };
  int key = hi > 0 ? next_tile(0) : 0, buf = 0;
  if (key < hi) copy(key, 0);

  // the wavefront's queries, their dO, and D_m
  bf16x8 qf[2][C::KS], dof[C::VS];
  const int64_t row0 = ((int64_t)b * 2 * a.heads + 2 * h) * a.q_len + i, row = ((int64_t)bh * a.q_len + i) * DV;
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
#pragma unroll
    for (int m = 0; m < 2; ++m)
      qf[m][s] = load8((const uint16_t*)a.q + (row0 + (int64_t)m * a.q_len) * D + 16 * s + 8 * hf, valid);
  float d[2] = {0.f, 0.f}, ref[2] = {0.f, 0.f}, factor = 1.f;  // ref: log-sum-exp in log2 units
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
  const int64_t all_rows = (int64_t)a.batch * 2 * a.heads * a.q_len;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    d[m] = add_halves(d[m]);
    if (valid) {
      const int64_t at = row0 + (int64_t)m * a.q_len;
      ref[m] = a.stats[3 * at] * kLog2e;
      d[m] *= a.stats[3 * at + 1];
      factor = a.stats[3 * at + 2];  // of the second map, in the end
      if (hf == 0) {
        a.rows[at] = ref[m];
        a.rows[all_rows + at] = d[m];
      }
    }
  }
  const float lam = a.lam[h];

  uint32_t kofs[C::KS], vofs[C::VS < 16 ? C::VS : 8], kcol[2][C::DT];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) kofs[s] = row_operand<C::KRB>(lane, s);
#pragma unroll
  for (int s = 0; s < (C::VS < 16 ? C::VS : 8); ++s) vofs[s] = 2 * C::KBYTES + row_operand<C::VRB>(lane, s);
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int c = 0; c < C::DT; ++c) kcol[j][c] = col_operand<C::KRB>(lane, c, j);

  const float c2 = a.scale * kLog2e;
  f32x16 dq[2][C::DT];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int c = 0; c < C::DT; ++c) clear(dq[m][c]);
  float lam_dot = 0.f, lam_lost = 0.f;

  while (key < hi) {
    const int next = next_tile(key + KB);
    WA_WAIT_VM(0);
    WA_BARRIER();
    if (next < hi) copy(next, buf ^ 1);
#pragma unroll 1
    for (int half = 0; half < KB; half += 32) {
      if (key + half >= some) break;
      const unsigned char* t = lds + buf * C::STAGE + half * C::KRB;
      const unsigned char* tv = lds + buf * C::STAGE + half * C::VRB;
      f32x16 s[2], dp;
      clear(s[0]);
      clear(s[1]);
      clear(dp);
#pragma unroll
      for (int x = 0; x < C::KS; ++x)
#pragma unroll
        for (int m = 0; m < 2; ++m) s[m] = mfma(read_row(t + m * C::KBYTES + kofs[x]), qf[m][x], s[m]);
#pragma unroll
      for (int x = 0; x < C::VS; ++x) dp = mfma(read_row(tv + vofs[x & 7] + (x >> 3) * 256), dof[x], dp);
      float p[2][16];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int v = 0; v < 16; ++v) p[m][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[m][v], c2, -ref[m]));
      if (key + half + 32 > all) {
        const int rest = limit - key - half - 4 * hf;
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v >> 2) + (v & 3) >= rest) p[0][v] = p[1][v] = 0.f;
      }
      float dot = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        dot = __builtin_fmaf(p[1][v], dp[v], dot);
        p[0][v] *= dp[v] - d[0];
        p[1][v] *= dp[v] - d[1];
      }
      const float add = dot - lam_lost, grown = lam_dot + add;
      lam_lost = (grown - lam_dot) - add;
      lam_dot = grown;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const bf16x8 ds = pack8(p[m] + 8 * x);
          const unsigned char* tk = t + m * C::KBYTES + 16 * x * C::KRB;
#pragma unroll
          for (int c = 0; c < C::DT; ++c) dq[m][c] = mfma(read_cols(tk + kcol[0][c], tk + kcol[1][c]), ds, dq[m][c]);
        }
    }
    key = next;
    buf ^= 1;
  }
  if (valid) {
    store_row(((uint16_t*)a.dq) + row0 * D, dq[0], a.scale, hf);
    store_row(((uint16_t*)a.dq) + (row0 + a.q_len) * D, dq[1], -lam * a.scale, hf);
  }
  double lam_row = (double)lam_dot * factor;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) lam_row += __shfl_xor(lam_row, x);
  if (lane == 0) lam_sum[w] = lam_row;
  __syncthreads();
  if (tid == 0) {
    double sum = 0.0;
    for (int x = 0; x < W; ++x) sum += lam_sum[x];
    a.lam_part[(int64_t)bh * tiles + tile] = sum;
  }
}

// One 4-byte-a-lane copy from global memory into LDS at the uniform address lds (lane i writes lds + 4 i).
__device__ __forceinline__ void dma4(const void* gbase, uint32_t voff, const unsigned char* lds) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)lds);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "global_load_lds_dword %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(m0), "v"(voff), "s"(gbase)
      : "memory");
}

template <int D, int DV, int W>
__global__ __launch_bounds__(64 * W, kDkvWaves<DV>) void diff_dkv_kernel(const WaDiffLaunch a, int tiles, int q_tiles) {
  using C = Bwd<D, DV, W>;
  constexpr int QB = C::TB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * C::STAGE];
  __shared__ __attribute__((aligned(1024))) float stat[2][4 * QB];  // of both maps: log-sum-exps (log2 units), then D_m

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // dlam: the parts that diff_dq_kernel left, in float64, in one order
  for (int h = blockIdx.x; h < a.heads; h += gridDim.x) {
    if (tid < 64) {
      double sum = 0.0;
      for (int b = 0; b < a.batch; ++b)
        for (int t = lane; t < q_tiles; t += 64) sum += a.lam_part[((int64_t)b * a.heads + h) * q_tiles + t];
      for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
      if (lane == 0) a.dlam[h] = (float)-sum;
    }
  }

  // the first tiles of keys, which the most queries see, come first
  const int bh = blockIdx.x / tiles, b = bh / a.kv_heads, hk = bh % a.kv_heads, per_key_head = a.heads / a.kv_heads;
  const int tile = blockIdx.x % tiles;
  const int keys = keys_of(a, b), start = start_of(a, b);
  const int k0 = tile * 32 * W + w * 32, kj = k0 + l32;
  const bool valid = kj < keys;
  // first query that sees this lane's key, the wavefront's first key, its last, the workgroup's first
  auto first_query = [&](int j) { return j >= keys ? a.q_len : a.causal ? min(max(j - start, 0), a.q_len) : 0; };
  const int from = first_query(kj);
  const int some = first_query(k0), all = first_query(min(k0 + 31, max(keys - 1, k0)));
  const bool whole = k0 + 31 < keys;
  const int lo = first_query(tile * 32 * W) / QB * QB, hi = a.q_len;

  const int64_t krow0 = ((int64_t)b * 2 * a.kv_heads + 2 * hk) * a.kv_len + kj, vrow = (int64_t)bh * a.kv_len + kj;
  bf16x8 kf[2][C::KS], vf[C::VS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
#pragma unroll
    for (int m = 0; m < 2; ++m)
      kf[m][s] = load8((const uint16_t*)a.k + (krow0 + (int64_t)m * a.kv_len) * D + 16 * s + 8 * hf, valid);
#pragma unroll
  for (int s = 0; s < C::VS; ++s) vf[s] = load8((const uint16_t*)a.v + vrow * DV + 16 * s + 8 * hf, valid);

  uint32_t qofs[C::KS], oofs[C::VS < 16 ? C::VS : 8], qcol[2][C::DT], ocol[2][C::VT < 8 ? C::VT : 4];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) qofs[s] = row_operand<C::KRB>(lane, s);
#pragma unroll
  for (int s = 0; s < (C::VS < 16 ? C::VS : 8); ++s) oofs[s] = 2 * C::KBYTES + row_operand<C::VRB>(lane, s);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
#pragma unroll
    for (int c = 0; c < C::DT; ++c) qcol[j][c] = col_operand<C::KRB>(lane, c, j);
#pragma unroll
    for (int c = 0; c < (C::VT < 8 ? C::VT : 4); ++c) ocol[j][c] = 2 * C::KBYTES + col_operand<C::VRB>(lane, c, j);
  }

  const float c2 = a.scale * kLog2e;
  f32x16 dk[2][C::DT], dv[C::VT];
#pragma unroll
  for (int c = 0; c < C::DT; ++c) {
    clear(dk[0][c]);
    clear(dk[1][c]);
  }
#pragma unroll
  for (int c = 0; c < C::VT; ++c) clear(dv[c]);

  const int shift = a.block == 128 ? 7 : 6;
  for (int g = 0; g < per_key_head; ++g) {
    const int h = hk * per_key_head + g;
    const float lam = a.lam[h];
    const int64_t qh = (int64_t)b * 2 * a.heads + 2 * h;
    const unsigned char* qg = (const unsigned char*)a.q + qh * a.q_len * C::KRB;
    const unsigned char* og = (const unsigned char*)a.dout + ((int64_t)b * a.heads + h) * a.q_len * C::VRB;
    const float* ref = a.rows + qh * a.q_len;
    const float* dots = ref + (int64_t)a.batch * 2 * a.heads * a.q_len;
    MaskWalk walk;
    if (a.mask) {
      walk.at = uniform_ptr(a.mask + ((int64_t)b * a.heads + h) * a.mb * a.nb + (tile * 32 * W >> shift));
      walk.step = a.nb;
      walk.entries = a.mb;
    }
    auto next_tile = [&](int i) {
      if (!a.mask || (i & (a.block - 1))) return i;
      return walk.next(i >> shift, lane) << shift;
    };
    auto copy = [&](int i, int buf) {
      const unsigned char* t = lds + buf * C::STAGE;
      copy_tile<C::KRB, QB, W>(t, qg, i, a.q_len - 1, w, lane);
      copy_tile<C::KRB, QB, W>(t + C::KBYTES, qg + (int64_t)a.q_len * C::KRB, i, a.q_len - 1, w, lane);
      copy_tile<C::VRB, QB, W>(t + 2 * C::KBYTES, og, i, a.q_len - 1, w, lane);
      // 4 QB statistics: QB / 16 copies of 64, wavefront w takes copies w, w + W, ...
#pragma unroll
      for (int c = w; c < QB / 16; c += W) {
        const int at = c * 64 + lane;  // statistic at / QB of query i + at % QB
        const int x = min(i + at % QB, a.q_len - 1) + (at / QB & 1) * a.q_len;
        dma4(c * 64 < 2 * QB ? ref : dots, (uint32_t)x * 4, (const unsigned char*)(stat[buf] + c * 64));
      }
    };
    // The first tile may begin inside a mask block that the walk has not looked at.
    int i = lo < hi ? (a.mask ? max(next_tile(lo & ~(a.block - 1)), lo) : lo) : hi, buf = 0;
    WA_BARRIER();  // everyone is done with the tiles of the head before
    if (i < hi) copy(i, 0);
    while (i < hi) {
      const int next = next_tile(i + QB);
      WA_WAIT_VM(0);
      WA_BARRIER();
      if (next < hi) copy(next, buf ^ 1);
#pragma unroll 1
      for (int half = 0; half < QB; half += 32) {
        const int i1 = i + half;
        if (i1 + 32 <= some || i1 >= hi) continue;
        const unsigned char* t = lds + buf * C::STAGE + half * C::KRB;
        const unsigned char* to = lds + buf * C::STAGE + half * C::VRB;
        f32x16 s[2], dp;
        clear(s[0]);
        clear(s[1]);
        clear(dp);
#pragma unroll
        for (int x = 0; x < C::KS; ++x)
#pragma unroll
          for (int m = 0; m < 2; ++m) s[m] = mfma(read_row(t + m * C::KBYTES + qofs[x]), kf[m][x], s[m]);
#pragma unroll
        for (int x = 0; x < C::VS; ++x) dp = mfma(read_row(to + oofs[x & 7] + (x >> 3) * 256), vf[x], dp);
        // register v holds query 8 (v / 4) + 4 hf + v % 4
        const float* st = stat[buf] + half + 4 * hf;
        float p[2][16], pc[16];
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float4 l0 = *(const float4*)(st + 8 * q4), l1 = *(const float4*)(st + QB + 8 * q4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = 4 * q4 + e;
            p[0][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][v], c2, -(&l0.x)[e]));
            p[1][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[1][v], c2, -(&l1.x)[e]));
          }
        }
        if (!whole || i1 < all || i1 + 32 > hi) {
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int q = i1 + 8 * (v >> 2) + 4 * hf + (v & 3);
            if (q < from || q >= hi) p[0][v] = p[1][v] = 0.f;
          }
        }
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float4 d0 = *(const float4*)(st + 2 * QB + 8 * q4), d1 = *(const float4*)(st + 3 * QB + 8 * q4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = 4 * q4 + e;
            const float p2 = -lam * p[1][v];
            pc[v] = p[0][v] + p2;
            p[0][v] *= dp[v] - (&d0.x)[e];
            p[1][v] = p2 * (dp[v] - (&d1.x)[e]);
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const bf16x8 pb = pack8(pc + 8 * x);
          const unsigned char* tc = to + 16 * x * C::VRB;
#pragma unroll
          for (int c = 0; c < C::VT; ++c)
            dv[c] = mfma(read_cols(tc + ocol[0][c & 3] + (c >> 2) * 256, tc + ocol[1][c & 3] + (c >> 2) * 256), pb, dv[c]);
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const bf16x8 ds = pack8(p[m] + 8 * x);
            const unsigned char* tq = t + m * C::KBYTES + 16 * x * C::KRB;
#pragma unroll
            for (int c = 0; c < C::DT; ++c) dk[m][c] = mfma(read_cols(tq + qcol[0][c], tq + qcol[1][c]), ds, dk[m][c]);
          }
        }
      }
      i = next;
      buf ^= 1;
    }
  }
  if (kj < a.kv_len) {  // keys that the sequence does not hold get 0
    store_row((uint16_t*)a.dk + krow0 * D, dk[0], a.scale, hf);
    store_row((uint16_t*)a.dk + (krow0 + a.kv_len) * D, dk[1], a.scale, hf);
    store_row((uint16_t*)a.dv + vrow * DV, dv, 1.f, hf);
  }
}

int waves_of(const WaDiffLaunch& a, int len) { return len <= 64 || (a.mask && a.block == 64) ? 2 : 4; }

template <int D, int DV, int W>
hipError_t launch_dq(const WaDiffLaunch& a, hipStream_t stream) {
  const int tiles = (a.q_len + 32 * W - 1) / (32 * W);
  hipLaunchKernelGGL((diff_dq_kernel<D, DV, W>), dim3((unsigned)(a.batch * a.heads * tiles)), dim3(64 * W), 0, stream, a, tiles);
  return hipGetLastError();
}
template <int D, int DV, int W>
hipError_t launch_dkv(const WaDiffLaunch& a, int q_tiles, hipStream_t stream) {
  const int tiles = (a.kv_len + 32 * W - 1) / (32 * W);
  hipLaunchKernelGGL((diff_dkv_kernel<D, DV, W>), dim3((unsigned)(a.batch * a.kv_heads * tiles)), dim3(64 * W), 0, stream, a, tiles,
                     q_tiles);
  return hipGetLastError();
}
template <int D, int DV>
hipError_t launch_dims(const WaDiffLaunch& a, hipStream_t stream) {
  const int wq = waves_of(a, a.q_len), wk = waves_of(a, a.kv_len), q_tiles = (a.q_len + 32 * wq - 1) / (32 * wq);
  const hipError_t e = wq == 2 ? launch_dq<D, DV, 2>(a, stream) : launch_dq<D, DV, 4>(a, stream);
  if (e != hipSuccess) return e;
  return wk == 2 ? launch_dkv<D, DV, 2>(a, q_tiles, stream) : launch_dkv<D, DV, 4>(a, q_tiles, stream);
}

}  // namespace

hipError_t wa_launch_diff_backward(const WaDiffLaunch& a, hipStream_t stream) {
  if (a.head_dim == 64 && a.value_dim == 64) return launch_dims<64, 64>(a, stream);
  if (a.head_dim == 64 && a.value_dim == 128) return launch_dims<64, 128>(a, stream);
  if (a.head_dim == 128 && a.value_dim == 128) return launch_dims<128, 128>(a, stream);
  if (a.head_dim == 128 && a.value_dim == 256) return launch_dims<128, 256>(a, stream);
  return hipErrorInvalidValue;
}
