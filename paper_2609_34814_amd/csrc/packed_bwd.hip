// Gradient of attention over packed sequences for gfx950 (MI355X). With P recomputed from the forward's log-sum-exps,
//   dP = dO V^T,   D = dO . O,   dS = P (dP - D),   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO.
//
// Two kernels, each owning what it writes, so nothing is added with atomics and equal calls give equal bits:
//   packed_dq_kernel: 128 queries of a head, over their keys; also writes what the other kernel's products of a query start from.
//   packed_dkv_kernel: 128 keys, over the queries of all heads that share them; in a call of few such tiles in parts, which
//   packed_parts_kernel adds in order.
// Both recompute the scores and dP. A wavefront holds 32 queries (keys) with their accumulators in registers, and the other side's
// tiles pass through LDS, copied one ahead. Scores come out with the wavefront's own index in the lanes and the other in the
// registers, so P and dS, rounded to bf16, are operands of the following products as they are. Two wavefronts share a SIMD.
//
// The lengths are known on the device only: workgroups are dealt tiles longest first over all sequences, each finding its own by counting
// the tiles that are longer (a sequence a lane).

#include "seq_attn.h"

#include <algorithm>

namespace {

using namespace wa;

constexpr int kRows = 128, kWaves = 4, kAhead = 2;

template <int D>
struct Bwd {
  static constexpr int RB = D * 2, DT = D / 32, KS = D / 16;
  // Values lie in LDS where, with the keys and the sums of dK and dV, they do not fit the registers; queries then pass 32 at a time.
  static constexpr bool kValuesInLds = D == 128;
  static constexpr int KB = 64, QB = kValuesInLds ? 32 : 64;
};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Tile number `rank` of all sequences, by descending level (a tile's number in its sequence, or that counted from the end): the sequence
// and the level, or false.
__device__ __forceinline__ bool tile_of(SeqArgs a, int64_t rank, int lane, int* b, int* level) {
  auto tiles_of = [&](int x) { return x < a->batch ? (int)(((int64_t)seq_of<false>(a, x).n + kRows - 1) / kRows) : 0; };
  const int mine = tiles_of(lane);
  // tiles of level t and above
  auto above = [&](int t) {
    int64_t sum = max(mine - t, 0);
    for (int base = 64; base < a->batch; base += 64) sum += max(tiles_of(base + lane) - t, 0);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
    return sum;
  };
  int most = mine;
  for (int base = 64; base < a->batch; base += 64) most = max(most, tiles_of(base + lane));
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) most = max(most, __shfl_xor(most, x));
  if (rank >= above(0)) return false;
  int lo = 0, hi = most;  // above(lo) > rank >= above(hi)
  while (hi - lo > 1) {
    const int mid = lo + ((hi - lo) >> 1);
    if (above(mid) > rank) lo = mid; else hi = mid;
  }
  int64_t k = rank - above(lo + 1);
  for (int base = 0; base < a->batch; base += 64) {
    uint64_t there = __ballot((base ? tiles_of(base + lane) : mine) > lo);
    const int n = __popcll(there);
    if (k < n) {
      for (; k > 0; --k) there &= there - 1;
      *b = base + __builtin_ctzll(there);
      *level = lo;
      return true;
    }
    k -= n;
  }
  return false;
}

// Neighbouring units, which may share keys, on one XCD where eight divides their number.
__device__ __forceinline__ int spread(int u, int units) { return units % 8 ? u : u % 8 * (units / 8) + u / 8; }

// Rows [row, row + ROWS) of g (`token` bytes apart) into a tile; rows past `last` are that row again.
template <int RB, int ROWS>
__device__ __forceinline__ void copy_rows(const unsigned char* tile, const unsigned char* g, uint32_t token, int row, int last, int w,
                                          int lane) {
  constexpr int RPI = 1024 / RB, LPR = RB / 16, N = ROWS * RB / 1024 / kWaves;
  static_assert(N * kWaves * 1024 == ROWS * RB, "a tile is whole copies of every wavefront");
  const unsigned char* from = g + (int64_t)row * token;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = (i * kWaves + w) * RPI + lane / LPR;
    dma16(from, min(r, last - row) * token + tile_chunk<RB>(r, lane % LPR) * 16, tile + (i * kWaves + w) * 1024);
  }
}

__device__ __forceinline__ float dot8(bf16x8 a, bf16x8 b, float sum) {
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = __builtin_fmaf((float)a[i], (float)b[i], sum);
  return sum;
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void packed_dq_kernel(const WaSeqLaunch a) {
  using C = Bwd<D>;
  constexpr int KB = C::KB, BYTES = KB * C::RB, STAGE = 2 * BYTES;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  int b = 0, tile = 0;
  if (!__builtin_amdgcn_readfirstlane(tile_of(seq_args(), blockIdx.x / a.heads, lane, &b, &tile))) return;
  b = __builtin_amdgcn_readfirstlane(b);
  tile = __builtin_amdgcn_readfirstlane(tile);
  const int h = spread(blockIdx.x % a.heads, a.heads), hk = h / (a.heads / a.kv_heads);
  const Seq s = Walk<false>::uniform(seq_of<false>(seq_args(), b));
  const int i0 = tile * kRows + w * 32, i = i0 + l32, i_last = s.n - 1;
  const bool valid = i <= i_last;
  const int limit = !valid ? 0 : a.causal ? i + 1 : s.n;
  const int some = i0 > i_last ? 0 : a.causal ? min(i0 + 32, s.n) : s.n, all = a.causal ? min(i0 + 1, s.n) : s.n;
  const int most = a.causal ? min((tile + 1) * kRows, s.n) : s.n;
  const unsigned char* kg = (const unsigned char*)a.k.at + (s.first * a.k.token + hk * a.k.head) * 2;
  const unsigned char* vg = (const unsigned char*)a.v.at + (s.first * a.v.token + hk * a.v.head) * 2;
  auto copy = [&](int key, int buf) {
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));  // the copies' offsets are not held across the loop
    const unsigned char* t = lds + buf * STAGE;
    copy_rows<C::RB, KB>(t, kg, (uint32_t)(a.k.token * 2), key, i_last, w, lane_o);
    copy_rows<C::RB, KB>(t + BYTES, vg, (uint32_t)(a.v.token * 2), key, i_last, w, lane_o);
  };
  copy(0, 0);

  // the wavefront's queries, their dO, and D
  bf16x8 qf[C::KS], dof[C::KS];
  const int64_t tok = s.first + i;
  const uint16_t* qg = (const uint16_t*)a.q.at + tok * a.q.token + h * a.q.head;
  const uint16_t* dog = (const uint16_t*)a.dout.at + tok * a.dout.token + h * a.dout.head;
  const uint16_t* og = (const uint16_t*)a.o.at + tok * a.o.token + h * a.o.head;
  float d = 0.f;
#pragma unroll
  for (int x = 0; x < C::KS; ++x) {
    qf[x] = load8(qg + 16 * x + 8 * hf, valid);
    dof[x] = load8(dog + 16 * x + 8 * hf, valid);
    d = dot8(dof[x], load8(og + 16 * x + 8 * hf, valid), d);
  }
  d = add_halves(d);
  const float c2 = a.scale * kLog2e;
  float ref = 0.f;  // log-sum-exp in log2 units
  if (valid) ref = a.lse_in[(int64_t)h * a.tokens + tok] * kLog2e;
  // For the side of the keys: what its products start from, scores from the log-sum-exp, so that P = exp2(c2 s), and dP from -D.
  if (valid && hf == 0) {
    float* to = a.rows + (int64_t)h * a.tokens + tok;
    to[0] = -ref / c2;
    to[(int64_t)a.heads * a.tokens] = -d;
  }

  const uint32_t k_row = row_operand<C::RB>(lane, 0), v_row = BYTES + row_operand<C::RB>(lane, 0);
  const uint32_t k_col0 = col_operand<C::RB>(lane, 0, 0), k_col1 = col_operand<C::RB>(lane, 0, 1);
  f32x16 dq[C::DT];
#pragma unroll
  for (int c = 0; c < C::DT; ++c) fill(dq[c], 0.f);

  // 32 keys; masked: this lane's query sees only `rest` of them, counted from its first register's.
  auto work = [&](uint32_t t, bool masked, int rest) {
    uint32_t kr = k_row + t, vr = v_row + t, kc0 = k_col0 + t, kc1 = k_col1 + t;
    asm volatile("" : "+v"(kr), "+v"(vr), "+v"(kc0), "+v"(kc1));
    auto row = [&](int x) {  // operand of product x of the scores, then of dP
      return x < C::KS ? read_row(lds + row_step(kr, x)) : read_row(lds + row_step(vr, x - C::KS));
    };
    auto col = [&](int x) {  // operand of product x of dQ: 16 keys, 32 columns
      const int at = 16 * (x / C::DT) * C::RB;
      return read_cols(lds + col_step(kc0, x % C::DT) + at, lds + col_step(kc1, x % C::DT) + at);
    };
    f32x16 sc, dp;
    fill(sc, 0.f);
    fill(dp, 0.f);
    float p[16];
    bf16x8 ring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) ring[x] = row(x);
#pragma unroll
    for (int x = 0; x < 2 * C::KS; ++x) {
      if (x < C::KS) sc = mfma(ring[x % kAhead], qf[x], sc); else dp = mfma(ring[x % kAhead], dof[x - C::KS], dp);
      if (x + kAhead < 2 * C::KS) ring[x % kAhead] = row(x + kAhead);
      if (x >= C::KS) {  // the exponentials run beside the products of dP
        constexpr int PER = 16 / C::KS;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int v = (x - C::KS) * PER + e;
          p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[v], c2, -ref));
        }
      }
    }
    bf16x8 cring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) cring[x] = col(x);
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + (v & 3) >= rest) p[v] = 0.f;
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] *= dp[v] - d;
    const bf16x8 ds[2] = {pack8(p), pack8(p + 8)};
#pragma unroll
    for (int x = 0; x < 2 * C::DT; ++x) {
      dq[x % C::DT] = mfma(cring[x % kAhead], ds[x / C::DT], dq[x % C::DT]);
      if (x + kAhead < 2 * C::DT) cring[x % kAhead] = col(x + kAhead);
    }
  };
  int buf = 0;
  for (int key = 0; key < most; key += KB) {
    WA_WAIT_VM(0);
    WA_BARRIER();
    if (key + KB < most) copy(key + KB, buf ^ 1);
    int end = KB;  // opaque: a loop, so that the two halves do not share registers
    asm volatile("" : "+s"(end));
#pragma unroll 1
    for (int half = 0; half < end; half += 32) {
      if (key + half >= some) break;
      work(buf * STAGE + half * C::RB, key + half + 32 > all, limit - key - half - 4 * hf);
    }
    buf ^= 1;
  }
  if (valid) store_row((uint16_t*)a.dq.at + tok * a.dq.token + h * a.dq.head, dq, a.scale, hf);
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void packed_dkv_kernel(const WaSeqLaunch a) {
  using C = Bwd<D>;
  constexpr int QB = C::QB, BYTES = QB * C::RB, STAGE = 2 * BYTES, VALUES = C::kValuesInLds ? kRows * C::RB : 0;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE + VALUES];
  __shared__ __attribute__((aligned(1024))) float stat[2][2 * QB];  // the rows of a.rows

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % a.parts, unit = blockIdx.x / a.parts;
  int b = 0, level = 0;
  if (!__builtin_amdgcn_readfirstlane(tile_of(seq_args(), unit / a.kv_heads, lane, &b, &level))) return;
  b = __builtin_amdgcn_readfirstlane(b);
  level = __builtin_amdgcn_readfirstlane(level);
  const int hk = spread(unit % a.kv_heads, a.kv_heads), group = a.heads / a.kv_heads;
  const Seq s = Walk<false>::uniform(seq_of<false>(seq_args(), b));
  // causal: the first tiles are seen by the most queries
  const int tile = a.causal ? (s.n + kRows - 1) / kRows - 1 - level : level;
  const int k0 = tile * kRows + w * 32, kj = k0 + l32;
  const bool valid = kj < s.n;
  const int from = !valid ? s.n : a.causal ? kj : 0;                      // first query that sees this lane's key,
  const int some = k0 >= s.n ? s.n : a.causal ? k0 : 0;                   // the wavefront's first
  const int all = a.causal ? min(k0 + 31, s.n - 1) : 0;                   // and its last
  const bool whole = k0 + 31 < s.n;
  // this part's tiles of queries, counted through the heads one after another
  const int first = (a.causal ? tile * kRows : 0) / QB * QB, q_tiles = (s.n - first + QB - 1) / QB;
  const int64_t all_tiles = (int64_t)group * q_tiles;
  const int64_t u0 = all_tiles * part / a.parts, u1 = all_tiles * (part + 1) / a.parts;

  const int64_t tok = s.first + kj;
  const uint16_t* kg = (const uint16_t*)a.k.at + tok * a.k.token + hk * a.k.head;
  const uint16_t* vg = (const uint16_t*)a.v.at + tok * a.v.token + hk * a.v.head;
  bf16x8 kf[C::KS], vf[C::kValuesInLds ? 1 : C::KS];
#pragma unroll
  for (int x = 0; x < C::KS; ++x) kf[x] = load8(kg + 16 * x + 8 * hf, valid);
  if constexpr (C::kValuesInLds) {
    copy_rows<C::RB, kRows>(lds + 2 * STAGE, (const unsigned char*)a.v.at + (s.first * a.v.token + hk * a.v.head) * 2,
                            (uint32_t)(a.v.token * 2), tile * kRows, s.n - 1, w, lane);
  } else {
#pragma unroll
    for (int x = 0; x < C::KS; ++x) vf[x] = load8(vg + 16 * x + 8 * hf, valid);
  }

  const uint32_t q_row = row_operand<C::RB>(lane, 0), o_row = BYTES + row_operand<C::RB>(lane, 0);
  const uint32_t q_col0 = col_operand<C::RB>(lane, 0, 0), q_col1 = col_operand<C::RB>(lane, 0, 1);
  const uint32_t v_row = 2 * STAGE + w * 32 * C::RB + row_operand<C::RB>(lane, 0);
  const float c2 = a.scale * kLog2e;
  f32x16 dk[C::DT], dv[C::DT];
#pragma unroll
  for (int c = 0; c < C::DT; ++c) {
    fill(dk[c], 0.f);
    fill(dv[c], 0.f);
  }

  auto copy = [&](int g, int i, int buf) {
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));
    const int h = hk * group + g;
    const unsigned char* t = lds + buf * STAGE;
    copy_rows<C::RB, QB>(t, (const unsigned char*)a.q.at + (s.first * a.q.token + h * a.q.head) * 2, (uint32_t)(a.q.token * 2), i,
                         s.n - 1, w, lane_o);
    copy_rows<C::RB, QB>(t + BYTES, (const unsigned char*)a.dout.at + (s.first * a.dout.token + h * a.dout.head) * 2,
                         (uint32_t)(a.dout.token * 2), i, s.n - 1, w, lane_o);
    // 2 QB statistics: QB / 32 copies of 64
    if (w < QB / 32) {
      const int at = w * 64 + lane_o;  // row at / QB of query i + at % QB
      const float* rows = a.rows + (int64_t)(at / QB * a.heads + h) * a.tokens + s.first + min(i + at % QB, s.n - 1);
      dma4_at(rows, (const unsigned char*)(stat[buf] + w * 64));
    }
  };
  // 32 queries; q0: the query of this lane's first register
  auto work = [&](uint32_t t, const float* st, bool masked, int q0) {
    uint32_t qr = q_row + t, orow = o_row + t, qc0 = q_col0 + t, qc1 = q_col1 + t, vr = v_row;
    asm volatile("" : "+v"(qr), "+v"(orow), "+v"(qc0), "+v"(qc1), "+v"(vr));
    auto row = [&](int x) { return x < C::KS ? read_row(lds + row_step(qr, x)) : read_row(lds + row_step(orow, x - C::KS)); };
    auto value = [&](int y) { return read_row(lds + row_step(vr, y)); };
    auto col = [&](int x) {  // of the products of 16 queries: dV's column tiles (of dO), then dK's (of Q)
      const int y = x % (2 * C::DT), at = 16 * (x / (2 * C::DT)) * C::RB + (y < C::DT ? BYTES : 0);
      return read_cols(lds + col_step(qc0, y % C::DT) + at, lds + col_step(qc1, y % C::DT) + at);
    };
    f32x16 sc, dp;
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sc[4 * q4 + e] = st[8 * q4 + e];
        dp[4 * q4 + e] = st[QB + 8 * q4 + e];
      }
    float p[16], ds[16];
    bf16x8 ring[kAhead], vring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) ring[x] = row(x);
#pragma unroll
    for (int x = 0; x < 2 * C::KS; ++x) {
      if (x < C::KS)
        sc = mfma(ring[x % kAhead], kf[x], sc);
      else
        dp = mfma(ring[x % kAhead], C::kValuesInLds ? vring[x % kAhead] : vf[C::kValuesInLds ? 0 : x - C::KS], dp);
      if (x + kAhead < 2 * C::KS) {
        ring[x % kAhead] = row(x + kAhead);
        if (C::kValuesInLds && x + kAhead >= C::KS) vring[x % kAhead] = value(x + kAhead - C::KS);
      }
      if (x >= C::KS) {
        constexpr int PER = 16 / C::KS;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int v = (x - C::KS) * PER + e;
          p[v] = __builtin_amdgcn_exp2f(sc[v] * c2);
        }
      }
    }
    bf16x8 cring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) cring[x] = col(x);
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int q = q0 + 8 * (v >> 2) + (v & 3);
        if (q < from || q >= s.n) p[v] = 0.f;
      }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) ds[v] = p[v] * dp[v];
    const bf16x8 pw[2] = {pack8(p), pack8(p + 8)}, dw[2] = {pack8(ds), pack8(ds + 8)};
#pragma unroll
    for (int x = 0; x < 4 * C::DT; ++x) {
      const int y = x % (2 * C::DT), c = y % C::DT;
      if (y < C::DT)
        dv[c] = mfma(cring[x % kAhead], pw[x / (2 * C::DT)], dv[c]);
      else
        dk[c] = mfma(cring[x % kAhead], dw[x / (2 * C::DT)], dk[c]);
      if (x + kAhead < 4 * C::DT) cring[x % kAhead] = col(x + kAhead);
    }
  };
  int g = (int)(u0 / q_tiles), i = first + (int)(u0 - (int64_t)g * q_tiles) * QB, buf = 0;
  int64_t u = u0;
  if (u < u1) copy(g, i, 0);
  for (; u < u1; ++u) {
    const int i0 = i;
    i += QB;
    if (i >= s.n) {
      i = first;
      ++g;
    }
    WA_WAIT_VM(0);
    WA_BARRIER();
    if (u + 1 < u1) copy(g, i, buf ^ 1);
    int end = QB;
    asm volatile("" : "+s"(end));
#pragma unroll 1
    for (int half = 0; half < end; half += 32) {
      const int i1 = i0 + half;
      if (i1 + 32 <= some || i1 >= s.n) continue;
      work(buf * STAGE + half * C::RB, stat[buf] + half + 4 * hf, !whole || i1 < all || i1 + 32 > s.n, i1 + 4 * hf);
    }
    buf ^= 1;
  }
  if (!valid) return;
  if (a.parts > 1) {
    float* to = a.part + (((int64_t)part * a.tokens + tok) * a.kv_heads + hk) * 2 * D;
    store_part(to, dk, a.scale, hf);
    store_part(to + D, dv, 1.f, hf);
  } else {
    store_row((uint16_t*)a.dk.at + tok * a.dk.token + hk * a.dk.head, dk, a.scale, hf);
    store_row((uint16_t*)a.dv.at + tok * a.dv.token + hk * a.dv.head, dv, 1.f, hf);
  }
}

// Adds the parts' results in order and rounds: a thread four columns of a row (D of dK, then D of dV).
template <int D>
__global__ __launch_bounds__(256) void packed_parts_kernel(const WaSeqLaunch a) {
  constexpr int QUADS = 2 * D / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / QUADS, tok = row / a.kv_heads;
  const int hk = (int)(row - tok * a.kv_heads), c = (int)(id % QUADS) * 4;
  if (tok < min(max(a.starts[0], 0), a.tokens) || tok >= min(max(a.starts[a.batch], 0), a.tokens)) return;
  const int64_t step = (int64_t)a.tokens * a.kv_heads * 2 * D;
  const float* at = a.part + row * 2 * D + c;
  float4 sum = *(const float4*)at;
#pragma unroll 4
  for (int x = 1; x < a.parts; ++x) {
    const float4 y = *(const float4*)(at + x * step);
    sum.x += y.x;
    sum.y += y.y;
    sum.z += y.z;
    sum.w += y.w;
  }
  uint16_t* out = c < D ? (uint16_t*)a.dk.at + tok * a.dk.token + hk * a.dk.head + c
                        : (uint16_t*)a.dv.at + tok * a.dv.token + hk * a.dv.head + c - D;
  *(uint2*)out = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
}

template <int D>
hipError_t launch(const WaSeqLaunch& a, hipStream_t stream) {
  const int64_t tiles = wa_packed_backward_tiles(a);
  hipLaunchKernelGGL(packed_dq_kernel<D>, dim3((unsigned)(tiles * a.heads)), dim3(64 * kWaves), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(packed_dkv_kernel<D>, dim3((unsigned)(tiles * a.kv_heads * a.parts)), dim3(64 * kWaves), 0, stream, a);
  if ((e = hipGetLastError()) != hipSuccess || a.parts == 1) return e;
  const int64_t threads = (int64_t)a.tokens * a.kv_heads * (2 * D / 4);
  hipLaunchKernelGGL(packed_parts_kernel<D>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// Sequences of n_b tokens have sum ceil(n_b / 128) tiles.
int64_t wa_packed_backward_tiles(const WaSeqLaunch& a) {
  return std::min<int64_t>(a.tokens, ((int64_t)a.tokens + (int64_t)(kRows - 1) * a.batch) / kRows);
}

// Parts of a tile of keys: as many as fill the 512 workgroups that the chip holds about once, twice where tiles are of
// different lengths, each of at least 256 queries of the longest that a sequence can be.
int32_t wa_packed_backward_parts(const WaSeqLaunch& a) {
  const int64_t items = std::max<int64_t>(1, ((int64_t)a.tokens + kRows - 1) / kRows * a.kv_heads);
  const int64_t queries = (int64_t)(a.heads / a.kv_heads) * a.tokens;
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>(1024 / items, std::min<int64_t>(queries / 256, 16)));
}

hipError_t wa_launch_packed_backward(const WaSeqLaunch& a, hipStream_t stream) {
  return a.head_dim == 64 ? launch<64>(a, stream) : launch<128>(a, stream);
}
