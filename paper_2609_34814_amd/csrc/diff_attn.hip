// Differential attention forward for gfx950 (MI355X): per head two softmax maps over the same kept keys,
//   O = P_1 V - lam_h P_2 V,   P_m = softmax(scale Q_m K_m^T).
//
// One workgroup computes one tile of 32 W query rows (W = 1, 2, 4) of both maps: W wavefronts a map, 32 rows each, so the V
// tile is read from memory once for both and the maps meet in LDS when the keys are done. In one pass over the keys, a
// tile of KB at a time (copied into LDS while the one before is worked on), a wavefront computes
//   S^T = K_m Q_m^T (v_mfma_f32_32x32x16_bf16: keys in registers, one query a lane), the running maximum and sum of its
//   queries, P^T rounded to bf16, and O_m^T += V^T P^T, whose operand P^T is in the registers that S^T came out in.
// Scores, maxima, sums and O are float32; P is rounded to bf16 because the matrix cores multiply that (half a step, 2^-9 of each
// probability, averages out over the keys of a row).
//
// Running maximum: O and l are rescaled only when a row's maximum grows by more than 2^8: probabilities up to 2^8 keep
// their bf16 and float32 precision, and after a row's first tiles it hardly ever happens.
//
// Few rows (tokens of a decoding step): the rows of all heads that share a key head fill one tile, and the keys are
// split over workgroups whose partial results a second kernel joins in key order, so a result does not depend on
// the order in which workgroups run.
//
// What bounds it: many rows of d 128, values 256 the power limit (2 x 8 heads of 4,096 tokens 392 us alone, 1.05 PFLOP/s, matrix
// cores 50% busy at 2.0 GHz; 441 in a row); of d 64 the exponentials beside the few products (values 64, 16 heads: 301 us,
// 0.91 PFLOP/s, vector unit 70% busy, matrix cores 44%); few rows the memory (one token of 16 sequences, 201 MB of keys and values:
// 36 us, 5.6 TB/s, and 4 for the join).

#include "diff_tiles.h"
#include "wavealign.h"

#include <algorithm>
#include <cmath>

namespace {

using namespace wa;

constexpr float kGrow = 8.f;  // log2 units
constexpr int kAheadRows = 4, kAheadCols = 4;  // operands read ahead
constexpr int kMaxSplits = 128, kFewSplits = 4;

template <int D, int DV, int W>
struct Fwd {
  // 64 keys a tile with four wavefronts a map (two tiles of 64 KiB for D 128, DV 256); with fewer, 32, so that two
  // workgroups fit a compute unit.
  static constexpr int KB = W == 4 ? 64 : 32;
  static constexpr int NWV = 2 * W;
  static constexpr int KRB = D * 2, VRB = DV * 2;
  static constexpr int KBYTES = KB * KRB, VBYTES = KB * VRB, STAGE = 2 * KBYTES + VBYTES;
  static constexpr int KT = KB / 32, DT = DV / 32, KS = D / 16;
  // Two tiles are held. More on their way (3 or 4 where they fit) took as long or longer, since they displace workgroups: one
  // token of 16 sequences 37, 38 and 41 us, 2 x 16 heads of 4,096 tokens (d 64, values 64) 353, 360 and 431 us.
  static_assert(W * 32 * DV * 4 <= 2 * STAGE, "the maps are joined in the tiles' memory");
};

template <int D, int DV, int W>
__global__ __launch_bounds__(128 * W, 2) void diff_fwd_kernel(const WaDiffLaunch a, const WaDiffPlan p) {
  using C = Fwd<D, DV, W>;
  constexpr int KB = C::KB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * C::STAGE];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int map = w / W, slice = w % W;

  Task task;
  if (!take_task<D == 64 && DV == 64 ? 2 : 1>(a, p.tiles, p.units, p.splits, a.causal, &task)) return;
  const int unit = task.unit, tile = task.tile;
  const int per_key_head = a.heads / a.kv_heads;
  const int heads = p.packed ? a.kv_heads : a.heads;
  const int b = unit / heads;
  const int hk = p.packed ? unit % heads : unit % heads / per_key_head;

  const int row = tile * 32 * W + slice * 32 + l32;
  const int sub = p.packed ? row / a.q_len : 0;
  const int h = p.packed ? hk * per_key_head + sub : unit % heads;
  const int i = row - sub * a.q_len;
  const bool valid = p.packed ? sub < per_key_head : i < a.q_len;

  // limits: of this lane's query, of the wavefront's (all below `some`, all at or past `all`), of the workgroup's
  const int start = start_of(a, b), keys = keys_of(a, b, start);
  const int limit = valid ? key_limit(a, keys, start, i) : 0;
  const int i0 = tile * 32 * W + slice * 32;  // not packed: the wavefront's first query
  const int i_last = a.q_len - 1;
  const int some = p.packed ? key_limit(a, keys, start, i_last) : i0 > i_last ? 0 : key_limit(a, keys, start, min(i0 + 31, i_last));
  const int all = key_limit(a, keys, start, p.packed ? 0 : min(i0, i_last));
  const int most = key_limit(a, keys, start, p.packed ? i_last : min(tile * 32 * W + 32 * W - 1, i_last));
  const unsigned char* kg[2];
#pragma unroll
  for (int m = 0; m < 2; ++m)
    kg[m] = (const unsigned char*)a.k + (((int64_t)b * 2 * a.kv_heads + 2 * hk + m) * a.kv_len) * C::KRB;
  const unsigned char* vg = (const unsigned char*)a.v + (((int64_t)b * a.kv_heads + hk) * a.kv_len) * C::VRB;

  MaskWalk walk;
  const int shift = a.block == 128 ? 7 : 6;
  if (a.mask) {
    walk.at = a.mask + (((int64_t)b * a.heads + h) * a.mb + (tile * 32 * W >> shift)) * a.nb;
    walk.at = uniform_ptr(walk.at);
  }
  int lo, hi;  // this workgroup's keys
  chunk_keys<KB>(a, task, walk, most, lane, &lo, &hi);
  walk.entries = (hi + a.block - 1) >> shift;
  // first kept tile at or past `key`, a multiple of KB
  auto next_tile = [&](int key) {
    if (!a.mask || (key & (a.block - 1))) return key;
    return walk.next(key >> shift, lane) << shift;
  };
  auto copy = [&](int key, int buf) {
    const unsigned char* t = lds + buf * C::STAGE;
    copy_tile<C::KRB, KB, C::NWV>(t, kg[0], key, keys - 1, w, lane);
    copy_tile<C::KRB, KB, C::NWV>(t + C::KBYTES, kg[1], key, keys - 1, w, lane);
    copy_tile<C::VRB, KB, C::NWV>(t + 2 * C::KBYTES, vg, key, keys - 1, w, lane);
  };

  const uint32_t kbase = map * C::KBYTES + row_operand<C::KRB>(lane, 0);
  const uint32_t vbase0 = 2 * C::KBYTES + col_operand<C::VRB>(lane, 0, 0), vbase1 = 2 * C::KBYTES + col_operand<C::VRB>(lane, 0, 1);

  const float c2 = a.scale * kLog2e;
  f32x16 acc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  bf16x8 qf[C::KS];
  auto work = [&](int key, uint32_t t) {
    // The operands' offsets are taken from their first in every tile, whose place is added before, one exclusive or each (opaque, so
    // that all of them are not held all along).
    uint32_t kb = kbase + t, vb0 = vbase0 + t, vb1 = vbase1 + t;
    asm volatile("" : "+v"(kb), "+v"(vb0), "+v"(vb1));
    auto row = [&](int x) { return read_row(lds + row_step(kb, x / C::KT) + x % C::KT * 32 * C::KRB); };
    auto col = [&](int x) {  // column tile x mod DT of 16 keys
      const int at = x / C::DT * 16 * C::VRB + (x % C::DT >> 2) * 256;
      return read_cols(lds + col_step(vb0, x % C::DT & 3) + at, lds + col_step(vb1, x % C::DT & 3) + at);
    };
    // Operands are read ahead of the products; fences keep the order written here (the scheduler sinks each read to its product).
    f32x16 s[C::KT];
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kt][v] = 0.f;
    constexpr int ROWS = C::KS * C::KT, COLS = 2 * C::KT * C::DT;
    bf16x8 ring[kAheadRows];
#pragma unroll
    for (int x = 0; x < kAheadRows; ++x) ring[x] = row(x);
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      WA_SCHED_FENCE();
      s[x % C::KT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[x % kAheadRows], qf[x / C::KT], s[x % C::KT], 0, 0, 0);
      if (x + kAheadRows < ROWS) ring[x % kAheadRows] = row(x + kAheadRows);
    }
    WA_SCHED_FENCE();
    bf16x8 cring[kAheadCols];
#pragma unroll
    for (int x = 0; x < kAheadCols; ++x) cring[x] = col(x);
    WA_SCHED_FENCE();
    if (key + KB > all) {
      const int rest = limit - key - 4 * hf;
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (kt * 32 + 8 * (v >> 2) + (v & 3) >= rest) s[kt][v] = -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, s[kt][v]);
    top = max_halves(top) * c2;
    const bool grow = top > m_run + kGrow;  // also from -inf; a row that has seen no key keeps -inf
    if (__ballot(grow)) {
      const float m_new = grow ? top : m_run;
      const float f = grow ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
      m_run = m_new;
      l_run *= f;
#pragma unroll
      for (int t2 = 0; t2 < C::DT; ++t2)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[t2][v] *= f;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    uint32_t pk[2 * C::KT][4];
    auto pair = [&](int k16, int j) {  // probabilities 2 j and 2 j + 1 of the lane's 8 of 16 keys
      const f32x16& x = s[k16 >> 1];
      const int v = 8 * (k16 & 1) + 2 * j;
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[v], c2, -ref));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[v + 1], c2, -ref));
      l_run += p0 + p1;
      pk[k16][j] = pack_bf16x2(p0, p1);
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) pair(0, j);
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      WA_SCHED_FENCE();
      const int k16 = x / C::DT, dt = x % C::DT;
      acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          cring[x % kAheadCols], as_bf16x8(make_uint4(pk[k16][0], pk[k16][1], pk[k16][2], pk[k16][3])), acc[dt], 0, 0, 0);
      if (x + kAheadCols < COLS) cring[x % kAheadCols] = col(x + kAheadCols);
#pragma unroll
      for (int j = 0; j < 4; ++j)  // the next 16 keys' probabilities beside this product
        if (k16 + 1 < 2 * C::KT && dt == j * C::DT / 4) pair(k16 + 1, j);
    }
    WA_SCHED_FENCE();
  };

  const uint16_t* qg = (const uint16_t*)a.q + (((int64_t)b * 2 * a.heads + 2 * h + map) * a.q_len + i) * D;
#pragma unroll
  for (int s = 0; s < C::KS; ++s) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (valid) u = *(const uint4*)(qg + 16 * s + 8 * hf);
    qf[s] = as_bf16x8(u);
  }

  int key = lo < hi ? next_tile(lo) : hi, buf = 0;
  if (key < hi) copy(key, 0);
  while (key < hi) {
    const int next = next_tile(key + KB);
    WA_WAIT_VM(0);  // this wavefront's part of the tile has arrived (and the queries, so that nothing waits for them below)
    WA_BARRIER();   // everyone's has, and everyone is done with the other buffer
    if (next < hi) copy(next, buf ^ 1);
    if (key < some) work(key, buf * C::STAGE);
    key = next;
    buf ^= 1;
  }

  const float l = add_halves(l_run);
  if (task.chunks > 1) {
    if (!valid) return;
    const int64_t rows = 32 * W, at = (task.part * 2 + map) * rows + slice * 32 + l32;
    float* out = a.part + at * DV;
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        *(float4*)(out + dt * 32 + 2 * v + 4 * hf) = make_float4(acc[dt][v], acc[dt][v + 1], acc[dt][v + 2], acc[dt][v + 3]);
    if (hf == 0) {
      float2* stat = (float2*)(a.part + a.part_tiles * 2 * rows * DV);
      stat[at] = make_float2(m_run, l);
    }
    return;
  }

  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[dt][v] *= inv;
  if (a.maps) {
    float big = 0.f;
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) big = fmaxf(big, fabsf(acc[dt][v]));
    const RowStats r = row_stats(m_run, l, max_halves(big));
    const float per_step = steps_per_unit(r.step);
    const int64_t at = ((int64_t)b * 2 * a.heads + 2 * h + map) * a.q_len + i;
    if (valid) {
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *(uint2*)(a.maps + at * DV + dt * 32 + 2 * v + 4 * hf) =
              make_uint2(pack_steps(acc[dt][v], acc[dt][v + 1], per_step), pack_steps(acc[dt][v + 2], acc[dt][v + 3], per_step));
      if (hf == 0) {
        a.stats[3 * at] = r.lse;
        a.stats[3 * at + 1] = r.step;
        a.stats[3 * at + 2] = r.factor;
      }
    }
  }
  // the second map's wavefronts hand their rows to the first's
  float* meet = (float*)lds + slice * 32 * DV;
  __syncthreads();
  if (map == 1) {
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) meet[(dt * 16 + v) * 64 + lane] = acc[dt][v];
  }
  __syncthreads();
  if (map == 1 || !valid) return;
  const float lam = a.lam[h];
  uint16_t* out = (uint16_t*)a.o + (((int64_t)b * a.heads + h) * a.q_len + i) * DV + 4 * hf;
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; v += 4) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = acc[dt][v + e] - lam * meet[(dt * 16 + v + e) * 64 + lane];
      *(uint2*)(out + dt * 32 + 2 * v) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    }
}

// The end of a row whose maps are whole: cols holds both maps' `E` columns from c on. top, l: of both maps; big: the
// largest of the row's columns on every lane.
template <int E, typename COLS>
__device__ __forceinline__ void finish_row(const WaDiffLaunch& a, const COLS (&o)[2], const float (&top)[2], const float (&l)[2],
                                           const float (&big)[2], int64_t bh, int i, int c, bool first) {
  const int dv = a.value_dim;
  if (a.maps) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const RowStats s = row_stats(top[m], l[m], big[m]);
      const float per_step = steps_per_unit(s.step);
      const int64_t to = (2 * bh + m) * a.q_len + i;
#pragma unroll
      for (int e = 0; e < E; ++e) a.maps[to * dv + c + e] = (int16_t)rintf(o[m][e] * per_step);
      if (first) {
        a.stats[3 * to] = s.lse;
        a.stats[3 * to + 1] = s.step;
        a.stats[3 * to + 2] = s.factor;
      }
    }
  }
  const float lam = a.lam[bh % a.heads];
  __bf16* out = (__bf16*)a.o + (bh * a.q_len + i) * dv + c;
#pragma unroll
  for (int e = 0; e < E; ++e) out[e] = (__bf16)(o[0][e] - lam * o[1][e]);
}

// Where a row's partial results lie: range c of map m at at + (2 c + m) rows, in rows of DV floats (or one float2 of
// statistics).
struct PartRow {
  int64_t bh, at;
  int i, rows;
  const float2* stat;
  __device__ __forceinline__ PartRow(const WaDiffLaunch& a, const WaDiffPlan& p, int64_t r, int dv) {
    i = r % a.q_len;
    bh = r / a.q_len;
    const int per_key_head = a.heads / a.kv_heads, h = bh % a.heads;
    const int64_t unit = p.packed ? bh / a.heads * a.kv_heads + h / per_key_head : bh;
    const int row = p.packed ? h % per_key_head * a.q_len + i : i;
    rows = 32 * p.waves;
    at = (unit * p.tiles + row / rows) * p.splits * 2 * rows + row % rows;
    stat = (const float2*)(a.part + a.part_tiles * 2 * rows * dv);
  }
};

// Joins the key ranges of split tiles, in a fixed order. Few ranges: four columns a lane, DV / 4 lanes a row, every lane with the
// row's weights.
template <int DV>
__global__ __launch_bounds__(256) void diff_join_few_kernel(const WaDiffLaunch a, const WaDiffPlan p) {
  typedef float cols __attribute__((ext_vector_type(4)));
  constexpr int L = DV / 4;
  const int64_t r = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  if (r >= (int64_t)a.batch * a.heads * a.q_len) return;
  const int lane = threadIdx.x % L;
  const PartRow row(a, p, r, DV);
  cols o[2];
  float top[2], l[2], big[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    float2 s[kFewSplits];
    cols x[kFewSplits];
#pragma unroll
    for (int c = 0; c < kFewSplits; ++c) {  // past the last range the last again, without weight
      const int64_t at = row.at + (2 * min(c, p.splits - 1) + m) * row.rows;
      s[c] = row.stat[at];
      x[c] = *(const cols*)(a.part + at * DV + 4 * lane);
    }
    top[m] = -INFINITY;
#pragma unroll
    for (int c = 0; c < kFewSplits; ++c) top[m] = fmaxf(top[m], s[c].x);
    l[m] = 0.f;
    o[m] = 0.f;
#pragma unroll
    for (int c = 0; c < kFewSplits; ++c) {
      if (c < p.splits) {
        const float f = s[c].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s[c].x - top[m]);
        l[m] += f * s[c].y;
        o[m] += x[c] * f;
      }
    }
    o[m] *= l[m] > 0.f ? 1.f / l[m] : l[m] == 0.f ? 0.f : NAN;
    big[m] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) big[m] = fmaxf(big[m], fabsf(o[m][e]));
    if (a.maps)
      for (int y = L / 2; y > 0; y >>= 1) big[m] = fmaxf(big[m], __shfl_xor(big[m], y));
  }
  finish_row<4>(a, o, top, l, big, row.bh, row.i, 4 * lane, lane == 0);
}

// Many ranges: a workgroup of R wavefronts a row, each taking every R-th range, DV / 64 columns a lane. 4 wavefronts, or 16 where
// there are more than 16 ranges (8 rows of 64 ranges of 256 columns: 8.7 us with 4, 7.9 with 16).
template <int DV, int R>
__global__ __launch_bounds__(64 * R) void diff_join_many_kernel(const WaDiffLaunch a, const WaDiffPlan p) {
  constexpr int E = DV / 64;
  typedef float cols __attribute__((ext_vector_type(E)));
  __shared__ float weight[2][kMaxSplits];
  __shared__ cols sums[R][2][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const PartRow row(a, p, blockIdx.x, DV);
  float top[2], l[2], big[2];
  cols o[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    float2 s[kMaxSplits / 64];  // a range a lane
    top[m] = -INFINITY;
#pragma unroll
    for (int x = 0; x < kMaxSplits / 64; ++x) {
      const int c = lane + 64 * x;
      s[x] = c < p.splits ? row.stat[row.at + (2 * c + m) * row.rows] : make_float2(-INFINITY, 0.f);
      top[m] = fmaxf(top[m], s[x].x);
    }
    for (int x = 32; x > 0; x >>= 1) top[m] = fmaxf(top[m], __shfl_xor(top[m], x));
    l[m] = 0.f;
#pragma unroll
    for (int x = 0; x < kMaxSplits / 64; ++x) {
      const float f = s[x].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s[x].x - top[m]);
      if (w == 0 && lane + 64 * x < p.splits) weight[m][lane + 64 * x] = f;
      l[m] += f * s[x].y;
    }
    for (int x = 32; x > 0; x >>= 1) l[m] += __shfl_xor(l[m], x);
    o[m] = 0.f;
  }
  __syncthreads();
#pragma unroll 4
  for (int c = w; c < p.splits; c += R)
#pragma unroll
    for (int m = 0; m < 2; ++m) o[m] += *(const cols*)(a.part + (row.at + (2 * c + m) * row.rows) * DV + lane * E) * weight[m][c];
#pragma unroll
  for (int m = 0; m < 2; ++m) sums[w][m][lane] = o[m];
  __syncthreads();
  if (w) return;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    for (int x = 1; x < R; ++x) o[m] += sums[x][m][lane];
    o[m] *= l[m] > 0.f ? 1.f / l[m] : l[m] == 0.f ? 0.f : NAN;
    big[m] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) big[m] = fmaxf(big[m], fabsf(o[m][e]));
    if (a.maps)
      for (int x = 32; x > 0; x >>= 1) big[m] = fmaxf(big[m], __shfl_xor(big[m], x));
  }
  finish_row<E>(a, o, top, l, big, row.bh, row.i, lane * E, lane == 0);
}

// The same for the cut tiles of a list of tasks: four columns a lane, DV / 4 lanes a row.
template <int DV>
__global__ __launch_bounds__(256) void diff_join_cut_kernel(const WaDiffLaunch a, const WaDiffPlan p) {
  typedef float cols __attribute__((ext_vector_type(4)));
  constexpr int L = DV / 4, PER = 256 / L;
  const int lane = threadIdx.x % L, rows = 32 * p.waves, all = a.tasks[1] * rows;
  const int4* cuts = (const int4*)(a.tasks + wa_diff_cut_list(a.task_items, wa_diff_slots(p.waves)));
  const float2* stat = (const float2*)(a.part + a.part_tiles * 2 * rows * DV);
  for (int r = blockIdx.x * PER + threadIdx.x / L; r < all; r += gridDim.x * PER) {
    const int4 e = cuts[r / rows];
    const int64_t bh = e.x / p.tiles;
    const int i = e.x % p.tiles * rows + r % rows;
    if (i >= a.q_len) continue;
    cols o[2];
    float top[2], l[2], big[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      auto at = [&](int c) { return ((int64_t)(e.z + c) * 2 + m) * rows + r % rows; };
      top[m] = -INFINITY;
      for (int c = 0; c < e.y; ++c) top[m] = fmaxf(top[m], stat[at(c)].x);
      l[m] = 0.f;
      o[m] = 0.f;
#pragma unroll 4
      for (int c = 0; c < e.y; ++c) {
        const float2 s = stat[at(c)];
        const float f = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - top[m]);
        l[m] += f * s.y;
        o[m] += *(const cols*)(a.part + at(c) * DV + 4 * lane) * f;
      }
      o[m] *= l[m] > 0.f ? 1.f / l[m] : l[m] == 0.f ? 0.f : NAN;
      big[m] = 0.f;
#pragma unroll
      for (int x = 0; x < 4; ++x) big[m] = fmaxf(big[m], fabsf(o[m][x]));
      if (a.maps)
        for (int y = L / 2; y > 0; y >>= 1) big[m] = fmaxf(big[m], __shfl_xor(big[m], y));
    }
    finish_row<4>(a, o, top, l, big, bh, i, 4 * lane, lane == 0);
  }
}

template <int D, int DV>
hipError_t launch_dims(WaDiffLaunch a, const WaDiffPlan& p, hipStream_t stream) {
  const int64_t items = (int64_t)p.units * p.tiles;
  const int slots = wa_diff_slots(p.waves);
  if (a.mask && p.splits == 1 && wa_diff_has_tasks(items)) {
    a.task_items = (int32_t)items;
    a.part_tiles = 2 * slots;
    const hipError_t e = wa_launch_diff_tasks(a, false, slots, stream);
    if (e != hipSuccess) return e;
  } else {
    a.tasks = nullptr;
    a.part_tiles = items * p.splits;
  }
  const int64_t grid = a.tasks ? items + slots : items * p.splits;
  const dim3 g((unsigned)grid), t(128 * p.waves);
  if (p.waves == 1) hipLaunchKernelGGL((diff_fwd_kernel<D, DV, 1>), g, t, 0, stream, a, p);
  if (p.waves == 2) hipLaunchKernelGGL((diff_fwd_kernel<D, DV, 2>), g, t, 0, stream, a, p);
  if (p.waves == 4) hipLaunchKernelGGL((diff_fwd_kernel<D, DV, 4>), g, t, 0, stream, a, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (p.splits == 1 && !a.tasks)) return e;
  const int64_t rows = (int64_t)a.batch * a.heads * a.q_len;
  if (a.tasks) {
    hipLaunchKernelGGL(diff_join_cut_kernel<DV>, dim3(1024), dim3(256), 0, stream, a, p);
  } else if (p.splits > 16) {
    hipLaunchKernelGGL((diff_join_many_kernel<DV, 16>), dim3((unsigned)rows), dim3(1024), 0, stream, a, p);
  } else if (p.splits > kFewSplits) {
    hipLaunchKernelGGL((diff_join_many_kernel<DV, 4>), dim3((unsigned)rows), dim3(256), 0, stream, a, p);
  } else {
    constexpr int PER = 256 / (DV / 4);
    hipLaunchKernelGGL(diff_join_few_kernel<DV>, dim3((unsigned)((rows + PER - 1) / PER)), dim3(256), 0, stream, a, p);
  }
  return hipGetLastError();
}

}  // namespace

WaDiffPlan wa_diff_plan(const WaDiffLaunch& a, bool masked) {
  WaDiffPlan p{};
  const int per_key_head = a.heads / a.kv_heads;
  // Heads that share keys share a tile while one head's queries would leave most of it empty; a mask is a head's own.
  p.packed = !masked && per_key_head > 1 && a.q_len <= 32;
  const int64_t rows = p.packed ? (int64_t)per_key_head * a.q_len : a.q_len;
  p.waves = rows <= 32 ? 1 : rows <= 64 || (masked && a.block == 64) ? 2 : 4;
  p.units = a.batch * (p.packed ? a.kv_heads : a.heads);
  p.tiles = (int32_t)((rows + 32 * p.waves - 1) / (32 * p.waves));
  // Key ranges: as many as keep 256 compute units busy (two workgroups each of less than four wavefronts a map), of
  // 256 keys at least.
  const int64_t slots = p.waves == 4 ? 256 : 512, items = (int64_t)p.units * p.tiles;
  p.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(slots / items, kMaxSplits), a.kv_len / 256));
  return p;
}

size_t wa_diff_part_floats(const WaDiffPlan& p, bool masked, int value_dim) {
  const int64_t items = (int64_t)p.units * p.tiles;
  const int64_t tiles = p.splits > 1 ? items * p.splits : masked && wa_diff_has_tasks(items) ? 2 * wa_diff_slots(p.waves) : 0;
  return (size_t)tiles * 2 * 32 * p.waves * (value_dim + 2);
}

hipError_t wa_launch_diff_attn(const WaDiffLaunch& a, hipStream_t stream) {
  const WaDiffPlan p = wa_diff_plan(a, a.mask != nullptr);
  if (a.head_dim == 64 && a.value_dim == 64) return launch_dims<64, 64>(a, p, stream);
  if (a.head_dim == 64 && a.value_dim == 128) return launch_dims<64, 128>(a, p, stream);
  if (a.head_dim == 128 && a.value_dim == 128) return launch_dims<128, 128>(a, p, stream);
  if (a.head_dim == 128 && a.value_dim == 256) return launch_dims<128, 256>(a, p, stream);
  return hipErrorInvalidValue;
}
