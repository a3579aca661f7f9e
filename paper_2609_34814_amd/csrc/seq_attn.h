// Attention over sequences of different lengths, for gfx950 (MI355X): the new tokens of each sequence over its keys, which are
// rows of the packed tensors or lie in pages of a cache,
//   O = softmax(scale Q K^T) V,   causal: the i-th of n queries of a sequence with L keys sees the keys up to L - n + i.
//
// A tile is 32 W query rows (W wavefronts): p tokens, a power of two, of all heads that share a key head (or of one head, where
// that would leave an eighth of the rows empty), so the heads of a group read a tile of keys once. A wavefront computes, a tile
// of KB keys at a time (copied into LDS while the one before is worked on), S^T = K Q^T (v_mfma_f32_32x32x16: keys in registers, one
// query a lane), the running maximum and sum of its queries, P^T rounded to 16 bits, and O^T += V^T P^T, whose operand P^T is in the
// registers that S^T came out in. Scores, maxima, sums and O are float32; P is rounded to the inputs' type because the matrix cores
// multiply that (half a step, 2^-9 or 2^-12 of each probability, which averages out over the keys of a row).
//
// Running maximum: O and l are rescaled only when a row's maximum grows by more than 2^8: probabilities up to 2^8 keep their
// precision, and after a row's first tiles it hardly ever happens. In fp16 they are held 2^7 times larger (up to 2^15), so that
// those down to 2^-21 of the largest keep all their bits.
//
// Who computes what: the work is a line of units, one for each tile of keys of each query tile, sequence after sequence and within
// one key head after key head. Worker w of G takes the units [w U / G, (w + 1) U / G), so all workers have the same to do whatever
// the lengths are, and neighbours (on one XCD) read the same keys. The lengths are known on the device only: each workgroup sums them
// itself, a sequence a lane, and finds its place in a sequence by a closed form, which costs no launch before this one. A border within
// a sixteenth of a share of a tile's end is moved there. A tile that several workers compute is joined by a second kernel, in key order: nothing
// is added with atomics, and equal calls give equal bits.
#pragma once

#include "diff_tiles.h"
#include "seq_launch.h"
#include "wavealign.h"

namespace wa {

constexpr float kSeqGrow = 8.f;  // log2 units
constexpr int kSeqAhead = 4;     // operands read ahead

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <bool HALF>
struct SeqType;
template <>
struct SeqType<false> {
  static constexpr float kBias = 0.f;
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
  static __device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct SeqType<true> {
  static constexpr float kBias = 7.f;  // log2 units
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
  }
  static __device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

template <int D, int W>
struct SeqTile {
  // Keys a tile: 64 with four wavefronts (two workgroups a compute unit); with one, 32, so that enough workgroups fit to keep the
  // memory busy.
  static constexpr int KB = W == 4 ? 64 : 32;
  static constexpr int RB = D * 2, BYTES = KB * RB, STAGE = 2 * BYTES;
  static constexpr int KT = KB / 32, DT = D / 32, KS = D / 16;
  static constexpr int LOG_KB = W == 4 ? 6 : 5;
};

// A launch's arguments where the hardware put them. They do not fit the scalar registers beside the kernel's state: again() forgets
// what was read of them, so that they are read again (from the scalar cache) where they are used next, and not held until then.
typedef const __attribute__((address_space(4))) WaSeqLaunch* SeqArgs;
__device__ __forceinline__ SeqArgs seq_args() { return (SeqArgs)__builtin_amdgcn_kernarg_segment_ptr(); }
__device__ __forceinline__ SeqArgs again(SeqArgs a) {
  asm volatile("" : "+s"(a));
  return a;
}

// A sequence, as the device's arrays have it, taken so that no value leads out of a tensor.
struct Seq {
  int first, n, keys;  // first query's row, queries, keys
};
template <bool PAGED>
__device__ __forceinline__ Seq seq_of(SeqArgs a, int b) {
  Seq s;
  s.first = min(max(a->starts[b], 0), a->tokens);
  s.n = min(max(a->starts[b + 1], s.first), a->tokens) - s.first;
  s.keys = s.n;
  if (PAGED) s.keys = (int)min((int64_t)max(a->kv_lens[b], 0), (int64_t)a->table_width << a->page_shift);
  return s;
}

// Units of the first t tiles of a sequence and head: tile t has ceil((before + (t + 1) p) / KB) of them, at least as many as tiles
// of keys that its queries see and at least one; without `causal` all have ceil(keys / KB).
struct Line {
  int log_p, log_kb, before;
  int whole;  // units of every tile, 0: causal
  __device__ __forceinline__ Line(int log_p_, int log_kb_, const Seq& s, bool causal) : log_p(log_p_), log_kb(log_kb_) {
    before = max(s.keys - s.n, 0);
    whole = causal ? 0 : max((int)(((int64_t)s.keys + (1 << log_kb) - 1) >> log_kb), 1);
  }
  __device__ __forceinline__ int64_t upto(int64_t t) const {
    if (whole) return t * whole;
    if (log_p >= log_kb) {
      const int64_t start = ((int64_t)before + (1 << log_kb) - 1) >> log_kb;
      return t * start + ((t * (t + 1) >> 1) << (log_p - log_kb));
    }
    // p divides KB: with c = ceil(before / p) and m = KB / p, the sum of ceil(u / m) for u from c + 1 to c + t
    const int s = log_kb - log_p;
    const int64_t c = ((int64_t)before + (1 << log_p) - 1) >> log_p;
    auto sum = [&](int64_t x) {
      const int64_t q = x >> s, r = x & ((1 << s) - 1);
      return ((q * (q + 1) >> 1) << s) + r * (q + 1);
    };
    return sum(c + t) - sum(c);
  }
};

// One tile's place in the line: rows [token, token + p) of sequence b for the heads of column col.
struct Item {
  int b, col, tile, tiles;
  Seq s;
  int64_t at;  // first unit
  int units;
};

template <bool PAGED>
struct Walk {
  SeqArgs a;
  int log_kb, log_tokens, cols, lane;

  __device__ __forceinline__ Walk(SeqArgs a_, int log_kb_, int lane_)
      : a(a_), log_kb(log_kb_), log_tokens(a_->plan.log_tokens), cols(a_->heads / a_->plan.per_tile), lane(lane_) {}
  __device__ __forceinline__ Line line(const Seq& s) const { return Line(log_tokens, log_kb, s, a->causal); }
  __device__ __forceinline__ int tiles(const Seq& s) const { return (int)(((int64_t)s.n + (1 << log_tokens) - 1) >> log_tokens); }

  // units of sequence base + lane, summed over the lanes up to this one
  __device__ __forceinline__ int64_t prefix(int base, int64_t* own) const {
    int64_t x = 0;
    if (base + lane < a->batch) {
      const Seq s = seq_of<PAGED>(a, base + lane);
      x = cols * line(s).upto(tiles(s));
    }
    *own = x;
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) {
      const int64_t y = __shfl_up(x, step);
      if (lane >= step) x += y;
    }
    return x;
  }
  __device__ __forceinline__ int64_t total() const {
    int64_t sum = 0, own;
    for (int base = 0; base < a->batch; base += 64) sum += __shfl(prefix(base, &own), 63);
    return sum;
  }
  // the item that holds unit x, which is below the total
  __device__ __forceinline__ Item find(int64_t x) const {
    int64_t before = 0, own, sum = 0;
    int base = 0, who = 0;
    for (;; base += 64) {
      sum = prefix(base, &own);
      const uint64_t past = __ballot(before + sum > x);
      if (past || base + 64 >= a->batch) {
        who = past ? __builtin_ctzll(past) : 0;
        break;
      }
      before += __shfl(sum, 63);
    }
    Item it;
    it.b = min(__builtin_amdgcn_readfirstlane(base + who), a->batch - 1);
    it.at = before + __shfl(sum - own, who);
    it.s = uniform(seq_of<PAGED>(a, it.b));
    const Line l = line(it.s);
    it.tiles = tiles(it.s);
    const int64_t column = l.upto(it.tiles);
    int64_t r = x - it.at;
    it.col = (int)(r / column);
    it.at += it.col * column;
    r -= it.col * column;
    int lo = 0, hi = it.tiles;  // upto(lo) <= r < upto(hi)
    while (hi - lo > 1) {
      const int mid = lo + ((hi - lo) >> 1);
      if (l.upto(mid) <= r) lo = mid; else hi = mid;
    }
    it.tile = lo;
    it.at += l.upto(lo);
    it.units = (int)(l.upto(lo + 1) - l.upto(lo));
    scalar(it);
    return it;
  }
  // the item behind `it`; there has to be one
  __device__ __forceinline__ Item next(Item it) const {
    it.at += it.units;
    if (++it.tile == it.tiles) {
      it.tile = 0;
      if (++it.col == cols) {
        it.col = 0;
        do it.s = uniform(seq_of<PAGED>(again(a), ++it.b)); while (it.s.n == 0 && it.b + 1 < a->batch);
        it.tiles = tiles(it.s);
      }
    }
    const Line l = line(it.s);
    it.units = (int)(l.upto(it.tile + 1) - l.upto(it.tile));
    scalar(it);
    return it;
  }
  static __device__ __forceinline__ int64_t uniform64(int64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uint64_t)v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
  }
  static __device__ __forceinline__ Seq uniform(Seq s) {
    s.first = __builtin_amdgcn_readfirstlane(s.first);
    s.n = __builtin_amdgcn_readfirstlane(s.n);
    s.keys = __builtin_amdgcn_readfirstlane(s.keys);
    return s;
  }
  static __device__ __forceinline__ void scalar(Item& it) {
    it.at = uniform64(it.at);
    it.col = __builtin_amdgcn_readfirstlane(it.col);
    it.tile = __builtin_amdgcn_readfirstlane(it.tile);
    it.units = __builtin_amdgcn_readfirstlane(it.units);
  }
};

// The shares of the line: of `total` units for `workers` workers.
struct Shares {
  int64_t total, near;  // near: how far a border moves to a tile's end
  int workers;
  __device__ __forceinline__ Shares(int64_t total_, SeqArgs a) : total(total_) {
    workers = (int)max((int64_t)1, min((int64_t)a->plan.workers, total / a->plan.min_units));
    near = total / workers >> 4;
  }
  __device__ __forceinline__ int64_t border(int w) const { return total * w / workers; }
  // where the border at unit x, inside `it`, is moved to
  __device__ __forceinline__ int64_t moved(int64_t x, const Item& it) const {
    if (x - it.at <= near) return it.at;
    if (it.at + it.units - x <= near) return it.at + it.units;
    return x;
  }
  // the worker whose share holds the first unit of `it`: the last whose border is at or before it, or is moved there
  __device__ __forceinline__ int first_of(const Item& it) const {
    const int64_t limit = it.at + min(near, (int64_t)it.units - 1);
    return (int)min((int64_t)workers - 1, ((limit + 1) * workers - 1) / total);
  }
};

// Zero rows, in the place of keys behind the last and of pages that the pool does not have.
static __device__ const uint4 kZeroRow[16] = {};

// The rows of one item's keys (or values) as tiles in LDS.
template <int D, int W, bool PAGED>
struct KeyRows {
  using C = SeqTile<D, W>;
  static constexpr int RPI = 1024 / C::RB, LPR = C::RB / 16, N = C::BYTES / 1024 / W;
  const unsigned char* base;  // packed: the sequence's first row; paged: the head of page 0
  uint32_t token;             // bytes
  int64_t page;

  // Rows [key, key + KB) into `tile`; last: the last key. Rows past it are that row again, or (whole copies of paged ones) zeros: what
  // they add is masked, and they hold no memory that the caller did not write. ids: the page of each 16 keys' (below 0: none), uniform.
  __device__ __forceinline__ void copy(const unsigned char* tile, int key, int last, int w, int lane, const int* ids, int page_mask) const {
    const int r0 = lane / LPR;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (i * W + w) * RPI, r = row + r0;
      const uint32_t chunk = tile_chunk<C::RB>(r, lane % LPR) * 16;
      const unsigned char* to = tile + (i * W + w) * 1024;
      if constexpr (!PAGED) {
        dma16(uniform_ptr(base + (int64_t)key * token), min(r, last - key) * token + chunk, to);
      } else {
        const int id = ids[row / 16];
        const unsigned char* from = base + id * page + (int64_t)((key + row) & page_mask) * token;
        const bool none = id < 0 || key + row > last;
        dma16(uniform_ptr(none ? (const unsigned char*)kZeroRow : from), (none ? 0 : min(r0, last - key - row) * token) + chunk, to);
      }
    }
  }
};

template <bool HALF, int D, int W, bool PAGED>
__global__ __launch_bounds__(64 * W, 2) void seq_attn_kernel(const WaSeqLaunch) {
  using C = SeqTile<D, W>;
  using T = SeqType<HALF>;
  constexpr int KB = C::KB, R = 32 * W;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * C::STAGE];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const SeqArgs a = seq_args();
  const Walk<PAGED> walk(a, C::LOG_KB, lane);
  const Shares shares(walk.uniform64(walk.total()), a);
  if (shares.total == 0) return;
  // workgroups go round the eight XCDs: each XCD takes neighbouring shares where there are shares for all
  const int me = shares.workers == a->plan.workers ? (blockIdx.x & 7) * (a->plan.workers >> 3) + (blockIdx.x >> 3) : blockIdx.x;
  if (me >= shares.workers) return;
  int64_t begin = shares.border(me), end = shares.border(me + 1);
  if (end < shares.total) end = shares.moved(end, walk.find(end));
  Item it = walk.find(begin);
  begin = shares.moved(begin, it);
  if (begin == it.at + it.units && begin < shares.total) it = walk.next(it);
  if (begin >= end) return;

  const int per_tile = a->plan.per_tile, log_p = a->plan.log_tokens, group = a->heads / a->kv_heads;
  const bool causal = a->causal;
  const float c2 = a->scale * kLog2e;
  const uint32_t kbase = row_operand<C::RB>(lane, 0);
  const uint32_t vbase0 = C::BYTES + col_operand<C::RB>(lane, 0, 0), vbase1 = C::BYTES + col_operand<C::RB>(lane, 0, 1);
  // this lane's row of a tile: token i of head `sub`
  const int row = w * 32 + l32, sub = row >> log_p, i_row = row & ((1 << log_p) - 1);
  const int i_first = log_p >= 5 ? (w * 32) & ((1 << log_p) - 1) : 0;  // the wavefront's tokens
  const int i_last = i_first + (log_p >= 5 ? 31 : (1 << log_p) - 1);
  const bool wave_used = (w * 32 >> log_p) < per_tile;

  // the keys of a worker's part of a tile
  struct Range {
    int lo, hi, most;
  };
  auto range = [&](const Item& x) {
    Range r;
    const int last = min(((x.tile + 1) << log_p), x.s.n) - 1;
    r.most = causal ? min(max(x.s.keys - x.s.n + last + 1, 0), x.s.keys) : x.s.keys;
    const int64_t u0 = max(begin - x.at, (int64_t)0), u1 = min(end - x.at, (int64_t)x.units);
    r.lo = (int)min(u0 * KB, (int64_t)r.most);
    r.hi = (int)min(u1 * KB, (int64_t)r.most);
    return r;
  };

  // Pages of a paged item: 64 entries of its table, one a lane; bad: those that the pool does not have.
  int window = -1, entry = 0, window_b = -1;
  uint64_t bad = 0;
  // copies a tile of keys and of values; returns which 16 keys of it lie in no page
  auto copy = [&](const Item& x, int key, int buf) -> uint32_t {
    const SeqArgs a = again(seq_args());
    const unsigned char* const kall = (const unsigned char*)(PAGED ? a->kp.at : a->k.at);
    const unsigned char* const vall = (const unsigned char*)(PAGED ? a->vp.at : a->v.at);
    const unsigned char* t = lds + buf * C::STAGE;
    const int hk = per_tile == 1 ? x.col / group : x.col;
    KeyRows<D, W, PAGED> rows[2];
    uint32_t none = 0;
    int ids[KB / 16];
    if constexpr (PAGED) {
      rows[0] = {kall + hk * a->kp.head * 2, (uint32_t)(a->kp.token * 2), a->kp.page * 2};
      rows[1] = {vall + hk * a->vp.head * 2, (uint32_t)(a->vp.token * 2), a->vp.page * 2};
      const int first = key >> a->page_shift;
      if (x.b != window_b || first >> 6 != window) {
        window_b = x.b;
        window = first >> 6;
        const int e = window * 64 + lane, used = (int)(((int64_t)x.s.keys + (1 << a->page_shift) - 1) >> a->page_shift);
        entry = e < used ? a->tables[x.b * a->table_stride + e] : 0;
        bad = __ballot((uint32_t)entry >= (uint32_t)a->n_pages);
      }
#pragma unroll
      for (int j = 0; j < KB / 16; ++j) {
        const int e = (key + 16 * j) >> a->page_shift & 63;
        const bool no = bad >> e & 1;
        ids[j] = no ? -1 : __builtin_amdgcn_readlane(entry, e);
        if (no) none |= 1u << j;
      }
    } else {
      rows[0] = {kall + (x.s.first * a->k.token + hk * a->k.head) * 2, (uint32_t)(a->k.token * 2), 0};
      rows[1] = {vall + (x.s.first * a->v.token + hk * a->v.head) * 2, (uint32_t)(a->v.token * 2), 0};
    }
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));  // the copies' offsets are not held across the loop
    const int mask = (1 << a->page_shift) - 1;
    rows[0].copy(t, key, x.s.keys - 1, w, lane_o, ids, mask);
    rows[1].copy(t + C::BYTES, key, x.s.keys - 1, w, lane_o, ids, mask);
    return none;
  };

  bf16x8 qf[C::KS];
  f32x16 acc[C::DT];
  float m_run, l_run;
  // One tile of keys. limit: of the lane's query; none: 16 keys without a page.
  auto work = [&](int key, uint32_t t, int limit, bool masked, uint32_t none) {
    // The operands' offsets are taken from their first in every tile, whose place is added before, one exclusive or each (opaque, so
    // that all of them are not held all along).
    uint32_t kb = kbase + t, vb0 = vbase0 + t, vb1 = vbase1 + t;
    asm volatile("" : "+v"(kb), "+v"(vb0), "+v"(vb1));
    auto key_row = [&](int x) { return read_row(lds + row_step(kb, x / C::KT) + x % C::KT * 32 * C::RB); };
    auto col = [&](int x) {  // column tile x mod DT of 16 keys
      const int at = x / C::DT * 16 * C::RB;
      return read_cols(lds + col_step(vb0, x % C::DT) + at, lds + col_step(vb1, x % C::DT) + at);
    };
    // Operands are read ahead of the products; fences keep the order written here (the scheduler sinks each read to its product).
    f32x16 s[C::KT];
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kt][v] = 0.f;
    constexpr int ROWS = C::KS * C::KT, COLS = 2 * C::KT * C::DT;
    bf16x8 ring[kSeqAhead];
#pragma unroll
    for (int x = 0; x < kSeqAhead; ++x) ring[x] = key_row(x);
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      WA_SCHED_FENCE();
      s[x % C::KT] = T::mfma(ring[x % kSeqAhead], qf[x / C::KT], s[x % C::KT]);
      if (x + kSeqAhead < ROWS) ring[x % kSeqAhead] = key_row(x + kSeqAhead);
    }
    WA_SCHED_FENCE();
    bf16x8 cring[kSeqAhead];
#pragma unroll
    for (int x = 0; x < kSeqAhead; ++x) cring[x] = col(x);
    WA_SCHED_FENCE();
    if (masked) {
      const int rest = limit - key - 4 * hf;
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (kt * 32 + 8 * (v >> 2) + (v & 3) >= rest || (PAGED && (none >> (2 * kt + (v >> 3)) & 1))) s[kt][v] = -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, s[kt][v]);
    top = max_halves(top) * c2;
    const bool grow = top > m_run + kSeqGrow;  // also from -inf; a row that has seen no key keeps -inf
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
    const float ref = m_run == -INFINITY ? 0.f : m_run - T::kBias;
    uint32_t pk[2 * C::KT][4];
    auto pair = [&](int k16, int j) {  // probabilities 2 j and 2 j + 1 of the lane's 8 of 16 keys
      const f32x16& x = s[k16 >> 1];
      const int v = 8 * (k16 & 1) + 2 * j;
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[v], c2, -ref));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[v + 1], c2, -ref));
      l_run += p0 + p1;
      pk[k16][j] = T::pack(p0, p1);
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) pair(0, j);
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      WA_SCHED_FENCE();
      const int k16 = x / C::DT, dt = x % C::DT;
      acc[dt] = T::mfma(cring[x % kSeqAhead], as_bf16x8(make_uint4(pk[k16][0], pk[k16][1], pk[k16][2], pk[k16][3])), acc[dt]);
      if (x + kSeqAhead < COLS) cring[x % kSeqAhead] = col(x + kSeqAhead);
#pragma unroll
      for (int j = 0; j < 4; ++j)  // the next 16 keys' probabilities beside this product
        if (k16 + 1 < 2 * C::KT && dt == j * C::DT / 4) pair(k16 + 1, j);
    }
    WA_SCHED_FENCE();
  };

  int buf = 0;
  bool ready = false;      // the item's first tile is on its way
  uint32_t none = 0, none_next = 0;
  bool any_bad = false;
  Range r = range(it);
  for (;;) {
    const bool more = it.at + it.units < end;
    Item nx = it;
    Range rn = {0, 0, 0};
    if (more) {
      nx = walk.next(it);
      rn = range(nx);
    }
    // the item's queries
    const SeqArgs a = again(seq_args());
    const int token = (it.tile << log_p) + i_row;
    const bool valid = sub < per_tile && token < it.s.n;
    const int head = it.col * per_tile + sub;
    const int before = it.s.keys - it.s.n;
    const int limit = !valid ? 0 : causal ? min(max(before + token + 1, 0), it.s.keys) : it.s.keys;
    const int t0 = (it.tile << log_p) + i_first, t1 = min((it.tile << log_p) + i_last, it.s.n - 1);
    // keys that any, and that all of the wavefront's queries see
    const int some = !wave_used || t0 >= it.s.n ? 0 : causal ? min(max(before + t1 + 1, 0), it.s.keys) : it.s.keys;
    const int all = causal ? min(max(before + t0 + 1, 0), it.s.keys) : it.s.keys;
    const uint16_t* qg = (const uint16_t*)a->q.at + (it.s.first + token) * a->q.token + head * a->q.head;
    if (!ready && r.lo < r.hi) none = copy(it, r.lo, buf);
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (valid) u = *(const uint4*)(qg + 16 * s + 8 * hf);
      qf[s] = as_bf16x8(u);
    }
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
    m_run = -INFINITY;
    l_run = 0.f;
    ready = false;
    for (int key = r.lo; key < r.hi; key += KB) {
      WA_WAIT_VM(0);  // this wavefront's part of the tile has arrived (and the queries, so that nothing waits for them below)
      WA_BARRIER();   // everyone's has, and everyone is done with the other buffer
      if (key + KB < r.hi) {
        none_next = copy(it, key + KB, buf ^ 1);
      } else if (rn.lo < rn.hi) {
        none_next = copy(nx, rn.lo, buf ^ 1);
        ready = true;
      }
      if (PAGED && none) any_bad = true;
      if (key < some) work(key, buf * C::STAGE, limit, key + KB > all || (PAGED && none), none);
      none = none_next;
      buf ^= 1;
    }

    // the item's end: whole rows to O, others to the worker's partial tiles
    {
    const SeqArgs a = again(seq_args());
    const float l = add_halves(l_run);
    const float ref = m_run == -INFINITY ? -INFINITY : m_run - T::kBias;
    const bool starts = begin <= it.at, finishes = it.at + it.units <= end;
    if (valid) {
      const int64_t tok = it.s.first + token;
      if (starts && finishes) {
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
        uint16_t* out = (uint16_t*)a->o.at + tok * a->o.token + head * a->o.head + 4 * hf;
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
          for (int v = 0; v < 16; v += 4)
            *(uint2*)(out + dt * 32 + 2 * v) =
                make_uint2(T::pack(acc[dt][v] * inv, acc[dt][v + 1] * inv), T::pack(acc[dt][v + 2] * inv, acc[dt][v + 3] * inv));
        if (a->lse && hf == 0) a->lse[(int64_t)head * a->tokens + tok] = l == 0.f ? -INFINITY : (ref + __log2f(l)) * kLn2;
        if (hf == 0) a->cuts[tok * a->heads + head] = make_int2(-1, 0);
      } else {
        // slot 0: a part that begins inside its tile; slot 1: one that begins with it
        const int64_t at = ((int64_t)me * 2 + (starts ? 1 : 0)) * R + row;
        float* out = a->part + at * D;
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
          for (int v = 0; v < 16; v += 4)
            *(float4*)(out + dt * 32 + 2 * v + 4 * hf) = make_float4(acc[dt][v], acc[dt][v + 1], acc[dt][v + 2], acc[dt][v + 3]);
        if (hf == 0) {
          ((float2*)(a->part + (int64_t)a->plan.workers * 2 * R * D))[at] = make_float2(ref, l);
          if (finishes) a->cuts[tok * a->heads + head] = make_int2(shares.first_of(it) | me << 16, row);
        }
      }
    }
    }
    if (!more) break;
    it = nx;
    r = rn;
  }
  if (PAGED && any_bad && a->status && tid == 0) atomicOr(a->status, WA_PAGE_BAD_INDEX);
}

// Joins the parts of a row, in key order: parts from worker cut.x & 0xffff to cut.x >> 16. TEAM wavefronts a row, each taking every
// TEAM-th part; the lanes hold the columns.
template <bool HALF, int D, int W, int TEAM>
__global__ __launch_bounds__(256) void seq_join_kernel(const WaSeqLaunch a, int rows_per_wave) {
  using T = SeqType<HALF>;
  constexpr int R = 32 * W, E = D / 64;
  typedef float cols __attribute__((ext_vector_type(E)));
  __shared__ cols sums[TEAM == 1 ? 1 : TEAM][64];
  __shared__ float totals[TEAM == 1 ? 1 : TEAM];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t all = (int64_t)a.tokens * a.heads;
  const int64_t first = TEAM == 1 ? ((int64_t)blockIdx.x * 4 + w) * rows_per_wave : blockIdx.x;
  // tokens of sequences: what lies before the first and behind the last stays as it is, and has no cuts
  const int64_t lo = (int64_t)min(max(a.starts[0], 0), a.tokens) * a.heads, hi = (int64_t)min(max(a.starts[a.batch], 0), a.tokens) * a.heads;
  const float2* stat = (const float2*)(a.part + (int64_t)a.plan.workers * 2 * R * D);
  int2 mine = make_int2(-1, 0);
  if (lane < rows_per_wave && first + lane >= lo && first + lane < min(hi, all)) mine = a.cuts[first + lane];
  uint64_t cut = __ballot(mine.x != -1);
  while (cut) {
    const int who = __builtin_ctzll(cut);
    cut &= cut - 1;
    const int x = __builtin_amdgcn_readlane(mine.x, who), r = __builtin_amdgcn_readlane(mine.y, who) & (R - 1);
    // taken into the workers that there are: nothing that the workspace holds leads out of it
    const int begin = min(x & 0xffff, a.plan.workers - 1), end = min((int)((uint32_t)x >> 16), a.plan.workers - 1);
    auto at = [&](int c) { return ((int64_t)c * 2 + (c == begin ? 1 : 0)) * R + r; };
    float top = -INFINITY;
    for (int c = begin + lane; c <= end; c += 64) top = fmaxf(top, stat[at(c)].x);
#pragma unroll
    for (int y = 32; y > 0; y >>= 1) top = fmaxf(top, __shfl_xor(top, y));
    cols o = 0.f;
    float l = 0.f;
#pragma unroll 8
    for (int c = begin + (TEAM == 1 ? 0 : w); c <= end; c += TEAM) {
      const float2 s = stat[at(c)];
      const float f = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - top);
      l += f * s.y;
      o += *(const cols*)(a.part + at(c) * D + lane * E) * f;
    }
    if constexpr (TEAM > 1) {
      sums[w][lane] = o;
      if (lane == 0) totals[w] = l;
      __syncthreads();
      if (w) return;
      for (int y = 1; y < TEAM; ++y) {
        o += sums[y][lane];
        l += totals[y];
      }
    }
    o *= l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
    const int64_t rr = first + who, token = rr / a.heads;
    const int head = (int)(rr - token * a.heads);
    uint16_t* out = (uint16_t*)a.o.at + token * a.o.token + head * a.o.head + lane * E;
    if constexpr (E == 2) {
      *(uint32_t*)out = T::pack(o[0], o[1]);
    } else {
      *out = (uint16_t)T::pack(o[0], 0.f);
    }
    if (a.lse && lane == 0) a.lse[(int64_t)head * a.tokens + token] = l == 0.f ? -INFINITY : (top + __log2f(l)) * kLn2;
  }
}

// Rows up to which a workgroup joins one alone: many parts each. With more, their tiles are cut in few.
constexpr int64_t kSeqTeamRows = 8192;

template <bool HALF, int D, int W, bool PAGED>
hipError_t seq_launch(const WaSeqLaunch& a, hipStream_t stream) {
  hipLaunchKernelGGL((seq_attn_kernel<HALF, D, W, PAGED>), dim3(a.plan.workers), dim3(64 * W), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)a.tokens * a.heads;
  if (rows <= kSeqTeamRows) {
    hipLaunchKernelGGL((seq_join_kernel<HALF, D, W, 4>), dim3((unsigned)rows), dim3(256), 0, stream, a, 1);
  } else {
    hipLaunchKernelGGL((seq_join_kernel<HALF, D, W, 1>), dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, stream, a, 64);
  }
  return hipGetLastError();
}

template <bool PAGED>
hipError_t seq_launch_any(WaSeqLaunch a, hipStream_t stream) {
  a.plan = wa_seq_plan(a);
  const int which = (a.half ? 4 : 0) | (a.head_dim == 128 ? 2 : 0) | (a.plan.waves == 4 ? 1 : 0);
  switch (which) {
    case 0: return seq_launch<false, 64, 1, PAGED>(a, stream);
    case 1: return seq_launch<false, 64, 4, PAGED>(a, stream);
    case 2: return seq_launch<false, 128, 1, PAGED>(a, stream);
    case 3: return seq_launch<false, 128, 4, PAGED>(a, stream);
    case 4: return seq_launch<true, 64, 1, PAGED>(a, stream);
    case 5: return seq_launch<true, 64, 4, PAGED>(a, stream);
    case 6: return seq_launch<true, 128, 1, PAGED>(a, stream);
    default: return seq_launch<true, 128, 4, PAGED>(a, stream);
  }
}

}  // namespace wa
