// Attention over sequences of different lengths, for gfx950 (MI355X): the new tokens of each sequence over its keys, which are
// rows of the packed tensors or lie in pages of a cache,
//   O = softmax(scale Q K^T) V,   causal: the i-th of n queries of a sequence with L keys sees the keys up to L - n + i.
//
// A tile is 32 W query rows (W wavefronts): p tokens, a power of two, of all heads that share a key head (or of one head, where
// that would leave an eighth of the rows empty), so the heads of a group read a tile of keys once. A wavefront computes, a tile
// of KB keys at a time (copied into LDS while the one before is worked on), S^T = K Q^T (v_mfma_f32_32x32x16: keys in registers, one
// query a lane), the running maximum and sum of its queries, P^T rounded to 16 bits, and O^T += V^T P^T, whose operand P^T is in the
// registers that S^T came out in. Of four wavefronts each computes the scores of a tile of keys beside the probabilities of the one
// before, so that matrix products and exponentials of one wavefront run at the same time (32,768 tokens, 32 heads over 8, d 128: 8.2 ms where
// they take turns, 7.8 so; 8,192 tokens of 7 documents, 16 over 4, d 64: 60 us and 51); one wavefront, which waits for the memory, has them take
// turns. Scores, maxima, sums and O are float32; P is rounded to the inputs' type because the matrix cores
// multiply that (half a step, 2^-9 or 2^-12 of each probability, which averages out over the keys of a row).
//
// Running maximum: O and l are rescaled only when a row's maximum grows by more than 2^8: probabilities up to 2^8 keep their
// precision, and after a row's first tiles it hardly ever happens. In fp16 they are held 2^7 times larger (up to 2^15), so that
// those down to 2^-21 of the largest keep all their bits.
//
// Who computes what. The lengths are known on the device only; each workgroup finds its work itself from the lengths, a sequence a lane,
// which costs no launch before this one.
//   Many tiles of four wavefronts, or ones of about equal length: a workgroup a tile, of packed sequences those with the most keys first, so
//   that the chip stays full to the end, and those that run together read the same keys at about the same time (one prompt of 32,768 tokens,
//   32 heads over 8, d 128: 9.6 ms where equal shares of the work begin anywhere in a tile, 8.2 so, when both were measured).
//   Others: the work is a line of units, one for each tile of keys of each query tile and two for its beginning and end, sequence after
//   sequence and within one key head after key head. Worker w of G takes the units [w U / G, (w + 1) U / G), found by a closed form, so all
//   workers have the same to do whatever the lengths are. A border within a sixteenth of a share of a tile's end is moved there. A tile
//   that several workers compute is joined by a second kernel, in key order: nothing is added with atomics, and equal calls give equal bits.
//   Calls of few keys, and packed sequences of few tokens: a workgroup a tile, without the second kernel.
#pragma once

#include "diff_tiles.h"
#include "seq_launch.h"
#include "wavealign.h"

#include <algorithm>
#include <type_traits>

namespace wa {

constexpr float kSeqGrow = 8.f;  // log2 units
constexpr int kSeqAhead = 4;     // operands read ahead
// Tiles of four wavefronts are dealt out whole where there are so many times the workers of them, and where that takes no longer than the line, in
// which a worker's share of s units takes about 22 + 2.2 s us, with parts to store and to join (fitted at d 128, units of 64 keys).
// Causal: whole tiles, of all lengths, take 4 + 1.05 longest + 0.7 s, so where longest <= 17 + 10/7 s. 2,400 tokens of 3 prompts, 32 heads over
// 8: 59 us along the line, 44 whole; 8,192 of one, 8 heads over 1: 168 and 185.
// Not causal, or behind many cached keys, tiles are about equal, and a last round of few of them counts: it takes 0.65 of a full one if it is
// half full or less, else 0.9. 6,000 tokens of 16 heads, not causal, 752 tiles: 323 us along the line, 298 whole; 4,800, 608 tiles: 207 and 251;
// over a cache 4,096 tokens behind 12,288, 32 heads over 8: 955 and 908; 1,024 behind 7,168: 152 and 175.
// Of 21 shapes timed both ways at either d, the choice is within 6% of the better (beside the join's launch, 2 to 3 us) but for: d 64, 130 us whole
// and 111 along the line (8,192 tokens of 7 documents, 16 heads, not causal), 91 along the line and 82 whole (6,000 of 2, 12 heads, causal); d 128, 96
// whole and 88 along the line (2,400 of 3, 32 heads, not causal).
constexpr int kSeqWhole = 4, kSeqLongest = 17;

// What a tile costs beside its keys, in tiles of keys.
constexpr int kSeqFixed = 2;

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
  // Keys a tile: 64 with four wavefronts (two workgroups a compute unit); with one, 32 of 256 bytes or 64 of 128, so that enough
  // workgroups fit to keep the memory busy.
  static constexpr int KB = W == 4 || D == 64 ? 64 : 32;
  static constexpr int RB = D * 2, BYTES = KB * RB, STAGE = 2 * BYTES;
  static constexpr int KT = KB / 32, DT = D / 32, KS = D / 16;
  static constexpr int LOG_KB = KB == 64 ? 6 : 5;
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

// Units of the first t tiles of a sequence and head: tile t has kSeqFixed for its queries and its end, and ceil((before + (t + 1) p) / KB)
// for its keys, at least as many as tiles of keys that its queries see; without `causal` all have ceil(keys / KB) + 1.
struct Line {
  int log_p, log_kb, before;
  int whole;  // units of every tile, 0: causal
  __device__ __forceinline__ Line(int log_p_, int log_kb_, const Seq& s, bool causal) : log_p(log_p_), log_kb(log_kb_) {
    before = max(s.keys - s.n, 0);
    whole = causal ? 0 : (int)(((int64_t)s.keys + (1 << log_kb) - 1) >> log_kb) + 1;
  }
  __device__ __forceinline__ int64_t upto(int64_t t) const {
    return t * kSeqFixed + keys_upto(t);
  }
  __device__ __forceinline__ int64_t keys_upto(int64_t t) const {
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

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uint64_t)v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t lane64(int64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)v >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}
// Sums over the lanes, the same in all of them, and up to each lane; numbers of 64 bits that are small take the short way.
__device__ __forceinline__ int lane_sum(int x) { return __builtin_amdgcn_readlane(lane_prefix_sum(x), 63); }
// The largest of numbers that are not negative.
__device__ __forceinline__ int lane_max(int x) {
  x = max(x, dpp32<0x111, 0xf>(0, x));  // as lane_prefix_sum
  x = max(x, dpp32<0x112, 0xf>(0, x));
  x = max(x, dpp32<0x114, 0xf>(0, x));
  x = max(x, dpp32<0x118, 0xf>(0, x));
  x = max(x, dpp32<0x142, 0xa>(0, x));
  x = max(x, dpp32<0x143, 0xc>(0, x));
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int64_t lane_prefix_sum64(int64_t x, int lane) {
  if (__ballot((uint64_t)x >> 25 != 0) == 0) return lane_prefix_sum((int)x);
#pragma unroll
  for (int step = 1; step < 64; step <<= 1) {
    const int64_t y = __shfl_up(x, step);
    if (lane >= step) x += y;
  }
  return x;
}
__device__ __forceinline__ uint64_t divide(uint64_t x, uint64_t y) {
  return (x | y) >> 32 ? x / y : (uint32_t)x / (uint32_t)y;
}

// Finds tiles: in the line of units, and by their length. The first 64 sequences are held, one a lane.
template <bool PAGED, int LOG_KB>
struct Walk {
  int lane, log_tokens, per_tile, cols, batch;
  bool causal;
  Seq mine;

  __device__ __forceinline__ Walk(SeqArgs a, int lane_)
      : lane(lane_), log_tokens(a->plan.log_tokens), per_tile(a->plan.per_tile), cols(a->heads / per_tile), batch(a->batch),
        causal(a->causal) {
    mine = seq_of<PAGED>(a, min(lane, batch - 1));
    if (lane >= batch) mine.n = 0;
  }
  __device__ __forceinline__ Line line(const Seq& s) const { return Line(log_tokens, LOG_KB, s, causal); }
  __device__ __forceinline__ int tiles(const Seq& s) const { return (int)(((int64_t)s.n + (1 << log_tokens) - 1) >> log_tokens); }
  // sequence base + lane, without queries if there is none
  __device__ __forceinline__ Seq seq_at(int base) const {
    if (base == 0) return mine;
    Seq s = seq_of<PAGED>(again(seq_args()), min(base + lane, batch - 1));
    if (base + lane >= batch) s.n = 0;
    return s;
  }
  __device__ __forceinline__ Seq seq(int b) const {
    Seq s;
    if (b < 64) {
      s.first = __builtin_amdgcn_readlane(mine.first, b);
      s.n = __builtin_amdgcn_readlane(mine.n, b);
      s.keys = __builtin_amdgcn_readlane(mine.keys, b);
    } else {
      s = seq_of<PAGED>(again(seq_args()), b);
      s.first = __builtin_amdgcn_readfirstlane(s.first);
      s.n = __builtin_amdgcn_readfirstlane(s.n);
      s.keys = __builtin_amdgcn_readfirstlane(s.keys);
    }
    return s;
  }

  // Units of sequence base + lane, and of all up to it from `base` on.
  struct Sums {
    int64_t own, upto;
  };
  __device__ __forceinline__ Sums sums(int base) const {
    const Seq s = seq_at(base);
    const int64_t x = s.n ? cols * line(s).upto(tiles(s)) : 0;
    return {x, lane_prefix_sum64(x, lane)};
  }
  __device__ __forceinline__ int64_t total(const Sums& head) const {
    int64_t sum = lane64(head.upto, 63);
    for (int base = 64; base < batch; base += 64) sum += lane64(sums(base).upto, 63);
    return sum;
  }
  // whether tiles are dealt out whole (see kSeqWhole)
  __device__ __forceinline__ bool even(int workers) const {
    int64_t all = 0;
    int longest = 0;
    for (int base = 0; base < batch; base += 64) {
      const Seq s = seq_at(base);
      const Line l = line(s);
      const int t = tiles(s);
      if (t == 0) continue;
      const int64_t units = l.upto(t);
      all += cols * units;
      longest = max(longest, (int)(units - l.upto(t - 1)));
    }
    all = lane64(lane_prefix_sum64(all, lane), 63);
    longest = lane_max(longest);
    if (!PAGED && causal) return (int64_t)(longest - kSeqLongest) * workers * 7 <= all * 10;
    const int64_t round = (int64_t)max(longest, 1) * workers, last = all - (int64_t)divide(all, round) * round;
    return last == 0 || (2 * last > round ? 90 : 65) * round - 100 * last <= (int64_t)1000 * workers + 9 * all;
  }
  // the item that holds unit x, which is below the total; head: sums(0)
  __device__ __forceinline__ Item find(int64_t x, const Sums& head) const {
    Item it;
    it.at = 0;
    Sums sum = head;
    int who = 0;
    for (int base = 0;; base += 64) {
      if (base) sum = sums(base);
      const uint64_t past = __ballot(it.at + sum.upto > x);
      it.b = base;
      if (past || base + 64 >= batch) {
        who = past ? __builtin_ctzll(past) : 0;
        break;
      }
      it.at += lane64(sum.upto, 63);
    }
    it.b = __builtin_amdgcn_readfirstlane(min(it.b + who, batch - 1));
    it.at += lane64(sum.upto - sum.own, who);
    it.s = seq(it.b);
    const Line l = line(it.s);
    it.tiles = tiles(it.s);
    const int64_t column = l.upto(it.tiles);
    int64_t r = uniform64(x - it.at);
    it.col = (int)divide(r, column);
    it.at += it.col * column;
    r -= it.col * column;
    int lo = 0, hi = it.tiles;  // upto(lo) <= r < upto(hi)
    while (hi - lo > 1) {
      const int mid = lo + ((hi - lo) >> 1);
      if (l.upto(mid) <= r) lo = mid; else hi = mid;
    }
    it.tile = lo;
    const int64_t from = l.upto(lo);
    it.at += from;
    it.units = (int)(l.upto(lo + 1) - from);
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
        do it.s = seq(++it.b); while (it.s.n == 0 && it.b + 1 < batch);
        it.tiles = tiles(it.s);
      }
    }
    measure(it);
    return it;
  }
  __device__ __forceinline__ void measure(Item& it) const {
    const Line l = line(it.s);
    it.units = (int)(l.upto(it.tile + 1) - l.upto(it.tile));
    scalar(it);
  }

  // Tiles of the sequences of one column, those of the first 512 held, one a lane, so that they are read once.
  struct Counts {
    static constexpr int kHeld = 8;
    int c[kHeld];
  };
  __device__ __forceinline__ Counts counts() const {
    Counts x;
#pragma unroll
    for (int i = 0; i < Counts::kHeld; ++i) x.c[i] = i == 0 ? tiles(mine) : 64 * i < batch ? tiles(seq_at(64 * i)) : 0;
    return x;
  }
  // f(first sequence, tiles of sequence first + lane) for all, while it says so
  template <typename F>
  __device__ __forceinline__ void each(const Counts& x, F&& f) const {
#pragma unroll
    for (int i = 0; i < Counts::kHeld; ++i)
      if (64 * i >= batch || !f(64 * i, x.c[i])) return;
    for (int base = 64 * Counts::kHeld; base < batch; base += 64)
      if (!f(base, tiles(seq_at(base)))) return;
  }
  // tiles that are number t and above in their sequences
  __device__ __forceinline__ int above(const Counts& x, int t) const {
    int sum = 0;
    each(x, [&](int, int n) {
      sum += max(n - t, 0);
      return true;
    });
    return lane_sum(sum);
  }
  // Tile `rank` of all, by falling number: of packed sequences those that see the most keys first. rank is below above(0) cols.
  __device__ __forceinline__ Item ranked(const Counts& x, int64_t rank) const {
    const int row = (int)divide(rank, cols);
    Item it;
    it.col = (int)(rank - (int64_t)row * cols);
    int most = 0;
    each(x, [&](int, int n) {
      most = max(most, n);
      return true;
    });
    int lo = 0, hi = lane_max(most), passed = 0;  // above(lo) > row >= above(hi) = passed
    while (hi - lo > 1) {
      const int mid = lo + ((hi - lo) >> 1), m = above(x, mid);
      if (m > row) {
        lo = mid;
      } else {
        hi = mid;
        passed = m;
      }
    }
    int k = row - passed, who = 0;
    each(x, [&](int base, int n) {
      uint64_t there = __ballot(n > lo);
      const int m = __popcll(there);
      if (k < m) {
        for (; k > 0; --k) there &= there - 1;
        who = base + __builtin_ctzll(there);
        return false;
      }
      k -= m;
      return true;
    });
    it.b = __builtin_amdgcn_readfirstlane(who);
    it.tile = lo;
    it.s = seq(it.b);
    it.tiles = tiles(it.s);
    it.at = 0;
    measure(it);
    return it;
  }
  static __device__ __forceinline__ void scalar(Item& it) {
    it.at = uniform64(it.at);
    it.col = __builtin_amdgcn_readfirstlane(it.col);
    it.tile = __builtin_amdgcn_readfirstlane(it.tile);
    it.tiles = __builtin_amdgcn_readfirstlane(it.tiles);
    it.units = __builtin_amdgcn_readfirstlane(it.units);
  }
};

// What bfloat16 lost of four values, as the next eight bits of each: differences of the bit patterns in steps of 2^8, so that a value and its
// rest are within 2^-17 of the float32 one.
__device__ __forceinline__ uint32_t rest4(float a, float b, float c, float d, uint2 o) {
  const float x[4] = {a, b, c, d};
  const uint32_t h[4] = {o.x << 16, o.x & 0xffff0000u, o.y << 16, o.y & 0xffff0000u};
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int lost = (int)(__builtin_bit_cast(uint32_t, x[i]) - h[i]);
    out |= (uint32_t)(min((lost + 128) >> 8, 127) & 255) << 8 * i;
  }
  return out;
}
// the i-th of four values from its bfloat16 and its rest
__device__ __forceinline__ float with_rest(uint32_t bf16_bits, uint32_t rest, int i) {
  return __builtin_bit_cast(float, (bf16_bits << 16) + ((uint32_t)(int)(int8_t)(rest >> 8 * i) << 8));
}

// Four columns of a row as 16-bit values are in the lane's half, the next four in the other half's, and so on in turn (a product's output):
// of eight and eight, each half gets its eight.
__device__ __forceinline__ uint4 gather8(uint2 even, uint2 odd) {
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(even.x), "+v"(odd.x));
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(even.y), "+v"(odd.y));
  return make_uint4(even.x, even.y, odd.x, odd.y);
}

// The shares of the line: of `total` units for `workers` workers.
struct Shares {
  int64_t total, near;  // near: how far a border moves to a tile's end; it never stays before a tile's first keys
  int workers;
  __device__ __forceinline__ Shares(int64_t total_, SeqArgs a) : total(total_) {
    workers = (int)max((int64_t)1, min((int64_t)a->plan.workers, (int64_t)divide(total, a->plan.min_units)));
    near = max((int64_t)divide(total, workers) >> 4, (int64_t)kSeqFixed);
  }
  __device__ __forceinline__ int64_t border(int w) const { return divide(total * w, workers); }
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

// One 16-byte-a-lane copy as dma16, for kernels in which nothing else uses M0 (the compiler writes it just before a use). The copy may
// read M0 one state after it is written, and an address five after the vector unit wrote it (a page's, read from a lane): the
// compiler does not look inside for that.
__device__ __forceinline__ void dma16_at(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(voff), "s"(base)
      : "memory");
}
__device__ __forceinline__ void dma16_late(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(voff), "s"(base)
      : "memory");
}

// Rows of keys or of values on their way to a tile in LDS: KB rows of RB bytes, `token` bytes apart in memory. A copy of a wavefront is
// RPI rows; the swizzle of a row's 16-byte chunks repeats after PERIOD copies, and so do the lanes' offsets from a copy's first row.
template <int D, int W>
struct Rows {
  using C = SeqTile<D, W>;
  static constexpr int RPI = 1024 / C::RB, LPR = C::RB / 16, N = C::BYTES / 1024 / W, STEP = W * RPI;
  static constexpr int PERIOD = STEP >= 16 ? 1 : 16 / STEP;
  uint32_t token;         // bytes
  uint32_t off[PERIOD];   // of this lane in copies 0 .. PERIOD - 1, from the tile's row 0 (copy i: of row i STEP)

  __device__ __forceinline__ void init(int64_t stride, int w, int lane) {
    token = (uint32_t)(stride * 2);
#pragma unroll
    for (int i = 0; i < PERIOD; ++i) {
      const int r = (i * W + w) * RPI + lane / LPR;
      off[i] = (w * RPI + lane / LPR) * token + tile_chunk<C::RB>(r, lane % LPR) * 16;
    }
  }
  // packed rows from `from` on, `left` of them: those past the last are the last again (what they add is masked, and they hold no memory
  // that the caller did not write)
  __device__ __forceinline__ void copy(const unsigned char* from, int left, uint32_t lds, int w, int lane) const {
    from = uniform_ptr(from);
    if (left >= C::KB) {
#pragma unroll
      for (int i = 0; i < N; ++i) dma16_at(from + (uint64_t)(i * STEP) * token, off[i % PERIOD], lds + i * W * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = (i * W + w) * RPI + lane / LPR;
        dma16_at(from, min(r, left - 1) * token + tile_chunk<C::RB>(r, lane % LPR) * 16, lds + i * W * 1024);
      }
    }
  }
  // Rows of pages. head: of page 0; ids: the page of each 16 rows, uniform; none: which of them have no page; at: the first row's place in
  // its page. Rows without a page and copies past the last row give zeros.
  __device__ __forceinline__ void copy_pages(const unsigned char* head, int64_t page, const int* ids, uint32_t none, int at, int shift,
                                             int left, uint32_t lds, int w, int lane) const {
    if (left >= C::KB && !none) {
      if (shift >= C::LOG_KB) {
        const unsigned char* from = uniform_ptr(head + ids[0] * page + (uint64_t)at * token);
#pragma unroll
        for (int i = 0; i < N; ++i) dma16_late(from + (uint64_t)(i * STEP) * token, off[i % PERIOD], lds + i * W * 1024);
      } else {
        const unsigned char* from[C::KB / 16];  // less the rows of the tile before them
#pragma unroll
        for (int j = 0; j < C::KB / 16; ++j)
          from[j] = head + ids[j] * page + ((int64_t)((at + 16 * j) & ((1 << shift) - 1)) - 16 * j) * token;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const unsigned char* to = from[i * STEP / 16];
          if (STEP == 32 && w >= 2) to = from[i * 2 + 1];
          dma16_late(uniform_ptr(to + (uint64_t)(i * STEP) * token), off[i % PERIOD], lds + i * W * 1024);
        }
      }
      return;
    }
    const int mask = (1 << shift) - 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (i * W + w) * RPI, r0 = lane / LPR;
      const uint32_t chunk = tile_chunk<C::RB>(row + r0, lane % LPR) * 16;
      const bool zero = none >> (row / 16) & 1 || row >= left;
      const unsigned char* from = zero ? (const unsigned char*)kZeroRow : head + ids[row / 16] * page + (uint64_t)((at + row) & mask) * token;
      dma16_late(uniform_ptr(from), (zero ? 0 : min(r0, left - 1 - row) * token) + chunk, lds + i * W * 1024);
    }
  }
};

template <bool HALF, int D, int W, bool PAGED>
__global__ __launch_bounds__(64 * W, D == 64 && W == 4 && !PAGED ? 3 : 2) void seq_attn_kernel(const WaSeqLaunch) {
  using C = SeqTile<D, W>;
  using T = SeqType<HALF>;
  constexpr int KB = C::KB, R = 32 * W;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * C::STAGE];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Walk<PAGED, C::LOG_KB> walk(seq_args(), lane);
  int64_t total, begin, end;
  Item it;
  int me = blockIdx.x;
  bool whole = (W == 1 && !PAGED) || seq_args()->plan.whole;
  typename Walk<PAGED, C::LOG_KB>::Counts counts;
  if (whole || !PAGED || W == 4) {
    counts = walk.counts();
    total = (int64_t)walk.above(counts, 0) * walk.cols;
    const int workers = seq_args()->plan.workers;
    if (!whole) whole = total >= (int64_t)(!PAGED && walk.causal ? kSeqWhole : 2 * kSeqWhole) * workers || walk.even(workers);
  }
  if (me == 0 && tid == 0) *seq_args()->any_cut = !whole;
  if (whole) {
    if (me >= total) return;
    it = walk.ranked(counts, me);
    begin = 0;
    end = it.units;
  } else {
    const SeqArgs a = seq_args();
    const auto sums = walk.sums(0);
    total = walk.total(sums);
    if (total == 0) return;
    const Shares shares(total, a);
    // workgroups go round the eight XCDs: each XCD takes neighbouring shares where there are shares for all
    if (shares.workers == a->plan.workers) me = (blockIdx.x & 7) * (a->plan.workers >> 3) + (blockIdx.x >> 3);
    if (blockIdx.x >= a->plan.workers || me >= shares.workers) return;
    begin = shares.border(me), end = shares.border(me + 1);
    if (end < total) end = shares.moved(end, walk.find(end, sums));
    it = walk.find(begin, sums);
    begin = shares.moved(begin, it);
    if (begin == it.at + it.units && begin < total) it = walk.next(it);
    if (begin >= end) return;
    begin = uniform64(begin);
    end = uniform64(end);
  }
  // A share that begins inside a tile ends with that one. So all workers begin with the first keys, and where tiles are of about a
  // share's length they meet the same keys at the same time (two chunks of 1,024 tokens over 16,384 keys among six tokens:
  // 672 -> 644 us).
  Item rest = it;
  int left = 0;  // of the share: 1: `rest` comes after the others; 2: it is the last
  if (PAGED && begin > it.at && it.at + it.units < end) {
    it = walk.next(it);
    left = 1;
  }
  const uint32_t kbase = row_operand<C::RB>(lane, 0);
  const uint32_t vbase0 = C::BYTES + col_operand<C::RB>(lane, 0, 0), vbase1 = C::BYTES + col_operand<C::RB>(lane, 0, 1);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)lds) + w * 1024;
  Rows<D, W> krows, vrows;
  krows.init(PAGED ? seq_args()->kp.token : seq_args()->k.token, w, lane);
  vrows.init(PAGED ? seq_args()->vp.token : seq_args()->v.token, w, lane);

  // the keys of this worker's part of a tile
  struct Range {
    int lo, hi;
  };
  auto range = [&](const Item& x) {
    Range r;
    const int last = min(((x.tile + 1) << walk.log_tokens), x.s.n) - 1;
    const int most = walk.causal ? min(max(x.s.keys - x.s.n + last + 1, 0), x.s.keys) : x.s.keys;
    const int64_t u0 = max(begin - x.at - kSeqFixed, (int64_t)0), u1 = min(end - x.at, (int64_t)x.units) - kSeqFixed;
    r.lo = (int)min(u0 * KB, (int64_t)most);
    r.hi = (int)min(max(u1, (int64_t)0) * KB, (int64_t)most);
    return r;
  };

  // Where the next copy comes from. Paged: 64 entries of the sequence's table, one a lane, and which of them name no page.
  const unsigned char *kfrom = nullptr, *vfrom = nullptr;
  int from_b = -1, from_keys = 0, window = -1, entry = 0, entry_ahead = 0, ahead_b = -1, ahead_window = 0;
  uint64_t bad = 0;
  // the entry of a sequence's table that this lane holds of the window of 64 around `key`
  auto load_entry = [&](int b, int keys, int key) {
    const SeqArgs a = again(seq_args());
    const int e = (key >> a->page_shift & ~63) + lane, used = (int)(((int64_t)keys + (1 << a->page_shift) - 1) >> a->page_shift);
    return e < used ? a->tables[b * a->table_stride + e] : 0;
  };
  auto aim = [&](const Item& x, int key) {
    const SeqArgs a = again(seq_args());
    const int hk = walk.per_tile == 1 ? x.col / (a->heads / a->kv_heads) : x.col;
    if (PAGED) {
      kfrom = (const unsigned char*)a->kp.at + hk * a->kp.head * 2;
      vfrom = (const unsigned char*)a->vp.at + hk * a->vp.head * 2;
    } else {
      kfrom = (const unsigned char*)a->k.at + ((x.s.first + key) * a->k.token + hk * a->k.head) * 2;
      vfrom = (const unsigned char*)a->v.at + ((x.s.first + key) * a->v.token + hk * a->v.head) * 2;
    }
    if (PAGED && x.b != from_b) window = -1;
    from_b = x.b;
    from_keys = x.s.keys;
  };
  // What the copies of a tile need of the arguments, read at once.
  struct Pool {
    int shift, pages;
    int64_t k, v;  // bytes of a page
  };
  auto pool = [&] {
    Pool p{};
    if constexpr (PAGED) {
      const SeqArgs a = again(seq_args());
      p = {a->page_shift, a->n_pages, a->kp.page * 2, a->vp.page * 2};
    }
    return p;
  };
  // Paged: the pages of the tile at `key`; returns which 16 keys of it lie in none.
  typedef int Ids[KB / 16];
  auto pages_at = [&](const Pool& pl, int key, Ids& ids) -> uint32_t {
    uint32_t none = 0;
    if constexpr (PAGED) {
      const int shift = pl.shift, first = key >> shift;
      if (first >> 6 != window) {
        window = first >> 6;
        entry = from_b == ahead_b && window == ahead_window ? entry_ahead : load_entry(from_b, from_keys, key);
        bad = __ballot((uint32_t)entry >= (uint32_t)pl.pages);
      }
#pragma unroll
      for (int j = 0; j < KB / 16; ++j) {
        const int e = (key + 16 * j) >> shift & 63;
        ids[j] = __builtin_amdgcn_readlane(entry, e);
        if (bad >> e & 1) none |= 1u << j;
      }
    }
    return none;
  };
  // copies the tile of keys, and that of values, at `key`
  auto copy_keys = [&](const Pool& pl, int key, int buf, const Ids& ids, uint32_t none) {
    const uint32_t to = lds0 + buf * C::STAGE;
    const int left = from_keys - key;
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));  // the last tiles' offsets are not held across the loop
    if constexpr (PAGED) {
      krows.copy_pages(kfrom, pl.k, ids, none, key & ((1 << pl.shift) - 1), pl.shift, left, to, w, lane_o);
    } else {
      krows.copy(kfrom, left, to, w, lane_o);
      kfrom += (uint64_t)KB * krows.token;
    }
  };
  auto copy_values = [&](const Pool& pl, int key, int buf, const Ids& ids, uint32_t none) {
    const uint32_t to = lds0 + buf * C::STAGE + C::BYTES;
    const int left = from_keys - key;
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));
    if constexpr (PAGED) {
      vrows.copy_pages(vfrom, pl.v, ids, none, key & ((1 << pl.shift) - 1), pl.shift, left, to, w, lane_o);
    } else {
      vrows.copy(vfrom, left, to, w, lane_o);
      vfrom += (uint64_t)KB * vrows.token;
    }
  };
  auto copy = [&](int key, int buf) -> uint32_t {
    const Pool pl = pool();
    Ids ids;
    const uint32_t none = pages_at(pl, key, ids);
    copy_keys(pl, key, buf, ids, none);
    copy_values(pl, key, buf, ids, none);
    return none;
  };

  // this lane's row of a tile: token i of head `sub`
  const int row = w * 32 + l32;
  struct Place {
    int token, head;
    bool valid;
  };
  auto place = [&](const Item& x) {
    const int log_p = walk.log_tokens, sub = row >> log_p;
    Place p;
    p.token = (x.tile << log_p) + (row & ((1 << log_p) - 1));
    p.head = x.col * walk.per_tile + sub;
    p.valid = sub < walk.per_tile && p.token < x.s.n;
    return p;
  };

  bf16x8 qf[C::KS], qn[C::KS];
  auto load_queries = [&](const Item& x, bf16x8 (&q)[C::KS]) {
    const Place p = place(x);
    const SeqArgs a = again(seq_args());
    const uint16_t* qg = (const uint16_t*)a->q.at + (x.s.first + p.token) * a->q.token + p.head * a->q.head;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) q[s] = load8(qg + 16 * s + 8 * hf, p.valid);
  };
  f32x16 acc[C::DT];
  float m_run, l_run;
  const float c2 = seq_args()->scale * kLog2e;
  // One wavefront: a tile of keys. limit: of the lane's query; none: 16 keys without a page.
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
    __builtin_amdgcn_s_setprio(1);
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
    __builtin_amdgcn_s_setprio(0);
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
    __builtin_amdgcn_s_setprio(1);
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
    __builtin_amdgcn_s_setprio(0);
  };

  // Four wavefronts: the scores of a tile of keys, at place t,
  constexpr int ROWS = C::KS * C::KT, COLS = 2 * C::KT * C::DT;
  auto scores = [&](f32x16 (&s)[C::KT], uint32_t t) {
    uint32_t kb = kbase + t;
    asm volatile("" : "+v"(kb));
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kt][v] = 0.f;
    bf16x8 ring[kSeqAhead];
#pragma unroll
    for (int x = 0; x < kSeqAhead; ++x) ring[x] = read_row(lds + row_step(kb, x / C::KT) + x % C::KT * 32 * C::RB);
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      WA_SCHED_FENCE();
      s[x % C::KT] = T::mfma(ring[x % kSeqAhead], qf[x / C::KT], s[x % C::KT]);
      const int y = x + kSeqAhead;
      if (y < ROWS) ring[x % kSeqAhead] = read_row(lds + row_step(kb, y / C::KT) + y % C::KT * 32 * C::RB);
    }
    WA_SCHED_FENCE();
  };
  // and what follows from them, `s`, for the tile at `key`, with the scores of the next tile, `sn`, if NEXT: the maxima and the first
  // probabilities beside the products of those scores, the others beside those of O. For 128 columns the scores' part goes first on a
  // SIMD (8,192 tokens, 14 heads over 2: 280 -> 258 us); for 64 columns, of which three wavefronts share a SIMD, it does not pay.
  auto step = [&](auto with_next, f32x16 (&s)[C::KT], f32x16 (&sn)[C::KT], int key, uint32_t t, int limit, bool masked, uint32_t none) {
    constexpr bool NEXT = decltype(with_next)::value;
    constexpr int PAIRS = 8 * C::KT, BEFORE = D == 128 ? 10 : 4;  // pairs of probabilities; those beside the scores (6 to 12: no change)
    uint32_t kb = kbase + (t ^ C::STAGE), vb0 = vbase0 + t, vb1 = vbase1 + t;
    asm volatile("" : "+v"(kb), "+v"(vb0), "+v"(vb1));
    auto key_row = [&](int x) { return read_row(lds + row_step(kb, x / C::KT) + x % C::KT * 32 * C::RB); };
    auto col = [&](int x) {
      const int at = x / C::DT * 16 * C::RB;
      return read_cols(lds + col_step(vb0, x % C::DT) + at, lds + col_step(vb1, x % C::DT) + at);
    };
    if (masked) {
      const int rest = limit - key - 4 * hf;
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (kt * 32 + 8 * (v >> 2) + (v & 3) >= rest || (PAGED && (none >> (2 * kt + (v >> 3)) & 1))) s[kt][v] = -INFINITY;
    }
    bf16x8 ring[kSeqAhead], cring[kSeqAhead];
    if constexpr (NEXT) {
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v) sn[kt][v] = 0.f;
#pragma unroll
      for (int x = 0; x < kSeqAhead; ++x) ring[x] = key_row(x);
    }
    float top = -INFINITY, ref = 0.f;
    auto rise = [&] {
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
      ref = m_run == -INFINITY ? 0.f : m_run - T::kBias;
    };
    uint32_t pk[2 * C::KT][4];
    auto pairs = [&](int from, int to) {  // of probabilities, four of 16 keys
#pragma unroll
      for (int i = 0; i < PAIRS; ++i)
        if (i >= from && i < to) {
          const int v = 2 * (i & 7);
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 3][v], c2, -ref));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 3][v + 1], c2, -ref));
          l_run += p0 + p1;
          pk[i >> 2][i & 3] = T::pack(p0, p1);
          asm volatile("" : "+v"(l_run));  // added here
        }
    };
    if (D == 128) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
      WA_SCHED_FENCE();
      if constexpr (NEXT) {
        sn[x % C::KT] = T::mfma(ring[x % kSeqAhead], qf[x / C::KT], sn[x % C::KT]);
        if (x + kSeqAhead < ROWS) ring[x % kSeqAhead] = key_row(x + kSeqAhead);
      }
      if (x >= ROWS - kSeqAhead) cring[x - (ROWS - kSeqAhead)] = col(x - (ROWS - kSeqAhead));
      if (x < 4) {
#pragma unroll
        for (int e = 0; e < 4 * C::KT; ++e) top = fmaxf(top, s[x / (4 / C::KT)][x % (4 / C::KT) * 4 * C::KT + e]);
        if (x == 3) rise();
      } else {
        pairs((BEFORE * (x - 4) + ROWS - 5) / (ROWS - 4), (BEFORE * (x - 3) + ROWS - 5) / (ROWS - 4));
      }
    }
    if (D == 128) __builtin_amdgcn_s_setprio(0);
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      WA_SCHED_FENCE();
      const int k16 = x / C::DT, dt = x % C::DT;
      acc[dt] = T::mfma(cring[x % kSeqAhead], as_bf16x8(make_uint4(pk[k16][0], pk[k16][1], pk[k16][2], pk[k16][3])), acc[dt]);
      if (x + kSeqAhead < COLS) cring[x % kSeqAhead] = col(x + kSeqAhead);
      constexpr int N = COLS - C::DT;
      pairs(BEFORE + ((PAIRS - BEFORE) * x + N - 1) / N, BEFORE + ((PAIRS - BEFORE) * (x + 1) + N - 1) / N);
    }
    WA_SCHED_FENCE();
  };

  int buf = 0;
  uint32_t none = 0, any_bad = 0, item_bad = 0;  // bad: of the keys that were passed, those without a page
  bool ready = false, stored = false;  // the item's first tile is on its way; stores of the item before come behind it
  Range r = range(it);
  for (;;) {
    const bool line = left < 2 && it.at + it.units < end, more = line || left == 1;
    Item nx;
    Range rn;
    bool known = false;  // nx
    auto look = [&] {
      if (line) {
        nx = walk.next(it);
      } else {
        nx = rest;
        left = 2;
      }
      rn = range(nx);
      known = true;
      if (PAGED && nx.b != it.b) {  // its pages are asked for ahead of its first copy
        ahead_b = nx.b;
        ahead_window = rn.lo >> again(seq_args())->page_shift >> 6;
        entry_ahead = load_entry(nx.b, nx.s.keys, rn.lo);
      }
    };
    Ids ids;  // of the next tile
    uint32_t none_next = 0;
    if constexpr (W == 4) {
      if (r.lo < r.hi) {
        WA_BARRIER();  // of the item before
        aim(it, r.lo);
        none = copy(r.lo, 0);
        if (r.lo + KB < r.hi) {
          const Pool pl = pool();
          none_next = pages_at(pl, r.lo + KB, ids);
          copy_keys(pl, r.lo + KB, 1, ids, none_next);
        }
      }
      load_queries(it, qf);
    } else if (ready) {
#pragma unroll
      for (int s = 0; s < C::KS; ++s) qf[s] = qn[s];
    } else {
      if (r.lo < r.hi) {
        aim(it, r.lo);
        none = copy(r.lo, buf);
      }
      load_queries(it, qf);
      stored = false;
    }
    int limit, some, all;  // keys that the lane's query sees; that any, and that all of the wavefront's queries see
    {
      const int log_p = walk.log_tokens, at = it.tile << log_p, before = it.s.keys - it.s.n;
      const int first = log_p >= 5 ? (w * 32) & ((1 << log_p) - 1) : 0;  // the wavefront's tokens
      const int t0 = at + first, t1 = min(at + first + (log_p >= 5 ? 31 : (1 << log_p) - 1), it.s.n - 1);
      const bool used = (w * 32 >> log_p) < walk.per_tile && t0 < it.s.n;
      const Place p = place(it);
      auto sees = [&](int t) { return walk.causal ? min(max(before + t + 1, 0), it.s.keys) : it.s.keys; };
      limit = p.valid ? sees(p.token) : 0;
      some = used ? sees(t1) : 0;
      all = sees(t0);
    }
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[t][v] = 0.f;
    m_run = -INFINITY;
    l_run = 0.f;
    ready = false;
    if constexpr (W == 4) {
      if (r.lo < r.hi) {
        f32x16 sa[C::KT];
        WA_WAIT_VM(0);
        WA_BARRIER();
        const int mine = min(some, r.hi);
        if (r.lo < mine) scores(sa, 0);
        int key = r.lo, at = 0;
        uint32_t now = 0;
        auto turn = [&] {
          const Pool pl = pool();
          WA_WAIT_VM(0);
          WA_BARRIER();  // everyone has the tile's values and the next one's keys, and is done with its keys and the values before
          now = none;
          if (PAGED) item_bad |= now;
          none = none_next;
          if (key + KB < r.hi) copy_values(pl, key + KB, at ^ 1, ids, none_next);
          if (key + 2 * KB < r.hi) {
            none_next = pages_at(pl, key + 2 * KB, ids);
            copy_keys(pl, key + 2 * KB, at, ids, none_next);
          }
        };
        for (; key + KB < mine; key += KB, at ^= 1) {
          turn();
          f32x16 sn[C::KT];
          step(std::true_type(), sa, sn, key, at * C::STAGE, limit, key + KB > all || (PAGED && now), now);
#pragma unroll
          for (int kt = 0; kt < C::KT; ++kt) sa[kt] = sn[kt];
        }
        if (key < mine) {
          turn();
          step(std::false_type(), sa, sa, key, at * C::STAGE, limit, key + KB > all || (PAGED && now), now);
          key += KB;
          at ^= 1;
        }
        for (; key < r.hi; key += KB, at ^= 1) turn();
      }
    } else for (int key = r.lo; key < r.hi; key += KB) {
      // This wavefront's part of the tile has arrived (and the queries, so that nothing waits for them below); stores behind it, at
      // least one for each eight columns that a lane holds, need not have.
      if (stored) WA_WAIT_VM(2 * C::DT); else WA_WAIT_VM(0);
      stored = false;
      WA_BARRIER();  // everyone's has, and everyone is done with the other buffer
      int next = key + KB;
      bool go = next < r.hi;
      if (!go && more) {
        if (!known) look();
        go = ready = rn.lo < rn.hi;
        next = rn.lo;
        if (go) {
          aim(nx, next);
          load_queries(nx, qn);
        }
      }
      none_next = go ? copy(next, buf ^ 1) : 0;
      if (more && !known) look();  // early, so that the last tile's copies do not wait for it
      item_bad |= none;
      if (key < some) work(key, buf * C::STAGE, limit, key + KB > all || (PAGED && none), none);
      none = none_next;
      buf ^= 1;
    }
    if (more && !known) look();

    // the item's end: whole rows to O, others to the worker's partial tiles
    const float l = add_halves(l_run);
    const float ref = m_run != -INFINITY ? m_run - T::kBias : l == 0.f ? -INFINITY : 0.f;  // the last: NaN, which a join has to find
    const bool starts = begin <= it.at, finishes = it.at + it.units <= end;
    const Place p = place(it);
    stored = __ballot(p.valid) != 0;
    // Where all scores are -inf (infinite queries, products past float32) a softmax is 0 / 0; where the row sees no key, O is 0. (Of packed
    // sequences each sees one.)
    const bool undefined = r.lo < r.hi && item_bad == 0 && (!PAGED || !walk.causal || it.s.keys - it.s.n + p.token >= r.lo);
    any_bad |= item_bad;
    item_bad = 0;
    const SeqArgs a = again(seq_args());
    const int64_t tok = it.s.first + p.token;
    if (starts && finishes) {
      const float inv = l > 0.f ? 1.f / l : l == 0.f && !undefined ? 0.f : NAN;
      uint16_t* out = (uint16_t*)a->o.at + tok * a->o.token + p.head * a->o.head + 8 * hf;
      float* stat = a->lse && p.valid ? a->lse + (p.head * (int64_t)a->tokens + tok) * a->lse_step : nullptr;
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; v += 8) {
          uint2 o16[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[dt][v + 4 * q + e] *= inv;
            o16[q] = make_uint2(T::pack(acc[dt][v + 4 * q], acc[dt][v + 4 * q + 1]), T::pack(acc[dt][v + 4 * q + 2], acc[dt][v + 4 * q + 3]));
            if (!HALF && !PAGED && stat)
              *(uint32_t*)(stat + 1 + dt * 8 + v / 2 + 2 * q + hf) =
                  rest4(acc[dt][v + 4 * q], acc[dt][v + 4 * q + 1], acc[dt][v + 4 * q + 2], acc[dt][v + 4 * q + 3], o16[q]);
          }
          const uint4 eight = gather8(o16[0], o16[1]);
          if (p.valid) *(uint4*)(out + dt * 32 + 2 * v) = eight;
        }
      if (stat && hf == 0) *stat = l == 0.f ? -INFINITY : (ref + __log2f(l)) * kLn2;
      if (!whole && p.valid && hf == 0) a->cuts[tok * a->heads + p.head] = make_int2(-1, 0);
    } else if (p.valid) {
      // slot 0: a part that begins inside its tile; slot 1: one that begins with it
      const int64_t at = ((int64_t)me * 2 + (starts ? 1 : 0)) * R + row;
      float* out = a->part + at * D;
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *(float4*)(out + dt * 32 + 2 * v + 4 * hf) = make_float4(acc[dt][v], acc[dt][v + 1], acc[dt][v + 2], acc[dt][v + 3]);
      if (hf == 0) ((float2*)(a->part + (int64_t)a->plan.workers * 2 * R * D))[at] = make_float2(ref, l == 0.f && undefined ? -1.f : l);
      if (finishes) {
        const int first = Shares(total, a).first_of(it);
        if (hf == 0) a->cuts[tok * a->heads + p.head] = make_int2(first | me << 16, row);
      }
    }
    if (!more) break;
    it = nx;
    r = rn;
  }
  if (PAGED && any_bad && seq_args()->status && tid == 0) atomicOr(seq_args()->status, WA_PAGE_BAD_INDEX);
}

// Where a row's parts lie, and its end.
template <bool HALF, int D, int W, bool PAGED>
struct JoinRow {
  static constexpr int R = 32 * W;
  int64_t token;
  int head, begin, end, row;
  const float2* stat;
  // cut: as seq_attn_kernel left it, taken into the workers that there are, so that nothing that the workspace holds leads out of it
  __device__ __forceinline__ JoinRow(const WaSeqLaunch& a, int64_t r, int2 cut) {
    token = r / a.heads;
    head = (int)(r - token * a.heads);
    begin = min(cut.x & 0xffff, a.plan.workers - 1);
    end = min((int)((uint32_t)cut.x >> 16), a.plan.workers - 1);
    row = cut.y & (R - 1);
    stat = (const float2*)(a.part + (int64_t)a.plan.workers * 2 * R * D);
  }
  // a part that begins with its tile lies in slot 1, others in slot 0
  __device__ __forceinline__ int64_t at(int c) const { return ((int64_t)c * 2 + (c == begin ? 1 : 0)) * R + row; }
  // columns [c, c + 4) of the row; o, l: summed over the parts, taken against `top`; undefined: a part has keys, whose scores are all -inf
  // (its l is -1)
  __device__ __forceinline__ void finish(const WaSeqLaunch& a, float4 o, float l, float top, bool undefined, int c) const {
    const float inv = l > 0.f ? 1.f / l : l == 0.f && !undefined ? 0.f : NAN;
    o.x *= inv;
    o.y *= inv;
    o.z *= inv;
    o.w *= inv;
    const uint2 o16 = make_uint2(SeqType<HALF>::pack(o.x, o.y), SeqType<HALF>::pack(o.z, o.w));
    *(uint2*)((uint16_t*)a.o.at + token * a.o.token + head * a.o.head + c) = o16;
    if (!a.lse) return;
    float* to = a.lse + (head * (int64_t)a.tokens + token) * a.lse_step;
    if (c == 0) *to = l == 0.f ? -INFINITY : (top + __log2f(l)) * kLn2;
    if (!HALF && !PAGED) *(uint32_t*)(to + 1 + c / 4) = rest4(o.x, o.y, o.z, o.w, o16);
  }
};
// Rows of sequences: what lies before the first and behind the last stays as it is, and has no cuts.
__device__ __forceinline__ bool seq_row(const WaSeqLaunch& a, int64_t r) {
  return r >= (int64_t)min(max(a.starts[0], 0), a.tokens) * a.heads && r < (int64_t)min(max(a.starts[a.batch], 0), a.tokens) * a.heads;
}

// Joins rows of few parts: four columns a lane, D / 4 lanes a row, which look at as many rows at once (those `groups` apart) and join the
// ones that are cut.
template <bool HALF, int D, int W, bool PAGED>
__global__ __launch_bounds__(256) void seq_join_few_kernel(const WaSeqLaunch a, int64_t groups) {
  constexpr int L = D / 4;
  if (!*a.any_cut) return;
  const int lane = threadIdx.x & (L - 1), c = 4 * lane;
  const int64_t group = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L, all = (int64_t)a.tokens * a.heads;
  for (int64_t base = group; base < all; base += groups * L) {
    const int64_t mine = base + lane * groups;
    int2 cut = make_int2(-1, 0);
    if (mine < all && seq_row(a, mine)) cut = a.cuts[mine];
    uint64_t some = __ballot(cut.x != -1) >> (threadIdx.x & 63 & ~(L - 1));
    if (L < 64) some &= ((uint64_t)1 << (L & 63)) - 1;
    while (some) {
      const int who = __builtin_ctzll(some);
      some &= some - 1;
      const JoinRow<HALF, D, W, PAGED> row(a, base + who * groups, make_int2(__shfl(cut.x, who, L), __shfl(cut.y, who, L)));
      float top = -INFINITY, l = 0.f;
      bool undefined = false;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = row.begin; w <= row.end; w += 4) {
        float2 s[4];
        float4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // past the last part the last again, without weight
          const int64_t at = row.at(min(w + i, row.end));
          s[i] = row.stat[at];
          x[i] = *(const float4*)(a.part + at * D + c);
        }
        float high = top;
#pragma unroll
        for (int i = 0; i < 4; ++i) high = fmaxf(high, s[i].x);
        const float keep = high == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - high);
        l *= keep;
        o.x *= keep;
        o.y *= keep;
        o.z *= keep;
        o.w *= keep;
        top = high;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = s[i].x == -INFINITY || w + i > row.end ? 0.f : __builtin_amdgcn_exp2f(s[i].x - high);
          undefined |= s[i].y < 0.f;
          l += f * s[i].y;
          o.x += f * x[i].x;
          o.y += f * x[i].y;
          o.z += f * x[i].z;
          o.w += f * x[i].w;
        }
      }
      row.finish(a, o, l, top, undefined, c);
    }
  }
}

// Joins rows of many parts: a workgroup a row, D / 4 lanes a part, 16 parts at a time.
template <bool HALF, int D, int W, bool PAGED>
__global__ __launch_bounds__(4 * D) void seq_join_many_kernel(const WaSeqLaunch a) {
  constexpr int L = D / 4, TEAMS = 16, AHEAD = 8;
  __shared__ float4 sums[TEAMS][L];
  __shared__ float2 stats[TEAMS];
  const int any = *a.any_cut;
  const int2 cut = a.cuts[blockIdx.x];
  if (!any || !seq_row(a, blockIdx.x) || cut.x == -1) return;
  const JoinRow<HALF, D, W, PAGED> row(a, blockIdx.x, cut);
  const int team = threadIdx.x / L, lane = threadIdx.x & (L - 1), c = 4 * lane;
  float top = -INFINITY, l = 0.f;
  bool undefined = false;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float high, const float2& s, const float4& x) {  // both taken against `high`
    const float f = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - high);
    undefined |= s.y < 0.f;
    l += f * s.y;
    o.x += f * x.x;
    o.y += f * x.y;
    o.z += f * x.z;
    o.w += f * x.w;
  };
  auto raise = [&](float high) {
    const float keep = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - high);
    l *= keep;
    o.x *= keep;
    o.y *= keep;
    o.z *= keep;
    o.w *= keep;
    top = high;
  };
  for (int w = row.begin + team; w <= row.end; w += AHEAD * TEAMS) {
    float2 s[AHEAD];
    float4 x[AHEAD];
    float high = top;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {  // past the last part the last again, without weight
      const int64_t at = row.at(min(w + i * TEAMS, row.end));
      s[i] = row.stat[at];
      x[i] = *(const float4*)(a.part + at * D + c);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (w + i * TEAMS > row.end) s[i] = make_float2(-INFINITY, 0.f);
      high = fmaxf(high, s[i].x);
    }
    raise(high);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) add(high, s[i], x[i]);
  }
  sums[team][lane] = o;
  if (lane == 0) stats[team] = make_float2(top, l == 0.f && undefined ? -1.f : l);
  __syncthreads();
  if (team) return;
  float high = top;
#pragma unroll
  for (int x = 1; x < TEAMS; ++x) high = fmaxf(high, stats[x].x);
  raise(high);
#pragma unroll
  for (int x = 1; x < TEAMS; ++x) add(high, stats[x], sums[x][lane]);  // in one order
  row.finish(a, o, l, top, undefined, c);
}

// Parts from which on a workgroup joins a row alone (one token of 64 sequences, 5 parts: 61 us where a workgroup of 1,024 threads does
// each, 5 us side by side; one of a long sequence, 256 parts: 6 us and 9).
constexpr int64_t kSeqManyParts = 12;

template <bool HALF, int D, int W, bool PAGED>
hipError_t seq_launch(const WaSeqLaunch& a, hipStream_t stream) {
  const int64_t most = wa_seq_most_tiles(a, a.plan);
  const int64_t grid = a.plan.whole ? most : PAGED && W == 1 ? a.plan.workers : std::max<int64_t>(most, a.plan.workers);
  hipLaunchKernelGGL((seq_attn_kernel<HALF, D, W, PAGED>), dim3((unsigned)grid), dim3(64 * W), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if constexpr (W == 4 || PAGED) {  // packed sequences of so few tokens are never cut (wa_seq_plan)
    if (e != hipSuccess || a.plan.whole) return e;
    const int64_t rows = (int64_t)a.tokens * a.heads;
    // a tile's parts, if all workers share the tiles that there are at least
    const int64_t tiles = std::max<int64_t>(std::min(a.batch, a.tokens), a.tokens >> a.plan.log_tokens) * (a.heads / a.plan.per_tile);
    if (a.plan.workers / tiles >= kSeqManyParts && rows <= (1 << 16)) {
      hipLaunchKernelGGL((seq_join_many_kernel<HALF, D, W, PAGED>), dim3((unsigned)rows), dim3(4 * D), 0, stream, a);
    } else {
      constexpr int PER = 256 / (D / 4);
      const int64_t wgs = std::min<int64_t>((rows + PER - 1) / PER, 2048);
      hipLaunchKernelGGL((seq_join_few_kernel<HALF, D, W, PAGED>), dim3((unsigned)wgs), dim3(256), 0, stream, a, wgs * PER);
    }
    return hipGetLastError();
  }
  return e;
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
