// Tiles, masks and row limits shared by the differential-attention kernels.
//
// Every operand tile lies in LDS as it lies in memory, one token a row, and serves two kinds of matrix operand:
// rows (16 consecutive bytes of one token, ds_read_b128) for products over the head's columns, and columns (4
// tokens of one column, ds_read_b64_tr_b16) for products over the tokens. So no tensor is transposed beforehand and no tile
// is held twice.
#pragma once

#include "diff_launch.h"
#include "tile_ops.h"

namespace wa {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Physical 16-byte chunk of (row, chunk) in a tile with rows of RB bytes. 64 banks of 4 bytes are 256 bytes: of
// 256-byte (or longer) rows, 16 rows read at one chunk fall on 16 different places, and 4 consecutive rows, of which a transposed read
// takes 64 bytes each, on 4 different quarters; of 128-byte rows, two make such a line and the same holds
// for pairs.
template <int RB>
__device__ __forceinline__ int tile_chunk(int row, int chunk) {
  return RB >= 256 ? chunk ^ ((row & 3) << 2 | (row >> 2 & 3)) : chunk ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3));
}

// Byte offset of the row operand: 8 columns from 16 s + 8 (lane / 32) of row lane % 32 (a multiple of 32 rows further
// is that many RB further).
template <int RB>
__device__ __forceinline__ uint32_t row_operand(int lane, int s) {
  const int row = lane & 31;
  return row * RB + tile_chunk<RB>(row, 2 * s + (lane >> 5)) * 16;
}

// Byte offset of half j of the column operand of column tile c (32 columns): the lane receives rows
// 4 (lane / 32) + 8 j + 0..3 of column 32 c + lane % 32 (a multiple of 16 rows further is that many RB further).
// Sixteen lanes read 4 rows of 16 columns, lane i row i / 4 and columns 4 (i % 4) on, and exchange them.
template <int RB>
__device__ __forceinline__ uint32_t col_operand(int lane, int c, int j) {
  const int g = lane >> 4, i = lane & 15;
  const int row = 8 * j + 4 * (g >> 1) + (i >> 2);
  return row * RB + tile_chunk<RB>(row, 4 * c + 2 * (g & 1) + (i >> 1 & 1)) * 16 + (i & 1) * 8;
}

// The same offsets of k-step s (below 8) and of column tile c (below 4) from those of the first: the swizzle is an exclusive or of
// the chunk's bits, so the step is too.
__device__ __forceinline__ uint32_t row_step(uint32_t first, int s) { return first ^ 32 * s; }
__device__ __forceinline__ uint32_t col_step(uint32_t first, int c) { return first ^ 64 * c; }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// The column operand from its two halves: rows (lane / 32) 4 + {0..3, 8..11} of 16, the order in which a product's
// output registers hold them, so a product over those rows takes them as they are.
__device__ __forceinline__ bf16x8 read_cols(const unsigned char* h0, const unsigned char* h1) {
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)h0);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)h1);
  const s16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ bf16x8 read_row(const unsigned char* p) { return as_bf16x8(*(const uint4*)p); }

// Copies rows [row0, row0 + ROWS) of g (rows of RB bytes) into a tile, by NWV wavefronts; rows past `last` are row
// `last` again (what they add is masked, and they hold no memory that the caller did not write).
template <int RB, int ROWS, int NWV>
__device__ __forceinline__ void copy_tile(const unsigned char* tile, const unsigned char* g, int row0, int last, int w,
                                          int lane) {
  constexpr int RPI = 1024 / RB, LPR = RB / 16, N = ROWS * RB / 1024 / NWV;
  static_assert(N >= 1 && N * NWV * 1024 == ROWS * RB, "a tile is whole copies of every wavefront");
  constexpr bool kSame = NWV * RPI % 16 == 0;  // the swizzle repeats from copy to copy
  const int r0 = w * RPI + lane / LPR;
  if (row0 + ROWS <= last + 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + i * NWV * RPI;
      dma16(g + (int64_t)(row0 + i * NWV * RPI) * RB,
            (uint32_t)(r0 * RB + tile_chunk<RB>(kSame ? r0 : r, lane % LPR) * 16), tile + (i * NWV + w) * 1024);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + i * NWV * RPI;
      dma16(g, (uint32_t)(min(row0 + r, last) * RB + tile_chunk<RB>(r, lane % LPR) * 16), tile + (i * NWV + w) * 1024);
    }
  }
}

// What a workgroup computes: chunk `chunk` of the `chunks` of a tile of a unit (a head or key head of a sequence).
struct Task {
  int unit, tile, chunk, chunks;
  int64_t item, part;  // the tile's number, and the chunk's among the partial results
};
// The workgroup's task; false if there is none. PER_CU: workgroups that a compute unit holds. Without a list of tasks, the chunks of a
// tile together, and the tiles of `group` units in turn, tile after tile (backwards: from the last), then those of the next units:
// workgroups go round the eight XCDs, so with eight units each XCD's cache holds the other side of one; causal ones take all units, so
// that long tiles come first (2 x 16 heads of 2,048 tokens, d 64, values 64: forward 55 us, dQ 78, dK and dV 88; by eights 58, 80 and
// 96), with neighbouring units, which may share keys, on one XCD where eight divides their number (forward and gradient of 32 heads over
// 8 of 16,384 tokens, d and values 128: 17.46 -> 16.88 ms); masked ones go unit after unit.
template <int PER_CU>
__device__ __forceinline__ bool take_task(const WaDiffLaunch& a, int tiles, int units, int chunks, bool backwards, Task* t) {
  if (a.tasks) {
    if ((int)blockIdx.x >= a.tasks[0]) return false;
    const int4 e = ((const int4*)(a.tasks + wa_diff_task_list(a.task_items)))[blockIdx.x];
    *t = {e.x / tiles, e.x % tiles, e.y, e.z, e.x, e.w + e.y};
    return true;
  }
  int id = blockIdx.x;
  // Causal tiles that all run at once, two a compute unit: the second ones shortest first, so that long ones share with short ones
  // (2 x 16 heads of 2,048 tokens, d 64, values 64: forward 61 -> 55 us, dQ 83 -> 80; 24 heads 57 -> 51, 80 -> 75).
  if (PER_CU == 2 && a.causal && !a.mask && gridDim.x <= 512 && id >= 256) id = 255 + gridDim.x - id;
  int turn = id / chunks;
  const int group = a.mask ? 1 : a.causal ? units : 8;
  const int first = turn / (tiles * group) * group, count = min(group, units - first);
  turn -= first * tiles;
  const int u = turn % count;
  t->unit = first + (count % 8 ? u : u % 8 * (count / 8) + u / 8);
  t->tile = backwards ? tiles - 1 - turn / count : turn / count;
  t->chunk = id % chunks;
  t->chunks = chunks;
  t->item = (int64_t)t->unit * tiles + t->tile;
  t->part = t->item * chunks + t->chunk;
  return true;
}

// The first query's position, taken so that no value of the device array leads out of a tensor.
__device__ __forceinline__ int start_of(const WaDiffLaunch& a, int b) {
  return a.q_start ? min(max(a.q_start[b], -a.q_len), a.kv_len) : a.kv_len - a.q_len;
}
// Query i sees the keys below this.
__device__ __forceinline__ int key_limit(const WaDiffLaunch& a, int keys, int start, int i) {
  return a.causal ? min(keys, max(start + i + 1, 0)) : keys;
}
// Keys of sequence b that its last query may see, so that any does: those behind them are neither read nor part of a tile, whatever
// they hold.
__device__ __forceinline__ int keys_of(const WaDiffLaunch& a, int b, int start) {
  const int keys = a.kv_lens ? min(max(a.kv_lens[b], 0), a.kv_len) : a.kv_len;
  return key_limit(a, keys, start, a.q_len - 1);
}

// A pointer that is the same in every lane, as scalar registers (the builtin returns signed words).
template <typename T>
__device__ __forceinline__ T* uniform_ptr(T* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
  return (T*)((uint64_t)hi << 32 | lo);
}

// Walks the kept blocks of one row (step 1) or column (step nb) of a head's mask: 64 entries at a time, one a lane, as
// a word of bits.
struct MaskWalk {
  const uint8_t* at = nullptr;  // entry 0; null: every block is kept
  int64_t step = 1;
  int entries = 0, word_i = -1;
  uint64_t word = 0;

  __device__ __forceinline__ void load(int w, int lane) {
    if (w == word_i) return;
    word_i = w;
    const int e = w * 64 + lane;
    word = __ballot(e < entries && at[e * step] != 0);
  }
  // Kept entry number k, or `entries` if there are fewer.
  __device__ __forceinline__ int nth(int k, int lane) {
    for (int w = 0; w * 64 < entries; ++w) {
      load(w, lane);
      const int n = __popcll(word);
      if (k < n) {
        uint64_t rest = word;
        for (; k > 0; --k) rest &= rest - 1;
        return w * 64 + __builtin_ctzll(rest);
      }
      k -= n;
    }
    return entries;
  }
  // First kept entry at or past j, or a value >= entries.
  __device__ __forceinline__ int next(int j, int lane) {
    while (j < entries) {
      load(j >> 6, lane);
      const uint64_t rest = word >> (j & 63);
      if (rest) return j + __builtin_ctzll(rest);
      j = (word_i + 1) * 64;
    }
    return j;
  }
};

// What the gradient takes from the forward, per row and map: the log-sum-exp of the scaled scores; the step in which the row of
// P_m V is held as 16-bit integers (its largest magnitude is 32767 steps, so dO . O_m is within 2^-16 of that times
// sum |dO|, where bfloat16 values gave dQ and dK a fifth more error in all); and the factor that takes probabilities recomputed
// from the float32 log-sum-exp (rounded by up to 2^-21) to the forward's, for the sum dlam.
struct RowStats {
  float lse, step, factor;
};
// top: the maximum the sum l was taken against, in log2 units; big: the row's largest |P_m V|
__device__ __forceinline__ RowStats row_stats(float top, float l, float big) {
  RowStats r = {-INFINITY, big * (1.f / 32767.f), 1.f};
  if (l != 0.f) {
    r.lse = (top + __log2f(l)) * kLn2;
    r.factor = __builtin_amdgcn_exp2f(r.lse * kLog2e - top) / l;
  }
  return r;
}
// Steps a unit; a row of nothing but 0, or too small for its step to have a reciprocal, is held as 0.
__device__ __forceinline__ float steps_per_unit(float step) { return step > 1e-37f ? 1.f / step : 0.f; }
__device__ __forceinline__ uint32_t pack_steps(float x, float y, float per_step) {
  return (uint32_t)(uint16_t)(int16_t)rintf(x * per_step) | (uint32_t)(uint16_t)(int16_t)rintf(y * per_step) << 16;
}

// The keys [*lo, *hi) of a chunk of a row tile that sees keys below `most`: of a listed task an equal number of the row's kept blocks,
// else equal ranges of whole blocks and tiles of KB.
template <int KB>
__device__ __forceinline__ void chunk_keys(const WaDiffLaunch& a, const Task& t, MaskWalk& walk, int most, int lane, int* lo, int* hi) {
  *lo = 0;
  *hi = most;
  if (t.chunks == 1) return;
  if (a.tasks) {
    const int shift = a.block == 128 ? 7 : 6, kept = a.tasks[4 + t.item];
    walk.entries = a.nb;
    if (t.chunk > 0) *lo = min(walk.nth(kept * t.chunk / t.chunks, lane) << shift, most);
    if (t.chunk + 1 < t.chunks) *hi = min(walk.nth(kept * (t.chunk + 1) / t.chunks, lane) << shift, most);
    walk.word_i = -1;
    return;
  }
  const int unit = a.mask ? max(a.block, KB) : KB, per = ((most + unit - 1) / unit + t.chunks - 1) / t.chunks;
  *lo = min((int64_t)t.chunk * per * unit, (int64_t)most);
  *hi = min((int64_t)*lo + per * unit, (int64_t)most);
}

// The value of lane % 32 and that of lane % 32 + 32. In assembly: the compiler reads both results of its builtin from
// one register. The exchange needs two wait states after a write of its operands.
__device__ __forceinline__ f32x2 both_halves(float x) {
  float lo = x, hi = x;
  asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(lo), "+v"(hi));
  const f32x2 v = {lo, hi};
  return v;
}
__device__ __forceinline__ float max_halves(float x) {
  const f32x2 v = both_halves(x);
  return fmaxf(v[0], v[1]);
}
__device__ __forceinline__ float add_halves(float x) {
  const f32x2 v = both_halves(x);
  return v[0] + v[1];
}

// Helpers of the gradients.
__device__ __forceinline__ void fill(f32x16& x, float f) {
#pragma unroll
  for (int v = 0; v < 16; ++v) x[v] = f;
}
// Registers 8 s to 8 s + 7 of a product as an operand over its rows.
__device__ __forceinline__ bf16x8 pack8(const float* p) {
  return as_bf16x8(make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])));
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

// The same from an address of the lane's own.
__device__ __forceinline__ void dma4_at(const void* from, const unsigned char* lds) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void_t*)lds);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %2, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(m0), "v"(from)
      : "memory");
}

}  // namespace wa
