// Internal launch interface of attention over packed sequences and over a paged cache (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

// [tokens][heads][head_dim] with free strides, in elements.
struct WaSeqRows {
  void* at;
  int64_t token, head;
};
// [pages][kv_heads][page][head_dim] with free strides, in elements.
struct WaSeqPages {
  void* at;
  int64_t page, head, token;
};

// How a forward call is cut into workgroups (see seq_attn.h).
struct WaSeqPlan {
  int32_t waves;      // wavefronts of a workgroup, 32 query rows each: 1 or 4
  int32_t per_tile;   // heads that share a tile: all of a key head, or 1
  int32_t log_tokens; // log2 of the tokens of a tile
  int32_t workers;    // workgroups, a multiple of 8
  int32_t min_units;  // tiles of keys that a worker gets at least
  int32_t whole;      // 1: no tile is cut
};
struct WaSeqLaunch {
  WaSeqRows q, k, v, o;    // k, v: of packed sequences
  WaSeqPages kp, vp;       // of a paged cache
  const int32_t* tables;   // [batch] rows of table_stride entries, table_width of them used
  int64_t table_stride;
  int32_t table_width, n_pages, page_shift;
  const int32_t* starts;   // [batch + 1]: first token of each sequence's queries, and their end
  const int32_t* kv_lens;  // [batch]: keys of each sequence; packed: its tokens
  float* lse;              // [heads][tokens] rows of lse_step, nullable: log-sum-exps, then (packed bf16) what O lost in rounding
  int32_t lse_step;
  int32_t* status;         // nullable
  int32_t batch, tokens, heads, kv_heads, head_dim, half, causal, paged;
  float scale;
  int32_t* any_cut;        // workspace: whether tiles are cut
  int2* cuts;              // workspace: [tokens][heads] (see seq_attn.h)
  float* part;             // workspace: partial tiles of the workers
  WaSeqPlan plan;
  // gradient
  WaSeqRows dout, dq, dk, dv;
  const float* lse_in;     // what the forward wrote, [heads][tokens] rows of lse_step
  float* rows;             // workspace: [2][heads][tokens]: what a query's products start from (packed_bwd.hip)
  void* cut_tiles;         // workspace: which tiles have parts (packed_bwd.hip)
  int64_t dq_part;         // floats of `part` that the parts of dQ may take; those of dK and dV lie behind
};

WaSeqPlan wa_seq_plan(const WaSeqLaunch& a);  // of its shape
int64_t wa_seq_most_tiles(const WaSeqLaunch& a, const WaSeqPlan& p);  // of all sequences and heads, at most
size_t wa_seq_part_floats(const WaSeqPlan& p, int head_dim);

hipError_t wa_launch_packed_attn(const WaSeqLaunch& a, hipStream_t stream);
hipError_t wa_launch_paged_attn(const WaSeqLaunch& a, hipStream_t stream);

// Gradient (packed_bwd.hip): tiles of 128 tokens of all sequences, at most; float32 results of tiles in parts, those of dQ and all.
int64_t wa_packed_backward_tiles(const WaSeqLaunch& a);
size_t wa_packed_backward_cut_bytes();
int64_t wa_packed_backward_dq_floats(const WaSeqLaunch& a);
int64_t wa_packed_backward_part_floats(const WaSeqLaunch& a);
hipError_t wa_launch_packed_backward(const WaSeqLaunch& a, hipStream_t stream);
