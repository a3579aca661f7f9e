// Internal launch interface of the differential-attention kernels (not part of the ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

struct WaDiffLaunch {
  const void* q;      // bf16 [batch][2 heads][q_len][head_dim]: maps 2h and 2h + 1 of head h
  const void* k;      // bf16 [batch][2 kv_heads][kv_len][head_dim]
  const void* v;      // bf16 [batch][kv_heads][kv_len][value_dim]
  const float* lam;   // [heads]
  const uint8_t* mask;     // [batch][heads][mb][nb], null: every block
  const int32_t* q_start;  // [batch], null: kv_len - q_len
  const int32_t* kv_lens;  // [batch], null: kv_len
  void* o;            // bf16 [batch][heads][q_len][value_dim]
  int16_t* maps;      // [batch][2 heads][q_len][value_dim]: P_m V in steps of its row's, nullable
  float* stats;       // [batch][2 heads][q_len][3]: log-sum-exp, step, correction (diff_tiles.h), with maps
  int32_t* order;     // workspace of masked calls: work items by falling length, then their lengths
  float* part;        // workspace of split calls: partial tiles, then (forward) their statistics
  int32_t batch, heads, kv_heads, q_len, kv_len, head_dim, value_dim, block, mb, nb, causal;
  float scale;
  // backward
  const void* dout;   // bf16 [batch][heads][q_len][value_dim]
  void* dq;
  void* dk;
  void* dv;
  float* dlam;        // [heads]
  float* rows;        // workspace: [batch][heads][4][q_len]: what the products of a query start from (diff_bwd.hip)
  double* lam_part;   // workspace: [batch][heads][tiles of q_len][parts] partial sums for dlam
};

// How a forward call is cut into workgroups (see diff_plan in diff_attn.hip).
struct WaDiffPlan {
  int32_t waves;   // wavefronts a map of a workgroup, 32 query rows each: 1, 2 or 4
  int32_t packed;  // 1: the rows of a tile run over the queries of all heads of a key head
  int32_t units;   // (sequence, head) or, packed, (sequence, key head) pairs
  int32_t tiles;   // row tiles of a unit
  int32_t splits;  // key ranges a tile is computed in
};
WaDiffPlan wa_diff_plan(const WaDiffLaunch& a, bool masked);
size_t wa_diff_part_floats(const WaDiffPlan& p, int value_dim);

// Tiles of masked calls run longest first where there are this many of them: fewer all run at once; with more, a long one
// that starts late is short next to the call, and running heads one after another keeps their keys in the caches.
constexpr int kDiffOrderMin = 257, kDiffOrderMax = 8192;
inline bool wa_diff_ordered(int64_t items) { return items >= kDiffOrderMin && items <= kDiffOrderMax; }
inline size_t wa_diff_order_ints(int64_t items) { return wa_diff_ordered(items) ? 2 * (size_t)items : 0; }
// Fills a.order for the rows of the mask, or for its columns summed over the heads of a key head (entry t of a unit u of n
// is item u n + t).
hipError_t wa_launch_diff_order(const WaDiffLaunch& a, bool columns, hipStream_t stream);

// How the gradient is cut: tiles of 32 * waves queries (keys), each tile's keys (queries of all heads) in so many parts.
struct WaDiffSide {
  int32_t waves, tiles, parts;
  int64_t items;  // tiles of all units
};
WaDiffSide wa_diff_dq_side(const WaDiffLaunch& a, bool masked);
WaDiffSide wa_diff_dkv_side(const WaDiffLaunch& a, bool masked);
// float32 of the parts' results, 0 where there is one
size_t wa_diff_dq_floats(const WaDiffLaunch& a, const WaDiffSide& s);
size_t wa_diff_dkv_floats(const WaDiffLaunch& a, const WaDiffSide& s);

hipError_t wa_launch_diff_attn(const WaDiffLaunch& a, hipStream_t stream);
hipError_t wa_launch_diff_backward(const WaDiffLaunch& a, hipStream_t stream);
