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
  float* stats;       // [batch][2 heads][q_len][3]: log-sum-exp, step, factor (diff_tiles.h), with maps
  int32_t* tasks;     // workspace of masked calls (see wa_diff_task_ints); null: tiles are dealt out by number
  int32_t task_items; // tiles that `tasks` is about
  float* part;        // workspace of split calls: part_tiles partial tiles, then (forward) their statistics
  int64_t part_tiles;
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

// How a forward call is cut into workgroups (see wa_diff_plan in diff_attn.hip).
struct WaDiffPlan {
  int32_t waves;   // wavefronts a map of a workgroup, 32 query rows each: 1, 2 or 4
  int32_t packed;  // 1: the rows of a tile run over the queries of all heads of a key head
  int32_t units;   // (sequence, head) or, packed, (sequence, key head) pairs
  int32_t tiles;   // row tiles of a unit
  int32_t splits;  // key ranges a tile is computed in
};
WaDiffPlan wa_diff_plan(const WaDiffLaunch& a, bool masked);
size_t wa_diff_part_floats(const WaDiffPlan& p, bool masked, int value_dim);

// Masked calls of this many tiles run a list of tasks, longest first, in which tiles of more kept blocks than a workgroup's share of
// the call are cut into chunks. Fewer tiles all run at once (or are cut into key ranges by their number alone); with more, a long one
// that starts late is short next to the call, and running heads one after another keeps their keys in the caches.
constexpr int kDiffTasksMin = 257, kDiffTasksMax = 8192, kDiffMaxChunks = 16;
inline bool wa_diff_has_tasks(int64_t items) { return items >= kDiffTasksMin && items <= kDiffTasksMax; }
// Workgroups that fill the chip, of so many wavefronts a map (or a workgroup of the gradient).
__host__ __device__ inline int wa_diff_slots(int waves) { return waves == 4 ? 256 : 512; }
// The list: [0] tasks, [1] cut tiles; from 4 the kept blocks of each tile; then tasks {tile, chunk, chunks, first partial tile}, at
// most one more a slot than there are tiles; then cut tiles {tile, chunks, first partial tile, 0}, at most one a slot. Their chunks
// are at most two a slot.
__host__ __device__ inline int wa_diff_task_list(int items) { return 4 + (items + 3) / 4 * 4; }
__host__ __device__ inline int wa_diff_cut_list(int items, int slots) { return wa_diff_task_list(items) + 4 * (items + slots); }
inline size_t wa_diff_task_ints(int64_t items, int slots) {
  return wa_diff_has_tasks(items) ? (size_t)wa_diff_cut_list((int)items, slots) + 4 * slots : 0;
}
// Fills a.tasks for the rows of the mask, or for its columns with the rows of all heads of a key head (entry t of a unit u of n is
// tile u n + t).
hipError_t wa_launch_diff_tasks(const WaDiffLaunch& a, bool columns, int slots, hipStream_t stream);

// How the gradient is cut: tiles of 32 * waves queries (keys), each tile's keys (queries of all heads) in so many parts.
struct WaDiffSide {
  int32_t waves, tiles, parts;
  int64_t items;  // tiles of all units
};
WaDiffSide wa_diff_dq_side(const WaDiffLaunch& a, bool masked);
WaDiffSide wa_diff_dkv_side(const WaDiffLaunch& a, bool masked);
// Partial tiles of a side: of its parts, or of its tasks; 0 where no tile is cut.
int64_t wa_diff_side_tiles(const WaDiffSide& s, bool masked);

hipError_t wa_launch_diff_attn(const WaDiffLaunch& a, hipStream_t stream);
hipError_t wa_launch_diff_backward(const WaDiffLaunch& a, hipStream_t stream);
