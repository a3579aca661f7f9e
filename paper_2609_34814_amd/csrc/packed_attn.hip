// Attention over packed sequences (seq_attn.h), and how the calls of it and of paged_attn.hip are cut.

#include "seq_attn.h"

#include <algorithm>

WaSeqPlan wa_seq_plan(const WaSeqLaunch& a) {
  WaSeqPlan p{};
  const int group = a.heads / a.kv_heads;
  // One wavefront a tile where a sequence's new tokens, on average, fill no more rows with all heads of a key head. The host knows the average
  // alone, and empty sequences count: 8,192 tokens of one, 32 heads over 8, take 530 us alone or in 256 slots, 1,223 in 1,024.
  const int64_t mean = ((int64_t)a.tokens + a.batch - 1) / std::max(a.batch, 1);
  p.waves = mean * group <= 32 ? 1 : 4;
  const int rows = 32 * p.waves;
  auto log_tokens = [&](int heads) {
    int l = 0;
    while ((heads << (l + 1)) <= rows) ++l;
    return l;
  };
  p.per_tile = group;
  p.log_tokens = group <= rows ? log_tokens(group) : 0;
  // heads that would leave more than an eighth of the rows empty go alone, but for few tokens
  if (group > rows || (mean * group > rows && (group << p.log_tokens) * 8 < rows * 7)) {
    p.per_tile = 1;
    p.log_tokens = log_tokens(1);
  }
  // Workgroups that the chip holds: two a compute unit of four wavefronts (of d 64 three fit, which as workers are no faster), four of one (a
  // fifth does not fit beside the LDS of four: one token of 32 sequences 162 us with 1,024, 197 with 1,280).
  p.workers = p.waves == 4 ? 512 : 1024;
  p.min_units = 4;
  // Calls whose tiles are never cut need no second kernel. Packed: tiles of fifteen tiles of keys at most, many short sequences
  // (1,000 tokens of 16: 21.7 -> 14.4 us; but 32,768 tokens of one head among 255 empty slots take 534 us, alone 286), and those of one wavefront
  // a tile. Over a cache, whose lengths the host does not know, tables of few keys: few keys a tile take less time than a join (one
  // wavefront: 100 sequences of up to 300 keys 23.5 -> 19.7 us, but 16 of 500 19.6 -> 24.6; four: 512 tokens of 32 heads 25.0 -> 18.0).
  if (a.paged) {
    const int64_t keys = (int64_t)a.table_width << a.page_shift;
    p.whole = keys <= (p.waves == 4 ? 512 : 256) || (p.waves == 1 && keys <= 512 && wa_seq_most_tiles(a, p) >= 256);
  } else {
    p.whole = a.tokens <= 960 || mean <= 128;
  }
  return p;
}

// Sequences of n_b queries have sum ceil(n_b / p) tiles of p tokens.
int64_t wa_seq_most_tiles(const WaSeqLaunch& a, const WaSeqPlan& p) {
  return ((a.tokens >> p.log_tokens) + std::min(a.batch, a.tokens)) * (int64_t)(a.heads / p.per_tile);
}

size_t wa_seq_part_floats(const WaSeqPlan& p, int head_dim) { return (size_t)p.workers * 2 * 32 * p.waves * (head_dim + 2); }

hipError_t wa_launch_packed_attn(const WaSeqLaunch& a, hipStream_t stream) { return wa::seq_launch_any<false>(a, stream); }
