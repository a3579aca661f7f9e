// Attention over packed sequences (seq_attn.h), and how the calls of it and of paged_attn.hip are cut.

#include "seq_attn.h"

#include <algorithm>

WaSeqPlan wa_seq_plan(const WaSeqLaunch& a) {
  WaSeqPlan p{};
  const int group = a.heads / a.kv_heads;
  // One wavefront a tile where a sequence's new tokens, on average, fill no more rows with all heads of a key head.
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
#ifndef NW1
#define NW1 1024
#endif
#ifndef MU
#define MU 4
#endif
  p.workers = p.waves == 4 ? 512 : NW1;
  p.min_units = MU;
  return p;
}

size_t wa_seq_part_floats(const WaSeqPlan& p, int head_dim) { return (size_t)p.workers * 2 * 32 * p.waves * (head_dim + 2); }

hipError_t wa_launch_packed_attn(const WaSeqLaunch& a, hipStream_t stream) { return wa::seq_launch_any<false>(a, stream); }
