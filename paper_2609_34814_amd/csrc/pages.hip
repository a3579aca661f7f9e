// A paged cache's pages for gfx950 (MI355X): tokens stored into them, and pages dealt out, shared, given back and moved, with all
// state on the device, so that no call waits for the host.
//
// Free pages are those without references, and they are dealt out lowest first, so equal states give equal results: where pages are
// counted, ranks come from prefix sums (64 lanes by lane moves, 16 wavefronts through LDS), and the only atomics are integer additions
// and minima, whose order does not matter. The copies of pages are the cost: 16 bytes a lane, four on their way, 16 KiB a workgroup
// (262 MB read and written by a compaction: 42 us, 6.2 TB/s through the last-level cache); a call that copies little costs its launches, of 2.4
// to 6.4 us each.

#include "common.h"
#include "pages_launch.h"
#include "wavealign.h"

#include <algorithm>

namespace {

using namespace wa;

constexpr int kThreads = 1024, kPerThread = 16;   // the one workgroup that deals pages out
constexpr int kScan = kThreads * kPerThread;      // pages it looks at at a time
constexpr int kChunk = 4096;                      // pages of a workgroup of a compaction, 16 a thread
constexpr int kCopyBytes = 16384;                 // bytes of a workgroup's copy
constexpr int kNone = -1;

__device__ __forceinline__ void report(int32_t* status, int bit) {
  if (status) atomicOr(status, bit);
}
__device__ __forceinline__ int pages_of(int len, int shift) { return (int)(((int64_t)max(len, 0) + (1 << shift) - 1) >> shift); }

// Sum over the workgroup's threads before this one; *total: over all. T / 64 wavefronts; `lds` holds one int each, and is free again
// after the next barrier.
template <int T>
__device__ __forceinline__ int before_me(int x, int* total, int* lds) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int sum = lane_prefix_sum(x);
  __syncthreads();
  if (lane == 63) lds[w] = sum;
  __syncthreads();
  int base = 0, all = 0;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    const int y = lds[i];
    if (i < w) base += y;
    all += y;
  }
  *total = all;
  return base + sum - x;
}

// The lowest `wanted` free pages, in order, into `list`; returns how many there are of them.
__device__ __forceinline__ int lowest_free(const int32_t* refs, int n, int wanted, int32_t* list, int* lds) {
  int have = 0;
  for (int base = 0; base < n && have < wanted; base += kScan) {
    const int at = base + threadIdx.x * kPerThread;
    uint32_t free_bits = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
      if (at + i < n && refs[at + i] <= 0) free_bits |= 1u << i;
    int total;
    int rank = have + before_me<kThreads>(__popc(free_bits), &total, lds);
    for (; free_bits && rank < wanted; free_bits &= free_bits - 1) list[rank++] = at + __builtin_ctz(free_bits);
    have += total;
  }
  __syncthreads();
  return min(have, wanted);
}

// ws: [sequences] where a sequence's pages begin in the list (kNone: it takes none), then the list.
__global__ __launch_bounds__(kThreads) void page_grow_kernel(const WaPageLaunch a) {
  __shared__ int lds[kThreads / 64];
  int32_t *offset = a.ws, *list = a.ws + a.sequences;
  auto need = [&](int s) {  // kNone: no room in the table
    const int have = pages_of(a.lens[s], a.shift), want = pages_of(a.first[s], a.shift);
    return want <= have ? 0 : want > a.width ? kNone : want - have;
  };
  // Pages wanted in all, where a need past the pool counts as one page more than it has, so that it always leaves `have` behind (1,024 needs
  // of up to 2^20 pages fit an int).
  int wanted = 0;
  for (int base = 0; base < a.sequences; base += kThreads) {
    const int s = base + threadIdx.x, n = s < a.sequences ? need(s) : 0;
    int total;
    const int at = before_me<kThreads>(min(max(n, 0), a.n_pages + 1), &total, lds);
    if (s < a.sequences) offset[s] = (int)min((int64_t)wanted + at, (int64_t)INT32_MAX);
    if (n == kNone) report(a.status, WA_PAGE_EXHAUSTED);
    wanted = (int)min((int64_t)wanted + total, (int64_t)a.n_pages + 1);
  }
  __syncthreads();
  const int have = lowest_free(a.refs, a.n_pages, min(wanted, a.n_pages), list, lds);
  const int lane = threadIdx.x & 63;
  if (wanted > have && threadIdx.x < 64) {  // one after another, 64 of them read at a time: who finds too few takes none
    if (lane == 0) report(a.status, WA_PAGE_EXHAUSTED);
    int at = 0;
    for (int base = 0; base < a.sequences; base += 64) {
      const int n = base + lane < a.sequences ? max(need(base + lane), 0) : 0;
      int mine = kNone;
      for (int i = 0; i < 64; ++i) {
        const int x = __builtin_amdgcn_readlane(n, i);
        if (x > have - at) continue;
        if (lane == i) mine = at;
        at += x;
      }
      if (base + lane < a.sequences) offset[base + lane] = mine;
    }
  }
  __syncthreads();
  for (int s = threadIdx.x >> 6; s < a.sequences; s += kThreads / 64) {
    const int n = need(s), from = offset[s], have_pages = pages_of(a.lens[s], a.shift);
    if (n == kNone || from == kNone || n > have - from) continue;
    for (int i = lane; i < n; i += 64) {
      const int p = list[from + i];
      a.tables[(int64_t)s * a.width + have_pages + i] = p;
      a.refs[p] = 1;
    }
    if (lane == 0 && a.first[s] > a.lens[s]) a.lens[s] = a.first[s];
  }
}

// One entry of a fork. len: the parent's tokens, of which whole pages are shared; the last page, if it is copied, goes from `from` to `to`.
struct Fork {
  int32_t parent, child, len, from, to;
};

// ws: [sequences] the entry that has a child, then the list of free pages, then the entries' Fork, child kNone: left out.
__device__ __forceinline__ Fork* forks_of(const WaPageLaunch& a) { return (Fork*)(a.ws + a.sequences + a.entries); }

__global__ __launch_bounds__(kThreads) void page_fork_kernel(const WaPageLaunch a) {
  __shared__ int lds[kThreads / 64];
  int32_t *owner = a.ws, *list = a.ws + a.sequences;
  Fork* forks = forks_of(a);
  auto known = [&](int s) { return (uint32_t)s < (uint32_t)a.sequences; };
  for (int i = threadIdx.x; i < a.entries; i += kThreads)
    if (known(a.second[i])) owner[a.second[i]] = INT32_MAX;
  __syncthreads();
  for (int i = threadIdx.x; i < a.entries; i += kThreads)
    if (known(a.second[i])) atomicMin(&owner[a.second[i]], i);
  __syncthreads();
  // until the free pages are known, `to` is a copy's rank
  int wanted = 0;
  for (int base = 0; base < a.entries; base += kThreads) {
    const int i = base + threadIdx.x;
    Fork f = {0, kNone, 0, kNone, kNone};
    if (i < a.entries) {
      f.parent = a.first[i];
      const int child = a.second[i];
      if (!known(f.parent) || !known(child)) {
        report(a.status, WA_PAGE_BAD_INDEX);
      } else if (a.lens[child] > 0 || atomicAdd(&owner[child], 0) != i) {
        report(a.status, WA_PAGE_BUSY);
      } else {
        f.child = child;
        f.len = max(a.lens[f.parent], 0);
        if (f.len & ((1 << a.shift) - 1)) {
          const int last = f.len >> a.shift;
          f.from = last < a.width ? a.tables[(int64_t)f.parent * a.width + last] : kNone;
          if ((uint32_t)f.from >= (uint32_t)a.n_pages) {
            report(a.status, WA_PAGE_BAD_INDEX);
            f.child = f.from = kNone;
          }
        }
      }
    }
    int total;
    const int rank = wanted + before_me<kThreads>(f.from != kNone ? 1 : 0, &total, lds);
    if (i < a.entries) {
      f.to = f.from != kNone ? rank : kNone;
      forks[i] = f;
    }
    wanted += total;
  }
  __syncthreads();
  const int have = lowest_free(a.refs, a.n_pages, wanted, list, lds);
  for (int i = threadIdx.x; i < a.entries; i += kThreads) {
    Fork f = forks[i];
    if (f.child == kNone) continue;
    if (f.to != kNone) {
      if (f.to >= have) {
        report(a.status, WA_PAGE_EXHAUSTED);
        forks[i].child = kNone;
        continue;
      }
      forks[i].to = list[f.to];
      a.refs[list[f.to]] = 1;
    }
  }
}

// 16 KiB at `at` of a page, 256 threads.
__device__ __forceinline__ void copy_chunk(const unsigned char* from, unsigned char* to, int64_t at, int64_t bytes) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t b = at + i * 4096 + threadIdx.x * 16;
    if (b < bytes) x[i] = *(const u32x4*)(from + b);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t b = at + i * 4096 + threadIdx.x * 16;
    if (b < bytes) *(u32x4*)(to + b) = x[i];
  }
}
__host__ __device__ inline int64_t chunks_of(int64_t page_bytes) { return (page_bytes + kCopyBytes - 1) / kCopyBytes; }
// chunk `job` of copying a page in every plane
__device__ __forceinline__ void copy_page(const WaPageLaunch& a, int from, int to, int64_t job) {
  const int64_t chunks = chunks_of(a.page_bytes), plane = job / chunks, at = (job - plane * chunks) * kCopyBytes;
  unsigned char* base = a.pool + plane * a.n_pages * a.page_bytes;
  copy_chunk(base + from * a.page_bytes, base + to * a.page_bytes, at, a.page_bytes);
}

// Workgroups [0, entries): the tables, references and lengths of the children; then those of the copies.
__global__ __launch_bounds__(256) void page_fork_fill_kernel(const WaPageLaunch a, int64_t jobs) {
  const Fork* forks = forks_of(a);
  if (blockIdx.x < (unsigned)a.entries) {
    const Fork f = forks[blockIdx.x];
    if (f.child == kNone) return;
    const int32_t* from = a.tables + (int64_t)f.parent * a.width;
    int32_t* to = a.tables + (int64_t)f.child * a.width;
    const int full = min(f.len >> a.shift, a.width);
    for (int i = threadIdx.x; i < full; i += 256) {
      const int p = from[i];
      to[i] = p;
      if ((uint32_t)p < (uint32_t)a.n_pages)
        atomicAdd(&a.refs[p], 1);
      else
        report(a.status, WA_PAGE_BAD_INDEX);
    }
    if (threadIdx.x == 0) {
      if (f.to != kNone) to[full] = f.to;
      a.lens[f.child] = f.len;
    }
    return;
  }
  const int64_t job = blockIdx.x - (int64_t)a.entries, entry = job / jobs;
  const Fork f = forks[entry];
  if (f.child != kNone && f.to != kNone) copy_page(a, f.from, f.to, job - entry * jobs);
}

__global__ __launch_bounds__(256) void page_free_kernel(const WaPageLaunch a) {
  __shared__ int held;
  const int s = a.first[blockIdx.x];
  if ((uint32_t)s >= (uint32_t)a.sequences) {
    if (threadIdx.x == 0) report(a.status, WA_PAGE_BAD_INDEX);
    return;
  }
  // the length is taken once, whichever of the entries of a sequence comes first
  if (threadIdx.x == 0) held = min(pages_of(atomicExch(&a.lens[s], 0), a.shift), a.width);
  __syncthreads();
  for (int i = threadIdx.x; i < held; i += 256) {
    const int p = a.tables[(int64_t)s * a.width + i];
    if ((uint32_t)p < (uint32_t)a.n_pages)
      atomicSub(&a.refs[p], 1);
    else
      report(a.status, WA_PAGE_BAD_INDEX);
  }
}

// Compaction. ws: [chunks] used pages of each chunk; then [n_pages] a moving page's rank, kNone for others; [n_pages] the holes by rank;
// [n_pages] the moving pages by rank; [2] how many move, how many are in use.
struct Compact {
  int32_t *counts, *rank, *hole, *from, *moves;
  __host__ __device__ explicit Compact(const WaPageLaunch& a) {
    const int chunks = (a.n_pages + kChunk - 1) / kChunk;
    counts = a.ws;
    rank = counts + chunks;
    hole = rank + a.n_pages;
    from = hole + a.n_pages;
    moves = from + a.n_pages;
  }
};

// used pages of [base + 16 thread, + 16) that lie below `end`, as bits
__device__ __forceinline__ uint32_t used_bits(const int32_t* refs, int base, int end) {
  const int at = base + threadIdx.x * 16;
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (at + i < end && refs[at + i] > 0) bits |= 1u << i;
  return bits;
}

__global__ __launch_bounds__(256) void page_count_kernel(const WaPageLaunch a) {
  __shared__ int lds[4];
  int total;
  before_me<256>(__popc(used_bits(a.refs, blockIdx.x * kChunk, a.n_pages)), &total, lds);
  if (threadIdx.x == 0) Compact(a).counts[blockIdx.x] = total;
}

__global__ __launch_bounds__(256) void page_plan_kernel(const WaPageLaunch a, int counted) {
  __shared__ int lds[4];
  const Compact c(a);
  const int chunks = gridDim.x, base = blockIdx.x * kChunk;
  const uint32_t bits = used_bits(a.refs, base, a.n_pages);
  int mine;
  const int rank_in = before_me<256>(__popc(bits), &mine, lds);
  // used pages of all chunks, of those before this one
  int u = mine, before = 0;
  if (counted) {
    int all = 0, front = 0;
    for (int i = threadIdx.x; i < chunks; i += 256) {
      all += c.counts[i];
      if (i < (int)blockIdx.x) front += c.counts[i];
    }
    before_me<256>(all, &u, lds);
    before_me<256>(front, &before, lds);
  }
  // used pages below u
  int below = 0;
  {
    const int whole = counted ? u / kChunk : 0, part = whole * kChunk;
    int x = 0;
    for (int i = threadIdx.x; i < whole; i += 256) x += c.counts[i];
    if (part < a.n_pages) x += __popc(used_bits(a.refs, part, u));
    before_me<256>(x, &below, lds);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    c.moves[0] = u - below;
    c.moves[1] = u;
    if (a.used) *a.used = u;
  }
  int rank = before + rank_in;  // used pages before the thread's first
  const int at = base + threadIdx.x * 16;
  for (int i = 0; i < 16 && at + i < a.n_pages; ++i) {
    const int p = at + i;
    const bool is_used = bits >> i & 1;
    c.rank[p] = is_used && p >= u ? rank - below : kNone;
    if (is_used && p >= u) c.from[rank - below] = p;
    if (!is_used && p < u) c.hole[p - rank] = p;
    rank += is_used;
  }
}

// Workgroups [0, table_wgs): the tables; then [0, ref_wgs): the references; then the copies, as many as come.
__global__ __launch_bounds__(256) void page_move_kernel(const WaPageLaunch a, int table_wgs, int ref_wgs) {
  const Compact c(a);
  int wg = blockIdx.x;
  if (wg < table_wgs) {
    const int64_t all = (int64_t)a.sequences * a.width;
    for (int64_t i = (int64_t)wg * 256 + threadIdx.x; i < all; i += (int64_t)table_wgs * 256) {
      const int s = (int)(i / a.width), e = (int)(i - (int64_t)s * a.width);
      int p = a.tables[i];
      if (e < pages_of(a.lens[s], a.shift)) {
        if ((uint32_t)p >= (uint32_t)a.n_pages) {
          report(a.status, WA_PAGE_BAD_INDEX);
        } else {
          const int r = c.rank[p];
          if (r != kNone) p = c.hole[r];
        }
      }
      a.out_tables[i] = p;
    }
    return;
  }
  wg -= table_wgs;
  const int moves = *c.moves;
  if (wg < ref_wgs) {
    for (int p = wg * 256 + threadIdx.x; p < a.n_pages; p += ref_wgs * 256) {
      if (p < moves) {  // the p-th move
        const int from = c.from[p], to = c.hole[p];
        a.out_refs[to] = a.refs[from];
        a.out_refs[from] = 0;
      }
      // what is neither a hole nor moves stays; where nothing is copied, refs change under this read and must not be asked
      if (a.out_refs != a.refs && c.rank[p] == kNone && !(a.refs[p] <= 0 && p < c.moves[1])) a.out_refs[p] = a.refs[p];
    }
    return;
  }
  wg -= ref_wgs;
  const int64_t jobs = a.planes * chunks_of(a.page_bytes), all = moves * jobs;
  for (int64_t i = wg; i < all; i += gridDim.x - table_wgs - ref_wgs) {
    const int k = (int)(i / jobs);
    copy_page(a, c.from[k], c.hole[k], i - k * jobs);
  }
}

__global__ __launch_bounds__(256) void page_copy_kernel(const WaPageLaunch a, int64_t jobs) {
  const int64_t entry = blockIdx.x / jobs, job = blockIdx.x - entry * jobs;
  const int from = a.first[entry], to = a.second[entry];
  if ((uint32_t)from >= (uint32_t)a.n_pages || (uint32_t)to >= (uint32_t)a.n_pages) {
    if (job == 0 && threadIdx.x == 0) report(a.status, WA_PAGE_BAD_INDEX);
    return;
  }
  copy_page(a, from, to, job);
}

// A wavefront TOKENS tokens: their keys and values, 16 bytes a lane. A token's sequence is the last that begins at or before it, found with a
// start a lane; its place is looked up by the lane of the token's number, for all tokens at once. One token a wavefront where there are few
// (32 tokens of 8 heads of 128, 4.3 us), else four, whose rows are on their way while the places are looked up (16,384 tokens 34.7 -> 29.7 us,
// 4.5 TB/s: their copy's bytes alone take 26.6).
template <int TOKENS>
__global__ __launch_bounds__(256) void page_store_kernel(const WaSeqLaunch a) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63;
  const int token0 = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)) * TOKENS);
  if (token0 >= a.tokens) return;
  const int log_row = a.head_dim == 128 ? 4 : 3, n = a.kv_heads << log_row, in_row = (1 << log_row) - 1;
  auto from = [&](int token, int x) {
    const WaSeqRows& r = x < n ? a.k : a.v;
    const int y = x < n ? x : x - n;
    return (const u32x4*)((const uint16_t*)r.at + (int64_t)token * r.token + (y >> log_row) * r.head + (y & in_row) * 8);
  };
  constexpr int kAhead = 4;  // rows of up to 16 heads of 64, or 8 of 128, wait for their place in registers
  u32x4 x[TOKENS][kAhead];
#pragma unroll
  for (int t = 0; t < TOKENS; ++t)
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (lane + 64 * i < 2 * n) x[t][i] = *from(min(token0 + t, a.tokens - 1), lane + 64 * i);
  int b[TOKENS];
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) b[t] = -1;
  for (int base = 0; base <= a.batch; base += 64) {
    const int y = base + lane <= a.batch ? a.starts[base + lane] : INT32_MAX;
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) b[t] += __popcll(__ballot(y <= token0 + t));
  }
  // lane t: token t's sequence, page and row; no page: below 0
  const int token = token0 + lane;
  int mine = b[0], page = -1, row = 0;
#pragma unroll
  for (int t = 1; t < TOKENS; ++t)
    if (lane == t) mine = b[t];
  if (lane < TOKENS && token < a.tokens && mine >= 0 && mine < a.batch) {
    const int first = a.starts[mine], end = min(a.starts[mine + 1], a.tokens);
    const int64_t at = (int64_t)a.kv_lens[mine] - (end - token);
    if (token >= first && token < end && at >= 0) {
      const int64_t entry = at >> a.page_shift;
      page = entry < a.table_width ? a.tables[mine * a.table_stride + entry] : -1;
      row = (int)at & ((1 << a.page_shift) - 1);
      if ((uint32_t)page >= (uint32_t)a.n_pages) {
        report(a.status, WA_PAGE_BAD_INDEX);
        page = -1;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) {
    const int64_t p = __builtin_amdgcn_readlane(page, t);
    if (p < 0) continue;
    const int r = __builtin_amdgcn_readlane(row, t);
    auto to = [&](int x) {
      const WaSeqPages& g = x < n ? a.kp : a.vp;
      const int y = x < n ? x : x - n;
      return (u32x4*)((uint16_t*)g.at + p * g.page + (y >> log_row) * g.head + r * g.token + (y & in_row) * 8);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (lane + 64 * i < 2 * n) *to(lane + 64 * i) = x[t][i];
    for (int i = lane + 64 * kAhead; i < 2 * n; i += 64) *to(i) = *from(token0 + t, i);
  }
}

}  // namespace

size_t wa_page_ws_ints(const WaPageLaunch& a) {
  const size_t grow = (size_t)a.sequences + a.n_pages;
  const size_t fork = (size_t)a.sequences + 6 * (size_t)a.entries;
  const size_t compact = ((size_t)a.n_pages + kChunk - 1) / kChunk + 3 * (size_t)a.n_pages + 2;
  return std::max({grow, fork, compact});
}

hipError_t wa_launch_page_grow(const WaPageLaunch& a, hipStream_t stream) {
  hipLaunchKernelGGL(page_grow_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t wa_launch_page_fork(const WaPageLaunch& a, hipStream_t stream) {
  hipLaunchKernelGGL(page_fork_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t jobs = a.planes * chunks_of(a.page_bytes);
  hipLaunchKernelGGL(page_fork_fill_kernel, dim3((unsigned)(a.entries * (jobs + 1))), dim3(256), 0, stream, a, jobs);
  return hipGetLastError();
}

hipError_t wa_launch_page_free(const WaPageLaunch& a, hipStream_t stream) {
  hipLaunchKernelGGL(page_free_kernel, dim3((unsigned)a.entries), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t wa_launch_page_compact(const WaPageLaunch& a, hipStream_t stream) {
  const int chunks = (a.n_pages + kChunk - 1) / kChunk;
  hipError_t e = hipSuccess;
  if (chunks > 1) {
    hipLaunchKernelGGL(page_count_kernel, dim3(chunks), dim3(256), 0, stream, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(page_plan_kernel, dim3(chunks), dim3(256), 0, stream, a, chunks > 1);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int table_wgs = (int)std::min<int64_t>(((int64_t)a.sequences * a.width + 1023) / 1024, 1024);
  const int ref_wgs = std::min((a.n_pages + 255) / 256, 256);
  // at most half of the pages move
  const int64_t most = (a.n_pages / 2) * a.planes * chunks_of(a.page_bytes);
  const int copy_wgs = (int)std::max<int64_t>(1, std::min<int64_t>(most, 4096));
  hipLaunchKernelGGL(page_move_kernel, dim3(table_wgs + ref_wgs + copy_wgs), dim3(256), 0, stream, a, table_wgs, ref_wgs);
  return hipGetLastError();
}

hipError_t wa_launch_page_copy(const WaPageLaunch& a, hipStream_t stream) {
  const int64_t jobs = a.planes * chunks_of(a.page_bytes);
  hipLaunchKernelGGL(page_copy_kernel, dim3((unsigned)(a.entries * jobs)), dim3(256), 0, stream, a, jobs);
  return hipGetLastError();
}

hipError_t wa_launch_page_store(const WaSeqLaunch& a, hipStream_t stream) {
  if (a.tokens >= 4096)
    hipLaunchKernelGGL(page_store_kernel<4>, dim3((unsigned)(((int64_t)a.tokens + 15) / 16)), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(page_store_kernel<1>, dim3((unsigned)(((int64_t)a.tokens + 3) / 4)), dim3(256), 0, stream, a);
  return hipGetLastError();
}
