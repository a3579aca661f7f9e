// Gradient of attention over packed sequences for gfx950 (MI355X). With P recomputed from the forward's log-sum-exps,
//   dP = dO V^T,   D = dO . O,   dS = P (dP - D),   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO.
//
// Three kernels. packed_rows_kernel: what the products of a query start from, its log-sum-exp and D. packed_grad_kernel: jobs of two kinds,
// each owning what it writes, so nothing is added with atomics and equal calls give equal bits:
//   keys     128 keys, over the queries of all heads that share them: dK and dV.
//   queries  128 queries of a head, over their keys: dQ.
// They run in one launch, those of keys first, which take longer, so that the others fill the chip while the last of them end (8,192 tokens of 7
// documents, 16 heads over 4, d 128: 163 + 121 us one after another, 240 together: 0.93 PFLOP/s of these seven products, 0.63 counting the formula's
// five, matrix cores 50% busy;
// what bounds it is two wavefronts a SIMD that take turns at products and exponentials). Long tiles are computed in parts, which
// packed_parts_kernel adds in order.
// Both recompute the scores and dP. A wavefront holds 32 queries (keys) with their accumulators in registers, and the other side's
// tiles pass through LDS, copied one ahead. Scores come out with the wavefront's own index in the lanes and the other in the
// registers, so P and dS, rounded to bf16, are operands of the following products as they are. Two wavefronts share a SIMD; the one that is
// at scores and dP goes first (16,384 tokens, 32 heads over 8, d 128: 7.24 -> 6.65 ms).

#include "packed_jobs.h"
#include "seq_attn.h"

#include <algorithm>

namespace {

using namespace wa;

constexpr int kRows = 128, kWaves = 4, kAhead = 2;

// Neighbouring units, which may share keys, on one XCD where eight divides their number.
__device__ __forceinline__ int spread(int u, int units) { return units % 8 ? u : u % 8 * (units / 8) + u / 8; }

template <int D>
struct Bwd {
  static constexpr int RB = D * 2, DT = D / 32, KS = D / 16;
  // Values lie in LDS where, with the keys and the sums of dK and dV, they do not fit the registers; queries then pass 32 at a time.
  static constexpr bool kValuesInLds = D == 128;
  static constexpr int KB = 64, QB = kValuesInLds ? 32 : 64;
};

// acc (rows: columns of the output) to the lane's output row, times f, 16 bytes a store
template <int T>
__device__ __forceinline__ void store_row16(uint16_t* out, const f32x16 (&acc)[T], float f, int hf, bool valid) {
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int v = 0; v < 16; v += 8) {
      const uint4 eight = gather8(
          make_uint2(pack_bf16x2(acc[t][v] * f, acc[t][v + 1] * f), pack_bf16x2(acc[t][v + 2] * f, acc[t][v + 3] * f)),
          make_uint2(pack_bf16x2(acc[t][v + 4] * f, acc[t][v + 5] * f), pack_bf16x2(acc[t][v + 6] * f, acc[t][v + 7] * f)));
      if (valid) *(uint4*)(out + t * 32 + 2 * v + 8 * hf) = eight;
    }
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ Seq one_seq(int b) {
  Seq s = seq_of<false>(seq_args(), b);
  s.first = __builtin_amdgcn_readfirstlane(s.first);
  s.n = __builtin_amdgcn_readfirstlane(s.n);
  s.keys = __builtin_amdgcn_readfirstlane(s.keys);
  return s;
}

// A tile of 128 rows, or the part of one, that a workgroup computes. Its length is the tiles of the other side that it meets.
struct Job {
  int b, tile, col;        // sequence, tile of it, head or key head
  int length, part, parts;  // the numbers of a tile's parts among all jobs are `cols` apart
  int number;               // the tile's, among all: those in parts come first
};

// All tiles of all sequences and `cols` heads, longest first, those longer than `most` in parts of about equal length: `most` takes as
// long as a 512th of all work, so that a call of few tiles fills the chip's workgroups (two a compute unit) once, and one of many is not cut.
// Where starts descend there are no jobs: sequences could overlap, which would write rows twice, in no order, and have more tiles and parts
// than there is room for. A pair of a key and a query takes four products for dK and dV and three for dQ.
// Causal tiles have the lengths 1 to T of a sequence of T tiles, others T. Each workgroup finds its job itself: the lengths are on the
// device. The tiles of the first 64 kHeld sequences are held, one a lane.
template <int kHeld>
struct Jobs {
  SeqArgs a;
  int lane, cols, batch, held[kHeld], longest, most;
  bool causal, queries;

  // share: of the kind of jobs in all work, in sevenths
  __device__ __forceinline__ Jobs(int lane_, int cols_, int share, bool queries_)
      : a(seq_args()), lane(lane_), cols(cols_), batch(a->batch), causal(a->causal), queries(queries_) {
    int64_t sum = 0;
    int n[kHeld], least = 0, top = 0;  // least: below 0 where starts descend
#pragma unroll
    for (int i = 0; i < kHeld; ++i) n[i] = 64 * i < batch ? tokens_of(64 * i + lane) : 0;
    auto add = [&](int x) {
      const int64_t t = tiles(x);
      least = min(least, x);
      top = max(top, (int)t);
      sum += causal ? t * (t + 1) / 2 : t * t;
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      held[i] = tiles(n[i]);
      if (64 * i < batch) add(n[i]);
    }
    for (int base = 64 * kHeld; base < batch; base += 64) add(tokens_of(base + lane));
    if (__ballot(least < 0)) batch = 0;
    sum = lane64(lane_prefix_sum64(sum, lane), 63) * cols;
    longest = lane_max(top);
    most = longest_whole(sum, share, longest);
  }
  // below 0 where the next sequence begins before this one
  __device__ __forceinline__ int tokens_of(int b) const {
    if (b >= batch) return 0;
    const SeqArgs x = again(a);
    return min(max(x->starts[b + 1], 0), x->tokens) - min(max(x->starts[b], 0), x->tokens);
  }
  static __device__ __forceinline__ int tiles(int n) { return (n + kRows - 1) / kRows; }
  // f(first sequence, tiles of sequence first + lane) for all, while it says so
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (64 * i >= batch || !f(64 * i, held[i])) return;
    for (int base = 64 * kHeld; base < batch; base += 64)
      if (!f(base, tiles(tokens_of(base + lane)))) return;
  }
  // those of tiles longer than `length`, of one column
  __device__ __forceinline__ int above(int length) const {
    int sum = 0;
    each([&](int, int t) {
      sum += t <= length ? 0 : causal ? jobs_upto(t, most) - jobs_upto(length, most) : t * parts_of(t, most);
      return true;
    });
    return lane_sum(sum);
  }
  // tiles longer than `length`, of one column
  __device__ __forceinline__ int longer(int length) const {
    int sum = 0;
    each([&](int, int t) {
      sum += t <= length ? 0 : causal ? t - length : t;
      return true;
    });
    return lane_sum(sum);
  }
  // job number `rank`; false if there is none
  __device__ __forceinline__ bool find(int64_t rank, Job* job) const {
    int lo = 0, hi = longest, passed = 0;  // above(lo) > row of jobs >= above(hi) = passed
    const int row = (int)(rank / cols);
    if (row >= above(0)) return false;
    while (hi - lo > 1) {
      const int mid = lo + ((hi - lo) >> 1), n = above(mid);
      if (n > row) {
        lo = mid;
      } else {
        hi = mid;
        passed = n;
      }
    }
    job->length = hi;
    job->parts = parts_of(hi, most);
    int k = (row - passed) / job->parts;
    job->part = row - passed - k * job->parts;
    job->number = (longer(hi) + k) * cols + (int)(rank - (int64_t)row * cols);
    job->col = spread((int)(rank - (int64_t)row * cols), cols);
    // the k-th tile of this length
    int who = 0, tile = 0, t = 0;
    each([&](int base, int x) {
      const int n = causal ? x >= hi : x == hi ? x : 0, sum = lane_prefix_sum(n);
      const uint64_t past = __ballot(sum > k);
      if (past) {
        const int l = __builtin_ctzll(past);
        who = base + l;
        tile = k - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(n, l));
        t = __builtin_amdgcn_readlane(x, l);
        return false;
      }
      k -= __builtin_amdgcn_readlane(sum, 63);
      return true;
    });
    job->b = __builtin_amdgcn_readfirstlane(who);
    job->tile = __builtin_amdgcn_readfirstlane(tile);
    t = __builtin_amdgcn_readfirstlane(t);
    if (causal) job->tile = queries ? hi - 1 : t - hi;  // the last queries meet the most keys, the first keys the most queries
    return true;
  }
};

// What packed_parts_kernel has to know of the jobs of a kind: how many tiles are in parts (each has two at least, of kMostParts), and of each its
// sequence, its number there, the number of its first part among the jobs, and its parts.
struct Cuts {
  int32_t tiles, unused[3];
  int4 tile[kMostParts / 2];
};
// The job of a workgroup; false if there is none.
template <int kHeld>
__device__ __forceinline__ bool find_job(const WaSeqLaunch& a, bool queries, int64_t rank, int cols, int share, Job* job) {
  const Jobs<kHeld> jobs(threadIdx.x & 63, cols, share, queries);
  Cuts* cuts = (Cuts*)a.cut_tiles + (queries ? 0 : 1);
  if (rank == 0) {
    const int n = jobs.longer(jobs.most) * cols;
    if (threadIdx.x == 0) cuts->tiles = n;
  }
  if (!jobs.find(rank, job)) return false;
  if (job->parts > 1 && job->part == 0 && threadIdx.x == 0) cuts->tile[job->number] = make_int4(job->b, job->tile, (int)rank, job->parts);
  return true;
}
// Up to 64 sequences have a path of their own (a step of 2,311 tokens in 5 documents: 55 us, 57 along the other; the gradient of 600 documents of
// 30 tokens, 8 heads of 64, takes 152 us so, and took 219, when the other took 160, where a path held 64).
__device__ __forceinline__ bool take_job(const WaSeqLaunch& a, bool queries, int64_t rank, int cols, int share, Job* job) {
  return a.batch <= 64 ? find_job<1>(a, queries, rank, cols, share, job) : find_job<8>(a, queries, rank, cols, share, job);
}

// Rows [row, row + ROWS) of g (`token` bytes apart) into a tile; rows past `last` are that row again.
template <int RB, int ROWS>
__device__ __forceinline__ void copy_rows(const unsigned char* tile, const unsigned char* g, uint32_t token, int row, int last, int w,
                                          int lane) {
  constexpr int RPI = 1024 / RB, LPR = RB / 16, N = ROWS * RB / 1024 / kWaves;
  static_assert(N * kWaves * 1024 == ROWS * RB, "a tile is whole copies of every wavefront");
  const unsigned char* from = g + (int64_t)row * token;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = (i * kWaves + w) * RPI + lane / LPR;
    dma16(from, min(r, last - row) * token + tile_chunk<RB>(r, lane % LPR) * 16, tile + (i * kWaves + w) * 1024);
  }
}

// dO . O of 8 columns, O with what its rounding left (dO . O of the rounded O alone gave dQ and dK an error of 0.0026 of their size where
// this gives 0.0024 and rounding them alone 0.0017)
__device__ __forceinline__ float dot8(bf16x8 a, bf16x8 o, uint32_t rest0, uint32_t rest1, float sum) {
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  const u16x8 bits = __builtin_bit_cast(u16x8, o);
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = __builtin_fmaf((float)a[i], with_rest(bits[i], i < 4 ? rest0 : rest1, i & 3), sum);
  return sum;
}

// rows[0]: scores from the log-sum-exp, so that P = exp2(c2 s); rows[1]: dP from -D. A wavefront 16 tokens of a head, D / 8 lanes a token.
template <int D>
__global__ __launch_bounds__(256) void packed_rows_kernel(const WaSeqLaunch a) {
  constexpr int L = D / 8, STEP = 64 / L;
  const int lane = threadIdx.x & 63, c = (lane & (L - 1)) * 8;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int h = (int)(id % a.heads), first = (int)(id / a.heads) * 16;
  const int begin = min(max(a.starts[0], 0), a.tokens), end = min(max(a.starts[a.batch], 0), a.tokens);
  const float c2 = a.scale * kLog2e;
  bf16x8 dof[16 / STEP], of[16 / STEP];
  float lse[16 / STEP];
  uint32_t rest[16 / STEP][2];
#pragma unroll
  for (int i = 0; i < 16 / STEP; ++i) {
    const int64_t tok = first + i * STEP + lane / L;
    const bool valid = tok >= begin && tok < end;
    dof[i] = load8((const uint16_t*)a.dout.at + tok * a.dout.token + h * a.dout.head + c, valid);
    of[i] = load8((const uint16_t*)a.o.at + tok * a.o.token + h * a.o.head + c, valid);
    const float* stat = a.lse_in + ((int64_t)h * a.tokens + tok) * a.lse_step;
    lse[i] = valid ? stat[0] : 0.f;
    rest[i][0] = valid ? *(const uint32_t*)(stat + 1 + c / 4) : 0;
    rest[i][1] = valid ? *(const uint32_t*)(stat + 2 + c / 4) : 0;
  }
#pragma unroll
  for (int i = 0; i < 16 / STEP; ++i) {
    const int64_t tok = first + i * STEP + lane / L;
    float d = dot8(dof[i], of[i], rest[i][0], rest[i][1], 0.f);
#pragma unroll
    for (int x = L / 2; x > 0; x >>= 1) d += __shfl_xor(d, x);
    if (c == 0 && tok >= begin && tok < end) {
      float* to = a.rows + (int64_t)h * a.tokens + tok;
      to[0] = -lse[i] * kLog2e / c2;
      to[(int64_t)a.heads * a.tokens] = -d;
    }
  }
}

// Job `rank` of queries. lds: 2 tiles of KB keys and values.
template <int D>
__device__ __forceinline__ void query_job(const WaSeqLaunch& a, int64_t rank, unsigned char* lds) {
  using C = Bwd<D>;
  constexpr int KB = C::KB, BYTES = KB * C::RB, STAGE = 2 * BYTES;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Job job;
  if (!take_job(a, true, rank, a.heads, 3, &job)) return;
  const int b = job.b, tile = job.tile, h = job.col, hk = h / (a.heads / a.kv_heads);
  const Seq s = one_seq(b);
  const int i0 = tile * kRows + w * 32, i = i0 + l32, i_last = s.n - 1;
  const bool valid = i <= i_last;
  // Keys that the lane's query sees; of one key alone dP = D, so dS is 0 and not what rounding leaves: none counts.
  const int sees = !valid ? 0 : a.causal ? i + 1 : s.n, limit = sees == 1 ? 0 : sees;
  const int some = i0 > i_last ? 0 : a.causal ? min(i0 + 32, s.n) : s.n, all = a.causal ? min(i0 + 1, s.n) : s.n;
  // this part's keys
  const int lo = job.length * job.part / job.parts * kRows, most = min(job.length * (job.part + 1) / job.parts * kRows, s.n);
  const unsigned char* kg = (const unsigned char*)a.k.at + (s.first * a.k.token + hk * a.k.head) * 2;
  const unsigned char* vg = (const unsigned char*)a.v.at + (s.first * a.v.token + hk * a.v.head) * 2;
  auto copy = [&](int key, int buf) {
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));  // the copies' offsets are not held across the loop
    const unsigned char* t = lds + buf * STAGE;
    copy_rows<C::RB, KB>(t, kg, (uint32_t)(a.k.token * 2), key, i_last, w, lane_o);
    copy_rows<C::RB, KB>(t + BYTES, vg, (uint32_t)(a.v.token * 2), key, i_last, w, lane_o);
  };
  copy(lo, 0);

  // the wavefront's queries and their dO
  bf16x8 qf[C::KS], dof[C::KS];
  const int64_t tok = s.first + i;
  const uint16_t* qg = (const uint16_t*)a.q.at + tok * a.q.token + h * a.q.head;
  const uint16_t* dog = (const uint16_t*)a.dout.at + tok * a.dout.token + h * a.dout.head;
#pragma unroll
  for (int x = 0; x < C::KS; ++x) {
    qf[x] = load8(qg + 16 * x + 8 * hf, valid);
    dof[x] = load8(dog + 16 * x + 8 * hf, valid);
  }
  const float c2 = a.scale * kLog2e;
  float ref = 0.f, d = 0.f;  // log-sum-exp in log2 units, D
  if (valid) {
    const float* from = a.rows + (int64_t)h * a.tokens + tok;
    ref = -from[0] * c2;
    d = -from[(int64_t)a.heads * a.tokens];
  }

  const uint32_t k_row = row_operand<C::RB>(lane, 0), v_row = BYTES + row_operand<C::RB>(lane, 0);
  const uint32_t k_col0 = col_operand<C::RB>(lane, 0, 0), k_col1 = col_operand<C::RB>(lane, 0, 1);
  f32x16 dq[C::DT];
#pragma unroll
  for (int c = 0; c < C::DT; ++c) fill(dq[c], 0.f);

  // 32 keys; masked: this lane's query sees only `rest` of them, counted from its first register's.
  auto work = [&](uint32_t t, bool masked, int rest) {
    uint32_t kr = k_row + t, vr = v_row + t, kc0 = k_col0 + t, kc1 = k_col1 + t;
    asm volatile("" : "+v"(kr), "+v"(vr), "+v"(kc0), "+v"(kc1));
    auto row = [&](int x) {  // operand of product x of the scores, then of dP
      return x < C::KS ? read_row(lds + row_step(kr, x)) : read_row(lds + row_step(vr, x - C::KS));
    };
    auto col = [&](int x) {  // operand of product x of dQ: 16 keys, 32 columns
      const int at = 16 * (x / C::DT) * C::RB;
      return read_cols(lds + col_step(kc0, x % C::DT) + at, lds + col_step(kc1, x % C::DT) + at);
    };
    f32x16 sc, dp;
    fill(sc, 0.f);
    fill(dp, 0.f);
    float p[16];
    bf16x8 ring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) ring[x] = row(x);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int x = 0; x < 2 * C::KS; ++x) {
      if (x < C::KS) sc = mfma(ring[x % kAhead], qf[x], sc); else dp = mfma(ring[x % kAhead], dof[x - C::KS], dp);
      if (x + kAhead < 2 * C::KS) ring[x % kAhead] = row(x + kAhead);
      if (x >= C::KS) {  // the exponentials run beside the products of dP
        constexpr int PER = 16 / C::KS;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int v = (x - C::KS) * PER + e;
          p[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[v], c2, -ref));
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    bf16x8 cring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) cring[x] = col(x);
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + (v & 3) >= rest) p[v] = 0.f;
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) p[v] *= dp[v] - d;
    const bf16x8 ds[2] = {pack8(p), pack8(p + 8)};
#pragma unroll
    for (int x = 0; x < 2 * C::DT; ++x) {
      dq[x % C::DT] = mfma(cring[x % kAhead], ds[x / C::DT], dq[x % C::DT]);
      if (x + kAhead < 2 * C::DT) cring[x % kAhead] = col(x + kAhead);
    }
  };
  int buf = 0;
  for (int key = lo; key < most; key += KB) {
    WA_WAIT_VM(0);
    WA_BARRIER();
    if (key + KB < most) copy(key + KB, buf ^ 1);
    int end = KB;  // opaque: a loop, so that the two halves do not share registers
    asm volatile("" : "+s"(end));
#pragma unroll 1
    for (int half = 0; half < end; half += 32) {
      if (key + half >= some) break;
      work(buf * STAGE + half * C::RB, key + half + 32 > all, limit - key - half - 4 * hf);
    }
    buf ^= 1;
  }
  if (job.parts > 1) {
    store_part(a.part + (rank * kRows + w * 32 + l32) * D, dq, a.scale, hf);
  } else {
    store_row16((uint16_t*)a.dq.at + tok * a.dq.token + h * a.dq.head, dq, a.scale, hf, valid);
  }
}

// Job `rank` of keys. lds: 2 tiles of QB queries and dO, and the values; stat: their rows of a.rows.
template <int D>
__device__ __forceinline__ void key_job(const WaSeqLaunch& a, int64_t rank, unsigned char* lds, float (*stat)[2 * Bwd<D>::QB]) {
  using C = Bwd<D>;
  constexpr int QB = C::QB, BYTES = QB * C::RB, STAGE = 2 * BYTES;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Job job;
  if (!take_job(a, false, rank, a.kv_heads, 4, &job)) return;
  const int b = job.b, tile = job.tile, hk = job.col, group = a.heads / a.kv_heads;
  const Seq s = one_seq(b);
  const int k0 = tile * kRows + w * 32, kj = k0 + l32;
  const bool valid = kj < s.n;
  const int from = !valid ? s.n : a.causal ? kj : 0;                      // first query that sees this lane's key,
  const int some = k0 >= s.n ? s.n : a.causal ? k0 : 0;                   // the wavefront's first
  const int all = a.causal ? min(k0 + 31, s.n - 1) : 0;                   // and its last
  const bool whole = k0 + 31 < s.n;
  const int lone = a.causal || s.n == 1 ? 0 : -1;                         // the query that sees one key, whose dS is 0; its tile is masked
  // this part's queries, in tiles of QB from the last on, of each tile all heads: so key tiles of different numbers, which begin with
  // different queries, meet the same ones at the same time, and the caches hold them
  const int lead = a.causal ? tile : 0, first = (lead + job.length * job.part / job.parts) * kRows;
  const int past = min((lead + job.length * (job.part + 1) / job.parts) * kRows, s.n);

  const int64_t tok = s.first + kj;
  const uint16_t* kg = (const uint16_t*)a.k.at + tok * a.k.token + hk * a.k.head;
  const uint16_t* vg = (const uint16_t*)a.v.at + tok * a.v.token + hk * a.v.head;
  bf16x8 kf[C::KS], vf[C::kValuesInLds ? 1 : C::KS];
#pragma unroll
  for (int x = 0; x < C::KS; ++x) kf[x] = load8(kg + 16 * x + 8 * hf, valid);
  if constexpr (C::kValuesInLds) {
    copy_rows<C::RB, kRows>(lds + 2 * STAGE, (const unsigned char*)a.v.at + (s.first * a.v.token + hk * a.v.head) * 2,
                            (uint32_t)(a.v.token * 2), tile * kRows, s.n - 1, w, lane);
  } else {
#pragma unroll
    for (int x = 0; x < C::KS; ++x) vf[x] = load8(vg + 16 * x + 8 * hf, valid);
  }

  const uint32_t q_row = row_operand<C::RB>(lane, 0), o_row = BYTES + row_operand<C::RB>(lane, 0);
  const uint32_t q_col0 = col_operand<C::RB>(lane, 0, 0), q_col1 = col_operand<C::RB>(lane, 0, 1);
  const uint32_t v_row = 2 * STAGE + w * 32 * C::RB + row_operand<C::RB>(lane, 0);
  const float c2 = a.scale * kLog2e;
  f32x16 dk[C::DT], dv[C::DT];
#pragma unroll
  for (int c = 0; c < C::DT; ++c) {
    fill(dk[c], 0.f);
    fill(dv[c], 0.f);
  }

  auto copy = [&](int g, int i, int buf) {
    int lane_o = lane;
    asm volatile("" : "+v"(lane_o));
    const int h = hk * group + g;
    const unsigned char* t = lds + buf * STAGE;
    copy_rows<C::RB, QB>(t, (const unsigned char*)a.q.at + (s.first * a.q.token + h * a.q.head) * 2, (uint32_t)(a.q.token * 2), i,
                         s.n - 1, w, lane_o);
    copy_rows<C::RB, QB>(t + BYTES, (const unsigned char*)a.dout.at + (s.first * a.dout.token + h * a.dout.head) * 2,
                         (uint32_t)(a.dout.token * 2), i, s.n - 1, w, lane_o);
    // 2 QB statistics: QB / 32 copies of 64
    if (w < QB / 32) {
      const int at = w * 64 + lane_o;  // row at / QB of query i + at % QB
      const float* rows = a.rows + (int64_t)(at / QB * a.heads + h) * a.tokens + s.first + min(i + at % QB, s.n - 1);
      dma4_at(rows, (const unsigned char*)(stat[buf] + w * 64));
    }
  };
  // 32 queries; q0: the query of this lane's first register
  auto work = [&](uint32_t t, const float* st, bool masked, int q0) {
    uint32_t qr = q_row + t, orow = o_row + t, qc0 = q_col0 + t, qc1 = q_col1 + t, vr = v_row;
    asm volatile("" : "+v"(qr), "+v"(orow), "+v"(qc0), "+v"(qc1), "+v"(vr));
    auto row = [&](int x) { return x < C::KS ? read_row(lds + row_step(qr, x)) : read_row(lds + row_step(orow, x - C::KS)); };
    auto value = [&](int y) { return read_row(lds + row_step(vr, y)); };
    auto col = [&](int x) {  // of the products of 16 queries: dV's column tiles (of dO), then dK's (of Q)
      const int y = x % (2 * C::DT), at = 16 * (x / (2 * C::DT)) * C::RB + (y < C::DT ? BYTES : 0);
      return read_cols(lds + col_step(qc0, y % C::DT) + at, lds + col_step(qc1, y % C::DT) + at);
    };
    f32x16 sc, dp;
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sc[4 * q4 + e] = st[8 * q4 + e];
        dp[4 * q4 + e] = st[QB + 8 * q4 + e];
      }
    float p[16], ds[16];
    bf16x8 ring[kAhead], vring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) ring[x] = row(x);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int x = 0; x < 2 * C::KS; ++x) {
      if (x < C::KS)
        sc = mfma(ring[x % kAhead], kf[x], sc);
      else
        dp = mfma(ring[x % kAhead], C::kValuesInLds ? vring[x % kAhead] : vf[C::kValuesInLds ? 0 : x - C::KS], dp);
      if (x + kAhead < 2 * C::KS) {
        ring[x % kAhead] = row(x + kAhead);
        if (C::kValuesInLds && x + kAhead >= C::KS) vring[x % kAhead] = value(x + kAhead - C::KS);
      }
      if (x >= C::KS) {
        constexpr int PER = 16 / C::KS;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int v = (x - C::KS) * PER + e;
          p[v] = __builtin_amdgcn_exp2f(sc[v] * c2);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    bf16x8 cring[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) cring[x] = col(x);
    if (masked) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int q = q0 + 8 * (v >> 2) + (v & 3);
        if (q < from || q >= s.n) p[v] = 0.f;
      }
      dp[0] *= q0 == lone ? 0.f : 1.f;
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) ds[v] = p[v] * dp[v];
    const bf16x8 pw[2] = {pack8(p), pack8(p + 8)}, dw[2] = {pack8(ds), pack8(ds + 8)};
#pragma unroll
    for (int x = 0; x < 4 * C::DT; ++x) {
      const int y = x % (2 * C::DT), c = y % C::DT;
      if (y < C::DT)
        dv[c] = mfma(cring[x % kAhead], pw[x / (2 * C::DT)], dv[c]);
      else
        dk[c] = mfma(cring[x % kAhead], dw[x / (2 * C::DT)], dk[c]);
      if (x + kAhead < 4 * C::DT) cring[x % kAhead] = col(x + kAhead);
    }
  };
  int g = 0, i = first + (past - first - 1) / QB * QB, buf = 0;
  copy(0, i, 0);
  while (i >= first) {
    const int i0 = i;
    if (++g == group) {
      g = 0;
      i -= QB;
    }
    WA_WAIT_VM(0);
    WA_BARRIER();
    if (i >= first) copy(g, i, buf ^ 1);
    int end = QB;
    asm volatile("" : "+s"(end));
#pragma unroll 1
    for (int half = 0; half < end; half += 32) {
      const int i1 = i0 + half;
      if (i1 + 32 <= some || i1 >= s.n) continue;
      work(buf * STAGE + half * C::RB, stat[buf] + half + 4 * hf, !whole || i1 < all || i1 + 32 > s.n, i1 + 4 * hf);
    }
    buf ^= 1;
  }
  if (job.parts > 1) {
    float* to = a.part + a.dq_part + (rank * kRows + w * 32 + l32) * 2 * D;
    store_part(to, dk, a.scale, hf);
    store_part(to + D, dv, 1.f, hf);
  } else {
    store_row16((uint16_t*)a.dk.at + tok * a.dk.token + hk * a.dk.head, dk, a.scale, hf, valid);
    store_row16((uint16_t*)a.dv.at + tok * a.dv.token + hk * a.dv.head, dv, 1.f, hf, valid);
  }
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 3 : 2) void packed_grad_kernel(const WaSeqLaunch a, int key_jobs) {
  using C = Bwd<D>;
  constexpr int KEYS = 4 * C::QB * C::RB + (C::kValuesInLds ? kRows * C::RB : 0), QUERIES = 4 * C::KB * C::RB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[KEYS > QUERIES ? KEYS : QUERIES];
  __shared__ __attribute__((aligned(1024))) float stat[2][2 * C::QB];
  if ((int)blockIdx.x < key_jobs)
    key_job<D>(a, blockIdx.x, lds, stat);
  else
    query_job<D>(a, blockIdx.x - key_jobs, lds);
}

// Adds the parts of cut tiles in order and rounds: four workgroups a tile, first those of dQ, then those of dK and dV.
template <int D>
__global__ __launch_bounds__(256) void packed_parts_kernel(const WaSeqLaunch a) {
  const bool keys = blockIdx.x >= 4 * kMostParts / 2;
  const int number = blockIdx.x / 4 % (kMostParts / 2);
  const Cuts* cuts = (const Cuts*)a.cut_tiles + (keys ? 1 : 0);
  const int4 cut = cuts->tile[number];
  if (number >= cuts->tiles) return;
  const int cols = keys ? a.kv_heads : a.heads, col = spread(cut.z % cols, cols), width = keys ? 2 * D : D;
  const Seq s = one_seq(__builtin_amdgcn_readfirstlane(cut.x));
  const int64_t step = (int64_t)cols * kRows * width;
  const float* from = a.part + (keys ? a.dq_part : 0) + (int64_t)cut.z * kRows * width;
  for (int x = threadIdx.x; x < kRows / 4 * width / 4; x += 256) {
    const int r = x / (width / 4) + blockIdx.x % 4 * (kRows / 4), c = x % (width / 4) * 4;
    if (cut.y * kRows + r >= s.n) break;
    const float* at = from + (int64_t)r * width + c;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int y = 0; y < cut.w; ++y) {
      const float4 z = *(const float4*)(at + y * step);
      sum.x += z.x;
      sum.y += z.y;
      sum.z += z.z;
      sum.w += z.w;
    }
    const int64_t tok = s.first + cut.y * kRows + r;
    const WaSeqRows& to = !keys ? a.dq : c < D ? a.dk : a.dv;
    *(uint2*)((uint16_t*)to.at + tok * to.token + col * to.head + c % D) = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
  }
}

// Tiles in parts are longer than a 512th of all, so that there are fewer than 1,024 parts (each of more than a half of that), of fewer
// than 512 tiles; and no more than the sequences' tiles have.
int64_t most_parts(const WaSeqLaunch& a, int cols) {
  return std::min<int64_t>(kMostParts, wa_packed_backward_tiles(a) * cols * (((int64_t)a.tokens + kRows - 1) / kRows));
}

template <int D>
hipError_t launch(const WaSeqLaunch& a, hipStream_t stream) {
  const int64_t tiles = wa_packed_backward_tiles(a);
  const int64_t row_waves = ((int64_t)a.tokens + 15) / 16 * a.heads;
  hipLaunchKernelGGL(packed_rows_kernel<D>, dim3((unsigned)((row_waves + 3) / 4)), dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // a job a tile, and for each part of a 512th of all one more at most; those of queries begin on the first XCD
  const int64_t key_jobs = (tiles * a.kv_heads + kSlots + 7) / 8 * 8, query_jobs = tiles * a.heads + kSlots;
  hipLaunchKernelGGL(packed_grad_kernel<D>, dim3((unsigned)(key_jobs + query_jobs)), dim3(64 * kWaves), 0, stream, a, (int)key_jobs);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(packed_parts_kernel<D>, dim3(4 * kMostParts), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// Sequences of n_b tokens have sum ceil(n_b / 128) tiles.
int64_t wa_packed_backward_tiles(const WaSeqLaunch& a) {
  return std::min<int64_t>(a.tokens, ((int64_t)a.tokens + (int64_t)(kRows - 1) * a.batch) / kRows);
}

size_t wa_packed_backward_cut_bytes() { return 2 * sizeof(Cuts); }
int64_t wa_packed_backward_dq_floats(const WaSeqLaunch& a) { return most_parts(a, a.heads) * kRows * a.head_dim; }
int64_t wa_packed_backward_part_floats(const WaSeqLaunch& a) {
  return wa_packed_backward_dq_floats(a) + most_parts(a, a.kv_heads) * kRows * 2 * a.head_dim;
}

hipError_t wa_launch_packed_backward(const WaSeqLaunch& a, hipStream_t stream) {
  return a.head_dim == 64 ? launch<64>(a, stream) : launch<128>(a, stream);
}
