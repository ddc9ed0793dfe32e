// Verification of drafted tokens against the target's logits (speculative sampling) from given random numbers.
//
//   p, q: softmax of scale * target's and draft's logits.  Draft i of a sequence is accepted while u_i q_i(d_i) < p_i(d_i).  At the first place that is not,
//   the next token is drawn from max(0, p - q), behind the last draft from p.  Drawn by a race: the token with the largest weight / e_j, where the e_j are
//   exponential random numbers, is token j with a probability in proportion to its weight.
#include "any_rows.cuh"

namespace iris {
namespace rows {

constexpr int kVerifyThreads = 256, kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifySplit = 16;     // blocks (one cluster) that share a row
constexpr int kMaxDrafts = 128;

// What is known of a place of a sequence: largest logit and sum exp(scale (z - largest)) of the target's row and the draft's, both logits of the
// drafted token; greedy: the column of the target's largest logit.
struct Seat {
  float m, s, mq, sq, z, zq;
  int best, pad;
};

struct VerifyParams {
  const void *logits, *draft_logits;   // draft_logits: nullptr if drafted tokens were certain
  int64_t stride, draft_stride;
  int sequences, drafts, vocab, split, each, draft_each;
  float scale;
  const float* scales;
  const int64_t* ids;
  const float *uniform, *noise;
  int64_t *tokens, *accepted;
  float* logprob;
  Seat* seats;   // [sequences, drafts + 1]
};

__device__ __forceinline__ float scale_of(const VerifyParams& p, int b) {
  const float s = p.scales ? p.scales[b] : p.scale;
  return s > 0.f ? s : NAN;
}
__device__ __forceinline__ bool is_greedy(float scale) { return scale > kMaxScale; }

// The block's share of a row: largest logit and sum; the next batch is under way while one is summed.
constexpr int kBatch = 4;   // granules of a thread
template <int DT>
__device__ __forceinline__ void fetch_first(const Row<DT>& row, const Part<DT>& part, uint4 (&g)[kBatch]) {
  if (kBatch * kVerifyThreads <= part.n_int)
#pragma unroll
    for (int u = 0; u < kBatch; ++u) g[u] = ld_once(row.at(part.w0 + u * kVerifyThreads + threadIdx.x));
}
// g: of fetch_first.
template <int DT>
__device__ __forceinline__ Acc sum_part(const Row<DT>& row, const Part<DT>& part, float k, float4* upper, uint4 (&g)[kBatch]) {
  constexpr int T = kVerifyThreads, U = kBatch, B = T * U;
  const int tid = threadIdx.x, n = part.n_all;
  Sums<DT, false, true> sums(k, upper + tid);
  const uint4* const from = reinterpret_cast<const uint4*>(row.at(part.w0)) + tid;
  uint4 h[U];
  const auto fetch = [&](int at, uint4(&to)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) to[u] = ld_once(from + at + u * T);
  };
  int b = 0;
  for (; b + 3 * B <= part.n_int; b += 2 * B) {
    fetch(b + B, h);
    sums.template add<true>(g, largest<DT, true>(g, 0, T));
    fetch(b + 2 * B, g);
    sums.template add<true>(h, largest<DT, true>(h, 0, T));
    sums.template pace<T, U>(b);
  }
  if (b + 2 * B <= part.n_int) {
    fetch(b + B, h);
    sums.template add<true>(g, largest<DT, true>(g, 0, T));
    sums.template add<true>(h, largest<DT, true>(h, 0, T));
    b += 2 * B;
  } else if (b + B <= part.n_int) {
    sums.template add<true>(g, largest<DT, true>(g, 0, T));
    b += B;
  }
  for (; b < n; b += B) {
    const int left = n - b - tid;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * T < left) g[u] = part.raw(row, b + u * T + tid);
    sums.template add<false>(g, largest<DT, false>(g, left, T), left, T);
  }
  return sums.done();
}
__device__ __forceinline__ uint64_t larger_key(uint64_t a, uint64_t b) { return a > b ? a : b; }

// The block's share of a row: the key of its largest logit, 0 where none is left.  A thread remembers its largest logit and the first of its batches that
// has it, and looks at that again in the end.  (What the row covers of granules in part comes last, and has keys of its own.)
template <int DT>
__device__ __forceinline__ uint64_t best_part(const Row<DT>& row, const Part<DT>& part, uint64_t (&of_warp)[kVerifyWarps], uint4 (&g)[kBatch]) {
  constexpr int T = kVerifyThreads, U = kBatch, B = T * U, VE = Elem<DT>::VE;
  const int tid = threadIdx.x, n = part.n_int;
  uint64_t key = 0;
  float best = -INFINITY;
  int at = -1;
  const uint4* const from = reinterpret_cast<const uint4*>(row.at(part.w0)) + tid;
  const auto keys_of = [&](const uint4& g, int granule) {
    float y[VE];
    Elem<DT>::unpack(g, y);
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (y[e] != -INFINITY) key = larger_key(key, order_key<DT>(y[e], granule * VE + e - row.ph));
  };
  uint4 h[U];
  const auto fetch = [&](int b, uint4(&to)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) to[u] = ld_once(from + b + u * T);
  };
  const auto look = [&](int b, const uint4(&x)[U]) {
    const float mx = largest<DT, true>(x, 0, T);
    if (mx > best || mx != mx) {   // NaN comes before all
      best = mx;
      at = b;
    }
  };
  int b = 0;
  for (; b + 2 * B <= n; b += 2 * B) {
    fetch(b + B, h);
    look(b, g);
    if (b + 3 * B <= n) fetch(b + 2 * B, g);
    look(b + B, h);
  }
  if (b + B <= n) {
    look(b, g);
    b += B;
  }
  for (int i = b + tid; i < part.n_all; i += T) keys_of(part.raw(row, i), part.granule(i));
  if (at >= 0)
#pragma unroll
    for (int u = 0; u < U; ++u) keys_of(from[at + u * T], part.w0 + at + u * T + tid);
#pragma unroll
  for (int o = 16; o; o >>= 1) key = larger_key(key, __shfl_xor_sync(~0u, key, o));
  if ((tid & 31) == 0) of_warp[tid >> 5] = key;
  __syncthreads();
  key = of_warp[tid & (kVerifyWarps - 1)];
#pragma unroll
  for (int o = kVerifyWarps / 2; o; o >>= 1) key = larger_key(key, __shfl_xor_sync(~0u, key, o));
  return key;
}

// One cluster of `split` blocks a row, the target's first: what the drawing needs of it.
//
// Bound by memory where there are many rows (64 sequences of 4 drafts over 128000 tokens, a quarter greedy: 29 us for 134 MB, 4.6 TB/s; 3584 rows of 16384: 29 us, six waves
// of blocks of 5 us).  Rows behind a draft that is refused need not be read, but to know that in time takes longer than to read them: places one
// after the other, in clusters that leave out what follows, took 53 us.
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads, 4) verify_rows_kernel(const __grid_constant__ VerifyParams p) {
  using E = Elem<DT>;
  __shared__ Warps<kVerifyWarps> buf;
  __shared__ Warps<kVerifySplit> parts;   // of the cluster's blocks, in the first one
  __shared__ uint64_t keys[kVerifySplit], of_warp[kVerifyWarps];
  __shared__ float4 upper[kVerifyThreads];
  const int split = p.split, rank = split > 1 ? (int)ptx::cluster_ctarank() : 0, tid = threadIdx.x;
  const int unit = blockIdx.x / split, targets = p.sequences * (p.drafts + 1);
  const bool draft = unit >= targets;
  const int each = p.drafts + !draft, in = draft ? unit - targets : unit, b = in / each, i = in - b * each;   // place i of sequence b
  if (tid < kVerifySplit) {
    parts.of[tid] = Acc{};
    keys[tid] = 0;
  }
  if (split > 1) ptx::cluster_arrive_release();   // behind the wait the others may write to the first block
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const Row<DT> row(draft ? p.draft_logits : p.logits, in, draft ? p.draft_stride : p.stride, p.vocab);
  const Part<DT> part(row, rank, draft ? p.draft_each : p.each);
  uint4 g[kBatch];
  fetch_first(row, part, g);   // under way while it turns out whether the row is needed
  const int64_t* const ids = p.ids + (int64_t)b * p.drafts;
  const float scale = scale_of(p, b), k = scale * kLog2e;
  const int64_t id = i < p.drafts ? ids[i] : -1;
  const bool there = id >= 0 && id < p.vocab;
  bool absent = draft && (!there || is_greedy(scale));   // or a draft before this place is: the row is not needed
  for (int j = tid; j < i; j += kVerifyThreads) absent |= ids[j] < 0 || ids[j] >= p.vocab;
  if (split > 1) ptx::cluster_wait();
  if (__syncthreads_or(absent)) return;   // all blocks of the cluster
  Seat* const seat = p.seats + (int64_t)b * (p.drafts + 1) + i;
  if (is_greedy(scale)) {
    uint64_t key = best_part<DT>(row, part, of_warp, g);
    if (split > 1) {
      if (tid == 0) ptx::st_shared_cluster_u64(ptx::mapa(ptx::smem_u32(&keys[rank]), 0), key);
      ptx::cluster_sync();
      key = 0;
      for (int s = 0; s < split; ++s) key = larger_key(key, keys[s]);
    }
    if (rank == 0 && tid == 0) seat->best = key && fabsf(key_value<DT>(key)) < INFINITY ? key_column(key) : -1;
    return;
  }
  const float z = rank == 0 && tid == 0 && there ? E::to(row.column((int)id)) : 0.f;
  Acc a = sum_part<DT>(row, part, k, upper, g);
  warp_share<false>(a, k, buf);
  __syncthreads();
  a = warps_join<false>(k, buf);
  if (split > 1) {
    if (tid == 0) {
      const uint32_t to = ptx::mapa(ptx::smem_u32(&parts.of[rank]), 0);
      ptx::st_shared_cluster_u32(to, __float_as_uint(a.m));
      ptx::st_shared_cluster_u32(to + 4, __float_as_uint(a.s));
    }
    ptx::cluster_sync();
    if (rank) return;
    a = warps_join<false>(k, parts);
  }
  if (tid == 0) {
    (draft ? seat->mq : seat->m) = a.m;
    (draft ? seat->sq : seat->s) = a.s;
    (draft ? seat->zq : seat->z) = z;
  }
}

__device__ __forceinline__ double prob(float z, float m, float s, float scale) {   // NaN in a row without a distribution, for masked tokens too
  return s != s ? (double)s : z == -INFINITY ? 0. : exp(((double)z - (double)m) * (double)scale) / (double)s;
}
// Whether a draft is accepted: in 32 bits, and in 64 where that is too near to tell (or NaN).
__device__ __forceinline__ bool accepts(const Seat& s, float u, bool with_q, float scale) {
  const float k = scale * kLog2e;
  const float pd = ex2((s.z - s.m) * k) / s.s, qd = with_q ? ex2((s.zq - s.mq) * k) / s.sq : 1.f, t = u * qd;
  if (fabsf(t - pd) > 1e-4f * fmaxf(t, pd) && fmaxf(t, pd) > 1e-30f) return t < pd;
  return (double)u * (with_q ? prob(s.zq, s.mq, s.sq, scale) : 1.) < prob(s.z, s.m, s.s, scale);
}
__device__ __forceinline__ float log_prob64(float z, const Seat& s, float scale) {   // rounded once but for the logarithm
  return (float)(((double)z - (double)s.m) * (double)scale - (double)logf(s.s));
}

__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// p - q counts as nothing up to so much of p.  The rows' sums are of 32 bits.  A term's exponent is rounded twice and up to 24 + 17 large on average (the slack
// of the reference that it is counted from, and what a row of 128000 columns has): 41 ln 2 2^-23; counting it from another reference 24 ln 2 2^-23; the
// exponential 2^-22; chains of at most 128 equal terms that round to one side 2^-20: together below 2^-17.  So two rows that are the same but lie unlike
// in 16 bytes, and are summed in other orders, leave less than 2^-16 of p.
constexpr float kNothing = 1.f / (1 << 16);
// How far, relative to p, a weight may be off in 32 bits: an exponent is at most 126 (below that the exponential is 0) and rounded four times (difference,
// scale's logarithm twice, product), 126 ln 2 2^-22 < 2^-15 of p with the exponential's and the sum's own 2^-22, and the same again for q <= p.
constexpr float kOff = 1.f / (1 << 14);
struct Runner {   // of the race: a column (-1: none) and between which bounds its score lies
  float low, high;
  int column;
};
// The winner's column among n runners, which all threads of the warp get: n <= 32, thread i has runner i.  Those that may be the best by their bounds are
// compared in 64 bits (`exactly`: the score of a column); the lowest column among equal ones; -1: none.
template <class F>
__device__ __forceinline__ int winner(Runner r, F exactly) {
  const float least = warp_max(r.column >= 0 ? r.low : 0.f);
  const uint32_t near = __ballot_sync(~0u, r.column >= 0 && r.high >= least);
  if (!near) return -1;
  double score = 0.;
  if (near & (near - 1)) score = near >> (threadIdx.x & 31) & 1 ? exactly(r.column) : 0.;
  int at = __ffs(near) - 1;
  for (uint32_t rest = near & (near - 1); rest; rest &= rest - 1) {
    const int i = __ffs(rest) - 1;
    const double a = __shfl_sync(~0u, score, at), b = __shfl_sync(~0u, score, i);
    const int ca = __shfl_sync(~0u, r.column, at), cb = __shfl_sync(~0u, r.column, i);
    if (b > a || (b == a && cb < ca)) at = i;
  }
  return __shfl_sync(~0u, r.column, at);
}

// One cluster of `split` blocks a sequence: accepts drafts up to the first that is refused, and draws the token behind them.
//
// 64 sequences over 128000: 19 us, of which the two rows and the noise (64 MB) account for 10; the rest is the chain of what has to be known first
// (statistics, where the sequence stops) and last (best of threads, of blocks, its column).  One sequence: 5 us of 11.  With the winners' columns kept in the pass
// instead of looked for in the end 29 us; their scores all in 64 bits, and two granules a thread at a time in half as many blocks, 47.  Where nothing is left
// of p - q all columns are compared in 64 bits before the second race: all 64 sequences of that kind 141 us a call instead of 43.
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads, 4) verify_draw_kernel(const __grid_constant__ VerifyParams p) {
  using E = Elem<DT>;
  constexpr int T = kVerifyThreads, VE = E::VE, ES = sizeof(typename E::T);
  __shared__ Runner block_best, parts[2][kVerifySplit];   // parts: of the cluster's blocks, of the first and the second race
  __shared__ float of_warp[kVerifyWarps];
  __shared__ unsigned long long exact_best;
  __shared__ int lowest, bound, runners;
  static_assert(kVerifySplit <= 32, "one a thread");
  __shared__ int stop_at;
  const int split = p.split, rank = split > 1 ? (int)ptx::cluster_ctarank() : 0, tid = threadIdx.x, lane = tid & 31;
  const int b = blockIdx.x / split, n = p.drafts;
  ptx::let_next_begin();
  if (split > 1) ptx::cluster_arrive_release();   // behind the wait the others may write to this block
  ptx::begin_after_previous();
  const float scale = scale_of(p, b);
  const bool greedy = is_greedy(scale);
  const int64_t* const ids = p.ids + (int64_t)b * n;
  const Seat* const seats = p.seats + (int64_t)b * (n + 1);
  if (tid < 32) {
    int stop = 0;
    for (;; stop += 32) {
      const int i = stop + lane;
      bool ok = i < n && ids[i] >= 0 && ids[i] < p.vocab;
      if (ok) ok = greedy ? seats[i].best == (int)ids[i] : accepts(seats[i], p.uniform[(int64_t)b * n + i], p.draft_logits != nullptr, scale);
      const uint32_t no = __ballot_sync(~0u, !ok);
      if (no) {
        stop += __ffs(no) - 1;
        break;
      }
    }
    if (lane == 0) stop_at = stop;
  }
  if (split > 1) ptx::cluster_wait();
  __syncthreads();
  const int stop = stop_at;
  const Seat seat = seats[stop];
  const bool refused = stop < n && ids[stop] >= 0 && ids[stop] < p.vocab;
  const int64_t r = (int64_t)b * (n + 1) + stop;
  const Row<DT> row(p.logits, r, p.stride, p.vocab);
  int next = seat.best;
  if (!greedy) {
    const Part<DT> part(row, rank, p.each);
    const float k = scale * kLog2e;
    const char* const noise = reinterpret_cast<const char*>(p.noise + (int64_t)b * p.vocab);
    for (int race = refused ? 0 : 1; race < 2; ++race) {
      const bool rest = race == 0, with_q = rest && p.draft_logits && seat.sq != 0.f;
      const int without = rest && !p.draft_logits ? (int)ids[stop] : -1;
      const Row<DT> draft_row(p.draft_logits, with_q ? (int64_t)b * n + stop : 0, p.draft_stride, p.vocab);
      const char* const draft = reinterpret_cast<const char*>(draft_row.granule0 + draft_row.ph);
      const float rs = (1.f + kOff) / seat.s, rsq = with_q ? 1.f / seat.sq : 0.f, mq = with_q ? seat.mq : 0.f;
      const uint32_t aq = phase(draft - (int64_t)row.ph * ES), ae = phase(noise - (int64_t)row.ph * 4);   // of every granule
      // The most that the scores of granule v may be, max(0, weight) / noise with p taken kOff too large, and the least: 0 where the weight may be nothing.
      const auto scores = [&](int v, float (&x)[VE], float (&low)[VE]) {
        const int c = v * VE - row.ph;
        uint4 zr[1], yr[1], e[VE / 4];
        if (c >= VE && c + 2 * VE <= p.vocab) {
          uint4 yn[1], en[VE / 4];
          zr[0] = ld_once(row.at(v));
          if (with_q) {
            const char* const from = draft + (int64_t)c * ES - aq;
            yr[0] = ld_global_v4(from);
            if (aq) yn[0] = ld_global_v4(from + 16);
          }
          const char* const from = noise + (int64_t)c * 4 - ae;
#pragma unroll
          for (int h = 0; h < VE / 4; ++h) e[h] = ld_global_v4(from + h * 16);
          if (ae) {
            en[VE / 4 - 1] = ld_global_v4(from + VE * 4);
#pragma unroll
            for (int h = 0; h + 1 < VE / 4; ++h) en[h] = e[h + 1];
            cut_all(e, en, ae);
          }
          if (with_q && aq) cut_all(yr, yn, aq);
        } else {   // what the columns' 16 bytes touch may leave the rows
          zr[0] = row.raw(v);
          if (with_q) yr[0] = load_piece<ES>(draft + (int64_t)c * ES, draft, draft + (int64_t)p.vocab * ES);
#pragma unroll
          for (int h = 0; h < VE / 4; ++h) e[h] = load_piece<4>(noise + ((int64_t)c + 4 * h) * 4, noise, noise + (int64_t)p.vocab * 4);
        }
        float z[VE], y[VE], f[VE];
        E::unpack(zr[0], z);
#pragma unroll
        for (int h = 0; h < VE / 4; ++h) {
          f[4 * h] = __uint_as_float(e[h].x), f[4 * h + 1] = __uint_as_float(e[h].y), f[4 * h + 2] = __uint_as_float(e[h].z), f[4 * h + 3] = __uint_as_float(e[h].w);
        }
#pragma unroll
        for (int u = 0; u < VE; ++u) {
          x[u] = ex2((z[u] - seat.m) * k) * rs;
          low[u] = x[u] * -(2.f * kOff + kNothing);
        }
        if (with_q) {
          E::unpack(yr[0], y);
#pragma unroll
          for (int u = 0; u < VE; ++u) x[u] = fmaf(ex2((y[u] - mq) * k), -rsq, x[u]);
        }
        if ((uint32_t)(without - c) < (uint32_t)VE) {
#pragma unroll
          for (int u = 0; u < VE; ++u) x[u] = c + u == without ? 0.f : x[u];
        }
#pragma unroll
        for (int u = 0; u < VE; ++u) {
          const float by = reciprocal(f[u]);
          low[u] = fmaxf(x[u] + low[u], 0.f) * by;
          x[u] = fmaxf(x[u], 0.f) * by;
        }
      };
      // The thread's best score, the first of its granules that has it, and the best of the others (NaN is no score).
      float score = 0.f, second = 0.f;
      int at = -1;
      for (int v = part.v0 + tid; v < part.v1; v += T) {
        float x[VE], low[VE], m = 0.f;
        scores(v, x, low);
#pragma unroll
        for (int u = 0; u < VE; ++u) m = fmaxf(m, x[u]);
        second = fmaxf(second, fminf(m, score));
        if (m > score) {
          score = m;
          at = v;
        }
      }
      const auto exactly = [&](int c) {
        double w = prob(E::to(row.column(c)), seat.m, seat.s, scale);
        if (with_q) {
          const double left = w - prob(E::to(draft_row.column(c)), seat.mq, seat.sq, scale);
          w = left > w * kNothing ? left : 0.;
        }
        return w > 0. ? w / (double)p.noise[(int64_t)b * p.vocab + c] : 0.;
      };
      // The block's: all columns that may be the best are at least as good, at most, as the best thread's is at least.  If there are several (or that is 0,
      // and it may be nothing), their 64-bit scores decide, and the lowest column of equal ones.
      const float of_this = warp_max(score);
      if (lane == 0) of_warp[tid >> 5] = of_this;
      if (tid == 0) {
        block_best = Runner{0.f, 0.f, -1};
        exact_best = 0;
        lowest = INT32_MAX;
        bound = runners = 0;
      }
      __syncthreads();
      const float top = warp_max(of_warp[lane & (kVerifyWarps - 1)]);
      // Threads that are not far behind look at their granule again for the bound, all together, and count their columns that reach their own.  Then, if
      // several threads or columns are near (or one that was far), each compares its own in 64 bits, in all of its granules if others may be near too.
      Runner mine{0.f, 0.f, -1};
      double exact = 0.;
      float least = 0.f;
      bool looks = at >= 0 && score >= top * 0.5f, all = false, several = false;
#pragma unroll 1
      for (int look = 0; look < 2; ++look) {
        int n_mine = looks ? 0 : 2;
        if (looks)
#pragma unroll 1
          for (int v = all ? part.v0 + tid : at; v < part.v1; v += T) {
            float x[VE], low[VE], m = 0.f;
            scores(v, x, low);
#pragma unroll
            for (int u = 0; u < VE; ++u) m = fmaxf(m, low[u]);
            if (look == 0) {
              least = m;
              atomicMax(&bound, __float_as_int(m));
            }
            uint32_t rest = 0;
#pragma unroll
            for (int u = VE - 1; u >= 0; --u)
              if (x[u] >= least && x[u] > 0.f) {
                rest |= 1u << u;
                if (look == 0) mine = Runner{low[u], x[u], v * VE - row.ph + u};
              }
            n_mine += __popc(rest);
            if (look)
#pragma unroll 1
              for (; rest; rest &= rest - 1) {
                const int c = v * VE - row.ph + __ffs(rest) - 1;
                const double e = exactly(c);
                if (e > exact) {
                  exact = e;
                  mine = Runner{__double2float_rd(e), __double2float_ru(e), c};
                }
              }
            if (!all) break;
          }
        if (look) break;
        __syncthreads();
        least = __int_as_float(bound);
        looks = at >= 0 && score >= least;   // from here on: is near
        all = second >= least;
        if (looks) atomicAdd(&runners, all ? 2 : n_mine);
        __syncthreads();
        several = runners > 1;
        if (!looks || several) mine.column = -1;
        if (!several) break;
      }
      if (several) {
        if (mine.column >= 0) atomicMax(&exact_best, (unsigned long long)__double_as_longlong(exact));   // of positive numbers the larger has the larger bits
        __syncthreads();
        if (mine.column >= 0 && (unsigned long long)__double_as_longlong(exact) == exact_best) atomicMin(&lowest, mine.column);
        __syncthreads();
        if (mine.column == lowest) block_best = mine;
      } else if (mine.column >= 0) {
        block_best = mine;
      }
      __syncthreads();
      const Runner best = block_best;
      next = best.column;
      if (split > 1) {
        if (tid < split) {
          const uint32_t to = ptx::mapa(ptx::smem_u32(&parts[race][rank]), tid);
          ptx::st_shared_cluster_u32(to, __float_as_uint(best.low));
          ptx::st_shared_cluster_u32(to + 4, __float_as_uint(best.high));
          ptx::st_shared_cluster_u32(to + 8, (uint32_t)best.column);
        }
        ptx::cluster_sync();
        next = winner(lane < split ? parts[race][lane] : Runner{0.f, 0.f, -1}, exactly);
      }
      if (next >= 0) break;   // all blocks of the cluster
      __syncthreads();
    }
  }
  if (rank) return;
  for (int i = tid; i <= n; i += T) {
    const int64_t token = i < stop ? ids[i] : i == stop ? (int64_t)next : -1;
    p.tokens[(int64_t)b * (n + 1) + i] = token;
    if (p.logprob) {
      const Seat s = i < stop ? seats[i] : seat;
      p.logprob[(int64_t)b * (n + 1) + i] = token < 0 || greedy ? 0.f : log_prob64(i < stop ? s.z : E::to(row.column(next)), s, scale);
    }
  }
  if (tid == 0) p.accepted[b] = stop;
}

template <int DT>
static int launch_verify(VerifyParams p, const iris_verify_args* a, cudaStream_t st) {
  IRIS_CHECK(allow_shared<verify_rows_kernel<DT>>(0, true));
  IRIS_CHECK(allow_shared<verify_draw_kernel<DT>>(0, true));
  const int64_t granules = part_granules(a->logits, p.stride, p.vocab, a->dtype, 1);
  const auto share = [&](int64_t rows, int least) {   // a row is shared while rows alone leave SMs without work and a block has at least so many granules
    int split = 1;
    while (split < kVerifySplit && rows * split * 2 <= kSms * 4 && granules > (int64_t)split * least) split *= 2;
    p.split = split;
    p.each = part_granules(a->logits, p.stride, p.vocab, a->dtype, split);
    p.draft_each = p.draft_logits ? part_granules(a->draft_logits, p.draft_stride, p.vocab, a->dtype, split) : 0;
  };
  const int64_t rows = (int64_t)p.sequences * (p.drafts + 1 + (p.draft_logits ? p.drafts : 0));
  share(rows, 512);
  IRIS_CHECK(launch_rows(verify_rows_kernel<DT>, p, (unsigned)(rows * p.split), p.split, kVerifyThreads, 0, st));
  share(p.sequences, 256);
  return launch_rows(verify_draw_kernel<DT>, p, (unsigned)(p.sequences * p.split), p.split, kVerifyThreads, 0, st);
}

}  // namespace rows
}  // namespace iris

using namespace iris;
using namespace iris::rows;

extern "C" size_t iris_verify_workspace_bytes(int64_t sequences, int drafts) {
  if (sequences <= 0 || drafts < 0 || drafts > kMaxDrafts || sequences > INT32_MAX / (kMaxDrafts + 1)) return 0;
  return (size_t)sequences * (drafts + 1) * sizeof(Seat);
}

extern "C" int iris_verify_drafts(const iris_verify_args* a, void* stream) {
  const char* fn = "iris_verify_drafts";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  if (a->drafts < 0 || a->drafts > kMaxDrafts) return fail(IRIS_ERR_ARG, "%s: drafts=%d not in [0, %d]", fn, a->drafts, kMaxDrafts);
  if (a->sequences < 0) return fail(IRIS_ERR_ARG, "%s: sequences=%lld", fn, (long long)a->sequences);
  if (a->sequences > INT32_MAX / (2 * kMaxDrafts + 1) / kVerifySplit) return fail(IRIS_ERR_UNSUPPORTED, "%s: too many sequences", fn);
  int64_t stride = a->row_stride, dstride = a->draft_stride;
  const int64_t rows = a->sequences * (a->drafts + 1);
  IRIS_CHECK(check_logits(fn, "logits", a->logits, a->dtype, rows, a->vocab, &stride));
  if (a->vocab < 1) return fail(IRIS_ERR_ARG, "%s: vocab=%lld", fn, (long long)a->vocab);
  const bool draft = a->draft_logits && a->drafts > 0;
  if (draft) IRIS_CHECK(check_logits(fn, "draft_logits", a->draft_logits, a->dtype, a->sequences * a->drafts, a->vocab, &dstride));
  if (!(a->scale > 0.f)) return fail(IRIS_ERR_ARG, "%s: scale has to be positive", fn);
  if (a->sequences == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "scales", a->scales, 4, false));
  IRIS_CHECK(check_aligned(fn, "draft_ids", a->draft_ids, 8, a->drafts > 0));
  const bool greedy = !a->scales && a->scale > kMaxScale;   // no random numbers needed
  IRIS_CHECK(check_aligned(fn, "uniform", a->uniform, 4, a->drafts > 0 && !greedy));
  IRIS_CHECK(check_aligned(fn, "noise", a->noise, 4, !greedy));
  IRIS_CHECK(check_aligned(fn, "tokens", a->tokens, 8, true));
  IRIS_CHECK(check_aligned(fn, "accepted", a->accepted, 8, true));
  IRIS_CHECK(check_aligned(fn, "logprob", a->logprob, 4, false));
  IRIS_CHECK(check_aligned(fn, "workspace", a->workspace, 16, true));
  const size_t need = iris_verify_workspace_bytes(a->sequences, a->drafts);
  if (a->workspace_bytes < need) return fail(IRIS_ERR_ARG, "%s: workspace has %zu bytes, the call needs %zu", fn, a->workspace_bytes, need);
  VerifyParams p{};
  p.logits = a->logits;
  p.draft_logits = draft && !greedy ? a->draft_logits : nullptr;   // greedy drafts are compared with the target's largest logit only
  p.stride = stride;
  p.draft_stride = dstride;
  p.sequences = (int)a->sequences;
  p.drafts = a->drafts;
  p.vocab = (int)a->vocab;
  p.scale = a->scale;
  p.scales = a->scales;
  p.ids = a->draft_ids;
  p.uniform = a->uniform;
  p.noise = a->noise;
  p.tokens = a->tokens;
  p.accepted = a->accepted;
  p.logprob = a->logprob;
  p.seats = static_cast<Seat*>(a->workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) return launch_verify<IRIS_BF16>(p, a, st);
  if (a->dtype == IRIS_F16) return launch_verify<IRIS_F16>(p, a, st);
  return launch_verify<IRIS_F32>(p, a, st);
}
