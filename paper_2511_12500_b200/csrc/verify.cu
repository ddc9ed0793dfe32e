// Verification of drafted tokens against the target's logits (speculative sampling) from given random numbers.
//
//   p, q: softmax of scale * target's and draft's logits.  Draft i of a sequence is accepted while u_i q_i(d_i) < p_i(d_i).  At the first place that is not,
//   the next token is drawn from max(0, p - q), behind the last draft from p.  Drawn by a race: the token with the largest weight / e_j, where the e_j are
//   exponential random numbers, is token j with a probability in proportion to its weight.
#include "any_rows.cuh"

namespace iris {
namespace rows {

constexpr int kVerifyThreads = 256, kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifySplit = 8;      // blocks (one cluster) that share a row
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

// The block's share of a row: largest logit and sum.
template <int DT>
__device__ __forceinline__ Acc sum_part(const Row<DT>& row, const Part<DT>& part, float k, float4* upper, Warps<kVerifyWarps>& buf) {
  constexpr int T = kVerifyThreads, U = 4;
  const int tid = threadIdx.x, n = part.n_all;
  Sums<DT, false, true> sums(k, upper + tid);
  batches<T, U>(part.n_int, [&](int b, auto all) {
    if constexpr (decltype(all)::value) {
      uint4 g[U];
#pragma unroll
      for (int u = 0; u < U; ++u) g[u] = ld_once(row.at(part.w0 + b + u * T + tid));
      sums.template pace<T, U>(b);
      sums.template add<true>(g, largest<DT, true>(g, 0, T));
    }
  });
  for (int b = part.n_int / (T * U) * (T * U); b < n; b += T * U) {
    const int left = n - b - tid;
    uint4 g[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * T < left) g[u] = part.raw(row, b + u * T + tid);
    sums.template pace<T, U>(b);
    sums.template add<false>(g, largest<DT, false>(g, left, T), left, T);
  }
  warp_share<false>(sums.done(), k, buf);
  __syncthreads();
  const Acc a = warps_join<false>(k, buf);
  __syncthreads();
  return a;
}

__device__ __forceinline__ uint64_t larger_key(uint64_t a, uint64_t b) { return a > b ? a : b; }

// The block's share of a row: the key of its largest logit, 0 where none is left.
template <int DT>
__device__ __forceinline__ uint64_t best_part(const Row<DT>& row, const Part<DT>& part, uint64_t (&of_warp)[kVerifyWarps]) {
  constexpr int T = kVerifyThreads, U = 4;
  const int tid = threadIdx.x, n = part.n_all;
  uint64_t key = 0;
  float best = -INFINITY;
  int at = -1;
  for (int b = 0; b < n; b += T * U) {
    const int left = n - b - tid;
    uint4 g[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * T < left) g[u] = part.raw(row, b + u * T + tid);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * T < left) {
        const float x = largest<DT>(g[u]);
        if (x > best || x != x) {
          best = x;
          at = part.granule(b + u * T + tid);
          float y[Elem<DT>::VE];   // columns of a thread need not rise (partial granules come last): keys decide
          Elem<DT>::unpack(g[u], y);
          uint64_t k = 0;
#pragma unroll
          for (int e = 0; e < Elem<DT>::VE; ++e) k = larger_key(k, y[e] == -INFINITY ? 0 : order_key<DT>(y[e], at * Elem<DT>::VE + e - row.ph));
          key = larger_key(key, k);
        } else if (x == best && at > part.granule(b + u * T + tid)) {
          float y[Elem<DT>::VE];
          at = part.granule(b + u * T + tid);
          Elem<DT>::unpack(g[u], y);
#pragma unroll
          for (int e = 0; e < Elem<DT>::VE; ++e)
            if (y[e] == best) key = larger_key(key, order_key<DT>(y[e], at * Elem<DT>::VE + e - row.ph));
        }
      }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) key = larger_key(key, __shfl_xor_sync(~0u, key, o));
  if ((tid & 31) == 0) of_warp[tid >> 5] = key;
  __syncthreads();
  key = of_warp[tid & (kVerifyWarps - 1)];
#pragma unroll
  for (int o = kVerifyWarps / 2; o; o >>= 1) key = larger_key(key, __shfl_xor_sync(~0u, key, o));
  return key;
}

// One cluster of `split` blocks a place of a sequence: what the drawing needs of its rows.
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads, 4) verify_rows_kernel(const __grid_constant__ VerifyParams p) {
  using E = Elem<DT>;
  __shared__ Warps<kVerifyWarps> buf;
  __shared__ Warps<kVerifySplit> parts, draft_parts;   // of the cluster's blocks, in the first one
  __shared__ uint64_t keys[kVerifySplit], of_warp[kVerifyWarps];
  __shared__ float4 upper[kVerifyThreads];
  const int split = p.split, rank = split > 1 ? (int)ptx::cluster_ctarank() : 0, tid = threadIdx.x;
  const int place = blockIdx.x / split, b = place % p.sequences, i = place / p.sequences;
  ptx::let_next_begin();
  if (tid < kVerifySplit) {
    parts.of[tid] = draft_parts.of[tid] = Acc{};
    keys[tid] = 0;
  }
  if (split > 1) ptx::cluster_sync();   // the others may write to the first block
  ptx::begin_after_previous();
  const int64_t* const ids = p.ids + (int64_t)b * p.drafts;
  bool gone = false;   // a draft before this place is absent
  for (int j = tid; j < i; j += kVerifyThreads) gone |= ids[j] < 0 || ids[j] >= p.vocab;
  if (__syncthreads_or(gone)) return;   // all blocks of the cluster
  const int64_t id = i < p.drafts ? ids[i] : -1;
  const bool drafted = id >= 0 && id < p.vocab;
  const float scale = scale_of(p, b), k = scale * kLog2e;
  const int64_t r = (int64_t)b * (p.drafts + 1) + i;
  const Row<DT> row(p.logits, r, p.stride, p.vocab);
  const Part<DT> part(row, rank, p.each);
  Seat* const seat = p.seats + r;
  if (is_greedy(scale)) {
    uint64_t key = best_part<DT>(row, part, of_warp);
    if (split > 1) {
      if (tid == 0) ptx::st_shared_cluster_u64(ptx::mapa(ptx::smem_u32(&keys[rank]), 0), key);
      ptx::cluster_sync();
      key = 0;
      for (int s = 0; s < split; ++s) key = larger_key(key, keys[s]);
    }
    if (rank == 0 && tid == 0) {
      const float x = key_value<DT>(key);
      seat->best = key && fabsf(x) < INFINITY ? key_column(key) : -1;
    }
    return;
  }
  const bool draft = drafted && p.draft_logits;
  const Row<DT> draft_row(p.draft_logits, draft ? (int64_t)b * p.drafts + i : 0, p.draft_stride, p.vocab);
  Acc a = sum_part<DT>(row, part, k, upper, buf), aq;
  if (draft) aq = sum_part<DT>(draft_row, Part<DT>(draft_row, rank, p.draft_each), k, upper, buf);
  if (split > 1) {
    if (tid == 0) {
      const uint32_t to = ptx::mapa(ptx::smem_u32(&parts.of[rank]), 0), to_q = ptx::mapa(ptx::smem_u32(&draft_parts.of[rank]), 0);
      ptx::st_shared_cluster_u32(to, __float_as_uint(a.m));
      ptx::st_shared_cluster_u32(to + 4, __float_as_uint(a.s));
      ptx::st_shared_cluster_u32(to_q, __float_as_uint(aq.m));
      ptx::st_shared_cluster_u32(to_q + 4, __float_as_uint(aq.s));
    }
    ptx::cluster_sync();
    if (rank) return;
    a = warps_join<false>(k, parts);
    aq = warps_join<false>(k, draft_parts);
  }
  if (tid == 0) {
    Seat s{a.m, a.s, aq.m, aq.s, 0.f, 0.f, -1, 0};
    if (drafted) s.z = E::to(row.column((int)id));
    if (draft) s.zq = E::to(draft_row.column((int)id));
    *seat = s;
  }
}

__device__ __forceinline__ double prob(float z, float m, float s, float scale) {
  return z == -INFINITY ? 0. : exp(((double)z - (double)m) * (double)scale) / (double)s;
}

struct Runner {   // of the race; column -1: none
  double score;
  int column;
  __device__ __forceinline__ void meet(double s, int c) {
    if (c >= 0 && (column < 0 || s > score || (s == score && c < column))) {
      score = s;
      column = c;
    }
  }
};

// One cluster of `split` blocks a sequence: accepts drafts up to the first that is refused, and draws the token behind them.
template <int DT>
__global__ void __launch_bounds__(kVerifyThreads) verify_draw_kernel(const __grid_constant__ VerifyParams p) {
  using E = Elem<DT>;
  constexpr int T = kVerifyThreads, VE = E::VE, ES = sizeof(typename E::T);
  __shared__ Runner of_warp[kVerifyWarps], parts[2][kVerifySplit];   // parts: of the cluster's blocks, of the first and the second race
  __shared__ int stop_at;
  const int split = p.split, rank = split > 1 ? (int)ptx::cluster_ctarank() : 0, tid = threadIdx.x, lane = tid & 31;
  const int b = blockIdx.x / split, n = p.drafts;
  ptx::let_next_begin();
  if (split > 1) ptx::cluster_sync();   // the others may write to this block
  ptx::begin_after_previous();
  const float scale = scale_of(p, b);
  const bool greedy = is_greedy(scale);
  const int64_t* const ids = p.ids + (int64_t)b * n;
  const Seat* const seats = p.seats + (int64_t)b * (n + 1);
  if (tid < 32) {
    int stop = 0;
    for (;; stop += 32) {
      const int i = stop + lane;
      bool ok = false;
      if (i < n && ids[i] >= 0 && ids[i] < p.vocab) {
        const Seat s = seats[i];
        if (greedy) {
          ok = s.best == (int)ids[i];
        } else {
          const double pd = prob(s.z, s.m, s.s, scale), qd = p.draft_logits ? prob(s.zq, s.mq, s.sq, scale) : 1.;
          ok = (double)p.uniform[(int64_t)b * n + i] * qd < pd;
        }
      }
      const uint32_t no = __ballot_sync(~0u, !ok);
      if (no) {
        stop += __ffs(no) - 1;
        break;
      }
    }
    if (lane == 0) stop_at = stop;
  }
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
      const float rs = 1.f / seat.s, rsq = with_q ? 1.f / seat.sq : 0.f, mq = with_q ? seat.mq : 0.f;
      float score = 0.f;
      Runner best{0., -1};
      for (int i = tid; i < part.n_all; i += T) {
        const int v = part.granule(i), column = v * VE - row.ph;
        float z[VE], y[VE], e[VE];
        E::unpack(part.raw(row, i), z);
        if (with_q) E::unpack(load_piece<ES>(draft + (int64_t)column * ES, draft, draft + (int64_t)p.vocab * ES), y);
#pragma unroll
        for (int h = 0; h < VE / 4; ++h) {
          float four[4];
          Elem<IRIS_F32>::unpack(load_piece<4>(noise + ((int64_t)column + 4 * h) * 4, noise, noise + (int64_t)p.vocab * 4), four);
#pragma unroll
          for (int u = 0; u < 4; ++u) e[4 * h + u] = four[u];
        }
#pragma unroll
        for (int u = 0; u < VE; ++u) {
          float w = ex2((z[u] - seat.m) * k) * rs;
          if (with_q) w -= ex2((y[u] - mq) * k) * rsq;
          if (column + u == without) w = 0.f;
          const float x = __fdividef(w, e[u]);
          if (w > 0.f && (x > score || (x == score && column + u < best.column))) {
            score = x;
            best.column = column + u;
          }
        }
      }
      if (best.column >= 0) {   // in 64 bits: the race between threads, blocks
        const int c = best.column;
        double w = prob(E::to(row.column(c)), seat.m, seat.s, scale);
        if (with_q) w -= prob(E::to(draft_row.column(c)), seat.mq, seat.sq, scale);
        best.score = w / (double)p.noise[(int64_t)b * p.vocab + c];
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        const double s = __shfl_xor_sync(~0u, best.score, o);
        const int c = __shfl_xor_sync(~0u, best.column, o);
        best.meet(s, c);
      }
      if (lane == 0) of_warp[tid >> 5] = best;
      __syncthreads();
      for (int w = 0; w < kVerifyWarps; ++w) best.meet(of_warp[w].score, of_warp[w].column);
      if (split > 1) {
        if (tid < split) {
          const uint32_t to = ptx::mapa(ptx::smem_u32(&parts[race][rank]), tid);
          ptx::st_shared_cluster_u64(to, (uint64_t)__double_as_longlong(best.score));
          ptx::st_shared_cluster_u32(to + 8, (uint32_t)best.column);
        }
        ptx::cluster_sync();
        for (int s = 0; s < split; ++s) best.meet(parts[race][s].score, parts[race][s].column);
      }
      next = best.column;
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
      double lp = 0.;
      if (token >= 0 && !greedy) lp = ((double)(i < stop ? s.z : E::to(row.column(next))) - (double)s.m) * (double)scale - log((double)s.s);
      p.logprob[(int64_t)b * (n + 1) + i] = (float)lp;
    }
  }
  if (tid == 0) p.accepted[b] = stop;
}

template <int DT>
static int launch_verify(VerifyParams p, const iris_verify_args* a, cudaStream_t st) {
  const auto split_for = [&](int64_t rows, int least, int full) {   // a row is shared while rows alone leave SMs without work
    const int64_t granules = part_granules(a->logits, p.stride, p.vocab, a->dtype, 1);
    int split = 1;
    while (split < kVerifySplit && rows * split < full && granules > (int64_t)split * least) split *= 2;
    p.split = split;
    p.each = part_granules(a->logits, p.stride, p.vocab, a->dtype, split);
    p.draft_each = a->draft_logits ? part_granules(a->draft_logits, p.draft_stride, p.vocab, a->dtype, split) : 0;
  };
  const int64_t places = (int64_t)p.sequences * (p.drafts + 1);
  split_for(places, 1024, kSms * 5 / 2);
  IRIS_CHECK(launch_rows(verify_rows_kernel<DT>, p, (unsigned)(places * p.split), p.split, kVerifyThreads, 0, st));
  split_for(p.sequences, 512, kSms * 5 / 2);
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
  if (a->sequences > INT32_MAX / (kMaxDrafts + 1) / kVerifySplit) return fail(IRIS_ERR_UNSUPPORTED, "%s: too many sequences", fn);
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
  IRIS_CHECK(check_aligned(fn, "uniform", a->uniform, 4, a->drafts > 0));
  IRIS_CHECK(check_aligned(fn, "noise", a->noise, 4, true));
  IRIS_CHECK(check_aligned(fn, "tokens", a->tokens, 8, true));
  IRIS_CHECK(check_aligned(fn, "accepted", a->accepted, 8, true));
  IRIS_CHECK(check_aligned(fn, "logprob", a->logprob, 4, false));
  IRIS_CHECK(check_aligned(fn, "workspace", a->workspace, 16, true));
  const size_t need = iris_verify_workspace_bytes(a->sequences, a->drafts);
  if (a->workspace_bytes < need) return fail(IRIS_ERR_ARG, "%s: workspace has %zu bytes, the call needs %zu", fn, a->workspace_bytes, need);
  VerifyParams p{};
  p.logits = a->logits;
  p.draft_logits = draft ? a->draft_logits : nullptr;
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
