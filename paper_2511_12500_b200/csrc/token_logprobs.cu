// Log probabilities of given tokens, entropy and the largest alternatives of rows of logits, and their gradient.
//
//   m = max z,  y_j = scale (z_j - m),  s = sum exp y_j;  log probability of t: y_t - ln s;
//   entropy: ln s - (sum y_j exp y_j) / s.
#include <type_traits>

#include "logit_grad.cuh"
#include "top_list.cuh"

namespace iris {
namespace rows {

constexpr int kScoreThreads = 256;
constexpr int kOneBatch = 2048;         // granules of a part that its block holds in registers, 8 a thread
enum { kNoTop, kTopPiecewise, kTopOneBatch };
constexpr int kMaxSplit = 8;            // blocks (one cluster) that share a row
static_assert(kScoreThreads == kTopThreads, "the list is kept by all threads of the block");

struct ScoreParams {
  const void* logits;
  int64_t stride;
  int vocab, n_targets, top_k, split, each;   // each: granules of a block's part of a row
  float scale;
  const int64_t* targets;
  float *logprob, *entropy, *stats, *top_logprob;
  int64_t* top_ids;
};

__device__ __forceinline__ float log_prob(float z, float m, float ls, float scale) {
  return ls == -INFINITY ? -INFINITY : (z - m) * scale - ls;
}

struct NoTop {};
// Where a thread's upper sums lie: the list is filled behind the pass (the kernel with pieces has shared memory for five blocks an SM and no more).
__device__ __forceinline__ float4* upper_of(NoTop&, float4* upper) { return upper + threadIdx.x; }
__device__ __forceinline__ float4* upper_of(TopShared& top, float4*) {
  static_assert(sizeof(top.key) >= kScoreThreads * sizeof(float4), "one for each thread");
  return reinterpret_cast<float4*>(top.key) + threadIdx.x;
}

// One cluster of `split` blocks a row; each takes an equal run of granules, and all get what each found.
//
// Bound by memory where a row is long and there are many (4096 x 128000 bf16: 189 us, 5.5 TB/s, 85 % of the copy rate; 7.0
// instructions an element, 60 % of the issue slots): without alternatives a batch of four granules a thread is fetched
// while one is summed, in four blocks an SM (without that 4 to 6 % more; five blocks spill far more registers than the 8 bytes
// that bf16 with entropy does with four: 194 us).  With alternatives five blocks of single batches hide the end of one row, about half of a
// block's time, behind the others' passes (4096 x 36864 fp16, 64 alternatives: 86 us; four blocks 91).  Short rows are bound by the
// chain of latencies: load, bound, list, places (1 x 16384: 4.6 us from first to last instruction).
//
// TOP: no alternatives; alternatives of a part of any length, of which pieces are read again; of a part of at most
// kOneBatch granules, which stays in registers.
template <int DT, bool ENTROPY, int TOP>
__global__ void __launch_bounds__(kScoreThreads, TOP == kTopPiecewise ? 5 : 4) score_kernel(const ScoreParams p) {
  using E = Elem<DT>;
  constexpr int T = kScoreThreads, U = TOP == kTopOneBatch ? kOneBatch / T : 4;
  __shared__ Warps<T / 32> buf;
  __shared__ Warps<kMaxSplit> parts;   // of the cluster's blocks
  __shared__ float4 upper[TOP == kNoTop ? T : 1];
  __shared__ typename std::conditional<TOP != kNoTop, TopShared, NoTop>::type top;
  extern __shared__ uint64_t lists[];   // TOP and split > 1: the blocks' sorted lists, top_k keys each, 0 where one is shorter
  const int split = p.split, rank = split > 1 ? (int)ptx::cluster_ctarank() : 0, tid = threadIdx.x;
  const int64_t r = blockIdx.x / split;
  if (split > 1) {
    if (tid < kMaxSplit) parts.of[tid] = Acc{};
    ptx::cluster_arrive_release();   // behind the wait the others may write there
  }
  const Row<DT> row(p.logits, r, p.stride, p.vocab);
  const Part<DT> part(row, rank, p.each);
  const float k = p.scale * kLog2e;
  ptx::begin_after_previous();
  float zt = 0.f;
  bool there = false;
  if (rank == 0 && tid < p.n_targets) {
    const int64_t t = p.targets[r * p.n_targets + tid];
    there = t >= 0 && t < p.vocab;
    if (there) zt = E::to(row.column((int)t));
  }
  Sums<DT, ENTROPY, TOP != kTopOneBatch> sums(k, upper_of(top, upper));
  const uint4* const from = reinterpret_cast<const uint4*>(row.at(part.w0)) + tid;
  const int n = part.n_all, shift = TOP == kTopPiecewise ? piece_shift(n) : 0;
  float best = -INFINITY, of_piece = -INFINITY;
  uint4 g[U];
  const auto load = [&](int b, auto all) {
    constexpr bool ALL = decltype(all)::value;
    const int left = n - b - tid;   // this thread has granules u with u * T < left
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (ALL) g[u] = ld_once(from + b + u * T);
      else if (u * T < left) g[u] = part.raw(row, b + u * T + tid);
    }
  };
  const auto batch = [&](int b, auto all) {
    constexpr bool ALL = decltype(all)::value;
    const int left = n - b - tid;
    load(b, all);
    const float mx = largest<DT, ALL>(g, left, T);
    sums.template pace<T, U>(b);
    sums.template add<ALL>(g, mx, left, T);
    if constexpr (TOP == kTopPiecewise) {   // the largest of each piece: 1 or 2 granules of the batch, all of them, or those of several batches
      static_assert(TOP != kTopPiecewise || U == 4, "pieces of 1, 2 and 4 granules lie in a batch");
      const int u0 = b / T, q = u0 >> shift;   // the batch's first granule of the thread, and its piece
      best = max_nan(best, mx);
      if (shift == 0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (ALL || u * T < left) top.largest[q + u][tid] = largest<DT>(g[u]);
      } else if (shift == 1) {
#pragma unroll
        for (int u = 0; u < U; u += 2)
          if (ALL || u * T < left)
            top.largest[q + u / 2][tid] = E::unfold(ALL || (u + 1) * T < left ? E::larger(E::fold(g[u]), E::fold(g[u + 1])) : E::fold(g[u]));
      } else {
        of_piece = u0 & ((1 << shift) - 1) ? max_nan(of_piece, mx) : mx;
        if (ALL || left > 0) top.largest[q][tid] = of_piece;
      }
    }
  };
  if constexpr (TOP == kTopOneBatch) {
    load(0, std::false_type{});
    best = largest<DT, false>(g, n - tid, T);
    top.ordinal[tid] = tid < n ? E::ordinal(best) : 0;
    if (tid == 0) top.n = top.n_queue = 0;
    __syncthreads();
    if (tid < 32) find_tau(top, p.top_k);   // while the other warps go on
    sums.template add<false>(g, best, n - tid, T);
  } else {
    int b = 0;
    if constexpr (TOP == kNoTop) {   // the next batch is under way while one is summed
      constexpr int B = T * U;
      uint4 h[U];
      const auto fetch = [&](int at, uint4(&to)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) to[u] = ld_once(from + at + u * T);
      };
      if (B <= part.n_int) fetch(0, g);
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
    }
    for (; b + T * U <= part.n_int; b += T * U) batch(b, std::true_type{});
    for (; b < n; b += T * U) batch(b, std::false_type{});
    if constexpr (TOP) {
      top.ordinal[tid] = tid < n ? E::ordinal(best) : 0;
      if (tid == 0) top.n = top.n_again = top.n_queue = 0;
    }
  }
  ptx::let_next_begin();
  warp_share<ENTROPY>(sums.done(), k, buf);
  __syncthreads();
  Acc a = warps_join<ENTROPY>(k, buf);
  const auto find_top = [&](auto emit) -> int {
    if constexpr (TOP == kTopPiecewise) {
      if (tid < 32) find_tau(top, p.top_k);
      __syncthreads();
    }
    if constexpr (TOP != kNoTop) {
      const Wanted<DT> wanted(top);
      if constexpr (TOP == kTopPiecewise) {
        queue_pieces<DT>(top, row, part, shift, wanted);
      } else if (!wanted.none && wanted(best)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * T < n - tid && wanted(largest<DT>(g[u]))) queue_granule(top, part.granule(u * T + tid), g[u]);
      }
      __syncthreads();
      list_queue<DT>(top, row, wanted);
      return finish_top<DT>(top, row, part, wanted.tau, p.top_k, emit);
    }
    return 0;
  };

  if (split > 1) {
    ptx::cluster_wait();   // all blocks have started and cleared their places
    if (tid < split) {
      const uint32_t to = ptx::mapa(ptx::smem_u32(&parts.of[rank]), tid);
      ptx::st_shared_cluster_u32(to, __float_as_uint(a.m));
      ptx::st_shared_cluster_u32(to + 4, __float_as_uint(a.s));
      ptx::st_shared_cluster_u32(to + 8, __float_as_uint(a.t));
    }
    if constexpr (TOP) {
      const uint32_t own = ptx::smem_u32(lists + rank * p.top_k);
      const auto share = [&](int place, uint64_t key, int sub, int group) {
        for (int s = sub; s < split; s += group) ptx::st_shared_cluster_u64(ptx::mapa(own + place * 8, s), key);
      };
      const int found = find_top(share);
      if (tid >= found && tid < p.top_k) share(tid, 0, 0, 1);
    }
    ptx::cluster_sync();
    a = warps_join<ENTROPY>(k, parts);
  }
  const float ls = log_sum(a);
  if (rank == 0 && tid == 0) {
    if (p.stats) {
      p.stats[2 * r] = ls == -INFINITY ? -INFINITY : a.m;
      p.stats[2 * r + 1] = ls;
    }
    if (ENTROPY) p.entropy[r] = a.s == 0.f ? 0.f : ls - a.t / a.s * kLn2;
  }
  if (rank == 0 && tid < p.n_targets) p.logprob[r * p.n_targets + tid] = there ? log_prob(zt, a.m, ls, p.scale) : 0.f;
  if constexpr (TOP) {
    const auto emit = [&](int place, uint64_t key, int sub, int) {
      if (sub) return;
      p.top_ids[r * p.top_k + place] = key_column(key);
      if (p.top_logprob) p.top_logprob[r * p.top_k + place] = log_prob(key_value<DT>(key), a.m, ls, p.scale);
    };
    if (split == 1) {
      find_top(emit);
    } else {   // every block finds the places of its own keys, with a group of threads each
      int group = 32;
      while (group * p.top_k > T) group /= 2;   // >= 2: top_k <= 128
      const int i = tid / group, n_all = split * p.top_k;
      const uint64_t key = i < p.top_k ? lists[rank * p.top_k + i] : 0;
      int place = 0;
      for (int j = tid % group; j < n_all; j += group) place += lists[j] > key;
      for (int o = group / 2; o; o /= 2) place += __shfl_xor_sync(~0u, place, o);
      if (key && place < p.top_k) emit(place, key, tid % group, group);
    }
  }
}

template <int DT, bool ENTROPY>
static int launch_score(const ScoreParams& p, int64_t rows, cudaStream_t st) {
  const auto kernel = !p.top_k             ? score_kernel<DT, ENTROPY, kNoTop>
                      : p.each > kOneBatch ? score_kernel<DT, ENTROPY, kTopPiecewise>
                                           : score_kernel<DT, ENTROPY, kTopOneBatch>;
  return launch_rows(kernel, p, (unsigned)(rows * p.split), p.split, kScoreThreads, p.split > 1 ? (size_t)p.split * p.top_k * 8 : 0, st);
}

template <int DT>
static int launch_score(const ScoreParams& p, int64_t rows, cudaStream_t st) {
  return p.entropy ? launch_score<DT, true>(p, rows, st) : launch_score<DT, false>(p, rows, st);
}

struct ScoreGradParams {
  const void* logits;
  int64_t stride, grad_stride;
  int vocab, n_targets, parts, each;
  float scale;
  const int64_t* targets;
  const float *stats, *entropy, *grad_logprob, *grad_entropy;
  void* dlogits;
};

// dz_j = scale [ sum_q g_q ([t_q = j] - q_j) - g_H q_j (ln q_j + H) ]
template <int DT, bool ENTROPY>
__global__ void __launch_bounds__(kGradThreads) score_grad_kernel(const ScoreGradParams p) {
  __shared__ List list;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const int64_t r = blockIdx.x / p.parts;
  const Row<DT> in(p.logits, r, p.stride, p.vocab), out(p.dlogits, r, p.grad_stride, p.vocab);
  const int n = p.grad_logprob ? p.n_targets : 0;
  const float ls = p.stats[2 * r + 1], gh = ENTROPY ? p.grad_entropy[r] : 0.f, h = ENTROPY ? p.entropy[r] : 0.f;
  if (threadIdx.x < kMaxList) {
    int id = -1;
    float add = 0.f;
    if ((int)threadIdx.x < n) {
      const int64_t t = p.targets[r * n + threadIdx.x];
      if (t >= 0 && t < p.vocab) {
        id = (int)t;
        add = p.scale * p.grad_logprob[r * n + threadIdx.x];
      }
    }
    list.id[threadIdx.x] = id;
    list.add[threadIdx.x] = add;
  }
  __syncthreads();
  float g = 0.f;
  for (int i = 0; i < n; ++i) g += list.add[i];
  Coef c;
  c.k = p.scale * kLog2e;
  c.m = c.m_l = p.stats[2 * r];
  c.off = c.off_l = ls * kLog2e;
  c.alpha = c.alpha_l = -(g + p.scale * gh * h);
  c.beta = -p.scale * gh * kLn2;
  c.zero = ls == -INFINITY;
  grad_part<DT, ENTROPY>(in, out, Part<DT>(in, blockIdx.x % p.parts, p.each), c, list, n);
}

template <int DT>
static int launch_score_grad(const ScoreGradParams& p, int64_t rows, cudaStream_t st) {
  const unsigned blocks = (unsigned)(rows * p.parts);
  if (p.grad_entropy) return launch_rows(score_grad_kernel<DT, true>, p, blocks, 1, kGradThreads, 0, st);
  return launch_rows(score_grad_kernel<DT, false>, p, blocks, 1, kGradThreads, 0, st);
}

}  // namespace rows
}  // namespace iris

using namespace iris;
using namespace iris::rows;

extern "C" int iris_token_logprobs(const iris_logprob_args* a, void* stream) {
  const char* fn = "iris_token_logprobs";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  int64_t stride = a->row_stride;
  IRIS_CHECK(check_logits(fn, "logits", a->logits, a->dtype, a->rows, a->vocab, &stride));
  IRIS_CHECK(check_scale(fn, "scale", a->scale, kMaxScale));
  if (a->n_targets < 0 || a->n_targets > kMaxList) return fail(IRIS_ERR_ARG, "%s: n_targets=%d not in [0, %d]", fn, a->n_targets, kMaxList);
  if (a->top_k < 0 || a->top_k > kMaxList) return fail(IRIS_ERR_ARG, "%s: top_k=%d not in [0, %d]", fn, a->top_k, kMaxList);
  if (a->top_k > a->vocab) return fail(IRIS_ERR_ARG, "%s: top_k=%d exceeds vocab=%lld", fn, a->top_k, (long long)a->vocab);
  if (a->rows == 0) return IRIS_OK;
  const bool want_lp = a->n_targets > 0;
  IRIS_CHECK(check_aligned(fn, "targets", a->targets, 8, want_lp));
  IRIS_CHECK(check_aligned(fn, "logprob", a->logprob, 4, want_lp));
  IRIS_CHECK(check_aligned(fn, "entropy", a->entropy, 4, false));
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, false));
  IRIS_CHECK(check_aligned(fn, "top_ids", a->top_ids, 8, a->top_k > 0));
  IRIS_CHECK(check_aligned(fn, "top_logprob", a->top_logprob, 4, false));
  // A row is shared by a cluster of blocks while the rows alone leave SMs without work, until a part fits registers.
  const int64_t granules = part_granules(a->logits, stride, a->vocab, a->dtype, 1);
  int split = 1;
  while (split < kMaxSplit && a->rows * split < kSms * 5 / 2 && granules > (int64_t)split * kOneBatch) split *= 2;
  ScoreParams p{a->logits, stride, (int)a->vocab, want_lp ? a->n_targets : 0, a->top_k, split, part_granules(a->logits, stride, a->vocab, a->dtype, split), a->scale, a->targets, a->logprob, a->entropy, a->stats,
                a->top_logprob, a->top_ids};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) return launch_score<IRIS_BF16>(p, a->rows, st);
  if (a->dtype == IRIS_F16) return launch_score<IRIS_F16>(p, a->rows, st);
  return launch_score<IRIS_F32>(p, a->rows, st);
}

extern "C" int iris_token_logprobs_backward(const iris_logprob_grad_args* a, void* stream) {
  const char* fn = "iris_token_logprobs_backward";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  int64_t stride = a->row_stride, gstride = a->grad_stride;
  IRIS_CHECK(check_logits(fn, "logits", a->logits, a->dtype, a->rows, a->vocab, &stride));
  IRIS_CHECK(check_logits(fn, "dlogits", a->dlogits, a->dtype, a->rows, a->vocab, &gstride));
  IRIS_CHECK(check_scale(fn, "scale", a->scale, kMaxScale));
  if (a->n_targets < 0 || a->n_targets > kMaxList) return fail(IRIS_ERR_ARG, "%s: n_targets=%d not in [0, %d]", fn, a->n_targets, kMaxList);
  IRIS_CHECK(check_in_place(fn, a->logits, stride, a->dlogits, gstride, a->rows, a->vocab, a->dtype));
  if (a->rows == 0 || a->vocab == 0) return IRIS_OK;
  const bool want_lp = a->n_targets > 0 && a->grad_logprob, want_h = a->grad_entropy != nullptr;
  IRIS_CHECK(check_aligned(fn, "targets", a->targets, 8, want_lp));
  IRIS_CHECK(check_aligned(fn, "grad_logprob", a->grad_logprob, 4, false));
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, true));
  IRIS_CHECK(check_aligned(fn, "grad_entropy", a->grad_entropy, 4, false));
  IRIS_CHECK(check_aligned(fn, "entropy", a->entropy, 4, want_h));
  const int parts = grad_parts(a->vocab, a->dtype);
  if (a->rows * parts > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 blocks", fn);
  ScoreGradParams p{a->logits, stride, gstride, (int)a->vocab, a->n_targets, parts, part_granules(a->logits, stride, a->vocab, a->dtype, parts), a->scale, a->targets, a->stats, a->entropy,
                    want_lp ? a->grad_logprob : nullptr, a->grad_entropy, a->dlogits};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) return launch_score_grad<IRIS_BF16>(p, a->rows, st);
  if (a->dtype == IRIS_F16) return launch_score_grad<IRIS_F16>(p, a->rows, st);
  return launch_score_grad<IRIS_F32>(p, a->rows, st);
}
