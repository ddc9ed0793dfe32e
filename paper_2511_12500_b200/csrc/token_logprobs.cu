// Log probabilities of given tokens, entropy and the largest alternatives of rows of logits, and their gradient.
//
//   m = max z,  y_j = scale (z_j - m),  s = sum exp y_j;  log probability of t: y_t - ln s;
//   entropy: ln s - (sum y_j exp y_j) / s.
#include "logit_grad.cuh"

namespace iris {
namespace rows {

constexpr int kScoreThreads = 256;

struct ScoreParams {
  const void* logits;
  int64_t stride;
  int vocab, n_targets, top_k;
  float scale;
  const int64_t* targets;
  float *logprob, *entropy, *stats, *top_logprob;
  int64_t* top_ids;
};

__device__ __forceinline__ float log_prob(float z, float m, float ls, float scale) {
  return ls == -INFINITY ? -INFINITY : (z - m) * scale - ls;
}

template <int DT>
__global__ void __launch_bounds__(kScoreThreads) score_kernel(const ScoreParams p) {
  constexpr int VE = Row<DT>::VE;
  __shared__ Acc buf[32];
  __shared__ uint64_t kbuf[32];
  const int64_t r = blockIdx.x;
  const Row<DT> row(p.logits, r, p.stride, p.vocab);
  const int nv = row.granules(), tid = threadIdx.x;
  const float k = p.scale * kLog2e;
  Acc a;
  for (int v = tid; v < nv; v += kScoreThreads) {
    float x[VE];
    row.load(v, x);
    a.add(x, k);
  }
  a = block_merge(a, k, buf);
  const float ls = log_sum(a);
  if (tid == 0) {
    if (p.stats) {
      p.stats[2 * r] = ls == -INFINITY ? -INFINITY : a.m;
      p.stats[2 * r + 1] = ls;
    }
    if (p.entropy) p.entropy[r] = a.s == 0.f ? 0.f : ls - a.t / a.s * kLn2;
  }
  if (p.logprob && tid < p.n_targets) {
    const int64_t t = p.targets[r * p.n_targets + tid];
    p.logprob[r * p.n_targets + tid] = t >= 0 && t < p.vocab ? log_prob(Elem<DT>::to(row.column((int)t)), a.m, ls, p.scale) : 0.f;
  }
  uint64_t last = ~0ull;
  for (int i = 0; i < p.top_k; ++i) {
    uint64_t best = 0;
    for (int v = tid; v < nv; v += kScoreThreads) {
      float x[VE];
      row.load(v, x);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int j = v * VE + e - row.ph;
        if (j >= 0 && j < p.vocab) {
          const uint64_t key = order_key(x[e], j);
          if (key > best && key < last) best = key;
        }
      }
    }
    for (int o = 16; o; o >>= 1) {
      const uint64_t b = __shfl_xor_sync(~0u, best, o);
      best = b > best ? b : best;
    }
    __syncthreads();
    if ((tid & 31) == 0) kbuf[tid >> 5] = best;
    __syncthreads();
    for (int w = 0; w < kScoreThreads / 32; ++w) best = kbuf[w] > best ? kbuf[w] : best;
    if (tid == 0) {
      p.top_ids[r * p.top_k + i] = key_column(best);
      if (p.top_logprob) p.top_logprob[r * p.top_k + i] = log_prob(key_value(best), a.m, ls, p.scale);
    }
    last = best;
  }
}

struct ScoreGradParams {
  const void* logits;
  int64_t stride, grad_stride;
  int vocab, n_targets;
  float scale;
  const int64_t* targets;
  const float *stats, *entropy, *grad_logprob, *grad_entropy;
  void* dlogits;
};

constexpr int kGradThreads = 256;

// dz_j = scale [ sum_q g_q ([t_q = j] - q_j) - g_H q_j (ln q_j + H) ]
template <int DT>
__global__ void __launch_bounds__(kGradThreads) score_grad_kernel(const ScoreGradParams p) {
  __shared__ List list;
  const int64_t r = blockIdx.x;
  const Row<DT> in(p.logits, r, p.stride, p.vocab), out(p.dlogits, r, p.grad_stride, p.vocab);
  const int n = p.grad_logprob ? p.n_targets : 0;
  const float ls = p.stats[2 * r + 1], gh = p.grad_entropy ? p.grad_entropy[r] : 0.f, h = p.grad_entropy ? p.entropy[r] : 0.f;
  if ((int)threadIdx.x < n) {
    const int64_t t = p.targets[r * n + threadIdx.x];
    const bool there = t >= 0 && t < p.vocab;
    list.id[threadIdx.x] = there ? (int)t : -1;
    list.add[threadIdx.x] = there ? p.scale * p.grad_logprob[r * n + threadIdx.x] : 0.f;
  }
  __syncthreads();
  float g = 0.f;
  for (int i = 0; i < n; ++i) g += list.add[i];
  Coef c;
  c.k = p.scale * kLog2e;
  c.m = p.stats[2 * r];
  c.off = c.off_l = ls * kLog2e;
  c.alpha = c.alpha_l = -(g + p.scale * gh * h);
  c.beta = -p.scale * gh * kLn2;
  c.zero = ls == -INFINITY;
  grad_range<DT>(in, out, 0, in.granules(), c, list, n);
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
  IRIS_CHECK(check_scale(fn, "scale", a->scale));
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
  ScoreParams p{a->logits, stride, (int)a->vocab, a->n_targets, a->top_k, a->scale, a->targets, want_lp ? a->logprob : nullptr, a->entropy, a->stats,
                a->top_logprob, a->top_ids};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) score_kernel<IRIS_BF16><<<(unsigned)a->rows, kScoreThreads, 0, st>>>(p);
  else if (a->dtype == IRIS_F16) score_kernel<IRIS_F16><<<(unsigned)a->rows, kScoreThreads, 0, st>>>(p);
  else score_kernel<IRIS_F32><<<(unsigned)a->rows, kScoreThreads, 0, st>>>(p);
  IRIS_CUDA_TRY(cudaGetLastError());
  return IRIS_OK;
}

extern "C" int iris_token_logprobs_backward(const iris_logprob_grad_args* a, void* stream) {
  const char* fn = "iris_token_logprobs_backward";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  int64_t stride = a->row_stride, gstride = a->grad_stride;
  IRIS_CHECK(check_logits(fn, "logits", a->logits, a->dtype, a->rows, a->vocab, &stride));
  IRIS_CHECK(check_logits(fn, "dlogits", a->dlogits, a->dtype, a->rows, a->vocab, &gstride));
  IRIS_CHECK(check_scale(fn, "scale", a->scale));
  if (a->n_targets < 0 || a->n_targets > kMaxList) return fail(IRIS_ERR_ARG, "%s: n_targets=%d not in [0, %d]", fn, a->n_targets, kMaxList);
  IRIS_CHECK(check_in_place(fn, a->logits, stride, a->dlogits, gstride, a->rows, a->vocab, a->dtype));
  if (a->rows == 0 || a->vocab == 0) return IRIS_OK;
  const bool want_lp = a->n_targets > 0 && a->grad_logprob, want_h = a->grad_entropy != nullptr;
  IRIS_CHECK(check_aligned(fn, "targets", a->targets, 8, want_lp));
  IRIS_CHECK(check_aligned(fn, "grad_logprob", a->grad_logprob, 4, false));
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, true));
  IRIS_CHECK(check_aligned(fn, "grad_entropy", a->grad_entropy, 4, false));
  IRIS_CHECK(check_aligned(fn, "entropy", a->entropy, 4, want_h));
  ScoreGradParams p{a->logits, stride, gstride, (int)a->vocab, a->n_targets, a->scale, a->targets, a->stats, a->entropy, want_lp ? a->grad_logprob : nullptr,
                    a->grad_entropy, a->dlogits};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) score_grad_kernel<IRIS_BF16><<<(unsigned)a->rows, kGradThreads, 0, st>>>(p);
  else if (a->dtype == IRIS_F16) score_grad_kernel<IRIS_F16><<<(unsigned)a->rows, kGradThreads, 0, st>>>(p);
  else score_grad_kernel<IRIS_F32><<<(unsigned)a->rows, kGradThreads, 0, st>>>(p);
  IRIS_CUDA_TRY(cudaGetLastError());
  return IRIS_OK;
}
