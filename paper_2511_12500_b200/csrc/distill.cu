// Distillation from a teacher's top logits: per row the Kullback-Leibler divergence of the student's distribution over
// the whole vocabulary from the teacher's on its listed tokens, and the gradient for the student's logits.
//
//   renormalised list: p = softmax(teacher_scale v),              L = sum_k p_k (ln p_k - ln q_k)
//   with remainder:    p_k = exp v_k, p_r = max(0, 1 - sum p_k),  L = the same + p_r (ln p_r - ln q_r), q_r = sum of q off the list
//   dL/dz_j = scale (P q_j - p_j) in the first form; in the second scale ((P + p_r) q_j - p_j) on the list and
//   scale ((P + p_r) q_j - p_r q_j / q_r) off it;  P = sum p_k.
#include "logit_grad.cuh"

namespace iris {
namespace rows {

constexpr int kDistillThreads = 256;
static_assert(kDistillThreads >= kMaxList, "one thread an entry of the list");

struct DistillParams {
  const void* logits;
  int64_t stride, grad_stride;
  int vocab, list_k, hold;   // hold: granules of a row that fit shared memory at once
  bool tail;
  float scale, teacher_scale;
  const float* teacher;
  const int64_t* ids;
  const float* weight;       // forward with gradient: loss weights; backward: grad_loss; nullptr = 1
  float *loss, *stats;
  void* dlogits;
};

// The teacher's list in shared memory: probabilities p[], columns in list.id (-1: absent).
struct Teacher {
  List list;
  float p[kMaxList];
};

// Fills t from the row's list; returns P and the remainder p_r.  Ends with a barrier.
__device__ __forceinline__ float2 load_teacher(const DistillParams& p, int64_t r, Teacher& t) {
  const int i = threadIdx.x, n = p.list_k;
  if (i < n) {
    const int64_t id = p.ids[r * n + i];
    const bool there = id >= 0 && id < p.vocab;
    t.list.id[i] = there ? (int)id : -1;
    const float v = p.teacher[r * n + i];
    t.p[i] = !there ? (p.tail ? 0.f : -INFINITY) : p.tail ? expf(v) : v * p.teacher_scale;
  }
  __syncthreads();
  if (!p.tail) {
    float m = -FLT_MAX;
    for (int j = 0; j < n; ++j) m = fmaxf(m, t.p[j]);
    const float e = i < n ? expf(t.p[i] - m) : 0.f;
    __syncthreads();
    if (i < n) t.p[i] = e;
    __syncthreads();
    float s = 0.f;
    for (int j = 0; j < n; ++j) s += t.p[j];
    __syncthreads();
    if (i < n) t.p[i] = s == 0.f ? 0.f : e / s;   // a list with no token left asks for nothing
    __syncthreads();
    return make_float2(s == 0.f ? 0.f : s == s ? 1.f : NAN, 0.f);
  }
  float s = 0.f;
  for (int j = 0; j < n; ++j) s += t.p[j];
  return make_float2(s, max_nan(0.f, 1.f - s));
}

// Coefficients of the gradient; also fills list.add.  Ends with a barrier.
__device__ __forceinline__ Coef distill_coef(const DistillParams& p, Teacher& t, float2 mass, float m, float ls, float lr, float w) {
  Coef c;
  c.k = p.scale * kLog2e;
  c.m = m;
  c.beta = 0.f;
  c.off_l = ls * kLog2e;
  c.alpha_l = w * p.scale * (mass.x + mass.y);
  if (p.tail) {
    const bool some = lr != -INFINITY;
    c.off = some ? lr * kLog2e : 0.f;
    c.alpha = some ? w * p.scale * ((mass.x + mass.y) * expf(lr - ls) - mass.y) : 0.f;
  } else {
    c.off = c.off_l;
    c.alpha = c.alpha_l;
  }
  c.zero = ls == -INFINITY || w == 0.f;
  if ((int)threadIdx.x < p.list_k) t.list.add[threadIdx.x] = -w * p.scale * t.p[threadIdx.x];
  __syncthreads();
  return c;
}

template <int DT>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams p) {
  using E = Elem<DT>;
  constexpr int VE = E::VE;
  extern __shared__ uint4 held[];
  __shared__ Teacher t;
  __shared__ Acc buf[32];
  __shared__ float red[32];
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, n = p.list_k;
  const Row<DT> in(p.logits, r, p.stride, p.vocab);
  const int nv = in.granules();
  const float k = p.scale * kLog2e;
  const float2 mass = load_teacher(p, r, t);
  const int id = tid < n ? t.list.id[tid] : -1;
  bool first = id >= 0;
  for (int j = 0; j < tid && j < n && first; ++j) first = t.list.id[j] != id;

  Acc a, on_list;
  float zk = -INFINITY;
  for (int v0 = 0; v0 < nv; v0 += p.hold) {
    const int v1 = min(nv, v0 + p.hold);
    __syncthreads();   // the previous tile has been read
    for (int v = v0 + tid; v < v1; v += kDistillThreads) {
      if (in.whole(v)) {
        held[v - v0] = ld_global_v4(in.at(v));
      } else {
        float x[VE];
        in.load(v, x);
        held[v - v0] = E::pack(x);
      }
    }
    __syncthreads();
    typename E::T* cells = reinterpret_cast<typename E::T*>(held);
    const int at = in.ph + id - v0 * VE;
    const bool here = id >= 0 && at >= 0 && at < (v1 - v0) * VE;
    if (here) {
      zk = E::to(cells[at]);
      const float one[1] = {zk};
      if (first) on_list.add(one, k);
    }
    if (p.tail) {   // listed tokens leave the sum over the remainder
      __syncthreads();
      if (here) cells[at] = E::from(-INFINITY);
      __syncthreads();
    }
    for (int v = tid; v < v1 - v0; v += kDistillThreads) {
      float x[VE];
      E::unpack(held[v], x);
      a.add(x, k);
    }
  }
  a = block_merge(a, k, buf);
  float lr = 0.f;
  Acc all = a;
  if (p.tail) {
    on_list = block_merge(on_list, k, buf);
    all.merge(on_list, k);
  }
  const float ls = log_sum(all);
  if (p.tail) lr = a.s == 0.f ? -INFINITY : (a.m - all.m) * p.scale + log_sum(a);
  float l = 0.f;
  if (id >= 0 && !(t.p[tid] == 0.f)) l = t.p[tid] * (logf(t.p[tid]) - ((zk - all.m) * p.scale - ls));
  if (tid == 0 && p.tail && !(mass.y == 0.f) && !(lr == -INFINITY && mass.y < 1e-5f)) l += mass.y * (logf(mass.y) - (lr - ls));
  if (ls == -INFINITY && id >= 0 && t.p[tid] > 0.f) l = INFINITY;
  if (ls == -INFINITY && tid == 0 && mass.y > 0.f) l = INFINITY;
  for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
  if ((tid & 31) == 0) red[tid >> 5] = l;
  __syncthreads();
  if (tid == 0) {
    float s = 0.f;
    for (int w = 0; w < kDistillThreads / 32; ++w) s += red[w];
    p.loss[r] = s;
    if (p.stats) {
      p.stats[3 * r] = ls == -INFINITY ? -INFINITY : all.m;
      p.stats[3 * r + 1] = ls;
      p.stats[3 * r + 2] = ls == -INFINITY && p.tail ? -INFINITY : lr;
    }
  }
  if (!p.dlogits) return;
  const Coef c = distill_coef(p, t, mass, all.m, ls, lr, p.weight ? p.weight[r] : 1.f);
  const Row<DT> out(p.dlogits, r, p.grad_stride, p.vocab);
  if (nv > p.hold) {
    grad_range<DT>(in, out, 0, nv, c, t.list, n);
    return;
  }
  for (int v = tid; v < nv; v += kDistillThreads) {
    float x[VE];
    E::unpack(held[v], x);
    dense_granule<DT>(x, c);
    store_granule<DT>(in, out, v, x);
  }
  __syncthreads();
  if (id >= 0 && !c.zero)
    out.column(id) = E::from(grad_of(zk, c.k, c.m, c.off_l, c.alpha_l, 0.f) + add_of_column(t.list, n, tid));
}

template <int DT>
__global__ void __launch_bounds__(kDistillThreads) distill_grad_kernel(const DistillParams p) {
  __shared__ Teacher t;
  const int64_t r = blockIdx.x;
  const Row<DT> in(p.logits, r, p.stride, p.vocab), out(p.dlogits, r, p.grad_stride, p.vocab);
  const float2 mass = load_teacher(p, r, t);
  const Coef c = distill_coef(p, t, mass, p.stats[3 * r], p.stats[3 * r + 1], p.stats[3 * r + 2], p.weight[r]);
  grad_range<DT>(in, out, 0, in.granules(), c, t.list, p.list_k);
}

}  // namespace rows
}  // namespace iris

using namespace iris;
using namespace iris::rows;

namespace {

constexpr int kHoldBytes = 192 * 1024;
constexpr int kMaxDevices = 64;

int check_distill(const char* fn, const iris_distill_args* a, int64_t* stride, int64_t* gstride) {
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  *stride = a->row_stride;
  IRIS_CHECK(check_logits(fn, "logits", a->logits, a->dtype, a->rows, a->vocab, stride));
  IRIS_CHECK(check_scale(fn, "scale", a->scale));
  IRIS_CHECK(check_scale(fn, "teacher_scale", a->teacher_scale));
  if (a->mode != IRIS_DISTILL_RENORM && a->mode != IRIS_DISTILL_TAIL) return fail(IRIS_ERR_ARG, "%s: unknown mode %d", fn, a->mode);
  if (a->list_k < 0 || a->list_k > kMaxList) return fail(IRIS_ERR_ARG, "%s: list_k=%d not in [0, %d]", fn, a->list_k, kMaxList);
  if (a->dlogits) {
    *gstride = a->grad_stride;
    IRIS_CHECK(check_logits(fn, "dlogits", a->dlogits, a->dtype, a->rows, a->vocab, gstride));
    IRIS_CHECK(check_in_place(fn, a->logits, *stride, a->dlogits, *gstride, a->rows, a->vocab, a->dtype));
  }
  if (a->rows == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "teacher", a->teacher, 4, a->list_k > 0));
  IRIS_CHECK(check_aligned(fn, "teacher_ids", a->teacher_ids, 8, a->list_k > 0));
  IRIS_CHECK(check_aligned(fn, "weight", a->weight, 4, false));
  return IRIS_OK;
}

DistillParams params_of(const iris_distill_args* a, int64_t stride, int64_t gstride) {
  DistillParams p{};
  p.logits = a->logits;
  p.stride = stride;
  p.grad_stride = gstride;
  p.vocab = (int)a->vocab;
  p.list_k = a->list_k;
  p.tail = a->mode == IRIS_DISTILL_TAIL;
  p.scale = a->scale;
  p.teacher_scale = a->teacher_scale;
  p.teacher = a->teacher;
  p.ids = a->teacher_ids;
  p.weight = a->weight;
  p.loss = a->loss;
  p.stats = a->stats;
  p.dlogits = a->dlogits;
  return p;
}

template <int DT>
int launch_distill(DistillParams p, int64_t rows, cudaStream_t st) {
  static bool configured[kMaxDevices] = {};
  int dev = -1;
  IRIS_CUDA_TRY(cudaGetDevice(&dev));
  if (dev >= kMaxDevices || !configured[dev]) {
    IRIS_CUDA_TRY(cudaFuncSetAttribute(distill_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHoldBytes));
    if (dev < kMaxDevices) configured[dev] = true;
  }
  const int64_t need = (p.vocab + 2 * Row<DT>::VE - 2) / Row<DT>::VE;   // granules of a row, wherever it starts
  p.hold = (int)(need * 16 <= kHoldBytes ? (need > 0 ? need : 1) : kHoldBytes / 16);
  distill_kernel<DT><<<(unsigned)rows, kDistillThreads, (size_t)p.hold * 16, st>>>(p);
  IRIS_CUDA_TRY(cudaGetLastError());
  return IRIS_OK;
}

}  // namespace

extern "C" int iris_distill_topk(const iris_distill_args* a, void* stream) {
  const char* fn = "iris_distill_topk";
  int64_t stride = 0, gstride = 0;
  IRIS_CHECK(check_distill(fn, a, &stride, &gstride));
  if (a->rows == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "loss", a->loss, 4, true));
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, false));
  const DistillParams p = params_of(a, stride, gstride);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) return launch_distill<IRIS_BF16>(p, a->rows, st);
  if (a->dtype == IRIS_F16) return launch_distill<IRIS_F16>(p, a->rows, st);
  return launch_distill<IRIS_F32>(p, a->rows, st);
}

extern "C" int iris_distill_topk_backward(const iris_distill_args* a, void* stream) {
  const char* fn = "iris_distill_topk_backward";
  int64_t stride = 0, gstride = 0;
  IRIS_CHECK(check_distill(fn, a, &stride, &gstride));
  if (a->rows == 0 || a->vocab == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, true));
  IRIS_CHECK(check_aligned(fn, "weight", a->weight, 4, true));
  if (!a->dlogits) return fail(IRIS_ERR_ARG, "%s: dlogits is NULL", fn);
  const DistillParams p = params_of(a, stride, gstride);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) distill_grad_kernel<IRIS_BF16><<<(unsigned)a->rows, kDistillThreads, 0, st>>>(p);
  else if (a->dtype == IRIS_F16) distill_grad_kernel<IRIS_F16><<<(unsigned)a->rows, kDistillThreads, 0, st>>>(p);
  else distill_grad_kernel<IRIS_F32><<<(unsigned)a->rows, kDistillThreads, 0, st>>>(p);
  IRIS_CUDA_TRY(cudaGetLastError());
  return IRIS_OK;
}
