// Distillation from a teacher's top logits: per row the Kullback-Leibler divergence of the student's distribution over
// the whole vocabulary from the teacher's on its listed tokens, and the gradient for the student's logits.
//
//   renormalised list: p = softmax(teacher_scale v),              L = sum_k p_k (ln p_k - ln q_k)
//   with remainder:    p_k = exp v_k, p_r = max(0, 1 - sum p_k),  L = the same + p_r (ln p_r - ln q_r), q_r = sum of q off the list
//   dL/dz_j = scale (P q_j - p_j) in the first form; in the second scale ((P + p_r) q_j - p_j) on the list and
//   scale ((P + p_r) q_j - p_r q_j / q_r) off it;  P = sum p_k.
#include <algorithm>

#include "logit_grad.cuh"
#include "sm100_ptx.cuh"

namespace iris {
namespace rows {

constexpr int kDistillThreads = 256;
constexpr int kMaxSplit = 8;   // blocks (one cluster) that share a row
static_assert(kDistillThreads >= kMaxList && kGradThreads == kDistillThreads, "one thread an entry of the list");

struct DistillParams {
  const void* logits;
  int64_t stride, grad_stride;
  int vocab, list_k, split, hold;   // hold: granules of its part that a block keeps in shared memory
  float scale, teacher_scale;
  const float* teacher;
  const int64_t* ids;
  const float* weight;       // forward with gradient: loss weights; backward: grad_loss; nullptr = 1
  float *loss, *stats;
  void* dlogits;
};

// The teacher's list in shared memory: probabilities p[], columns in list.id (-1: absent), their sum and the remainder p_r.
struct Teacher {
  List list;
  float p[kMaxList];
  float sum, rest;
};

// Fills t from the row's list, by the first warp; visible to the others after the next barrier.
template <bool TAIL>
__device__ __forceinline__ void load_teacher(const DistillParams& p, int64_t r, Teacher& t) {
  if (threadIdx.x >= 32) return;
  constexpr int N = kMaxList / 32;
  const int lane = threadIdx.x, n = p.list_k;
  float v[N];
  float m = TAIL ? 0.f : -FLT_MAX;   // log probabilities are taken as they are
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int j = lane + 32 * i;
    int id = -1;
    v[i] = -INFINITY;
    if (j < n) {
      const int64_t id64 = p.ids[r * n + j];
      if (id64 >= 0 && id64 < p.vocab) {
        id = (int)id64;
        v[i] = p.teacher[r * n + j] * (TAIL ? 1.f : p.teacher_scale);
      }
    }
    t.list.id[j] = id;
    if (!TAIL) m = fmaxf(m, v[i]);
  }
  if (!TAIL) m = warp_max(m);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 32 * i < n ? expf(v[i] - m) : 0.f;
    s += v[i];
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
#pragma unroll
  for (int i = 0; i < N; ++i) t.p[lane + 32 * i] = TAIL ? v[i] : s == 0.f ? 0.f : v[i] / s;   // a list with no token left asks for nothing
  if (lane == 0) {
    t.sum = TAIL ? s : s == 0.f ? 0.f : s == s ? 1.f : NAN;
    t.rest = TAIL ? max_nan(0.f, 1.f - s) : 0.f;
  }
}

template <bool TAIL>
__device__ __forceinline__ Coef distill_coef(const DistillParams& p, const Teacher& t, float m, float ls, float lr, float w) {
  Coef c;
  c.k = p.scale * kLog2e;
  c.m = m;
  c.beta = 0.f;
  c.off_l = ls * kLog2e;
  c.alpha_l = w * p.scale * (t.sum + t.rest);
  if (TAIL) {
    const bool some = lr != -INFINITY;
    c.off = some ? lr * kLog2e : 0.f;
    c.alpha = some ? w * p.scale * ((t.sum + t.rest) * expf(lr - ls) - t.rest) : 0.f;
  } else {
    c.off = c.off_l;
    c.alpha = c.alpha_l;
  }
  c.zero = ls == -INFINITY || w == 0.f;
  return c;
}

// What a block of the cluster found in its part: the tokens off the list (all, without remainder) and those on it.
struct Found {
  Acc dense, listed;
};

// Rows are read once: every block of the cluster copies its part to shared memory, the blocks exchange their sums, and
// the gradient is computed from the copy.  A part that does not fit is taken in pieces and read again for the gradient.
template <int DT, bool TAIL>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams p) {
  using E = Elem<DT>;
  constexpr int VE = E::VE, T = kDistillThreads, U = 4;
  extern __shared__ uint4 held[];
  __shared__ Teacher t;
  __shared__ Warps8 buf[2];
  __shared__ Found found[kMaxSplit];
  __shared__ float red[kMaxList / 32];
  const int split = p.split, rank = split > 1 ? (int)ptx::cluster_ctarank() : 0, tid = threadIdx.x, n = p.list_k;
  const int64_t r = blockIdx.x / split;
  if (split > 1) ptx::cluster_arrive_relaxed();
  const Row<DT> in(p.logits, r, p.stride, p.vocab);
  const Part<DT> part(in, rank, split);
  const float k = p.scale * kLog2e;
  typename E::T* cells = reinterpret_cast<typename E::T*>(held);

  Sums<DT, false> sums(k);
  Acc listed;
  float zk = -INFINITY;   // the listed token's logit: of all tokens in the first block, of the part's own in the others
  int id = -1;
  bool first = false;     // not a repetition of an earlier entry
  for (int b0 = 0; b0 < part.n_all || b0 == 0; b0 += p.hold) {
    const int size = min(part.n_all - b0, p.hold);
    if (b0 > 0) __syncthreads();   // the previous piece has been read
    for (int i = tid; i < size; i += T) {
      if (b0 + i < part.n_int) copy_async(&held[i], in.at(part.w0 + b0 + i));
      else held[i] = part.raw(in, b0 + i);
    }
    if (b0 == 0) load_teacher<TAIL>(p, r, t);
    copy_async_wait();
    __syncthreads();
    if (b0 == 0 && tid < n) {
      id = t.list.id[tid];
      if (rank == 0 && id >= 0) zk = E::to(in.column(id));
      first = TAIL && id >= 0 && !repeated(t.list, n, tid, true);
    }
    bool here = id >= 0 && part.has(in.ph + id);
    int at = 0;
    if (here) {
      at = (part.place((in.ph + id) / VE) - b0) * VE + (in.ph + id) % VE;
      here = at >= 0 && at < size * VE;
    }
    if (here) {
      zk = E::to(cells[at]);
      if (first) listed.add_one(zk, k);
    }
    if (TAIL) {   // listed tokens leave the sum over the remainder
      __syncthreads();
      if (here) cells[at] = E::from(-INFINITY);
      __syncthreads();
    }
    for (int i = tid; i < size; i += T * U) {
      uint4 g[U];
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * T < size) {
          g[u] = held[i + u * T];
          mx = max_nan(mx, E::largest(g[u]));
        }
      sums.raise(mx);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * T < size) sums.add(g[u]);
    }
  }
  sums.flush();
  warp_share<false>(sums.a, k, buf[0]);
  if (TAIL) warp_share<false>(listed, k, buf[1]);
  __syncthreads();
  Acc dense = warps_join<false>(k, buf[0]);
  if (TAIL) listed = warps_join<false>(k, buf[1]);
  if (split > 1) {
    ptx::cluster_wait();   // all blocks have started
    if (tid < split) {
      const uint32_t to = ptx::mapa(ptx::smem_u32(&found[rank]), tid);
      ptx::st_shared_cluster_u32(to, __float_as_uint(dense.m));
      ptx::st_shared_cluster_u32(to + 4, __float_as_uint(dense.s));
      if (TAIL) {
        ptx::st_shared_cluster_u32(to + sizeof(Acc), __float_as_uint(listed.m));
        ptx::st_shared_cluster_u32(to + sizeof(Acc) + 4, __float_as_uint(listed.s));
      }
    }
    ptx::cluster_sync();
    dense = listed = Acc{};
    for (int i = 0; i < split; ++i) {
      dense.merge(Acc{found[i].dense.m, found[i].dense.s, 0.f}, k);
      if (TAIL) listed.merge(Acc{found[i].listed.m, found[i].listed.s, 0.f}, k);
    }
  }
  Acc all = dense;
  if (TAIL) all.merge(listed, k);
  const float ls = log_sum(all);
  const float lr = !TAIL ? 0.f : dense.s == 0.f ? -INFINITY : (dense.m - all.m) * p.scale + log_sum(dense);
  const float pk = id >= 0 ? t.p[tid] : 0.f;
  if (rank == 0 && tid < kMaxList) {
    float l = 0.f;
    if (!(pk == 0.f)) l = ls == -INFINITY && pk > 0.f ? INFINITY : pk * (logf(pk) - ((zk - all.m) * p.scale - ls));
    if (TAIL && tid == 0 && !(t.rest == 0.f)) {
      if (ls == -INFINITY && t.rest > 0.f) l = INFINITY;
      else if (!(lr == -INFINITY && t.rest < 1e-5f)) l += t.rest * (logf(t.rest) - (lr - ls));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
    if ((tid & 31) == 0) red[tid >> 5] = l;
  }
  if (p.dlogits) {
    const float w = p.weight ? p.weight[r] : 1.f;
    const Coef c = distill_coef<TAIL>(p, t, all.m, ls, lr, w);
    const Row<DT> out(p.dlogits, r, p.grad_stride, p.vocab);
    if (tid < n) t.list.add[tid] = -w * p.scale * pk;
    if (part.n_all > p.hold) {
      __syncthreads();
      grad_part<DT, false>(in, out, part, c, t.list, n);
    } else {
      const Dense<DT, false> of(c);
      const bool alike = in.ph == out.ph;
      for (int i = tid; i < part.n_all; i += T) {
        float x[VE];
        of(held[i], x);
        store_granule<DT>(in, out, part, alike, i, x);
      }
      __syncthreads();   // the dense part of the listed columns is written before what replaces it
      if (id >= 0 && part.has(in.ph + id) && !c.zero) out.column(id) = E::from(grad_of(zk, c) + add_of_column(t.list, n, tid));
    }
  } else {
    __syncthreads();
  }
  if (rank == 0 && tid == 0) {
    p.loss[r] = red[0] + red[1] + red[2] + red[3];
    if (p.stats) {
      p.stats[3 * r] = ls == -INFINITY ? -INFINITY : all.m;
      p.stats[3 * r + 1] = ls;
      p.stats[3 * r + 2] = ls == -INFINITY && TAIL ? -INFINITY : lr;
    }
  }
}

template <int DT, bool TAIL>
__global__ void __launch_bounds__(kDistillThreads) distill_grad_kernel(const DistillParams p) {
  __shared__ Teacher t;
  const int64_t r = blockIdx.x / p.split;
  const Row<DT> in(p.logits, r, p.stride, p.vocab), out(p.dlogits, r, p.grad_stride, p.vocab);
  load_teacher<TAIL>(p, r, t);
  __syncthreads();
  const float w = p.weight[r];
  const Coef c = distill_coef<TAIL>(p, t, p.stats[3 * r], p.stats[3 * r + 1], p.stats[3 * r + 2], w);
  if (threadIdx.x < kMaxList) t.list.add[threadIdx.x] = -w * p.scale * t.p[threadIdx.x];
  __syncthreads();
  grad_part<DT, false>(in, out, Part<DT>(in, blockIdx.x % p.split, p.split), c, t.list, p.list_k);
}

}  // namespace rows
}  // namespace iris

using namespace iris;
using namespace iris::rows;

namespace {

constexpr int kHoldBytes = 192 * 1024;   // of shared memory at most for a part
static int part_kb() { const char* e = getenv("PARTKB"); return e ? atoi(e) : 56; }
#define kPartBytes (part_kb() * 1024)
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

template <int DT, bool TAIL>
int launch_distill(DistillParams p, int64_t rows, cudaStream_t st) {
  static bool configured[kMaxDevices] = {};
  int dev = -1;
  IRIS_CUDA_TRY(cudaGetDevice(&dev));
  if (dev >= kMaxDevices || !configured[dev]) {
    IRIS_CUDA_TRY(cudaFuncSetAttribute(distill_kernel<DT, TAIL>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHoldBytes));
    if (dev < kMaxDevices) configured[dev] = true;
  }
  // A row is shared by a cluster of blocks until a part is at most kPartBytes, or while the rows alone leave SMs without
  // work and every thread still has a granule.
  const int64_t granules = (p.vocab + 2 * Row<DT>::VE - 2) / Row<DT>::VE;   // of a row, wherever it starts
  int split = 1;
  while (split < kMaxSplit && (granules * 16 > (int64_t)split * kPartBytes || (rows * split < 2 * kSms && granules >= (int64_t)split * 2 * kDistillThreads))) ++split;
  p.split = split;
  const int64_t need = std::max<int64_t>(1, (granules + split - 1) / split);
  p.hold = (int)std::min<int64_t>(need, kHoldBytes / 16);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(rows * split));
  cfg.blockDim = dim3(kDistillThreads);
  cfg.dynamicSmemBytes = (size_t)p.hold * 16;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)split;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = split > 1 ? 1 : 0;
  IRIS_CUDA_TRY(cudaLaunchKernelEx(&cfg, distill_kernel<DT, TAIL>, p));
  return IRIS_OK;
}

template <int DT, bool TAIL>
int launch_distill_grad(const DistillParams& p, int64_t rows, cudaStream_t st) {
  distill_grad_kernel<DT, TAIL><<<(unsigned)(rows * p.split), kDistillThreads, 0, st>>>(p);
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
  if (a->rows > INT32_MAX / kMaxSplit) return fail(IRIS_ERR_UNSUPPORTED, "%s: more than 2^28 rows", fn);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tail = a->mode == IRIS_DISTILL_TAIL;
  if (a->dtype == IRIS_BF16) return tail ? launch_distill<IRIS_BF16, true>(p, a->rows, st) : launch_distill<IRIS_BF16, false>(p, a->rows, st);
  if (a->dtype == IRIS_F16) return tail ? launch_distill<IRIS_F16, true>(p, a->rows, st) : launch_distill<IRIS_F16, false>(p, a->rows, st);
  return tail ? launch_distill<IRIS_F32, true>(p, a->rows, st) : launch_distill<IRIS_F32, false>(p, a->rows, st);
}

extern "C" int iris_distill_topk_backward(const iris_distill_args* a, void* stream) {
  const char* fn = "iris_distill_topk_backward";
  int64_t stride = 0, gstride = 0;
  IRIS_CHECK(check_distill(fn, a, &stride, &gstride));
  if (a->rows == 0 || a->vocab == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, true));
  IRIS_CHECK(check_aligned(fn, "weight", a->weight, 4, true));
  if (!a->dlogits) return fail(IRIS_ERR_ARG, "%s: dlogits is NULL", fn);
  DistillParams p = params_of(a, stride, gstride);
  p.split = grad_parts(a->vocab, a->dtype);
  if (a->rows * p.split > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 blocks", fn);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tail = a->mode == IRIS_DISTILL_TAIL;
  if (a->dtype == IRIS_BF16) return tail ? launch_distill_grad<IRIS_BF16, true>(p, a->rows, st) : launch_distill_grad<IRIS_BF16, false>(p, a->rows, st);
  if (a->dtype == IRIS_F16) return tail ? launch_distill_grad<IRIS_F16, true>(p, a->rows, st) : launch_distill_grad<IRIS_F16, false>(p, a->rows, st);
  return tail ? launch_distill_grad<IRIS_F32, true>(p, a->rows, st) : launch_distill_grad<IRIS_F32, false>(p, a->rows, st);
}
