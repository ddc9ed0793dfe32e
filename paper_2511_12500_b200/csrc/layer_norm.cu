// Layer norm over rows and its gradient.
//
//   mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), h = (x - mu) r;   y = h w + b
//   g = dy w:   dx = r (g - mean g - h mean(g h)),   dw = sum over rows dy h,   db = sum over rows dy
//
// A row is held in registers by a group of warps, 8 columns a thread and a few such runs, and where that is not enough by a cluster of blocks.
#include "any_rows.cuh"

namespace iris {
namespace rows {

constexpr int kNormRuns = 4, kNormGradRuns = 2;   // runs of 8 columns that a thread holds
constexpr int kNormWarps = 16;                  // of a block
constexpr int kNormSplit = 8;                   // blocks (one cluster) that share a row
constexpr int64_t kNormMaxDim = (int64_t)kNormGradRuns * kWarpColumns * kNormWarps * kNormSplit;

struct NormParams {
  const char* x;
  char* y;
  int64_t x_stride, y_stride;   // bytes
  const char *weight, *bias;
  float* stats;
  int64_t rows;
  int dim, warps, split;        // warps: of a row in one block
  float eps;
};

struct NormGradParams {
  const char *x, *dy;
  char* dx;
  int64_t x_stride, dy_stride, dx_stride;
  const char* weight;
  const float* stats;
  float* parts;                 // [blocks / split, 2, dim]: sums of dy h and of dy over a block's rows; nullptr: not wanted
  int64_t rows;
  int dim, warps, split;
};

// What a warp knows of a row, and the sum over the warps of a row, which all of its threads get.
struct NormShared {
  float2 of[2][kNormWarps * kNormSplit];   // twice: one is read while the next row's is written
};
struct Group {
  int warps, split, rank, index, warp, lane, id;   // index: of the group in its block; warp: in its row, over all blocks; id: of its barrier
  __device__ __forceinline__ Group(int warps_, int split_) : warps(warps_), split(split_) {
    rank = split > 1 ? (int)ptx::cluster_ctarank() : 0;
    lane = threadIdx.x & 31;
    index = (int)(threadIdx.x >> 5) / warps;
    warp = (int)(threadIdx.x >> 5) % warps + rank * warps;
    id = 1 + index;
  }
  // Every warp of the row puts its value into `turn`'s half and waits for the others'.
  __device__ __forceinline__ void exchange(NormShared& s, int turn, float2 v) const {
    if (split > 1) {
      if (lane < split) {
        const uint32_t to = ptx::mapa(ptx::smem_u32(&s.of[turn][warp]), lane);
        ptx::st_shared_cluster_u64(to, pair(v.x, v.y));
      }
      ptx::cluster_sync();
    } else {
      if (lane == 0) s.of[turn][index * warps + warp] = v;
      asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
    }
  }
  __device__ __forceinline__ int all() const { return warps * split; }
  __device__ __forceinline__ const float2* of(const NormShared& s, int turn) const { return s.of[turn] + (split > 1 ? 0 : index * warps); }
};
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  return x;
}

template <int DT, int PT, int I>
__global__ void __launch_bounds__(kNormWarps * 32) norm_kernel(const NormParams p) {
  using C = Columns<DT>;
  using W = Columns<PT>;
  __shared__ NormShared shared;
  const Group group(p.warps, p.split);
  const int64_t r = (int64_t)(blockIdx.x / p.split) * (blockDim.x / (p.warps * 32)) + group.index;
  const int begin = group.warp * I * kWarpColumns, first = begin + group.lane * kLaneColumns;
  ptx::let_next_begin();
  if (p.split > 1) ptx::cluster_sync();   // the others may write to this block's shared memory
  ptx::begin_after_previous();
  if (r >= p.rows) return;   // a whole group, and of one block only
  uint4 raw[I * C::N];
  C::template load<I>(p.x + r * p.x_stride, first, p.dim, raw);
  float x[I][kLaneColumns], sum = 0.f;
#pragma unroll
  for (int i = 0; i < I; ++i) {
    C::unpack(raw + i * C::N, x[i]);
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) sum += x[i][e];
  }
  // The warp's mean, and the squares' sum about it: nothing is lost where the mean is large.
  const int has = max(0, min(p.dim - begin, I * kWarpColumns));
  const float mine = has ? warp_sum(sum) / (float)has : 0.f;
  float squares = 0.f;
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) {
      const float d = first + i * kWarpColumns + e < p.dim ? x[i][e] - mine : 0.f;
      squares = fmaf(d, d, squares);
    }
  squares = warp_sum(squares);
  float mean = mine;
  if (group.all() > 1) {
    group.exchange(shared, 0, make_float2(mine, squares));
    const float2* const of = group.of(shared, 0);
    float s = 0.f, q = 0.f;
    for (int w = group.lane; w < group.all(); w += 32) {
      s = fmaf(of[w].x, (float)max(0, min(p.dim - w * I * kWarpColumns, I * kWarpColumns)), s);
    }
    mean = warp_sum(s) / (float)p.dim;
    for (int w = group.lane; w < group.all(); w += 32) {
      const float d = of[w].x - mean;
      q += fmaf(d * d, (float)max(0, min(p.dim - w * I * kWarpColumns, I * kWarpColumns)), of[w].y);
    }
    squares = warp_sum(q);
  }
  const float rstd = 1.f / sqrtf(squares / (float)p.dim + p.eps);
  if (p.stats && group.warp == 0 && group.lane == 0) {
    p.stats[2 * r] = mean;
    p.stats[2 * r + 1] = rstd;
  }
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) x[i][e] = (x[i][e] - mean) * rstd;
  if (p.weight) {
    uint4 v[I * W::N];
    W::template load<I>(p.weight, first, p.dim, v);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      float w[kLaneColumns];
      W::unpack(v + i * W::N, w);
#pragma unroll
      for (int e = 0; e < kLaneColumns; ++e) x[i][e] *= w[e];
    }
  }
  if (p.bias) {
    uint4 v[I * W::N];
    W::template load<I>(p.bias, first, p.dim, v);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      float w[kLaneColumns];
      W::unpack(v + i * W::N, w);
#pragma unroll
      for (int e = 0; e < kLaneColumns; ++e) x[i][e] += w[e];
    }
  }
#pragma unroll
  for (int i = 0; i < I; ++i) C::pack(x[i], raw + i * C::N);
  C::template store<I>(p.y + r * p.y_stride, first, p.dim, raw);
}

// A block's groups take rows in turn and add up dw and db of their columns in registers, in chains of at most kNormChain rows, then of such sums.
constexpr int kNormChain = 128;

template <int DT, int PT, int I>
__global__ void __launch_bounds__(kNormWarps * 32) norm_grad_kernel(const NormGradParams p) {
  using C = Columns<DT>;
  using W = Columns<PT>;
  __shared__ NormShared shared;
  extern __shared__ float sums[];   // [groups, 2, columns of the block]
  const Group group(p.warps, p.split);
  const int groups = blockDim.x / (p.warps * 32);
  const int begin = group.warp * I * kWarpColumns, first = begin + group.lane * kLaneColumns;
  const int64_t step = (int64_t)(gridDim.x / p.split) * groups;
  const int columns = p.warps * I * kWarpColumns;   // of the block
  float* const own = sums + group.index * 2 * columns + first - group.rank * columns;
  if (p.split > 1) ptx::cluster_sync();   // the others may write to this block's shared memory
  ptx::begin_after_previous();
  float dw[I][kLaneColumns] = {}, db[I][kLaneColumns] = {};
  const auto put = [&](bool more) {
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int e = 0; e < kLaneColumns; ++e) {
        float* const s = own + i * kWarpColumns + e;
        s[0] = more ? s[0] + dw[i][e] : dw[i][e];
        s[columns] = more ? s[columns] + db[i][e] : db[i][e];
        dw[i][e] = db[i][e] = 0.f;
      }
  };
  int turn = 0, chain = 0;
  bool more = false;
  for (int64_t r = (int64_t)(blockIdx.x / p.split) * groups + group.index; r < p.rows; r += step, turn ^= 1) {
    if (p.parts && chain++ == kNormChain) {
      put(more);
      more = true;
      chain = 1;
    }
    uint4 xr[I * C::N], gr[I * C::N];
    C::template load<I>(p.x + r * p.x_stride, first, p.dim, xr);
    C::template load<I>(p.dy + r * p.dy_stride, first, p.dim, gr);
    const float mean = p.stats[2 * r], rstd = p.stats[2 * r + 1];
    float h[I][kLaneColumns], g[I][kLaneColumns];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      C::unpack(xr + i * C::N, h[i]);
      C::unpack(gr + i * C::N, g[i]);
#pragma unroll
      for (int e = 0; e < kLaneColumns; ++e) {
        h[i][e] = (h[i][e] - mean) * rstd;
        dw[i][e] = fmaf(g[i][e], h[i][e], dw[i][e]);
        db[i][e] += g[i][e];
      }
    }
    if (!p.dx) continue;
    if (p.weight) {
      uint4 v[I * W::N];
      W::template load<I>(p.weight, first, p.dim, v);
#pragma unroll
      for (int i = 0; i < I; ++i) {
        float w[kLaneColumns];
        W::unpack(v + i * W::N, w);
#pragma unroll
        for (int e = 0; e < kLaneColumns; ++e) g[i][e] *= w[e];
      }
    }
    float a = 0.f, b = 0.f;   // dy is 0 behind the row's end
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int e = 0; e < kLaneColumns; ++e) {
        a += g[i][e];
        b = fmaf(g[i][e], h[i][e], b);
      }
    a = warp_sum(a);
    b = warp_sum(b);
    if (group.all() > 1) {
      group.exchange(shared, turn, make_float2(a, b));
      const float2* const of = group.of(shared, turn);
      a = b = 0.f;
      for (int w = group.lane; w < group.all(); w += 32) {
        a += of[w].x;
        b += of[w].y;
      }
      a = warp_sum(a);
      b = warp_sum(b);
    }
    a /= (float)p.dim;
    b /= (float)p.dim;
#pragma unroll
    for (int i = 0; i < I; ++i) {
#pragma unroll
      for (int e = 0; e < kLaneColumns; ++e) g[i][e] = (g[i][e] - a - h[i][e] * b) * rstd;
      C::pack(g[i], xr + i * C::N);
    }
    C::template store<I>(p.dx + r * p.dx_stride, first, p.dim, xr);
  }
  if (!p.parts) return;
  put(more);
  __syncthreads();
  float* const to = p.parts + (int64_t)(blockIdx.x / p.split) * 2 * p.dim;
  for (int c = threadIdx.x; c < columns; c += blockDim.x) {
    const int column = group.rank * columns + c;
    if (column >= p.dim) continue;
    float w = sums[c], b = sums[columns + c];
    for (int q = 1; q < groups; ++q) {
      w += sums[q * 2 * columns + c];
      b += sums[(q * 2 + 1) * columns + c];
    }
    to[column] = w;
    to[p.dim + column] = b;
  }
}

// dw and db: the sums of `n` parts.  32 columns a block, its warps take parts in turn.
struct NormJoinParams {
  const float* parts;
  int n, dim;
  void* out[2];
};
template <int PT>
__global__ void __launch_bounds__(512) norm_join_kernel(const NormJoinParams p) {
  __shared__ float s[16][32];
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.x & 1, c = (blockIdx.x >> 1) * 32 + lane;
  void* const out = which ? p.out[1] : p.out[0];
  if (!out) return;
  float sum = 0.f;
  if (c < p.dim)
    for (int i = warp; i < p.n; i += 16) sum += p.parts[((int64_t)2 * i + which) * p.dim + c];
  s[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && c < p.dim) {
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) all += s[w][lane];
    static_cast<typename Elem<PT>::T*>(out)[c] = Elem<PT>::from(all);
  }
}

// ---- host side -----------------------------------------------------------------------------------------------------
struct NormPlan {
  int split, warps, runs, groups;
};
static NormPlan norm_plan(int64_t dim, int most) {   // most: runs that a thread can hold
  NormPlan n;
  n.split = 1;
  while ((int64_t)n.split * most * kWarpColumns * kNormWarps < dim) n.split *= 2;
  const int runs = (int)((dim + (int64_t)n.split * kWarpColumns - 1) / ((int64_t)n.split * kWarpColumns));   // of 256 columns in a block
  n.warps = (runs + most - 1) / most;
  n.runs = (runs + n.warps - 1) / n.warps;
  n.groups = n.split > 1 ? 1 : kNormWarps / n.warps;
  return n;
}
static int64_t norm_grad_blocks(const NormPlan& n, int64_t rows) {   // times split
  const int64_t full = (rows + n.groups - 1) / n.groups, room = kSms / n.split;
  return full < room ? full : room;
}

template <int DT, int PT>
static int launch_norm(const NormParams& p, const NormPlan& n, cudaStream_t st) {
  void (*const kernels[kNormRuns])(NormParams) = {norm_kernel<DT, PT, 1>, norm_kernel<DT, PT, 2>, norm_kernel<DT, PT, 3>, norm_kernel<DT, PT, 4>};
  const int64_t blocks = (p.rows + n.groups - 1) / n.groups * n.split;
  if (blocks > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "iris_layer_norm: more than 2^31 - 1 blocks");
  return launch_rows(kernels[n.runs - 1], p, (unsigned)blocks, n.split, n.warps * n.groups * 32, 0, st);
}
template <int DT, int PT, int I>
static int launch_norm_grad(const NormGradParams& p, const NormPlan& n, int64_t blocks, cudaStream_t st) {
  constexpr auto kernel = norm_grad_kernel<DT, PT, I>;
  const size_t bytes = p.parts ? (size_t)2 * n.groups * n.warps * I * kWarpColumns * sizeof(float) : 0;
  if (bytes > 48 * 1024) IRIS_CHECK(allow_shared<kernel>(2 * kNormWarps * I * kWarpColumns * (int)sizeof(float)));
  return launch_rows(kernel, p, (unsigned)(blocks * n.split), n.split, n.warps * n.groups * 32, bytes, st);
}
template <int DT, int PT>
static int launch_norm_grad(const NormGradParams& p, const NormPlan& n, void* dweight, void* dbias, cudaStream_t st) {
  int64_t blocks = norm_grad_blocks(n, p.rows);
  IRIS_CHECK(n.runs == 1 ? launch_norm_grad<DT, PT, 1>(p, n, blocks, st) : launch_norm_grad<DT, PT, 2>(p, n, blocks, st));
  if (!p.parts) return IRIS_OK;
  return launch_rows(norm_join_kernel<PT>, NormJoinParams{p.parts, (int)blocks, p.dim, {dweight, dbias}}, (unsigned)((p.dim + 31) / 32 * 2), 1, 512, 0, st);
}

static int check_norm(const char* fn, int64_t rows, int64_t dim, int dtype, int param_dtype) {
  if (dtype != IRIS_F16 && dtype != IRIS_BF16 && dtype != IRIS_F32) return fail(IRIS_ERR_ARG, "%s: unknown dtype %d", fn, dtype);
  if (param_dtype != IRIS_F32 && param_dtype != dtype) return fail(IRIS_ERR_ARG, "%s: param_dtype %d is neither fp32 nor the rows' type", fn, param_dtype);
  if (rows < 0 || dim < 1) return fail(IRIS_ERR_ARG, "%s: rows=%lld, dim=%lld", fn, (long long)rows, (long long)dim);
  if (dim > kNormMaxDim || rows > INT32_MAX)
    return fail(IRIS_ERR_UNSUPPORTED, "%s: at most 2^31 - 1 rows of %lld columns", fn, (long long)kNormMaxDim);
  return IRIS_OK;
}
static int check_params(const char* fn, const char* what, const void* p, int param_dtype, bool needed) {
  return check_aligned(fn, what, p, elem_size(param_dtype), needed);
}

}  // namespace rows
}  // namespace iris

using namespace iris;
using namespace iris::rows;

extern "C" int iris_layer_norm(const iris_layer_norm_args* a, void* stream) {
  const char* fn = "iris_layer_norm";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  IRIS_CHECK(check_norm(fn, a->rows, a->dim, a->dtype, a->param_dtype));
  int64_t xs = a->row_stride, ys = a->out_stride;
  IRIS_CHECK(check_matrix(fn, "x", a->x, a->dtype, a->rows, a->dim, &xs));
  IRIS_CHECK(check_matrix(fn, "y", a->y, a->dtype, a->rows, a->dim, &ys));
  IRIS_CHECK(check_params(fn, "weight", a->weight, a->param_dtype, false));
  IRIS_CHECK(check_params(fn, "bias", a->bias, a->param_dtype, false));
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, false));
  if (!(a->eps >= 0.f) || std::isinf(a->eps)) return fail(IRIS_ERR_ARG, "%s: eps has to be finite and not negative", fn);
  IRIS_CHECK(check_overlap(fn, "y", "x", a->x, xs, a->y, ys, a->rows, a->dim, a->dtype));
  if (a->rows == 0) return IRIS_OK;
  const int64_t es = (int64_t)elem_size(a->dtype);
  const NormPlan n = norm_plan(a->dim, kNormRuns);
  NormParams p{static_cast<const char*>(a->x), static_cast<char*>(a->y), xs * es, ys * es, static_cast<const char*>(a->weight),
               static_cast<const char*>(a->bias), a->stats, a->rows, (int)a->dim, n.warps, n.split, a->eps};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = a->param_dtype == IRIS_F32;
  if (a->dtype == IRIS_BF16) return wide ? launch_norm<IRIS_BF16, IRIS_F32>(p, n, st) : launch_norm<IRIS_BF16, IRIS_BF16>(p, n, st);
  if (a->dtype == IRIS_F16) return wide ? launch_norm<IRIS_F16, IRIS_F32>(p, n, st) : launch_norm<IRIS_F16, IRIS_F16>(p, n, st);
  return launch_norm<IRIS_F32, IRIS_F32>(p, n, st);
}

extern "C" size_t iris_layer_norm_workspace_bytes(int64_t rows, int64_t dim) {
  if (rows <= 0 || dim <= 0 || dim > kNormMaxDim) return 0;
  return (size_t)norm_grad_blocks(norm_plan(dim, kNormGradRuns), rows) * 2 * dim * sizeof(float);
}

extern "C" int iris_layer_norm_backward(const iris_layer_norm_grad_args* a, void* stream) {
  const char* fn = "iris_layer_norm_backward";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  IRIS_CHECK(check_norm(fn, a->rows, a->dim, a->dtype, a->param_dtype));
  int64_t xs = a->row_stride, gs = a->dy_stride, ds = a->dx_stride;
  IRIS_CHECK(check_matrix(fn, "x", a->x, a->dtype, a->rows, a->dim, &xs));
  IRIS_CHECK(check_matrix(fn, "dy", a->dy, a->dtype, a->rows, a->dim, &gs));
  if (a->dx) {
    IRIS_CHECK(check_matrix(fn, "dx", a->dx, a->dtype, a->rows, a->dim, &ds));
    IRIS_CHECK(check_overlap(fn, "dx", "x", a->x, xs, a->dx, ds, a->rows, a->dim, a->dtype));
    IRIS_CHECK(check_overlap(fn, "dx", "dy", a->dy, gs, a->dx, ds, a->rows, a->dim, a->dtype));
  }
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, a->rows > 0));
  IRIS_CHECK(check_params(fn, "weight", a->weight, a->param_dtype, false));
  IRIS_CHECK(check_params(fn, "dweight", a->dweight, a->param_dtype, false));
  IRIS_CHECK(check_params(fn, "dbias", a->dbias, a->param_dtype, false));
  const bool sums = a->dweight || a->dbias;
  const size_t need = iris_layer_norm_workspace_bytes(a->rows, a->dim);
  if (sums && need) {
    IRIS_CHECK(check_aligned(fn, "workspace", a->workspace, 16, true));
    if (a->workspace_bytes < need) return fail(IRIS_ERR_ARG, "%s: workspace has %zu bytes, the call needs %zu", fn, a->workspace_bytes, need);
  }
  if (!sums && !a->dx) return IRIS_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->rows == 0) {   // sums of nothing
    for (void* d : {a->dweight, a->dbias})
      if (d) IRIS_CUDA_TRY(cudaMemsetAsync(d, 0, a->dim * elem_size(a->param_dtype), st));
    return IRIS_OK;
  }
  const int64_t es = (int64_t)elem_size(a->dtype);
  const NormPlan n = norm_plan(a->dim, kNormGradRuns);
  NormGradParams p{static_cast<const char*>(a->x), static_cast<const char*>(a->dy), static_cast<char*>(a->dx), xs * es, gs * es, ds * es,
                   static_cast<const char*>(a->weight), a->stats, sums ? static_cast<float*>(a->workspace) : nullptr, a->rows, (int)a->dim, n.warps,
                   n.split};
  const bool wide = a->param_dtype == IRIS_F32;
  if (a->dtype == IRIS_BF16)
    return wide ? launch_norm_grad<IRIS_BF16, IRIS_F32>(p, n, a->dweight, a->dbias, st) : launch_norm_grad<IRIS_BF16, IRIS_BF16>(p, n, a->dweight, a->dbias, st);
  if (a->dtype == IRIS_F16)
    return wide ? launch_norm_grad<IRIS_F16, IRIS_F32>(p, n, a->dweight, a->dbias, st) : launch_norm_grad<IRIS_F16, IRIS_F16>(p, n, a->dweight, a->dbias, st);
  return launch_norm_grad<IRIS_F32, IRIS_F32>(p, n, a->dweight, a->dbias, st);
}
