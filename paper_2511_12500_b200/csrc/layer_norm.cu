// Layer norm over rows and its gradient.
//
//   mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), h = (x - mu) r;   y = h w + b
//   g = dy w:   dx = r (g - mean g - h mean(g h)),   dw = sum over rows dy h,   db = sum over rows dy
//
// A row is held in registers by a group of warps, 8 columns a thread and a few such runs, and where that is not enough by a cluster of blocks.
// Blocks stay and take rows in turn; the next ones are under way to shared memory meanwhile.
#include "any_rows.cuh"
#include "norm_rows.h"

namespace iris {
namespace rows {

constexpr int kNormRuns = 4, kNormGradRuns = 2;   // runs of 8 columns that a thread holds, of one row or of several short ones
constexpr int kNormRowWarps = 8, kNormGradRowWarps = 16;   // of a row in a block, at most
constexpr int kNormSplitGroups = 4;             // of a block in a cluster, at most (a row has 5 of the block's 16 warps or more)
constexpr int kNormSplit = 8;                   // blocks (one cluster) that share a row
constexpr int64_t kNormMaxDim = (int64_t)kNormRuns * kWarpColumns * kNormRowWarps * kNormSplit;
static_assert(kNormRuns * kNormRowWarps == kNormGradRuns * kNormGradRowWarps, "the same limit for both directions");
constexpr int kNormRows = 2;                    // that several warps have at a time, at most
// Warps of a block, which has an SM to itself, and rows (or R of them) in shared memory: what registers and shared memory allow.
constexpr int norm_warps(int dtype, int rows_runs) { return dtype == IRIS_F32 || rows_runs > 4 ? 16 : 24; }
constexpr int norm_stages(int dtype, int rows_runs) { return dtype == IRIS_F32 || rows_runs > 4 ? 2 : 3; }
constexpr int norm_grad_warps(int rows_runs) { return rows_runs > 2 ? 12 : 16; }
constexpr int norm_grad_stages(int dtype) { return dtype == IRIS_F32 ? 2 : 3; }
// Another block's values are taken for lost after so many looks, of 4 us at most each (a second in all; looks are counted, as a clock runs on while the kernel is
// off the GPU).  sends: to how many blocks a warp sends its values.
struct NormPatience {
  uint32_t looks, sends;
};
constexpr uint32_t kNormLooks = 1 << 18;
__device__ int32_t norm_status[kStatusWords];   // the first wait that ran out on the device, as the status block of a heap has it
constexpr int kNormChain = 128;                 // rows that a thread adds up before the sum goes to the sum of such sums

// How rows lie: all at 16 bytes, and their lengths multiples of that; those of all matrices alike, at any places of 16 bytes; anyhow.
enum { kAny, kAligned, kSame };

struct NormParams {
  const char* x;
  char* y;
  int64_t x_stride, y_stride;   // bytes
  const char *weight, *bias;
  float* stats;
  int64_t rows;
  int dim, warps, split;        // warps: of a row in one block
  int period;                   // kSame: rows that far apart begin at the same place of 16 bytes
  float eps;
  NormPatience patience;
};

struct NormGradParams {
  const char *x, *dy;
  char* dx;
  int64_t x_stride, dy_stride, dx_stride;
  const char* weight;
  const float* stats;
  float* parts;                 // [blocks / split (times groups if by_group), 2, dim]: sums of dy h and of dy; nullptr: not wanted
  int64_t rows;
  int dim, warps, split, period, by_group;   // by_group: of norm_by_group
  NormPatience patience;
};

// What a warp knows of a row, and the sum over the warps of a row, which all of its threads get.
struct NormShared {
  uint64_t arrived[kNormSplitGroups][2];   // of a group's values in a cluster, one for each half
  int lost[kNormGradRowWarps];             // of a warp: its wait has run out
  float2 of[2][kNormRows][kNormGradRowWarps * kNormSplit];   // twice: one is read while the next rows' is written
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
  // Before the first exchange; all blocks of the cluster.
  template <int R>
  __device__ __forceinline__ void prepare(NormShared& s) const {
    if (split == 1) return;
    if (lane == 0) s.lost[threadIdx.x >> 5] = 0;
    if (warp == rank * warps && lane == 0) {
      for (int h = 0; h < 2; ++h) {
        ptx::mbar_init(ptx::smem_u32(&s.arrived[index][h]), 1);
        ptx::mbar_arrive_expect_tx(ptx::smem_u32(&s.arrived[index][h]), all() * R * 8);
      }
      ptx::fence_mbar_init();
    }
    ptx::cluster_sync();
  }
  // The last thing a block does: the others may still write to its shared memory.
  __device__ __forceinline__ void finish() const {
    __syncwarp();
    if (split > 1) ptx::cluster_sync();
  }
  // In the end: a wait that ran out is recorded.  Values may still be on their way to this block, which is to outlive them: about a second.
  __device__ __forceinline__ void report_lost(const NormShared& s) const {
    __syncwarp();
    if (!*reinterpret_cast<const volatile int*>(&s.lost[threadIdx.x >> 5])) return;
    if (lane == 0) report_timeout(norm_status, KID_NORM, index, warp, 0, 0);
#pragma unroll 1
    for (int i = 0; i < 1000000; ++i) __nanosleep(1000);
  }
  // Every warp of the rows puts its values into a half of the shared memory (the halves in turn) and waits for the others'.  `lost` becomes NaN, and stays it,
  // for a thread that has not seen them come: its columns are NaN from then on.  It sends nothing more and prepares nothing, so that the others give up in turn
  // and no mbarrier is used out of step.
  //
  // In a cluster the values count themselves on the mbarrier of the block that they go to.  A barrier of the cluster would wait for
  // the stores of the row before as well.  A warp writes to a half again when all values of the exchange after have come, which each warp
  // sends when it has read that half; for the same reason one thread may prepare the mbarrier for its next use as soon as it has seen the values come.
  template <int R>
  __device__ __forceinline__ void exchange(NormShared& s, uint32_t count, const float (&a)[R], const float (&b)[R], float& lost, const NormPatience& patience) const {
    static_assert(R <= kNormRows, "room for them");
    const uint32_t turn = count & 1;
    if (split > 1) {
      const uint32_t bar = ptx::smem_u32(&s.arrived[index][turn]), parity = count >> 1 & 1;
      if (lane < patience.sends && lost == 0.f) {
#pragma unroll
        for (int q = 0; q < R; ++q) ptx::st_async_u64(ptx::mapa(ptx::smem_u32(&s.of[turn][q][index * all() + warp]), lane), pair(a[q], b[q]), ptx::mapa(bar, lane));
      }
      if (!ptx::mbar_try_wait_cluster(bar, parity)) {
        uint32_t looks = 1;
        while (lost == 0.f && !ptx::mbar_try_wait_cluster(bar, parity))
          if (++looks >= patience.looks) {
            lost = NAN;
            *reinterpret_cast<volatile int*>(&s.lost[threadIdx.x >> 5]) = 1;
          }
      }
      __syncwarp();
      if (warp == rank * warps && lane == 0 && lost == 0.f) ptx::mbar_arrive_expect_tx(bar, all() * R * 8);
    } else {
      if (lane == 0) {
#pragma unroll
        for (int q = 0; q < R; ++q) s.of[turn][q][index * warps + warp] = make_float2(a[q], b[q]);
      }
      asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
    }
  }
  __device__ __forceinline__ int all() const { return warps * split; }
  __device__ __forceinline__ const float2* of(const NormShared& s, int turn, int q) const { return s.of[turn][q] + index * all(); }
};

// How the columns of a row are shared by its warps: `each` a warp, `rest` in the last one that has any, of which the first has `none` that are not the row's.
struct Shares {
  int last;
  float each, rest, none, dim;
  __device__ __forceinline__ Shares(int each_, int dim_, int none_) {
    last = (dim_ - 1) / each_;
    each = (float)each_;
    rest = (float)(dim_ - last * each_);
    none = (float)none_;
    dim = (float)(dim_ - none_);
  }
  __device__ __forceinline__ float of(int warp) const { return (warp < last ? each : warp == last ? rest : 0.f) - (warp == 0 ? none : 0.f); }
};
// The rows of a group.  SAME (mode kSame): those of a block begin at the same place of 16 bytes (`ph`, in bytes).  Columns are then counted from there, `none`
// are not the row's, and rows are addressed so.
struct Rows : NormWalk {
  int ph, none;
  template <bool SAME, int R>
  static __device__ __forceinline__ Rows of(const Group& group, int groups, int period_, const char* base, int64_t stride, int es) {
    const int64_t block = blockIdx.x / group.split, blocks = gridDim.x / group.split, period = SAME ? period_ : 1, set = norm_set(block, period);
    Rows r;
    static_cast<NormWalk&>(r) = norm_walk(block, blocks, group.index, groups, period, set, R);
    r.ph = SAME ? (int)phase(base + set * stride) : 0;
    r.none = r.ph / es;
    return r;
  }
};
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
  return x;
}

// A vector of parameters in shared memory, in 32 bits, so that a thread's columns of run i are two accesses of 16 bytes side by side with the other
// threads': [runs of the block, 2, 32 threads, 4].  `none`: what stands for a vector that is not there.
template <int PT, int I>
__device__ __forceinline__ void put_params(float* to, const char* from, float none, const Group& group, int begin, int dim) {
  if (group.index) return;   // the other groups have the same columns
#pragma unroll 1
  for (int i = 0; i < I; ++i) {
    float x[kLaneColumns];
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) x[e] = none;
    if (from) Columns<PT>::load(from, begin + group.lane * kLaneColumns + i * kWarpColumns, dim, x);
    float4* const at = reinterpret_cast<float4*>(to) + ((group.warp - group.rank * group.warps) * I + i) * 64 + group.lane;
    at[0] = make_float4(x[0], x[1], x[2], x[3]);
    at[32] = make_float4(x[4], x[5], x[6], x[7]);
  }
}
// `at`: of the thread's run 0.
__device__ __forceinline__ void get_params(uint32_t at, int i, uint64_t (&x)[kLaneColumns / 2]) {
  const uint4 a = ld_shared_v4(at + i * 1024), b = ld_shared_v4(at + i * 1024 + 512);
  x[0] = (uint64_t)a.y << 32 | a.x;
  x[1] = (uint64_t)a.w << 32 | a.z;
  x[2] = (uint64_t)b.y << 32 | b.x;
  x[3] = (uint64_t)b.w << 32 | b.z;
}
__device__ __forceinline__ float both(uint64_t x) {
  const float2 f = unpair(x);
  return f.x + f.y;
}

// R rows at a time.
//
// Statistics in one exchange among a row's warps: each sums the squares about its own mean, and means and squares' sums are joined (squares of the differences
// of means, weighted by columns, come on top).  Long rows are read once and written once: 32768 x 4096 bf16 102 us, 5.2 TB/s.  With rows fetched ahead to
// shared memory nothing waits for memory long (1.0 warps an issue); what is left is chains of dependent instructions, shuffles and barriers at 16 warps an SM, so
// the rows in work count: 4104 columns, whose fifth warp has 8 of them, take 69 us for 16001 rows, 4096 columns 52; rows of 4096 that begin at
// any element 90.  Held in registers one row ahead instead of copied ahead: 244; parameters read from L1 instead of shared memory: 212; one row at a time 110.
// Rows of more than 8192 columns are shared by a cluster (SPLIT): 4096 x 16384 77 us, 1024 x 65536 91; 111 the former with a cluster's barrier in every turn and one group of 8 warps a block.
template <int DT, int PT, int R, int I, int MODE, bool SPLIT>
__global__ void __launch_bounds__(norm_warps(DT, R * I) * 32) norm_kernel(const NormParams p) {
  using C = Columns<DT>;
  using G = Segment<DT, I, MODE == kAligned>;
  using A = Aligned<DT, I>;
  constexpr bool SAME = MODE == kSame;
  constexpr int kStages = norm_stages(DT, R * I), H = kLaneColumns / 2;
  __shared__ NormShared shared;
  extern __shared__ __align__(16) char ring[];   // [warps, stages, R] segments; weight, bias
  const Group group(p.warps, SPLIT ? p.split : 1);
  const int groups = blockDim.x / (p.warps * 32);
  const int begin = group.warp * G::kColumns;
  const uint32_t own = ptx::smem_u32(ring) + (threadIdx.x >> 5) * (kStages * R * G::kBytes);
  float* const params = reinterpret_cast<float*>(ring + (blockDim.x >> 5) * (kStages * R * G::kBytes));
  const int columns = p.warps * G::kColumns;   // of the block
  const uint32_t weight = ptx::smem_u32(params) + ((group.warp - group.rank * group.warps) * I * 64 + group.lane) * 16, bias = weight + columns * 4;
  const Rows rows = Rows::of<SAME, R>(group, groups, p.period, p.x, p.x_stride, C::ES);
  const int dim = p.dim + rows.none, first = begin + group.lane * kLaneColumns;   // counted as rows are
  group.prepare<R <= kNormRows ? R : 1>(shared);
  ptx::let_next_begin();
  ptx::begin_after_previous();
  typename G::Lone lone[R];
  const auto fetch = [&](int64_t r, const char* from, int stage) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      lone[q].settle();
      if (r + q * rows.each < p.rows) {
        const uint32_t to = own + (stage * R + q) * G::kBytes;
        if constexpr (SAME) A::fetch(to, from + q * rows.each * p.x_stride, begin, dim, rows.ph, r + q * rows.each == 0, r + q * rows.each == p.rows - 1, lone[q]);
        else G::fetch(to, from + q * rows.each * p.x_stride, begin, dim, lone[q]);
      }
    }
    copy_async_commit();
  };
  int64_t r = rows.first;
  const char* x_row = p.x + r * p.x_stride - rows.ph;
  char* y_row = p.y + r * p.y_stride - rows.ph;
  const int64_t x_step = rows.step * p.x_stride, y_step = rows.step * p.y_stride;
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) fetch(r + k * rows.step, x_row + k * x_step, k);
  put_params<PT, I>(params, p.weight, 1.f, group, begin - rows.none, p.dim);
  put_params<PT, I>(params + columns, p.bias, 0.f, group, begin - rows.none, p.dim);
  __syncthreads();
  const Shares shares(G::kColumns, dim, rows.none);
  const float mine = fmaxf(shares.of(group.warp), 1.f), whole = 1.f / shares.dim;
  const bool full = begin >= rows.none && begin + G::kColumns <= dim;
  int stage = 0;
  float lost = 0.f;
  for (uint32_t count = 0; r < p.rows; r += rows.step, x_row += x_step, y_row += y_step, ++count) {
#pragma unroll
    for (int q = 0; q < R; ++q) lone[q].settle();
    copy_async_wait_but<kStages - 2>();
    __syncwarp();
    const uint32_t here = own + stage * (R * G::kBytes);
    fetch(r + (kStages - 1) * rows.step, x_row + (kStages - 1) * x_step, stage == 0 ? kStages - 1 : stage - 1);   // where the row before was
    stage = stage + 1 == kStages ? 0 : stage + 1;
    uint64_t x[R][I][H];
    float mean[R], squares[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      uint64_t s = 0;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        if constexpr (SAME) A::read(here + q * G::kBytes, begin, dim, rows.ph, i, x[q][i]);
        else G::read(here + q * G::kBytes, x_row + q * rows.each * p.x_stride, begin, dim, i, x[q][i]);
#pragma unroll
        for (int e = 0; e < H; ++e) s = add2f(s, x[q][i][e]);
      }
      mean[q] = both(s);
    }
    // The warp's mean, and the squares' sum about it: nothing is lost where the mean is large.  A quotient, so that the mean of equal small whole
    // numbers is that number.
#pragma unroll
    for (int q = 0; q < R; ++q) mean[q] = warp_sum(mean[q]) / mine;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const uint64_t minus = pair(-mean[q], -mean[q]);
      uint64_t s = 0;
      if (full) {
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
          for (int e = 0; e < H; ++e) {
            const uint64_t d = add2f(x[q][i][e], minus);
            s = fma2f(d, d, s);
          }
      } else {   // columns that are not the row's do not count
#pragma unroll
        for (int i = 0; i < I; ++i) {
          uint64_t t = 0;
#pragma unroll
          for (int e = 0; e < H; ++e) {
            const uint64_t d = add2f(x[q][i][e], minus);
            t = fma2f(d, d, t);
          }
          const int c = first + i * kWarpColumns;
          if (c < rows.none || c + kLaneColumns > dim) {   // few threads
            t = 0;
            if (c < dim)
#pragma unroll
              for (int e = 0; e < H; ++e) {
                const float2 d = unpair(add2f(x[q][i][e], minus));
                const uint64_t there = pair(c + 2 * e >= rows.none && c + 2 * e < dim ? d.x : 0.f, c + 2 * e + 1 >= rows.none && c + 2 * e + 1 < dim ? d.y : 0.f);
                t = fma2f(there, there, t);
              }
          }
          s = add2f(s, t);
        }
      }
      squares[q] = both(s);
    }
#pragma unroll
    for (int q = 0; q < R; ++q) squares[q] = warp_sum(squares[q]);
    if constexpr (R <= kNormRows)
      if (group.all() > 1) {
        group.exchange(shared, count, mean, squares, lost, p.patience);
#pragma unroll
        for (int q = 0; q < R; ++q) {
          const float2* const of = group.of(shared, count & 1, q);
          float m = lost, s = 0.f;
          if (SPLIT && group.all() > 16) {   // a lane takes a warp, or a few (1024 x 65536, with one group a block: 200 us instead of 367; at 16 warps the same within 5 %)
            for (int w = group.lane; w < group.all(); w += 32) m = fmaf(of[w].x, shares.of(w), m);
            mean[q] = warp_sum(m) / shares.dim;
            for (int w = group.lane; w < group.all(); w += 32) {
              const float2 v = of[w];
              const float d = v.x - mean[q];
              s += fmaf(d * d, shares.of(w), v.y);
            }
            squares[q] = warp_sum(s);
            continue;
          }
#pragma unroll 4
          for (int w = 0; w < group.all(); ++w) m = fmaf(of[w].x, shares.of(w), m);
          mean[q] = m / shares.dim;
#pragma unroll 4
          for (int w = 0; w < group.all(); ++w) {   // from the warp's mean to the row's
            const float2 v = of[w];
            const float d = v.x - mean[q];
            s += fmaf(d * d, shares.of(w), v.y);
          }
          squares[q] = s;
        }
      }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      squares[q] = rsqrtf(fmaf(squares[q], whole, p.eps));
      if (p.stats && group.warp == 0 && group.lane == 0 && r + q * rows.each < p.rows)
        *reinterpret_cast<float2*>(p.stats + 2 * (r + q * rows.each)) = make_float2(mean[q], squares[q]);
    }
#pragma unroll
    for (int i = 0; i < I; ++i) {
      uint64_t w[H], b[H];
      get_params(weight, i, w);
      get_params(bias, i, b);
#pragma unroll
      for (int q = 0; q < R; ++q)
#pragma unroll
        for (int e = 0; e < H; ++e) x[q][i][e] = fma2f(mul2f(add2f(x[q][i][e], pair(-mean[q], -mean[q])), pair(squares[q], squares[q])), w[e], b[e]);
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (r + q * rows.each >= p.rows) break;
      uint4 out[I * C::N];
#pragma unroll
      for (int i = 0; i < I; ++i) C::pack2(x[q][i], out + i * C::N);
      if constexpr (SAME) A::write(y_row + q * rows.each * p.y_stride, begin, dim, rows.ph, out);
      else G::write(here + q * G::kBytes, y_row + q * rows.each * p.y_stride, begin, dim, out);
    }
  }
  if (SPLIT) group.report_lost(shared);
  group.finish();
}

// A block's groups add up dw and db of their columns in registers, so blocks stay and a thread has the same columns of every row.  R rows at a time.
//
// 16384 x 4096 bf16: 78 us and 6 for norm_join_kernel, 4.8 TB/s together; issue slots 58 %, bound like norm_kernel by dependent instructions at the 16 warps that
// the sums' registers allow (32 of 128).  5003 x 2563 fp16, rows at any element: 33 us; a third of that goes by before the first rows are there and
// after the last ones (50030 rows: 253 us).  Held for 1024 columns a warp instead of 512, 8 warps: 87 us; x and dy read twice instead of held: 86, 32-bit rows
// 257 instead of 161.
template <int DT, int R, int I>
constexpr int norm_grad_stage_bytes() { return R * (2 * Segment<DT, I>::kBytes + 16); }   // x, dy, statistics

template <int DT, int PT, int R, int I, int MODE, bool SPLIT>
__global__ void __launch_bounds__(norm_grad_warps(R * I) * 32) norm_grad_kernel(const NormGradParams p) {
  using C = Columns<DT>;
  using G = Segment<DT, I, MODE == kAligned>;
  using A = Aligned<DT, I>;
  constexpr bool SAME = MODE == kSame;
  constexpr int kStages = norm_grad_stages(DT), kRow = 2 * G::kBytes + 16, kStage = norm_grad_stage_bytes<DT, R, I>(), H = kLaneColumns / 2;
  __shared__ NormShared shared;
  extern __shared__ __align__(16) char ring[];   // [warps, stages, R] segments of x, of dy, statistics; weight
  const Group group(p.warps, SPLIT ? p.split : 1);
  const int groups = blockDim.x / (p.warps * 32);
  const int begin = group.warp * G::kColumns, first = begin + group.lane * kLaneColumns;
  const int columns = p.warps * G::kColumns;   // of the block
  const Rows rows = Rows::of<SAME, R>(group, groups, p.period, p.x, p.x_stride, C::ES);
  const int dim = p.dim + rows.none;   // counted as rows are, like `first`
  const uint32_t own = ptx::smem_u32(ring) + (threadIdx.x >> 5) * (kStages * kStage);
  float* const params = reinterpret_cast<float*>(ring + (blockDim.x >> 5) * (kStages * kStage));
  const uint32_t weight = ptx::smem_u32(params) + ((group.warp - group.rank * group.warps) * I * 64 + group.lane) * 16;
  const float whole = 1.f / (float)p.dim;
  group.prepare<R <= kNormRows ? R : 1>(shared);
  ptx::begin_after_previous();
  uint64_t dw[I][H] = {}, db[I][H] = {};
  // The sums so far, to this group's part.
  const int64_t block = blockIdx.x / group.split;
  const auto put = [&](bool more) {
    float* const to = p.parts + (p.by_group ? block * groups + group.index : block) * 2 * p.dim;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const int c = first - rows.none + i * kWarpColumns + 2 * e;
        const float2 w = unpair(dw[i][e]), b = unpair(db[i][e]);
        if (c >= 0 && c < p.dim) {
          to[c] = more ? to[c] + w.x : w.x;
          to[p.dim + c] = more ? to[p.dim + c] + b.x : b.x;
        }
        if (c + 1 >= 0 && c + 1 < p.dim) {
          to[c + 1] = more ? to[c + 1] + w.y : w.y;
          to[p.dim + c + 1] = more ? to[p.dim + c + 1] + b.y : b.y;
        }
        dw[i][e] = db[i][e] = 0;
      }
  };
  typename G::Lone lone[R][2];
  const auto fetch = [&](int64_t r, const char* x, const char* dy, int stage) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      lone[q][0].settle();
      lone[q][1].settle();
      if (r + q * rows.each < p.rows) {
        const uint32_t to = own + stage * kStage + q * kRow;
        const int64_t at = q * rows.each;
        if constexpr (SAME) {
          A::fetch(to, x + at * p.x_stride, begin, dim, rows.ph, r + at == 0, r + at == p.rows - 1, lone[q][0]);
          A::fetch(to + G::kBytes, dy + at * p.dy_stride, begin, dim, rows.ph, r + at == 0, r + at == p.rows - 1, lone[q][1]);
        } else {
          G::fetch(to, x + at * p.x_stride, begin, dim, lone[q][0]);
          G::fetch(to + G::kBytes, dy + at * p.dy_stride, begin, dim, lone[q][1]);
        }
        if (group.lane == 0) copy_async_pair(to + 2 * G::kBytes, p.stats + 2 * (r + at));
      }
    }
    copy_async_commit();
  };
  int64_t r = rows.first;
  const char *x_row = p.x + r * p.x_stride - rows.ph, *dy_row = p.dy + r * p.dy_stride - rows.ph;
  char* dx_row = p.dx + r * p.dx_stride - rows.ph;
  const int64_t x_step = rows.step * p.x_stride, dy_step = rows.step * p.dy_stride, dx_step = rows.step * p.dx_stride;
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) fetch(r + k * rows.step, x_row + k * x_step, dy_row + k * dy_step, k);
  put_params<PT, I>(params, p.weight, 1.f, group, begin - rows.none, p.dim);
  __syncthreads();
  int chain = 0, stage = 0;
  bool more = false;
  float lost = 0.f;
  for (uint32_t count = 0; r < p.rows; r += rows.step, x_row += x_step, dy_row += dy_step, dx_row += dx_step, ++count) {
    if (p.by_group && chain >= kNormChain) {
      put(more);
      more = true;
      chain = 0;
    }
    chain += R;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      lone[q][0].settle();
      lone[q][1].settle();
    }
    copy_async_wait_but<kStages - 2>();
    __syncwarp();
    const uint32_t here = own + stage * kStage;
    fetch(r + (kStages - 1) * rows.step, x_row + (kStages - 1) * x_step, dy_row + (kStages - 1) * dy_step,
          stage == 0 ? kStages - 1 : stage - 1);   // where the row before was
    stage = stage + 1 == kStages ? 0 : stage + 1;
    uint64_t h[R][I][H], g[R][I][H];
    float rstd[R], a[R], b[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const float2 stats = unpair(ld_shared_u64(here + q * kRow + 2 * G::kBytes));
      rstd[q] = stats.y;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        if constexpr (SAME) {
          A::read(here + q * kRow, begin, dim, rows.ph, i, h[q][i]);
          A::read(here + q * kRow + G::kBytes, begin, dim, rows.ph, i, g[q][i]);
        } else {
          G::read(here + q * kRow, x_row + q * rows.each * p.x_stride, begin, dim, i, h[q][i]);
          G::read(here + q * kRow + G::kBytes, dy_row + q * rows.each * p.dy_stride, begin, dim, i, g[q][i]);
        }
#pragma unroll
        for (int e = 0; e < H; ++e) h[q][i][e] = mul2f(add2f(h[q][i][e], pair(-stats.x, -stats.x)), pair(stats.y, stats.y));
        if (q == 0 || r + q * rows.each < p.rows) {
#pragma unroll
          for (int e = 0; e < H; ++e) {
            dw[i][e] = fma2f(g[q][i][e], h[q][i][e], dw[i][e]);
            db[i][e] = add2f(g[q][i][e], db[i][e]);
          }
        }
      }
    }
    if (!p.dx) continue;
    uint64_t a2[R] = {}, b2[R] = {};   // dy is 0 behind the row's end
#pragma unroll
    for (int i = 0; i < I; ++i) {
      uint64_t w[H];
      get_params(weight, i, w);
#pragma unroll
      for (int q = 0; q < R; ++q)
#pragma unroll
        for (int e = 0; e < H; ++e) {
          g[q][i][e] = mul2f(g[q][i][e], w[e]);
          a2[q] = add2f(g[q][i][e], a2[q]);
          b2[q] = fma2f(g[q][i][e], h[q][i][e], b2[q]);
        }
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      a[q] = warp_sum(both(a2[q]));
      b[q] = warp_sum(both(b2[q]));
    }
    if (group.all() > 1) {
      group.exchange(shared, count, a, b, lost, p.patience);
#pragma unroll
      for (int q = 0; q < R; ++q) {
        const float2* const of = group.of(shared, count & 1, q);
        a[q] = b[q] = lost;
        if (SPLIT && group.all() > 16) {   // a lane takes a warp, or a few
          for (int w = group.lane; w < group.all(); w += 32) {
            const float2 v = of[w];
            a[q] += v.x;
            b[q] += v.y;
          }
          a[q] = warp_sum(a[q]);
          b[q] = warp_sum(b[q]);
          continue;
        }
#pragma unroll 4
        for (int w = 0; w < group.all(); ++w) {
          const float2 v = of[w];
          a[q] += v.x;
          b[q] += v.y;
        }
      }
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (r + q * rows.each >= p.rows) break;
      uint4 out[I * C::N];
      const uint64_t minus_a = pair(-a[q] * whole, -a[q] * whole), minus_b = pair(-b[q] * whole, -b[q] * whole), by = pair(rstd[q], rstd[q]);
#pragma unroll
      for (int i = 0; i < I; ++i) {
#pragma unroll
        for (int e = 0; e < H; ++e) g[q][i][e] = mul2f(fma2f(h[q][i][e], minus_b, add2f(g[q][i][e], minus_a)), by);
        C::pack2(g[q][i], out + i * C::N);
      }
      if constexpr (SAME) A::write(dx_row + q * rows.each * p.dx_stride, begin, dim, rows.ph, out);
      else G::write(here + q * kRow, dx_row + q * rows.each * p.dx_stride, begin, dim, out);
    }
  }
  ptx::let_next_begin();
  const auto end = [&] {   // behind the parts: between the rows and them it costs registers (8192 x 8192: 101 us instead of 97)
    if (SPLIT) group.report_lost(shared);
    group.finish();
  };
  if (!p.parts) return end();
  if (p.by_group || groups == 1) {
    put(more);
    return end();
  }
  // The groups' sums, through the ring: [groups, 2, columns].
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(ring);
  float2* const to = reinterpret_cast<float2*>(sums + group.index * 2 * columns + first - group.rank * columns);
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int e = 0; e < H; ++e) {
      to[i * (kWarpColumns / 2) + e] = unpair(dw[i][e]);
      to[columns / 2 + i * (kWarpColumns / 2) + e] = unpair(db[i][e]);
    }
  __syncthreads();
  float* const part = p.parts + block * 2 * p.dim;
  const int from = group.rank * columns - rows.none;   // the block's first column
  for (int c = threadIdx.x; c < columns; c += blockDim.x) {
    if (from + c < 0 || from + c >= p.dim) continue;
    float w = 0.f, b = 0.f;
    for (int q = 0; q < groups; ++q) {
      w += sums[q * 2 * columns + c];
      b += sums[(q * 2 + 1) * columns + c];
    }
    part[from + c] = w;
    part[p.dim + from + c] = b;
  }
  end();
}

// dw and db: the sums of `n` parts.  32 columns a block, its warps take parts in turn, eight loads of a thread under way (148 parts of 4096 columns: 6 us,
// of which most is the launch and two latencies).
constexpr int kJoinWarps = 16;
struct NormJoinParams {
  const float* parts;
  int n, dim;
  void* out[2];
};
template <int PT>
__global__ void __launch_bounds__(kJoinWarps * 32) norm_join_kernel(const NormJoinParams p) {
  __shared__ float s[kJoinWarps][32];
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.x & 1, c = (blockIdx.x >> 1) * 32 + lane;
  void* const out = which ? p.out[1] : p.out[0];
  if (!out) return;
  const float* const from = p.parts + (int64_t)which * p.dim + min(c, p.dim - 1);
  float sum = 0.f;
  for (int i = warp; i < p.n; i += kJoinWarps * 8) {
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = i + u * kJoinWarps < p.n ? __ldcg(from + (int64_t)2 * (i + u * kJoinWarps) * p.dim) : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += x[u];
  }
  s[warp][lane] = sum;
  __syncthreads();
  if (warp == 0 && c < p.dim) {
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) all += s[w][lane];
    static_cast<typename Elem<PT>::T*>(out)[c] = Elem<PT>::from(all);
  }
}

// ---- host side -----------------------------------------------------------------------------------------------------
static std::atomic<bool> norm_withhold{false};
static NormPatience norm_patience(int split) { return norm_withhold.load() ? NormPatience{16, 0} : NormPatience{kNormLooks, (uint32_t)split}; }
struct NormPlan {
  int split, warps, runs, rows, groups;   // rows: at a time (several only of one run, or of two); groups: of a block
};
static void plan_runs(NormPlan& n, int64_t columns, int most, int row_warps) {   // most: runs that a thread holds of a row
  n.split = 1;
  while ((int64_t)n.split * most * kWarpColumns * row_warps < columns) n.split *= 2;
  const int runs = (int)((columns + (int64_t)n.split * kWarpColumns - 1) / ((int64_t)n.split * kWarpColumns));   // of 256 columns in a block
  n.warps = (runs + most - 1) / most;
  n.runs = (runs + n.warps - 1) / n.warps;
}
static void plan_groups(NormPlan& n, int64_t rows, int warps) {   // warps: of a block
  if (n.split > 1 && warps > kNormGradRowWarps) warps = kNormGradRowWarps;   // that there is room for in NormShared
  n.groups = warps / n.warps;
  if (n.split > 1 && n.groups > kNormSplitGroups) n.groups = kNormSplitGroups;
  const int64_t each = (rows * n.split + (int64_t)kSms * n.rows - 1) / ((int64_t)kSms * n.rows);   // few rows are spread over the SMs
  if (n.groups > each) n.groups = each < 1 ? 1 : (int)each;
}
static int64_t norm_grid(const NormPlan& n, int64_t rows, int64_t room) { return norm_grid(n.groups, n.rows, rows, room); }
// Whether the rows of two matrices lie alike in 16 bytes.
static bool lie_alike(const void* a, int64_t a_stride, const void* b, int64_t b_stride) {
  return (reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b)) % 16 == 0 && (a_stride - b_stride) % 16 == 0;
}
static int period_of(int64_t stride) {   // bytes
  int n = 1;
  while (stride * n % 16) n *= 2;
  return n;
}
// How the rows lie that a call reads and writes (`alike`: the others as x's).  Comes back with the columns counted as the kernel does.
static int norm_mode(const void* x, int64_t stride, bool alike, int64_t row_bytes, int64_t* columns) {
  if (!alike || stride < 16) return kAny;   // kSame reads whole 16 bytes where rows begin and end, which are to lie between the rows before and behind
  if (reinterpret_cast<uintptr_t>(x) % 16 == 0 && stride % 16 == 0) return row_bytes % 16 == 0 ? kAligned : kSame;
  if (*columns + kNormPeriod - 1 > kNormMaxDim) return kAny;
  *columns += kNormPeriod - 1;
  return kSame;
}
static NormPlan norm_plan(int64_t rows, int64_t columns, int dtype) {
  NormPlan n;
  plan_runs(n, columns, kNormRuns, kNormRowWarps);
  // Two rows at a time share a barrier and the parameters; short ones are four, or two; few rows are spread over the SMs first.
  n.rows = n.warps == 1 && n.split == 1 && n.runs < 3 ? kNormRuns / n.runs : dtype != IRIS_F32 && rows > 2 * kSms ? 2 : 1;
  plan_groups(n, rows, norm_warps(dtype, n.rows * n.runs));
  return n;
}
static NormPlan norm_grad_plan(int64_t rows, int64_t columns, int dtype) {
  NormPlan n;
  // Rows of more than 8 warps are shared by two blocks of two groups rather than held by one group (8192 x 8192 bf16 98 us instead of 101);
  // four blocks instead of two leave 16 of 148 SMs without a cluster (5500 x 12000: 2 % longer).
  const bool pairs = columns > kNormGradRuns * kWarpColumns * kNormGradRowWarps / 2 && columns <= kNormGradRuns * kWarpColumns * kNormGradRowWarps;
  plan_runs(n, columns, kNormGradRuns, pairs ? kNormGradRowWarps / 2 : kNormGradRowWarps);
  // Two rows at a time leave room for fewer warps: where rows have so many that it makes no difference.
  const bool two = n.runs == 1 ? n.warps == 1 && n.split == 1
                               : dtype != IRIS_F32 && rows > 2 * kSms && norm_grad_warps(4) / n.warps * n.warps >= norm_grad_warps(2) / n.warps * n.warps;
  n.rows = two ? 2 : 1;
  plan_groups(n, rows, norm_grad_warps(n.rows * n.runs));
  return n;
}
// Whether a group has more than kNormChain rows, and its sums their own part.
static bool norm_by_group(const NormPlan& n, int64_t rows, int64_t grid) { return rows > grid * n.groups * kNormChain; }
static int64_t norm_parts(const NormPlan& n, int64_t rows) {   // at most: a device may have fewer clusters at once, and more rows for each
  const int64_t grid = norm_grid(n, rows, kSms / n.split);
  return grid * (n.split > 1 || norm_by_group(n, rows, grid) ? n.groups : 1);
}

template <int DT, int PT, int R, int I, int MODE, bool SPLIT = false>
static int launch_norm(const NormParams& p, const NormPlan& n, cudaStream_t st) {
  if constexpr (!SPLIT && I == kNormRuns)   // as rows of several blocks have
    if (n.split > 1) return launch_norm<DT, PT, R, I, MODE, true>(p, n, st);
  constexpr auto kernel = norm_kernel<DT, PT, R, I, MODE, SPLIT>;
  constexpr int stages = norm_stages(DT, R * I) * R * Segment<DT, I>::kBytes, params = 2 * I * kWarpColumns * (int)sizeof(float);   // of a warp, of a warp of a row
  constexpr int most = norm_warps(DT, R * I) * stages + kNormRowWarps * params;
  int room;
  IRIS_CHECK(allow_shared<kernel>(most));
  IRIS_CHECK(clusters_at_once<kernel>(n.split, norm_warps(DT, R * I) * 32, most, &room));
  return launch_rows(kernel, p, (unsigned)(norm_grid(n, p.rows, room) * n.split), n.split, n.warps * n.groups * 32,
                     (size_t)n.warps * (n.groups * stages + params), st);
}
template <int DT, int PT, int MODE>
static int launch_norm(const NormParams& p, const NormPlan& n, cudaStream_t st) {
  if (n.runs == 1) return launch_norm<DT, PT, 4, 1, MODE>(p, n, st);
  if (n.runs == 2) return launch_norm<DT, PT, 2, 2, MODE>(p, n, st);
  if constexpr (DT != IRIS_F32)
    if (n.rows == 2) return n.runs == 3 ? launch_norm<DT, PT, 2, 3, MODE>(p, n, st) : launch_norm<DT, PT, 2, 4, MODE>(p, n, st);
  return n.runs == 3 ? launch_norm<DT, PT, 1, 3, MODE>(p, n, st) : launch_norm<DT, PT, 1, 4, MODE>(p, n, st);
}
template <int DT, int PT>
static int launch_norm(const NormParams& p, const NormPlan& n, int mode, cudaStream_t st) {
  return mode == kAligned ? launch_norm<DT, PT, kAligned>(p, n, st) : mode == kSame ? launch_norm<DT, PT, kSame>(p, n, st) : launch_norm<DT, PT, kAny>(p, n, st);
}
template <int DT, int PT, int R, int I, int MODE, bool SPLIT = false>
static int launch_norm_grad(NormGradParams p, const NormPlan& n, cudaStream_t st, int* parts) {
  if constexpr (!SPLIT && I == kNormGradRuns)
    if (n.split > 1) return launch_norm_grad<DT, PT, R, I, MODE, true>(p, n, st, parts);
  constexpr auto kernel = norm_grad_kernel<DT, PT, R, I, MODE, SPLIT>;
  constexpr int stages = norm_grad_stages(DT) * norm_grad_stage_bytes<DT, R, I>(), params = I * kWarpColumns * (int)sizeof(float);   // of a warp, of a warp of a row
  static_assert(stages >= 2 * params, "the groups' sums take the place of the rows");
  constexpr int most = norm_grad_warps(R * I) * (stages + params);
  int room;
  IRIS_CHECK(allow_shared<kernel>(most));
  IRIS_CHECK(clusters_at_once<kernel>(n.split, norm_grad_warps(R * I) * 32, most, &room));
  const int64_t grid = norm_grid(n, p.rows, room);
  p.by_group = p.parts && norm_by_group(n, p.rows, grid);
  *parts = (int)(grid * (p.by_group ? n.groups : 1));
  return launch_rows(kernel, p, (unsigned)(grid * n.split), n.split, n.warps * n.groups * 32, (size_t)n.warps * (n.groups * stages + params), st);
}
template <int DT, int PT, int MODE>
static int launch_norm_grad(const NormGradParams& p, const NormPlan& n, cudaStream_t st, int* parts) {
  if (n.runs == 1) return launch_norm_grad<DT, PT, 2, 1, MODE>(p, n, st, parts);
  if constexpr (DT != IRIS_F32)
    if (n.rows == 2) return launch_norm_grad<DT, PT, 2, 2, MODE>(p, n, st, parts);
  return launch_norm_grad<DT, PT, 1, 2, MODE>(p, n, st, parts);
}
template <int DT, int PT>
static int launch_norm_grad(const NormGradParams& p, const NormPlan& n, int mode, void* dweight, void* dbias, cudaStream_t st) {
  int parts = 0;
  IRIS_CHECK(mode == kAligned ? launch_norm_grad<DT, PT, kAligned>(p, n, st, &parts) : mode == kSame ? launch_norm_grad<DT, PT, kSame>(p, n, st, &parts)
                                                                                              : launch_norm_grad<DT, PT, kAny>(p, n, st, &parts));
  if (!p.parts) return IRIS_OK;
  return launch_rows(norm_join_kernel<PT>, NormJoinParams{p.parts, parts, p.dim, {dweight, dbias}}, (unsigned)((p.dim + 31) / 32 * 2), 1,
                     kJoinWarps * 32, 0, st);
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
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 8, false));
  if (!(a->eps >= 0.f) || std::isinf(a->eps)) return fail(IRIS_ERR_ARG, "%s: eps has to be finite and not negative", fn);
  IRIS_CHECK(check_overlap(fn, "y", "x", a->x, xs, a->y, ys, a->rows, a->dim, a->dtype));
  if (a->rows == 0) return IRIS_OK;
  const int64_t es = (int64_t)elem_size(a->dtype);
  int64_t columns = a->dim;
  const int mode = norm_mode(a->x, xs * es, lie_alike(a->x, xs * es, a->y, ys * es), a->dim * es, &columns);
  const NormPlan n = norm_plan(a->rows, columns, a->dtype);
  NormParams p{static_cast<const char*>(a->x), static_cast<char*>(a->y), xs * es, ys * es, static_cast<const char*>(a->weight),
               static_cast<const char*>(a->bias), a->stats, a->rows, (int)a->dim, n.warps, n.split, period_of(xs * es), a->eps, norm_patience(n.split)};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = a->param_dtype == IRIS_F32;
  if (a->dtype == IRIS_BF16) return wide ? launch_norm<IRIS_BF16, IRIS_F32>(p, n, mode, st) : launch_norm<IRIS_BF16, IRIS_BF16>(p, n, mode, st);
  if (a->dtype == IRIS_F16) return wide ? launch_norm<IRIS_F16, IRIS_F32>(p, n, mode, st) : launch_norm<IRIS_F16, IRIS_F16>(p, n, mode, st);
  return launch_norm<IRIS_F32, IRIS_F32>(p, n, mode, st);
}

extern "C" size_t iris_layer_norm_workspace_bytes(int64_t rows, int64_t dim) {
  if (rows <= 0 || rows > INT32_MAX || dim <= 0 || dim > kNormMaxDim) return 0;
  int64_t parts = 0;
  for (int dtype : {(int)IRIS_F16, (int)IRIS_F32})
    for (int64_t columns : {dim, dim + kNormPeriod - 1})   // rows may begin anywhere
      if (columns <= kNormMaxDim || columns == dim) {
        const int64_t n = norm_parts(norm_grad_plan(rows, columns, dtype), rows);
        parts = n > parts ? n : parts;
      }
  return (size_t)parts * 2 * dim * sizeof(float);
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
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 8, a->rows > 0));
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
  int64_t columns = a->dim;
  const bool alike = lie_alike(a->x, xs * es, a->dy, gs * es) && (!a->dx || lie_alike(a->x, xs * es, a->dx, ds * es));
  const int mode = norm_mode(a->x, xs * es, alike && gs * es >= 16, a->dim * es, &columns);
  const NormPlan n = norm_grad_plan(a->rows, columns, a->dtype);
  NormGradParams p{static_cast<const char*>(a->x), static_cast<const char*>(a->dy), static_cast<char*>(a->dx), xs * es, gs * es, ds * es,
                   static_cast<const char*>(a->weight), a->stats, sums ? static_cast<float*>(a->workspace) : nullptr, a->rows, (int)a->dim, n.warps,
                   n.split, period_of(xs * es), 0, norm_patience(n.split)};
  const bool wide = a->param_dtype == IRIS_F32;
  if (a->dtype == IRIS_BF16)
    return wide ? launch_norm_grad<IRIS_BF16, IRIS_F32>(p, n, mode, a->dweight, a->dbias, st) : launch_norm_grad<IRIS_BF16, IRIS_BF16>(p, n, mode, a->dweight, a->dbias, st);
  if (a->dtype == IRIS_F16)
    return wide ? launch_norm_grad<IRIS_F16, IRIS_F32>(p, n, mode, a->dweight, a->dbias, st) : launch_norm_grad<IRIS_F16, IRIS_F16>(p, n, mode, a->dweight, a->dbias, st);
  return launch_norm_grad<IRIS_F32, IRIS_F32>(p, n, mode, a->dweight, a->dbias, st);
}

extern "C" int iris_layer_norm_status(void* stream, int32_t* detail) {
  int32_t host[kStatusWords];
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  IRIS_CUDA_TRY(cudaMemcpyFromSymbolAsync(host, norm_status, sizeof(host), 0, cudaMemcpyDeviceToHost, st));
  IRIS_CUDA_TRY(cudaStreamSynchronize(st));
  if (detail)
    for (int i = 0; i < kStatusWords; ++i) detail[i] = host[i];
  if (!host[0]) return IRIS_OK;
  const int32_t none[kStatusWords] = {};
  IRIS_CUDA_TRY(cudaMemcpyToSymbolAsync(norm_status, none, sizeof(none), 0, cudaMemcpyHostToDevice, st));
  IRIS_CUDA_TRY(cudaStreamSynchronize(st));
  return fail(host[0], "iris_layer_norm: a wait of a block for the others of its rows ran out: kernel=%d block=%d group=%d warp=%d", host[1], host[2], host[3], host[4]);
}

extern "C" void iris_layer_norm_withhold(int on) { norm_withhold.store(on != 0); }
