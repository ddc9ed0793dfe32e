// The k largest of a row's logits.  The pass over the row keeps every thread's largest logits, by pieces of the row.  If k
// threads hold a logit >= tau, then k logits are >= tau: the largest such tau that a few halvings find leaves little more
// than k logits from it up (each of 256 threads has a share of the row, and few hold two of the k largest).  The pieces with
// such logits, about k of them, are read again, from L2, a granule a thread, and the logits are listed; a key's place among
// the k is the number of larger keys on the list.
//
// Where far more than k threads hold tau or more (equal logits; a mask that leaves fewer than k, in which case tau is the
// mask's value), the list takes what is above tau, and the ties it lacks are fetched in column order.  A row laid out so that
// the list overflows is selected digit by digit.  So is, from k = 114 on, a long row whose mask leaves fewer than k: "far more"
// is then more threads than there are (4096 x 36864 bf16, 99.8 % masked: 127 us with 113 alternatives, 688 with 114).
//
// One search of the row for each alternative took 8.9 ms for 4096 x 36864 with 64 (86 us now); a list filled during the pass,
// with a bound after every batch, 179 us: two barriers and a search for the bound a batch.
#pragma once

#include "logit_rows.cuh"
#include "sm100_ptx.cuh"

namespace iris {
namespace rows {

constexpr int kTopThreads = 256;
constexpr int kTopPieces = 16;
constexpr int kTopCap = 1024;   // > 127 granules of 8, what a block can hold with fewer than k threads at work
static_assert(kTopThreads >= kMaxList && kTopCap >= (kMaxList - 1) * 8, "the list holds all of a part that has fewer granules than k");

constexpr int kTopQueue = 768;   // granules with wanted logits

struct TopShared {
  alignas(16) uint64_t key[kTopCap];
  union {
    float largest[kTopPieces][kTopThreads];   // of a thread's logits in a piece
    struct {
      uint4 granule[kTopQueue];
      int index[kTopQueue];
    } queue;
  };
  uint32_t ordinal[kTopThreads];            // of a thread's largest logit; 0 = it has none
  uint16_t again[kTopPieces * kTopThreads]; // pieces to be read again: piece * kTopThreads + thread
  uint32_t hist[256];
  uint32_t tau;
  int with_tau;   // logits equal to tau are listed too
  int n, n_again, n_queue, warp_sum[kTopThreads / 32];
};

// By one warp: the largest tau it finds with at least k of sh.ordinal >= tau (0 if fewer than k are not 0), by quartering;
// a few more than k are near enough.
__device__ __forceinline__ void find_tau(TopShared& sh, int k) {
  const int lane = threadIdx.x & 31, enough = k + max(8, k / 8);
  int above = kTopThreads;   // threads that hold lo or more
  uint32_t c[kTopThreads / 32], lo = ~0u, hi = 0;
#pragma unroll
  for (int i = 0; i < kTopThreads / 32; ++i) {
    c[i] = sh.ordinal[lane + 32 * i];
    lo = min(lo, c[i]);
    hi = max(hi, c[i]);
  }
  lo = __reduce_min_sync(~0u, lo);   // all kTopThreads >= k are at least this large
  hi = __reduce_max_sync(~0u, hi);
  for (int it = 0; it < 10 && lo < hi; ++it) {
    const uint32_t step = (hi - lo) / 4, m1 = lo + max(1u, step), m2 = max(m1, lo + 2 * step), m3 = max(m2, lo + 3 * step);   // in (lo, hi]
    uint32_t cnt = 0;   // three counts up to 256, 10 bits each
#pragma unroll
    for (int i = 0; i < kTopThreads / 32; ++i) cnt += (c[i] >= m1 ? 1u : 0u) + (c[i] >= m2 ? 1u << 10 : 0u) + (c[i] >= m3 ? 1u << 20 : 0u);
    cnt = __reduce_add_sync(~0u, cnt);
    const int n1 = cnt & 1023, n2 = cnt >> 10 & 1023, n3 = cnt >> 20;
    if (n3 >= k) lo = m3, above = n3;
    else if (n2 >= k) lo = m2, hi = m3 - 1, above = n2;
    else if (n1 >= k) lo = m1, hi = m2 - 1, above = n1;
    else hi = m1 - 1;
    if (above <= enough) break;
  }
  if (lane == 0) {
    sh.tau = lo;
    sh.with_tau = lo == 0 || above <= 2 * enough;
  }
}

// Exact tau by passes over 8 bits each, and the keys above it (fewer than k) on the list.
template <int DT>
__device__ __noinline__ void select_by_digits(TopShared& sh, const Row<DT>& row, int v0, int v1, int k) {
  using E = Elem<DT>;
  constexpr int VE = E::VE, kBits = VE == 8 ? 16 : 32;
  uint32_t prefix = 0, mask = 0;
  int need = k;
  for (int shift = kBits - 8; shift >= 0; shift -= 8) {
    sh.hist[threadIdx.x] = 0;
    __syncthreads();
    for (int v = v0 + (int)threadIdx.x; v < v1; v += kTopThreads) {
      float x[VE];
      row.load(v, x);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int i = v * VE + e;
        const uint32_t n = E::ordinal(x[e]);
        if (i >= row.ph && i < row.end && (n & mask) == prefix) atomicAdd(&sh.hist[n >> shift & 255], 1u);
      }
    }
    __syncthreads();
    int digit = 255, above = 0;   // every thread walks down the same counts
    while (digit > 0 && above + (int)sh.hist[digit] < need) above += (int)sh.hist[digit--];
    need -= above;
    prefix |= (uint32_t)digit << shift;
    mask |= 255u << shift;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    sh.tau = prefix;
    sh.n = 0;
  }
  __syncthreads();
  for (int v = v0 + (int)threadIdx.x; v < v1; v += kTopThreads) {
    float x[VE];
    row.load(v, x);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int i = v * VE + e;
      if (i >= row.ph && i < row.end && E::ordinal(x[e]) > prefix) sh.key[atomicAdd(&sh.n, 1)] = order_key<DT>(x[e], i - row.ph);
    }
  }
  __syncthreads();
}

// Appends to the list the `need` lowest columns whose logit is equal to tau.
template <int DT>
__device__ __noinline__ void fetch_ties(TopShared& sh, const Row<DT>& row, int v0, int v1, uint32_t tau, int need) {
  using E = Elem<DT>;
  constexpr int VE = E::VE;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = sh.n;
  int got = 0;
  for (int base = v0; base < v1 && got < need; base += kTopThreads) {
    const int v = base + (int)threadIdx.x;
    uint32_t hits = 0;
    float x[VE];
    if (v < v1) {
      row.load(v, x);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int i = v * VE + e;
        if (i >= row.ph && i < row.end && E::ordinal(x[e]) == tau) hits |= 1u << e;
      }
    }
    const int mine = __popc(hits);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(~0u, upto, o);
      if (lane >= o) upto += y;
    }
    __syncthreads();   // the sums of the previous round, or sh.n, have been read
    if (lane == 31) sh.warp_sum[warp] = upto;
    __syncthreads();
    int at = got + upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kTopThreads / 32; ++w) {
      at += w < warp ? sh.warp_sum[w] : 0;
      total += sh.warp_sum[w];
    }
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (hits >> e & 1) {
        if (at < need) sh.key[first + at] = (uint64_t)tau << 32 | (0xffffffffu - (uint32_t)(v * VE + e - row.ph));
        ++at;
      }
    got += total;
  }
  __syncthreads();
  if (threadIdx.x == 0) sh.n = first + min(got, need);
  __syncthreads();
}

// Granules of a thread in a piece, as a power of two: at most kTopPieces pieces.
__device__ __forceinline__ int piece_shift(int n_all) {
  const int each = (n_all + kTopThreads - 1) / kTopThreads;
  int s = 0;
  while ((each + (1 << s) - 1) >> s > kTopPieces) ++s;
  return s;
}

// Which logits the list takes; NaN is wanted, and everything for tau = 0.
template <int DT>
struct Wanted {
  uint32_t tau;
  float at_tau;
  bool with_tau, none;
  __device__ __forceinline__ explicit Wanted(const TopShared& sh) : tau(sh.tau) {
    using E = Elem<DT>;
    none = tau == E::ordinal(NAN);   // nothing is above NaN: they are fetched as ties
    with_tau = sh.with_tau && !none;
    at_tau = tau ? E::value(tau) : NAN;
  }
  __device__ __forceinline__ bool operator()(float x) const { return with_tau ? !(x < at_tau) : !(x <= at_tau); }
};

// Granules with wanted logits are queued with their bits, and then looked through an element a thread: inside the pass, or
// where a thread has read a granule again, one that holds a wanted logit would stop its warp for all its elements.
__device__ __forceinline__ void queue_granule(TopShared& sh, int v, const uint4& g) {
  const int at = atomicAdd(&sh.n_queue, 1);
  if (at < kTopQueue) {
    sh.queue.granule[at] = g;
    sh.queue.index[at] = v;
  }
}
template <int DT>
__device__ __forceinline__ void list_queue(TopShared& sh, const Row<DT>& row, const Wanted<DT>& wanted) {   // behind a barrier
  using E = Elem<DT>;
  constexpr int VE = E::VE;
  const int n = sh.n_queue;
  if (n > kTopQueue) {
    if (threadIdx.x == 0) sh.n = kTopCap + 1;   // too many for the list, too
    return;
  }
  for (int j = threadIdx.x; j < n * VE; j += kTopThreads) {
    const int i = sh.queue.index[j / VE] * VE + j % VE;
    const float x = E::to(reinterpret_cast<const typename E::T*>(&sh.queue.granule[j / VE])[j % VE]);
    if (wanted(x) && i >= row.ph && i < row.end) {
      const int at = atomicAdd(&sh.n, 1);
      if (at < kTopCap) sh.key[at] = order_key<DT>(x, i - row.ph);
    }
  }
}

// Queues what is wanted of a part, of which sh.largest has the pieces' largest logits.  One barrier.
template <int DT>
__device__ __forceinline__ void queue_pieces(TopShared& sh, const Row<DT>& row, const Part<DT>& part, int shift, const Wanted<DT>& wanted) {
  constexpr int T = kTopThreads;
  const int tid = threadIdx.x, lane = tid & 31;
  uint32_t pieces = 0;
  if (!wanted.none)
    for (int q = 0; (q << shift) * T + tid < part.n_all; ++q) pieces |= wanted(sh.largest[q][tid]) ? 1u << q : 0u;
  const int mine = __popc(pieces);
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(~0u, upto, o);
    if (lane >= o) upto += y;
  }
  int at = 0;
  if (lane == 31 && upto) at = atomicAdd(&sh.n_again, upto);
  at = __shfl_sync(~0u, at, 31) + upto - mine;
  for (; pieces; pieces &= pieces - 1) sh.again[at++] = (uint16_t)((__ffs(pieces) - 1) * T + tid);
  __syncthreads();
  for (int j = tid; j < sh.n_again << shift; j += T) {
    const int which = sh.again[j >> shift], i = ((which / T << shift) + (j & ((1 << shift) - 1))) * T + which % T;
    if (i >= part.n_all) continue;
    const uint4 g = part.raw(row, i);
    if (wanted(largest<DT>(g))) queue_granule(sh, part.granule(i), g);
  }
}

// Once all threads have listed what is wanted: emit(place, key, sub, group) for the part's largest, place = 0 ..
// min(k, its length) - 1, by threads sub = 0 .. group - 1 each.  Returns that count.
template <int DT, class Emit>
__device__ __forceinline__ int finish_top(TopShared& sh, const Row<DT>& row, const Part<DT>& part, uint32_t tau, int k, Emit emit) {
  constexpr int T = kTopThreads;
  const int tid = threadIdx.x;
  __syncthreads();
  if (sh.n > kTopCap) {
    select_by_digits<DT>(sh, row, part.v0, part.v1, k);
    tau = sh.tau;
  }
  if (tau && sh.n < k) fetch_ties<DT>(sh, row, part.v0, part.v1, tau, k - sh.n);
  const int n = sh.n;
  int group = 32;   // threads that share a key's comparisons
  while (group > 1 && group * n > T) group /= 2;
  for (int b = 0; b < n; b += T / group) {
    const int i = b + tid / group, sub = tid % group;
    uint64_t key = 0;
    int place = 0;
    if (i < n) {
      key = sh.key[i];
      for (int j = 2 * sub; j < n; j += 2 * group) {
        const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(&sh.key[j]);
        place += (two.x > key) + (two.y > key && j + 1 < n);
      }
    }
    for (int o = group / 2; o; o /= 2) place += __shfl_xor_sync(~0u, place, o);
    if (i < n && place < k) emit(place, key, sub, group);
  }
  return min(n, k);
}

}  // namespace rows
}  // namespace iris
