// The k largest of a row's logits.  The pass over the row keeps every thread's largest logits, by pieces of the row.  If k
// threads hold a logit >= tau, then k logits are >= tau: the largest such tau that a few halvings find leaves little more
// than k logits above it (each of 256 threads has a share of the row, and few hold two of the k largest).  Threads read the
// pieces again whose largest logit is above tau (from L2: about k of them) and list what is; a key's place among the k is
// the number of larger keys on the list.
//
// Ties are cut by the column, so logits equal to tau may be needed too (a row whose mask leaves fewer than k logits always
// needs some); those are fetched in column order.  A row laid out so that the list overflows is selected digit by digit.
#pragma once

#include "logit_rows.cuh"
#include "sm100_ptx.cuh"

namespace iris {
namespace rows {

constexpr int kTopThreads = 256;
constexpr int kTopPieces = 16;
constexpr int kTopCap = 1024;   // > 127 granules of 8, what a block can hold with fewer than k threads at work
static_assert(kTopThreads >= kMaxList && kTopCap >= (kMaxList - 1) * 8, "the list holds all of a part that has fewer granules than k");

struct TopShared {
  uint64_t key[kTopCap];
  float largest[kTopPieces][kTopThreads];   // of a thread's logits in a piece of the row
  uint32_t ordinal[kTopThreads];            // of a thread's largest logit; 0 = it has none
  uint32_t hist[256];
  uint32_t tau;
  int n, warp_sum[kTopThreads / 32];
};

// By one warp: the largest tau it finds in 16 halvings with at least k of sh.ordinal >= tau (0 if fewer than k are not 0);
// a count within an eighth of k is near enough.
__device__ __forceinline__ void bisect_tau(TopShared& sh, int k) {
  const int lane = threadIdx.x & 31;
  uint32_t c[kTopThreads / 32], lo = ~0u, hi = 0;
#pragma unroll
  for (int i = 0; i < kTopThreads / 32; ++i) {
    c[i] = sh.ordinal[lane + 32 * i];
    lo = min(lo, c[i]);
    hi = max(hi, c[i]);
  }
  lo = __reduce_min_sync(~0u, lo);   // all kTopThreads >= k are at least this large
  hi = __reduce_max_sync(~0u, hi);
  for (int it = 0; it < 16 && lo < hi; ++it) {
    const uint32_t mid = lo + (hi - lo - 1) / 2 + 1;   // in (lo, hi]
    int cnt = 0;
#pragma unroll
    for (int i = 0; i < kTopThreads / 32; ++i) cnt += c[i] >= mid;
    cnt = __reduce_add_sync(~0u, cnt);
    if (cnt >= k) {
      lo = mid;
      if (cnt <= k + k / 8) break;
    } else {
      hi = mid - 1;
    }
  }
  if (lane == 0) sh.tau = lo;
}

// Lists the columns of the logits above tau among this thread's granules g[0 .. U), granule u being the part's
// i0 + u * T-th, where u * T < left: one mark a logit, made two at a time, and few that are set.
template <int DT, int U>
__device__ __forceinline__ void collect(TopShared& sh, const Row<DT>& row, const Part<DT>& part, const uint4 (&g)[U], int i0, int left, uint32_t tau2) {
  using E = Elem<DT>;
  uint32_t m[E::kMarkWords] = {};
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (u * kTopThreads < left) E::mark(g[u], u, tau2, m);
#pragma unroll
  for (int w = 0; w < E::kMarkWords; ++w)
    while (m[w]) {
      const int bit = __ffs(m[w]) - 1;
      m[w] &= m[w] - 1;
      const int i = part.granule(i0 + E::marked_granule(w, bit) * kTopThreads) * E::VE + E::marked_element(bit);
      if (i >= row.ph && i < row.end) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < kTopCap) sh.key[at] = (uint32_t)(i - row.ph);
      }
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

// After the pass, sh.largest and sh.ordinal written and sh.n 0 behind a barrier: emit(place, key) for the part's largest,
// place = 0 .. min(k, its length) - 1.  Returns that count.  `piece`: granules of a thread in a piece, a multiple of U.
template <int DT, int U, class Emit>
__device__ __forceinline__ int find_top(TopShared& sh, const Row<DT>& row, const Part<DT>& part, int piece, int k, Emit emit) {
  using E = Elem<DT>;
  constexpr int T = kTopThreads;
  const int tid = threadIdx.x;
  if (tid < 32) bisect_tau(sh, k);
  __syncthreads();
  uint32_t tau = sh.tau;
  if (tau != E::ordinal(NAN)) {   // nothing is above NaN
    const float at_tau = tau ? E::value(tau) : NAN;   // everything is above tau = 0
    const uint32_t tau2 = E::twice(at_tau);
    for (int q = 0, i0 = tid; i0 < part.n_all; ++q, i0 += T * piece) {
      if (sh.largest[q][tid] <= at_tau) continue;
      for (int i = i0; i < min(i0 + T * piece, part.n_all); i += T * U) {
        uint4 g[U];
        const int left = part.n_all - i;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * T < left) g[u] = part.raw(row, i + u * T);
        collect<DT>(sh, row, part, g, i, left, tau2);
      }
    }
  }
  __syncthreads();
  if (sh.n > kTopCap) {
    select_by_digits<DT>(sh, row, part.v0, part.v1, k);
    tau = sh.tau;
  } else {   // the listed logits once more, for their keys
    for (int i = tid; i < sh.n; i += T) {
      const int column = (int)sh.key[i];
      sh.key[i] = order_key<DT>(E::to(row.column(column)), column);
    }
    __syncthreads();
  }
  if (tau && sh.n < k) fetch_ties<DT>(sh, row, part.v0, part.v1, tau, k - sh.n);
  const int n = sh.n;
  for (int i = tid; i < n; i += T) {
    const uint64_t key = sh.key[i];
    int place = 0;
    for (int j = 0; j < n; ++j) place += sh.key[j] > key;
    if (place < k) emit(place, key);
  }
  return min(n, k);
}

}  // namespace rows
}  // namespace iris
