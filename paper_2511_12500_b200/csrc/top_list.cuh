// The k largest of a row's logits, found in the pass over them: a block keeps a lower bound tau of its k-th largest and
// puts every logit above tau on a list in shared memory.
//
// The bound comes from the threads' maxima: if k threads hold a logit >= tau, then k logits are >= tau.  With 256 threads
// and k of them above, the list grows by little more than k for the first 64 logits a thread, and by ever less after that.
// Ties are cut by the column, so a logit equal to the final tau may still be needed (a row whose mask leaves fewer than k
// logits always needs some); those are fetched in column order at the end.  A row that is laid out so that the list
// overflows is selected digit by digit instead.
#pragma once

#include "logit_rows.cuh"
#include "sm100_ptx.cuh"

namespace iris {
namespace rows {

constexpr int kTopThreads = 256;
constexpr int kTopCap = 1024;   // > 127 granules of 8, what a block can hold with fewer than k threads at work
static_assert(kTopThreads >= kMaxList && kTopCap >= (kMaxList - 1) * 8, "the list holds all of a part that has fewer granules than k");

struct TopShared {
  uint64_t key[kTopCap];      // candidates as they come
  uint64_t kept[kTopCap];     // those above the final tau, and the ties that are needed
  uint32_t code[kTopThreads]; // the threads' maxima (order_bits); 0 = no logit yet
  uint32_t hist[256];
  uint32_t tau;
  int n, n_kept, warp_sum[kTopThreads / 32];
};

// By one warp: the largest tau it finds in 16 halvings with at least k of sh.code >= tau (0 if fewer than k are not 0);
// a count within an eighth of k is near enough.
__device__ __forceinline__ void bisect_tau(TopShared& sh, int k) {
  const int lane = threadIdx.x & 31;
  uint32_t c[kTopThreads / 32], lo = ~0u, hi = 0;
#pragma unroll
  for (int i = 0; i < kTopThreads / 32; ++i) {
    c[i] = sh.code[lane + 32 * i];
    lo = min(lo, c[i]);
    hi = max(hi, c[i]);
  }
  lo = __reduce_min_sync(~0u, lo);   // all kTopThreads >= k are at least this large
  hi = __reduce_max_sync(~0u, hi);
  for (int it = 0; it < 16 && lo < hi; ++it) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;   // in (lo, hi]; (hi - lo + 1) is 0 only for the whole range, which 0 and NaN make
    const uint32_t m = hi - lo == ~0u ? 0x80000000u : mid;
    int cnt = 0;
#pragma unroll
    for (int i = 0; i < kTopThreads / 32; ++i) cnt += c[i] >= m;
    cnt = __reduce_add_sync(~0u, cnt);
    if (cnt >= k) {
      lo = m;
      if (cnt <= k + k / 8) break;
    } else {
      hi = m - 1;
    }
  }
  if (lane == 0) sh.tau = max(sh.tau, lo);   // never back: what was left out was not above the earlier one
}

// Puts granule v's logits above tau on the list; at_tau: tau as a float, NaN for tau = 0 (every logit is above it).  Not
// inlined: few granules have such a logit, and the pass over the row keeps its registers.
template <int DT>
__device__ __noinline__ void collect(TopShared& sh, int ph, int end, int v, uint4 g, float at_tau) {
  using E = Elem<DT>;
  constexpr int VE = E::VE;
  float x[VE];
  E::unpack(g, x);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    if (!(x[e] <= at_tau)) {
      const int i = v * VE + e;
      if (i >= ph && i < end) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < kTopCap) sh.key[at] = order_key(x[e], i - ph);
      }
    }
  }
}

// Exact tau by four passes over 8 bits each, and the logits above it (fewer than k) on the list.
template <int DT>
__device__ __noinline__ void select_by_digits(TopShared& sh, const Row<DT>& row, int v0, int v1, int k) {
  constexpr int VE = Row<DT>::VE;
  uint32_t prefix = 0, mask = 0;
  int need = k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    sh.hist[threadIdx.x] = 0;
    __syncthreads();
    for (int v = v0 + (int)threadIdx.x; v < v1; v += kTopThreads) {
      float x[VE];
      row.load(v, x);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int i = v * VE + e;
        const uint32_t code = order_bits(x[e]);
        if (i >= row.ph && i < row.end && (code & mask) == prefix) atomicAdd(&sh.hist[code >> shift & 255], 1u);
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
      if (i >= row.ph && i < row.end && order_bits(x[e]) > prefix) sh.key[atomicAdd(&sh.n, 1)] = order_key(x[e], i - row.ph);
    }
  }
  __syncthreads();
}

// Appends to sh.kept the `need` lowest columns whose logit is equal to tau.
template <int DT>
__device__ __noinline__ void fetch_ties(TopShared& sh, const Row<DT>& row, int v0, int v1, uint32_t tau, int need) {
  constexpr int VE = Row<DT>::VE;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = sh.n_kept;
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
        if (i >= row.ph && i < row.end && order_bits(x[e]) == tau) hits |= 1u << e;
      }
    }
    const int mine = __popc(hits);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(~0u, upto, o);
      if (lane >= o) upto += y;
    }
    __syncthreads();   // the sums of the previous round have been read
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
        if (at < need) sh.kept[first + at] = (uint64_t)tau << 32 | (0xffffffffu - (uint32_t)(v * VE + e - row.ph));
        ++at;
      }
    got += total;
  }
  __syncthreads();
  if (threadIdx.x == 0) sh.n_kept = first + min(got, need);
  __syncthreads();
}

// After the pass: emit(place, key) for the part's largest, place = 0 .. min(k, its length) - 1.  Returns that count.
template <int DT, class Emit>
__device__ __forceinline__ int finish_top(TopShared& sh, const Row<DT>& row, int v0, int v1, int k, Emit emit) {
  __syncthreads();
  if (sh.n > kTopCap) select_by_digits<DT>(sh, row, v0, v1, k);
  const int n = sh.n;
  const uint32_t tau = sh.tau;
  for (int i = threadIdx.x; i < n; i += kTopThreads) {
    const uint64_t key = sh.key[i];
    if ((uint32_t)(key >> 32) > tau) sh.kept[atomicAdd(&sh.n_kept, 1)] = key;
  }
  __syncthreads();
  if (tau && sh.n_kept < k) fetch_ties<DT>(sh, row, v0, v1, tau, k - sh.n_kept);
  const int m = sh.n_kept;
  for (int i = threadIdx.x; i < m; i += kTopThreads) {
    const uint64_t key = sh.kept[i];
    int place = 0;
    for (int j = 0; j < m; ++j) place += sh.kept[j] > key;
    if (place < k) emit(place, key);
  }
  return min(m, k);
}

}  // namespace rows
}  // namespace iris
