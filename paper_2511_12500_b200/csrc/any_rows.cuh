// Rows that start at any element, seen in pieces of 16 bytes counted from the row's first element (not from a 16-byte boundary as in
// logit_rows.cuh), so that a thread has the same columns of every row: what the operators on embeddings and norms need, whose weights and sums
// belong to columns.
//
// A piece that does not start on a 16-byte boundary is cut out of the two aligned 16 bytes that it touches (the second is the next thread's
// first and comes from L1).  Stores go the other way: a warp holds consecutive pieces, and each thread joins the end of its neighbour's piece
// with the start of its own.  Nothing outside a row is read or written: at a row's ends, elements are moved one at a time.
#pragma once

#include <atomic>

#include "logit_rows.cuh"

namespace iris {
namespace rows {

constexpr int kLaneColumns = 8;                  // of a thread: one piece of 16-bit elements, two of 32-bit ones
constexpr int kWarpColumns = 32 * kLaneColumns;  // that the threads of a warp hold at a time

// Bytes a .. a + 15 of the 32 bytes lo, hi.
__device__ __forceinline__ uint4 cut(const uint4& lo, const uint4& hi, uint32_t a) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  if (a & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (a & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const uint32_t bits = (a & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}

// The 16 bytes at `at` of which [lo, hi) may be read; zeros elsewhere.  ES: bytes of an element.
template <int ES>
__device__ __forceinline__ uint4 load_elements(const char* at, const char* lo, const char* hi) {
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 16 / ES; ++e) {
    const char* p = at + e * ES;
    if (p >= lo && p < hi) {
      const uint32_t v = ES == 4 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
      w[e * ES / 4] |= v << (e * ES % 4 * 8);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int ES>
__device__ __forceinline__ void store_elements(char* at, const char* lo, const char* hi, const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 16 / ES; ++e) {
    char* p = at + e * ES;
    if (p >= lo && p < hi) {
      const uint32_t x = w[e * ES / 4] >> (e * ES % 4 * 8);
      if (ES == 4) *reinterpret_cast<uint32_t*>(p) = x;
      else *reinterpret_cast<uint16_t*>(p) = (uint16_t)x;
    }
  }
}
// Aligned 16 bytes, as above.
template <int ES>
__device__ __forceinline__ void store16(char* at, const char* lo, const char* hi, const uint4& v) {
  if (at >= lo && at + 16 <= hi) st_global_v4(at, v);
  else store_elements<ES>(at, lo, hi, v);
}
__device__ __forceinline__ uint32_t phase(const void* p) { return (uint32_t)reinterpret_cast<uintptr_t>(p) & 15; }

// N pieces: piece i at `at` + i * step, of the row [lo, hi).  All loads are under way before the first result is used.
template <int ES, int N>
__device__ __forceinline__ void load_pieces(const char* at, int step, const char* lo, const char* hi, uint4 (&v)[N]) {
  const uint32_t a = phase(at);   // of every piece: step is a multiple of 16
  if (a == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const char* p = at + (int64_t)i * step;
      if (p >= lo && p + 16 <= hi) v[i] = ld_global_v4(p);
      else v[i] = load_elements<ES>(p, lo, hi);
    }
    return;
  }
  uint4 next[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const char* p = at + (int64_t)i * step - a;
    const bool inside = p >= lo && p + 32 <= hi;
    v[i] = inside ? ld_global_v4(p) : load_elements<ES>(p, lo, hi);
    next[i] = inside ? ld_global_v4(p + 16) : load_elements<ES>(p + 16, lo, hi);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = cut(v[i], next[i], a);
}
template <int ES>
__device__ __forceinline__ uint4 load_piece(const char* at, const char* lo, const char* hi) {
  uint4 v[1];
  load_pieces<ES, 1>(at, 16, lo, hi, v);
  return v[0];
}

// A thread's 8 columns of a type: 1 piece or 2.
template <int DT>
struct Columns {
  using E = Elem<DT>;
  static constexpr int ES = sizeof(typename E::T), N = kLaneColumns / E::VE;   // N: pieces
  static __device__ __forceinline__ void unpack(const uint4* v, float (&x)[kLaneColumns]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float y[E::VE];
      E::unpack(v[i], y);
#pragma unroll
      for (int e = 0; e < E::VE; ++e) x[i * E::VE + e] = y[e];
    }
  }
  static __device__ __forceinline__ void pack(const float (&x)[kLaneColumns], uint4* v) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float y[E::VE];
#pragma unroll
      for (int e = 0; e < E::VE; ++e) y[e] = x[i * E::VE + e];
      v[i] = E::pack(y);
    }
  }
  // Columns first + i * kWarpColumns ... of the row's `dim`; zeros behind its end.
  template <int I>
  static __device__ __forceinline__ void load(const char* row, int first, int dim, uint4 (&v)[I * N]) {
    const char* hi = row + (int64_t)dim * ES;
    const char* at = row + (int64_t)first * ES;
    if constexpr (N == 1) {
      load_pieces<ES, I>(at, kWarpColumns * ES, row, hi, v);
    } else {
      uint4 a[I], b[I];
      load_pieces<ES, I>(at, kWarpColumns * ES, row, hi, a);
      load_pieces<ES, I>(at + 16, kWarpColumns * ES, row, hi, b);
#pragma unroll
      for (int i = 0; i < I; ++i) {
        v[2 * i] = a[i];
        v[2 * i + 1] = b[i];
      }
    }
  }
  // The other way; all threads of a warp, whose columns are lane * kLaneColumns on from the first one's.
  template <int I>
  static __device__ __forceinline__ void store(char* row, int first, int dim, const uint4 (&v)[I * N]) {
    const int lane = threadIdx.x & 31, begin = first - lane * kLaneColumns;
    const char* lo = row + (int64_t)begin * ES;
    const char* hi = row + (int64_t)min(dim, begin + I * kWarpColumns) * ES;
    char* at = row + (int64_t)first * ES;
    const uint32_t a = phase(at);
    if (a == 0) {
#pragma unroll
      for (int i = 0; i < I * N; ++i) store16<ES>(at + (int64_t)(i / N) * kWarpColumns * ES + i % N * 16, lo, hi, v[i]);
      return;
    }
    uint4 carry = make_uint4(0, 0, 0, 0);   // the piece in front of the warp's next 256 columns
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const uint4 last = v[i * N + N - 1];
      uint4 before = make_uint4(__shfl_up_sync(~0u, last.x, 1), __shfl_up_sync(~0u, last.y, 1), __shfl_up_sync(~0u, last.z, 1),
                                __shfl_up_sync(~0u, last.w, 1));
      if (lane == 0) before = carry;
      carry = make_uint4(__shfl_sync(~0u, last.x, 31), __shfl_sync(~0u, last.y, 31), __shfl_sync(~0u, last.z, 31), __shfl_sync(~0u, last.w, 31));
#pragma unroll
      for (int n = 0; n < N; ++n)
        store16<ES>(at + (int64_t)i * kWarpColumns * ES + n * 16 - a, lo, hi, cut(n ? v[i * N + n - 1] : before, v[i * N + n], 16 - a));
    }
    if (lane == 31) store16<ES>(at + (int64_t)(I - 1) * kWarpColumns * ES + N * 16 - a, lo, hi, cut(carry, carry, 16 - a));
  }
};

// ---- host side -----------------------------------------------------------------------------------------------------
// Lets a kernel have up to `bytes` of dynamic shared memory on the current device, once.
template <auto KERNEL>
inline int allow_shared(int bytes) {
  constexpr int kDevices = 64;
  static std::atomic<bool> done[kDevices] = {};   // calls may come from several threads; the setting may be made twice
  int dev = -1;
  IRIS_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < kDevices && done[dev].load(std::memory_order_acquire)) return IRIS_OK;
  IRIS_CUDA_TRY(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (dev < kDevices) done[dev].store(true, std::memory_order_release);
  return IRIS_OK;
}
// A matrix of rows; `stride` comes back as the elements between rows.
inline int check_matrix(const char* fn, const char* what, const void* p, int dtype, int64_t rows, int64_t columns, int64_t* stride) {
  if (*stride == 0) *stride = columns;
  if (*stride < columns) return fail(IRIS_ERR_ARG, "%s: %s: row stride %lld is less than a row's %lld elements", fn, what, (long long)*stride, (long long)columns);
  if (rows > 1 && *stride > INT64_MAX / 8 / rows) return fail(IRIS_ERR_ARG, "%s: %s: row stride %lld is too large", fn, what, (long long)*stride);
  return check_aligned(fn, what, p, elem_size(dtype), rows > 0 && columns > 0);
}

}  // namespace rows
}  // namespace iris
