// Rows that start at any element, seen by columns (not by 16-byte granules as in logit_rows.cuh), so that a thread has the same columns of every row:
// what the operators on embeddings and norms need, whose weights and sums belong to columns.
//
// A warp takes 256 columns of a row, or a few times that, through shared memory of its own.  Aligned 16 bytes are copied asynchronously, several rows
// ahead, without passing through registers; where the row begins elsewhere than at 16 bytes, each thread cuts its columns out of two of
// them there, and results go the same way back.  Nothing outside a row is written: what does not fill 16 bytes is stored by elements.  Segment reads nothing
// outside it either: its first elements are copied by words (and one by itself, where it begins at half a word), and the copy of its last 16 bytes is cut
// short.  Aligned (rows that all begin at the same place of 16 bytes) also reads what lies between two rows within the 16 bytes that one of them touches.
#pragma once

#include <atomic>

#include "logit_rows.cuh"

namespace iris {
namespace rows {

constexpr int64_t kMaxDim = 1 << 24;             // bytes of a row are counted in 32 bits
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

// The same where `a` is the same in all threads of the warp: four instructions for each instead of fifteen.
template <int U>
__device__ __forceinline__ void cut_all(uint4 (&v)[U], const uint4 (&next)[U], uint32_t a) {
  const uint32_t bits = (a & 3) * 8;
  switch (a >> 2) {
    case 0:
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = make_uint4(__funnelshift_r(v[u].x, v[u].y, bits), __funnelshift_r(v[u].y, v[u].z, bits), __funnelshift_r(v[u].z, v[u].w, bits),
                          __funnelshift_r(v[u].w, next[u].x, bits));
      break;
    case 1:
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = make_uint4(__funnelshift_r(v[u].y, v[u].z, bits), __funnelshift_r(v[u].z, v[u].w, bits), __funnelshift_r(v[u].w, next[u].x, bits),
                          __funnelshift_r(next[u].x, next[u].y, bits));
      break;
    case 2:
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = make_uint4(__funnelshift_r(v[u].z, v[u].w, bits), __funnelshift_r(v[u].w, next[u].x, bits), __funnelshift_r(next[u].x, next[u].y, bits),
                          __funnelshift_r(next[u].y, next[u].z, bits));
      break;
    default:
#pragma unroll
      for (int u = 0; u < U; ++u)
        v[u] = make_uint4(__funnelshift_r(v[u].w, next[u].x, bits), __funnelshift_r(next[u].x, next[u].y, bits), __funnelshift_r(next[u].y, next[u].z, bits),
                          __funnelshift_r(next[u].z, next[u].w, bits));
  }
}

// The 16 bytes at `at` of which [lo, hi) may be read; zeros elsewhere.  ES: bytes of an element.  (Loops, as these are rare: unrolled they cost
// the kernels registers.)
template <int ES>
__device__ __forceinline__ uint4 load_elements(const char* at, const char* lo, const char* hi) {
  uint4 v = make_uint4(0, 0, 0, 0);
#pragma unroll 1
  for (const char* p = at + 16 - ES; p >= at; p -= ES) {
    const uint32_t x = p < lo || p >= hi ? 0 : ES == 4 ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
    v = ES == 4 ? make_uint4(x, v.x, v.y, v.z)
                : make_uint4(v.x << 16 | x, __funnelshift_l(v.x, v.y, 16), __funnelshift_l(v.y, v.z, 16), __funnelshift_l(v.z, v.w, 16));
  }
  return v;
}
template <int ES>
__device__ __forceinline__ void store_elements(char* at, const char* lo, const char* hi, uint4 v) {
#pragma unroll 1
  for (char* p = at; p < at + 16; p += ES) {
    if (p >= lo && p < hi) {
      if (ES == 4) *reinterpret_cast<uint32_t*>(p) = v.x;
      else *reinterpret_cast<uint16_t*>(p) = (uint16_t)v.x;
    }
    v = ES == 4 ? make_uint4(v.y, v.z, v.w, 0)
                : make_uint4(__funnelshift_r(v.x, v.y, 16), __funnelshift_r(v.y, v.z, 16), __funnelshift_r(v.z, v.w, 16), v.w >> 16);
  }
}
// Aligned 16 bytes, as above.
template <int ES>
__device__ __forceinline__ void store16(char* at, const char* lo, const char* hi, const uint4& v) {
  if (at >= lo && at + 16 <= hi) st_global_v4(at, v);
  else store_elements<ES>(at, lo, hi, v);
}
__device__ __forceinline__ uint32_t phase(const void* p) { return (uint32_t)reinterpret_cast<uintptr_t>(p) & 15; }

// The 16 bytes from byte `b` of a row of `bytes` on, which are aligned; zeros outside the row.
template <int ES>
__device__ __forceinline__ uint4 edge_load(const char* row, int b, int bytes) {
  if (b >= 0 && b + 16 <= bytes) return ld_global_v4(row + b);
  if (b <= -16 || b >= bytes) return make_uint4(0, 0, 0, 0);
  return load_elements<ES>(row + b, row, row + bytes);
}
// The piece at `at` of the row [lo, hi), by one thread alone.
template <int ES>
__device__ __forceinline__ uint4 load_piece(const char* at, const char* lo, const char* hi) {
  const uint32_t a = phase(at);
  const char* p = at - a;
  if (a == 0) return p >= lo && p + 16 <= hi ? ld_global_v4(p) : load_elements<ES>(p, lo, hi);
  const bool inside = p >= lo && p + 32 <= hi;
  const uint4 v = inside ? ld_global_v4(p) : load_elements<ES>(p, lo, hi), next = inside ? ld_global_v4(p + 16) : load_elements<ES>(p + 16, lo, hi);
  return cut(v, next, a);
}

__device__ __forceinline__ uint4 ld_shared_v4(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
// `bytes` <= 16 of 16, the rest zeros.
__device__ __forceinline__ void copy_async_part(uint32_t shared, const void* global, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(shared), "l"(global), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async_word(uint32_t shared, const void* global) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(shared), "l"(global) : "memory");
}
__device__ __forceinline__ void copy_async_pair(uint32_t shared, const float* global) {   // 8-byte aligned
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(shared), "l"(global) : "memory");
}
__device__ __forceinline__ uint64_t ld_shared_u64(uint32_t at) {
  uint64_t v;
  asm volatile("ld.shared.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait_but() {   // until at most N groups of this thread are under way
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A thread's 8 columns of a type.
template <int DT>
struct Columns {
  using E = Elem<DT>;
  static constexpr int ES = sizeof(typename E::T), N = kLaneColumns / E::VE;   // N: times 16 bytes
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
  // As pairs, for arithmetic on two at once.
  static __device__ __forceinline__ void unpack2(const uint4* v, uint64_t (&x)[kLaneColumns / 2]) {
    float y[kLaneColumns];
    unpack(v, y);
#pragma unroll
    for (int e = 0; e < kLaneColumns / 2; ++e) x[e] = pair(y[2 * e], y[2 * e + 1]);
  }
  static __device__ __forceinline__ void pack2(const uint64_t (&x)[kLaneColumns / 2], uint4* v) {
    float y[kLaneColumns];
#pragma unroll
    for (int e = 0; e < kLaneColumns / 2; ++e) {
      const float2 f = unpair(x[e]);
      y[2 * e] = f.x;
      y[2 * e + 1] = f.y;
    }
    pack(y, v);
  }
  // Straight from memory: columns `first` ... of a vector of `dim`, zeros behind its end.
  static __device__ __forceinline__ void load(const char* row, int first, int dim, float (&x)[kLaneColumns]) {
    uint4 v[N];
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = load_piece<ES>(row + first * ES + n * 16, row, row + dim * ES);
    unpack(v, x);
  }
};

// I times 256 columns of a row, from column `begin`, in a warp's shared memory at `at` (16-byte aligned, kBytes): bytes from the aligned 16
// in which they begin.  ALIGNED: rows begin at 16 bytes, and their lengths are multiples of that.
template <int DT, int I, bool ALIGNED = false>
struct Segment {
  using C = Columns<DT>;
  static constexpr int ES = C::ES, N = C::N, kColumns = I * kWarpColumns, kBytes = kColumns * ES + 32;
  // Starts the copies.  An element that begins at half a word, if there is one, comes back with its place in shared memory, where `settle` puts it; later,
  // so that nobody waits for it here.
  struct Lone {
    uint32_t at = 0;   // 0: none
    uint16_t value;
    __device__ __forceinline__ void settle() {
      if (at) asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(value) : "memory");
      at = 0;
    }
  };
  static __device__ __forceinline__ void fetch(uint32_t at, const char* row, int begin, int dim, Lone& lone) {
    const int lane = threadIdx.x & 31, bytes = dim * ES, start = begin * ES;
    if constexpr (ALIGNED) {
      const char* const p = row + start + lane * 16;
      const int left = bytes - start - lane * 16;
#pragma unroll
      for (int k = 0; k < I * N; ++k)
        if (begin + kColumns <= dim || k * 512 < left) copy_async(at + (k * 32 + lane) * 16, p + k * 512);
        else ptx::st_shared_v4(at + (k * 32 + lane) * 16, make_uint4(0, 0, 0, 0));
      return;
    }
    const int a = (int)phase(row + start);
    const char* const somewhere = row - phase(row);   // aligned, for copies of 0 bytes
    if (begin + kColumns <= dim) {
      const char* const p = row + (start - a + lane * 16);
#pragma unroll
      for (int k = 0; k < I * N; ++k)
        if (k || start - a + lane * 16 >= 0) copy_async(at + (k * 32 + lane) * 16, p + k * 512);
    } else {
#pragma unroll
      for (int k = 0; k < I * N; ++k) {
        const int g = k * 32 + lane, from = start - a + g * 16;   // counted from the row's first byte
        if (from >= 0) copy_async_part(at + g * 16, from < bytes ? row + from : somewhere, max(0, min(16, bytes - from)));
      }
    }
    if (a == 0) return;
    if (lane == 0) {
      const int from = start - a + I * N * 512;
      copy_async_part(at + I * N * 512, from < bytes ? row + from : somewhere, max(0, min(16, bytes - from)));
    }
    if (begin == 0) {   // the row's first elements
      const int word = (a + 3) / 4 + lane, from = word * 4 - a;
      if (word < 4) {
        if (from + 4 <= bytes) copy_async_word(at + word * 4, row + from);
        else if (from < bytes) asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + word * 4), "h"(*reinterpret_cast<const uint16_t*>(row + from)) : "memory");
      }
      if (ES == 2 && lane == 0 && (a & 2)) {
        lone.at = at + a;
        lone.value = *reinterpret_cast<const uint16_t*>(row);
      }
    }
  }
  // Run i of the thread's columns; zeros behind the row's end.  After a barrier of the warp behind the copies and `settle`.
  static __device__ __forceinline__ void read(uint32_t at, const char* row, int begin, int dim, int i, uint64_t (&x)[kLaneColumns / 2]) {
    const uint32_t a = ALIGNED ? 0 : phase(row + begin * ES);
    uint4 v[N];
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = ld_shared_v4(at + (i * 32 + (threadIdx.x & 31)) * N * 16 + n * 16);
    if (a) {
      uint4 next[N];
#pragma unroll
      for (int n = 0; n < N; ++n) next[n] = n + 1 < N ? v[n + 1 < N ? n + 1 : 0] : ld_shared_v4(at + (i * 32 + (threadIdx.x & 31)) * N * 16 + n * 16 + 16);
      cut_all(v, next, a);
    }
    if (a && dim * ES < 16) {   // the copies have left nothing behind the end of such a row
#pragma unroll
      for (int n = 0; n < N; ++n) {
        uint32_t w[4] = {v[n].x, v[n].y, v[n].z, v[n].w};
        const int there = dim - begin - i * kWarpColumns - (int)(threadIdx.x & 31) * kLaneColumns - n * C::E::VE;
#pragma unroll
        for (int e = 0; e < C::E::VE; ++e)
          if (e >= there) w[e * ES / 4] &= ES == 4 ? 0u : e % 2 ? 0xffffu : 0xffff0000u;
        v[n] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    C::unpack2(v, x);
  }
  // Stores the threads' columns; `at`: kBytes of the warp's shared memory that nobody reads any more.
  static __device__ __forceinline__ void write(uint32_t at, char* row, int begin, int dim, const uint4 (&v)[I * N]) {
    const int lane = threadIdx.x & 31, bytes = min(dim - begin, kColumns) * ES;   // of the segment
    if (bytes <= 0) return;
    char* const to = row + begin * ES;
    const int a = ALIGNED ? 0 : (int)phase(to);
    if (ALIGNED || (a == 0 && bytes % 16 == 0)) {
#pragma unroll
      for (int k = 0; k < I * N; ++k) {
        const int b = ((k / N * 32 + lane) * N + k % N) * 16;
        if (b < bytes) st_global_v4(to + b, v[k]);
      }
      return;
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < I * N; ++k) ptx::st_shared_v4(at + 16 + ((k / N * 32 + lane) * N + k % N) * 16, v[k]);
    __syncwarp();
    uint4 w[I * N];
    if (a) {
      uint4 next[I * N];
#pragma unroll
      for (int k = 0; k < I * N; ++k) {
        w[k] = ld_shared_v4(at + (k * 32 + lane) * 16);
        next[k] = ld_shared_v4(at + (k * 32 + lane) * 16 + 16);
      }
      cut_all(w, next, 16 - a);
    } else {
#pragma unroll
      for (int k = 0; k < I * N; ++k) w[k] = ld_shared_v4(at + (k * 32 + lane) * 16 + 16);
    }
#pragma unroll
    for (int k = 0; k < I * N; ++k) {
      const int b = (k * 32 + lane) * 16 - a;
      if (b >= 0 && b + 16 <= bytes) st_global_v4(to + b, w[k]);
    }
    // what does not fill 16 bytes: at the begin (if it is not aligned) and at the end, an element a thread
    const int head = a ? min(16 - a, bytes) : 0, end = ((bytes + a) & ~15) - a;
    const int b = lane < 8 ? lane * ES : end + (lane - 8) * ES;
    if (lane < 8 ? b < head : end >= 0 && lane < 16 && b < bytes) {
      if (ES == 4) {
        uint32_t x;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at + 16 + b) : "memory");
        *reinterpret_cast<uint32_t*>(to + b) = x;
      } else {
        uint16_t x;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at + 16 + b) : "memory");
        *reinterpret_cast<uint16_t*>(to + b) = x;
      }
    }
  }
};

__device__ __forceinline__ uint32_t ones_below(int bit) {   // of a word; none below 0, all from 32 on
  uint32_t m;
  asm("bmsk.clamp.b32 %0, 0, %1;" : "=r"(m) : "r"(max(0, bit)));
  return m;
}
// Bytes lo .. hi - 1 of 16, zeros elsewhere.
__device__ __forceinline__ uint4 between(const uint4& v, int lo, int hi) {
  lo *= 8;
  hi *= 8;
  return make_uint4(v.x & ones_below(hi) & ~ones_below(lo), v.y & ones_below(hi - 32) & ~ones_below(lo - 32),
                    v.z & ones_below(hi - 64) & ~ones_below(lo - 64), v.w & ones_below(hi - 96) & ~ones_below(lo - 96));
}
// Elements of v from byte lo on and before byte hi, to `at` + their place.
template <int ES>
__device__ __forceinline__ void store_between(char* at, const uint4& v, int lo, int hi) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 16 / ES; ++e)
    if (e * ES >= lo && e * ES < hi) {
      if (ES == 4) *reinterpret_cast<uint32_t*>(at + e * ES) = w[e * ES / 4];
      else *reinterpret_cast<uint16_t*>(at + e * ES) = (uint16_t)(w[e * ES / 4] >> (e % 2 * 16));
    }
}
// The same for rows that all begin at the same place of 16 bytes (`ph`, in bytes): columns are counted from the aligned 16 bytes in which a row begins, so
// that no piece has to be cut.  row: that place; dim: columns counted so, up to the row's end; the first ph / ES of them are not the row's.
// Of the aligned 16 bytes in which a row begins or ends, all are read, as they lie between the matrix's rows; but not in front of the first row and behind
// the last one (`first`, `last`).
template <int DT, int I>
struct Aligned {
  using C = Columns<DT>;
  using Lone = typename Segment<DT, I>::Lone;
  static constexpr int ES = C::ES, N = C::N, VE = C::E::VE, kColumns = I * kWarpColumns, kBytes = kColumns * ES;
  static __device__ __forceinline__ bool whole(int begin, int dim, int ph) { return (begin > 0 || ph == 0) && begin + kColumns <= dim; }   // all are the row's
  static __device__ __forceinline__ void fetch(uint32_t at, const char* row, int begin, int dim, int ph, bool first, bool last, Lone& lone) {
    const int lane = threadIdx.x & 31;
    const char* const p = row + begin * ES + lane * 16;
    const int left = dim * ES - begin * ES - lane * 16;
    const bool careful = (first && ph) || (last && dim * ES % 16);
    if (!careful) {
#pragma unroll
      for (int k = 0; k < I * N; ++k)
        if (k * 512 < left) copy_async(at + (k * 32 + lane) * 16, p + k * 512);
        else ptx::st_shared_v4(at + (k * 32 + lane) * 16, make_uint4(0, 0, 0, 0));
      return;
    }
#pragma unroll 1
    for (int k = 0; k < I * N; ++k) {
      if (k == 0 && first && ph && begin + lane == 0) continue;
      if (k * 512 < left) copy_async_part(at + (k * 32 + lane) * 16, p + k * 512, last ? min(16, left - k * 512) : 16);
      else ptx::st_shared_v4(at + (k * 32 + lane) * 16, make_uint4(0, 0, 0, 0));
    }
    if (first && ph && begin == 0) {   // the row's first elements
      const int from = lane * 4, bytes = dim * ES;
      if (lane < 4 && from + 4 > ph && from < bytes) {
        if (from >= ph && from + 4 <= bytes) {
          copy_async_word(at + from, row + from);
        } else if (ES == 2) {   // half a word
          const int half = from >= ph ? from : from + 2;
          if (half < bytes) {
            lone.at = at + half;
            lone.value = *reinterpret_cast<const uint16_t*>(row + half);
          }
        }
      }
    }
  }
  static __device__ __forceinline__ void read(uint32_t at, int begin, int dim, int ph, int i, uint64_t (&x)[kLaneColumns / 2]) {
    const int lane = threadIdx.x & 31;
    uint4 v[N];
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = ld_shared_v4(at + ((i * 32 + lane) * N + n) * 16);
    // Zeros where a column is not the row's; 16 bytes that lie behind it altogether are 0 already.
    const int from = (begin + i * kWarpColumns) * ES, bytes = dim * ES;
    if ((i == 0 && begin == 0 && ph) || (from < bytes && bytes < from + kWarpColumns * ES && bytes % 16)) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int b = from + (lane * N + n) * 16;
        if (b < ph || (b < bytes && bytes < b + 16)) v[n] = between(v[n], ph - b, bytes - b);
      }
    }
    C::unpack2(v, x);
  }
  static __device__ __forceinline__ void write(char* row, int begin, int dim, int ph, const uint4 (&v)[I * N]) {
    const int lane = threadIdx.x & 31;
    char* const p = row + (begin + lane * kLaneColumns) * ES;
    if (whole(begin, dim, ph)) {
#pragma unroll
      for (int k = 0; k < I * N; ++k) st_global_v4(p + k / N * kWarpColumns * ES + k % N * 16, v[k]);
      return;
    }
    // The 16 bytes in which the row begins, and those in which it ends, by elements.
    const int from = begin * ES + lane * (N * 16), bytes = dim * ES;
    uint4 end = v[0];
    int end_at = -1;
#pragma unroll
    for (int k = 0; k < I * N; ++k) {
      const int b = from + k / N * (kWarpColumns * ES) + k % N * 16;
      if (k == 0 && b < ph) continue;
      if (b + 16 <= bytes) {
        st_global_v4(row + b, v[k]);
      } else if (b < bytes) {
        end = v[k];
        end_at = b;
      }
    }
    if (end_at >= 0) store_between<ES>(row + end_at, end, 0, bytes - end_at);
    if (from < ph) store_between<ES>(row, v[0], ph, bytes);
  }
};

// ---- host side -----------------------------------------------------------------------------------------------------
// Lets a kernel have up to `bytes` of dynamic shared memory on the current device, and clusters of more than 8 blocks, once.
template <auto KERNEL>
inline int allow_shared(int bytes, bool large_clusters = false) {
  constexpr int kDevices = 64;
  static std::atomic<bool> done[kDevices] = {};   // calls may come from several threads; the setting may be made twice
  int dev = -1;
  IRIS_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < kDevices && done[dev].load(std::memory_order_acquire)) return IRIS_OK;
  IRIS_CUDA_TRY(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (large_clusters) IRIS_CUDA_TRY(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  if (dev < kDevices) done[dev].store(true, std::memory_order_release);
  return IRIS_OK;
}
// How many clusters of `split` blocks (a power of two, at most 8) of a kernel whose blocks have an SM to themselves are there at once: an SM that is left over in its
// part of the chip has none, so that clusters of 4 and 8 do not get all of them (33 and 15; blocks that stay and take rows in turn took
// up to twice as long with 37 and 18 clusters: 2048 x 32768 131 us instead of 79).  threads, bytes: the kernel's most.
template <auto KERNEL>
inline int clusters_at_once(int split, int threads, int bytes, int* clusters) {
  constexpr int kDevices = 64, kSplits = 4;
  static std::atomic<int> known[kDevices][kSplits] = {};
  int dev = -1, which = 0;
  if (split == 1) {
    *clusters = kSms;
    return IRIS_OK;
  }
  while (1 << which < split) ++which;
  IRIS_CUDA_TRY(cudaGetDevice(&dev));
  int n = dev < kDevices ? known[dev][which].load(std::memory_order_acquire) : 0;
  if (!n) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)split);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)bytes;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    IRIS_CUDA_TRY(cudaOccupancyMaxActiveClusters(&n, KERNEL, &cfg));
    n = n < 1 ? 1 : n > kSms / split ? kSms / split : n;
    if (dev < kDevices) known[dev][which].store(n, std::memory_order_release);
  }
  *clusters = n;
  return IRIS_OK;
}
// Whether rows `stride` bytes apart all begin at 16 bytes.
inline bool aligned_rows(const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 16 == 0; }
// A matrix of rows; `stride` comes back as the elements between rows.
inline int check_matrix(const char* fn, const char* what, const void* p, int dtype, int64_t rows, int64_t columns, int64_t* stride) {
  if (*stride == 0) *stride = columns;
  if (*stride < columns) return fail(IRIS_ERR_ARG, "%s: %s: row stride %lld is less than a row's %lld elements", fn, what, (long long)*stride, (long long)columns);
  if (rows > 1 && *stride > INT64_MAX / 8 / rows) return fail(IRIS_ERR_ARG, "%s: %s: row stride %lld is too large", fn, what, (long long)*stride);
  return check_aligned(fn, what, p, elem_size(dtype), rows > 0 && columns > 0);
}

}  // namespace rows
}  // namespace iris
