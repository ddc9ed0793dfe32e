// What the operators on rows of logits share: element types, 16-byte pieces of a row that may start at any element,
// the running softmax statistics and their reductions, and the argument checks.
//
// A row of `vocab` elements starts at any multiple of the element size.  Its memory is seen as 16-byte granules: with
// `ph` = the row's first element's place in its granule, granule v holds columns v*VE - ph ... v*VE - ph + VE - 1.
// Granules that lie inside the row are moved with one 16-byte access, the first and the last one, where the row covers
// them in part, element by element: nothing outside the row is read or written.
#pragma once

#include <cfloat>
#include <cmath>
#include <type_traits>

#include "iris_device.cuh"
#include "sm100_ptx.cuh"

namespace iris {
namespace rows {

constexpr int kMaxList = 128;               // targets, alternatives or teacher's tokens of one row
constexpr int64_t kMaxVocab = 1 << 30;      // columns are counted in 32 bits inside a row
constexpr int kSms = 148;                    // of a B200
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kMaxScale = 2e38f;           // times log2(e) it is in the type's range, so that times a difference of 0 it is 0
constexpr float kFloor = -1024.f;           // exponents (base 2) are cut here: 2^-1024 is 0 in 32 bits, and 0 * -1024 is not NaN

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two 32-bit floats at once (one instruction on sm_100a).
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t add2f(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2f(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2f(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// 16 bytes that are read once: not kept in L1.  Volatile, with memory clobbered: it must not move ahead of the wait for the
// kernel before, nor behind a store where the gradient replaces the logits.
__device__ __forceinline__ uint4 ld_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
// 16 bytes to shared memory without passing through registers; visible to the copying thread after copy_async_wait, to
// the block after a barrier behind that.
__device__ __forceinline__ void copy_async(uint32_t shared, const void* global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(shared), "l"(global) : "memory");
}
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// The larger of two, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// An element type.  VE: elements of a granule; kMasked: 32 bits of -inf; kLowest: about the lowest finite value; fold(): a
// granule's largest values in two halves, larger() of two such, unfold() the larger half, NaN if one is; at_least(): none
// below floor, which is twice() a value, NaN stays; ordinal() and value(): below.
template <int DT> struct Elem;
template <> struct Elem<IRIS_F16> {
  using T = __half;
  static constexpr int VE = 8;
  static constexpr uint32_t kMasked = 0xfc00fc00u;
  static constexpr float kLowest = -65504.f;
  static __device__ __forceinline__ uint32_t twice(float x) {
    const __half2 h = __floats2half2_rn(x, x);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  // A number that orders the type's values, 0 below all of them, the largest for NaN, and back.
  static __device__ __forceinline__ uint32_t ordinal(float x) {
    const uint32_t b = (uint32_t)__half_as_ushort(__float2half_rn(x + 0.f));   // -0 counts as +0
    return x != x ? 0xffffu : b & 0x8000u ? ~b & 0xffffu : b | 0x8000u;
  }
  static __device__ __forceinline__ float value(uint32_t n) {
    const uint32_t b = n & 0x8000u ? n & 0x7fffu : ~n & 0xffffu;
    return n == 0xffffu ? NAN : __half2float(__ushort_as_half((unsigned short)b));
  }
  static __device__ __forceinline__ uint4 at_least(uint4 v, uint32_t floor) {
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(v.x) : "r"(floor));
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(v.y) : "r"(floor));
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(v.z) : "r"(floor));
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(v.w) : "r"(floor));
    return v;
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  }
  static __device__ __forceinline__ uint32_t fold(const uint4& v) { return larger(larger(v.x, v.y), larger(v.z, v.w)); }
  static __device__ __forceinline__ float unfold(uint32_t m) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return max_nan(f.x, f.y);
  }
  static __device__ __forceinline__ float to(T x) { return __half2float(x); }
  static __device__ __forceinline__ T from(float x) { return __float2half_rn(x); }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Elem<IRIS_BF16> {
  using T = __nv_bfloat16;
  static constexpr int VE = 8;
  static constexpr uint32_t kMasked = 0xff80ff80u;
  static constexpr float kLowest = -3.38e38f;
  static __device__ __forceinline__ uint32_t twice(float x) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, x);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  // A number that orders the type's values, 0 below all of them, the largest for NaN, and back.
  static __device__ __forceinline__ uint32_t ordinal(float x) {
    const uint32_t b = __float_as_uint(x + 0.f) >> 16;   // -0 counts as +0
    return x != x ? 0xffffu : b & 0x8000u ? ~b & 0xffffu : b | 0x8000u;
  }
  static __device__ __forceinline__ float value(uint32_t n) {
    const uint32_t b = n & 0x8000u ? n & 0x7fffu : ~n & 0xffffu;
    return n == 0xffffu ? NAN : __uint_as_float(b << 16);
  }
  static __device__ __forceinline__ uint4 at_least(uint4 v, uint32_t floor) {
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.x) : "r"(floor));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.y) : "r"(floor));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.z) : "r"(floor));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.w) : "r"(floor));
    return v;
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  }
  static __device__ __forceinline__ uint32_t fold(const uint4& v) { return larger(larger(v.x, v.y), larger(v.z, v.w)); }
  static __device__ __forceinline__ float unfold(uint32_t m) {
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  static __device__ __forceinline__ float to(T x) { return __bfloat162float(x); }
  static __device__ __forceinline__ T from(float x) { return __float2bfloat16_rn(x); }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Elem<IRIS_F32> {
  using T = float;
  static constexpr int VE = 4;
  static constexpr uint32_t kMasked = 0xff800000u;
  static constexpr float kLowest = -3.38e38f;
  static __device__ __forceinline__ uint32_t twice(float x) { return __float_as_uint(x); }
  static __device__ __forceinline__ uint32_t ordinal(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return x != x ? ~0u : b & 0x80000000u ? ~b : b | 0x80000000u;
  }
  static __device__ __forceinline__ float value(uint32_t n) { return n == ~0u ? NAN : __uint_as_float(n & 0x80000000u ? n & 0x7fffffffu : ~n); }
  static __device__ __forceinline__ uint4 at_least(const uint4& v, uint32_t floor) {
    const float f = __uint_as_float(floor);
    return make_uint4(__float_as_uint(max_nan(__uint_as_float(v.x), f)), __float_as_uint(max_nan(__uint_as_float(v.y), f)),
                      __float_as_uint(max_nan(__uint_as_float(v.z), f)), __float_as_uint(max_nan(__uint_as_float(v.w), f)));
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b))); }
  static __device__ __forceinline__ uint32_t fold(const uint4& v) { return larger(larger(v.x, v.y), larger(v.z, v.w)); }
  static __device__ __forceinline__ float unfold(uint32_t m) { return __uint_as_float(m); }
  static __device__ __forceinline__ float to(T x) { return x; }
  static __device__ __forceinline__ T from(float x) { return x; }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};

template <int DT>
__device__ __forceinline__ float largest(const uint4& g) {
  return Elem<DT>::unfold(Elem<DT>::fold(g));
}
// Of the granules g[u] with u * T < left (all of them if ALL); -inf if there are none.
template <int DT, bool ALL, int U>
__device__ __forceinline__ float largest(const uint4 (&g)[U], int left, int T) {
  uint32_t m = Elem<DT>::kMasked;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (ALL || u * T < left) m = ALL && u == 0 ? Elem<DT>::fold(g[0]) : Elem<DT>::larger(m, Elem<DT>::fold(g[u]));
  return Elem<DT>::unfold(m);
}

// The granule with -inf in the places whose bit is set.
template <int DT>
__device__ __forceinline__ uint4 without(const uint4& g, uint32_t bits) {
  float x[Elem<DT>::VE];
  Elem<DT>::unpack(g, x);
#pragma unroll
  for (int e = 0; e < Elem<DT>::VE; ++e) x[e] = bits >> e & 1 ? -INFINITY : x[e];
  return Elem<DT>::pack(x);
}

// A row of the logits (or of the gradient) as granules.
template <int DT>
struct Row {
  using E = Elem<DT>;
  using T = typename E::T;
  static constexpr int VE = E::VE;
  T* granule0;   // 16-byte aligned; the row's element 0 is granule0[ph]
  int ph, end;   // elements ph .. end - 1 counted from granule0 belong to the row
  __device__ __forceinline__ Row(const void* base, int64_t row, int64_t stride, int vocab) {
    T* p = static_cast<T*>(const_cast<void*>(base)) + row * stride;
    ph = (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    granule0 = p - ph;
    end = ph + vocab;
  }
  __device__ __forceinline__ int granules() const { return (end + VE - 1) / VE; }
  __device__ __forceinline__ bool whole(int v) const { return v * VE >= ph && (v + 1) * VE <= end; }
  __device__ __forceinline__ T* at(int v) const { return granule0 + (int64_t)v * VE; }
  __device__ __forceinline__ T& column(int j) const { return granule0[ph + (int64_t)j]; }
  // The granule's bits; -inf in the places that do not belong to the row.
  __device__ __forceinline__ uint4 raw(int v) const {
    if (whole(v)) return ld_once(at(v));
    float x[VE];
    load(v, x);
    return E::pack(x);
  }
  // The granule's values, likewise.
  __device__ __forceinline__ void load(int v, float (&x)[VE]) const {
    if (whole(v)) {
      E::unpack(ld_global_v4(at(v)), x);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int i = v * VE + e;
        x[e] = i >= ph && i < end ? E::to(granule0[i]) : -INFINITY;
      }
    }
  }
};

// What a block does of a row: granules [v0, v1).  Counted i = 0 .. n_all - 1 so that those that lie inside the row come
// first (n_int of them, w0 + i), and what the row covers in part, at most two, comes last.
template <int DT>
struct Part {
  static constexpr int VE = Elem<DT>::VE;
  int v0, v1, w0, n_int, n_all;
  __device__ __forceinline__ Part(const Row<DT>& row, int part, int each) {   // each: granules of a part, the last ones have fewer
    const int nv = row.granules();
    v0 = min(nv, part * each);
    v1 = min(nv, v0 + each);
    w0 = v0 + (v0 < v1 && v0 * VE < row.ph);
    n_int = v1 - (v1 > w0 && v1 * VE > row.end) - w0;
    n_all = v1 - v0;
  }
  __device__ __forceinline__ int granule(int i) const { return i < n_int ? w0 + i : v0 < w0 && i == n_int ? v0 : v1 - 1; }
  __device__ __forceinline__ int place(int v) const { return v < w0 ? n_int : v < w0 + n_int ? v - w0 : n_all - 1; }
  __device__ __forceinline__ bool has(int element) const { return element >= v0 * VE && element < v1 * VE; }   // counted from granule0
  __device__ __forceinline__ uint4 raw(const Row<DT>& row, int i) const { return i < n_int ? ld_once(row.at(w0 + i)) : row.raw(granule(i)); }
};

// Running statistics of a set of logits: m >= every one of them (and >= -FLT_MAX, so that z - m is never inf - inf for
// a masked z), s = sum 2^y, t = sum y 2^y, y = (z - m) k cut at about kFloor, k = scale log2(e).
struct Acc {
  float m = -FLT_MAX, s = 0.f, t = 0.f;
  __device__ __forceinline__ void rebase(float mx, float k) {   // to another m, if not too far below
    const float d = max_nan((m - mx) * k, kFloor), f = ex2(d);
    t = __fmul_rn(fmaf(s, d, t), f);
    s = __fmul_rn(s, f);
    m = mx;
  }
  __device__ __forceinline__ void merge(const Acc& o, float k) {
    Acc b = o;
    const float mx = max_nan(m, o.m);
    rebase(mx, k);
    b.rebase(mx, k);
    s = __fadd_rn(s, b.s);
    t = __fadd_rn(t, b.t);
  }
  __device__ __forceinline__ void add_one(float z, float k) { merge(Acc{max_nan(z, -FLT_MAX), z == -INFINITY ? 0.f : z == z && z != INFINITY ? 1.f : NAN, 0.f}, k); }
};

// The lowest logit that has to be told apart: one below low(m, k) has 2^y = 0 and is lifted to it, so that y 2^y is 0 and
// not NaN for -inf.  Rounding to the type leaves it well below m (by 1000 / k and 1 / 64 of itself).  False where the type
// has no such value (masks of the lowest finite value and nothing above them, scales beyond the type's range): then y is
// cut instead.
template <int DT>
__device__ __forceinline__ bool lift_floor(float m, float k, uint32_t& word) {
  const float z = m + kFloor / k, low = z - fabsf(z) * (1.f / 64);
  word = Elem<DT>::twice(low);
  return low >= Elem<DT>::kLowest && low * k > -1e38f && m * k < 1e38f && k < 1e8f;
}

// A thread's statistics of granules, counted from a logit near the largest: it is raised only when one comes that is
// 2^kSlack times as probable, so that in most rows it is the largest of the first batch and the sums need no further care.
// 2^24 times 2^30 columns is far from overflow, and s loses nothing by larger terms; t does, as s kSlack is taken from it in
// the end: its slack is 8 (entropies of 4096 x 128000: 1.1e-6 off with a slack of 24, 1e-7 with 8; 2 takes 4 % longer).  Per element one
// instruction to unpack, half of one each to subtract, scale and add, and the exponential; with the entropy half of one each
// for the lift (on packed 16-bit values) and the second sum.
//
// Sums are taken in two levels, as each addition rounds, and equal terms round to the same side (a chain of 4096 terms 0.7: 3e-5 off): pace() ends
// a chain of at most 128 terms in each of two halves.  LONG, for parts of any length: the sums above them keep what their additions lose, so that a
// row of 2^30 columns is as near as a short one.  They lie in shared memory, as they are seldom touched: in registers they made the kernels spill
// (1 to 4 %).
template <int DT, bool ENTROPY, bool LONG>
struct Sums {
  static constexpr float kSlack = ENTROPY ? 8.f : 24.f;
  Acc a;           // LONG: s and t in the end
  float4* upper;   // LONG: s, t, and what the additions to them lost
  float k, top = -FLT_MAX;   // top: the largest logit so far
  bool lift = false;
  uint32_t floor = 0;
  uint64_t s2 = 0, t2 = 0;   // sums of even and odd places since the last raise
  uint64_t k2, minus_m2;
  __device__ __forceinline__ Sums(float k_, float4* upper_) : upper(upper_), k(k_), k2(pair(k_, k_)), minus_m2(pair(FLT_MAX, FLT_MAX)) {
    if (LONG) *upper = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  static __device__ __forceinline__ void add_exactly(float& sum, float& lost, float x) {
    const float more = __fadd_rn(x, lost), to = __fadd_rn(sum, more);
    lost = __fsub_rn(more, __fsub_rn(to, sum));
    sum = to;
  }
  __device__ __forceinline__ void flush() {
    const float2 s = unpair(s2), t = unpair(t2);
    s2 = t2 = 0;
    if (LONG) {
      float4 u = *upper;
      add_exactly(u.x, u.z, s.x + s.y);
      if (ENTROPY) add_exactly(u.y, u.w, t.x + t.y);
      *upper = u;
    } else {
      a.s += s.x + s.y;
      if (ENTROPY) a.t += t.x + t.y;
    }
  }
  __device__ __forceinline__ void rebase(float mx) {
    flush();
    if (LONG) {
      a.s = upper->x;
      a.t = upper->y;
    }
    a.rebase(mx, k);
    if (LONG) *upper = make_float4(a.s, a.t, 0.f, 0.f);
  }
  // Before a batch of U granules of every thread that begins at granule b = i T U of its loop.
  template <int T, int U>
  __device__ __forceinline__ void pace(int b) {
    constexpr int kBatches = 128 / (U * Elem<DT>::VE / 2);
    static_assert((kBatches & (kBatches - 1)) == 0 && (T * U & (T * U - 1)) == 0, "powers of two");
    if ((b & (kBatches * T * U - 1)) == 0) flush();
  }
  __device__ __forceinline__ void raise(float mx) {   // before adding logits of which mx is the largest
    top = max_nan(top, mx);
    if ((mx - a.m) * k <= kSlack) return;
    rebase(max_nan(a.m, mx));
    minus_m2 = pair(-a.m, -a.m);
    if (ENTROPY) lift = lift_floor<DT>(a.m, k, floor);
  }
  __device__ __forceinline__ Acc done() {   // counted from the largest logit
    rebase(top);
    return a;
  }
  __device__ __forceinline__ void add_lifted(const uint4& g) {
    constexpr int VE = Elem<DT>::VE;
    float x[VE];
    Elem<DT>::unpack(ENTROPY ? Elem<DT>::at_least(g, floor) : g, x);
#pragma unroll
    for (int e = 0; e < VE; e += 2) {
      const uint64_t y2 = mul2f(add2f(pair(x[e], x[e + 1]), minus_m2), k2);
      const float2 y = unpair(y2);
      const uint64_t f = pair(ex2(y.x), ex2(y.y));
      s2 = add2f(s2, f);
      if (ENTROPY) t2 = fma2f(f, y2, t2);
    }
  }
  __device__ __forceinline__ void add_cut(const uint4& g) {
    constexpr int VE = Elem<DT>::VE;
    float x[VE];
    Elem<DT>::unpack(g, x);
#pragma unroll
    for (int e = 0; e < VE; e += 2) {
      const float y0 = max_nan((x[e] - a.m) * k, kFloor), y1 = max_nan((x[e + 1] - a.m) * k, kFloor);
      const uint64_t f = pair(ex2(y0), ex2(y1));
      s2 = add2f(s2, f);
      t2 = fma2f(f, pair(y0, y1), t2);
    }
  }
  // Granules g[0 .. U), the first `left` of every T-th (all of them if ALL), of which mx is the largest logit.
  template <bool ALL, int U>
  __device__ __forceinline__ void add(const uint4 (&g)[U], float mx, int left = 0, int T = 1) {
    raise(mx);
    if (!ENTROPY || lift) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (ALL || u * T < left) add_lifted(g[u]);
    } else if (mx != -INFINITY) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (ALL || u * T < left) add_cut(g[u]);
    }
  }
};

// Calls f(b, all) for batches b of T * U consecutive granules until n: with std::true_type for whole ones, of which thread
// tid has granules b + u * T + tid, then with std::false_type for the rest, where f looks which of its own are below n.
template <int T, int U, class F>
__device__ __forceinline__ void batches(int n, F f) {
  int b = 0;
  for (; b + T * U <= n; b += T * U) f(b, std::true_type{});
  if (b < n) f(b, std::false_type{});
}

__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

// All threads of a block of W warps (a power of two) get the merged statistics, the same bits: warp_share, a barrier,
// warps_join.
template <int W>
struct Warps {
  Acc of[W];
};
template <bool ENTROPY, int W>
__device__ __forceinline__ void warp_share(Acc a, float k, Warps<W>& buf) {
  a.rebase(warp_max(a.m), k);
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, o);
    if (ENTROPY) a.t += __shfl_xor_sync(~0u, a.t, o);
  }
  if ((threadIdx.x & 31) == 0) buf.of[threadIdx.x >> 5] = a;
}
template <bool ENTROPY, int W>
__device__ __forceinline__ Acc warps_join(float k, const Warps<W>& buf) {
  Acc a = buf.of[threadIdx.x & (W - 1)];
  a.rebase(warp_max(a.m), k);
#pragma unroll
  for (int o = W / 2; o; o >>= 1) {
    a.s += __shfl_xor_sync(~0u, a.s, o);
    if (ENTROPY) a.t += __shfl_xor_sync(~0u, a.t, o);
  }
  return a;
}

// ln sum exp(scale (z - m)): -inf where no logit is left.
__device__ __forceinline__ float log_sum(const Acc& a) { return a.s > 0.f ? logf(a.s) : a.s == 0.f ? -INFINITY : NAN; }

// A larger logit, and among equal ones the lower column, has the larger key; 0 is no logit's.  NaN comes above +inf.
template <int DT>
__device__ __forceinline__ uint64_t order_key(float x, int column) {
  return (uint64_t)Elem<DT>::ordinal(x) << 32 | (0xffffffffu - (uint32_t)column);
}
__device__ __forceinline__ int key_column(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }
template <int DT>
__device__ __forceinline__ float key_value(uint64_t key) {
  return Elem<DT>::value((uint32_t)(key >> 32));
}

// ---- host side -----------------------------------------------------------------------------------------------------
inline size_t elem_size(int dtype) { return dtype == IRIS_F32 ? 4 : 2; }

// Checks shared by all calls; `stride` comes back as the elements between rows.
inline int check_logits(const char* fn, const char* what, const void* p, int dtype, int64_t rows, int64_t vocab, int64_t* stride) {
  if (dtype != IRIS_F16 && dtype != IRIS_BF16 && dtype != IRIS_F32) return fail(IRIS_ERR_ARG, "%s: unknown dtype %d", fn, dtype);
  if (rows < 0 || vocab < 0) return fail(IRIS_ERR_ARG, "%s: rows=%lld, vocab=%lld", fn, (long long)rows, (long long)vocab);
  if (vocab > kMaxVocab || rows > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "%s: at most 2^31 - 1 rows of 2^30 columns", fn);
  if (*stride == 0) *stride = vocab;
  if (*stride < vocab) return fail(IRIS_ERR_ARG, "%s: %s: row stride %lld is less than vocab %lld", fn, what, (long long)*stride, (long long)vocab);
  if (rows > 1 && *stride > INT64_MAX / 8 / rows) return fail(IRIS_ERR_ARG, "%s: %s: row stride %lld is too large", fn, what, (long long)*stride);
  if (rows == 0 || vocab == 0) return IRIS_OK;
  if (!p) return fail(IRIS_ERR_ARG, "%s: %s is NULL", fn, what);
  if (reinterpret_cast<uintptr_t>(p) % elem_size(dtype)) return fail(IRIS_ERR_ARG, "%s: %s is not aligned to its elements", fn, what);
  return IRIS_OK;
}
// Granules of a row, wherever it starts, in equal parts.
inline int part_granules(const void* p, int64_t stride, int64_t vocab, int dtype, int parts) {
  const int64_t es = (int64_t)elem_size(dtype), ve = 16 / es;
  const bool aligned = reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % ve == 0;
  const int64_t granules = (vocab + (aligned ? ve - 1 : 2 * ve - 2)) / ve;
  return (int)((granules + parts - 1) / parts);
}
inline int check_scale(const char* fn, const char* what, float s, float most = FLT_MAX) {
  if (!(s > 0.f) || std::isinf(s)) return fail(IRIS_ERR_ARG, "%s: %s has to be positive and finite", fn, what);
  if (s > most) return fail(IRIS_ERR_ARG, "%s: %s is at most %g", fn, what, most);
  return IRIS_OK;
}
inline int check_aligned(const char* fn, const char* what, const void* p, size_t a, bool needed) {
  if (needed && !p) return fail(IRIS_ERR_ARG, "%s: %s is NULL", fn, what);
  if (reinterpret_cast<uintptr_t>(p) % a) return fail(IRIS_ERR_ARG, "%s: %s is not %zu-byte aligned", fn, what, a);
  return IRIS_OK;
}
// `out` may be `in` itself (same address and stride) or share no element with it.
inline int check_overlap(const char* fn, const char* out_name, const char* in_name, const void* in, int64_t stride, const void* out, int64_t ostride,
                         int64_t rows, int64_t columns, int dtype) {
  if (rows == 0 || columns == 0) return IRIS_OK;
  const size_t es = elem_size(dtype);
  const uint64_t a = reinterpret_cast<uint64_t>(in), b = reinterpret_cast<uint64_t>(out);
  if (a == b && (stride == ostride || rows == 1)) return IRIS_OK;
  const uint64_t row = columns * es, ea = a + (uint64_t)(rows - 1) * stride * es + row, eb = b + (uint64_t)(rows - 1) * ostride * es + row;
  if (ea <= b || eb <= a) return IRIS_OK;
  if (stride == ostride && rows > 1) {   // two column ranges of one matrix
    const uint64_t s = stride * es, d = (a < b ? b - a : a - b) % s;
    if (d >= row && s - d >= row) return IRIS_OK;
  }
  return fail(IRIS_ERR_ARG, "%s: %s overlaps %s and is not the same matrix", fn, out_name, in_name);
}
inline int check_in_place(const char* fn, const void* logits, int64_t stride, const void* grad, int64_t gstride, int64_t rows, int64_t vocab, int dtype) {
  return check_overlap(fn, "dlogits", "logits", logits, stride, grad, gstride, rows, vocab, dtype);
}
// Launches clusters of `split` blocks.  A kernel may begin while the one before it in the stream ends (it waits for that
// one before it reads anything): a decoding step's calls are about as long as the gap between two launches.
template <class P>
inline int launch_rows(void (*kernel)(P), const P& p, unsigned blocks, int split, int threads, size_t bytes, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)split;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = split > 1 ? 2 : 1;
  if (cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p)) {
    cudaGetLastError();   // reported here, not by the next call
    return fail(IRIS_ERR_CUDA, "kernel launch: %s", cudaGetErrorString(e));
  }
  return IRIS_OK;
}
#define IRIS_CHECK(...)                      \
  do {                                       \
    if (int rc_ = (__VA_ARGS__)) return rc_; \
  } while (0)

}  // namespace rows
}  // namespace iris
