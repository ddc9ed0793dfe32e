// The gradient of a loss on a row's softmax, from saved statistics: a dense part that is the same function of every
// logit, and a list of at most kMaxList columns where it differs (the targets, the teacher's tokens).
#pragma once

#include "logit_rows.cuh"

namespace iris {
namespace rows {

// dz_j = 2^(y_j - off) (alpha + beta max(y_j - off, kFloor)) for columns off the list, y_j = (z_j - m) k,
//        2^(y_j - off_l) (alpha_l + beta max(y_j - off_l, kFloor)) + add for those on it, y_j = (z_j - m_l) k.
// zero: the whole row is 0, whatever its logits are.
struct Coef {
  float k, m, off, alpha, m_l, off_l, alpha_l, beta;
  bool zero;
};

// The list in shared memory.  `id` < 0: no entry, also behind the last one.  `add` is what the listed column's gradient
// gets besides; entries with one column all write the sum of theirs, so that their order does not matter.
struct List {
  alignas(16) int id[kMaxList];
  float add[kMaxList];
};

// ex2 gives 0 below 2^-126, and alpha + beta y may be large: exponents are raised by 8 and the factor lowered by 2^-8, a
// power of two, so that a y of 0 still gives alpha.  (By 32, the rounding of exponents near 32 was 1e-6 of the result.)
constexpr float kRaise = 8.f, kLower = 1.f / 256.f;

// 2^y (alpha + beta y): beta y would overflow for a large beta where 2^y is 0.
__device__ __forceinline__ float raised(float y, float alpha, float beta) {
  const float e = ex2(y + kRaise);
  return fmaf(e * max_nan(y, kFloor), beta, e * alpha) * kLower;
}
__device__ __forceinline__ float grad_of(float z, const Coef& c) {   // on the list
  const float y = (z - c.m_l) * c.k - c.off_l;
  return raised(y, c.alpha_l, c.beta);
}

// Whether another entry of the first n has entry i's column.
__device__ __forceinline__ bool repeated(const List& l, int n, int i) {
  const int id = l.id[i];
  int same = 0;
  for (int j = 0; j < n; j += 4) {
    const int4 o = *reinterpret_cast<const int4*>(&l.id[j]);
    same += (o.x == id) + (o.y == id) + (o.z == id) + (o.w == id);
  }
  return same > 1;
}
// Whether an entry before entry i has its column.
__device__ __forceinline__ bool comes_again(const List& l, int i) {
  const int id = l.id[i];
  int same = 0;
  for (int j = 0; j < i; j += 4) {
    const int4 o = *reinterpret_cast<const int4*>(&l.id[j]);
    same += (o.x == id) + (o.y == id && j + 1 < i) + (o.z == id && j + 2 < i) + (o.w == id && j + 3 < i);
  }
  return same > 0;
}
__device__ __forceinline__ float sum_of_column(const List& l, int n, int i) {
  float s = 0.f;
  const int id = l.id[i];
  for (int j = 0; j < n; ++j) s += l.id[j] == id ? l.add[j] : 0.f;
  return s;
}

// The dense part, two elements at a time: per element one instruction to unpack, the exponential, and half of one each to
// subtract, scale, multiply and pack.
template <int DT, bool BETA>
struct Dense {
  static constexpr int VE = Elem<DT>::VE;
  uint64_t k2, minus_m2, minus_off2, alpha2, beta2;
  uint32_t floor = 0;
  bool lift = true;
  Coef c;
  __device__ __forceinline__ explicit Dense(const Coef& c_) : c(c_) {
    k2 = pair(c.k, c.k);
    minus_m2 = pair(-c.m, -c.m);
    const float off = c.off - kRaise, alpha = (c.alpha - kRaise * c.beta) * kLower, beta = c.beta * kLower;
    minus_off2 = pair(-off, -off);
    alpha2 = pair(alpha, alpha);
    beta2 = pair(beta, beta);
    if (BETA) lift = lift_floor<DT>(c.m, c.k, floor);   // off >= 0 lowers the exponents further
  }
  __device__ __forceinline__ bool plain() const { return c.zero || lift; }
  __device__ __forceinline__ void operator()(const uint4& g, float (&x)[VE]) const {   // where lift and not zero
    Elem<DT>::unpack(BETA ? Elem<DT>::at_least(g, floor) : g, x);
#pragma unroll
    for (int e = 0; e < VE; e += 2) {
      const uint64_t y2 = fma2f(add2f(pair(x[e], x[e + 1]), minus_m2), k2, minus_off2);
      const float2 y = unpair(y2);
      const float2 d = unpair(mul2f(pair(ex2(y.x), ex2(y.y)), BETA ? fma2f(beta2, y2, alpha2) : alpha2));
      x[e] = d.x;
      x[e + 1] = d.y;
    }
  }
  __device__ __forceinline__ void one_by_one(const uint4& g, float (&x)[VE]) const {
    Elem<DT>::unpack(g, x);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float y = (x[e] - c.m) * c.k - c.off;
      x[e] = c.zero ? 0.f : raised(y, c.alpha, c.beta);
    }
  }
};

constexpr int kGradThreads = 256;
constexpr int kGradGranules = 4;   // that a thread has in flight

// The dense gradient of a granule element by element, for what the row covers in part and where the rows of the gradient
// do not lie in memory as those of the logits.
template <int DT, bool BETA>
__device__ __forceinline__ void write_elements(const Row<DT>& in, const Row<DT>& out, const Dense<DT, BETA>& dense, int granule, const uint4& g) {
  using E = Elem<DT>;
  float x[E::VE];
  dense.one_by_one(g, x);
  const int at = granule * E::VE;
#pragma unroll
  for (int e = 0; e < E::VE; ++e)
    if (at + e >= in.ph && at + e < in.end) out.column(at + e - in.ph) = E::from(x[e]);
}
template <int DT, bool BETA>
__device__ __forceinline__ uint4 dense_of(const Dense<DT, BETA>& dense, const uint4& g) {
  if (dense.c.zero) return make_uint4(0, 0, 0, 0);
  float x[Elem<DT>::VE];
  dense(g, x);
  return Elem<DT>::pack(x);
}

// Streamed gradients are bound by memory: 8192 x 16384 bf16 with the entropy's part in 87 us, 6.2 TB/s read and written, 94 %
// of the copy rate; four granules of a thread under way in five to six blocks an SM, 2048 granules a block or more.
//
// A part of a row; listed columns outside it are another block's.  The list has been written before the last barrier
// (id) or the next one (add).
template <int DT, bool BETA>
__device__ __forceinline__ void grad_part(const Row<DT>& in, const Row<DT>& out, const Part<DT>& part, const Coef& c, const List& list, int n) {
  const int tid = threadIdx.x;
  float zl = 0.f;
  bool rep = false;
  const bool mine = tid < n && !c.zero && list.id[tid] >= 0 && part.has(in.ph + list.id[tid]);
  if (mine) {
    zl = Elem<DT>::to(in.column(list.id[tid]));
    rep = repeated(list, n, tid);
  }
  __syncthreads();   // the gradient may replace the logits: listed ones have been read
  const Dense<DT, BETA> dense(c);
  constexpr int T = kGradThreads, U = kGradGranules;
  if (in.ph == out.ph && dense.plain()) {
    const uint4* const from = reinterpret_cast<const uint4*>(in.at(part.w0)) + tid;
    uint4* const to = reinterpret_cast<uint4*>(out.at(part.w0)) + tid;
    batches<T, U>(part.n_int, [&](int b, auto all) {
      constexpr bool ALL = decltype(all)::value;
      const int left = part.n_int - b - tid;
      uint4 g[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if ((ALL || u * T < left) && !c.zero) g[u] = ld_once(from + b + u * T);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (ALL || u * T < left) st_global_v4(to + b + u * T, dense_of(dense, g[u]));
    });
    if (tid < part.n_all - part.n_int) write_elements(in, out, dense, part.granule(part.n_int + tid), part.raw(in, part.n_int + tid));
  } else {
#pragma unroll 1
    for (int i = tid; i < part.n_all; i += T) write_elements(in, out, dense, part.granule(i), part.raw(in, i));
  }
  __syncthreads();   // the dense part of the listed columns is written before what replaces it
  if (mine) out.column(list.id[tid]) = Elem<DT>::from(grad_of(zl, c) + (rep ? sum_of_column(list, n, tid) : list.add[tid]));
}

// Blocks a row is cut into for a streamed gradient: 8 granules a thread or more (2048 x 36864 fp16: 53.3 us; 4: 58.8,
// 16: 55.2).
inline int grad_parts(int64_t vocab, int dtype) {
  const int64_t granules = vocab * (int64_t)elem_size(dtype) / 16, each = kGradThreads * 8;
  return (int)(granules / each > 0 ? granules / each : 1);
}

}  // namespace rows
}  // namespace iris
