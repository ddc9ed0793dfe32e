// The gradient of a loss on a row's softmax, from saved statistics: a dense part that is the same function of every
// logit, and a list of at most kMaxList columns where it differs (the targets, the teacher's tokens).
#pragma once

#include "logit_rows.cuh"

namespace iris {
namespace rows {

// dz_j = 2^(y_j - off) (alpha + beta max(y_j - off, kFloor)) for columns off the list,
//        2^(y_j - off_l) (alpha_l + beta max(y_j - off_l, kFloor)) + add for those on it,   y_j = (z_j - m) k.
// zero: the whole row is 0, whatever its logits are.
struct Coef {
  float k, m, off, alpha, off_l, alpha_l, beta;
  bool zero;
};

// The list in shared memory.  `id` < 0: no entry, also behind the last one.  `add` is what the listed column's gradient
// gets besides; entries with one column all write the sum of theirs, so that their order does not matter.
struct List {
  alignas(16) int id[kMaxList];
  float add[kMaxList];
};

__device__ __forceinline__ float grad_of(float z, const Coef& c) {   // on the list
  const float y = (z - c.m) * c.k - c.off_l;
  return ex2(y) * fmaf(c.beta, max_nan(y, kFloor), c.alpha_l);
}

// Whether another entry of the first n has entry i's column; `before`: an earlier one.
__device__ __forceinline__ bool repeated(const List& l, int n, int i, bool before) {
  const int id = l.id[i];
  int same = 0;
  for (int j = 0; j < n; j += 4) {
    const int4 o = *reinterpret_cast<const int4*>(&l.id[j]);
    same += (o.x == id && (!before || j < i)) + (o.y == id && (!before || j + 1 < i)) + (o.z == id && (!before || j + 2 < i)) +
            (o.w == id && (!before || j + 3 < i));
  }
  return same > (before ? 0 : 1);
}
__device__ __forceinline__ float add_of_column(const List& l, int n, int i) {
  if (!repeated(l, n, i, false)) return l.add[i];
  float s = 0.f;
  const int id = l.id[i];
  for (int j = 0; j < n; ++j) s += l.id[j] == id ? l.add[j] : 0.f;
  return s;
}

// The dense part, two elements at a time: per element one instruction to unpack, the exponential, and half of one each to
// subtract, scale, multiply and pack.
template <int DT, bool BETA>
struct Dense {
  uint64_t k2, minus_m2, minus_off2, alpha2, beta2;
  uint32_t floor = 0;
  bool lift = false;
  Coef c;
  __device__ __forceinline__ explicit Dense(const Coef& c_) : c(c_) {
    k2 = pair(c.k, c.k);
    minus_m2 = pair(-c.m, -c.m);
    minus_off2 = pair(-c.off, -c.off);
    alpha2 = pair(c.alpha, c.alpha);
    beta2 = pair(c.beta, c.beta);
    if (BETA) lift = lift_floor<DT>(c.m, c.k, floor);   // off >= 0 lowers the exponents further
  }
  __device__ __forceinline__ void operator()(const uint4& g, float (&x)[Elem<DT>::VE]) const {
    constexpr int VE = Elem<DT>::VE;
    if (c.zero) {
#pragma unroll
      for (int e = 0; e < VE; ++e) x[e] = 0.f;
    } else if (!BETA || lift) {
      Elem<DT>::unpack(BETA ? Elem<DT>::at_least(g, floor) : g, x);
#pragma unroll
      for (int e = 0; e < VE; e += 2) {
        const uint64_t y2 = fma2f(add2f(pair(x[e], x[e + 1]), minus_m2), k2, minus_off2);
        const float2 y = unpair(y2);
        const float2 d = unpair(mul2f(pair(ex2(y.x), ex2(y.y)), BETA ? fma2f(beta2, y2, alpha2) : alpha2));
        x[e] = d.x;
        x[e + 1] = d.y;
      }
    } else {
      Elem<DT>::unpack(g, x);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float y = (x[e] - c.m) * c.k - c.off;
        x[e] = ex2(y) * fmaf(c.beta, max_nan(y, kFloor), c.alpha);
      }
    }
  }
};

// Granule i of a part of the gradient: at once where it lies inside the row and the two matrices' rows lie alike in
// memory, else element by element.
template <int DT>
__device__ __forceinline__ void store_granule(const Row<DT>& in, const Row<DT>& out, const Part<DT>& part, bool alike, int i,
                                              const float (&x)[Elem<DT>::VE]) {
  using E = Elem<DT>;
  if (alike && i < part.n_int) {
    st_global_v4(out.at(part.w0 + i), E::pack(x));
  } else {
    const int at = part.granule(i) * E::VE;
#pragma unroll
    for (int e = 0; e < E::VE; ++e)
      if (at + e >= in.ph && at + e < in.end) out.column(at + e - in.ph) = E::from(x[e]);
  }
}

constexpr int kGradThreads = 256;
constexpr int kGradGranules = 4;   // that a thread has in flight

// A part of a row, by all kGradThreads threads of the block; listed columns outside it are another block's.
template <int DT, bool BETA>
__device__ __forceinline__ void grad_part(const Row<DT>& in, const Row<DT>& out, const Part<DT>& part, const Coef& c, const List& list, int n) {
  constexpr int VE = Elem<DT>::VE, U = kGradGranules, T = kGradThreads;
  const int tid = threadIdx.x;
  float zl = 0.f, add = 0.f;
  bool mine = false;
  if (tid < n && !c.zero) {
    mine = list.id[tid] >= 0 && part.has(in.ph + list.id[tid]);
    if (mine) {
      zl = Elem<DT>::to(in.column(list.id[tid]));
      add = add_of_column(list, n, tid);
    }
  }
  const Dense<DT, BETA> dense(c);
  const bool alike = in.ph == out.ph;
  __syncthreads();   // the gradient may replace the logits: listed ones have been read
  for (int i = tid; i < part.n_all; i += T * U) {
    uint4 g[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * T < part.n_all) g[u] = part.raw(in, i + u * T);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * T < part.n_all) {
        float x[VE];
        dense(g[u], x);
        store_granule<DT>(in, out, part, alike, i + u * T, x);
      }
  }
  __syncthreads();   // the dense part of the listed columns is written before what replaces it
  if (mine) out.column(list.id[tid]) = Elem<DT>::from(grad_of(zl, c) + add);
}

// Blocks a row is cut into for a streamed gradient: about 8 granules a thread.
inline int grad_parts(int64_t vocab, int dtype) {
  const int64_t granules = vocab * (int64_t)elem_size(dtype) / 16, each = kGradThreads * 8;
  return (int)(granules / each > 0 ? granules / each : 1);
}

}  // namespace rows
}  // namespace iris
