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

// The list in shared memory.  `id` < 0: no entry.  `add` of entries with one column is their sum, in all of them, so
// that the order in which they are written does not matter.
struct List {
  int id[kMaxList];
  float add[kMaxList];
};

__device__ __forceinline__ float grad_of(float z, float k, float m, float off, float alpha, float beta) {
  const float y = (z - m) * k - off;
  return ex2(y) * fmaf(beta, max_nan(y, kFloor), alpha);
}

// The sum of add over the entries that share entry i's column.
__device__ __forceinline__ float add_of_column(const List& l, int n, int i) {
  float s = 0.f;
  const int id = l.id[i];
  for (int j = 0; j < n; ++j) s += l.id[j] == id ? l.add[j] : 0.f;
  return s;
}

// Granules of the gradient: whole ones at once where its rows lie in memory as the logits' do, else element by element.
template <int DT>
__device__ __forceinline__ void store_granule(const Row<DT>& in, const Row<DT>& out, int v, const float (&x)[Row<DT>::VE]) {
  using E = Elem<DT>;
  constexpr int VE = E::VE;
  if (in.whole(v) && in.ph == out.ph) {
    st_global_v4(out.at(v), E::pack(x));
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int i = v * VE + e;
      if (i >= in.ph && i < in.end) out.column(i - in.ph) = E::from(x[e]);
    }
  }
}

template <int DT>
__device__ __forceinline__ void dense_granule(float (&x)[Row<DT>::VE], const Coef& c) {
#pragma unroll
  for (int e = 0; e < Row<DT>::VE; ++e) x[e] = c.zero ? 0.f : grad_of(x[e], c.k, c.m, c.off, c.alpha, c.beta);
}

// Granules [v0, v1) of a row, by all threads of the block; listed columns outside them are another block's.
template <int DT>
__device__ void grad_range(const Row<DT>& in, const Row<DT>& out, int v0, int v1, const Coef& c, const List& list, int n) {
  constexpr int VE = Row<DT>::VE;
  const int i = threadIdx.x;
  float zl = 0.f, add = 0.f;
  bool mine = false;
  if (i < n && !c.zero) {
    const int g = in.ph + list.id[i];
    mine = list.id[i] >= 0 && g >= v0 * VE && g < v1 * VE;
    if (mine) {
      zl = Elem<DT>::to(in.column(list.id[i]));
      add = add_of_column(list, n, i);
    }
  }
  __syncthreads();   // the gradient may replace the logits: listed ones have been read
  for (int v = v0 + (int)threadIdx.x; v < v1; v += (int)blockDim.x) {
    float x[VE];
    in.load(v, x);
    dense_granule<DT>(x, c);
    store_granule<DT>(in, out, v, x);
  }
  __syncthreads();   // the dense part of the listed columns is written before what replaces it
  if (mine) out.column(list.id[i]) = Elem<DT>::from(grad_of(zl, c.k, c.m, c.off_l, c.alpha_l, c.beta) + add);
}

}  // namespace rows
}  // namespace iris
