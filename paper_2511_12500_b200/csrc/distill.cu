// Distillation from a teacher's top logits: per row the Kullback-Leibler divergence of the student's distribution over
// the whole vocabulary from the teacher's on its listed tokens, and the gradient for the student's logits.
//
//   renormalised list: p = softmax(teacher_scale v),              L = sum_k p_k (ln p_k - ln q_k)
//   with remainder:    p_k = exp v_k, p_r = max(0, 1 - sum p_k),  L = the same + p_r (ln p_r - ln q_r), q_r = sum of q off the list
//   dL/dz_j = scale (P q_j - p_j) in the first form; in the second scale ((P + p_r) q_j - p_j) on the list and
//   scale ((P + p_r) q_j - p_r q_j / q_r) off it;  P = sum p_k.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "logit_grad.cuh"
#include "sm100_ptx.cuh"

namespace iris {
namespace rows {

constexpr int kDistillThreads = 128;
constexpr int kDistillBlocks = 4;   // an SM's registers are shared out for
constexpr int kLossBlocks = 8;
enum { kLossOnly, kHeld, kReadTwice };
constexpr int kMaxSplit = 8;   // blocks (one cluster) that share a row
static_assert(kDistillThreads >= kMaxList && kGradThreads >= kMaxList, "one thread an entry of the list");

struct DistillParams {
  const void* logits;
  int64_t stride, grad_stride;
  int rows, vocab, list_k, split, each, hold;   // each: granules of a block's part of a row; hold: of those in shared memory
  float scale, teacher_scale;
  const float* teacher;
  const int64_t* ids;
  const float* weight;       // forward with gradient: loss weights; backward: grad_loss; nullptr = 1
  float *loss, *stats;
  void* dlogits;
};

// The teacher's list: thread i has entry i, its column (-1: absent) and its value, and with the others of the first four
// warps its probability p, the sum P and the remainder p_r.
struct Entry {
  int id;
  float v;
};
struct RawEntry {   // as loaded: nothing waits for it yet
  int64_t id = -1;
  float v = 0.f;
  __device__ __forceinline__ Entry checked(const DistillParams& p) const {
    const bool there = id >= 0 && id < p.vocab;
    return Entry{there ? (int)id : -1, there ? v : -INFINITY};
  }
};
struct TeacherSums {
  float m[kMaxList / 32], s[kMaxList / 32];
};

__device__ __forceinline__ RawEntry load_entry(const DistillParams& p, int64_t r) {
  RawEntry e;
  if ((int)threadIdx.x < p.list_k) {
    const int64_t at = r * p.list_k + threadIdx.x;
    e.id = p.ids[at];
    e.v = p.teacher[at];
  }
  return e;
}

// Before a barrier: what a warp of the list gives to the sum.  Returns exp(scale (v - the warp's m)): differences are scaled, as a mask's finite value
// times the scale may overflow.
template <bool TAIL>
__device__ __forceinline__ float share_entry(const Entry& e, float scale, TeacherSums& t) {
  if (threadIdx.x >= kMaxList) return 0.f;
  const float m = TAIL ? 0.f : fmaxf(warp_max(e.v == e.v ? e.v : -FLT_MAX), -FLT_MAX);   // log probabilities are taken as they are
  const float x = expf(TAIL ? e.v : (e.v - m) * scale);
  float s = x;
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
  if ((threadIdx.x & 31) == 0) {
    t.m[threadIdx.x >> 5] = m;
    t.s[threadIdx.x >> 5] = s;
  }
  return x;
}
// Behind it: the entry's p, P and p_r, the latter two in all threads.
template <bool TAIL>
__device__ __forceinline__ float3 join_entries(float x, float scale, const TeacherSums& t) {
  constexpr int N = kMaxList / 32;
  if (TAIL) {
    const float s = t.s[0] + t.s[1] + t.s[2] + t.s[3];
    return make_float3(x, s, max_nan(0.f, 1.f - s));
  }
  float m = t.m[0], s = 0.f;
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, t.m[i]);
#pragma unroll
  for (int i = 0; i < N; ++i) s += t.s[i] * ex2((t.m[i] - m) * scale * kLog2e);
  if (s == 0.f) return make_float3(0.f, 0.f, 0.f);   // a list with no token left asks for nothing
  const float own = threadIdx.x < kMaxList ? t.m[threadIdx.x >> 5] : m;
  return make_float3(x * ex2((own - m) * scale * kLog2e) / s, s == s ? 1.f : NAN, 0.f);
}

// ln of the sum of the tokens off the list (`dense`), counted from m; what is less than the type holds is its lowest value, as -inf says
// that there is no such token.
__device__ __forceinline__ float log_rest(const Acc& dense, float ls_off, float m, float scale) {
  return dense.s == 0.f ? -INFINITY : max_nan((dense.m - m) * scale + ls_off, -FLT_MAX);
}

// The remainder that counts: against tokens off the list that have no probability in 32 bits (the largest is masked, by -inf or by a finite value),
// what rounding may have left of 1 - sum p is no remainder.  The rows of -inf (ls) keep theirs.
__device__ __forceinline__ float kept_rest(float rest, float ls, float lr) {
  return rest < 1e-5f && ex2((lr - ls) * kLog2e) == 0.f ? 0.f : rest;
}

// m_off, ls_off: with a remainder, a logit and ln of the sum of the tokens off the list counted from it.  Their largest one, or (m, lr): but where
// they are all masked by a finite value, (z - m) k and lr are so far below 0 that their difference, the logarithm of a share, is lost.
template <bool TAIL>
__device__ __forceinline__ Coef distill_coef(float scale, float sum, float rest, float m, float ls, float lr, float m_off, float ls_off, float w) {
  Coef c;
  c.k = scale * kLog2e;
  c.m = c.m_l = m;
  c.beta = 0.f;
  c.off_l = ls * kLog2e;
  c.alpha_l = w * scale * (sum + rest);
  if (TAIL && !(rest == 0.f)) {
    const bool some = ls_off != -INFINITY;
    if (some) c.m = m_off;
    c.off = some ? ls_off * kLog2e : 0.f;
    c.alpha = some ? w * scale * ((sum + rest) * ex2((lr - ls) * kLog2e) - rest) : 0.f;
  } else {
    c.off = c.off_l;
    c.alpha = c.alpha_l;
  }
  c.zero = ls == -INFINITY || w == 0.f;
  return c;
}

// What the blocks of the cluster found in their parts: of the tokens off the list (all, without remainder) and of those on it.
struct Found {
  Warps<kMaxSplit> dense, listed;
};

// The one or two granules of a part that the row covers in part, held by threads 0 and 1 of the block.
template <int DT>
struct Edge {
  using T = typename Elem<DT>::T;
  T v[Elem<DT>::VE];
  __device__ __forceinline__ void load(const Row<DT>& row, const Part<DT>& part) {   // bits as they are: nothing waits for them yet
    if ((int)threadIdx.x >= part.n_all - part.n_int) return;
    const int at = part.granule(part.n_int + threadIdx.x) * Elem<DT>::VE;
#pragma unroll
    for (int e = 0; e < Elem<DT>::VE; ++e) v[e] = at + e >= row.ph && at + e < row.end ? row.granule0[at + e] : Elem<DT>::from(-INFINITY);
  }
  __device__ __forceinline__ uint4 raw() const {
    float x[Elem<DT>::VE];
#pragma unroll
    for (int e = 0; e < Elem<DT>::VE; ++e) x[e] = Elem<DT>::to(v[e]);
    return Elem<DT>::pack(x);
  }
};

// A cluster of `split` blocks takes rows one after the other; each block has a part of the row.
//   kHeld       The part lies in shared memory, where a thread uses only the granules that it copied itself, and the
//               gradient is computed from there, so a row is read once.  As soon as a granule has been used for the last
//               time its place takes the next row's, which is under way while this one is finished.
//   kLossOnly   Nothing has to be held; a cluster for every row.
//   kReadTwice  The gradient of a part too large for shared memory.
// A byte a granule (on_list) says which of its tokens are on the list: with a remainder they leave the sum.
//
// What bounds it: 8192 x 28672 bf16 with 64 teacher's tokens takes 193 us, 4.9 TB/s read and written, 74 % of the copy rate;
// 2 exponentials an element keep the special function unit 60 % busy and 12.7 instructions an element the issue slots 50 %.
// Without its loads and stores the kernel takes 170 us, without its arithmetic 175: three rows in an SM do not overlap them
// better.  Blocks of 128 threads: what a row costs besides its elements is 670 instructions a warp, so few warps (256
// threads: 195 us), with four blocks' worth of registers; rows of one block up to 60 KB (two blocks of 28 KB: 236 us), as
// many clusters as fit at once (one wave more, as an SM count would give for clusters of four, is twice the time).
// 4096 x 128000 with remainder, clusters of five: 455 us, 70 %; about 2 us of a row's 12 wait for the exchange.
// The loss alone streams: 1024 x 50021 fp32 with remainder 37 us, 85 %; 4096 x 36864 bf16 54 us renormalised, 60 with remainder (86 and 77 %).  Of its
// eight blocks an SM only fp32 renormalised spills registers (84 bytes; 36 us, 86 %).
template <int DT, bool TAIL, int MODE>
__global__ void __launch_bounds__(kDistillThreads, MODE == kLossOnly ? kLossBlocks : kDistillBlocks) distill_kernel(const DistillParams p) {
  using E = Elem<DT>;
  constexpr int VE = E::VE, T = kDistillThreads, U = 4;   // granules of a batch
  constexpr bool HELD = MODE == kHeld, grad = MODE != kLossOnly;
  extern __shared__ uint4 held[];
  __shared__ List lists[2];          // of this row and the one before
  __shared__ TeacherSums teacher;
  __shared__ Warps<T / 32> buf[2];
  __shared__ Found found[2];         // as the lists
  __shared__ float red[kMaxList / 32];
  __shared__ float4 upper[HELD ? 1 : T];
  __shared__ int repeats[2];         // whether a column comes twice on the list
  uint32_t* const on_list = reinterpret_cast<uint32_t*>(held + (HELD ? p.hold : 0));
  const uint8_t* const marks = reinterpret_cast<const uint8_t*>(on_list);
  uint4* const mine = held + threadIdx.x;
  const uint32_t held_at = ptx::smem_u32(held), mine_at = held_at + threadIdx.x * 16;
  const int split = p.split, rank = split > 1 ? (int)ptx::cluster_ctarank() : 0, tid = threadIdx.x, n = p.list_k;
  const int64_t step = gridDim.x / split;
  int64_t r = blockIdx.x / split;
  if (split > 1) {
    if (tid < kMaxSplit) found[0].dense.of[tid] = found[0].listed.of[tid] = found[1].dense.of[tid] = found[1].listed.of[tid] = Acc{};
    ptx::cluster_arrive_release();
  }
  ptx::begin_after_previous();
  const float k = p.scale * kLog2e;

  RawEntry ahead = load_entry(p, r);
  float w = p.weight ? p.weight[r] : 1.f;
  Row<DT> in(p.logits, r, p.stride, p.vocab);
  Part<DT> part(in, rank, p.each);
  Edge<DT> edge;
  if (HELD) {
    const uint4* const from = reinterpret_cast<const uint4*>(in.at(part.w0));
#pragma unroll 4
    for (int i = tid; i < part.n_int; i += T) copy_async(held_at + i * 16, from + i);
    edge.load(in, part);
  }
  for (int i = tid; i * 4 < p.hold; i += T) on_list[i] = 0;
  if (tid == 0) repeats[0] = 0;
  if (split > 1) ptx::cluster_wait();   // all blocks have started and have cleared their places for the others' sums
  __syncthreads();
  for (int turn = 0; r < p.rows; r += step, turn ^= 1) {
    List& list = lists[turn];
    const Entry entry = ahead.checked(p);
    Sums<DT, false, !HELD> sums(k, upper + (HELD ? 0 : tid));
    const bool own = entry.id >= 0 && part.has(in.ph + entry.id);
    typename E::T z_listed = E::from(-INFINITY);   // the listed token's logit: of all tokens in the first block, of the part's own in the others
    if (own || (rank == 0 && entry.id >= 0)) z_listed = in.column(entry.id);
    if (tid < kMaxList) list.id[tid] = entry.id;
    const float x = share_entry<TAIL>(entry, p.teacher_scale, teacher);
    const int mark = own ? part.place((in.ph + entry.id) / VE) : -1;   // the listed token's granule and its bit in there
    const uint32_t bit = own ? 1u << (mark % 4 * 8 + (in.ph + entry.id) % VE) : 0;
    bool first = false;                                                // of entries with the same column: the one whose logit is summed
    if (tid == 0) repeats[turn ^ 1] = 0;
    const int64_t r_next = r + step;
    const bool more = MODE != kLossOnly && r_next < p.rows;
    const Row<DT> next(p.logits, more ? r_next : r, p.stride, p.vocab);
    const Part<DT> next_part(next, rank, p.each);
    const uint4* const from = reinterpret_cast<const uint4*>(next.at(next_part.w0));
    const int n_next = HELD && more ? next_part.n_int : 0;

    if (HELD) {
      if (own) {
        first = !(atomicOr(&on_list[mark / 4], bit) & bit);
        if (!first) repeats[turn] = 1;
      }
      if (TAIL) __syncthreads();
      copy_async_wait();
      batches<T, U>(part.n_int, [&](int b, auto all) {
        constexpr bool ALL = decltype(all)::value;
        const int left = part.n_int - b - tid;
        uint4 g[U];
        uint32_t bits[U], any = 0;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (ALL || u * T < left) {
            g[u] = mine[b + u * T];
            if (TAIL) any |= bits[u] = marks[b + u * T + tid];
          }
        if (TAIL && any) {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if ((ALL || u * T < left) && bits[u]) g[u] = without<DT>(g[u], bits[u]);
        }
        sums.template pace<T, U>(b);
        sums.template add<ALL>(g, largest<DT, ALL>(g, left, T), left, T);
      });
      if (tid < part.n_all - part.n_int) {
        const uint4 g[1] = {without<DT>(edge.raw(), TAIL ? marks[part.n_int + tid] : 0)};
        sums.template add<true>(g, largest<DT>(g[0]));
      }
    } else {
      for (int b0 = 0; b0 < part.n_all; b0 += p.hold) {   // p.hold granules at a time have marks
        const bool in_piece = TAIL && own && mark >= b0 && mark < b0 + p.hold;
        if (TAIL) {
          if (in_piece) {
            first = !(atomicOr(&on_list[(mark - b0) / 4], bit) & bit);
            if (!first) repeats[turn] = 1;
          }
          __syncthreads();
        }
        const int size = min(part.n_all - b0, p.hold), inside = min(part.n_int - b0, size);
        const uint4* const at = reinterpret_cast<const uint4*>(in.at(part.w0)) + b0 + tid;
        const auto batch = [&](int b, auto all) {
          constexpr bool ALL = decltype(all)::value;
          const int left = size - b - tid;
          uint4 g[U];
          uint32_t bits[U], any = 0;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (ALL) g[u] = ld_once(at + b + u * T);
            else if (u * T < left) g[u] = part.raw(in, b0 + b + u * T + tid);
          }
          if (TAIL) {
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (ALL || u * T < left) any |= bits[u] = marks[b + u * T + tid];
            if (any) {
#pragma unroll
              for (int u = 0; u < U; ++u)
                if ((ALL || u * T < left) && bits[u]) g[u] = without<DT>(g[u], bits[u]);
            }
          }
          sums.template pace<T, U>(b);
          sums.template add<ALL>(g, largest<DT, ALL>(g, left, T), left, T);
        };
        int b = 0;
        for (; b + T * U <= inside; b += T * U) batch(b, std::true_type{});
        for (; b < size; b += T * U) batch(b, std::false_type{});
        if (TAIL) {
          __syncthreads();
          if (in_piece) on_list[(mark - b0) / 4] = 0;
          __syncthreads();
        }
      }
    }
    warp_share<false>(sums.done(), k, buf[0]);
    if (TAIL) {
      Acc listed;
      if (repeats[turn] && own) first = !comes_again(list, tid);   // not the one that came first: sums must not depend on that
      if (first) listed.add_one(E::to(z_listed), k);
      warp_share<false>(listed, k, buf[1]);
    }
    __syncthreads();
    if (HELD && own) on_list[mark / 4] = 0;
    Acc dense = warps_join<false>(k, buf[0]), listed;
    if (TAIL) listed = warps_join<false>(k, buf[1]);
    if (split > 1) {
      if (tid < split) {
        const uint32_t to = ptx::mapa(ptx::smem_u32(&found[turn].dense.of[rank]), tid), to_listed = ptx::mapa(ptx::smem_u32(&found[turn].listed.of[rank]), tid);
        ptx::st_shared_cluster_u32(to, __float_as_uint(dense.m));
        ptx::st_shared_cluster_u32(to + 4, __float_as_uint(dense.s));
        if (TAIL) {
          ptx::st_shared_cluster_u32(to_listed, __float_as_uint(listed.m));
          ptx::st_shared_cluster_u32(to_listed + 4, __float_as_uint(listed.s));
        }
      }
      ptx::cluster_arrive_release();
    }
    const float w_row = w;
    if (more) {
      ahead = load_entry(p, r_next);
      if (p.weight) w = p.weight[r_next];
    }
    const float3 teach = join_entries<TAIL>(x, p.teacher_scale, teacher);
    const float pk = entry.id >= 0 ? teach.x : 0.f;
    if (split > 1) {
      ptx::cluster_wait();   // behind it no block reads logits of another's part, and the gradient may replace them
      dense = warps_join<false>(k, found[turn].dense);
      if (TAIL) listed = warps_join<false>(k, found[turn].listed);
    }
    Acc all = dense;
    if (TAIL) all.merge(listed, k);
    const float ls = log_sum(all);
    const float ls_off = TAIL ? log_sum(dense) : 0.f, lr = TAIL ? log_rest(dense, ls_off, all.m, p.scale) : 0.f;
    const float rest = TAIL ? kept_rest(teach.z, ls, lr) : 0.f;
    const float zk = E::to(z_listed);
    Coef coef;
    const Row<DT> out(p.dlogits, grad ? r : 0, p.grad_stride, p.vocab);
    bool rep = false;
    float listed_grad = 0.f, add = 0.f;
    if constexpr (grad) {
      coef = distill_coef<TAIL>(p.scale, teach.y, rest, all.m, ls, lr, dense.m, ls_off, w_row);
      add = -w_row * p.scale * pk;
      listed_grad = grad_of(zk, coef);
      if (tid < n) list.add[tid] = add;
      rep = own && (HELD ? repeats[turn] != 0 : repeated(list, n, tid));
      const Dense<DT, false> dense_part(coef);
      if (HELD) {
        if (tid < part.n_all - part.n_int) write_elements(in, out, dense_part, part.granule(part.n_int + tid), edge.raw());
        if (more) edge.load(next, next_part);
        const bool alike = in.ph == out.ph && dense_part.plain();
        const int both = alike ? more ? min(part.n_int, n_next) : part.n_int : 0;
        uint4* const to = reinterpret_cast<uint4*>(out.at(part.w0)) + tid;
        int b = 0;
        for (; b + T * U <= both; b += T * U) {
          uint4 g[U];
#pragma unroll
          for (int u = 0; u < U; ++u) g[u] = mine[b + u * T];
#pragma unroll
          for (int u = 0; u < U; ++u) st_global_v4(to + b + u * T, dense_of(dense_part, g[u]));
          if (more) {
#pragma unroll
            for (int u = 0; u < U; ++u) copy_async(mine_at + (b + u * T) * 16, from + b + u * T + tid);
          }
        }
        for (int i = b + tid; i < max(part.n_int, n_next); i += T) {
          if (i < part.n_int) {
            if (alike) st_global_v4(to + i - tid, dense_of(dense_part, held[i]));
            else write_elements(in, out, dense_part, part.w0 + i, held[i]);
          }
          if (i < n_next) copy_async(held_at + i * 16, from + i);
        }
      } else {
        if (split == 1) __syncthreads();   // the listed logits have been read
        if (in.ph == out.ph && dense_part.plain()) {
          const uint4* const at = reinterpret_cast<const uint4*>(in.at(part.w0)) + tid;
          uint4* const to = reinterpret_cast<uint4*>(out.at(part.w0)) + tid;
          batches<T, U>(part.n_int, [&](int b, auto all) {
            constexpr bool ALL = decltype(all)::value;
            const int left = part.n_int - b - tid;
            uint4 g[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
              if ((ALL || u * T < left) && !coef.zero) g[u] = ld_once(at + b + u * T);
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (ALL || u * T < left) st_global_v4(to + b + u * T, dense_of(dense_part, g[u]));
          });
          if (tid < part.n_all - part.n_int) write_elements(in, out, dense_part, part.granule(part.n_int + tid), part.raw(in, part.n_int + tid));
        } else {
          for (int i = tid; i < part.n_all; i += T) write_elements(in, out, dense_part, part.granule(i), part.raw(in, i));
        }
      }
    }
    if (rank == 0 && tid < kMaxList) {
      float l = 0.f;   // log probabilities in parts: their products with p are in range where a mask's own is not
      if (ls != ls) l = NAN;   // also where nothing is asked of the row
      else if (!(pk == 0.f)) l = ls == -INFINITY && pk > 0.f ? INFINITY : pk * (logf(pk) + ls) + pk * (all.m - zk) * p.scale;
      if (TAIL && tid == 0 && !(rest == 0.f)) {
        if (ls == -INFINITY && rest > 0.f) l = INFINITY;
        else l += rest * (logf(rest) - ls_off + ls) + rest * (all.m - dense.m) * p.scale;
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(~0u, l, o);
      if ((tid & 31) == 0) red[tid >> 5] = l;
    }
    __syncthreads();   // the dense part of the listed columns is written before what replaces it
    if (grad && own && !coef.zero) out.column(entry.id) = E::from(listed_grad + (rep ? sum_of_column(list, n, tid) : add));
    if (rank == 0 && tid == 0) {
      p.loss[r] = red[0] + red[1] + red[2] + red[3];
      if (p.stats) {
        p.stats[3 * r] = ls == -INFINITY ? -INFINITY : all.m;
        p.stats[3 * r + 1] = ls;
        p.stats[3 * r + 2] = ls == -INFINITY && TAIL ? -INFINITY : lr;
      }
    }
    if (MODE == kLossOnly) break;
    in = next;
    part = next_part;
  }
  ptx::let_next_begin();
}

// The statistics of a whole row's tokens off the list, by all threads of a block of kGradThreads.  list.id has been written before the last barrier.
constexpr int kSieve = 4096;   // granules are looked up on the list where granule mod kSieve is that of a listed token
struct OffList {
  uint32_t sieve[kSieve / 32];
  Warps<kGradThreads / 32> buf;
  float4 upper[kGradThreads];
};
struct NoOffList {};
template <int DT>
__device__ __forceinline__ Acc sum_off_list(const Row<DT> row, const List& list, int n, float k, OffList& sh) {
  constexpr int VE = Elem<DT>::VE, T = kGradThreads;
  const int tid = threadIdx.x;
  for (int i = tid; i < kSieve / 32; i += T) sh.sieve[i] = 0;
  __syncthreads();
  if (tid < n && list.id[tid] >= 0) {
    const int v = (row.ph + list.id[tid]) / VE % kSieve;
    atomicOr(&sh.sieve[v / 32], 1u << v % 32);
  }
  __syncthreads();
  const Part<DT> whole(row, 0, row.granules());
  Sums<DT, false, true> sums(k, sh.upper + tid);
  for (int i = tid; i < whole.n_all; i += T) {
    uint4 g[1] = {whole.raw(row, i)};
    const int v = whole.granule(i);
    if (sh.sieve[v % kSieve / 32] >> v % 32 & 1) {
      uint32_t bits = 0;
      for (int j = 0; j < n; ++j) {
        const int at = row.ph + list.id[j];
        if (list.id[j] >= 0 && at / VE == v) bits |= 1u << at % VE;
      }
      g[0] = without<DT>(g[0], bits);
    }
    sums.template pace<T, 1>(i - tid);
    sums.template add<true>(g, largest<DT>(g[0]));
  }
  warp_share<false>(sums.done(), k, sh.buf);
  __syncthreads();
  return warps_join<false>(k, sh.buf);
}

// A row whose student gives the tokens off the list no probability in 32 bits, but not -inf, is one block's: saved statistics do not hold how its
// remainder is spread (distill_coef), so the row is summed again, before any of it is replaced.  Not inlined, so that
// its registers are not other rows'.
template <int DT>
__device__ __noinline__ void grad_of_masked_rest(const DistillParams& p, int64_t r, const List& list, OffList& sh, float sum, float rest) {
  const Row<DT> in(p.logits, r, p.stride, p.vocab), out(p.dlogits, r, p.grad_stride, p.vocab);
  const int n = p.list_k;
  const float scale = p.scale, w = p.weight[r], m = p.stats[3 * r], ls = p.stats[3 * r + 1], lr = p.stats[3 * r + 2];
  const Acc dense = sum_off_list<DT>(in, list, n, scale * kLog2e, sh);
  const Coef c = distill_coef<true>(scale, sum, rest, m, ls, lr, dense.m, log_sum(dense), w);
  grad_part<DT, false>(in, out, Part<DT>(in, 0, in.granules()), c, list, n);
}

// With a remainder as many blocks an SM as the other form has by itself.
template <int DT, bool TAIL>
__global__ void __launch_bounds__(kGradThreads, TAIL ? 6 : 0) distill_grad_kernel(const __grid_constant__ DistillParams p) {
  __shared__ List list;
  __shared__ TeacherSums teacher;
  __shared__ typename std::conditional<TAIL, OffList, NoOffList>::type off;
  const int64_t r = blockIdx.x / p.split;
  const int tid = threadIdx.x;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const Row<DT> in(p.logits, r, p.stride, p.vocab), out(p.dlogits, r, p.grad_stride, p.vocab);
  const float w = p.weight[r], m = p.stats[3 * r], ls = p.stats[3 * r + 1], lr = p.stats[3 * r + 2];
  const Entry e = load_entry(p, r).checked(p);
  if (tid < kMaxList) list.id[tid] = e.id;
  const float x = share_entry<TAIL>(e, p.teacher_scale, teacher);
  __syncthreads();
  const float3 teach = join_entries<TAIL>(x, p.teacher_scale, teacher);
  if (tid < kMaxList) list.add[tid] = -w * p.scale * (e.id >= 0 ? teach.x : 0.f);
  const float rest = TAIL ? kept_rest(teach.z, ls, lr) : 0.f;
  const int part = blockIdx.x % p.split;
  if constexpr (TAIL) {
    if (!(rest == 0.f) && w != 0.f && lr != -INFINITY && ex2((lr - ls) * kLog2e) == 0.f) {   // alike in all blocks of the row
      if (part == 0) grad_of_masked_rest<DT>(p, r, list, off, teach.y, rest);
      return;
    }
  }
  const Coef c = distill_coef<TAIL>(p.scale, teach.y, rest, m, ls, lr, m, lr, w);
  grad_part<DT, false>(in, out, Part<DT>(in, part, p.each), c, list, p.list_k);
}

}  // namespace rows
}  // namespace iris

using namespace iris;
using namespace iris::rows;

namespace {

constexpr int kHoldBytes = 192 * 1024;   // of shared memory at most for a part
constexpr int kPartBytes = 60 * 1024;    // ... and where the row can be split further: three blocks' worth in an SM
constexpr int kMaxDevices = 64;

int check_distill(const char* fn, const iris_distill_args* a, int64_t* stride, int64_t* gstride) {
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  *stride = a->row_stride;
  IRIS_CHECK(check_logits(fn, "logits", a->logits, a->dtype, a->rows, a->vocab, stride));
  IRIS_CHECK(check_scale(fn, "scale", a->scale, kMaxScale));
  IRIS_CHECK(check_scale(fn, "teacher_scale", a->teacher_scale));
  if (a->mode != IRIS_DISTILL_RENORM && a->mode != IRIS_DISTILL_TAIL) return fail(IRIS_ERR_ARG, "%s: unknown mode %d", fn, a->mode);
  if (a->list_k < 0 || a->list_k > kMaxList) return fail(IRIS_ERR_ARG, "%s: list_k=%d not in [0, %d]", fn, a->list_k, kMaxList);
  if (a->dlogits) {
    *gstride = a->grad_stride;
    IRIS_CHECK(check_logits(fn, "dlogits", a->dlogits, a->dtype, a->rows, a->vocab, gstride));
    IRIS_CHECK(check_in_place(fn, a->logits, *stride, a->dlogits, *gstride, a->rows, a->vocab, a->dtype));
  }
  if (a->rows == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "teacher", a->teacher, 4, a->list_k > 0));
  IRIS_CHECK(check_aligned(fn, "teacher_ids", a->teacher_ids, 8, a->list_k > 0));
  IRIS_CHECK(check_aligned(fn, "weight", a->weight, 4, false));
  return IRIS_OK;
}

DistillParams params_of(const iris_distill_args* a, int64_t stride, int64_t gstride) {
  DistillParams p{};
  p.logits = a->logits;
  p.stride = stride;
  p.grad_stride = gstride;
  p.rows = (int)a->rows;
  p.vocab = (int)a->vocab;
  p.list_k = a->list_k;
  p.scale = a->scale;
  p.teacher_scale = a->teacher_scale;
  p.teacher = a->teacher;
  p.ids = a->teacher_ids;
  p.weight = a->weight;
  p.loss = a->loss;
  p.stats = a->stats;
  p.dlogits = a->dlogits;
  return p;
}

template <int DT, bool TAIL, int MODE>
int launch_distill(const DistillParams& p, cudaStream_t st) {
  const auto kernel = distill_kernel<DT, TAIL, MODE>;
  const int bytes = (MODE == kHeld ? p.hold * 16 : 0) + (p.hold + 3) / 4 * 4;
  static std::atomic<bool> configured[kMaxDevices] = {};   // calls may come from several threads; the setting may be made twice
  int dev = -1;
  IRIS_CUDA_TRY(cudaGetDevice(&dev));
  if (dev >= kMaxDevices || !configured[dev].load(std::memory_order_acquire)) {
    IRIS_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHoldBytes + kHoldBytes / 16));
    if (dev < kMaxDevices) configured[dev].store(true, std::memory_order_release);
  }
  if (MODE == kLossOnly) return launch_rows(kernel, p, (unsigned)((int64_t)p.rows * p.split), p.split, kDistillThreads, (size_t)bytes, st);
  // As many clusters as the device holds at a time: one more would run after the others have done all their rows.  The
  // answer is kept (it depends on the kernel, the split and the bytes alone), as asking takes longer than a small launch.
  int clusters = 0;
  static std::atomic<uint64_t> known[kMaxSplit + 1];
  const uint64_t key = (uint64_t)(dev + 1) << 48 | (uint64_t)bytes << 16;
  const uint64_t was = known[p.split].load(std::memory_order_relaxed);
  if ((was & ~0xffffull) == key) {
    clusters = (int)(was & 0xffff);
  } else {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)p.split);
    cfg.blockDim = dim3(kDistillThreads);
    cfg.dynamicSmemBytes = (size_t)bytes;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)p.split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = p.split > 1 ? 1 : 0;
    if (p.split > 1) IRIS_CUDA_TRY(cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg));
    else IRIS_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&clusters, kernel, kDistillThreads, (size_t)bytes));
    if (p.split == 1) clusters *= kSms;
    clusters = std::max(1, std::min(clusters, 0xffff));
    known[p.split].store(key | (uint64_t)clusters, std::memory_order_relaxed);
  }
  return launch_rows(kernel, p, (unsigned)(std::min(clusters, p.rows) * p.split), p.split, kDistillThreads, (size_t)bytes, st);
}

template <int DT>
int launch_distill(DistillParams p, bool tail, cudaStream_t st) {
  // With a gradient a row is shared by a cluster of blocks until a part is at most kPartBytes of shared memory (parts of 36,
  // 48, 60, 72 and 100 KB: 642, 585, 559, 611 and 672 us for 4096 x 128000 at the time); with or without one, while the
  // rows alone leave SMs without work and every thread still has a granule.
  const int64_t granules = part_granules(p.logits, p.stride, p.vocab, DT, 1);
  int split = 1;
  while (split < kMaxSplit && ((p.dlogits && granules * 16 > (int64_t)split * kPartBytes) ||
                               ((int64_t)p.rows * split < 2 * kSms && granules >= (int64_t)split * 2 * kDistillThreads)))
    ++split;
  p.split = split;
  p.each = part_granules(p.logits, p.stride, p.vocab, DT, split);
  p.hold = std::max(1, std::min(p.each, kHoldBytes / 16));
  if (!p.dlogits) return tail ? launch_distill<DT, true, kLossOnly>(p, st) : launch_distill<DT, false, kLossOnly>(p, st);
  if (p.each <= kHoldBytes / 16) return tail ? launch_distill<DT, true, kHeld>(p, st) : launch_distill<DT, false, kHeld>(p, st);
  return tail ? launch_distill<DT, true, kReadTwice>(p, st) : launch_distill<DT, false, kReadTwice>(p, st);
}

template <int DT, bool TAIL>
int launch_distill_grad(const DistillParams& p, int64_t rows, cudaStream_t st) {
  return launch_rows(distill_grad_kernel<DT, TAIL>, p, (unsigned)(rows * p.split), 1, kGradThreads, 0, st);
}

}  // namespace

extern "C" int iris_distill_topk(const iris_distill_args* a, void* stream) {
  const char* fn = "iris_distill_topk";
  int64_t stride = 0, gstride = 0;
  IRIS_CHECK(check_distill(fn, a, &stride, &gstride));
  if (a->rows == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "loss", a->loss, 4, true));
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, false));
  const DistillParams p = params_of(a, stride, gstride);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tail = a->mode == IRIS_DISTILL_TAIL;
  if (a->dtype == IRIS_BF16) return launch_distill<IRIS_BF16>(p, tail, st);
  if (a->dtype == IRIS_F16) return launch_distill<IRIS_F16>(p, tail, st);
  return launch_distill<IRIS_F32>(p, tail, st);
}

extern "C" int iris_distill_topk_backward(const iris_distill_args* a, void* stream) {
  const char* fn = "iris_distill_topk_backward";
  int64_t stride = 0, gstride = 0;
  IRIS_CHECK(check_distill(fn, a, &stride, &gstride));
  if (a->rows == 0 || a->vocab == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "stats", a->stats, 4, true));
  IRIS_CHECK(check_aligned(fn, "weight", a->weight, 4, true));
  if (!a->dlogits) return fail(IRIS_ERR_ARG, "%s: dlogits is NULL", fn);
  DistillParams p = params_of(a, stride, gstride);
  p.split = grad_parts(a->vocab, a->dtype);
  p.each = part_granules(a->logits, stride, a->vocab, a->dtype, p.split);
  if (a->rows * p.split > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 blocks", fn);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool tail = a->mode == IRIS_DISTILL_TAIL;
  if (a->dtype == IRIS_BF16) return tail ? launch_distill_grad<IRIS_BF16, true>(p, a->rows, st) : launch_distill_grad<IRIS_BF16, false>(p, a->rows, st);
  if (a->dtype == IRIS_F16) return tail ? launch_distill_grad<IRIS_F16, true>(p, a->rows, st) : launch_distill_grad<IRIS_F16, false>(p, a->rows, st);
  return tail ? launch_distill_grad<IRIS_F32, true>(p, a->rows, st) : launch_distill_grad<IRIS_F32, false>(p, a->rows, st);
}
