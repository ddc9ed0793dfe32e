// Embedding lookup in a table cut by rows into shards (the head's B shards are one), and its gradient by sorted tokens.
//
//   y_i = scale E[t_i];   dE[v] = scale * sum over i with t_i = v of dy_i
#include "any_rows.cuh"

namespace iris {
namespace rows {

// ---- lookup --------------------------------------------------------------------------------------------------------
constexpr int64_t kMaxTokens = 1 << 30;   // places, and those a little behind the last, are counted in 32 bits
constexpr int kEmbedThreads = 256;

struct EmbedParams {
  const char* shard[IRIS_MAX_WORLD];
  int64_t shard_stride, out_stride;   // bytes
  const int64_t* tokens;
  char* out;
  int64_t n, vocab;
  uint32_t per, each;                 // rows of a shard; warps of a row
  int bytes;                          // of a row
  float scale;
};

// 16 bytes from byte b of the row on, all of which lie in it, though the aligned ones that they touch do not.
template <int ES>
__device__ __forceinline__ uint4 load_apart(const char* from, int b) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = ES == 4 ? *reinterpret_cast<const uint32_t*>(from + b + i * 4)
                   : *reinterpret_cast<const uint16_t*>(from + b + i * 4) | (uint32_t)*reinterpret_cast<const uint16_t*>(from + b + i * 4 + 2) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// For those 16 bytes of each 512 that lie in the row; begin: byte of the row, of this thread.
template <int ES, int U>
__device__ __forceinline__ void load_like(const char* from, int begin, int bytes, uint4 (&v)[U]) {
  const int a = (int)phase(from + begin), lane = threadIdx.x & 31;   // a: the same for all threads
  const bool inside = begin - lane * 16 - a >= 0 && begin - lane * 16 - a + U * 512 + 16 <= bytes;
  const char* const p = from + begin - a;
  uint4 next[U];
  if (inside) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[u] = ld_global_v4(p + u * 512);
      if (a) next[u] = ld_global_v4(p + u * 512 + 16);
    }
    if (a) cut_all(v, next, a);
    return;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int b = begin + u * 512;
    v[u] = next[u] = make_uint4(0, 0, 0, 0);
    if (b - a >= 0 && b - a + (a ? 32 : 16) <= bytes) {
      v[u] = ld_global_v4(p + u * 512);
      if (a) next[u] = ld_global_v4(p + u * 512 + 16);
    }
  }
  if (a) cut_all(v, next, a);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int b = begin + u * 512;
    if (a && b >= 0 && b + 16 <= bytes && !(b - a >= 0 && b - a + 32 <= bytes)) v[u] = load_apart<ES>(from, b);
  }
}
// What does not fill 16 aligned bytes of the output: its first elements and its last ones, one a thread.  `first`, `last`: whether the warp looks after them.
template <int DT>
__device__ __forceinline__ void move_ends(const char* from, char* to, int bytes, float scale, bool first, bool last) {
  using E = Elem<DT>;
  using T = typename E::T;
  constexpr int ES = sizeof(T);
  const int lane = threadIdx.x & 31, head = (int)(-phase(to) & 15), tail = bytes - (int)phase(to + bytes);
  int b = -1;
  if (lane < 8) {
    if (first && lane * ES < min(head, bytes)) b = lane * ES;
  } else if (lane < 16) {
    if (last && tail >= head && tail + (lane - 8) * ES < bytes) b = tail + (lane - 8) * ES;
  }
  if (b < 0) return;
  const T x = from ? *reinterpret_cast<const T*>(from + b) : E::from(0.f);
  *reinterpret_cast<T*>(to + b) = scale == 1.f ? x : E::from(E::to(x) * scale);
}
template <int DT>
__device__ __forceinline__ uint4 scaled(const uint4& v, float scale) {
  using E = Elem<DT>;
  float x[E::VE];
  E::unpack(v, x);
#pragma unroll
  for (int e = 0; e < E::VE; ++e) x[e] *= scale;
  return E::pack(x);
}
__device__ __forceinline__ const char* embed_row(const EmbedParams& p, int64_t i) {
  const int64_t t = p.tokens[i];
  if (t < 0 || t >= p.vocab) return nullptr;
  const uint32_t r = (uint32_t)t / p.per;
  return p.shard[r] ? p.shard[r] + (int64_t)((uint32_t)t - r * p.per) * p.shard_stride : nullptr;
}

// A warp moves U times 512 bytes of a row of the output, 16 aligned bytes a thread at a time.  Where the table's row does not lie like the output's,
// those are cut out of two of the table's, of which the second are the next thread's first and come from L1.
//
// 32768 x 4096 bf16 70 us, 74 % of the copy rate; 32771 x 4099 fp16, where no two rows lie alike, 84 us (62 %): token, row and store come one after the other
// in a warp, 32 warps an SM.  With the ends of a row moved by single threads one element after the other 116 us; shifts by selections instead of cases 118; parts
// of all rows counted through, with a division a thread, 147.  64 rows of 8192: 6.2 us, of which the launch and three latencies are nearly all.
template <int DT, int U>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const __grid_constant__ EmbedParams p) {
  constexpr int ES = sizeof(typename Elem<DT>::T);
  const int lane = threadIdx.x & 31;
  constexpr uint32_t kWarps = kEmbedThreads / 32;
  const uint32_t q = blockIdx.x / p.each, in = (blockIdx.x - q * p.each) * kWarps + (threadIdx.x >> 5), down = in / p.each;
  const int64_t i = (int64_t)q * kWarps + down;
  const int part = (int)(in - down * p.each);
  ptx::let_next_begin();
  ptx::begin_after_previous();
  if (i >= p.n) return;
  char* const to = p.out + i * p.out_stride;
  const char* const from = embed_row(p, i);
  const int begin = part * (U * 512) - (int)phase(to) + lane * 16;   // byte of the row
  uint4 v[U];
  if (from) {
    load_like<ES>(from, begin, p.bytes, v);
    if (p.scale != 1.f) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = scaled<DT>(v[u], p.scale);
    }
  } else {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int b = begin + u * 512;
    if (b >= 0 && b + 16 <= p.bytes) st_global_v4(to + b, v[u]);
  }
  if (part == 0 || part + 1 == (int)p.each) move_ends<DT>(from, to, p.bytes, p.scale, part == 0, part + 1 == (int)p.each);
}

// Short rows, of at most 16 * L bytes with what their ends touch: L threads a row, and U rows of theirs under way at a time.
template <int DT, int L>
__global__ void __launch_bounds__(kEmbedThreads) embed_short_kernel(const __grid_constant__ EmbedParams p) {
  constexpr int ES = sizeof(typename Elem<DT>::T), U = 4;
  const int64_t first = ((int64_t)blockIdx.x * kEmbedThreads + threadIdx.x) / L * U;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const char* from[U];
#pragma unroll
  for (int u = 0; u < U; ++u) from[u] = first + u < p.n ? embed_row(p, first + u) : nullptr;
  uint4 v[U], next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    v[u] = next[u] = make_uint4(0, 0, 0, 0);
    if (!from[u]) continue;
    const int begin = (threadIdx.x % L) * 16 - (int)phase(p.out + (first + u) * p.out_stride), a = (int)phase(from[u] + begin);
    v[u] = edge_load<ES>(from[u], begin - a, p.bytes);
    if (a) next[u] = edge_load<ES>(from[u], begin - a + 16, p.bytes);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (first + u >= p.n) break;
    char* const to = p.out + (first + u) * p.out_stride;
    const int b = (threadIdx.x % L) * 16 - (int)phase(to);
    uint4 w = cut(v[u], next[u], phase(from[u] + b));
    if (p.scale != 1.f) w = scaled<DT>(w, p.scale);
    if (b >= 0 && b + 16 <= p.bytes) st_global_v4(to + b, w);
    else if (b > -16 && b < p.bytes) store_elements<ES>(to + b, to, to + p.bytes, w);
  }
}

template <int DT>
static int launch_embed(EmbedParams p, bool aligned, cudaStream_t st) {
  const int bytes = p.bytes + (aligned ? 0 : 16 - (int)elem_size(DT));   // that the aligned 16 bytes touched by a row may have
  const bool few = p.n * ((bytes + 2047) / 2048) < (int64_t)kSms * 64;   // rather more warps
  int64_t blocks;
  void (*kernel)(EmbedParams);
  if (bytes <= 512 && !few) {
    const int threads = bytes <= 128 ? 8 : bytes <= 256 ? 16 : 32;   // of a row
    kernel = threads == 8 ? embed_short_kernel<DT, 8> : threads == 16 ? embed_short_kernel<DT, 16> : embed_short_kernel<DT, 32>;
    blocks = ((p.n + 3) / 4 * threads + kEmbedThreads - 1) / kEmbedThreads;
  } else {
    const int runs = (bytes + 511) / 512, most = few ? 1 : 4, each = (runs + most - 1) / most, u = (runs + each - 1) / each;   // equal parts of a row
    p.each = (uint32_t)((runs + u - 1) / u);
    kernel = u == 1 ? embed_kernel<DT, 1> : u == 2 ? embed_kernel<DT, 2> : u == 3 ? embed_kernel<DT, 3> : embed_kernel<DT, 4>;
    blocks = (p.n * p.each + kEmbedThreads / 32 - 1) / (kEmbedThreads / 32);
  }
  if (blocks > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "iris_embed_tokens: more than 2^31 - 1 blocks");
  return launch_rows(kernel, p, (unsigned)blocks, 1, kEmbedThreads, 0, st);
}

// ---- gradient: sorted tokens ---------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kSortBlocks = 16;     // one cluster
constexpr int kSortMaxBits = 10;    // of a digit

struct SortParams {
  const int64_t* tokens;
  int n;
  uint32_t vocab, per, present;     // present: a bit for each shard that is there, all set: each is
  uint2* lists[2];                  // (token, place): of pass 0, 2, .. and 1, 3, ..
  uint32_t* used;                   // a bit for each row of the table that a token names; nullptr: not wanted
  int passes, split;
};

template <class P>
__device__ __forceinline__ uint32_t key_of(const P& p, int64_t t) {   // vocab: no token, behind all others
  if (t < 0 || t >= p.vocab) return p.vocab;
  return p.present == ~0u || p.present >> ((uint32_t)t / p.per) & 1 ? (uint32_t)t : p.vocab;
}

// Tokens in rising order, equal ones in the order of their places, so that the sums over them have one order: a radix sort by one cluster.
// Each warp has a run of the places and counts its digits; a digit's places follow from the counts of all warps before; then the warps
// place their runs, 32 at a time.  Buffers lie in global memory (L2); what one block writes and another reads is ordered by the cluster's barrier.
// Bound by latencies and the instructions of 16 SMs (65536 tokens of 16 bits: 25 us; 9001: 15; 1000, by one block: 9): kSortItems loads of a thread are under way at a time, and keys stay in registers between counting and placing where a thread has no more
// than that.  Threads with equal digits find one another by a vote on each bit, as the instruction that finds them at once takes far longer (65536
// tokens of 16 bits: 40 us with it).
constexpr int kSortItems = 8;

// The threads of the warp that are there and have the same digit.
template <int BITS>
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, bool there) {
  uint32_t same = __ballot_sync(~0u, there);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const bool one = digit >> b & 1;
    const uint32_t ones = __ballot_sync(~0u, one);
    same &= one ? ones : ~ones;
  }
  return same;
}

template <int BITS>
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ uint32_t count[];   // [kSortWarps, digits]; totals [split, digits]; base [digits]
  __shared__ uint32_t of_warp[kSortWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int digits = 1 << BITS;
  const int rank = p.split > 1 ? (int)ptx::cluster_ctarank() : 0;
  uint32_t* const mine = count + warp * digits;
  uint32_t* const totals = count + kSortWarps * digits;
  uint32_t* const base = totals + p.split * digits;
  const int each = (int)(((int64_t)p.n + p.split * kSortWarps * 32 - 1) / (p.split * kSortWarps * 32)) * 32;
  const int64_t b64 = (int64_t)(rank * kSortWarps + warp) * each;
  const int begin = (int)(b64 < p.n ? b64 : p.n), end = (int)(b64 + each < p.n ? b64 + each : p.n);
  if (p.split > 1) ptx::cluster_arrive_release();
  ptx::let_next_begin();
  ptx::begin_after_previous();
  if (p.used)   // set behind the first pass's barrier
    for (uint32_t i = rank * kSortThreads + tid; i < (p.vocab + 31) / 32; i += p.split * kSortThreads) p.used[i] = 0;
  const bool held = each <= 32 * kSortItems;
  uint32_t key[kSortItems], place[kSortItems], same[kSortItems];
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * BITS;
    const uint2* const from = p.lists[pass & 1 ^ 1];
    uint2* const list = p.lists[pass & 1];
    const auto load = [&](int at) {
      if (pass) {
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
          const uint2 x = at + k * 32 + lane < end ? __ldcg(from + at + k * 32 + lane) : make_uint2(0, 0);
          key[k] = x.x;
          place[k] = x.y;
        }
      } else {
        int64_t t[kSortItems];
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) t[k] = at + k * 32 + lane < end ? p.tokens[at + k * 32 + lane] : -1;
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
          key[k] = key_of(p, t[k]);
          place[k] = (uint32_t)(at + k * 32 + lane);
        }
      }
    };
    for (int i = tid; i < kSortWarps * digits; i += kSortThreads) count[i] = 0;
    __syncthreads();
    for (int at = begin; at < end; at += 32 * kSortItems) {
      load(at);
#pragma unroll
      for (int k = 0; k < kSortItems; ++k) {
        if (at + k * 32 >= end) break;
        const bool there = at + k * 32 + lane < end;
        const uint32_t d = key[k] >> shift & (digits - 1);
        same[k] = same_digit<BITS>(d, there);
        if (there && (same[k] & ((1u << lane) - 1)) == 0) mine[d] += __popc(same[k]);
        __syncwarp();
      }
    }
    if (p.split > 1 && pass == 0) ptx::cluster_wait();   // all blocks have started
    __syncthreads();
    if (tid < digits) {
      uint32_t c[kSortWarps], sum = 0;
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) c[w] = count[w * digits + tid];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        count[w * digits + tid] = sum;
        sum += c[w];
      }
      if (p.split > 1)
        for (int s = 0; s < p.split; ++s) ptx::st_shared_cluster_u32(ptx::mapa(ptx::smem_u32(totals + rank * digits + tid), s), sum);
      else totals[tid] = sum;
    }
    if (p.split > 1) ptx::cluster_sync();
    else __syncthreads();
    uint32_t all = 0, before = 0;
    if (tid < digits)
      for (int s = 0; s < p.split; ++s) {
        const uint32_t c = totals[s * digits + tid];
        before += s < rank ? c : 0;
        all += c;
      }
    uint32_t up = all;   // sums over the digits up to this one
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t x = __shfl_up_sync(~0u, up, o);
      if (lane >= o) up += x;
    }
    if (lane == 31) of_warp[warp] = up;
    __syncthreads();
    uint32_t w = of_warp[lane];
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const uint32_t x = __shfl_up_sync(~0u, w, o);
      if (lane >= o) w += x;
    }
    w = __shfl_sync(~0u, w, max(warp - 1, 0));
    if (tid < digits) base[tid] = up - all + (warp ? w : 0) + before;
    __syncthreads();
    for (int at = begin; at < end; at += 32 * kSortItems) {
      if (!held) load(at);
#pragma unroll
      for (int k = 0; k < kSortItems; ++k) {
        if (at + k * 32 >= end) break;
        const bool there = at + k * 32 + lane < end;
        const uint32_t d = key[k] >> shift & (digits - 1);
        if (!held) same[k] = same_digit<BITS>(d, there);
        const uint32_t lower = same[k] & ((1u << lane) - 1);
        if (there) {
          const uint32_t to = base[d] + mine[d] + __popc(lower);
          list[to] = make_uint2(key[k], place[k]);
          if (pass == 0 && p.used && key[k] < p.vocab) atomicOr(p.used + (key[k] >> 5), 1u << (key[k] & 31));
        }
        __syncwarp();
        if (there && lower == 0) mine[d] += __popc(same[k]);
        __syncwarp();
      }
    }
    if (p.split > 1) ptx::cluster_sync();
    else __syncthreads();
  }
}

// ---- gradient: sums ------------------------------------------------------------------------------------------------
constexpr int kSumThreads = 256, kSumWarps = kSumThreads / 32;
constexpr int kFillBytes = 8192;    // that a warp clears

struct EmbedGradParams {
  const char* dy;
  int64_t dy_stride;                // bytes
  char* shard[IRIS_MAX_WORLD];
  int64_t shard_stride;             // bytes
  const uint2* list;                // (token, place), sorted
  const uint32_t* used;
  const int64_t* tokens;            // of the kernel for few of them
  float* parts;                     // [chunks, 2, part_stride]: sums of the run at a chunk's start and of the one at its end, where they go on beyond it
  int n, chunk, chunks, dim, part_stride, tiles, fill_parts, fill_shift;   // chunk: sorted places of a chunk
  uint32_t vocab, per, present;     // present: see SortParams
  unsigned sum_blocks;
  float scale;
  int accumulate, aligned;          // aligned: grad_out and the shards begin at 16 bytes
};

template <int ES>
__device__ __forceinline__ void store_zero(char* at) {
  if (ES == 4) *reinterpret_cast<uint32_t*>(at) = 0;
  else *reinterpret_cast<uint16_t*>(at) = 0;
}
__device__ __forceinline__ char* table_row(const EmbedGradParams& p, uint32_t v) {
  const uint32_t r = v / p.per;
  return p.shard[r] ? p.shard[r] + (int64_t)(v - r * p.per) * p.shard_stride : nullptr;
}
__device__ __forceinline__ uint4 pairs(uint64_t a, uint64_t b) { return make_uint4((uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)); }
// All threads of a warp: their columns of row v, from column `begin` on; `at`: shared memory of the warp's, Segment<GT, I>::kBytes.
template <int GT, int I, bool ALIGNED>
__device__ __forceinline__ void write_row(const EmbedGradParams& p, uint32_t v, uint32_t at, int begin, const uint64_t (&sum)[I][kLaneColumns / 2]) {
  using C = Columns<GT>;
  char* const row = table_row(p, v);
  uint4 w[I * C::N];
#pragma unroll
  for (int i = 0; i < I; ++i) {
    uint64_t x[kLaneColumns / 2];
#pragma unroll
    for (int e = 0; e < kLaneColumns / 2; ++e) x[e] = mul2f(sum[i][e], pair(p.scale, p.scale));
    if (p.accumulate) {
      float old[kLaneColumns];
      C::load(row, begin + i * kWarpColumns + (threadIdx.x & 31) * kLaneColumns, p.dim, old);
#pragma unroll
      for (int e = 0; e < kLaneColumns / 2; ++e) x[e] = add2f(x[e], pair(old[2 * e], old[2 * e + 1]));
    }
    C::pack2(x, w + i * C::N);
  }
  __syncwarp();
  Segment<GT, I, ALIGNED>::write(at, row, begin, p.dim, w);
}

// Zeros in bytes lo .. hi - 1, by a warp.
template <int ES>
__device__ __forceinline__ void clear(char* lo, char* hi) {
  const int lane = threadIdx.x & 31;
  char* const begin = lo + (-phase(lo) & 15);
  char* const end = hi - phase(hi);
  if (begin > end) {   // within 16 aligned bytes
    if (lo + lane * ES < hi) store_zero<ES>(lo + lane * ES);
    return;
  }
  if (lane < 8) {
    if (lo + lane * ES < begin) store_zero<ES>(lo + lane * ES);
  } else if (lane < 16) {
    if (end + (lane - 8) * ES < hi) store_zero<ES>(end + (lane - 8) * ES);
  }
  for (char* at = begin + lane * 16; at < end; at += 512) st_global_v4(at, make_uint4(0, 0, 0, 0));
}
// Zeros in the rows that no token names: a warp has 2^fill_shift rows, or kFillBytes of one.  used: a bit for each of the rows.
template <int GT>
__device__ __forceinline__ void fill_rows(const EmbedGradParams& p, int64_t v0, int part, uint32_t used) {
  constexpr int ES = Columns<GT>::ES;
  const int64_t bytes = (int64_t)p.dim * ES;
  const int64_t left = p.vocab - v0;
  const int rows = 1 << p.fill_shift, n = left < rows ? (int)left : rows;
  if (n <= 0) return;
  if (p.fill_parts > 1) {
    char* const row = used & 1 ? nullptr : table_row(p, (uint32_t)v0);
    if (row) clear<ES>(row + (int64_t)part * kFillBytes, row + min(bytes, (int64_t)(part + 1) * kFillBytes));
    return;
  }
  for (int b = 0; b < n;) {   // rows side by side are cleared at once
    int m = used >> b & 1 ? 0 : 1;
    char* const row = m ? table_row(p, (uint32_t)v0 + b) : nullptr;
    if (row) {
      if (p.shard_stride == bytes)
        while (b + m < n && !(used >> (b + m) & 1) && table_row(p, (uint32_t)v0 + b + m) == row + m * bytes) ++m;
      clear<ES>(row, row + m * bytes);
    }
    b += m ? m : 1;
  }
}

// A warp adds up a chunk of the sorted places over 256 columns.  A run of equal tokens that lies inside a chunk is finished here; one that goes on
// in other chunks leaves its sums in `parts`, for embed_join_kernel.
//
// The rows are on their way to shared memory up to 12 ahead.  The rows that no token names are cleared by further warps of the same launch: nearly free beside the
// sums (65536 x 4096 bf16 to 32768 fp32 rows: 164 us with them, 162 without; 6.5 TB/s).  256 columns a warp: 245 us.  Rows at any element: 9001 x 2561 in 30 us,
// bound by instructions.
template <int DT, int I>
constexpr int sum_stages() { return (DT == IRIS_F32 ? 8 : 12) / I; }   // about 8 KB or 6 KB a warp
template <int DT, int GT, int I>
constexpr int sum_bytes() { return sum_stages<DT, I>() * Segment<DT, I>::kBytes + Segment<GT, I>::kBytes; }   // of a warp

template <int DT, int GT, int I, bool ALIGNED>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const __grid_constant__ EmbedGradParams p) {
  using G = Segment<DT, I, ALIGNED>;
  constexpr int kStages = sum_stages<DT, I>(), H = kLaneColumns / 2;
  extern __shared__ __align__(16) char ring[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  if (blockIdx.x >= p.sum_blocks) {
    const int64_t unit = (int64_t)(blockIdx.x - p.sum_blocks) * kSumWarps + warp, v0 = unit / p.fill_parts << p.fill_shift;
    if (v0 < p.vocab) fill_rows<GT>(p, v0, (int)(unit % p.fill_parts), p.used[v0 >> 5] >> (v0 & 31));
    return;
  }
  const int64_t unit = (int64_t)blockIdx.x * kSumWarps + warp;
  const int c = (int)(unit / p.tiles), column = (int)(unit % p.tiles) * G::kColumns, first = column + lane * kLaneColumns;
  if (c >= p.chunks) return;
  const uint32_t own = ptx::smem_u32(ring) + warp * sum_bytes<DT, GT, I>(), out = own + kStages * G::kBytes;
  const int begin = c * p.chunk, end = min(p.n, begin + p.chunk);
  // 32 entries are held by the threads, and the next 32, as copies begin ahead.
  const auto entry = [&](int i) { return i < end ? p.list[i] : make_uint2(p.vocab, 0); };
  uint32_t now = p.list[begin].x;
  if (now >= p.vocab) return;
  bool goes_on = begin > 0 && p.list[begin - 1].x == now;   // the run came from the chunk before
  uint2 held = entry(begin + lane), next = entry(begin + 32 + lane);
  uint64_t sum[I][H] = {};
  typename G::Lone lone;
  const auto row_of = [&](uint32_t i) { return p.dy + (int64_t)i * p.dy_stride; };
  const auto fetch = [&](int i, int base, uint32_t to) {   // base: of `held`
    lone.settle();
    if (i < end) {
      const uint32_t at = __shfl_sync(~0u, i - base < 32 ? held.y : next.y, (i - base) & 31);
      G::fetch(to, row_of(at), column, p.dim, lone);
    }
    copy_async_commit();
  };
  const auto finish = [&](bool more) {   // more: the run goes on in the next chunk
    if (!goes_on && !more) {
      write_row<GT, I, ALIGNED>(p, now, out, column, sum);
    } else {
      float* const to = p.parts + ((int64_t)2 * c + !goes_on) * p.part_stride + first;
#pragma unroll
      for (int i = 0; i < I; ++i)
        if (first + i * kWarpColumns < p.dim) {
          st_global_v4(to + i * kWarpColumns, pairs(sum[i][0], sum[i][1]));
          st_global_v4(to + i * kWarpColumns + 4, pairs(sum[i][2], sum[i][3]));
        }
    }
  };
#pragma unroll 1
  for (int k = 0; k < kStages - 1; ++k) fetch(begin + k, begin, own + k * G::kBytes);
  int base = begin;
  uint32_t here = own, before = own + (kStages - 1) * G::kBytes;
#pragma unroll 1
  for (int i = begin; i < end; ++i) {
    if (i - base == 32) {
      base = i;
      held = next;
      next = entry(base + 32 + lane);
    }
    const uint32_t k = __shfl_sync(~0u, held.x, i - base);
    if (k != now) {
      finish(false);
      if (k >= p.vocab) break;
      now = k;
      goes_on = false;
#pragma unroll
      for (int r = 0; r < I; ++r)
#pragma unroll
        for (int e = 0; e < H; ++e) sum[r][e] = 0;
    }
    lone.settle();
    copy_async_wait_but<kStages - 2>();
    __syncwarp();
    fetch(i + kStages - 1, base, before);
    const char* const row = ALIGNED ? nullptr : row_of(__shfl_sync(~0u, held.y, i - base));
#pragma unroll
    for (int r = 0; r < I; ++r) {
      uint64_t x[H];
      G::read(here, row, column, p.dim, r, x);
#pragma unroll
      for (int e = 0; e < H; ++e) sum[r][e] = add2f(sum[r][e], x[e]);
    }
    before = here;
    here = here == own + (kStages - 1) * G::kBytes ? own : here + G::kBytes;
    if (i + 1 == end) finish(end < p.n && p.list[end].x == now);
  }
  copy_async_wait();   // a block does not end while copies are under way
}

// Runs that go over several chunks: the sums of their parts (13 us where 65536 tokens have 591 chunks: two waves of a launch and four latencies).  A warp looks after the run that begins in a chunk and goes on beyond it, over 256 columns;
// the parts of a long one are shared by the warps of the block.
constexpr int kJoinWarps = 16, kLongRun = 16;

template <int GT>
__global__ void __launch_bounds__(kJoinWarps * 32) embed_join_kernel(const __grid_constant__ EmbedGradParams p) {
  constexpr int kOut = Segment<GT, 1>::kBytes;
  __shared__ __align__(16) char out[kJoinWarps][kOut > kWarpColumns * 4 ? kOut : kWarpColumns * 4];
  __shared__ int lasts[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const int tiles = (p.dim + kWarpColumns - 1) / kWarpColumns;
  const int c0 = (int)(blockIdx.x / tiles) * kJoinWarps, column = (int)(blockIdx.x % tiles) * kWarpColumns, first = column + lane * kLaneColumns;
  const auto key_at = [&](int64_t i) { return i < p.n ? p.list[i].x : p.vocab; };   // vocab: no token
  // The chunks c + 1 .. last - 1 begin with the run of chunk c (or there is none: 0).
  const auto last_of = [&](int c) -> int {
    const int64_t begin = (int64_t)c * p.chunk, end = begin + p.chunk;
    const uint32_t key = key_at(end - 1), after = key_at(end), before = begin ? key_at(begin - 1) : p.vocab;
    if (key >= p.vocab || after != key || before == key) return 0;
    int last = c + 1;
    for (;;) {
      const uint32_t there = __ballot_sync(~0u, last + lane < p.chunks && key_at((int64_t)(last + lane) * p.chunk) == key);
      last += __popc(there);   // of consecutive chunks, as the keys are sorted
      if (there != ~0u) return last;
    }
  };
  float sum[kLaneColumns];
  const auto add = [&](int c, int from, int step, int last) {   // parts from, from + step .. of the run of chunk c
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) sum[e] = 0.f;
    for (int i = from; i < last; i += 4 * step) {
      float x[4][kLaneColumns];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = i + u * step;
        const float* const at = p.parts + ((int64_t)2 * k + (k == c)) * p.part_stride + first;
        const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 a = k < last && first < p.dim ? __ldcg(reinterpret_cast<const float4*>(at)) : none;
        const float4 b = k < last && first < p.dim ? __ldcg(reinterpret_cast<const float4*>(at + 4)) : none;
        x[u][0] = a.x, x[u][1] = a.y, x[u][2] = a.z, x[u][3] = a.w, x[u][4] = b.x, x[u][5] = b.y, x[u][6] = b.z, x[u][7] = b.w;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < kLaneColumns; ++e) sum[e] += x[u][e];
    }
  };
  const auto write = [&](int c, uint32_t at) {
    uint64_t x[1][kLaneColumns / 2];
#pragma unroll
    for (int e = 0; e < kLaneColumns / 2; ++e) x[0][e] = pair(sum[2 * e], sum[2 * e + 1]);
    write_row<GT, 1, false>(p, p.list[(int64_t)c * p.chunk + p.chunk - 1].x, at, column, x);
  };
  const int c = c0 + warp, last = c < p.chunks ? last_of(c) : 0;
  if (lane == 0) lasts[warp] = last - c > kLongRun ? last : 0;
  if (last && last - c <= kLongRun) {
    add(c, c, 1, last);
    write(c, ptx::smem_u32(out[warp]));
  }
  for (int w = 0; w < kJoinWarps; ++w) {
    __syncthreads();
    const int run = c0 + w, until = lasts[w];
    if (!until) continue;   // all warps
    add(run, run + warp, kJoinWarps, until);
    float* const own = reinterpret_cast<float*>(out[warp]);
    __syncwarp();
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) own[lane * kLaneColumns + e] = sum[e];
    __syncthreads();
    if (warp == 0) {
      for (int v = 1; v < kJoinWarps; ++v)
#pragma unroll
        for (int e = 0; e < kLaneColumns; ++e) sum[e] += reinterpret_cast<const float*>(out[v])[lane * kLaneColumns + e];
      write(run, ptx::smem_u32(out[0]));
    }
  }
}

// Few tokens, without sorting: a warp looks after one place and 256 columns, and adds up the rows of all places with its token, in their order, if it
// is the first of them; other warps clear the rows that no token names.  64 tokens, 8192 rows of 1024: 8 us instead of 24; 400: 10.5 instead of 25.
// Where nearly all tokens are one, its warps take 0.11 us a row, the latency of the seven rows under way: 150 of 500 make it 22 us, all 500 55, sorting 20.
constexpr int kFewTokens = 512;

template <int DT, int GT, bool ALIGNED>
struct Few {
  using G = Segment<DT, 1, ALIGNED>;
  static constexpr int kStages = 8, kWarp = kStages * G::kBytes + Segment<GT, 1>::kBytes + kFewTokens * 2;   // rows, a row of the result, places
  static constexpr int kBytes = kFewTokens * 4 + kSumWarps * kWarp;                                          // tokens
};
template <int DT, int GT, bool ALIGNED>
__global__ void __launch_bounds__(kSumThreads) embed_few_kernel(const __grid_constant__ EmbedGradParams p) {
  using F = Few<DT, GT, ALIGNED>;
  using G = typename F::G;
  constexpr int H = kLaneColumns / 2, kStages = F::kStages;
  extern __shared__ __align__(16) char few[];
  uint32_t* const keys = reinterpret_cast<uint32_t*>(few);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const int64_t unit = (int64_t)blockIdx.x * kSumWarps + warp;
  for (int i = threadIdx.x; i < kFewTokens; i += kSumThreads) keys[i] = i < p.n ? key_of(p, p.tokens[i]) : p.vocab;
  __syncthreads();
  if (blockIdx.x >= p.sum_blocks) {
    const int64_t at = unit - (int64_t)p.sum_blocks * kSumWarps;
    const int64_t v0 = at / p.fill_parts << p.fill_shift;
    uint32_t used = 0;
    for (int i = lane; i < p.n; i += 32) used |= keys[i] >= v0 && keys[i] < v0 + (1 << p.fill_shift) && keys[i] < p.vocab ? 1u << (keys[i] - v0) : 0u;
    fill_rows<GT>(p, v0, (int)(at % p.fill_parts), __reduce_or_sync(~0u, used));
    return;
  }
  const int place = (int)(unit / p.tiles), column = (int)(unit % p.tiles) * kWarpColumns;
  if (place >= p.n) return;
  const uint32_t key = keys[place];
  if (key >= p.vocab) return;
  char* const mine = few + kFewTokens * 4 + warp * F::kWarp;
  const uint32_t own = ptx::smem_u32(mine);
  uint16_t* const list = reinterpret_cast<uint16_t*>(mine + kStages * G::kBytes + Segment<GT, 1>::kBytes);
  int m = 0;   // places with this token
  for (int at = 0; at < p.n; at += 32) {
    const bool one = keys[at + lane] == key;
    const uint32_t same = __ballot_sync(~0u, one);
    if (m == 0 && same && at + __ffs(same) - 1 < place) return;   // it is not the first
    if (one) list[m + __popc(same & ((1u << lane) - 1))] = (uint16_t)(at + lane);
    m += __popc(same);
  }
  __syncwarp();
  uint64_t sum[1][H] = {};
  typename G::Lone lone;
  const auto row_of = [&](int i) { return p.dy + (int64_t)list[i] * p.dy_stride; };
  const auto fetch = [&](int i, uint32_t to) {
    lone.settle();
    if (i < m) G::fetch(to, row_of(i), column, p.dim, lone);
    copy_async_commit();
  };
#pragma unroll 1
  for (int k = 0; k < kStages - 1; ++k) fetch(k, own + k * G::kBytes);
  uint32_t here = own, before = own + (kStages - 1) * G::kBytes;
#pragma unroll 1
  for (int i = 0; i < m; ++i) {
    lone.settle();
    copy_async_wait_but<kStages - 2>();
    __syncwarp();
    fetch(i + kStages - 1, before);
    uint64_t x[H];
    G::read(here, row_of(i), column, p.dim, 0, x);
#pragma unroll
    for (int e = 0; e < H; ++e) sum[0][e] = add2f(sum[0][e], x[e]);
    before = here;
    here = here == own + (kStages - 1) * G::kBytes ? own : here + G::kBytes;
  }
  write_row<GT, 1, ALIGNED>(p, key, own + kStages * G::kBytes, column, sum);
}

// ---- host side -----------------------------------------------------------------------------------------------------
struct EmbedGradPlan {
  int chunk, chunks, runs, tiles;   // runs: of 256 columns that a warp adds up
  size_t list, used, parts, bytes;   // list: of one list of n; offsets of the others
};
static int part_stride(int64_t dim) { return (int)((dim + kLaneColumns - 1) / kLaneColumns * kLaneColumns); }
static EmbedGradPlan embed_grad_plan(int64_t n, int64_t vocab, int64_t dim) {
  EmbedGradPlan g;
  g.runs = dim > kWarpColumns ? 2 : 1;
  g.tiles = (int)((dim + g.runs * kWarpColumns - 1) / (g.runs * kWarpColumns));
  // About 32 warps an SM, chunks of 16 to 256 (their parts are written and read again: 16 bytes a column for two).
  int64_t chunk = n * g.tiles / (kSms * 32) + 1;
  chunk = chunk < 16 ? 16 : chunk > 256 ? 256 : chunk;
  g.chunk = (int)chunk;
  g.chunks = (int)((n + chunk - 1) / chunk);
  g.list = align_up((uint64_t)n * 8, 256);
  g.used = 2 * g.list;
  g.parts = g.used + align_up((uint64_t)(vocab + 31) / 32 * 4, 256);
  g.bytes = g.parts + (uint64_t)g.chunks * 2 * part_stride(dim) * 4;
  return g;
}

template <int BITS>
static int launch_sort(const SortParams& p, cudaStream_t st) {
  constexpr auto kernel = sort_tokens_kernel<BITS>;
  constexpr int bytes = (kSortWarps + kSortBlocks + 1) * 4 << BITS;
  IRIS_CHECK(allow_shared<kernel>(bytes, true));
  return launch_rows(kernel, p, (unsigned)p.split, p.split, kSortThreads, bytes, st);
}
template <int DT, int GT, int I, bool ALIGNED>
static int launch_sum(const EmbedGradParams& p, unsigned fill_blocks, cudaStream_t st) {
  constexpr auto kernel = embed_sum_kernel<DT, GT, I, ALIGNED>;
  constexpr int bytes = kSumWarps * sum_bytes<DT, GT, I>();
  IRIS_CHECK(allow_shared<kernel>(bytes));
  return launch_rows(kernel, p, p.sum_blocks + fill_blocks, 1, kSumThreads, bytes, st);
}
template <int DT, int GT, bool ALIGNED>
static int launch_few(const EmbedGradParams& p, unsigned fill_blocks, cudaStream_t st) {
  constexpr auto kernel = embed_few_kernel<DT, GT, ALIGNED>;
  IRIS_CHECK(allow_shared<kernel>(Few<DT, GT, ALIGNED>::kBytes));
  return launch_rows(kernel, p, p.sum_blocks + fill_blocks, 1, kSumThreads, Few<DT, GT, ALIGNED>::kBytes, st);
}
template <int DT, int GT>
static int launch_embed_grad(const EmbedGradParams& p, const EmbedGradPlan& g, unsigned fill_blocks, cudaStream_t st) {
  const bool few = p.n <= kFewTokens, aligned = p.dim * Columns<DT>::ES % 16 == 0 && p.dim * Columns<GT>::ES % 16 == 0 && p.aligned && p.dy_stride % 16 == 0 && p.shard_stride % 16 == 0;
  if (few) return aligned ? launch_few<DT, GT, true>(p, fill_blocks, st) : launch_few<DT, GT, false>(p, fill_blocks, st);
  if (g.runs == 1) IRIS_CHECK(aligned ? launch_sum<DT, GT, 1, true>(p, fill_blocks, st) : launch_sum<DT, GT, 1, false>(p, fill_blocks, st));
  else IRIS_CHECK(aligned ? launch_sum<DT, GT, 2, true>(p, fill_blocks, st) : launch_sum<DT, GT, 2, false>(p, fill_blocks, st));
  if (p.chunks < 2) return IRIS_OK;
  const int64_t blocks = (int64_t)((p.chunks + kJoinWarps - 1) / kJoinWarps) * ((p.dim + kWarpColumns - 1) / kWarpColumns);
  return launch_rows(embed_join_kernel<GT>, p, (unsigned)blocks, 1, kJoinWarps * 32, 0, st);
}

static int check_table(const char* fn, int dtype, int world, int64_t vocab, int64_t dim, int64_t n) {
  if (dtype != IRIS_F16 && dtype != IRIS_BF16 && dtype != IRIS_F32) return fail(IRIS_ERR_ARG, "%s: unknown dtype %d", fn, dtype);
  if (world < 1 || world > IRIS_MAX_WORLD) return fail(IRIS_ERR_ARG, "%s: world=%d not in [1, %d]", fn, world, IRIS_MAX_WORLD);
  if (vocab < 0 || dim < 0 || n < 0) return fail(IRIS_ERR_ARG, "%s: vocab=%lld, dim=%lld, n=%lld", fn, (long long)vocab, (long long)dim, (long long)n);
  if (vocab > kMaxVocab || dim > kMaxDim || n > kMaxTokens) return fail(IRIS_ERR_UNSUPPORTED, "%s: at most 2^30 tokens, 2^30 rows of 2^24 columns", fn);
  if (vocab % world) return fail(IRIS_ERR_ARG, "%s: vocab=%lld is not a multiple of world=%d", fn, (long long)vocab, world);
  return IRIS_OK;
}
static int check_finite(const char* fn, const char* what, float x) {
  if (!std::isfinite(x)) return fail(IRIS_ERR_ARG, "%s: %s has to be finite", fn, what);
  return IRIS_OK;
}

}  // namespace rows
}  // namespace iris

using namespace iris;
using namespace iris::rows;

extern "C" int iris_embed_tokens(const iris_embed_args* a, void* stream) {
  const char* fn = "iris_embed_tokens";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  IRIS_CHECK(check_table(fn, a->dtype, a->world, a->vocab, a->dim, a->n));
  IRIS_CHECK(check_finite(fn, "scale", a->scale));
  const int64_t es = (int64_t)elem_size(a->dtype), per = a->vocab / a->world;
  int64_t ss = a->shard_stride, os = a->out_stride;
  EmbedParams p{};
  for (int r = 0; r < a->world; ++r) {
    ss = a->shard_stride;
    IRIS_CHECK(check_matrix(fn, "shard", a->shards[r] ? a->shards[r] : reinterpret_cast<const void*>(es), a->dtype, per, a->dim, &ss));
    p.shard[r] = static_cast<const char*>(a->shards[r]);
  }
  IRIS_CHECK(check_matrix(fn, "out", a->out, a->dtype, a->n, a->dim, &os));
  if (a->n == 0 || a->dim == 0) return IRIS_OK;
  IRIS_CHECK(check_aligned(fn, "tokens", a->tokens, 8, true));
  p.shard_stride = ss * es;
  p.out_stride = os * es;
  p.tokens = a->tokens;
  p.out = static_cast<char*>(a->out);
  p.n = a->n;
  p.vocab = a->vocab;
  p.per = (uint32_t)(per ? per : 1);
  const bool aligned = aligned_rows(a->out, os * es);
  p.bytes = (int)(a->dim * es);
  p.scale = a->scale;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) return launch_embed<IRIS_BF16>(p, aligned, st);
  if (a->dtype == IRIS_F16) return launch_embed<IRIS_F16>(p, aligned, st);
  return launch_embed<IRIS_F32>(p, aligned, st);
}

extern "C" size_t iris_embed_workspace_bytes(int64_t n, int64_t vocab, int64_t dim) {
  if (n < 0 || vocab < 0 || dim < 0 || n > kMaxTokens || vocab > kMaxVocab || dim > kMaxDim) return 0;
  return embed_grad_plan(n, vocab, dim).bytes;
}

extern "C" int iris_embed_tokens_backward(const iris_embed_grad_args* a, void* stream) {
  const char* fn = "iris_embed_tokens_backward";
  if (!a) return fail(IRIS_ERR_ARG, "%s: args is NULL", fn);
  IRIS_CHECK(check_table(fn, a->dtype, a->world, a->vocab, a->dim, a->n));
  if (a->grad_dtype != IRIS_F32 && a->grad_dtype != a->dtype) return fail(IRIS_ERR_ARG, "%s: grad_dtype %d is neither fp32 nor the rows' type", fn, a->grad_dtype);
  IRIS_CHECK(check_finite(fn, "scale", a->scale));
  const int64_t es = (int64_t)elem_size(a->dtype), gs = (int64_t)elem_size(a->grad_dtype), per = a->vocab / a->world;
  int64_t ss = a->shard_stride, ds = a->grad_out_stride;
  IRIS_CHECK(check_matrix(fn, "grad_out", a->grad_out, a->dtype, a->n, a->dim, &ds));
  EmbedGradParams p{};
  uint32_t present = 0;
  for (int r = 0; r < a->world; ++r) {
    ss = a->shard_stride;
    IRIS_CHECK(check_matrix(fn, "grad_shard", a->grad_shards[r] ? a->grad_shards[r] : reinterpret_cast<const void*>(gs), a->grad_dtype, per, a->dim, &ss));
    p.shard[r] = static_cast<char*>(a->grad_shards[r]);
    present |= (uint32_t)(a->grad_shards[r] != nullptr) << r;
  }
  if (a->vocab == 0 || a->dim == 0 || !present || (a->n == 0 && a->accumulate)) return IRIS_OK;
  const EmbedGradPlan g = embed_grad_plan(a->n, a->vocab, a->dim);
  IRIS_CHECK(check_aligned(fn, "tokens", a->tokens, 8, a->n > 0));
  IRIS_CHECK(check_aligned(fn, "workspace", a->workspace, 16, true));
  if (a->workspace_bytes < g.bytes) return fail(IRIS_ERR_ARG, "%s: workspace has %zu bytes, the call needs %zu", fn, a->workspace_bytes, g.bytes);
  const bool few = a->n <= kFewTokens;
  const int fill_parts = (int)((a->dim * gs + kFillBytes - 1) / kFillBytes);
  int fill_shift = 0;
  while (fill_shift < 5 && (a->dim * gs << (fill_shift + 1)) <= kFillBytes) ++fill_shift;
  const int tiles = few ? (int)((a->dim + kWarpColumns - 1) / kWarpColumns) : g.tiles;
  const int64_t units = few ? a->n * tiles : (int64_t)g.chunks * g.tiles, sum_blocks = (units + kSumWarps - 1) / kSumWarps;
  const int64_t fill_blocks = a->accumulate ? 0 : (((a->vocab + (1 << fill_shift) - 1) >> fill_shift) * fill_parts + kSumWarps - 1) / kSumWarps;
  if (sum_blocks + fill_blocks > INT32_MAX || units > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 blocks", fn);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* const ws = static_cast<char*>(a->workspace);
  p.dim = (int)a->dim;
  p.part_stride = part_stride(a->dim);
  p.fill_parts = fill_parts;
  p.fill_shift = fill_shift;
  p.tiles = tiles;
  p.sum_blocks = (unsigned)sum_blocks;
  p.n = (int)a->n;
  p.chunk = g.chunk;
  p.chunks = g.chunks;
  p.vocab = (uint32_t)a->vocab;
  p.per = (uint32_t)per;
  p.present = present == (1u << a->world) - 1 ? ~0u : present;
  p.tokens = a->tokens;
  p.scale = a->scale;
  p.accumulate = a->accumulate;
  p.dy = static_cast<const char*>(a->grad_out);
  p.dy_stride = ds * es;
  p.shard_stride = ss * gs;
  p.aligned = reinterpret_cast<uintptr_t>(a->grad_out) % 16 == 0;
  for (int r = 0; r < a->world; ++r) p.aligned &= reinterpret_cast<uintptr_t>(a->grad_shards[r]) % 16 == 0;
  if (!few) {
    SortParams s{};
    s.tokens = a->tokens;
    s.n = p.n;
    s.vocab = p.vocab;
    s.per = p.per;
    s.present = p.present;
    for (int i = 0; i < 2; ++i) s.lists[i] = reinterpret_cast<uint2*>(ws + i * g.list);
    s.used = a->accumulate ? nullptr : reinterpret_cast<uint32_t*>(ws + g.used);
    int bits = 1;
    while (a->vocab >> bits) ++bits;   // vocab itself is a key
    s.passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
    bits = (bits + s.passes - 1) / s.passes;
    s.split = p.n > kSortItems * kSortThreads ? kSortBlocks : 1;
    IRIS_CHECK(bits <= 6 ? launch_sort<6>(s, st) : bits == 7 ? launch_sort<7>(s, st) : bits == 8 ? launch_sort<8>(s, st) : bits == 9 ? launch_sort<9>(s, st) : launch_sort<10>(s, st));
    p.list = s.lists[s.passes & 1 ^ 1];
    p.used = s.used;
    p.parts = reinterpret_cast<float*>(ws + g.parts);
  }
  const bool wide = a->grad_dtype == IRIS_F32;
  const unsigned f = (unsigned)fill_blocks;
  if (a->dtype == IRIS_BF16) return wide ? launch_embed_grad<IRIS_BF16, IRIS_F32>(p, g, f, st) : launch_embed_grad<IRIS_BF16, IRIS_BF16>(p, g, f, st);
  if (a->dtype == IRIS_F16) return wide ? launch_embed_grad<IRIS_F16, IRIS_F32>(p, g, f, st) : launch_embed_grad<IRIS_F16, IRIS_F16>(p, g, f, st);
  return launch_embed_grad<IRIS_F32, IRIS_F32>(p, g, f, st);
}
