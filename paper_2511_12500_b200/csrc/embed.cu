// Embedding lookup in a table cut by rows into shards (the head's B shards are one), and its gradient by sorted tokens.
//
//   y_i = scale E[t_i];   dE[v] = scale * sum over i with t_i = v of dy_i
#include "any_rows.cuh"

namespace iris {
namespace rows {

// ---- lookup --------------------------------------------------------------------------------------------------------
constexpr int kEmbedThreads = 256;

struct EmbedParams {
  const char* shard[IRIS_MAX_WORLD];
  int64_t shard_stride, out_stride;   // bytes
  const int64_t* tokens;
  char* out;
  int64_t n, vocab;
  uint32_t per, each;                 // rows of a shard; 16-byte granules that a row of the output may touch
  int bytes;                          // of a row
  float scale;
};

// A thread moves granules of the output, counted over all rows, so that blocks are full whatever a row's length is.
template <int DT, int U>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const __grid_constant__ EmbedParams p) {
  using E = Elem<DT>;
  constexpr int ES = sizeof(typename E::T), T = kEmbedThreads;
  const int64_t f0 = (int64_t)blockIdx.x * (T * U), row0 = f0 / p.each;
  const uint32_t in_row = (uint32_t)(f0 - row0 * p.each);
  ptx::let_next_begin();
  ptx::begin_after_previous();
  char* to[U];
  const char* from[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t at = in_row + u * T + threadIdx.x, down = at / p.each;
    const int64_t i = row0 + down;
    to[u] = nullptr;
    from[u] = nullptr;
    if (i >= p.n) continue;
    const int64_t t = p.tokens[i];
    to[u] = p.out + i * p.out_stride;
    if (t >= 0 && t < p.vocab) {
      const uint32_t r = (uint32_t)t / p.per;
      if (p.shard[r]) from[u] = p.shard[r] + (int64_t)((uint32_t)t - r * p.per) * p.shard_stride;
    }
  }
  uint4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t at = in_row + u * T + threadIdx.x;
    const int byte = (int)(at - at / p.each * p.each) * 16 - (int)phase(to[u]);
    v[u] = from[u] ? load_piece<ES>(from[u] + byte, from[u], from[u] + p.bytes) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!to[u]) continue;
    const uint32_t at = in_row + u * T + threadIdx.x;
    const int byte = (int)(at - at / p.each * p.each) * 16 - (int)phase(to[u]);
    if (p.scale != 1.f) {
      float x[E::VE];
      E::unpack(v[u], x);
#pragma unroll
      for (int e = 0; e < E::VE; ++e) x[e] *= p.scale;
      v[u] = E::pack(x);
    }
    store16<ES>(to[u] + byte, to[u], to[u] + p.bytes, v[u]);
  }
}

template <int DT>
static int launch_embed(const EmbedParams& p, cudaStream_t st) {
  const int64_t granules = p.n * p.each;
  const bool few = granules < (int64_t)kSms * 8 * kEmbedThreads * 4;
  const int64_t blocks = (granules + kEmbedThreads * (few ? 1 : 4) - 1) / (kEmbedThreads * (few ? 1 : 4));
  if (blocks > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "iris_embed_tokens: more than 2^31 - 1 blocks");
  return launch_rows(few ? embed_kernel<DT, 1> : embed_kernel<DT, 4>, p, (unsigned)blocks, 1, kEmbedThreads, 0, st);
}

// ---- gradient: sorted tokens ---------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kSortBlocks = 8;      // one cluster
constexpr int kSortMaxBits = 10;    // of a digit

struct SortParams {
  const int64_t* tokens;
  int n;
  uint32_t vocab, per, present;     // present: a bit for each shard that is there
  uint32_t *keys[2], *places[2];    // of pass 0, 2, .. and 1, 3, ..
  uint32_t* used;                   // a bit for each row of the table that a token names; nullptr: not wanted
  int passes, bits, split;
};

__device__ __forceinline__ uint32_t sort_key(const SortParams& p, int64_t t) {   // vocab: no token, behind all others
  if (t < 0 || t >= p.vocab) return p.vocab;
  return p.present >> ((uint32_t)t / p.per) & 1 ? (uint32_t)t : p.vocab;
}

// Tokens in rising order, equal ones in the order of their places, so that the sums over them have one order: a radix sort by one cluster.
// Each warp has a run of the places and counts its digits; a digit's places follow from the counts of all warps before; then the warps
// place their runs, 32 at a time.  Buffers lie in global memory (L2); what one block writes and another reads is ordered by the cluster's barrier.
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ uint32_t count[];   // [kSortWarps, digits]; totals [split, digits]; base [digits]
  __shared__ uint32_t of_warp[kSortWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, digits = 1 << p.bits;
  const int rank = p.split > 1 ? (int)ptx::cluster_ctarank() : 0;
  uint32_t* const mine = count + warp * digits;
  uint32_t* const totals = count + kSortWarps * digits;
  uint32_t* const base = totals + p.split * digits;
  const int each = (int)(((int64_t)p.n + p.split * kSortWarps * 32 - 1) / (p.split * kSortWarps * 32)) * 32;
  const int64_t b64 = (int64_t)(rank * kSortWarps + warp) * each;
  const int begin = (int)(b64 < p.n ? b64 : p.n), end = (int)(b64 + each < p.n ? b64 + each : p.n);
  ptx::let_next_begin();
  if (p.split > 1) ptx::cluster_sync();
  ptx::begin_after_previous();
  if (p.used)
    for (uint32_t i = rank * kSortThreads + tid; i < (p.vocab + 31) / 32; i += p.split * kSortThreads) p.used[i] = 0;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits;
    const uint32_t *const keys = p.keys[pass & 1 ^ 1], *const places = p.places[pass & 1 ^ 1];
    uint32_t *const to_keys = p.keys[pass & 1], *const to_places = p.places[pass & 1];
    const auto key_at = [&](int i) { return pass ? __ldcg(keys + i) : sort_key(p, p.tokens[i]); };
    for (int i = tid; i < kSortWarps * digits; i += kSortThreads) count[i] = 0;
    __syncthreads();
    for (int i = begin + lane; i - lane < end; i += 32) {
      const uint32_t d = i < end ? key_at(i) >> shift & (digits - 1) : ~0u;
      const uint32_t same = __match_any_sync(~0u, d);
      if (i < end && (same & ((1u << lane) - 1)) == 0) mine[d] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    if (tid < digits) {
      uint32_t sum = 0;
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = count[w * digits + tid];
        count[w * digits + tid] = sum;
        sum += c;
      }
      for (int s = 0; s < p.split; ++s)
        if (p.split > 1) ptx::st_shared_cluster_u32(ptx::mapa(ptx::smem_u32(totals + rank * digits + tid), s), sum);
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
    for (int i = begin + lane; i - lane < end; i += 32) {
      const uint32_t key = i < end ? key_at(i) : 0, d = i < end ? key >> shift & (digits - 1) : ~0u;
      const uint32_t same = __match_any_sync(~0u, d), lower = same & ((1u << lane) - 1);
      uint32_t at = 0;
      if (i < end) {
        at = base[d] + mine[d] + __popc(lower);
        to_keys[at] = key;
        to_places[at] = pass ? __ldcg(places + i) : (uint32_t)i;
      }
      __syncwarp();
      if (i < end && lower == 0) mine[d] += __popc(same);
      __syncwarp();
    }
    if (p.split > 1) ptx::cluster_sync();
    else __syncthreads();
  }
  if (!p.used) return;
  const uint32_t* const keys = p.keys[p.passes & 1 ^ 1];
  for (int i = begin + lane; i < end; i += 32) {
    const uint32_t key = __ldcg(keys + i);
    if (key < p.vocab && (i == 0 || __ldcg(keys + i - 1) != key)) atomicOr(p.used + (key >> 5), 1u << (key & 31));
  }
}

// ---- gradient: sums ------------------------------------------------------------------------------------------------
constexpr int kSumThreads = 256, kSumWarps = kSumThreads / 32;
constexpr int kFillBytes = 2048;    // of a row that a warp clears at a time

struct EmbedGradParams {
  const char* dy;
  int64_t dy_stride;                // bytes
  char* shard[IRIS_MAX_WORLD];
  int64_t shard_stride;             // bytes
  const uint32_t *keys, *places, *used;
  float* parts;                     // [chunks, 2, dim]: sums of the run at a chunk's start and of the one at its end, where they go on beyond it
  int n, chunk, chunks, dim, tiles, fill_parts;   // chunk: sorted places of a chunk
  uint32_t vocab, per;
  unsigned sum_blocks;
  float scale;
  int accumulate, aligned;
};

template <int GT>
__device__ __forceinline__ char* table_row(const EmbedGradParams& p, uint32_t v) {
  const uint32_t r = v / p.per;
  return p.shard[r] ? p.shard[r] + (int64_t)(v - r * p.per) * p.shard_stride : nullptr;
}
// All threads of a warp: their columns of row v, from column `begin` on; `at`: shared memory of the warp's, Segment<GT, 1>::kBytes.
template <int GT>
__device__ __forceinline__ void write_row(const EmbedGradParams& p, uint32_t v, uint32_t at, int begin, const float (&sum)[kLaneColumns]) {
  using C = Columns<GT>;
  char* const row = table_row<GT>(p, v);
  float x[kLaneColumns];
#pragma unroll
  for (int e = 0; e < kLaneColumns; ++e) x[e] = sum[e] * p.scale;
  uint4 w[C::N];
  if (p.accumulate) {
    float old[kLaneColumns];
    C::load(row, begin + (threadIdx.x & 31) * kLaneColumns, p.dim, old);
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) x[e] += old[e];
  }
  C::pack(x, w);
  __syncwarp();
  Segment<GT, 1>::write(at, row, begin, p.dim, w);
}

// Zeros in the rows that no token names: a warp has 32 rows and kFillBytes of each.
template <int GT>
__device__ __forceinline__ void fill_rows(const EmbedGradParams& p, int64_t unit) {
  constexpr int ES = Columns<GT>::ES;
  const uint32_t word = (uint32_t)(unit / p.fill_parts);
  const int part = (int)(unit % p.fill_parts), lane = threadIdx.x & 31;
  if (word >= (p.vocab + 31) / 32) return;
  const uint32_t used = p.used[word];
  for (int b = 0; b < 32; ++b) {
    const uint32_t v = word * 32 + b;
    if (v >= p.vocab) return;
    if (used >> b & 1) continue;
    char* const row = table_row<GT>(p, v);
    if (!row) continue;
    char* const lo = row + (int64_t)part * kFillBytes;
    char* const hi = row + min((int64_t)p.dim * ES, (int64_t)(part + 1) * kFillBytes);
    for (char* at = lo - phase(lo) + lane * 16; at < hi; at += 32 * 16) store16<ES>(at, lo, hi, make_uint4(0, 0, 0, 0));
  }
}

// A warp adds up a chunk of the sorted places over 256 columns.  A run of equal tokens that lies inside a chunk is finished here; one that goes on
// in other chunks leaves its sums in `parts`, for embed_join_kernel.
//
// The rows are on their way to shared memory kSumStages ahead.
template <int DT>
constexpr int sum_stages() { return DT == IRIS_F32 ? 8 : 12; }   // 8 KB or 6 KB a warp
template <int DT, int GT>
constexpr int sum_bytes() { return sum_stages<DT>() * Segment<DT, 1>::kBytes + Segment<GT, 1>::kBytes; }   // of a warp

template <int DT, int GT>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const __grid_constant__ EmbedGradParams p) {
  using G = Segment<DT, 1>;
  constexpr int kStages = sum_stages<DT>();
  extern __shared__ __align__(16) char ring[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  if (blockIdx.x >= p.sum_blocks) {
    fill_rows<GT>(p, (int64_t)(blockIdx.x - p.sum_blocks) * kSumWarps + warp);
    return;
  }
  const int64_t unit = (int64_t)blockIdx.x * kSumWarps + warp;
  const int c = (int)(unit / p.tiles), column = (int)(unit % p.tiles) * kWarpColumns, first = column + lane * kLaneColumns;
  if (c >= p.chunks) return;
  const uint32_t own = ptx::smem_u32(ring) + warp * sum_bytes<DT, GT>(), out = own + kStages * G::kBytes;
  const int begin = c * p.chunk, end = min(p.n, begin + p.chunk);
  // The places and tokens of 32 entries are held by the threads, and the next 32 places, as copies begin ahead.
  const auto key_of = [&](int i) { return i < end ? p.keys[i] : p.vocab; };
  const auto place_of = [&](int i) { return i < end ? p.places[i] : 0u; };
  uint32_t now = p.keys[begin];
  if (now >= p.vocab) return;
  bool goes_on = begin > 0 && p.keys[begin - 1] == now;   // the run came from the chunk before
  uint32_t key = key_of(begin + lane), place = place_of(begin + lane), next_place = place_of(begin + 32 + lane);
  uint64_t sum[kLaneColumns / 2] = {};
  typename G::Lone lone;
  const auto row_of = [&](uint32_t i) { return p.dy + (int64_t)i * p.dy_stride; };
  const auto fetch = [&](int i, int base, int stage) {   // base: of `place`
    lone.settle();
    if (i < end) {
      const uint32_t at = __shfl_sync(~0u, i - base < 32 ? place : next_place, (i - base) & 31);
      G::fetch(own + stage * G::kBytes, row_of(at), column, p.dim, lone);
    }
    copy_async_commit();
  };
  const auto finish = [&](bool more) {   // more: the run goes on in the next chunk
    float s[kLaneColumns];
#pragma unroll
    for (int e = 0; e < kLaneColumns / 2; ++e) {
      const float2 f = unpair(sum[e]);
      s[2 * e] = f.x;
      s[2 * e + 1] = f.y;
    }
    if (!goes_on && !more) {
      write_row<GT>(p, now, out, column, s);
    } else {
      float* const to = p.parts + ((int64_t)2 * c + !goes_on) * p.dim;
#pragma unroll
      for (int e = 0; e < kLaneColumns; ++e)
        if (first + e < p.dim) to[first + e] = s[e];
    }
  };
#pragma unroll 1
  for (int k = 0; k < kStages - 1; ++k) fetch(begin + k, begin, k);
  int base = begin, stage = 0;
#pragma unroll 1
  for (int i = begin; i < end; ++i) {
    if (i - base == 32) {
      base = i;
      place = next_place;
      key = key_of(base + lane);
      next_place = place_of(base + 32 + lane);
    }
    const uint32_t k = __shfl_sync(~0u, key, i - base), at = __shfl_sync(~0u, place, i - base);
    if (k != now) {
      finish(false);
      if (k >= p.vocab) break;
      now = k;
      goes_on = false;
#pragma unroll
      for (int e = 0; e < kLaneColumns / 2; ++e) sum[e] = 0;
    }
    lone.settle();
    copy_async_wait_but<kStages - 2>();
    __syncwarp();
    fetch(i + kStages - 1, base, stage == 0 ? kStages - 1 : stage - 1);
    uint64_t x[kLaneColumns / 2];
    G::read(own + stage * G::kBytes, row_of(at), column, p.dim, 0, x);
#pragma unroll
    for (int e = 0; e < kLaneColumns / 2; ++e) sum[e] = add2f(sum[e], x[e]);
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (i + 1 == end) finish(end < p.n && p.keys[end] == now);
  }
  copy_async_wait();   // a block does not end while copies are under way
}

// Runs that go over several chunks: the sums of their parts, by the block of the chunk where a run begins; its warps take the parts in turn.
template <int GT>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(const __grid_constant__ EmbedGradParams p) {
  __shared__ float sums[kSumWarps][kWarpColumns];
  __shared__ __align__(16) char out[Segment<GT, 1>::kBytes];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ptx::let_next_begin();
  ptx::begin_after_previous();
  const int c = (int)(blockIdx.x / p.tiles), first = (int)(blockIdx.x % p.tiles) * kWarpColumns + lane * kLaneColumns;
  const int begin = c * p.chunk, end = min(p.n, begin + p.chunk);
  if (end >= p.n) return;
  const uint32_t key = p.keys[end - 1];
  if (key >= p.vocab || p.keys[end] != key || (begin > 0 && p.keys[begin - 1] == key)) return;
  int last = c + 1;   // the chunks c + 1 .. last - 1 begin with the run
  for (;;) {
    const int i = last + lane;
    const uint32_t there = __ballot_sync(~0u, i < p.chunks && p.keys[(int64_t)i * p.chunk < p.n ? i * p.chunk : 0] == key);
    last += __popc(there);   // of consecutive chunks, as the keys are sorted
    if (there != ~0u) break;
  }
  float sum[kLaneColumns] = {};
  for (int i = c + warp; i < last; i += kSumWarps) {
    const float* const from = p.parts + ((int64_t)2 * i + (i == c)) * p.dim;
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) sum[e] += first + e < p.dim ? from[first + e] : 0.f;
  }
#pragma unroll
  for (int e = 0; e < kLaneColumns; ++e) sums[warp][lane * kLaneColumns + e] = sum[e];
  __syncthreads();
  if (warp) return;
  for (int w = 1; w < min(kSumWarps, last - c); ++w)
#pragma unroll
    for (int e = 0; e < kLaneColumns; ++e) sum[e] += sums[w][lane * kLaneColumns + e];
  write_row<GT>(p, key, ptx::smem_u32(out), first - lane * kLaneColumns, sum);
}

// ---- host side -----------------------------------------------------------------------------------------------------
struct EmbedGradPlan {
  int chunk, chunks, tiles;
  size_t list, used, parts, bytes;   // list: of one list of n; offsets of the others
};
static EmbedGradPlan embed_grad_plan(int64_t n, int64_t vocab, int64_t dim) {
  EmbedGradPlan g;
  g.tiles = (int)((dim + kWarpColumns - 1) / kWarpColumns);
  // About 32 warps an SM, chunks of 16 to 256 (their parts are written and read again: 16 bytes a column for two).
  int64_t chunk = n * g.tiles / (kSms * 32) + 1;
  chunk = chunk < 16 ? 16 : chunk > 256 ? 256 : chunk;
  g.chunk = (int)chunk;
  g.chunks = (int)((n + chunk - 1) / chunk);
  g.list = align_up((uint64_t)n * 4, 256);
  g.used = 4 * g.list;
  g.parts = g.used + align_up((uint64_t)(vocab + 31) / 32 * 4, 256);
  g.bytes = g.parts + (uint64_t)g.chunks * 2 * dim * 4;
  return g;
}

template <int DT, int GT>
static int launch_embed_grad(const EmbedGradParams& p, unsigned fill_blocks, cudaStream_t st) {
  constexpr auto kernel = embed_sum_kernel<DT, GT>;
  constexpr int bytes = kSumWarps * sum_bytes<DT, GT>();
  IRIS_CHECK(allow_shared<kernel>(bytes));
  IRIS_CHECK(launch_rows(kernel, p, p.sum_blocks + fill_blocks, 1, kSumThreads, bytes, st));
  if (p.chunks < 2) return IRIS_OK;
  return launch_rows(embed_join_kernel<GT>, p, (unsigned)((int64_t)p.chunks * p.tiles), 1, kSumThreads, 0, st);
}

static int check_table(const char* fn, int dtype, int world, int64_t vocab, int64_t dim, int64_t n) {
  if (dtype != IRIS_F16 && dtype != IRIS_BF16 && dtype != IRIS_F32) return fail(IRIS_ERR_ARG, "%s: unknown dtype %d", fn, dtype);
  if (world < 1 || world > IRIS_MAX_WORLD) return fail(IRIS_ERR_ARG, "%s: world=%d not in [1, %d]", fn, world, IRIS_MAX_WORLD);
  if (vocab < 0 || dim < 0 || n < 0) return fail(IRIS_ERR_ARG, "%s: vocab=%lld, dim=%lld, n=%lld", fn, (long long)vocab, (long long)dim, (long long)n);
  if (vocab > kMaxVocab || dim > kMaxDim || n > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "%s: at most 2^31 - 1 tokens, 2^30 rows of 2^24 columns", fn);
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
  p.each = (uint32_t)part_granules(a->out, os, a->dim, a->dtype, 1);
  p.bytes = (int)(a->dim * es);
  p.scale = a->scale;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a->dtype == IRIS_BF16) return launch_embed<IRIS_BF16>(p, st);
  if (a->dtype == IRIS_F16) return launch_embed<IRIS_F16>(p, st);
  return launch_embed<IRIS_F32>(p, st);
}

extern "C" size_t iris_embed_workspace_bytes(int64_t n, int64_t vocab, int64_t dim) {
  if (n < 0 || vocab < 0 || dim < 0 || n > INT32_MAX || vocab > kMaxVocab || dim > kMaxDim) return 0;
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
  p.dim = (int)a->dim;
  p.fill_parts = (int)((a->dim * gs + kFillBytes - 1) / kFillBytes);
  const int64_t sum_blocks = ((int64_t)g.chunks * g.tiles + kSumWarps - 1) / kSumWarps;
  const int64_t fill_blocks = a->accumulate ? 0 : ((a->vocab + 31) / 32 * p.fill_parts + kSumWarps - 1) / kSumWarps;
  if (sum_blocks + fill_blocks > INT32_MAX || (int64_t)g.chunks * g.tiles > INT32_MAX) return fail(IRIS_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 blocks", fn);
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  char* const ws = static_cast<char*>(a->workspace);
  SortParams s{};
  s.tokens = a->tokens;
  s.n = (int)a->n;
  s.vocab = (uint32_t)a->vocab;
  s.per = (uint32_t)per;
  s.present = present;
  for (int i = 0; i < 2; ++i) {
    s.keys[i] = reinterpret_cast<uint32_t*>(ws + i * g.list);
    s.places[i] = reinterpret_cast<uint32_t*>(ws + (2 + i) * g.list);
  }
  s.used = a->accumulate ? nullptr : reinterpret_cast<uint32_t*>(ws + g.used);
  int bits = 1;
  while (a->vocab >> bits) ++bits;   // vocab itself is a key
  s.passes = (bits + kSortMaxBits - 1) / kSortMaxBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  s.split = a->n > 4 * kSortThreads ? kSortBlocks : 1;
  const size_t shared = (size_t)(kSortWarps + s.split + 1) * 4 << s.bits;
  IRIS_CHECK(allow_shared<sort_tokens_kernel>((kSortWarps + kSortBlocks + 1) * 4 << kSortMaxBits));
  IRIS_CHECK(launch_rows(sort_tokens_kernel, s, (unsigned)s.split, s.split, kSortThreads, shared, st));

  p.dy = static_cast<const char*>(a->grad_out);
  p.dy_stride = ds * es;
  p.shard_stride = ss * gs;
  p.keys = s.keys[s.passes & 1 ^ 1];
  p.places = s.places[s.passes & 1 ^ 1];
  p.used = s.used;
  p.parts = reinterpret_cast<float*>(ws + g.parts);
  p.n = (int)a->n;
  p.chunk = g.chunk;
  p.chunks = g.chunks;
  p.tiles = g.tiles;
  p.vocab = (uint32_t)a->vocab;
  p.per = (uint32_t)per;
  p.sum_blocks = (unsigned)sum_blocks;
  p.scale = a->scale;
  p.accumulate = a->accumulate;
  const bool wide = a->grad_dtype == IRIS_F32;
  const unsigned f = (unsigned)fill_blocks;
  if (a->dtype == IRIS_BF16) return wide ? launch_embed_grad<IRIS_BF16, IRIS_F32>(p, f, st) : launch_embed_grad<IRIS_BF16, IRIS_BF16>(p, f, st);
  if (a->dtype == IRIS_F16) return wide ? launch_embed_grad<IRIS_F16, IRIS_F32>(p, f, st) : launch_embed_grad<IRIS_F16, IRIS_F16>(p, f, st);
  return launch_embed_grad<IRIS_F32, IRIS_F32>(p, f, st);
}
