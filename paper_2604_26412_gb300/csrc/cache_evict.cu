// cache_evict.cu -- eviction: the kept tokens' K, V and weights moved to the front of their cache, and the pages that are
// left over put back on the list of free pages.
#include <algorithm>
#include <climits>

#include "kvshot_partial.cuh"

namespace kvshot {
namespace {

using namespace dev;
using partial::aligned;

struct EvictParams {
  const uint8_t *k, *v;
  uint8_t *k_out, *v_out;
  const float* weights;
  float* weights_out;
  const int32_t *page_table, *page_table_out, *seq_lens, *kept, *kept_count, *free_count;
  int32_t *seq_lens_out, *free_pages, *free_count_out, *err;
  int C, hkv, P, max_pages, num_pages, max_pages_out, num_pages_out, max_kept, weights_len, weights_len_out, num_free;
  int heads_each;  // of 2 hkv (K and V), that a CTA moves into another pool
};

// Length and number of kept tokens of cache c; kept < 0: the cache stays as it is.
struct CacheKeep {
  int len, kept;
};
__device__ __forceinline__ CacheKeep cache_keep(const EvictParams& p, int c, int L, int m) {
  const int room = min(static_cast<int64_t>(p.max_pages) * p.P, static_cast<int64_t>(INT_MAX));
  bool ok = L >= 0 && L <= room;
  L = min(max(L, 0), room);
  ok = ok && m >= 0 && m <= L && m <= p.max_kept && m <= static_cast<int64_t>(p.max_pages_out) * p.P;
  if (p.weights != nullptr) ok = ok && L <= p.weights_len && m <= p.weights_len_out;
  if (!ok) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
  return CacheKeep{L, ok ? m : -1};
}

// Old place of token i, or -1 if the list is out of order or range there.
__device__ __forceinline__ int old_place(const EvictParams& p, const int32_t* kept, int i, int L) {
  const int j = kept[i];
  if (j >= i && j < L && (i == 0 || kept[i - 1] < j)) return j;
  set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
  return -1;
}

__device__ __forceinline__ int checked_page(const EvictParams& p, const int32_t* table, int row, int c, int page, int pool) {
  const int id = table[static_cast<size_t>(c) * row + page];
  if (static_cast<unsigned>(id) < static_cast<unsigned>(pool)) return id;
  set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
  return -1;
}

// A row of 256 bytes is 16 pieces of 16; a thread moves one piece of several rows.  A chunk of rows is loaded whole, then
// stored, and the next chunk's places are looked up while its bytes are on their way.
//
// Into another pool a CTA takes one chunk of several heads' K and V, whose rows' places are the same but for the head.  In
// place chunks go in ascending order: a token's new place is never behind its old one and both ascend, so a chunk's stores
// never reach what a later chunk loads, and one barrier between a chunk's loads and its stores is enough.  There a CTA takes
// all chunks, and where that leaves SMs idle only 4 or 8 of the 16 pieces, which are independent of one another.
// Bound by HBM: 4096 of 32K tokens of 16 caches into another pool 88 us (6.1 TB/s; 97 with a head's K or V to a CTA, 189 with
// places looked up by each row's loads); 512 of up to 8K tokens of 64 caches 54 us, where most CTAs end after one chunk.  In
// place, in a graph: the same 98 and 52 us; 4096 of 32K tokens of one cache 27 us (1.3 TB/s), 2048 of 8K 13 us, where each of the
// 64 CTAs goes through its chunks one after the other, one chunk's loads on their way.
constexpr int kMoveThreads = 256;
constexpr int kMoveLoads = 8;  // rows of a thread and chunk
constexpr int kHeadsEach = 4;  // heads' K or V that a CTA moves into another pool
constexpr int kRowPieces = kHeadDim * 2 / 16;
constexpr int kMoveItems = kMoveThreads * kMoveLoads;

template <bool kInPlace, int kPieces>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(EvictParams p) {
  constexpr int kRows = kMoveItems / kPieces;  // of a chunk
  __shared__ int s_src[2][kRows], s_dst[2][kRows];  // row of KV head 0 in its pool, or -1
  allow_dependent_launch();
  const int c = blockIdx.z, y = blockIdx.y, tid = threadIdx.x;
  const CacheKeep ck = cache_keep(p, c, p.seq_lens[c], p.kept_count[c]);
  const int32_t* kept = p.kept + static_cast<size_t>(c) * p.max_kept;
  if (y == static_cast<int>(gridDim.y) - 1) {  // the weights: one CTA
    if (p.weights == nullptr || blockIdx.x != 0) return;
    const float* src = p.weights + static_cast<size_t>(c) * p.weights_len;
    float* dst = p.weights_out + static_cast<size_t>(c) * p.weights_len_out;
    for (int i0 = 0; i0 < ck.kept; i0 += 8 * kMoveThreads) {
      float x[8];
      int j[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = i0 + i * kMoveThreads + tid;
        j[i] = at < ck.kept ? old_place(p, kept, at, ck.len) : -1;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (j[i] >= 0) x[i] = src[j[i]];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (j[i] >= 0) dst[i0 + i * kMoveThreads + tid] = x[i];
    }
    __syncthreads();  // (in place, what is behind the kept tokens' weights has been read)
    if (ck.kept >= 0)
      for (int i = ck.kept + tid; i < p.weights_len_out; i += kMoveThreads) dst[i] = 0.f;
    return;
  }
  const int piece = (kInPlace ? blockIdx.x * kPieces : 0) + tid % kPieces;
  auto look_up = [&](int i0, int buf) {
#pragma unroll
    for (int r = tid; r < kRows; r += kMoveThreads) {
      const int at = i0 + r, j = at < ck.kept ? old_place(p, kept, at, ck.len) : -1;
      int from = -1, to = -1;
      if (j >= 0 && !(kInPlace && j == at)) {
        const int pj = j / p.P, pa = at / p.P;
        const int a = checked_page(p, p.page_table, p.max_pages, c, pj, p.num_pages);
        const int b = checked_page(p, p.page_table_out, p.max_pages_out, c, pa, p.num_pages_out);
        if (a >= 0 && b >= 0) {
          from = a * p.hkv * p.P + (j - pj * p.P);
          to = b * p.hkv * p.P + (at - pa * p.P);
        }
      }
      s_src[buf][r] = from;
      s_dst[buf][r] = to;
    }
  };
  int i0 = kInPlace ? 0 : blockIdx.x * kRows;
  if (i0 >= ck.kept) return;
  look_up(i0, 0);
  __syncthreads();
  // One head's K or V (0 .. 2 hkv - 1) after the other; in place there is one.
  auto source = [&](int i) {
    return reinterpret_cast<const uint4*>((i & 1) != 0 ? p.v : p.k) + static_cast<size_t>((i >> 1) * p.P) * kRowPieces + piece;
  };
  auto destination = [&](int i) {
    return reinterpret_cast<uint4*>((i & 1) != 0 ? p.v_out : p.k_out) + static_cast<size_t>((i >> 1) * p.P) * kRowPieces + piece;
  };
  if (!kInPlace) {
    int from[kMoveLoads], to[kMoveLoads];
#pragma unroll
    for (int i = 0; i < kMoveLoads; ++i) {
      from[i] = s_src[0][i * (kMoveThreads / kPieces) + tid / kPieces];
      to[i] = s_dst[0][i * (kMoveThreads / kPieces) + tid / kPieces];
    }
    for (int head = y * p.heads_each; head < min(2 * p.hkv, (y + 1) * p.heads_each); ++head) {
      const uint4* src = source(head);
      uint4* dst = destination(head);
      uint4 x[kMoveLoads];
#pragma unroll
      for (int i = 0; i < kMoveLoads; ++i)
        if (from[i] >= 0) x[i] = __ldg(src + static_cast<size_t>(from[i]) * kRowPieces);
#pragma unroll
      for (int i = 0; i < kMoveLoads; ++i)
        if (from[i] >= 0) dst[static_cast<size_t>(to[i]) * kRowPieces] = x[i];
    }
    return;
  }
  const uint4* src = source(y);
  uint4* dst = destination(y);
  for (int buf = 0;; buf ^= 1) {
    uint4 x[kMoveLoads];
    int to[kMoveLoads];  // (read before the barrier: behind it these places may already be a later chunk's)
#pragma unroll
    for (int i = 0; i < kMoveLoads; ++i) {
      const int from = s_src[buf][i * (kMoveThreads / kPieces) + tid / kPieces];
      to[i] = s_dst[buf][i * (kMoveThreads / kPieces) + tid / kPieces];
      if (from >= 0) x[i] = src[static_cast<size_t>(from) * kRowPieces];
    }
    i0 += kRows;
    if (i0 < ck.kept) look_up(i0, buf ^ 1);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMoveLoads; ++i)
      if (to[i] >= 0) dst[static_cast<size_t>(to[i]) * kRowPieces] = x[i];
    if (i0 >= ck.kept) break;
  }
}

template <bool kInPlace, int kPieces>
cudaError_t launch_move(const EvictParams& p, cudaStream_t stream) {
  const int room = static_cast<int>(std::min<int64_t>(p.max_kept, static_cast<int64_t>(p.max_pages_out) * p.P));
  const int x = kInPlace ? kRowPieces / kPieces : (room + kMoveItems / kPieces - 1) / (kMoveItems / kPieces);
  const int y = kInPlace ? 2 * p.hkv : (2 * p.hkv + p.heads_each - 1) / p.heads_each;
  return launch_maybe_pdl(move_kernel<kInPlace, kPieces>, dim3(x, y + 1, p.C), dim3(kMoveThreads), 0, false, stream, p);
}

// Lengths and free pages: one CTA, a thread per cache, then a warp per cache writes its pages.  Beside the last rows' moves, which
// read neither list nor count; the lengths, which they may still read, are written when the moves have ended.
constexpr int kEndThreads = 1024;
static_assert(kEndThreads >= kMaxCaches, "a thread per cache");

__global__ void __launch_bounds__(kEndThreads) evict_end_kernel(EvictParams p) {
  __shared__ int s_first[kMaxCaches], s_gone[kMaxCaches], s_base[kMaxCaches], s_warp[32];
  const int c = threadIdx.x, lane = c & 31, warp = c >> 5;
  CacheKeep ck{0, -1};
  if (c < p.C) ck = cache_keep(p, c, p.seq_lens[c], p.kept_count[c]);
  const int used = (ck.len + p.P - 1) / p.P, first = ck.kept >= 0 ? (ck.kept + p.P - 1) / p.P : used;
  const int gone = p.free_pages != nullptr ? used - first : 0;
  int scan = gone;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += x;
  }
  if (lane == 31) s_warp[warp] = scan;
  __syncthreads();
  int base = scan - gone, total = 0;
  for (int w = 0; w < 32; ++w) {
    if (w < warp) base += s_warp[w];
    total += s_warp[w];
  }
  const int F = p.free_pages != nullptr ? *p.free_count : 0;
  s_first[c] = first;
  s_gone[c] = gone;
  s_base[c] = base;
  __syncthreads();  // (free_count has been read by all)
  if (p.free_pages != nullptr) {
    const bool room = F >= 0 && static_cast<int64_t>(F) + total <= p.num_free;
    if (c == 0) {
      if (!room) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
      *p.free_count_out = room ? F + total : F;
    }
    if (room)
      for (int i = warp; i < p.C; i += 32)
        for (int j = lane; j < s_gone[i]; j += 32) {
          const int id = p.page_table[static_cast<size_t>(i) * p.max_pages + s_first[i] + j];
          if (static_cast<unsigned>(id) >= static_cast<unsigned>(p.num_pages)) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
          p.free_pages[F + s_base[i] + j] = id;
        }
  }
  wait_for_prerequisite_grid();  // (by all: what follows this kernel follows the moves, too)
  if (c < p.C) p.seq_lens_out[c] = ck.kept >= 0 ? ck.kept : ck.len;
}

}  // namespace
}  // namespace kvshot

using namespace kvshot;

extern "C" kvshot_status kvshot_cache_evict(const kvshot_evict_desc* d, const void* k, const void* v,
                                            const int32_t* page_table, const int32_t* seq_lens, const int32_t* kept,
                                            const int32_t* kept_count, const float* weights, void* k_out, void* v_out,
                                            const int32_t* page_table_out, int32_t* seq_lens_out, float* weights_out,
                                            int32_t* free_pages, const int32_t* free_count, int32_t* free_count_out,
                                            kvshot_stream_t stream) {
  if (d == nullptr) return KVSHOT_ERR_NULL;
  if (d->num_caches < 1 || d->hkv < 1 || d->page_size < 1 || d->max_pages_per_seq < 1 || d->num_pages < 1 ||
      d->max_pages_out < 1 || d->num_pages_out < 1 || d->max_kept < 1 || d->weights_len < 0 || d->weights_len_out < 0 ||
      d->num_free < 0)
    return KVSHOT_ERR_SHAPE;
  const int64_t page_rows = static_cast<int64_t>(d->hkv) * d->page_size;
  if (d->num_caches > kMaxCaches || d->head_dim != kHeadDim || d->hkv > 16383 || page_rows >= INT_MAX ||
      d->num_pages * page_rows >= INT_MAX || d->num_pages_out * page_rows >= INT_MAX ||
      static_cast<int64_t>(d->num_caches) * d->max_pages_per_seq >= INT_MAX / 2 ||
      static_cast<int64_t>(d->num_caches) * d->max_pages_out >= INT_MAX / 2 || d->max_kept > 1 << 30 ||
      d->weights_len > 1 << 30 || d->weights_len_out > 1 << 30)
    return KVSHOT_ERR_UNSUPPORTED;
  if (!k || !v || !page_table || !seq_lens || !kept || !kept_count || !k_out || !v_out || !page_table_out || !seq_lens_out)
    return KVSHOT_ERR_NULL;
  if ((weights == nullptr) != (weights_out == nullptr)) return KVSHOT_ERR_NULL;
  const int given = (free_pages != nullptr) + (free_count != nullptr) + (free_count_out != nullptr);
  if (given != 0 && given != 3) return KVSHOT_ERR_NULL;
  for (const void* x : {k, v, static_cast<const void*>(k_out), static_cast<const void*>(v_out)})
    if (!aligned(x, 16)) return KVSHOT_ERR_ALIGN;
  for (const void* x : {static_cast<const void*>(page_table), static_cast<const void*>(seq_lens),
                        static_cast<const void*>(kept), static_cast<const void*>(kept_count),
                        static_cast<const void*>(weights), static_cast<const void*>(page_table_out),
                        static_cast<const void*>(seq_lens_out), static_cast<const void*>(weights_out),
                        static_cast<const void*>(free_pages), static_cast<const void*>(free_count),
                        static_cast<const void*>(free_count_out)})
    if (!aligned(x, 4)) return KVSHOT_ERR_ALIGN;
  // In place means K, V and the table; weights in place keep their rows.
  const bool in_place = k_out == k;
  if (in_place != (v_out == v) || (in_place && (page_table_out != page_table || d->max_pages_out != d->max_pages_per_seq ||
                                                d->num_pages_out != d->num_pages)))
    return KVSHOT_ERR_SHAPE;
  if (weights != nullptr && weights_out == weights && d->weights_len_out != d->weights_len) return KVSHOT_ERR_SHAPE;
  const EvictParams p{static_cast<const uint8_t*>(k), static_cast<const uint8_t*>(v), static_cast<uint8_t*>(k_out),
                      static_cast<uint8_t*>(v_out), weights, weights_out, page_table, page_table_out, seq_lens, kept,
                      kept_count, free_count, seq_lens_out, free_pages, free_count_out, d->err_flag, d->num_caches, d->hkv,
                      d->page_size, d->max_pages_per_seq, d->num_pages, d->max_pages_out, d->num_pages_out, d->max_kept,
                      d->weights_len, d->weights_len_out, d->num_free, kHeadsEach};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // In place: whole rows while those alone are two CTAs to an SM.
  const int64_t ctas = 2LL * d->hkv * d->num_caches, enough = 2LL * sm_count();
  const cudaError_t moved = !in_place            ? launch_move<false, 16>(p, s)
                            : ctas >= enough     ? launch_move<true, 16>(p, s)
                            : 2 * ctas >= enough ? launch_move<true, 8>(p, s)
                                                 : launch_move<true, 4>(p, s);
  if (moved != cudaSuccess) return KVSHOT_ERR_CUDA;
  const cudaError_t e = launch_maybe_pdl(evict_end_kernel, dim3(1), dim3(kEndThreads), 0, true, s, p);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
