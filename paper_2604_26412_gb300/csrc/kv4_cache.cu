// kv4_cache.cu -- the 4-bit target cache beside its attention: room for new tokens (block tables and slot maps),
// quantisation of K and V into slots, and the values of slots read back.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdlib>

#include "kvshot_attn_common.cuh"
#include "kvshot_kv4.cuh"

namespace kvshot {
namespace {

using namespace dev;
using namespace kv4;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// ------------------------------------------------------------ room for new tokens

constexpr int kPlanThreads = 1024;  // one cache each
static_assert(kPlanThreads >= kMaxCaches, "a thread per cache");
constexpr int kFillThreads = 256;
constexpr int kExtendCluster = 8;
constexpr int kClusterItems = 16 * kExtendCluster * kPlanThreads;

struct ExtendParams {
  const int32_t *seq_lens, *new_tokens, *page_table, *free_pages, *free_count;
  int32_t *seq_lens_out, *page_table_out, *free_count_out, *token_start, *slots, *token_cache, *positions;
  int32_t* err;
  int C, P, max_pages, num_pages, num_free, max_tokens;
  Div by_page, by_entry;  // page size, table entries of a cache
};

// What follows from the lengths and the counts: first new token, length before, first new page of each cache.
struct ExtendPlan {
  int start[kMaxCaches + 1], len[kMaxCaches], base[kMaxCaches];
};

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int P) { return (tokens + P - 1) / P; }
__device__ __forceinline__ int pages_of(const ExtendParams& p, int tokens) {
  const int q = p.by_page(tokens);
  return q + (q * p.P < tokens ? 1 : 0);
}

// Sums over the threads up to and including this one, of two numbers; `warp_sums` [2][32] is scratch.  *total_a, *total_b:
// over the block.
__device__ __forceinline__ void block_scan(int64_t& a, int64_t& b, int64_t* warp_sums, int64_t* total_a, int64_t* total_b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) {
      a += x;
      b += y;
    }
  }
  __syncthreads();
  if (lane == 31) {
    warp_sums[warp] = a;
    warp_sums[32 + warp] = b;
  }
  __syncthreads();
  // Each warp sums the warps' numbers: lane w those up to warp w.
  int64_t sa = lane < warps ? warp_sums[lane] : 0, sb = lane < warps ? warp_sums[32 + lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, sa, o), y = __shfl_up_sync(0xffffffffu, sb, o);
    if (lane >= o) {
      sa += x;
      sb += y;
    }
  }
  *total_a = __shfl_sync(0xffffffffu, sa, 31);
  *total_b = __shfl_sync(0xffffffffu, sb, 31);
  const int64_t below_a = __shfl_sync(0xffffffffu, sa, max(warp - 1, 0)), below_b = __shfl_sync(0xffffffffu, sb, max(warp - 1, 0));
  a += warp > 0 ? below_a : 0;
  b += warp > 0 ? below_b : 0;
}

// Whether the call can be met at all (the same answer in all threads), and what this thread's cache gets: tokens before
// and with its own, length, pages before it.  kPlanThreads threads.
struct CachePlan {
  int len, count, start, base;
  int free_count, need, total;  // before the call; of all caches
};
__device__ __forceinline__ bool extend_plan(const ExtendParams& p, int64_t* scratch, CachePlan* out) {
  const int c = threadIdx.x;
  const int L = c < p.C ? p.seq_lens[c] : 0, n = c < p.C ? p.new_tokens[c] : 0;
  const int F = *p.free_count;
  bool ok = L >= 0 && n >= 0 && F >= 0 && F <= p.num_free;
  const int64_t used = ok ? pages_of(L, p.P) : 0, after = ok ? pages_of(static_cast<int64_t>(L) + n, p.P) : 0;
  ok = ok && after <= p.max_pages;
  if (ok && c < p.C && n > 0 && L % p.P != 0) {  // the page that the first new token joins
    const int pid = p.page_table[static_cast<size_t>(c) * p.max_pages + used - 1];
    ok = pid >= 0 && pid < p.num_pages;
  }
  int64_t pages = after - used, tokens = n, need, total;
  block_scan(pages, tokens, scratch, &need, &total);
  ok = ok && need <= F && total <= p.max_tokens;
  ok = __syncthreads_and(ok);
  if (ok) {
    // The pages that the call takes: eight loads in flight to a thread (one at a time took 20 us for 65k pages).
    int worst = 0;
#pragma unroll 1
    for (int64_t i0 = F - need + threadIdx.x; i0 < F; i0 += 8 * kPlanThreads) {
      int pid[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) pid[i] = i0 + i * kPlanThreads < F ? p.free_pages[i0 + i * kPlanThreads] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) worst |= static_cast<unsigned>(pid[i]) >= static_cast<unsigned>(p.num_pages);
    }
    ok = worst == 0;
  }
  ok = __syncthreads_and(ok);
  *out = CachePlan{L, n, static_cast<int>(tokens) - n, static_cast<int>(pages - (after - used)), F, static_cast<int>(need),
                   static_cast<int>(total)};
  return ok;
}

// The outputs per cache and the error, of a plan.
__device__ __forceinline__ void write_plan(const ExtendParams& p, const CachePlan& w, bool ok) {
  const int c = threadIdx.x;
  if (!ok && c == 0) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
  if (c < p.C) {
    p.seq_lens_out[c] = ok ? w.len + w.count : w.len;
    p.token_start[c + 1] = ok ? w.start + w.count : 0;
  }
  if (c == 0) {
    p.token_start[0] = 0;
    *p.free_count_out = ok ? w.free_count - w.need : w.free_count;
  }
}

// The table's entries and the packed tokens' maps: this thread's, of `threads`.  free_count: before the call.
__device__ __forceinline__ void extend_fill(const ExtendParams& p, const ExtendPlan& s, int free_count, int thread, int threads) {
  const bool in_place = p.page_table == p.page_table_out;
  const int entries = p.C * p.max_pages;
#pragma unroll 4
  for (int i = thread; i < entries; i += threads) {
    const int c = p.by_entry(i), j = i - c * p.max_pages;
    const int used = pages_of(p, s.len[c]), after = pages_of(p, s.len[c] + s.start[c + 1] - s.start[c]);
    if (j >= used && j < after) p.page_table_out[i] = p.free_pages[free_count - 1 - (s.base[c] + j - used)];
    else if (!in_place) p.page_table_out[i] = p.page_table[i];
  }
  const int total = s.start[p.C];
  for (int t = thread; t < p.max_tokens; t += threads) {
    int slot = -1, cache = -1, pos = -1;
    if (t < total) {
      int lo = 0, hi = p.C - 1;  // last cache whose first token is <= t
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s.start[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
      cache = lo;
      const int L = s.len[lo];
      pos = L + t - s.start[lo];
      const int j = p.by_page(pos), used = pages_of(p, L);
      const int32_t* entry = j < used ? p.page_table + static_cast<size_t>(lo) * p.max_pages + j
                                      : p.free_pages + free_count - 1 - (s.base[lo] + j - used);
      slot = *entry * p.P + (pos - j * p.P);
    }
    if (p.slots) p.slots[t] = slot;
    if (p.token_cache) p.token_cache[t] = cache;
    if (p.positions) p.positions[t] = pos;
  }
}

// All of a small call in one cluster.  Every CTA makes the plan for itself; the lengths are written once all have read them.
__global__ void __cluster_dims__(kExtendCluster, 1, 1) __launch_bounds__(kPlanThreads)
    extend_cluster_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ int64_t scratch[64];
  __shared__ ExtendPlan s;
  CachePlan w;
  const bool ok = extend_plan(p, scratch, &w);
  const int c = threadIdx.x;
  if (c < p.C) {
    s.start[c] = ok ? w.start : 0;
    s.len[c] = w.len;
    s.base[c] = w.base;
  }
  if (c == 0) s.start[p.C] = ok ? w.total : 0;
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (blockIdx.x == 0) write_plan(p, w, ok);
  extend_fill(p, s, w.free_count, blockIdx.x * kPlanThreads + threadIdx.x, kExtendCluster * kPlanThreads);
}

// A large call: the plan in one CTA, its outputs to the fill kernel's CTAs.
__global__ void __launch_bounds__(kPlanThreads) extend_plan_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ int64_t scratch[64];
  allow_dependent_launch();
  CachePlan w;
  const bool ok = extend_plan(p, scratch, &w);
  write_plan(p, w, ok);
}

__global__ void __launch_bounds__(kFillThreads) extend_fill_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ int64_t scratch[64];
  __shared__ ExtendPlan s;
  wait_for_prerequisite_grid();
  int64_t base = 0;
  for (int c0 = 0; c0 < p.C; c0 += kFillThreads) {
    const int c = c0 + threadIdx.x;
    int64_t need = 0, none = 0, total, zero;
    if (c < p.C) {
      const int a = p.token_start[c], n = p.token_start[c + 1] - a, L = p.seq_lens_out[c] - n;
      s.start[c] = a;
      s.len[c] = L;
      need = pages_of(p, L + n) - pages_of(p, L);
    }
    int64_t upto = need;
    block_scan(upto, none, scratch, &total, &zero);
    if (c < p.C) s.base[c] = static_cast<int>(base + upto - need);
    base += total;
  }
  if (threadIdx.x == 0) s.start[p.C] = p.token_start[p.C];
  __syncthreads();
  extend_fill(p, s, *p.free_count_out + static_cast<int>(base), blockIdx.x * kFillThreads + threadIdx.x, gridDim.x * kFillThreads);
}

// ------------------------------------------------------------ store, load

struct RowParams {
  const uint8_t* k;  // (store: read only)
  const uint8_t* v;
  const int32_t* slots;
  uint8_t* cache;
  int32_t* err;
  int64_t k_stride, v_stride;  // bytes
  int T, hkv, P, num_slots;
  Div by_page;
  float k_unit, v_unit;        // 2^exp; store: 2^-exp
};

constexpr int kRowThreads = 256;
constexpr int kRowLanes = kHeadDim / 8;  // threads to a token's K or V of one head: 8 dims each, half a block
constexpr int kRowTokens = kRowThreads / kRowLanes;

// A thread's place: token t, dims 8 j .. 8 j + 7 of the units [u0, u0 + kUnits) (unit: K or V of a head).
struct RowPlace {
  int j, t, u0, slot;
  uint32_t code;  // byte of its codes in a group's K codes
  size_t group;   // byte of the slot's group for head 0
  size_t head;    // from a head's group to the next one's
};

template <int kUnits>
__device__ __forceinline__ RowPlace row_place(const RowParams& p) {
  RowPlace w;
  w.j = threadIdx.x % kRowLanes;
  w.t = blockIdx.x * kRowTokens + threadIdx.x / kRowLanes;
  w.u0 = blockIdx.y * kUnits;
  w.slot = w.t < p.T ? p.slots[w.t] : -1;
  if (w.slot < 0 || w.slot >= p.num_slots) {
    if (w.slot != -1) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
    w.slot = -1;
  }
  const int page = p.by_page(max(w.slot, 0)), at = max(w.slot, 0) - page * p.P, groups = p.P / kKv4Tokens;
  w.head = static_cast<size_t>(groups) * kKv4Bytes;
  w.group = (static_cast<size_t>(page) * p.hkv * groups + at / kKv4Tokens) * kKv4Bytes;
  w.code = (w.j >> 2) * kChunkStride + at % kKv4Tokens * kChunkBytes + (w.j & 3) * 4;
  return w;
}
__device__ __forceinline__ uint32_t scale_at(const RowParams& p, const RowPlace& w) {
  return kScales + w.slot % kKv4Tokens * (kHeadDim / kBlockDims) + (w.j >> 1);  // (pages are whole groups)
}

// Quantises: two threads to a block of 16 dims.  y / s rounds to e2m1, and top / 6 to e4m3, as the exact quotients do:
// the reciprocal is taken as a number of fp32 below it and the rest, so that the quotient's error is far below the gap
// between a tie and any other quotient of a bf16 number by an e4m3 one, and a quotient that is a tie comes out as that.
template <int kUnits>
__global__ void __launch_bounds__(kRowThreads) store_kernel(const __grid_constant__ RowParams p) {
  const int t = blockIdx.x * kRowTokens + threadIdx.x / kRowLanes, u0 = blockIdx.y * kUnits;
  uint4 x[kUnits];  // (loaded beside the slot, not after it)
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = u0 + i, h = u >> 1;
    x[i] = make_uint4(0u, 0u, 0u, 0u);
    if (t < p.T && u < 2 * p.hkv)
      x[i] = *reinterpret_cast<const uint4*>(((u & 1) ? p.v + t * p.v_stride : p.k + t * p.k_stride) + (h * kHeadDim + threadIdx.x % kRowLanes * 8) * 2);
  }
  const RowPlace w = row_place<kUnits>(p);
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = u0 + i;
    const uint32_t d[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    uint32_t m = 0;  // largest magnitudes, as their bits: a NaN is above infinity
#pragma unroll
    for (int k = 0; k < 4; ++k) m = __vmaxu2(m, d[k] & 0x7fff7fffu);
    m = max(m & 0xffffu, m >> 16);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const float unit = u & 1 ? p.v_unit : p.k_unit, top = __uint_as_float(m << 16) * unit;
    const bool nan = m > 0x7f80u;
    const float sixth = fmaf(top, 0x1.555554p-3f, top * 0x1.555556p-27f);
    const uint32_t scale = nan ? 0x7fu : f32_to_e4m3(fminf(fmaxf(sixth, 0x1p-9f), 448.f));
    const float s = __half2float(__ushort_as_half(static_cast<unsigned short>(e4m3x2_to_f16x2(scale) & 0xffffu)));
    // (The rest is kept above zero: infinity times it has to be infinity, and -0 times it -0.)
    const float r = __frcp_rd(s), rest = fmaxf(fmaf(-r, s, 1.f) * r, r * 0x1p-60f);
    const float r1 = r * unit, r0 = rest * unit;
    uint32_t codes = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float lo = bf16_lo(d[k]), hi = bf16_hi(d[k]);
      codes |= f32x2_to_e2m1(fmaf(lo, r1, lo * r0), fmaf(hi, r1, hi * r0)) << (8 * k);
    }
    if (w.slot < 0 || u >= 2 * p.hkv) continue;
    uint8_t* g = p.cache + w.group + (u >> 1) * w.head;
    *reinterpret_cast<uint32_t*>(g + (u & 1) * kVCodes + w.code) = nan ? 0u : codes;
    if (!(w.j & 1)) g[(u & 1) * kScaleBytes + scale_at(p, w)] = static_cast<uint8_t>(scale);
  }
}

// A thread decodes 8 dims of some K and V.
template <int kUnits>
__global__ void __launch_bounds__(kRowThreads) load_kernel(const __grid_constant__ RowParams p, uint8_t* k, uint8_t* v) {
  const RowPlace w = row_place<kUnits>(p);
  if (w.t >= p.T) return;
  uint32_t codes[kUnits], s1[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = w.u0 + i;
    codes[i] = s1[i] = 0;
    if (w.slot >= 0 && u < 2 * p.hkv) {
      const uint8_t* g = p.cache + w.group + (u >> 1) * w.head;
      codes[i] = *reinterpret_cast<const uint32_t*>(g + (u & 1) * kVCodes + w.code);
      s1[i] = g[(u & 1) * kScaleBytes + scale_at(p, w)];
    }
  }
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int u = w.u0 + i;
    if (u >= 2 * p.hkv) break;
    const uint32_t s2 = e4m3x2_to_f16x2(s1[i] | (s1[i] << 8));
    const float unit = u & 1 ? p.v_unit : p.k_unit;
    uint32_t f[4], out[4];
    e2m1x8_to_f16(codes[i], f);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint32_t x = mul_f16x2(f[n], s2);
      const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&x));
      out[n] = pack_bf16x2(y.x * unit, y.y * unit);
    }
    uint8_t* dst = ((u & 1) ? v + w.t * p.v_stride : k + w.t * p.k_stride) + ((u >> 1) * kHeadDim + w.j * 8) * 2;
    *reinterpret_cast<uint4*>(dst) = make_uint4(out[0], out[1], out[2], out[3]);
  }
}

kvshot_status check_kv4(const kvshot_kv4_desc* d, bool store, RowParams* p) {
  if (d == nullptr) return KVSHOT_ERR_NULL;
  if (d->num_tokens < 0 || d->hkv < 1 || d->num_pages < 1) return KVSHOT_ERR_SHAPE;
  if (d->head_dim != kHeadDim) return KVSHOT_ERR_UNSUPPORTED;
  if (d->page_size < 1) return KVSHOT_ERR_SHAPE;
  if (d->page_size % kKv4Tokens != 0) return KVSHOT_ERR_UNSUPPORTED;
  if (std::abs(static_cast<int64_t>(d->k_scale_exp)) > 64 || std::abs(static_cast<int64_t>(d->v_scale_exp)) > 64)
    return KVSHOT_ERR_SHAPE;
  if (static_cast<double>(d->num_pages) * d->hkv * d->page_size >= INT_MAX || d->hkv > 16384)
    return KVSHOT_ERR_UNSUPPORTED;
  const int64_t row = static_cast<int64_t>(d->hkv) * kHeadDim;
  for (const int64_t s : {d->k_stride, d->v_stride}) {
    if (s != 0 && s < row) return KVSHOT_ERR_SHAPE;
    if (s % 8 != 0) return KVSHOT_ERR_ALIGN;
    if (s > INT64_MAX / 2 / std::max(1, d->num_tokens)) return KVSHOT_ERR_SHAPE;
  }
  p->k_stride = 2 * (d->k_stride ? d->k_stride : row);
  p->v_stride = 2 * (d->v_stride ? d->v_stride : row);
  p->T = d->num_tokens;
  p->hkv = d->hkv;
  p->P = d->page_size;
  p->by_page = Div::by(d->page_size);
  p->num_slots = d->num_pages * d->page_size;
  p->k_unit = std::ldexp(1.f, store ? -d->k_scale_exp : d->k_scale_exp);
  p->v_unit = std::ldexp(1.f, store ? -d->v_scale_exp : d->v_scale_exp);
  p->err = d->err_flag;
  return KVSHOT_OK;
}

// Units (K or V of a head) to a thread: several, whose loads are in flight together, once that leaves every SM enough
// threads.
constexpr int kManyUnits = 4;
bool many_units(const RowParams& p, int sms) {
  return static_cast<int64_t>(p.T) * kRowLanes * 2 * p.hkv / kManyUnits >= static_cast<int64_t>(sms) * 2048;
}
dim3 row_grid(const RowParams& p, int units) {
  return dim3((p.T + kRowTokens - 1) / kRowTokens, (2 * p.hkv + units - 1) / units);
}

}  // namespace
}  // namespace kvshot

using namespace kvshot;

extern "C" kvshot_status kvshot_cache_extend(const kvshot_extend_desc* d, const int32_t* seq_lens,
                                             const int32_t* new_tokens, const int32_t* page_table,
                                             const int32_t* free_pages, const int32_t* free_count,
                                             int32_t* seq_lens_out, int32_t* page_table_out, int32_t* free_count_out,
                                             int32_t* token_start, int32_t* slots, int32_t* token_cache,
                                             int32_t* positions, kvshot_stream_t stream) {
  if (d == nullptr) return KVSHOT_ERR_NULL;
  if (d->num_caches < 1 || d->page_size < 1 || d->max_pages_per_seq < 1 || d->num_pages < 1 || d->num_free < 0 ||
      d->max_tokens < 0)
    return KVSHOT_ERR_SHAPE;
  // Token positions, table entries and slots are 32-bit numbers.
  if (d->num_caches > kMaxCaches || static_cast<int64_t>(d->max_pages_per_seq) * d->page_size >= INT_MAX ||
      static_cast<int64_t>(d->num_pages) * d->page_size >= INT_MAX ||
      static_cast<int64_t>(d->num_caches) * d->max_pages_per_seq >= INT_MAX / 2 || d->max_tokens >= INT_MAX / 2)
    return KVSHOT_ERR_UNSUPPORTED;
  if (!seq_lens || !new_tokens || !page_table || !free_pages || !free_count || !seq_lens_out || !page_table_out ||
      !free_count_out || !token_start)
    return KVSHOT_ERR_NULL;
  for (const void* p : {static_cast<const void*>(seq_lens), static_cast<const void*>(new_tokens),
                        static_cast<const void*>(page_table), static_cast<const void*>(free_pages),
                        static_cast<const void*>(free_count), static_cast<const void*>(seq_lens_out),
                        static_cast<const void*>(page_table_out), static_cast<const void*>(free_count_out),
                        static_cast<const void*>(token_start), static_cast<const void*>(slots),
                        static_cast<const void*>(token_cache), static_cast<const void*>(positions)})
    if (!aligned(p, 4)) return KVSHOT_ERR_ALIGN;
  ExtendParams p{seq_lens,       new_tokens,     page_table,    free_pages,  free_count,
                 seq_lens_out,   page_table_out, free_count_out, token_start, slots,
                 token_cache,    positions,      d->err_flag,   d->num_caches, d->page_size,
                 d->max_pages_per_seq, d->num_pages, d->num_free, d->max_tokens,
                 Div::by(d->page_size), Div::by(d->max_pages_per_seq)};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int most = std::max(d->max_tokens, d->num_caches * d->max_pages_per_seq);
  if (most <= kClusterItems) {
    const cudaError_t e = launch_maybe_pdl(extend_cluster_kernel, dim3(kExtendCluster), dim3(kPlanThreads), 0, false, s, p);
    return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
  }
  if (launch_maybe_pdl(extend_plan_kernel, dim3(1), dim3(kPlanThreads), 0, false, s, p) != cudaSuccess)
    return KVSHOT_ERR_CUDA;
  const int grid = std::min((most + kFillThreads - 1) / kFillThreads, 1024);
  const cudaError_t e = launch_maybe_pdl(extend_fill_kernel, dim3(grid), dim3(kFillThreads), 0, true, s, p);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}

extern "C" size_t kvshot_kv4_cache_bytes(int32_t num_pages, int32_t hkv, int32_t page_size) {
  if (num_pages < 1 || hkv < 1 || page_size < 1 || page_size % kKv4Tokens != 0) return 0;
  if (static_cast<double>(num_pages) * hkv * page_size >= INT_MAX) return 0;
  return static_cast<size_t>(num_pages) * hkv * (page_size / kKv4Tokens) * kKv4Bytes;
}

extern "C" kvshot_status kvshot_kv4_store(const kvshot_kv4_desc* d, const void* k, const void* v, const int32_t* slots,
                                          void* cache, kvshot_stream_t stream) {
  RowParams p;
  if (kvshot_status st = check_kv4(d, true, &p)) return st;
  if (p.T == 0) return KVSHOT_OK;
  if (!k || !v || !slots || !cache) return KVSHOT_ERR_NULL;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cache, 16) || !aligned(slots, 4)) return KVSHOT_ERR_ALIGN;
  p.k = static_cast<const uint8_t*>(k);
  p.v = static_cast<const uint8_t*>(v);
  p.slots = slots;
  p.cache = static_cast<uint8_t*>(cache);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e =
      many_units(p, sm_count())
          ? launch_maybe_pdl(store_kernel<kManyUnits>, row_grid(p, kManyUnits), dim3(kRowThreads), 0, false, s, p)
          : launch_maybe_pdl(store_kernel<1>, row_grid(p, 1), dim3(kRowThreads), 0, false, s, p);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}

extern "C" kvshot_status kvshot_kv4_load(const kvshot_kv4_desc* d, const void* cache, const int32_t* slots, void* k,
                                         void* v, kvshot_stream_t stream) {
  RowParams p;
  if (kvshot_status st = check_kv4(d, false, &p)) return st;
  if (p.T == 0) return KVSHOT_OK;
  if (!k || !v || !slots || !cache) return KVSHOT_ERR_NULL;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cache, 16) || !aligned(slots, 4)) return KVSHOT_ERR_ALIGN;
  p.k = p.v = nullptr;
  p.slots = slots;
  p.cache = const_cast<uint8_t*>(static_cast<const uint8_t*>(cache));  // read only
  uint8_t *kb = static_cast<uint8_t*>(k), *vb = static_cast<uint8_t*>(v);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e =
      many_units(p, sm_count())
          ? launch_maybe_pdl(load_kernel<kManyUnits>, row_grid(p, kManyUnits), dim3(kRowThreads), 0, false, s, p, kb, vb)
          : launch_maybe_pdl(load_kernel<1>, row_grid(p, 1), dim3(kRowThreads), 0, false, s, p, kb, vb);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
