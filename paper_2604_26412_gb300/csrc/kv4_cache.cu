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

struct ExtendParams {
  const int32_t *seq_lens, *new_tokens, *page_table, *free_pages, *free_count;
  int32_t *seq_lens_out, *page_table_out, *free_count_out, *token_start, *slots, *token_cache, *positions;
  int32_t* err;
  int C, P, max_pages, num_pages, num_free, max_tokens;
};

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int P) { return (tokens + P - 1) / P; }

// Sum over the threads up to and including this one; `warp_sums` [32] is scratch.  *total: over the block.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* warp_sums, int64_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t t = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += t;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  int64_t below = 0, all = 0;
  for (int w = 0; w < warps; ++w) {
    below += w < warp ? warp_sums[w] : 0;
    all += warp_sums[w];
  }
  *total = all;
  return below + v;
}

// Lengths, counts and token starts, and whether the call can be met at all: everything that the fill kernel needs.
__global__ void __launch_bounds__(kPlanThreads) extend_plan_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ int64_t sums[32];
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
  int64_t need, total;
  block_scan(after - used, sums, &need);
  const int64_t end = block_scan(n, sums, &total);
  ok = ok && need <= F && total <= p.max_tokens;
  ok = __syncthreads_and(ok);
  if (ok) {
    bool good = true;
    for (int64_t i = F - need + threadIdx.x; i < F; i += blockDim.x)
      good = good && p.free_pages[i] >= 0 && p.free_pages[i] < p.num_pages;
    ok = good;
  }
  ok = __syncthreads_and(ok);
  if (!ok && threadIdx.x == 0) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
  if (c < p.C) {
    p.seq_lens_out[c] = ok ? L + n : L;
    p.token_start[c + 1] = ok ? static_cast<int32_t>(end) : 0;
  }
  if (c == 0) {
    p.token_start[0] = 0;
    *p.free_count_out = ok ? F - static_cast<int32_t>(need) : F;
  }
}

// The table's entries and the packed tokens' maps, from what the plan kernel wrote.
__global__ void __launch_bounds__(kFillThreads) extend_fill_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ int64_t sums[32];
  __shared__ int s_start[kMaxCaches + 1], s_len[kMaxCaches], s_base[kMaxCaches];
  wait_for_prerequisite_grid();
  int64_t base = 0;
  for (int c0 = 0; c0 < p.C; c0 += kFillThreads) {
    const int c = c0 + threadIdx.x;
    int64_t need = 0;
    if (c < p.C) {
      const int a = p.token_start[c], n = p.token_start[c + 1] - a, L = p.seq_lens_out[c] - n;
      s_start[c] = a;
      s_len[c] = L;
      need = pages_of(static_cast<int64_t>(L) + n, p.P) - pages_of(L, p.P);
    }
    int64_t total;
    const int64_t upto = block_scan(need, sums, &total);
    if (c < p.C) s_base[c] = static_cast<int>(base + upto - need);
    base += total;
  }
  if (threadIdx.x == 0) s_start[p.C] = p.token_start[p.C];
  __syncthreads();
  const int F = *p.free_count_out + static_cast<int>(base);  // before the call
  const int stride = gridDim.x * kFillThreads, i0 = blockIdx.x * kFillThreads + threadIdx.x;
  // Page j of cache c.
  auto page = [&](int c, int j) {
    const int used = static_cast<int>(pages_of(s_len[c], p.P));
    return j < used ? p.page_table[static_cast<size_t>(c) * p.max_pages + j] : p.free_pages[F - 1 - (s_base[c] + j - used)];
  };
  const bool in_place = p.page_table == p.page_table_out;
  const int entries = p.C * p.max_pages;
  for (int i = i0; i < entries; i += stride) {
    const int c = i / p.max_pages, j = i - c * p.max_pages;
    const int n = s_start[c + 1] - s_start[c];
    const bool fresh = j >= pages_of(s_len[c], p.P) && j < pages_of(static_cast<int64_t>(s_len[c]) + n, p.P);
    if (fresh) p.page_table_out[i] = page(c, j);
    else if (!in_place) p.page_table_out[i] = p.page_table[i];
  }
  const int total = s_start[p.C];
  for (int t = i0; t < p.max_tokens; t += stride) {
    int slot = -1, cache = -1, pos = -1;
    if (t < total) {
      int lo = 0, hi = p.C - 1;  // last cache whose first token is <= t
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_start[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
      cache = lo;
      pos = s_len[lo] + t - s_start[lo];
      const int j = pos / p.P;
      slot = page(lo, j) * p.P + (pos - j * p.P);
    }
    if (p.slots) p.slots[t] = slot;
    if (p.token_cache) p.token_cache[t] = cache;
    if (p.positions) p.positions[t] = pos;
  }
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
  float k_unit, v_unit;        // 2^exp; store: 2^-exp
};

constexpr int kRowThreads = 256;
constexpr int kRowLanes = kHeadDim / kBlockDims;  // threads to a token's K or V of one head: a block of 16 dims each

// Byte of the group of `slot` and head h, and the token's place in it.
__device__ __forceinline__ size_t group_of(const RowParams& p, int slot, int h) {
  const int page = slot / p.P, groups = p.P / kKv4Tokens;
  return ((static_cast<size_t>(page) * p.hkv + h) * groups + (slot - page * p.P) / kKv4Tokens) * kKv4Bytes;
}

__device__ __forceinline__ bool slot_valid(const RowParams& p, int slot) {
  if (slot >= 0 && slot < p.num_slots) return true;
  if (slot != -1) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
  return false;
}

// A thread quantises a block of 16 dims; blockIdx.y: K or V of a head.
__global__ void __launch_bounds__(kRowThreads) store_kernel(const __grid_constant__ RowParams p) {
  const int b = threadIdx.x % kRowLanes, t = blockIdx.x * (kRowThreads / kRowLanes) + threadIdx.x / kRowLanes;
  const int kind = blockIdx.y & 1, h = blockIdx.y >> 1;
  const int slot = t < p.T ? p.slots[t] : -1;
  const bool live = slot_valid(p, slot);
  uint32_t scale = 0;
  uint2 codes = make_uint2(0u, 0u);
  if (live) {
    const uint8_t* src = (kind ? p.v + t * p.v_stride : p.k + t * p.k_stride) + (h * kHeadDim + b * kBlockDims) * 2;
    const uint4 a = *reinterpret_cast<const uint4*>(src), c = *reinterpret_cast<const uint4*>(src + 16);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, c.x, c.y, c.z, c.w};
    const float unit = kind ? p.v_unit : p.k_unit;
    float y[16];
    uint32_t top = 0;  // largest magnitude, as its bits: a NaN is above infinity
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[2 * i] = bf16_lo(w[i]) * unit;
      y[2 * i + 1] = bf16_hi(w[i]) * unit;
      top = max(top, max(__float_as_uint(y[2 * i]) & 0x7fffffffu, __float_as_uint(y[2 * i + 1]) & 0x7fffffffu));
    }
    if (top > 0x7f800000u) {
      scale = 0x7fu;
    } else {
      scale = f32_to_e4m3(fminf(fmaxf(__fdiv_rn(__uint_as_float(top), 6.f), 0x1p-9f), 448.f));
      const float s = __half2float(__ushort_as_half(static_cast<unsigned short>(e4m3x2_to_f16x2(scale) & 0xffffu)));
      // y / s, correctly rounded (one step from y times the rounded reciprocal), so that ties stay ties.
      const float r = __frcp_rn(s), most = 8.f * s;
      float q[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = fminf(fmaxf(y[i], -most), most);
        const float q0 = x * r;
        q[i] = copysignf(fmaf(fmaf(-q0, s, x), r, q0), x);  // (the sign: of a zero)
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        codes.x |= f32x2_to_e2m1(q[2 * i], q[2 * i + 1]) << (8 * i);
        codes.y |= f32x2_to_e2m1(q[8 + 2 * i], q[9 + 2 * i]) << (8 * i);
      }
    }
  }
  // The scales of a token's eight blocks, eight lanes next to one another, in one store.
  uint32_t lo = scale << (8 * (b & 3)), hi = b < 4 ? 0u : lo;
  lo = b < 4 ? lo : 0u;
#pragma unroll
  for (int o = 1; o < kRowLanes; o <<= 1) {
    lo |= __shfl_xor_sync(0xffffffffu, lo, o);
    hi |= __shfl_xor_sync(0xffffffffu, hi, o);
  }
  if (!live) return;
  uint8_t* g = p.cache + group_of(p, slot, h);
  const int row = slot % kKv4Tokens;
  *reinterpret_cast<uint2*>(g + kind * kVCodes + (b >> 1) * kChunkStride + row * kChunkBytes + (b & 1) * 8) = codes;
  if (b == 0) *reinterpret_cast<uint2*>(g + kScales + kind * kScaleBytes + row * kRowLanes) = make_uint2(lo, hi);
}

// A thread decodes a block of 16 dims.
__global__ void __launch_bounds__(kRowThreads) load_kernel(const __grid_constant__ RowParams p, uint8_t* k, uint8_t* v) {
  const int b = threadIdx.x % kRowLanes, t = blockIdx.x * (kRowThreads / kRowLanes) + threadIdx.x / kRowLanes;
  const int kind = blockIdx.y & 1, h = blockIdx.y >> 1;
  if (t >= p.T) return;
  const int slot = p.slots[t];
  uint32_t out[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
  if (slot_valid(p, slot)) {
    const uint8_t* g = p.cache + group_of(p, slot, h);
    const int row = slot % kKv4Tokens;
    const uint2 codes =
        *reinterpret_cast<const uint2*>(g + kind * kVCodes + (b >> 1) * kChunkStride + row * kChunkBytes + (b & 1) * 8);
    const uint32_t s1 = g[kScales + kind * kScaleBytes + row * kRowLanes + b];
    const uint32_t s2 = e4m3x2_to_f16x2(s1 | (s1 << 8));
    const float unit = kind ? p.v_unit : p.k_unit;
    uint32_t f[8];
    e2m1x8_to_f16(codes.x, *reinterpret_cast<uint32_t(*)[4]>(&f[0]));
    e2m1x8_to_f16(codes.y, *reinterpret_cast<uint32_t(*)[4]>(&f[4]));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = mul_f16x2(f[i], s2);
      const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&x));
      out[i] = pack_bf16x2(y.x * unit, y.y * unit);
    }
  }
  uint8_t* dst = (kind ? v + t * p.v_stride : k + t * p.k_stride) + (h * kHeadDim + b * kBlockDims) * 2;
  *reinterpret_cast<uint4*>(dst) = make_uint4(out[0], out[1], out[2], out[3]);
  *reinterpret_cast<uint4*>(dst + 16) = make_uint4(out[4], out[5], out[6], out[7]);
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
  p->num_slots = d->num_pages * d->page_size;
  p->k_unit = std::ldexp(1.f, store ? -d->k_scale_exp : d->k_scale_exp);
  p->v_unit = std::ldexp(1.f, store ? -d->v_scale_exp : d->v_scale_exp);
  p->err = d->err_flag;
  return KVSHOT_OK;
}

dim3 row_grid(const RowParams& p) {
  constexpr int tokens = kRowThreads / kRowLanes;
  return dim3((p.T + tokens - 1) / tokens, 2 * p.hkv);
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
                 d->max_pages_per_seq, d->num_pages, d->num_free, d->max_tokens};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (launch_maybe_pdl(extend_plan_kernel, dim3(1), dim3(kPlanThreads), 0, false, s, p) != cudaSuccess)
    return KVSHOT_ERR_CUDA;
  const int most = std::max(d->max_tokens, d->num_caches * d->max_pages_per_seq);
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
  const cudaError_t e = launch_maybe_pdl(store_kernel, row_grid(p), dim3(kRowThreads), 0, false,
                                         reinterpret_cast<cudaStream_t>(stream), p);
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
  const cudaError_t e =
      launch_maybe_pdl(load_kernel, row_grid(p), dim3(kRowThreads), 0, false, reinterpret_cast<cudaStream_t>(stream), p,
                       static_cast<uint8_t*>(k), static_cast<uint8_t*>(v));
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
