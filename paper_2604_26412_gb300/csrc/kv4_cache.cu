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

// What bounds an extension: a chain of dependent loads (lengths, the pages they join, the free pages, the table) between
// two barriers, 6 us in a graph for 64 caches; its bytes would take 0.04.  So a small one is one launch, of a cluster whose
// CTAs make the plan each for itself and check the pages taken each in part (one CTA, loads one at a time: 20 us for
// 65k pages), and a large one is two, the second of many CTAs (256 prompts of up to 8191 tokens 14.8 us; in one cluster 88.
// 64 caches of 1 to 8 new tokens 8.4 us, in two launches 9.2).
constexpr int kPlanThreads = 1024;  // one cache each
static_assert(kPlanThreads >= kMaxCaches, "a thread per cache");
constexpr int kFillThreads = 256;
constexpr int kExtendCluster = 8;
constexpr int kClusterItems = 16 * kExtendCluster * kPlanThreads;  // table entries or tokens of a small extension, at most

struct ExtendParams {
  const int32_t *seq_lens, *new_tokens, *page_table, *free_pages, *free_count;
  int32_t *seq_lens_out, *page_table_out, *free_count_out, *token_start, *slots, *token_cache, *positions;
  int32_t* err;
  int C, P, max_pages, num_pages, num_free, max_tokens;
  int search;             // the largest power of two below C
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

// Sums over the threads up to and including this one, of two numbers below 2^31 each; `warp_sums` [64] is scratch.
// *total_a, *total_b: over the block.  Sums stop at 2^31 - 1, which no call's max_tokens allows (nor, with it, the pages of so
// many tokens).
__device__ __forceinline__ uint32_t sum31(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }
__device__ __forceinline__ void warp_scan(uint32_t& a, uint32_t& b, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) {
      a = sum31(a, x);
      b = sum31(b, y);
    }
  }
}
__device__ __forceinline__ void block_scan(uint32_t& a, uint32_t& b, uint32_t* warp_sums, uint32_t* total_a, uint32_t* total_b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  warp_scan(a, b, lane);
  if (lane == 31) {
    warp_sums[warp] = a;
    warp_sums[32 + warp] = b;
  }
  __syncthreads();
  // Each warp sums the warps' numbers: lane w those up to warp w.
  uint32_t sa = lane < warps ? warp_sums[lane] : 0, sb = lane < warps ? warp_sums[32 + lane] : 0;
  warp_scan(sa, sb, lane);
  *total_a = __shfl_sync(0xffffffffu, sa, 31);
  *total_b = __shfl_sync(0xffffffffu, sb, 31);
  const uint32_t below_a = __shfl_sync(0xffffffffu, sa, max(warp - 1, 0)), below_b = __shfl_sync(0xffffffffu, sb, max(warp - 1, 0));
  if (warp > 0) {
    a = sum31(a, below_a);
    b = sum31(b, below_b);
  }
}

// Whether the call can be met at all (the same answer in all threads of the cluster), and what this thread's cache gets:
// tokens before its own, pages before them.  A cluster of kExtendCluster x kPlanThreads threads; every CTA makes the plan
// for itself, but for the pages that the call takes, which are checked once.  All inputs that an output may be have been
// read when it returns.
struct CachePlan {
  int len, count, start, base;
  int free_count, need, total;  // before the call; of all caches
};
struct PlanShared {
  uint32_t sums[64];
  int ok[kExtendCluster];  // a CTA's answer to the pages it checked
};
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ bool extend_plan(const ExtendParams& p, PlanShared& s, CachePlan* out) {
  cluster_arrive();
  const int c = threadIdx.x;
  const int L = c < p.C ? p.seq_lens[c] : 0, n = c < p.C ? p.new_tokens[c] : 0;
  const int F = *p.free_count;
  bool ok = L >= 0 && n >= 0 && F >= 0 && F <= p.num_free;
  const int64_t used = ok ? pages_of(L, p.P) : 0, after = ok ? pages_of(static_cast<int64_t>(L) + n, p.P) : 0;
  ok = ok && after <= p.max_pages;
  int joined = 0;  // the page that the first new token joins (looked at after the sums, which its load need not hold up)
  if (ok && c < p.C && n > 0 && L % p.P != 0) joined = p.page_table[static_cast<size_t>(c) * p.max_pages + used - 1];
  const uint32_t own = ok ? static_cast<uint32_t>(after - used) : 0;  // (at most max_pages)
  uint32_t pages = own, tokens = ok ? n : 0, need, total;
  block_scan(pages, tokens, s.sums, &need, &total);
  ok = ok && need <= static_cast<uint32_t>(F) && total <= static_cast<uint32_t>(p.max_tokens) && joined >= 0 && joined < p.num_pages;
  ok = __syncthreads_and(ok);
  bool good = ok;
  if (ok) {  // (eight loads of a thread in flight)
    constexpr int threads = kExtendCluster * kPlanThreads;
#pragma unroll 1
    for (int64_t i0 = F - static_cast<int64_t>(need) + blockIdx.x * kPlanThreads + threadIdx.x; i0 < F; i0 += 8 * threads) {
      int pid[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) pid[i] = i0 + i * threads < F ? p.free_pages[i0 + i * threads] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) good = good && static_cast<unsigned>(pid[i]) < static_cast<unsigned>(p.num_pages);
    }
  }
  good = __syncthreads_and(good);
  cluster_wait();  // (every CTA has started)
  if (threadIdx.x < kExtendCluster)
    asm volatile("{\n\t.reg .u32 ra;\n\tmapa.shared::cluster.u32 ra, %0, %1;\n\tst.shared::cluster.s32 [ra], %2;\n\t}" ::"r"(
                     smem_addr(s.ok + blockIdx.x)),
                 "r"(threadIdx.x), "r"(static_cast<int>(good))
                 : "memory");
  cluster_arrive();
  cluster_wait();
#pragma unroll
  for (int i = 0; i < kExtendCluster; ++i) ok = ok && s.ok[i] != 0;
  *out = CachePlan{L, n, static_cast<int>(tokens - n), static_cast<int>(pages - own), F, static_cast<int>(need),
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

// The table's entries and the packed tokens' maps: this thread's, of `threads`, four at a time.  free_count: before the
// call.
__device__ __forceinline__ void extend_fill(const ExtendParams& p, const ExtendPlan& s, int free_count, int thread, int threads) {
  const bool in_place = p.page_table == p.page_table_out;
  const int entries = p.C * p.max_pages;
#pragma unroll 1
  for (int i0 = thread; i0 < entries; i0 += 4 * threads) {
    const int32_t* from[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = i0 + k * threads;
      from[k] = nullptr;
      if (i >= entries) continue;
      const int c = p.by_entry(i), j = i - c * p.max_pages, L = s.len[c];
      const int used = pages_of(p, L), after = pages_of(p, L + s.start[c + 1] - s.start[c]);
      if (j >= used && j < after) from[k] = p.free_pages + free_count - 1 - (s.base[c] + j - used);
      else if (!in_place) from[k] = p.page_table + i;
    }
    int pid[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) pid[k] = from[k] ? *from[k] : 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (from[k]) p.page_table_out[i0 + k * threads] = pid[k];
  }
  const int total = s.start[p.C];
#pragma unroll 1
  for (int t0 = thread; t0 < p.max_tokens; t0 += 4 * threads) {
    int c[4] = {0, 0, 0, 0};  // last cache whose first token is <= t
    for (int step = p.search; step > 0; step >>= 1)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c[k] + step < p.C && s.start[c[k] + step] <= t0 + k * threads) c[k] += step;
    int pos[4], page[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int t = t0 + k * threads, L = s.len[c[k]];
      pos[k] = L + t - s.start[c[k]];
      page[k] = 0;
      if (t >= total) continue;
      const int j = p.by_page(pos[k]), used = pages_of(p, L);
      page[k] = j < used ? p.page_table[static_cast<size_t>(c[k]) * p.max_pages + j]
                         : p.free_pages[free_count - 1 - (s.base[c[k]] + j - used)];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int t = t0 + k * threads;
      if (t >= p.max_tokens) break;
      const bool live = t < total;
      if (p.slots) p.slots[t] = live ? page[k] * p.P + pos[k] - p.by_page(pos[k]) * p.P : -1;
      if (p.token_cache) p.token_cache[t] = live ? c[k] : -1;
      if (p.positions) p.positions[t] = live ? pos[k] : -1;
    }
  }
}

// All of a small call in one cluster.
__global__ void __cluster_dims__(kExtendCluster, 1, 1) __launch_bounds__(kPlanThreads)
    extend_cluster_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ PlanShared shared;
  __shared__ ExtendPlan s;
  CachePlan w;
  const bool ok = extend_plan(p, shared, &w);
  const int c = threadIdx.x;
  if (c < p.C) {
    s.start[c] = ok ? w.start : 0;
    s.len[c] = w.len;
    s.base[c] = w.base;
  }
  if (c == 0) s.start[p.C] = ok ? w.total : 0;
  if (blockIdx.x == 0) write_plan(p, w, ok);
  __syncthreads();
  extend_fill(p, s, w.free_count, blockIdx.x * kPlanThreads + threadIdx.x, kExtendCluster * kPlanThreads);
}

// A large call: the plan in one cluster, its outputs to the fill kernel's CTAs.
__global__ void __cluster_dims__(kExtendCluster, 1, 1) __launch_bounds__(kPlanThreads)
    extend_plan_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ PlanShared shared;
  allow_dependent_launch();
  CachePlan w;
  const bool ok = extend_plan(p, shared, &w);
  if (blockIdx.x == 0) write_plan(p, w, ok);
}

__global__ void __launch_bounds__(kFillThreads) extend_fill_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ int sums[kFillThreads / 32];
  __shared__ ExtendPlan s;
  wait_for_prerequisite_grid();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int base = 0;  // (what the plan grants is below 2^31 pages)
  for (int c0 = 0; c0 < p.C; c0 += kFillThreads) {
    const int c = c0 + threadIdx.x;
    int need = 0;
    if (c < p.C) {
      const int a = p.token_start[c], n = p.token_start[c + 1] - a, L = p.seq_lens_out[c] - n;
      s.start[c] = a;
      s.len[c] = L;
      need = pages_of(p, L + n) - pages_of(p, L);
    }
    int upto = need;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    int below = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kFillThreads / 32; ++w) {
      below += w < warp ? sums[w] : 0;
      all += sums[w];
    }
    if (c < p.C) s.base[c] = base + below + upto - need;
    base += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) s.start[p.C] = p.token_start[p.C];
  __syncthreads();
  extend_fill(p, s, *p.free_count_out + base, blockIdx.x * kFillThreads + threadIdx.x, gridDim.x * kFillThreads);
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

// 512 bytes of K or V of a head's two tokens to a warp's load or store, 128 of their codes.  Bounded by HBM: 131009 tokens
// of 8 heads read back in 107 us (6.4 TB/s, 0.94 of the copy's rate); 32771 stored in 33 us (5.2 TB/s: the quantising, 40
// instructions to 8 numbers, is not all hidden) and read back in 27.  A small call is its launch (3 us).
constexpr int kRowThreads = 256;
constexpr int kRowLanes = kHeadDim / 8;  // threads to a token's K or V of one head: 8 dims each, half a block
constexpr int kRowTokens = kRowThreads / kRowLanes;

// A thread's place: token t, dims 8 j .. 8 j + 7 of some heads.
struct RowPlace {
  bool live;
  uint32_t code, scale;  // bytes of its codes and scale in a group (K's)
  size_t group, head;    // byte of the slot's group for head 0; from a head's group to the next one's
};

__device__ __forceinline__ RowPlace row_place(const RowParams& p, int slot, int j) {
  RowPlace w;
  w.live = slot >= 0 && slot < p.num_slots;
  if (!w.live) {
    if (slot != -1) set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
    slot = 0;
  }
  const int page = p.by_page(slot), at = slot - page * p.P, groups = p.P / kKv4Tokens, row = at % kKv4Tokens;
  w.head = static_cast<size_t>(groups) * kKv4Bytes;
  w.group = (static_cast<size_t>(page) * p.hkv * groups + at / kKv4Tokens) * kKv4Bytes;
  w.code = (j >> 2) * kChunkStride + row * kChunkBytes + (j & 3) * 4;
  w.scale = kScales + row * (kHeadDim / kBlockDims) + (j >> 1);
  return w;
}

__device__ __forceinline__ float rcp_approx(float x) {  // to an fp32 step
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\t"
      "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// Eight numbers of a block of 16 (the next lane, an odd one, has the others) to codes and the block's scale.
//
// y / s rounds to e2m1, and top / 6 to e4m3, as the exact quotients do.  Those are quotients of numbers of at most 8 bits,
// so any of them is either a tie or at least 2^-9 of itself away from one; and each is computed as y r + y rest with
// r + rest = 1 / s to some 2^-44, whose fp32 rounding gives a tie exactly.  r lies below 1 / s, so that the rest is above
// zero: it keeps the sign of a zero, and infinity infinite.
__device__ __forceinline__ uint32_t quantise(const uint4& x, float unit, uint32_t* scale) {
  const uint32_t d[4] = {x.x, x.y, x.z, x.w};
  uint32_t m = 0;  // largest magnitudes, as their bits: a NaN is above infinity
#pragma unroll
  for (int k = 0; k < 4; ++k) m = __vmaxu2(m, d[k] & 0x7fff7fffu);
  m = max(m & 0xffffu, m >> 16);
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  const float top = __uint_as_float(m << 16) * unit;
  const bool nan = m > 0x7f80u;
  const uint32_t sc = f32_to_e4m3(fmaxf(fmaf(top, 0x1.555554p-3f, top * 0x1.555556p-27f), 0x1p-9f));  // (saturates)
  const float s = __half2float(__ushort_as_half(static_cast<unsigned short>(e4m3x2_to_f16x2(sc) & 0xffffu)));
  const float r = rcp_approx(s) * (1.f - 0x1p-22f), r1 = r * unit, r0 = fmaf(-r, s, 1.f) * r1;
  uint32_t codes[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 y = make_float2(bf16_lo(d[k]), bf16_hi(d[k])), q = fma2(y, make_float2(r1, r1), mul2(y, make_float2(r0, r0)));
    codes[k] = f32x2_to_e2m1(q.x, q.y);
  }
  *scale = nan ? 0x7fu : sc;
  return nan ? 0u : __byte_perm(__byte_perm(codes[0], codes[1], 0x0040), __byte_perm(codes[2], codes[3], 0x0040), 0x5410);
}

// Five CTAs to an SM: 32771 tokens stored and read back in 61.2 us, with six 63.8, as the compiler has it (four) 64.6.
template <int kHeads>
__global__ void __launch_bounds__(kRowThreads, 5) store_kernel(const __grid_constant__ RowParams p) {
  const int j = threadIdx.x % kRowLanes, t = blockIdx.x * kRowTokens + threadIdx.x / kRowLanes, h0 = blockIdx.y * kHeads;
  const uint8_t* k = p.k + t * p.k_stride + (h0 * kHeadDim + j * 8) * 2;
  const uint8_t* v = p.v + t * p.v_stride + (h0 * kHeadDim + j * 8) * 2;
  uint4 xk[kHeads], xv[kHeads];  // (loaded beside the slot, not after it)
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    xk[i] = xv[i] = make_uint4(0u, 0u, 0u, 0u);
    if (t < p.T && h0 + i < p.hkv) {
      xk[i] = *reinterpret_cast<const uint4*>(k + i * 2 * kHeadDim);
      xv[i] = *reinterpret_cast<const uint4*>(v + i * 2 * kHeadDim);
    }
  }
  const RowPlace w = row_place(p, t < p.T ? p.slots[t] : -1, j);
  uint8_t* g = p.cache + w.group + h0 * w.head;
#pragma unroll
  for (int i = 0; i < kHeads; ++i, g += w.head) {
    uint32_t sk, sv;
    const uint32_t ck = quantise(xk[i], p.k_unit, &sk), cv = quantise(xv[i], p.v_unit, &sv);
    if (!w.live || h0 + i >= p.hkv) continue;
    *reinterpret_cast<uint32_t*>(g + w.code) = ck;
    *reinterpret_cast<uint32_t*>(g + kVCodes + w.code) = cv;
    if (j & 1) g[kScaleBytes + w.scale] = static_cast<uint8_t>(sv);
    else g[w.scale] = static_cast<uint8_t>(sk);
  }
}

// Eight codes and their scale to bf16 numbers.
__device__ __forceinline__ uint4 dequantise(uint32_t codes, uint32_t scale, float unit) {
  const uint32_t s2 = e4m3x2_to_f16x2(scale | (scale << 8));
  uint32_t f[4], out[4];
  e2m1x8_to_f16(codes, f);
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const uint32_t x = mul_f16x2(f[n], s2);
    const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&x));
    out[n] = pack_bf16x2(y.x * unit, y.y * unit);
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

template <int kHeads>
__global__ void __launch_bounds__(kRowThreads) load_kernel(const __grid_constant__ RowParams p, uint8_t* ko, uint8_t* vo) {
  const int j = threadIdx.x % kRowLanes, t = blockIdx.x * kRowTokens + threadIdx.x / kRowLanes, h0 = blockIdx.y * kHeads;
  if (t >= p.T) return;
  const RowPlace w = row_place(p, p.slots[t], j);
  const uint8_t* g = p.cache + w.group + h0 * w.head;
  uint32_t ck[kHeads], cv[kHeads], sk[kHeads], sv[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i, g += w.head) {
    ck[i] = cv[i] = sk[i] = sv[i] = 0;
    if (w.live && h0 + i < p.hkv) {
      ck[i] = *reinterpret_cast<const uint32_t*>(g + w.code);
      cv[i] = *reinterpret_cast<const uint32_t*>(g + kVCodes + w.code);
      sk[i] = g[w.scale];
      sv[i] = g[kScaleBytes + w.scale];
    }
  }
  uint8_t* k = ko + t * p.k_stride + (h0 * kHeadDim + j * 8) * 2;
  uint8_t* v = vo + t * p.v_stride + (h0 * kHeadDim + j * 8) * 2;
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (h0 + i >= p.hkv) break;
    *reinterpret_cast<uint4*>(k + i * 2 * kHeadDim) = dequantise(ck[i], sk[i], p.k_unit);
    *reinterpret_cast<uint4*>(v + i * 2 * kHeadDim) = dequantise(cv[i], sv[i], p.v_unit);
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

// Heads to a thread: four, whose loads are in flight together, once that leaves every SM enough threads (131009 tokens
// read back in 107 us, two heads 110, one 137; 2048 tokens, one head each, 4.4).
constexpr int kManyHeads = 4;
bool many_heads(const RowParams& p, int sms) {
  return static_cast<int64_t>(p.T) * kRowLanes * p.hkv / kManyHeads >= static_cast<int64_t>(sms) * 2048;
}
dim3 row_grid(const RowParams& p, int heads) { return dim3((p.T + kRowTokens - 1) / kRowTokens, (p.hkv + heads - 1) / heads); }

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
  int search = 0;
  for (int s = 1; s < d->num_caches; s *= 2) search = s;
  ExtendParams p{seq_lens,       new_tokens,     page_table,    free_pages,  free_count,
                 seq_lens_out,   page_table_out, free_count_out, token_start, slots,
                 token_cache,    positions,      d->err_flag,   d->num_caches, d->page_size,
                 d->max_pages_per_seq, d->num_pages, d->num_free, d->max_tokens,
                 search, Div::by(d->page_size), Div::by(d->max_pages_per_seq)};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int most = std::max(d->max_tokens, d->num_caches * d->max_pages_per_seq);
  if (most <= kClusterItems) {
    const cudaError_t e = launch_maybe_pdl(extend_cluster_kernel, dim3(kExtendCluster), dim3(kPlanThreads), 0, false, s, p);
    return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
  }
  if (launch_maybe_pdl(extend_plan_kernel, dim3(kExtendCluster), dim3(kPlanThreads), 0, false, s, p) != cudaSuccess)
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
      many_heads(p, sm_count())
          ? launch_maybe_pdl(store_kernel<kManyHeads>, row_grid(p, kManyHeads), dim3(kRowThreads), 0, false, s, p)
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
      many_heads(p, sm_count())
          ? launch_maybe_pdl(load_kernel<kManyHeads>, row_grid(p, kManyHeads), dim3(kRowThreads), 0, false, s, p, kb, vb)
          : launch_maybe_pdl(load_kernel<1>, row_grid(p, 1), dim3(kRowThreads), 0, false, s, p, kb, vb);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
