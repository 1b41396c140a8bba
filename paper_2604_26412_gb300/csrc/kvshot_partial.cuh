// kvshot_partial.cuh -- what the entry points that draft over a part of a long cache have in common: the cache's view,
// its checks, and operand fragments of mma.sync read straight from rows in global memory.
#pragma once

#include <cudaTypedefs.h>

#include "kvshot_attn_common.cuh"

namespace kvshot {
namespace partial {
namespace {  // internal linkage: every translation unit gets its own copy

constexpr int kMaxGroup = 32;  // q heads of a KV head

// A bf16 cache: paged (page_table) or contiguous (one page of l_cap tokens per cache).
struct CacheView {
  const int32_t *page_table, *seq_lens;
  int32_t* err;
  int C, hkv, P, max_pages, num_pages, len_bound;
};

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Checks of the descriptor that all of them make: heads and nodes as kvshot_draft_attn has them (valid, too, in a descriptor that
// gives none of them but hq = hkv), then the cache's layout.
inline kvshot_status check_partial(const kvshot_attn_desc* d, bool paged) {
  if (kvshot_status st = check_common(d)) return st;
  const int64_t kRows = int64_t{1} << 31;  // rows of K, of tables and of q are 32-bit numbers
  if (paged) {
    const int P = d->page_size;  // groups of 8 keys, and boxes of up to 64, lie in one page
    if (P < 8 || P > 256 || !(64 % P == 0 || P % 64 == 0)) return KVSHOT_ERR_UNSUPPORTED;
    if (d->max_pages_per_seq < 1 || d->num_pages < 1) return KVSHOT_ERR_SHAPE;
    if (static_cast<int64_t>(d->num_pages) * d->hkv * P >= kRows - 1 ||
        static_cast<int64_t>(d->num_caches) * d->max_pages_per_seq >= kRows - 1)
      return KVSHOT_ERR_UNSUPPORTED;
  } else {
    if (d->l_cap < 1) return KVSHOT_ERR_SHAPE;
    if (static_cast<int64_t>(d->num_caches) * d->hkv * d->l_cap >= kRows - 1) return KVSHOT_ERR_UNSUPPORTED;
  }
  if (d->flags & (KVSHOT_TARGET_FP8 | KVSHOT_FORCE_CC | KVSHOT_FORCE_MMA | KVSHOT_FORCE_TC)) return KVSHOT_ERR_UNSUPPORTED;
  // (Places of tokens stay 32-bit numbers where they are rounded up.)
  const int64_t room = paged ? static_cast<int64_t>(d->max_pages_per_seq) * d->page_size : d->l_cap;
  if ((room < d->max_seq_len ? room : d->max_seq_len) > kRows - 4096) return KVSHOT_ERR_UNSUPPORTED;
  if (d->hq / d->hkv > kMaxGroup || d->hkv > 65535) return KVSHOT_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(d->num_caches) * d->n_query * d->hq >= kRows) return KVSHOT_ERR_UNSUPPORTED;
  return KVSHOT_OK;
}

// Tensor map of a bf16 tensor of `rank` dimensions, 128-byte swizzle; strides (of dimensions 1 ...) in bytes.  False if the
// encoder is not there or refuses.
inline bool encode_bf16(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                        const cuuint32_t* box) {
  static const PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f) : nullptr;
  }();
  const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
  return encode != nullptr && encoded([&] {
           return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, ones,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
         });
}
// Rows of 128 dims landed in groups of 8 (kGroupBytes): {64 dims, 8 rows, 2 halves, rows / 8}, `groups` of them to a box ...
inline bool map_groups(CUtensorMap* map, const void* base, uint64_t rows, uint32_t groups) {
  const cuuint64_t dims[4] = {64, 8, 2, rows / 8}, strides[3] = {256, 128, 2048};
  const cuuint32_t box[4] = {64, 8, 2, groups};
  return rows % 8 == 0 && encode_bf16(map, base, 4, dims, strides, box);
}
// ... or one, from any row: {64 dims, rows, 2 halves}.
inline bool map_any_8(CUtensorMap* map, const void* base, uint64_t rows) {
  const cuuint64_t dims[3] = {64, rows, 2}, strides[2] = {256, 128};
  const cuuint32_t box[3] = {64, 8, 2};
  return encode_bf16(map, base, 3, dims, strides, box);
}
// Half the dims of `heads` heads of `nodes` rows of q [C, Nq, hq, 128].
inline bool map_q(CUtensorMap* map, const void* q, int C, int Nq, int hq, uint32_t heads, uint32_t nodes) {
  const cuuint64_t row = kHeadDim * 2;
  const cuuint64_t dims[4] = {kHeadDim, static_cast<cuuint64_t>(hq), static_cast<cuuint64_t>(Nq), static_cast<cuuint64_t>(C)};
  const cuuint64_t strides[3] = {row, row * hq, row * hq * Nq};
  const cuuint32_t box[4] = {64, heads, nodes, 1};
  return encode_bf16(map, q, 4, dims, strides, box);
}

inline CacheView cache_view(const kvshot_attn_desc* d, const int32_t* page_table, const int32_t* seq_lens) {
  CacheView v;
  const bool paged = page_table != nullptr;
  v.page_table = page_table;
  v.seq_lens = seq_lens;
  v.err = d->err_flag;
  v.C = d->num_caches;
  v.hkv = d->hkv;
  v.P = paged ? d->page_size : d->l_cap;
  v.max_pages = paged ? d->max_pages_per_seq : 1;
  v.num_pages = paged ? d->num_pages : d->num_caches;
  const int64_t room = static_cast<int64_t>(v.max_pages) * v.P;
  v.len_bound = static_cast<int>(room < d->max_seq_len ? room : d->max_seq_len);
  return v;
}

inline float score_scale(const kvshot_attn_desc* d) {
  return d->scale != 0.f ? d->scale : 0.08838834764831845f;  // 1 / sqrt(128)
}

__device__ __forceinline__ int clamped_len(const CacheView& v, int c) {
  const int L = v.seq_lens[c];
  if (L >= 0 && L <= v.len_bound) return L;
  dev::set_error(v.err, KVSHOT_ERR_DEVICE_BOUNDS);
  return L < 0 ? 0 : v.len_bound;
}

// Pool page of page p of cache c, or -1 (recorded) if its id is outside the pool.
__device__ __forceinline__ int page_id(const CacheView& v, int c, int p) {
  if (v.page_table == nullptr) return c;
  const int id = v.page_table[static_cast<size_t>(c) * v.max_pages + p];
  if (static_cast<unsigned>(id) < static_cast<unsigned>(v.num_pages)) return id;
  dev::set_error(v.err, KVSHOT_ERR_DEVICE_BOUNDS);
  return -1;
}

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n));
  return n;
}
__device__ __forceinline__ void cluster_sync_all() {
  __syncwarp();  // (.aligned: the whole warp at once, which loops and branches of single lanes before it do not promise)
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float remote_float(uint32_t addr, uint32_t rank) {
  float x;
  asm volatile("{\n\t.reg .u32 ra;\n\tmapa.shared::cluster.u32 ra, %1, %2;\n\tld.shared::cluster.f32 %0, [ra];\n\t}"
               : "=f"(x) : "r"(addr), "r"(rank) : "memory");
  return x;
}

__device__ __forceinline__ float4 remote_float4(uint32_t addr, uint32_t rank) {
  float4 x;
  asm volatile("{\n\t.reg .u32 ra;\n\tmapa.shared::cluster.u32 ra, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [ra];\n\t}"
               : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr), "r"(rank) : "memory");
  return x;
}

__device__ __forceinline__ uint32_t word(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

// Dot products of rows (keys, or bounds) with rows of q run as mma.sync m16n8k16 with the rows as M.  A sum over the dims
// does not depend on their order, so lane (g, t) = (lane / 4, lane % 4) takes, of rows g and g + 8, the 16-byte pieces
// 4 j + t: a load of the warp covers whole 64-byte segments of 8 rows, and piece j holds the A (and from a row of q alike
// the B) operands of the k-steps 2 j and 2 j + 1.
__device__ __forceinline__ void mma_piece(float (&d)[4], const uint4& a, const uint4& a8, const uint4& b) {
  const uint32_t lo[4] = {a.x, a8.x, a.y, a8.y}, hi[4] = {a.z, a8.z, a.w, a8.w};
  dev::mma_bf16_16816(d, lo, b.x, b.y);
  dev::mma_bf16_16816(d, hi, b.z, b.w);
}

// A wait that looks a few times before it takes the time (reading the clock takes long enough to be late).
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, int32_t* err, uint64_t limit) {
  if (limit >= dev::kPollBelowNs) {
    for (int i = 0; i < 32; ++i)
      if (dev::mbar_try_wait(bar, parity)) return true;
  }
  return dev::mbar_wait(bar, parity, err, limit);
}

// 32 bytes of a row by one load: half the requests of 16-byte loads for the same bytes.
struct Row32 {
  uint4 lo, hi;
};
__device__ __forceinline__ Row32 load32(const uint4* p) {
  Row32 r;
  asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r.lo.x), "=r"(r.lo.y), "=r"(r.lo.z), "=r"(r.lo.w), "=r"(r.hi.x), "=r"(r.hi.y), "=r"(r.hi.z), "=r"(r.hi.w)
               : "l"(p));
  return r;
}

// Rows of q staged in shared memory, 16 pieces and 64 bytes of padding each: 8 rows' pieces 4 j .. 4 j + 3 are in different
// banks.
constexpr int kQRowBytes = 256 + 64;

}  // namespace
}  // namespace partial
}  // namespace kvshot
