// page_select.cu -- which pages or tokens of a cache matter: bounds of the pages' keys, scores of pages, and the best
// entries of rows of scores.
#include <algorithm>
#include <climits>

#include "kvshot_partial.cuh"
#include "kvshot_tcgen05.cuh"

namespace kvshot {
namespace {

using namespace dev;
using namespace partial;

// ------------------------------------------------------------ bounds

constexpr int kBoundsThreads = 256;

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  __nv_bfloat162 r = __hmin2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}

// A warp takes one (page, KV head): P rows of 256 bytes, two to a load.  Bound by HBM: 16 caches of 32K tokens in 166 us, 6.6
// TB/s.  After growth, by the launch and three dependent loads (length, table, keys): 64 caches of up to 8K tokens 6.1 us (3.4 in
// a graph).
__global__ void __launch_bounds__(kBoundsThreads) bounds_kernel(CacheView v, const uint4* __restrict__ k,
                                                               const int32_t* __restrict__ from, uint4* bounds) {
  const int c = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int since = from == nullptr ? 0 : from[c];
  const int L = clamped_len(v, c);
  const int p0 = max(0, since) / v.P, pages = (L + v.P - 1) / v.P;
  const int64_t units = static_cast<int64_t>(max(0, pages - p0)) * v.hkv;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kBoundsThreads / 32) + warp; u < units;
       u += static_cast<int64_t>(gridDim.x) * (kBoundsThreads / 32)) {
    const int p = p0 + static_cast<int>(u / v.hkv), h = static_cast<int>(u % v.hkv);
    const int id = page_id(v, c, p);
    if (id < 0) continue;
    const int rows = min(v.P, L - p * v.P);
    const uint4* src = k + (static_cast<size_t>(id) * v.hkv + h) * v.P * 16 + lane;
    const int own = lane >> 4;  // this half-warp's rows: own, own + 2, ...
    uint4 lo = make_uint4(0x7f807f80u, 0x7f807f80u, 0x7f807f80u, 0x7f807f80u);  // +inf
    uint4 hi = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
    for (int r = own; r < rows; r += 16) {
      uint4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + 2 * i < rows) x[i] = __ldg(src + (r - own + 2 * i) * 16);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + 2 * i < rows) {
          lo = make_uint4(min2(lo.x, x[i].x), min2(lo.y, x[i].y), min2(lo.z, x[i].z), min2(lo.w, x[i].w));
          hi = make_uint4(max2(hi.x, x[i].x), max2(hi.y, x[i].y), max2(hi.z, x[i].z), max2(hi.w, x[i].w));
        }
    }
    // The two half-warps' rows; then lanes 0 .. 15 hold the least and lanes 16 .. 31 the greatest.
    auto other = [](uint32_t x) { return __shfl_xor_sync(0xffffffffu, x, 16); };
    const uint4 lo2 = make_uint4(other(lo.x), other(lo.y), other(lo.z), other(lo.w));
    const uint4 hi2 = make_uint4(other(hi.x), other(hi.y), other(hi.z), other(hi.w));
    lo = make_uint4(min2(lo.x, lo2.x), min2(lo.y, lo2.y), min2(lo.z, lo2.z), min2(lo.w, lo2.w));
    hi = make_uint4(max2(hi.x, hi2.x), max2(hi.y, hi2.y), max2(hi.z, hi2.z), max2(hi.w, hi2.w));
    bounds[(static_cast<size_t>(id) * v.hkv + h) * 32 + lane] = own == 0 ? lo : hi;
  }
}

// ------------------------------------------------------------ scores

// max(q lo, q hi) = max(q, 0) hi + min(q, 0) lo, so a page's score is the product of [min(q, 0), max(q, 0)] with its
// bounds [lo, hi], a row of 256 elements: 16 steps of mma.sync with 16 pages as M.  The two halves of a row of q lie in shared
// memory; lane (g, t) has pieces 2 t, 2 t + 1 of every 128 bytes of rows g and g + 8 (32-byte loads of the bounds).
// Bound by the loads in flight of 16 warps an SM: 12 nodes of 4 q heads over 64 caches of up to 8K tokens 30 us.  Small calls are
// a launch and two dependent loads: one row over 8K tokens 2.4 us in a graph.
constexpr int kScoreWarps = 4;
constexpr int kScoreRows = 64;                   // rows of q in shared memory at a time
constexpr int kScoreRowBytes = 2 * 256 + 64;     // 8 rows' pieces are in different banks

struct ScoreParams {
  CacheView v;
  const uint4* q;       // rows [C, Nq, hq]
  const uint4* bounds;  // 32 pieces per (page, head): lo, hi
  float* scores;
  int hq, G, Nq;
  float scale;
};

// kLogGp: G is padded to 2^kLogGp columns (4: to 16 or 32, in log_gp).
template <int kLogGp>
__global__ void __launch_bounds__(kScoreWarps * 32) scores_kernel(ScoreParams p, int log_gp_arg) {
  extern __shared__ __align__(16) uint8_t s_q[];  // up to kScoreRows rows
  const int log_gp = kLogGp < 4 ? kLogGp : log_gp_arg, gp = 1 << log_gp;
  const int c = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const int rows = p.Nq << log_gp;
  const size_t stride = static_cast<size_t>(p.v.max_pages) * p.v.hkv;
  float* out = p.scores + (static_cast<size_t>(c) * p.Nq * p.v.hkv + h) * p.v.max_pages;
  auto stage = [&](int r0) {
    const int here = min(kScoreRows, (rows - r0 + 15) / 16 * 16);
    for (int i = threadIdx.x; i < here * 16; i += kScoreWarps * 32) {
      const int r = r0 + i / 16, n = r >> log_gp, j = r & (gp - 1);
      const bool live = n < p.Nq && j < p.G;
      const uint4 x = live ? __ldg(p.q + ((static_cast<size_t>(c) * p.Nq + n) * p.hq + h * p.G + j) * 16 + i % 16) : zero;
      // (of 128 bytes the even pieces, then the odd ones: a load of the warp has no two rows in one bank)
      uint4* row = reinterpret_cast<uint4*>(s_q + (i / 16) * kScoreRowBytes) + (i & 8) + (i & 1) * 4 + (i >> 1 & 3);
      row[0] = make_uint4(min2(x.x, 0), min2(x.y, 0), min2(x.z, 0), min2(x.w, 0));
      row[16] = make_uint4(max2(x.x, 0), max2(x.y, 0), max2(x.z, 0), max2(x.w, 0));
    }
    return here;
  };
  // (Table entries are looked up beside the length: their number is the table's, not the length's.)
  const int32_t* table = p.v.page_table + static_cast<size_t>(c) * p.v.max_pages;
  int id[2];
  auto look_up = [&](int cta0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int page = cta0 + warp * 16 + g + 8 * i;
      id[i] = page < p.v.max_pages ? __ldg(table + page) : 0;
    }
  };
  constexpr int kPages = kScoreWarps * 16;
  int cta0 = blockIdx.x * kPages;
  look_up(cta0);
  const int L = clamped_len(p.v, c);
  const int pages = (L + p.v.P - 1) / p.v.P;
  if (cta0 >= pages) return;
  const bool masked = p.G != gp;
  bool staged = false;
  for (; cta0 < pages; cta0 += gridDim.x * kPages) {
    const int page[2] = {cta0 + warp * 16 + g, cta0 + warp * 16 + g + 8};
    Row32 b[2][4];  // the 128-byte parts of the two pages' rows: lo, lo, hi, hi
    bool live[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      live[i] = page[i] < pages && static_cast<unsigned>(id[i]) < static_cast<unsigned>(p.v.num_pages);
      if (page[i] < pages && !live[i]) set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
      const uint4* src = p.bounds + (static_cast<size_t>(live[i] ? id[i] : 0) * p.v.hkv + h) * 32 + 2 * t;
#pragma unroll
      for (int j = 0; j < 4; ++j) b[i][j] = live[i] ? load32(src + 8 * j) : Row32{zero, zero};
    }
    look_up(cta0 + gridDim.x * kPages);
    float best[2] = {-INFINITY, -INFINITY};  // of a node whose columns are several tiles (gp > 8)
    for (int r0 = 0; r0 < rows; r0 += kScoreRows) {
      int here = min(kScoreRows, (rows - r0 + 15) / 16 * 16);
      if (!staged || rows > kScoreRows) {
        __syncthreads();
        here = stage(r0);
        __syncthreads();
        staged = true;
      }
      for (int pair = 0; pair < here / 16; ++pair) {
        // Two tiles of 8 columns, the products with the least and the greatest keys apart: four chains.
        float d[2][4] = {}, d2[2][4] = {};
        const uint8_t* row = s_q + (pair * 16 + g) * kScoreRowBytes + t * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint4* q = reinterpret_cast<const uint4*>(row + x * 8 * kScoreRowBytes + j * 128);
            float (&acc)[4] = j < 2 ? d[x] : d2[x];
            mma_piece(acc, b[0][j].lo, b[1][j].lo, q[0]);
            mma_piece(acc, b[0][j].hi, b[1][j].hi, q[4]);
          }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          // d: page g, columns 2 t and 2 t + 1; page g + 8, the same columns.
          const int col = r0 + pair * 16 + x * 8 + 2 * t;
          auto put = [&](int i, int n, float s) {
            if (n < p.Nq && live[i]) out[n * stride + page[i]] = s * p.scale;
          };
          float s[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) s[i] = d[x][i] + d2[x][i];
          if (kLogGp == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) put(i >> 1, col + (i & 1), s[i]);
            continue;
          }
          if (masked)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (((col + (i & 1)) & (gp - 1)) >= p.G) s[i] = -INFINITY;
          float m[2] = {fmaxf(s[0], s[1]), fmaxf(s[2], s[3])};
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (kLogGp > 1) m[i] = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], 1));
            if (kLogGp > 2) m[i] = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], 2));
          }
          if (kLogGp > 3) {
            const bool last = ((col & (gp - 1)) >> 3) == (gp >> 3) - 1;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              best[i] = fmaxf(best[i], m[i]);
              m[i] = best[i];
              if (last) best[i] = -INFINITY;
            }
            if (!last) continue;
          }
          if ((2 * t & (gp - 1)) == 0)
#pragma unroll
            for (int i = 0; i < 2; ++i) put(i, col >> log_gp, m[i]);
        }
      }
    }
  }
}

// Many rows over many pages: tcgen05.  128 pages are the M rows of a product of 256 dims, and the query rows (up to 128 of
// whole nodes) its N columns, so that a thread has a page's row of scores, finds each node's best in its own registers, and a
// warp stores 32 consecutive pages.  One persistent CTA per SM takes an equal run of the caches' tiles, KV head after KV
// head.  Pages are 512 bytes at any place of the pool: four warps copy them 16 bytes a lane, half a page (lo, hi) to a stage,
// all but two of the stages on their way.  (A tensor map's gather, four rows to an instruction, was not tried.)  The next head's
// q is loaded meanwhile.
//   warps 0..3 scores;  4..7 copies, and q's two halves;  8 MMA, and the owner of tensor memory
// 12 nodes of 4 q heads over 16 caches of 20K to 32K tokens: 28.8 us (mma.sync 36.5).  Once begun, a CTA takes a tile in 1.5 us
// (6.5 TB/s with the scores that are written); its start, q and the first tile take 7.
constexpr int kStPages = 128;
constexpr int kStCols = 128;
constexpr int kStStageBytes = kStPages * 256, kStChunkBytes = kStPages * 128;
constexpr int kStMaxStages = 5, kStMinStages = 3;
constexpr int kStSmem = 232448;  // what a CTA can have
constexpr int kStRooms = 4;  // of kStCols columns in tensor memory
constexpr int kStThreads = 9 * 32;
constexpr int kStQEach = kStCols * 16 / 128;

struct ScoreTcParams {
  ScoreParams s;
  int nodes_per_block, blocks, cols;  // blocks of whole nodes; cols: a block's columns rounded up to 16
  int stages;
  uint32_t wait_ns;
};
struct ScoreTcBarriers {
  uint64_t kfull[kStMaxStages], kempty[kStMaxStages], qfull[2], qempty[2], sfull[kStRooms], sempty[kStRooms], done;
  uint32_t tmem;
};
struct ScoreUnit {
  int c, hr, tile, pages;  // hr: KV head and block of nodes; pages: of the cache
  bool fresh;              // its q is another one's than the last unit's
};

// A CTA's run of units.
struct ScoreCursor {
  int c, hr, tile, pages;
  int64_t left;
  bool fresh;
  __device__ __forceinline__ static int pages_of(const ScoreTcParams& p, int c) {
    const int L = clamped_len(p.s.v, c);
    return (L + p.s.v.P - 1) / p.s.v.P;
  }
  __device__ __forceinline__ static int tiles(int pages) { return (pages + kStPages - 1) / kStPages; }
  __device__ __forceinline__ void init(const ScoreTcParams& p) {
    const int lane = threadIdx.x & 31, heads = p.s.v.hkv * p.blocks;
    const int own = lane < p.s.v.C ? pages_of(p, lane) : 0;  // (of up to 32 caches, looked at once)
    int64_t total = static_cast<int64_t>(tiles(own)) * heads;
    for (int i = lane + 32; i < p.s.v.C; i += 32) total += static_cast<int64_t>(tiles(pages_of(p, i))) * heads;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    const int64_t t0 = total * blockIdx.x / gridDim.x;
    left = total * (blockIdx.x + 1) / gridDim.x - t0;
    c = hr = tile = pages = 0;
    fresh = true;
    if (left == 0) return;
    int64_t before = 0;
    for (int base = 0;; base += 32) {  // (t0 is below the total)
      const int here = base == 0 ? own : base + lane < p.s.v.C ? pages_of(p, base + lane) : 0;
      const int64_t n = static_cast<int64_t>(tiles(here)) * heads;
      int64_t scan = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += x;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + scan > t0);
      if (past != 0) {
        const int at = __ffs(past) - 1;
        c = base + at;
        pages = __shfl_sync(0xffffffffu, here, at);
        const int64_t in = t0 - before - __shfl_sync(0xffffffffu, scan - n, at);
        hr = static_cast<int>(in / tiles(pages));
        tile = static_cast<int>(in % tiles(pages));
        return;
      }
      before += __shfl_sync(0xffffffffu, scan, 31);
    }
  }
  __device__ __forceinline__ bool next(const ScoreTcParams& p, ScoreUnit* out) {
    if (left == 0) return false;
    while (tile == tiles(pages)) {
      tile = 0;
      fresh = true;
      if (pages > 0 && ++hr < p.s.v.hkv * p.blocks) continue;
      hr = 0;
      pages = pages_of(p, ++c);
    }
    *out = ScoreUnit{c, hr, tile++, pages, fresh};
    fresh = false;
    --left;
    return true;
  }
};

__device__ __forceinline__ void copy_async_16(uint32_t dst, const void* src, bool live) {  // zeros if not
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void wait_ld_of(uint32_t (&v)[32]) {  // nothing computed from v moves before the wait
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                 "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                 "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                 "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}

template <int kLogGp>
__global__ void __launch_bounds__(kStThreads, 1) scores_tc_kernel(ScoreTcParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr int kGp = 1 << kLogGp;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (known to be uniform)
  const ScoreParams& s = p.s;
  const int hkv = s.v.hkv, q_chunk = p.cols * 128;  // bytes of 64 dims of the block's rows
  const int stages = p.stages;
  uint8_t* q_at = smem + stages * kStStageBytes;
  ScoreTcBarriers& bar = *reinterpret_cast<ScoreTcBarriers*>(q_at + 2 * 4 * q_chunk);
  int32_t* err = s.v.err;
  const uint64_t limit = p.wait_ns;
  if ((smem_addr(smem) & 1023u) != 0) {  // (the swizzled tiles' layout counts on it; dynamic shared memory is, alone)
    set_error(err, KVSHOT_ERR_CUDA);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(smem_addr(&bar.kfull[i]), 4);
      mbar_init(smem_addr(&bar.kempty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&bar.qfull[i]), 4);
      mbar_init(smem_addr(&bar.qempty[i]), 1);
    }
    for (int i = 0; i < kStRooms; ++i) {
      mbar_init(smem_addr(&bar.sfull[i]), 1);
      mbar_init(smem_addr(&bar.sempty[i]), 4);
    }
    mbar_init(smem_addr(&bar.done), 1);
    fence_mbar_init();
  }
  ScoreCursor cu;  // (the lengths are on their way beside the rest of the start)
  cu.init(p);
  if (warp == 8) {
    tc::tmem_alloc(smem_addr(&bar.tmem), kStRooms * kStCols);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = bar.tmem;
  ScoreUnit u;
  bool ok = true;

  if (warp == 8) {  // ---- products
    const uint32_t idesc = tc::idesc_bf16(kStPages, p.cols, false);
    int stage = 0, n = 0, group = -1;
    uint32_t phase = 0;
    while (__all_sync(0xffffffffu, ok && cu.next(p, &u))) {
      if (__any_sync(0xffffffffu, u.fresh)) {
        if (group >= 0) tc::tc_commit_elect(smem_addr(&bar.qempty[group & 1]));
        ++group;
        ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.qfull[group & 1]), (group >> 1) & 1, err, limit));
        if (!ok) break;
      }
      const int room = n % kStRooms;
      if (n >= kStRooms) ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.sempty[room]), (n / kStRooms - 1) & 1, err, limit));
      const uint32_t q = smem_addr(q_at) + (group & 1) * 4 * q_chunk;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (ok) ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.kfull[stage]), phase, err, limit));
        if (!ok) break;
        tc::tc_fence_after();
        const uint32_t k = smem_addr(smem) + stage * kStStageBytes;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
          tc::tc_mma_elect(tmem + room * kStCols, tc::smem_desc_sw128(k + (ks >> 2) * kStChunkBytes + (ks & 3) * 32, 16, 1024),
                           tc::smem_desc_sw128(q + (2 * half + (ks >> 2)) * q_chunk + (ks & 3) * 32, 16, 1024), idesc,
                           half > 0 || ks > 0);
        tc::tc_commit_elect(smem_addr(&bar.kempty[stage]));
        if (++stage == stages) {
          stage = 0;
          phase ^= 1u;
        }
      }
      if (!ok) break;
      tc::tc_commit_elect(smem_addr(&bar.sfull[room]));
      ++n;
    }
    tc::tc_commit_elect(smem_addr(&bar.done));  // every product this warp issued has completed
    mbar_wait(smem_addr(&bar.done), 0, err);
  } else if (warp >= 4) {  // ---- copies
    const int w = warp - 4, tid = threadIdx.x - 128;
    int issued = 0, arrived = 0, group = -1, first = 0;  // halves; the first of the present group
    int stage = 0, arrive_stage = 0;
    uint32_t phase = 1;  // of the kempty barriers (a stage's first use waits for none)
    auto arrive = [&](int until) {  // (those copies of this warp have landed)
      fence_proxy_async_smem();
      __syncwarp();
      for (; arrived < until; ++arrived) {
        if (lane == 0) mbar_arrive(smem_addr(&bar.kfull[arrive_stage]));
        if (++arrive_stage == stages) arrive_stage = 0;
      }
    };
    auto look_up = [&](const ScoreUnit& x) {  // this lane's page, looked at a unit later
      const int page = x.tile * kStPages + w * 32 + lane;
      return page < x.pages ? __ldg(s.v.page_table + static_cast<size_t>(x.c) * s.v.max_pages + page) : 0;
    };
    uint4 x[kStQEach];
    auto load_q = [&](const ScoreUnit& v) {
      const int h = v.hr / p.blocks, n0 = v.hr % p.blocks * p.nodes_per_block, nodes = min(p.nodes_per_block, s.Nq - n0);
      const uint4* q = s.q + ((static_cast<size_t>(v.c) * s.Nq + n0) * s.hq + h * s.G) * 16 + (tid & 15);
      // (Rows past the last one are other rows' here, and zeros in shared memory: without branches all loads are on their way.)
      auto load = [&](int e) {  // 8 rows
        const int r = e * 8 + (tid >> 4), n = min(r >> kLogGp, nodes - 1), j = min(r & (kGp - 1), s.G - 1);
        x[e] = __ldg(q + (n * s.hq + j) * 16);
      };
#pragma unroll
      for (int e = 0; e < kStQEach / 2; ++e) load(e);
      if (p.cols > kStCols / 2)
#pragma unroll
        for (int e = kStQEach / 2; e < kStQEach; ++e) load(e);
    };
    auto put_q = [&](const ScoreUnit& v) {  // of the next group
      if (arrived < first) {  // (what waits for the halves of the group before this one must not be waited for)
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        arrive(issued);
      }
      first = issued;
      ++group;
      if (group >= 2) ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.qempty[group & 1]), ((group >> 1) - 1) & 1, err, limit));
      if (!ok) return;
      uint8_t* q = q_at + (group & 1) * 4 * q_chunk + (tid >> 3 & 1) * q_chunk + (tid >> 4) * 128 + (((tid & 7) ^ (tid >> 4)) << 4);
      const int nodes = min(p.nodes_per_block, s.Nq - v.hr % p.blocks * p.nodes_per_block);
#pragma unroll
      for (int e = 0; e < kStQEach; ++e) {
        if (e * 8 >= p.cols) break;
        const int r = e * 8 + (tid >> 4);
        if (r >> kLogGp >= nodes || (r & (kGp - 1)) >= s.G) x[e] = make_uint4(0, 0, 0, 0);
        uint4* dst = reinterpret_cast<uint4*>(q + e * 1024);
        *dst = make_uint4(min2(x[e].x, 0), min2(x[e].y, 0), min2(x[e].z, 0), min2(x[e].w, 0));
        dst[2 * q_chunk / 16] = make_uint4(max2(x[e].x, 0), max2(x[e].y, 0), max2(x[e].z, 0), max2(x[e].w, 0));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_addr(&bar.qfull[group & 1]));
    };
    bool more = cu.next(p, &u);
    int next_id = more ? look_up(u) : 0;
    if (more) {
      load_q(u);
      put_q(u);
    }
    while (ok && more) {
      const ScoreUnit now = u;
      const int id = next_id;
      more = cu.next(p, &u);
      next_id = more ? look_up(u) : 0;
      const bool another = more && u.fresh;
      if (another) load_q(u);
      const bool in_pool = static_cast<unsigned>(id) < static_cast<unsigned>(s.v.num_pages);
      const bool there = now.tile * kStPages + w * 32 + lane < now.pages;
      if (there && !in_pool) set_error(err, KVSHOT_ERR_DEVICE_BOUNDS);
      const int row = there && in_pool ? id * hkv + now.hr / p.blocks : -1;
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        if (issued >= stages) ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.kempty[stage]), phase, err, limit));
        if (!ok) break;
        // Rows r = 2 i and 2 i + 1 of the warp's 32: piece 0 .. 15 of the half, at (piece & 7) ^ (r & 7) of its 128 bytes.
        const uint32_t dst = smem_addr(smem) + stage * kStStageBytes + (lane >> 3 & 1) * kStChunkBytes + w * 4096 + (lane >> 4) * 128;
        const uint4* src = s.bounds + half * 16 + (lane & 15);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int from = __shfl_sync(0xffffffffu, row, 2 * i + (lane >> 4));
          copy_async_16(dst + 256 * i + (((lane & 7) ^ (lane >> 4) ^ (2 * i & 7)) << 4), src + static_cast<size_t>(max(from, 0)) * 32,
                        from >= 0);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++stage == stages) {
          stage = 0;
          phase ^= 1u;
        }
        if (++issued - arrived > stages - 2) {  // (two stages are not on their way: one multiplied, one full)
          if (stages == 5) asm volatile("cp.async.wait_group 3;" ::: "memory");
          else if (stages == 4) asm volatile("cp.async.wait_group 2;" ::: "memory");
          else asm volatile("cp.async.wait_group 1;" ::: "memory");
          arrive(arrived + 1);
        }
      }
      if (ok && another) put_q(u);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    arrive(issued);
  } else {  // ---- scores
    int n = 0;
    while (ok && cu.next(p, &u)) {
      const int room = n % kStRooms, page = u.tile * kStPages + threadIdx.x;
      const int h = u.hr / p.blocks, n0 = u.hr % p.blocks * p.nodes_per_block, nodes = min(p.nodes_per_block, s.Nq - n0);
      const unsigned id = page < u.pages ? __ldg(s.v.page_table + static_cast<size_t>(u.c) * s.v.max_pages + page) : 0xffffffffu;
      ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.sfull[room]), (n / kStRooms) & 1, err, limit));
      if (!ok) break;
      tc::tc_fence_after();
      const uint32_t at = tmem + room * kStCols + (static_cast<uint32_t>(warp) << 21);
      const size_t stride = static_cast<size_t>(s.v.max_pages) * hkv;
      float* out = s.scores + ((static_cast<size_t>(u.c) * s.Nq + n0) * hkv + h) * s.v.max_pages + page;
      const bool live = id < static_cast<unsigned>(s.v.num_pages);
#pragma unroll
      for (int half = 0; half < kStCols / 64; ++half) {
        if (half * 64 >= p.cols) break;
        __syncwarp();
        uint32_t v[2][32];
        tc::tmem_ld32(at + half * 64, v[0]);
        tc::tmem_ld32(at + half * 64 + 32, v[1]);  // (what is behind the columns is not used)
        wait_ld_of(v[0]);
        wait_ld_of(v[1]);
        if ((half + 1) * 64 >= p.cols) {
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_addr(&bar.sempty[room]));
        }
#pragma unroll
        for (int x = 0; x < 64 / kGp; ++x) {
          float best = __uint_as_float(v[x * kGp >> 5][x * kGp & 31]);
#pragma unroll
          for (int j = 1; j < kGp; ++j)
            if (j < s.G) best = fmaxf(best, __uint_as_float(v[(x * kGp + j) >> 5][(x * kGp + j) & 31]));
          const int node = half * (64 / kGp) + x;
          if (node < nodes && live) out[node * stride] = best * s.scale;
        }
      }
      ++n;
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == 8) tc::tmem_dealloc(tmem, kStRooms * kStCols);
}

template <int kLogGp>
cudaError_t launch_scores_tc(const ScoreParams& s, int64_t most_tiles, uint32_t wait_ns, cudaStream_t stream) {
  ScoreTcParams p;
  p.s = s;
  const int most = kStCols >> kLogGp;
  p.blocks = (s.Nq + most - 1) / most;
  p.nodes_per_block = (s.Nq + p.blocks - 1) / p.blocks;
  p.cols = ((p.nodes_per_block << kLogGp) + 15) / 16 * 16;
  p.wait_ns = wait_ns;
  const int rest = kStSmem - 2 * 4 * p.cols * 128 - static_cast<int>(sizeof(ScoreTcBarriers));
  static_assert(kStSmem - 2 * 4 * kStCols * 128 - sizeof(ScoreTcBarriers) >= kStMinStages * kStStageBytes, "room for the stages");
  p.stages = std::min(kStMaxStages, rest / kStStageBytes);
  const size_t smem = p.stages * kStStageBytes + 2 * 4 * p.cols * 128 + sizeof(ScoreTcBarriers);
  // (The limit is the process's, and the same in every call: another thread's call of another size must not lower it.)
  cudaError_t e = cudaFuncSetAttribute(scores_tc_kernel<kLogGp>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStSmem);
  if (e != cudaSuccess) return e;
  const int grid = static_cast<int>(std::min<int64_t>(sm_count(), most_tiles * p.blocks));
  return launch_maybe_pdl(scores_tc_kernel<kLogGp>, dim3(grid), dim3(kStThreads), smem, false, stream, p);
}

// ------------------------------------------------------------ selection

// A radix selection: the scores as integers of the same order, the last one to be picked found digit by digit from counts of
// the digits, then one ordered pass that writes what is above it and the first of what is equal.
struct SelectParams {
  const float* scores;
  const int32_t* seq_lens;
  int32_t *picks, *counts, *err;
  int row_len, rows_per_len, tokens_per_entry, keep, first, last;
};

__device__ __forceinline__ uint32_t order_key(float f) {
  uint32_t u;
  asm("add.rn.f32 %0, %1, 0f00000000;" : "=r"(u) : "r"(__float_as_uint(f)));  // -0 is 0, and every NaN 0x7fffffff
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}

struct SelectRow {
  int n, count;  // entries; picks
};
__device__ __forceinline__ SelectRow select_row(const SelectParams& p, int row) {
  const int len = p.seq_lens[row / p.rows_per_len];
  int n = len > 0 ? (len - 1) / p.tokens_per_entry + 1 : 0;
  if (len < 0 || n > p.row_len) {
    set_error(p.err, KVSHOT_ERR_DEVICE_BOUNDS);
    n = min(n, p.row_len);
  }
  return SelectRow{n, min(n, p.keep)};
}

// One more in bin i, if i < bins.  (Without a branch: a row has a dozen of these a thread and round.)
__device__ __forceinline__ void count_in(uint32_t hist, uint32_t i, uint32_t bins) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.u32 p, %1, %2;\n\t@p red.shared.add.s32 [%0], 1;\n\t}" ::"r"(hist + 4 * i),
               "r"(i), "r"(bins)
               : "memory");
}

// The bin in which the need-th greatest entry is, from the bins' counts: each thread takes consecutive bins, the top ones
// first.  s_warp [warps of the block] is scratch.  Found by one thread, which calls found(bin, entries above it).
template <int kThreads, int kBins, typename Found>
__device__ __forceinline__ void find_bin(const int* hist, int need, int* s_warp, Found found) {
  constexpr int kPer = kBins / kThreads;
  static_assert(kPer * kThreads == kBins, "whole bins");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, top = kBins - 1 - tid * kPer;
  int h[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += h[i] = hist[top - i];
  int scan = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += x;
  }
  if (lane == 31) s_warp[warp] = scan;
  __syncthreads();
  int above = scan - sum;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w)
    if (w < warp) above += s_warp[w];
  if (above < need && above + sum >= need) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (above < need && above + h[i] >= need) found(top - i, above);
      above += h[i];
    }
  }
}

__device__ __forceinline__ void remote_add(int* at, uint32_t rank, int v) {
  asm volatile("{\n\t.reg .u32 ra;\n\tmapa.shared::cluster.u32 ra, %0, %1;\n\tred.shared::cluster.add.s32 [ra], %2;\n\t}" ::"r"(
                   smem_addr(at)),
               "r"(rank), "r"(v)
               : "memory");
}
__device__ __forceinline__ int remote_int(const int* at, uint32_t rank) {
  int v;
  asm volatile("{\n\t.reg .u32 ra;\n\tmapa.shared::cluster.u32 ra, %1, %2;\n\tld.shared::cluster.s32 %0, [ra];\n\t}"
               : "=r"(v) : "r"(smem_addr(at)), "r"(rank) : "memory");
  return v;
}

// A row is read once: a cluster of CTAs (one, for rows of up to kThreads x kSelectKeys entries) holds its keys in registers,
// every thread a run of consecutive entries, so that the picks' places follow from one scan of the threads' numbers.  Each
// CTA counts the digits of its own keys that are still in question and adds what it counted to the counts of all CTAs, which
// then each find the digit for themselves.  What bounds it: the latencies of a load, two to four rounds of counts and a
// scan, and, where there are many rows, the instructions of each key (keys that do not compete are 0, so that a key in
// question is one subtraction and one comparison).  In a graph, and as calls one after another where that is said: 4096 of 32K
// entries in 16 rows 11.8 us, calls 14.3 (89 with one CTA that reads the scores for every digit; 13.5 with eight CTAs of 4096
// entries to a row and not four of 8192).  1536 rows of 1250 to 2048 entries 11.7 us, calls 14.3; a warp to a row with its keys in registers, bit by bit, took 25.8, a set of keys in question kept as bits
// 17.1, digits of 8 and 10 bits 12.5 and 11.8, 256 threads to a row 15.2.
constexpr int kSelectKeys = 16;
constexpr int kMaxSelectCluster = 8;

template <int kThreads, int kBits, bool kCluster>
struct SelectSpace {
  static constexpr int kBins = 1 << kBits, kWarps = kThreads / 32, kPasses = (32 + kBits - 1) / kBits;
  int hist[2][kBins];
  int total[kCluster ? kPasses : 1][kCluster ? kBins : 1];  // over the cluster
  float scores[kWarps][33 * kSelectKeys];
  int warp[kWarps], sum, bin, above;
};

template <int kThreads, int kBits, bool kCluster>
__global__ void __launch_bounds__(kThreads) select_kernel(SelectParams p) {
  using Space = SelectSpace<kThreads, kBits, kCluster>;
  constexpr int kBins = Space::kBins, kWarps = Space::kWarps, kPasses = Space::kPasses;
  extern __shared__ __align__(16) uint8_t s_raw[];
  Space& sm = *reinterpret_cast<Space*>(s_raw);
  int(&s_hist)[2][kBins] = sm.hist;
  auto& s_total = sm.total;
  int(&s_warp)[kWarps] = sm.warp;
  int &s_sum = sm.sum, &s_bin = sm.bin, &s_above = sm.above;
  const int S = kCluster ? static_cast<int>(cluster_size()) : 1, rank = kCluster ? blockIdx.x % S : 0;
  const int row = blockIdx.x / S, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const SelectRow r = select_row(p, row);
  const int n = r.n;
  int32_t* picks = p.picks + static_cast<size_t>(row) * p.keep;
  if (rank == 0 && tid == 0) p.counts[row] = r.count;
  for (int i = r.count + rank * kThreads + tid; i < p.keep; i += S * kThreads) picks[i] = -1;
  if (n <= p.keep) {
    for (int i = rank * kThreads + tid; i < n; i += S * kThreads) picks[i] = i;
    return;  // (the whole cluster)
  }
  // This CTA's entries [e0, e1); this thread's: `rounds` from `first` on.
  const int chunk = (n + S - 1) / S, e0 = min(n, rank * chunk), e1 = min(n, e0 + chunk);
  const int rounds = (chunk + kThreads - 1) / kThreads, first = e0 + tid * rounds, mine = min(max(e1 - first, 0), rounds);
  // (A warp reads its threads' runs together, and hands them out through shared memory; a gap in 33 keeps the banks apart.)
  const int of_warp = min(max(e1 - (e0 + warp * 32 * rounds), 0), 32 * rounds);
  const float* s = p.scores + static_cast<size_t>(row) * p.row_len + e0 + warp * 32 * rounds;
  int need = p.keep - p.first - p.last;
  float f[kSelectKeys];
#pragma unroll
  for (int k = 0; k < kSelectKeys; ++k) f[k] = k * 32 + lane < of_warp ? __ldg(s + k * 32 + lane) : 0.f;
  for (int i = tid; i < 2 * kBins; i += kThreads) s_hist[i / kBins][i % kBins] = 0;
  if (kCluster)
    for (int i = tid; i < kPasses * kBins; i += kThreads) s_total[kCluster ? i / kBins : 0][kCluster ? i % kBins : 0] = 0;
#pragma unroll
  for (int k = 0; k < kSelectKeys; ++k)
    if (k < rounds) sm.scores[warp][k * 33 + lane] = f[k];
  if (kCluster) cluster_sync_all();
  else __syncthreads();
  // Of this thread's entries those past the row's, and those that are picked anyway, have key 0, which no score has.
  const uint32_t all = (1u << mine) - 1;
  auto below = [&](int e) { return (1u << min(max(e - first, 0), mine)) - 1; };
  const uint32_t anyway = all & (below(p.first) | ~below(n - p.last)), competing = all & ~anyway;
  const bool edge = __any_sync(0xffffffffu, competing != (1u << rounds) - 1);
  uint32_t key[kSelectKeys];
#pragma unroll
  for (int k = 0; k < kSelectKeys; ++k) {
    if (k >= rounds) break;
    const int at = lane * rounds + k;
    key[k] = order_key(sm.scores[warp][at + (at >> 5)]);
    if (edge && (competing >> k & 1) == 0) key[k] = 0;
  }
  // Still in question: keys from lo on, of which the bits below `width` are open.
  uint32_t lo = 0;
  int width = 32;
  for (int pass = 0; need > 0; ++pass) {
    int* hist = s_hist[pass & 1];
    const int shift = max(width - kBits, 0);
    const uint32_t bins = 1u << (width - shift), hist_at = smem_addr(hist);
#pragma unroll
    for (int k = 0; k < kSelectKeys; ++k) {
      if (k >= rounds) break;
      count_in(hist_at, (key[k] - lo) >> shift, bins);
    }
    __syncthreads();
    if (kCluster) {
      int* total = s_total[kCluster ? pass : 0];
      for (int i = tid; i < kBins; i += kThreads) {
        const int v = hist[i];
        if (v == 0) continue;
        hist[i] = 0;
        for (int x = 0; x < S; ++x) remote_add(total + i, x, v);
      }
      cluster_sync_all();
      hist = total;
    } else {
      for (int i = tid; i < kBins; i += kThreads) s_hist[(pass + 1) & 1][i] = 0;
    }
    find_bin<kThreads, kBins>(hist, need, s_warp, [&](int bin, int above) {
      s_bin = bin;
      s_above = above;
    });
    __syncthreads();
    lo += static_cast<uint32_t>(s_bin) << shift;
    need -= s_above;
    width = shift;
    if (width == 0 || hist[s_bin] == need) break;  // (the whole bin is taken)
  }
  // Picked is what is above; what is still in question is equal, and the first `need` of it are picked.
  uint32_t over = anyway, open = 0;
  if (p.keep > p.first + p.last) {
    const uint32_t span = (1u << width) - 1;  // (width < 32 after a pass)
#pragma unroll
    for (int k = 0; k < kSelectKeys; ++k) {
      if (k >= rounds) break;
      if (key[k] > lo + span) over |= 1u << k;
      if (key[k] - lo <= span) open |= 1u << k;
    }
  }
  // Places: numbers picked and equal before.
  const int overs = __popc(over), equals = __popc(open);
  int place = overs | equals << 16;  // (each below 2^14 in a CTA)
  int scan = place;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += x;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = scan;
  __syncthreads();
  place = scan - place;
  int total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w == warp) place += total;
    total += s_warp[w];
  }
  int overs_before = place & 0xffff, equals_before = place >> 16;
  if (kCluster) {
    if (tid == 0) s_sum = total;
    cluster_sync_all();
    for (int x = 0; x < rank; ++x) {
      const int t = remote_int(&s_sum, x);
      overs_before += t & 0xffff;
      equals_before += t >> 16;
    }
  }
  for (uint32_t left = over | open; left != 0; left &= left - 1) {
    const int k = __ffs(left) - 1;
    const bool equal = (open >> k & 1u) != 0;
    if (!equal || equals_before < need) picks[overs_before + min(equals_before, need)] = first + k;
    if (equal) ++equals_before;
    else ++overs_before;
  }
  if (kCluster) cluster_sync_all();  // (another CTA may still read this one's sum)
}

// Rows too long for a cluster's registers: one CTA, which reads the scores again for every digit.
constexpr int kLongThreads = 1024;
constexpr int kLongBits = 11;

__global__ void __launch_bounds__(kLongThreads) select_long_kernel(SelectParams p) {
  constexpr int kWarps = kLongThreads / 32, kBins = 1 << kLongBits;
  __shared__ int s_hist[kBins];
  __shared__ int s_warp[2][kWarps];
  __shared__ int s_bin, s_above;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const SelectRow r = select_row(p, row);
  const int n = r.n;
  int32_t* picks = p.picks + static_cast<size_t>(row) * p.keep;
  if (tid == 0) p.counts[row] = r.count;
  for (int i = r.count + tid; i < p.keep; i += kLongThreads) picks[i] = -1;
  if (n <= p.keep) {
    for (int i = tid; i < n; i += kLongThreads) picks[i] = i;
    return;
  }
  const float* s = p.scores + static_cast<size_t>(row) * p.row_len;
  const int a = p.first, b = n - p.last;
  int need = p.keep - p.first - p.last;
  uint32_t prefix = 0, mask = 0;
  if (need == 0) prefix = mask = 0xffffffffu;
  for (int shift = 32 - kLongBits; need > 0; shift = max(0, shift - kLongBits)) {
    const uint32_t digit_mask = (mask == 0 ? 0xffffffffu : ~mask) >> shift;
    __syncthreads();
    for (int i = tid; i < kBins; i += kLongThreads) s_hist[i] = 0;
    __syncthreads();
    for (int i = a + tid; i < b; i += kLongThreads) {
      const uint32_t key = order_key(__ldg(s + i));
      if ((key & mask) == prefix) atomicAdd(&s_hist[(key >> shift) & digit_mask], 1);
    }
    __syncthreads();
    find_bin<kLongThreads, kBins>(s_hist, need, s_warp[0], [&](int bin, int above) {
      s_bin = bin;
      s_above = above;
    });
    __syncthreads();
    prefix |= static_cast<uint32_t>(s_bin) << shift;
    mask |= digit_mask << shift;
    need -= s_above;
    if (shift == 0 || s_hist[s_bin] == need) break;
  }
  // Each warp counts, then writes, a run of consecutive entries.
  const int run = ((n + kWarps - 1) / kWarps + 31) / 32 * 32;
  const int i0 = min(n, warp * run), i1 = min(n, i0 + run);
  auto classify = [&](int i, bool& over, bool& equal) {
    over = equal = false;
    if (i >= i1) return;
    if (i < a || i >= b) {
      over = true;
      return;
    }
    const uint32_t key = order_key(__ldg(s + i)) & mask;
    over = key > prefix;
    equal = key == prefix;
  };
  int overs = 0, equals = 0;
  for (int i = i0; i < i1; i += 32) {
    bool over, equal;
    classify(i + lane, over, equal);
    overs += __popc(__ballot_sync(0xffffffffu, over));
    equals += __popc(__ballot_sync(0xffffffffu, equal));
  }
  __syncthreads();
  if (lane == 0) {
    s_warp[0][warp] = overs;
    s_warp[1][warp] = equals;
  }
  __syncthreads();
  overs = equals = 0;
  for (int w = 0; w < warp; ++w) {
    overs += s_warp[0][w];
    equals += s_warp[1][w];
  }
  for (int i = i0; i < i1; i += 32) {
    bool over, equal;
    classify(i + lane, over, equal);
    const uint32_t mo = __ballot_sync(0xffffffffu, over), me = __ballot_sync(0xffffffffu, equal);
    const uint32_t below = (1u << lane) - 1;
    const int before = equals + __popc(me & below);
    if (over || (equal && before < need)) picks[overs + __popc(mo & below) + min(before, need)] = i + lane;
    overs += __popc(mo);
    equals += __popc(me);
  }
}

template <int kThreads, int kBits, bool kCluster>
cudaError_t launch_select(const SelectParams& p, int rows, int S, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(rows * S);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(SelectSpace<kThreads, kBits, kCluster>);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = kCluster ? 1 : 0;
  if (cfg.dynamicSmemBytes > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(select_kernel<kThreads, kBits, kCluster>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(cfg.dynamicSmemBytes));
    if (e != cudaSuccess) return e;
  }
  return cudaLaunchKernelEx(&cfg, select_kernel<kThreads, kBits, kCluster>, p);
}

}  // namespace
}  // namespace kvshot

using namespace kvshot;

extern "C" kvshot_status kvshot_page_bounds(const kvshot_attn_desc* d, const void* target_k, const int32_t* page_table,
                                            const int32_t* seq_lens, const int32_t* from_tokens, void* bounds,
                                            kvshot_stream_t stream) {
  kvshot_attn_desc heads;
  if (d != nullptr && d->hq == 0) {  // no query heads are read: a descriptor without them is as good
    heads = *d;
    heads.hq = heads.hkv;
    d = &heads;
  }
  if (kvshot_status st = check_partial(d, true)) return st;
  if (!target_k || !page_table || !seq_lens || !bounds) return KVSHOT_ERR_NULL;
  if (!aligned(target_k, 16) || !aligned(bounds, 16) || !aligned(page_table, 4) || !aligned(seq_lens, 4) ||
      !aligned(from_tokens, 4))
    return KVSHOT_ERR_ALIGN;
  const CacheView v = cache_view(d, page_table, seq_lens);
  const int64_t units = static_cast<int64_t>((v.len_bound + v.P - 1) / v.P) * v.hkv;
  // After growth most caches have a page or two to do, and CTAs without work are what costs.
  const int64_t most = std::max<int64_t>(1, static_cast<int64_t>(sm_count()) * (from_tokens != nullptr ? 8 : 64) / v.C);
  // (One CTA at least: lengths are looked at even without room.)
  const int x = static_cast<int>(std::clamp<int64_t>((units + kBoundsThreads / 32 - 1) / (kBoundsThreads / 32), 1, most));
  const cudaError_t e = launch_maybe_pdl(bounds_kernel, dim3(x, v.C), dim3(kBoundsThreads), 0, false,
                                         reinterpret_cast<cudaStream_t>(stream), v, static_cast<const uint4*>(target_k),
                                         from_tokens, static_cast<uint4*>(bounds));
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}

extern "C" kvshot_status kvshot_page_scores(const kvshot_attn_desc* d, const void* q, const void* bounds,
                                            const int32_t* page_table, const int32_t* seq_lens, float* scores,
                                            kvshot_stream_t stream) {
  if (kvshot_status st = check_partial(d, true)) return st;
  if (d->n_query == 0) return KVSHOT_OK;
  if (!q || !bounds || !page_table || !seq_lens || !scores) return KVSHOT_ERR_NULL;
  if (!aligned(q, 16) || !aligned(bounds, 32) || !aligned(page_table, 4) || !aligned(seq_lens, 4) || !aligned(scores, 4))
    return KVSHOT_ERR_ALIGN;
  ScoreParams p;
  p.v = cache_view(d, page_table, seq_lens);
  p.q = static_cast<const uint4*>(q);
  p.bounds = static_cast<const uint4*>(bounds);
  p.scores = scores;
  p.hq = d->hq;
  p.G = d->hq / d->hkv;
  p.Nq = d->n_query;
  int log_gp = 0;
  while ((1 << log_gp) < p.G) ++log_gp;
  if ((static_cast<int64_t>(p.Nq) << log_gp) >= INT_MAX || static_cast<int64_t>(p.v.max_pages) * p.v.hkv >= INT_MAX)
    return KVSHOT_ERR_UNSUPPORTED;
  p.scale = score_scale(d);
  const int pages = (p.v.len_bound + p.v.P - 1) / p.v.P, per_cta = kScoreWarps * 16;
  const int64_t tiles = static_cast<int64_t>((pages + kStPages - 1) / kStPages) * p.v.hkv * p.v.C;
  // Graph times (us, mma.sync against tcgen05) of 16 caches of 20K to 32K tokens: 16 rows 23, 25; 32: 28, 26; 48: 35, 27; 64: 41,
  // 29; 256: 141, 68.  64 caches of up to 8K: 32 rows 25, 32; 48: 30, 33; 64: 35, 35; 128: 64, 43.  4 of 32K: 48 rows 10.7,
  // 12.3; 64: 12.8, 12.6.  One of 32K: 64 rows 5.9, 7.6; 128: 9.1, 8.5.  One of 8K: 128 rows 7.1, 8.0; 256: 12, 8.1.
  const int64_t columns = static_cast<int64_t>(p.Nq) << log_gp;
  // Tiles that no cache fills: 192 rows, 50 caches of 68 pages 17, 27; 256 rows, 64 of 128 pages 42, 35.
  if (columns >= 48 && pages >= kStPages && columns * tiles >= (columns >= 128 ? 8 : 48) * 1024) {
    const uint32_t wait_ns = d->wait_limit_ns != 0 ? d->wait_limit_ns : static_cast<uint32_t>(kWaitLimitNs);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const cudaError_t e = log_gp == 0   ? launch_scores_tc<0>(p, tiles, wait_ns, st)
                          : log_gp == 1 ? launch_scores_tc<1>(p, tiles, wait_ns, st)
                          : log_gp == 2 ? launch_scores_tc<2>(p, tiles, wait_ns, st)
                          : log_gp == 3 ? launch_scores_tc<3>(p, tiles, wait_ns, st)
                          : log_gp == 4 ? launch_scores_tc<4>(p, tiles, wait_ns, st)
                                        : launch_scores_tc<5>(p, tiles, wait_ns, st);
    return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
  }
  const size_t smem = static_cast<size_t>(std::min(kScoreRows, ((p.Nq << log_gp) + 15) / 16 * 16)) * kScoreRowBytes;
  // Where there are more than twelve CTAs to an SM, each takes several chunks of pages, and q once.
  const int64_t heads = static_cast<int64_t>(p.v.hkv) * p.v.C;
  const int chunks = std::max(1, (pages + per_cta - 1) / per_cta);  // (lengths are looked at even without room)
  const int64_t each = std::max<int64_t>(1, (chunks * heads + 12 * sm_count() - 1) / (12 * sm_count()));
  const int x = static_cast<int>((chunks + each - 1) / each);
  auto* kernel = log_gp == 0   ? scores_kernel<0>
                 : log_gp == 1 ? scores_kernel<1>
                 : log_gp == 2 ? scores_kernel<2>
                 : log_gp == 3 ? scores_kernel<3>
                               : scores_kernel<4>;
  const cudaError_t e = launch_maybe_pdl(kernel, dim3(x, p.v.hkv, p.v.C), dim3(kScoreWarps * 32), smem, false,
                                         reinterpret_cast<cudaStream_t>(stream), p, log_gp);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}

extern "C" kvshot_status kvshot_select_top(const kvshot_select_desc* d, const float* scores, const int32_t* seq_lens,
                                           int32_t* picks, int32_t* counts, kvshot_stream_t stream) {
  if (d == nullptr) return KVSHOT_ERR_NULL;
  if (d->num_rows < 0 || d->row_len < 1 || d->rows_per_len < 1 || d->num_rows % d->rows_per_len != 0 ||
      d->tokens_per_entry < 1 || d->keep < 1 || d->first < 0 || d->last < 0 ||
      static_cast<int64_t>(d->first) + d->last > d->keep)
    return KVSHOT_ERR_SHAPE;
  if (d->num_rows >= INT_MAX / kMaxSelectCluster || d->row_len > 1 << 30 || d->keep > 1 << 30) return KVSHOT_ERR_UNSUPPORTED;
  if (d->num_rows == 0) return KVSHOT_OK;
  if (!scores || !seq_lens || !picks || !counts) return KVSHOT_ERR_NULL;
  if (!aligned(scores, 4) || !aligned(seq_lens, 4) || !aligned(picks, 4) || !aligned(counts, 4)) return KVSHOT_ERR_ALIGN;
  const SelectParams p{scores,          seq_lens,          picks,               counts,  d->err_flag, d->row_len,
                       d->rows_per_len, d->tokens_per_entry, d->keep, d->first, d->last};
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int n = d->row_len, rows = d->num_rows;  // (the longest that a row can be: lengths are known to the device alone)
  auto cluster = [&](int per_cta) {
    int S = 2;
    while (S < kMaxSelectCluster && S * per_cta < n) S *= 2;
    return S;
  };
  cudaError_t e;
  if (n <= 128 * kSelectKeys) e = launch_select<128, 9, false>(p, rows, 1, st);
  else if (n <= 512 * kSelectKeys && 2 * rows > sm_count()) e = launch_select<512, 11, false>(p, rows, 1, st);
  else if (n <= 512 * kSelectKeys * kMaxSelectCluster) e = launch_select<512, 11, true>(p, rows, cluster(8192), st);
  else if (n <= 1024 * kSelectKeys * kMaxSelectCluster) e = launch_select<1024, 11, true>(p, rows, kMaxSelectCluster, st);
  else e = launch_maybe_pdl(select_long_kernel, dim3(rows), dim3(kLongThreads), 0, false, st, p);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
