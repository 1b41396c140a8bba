// key_weights.cu -- the softmax weight that each cached token got from the query rows, accumulated.
//   w_out[c, j] = decay w[c, j] + sum over rows n and q heads of exp(scale q . k_j - lse[c, n, head])
#include <algorithm>
#include <cmath>

#include "kvshot_partial.cuh"
#include "kvshot_tcgen05.cuh"

namespace kvshot {
namespace {

using namespace dev;
using namespace partial;

struct WeightParams {
  CacheView v;
  const uint4 *q, *k;
  const float *lse, *weights;
  float* weights_out;
  int hq, G, Nq, weights_len;
  float qscale, decay;  // scale * log2(e)
  uint32_t wait_ns;
};

__device__ __forceinline__ int weights_len_of(const WeightParams& p, int c) {
  const int L = clamped_len(p.v, c);
  if (L <= p.weights_len) return L;
  set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
  return p.weights_len;
}

// lse of a row in the log2 domain, negated; a row that is empty gives nothing.
__device__ __forceinline__ float neg_log2_sum(float z) { return z == -INFINITY ? -INFINITY : z * -1.4426950408889634f; }

// ------------------------------------------------------------ few rows

// Up to 8 rows per KV head, 64 in small calls.  A warp's keys are the M rows of mma.sync, the query rows its columns; operands go
// from global memory straight to registers, the next keys' while the present ones' are multiplied.  A lane sums the exponentials of
// its keys' columns over its heads; the heads are shared out over a cluster of CTAs where there are few keys, whose sums
// meet in shared memory in rank order.
constexpr int kDirectRows = 64;  // rows of a KV head, at most
constexpr int kDirectWarps = 4;
constexpr int kDirectChunks = 2;  // of 16 keys, per warp
constexpr int kDirectKeys = kDirectWarps * kDirectChunks * 16;

template <int NT>
__global__ void __launch_bounds__(kDirectWarps * 32) weights_kernel(WeightParams p) {
  __shared__ float s_w[kDirectKeys];
  const int S = static_cast<int>(cluster_size());
  const int rank = blockIdx.x % S, c = blockIdx.y;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int cta0 = blockIdx.x / S * kDirectKeys;
  // (Table entries are looked up beside the length, and what the keys had before beside everything.)
  int id[kDirectChunks][2];
#pragma unroll
  for (int i = 0; i < kDirectChunks; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int page = (cta0 + (warp * kDirectChunks + i) * 16 + g + 8 * e) / p.v.P;
      id[i][e] = p.v.page_table == nullptr ? c : page < p.v.max_pages ? __ldg(p.v.page_table + static_cast<size_t>(c) * p.v.max_pages + page) : -1;
    }
  const int key0 = cta0 + threadIdx.x;
  const bool sums = static_cast<int>(threadIdx.x) % S == rank && key0 < p.weights_len;  // this thread ends key0's
  const size_t key_at = static_cast<size_t>(c) * p.weights_len + key0;
  const float had = sums && p.weights != nullptr ? p.weights[key_at] : 0.f;
  const int L = weights_len_of(p, c);
  if (cta0 >= L) return;  // (the whole cluster)
  const uint4 zero = make_uint4(0, 0, 0, 0);
  bool live[kDirectChunks][2];
  size_t row[kDirectChunks][2];  // of KV head 0
  float w[kDirectChunks][2] = {};
#pragma unroll
  for (int i = 0; i < kDirectChunks; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = cta0 + (warp * kDirectChunks + i) * 16 + g + 8 * e, page = j / p.v.P;
      live[i][e] = j < L && static_cast<unsigned>(id[i][e]) < static_cast<unsigned>(p.v.num_pages);
      if (j < L && !live[i][e]) set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
      row[i][e] = (static_cast<size_t>(live[i][e] ? id[i][e] : 0) * p.v.hkv * p.v.P + (j - page * p.v.P)) * 16 + t;
    }
  const int h0 = p.v.hkv * rank / S, h1 = p.v.hkv * (rank + 1) / S, rows = p.Nq * p.G;
  const size_t head = static_cast<size_t>(p.v.P) * 16;
  uint4 a[kDirectChunks][2][4];
  auto load = [&](int i, int h) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) a[i][e][j] = live[i][e] ? __ldg(p.k + row[i][e] + h * head + 4 * j) : zero;
  };
#pragma unroll
  for (int i = 0; i < kDirectChunks; ++i) load(i, h0);
  for (int h = h0; h < h1; ++h) {
    uint4 q[NT][4];
    float z[NT][2];
    bool in[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 8 + g;
      const size_t at = ((static_cast<size_t>(c) * p.Nq + r / p.G) * p.hq + h * p.G + r % p.G) * 16 + t;
#pragma unroll
      for (int j = 0; j < 4; ++j) q[nt][j] = r < rows ? __ldg(p.q + at + 4 * j) : zero;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r2 = nt * 8 + 2 * t + e;
        in[nt][e] = r2 < rows;
        z[nt][e] = in[nt][e] ? neg_log2_sum(__ldg(p.lse + (static_cast<size_t>(c) * p.Nq + r2 / p.G) * p.hq + h * p.G + r2 % p.G)) : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < kDirectChunks; ++i) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) mma_piece(d, a[i][0][j], a[i][1][j], q[nt][j]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (in[nt][e & 1]) w[i][e >> 1] += ex2(fmaf(d[e], p.qscale, z[nt][e & 1]));
      }
      if (h + 1 < h1) load(i, h + 1);
    }
  }
#pragma unroll
  for (int i = 0; i < kDirectChunks; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float x = w[i][e];
      x += __shfl_xor_sync(0xffffffffu, x, 1);
      x += __shfl_xor_sync(0xffffffffu, x, 2);
      if (t == 0) s_w[(warp * kDirectChunks + i) * 16 + g + 8 * e] = live[i][e] ? x : -1.f;  // (a page passed over)
    }
  if (S > 1) cluster_sync_all();
  else __syncthreads();
  if (sums && key0 < L) {
    float x[8], sum = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) x[r] = r < S ? remote_float(smem_addr(&s_w[threadIdx.x]), r) : 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) sum += x[r];
    if (!(s_w[threadIdx.x] == -1.f)) p.weights_out[key_at] = fmaf(p.decay, had, sum);
  }
  if (S > 1) cluster_sync_all();  // (another CTA may still read this one's sums)
}
static_assert(kDirectWarps * 32 == kDirectKeys, "a thread per key");

// ------------------------------------------------------------ many rows

// More rows per KV head: tcgen05.  128 keys are the M rows of S = K Q^T and the query rows (up to 256 of whole
// nodes) its N columns, so that a key is a lane of tensor memory and its thread sums its own columns: no exchange between
// threads.  One persistent CTA per SM takes an equal run of the caches' tiles, cut into pieces of one cache; a piece is
// passed over once per KV head and block of rows, K tiles streaming through a ring while the next pass's q is loaded.
//   warps 0..3, 4..7  sums of the piece's even and odd tiles.  S comes in units of up to 128 columns; each warpgroup has two
//                     units' room in tensor memory.  Its keys' sums stay with their threads until the piece's end.
//   warp 8            TMA, and the rows' lse;  warp 9: MMA, and the owner of tensor memory
// Up to 128 rows the call reads K at the copy's rate (16 x 32K tokens 166 to 170 us, floor 160).  With 256 rows (20K to 32K
// tokens each) it takes 188 to 192 us in a graph, 1.2 PFLOP/s, and 190 to 209 by box as calls one after another: the bytes and
// the hand-overs alone take 149, with the products 182, with the exponentials 175.  No faster: both units of a tile as one product (198), five tiles in the ring with one place for q (197),
// four warpgroups of a unit each (192).  Operands not in uniform registers cost 26 us, rooms given back after their sums 11.
constexpr int kTcGroups = 2;  // warpgroups
constexpr int kTcLoadWarp = 4 * kTcGroups, kTcMmaWarp = kTcLoadWarp + 1;
constexpr int kTcThreads = (kTcMmaWarp + 1) * 32;
constexpr int kTcKeys = 128;
constexpr int kTcMaxRows = 256;
constexpr int kTcTileBytes = kTcKeys * 256;
constexpr int kTcMaxStages = 6;
constexpr int kTcPart = 128;      // columns of S handed over at a time
constexpr int kTcUnits = 4;       // room for them in tensor memory
constexpr int kTcTmemCols = kTcUnits * kTcPart;
constexpr int kTcSmem = 232448;                      // what a CTA can have
constexpr int kTcTail = 2 * kTcMaxRows * 4 + 512;    // row sums, barriers
// Tiles of a piece, at most: one pass's K of all CTAs stays in L2 for the next block of rows; and 32 where there is one block.
constexpr int kTcPiece = 32, kTcPieceBlocks = 16;

struct WeightTcParams {
  WeightParams w;
  int nodes_per_block, blocks, cols;  // row blocks of whole nodes; cols: their rows rounded up to 16
  int stages, box_rows;               // ring; keys of a box of K
  int grouped;                        // boxes of whole row groups (else of 8 rows from any row)
};
struct WeightMaps {
  CUtensorMap k, q;
};

struct TcPiece {
  int c, tile, tiles, len;
};
// The CTA's pieces in order.  The whole warp calls, with the same arguments.
struct TcCursor {
  int c, tile, left, L, cap;
  __device__ __forceinline__ void init(const WeightTcParams& p) {
    const int lane = threadIdx.x & 31;
    int total = 0;
    for (int i = lane; i < p.w.v.C; i += 32) total += (weights_len_of(p.w, i) + kTcKeys - 1) / kTcKeys;
    total = __reduce_add_sync(0xffffffffu, total);
    const int t0 = static_cast<int>(static_cast<int64_t>(total) * blockIdx.x / gridDim.x);
    left = static_cast<int>(static_cast<int64_t>(total) * (blockIdx.x + 1) / gridDim.x) - t0;
    cap = p.blocks > 1 ? kTcPieceBlocks : kTcPiece;
    c = tile = L = 0;
    if (left == 0) return;
    int before = 0;
    for (int base = 0;; base += 32) {  // (t0 is below the total)
      const int n = base + lane < p.w.v.C ? (weights_len_of(p.w, base + lane) + kTcKeys - 1) / kTcKeys : 0;
      int scan = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += x;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + scan > t0);
      if (past != 0) {
        const int at = __ffs(past) - 1;
        c = base + at;
        tile = t0 - before - __shfl_sync(0xffffffffu, scan - n, at);
        break;
      }
      before += __shfl_sync(0xffffffffu, scan, 31);
    }
    L = weights_len_of(p.w, c);
  }
  __device__ __forceinline__ bool next(const WeightTcParams& p, TcPiece* out) {
    if (left == 0) return false;
    while (tile * kTcKeys >= L) {
      ++c;
      tile = 0;
      L = weights_len_of(p.w, c);
    }
    const int here = min(min(left, cap), (L + kTcKeys - 1) / kTcKeys - tile);
    *out = TcPiece{c, tile, here, L};
    left -= here;
    tile += here;
    return true;
  }
};

struct TcBarriers {
  uint64_t kfull[kTcMaxStages], kempty[kTcMaxStages], qfull[2], qempty[2], zfull[2], zempty[2];
  uint64_t sfull[kTcUnits], sempty[kTcUnits], done;
  uint32_t tmem;
};

// Waits for this warp's loads from tensor memory, of which v is one: what is computed from v cannot move before it.
__device__ __forceinline__ void wait_ld_of(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                 "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                 "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                 "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}

// exp2(s qscale - z) of 32 columns, added to the sums.
__device__ __forceinline__ void add_columns(const uint32_t (&v)[32], const float* z, float qscale, float2 (&sum)[2]) {
  const float2 qs = make_float2(qscale, qscale);
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const float4 n = *reinterpret_cast<const float4*>(z + i);
    const float2 x = fma2(make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), qs, make_float2(n.x, n.y));
    const float2 y = fma2(make_float2(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), qs, make_float2(n.z, n.w));
    sum[0] = add2(sum[0], make_float2(ex2(x.x), ex2(x.y)));
    sum[1] = add2(sum[1], make_float2(ex2(y.x), ex2(y.y)));
  }
}

__global__ void __launch_bounds__(kTcThreads, 1)
    weights_tc_kernel(const __grid_constant__ WeightTcParams p, const __grid_constant__ WeightMaps maps) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (known to be uniform)
  const int qbytes = p.cols * 256, hkv = p.w.v.hkv, G = p.w.G;
  uint8_t* ring = smem + 2 * qbytes;
  float* s_z = reinterpret_cast<float*>(ring + p.stages * kTcTileBytes);  // [2][kTcMaxRows], by pass
  TcBarriers& bar = *reinterpret_cast<TcBarriers*>(s_z + 2 * kTcMaxRows);
  if ((smem_addr(smem) & 1023u) != 0) {  // (the swizzled tiles' layout counts on it; dynamic shared memory is, alone)
    set_error(p.w.v.err, KVSHOT_ERR_CUDA);
    return;
  }
  // Rows of q past a block's are zeros (no copy ever writes them).
  for (int i = threadIdx.x; i < 2 * qbytes / 16; i += kTcThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(smem_addr(&bar.kfull[i]), 1);
      mbar_init(smem_addr(&bar.kempty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_addr(&bar.qfull[i]), 1);
      mbar_init(smem_addr(&bar.qempty[i]), 1);
      mbar_init(smem_addr(&bar.zfull[i]), 1);
      mbar_init(smem_addr(&bar.zempty[i]), 4 * kTcGroups);
    }
    for (int i = 0; i < kTcUnits; ++i) {
      mbar_init(smem_addr(&bar.sfull[i]), 1);
      mbar_init(smem_addr(&bar.sempty[i]), 4);
    }
    mbar_init(smem_addr(&bar.done), 1);
    fence_mbar_init();
    prefetch_tensormap(&maps.k);
    prefetch_tensormap(&maps.q);
  }
  TcCursor cu;  // (the lengths are on their way beside the rest of the start)
  cu.init(p);
  if (warp == kTcMmaWarp) {
    tc::tmem_alloc(smem_addr(&bar.tmem), kTcTmemCols);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = bar.tmem;
  const uint64_t limit = p.w.wait_ns;
  int32_t* err = p.w.v.err;
  TcPiece pc;
  const int passes = hkv * p.blocks;

  if (warp == kTcLoadWarp) {  // ---- loads
    const uint64_t once = l2_policy_evict_first();
    const int boxes = kTcKeys / p.box_rows, P = p.w.v.P;
    int stage = 0, pass_no = 0, q_issued = 0;
    uint32_t phase = 1, issued = 0;  // of the kempty barriers (their first use needs no wait); stages ever filled
    bool ok = true;
    // Row (of the [rows, 128] matrix, KV head 0) of this lane's box of a tile, or -1.
    auto box_row = [&](int c, int tile, int L) -> int64_t {
      const int key = tile * kTcKeys + lane * p.box_rows;
      if (lane >= boxes || key >= L) return -1;
      const int page = key / P, id = page_id(p.w.v, c, page);
      return id < 0 ? -1 : static_cast<int64_t>(id) * hkv * P + (key - page * P);
    };
    while (ok && cu.next(p, &pc)) {
      int64_t next = box_row(pc.c, pc.tile, pc.len);
      for (int pass = 0; ok && pass < passes; ++pass, ++pass_no) {
        const int h = pass / p.blocks, rb = pass % p.blocks, qb = pass_no & 1;
        const uint32_t qbar = smem_addr(&bar.qfull[qb]);
        if (pass_no >= 2) ok = wait(smem_addr(&bar.qempty[qb]), ((pass_no >> 1) - 1) & 1, err, limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) {
          const int rows = p.nodes_per_block * G;
          const uint32_t dst = smem_addr(smem) + qb * qbytes;
          mbar_arrive_expect_tx(qbar, rows * 256);
          tma_load_4d(dst, &maps.q, 0, h * G, rb * p.nodes_per_block, pc.c, qbar);
          tma_load_4d(dst + p.cols * 128, &maps.q, 64, h * G, rb * p.nodes_per_block, pc.c, qbar);
        }
        ++q_issued;
        // The rows' lse.  (Its loads are under way while the pass's first tiles are asked for.)
        const int n0 = rb * p.nodes_per_block, rows = min(p.nodes_per_block, p.w.Nq - n0) * G;
        float z[kTcMaxRows / 32];
#pragma unroll
        for (int i = 0; i < kTcMaxRows / 32; ++i) {
          const int r = i * 32 + lane;
          z[i] = r < rows ? __ldg(p.w.lse + (static_cast<size_t>(pc.c) * p.w.Nq + n0 + r / G) * p.w.hq + h * G + r % G) : -INFINITY;
        }
        auto put_lse = [&] {
          if (pass_no >= 2) ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.zempty[qb]), ((pass_no >> 1) - 1) & 1, err, limit));
#pragma unroll
          for (int i = 0; i < kTcMaxRows / 32; ++i) s_z[qb * kTcMaxRows + i * 32 + lane] = neg_log2_sum(z[i]);
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_addr(&bar.zfull[qb]));
        };
        for (int i = 0; i < pc.tiles; ++i) {
          const int64_t row = next;
          // (the next tile's look-up is under way while this one waits for room)
          next = box_row(pc.c, pc.tile + (i + 1 < pc.tiles ? i + 1 : 0), pc.len);
          if (issued >= static_cast<uint32_t>(p.stages)) ok = wait(smem_addr(&bar.kempty[stage]), phase, err, limit);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const uint32_t full = smem_addr(&bar.kfull[stage]);
          const int live = __popc(__ballot_sync(0xffffffffu, row >= 0));
          if (lane == 0) mbar_arrive_expect_tx(full, live * p.box_rows * 256);
          __syncwarp();
          if (row >= 0) {
            const uint32_t dst = smem_addr(ring) + stage * kTcTileBytes + lane * p.box_rows * 256;
            const int64_t y = row + static_cast<int64_t>(h) * P;
            if (p.grouped) tma_load_4d_hint(dst, &maps.k, 0, 0, 0, static_cast<int>(y >> 3), full, once);
            else tma_load_3d(dst, &maps.k, 0, static_cast<int>(y), 0, full, once);
          }
          ++issued;
          if (++stage == p.stages) {
            stage = 0;
            phase ^= 1u;
          }
          if (i == 0) put_lse();
          if (!ok) break;
        }
      }
    }
    // No copy is in flight when the CTA ends: every phase that was filled has to complete.
    for (uint32_t i = issued > static_cast<uint32_t>(p.stages) ? issued - p.stages : 0; i < issued; ++i)
      mbar_wait(smem_addr(&bar.kfull[i % p.stages]), (i / p.stages) & 1, err);
    for (int i = max(0, q_issued - 2); i < q_issued; ++i) mbar_wait(smem_addr(&bar.qfull[i & 1]), (i >> 1) & 1, err);
  } else if (warp == kTcMmaWarp) {  // ---- products
    // (All control is uniform, so that operands are in uniform registers: 26 cycles to issue an MMA, and not 50.)
    int stage = 0, pass_no = 0;
    uint32_t phase = 0;
    uint32_t units0 = 0, units1 = 0;  // that each warpgroup has been given
    bool ok = true;
    while (__all_sync(0xffffffffu, ok && cu.next(p, &pc))) {
      const int tiles = __shfl_sync(0xffffffffu, pc.tiles, 0);
      for (int pass = 0; ok && pass < passes; ++pass, ++pass_no) {
        const int qb = pass_no & 1;
        ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.qfull[qb]), (pass_no >> 1) & 1, err, limit));
        const uint32_t qbase = smem_addr(smem) + qb * qbytes;
        for (int i = 0; ok && i < tiles; ++i) {
          uint32_t& n = (i & 1) != 0 ? units1 : units0;
          for (int col = 0; col < p.cols; col += kTcPart, ++n) {
            const int room = 2 * (i & 1) + (n & 1);
            if (n >= 2) ok = wait(smem_addr(&bar.sempty[room]), ((n >> 1) - 1) & 1, err, limit);
            if (col == 0) ok = ok && wait(smem_addr(&bar.kfull[stage]), phase, err, limit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t idesc = tc::idesc_bf16(kTcKeys, min(kTcPart, p.cols - col), false);
            const uint32_t kbase = smem_addr(ring) + stage * kTcTileBytes, qpart = qbase + col * 128;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
              const uint64_t ad = tc::smem_desc_sw128(kbase + (ks >> 2) * kGroupHalfBytes + (ks & 3) * 32, 16, kGroupBytes);
              const uint64_t bd = tc::smem_desc_sw128(qpart + (ks >> 2) * (p.cols * 128) + (ks & 3) * 32, 16, 1024);
              tc::tc_mma_elect(tmem + room * kTcPart, ad, bd, idesc, ks > 0);
            }
            tc::tc_commit_elect(smem_addr(&bar.sfull[room]));
          }
          if (!ok) break;
          tc::tc_commit_elect(smem_addr(&bar.kempty[stage]));
          if (++stage == p.stages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (ok) tc::tc_commit_elect(smem_addr(&bar.qempty[qb]));
      }
    }
    tc::tc_commit_elect(smem_addr(&bar.done));  // every product this warp issued has completed
    mbar_wait(smem_addr(&bar.done), 0, err);
  } else {  // ---- sums
    const int wg = warp >> 2, tid = threadIdx.x & 127;
    const uint32_t my_tmem = tmem + 2 * wg * kTcPart + (static_cast<uint32_t>(warp & 3) << 21);
    int pass_no = 0;
    uint32_t units = 0;
    bool ok = true;
    while (ok && cu.next(p, &pc)) {
      float acc[kTcPiece / kTcGroups];
      for (int x = 0; x < kTcPiece / kTcGroups; ++x) acc[x] = 0.f;
      for (int pass = 0; ok && pass < passes; ++pass, ++pass_no) {
        const int rb = pass % p.blocks, rows = min(p.nodes_per_block, p.w.Nq - rb * p.nodes_per_block) * G;
        const float* z0 = s_z + (pass_no & 1) * kTcMaxRows;
        ok = __all_sync(0xffffffffu, wait(smem_addr(&bar.zfull[pass_no & 1]), (pass_no >> 1) & 1, err, limit));
        for (int i = wg; ok && i < pc.tiles; i += kTcGroups) {
          float2 sum[2] = {};
          for (int col = 0; col < p.cols; col += kTcPart, ++units) {
            const int room = units & 1, here = min(kTcPart, rows - col), whole = here >> 5;
            ok = wait(smem_addr(&bar.sfull[2 * wg + room]), (units >> 1) & 1, err, limit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t at = my_tmem + room * kTcPart;
            const float* z = z0 + col;
            uint32_t v[32], v2[32];
            // (The room is given back as soon as its last columns are in registers.)
            auto give_back = [&] {
              tc::tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_addr(&bar.sempty[2 * wg + room]));
            };
            if (whole > 0) tc::tmem_ld32(at, v);
            if (here == kTcPart) {  // (the common case without a branch between its loads)
#pragma unroll
              for (int cc = 0; cc < kTcPart / 32; cc += 2) {
                wait_ld_of(v);
                tc::tmem_ld32(at + 32 * (cc + 1), v2);
                add_columns(v, z + 32 * cc, p.w.qscale, sum);
                wait_ld_of(v2);
                if (cc + 2 < kTcPart / 32) tc::tmem_ld32(at + 32 * (cc + 2), v);
                else give_back();
                add_columns(v2, z + 32 * (cc + 1), p.w.qscale, sum);
              }
              continue;
            }
            for (int cc = 0; cc < whole; ++cc) {
              wait_ld_of(v);
              add_columns(v, z + 32 * cc, p.w.qscale, sum);
              if (cc + 1 < whole) tc::tmem_ld32(at + 32 * (cc + 1), v);
            }
            for (int x = max(whole, 0) * 32; x < here; x += 4) {
              uint32_t u[4];
              tc::tmem_ld4(at + x, u);
              asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3])::"memory");
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (x + e < here) sum[e & 1].x += ex2(fmaf(__uint_as_float(u[e]), p.w.qscale, z[x + e]));
            }
            give_back();
          }
          acc[i / kTcGroups] += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&bar.zempty[pass_no & 1]));
      }
      // What the keys had, and their pages (those passed over are left as they are): eight tiles' loads at a time.
      for (int i0 = wg; i0 < pc.tiles; i0 += 8 * kTcGroups) {
        int page[8];
        float before[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int i = i0 + x * kTcGroups, j = (pc.tile + i) * kTcKeys + tid;
          const bool live = i < pc.tiles && j < pc.len;
          page[x] = !live                          ? -1
                    : p.w.v.page_table == nullptr ? 0
                                                  : __ldg(p.w.v.page_table + static_cast<size_t>(pc.c) * p.w.v.max_pages + j / p.w.v.P);
          before[x] = live && p.w.weights != nullptr ? p.w.weights[static_cast<size_t>(pc.c) * p.w.weights_len + j] : 0.f;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int j = (pc.tile + i0 + x * kTcGroups) * kTcKeys + tid;
          if (static_cast<unsigned>(page[x]) < static_cast<unsigned>(p.w.v.num_pages))
            p.w.weights_out[static_cast<size_t>(pc.c) * p.w.weights_len + j] = fmaf(p.w.decay, before[x], acc[i0 / kTcGroups + x]);
        }
      }
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == kTcMmaWarp) tc::tmem_dealloc(tmem, kTcTmemCols);
}

template <int NT>
cudaError_t launch_direct(const WeightParams& p, int tiles, int S, cudaStream_t stream) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles * S, p.v.C);
  cfg.blockDim = dim3(kDirectWarps * 32);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, weights_kernel<NT>, p);
}

cudaError_t launch_tc(const WeightParams& w, const void* q, const void* k, int64_t tiles, cudaStream_t stream) {
  WeightTcParams p;
  p.w = w;
  // Blocks of whole nodes, of equal size.
  const int most = kTcMaxRows / w.G;
  p.blocks = (w.Nq + most - 1) / most;
  p.nodes_per_block = (w.Nq + p.blocks - 1) / p.blocks;
  p.cols = (p.nodes_per_block * w.G + 15) / 16 * 16;
  p.stages = std::min(kTcMaxStages, (kTcSmem - kTcTail - 2 * p.cols * 256) / kTcTileBytes);
  const bool paged = w.v.page_table != nullptr;
  p.grouped = paged || w.v.P % 8 == 0;
  p.box_rows = !p.grouped ? 8 : paged ? std::min(w.v.P, 64) : 64;
  const uint64_t rows = static_cast<uint64_t>(w.v.num_pages) * w.v.hkv * w.v.P;
  WeightMaps maps;
  const bool kmap = p.grouped ? map_groups(&maps.k, k, rows, p.box_rows / 8) : map_any_8(&maps.k, k, rows);
  if (!kmap || !map_q(&maps.q, q, w.v.C, w.Nq, w.hq, w.G, p.nodes_per_block)) return cudaErrorInvalidValue;
  const size_t smem = 2 * p.cols * 256 + p.stages * kTcTileBytes + kTcTail;
  static_assert(sizeof(TcBarriers) <= 512, "barriers fit the tail");
  cudaError_t e = cudaFuncSetAttribute(weights_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kTcSmem);
  if (e != cudaSuccess) return e;
  const int grid = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(sm_count(), tiles)));
  return launch_maybe_pdl(weights_tc_kernel, dim3(grid), dim3(kTcThreads), smem, false, stream, p, maps);
}

}  // namespace
}  // namespace kvshot

using namespace kvshot;

extern "C" kvshot_status kvshot_key_weights(const kvshot_attn_desc* d, const void* q, const void* target_k,
                                            const int32_t* page_table, const int32_t* seq_lens, const float* lse,
                                            float decay, int32_t weights_len, const float* weights, float* weights_out,
                                            kvshot_stream_t stream) {
  if (kvshot_status st = check_partial(d, page_table != nullptr)) return st;
  if (!(decay >= 0.f && decay <= 1.f) || weights_len < 0) return KVSHOT_ERR_SHAPE;
  if (!target_k || !seq_lens || !weights_out || (d->n_query > 0 && (!q || !lse))) return KVSHOT_ERR_NULL;
  if (!aligned(q, 16) || !aligned(target_k, 16) || !aligned(page_table, 4) || !aligned(seq_lens, 4) || !aligned(lse, 4) ||
      !aligned(weights, 4) || !aligned(weights_out, 4))
    return KVSHOT_ERR_ALIGN;
  WeightParams p;
  p.v = cache_view(d, page_table, seq_lens);
  p.q = static_cast<const uint4*>(q);
  p.k = static_cast<const uint4*>(target_k);
  p.lse = lse;
  p.weights = decay > 0.f ? weights : nullptr;
  p.weights_out = weights_out;
  p.hq = d->hq;
  p.G = d->hq / d->hkv;
  p.Nq = d->n_query;
  p.weights_len = weights_len;
  p.qscale = score_scale(d) * 1.4426950408889634f;
  p.decay = decay;
  p.wait_ns = d->wait_limit_ns != 0 ? d->wait_limit_ns : static_cast<uint32_t>(kWaitLimitNs);
  const int most = std::min(p.v.len_bound, weights_len), rows = p.G * p.Nq;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e;
  // 9 to 64 rows: two to eight n-tiles of registers a key cost the direct kernel its occupancy, which does not matter before the
  // SMs have tiles enough (us in a graph, direct against tcgen05; 16 rows over 8K tokens 11, 16, over 16 x 32K 221, 168; 32 rows
  // over 4K 7.0, 16.2, over 8K 13.1, 16.6, over 16K 18.5, 17.0; 64 rows over 4K 10.3, 17.9, over 8K 19.6, 17.3).
  const int64_t tc_tiles = static_cast<int64_t>((most + kTcKeys - 1) / kTcKeys) * p.v.C;
  const int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : rows <= 32 ? 4 : 8;
  if (rows > kDirectRows || (nt > 1 && nt / 2 * tc_tiles > sm_count())) {
    e = launch_tc(p, q, target_k, tc_tiles, s);
  } else {
    const int tiles = std::max(1, (most + kDirectKeys - 1) / kDirectKeys);  // (lengths are looked at even without room)
    int S = 1;  // CTAs that share the heads: until the SMs have two each
    while (S < 8 && 2 * S <= p.v.hkv && static_cast<int64_t>(tiles) * p.v.C * S < 2 * sm_count()) S *= 2;
    e = nt == 1   ? launch_direct<1>(p, tiles, S, s)
        : nt == 2 ? launch_direct<2>(p, tiles, S, s)
        : nt == 4 ? launch_direct<4>(p, tiles, S, s)
                  : launch_direct<8>(p, tiles, S, s);
  }
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
