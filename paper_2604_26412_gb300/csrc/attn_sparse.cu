// attn_sparse.cu -- draft attention over the pages picked for each query row and KV head, and the draft K/V.
#include <algorithm>
#include <cmath>

#include "kvshot_partial.cuh"

namespace kvshot {
namespace {

using namespace dev;
using namespace partial;

constexpr int kSparseWarps = 4;
constexpr int kSparseThreads = kSparseWarps * 32;
constexpr int kPartStride = kHeadDim + 4;  // floats of a row of a warp's partial result in shared memory

struct SparseParams {
  CacheView v;
  const uint4 *q, *k, *val, *dk, *dv;
  __nv_bfloat16* out;
  float* lse;
  const int32_t *picks, *counts, *tree_parent;
  int per_seq, hq, G, Nq, N, n_max, max_picks;
  float qscale;  // scale * log2(e)
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void tma_load_3d_plain(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

// Running softmax of one warp: the q heads of the KV head (padded to 8 NT rows) are the N columns of both products, so a
// decoded row costs each MMA little padding; 16 keys at a time are the M rows of S^T = K Q^T and the depth of
// O^T = V^T P^T.  Lane (g, t) keeps for rows 2 t, 2 t + 1 of each n-tile the reference, its part of the sum, and the
// dims 16 g .. 16 g + 15 of O.
template <int NT>
struct WarpState {
  uint4 q[NT][4];
  float m[NT][2], l[NT][2], o[NT][8][4];

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
    }
  }

  // kr: this lane's rows of K (keys g and g + 8 of the 16), vr: of V (keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9); -1: no key.
  __device__ __forceinline__ void step(const uint4* __restrict__ k, const uint4* __restrict__ v, const int (&kr)[2],
                                       const int (&vr)[4], float qscale, int g, int t) {
    // 32-byte loads: lane (g, t) has pieces 2 t, 2 t + 1 of each half of its key rows, and 2 g, 2 g + 1 of its value rows.
    const Row32 none = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    Row32 a[2][2], b[4];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < 2; ++j) a[e][j] = kr[e] >= 0 ? load32(k + static_cast<size_t>(kr[e]) * 16 + 8 * j + 2 * t) : none;
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = vr[e] >= 0 ? load32(v + static_cast<size_t>(vr[e]) * 16 + 2 * g) : none;
    uint32_t p0[NT], p1[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};  // (two chains of products)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        mma_piece(s, a[0][j].lo, a[1][j].lo, q[nt][2 * j]);
        mma_piece(s2, a[0][j].hi, a[1][j].hi, q[nt][2 * j + 1]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = kr[e >> 1] >= 0 ? (s[e] + s2[e]) * qscale : -INFINITY;
      const float top0 = fmaxf(s[0], s[2]), top1 = fmaxf(s[1], s[3]);
      // The reference moves only when a score is more than 2^8 above it: P stays in range, and the exchange and the
      // rescaling are rare.
      if (__any_sync(0xffffffffu, top0 > m[nt][0] + 8.f || top1 > m[nt][1] + 8.f)) {
        float top[2] = {top0, top1};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], x));
          const float now = fmaxf(m[nt][e], top[e]);
          const float f = now == -INFINITY ? 1.f : ex2(m[nt][e] - now);
          m[nt][e] = now;
          l[nt][e] *= f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[nt][i][e] *= f;
            o[nt][i][2 + e] *= f;
          }
        }
      }
      const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
      s[0] = ex2(s[0] - m0);
      s[1] = ex2(s[1] - m1);
      s[2] = ex2(s[2] - m0);
      s[3] = ex2(s[3] - m1);
      l[nt][0] += s[0] + s[2];
      l[nt][1] += s[1] + s[3];
      // (key, row pair) -> (row, key pair): the B operand of the second product.  bf16: the range of P's products with V.
      p0[nt] = transpose8x8(pack_bf16x2(s[0], s[1]));
      p1[nt] = transpose8x8(pack_bf16x2(s[2], s[3]));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w0 = word(i < 4 ? b[0].lo : b[0].hi, i & 3), w1 = word(i < 4 ? b[1].lo : b[1].hi, i & 3);
      const uint32_t w2 = word(i < 4 ? b[2].lo : b[2].hi, i & 3), w3 = word(i < 4 ? b[3].lo : b[3].hi, i & 3);
      const uint32_t av[4] = {__byte_perm(w0, w1, 0x5410), __byte_perm(w0, w1, 0x7632), __byte_perm(w2, w3, 0x5410),
                              __byte_perm(w2, w3, 0x7632)};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(o[nt][i], av, p0[nt], p1[nt]);
    }
  }
};

// A unit is one (cache, KV head, query row); the CTAs of a cluster (1 to 8) take its picks in turn, the last one the draft keys
// too, and a CTA's warps 16 keys in turn.  Nodes of one cache and head are next to one another in the grid: their pages
// overlap, and meet in L2.  A call of few units is a chain of latencies: picks, table, K and V, the states' meeting.  So picks
// and table entries are loaded before the length and the count are known, as far as the lists and the table reach.
template <int NT>
__global__ void __launch_bounds__(kSparseThreads) sparse_kernel(SparseParams p) {
  extern __shared__ __align__(16) float s_part[];  // [warps][8 NT][kPartStride]; the CTA's state is joined in the first warp's
  __shared__ int s_row[kSparseThreads], s_valid[kSparseThreads];
  __shared__ float s_m[kSparseWarps][8 * NT], s_l[kSparseWarps][8 * NT];
  __shared__ int s_parent[kMaxTreeNodes], s_line[kMaxTreeNodes];
  __shared__ int s_line_len;
  const int S = static_cast<int>(cluster_size());
  const int rank = blockIdx.x % S, unit = blockIdx.x / S;
  const int n = unit % p.Nq, h = unit / p.Nq % p.v.hkv, c = unit / p.Nq / p.v.hkv;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const size_t list = (static_cast<size_t>(c) * p.Nq + n) * p.v.hkv + h;
  const int32_t* picks = p.picks + list * p.max_picks;
  const int32_t* table = p.v.page_table + static_cast<size_t>(c) * p.v.max_pages;
  // This CTA's picks are rank, rank + S, ...; a thread looks up one of a batch.
  int pick = -1, before = -1, id = -1;
  auto look_up = [&](int base) {
    const int64_t at = (static_cast<int64_t>(base) + tid) * S + rank;
    pick = at < p.max_picks ? __ldg(picks + at) : -1;
    before = at > 0 && at < p.max_picks ? __ldg(picks + at - 1) : -1;
    id = pick >= 0 && pick < p.v.max_pages ? __ldg(table + pick) : -1;
  };
  look_up(0);
  int count = p.counts[list];
  const int L = clamped_len(p.v, c);
  const bool draft = rank == S - 1, tree = p.tree_parent != nullptr;
  if (draft && tree && tid < p.N) s_parent[tid] = p.tree_parent[static_cast<size_t>(c / p.per_seq) * p.N + tid];
  if (count < 0 || count > p.max_picks) {
    set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
    count = min(max(count, 0), p.max_picks);
  }

  WarpState<NT> st;
  st.init();
  const size_t qrow = (static_cast<size_t>(c) * p.Nq + n) * p.hq + h * p.G;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      st.q[nt][j] = nt * 8 + g < p.G ? __ldg(p.q + (qrow + nt * 8 + g) * 16 + 8 * (j >> 1) + 2 * t + (j & 1)) : make_uint4(0, 0, 0, 0);

  const int own = count > rank ? (count - rank + S - 1) / S : 0;  // picks of this CTA
  const int groups_per_page = p.v.P / 8;
  for (int base = 0; base < own; base += kSparseThreads) {
    if (base > 0) {
      __syncthreads();
      look_up(base);
    }
    const int here = min(kSparseThreads, own - base);
    if (tid < here) {
      int row = 0, valid = 0;
      if (pick >= 0 && pick > before && static_cast<int64_t>(pick) * p.v.P < L) {
        if (static_cast<unsigned>(id) < static_cast<unsigned>(p.v.num_pages)) {
          row = (id * p.v.hkv + h) * p.v.P;
          valid = min(p.v.P, L - pick * p.v.P);
        }
      }
      if (valid == 0) set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
      s_row[tid] = row;
      s_valid[tid] = valid;
    }
    __syncthreads();
    const int groups = here * groups_per_page;  // of 8 keys; a group is in one page
    for (int s = warp; 2 * s < groups; s += kSparseWarps) {
      int first[2], live[2];  // row of the group's first key, and its keys
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int grp = 2 * s + e, page = min(grp / groups_per_page, here - 1), off = (grp - page * groups_per_page) * 8;
        first[e] = s_row[page] + off;
        live[e] = grp < groups ? s_valid[page] - off : 0;
      }
      const int kr[2] = {g < live[0] ? first[0] + g : -1, g < live[1] ? first[1] + g : -1};
      const int vr[4] = {2 * t < live[0] ? first[0] + 2 * t : -1, 2 * t + 1 < live[0] ? first[0] + 2 * t + 1 : -1,
                         2 * t < live[1] ? first[1] + 2 * t : -1, 2 * t + 1 < live[1] ? first[1] + 2 * t + 1 : -1};
      st.step(p.k, p.val, kr, vr, p.qscale, g, t);
    }
  }

  if (draft) {  // the node itself and its ancestors
    const int node = p.N - p.Nq + n;
    if (tree) {
      __syncthreads();
      if (tid == 0) {
        int at = node, len = 0;
        while (at >= 0) {
          s_line[len++] = at;
          const int up = s_parent[at];
          if (up < -1 || up >= at) {
            set_error(p.v.err, KVSHOT_ERR_TREE);
            break;
          }
          at = up;
        }
        s_line_len = len;
      }
      __syncthreads();
    }
    const int line = tree ? s_line_len : node + 1;
    const int draft0 = (c * p.v.hkv + h) * p.n_max;
    auto slot = [&](int i) { return i >= line ? -1 : draft0 + (tree ? s_line[i] : i); };
    // (From the last warp down: it has the fewest of the pages' keys.)
    for (int s = kSparseWarps - 1 - warp; s * 16 < line; s += kSparseWarps) {
      const int kr[2] = {slot(s * 16 + g), slot(s * 16 + g + 8)};
      const int vr[4] = {slot(s * 16 + 2 * t), slot(s * 16 + 2 * t + 1), slot(s * 16 + 2 * t + 8), slot(s * 16 + 2 * t + 9)};
      st.step(p.dk, p.dv, kr, vr, p.qscale, g, t);
    }
  }

  // The warps' states joined, then the CTAs': reference and sum of every row, and a weighted sum of the O's.
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = st.l[nt][e];
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
      const int r = nt * 8 + 2 * t + e;
      if (g == 0) {
        s_m[warp][r] = st.m[nt][e];
        s_l[warp][r] = l;
      }
      float* dst = s_part + (warp * 8 * NT + r) * kPartStride + 16 * g;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(st.o[nt][i][e], st.o[nt][i][2 + e]);
    }
  __syncthreads();
  __shared__ float s_top[8 * NT], s_sum[8 * NT];  // of the CTA
  for (int i = tid; i < p.G * kHeadDim; i += kSparseThreads) {
    const int r = i / kHeadDim, d = i % kHeadDim;
    float top = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kSparseWarps; ++w) top = fmaxf(top, s_m[w][r]);
    float sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < kSparseWarps; ++w) {
      const float f = s_m[w][r] == -INFINITY ? 0.f : ex2(s_m[w][r] - top);
      sum += f * s_l[w][r];
      o += f * s_part[(w * 8 * NT + r) * kPartStride + d];
    }
    s_part[r * kPartStride + d] = o;
    if (d == 0) {
      s_top[r] = top;
      s_sum[r] = sum;
    }
  }
  if (S > 1) cluster_sync_all();
  else __syncthreads();
  for (int i = rank * kSparseThreads + tid; i < p.G * kHeadDim; i += S * kSparseThreads) {
    const int r = i / kHeadDim, d = i % kHeadDim;
    float m[8], top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      m[x] = x < S ? remote_float(smem_addr(&s_top[r]), x) : -INFINITY;
      top = fmaxf(top, m[x]);
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      if (x >= S) break;
      const float f = m[x] == -INFINITY ? 0.f : ex2(m[x] - top);
      sum += f * remote_float(smem_addr(&s_sum[r]), x);
      o += f * remote_float(smem_addr(s_part + r * kPartStride + d), x);
    }
    p.out[(qrow + r) * kHeadDim + d] = __float2bfloat16_rn(o / sum);
    if (d == 0) p.lse[qrow + r] = (top + log2f(sum)) * 0.6931471805599453f;
  }
  if (S > 1) cluster_sync_all();  // (another CTA may still read this one's state)
}

template <int NT>
cudaError_t launch_sparse(const SparseParams& p, int units, int S, cudaStream_t stream) {
  const size_t smem = sizeof(float) * kSparseWarps * 8 * NT * kPartStride;
  if (smem > 48 * 1024) {
    const cudaError_t e =
        cudaFuncSetAttribute(sparse_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(units * S);
  cfg.blockDim = dim3(kSparseThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sparse_kernel<NT>, p);
}

// ------------------------------------------------------------ several query rows

// Nodes of one level pick much the same pages.  Here a CTA takes up to 64 rows (nodes x q heads of the KV head) of a cache, and
// each page that any of its nodes picked once: by TMA into a ring in shared memory, from where the warps, 8 rows each, take
// those that a node of theirs picked.  A cluster shares out the pages, by their number; its CTAs' states meet in shared memory.
//   a window of pages: the nodes' picks as a bit set for each page, then the list of the pages that have any
//   a ring of stages of 32 keys in groups of 8 (2 KB: dims 0 .. 63, then 64 .. 127, 128-byte swizzled rows); one warp loads
// The tree's level of 16 x 32K tokens (12 nodes, 128 pages each, 3 to 4 nodes to a page) reads 400 MB so, and not 1.6 GB:
// 110 us, 162 with a CTA for each node.
constexpr int kSharedWarps = 8;                      // at most: 8 rows each (and one more warp, which loads)
constexpr int kWindow = 1024;                        // pages
constexpr int kStageKeys = 32;
constexpr int kStageHalf = kStageKeys * kHeadDim * 2;  // K; V is behind it
constexpr int kStageBytes = 2 * kStageHalf;
constexpr int kRingStages = 5;

struct SharedSpace {
  uint8_t ring[kRingStages * kStageBytes];           // at the end: the warps' states
  unsigned long long mask[kWindow], line[kMaxTreeNodes];  // nodes (of this block) by page; by draft slot of a tree
  unsigned long long list_mask[kWindow];
  int list_row[kWindow];                             // first row of the page in the pool, KV head included; -1: passed over
  uint16_t list_live[kWindow];                       // its tokens below the length
  uint16_t list_page[kWindow];                       // page, from the window's first
  uint64_t full[kRingStages], empty[kRingStages];
  int counts[64], parent[kMaxTreeNodes], warp_sum[kSharedWarps + 1];
  float m[64], l[64];
};
static_assert(sizeof(float) * 64 * kPartStride <= kRingStages * kStageBytes, "the states fit the ring");

struct SharedParams {
  SparseParams s;
  int nodes_per_block, log_gp;
  int box_keys;         // keys of a box: a page, or 32 keys of one
  uint32_t by_page;     // ceil(2^32 / groups of a page)
  uint32_t wait_ns;
};
struct SharedMaps {
  CUtensorMap k, v, dk, dv;
};

// Offset in a stage's K or V of 16-byte piece `piece` of key `row`.
__device__ __forceinline__ uint32_t stage_off(int row, int piece) {
  return static_cast<uint32_t>((row >> 3) * kGroupBytes + (piece >> 3) * kGroupHalfBytes + (row & 7) * 128 +
                               (((piece & 7) ^ (row & 7)) << 4));
}

// kConsumers: the most warps that multiply (two CTAs to an SM: 144 registers with 6 of them, 112 with 8).
template <int kConsumers>
__global__ void __launch_bounds__((kConsumers + 1) * 32, 2)
    sparse_shared_kernel(const __grid_constant__ SharedParams sp, const __grid_constant__ SharedMaps maps) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  SharedSpace& sm = *reinterpret_cast<SharedSpace*>(smem_raw);
  const SparseParams& p = sp.s;
  const int S = static_cast<int>(cluster_size()), rank = blockIdx.x % S;
  const int h = blockIdx.x / S % p.v.hkv, c = blockIdx.x / S / p.v.hkv;
  const int n0 = blockIdx.y * sp.nodes_per_block, nodes = min(sp.nodes_per_block, p.Nq - n0);
  const int gp = 1 << sp.log_gp, threads = blockDim.x, consumers = threads / 32 - 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int L = clamped_len(p.v, c), P = p.v.P;
  const uint64_t limit = sp.wait_ns;
  int32_t* err = p.v.err;

  if (tid == 0) {
    for (int i = 0; i < kRingStages; ++i) {
      mbar_init(smem_addr(&sm.full[i]), 1);
      mbar_init(smem_addr(&sm.empty[i]), consumers);
    }
    fence_mbar_init();
    prefetch_tensormap(&maps.k);
    prefetch_tensormap(&maps.v);
  }
  // The nodes' counts, and of a tree the lines of ancestors as bits of the draft slots.
  if (tid < nodes) {
    int count = p.counts[(static_cast<size_t>(c) * p.Nq + n0 + tid) * p.v.hkv + h];
    if (count < 0 || count > p.max_picks) {
      set_error(err, KVSHOT_ERR_DEVICE_BOUNDS);
      count = min(max(count, 0), p.max_picks);
    }
    sm.counts[tid] = count;
  }
  const bool draft = rank == S - 1, tree = p.tree_parent != nullptr;
  if (draft && tree) {
    for (int i = tid; i < p.N; i += threads) {
      sm.parent[i] = p.tree_parent[static_cast<size_t>(c / p.per_seq) * p.N + i];
      sm.line[i] = 0;
    }
    __syncthreads();
    if (tid < nodes) {
      for (int at = p.N - p.Nq + n0 + tid; at >= 0;) {
        atomicOr(&sm.line[at], 1ull << tid);
        const int up = sm.parent[at];
        if (up < -1 || up >= at) {
          set_error(err, KVSHOT_ERR_TREE);
          break;
        }
        at = up;
      }
    }
  }

  // A consumer's rows: columns 2 t, 2 t + 1 of its products, and column g's q.
  uint32_t q[8][2];
  {
    const int r = warp * 8 + g, node = r >> sp.log_gp, j = r & (gp - 1);
    const bool live = node < nodes && j < p.G;
    const uint32_t* src = reinterpret_cast<const uint32_t*>(p.q) + ((static_cast<size_t>(c) * p.Nq + n0 + node) * p.hq + h * p.G + j) * 64 + t;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      q[ks][0] = live ? __ldg(src + 8 * ks) : 0;
      q[ks][1] = live ? __ldg(src + 8 * ks + 4) : 0;
    }
  }
  // Nodes of the warp's rows: node0 and up to 7 more, of which columns 2 t and 2 t + 1 are the bits bit[0] and bit[1].
  const int node0 = warp * 8 >> sp.log_gp;
  uint32_t bit[2], tile_nodes = 0;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int node = (warp * 8 + 2 * t + e) >> sp.log_gp;
    bit[e] = node < nodes ? 1u << (node - node0) : 0;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int node = (warp * 8 + i) >> sp.log_gp;
    if (node < nodes) tile_nodes |= 1u << (node - node0);
  }
  // Offsets of this lane's rows for ldmatrix: K by pairs of pieces of a half, V transposed alike.
  uint32_t koff[4], voff[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    koff[i] = stage_off(lane & 15, 2 * i + (lane >> 4));
    voff[i] = kStageHalf + stage_off((lane & 7) + ((lane >> 4) << 3), 2 * i + ((lane >> 3) & 1));
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[i][e] = 0.f;

  // S^T = K Q^T of 16 keys from `base` on; see: the tile's nodes that see keys g and g + 8.
  auto scores = [&](uint32_t base, uint32_t see0, uint32_t see1, float (&s)[4]) {
    float d[2][4] = {};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      uint32_t a[4];
      ldmatrix_x4(base + koff[ks & 3] + (ks >> 2) * kGroupHalfBytes, a[0], a[1], a[2], a[3]);
      mma_bf16_16816(d[ks & 1], a, q[ks][0], q[ks][1]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      s[e] = ((e < 2 ? see0 : see1) & bit[e & 1]) != 0 ? (d[0][e] + d[1][e]) * p.qscale : -INFINITY;
  };
  // O^T += V^T P^T; mask: which of this lane's keys (2 t, 2 t + 1 of each group) are tokens: of others V may hold anything.
  auto values = [&](uint32_t base, uint32_t p0, uint32_t p1, bool whole, uint32_t mask0, uint32_t mask1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t a[4];
      ldmatrix_x4_trans(base + voff[i & 3] + (i >> 2) * kGroupHalfBytes, a[0], a[1], a[2], a[3]);
      if (!whole) {
        a[0] &= mask0;
        a[1] &= mask0;
        a[2] &= mask1;
        a[3] &= mask1;
      }
      mma_bf16_16816(o[i], a, p0, p1);
    }
  };
  auto raise = [&](float top0, float top1) {  // the reference, when a score is more than 2^8 above it
    if (!__any_sync(0xffffffffu, top0 > m[0] + 8.f || top1 > m[1] + 8.f)) return;
    float top[2] = {top0, top1};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], x));
      const float now = fmaxf(m[e], top[e]);
      const float f = now == -INFINITY ? 1.f : ex2(m[e] - now);
      m[e] = now;
      l[e] *= f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[i][e] *= f;
        o[i][2 + e] *= f;
      }
    }
  };
  auto weigh = [&](float (&s)[4], uint32_t* p0, uint32_t* p1) {
    const float m0 = m[0] == -INFINITY ? 0.f : m[0], m1 = m[1] == -INFINITY ? 0.f : m[1];
    s[0] = ex2(s[0] - m0);
    s[1] = ex2(s[1] - m1);
    s[2] = ex2(s[2] - m0);
    s[3] = ex2(s[3] - m1);
    l[0] += s[0] + s[2];
    l[1] += s[1] + s[3];
    *p0 = transpose8x8(pack_bf16x2(s[0], s[1]));
    *p1 = transpose8x8(pack_bf16x2(s[2], s[3]));
  };
  // A stage.  Lane x < 4 knows of group x its tokens (none below 1, 8 or more: all); see[i]: the tile's nodes that see key g of
  // group i.
  auto consume = [&](uint32_t base, int lane_live, const uint32_t (&see)[4]) {
    const bool both0 = __any_sync(0xffffffffu, ((see[0] | see[1]) & tile_nodes) != 0);
    const bool both1 = __any_sync(0xffffffffu, ((see[2] | see[3]) & tile_nodes) != 0);
    if (!both0 && !both1) return;
    const bool whole = __all_sync(0xffffffffu, lane >= 4 || lane_live >= 8);
    uint32_t mask[4] = {};
    if (!whole)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int live = __shfl_sync(0xffffffffu, lane_live, i);
        mask[i] = (2 * t < live ? 0xffffu : 0u) | (2 * t + 1 < live ? 0xffff0000u : 0u);
      }
    constexpr uint32_t kSecond = 2 * kGroupBytes;  // the stage's keys 16 .. 31
    uint32_t p0, p1;
    if (both0 && both1) {
      float s[4], s2[4];
      scores(base, see[0], see[1], s);
      scores(base + kSecond, see[2], see[3], s2);
      raise(max3(fmaxf(s[0], s[2]), s2[0], s2[2]), max3(fmaxf(s[1], s[3]), s2[1], s2[3]));
      uint32_t p2, p3;
      weigh(s, &p0, &p1);
      weigh(s2, &p2, &p3);
      values(base, p0, p1, whole, mask[0], mask[1]);
      values(base + kSecond, p2, p3, whole, mask[2], mask[3]);
    } else {
      float s[4];
      const uint32_t from = both0 ? base : base + kSecond;
      scores(from, both0 ? see[0] : see[2], both0 ? see[1] : see[3], s);
      raise(fmaxf(s[0], s[2]), fmaxf(s[1], s[3]));
      weigh(s, &p0, &p1);
      values(from, p0, p1, whole, both0 ? mask[0] : mask[2], both0 ? mask[1] : mask[3]);
    }
  };

  uint32_t filled = 0;  // stages so far, the same in all warps
  bool ok = true;
  // `stages` stages through the ring: load(stage, base, bar) issues a stage's copies and returns its bytes (the whole loading warp;
  // it announces them first), use(stage, base).
  auto stream = [&](int stages, auto load, auto use) {
    for (int st = 0; ok && st < stages; ++st, ++filled) {
      const uint32_t slot = filled % kRingStages, round = filled / kRingStages;
      const uint32_t base = smem_addr(sm.ring) + slot * kStageBytes;
      if (warp == consumers) {
        if (round > 0) ok = __all_sync(0xffffffffu, wait(smem_addr(&sm.empty[slot]), (round - 1) & 1, err, limit));
        if (!ok) break;
        load(st, base, smem_addr(&sm.full[slot]));
      } else {
        ok = __all_sync(0xffffffffu, wait(smem_addr(&sm.full[slot]), round & 1, err, limit));
        if (!ok) break;
        use(st, base);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&sm.empty[slot]));
      }
    }
  };

  const int pages = (L + P - 1) / P, groups_per_page = P / 8;
  const int page0 = static_cast<int>(static_cast<int64_t>(pages) * rank / S);
  const int page1 = static_cast<int>(static_cast<int64_t>(pages) * (rank + 1) / S);
  const int32_t* picks = p.picks + ((static_cast<size_t>(c) * p.Nq + n0) * p.v.hkv + h) * p.max_picks;
  const size_t list_stride = static_cast<size_t>(p.v.hkv) * p.max_picks;
  // (Every CTA of the cluster has a window at least, in which it checks all picks.)
  for (int w0 = page0; w0 < page1 || w0 == page0; w0 += kWindow) {
    const int w1 = min(page1, w0 + kWindow);
    __syncthreads();
    for (int i = tid; i < w1 - w0; i += threads) sm.mask[i] = 0;
    __syncthreads();
    const int total = nodes * p.max_picks;
    for (int i0 = tid; i0 < total; i0 += 8 * threads) {
      int pick[8], before[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int i = i0 + x * threads, node = i / p.max_picks, at = i - node * p.max_picks;
        const bool live = i < total && at < sm.counts[node];
        pick[x] = live ? __ldg(picks + node * list_stride + at) : -2;
        before[x] = live && at > 0 ? __ldg(picks + node * list_stride + at - 1) : -1;
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int i = i0 + x * threads, node = i / p.max_picks, at = i - node * p.max_picks;
        if (i >= total || at >= sm.counts[node]) continue;
        if (pick[x] >= w0 && pick[x] < w1 && pick[x] > before[x]) atomicOr(&sm.mask[pick[x] - w0], 1ull << node);
        else if (pick[x] < 0 || pick[x] >= pages || pick[x] <= before[x]) set_error(err, KVSHOT_ERR_DEVICE_BOUNDS);
      }
    }
    __syncthreads();
    // The pages that some node picked, in order.
    const int per = (w1 - w0 + threads - 1) / threads;
    int mine = 0;
    for (int i = tid * per; i < min(w1 - w0, tid * per + per); ++i) mine += sm.mask[i] != 0;
    int scan = mine;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, scan, x);
      if (lane >= x) scan += y;
    }
    if (lane == 31) sm.warp_sum[warp] = scan;
    __syncthreads();
    int at = scan - mine, listed = 0;
    for (int x = 0; x <= consumers; ++x) {
      if (x < warp) at += sm.warp_sum[x];
      listed += sm.warp_sum[x];
    }
    for (int i = tid * per; i < min(w1 - w0, tid * per + per); ++i)
      if (sm.mask[i] != 0) {
        sm.list_page[at] = static_cast<uint16_t>(i);
        sm.list_mask[at++] = sm.mask[i];
      }
    __syncthreads();
    for (int i = tid; i < listed; i += threads) {
      const int page = w0 + sm.list_page[i], id = page_id(p.v, c, page);
      sm.list_row[i] = id >= 0 ? (id * p.v.hkv + h) * P : -1;
      sm.list_live[i] = static_cast<uint16_t>(id >= 0 ? min(P, L - page * P) : 0);
    }
    __syncthreads();
    // Group i (8 keys of one page): the page's place in the list, and its first key there.
    const uint32_t groups = listed * groups_per_page;
    auto page_of = [&](uint32_t i) { return groups_per_page == 1 ? i : __umulhi(i, sp.by_page); };
    const int box_groups = sp.box_keys / 8, boxes = kStageKeys / sp.box_keys;
    stream(static_cast<int>(groups * 8 + kStageKeys - 1) / kStageKeys,
           [&](int st, uint32_t base, uint32_t bar) {
             const uint32_t i = st * (kStageKeys / 8) + lane * box_groups, page = page_of(min(i, groups));
             int row = -1;
             if (lane < boxes && i < groups && sm.list_row[page] >= 0) row = sm.list_row[page] + (i - page * groups_per_page) * 8;
             const int live = __popc(__ballot_sync(0xffffffffu, row >= 0));
             if (lane == 0) mbar_arrive_expect_tx(bar, live * sp.box_keys * 512);
             __syncwarp();
             if (row >= 0) {
               const uint32_t dst = base + lane * sp.box_keys * 256;
               tma_load_4d(dst, &maps.k, 0, 0, 0, row >> 3, bar);
               tma_load_4d(dst + kStageHalf, &maps.v, 0, 0, 0, row >> 3, bar);
             }
           },
           [&](int st, uint32_t base) {
             int live = 0;
             uint32_t nodes_of = 0;
             const uint32_t i = st * (kStageKeys / 8) + lane;
             if (lane < 4 && i < groups) {
               const uint32_t page = page_of(i);
               live = sm.list_live[page] - static_cast<int>(i - page * groups_per_page) * 8;
               nodes_of = static_cast<uint32_t>(sm.list_mask[page] >> node0) & 0xffu;
             }
             uint32_t see[4];
#pragma unroll
             for (int x = 0; x < 4; ++x) {
               const uint32_t both = __shfl_sync(0xffffffffu, nodes_of | static_cast<uint32_t>(min(max(live, 0), 8)) << 8, x);
               see[x] = g < static_cast<int>(both >> 8) ? both & 0xffu : 0u;
             }
             consume(base, live, see);
           });
  }

  if (draft) {  // the nodes themselves and their ancestors
    const int first_row = (c * p.v.hkv + h) * p.n_max, first_node = p.N - p.Nq + n0;
    const int slots = min(p.N, first_node + nodes);  // (no node sees a later one)
    stream((slots + kStageKeys - 1) / kStageKeys,
           [&](int st, uint32_t base, uint32_t bar) {
             const int slot = st * kStageKeys + lane * 8;
             const bool live = lane < kStageKeys / 8 && slot < slots;
             const int boxes = __popc(__ballot_sync(0xffffffffu, live));
             if (lane == 0) mbar_arrive_expect_tx(bar, boxes * 2 * kGroupBytes);
             __syncwarp();
             if (live) {
               const uint32_t dst = base + lane * kGroupBytes;
               tma_load_3d_plain(dst, &maps.dk, 0, first_row + slot, 0, bar);
               tma_load_3d_plain(dst + kStageHalf, &maps.dv, 0, first_row + slot, 0, bar);
             }
           },
           [&](int st, uint32_t base) {
             uint32_t see[4];
#pragma unroll
             for (int x = 0; x < 4; ++x) {
               const int slot = st * kStageKeys + 8 * x + g;
               // A chain's node sees the slots up to its own: nodes from slot - first_node on see this one.
               const unsigned long long nodes_of = slot >= slots ? 0ull : tree ? sm.line[slot] : ~0ull << max(0, slot - first_node);
               see[x] = static_cast<uint32_t>(nodes_of >> node0) & 0xffu;
             }
             consume(base, slots - st * kStageKeys - 8 * lane, see);
           });
  }
  if (warp == consumers)  // no copy is in flight when the ring becomes the states' place, or the CTA ends
    for (uint32_t i = filled > kRingStages ? filled - kRingStages : 0; i < filled; ++i)
      mbar_wait(smem_addr(&sm.full[i % kRingStages]), (i / kRingStages) & 1, err);
  __syncthreads();

  // The CTAs' states joined.
  float* part = reinterpret_cast<float*>(sm.ring);  // [64 rows][kPartStride]
  if (warp < consumers) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float sum = l[e];
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      const int r = warp * 8 + 2 * t + e;
      if (g == 0) {
        sm.m[r] = m[e];
        sm.l[r] = sum;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        part[r * kPartStride + 16 * i + g] = o[i][e];
        part[r * kPartStride + 16 * i + g + 8] = o[i][2 + e];
      }
    }
  }
  if (S > 1) cluster_sync_all();
  else __syncthreads();
  const int rows = nodes << sp.log_gp;
  for (int i = rank * threads + tid; i < rows * kHeadDim; i += S * threads) {
    const int r = i / kHeadDim, d = i % kHeadDim, j = r & (gp - 1);
    if (j >= p.G) continue;
    float top = -INFINITY;
    for (int x = 0; x < S; ++x) top = fmaxf(top, remote_float(smem_addr(&sm.m[r]), x));
    float sum = 0.f, out = 0.f;
    for (int x = 0; x < S; ++x) {
      const float mx = remote_float(smem_addr(&sm.m[r]), x);
      const float f = mx == -INFINITY ? 0.f : ex2(mx - top);
      sum += f * remote_float(smem_addr(&sm.l[r]), x);
      out += f * remote_float(smem_addr(part + r * kPartStride + d), x);
    }
    const size_t row = (static_cast<size_t>(c) * p.Nq + n0 + (r >> sp.log_gp)) * p.hq + h * p.G + j;
    p.out[row * kHeadDim + d] = __float2bfloat16_rn(out / sum);
    if (d == 0) p.lse[row] = (top + log2f(sum)) * 0.6931471805599453f;
  }
  if (S > 1) cluster_sync_all();  // (another CTA may still read this one's state)
}

cudaError_t launch_shared(const SparseParams& s, int caches, int S, uint32_t wait_ns, cudaStream_t stream) {
  SharedParams p;
  p.s = s;
  p.log_gp = 0;
  while ((1 << p.log_gp) < s.G) ++p.log_gp;
  const int most = 64 >> p.log_gp, blocks = (s.Nq + most - 1) / most;
  p.nodes_per_block = (s.Nq + blocks - 1) / blocks;
  p.box_keys = std::min(s.v.P, kStageKeys);
  const uint32_t groups = s.v.P / 8;
  p.by_page = groups > 1 ? static_cast<uint32_t>(((uint64_t{1} << 32) + groups - 1) / groups) : 0;
  p.wait_ns = wait_ns;
  SharedMaps maps;
  const uint64_t rows = static_cast<uint64_t>(s.v.num_pages) * s.v.hkv * s.v.P;
  const uint64_t drows = static_cast<uint64_t>(caches) * s.v.hkv * s.n_max;
  if (!map_groups(&maps.k, s.k, rows, p.box_keys / 8) || !map_groups(&maps.v, s.val, rows, p.box_keys / 8) ||
      !map_any_8(&maps.dk, s.dk, drows) || !map_any_8(&maps.dv, s.dv, drows))
    return cudaErrorInvalidValue;
  const int warps = ((p.nodes_per_block << p.log_gp) + 7) / 8 + 1;
  auto* kernel = warps <= 7 ? sparse_shared_kernel<6> : sparse_shared_kernel<kSharedWarps>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SharedSpace));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(caches * s.v.hkv * S, blocks);
  cfg.blockDim = dim3(warps * 32);
  cfg.dynamicSmemBytes = sizeof(SharedSpace);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p, maps);
}

constexpr size_t kSparseWorkspace = 256;

kvshot_status check_sparse(const kvshot_attn_desc* d, int max_picks) {
  if (kvshot_status st = check_partial(d, true)) return st;
  if (max_picks < 1) return KVSHOT_ERR_SHAPE;
  if (max_picks > 1 << 24) return KVSHOT_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(d->num_caches) * d->hkv * d->n_query >= (int64_t{1} << 27)) return KVSHOT_ERR_UNSUPPORTED;
  return KVSHOT_OK;
}

}  // namespace
}  // namespace kvshot

using namespace kvshot;

extern "C" size_t kvshot_draft_attn_sparse_workspace_size(const kvshot_attn_desc* d, int32_t max_picks) {
  return check_sparse(d, max_picks) == KVSHOT_OK ? kSparseWorkspace : 0;
}

extern "C" kvshot_status kvshot_draft_attn_sparse(const kvshot_attn_desc* d, const void* q, const void* target_k,
                                                  const void* target_v, const int32_t* page_table,
                                                  const int32_t* seq_lens, const int32_t* picks, const int32_t* counts,
                                                  int32_t max_picks, const void* draft_k, const void* draft_v,
                                                  const int32_t* tree_parent, void* out, float* lse,
                                                  kvshot_stream_t stream) {
  if (kvshot_status st = check_sparse(d, max_picks)) return st;
  if (d->n_query == 0) return KVSHOT_OK;
  const bool tree = (d->flags & KVSHOT_TREE) != 0;
  if (!q || !target_k || !target_v || !page_table || !seq_lens || !picks || !counts || !draft_k || !draft_v || !out || !lse ||
      (tree && !tree_parent))
    return KVSHOT_ERR_NULL;
  for (const void* x : {q, static_cast<const void*>(out)})
    if (!aligned(x, 16)) return KVSHOT_ERR_ALIGN;
  for (const void* x : {target_k, target_v, draft_k, draft_v})  // (read 32 bytes at a time)
    if (!aligned(x, 32)) return KVSHOT_ERR_ALIGN;
  for (const void* x : {static_cast<const void*>(page_table), static_cast<const void*>(seq_lens),
                        static_cast<const void*>(picks), static_cast<const void*>(counts),
                        static_cast<const void*>(tree ? tree_parent : nullptr), static_cast<const void*>(lse)})
    if (!aligned(x, 4)) return KVSHOT_ERR_ALIGN;
  if (d->workspace == nullptr || !aligned(d->workspace, 256) || d->workspace_bytes < kSparseWorkspace)
    return KVSHOT_ERR_WORKSPACE;
  SparseParams p;
  p.v = cache_view(d, page_table, seq_lens);
  p.q = static_cast<const uint4*>(q);
  p.k = static_cast<const uint4*>(target_k);
  p.val = static_cast<const uint4*>(target_v);
  p.dk = static_cast<const uint4*>(draft_k);
  p.dv = static_cast<const uint4*>(draft_v);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.picks = picks;
  p.counts = counts;
  p.tree_parent = tree ? tree_parent : nullptr;
  p.per_seq = d->num_caches / d->num_seqs;
  p.hq = d->hq;
  p.G = d->hq / d->hkv;
  p.Nq = d->n_query;
  p.N = d->n_nodes;
  p.n_max = d->n_max;
  p.max_picks = max_picks;
  p.qscale = score_scale(d) * 1.4426950408889634f;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  // Pages are shared between nodes from 32 rows on, and where that leaves the SMs enough to do (us with a CTA for each node
  // against shared; 16 caches of 20K to 32K tokens and 128 pages a node, 48 rows: 162, 110; 8 rows: 44, 56; 256 rows and 64
  // pages: 403, 347; 16 caches of 4K tokens and 32 pages, 48 rows: 59, 45; one of 8K and 64 pages, 256 rows: 33, 47).  Two CTAs
  // of a cluster fill the SMs' two places, and more are slower.
  int log_gp = 0;
  while ((1 << log_gp) < p.G) ++log_gp;
  const int64_t rows = static_cast<int64_t>(p.Nq) << log_gp, shared = int64_t{d->num_caches} * d->hkv * ((rows + 63) / 64);
  if (rows >= 32 && 3 * shared >= 2 * sm_count() && rows < 64 * 65535) {
    const uint32_t wait_ns = d->wait_limit_ns != 0 ? d->wait_limit_ns : static_cast<uint32_t>(kWaitLimitNs);
    const int S = shared < 2 * sm_count() ? 2 : 1;
    return launch_shared(p, d->num_caches, S, wait_ns, s) == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
  }
  const int64_t steps = static_cast<int64_t>(max_picks) * d->page_size / 16;
  const int units = d->num_caches * d->hkv * d->n_query;
  // CTAs per unit: until the SMs have two each, while a warp still has 16 keys.
  int S = 1;
  while (S < 8 && static_cast<int64_t>(units) * S < 2 * sm_count() && steps > 2 * S * kSparseWarps) S *= 2;
  const cudaError_t e = p.G <= 8    ? launch_sparse<1>(p, units, S, s)
                        : p.G <= 16 ? launch_sparse<2>(p, units, S, s)
                                    : launch_sparse<4>(p, units, S, s);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
