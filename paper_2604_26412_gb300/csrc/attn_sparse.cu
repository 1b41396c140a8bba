// attn_sparse.cu -- draft attention over the pages picked for each query row and KV head, and the draft K/V.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "kvshot_partial.cuh"
#include "kvshot_tcgen05.cuh"

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
      // (key, row pair) -> (row, key pair): the B operand of the second product.  bf16, as the draft attention has it: V is bf16
      // and a product's operands have one type.  A weight is off by 2^-8 of itself at most; the sums are of what it was before.
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
// each page that any of its nodes picked once, 128 keys to a tile, on tcgen05: keys are the M rows of S^T = K Q^T, so that a
// thread has one key and knows with one 64-bit word which columns, rows of q, picked its page; dims are the M rows of
// O^T += V^T P^T, whose accumulator never leaves tensor memory.  The columns' sums stay in the threads' registers, each its own
// keys' share, to the end.  A cluster's CTAs take its pages in turn, by their number; their states meet in shared memory.
//   a window of pages: the nodes' picks as a set of columns for each page, then the list of the pages that have any
//   warps 0..7  softmax, a key to a thread: the first four of columns 0 to 31, the others of the rest
//   warp 8      TMA;  warp 9: MMA, and the owner of tensor memory
// Two CTAs to an SM, each with one K and one V tile: while one waits for its bytes the other multiplies.
// The tree's level of 16 x 32K tokens (12 nodes, 128 pages each, 3 to 4 nodes to a page) reads 400 MB so, and not 1.6 GB:
// 95 us, 162 with a CTA for each node, 110 with mma.sync and eight rows to a warp (five times the instructions).  Of the 95 the
// list of pages takes 8, the tiles 50 to 75 (6.5 TB/s in all; the 104 of 152 SMs that have two of the 256 CTAs are the slower
// ones), the wait for the cluster's other CTA and the join 5.  Four softmax warps of 64 columns each in turn were 112, a join
// by single floats 15 us longer, references that start at the first tile's greatest scores 1.5 us.
constexpr int kTileKeys128 = 128;
constexpr int kTileBytes128 = kTileKeys128 * kHeadDim * 2;  // of K, and of V
constexpr int kColumns = 64;
constexpr int kWindow = 1024;                      // pages
constexpr int kSharedThreads = 10 * 32;
constexpr int kSoftmaxThreads = 128;               // of 32 columns
constexpr int kPagesEach = (kWindow + kSharedThreads - 1) / kSharedThreads, kPicksEach = 6;
constexpr int kQEach = (kColumns * 16 + kSharedThreads - 1) / kSharedThreads;
constexpr int kSharedTmem = 128;                   // columns: O 64, S 64
constexpr int kTmemS = 64;

struct SharedSpace {
  uint8_t k[kTileBytes128], v[kTileBytes128];      // in groups of 8 keys; at the end: the CTA's state
  uint8_t q[kColumns * 256], p[kTileKeys128 * 128];
  uint32_t mask[kWindow][2];                       // columns by page of the window; then those of the pages that have any,
  int list_row[kWindow];                           // and such a page's first row in the pool, KV head included; -1: passed over
  unsigned long long line[kMaxTreeNodes];          // columns by draft slot of a tree
  float neg_ref[kColumns], factor[kColumns], m[kColumns], l[kColumns], part_l[4][kColumns];
  int top[8][32];
  uint64_t kfull, vfull, sdone, pfull, pvdone, done;
  int counts[kColumns], parent[kMaxTreeNodes], warp_sum[kSharedThreads / 32], ends;  // ends: the cache's last page is listed
  uint32_t tmem;
};
static_assert(sizeof(float) * kColumns * kPartStride <= 2 * kTileBytes128, "the state fits the tiles' place");
static_assert(2 * (sizeof(SharedSpace) + 1024) <= 228 * 1024, "two CTAs to an SM");

struct SharedParams {
  SparseParams s;
  int nodes_per_block, cols;  // cols: the block's rows rounded up to 16
  int box_keys;               // keys of a box: a page, or 64 keys of one
  uint32_t by_page;           // ceil(2^32 / groups of a page)
  uint32_t wait_ns;
};
struct SharedMaps {
  CUtensorMap k, v, dk, dv;
};

// Whether x holds in any of the softmax threads of one half of the columns: one barrier of theirs.
__device__ __forceinline__ bool any_softmax(int barrier, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred in, out;\n\tsetp.ne.u32 in, %1, 0;\n\tbar.red.or.pred out, %3, %2, in;\n\tselp.u32 %0, 1, 0, out;\n\t}"
      : "=r"(r) : "r"(static_cast<uint32_t>(x)), "n"(kSoftmaxThreads), "r"(barrier) : "memory");
  return r != 0;
}
// Floats as integers of the same order.
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i >= 0 ? i : i ^ 0x7fffffff;
}
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i >= 0 ? i : i ^ 0x7fffffff); }

__device__ __forceinline__ void wait_columns(uint32_t (&v)[32]) {  // nothing computed from v moves before the wait
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                 "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                 "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                 "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}

__global__ void __launch_bounds__(kSharedThreads, 2)
    sparse_shared_kernel(const __grid_constant__ SharedParams sp, const __grid_constant__ SharedMaps maps) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  SharedSpace& sm = *reinterpret_cast<SharedSpace*>(smem_raw);
  const SparseParams& p = sp.s;
  const int S = static_cast<int>(cluster_size()), rank = blockIdx.x % S;
  const int h = blockIdx.x / S % p.v.hkv, c = blockIdx.x / S / p.v.hkv;
  const int n0 = blockIdx.y * sp.nodes_per_block, nodes = min(sp.nodes_per_block, p.Nq - n0), rows = nodes * p.G;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int L = clamped_len(p.v, c), P = p.v.P;
  const uint64_t limit = sp.wait_ns;
  int32_t* err = p.v.err;
  if ((smem_addr(smem_raw) & 1023u) != 0) {  // (the swizzled tiles' layout counts on it; dynamic shared memory is, alone)
    set_error(err, KVSHOT_ERR_CUDA);
    return;
  }

  if (tid == 0) {
    mbar_init(smem_addr(&sm.kfull), 1);
    mbar_init(smem_addr(&sm.vfull), 1);
    mbar_init(smem_addr(&sm.sdone), 1);
    mbar_init(smem_addr(&sm.pfull), sp.cols > 32 ? 8 : 4);
    mbar_init(smem_addr(&sm.pvdone), 1);
    mbar_init(smem_addr(&sm.done), 1);
    fence_mbar_init();
    prefetch_tensormap(&maps.k);
    prefetch_tensormap(&maps.v);
  }
  if (warp == 9) {
    tc::tmem_alloc(smem_addr(&sm.tmem), kSharedTmem);
    tc::tmem_relinquish();
  }
  const int pages = (L + P - 1) / P, groups_per_page = P / 8, total = nodes * p.max_picks;
  const int own = (pages - rank + S - 1) / S;  // pages of this CTA: rank, rank + S, ... (what is picked tends to be close together)
  const int32_t* picks = p.picks + ((static_cast<size_t>(c) * p.Nq + n0) * p.v.hkv + h) * p.max_picks;
  const size_t list_stride = static_cast<size_t>(p.v.hkv) * p.max_picks;
  // A window's page ids, consecutive ones to a thread, and the first of the picks: on their way together.
  int pick[kPicksEach], before[kPicksEach], id[kPagesEach];
  auto fetch_picks = [&](int i0) {
#pragma unroll
    for (int x = 0; x < kPicksEach; ++x) {
      const int i = i0 + x * kSharedThreads, node = i / p.max_picks, at = i - node * p.max_picks;
      pick[x] = i < total ? __ldg(picks + node * list_stride + at) : -2;
      before[x] = i < total && at > 0 ? __ldg(picks + node * list_stride + at - 1) : -1;
    }
  };
  auto fetch = [&](int w0) {
#pragma unroll
    for (int x = 0; x < kPagesEach; ++x) {
      const int at = w0 + tid * kPagesEach + x, page = at * S + rank;
      id[x] = at >= own ? -1 : p.v.page_table == nullptr ? c : __ldg(p.v.page_table + static_cast<size_t>(c) * p.v.max_pages + page);
    }
    fetch_picks(tid);
  };
  fetch(0);
  // The nodes' counts, and of a tree the lines of ancestors as columns of the draft slots.
  const unsigned long long node_columns = (1ull << p.G) - 1;  // of node 0
  const unsigned long long all_columns = rows < 64 ? (1ull << rows) - 1 : ~0ull;
  if (tid >= rows && tid < kColumns) sm.neg_ref[tid] = INFINITY;  // (no row, and no key that it sees)
  // q as the B operand: rows of 64 dims, 128-byte swizzled, the first half of the dims of all rows, then the second.
  int count = tid < nodes ? __ldg(p.counts + (static_cast<size_t>(c) * p.Nq + n0 + tid) * p.v.hkv + h) : 0;
  // A row's first reference is its score for the node itself, which every row sees: a sum then cannot vanish.
  uint4 qx[kQEach], self[kQEach];
#pragma unroll
  for (int x = 0; x < kQEach; ++x) {
    const int i = tid + x * kSharedThreads, r = min(i / 16, rows - 1), node = r / p.G;
    qx[x] = __ldg(p.q + ((static_cast<size_t>(c) * p.Nq + n0 + node) * p.hq + h * p.G + (r - node * p.G)) * 16 + i % 16);
    self[x] = __ldg(p.dk + (static_cast<size_t>(c * p.v.hkv + h) * p.n_max + p.N - p.Nq + n0 + node) * 16 + i % 16);
  }
  if (tid < nodes) {
    if (count < 0 || count > p.max_picks) {
      set_error(err, KVSHOT_ERR_DEVICE_BOUNDS);
      count = min(max(count, 0), p.max_picks);
    }
    sm.counts[tid] = count;
  }
#pragma unroll
  for (int x = 0; x < kQEach; ++x) {
    const int i = tid + x * kSharedThreads, r = i / 16, piece = i % 16;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t a = word(qx[x], e), b = word(self[x], e);
      s = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), s);
      s = fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), s);
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (piece == 0 && r < rows) sm.neg_ref[r] = fminf(-s * p.qscale, FLT_MAX);  // (finite: a score of -inf less itself is no number)
    if (r >= rows) qx[x] = make_uint4(0, 0, 0, 0);
    if (r < sp.cols) *reinterpret_cast<uint4*>(sm.q + (piece >> 3) * (sp.cols * 128) + r * 128 + (((piece & 7) ^ (r & 7)) << 4)) = qx[x];
  }
  fence_proxy_async_smem();
  const bool draft = rank == S - 1, tree = p.tree_parent != nullptr;
  if (draft && tree) {
    for (int i = tid; i < p.N; i += kSharedThreads) {
      sm.parent[i] = p.tree_parent[static_cast<size_t>(c / p.per_seq) * p.N + i];
      sm.line[i] = 0;
    }
    __syncthreads();
    if (tid < nodes) {
      for (int at = p.N - p.Nq + n0 + tid; at >= 0;) {
        atomicOr(&sm.line[at], node_columns << (tid * p.G));
        const int up = sm.parent[at];
        if (up < -1 || up >= at) {
          set_error(err, KVSHOT_ERR_TREE);
          break;
        }
        at = up;
      }
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sm.tmem, quarter = static_cast<uint32_t>(warp & 3) << 21;

  const int half = warp >> 2;  // of the columns, in the softmax warps
  float2 sums[16] = {};        // of the softmax threads: their keys' shares of the columns'
  int done = 0;  // tiles so far, the same in all warps while nothing fails
  int k_issued = 0, v_issued = 0;
  bool ok = true;
  // `tiles` tiles through the two products.  load(tile, kdst, vdst, kbar or vbar, which) issues a tile's copies (the whole loading
  // warp, which announces their bytes first); columns(tile, key, half, &live) which of the half's
  // columns see this key, and whether it is a token that any column of either half sees.
  auto stream = [&](int tiles, auto load, auto columns) {
    if (warp == 8) {
      for (int t = 0; ok && t < tiles; ++t, ++done) {
        if (done > 0) ok = __all_sync(0xffffffffu, wait(smem_addr(&sm.sdone), (done - 1) & 1, err, limit));
        if (!ok) break;
        load(t, false, smem_addr(sm.k), smem_addr(&sm.kfull));
        ++k_issued;
        if (done > 0) ok = __all_sync(0xffffffffu, wait(smem_addr(&sm.pvdone), (done - 1) & 1, err, limit));
        if (!ok) break;
        load(t, true, smem_addr(sm.v), smem_addr(&sm.vfull));
        ++v_issued;
      }
    } else if (warp == 9) {
      const uint32_t idesc_s = tc::idesc_bf16(128, sp.cols, false);
      const uint32_t idesc_o = tc::idesc_bf16(128, sp.cols, true) | 1u << 15;  // V^T: A is MN-major too
      const uint32_t k = smem_addr(sm.k), v = smem_addr(sm.v), q = smem_addr(sm.q), pb = smem_addr(sm.p);
      for (int t = 0; ok && t < tiles; ++t, ++done) {
        ok = __all_sync(0xffffffffu, wait(smem_addr(&sm.kfull), done & 1, err, limit));
        if (!ok) break;
        tc::tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
          tc::tc_mma_elect(tmem + kTmemS, tc::smem_desc_sw128(k + (ks >> 2) * kGroupHalfBytes + (ks & 3) * 32, 16, kGroupBytes),
                           tc::smem_desc_sw128(q + (ks >> 2) * (sp.cols * 128) + (ks & 3) * 32, 16, 1024), idesc_s, ks > 0);
        tc::tc_commit_elect(smem_addr(&sm.sdone));
        ok = wait(smem_addr(&sm.vfull), done & 1, err, limit);
        ok = ok && wait(smem_addr(&sm.pfull), done & 1, err, limit);  // (S has been read by then)
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc::tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)  // 16 keys: two groups
          tc::tc_mma_elect(tmem, tc::smem_desc_sw128(v + ks * 2 * kGroupBytes, kGroupHalfBytes, kGroupBytes),
                           tc::smem_desc_sw128(pb + ks * 2048, 16, 1024), idesc_o, done > 0 || ks > 0);
        tc::tc_commit_elect(smem_addr(&sm.pvdone));
      }
    } else {
      const uint32_t s_at = tmem + quarter + kTmemS + 32 * half;
      const int barrier = 1 + half, key = tid & 127;
      float* neg_ref = sm.neg_ref + 32 * half;
      float* factor = sm.factor + 32 * half;
      if (32 * half >= sp.cols) {  // nothing to do
        done += tiles;
        tiles = 0;
      }
      for (int t = 0; ok && t < tiles; ++t, ++done) {
        bool live;
        const uint32_t see = columns(t, key, half, &live);
        ok = wait(smem_addr(&sm.sdone), done & 1, err, limit);
        if (done > 0) ok = ok && wait(smem_addr(&sm.pvdone), (done - 1) & 1, err, limit);  // (P's place is free, O at rest)
        if (!live && ok && half == 0) {
          // V of what no column sees may hold anything, and a NaN times P's 0 is one: zeros.
          ok = wait(smem_addr(&sm.vfull), done & 1, err, limit);
          uint4* row = reinterpret_cast<uint4*>(sm.v + (key >> 3) * kGroupBytes + (key & 7) * 128);
#pragma unroll
          for (int i = 0; i < 8; ++i) row[i] = row[i + kGroupHalfBytes / 16] = make_uint4(0, 0, 0, 0);
        }
        __syncwarp();
        tc::tc_fence_after();
        uint32_t x[32];
        float top = -INFINITY;
        auto refer = [&] {  // scores less the reference, where the key is seen
          tc::tmem_ld32(s_at, x);
          wait_columns(x);
          const float2 qs = make_float2(p.qscale, p.qscale);
          top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 r = *reinterpret_cast<const float4*>(neg_ref + i);
            const float2 a = fma2(make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), qs, make_float2(r.x, r.y));
            const float2 b = fma2(make_float2(__uint_as_float(x[i + 2]), __uint_as_float(x[i + 3])), qs, make_float2(r.z, r.w));
            const float y0 = see >> i & 1 ? a.x : -INFINITY, y1 = see >> (i + 1) & 1 ? a.y : -INFINITY;
            const float y2 = see >> (i + 2) & 1 ? b.x : -INFINITY, y3 = see >> (i + 3) & 1 ? b.y : -INFINITY;
            top = max3(top, y0, y1);
            top = max3(top, y2, y3);
            x[i] = __float_as_uint(y0);
            x[i + 1] = __float_as_uint(y1);
            x[i + 2] = __float_as_uint(y2);
            x[i + 3] = __float_as_uint(y3);
          }
        };
        // References move only when a score is more than 2^32 above its column's: P and the sums stay in range.
        bool moved = false;
        for (;;) {
          refer();
          if (moved || !any_softmax(barrier, !ok || top > 32.f)) break;
          if (any_softmax(barrier, !ok)) {
            ok = false;
            break;
          }
          moved = true;
          tc::tmem_ld32(s_at, x);
          wait_columns(x);
          int mine = 0;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const int best = __reduce_max_sync(0xffffffffu, ordered(see >> i & 1 ? __uint_as_float(x[i]) * p.qscale : -INFINITY));
            if (lane == i) mine = best;
          }
          sm.top[warp][lane] = mine;
          named_barrier_sync(barrier, kSoftmaxThreads);
          if (key < 32) {
            const int(*tops)[32] = sm.top + 4 * half;
            const float best = unordered(max(max(tops[0][key], tops[1][key]), max(tops[2][key], tops[3][key])));
            const float old = -neg_ref[key], now = fmaxf(old, best);
            factor[key] = now == -INFINITY ? 1.f : ex2(old - now);
            neg_ref[key] = -now;
          }
          named_barrier_sync(barrier, kSoftmaxThreads);
          if (done > 0) {
            tc::tmem_ld32(tmem + quarter + 32 * half, x);
            wait_columns(x);
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * factor[i]);
            tc::tmem_st32(tmem + quarter + 32 * half, x);
            tc::tmem_wait_st();
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            sums[i].x *= factor[2 * i];
            sums[i].y *= factor[2 * i + 1];
          }
        }
        if (!ok) break;
        // P, rounded to bf16 (2^-8 of a weight at most) as the second product takes it beside a bf16 V; the sums are of what it
        // was before.
        uint4* prow = reinterpret_cast<uint4*>(sm.p + key * 128);
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 y = make_float2(ex2(__uint_as_float(x[i + 2 * e])), ex2(__uint_as_float(x[i + 2 * e + 1])));
            sums[i / 2 + e] = add2(sums[i / 2 + e], y);
            w[e] = pack_bf16x2(y.x, y.y);
          }
          prow[(4 * half + i / 8) ^ (key & 7)] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        fence_proxy_async_smem();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&sm.pfull));
      }
    }
  };

  // (Every CTA of the cluster has a window at least, in which it checks all picks.)
  for (int w0 = 0; w0 < own || w0 == 0; w0 += kWindow) {
    const int w1 = min(own, w0 + kWindow);
    if (w0 > 0) fetch(w0);
    __syncthreads();  // (the list is no longer read)
    for (int i = tid; i < w1 - w0; i += kSharedThreads) sm.mask[i][0] = sm.mask[i][1] = 0;
    if (tid == 0) sm.ends = 0;
    __syncthreads();
    for (int i0 = tid; i0 < total; i0 += kPicksEach * kSharedThreads) {
      if (i0 > tid) fetch_picks(i0);
#pragma unroll
      for (int x = 0; x < kPicksEach; ++x) {
        const int i = i0 + x * kSharedThreads, node = i / p.max_picks, at = i - node * p.max_picks;
        if (i >= total || at >= sm.counts[node]) continue;
        if (pick[x] < 0 || pick[x] >= pages || pick[x] <= before[x]) {
          set_error(err, KVSHOT_ERR_DEVICE_BOUNDS);
          continue;
        }
        const int own_at = pick[x] / S;
        if (pick[x] - own_at * S != rank || own_at < w0 || own_at >= w1) continue;
        const unsigned long long columns = node_columns << (node * p.G);
        if (static_cast<uint32_t>(columns) != 0) atomicOr(&sm.mask[own_at - w0][0], static_cast<uint32_t>(columns));
        if (columns >> 32 != 0) atomicOr(&sm.mask[own_at - w0][1], static_cast<uint32_t>(columns >> 32));
      }
    }
    __syncthreads();
    // The pages that some node picked, in order.
    uint2 mask[kPagesEach];
    int mine = 0;
#pragma unroll
    for (int x = 0; x < kPagesEach; ++x) {
      const int i = tid * kPagesEach + x;
      mask[x] = i < w1 - w0 ? *reinterpret_cast<const uint2*>(sm.mask[i]) : make_uint2(0, 0);
      mine += (mask[x].x | mask[x].y) != 0;
    }
    int scan = mine;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, scan, x);
      if (lane >= x) scan += y;
    }
    if (lane == 31) sm.warp_sum[warp] = scan;
    __syncthreads();
    int at = scan - mine, listed = 0;
#pragma unroll
    for (int x = 0; x < kSharedThreads / 32; ++x) {
      if (x < warp) at += sm.warp_sum[x];
      listed += sm.warp_sum[x];
    }
#pragma unroll
    for (int x = 0; x < kPagesEach; ++x)
      if ((mask[x].x | mask[x].y) != 0) {
        const bool bad = static_cast<unsigned>(id[x]) >= static_cast<unsigned>(p.v.num_pages);
        if (bad) set_error(err, KVSHOT_ERR_DEVICE_BOUNDS);
        sm.list_row[at] = bad ? -1 : (id[x] * p.v.hkv + h) * P;
        *reinterpret_cast<uint2*>(sm.mask[at++]) = mask[x];
        if ((w0 + tid * kPagesEach + x) * S + rank == pages - 1) sm.ends = 1;
      }
    __syncthreads();
    const int last = listed - 1;  // in whose page the cache may end
    const int last_live = sm.ends != 0 ? L - (pages - 1) * P : P;
    // Group i (8 keys of one page): the page's place in the list, and its first key there.
    const uint32_t groups = listed * groups_per_page;
    auto page_of = [&](uint32_t i) { return groups_per_page == 1 ? i : __umulhi(i, sp.by_page); };
    const int box_groups = sp.box_keys / 8, boxes = kTileKeys128 / sp.box_keys;
    stream(static_cast<int>(groups * 8 + kTileKeys128 - 1) / kTileKeys128,
           [&](int t, bool values, uint32_t base, uint32_t bar) {
             const uint32_t i = t * (kTileKeys128 / 8) + lane * box_groups;
             int row = -1;
             if (lane < boxes && i < groups) {
               const uint32_t page = page_of(i);
               if (sm.list_row[page] >= 0) row = sm.list_row[page] + (i - page * groups_per_page) * 8;
             }
             const int live = __popc(__ballot_sync(0xffffffffu, row >= 0));
             if (lane == 0) mbar_arrive_expect_tx(bar, live * sp.box_keys * 256);
             __syncwarp();
             if (row >= 0) tma_load_4d(base + lane * sp.box_keys * 256, values ? &maps.v : &maps.k, 0, 0, 0, row >> 3, bar);
           },
           [&](int t, int key, int half, bool* live) {
             const uint32_t i = t * (kTileKeys128 / 8) + (key >> 3);
             *live = false;
             if (i >= groups) return 0u;
             const uint32_t page = page_of(i);
             const int at = static_cast<int>(i - page * groups_per_page) * 8 + (key & 7);
             *live = sm.list_row[page] >= 0 && at < (static_cast<int>(page) == last ? last_live : P);
             return *live ? sm.mask[page][half] : 0u;
           });
  }

  if (draft) {  // the nodes themselves and their ancestors
    const int first_row = (c * p.v.hkv + h) * p.n_max, first_node = p.N - p.Nq + n0;
    const int slots = min(p.N, first_node + nodes);  // (no node sees a later one)
    stream((slots + kTileKeys128 - 1) / kTileKeys128,
           [&](int t, bool values, uint32_t base, uint32_t bar) {
             const int slot = t * kTileKeys128 + lane * 8;
             const bool live = lane < kTileKeys128 / 8 && slot < slots;
             const int boxes = __popc(__ballot_sync(0xffffffffu, live));
             if (lane == 0) mbar_arrive_expect_tx(bar, boxes * kGroupBytes);
             __syncwarp();
             if (live) tma_load_3d_plain(base + lane * kGroupBytes, values ? &maps.dv : &maps.dk, 0, first_row + slot, 0, bar);
           },
           [&](int t, int key, int half, bool* live) {
             const int slot = t * kTileKeys128 + key;
             // A chain's node sees the slots up to its own: nodes from slot - first_node on see this one.
             const unsigned long long see =
                 slot >= slots ? 0ull : tree ? sm.line[slot] : all_columns & ~0ull << (max(0, slot - first_node) * p.G);
             *live = see != 0;  // (a tree's branch without any of these nodes may hold anything)
             return static_cast<uint32_t>(see >> (32 * half));
           });
  }
  // Every product has completed, and every copy landed, when the tiles' place becomes the state's.
  if (warp == 9) {
    tc::tc_commit_elect(smem_addr(&sm.done));
    mbar_wait(smem_addr(&sm.done), 0, err);
  }
  if (warp == 8) {
    if (k_issued > 0) mbar_wait(smem_addr(&sm.kfull), (k_issued - 1) & 1, err);
    if (v_issued > 0) mbar_wait(smem_addr(&sm.vfull), (v_issued - 1) & 1, err);
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  float* part = reinterpret_cast<float*>(sm.k);  // [64 rows][kPartStride]
  if (warp < 8) {
    uint32_t o[32];
    if (done > 0 && 32 * half < sp.cols) {
      tc::tmem_ld32(tmem + quarter + 32 * half, o);
      wait_columns(o);
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = 0;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) part[(32 * half + i) * kPartStride + (tid & 127)] = __uint_as_float(o[i]);
    tc::tc_fence_before();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float2 x = sums[i];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) x = add2(x, make_float2(__shfl_xor_sync(0xffffffffu, x.x, o), __shfl_xor_sync(0xffffffffu, x.y, o)));
      if (lane == i) *reinterpret_cast<float2*>(&sm.part_l[warp & 3][32 * half + 2 * i]) = x;
    }
    named_barrier_sync(1 + half, kSoftmaxThreads);
    if ((tid & 127) < 32) {
      const int r = 32 * half + lane;
      sm.m[r] = -sm.neg_ref[r];
      sm.l[r] = (sm.part_l[0][r] + sm.part_l[1][r]) + (sm.part_l[2][r] + sm.part_l[3][r]);
    }
  }

  // The CTAs' states joined: a row's weight of each, then the sums of four dims to a thread.
  if (S > 1) cluster_sync_all();
  else __syncthreads();
  if (warp == 9) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, kSharedTmem);
  }
  float(*weight)[kColumns] = reinterpret_cast<float(*)[kColumns]>(sm.p);  // [S]
  if (tid < rows) {
    float top = -INFINITY, sum = 0.f;
    for (int x = 0; x < S; ++x) top = fmaxf(top, remote_float(smem_addr(&sm.m[tid]), x));
    for (int x = 0; x < S; ++x) {
      const float mx = remote_float(smem_addr(&sm.m[tid]), x), f = mx == -INFINITY ? 0.f : ex2(mx - top);
      weight[x][tid] = f;
      sum += f * remote_float(smem_addr(&sm.l[tid]), x);
    }
    sm.factor[tid] = sum;
    if (tid % S == rank) {
      const int node = tid / p.G;
      p.lse[(static_cast<size_t>(c) * p.Nq + n0 + node) * p.hq + h * p.G + (tid - node * p.G)] =
          (top + log2f(sum)) * 0.6931471805599453f;
    }
  }
  __syncthreads();
  for (int i = rank * kSharedThreads + tid; i < rows * (kHeadDim / 4); i += S * kSharedThreads) {
    const int r = i / (kHeadDim / 4), d = i % (kHeadDim / 4) * 4, node = r / p.G;
    const float sum = sm.factor[r];
    float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int x = 0; x < S; ++x) {
      const float f = weight[x][r];
      if (f == 0.f) continue;
      const float4 y = remote_float4(smem_addr(part + r * kPartStride + d), x);
      out.x += f * y.x;
      out.y += f * y.y;
      out.z += f * y.z;
      out.w += f * y.w;
    }
    const size_t row = (static_cast<size_t>(c) * p.Nq + n0 + node) * p.hq + h * p.G + (r - node * p.G);
    *reinterpret_cast<uint2*>(p.out + row * kHeadDim + d) =
        make_uint2(pack_bf16x2(out.x / sum, out.y / sum), pack_bf16x2(out.z / sum, out.w / sum));
  }
  if (S > 1) cluster_sync_all();  // (another CTA may still read this one's state)
}

cudaError_t launch_shared(const SparseParams& s, int caches, int S, uint32_t wait_ns, cudaStream_t stream) {
  SharedParams p;
  p.s = s;
  const int most = kColumns / s.G, blocks = (s.Nq + most - 1) / most;
  p.nodes_per_block = (s.Nq + blocks - 1) / blocks;
  p.cols = (p.nodes_per_block * s.G + 15) / 16 * 16;
  p.box_keys = std::min(s.v.P, 64);
  const uint32_t groups = s.v.P / 8;
  p.by_page = groups > 1 ? static_cast<uint32_t>(((uint64_t{1} << 32) + groups - 1) / groups) : 0;
  p.wait_ns = wait_ns;
  SharedMaps maps;
  const uint64_t rows = static_cast<uint64_t>(s.v.num_pages) * s.v.hkv * s.v.P;
  const uint64_t drows = static_cast<uint64_t>(caches) * s.v.hkv * s.n_max;
  if (!map_groups(&maps.k, s.k, rows, p.box_keys / 8) || !map_groups(&maps.v, s.val, rows, p.box_keys / 8) ||
      !map_any_8(&maps.dk, s.dk, drows) || !map_any_8(&maps.dv, s.dv, drows))
    return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(sparse_shared_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SharedSpace));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(caches * s.v.hkv * S, blocks);
  cfg.blockDim = dim3(kSharedThreads);
  cfg.dynamicSmemBytes = sizeof(SharedSpace);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sparse_shared_kernel, p, maps);
}

// The states meet in shared memory, and nothing is written here: the call asks for a workspace as the other attention calls do.
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
  // against shared; 16 caches of 20K to 32K tokens and 128 pages a node, 48 rows: 162, 95; 8 rows: 43, 58; 256 rows and 64
  // pages: 403, 224; 64 caches of up to 8K and 32 pages, 16 rows: 79, 84; 16 caches of 4K and 32 pages, 48 rows: 59, 43; one of
  // 8K and 64 pages, 256 rows: 33, 36).  Two CTAs of a cluster fill the SMs' two places (one: 131, and four: 122 for the 95).
  const int each = kColumns / p.G;
  const int64_t rows = static_cast<int64_t>(p.Nq) * p.G, blocks = (p.Nq + each - 1) / each, shared = blocks * d->num_caches * d->hkv;
  // What a node picks has to be worth the list (12 nodes of 16 caches of 4K: 16 tokens 19, 21; 128 27, 27; 256 40, 34).
  const int64_t picked = std::min<int64_t>(static_cast<int64_t>(max_picks) * d->page_size, p.v.len_bound);
  if (rows >= 32 && picked >= 128 && 3 * shared >= 2 * sm_count() && blocks < 65536) {
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
