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

// A unit is one (cache, KV head, query row); its CTAs (a cluster of 1 to 8) take equal parts of its pages, the last one
// the draft keys too, and the CTA's warps 16 keys in turn.  Nodes of one cache and head are next to one another in the
// grid: their pages overlap, and meet in L2.
template <int NT>
__global__ void __launch_bounds__(kSparseThreads) sparse_kernel(SparseParams p) {
  extern __shared__ __align__(16) float s_part[];  // [warps][8 NT][kPartStride]
  __shared__ int s_row[kSparseThreads], s_valid[kSparseThreads];
  __shared__ float s_m[kSparseWarps][8 * NT], s_l[kSparseWarps][8 * NT];
  __shared__ int s_parent[kMaxTreeNodes], s_line[kMaxTreeNodes];
  __shared__ int s_line_len;
  const int S = static_cast<int>(cluster_size());
  const int rank = blockIdx.x % S, unit = blockIdx.x / S;
  const int n = unit % p.Nq, h = unit / p.Nq % p.v.hkv, c = unit / p.Nq / p.v.hkv;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int L = clamped_len(p.v, c);
  const size_t list = (static_cast<size_t>(c) * p.Nq + n) * p.v.hkv + h;
  int count = p.counts[list];
  if (count < 0 || count > p.max_picks) {
    set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
    count = min(max(count, 0), p.max_picks);
  }
  const int32_t* picks = p.picks + list * p.max_picks;

  WarpState<NT> st;
  st.init();
  const size_t qrow = (static_cast<size_t>(c) * p.Nq + n) * p.hq + h * p.G;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      st.q[nt][j] = nt * 8 + g < p.G ? __ldg(p.q + (qrow + nt * 8 + g) * 16 + 8 * (j >> 1) + 2 * t + (j & 1)) : make_uint4(0, 0, 0, 0);

  const int i0 = static_cast<int>(static_cast<int64_t>(count) * rank / S);
  const int i1 = static_cast<int>(static_cast<int64_t>(count) * (rank + 1) / S);
  const int groups_per_page = p.v.P / 8;
  for (int base = i0; base < i1; base += kSparseThreads) {
    __syncthreads();
    const int here = min(kSparseThreads, i1 - base);
    if (tid < here) {
      const int pick = picks[base + tid], before = base + tid > 0 ? picks[base + tid - 1] : -1;
      int row = 0, valid = 0;
      if (pick >= 0 && pick > before && static_cast<int64_t>(pick) * p.v.P < L) {
        const int id = page_id(p.v, c, pick);
        if (id >= 0) {
          row = (id * p.v.hkv + h) * p.v.P;
          valid = min(p.v.P, L - pick * p.v.P);
        }
      } else {
        set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
      }
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

  if (rank == S - 1) {  // the node itself and its ancestors
    const int node = p.N - p.Nq + n;
    if (p.tree_parent != nullptr) {
      const int32_t* parent = p.tree_parent + static_cast<size_t>(c / p.per_seq) * p.N;
      if (tid < p.N) s_parent[tid] = parent[tid];
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
    const int line = p.tree_parent != nullptr ? s_line_len : node + 1;
    const int draft0 = (c * p.v.hkv + h) * p.n_max;
    auto slot = [&](int i) { return i >= line ? -1 : draft0 + (p.tree_parent != nullptr ? s_line[i] : i); };
    for (int s = warp; s * 16 < line; s += kSparseWarps) {
      const int kr[2] = {slot(s * 16 + g), slot(s * 16 + g + 8)};
      const int vr[4] = {slot(s * 16 + 2 * t), slot(s * 16 + 2 * t + 1), slot(s * 16 + 2 * t + 8), slot(s * 16 + 2 * t + 9)};
      st.step(p.dk, p.dv, kr, vr, p.qscale, g, t);
    }
  }

  // The warps' states joined: reference and sum of every row, then a weighted sum of the O's.
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
  if (S > 1) cluster_sync_all();
  else __syncthreads();
  for (int i = rank * kSparseThreads + tid; i < p.G * kHeadDim; i += S * kSparseThreads) {
    const int r = i / kHeadDim, d = i % kHeadDim;
    float top = -INFINITY;
    for (int x = 0; x < S; ++x)
      for (int w = 0; w < kSparseWarps; ++w) top = fmaxf(top, remote_float(smem_addr(&s_m[w][r]), x));
    float sum = 0.f, o = 0.f;
    for (int x = 0; x < S; ++x)
      for (int w = 0; w < kSparseWarps; ++w) {
        const float m = remote_float(smem_addr(&s_m[w][r]), x);
        const float f = m == -INFINITY ? 0.f : ex2(m - top);
        sum += f * remote_float(smem_addr(&s_l[w][r]), x);
        o += f * remote_float(smem_addr(s_part + (w * 8 * NT + r) * kPartStride + d), x);
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

constexpr size_t kSparseWorkspace = 256;

kvshot_status check_sparse(const kvshot_attn_desc* d, int max_picks) {
  if (kvshot_status st = check_partial(d, true)) return st;
  if (max_picks < 1) return KVSHOT_ERR_SHAPE;
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
  const int units = d->num_caches * d->hkv * d->n_query;
  // CTAs per unit: until the SMs have two each, while a warp still has 16 keys.
  const int64_t steps = static_cast<int64_t>(max_picks) * d->page_size / 16;
  int S = 1;
  while (S < 8 && static_cast<int64_t>(units) * S < 2 * sm_count() && steps > 2 * S * kSparseWarps) S *= 2;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = p.G <= 8    ? launch_sparse<1>(p, units, S, s)
                        : p.G <= 16 ? launch_sparse<2>(p, units, S, s)
                                    : launch_sparse<4>(p, units, S, s);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
