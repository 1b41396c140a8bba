// attn_kv4.cu -- draft attention over a 4-bit target cache, with an optional sliding window and sink tokens.
//
// One CTA per query row (cache, node, head): 128 keys at a time, a key to a thread for the scores, a dim to a thread
// for the weighted sum, with a running maximum and sum in fp32.
#include <algorithm>
#include <climits>
#include <cmath>

#include "kvshot_attn_common.cuh"
#include "kvshot_kv4.cuh"

namespace kvshot {
namespace {

using namespace dev;
using namespace kv4;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

constexpr int kThreads = 128;

struct Kv4Params {
  AttnParams a;
  const uint8_t* cache;
  const __nv_bfloat16 *draft_k, *draft_v;
  int window, sinks;
};

__device__ __forceinline__ float kv4_value(const uint8_t* g, int kind, int row, int d) {
  const uint32_t byte = g[kind * kVCodes + (d >> 5) * kChunkStride + row * kChunkBytes + ((d & 31) >> 1)];
  const uint32_t n = (d & 1) ? byte >> 4 : byte & 15u;
  const float mag = (n & 7u) < 2u ? 0.5f * (n & 7u) : (1.f + 0.5f * (n & 1u)) * static_cast<float>(1u << ((n & 7u) / 2 - 1));
  const uint32_t s = e4m3x2_to_f16x2(g[kScales + kind * kScaleBytes + row * 8 + (d >> 4)]);
  const float v = mag * __half2float(__ushort_as_half(static_cast<unsigned short>(s & 0xffffu)));
  return (n & 8u) ? -v : v;
}

__global__ void __launch_bounds__(kThreads) attn_kv4_kernel(const __grid_constant__ Kv4Params kp) {
  const AttnParams& p = kp.a;
  __shared__ float s_q[kHeadDim], s_p[kThreads], s_red[kThreads];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % p.hq, nl = blockIdx.x / p.hq, c = blockIdx.y;
  const int kh = h / p.G, node = p.N - p.Nq + nl;
  wait_for_prerequisite_grid();
  const int L = clamp_len(p, c);
  const size_t row = (static_cast<size_t>(c) * p.Nq + nl) * p.hq + h;
  s_q[tid] = __bfloat162float(p.q[row * kHeadDim + tid]);
  // Depth of the node, and of its ancestors: tree walks are short.
  const int* par = p.tree ? p.tree_parent + static_cast<size_t>(c / (p.C / p.B)) * p.N : nullptr;
  auto parent = [&](int m) {
    if (!par) return m - 1;
    const int v = par[m];
    if (v < -1 || v >= m) {
      set_error(p.err, KVSHOT_ERR_TREE);
      return -1;
    }
    return v;
  };
  auto depth = [&](int m) {
    int d = 0;
    for (; m >= 0; m = parent(m)) ++d;
    return d;
  };
  const int pos = L + (par ? depth(node) : node + 1) - 1;
  auto seen = [&](int at) { return kp.window == 0 || pos - at < kp.window || at < kp.sinks; };
  auto draft_seen = [&](int m) {
    if (m > node) return false;
    if (!par) return seen(L + m);
    int a = node;
    while (a > m) a = parent(a);
    return a == m && seen(L + depth(m) - 1);
  };
  __syncthreads();
  float m_run = -INFINITY, l_run = 0.f, o = 0.f;
  const int keys = L + p.N, ps = p.page_size, groups = ps / kKv4Tokens;
  const int first = kp.window == 0 ? 0 : max(0, pos - kp.window + 1);
  for (int k0 = 0; k0 < keys; k0 += kThreads) {
    // (tiles between the sinks and the window hold nothing to see)
    if (kp.window != 0 && k0 >= kp.sinks && k0 + kThreads <= min(first, L)) continue;
    const int j = k0 + tid;
    auto group = [&](int key) {
      const int pg = key / ps;
      const int pid = p.paged ? valid_page_id(p, p.page_table[static_cast<size_t>(c) * p.max_pages + pg]) : c;
      return kp.cache + ((static_cast<size_t>(pid) * p.hkv + kh) * groups + (key - pg * ps) / kKv4Tokens) * kKv4Bytes;
    };
    float s = -INFINITY;
    if (j < L ? seen(j) : j < keys && draft_seen(j - L)) {
      s = 0.f;
      if (j < L) {
        const uint8_t* g = group(j);
        for (int d = 0; d < kHeadDim; ++d) s += s_q[d] * kv4_value(g, 0, j % kKv4Tokens, d);
        s *= p.qscale * p.k_scale;
      } else {
        const __nv_bfloat16* k = kp.draft_k + ((static_cast<size_t>(c) * p.hkv + kh) * p.n_max + j - L) * kHeadDim;
        for (int d = 0; d < kHeadDim; ++d) s += s_q[d] * __bfloat162float(k[d]);
        s *= p.qscale;
      }
    }
    s_red[tid] = s;
    __syncthreads();
    float mx = m_run;
    for (int i = 0; i < kThreads; ++i) mx = fmaxf(mx, s_red[i]);
    const float e = s == -INFINITY ? 0.f : exp2f(s - mx);
    s_p[tid] = e;
    __syncthreads();
    const float alpha = m_run == -INFINITY ? 0.f : exp2f(m_run - mx);
    m_run = mx;
    o *= alpha;
    l_run *= alpha;
    for (int i = 0; i < kThreads; ++i) {
      const float w = s_p[i];
      if (w == 0.f) continue;
      l_run += w;
      const int key = k0 + i;
      if (key < L) {
        o += w * p.v_scale * kv4_value(group(key), 1, key % kKv4Tokens, tid);
      } else {
        o += w * __bfloat162float(kp.draft_v[((static_cast<size_t>(c) * p.hkv + kh) * p.n_max + key - L) * kHeadDim + tid]);
      }
    }
    __syncthreads();
  }
  p.out[row * kHeadDim + tid] = __float2bfloat16(o / l_run);
  if (tid == 0) p.lse[row] = (m_run + log2f(l_run)) * 0.69314718055994531f;
}

kvshot_status check_attn_kv4(const kvshot_attn_desc* d, int32_t window, int32_t sinks) {
  if (kvshot_status st = check_common(d)) return st;
  if ((d->flags & ~(KVSHOT_TREE | KVSHOT_OVERLAP_PREVIOUS)) != 0) return KVSHOT_ERR_UNSUPPORTED;
  if (d->k_scale_exp < -64 || d->k_scale_exp > 64 || d->v_scale_exp < -64 || d->v_scale_exp > 64)
    return KVSHOT_ERR_SHAPE;
  if (window < 0 || sinks < 0) return KVSHOT_ERR_SHAPE;
  return KVSHOT_OK;
}

}  // namespace
}  // namespace kvshot

using namespace kvshot;

extern "C" size_t kvshot_draft_attn_kv4_workspace_size(const kvshot_attn_desc* d, int32_t window, int32_t sinks) {
  return check_attn_kv4(d, window, sinks) == KVSHOT_OK ? 256 : 0;
}

extern "C" kvshot_status kvshot_draft_attn_kv4(const kvshot_attn_desc* d, const void* q, const void* cache,
                                               const int32_t* page_table, const int32_t* seq_lens, const void* draft_k,
                                               const void* draft_v, const int32_t* tree_parent, int32_t window,
                                               int32_t sinks, void* out, float* lse, kvshot_stream_t stream) {
  if (kvshot_status st = check_attn_kv4(d, window, sinks)) return st;
  const bool paged = page_table != nullptr, tree = d->flags & KVSHOT_TREE;
  if (paged) {
    if (d->page_size < 1) return KVSHOT_ERR_SHAPE;
    if (d->page_size % kKv4Tokens != 0) return KVSHOT_ERR_UNSUPPORTED;
    if (d->max_pages_per_seq < 1 || d->num_pages < 1) return KVSHOT_ERR_SHAPE;
    if (static_cast<double>(d->num_pages) * d->hkv * d->page_size >= INT_MAX ||
        static_cast<int64_t>(d->num_caches) * d->max_pages_per_seq >= INT_MAX ||
        static_cast<int64_t>(d->max_pages_per_seq) * d->page_size >= INT_MAX)
      return KVSHOT_ERR_UNSUPPORTED;
  } else {
    if (d->l_cap < 1) return KVSHOT_ERR_SHAPE;
    if (d->l_cap % kKv4Tokens != 0) return KVSHOT_ERR_UNSUPPORTED;
    if (static_cast<double>(d->num_caches) * d->hkv * d->l_cap >= INT_MAX) return KVSHOT_ERR_UNSUPPORTED;
  }
  if (d->n_query == 0) return KVSHOT_OK;
  if (!q || !cache || !seq_lens || !draft_k || !draft_v || !out || !lse || (tree && !tree_parent)) return KVSHOT_ERR_NULL;
  if (!aligned(q, 16) || !aligned(cache, 16) || !aligned(draft_k, 16) || !aligned(draft_v, 16) || !aligned(out, 16) ||
      !aligned(lse, 4) || !aligned(seq_lens, 4) || (paged && !aligned(page_table, 4)) || (tree && !aligned(tree_parent, 4)))
    return KVSHOT_ERR_ALIGN;
  if (d->workspace == nullptr || !aligned(d->workspace, 256) || d->workspace_bytes < 256) return KVSHOT_ERR_WORKSPACE;
  Kv4Params kp = {};
  AttnParams& p = kp.a;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.page_table = page_table;
  p.seq_lens = seq_lens;
  p.tree_parent = tree_parent;
  p.err = d->err_flag;
  p.C = d->num_caches;
  p.B = d->num_seqs;
  p.hq = d->hq;
  p.hkv = d->hkv;
  p.G = d->hq / d->hkv;
  p.paged = paged;
  p.page_size = paged ? d->page_size : d->l_cap;
  p.max_pages = paged ? d->max_pages_per_seq : 1;
  p.num_pages = paged ? d->num_pages : d->num_caches;
  const int64_t cap = static_cast<int64_t>(p.max_pages) * p.page_size;
  p.len_bound = static_cast<int>(std::min<int64_t>(d->max_seq_len, cap));
  p.N = d->n_nodes;
  p.Nq = d->n_query;
  p.n_max = d->n_max;
  p.tree = tree;
  const double scale = d->scale != 0.f ? static_cast<double>(d->scale) : 1.0 / std::sqrt(static_cast<double>(kHeadDim));
  p.qscale = static_cast<float>(scale * 1.4426950408889634);
  p.k_scale = std::ldexp(1.f, d->k_scale_exp);
  p.v_scale = std::ldexp(1.f, d->v_scale_exp);
  kp.cache = static_cast<const uint8_t*>(cache);
  kp.draft_k = static_cast<const __nv_bfloat16*>(draft_k);
  kp.draft_v = static_cast<const __nv_bfloat16*>(draft_v);
  kp.window = window;
  kp.sinks = sinks;
  const bool pdl = (d->flags & KVSHOT_OVERLAP_PREVIOUS) != 0;
  const cudaError_t e = launch_maybe_pdl(attn_kv4_kernel, dim3(p.Nq * p.hq, p.C), dim3(kThreads), 0, pdl,
                                         reinterpret_cast<cudaStream_t>(stream), kp);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
