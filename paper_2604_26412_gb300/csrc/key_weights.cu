// key_weights.cu -- the softmax weight that each cached token got from the query rows, accumulated.
//   w_out[c, j] = decay w[c, j] + sum over rows n and q heads of exp(scale q . k_j - lse[c, n, head])
#include <algorithm>
#include <cmath>

#include "kvshot_partial.cuh"

namespace kvshot {
namespace {

using namespace dev;
using namespace partial;

constexpr int kWeightWarps = 4;
constexpr int kWeightChunks = 2;  // of 16 keys, per warp
constexpr int kWeightKeys = kWeightWarps * kWeightChunks * 16;
constexpr int kWeightRows = 128;  // rows of q in shared memory at a time

struct WeightParams {
  CacheView v;
  const uint4 *q, *k;
  const float *lse, *weights;
  float* weights_out;
  int hq, G, Nq, weights_len;
  float qscale, decay;  // scale * log2(e)
};

// A warp's keys are the M rows of mma.sync, the query rows of one KV head its columns; a lane sums the exponentials of its
// keys' columns over all heads.
__global__ void __launch_bounds__(kWeightWarps * 32) weights_kernel(WeightParams p) {
  __shared__ __align__(16) uint8_t s_q[kWeightRows * kQRowBytes];
  __shared__ float s_lse[kWeightRows];
  const int c = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  int L = clamped_len(p.v, c);
  if (L > p.weights_len) {
    set_error(p.v.err, KVSHOT_ERR_DEVICE_BOUNDS);
    L = p.weights_len;
  }
  const int cta0 = blockIdx.x * kWeightKeys;
  if (cta0 >= L) return;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  int key[kWeightChunks][2];
  size_t row[kWeightChunks][2];  // of KV head 0
  float w[kWeightChunks][2] = {};
#pragma unroll
  for (int i = 0; i < kWeightChunks; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      int j = cta0 + (i * kWeightWarps + warp) * 16 + g + 8 * e;
      const int page = j / p.v.P, id = j < L ? page_id(p.v, c, page) : -1;
      row[i][e] = static_cast<size_t>(max(id, 0)) * p.v.hkv * p.v.P + (j - page * p.v.P);
      key[i][e] = id >= 0 ? j : -1;
    }
  const int rows = p.Nq * p.G;
  for (int h = 0; h < p.v.hkv; ++h) {
    for (int r0 = 0; r0 < rows; r0 += kWeightRows) {
      __syncthreads();
      const int here = min(kWeightRows, (rows - r0 + 7) / 8 * 8);
      for (int i = threadIdx.x; i < here * 16; i += kWeightWarps * 32) {
        const int r = r0 + i / 16, n = r / p.G, head = h * p.G + r % p.G;
        const size_t at = (static_cast<size_t>(c) * p.Nq + n) * p.hq + head;
        *reinterpret_cast<uint4*>(s_q + (i / 16) * kQRowBytes + (i % 16) * 16) = r < rows ? __ldg(p.q + at * 16 + i % 16) : zero;
        if (i % 16 == 0) {
          const float z = r < rows ? p.lse[at] : INFINITY;
          s_lse[i / 16] = z == -INFINITY ? INFINITY : z * 1.4426950408889634f;  // (an empty row gives nothing)
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWeightChunks; ++i) {
        uint4 a[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            a[e][j] = key[i][e] >= 0 ? __ldg(p.k + (row[i][e] + static_cast<size_t>(h) * p.v.P) * 16 + 4 * j + t) : zero;
        for (int tile = 0; tile < here / 8; ++tile) {
          float d[4] = {0.f, 0.f, 0.f, 0.f};
          const uint8_t* qrow = s_q + (tile * 8 + g) * kQRowBytes + t * 16;
#pragma unroll
          for (int j = 0; j < 4; ++j) mma_piece(d, a[0][j], a[1][j], *reinterpret_cast<const uint4*>(qrow + j * 64));
          const float z0 = s_lse[tile * 8 + 2 * t], z1 = s_lse[tile * 8 + 2 * t + 1];
          w[i][0] += ex2(fmaf(d[0], p.qscale, -z0)) + ex2(fmaf(d[1], p.qscale, -z1));
          w[i][1] += ex2(fmaf(d[2], p.qscale, -z0)) + ex2(fmaf(d[3], p.qscale, -z1));
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kWeightChunks; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float x = w[i][e];
      x += __shfl_xor_sync(0xffffffffu, x, 1);
      x += __shfl_xor_sync(0xffffffffu, x, 2);
      if (t != 0 || key[i][e] < 0) continue;
      const size_t at = static_cast<size_t>(c) * p.weights_len + key[i][e];
      p.weights_out[at] = p.weights != nullptr ? fmaf(p.decay, p.weights[at], x) : x;
    }
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
  const int most = std::min(p.v.len_bound, weights_len);
  // (With no room at all the lengths still have to be looked at.)
  const cudaError_t e =
      launch_maybe_pdl(weights_kernel, dim3(std::max(1, (most + kWeightKeys - 1) / kWeightKeys), p.v.C),
                       dim3(kWeightWarps * 32), 0, false, reinterpret_cast<cudaStream_t>(stream), p);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
