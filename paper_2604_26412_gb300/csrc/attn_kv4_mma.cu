// attn_kv4_mma.cu -- draft attention over a 4-bit target cache for stacks of up to 16 query rows per KV head, on
// mma.sync tensor cores, with an optional sliding window and sink tokens.
//
// What bounds it: 144 B per key and KV head come from HBM, and each of its 256 codes has to become an f16 before it can be
// multiplied: 128 conversions of two codes and 128 products with a scale per key, 8 of the kernel's ~17 (8 rows) to 22 (16)
// warp instructions per key.  So a warp keeps everything in registers from the codes to O, and waits for no other warp:
//  - Keys are the M dimension (as in attn_f8.cu): S^T = K Q^T, O^T = V^T P^T (m16n8k16, f16, fp32 sums); the query rows
//    are N in steps of 8.  An m16 tile of keys is a 16-token group of the cache.
//  - K: ldmatrix gives a lane 8 dims of each chunk of its key row, which feed k-steps 2 c and 2 c + 1; q's dims are taken
//    in the same order.  V: a transposing ldmatrix of 16-bit words gives a lane four dims of two neighbouring keys; two
//    shifts and two selections pair their codes dim by dim, the m-tile's rows being dims 4 g + kk and 4 g + kk + 2 of a
//    chunk.  Scales ride on the converted pairs, whose products are exact.
//  - P^T comes from S^T by one 8x8 transpose (movmatrix) per 8 keys x 8 rows.
//  - A row's reference is 2^8 below the maximum it was taken from and moves when a score passes it by 2^15, so O is
//    rescaled rarely and P stays in f16's normal range for scores down to 2^-22 of the maximum.
// A CTA is four warps, 32 keys of a tile each, and a loading warp; several CTAs share an SM.
#include <algorithm>

#include "kvshot_kv4_attn.cuh"

namespace kvshot {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = (kWarps + 1) * 32;
constexpr int kCombStride = kHeadDim + 4;  // padded fp32 row of the combine buffer

// NR: 8-row steps.
template <int NR, int STAGES, int MINB>
struct Cfg {
  static constexpr int kNR = NR;
  static constexpr int kStages = STAGES;
  static constexpr int kMinBlocks = MINB;
  static constexpr int kRows = 8 * NR;
};

struct Smem : Ring {
  Rows* rows;
  uint32_t joined;      // barrier of the consumer warps
  float* comb_o;        // [kWarps][rows][kCombStride] a piece's O of each warp
  float *ref, *sum;     // [kWarps][rows] its references and sums; then (ref) its weights
};

template <class CF>
__host__ __device__ constexpr size_t smem_bytes(int C) {
  return 128 + CF::kStages * kStageSize + sizeof(float) * kWarps * CF::kRows * (kCombStride + 2) +
         sizeof(TileMeta) * kMetas + sizeof(Rows) + sizeof(uint64_t) * (2 * CF::kStages + 2) + sizeof(int) * (4 + 2 * C + 1);
}

template <class CF>
__device__ __forceinline__ Smem carve(uint8_t* raw, int C) {
  Smem s;
  uint8_t* b = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~uintptr_t(127));
  s.ring = smem_addr(b);
  s.comb_o = reinterpret_cast<float*>(b + CF::kStages * kStageSize);
  s.ref = s.comb_o + kWarps * CF::kRows * kCombStride;
  s.sum = s.ref + kWarps * CF::kRows;
  TileMeta* meta = reinterpret_cast<TileMeta*>(s.sum + kWarps * CF::kRows);
  s.meta = smem_addr(meta);
  uint64_t* m = reinterpret_cast<uint64_t*>(meta + kMetas);
  s.cfull = smem_addr(m);
  s.cempty = s.cfull + 8 * CF::kStages;
  s.joined = s.cempty + 8 * CF::kStages;
  s.rows = reinterpret_cast<Rows*>(m + 2 * CF::kStages + 2);
  int* words = reinterpret_cast<int*>(s.rows + 1);
  s.issued = words;
  s.len = words + 4;
  s.base = s.len + C;
  return s;
}

// 8x8 transpose of b16 elements across the warp.
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// D += A * B, m16n8k16, f16 inputs, fp32 accumulate.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two bytes of (a, b) picked by sel's first two places, and two by its last, as scales: e4m3 -> f16x2 each.
__device__ __forceinline__ uint2 scales_of(uint32_t a, uint32_t b, uint32_t sel) {
  const uint32_t x = __byte_perm(a, b, sel);
  uint2 r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
      : "=r"(r.x), "=r"(r.y)
      : "r"(x));
  return r;
}

// Bits of a where m is set, of b elsewhere.
__device__ __forceinline__ uint32_t select_bits(uint32_t a, uint32_t b, uint32_t m) { return (a & m) | (b & ~m); }

// Join the warps' parts of a piece, which lie in shared memory, and write it: the final bf16 output + lse if it is the
// whole unit, else the normalised fp32 part + log2-domain lse.  All consumer threads (thread = dim).
template <int n>
__device__ __noinline__ bool join_warps(const AttnParams& p, const Smem& sm, const TileMeta& w, WarpSync& sync, const Waiter& wait) {
  const int tid = threadIdx.x;
  if (!sync(wait)) return false;
  const int rows = min(p.rows_per_unit, p.rows_total - w.rb * p.rows_per_unit);
  const bool whole = w.flags & kWhole;
  const size_t part = static_cast<size_t>((w.c * p.hkv + w.h) * p.row_blocks + w.rb + blockIdx.x) * p.rows_per_unit;
  const size_t orow0 = static_cast<size_t>(w.c) * p.Nq * p.hq + w.h * p.G;
  if (tid < rows) {
    float top = kNoRef, total = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) top = fmaxf(top, sm.ref[k * n + tid]);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) total += ex2(sm.ref[k * n + tid] - top) * sm.sum[k * n + tid];
    const float inv = total == 0.f ? 0.f : __fdividef(1.f, total);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) sm.ref[k * n + tid] = ex2(sm.ref[k * n + tid] - top) * inv;
    const float lse2 = total == 0.f ? -INFINITY : top + __log2f(total);
    if (whole) p.lse[orow0 + sm.rows->place[tid]] = lse2 * 0.69314718055994531f;
    else p.ws_lse[part + tid] = lse2;
  }
  if (!sync(wait)) return false;
#pragma unroll 1
  for (int r = 0; r < rows; ++r) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) v = fmaf(sm.ref[k * n + r], sm.comb_o[(k * n + r) * kCombStride + tid], v);
    if (whole) p.out[(orow0 + sm.rows->place[r]) * kHeadDim + tid] = __float2bfloat16(v);
    else p.ws_o[(part + r) * kHeadDim + tid] = v;
  }
  return true;
}

template <class CF>
__device__ __forceinline__ void run_consumer(const Kv4Params& kp, const Smem& smem, const Waiter& wait) {
  constexpr int NR = CF::kNR;
  const AttnParams& p = kp.a;
  const Smem sm = smem;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
  // This lane's places in a group: ldmatrix rows of K (chunk lane / 8, token lane % 8) and of V (chunk lane / 16, token
  // lane % 16), the scales of its keys (K: token g; V: tokens 2 q4, 2 q4 + 1) and which of them it takes.
  const uint32_t kaddr = (lane >> 3) * kChunkStride + (lane & 7) * kChunkBytes;
  const uint32_t vaddr = kVCodes + (lane >> 4) * kChunkStride + (lane & 15) * kChunkBytes;
  const uint32_t kscale = kScales + g * 8, vscale = kScales + kScaleBytes + q4 * 16;
  const uint32_t ksel = q4 & 2 ? 0x3311u : 0x2200u, vsel = g & 4 ? 0x7351u : 0x6240u;
  WarpSync sync{sm.joined, 0};
  // Q^T fragments (f16): k-step 2 c + h on dims 32 c + 8 q4 + 4 h + {0, 1}, {2, 3} of row 8 nr + g.
  uint2 q[8][NR];
  float o[8][NR][4], ref[NR][2], l[NR][2];  // rows 8 nr + 2 q4 + e; l: this lane's keys only
  bool in_codes = false;                    // O is in units of the value codes (a warp without draft keys keeps it so)
  wait_for_prerequisite_grid();             // q and the outputs may be the preceding kernel's
  int stage = 0, rb = 0;
  uint32_t phase = 0;
#pragma unroll 1
  for (int t = 0;; ++t) {
    if (!__all_sync(0xffffffffu, wait(sm.cfull + 8 * stage, phase))) return;
    const int4 meta = tile_words(sm, t);  // flags, key0, nkeys, L
    if (meta.x & kStop) return;
    const bool draft = meta.x & kDraft, masked = meta.x & kMasked;
    if (meta.x & kFirst) {
      const TileMeta w = tile_meta(sm, t);
      if (!sync(wait)) return;  // the piece before has been written out
      rb = w.rb;
      if (w.flags & kNewRows) {
        if (warp == 0) build_rows(kp, *sm.rows, CF::kRows, w.rb, w.seq, w.flags & kNewTree);
        if (!sync(wait)) return;
      }
      const __nv_bfloat16* qrow = p.q + (static_cast<size_t>(w.c) * p.Nq * p.hq + w.h * p.G) * kHeadDim + 8 * q4;
      const int rows = min(p.rows_per_unit, p.rows_total - w.rb * p.rows_per_unit);
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        const uint4* src = reinterpret_cast<const uint4*>(qrow + static_cast<size_t>(sm.rows->place[8 * nr + g]) * kHeadDim);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint4 x = make_uint4(0u, 0u, 0u, 0u);
          if (8 * nr + g < rows) x = src[4 * c];
          q[2 * c][nr] = make_uint2(bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(x.y));
          q[2 * c + 1][nr] = make_uint2(bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(x.w));
        }
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) o[mt][nr][0] = o[mt][nr][1] = o[mt][nr][2] = o[mt][nr][3] = 0.f;
        ref[nr][0] = ref[nr][1] = kNoRef;
        l[nr][0] = l[nr][1] = 0.f;
      }
      in_codes = !draft;
    }
    const float qs = draft ? p.qscale : p.qscale * p.k_scale;
    const uint32_t tile = sm.ring + stage * kStageSize;
    // 16 keys (a group of the cache) at a time: two groups of a prefix tile to a warp, one of a draft tile.
    const int last = draft ? warp + 1 : 2 * warp + 2;
#pragma unroll 1
    for (int grp = draft ? warp : 2 * warp; grp < last; ++grp) {
      const int kw = 16 * grp;
      if (kw >= meta.z) break;
      const uint32_t at = tile + grp * kKv4Bytes;
      // S^T: s[nr][2 a + e] is key kw + 8 a + g, row 8 nr + 2 q4 + e.
      float s[NR][4];
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) s[nr][0] = s[nr][1] = s[nr][2] = s[nr][3] = 0.f;
      if (!draft) {
        uint32_t a[4], b[4];  // keys g and g + 8: a word of each chunk
        ldmatrix_x4(at + kaddr, a[0], a[1], a[2], a[3]);
        ldmatrix_x4(at + kaddr + 8 * kChunkBytes, b[0], b[1], b[2], b[3]);
        const uint2 sa = lds64(at + kscale), sb = lds64(at + kscale + 64);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint2 sca = scales_of(c < 2 ? sa.x : sa.y, 0, ksel), scb = scales_of(c < 2 ? sb.x : sb.y, 0, ksel);
          const uint32_t s2a = c & 1 ? sca.y : sca.x, s2b = c & 1 ? scb.y : scb.x;
          uint32_t fa[4], fb[4];
          e2m1x8_to_f16(a[c], fa);
          e2m1x8_to_f16(b[c], fb);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            fa[k] = mul_f16x2(fa[k], s2a);
            fb[k] = mul_f16x2(fb[k], s2b);
          }
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            mma_f16(s[nr], fa[0], fb[0], fa[1], fb[1], q[2 * c][nr].x, q[2 * c][nr].y);
            mma_f16(s[nr], fa[2], fb[2], fa[3], fb[3], q[2 * c + 1][nr].x, q[2 * c + 1][nr].y);
          }
        }
      } else {
        const uint32_t krow = tile + (kw + g) * kDraftRow + 16 * q4;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint4 x = lds128(krow + 64 * c), y = lds128(krow + 8 * kDraftRow + 64 * c);
          const uint32_t f[8] = {bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(y.x), bf16x2_to_f16x2(x.y), bf16x2_to_f16x2(y.y),
                                 bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(y.z), bf16x2_to_f16x2(x.w), bf16x2_to_f16x2(y.w)};
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            mma_f16(s[nr], f[0], f[1], f[2], f[3], q[2 * c][nr].x, q[2 * c][nr].y);
            mma_f16(s[nr], f[4], f[5], f[6], f[7], q[2 * c + 1][nr].x, q[2 * c + 1][nr].y);
          }
        }
      }
      if (masked) {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const uint64_t vis = rows_seeing(kp, *sm.rows, meta, rb, kw + 8 * a + g) >> (2 * q4);
#pragma unroll
          for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (!((vis >> (8 * nr + e)) & 1ull)) s[nr][2 * a + e] = -INFINITY;
        }
      }
      bool grow = draft && in_codes && p.v_scale != 1.f;  // (O leaves the codes)
      float mx[NR][2];
#pragma unroll
      for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mx[nr][e] = fmaf(fmaxf(s[nr][e], s[nr][2 + e]), qs, -ref[nr][e]);
          grow |= mx[nr][e] > kRefLimit;
        }
      if (__any_sync(0xffffffffu, grow)) {
        const float vs = draft && in_codes ? p.v_scale : 1.f;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float v = fmaxf(s[nr][e], s[nr][2 + e]) * qs;
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
            const float to = v - ref[nr][e] > kRefLimit ? v - kRefBelow : ref[nr][e];
            const float alpha = ex2(ref[nr][e] - to), o_alpha = alpha * vs;
            ref[nr][e] = to;
            l[nr][e] *= alpha;
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) {
              o[mt][nr][e] *= o_alpha;
              o[mt][nr][2 + e] *= o_alpha;
            }
          }
      }
      if (draft) in_codes = false;
      uint32_t pb[NR][2];  // P^T fragments
#pragma unroll
      for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const float e0 = ex2(fmaf(s[nr][2 * a], qs, -ref[nr][0])), e1 = ex2(fmaf(s[nr][2 * a + 1], qs, -ref[nr][1]));
          l[nr][0] += e0;
          l[nr][1] += e1;
          pb[nr][a] = movmatrix_trans(pack_f16x2(e0, e1));
        }
      if (!draft) {
        uint32_t v[4][2];  // chunk; tokens 0..7 and 8..15
        ldmatrix_x4_trans(at + vaddr, v[0][0], v[0][1], v[1][0], v[1][1]);
        ldmatrix_x4_trans(at + vaddr + 2 * kChunkStride, v[2][0], v[2][1], v[3][0], v[3][1]);
        uint4 sc[2] = {lds128(at + vscale), lds128(at + vscale + 64)};  // tokens 2 q4, 2 q4 + 1 and those + 8
        if (masked) {
          // Keys that no row sees may hold anything, NaN scales among it: 0 times them must be 0.
          const int lo = p.window > 0 ? meta.w + p.min_depth - p.window : 0;
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            const int key = kw + 8 * a + 2 * q4, pos = meta.y + key;
            if (key >= meta.z || (pos < lo && pos >= p.sinks)) sc[a].x = sc[a].y = 0u;
            if (key + 1 >= meta.z || (pos + 1 < lo && pos + 1 >= p.sinks)) sc[a].z = sc[a].w = 0u;
          }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          // Codes of dims 4 g .. 4 g + 3: of keys 2 q4 and 2 q4 + 8, and of the keys after them; then dim by dim the
          // codes of two neighbouring keys in a byte (dims 0, 2 of the keys and of those + 8; dims 1, 3).
          const uint32_t x = __byte_perm(v[c][0], v[c][1], 0x5410), y = __byte_perm(v[c][0], v[c][1], 0x7632);
          uint32_t f[8];
          e2m1x8_to_f16(select_bits(x, y << 4, 0x0f0f0f0fu), *reinterpret_cast<uint32_t(*)[4]>(&f[0]));
          e2m1x8_to_f16(select_bits(x >> 4, y, 0x0f0f0f0fu), *reinterpret_cast<uint32_t(*)[4]>(&f[4]));
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            const uint2 pair = scales_of(c < 2 ? sc[a].x : sc[a].y, c < 2 ? sc[a].z : sc[a].w, vsel);
            const uint32_t s2 = c & 1 ? pair.y : pair.x;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              f[2 * a + k] = mul_f16x2(f[2 * a + k], s2);
              f[4 + 2 * a + k] = mul_f16x2(f[4 + 2 * a + k], s2);
            }
          }
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            mma_f16(o[2 * c][nr], f[0], f[1], f[2], f[3], pb[nr][0], pb[nr][1]);
            mma_f16(o[2 * c + 1][nr], f[4], f[5], f[6], f[7], pb[nr][0], pb[nr][1]);
          }
        }
      } else {
        const uint32_t vrow = tile + kDraftV + (kw + 2 * q4) * kDraftRow + 8 * g;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t f[8];
#pragma unroll
          for (int a = 0; a < 2; ++a) {  // keys 2 q4 + 8 a, + 1: dims 4 g .. 4 g + 3 of the chunk
            uint2 x = lds64(vrow + 8 * a * kDraftRow + 64 * c), y = lds64(vrow + (8 * a + 1) * kDraftRow + 64 * c);
            if (kw + 2 * q4 + 8 * a >= meta.z) x = make_uint2(0u, 0u);
            if (kw + 2 * q4 + 8 * a + 1 >= meta.z) y = make_uint2(0u, 0u);
            f[2 * a] = bf16x2_to_f16x2(__byte_perm(x.x, y.x, 0x5410));
            f[2 * a + 1] = bf16x2_to_f16x2(__byte_perm(x.y, y.y, 0x5410));
            f[4 + 2 * a] = bf16x2_to_f16x2(__byte_perm(x.x, y.x, 0x7632));
            f[4 + 2 * a + 1] = bf16x2_to_f16x2(__byte_perm(x.y, y.y, 0x7632));
          }
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            mma_f16(o[2 * c][nr], f[0], f[1], f[2], f[3], pb[nr][0], pb[nr][1]);
            mma_f16(o[2 * c + 1][nr], f[4], f[5], f[6], f[7], pb[nr][0], pb[nr][1]);
          }
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(sm.cempty + 8 * stage);
    if (++stage == CF::kStages) {
      stage = 0;
      phase ^= 1u;
    }
    if (!(meta.x & kLast)) continue;
    // This warp's part: o[2 c + kk][nr][2 a + e] is dim 32 c + 4 g + kk + 2 a of row 8 nr + 2 q4 + e.
    const float vs = in_codes ? p.v_scale : 1.f;
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = warp * CF::kRows + 8 * nr + 2 * q4 + e;
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[nr][e] += __shfl_xor_sync(0xffffffffu, l[nr][e], d);
        if (g == 0) {
          sm.ref[row] = ref[nr][e];
          sm.sum[row] = l[nr][e];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<float4*>(sm.comb_o + row * kCombStride + 32 * c + 4 * g) =
              make_float4(o[2 * c][nr][e] * vs, o[2 * c + 1][nr][e] * vs, o[2 * c][nr][2 + e] * vs, o[2 * c + 1][nr][2 + e] * vs);
      }
    if (!join_warps<CF::kRows>(p, smem, tile_meta(sm, t), sync, wait)) return;
  }
}

template <class CF>
__global__ void __launch_bounds__(kThreads, CF::kMinBlocks) attn_kv4_mma_kernel(const __grid_constant__ Kv4Params kp) {
  extern __shared__ uint8_t smem_raw[];
  const AttnParams& p = kp.a;
  const Smem sm = carve<CF>(smem_raw, p.C);
  if (threadIdx.x == 0) {
    allow_dependent_launch();  // the merge may be scheduled as CTAs finish
#pragma unroll 1
    for (int s = 0; s < CF::kStages; ++s) {
      mbar_init(sm.cfull + 8 * s, 1);
      mbar_init(sm.cempty + 8 * s, kWarps);
    }
    mbar_init(sm.joined, kWarps);
    init_waits(p);
    *sm.issued = 0;
    fence_mbar_init();
  }
  __syncthreads();
  const Waiter wait{p.wait_ns < kPollBelowNs};
  if (threadIdx.x >= 32 * kWarps) run_loader<CF::kStages, 1>(kp, sm, wait);
  else run_consumer<CF>(kp, sm, wait);
  __syncthreads();
  if (threadIdx.x == 0) drain<CF::kStages>(p, sm);
}

using Cfg8 = Cfg<1, 2, 3>;
using Cfg16 = Cfg<2, 3, 2>;

// Every plan that kMaxCaches allows fits an SM.
static_assert(smem_bytes<Cfg8>(kMaxCaches) <= 227 * 1024 && smem_bytes<Cfg16>(kMaxCaches) <= 227 * 1024,
              "shared memory at the largest number of caches");

template <class CF>
cudaError_t set_smem(int C, size_t* smem) {
  *smem = smem_bytes<CF>(C);
  return cudaFuncSetAttribute(attn_kv4_mma_kernel<CF>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(*smem));
}

template <class CF>
cudaError_t occupancy_cfg(int C, int* ctas) {
  size_t smem;
  const cudaError_t e = set_smem<CF>(C, &smem);
  if (e != cudaSuccess) return e;
  return cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas, attn_kv4_mma_kernel<CF>, kThreads, smem);
}

template <class CF>
cudaError_t launch_cfg(const Kv4Params& kp, bool pdl, cudaStream_t stream) {
  size_t smem;
  const cudaError_t e = set_smem<CF>(kp.a.C, &smem);
  if (e != cudaSuccess) return e;
  return launch_maybe_pdl(attn_kv4_mma_kernel<CF>, dim3(kp.a.num_ctas), dim3(kThreads), smem, pdl, stream, kp);
}

}  // namespace

cudaError_t attn_kv4_mma_occupancy(int rows_per_unit, int C, int* ctas_per_sm) {
  return rows_per_unit == 8 ? occupancy_cfg<Cfg8>(C, ctas_per_sm) : occupancy_cfg<Cfg16>(C, ctas_per_sm);
}

cudaError_t launch_attn_kv4_mma(const Kv4Params& p, bool pdl, cudaStream_t stream) {
  return p.a.rows_per_unit == 8 ? launch_cfg<Cfg8>(p, pdl, stream) : launch_cfg<Cfg16>(p, pdl, stream);
}

}  // namespace kvshot
