// attn_kv4_mma.cu -- draft attention over a 4-bit target cache for stacks of up to 16 query rows per KV head, on
// mma.sync tensor cores, with an optional sliding window and sink tokens.
//
// What bounds it: 144 B per key and KV head come from HBM, and each of its 256 codes has to become an f16 before it can be
// multiplied: 128 conversions of two codes and 128 products with a scale per key, 8 of the kernel's ~15 (8 rows) to 19 (16)
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
//  - A warp takes 32 keys together: one vote on the references, two independent chains of products (64 ragged sequences
//    104 -> 97 us, 16 rows of 4 x 4 x 32k tokens 210 -> 174 with q's fragments in shared memory, which makes the registers
//    for it).
// A CTA is four warps, 32 keys of a tile each, and a loading warp; three CTAs share an SM (16 rows: two).  One more, in
// the fewer registers that leaves a thread, is slower (105 against 97 us; 16 rows 202 against 173), and so is one less (110).
// Measured, attention and merge: 8 rows, 64 sequences of 512 to 8192 tokens 94 us (3.9 TB/s, 0.57 of the copy's rate);
// 16 rows, 4 x 4 x 32k tokens 166 us (3.7 TB/s); 8 rows, a window of 4096 32 us; one sequence of 2048 tokens 12.3 us.
// It issues at half of the rate; what it waits for most is its own fixed latencies (1.2 cycles an instruction).
// From 17 rows on attn_kv4.cu is faster; at 16 it takes 168 us (4 x 4 x 32k) where this kernel takes 166, and 41.5 against
// 37.5 for 16 sequences of 4096 tokens.
#include <algorithm>
#include <climits>

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

template <int NR>
constexpr int kQChunk = NR * 32 * 16;  // bytes of a chunk's Q^T fragments

struct Smem : Ring {
  Rows* rows;
  uint32_t joined;      // barrier of the consumer warps
  uint32_t q;           // [chunk][row step][lane] 16 B: Q^T fragments of the piece's rows
  float* comb_o;        // [kWarps][rows][kCombStride] a piece's O of each warp
  float *ref, *sum;     // [kWarps][rows] its references and sums; then (ref) its weights
};

template <class CF>
__host__ __device__ constexpr size_t smem_bytes() {
  return 128 + CF::kStages * kStageSize + kQChunk<CF::kNR> * 4 + sizeof(float) * kWarps * CF::kRows * (kCombStride + 2) +
         sizeof(TileMeta) * kMetas + kFirstBytes + sizeof(Rows) + sizeof(uint64_t) * (2 * CF::kStages + 2) + sizeof(int) * 4;
}

template <class CF>
__device__ __forceinline__ Smem carve(uint8_t* raw) {
  Smem s;
  uint8_t* b = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~uintptr_t(127));
  s.ring = smem_addr(b);
  s.q = s.ring + CF::kStages * kStageSize;
  s.comb_o = reinterpret_cast<float*>(b + CF::kStages * kStageSize + 4 * kQChunk<CF::kNR>);
  s.ref = s.comb_o + kWarps * CF::kRows * kCombStride;
  s.sum = s.ref + kWarps * CF::kRows;
  TileMeta* meta = reinterpret_cast<TileMeta*>(s.sum + kWarps * CF::kRows);
  s.meta = smem_addr(meta);
  s.first = smem_addr(meta + kMetas);
  uint64_t* m = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(meta + kMetas) + kFirstBytes);
  s.cfull = smem_addr(m);
  s.cempty = s.cfull + 8 * CF::kStages;
  s.joined = s.cempty + 8 * CF::kStages;
  s.rows = reinterpret_cast<Rows*>(m + 2 * CF::kStages + 2);
  int* words = reinterpret_cast<int*>(s.rows + 1);
  s.issued = words;
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
// whole unit, else the normalised fp32 part + log2-domain lse.  All consumer threads.
template <int n>
__device__ __noinline__ bool join_warps(const AttnParams& p, const Smem& sm, const TileMeta& w, WarpSync& sync,
                                        const Waiter& wait) {
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
  const int lane = tid & 31;  // four dims, of a row of this warp
#pragma unroll 1
  for (int r = tid >> 5; r < rows; r += kWarps) {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float a = sm.ref[k * n + r];
      const float4 o = *reinterpret_cast<const float4*>(sm.comb_o + (k * n + r) * kCombStride + 4 * lane);
      v.x = fmaf(a, o.x, v.x);
      v.y = fmaf(a, o.y, v.y);
      v.z = fmaf(a, o.z, v.z);
      v.w = fmaf(a, o.w, v.w);
    }
    if (whole)
      reinterpret_cast<uint2*>(p.out + (orow0 + sm.rows->place[r]) * kHeadDim)[lane] =
          make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    else
      reinterpret_cast<float4*>(p.ws_o + (part + r) * kHeadDim)[lane] = v;
  }
  return true;
}

// A warp's part of a piece.
template <int NR>
struct State {
  float o[8][NR][4];  // o[2 c + kk][nr][2 a + e]: dim 32 c + 4 g + kk + 2 a of row 8 nr + 2 q4 + e
  float ref[NR][2], l[NR][2];  // rows 8 nr + 2 q4 + e; l: this lane's keys only
};

// Scores to P^T fragments: s[i][nr][2 a + e] is key 16 i + 8 a + g, row 8 nr + 2 q4 + e.  `units`: what O is multiplied
// with when it changes its units (then `change`), which moves the references, too.
template <int NR, int KG>
__device__ __forceinline__ void softmax_step(State<NR>& st, const float (&s)[KG][NR][4], float qs, bool change, float units,
                                             uint32_t (&pb)[KG][NR][2]) {
  float top[NR][2];
  bool grow = change;
#pragma unroll
  for (int nr = 0; nr < NR; ++nr)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float v = fmaxf(s[0][nr][e], s[0][nr][2 + e]);
#pragma unroll
      for (int i = 1; i < KG; ++i) v = max3(v, s[i][nr][e], s[i][nr][2 + e]);
      top[nr][e] = v;
      grow |= fmaf(v, qs, -st.ref[nr][e]) > kRefLimit;
    }
  if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float v = top[nr][e] * qs;
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
        const float to = v - st.ref[nr][e] > kRefLimit ? v - kRefBelow : st.ref[nr][e];
        const float alpha = ex2(st.ref[nr][e] - to), o_alpha = alpha * units;
        st.ref[nr][e] = to;
        st.l[nr][e] *= alpha;
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) {
          st.o[mt][nr][e] *= o_alpha;
          st.o[mt][nr][2 + e] *= o_alpha;
        }
      }
  }
#pragma unroll
  for (int i = 0; i < KG; ++i)
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const float e0 = ex2(fmaf(s[i][nr][2 * a], qs, -st.ref[nr][0])), e1 = ex2(fmaf(s[i][nr][2 * a + 1], qs, -st.ref[nr][1]));
        st.l[nr][0] += e0;
        st.l[nr][1] += e1;
        pb[i][nr][a] = movmatrix_trans(pack_f16x2(e0, e1));
      }
}

// Keys that the rows' masks hide: scores of keys `key` and `key` + 8 (of the tile) of s[...][nr][2 a + e].  Returns whether
// any row sees them, as bits.
template <int NR>
__device__ __forceinline__ uint32_t hide(float (&s)[NR][4], const Kv4Params& kp, const Rows& rows, const int4& meta, int rb,
                                         int key, int q4) {
  uint32_t seen = 0;
#pragma unroll 1
  for (int a = 0; a < 2; ++a) {
    const uint64_t all = rows_seeing(kp, rows, meta, rb, key + 8 * a), vis = all >> (2 * q4);
    seen |= static_cast<uint32_t>(any_row(rows, all)) << a;
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (!((vis >> (8 * nr + e)) & 1ull)) {
          if (a == 0) s[nr][e] = -INFINITY;
          else s[nr][2 + e] = -INFINITY;
        }
  }
  return seen;
}

// Prefix keys, 8 rows: a row of depth d sees the sinks and the positions from L + d - window on.  `from`: of rows 2 q4 + e.
__device__ __forceinline__ void hide_prefix(float (&s)[4], const int (&from)[2], const int4& meta, int sinks, int key) {
#pragma unroll
  for (int a = 0; a < 2; ++a) {
    const int at = key + 8 * a, pos = meta.y + at;
    const int bound = at >= meta.z ? INT_MIN : pos < sinks ? INT_MAX : pos;  // (no key: no row; a sink: every row)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (bound < from[e]) s[2 * a + e] = -INFINITY;
  }
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
  const uint32_t qaddr = sm.q + lane * 16;
  const uint32_t kscale = kScales + g * 8, vscale = kScales + kScaleBytes + q4 * 16;
  const uint32_t ksel = q4 & 2 ? 0x3311u : 0x2200u, vsel = g & 4 ? 0x7351u : 0x6240u;
  WarpSync sync{sm.joined, 0};
  State<NR> st;
  bool in_codes = false;                    // O is in units of the value codes (a warp without draft keys keeps it so)
  wait_for_prerequisite_grid();             // q and the outputs may be the preceding kernel's
  int stage = 0, rb = 0;
  uint32_t phase = 0;
#pragma unroll 1
  for (int t = -1;; ++t) {
    // The first piece begins (t = -1) before its first tile has landed, the others with theirs.
    int4 meta = make_int4(kFirst, 0, 0, 0);  // flags, key0, nkeys, L
    if (t >= 0) {
      if (!wait.landed(sm.cfull + 8 * stage, phase)) return;
      meta = tile_words(sm, t);
      if (meta.x & kStop) return;
    }
    const bool draft = meta.x & kDraft, masked = meta.x & kMasked;
    if ((meta.x & kFirst) && t != 0) {
      const TileMeta w = tile_meta_at(t < 0 ? sm.first : sm.meta + t % kMetas * sizeof(TileMeta));
      if (!(w.flags & kFirst)) continue;  // (a CTA without tiles: its stop is next)
      if (!sync(wait)) return;  // the piece before has been written out
      rb = w.rb;
      if (w.flags & kNewRows) {
        if (warp == 0) build_rows(kp, *sm.rows, CF::kRows, w.rb, w.seq, w.flags & kNewTree);
        if (!sync(wait)) return;
      }
      // Q^T fragments (f16), a chunk by each warp: lane (g, q4) holds dims 32 c + 8 q4 .. + 7 of row 8 nr + g, for the
      // chunk's two k-steps.
      const __nv_bfloat16* qrow =
          p.q + (static_cast<size_t>(w.c) * p.Nq * p.hq + w.h * p.G) * kHeadDim + 32 * warp + 8 * q4;
      const int rows = min(p.rows_per_unit, p.rows_total - w.rb * p.rows_per_unit);
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (8 * nr + g < rows)
          x = *reinterpret_cast<const uint4*>(qrow + static_cast<size_t>(sm.rows->place[8 * nr + g]) * kHeadDim);
        sts128(sm.q + warp * kQChunk<NR> + nr * 512 + lane * 16,
               make_uint4(bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(x.y), bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(x.w)));
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) st.o[mt][nr][0] = st.o[mt][nr][1] = st.o[mt][nr][2] = st.o[mt][nr][3] = 0.f;
        st.ref[nr][0] = st.ref[nr][1] = kNoRef;
        st.l[nr][0] = st.l[nr][1] = 0.f;
      }
      in_codes = true;
      if (!sync(wait)) return;
      if (t < 0) continue;
    }
    const uint32_t tile = sm.ring + stage * kStageSize;
    if (!draft) {
      // A warp takes two groups of the cache (32 keys) together.
      const int kw = 32 * warp;
      if (kw < meta.z) {
        const uint32_t at = tile + 2 * warp * kKv4Bytes;
        float s[2][NR][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) s[i][nr][0] = s[i][nr][1] = s[i][nr][2] = s[i][nr][3] = 0.f;
        uint32_t w[2][2][4];  // group, keys g and g + 8: a word of each chunk
        uint2 sk[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            ldmatrix_x4(at + i * kKv4Bytes + kaddr + 8 * a * kChunkBytes, w[i][a][0], w[i][a][1], w[i][a][2], w[i][a][3]);
            sk[i][a] = lds64(at + i * kKv4Bytes + kscale + 64 * a);
          }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint4 q[NR];
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) q[nr] = lds128(qaddr + c * kQChunk<NR> + nr * 512);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t f[2][4];
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const uint2 pair = scales_of(c < 2 ? sk[i][a].x : sk[i][a].y, 0, ksel);
              const uint32_t s2 = c & 1 ? pair.y : pair.x;
              e2m1x8_to_f16(w[i][a][c], f[a]);
#pragma unroll
              for (int k = 0; k < 4; ++k) f[a][k] = mul_f16x2(f[a][k], s2);
            }
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
              mma_f16(s[i][nr], f[0][0], f[1][0], f[0][1], f[1][1], q[nr].x, q[nr].y);
              mma_f16(s[i][nr], f[0][2], f[1][2], f[0][3], f[1][3], q[nr].z, q[nr].w);
            }
          }
        }
        if (masked) {
          // (8 rows by compares: a window of 4096 31.8 us, by the rows' bits 35.4.  At 16 rows the compares' registers cost
          // every tile: 4 x 4 x 32k tokens 171 us, by the bits 166.)
          if constexpr (NR == 1) {
            const int2 depth = *reinterpret_cast<const int2*>(sm.rows->depth + 2 * q4);
            const int from[2] = {kp.window > 0 ? meta.w + depth.x - kp.window : INT_MIN + 1,
                                 kp.window > 0 ? meta.w + depth.y - kp.window : INT_MIN + 1};
#pragma unroll
            for (int i = 0; i < 2; ++i) hide_prefix(s[i][0], from, meta, kp.sinks, kw + 16 * i + g);
          } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) hide<NR>(s[i], kp, *sm.rows, meta, rb, kw + 16 * i + g, q4);
          }
        }
        uint32_t pb[2][NR][2];
        softmax_step<NR, 2>(st, s, p.qscale * p.k_scale, false, 1.f, pb);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t vat = at + i * kKv4Bytes;
          uint32_t v[4][2];  // chunk; tokens 0..7 and 8..15
          ldmatrix_x4_trans(vat + vaddr, v[0][0], v[0][1], v[1][0], v[1][1]);
          ldmatrix_x4_trans(vat + vaddr + 2 * kChunkStride, v[2][0], v[2][1], v[3][0], v[3][1]);
          uint4 sc[2] = {lds128(vat + vscale), lds128(vat + vscale + 64)};  // tokens 2 q4, 2 q4 + 1 and those + 8
          if (masked) {
            // Keys that no row sees may hold anything, NaN scales among it: 0 times them must be 0.
            const int lo = kp.window > 0 ? meta.w + sm.rows->min_depth - kp.window : 0;
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const int key = kw + 16 * i + 8 * a + 2 * q4, pos = meta.y + key;
              if (key >= meta.z || (pos < lo && pos >= kp.sinks)) sc[a].x = sc[a].y = 0u;
              if (key + 1 >= meta.z || (pos + 1 < lo && pos + 1 >= kp.sinks)) sc[a].z = sc[a].w = 0u;
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
              mma_f16(st.o[2 * c][nr], f[0], f[1], f[2], f[3], pb[i][nr][0], pb[i][nr][1]);
              mma_f16(st.o[2 * c + 1][nr], f[4], f[5], f[6], f[7], pb[i][nr][0], pb[i][nr][1]);
            }
          }
        }
      }
    } else {
      // 16 keys to a warp, bf16 (the first two warps).
      const int kw = 16 * warp;
      if (kw < meta.z) {
        float s[1][NR][4];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) s[0][nr][0] = s[0][nr][1] = s[0][nr][2] = s[0][nr][3] = 0.f;
        const uint32_t krow = tile + (kw + g) * kDraftRow + 16 * q4;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint4 x = lds128(krow + 64 * c), y = lds128(krow + 8 * kDraftRow + 64 * c);
          const uint32_t f[8] = {bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(y.x), bf16x2_to_f16x2(x.y), bf16x2_to_f16x2(y.y),
                                 bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(y.z), bf16x2_to_f16x2(x.w), bf16x2_to_f16x2(y.w)};
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            const uint4 q = lds128(qaddr + c * kQChunk<NR> + nr * 512);
            mma_f16(s[0][nr], f[0], f[1], f[2], f[3], q.x, q.y);
            mma_f16(s[0][nr], f[4], f[5], f[6], f[7], q.z, q.w);
          }
        }
        const uint32_t seen = hide<NR>(s[0], kp, *sm.rows, meta, rb, kw + g, q4);
        // Of keys 8 a .. 8 a + 7, a bit in each lane of theirs: this lane's V are keys 2 q4 and 2 q4 + 1.
        const uint32_t live[2] = {__ballot_sync(0xffffffffu, seen & 1u) >> (8 * q4), __ballot_sync(0xffffffffu, seen & 2u) >> (8 * q4)};
        uint32_t pb[1][NR][2];
        softmax_step<NR, 1>(st, s, p.qscale, in_codes && p.v_scale != 1.f, in_codes ? p.v_scale : 1.f, pb);
        in_codes = false;
        const uint32_t vrow = tile + kDraftV + (kw + 2 * q4) * kDraftRow + 8 * g;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t f[8];
#pragma unroll
          for (int a = 0; a < 2; ++a) {  // keys 2 q4 + 8 a, + 1: dims 4 g .. 4 g + 3 of the chunk
            uint2 x = lds64(vrow + 8 * a * kDraftRow + 64 * c), y = lds64(vrow + (8 * a + 1) * kDraftRow + 64 * c);
            if (!(live[a] & 0x01u)) x = make_uint2(0u, 0u);  // (no row sees it, or there is no such key)
            if (!(live[a] & 0x10u)) y = make_uint2(0u, 0u);
            f[2 * a] = bf16x2_to_f16x2(__byte_perm(x.x, y.x, 0x5410));
            f[2 * a + 1] = bf16x2_to_f16x2(__byte_perm(x.y, y.y, 0x5410));
            f[4 + 2 * a] = bf16x2_to_f16x2(__byte_perm(x.x, y.x, 0x7632));
            f[4 + 2 * a + 1] = bf16x2_to_f16x2(__byte_perm(x.y, y.y, 0x7632));
          }
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            mma_f16(st.o[2 * c][nr], f[0], f[1], f[2], f[3], pb[0][nr][0], pb[0][nr][1]);
            mma_f16(st.o[2 * c + 1][nr], f[4], f[5], f[6], f[7], pb[0][nr][0], pb[0][nr][1]);
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
        for (int d = 4; d < 32; d <<= 1) st.l[nr][e] += __shfl_xor_sync(0xffffffffu, st.l[nr][e], d);
        if (g == 0) {
          sm.ref[row] = st.ref[nr][e];
          sm.sum[row] = st.l[nr][e];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<float4*>(sm.comb_o + row * kCombStride + 32 * c + 4 * g) =
              make_float4(st.o[2 * c][nr][e] * vs, st.o[2 * c + 1][nr][e] * vs, st.o[2 * c][nr][2 + e] * vs,
                          st.o[2 * c + 1][nr][2 + e] * vs);
      }
    if (!join_warps<CF::kRows>(p, smem, tile_meta(sm, t), sync, wait)) return;
  }
}

template <class CF>
__global__ void __launch_bounds__(kThreads, CF::kMinBlocks) attn_kv4_mma_kernel(const __grid_constant__ Kv4Params kp) {
  extern __shared__ uint8_t smem_raw[];
  const AttnParams& p = kp.a;
  const Smem sm = carve<CF>(smem_raw);
  if (threadIdx.x == 0) {
    allow_dependent_launch();  // the merge may be scheduled as CTAs finish
#pragma unroll 1
    for (int s = 0; s < CF::kStages; ++s) {
      mbar_init(sm.cfull + 8 * s, 1);
      mbar_init(sm.cempty + 8 * s, kWarps);
    }
    mbar_init(sm.joined, kWarps);
    init_waits(p);
    fence_mbar_init();
  }
  const bool loads = threadIdx.x >= 32 * kWarps;
  if (loads) plan_loader(kp, sm);
  __syncthreads();
  const Waiter wait(p);
  if (loads) run_loader<CF::kStages, 1>(kp, sm, wait);
  else run_consumer<CF>(kp, sm, wait);
  __syncthreads();
  if (threadIdx.x == 0) drain<CF::kStages>(p, sm);
}

using Cfg8 = Cfg<1, 2, 3>;
using Cfg16 = Cfg<2, 2, 2>;

template <class CF>
cudaError_t set_smem() {
  return cudaFuncSetAttribute(attn_kv4_mma_kernel<CF>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(smem_bytes<CF>()));
}

template <class CF>
cudaError_t occupancy_cfg(int* ctas) {
  const cudaError_t e = set_smem<CF>();
  if (e != cudaSuccess) return e;
  return cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas, attn_kv4_mma_kernel<CF>, kThreads, smem_bytes<CF>());
}

template <class CF>
cudaError_t launch_cfg(const Kv4Params& kp, bool pdl, cudaStream_t stream) {
  const cudaError_t e = set_smem<CF>();
  if (e != cudaSuccess) return e;
  return launch_maybe_pdl(attn_kv4_mma_kernel<CF>, dim3(kp.a.num_ctas), dim3(kThreads), smem_bytes<CF>(), pdl, stream, kp);
}

}  // namespace

cudaError_t attn_kv4_mma_occupancy(int rows_per_unit, int* ctas_per_sm) {
  return rows_per_unit == 8 ? occupancy_cfg<Cfg8>(ctas_per_sm) : occupancy_cfg<Cfg16>(ctas_per_sm);
}

cudaError_t launch_attn_kv4_mma(const Kv4Params& p, bool pdl, cudaStream_t stream) {
  return p.a.rows_per_unit == 8 ? launch_cfg<Cfg8>(p, pdl, stream) : launch_cfg<Cfg16>(p, pdl, stream);
}

}  // namespace kvshot
