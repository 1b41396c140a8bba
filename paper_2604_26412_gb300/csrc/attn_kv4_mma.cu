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
#include <type_traits>

#include "kvshot_kv4_attn.cuh"

namespace kvshot {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = (kWarps + 1) * 32;
constexpr int kBarConsumers = 1;
constexpr int kCombStride = kHeadDim + 4;  // padded fp32 row of the combine buffer

// NR: 8-row steps.
template <int NR, int STAGES, int MINB>
struct Cfg {
  static constexpr int kNR = NR;
  static constexpr int kStages = STAGES;
  static constexpr int kMinBlocks = MINB;
  static constexpr int kRows = 8 * NR;
  static constexpr bool kQSmem = NR > 1;  // Q^T fragments: in registers for 8 rows, else in shared memory
};

struct Smem : Ring, Rows {
  uint2* qf;      // [8 k-steps][NR][32 lanes] Q^T fragments of the piece (kQSmem)
  float* comb_o;  // [rows][kCombStride]
  float* comb_m;  // [kWarps][rows]
  float* comb_l;  // [kWarps][rows]
  volatile int* abort;
  int* consumed;
};

template <class CF>
__host__ __device__ constexpr size_t smem_bytes(int C) {
  return 128 + CF::kStages * kStageSize + (CF::kQSmem ? 8 * CF::kNR * 32 * 8 : 0) +
         sizeof(float) * CF::kRows * (kCombStride + 2 * kWarps) + sizeof(uint64_t) * (2 * CF::kStages + 128) +
         sizeof(int) * (3 * 64 + 4 + 2 * C + 1);
}

template <class CF>
__device__ __forceinline__ Smem carve(uint8_t* raw, int C) {
  Smem s;
  uint8_t* b = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~uintptr_t(127));
  s.ring = smem_addr(b);
  s.comb_o = reinterpret_cast<float*>(b + CF::kStages * kStageSize);
  s.qf = reinterpret_cast<uint2*>(s.comb_o + CF::kRows * kCombStride);
  uint64_t* m = reinterpret_cast<uint64_t*>(s.qf + (CF::kQSmem ? 8 * CF::kNR * 32 : 0));
  s.cfull = smem_addr(m);
  s.cempty = s.cfull + 8 * CF::kStages;
  s.anc = m + 2 * CF::kStages;
  s.row_anc = s.anc + 64;
  s.comb_m = reinterpret_cast<float*>(s.row_anc + 64);
  s.comb_l = s.comb_m + kWarps * CF::kRows;
  s.depth = reinterpret_cast<int*>(s.comb_l + kWarps * CF::kRows);
  s.place = s.depth + 64;
  s.par = s.place + 64;
  s.abort = reinterpret_cast<volatile int*>(s.par + 64);
  s.issued = s.par + 65;
  s.consumed = s.par + 66;
  s.len = s.par + 68;
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

// Two e2m1 codes in each of the low two bytes -> two f16x2.
__device__ __forceinline__ uint2 e2m1x4_to_f16(uint32_t codes) {
  uint2 r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t}"
      : "=r"(r.x), "=r"(r.y)
      : "r"(codes));
  return r;
}

// Bits of a where m is set, of b elsewhere.
__device__ __forceinline__ uint32_t select_bits(uint32_t a, uint32_t b, uint32_t m) { return (a & m) | (b & ~m); }

// Combine the warps and write the piece: the final bf16 output + lse if it is the whole unit, else the normalised fp32
// part + log2-domain lse.  o[2 c + kk][nr][2 a + e]: dim 32 c + 4 g + kk + 2 a of row 8 nr + 2 q4 + e.
template <class CF>
__device__ __forceinline__ void finalize(const AttnParams& p, const Smem& sm, const Piece& w, float o_scale,
                                      float (&o)[8][CF::kNR][4], const float (&ref)[CF::kNR][2], float (&l)[CF::kNR][2]) {
  constexpr int NR = CF::kNR;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
#pragma unroll
  for (int nr = 0; nr < NR; ++nr)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[nr][e] += __shfl_xor_sync(0xffffffffu, l[nr][e], d);
      if (g == 0) {
        sm.comb_m[warp * CF::kRows + 8 * nr + 2 * q4 + e] = ref[nr][e];
        sm.comb_l[warp * CF::kRows + 8 * nr + 2 * q4 + e] = l[nr][e];
      }
    }
  named_barrier_sync(kBarConsumers, kWarps * 32);
  float top[NR][2], sum[NR][2];
#pragma unroll
  for (int nr = 0; nr < NR; ++nr)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 8 * nr + 2 * q4 + e;
      float mx = kNoRef, s = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) mx = fmaxf(mx, sm.comb_m[k * CF::kRows + row]);
#pragma unroll
      for (int k = 0; k < kWarps; ++k) s += ex2(sm.comb_m[k * CF::kRows + row] - mx) * sm.comb_l[k * CF::kRows + row];
      top[nr][e] = mx;
      sum[nr][e] = s;
      const float x = ex2(ref[nr][e] - mx) * o_scale;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        o[mt][nr][e] *= x;
        o[mt][nr][2 + e] *= x;
      }
    }
  const int row0 = w.rb * p.rows_per_unit, rows = min(p.rows_per_unit, p.rows_total - row0);
  const bool whole = w.whole();
  const size_t part = static_cast<size_t>(w.c * p.hkv * p.row_blocks + w.hr + blockIdx.x) * p.rows_per_unit;
  const size_t orow0 = static_cast<size_t>(w.c) * p.Nq * p.hq + w.h * p.G;
  // The warps add to the buffer one after another; the last one writes out.
#pragma unroll 1
  for (int k = 0; k < kWarps; ++k) {
    if (warp == k) {
#pragma unroll
      for (int nr = 0; nr < NR; ++nr)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int rl = 8 * nr + 2 * q4 + e;
          const float inv = sum[nr][e] == 0.f ? 0.f : 1.f / sum[nr][e];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float4* buf = reinterpret_cast<float4*>(sm.comb_o + rl * kCombStride + 32 * c + 4 * g);
            float4 v = make_float4(o[2 * c][nr][e], o[2 * c + 1][nr][e], o[2 * c][nr][2 + e], o[2 * c + 1][nr][2 + e]);
            if (k > 0) {
              const float4 a = *buf;
              v = make_float4(v.x + a.x, v.y + a.y, v.z + a.z, v.w + a.w);
            }
            if (k < kWarps - 1) {
              *buf = v;
            } else if (rl < rows) {
              if (whole)
                *reinterpret_cast<uint2*>(p.out + (orow0 + sm.place[rl]) * kHeadDim + 32 * c + 4 * g) =
                    make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
              else
                *reinterpret_cast<float4*>(p.ws_o + (part + rl) * kHeadDim + 32 * c + 4 * g) =
                    make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
            }
          }
          if (k == kWarps - 1 && g == 0 && rl < rows) {
            const float lse2 = sum[nr][e] == 0.f ? -INFINITY : top[nr][e] + __log2f(sum[nr][e]);
            if (whole) p.lse[orow0 + sm.place[rl]] = lse2 * 0.69314718055994531f;
            else p.ws_lse[part + rl] = lse2;
          }
        }
    }
    named_barrier_sync(kBarConsumers, kWarps * 32);
  }
}

template <class CF>
__device__ __forceinline__ void run_consumer(const Kv4Params& kp, const Smem& smem, const Waiter& wait, Piece next) {
  constexpr int NR = CF::kNR;
  const AttnParams& p = kp.a;
  const Smem sm = smem;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q4 = lane & 3;
  // This lane's places in a group: ldmatrix rows of K (chunk lane / 8, token lane % 8) and of V (chunk lane / 16, token
  // 8 (lane / 8 % 2) + lane % 8), the scales of its keys (K: token g; V: tokens 2 q4, 2 q4 + 1) and which of them it takes.
  const uint32_t kaddr = (lane >> 3) * kChunkStride + (lane & 7) * kChunkBytes;
  const uint32_t vaddr = kVCodes + (lane >> 4) * kChunkStride + (lane & 15) * kChunkBytes;
  const uint32_t kscale = kScales + g * 8, vscale = kScales + kScaleBytes + q4 * 16;
  const uint32_t ksel = q4 & 2 ? 0x3311u : 0x2200u, vsel = g & 4 ? 0x7351u : 0x6240u;
  uint2 qreg[CF::kQSmem ? 1 : 8] = {};
  uint2* qf = sm.qf + lane;
  auto q_frag = [&](int kstep, int nr) -> uint2 {
    if constexpr (CF::kQSmem) return qf[(kstep * NR + nr) * 32];
    else return qreg[kstep];
  };
  int stage = 0, consumed = 0, unit_rb = -1, unit_seq = -1;
  uint32_t phase = 0;
  bool live = true;
  wait_for_prerequisite_grid();  // q and the outputs may be the preceding kernel's
  while (next_piece(p, sm.len, next)) {
    const Piece w = next;
    if (w.rb != unit_rb || (p.tree && w.seq != unit_seq)) {
      load_rows(p, smem, CF::kRows, w.rb, w.seq, p.tree && w.seq != unit_seq, kBarConsumers, kWarps * 32);
      unit_rb = w.rb;
      unit_seq = w.seq;
      named_barrier_sync(kBarConsumers, kWarps * 32);
    }
    float o[8][NR][4], ref[NR][2], l[NR][2];  // rows 8 nr + 2 q4 + e; l: this lane's keys only
    {
      const int row0 = w.rb * p.rows_per_unit, rows = min(p.rows_per_unit, p.rows_total - row0);
      const __nv_bfloat16* q = p.q + (static_cast<size_t>(w.c) * p.Nq * p.hq + w.h * p.G) * kHeadDim + 8 * q4;
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        const int r = 8 * nr + g;
        constexpr int kChunks = CF::kQSmem ? 4 / kWarps : 4;  // chunks of 32 dims: the warps share them
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int c = CF::kQSmem ? warp * kChunks + i : i;
          uint4 x = make_uint4(0u, 0u, 0u, 0u);
          if (r < rows) x = *reinterpret_cast<const uint4*>(q + static_cast<size_t>(sm.place[r]) * kHeadDim + 32 * c);
          const uint2 f0 = make_uint2(bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(x.y));
          const uint2 f1 = make_uint2(bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(x.w));
          if constexpr (CF::kQSmem) {
            qf[(2 * c * NR + nr) * 32] = f0;
            qf[((2 * c + 1) * NR + nr) * 32] = f1;
          } else {
            qreg[2 * i] = f0;
            qreg[2 * i + 1] = f1;
          }
        }
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) o[mt][nr][0] = o[mt][nr][1] = o[mt][nr][2] = o[mt][nr][3] = 0.f;
        ref[nr][0] = ref[nr][1] = kNoRef;
        l[nr][0] = l[nr][1] = 0.f;
      }
      if constexpr (CF::kQSmem) named_barrier_sync(kBarConsumers, kWarps * 32);
    }
    int seen_from = 0;  // prefix tiles from here on (or before the sinks' end) are seen whole by every row
    if (p.window > 0) {
      int dmax = 0;
#pragma unroll 1
      for (int j = 0; j < CF::kRows; ++j) dmax = max(dmax, sm.depth[j]);
      seen_from = w.L + dmax - p.window;
    }
    bool in_codes = !w.draft(w.lt0);  // O is in units of the value codes
#pragma unroll 1
    for (int lt = w.lt0; lt < w.lt1; ++lt) {
      const bool draft = w.draft(lt);
      const int key0 = w.key0(lt), nkeys = w.nkeys(lt, p.N);
      const bool masked = draft || w.masked(lt, seen_from, p.sinks);
      const float qs = draft ? p.qscale : p.qscale * p.k_scale;
      live = __all_sync(0xffffffffu, live && wait(sm.cfull + 8 * stage, phase));
      const uint32_t tile = sm.ring + stage * kStageSize;
      // Softmax of M x 16 keys from key kw of the tile on: s to P^T fragments.  s[m][nr][2 a + e]: key kw + 16 m + 8 a + g.
      auto softmax = [&](auto& s, auto& pb, int kw) {
        constexpr int M = std::extent<std::remove_reference_t<decltype(s)>, 0>::value;
        if (masked) {
#pragma unroll
          for (int m = 0; m < M; ++m)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const int key = kw + 16 * m + 8 * a + g;
              const uint64_t vis = key < nkeys ? visible_rows(p, smem, 2 * q4, CF::kRows - 2 * q4, draft, key0 + key, w.L) : 0ull;
#pragma unroll
              for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (!((vis >> (8 * nr + e)) & 1ull)) s[m][nr][2 * a + e] = -INFINITY;
            }
        }
        bool grow = false;
        float mx[NR][2];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            mx[nr][e] = fmaxf(s[0][nr][e], s[0][nr][2 + e]);
            if constexpr (M == 2) mx[nr][e] = max3(mx[nr][e], s[1][nr][e], s[1][nr][2 + e]);
            mx[nr][e] *= qs;
            grow |= mx[nr][e] - ref[nr][e] > kRefLimit;
          }
        const bool leave_codes = draft && in_codes && p.v_scale != 1.f;  // warp-uniform
        if (__any_sync(0xffffffffu, grow || leave_codes)) {
#pragma unroll
          for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v = mx[nr][e];
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
              const float to = v - ref[nr][e] > kRefLimit ? v - kRefBelow : ref[nr][e];
              const float alpha = ex2(ref[nr][e] - to), o_alpha = leave_codes ? alpha * p.v_scale : alpha;
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
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
          for (int m = 0; m < M; ++m)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const float e0 = ex2(fmaf(s[m][nr][2 * a], qs, -ref[nr][0])), e1 = ex2(fmaf(s[m][nr][2 * a + 1], qs, -ref[nr][1]));
              l[nr][0] += e0;
              l[nr][1] += e1;
              pb[m][nr][a] = movmatrix_trans(pack_f16x2(e0, e1));
            }
      };
      if (live && !draft) {
        const int kw = 32 * warp;
        if (kw < nkeys) {
          float s[2][NR][4];
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const uint32_t grp = tile + (2 * warp + m) * kKv4Bytes;
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) s[m][nr][0] = s[m][nr][1] = s[m][nr][2] = s[m][nr][3] = 0.f;
            uint32_t a[4], b[4];  // rows g and g + 8: a word of each chunk
            ldmatrix_x4(grp + kaddr, a[0], a[1], a[2], a[3]);
            ldmatrix_x4(grp + kaddr + 8 * kChunkBytes, b[0], b[1], b[2], b[3]);
            const uint2 sa = lds64(grp + kscale), sb = lds64(grp + kscale + 64);
#pragma unroll
            for (int cc = 0; cc < 2; ++cc) {  // chunks 2 cc, 2 cc + 1
              const uint32_t pa = __byte_perm(cc ? sa.y : sa.x, 0, ksel), pb = __byte_perm(cc ? sb.y : sb.x, 0, ksel);
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int c = 2 * cc + i;
                const uint32_t s2a = e4m3x2_to_f16x2(i ? pa >> 16 : pa), s2b = e4m3x2_to_f16x2(i ? pb >> 16 : pb);
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
                  const uint2 q0 = q_frag(2 * c, nr), q1 = q_frag(2 * c + 1, nr);
                  mma_f16(s[m][nr], fa[0], fb[0], fa[1], fb[1], q0.x, q0.y);
                  mma_f16(s[m][nr], fa[2], fb[2], fa[3], fb[3], q1.x, q1.y);
                }
              }
            }
          }
          uint32_t pb[2][NR][2];
          softmax(s, pb, kw);
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const uint32_t grp = tile + (2 * warp + m) * kKv4Bytes;
            uint32_t v[4][2];  // chunk; tokens 0..7 and 8..15
            ldmatrix_x4_trans(grp + vaddr, v[0][0], v[0][1], v[1][0], v[1][1]);
            ldmatrix_x4_trans(grp + vaddr + 2 * kChunkStride, v[2][0], v[2][1], v[3][0], v[3][1]);
            uint4 sc[2] = {lds128(grp + vscale), lds128(grp + vscale + 64)};  // tokens 2 q4, 2 q4 + 1 and those + 8
            if (masked) {
              // Keys that no row sees may hold anything, NaN scales among it: 0 times them must be 0.
              const int lo = p.window > 0 ? w.L + p.min_depth - p.window : 0;
#pragma unroll
              for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const int key = kw + 16 * m + 8 * a + 2 * q4 + k, at = key0 + key;
                  if (key >= nkeys || (at < lo && at >= p.sinks)) {
                    if (k == 0) sc[a].x = sc[a].y = 0u;
                    else sc[a].z = sc[a].w = 0u;
                  }
                }
            }
#pragma unroll
            for (int cc = 0; cc < 2; ++cc) {
              uint32_t bytes[2];  // scales of (key, next key) for chunks 2 cc and 2 cc + 1
#pragma unroll
              for (int a = 0; a < 2; ++a) bytes[a] = __byte_perm(cc ? sc[a].y : sc[a].x, cc ? sc[a].w : sc[a].z, vsel);
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int c = 2 * cc + i;
                uint2 even[2], odd[2];  // dims 4 g, 4 g + 2 and 4 g + 1, 4 g + 3 of keys 2 q4, 2 q4 + 1 (+ 8)
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                  const uint32_t r = v[c][a], s2 = e4m3x2_to_f16x2(i ? bytes[a] >> 16 : bytes[a]);
                  even[a] = e2m1x4_to_f16(select_bits(r, r >> 12, 0x0f0fu));
                  odd[a] = e2m1x4_to_f16(select_bits(r >> 4, r >> 16, 0x0f0fu));
                  even[a].x = mul_f16x2(even[a].x, s2);
                  even[a].y = mul_f16x2(even[a].y, s2);
                  odd[a].x = mul_f16x2(odd[a].x, s2);
                  odd[a].y = mul_f16x2(odd[a].y, s2);
                }
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) {
                  mma_f16(o[2 * c][nr], even[0].x, even[0].y, even[1].x, even[1].y, pb[m][nr][0], pb[m][nr][1]);
                  mma_f16(o[2 * c + 1][nr], odd[0].x, odd[0].y, odd[1].x, odd[1].y, pb[m][nr][0], pb[m][nr][1]);
                }
              }
            }
          }
        }
      } else if (live && 16 * warp < nkeys) {
        // A draft tile: bf16 rows, 16 keys to a warp.
        const int kw = 16 * warp;
        float s[1][NR][4];
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) s[0][nr][0] = s[0][nr][1] = s[0][nr][2] = s[0][nr][3] = 0.f;
        const uint32_t krow = tile + (kw + g) * kDraftRow + 16 * q4;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          const uint4 x = lds128(krow + 64 * c), y = lds128(krow + 8 * kDraftRow + 64 * c);
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            uint2 q0, q1;
            if constexpr (CF::kQSmem) {
              q0 = q_frag(2 * c, nr);
              q1 = q_frag(2 * c + 1, nr);
            } else {
              q0 = c == 0 ? qreg[0] : c == 1 ? qreg[2] : c == 2 ? qreg[4] : qreg[6];
              q1 = c == 0 ? qreg[1] : c == 1 ? qreg[3] : c == 2 ? qreg[5] : qreg[7];
            }
            mma_f16(s[0][nr], bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(y.x), bf16x2_to_f16x2(x.y), bf16x2_to_f16x2(y.y), q0.x, q0.y);
            mma_f16(s[0][nr], bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(y.z), bf16x2_to_f16x2(x.w), bf16x2_to_f16x2(y.w), q1.x, q1.y);
          }
        }
        uint32_t pb[1][NR][2];
        softmax(s, pb, kw);
        const uint32_t vrow = tile + kDraftV + (kw + 2 * q4) * kDraftRow + 8 * g;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint2 x[4];  // keys 2 q4, 2 q4 + 1 and those + 8: dims 4 g .. 4 g + 3 of the chunk
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int key = (k & 1) + 8 * (k >> 1);
            x[k] = lds64(vrow + key * kDraftRow + 64 * c);
            if (kw + 2 * q4 + key >= nkeys) x[k] = make_uint2(0u, 0u);
          }
          auto pair = [](uint32_t a, uint32_t b, uint32_t sel) { return bf16x2_to_f16x2(__byte_perm(a, b, sel)); };
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) {
            mma_f16(o[2 * c][nr], pair(x[0].x, x[1].x, 0x5410), pair(x[0].y, x[1].y, 0x5410), pair(x[2].x, x[3].x, 0x5410),
                    pair(x[2].y, x[3].y, 0x5410), pb[0][nr][0], pb[0][nr][1]);
            mma_f16(o[2 * c + 1][nr], pair(x[0].x, x[1].x, 0x7632), pair(x[0].y, x[1].y, 0x7632),
                    pair(x[2].x, x[3].x, 0x7632), pair(x[2].y, x[3].y, 0x7632), pb[0][nr][0], pb[0][nr][1]);
          }
        }
      }  // (a warp without keys of the draft tiles keeps O in units of the codes)
      __syncwarp();
      if (live) {
        if (lane == 0) mbar_arrive(sm.cempty + 8 * stage);
        ++consumed;
      }
      if (++stage == CF::kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    finalize<CF>(p, sm, w, in_codes ? p.v_scale : 1.f, o, ref, l);
  }
  if (threadIdx.x == 0) *sm.consumed = consumed;
}

template <class CF>
__global__ void __launch_bounds__(kThreads, CF::kMinBlocks) attn_kv4_mma_kernel(const __grid_constant__ Kv4Params kp) {
  extern __shared__ uint8_t smem_raw[];
  const AttnParams& p = kp.a;
  if (threadIdx.x == 0) allow_dependent_launch();  // the merge may be scheduled as CTAs finish
  const Smem sm = carve<CF>(smem_raw, p.C);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int s = 0; s < CF::kStages; ++s) {
      mbar_init(sm.cfull + 8 * s, 1);
      mbar_init(sm.cempty + 8 * s, kWarps);
    }
    *sm.abort = 0;
    *sm.issued = 0;
    *sm.consumed = 0;
    fence_mbar_init();
  }
  build_kv4_plan(p, sm.len, sm.base);  // (barriers inside)
  const Waiter wait{p.err, p.wait_ns, sm.abort, p.wait_ns < kPollBelowNs};
  Piece w;
  begin_pieces(p, sm.len, sm.base, w);
  if (warp == kWarps) run_loader<CF::kStages>(kp, sm, wait, w);
  else run_consumer<CF>(kp, sm, wait, w);
  __syncthreads();
  if (threadIdx.x == 0) {  // no copy outlives the CTA, whatever ended it
    for (int k = *sm.consumed; k < *sm.issued; ++k)
      if (!mbar_wait(sm.cfull + 8 * (k % CF::kStages), (k / CF::kStages) & 1, p.err)) break;
  }
}

using Cfg8 = Cfg<1, 3, 3>;
using Cfg16 = Cfg<2, 4, 2>;

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
