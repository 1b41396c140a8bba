// attn_kv4.cu -- draft attention over a 4-bit target cache, with an optional sliding window and sink tokens: the call,
// its plan, and the kernel for stacks of 17 query rows and more per KV head, on the 5th-generation tensor cores (tcgen05).
// (Up to 16 rows: attn_kv4_mma.cu.)
//
// Per unit (cache, KV head, block of up to 64 stacked GQA rows), per tile of 128 keys, with keys as the MMA's M and the
// query rows as its N, so that few rows waste nothing:
//   S^T = K Q^T    M = 128 keys, N rows, K = 128 dims:  A = K (f16, tensor memory), B = Q (shared memory)
//   P^T = 2^(S^T qs - m)   a key to a thread; m per row moves only when a score passes it by 2^15 / 2^8
//   O^T += V^T P^T M = 128 dims, N rows, K = 128 keys:  A = V (f16, shared memory, MN-major), B = P (shared memory)
// The cache's bytes stream through a ring of tiles (one bulk copy per run of groups) and are decoded by warps of their
// own: a thread takes one key's codes, two per conversion (e2m1 -> f16, times the block's scale: both exact), K into
// tensor memory, V into shared memory.  P and q are rounded to f16 (11 bits: P in [2^-14, 2^15]), sums are fp32.
// Warp roles: a softmax warpgroup per 16 rows (thread = key, then dim), two decoding warpgroups (thread = key; the tiles
// t % 2 == w, K and then V), and a warp each that loads, issues QK^T and owns tensor memory, issues P.V, stages q.  A
// tile's buffers (K and S in tensor memory, V and P in shared memory) are pair t % 2.
//
// What bounds it: instructions.  A tile takes ~5300 warp instructions at 48 rows (3100 of softmax, 1600 of decoding), at
// 57% of the issue rate 0.85 us; its 18 KB are 0.41 us of the copy's bandwidth, its products 0.2 us.  Without the
// conversions a tile takes 0.79 us, without the exponentials 0.83, with a quarter of the products 0.85.  Beside the tiles,
// a call's 20 us are its start (5 us to the first scores), a piece's first tile, draft tiles and end (~6 us) and the merge.
// What the layout rests on (16 sequences of 4096 tokens):
//  - More softmax warps, not more rows to a thread: their steps wait for one another's latencies.  48 rows on two
//    warpgroups 61.7 us, on three 59.6; 32 rows, two warpgroups on tiles in turn 52.2, on 16 rows each of every tile 48.5.
//    Threads of 48 rows that take the scores twice (their registers hold the sums alone): 75 against 64.
//  - Little code in the tiles' path: the roles share an instruction cache that they about fill, and code that runs once
//    costs ~20 cycles an instruction.  So the plan is code of one warp, the other roles follow its words for each tile,
//    decoding is rolled, rare steps are out of line (48 rows 118 -> 69 us on the way).
//  - MMAs issued by an elected lane in uniform control flow: 10 cycles each, 45 by `if (lane == 0)`.
//  - What a piece needs beside its tiles is made beside them: rows' tables after q (69 -> 64 us), the CTA's plan and first
//    q before its first tile (64 -> 61.7), tables by jumps and whole nodes (59.6 -> 53.8), a warpgroup that ends its rows
//    by itself (53.5 -> 49.8).
// Measured, attention and merge: 32 rows 42 us, 48 rows 49.2, 64 rows 55.8, 256 rows 170 (the tree's 64 nodes in four
// blocks, each of which decodes the cache for itself).  Many short contexts cost their pieces: 82 caches of 5 tokens, 48
// rows, 656 pieces of three tiles 60 us (20k cycles each, most of it code fetched anew).
// Work plan: the units' tiles laid end to end and cut into equal ranges, one per persistent CTA (kvshot_internal.h);
// with a window a unit's tiles are those of the sinks and those of the window.
#include <algorithm>
#include <climits>
#include <cmath>

#include "kvshot_kv4_attn.cuh"
#include "kvshot_tcgen05.cuh"

namespace kvshot {
namespace {

using namespace tc;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

constexpr int kVHalf = kTile * 128;                // 64 dims of a tile's V: 128 rows of 128 bytes, 128-byte swizzle
constexpr int kVTile = 2 * kVHalf;
constexpr int kPTile = kTile * 128;                // P^T: a row of up to 64 query rows per key, 128-byte swizzle
constexpr int kCols = 16;                          // query rows of a softmax thread
constexpr int kGroupThreads = 128;                 // a warpgroup
constexpr int kBarTmem = 5;                        // named barrier: all but the loading warp and q's
constexpr int kBarGroup = 1;                       // named barriers 1 to 4: the threads of a softmax warpgroup
// NC: query rows of a unit, a multiple of 16 (and the MMAs' N).
template <int NC>
struct Cfg {
  static constexpr int kNC = NC;
  static constexpr int kGroups = NC / kCols;           // softmax warpgroups
  // Warps: the softmax warpgroups, two that decode, then the loading one, QK^T's, P.V's and q's.
  static constexpr int kWarpDecode = 4 * kGroups, kWarpLoad = kWarpDecode + 8, kWarpQk = kWarpLoad + 1,
                       kWarpQ = kWarpLoad + 3, kThreads = 32 * (kWarpLoad + 4);
  static constexpr int kStages = NC <= 32 ? 5 : 4;
  static constexpr int kQTile = NC * 256;
  static constexpr uint32_t kTmemK = 0, kTmemS = 128, kTmemO = 128 + 2 * NC;  // columns
  static constexpr uint32_t kTmemCols = kTmemO + NC <= 256 ? 256 : 512;
  static_assert(kTmemO + NC <= 512, "tensor memory");
};

struct Smem : Ring {
  Rows* rows;                        // [kRowSets]
  uint32_t v, p, q;                  // shared-memory addresses
  uint32_t kfull, vfull;             // [2] K, V decoded
  uint32_t qkdone, pfull, pvdone;    // [2] QK^T done; P written (and S read); P.V done
  uint32_t qfull, qempty;            // [2] q of a piece staged; its last QK^T done
  uint32_t ofree, mmadone;           // epilogue has read O; [2] every MMA issued is done
  uint32_t rfull, rfree;             // [kRowSets] a piece's rows built; the piece ended
  float *ref, *alpha;                // [64] per row (ref: negated)
  float* sums;                       // [softmax warp][16] of a piece's rows
  int* wmax;                         // [softmax warp][64] per warp and row
  uint32_t* tmem;
};

constexpr int kBarriers = 18 + 2 * kRowSets;  // besides the ring's (an even number: what follows is aligned to 16 bytes)

template <class CF>
__host__ __device__ constexpr size_t smem_bytes() {
  return 1024 + 2 * kVTile + 2 * kPTile + 2 * CF::kQTile + CF::kStages * kStageSize +
         sizeof(TileMeta) * kMetas + kFirstBytes + sizeof(uint64_t) * (2 * CF::kStages + kBarriers) + kRowSets * sizeof(Rows) +
         sizeof(int) * (2 * 64 + 4 * CF::kNC + CF::kGroups * 4 * 64 + 4);
}

template <class CF>
__device__ __forceinline__ Smem carve(uint8_t* raw) {
  Smem s;
  uint8_t* b = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  s.v = smem_addr(b);
  s.p = s.v + 2 * kVTile;
  s.q = s.p + 2 * kPTile;
  s.ring = s.q + 2 * CF::kQTile;
  b += 2 * kVTile + 2 * kPTile + 2 * CF::kQTile + CF::kStages * kStageSize;
  s.meta = smem_addr(b);
  s.first = s.meta + kMetas * sizeof(TileMeta);
  b += sizeof(TileMeta) * kMetas + kFirstBytes;
  s.cfull = smem_addr(b);
  s.cempty = s.cfull + 8 * CF::kStages;
  s.kfull = s.cempty + 8 * CF::kStages;
  s.vfull = s.kfull + 16;
  s.qkdone = s.vfull + 16;
  s.pfull = s.qkdone + 16;
  s.pvdone = s.pfull + 16;
  s.qfull = s.pvdone + 16;
  s.qempty = s.qfull + 16;
  s.mmadone = s.qempty + 16;
  s.ofree = s.mmadone + 16;
  s.rfull = s.ofree + 16;
  s.rfree = s.rfull + 8 * kRowSets;
  s.rows = reinterpret_cast<Rows*>(b + 8 * (2 * CF::kStages + kBarriers));
  s.ref = reinterpret_cast<float*>(s.rows + kRowSets);
  s.alpha = s.ref + 64;
  s.sums = s.alpha + 64;
  s.wmax = reinterpret_cast<int*>(s.sums + 4 * CF::kNC);
  s.tmem = reinterpret_cast<uint32_t*>(s.wmax + CF::kGroups * 4 * 64);
  s.issued = reinterpret_cast<int*>(s.tmem + 2);
  return s;
}

// q of every piece as f16, rows of 64 dims in two halves (K-major B of QK^T, 128-byte swizzle), and the rows' nodes.  This
// warp reads every tile's words, and counts among the readers of a stage, so that it cannot fall behind the ring.
template <class CF>
__device__ __forceinline__ void run_q(const Kv4Params& kp, const Smem& smem, const Waiter& wait) {
  const AttnParams& p = kp.a;
  const Smem sm = smem;
  const int lane = threadIdx.x & 31;
  wait_for_prerequisite_grid();
  int stage = 0, piece = 0, set = -1;
  uint32_t phase = 0;
#pragma unroll 1
  for (int t = -1;; ++t) {
    // The first piece's (t = -1) before its first tile has landed, the others' with theirs.
    TileMeta w = tile_meta_at(sm.first);
    if (t >= 0) {
      if (!wait.landed(sm.cfull + 8 * stage, phase)) return;
      w = tile_meta(sm, t);
      if (lane == 0) mbar_arrive(sm.cempty + 8 * stage);
      if (++stage == CF::kStages) {
        stage = 0;
        phase ^= 1u;
      }
      if (w.flags & kStop) return;
    }
    if (!(w.flags & kFirst) || t == 0) continue;
    const int b = piece & 1;
    if (!wait(sm.qempty + 8 * b, ((piece >> 1) & 1) ^ 1u)) return;
    const __nv_bfloat16* q = p.q + (static_cast<size_t>(w.c) * p.Nq * p.hq + w.h * p.G) * kHeadDim;
    const int row0 = w.rb * p.rows_per_unit, rows = min(p.rows_per_unit, p.rows_total - row0);
    // 16 bytes of two rows at a time per warp; eight loads of a lane on their way together.
    const int ch = lane & 15;
    const uint32_t dst = sm.q + b * CF::kQTile + (ch >> 3) * (CF::kNC * 128);
#pragma unroll 1
    for (int r0 = lane >> 4; r0 < CF::kNC; r0 += 16) {
      uint4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = r0 + 2 * i, nl = kp.by_group(row0 + r);
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows)
          x[i] = reinterpret_cast<const uint4*>(q + (static_cast<size_t>(nl) * p.hq + row0 + r - nl * p.G) * kHeadDim)[ch];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = r0 + 2 * i;
        sts128(dst + r * 128 + (((ch & 7) ^ (r & 7)) << 4),
               make_uint4(bf16x2_to_f16x2(x[i].x), bf16x2_to_f16x2(x[i].y), bf16x2_to_f16x2(x[i].z), bf16x2_to_f16x2(x[i].w)));
      }
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(sm.qfull + 8 * b);
    // A set's last reader is the end of a piece, at the latest of the fourth before this one.
    if (!wait(sm.rfree + 8 * (piece & (kRowSets - 1)), ((piece / kRowSets) & 1) ^ 1u)) return;
    if (w.flags & kNewRows) {
      // (A set of another row block has the tree of the one before it copied along.)
      const int before = set & (kRowSets - 1);
      set = (set + 1) & (kRowSets - 1);
      if (p.tree && !(w.flags & kNewTree)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) sm.rows[set].anc[lane + 32 * k] = sm.rows[before].anc[lane + 32 * k];
        __syncwarp();
      }
      build_rows(kp, sm.rows[set], CF::kNC, w.rb, w.seq, w.flags & kNewTree);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(sm.rfull + 8 * (piece & (kRowSets - 1)));
    ++piece;
  }
}

// ------------------------------------------------------------ decode

// 32 dims of one key (16 words) into its row of the V tile: 16-byte chunks 4 c .. 4 c + 3, 128-byte swizzle.
__device__ __forceinline__ void put_v(uint32_t row, uint32_t sw, int c, const uint32_t* o) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    sts128(row + (c >> 1) * kVHalf + ((((c & 1) * 4 + i) << 4) ^ sw),
           make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
}

// A draft tile's key (bf16 row at `src`, zeros past the valid keys) into tensor memory (K) or the V tile.
template <bool kV>
__device__ __noinline__ void decode_draft(uint32_t src, bool live, uint32_t dst, uint32_t sw) {
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    uint32_t o[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (live) x = lds128(src + (4 * c + i) * 16);
      o[4 * i] = bf16x2_to_f16x2(x.x);
      o[4 * i + 1] = bf16x2_to_f16x2(x.y);
      o[4 * i + 2] = bf16x2_to_f16x2(x.z);
      o[4 * i + 3] = bf16x2_to_f16x2(x.w);
    }
    if constexpr (kV) put_v(dst, sw, c, o);
    else tmem_st16(dst + 16 * c, o);
  }
}

// The codes of 32 dims of one key (a chunk) with the two scales in the low bytes of `scales`, as 16 f16x2 words.
__device__ __forceinline__ void decode32(uint32_t src, uint32_t scales, uint32_t (&o)[16]) {
  const uint4 x = lds128(src);
  const uint2 s = scale_pair(scales);
  decode16(x.x, x.y, s.x, o);
  decode16(x.z, x.w, s.y, o + 8);
}

// A decoding warpgroup: the tiles t % 2 == wg, a key to a thread.
template <class CF>
__device__ __forceinline__ void run_decode(const Kv4Params& kp, const Smem& smem, const Waiter& wait, uint32_t tmem) {
  const AttnParams& p = kp.a;
  const Smem sm = smem;
  const int lane = threadIdx.x & 31, key = threadIdx.x & 127, wg = (threadIdx.x >> 7) & 1;
  const uint32_t src0 = sm.ring + (key >> 4) * kKv4Bytes + (key & 15) * kChunkBytes;
  const uint32_t scale0 = kScales + (key & 15) * 8 - (key & 15) * kChunkBytes;  // from there
  const uint32_t draft0 = sm.ring + key * kDraftRow;
  const uint32_t kdst = tmem + (static_cast<uint32_t>(key & 96) << 16) + CF::kTmemK + 64 * wg;
  const uint32_t vdst = sm.v + wg * kVTile + key * 128, sw = static_cast<uint32_t>(key & 7) << 4;
  const uint32_t qkdone = sm.qkdone + 8 * wg, pvdone = sm.pvdone + 8 * wg, kfull = sm.kfull + 8 * wg, vfull = sm.vfull + 8 * wg;
  int stage = wg;
  uint32_t phase = 0, freed = 1;
#pragma unroll 1
  for (int t = wg;; t += 2) {
    // The tile's bytes; K's buffer: QK^T of its previous tile is done.
    uint32_t flags = tile_flags(sm, t);
    if (!wait.landed(sm.cfull + 8 * stage, phase, qkdone, freed)) return;
    tc_fence_after();
    if (!is_of(flags)) flags = tile_flags(sm, t);
    if (flags & kStop) {
      // (P.V of the tile before has to have seen its V, whose phase this one ends.)
      if (!wait(pvdone, freed)) return;
      if (lane == 0) {
        mbar_arrive(kfull);
        mbar_arrive(vfull);
      }
      return;
    }
    const bool draft = flags & kDraft;
    const uint32_t src = src0 + stage * kStageSize;
    if (!draft) {
      uint2 sc = lds64(src + scale0);
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t o[16];
        decode32(src + c * kChunkStride, sc.x, o);
        tmem_st16(kdst + 16 * c, o);
        sc.x = __funnelshift_r(sc.x, sc.y, 16);
        sc.y >>= 16;
      }
    } else {
      decode_draft<false>(draft0 + stage * kStageSize, key < tile_words(sm, t).z, kdst, sw);
    }
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(kfull);
    // V's buffer: P.V of its previous tile is done.
    if (!wait(pvdone, freed)) return;
    bool seen = true;
    if (flags & kMasked) {
      // Keys that no row sees count as zeros; whether one does, for drafts and in a window, the piece's rows say.  (The phase
      // is theirs: the fourth piece before has its rows, since they are built before q of the next piece is staged, and the
      // products of the tile before the last, whose K this warp has replaced, have had their q.)
      const int4 meta = tile_words(sm, t);
      const uint32_t piece = static_cast<uint32_t>(meta.x) >> kPieceShift, set = static_cast<uint32_t>(meta.x) >> kSetShift;
      if (draft || kp.window > 0) {
        if (!wait(sm.rfull + 8 * (piece % kRowSets), piece / kRowSets & 1u)) return;
        const Rows& rows = sm.rows[set % kRowSets];
        seen = any_row(rows, rows_seeing(kp, rows, meta, tile_meta(sm, t).rb, key));
      } else {
        seen = key < meta.z;
      }
    }
    if (!draft) {
      uint2 sc = lds64(src + scale0 + kScaleBytes);
      if (!seen) sc = make_uint2(0u, 0u);  // (any code times 0 is 0)
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t o[16];
        decode32(src + kVCodes + c * kChunkStride, sc.x, o);
        put_v(vdst, sw, c, o);
        sc.x = __funnelshift_r(sc.x, sc.y, 16);
        sc.y >>= 16;
      }
    } else {
      decode_draft<true>(draft0 + kDraftV + stage * kStageSize, seen, vdst, sw);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(sm.cempty + 8 * stage);
      mbar_arrive(vfull);
    }
    freed ^= 1u;
    stage += 2;
    if (stage >= CF::kStages) {
      stage -= CF::kStages;
      phase ^= 1u;
    }
  }
}

// ------------------------------------------------------------ MMA issue (one warp each)

// A value that is the same in every lane, known to be so.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_max_sync(0xffffffffu, x); }

template <class CF>
__device__ __forceinline__ void run_qk(const Smem& smem, const Waiter& wait, uint32_t tmem_base) {
  const Smem sm = smem;
  constexpr uint32_t idesc = idesc_f16(128, CF::kNC, false);
  const uint32_t tmem = uniform(tmem_base);
  const uint64_t q0 = smem_desc_sw128(sm.q, 16, 1024);
  int piece = -1;
#pragma unroll 1
  for (int t = 0, stops = 0; stops < 2; ++t) {
    const uint32_t b = t & 1, phase = (t >> 1) & 1;
    uint32_t flags = uniform(tile_flags(sm, t));
    if (!wait(sm.pfull + 8 * b, phase ^ 1u, sm.kfull + 8 * b, phase)) break;  // (S of the tile before the last has been read)
    if (!is_of(flags)) flags = uniform(tile_flags(sm, t));
    if (flags & kFirst) {
      ++piece;
      if (!wait(sm.qfull + 8 * (piece & 1), (piece >> 1) & 1)) break;
    }
    if (flags & kStop) {
      ++stops;  // (its S is nothing, and the softmax sees that)
    } else {
      tc_fence_after();
      const uint32_t d = tmem + CF::kTmemS + b * CF::kNC;
      uint32_t k = tmem + CF::kTmemK + 64 * b;
      uint64_t q = q0 + (piece & 1) * (CF::kQTile >> 4);
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {  // of the dims
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) tc_mma_tmem_a_elect(d, k + 8 * ks, q + 2 * ks, idesc, half + ks > 0);
        k += 32;
        q += CF::kNC * 128 >> 4;
      }
      if (flags & kLast) tc_commit_elect(sm.qempty + 8 * (piece & 1));
    }
    tc_commit_elect(sm.qkdone + 8 * b);
  }
  tc_commit_elect(sm.mmadone);
}

template <class CF>
__device__ __forceinline__ void run_pv(const Smem& smem, const Waiter& wait, uint32_t tmem_base) {
  const Smem sm = smem;
  constexpr uint32_t idesc = idesc_f16(128, CF::kNC, true, true);
  const uint32_t tmem = uniform(tmem_base);
  const uint64_t v0 = smem_desc_sw128(sm.v, kVHalf, 1024), p0 = smem_desc_sw128(sm.p, kPTile, 1024);
  int piece = -1, in_piece = 0;
#pragma unroll 1
  for (int t = 0;; ++t, ++in_piece) {
    const uint32_t b = t & 1, phase = (t >> 1) & 1;
    uint32_t flags = uniform(tile_flags(sm, t));
    if (!wait(sm.vfull + 8 * b, phase)) break;
    if (!is_of(flags)) flags = uniform(tile_flags(sm, t));
    if (flags & kStop) break;
    if (!wait(sm.pfull + 8 * b, phase)) break;
    if (flags & kFirst) {
      in_piece = 0;
      if (++piece > 0 && !wait(sm.ofree, (piece - 1) & 1)) break;
    }
    tc_fence_after();
    const uint32_t o = tmem + CF::kTmemO;
    uint64_t v = v0 + b * (kVTile >> 4), x = p0 + b * (kPTile >> 4);
    uint32_t more = in_piece > 0;  // the accumulator holds tiles of this piece
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int k16 = 0; k16 < kTile / 32; ++k16) {  // two 8-key groups of 1 KB each
        tc_mma_elect(o, v + k16 * 128, x + k16 * 128, idesc, more);
        more = 1;
      }
      v += kTile / 32 * 128;
      x += kTile / 32 * 128;
    }
    tc_commit_elect(sm.pvdone + 8 * b);
  }
  tc_commit_elect(sm.mmadone + 8);
}

// ------------------------------------------------------------ softmax and epilogue

// Whether `x` holds for any of the `threads` threads of a named barrier (all of which call it).
__device__ __forceinline__ bool any_of(int bar, int threads, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(x)), "r"(bar), "r"(threads)
      : "memory");
  return r != 0;
}

// Sums of the columns over the warp's lanes: N sums to 32 lanes by halving, then plain for what is left.  Lane's v[i],
// i < the final width, is then the sum of column column0 + i.
template <int N>
__device__ __forceinline__ int column_sums(float (&v)[N], int lane, int* column0) {
  int width = N, col = 0;
#pragma unroll
  for (int bit = 16; bit > 0; bit >>= 1) {
    if (width % 2 == 0) {
      width /= 2;
      const bool up = lane & bit;
      col += up ? width : 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < width) {
          const float send = up ? v[i] : v[i + width], keep = up ? v[i + width] : v[i];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
        }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < width) v[i] += __shfl_xor_sync(0xffffffffu, v[i], bit);
    }
  }
  *column0 = col;
  return width;
}

// The references of rows whose scores have passed their limit move: refs (negated), and alpha with what O and the sums are to be
// multiplied by.  The threads of warpgroup wg; n rows from the first of `scores`, `ref` and `alpha` on.
__device__ __noinline__ void move_references(int* wmax, float* refs, float* alpha, int wg, int n, uint32_t scores, float qs,
                                             uint32_t vis, bool fresh) {
  const int tid = threadIdx.x & 127, warp = tid >> 5;
#pragma unroll 1
  for (int j = 0; j < n; j += 8) {
    uint32_t s[8];
    tmem_ld8(scores + j, s);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = (vis >> (j + i)) & 1u ? __uint_as_float(s[i]) * qs : -INFINITY;
      const int m = __reduce_max_sync(0xffffffffu, ordered(x));
      if ((tid & 31) == 0) wmax[warp * 64 + j + i] = m;
    }
  }
  named_barrier_sync(kBarGroup + wg, kGroupThreads);
  if (tid < n) {
    const float m = unordered(max(max(wmax[tid], wmax[64 + tid]), max(wmax[128 + tid], wmax[192 + tid])));
    const float old = fresh ? kNoRef : -refs[tid], ref = m - old > kRefLimit ? m - kRefBelow : old;
    refs[tid] = -ref;
    alpha[tid] = ex2(old - ref);
  }
  named_barrier_sync(kBarGroup + wg, kGroupThreads);
}

// n rows of O of this thread's dim times alpha and vs.
__device__ __noinline__ void rescale_o(const float* alpha, int n, uint32_t o_cols, float vs) {
#pragma unroll 1
  for (int j = 0; j < n; j += 8) {
    uint32_t o[8];
    tmem_ld8(o_cols + j, o);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * (alpha[j + i] * vs));
    tmem_st8(o_cols + j, o);
  }
  tmem_wait_st();
}

// A piece's rows row .. row + kCols - 1, a warpgroup's, of this thread's dim: the final ones, or the piece's part in the
// workspace.  `sums`: [4][kCols] of the rows, by its warps; `refs`: negated.
__device__ __noinline__ void write_rows(const AttnParams& p, const Rows& rows, const TileMeta& w, int row, const float* sums,
                                        const float* refs, uint32_t o_cols, float units) {
  const int tid = threadIdx.x & 127, lane = tid & 31, j = lane % kCols;
  const bool whole = w.flags & kWhole;
  // (A part has room for all rows.)
  const int end = whole ? min(p.rows_per_unit, p.rows_total - w.rb * p.rows_per_unit) : p.rows_per_unit;
  const size_t row0 = static_cast<size_t>(w.c) * p.Nq * p.hq + w.h * p.G;
  const size_t part = static_cast<size_t>((w.c * p.hkv + w.h) * p.row_blocks + w.rb + blockIdx.x) * p.rows_per_unit + row;
  // Lane j: row + j.
  const float sum = (sums[j] + sums[kCols + j]) + (sums[2 * kCols + j] + sums[3 * kCols + j]);
  const float inv = sum == 0.f ? 0.f : __fdividef(units, sum);
  const int place = rows.place[row + j];
  if (tid < kCols && row + j < end) {
    const float lse2 = sum == 0.f ? -INFINITY : __log2f(sum) - refs[j];
    if (whole) p.lse[row0 + place] = lse2 * 0.69314718055994531f;
    else p.ws_lse[part + j] = lse2;
  }
  __nv_bfloat16* out = p.out + row0 * kHeadDim + tid;
  float* ws = p.ws_o + part * kHeadDim + tid;
#pragma unroll 1
  for (int i0 = 0; i0 < kCols; i0 += 4) {
    uint32_t o[4];
    tmem_ld4(o_cols + i0, o);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = __shfl_sync(0xffffffffu, inv, i0 + i);
      const int to = __shfl_sync(0xffffffffu, place, i0 + i);
      const float v = a != 0.f ? __uint_as_float(o[i]) * a : 0.f;
      if (!whole) ws[i * kHeadDim] = v;
      else if (row + i0 + i < end) out[static_cast<size_t>(to) * kHeadDim] = __float2bfloat16(v);
    }
    ws += 4 * kHeadDim;
  }
}

template <class CF>
__device__ __forceinline__ void run_softmax(const Kv4Params& kp, const Smem& smem, const Waiter& wait, uint32_t tmem) {
  constexpr int NC = kCols;
  const AttnParams& p = kp.a;
  const Smem sm = smem;
  const int lane = threadIdx.x & 31, key = threadIdx.x & 127, wg = threadIdx.x >> 7;
  const int col0 = wg * NC;  // this thread's first row
  const uint32_t trow = tmem + (static_cast<uint32_t>(key & 96) << 16);
  const uint32_t o_cols = trow + CF::kTmemO + col0;
  const uint32_t pdst = sm.p + key * 128, sw = static_cast<uint32_t>(key & 7) << 4;
  float* ref = sm.ref + col0;
  float* alpha = sm.alpha + col0;
  int* wmax = sm.wmax + 256 * wg;
  const int bar = kBarGroup + wg;
  float2 l[NC / 2];               // sums over this thread's keys
  bool in_codes = false;          // O is in units of the value codes
  wait_for_prerequisite_grid();   // outputs and scratch may be the preceding kernel's
  bool fresh = true;              // the piece has had no tile yet
  bool good = true;               // no wait of this warp has given up
  const float qs_prefix = p.qscale * p.k_scale;
  int set = -1, piece = -1;       // the piece's set of rows, and its number
  auto begin = [&](int t) {
    ++piece;
    if (tile_words(sm, t).x & kNewRows) set = (set + 1) & (kRowSets - 1);
#pragma unroll
    for (int j = 0; j < NC / 2; ++j) l[j] = make_float2(0.f, 0.f);
    in_codes = fresh = true;
  };
  auto rows_built = [&]() { return wait(sm.rfull + 8 * (piece & (kRowSets - 1)), (piece / kRowSets) & 1); };
  // A piece's end, at its last tile t: a warpgroup has all of its rows.
  auto end = [&](int t) {
    int col = 0;
    float sums[NC];
#pragma unroll
    for (int j = 0; j < NC / 2; ++j) {
      sums[2 * j] = l[j].x;
      sums[2 * j + 1] = l[j].y;
    }
    const int width = column_sums(sums, lane, &col);
    float* all = sm.sums + wg * 4 * NC;  // (read until this warpgroup's next vote)
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (i < width) all[(key >> 5) * NC + col + i] = sums[i];
    // O is at rest: P.V of the piece's last tile is done.
    const bool ok = wait(sm.pvdone + 8 * (t & 1), (t >> 1) & 1) && rows_built();
    if (any_of(bar, kGroupThreads, !ok)) return false;
    tc_fence_after();
    write_rows(p, sm.rows[set], tile_meta(sm, t), col0, all, ref, o_cols, in_codes ? p.v_scale : 1.f);
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(sm.ofree);
      mbar_arrive(sm.rfree + 8 * (piece & (kRowSets - 1)));
    }
    return true;
  };
#pragma unroll 1
  for (int t = 0;; ++t) {
    const int b = t & 1;
    const uint32_t phase = (t >> 1) & 1;
    // S, and with it the words of the tile and of those before it; and the buffer of P, free when P.V of the tile before
    // the last is done.  (A warp whose wait gives up goes on to the vote: the warps of a
    // warpgroup leave there, together.)
    uint32_t flags = tile_flags(sm, t);
    good = good && wait(sm.qkdone + 8 * b, phase, sm.pvdone + 8 * b, phase ^ 1u);
    if (!is_of(flags)) flags = tile_flags(sm, t);
    float qs = qs_prefix;
    uint32_t vis = ~0u;  // bits of this thread's rows that see the key
    bool stop = false, leave_codes = false, odd = !good;
    if (flags != 0 && good) {  // (most tiles have none)
      stop = flags & kStop;
      if ((flags & kFirst) && !stop) begin(t);
      if ((flags & kMasked) && !stop) {
        good = rows_built();
        if (good) vis = static_cast<uint32_t>(rows_seeing(kp, sm.rows[set], tile_words(sm, t), tile_meta(sm, t).rb, key) >> col0);
      }
      if (flags & kDraft) {
        qs = p.qscale;
        leave_codes = in_codes && !fresh && p.v_scale != 1.f;
        in_codes = false;
      }
      odd = !good || fresh || leave_codes || stop;
    }
    tc_fence_after();
    const uint32_t scores = trow + CF::kTmemS + b * CF::kNC + col0;
    float2 x[NC / 2];
    for (bool moved = false;; moved = true) {
      uint32_t s[NC];
      tmem_ld16(scores, s);
      tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < NC; j += 4) {
        const float4 m = *reinterpret_cast<const float4*>(ref + j);  // (negated)
        const float2 lo = make_float2(__uint_as_float(s[j]), __uint_as_float(s[j + 1]));
        const float2 hi = make_float2(__uint_as_float(s[j + 2]), __uint_as_float(s[j + 3]));
        x[j / 2] = fma2(lo, make_float2(qs, qs), make_float2(m.x, m.y));
        x[j / 2 + 1] = fma2(hi, make_float2(qs, qs), make_float2(m.z, m.w));
      }
      if (flags & kMasked) {
#pragma unroll
        for (int j = 0; j < NC; j += 2) {
          if (!((vis >> j) & 1u)) x[j / 2].x = -INFINITY;
          if (!((vis >> j) & 2u)) x[j / 2].y = -INFINITY;
        }
      }
      if (moved) break;
      float top = kRefLimit;
#pragma unroll
      for (int j = 0; j < NC / 2; ++j) top = max3(top, x[j].x, x[j].y);
      if (!any_of(bar, kGroupThreads, top > kRefLimit || odd)) break;
      if (any_of(bar, kGroupThreads, !good) || stop) return;
      move_references(wmax, ref, alpha, wg, NC, scores, qs, vis, fresh);  // always with a warpgroup's first keys of a piece
#pragma unroll
      for (int j = 0; j < NC / 2; ++j) {
        l[j].x *= alpha[2 * j];
        l[j].y *= alpha[2 * j + 1];
      }
      if (!fresh) {
        if (any_of(bar, kGroupThreads, !wait(sm.pvdone + 8 * (b ^ 1), ((t - 1) >> 1) & 1))) return;
        tc_fence_after();
        rescale_o(alpha, NC, o_cols, leave_codes ? p.v_scale : 1.f);
      }
    }
#pragma unroll
    for (int j = 0; j < NC; j += 8) {
      uint32_t pk[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 e = make_float2(ex2(x[j / 2 + i].x), ex2(x[j / 2 + i].y));
        l[j / 2 + i] = add2(l[j / 2 + i], e);
        pk[i] = pack_f16x2(e.x, e.y);
      }
      sts128(pdst + b * kPTile + ((static_cast<uint32_t>(col0 + j) << 1) ^ sw), make_uint4(pk[0], pk[1], pk[2], pk[3]));
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(sm.pfull + 8 * b);
    if (flags != 0) {
      fresh = false;
      if (flags & kLast) good = end(t);
    }
  }
}

// (With 28 warps a thread has 72 registers, and the plan inline would spill; the call costs 0.5 us, the spills 4.)
__device__ __noinline__ void plan_loader_apart(const Kv4Params& kp, const Ring& sm) { plan_loader(kp, sm); }

template <class CF>
__global__ void __launch_bounds__(CF::kThreads, 1) attn_kv4_kernel(const __grid_constant__ Kv4Params kp) {
  extern __shared__ uint8_t smem_raw[];
  const AttnParams& p = kp.a;
  if (threadIdx.x == 0) allow_dependent_launch();  // the merge may be scheduled as CTAs finish
  const Smem sm = carve<CF>(smem_raw);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) init_waits(p);
  if (threadIdx.x < 2 * CF::kStages + kBarriers) {
    // Arrivals, in the order of carve(): the ring (of a stage, a decoding warpgroup's warps and the one that stages q), K and
    // V decoded, then the rest.
    const int j = threadIdx.x - 2 * CF::kStages;
    const bool softmax = (j >> 1) == 3 || (j >> 1) == 8 || j >= 18 + kRowSets;  // P written, O read, a piece ended
    const int n = softmax ? 4 * CF::kGroups : j < -CF::kStages ? 1 : j < 0 ? 5 : j < 4 ? 4 : 1;
    mbar_init(sm.cfull + 8 * threadIdx.x, n);
    fence_mbar_init();
  }
  if (warp == CF::kWarpQ && (threadIdx.x & 31) < kMetas)  // (what an earlier CTA left there is of no tile)
    sts128(sm.meta + (threadIdx.x & 31) * sizeof(TileMeta), make_uint4(~0u, 0u, 0u, 0u));
  if (warp == CF::kWarpLoad) {
    if constexpr (CF::kThreads > 24 * 32) plan_loader_apart(kp, sm);
    else plan_loader(kp, sm);
  }
  __syncthreads();
  const Waiter wait(p);
  uint32_t tmem = 0;
  if (warp == CF::kWarpLoad) {
    run_loader<CF::kStages, 2>(kp, sm, wait);  // (a last word for each warpgroup)
  } else if (warp == CF::kWarpQ) {
    run_q<CF>(kp, sm, wait);
  } else {
    // The roles that use tensor memory wait for it (and the others need not).
    if (warp == CF::kWarpQk) {
      tmem_alloc(smem_addr(sm.tmem), CF::kTmemCols);
      tmem_relinquish();
    }
    tc_fence_before();
    named_barrier_sync(kBarTmem, CF::kThreads - 64);
    tc_fence_after();
    tmem = *sm.tmem;
    if (warp < CF::kWarpDecode) run_softmax<CF>(kp, sm, wait, tmem);
    else if (warp < CF::kWarpLoad) run_decode<CF>(kp, sm, wait, tmem);
    else if (warp == CF::kWarpQk) run_qk<CF>(sm, wait, tmem);
    else run_pv<CF>(sm, wait, tmem);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    // No copy or MMA outlives the CTA, whatever ended it (each wait is bounded).
    drain<CF::kStages>(p, sm);
    mbar_wait(sm.mmadone, 0, p.err);
    mbar_wait(sm.mmadone + 8, 0, p.err);
  }
  __syncthreads();
  tc_fence_after();
  if (warp == CF::kWarpQk) tmem_dealloc(tmem, CF::kTmemCols);
}

// Join the pieces of the units that the CTAs' ranges cut, out = sum_k 2^(lse_k - m) o_k / sum_k 2^(lse_k - m): a warp per
// row, lane = 4 dims.  blockIdx.x: a boundary between two ranges, whose unit it joins if it is the first one inside of it
// (or, units cut by themselves, the unit).  So the CTAs are as many as the cuts need: 256 rows of 16 sequences, 512 units
// of which 151 are cut, took 8 us of 174 with a warp for every row of all units.
constexpr int kMergeWarps = 8;  // rows of a CTA
// kMergeBatch: pieces loaded together.
template <int kMergeBatch, int kCtasPerSm>
__global__ void __launch_bounds__(32 * kMergeWarps, kCtasPerSm) merge_kv4_kernel(const __grid_constant__ Kv4Params kp) {
  const AttnParams& p = kp.a;
  // CTA 0 waits in any case: a kernel that depends on this grid alone then comes after the attention, too.
  if (blockIdx.x == 0 && blockIdx.y == 0) wait_for_prerequisite_grid();
  if (threadIdx.x == 0) allow_dependent_launch();
  const int lane = threadIdx.x & 31, r = blockIdx.y * kMergeWarps + (threadIdx.x >> 5);
  const RangeStart u = range_of<true>(kp);
  if (u.t >= u.t_end || (u.per == 0 && (u.lt == 0 || u.lt > u.tpc))) return;
  const int b0 = blockIdx.x * max(u.per, 1);  // the CTAs that held the unit
  const int b1 = u.per > 0 ? b0 + tiles_per_cta(u.ut, u.tpc) - 1 : (u.t - u.lt + u.ut - 1) / u.tpc;
  const int h = kp.by_blocks(u.hr), rb = u.hr - h * p.row_blocks, rr = rb * p.rows_per_unit + r, np = b1 - b0 + 1;
  if (np < 2 || r >= p.rows_per_unit || rr >= p.rows_total) return;
  const int nl = kp.by_group(rr);
  const size_t orow = (static_cast<size_t>(u.c) * p.Nq + nl) * p.hq + h * p.G + rr - nl * p.G;
  const size_t row0 = static_cast<size_t>(u.c * p.hkv * p.row_blocks + u.hr + b0) * p.rows_per_unit + r;
  const float4* parts = reinterpret_cast<const float4*>(p.ws_o + row0 * kHeadDim) + lane;
  const int stride = p.rows_per_unit * (kHeadDim / 4);  // from one piece's row to the next one's
  wait_for_prerequisite_grid();
  float m = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int k0 = 0; k0 < np; k0 += 32) {  // lane k: piece k0 + k
    const float ls = k0 + lane < np ? p.ws_lse[row0 + static_cast<size_t>(k0 + lane) * p.rows_per_unit] : -INFINITY;
    float w = 0.f;
#pragma unroll 1
    for (int k = 0; k < min(32, np - k0); k += kMergeBatch) {
      float4 x[kMergeBatch];  // (of the first batch, loaded beside the lse)
#pragma unroll
      for (int i = 0; i < kMergeBatch; ++i)
        x[i] = k0 + k + i < np ? parts[static_cast<size_t>(k0 + k + i) * stride] : make_float4(0.f, 0.f, 0.f, 0.f);
      if (k == 0) {
        float top = ls;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        top = fmaxf(top, m);
        const float keep = m == -INFINITY ? 0.f : exp2f(m - top);
        w = ls == -INFINITY ? 0.f : exp2f(ls - top);
        m = top;
        sum *= keep;
        acc = make_float4(acc.x * keep, acc.y * keep, acc.z * keep, acc.w * keep);
      }
#pragma unroll
      for (int i = 0; i < kMergeBatch; ++i) {
        const float a = __shfl_sync(0xffffffffu, w, k + i);  // 0 past the last piece
        sum += a;
        acc.x = fmaf(a, x[i].x, acc.x);
        acc.y = fmaf(a, x[i].y, acc.y);
        acc.z = fmaf(a, x[i].z, acc.z);
        acc.w = fmaf(a, x[i].w, acc.w);
      }
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  reinterpret_cast<uint2*>(p.out + orow * kHeadDim)[lane] =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  if (lane == 0) p.lse[orow] = sum > 0.f ? (m + log2f(sum)) * 0.69314718055994531f : -INFINITY;
}

constexpr int kMaxRows = 64;  // query rows of a unit

int rows_of_unit(int rows) {
  const int blocks = (rows + kMaxRows - 1) / kMaxRows, r = (rows + blocks - 1) / blocks;
  return r <= 8 ? 8 : (r + 15) / 16 * 16;
}

template <class CF>
cudaError_t launch_cfg(const Kv4Params& kp, bool pdl, cudaStream_t stream) {
  constexpr size_t smem = smem_bytes<CF>();
  static_assert(smem <= 227 * 1024, "shared memory");
  const cudaError_t e =
      cudaFuncSetAttribute(attn_kv4_kernel<CF>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  return launch_maybe_pdl(attn_kv4_kernel<CF>, dim3(kp.a.num_ctas), dim3(CF::kThreads), smem, pdl, stream, kp);
}

cudaError_t launch(const Kv4Params& kp, bool pdl, cudaStream_t stream) {
  switch (kp.a.rows_per_unit) {
    case 8:
    case 16: return launch_attn_kv4_mma(kp, pdl, stream);
    case 32: return launch_cfg<Cfg<32>>(kp, pdl, stream);
    case 48: return launch_cfg<Cfg<48>>(kp, pdl, stream);
    case 64: return launch_cfg<Cfg<64>>(kp, pdl, stream);
    default: return cudaErrorInvalidValue;
  }
}

kvshot_status check_attn_kv4(const kvshot_attn_desc* d, int32_t window, int32_t sinks) {
  if (kvshot_status st = check_common(d)) return st;
  if ((d->flags & ~(KVSHOT_TREE | KVSHOT_OVERLAP_PREVIOUS)) != 0) return KVSHOT_ERR_UNSUPPORTED;
  if (d->k_scale_exp < -64 || d->k_scale_exp > 64 || d->v_scale_exp < -64 || d->v_scale_exp > 64)
    return KVSHOT_ERR_SHAPE;
  if (window < 0 || sinks < 0) return KVSHOT_ERR_SHAPE;
  return KVSHOT_OK;
}

struct Plan {
  int rows_per_unit, row_blocks, units, num_ctas, draft_tiles;
  size_t off_o, bytes;
};

// Tiles that a CTA's range may grow by where that leaves it one piece, about what a second piece and the merge cost: of this
// kernel (64 rows, 16 sequences of 4096 tokens, 34 tiles instead of 29: 59.5 -> 55.8 us; 48 rows 50.3 -> 49.5), and of the
// other with 16 rows (12 instead of 9: 39.1 -> 37.8) and 8 (34.2 -> 33.2; with three a window of 4096 32.3 -> 32.9).  Of 75
// calls of 4 to 64 rows over 4 to 28 caches of 1500, 4100 or 9000 tokens none loses more than 0.8% against ranges laid end to
// end, and 35 gain 5% and more (48 rows, 17 caches of 1500: 33.1 -> 27.1 us).
constexpr int kSpareTiles = 6, kSpareTiles16 = 3, kSpareTiles8 = 1;

// Fewest tiles per CTA.  (One a CTA is no faster: a sequence of 2048 tokens takes 12.4 us with either.)
constexpr int64_t kMinTiles = 2;

kvshot_status make_kv4_plan(const kvshot_attn_desc* d, int32_t window, int32_t sinks, Plan* pl) {
  const int64_t rows = static_cast<int64_t>(d->hq / d->hkv) * d->n_query;
  if (rows >= INT_MAX / 2) return KVSHOT_ERR_UNSUPPORTED;
  pl->rows_per_unit = rows_of_unit(static_cast<int>(rows));
  pl->row_blocks = static_cast<int>((rows + pl->rows_per_unit - 1) / pl->rows_per_unit);
  pl->draft_tiles = (d->n_nodes + kDraftTile - 1) / kDraftTile;
  const int64_t units = static_cast<int64_t>(d->num_caches) * d->hkv * pl->row_blocks;
  int64_t prefix = (static_cast<int64_t>(d->max_seq_len) + kTile - 1) / kTile;
  if (window > 0) {  // at most: the sinks' tiles and the window's, each cut at both ends
    const int64_t seen =
        (static_cast<int64_t>(window) + kTile - 1) / kTile + 1 + (static_cast<int64_t>(sinks) + kTile - 1) / kTile;
    prefix = std::min(prefix, seen);
  }
  const int64_t max_tiles = units * (prefix + pl->draft_tiles);
  if (units >= INT_MAX / 2 || max_tiles >= INT_MAX / 2) return KVSHOT_ERR_UNSUPPORTED;
  pl->units = static_cast<int>(units);
  int64_t grid = d->num_ctas;
  if (grid == 0) {
    const int sms = sm_count();
    int per_sm = 1;
    if (pl->rows_per_unit <= 16 && attn_kv4_mma_occupancy(pl->rows_per_unit, &per_sm) != cudaSuccess)
      return KVSHOT_ERR_CUDA;
    if (sms < 1 || per_sm < 1) return KVSHOT_ERR_CUDA;
    grid = std::min<int64_t>(sms * per_sm, std::max((max_tiles + kMinTiles - 1) / kMinTiles, units));
  }
  pl->num_ctas = static_cast<int>(std::max<int64_t>(1, std::min(grid, max_tiles)));
  const size_t slots = static_cast<size_t>(pl->units) + pl->num_ctas;
  pl->off_o = round_up(sizeof(float) * slots * pl->rows_per_unit, 256);
  pl->bytes = pl->off_o + sizeof(float) * slots * pl->rows_per_unit * kHeadDim;
  return KVSHOT_OK;
}

}  // namespace
}  // namespace kvshot

using namespace kvshot;

extern "C" size_t kvshot_draft_attn_kv4_workspace_size(const kvshot_attn_desc* d, int32_t window, int32_t sinks) {
  if (check_attn_kv4(d, window, sinks) != KVSHOT_OK) return 0;
  if (d->n_query == 0) return 256;
  Plan pl;
  return make_kv4_plan(d, window, sinks, &pl) == KVSHOT_OK ? pl.bytes : 0;
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
  // Positions and the ends of tiles are 32-bit numbers, and so is a window's reach from a draft node.
  const int64_t room = paged ? static_cast<int64_t>(d->max_pages_per_seq) * d->page_size : d->l_cap;
  const int64_t len_bound = std::min<int64_t>(d->max_seq_len, room);
  if (len_bound + 2 * static_cast<int64_t>(d->n_nodes) > INT_MAX - kTile) return KVSHOT_ERR_UNSUPPORTED;
  if (d->n_query == 0) return KVSHOT_OK;
  if (!q || !cache || !seq_lens || !draft_k || !draft_v || !out || !lse || (tree && !tree_parent)) return KVSHOT_ERR_NULL;
  if (!aligned(q, 16) || !aligned(cache, 16) || !aligned(draft_k, 16) || !aligned(draft_v, 16) || !aligned(out, 16) ||
      !aligned(lse, 4) || !aligned(seq_lens, 4) || (paged && !aligned(page_table, 4)) || (tree && !aligned(tree_parent, 4)))
    return KVSHOT_ERR_ALIGN;
  Plan pl;
  if (kvshot_status st = make_kv4_plan(d, window, sinks, &pl)) return st;
  if (d->workspace == nullptr || !aligned(d->workspace, 256) || d->workspace_bytes < pl.bytes)
    return KVSHOT_ERR_WORKSPACE;
  Kv4Params kp = {};
  AttnParams& p = kp.a;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.page_table = page_table;
  p.seq_lens = seq_lens;
  p.tree_parent = tree_parent;
  p.err = d->err_flag;
  p.ws_lse = static_cast<float*>(d->workspace);
  p.ws_o = reinterpret_cast<float*>(static_cast<uint8_t*>(d->workspace) + pl.off_o);
  p.C = d->num_caches;
  p.B = d->num_seqs;
  p.hq = d->hq;
  p.hkv = d->hkv;
  p.G = d->hq / d->hkv;
  p.rows_total = p.G * d->n_query;
  p.rows_per_unit = pl.rows_per_unit;
  p.row_blocks = pl.row_blocks;
  p.paged = paged;
  p.page_size = paged ? d->page_size : d->l_cap;
  p.max_pages = paged ? d->max_pages_per_seq : 1;
  p.num_pages = paged ? d->num_pages : d->num_caches;
  p.len_bound = static_cast<int>(len_bound);
  p.N = d->n_nodes;
  p.Nq = d->n_query;
  p.n_max = d->n_max;
  p.tree = tree;
  p.draft_tiles = pl.draft_tiles;
  const double scale = d->scale != 0.f ? static_cast<double>(d->scale) : 1.0 / std::sqrt(static_cast<double>(kHeadDim));
  p.qscale = static_cast<float>(scale * 1.4426950408889634);
  p.num_ctas = pl.num_ctas;
  p.wait_ns = d->wait_limit_ns != 0 ? d->wait_limit_ns : 2000000000u;
  // (As for the fp8 cache: a prefix score's scale that underflows to 0 would make masked scores 0 * -inf.)
  p.k_scale = std::max(std::ldexp(1.f, d->k_scale_exp), std::ldexp(1.f, -100) / p.qscale);
  p.v_scale = std::ldexp(1.f, d->v_scale_exp);
  kp.window = window < static_cast<int64_t>(p.len_bound) + p.N ? window : 0;  // (a window that no key is out of is none)
  kp.sinks = sinks;
  kp.min_depth = tree ? 1 : d->n_nodes - d->n_query + 1;
  kp.cache = static_cast<const uint8_t*>(cache);
  kp.draft_k = static_cast<const __nv_bfloat16*>(draft_k);
  kp.draft_v = static_cast<const __nv_bfloat16*>(draft_v);
  kp.groups_per_page = p.page_size / kKv4Tokens;
  kp.run_groups = std::min(kTileGroups, kp.groups_per_page & -kp.groups_per_page);
  kp.by_page = Div::by(kp.groups_per_page);
  kp.by_blocks = Div::by(p.row_blocks);
  kp.by_seq = Div::by(p.C / p.B);
  kp.by_group = Div::by(p.G);
  kp.by_cache = Div::by(p.hkv * p.row_blocks);
  kp.ctas_per_unit = pl.num_ctas / pl.units;
  kp.spare_tiles = p.rows_per_unit == 8 ? kSpareTiles8 : p.rows_per_unit == 16 ? kSpareTiles16 : kSpareTiles;
  if (!paged) kp.run_groups = kTileGroups;  // one page: a tile's groups are neighbours
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (launch(kp, (d->flags & KVSHOT_OVERLAP_PREVIOUS) != 0, s) != cudaSuccess) return KVSHOT_ERR_CUDA;
  // A CTA takes whole units, whatever the lengths: nothing to merge.
  if (pl.num_ctas == 1 || (d->num_caches == 1 && (kp.ctas_per_unit == 1 || pl.units % pl.num_ctas == 0))) return KVSHOT_OK;
  const int rows = std::min(p.rows_per_unit, p.rows_total);
  const dim3 grid(pl.num_ctas - 1, (rows + kMergeWarps - 1) / kMergeWarps);
  const bool few = static_cast<int64_t>(grid.x) * grid.y <= 2 * static_cast<int64_t>(sm_count());
  const cudaError_t e = launch_maybe_pdl(few ? merge_kv4_kernel<8, 2> : merge_kv4_kernel<2, 6>, grid, dim3(32 * kMergeWarps), 0, true, s, kp);
  return e == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
