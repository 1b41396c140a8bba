// attn_kv4.cu -- draft attention over a 4-bit target cache, with an optional sliding window and sink tokens, on the
// 5th-generation tensor cores (tcgen05).
//
// Per unit (cache, KV head, block of up to 64 stacked GQA rows), per tile of 128 keys, with keys as the MMA's M and the
// query rows as its N, so that few rows waste nothing:
//   S^T = K Q^T    M = 128 keys, N rows, K = 128 dims:  A = K (f16, tensor memory), B = Q (shared memory)
//   P^T = 2^(S^T qs - m)   a key to a thread; m per row moves only when a score passes it by 2^15 / 2^8
//   O^T += V^T P^T M = 128 dims, N rows, K = 128 keys:  A = V (f16, shared memory, MN-major), B = P (shared memory)
// The cache's bytes stream through a ring of tiles (one bulk copy per run of groups) and are decoded by warps of their
// own: a thread takes one key's codes, two per conversion (e2m1 -> f16, times the block's scale: both exact), K into
// tensor memory, V into shared memory.
// Warp roles: 0..3 softmax and epilogue (thread = key, then dim), 4..7 decode K, 8..11 decode V, 12 loads, 13 issues
// QK^T and owns tensor memory, 14 issues P.V, 15 stages q (f16).
// Work plan: the units' tiles laid end to end and cut into equal ranges, one per persistent CTA (kvshot_internal.h);
// with a window a unit's tiles are those of the sinks and those of the window.
#include <algorithm>
#include <climits>
#include <cmath>

#include "kvshot_attn_common.cuh"
#include "kvshot_kv4.cuh"
#include "kvshot_tcgen05.cuh"

namespace kvshot {
namespace {

using namespace dev;
using namespace kv4;
using namespace tc;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

constexpr int kTile = kKv4PrefixTile;              // keys per prefix tile
constexpr int kTileGroups = kTile / kKv4Tokens;
constexpr int kStageSize = kTileGroups * kKv4Bytes;
constexpr int kDraftTile = 32;                     // keys per draft tile: bf16 rows of K and V fill a stage
constexpr int kDraftRow = 2 * kHeadDim + 16;       // padded: rows 16 bytes apart mod 128, free of bank conflicts
constexpr int kDraftV = kDraftTile * kDraftRow;
static_assert(2 * kDraftV <= kStageSize, "a draft tile fits a stage");
constexpr int kVHalf = kTile * 128;                // 64 dims of a tile's V: 128 rows of 128 bytes, 128-byte swizzle
constexpr int kVTile = 2 * kVHalf;
constexpr int kPTile = kTile * 128;                // P^T: a row of up to 64 query rows per key, 128-byte swizzle
constexpr int kThreads = 16 * 32;
constexpr int kSoftmaxThreads = 128;
constexpr int kWarpK = 4, kWarpV = 8, kWarpLoad = 12, kWarpQk = 13, kWarpPv = 14, kWarpQ = 15;
constexpr int kBarSoftmax = 1;
// The reference of a row is 2^8 below the maximum it was taken from and moves when a score passes it by 2^15: P stays in
// f16's normal range for scores down to 2^-22 of the maximum and below its largest number.
constexpr float kRefBelow = 8.f, kRefLimit = 15.f;
constexpr float kNoRef = -1e30f;                   // no score yet

struct Kv4Params {
  AttnParams a;
  const uint8_t* cache;
  const __nv_bfloat16 *draft_k, *draft_v;
  int groups_per_page;
  int run_groups;  // groups of a tile that are always neighbours in memory (a power of two, at most kTileGroups)
};

// NC: query rows of a unit, a multiple of 8.
template <int NC>
struct Cfg {
  static constexpr int kNC = NC;
  static constexpr int kNT = (NC + 15) / 16 * 16;  // the MMA's N
  static constexpr int kStages = NC <= 16 ? 6 : NC <= 32 ? 5 : 4;
  static constexpr int kQTile = kNT * 256;
  static constexpr uint32_t kTmemK = 0, kTmemS = 128, kTmemO = 128 + 2 * kNT;  // columns
  static constexpr uint32_t kTmemCols = kTmemO + kNT <= 256 ? 256 : 512;
};

struct Smem {
  uint32_t v, p, q, ring;          // shared-memory addresses
  uint64_t *cfull, *cempty;        // [stages] bytes landed; read by the eight decode warps
  uint64_t *kfull, *kempty;        // [2] K decoded; QK^T done
  uint64_t *vfull;                 // [2] V decoded
  uint64_t *sfull, *pfull, *pvdone;  // [2] QK^T done; P written (and S read); P.V done
  uint64_t *qfull, *qempty;        // [2] q of a piece staged; its last QK^T done
  uint64_t* ofree;                 // epilogue has read O
  uint64_t* mmadone;               // [2]
  uint64_t* anc;                   // [64] each node's ancestors and itself (tree)
  uint64_t* row_anc;               // [64] those of each query row's node
  float *ref, *alpha, *inv;        // [64] per row
  int* depth;                      // [64] per row
  int* wmax;                       // [4][64] per warp and row; sums at a piece's end
  int* par;                        // [64]
  uint32_t* tmem;
  int* misc;                       // [0] abort, [1] tiles issued by the loader
  int *len, *base;
};

constexpr int kBarriers = 20;  // besides the ring's: 19, and one for the alignment of what follows

template <class CF>
__host__ __device__ constexpr size_t smem_bytes(int C) {
  return 1024 + 2 * kVTile + 2 * kPTile + 2 * CF::kQTile + CF::kStages * kStageSize +
         sizeof(uint64_t) * (2 * CF::kStages + kBarriers) + sizeof(uint64_t) * 128 + sizeof(int) * (64 * 9) +
         sizeof(int) * (4 + 2 * C + 1);
}

template <class CF>
__device__ __forceinline__ Smem carve(uint8_t* raw, int C) {
  Smem s;
  uint8_t* b = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  s.v = smem_addr(b);
  s.p = s.v + 2 * kVTile;
  s.q = s.p + 2 * kPTile;
  s.ring = s.q + 2 * CF::kQTile;
  uint64_t* m = reinterpret_cast<uint64_t*>(b + 2 * kVTile + 2 * kPTile + 2 * CF::kQTile + CF::kStages * kStageSize);
  s.cfull = m;
  s.cempty = s.cfull + CF::kStages;
  s.kfull = s.cempty + CF::kStages;
  s.kempty = s.kfull + 2;
  s.vfull = s.kempty + 2;
  s.sfull = s.vfull + 2;
  s.pfull = s.sfull + 2;
  s.pvdone = s.pfull + 2;
  s.qfull = s.pvdone + 2;
  s.qempty = s.qfull + 2;
  s.ofree = s.qempty + 2;
  s.mmadone = s.ofree + 1;
  s.anc = m + 2 * CF::kStages + kBarriers;
  s.row_anc = s.anc + 64;
  s.ref = reinterpret_cast<float*>(s.row_anc + 64);
  s.alpha = s.ref + 64;
  s.inv = s.alpha + 64;
  s.depth = reinterpret_cast<int*>(s.inv + 64);
  s.wmax = s.depth + 64;
  s.par = s.wmax + 4 * 64;
  s.tmem = reinterpret_cast<uint32_t*>(s.par + 64);
  s.misc = reinterpret_cast<int*>(s.tmem + 1);
  s.len = s.misc + 3;
  s.base = s.len + C;
  return s;
}

// ------------------------------------------------------------ work plan

__device__ __forceinline__ void build_kv4_plan(const AttnParams& p, int* s_len, int* s_base) {
  const int HR = p.hkv * p.row_blocks;
  for (int c = threadIdx.x; c < p.C; c += blockDim.x) {
    const int L = clamp_len(p, c);
    s_len[c] = L;
    s_base[c + 1] = (window_span<kTile>(p, L).tiles + p.draft_tiles) * HR;
  }
  __syncthreads();
  if (p.unit_ctas > 0) return;  // one cache: the cut needs its length alone
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, per = (p.C + 31) / 32, c0 = min(p.C, lane * per), c1 = min(p.C, c0 + per);
    int v = 0;
    for (int c = c0; c < c1; ++c) v += s_base[c + 1];
    int scan = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += t;
    }
    int below = scan - v;
    for (int c = c0; c < c1; ++c) {
      below += s_base[c + 1];
      s_base[c + 1] = below;
    }
    if (lane == 0) s_base[0] = 0;
  }
  __syncthreads();
}

struct Walk {
  int t, t_begin, t_end;  // tile of this CTA's range
  int c, hr, lt;          // cache, KV head x row block, tile of the unit
  int L, ut;              // prefix length, tiles of a unit
  WindowSpan span;

  __device__ __forceinline__ void load_cache(const AttnParams& p, const int* s_len) {
    L = s_len[c];
    span = window_span<kTile>(p, L);
    ut = span.tiles + p.draft_tiles;
  }
  __device__ __forceinline__ void begin(const AttnParams& p, const int* s_len, const int* s_base) {
    c = hr = lt = 0;
    t = t_begin = t_end = 0;
    if (p.unit_ctas > 0) {
      load_cache(p, s_len);
      const UnitCut u = unit_cut(p.unit_ctas, ut);
      hr = blockIdx.x / u.per;
      lt = (blockIdx.x - hr * u.per) * u.tpc;
      t_end = hr < p.hkv * p.row_blocks ? min(u.tpc, ut - lt) : 0;
      return;
    }
    const int total = s_base[p.C], tpc = tiles_per_cta(total, p.num_ctas);
    t = t_begin = min(total, static_cast<int>(blockIdx.x) * tpc);
    t_end = min(total, t + tpc);
    if (t >= t_end) return;
    int lo = 0, hi = p.C - 1;  // last cache whose first tile is <= t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_base[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
    c = lo;
    load_cache(p, s_len);
    const int rem = t - s_base[lo];
    hr = rem / ut;
    lt = rem - hr * ut;
  }
  __device__ __forceinline__ void next(const AttnParams& p, const int* s_len) {
    ++t;
    if (++lt == ut) {
      lt = 0;
      if (++hr == p.hkv * p.row_blocks) {
        hr = 0;
        ++c;
        if (t < t_end) load_cache(p, s_len);
      }
    }
  }
  __device__ __forceinline__ bool draft() const { return lt >= span.tiles; }
  __device__ __forceinline__ bool first() const { return t == t_begin || lt == 0; }
  __device__ __forceinline__ bool last() const { return t == t_end - 1 || lt == ut - 1; }
  // First key of the tile (token, or draft slot), and its valid keys.
  __device__ __forceinline__ int key0() const {
    return draft() ? (lt - span.tiles) * kDraftTile : (lt < span.sink_tiles ? lt : lt + span.skip) * kTile;
  }
  __device__ __forceinline__ int nkeys(const AttnParams& p) const {
    return draft() ? min(kDraftTile, p.N - key0()) : min(kTile, L - key0());
  }
};

// ------------------------------------------------------------ loads

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
               : "memory");
}

template <class CF>
__device__ __forceinline__ void run_loader(const Kv4Params& kp, const Smem& sm, Walk w) {
  const AttnParams& p = kp.a;
  volatile int* abort = &sm.misc[0];
  const int lane = threadIdx.x & 31;
  int stage = 0, issued = 0;
  uint32_t phase = 0;
  bool waited = false;
  const int runs = kTileGroups / kp.run_groups;
  // Page of this lane's run of groups in the tile at `w` (checked when it is used).
  auto page_of = [&](const Walk& x) {
    if (x.t >= x.t_end || x.draft() || lane >= runs) return 0;
    const int g = x.key0() / kKv4Tokens + lane * kp.run_groups;
    if (g * kKv4Tokens >= x.L) return 0;
    return p.paged ? p.page_table[static_cast<size_t>(x.c) * p.max_pages + g / kp.groups_per_page] : x.c;
  };
  int next_page = page_of(w);
  while (w.t < w.t_end) {
    const bool draft = w.draft();
    const int h = w.hr / p.row_blocks, key0 = w.key0(), nkeys = w.nkeys(p), c = w.c;
    int pid = next_page;
    w.next(p, sm.len);
    next_page = page_of(w);
    if (draft && !waited) {  // the draft K/V may come from the preceding kernel
      wait_for_prerequisite_grid();
      waited = true;
    }
    int ok = 1;
    if (lane == 0) ok = mbar_wait(smem_addr(&sm.cempty[stage]), phase ^ 1u, p.err, p.wait_ns) && !*abort;
    ok = __shfl_sync(0xffffffffu, ok, 0);
    if (!ok) {
      if (lane == 0) *abort = 1;
      break;
    }
    const uint32_t bar = smem_addr(&sm.cfull[stage]), dst = sm.ring + stage * kStageSize;
    if (draft) {
      if (lane == 0) mbar_arrive_expect_tx(bar, static_cast<uint32_t>(nkeys) * 4 * kHeadDim);
      __syncwarp();
      if (lane < nkeys) {
        const size_t row = (static_cast<size_t>(c) * p.hkv + h) * p.n_max + key0 + lane;
        bulk_load(dst + lane * kDraftRow, kp.draft_k + row * kHeadDim, 2 * kHeadDim, bar);
        bulk_load(dst + kDraftV + lane * kDraftRow, kp.draft_v + row * kHeadDim, 2 * kHeadDim, bar);
      }
    } else {
      const int groups = (nkeys + kKv4Tokens - 1) / kKv4Tokens;
      if (lane == 0) mbar_arrive_expect_tx(bar, static_cast<uint32_t>(groups) * kKv4Bytes);
      __syncwarp();
      const int g0 = lane * kp.run_groups, n = min(kp.run_groups, groups - g0);
      if (lane < runs && n > 0) {
        if (p.paged) pid = valid_page_id(p, pid);
        const int g = key0 / kKv4Tokens + g0, in_page = p.paged ? g % kp.groups_per_page : g;
        const uint8_t* src =
            kp.cache + ((static_cast<size_t>(pid) * p.hkv + h) * kp.groups_per_page + in_page) * kKv4Bytes;
        bulk_load(dst + g0 * kKv4Bytes, src, static_cast<uint32_t>(n) * kKv4Bytes, bar);
      }
    }
    ++issued;
    if (++stage == CF::kStages) {
      stage = 0;
      phase ^= 1u;
    }
  }
  if (lane == 0) sm.misc[1] = issued;
}

__device__ __forceinline__ uint32_t bf16x2_to_f16x2(uint32_t w) {
  const __half2 v = __floats2half2_rn(bf16_lo(w), bf16_hi(w));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
               : "memory");
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}

// q of every piece as f16, rows of 64 dims in two halves (K-major B of QK^T, 128-byte swizzle).
template <class CF>
__device__ __forceinline__ void run_q(const Kv4Params& kp, const Smem& sm, Walk w) {
  const AttnParams& p = kp.a;
  volatile int* abort = &sm.misc[0];
  const int lane = threadIdx.x & 31;
  wait_for_prerequisite_grid();
  int piece = 0;
  for (; w.t < w.t_end; w.next(p, sm.len)) {
    if (!w.first()) continue;
    const int b = piece & 1;
    const bool ok = __all_sync(0xffffffffu, mbar_wait(smem_addr(&sm.qempty[b]), ((piece >> 1) & 1) ^ 1u, p.err, p.wait_ns)) &&
                    !__any_sync(0xffffffffu, *abort);
    if (!ok) {
      *abort = 1;
      return;
    }
    const int h = w.hr / p.row_blocks, rb = w.hr - h * p.row_blocks;
#pragma unroll 4
    for (int i = lane; i < CF::kNT * 16; i += 32) {
      const int r = i >> 4, ch = i & 15, rr = rb * p.rows_per_unit + r;
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (r < p.rows_per_unit && rr < p.rows_total) {
        const int nl = rr / p.G, gh = rr - nl * p.G;
        x = *(reinterpret_cast<const uint4*>(
                  p.q + ((static_cast<size_t>(w.c) * p.Nq + nl) * p.hq + h * p.G + gh) * kHeadDim) +
              ch);
      }
      sts128(sm.q + b * CF::kQTile + (ch >> 3) * (CF::kNT * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4),
             make_uint4(bf16x2_to_f16x2(x.x), bf16x2_to_f16x2(x.y), bf16x2_to_f16x2(x.z), bf16x2_to_f16x2(x.w)));
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_addr(&sm.qfull[b]));
    ++piece;
  }
}

// ------------------------------------------------------------ decode

// 16 codes (8 bytes) of one block times its scale, as 8 f16x2 words.
__device__ __forceinline__ void decode16(uint32_t lo, uint32_t hi, uint32_t scale2, uint32_t* o) {
  uint32_t a[4], b[4];
  e2m1x8_to_f16(lo, a);
  e2m1x8_to_f16(hi, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[i] = mul_f16x2(a[i], scale2);
    o[4 + i] = mul_f16x2(b[i], scale2);
  }
}

// The scales of blocks 2 c and 2 c + 1, each in both halves.
__device__ __forceinline__ uint2 scale_pair(const uint2& sc, int c) {
  const uint32_t two = e4m3x2_to_f16x2(((c & 2) ? sc.y : sc.x) >> (16 * (c & 1)));
  return make_uint2(__byte_perm(two, two, 0x1010), __byte_perm(two, two, 0x3232));
}

// Warps 4..7 (K, into tensor memory) and 8..11 (V, into shared memory): a thread decodes one key.
template <class CF, bool kV>
__device__ __forceinline__ void run_decode(const Kv4Params& kp, const Smem& sm, uint32_t tmem, Walk w) {
  const AttnParams& p = kp.a;
  volatile int* abort = &sm.misc[0];
  const int lane = threadIdx.x & 31, key = threadIdx.x & 127;
  const uint32_t src = sm.ring + (key >> 4) * kKv4Bytes + (key & 15) * kChunkBytes + (kV ? kVCodes : 0);
  const uint32_t ssrc = sm.ring + (key >> 4) * kKv4Bytes + kScales + (kV ? kScaleBytes : 0) + (key & 15) * 8;
  const uint32_t dsrc = sm.ring + key * kDraftRow + (kV ? kDraftV : 0);
  const uint32_t trow = tmem + (static_cast<uint32_t>(key & 96) << 16) + CF::kTmemK;
  int stage = 0;
  uint32_t phase = 0;
  for (int t = 0; w.t < w.t_end; ++t, w.next(p, sm.len)) {
    const int nkeys = w.nkeys(p), b = t & 1;
    const bool draft = w.draft();
    // Keys that no row sees may hold anything; V of them must not be NaN (0 * NaN).
    bool live = key < nkeys;
    if (kV && !draft && p.window > 0) {
      const int k = w.key0() + key;
      live = live && (k >= w.L + p.min_depth - p.window || k < p.sinks);
    }
    bool ok = !*abort && mbar_wait(smem_addr(&sm.cfull[stage]), phase, p.err, p.wait_ns);
    // The buffer's previous tile has been multiplied.
    uint64_t* freed = kV ? &sm.pvdone[b] : &sm.kempty[b];
    auto wait_buffer = [&] {
      if (ok && t >= 2) ok = mbar_wait(smem_addr(freed), ((t >> 1) & 1) ^ 1u, p.err, p.wait_ns);
      ok = __all_sync(0xffffffffu, ok);
      if (kV) return;
      tc_fence_after();
    };
    const uint32_t vdst = sm.v + b * kVTile + key * 128, sw = static_cast<uint32_t>(key & 7) << 4;
    // 32 dims as 16 words.
    auto put = [&](int c, const uint32_t* o) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 4 * c + i;
        sts128(vdst + (ch >> 3) * kVHalf + ((static_cast<uint32_t>(ch & 7) << 4) ^ sw),
               make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
      }
    };
    if (__all_sync(0xffffffffu, ok)) {
      if (!draft) {
        uint4 x[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = lds128(src + stage * kStageSize + c * kChunkStride);
        uint2 sc = lds64(ssrc + stage * kStageSize);
        if (kV && !live) {
          sc = make_uint2(0u, 0u);
#pragma unroll
          for (int c = 0; c < 4; ++c) x[c] = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&sm.cempty[stage]));
        wait_buffer();
        if (ok) {
          if constexpr (kV) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              uint32_t o[16];
              const uint2 s2 = scale_pair(sc, c);
              decode16(x[c].x, x[c].y, s2.x, o);
              decode16(x[c].z, x[c].w, s2.y, o + 8);
              put(c, o);
            }
          } else {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              uint32_t o[32];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int c = 2 * hf + i;
                const uint2 s2 = scale_pair(sc, c);
                decode16(x[c].x, x[c].y, s2.x, o + 16 * i);
                decode16(x[c].z, x[c].w, s2.y, o + 16 * i + 8);
              }
              tmem_st32(trow + 64 * b + 32 * hf, o);
            }
          }
        }
      } else {
        wait_buffer();
        if (ok) {
#pragma unroll 1
          for (int hf = 0; hf < 2; ++hf) {
            uint32_t o[32];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              uint4 x = make_uint4(0u, 0u, 0u, 0u);
              if (live) x = lds128(dsrc + stage * kStageSize + (8 * hf + i) * 16);
              o[4 * i] = bf16x2_to_f16x2(x.x);
              o[4 * i + 1] = bf16x2_to_f16x2(x.y);
              o[4 * i + 2] = bf16x2_to_f16x2(x.z);
              o[4 * i + 3] = bf16x2_to_f16x2(x.w);
            }
            if constexpr (kV) {
              put(2 * hf, o);
              put(2 * hf + 1, o + 16);
            } else {
              tmem_st32(trow + 64 * b + 32 * hf, o);
            }
          }
        }
        __syncwarp();
        if (lane == 0 && ok) mbar_arrive(smem_addr(&sm.cempty[stage]));
      }
    } else {
      ok = false;
    }
    if (!ok) {
      *abort = 1;
      return;
    }
    if constexpr (kV) {
      fence_proxy_async_smem();
    } else {
      tmem_wait_st();
      tc_fence_before();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_addr(kV ? &sm.vfull[b] : &sm.kfull[b]));
    if (++stage == CF::kStages) {
      stage = 0;
      phase ^= 1u;
    }
  }
}

// ------------------------------------------------------------ MMA issue (one thread each)

template <class CF>
__device__ __forceinline__ void run_qk(const Kv4Params& kp, const Smem& sm, uint32_t tmem, Walk w) {
  const AttnParams& p = kp.a;
  volatile int* abort = &sm.misc[0];
  constexpr uint32_t idesc = idesc_f16(128, CF::kNT, false);
  int piece = -1;
  for (int t = 0; w.t < w.t_end; ++t, w.next(p, sm.len)) {
    const int b = t & 1;
    bool ok = !*abort;
    if (w.first()) {
      ++piece;
      ok = ok && mbar_wait(smem_addr(&sm.qfull[piece & 1]), (piece >> 1) & 1, p.err, p.wait_ns);
    }
    if (t >= 2) ok = ok && mbar_wait(smem_addr(&sm.pfull[b]), ((t >> 1) & 1) ^ 1u, p.err, p.wait_ns);  // S has been read
    ok = ok && mbar_wait(smem_addr(&sm.kfull[b]), (t >> 1) & 1, p.err, p.wait_ns);
    if (!ok) {
      *abort = 1;
      break;
    }
    tc_fence_after();
    const uint32_t q = sm.q + (piece & 1) * CF::kQTile;
#pragma unroll
    for (int ks = 0; ks < kHeadDim / 16; ++ks)
      tc_mma_tmem_a(tmem + CF::kTmemS + b * CF::kNT, tmem + CF::kTmemK + 64 * b + 8 * ks,
                    smem_desc_sw128(q + (ks >> 2) * (CF::kNT * 128) + (ks & 3) * 32, 16, 1024), idesc, ks > 0);
    tc_commit(smem_addr(&sm.sfull[b]));
    tc_commit(smem_addr(&sm.kempty[b]));
    if (w.last()) tc_commit(smem_addr(&sm.qempty[piece & 1]));
  }
  tc_commit(smem_addr(&sm.mmadone[0]));
}

template <class CF>
__device__ __forceinline__ void run_pv(const Kv4Params& kp, const Smem& sm, uint32_t tmem, Walk w) {
  const AttnParams& p = kp.a;
  volatile int* abort = &sm.misc[0];
  constexpr uint32_t idesc = idesc_f16(128, CF::kNT, true, true);
  int piece = -1;
  for (int t = 0; w.t < w.t_end; ++t, w.next(p, sm.len)) {
    const int b = t & 1;
    bool ok = !*abort;
    const bool first = w.first();
    if (first && ++piece > 0) ok = ok && mbar_wait(smem_addr(sm.ofree), (piece - 1) & 1, p.err, p.wait_ns);
    ok = ok && mbar_wait(smem_addr(&sm.vfull[b]), (t >> 1) & 1, p.err, p.wait_ns);
    ok = ok && mbar_wait(smem_addr(&sm.pfull[b]), (t >> 1) & 1, p.err, p.wait_ns);
    if (!ok) {
      *abort = 1;
      break;
    }
    tc_fence_after();
#pragma unroll
    for (int k16 = 0; k16 < kTile / 16; ++k16)  // two 8-key groups of 1 KB each
      tc_mma(tmem + CF::kTmemO, smem_desc_sw128(sm.v + b * kVTile + k16 * 2048, kVHalf, 1024),
             smem_desc_sw128(sm.p + b * kPTile + k16 * 2048, kPTile, 1024), idesc, !(first && k16 == 0));
    tc_commit(smem_addr(&sm.pvdone[b]));
  }
  tc_commit(smem_addr(&sm.mmadone[1]));
}

// ------------------------------------------------------------ softmax and epilogue

// Whether `x` holds for any of the softmax threads (all of which call it): a barrier with a reduction.
__device__ __forceinline__ bool any_softmax(bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(x)), "n"(kBarSoftmax), "n"(kSoftmaxThreads)
      : "memory");
  return r != 0;
}

// Floats as integers of the same order.
__device__ __forceinline__ int ordered(float f) {
  const int i = __float_as_int(f);
  return i >= 0 ? i : i ^ 0x7fffffff;
}
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i >= 0 ? i : i ^ 0x7fffffff); }

template <class CF>
__device__ __forceinline__ void run_softmax(const Kv4Params& kp, const Smem& sm, uint32_t tmem, Walk w) {
  constexpr int NC = CF::kNC;
  const AttnParams& p = kp.a;
  volatile int* abort = &sm.misc[0];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t trow = tmem + (static_cast<uint32_t>(tid & 96) << 16);
  const int HR = p.hkv * p.row_blocks;
  float l[NC];         // this thread's keys only
  int unit_rb = -1, unit_seq = -1, dmax = 0, piece_lt0 = 0, h = 0, rb = 0;
  bool in_codes = false;  // O is in units of the value codes
  wait_for_prerequisite_grid();  // outputs and scratch may be the preceding kernel's
  for (int t = 0; w.t < w.t_end; ++t, w.next(p, sm.len)) {
    const int b = t & 1, key0 = w.key0(), nkeys = w.nkeys(p);
    const bool draft = w.draft(), first = w.first();
    if (first) {
      h = w.hr / p.row_blocks;
      rb = w.hr - h * p.row_blocks;
      piece_lt0 = w.lt;
      in_codes = !draft;
      const int seq = w.c / (p.C / p.B);
      if (rb != unit_rb || (p.tree && seq != unit_seq)) {
        // The rows' nodes: depths and ancestors.
        if (p.tree && seq != unit_seq) {
          named_barrier_sync(kBarSoftmax, kSoftmaxThreads);
          for (int i = tid; i < p.N; i += kSoftmaxThreads) {
            int v = p.tree_parent[static_cast<size_t>(seq) * p.N + i];
            if (v < -1 || v >= i) {
              set_error(p.err, KVSHOT_ERR_TREE);
              v = -1;
            }
            sm.par[i] = v;
          }
          named_barrier_sync(kBarSoftmax, kSoftmaxThreads);
          for (int i = tid; i < p.N; i += kSoftmaxThreads) {
            uint64_t bits = 0;
            for (int m = i; m >= 0; m = sm.par[m]) bits |= 1ull << m;  // parents strictly decrease
            sm.anc[i] = bits;
          }
        }
        named_barrier_sync(kBarSoftmax, kSoftmaxThreads);
        if (tid < NC) {
          const int rr = min(rb * p.rows_per_unit + tid, p.rows_total - 1);
          const int node = p.N - p.Nq + rr / p.G;
          if (p.tree) sm.row_anc[tid] = sm.anc[node];
          sm.depth[tid] = p.tree ? __popcll(sm.anc[node]) : node + 1;
        }
        unit_rb = rb;
        unit_seq = seq;
      }
      if (tid < NC) sm.ref[tid] = kNoRef;
      named_barrier_sync(kBarSoftmax, kSoftmaxThreads);
      dmax = 0;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        dmax = max(dmax, sm.depth[j]);
        l[j] = 0.f;
      }
    }
    // Where the tile holds keys that some row does not see.
    const bool full = !draft && nkeys == kTile &&
                      (p.window == 0 || key0 >= w.L + dmax - p.window || key0 + kTile <= p.sinks);
    const float qs = draft ? p.qscale : p.qscale * p.k_scale;
    const int key = key0 + tid;
    int key_depth = 0;
    bool sink = false;
    if (draft && tid < nkeys) {
      key_depth = p.tree ? __popcll(sm.anc[key]) : key + 1;
      sink = w.L + key_depth - 1 < p.sinks;
    }
    auto sees = [&](int j) {  // row j sees this thread's key
      if (tid >= nkeys) return false;
      const int d = sm.depth[j];
      if (draft) {
        const bool line = p.tree ? (sm.row_anc[j] >> key) & 1ull : key < d;
        return line && (p.window == 0 || d - key_depth < p.window || sink);
      }
      return p.window == 0 || key >= w.L + d - p.window || key < p.sinks;
    };
    bool ok = !*abort && mbar_wait(smem_addr(&sm.sfull[b]), (t >> 1) & 1, p.err, p.wait_ns);
    ok = __all_sync(0xffffffffu, ok);
    tc_fence_after();
    float x[NC];
    auto load_scores = [&] {
      uint32_t s[NC];
      tmem_ld_cols<NC>(trow + CF::kTmemS + b * CF::kNT, s);
      tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < NC; ++j) x[j] = __uint_as_float(s[j]);
    };
    float top = -INFINITY;
    if (ok) {
      load_scores();
#pragma unroll
      for (int j = 0; j < NC; j += 4) {
        const float4 m = *reinterpret_cast<const float4*>(sm.ref + j);
        x[j] = fmaf(x[j], qs, -m.x);
        x[j + 1] = fmaf(x[j + 1], qs, -m.y);
        x[j + 2] = fmaf(x[j + 2], qs, -m.z);
        x[j + 3] = fmaf(x[j + 3], qs, -m.w);
      }
      if (!full) {
#pragma unroll
        for (int j = 0; j < NC; ++j)
          if (!sees(j)) x[j] = -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < NC; ++j) top = fmaxf(top, x[j]);
    }
    const bool leave_codes = draft && in_codes && p.v_scale != 1.f;
    if (any_softmax(top > kRefLimit || leave_codes || !ok)) {
      // A row's reference moves (always with a piece's first keys).
      if (any_softmax(!ok)) {
        *abort = 1;
        return;
      }
      load_scores();
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        x[j] = full || sees(j) ? x[j] * qs : -INFINITY;
        const int m = __reduce_max_sync(0xffffffffu, ordered(x[j]));
        if (lane == 0) sm.wmax[warp * 64 + j] = m;
      }
      named_barrier_sync(kBarSoftmax, kSoftmaxThreads);
      if (tid < NC) {
        const float m = unordered(max(max(sm.wmax[tid], sm.wmax[64 + tid]), max(sm.wmax[128 + tid], sm.wmax[192 + tid])));
        const float old = sm.ref[tid], ref = m - old > kRefLimit ? m - kRefBelow : old;
        sm.ref[tid] = ref;
        sm.alpha[tid] = ex2(old - ref);
      }
      named_barrier_sync(kBarSoftmax, kSoftmaxThreads);
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        l[j] *= sm.alpha[j];
        x[j] -= sm.ref[j];
      }
      if (!first) {
        ok = mbar_wait(smem_addr(&sm.pvdone[b ^ 1]), ((t - 1) >> 1) & 1, p.err, p.wait_ns);
        if (any_softmax(!ok)) {
          *abort = 1;
          return;
        }
        tc_fence_after();
        const float vs = leave_codes ? p.v_scale : 1.f;
        uint32_t o[NC];
        tmem_ld_cols<NC>(trow + CF::kTmemO, o);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < NC; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * (sm.alpha[j] * vs));
        tmem_st_cols<NC>(trow + CF::kTmemO, o);
        tmem_wait_st();
      }
    }
    if (draft) in_codes = false;
    // P's buffer is free when P.V of the tile before the last is done.
    ok = t < 2 || mbar_wait(smem_addr(&sm.pvdone[b]), ((t >> 1) & 1) ^ 1u, p.err, p.wait_ns);
    const uint32_t pdst = sm.p + b * kPTile + tid * 128, sw = static_cast<uint32_t>(tid & 7) << 4;
#pragma unroll
    for (int j = 0; j < NC; j += 8) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = ex2(x[j + i]);
        l[j + i] += e[i];
      }
      if (ok)
        sts128(pdst + ((static_cast<uint32_t>(j) << 1) ^ sw),
               make_uint4(pack_f16x2(e[0], e[1]), pack_f16x2(e[2], e[3]), pack_f16x2(e[4], e[5]), pack_f16x2(e[6], e[7])));
    }
    fence_proxy_async_smem();
    tc_fence_before();
    ok = __all_sync(0xffffffffu, ok);
    if (lane == 0 && ok) mbar_arrive(smem_addr(&sm.pfull[b]));
    if (!ok) *abort = 1;  // (the next vote takes every softmax thread out)
    if (w.last()) {
      // Sums over the keys' threads, then the rows.
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        float v = l[j];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (lane == 0) sm.wmax[warp * 64 + j] = __float_as_int(v);
      }
      ok = ok && mbar_wait(smem_addr(&sm.pvdone[b]), (t >> 1) & 1, p.err, p.wait_ns);
      if (any_softmax(!ok)) {
        *abort = 1;
        return;
      }
      tc_fence_after();
      const bool whole = piece_lt0 == 0 && w.lt == w.ut - 1;
      const int slot = w.c * HR + w.hr + blockIdx.x;
      const int rows = min(p.rows_per_unit, p.rows_total - rb * p.rows_per_unit);
      auto out_row = [&](int j) {
        const int rr = rb * p.rows_per_unit + j, nl = rr / p.G;
        return (static_cast<size_t>(w.c) * p.Nq + nl) * p.hq + h * p.G + rr - nl * p.G;
      };
      if (tid < NC) {
        const float sum = (__int_as_float(sm.wmax[tid]) + __int_as_float(sm.wmax[64 + tid])) +
                          (__int_as_float(sm.wmax[128 + tid]) + __int_as_float(sm.wmax[192 + tid]));
        sm.inv[tid] = sum > 0.f ? (in_codes ? p.v_scale : 1.f) / sum : sum == 0.f ? 0.f : sum;  // (NaN stays)
        const float lse2 = sum == 0.f ? -INFINITY : sm.ref[tid] + __log2f(sum);
        if (tid < rows) {
          if (whole) p.lse[out_row(tid)] = lse2 * 0.69314718055994531f;
          else p.ws_lse[static_cast<size_t>(slot) * p.rows_per_unit + tid] = lse2;
        }
      }
      uint32_t o[NC];
      tmem_ld_cols<NC>(trow + CF::kTmemO, o);
      tmem_wait_ld();
      tc_fence_before();
      named_barrier_sync(kBarSoftmax, kSoftmaxThreads);  // (and wmax has been read)
      if (lane == 0) mbar_arrive(smem_addr(sm.ofree));
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        if (j >= rows) break;
        const float v = __uint_as_float(o[j]) * sm.inv[j];
        if (whole) p.out[out_row(j) * kHeadDim + tid] = __float2bfloat16(v);
        else p.ws_o[(static_cast<size_t>(slot) * p.rows_per_unit + j) * kHeadDim + tid] = v;
      }
    }
  }
}

template <class CF>
__global__ void __launch_bounds__(kThreads, 1) attn_kv4_kernel(const __grid_constant__ Kv4Params kp) {
  extern __shared__ uint8_t smem_raw[];
  const AttnParams& p = kp.a;
  if (threadIdx.x == 0) allow_dependent_launch();  // the merge may be scheduled as CTAs finish
  const Smem sm = carve<CF>(smem_raw, p.C);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < CF::kStages; ++s) {
      mbar_init(smem_addr(&sm.cfull[s]), 1);
      mbar_init(smem_addr(&sm.cempty[s]), 8);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_addr(&sm.kfull[b]), 4);
      mbar_init(smem_addr(&sm.kempty[b]), 1);
      mbar_init(smem_addr(&sm.vfull[b]), 4);
      mbar_init(smem_addr(&sm.sfull[b]), 1);
      mbar_init(smem_addr(&sm.pfull[b]), 4);
      mbar_init(smem_addr(&sm.pvdone[b]), 1);
      mbar_init(smem_addr(&sm.qfull[b]), 1);
      mbar_init(smem_addr(&sm.qempty[b]), 1);
      mbar_init(smem_addr(&sm.mmadone[b]), 1);
    }
    mbar_init(smem_addr(sm.ofree), 4);
    sm.misc[0] = sm.misc[1] = 0;
    fence_mbar_init();
  }
  if (warp == kWarpQk) {
    tmem_alloc(smem_addr(sm.tmem), CF::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  build_kv4_plan(p, sm.len, sm.base);  // (barriers inside)
  tc_fence_after();
  const uint32_t tmem = *sm.tmem;
  Walk w;
  w.begin(p, sm.len, sm.base);
  if (warp < kWarpK) run_softmax<CF>(kp, sm, tmem, w);
  else if (warp < kWarpV) run_decode<CF, false>(kp, sm, tmem, w);
  else if (warp < kWarpLoad) run_decode<CF, true>(kp, sm, tmem, w);
  else if (warp == kWarpLoad) run_loader<CF>(kp, sm, w);
  else if (warp == kWarpQk && lane == 0) run_qk<CF>(kp, sm, tmem, w);
  else if (warp == kWarpPv && lane == 0) run_pv<CF>(kp, sm, tmem, w);
  else if (warp == kWarpQ) run_q<CF>(kp, sm, w);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0) {
    // No copy or MMA outlives the CTA, whatever ended it (each wait is bounded).
    for (int k = max(0, sm.misc[1] - CF::kStages); k < sm.misc[1]; ++k)
      if (!mbar_wait(smem_addr(&sm.cfull[k % CF::kStages]), (k / CF::kStages) & 1, p.err)) break;
    mbar_wait(smem_addr(&sm.mmadone[0]), 0, p.err);
    mbar_wait(smem_addr(&sm.mmadone[1]), 0, p.err);
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kWarpQk) tmem_dealloc(tmem, CF::kTmemCols);
}

constexpr int kMaxRows = 64;  // query rows of a unit

int rows_of_unit(int rows) {
  const int blocks = (rows + kMaxRows - 1) / kMaxRows, r = (rows + blocks - 1) / blocks;
  return r <= 8 ? 8 : (r + 15) / 16 * 16;
}

template <class CF>
cudaError_t launch_cfg(const Kv4Params& kp, bool pdl, cudaStream_t stream) {
  static_assert(smem_bytes<CF>(kMaxCaches) <= 227 * 1024, "shared memory at the largest number of caches");
  const size_t smem = smem_bytes<CF>(kp.a.C);
  const cudaError_t e =
      cudaFuncSetAttribute(attn_kv4_kernel<CF>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  return launch_maybe_pdl(attn_kv4_kernel<CF>, dim3(kp.a.num_ctas), dim3(kThreads), smem, pdl, stream, kp);
}

cudaError_t launch(const Kv4Params& kp, bool pdl, cudaStream_t stream) {
  switch (kp.a.rows_per_unit) {
    case 8: return launch_cfg<Cfg<8>>(kp, pdl, stream);
    case 16: return launch_cfg<Cfg<16>>(kp, pdl, stream);
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

// Fewest tiles per CTA.
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
    const int64_t seen = (static_cast<int64_t>(window) + kTile - 1) / kTile + 1 + (static_cast<int64_t>(sinks) + kTile - 1) / kTile;
    prefix = std::min(prefix, seen);
  }
  const int64_t max_tiles = units * (prefix + pl->draft_tiles);
  if (units >= INT_MAX / 2 || max_tiles >= INT_MAX / 2) return KVSHOT_ERR_UNSUPPORTED;
  pl->units = static_cast<int>(units);
  int64_t grid = d->num_ctas;
  if (grid == 0) {
    const int sms = sm_count();
    if (sms < 1) return KVSHOT_ERR_CUDA;
    grid = std::min<int64_t>(sms, std::max((max_tiles + kMinTiles - 1) / kMinTiles, units));
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
  p.len_bound = static_cast<int>(std::min<int64_t>(d->max_seq_len, static_cast<int64_t>(p.max_pages) * p.page_size));
  p.N = d->n_nodes;
  p.Nq = d->n_query;
  p.n_max = d->n_max;
  p.tree = tree;
  p.draft_tiles = pl.draft_tiles;
  p.prefix_tile = kTile;
  const double scale = d->scale != 0.f ? static_cast<double>(d->scale) : 1.0 / std::sqrt(static_cast<double>(kHeadDim));
  p.qscale = static_cast<float>(scale * 1.4426950408889634);
  p.num_ctas = pl.num_ctas;
  p.unit_ctas = d->num_caches == 1 ? pl.num_ctas / pl.units : 0;
  p.wait_ns = d->wait_limit_ns != 0 ? d->wait_limit_ns : 2000000000u;
  p.k_scale = std::ldexp(1.f, d->k_scale_exp);
  p.v_scale = std::ldexp(1.f, d->v_scale_exp);
  p.window = window;
  p.sinks = sinks;
  p.min_depth = tree ? 1 : d->n_nodes - d->n_query + 1;
  kp.cache = static_cast<const uint8_t*>(cache);
  kp.draft_k = static_cast<const __nv_bfloat16*>(draft_k);
  kp.draft_v = static_cast<const __nv_bfloat16*>(draft_v);
  kp.groups_per_page = p.page_size / kKv4Tokens;
  kp.run_groups = std::min(kTileGroups, kp.groups_per_page & -kp.groups_per_page);
  if (!paged) kp.run_groups = kTileGroups;  // one page: a tile's groups are neighbours
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (launch(kp, (d->flags & KVSHOT_OVERLAP_PREVIOUS) != 0, s) != cudaSuccess) return KVSHOT_ERR_CUDA;
  // A CTA takes whole units, whatever the lengths: nothing to merge.
  if (pl.num_ctas == 1 || p.unit_ctas == 1 || (d->num_caches == 1 && pl.units % pl.num_ctas == 0)) return KVSHOT_OK;
  return launch_merge(p, sm_count(), s) == cudaSuccess ? KVSHOT_OK : KVSHOT_ERR_CUDA;
}
