// kvshot_kv4_attn.cuh -- what the two attention kernels over a 4-bit target cache share: the work plan with a sliding
// window, the loader of the cache's bytes, the query rows' nodes and masks, and the bounded waits.
#pragma once

#include "kvshot_attn_common.cuh"
#include "kvshot_kv4.cuh"

namespace kvshot {

struct Kv4Params {
  AttnParams a;
  const uint8_t* cache;
  const __nv_bfloat16 *draft_k, *draft_v;
  int groups_per_page;
  int run_groups;  // groups of a tile that are always neighbours in memory (a power of two, at most kTileGroups)
};

// attn_kv4_mma.cu: stacks of up to 16 query rows per KV head.
cudaError_t attn_kv4_mma_occupancy(int rows_per_unit, int C, int* ctas_per_sm);
cudaError_t launch_attn_kv4_mma(const Kv4Params& p, bool pdl, cudaStream_t stream);

namespace {  // internal linkage: every translation unit gets its own copy

using namespace dev;
using namespace kv4;

constexpr int kTile = kKv4PrefixTile;              // keys per prefix tile
constexpr int kTileGroups = kTile / kKv4Tokens;
constexpr int kStageSize = kTileGroups * kKv4Bytes;
constexpr int kDraftTile = 32;                     // keys per draft tile: bf16 rows of K and V fill a stage
constexpr int kDraftRow = 2 * kHeadDim + 16;       // padded: rows 16 bytes apart mod 128, free of bank conflicts
constexpr int kDraftV = kDraftTile * kDraftRow;
static_assert(2 * kDraftV <= kStageSize, "a draft tile fits a stage");
// The reference of a row is 2^8 below the maximum it was taken from and moves when a score passes it by 2^15: P stays in
// f16's normal range for scores down to 2^-22 of the maximum and below its largest number.
constexpr float kRefBelow = 8.f, kRefLimit = 15.f;
constexpr float kNoRef = -1e30f;                   // no score yet


// Shared-memory parts that both kernels have: the ring of the cache's bytes (addresses of its stages and of its barriers,
// landed and read), and the query rows' nodes.
struct Ring {
  uint32_t ring, cfull, cempty;
  int* issued;      // tiles issued by the loader
  int *len, *base;  // the plan
};
struct Rows {
  uint64_t *anc, *row_anc;  // [64] each node's ancestors and itself (tree); of each query row's node
  int *depth, *place;       // [64] per row: the node's depth; the row's place in a cache's q and out
  int* par;                 // [64]
};

// Every wait ends: when its phase completes, when another role has given up, or (which gives up) after the call's limit.
// The inline part is one try, which blocks for a while (a call for each wait took more instructions than it waited for).
__device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, int32_t* err, uint64_t limit_ns, volatile int* abort) {
  const bool poll = limit_ns < kPollBelowNs;  // (a blocking try could sit out a short limit)
  const uint64_t t0 = global_timer_ns();
  for (;;) {
    for (int i = 0; i < (poll ? 1 : 16); ++i)
      if (poll ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
    if (*abort) return false;
    if (global_timer_ns() - t0 > limit_ns) break;
  }
  set_error(err, KVSHOT_ERR_TIMEOUT);
  *abort = 1;
  return false;
}

struct Waiter {
  int32_t* err;
  uint64_t limit;
  volatile int* abort;
  bool poll;
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
    if (poll ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
    return wait_slow(bar, parity, err, limit, abort);
  }
};

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

// A run of tiles of one unit that this CTA takes.
struct Piece {
  int t, t_end;        // tile of this CTA's range: the piece's first one (its end after next_piece), and the range's end
  int c, hr;           // cache, KV head x row block
  int lt0, lt1, ut;    // the piece's tiles of the unit [lt0, lt1), tiles of the unit
  int h, rb, seq, L;   // KV head, row block, sequence, prefix length
  WindowSpan span;

  // First key of tile lt (token, or draft slot), and its valid keys.
  __device__ __forceinline__ bool draft(int lt) const { return lt >= span.tiles; }
  __device__ __forceinline__ int key0(int lt) const {
    return draft(lt) ? (lt - span.tiles) * kDraftTile : (lt < span.sink_tiles ? lt : lt + span.skip) * kTile;
  }
  __device__ __forceinline__ int nkeys(int lt, int n_nodes) const {
    return draft(lt) ? min(kDraftTile, n_nodes - key0(lt)) : min(kTile, L - key0(lt));
  }
  // Whether prefix tile lt holds keys past the last one, or from the sinks' end up to `from`, where a window begins.
  __device__ __forceinline__ bool masked(int lt, int from, int sinks) const {
    const int k = key0(lt);
    return k + kTile > L || (k < from && k + kTile > sinks);
  }
  __device__ __forceinline__ bool whole() const { return lt0 == 0 && lt1 == ut; }
};

// The CTA's range; next_piece finds its first piece.
__device__ __noinline__ void begin_pieces(const AttnParams& p, const int* s_len, const int* s_base, Piece& w) {
  w.c = w.hr = w.lt1 = w.ut = w.t = w.t_end = 0;
  if (p.unit_ctas > 0) {
    w.ut = window_span<kTile>(p, s_len[0]).tiles + p.draft_tiles;
    const UnitCut u = unit_cut(p.unit_ctas, w.ut);
    w.hr = blockIdx.x / u.per;
    w.lt1 = (blockIdx.x - w.hr * u.per) * u.tpc;
    w.t_end = w.hr < p.hkv * p.row_blocks ? min(u.tpc, w.ut - w.lt1) : 0;
    return;
  }
  const int total = s_base[p.C], tpc = tiles_per_cta(total, p.num_ctas);
  w.t = min(total, static_cast<int>(blockIdx.x) * tpc);
  w.t_end = min(total, w.t + tpc);
  if (w.t >= w.t_end) return;
  int lo = 0, hi = p.C - 1;  // last cache whose first tile is <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s_base[mid] <= w.t) lo = mid;
    else hi = mid - 1;
  }
  w.c = lo;
  w.ut = window_span<kTile>(p, s_len[lo]).tiles + p.draft_tiles;
  const int rem = w.t - s_base[lo];
  w.hr = rem / w.ut;
  w.lt1 = rem - w.hr * w.ut;
}

// Moves on to the next piece of the range; false at its end.  (Out of line: the roles' loops over the tiles are short.)
__device__ __noinline__ bool next_piece(const AttnParams& p, const int* s_len, Piece& w) {
  if (w.t >= w.t_end) return false;
  if (w.lt1 == w.ut) {
    w.lt1 = 0;
    if (++w.hr == p.hkv * p.row_blocks) {
      w.hr = 0;
      ++w.c;
    }
  }
  w.L = s_len[w.c];
  w.span = window_span<kTile>(p, w.L);
  w.ut = w.span.tiles + p.draft_tiles;
  w.lt0 = w.lt1;
  w.lt1 = min(w.ut, w.lt0 + w.t_end - w.t);
  w.t += w.lt1 - w.lt0;
  w.h = w.hr / p.row_blocks;
  w.rb = w.hr - w.h * p.row_blocks;
  w.seq = w.c / (p.C / p.B);
  return true;
}

// ------------------------------------------------------------ loads

// The roles keep copies of their own of what they also hand to functions out of line: a variable whose address has been
// given away is read from local memory again after every barrier and copy.

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
               : "memory");
}

// The loading warp: one stage per tile, a copy per run of groups (a draft tile: two per row).
template <int kStages>
__device__ __forceinline__ void run_loader(const Kv4Params& kp, const Ring& ring, const Waiter& wait, Piece next) {
  const AttnParams& p = kp.a;
  const Ring sm = ring;
  const int lane = threadIdx.x & 31;
  int stage = 0, issued = 0;
  uint32_t phase = 0;
  bool waited = false, ok = true;
  // Page ids come 32 to a load, a window of tiles ahead: lane i holds the address of run i % runs of the window's tile
  // i / runs, and issues that copy.
  const int runs = kTileGroups / kp.run_groups, ahead = 32 / runs;
  const int my_tile = lane / runs, my_g0 = (lane % runs) * kp.run_groups;
  while (ok && next_piece(p, sm.len, next)) {
    const Piece w = next;
    const int32_t* table = p.page_table + (p.paged ? static_cast<size_t>(w.c) * p.max_pages : 0);
    auto group_of = [&](int lt) {  // this lane's first group of the window from tile lt on, or -1
      lt += my_tile;
      if (lt >= w.lt1 || w.draft(lt)) return -1;
      const int g = w.key0(lt) / kKv4Tokens + my_g0;
      return g * kKv4Tokens < w.L ? g : -1;
    };
    auto page_of = [&](int g) { return g < 0 ? 0 : p.paged ? table[g / kp.groups_per_page] : w.c; };
    int window = w.lt0, g = group_of(window), pid = page_of(g);
    const uint8_t* src = nullptr;
    uint32_t bytes = 0;
    for (int lt = w.lt0; lt < w.lt1; ++lt) {
      if (lt == window) {
        if (p.paged && g >= 0) pid = valid_page_id(p, pid);
        src = kp.cache + ((static_cast<size_t>(pid) * p.hkv + w.h) * kp.groups_per_page +
                          (p.paged ? g % kp.groups_per_page : g)) * kKv4Bytes;
        bytes = g < 0 ? 0 : min(kp.run_groups, (w.L + kKv4Tokens - 1) / kKv4Tokens - g) * kKv4Bytes;
        window += ahead;
        g = group_of(window);
        pid = page_of(g);
      }
      const bool draft = w.draft(lt);
      const int nkeys = w.nkeys(lt, p.N);
      if (draft && !waited) {  // the draft K/V may come from the preceding kernel
        wait_for_prerequisite_grid();
        waited = true;
      }
      ok = __all_sync(0xffffffffu, wait(sm.cempty + 8 * stage, phase ^ 1u));
      if (!ok) break;
      const uint32_t bar = sm.cfull + 8 * stage, dst = sm.ring + stage * kStageSize;
      if (lane == 0)
        mbar_arrive_expect_tx(bar, draft ? nkeys * 4 * kHeadDim : (nkeys + kKv4Tokens - 1) / kKv4Tokens * kKv4Bytes);
      __syncwarp();
      if (draft) {
        if (lane < nkeys) {
          const size_t row = (static_cast<size_t>(w.c) * p.hkv + w.h) * p.n_max + w.key0(lt) + lane;
          bulk_load(dst + lane * kDraftRow, kp.draft_k + row * kHeadDim, 2 * kHeadDim, bar);
          bulk_load(dst + kDraftV + lane * kDraftRow, kp.draft_v + row * kHeadDim, 2 * kHeadDim, bar);
        }
      } else if (my_tile == lt - (window - ahead) && bytes > 0) {
        bulk_load(dst + my_g0 * kKv4Bytes, src, bytes, bar);
      }
      ++issued;
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
  }
  if (lane == 0) *sm.issued = issued;
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

// Two blocks' scales (the low two bytes), each in both halves.
__device__ __forceinline__ uint2 scale_pair(uint32_t bytes) {
  const uint32_t two = e4m3x2_to_f16x2(bytes);
  return make_uint2(__byte_perm(two, two, 0x1010), __byte_perm(two, two, 0x3232));
}

// Floats as integers of the same order.
__device__ __forceinline__ int ordered(float f) {
  const int i = __float_as_int(f);
  return i >= 0 ? i : i ^ 0x7fffffff;
}
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i >= 0 ? i : i ^ 0x7fffffff); }

// The nodes of a unit's rows, by the first `threads` threads of the CTA, which all call it (named barrier `bar`).
__device__ __noinline__ void load_rows(const AttnParams& p, const Rows& sm, int nc, int rb, int seq, bool new_seq, int bar,
                                       int threads) {
  const int tid = threadIdx.x;
  named_barrier_sync(bar, threads);  // the rows before are no longer read
  if (new_seq) {
    for (int i = tid; i < p.N; i += threads) {
      int v = p.tree_parent[static_cast<size_t>(seq) * p.N + i];
      if (v < -1 || v >= i) {
        set_error(p.err, KVSHOT_ERR_TREE);
        v = -1;
      }
      sm.par[i] = v;
    }
    named_barrier_sync(bar, threads);
    for (int i = tid; i < p.N; i += threads) {
      uint64_t bits = 0;
      for (int m = i; m >= 0; m = sm.par[m]) bits |= 1ull << m;  // parents strictly decrease
      sm.anc[i] = bits;
    }
    named_barrier_sync(bar, threads);
  }
  if (tid < nc) {
    const int rr = rb * p.rows_per_unit + tid;
    const int nl = min(rr, p.rows_total - 1) / p.G, node = p.N - p.Nq + nl;
    if (p.tree) sm.row_anc[tid] = sm.anc[node];
    sm.depth[tid] = p.tree ? __popcll(sm.anc[node]) : node + 1;
    sm.place[tid] = nl * p.hq + rr - nl * p.G;
  }
}

// Bit j: row j0 + j sees this thread's key.  `at`: token position or draft slot of the key, which is valid.
__device__ __noinline__ uint64_t visible_rows(const AttnParams& p, const Rows& sm, int j0, int n, bool draft, int at, int L) {
  uint64_t bits = 0;
  const int key_depth = !draft ? 0 : p.tree ? __popcll(sm.anc[at]) : at + 1;
  const int pos = draft ? L + key_depth - 1 : at;
  const bool always = p.window == 0 || pos < p.sinks;
#pragma unroll 1
  for (int j = 0; j < n; ++j) {
    const int d = sm.depth[j0 + j];
    bool v = always || L + d - 1 - pos < p.window;
    if (draft) v = v && (p.tree ? (sm.row_anc[j0 + j] >> at) & 1ull : at < d);
    bits |= static_cast<uint64_t>(v) << j;
  }
  return bits;
}


}  // namespace
}  // namespace kvshot
