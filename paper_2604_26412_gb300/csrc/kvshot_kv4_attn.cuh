// kvshot_kv4_attn.cuh -- what the two attention kernels over a 4-bit target cache share: the work plan with a sliding
// window, the loader of the cache's bytes, the query rows' nodes and masks, and the bounded waits.
#pragma once

#include <climits>

#include "kvshot_attn_common.cuh"
#include "kvshot_kv4.cuh"

namespace kvshot {

struct Kv4Params {
  AttnParams a;
  const uint8_t* cache;
  const __nv_bfloat16 *draft_k, *draft_v;
  int groups_per_page;
  Div by_page, by_blocks, by_seq, by_group;  // groups per page, row blocks, caches per sequence, heads per KV head
  Div by_cache;    // units of a cache
  int ctas_per_unit;
  int spare_tiles; // a CTA may take as many tiles more if that leaves it one piece
  int window, sinks;  // sliding window (0: none) and sink tokens
  int min_depth;      // depth of the shallowest query node (a lower bound), for the window
  int run_groups;     // groups of a tile that are always neighbours in memory (a power of two, at most kTileGroups)
};

// attn_kv4_mma.cu: stacks of up to 16 query rows per KV head.
cudaError_t attn_kv4_mma_occupancy(int rows_per_unit, int* ctas_per_sm);
cudaError_t launch_attn_kv4_mma(const Kv4Params& p, bool pdl, cudaStream_t stream);

namespace {  // internal linkage: every translation unit gets its own copy

using namespace dev;
using namespace kv4;

constexpr int kTile = 128;                         // keys per prefix tile
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


// What the loading warp says of a tile, beside the tile's bytes.  The other warps follow these words alone: the plan, with
// its divisions, is code of one warp.  (Code that a CTA runs once costs it ~20 cycles per instruction, most of them spent
// fetching it: with the plan in every role, finding a piece took each of them 1300 to 3300 cycles.)
constexpr int kFirst = 1, kLast = 2;   // of the CTA's piece of a unit
constexpr int kDraft = 4;              // bf16 draft keys, else codes
constexpr int kMasked = 8;             // holds keys that some query row does not see
constexpr int kWhole = 16;             // (with kLast) the piece is the whole unit
constexpr int kNewRows = 32;           // the query rows' nodes differ from the piece's before
constexpr int kNewTree = 64;           // and so does the draft tree
constexpr int kStop = 128;             // no tile: the CTA's work is done
constexpr int kPieceShift = 8, kSetShift = 11;  // (with kMasked) bits 8 to 10: the piece's number; 11 and 12: its set of rows
constexpr int kRowSets = 4;            // sets of rows, of as many pieces (tcgen05 kernel)
struct TileMeta {
  int flags, key0, nkeys, L;  // (and the tile's number above bit 16); first key (token, or draft slot), valid keys, prefix length
  int c, h, rb, seq;          // cache, KV head, row block, sequence
};
constexpr int kMetas = 16;    // more than the tiles between the loader and the last reader
constexpr int kTagShift = 16;

// Shared-memory parts that both kernels have: the ring of the cache's bytes (addresses of its stages and of its barriers,
// landed and read) with the tiles' words.
struct Ring {
  uint32_t ring, cfull, cempty;
  uint32_t meta;    // [kMetas] TileMeta
  uint32_t first;   // TileMeta of the CTA's first piece, whose q and rows need not wait for a tile (flags 0: there is none)
  int* issued;      // tiles issued by the loader
};
// The query rows of a unit: their places in a cache's q and out, and, of a draft tree, who sees what, as bits of rows.
struct alignas(16) Rows {
  int place[64];
  int depth[64];                      // of the row's node
  uint64_t line[kMaxTreeNodes];       // rows whose node is this one or descends from it
  uint64_t upto[kMaxTreeNodes + 1];   // rows whose depth is at most x
  uint64_t anc[kMaxTreeNodes];        // nodes: itself and its ancestors
  int parent[kMaxTreeNodes];          // (of build_rows)
  int count, min_depth;               // rows that there are; depth of the shallowest of them
};

// Every wait ends: when its phase completes, when another role has given up, or (which gives up) after the call's limit.
// A warp waits as one.  The inline part is one try of all lanes, which blocks for a while; what the rest needs lies in
// shared memory, so that the many places that wait are short.  A blocking try may sit out more than the time it is given
// (with a limit of 1 ns, and that as its time, no wait ever gave up).  So with limits below kPollBelowNs a try is given none,
// which keeps it to a few microseconds, and the waits for a tile's bytes are polled.  (A look at the limit at every wait
// costs 256 rows 2.5 us of 170, polling inline 13.)
struct WaitLimits {
  int32_t* err;
  uint64_t limit_ns;
  int abort;  // a wait has given up
};
__device__ __forceinline__ WaitLimits* wait_limits() {
  __shared__ WaitLimits s_limits;
  return &s_limits;
}
// One thread, before the first wait and a barrier.
__device__ __forceinline__ void init_waits(const AttnParams& p) {
  WaitLimits* w = wait_limits();
  w->err = p.err;
  w->limit_ns = p.wait_ns;
  w->abort = 0;
}
// Blocks for about `hint_ns`, or a few microseconds.
__device__ __forceinline__ bool try_wait_for(uint32_t bar, uint32_t parity, uint32_t hint_ns) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}\n"
      : "=r"(done)
      : "r"(bar), "r"(parity), "r"(hint_ns)
      : "memory");
  return done != 0;
}
__device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, uint32_t hint_ns) {
  volatile WaitLimits* w = wait_limits();
  const uint64_t t0 = global_timer_ns(), limit = w->limit_ns;
  for (;;) {
    if (__all_sync(0xffffffffu, hint_ns == 0 ? mbar_test_wait(bar, parity) : try_wait_for(bar, parity, hint_ns))) return true;
    if (__any_sync(0xffffffffu, w->abort)) return false;
    if (__any_sync(0xffffffffu, global_timer_ns() - t0 > limit)) break;
  }
  if ((threadIdx.x & 31) == 0) {
    set_error(w->err, KVSHOT_ERR_TIMEOUT);
    w->abort = 1;
  }
  return false;
}
struct Waiter {
  uint32_t hint_ns;  // of a try
  __device__ __forceinline__ explicit Waiter(const AttnParams& p) : hint_ns(p.wait_ns < kPollBelowNs ? 0 : 20000) {}
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
    return __all_sync(0xffffffffu, try_wait_for(bar, parity, hint_ns)) || wait_slow(bar, parity, hint_ns);
  }
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity, uint32_t bar2, uint32_t parity2) const {
    const bool one = try_wait_for(bar, parity, hint_ns), two = try_wait_for(bar2, parity2, hint_ns);
    return __all_sync(0xffffffffu, one && two) || (wait_slow(bar, parity, hint_ns) && wait_slow(bar2, parity2, hint_ns));
  }
  // The same for a tile's bytes to land (and for another barrier).
  __device__ __forceinline__ bool landed(uint32_t bar, uint32_t parity) const {
    return hint_ns == 0 ? wait_slow(bar, parity, 0) : (*this)(bar, parity);
  }
  __device__ __forceinline__ bool landed(uint32_t bar, uint32_t parity, uint32_t bar2, uint32_t parity2) const {
    return hint_ns == 0 ? wait_slow(bar, parity, 0) && wait_slow(bar2, parity2, 0) : (*this)(bar, parity, bar2, parity2);
  }
};

__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
               : "memory");
}
__device__ __forceinline__ void sts32(uint32_t addr, int v) {
  asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ int lds32(uint32_t addr) {
  int v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// The words of tile t, once something that follows from its landing has been waited for.
__device__ __forceinline__ int4 tile_words(const Ring& r, int t) {
  const uint4 v = lds128(r.meta + t % kMetas * sizeof(TileMeta));
  return make_int4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ TileMeta tile_meta_at(uint32_t at) {
  const uint4 v = lds128(at), w = lds128(at + 16);
  return TileMeta{static_cast<int>(v.x), static_cast<int>(v.y), static_cast<int>(v.z), static_cast<int>(v.w),
                  static_cast<int>(w.x), static_cast<int>(w.y), static_cast<int>(w.z), static_cast<int>(w.w)};
}
__device__ __forceinline__ TileMeta tile_meta(const Ring& r, int t) {
  return tile_meta_at(r.meta + t % kMetas * sizeof(TileMeta));
}
// Its flags alone, read ahead of the wait; they are the tile's if is_of says so, and else are read again after it.
__device__ __forceinline__ uint32_t tile_flags(const Ring& r, int t) {
  return lds32(r.meta + t % kMetas * sizeof(TileMeta)) ^ (static_cast<uint32_t>(t) << kTagShift);
}
__device__ __forceinline__ bool is_of(uint32_t flags) { return flags < (1u << kTagShift); }

// ------------------------------------------------------------ the plan

// The prefix tiles of a cache of L tokens that some query row may see, with a sliding window: tiles [0, sink_tiles) and,
// `skip` tiles further on, those from the window's first key to the last one.  (The shallowest query node stands at
// L + min_depth - 1 and sees keys from L + min_depth - window on.)
// Of these tiles the groups of 16 tokens [hide0, hide1) hold neither a sink nor a key that the shallowest node sees.
struct WindowSpan {
  int tiles, sink_tiles, skip, hide0, hide1;
};
__device__ __forceinline__ WindowSpan window_span(const Kv4Params& p, int L) {
  const int all = (L + kTile - 1) / kTile;
  if (p.window == 0) return WindowSpan{all, all, 0, 0, 0};
  const int lo = min(L, max(0, L + p.min_depth - p.window));
  const int sink_tiles = min(all, (min(p.sinks, lo) + kTile - 1) / kTile);
  const int skip = max(0, min(all, lo / kTile) - sink_tiles);
  const int hide0 = p.sinks / kKv4Tokens + (p.sinks % kKv4Tokens > 0);
  return WindowSpan{all - skip, sink_tiles, skip, hide0, (lo == L ? lo + kKv4Tokens - 1 : lo) / kKv4Tokens};
}

// ------------------------------------------------------------ loads

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
               : "memory");
}

// Where a CTA's range of tiles [t, t_end) begins: cache c (of length L), KV head x row block hr, tile lt of the unit's ut;
// tpc: tiles of a range.  The units' tiles laid end to end are cut into equal ranges; or, if there are CTAs for it and the
// longest range gets no more than spare_tiles longer (and with one cache), each unit by itself into `per` pieces, so that no
// CTA takes the end of one unit and the start of the next one: a second piece costs it a start and an end, and the units
// that it cuts a merge.  (per 0: equal ranges.)
struct RangeStart {
  int t, t_end, c, L, hr, lt, ut, tpc, per;
};
// By a warp.  kMerge: not this CTA's, but the range that begins at the boundary after range blockIdx.x, or unit blockIdx.x.
template <bool kMerge>
__device__ __forceinline__ RangeStart range_of(const Kv4Params& kp) {
  const AttnParams& p = kp.a;
  const int lane = threadIdx.x & 31, HR = p.hkv * p.row_blocks;
  auto unit_tiles = [&](int L) { return window_span(kp, L).tiles + p.draft_tiles; };
  RangeStart r{0, 0, 0, 0, 0, 0, 0, 0, 0};
  // A lane's cache of 32 from c0 on: its length, and the tiles up to and including it.
  int L = 0, upto = 0, total = 0, longest = 0;
  auto sum = [&](int c0) {
    const int c = c0 + lane;
    L = c < p.C ? clamp_len(p, c) : 0;
    upto = c < p.C ? unit_tiles(L) : 0;
    longest = max(longest, upto);
    upto *= HR;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
  };
  r.per = kp.ctas_per_unit;
  const bool alone = p.C == 1 && r.per > 0;  // (needs no sums)
#pragma unroll 1
  for (int c0 = 0; !alone && c0 < p.C; c0 += 32) {
    sum(c0);
    total += __shfl_sync(0xffffffffu, upto, 31);
  }
  r.tpc = tiles_per_cta(total, p.num_ctas);
  if (alone || (r.per > 0 && tiles_per_cta(__reduce_max_sync(0xffffffffu, longest), r.per) <= r.tpc + kp.spare_tiles)) {
    const int unit = kMerge ? blockIdx.x : blockIdx.x / r.per, piece = kMerge ? 0 : blockIdx.x - unit * r.per;
    r.c = kp.by_cache(unit);
    r.hr = unit - r.c * HR;
    if (r.c < p.C) {
      r.L = clamp_len(p, r.c);
      r.ut = unit_tiles(r.L);
      r.tpc = tiles_per_cta(r.ut, r.per);
      r.lt = piece * r.tpc;
      r.t_end = max(0, min(r.tpc, r.ut - r.lt));
    }
    return r;
  }
  r.per = 0;
  r.t = min(total, static_cast<int>(blockIdx.x + kMerge) * r.tpc);
  r.t_end = min(total, r.t + r.tpc);
  int below = 0, c0 = 0;
#pragma unroll 1
  for (; r.t < r.t_end; c0 += 32) {
    if (p.C > 32) sum(c0);
    const int all = __shfl_sync(0xffffffffu, upto, 31);
    if (r.t < below + all) break;
    below += all;
  }
  if (r.t < r.t_end) {
    const int i = __popc(__ballot_sync(0xffffffffu, below + upto <= r.t));  // caches of these that end before it
    r.c = c0 + i;
    r.L = __shfl_sync(0xffffffffu, L, i);
    const int before = __shfl_sync(0xffffffffu, upto, max(i - 1, 0));
    const int rem = r.t - below - (i > 0 ? before : 0);
    r.ut = unit_tiles(r.L);
    r.hr = rem / r.ut;
    r.lt = rem - r.hr * r.ut;
  }
  return r;
}
constexpr int kFirstBytes = sizeof(TileMeta) + 16;
// By the loading warp, before the barrier that the roles begin with; left at sm.first: the first piece's words, with t,
// t_end and L in place of a tile's, then hr and lt.
__device__ __forceinline__ void plan_loader(const Kv4Params& kp, const Ring& sm) {
  const AttnParams& p = kp.a;
  const RangeStart r = range_of<false>(kp);
  if ((threadIdx.x & 31) == 0) {
    const int h = kp.by_blocks(r.hr);
    *sm.issued = 0;
    sts128(sm.first, make_uint4(r.t < r.t_end ? kFirst | kNewRows | (p.tree ? kNewTree : 0) : 0, r.t, r.t_end, r.L));
    sts128(sm.first + 16, make_uint4(r.c, h, r.hr - h * p.row_blocks, kp.by_seq(r.c)));
    sts128(sm.first + 32, make_uint4(r.hr, r.lt, 0, 0));
  }
}

// The loading warp: the CTA's tiles, one after another, each a stage of the ring with a copy per run of groups (a draft
// tile: two per row); at the end `kStops` tiles that say so.
template <int kStages, int kStops>
__device__ __forceinline__ void run_loader(const Kv4Params& kp, const Ring& ring, const Waiter& wait) {
  const AttnParams& p = kp.a;
  const Ring sm = ring;
  const int lane = threadIdx.x & 31, HR = p.hkv * p.row_blocks;
  const TileMeta first = tile_meta_at(sm.first);
  const int t_end = first.nkeys;
  int t = first.key0, c = first.c, hr = lds32(sm.first + 32), lt = lds32(sm.first + 36);
  int stage = 0, issued = 0, last_rb = -1, last_seq = -1, piece = -1, set = -1;
  uint32_t phase = 0;
  bool waited = false, ok = true;
  // Page ids come 32 to a load, a window of tiles ahead: lane i holds the address of run i % runs of the window's tile
  // i / runs, and issues that copy.
  const int runs = kTileGroups / kp.run_groups, ahead = 32 / runs;
  const int my_tile = lane / runs, my_g0 = (lane % runs) * kp.run_groups;
#pragma unroll 1
  for (; ok && t < t_end; lt = 0) {  // a piece
    const int L = lds32(sm.first + 12);
    const WindowSpan span = window_span(kp, L);
    const int ut = span.tiles + p.draft_tiles, lt1 = min(ut, lt + t_end - t);
    const int h = kp.by_blocks(hr), rb = hr - h * p.row_blocks, seq = kp.by_seq(c);
    const int last = kLast | (lt == 0 && lt1 == ut ? kWhole : 0);
    int flags = kFirst;
    if (rb != last_rb) flags |= kNewRows;
    if (p.tree && seq != last_seq) flags |= kNewRows | kNewTree;
    last_rb = rb;
    last_seq = seq;
    ++piece;
    if (flags & kNewRows) ++set;
    const int masked = kMasked | (piece & (2 * kRowSets - 1)) << kPieceShift | (set & (kRowSets - 1)) << kSetShift;
    t += lt1 - lt;
    // A window: rows see keys from L + their depth - window on (and the sinks); a depth is at most N.
    const int seen_from = kp.window > 0 ? L + p.N - kp.window : 0;
    const int32_t* table = p.page_table + (p.paged ? static_cast<size_t>(c) * p.max_pages : 0);
    auto key_of = [&](int x) { return (x < span.sink_tiles ? x : x + span.skip) * kTile; };  // of a prefix tile
    const int groups = (L + kKv4Tokens - 1) / kKv4Tokens;
    // A run of groups loses the hidden ones at its two ends, and with them all of it (its page is not looked up then).
    auto hidden = [&](int g) { return g >= span.hide0 && g < span.hide1; };
    auto run_end = [&](int g) {  // of the run that holds group g
      const int end = min((g | (kp.run_groups - 1)) + 1, groups);
      return hidden(end - 1) ? max(span.hide0, g) : end;
    };
    auto group_of = [&](int x) {  // this lane's first group to load of the window from tile x on, or -1
      x += my_tile;
      if (x >= lt1 || x >= span.tiles) return -1;
      const int g0 = key_of(x) / kKv4Tokens + my_g0, g = hidden(g0) ? span.hide1 : g0;
      return g < min(g0 + kp.run_groups, groups) ? g : -1;
    };
    auto page_of = [&](int g) { return g < 0 ? 0 : p.paged ? table[kp.by_page(g)] : c; };
    int window = lt, g = group_of(window), pid = page_of(g);
    const uint8_t* src = nullptr;
    uint32_t bytes = 0, at = 0;  // of this lane's copy, and its place in the tile
#pragma unroll 1
    for (; lt < lt1; ++lt) {
      if (lt == window) {
        if (p.paged && g >= 0) pid = valid_page_id(p, pid);
        src = kp.cache + ((static_cast<size_t>(pid) * p.hkv + h) * kp.groups_per_page +
                          (p.paged ? g - kp.by_page(g) * kp.groups_per_page : g)) * kKv4Bytes;
        bytes = g < 0 ? 0 : (run_end(g) - g) * kKv4Bytes;
        at = g % kTileGroups * kKv4Bytes;
        window += ahead;
        g = group_of(window);
        pid = page_of(g);
      }
      const bool draft = lt >= span.tiles;
      const int key0 = draft ? (lt - span.tiles) * kDraftTile : key_of(lt);
      const int nkeys = draft ? min(kDraftTile, p.N - key0) : min(kTile, L - key0);
      if (draft) flags |= kDraft | masked;
      else if (nkeys < kTile || (key0 < seen_from && key0 + kTile > kp.sinks)) flags |= masked;
      if (lt == lt1 - 1) flags |= last;
      if (draft && !waited) {  // the draft K/V may come from the preceding kernel
        wait_for_prerequisite_grid();
        waited = true;
      }
      const bool mine = !draft && my_tile == lt - (window - ahead);
      int tx = draft ? nkeys * 4 * kHeadDim : (nkeys + kKv4Tokens - 1) / kKv4Tokens * kKv4Bytes;
      if (kp.window > 0 && !draft) tx = __reduce_add_sync(0xffffffffu, mine ? bytes : 0);
      ok = wait(sm.cempty + 8 * stage, phase ^ 1u);
      if (!ok) break;
      const uint32_t bar = sm.cfull + 8 * stage, dst = sm.ring + stage * kStageSize;
      if (lane == 0) {
        const uint32_t m = sm.meta + issued % kMetas * sizeof(TileMeta);
        sts128(m, make_uint4(flags | issued << kTagShift, key0, nkeys, L));
        sts128(m + 16, make_uint4(c, h, rb, seq));
        mbar_arrive_expect_tx(bar, tx);
      }
      __syncwarp();
      if (draft) {
        if (lane < nkeys) {
          const size_t row = (static_cast<size_t>(c) * p.hkv + h) * p.n_max + key0 + lane;
          bulk_load(dst + lane * kDraftRow, kp.draft_k + row * kHeadDim, 2 * kHeadDim, bar);
          bulk_load(dst + kDraftV + lane * kDraftRow, kp.draft_v + row * kHeadDim, 2 * kHeadDim, bar);
        }
      } else if (mine && bytes > 0) {
        bulk_load(dst + at, src, bytes, bar);
      }
      flags = 0;
      ++issued;
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (++hr == HR) {  // (a piece that ends before its unit is the CTA's last)
      hr = 0;
      ++c;
      if (t < t_end) {
        const int next = clamp_len(p, c);
        __syncwarp();
        if (lane == 0) sts32(sm.first + 12, next);
        __syncwarp();
      }
    }
  }
#pragma unroll 1
  for (int i = 0; ok && i < kStops; ++i) {
    ok = wait(sm.cempty + 8 * stage, phase ^ 1u);
    if (!ok) break;
    if (lane == 0) {
      sts128(sm.meta + issued % kMetas * sizeof(TileMeta), make_uint4(kStop | issued << kTagShift, 0, 0, 0));
      mbar_arrive(sm.cfull + 8 * stage);
    }
    ++issued;
    if (++stage == kStages) {
      stage = 0;
      phase ^= 1u;
    }
  }
  if (lane == 0) *sm.issued = issued;
}

// After the roles have ended: no copy outlives the CTA, whatever ended it (each wait is bounded).  One thread.
template <int kStages>
__device__ __forceinline__ void drain(const AttnParams& p, const Ring& sm) {
#pragma unroll 1
  for (int k = max(0, *sm.issued - kStages); k < *sm.issued; ++k)
    if (!mbar_wait(sm.cfull + 8 * (k % kStages), (k / kStages) & 1, p.err)) break;
}

// A barrier among warps that ends like every wait (count: warps; a warp passes it with the phase it has counted).
struct WarpSync {
  uint32_t bar, phase;
  __device__ __forceinline__ bool operator()(const Waiter& wait) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
    const bool ok = wait(bar, phase);
    phase ^= 1u;
    return ok;
  }
};

__device__ __forceinline__ uint32_t bf16x2_to_f16x2(uint32_t w) {
  const __half2 v = __floats2half2_rn(bf16_lo(w), bf16_hi(w));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
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

// The rows of row block rb, of sequence seq's draft tree, by one warp.
__device__ __noinline__ void build_rows(const Kv4Params& kp, Rows& r, int nc, int rb, int seq, bool new_tree) {
  const AttnParams& p = kp.a;
  const int lane = threadIdx.x & 31;
  if (new_tree) {
    const int* tree = p.tree_parent + static_cast<size_t>(seq) * p.N;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = lane + 32 * k;
      int v = i < p.N ? tree[i] : -1;
      if (v < -1 || v >= i) {
        if (i < p.N) set_error(p.err, KVSHOT_ERR_TREE);
        v = -1;
      }
      r.parent[i] = v;
    }
    __syncwarp();
    // Ancestors, by jumps that double: a node's bits so far end above r.parent, where the next ones begin.
    uint64_t bits[2] = {1ull << lane, 1ull << (lane + 32)};
    int up[2] = {r.parent[lane], r.parent[lane + 32]};
#pragma unroll
    for (int k = 0; k < 2; ++k) r.anc[lane + 32 * k] = bits[k];
    __syncwarp();
#pragma unroll 1
    while (__any_sync(0xffffffffu, max(up[0], up[1]) >= 0)) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (up[k] >= 0) {
          bits[k] |= r.anc[up[k]];
          up[k] = r.parent[up[k]];
        }
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        r.anc[lane + 32 * k] = bits[k];
        r.parent[lane + 32 * k] = up[k];
      }
      __syncwarp();
    }
  }
  const int row0 = rb * p.rows_per_unit;
  int least = INT_MAX;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int j = lane + 32 * k, nl = kp.by_group(min(row0 + j, p.rows_total - 1));  // (past the last row: its node)
    if (j < nc) {
      const int depth = p.tree ? __popcll(r.anc[p.N - p.Nq + nl]) : p.N - p.Nq + nl + 1;
      r.place[j] = nl * p.hq + row0 + j - nl * p.G;
      r.depth[j] = depth;
      least = min(least, depth);
    }
  }
  least = __reduce_min_sync(0xffffffffu, least);
  if (lane == 0) {
    r.count = min(p.rows_per_unit, p.rows_total - row0);
    r.min_depth = least;
  }
  if (p.tree) {
    // The query nodes one after another, whose rows are neighbours: lane m has the rows of nodes m, m + 32, and of depths.
    uint64_t line[2] = {0ull, 0ull}, upto[2] = {0ull, 0ull};
    const int last = kp.by_group(min(row0 + 63, p.rows_total - 1));
#pragma unroll 1
    for (int nl = kp.by_group(row0); nl <= last; ++nl) {
      const uint64_t anc = r.anc[p.N - p.Nq + nl];
      const int a = max(nl * p.G - row0, 0), b = min(nl * p.G + p.G - row0, 64);
      const uint64_t rows = ~0ull >> (64 - b + a) << a;
      if ((static_cast<uint32_t>(anc) >> lane) & 1) line[0] |= rows;
      if ((static_cast<uint32_t>(anc >> 32) >> lane) & 1) line[1] |= rows;
      const int depth = __popcll(anc);
      if (depth <= lane) upto[0] |= rows;
      if (depth <= lane + 32) upto[1] |= rows;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      r.line[lane + 32 * k] = line[k];
      r.upto[lane + 32 * k] = upto[k];
    }
    if (lane == 0) r.upto[kMaxTreeNodes] = ~0ull;
  }
  __syncwarp();
}

// Bits of the unit's rows that see key `key` of a masked tile (m: its words' flags, key0, nkeys, L).
__device__ __noinline__ uint64_t rows_seeing(const Kv4Params& kp, const Rows& r, const int4& m, int rb, int key) {
  const AttnParams& p = kp.a;
  if (key >= m.z) return 0ull;
  const bool draft = m.x & kDraft;
  if (!draft && kp.window == 0) return ~0ull;
  const int at = m.y + key, L = m.w;
  // Rows whose node's depth is at most x.  A chain's rows are in the order of depth.
  auto upto = [&](int x) -> uint64_t {
    if (p.tree) return x < 0 ? 0ull : r.upto[min(x, p.N)];
    const int nodes = min(x - (p.N - p.Nq), p.Nq);
    if (nodes <= 0) return 0ull;  // (x may be as low as -L: no product with it)
    const int n = nodes * p.G - rb * p.rows_per_unit;
    return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull;
  };
  if (!draft) return at < kp.sinks ? ~0ull : upto(at - L + kp.window);
  uint64_t bits = p.tree ? r.line[at] : ~upto(at);
  if (kp.window > 0) {
    const int depth = p.tree ? __popcll(r.anc[at]) : at + 1;
    if (L + depth - 1 >= kp.sinks) bits &= upto(depth + kp.window - 1);
  }
  return bits;
}
// Whether any row of the unit is among them.  The other keys' values count as zeros: what stands there may be anything, and
// 0 times an infinity or a NaN is none.
__device__ __forceinline__ bool any_row(const Rows& r, uint64_t bits) { return (bits << (64 - r.count)) != 0; }

}  // namespace
}  // namespace kvshot
