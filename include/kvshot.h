/*
 * kvshot.h -- C ABI of libkvshot, GB300 (sm_103a) draft attention for
 * KV-reuse speculative drafting.
 *
 * The drafter of a KV-reuse speculative decoder re-attends, with its own
 * query, to the target model's key/value cache instead of (or next to) the
 * target's hidden state: a' = sum_i alpha_i(q') v_i with
 * alpha_i(q') = softmax_i(q'^T k_i)  (arXiv 2604.26412, Sec. 2.2,
 * Eq. "kv-reattention").  Its memory M_i holds the target K/V of the verified
 * prefix (j <= t) followed by K/V the drafter produced for its own earlier
 * draft positions (j > t)  (Sec. 3.4, Eq. "cross-attn"; App. B,
 * "Cross-attention memory").  The same attention step serves the KV-only
 * drafter (Sec. 3.2) and the cross-attention branch o_i of the hybrid
 * gated-delta drafter (Sec. 3.4).  Draft positions form a chain (K draft
 * tokens drafted one after another, Sec. 4.2) or a tree (tree verification
 * with a (8, 10, 60) draft tree, Sec. 3.1 and 3.5); a draft node sees every
 * verified prefix token plus itself and its ancestors among the draft nodes.
 *
 * Conventions for every entry point:
 *  - All tensor pointers are DEVICE pointers owned by the caller.  The
 *    library never allocates; scratch space is the caller's workspace.
 *  - Work is enqueued on `stream` (a cudaStream_t; NULL = legacy default
 *    stream).  Nothing synchronises the host.
 *  - Argument errors are found on the host, before anything is enqueued, and
 *    returned as a kvshot_status; nothing is launched then.
 *  - Errors only visible on the device (a page id outside the pool, a
 *    sequence length above the stated bound, a parent index that is not an
 *    earlier node, a pipeline wait that timed out) are recorded in
 *    desc->err_flag (if non-NULL): the first error code is stored with an
 *    atomic compare-and-swap from 0.  Outputs of the affected call are then
 *    unspecified.  No kernel traps.
 *  - bf16 tensors are row-major with the innermost dimension head_dim (= 128).
 */
#ifndef KVSHOT_H
#define KVSHOT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* kvshot_stream_t; /* same handle type as cudaStream_t */

typedef enum kvshot_status {
  KVSHOT_OK = 0,
  KVSHOT_ERR_NULL = 1,          /* a required pointer is NULL */
  KVSHOT_ERR_SHAPE = 2,         /* inconsistent or out-of-range sizes in the descriptor */
  KVSHOT_ERR_ALIGN = 3,         /* a pointer is not aligned as stated below */
  KVSHOT_ERR_UNSUPPORTED = 4,   /* valid but outside this build (head_dim != 128, tree with > 64 nodes, ...) */
  KVSHOT_ERR_TREE = 5,          /* (device) tree_parent[i] is not in [-1, i) */
  KVSHOT_ERR_WORKSPACE = 6,     /* workspace missing, misaligned or smaller than the size query returns */
  KVSHOT_ERR_CUDA = 7,          /* a CUDA runtime/driver call failed (tensor map encode, launch) */
  KVSHOT_ERR_DEVICE_BOUNDS = 8, /* (device) page id outside the pool or seq_len above its bound */
  KVSHOT_ERR_TIMEOUT = 9        /* (device) a pipeline wait gave up after its time limit */
} kvshot_status;

/* desc->flags */
#define KVSHOT_TREE 0x1u       /* draft nodes form a tree given by tree_parent (else a chain) */
#define KVSHOT_FORCE_CC 0x2u   /* use the CUDA-core kernel whatever the row count (measurement aid) */
#define KVSHOT_FORCE_MMA 0x4u  /* use the mma.sync tensor-core kernel whatever the row count (measurement aid) */
#define KVSHOT_FORCE_TC 0x8u   /* use the tcgen05 / tensor-memory kernel (needs 128 % (hq / hkv) == 0) */
/* Let the attention kernel start while the kernel enqueued just before the call is still running
 * (programmatic dependent launch): it then reads seq_lens, page_table, target_k/v and tree_parent,
 * and starts the first target K/V loads, before that kernel has finished, and waits for it only
 * before it reads q or draft_k/v or writes anything.  Set it only when the preceding kernel does
 * not write seq_lens, page_table, target_k, target_v or tree_parent (kvshot_draft_append, which
 * writes q and the draft K/V, qualifies). */
#define KVSHOT_OVERLAP_PREVIOUS 0x10u
/* The target cache (target_k, target_v) holds fp8 E4M3 codes (OCP FP8: 1 sign bit, 4 exponent
 * bits with bias 7, 3 mantissa bits, subnormals, codes 0x7F and 0xFF NaN, no infinities), one byte
 * per element in the same row layout as the bf16 cache ([..][128] per token and KV head).  The
 * key and value of a target token are decoded as
 *   k = e4m3(code) * 2^desc->k_scale_exp,   v = e4m3(code) * 2^desc->v_scale_exp
 * which is exact in bf16 for |exponent| <= 64; attention then proceeds as for a bf16 cache.  The
 * draft K/V stay bf16.  Both tensor-core kernels then multiply in f16 (e4m3 -> f16 is exact; q,
 * P and the draft K/V are rounded to f16, which keeps more mantissa than bf16; only magnitudes below
 * 2^-14 lose bits).  Stacks of 17 rows and more run on the tcgen05 kernel (128 rows at a time),
 * which decodes the codes into f16 tiles in shared memory; the others on the m16n8k16 kernel, which
 * decodes them in registers.  KVSHOT_FORCE_TC with more than 128 rows and KVSHOT_FORCE_CC return
 * KVSHOT_ERR_UNSUPPORTED.  Not in the paper: a cache-compression variant that halves the bytes the
 * kernel reads per target token. */
#define KVSHOT_TARGET_FP8 0x20u

/*
 * Problem descriptor shared by kvshot_draft_attn and kvshot_draft_append.
 *
 * A "cache" is one independent KV cache: one sequence when one target layer
 * is reused, or one (sequence, reused target layer) pair when several target
 * layers are attended separately (KV-only head concatenation, Sec. 3.2).
 * Caches of one sequence are consecutive and share that sequence's draft tree.
 */
typedef struct kvshot_attn_desc {
  int32_t num_caches;        /* C >= 1 (<= 1024) */
  int32_t num_seqs;          /* B >= 1, C % B == 0; cache c belongs to sequence c / (C / B) */
  int32_t hq;                /* query heads */
  int32_t hkv;               /* KV heads; hq % hkv == 0 (GQA group G = hq / hkv) */
  int32_t head_dim;          /* must be 128 */
  int32_t page_size;         /* paged layout: tokens per page: 8, 16, 32, 64, 128, 192 or 256 */
  int32_t max_pages_per_seq; /* paged layout: row stride of page_table */
  int32_t num_pages;         /* paged layout: pages in the target_k / target_v pools */
  int32_t l_cap;             /* contiguous layout: token capacity per (cache, KV head) */
  int32_t max_seq_len;       /* host-known upper bound on every seq_lens[c]; sizes the work plan */
  int32_t n_nodes;           /* N: draft nodes present; draft slots 0..N-1 hold their K/V */
  int32_t n_query;           /* Nq: the last Nq draft nodes are the query rows (Nq <= N) */
  int32_t n_max;             /* draft buffer capacity in slots (N <= n_max) */
  float scale;               /* softmax scale on q.k, > 0; 0 selects 1/sqrt(head_dim); negative -> KVSHOT_ERR_SHAPE */
  uint32_t flags;            /* KVSHOT_TREE, at most one of KVSHOT_FORCE_CC / _MMA / _TC */
  int32_t num_ctas;          /* persistent CTAs to launch; 0 = one full wave on this GPU */
  void* workspace;           /* device scratch, 256-byte aligned; see kvshot_draft_attn_workspace_size */
  size_t workspace_bytes;
  int32_t* err_flag;         /* optional device int32, 0 before the call; see conventions above */
  int32_t k_scale_exp;       /* KVSHOT_TARGET_FP8: target keys are e4m3 x 2^k_scale_exp, |exp| <= 64 (and the 4-bit cache's) */
  int32_t v_scale_exp;       /* KVSHOT_TARGET_FP8: target values are e4m3 x 2^v_scale_exp, |exp| <= 64 (likewise) */
  uint32_t wait_limit_ns;    /* watchdog: longest any one wait of the attention kernels' load/compute
                                pipeline may take, in ns; 0 = 2 s.  A wait that runs past it records
                                KVSHOT_ERR_TIMEOUT; the kernel then stops computing, waits (2 s at most
                                each) for the copies and tensor-core operations it already issued, and
                                returns, leaving the outputs unspecified.  Setting it near zero makes every
                                CTA give up on its first unfinished wait: a way to exercise that path. */
} kvshot_attn_desc;

/*
 * Bytes of workspace kvshot_draft_attn needs for `desc` on the current device
 * (partial softmax states of work pieces that straddle CTAs).  Returns 0 if the descriptor is invalid.  The size depends on the
 * shape fields, flags, num_ctas and the device's SM count, not on pointers.
 */
size_t kvshot_draft_attn_workspace_size(const kvshot_attn_desc* desc);

/*
 * Draft attention.  For every cache c, query row n_local in [0, Nq) (draft
 * node n = N - Nq + n_local) and query head h (KV head h / G):
 *
 *   keys  = { prefix tokens j in [0, L_c) }  U  { draft slots m : m == n or m is an ancestor of n }
 *   s_k   = scale * q . k_k
 *   lse   = log sum_k exp(s_k)                          (natural log)
 *   out   = sum_k exp(s_k - lse) v_k                    (fp32 accumulate, rounded to bf16)
 *
 * where L_c = seq_lens[c] (Sec. 2.2 Eq. "kv-reattention" over M_i of Sec. 3.4 / App. B).
 * A chain (flags without KVSHOT_TREE) means node n's ancestors are 0..n-1.
 *
 * q:           [C, Nq, hq, 128] bf16, 16-byte aligned.
 * target_k/v:  paged (page_table != NULL): [num_pages, hkv, page_size, 128] bf16;
 *              contiguous (page_table == NULL): [C, hkv, l_cap, 128] bf16.  16-byte aligned.
 *              Rows past L_c may hold anything (NaN included); they are never used.
 * page_table:  [C, max_pages_per_seq] int32; entry p of cache c is the pool page of tokens
 *              [p * page_size, (p + 1) * page_size).  Only the first ceil(L_c / page_size) entries are read.
 * seq_lens:    [C] int32, 0 <= L_c <= min(max_seq_len, capacity).
 * draft_k/v:   [C, hkv, n_max, 128] bf16, 16-byte aligned; slots 0..N-1 are read.
 * tree_parent: [B, N] int32, parent[i] in [-1, i) (-1 = child of the last verified token);
 *              read only with KVSHOT_TREE (then N <= 64).  May be NULL for a chain.
 * out:         [C, Nq, hq, 128] bf16, 16-byte aligned, must not alias any input.
 * lse:         [C, Nq, hq] fp32 (natural log), 4-byte aligned.
 * Nq == 0 is a no-op returning KVSHOT_OK.
 */
kvshot_status kvshot_draft_attn(const kvshot_attn_desc* desc, const void* q, const void* target_k,
                                const void* target_v, const int32_t* page_table, const int32_t* seq_lens,
                                const void* draft_k, const void* draft_v, const int32_t* tree_parent,
                                void* out, float* lse, kvshot_stream_t stream);

/* Bytes of device scratch built into the library for kvshot_draft_attn_static (64 MiB: enough for the
 * plan of a 64-node whole tree over 16 caches x 8 KV heads, 256 stacked rows per head, ~34 MB). */
#define KVSHOT_STATIC_WORKSPACE_BYTES (64u * 1024u * 1024u)

/*
 * kvshot_draft_attn_static -- the same computation, arguments and results as
 * kvshot_draft_attn, for callers that cannot allocate device memory: code
 * handed only device pointers by a host framework that owns all allocation,
 * a serving loop whose memory pool is fully reserved up front, or a hot path
 * that must not call cudaMalloc (which can synchronise the device and stall
 * every other stream).  The paper has no counterpart; this is an interface
 * convenience only.
 *
 * Instead of desc->workspace (ignored, as is desc->workspace_bytes) the call
 * uses a fixed scratch array of KVSHOT_STATIC_WORKSPACE_BYTES inside the
 * library; every GPU that loads the library holds that array until the
 * process exits.  The call itself allocates nothing.
 *  - Descriptors whose work plan needs more scratch than that
 *    (kvshot_draft_attn_workspace_size(desc) > KVSHOT_STATIC_WORKSPACE_BYTES)
 *    are rejected with KVSHOT_ERR_WORKSPACE before anything is launched.
 *  - The first call on each device looks up the array's device address (with
 *    that device current) and keeps it for the life of the process; make that
 *    first call before any stream capture.  The kept address belongs to the
 *    device's primary context: after cudaDeviceReset (or any teardown of that
 *    context) it is stale, and the entry point must not be called again in
 *    that process.
 *  - All calls on a device share the one array and it keeps the last call's
 *    contents.  Nothing in it has to start at zero, but two calls whose
 *    kernels overlap on the GPU (e.g. on different streams without ordering)
 *    race on it and corrupt each other's results; keep such calls ordered.
 */
kvshot_status kvshot_draft_attn_static(const kvshot_attn_desc* desc, const void* q, const void* target_k,
                                       const void* target_v, const int32_t* page_table, const int32_t* seq_lens,
                                       const void* draft_k, const void* draft_v, const int32_t* tree_parent,
                                       void* out, float* lse, kvshot_stream_t stream);

/*
 * Draft append with RoPE: the drafter's new K/V for draft positions j > t
 * enter M_i (App. B: past the verified prefix the memory holds keys and
 * values that the drafter computes itself with its own projection weights;
 * those projections are upstream GEMMs), with rotary position embedding
 * applied to q and k (RoPE re-application, Sec. 3.2).
 *
 * For cache c and new node i in [0, n_new) at position pos = positions[c, i]:
 *   theta_j = pos * rope_base^(-2j / 128),  j in [0, 64)
 *   rot(x)[j]      = x[j] cos(theta_j) - x[j + 64] sin(theta_j)
 *   rot(x)[j + 64] = x[j + 64] cos(theta_j) + x[j] sin(theta_j)
 *   q_out[c, i, h]              = bf16(rot(q_in[c, i, h]))      for h < hq
 *   draft_k[c, kh, n0 + i]      = bf16(rot(k_in[c, i, kh]))     for kh < hkv
 *   draft_v[c, kh, n0 + i]      = v_in[c, i, kh]                (copied bit for bit)
 * The stored values are those of angles and rotations evaluated in fp64 and rounded once to bf16 (nearest even).
 *
 * q_in:  [C, n_new, hq, 128] bf16; k_in, v_in: [C, n_new, hkv, 128] bf16; positions: [C, n_new] int32 >= 0.
 * draft_k/v: [C, hkv, n_max, 128] bf16 (desc->n_max); requires 0 <= n0 and n0 + n_new <= n_max.
 * q_out: [C, n_new, hq, 128] bf16; may equal q_in (in place) but must not partially overlap it.
 * All bf16 pointers 16-byte aligned.  Only num_caches, hq, hkv, head_dim and n_max of desc are read.
 * n_new == 0 is a no-op returning KVSHOT_OK.
 */
kvshot_status kvshot_draft_append(const kvshot_attn_desc* desc, const void* q_in, const void* k_in,
                                  const void* v_in, const int32_t* positions, int32_t n0, int32_t n_new,
                                  float rope_base, void* draft_k, void* draft_v, void* q_out,
                                  kvshot_stream_t stream);

/*
 * Gated-delta fusion of the hybrid drafter (Sec. 3.4, Eqs. "self-attn",
 * "cross-attn", "delta" and "fusion").  For every draft token t, with n_t the
 * self-attention branch (the EAGLE-3 path) and o_t the cross-attention
 * branch (re-attention to the target KV):
 *   delta_t = o_t - n_t
 *   g_t     = sigmoid(W_g [n_t; o_t; delta_t] + b_g)
 *   h_t     = n_t + g_t (.) (W_delta delta_t)
 * The attention of both branches is kvshot_draft_attn: over the target prefix
 * and the draft KV for o, over the drafter's own draft KV alone (every
 * seq_lens[c] = 0) for n.  Products accumulate in fp32 and delta is never
 * rounded (W delta is formed as W o - W n in fp32); h is rounded once to bf16
 * (nearest even).
 *
 * n, o:     [T, d] bf16, row-major (token-major), 16-byte aligned.
 * w_g:      [d, 3d] bf16, row-major: row i holds output feature i's weights
 *           over the inputs [n; o; delta].  16-byte aligned.
 * b_g:      [d] bf16, 8-byte aligned.
 * w_delta:  [d, d] bf16, row-major, 16-byte aligned.
 * h:        [T, d] bf16, 8-byte aligned; must not overlap n, o or the workspace.
 * desc->hidden = d: a positive multiple of 128, at most 32768 (else
 * KVSHOT_ERR_UNSUPPORTED); desc->num_tokens = T >= 0 (0: no-op), T * d < 2^31.
 * Workspace: kvshot_gated_delta_workspace_size(desc) bytes (the fp32 partial
 * products, 16 T d bytes), 256-byte aligned; nothing in it has to be
 * initialised.  Errors follow the conventions at the top of this file.
 */
typedef struct kvshot_fusion_desc {
  int32_t num_tokens;        /* T */
  int32_t hidden;            /* d */
  void* workspace;           /* device scratch, 256-byte aligned */
  size_t workspace_bytes;
  int32_t* err_flag;         /* optional device int32, 0 before the call (KVSHOT_ERR_TIMEOUT) */
} kvshot_fusion_desc;

/* Bytes of workspace kvshot_gated_delta needs; 0 if the descriptor is invalid. */
size_t kvshot_gated_delta_workspace_size(const kvshot_fusion_desc* desc);

kvshot_status kvshot_gated_delta(const kvshot_fusion_desc* desc, const void* n, const void* o, const void* w_g,
                                 const void* b_g, const void* w_delta, void* h, kvshot_stream_t stream);

/*
 * Linear projection of multi-layer target KV for the KV-only drafter
 * (Sec. 3.2, injection strategy "linear projection"; "Proj + RoPE fix").
 * For every newly verified token t (desc->num_tokens = T of them), with
 * d_kv = hkv * 128 and L = desc->num_layers sampled target layers:
 *   K'(t) = W_K [K_1(t); ...; K_L(t)],   V'(t) = W_V [V_1(t); ...; V_L(t)]
 * and, with KVSHOT_PROJECT_ROPE, K'(t) is rotated again by RoPE at the
 * token's position (rotate-half pairs (j, j + 64) of every head,
 * theta_j = pos * rope_base^(-2j/128), as in kvshot_draft_append).  K'(t) and
 * V'(t) are rounded to bf16 and stored in slot positions[t] of cache
 * token_cache[t] of the reused cache that kvshot_draft_attn reads as its
 * target K/V; other slots are left untouched.  Products accumulate in fp32.
 *
 * k_in, v_in:  [T, L, hkv, 128] bf16: the tokens' K / V of the L layers (K post-RoPE, as cached).
 * w_k, w_v:    [d_kv, L * d_kv] bf16, row-major (row i: output feature i over the concatenated inputs).
 * token_cache: [T] int32 in [0, num_caches); positions: [T] int32 >= 0, below the cache's capacity.
 * page_table:  paged cache (non-NULL): [num_caches, max_pages_per_seq] int32; k_out / v_out are
 *              [num_pages, hkv, page_size, 128] bf16.  Contiguous (NULL): k_out / v_out are
 *              [num_caches, hkv, l_cap, 128] bf16.
 * All bf16 pointers 16-byte aligned, int32 pointers 4-byte aligned.  num_layers <= 8, hkv <= 64.
 * Device-side errors (a cache, position or page id out of range) skip that token's store and set
 * KVSHOT_ERR_DEVICE_BOUNDS.  T == 0 is a no-op.
 * Workspace: kvshot_kv_project_workspace_size(desc) bytes (8 L T d_kv), 256-byte aligned.  It is checked as
 * before, but not read or written: the partial sums stay on the chip.
 */
#define KVSHOT_PROJECT_ROPE 0x1u /* re-apply RoPE to the projected keys ("Proj + RoPE fix") */

typedef struct kvshot_project_desc {
  int32_t num_tokens;        /* T */
  int32_t num_layers;        /* L >= 1 */
  int32_t hkv;               /* KV heads */
  int32_t head_dim;          /* must be 128 */
  int32_t num_caches;        /* caches of the output (reused) cache */
  int32_t page_size;         /* paged output: tokens per page */
  int32_t max_pages_per_seq; /* paged output: row stride of page_table */
  int32_t num_pages;         /* paged output: pages in the pools */
  int32_t l_cap;             /* contiguous output: token capacity per (cache, KV head) */
  float rope_base;           /* > 0 (used with KVSHOT_PROJECT_ROPE) */
  uint32_t flags;            /* KVSHOT_PROJECT_ROPE or 0 */
  void* workspace;           /* device scratch, 256-byte aligned */
  size_t workspace_bytes;
  int32_t* err_flag;         /* optional device int32, 0 before the call */
} kvshot_project_desc;

/* Bytes of workspace kvshot_kv_project needs (0 if the descriptor is invalid; the layout is read
 * from page_size > 0 for this query). */
size_t kvshot_kv_project_workspace_size(const kvshot_project_desc* desc);

kvshot_status kvshot_kv_project(const kvshot_project_desc* desc, const void* k_in, const void* v_in,
                                const void* w_k, const void* w_v, const int32_t* token_cache,
                                const int32_t* positions, const int32_t* page_table, void* k_out, void* v_out,
                                kvshot_stream_t stream);

/*
 * kvshot_draft_append with QK-norm (App. D, Tab. ablations, the "QK-Norm"
 * training regime, which the paper names without a formula; read as Qwen3's
 * attention, which normalises q and k per head before RoPE): every
 * 128-wide q and k head is first scaled to unit RMS and by its weights,
 *   x <- x / sqrt(mean_j x_j^2 + eps) * w        (w = q_norm_w or k_norm_w)
 * and then rotated exactly as kvshot_draft_append does; v is stored as is.
 * Computed in fp32 and rounded once to bf16 (so not bit-identical to an fp64
 * evaluation: the results are within one bf16 rounding step of it).
 * q_norm_w, k_norm_w: [128] bf16, 4-byte aligned.  eps > 0 (Qwen3: 1e-6).
 * Every other argument as for kvshot_draft_append.
 */
kvshot_status kvshot_draft_append_qknorm(const kvshot_attn_desc* desc, const void* q_in, const void* k_in,
                                         const void* v_in, const int32_t* positions, int32_t n0, int32_t n_new,
                                         float rope_base, const void* q_norm_w, const void* k_norm_w, float eps,
                                         void* draft_k, void* draft_v, void* q_out, kvshot_stream_t stream);

/*
 * The 4-bit target cache (not in the paper: a cache-compression variant, a quarter of the bf16 cache's bytes and a bit
 * more than half of the fp8 one's) and its four entry points: kvshot_cache_extend finds the slots of newly verified
 * tokens, kvshot_kv4_store quantises their K and V into them, kvshot_draft_attn_kv4 attends to the cache and
 * kvshot_kv4_load reads values back.
 *
 * Values.  A token's K (or V) of one KV head is 8 blocks of 16 consecutive dims.  A block has a scale s, an e4m3 number
 * (OCP FP8) in [2^-9, 448], and 16 codes, e2m1 numbers (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3,
 * 4, 6 and their negatives); the value of a dim is code * s * 2^k_scale_exp (keys) or 2^v_scale_exp (values).  It has
 * at most 6 significant bits, so it is exact in bf16, and without the power of two exact in f16.
 * Quantising a block of x_i, exactly as written (roundings to nearest, ties to the even code):
 *   y_i = x_i 2^-exp,   s = e4m3(min(max(max_i |y_i| / 6, 2^-9), 448)),   code_i = e2m1(y_i / s), saturating at 6.
 * An infinity saturates; a NaN makes the block's scale NaN (0x7F), and with it all 16 values.
 *
 * Layout.  KVSHOT_KV4_GROUP_TOKENS = 16 consecutive tokens of one KV head are a group of KVSHOT_KV4_GROUP_BYTES = 2304
 * bytes; a page of page_size tokens (a multiple of 16) holds page_size / 16 groups per KV head:
 *   cache: [num_pages][hkv][page_size / 16][2304]
 * Inside a group, with token t in [0, 16):
 *   byte  c * 256 + t * 16 + i          K codes of dims 32 c + 2 i (low nibble) and 32 c + 2 i + 1, c in [0, 4), i in [0, 16)
 *   byte  1024 + ...                    V codes, laid out alike
 *   byte  2048 + t * 8 + b              K scale of block b (dims 16 b .. 16 b + 15)
 *   byte  2176 + t * 8 + b              V scale of block b
 * A slot is page * page_size + (place in the page).  A contiguous cache [num_caches][hkv][l_cap / 16][2304] is the same
 * with one page of l_cap tokens (a multiple of 16) per cache.
 */
#define KVSHOT_KV4_GROUP_TOKENS 16
#define KVSHOT_KV4_GROUP_BYTES 2304

/*
 * Room for newly verified tokens: block tables and slot maps from lengths, on the device.
 * Cache c holds seq_lens[c] = L_c tokens in its first ceil(L_c / page_size) pages and gets n_c = new_tokens[c] >= 0
 * more.  Pages that it lacks come off the end of the list of free pages, in cache order: with need_c new pages for cache
 * c and base_c = sum over b < c of need_b, its new pages are free_pages[F - 1 - base_c], free_pages[F - 2 - base_c], ...
 * (F = *free_count), in that order.  Written:
 *   page_table_out  page_table with the new pages' entries (other entries are copied; in place only new ones are written)
 *   seq_lens_out    L_c + n_c
 *   free_count_out  F - sum need_c
 *   token_start     [C + 1]: cache c's new tokens are token_start[c] .. token_start[c + 1] - 1 of the packed order
 *   slots, token_cache, positions   [max_tokens]: slot, cache and position L_c + i of each packed token; -1 past the last
 *                   (a fixed max_tokens keeps the sizes that a captured graph needs).  Any of the three may be NULL.
 * The slots are those of kvshot_kv4_store, and (page, offset) of any paged cache of this library.
 * seq_lens_out, page_table_out and free_count_out may be seq_lens, page_table and free_count; nothing else may overlap.
 * All or nothing: if a length or count is negative or a row, the free list or max_tokens too small, or a free page's id
 * outside [0, num_pages), KVSHOT_ERR_DEVICE_BOUNDS is recorded and nothing is taken: lengths, table and free list are
 * copied as they are, token_start is all 0 and the maps all -1.
 */
typedef struct kvshot_extend_desc {
  int32_t num_caches;        /* C in [1, 1024] */
  int32_t page_size;         /* tokens per page, >= 1 */
  int32_t max_pages_per_seq; /* row length of page_table */
  int32_t num_pages;         /* pages in the pool */
  int32_t num_free;          /* entries of free_pages (an upper bound of *free_count) */
  int32_t max_tokens;        /* entries of slots, token_cache and positions */
  int32_t* err_flag;         /* optional device int32, 0 before the call */
} kvshot_extend_desc;

kvshot_status kvshot_cache_extend(const kvshot_extend_desc* desc, const int32_t* seq_lens, const int32_t* new_tokens,
                                  const int32_t* page_table, const int32_t* free_pages, const int32_t* free_count,
                                  int32_t* seq_lens_out, int32_t* page_table_out, int32_t* free_count_out,
                                  int32_t* token_start, int32_t* slots, int32_t* token_cache, int32_t* positions,
                                  kvshot_stream_t stream);

/*
 * kvshot_kv4_store: K and V of num_tokens tokens quantised into the slots slots[t] of the cache.
 * kvshot_kv4_load:  the values in those slots, as bf16 (exact; beyond bf16's range, infinite).
 * k, v: [num_tokens][hkv][128] bf16, 16-byte aligned, token t at t * k_stride (v_stride) elements, multiples of 8 and
 * at least hkv * 128 (0 selects hkv * 128): K and V may be slices of a fused projection's rows.
 * slots: [num_tokens] int32.  A slot of -1 is passed over (load: zeros); one outside the cache is too, and recorded as
 * KVSHOT_ERR_DEVICE_BOUNDS.  Slots of one store must differ, or either token may be what the slot then holds.
 * cache: 16-byte aligned, kvshot_kv4_cache_bytes bytes; other slots keep their values.
 * num_tokens == 0 is a no-op.
 */
typedef struct kvshot_kv4_desc {
  int32_t num_tokens;  /* T >= 0 */
  int32_t hkv;         /* KV heads */
  int32_t head_dim;    /* must be 128 */
  int32_t page_size;   /* tokens per page, a multiple of 16 (contiguous cache: l_cap) */
  int32_t num_pages;   /* pages in the cache (contiguous cache: num_caches); num_pages * hkv * page_size < 2^31 */
  int32_t k_scale_exp; /* |exp| <= 64 */
  int32_t v_scale_exp;
  int64_t k_stride;    /* elements between tokens of k, v; 0: hkv * 128 */
  int64_t v_stride;
  int32_t* err_flag;   /* optional device int32, 0 before the call */
} kvshot_kv4_desc;

/* Bytes of a 4-bit cache, 0 if the sizes are invalid. */
size_t kvshot_kv4_cache_bytes(int32_t num_pages, int32_t hkv, int32_t page_size);

kvshot_status kvshot_kv4_store(const kvshot_kv4_desc* desc, const void* k, const void* v, const int32_t* slots,
                               void* cache, kvshot_stream_t stream);
kvshot_status kvshot_kv4_load(const kvshot_kv4_desc* desc, const void* cache, const int32_t* slots, void* k, void* v,
                              kvshot_stream_t stream);

/*
 * kvshot_draft_attn over a 4-bit target cache, with an optional sliding window.  Arguments, results and errors as
 * there, except:
 *  - cache: the 4-bit cache, paged (page_table != NULL, desc->page_size a multiple of 16) or contiguous (page_table
 *    NULL, desc->l_cap a multiple of 16), 16-byte aligned; scales 2^desc->k_scale_exp and 2^desc->v_scale_exp.
 *  - desc->flags: KVSHOT_TREE and KVSHOT_OVERLAP_PREVIOUS (which then covers seq_lens, page_table, cache and
 *    tree_parent); others return KVSHOT_ERR_UNSUPPORTED.
 *  - Lengths (max_seq_len, or the room that the table or the cache has, if that is less) and twice n_nodes sum up to
 *    2^31 - 129 at most (else KVSHOT_ERR_UNSUPPORTED): positions are 32-bit numbers.
 *  - window = W > 0: a node at position p (a node of depth d, 1 for a child of the last verified token, stands at
 *    L_c + d - 1; the target token j at j) sees a key that it would see otherwise only if the key's position is above
 *    p - W, or below `sinks`.  A node always sees itself.  window = 0: no window (sinks is not used then).
 *    A page is not read, nor its entry of page_table, if it holds no sink and no token that a node of the least depth
 *    sees: of depth n_nodes - n_query + 1, for a tree 1.  Of other pages, too, most such tokens are not read.
 *  - q, the softmax weights and the draft K/V are rounded to f16 for the tensor cores (finite magnitudes up to 65504;
 *    those below 2^-14 lose bits), the cache's values are exact.  The running sums are fp32.
 *  - A NaN stored in a token or draft slot that some query row sees may reach the other rows of its KV head's group.
 * The workspace is kvshot_draft_attn_kv4_workspace_size bytes (0 if the descriptor is invalid).
 */
size_t kvshot_draft_attn_kv4_workspace_size(const kvshot_attn_desc* desc, int32_t window, int32_t sinks);
kvshot_status kvshot_draft_attn_kv4(const kvshot_attn_desc* desc, const void* q, const void* cache,
                                    const int32_t* page_table, const int32_t* seq_lens, const void* draft_k,
                                    const void* draft_v, const int32_t* tree_parent, int32_t window, int32_t sinks,
                                    void* out, float* lse, kvshot_stream_t stream);

/*
 * Drafting over a part of a long target cache (not in the paper).  A page of the target cache none of whose keys can score
 * high need not be read for a draft token, and a token that draft tokens gave little weight need not be kept.
 *   kvshot_page_bounds   least and greatest key of each page             (after the cache grew)
 *   kvshot_page_scores   greatest possible score of each page, for every draft token and KV head
 *   kvshot_select_top    the best entries of each row of scores: pages to read, or tokens to keep
 *   kvshot_draft_attn_sparse   draft attention over the selected pages and the draft K/V
 *   kvshot_key_weights   softmax weights that the cached tokens got, accumulated
 *   kvshot_cache_evict   the tokens to keep moved to the front, and the other pages given back
 * The first two, the fourth and the fifth take a kvshot_attn_desc and read of it num_caches, num_seqs, hq, hkv, head_dim,
 * page_size, max_pages_per_seq, num_pages, max_seq_len, n_nodes, n_query, n_max, scale, flags, err_flag and wait_limit_ns as
 * kvshot_draft_attn does (kvshot_page_bounds no query heads' or nodes' fields: they may be 0, and are checked if they are
 * not).  Caches are bf16 and paged (kvshot_key_weights: or contiguous), q is [C, Nq, hq, 128] bf16, and the q heads of one
 * KV head are at most 32.
 * KVSHOT_TARGET_FP8 and the KVSHOT_FORCE_ flags return KVSHOT_ERR_UNSUPPORTED; KVSHOT_OVERLAP_PREVIOUS has no effect.
 * A length outside [0, min(max_seq_len, capacity)] is recorded as KVSHOT_ERR_DEVICE_BOUNDS and clamped to it, a page id
 * outside the pool recorded and its page passed over.  16-byte alignment of all bf16 pointers, 4 of int32 and fp32.
 */

/*
 * bounds[pid, h, 0, d] = min, bounds[pid, h, 1, d] = max over the tokens of the page below the cache's length, of key
 * element d of KV head h (NaN if one of them is): [num_pages, hkv, 2, 128] bf16, by pool page, so that bounds stay with
 * their page.  Computed for the pages that hold a token at or past from_tokens[c] (a length before the cache grew; NULL:
 * all pages); other entries are left as they are.  Whatever else writes keys below a length, kvshot_cache_evict in place
 * among it, leaves bounds behind that are not of these keys: compute them anew with NULL.  A page that several caches
 * share has to hold the same number of tokens below each one's length.
 */
kvshot_status kvshot_page_bounds(const kvshot_attn_desc* desc, const void* target_k, const int32_t* page_table,
                                 const int32_t* seq_lens, const int32_t* from_tokens, void* bounds,
                                 kvshot_stream_t stream);

/*
 * scores[c, n, h, p] = scale * max over the q heads g of KV head h of sum_d max(q_gd min_d, q_gd max_d), with the bounds
 * of page p of cache c: no key of the page scores higher for draft token n.  [C, Nq, hkv, max_pages_per_seq] fp32; entries
 * past a cache's last page are left as they are.  Products accumulate in fp32.  Bounds and q must be finite, and bounds
 * 32-byte aligned.
 */
kvshot_status kvshot_page_scores(const kvshot_attn_desc* desc, const void* q, const void* bounds,
                                 const int32_t* page_table, const int32_t* seq_lens, float* scores,
                                 kvshot_stream_t stream);

/*
 * The best entries of each row.  Row r has n_r = ceil(seq_lens[r / rows_per_len] / tokens_per_entry) entries, of which
 * min(n_r, keep) are picked: the first `first`, the last `last`, and of the others those with the highest scores; of equal
 * ones (0 and -0 are) the lowest index, and a NaN is above every number.
 * picks: [num_rows, keep] int32, ascending, -1 past the last; counts: [num_rows] int32.
 * scores: [num_rows, row_len] fp32.  A row that is longer than row_len is recorded as KVSHOT_ERR_DEVICE_BOUNDS and has
 * row_len entries, a negative length 0.  num_rows == 0 is a no-op.
 * For kvshot_page_scores: num_rows = C Nq hkv, row_len = max_pages_per_seq, rows_per_len = Nq hkv, tokens_per_entry =
 * page_size.  For weights of tokens: num_rows = C, rows_per_len = tokens_per_entry = 1.
 */
typedef struct kvshot_select_desc {
  int32_t num_rows;
  int32_t row_len;
  int32_t rows_per_len;     /* >= 1; num_rows is a multiple of it */
  int32_t tokens_per_entry; /* >= 1 */
  int32_t keep;             /* >= 1 */
  int32_t first;            /* >= 0 */
  int32_t last;             /* >= 0; first + last <= keep */
  int32_t* err_flag;        /* optional device int32, 0 before the call */
} kvshot_select_desc;

kvshot_status kvshot_select_top(const kvshot_select_desc* desc, const float* scores, const int32_t* seq_lens,
                                int32_t* picks, int32_t* counts, kvshot_stream_t stream);

/*
 * kvshot_draft_attn with the prefix tokens of each query row and KV head limited to the pages picked for it: out and lse of
 * row n and the q heads of KV head h are over the tokens below L_c in the pages page_table[c, picks[c, n, h, i]],
 * i < counts[c, n, h], and the draft keys that kvshot_draft_attn gives that row.
 * picks: [C, Nq, hkv, max_picks] int32, each list ascending; counts: [C, Nq, hkv] int32 in [0, max_picks].  A pick that
 * is not above its predecessor or not a page below the cache's length is recorded as KVSHOT_ERR_DEVICE_BOUNDS and passed
 * over (a page that comes again later in such a list may count twice), a count out of range recorded and clamped; entries
 * of picks past a count may be anything.  Other arguments as for kvshot_draft_attn, but target_k/v and draft_k/v 32-byte
 * aligned.
 * The softmax weights are rounded to bf16 for the tensor cores, sums are fp32.  A NaN or infinity stored in a value that some
 * row of the KV head sees may reach the cache's other rows of that head.
 * Workspace: kvshot_draft_attn_sparse_workspace_size bytes (0 if the descriptor is invalid), as for kvshot_draft_attn.
 */
size_t kvshot_draft_attn_sparse_workspace_size(const kvshot_attn_desc* desc, int32_t max_picks);
kvshot_status kvshot_draft_attn_sparse(const kvshot_attn_desc* desc, const void* q, const void* target_k,
                                       const void* target_v, const int32_t* page_table, const int32_t* seq_lens,
                                       const int32_t* picks, const int32_t* counts, int32_t max_picks,
                                       const void* draft_k, const void* draft_v, const int32_t* tree_parent, void* out,
                                       float* lse, kvshot_stream_t stream);

/*
 * weights_out[c, j] = decay * weights[c, j] + sum over the query rows n and q heads of exp(scale q . k_j - lse[c, n, head])
 * for every token j < L_c: what the softmax whose lse kvshot_draft_attn returned gave the token, summed.  A row whose lse
 * is -inf adds nothing.  q, and keys below the length, must be finite.  [C, weights_len] fp32; entries past the length are
 * left as they are.  weights may be weights_out, or NULL (zeros).  decay in [0, 1]; with 0 weights is not read.  Sums are
 * fp32 and their order fixed.
 * page_table NULL: a contiguous cache [C, hkv, l_cap, 128].  A length above weights_len is recorded as out of bounds, too.
 */
kvshot_status kvshot_key_weights(const kvshot_attn_desc* desc, const void* q, const void* target_k,
                                 const int32_t* page_table, const int32_t* seq_lens, const float* lse, float decay,
                                 int32_t weights_len, const float* weights, float* weights_out, kvshot_stream_t stream);

/*
 * Eviction.  Cache c keeps m_c = kept_count[c] of its L_c tokens: token kept[c, i] becomes token i, for all KV heads of K
 * and V and in the weights.
 *   k, v -> k_out, v_out    [num_pages, hkv, page_size, 128] bf16, in place (k_out = k, v_out = v, page_table_out =
 *                           page_table), or into other pools of num_pages_out pages through page_table_out, a smaller
 *                           copy for instance.  Slots past the last kept token are left as they are.  Bounds of the
 *                           pages (kvshot_page_bounds) do not follow: compute them anew for all pages.
 *   weights -> weights_out  [C, weights_len] -> [C, weights_len_out] fp32, 0 past the kept tokens' (what a token that comes
 *                           later starts with); in place, or not overlapping; both may be NULL
 *   seq_lens_out            m_c
 *   free_pages, free_count_out   page_table's pages past the first ceil(m_c / page_size) of cache c's ceil(L_c / page_size),
 *                           put behind the *free_count free ones, cache after cache, ascending: what kvshot_cache_extend
 *                           takes from.  free_pages, free_count and free_count_out may all be NULL.
 * seq_lens_out may be seq_lens, free_count_out may be free_count; nothing else may overlap.  Pages must not be shared
 * between caches.  kept: [C, max_kept] int32, ascending, below L_c.
 * Device errors are recorded as KVSHOT_ERR_DEVICE_BOUNDS: a length that the table has no room for, or a count below 0 or
 * above what the length, max_kept, page_table_out or weights_len_out has room for (that cache's tokens, length and pages stay
 * as they are; seq_lens_out is the length, clamped to the table's room); a kept index out of order or range (that cache's
 * contents are then unspecified); page ids outside their pool (nothing is moved there; one that is given back goes on the
 * list as it is); more free pages than num_free (none is given back).
 */
typedef struct kvshot_evict_desc {
  int32_t num_caches;        /* C in [1, 1024] */
  int32_t hkv;
  int32_t head_dim;          /* must be 128 */
  int32_t page_size;         /* >= 1 */
  int32_t max_pages_per_seq; /* row length of page_table */
  int32_t num_pages;         /* pages in k and v */
  int32_t max_pages_out;     /* row length of page_table_out */
  int32_t num_pages_out;     /* pages in k_out and v_out */
  int32_t max_kept;          /* row length of kept */
  int32_t weights_len;       /* row lengths of weights and weights_out */
  int32_t weights_len_out;
  int32_t num_free;          /* entries of free_pages */
  int32_t* err_flag;         /* optional device int32, 0 before the call */
} kvshot_evict_desc;

kvshot_status kvshot_cache_evict(const kvshot_evict_desc* desc, const void* k, const void* v, const int32_t* page_table,
                                 const int32_t* seq_lens, const int32_t* kept, const int32_t* kept_count,
                                 const float* weights, void* k_out, void* v_out, const int32_t* page_table_out,
                                 int32_t* seq_lens_out, float* weights_out, int32_t* free_pages,
                                 const int32_t* free_count, int32_t* free_count_out, kvshot_stream_t stream);

/* Static description of a status code (never NULL). */
const char* kvshot_status_string(kvshot_status status);

/* Library version, major * 10000 + minor * 100 + patch. */
int32_t kvshot_version(void);

#ifdef __cplusplus
}
#endif
#endif /* KVSHOT_H */
