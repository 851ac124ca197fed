/*
 * routerelay.h -- C ABI of librouterelay.so, the MI355X (gfx950) route-
 * maintenance path of RouteRelay (arXiv 2609.07306).
 *
 * Problem (Sec. 2.1, Eq. (1)-(2)): per query head h, chunk representations
 * Qc[h] in R^{n_q x d} and Kc[g] in R^{n_k x d} (g = h / (H_q / H_kv)) give
 * scores S = Qc Kc^T, and row i routes to the k best key chunks.  RouteRelay
 * (Sec. 3) keeps, per row, a ledger of the selected set R, m near-miss and r
 * random sentinels C, and the layer the entry was built at.  Anchor layers
 * rebuild every entry; intermediate (relay) layers rescore R u C, keep the
 * route of a row when its weakest selected score beats its strongest sentinel
 * by more than gamma, and fully reroute the other rows only (Sec. 3.2,
 * Sec. 4.1-4.2).
 *
 * Conventions shared by every call:
 *   - Tensors are DEVICE pointers owned by the caller, row-major, contiguous.
 *     Qc is [H_q, n_q, d] and Kc is [H_kv, n_k, d], binary32 (RR_F32) or bf16
 *     (RR_BF16, 16-bit storage).  Scores are accumulated in binary32.
 *   - Row index: row = h * n_q + i.  The causal chunk mask lets row i select
 *     key chunks j <= i only (needs n_q == n_k); such a row has n_i = i + 1
 *     valid chunks, a row without the mask has n_i = n_k.
 *   - A route is a SET, stored sorted by ascending chunk id and padded with
 *     -1 (a row with n_i < k routes to all of its valid chunks).  Ties in
 *     score are broken toward the lower chunk id; -0 equals +0.
 *   - Scores may be any finite float or infinity.  A NaN ranks with -inf in the
 *     tiles that keep their scores in registers (see the options); the two-sweep
 *     tiles must not meet one.
 *   - Every call enqueues work on the given HIP stream (NULL: the null
 *     stream) and returns; outputs, including device counters, are valid once
 *     that stream has reached the enqueued work.  No call synchronises the
 *     host with the device and none allocates memory, except
 *     rr_ledger_create.
 *   - The caller keeps Qc, Kc and the output buffers alive until the stream
 *     has passed the call.  A ledger is used by one host thread on one stream
 *     at a time.
 *   - Errors are reported by the return value; rr_last_error() returns a
 *     message for the calling thread's most recent failure.  Argument errors
 *     are detected before any work is enqueued.
 */
#ifndef ROUTERELAY_H
#define ROUTERELAY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RR_OK = 0,
    RR_ERR_INVALID = -1,     /* an argument or configuration value is invalid */
    RR_ERR_OOM = -2,         /* device allocation failed */
    RR_ERR_HIP = -3,         /* a HIP runtime call failed (message in rr_last_error) */
    RR_ERR_STATE = -4,       /* call order violated (relay before any anchor, layer going back) */
    RR_ERR_UNSUPPORTED = -5  /* valid but outside the shapes the library supports */
} rr_status;

/* (RR_E4M3, eight bits of the OCP e4m3 form, is a type of paged caches only.) */
typedef enum { RR_F32 = 0, RR_BF16 = 1, RR_E4M3 = 2 } rr_dtype;

/* Shape and rule parameters.  Supported: d in {32, 64, 128} (and 256 for
 * bf16); 1 <= k <= n_k; k + m <= 128; k + m + r + n_sink + n_recent <= 256;
 * n_k <= 8192;
 * n_heads a multiple of n_kv_heads; gamma not NaN.  gamma is the guard
 * margin of Eq. (8); the paper uses gamma >= 0 (0 by default, Table 1);
 * +INFINITY refreshes every row that has a sentinel and -INFINITY refreshes
 * none.  seed keys the random-sentinel probes. */
/* Options (rr_config.options).  A relay layer (Sec. 3.2) runs as one of two
 * schedules with the same results:
 *   one pass -- over the row tiles of every head, the tile's scores rescore
 *     its rows' ledgers, the trigger flags rows, and the same pass routes the
 *     flagged ones.  Up to 2048 key chunks, and up to 4096 unless a row has
 *     more than 440 route, sentinel and draw slots, a 32-row tile keeps its
 *     scores in registers; other tiles sweep the keys twice and hold the
 *     ledgers as bitmaps in LDS (n_k up to 3072; k + m > 64: 4608; rows of 512
 *     bytes, d = 128 binary32 or 256 bf16: 3072 with k + m > 64 only);
 *   split -- rescoring and trigger, then the routing of the flagged rows
 *     compacted per head (Sec. 4.2).
 * By default the one measured faster for the shape runs: one pass up to 2048
 * chunks and for causal inputs where it fits, but the split schedule for many
 * bf16 rows with k + m up to about 52 over more than 1024 chunks, and for
 * non-causal inputs beyond.  Where most rows keep their route and rows are
 * many, the split schedule can be the faster one elsewhere too.
 * RR_OPT_SPLIT_RELAY forces the split schedule, RR_OPT_ONE_PASS_RELAY the one
 * pass (RR_ERR_UNSUPPORTED where no tile takes it); not both. */
typedef enum { RR_OPT_SPLIT_RELAY = 1, RR_OPT_ONE_PASS_RELAY = 2 } rr_option;

typedef struct {
    int32_t n_heads;    /* H_q */
    int32_t n_kv_heads; /* H_kv */
    int32_t n_q;        /* query chunks per head */
    int32_t n_k;        /* key chunks per head */
    int32_t d;          /* representation width */
    int32_t k;          /* route width */
    int32_t m;          /* near-miss sentinels */
    int32_t r;          /* random sentinels */
    int32_t dtype;      /* rr_dtype of Qc and Kc */
    int32_t causal;     /* 1: chunk mask j <= i */
    float gamma;        /* guard margin */
    uint32_t options;   /* rr_option bits (0: defaults) */
    uint64_t seed;
    /* Mandatory sentinels (Sec. 3.1, item 3): the sink chunks j < n_sink and
     * the recent chunks -- the n_recent valid chunks up to the row's position
     * (row i when n_q == n_k, else the last key chunk) -- that are not in R or
     * N, kept ascending in n_sink + n_recent extra sentinel slots after the
     * random ones (-1 padded) and left out of the random draws. */
    int32_t n_sink;
    int32_t n_recent;
    /* Minimum reuse horizon (Sec. 3.2, Hysteresis): a row (re)built at layer
     * b is not rerouted at layers b+1 .. b+min_reuse.  0: off. */
    int32_t min_reuse;
    int32_t reserved;           /* must be 0 */
    /* Per-row guard margins gamma_i of Eq. (8): a device array of H_q*n_q
     * binary32 values read by every relay (the caller may change them between
     * layers, e.g. to raise the margin of recently refreshed rows); NULL: the
     * scalar gamma for every row.  Values must not be NaN. */
    const float *gamma_rows;
    /* Query-dependent route budgets (Sec. 4.3): a device array of H_q*n_q
     * int32 route widths k_i, read by every routing call (full, anchor,
     * relay).  Row i routes to its k_i best chunks, in its first k_i route
     * slots (the other k - k_i are -1), and its near-miss sentinels are the m
     * chunks ranked after them.  Rows of every width share the launches (one
     * bucket).  Values outside [1, k] are clamped to it.  NULL: k for every
     * row. */
    const int32_t *k_rows;
} rr_config;

typedef struct rr_ledger rr_ledger;

/* Route ledger (Sec. 3.1, Eq. (4); state tensors of Sec. 4.1).  Allocates,
 * on the current HIP device, the structure-of-arrays ledger -- routes
 * [H_q*n_q, k], sentinels [H_q*n_q, m+r+n_sink+n_recent] (near-miss slots
 * first, sorted by id; then random slots in draw order; then mandatory slots,
 * sorted by id; -1 padded), build layer and age
 * [H_q*n_q] int32 -- plus the per-row scratch of the relay path.  *out
 * receives the handle (NULL on failure).  Returns RR_ERR_INVALID /
 * RR_ERR_UNSUPPORTED for a bad config, RR_ERR_OOM if allocation fails. */
rr_status rr_ledger_create(const rr_config *cfg, rr_ledger **out);

/* Frees the ledger's device memory after synchronising the device.  NULL is
 * a no-op. */
rr_status rr_ledger_destroy(rr_ledger *ledger);

/* Anchor layer (Sec. 3.1; forced anchors, Sec. 3.2): full routing of every
 * row (Eq. (1)-(2)) that also keeps the chunks ranked k+1..k+m as near-miss
 * sentinels and draws r random sentinels from the remaining valid chunks;
 * every ledger entry is rebuilt with build layer = layer and age 0.
 *   layer   >= 0; it keys the random probes.  An anchor may restart the layer
 *           sequence (a new forward pass): later relays must not go below it.
 *   Qc, Kc  device inputs as above.
 *   routes  optional device output [H_q*n_q, k] int32 (a copy of the ledger's
 *           routes); may be NULL.
 *   pairs   optional device int64: number of scores evaluated (sum of n_i).
 */
rr_status rr_anchor_route(rr_ledger *ledger, int32_t layer, const void *Qc, const void *Kc,
                          int32_t *routes, int64_t *pairs, void *hip_stream);

/* Relay layer (Sec. 3.2, Eq. (5)-(8); dataflow of Sec. 4.1-4.2).  Each row
 * rescores its candidates A = R u C at this layer: alpha = min over R,
 * beta = max over C.  A row with a non-empty C and beta + gamma >= alpha is
 * rerouted: its full score row is computed and its ledger entry rebuilt as at
 * an anchor (build layer = layer, age 0).  Other rows keep their entry and get
 * age = layer - build layer.  Only the rerouted rows run the selection and
 * the ledger rebuild: compacted per head for a second launch (split
 * schedule), or within the rescoring launch's own tiles (one-pass schedule);
 * rr_config.options and the inputs choose the schedule, the results are the
 * same.
 *   routes      optional device output [H_q*n_q, k] int32 (copy of the
 *               ledger's routes after the update); NULL to read the ledger
 *               through rr_ledger_routes instead.
 *   mask        optional device output [H_q*n_q] uint8: 1 = rerouted.
 *   pairs       optional device int64: scores evaluated, i.e. the sum over
 *               rows of |A_i| (valid candidate slots) plus n_i per rerouted
 *               row.
 *   n_rerouted  optional device int32: number of rerouted rows.
 * Returns RR_ERR_STATE if no anchor (or import) preceded it or if layer is
 * below the previous call's layer. */
rr_status rr_relay_layer(rr_ledger *ledger, int32_t layer, const void *Qc, const void *Kc,
                         int32_t *routes, uint8_t *mask, int64_t *pairs, int32_t *n_rerouted,
                         void *hip_stream);

/* Relay layer that allocates nothing, for callers that cannot allocate
 * device memory at call time: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  The same computation and kernels as
 * rr_relay_layer, on a ledger the caller owns, in the layout rr_ledger_export
 * writes: led_routes [H_q*n_q, k], led_sent [H_q*n_q, m+r+n_sink+n_recent]
 * (may be NULL when that width is 0), led_build and led_age [H_q*n_q]
 * int32, all device memory,
 * updated in place.  The relay's scratch (flags, alpha / beta, per-workgroup
 * partials, call totals, threshold seeds, a completion counter) lives in a
 * static device area of the library, 4 MiB per GPU, held until the process
 * ends; a configuration whose scratch exceeds it (beyond about 200 000 routed
 * rows) returns RR_ERR_UNSUPPORTED before any work is enqueued.  There is no
 * call-order state: the caller keeps layers non-decreasing after an anchor
 * built the ledger.  Every call on one GPU shares that GPU's area, so calls
 * that overlap on one GPU (concurrent streams or threads) race; calls
 * ordered on one stream do not.  routes, mask, pairs and n_rerouted are as in
 * rr_relay_layer. */
rr_status rr_relay_layer_static(const rr_config *cfg, int32_t layer, const void *Qc, const void *Kc,
                                int32_t *led_routes, int32_t *led_sent, int32_t *led_build,
                                int32_t *led_age, int32_t *routes, uint8_t *mask, int64_t *pairs,
                                int32_t *n_rerouted, void *hip_stream);

/* Full routing baseline (Eq. (1)-(2)) with the same GEMM + TopK kernels and
 * no ledger: routes [H_q*n_q, cfg->k] int32 receives every row's route.
 * cfg->m and cfg->r are ignored.  route_scores (optional, [H_q*n_q, k]
 * binary32) receives the score of each route slot (padding: -INFINITY).
 * pairs (optional device int64) receives the number of scores evaluated. */
rr_status rr_full_route(const rr_config *cfg, const void *Qc, const void *Kc, int32_t *routes,
                        float *route_scores, int64_t *pairs, void *hip_stream);

/* Borrowed device view of the ledger's routes [H_q*n_q, k]; valid until the
 * next call that mutates or destroys the ledger.  NULL for a NULL ledger. */
const int32_t *rr_ledger_routes(const rr_ledger *ledger);

/* Copies the ledger state into caller device buffers (each may be NULL):
 * routes [rows,k], sent [rows,m+r+n_sink+n_recent], build [rows], age [rows]
 * int32. */
rr_status rr_ledger_export(const rr_ledger *ledger, int32_t *routes, int32_t *sent,
                           int32_t *build, int32_t *age, void *hip_stream);

/* Replaces the ledger state from caller device buffers (all four required)
 * and records `layer` as the last layer seen, so that a relay may follow.
 * The contents are trusted: ids must lie in [-1, n_i) with R sorted. */
rr_status rr_ledger_import(rr_ledger *ledger, int32_t layer, const int32_t *routes,
                           const int32_t *sent, const int32_t *build, const int32_t *age,
                           void *hip_stream);

/* Diagnostics of the most recent relay: per-row alpha and beta (binary32,
 * beta = -INFINITY for an empty C) and the compacted rerouted row ids, one
 * ascending list per head at ids[h*n_q .. h*n_q + count_h), -1 after it
 * (formed from the relay's flags when asked for).  Each output may be NULL. */
rr_status rr_ledger_relay_stats(const rr_ledger *ledger, float *alpha, float *beta,
                                int32_t *ids, void *hip_stream);

/* Kernel timing for measurement.  Between rr_profile_start and
 * rr_profile_stop every kernel the library launches is bracketed by HIP
 * events recorded on its own stream.  rr_profile_stop waits for those events
 * and returns, per kernel kind, the summed duration in milliseconds and the
 * number of launches.  total_ms and launches are caller arrays of n_kinds
 * entries (each may be NULL); RR_KERNEL_KINDS entries are written (of n_kinds
 * = 8, the kinds before RR_KERNEL_APPEND that an earlier header had, those),
 * and any other n_kinds < RR_KERNEL_KINDS with a non-NULL array returns
 * RR_ERR_INVALID without writing anything (profiling then stays on).
 * Process-wide; not for concurrent use from several threads. */
typedef enum {
    RR_KERNEL_FULL = 0,     /* GEMM + TopK, full routing */
    RR_KERNEL_ANCHOR = 1,   /* GEMM + TopK + ledger build, every row */
    RR_KERNEL_REROUTE = 2,  /* GEMM + TopK + ledger build, compacted rows */
    RR_KERNEL_RESCORE = 3,  /* rescoring (dense tiles or gather), trigger, compaction counts, ages */
    RR_KERNEL_RELAY = 4,    /* one-pass relay: rescoring + trigger + GEMM + TopK + ledger build of the flagged rows */
    RR_KERNEL_POOL = 5,     /* chunk pooling */
    RR_KERNEL_EXPAND = 6,   /* token expansion */
    RR_KERNEL_ATTENTION = 7, /* sparse attention over routed chunks */
    RR_KERNEL_APPEND = 8,   /* new tokens into the paged cache */
    RR_KERNEL_PAGED = 9,    /* attention over the paged cache */
    RR_KERNEL_JOIN = 10,    /* its parts joined, where that is a launch of its own: always behind a
                               shared prefix, otherwise for few items of many parts */
    RR_KERNEL_KINDS = 11
} rr_kernel_kind;

rr_status rr_profile_start(void);
rr_status rr_profile_stop(double *total_ms, int64_t *launches, int32_t n_kinds);

/* Exact selection (Eq. (2)) runs collection sweeps over a row's keys until
 * the row's candidate list holds exactly its top k+m (bisection on the score,
 * then on the chunk id of a tied score); the number of sweeps is capped above
 * what the bisections can need.  A row that still had not settled at the cap
 * would get an empty routed and near-miss set, and is counted here.
 * rr_unconverged_rows synchronises the current device and stores, in *count
 * (host memory), the number of such rows over every call on that device since
 * the library was loaded: 0 unless something is wrong.  A diagnostic, not for
 * the hot path. */
rr_status rr_unconverged_rows(uint64_t *count);

/* Test hook: caps the collection sweeps per route tile at `cap` for later
 * launches from this process (0 restores the default cap; the default always
 * suffices).  A lowered cap exists only to exercise rr_unconverged_rows. */
rr_status rr_set_sweep_cap(int32_t cap);

/* Number of bytes of ledger index storage (routes plus sentinels) for a
 * config: H_q * n_q * (k + m + r + n_sink + n_recent) * 4. */
size_t rr_ledger_index_bytes(const rr_config *cfg);

const char *rr_status_string(rr_status status);

/* Message of the calling thread's most recent failure ("" if none). */
const char *rr_last_error(void);

/* ------------------------------------------------------------------------
 * The steps either side of route maintenance.  Chunks are consecutive runs of
 * `chunk` tokens, the last one possibly shorter: n_chunks =
 * ceil(n_tokens / chunk), chunk j holds tokens j*chunk .. min((j+1)*chunk,
 * n_tokens) - 1.  All pointers are device memory; every call enqueues on the
 * given HIP stream (NULL: the default stream) and returns.
 * ---------------------------------------------------------------------- */

/* Chunk representations (Sec. 2.1: the router forms one representation per
 * chunk of tokens; here the mean of the chunk's token vectors).  X is
 * [n_heads, n_tokens, d] of dtype (rr_dtype), Xc receives [n_heads, n_chunks,
 * d] of the same dtype: each chunk's mean, summed in binary32 and rounded to
 * nearest even for bf16.  d a multiple of 8, at most 1024; chunk >= 1.
 * Returns RR_ERR_INVALID for bad sizes or NULL pointers. */
rr_status rr_pool_chunks(const void *X, int32_t n_heads, int32_t n_tokens, int32_t d, int32_t chunk,
                         int32_t dtype, void *Xc, void *hip_stream);

/* Token expansion (Sec. 2.1: selected chunks are expanded into token
 * indices).  routes is [rows, k] chunk ids (a ledger's or rr_full_route's
 * layout), tokens receives [rows, k*chunk] int32: route slot s fills columns
 * s*chunk .. s*chunk + chunk - 1 with its chunk's token ids ascending, -1
 * past the sequence's last token and for an empty (-1) or out-of-range slot.
 * Returns RR_ERR_INVALID for bad sizes or NULL pointers. */
rr_status rr_expand_tokens(const int32_t *routes, int64_t rows, int32_t k, int32_t chunk, int32_t n_tokens,
                           int32_t *tokens, void *hip_stream);

/* Sparse attention over routed chunks (Sec. 2.2 Eq. (3)): every query token t
 * of chunk i of head h attends, with one softmax scaled by `scale`, to the
 * tokens of the chunks in row h*n_chunks + i of routes; when causal, keys
 * after t are excluded (and routed chunks after i contribute nothing).  Slots
 * holding -1 or an id outside [0, n_chunks) are skipped; a query with no
 * admissible key gets a zero output.  Query head h reads key / value head
 * h / (n_heads / n_kv_heads).  Layouts: Q and O [n_heads, n_tokens, d], K and
 * V [n_kv_heads, n_tokens, d], bf16, row-major; routes [n_heads*n_chunks, k]
 * int32.  Scores and sums in binary32, the softmax weights rounded to bf16
 * for the value product, O rounded to nearest even.  Supported: bf16 with
 * d = 64 or 128, 1 <= k <= 256.  Returns RR_ERR_INVALID for bad sizes or NULL
 * pointers, RR_ERR_UNSUPPORTED for other dtypes or d. */
typedef struct {
    int32_t n_heads;
    int32_t n_kv_heads;
    int32_t n_tokens;
    int32_t d;
    int32_t chunk;      /* tokens per chunk */
    int32_t k;          /* route slots per row */
    int32_t causal;     /* 1: key token u is visible to query token t iff u <= t */
    int32_t dtype;      /* rr_dtype of Q, K, V and O (RR_BF16) */
    float scale;        /* softmax scale; 0: 1/sqrt(d) */
    int32_t reserved;   /* must be 0 */
} rr_attn_config;

rr_status rr_sparse_attention(const rr_attn_config *cfg, const void *Q, const void *K, const void *V,
                              const int32_t *routes, void *O, void *hip_stream);

/* ------------------------------------------------------------------------
 * The paged cache: keys and values of a batch of sequences that grow a few
 * tokens at a time, and attention of their newest tokens.
 *
 * A cache is two pools K_cache and V_cache, [n_pages, n_kv_heads, page, d]
 * each: page p holds `page` consecutive tokens of one sequence (or of several
 * that begin alike).  Token u of sequence b lies in page page_table[b][u /
 * page] at place u % page; page_table is [n_seqs, max_pages] int32.  A page is
 * a chunk: rr_pool_chunks over a pool taken as [n_pages * n_kv_heads, page, d]
 * gives the representations of whole pages, and rr_full_route with n_q = 1
 * and the batch folded into the heads routes over them.
 *
 * lengths [n_seqs] int32 counts each sequence's tokens, those new in this
 * step included, for the append and for the attention after it.  Entries of
 * page_table outside [0, n_pages) hold no page: nothing is written there and
 * no query sees their tokens.  A length is meant to lie between 0 and
 * max_pages * page.  One outside is no fault: the attention takes the nearer
 * end, and its queries as the newest tokens up to there; the append takes it as
 * it is and leaves out the tokens without a place.  (So the queries of a
 * sequence that has outgrown its table are off by what it lacks.)  Sequences
 * may share pages that none of them writes.
 *
 * Types: dtype RR_BF16 with cache_dtype RR_BF16 or RR_E4M3, or RR_F32 with
 * RR_F32.  An RR_E4M3 cache holds x / scale of key head g, k_scale[g] for
 * keys and v_scale[g] for values ([n_kv_heads] binary32, positive), rounded
 * to nearest even, past the largest finite value (448) clamped to it.  The
 * scales are NULL for other caches.
 *
 * Pointers to vectors that the attention reads (Q, the pools) or writes (O)
 * and the workspace are 16-byte aligned (RR_ERR_INVALID otherwise).
 * ---------------------------------------------------------------------- */

typedef struct {
    int32_t n_heads;      /* of Q; not read where Q is NULL */
    int32_t n_kv_heads;
    int32_t d;            /* a multiple of 8, at most 1024 */
    int32_t page;         /* tokens a page */
    int32_t n_pages;      /* pages of each pool */
    int32_t max_pages;    /* page_table entries of a sequence */
    int32_t n_seqs;
    int32_t n_tokens;     /* new tokens, all sequences' (0: nothing to do), below 2^24 */
    int32_t rot;          /* leading features of a head that are rotated: even, 0 .. d */
    int32_t interleaved;  /* partners: 1: features 2j and 2j + 1; 0: j and j + rot / 2 */
    int32_t dtype;        /* of K, V, Q and Q_out */
    int32_t cache_dtype;
    int64_t ldq, ldk, ldv;  /* elements from one token's rows to the next one's, >= 0 (0: one token's rows for all) */
    const float *k_scale, *v_scale;
} rr_append_config;

/* Appends new tokens: K and V [n_tokens, n_kv_heads, d] go into the pools,
 * keys rotated by their positions; queries Q [n_tokens, n_heads, d] (or NULL)
 * get the same rotation into Q_out [n_tokens, n_heads, d], which may be Q
 * itself where ldq = n_heads * d and must not overlap it otherwise.  Tokens
 * are packed: those of sequence b are tokens seq_start[b] .. seq_start[b+1] - 1
 * ([n_seqs + 1] int32, ascending); NULL: n_tokens / n_seqs each.  The last one
 * of sequence b is token lengths[b] - 1 of the sequence.  Tokens outside
 * every sequence, and those that would lie before a sequence's first token
 * or past its page table, are left out: their rows of Q_out keep what they
 * held.  Position p turns partners (x, y) into (x cos a - y sin a, y cos a +
 * x sin a), a = p * freqs[j], freqs [rot / 2] binary64 radians; angles are
 * reduced in binary64, the rotation is computed in binary32 and rounded
 * once.  Two new tokens must not lie in the same place.
 * Returns RR_ERR_INVALID for bad sizes, types or NULL pointers,
 * RR_ERR_UNSUPPORTED for 2^24 tokens or more, or for more than 2^30 elements of
 * keys and queries in a token. */
rr_status rr_cache_append(const rr_append_config *cfg, const void *K, const void *V, const void *Q,
                          const int32_t *seq_start, const int32_t *lengths, const int32_t *page_table,
                          const double *freqs, void *K_cache, void *V_cache, void *Q_out, void *hip_stream);

typedef struct {
    int32_t n_heads;
    int32_t n_kv_heads;
    int32_t d;           /* 64, 128, or 256 for bf16 */
    int32_t page;
    int32_t n_pages;
    int32_t max_pages;
    int32_t n_seqs;
    int32_t n_q;         /* query tokens of each sequence: its newest */
    int32_t k;           /* route slots (0: no routes) */
    int32_t n_sink;      /* first pages ... */
    int32_t n_recent;    /* ... and last pages that every query sees besides its routes */
    int32_t n_prefix;    /* rr_prefix_attention: tokens that all sequences begin with (otherwise 0) */
    int32_t dtype;       /* of Q and O */
    int32_t cache_dtype;
    float scale;         /* softmax scale; 0: 1/sqrt(d) */
    int32_t reserved;    /* must be 0 */
    const float *k_scale, *v_scale;
} rr_paged_config;

/* Bytes of workspace that rr_paged_attention and rr_prefix_attention need for
 * a config (0: the config is not valid, see rr_last_error).  A workspace is
 * filled with zeros before its first use; calls leave the part of it that has
 * to be zero (the first 2048 bytes) at zero, so it serves any calls that follow
 * one another.  Calls that may run at the same time need one each. */
size_t rr_paged_workspace_bytes(const rr_paged_config *cfg);

/* Attention of the newest n_q tokens of every sequence over its cache (Sec.
 * 2.2 Eq. (3) where a token is all that is new): query t of Q [n_seqs, n_q,
 * n_heads, d] stands at position p = lengths[b] - n_q + t of sequence b and
 * attends, with one softmax scaled by `scale`, to the sequence's tokens u <= p;
 * query head h reads key head h / (n_heads / n_kv_heads).  A query that sees
 * no token (p < 0), or whose scores are all -INFINITY, gets a zero output.
 *   routes  [n_seqs * n_heads * n_q, k] int32 (row (b * n_heads + h) * n_q + t)
 *           page indices within the sequence: the query sees the tokens u <= p
 *           of those pages, of its first n_sink and of the n_recent up to the
 *           one that holds p, each once; other slots (-1, or a page that begins
 *           after p) are skipped.  NULL with k = 0: its first n_sink and last
 *           n_recent pages alone; every token where these are 0 too.
 *           k + n_sink + n_recent <= 256.
 *   O       [n_seqs, n_q, n_heads, d] of dtype.
 *   lse     optional [n_seqs, n_q, n_heads] binary32: the logarithm of the sum
 *           of exp(scaled score), -INFINITY where no token is seen.
 * Scores, softmax and sums in binary32.  With bf16 queries the softmax weights
 * enter the value product as the sum of two bf16 numbers (2^-16 off) where at
 * most 64 query rows are multiplied with a key head's tokens together (n_q *
 * n_heads / n_kv_heads of a sequence, n_seqs times that behind a shared prefix),
 * rounded to bf16 (2^-8 off) at worst where more are.  Tokens that a
 * query does not see have no part in its output, whatever their rows hold;
 * where it sees a value that is not finite, that feature of its output is
 * infinite or NaN, however low the score.
 * Returns RR_ERR_INVALID for bad sizes, NULL or unaligned pointers or a
 * workspace too small, RR_ERR_UNSUPPORTED for other types or d, for 2^31
 * query rows (n_seqs * n_q * n_heads; 2^24 with a prefix) or more, or where
 * 1 + max_pages * page / 128 times n_seqs, n_kv_heads and the tiles of (16 to
 * 128) rows of a key head comes near 2^31. */
rr_status rr_paged_attention(const rr_paged_config *cfg, const void *Q, const void *K_cache, const void *V_cache,
                             const int32_t *page_table, const int32_t *lengths, const int32_t *routes, void *O,
                             float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

/* The same without routes for sequences whose first n_prefix tokens are the
 * same: prefix_pages [ceil(n_prefix / page)] int32 holds their pages (in the
 * last one the first n_prefix % page places, if any), which are read once for
 * up to 128 query rows of the batch on a key head (binary32: 32) in place of
 * once a sequence; page_table serves the tokens from n_prefix on (its
 * earlier entries are not read, n_prefix may lie inside a page). */
rr_status rr_prefix_attention(const rr_paged_config *cfg, const void *Q, const void *K_cache, const void *V_cache,
                              const int32_t *page_table, const int32_t *lengths, const int32_t *prefix_pages, void *O,
                              float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* ROUTERELAY_H */
