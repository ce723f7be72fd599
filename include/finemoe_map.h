/*
 * finemoe_map.h - C ABI of the expert-map matching and prefetch-selection
 * library for AMD Instinct MI355X (gfx950).
 *
 * The library implements the per-iteration search of FineMoE (arXiv
 * 2502.05370): a batch of queries is scored by cosine similarity against a
 * GPU-resident store of historical iterations, the best stored iteration(s)
 * are kept per query, and the matched expert map is turned into per-layer
 * expert prefetch sets by probability thresholding.
 *
 *   expert map (Section 4.1)      L rows of E gate probabilities, one row per
 *                                 MoE layer (the paper's J experts are E here)
 *   semantic search (Eq. 4)       cosine of embedding-layer outputs
 *   trajectory search (Eq. 5)     cosine of the first p observed layers of
 *                                 gate probabilities, flattened
 *   threshold (Section 4.3)       fixed tau, or delta = Clip(1 - score, 0, 1)
 *   prefetch set (Eq. 6-8)        fewest experts, highest probability first,
 *                                 whose summed probability reaches the
 *                                 threshold, clamped to [k_min, k_max]
 *
 * Conventions shared by every call:
 *   - All pointers marked "device" are HIP device pointers owned by the
 *     caller; the library never allocates device memory and never frees a
 *     caller buffer.  A store handle only borrows its buffer.
 *   - Work is enqueued asynchronously on the given stream (a hipStream_t
 *     passed as void*; NULL means the null stream).  Outputs are valid once
 *     the caller has synchronised that stream.  No call synchronises the
 *     stream except fm_store_check.
 *   - Arguments are validated on the host before anything is enqueued; an
 *     invalid call returns a non-zero fm_status, enqueues nothing and leaves
 *     every output untouched.  fm_last_error() then describes the problem
 *     (thread-local, valid until the next call on the same thread).
 *   - Ranking order is (score descending, store index ascending); a NaN
 *     score ranks below every number.  Missing matches (an empty store, or
 *     k larger than the store) are returned as index -1 and score -inf, and
 *     select nothing.
 *   - bf16 values are IEEE-754 binary32 values truncated to their upper 16
 *     bits (as produced by round-to-nearest-even), stored as uint16.
 */
#ifndef FINEMOE_MAP_H
#define FINEMOE_MAP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FM_OK = 0,
    FM_ERR_INVALID = 1,      /* bad argument: NULL pointer, out-of-range size or parameter */
    FM_ERR_UNSUPPORTED = 2,  /* valid but not implemented (e.g. E > 64, d_emb not a multiple of 128) */
    FM_ERR_FULL = 3,         /* insert would exceed the store capacity */
    FM_ERR_HIP = 4,          /* a HIP runtime call failed (message from the runtime) */
    FM_ERR_DEVICE = 5        /* fm_store_check found a sticky device-side range error */
} fm_status;

/* The argument enums below end in a 32-bit sentinel so that any int a caller
 * passes is a value of the type, which the library then checks and rejects
 * if it is not one of the listed ones (FM_ERR_INVALID); the sentinels are not
 * valid arguments. */
typedef enum { FM_F32 = 0, FM_BF16 = 1, FM_DTYPE_ENUM_INT32_ = 0x7fffffff } fm_dtype;

/* Threshold of Section 4.3: FIXED uses params.tau for every layer; DYNAMIC
 * uses delta = Clip(1 - score, 0, 1) with the best match's score (a NaN score
 * gives delta = 1). */
typedef enum { FM_TAU_FIXED = 0, FM_TAU_DYNAMIC = 1, FM_TAU_ENUM_INT32_ = 0x7fffffff } fm_tau_mode;

/* Which probabilities guide a layer: NONE = the layer's row of the best match
 * (Sections 4.2.1 and 4.2.2 use the single highest-scoring map); SCORE = the
 * similarity-weighted mean of that row over the k kept matches, with weights
 * max(score, 0) (plain mean if every weight is 0). */
typedef enum { FM_BLEND_NONE = 0, FM_BLEND_SCORE = 1, FM_BLEND_ENUM_INT32_ = 0x7fffffff } fm_blend;

/* Which Section 4.5 priority fm_priority_order ranks by. */
typedef enum { FM_PRI_PREFETCH = 0, FM_PRI_EVICT = 1, FM_PRI_ENUM_INT32_ = 0x7fffffff } fm_pri_kind;

/* Sticky device-side flags reported by fm_store_check. */
#define FM_FLAG_DEPTH_CLAMPED 0x1u   /* a trajectory depth was outside [1, max_depth] and was clamped */
#define FM_FLAG_INDEX_RANGE   0x2u   /* fm_select_prefetch met an index >= the store size (row skipped); the model
                                        operators met a token, expert or slot past its range (left out) */
#define FM_FLAG_STATE_STALE   0x4u   /* fm_traj_step: the store size changed since layer 0, or layers out of order */
#define FM_FLAG_VALUE_RANGE   0x8u   /* a float32 map or trajectory-query value exceeds 8 in magnitude (gate
                                        probabilities lie in [0, 1]); float32 trajectory scores are then unspecified */
#define FM_FLAG_EXPERT_MISSING 0x10u /* fm_moe_experts: an expert that a token takes is in no slot (left out) */
#define FM_FLAG_PAGES_FULL     0x20u /* fm_kv_resize: a slot's tokens found no page or passed its table (not added) */
#define FM_FLAG_PAGE_SHARED    0x40u /* fm_kv_write: a token lies in a page that several slots hold (not written) */

typedef struct fm_store fm_store;   /* opaque host-side handle */

typedef struct {
    int32_t cap;         /* capacity C in stored iterations, >= 1 */
    int32_t L;           /* MoE layers, 1..64 */
    int32_t E;           /* experts per layer, 1..64 (a prefetch set is a 64-bit mask) */
    int32_t d_emb;       /* semantic embedding size (hidden size h); 0 = no embeddings,
                            otherwise a positive multiple of 128 */
    fm_dtype map_dtype;  /* element type of stored maps and trajectory queries */
    void* buffer;        /* device, at least fm_store_bytes(...) bytes, 256-byte aligned */
    size_t buffer_bytes;
} fm_store_desc;

typedef struct {
    fm_tau_mode mode;
    float tau;           /* FIXED threshold; compared as the exact float value */
    int32_t k_min;       /* Eq. 8 floor (the model's K), 0 <= k_min <= k_max */
    int32_t k_max;       /* cap on the set size, k_max <= E */
    fm_blend blend;
} fm_select_params;

/* Bytes of the layer-major map planes alone: L planes of cap (rounded up to
 * 16) rows of E elements rounded up to a multiple of 4 (the padding is stored
 * as zeros), each plane padded to 256 bytes.  Inside a plane the maps are
 * stored in tiles of 16: for every quad of 4 consecutive experts, the tile's
 * 16 rows of that quad are contiguous.  For cap = 32768 maps of 24 x 60
 * float32 (Section 6.8's largest store, Qwen1.5-MoE shape) this is
 * 188,743,680 bytes. */
size_t fm_map_bytes(int32_t cap, int32_t L, int32_t E, fm_dtype map_dtype);

/* Bytes of the whole device buffer a store needs: map planes, the prefix
 * inverse norms 1/|x[y][0:l+1]| of every map at every depth (L x cap float32,
 * cap rounded up to 64, computed at insert time in float64), embeddings
 * (cap x d_emb bf16), their float32 norms and 256 bytes of device flags, each
 * part 256-byte aligned.  Returns 0 for invalid sizes. */
size_t fm_store_bytes(int32_t cap, int32_t L, int32_t E, int32_t d_emb, fm_dtype map_dtype);

/* Bytes of match workspace for a store of L layers of E experts (map_dtype)
 * and d_emb embedding dimensions (0 or a multiple of 128), serving batches of
 * up to B_max queries keeping up to k_max matches each (device memory,
 * 256-byte aligned, owned by the caller).  It holds the staged queries of one
 * launch (depth-sorted trajectory planes, or tiled semantic embeddings), the
 * query norms, ranking floors and the per-workgroup partial top-k lists.  Every match call
 * rewrites what it reads, so the contents need no initialisation.  Calls that
 * share a workspace must be ordered (same stream, or synchronised); concurrent
 * calls on one workspace race.  Returns 0 for invalid arguments. */
size_t fm_workspace_bytes(int32_t L, int32_t E, int32_t d_emb, fm_dtype map_dtype, int32_t B_max,
                          int32_t k_max);

/* Create a host handle over a caller-owned device buffer (Expert Map Store,
 * Section 4.4).  The store starts empty.  The buffer contents are not read;
 * the current HIP device at this call is the store's device.  Errors:
 * FM_ERR_INVALID for NULL pointers, out-of-range sizes or a short or
 * misaligned buffer; FM_ERR_UNSUPPORTED for E or L above 64, a d_emb that is
 * not a multiple of 128, or map planes so large that one group of layer
 * planes scanned together (32/E planes when E in {8, 16, 32}, else one)
 * exceeds 0xF0000000 bytes (e.g. cap above ~15.7 million maps of 64 float32
 * experts). */
fm_status fm_store_build(fm_store** out, const fm_store_desc* desc);

/* Append n iterations (Step 5 of Section 3.2: new expert maps enter the
 * store).  maps: device [n][L][E] of map_dtype, map-major; embs: device
 * [n][d_emb] bf16, 16-byte aligned, required when d_emb > 0 and ignored
 * otherwise.  The maps
 * are transposed into the layer-major planes, and their prefix norms and the
 * embedding norms are computed.  slots_out: device [n] int32 receiving the store index of each
 * inserted iteration, or NULL.  FM_ERR_FULL if size + n > cap (nothing is
 * inserted).  n == 0 is a no-op. */
fm_status fm_store_insert(fm_store* store, const void* maps, const void* embs, int32_t n,
                          int32_t* slots_out, void* stream);

/* Bytes of scratch (device memory owned by the caller, 256-byte aligned)
 * that fm_store_insert_dedup needs for batches of up to n_max new iterations
 * on a store of capacity cap: two dense float32 matrices of n_max x cap
 * scores plus 72 KB of index arrays.  Returns 0 unless cap >= 1 and
 * 1 <= n_max <= 1024. */
size_t fm_dedup_scratch_bytes(int32_t cap, int32_t n_max);

/* Insert with deduplication (Section 4.4, Expert map deduplication).  maps,
 * embs and slots_out as for fm_store_insert, 1 <= n <= 1024 (n == 0 is a
 * no-op).  While the store has room, new iterations are appended in batch
 * order.  The rest replace stored iterations: for each such new iteration x
 * the redundancy score against every iteration y stored before this call is
 *     RDY[x][y] = (d/L) score_sem[x][y] + ((L-d)/L) score_traj[x][y]
 * with d = prefetch_distance (0..L), score_sem the Eq. 4 cosine of the
 * embeddings and score_traj the Eq. 5 cosine over all L layers, both as the
 * match calls compute them (float32), weighted in float64 and rounded to
 * float32; a term with weight 0 is not computed.  In batch order, each x
 * overwrites the y with the highest RDY (lower index on equal values, NaN
 * last) that no earlier x of this call took; an x left without a candidate
 * (a store of fewer than n entries) is dropped and gets slot -1.  The
 * store size becomes min(size + n, cap).
 * workspace: as for the match calls, sized with B_max >= n.  scratch: at least
 * fm_dedup_scratch_bytes(cap, n) bytes, rewritten by the call.  Calls sharing
 * a workspace or scratch must be ordered.
 * Errors: FM_ERR_INVALID for NULL or misaligned pointers, n or d out of
 * range, d > 0 on a store without embeddings, or a short workspace or
 * scratch; nothing is enqueued then. */
fm_status fm_store_insert_dedup(fm_store* store, const void* maps, const void* embs, int32_t n,
                                int32_t prefetch_distance, int32_t* slots_out, void* workspace,
                                size_t workspace_bytes, void* scratch, size_t scratch_bytes, void* stream);

/* Current number of stored iterations (host-side count, no synchronisation). */
fm_status fm_store_size(const fm_store* store, int32_t* n_out);

/* Synchronise the stream, read and clear the sticky device flags
 * (FM_FLAG_*).  Returns FM_ERR_DEVICE when any flag was set; *flags_out (may
 * be NULL) receives them. */
fm_status fm_store_check(fm_store* store, void* stream, uint32_t* flags_out);

/* Release the host handle (the caller's buffer is untouched). */
fm_status fm_store_destroy(fm_store* store);

/* Semantic search, Eq. 4: for each query embedding q[b] (device [B][d_emb]
 * bf16, 16-byte aligned) the k stored iterations with the highest cosine
 * q[b].x[y] / (|q[b]| |x[y]|) over y < size, accumulated in float32.  A zero
 * norm gives score 0.  Outputs: idx_out device [B][k] int32, score_out device
 * [B][k] float32, in ranking order.  1 <= k <= 8, 1 <= B <= 65536.
 * FM_ERR_INVALID if the store has no embeddings, q is misaligned or the
 * workspace is too small. */
fm_status fm_match_semantic(const fm_store* store, const void* q, int32_t B, int32_t k,
                            int32_t* idx_out, float* score_out,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Trajectory search, Eq. 5: query b observed its first p_b = depth[b] layers
 * (device [B] int32); q is device [B][L][E] of map_dtype, map-major, and rows
 * l >= p_b are never read.  Score = cosine between q[b][0:p_b] and
 * x[y][0:p_b], both flattened over (layer, expert), accumulated in float32.
 * max_depth (1..L) is a host-side bound on the depths that sizes the scan;
 * a depth outside [1, max_depth] is clamped and sets FM_FLAG_DEPTH_CLAMPED.
 * Outputs and limits as for fm_match_semantic. */
fm_status fm_match_trajectory(const fm_store* store, const void* q, const int32_t* depth,
                              int32_t max_depth, int32_t B, int32_t k,
                              int32_t* idx_out, float* score_out,
                              void* workspace, size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * fm_match_trajectory without a workspace argument.  Its workspace is a
 * device array of the library of FM_NOALLOC_SCRATCH_BYTES, one per GPU,
 * which every GPU the call runs on holds until the process ends; its address
 * is looked up on the first call on each device.  The call allocates and
 * frees nothing.  Arguments, results, limits and errors as for
 * fm_match_trajectory, plus FM_ERR_UNSUPPORTED when a trajectory search of
 * the store's L x E needs more workspace than the array holds (no shape with
 * L, E <= 64 does) and FM_ERR_HIP when the array's address cannot be
 * obtained.  All calls on one GPU share the array: calls that overlap in time
 * on one GPU (other streams, or host threads without ordering) race, and
 * their results are unspecified.  Nothing in it needs to start at zero
 * (every call rewrites what it reads). */
#define FM_NOALLOC_SCRATCH_BYTES (40u << 20)
fm_status fm_match_trajectory_noalloc(const fm_store* store, const void* q, const int32_t* depth,
                                      int32_t max_depth, int32_t B, int32_t k, int32_t* idx_out,
                                      float* score_out, void* stream);

/* Prefetch sets, Section 4.3 (Eq. 6-8): for query b and every layer l in
 * [layer_begin[b], layer_end[b]) (device [B] int32 each, clamped to [0, L]),
 * take the guiding probabilities (fm_blend), the threshold (fm_tau_mode) from
 * score[b][0], order the experts by probability (descending, lower expert
 * index first on equal values), find the smallest k* whose running float64
 * sum of the first k* reaches the threshold (k* = E if none does) and keep
 * the first min(max(k*, k_min), k_max).  idx/score: device [B][k] as written
 * by a match call.  mask_out: device [B][L] uint64, bit j = expert j;
 * count_out: device [B][L] uint8.  Layers outside the range, and queries whose
 * idx[b][0] is -1, get mask 0 and count 0. */
fm_status fm_select_prefetch(const fm_store* store, const int32_t* idx, const float* score,
                             int32_t B, int32_t k, const int32_t* layer_begin,
                             const int32_t* layer_end, const fm_select_params* params,
                             uint64_t* mask_out, uint8_t* count_out, void* stream);

/* A match call and the selection of its rows in one call: the semantic
 * search of Section 4.2.1 (Eq. 4) or the trajectory search of Section 4.2.2
 * (Eq. 5), then the prefetch sets of Section 4.3 (Eq. 6-8) of every row of
 * the batch, with the merge of the search's per-workgroup lists and the
 * selection in one launch.  Arguments, results and errors as for
 * fm_match_semantic / fm_match_trajectory followed by fm_select_prefetch on
 * the same B rows with the same k: idx_out/score_out receive the matches
 * (device [B][k]), mask_out/count_out the sets (device [B][L]); layer_begin,
 * layer_end and params as for fm_select_prefetch.  The results are those of
 * the two separate calls. */
fm_status fm_match_semantic_select(const fm_store* store, const void* q, int32_t B, int32_t k,
                                   const int32_t* layer_begin, const int32_t* layer_end,
                                   const fm_select_params* params, int32_t* idx_out, float* score_out,
                                   uint64_t* mask_out, uint8_t* count_out, void* workspace,
                                   size_t workspace_bytes, void* stream);
fm_status fm_match_trajectory_select(const fm_store* store, const void* q, const int32_t* depth,
                                     int32_t max_depth, int32_t B, int32_t k, const int32_t* layer_begin,
                                     const int32_t* layer_end, const fm_select_params* params,
                                     int32_t* idx_out, float* score_out, uint64_t* mask_out,
                                     uint8_t* count_out, void* workspace, size_t workspace_bytes,
                                     void* stream);

/* Misses of prefetch sets (Section 3: R_{l,j} = 1 iff expert j of layer l is
 * activated and not cached).  q: device [B][L][E] of map_dtype, each query's
 * own gate probabilities (the experts its layers actually route to); the
 * activated experts of a row are its K highest (lower expert index first on
 * equal values, NaN last), the cached ones its prefetch set (masks: device
 * [B][L] uint64 as written by fm_select_prefetch).  miss_out: device [B][L]
 * uint8, the number of activated experts outside the set for layers in
 * [layer_begin[b], layer_end[b]) (clamped to [0, L]), 0 elsewhere.
 * 1 <= K <= E, 1 <= B <= 65536.  Errors: FM_ERR_INVALID for NULL pointers or
 * out-of-range arguments; nothing is enqueued then. */
fm_status fm_miss_count(const fm_store* store, const void* q, int32_t B, int32_t K, const uint64_t* masks,
                        const int32_t* layer_begin, const int32_t* layer_end, uint8_t* miss_out, void* stream);

/* Expert priorities of Section 4.5, one ordered list per query.
 * FM_PRI_PREFETCH: the candidates are the experts of query b's prefetch set
 * (masks: device [B][L] uint64 as written by fm_select_prefetch) in the
 * layers after its current layer, l > l_now[b] (l_now: device [B] int32,
 * 0-based; -1 lists every layer); PRI = p_{l,j} / (l - l_now[b]).
 * FM_PRI_EVICT: the candidates are the cached experts (masks: device [L]
 * uint64, bit j of layer l = expert cached, one mask for all queries);
 * PRI = 1 / (p_{l,j} * freq[l][j]) with freq device [L][E] float32 visit
 * counts (p * freq = 0 gives +inf).  p_{l,j} is the query's guiding
 * probability, exactly as fm_select_prefetch computes it from idx/score/blend.
 * PRI is computed in float64 and rounded to float32.  Each query's
 * candidates are ordered by PRI descending, the lower l * E + j first on
 * equal values, NaN last; the first cap are written: order_out device
 * [B][cap] int32 (l * E + j, -1 past the candidates), pri_out device [B][cap]
 * float32 (-inf past the candidates); count_out device [B] int32 receives
 * the number of candidates.  A query whose idx[b][0] is -1 has none (an
 * index >= the store size also sets FM_FLAG_INDEX_RANGE).  1 <= k <= 8,
 * 1 <= B <= 65536, 1 <= cap <= 4096.  Errors: FM_ERR_INVALID for NULL
 * pointers (l_now for PREFETCH, freq for EVICT) or out-of-range arguments;
 * nothing is enqueued then. */
fm_status fm_priority_order(const fm_store* store, const int32_t* idx, const float* score, int32_t B, int32_t k,
                            fm_blend blend, fm_pri_kind kind, const uint64_t* masks, const int32_t* l_now,
                            const float* freq, int32_t cap, int32_t* order_out, float* pri_out,
                            int32_t* count_out, void* stream);

/* Bytes of state (device memory owned by the caller, 256-byte aligned) for
 * fm_traj_step passes of up to B_max queries (1..65536) on a store of
 * capacity cap: per group of 64 queries a 1,280-byte header (store size at
 * layer 0, last layer, float64 running query sums of squares in two slots)
 * and the running float32 dot products of each query with each stored map
 * (cap rounded up to 16, 4 query tiles of 16): 1,280 + 1,024 * ceil(cap / 16)
 * * 4 bytes per group, each group 256-byte aligned.
 * 0 for invalid arguments. */
size_t fm_traj_state_bytes(int32_t cap, int32_t B_max);

/* Incremental trajectory re-search (Section 4.2.2: after each newly observed
 * layer the trajectory search runs again with the prefix grown by one layer).
 * q_layer: device [B][E] of map_dtype, each query's gate probabilities at
 * layer `layer` (0-based).  layer == 0 starts a pass and overwrites the
 * state; every later call of the pass passes the next layer for the same B
 * queries, in the same order, on an unchanged store.  The state keeps the
 * running dot product of every (query, stored map) pair, so a step reads one
 * layer plane of the store instead of layer + 1.  Outputs as for
 * fm_match_trajectory with depth[b] = layer + 1 for every b (Eq. 5 over the
 * first layer + 1 layers, float32 accumulation, rows of the store beyond its
 * size at the call never ranked).  A step whose store size differs from the
 * size at layer 0, or whose layer does not follow the previous one, sets
 * FM_FLAG_STATE_STALE and its results are unspecified.  1 <= k <= 8,
 * 1 <= B <= 65536, 0 <= layer < L.  Errors: FM_ERR_INVALID for NULL or
 * misaligned pointers, out-of-range arguments, or a short state or
 * workspace; nothing is enqueued then. */
fm_status fm_traj_step(fm_store* store, void* state, size_t state_bytes, const void* q_layer, int32_t layer,
                       int32_t B, int32_t k, int32_t* idx_out, float* score_out, void* workspace,
                       size_t workspace_bytes, void* stream);

/* ---- Model operators around the search -------------------------------
 *
 * What the search works on and for: token embeddings (the semantic queries of
 * Section 4.2.1), the gate of an MoE layer (a row of an expert map and of a
 * trajectory query, Sections 4.1 and 4.2.2), and the chosen experts' products
 * on experts that a cache holds (the prefetched ones of Section 4.3).  They
 * take no store: work is enqueued on the current device, which must hold every
 * buffer; T <= 2^24 tokens, B <= 65536 requests, d <= 16384.  flags, where a call takes it, is a device uint32 that collects
 * sticky FM_FLAG_* bits, or NULL.  Sizes of zero tokens or requests are
 * no-ops.  All sums are float32; bf16 inputs are widened exactly and results
 * rounded once, to nearest even.  Results do not depend on timing: the same
 * inputs give the same bits. */

/* Embedding lookup: out[t] = scale * table[tokens[t]].  table: device [V][d]
 * of dtype; tokens: device [T] int32; out: device [T][d] of dtype, apart from
 * the table.  A negative token is padding and gives a row of zeros, and so
 * does a token >= V, which also sets FM_FLAG_INDEX_RANGE.  Pointers are
 * aligned to their elements. */
fm_status fm_embed_lookup(const void* table, int32_t V, int32_t d, fm_dtype dtype, const int32_t* tokens, int32_t T,
                          float scale, void* out, uint32_t* flags, void* stream);

/* Mean embedding of each request, the query form of fm_match_semantic:
 * out[b] = scale * mean of table[tokens[t]] over the tokens of request b that
 * select a row, offsets[b] <= t < offsets[b + 1] (padding and tokens >= V are
 * left out of the sum and of the count); a request without any gives zeros.
 * offsets: device [B + 1] int32, clamped to [0, T] (an end before its start
 * is an empty request); tokens: device [T]; out: device [B][d] bf16.
 * Otherwise as fm_embed_lookup. */
fm_status fm_embed_pool(const void* table, int32_t V, int32_t d, fm_dtype dtype, const int32_t* tokens, int32_t T,
                        const int32_t* offsets, int32_t B, float scale, void* out, uint32_t* flags, void* stream);

/* Bytes of scratch (device memory owned by the caller, 256-byte aligned) for
 * fm_embed_grad calls of up to T_max tokens on a table of V rows: two int32
 * per row, one per token, and the list of frequent tokens.  Returns 0 unless
 * 1 <= V <= 2^24 and 0 <= T_max <= 2^24. */
size_t fm_embed_grad_scratch_bytes(int32_t T_max, int32_t V);

/* Gradient of fm_embed_lookup with respect to the table:
 * dtable[v] = scale * sum of dout[t] over tokens[t] == v, summed in float32 in
 * an order fixed by the tokens.  dout: device [T][d] of dtype; dtable: device
 * [V][d] of grad_dtype.  accumulate == 0 writes every row (zeros where no
 * token selects it); otherwise the sum is added to the rows that tokens
 * select and no other row is touched.  Padding and tokens >= V contribute
 * nothing.  The positions of a row that more than 32 tokens select are found by
 * reading all tokens, once per 128 or 256 of its columns, so that the time of
 * long batches grows with their length times the number of such rows (fast up
 * to some 10^5 tokens: 65,536 over 128,000 rows of 2,048 bf16 0.21 ms, 1,048,576
 * 13 ms).  T == 0 with accumulate == 0 writes zeros.  scratch: at least
 * fm_embed_grad_scratch_bytes(T, V) bytes, rewritten by the call. */
fm_status fm_embed_grad(const void* dout, fm_dtype dtype, const int32_t* tokens, int32_t T, int32_t V, int32_t d,
                        float scale, int32_t accumulate, void* dtable, fm_dtype grad_dtype, void* scratch,
                        size_t scratch_bytes, uint32_t* flags, void* stream);

/* The gate of one MoE layer: logits l[t][e] = x[t] . gate[e], probabilities
 * p = softmax over e (float32), and each token's K experts with the largest
 * logits (lower index first on equal logits, NaN last).  x: device [T][d],
 * gate: device [E][d], both of dtype and 16-byte aligned, d a multiple of 8;
 * active: device [T] uint8 or NULL: a token with 0 has no request (its
 * probabilities and weights are 0, its experts -1, its mask 0).
 * probs_out: row t at probs_out + t * probs_stride elements of probs_dtype
 * (probs_stride >= E), so that a layer's probabilities land in the rows
 * [t][layer] of a batch of maps or trajectory queries; ids_out: device [T][K]
 * int32, by falling logit; weight_out: device [T][K] float32, the chosen
 * probabilities, divided by their sum if renorm != 0; mask_out: device [T]
 * uint64 (bit e = expert e chosen, as the masks of fm_select_prefetch) or
 * NULL.  1 <= E <= 64, 1 <= K <= min(8, E). */
fm_status fm_moe_route(const void* x, const void* gate, fm_dtype dtype, int32_t T, int32_t d, int32_t E, int32_t K,
                       int32_t renorm, const uint8_t* active, void* probs_out, fm_dtype probs_dtype,
                       int64_t probs_stride, int32_t* ids_out, float* weight_out, uint64_t* mask_out, void* stream);

/* A layer's experts as an expert cache holds them.  slots: device
 * [n_slots][3 d f] of dtype, 16-byte aligned; a slot is one expert's weights
 * as one block, so that loading it is one copy: the gate projection [f][d],
 * the up projection [f][d], the down projection [d][f].  slot_of: device [E]
 * int32, the slot of each expert (-1: in no slot). */
typedef struct {
    int32_t E;           /* experts of the layer, 1..64 */
    int32_t n_slots;     /* >= 1 */
    int32_t d;           /* hidden size, a positive multiple of 8 */
    int32_t f;           /* expert width, a positive multiple of 8, up to 65536 */
    fm_dtype dtype;      /* of the weights, inputs and outputs */
    const void* slots;
    const int32_t* slot_of;
} fm_expert_cache;

/* Bytes of workspace (device memory owned by the caller, 256-byte aligned)
 * for fm_moe_experts calls of up to T_max tokens of K experts each: the
 * activated products of one pass over the experts and its partial sums.  Above
 * 128 tokens it does not depend on T_max.
 * Returns 0 for sizes that fm_moe_experts refuses or T_max < 1. */
size_t fm_moe_workspace_bytes(int32_t d, int32_t f, fm_dtype dtype, int32_t T_max, int32_t K);

/* The chosen experts' products of one MoE layer:
 *   out[t] = residual[t] + sum over k of
 *            weight[t][k] * Down_e (silu(Gate_e x[t]) * (Up_e x[t])),  e = ids[t][k],
 * silu(z) = z / (1 + exp(-z)).  x, residual (or NULL: zeros) and out: device
 * [T][d] of the cache's dtype, 16-byte aligned; out may be x or residual
 * (not overlap them otherwise); ids: device [T][K] int32, weight: device [T][K] float32, as written by
 * fm_moe_route.  An expert of -1 contributes nothing; an expert that is in no
 * slot contributes nothing and sets FM_FLAG_EXPERT_MISSING; experts >= E and
 * slots >= n_slots contribute nothing and set FM_FLAG_INDEX_RANGE.  An expert
 * that a token lists twice counts with the sum of its weights.  An expert
 * that every token takes (a shared expert of m times the width) is m experts
 * in every token's list.  Up to 128 tokens (a decode iteration) an expert's
 * weights are read once per 64 of its tokens; longer batches (prompts) take
 * passes of up to 4,096 tokens, or of as many as 256 MB hold of K max(d, f)
 * float32 values.  1 <= K <= 8.  Infinities and NaN follow the formula.  The
 * weights of one slot must not exceed 0xF0000000 bytes.  workspace: at least
 * fm_moe_workspace_bytes(d, f, dtype, T, K) bytes, rewritten by the call;
 * calls sharing one must be ordered. */
fm_status fm_moe_experts(const fm_expert_cache* cache, const void* x, const int32_t* ids, const float* weight,
                         int32_t T, int32_t K, const void* residual, void* out, uint32_t* flags, void* workspace,
                         size_t workspace_bytes, void* stream);

/* ---- Attention of one new token over a paged cache --------------------
 *
 * The other half of a serving iteration's layer: keys and values of a batch's
 * requests in pages, and each request's new token attending to its own.  Under
 * the conventions of the model operators above: the current device must hold
 * every buffer, flags is a device uint32 or NULL, sums are float32, results do
 * not depend on timing.
 *
 * A cache serves n_slots requests (batch slots).  Slot s holds length[s]
 * tokens; token t lies in page table[s][t / page], at place t % page.  A page
 * holds `page` tokens of all layers and heads as one block, so that copying or
 * moving it is one copy.  Several slots may hold the same page (after
 * fm_kv_fork): refs[p] counts them, and a page with refs[p] == 0 is free.  A
 * caller starts with length and refs of zeros and a table of -1, and may fill
 * or restore the arrays itself as long as they agree; pages need no
 * initialisation.  Table entries from a slot's last page on are -1.
 *
 * Layout of a page: [layers][2: keys, values][heads][page / 16 blocks of 16
 * tokens], every block in pieces of 1 KB that hold 64 bytes of each of its
 * tokens' rows (head_dim is padded with zeros to such a multiple): 32 bf16 or
 * 16 float32 values.  With n = 16 / sizeof(element) and lane = 0..63, a piece p
 * of keys holds at 16-byte place `lane` the dimensions 4 n p + n (lane / 16) ..
 * + n - 1 of token lane % 16; a piece of values holds there, for i = 0 ..
 * n / 4 - 1 and j = 0..3, dimension 4 n p + 16 i + lane % 16 of token
 * 4 (lane / 16) + j at element 4 i + j.
 *
 * Calls that change a cache (fm_kv_resize, _fork, _compact, _copy, _write) must
 * be ordered with every other call on it; the others need no order among
 * themselves.  A page number outside [0, n_pages) in a visible place of a table
 * is never followed: its tokens are left out and FM_FLAG_INDEX_RANGE is set.
 * Lengths are taken as clamped to [0, max_pages * page]. */
typedef struct {
    int32_t n_slots;     /* requests, 1..65536 */
    int32_t max_pages;   /* pages of one slot, >= 1; max_pages * page <= 2^30, n_slots * max_pages <= 2^28 */
    int32_t n_pages;     /* pages of the pool, 1..2^24 */
    int32_t page;        /* tokens of a page, a multiple of 16 in 16..1024 */
    int32_t layers;      /* 1..1024 */
    int32_t heads;       /* key (and value) heads, 1..1024 */
    int32_t head_dim;    /* a multiple of 8 in 8..256 */
    fm_dtype dtype;      /* of keys and values, and of queries and outputs */
    void* pages;         /* device [n_pages][fm_kv_page_bytes(...)], 256-byte aligned */
    int32_t* table;      /* device [n_slots][max_pages] */
    int32_t* length;     /* device [n_slots] */
    int32_t* refs;       /* device [n_pages] */
} fm_kv_cache;

/* Bytes of one page (at most 2^31).  Returns 0 for sizes that the calls below refuse. */
size_t fm_kv_page_bytes(int32_t layers, int32_t heads, int32_t head_dim, int32_t page, fm_dtype dtype);

/* Bytes of scratch (device memory owned by the caller, 256-byte aligned,
 * rewritten by every call) for fm_kv_resize, _fork, _compact and _copy on a
 * cache of these sizes (its pointers are not looked at).  Returns 0 for sizes
 * that they refuse. */
size_t fm_kv_scratch_bytes(const fm_kv_cache* cache);

/* Tokens come and go: delta[s] > 0 makes room for that many tokens behind slot
 * s, delta[s] < 0 drops its last -delta[s] (all of them if it has fewer: any
 * request ends with -2^31), 0 leaves it alone.  delta: device [n_slots] int32.
 * Dropping comes first: pages without a token left are released (refs - 1).
 * Then slots grow in order of their numbers.  New pages are the free ones of
 * the lowest numbers (that are free after the drops); a partly filled last page
 * that other slots hold too is copied to a new page first, so that no token is
 * ever added to a shared page (slots that share one and grow in the same call
 * get a copy each, and the original is released if all of its holders do).
 * A slot whose pages do not fit any more is refused (its length, pages and the
 * free ones stay), and so is every later one that needs a page; one that would
 * pass max_pages is refused alone.  Refusals set FM_FLAG_PAGES_FULL.
 * granted_out: device [n_slots] uint8 or NULL: 1 where tokens were added, else
 * 0: the `active` of the calls that follow. */
fm_status fm_kv_resize(const fm_kv_cache* cache, const int32_t* delta, uint8_t* granted_out, uint32_t* flags,
                       void* scratch, size_t scratch_bytes, void* stream);

/* Slots go on from other slots: slot s becomes what slot parent[s] was before
 * the call, sharing its pages, and releases its own.  parent: device [n_slots]
 * int32; -1 (or s itself) leaves slot s alone; a parent >= n_slots does too and
 * sets FM_FLAG_INDEX_RANGE.  Any parents are fine: many of one, chains, cycles. */
fm_status fm_kv_fork(const fm_kv_cache* cache, const int32_t* parent, uint32_t* flags, void* scratch,
                     size_t scratch_bytes, void* stream);

/* Live pages to the front: of the n pages that are held, those numbered n and
 * above move to the free numbers below n, in order, and the tables follow, so
 * that the pool's upper part is free (for expert slots, say).  Entries that a
 * slot does not use are left as they are if they are -1.  live_out: device int32 or
 * NULL: n. */
fm_status fm_kv_compact(const fm_kv_cache* cache, int32_t* live_out, uint32_t* flags, void* scratch,
                        size_t scratch_bytes, void* stream);

/* Contents of page src[i] to page dst[i], i < n <= n_pages; tables and counts
 * stay.  src, dst: device [n] int32.  A pair is left out, and sets
 * FM_FLAG_INDEX_RANGE, if one of its pages is outside the pool, or its
 * destination occurs again among the sources or destinations. */
fm_status fm_kv_copy(const fm_kv_cache* cache, const int32_t* src, const int32_t* dst, int32_t n, uint32_t* flags,
                     void* scratch, size_t scratch_bytes, void* stream);

/* Keys and values of new tokens into their pages of one layer.  k, v: device
 * [T][heads][head_dim] of the cache's dtype, rows of k_stride and v_stride
 * elements (the parts of one projection's output, say), 16-byte aligned, strides
 * multiples of 16 bytes.  offsets NULL: T = n_slots, and row s is slot s's last token.  Otherwise
 * offsets: device [n_slots + 1] int32, clamped to [0, T], and rows offsets[s]
 * .. offsets[s + 1] - 1 are the last tokens of slot s (an end before its start:
 * none).  active: device [n_slots] uint8 or NULL; a slot with 0 writes nothing,
 * nor does one without a token (offsets NULL).  A slot with more rows than
 * tokens writes nothing and sets FM_FLAG_INDEX_RANGE; tokens in a page that
 * several slots hold are not written and set FM_FLAG_PAGE_SHARED. */
fm_status fm_kv_write(const fm_kv_cache* cache, int32_t layer, const void* k, int64_t k_stride, const void* v,
                      int64_t v_stride, const int32_t* offsets, int32_t T, const uint8_t* active, uint32_t* flags,
                      void* stream);

/* The reverse of fm_kv_write: the slots' last tokens out of their pages (to
 * store a prefix elsewhere, say).  Arguments as there; rows that it would not
 * write are not touched, tokens in shared pages are read. */
fm_status fm_kv_read(const fm_kv_cache* cache, int32_t layer, void* k, int64_t k_stride, void* v, int64_t v_stride,
                     const int32_t* offsets, int32_t T, const uint8_t* active, uint32_t* flags, void* stream);

/* Bytes of workspace (device memory owned by the caller, 256-byte aligned) for
 * fm_attn_decode calls with q_heads query heads on a cache of these sizes.  It
 * must be zero before its first call; every call leaves its first
 * FM_ATTN_TICKET_BYTES bytes zero (they count which parts of split sequences are
 * there) and needs no more.  Returns 0 for sizes that it refuses. */
#define FM_ATTN_TICKET_BYTES 2048
size_t fm_attn_workspace_bytes(const fm_kv_cache* cache, int32_t q_heads);

/* Attention of every slot's last token over the slot's tokens in one layer:
 *   out[s][h] = sum over j of p_j v_j / sum over j of p_j,   p_j = exp(scale q[s][h] . k_j),
 * j from max(0, first[s], length[s] - window if window > 0) up to length[s] - 1;
 * query head h reads key head h / (q_heads / heads).  q: device
 * [n_slots][q_heads][head_dim] of the cache's dtype, 16-byte aligned, rows of
 * q_stride elements (a multiple of 16 bytes); q_heads a multiple of heads, at
 * most 1024.  first: device [n_slots] int32 or NULL.  active: device
 * [n_slots] uint8 or NULL: a slot with 0 has no query.  out: device
 * [n_slots][q_heads][head_dim] of the cache's dtype, apart from q, 16-byte
 * aligned.  lse_out: device [n_slots][q_heads] float32 or NULL: log of the sum
 * of p_j, for joining with attention over other tokens.  A query that sees no
 * token, or only tokens whose score is minus infinity, gives zeros and -inf;
 * tokens outside the range have no part in the result, whatever their pages
 * hold; other infinities and NaN follow the formula, but that a score of plus
 * infinity gives a lse_out of NaN.  bf16 caches: p_j meets v_j as two bf16
 * (2^-15 relative, or 2^-133 where that is more).  p_j and their sums with v_j
 * are float32, relative to the largest score that a part of the tokens has: below
 * 2^-126 p_j is zero, and values of which a sum passes 3.4e38 give infinities or
 * NaN.  Calls sharing a workspace must be ordered. */
fm_status fm_attn_decode(const fm_kv_cache* cache, int32_t layer, const void* q, int64_t q_stride, int32_t q_heads,
                         float scale, int32_t window, const int32_t* first, const uint8_t* active, void* out,
                         float* lse_out, uint32_t* flags, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Norms around a block ----------------------------------------------
 *
 * A block's output y joins the residual stream x and the next block's input is
 * normed, in one pass:
 *   n[t] = y[t] * rsqrt(mean(y[t]^2) + eps) * post      (post NULL: n = y)
 *   r[t] = x[t] + scale * gate * n[t]                    (gate NULL: 1)
 *   h[t] = r[t] * rsqrt(mean(r[t]^2) + eps) * pre        (pre NULL: no h)
 * y NULL: r = x, the norm before a first block (post and gate NULL, r_out NULL).
 * gate is [d] (FM_GATE_CHANNEL), [T] (FM_GATE_TOKEN) or [T][d] (FM_GATE_EACH).
 * All of dtype, d a multiple of 8, [T][d] and [d] tensors 16-byte aligned; h
 * comes from r before its rounding.  r_out may be x or y, h_out may be y
 * (no other overlap).  eps >= 0. */
typedef enum {
    FM_GATE_NONE = 0, FM_GATE_CHANNEL = 1, FM_GATE_TOKEN = 2, FM_GATE_EACH = 3, FM_GATE_ENUM_INT32_ = 0x7fffffff
} fm_gate_kind;

fm_status fm_block_norm(const void* x, const void* y, const void* post, const void* gate, fm_gate_kind gate_kind,
                        float scale, const void* pre, float eps, int32_t T, int32_t d, fm_dtype dtype, void* r_out,
                        void* h_out, void* stream);

/* Bytes of scratch (device memory owned by the caller, 256-byte aligned,
 * rewritten by every call) for fm_block_norm_grad calls of up to T_max tokens.
 * Returns 0 for sizes that it refuses (T_max = 0 is fine). */
size_t fm_block_norm_scratch_bytes(int32_t T_max, int32_t d);

/* Gradient of fm_block_norm: dr is the gradient of r from elsewhere (NULL:
 * zeros), dh that of h (NULL exactly where pre is; one of the two is given).
 * x, y and the rest are the forward call's arguments.  dx, dy (NULL where y
 * is): device [T][d] of dtype; dpost, dpre, dgate of FM_GATE_CHANNEL: device
 * [d] float32, sums over the tokens in a fixed order, with accumulate != 0
 * added to what is there; dgate of FM_GATE_TOKEN: device [T] float32, of
 * FM_GATE_EACH [T][d] of dtype, both written.  A gradient is given exactly
 * where its input is.  dx may be dr, dy may be y or dh, dgate of FM_GATE_EACH
 * may be gate (no other overlap).  T == 0 with accumulate == 0 writes zeros to
 * the [d] gradients. */
fm_status fm_block_norm_grad(const void* dr, const void* dh, const void* x, const void* y, const void* post,
                             const void* gate, fm_gate_kind gate_kind, float scale, const void* pre, float eps,
                             int32_t T, int32_t d, fm_dtype dtype, int32_t accumulate, void* dx, void* dy,
                             float* dpost, void* dgate, float* dpre, void* scratch, size_t scratch_bytes,
                             void* stream);

/* Test support: the dense float32 score matrix of a trajectory (q, depth
 * non-NULL) or semantic (q_sem non-NULL) search, written to scores_out device
 * [B][size] with the arithmetic of the match calls (the same kernels, but for
 * semantic searches of a size that the match calls run on their split-k scan,
 * whose float32 sums are taken in another order).
 * Exactly one of q / q_sem must be non-NULL. */
fm_status fm_debug_scores(const fm_store* store, const void* q, const int32_t* depth,
                          int32_t max_depth, const void* q_sem, int32_t B, float* scores_out,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Test support: the scan kernel that a match call launches for a batch of B
 * queries keeping k matches (its first 1,024 queries, if there are more) on a
 * store of n iterations of L x E maps and d_emb-wide embeddings: a trajectory
 * search to max_depth >= 1, or a semantic search with max_depth = 0.  k = 0
 * names the dense form (fm_debug_scores).  A name, then for a kernel of several
 * shapes a space and the shape: "k_traj_scan", "k_traj_mm", "k_traj_split RxC"
 * (blocks of 16 maps by tiles of 16 queries), "k_sem_scan", "k_sem_mm Q"
 * (queries per group), "k_sem_split RxC"; "k_traj_scan floors" is k_traj_scan
 * with the ranking floors that a query group's workgroups share.  A constant
 * string; NULL for sizes that the match calls refuse.  Runs on the host,
 * without a GPU. */
const char* fm_debug_scan_name(int32_t L, int32_t E, int32_t d_emb, fm_dtype map_dtype, int32_t n,
                               int32_t max_depth, int32_t B, int32_t k);

/* Measurement support: start and stop are hipEvent_t handles (passed as
 * void*) created by the caller, or both NULL to switch this off.  While set,
 * every match call made on this thread records start on its stream right
 * before the launch of its scan kernel (k_traj_* or k_sem_*; k_traj_step
 * for fm_traj_step) and stop right after it, so the events bracket exactly
 * that kernel (for a batch of more than one launch, the last launch's).  The library does not own or
 * destroy the events.  FM_ERR_INVALID if exactly one of them is NULL. */
fm_status fm_debug_scan_events(void* start, void* stop);

/* Description of the last non-OK status on this thread ("" if none). */
const char* fm_last_error(void);

/* ABI version: (major << 16) | minor. */
int32_t fm_version(void);

#ifdef __cplusplus
}
#endif

#endif /* FINEMOE_MAP_H */
