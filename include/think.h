/*
 * think.h -- C ABI of the ThinK hot path (query-driven key-cache channel pruning)
 * for NVIDIA B200 (sm_100a).
 *
 * Problem statement (paper, Sec. 1 and Sec. 3.1): the key and value caches are
 * tensors K, V in R^{B x S x L x N x D} (batch, tokens, layers, heads, head
 * dimension).  Given a pruning ratio lambda, T = floor((1 - lambda) D) key
 * channels are kept per head (Sec. 3.1, Eq. 2); the channels are chosen by the
 * query-driven score of Sec. 3.2 evaluated with the last S_obs queries
 * ("Observation Window"); the most recent S_recent prompt tokens and all newly
 * decoded tokens keep all D key channels (Sec. 3.3).
 *
 * Call order:   thinK_cache_bytes -> thinK_create -> thinK_score_select -> thinK_compact
 *               (or thinK_prefill for both) -> { thinK_append -> thinK_decode_attn }* -> thinK_destroy
 *
 * Conventions that hold for every entry point
 *  - All tensor pointers are DEVICE pointers unless marked "host".  The caller
 *    allocates and owns every device buffer; the library never allocates device
 *    memory and never frees anything but its own host-side handle.
 *  - `stream` is a cudaStream_t passed as void*.  Calls enqueue work on it and
 *    return without synchronising.  Calls on one handle must be stream-ordered
 *    with respect to each other.
 *  - Errors are return codes.  Arguments are validated on the host before any
 *    launch; an invalid call launches nothing.  Inputs are assumed finite:
 *    NaN/Inf in K or Q sets a bit of the device error word and leaves the
 *    choice among the affected channels unspecified (never an out-of-range write).
 *  - Element type (`dtype`): bf16 or fp32 for K, V, Q, q, k_new, v_new and out.
 */
#ifndef THINK_H_
#define THINK_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  THINK_OK = 0,
  THINK_ERR_INVALID_ARG = 1, /* null / misaligned pointer, bad shape, bad layer range */
  THINK_ERR_UNSUPPORTED = 2, /* head dimension, group size or dtype without a kernel */
  THINK_ERR_STATE = 3,       /* call out of order */
  THINK_ERR_CAPACITY = 4,    /* tail full (max_new_tokens) or buffer too small */
  THINK_ERR_CUDA = 5         /* a CUDA runtime call or launch failed */
} thinK_status;

typedef enum { THINK_BF16 = 0, THINK_F32 = 1 } thinK_dtype;

/* Score used to rank the channels of a key head. */
typedef enum {
  THINK_SCORE_QUERY_DRIVEN = 0, /* Sec. 3.2: ||Q[-S_obs:, j] K[:, j]^T||_F                      */
  THINK_SCORE_KEY_L2 = 1,       /* Sec. 3.1, Eq. 1 with p = 2: ||K[:, j]||_2 (paper's baseline) */
  THINK_SCORE_KEY_L1 = 2        /* Sec. 3.1, Eq. 1 with p = 1: ||K[:, j]||_1                    */
} thinK_criterion;

/* Kernel behind the value-channel score of App. D (thinK_score_select_kv). */
typedef enum {
  THINK_VALUE_SCORE_AUTO = 0,     /* tcgen05.mma with accumulators in tensor memory where the shape allows it
                                     (blocks of 128 stacked window rows, D = 128), mma.sync elsewhere */
  THINK_VALUE_SCORE_MMA_SYNC = 1  /* the mma.sync kernel everywhere (same results within the stated tolerance) */
} thinK_value_score_kernel;

typedef struct {
  int32_t B;              /* batch entries */
  int32_t L;              /* layers held by this cache */
  int32_t N_q;            /* query heads; N_q % N_kv == 0, group size G = N_q / N_kv in {1,2,4,8} */
  int32_t N_kv;           /* key/value heads */
  int32_t D;              /* head dimension: 64 or 128 */
  int32_t S_max;          /* rows allocated along S in K and V (>= every seq_len) */
  int32_t S_obs;          /* observation window (Sec. 3.2); seq_len >= S_obs */
  int32_t S_recent;       /* prompt tokens left unpruned (Sec. 3.3, Sec. 4.3 "recent size") */
  int32_t max_new_tokens; /* decode steps the unpruned tail can take */
  int32_t dtype;          /* thinK_dtype */
  int32_t criterion;      /* thinK_criterion */
  int32_t value_score_kernel; /* thinK_value_score_kernel; only read when lambda_v > 0 */
  double lambda;          /* pruning ratio, 0 <= lambda < 1 */
  double lambda_v;        /* pruning ratio of the value channels (App. D); 0 = values untouched (the default path) */
} thinK_config;

/* A strided view of a B x S x L x N x D tensor.  Strides are in ELEMENTS; the D
 * axis is contiguous.  `ptr` and every stride must be multiples of 16 bytes.
 * The paper's layout is stride_b = S*L*N*D, stride_s = L*N*D, stride_l = N*D,
 * stride_n = D; a per-layer cache [B, N, S, D] is expressed by other strides. */
typedef struct {
  void* ptr;
  int64_t stride_b, stride_s, stride_l, stride_n;
} thinK_tensor5;

/* Byte sizes of the caller-allocated device buffers (each 256-byte aligned). */
typedef struct {
  size_t k_thin;    /* pruned prefix keys, library layout (below) */
  size_t tail_k;    /* unpruned keys: recent prompt rows + decoded tokens */
  size_t tail_v;    /* values of the same tokens, [B, L, N_kv, cap, D] */
  size_t idx;       /* kept channels, uint8 [B, L, N_kv, T], ascending */
  size_t scores;    /* channel scores, fp64 [B, L, N_kv, D] */
  size_t workspace; /* reduction partials, split-softmax states, counters */
  /* The paper's accounting of the same cache (Sec. 3.1, Sec. 3.3), in bytes:
   * keys of the pruned prefix at T channels + unpruned keys at D + all values,
   * with the tail at full capacity; and the unpruned cache 2*B*S*L*N*D*e with
   * the same number of tokens. */
  size_t model_think_bytes;
  size_t model_dense_bytes;
  /* Only with lambda_v > 0 (else 0): */
  size_t v_thin;    /* pruned prefix values, bf16 [rows of T_v kept channels padded to a multiple of 16] */
  size_t perm_v;    /* uint8 [B, L, N_kv, D]: kept value channels ascending, then the pruned ones ascending */
} thinK_sizes;

typedef struct thinK_cache thinK_cache; /* opaque, host side */

/* T = floor((1 - lambda) * D) (Sec. 3.1); returns 0 when lambda is outside
 * [0, 1) or T would be 0. */
int32_t thinK_T(double lambda, int32_t D);

const char* thinK_status_string(thinK_status s);

/* Sizes of the buffers thinK_create needs.  `seq_lens` (host, [B]) are the
 * prompt lengths S_b; S_recent <= S_b, S_obs <= S_b <= S_max.
 *
 * Library layout of k_thin and tail_k.  For every (b, l, h) the S_p = S_b - S_recent prefix tokens
 * are cut into tiles of 64 tokens; tile t of head (b, l, h) is tile number
 *   thin_tile_base(b) + (l*N_kv + h)*n_tiles(b) + t,   n_tiles(b) = ceil(S_p(b)/64),
 *   thin_tile_base(b) = sum_{b'<b} L*N_kv*n_tiles(b'),
 * and a tile holds Tp x 64 elements (tokens past S_p are zero).
 *  - fp32: Tp = T; channel-major [T][64], rows of 64 tokens whose 16-byte chunks are XOR-swizzled with
 *    (row & 7): element (token u, channel c) at c*64 + swz(c, u),
 *    swz(c, u) = (((u*4/16) ^ (c & 7)) * 16 + (u*4)%16) / 4.
 *  - bf16: Tp = T rounded up to a multiple of 8 (extra channels are zero); the tile is stored in the
 *    operand order of the tensor-core instruction that consumes it: four 16-token steps of Tp*32
 *    bytes; in a step, for each group s of 16 channels a 512-byte chunk with 16 bytes per lane i
 *    (r = i/4, q = i%4): for jx = 0,1 the channel pairs (16s+2q, +1) and (16s+2q+8, +9) of token
 *    16*step + 8*jx + r; a trailing group of 8 channels is a 256-byte block with 8 bytes per lane
 *    (pair (16*n16+2q, +1) for jx = 0,1).
 * tail_k uses the same tile layout with all D channels: [B, L, N_kv, ceil(cap/64)] tiles of D x 64,
 * cap = S_recent + max_new_tokens.
 * After the n_tiles(b) prompt tiles every head owns ceil(cap/64) more tiles in k_thin, which receive the
 * tail blocks that thinK_reprune_tail thins (so the tile number above uses n_tiles(b) + ceil(cap/64)
 * per head).
 * v_thin (lambda_v > 0): token-major rows of Tvp = T_v rounded up to 16 bf16 elements, row t of head
 * (b, l, h) at element v_base(b) + ((l*N_kv + h)*S_p(b) + t)*Tvp, v_base(b) = sum_{b'<b} L*N_kv*S_p(b')*Tvp;
 * element c < T_v of a row is channel perm_v[b][l][h][c] of the value, the padding is zero.  With
 * lambda_v > 0 the rows of tail_v are stored in the channel order perm_v[b][l][h][0..D). */
thinK_status thinK_cache_bytes(const thinK_config* cfg, const int32_t* seq_lens, thinK_sizes* out);

/* Builds the host-side handle and writes the small device tables (lengths,
 * tile offsets, zeroed counters) into `workspace` with synchronous copies.
 * `sizes` (host) states the bytes the caller actually allocated for each buffer
 * (v_thin and perm_v: for the later thinK_attach_value_cache); a buffer smaller
 * than thinK_cache_bytes reports for this configuration is refused with
 * THINK_ERR_CAPACITY before anything is written.  The buffers stay valid until
 * thinK_destroy.  `scores` may be NULL (scores are then not kept). */
thinK_status thinK_create(const thinK_config* cfg, const int32_t* seq_lens, const thinK_sizes* sizes, void* k_thin,
                          void* tail_k, void* tail_v, void* idx, void* scores, void* workspace, thinK_cache** out);

/* Prefill, Sec. 3.2: channel scores and I = Top_T(Score, T) for layers
 * [layer0, layer0 + nlayers) of every (b, h).
 *   q_obs: [B, S_obs, L, N_q, D] view -- row s of entry b is the query of prompt
 *          token S_b - S_obs + s ("Observation Window"); ignored (may hold a NULL
 *          ptr) for the key-norm criteria of Eq. 1.
 *   k:     [B, S_max, L, N_kv, D] view; rows >= S_b are never read.
 * Score[j] = sqrt(sum_g sum_s q^2 * sum_t k^2): the closed form of the Frobenius
 * norm of the rank-one product, with the G query heads of a group stacked.  All
 * S_b key rows enter the score.  Sums run in fp64 over fp32 partial chains of
 * at most 8 terms (bf16) or directly in fp64 (fp32), in a fixed order: results
 * are deterministic.  Equal scores go to the lower channel.  Writes idx (and
 * scores).  Layer indices address both the views and the cache. */
thinK_status thinK_score_select(thinK_cache* c, thinK_tensor5 q_obs, thinK_tensor5 k, int32_t layer0,
                                int32_t nlayers, void* stream);

/* Value-channel pruning (App. D, "ThinKV"), bf16 caches only.  With cfg.lambda_v > 0 the caller hands
 * over the two extra buffers of thinK_sizes (v_thin, perm_v) right after thinK_create; the path is then
 *   thinK_score_select_kv -> thinK_compact -> { thinK_append -> thinK_decode_attn }*
 * (thinK_prefill takes both steps).  `scores_v` (fp64 [B, L, N_kv, D], thinK_sizes.scores bytes) may be
 * NULL: the value scores are then not kept.  THINK_ERR_STATE if lambda_v == 0. */
thinK_status thinK_attach_value_cache(thinK_cache* c, void* v_thin, void* perm_v, void* scores_v);

/* thinK_score_select plus the value-channel score of App. D, Eqs. 3-4:
 *   Score_v[j] = || softmax(Q[-S_obs:] K^T / sqrt(D)) V[:, j] ||_F,   I_v = Top_T(Score_v, T_v),
 * T_v = floor((1 - lambda_v) D).  All S_b rows of K and V enter, no causal mask inside the window
 * (the formula has none), the G query heads of a group are stacked row-wise as for the key score, ties
 * go to the lower channel.  Both products run on tensor cores in bf16 with fp32 accumulation, the
 * softmax weights as a bf16 pair hi + lo; column norms in fp64.  Against an fp64 evaluation the scores
 * carry a relative error of about 1e-5, so two channels whose scores are closer than that may swap.
 * Writes perm_v (kept channels ascending, then the rest ascending).  `v` as for thinK_compact.
 * Kernels: blocks of 128 stacked window rows at D = 128 run on tcgen05.mma with accumulators in tensor memory,
 * everything else on mma.sync; cfg.value_score_kernel = THINK_VALUE_SCORE_MMA_SYNC keeps the mma.sync kernel
 * everywhere (same results within the tolerance above).
 * The tcgen05 kernel bounds its waits: if one runs out, the device error word gets bit 2 (see
 * thinK_device_error) and the scores of that call are unspecified; the next call starts clean. */
thinK_status thinK_score_select_kv(thinK_cache* c, thinK_tensor5 q_obs, thinK_tensor5 k, thinK_tensor5 v,
                                   int32_t layer0, int32_t nlayers, void* stream);

/* Prefill, Sec. 3.3: builds the two-part key cache for the given layers from
 * the idx thinK_score_select stored: K_T[t][c] = K[t][idx[c]] for t < S_p, and
 * the last S_recent rows of K and V copied unpruned to the tail.  After this
 * call K may be released by the caller; V rows [0, S_p) of `v` stay BORROWED:
 * thinK_decode_attn reads them in place on every step.  One view serves all
 * layers: a call with a different `v` starts a new prompt, i.e. the layers
 * outside its range count as not compacted until they are compacted again.
 * With lambda_v > 0 (after thinK_score_select_kv) the prefix values are thinned too:
 * V_T[t][c] = V[t][perm_v[c]], c < T_v, written to v_thin; the recent rows keep all D channels
 * (declared reading: App. D gives the criterion only; the split mirrors the keys').  `v` is then
 * not borrowed. */
thinK_status thinK_compact(thinK_cache* c, thinK_tensor5 k, thinK_tensor5 v, int32_t layer0, int32_t nlayers,
                           void* stream);

/* Prefill in one call: thinK_score_select followed by thinK_compact for the same layers on the
 * same stream (Sec. 3.2 + 3.3).  Arguments as for those two calls. */
thinK_status thinK_prefill(thinK_cache* c, thinK_tensor5 q_obs, thinK_tensor5 k, thinK_tensor5 v, int32_t layer0,
                           int32_t nlayers, void* stream);

/* Prefill behind a token-eviction method (the setting of the paper's main experiments, Sec. 4.1-4.2:
 * H2O or SnapKV first reduce every head to "KV-size" tokens, then the channels of the surviving keys
 * are pruned).  Instead of gathered K/V tensors the caller passes the method's per-head list of kept
 * tokens; scoring, compaction and the tail seed read the kept rows straight from the prompt tensors.
 *   The cache must have been created with seq_lens[b] = n_b, the number of tokens KEPT for entry b
 *   (the same for every head), and S_max >= max n_b.
 *   tok:        device int32 [B, L, N_kv, tok_stride]; tok[b][l][h][i], i < n_b, is the row of `k`
 *               and `v` that holds kept token i of that head.  The order of the list is the token
 *               order of the compressed cache: its last S_recent entries stay unpruned.  4-byte aligned.
 *   src_tokens: rows of `k` and `v` per entry; every used tok value must lie in [0, src_tokens).
 *               The host cannot see the list: an entry outside the range is read as row 0 and sets
 *               the device error word (thinK_device_error != 0), results are then unspecified.
 *   q_obs:      as for thinK_score_select (the window's queries are not evicted).
 *   v_kept:     device buffer of thinK_v_kept_bytes(c); receives the values of the kept tokens as
 *               dense [B, L, N_kv, S_max, D] and is BORROWED until thinK_destroy (decode reads it);
 *               `k` and `v` themselves may be released after the call.  One buffer for all layers.
 * Score[j] sums the squared keys over the kept rows only; everything downstream is thinK_compact
 * on the gathered tensors.  THINK_ERR_INVALID_ARG if tok_stride < n_b or n_b > src_tokens. */
thinK_status thinK_prefill_evicted(thinK_cache* c, thinK_tensor5 q_obs, thinK_tensor5 k, thinK_tensor5 v,
                                   const int32_t* tok, int64_t tok_stride, int32_t src_tokens, void* v_kept,
                                   int32_t layer0, int32_t nlayers, void* stream);

/* Bytes of the v_kept buffer of thinK_prefill_evicted: B * L * N_kv * S_max * D elements (0 if c is NULL). */
size_t thinK_v_kept_bytes(const thinK_cache* c);

/* Decode, Sec. 3.3: the new token's key and value join the unpruned tail.
 * k_new, v_new: dense [B, nlayers, N_kv, D].  Every layer of the cache must be
 * appended once per step (any split into layer ranges); THINK_ERR_CAPACITY once
 * max_new_tokens have been appended. */
thinK_status thinK_append(thinK_cache* c, const void* k_new, const void* v_new, int32_t layer0, int32_t nlayers,
                          void* stream);

/* Decode, Sec. 3.3 / Fig. 2 with the attention of Sec. 3.2: for each query head
 * the query is gathered to the kept channels and multiplied with the pruned
 * keys, the full query with the unpruned tail keys; the logits are concatenated,
 * scaled by 1/sqrt(D) (original D) and normalised by ONE softmax; the result is
 * the weighted sum of all value rows (prompt V in place + tail).
 *   q, out: dense [B, nlayers, N_q, D] in the cache dtype.
 * bf16: fp32 accumulation; fp32: logits in fp64, fp32 accumulation of p.V.
 * All layers in the range must hold the same number of tail tokens.
 * With lambda_v > 0 a pruned value channel of a prefix token counts as zero: output channel j sums the
 * tail tokens' share always and the prefix tokens' share only if j is kept. */
thinK_status thinK_decode_attn(thinK_cache* c, const void* q, void* out, int32_t layer0, int32_t nlayers,
                               void* stream);

/* One decode step in one call: thinK_append followed by thinK_decode_attn for the same layers (Sec. 3.3),
 * same arguments and results.  The attention kernel is launched as a programmatic dependent of the append
 * kernel: it starts streaming the pruned prefix while the append is still running and waits for it only
 * where it first touches the tail, which takes the append and the launch gap off the step's critical path.
 * bf16 caches; fp32 caches run the two launches back to back. */
thinK_status thinK_append_decode(thinK_cache* c, const void* k_new, const void* v_new, const void* q, void* out,
                                 int32_t layer0, int32_t nlayers, void* stream);

/* Score + select without any caller- or library-side allocation.  (The paper has no counterpart:
 * this is a packaging variant of thinK_score_select, same kernel, same results.)
 *
 * Who needs it: code that may not call cudaMalloc where it runs -- a plugin inside a host
 * application that hands out all device memory itself, a callback running under a memory pool that
 * forbids side allocations, or a process whose memory budget was fixed at start-up.  Such a caller
 * cannot provide the `workspace` that thinK_create asks for, so this call needs no handle and no
 * workspace: its scratch (lengths, ticket counters, fp64 partial sums) is a fixed 8 MiB array
 * compiled into the library.  Every GPU that loads the library holds those 8 MiB until exit.
 *
 *   cfg, seq_lens: as for thinK_cache_bytes (seq_lens on the HOST; copied with the stream).
 *   q_obs, k, layer0, nlayers: as for thinK_score_select.
 *   idx:    device out, uint8 [B, L, N_kv, T]; rows of the given layers are written.
 *   scores: device out, fp64 [B, L, N_kv, D], or NULL.
 *
 * Limit: lengths + counters + 2 * B * nlayers * C * 8 bytes per token split must fit in 8 MiB, where
 * C = N_kv*D when a token's keys are at most 4096 bytes, else N_kv*D rounded up to a whole number of
 * 4096-byte column blocks (2048 bf16 or 1024 fp32 columns each).  The call lowers its token split to
 * fit; if even one split does not fit it launches nothing and returns THINK_ERR_CAPACITY -- pass
 * fewer layers per call.
 * The first call on a device looks up the array's device address (once per device; make that first
 * call outside of any stream capture).  No cudaMalloc/cudaFree is called, here or later.
 * All calls share the one array, which still holds the previous call's contents: the call rewrites
 * the lengths and zeroes the tickets on `stream` before the kernel.  Two calls whose GPU work can
 * overlap (different streams, or different host threads without ordering) race on it: order them. */
thinK_status thinK_score_select_static(const thinK_config* cfg, const int32_t* seq_lens, thinK_tensor5 q_obs,
                                       thinK_tensor5 k, int32_t layer0, int32_t nlayers, uint8_t* idx,
                                       double* scores, void* stream);

/* Periodic re-pruning of the tail (App. C.1 of the paper, without its quantiser): the oldest unpruned
 * keys are thinned with the channels selected at prefill and joined to the pruned part, so the
 * full-width tail stops growing over a long generation.  Moves whole blocks of 64 tokens, oldest
 * first, for as long as at least `keep_recent` tokens stay unpruned; fewer movable tokens than 64 is
 * not an error (nothing happens).  The values of the moved tokens stay where they are (tail_v).
 * Attention afterwards treats those tokens like prefix tokens: gathered query x thinned keys.
 * bf16 caches only (THINK_ERR_UNSUPPORTED otherwise).  All layers of a decode call must have been
 * re-pruned alike.
 * What it saves is HBM traffic per decode step (the moved keys are read at T channels instead of D) and,
 * in the paper's accounting, cache size; it gives no ALLOCATED memory back: tail_k and tail_v stay sized
 * for S_recent + max_new_tokens full-width rows, positions keep counting against that capacity, and
 * k_thin carries ceil(cap/64) spare tiles per head for the moved blocks whether or not they are used.
 * thinK_sizes.model_think_bytes does not account for re-pruning. */
thinK_status thinK_reprune_tail(thinK_cache* c, int32_t keep_recent, int32_t layer0, int32_t nlayers, void* stream);

/* Tokens of the tail buffers of `layer` whose keys have been re-pruned (a multiple of 64), or -1. */
int32_t thinK_repruned_len(const thinK_cache* c, int32_t layer);

/* Tokens in the tail buffers of `layer` (S_recent + appended; re-pruned ones included), or -1. */
int32_t thinK_tail_len(const thinK_cache* c, int32_t layer);

/* Reads the device-side error word (0 = none) with a synchronous copy.  Bits: 1 a kept-token index of
 * thinK_prefill_evicted was out of range; 2 a bounded wait inside a kernel ran out (value-score kernel: that unit's
 * selection is missing; compaction: a tile whose row copies did not complete within about a second is left
 * unwritten -- re-create the cache); 4 a kernel found its shared memory misaligned; 8 a channel score was NaN or infinite (non-finite K or Q: exactly T channels
 * are still selected, NaN scores ranking lowest). */
thinK_status thinK_device_error(thinK_cache* c, int32_t* out_code);

thinK_status thinK_destroy(thinK_cache* c);

/* ---------------------------------------------------------------------------------------------------------
 * Paged key-value cache: the unpruned side of a serving process.  (The paper has no counterpart; its App. C.1
 * runs ThinK next to a quantised cache.)  Sequences whose keys are not (or not yet) thinned live in a pool of
 * pages; their lengths and page tables are DEVICE arrays, so a captured graph serves any batch.  A prompt that
 * is to be thinned is read back (thinK_paged_read) into the tensors thinK_prefill takes.
 *
 * A page holds 64 tokens of every layer and key head.  The pool is [L][num_pages][N_kv] blocks; a block is
 *     64 key rows | 64 value rows | scales of the 64 key rows | scales of the 64 value rows
 * and a row is the D channels of one token in order (no swizzle, no padding):
 *   THINK_PAGE_PLAIN  the elements themselves (cfg.dtype), no scales.
 *   THINK_PAGE_E4M3   one e4m3 byte per channel, one scale byte per row: byte e is 2^(e - 127), 255 a NaN.  Written rows
 *                     use the smallest power of two >= 2^-126 under which the row's largest magnitude is at
 *                     most 448; codes are x / scale rounded to nearest even.  bf16 caches only.
 *   THINK_PAGE_INT4   4 bits per channel (the even channel of a pair in the low half of the byte), code = n + 8,
 *                     one bf16 scale per 32 channels, channel groups in order: s = amax / 7 rounded to bf16,
 *                     n = x / s rounded to nearest even and limited to [-7, 7]; s = 0 gives n = 0.  Stored scales
 *                     are finite or NaN.  bf16 caches only.
 * A row (E4M3) or a group of 32 channels (INT4) that holds a NaN or an infinity is stored so that all of it reads
 * back as NaN, and sets bit 8 of the device error word.
 *
 * Sequence b of a call owns row b of the page table: its token t lies in page table[b * table_stride + t / 64],
 * slot t % 64.  Only the entries that a call needs are read, and what lies in a page outside of the tokens a call
 * names is never looked at (it may hold NaN) nor changed.  The host cannot see table, lengths and positions: an
 * entry outside [0, num_pages), a position outside [0, 64 * max_pages), a length above 64 * max_pages or a row
 * count above max_rows sets bit 16 of the error word; the tokens concerned are left out (not written, not read,
 * no weight in the softmax), and lengths and counts are cut to the limit.  Negative lengths and counts mean zero.
 *
 * A handle is constant after creation apart from its error word: calls that write different pages, or only read,
 * may run at the same time on any streams of its device, except that attention calls need a scratch buffer each
 * (see thinK_paged_decode_attn).  Calls enqueue on `stream`, which must belong to the device that was current
 * when the handle was created; that device must be current in every call. */
typedef enum { THINK_PAGE_PLAIN = 0, THINK_PAGE_E4M3 = 1, THINK_PAGE_INT4 = 2 } thinK_page_format;

typedef struct {
  int32_t L;             /* layers held by the pool */
  int32_t N_q, N_kv;     /* N_q % N_kv == 0, group size N_q / N_kv from 1 to 8 */
  int32_t D;             /* head dimension: 64 or 128 */
  int32_t num_pages;     /* pages of the pool */
  int32_t max_batch;     /* sequences a call may name, at most 4096 */
  int32_t dtype;         /* thinK_dtype of rows, queries and outputs */
  int32_t page_format;   /* thinK_page_format */
  double softmax_scale;  /* factor on q.k; 0 means 1/sqrt(D) */
} thinK_paged_config;

typedef struct {
  size_t pages;          /* bytes of the pool: L * num_pages * N_kv * block */
  size_t workspace;      /* bytes of the workspace, and of a scratch buffer */
  size_t block;          /* bytes of one (layer, page, key head) block */
} thinK_paged_sizes;

/* Page table of a call (device memory, int32 [B][table_stride], the first max_pages entries of a row usable). */
typedef struct {
  const int32_t* table;
  int64_t table_stride;  /* in entries, >= max_pages */
  int32_t max_pages;
  int32_t B;             /* sequences of this call, 1 <= B <= max_batch */
} thinK_page_table;

typedef struct thinK_paged thinK_paged; /* opaque, host side */

thinK_status thinK_paged_bytes(const thinK_paged_config* cfg, thinK_paged_sizes* out);

/* Builds the host-side handle; zeroes the counters in `workspace` (synchronously) and leaves `pages` alone.  `sizes`
 * (host) states the bytes allocated for the two buffers (256-byte aligned), THINK_ERR_CAPACITY if too few.  The
 * buffers stay valid until thinK_paged_destroy. */
thinK_status thinK_paged_create(const thinK_paged_config* cfg, const thinK_paged_sizes* sizes, void* pages,
                                void* workspace, thinK_paged** out);

/* Parts of a block, for thinK_paged_offset. */
typedef enum { THINK_PART_K = 0, THINK_PART_V = 1, THINK_PART_K_SCALE = 2, THINK_PART_V_SCALE = 3 } thinK_page_part;

/* Byte offset in the pool of a token's row (or of its scales) in the given part, for programs that move pages
 * themselves; -1 if anything is out of range or the format has no such part. */
int64_t thinK_paged_offset(const thinK_paged_config* cfg, int32_t layer, int32_t page, int32_t head, int32_t slot,
                           int32_t part);

/* Writes rows to their pages, quantising them.  k, v: [B, max_rows, nlayers, N_kv, D] views; layer index i of the
 * views is layer layer0 + i of the pool.  Row s < rows[b] of entry b becomes token pos[b] + s.
 *   pos, rows: device int32 [B]; NULL means 0 for all, max_rows for all.
 * One-token appends (max_rows = 1, pos = the lengths so far) and whole prompts use the same call.  Rows at and
 * behind rows[b] are not read.  No two rows of a call may go to the same slot of the same page (what that slot
 * holds afterwards is unspecified). */
thinK_status thinK_paged_write(thinK_paged* p, thinK_tensor5 k, thinK_tensor5 v, thinK_page_table table,
                               const int32_t* pos, const int32_t* rows, int32_t max_rows, int32_t layer0,
                               int32_t nlayers, void* stream);

/* A step of a packed batch: the new tokens of all sequences stand one behind the other, sequence after sequence
 * ("packed token" i).  From the tokens that each sequence holds and those it is to gain (change[b] > 0) or to lose (< 0,
 * from its end; more than it holds: all) the call takes pages from the list of free ones, gives pages back to it, and says
 * where each packed token goes.  Everything is device memory, so a captured graph plans every step.
 *   free_pages: int32 [num_pages], the first free_count[0] of which are the free pages.  Pages given back are put
 *           behind them, in the order of their sequences and tokens; pages are taken from the end, first sequence
 *           first.  Entries behind the pages that are left hold whatever they held.
 *   table:  the entries that a sequence gains are written; those that it loses stay as they are.
 * A sequence gains what it asked for or nothing: nothing if it would pass 64 * max_pages tokens (it then counts as asking
 * for nothing), if it needs pages and all that it and the sequences in front of it ask for are more than there are
 * (those given back in this call among them), or if their tokens are more than max_tokens.
 * Results:
 *   pos:    int32 [B], tokens held before the new ones: the position of the first new token.
 *   rows:   int32 [B], tokens gained.            start: int32 [B + 1], packed tokens in front of a sequence's first; the
 *           last entry is their number.
 *   token_pos, slots: int32 [max_tokens], position and slot (64 * page + place in the page) of every packed token; -1 behind
 *           the last one.  16-byte aligned.
 *   seq_len_out: int32 [B], pos + rows; may be seq_len itself.   free_left: int32 [1]; may be free_count itself.
 * No other two of the arrays may overlap (THINK_ERR_INVALID_ARG).  A length above 64 * max_pages (cut), a change that does
 * not fit the table, a count of free pages outside [0, num_pages] (cut) and a page outside the pool (it is moved as it is, its
 * tokens get slot -1) set bit 16 of the error word.  Calls on one list of free pages must be ordered.
 * THINK_ERR_UNSUPPORTED for more than 2^25 - 1 pages, or tables of more than 2^31 - 1 entries. */
typedef struct {
  int32_t* table;            /* [B][table_stride], the first max_pages entries of a row usable */
  int64_t table_stride;
  int32_t max_pages;
  int32_t B;                 /* 1 <= B <= max_batch */
  const int32_t* seq_len;    /* [B] tokens held */
  const int32_t* change;     /* [B] tokens to gain or to lose */
  int32_t* free_pages;       /* [num_pages] */
  const int32_t* free_count; /* [1] */
  int32_t *pos, *rows, *start, *token_pos, *slots, *seq_len_out, *free_left;
  int32_t max_tokens;        /* room for packed tokens, at most 2^30 */
} thinK_paged_step;

thinK_status thinK_paged_plan(thinK_paged* p, const thinK_paged_step* step, void* stream);

/* Writes packed rows to their slots, quantising them as thinK_paged_write does.  k, v: [tokens, nlayers, N_kv, D] views (the
 * s axis of the view is the token, its b axis is not looked at).  Row i goes to slot slots[i] of thinK_paged_plan; a
 * negative one means nowhere (the row is not stored), one behind the pool sets bit 16 of the error word.
 * No two rows may go to the same slot. */
thinK_status thinK_paged_write_slots(thinK_paged* p, thinK_tensor5 k, thinK_tensor5 v, const int32_t* slots, int32_t tokens,
                                     int32_t layer0, int32_t nlayers, void* stream);

/* Reads rows back: the reverse of thinK_paged_write, same arguments; k and v are written.  Values are the stored
 * ones rounded to cfg.dtype (E4M3: exact; INT4: n * s to nearest even).  Rows at and behind rows[b] of the views, and
 * rows whose page is out of range, are left as they were.  No two rows of the views, k's and v's together, may share
 * memory, whether the call fills them or not: THINK_ERR_INVALID_ARG.  (Strides of 0 only where there is one index;
 * interleaved views are fine; views so entangled that some ten thousand steps do not tell count as sharing.) */
thinK_status thinK_paged_read(thinK_paged* p, thinK_tensor5 k, thinK_tensor5 v, thinK_page_table table,
                              const int32_t* pos, const int32_t* rows, int32_t max_rows, int32_t layer0,
                              int32_t nlayers, void* stream);

/* Attention of one new token per sequence over its first seq_len[b] tokens (append the token's own key and value
 * first): out = softmax(softmax_scale * q K^T) V for every query head, head h of the queries reading key head
 * h / (N_q / N_kv).
 *   q, out: dense [B, nlayers, N_q, D] in cfg.dtype.  q, out and lse may not overlap.
 *   lse:    fp32 [B, nlayers, N_q], the natural logarithm of the softmax's sum (for joining with attention over
 *           other tokens), or NULL.
 *   seq_len: device int32 [B].  A sequence without tokens gets out = 0 and lse = -infinity; one with tokens
 *           whose logits are all -infinity (keys of infinities) gets out = NaN and lse = -infinity.
 *   scratch: NULL for the handle's own workspace, or a device buffer of scratch_bytes >= thinK_paged_sizes.workspace
 *           (of the handle that it is given to), 256-byte aligned, that was filled with zeros once before its first use.
 *           A call leaves it ready for the next one, of the same handle or of any other.  Calls that may run at the
 *           same time - on two streams, or as two captured graphs - need a scratch buffer each.
 * A call names at most 2^29 table entries (4 * B * max_pages + 2 * B below 2^31), THINK_ERR_UNSUPPORTED otherwise.
 * Logits, softmax sums and outputs are accumulated in fp32.  On bf16 caches a weight (of quantised pages: times its
 * value's scale) meets the values as a pair of bf16, within 2^-16 of itself or, if it is smaller than 2^-117, 2^-133
 * (in any cache weights below 2^-117 of the largest may count as none);
 * queries are exact, on E4M3 pages relative to the row's largest channel, 2^-39 of which is the smallest step.  fp32
 * caches compute in fp32.  Results do not depend on timing: partial results are joined in token order. */
thinK_status thinK_paged_decode_attn(thinK_paged* p, const void* q, void* out, float* lse, thinK_page_table table,
                                     const int32_t* seq_len, void* scratch, size_t scratch_bytes, int32_t layer0,
                                     int32_t nlayers, void* stream);

/* Attention of many new tokens per sequence, causal, over the pages (write the tokens' keys and values first): row s <
 * rows[b] of entry b is the query of token pos[b] + s and sees tokens 0 .. pos[b] + s of its sequence.  Prompts from their
 * beginning, later parts of a prompt, a few guessed tokens and single ones may stand side by side.
 *   q, out: start = NULL: [B, max_rows, nlayers, N_q, D] views; else packed, [max_rows, nlayers, N_q, D] (their b axis is not
 *           looked at), with row s of entry b at start[b] + s and max_rows the packed rows of all entries.  Rows that no
 *           entry has are left as they were.  No row of out may share memory with another, nor with one of q.
 *   lse:    fp32, dense [B, max_rows, nlayers, N_q] or [max_rows, nlayers, N_q], as in thinK_paged_decode_attn; or NULL.
 *   pos, rows, start: device int32 [B]; NULL means 0 for all, max_rows for all (not with start), padded.
 *   scratch: device buffer of scratch_bytes >= thinK_paged_prompt_scratch(p), 256-byte aligned; its contents do not matter.
 *           Calls that may run at the same time need a scratch buffer each.
 * A count of rows above max_rows, a start outside the packed rows, a negative position and tokens behind the table's end
 * set bit 16 of the error word: rows are cut to what there is, tokens that have no page are left out.  A row without
 * tokens gets out = 0 and lse = -infinity; one with tokens whose logits are all -infinity out = NaN and lse = -infinity.
 * What a row does not see does not reach it, whatever it holds (NaN, infinities); what it sees does: an infinite value gives an
 * infinity or a NaN, however small its weight.
 * Logits, softmax sums and outputs are accumulated in fp32 from the stored values, which enter exactly (4-bit ones, of 11
 * bits, as the sum of two bf16; values past bf16's largest, which a row that holds that number may be stored as in E4M3, count as
 * infinite as they do when read back, 4-bit ones from 2^129 - 2^121 on, which no written row holds).  On bf16 caches a weight meets the values rounded to bf16 (2^-8 of itself at most; weights
 * below 2^-118 of the largest may count as none); the softmax sum takes it unrounded.  fp32 caches compute in fp32.  Results do not
 * depend on timing.
 * THINK_ERR_UNSUPPORTED where 64 * max_pages + max_rows passes 2^31 - 1, where (max_rows * N_q / N_kv / 256 + 1) * (64 * max_pages +
 * max_rows + 384) * B * nlayers * N_kv passes 4e15 (fp32: 64 in place of 256 and 384; packed rows count for every entry), and where
 * the kernel could not be set up when the handle was created (its other calls work all the same). */
thinK_status thinK_paged_prompt_attn(thinK_paged* p, thinK_tensor5 q, thinK_tensor5 out, float* lse, thinK_page_table table,
                                     const int32_t* pos, const int32_t* rows, const int32_t* start, int32_t max_rows,
                                     void* scratch, size_t scratch_bytes, int32_t layer0, int32_t nlayers, void* stream);

/* Bytes of the scratch buffer of thinK_paged_prompt_attn (0 if p is NULL). */
size_t thinK_paged_prompt_scratch(const thinK_paged* p);

/* The handle's error word, read with a synchronous copy; wait for the calls that it is to cover first.  Bits: 8 and 16 as
 * above; of thinK_paged_prompt_attn on bf16 caches also 2, a bounded wait inside the kernel ran out, and 4, a block found its
 * shared memory misaligned (rows that such a block had to compute are not to be relied on).  The word keeps its bits as long as
 * the handle lives. */
thinK_status thinK_paged_device_error(thinK_paged* p, int32_t* out_code);

thinK_status thinK_paged_destroy(thinK_paged* p);

/* ---------------------------------------------------------------------------------------------------------
 * Rotary positions, which queries and keys carry before they go to thinK_paged_write_slots, thinK_paged_write,
 * thinK_append or thinK_prefill.  (The paper takes rotated keys as given.)  The first rot_dim channels of a row make
 * rot_dim / 2 pairs; pair j of a token at position t becomes
 *     (a, b) -> m (a cos(t f_j) - b sin(t f_j),  b cos(t f_j) + a sin(t f_j)),      f_j = theta^(-2 j / rot_dim)
 * with frequencies scaled for contexts longer than the one that a model was trained on:
 *   LINEAR  f_j / factor
 *   NTK     theta * factor^(rot_dim / (rot_dim - 2)) in theta's place
 *   YARN    f_j (1 - r_j) + r_j f_j / factor, r_j = (j - low) / (high - low) within [0, 1], where low and high are the pairs
 *           that make `fast` (32) and `slow` (1) turns over the trained context, rot_dim ln(trained / (2 pi turns)) /
 *           (2 ln theta), rounded down and up into [0, rot_dim - 1]; m = 0.1 ln(factor) + 1   (Peng et al., 2023)
 *   BANDS   f_j (1 - r_j) + r_j f_j / factor, r_j = (fast - turns_j) / (fast - slow) within [0, 1] for the turns that the pair
 *           makes over the trained context; slow 1, fast 4
 * Angles are exact to 2^-27 turns at any position; products and sums are fp32, rounded once to the rows' type. */
typedef enum {
  THINK_ROPE_HALVES = 0, /* pair j: channels j and j + rot_dim / 2 */
  THINK_ROPE_PAIRS = 1   /* pair j: channels 2 j and 2 j + 1       */
} thinK_rope_layout;
typedef enum {
  THINK_ROPE_PLAIN = 0, THINK_ROPE_LINEAR = 1, THINK_ROPE_NTK = 2, THINK_ROPE_YARN = 3, THINK_ROPE_BANDS = 4
} thinK_rope_scaling;

typedef struct {
  int32_t D;             /* channels of a row, at most 256; a row is a multiple of 16 bytes */
  int32_t rot_dim;       /* channels that turn: even, 2 <= rot_dim <= D; the others stay as they are */
  int32_t layout;        /* thinK_rope_layout */
  int32_t scaling;       /* thinK_rope_scaling */
  int32_t dtype;         /* thinK_dtype of the rows */
  double theta;          /* base, at least 1 */
  double factor;         /* context extension, at least 1 (not read for PLAIN) */
  double trained;        /* tokens of the trained context (YARN, BANDS) */
  double slow, fast;     /* turns; 0 means the defaults above (YARN, BANDS) */
  double attention_factor; /* m; 0 means 1, for YARN 0.1 ln(factor) + 1 */
} thinK_rope_config;

typedef struct thinK_rope thinK_rope; /* opaque, host side, constant: any number of calls may use it at once */

thinK_status thinK_rope_create(const thinK_rope_config* cfg, thinK_rope** out);

/* Radians per token of a pair, -1 if there is no such pair. */
double thinK_rope_frequency(const thinK_rope* r, int32_t pair);

/* Turns queries and keys in one launch: q, q_out are [B, S, nlayers, N_q, D] views, k, k_out [B, S, nlayers, N_kv, D]; N_q or
 * N_kv may be 0, the views concerned are then not looked at.
 *   pos:    device int32.  pos_stride = 0: row s of entry b has position pos[b] + s; else pos[b * pos_stride + s].
 *           A row whose position is negative (or passes 2^31 - 1) is left as it was in q_out and k_out.
 *   rows:   device int32 [B], rows of an entry (the others are left as they were), or NULL for S.
 *   transpose: 1 turns by -t f_j (with the same m): the gradient of a loss with respect to q and k from those with
 *           respect to q_out and k_out.
 * q_out may be q itself (same pointer and strides), k_out k; apart from that no row of q_out and k_out may share memory with
 * another row of the two, nor with one of q or k (THINK_ERR_INVALID_ARG).  q and k may repeat rows (strides of 0).
 * THINK_ERR_UNSUPPORTED for more than 2^24 pieces of 16 bytes in all rows of a token, and for more than 2^31 - 1 blocks of tokens. */
thinK_status thinK_rope_apply(const thinK_rope* r, thinK_tensor5 q, thinK_tensor5 k, thinK_tensor5 q_out, thinK_tensor5 k_out,
                              int32_t B, int32_t S, int32_t nlayers, int32_t N_q, int32_t N_kv, const int32_t* pos,
                              int64_t pos_stride, const int32_t* rows, int32_t transpose, void* stream);

thinK_status thinK_rope_destroy(thinK_rope* r);

#ifdef __cplusplus
}
#endif
#endif /* THINK_H_ */
