/*
 * madakv.h - C ABI of the MadaKV eviction + ragged-decode hot path for one AMD
 * MI355X (gfx950).
 *
 * The calls follow the method of "MadaKV: Adaptive Modality-Perception KV Cache
 * Eviction" (arxiv 2506.15724), Section 3:
 *
 *   madakv_score          Sec. 3.3 Eq. 7 (proxy-token scores), Eq. 6 (modality
 *                         mass), Eq. 9 (theta-mass sparsity counts), plus score
 *                         pooling used for ranking only
 *   madakv_allocate       Sec. 3.3 Eq. 8 (per-head, per-modality budgets) and
 *                         Eq. 10-11 (layer compensation, budget recurrence)
 *   madakv_select_gather  Sec. 3.3, end of the MPA paragraph: per-head,
 *                         per-modality eviction; builds the reduced KV cache
 *   madakv_decode_attn    Sec. 3.1 Eq. 3-5: append K_t, V_t and attend over the
 *                         reduced cache
 *   madakv_evict          Sec. 3.3 Eq. 6-11 and the eviction itself: the first three calls in one
 *   madakv_score_lse      Sec. 3.3 Eq. 7 with the softmax normalisers of the proxy rows given
 *                         (the prefill attention of Sec. 3.1 Eq. 5 has them)
 *   madakv_score_prompt   Eq. 7 with every position of the prompt as a proxy token: the attention weight a key has
 *                         accumulated over the whole prompt
 *   madakv_decode_attn_weights  a decode step that goes on accumulating it, and the eviction of one row per step by it
 *   madakv_cache_rows     the rows of an 8-bit or 4-bit reduced cache in the type of the model
 *   madakv_prompt_attn    that prefill attention for every position (Sec. 3.1 Eq. 5), whose normalisers madakv_score_prompt takes
 *   madakv_tree_attn      Eq. 5 for several drafted tokens per step over the reduced cache
 *   madakv_tree_commit    Eq. 4 for those of them that are accepted
 *   madakv_window_attn_score  that prefill attention for the proxy rows (Sec. 3.1 Eq. 5) with Eq. 7, 6, 9 as
 *                         by-products of the same pass
 *
 * General rules
 *   - Plain C, no exceptions.  Every call returns a madakv_status (0 = OK).
 *   - Every tensor pointer is a DEVICE pointer owned by the caller, contiguous,
 *     row-major in the stated shape.  Q/K/V-like tensors (q_win, k, v, k_c, v_c, q,
 *     k_new, v_new, out) and the workspaces must be aligned to 16 bytes; the other
 *     arrays to their element size (kv_off 8, float / int32 arrays and stats 4).
 *     The library never allocates, frees or keeps tensor memory.  A null or
 *     misaligned pointer gives MADAKV_ERR_INVALID_ARG; nothing is enqueued then.
 *   - All work is ordered on the caller's stream (a hipStream_t passed as void*, NULL = the
 *     null stream): it starts after what the stream held before the call and is complete, as far
 *     as the stream is concerned, before anything enqueued after it.  madakv_allocate,
 *     madakv_score_prompt, madakv_prompt_attn, madakv_cache_rows, the tree and the decode calls enqueue on that stream only.  madakv_score, madakv_score_lse,
 *     madakv_select_gather and madakv_evict over four or more layers also use the handle's own
 *     stream for the per-head statistics / selection kernels of one layer group while another
 *     group is scored or gathered; that stream forks from and joins the caller's stream through
 *     events inside the call.  No call synchronises the device.
 *   - Arguments are validated on the host before anything is enqueued.  Errors
 *     found there leave all outputs untouched.
 *   - The handle belongs to the HIP device that was current in madakv_create; that device must
 *     be current in every later call on it.  It owns device memory: carry state (layer recurrence, cache
 *     cursors), per KV head of the model 128 bytes per query head that it serves and 4 more (at most 1028) in which
 *     decode's pieces count themselves, the words in which the scoring kernels exchange row statistics
 *     (per head up to about 1 byte per key of the prompt with G * W <= 64, up to 4.3
 *     beyond, or less than 1 MB in all), up to MADAKV_STATIC_SCRATCH_BYTES for madakv_decode_attn_static, with a paged cache
 *     its page table, and for contexts of four or more 16384-token chunks on at most 128 heads per layer 25 to 72 KB per
 *     chunk of up to 128 heads for the lists and histograms that the per-head statistics and selection kernels share
 *     between launches; and a little pinned
 *     host memory, one extra stream of default priority and a few events.  Calls on one handle
 *     must not overlap, a graph that holds captured calls is not replayed after madakv_destroy, and a handle's
 *     lengths are those of one cache: a second cache that is evicted while the first is still decoded has a handle of its own.
 *   - Layers are addressed as a range [layer0, layer0 + n).  Tensor arguments hold
 *     only the n layers of the call, layer-major.  madakv_allocate and
 *     madakv_select_gather carry state from layer to layer and must be called in
 *     increasing layer order, starting at layer 0 (which resets the state).
 *   - Modality ids: 0 = text, 1 = image (2, 3: further modalities when n_modalities says so).
 *     Query head j reads KV head j / G,
 *     G = n_q_heads / n_kv_heads.
 */
#ifndef MADAKV_H
#define MADAKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MADAKV_OK = 0,
  MADAKV_ERR_INVALID_ARG = -1,        /* null / misaligned pointer, bad layer range, out of decode slack */
  MADAKV_ERR_BAD_SHAPE = -2,          /* n_q_heads % n_kv_heads, window > ctx_len, unsupported head_dim ... */
  MADAKV_ERR_BAD_BUDGET = -3,         /* budget <= window while budget < ctx_len */
  MADAKV_ERR_WORKSPACE_TOO_SMALL = -4,
  MADAKV_ERR_UNSUPPORTED_DTYPE = -5,
  MADAKV_ERR_HIP = -6,                /* see madakv_last_hip_error */
  MADAKV_ERR_UNIMPLEMENTED = -7
} madakv_status;

enum { MADAKV_FP32 = 0, MADAKV_BF16 = 1 };

/* Hyper-parameters and shapes.  The paper names the proxy-token count, theta and
 * the layer budget (Sec. 3.3) without giving values; they are set here. */
typedef struct {
  int32_t n_layers;        /* 1 .. 1024 */
  int32_t batch;           /* >= 1 */
  int32_t n_q_heads;       /* multiple of n_kv_heads */
  int32_t n_kv_heads;      /* 1 .. 64 */
  int32_t head_dim;        /* 64 or 128 */
  int32_t ctx_len;         /* L, prompt length, <= 2^20 */
  int32_t window;          /* W = number of proxy tokens (the last W prompt positions); G*W <= 256 */
  int32_t budget;          /* tokens kept per KV head per layer, window included; >= ctx_len keeps all */
  int32_t dtype;           /* MADAKV_FP32 / MADAKV_BF16: type of Q, K, V and of the reduced cache */
  int32_t pool_k;          /* odd, 1 .. 63: max-pool width on the scores used for ranking; 1 = none */
  int32_t mpa_mode;        /* 1 = Eq. 8 modality split; 0 = modality-agnostic top-k; 2 / 3 = fixed priority
                              baselines: text / image takes all it can, the other modality the rest */
  int32_t hcc_mode;        /* 1 = Eq. 9-11 compensation, head totals follow demand; 0 = every head gets
                              budget - window; 2 = Eq. 9-11 layer totals shared equally by the heads */
  int32_t hcc_rho;         /* >= 1: demand clamp ratio around the running nominal budget */
  float   theta;           /* Eq. 9 threshold, in (0, 1] */
  float   softmax_scale;   /* 0 = 1/sqrt(head_dim) */
  int32_t max_new_tokens;  /* decode slack per head in the reduced cache */
  int32_t out_fp32;        /* decode output: 1 = float, 0 = same as dtype */
  int32_t pool_mode;       /* 0 = max-pool, 1 = average-pool (same clipped neighbourhood) */
  int32_t share_mode;      /* Eq. 6 masses over 0 = the candidates, 1 = all L columns (window included) */
  int32_t select_mode;     /* 0 = top scores per modality; 1 = score-free baseline: the first sink_tokens
                              candidates and the most recent ones, b_t + b_v in total */
  int32_t sink_tokens;     /* >= 0, used by select_mode 1 */
  int32_t cache_fp8;       /* 1 = the reduced cache k_c, v_c holds 8-bit floats (OCP E4M3: round to nearest even,
                              magnitudes above 448 saturate), one byte per element, instead of dtype; needs
                              dtype = MADAKV_BF16.  Q, K, V, k_new, v_new and out stay in dtype.
                              4 = 4-bit floats (needs dtype = MADAKV_BF16): k_c holds capacity_tokens * (head_dim / 2 +
                              head_dim / 32) bytes, and v_c likewise: first the codes of all rows, head_dim / 2 bytes each
                              (element 2i of a row is the low half of its byte i), then their scales, head_dim / 32
                              bytes per row.  An element is an E2M1 float (0, 0.5, 1, 1.5, 2, 3, 4, 6, the high bit the sign)
                              times 2^(b - 127), b the scale byte of its block of 32 dims: the least that leaves the largest
                              magnitude of the block at most 7, within 7 .. 252; elements are rounded to nearest even and
                              saturate at 6; infinities and NaN are taken for the largest finite bf16.  The row numbers
                              in kv_off, kept_idx and the page table count rows as ever. */
  int32_t n_modalities;    /* M, 2 .. 4: modality ids in the mask are 0 .. M-1 (the paper has text = 0 and
                              image = 1; more modalities are the extension its Sec. 6 names) */
  int32_t page_rows;       /* 0 = every head's segment of the reduced cache is its kept rows followed by
                              max_new_tokens free rows; 16, 32, 64, 128 or 256 = paged reduced cache: a segment
                              is the kept rows rounded up to whole pages of that many rows, and the rows decode
                              appends (Sec. 3.1 Eq. 4) continue in pages taken on demand from a pool all heads
                              of a batch item share, so no head reserves room for generation up front */
} madakv_config;

/* Per-head statistics that madakv_score hands to madakv_allocate: a record of M floats
 * (Eq. 6 attention mass per modality) followed by M int32 (Eq. 9 theta-mass counts).  With
 * two modalities the record is this struct. */
typedef struct {
  float   w_t, w_v;        /* Eq. 6 attention mass on text / image candidates */
  int32_t k_t, k_v;        /* Eq. 9 theta-mass counts */
} madakv_head_stats;

typedef struct madakv_handle madakv_handle;

/* Creates a handle on the current HIP device.  *out is set only on success.  The handle's memory is set
 * up when the call returns: its first call may be on any stream, under graph capture too.
 * Errors: INVALID_ARG (null), BAD_SHAPE, BAD_BUDGET, UNSUPPORTED_DTYPE, HIP. */
int32_t madakv_create(const madakv_config* cfg, madakv_handle** out);
int32_t madakv_destroy(madakv_handle* h);

/* hipError_t of the last failing HIP call made through this handle (0 if none). */
int32_t madakv_last_hip_error(const madakv_handle* h);

/* Bytes of caller-provided scratch that serve calls over up to n layers (the worst case over all
 * such layer ranges: a call over fewer layers can need more than one over n).  So do the other calls named
 * madakv_*_workspace_bytes.  Any out pointer may be NULL. */
int32_t madakv_workspace_bytes(const madakv_handle* h, int32_t n_layers_per_call,
                               size_t* score_ws, size_t* select_ws, size_t* decode_ws);

/* Rows (tokens) the reduced cache k_c / v_c and kept_idx must hold for the whole
 * model: n_layers * batch * n_kv_heads * (min(budget, ctx_len) + max_new_tokens); with a paged
 * cache n_layers * batch * n_kv_heads * (ceil(min(budget, ctx_len) / page_rows) + 1 +
 * ceil(max_new_tokens / page_rows)) pages of page_rows rows.
 * Known without a device sync because the sum of budgets is conserved exactly. */
int32_t madakv_compact_capacity_tokens(const madakv_handle* h, int64_t* tokens);

/* Environment variables (diagnostics, read at every call they concern; not needed in normal use):
 *   MADAKV_SCORE_TWO_SWEEPS=1   score with the two-sweep kernels (K read twice) everywhere
 *   MADAKV_SCORE_SPIN_LIMIT=n   polls a workgroup of the one-sweep scoring kernel spends on a missing word
 *                               before it computes the head's row statistics alone (default 65536)
 *   MADAKV_LAYER_GROUPS=n       layer groups a call over several layers is pipelined in (1..4; default: as many as
 *                               leave a group 256 heads)
 *   MADAKV_SCORE_NO_PARKED_CHUNKS=1   long heads: all chunks of a head in one launch of the one-sweep kernel, also
 *                               where a few of them are in the way of one more head fitting the chip */

/* Eq. 7, Eq. 6, Eq. 9 and pooling for layers [layer0, layer0 + n).
 *   q_win    [n, B, Hq, W, d]  queries of the last W prompt positions
 *   k        [n, B, H, L, d]   prompt keys
 *   mask     [B, L] uint8      modality id per position
 *   psi      [n, B, H, L]      out: psi(i) = sum over the G*W proxy rows of the causal
 *                              softmax(scale * q k^T) they pay to key i
 *   psi_pool [n, B, H, L-W]    out: max of psi over |j - i| <= (pool_k-1)/2 within the
 *                              candidates [0, L-W)
 *   stats    [n, B, H]         out: records {float w[M]; int32 k[M]} over the candidates
 *   n_mod    [B, M] int32      out: candidate count per modality
 * ws / ws_bytes: scratch of at least score_ws bytes.  Its first int32 is a diagnostic counter the
 * library only ever adds to: workgroups of the one-sweep scoring kernel that gave up waiting for the
 * row statistics of their head's other workgroups and computed them alone (0 in normal operation if
 * the caller cleared it). */
int32_t madakv_score(madakv_handle* h, int32_t layer0, int32_t n,
                     const void* q_win, const void* k, const uint8_t* mask,
                     float* psi, float* psi_pool, void* stats, int32_t* n_mod,
                     void* ws, size_t ws_bytes, void* stream);

/* Sec. 3.3 Eq. 7 (then Eq. 6, Eq. 9, pooling as in madakv_score) for a caller whose prefill attention
 * (Sec. 3.1 Eq. 5 on the last W prompt positions) kept the softmax normalisers of the proxy
 * rows (any flash-attention kernel has them): with
 *   row_lse  [n, B, Hq, W] float  natural log of sum_i exp(scale * q_r . k_i) over the keys row r sees
 * the first of the two passes over K is not needed and psi costs one pass.  Everything else as
 * in madakv_score; the results are the same up to the rounding of row_lse. */
int32_t madakv_score_lse(madakv_handle* h, int32_t layer0, int32_t n,
                         const void* q_win, const void* k, const uint8_t* mask, const float* row_lse,
                         float* psi, float* psi_pool, void* stats, int32_t* n_mod,
                         void* ws, size_t ws_bytes, void* stream);

/* The step before the eviction path, fused with its first step: the prefill attention of the last W prompt
 * positions (Sec. 3.1 Eq. 5 for the proxy rows of Sec. 3.3), whose softmax rows are the alpha of Eq. 7.  One pass
 * over K and V gives
 *   out      [n, B, Hq, W, d]  softmax(scale * q_win k^T) v over the keys each proxy row sees (float if out_fp32
 *                              else dtype)
 *   row_lse  [n, B, Hq, W]     optional (may be NULL): natural log-sum-exp of each row
 * and psi, psi_pool, stats, n_mod exactly as madakv_score defines them (up to the rounding order of psi).  A model
 * whose prefill calls this for its last W positions needs no scoring sweep of its own: madakv_allocate and
 * madakv_select_gather follow directly.  v [n, B, H, L, d]; ws: madakv_window_attn_workspace_bytes(h, n) bytes;
 * everything else as in madakv_score.  With more than 32 proxy rows (grouped queries, wide windows) the rows are
 * taken in blocks of 32, each with a pass over K and V of its own, or, above 64 rows in calls with enough workgroups
 * that way, in one pass for all rows behind a sweep over K.  MADAKV_ERR_UNIMPLEMENTED unless dtype is bf16
 * and ctx_len <= 131072 (head_dim 128) / 196608 (head_dim 64). */
int32_t madakv_window_attn_workspace_bytes(const madakv_handle* h, int32_t n_layers_per_call, size_t* bytes);
int32_t madakv_window_attn_score(madakv_handle* h, int32_t layer0, int32_t n,
                                 const void* q_win, const void* k, const void* v, const uint8_t* mask,
                                 void* out, float* row_lse,
                                 float* psi, float* psi_pool, void* stats, int32_t* n_mod,
                                 void* ws, size_t ws_bytes, void* stream);

/* Eq. 7 with every position of the prompt as a proxy token, the scores of heavy-hitter eviction: the attention weight each
 * key has received from all queries.
 *   q        [n, B, Hq, L, d]  queries of the whole prompt
 *   k        [n, B, H, L, d]
 *   row_lse  [n, B, Hq, L] float or NULL  natural log of sum_i exp(scale * q_r . k_i) over the keys i <= r, which the prefill
 *                              attention has; without it the call forms the logits of prompts
 *                              of more than 256 positions twice
 *   psi      [n, B, H, L]      out: sum over the G * L query rows of the causal softmax weight they pay to key i
 * mask, psi_pool, stats, n_mod: all NULL (the scores alone), or as in madakv_score, for madakv_allocate and
 * madakv_select_gather to go on with; they are those of psi * 2^-s, s the least with W * 2^s >= L, so that they have the
 * range that W proxy tokens give (budgets, counts and rankings do not depend on it).
 *   ws       madakv_score_prompt_workspace_bytes(h, n) bytes
 * A row's normaliser is one float: a weight is off by 2^-24 of the magnitude of its row's log-sum-exp, relative to the weight (1e-5 at 200).
 * MADAKV_ERR_UNIMPLEMENTED unless dtype is bf16. */
int32_t madakv_score_prompt_workspace_bytes(const madakv_handle* h, int32_t n_layers_per_call, size_t* bytes);
int32_t madakv_score_prompt(madakv_handle* h, int32_t layer0, int32_t n,
                            const void* q, const void* k, const uint8_t* mask, const float* row_lse,
                            float* psi, float* psi_pool, void* stats, int32_t* n_mod,
                            void* ws, size_t ws_bytes, void* stream);

/* The prefill attention of the whole prompt (Sec. 3.1 Eq. 5 at every position), causal, with grouped heads.
 *   q        [n, B, Hq, L, d]
 *   k, v     [n, B, H, L, d]
 *   seq_off  [B, n_seq + 1] int32 on the device, ascending within 0 .. L, or NULL with n_seq = 0.  Sequence s of batch item b has the
 *            positions seq_off[b][s] .. seq_off[b][s + 1] - 1 (possibly none); a position sees those of its own sequence up to itself.
 *            One sequence of each item is a padded batch, several are packed prompts.  NULL: all L positions are one sequence
 *   out      [n, B, Hq, L, d]  softmax(scale * q k^T) v (float if out_fp32 else dtype).  Of bf16 outputs each weight is rounded to bf16, by up to
 *            2^-8 of it, in front of the product with v; of float ones it is not
 *   row_lse  [n, B, Hq, L]     optional (may be NULL): natural log-sum-exp of each row, as madakv_score_prompt takes it
 * Rows of out and row_lse at positions of no sequence are left as they are, and what k and v hold where a position does not look
 * has no influence on it, whatever it is.  (A caller that has filled row_lse with +infinity has madakv_score_prompt count nothing from the queries of
 * positions of no sequence.)  No workspace. */
int32_t madakv_prompt_attn(madakv_handle* h, int32_t layer0, int32_t n, const void* q, const void* k, const void* v,
                           const int32_t* seq_off, int32_t n_seq, void* out, float* row_lse, void* stream);

/* Eq. 8, Eq. 10-11 for layers [layer0, layer0 + n) in order.
 *   stats    [n, B, H]        from madakv_score
 *   n_mod    [B, M]
 *   budgets  [n, B, H, M] int32  out: candidate tokens to keep per modality ((b_t, b_v) for M = 2);
 *                              their sum over modalities, heads and the whole model is
 *                              exactly n_layers * H * (budget - W) per batch item.
 *                              With mpa_mode = 0 the head total is in slot 0, the others are 0.
 * The remaining pool of each batch item is carried in the handle; layer0 = 0 resets it. */
int32_t madakv_allocate(madakv_handle* h, int32_t layer0, int32_t n,
                        const void* stats, const int32_t* n_mod,
                        int32_t* budgets, void* stream);

/* Per head and modality: keep the b_m candidates with the largest psi_pool (equal scores:
 * lower position first), in ascending position, then the W window positions; copy their
 * K and V rows into the reduced cache.
 *   psi_pool [n, B, H, L-W], mask [B, L], budgets [n, B, H, M] (0 <= b_m <= n_mod[m])
 *   k, v     [n, B, H, L, d]
 *   kept_idx int32, ragged  out: head (l,b,h) owns kept_idx[kv_off .. kv_off + kv_len)
 *   kv_off   [n, B, H] int64 out: first row of the head's segment in k_c / v_c / kept_idx
 *   kv_len   [n, B, H] int32 out: sum of the head's budgets + W
 *   k_c, v_c [capacity_tokens, d]  out: the reduced cache (dtype, or bytes with cache_fp8); a head's segment has kv_len
 *                              rows followed by max_new_tokens free rows
 * Batch item b owns rows [b, b+1) * capacity_tokens / B; inside, layers then heads follow
 * each other.  Budgets from madakv_allocate fill that space exactly.  If hand-made budgets
 * add up to more, the first head that does not fit and every head after it in the batch
 * item get an empty segment (kv_len = 0): nothing is written for them, decode neither
 * appends to them nor produces a finite output for them.  The write cursor per batch item is carried in the handle; layer0 = 0
 * resets it.  The decode-step counters of the layers in the call are reset. */
int32_t madakv_select_gather(madakv_handle* h, int32_t layer0, int32_t n,
                             const float* psi_pool, const uint8_t* mask, const int32_t* budgets,
                             const void* k, const void* v,
                             int32_t* kept_idx, int64_t* kv_off, int32_t* kv_len,
                             void* k_c, void* v_c,
                             void* ws, size_t ws_bytes, void* stream);

/* Sec. 3.3 as a whole (Eq. 7, 6, 9, then Eq. 8, 10, 11, then the per-head, per-modality eviction):
 * madakv_score + madakv_allocate + madakv_select_gather for layers [layer0, layer0 + n) in one call,
 * with the same arguments and the same results bit for bit.  A call over four or more layers is
 * cut into four layer groups: the statistics, allocation and selection of a group run on a side
 * stream while the caller's stream holds the score passes of the next group and the gather of the
 * group before.  Keep-all configurations (budget >= ctx_len) have nothing to score: use
 * madakv_select_gather for them.  score_ws / select_ws: at least what madakv_workspace_bytes
 * reports for n layers. */
int32_t madakv_evict(madakv_handle* h, int32_t layer0, int32_t n,
                     const void* q_win, const void* k, const void* v, const uint8_t* mask,
                     float* psi, float* psi_pool, void* stats, int32_t* n_mod, int32_t* budgets,
                     int32_t* kept_idx, int64_t* kv_off, int32_t* kv_len, void* k_c, void* v_c,
                     void* score_ws, size_t score_ws_size, void* select_ws, size_t select_ws_size, void* stream);

/* One decode step for layers [layer0, layer0 + n): append k_new, v_new to every head's
 * segment (Eq. 4), then out = softmax(scale * q k_c^T) v_c over the head's rows (Eq. 5).
 *   q        [n, B, Hq, d]
 *   k_new, v_new [n, B, H, d]  both NULL = attend only
 *   k_c, v_c, kv_off          as produced by madakv_select_gather
 *   kv_len   [n, B, H]        in/out: the array madakv_select_gather filled (the library sizes
 *                              its launch from the lengths it produced); incremented by the append
 *   out      [n, B, Hq, d]    float if out_fp32 else dtype
 *   ws, ws_bytes               at least what madakv_workspace_bytes reports; the partial results of heads that are cut
 *                              into several pieces go through it
 * INVALID_ARG if a layer in the range has already appended max_new_tokens rows.  Of rows that replays have appended the host does not know: a head
 * whose segment is full stores nothing and attends over the rows it has. */
int32_t madakv_decode_attn(madakv_handle* h, int32_t layer0, int32_t n,
                           const void* q, const void* k_new, const void* v_new,
                           void* k_c, void* v_c, const int64_t* kv_off, int32_t* kv_len,
                           void* out, void* ws, size_t ws_bytes, void* stream);

/* One decode step that keeps an account of the attention it pays (the accumulated weight by which heavy-hitter eviction
 * ranks tokens), and the eviction of one row per step by that account.  Arguments up to out as in madakv_decode_attn; then
 *   acc_in, acc_out [capacity_tokens] float, indexed like the rows of k_c (the same array, or two): for every row r of the
 *            heads in the call acc_out[r] = decay * acc_in[r] + the sum over the G query heads of the weight they pay to r
 *            in this step; of a row that is new in this step the weights alone.  Entries of other rows are left as they are.
 *            What acc_in holds at first is the caller's choice: zeros, or psi of the kept positions.  The sums stay where
 *            they are when a (re-)eviction moves rows.
 *   decay    0 .. 1; 1 = the plain sum
 *   slot_in  [n, B, H] or NULL.  NULL: k_new, v_new are appended as in madakv_decode_attn (or NULL too: attend only).  Else:
 *            they replace row slot_in of the head's segment (0 .. kv_len - 1); the segment keeps its length.  A head whose
 *            entry is no row of it stores nothing in this step and attends over the rows it has.
 *   slot_out [n, B, H] or NULL (may be slot_in): the row with the smallest acc_out among those whose original position is at
 *            most pos - recent (equal sums: the lower row), -1 if there is none: what the next step's slot_in takes.  A
 *            sum that is NaN comes last.
 *   kept_idx, pos  both or neither (slot_out needs them): original positions of the cache's rows, as madakv_select_gather
 *            left them, and the position of this step's token per batch item, [B] int32 on the device.  kept_idx of the new
 *            row becomes pos; rows appended by other calls have none until a re-eviction.
 *   recent   >= 0: the newest tokens that slot_out spares, the one of this step among them
 *   ws       madakv_decode_attn_weights_workspace_bytes(h, n) bytes
 * Once rows have been replaced, a segment is no longer in order of position: madakv_reevict gives
 * MADAKV_ERR_INVALID_ARG for its layer until the next eviction, and for good once a replacing step has been captured, whose
 * replays the host does not see.  Nothing depends on the host from step to step: a
 * captured replacing step can be replayed any number of times (pos is the caller's to advance on the device). */
int32_t madakv_decode_attn_weights_workspace_bytes(const madakv_handle* h, int32_t n_layers_per_call, size_t* bytes);
int32_t madakv_decode_attn_weights(madakv_handle* h, int32_t layer0, int32_t n,
                                   const void* q, const void* k_new, const void* v_new,
                                   void* k_c, void* v_c, const int64_t* kv_off, int32_t* kv_len, void* out,
                                   const float* acc_in, float* acc_out, float decay,
                                   const int32_t* slot_in, int32_t* slot_out,
                                   int32_t* kept_idx, const int32_t* pos, int32_t recent,
                                   void* ws, size_t ws_bytes, void* stream);

/* Attention of several drafted tokens at once (Eq. 5 for the nodes of a tree, each following its parent): every node attends over the rows of the
 * reduced cache and over the nodes that its mask names.  Nothing is stored: madakv_tree_commit does that for the nodes that are accepted.
 *   n_nodes  T, 1 .. 64 (else MADAKV_ERR_BAD_SHAPE)
 *   q        [n, B, Hq, T, d]
 *   k_new, v_new [n, B, H, T, d]  the nodes' rows; they count with the values that the cache would hold of them (cache_fp8), so that a
 *            node's output is what madakv_decode_attn gives for its token behind its ancestors, up to rounding: with out_fp32, and with bf16 outputs while
 *            G * n_nodes <= 64, softmax weights have 16 bits or more, as in that call; with bf16 outputs of larger trees each may be rounded to bf16, by
 *            up to 2^-8 of it, in front of the product with v
 *   tree     [B, T] uint64     bit i of entry t: node t sees node i (its ancestors, and as a rule itself); bits from T on mean nothing.  A node may
 *                              see none
 *   k_c, v_c, kv_off, kv_len   as in madakv_decode_attn; none of them is written
 *   out      [n, B, Hq, T, d]  float if out_fp32 else dtype; not finite for a head with an empty segment
 *   ws       madakv_tree_attn_workspace_bytes(h, n, T) bytes; what it reports serves calls over up to n layers and T nodes */
int32_t madakv_tree_attn_workspace_bytes(const madakv_handle* h, int32_t n_layers_per_call, int32_t n_nodes, size_t* bytes);
int32_t madakv_tree_attn(madakv_handle* h, int32_t layer0, int32_t n, int32_t n_nodes, const void* q, const void* k_new, const void* v_new,
                         const uint64_t* tree, const void* k_c, const void* v_c, const int64_t* kv_off, const int32_t* kv_len,
                         void* out, void* ws, size_t ws_bytes, void* stream);

/* The accepted nodes' rows into the cache (Eq. 4 for several tokens, of every batch item as many as it has accepted).
 *   k_new, v_new [n, B, H, T, d]  as in madakv_tree_attn
 *   path     [B, max_path] int32 on the device: the accepted nodes, in order; an entry that is no node ends the path.  max_path 1 .. 64
 *   n_path   [B] int32 on the device: how many there are (0 .. max_path)
 *   start    [B] int32 on the device: the rows that the heads of the item have behind those that the last (re-)eviction left them, in front of the
 *            accepted ones.  Fewer than a head has: its later rows are taken back.  More, or less than 0: there is a mistake, and the
 *            heads of the item are left as they are.  In a paged cache rows are not taken back: heads that have more rows are left as they are, too
 *   most     the most rows that any head of these layers has behind those of the eviction after the call (0 .. max_new_tokens, else
 *            MADAKV_ERR_INVALID_ARG): accepted rows beyond it are not stored, and contiguous segments with more rows are cut to it.  The host counts `most` rows as
 *            appended (madakv_decode_attn refuses a layer from max_new_tokens on); a caller that does not know the lengths gives an upper bound
 *   kv_len   in/out: the rows that the (re-)eviction left + start + the rows stored
 * A call repeated with the same arguments does the same again.  kept_idx has no entries for these rows until a re-eviction, and their entries in the sums of
 * madakv_decode_attn_weights are the caller's to set.  Segments that are empty, or that this handle has not evicted, are left as they are.
 * A captured call can be replayed any number of times: `most` bounds the rows whatever the path says, and every other call covers the rows that replays may
 * have left, those of an ordinary decode step among them. */
int32_t madakv_tree_commit(madakv_handle* h, int32_t layer0, int32_t n, int32_t n_nodes, const void* k_new, const void* v_new,
                           const int32_t* path, const int32_t* n_path, int32_t max_path, const int32_t* start, int32_t most,
                           void* k_c, void* v_c, const int64_t* kv_off, int32_t* kv_len, void* stream);

/* The rows that the heads of layers [layer0, layer0 + n) hold in an 8-bit or 4-bit reduced cache, as values of dtype:
 *   k_rows, v_rows [capacity_tokens, d]  out: row i holds what row i of k_c / v_c stands for (every value is exact in
 *                  bf16); rows of no head are left as they are
 * For a handle whose cache holds rows of dtype: MADAKV_ERR_UNIMPLEMENTED (k_c and v_c are the rows). */
int32_t madakv_cache_rows(madakv_handle* h, int32_t layer0, int32_t n, const void* k_c, const void* v_c,
                          const int64_t* kv_off, const int32_t* kv_len, void* k_rows, void* v_rows, void* stream);

/* Re-eviction during generation (the paper evicts once, after the prefill, Sec. 3.3; its Sec. 6 leaves long
 * generation open).  After some decode steps every head's segment holds its kept rows, the W window rows and
 * the appended rows.  The call brings each head of layers [layer0, layer0 + n) back to the length the prompt
 * eviction gave it, in place:
 *   - the last W rows of the segment are the new proxy set; q_recent holds their queries;
 *   - every earlier row is a candidate, scored as in Eq. 7 over the rows of the segment (proxy row r sees
 *     the rows up to its own), pooled over neighbouring rows as configured;
 *   - the head's total stays budgets_total = (length after the last (re-)eviction) - W: the layer
 *     compensation of Eq. 9-11 is a prefill decision and is not re-run;
 *   - the total is split over the modalities by the current masses (Eq. 6, Eq. 8, same integer rules as
 *     madakv_allocate; a prompt token has the modality of its position in `mask`, a generated token is text);
 *   - per modality the best-scored candidates survive (equal scores: lower row), in row order, followed by
 *     the W proxy rows; K, V and kept_idx rows move down inside the segment.
 *   q_recent [n, B, Hq, W, d]   queries of the tokens in the last W rows of every segment, oldest first
 *   mask     [B, L]
 *   k_c, v_c, kept_idx, kv_off  as left by madakv_select_gather / madakv_evict and madakv_decode_attn;
 *                               kept_idx entries of generated tokens read ctx_len + (index of the token
 *                               in the generation) afterwards
 *   kv_len   [n, B, H]          in/out: back to its value after the prompt eviction
 *   budgets  [n, B, H, M]       out: the new split
 *   ws                          madakv_reevict_workspace_bytes(h, n) bytes
 * The decode-step counters of the layers are reset: max_new_tokens rows can be appended again.
 * An 8-bit or 4-bit cache is scored by the values it holds and moved as it is stored (4 bits: the workspace holds K as bf16, of the
 * rows that n layers can have).  A paged cache is re-evicted as a whole
 * (layer0 = 0, n = n_layers, else MADAKV_ERR_INVALID_ARG): the survivors end up in the heads' initial pages
 * and every page taken since the eviction goes back to the pools, which all layers share; the work is done
 * on a linear copy of the rows in the workspace (as many rows as the cache holds).
 * MADAKV_ERR_UNIMPLEMENTED with dtype fp32 or segments longer than 64 chunks of the
 * scoring kernel (65536 rows at G * W <= 32, 49152 beyond); MADAKV_ERR_BAD_BUDGET when budget >= ctx_len
 * (nothing was evicted). */
int32_t madakv_reevict_workspace_bytes(const madakv_handle* h, int32_t n_layers_per_call, size_t* bytes);
int32_t madakv_reevict(madakv_handle* h, int32_t layer0, int32_t n,
                       const void* q_recent, const uint8_t* mask,
                       void* k_c, void* v_c, int32_t* kept_idx, const int64_t* kv_off, int32_t* kv_len,
                       int32_t* budgets, void* ws, size_t ws_bytes, void* stream);

/* Paged reduced cache (page_rows > 0): where the rows of a head are.  Rows [0, table[0] * page_rows) of head
 * (l, b, h) sit at kv_off[l, b, h] + r (its initial pages follow each other); row r beyond that sits in page
 * table[1 + (r - table[0] * page_rows) / page_rows] at slot r % page_rows, a page p covering rows
 * [p * page_rows, (p + 1) * page_rows) of k_c / v_c.  *table is a device pointer into the handle (valid
 * until madakv_destroy, NULL without paging) to int32 [n_layers * batch * n_kv_heads][*entries_per_head],
 * head-major in (layer, batch, head) order; madakv_select_gather / madakv_evict write entry 0,
 * madakv_decode_attn the others as pages get taken (from the top of the batch item's region downwards;
 * a new pass starting at layer 0 returns them all). */
int32_t madakv_page_table(const madakv_handle* h, const int32_t** table, int32_t* entries_per_head);

/* madakv_decode_attn for callers that cannot allocate device memory and so have no workspace to
 * pass: code running under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, kernels and results as madakv_decode_attn, without ws: the partial results go to a
 * scratch array of the handle's, of at most MADAKV_STATIC_SCRATCH_BYTES.  The call allocates and frees nothing.
 *   - MADAKV_ERR_WORKSPACE_TOO_SMALL if that might not hold what this launch needs, taken as
 *     (heads in the call) * (chunks of the longest head) * G * (head_dim + 2) * 4 bytes, with
 *     chunks of 256 .. 1024 rows (512 once the call covers >= 1024 heads); the longest head is
 *     taken from what the eviction produced once that has reached the host, from ctx_len +
 *     max_new_tokens before.  One layer of 128 heads of up to 16K rows fits.  Nothing is
 *     enqueued in that case.
 *   - On a stream under graph capture (this call, madakv_decode_attn or madakv_decode_attn_weights) the launch is sized for every
 *     row the segments have room for, so that the captured step can be replayed while the heads
 *     grow; each replay appends a row like a call would, but the library's count of appended rows
 *     only sees the capture itself: the caller must not replay beyond max_new_tokens rows per
 *     head, and takes up eager decode calls again only after a new eviction or re-eviction.  (The calls themselves go by the lengths on
 *     the device and take whatever rows the replays have left: once an appending step or a madakv_tree_commit of a layer has been captured, its launches cover
 *     every row the segments have room for.) */
#define MADAKV_STATIC_SCRATCH_BYTES ((size_t)8 << 20)
int32_t madakv_decode_attn_static(madakv_handle* h, int32_t layer0, int32_t n,
                                  const void* q, const void* k_new, const void* v_new,
                                  void* k_c, void* v_c, const int64_t* kv_off, int32_t* kv_len,
                                  void* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MADAKV_H */
