/*
 * cc.h -- C ABI of the counter-causal refresh-scoring library (libcc.so, gfx950).
 *
 * The library implements the memory-refresh cycle of counter-causal KV-cache
 * eviction (Gould & van den Hengel, "Back from the Future: Key-Value Cache
 * Management by Counter-Causal Surprise"):
 *
 *   cc_score        per-entry surprise scores of the cached tokens (Sec. 3.1):
 *                   attention over the stored keys/values under the
 *                   counter-causal mask, the output projection, the LM head and
 *                   the log-softmax at the cached token id;
 *   cc_select_keep  the k highest-scoring entries of each segment (Sec. 3.2,
 *                   memory refresh: argsort and keep the top J);
 *   cc_compact_kv   gather the kept entries of the KV cache, token ids and
 *                   position ids (Sec. 3.2, memory refresh: K', V', X updates).
 *
 * Conventions shared by every entry point
 *   - Pointers are device pointers unless the name ends in _h (host memory).
 *   - Every call only enqueues work on `stream` (a hipStream_t; NULL is the
 *     default stream) and returns; results are ready when the stream is.
 *     Host arrays (_h) are read before the call returns.
 *   - The caller owns every buffer.  The library allocates no device memory;
 *     scratch space comes from the caller's workspace, whose size the matching
 *     *_workspace query returns (a NULL workspace with size 0 is valid when the
 *     query returned 0).  Small planning tables are copied from host memory
 *     into the workspace on `stream`.
 *   - Arguments are checked on the host before anything is enqueued.  A call
 *     that returns a status other than CC_OK has enqueued nothing and written
 *     nothing.  Faults inside kernels surface at the caller's next
 *     synchronisation.  Token ids outside [0, vocab) and position ids outside
 *     the cache are a caller error with undefined results for that row.
 *   - Element types: CC_BF16 tensors are bfloat16, CC_F32 tensors are float32;
 *     scores are always float32.  Matrices are row-major.
 *   - Calls that share a workspace must be ordered (same stream or synchronised).
 *   - The same call repeats bit for bit.  An entry's results do not depend on the entries beside it
 *     beyond that, except in rounding: attention sums a row's keys in one or two chains (fp32: in
 *     four or eight) by the size of the launch, and the projections of FULL and LAST_LAYER_H cut
 *     their sums by the number of entries.  A sequence scored alone and in a batch can therefore
 *     differ in the last bits, and a selection with it where scores nearly tie.  cc_linear and the LM
 *     head calls on the same rows, selection and compaction do not depend on the batch at all.
 */
#ifndef CC_H
#define CC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum cc_status {
  CC_OK = 0,
  CC_ERR_ARG = 1,          /* a NULL required pointer, a bad enum value, a bad count */
  CC_ERR_SHAPE = 2,        /* inconsistent sizes (e.g. n_heads_q % n_heads_kv != 0) */
  CC_ERR_DTYPE = 3,        /* dtype not valid for this call */
  CC_ERR_WORKSPACE = 4,    /* workspace smaller than the query returned */
  CC_ERR_UNSUPPORTED = 5,  /* a valid problem this library has no kernel for */
  CC_ERR_HIP = 6,          /* the HIP runtime rejected a launch or copy */
  CC_ERR_SCRATCH = 7       /* the call needs more than the static scratch of the
                              allocation-free entry point holds */
} cc_status;

typedef enum cc_dtype { CC_F32 = 0, CC_BF16 = 1 } cc_dtype;

/* Counter-causal mask (Sec. 3.1): position i attends to cache positions j > i of
 * its own sequence (STRICT, the paper's mask).  INCLUSIVE (j >= i) is provided for
 * testing.  A row with no allowed key has a zero attention output. */
typedef enum cc_diag { CC_DIAG_STRICT = 0, CC_DIAG_INCLUSIVE = 1 } cc_diag;

/* LAST_LAYER: the fast single-layer approximation (Sec. 3.1): queries are given,
 * attention runs on the cache's last layer, then W_o and the LM head.
 * FULL: every layer runs with fresh queries from the token embeddings against the
 * stored keys/values of that layer (Sec. 3.1, full counter-causal pass).
 * LAST_LAYER_H: the fast approximation in its exact form (Sec. 3.1, fast single-layer
 * approximation): from the stored activations H entering the last layer, RMSNorm,
 * W_q and RoPE at the original positions, attention on the cache's last layer, the
 * layer's output processing (W_o + residual, RMSNorm, SwiGLU MLP + residual), the
 * final RMSNorm and the LM head.
 * LAST_LAYER_FUSED: LAST_LAYER with W_o folded into the LM head.  With queries given,
 * the output processing of the fast approximation (Sec. 3.1) is the bare projection
 * W_o, so z = W_lm (W_o y) = (W_lm W_o) y: inputs.w_lm holds the product
 * [V][Hq*head_dim] (from cc_fuse_wo_lmhead, once per model) and inputs.w_o is unused.
 * The scores equal LAST_LAYER's up to rounding. */
typedef enum cc_mode {
  CC_MODE_LAST_LAYER = 0,
  CC_MODE_FULL = 1,
  CC_MODE_LAST_LAYER_H = 2,
  CC_MODE_LAST_LAYER_FUSED = 3
} cc_mode;

typedef enum cc_kv_layout { CC_KV_CONTIGUOUS = 0, CC_KV_PAGED = 1 } cc_kv_layout;

/* A view of the KV cache (keys and values share the layout).  head_dim elements of
 * one (layer, KV head, token) are contiguous; strides are in elements.
 *   CONTIGUOUS: element (seq b, layer l, head h, token t, e) is at
 *       base + b*seq_stride + l*layer_stride + h*head_stride + t*tok_stride + e
 *   PAGED: token t of sequence b lives in page block_table[b*max_pages + t/page_size],
 *       slot t % page_size:
 *       base + l*layer_stride + page*page_stride + h*head_stride + slot*tok_stride + e
 * Token t is the t-th cached entry of its sequence in cache order (ascending
 * original position after any number of refreshes). */
typedef struct cc_kv {
  int32_t layout;              /* cc_kv_layout */
  int32_t n_layers;            /* layers held by the cache */
  void* k;                     /* device base of keys */
  void* v;                     /* device base of values */
  int64_t seq_stride;          /* CONTIGUOUS only */
  int64_t layer_stride;
  int64_t head_stride;
  int64_t tok_stride;
  int64_t page_stride;         /* PAGED only: one page spans less than 4 GiB, i.e.
                                  page_stride and page_size*tok_stride, in bytes, are
                                  below 2^32 (CC_ERR_UNSUPPORTED otherwise) */
  const int32_t* block_table;  /* PAGED only: device [n_seqs][max_pages] page ids */
  int32_t page_size;           /* PAGED only: tokens per page, a power of two >= 16 */
  int32_t max_pages;           /* PAGED only: row length of block_table */
} cc_kv;

/* Shape of one refresh.  Sequences are ragged: sequence b holds cache entries
 * [cu_seqlens[b], cu_seqlens[b+1]) of every token-major array (N = cu_seqlens[n_seqs]).
 * With GQA, query head h reads KV head h / (n_heads_q / n_heads_kv). */
typedef struct cc_problem {
  int32_t dtype;               /* cc_dtype of q, k, v and all weights */
  int32_t mode;                /* cc_mode */
  int32_t diag;                /* cc_diag */
  int32_t n_seqs;              /* >= 1 */
  const int32_t* cu_seqlens_h; /* host [n_seqs+1], cu[0] = 0, non-decreasing */
  const int32_t* cu_seqlens_d; /* the same values in device memory */
  int32_t n_heads_q;
  int32_t n_heads_kv;          /* divides n_heads_q */
  int32_t head_dim;            /* 64 or 128 (FULL and LAST_LAYER_H: 128) */
  int32_t hidden;              /* D: model width, rows of W_o (bf16: a multiple of 64) */
  int32_t vocab;               /* V: rows of the LM head */
  int32_t n_layers;            /* FULL only: transformer layers (<= kv.n_layers) */
  int32_t ffn;                 /* FULL, LAST_LAYER_H: SwiGLU width */
  float softmax_scale;         /* 0 selects 1/sqrt(head_dim) (Eq. (2)) */
  float rope_theta;            /* FULL, LAST_LAYER_H: rotary base */
  float rms_eps;               /* FULL, LAST_LAYER_H: RMSNorm epsilon */
  int32_t n_frozen;            /* first n_frozen entries of each sequence are sink
                                  slots that are never evicted (score +inf) */
  int32_t lmhead_packed;       /* bf16 only: 1 = the LM head reads the packed weight
                                  cc_inputs.w_lm_packed (cc_pack_lmhead; cc_inputs.w_lm
                                  is then not read and may be NULL); 0 = row-major w_lm */
} cc_problem;

/* Weights of one transformer layer (FULL, LAST_LAYER_H), device pointers in `dtype`. */
typedef struct cc_layer_weights {
  const void* attn_norm;       /* [D] RMSNorm gain before attention */
  const void* wq;              /* [Hq*d][D] query projection */
  const void* wo;              /* [D][Hq*d] output projection */
  const void* mlp_norm;        /* [D] RMSNorm gain before the MLP */
  const void* w_gate;          /* [F][D] */
  const void* w_up;            /* [F][D] */
  const void* w_down;          /* [D][F] */
} cc_layer_weights;

typedef struct cc_inputs {
  const void* q;               /* LAST_LAYER(_FUSED): [N][Hq][d] queries (already
                                  rotated) */
  cc_kv kv;                    /* LAST_LAYER scores layer kv.n_layers-1; FULL uses
                                  layers 0..n_layers-1 (keys already rotated) */
  const int32_t* token_ids;    /* [N] cached token ids X */
  const int32_t* pos_ids;      /* FULL, LAST_LAYER_H: [N] original positions,
                                  NULL -> 0..n_b-1 */
  const void* w_o;             /* LAST_LAYER: [D][Hq*d] */
  const void* w_lm;            /* [V][D] LM head; LAST_LAYER_FUSED: [V][Hq*d], the
                                  product W_lm W_o.  Not read (may be NULL) when
                                  lmhead_packed = 1 */
  const void* embed;           /* FULL: [V][D] token embeddings */
  const cc_layer_weights* layers_h; /* FULL: host array [n_layers]; LAST_LAYER_H:
                                  host array [1], the last layer's weights */
  const void* final_norm;      /* FULL, LAST_LAYER_H: [D] final RMSNorm gain */
  const void* h_last;          /* LAST_LAYER_H: [N][D] stored activations entering
                                  the last layer (dtype), token-major like ids */
  const void* w_lm_packed;     /* lmhead_packed = 1: the LM head in the packed layout
                                  of cc_pack_lmhead */
} cc_inputs;

/* Human-readable name of a status code (static string). */
const char* cc_status_str(cc_status s);

/* Library build identifier, e.g. "libcc gfx950 <date>". */
const char* cc_version(void);

/* ------------------------------------------------------------------ scoring */

/* Workspace bytes cc_score needs for problem p (sizes only; pointers unused). */
cc_status cc_score_workspace(const cc_problem* p, size_t* bytes);

/* Surprise score of every cached entry (Eq. (5), Sec. 3.1):
 *   scores[i] = logsumexp_v(z_i) - z_i[x_i] = -log P(x_i | x_{i+1..n_b-1}),
 * a strictly decreasing function of P, where z_i are the LM-head logits of entry i
 * after the counter-causal pass.  The last entry of each sequence (no future) and
 * the first n_frozen entries score +inf.  scores: device float32 [N].
 * The [N][V] logits are never materialised. */
cc_status cc_score(const cc_problem* p, const cc_inputs* in, float* scores,
                   void* workspace, size_t workspace_bytes, void* stream);

/* Sub-steps of cc_score, exposed for testing and measurement. */

/* Workspace for cc_attention_cc. */
cc_status cc_attention_workspace(const cc_problem* p, size_t* bytes);

/* Counter-causal attention (Eq. (2) under the mask of Sec. 3.1) over cache layer
 * `layer`: o[i][h][:] = sum_{j allowed} softmax_j(scale * q[i][h].k[j][c]) v[j][c],
 * c = h / g.  q, o: [N][Hq][d] in dtype (o may not alias q). */
cc_status cc_attention_cc(const cc_problem* p, const void* q, const cc_kv* kv,
                          int32_t layer, void* o, void* workspace,
                          size_t workspace_bytes, void* stream);

/* Workspace for cc_lmhead_score. */
cc_status cc_lmhead_workspace(const cc_problem* p, size_t* bytes);

/* LM head, log-softmax and target gather (Eq. (5)): for hidden rows u [N][D]
 * (dtype), scores[i] = logsumexp(W_lm u_i) - (W_lm u_i)[ids[i]], with the
 * last-entry / frozen rule applied.  The target logit is taken from the same
 * accumulators as the log-sum-exp, and a difference that rounding takes below zero is
 * returned as 0 (-log P >= 0).  lse (nullable) receives logsumexp.  This is the
 * log-probability sub-step: log P(x_i | future) = -scores[i] for every finite score. */
cc_status cc_lmhead_score(const cc_problem* p, const void* u, const void* w_lm,
                          const int32_t* token_ids, float* scores, float* lse,
                          void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of the static device scratch behind cc_lmhead_score_noalloc (per GPU). */
#define CC_NOALLOC_SCRATCH_BYTES (32u << 20)

/* cc_lmhead_score without a workspace, for callers that cannot allocate device memory
 * (code under HIP graph capture, tight serving loops, harnesses that forbid allocation).
 * Arguments, results and errors are those of cc_lmhead_score with p->lmhead_packed = 0
 * (a packed problem returns CC_ERR_ARG); the scratch that cc_lmhead_workspace(p) would
 * size -- the per-(vocabulary tile, entry) log-sum-exp partials and the target logits,
 * written in full by every call -- lives in a static device array of
 * CC_NOALLOC_SCRATCH_BYTES that each GPU the library runs on holds until the process
 * ends.  A problem whose cc_lmhead_workspace exceeds it returns CC_ERR_SCRATCH before
 * anything is enqueued (32 MiB covers, e.g., 4096 entries of a 128256-word vocabulary:
 * about 8 B per entry per 256 words).  The call allocates nothing.  Every call on one GPU
 * shares that GPU's array: calls whose execution overlaps on one GPU (two streams, or two
 * host threads) race and must be ordered by the caller. */
cc_status cc_lmhead_score_noalloc(const cc_problem* p, const void* u, const void* w_lm,
                                  const int32_t* token_ids, float* scores, float* lse,
                                  void* stream);

/* Workspace for cc_fuse_wo_lmhead: the transposed W_o. */
cc_status cc_fuse_wo_lmhead_workspace(int32_t dtype, int32_t hidden, int32_t qdim,
                                      size_t* bytes);

/* The weight of mode LAST_LAYER_FUSED: out[v][c] = sum_d w_lm[v][d] w_o[d][c], with
 * w_lm [V][hidden], w_o [hidden][qdim] (qdim = Hq*head_dim) and out [V][qdim], all in
 * dtype (fp32 accumulation, one rounding to dtype).  A one-time weight preparation,
 * not part of a refresh.  bf16 needs hidden % 64 == 0 and 16-byte aligned pointers. */
cc_status cc_fuse_wo_lmhead(int32_t dtype, const void* w_lm, const void* w_o, void* out,
                            int32_t vocab, int32_t hidden, int32_t qdim, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Dense projection y[m][n] = sum_k x[m][k] w[n][k] (x: [M][K], w: [N][K], y: [M][N],
 * all in dtype), the layer's output projection of the fast variant. */
cc_status cc_linear(int32_t dtype, const void* x, const void* w, void* y, int32_t M,
                    int32_t N, int32_t K, void* stream);

/* ------------------------------------------------------------------ FP8 LM head */

/* Workspace for cc_quantize_fp8 on `rows` rows. */
cc_status cc_quantize_fp8_workspace(int64_t rows, size_t* bytes);

/* OCP FP8 E4M3 quantization of x [rows][cols] (dtype): per_row = 1 gives each row its own
 * scale, per_row = 0 one scale for the matrix.  amax = max |x| over the row (matrix),
 * codes = E4M3(x * (448 / amax)) rounded to nearest even, scale = amax / 448, every step
 * in fp32; an all-zero row (matrix) gets codes 0 and scale 0.  x aligned to four
 * elements; codes: device uint8 [rows][cols] (4-byte aligned); scale: device float
 * [rows] (per_row) or [1].
 * cols must be a positive multiple of 4.  A weight preparation for cc_lmhead_score_fp8
 * (the LM head, one scale); not part of the method (the paper fixes no precision). */
cc_status cc_quantize_fp8(int32_t dtype, const void* x, int64_t rows, int32_t cols,
                          int32_t per_row, uint8_t* codes, float* scale, void* workspace,
                          size_t workspace_bytes, void* stream);

/* Workspace for cc_lmhead_score_fp8. */
cc_status cc_lmhead_fp8_workspace(const cc_problem* p, size_t* bytes);

/* cc_lmhead_score on an FP8 LM head: u [N][D] (dtype) is quantized per row into the
 * workspace as in cc_quantize_fp8; w_codes [V][D] are the LM head's E4M3 codes with one
 * device scale w_scale[0]; the logits are z = (sum_d code products) * scale_u * scale_w,
 * accumulated in fp32 on the FP8 matrix cores, and the score follows Eq. (5) as in
 * cc_lmhead_score.  D = p->hidden must be a multiple of 128; w_codes 16-byte aligned. */
cc_status cc_lmhead_score_fp8(const cc_problem* p, const void* u, const uint8_t* w_codes,
                              const float* w_scale, const int32_t* token_ids, float* scores,
                              float* lse, void* workspace, size_t workspace_bytes,
                              void* stream);

/* Bytes of the packed LM-head layout of a bf16 [rows][cols] matrix: rows rounded up
 * to a multiple of 256, times cols, times 2. */
cc_status cc_pack_lmhead_bytes(int64_t rows, int32_t cols, size_t* bytes);

/* Packs a bf16 matrix x [rows][cols] (row stride cols; cols a positive multiple of 32;
 * x 16-byte aligned) into the layout the packed LM head stages: for each 256-row tile
 * and 32-column step, one 16 KB block in which row r (64 bytes at 64r) holds its
 * 16-byte chunk c (columns 8c .. 8c+7 of the step) at chunk position c ^ ((r >> 1) & 3);
 * rows past `rows` are zero.  A bit copy that changes the layout only: the weight
 * preparation for lmhead_packed = 1, made once per model.  out: device, cc_pack_lmhead_bytes bytes, 16-byte aligned,
 * not overlapping x. */
cc_status cc_pack_lmhead(const void* x, int64_t rows, int32_t cols, void* out,
                         size_t out_bytes, void* stream);

/* cc_lmhead_score with p->lmhead_packed = 1: w_packed is w_lm [V][D] packed by
 * cc_pack_lmhead (the row-major weight is not needed).  The result equals
 * cc_lmhead_score (the same sums on another layout of the weight).  Workspace: cc_lmhead_workspace(p). */
cc_status cc_lmhead_score_packed(const cc_problem* p, const void* u, const void* w_packed,
                                 const int32_t* token_ids, float* scores, float* lse,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ selection */

/* Workspace for cc_select_keep with n_segs segments. */
cc_status cc_select_workspace(int32_t n_segs, size_t* bytes);

/* Keep selection (Sec. 3.2): segment s is scores[seg_start_h[s] .. +seg_len_h[s]).
 * Its k = k_h[s] kept entries are the first k under the order (score descending,
 * -0 == +0, NaN below -inf; ties to the lower index), written in ascending order as
 * segment-local indices to keep_idx[off_s .. off_s + k), off_s = sum_{t<s} k_h[t].
 * 0 <= k <= seg_len.  Segments may overlap (e.g. one per KV head over the same
 * per-token scores).  keep_idx: device int32 [sum k]. */
cc_status cc_select_keep(const float* scores, int32_t n_segs, const int64_t* seg_start_h,
                         const int32_t* seg_len_h, const int32_t* k_h, int32_t* keep_idx,
                         void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ compaction */

/* Workspace for cc_compact_kv on a cache of cache_layers layers. */
cc_status cc_compact_workspace(const cc_problem* p, int32_t cache_layers, int32_t per_head,
                               size_t* bytes);

/* KV compaction (Sec. 3.2): for every cache layer, KV head and sequence b,
 *   dst[j] = src[keep[j]] for j < k_b   (a bit copy of head_dim elements),
 * with keep the list from cc_select_keep.  Lists are packed back to back:
 * per_head = 0: one list per sequence (k_h[b]); per_head = 1: one list per
 * (sequence, KV head) in order b*n_heads_kv + h (k_h[b*Hkv+h]).
 * dst is `out` (same geometry as `kv`) or, when out is NULL, `kv` itself (in
 * place; safe because lists are ascending so keep[j] >= j).  token_ids and pos_ids
 * (nullable, device int32 [N], token-major by cu_seqlens) are compacted in place
 * with the first list of each sequence: ids[cu_b + j] = ids[cu_b + keep[j]].
 * Entries at and past k_b are left untouched (paged: pages past ceil(k_b/P) are free
 * for the caller to reuse). */
cc_status cc_compact_kv(const cc_problem* p, const cc_kv* kv, const int32_t* keep_idx,
                        const int32_t* k_h, int32_t per_head, int32_t* token_ids,
                        int32_t* pos_ids, const cc_kv* out, void* workspace,
                        size_t workspace_bytes, void* stream);

/* Workspace for cc_compact_rows. */
cc_status cc_compact_rows_workspace(const cc_problem* p, int32_t row_bytes, int32_t per_head,
                                    size_t* bytes);

/* Compaction of a token-major per-entry array that travels with the cache, such as the
 * stored activations H of the exact fast variant (Sec. 3.1: H is recorded per cache
 * entry, so the memory refresh of Sec. 3.2 keeps the same rows):
 *   rows[cu[b] + j] = rows[cu[b] + keep_b[j]] for j < k_b,
 * with the same keep lists as cc_compact_kv (per_head = 1: the first list of each
 * sequence is used).  rows: device [N][row_bytes] (row_bytes a multiple of 16, rows
 * 16-byte aligned); out_rows NULL compacts in place, else writes out_rows (same shape,
 * no overlap with rows).  A bit copy. */
cc_status cc_compact_rows(const cc_problem* p, void* rows, int32_t row_bytes,
                          const int32_t* keep_idx, const int32_t* k_h, int32_t per_head,
                          void* out_rows, void* workspace, size_t workspace_bytes,
                          void* stream);

/* ------------------------------------------------------------------ cache in 8 bits */

/* A KV cache in 8 bits: OCP E4M3 codes, and for each block of scale_block consecutive
 * entries of one (sequence, layer, KV head) one power-of-two scale, stored as the exponent
 * byte x of the scale 2^(x-127) (E8M0; 0 and 255 are never written and read as 2^-127 and
 * 2^127).  An entry's element is code * scale.
 * `codes` has the fields of a cc_kv, its elements being bytes (strides in bytes, multiples
 * of 16).  The scale of token t is at
 *   CONTIGUOUS: k_scale + b*scale_seq_stride + l*scale_layer_stride + h*scale_head_stride
 *               + t/scale_block
 *   PAGED:      k_scale + l*scale_layer_stride + page*scale_page_stride
 *               + h*scale_head_stride + slot/scale_block
 * (v_scale alike).  scale_block: a power of two from 16 to 128, at most page_size. */
typedef struct cc_kv8 {
  cc_kv codes;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int64_t scale_seq_stride;    /* CONTIGUOUS only */
  int64_t scale_layer_stride;
  int64_t scale_head_stride;
  int64_t scale_page_stride;   /* PAGED only */
  int32_t scale_block;
} cc_kv8;

/* ------------------------------------------------------------------ appending */

/* Rows of new tokens: element (layer l, token i, head h, e) is at
 * base + l*layer_stride + i*tok_stride + h*head_stride + e (strides in elements; rows of
 * head_dim elements are contiguous and 16-byte aligned).  Slices of one fused projection
 * output are such views. */
typedef struct cc_rows {
  const void* base;
  int64_t layer_stride, tok_stride, head_stride;
} cc_rows;

/* What is appended.  The problem's cu_seqlens count the NEW tokens of each sequence (0 is
 * valid), M = cu_seqlens[n_seqs] in all; cached[b] entries are in the cache before. */
typedef struct cc_append {
  cc_rows k, v;                /* [n_layers][M][Hkv][head_dim] in p->dtype */
  cc_rows q;                   /* base NULL: none; [M][Hq][head_dim], n_layers = 1 only */
  void* q_out;                 /* with q: [M][Hq][head_dim] packed, in p->dtype; may be q
                                  itself where q is packed like that */
  const int32_t* cached;       /* device [n_seqs]; negative ones are 0 */
  const int32_t* pos_ids;      /* device [M] original positions, NULL -> cached[b] + i */
  int64_t capacity;            /* entries that a sequence's place in the cache holds.  Paged:
                                  0 selects max_pages * page_size, which is also the limit */
  int32_t layer;               /* first cache layer written */
  int32_t n_layers;            /* layers written, >= 1 */
  int32_t rotate;              /* 1: k and q are rotated (elements e and e + head_dim/2 by
                                  position * rope_theta^(-2e/head_dim)); 0: they are already */
} cc_append;

/* Appends the new tokens' keys and values to a cache in p->dtype, at entries cached[b],
 * cached[b] + 1, ... of each sequence, rotating keys on the way (angles in fp64, the
 * rotation in fp32, one rounding to the cache's type); rotates q into q_out alike.  Tokens
 * at or past the capacity, and those whose page id is negative, are not written.  `cached`
 * is read on the device, so a captured call follows lengths that advance between replays.
 * No other entry is touched.  Sequences must not share pages that are written.  Some 40 million
 * tokens, or 4 million sequences, are the most of a call. */
cc_status cc_append_kv(const cc_problem* p, const cc_append* a, const cc_kv* kv, void* stream);

/* The same into a cache in 8 bits (p->dtype: the type of k, v and q; fp32 values are
 * rounded once).  A block that held no entry gets the smallest scale s = 2^e, e >= -100, with
 * max |x| <= 448 s over its new elements; a block that held some keeps the larger of that
 * and its scale, its entries' codes being rounded again where the scale grows (exact but for
 * elements below 2^-6 of the new scale).  Codes are E4M3(x / s), nearest even; NaN and infinities
 * become NaN codes and do not count for the scale. */
cc_status cc_append_kv8(const cc_problem* p, const cc_append* a, const cc_kv8* kv, void* stream);

/* ------------------------------------------------------------------ compaction in 8 bits */

/* cc_compact_kv on a cache in 8 bits: the kept entries move to the front of their planes.
 * A destination block gets the smallest scale s = 2^e, e >= -100, with max |x| <= 448 s over the
 * kept elements in it (NaN not counted), and their codes are rounded again (exact but for
 * elements below 2^-6 of the new scale; NaN codes stay).  keep_idx, k_h, per_head,
 * token_ids and pos_ids as in cc_compact_kv; `out` NULL compacts in place, else a cache of
 * the same layout, layers and scale_block that does not overlap kv.  Codes past entry k_b
 * and scales past its block are left untouched.  n_layers * n_heads_kv is below 2^20, and with
 * per_head n_heads_kv at most 64.  Needs no workspace. */
cc_status cc_compact_kv8(const cc_problem* p, const cc_kv8* kv, const int32_t* keep_idx,
                         const int32_t* k_h, int32_t per_head, int32_t* token_ids,
                         int32_t* pos_ids, const cc_kv8* out, void* stream);

/* ------------------------------------------------------------------ attention in 8 bits */

/* Which entries a query attends to.  With n_b = kv_lens[b] entries in the cache and m_b
 * queries in the call, query i of a sequence stands at entry n_b - m_b + i (the queries are
 * the last entries).  CAUSAL: entries up to and including its own.  COUNTER_CAUSAL: those
 * after its own (p->diag STRICT) or from its own on (INCLUSIVE).  With more queries than entries
 * the first stand before entry 0: they attend to none (CAUSAL) or to all (COUNTER_CAUSAL).  A
 * query with no entry to attend to has a zero output. */
typedef enum cc_mask { CC_MASK_CAUSAL = 0, CC_MASK_COUNTER_CAUSAL = 1 } cc_mask;

/* Workspace for cc_attention_kv8 (partial results of rows whose entries are shared out). */
cc_status cc_attention_kv8_workspace(const cc_problem* p, int32_t mask, int32_t max_kv_len,
                                     size_t* bytes);

/* Attention over layer `layer` of a cache in 8 bits: o[i][h][:] = sum_j softmax_j(scale *
 * q[i][h] . k[j][c]) v[j][c], c = h / g, over the entries that `mask` allows.  The problem's
 * cu_seqlens count the QUERIES of each sequence; q, o: [N][Hq][head_dim] bf16, packed, not
 * overlapping.  kv_lens: device [n_seqs] entries in the cache (the queries' own among them),
 * read on the device; max_kv_len: host, at least every kv_lens[b] (longer ones are cut there,
 * negative ones are 0), sizes the launch and the workspace.  The pages of a sequence's entries
 * have valid ids; tok_stride is below 2^28.  Entries past kv_lens[b] are not read, and one that
 * a query may not attend to does not reach it, whatever it holds; a NaN code in one that it
 * attends to gives NaN.  Elements are taken in bf16 (exactly, from 2^-126 to below 2^128; those of
 * 2^128 and more, which scales above 2^119 can have, are infinite and make what they reach infinite or NaN).
 * Sums, maxima and outputs are kept in fp32 until the last rounding (weighted sums before the
 * division, of weights up to 2^8: values that take these past fp32 give infinities); the
 * probabilities enter the second product in bf16.  n_seqs * n_heads_kv is below 2^24. */
cc_status cc_attention_kv8(const cc_problem* p, const void* q, const cc_kv8* kv, int32_t layer,
                           int32_t mask, const int32_t* kv_lens, int32_t max_kv_len, void* o,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ log-probabilities */

/* Most alternatives per row of cc_lmhead_logprobs. */
#define CC_LOGPROBS_MAX_TOP 32

/* Workspace for cc_lmhead_logprobs. */
cc_status cc_lmhead_logprobs_workspace(int32_t dtype, int32_t n, int32_t vocab, int32_t hidden,
                                       int32_t top, size_t* bytes);

/* Log-probabilities of the LM head's distribution, row by row: with z = W_lm u_i,
 *   logprob[i] = z[ids[i]] - logsumexp(z),   entropy[i] = -sum_v p_v log p_v,
 *   top_ids[i][0..top) the words of the largest logits, falling (ties: the lower id first),
 *   top_logprob[i][r] = z[top_ids[i][r]] - logsumexp(z).
 * u [n][hidden] and w_lm [vocab][hidden] bf16 (packed = 1: w_lm in the layout of
 * cc_pack_lmhead), hidden a multiple of 64, fp32 accumulation.  0 <= top <= min(vocab,
 * CC_LOGPROBS_MAX_TOP).  logprob and ids (both or neither), entropy, and with top = 0 the top
 * arrays may be NULL.  An id outside [0, vocab), as in the rows that pad a batch, gives a NaN
 * log-probability.  The [n][vocab] logits are never materialised.  A NaN logit ranks below every
 * other (the row's log-probabilities and entropy are then NaN). */
cc_status cc_lmhead_logprobs(int32_t dtype, const void* u, const void* w_lm, int32_t packed, int32_t n,
                             int32_t vocab, int32_t hidden, const int32_t* ids, int32_t top,
                             float* logprob, float* entropy, int32_t* top_ids, float* top_logprob,
                             void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CC_H */
