/*
 * liblfps — the decode-step hot path of LFPS ("Learn from the Past: Fast Sparse Indexing
 * for LLM Decoding") as hand-written HIP kernels for gfx950 (MI355X), behind a C ABI.
 *
 * One decode step of one attention layer, for B requests in GQA form (Hq query heads,
 * Hkv KV heads, G = Hq/Hkv heads per group, head_dim D = 128), with the KV cache resident
 * in device memory:
 *
 *   S1  candidates   previous step's per-head Top-k  ->  sorted candidate positions per KV group
 *   S2  score        q . K_j / sqrt(D) for candidate rows only (all G heads of the group)
 *   S3  select       per query head, the k best candidates  ->  Top-k index set of this step
 *   S4  sparse attn  Softmax over the selected scores, weighted sum of the selected V rows
 *
 * plus two baselines over the whole context: full attention and exact Top-k.
 *
 * Conventions
 *   - Every function returns an int status: LFPS_OK (0) or a negative lfps_status.  Nothing
 *     throws, exits, or synchronises the host (except lfps_create/destroy, lfps_timing_read and
 *     lfps_poll_status, which say so).  After lfps_create no entry point allocates memory.
 *   - All array arguments are DEVICE pointers owned by the caller, unless marked "host".
 *     The context owns only its workspace (candidate scores, split partials, event pool).
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work is
 *     enqueued asynchronously on it, in order.  Use one context per stream at a time.
 *   - Entry points that only enqueue kernels (the S1..S4 calls, lfps_step, the lfps_table_* steps, the
 *     baselines) keep all their state in device memory and may be recorded into a HIP graph; the ones that
 *     synchronise, copy to the host or read events (create/destroy, poll_status, timing_read) may not.
 *   - Positions and counts are int32.  A negative entry in an index array is padding.
 *   - q is fp32 [B, Hq, D].  With an fp16 cache every |q| element must stay below 65504, the fp16 range: an
 *     element beyond it is clamped to +-65504 by the scoring kernels (the scores stay finite but belong to the
 *     clamped query) and LFPS_FLAG_Q_RANGE is raised.
 *     K and V rows are D contiguous elements (bf16, fp16 or fp32); the view
 *     struct gives the element strides between requests, KV heads and rows.
 *   - Argument errors that the host can see (NULL pointers, bad shapes/strides) return
 *     LFPS_EINVAL before anything is launched.  Values that live in device memory (k, seq_lens,
 *     indices) are clamped by the kernels: k_b to [0, max_k], seq_lens to [0, max_seq_len],
 *     index entries outside [0, n_b) are ignored.
 */
#ifndef LFPS_H
#define LFPS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif
#pragma GCC visibility push(default) /* the declarations below are the library's whole export list */

typedef struct lfps_ctx lfps_ctx;

typedef enum {
  LFPS_OK = 0,
  LFPS_EINVAL = -1, /* NULL pointer, unsupported shape/dtype, bad stride */
  LFPS_ECAP = -2,   /* a capacity in lfps_config cannot be met (LDS bitmap, workspace) */
  LFPS_EHIP = -3,   /* HIP runtime error; text via lfps_last_error */
  LFPS_ENOMEM = -4  /* workspace allocation failed in lfps_create */
} lfps_status;

typedef enum { LFPS_F32 = 0, LFPS_BF16 = 1, LFPS_F16 = 2 } lfps_dtype;   /* fp32, bfloat16, IEEE half */

typedef struct {
  int32_t batch;       /* B >= 1; B * Hq <= 65535 */
  int32_t n_q_heads;   /* Hq, a multiple of n_kv_heads; Hq/Hkv must be 1, 2 or 4 */
  int32_t n_kv_heads;  /* Hkv */
  int32_t head_dim;    /* D, must be 128 */
  int32_t kv_dtype;    /* lfps_dtype of the K/V cache */
  int32_t max_seq_len; /* Lcap: rows allocated per (request, KV head); n_b <= Lcap always */
  int32_t max_k;       /* kmax: row length of every Top-k array; k_b <= kmax */
  int32_t radius;      /* r >= 0: positional expansion radius around each predicted position */
  int32_t n_recent;    /* the newest n_recent rows are always candidates (>= 0) */
  int32_t n_sink;      /* the first n_sink rows are always candidates (>= 0) */
  int32_t cand_cap;    /* row length of candidate arrays; 0 = min(Lcap, G*kmax*(2r+2)+n_recent+n_sink), or Lcap in table mode */
  int32_t device;      /* HIP device ordinal */
  int32_t table_mode;  /* 1: also allocate the per-head score tables used by the lfps_table_* entry points */
  float table_decay;   /* gamma of Eq. 10 (the paper's decay factor r = 0.95); table mode needs 0 < gamma < 1 */
  float table_a;       /* a of Eq. 8 (0.2 / 0.3 in the paper); table mode needs a > 0 */
  int32_t k_fp8;       /* 1: K is stored as OCP FP8 E4M3, one byte per element (needs kv_dtype = LFPS_BF16, which then
                          describes V).  The values are used as they are; a dequantisation scale is the caller's to
                          fold into q. */
  int32_t v_fp8;       /* 1: V is stored as OCP FP8 E4M3 as well (needs kv_dtype = LFPS_BF16; a scale of V is a factor
                          on the output rows and the caller's to apply) */
} lfps_config;

/* View of the KV cache.  The struct itself is host memory; k, v, seq_lens and block_table are device
 * pointers.  seq_lens[b] = n_b, the number of valid rows of request b at this step.
 *
 * Contiguous cache (block_table == NULL): element (b, g, i, c) of K is
 *   k[b*stride_b + g*stride_h + i*stride_n + c]
 * (strides in elements, stride_n >= D, rows 16-byte aligned), same for v.  K and V share the element
 * strides also when only one of them is FP8 (cfg.k_fp8, cfg.v_fp8): an FP8 element is one byte.
 *
 * Paged cache (block_table != NULL): k and v are pools of n_blocks blocks of block_size rows, and
 * block_table[b*block_table_stride + i/block_size] names the block that holds row i of request b:
 *   k[block*stride_b + g*stride_h + (i % block_size)*stride_n + c]
 * so stride_b is the distance between blocks.  block_size is a power of two in [1, 65536];
 * block_table_stride*block_size >= max_seq_len; n_blocks*block_size < 2^31.  Table entries are
 * read by the kernels and clamped into [0, n_blocks); only the entries of rows below n_b are read,
 * and the first entry of every request (padding slots read row 0, also when n_b = 0).
 * The method itself (positions, candidates, Top-k indices) always speaks in logical rows i. */
/* Host-resident cache (the paper's placement, Sec. 4 overview: the KV cache in host memory): k and v may also
 * point to pinned host memory that the device can address (hipHostMalloc; pass what lfps_host_device_pointer
 * returns for it).  Every kernel then fetches exactly the rows it touches over the host link: the candidate rows
 * of K once per KV group, the selected rows of V per head; nothing else changes, results are bit-identical to a
 * device-resident cache.  seq_lens and block_table stay in device memory. */
typedef struct {
  const void* k;
  const void* v;
  int64_t stride_b, stride_h, stride_n;
  const int32_t* seq_lens; /* [B] */
  const int32_t* block_table; /* [B, block_table_stride] or NULL */
  int32_t block_size;
  int32_t block_table_stride;
  int32_t n_blocks;
} lfps_kv;

/* The address at which the current device sees a pinned host allocation (hipHostMalloc'ed memory, e.g. a pinned
 * torch tensor): host in, *dev out.  LFPS_EHIP if the memory is not mapped for the device. */
int lfps_host_device_pointer(const void* host, void** dev);

/* Create / destroy.  lfps_create validates the config, selects cfg->device, allocates the
 * workspace (lfps_workspace_bytes) and synchronises the device once.  *out is NULL on error. */
int lfps_create(const lfps_config* cfg, lfps_ctx** out);
int lfps_destroy(lfps_ctx* ctx);
/* Text of the last error on this context (host string owned by the context; "" if none).
 * With ctx == NULL: text of the last failure of a call that takes no context (lfps_create,
 * lfps_workspace_bytes, lfps_sparse_attn_noalloc, lfps_pages_workspace_bytes) in this thread. */
const char* lfps_last_error(const lfps_ctx* ctx);
/* Device bytes lfps_create will allocate for this config (host out-pointer). */
int lfps_workspace_bytes(const lfps_config* cfg, int64_t* out);
/* The candidate row length in effect (cfg.cand_cap or its default). */
int32_t lfps_cand_cap(const lfps_ctx* ctx);

/* S1 — candidate set (Alg. 1 lines 6-7; Eq. 7 and Eq. 9 in their memoryless form).
 * For every (b, g):  C = clip_[0,n_b)( U_{h in g} U_{i in prev_topk[b,h,0:k_b]} {i-r, ..., i+r+1} )
 *                        U {n_b - n_recent, ..., n_b - 1} U {0, ..., n_sink - 1}
 * i.e. the previous Top-k itself (vertical pattern), the same positions shifted by +1 (slash
 * pattern, the direction Eq. 10 moves slash history), each widened by +-r (at r = 1 the offsets
 * are the {-1,0,1,2} of Sec. 4.2 stage 3).  Output is ascending and duplicate-free, hence
 * bit-reproducible.
 *   prev_topk  [B, Hq, kmax] int32, first k_b entries of a row are used, entries outside [0,n_b) ignored
 *   k          [B] int32;  seq_lens [B] int32
 *   cand       [B, Hkv, cand_cap] int32 out (entries past cand_count are left untouched)
 *   cand_count [B, Hkv] int32 out.  If a set would exceed cand_cap it is truncated to its
 *              cand_cap smallest positions and LFPS_FLAG_CAND_OVERFLOW is raised (lfps_poll_status). */
int lfps_candidates(lfps_ctx* ctx, const int32_t* prev_topk, const int32_t* k, const int32_t* seq_lens,
                    int32_t* cand, int32_t* cand_count, void* stream);

/* S2 + S3 — exact dot products over the candidates only, then the k best per query head
 * (Alg. 1 line 8; Sec. 1 Steps 1-2 restricted to the candidate set).
 * score(b,h,j) = q[b,h] . K[b,g(h),cand[b,g,j]] / sqrt(D), fp32 accumulate.
 *   cand, cand_count  as produced by lfps_candidates (ascending positions in [0, n_b)).  An entry outside
 *              [0, n_b) scores -inf: it is taken only when fewer than k_b valid candidates exist, and then
 *              written as -1 (score 0) where it would stand.
 *   topk_idx   [B, Hq, kmax] int32 out: the min(k_b, c) selected positions, ascending; rest -1.
 *              Equal scores at the cut are resolved towards the lower position.
 *   topk_score [B, Hq, kmax] fp32 out or NULL: the score of each selected position (0 for padding)
 *   cand_score [B, Hq, cand_cap] fp32 out or NULL: every candidate's score (parity/debug dump) */
int lfps_score_topk(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* cand,
                    const int32_t* cand_count, const int32_t* k, int32_t* topk_idx, float* topk_score,
                    float* cand_score, void* stream);

/* S4 — sparse attention output (Eq. 1):  out[b,h] = sum_i softmax_i(s_i) V[b,g(h),i],  i in idx[b,h,0:k_b],
 * s_i = q.K_i/sqrt(D).  Negative entries and entries >= n_b are skipped.
 *   idx       [B, Hq, kmax] int32
 *   idx_score [B, Hq, kmax] fp32 scores of those positions, or NULL to recompute q.K from the cache
 *   out       [B, Hq, D] fp32 (zeros for a head with no valid index) */
int lfps_sparse_attn(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* idx,
                     const float* idx_score, const int32_t* k, float* out, void* stream);

/* S4 for callers that cannot allocate device memory (code recorded into a HIP graph, serving loops and harnesses
 * that forbid hipMalloc): the same result as lfps_sparse_attn(ctx, q, kv, idx, NULL, k, out) without a context.
 * Nothing is allocated, by this call or before it: the scores of the selected rows, which lfps_sparse_attn keeps in
 * its context's workspace between its two kernels, go to a static device array of LFPS_NOALLOC_MAX_SCORES floats
 * (8 MiB, held by every GPU the library runs on until the process ends).
 *   cfg   the shapes and cache format as for lfps_create (batch, heads, head_dim, kv_dtype, k_fp8 / v_fp8,
 *         max_seq_len, max_k; the other fields must be valid but are not used); cfg->device must be the
 *         CURRENT device.  batch * n_q_heads * max_k must not exceed LFPS_NOALLOC_MAX_SCORES: LFPS_ECAP otherwise.
 *   q [B, Hq, D], idx [B, Hq, kmax], k [B], out [B, Hq, D]: device pointers owned by the caller, as for
 *         lfps_sparse_attn.
 * Errors are returned as lfps_status; their text is lfps_last_error(NULL) in the calling thread.
 * All calls on one GPU share that GPU's array: two calls that overlap in time on one GPU (different streams or
 * threads) race on it.  The array keeps the previous call's scores; nothing in it needs clearing (every entry
 * that is read has been written by the same call).  The first call on a device looks the array's address up
 * (hipGetSymbolAddress), so make that call outside stream capture. */
#define LFPS_NOALLOC_MAX_SCORES 2097152
int lfps_sparse_attn_noalloc(const lfps_config* cfg, const float* q, const lfps_kv* kv, const int32_t* idx,
                             const int32_t* k, float* out, void* stream);

/* S1..S4 in one call (Alg. 1 lines 6-8 and 10, then Eq. 1): candidates from prev_topk, score,
 * select into topk_idx (this step's index set, the next step's prev_topk), attention into out.
 * S4 reuses S3's scores, so only V rows are gathered.  prev_topk and topk_idx must not overlap.
 *   topk_score [B, Hq, kmax] fp32 out or NULL
 * With a bf16 or fp16 cache the scoring pass keeps, per head, only rows whose score reaches the k-th best
 * score of the PREVIOUS lfps_step call on this context minus a margin (the context remembers one
 * float per head); a head for which that leaves fewer than k rows is rescored without the filter
 * in the same call (by that head's workgroup of the select kernel: no extra launches); a head with so few candidates that
 * filtering would save little keeps them all in the next step.  The result is therefore
 * the same exact Top-k over the candidates whatever the remembered value is; only the time differs.  The first
 * chained step after lfps_create or lfps_reset_history has nothing remembered and takes the unfiltered kernels; that
 * is decided on the host, so a HIP graph captured from such a call replays the unfiltered form: capture a later step.  (A context whose max_k exceeds ~13 000 starts with the
 * filter off: a head's survivors would not fit the select's on-chip list.)  lfps_set_filter(ctx, 0) turns the filter off,
 * lfps_reset_history forgets the remembered scores (e.g. when the context moves to other requests). */
int lfps_step(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* prev_topk, const int32_t* k,
              int32_t* topk_idx, float* topk_score, float* out, void* stream);

/* Baseline: full attention decode, softmax(q K^T / sqrt(D)) V over all n_b rows
 * (Sec. 1 with idx = all; the "full attention" upper bound of Sec. 5).  out [B, Hq, D] fp32. */
int lfps_full_attn_decode(lfps_ctx* ctx, const float* q, const lfps_kv* kv, float* out, void* stream);

/* Baseline: exact Top-k, Sec. 1 Steps 1-2 over all n_b keys (the "exact Top-k" upper bound of
 * Sec. 5): scores every row, selects the k_b best per head.  Outputs as lfps_score_topk.
 * Also the seed of step 0 (the previous Top-k of the first LFPS step).
 * With a 16-bit or FP8-key cache of about a million rows or more (batch * n_kv_heads * max_seq_len) and the score
 * filter on, the scores are not written out and read back: a threshold per head is taken from a scored sample of
 * the rows, one filtered pass over all rows keeps what reaches it, and heads left short are rescored the plain
 * way, so the result is the same exact Top-k either way. */
int lfps_exact_topk(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* k, int32_t* topk_idx,
                    float* topk_score, void* stream);

/* ---- LFPS with score tables: the paper's own candidate rule (Sec. 4.2, Alg. 1 lines 5-9) --------------
 * The context (created with table_mode = 1) keeps, per query head, a vertical and a slash score table over
 * positions.  Sink rows (< n_sink) are outside the tables, as in the paper: always candidates, never
 * counted or updated.  Radius must be <= 30.  Rows appended since the last update enter the tables as zeros. */

/* Eq. 4: tables from the attention weights of the last s = n_queries prefill queries.
 *   q_hist [n_queries, B, Hq, D] fp32, q_hist[j-1] = the j-th most recent query (j = 1: the last one).
 * Query j sees rows [0, n_b - j + 1); w = softmax over the offloaded rows it sees of q.K/sqrt(D);
 *   Phi_ver(i) = 1/(2 s (1 - gamma)) sum_j w_j(i),    Phi_sla(i) = 1/(2 s (1 - gamma)) sum_j w_j(i - j + 1)
 * (the paper uses s = 32).  Two passes over K for every 32 queries (one for a single query); fp32 caches: one scoring
 * pass per query. */
int lfps_tables_init(lfps_ctx* ctx, const float* q_hist, int32_t n_queries, const lfps_kv* kv, void* stream);
/* Set / read the tables as true values per position: phi_ver, phi_sla [B, Hq, max_seq_len], rows
 * [0, seq_lens[b]) used (fp32 in, fp64 out; entries of sink rows and rows >= n_b read as 0). */
int lfps_tables_import(lfps_ctx* ctx, const float* phi_ver, const float* phi_sla, const int32_t* seq_lens,
                       void* stream);
int lfps_tables_export(lfps_ctx* ctx, double* phi_ver, double* phi_sla, const int32_t* seq_lens, void* stream);
/* S1 in table form (Eq. 7, 8, 9): per head the positions whose vertical or slash score exceeds
 * tau = a * mean / kappa of its table, widened by the offsets -r ... r+1 and kept where the vertical or the
 * slash score exceeds the table mean; union over the heads of a KV group, plus the newest n_recent and
 * the n_sink first rows.  Outputs as lfps_candidates. */
int lfps_table_candidates(lfps_ctx* ctx, const int32_t* seq_lens, int32_t* cand, int32_t* cand_count, void* stream);
/* Eq. 10: decay by gamma, slash history moved from i-1 to i, and on the selected positions
 * idx[b,h,0:k_b] (scaled scores idx_score) the softmax weight over the selected set minus 1/(2|C_2|).
 * seq_lens is the length the step saw.  The slash table has room for max_seq_len - 1 updates after an
 * import or init: the call that would exceed it returns LFPS_ECAP, and (for updates replayed from a
 * recorded graph, which the host does not see) the kernel leaves the tables alone and raises
 * LFPS_FLAG_TABLE_FULL.  The table calls keep their state in device memory and may be recorded into a graph. */
int lfps_table_update(lfps_ctx* ctx, const int32_t* idx, const float* idx_score, const int32_t* k,
                      const int32_t* seq_lens, void* stream);
/* Alg. 1 lines 5-9 then Eq. 1: table candidates, exact scores over them, per-head Top-k (fewer than k_b
 * when the candidate set is smaller: padded with -1), sparse attention, table update. */
int lfps_table_step(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* k, int32_t* topk_idx,
                    float* topk_score, float* out, void* stream);

/* ---- Head sparsity estimate and bypass (Sec. 4.2 stage 1, Eq. 5-6, App. B.1; Alg. 1 lines 1-4) ------------
 * Priors of the prefill stage (Sec. 4.2 "Prefilling", last paragraph), from the last prefill query q:
 *   kbar, vbar  [B, Hkv, D] fp32  mean K row / V row over rows [n_sink, n_b)
 *   sigma2_hat  [B, Hq]     fp32  variance over those rows of q.K_i/sqrt(D), divided by |q|^2 */
int lfps_priors(lfps_ctx* ctx, const float* q, const lfps_kv* kv, float* kbar, float* vbar, float* sigma2_hat,
                void* stream);
/* rho[b,h] = w_sink / (w_sink + w_global + w_local)  (Eq. 6) with
 *   w_sink = sum_{i < n_sink} exp(q.K_i/sqrt(D)),  w_local = the same sum over the newest n_local rows (the paper: 6),
 *   w_global = n_b * exp(q.kbar/sqrt(D) + |q|^2 sigma2_hat / 2);   gate[b,h] = rho > eps (the paper: 0.85).
 * rho [B, Hq] fp32 or NULL; gate [B, Hq] int32. */
int lfps_head_sparsity(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const float* kbar, const float* sigma2_hat,
                       int32_t n_local, float eps, float* rho, int32_t* gate, void* stream);
/* lfps_table_step with the bypass in front (Alg. 1 in full): a head with rho > eps outputs vbar[b, g(h)],
 * selects nothing (its topk_idx row is -1), proposes no candidates and keeps its tables as they are.
 * gate_out [B, Hq] int32 or NULL receives the marks. */
int lfps_table_step_gated(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* k, const float* kbar,
                          const float* vbar, const float* sigma2_hat, int32_t n_local, float eps, int32_t* topk_idx,
                          float* topk_score, float* out, int32_t* gate_out, void* stream);

/* ---- Prompts, forks and pages: what brings rows into a cache and shares them ---------------------------------
 * Packed tokens: the new tokens of all requests lie one behind the other in the token arrays; those of request b are
 * cu[b] <= t < cu[b+1] (cu: [B+1] int32, rising), and they are the request's newest: token cu[b] + i is row
 * n_b - (cu[b+1] - cu[b]) + i of its cache, n_b (seq_lens) with the new rows counted in.  A request may have none.  Tokens
 * of no request (in front of cu[0], from cu[B] on) are neither read nor written; a request with more new tokens than rows
 * has its first ones at no row.  n_tokens bounds the arrays: entries of cu are clamped to it. */

/* The newest K and V rows into the cache: k_new, v_new [n_tokens, Hkv, D] of cfg.kv_dtype, element (t, g, c) at
 * t*stride_t + g*D + c (slices of a fused projection; rows 16-byte aligned, stride_t >= Hkv*D).  The cache behind kv is
 * WRITTEN, at the rows named above and nowhere else; tokens at no row are dropped.  FP8 caches: rounded to nearest even,
 * values beyond +-448 and infinities become +-448, NaN stays NaN.  Two requests whose tables name the same block for a row
 * that both append leave either's (lfps_pages_update gives each its own); rows whose entry names no block of the pool are dropped. */
int lfps_append(lfps_ctx* ctx, const void* k_new, const void* v_new, int64_t stride_t, const int32_t* cu,
                int32_t n_tokens, const lfps_kv* kv, void* stream);

/* Causal attention of the new tokens over the cache, their own rows in it included (append first): the token at row p of
 * request b attends rows 0 ... p:  out[t,h] = sum_j softmax_j(q[t,h].K[b,g(h),j]/sqrt(D)) V[b,g(h),j],  j <= p.  One call takes
 * whole prompts (n_b tokens), chunks behind rows that are there already, drafted tokens and single ones, mixed.
 *   q    [n_tokens, Hq, D] of cfg.kv_dtype (bf16 beside FP8 caches), element (t, h, c) at t*stride_t + h*D + c (rows 16-byte
 *        aligned, stride_t >= Hq*D)
 *   out  [n_tokens, Hq, D] of the same type, contiguous, 16-byte aligned; must not overlap q.  A token at no row gets zeros, rows
 *        of tokens of no request are left as they were.
 * Products and sums are fp32; 16-bit types round the weights to 16 bits for the product with V.  n_tokens * Hq <= 2^27. */
int lfps_prompt_attn(lfps_ctx* ctx, const void* q, int64_t stride_t, const int32_t* cu, int32_t n_tokens,
                     const lfps_kv* kv, void* out, void* stream);

/* What stands between the projection and the attention, in one pass: every head of q and k_new is brought to unit mean square,
 *   y_c = x_c / sqrt(mean_c x_c^2 + eps) * weight_c       (weight NULL: y = x),
 * its first rotary_dim channels are turned in pairs by the token's position,
 *   (y_a, y_b) -> (y_a cos x - y_b sin x, y_b cos x + y_a sin x),   x = positions[pair_axis[i]][t] * inv_freq[i]   for pair i = (a, b),
 * and keys and values go into the cache as in lfps_append (which takes keys that are turned already). */
typedef struct {
  const float* q_weight;    /* [D] fp32, 16-byte aligned, or NULL: the query heads are not normed */
  const float* k_weight;    /* the same of the key heads */
  const float* inv_freq;    /* [rotary_dim / 2] fp32: a pair's angle per position */
  const int32_t* pair_axis; /* [rotary_dim / 2]: the row of positions that turns a pair (time, height, width, ...), clamped to n_axes; NULL: row 0 */
  float eps;                /* >= 0 */
  int32_t rotary_dim;       /* a multiple of 16 in [0, D]; channels behind them are not turned */
  int32_t n_axes;           /* rows of positions, 1 to 8; more than one needs pair_axis and positions */
  int32_t interleaved;      /* pair i is the channels 0: i and i + rotary_dim / 2, 1: 2 i and 2 i + 1 */
} lfps_rotary;
/*   q, k_new, v_new  [n_tokens, Hq or Hkv, D] of cfg.kv_dtype, element (t, h, c) at t*stride_t + h*D + c (slices of one fused projection; rows 16-byte
 *              aligned, stride_t >= Hq*D)
 *   positions  [n_axes, n_tokens] int32, any values; NULL: a token's cache row, which is its place in the text as long as no rows were evicted:
 *              after lfps_evict new rows lie below the places at which the kept keys were turned, and positions have to be given
 *   q_out      [n_tokens, Hq, D], contiguous, 16-byte aligned, of q_out_dtype: LFPS_F32 (what the decode steps take: one token a request makes [B, Hq, D])
 *              or cfg.kv_dtype (lfps_prompt_attn, lfps_window_attn).  It must not overlap the inputs.  A token at no row gets zeros, rows of
 *              tokens of no request are left as they were.
 * Norms, angles and turns are fp32, with angles reduced in 64 bits; every value is rounded once, to the type that it is stored in (FP8: as in lfps_append). */
int lfps_rotate_append(lfps_ctx* ctx, const lfps_rotary* rot, const void* q, const void* k_new, const void* v_new, int64_t stride_t,
                       const int32_t* positions, const int32_t* cu, int32_t n_tokens, const lfps_kv* kv, void* q_out, int32_t q_out_dtype,
                       void* stream);

/* lfps_prompt_attn and lfps_full_attn_decode over a sliding window and the first rows: the token at row p sees the rows j <= p with
 * j > p - window (window >= 1: its own row is the last of them) or j < n_sink.  Arguments and roundings else as there (lfps_window_attn of 16-bit types:
 * weights of 16 bits for the product with V, bf16 over FP8 caches; the decode form fp32 throughout); out must not overlap q. */
int lfps_window_attn(lfps_ctx* ctx, const void* q, int64_t stride_t, const int32_t* cu, int32_t n_tokens, const lfps_kv* kv, int32_t window,
                     int32_t n_sink, void* out, void* stream);
int lfps_window_attn_decode(lfps_ctx* ctx, const float* q, const lfps_kv* kv, int32_t window, int32_t n_sink, float* out, void* stream);

/* Accumulated attention weight.  For all rows j < n_b:
 *   mass[b,g,j] = (j < held[b] ? decay * mass[b,g,j] : 0) + sum over the new tokens t of b and the heads h of g of softmax_j(q[t,h].K[b,g,j]/sqrt(D))
 * with the rows that lfps_prompt_attn gives a token (its own and those before).  The tokens may be fewer than were appended last: the newest 32 of a
 * prompt are packed as a call with cu of their own.
 *   held   [B] int32: rows that have a weight already (0 after a prompt's first call, the rows before the new ones later); NULL: none, mass
 *          is written whole.  decay in [0, 1].
 *   mass   [B, Hkv, max_seq_len] fp32, 16-byte aligned; rows from n_b on are left as they were
 * mass must not overlap what is read.  kv->v is not read.  Products and sums are fp32; sums come in the same order every time. */
int lfps_attn_mass(lfps_ctx* ctx, const void* q, int64_t stride_t, const int32_t* cu, int32_t n_tokens, const lfps_kv* kv, const int32_t* held,
                   float decay, float* mass, void* stream);
/* lfps_full_attn_decode that adds its weights up too (q, out [B, Hq, D] fp32; mass as above, the one token of a request being its row n_b - 1).
 * q, out and mass must not overlap. */
int lfps_full_attn_mass_decode(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* held, float decay, float* mass, float* out,
                               void* stream);

/* Eviction: every KV head of request b keeps m_b = min(n_b, budget[b]) of its rows: the first n_sink, the n_recent newest (as far as there is room), and
 * between them those of the largest mass (of equal ones the lower rows; NaN counts as least).  The kept rows move to the front in order: row i of the
 * result is row kept[b,g,i] of K and V.  Keys stay as they were turned: from then on lfps_rotate_append has to be given positions.
 *   mass, mass_out [B, Hkv, max_seq_len] fp32; mass_out[b,g,i] = mass[b,g,kept[b,g,i]]
 *   budget [B] int32, clamped to [0, n_b];  lens_out [B] int32: m_b
 *   kept   [B, Hkv, max_seq_len] int32.  Entries of mass_out and kept from m_b on are left as they were.
 *   to     NULL: in place; K and V of kv are WRITTEN, at rows below m_b that change.  No other request may then have these rows (a shared block
 *          would change for all of them).  Else the view that receives the rows (its k, v, strides, table; its seq_lens are not read): other
 *          slabs, or blocks that no request of kv has, of the same pool too; rows whose table entry names no block are dropped.
 * The calls of several layers read the same lengths: swap lens_out in when all have been made (lfps_pages_update with new_lens = m_b then frees the
 * blocks behind).  Written arrays must not overlap read ones, nor each other. */
int lfps_evict(lfps_ctx* ctx, const lfps_kv* kv, const float* mass, const int32_t* budget, int32_t n_sink, int32_t n_recent, const lfps_kv* to,
               float* mass_out, int32_t* kept, int32_t* lens_out, void* stream);

/* lfps_full_attn_decode for a batch in which groups of requests share their first rows, which are then read once a group.
 *   group_start [n_groups + 1] int32, rising: group i is the requests group_start[i] <= b < group_start[i+1]
 *   prefix_len  [n_groups] int32, clamped to [0, n of the group's first request]: row j < prefix_len[i] of any of them is row
 *               j of the group's first request (as far as the request has rows); what the others' own slabs or tables hold
 *               there is not read.
 *   q, out      [B, Hq, D] fp32.  Rows of out of requests in no group are left as they were.  1 <= n_groups <= B.
 * Requests that share nothing are best one group with a prefix_len of 0: the call is made for few groups of like sizes and prefixes.
 * Over shared rows, products with 16-bit and FP8 rows take the query and the softmax weights as sums of 16-bit terms: to 2^-22 of each
 * (fp16; FP8 keys and values), else the query whole and the weights whole for groups of up to 64 query rows (requests * Hq / Hkv, by
 * the average size), to 2^-18 for larger ones, so the last bits of a result depend on the groups.  Sums are fp32. */
int lfps_prefix_attn_decode(lfps_ctx* ctx, const float* q, const lfps_kv* kv, const int32_t* group_start,
                            const int32_t* prefix_len, int32_t n_groups, float* out, void* stream);

/* Pages.  The state of a paged cache is its block table and lengths (the view's); a block is live if the table names it for a
 * row below some n_b, or if the caller holds it for something else (held [n_blocks] int32, not 0; or NULL).  The calls below
 * read the view's table and lengths and write new ones: swap the two, as the Top-k arrays of two steps.  What a call writes
 * (its results and work) must not overlap what it reads, nor another result.  They compute whole numbers only and plan the copies
 * of rows as a list [.., 3] of (from block, to block, leading rows; -1, -1, 0: none), which lfps_pages_copy carries out in the pool of
 * every layer that shares the table.
 * work: lfps_pages_workspace_bytes(n_blocks) bytes of device memory, 16-byte aligned, that no other call uses meanwhile; nothing
 * in it is kept from one call to the next.  The view must be paged; n_blocks <= 2^24. */
int lfps_pages_workspace_bytes(int32_t n_blocks, int64_t* out);

/* The next step's pages.  For every request b (all of it from the state before the call):
 *   parent [B] int32 or NULL (all continue)   b: continues itself, p: forks request p (p may go on, too), outside [0, B): ends
 *   new_lens [B] int32    its new length, clamped to [0, max_seq_len]: grows (parent's length + new rows), stays, or is cut
 *   table_out [B, block_table_stride], lens_out [B]   entries of rows that it has not are -1
 *   copies [B, 3]         entry b: the copy that request b needs
 * It keeps the parent's blocks as far as it has rows of them.  New blocks are the lowest ones that are not live before the call,
 * dealt to the requests in order, to each first the copy of its last block, then those of its growth.  That copy is made where it
 * will write behind the parent's rows in a block of which others keep rows, or which is held; where all who keep it
 * write into it, the one with the most rows in it (of those, the first) keeps the block itself.  Copy before anything is appended.
 * If the blocks do not suffice, a request gets what is left: lens_out says how many rows it has room for (never fewer than it kept,
 * and nobody's growth reaches rows that another kept) and LFPS_FLAG_PAGES_FULL is raised.  Append no more tokens than it grew by: they
 * are the newest rows of lens_out.  Blocks that this call frees can be had from the next one on. */
int lfps_pages_update(lfps_ctx* ctx, const lfps_kv* kv, const int32_t* parent, const int32_t* new_lens,
                      const int32_t* held, int32_t* table_out, int32_t* lens_out, int32_t* copies, void* work,
                      int64_t work_bytes, void* stream);

/* Moves the live blocks to the front of the pool: with m of them, those numbered m and above go to the free numbers below m, both
 * in rising order.  table_out as above, moves [n_blocks / 2, 3] (the moves first, then empty entries), block_map [n_blocks]
 * (a block's new number; -1: it was free) for the caller's own tables, n_live [1] = m.  Lengths do not change. */
int lfps_pages_compact(lfps_ctx* ctx, const lfps_kv* kv, const int32_t* held, int32_t* table_out, int32_t* moves,
                       int32_t* block_map, int32_t* n_live, void* work, int64_t work_bytes, void* stream);

/* Carries out a list of n copies (device array; entries outside the pool, of no rows or onto themselves are skipped; rows are
 * clamped to the block) in the pools of kv, which are WRITTEN.  For lists of one's own: no block may be written twice, or written
 * and read, in one list. */
int lfps_pages_copy(lfps_ctx* ctx, const lfps_kv* kv, const int32_t* list, int32_t n, void* stream);

/* Switches the score filter of the chained steps on or off (on: only for caches it exists for, bf16 / fp16 / FP8
 * keys; a no-op otherwise).  lfps_reset_history makes every head start without a remembered score. */
int lfps_set_filter(lfps_ctx* ctx, int32_t on);
int lfps_reset_history(lfps_ctx* ctx, void* stream);
/* Copies the candidate counts [B, Hkv] of the last lfps_step call into dst (device, int32),
 * asynchronously on `stream` (for benchmarks: bytes moved per step). */
int lfps_copy_cand_count(lfps_ctx* ctx, int32_t* dst, void* stream);

/* Status flags raised by kernels since the last poll.  Synchronises `stream`, copies the flag
 * word to *flags (host) and clears it. */
#define LFPS_FLAG_CAND_OVERFLOW 1
#define LFPS_FLAG_TABLE_FULL 2      /* a table update was skipped: max_seq_len - 1 updates since the last import / init */
#define LFPS_FLAG_PAGES_FULL 8      /* lfps_pages_update: a request did not get the blocks it wanted (lens_out) */
#define LFPS_FLAG_Q_RANGE 4         /* fp16 cache: a query element beyond +-65504 was clamped to the fp16 range by a
                                       scoring kernel (the scores of that head are those of the clamped query) */
int lfps_poll_status(lfps_ctx* ctx, int32_t* flags, void* stream);
/* Heads that the filtered scoring pass of lfps_step / lfps_table_step left with fewer than k rows (or more than the
 * select's list holds) and that were therefore rescored without the filter, since the last call (host out-pointer;
 * synchronises `stream` and clears the count).  Results do not depend on it: it tells how often the remembered
 * k-th score was of no use (first step after a reset, a sudden change of the query). */
int lfps_poll_rescored(lfps_ctx* ctx, int32_t* n_heads, void* stream);

/* Per-kernel timing for benchmarks.  While enabled, every kernel launch is bracketed by HIP
 * events on the launch stream (at most LFPS_TIMING_MAX_LAUNCHES launches between reads; later
 * ones go untimed).  lfps_timing_read synchronises the stream and writes, for kernel slot i,
 * the summed milliseconds to ms[i] and the number of timed launches to launches[i] (host
 * arrays of LFPS_N_KERNELS), then resets the accumulators. */
enum {
  LFPS_KERNEL_CANDIDATES = 0,   /* steps that find their candidates inside the filter_score launch (but for the longest contexts of large
                                   batches and capacities below the bound; table form up to four million rows) or the
                                   gather_score launch (fp32 caches of up to 8192 rows) count it here too, with next to no time; so
                                   TABLE_CANDIDATES */
  LFPS_KERNEL_GATHER_SCORE = 1,
  LFPS_KERNEL_SELECT = 2,
  LFPS_KERNEL_SPARSE_ATTN = 3,
  LFPS_KERNEL_DENSE_SCORE = 4,
  LFPS_KERNEL_FULL_ATTN = 5,
  LFPS_KERNEL_FULL_MERGE = 6,
  LFPS_KERNEL_HEAD_SCORE = 7,
  LFPS_KERNEL_FILTER_SCORE = 8,
  LFPS_KERNEL_FILTER_SELECT = 9,
  LFPS_KERNEL_TABLE_FLAGS = 10,
  LFPS_KERNEL_TABLE_CANDIDATES = 11,
  LFPS_KERNEL_TABLE_UPDATE = 12,
  LFPS_KERNEL_FILTER_SELECT_ATTEND = 13,   /* S3 + S4 from the filtered pass's survivor lists (chained steps) */
  LFPS_KERNEL_SELECT_ATTEND = 14,          /* S3 + S4 from full score rows (heads the filter left short; unfiltered contexts) */
  LFPS_KERNEL_PROMPT_ATTN = 15,            /* all launches of a call counted as one, here and below */
  LFPS_KERNEL_PREFIX_ATTN = 16,
  LFPS_KERNEL_APPEND = 17,
  LFPS_KERNEL_PAGES_PLAN = 18,
  LFPS_KERNEL_PAGES_COPY = 19,
  LFPS_KERNEL_ROTATE_APPEND = 20,
  LFPS_KERNEL_WINDOW_ATTN = 21,
  LFPS_KERNEL_ATTN_MASS = 22,
  LFPS_KERNEL_EVICT = 23,
  LFPS_N_KERNELS = 24
};
#define LFPS_TIMING_MAX_LAUNCHES 4096
int lfps_timing_enable(lfps_ctx* ctx, int32_t on);
int lfps_timing_read(lfps_ctx* ctx, float* ms, int32_t* launches, void* stream);
const char* lfps_kernel_name(int32_t slot);

/* Plain device-to-device copy of `bytes` bytes (a multiple of 16; both pointers 16-byte aligned),
 * one 16-byte load and store per lane, grid-strided.  Not part of the method: it exists so that
 * hardware memory counters (bytes fetched / written per dispatch) can be scaled against a kernel
 * whose traffic is known exactly. */
int lfps_calib_copy(void* dst, const void* src, int64_t bytes, void* stream);

#pragma GCC visibility pop
#ifdef __cplusplus
}
#endif
#endif /* LFPS_H */
