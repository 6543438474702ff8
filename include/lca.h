/* Latent-Condensed Attention (LCA) for NVIDIA B200 (sm_100a) -- C ABI.
 *
 * The library computes the prefill / decode hot path of LCA: condensation of the distant
 * history in MLA's latent space (query-aware weighted pooling of C^KV, arg-max anchor selection
 * of K^R) followed by attention of the absorbed-form queries [q_latent | q_rope] over the
 * condensed representatives plus the uncondensed local window, and the same dual path for
 * grouped-query attention (pool V, select K).  Section / equation numbers below refer to the
 * paper "Latent-Condensed Transformer for Efficient Long Context Modeling".
 *
 * Conventions that hold for every entry point
 *   - All tensor pointers are DEVICE pointers owned by the caller, 16-byte aligned, dense
 *     row-major with the shapes stated; element type bf16 unless stated.  `lca_params*` is a
 *     HOST pointer.  `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *   - Calls are asynchronous on `stream`; nothing is allocated, freed or kept between calls
 *     unless an entry point says otherwise; the workspace `ws` may be reused by the next call
 *     on the same stream.
 *   - Return value: LCA_OK (0) or a negative lca_status.  Arguments are validated on the host
 *     first; an invalid call launches nothing and writes nothing.
 *   - Token positions are 0-based in the ABI (the paper's formulas are 1-based).
 *
 * Partition of a length-L sequence (Sec. 4.2): m = floor((L-w)/g) groups of g tokens,
 * G_j = {j*g .. (j+1)*g-1}; the last k = L - m*g = w + (L-w) mod g tokens form the local window.
 * When L < w+g there is no group: m = 0, k = L and every entry point degenerates to plain
 * causal attention (Sec. 4.3).  `lca_partition` returns (m, k).
 *
 * Condensed-cache layout (Sec. 4.3 "Decoding and Online Cache Update"), per sequence:
 *   rows 0..m-1   representatives in group order: cache_sem[j] = c_rep_j (Eq. 7, rounded to
 *                 nearest-even bf16), cache_pos[j] = k^R of the anchor token I_j (Eq. 8, bit copy)
 *   rows m..m+k-1 the last k tokens in token order (bit copies)
 * GQA (Sec. 5.4): the same per KV head with cache_sem = pooled V, cache_pos = selected K.
 */
#ifndef LCA_H_
#define LCA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum lca_status {
  LCA_OK = 0,
  LCA_ERR_INVALID_ARG = -1,        /* NULL where a pointer is required, non-positive size, ...   */
  LCA_ERR_UNSUPPORTED_SHAPE = -2,  /* a head dimension / group size no kernel is built for       */
  LCA_ERR_MISALIGNED = -3,         /* a tensor pointer that is not 16-byte aligned               */
  LCA_ERR_WORKSPACE_TOO_SMALL = -4,
  LCA_ERR_CUDA = -5,               /* a CUDA runtime call or a launch failed                     */
  LCA_ERR_DEVICE_TIMEOUT = -6,     /* a bounded device-side wait expired (reported by lca_last_device_status) */
  LCA_ERR_STATIC_SCRATCH_EXCEEDED = -7  /* lca_condense_static_scratch: the problem needs more than LCA_STATIC_SCRATCH_BYTES */
} lca_status;

enum { LCA_VARIANT_MLA = 0, LCA_VARIANT_GQA = 1 };
/* How a group is reduced to one vector (Table 5 ablates these for c_rep and for k^R_rep):
 *   MAXPOOL  element-wise maximum over the g tokens      MEANPOOL  plain mean
 *   WEIGHTED sum_i alpha_i x_i with the Eq. 6 weights    MAXSEL    the vector of the arg-max token (Eq. 8)
 * DEFAULT is the method itself: WEIGHTED for the semantic part (Eq. 7), MAXSEL for the positional part. */
enum { LCA_REDUCE_DEFAULT = 0, LCA_REDUCE_MAXPOOL = 1, LCA_REDUCE_MEANPOOL = 2, LCA_REDUCE_WEIGHTED = 3, LCA_REDUCE_MAXSEL = 4 };
enum { LCA_WS_CONDENSE = 0, LCA_WS_PREFILL = 1, LCA_WS_DECODE = 2, LCA_WS_UPDATE = 3,
       LCA_WS_CONDENSE_VARLEN = 4, LCA_WS_PREFILL_VARLEN = 5 };

/* Problem statement = the REQUIRE line of Alg. 1 (L, C^KV, K^R, Q, w, g) plus the head layout.
 *   MLA: n_kv_heads = 1, d_sem = d_c (512), d_pos = d_R (64); logits use [sem | pos], values = sem.
 *   GQA: d_sem = d_pos = head_dim (128); logits use pos (= K) only, values = sem (= V);
 *        n_q_heads must be a multiple of n_kv_heads.
 *   n_summary_q: number of trailing queries averaged into the summary query (Alg. 1, first step;
 *                Table 8 varies it); 0 means g; clamped to L.
 *   softmax_scale: 1/sqrt(d_h), used for the importance scores (Sec. 4.2) and the attention (Eq. 10).
 *   rep_logit_bias: added to the logit of every representative; 0 = Alg. 1 as printed,
 *                log(g) = the group-size-weighted form analysed in the proof of Theorem 1.
 *   sem_reducer / pos_reducer: 0 = the method (Eq. 7 / Eq. 8); other values reproduce the operators
 *                ablated in Table 5 (lca_condense only; lca_decode_update always uses the method's). */
typedef struct lca_params {
  int32_t variant;
  int32_t batch;
  int32_t seq_len;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t d_sem;
  int32_t d_pos;
  int32_t group_size;
  int32_t window;
  int32_t n_summary_q;
  float softmax_scale;
  float rep_logit_bias;
  int32_t sem_reducer;   /* LCA_REDUCE_*: how lca_condense forms cache_sem[j] (c_rep; GQA: v_rep) */
  int32_t pos_reducer;   /* LCA_REDUCE_*: how it forms cache_pos[j] (k^R_rep; GQA: k_rep).  anchor_idx is always the arg-max token */
} lca_params;

/* (m, k) of Sec. 4.2 for one sequence of p->seq_len tokens.  Host only, no device work. */
int lca_partition(const lca_params* p, int32_t* m, int32_t* k);

/* Bytes of device workspace `which` (LCA_WS_*) needs for these parameters (0 is possible).
 * Returns 0 for invalid parameters as well; the entry point then reports the error. */
size_t lca_workspace_bytes(const lca_params* p, int32_t which);

/* Condensation: Alg. 1 up to the local window (summary query, Eq. 6 group softmax, Eq. 7 pooling, Eq. 8
 * anchors, Eq. 9 local window) for `batch` sequences.
 *   q_tail_sem [B, n, H, d_sem], q_tail_pos [B, n, H, d_pos]: the LAST n = n_summary_q query
 *       positions of each sequence (MLA: q_latent and q_rope; GQA: q_tail_sem = NULL and
 *       q_tail_pos = Q).  q_tail_batch_stride = rows (positions) between consecutive sequences
 *       in these arrays (n for a packed tail, L when pointing into a full [B,L,H,d] tensor).
 *       Ignored (may be NULL) when qbar_opt is given.
 *   qbar_opt   [B, n_kv_heads, dk] fp32, dk = d_sem+d_pos (MLA) or d_pos (GQA), or NULL: a
 *       caller-supplied summary query (e.g. the streaming update of Sec. 4.3).
 *   kv_sem [B, L, n_kv_heads, d_sem], kv_pos [B, L, n_kv_heads, d_pos]: C^KV, K^R (GQA: V, K).
 *   cache_sem [B, m+k, n_kv_heads, d_sem], cache_pos [B, m+k, n_kv_heads, d_pos]: out, layout above.
 *   anchor_idx [B, m, n_kv_heads] int32 out: absolute token index of I_j (lowest index on ties).
 *   scores_opt [B, n_kv_heads, m*g] fp64 out or NULL: the importance scores s_i the kernel used.
 *   ws / ws_bytes: >= lca_workspace_bytes(p, LCA_WS_CONDENSE).
 * The summary query and the importance scores are evaluated in fp64, so the arg-max anchors
 * follow the exact scores (lowest index on exact ties); the group softmax (Eq. 6) and the
 * pooling (Eq. 7) are fp32, and c_rep is rounded once, to bf16 (nearest even). */
int lca_condense(const lca_params* p, const void* q_tail_sem, const void* q_tail_pos,
                 int64_t q_tail_batch_stride, const float* qbar_opt, const void* kv_sem,
                 const void* kv_pos, void* cache_sem, void* cache_pos, int32_t* anchor_idx,
                 double* scores_opt, void* ws, size_t ws_bytes, void* stream);

/* The same condensation for callers that cannot allocate device memory.  (The paper has no
 * counterpart: this entry point exists only for the way the library is called.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- a plug-in inside a serving
 * process whose memory is handed out once at start-up by its own pool, a real-time loop that
 * may not take the allocator's lock, a host thread that is not allowed to synchronise the
 * device (cudaMalloc and cudaFree may do that).  lca_condense needs a few hundred KB of scratch
 * for the summary query; here that scratch is a fixed array of LCA_STATIC_SCRATCH_BYTES that is
 * part of the library image on every GPU that loads it, from load until the process exits.
 *
 * Arguments, results and arithmetic are those of lca_condense without `ws` / `ws_bytes`; the
 * output is bit-identical.  The call allocates nothing and frees nothing.
 *   - Limit: lca_workspace_bytes(p, LCA_WS_CONDENSE) must not exceed LCA_STATIC_SCRATCH_BYTES
 *     (1 MiB: one MLA sequence with up to 128 heads and 64 summary positions uses 0.6 MB; a
 *     batch of 64 such sequences does not fit).  Larger problems return
 *     LCA_ERR_STATIC_SCRATCH_EXCEEDED and launch nothing: use lca_condense with your own buffer.
 *   - The first call on each device looks up the array's device address (the device that is
 *     current at the call).  Make that first call outside any stream capture; later calls on the
 *     same device do no set-up work.
 *   - All calls on one device share the one array, and it keeps whatever the previous call left
 *     there.  Nothing in it has to start at zero: every element a call reads was written earlier
 *     in that same call.  Two calls that may overlap on the GPU (different streams, no
 *     dependency between them) race on the array and give wrong results; order them. */
#define LCA_STATIC_SCRATCH_BYTES (1u << 20)
int lca_condense_static_scratch(const lca_params* p, const void* q_tail_sem, const void* q_tail_pos,
                                int64_t q_tail_batch_stride, const float* qbar_opt,
                                const void* kv_sem, const void* kv_pos, void* cache_sem,
                                void* cache_pos, int32_t* anchor_idx, double* scores_opt,
                                void* stream);

/* Prefill attention, Eq. 10 evaluated at every prefix length (causal): the query at position t
 * attends to the representatives of the m_t = floor((t+1-w)/g) groups that lie wholly outside its
 * window (0 if t+1 < w+g; read from rows 0..m_t-1 of the cache) and to the tokens m_t*g..t
 * (read from kv_sem / kv_pos).  window >= seq_len gives dense causal attention (Eq. 5).
 *   q_sem [B, L, H, d_sem] (MLA; NULL for GQA), q_pos [B, L, H, d_pos]
 *   kv_sem, kv_pos, cache_sem, cache_pos: as for lca_condense (the cache may be NULL when m = 0)
 *   out [B, L, H, d_sem] bf16: softmax-weighted sum of the sem vectors (latent space for MLA)
 *   lse_opt [B, L, H] fp32 or NULL: natural-log sum-exp of the logits of each row
 * fp32 softmax and accumulation, bf16 tensor-core products.  `out` may be aligned to 16 bytes only;
 * where it is aligned to 32 bytes the tensor-core kernels store 32 bytes per instruction. */
int lca_prefill_attention(const lca_params* p, const void* q_sem, const void* q_pos,
                          const void* kv_sem, const void* kv_pos, const void* cache_sem,
                          const void* cache_pos, void* out, float* lse_opt, void* ws,
                          size_t ws_bytes, void* stream);

/* Batches of sequences of different lengths (Alg. 1 takes one L per sequence: a batch is `batch` independent runs,
 * each with its own L_b, m_b = floor((L_b - w)/g) and k_b).  The sequences are packed one after the other, without
 * padding, in every tensor:
 *   q_sem / q_pos  [T, H, d]          T = sum of L_b           kv_sem / kv_pos [T, n_kv_heads, d]
 *   cache_sem / cache_pos [R, n_kv_heads, d]   R = sum of (m_b + k_b), each sequence in the layout stated at the top
 *   anchor_idx [M, n_kv_heads]        M = sum of m_b (token indices count from the start of their own sequence)
 *   out [T, H, d_sem], lse_opt [T, H]
 * seq_lens [batch] is a HOST array of positive lengths; p->seq_len is ignored, except that lca_workspace_bytes(p,
 * LCA_WS_CONDENSE_VARLEN / LCA_WS_PREFILL_VARLEN) sizes the workspace for sequences of at most p->seq_len tokens.
 * lca_varlen_layout fills the prefix sums (batch + 1 entries each, any of them may be NULL): first token row, first
 * cache row and first anchor_idx row of every sequence, totals in the last entry.  Host only.
 * lca_condense_varlen takes the WHOLE packed query tensors and averages the last min(n_summary_q, L_b) positions of
 * each sequence (or uses qbar_opt [batch, n_kv_heads, dk]); it does not return the scores.  Results are those of one
 * call per sequence, bit for bit.  The calls copy a few small tables to the device from pageable host memory, which
 * orders the host behind earlier work of `stream`. */
int lca_varlen_layout(const lca_params* p, const int32_t* seq_lens, int64_t* token_offsets,
                      int64_t* cache_row_offsets, int64_t* group_offsets);
int lca_condense_varlen(const lca_params* p, const int32_t* seq_lens, const void* q_sem, const void* q_pos,
                        const float* qbar_opt, const void* kv_sem, const void* kv_pos, void* cache_sem,
                        void* cache_pos, int32_t* anchor_idx, void* ws, size_t ws_bytes, void* stream);
int lca_prefill_attention_varlen(const lca_params* p, const int32_t* seq_lens, const void* q_sem,
                                 const void* q_pos, const void* kv_sem, const void* kv_pos,
                                 const void* cache_sem, const void* cache_pos, void* out, float* lse_opt,
                                 void* ws, size_t ws_bytes, void* stream);

/* Decode attention (Sec. 4.3): one new query per sequence attends to every valid row of that
 * sequence's condensed cache (the caller has appended the new token's own row).
 *   q_sem [B, H, d_sem] (NULL for GQA), q_pos [B, H, d_pos]
 *   cache_sem [B, cache_row_capacity, n_kv_heads, d_sem], cache_pos likewise with d_pos
 *   cache_rows [B] int32 (device): valid rows of each sequence, clamped to [0, cache_row_capacity]
 *       (the tensor-core kernels fetch whole tiles of 128 rows: rows between cache_rows[b] and the
 *       end of the buffers take no part in the result but must hold finite numbers, e.g. zeros)
 *   n_rep: leading rows that are representatives (they receive rep_logit_bias)
 *   out [B, H, d_sem] bf16, lse_opt [B, H] fp32 or NULL
 * p->seq_len, group_size and window are not used here. */
int lca_decode_attention(const lca_params* p, const void* q_sem, const void* q_pos,
                         const void* cache_sem, const void* cache_pos, const int32_t* cache_rows,
                         int32_t cache_row_capacity, int32_t n_rep, void* out, float* lse_opt,
                         void* ws, size_t ws_bytes, void* stream);

/* Online cache update while decoding (Sec. 4.3 "Decoding and Online Cache Update").  The caller
 * appends the row of every newly generated token after the valid rows of its sequence and counts
 * it in cache_rows[b].  This call then looks at every sequence: when its uncondensed tokens
 * (cache_rows[b] - n_rep[b]) have reached window + group_size, the EARLIEST group_size of them are
 * condensed into one representative with the summary query of the last queries (importance
 * scores as in Sec. 4.2, Eq. 6 softmax, Eq. 7 pooling, Eq. 8 anchor), the representative is
 * written to row n_rep[b], the remaining tokens move up by group_size - 1 rows, n_rep[b] grows by
 * one and cache_rows[b] shrinks by group_size - 1: the cache stays at m + w .. m + w + g - 1 rows
 * in the layout [representatives ; tokens in order].  Sequences below the threshold are untouched.
 *   q_tail_sem / q_tail_pos / q_tail_batch_stride / qbar_opt: the last n_summary_q (0 = g) queries
 *       of each sequence or a ready summary query, exactly as for lca_condense
 *   cache_sem [B, cache_row_capacity, n_kv_heads, d_sem], cache_pos likewise: in / out
 *   n_rep [B], cache_rows [B] int32 (device): in / out
 *   anchor_out [B, n_kv_heads] int32 (device): offset 0..g-1 of the anchor token inside the
 *       condensed group, or -1 where nothing was condensed
 *   ws / ws_bytes: >= lca_workspace_bytes(p, LCA_WS_UPDATE); p->seq_len is not used. */
int lca_decode_update(const lca_params* p, const void* q_tail_sem, const void* q_tail_pos,
                      int64_t q_tail_batch_stride, const float* qbar_opt, void* cache_sem,
                      void* cache_pos, int32_t cache_row_capacity, int32_t* n_rep,
                      int32_t* cache_rows, int32_t* anchor_out, void* ws, size_t ws_bytes,
                      void* stream);

/* ---- Ring layout of the decode cache -------------------------------------------------------
 * Sec. 4.3 fixes what the cache holds while decoding (the m representatives and the most recent
 * tokens) and how a group is condensed, not where the rows live.  In the packed layout above the
 * representatives are followed by the tokens in order, so every update moves the whole window up
 * by group_size - 1 rows.  In the ring layout nothing moves:
 *   rows [0, R), R = window + group_size: the uncondensed tokens; token number n of the sequence
 *                (0-based, counted from the start of the sequence) is at row n % R
 *   rows [R, R + n_rep[b]): the representatives in group order
 * State per sequence: n_rep[b] and n_tok[b] (tokens of the sequence so far); the uncondensed tokens
 * are n_rep[b]*group_size .. n_tok[b]-1, at most R of them (and, once a sequence has representatives,
 * at least `window` of them: the state lca_ring_from_packed and every update leave; with fewer, ring rows
 * of condensed tokens would be attended to).  The caller writes the row of a new
 * token at row n_tok[b] % R and then counts it in n_tok[b].  window must be a multiple of group_size
 * (groups leave the ring whole), ring_row_capacity >= R + the representatives the sequence will have;
 * buffers are [B, ring_row_capacity, n_kv_heads, d_sem | d_pos].  Rows that hold nothing yet must hold
 * finite numbers (e.g. zeros), as for lca_decode_attention.
 *
 * lca_ring_from_packed: the step from a packed cache (lca_condense output, or a packed decode cache)
 * to the ring layout: representatives to rows R.., token i of the packed tail to row
 * (n_rep[b]*group_size + i) % R, n_tok_out[b] = n_rep[b]*group_size + packed_rows[b] - n_rep[b].
 *   packed_rows [B], n_rep [B] int32 (device); packed_sem / packed_pos [B, packed_row_capacity, ...].
 *   A sequence with more than R packed tokens, or more representatives than fit behind the ring, is
 *   truncated to what fits (the caller sizes the buffers; nothing is written out of bounds). */
int lca_ring_from_packed(const lca_params* p, const void* packed_sem, const void* packed_pos,
                         const int32_t* packed_rows, const int32_t* n_rep, int32_t packed_row_capacity,
                         void* ring_sem, void* ring_pos, int32_t ring_row_capacity, int32_t* n_tok_out,
                         void* stream);

/* lca_decode_attention over the ring layout: the query attends to the n_rep[b] representatives (each
 * with rep_logit_bias) and to the uncondensed tokens n_rep[b]*g .. n_tok[b]-1 (the caller has written
 * and counted the new token's own row).  Ring rows that still hold tokens of an already condensed
 * group are left out.  Same arithmetic, outputs and workspace (LCA_WS_DECODE) as lca_decode_attention;
 * n_rep, n_tok [B] int32 (device). */
int lca_decode_attention_ring(const lca_params* p, const void* q_sem, const void* q_pos,
                              const void* ring_sem, const void* ring_pos, const int32_t* n_rep,
                              const int32_t* n_tok, int32_t ring_row_capacity, void* out, float* lse_opt,
                              void* ws, size_t ws_bytes, void* stream);

/* lca_decode_update over the ring layout: a sequence with window + group_size uncondensed tokens has
 * its earliest group (ring rows (n_rep[b]*g) % R .. +g-1) condensed exactly as in lca_decode_update;
 * the representative is written to row R + n_rep[b] and n_rep[b] grows by one.  No other row and no
 * other counter changes (n_tok is read only).  A sequence whose representative region is full
 * (R + n_rep[b] == ring_row_capacity) is left alone, anchor_out = -1.
 * Summary-query arguments, anchor_out and workspace (LCA_WS_UPDATE) as for lca_decode_update. */
int lca_decode_update_ring(const lca_params* p, const void* q_tail_sem, const void* q_tail_pos,
                           int64_t q_tail_batch_stride, const float* qbar_opt, void* ring_sem,
                           void* ring_pos, int32_t ring_row_capacity, int32_t* n_rep, const int32_t* n_tok,
                           int32_t* anchor_out, void* ws, size_t ws_bytes, void* stream);

/* The update on the ring layout with a running summary query, called once per decode step after the
 * step's token has been written and counted (Sec. 4.3: an update scores with the mean of the last g queries):
 *   1. qsum[b, hk, :] += sum over the query heads of KV head hk of this step's [q_sem | q_pos] (fp64;
 *      MLA: dk = d_sem + d_pos, GQA: dk = d_pos), qcount[b] += 1;
 *   2. every sequence that is due (window + group_size uncondensed tokens) is condensed exactly as by
 *      lca_decode_update_ring with the summary query qsum / (qcount * heads per KV head), i.e. the mean of
 *      the queries of all steps since its previous update (the last group_size queries when this is
 *      called at every step), and its qsum and qcount are cleared.
 * No query tail is re-read: a step costs the bytes of that step's queries.
 *   q_sem [B, H, d_sem] (NULL for GQA), q_pos [B, H, d_pos]: this step's queries
 *   qsum [B, n_kv_heads, dk] fp64, qcount [B] int32 (device, in / out): zero them when a sequence
 *        starts; to include queries of the prefill, call this with them before decoding starts (a
 *        sequence that is not due only accumulates)
 *   the other arguments as for lca_decode_update_ring; p->n_summary_q must be 0 or group_size. */
int lca_decode_step_update_ring(const lca_params* p, const void* q_sem, const void* q_pos, double* qsum,
                                int32_t* qcount, void* ring_sem, void* ring_pos, int32_t ring_row_capacity,
                                int32_t* n_rep, const int32_t* n_tok, int32_t* anchor_out, void* ws,
                                size_t ws_bytes, void* stream);

/* ---- Paged 8-bit cache ----------------------------------------------------------------------
 * The decode cache of many sequences in one pool of pages, each row element held in 8 bits (e4m3) with one
 * fp32 scale for each (page, KV head): value = code * scale.  Scales are positive, from 2^-100 (the attention takes smaller
 * ones of values as that) to 2^120; they need not be powers of two.
 *
 * Rows are addressed by position, so nothing moves when a group is condensed: token number n of a sequence is
 * row n; representative j is row j, which belonged to a token condensed long before (n_rep <= n_rep * group_size).
 * Of the row space of a sequence with n_rep representatives and n_tok tokens the rows
 *     [0, n_rep)   and   [n_rep * group_size, n_tok)
 * are present; lca_condense's [representatives ; tokens] order is exactly this order without the gap.  A cache that
 * is never condensed is the case n_rep = NULL (no representatives, rows [0, n_tok)).
 * Row x is on page block_table[b][x / page_size], at place x % page_size.  An entry outside [0, n_pages) (for
 * instance -1) is no page: its rows take no part.  With n_rep, group_size must be a multiple of page_size, so that
 * tokens and representatives never share a page. */
typedef struct lca_paged8 {
  void* pages_sem;        /* [n_pages, n_kv_heads, page_size, d_sem] e4m3 codes: latents (GQA: V) */
  void* pages_pos;        /* [n_pages, n_kv_heads, page_size, d_pos] e4m3 codes: rope keys (GQA: K) */
  float* scale_sem;       /* [n_pages, n_kv_heads]: scale of pages_sem (MLA: of both, the logit is one sum) */
  float* scale_pos;       /* [n_pages, n_kv_heads]: GQA scale of pages_pos; MLA: NULL */
  int32_t* block_table;   /* [batch, table_width] */
  int32_t n_pages;        /* pages of the pool; n_pages * page_size < 2^31 */
  int32_t page_size;      /* 16, 32, 64 or 128 rows */
  int32_t table_width;    /* entries per sequence; table_width * page_size and batch * table_width < 2^31.
                           * Rows behind the table are absent */
} lca_paged8;             /* a HOST structure of device pointers; pages 16-byte aligned */

/* Block tables, free list and slot maps on the GPU, from the lengths of the requests.  The caller states how many
 * representatives and tokens every sequence is to hold; the call compares that with what it holds, gives back the
 * pages that no present row needs any more, takes pages for new rows from the free list and names the slot of every
 * new row.  Growth, condensation (n_rep grows), rollback of rejected tokens (n_tok shrinks) and the end of a request
 * (n_rep = n_tok = 0) are the same call.
 *   n_rep (or NULL: 0), n_tok [batch] int32: target state.  A target must satisfy n_rep * group_size <= n_tok and
 *       fit the table; n_rep does not shrink except to 0 together with n_tok
 *   held_rep (NULL with n_rep), held_tok [batch] int32, in / out: what the tables cover now (0 at first)
 *   cache->block_table in / out: entries that no present row needs become -1; only block_table, n_pages, page_size and
 *       table_width of `cache` are used
 *   free_pages [n_pages] int32, n_free [1] int32, in / out: stack of free pages.  Pages given back are pushed in
 *       descending (sequence, entry) order, pages taken are popped in ascending order: taking and giving back the same
 *       pages leaves the stack as it was
 *   slot_map [n_rows] int32 out (NULL: not wanted): slot = page * page_size + place of every new row: of each sequence
 *       the representatives [held_rep, n_rep), then the tokens [max(held_tok, n_rep * group_size), n_tok).
 *       rows_per_seq = 0: packed, sequence after sequence; rows_per_seq = s > 0: sequence b starts at b * s.
 *       Entries of no row are -1
 *   row_offsets [batch + 1] int32 out: first new row of each sequence in the packed order (may be NULL when no packed
 *       slot_map is wanted)
 *   status [1] int32 out: 0; k > 0: k pages are missing; -1: a target (or the held state) is not valid; -2: slot_map
 *       is too small.  Unless it is 0 nothing has changed, and all slots are -1
 * Uses batch and group_size of p.  Needs no workspace. */
int lca_page_update(const lca_params* p, const lca_paged8* cache, const int32_t* n_rep, const int32_t* n_tok,
                    int32_t* held_rep, int32_t* held_tok, int32_t* free_pages, int32_t* n_free, int32_t* slot_map,
                    int32_t n_rows, int32_t rows_per_seq, int32_t* row_offsets, int32_t* status, void* stream);

/* Writes rows into the paged cache.
 *   rows_sem [n_rows, n_kv_heads, d_sem], rows_pos [n_rows, n_kv_heads, d_pos] bf16
 *   slot_map [n_rows] int32: slot of every row; a negative one (or one behind the pool) is skipped
 * Rows are appended: the rows of one page come together, in the order of their places, and a page is first written at
 * place 0, which sets its scale anew (so a page needs no clearing between owners).  Two rows with the same slot, or two
 * separate runs of rows for one page, in one call leave that page undefined.
 * Scale of a block (page, KV head): the smallest power of two with max|x| <= 448 * scale over the finite elements (MLA:
 * over latent and rope key together) of every row written since place 0 of its page, at least 2^-100.  A later row with a larger
 * element raises the scale; the rows the block holds already are then rounded again, which is exact except where a code
 * falls below the normal range.  Rows taken back by lca_page_update count too: what a large element in a rejected token did to
 * the scale and to the rows before it on that page is not undone, and a row appended in its place uses that scale.  Write
 * tokens once they are accepted where that matters.
 * Codes are rounded to nearest even; infinities become +-448 * scale, NaN stays NaN.
 * Of `cache` the pages, scales, n_pages and page_size are used, of p variant, n_kv_heads, d_sem and d_pos. */
int lca_paged8_write(const lca_params* p, const lca_paged8* cache, const void* rows_sem, const void* rows_pos,
                     const int32_t* slot_map, int64_t n_rows, void* stream);

/* Decode attention over the paged cache (Sec. 4.3): q_len new tokens per sequence attend to the present rows.
 *   q_sem [B, q_len, H, d_sem] (NULL for GQA), q_pos [B, q_len, H, d_pos] bf16
 *   n_rep (or NULL), n_tok [B] int32 (device): state of each sequence, the rows of the q_len tokens included; values
 *       outside the table are clamped to it
 *   out [B, q_len, H, d_sem] bf16, lse_opt [B, q_len, H] fp32 or NULL
 * The q_len tokens are the last ones of their sequence: query i sees the present rows below n_tok - q_len + 1 + i.
 * Representatives get rep_logit_bias.  A query that sees no row (an empty sequence, fewer tokens than q_len) gives
 * out = 0 and lse = -inf.  What absent rows and unused pages hold does not matter; a NaN in a present row reaches every
 * query of that sequence and KV head that sees the row, and through its value those of the q_len that do not see it may become NaN too.
 * Products on the tensor cores with queries and softmax weights as sums of two 8-bit terms: a query element is exact to
 * 2^-17 of the largest of its row, a weight to 2^-8 of itself or to a step of 2^-17 of the largest weight, whichever is more; weights
 * near that step are rounded with offsets spread evenly over the rows, so that many of them keep their sum, whatever
 * the period of the values, to a few dozen steps.  fp32 softmax and sums, one rounding to bf16.  Results do not depend on anything
 * but the arguments (no atomics).
 * ws / ws_bytes: lca_paged8_workspace_bytes. */
size_t lca_paged8_workspace_bytes(const lca_params* p, const lca_paged8* cache, int32_t q_len);
int lca_decode_attention_paged8(const lca_params* p, const lca_paged8* cache, const void* q_sem, const void* q_pos,
                                int32_t q_len, const int32_t* n_rep, const int32_t* n_tok, void* out, float* lse_opt,
                                void* ws, size_t ws_bytes, void* stream);

/* Online update (Sec. 4.3) over the paged cache: every sequence with at least window + group_size uncondensed tokens
 * (n_tok - n_rep * group_size) has its earliest group condensed, with the arithmetic of lca_decode_update on the values
 * the cache stands for.  The call reads the cache and returns the representative; nothing is written to the pages:
 * pass n_rep_new to lca_page_update (it gives back the group's pages and names the slot of the representative) and the
 * rows to lca_paged8_write.
 *   q_tail_sem / q_tail_pos / q_tail_batch_stride / qbar_opt: summary query, as for lca_decode_update
 *   n_rep, n_tok [B] int32; n_rep_new [B] int32 out (another array): n_rep + 1 where a group was condensed, else n_rep
 *   rep_sem [B, n_kv_heads, d_sem], rep_pos [B, n_kv_heads, d_pos] bf16 out: rows of sequences that are not due are
 *       left as they are
 *   anchor_out [B, n_kv_heads] int32: offset 0..g-1 of the anchor token, -1 where nothing was condensed
 * A sequence whose group is not wholly on pages is left alone.  ws: LCA_WS_UPDATE. */
int lca_decode_update_paged8(const lca_params* p, const lca_paged8* cache, const void* q_tail_sem,
                             const void* q_tail_pos, int64_t q_tail_batch_stride, const float* qbar_opt,
                             const int32_t* n_rep, const int32_t* n_tok, int32_t* n_rep_new, void* rep_sem,
                             void* rep_pos, int32_t* anchor_out, void* ws, size_t ws_bytes, void* stream);

/* ---- Paged 4-bit cache ----------------------------------------------------------------------
 * The paged cache with each row element held in 4 bits, about half of the 8-bit cache's bytes (MLA 512 + 64: 298 a row, 8 KV heads
 * of 128: 1072 instead of 2048).  Row space, pages, block tables and counters are those of lca_paged8, and lca_page_update manages
 * them: pass it an lca_paged8 with the same block_table, n_pages, page_size and table_width (it uses nothing else).
 *
 *     value = code * 2^(exponent of its row and KV head - shift of its block of 32 columns)
 *   code      a sign and a magnitude 0, 1/2, 1, 3/2, 2, 3, 4 or 6 (index 0..7).  Eight codes fill a little-endian 32-bit word: value
 *             i has its magnitude's index in bits 4 i .. 4 i + 2 and its sign in bit 8 i + 7 (i < 4) or 8 (i - 4) + 3
 *   exponent  a byte, 127 more than the exponent: 33 (-94) to 253 (126); smaller ones are taken as 33.  MLA: latent and rope key
 *             share it, the logit is one sum
 *   shift     four bits, 0 to 14; 15: the values of the block are NaN.  Two blocks to a byte, the first in the low half */
typedef struct lca_paged4 {
  void* pages_sem;        /* [n_pages, n_kv_heads, page_size, d_sem / 2] bytes: latents (GQA: V) */
  void* pages_pos;        /* [n_pages, n_kv_heads, page_size, d_pos / 2] bytes: rope keys (GQA: K) */
  uint8_t* shift_sem;     /* [n_pages, n_kv_heads, page_size, d_sem / 64] */
  uint8_t* shift_pos;     /* [n_pages, n_kv_heads, page_size, d_pos / 64] */
  uint8_t* exp_sem;       /* [n_pages, n_kv_heads, page_size] */
  uint8_t* exp_pos;       /* [n_pages, n_kv_heads, page_size]; MLA: NULL */
  int32_t* block_table;   /* [batch, table_width] */
  int32_t n_pages;        /* as in lca_paged8 */
  int32_t page_size;
  int32_t table_width;
} lca_paged4;             /* a HOST structure of device pointers; pages, shifts and exponents 16-byte aligned */

/* Writes rows into the paged cache.  Arguments as for lca_paged8_write; but rows do not depend on one another, so they may come in
 * any order and any number to a page, and a row is replaced by writing its slot again.  Two rows with the same slot in one call leave
 * that row undefined.
 * Scale of a block: the smallest power of two with max|x| <= 6 * scale over its finite elements.  The row's exponent is that of
 * its largest block, at least -94 (MLA: over latent and rope key together), and no block is given less than 2^-14 of the row's scale.
 * Codes are the nearest ones, ties to the even index; infinities become +-6 * scale; a NaN makes its block NaN. */
int lca_paged4_write(const lca_params* p, const lca_paged4* cache, const void* rows_sem, const void* rows_pos,
                     const int32_t* slot_map, int64_t n_rows, void* stream);

/* The values of rows of the cache, in bf16, exact but for those of 2^128 and more, which are infinity: codes that elements from 7/8 of 2^128 on, or
 * infinities beside elements above 3/4 of it, were rounded to.
 *   slot_map [n_rows] int32: slot of every row wanted, in any order, the same one any number of times
 *   rows_sem [n_rows, n_kv_heads, d_sem], rows_pos [n_rows, n_kv_heads, d_pos] bf16 out: rows whose slot is negative or behind
 *       the pool are left as they are */
int lca_paged4_read(const lca_params* p, const lca_paged4* cache, void* rows_sem, void* rows_pos, const int32_t* slot_map,
                    int64_t n_rows, void* stream);

/* Decode attention over the paged 4-bit cache: lca_decode_attention_paged8 on the values that this cache stands for, with the same
 * arguments and the same treatment of absent rows, of queries that see no row and of NaN.  The cached values enter the products
 * exactly; queries and weights are sums of two 8-bit terms as there: a weight to 2^-9 of itself or to a step of 2^-18 of the largest; MLA
 * 512 + 64 with more than 64 rows (q_len * n_q_heads): 2^-8 and 2^-17. */
size_t lca_paged4_workspace_bytes(const lca_params* p, const lca_paged4* cache, int32_t q_len);
int lca_decode_attention_paged4(const lca_params* p, const lca_paged4* cache, const void* q_sem, const void* q_pos,
                                int32_t q_len, const int32_t* n_rep, const int32_t* n_tok, void* out, float* lse_opt,
                                void* ws, size_t ws_bytes, void* stream);

/* Online update over the paged 4-bit cache: lca_decode_update_paged8 on the values that this cache stands for. */
int lca_decode_update_paged4(const lca_params* p, const lca_paged4* cache, const void* q_tail_sem,
                             const void* q_tail_pos, int64_t q_tail_batch_stride, const float* qbar_opt,
                             const int32_t* n_rep, const int32_t* n_tok, int32_t* n_rep_new, void* rep_sem,
                             void* rep_pos, int32_t* anchor_out, void* ws, size_t ws_bytes, void* stream);

/* ---- Rotary positions -----------------------------------------------------------------------
 * The attention calls take queries and keys that carry their positions (q_pos, kv_pos; GQA: the whole head).  This call rotates
 * them, from the layout that a projection leaves them in: for each token t, head and pair i of columns
 *     (a, b) -> factor * (a cos - b sin, a sin + b cos) of the angle  positions[t] * freqs[i]
 * Pairs are columns (2 i, 2 i + 1) where `interleaved`, else (i, i + rot_dim / 2).  Columns behind the first rot_dim are copied as they are
 * (not multiplied by `factor`).  With `inverse` the angle is negated: that is also the gradient of the call.  Angles and their whole
 * turns are taken in 64 bits, what is left of half a turn, its cosine and sine (to 2^-22) and the products in fp32; rounded once. */
enum { LCA_DTYPE_BF16 = 0, LCA_DTYPE_FP32 = 1 };
typedef struct lca_rope_args {
  int32_t dtype;              /* of q, k and the outputs */
  int32_t interleaved;        /* 0 or 1 */
  int32_t inverse;            /* 0 or 1 */
  int32_t n_q_heads, n_k_heads;
  int32_t head_dim;           /* columns of a head */
  int32_t rot_dim;            /* even, 2 to min(head_dim, 8192): the first columns of a head */
  float factor;
  int64_t n_tokens;
  const int32_t* positions;   /* [n_tokens] */
  const double* freqs;        /* [rot_dim / 2] on the device (lca_rope_frequencies) */
  /* Element (token, head, column) of a tensor is at token * token_stride + head * head_stride + column, in elements.  Tensors need
   * only their element's alignment; 16-byte aligned rows and rot_dim a multiple of 16 are fast.  An output may be its input (same
   * address and strides); otherwise no output overlaps an input, its own or the other one, or the other output, nor do the heads of
   * an output overlap.  Either of q and k may be NULL (its output too). */
  const void* q; int64_t q_token_stride, q_head_stride;
  void* q_out; int64_t q_out_token_stride, q_out_head_stride;
  const void* k; int64_t k_token_stride, k_head_stride;
  void* k_out; int64_t k_out_token_stride, k_out_head_stride;
} lca_rope_args;              /* a HOST structure of device pointers */
int lca_rope(const lca_rope_args* args, void* stream);

/* Frequencies of the pairs on the HOST, f_i = base^(-2 i / rot_dim), and the factor that goes with them, for contexts `scale` times as
 * long as `trained_len` tokens:
 *   PLAIN   as they are, factor 1
 *   LINEAR  f_i / scale
 *   BASE    base * scale^(rot_dim / (rot_dim - 2)) in place of base: the fastest pair keeps its frequency, the slowest is divided by scale
 *   RAMP    pairs that make more than `fast` turns in trained_len tokens keep f_i, those with less than `slow` take f_i / scale, between
 *           them the share that is kept grows linearly with the turns; factor 0.1 ln(scale) + 1 where scale > 1
 *           (one of two customs: others let the share grow with the pair's index between two bounds, and put part of the factor into the
 *           softmax scale.  A model trained that way needs its own frequencies; lca_rope takes any)
 * trained_len, fast and slow are only used by RAMP (customary: fast = 32, slow = 1). */
enum { LCA_ROPE_PLAIN = 0, LCA_ROPE_LINEAR = 1, LCA_ROPE_BASE = 2, LCA_ROPE_RAMP = 3 };
int lca_rope_frequencies(int32_t kind, int32_t rot_dim, double base, double scale, double trained_len, double fast,
                         double slow, double* freqs_host, float* factor_host);

/* ---- Verification of drafted tokens ----------------------------------------------------------
 * Which of the drafted tokens of each request the target accepts, and the token that follows them, so that the outcome is distributed
 * as the target's own samples.  With p_i the target's probabilities at draft i, q_i the drafter's and x_i the draft:
 *   draft i is accepted while u_accept[i] * q_i(x_i) < p_i(x_i)  (the product in 64 bits, where it is exact)
 *   the next token is drawn from max(p_i - q_i, 0) at the first rejected draft i, or from p after the last accepted one: the first
 *       token v whose cumulative sum exceeds u_sample times the whole sum, in 64-bit sums
 * A token has mass where the difference (where it is drawn from p: the entry) is a positive finite fp32 number.  Where p_i - q_i leaves none, the token
 * is drawn from p_i; where that has none either it is -1.  A draft outside the vocabulary is rejected (and with it all behind it). */
typedef struct lca_verify_args {
  int32_t dtype;                /* of both probabilities: LCA_DTYPE_FP32 or LCA_DTYPE_BF16 */
  int32_t batch, n_drafts, vocab;       /* n_drafts >= 0; n_drafts and vocab below 2^31 - 4096 */
  const void* target_probs;     /* [batch, n_drafts + 1, vocab]; they need not add up to 1 */
  const void* draft_probs;      /* [batch, n_drafts, vocab]; NULL: the drafter is certain (q_i(x_i) = 1, 0 elsewhere) */
  const int32_t* draft_tokens;  /* [batch, n_drafts] */
  const int32_t* n_draft;       /* [batch]: drafts of each request, clamped to 0 .. n_drafts; NULL: n_drafts */
  const float* u_accept;        /* [batch, n_drafts] in [0, 1) */
  const float* u_sample;        /* [batch] in [0, 1) */
  const int32_t* n_tok;         /* [batch], or NULL with n_tok_out: tokens in the cache, the drafts included */
  int32_t* accepted;            /* [batch] out: number of accepted drafts */
  int32_t* tokens_out;          /* [batch, n_drafts + 1] out: accepted drafts, the next token, then -1 */
  int32_t* n_tok_out;           /* [batch] out, may be n_tok: n_tok less the rejected drafts, the target state for lca_page_update */
} lca_verify_args;              /* a HOST structure of device pointers, each aligned to its element */
int lca_verify_drafts(const lca_verify_args* args, void* stream);

/* Value up-projection of the latent attention output (Alg. 1: v = c W^UV; Sec. 4.3: in the absorbed
 * form the attention result lives in the latent space and W^UV is applied to it once per query and
 * head):   out_v[t, h, :] = attn_latent[t, h, :] . W^UV[h]
 *   attn_latent [n_tokens, n_heads, d_latent] bf16: `out` of lca_prefill_attention / lca_decode_attention
 *                                                   (n_tokens = batch * seq_len, or batch for decode)
 *   w_uv        [n_heads, d_latent, d_v] bf16 (d_v contiguous)
 *   out_v       [n_tokens, n_heads, d_v] bf16 (products in bf16 on the tensor cores, fp32 sums, one rounding)
 * Built for d_latent = 512, d_v = 128 (DeepSeek-V2 / V3); other sizes return LCA_ERR_UNSUPPORTED_SHAPE.
 * Needs no workspace.  n_tokens = 0 is a no-op. */
int lca_latent_to_value(const void* attn_latent, const void* w_uv, void* out_v, int64_t n_tokens,
                        int32_t n_heads, int32_t d_latent, int32_t d_v, void* stream);

/* Which attention implementation lca_prefill_attention / lca_decode_attention use:
 *   0 = automatic (tensor-core kernels where the shape is supported, else the scalar kernel),
 *   1 = force the scalar (CUDA-core) kernel, 2 = force the tensor-core kernel (unsupported
 *   shapes then return LCA_ERR_UNSUPPORTED_SHAPE).  Process-wide; returns the previous value. */
int lca_set_attention_impl(int impl);

/* Number of kernels the library has launched since it was loaded (all entry points). */
int64_t lca_launch_count(void);

/* Status word written by bounded device-side waits of the most recent tensor-core launch on the
 * current device: 0 = none expired.  Synchronises `stream`.  Returns LCA_OK or
 * LCA_ERR_DEVICE_TIMEOUT / LCA_ERR_CUDA. */
int lca_last_device_status(void* stream);

/* Self-test of the time-out mechanism (the paper has no counterpart).  Every device-side wait of
 * the tensor-core kernels gives up after a fixed number of SM cycles, records a code in the status
 * word that lca_last_device_status reads, and the kernel returns in an orderly way.  This call
 * launches a one-thread kernel that waits, with the same routine and a limit of `limit_cycles`
 * (1 .. 1e8), on a barrier nobody ever arrives on: afterwards lca_last_device_status returns
 * LCA_ERR_DEVICE_TIMEOUT once, and the next ordinary call works as usual.  Nothing faults, traps or
 * waits longer than the limit. */
int lca_selftest_bounded_wait(int64_t limit_cycles, void* stream);

const char* lca_status_string(int status);
int lca_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LCA_H_ */
