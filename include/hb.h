/*
 * hb.h -- C ABI of the heterogeneous-batching step library (B200 / sm_100a).
 *
 * One call, hb_mixed_step, runs ONE transformer forward over a ragged mixed
 * batch: the "forward" stage of the paper's inference loop (Algorithm 1) over
 * the batch unit of Section 3.2 (embedding chunks, generation prefill chunks,
 * decode tokens), followed by the two output paths of Algorithm 1: the
 * incremental pooler of Section 3.3 (Eq. 1-2 and the last-token head) on the
 * embedding rows and the logits for the sampler on the generation rows.
 *
 * Conventions
 *  - every function returns an int status: HB_OK (0) or a negative HB_ERR_*;
 *    nothing throws or aborts across this boundary;
 *  - "host" / "device" is stated for every pointer; device pointers are plain
 *    CUDA device addresses on the current device; `stream` is a cudaStream_t
 *    passed as void* (NULL = the legacy default stream);
 *  - the library never frees caller memory; hb_mixed_step allocates no device
 *    memory, and its host scratch (work lists, validation marks, the pinned
 *    descriptor staging) belongs to the context: it is reserved by hb_create
 *    for the context's limits and only grows if a step meets a KV cache or
 *    pool with more pages / slots than any step before (per-class timing,
 *    hb_profile_enable, creates its CUDA events on demand);
 *  - all work is enqueued on `stream`; outputs are valid once the caller has
 *    synchronised that stream;
 *  - there is no CPU path: without a CUDA device every compute call fails.
 */
#ifndef HB_H_
#define HB_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define HB_API __attribute__((visibility("default")))
#else
#define HB_API
#endif

/* ---- status codes ------------------------------------------------------- */
enum {
  HB_OK = 0,
  HB_ERR_BAD_ARG = -1,       /* null pointer, bad size, double free ...        */
  HB_ERR_CUDA = -2,          /* a CUDA runtime/driver call failed              */
  HB_ERR_OOM_PAGES = -3,     /* hb_kv_alloc_pages: not enough free pages       */
  HB_ERR_OOM_SLOTS = -4,     /* hb_pool_alloc_slot: no free slot               */
  HB_ERR_TOO_LARGE = -5,     /* batch exceeds the limits given to hb_create    */
  HB_ERR_BAD_DESC = -6,      /* batch descriptor failed validation             */
  HB_ERR_DEVICE_STATUS = -7, /* a kernel reported a bounded-wait expiry/index  */
  HB_ERR_UNSUPPORTED = -8    /* model shape outside what the kernels cover     */
};

/* Row kinds of the batch unit (Section 3.2).  Rows of one kind are contiguous
 * and kinds appear in this order (Section 3.2 has the scheduler hand over each
 * batch already grouped by kind, so every output head reads one slice). */
enum { HB_KIND_DECODE = 0, HB_KIND_PREFILL_CHUNK = 1, HB_KIND_EMBED_CHUNK = 2 };

/* Pooling heads (Section 3.3).  Additive (Eq. 1-2): mean (w = 1) and weighted
 * mean with w = 1-based position of the token in its request (the paper
 * leaves the weights open; this is the common position weighting).
 * Positional: last token (H of the last row of the final chunk) and CLS (H of
 * the first row of the first chunk, retained in the slot). */
enum { HB_POOL_NONE = 0, HB_POOL_MEAN = 1, HB_POOL_LAST = 2, HB_POOL_CLS = 3, HB_POOL_WMEAN = 4, HB_POOL_MAX = 5 };

typedef struct hb_ctx hb_ctx;
typedef struct hb_kv hb_kv;
typedef struct hb_pool hb_pool;

/* Decoder-only model: pre-norm RMSNorm, rotate-half RoPE, grouped-query causal
 * attention, SwiGLU FFN, no biases, untied LM head.  head_dim must be 64 or
 * 128; d_model, n_heads*head_dim, d_ffn multiples of 64; page_size 16.
 * Precision: bf16 model weights, repacked to fp16 for the tensor cores;
 * activations between kernels, the KV cache and the attention probabilities
 * fp16; residual stream, norms, softmax, pooling and every accumulation fp32. */
typedef struct {
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab;
  int32_t page_size;    /* tokens per KV page (16)                              */
  int32_t max_pos;      /* largest position + 1 any request may reach          */
  float rope_theta;
  float rms_eps;
} hb_model_cfg;

/* Weights are row-major [out, in] (y = x * W^T), device memory owned by the
 * caller.  The projection matrices are fp16: the model's bf16 values repacked
 * once with hb_weights_pack_f16 (the tensor cores take one 16-bit format for
 * both operands, and activations are fp16).  Gains and the token embedding
 * stay bf16.
 *   wqkv      fp16 [(n_heads + 2 n_kv_heads) * head_dim, d_model]: q rows, then k, then v;
 *             inside every q and k head the rows are pair-interleaved for the rotary
 *             step: row 2i = the head's row i, row 2i+1 = its row i + head_dim/2
 *             (a fixed permutation of the head dimension, applied alike to q and k,
 *             so q.k is unchanged; the KV cache holds k in this order)
 *   wo        fp16 [d_model, n_heads * head_dim]
 *   w_gate_up fp16 [2 * d_ffn, d_model]: row 2j = gate row j, row 2j+1 = up row j
 *   w_down    fp16 [d_model, d_ffn]
 *   lm_head   fp16 [vocab, d_model]
 *   attn_norm, ffn_norm, final_norm bf16 [d_model] gains
 *   tok_emb   bf16 [vocab, d_model] */
typedef struct {
  const void* attn_norm;
  const void* wqkv;
  const void* wo;
  const void* ffn_norm;
  const void* w_gate_up;
  const void* w_down;
} hb_layer_weights;

typedef struct {
  const void* tok_emb;               /* device */
  const hb_layer_weights* layers;    /* HOST array [n_layers] of device ptrs   */
  const void* final_norm;            /* device */
  const void* lm_head;               /* device */
} hb_weights;

/* One segment = the rows one request contributes to this step (Section 3.2).
 *   kind        HB_KIND_*
 *   q_start     first token row of the segment (prefix sum of q_len)
 *   q_len       rows: 1 for DECODE, chunk size c_k otherwise (>= 1)
 *   pos_start   tokens of this request already in the KV cache; row j has
 *               position pos_start + j, writes its K/V there and attends to
 *               positions 0 .. pos_start + j of its own request
 *   pt_start    offset of this request's page list inside page_ids
 *   pt_len      entries of that list; must cover pos_start + q_len tokens
 *   pool_slot   pool slot (EMBED_CHUNK) or -1
 *   pool_mode   HB_POOL_* (NONE unless EMBED_CHUNK)
 *   is_final    last chunk of the request: emit embedding / logits
 *   logits_row  row of out_logits to write (DECODE, final PREFILL_CHUNK), else -1
 *   emb_row     row of out_emb to write (final EMBED_CHUNK), else -1 */
typedef struct {
  int32_t kind, q_start, q_len, pos_start;
  int32_t pt_start, pt_len, pool_slot, pool_mode;
  int32_t is_final, logits_row, emb_row, reserved;
} hb_seg;

/* Batch descriptor; every pointer is HOST memory, read during the call only. */
typedef struct {
  int32_t n_tokens;       /* total rows T                                       */
  int32_t n_segs;         /* segments R                                         */
  int32_t n_page_ids;     /* length of page_ids                                 */
  int32_t n_logit_rows;   /* rows of out_logits produced this step              */
  int32_t n_emb_rows;     /* rows of out_emb produced this step                 */
  const int32_t* token_ids; /* [n_tokens] ids in [0, vocab)                     */
  const hb_seg* segs;       /* [n_segs]                                         */
  const int32_t* page_ids;  /* [n_page_ids] physical page numbers               */
} hb_batch_desc;

/* ---- context -------------------------------------------------------------- */

/* Bytes of device workspace a context needs for steps of at most max_tokens
 * rows, max_segs segments and max_page_ids page-list entries.  Host only. */
HB_API int hb_workspace_bytes(const hb_model_cfg* cfg, int32_t max_tokens, int32_t max_segs,
                       int32_t max_page_ids, size_t* out_bytes);

/* Create a context on the current device.  `workspace` (device, 256-byte
 * aligned, hb_workspace_bytes big) stays owned by the caller; pass NULL to let
 * the library allocate (and later free) it.  Builds the rotary table and the
 * activation tensor maps.  Synchronises the device once. */
HB_API int hb_create(const hb_model_cfg* cfg, int32_t max_tokens, int32_t max_segs,
              int32_t max_page_ids, void* workspace, size_t workspace_bytes,
              hb_ctx** out);
HB_API int hb_destroy(hb_ctx* ctx);

/* ---- paged KV cache ------------------------------------------------------- */

/* Bytes of an arena of n_pages.  Arena layout (fp16; post-rotary K and V):
 * [layer][page][kv_head][slot group][K|V][head_dim/64][8 slots][64]: slots 0-7
 * and 8-15 of a page form two groups, the head dimension is split into
 * 64-element halves, and the K+V block of one (layer, page, head) is contiguous
 * (4-8 KiB), so one TMA copy fetches it and the blocks of consecutive pages
 * line up in shared memory the way the tensor-core descriptors need.
 * Host only. */
HB_API int hb_kv_arena_bytes(const hb_model_cfg* cfg, int32_t n_pages, size_t* out_bytes);

/* Wrap a caller-owned device arena.  Only the free list lives in the library
 * (host memory); no device work.  `arena` may be NULL for host-side
 * bookkeeping tests. */
HB_API int hb_kv_create(const hb_model_cfg* cfg, void* arena, size_t arena_bytes, int32_t n_pages,
                 hb_kv** out);
HB_API int hb_kv_destroy(hb_kv* kv);
/* Take n pages (lowest free ids first); all-or-nothing: HB_ERR_OOM_PAGES. */
HB_API int hb_kv_alloc_pages(hb_kv* kv, int32_t n, int32_t* out_ids /* host [n] */);
/* Return pages; a page not currently allocated -> HB_ERR_BAD_ARG, nothing freed. */
HB_API int hb_kv_free_pages(hb_kv* kv, int32_t n, const int32_t* ids /* host [n] */);
HB_API int hb_kv_free_count(const hb_kv* kv, int32_t* out_free);

/* ---- pooling state (Section 3.3: O(d) state per request) ------------------ */

/* Arena layout: float sum[n_slots][d_model], then uint32 meta[n_slots][4] =
 * {count, chunks, mode, state}; state 0 = open, 1 = emitted.  Host only. */
HB_API int hb_pool_arena_bytes(const hb_model_cfg* cfg, int32_t n_slots, size_t* out_bytes);
HB_API int hb_pool_create(const hb_model_cfg* cfg, void* arena, size_t arena_bytes, int32_t n_slots,
                   hb_pool** out);
HB_API int hb_pool_destroy(hb_pool* pool);
/* Take a slot (lowest free id).  No device work: the first chunk of a request
 * (pos_start == 0) overwrites the slot, which realises S(0) = 0, W(0) = 0. */
HB_API int hb_pool_alloc_slot(hb_pool* pool, int32_t* out_slot);
HB_API int hb_pool_free_slot(hb_pool* pool, int32_t slot);

/* Row buffer for buffered heads (Section 3.3: a head that is neither additive
 * nor positional keeps A(k) = [A(k-1); H(k)], every final hidden state of the
 * request, at O(n d) memory, and runs after the final chunk).  Layout:
 * float rows[n_slots][max_rows][d_model]; row p of a slot holds the final
 * RMSNorm output of the request's token at position p.  The caller owns the
 * memory (device, 256-byte aligned); attach it once, before the first step
 * that uses HB_POOL_MAX.  HB_POOL_MAX is the buffered head built in: every
 * chunk appends its rows, the final chunk emits the element-wise maximum over
 * all n rows, L2-normalised.  After the final chunk the buffer holds all n
 * rows, so a caller can run any other head over them itself.  A segment with
 * pos_start + q_len > max_rows, or HB_POOL_MAX without an attached buffer, is
 * HB_ERR_BAD_DESC.  max_rows in 1..cfg.max_pos.  Host only. */
HB_API int hb_pool_row_buffer_bytes(const hb_model_cfg* cfg, int32_t n_slots, int32_t max_rows, size_t* out_bytes);
HB_API int hb_pool_attach_row_buffer(hb_pool* pool, void* buf, size_t bytes, int32_t max_rows);

/* ---- the step ------------------------------------------------------------- */

/* Host-only validation of a descriptor against the limits (what hb_mixed_step
 * checks before it enqueues anything): sizes, kind order, q_start prefix sums,
 * page lists cover pos_start + q_len, page ids in [0, n_pages), a page written
 * this step belongs to one segment only, pool slots in range and used once,
 * output rows in range and used once, token ids in range. */
HB_API int hb_validate_desc(const hb_model_cfg* cfg, int32_t max_tokens, int32_t max_segs,
                     int32_t max_page_ids, int32_t n_pages, int32_t n_slots,
                     const hb_batch_desc* desc);

/* One forward step over the mixed batch (Algorithm 1: Forward, IncPooler,
 * and the logits the Sampler consumes).
 *   desc        host descriptor (copied; may be reused after return)
 *   w           host struct of device weight pointers
 *   kv, pool    caches created above; K/V of every row is appended to its
 *               page; pool slots of EMBED_CHUNK segments are updated
 *   out_logits  device float [>= n_logit_rows, vocab]; row seg.logits_row gets
 *               the logits of the segment's last row
 *   out_emb     device float [>= n_emb_rows, d_model]; row seg.emb_row gets the
 *               L2-normalised embedding of a request whose final chunk ran
 * Rows of the outputs not named by a segment are left untouched.  Returns
 * after enqueueing; no synchronisation, no device allocation.  A failed
 * validation enqueues nothing.  Alignment (checked, HB_ERR_BAD_ARG): out_logits,
 * out_emb and tok_emb 16 bytes, every norm gain 8 bytes (the kernels use
 * 16-byte and 8-byte vector accesses); projection weights 16 bytes. */
HB_API int hb_mixed_step(hb_ctx* ctx, const hb_batch_desc* desc, const hb_weights* w, hb_kv* kv,
                  hb_pool* pool, float* out_logits, float* out_emb, void* stream);

/* ---- low-rank adapters on embedding rows ------------------------------------
 *
 * With a shared backbone the embedding model is the generation model plus a
 * low-rank adapter (Section 2.1, paragraph on parameter sharing; in Section
 * 5.1 both request types share one GPU through such adapters).  Inside the one forward
 * pass, rows of EMBED_CHUNK segments compute every projection as
 *     y = x W^T + (alpha / r) (x A^T) B^T,        A [r, in], B [out, r],
 * and rows of DECODE / PREFILL_CHUNK segments compute y = x W^T.  The paper
 * does not say which projections carry the adapter; here all seven of a layer
 * do (q, k, v, o, gate, up, down).  Token embedding, norm gains and LM head
 * are shared unchanged.
 *
 * Packed layout (device, fp16, row-major, 16-byte aligned; the caller packs
 * once).  R(n) = n * r rounded up to a multiple of 64; unused rows / columns
 * are zero.  Row orders of the B factors follow the fused weights they pair
 * with (hb_layer_weights):
 *   a_qkv  [R(3), d]          rows [0,r) = A_q, [r,2r) = A_k, [2r,3r) = A_v
 *   b_qkv  [(Hq+2Hkv)Dh, R(3)] rows as wqkv (q and k rows pair-interleaved per
 *                             head); q rows hold B_q in columns [0,r), k rows
 *                             B_k in [r,2r), v rows B_v in [2r,3r), zero elsewhere
 *   a_o    [R(1), Hq*Dh]      A_o;           b_o  [d, R(1)]   B_o
 *   a_gu   [R(2), d]          A_gate, A_up;  b_gu [2F, R(2)]  rows as w_gate_up
 *                             (gate_j, up_j interleaved): gate rows hold B_gate
 *                             in [0,r), up rows B_up in [r,2r)
 *   a_d    [R(1), F]          A_down;        b_d  [d, R(1)]   B_down
 * scale = alpha / r multiplies the rank-r activations in fp32 before they are
 * rounded to fp16.  rank in 1..64. */
typedef struct hb_lora_layer {
  const void *a_qkv, *b_qkv, *a_o, *b_o, *a_gu, *b_gu, *a_d, *b_d;
} hb_lora_layer;

typedef struct hb_lora {
  int32_t rank;
  float scale;
  const hb_lora_layer* layers; /* host array [n_layers] */
} hb_lora;

/* hb_mixed_step with adapters on the EMBED_CHUNK rows.  lora == NULL, or a
 * step without EMBED_CHUNK rows, is exactly hb_mixed_step.  Per layer this
 * adds four thin GEMMs (the rank-r activations of the rows, zero for rows
 * that carry no adapter) and extends the K loop of the four projection GEMMs
 * by R / 64 blocks.  The context must have been created after
 * hb_workspace_bytes (the workspace always includes the rank-r buffer). */
HB_API int hb_mixed_step_lora(hb_ctx* ctx, const hb_batch_desc* desc, const hb_weights* w, const hb_lora* lora,
                       hb_kv* kv, hb_pool* pool, float* out_logits, float* out_emb, void* stream);

/* Repack bf16 values to fp16, element by element, on `stream` (device
 * pointers, 16-byte aligned; dst may equal src for an in-place repack, partial
 * overlap is rejected).  Exact for 2^-14 <= |w| <= 65504; smaller magnitudes
 * round to the fp16 subnormal grid (absolute error <= 2^-25), larger saturate. */
HB_API int hb_weights_pack_f16(const void* src_bf16, void* dst_f16, size_t n_elems, void* stream);

/* Greedy sampler over logits rows (Algorithm 1 "Sampler", greedy case): lowest
 * index of the maximum of each row.  logits device float [n_rows, vocab],
 * out_tokens device int32 [n_rows]. */
HB_API int hb_argmax(hb_ctx* ctx, const float* logits, int32_t n_rows, int32_t* out_tokens,
              void* stream);

/* Read (and clear) the device status word; synchronises `stream`.  0 = clean.
 * Non-zero: *out_code holds the OR of the bits below and the call returns
 * HB_ERR_DEVICE_STATUS.  Bits 0-5 and 7-11 mean a kernel gave up (a bounded wait
 * expired, an index check failed: outputs of that step are not valid); bit 6 is a
 * value report: the step ran, but an activation did not fit fp16. */
enum {
  HB_STATUS_GEMM_WAIT = 1,        /* projection GEMM: a pipeline wait expired                 */
  HB_STATUS_ATTN_INDEX = 2,       /* attention: page id out of range                          */
  HB_STATUS_APPEND_INDEX = 4,     /* KV append: page id out of range (row not written)        */
  HB_STATUS_POOL_INDEX = 8,       /* pooler: slot / row buffer out of range                   */
  HB_STATUS_ATTN_WAIT = 16,       /* attention: a pipeline wait expired                       */
  HB_STATUS_SELFTEST_WAIT = 32,   /* hb_selftest_wait_expiry                                  */
  HB_STATUS_TOKEN_INDEX = 128,    /* hb_logprobs: a token id beyond the vocabulary (its row got NaN) */
  HB_STATUS_LOGPROBS_WAIT = 256,  /* hb_logprobs: a pipeline wait expired                 */
  HB_STATUS_ROW_INDEX = 512,      /* hb_quant_rows: an index beyond the source's rows (its row was not written) */
  HB_STATUS_GROUP_INDEX = 1024,   /* hb_linear_grouped: bounds that decrease or pass the rows (that group was not computed) */
  HB_STATUS_LINEAR_WAIT = 2048,   /* hb_linear, hb_linear_grouped: a pipeline wait expired */
  HB_STATUS_F16_RANGE = 64        /* a normed row or a SwiGLU output was NaN or beyond +-65504:
                                     finite values were stored saturated, NaN was stored as NaN */
};
HB_API int hb_status_poll(hb_ctx* ctx, void* stream, uint32_t* out_code);

/* Per-kernel-class device timing.  While enabled, hb_mixed_step brackets every launch with a
 * pair of CUDA events on the step's stream; hb_profile_read synchronises them, adds the
 * elapsed milliseconds and launch counts per class into the two arrays of HB_N_CLASSES
 * entries, and clears the record.  While enabled, launches do not overlap one another and
 * the layer's one attention launch is issued once per item list (classes 1 and 5), so the
 * launch count of a step is higher than in normal operation.  Classes: */
enum {
  HB_CLASS_GEMM = 0,      /* QKV, O, gate/up, down projections                          */
  HB_CLASS_ATTENTION = 1, /* attention launch (when timed: the decode splits alone) */
  HB_CLASS_NORM_ROPE = 2, /* gather + RMSNorm, RMSNorm, RoPE + KV append                */
  HB_CLASS_POOL = 3,      /* final RMSNorm + pooler / logits-row preparation            */
  HB_CLASS_LM_HEAD = 4,   /* LM-head projection                                         */
  HB_CLASS_ATTENTION_TC = 5, /* when timed: the attention launch's tcgen05 chunk tiles alone */
  HB_CLASS_LORA = 6,      /* adapters: rank-r activations of the embedding rows         */
  HB_N_CLASSES = 7
};
HB_API int hb_profile_enable(hb_ctx* ctx, int on);
HB_API int hb_profile_read(hb_ctx* ctx, float* ms_by_class, int32_t* launches_by_class);

/* Failure-path self-test.  Every wait inside the kernels (on an mbarrier fed by TMA, by the tensor
 * cores or by another warp role) is bounded in time; when a bound expires the kernel raises a bit
 * in the status word and returns normally.  This call launches a one-thread kernel that runs the
 * same bounded wait on a barrier nothing arrives on, with a limit of limit_ms (1..1000)
 * milliseconds, so that the path "wait expires -> status bit -> hb_status_poll returns
 * HB_ERR_DEVICE_STATUS -> context still usable" can be exercised without faulting or hanging the
 * GPU.  The status code it raises is 32. */
HB_API int hb_selftest_wait_expiry(hb_ctx* ctx, uint32_t limit_ms, void* stream);

/* Kernels launched by the last hb_mixed_step on this context. */
HB_API int hb_last_launch_count(const hb_ctx* ctx, int32_t* out_count);

/* ---- kernel-level entry points (used by the parity tests) ----------------- */

/* Epilogues of the projection GEMM (the dense contractions of the forward,
 * Section 3.1: the attention and feed-forward projections every row passes through). */
enum {
  HB_EPI_F16 = 0,       /* C fp16 [M,N] = A * B^T                               */
  HB_EPI_F32 = 1,       /* C float [M,N] = A * B^T                              */
  HB_EPI_RESID_F32 = 2, /* C float [M,N] += A * B^T (residual stream update)    */
  HB_EPI_SWIGLU = 3     /* C fp16 [M,N/2]: silu(acc[2j]) * acc[2j+1]            */
};

/* C = epilogue(A * B^T): A fp16 [M,K] row-major (activations), B fp16 [N,K]
 * row-major (weights), both K-major, fp32 accumulation on the tcgen05 tensor
 * cores; fp16 outputs saturate at +-65504.  All device pointers, 16-byte
 * aligned; K and N multiples of 8.  M may be any value >= 1. */
HB_API int hb_gemm(hb_ctx* ctx, const void* A, const void* B, void* C, int32_t M, int32_t N,
            int32_t K, int32_t epilogue, void* stream);

/* hb_gemm with a second operand pair accumulated after the first:
 * C = epilogue(A * B^T + A2 * B2^T), A2 fp16 [M,K2], B2 fp16 [N,K2], K2 a
 * multiple of 64.  This is how an adapted projection adds its low-rank branch
 * (hb_mixed_step_lora): A2 = the rows' rank-r activations, B2 = the up factor. */
HB_API int hb_gemm_pair(hb_ctx* ctx, const void* A, const void* B, const void* A2, const void* B2, void* C,
                 int32_t M, int32_t N, int32_t K, int32_t K2, int32_t epilogue, void* stream);

/* Tile walk of the projection GEMM, for tests and tuning.  A launch normally chooses by itself in
 * which order its workers take the output tiles (rows fastest over the whole M, or in bands of row
 * tiles when A's share of a work item would not stay in L2) and whether its loads carry L2 eviction
 * hints.  The walk never changes the K order of an element's sum, so results are bit-identical under
 * every setting; this call forces one for all later launches of the process so that a test can show
 * exactly that, and a profile can compare DRAM traffic.  band >= 1: row tiles per band; band = 0: whole
 * M; hints 0 / 1; -1 for either = automatic again.  Host only, not thread-safe against launches. */
HB_API int hb_gemm_set_walk(int32_t band, int32_t hints);
/* Tuning: cap the CTAs of every projection launch at max_ctas (even; 0 = one per SM again), e.g. to
 * leave SMs to kernels of another stream.  Changes the work split between workers only, never a
 * result bit.  Host only, process-wide. */
HB_API int hb_gemm_set_cta_limit(int32_t max_ctas);
/* The attention launch of a step runs min(items, 2 per SM) resident blocks that take the step's
 * attention items (decode splits, chunk tiles) one after the other from a ticket.  This call caps the
 * blocks of every later attention launch of the process at max_blocks (0 = automatic again), so that a
 * test can make one block walk through many items of both kinds.  Which block runs an item never
 * changes a result bit (an item's arithmetic is its own; the splits of a decode row are merged in
 * split order by whichever block arrives last).  Host only, not thread-safe against launches. */
HB_API int hb_attn_set_block_limit(int32_t max_blocks);
/* Keys per decode attention item.  A decode row with n = context + 1 keys is cut into
 * max(1, (n + keys / 2) div keys) equal splits (rounded up to whole 64-key tiles) that different blocks
 * may run; their partial results are merged in split order.  The count depends on the row's own context
 * and on this value only, never on the rest of the batch, so a request's result does not depend on its
 * batch; it does depend on this value (another summation order: results differ in the last bits).
 * Default 2048 (keys = 0 restores it); multiples of 64 from 256 to 65536.  A smaller value keeps more
 * blocks busy when steps hold only a few long decode rows, at the cost of a partial record, a fence, an
 * atomic and a share of the merge per split.  Process-wide; hb_workspace_bytes and hb_create read it,
 * and a context keeps the value it was created with.  Host only. */
HB_API int hb_attn_set_split_keys(int32_t keys);

/* The incremental pooler on its own (Section 3.3, Eq. 1-2 and the last-token
 * head), as hb_mixed_step runs it on an embedding segment: final RMSNorm of
 * the chunk's rows, then
 *   mean / weighted mean: S <- S + sum_j w_j rmsnorm(x_j) * gain, count <-
 *         count + n_rows (first_chunk != 0 starts from S = 0, count = 0; the
 *         position weights continue from the slot's count);
 *   last: only the counters move until the final chunk; cls: the first
 *         chunk's first normed row is kept in S;
 * and on the final chunk out_emb = L2-normalised S / W (W = count, or
 * count (count + 1) / 2 for position weights) or the retained row.
 *   x          device float [n_rows, d_model] residual-stream rows of the chunk
 *   gain       device bf16 [d_model] final-norm gain
 *   slot_sum   device float [d_model], slot_meta device uint32 [4] =
 *              {count, chunks, mode, state}: the request's pool slot (in/out)
 *   out_emb    device float [d_model] (written when is_final != 0)
 * n_rows <= the context's max_tokens.  Uses the context's scratch.  x,
 * slot_sum and out_emb must be 16-byte aligned, gain 8-byte aligned (vector
 * accesses); a misaligned pointer is HB_ERR_BAD_ARG and nothing is launched. */
HB_API int hb_pool_chunk(hb_ctx* ctx, const float* x, const void* gain, int32_t n_rows, int32_t mode,
                         int32_t first_chunk, int32_t is_final, float* slot_sum, uint32_t* slot_meta,
                         float* out_emb, void* stream);

/* ---- entry point that allocates nothing ------------------------------------ */

/* Largest chunk and hidden size hb_pool_chunk_noalloc accepts. */
#define HB_NOALLOC_MAX_ROWS 2048
#define HB_NOALLOC_MAX_DMODEL 4096

/* (The paper has no counterpart to this call; it exists for deployment.)
 * hb_pool_chunk without a context and without any allocation: same arguments
 * and results as hb_pool_chunk, with d_model and rms_eps passed directly.
 *
 * Who needs it: a caller that cannot allocate device memory -- for example a
 * serving process whose own allocator claimed the whole device at start-up, or
 * code running where a device allocation would fail or stall the GPU -- cannot
 * create an hb_ctx (that allocates the workspace) and so cannot reach any other
 * compute call.  Here the pooler's scratch (partial sums of 32-row blocks, an
 * arrival counter, a status word) lives in a fixed array inside the library
 * image instead: 1 MiB + 256 bytes on every GPU that loads the library, held
 * until the process exits.  The call itself uses no cudaMalloc, cudaFree or
 * any other allocating routine.
 *
 * Limits and rules
 *  - n_rows <= HB_NOALLOC_MAX_ROWS and d_model <= HB_NOALLOC_MAX_DMODEL
 *    (d_model a multiple of 4); anything larger returns HB_ERR_TOO_LARGE and
 *    does nothing;
 *  - the first call on a device looks up the array's device address (once per
 *    device, with that device current); make that first call before starting
 *    any stream capture;
 *  - all calls on a device share the one array, which keeps the previous
 *    call's contents (the call clears the words that must start at zero).
 *    Two calls whose kernels can run at the same time on that device -- from
 *    different streams or threads -- race on it: serialise them;
 *  - the caller still owns and passes every input and output (x, gain,
 *    slot_sum, slot_meta, out_emb: device pointers as in hb_pool_chunk), with
 *    the same alignment rule: x, slot_sum, out_emb 16 bytes, gain 8 bytes.  A
 *    view cut out of a larger arena at an odd offset is refused with
 *    HB_ERR_BAD_ARG before anything is launched;
 *  - the looked-up address is cached for the life of the process.  After
 *    cudaDeviceReset on that device it is stale: do not call this entry again
 *    in a process that reset the device;
 *  - there is no context, so no hb_status_poll: the status word the kernel
 *    keeps in the array's tail is write-only for callers.  The only device
 *    check behind it (pool slot in range) cannot fail here, because this entry
 *    always runs on a one-slot pool it builds itself. */
HB_API int hb_pool_chunk_noalloc(const float* x, const void* gain, int32_t n_rows, int32_t d_model,
                                 float rms_eps, int32_t mode, int32_t first_chunk, int32_t is_final,
                                 float* slot_sum, uint32_t* slot_meta, float* out_emb, void* stream);

/* ---- 8-bit KV cache ---------------------------------------------------------
 *
 * The paged KV cache with one byte per element (e4m3: 4 exponent and 3 mantissa bits) and a scale
 * for each block of one page (16 tokens) and KV head, K and V apart: half the memory and half the
 * bytes a decode row has to read.  Arena layout: [layer][page][kv head][block], block =
 *   16 * head_dim codes of K: token t, dimension d at byte (d / 64) * 1024 + t * 64 + d % 64
 *   16 * head_dim codes of V: token t, dimension d at byte
 *       (d / 32) * 512 + (d % 8 * 4 + t % 8 / 2) * 16 + d % 32 / 8 * 4 + t / 8 * 2 + t % 2
 *   32 bytes: float scale of K, float scale of V (powers of two), 24 bytes reserved
 * (a block is read with ONE bulk copy and its 16-byte pieces are the matrix-instruction fragments).
 * A code c stands for c * scale.  The scale is the smallest 2^e, -32 <= e <= 24, with
 * max |x| <= 448 * 2^e over the rows appended to the block (448 is the largest e4m3 value).  A power
 * of two, because then neither the codes nor the products with them are rounded by it, and a code
 * that has to be stored again under a larger scale only changes where it falls below the smallest
 * normal e4m3 value.  An append that starts at slot 0 of a page starts the block afresh (its
 * unused slots become zero); one that starts later keeps the larger of the block's scale and its own,
 * and stores the block's codes again if the scale grew.  Infinite elements saturate, NaN stays NaN. */

/* Bytes of an 8-bit arena of n_pages.  Host only. */
HB_API int hb_kv8_arena_bytes(const hb_model_cfg* cfg, int32_t n_pages, size_t* out_bytes);
/* hb_kv_create for the 8-bit format: an hb_kv whose pages are allocated, freed and destroyed with
 * the hb_kv_* calls above, and which hb_mixed_step[_lora] takes in place of a 16-bit cache (the
 * step's QKV projection then leaves fp16 rows for hb_kv8_append, and hb_kv8_attention reads the
 * pages; its rows are rounded to fp16 before their rotation).  Such a step has at most 8192 segments.  Arena
 * 256-byte aligned. */
HB_API int hb_kv8_create(const hb_model_cfg* cfg, void* arena, size_t arena_bytes, int32_t n_pages, hb_kv** out);

/* The rows of a step, in DEVICE memory the caller owns.  Of each segment q_start, q_len, pos_start,
 * pt_start and pt_len are read (the other fields are not).  Unlike in hb_batch_desc, segments need
 * not be adjacent and q_len may be 0; rows whose row_seg is -1 belong to nobody (padding): what
 * the calls write for rows is left untouched there.  Nothing is read on the host, so a captured
 * call sees what the arrays hold when it is replayed.  row_seg[r] = s exactly for the rows of
 * segment s, and no row belongs to two segments.  Limits (HB_ERR_TOO_LARGE beyond them): 8192
 * segments, 2^26 rows, max_keys 2^30.  The two bounds size the launches: a segment beyond one of
 * them, a page id outside the arena, or any other inconsistent field is reported
 * through the status word (HB_STATUS_APPEND_INDEX / HB_STATUS_ATTN_INDEX) and skipped. */
typedef struct {
  const hb_seg* segs;        /* device [n_segs], 16-byte aligned                        */
  const int32_t* page_ids;   /* device [n_page_ids]                                     */
  const int32_t* row_seg;    /* device [n_rows]: the row's segment, -1 = padding        */
  int32_t n_segs, n_page_ids, n_rows;
  int32_t max_q_len;         /* no segment has more rows                                */
  int32_t max_keys;          /* no segment has a larger pos_start + q_len               */
} hb_rows;

/* Which pairs of a head's first rot_dim dimensions turn together: (2i, 2i + 1), or (i, i + rot_dim / 2). */
enum { HB_ROPE_PAIRS = 0, HB_ROPE_HALVES = 1 };

/* What hb_kv8_append reads and writes besides the cache.  Device pointers.
 *   qkv       fp16 [n_rows, qkv_stride]: per row n_heads q heads, n_kv_heads k heads, n_kv_heads v
 *             heads of head_dim; 16-byte aligned, stride a multiple of 8
 *   q_out     fp16 [n_rows, q_stride]: the row's normed and rotated q heads; may be the q part of qkv
 *   q_gain, k_gain  bf16 [head_dim] (16-byte aligned) or NULL: x <- x / sqrt(mean(x^2) + norm_eps) * gain per head
 *   rope_cos, rope_sin  fp32 [rope_rows, rot_dim / 2] (16-byte aligned), row = position; rot_dim a
 *             multiple of 16 up to head_dim, 0 = no rotation (the tables are not read)
 * Norm, rotation and scaling run in fp32; q is rounded once to fp16 (saturating), k once to e4m3. */
typedef struct {
  const void* qkv;
  void* q_out;
  int64_t qkv_stride, q_stride;   /* elements */
  const void *q_gain, *k_gain;
  float norm_eps;
  const float *rope_cos, *rope_sin;
  int32_t rope_rows, rot_dim, rope_layout;
} hb_append_args;

/* Norms, rotates and appends the k and v of every row to layer `layer` of an 8-bit cache at position
 * pos_start + (row - q_start), and writes the rotated q.  A page written by one segment must not be
 * written by another of the same call.  ctx supplies the status word (same cfg as the cache's). */
HB_API int hb_kv8_append(hb_ctx* ctx, hb_kv* kv, int32_t layer, const hb_rows* rows, const hb_append_args* args, void* stream);

/* Causal attention of every row over its own request's pages of an 8-bit cache (the rows' own k and
 * v included: append first): row j of a segment sees positions 0 .. pos_start + j.
 *   q    fp16 [n_rows, q_stride], out fp16 [n_rows, out_stride]: n_heads heads of head_dim; 16-byte
 *        aligned, strides multiples of 8; out may not overlap q
 *   scale  factor of the scores, up to 2^60 (0 = 1 / sqrt(head_dim)): with it the scores of finite q and k are finite
 *   workspace  device, 256-byte aligned, hb_kv8_attention_workspace bytes for these rows; needs no
 *        initialisation and belongs to the call until it has run: calls that may run at the same
 *        time need a workspace each
 * Scores, softmax and sums in fp32, probabilities rounded to fp16 for the tensor cores.  A NaN in
 * a key makes the rows that see it NaN; a NaN in a value makes at least that dimension of them NaN
 * (the whole row where other rows of the segment come before the token).  Rows before the token
 * are not touched by it.  How a segment's keys are split depends on its own lengths only, never on
 * the rest of the batch.  Inside hb_mixed_step the splits may be longer than the 512 keys of this call: there
 * they are 512 keys times the least power of two for which the records of max_segs requests of max_pos tokens fit
 * into the context's activation buffer.  A context of 4096 rows of a 7B-class model has 512 up to 64 segments of 8192 positions,
 * 4096 for 64 of 65552 and 32768 for 256 of 131072: with limits far beyond the requests, few long decode rows have too few
 * splits to fill the GPU.  Scores beyond 2^20 in size are as coarse as fp32 is there, and an infinite q has no defined result. */
HB_API int hb_kv8_attention_workspace(const hb_model_cfg* cfg, const hb_rows* rows, size_t* out_bytes);
HB_API int hb_kv8_attention(hb_ctx* ctx, hb_kv* kv, int32_t layer, const hb_rows* rows, const void* q, int64_t q_stride,
                     void* out, int64_t out_stride, float scale, void* workspace, size_t workspace_bytes, void* stream);

/* Rotary tables for hb_kv8_append: out_cos / out_sin HOST float [n_pos, rot_dim / 2], angle(p, i) =
 * p * f_i with f_i = theta^(-2i / rot_dim), formed in double and stored as float.  Scaling for
 * contexts longer than the trained one (NULL = none):
 *   HB_ROPE_LINEAR  f_i / factor for every i
 *   HB_ROPE_BY_PARTS  with r_i = orig_len * f_i / (2 pi) turns over the trained length:
 *       g_i = clamp((r_i - lo) / (hi - lo), 0, 1);  f_i * (g_i + (1 - g_i) / factor)
 *       (fast dimensions stay, slow ones are interpolated; Peng et al. 2023, "YaRN", section 3.2)
 *   both: cos and sin are multiplied by `attn_factor` (1 = unchanged)
 * Host only. */
enum { HB_ROPE_LINEAR = 1, HB_ROPE_BY_PARTS = 2 };
typedef struct {
  int32_t kind;
  double factor;        /* >= 1 */
  double orig_len, lo, hi;   /* BY_PARTS: orig_len > 0, 0 <= lo < hi */
  double attn_factor;   /* > 0 */
} hb_rope_scaling;
HB_API int hb_rope_table(int32_t n_pos, int32_t rot_dim, double theta, const hb_rope_scaling* scaling, float* out_cos, float* out_sin);

/* ---- scoring of logits -------------------------------------------------------- */

/* Largest number of alternatives hb_logprobs gives. */
#define HB_LOGPROBS_MAX_K 32
enum { HB_DTYPE_F32 = 0, HB_DTYPE_F16 = 1, HB_DTYPE_BF16 = 2, HB_DTYPE_E4M3 = 3 };   /* hb_logprobs takes the first two */

/* Scores logits rows (the sampler's side of Algorithm 1: what hb_argmax decides, this measures).
 *   logits   device [n_rows, row_stride] of dtype, the first `vocab` of each row count; rows need no
 *            alignment beyond their type's
 *   tokens   device int32 [n_rows]: the token whose log probability is asked for; negative = none
 *            (0 is written); >= vocab: NaN is written and HB_STATUS_TOKEN_INDEX raised
 *   out_logprob  float [n_rows]: x[token] - log sum exp x
 *   out_entropy  float [n_rows]: -sum p log p, in nats
 *   out_top_ids, out_top_logprobs  int32 / float [n_rows, k]: the k largest, best first, the lower
 *            token first among equals; 0 <= k <= min(vocab, HB_LOGPROBS_MAX_K); unused (may be NULL) if k = 0
 * tokens and out_logprob (both or neither), and out_entropy, may be NULL.  vocab up to 2^20.  A logit of -inf has probability 0.  A row that
 * holds NaN or +inf, or nothing but -inf, has no probabilities: its floats become NaN (NaN logits rank last among
 * the alternatives).  Statistics in fp32; a row's result does not depend on the other rows. */
HB_API int hb_logprobs(hb_ctx* ctx, const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t row_stride,
                const int32_t* tokens, int32_t k, float* out_logprob, float* out_entropy, int32_t* out_top_ids,
                float* out_top_logprobs, void* stream);

/* ---- dense operators in 8 and 16 bits ------------------------------------------
 *
 * The projections of a layer with what stands around them, as calls of their own: the norm that
 * feeds a product (hb_norm), rows brought to 8 bits (hb_quant_rows), and the product with scales,
 * bias, activation and residual in its epilogue, with one weight (hb_linear) or one per run of rows
 * (hb_linear_grouped).  Types are HB_DTYPE_*; strides are in elements and may exceed the row length.
 * E4M3 rows carry one fp32 scale each, max(their largest magnitude, 2^-100) / 448 (by the rounded
 * reciprocal): code c stands for c * scale.  A row that holds a NaN or an infinity has scale NaN and NaN codes.  fp16 outputs
 * saturate at +-65504 (NaN stays NaN).  Nothing is allocated, and no call keeps anything for the next: calls of one context may run at
 * the same time on different streams. */

/* y = s / sqrt(mean(s^2) + eps) * gain with s = x (+ residual), one pass over the row.  Device pointers.
 *   x         [n_rows, d] F32, F16 or BF16
 *   residual  [n_rows, d] F32, F16 or BF16, or NULL
 *   sum_out   [n_rows, d] of residual_dtype: s, rounded once (the norm takes the unrounded s); may be residual
 *             itself; NULL if it is not wanted; without a residual it has to be NULL
 *   gain      bf16 [d], or NULL = ones
 *   y         [n_rows, d] F32, F16, BF16 or E4M3; may be x itself where type and stride are x's
 *   y_scale   float [n_rows], E4M3 only (NULL otherwise)
 * Pointers aligned to their type, 1 <= d <= HB_NORM_MAX_D; rows are read and written in wide accesses where the arrays' rows
 * lie alike against 16-byte boundaries (8 for E4M3) and the gain starts on one, whatever d.  Statistics in fp32; a row whose
 * squares sum beyond fp32 norms to zero, as the formula does in fp32. */
#define HB_NORM_MAX_D 32768
typedef struct {
  const void* x;
  const void* residual;
  void* sum_out;
  const void* gain;
  void* y;
  float* y_scale;
  int64_t x_stride, residual_stride, sum_stride, y_stride;
  int32_t x_dtype, residual_dtype, y_dtype;
  int32_t n_rows, d;
  float eps;
} hb_norm_args;
HB_API int hb_norm(hb_ctx* ctx, const hb_norm_args* args, void* stream);

/* Rows to E4M3 with a scale each: row r of codes is row index[r] of x, or row r where index is NULL (then
 * n_src >= n_rows).  x [n_src, d] F32, F16 or BF16; index device int32 [n_rows]: a negative entry leaves its row as
 * it is, one >= n_src too and raises HB_STATUS_ROW_INDEX.  The same source row may be taken more than once.
 * codes [n_rows, d], scale float [n_rows]: a code is the e4m3 value nearest to the fp32 quotient x / scale.  Limits and alignment
 * as hb_norm's.  Without an index, codes may lie in x's own rows, each at the start of its row (the strides' bytes equal). */
HB_API int hb_quant_rows(hb_ctx* ctx, const void* x, int32_t x_dtype, int64_t x_stride, int32_t n_src, const int32_t* index,
                         int32_t n_rows, int32_t d, void* codes, int64_t codes_stride, float* scale, void* stream);

/* Activations of hb_linear; GELU is x Phi(x), GELU_TANH its form with tanh.  Their errors are 2^-20 of |x| at most, not of the result:
 * where GELU is small beside x (x = -5: 3e-7 x), some of its own bits are lost. */
enum { HB_ACT_NONE = 0, HB_ACT_RELU = 1, HB_ACT_SILU = 2, HB_ACT_GELU = 3, HB_ACT_GELU_TANH = 4 };

/* C = act(z) + residual,  z[i, j] = a_scale[i] * w_scale[j] * sum_k a[i, k] * w[j, k] + bias[j]
 * gated: w's rows are pairs (gate, up) as in hb_layer_weights.w_gate_up, C has n / 2 columns,
 *        C[i, j] = act(z[i, 2j]) * z[i, 2j + 1] + residual[i, j].
 *   a         [m, k] and w [n, k], both of ab_dtype: F16, BF16 or E4M3; 16-byte aligned, every row starts on a
 *             16-byte boundary (k may be any)
 *   a_scale   float [m] or NULL, w_scale float [n] or NULL (any ab_dtype), bias float [n] or NULL
 *   residual  [m, columns of C] F32, F16 or BF16, or NULL; may be c itself where type and stride are c's
 *   c         [m, n or n / 2] F32, F16 or BF16; may not overlap a or w
 * Device pointers.  Products are summed in fp32 on the tensor cores, everything after them in fp32, rounded once.  The tensor cores
 * truncate: terms of one sign lose up to 2.5e-5 of their sum before it is added in registers that round (1e-4 with 16 bits out).
 * The order of a sum depends on the sizes (m among them), never on values or timing: equal calls give equal bits. */
typedef struct {
  const void* a;
  const void* w;
  const float* a_scale;
  const float* w_scale;
  const float* bias;
  const void* residual;
  void* c;
  int64_t a_stride, w_stride, residual_stride, c_stride;
  int32_t m, n, k;
  int32_t ab_dtype, c_dtype, residual_dtype;
  int32_t act, gated;
} hb_linear_args;
HB_API int hb_linear(hb_ctx* ctx, const hb_linear_args* args, void* stream);

/* hb_linear where rows group_start[g] .. group_start[g + 1] - 1 of a, c and residual take the g-th w, w_scale and
 * bias: w [n_groups][n, k] with w_group_stride elements between them (a multiple of 16 bytes), w_scale and bias
 * [n_groups, n].  Groups are an expert's rows, or the requests that share an adapter; a group may be empty.
 * group_start: device int32 [n_groups + 1], not decreasing, in 0 .. m; read on the device only, so a captured call sees what
 * it holds when it is replayed.  Rows before the first and behind the last group are left as they are.  A group that
 * starts below an earlier bound, ends before it starts or leaves 0 .. m is skipped and raises HB_STATUS_GROUP_INDEX.
 * n_groups <= HB_LINEAR_MAX_GROUPS. */
#define HB_LINEAR_MAX_GROUPS 512
HB_API int hb_linear_grouped(hb_ctx* ctx, const hb_linear_args* args, const int32_t* group_start, int32_t n_groups,
                             int64_t w_group_stride, void* stream);

/* Which kernel the two calls take for these sizes and types on a device of num_sms SMs (n_groups 0: hb_linear); host only, pointers and
 * strides are not looked at.  out[0]: rows of A per tile (8 and 16: the kernel for few rows; 256: a pair of CTAs), out[1]: blocks of 16
 * features of such a small tile, or the CTAs that share a tile's K, out[2]: how the sums leave (0 plain, 1 in segments, 2 sixteen warps). */
HB_API int hb_linear_variant(const hb_linear_args* args, int32_t n_groups, int32_t num_sms, int32_t out[3]);

/* The step with 8-bit projection weights: hb_mixed_step over an 8-bit cache (hb_kv8_create) whose four projections per layer
 * run on E4M3 operands.  Per layer: hb_norm to codes, hb_linear QKV, append and attention over the 8-bit cache,
 * hb_quant_rows of the attention's output, hb_linear O onto the residual stream, hb_norm, hb_linear gate/up with SwiGLU,
 * hb_quant_rows, hb_linear down onto the residual stream.  Embedding, gains, LM head, pooling and outputs are hb_mixed_step's.
 * Every projection weight is E4M3 codes, row-major [out, in] in hb_layer_weights' row order, 16-byte aligned, with a float
 * scale per row (hb_quant_rows of the model's rows gives both).  No adapters.  d_ffn and n_heads * head_dim are at most
 * HB_NORM_MAX_D (HB_ERR_TOO_LARGE).  A row's projections depend on the number of rows of the step in their last bits
 * (hb_linear), unlike hb_mixed_step's.
 * HB_STATUS_F16_RANGE: a normed row held a NaN or an infinity, or a row of the attention's output or of the SwiGLU held a
 * NaN or reached +-65504, where hb_linear saturates. */
typedef struct {
  const void *attn_norm, *ffn_norm;                 /* bf16 [d_model] */
  const void *wqkv, *wo, *w_gate_up, *w_down;       /* E4M3 codes */
  const float *wqkv_scale, *wo_scale, *gate_up_scale, *down_scale;
} hb_layer_weights8;
typedef struct {
  const void* tok_emb;               /* device */
  const hb_layer_weights8* layers;   /* HOST array [n_layers] of device ptrs   */
  const void* final_norm;            /* device */
  const void* lm_head;               /* device, fp16 */
} hb_weights8;
HB_API int hb_mixed_step8(hb_ctx* ctx, const hb_batch_desc* desc, const hb_weights8* w, hb_kv* kv, hb_pool* pool,
                          float* out_logits, float* out_emb, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HB_H_ */
