/*
 * tdp.h - C ABI of the MI355X pipeline-stage library.
 *
 * One "stage" is a contiguous slice of a Llama-style model's decoder layers held by one GPU
 * (paper Sec. 2.2.3: pipeline parallelism splits the model layer-wise, each device owning a
 * subset of layers).  A stage is told which batch to run and in which phase (Sec. 3.2: the
 * engine packs prompts for the prefill phase and decode steps for the decode phase; a worker
 * only knows what to compute); batches are never mixed (separate batching, Sec. 2.3, Sec. 3.1).
 * Hidden states come in from the previous stage and go out to the next: no embedding, no final
 * norm, no LM head.
 *
 * Conventions
 *  - All functions return TDP_OK (0) or a negative error code; tdp_last_error() gives a
 *    thread-local message for the most recent failure.
 *  - Argument checks run on the host before any GPU work, so a bad argument never launches.
 *  - "dev" pointers are device (HBM) addresses, "host" pointers are ordinary host addresses.
 *  - bf16 is the raw 16-bit brain-float encoding; matrices are row-major.
 *  - Calls that take a `stream` (a hipStream_t passed as void*, NULL = the default stream) only
 *    enqueue work and return; nothing synchronises with the host.  One stage must not be driven
 *    from two streams at once: its scratch buffers are shared.
 *  - The caller owns page allocation: which physical page belongs to which request is the
 *    engine's business (Sec. 3.2.1).  The stage only writes the slot the tables name.
 *    Contents of device-side tables are trusted by the prefill / decode / import / export calls:
 *    a page id outside [0, num_pages) or a position beyond 16 * max_pages_per_seq is undefined
 *    behaviour there (a decode step takes the nearest position of the row instead: that request's
 *    result means nothing, the others' and those of later calls are not touched).
 *    tdp_stage_check_decode / tdp_stage_check_prefill validate them first for a caller that wants
 *    that (they cost a synchronisation, so they are not part of the hot calls).
 */
#ifndef TDP_H_
#define TDP_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TDP_API __attribute__((visibility("default")))

#define TDP_OK       0
#define TDP_EINVAL  (-1)   /* null pointer, bad shape, size beyond the configured maximum */
#define TDP_ENOMEM  (-2)   /* device or host allocation failed */
#define TDP_EHIP    (-3)   /* a HIP runtime call failed (message holds the HIP error string) */

/* weight identifiers for tdp_stage_set_weight */
#define TDP_WQ      0      /* [d_model, n_q_heads*head_dim]  */
#define TDP_WK      1      /* [d_model, n_kv_heads*head_dim] */
#define TDP_WV      2      /* [d_model, n_kv_heads*head_dim] */
#define TDP_WO      3      /* [n_q_heads*head_dim, d_model]  */
#define TDP_WG      4      /* [d_model, d_ff]   gate         */
#define TDP_WU      5      /* [d_model, d_ff]   up           */
#define TDP_WD      6      /* [d_ff, d_model]   down         */
#define TDP_G_ATTN  7      /* [d_model] RMSNorm gain before attention */
#define TDP_G_MLP   8      /* [d_model] RMSNorm gain before the MLP   */
/* optional biases of the q / k / v projections (the Qwen2.5-32B model of the paper's Table 2 has
 * them; a stage whose biases are never set runs without): vectors [d_q, 1], [d_kv, 1], [d_kv, 1] */
#define TDP_BQ 9
#define TDP_BK 10
#define TDP_BV 11

#define TDP_F32     0
#define TDP_BF16    1

#define TDP_HOST    0
#define TDP_DEVICE  1

/* element type of the KV pools (tdp_stage_config.kv_dtype) */
#define TDP_KV_BF16      0
#define TDP_KV_FP8_E4M3  1   /* OCP 8-bit float, 4 exponent bits (bias 7), 3 mantissa bits, max 448, no infinities */

typedef struct tdp_stage tdp_stage;   /* opaque: owns weights, KV pools and scratch (all in HBM) */

typedef struct tdp_stage_config {
  int32_t n_layers;            /* decoder layers in this stage (>= 1) */
  int32_t d_model;             /* multiple of 64 */
  int32_t n_q_heads;           /* multiple of n_kv_heads; group size n_q_heads/n_kv_heads <= 16 */
  int32_t n_kv_heads;
  int32_t head_dim;            /* 64 or 128 */
  int32_t d_ff;                /* SwiGLU width, multiple of 4 */
  float   rms_eps;
  float   rope_base;
  int32_t page_size;           /* tokens per KV page; must be 16 */
  int32_t num_pages;           /* physical pages per layer in the KV pool */
  int32_t max_batch;           /* largest decode batch */
  int32_t max_tokens;          /* largest packed prefill token count */
  int32_t max_seqs;            /* largest number of prompts in one prefill */
  int32_t max_pages_per_seq;   /* width of a block-table row */
  /* KV-cache element type.  The decode phase is bound by reading the cache (Sec. 2.1); the paper keeps
   * it in the model's 16-bit type (TDP_KV_BF16, the default and what every headline number uses).
   * TDP_KV_FP8_E4M3 stores each key (after rotation) and value as the E4M3 code of value / scale:
   * round to nearest, ties to the even code, magnitudes from 448 up saturate, NaN stays NaN; the
   * quotient is an fp32 division.  Attention in both phases reads the cache, i.e. code * scale (the
   * code value is exact in bf16; the scales join the softmax scale and the final normalisation), and
   * is otherwise unchanged.  k_scale / v_scale: per stage, > 0; 0 means 1. */
  int32_t kv_dtype;
  float   k_scale, v_scale;
  /* Decode batches as two half-batches on two streams (0 or 1: off, the default; 2: on).  The decode
   * phase alternates a step bound by reading the cache (attention) with steps bound by the matrix
   * cores (the projections, Sec. 2.1 and Sec. 3.4); with two half-batches in flight one half's attention
   * may run beside the other half's projections.  The stage then holds a second set of scratch buffers
   * and a second stream of its own (default priority); tdp_stage_decode forks it behind the work already
   * queued on the caller's stream and joins it before returning control of that stream, so callers see
   * the same semantics (graph capture included).  Results equal the one-batch form's within rounding;
   * per-class timing is not recorded in this form.  Measured slower than one batch on MI355X at the
   * benchmark shapes (each half streams all weights again): an option, not the default. */
  int32_t decode_micro_batches;
} tdp_stage_config;

/* Version of this ABI (bumped on incompatible change). */
TDP_API int tdp_abi_version(void);

/* Message for the calling thread's most recent error ("" if none).  Never NULL. */
TDP_API const char* tdp_last_error(void);

/*
 * Create a stage: allocates weights (zeroed), per-layer K and V pools and scratch on the current
 * HIP device.  `*out` is set only on success.  Errors: TDP_EINVAL (bad config), TDP_ENOMEM,
 * TDP_EHIP.  The config is checked before any HIP call.
 */
TDP_API int tdp_stage_create(const tdp_stage_config* cfg, tdp_stage** out);

/* Free everything the stage owns.  NULL is allowed.  Synchronises the device first. */
TDP_API void tdp_stage_destroy(tdp_stage* st);

/*
 * Load one weight.  `src` is a row-major [rows, cols] = [in, out] matrix (y = x W) or a vector
 * [rows] with cols = 1, of type `dtype` (TDP_F32 or TDP_BF16; fp32 is rounded to bf16 with
 * round-to-nearest-even, gains are kept in fp32), living where `mem` says (TDP_HOST or
 * TDP_DEVICE).  The library repacks it once into its own MFMA-friendly layout; `src` is not
 * referenced after the call returns.  The call waits for the device's work on all streams before it reads
 * the source and replaces the weight, and for its own before it returns.  Shapes must match the config.
 */
TDP_API int tdp_stage_set_weight(tdp_stage* st, int32_t layer, int32_t which, const void* src,
                         int32_t dtype, int32_t mem, int64_t rows, int64_t cols);

/*
 * Raw access to one layer's KV pools, for tests that poison, inject or dump them.
 * Layout:  K pool [num_pages][n_kv_heads][R / 64][16][64 bytes]   (R = bytes of one key row)
 *          V pool [num_pages][n_kv_heads][head_dim][16]             (token slot fastest)
 * of bf16 elements, or of one-byte E4M3 codes when kv_dtype = TDP_KV_FP8_E4M3.  A key row (head_dim
 * elements, R = 64 ... 256 bytes) is stored in 64-byte pieces, piece g of the page's 16 token slots
 * together: byte r of the key of (page, head, slot) lies at
 *   ((page * n_kv_heads + head) * 16 * R) + (r / 64) * 1024 + slot * 64 + r % 64
 * (what one decode-attention load instruction fetches, 64 bytes of each of 16 tokens, is then four
 * runs of 256 bytes instead of sixteen half cache lines).
 * Keys are stored after the rotary embedding.  `*bytes` = size of EACH pool.
 */
TDP_API int tdp_stage_kv_pool(tdp_stage* st, int32_t layer, void** k_dev, void** v_dev, int64_t* bytes);

/*
 * Copy K/V between packed logical order and the pages (the path a recompute-free migration or a
 * test would use).  k_packed / v_packed: dev bf16 [total_tokens][n_kv_heads][head_dim], the
 * sequences' tokens concatenated; token t of sequence s (cu_seqlens[s] <= t < cu_seqlens[s+1])
 * lives at position t - cu_seqlens[s], i.e. page block_tables[s][pos/16], slot pos%16.
 * cu_seqlens: dev int32 [n_seqs+1]; block_tables: dev int32 [n_seqs][max_pages_per_seq].
 * import writes pages from the packed arrays, export reads pages into them.  With an 8-bit cache
 * the packed side stays bf16: import stores the code of value / scale, export returns
 * bf16(code * scale).
 */
TDP_API int tdp_stage_kv_import(tdp_stage* st, int32_t layer, const void* k_packed, const void* v_packed,
                        const int32_t* cu_seqlens, const int32_t* block_tables, int32_t n_seqs,
                        int32_t total_tokens, void* stream);
TDP_API int tdp_stage_kv_export(tdp_stage* st, int32_t layer, void* k_packed, void* v_packed,
                        const int32_t* cu_seqlens, const int32_t* block_tables, int32_t n_seqs,
                        int32_t total_tokens, void* stream);

/*
 * Prefill phase (Sec. 2.1: all prompt tokens are processed concurrently and the KV cache is
 * initialised).  Runs every layer of the stage over `total_tokens` packed prompt tokens.
 *   hidden_in    dev bf16 [total_tokens][d_model]   packed var-length prompts
 *   cu_seqlens   dev int32 [n_seqs+1]               prefix sums of prompt lengths, [0] = 0
 *   block_tables dev int32 [n_seqs][max_pages_per_seq]; row s needs ceil(len_s/16) valid entries
 *   hidden_out   dev bf16 [total_tokens][d_model]   (may alias hidden_in)
 * Every prompt starts at position 0 on an empty cache (no chunked prefill, Sec. 2.3); attention
 * is causal within a prompt; K (rotated) and V of every token and layer are written to the
 * pages.  n_seqs <= max_seqs, total_tokens <= max_tokens, each prompt <= 16*max_pages_per_seq.
 * n_seqs = 0 or total_tokens = 0 is a successful no-op.
 */
TDP_API int tdp_stage_prefill(tdp_stage* st, const void* hidden_in, const int32_t* cu_seqlens,
                      const int32_t* block_tables, int32_t n_seqs, int32_t total_tokens,
                      void* hidden_out, void* stream);

/*
 * Decode phase (Sec. 2.1: each step processes one new token per request using the KV cache).
 *   hidden_in    dev bf16 [batch][d_model]          one token per request
 *   ctx_lens     dev int32 [batch]                  tokens ALREADY cached for request b; the new
 *                                                   token takes position ctx_lens[b]
 *   block_tables dev int32 [batch][max_pages_per_seq]; row b needs ceil((ctx_lens[b]+1)/16) entries
 *   hidden_out   dev bf16 [batch][d_model]          (may alias hidden_in)
 * For every layer the new token's K (rotated) and V are appended at page
 * block_tables[b][ctx/16], slot ctx%16 BEFORE attention, which then spans ctx+1 tokens.
 * ctx_lens[b] = 0 is legal.  batch <= max_batch; batch = 0 is a successful no-op.  Re-running a
 * step with the same inputs rewrites the same slots with the same values.
 */
TDP_API int tdp_stage_decode(tdp_stage* st, const void* hidden_in, const int32_t* ctx_lens,
                     const int32_t* block_tables, int32_t batch, void* hidden_out, void* stream);

/*
 * Validate the device-side tables of a decode or prefill call before making it.  Checked, for every
 * row of the batch: the length (decode: 0 <= ctx_lens[b] and ctx_lens[b] + 1 <= 16 * max_pages_per_seq;
 * prefill: 0 <= len_s <= 16 * max_pages_per_seq, cu_seqlens[0] = 0, cu_seqlens[n_seqs] = total_tokens);
 * every table entry the call would use lies in [0, num_pages); and no page that the call writes
 * (decode: the page of position ctx_lens[b]; prefill: every page of every prompt) appears a second
 * time among the entries the call uses - two requests writing one page, or one reading what another
 * writes, is how a page-allocation mistake shows (the engine owns allocation, Sec. 3.2.1).  Pages
 * that are only read may be shared.  The kernels read the tables inside [rows][max_pages_per_seq]
 * whatever the lengths say, so the check itself is safe on arbitrary input.
 * Returns TDP_OK, or TDP_EINVAL with a message naming the first offending row and what is wrong
 * with it.  Same size limits and pointer kinds as the call it guards.  Runs on `stream` and waits for it.
 */
TDP_API int tdp_stage_check_decode(tdp_stage* st, const int32_t* ctx_lens, const int32_t* block_tables,
                                   int32_t batch, void* stream);
TDP_API int tdp_stage_check_prefill(tdp_stage* st, const int32_t* cu_seqlens, const int32_t* block_tables,
                                    int32_t n_seqs, int32_t total_tokens, void* stream);

/*
 * Restrict the following prefill/decode calls to layers [first, first + count) of the stage, as
 * if the stage were that sub-slice (a finer pipeline split, or a layer-by-layer check against a
 * reference).  The hand-over format at both ends stays bf16.  count = 0 restores the whole stage.
 * Errors: TDP_EINVAL when the range does not lie inside [0, n_layers).
 */
TDP_API int tdp_stage_set_layer_range(tdp_stage* st, int32_t first, int32_t count);

/*
 * Decode attention splits a request's context into spans of `span_tokens` logical tokens, one
 * workgroup per (span, K/V head), and merges the spans' partial softmax states in a fixed logical
 * order (Sec. 2.1: a decode step reads the request's whole cache).  By default the span is chosen
 * from batch x K/V heads so that small batches still fill the GPU; this call pins it for the
 * following decode calls (tuning, and tests that walk every span length).  span_tokens: 0 =
 * automatic, else 256, 512, 1024, 2048 or 4096.  Results agree within rounding whatever the span.
 */
TDP_API int tdp_stage_set_decode_span(tdp_stage* st, int32_t span_tokens);

/*
 * Diagnostic: one projection GEMM through the library's kernels, out = A * W with W given as
 * a row-major [K, N] bf16 device matrix (repacked internally on every call: not a fast path).
 * A dev bf16 [M][K]; out dev bf16 [M][N].  K multiple of 64, N multiple of 4.
 * tile: 0 = automatic, 1..3 force a kernel variant (256 x 256, 128 x 256, 128 x 128 output tile);
 * splits: 0 = automatic, else force the split-K factor.  epilogue: 0 = plain store; 1 = out =
 * residual + A*W (residual dev bf16 [M][N]); 2 = the gated MLP epilogue (Sec. 3.4 counts the MLP among
 * the linear layers that dominate a decode step): W = [W_gate | W_up] side by side, N = 2 F, and
 * out dev bf16 [M][F] = silu(A*W_gate) * (A*W_up) with silu(z) = z / (1 + exp(-z)); F multiple of 4.
 */
TDP_API int tdp_gemm_bf16(const void* A, const void* W, const void* residual, void* out, int32_t M, int32_t N,
                  int32_t K, int32_t epilogue, int32_t tile, int32_t splits, void* stream);

/*
 * Diagnostic, on the host alone: how the library makes a projection of this shape (epilogues as in
 * tdp_gemm_bf16).  deferred = 1: as a stage makes its QKV (epilogue 0), O and down (1) projections,
 * the fp32 partials of a split summed by the kernel behind it.  workspace_elems: floats that the partials
 * may take (tdp_gemm_bf16: 16 * M * N with N rounded up to 256, or to 2 * 128 columns of F).  plan (host int32 [5]):
 * tile number, output rows and weight rows of a tile, split-K factor, and the k of one chunk where a
 * workgroup sums its K range in chunks (0: in one go).
 */
TDP_API int tdp_gemm_plan(int32_t M, int32_t N, int32_t K, int32_t epilogue, int32_t deferred, int64_t workspace_elems,
                          int32_t* plan);

/*
 * Diagnostic, on the host alone: the same for a product of 8-bit integers (tdp_linear_i8_run, TDP_E_LM_HEAD_I8) that is made in
 * tiles; the kernels for small batches have none.  workspace_elems: of a tdp_linear_i8 as tdp_linear_i8_set_form says, of a tdp_ends
 * 2 * min(rows, 512) * N, rows = max_tokens rounded up to 2 and N to 256.  plan (host int32 [4]): as the first four there.
 */
TDP_API int tdp_gemm_plan_i8(int32_t M, int32_t N, int32_t K, int32_t gated, int64_t workspace_elems, int32_t* plan);

/*
 * Diagnostic: tdp_gemm_bf16 made in exactly one way, so that every kernel variant can be tested whatever
 * the plan would take: tile = a tile number of tdp_gemm_plan (from 1), splits = the split-K factor (one
 * that leaves no split empty), chunk_k = 0 or a multiple of 64: a workgroup sums its K range in chunks of
 * that many (splits = 1, tiles of at most 96 x 128 and the 128 x 128 one made for it).  TDP_EINVAL if
 * there is no such form.
 */
TDP_API int tdp_gemm_bf16_form(const void* A, const void* W, const void* residual, void* out, int32_t M, int32_t N,
                               int32_t K, int32_t epilogue, int32_t tile, int32_t splits, int32_t chunk_k,
                               void* stream);

/*
 * tdp_gemm_bf16 (epilogues 0 and 1) for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): same kernels, same results, but
 * the repacked weights and the split-K partials live in a device array that is part of the library
 * image (64 MiB per GPU, held until the process ends) instead of two allocations per call.  The
 * call allocates and frees nothing and only enqueues on `stream` (it does not wait; the caller
 * synchronises before reading `out`).  Limits: N rounded up to a multiple of 256, times K, at most
 * 8 Mi elements (16 MiB of weights); (splits, or 16 when splits = 0) * M * that N at most 12 Mi
 * floats (48 MiB of partials); anything larger is TDP_EINVAL with a message naming the limit, checked
 * before any GPU work.  All calls on one GPU share the one array: calls that may overlap (different
 * streams without an order between them, or several threads) race; calls on one stream are safe.
 */
TDP_API int tdp_gemm_bf16_static(const void* A, const void* W, const void* residual, void* out, int32_t M,
                                 int32_t N, int32_t K, int32_t epilogue, int32_t tile, int32_t splits, void* stream);

/*
 * Diagnostics for the 8-bit cache format: the conversions exactly as the KV kernels perform them.
 * tdp_e4m3_from_f32: codes[i] = E4M3 code of src[i] / scale (dev fp32 -> dev bytes; scale > 0).
 * tdp_e4m3_to_f32:   dst[i] = value of codes[i] (dev bytes -> dev fp32), through the conversion
 *                    instruction the decode-attention kernel uses; n a multiple of 4, codes 4-byte
 *                    and dst 16-byte aligned.
 */
TDP_API int tdp_e4m3_from_f32(const float* src, uint8_t* codes, int64_t n, float scale, void* stream);
TDP_API int tdp_e4m3_to_f32(const uint8_t* codes, float* dst, int64_t n, void* stream);

/*
 * Empirical ceilings of the GPU the library runs on, for the benchmark's roofline context (the
 * decode phase is bound by memory bandwidth and the prefill phase by compute, Sec. 2.1; these say
 * what the part sustains for either with no other work in the way).  Both calls launch a trivial
 * kernel `launches` times (1..1000) after one warm-up, time the launches with HIP events on
 * `stream`, wait for them and return the average milliseconds per launch in *ms_per_launch (host).
 * tdp_probe_hbm_read: reads the first 2^k * 4 KiB of `buf` (dev, 16-byte aligned, at least 512 KiB;
 *   2^k * 4 KiB is the largest such size <= bytes, returned in *bytes_per_launch) exactly once per
 *   launch, 16 bytes per lane per instruction, 16 KiB in flight per wave.  pattern bit 0: 0 walks the
 *   4 KiB pieces in address order, 1 in a fixed pseudo-random order (how a paged KV cache is read);
 *   bit 1: the loads are marked non-temporal, as the library's own kernels mark data they read once
 *   (keys and values in decode, weights of a GEMM with a single row of tiles).  Nothing is written to `buf`.
 * tdp_probe_mfma_bf16: `iters` (1..2^22) rounds of sixteen independent 16x16x32 bf16 MFMAs per wave on
 *   register operands, two waves per SIMD on every CU; *flop_per_launch (host) = multiply-adds * 2.
 *   random_operands = 1: operands uniform in (-1, 1), different in every lane and element; 0: the
 *   same constants everywhere (the rate depends on it: the part is power-limited and an MFMA's
 *   power grows with the operand bits that toggle).
 * Errors: TDP_EINVAL (null pointer, size or count out of range), TDP_ENOMEM, TDP_EHIP.
 */
TDP_API int tdp_probe_hbm_read(const void* buf, int64_t bytes, int32_t pattern, int32_t launches,
                               int64_t* bytes_per_launch, float* ms_per_launch, void* stream);
TDP_API int tdp_probe_mfma_bf16(int32_t iters, int32_t launches, int32_t random_operands, double* flop_per_launch,
                                float* ms_per_launch, void* stream);

/*
 * Timing hooks: when enabled, prefill/decode record HIP events around each kernel class on the
 * call's stream; tdp_stage_timing_read synchronises and returns the summed milliseconds of the
 * most recent call per class (order: rmsnorm, gemm_qkv, rope_kv, attention, gemm_o, gemm_gate_up,
 * gemm_down, attention_merge) into ms[8].  "attention" is the attention kernel (prefill or
 * decode).  The partial results of decode requests longer than one span are combined inside it, or, for
 * large batches of long contexts, by a kernel behind it, whose class is "attention_merge" (0 otherwise).  It also
 * rotates and appends in small decode batches: "rope_kv" is 0 there.  In a prefill whose QKV projection is made
 * unsplit in tiles of 256 weight rows, on a 16-bit cache, queries and keys are rotated and keys appended by the
 * projection, within "gemm_qkv"; "rope_kv" is then the append of the values alone.
 */
TDP_API int tdp_stage_timing_enable(tdp_stage* st, int32_t on);
TDP_API int tdp_stage_timing_read(tdp_stage* st, float* ms /* host [8] */);

/* ---- projections in 8-bit integers -----------------------------------------------------------------
 * y = x W with both held as 8-bit integers, a scale for each row of x (token) and each column of W (output
 * channel), and exact sums: half the bytes of a bf16 projection to stream (what bounds a decode step's projections,
 * Sec. 3.4) and twice its matrix rate.  A vector v is held as codes c and a scale: with a = max |v| the scale is a / 127
 * and c = rint(v * (127 / a)), each operation rounded in fp32; an element is off by at most (1/2 + 2^-15) scales, and 2^-143 more
 * where the scale is subnormal (a below 127 * 2^-126; a vector below 127 * 2^-150 has scale 0).
 *   y[m][n] = scale_x[m] * scale_w[n] * sum_k c_x[m][k] c_w[k][n]
 * The sum is a whole number, so a row's result does not depend on the other rows of the call.  A row or column that holds an
 * infinity or a NaN has scale NaN, and with it its whole result; one of zeros has scale 0.
 * A tdp_linear_i8 owns the codes and scales of one weight matrix and scratch for max_rows rows.  It lives on the
 * device that is current when it is created, and calls on it need that device current.  Like a stage it must not be driven from two
 * streams at once, nor by two captured graphs that replay at once.  Calls that set something wait for the device's work on all streams
 * first, and return when they are done. */
typedef struct tdp_linear_i8 tdp_linear_i8;
typedef struct {
  int32_t in_features;   /* K: a multiple of 8, at most 131072 */
  int32_t out_features;  /* N: a multiple of 4; gated: of 8; at most 2^24 */
  int32_t gated;         /* 1: W = [W_gate | W_up] side by side, as in tdp_gemm_bf16: the result has N / 2 columns */
  int32_t max_rows;      /* rows per call, at most 2^21 */
} tdp_linear_i8_config;
TDP_API int tdp_linear_i8_create(const tdp_linear_i8_config* cfg, tdp_linear_i8** out);
TDP_API void tdp_linear_i8_destroy(tdp_linear_i8* h);
/* W row-major [K, N], host or device, fp32 or bf16: quantised column by column and laid out.  Synchronous. */
TDP_API int tdp_linear_i8_set_weight(tdp_linear_i8* h, const void* src, int32_t dtype, int32_t mem, int64_t rows, int64_t cols);
/* A matrix that is quantised already: codes int8 row-major [K, N] and fp32 scales [N], both where mem says.  Synchronous. */
TDP_API int tdp_linear_i8_set_codes(tdp_linear_i8* h, const int8_t* codes, const float* scales, int32_t mem, int64_t rows, int64_t cols);
/* Added to every row of an ungated result: [N], fp32 or bf16.  Synchronous. */
TDP_API int tdp_linear_i8_set_bias(tdp_linear_i8* h, const void* src, int32_t dtype, int32_t mem, int64_t n);
/* Tuning and tests: the following calls make the product in exactly one way, tile = a tile number of tdp_gemm_plan (not the one that is
 * made for chunked sums), splits = the split-K factor (over k-tiles of 128, none of them empty); tile = 0: planned, the default.  A call whose
 * partials exceed the workspace (8 * min(max_rows, 512) * N, N rounded up to 256, at most 64 Mi) is then TDP_EINVAL.  Results are the same
 * to the bit. */
TDP_API int tdp_linear_i8_set_form(tdp_linear_i8* h, int32_t tile, int32_t splits);
/* out[m] = y[m] (+ bias) (+ residual[m]), or silu(gate) * up if gated, for M <= max_rows rows (M = 0: nothing to do).
 *   x          dev, x_dtype, rows ld_x elements apart, 16-byte aligned: quantised by the call
 *   residual   dev, out_dtype, rows ld_residual elements apart, or null; gated: null.  May be out itself (address and ld_out)
 *   out        dev, out_dtype, rows ld_out elements apart: [M][N], gated [M][N / 2]; columns behind those are left as they are.  Shares
 *              no element with x
 * TDP_F32 or TDP_BF16 each; out and residual aligned to four elements, row by row.  Sums, scales, bias and residual are joined in fp32
 * and rounded once.  With u = 2^-24 the fp32 number is off by 3 u of y (sum, times scale_w, times scale_x, while these are normal
 * numbers), and u of what each addition gives; gated by (4 |g| + 16) u of itself, g the gate in front of silu, and gates below -87 may
 * give 0. */
TDP_API int tdp_linear_i8_run(tdp_linear_i8* h, const void* x, int32_t x_dtype, int64_t ld_x, int32_t M, const void* residual,
                              int64_t ld_residual, void* out, int32_t out_dtype, int64_t ld_out, void* stream);

/* ---- the two ends of the pipeline ---------------------------------------------------------------
 * What runs in front of the first stage and behind the last one so that a chain of stages turns
 * token ids into token ids (the paper measures generated tokens per second on whole models, Sec.
 * 4.1 and Table 2): the token-embedding lookup, and the final RMSNorm + vocabulary projection +
 * greedy selection.  A tdp_ends owns the embedding table (bf16 [vocab, d_model]), the final norm
 * gain (fp32) and the vocabulary projection (bf16, repacked once), plus scratch for max_tokens rows.
 * vocab_size must be a multiple of 4, d_model a multiple of 64.
 * The object lives on the device that is current when it is created, and calls on it need that device current (TDP_EINVAL). */
typedef struct tdp_ends tdp_ends;
typedef struct {
  int32_t vocab_size, d_model;
  float rms_eps;
  int32_t max_tokens; /* rows per call */
} tdp_ends_config;
#define TDP_E_EMBEDDING 0  /* [vocab_size, d_model] */
#define TDP_E_FINAL_NORM 1 /* [d_model, 1] */
#define TDP_E_LM_HEAD 2    /* [d_model, vocab_size] row-major ([in, out] like every projection) */
#define TDP_E_LM_HEAD_I8 3 /* the same, held in 8-bit integers with a scale for each token of the vocabulary (see tdp_linear_i8); the
                              rows are then quantised behind the final norm.  d_model is at most 131072.  The projection is in the
                              form that was set last.  The bf16 matrix's memory is given back if none was set before and no call has
                              read it (zeros); setting one takes it again. */
TDP_API int tdp_ends_create(const tdp_ends_config* cfg, tdp_ends** out);
TDP_API void tdp_ends_destroy(tdp_ends* e);
/* src: host or device (mem), fp32 or bf16 (dtype).  Waits for the device's work on all streams first (a source may be written by any,
 * and calls on any may still read the weight that is replaced), and returns when it is done. */
TDP_API int tdp_ends_set_weight(tdp_ends* e, int32_t which, const void* src, int32_t dtype, int32_t mem,
                                int64_t rows, int64_t cols);
/* hidden_out[m][:] = embedding[token_ids[m]][:].  token_ids dev int32 [M]; hidden_out dev bf16
 * [M, d_model].  An id outside the vocabulary is clamped into it (never a wild read).  Enqueues on
 * stream and returns. */
TDP_API int tdp_embed_tokens(tdp_ends* e, const int32_t* token_ids, int32_t M, void* hidden_out, void* stream);
/* For row m: x = hidden_in[row_index ? row_index[m] : m]; logits[m] = RMSNorm(x; gain) * W_head;
 * next_token[m] = the lowest index among the largest logits.  hidden_in dev bf16 [n_rows_in,
 * d_model]; row_index dev int32 [M] or null (prefill: the last token of each prompt), entries are
 * clamped to [0, n_rows_in); logits_out dev fp32 [M, vocab_size] or null (internal scratch);
 * next_token dev int32 [M] or null.  M <= max_tokens.  fp32 accumulation, fp32 logits. */
TDP_API int tdp_lm_head(tdp_ends* e, const void* hidden_in, int32_t n_rows_in, const int32_t* row_index, int32_t M,
                        float* logits_out, int32_t* next_token, void* stream);
/* Greedy selection alone: out[m] = lowest index among the maxima of logits[m][0..n), rows ld apart.
 * All device pointers.  NaN entries never win; a row of NaNs gives 0. */
TDP_API int tdp_argmax_rows(const float* logits, int32_t M, int32_t n, int64_t ld, int32_t* out, void* stream);

/* Log-probabilities of given logits: for every row m of [M][n] logits (dev, TDP_F32 or TDP_BF16, rows ld >= n elements apart, at any
 * alignment of their type; n up to 2^30)
 *   logprob[m]     ln p of token targets[m] (dev int32 [M]); a target outside [0, n), such as -1 for none, has minus infinity.
 *                  targets null: of the row's largest logit
 *   entropy[m]     - sum p ln p, in nats
 *   top_index[m][j], top_logprob[m][j], j < n_top: the likeliest tokens in order, of equal ones the lower index first (dev int32 / fp32
 *                  [M][n_top]); n_top 0 .. TDP_MAX_TOP, at most n
 * with p = softmax of the row.  logprob and entropy may be null, and top_index and top_logprob with n_top = 0.  Logits of minus infinity are
 * tokens of probability 0.  A row with a NaN or plus infinity, or with nothing but minus infinity, has no distribution: its logprob
 * (but for targets outside), entropy and top_logprob are NaN; top_index still orders its logits, without the NaN, and is -1 behind
 * the last.  Sums are fp32, relative to the row's maximum. */
#define TDP_MAX_TOP 32
TDP_API int tdp_logprob_rows(const void* logits, int32_t dtype, int32_t M, int32_t n, int64_t ld, const int32_t* targets, int32_t n_top,
                             float* logprob, float* entropy, int32_t* top_index, float* top_logprob, void* stream);
/* The same behind tdp_lm_head's norm and projection (hidden_in, n_rows_in, row_index, M as there), with the greedy token as
 * there in next_token (dev int32 [M] or null): what an engine answers a token with, or, with a prompt's own next tokens as targets, what
 * scores it.  Logits are kept inside, and where neither next_token nor n_top asks for tokens they are not stored at all.  An ends
 * object must not be driven from two streams at once, nor by two captured graphs that replay at once. */
TDP_API int tdp_lm_head_logprobs(tdp_ends* e, const void* hidden_in, int32_t n_rows_in, const int32_t* row_index, int32_t M,
                                 const int32_t* targets, int32_t n_top, int32_t* next_token, float* logprob, float* entropy,
                                 int32_t* top_index, float* top_logprob, void* stream);

/* ---- several continuations of a prompt -------------------------------------------------------------
 * What a batch needs whose rows continue one another's tokens: the choice of the likeliest continuations over beams and vocabulary,
 * block tables that fork and pages that are copied when they do, and attention that reads a prefix which several rows share
 * once.  All of it works on device memory and only enqueues, so that a step (attention, head, choice, tables, copies) needs no host. */

/* Beam selection.  The rows of logits are beams, `beams` of them to a group (a request).  Beam b of a group, with the score s_b it has so
 * far, can be continued by every token t at
 *   c(b, t) = s_b + z_b[t] - ln sum_j exp z_b[j];      a finished beam by end_token alone, at s_b.
 * For every group the n_out best continuations are given in order, of equal ones the lower beam first, then the larger logit, then the lower
 * token:
 *   parent[g][j]    row of logits that it continues (group * beams + beam)
 *   token[g][j], score[g][j]
 *   finished_out[g][j]   1 if the token is end_token, else 0 (may be null)
 * A continuation of minus infinity or NaN is none (a beam whose score is minus infinity, a masked token, and a row with a NaN, with plus
 * infinity or with nothing but minus infinity, which has no distribution); places behind the last have parent and token -1, score minus
 * infinity, finished_out 0.  The candidates are formed and compared in 64 bits, but for the exponentials, which are fp32 numbers relative to
 * the row's largest logit m: its own is exactly 1 (a row held to one token costs nothing), and ln sum is off by at most
 * 2^-23 sum_{z < m} p (1 + m - z) + n 2^-53, p the tokens' probabilities.
 *   logits   dev, TDP_F32 or TDP_BF16, [n_groups * beams][n], rows ld >= n elements apart, at any alignment of their type
 *   scores   dev fp32 [n_groups * beams]; the results overlap neither them nor one another (finished_out may be finished itself)
 *   finished dev int32 [n_groups * beams], not 0: finished; or null.  end_token: in [0, n), or, with finished null, -1: none
 * beams 1 .. TDP_MAX_BEAMS, n_out 1 .. TDP_MAX_TOP and at most beams * n, n up to 2^27, n_groups * beams <= max_rows (0: nothing to do).
 * A tdp_beams owns scratch.  It lives on the device that is current when it is created, calls on it need that device current, and it must
 * not be driven from two streams at once, nor by two captured graphs that replay at once. */
#define TDP_MAX_BEAMS 32
typedef struct tdp_beams tdp_beams;
typedef struct {
  int32_t max_rows; /* rows of logits per call, 1 .. 2^16 */
  int32_t max_out;  /* n_out, 1 .. TDP_MAX_TOP */
} tdp_beams_config;
TDP_API int tdp_beams_create(const tdp_beams_config* cfg, tdp_beams** out);
TDP_API void tdp_beams_destroy(tdp_beams* h);
TDP_API int tdp_beams_select(tdp_beams* h, const void* logits, int32_t dtype, int32_t n_groups, int32_t beams, int32_t n, int64_t ld,
                             const float* scores, const int32_t* finished, int32_t end_token, int32_t n_out, int32_t* parent,
                             int32_t* token, float* score, int32_t* finished_out, void* stream);

/* Block tables that fork.  A row is a length, lens[r] tokens, and the ceil(lens[r] / 16) first entries of its table row: the pages that hold
 * them.  refs[p] counts the table entries that name page p, and whoever else holds it (prompts kept for later, other batches); a page with
 * refs 0 is free.  tdp_pages_fork makes n_dst new rows from n_src old ones:
 *   - row r continues row parents[r] (-1: a new, empty row) with room for add[r] more tokens (add null: add_all for every row), so
 *     dst_lens[r] = src_lens[parents[r]] + add[r].  parents null: row r continues row r, rows from n_src on are new
 *   - full pages are shared.  A last page that is partly filled can be written by one row only: the first (lowest) row that continues its
 *     row takes it over, if it is named nowhere else (refs 1); every other one gets a fresh page in its place, and copies[r] = (that page, the
 *     fresh one), to be given to tdp_stage_kv_copy_pages of every stage that holds these pages; copies[r] = (-1, -1) otherwise
 *   - old rows that nothing continues are released, and with them the pages that nothing names any more
 * Fresh pages are those with refs_in 0, lowest ids first, dealt to the rows in order and within a row to its entries in order; pages
 * released by a call are free from the next one on, so no page is read and written by the copies of one call.
 * refs_out may be refs_in itself.  status (dev int32 [4]): pages that are missing, rows that are refused (a parent or length out of range, a
 * last page outside the pool), fresh pages taken, pages that were free.  If a page is missing or a row refused nothing happens: refs_out is
 * refs_in, copies are (-1, -1), dst_tables and dst_lens are left as they are.  Entries of dst_tables behind a row's pages are -1.
 * n_src = 0 makes new rows alone, n_dst = 0 releases all.  Page ids in src_tables are trusted as everywhere; reference counts of ids
 * outside the pool are skipped.
 *   parents, add, dst_lens dev int32 [n_dst]; copies dev int32 [n_dst][2]; src_lens dev int32 [n_src]; src_tables, dst_tables
 *   dev int32 [n_src], [n_dst] [max_pages_per_seq]; refs_in, refs_out dev int32 [num_pages].  But for refs_out, no output overlaps an input or
 *   another output. */
typedef struct tdp_pages tdp_pages;
typedef struct {
  int32_t num_pages;          /* 1 .. 2^22 */
  int32_t max_rows;           /* rows on either side, 1 .. 8192 */
  int32_t max_pages_per_seq;  /* width of a block-table row, up to 2^16 */
} tdp_pages_config;
TDP_API int tdp_pages_create(const tdp_pages_config* cfg, tdp_pages** out);
TDP_API void tdp_pages_destroy(tdp_pages* h); /* owns scratch alone; a device, streams and graphs as a tdp_beams */
TDP_API int tdp_pages_fork(tdp_pages* h, const int32_t* parents, const int32_t* src_tables, const int32_t* src_lens, int32_t n_src,
                           const int32_t* add, int32_t add_all, int32_t n_dst, const int32_t* refs_in, int32_t* refs_out,
                           int32_t* dst_tables, int32_t* dst_lens, int32_t* copies, int32_t* status, void* stream);
/* Pages in use moved towards the front of the pool, at most max_moves of them: the k-th move takes the k-th highest movable page to the k-th
 * lowest free one, as long as that is lower.  Movable are pages that the n_rows given rows name and nobody else holds (refs equal to
 * the entries that name them); others stay.  dst_tables (may be src_tables itself) are the rows with the new ids, -1 behind a row's pages,
 * moves (dev int32 [max_moves][2]) the (old, new) ids for tdp_stage_kv_copy_pages, (-1, -1) behind the last.  status: 0, rows that are
 * refused (a length out of range, an id outside the pool; nothing moves then), moves, pages in use.  max_moves 1 .. 2^22.  refs_out may be
 * refs_in itself; apart from these two no output overlaps an input or another output. */
TDP_API int tdp_pages_compact(tdp_pages* h, const int32_t* src_tables, const int32_t* lens, int32_t n_rows, int32_t max_moves,
                              const int32_t* refs_in, int32_t* refs_out, int32_t* dst_tables, int32_t* moves, int32_t* status,
                              void* stream);
/* Keys and values of whole pages copied within the stage, in all its layers: page pairs[i][0] to page pairs[i][1], i < n (dev int32
 * [n][2]).  Pairs with an id outside [0, num_pages) are skipped.  The pairs are independent: no page is the target of two, nor the target
 * of one and the source of another. */
TDP_API int tdp_stage_kv_copy_pages(tdp_stage* st, const int32_t* pairs, int32_t n, void* stream);

/* Attention of rows that share prefixes.  Rows group_starts[g] .. group_starts[g + 1] - 1 of the batch (dev int32 [n_groups + 1], from 0 to batch,
 * ascending; a group may be empty) are a group: rows whose block tables may begin with the same pages, such as the beams of a prompt or requests
 * behind one system prompt.  The leading whole pages in which the tables of all rows of a group agree, in front of every row's last
 * token, are found in the tables and read once for the group; so results are those of attention row by row, within rounding, whatever
 * the groups are.  n_groups = 0 (group_starts null): every row for itself.  n_groups <= max_batch.
 * Pages that only some rows of a group share are read by each of them: a row of other origin belongs into a group of its own.  A prefix of
 * fewer than 16 pages is shared only as long as no row of the group has more than 256 tokens behind it.  (tdp_stage_prefill begins at position 0 and
 * writes all pages of its prompts, so what a request has of its own behind a prefix that exists already is fed to decode steps.)  Groups pay from some
 * 130 to 350 MB of keys and values per layer on that rows would read of their prefixes one by one; below 100 MB tdp_stage_decode is the faster
 * step, by up to 20 us a layer.
 * tdp_stage_decode_shared is tdp_stage_decode with groups (one batch, whatever decode_micro_batches says).
 * tdp_stage_attend is the attention alone, on one layer's pools: row b attends to the lens[b] tokens that its pages hold,
 *   out[b][h] = sum_t softmax_t(q[b][h] . k[t][h / group] / sqrt(head_dim)) v[t][h / group],
 * zeros where lens[b] is 0 (or less; a length beyond 16 * max_pages_per_seq counts as that).  q dev bf16 [batch][n_q_heads][head_dim], rotated as
 * the keys are, 16-byte aligned; out the same, 8-byte aligned, not overlapping q; lens dev int32 [batch].  It writes no page.
 * Scores, softmax statistics and sums are fp32; probabilities are rounded to bf16 for the product with the values.  Both calls use the stage's
 * scratch, so they are ordered with its other calls, and need its device current. */
TDP_API int tdp_stage_attend(tdp_stage* st, int32_t layer, const void* q, const int32_t* lens, const int32_t* block_tables, int32_t batch,
                             const int32_t* group_starts, int32_t n_groups, void* out, void* stream);
TDP_API int tdp_stage_decode_shared(tdp_stage* st, const void* hidden_in, const int32_t* ctx_lens, const int32_t* block_tables, int32_t batch,
                                    const int32_t* group_starts, int32_t n_groups, void* hidden_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TDP_H_ */
