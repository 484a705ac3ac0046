/*
 * nnc.h - C ABI of the MI355X (gfx950) Qwen3-style decoder forward pass.
 *
 * The workload is the one the nncase paper compiles and times: the decode stage
 * (and the prompt pass before it) of Qwen3-0.6B / 1.7B at batch 1, tokens/s over
 * the decoding stage (Section 4, experimental setup; Sections 4.1 and 4.2), with
 * weights laid out once, ahead of time, in the layout the matmul micro-kernel
 * wants (Section 3.1.2 "Auto Vectorize": packed / blocked layouts; Section 3.3.1:
 * constants are pre-split and pinned; Section 3.3.2: MatMul micro-kernels over
 * packed operands).  Here the packed layout is the CDNA4 matrix-core fragment
 * order and the micro-kernels are hand-written HIP.
 *
 * Conventions for every entry point
 *   - returns nnc_status; never throws, never aborts; on error the out-params and
 *     the model state are left untouched and nnc_last_error() describes the cause;
 *   - "host" pointers are ordinary CPU memory read during the call only;
 *     "device" pointers are GPU memory owned by the caller, read or written by
 *     work enqueued on the model's stream; calls do not synchronise the stream
 *     (a long prompt's last pass runs on a second stream that the library creates
 *     and joins back to the model's stream with events before the call returns,
 *     see NNC_OPT_TAIL_OVERLAP: a caller still orders its work on the one stream);
 *   - a model is bound to the GPU that was current at nnc_model_create and to one
 *     stream; calls on one model must not overlap (not thread-safe);
 *   - positions are implicit: each KV slot remembers its length, nnc_prefill and
 *     nnc_decode_step append at that length.
 *
 * Canonical weight blob (host memory, little endian, tensors contiguous,
 * matrices row-major [out, in] in blob_dtype, gains always fp32), in order:
 *   embed [V,H]                                   if has_embed_and_head
 *   per layer: g_in [H], Wq [Dq,H], Wk [Dkv,H], Wv [Dkv,H], g_q [d], g_k [d],
 *              Wo [H,Dq], g_post [H], Wgate [F,H], Wup [F,H], Wdown [H,F]
 *   g_final [H]                                   if has_embed_and_head
 *   lm_head [V,H]                                 if has_embed_and_head && !tied_lm_head
 * with Dq = n_q_heads*head_dim, Dkv = n_kv_heads*head_dim.
 * blob_dtype NNC_W8 (weight-only 8 bits; the paper has no low-bit format: this extends its
 * 16-bit runs of Section 4 towards the memory wall it names in Sections 4.1 and 4.2): every
 * matrix of a layer is [out, in] signed bytes q followed by [out] fp32 scales s, the weight being
 * s[row] * q[row][col]; embed and lm_head are bf16; hidden and ffn are multiples of 64.
 */
#ifndef NNC_H_
#define NNC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct nnc_model nnc_model; /* opaque; owned by the library */

typedef enum {
  NNC_OK = 0,
  NNC_E_ARG = 1,     /* null pointer, slot/batch/token out of range, duplicate slots */
  NNC_E_CONFIG = 2,  /* unsupported or inconsistent nnc_config */
  NNC_E_BLOB = 3,    /* blob_bytes does not match the config */
  NNC_E_NOMEM = 4,   /* device allocation failed */
  NNC_E_KV_FULL = 5, /* a slot would exceed max_seq */
  NNC_E_DEVICE = 6,  /* HIP error, or no gfx950 device */
  NNC_E_STATE = 7    /* call not valid for this model (e.g. token API on a hidden-state model) */
} nnc_status;

typedef enum {
  NNC_F32 = 0,
  NNC_BF16 = 1,
  NNC_F16 = 2, /* IEEE binary16, the paper's F16 (Section 4, setup) */
  NNC_W8 = 3,  /* blob_dtype only: bytes with one scale per output row in the layers, bf16 elsewhere */
  NNC_I8 = 4,  /* paged KV cache only: signed bytes -127 .. 127 with one fp32 scale per row and kv head */
  NNC_E4M3 = 5 /* paged KV cache only: OCP 8-bit floats (4 exponent bits, largest 448), scales likewise */
} nnc_dtype;

typedef struct {
  uint32_t struct_bytes; /* = sizeof(nnc_config) */
  uint32_t hidden, n_layers, n_q_heads, n_kv_heads, head_dim, ffn, vocab;
  float rms_eps, rope_theta;
  uint32_t has_embed_and_head; /* 0: hidden state in, hidden state out (one-layer fp32 config) */
  uint32_t tied_lm_head;       /* 1: LM head is the embedding matrix, blob holds no lm_head */
  uint32_t blob_dtype;         /* nnc_dtype of the matrices in the blob */
  uint32_t compute_dtype;      /* NNC_F32: fp32 weights, fp32 KV cache, fp32 matrix-core math;
                                  NNC_BF16 / NNC_F16: 16-bit weights and KV cache in that format,
                                  fp32 accumulation (activations enter the matrix cores as 16-bit
                                  pieces of that format).  Must equal blob_dtype, or be a 16-bit type
                                  with an NNC_F32 blob (weights are then rounded to nearest even
                                  once, at create).  An NNC_W8 blob computes in NNC_BF16: the decode
                                  GEMMs stream the bytes, widen them to bf16 exactly in registers and
                                  multiply the row sums by the scales; bf16 KV cache, embedding and
                                  LM head.  Prompt blocks widen each matrix (exactly) into a scratch matrix of
                                  bf16 tiles first and scale the rows in the GEMM's epilogue, short ones (up to
                                  256 tokens, see NNC_OPT_PLANNER) stream the bytes as decode does;
                                  batch-1 decode runs through the per-stage kernels (the resident decode
                                  kernel takes 16-bit weights only). */
  uint32_t max_batch;          /* number of KV slots */
  uint32_t max_seq;            /* positions per slot */
} nnc_config;

/* Device memory and stream come from the caller (e.g. PyTorch's allocator and
 * current stream).  alloc returns device memory aligned to >= 256 bytes or NULL;
 * both callbacks are invoked only inside nnc_model_create / nnc_model_destroy.
 * A NULL nnc_device, or NULL alloc/free, selects hipMalloc/hipFree and the
 * default stream. */
typedef struct {
  void *(*alloc)(size_t bytes, void *ctx);
  void (*free)(void *p, void *ctx);
  void *ctx;
  void *stream; /* hipStream_t; NULL = default stream */
} nnc_device;

/*
 * Build a model: validate the config, check blob_bytes, allocate weights / KV
 * cache / workspace, upload and repack every matrix once into the matrix-core
 * tile layout (the on-GPU counterpart of the paper's packed constant layouts,
 * Sections 3.1.2 and 3.3.1): Wq|Wk|Wv fused row-wise, Wgate/Wup interleaved in
 * 16-row tiles, bf16 rounding if requested.  blob is host memory borrowed for
 * the duration of the call.  Synchronises the stream before returning.
 */
nnc_status nnc_model_create(const nnc_config *cfg, const void *blob, size_t blob_bytes,
                            const nnc_device *dev, nnc_model **out);

/* Release everything obtained through nnc_device.alloc.  NULL is allowed.
 * Synchronises the stream first.  (Lifetime management: the paper is silent; defined here.) */
void nnc_model_destroy(nnc_model *m);

/*
 * Prompt pass (the paper's pre-decode stage, Section 4 setup): run n tokens
 * (host int32, each in [0, vocab)) through the model for one KV slot, appending
 * K/V at positions len..len+n-1.  logits_out: device, vocab floats, logits of the
 * LAST position; may be NULL.  next_out: device int32, greedy arg-max of those
 * logits (lowest index wins ties); may be NULL.  Chunked prefill = repeated calls.
 * NNC_E_KV_FULL if len + n > max_seq.
 */
nnc_status nnc_prefill(nnc_model *m, uint32_t slot, const int32_t *tokens, uint32_t n,
                       float *logits_out, int32_t *next_out);

/*
 * One decode step (the stage the paper's tokens/s metric covers): one token for
 * each of `batch` distinct slots (host arrays slots[batch], tokens[batch]).
 * logits_out: device [batch, vocab] floats or NULL.  next_out: device [batch]
 * int32 greedy tokens or NULL.
 */
nnc_status nnc_decode_step(nnc_model *m, const uint32_t *slots, const int32_t *tokens,
                           uint32_t batch, float *logits_out, int32_t *next_out);

/*
 * Greedy decode loop with the token fed back on the device: n_steps decode steps
 * for `batch` distinct slots starting from first_tokens (host), no host
 * synchronisation between steps.  tokens_out: device [n_steps, batch] int32, the
 * token produced by each step.  logits_out: device [n_steps, batch, vocab] floats
 * or NULL.  NNC_E_KV_FULL if any slot would exceed max_seq during the run.
 * A run of two to four sequences that the resident kernel takes (NNC_OPT_PERSISTENT; its choice looks at the
 * contexts at the end of the run) computes what the same steps by nnc_decode_step compute, to fp32 rounding
 * but not bit for bit: those run one kernel per stage, and a value that is cached may round the other way
 * in its last bit.  With NNC_OPT_PERSISTENT 0 a run gives the same bits however it is cut into calls.
 */
nnc_status nnc_decode_greedy(nnc_model *m, const uint32_t *slots, const int32_t *first_tokens,
                             uint32_t batch, uint32_t n_steps, int32_t *tokens_out,
                             float *logits_out);

/*
 * nnc_decode_step for callers that cannot allocate: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and the same
 * results bit for bit as nnc_decode_step when that is called with a logits buffer (one kernel
 * per stage, launched eagerly on the model's stream), but the call allocates nothing: no
 * device or host memory, no graph, no event.  Its workspace is a fixed array of
 * NNC_STATIC_SCRATCH_MIB MiB inside the library's code object, one copy per GPU, held from
 * the first use until the process ends.
 * Limits: batch <= NNC_STATIC_MAX_BATCH, and the step's workspace (it grows with batch x
 * hidden / ffn sizes and with batch x query heads x cached positions; without logits_out also
 * batch x vocab floats) must fit the array: NNC_E_ARG with the byte counts otherwise, state
 * untouched.  NNC_E_STATE while nnc_profile_begin is active or if the model's GPU is not the
 * current device.
 * Every call on one GPU shares that GPU's array, whatever the model or stream: calls that
 * overlap on one GPU race.  Nothing in the array has to start at zero (every word a kernel
 * reads was written earlier in the same call), so no call clears it.
 */
#define NNC_STATIC_SCRATCH_MIB 24
#define NNC_STATIC_MAX_BATCH 8
nnc_status nnc_decode_step_static(nnc_model *m, const uint32_t *slots, const int32_t *tokens,
                                  uint32_t batch, float *logits_out, int32_t *next_out);

/* Forget the contents of one slot (slot >= 0) or of all slots (slot = -1): the slot's length
 * becomes 0, nothing is cleared on the device, no work is enqueued.  The paper is silent on
 * cache management (its runs are one prompt + one decode loop, Section 4 setup); defined here
 * so that one model serves request after request. */
nnc_status nnc_kv_reset(nnc_model *m, int32_t slot);

/*
 * Wait for all work enqueued on the model's stream and report deferred failures: the resident
 * decode kernel bounds every wait for an exchange word; if one ran out, all its workgroups
 * exited early, the outputs of that call are invalid and NNC_E_DEVICE is returned here and
 * by every later prompt / decode call on the model (they check without waiting).
 */
nnc_status nnc_synchronize(nnc_model *m);

/* Current length of a slot (host out-param).  (Paper silent; bookkeeping of this library.) */
nnc_status nnc_slot_len(const nnc_model *m, uint32_t slot, uint32_t *len_out);

/*
 * Hidden-state variants for models created with has_embed_and_head = 0: one decoder layer
 * (or several) without embedding and LM head, the unit the paper's operator-level
 * discussion is about (Section 3.1.2, the attention-like MatMul / Exp / MatMul chain) and the shape
 * of the smallest benchmark configuration.  The paper defines no such call; defined here.
 * x: device [n, hidden] floats in; y: device [n, hidden] floats out (the residual
 * stream after the last layer).  nnc_prefill_hidden treats the n rows as
 * consecutive positions of one slot; nnc_decode_step_hidden treats row i as the
 * next position of slots[i].
 */
nnc_status nnc_prefill_hidden(nnc_model *m, uint32_t slot, const float *x, uint32_t n, float *y);
nnc_status nnc_decode_step_hidden(nnc_model *m, const uint32_t *slots, const float *x,
                                  uint32_t batch, float *y);

/*
 * Copy cached rows out for inspection: positions pos0..pos0+n-1 of one layer and
 * slot, widened to fp32, as [n, Dkv] (kv head major inside a row) into device
 * memory `out`.  which: 0 = K (after QK-norm and RoPE), 1 = V.
 */
nnc_status nnc_kv_read(nnc_model *m, uint32_t layer, uint32_t slot, uint32_t which, uint32_t pos0,
                       uint32_t n, float *out);

/* Runtime switches. */
typedef enum {
  NNC_OPT_GRAPH = 0,        /* 1 (default): replay decode steps as captured HIP graphs; 0: eager */
  NNC_OPT_PREFILL_EXACT = 1, /* precision of the prompt pass of bf16 models.
                               0 (default): blocks of up to 4096 tokens with LDS-staged
                               matrix-core GEMMs and matrix-core attention.  Blocks of up to 512
                               tokens carry every matrix-core input as two bf16 pieces (16
                               significant bits); longer blocks round those inputs to bf16 once.
                               A call with more than 512 tokens runs its last 16 tokens through
                               the three-piece path of mode 1, so that the logits of the last
                               position see single-piece noise only through the cache; the LM
                               head itself is always fp32-grade.
                               2: the same blocks, two pieces at every length (twice the
                               matrix-core work of long blocks).
                               1: 21-token chunks through the decode kernels, three bf16 pieces
                               (fp32-grade) */
  NNC_OPT_PERSISTENT = 2,   /* 1 (default): batch-1 decode steps of 16-bit models, and nnc_decode_greedy
                               runs of two to four sequences of the smaller shapes (hidden sizes up to
                               1024, two sequences up to 2048) whose contexts are not too long, run in one
                               resident kernel per call (all steps of nnc_decode_greedy in a
                               single launch); 0: one kernel per stage.
                               That kernel takes every compute unit, and its workgroups wait for each
                               other (NNC_OPT_SPIN_LIMIT bounds the wait).  Launches of one process, of
                               whatever model and stream, take turns on a GPU; nothing orders them with
                               the kernels of other processes, or with kernels of the caller's own that stay
                               on the GPU for as long as that bound: where such share the GPU, set 0.
                               While the caller captures the model's stream, every call is one kernel per
                               stage, as each replay of a resident launch would need tags of its own */
  NNC_OPT_PREFILL_TILE = 4, /* block tile of the large-block prompt GEMMs: -1 (default) chosen from
                               each launch's size; 0: 64 x 128, 1: 256 x 128, 2: 128 x 128, 3: 64 x 64,
                               4: 192 x 128, 5: 256 x 256, 6: 192 x 256 (rows x operand columns).  Same k order per output
                               element in all of 0 .. 6, hence bit-identical results, except where the k range of
                               a narrow (residual) projection is split over several workgroups (partial
                               sums added in a fixed order): with a forced tile only the 64-row tiles do
                               that by themselves, for short blocks; see NNC_OPT_PREFILL_KSLICES.
                               With -1 and NNC_OPT_PLANNER 1, blocks of up to 512 tokens (the smaller the
                               hidden size, the longer) run through kernels of their own, which sum k in
                               another order: two pieces as well, equal to the tiles' to rounding */
  NNC_OPT_PREFILL_KSLICES = 13, /* with a forced NNC_OPT_PREFILL_TILE: k slices (1 .. 4) of the output and
                               down projections of a large prompt block, 0 (default): by the rule above.
                               Without a forced tile the tile model picks tile and slices together */
  NNC_OPT_PREFILL_ATTN = 6, /* attention of large prompt blocks.  0 .. 3: the kernel of 16 x 16 products, bit 0:
                               every workgroup takes a long and a short 64-token block, bit 1: two query
                               heads per wave; bit-identical for 0 .. 3 (a wave's arithmetic per head is the
                               same).  -1 (default): chosen from each launch's size: that kernel, or, while
                               NNC_OPT_PLANNER is 1, one of 32 x 32 products for blocks of one piece with at least
                               80 pairs of (128 tokens, query head), and for two-piece blocks that end at position
                               1600 or later and leave compute units idle, their positions split over up to 8
                               workgroups.  Its results differ from those of 0 .. 3: with one piece the
                               softmax weights are rounded to 16 bits against another running maximum, with two
                               the sums run in another order.
                               Short blocks with few workgroups that -1 does not split use a kernel of their
                               own, whatever this says, while NNC_OPT_PLANNER is 1 */
  NNC_OPT_FUSE_QK = 7,      /* 1 (default): per-stage decode passes (fp32 models, 16-bit models of at most
                               eight query heads per kv head) do QK-norm, RoPE and the cache append inside
                               the attention kernel (one kernel less per layer); 0: in a kernel of their
                               own.  Bit-identical results while the QKV projection has one k slice (with
                               NNC_OPT_PLANNER 0 always); the planner may give the attention kernel up to
                               four partial sums of it, whose order of addition is another (fp32 rounding) */
  NNC_OPT_TAIL_OVERLAP = 8, /* 1 (default): the fp32-grade pass over the last tokens of a long prompt is
                               enqueued on a second stream of the library's own and runs beside the
                               prompt's last block, each of its layers waiting (event) for that
                               layer's cache rows; the model's stream waits for it before the call
                               returns to the caller's later work.  0: it follows the block on the
                               model's stream.  Bit-identical results */
  NNC_OPT_PREFILL_BLOCK = 9, /* tokens per block of the large-block prompt pass: 0 (default) = the largest
                               (4096, or max_seq rounded up to 128 if that is less); else a multiple of
                               128.  Longer blocks give the narrow projections enough workgroups for the
                               largest block tile; the blocking does not change which inputs are rounded
                               (every block of more than 512 tokens carries one bf16 piece) */
  NNC_OPT_PLANNER = 10,     /* 1 (default): block tiles, row tiles per workgroup and k slices of the GEMM
                               launches come from the analytic model behind nnc_plan_*_query, and short
                               prompt blocks have kernels of their own (see NNC_OPT_PREFILL_TILE and
                               NNC_OPT_PREFILL_ATTN); 0: from the hand-written rules that preceded it, the
                               block tiles at every length (kept for comparison) */
  NNC_OPT_FUSE_NORM = 11,   /* 1: in per-stage decode passes the RMSNorm after an output / down
                               projection runs in the tail of that GEMM launch (its last workgroups to
                               finish wait for the others, one per sequence, and norm the rows): two
                               kernels less per layer, same arithmetic, bit-identical results; the wait
                               is bounded by NNC_OPT_SPIN_LIMIT.  0 (default): in a kernel of its own --
                               the hand-over inside the launch (store acknowledgement, counter, reads
                               past the caches) takes as long as the kernel boundary it replaces */
  NNC_OPT_DECODE_PIECES = 12, /* bf16 / binary16 pieces an activation is split into before a decode GEMM of
                               a batch of two or more sequences: 0 (default) the library's choice, 2 or 3
                               forced.  Three pieces carry an fp32 value to 2^-25 relative, two to 2^-17
                               (a third fewer operand columns) */
  NNC_OPT_SPIN_LIMIT = 5,   /* polls after which a wait inside the resident kernel gives up (sets
                               the failure flag and lets every workgroup exit); 0 (default):
                               2^20, about a second.  A tiny value makes the give-up path testable */
  NNC_OPT_TAG_LIMIT = 14,   /* the resident kernel marks every exchanged word with a 32-bit tag, 5 x layers + 1
                               tags per decode step; when they reach this limit, the exchange buffers are
                               cleared (on the model's stream) and the tags start again: no run of calls ends
                               there.  0 (default): 2^32 - 1.  A small value makes the restart testable; one
                               run that needs more tags by itself is NNC_E_STATE at batch 1 and runs one
                               kernel per stage at larger batches */
  NNC_OPT_STAGE_TRACE = 3   /* s + 1: the resident kernel stamps the 100 MHz wall clock at every
                               stage boundary of decode step s of each following launch (read them
                               with nnc_stage_trace); 0 (default): off */
} nnc_option;
nnc_status nnc_set_option(nnc_model *m, nnc_option opt, int32_t value);

/*
 * Per-kernel timing with HIP events on the model's stream.  After
 * nnc_profile_begin, every launch of the forward pass runs eagerly and is
 * bracketed by events; nnc_profile_end synchronises, stops profiling and fills up
 * to `cap` records (host), returning the number written in *n_out.  (A step on pages waits for the
 * stream once while it is profiled: the lengths that its bytes follow from lie in device memory.)
 */
typedef struct {
  char name[48];        /* kernel family, e.g. "attn_partial"; the skinny GEMM reports one record per
                           matrix it streams: "gemm_skinny.qkv", ".o", ".gate_up", ".down", ".lm_head" */
  uint64_t launches;
  double total_ms;      /* sum of event-to-event times */
  double bytes;         /* algorithmic bytes those launches had to move */
  double flops;         /* algorithmic flops (2 per multiply-add) */
} nnc_kernel_stat;
nnc_status nnc_profile_begin(nnc_model *m);
nnc_status nnc_profile_end(nnc_model *m, nnc_kernel_stat *out, uint32_t cap, uint32_t *n_out);

/*
 * Stage stamps of the last traced resident-kernel launch (see NNC_OPT_STAGE_TRACE), for
 * tuning: host buffer out[workgroups][points] of 64-bit wall-clock ticks (10 ns each).
 * Per layer 8 points: layer start, QKV operand ready, q|k|v published, attention partials
 * published, attention block output published, gate/up operand ready, activations
 * published, MLP output published; then LM-head operand ready, per-workgroup winners
 * published, token known.  Synchronises the stream.  NNC_E_ARG if cap (in
 * 64-bit words) is too small; NNC_E_STATE if tracing is off.
 */
nnc_status nnc_stage_trace(nnc_model *m, uint64_t *out, uint32_t cap, uint32_t *workgroups,
                           uint32_t *points);

/*
 * The analytic tile chooser the library plans its GEMM launches with, exposed for inspection and
 * tests (host code only, no GPU needed).  It follows the paper's parametric optimisation
 * (Section 3.2.2): tile variables, capacity constraints per storage level (LDS bytes of the
 * staged operands, registers per wave), and the objective minimise max(T_mem, T_comp) with T_comp
 * from a linear regression of the micro-kernel's time per k step and T_mem = traffic / bandwidth,
 * plus launch and epilogue-traffic time.  The search space is the block tiles the kernels are
 * instantiated for, times the k slices a launch may use, so the problem is solved by enumeration.
 * epilogue: 0 store, 1 add to the residual stream, 2 SwiGLU.  n_cus: compute units (0 = 256).
 *   nnc_plan_prefill_gemm_query  prompt GEMM [rows x k] x [k x n_tokens] with `pieces` 16-bit
 *                                pieces per activation; may use up to max_k_slices k slices
 *   nnc_plan_skinny_gemm_query   weight-streaming GEMM of a decode pass with n_seq sequences of
 *                                `pieces` pieces each; T_mem has two levels here: t_mem_us = the
 *                                weights from HBM, t_comp_us = what the busiest compute unit moves
 *                                through its vector memory path (its workgroups' weight tiles and
 *                                operand reads); tile_rows = rows per workgroup (16 x 1, 2, 3, 4, 6
 *                                or 8 row tiles; with epilogue 0 and max_k_slices 1 they need not divide
 *                                `rows`: the last workgroup then has fewer); max_k_slices = partial sums
 *                                the consumer can add
 */
typedef struct {
  uint32_t tile_rows, tile_cols;  /* block tile (rows x operand columns) */
  int32_t tile_code;              /* the library's code of that tile (NNC_OPT_PREFILL_TILE) / row tiles per workgroup */
  uint32_t k_slices, workgroups;
  double t_comp_us, t_mem_us, t_us; /* model times of the choice */
  uint32_t candidates, rejected_by_capacity; /* prompt GEMM: tiles enumerated / ruled out by LDS or registers */
} nnc_gemm_plan;
nnc_status nnc_plan_prefill_gemm_query(uint32_t rows, uint32_t k, uint32_t n_tokens, uint32_t pieces,
                                       uint32_t epilogue, uint32_t max_k_slices, uint32_t n_cus,
                                       nnc_gemm_plan *out);
nnc_status nnc_plan_skinny_gemm_query(uint32_t rows, uint32_t k, uint32_t n_seq, uint32_t pieces,
                                      uint32_t epilogue, uint32_t max_k_slices, uint32_t n_cus,
                                      nnc_gemm_plan *out);

/* =============================================================================================
 * Paged KV cache, and the search that shares its pages.  (The paper's runs are one sequence in one
 * cache; nothing of this section is in it, all of it is defined here.)
 *
 * Operators of their own, without a model: nnc_page_append, nnc_page_read, nnc_page_attention,
 * nnc_page_attention_shared, nnc_page_bound, nnc_page_pick, nnc_page_attention_picked, nnc_page_reorder, nnc_beam_select,
 * nnc_draft_verify.  They enqueue on `stream` (hipStream_t, NULL = default stream) of
 * the current device, which must be the one that holds every buffer named in the call; they allocate
 * nothing, keep nothing and may be captured into a graph.  Buffers belong to the caller and must live
 * until the work has run; a workspace may serve any number of calls that follow each other in one
 * stream, not calls (or replays of graphs that captured it) that may run side by side.
 * What the host can see is checked (NNC_E_ARG); page numbers, positions and lengths lie in device
 * memory and are checked on the device: what each call does about a wrong one is said there.
 *
 * nnc_pages: one pool for all layers, memory of the caller:
 *   k, v              [n_layers][n_pages][n_kv_heads][page_tokens][head_dim] of dtype, on a multiple of 16 bytes
 *   k_scale, v_scale  [n_layers][n_pages][n_kv_heads][page_tokens] fp32 for NNC_I8 and NNC_E4M3, else NULL
 * dtype: NNC_F32, NNC_BF16, NNC_F16, NNC_I8 or NNC_E4M3.  head_dim: 64 or 128.  page_tokens: 1 .. 4096,
 * n_kv_heads and n_layers: up to 1024.  Pages need no initial contents.
 * nnc_page_table: entries [n_seqs][max_pages], device: position p of sequence i is row p % page_tokens of
 * page entries[i][p / page_tokens].  Sequences may name the same page (a shared prompt) as long as nobody writes to it.
 */
typedef struct {
  uint32_t struct_bytes; /* = sizeof(nnc_pages) */
  uint32_t dtype, n_layers, n_pages, page_tokens, n_kv_heads, head_dim;
  void *k, *v;
  float *k_scale, *v_scale;
} nnc_pages;

typedef struct {
  const int32_t *entries;
  uint32_t n_seqs, max_pages;
} nnc_page_table;

/* Rows of K and V: row i, kv head h, element e at k[i * k_row_stride + h * k_head_stride + e] (elements of dtype:
 * NNC_F32, NNC_BF16 or NNC_F16; any strides), likewise v.  Row i is position pos[i] of sequence seq[i] (device
 * arrays of n; NULL: every row is of sequence seq0; row i is position pos0 + i). */
typedef struct {
  void *k, *v;
  uint32_t dtype;
  int64_t k_row_stride, k_head_stride, v_row_stride, v_head_stride;
  uint32_t n;
  const int32_t *seq, *pos;
  int32_t seq0, pos0;
} nnc_page_rows;

/*
 * Write rows into the pages of one layer.  16- and 32-bit pools round to nearest even.  8-bit pools take, for each row
 * and kv head, scale = max(max |x| / T, 2^-80) in fp32 (T = 127 for NNC_I8, 448 for NNC_E4M3) and store x / scale, rounded
 * to the nearest value of the format (ties to even): off by at most scale / 2, or by 2^-4 of the value (2^-10 scale at the
 * least).  A row of which one value is not finite becomes NaN as a whole (its scale does).
 * A row with a negative position is padding and is not written; nor is one whose sequence, position or page
 * does not exist.  Rows of one call must be different positions.  The rows are only read.
 */
nnc_status nnc_page_append(const nnc_pages *pages, uint32_t layer, const nnc_page_table *table,
                           const nnc_page_rows *rows, void *stream);

/*
 * The way back: read the named positions of one layer into rows (k or v may be NULL).  Values are value * scale in
 * fp32, rounded once to the rows' type.  A row whose sequence, position or page does not exist becomes NaN.
 */
nnc_status nnc_page_read(const nnc_pages *pages, uint32_t layer, const nnc_page_table *table,
                         const nnc_page_rows *rows, void *stream);

/* One query row per sequence of the table: q head a of row i at q[i * q_row_stride + a * q_head_stride], reading kv
 * head a / (n_q_heads / n_kv_heads); out in the same type, with strides of its own (it may be q itself). */
typedef struct {
  const void *q;
  void *out;
  uint32_t dtype, n_q_heads;
  int64_t q_row_stride, q_head_stride, out_row_stride, out_head_stride;
  const int32_t *lens; /* device [n_seqs]: cached positions of each sequence */
  uint32_t max_len;    /* none of them is larger (it sizes the launch); 0: what the table holds */
  uint32_t window;     /* only the last `window` positions are attended to; 0: all */
  float scale;         /* of the scores, e.g. 1 / sqrt(head_dim) */
} nnc_page_query;

/*
 * Attention of one new token per sequence over one layer: softmax(scale * q K^T) V over positions 0 .. lens[i] - 1
 * (the last `window` of them).  Sums, softmax statistics, scores and weights are fp32-grade whatever the types (weights 22 bits for
 * binary16 queries over a binary16 pool); out is rounded once.  A sequence of length 0 gives zeros; a negative length, one above max_len and a missing page
 * give NaN.  What pages hold beyond a sequence's length is not looked at.  A NaN or an infinity in reach shows in the results
 * of the heads that read it, as NaN or an infinity, but for scores of -infinity: out of an fp32 pool they weigh nothing (where
 * nothing else is left the result is zero), out of others they do that or give NaN.
 * Long sequences are split over several workgroups and their results joined in a fixed order: the same call gives the same
 * bits.  How they are split depends on max_len, n_seqs and the heads, so results for another max_len
 * differ in rounding.  workspace: nnc_page_attention_workspace bytes (which may be 0), on a multiple of 16.
 */
nnc_status nnc_page_attention_workspace(const nnc_pages *pages, const nnc_page_table *table,
                                        const nnc_page_query *query, size_t *bytes);
nnc_status nnc_page_attention(const nnc_pages *pages, uint32_t layer, const nnc_page_table *table,
                              const nnc_page_query *query, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention of rows that share the first positions of their contexts (a batch behind one prompt, the beams of a search, the new
 * tokens of one sequence).  Query row g * width + w is row w of group g; query->lens: device [rows].
 *   prefix not NULL: device [groups]; the table has a row for every query row.  Positions below prefix[g] are read for the
 *     whole group (once for up to 128 rows x query heads of a kv head, 64 where the queries are not of the type that the pool's products are
 *     in, 16 of an fp32 pool) through the table row of its first query row, the others through the row's own.  max_own: no row has
 *     more positions behind its prefix (0: none has any).
 *   prefix NULL: the table has a row for every group, whose query rows are new tokens of one sequence: row r sees its first lens[r]
 *     positions, all of them read in the same way (max_own is not looked at).
 * The result of a row is that of nnc_page_attention for its length, but for the order of sums and, with NNC_BF16 queries over an NNC_BF16 pool or one of 8
 * bits, where a group has more than sixteen rows (width x query heads of a kv head) or none has positions of its own, the products' weights, which have 17 bits
 * (2^-18 of sum w |v| is left out; the output's own rounding is 2^-9 of it).  Weights of up to 2^20 stand in those sums: values of V beyond 2^107 / positions may
 * make them infinite.  A length may end
 * inside the prefix; it gives zeros where it is 0, and NaN where it is negative, above max_len or more than max_own behind the prefix, as
 * does a negative prefix.  A row is NaN as a whole where one of its positions has no page or a value of V that is not finite
 * and that other rows do not see.  What positions behind a row's own length hold does not reach it.  query->window must be 0.
 * width: up to 65535; rows: up to 65535.  workspace: nnc_page_attention_shared_workspace bytes (which may be 0), on a multiple of 16.
 */
typedef struct {
  uint32_t width;
  const int32_t *prefix;
  uint32_t max_own;
} nnc_page_share;
nnc_status nnc_page_attention_shared_workspace(const nnc_pages *pages, const nnc_page_table *table,
                                               const nnc_page_query *query, const nnc_page_share *share, size_t *bytes);
nnc_status nnc_page_attention_shared(const nnc_pages *pages, uint32_t layer, const nnc_page_table *table,
                                     const nnc_page_query *query, const nnc_page_share *share, void *workspace,
                                     size_t workspace_bytes, void *stream);

/*
 * Attention to a part of a long context: the pages whose keys promise the largest scores.
 * nnc_page_bounds: for every page and kv head the smallest and the largest key, dimension by dimension, memory of the caller:
 *   lo, hi  [n_layers][n_pages][n_kv_heads][head_dim], on a multiple of 16 bytes; in the pool's dtype, NNC_BF16 for pools of 8 bits
 *           (whose values, with their scales, are rounded outwards: downwards in lo, upwards in hi).  lo <= hi, or a NaN in one of them
 */
typedef struct {
  void *lo, *hi;
} nnc_page_bounds;

/*
 * Bring the bounds of a layer up to date: of every sequence i those of the pages that hold positions since[i] .. lens[i] - 1 (device
 * arrays of n_seqs; since NULL: since0 for all), each from all of the page's positions below lens[i].  max_new: no sequence has more such
 * positions (0: what the table holds); pages behind that many are left as they are.  A NaN among a page's keys makes the bounds of its dimension NaN.
 * Nothing is done for a negative length or since, for a since that is not below the length, nor for a page that does not exist.  A page that several of the sequences name gets
 * the bounds that one of them gives it: they are to see the same positions of it.
 */
nnc_status nnc_page_bound(const nnc_pages *pages, uint32_t layer, const nnc_page_bounds *bounds, const nnc_page_table *table,
                          const int32_t *lens, const int32_t *since, int32_t since0, uint32_t max_new, void *stream);

/* One query row per sequence, as in nnc_page_query, and how many pages it picks. */
typedef struct {
  const void *q;
  uint32_t dtype, n_q_heads;
  int64_t q_row_stride, q_head_stride;
  const int32_t *lens;          /* device [n_seqs] */
  uint32_t max_len;             /* none of them is larger; 0: what the table holds */
  uint32_t keep;                /* pages picked for each kv head, 1 .. 65536 */
  uint32_t first, last;         /* of them, the first ones and the last ones of the sequence, whatever they score; last >= 1 */
  int32_t *tables_out;          /* device [n_seqs][n_kv_heads][keep] */
  int32_t *lens_out;            /* device [n_seqs][n_kv_heads] */
} nnc_pick;

/*
 * For every sequence and kv head, the `keep` pages with the largest scores, in the order of the sequence:
 *   score of a page = the largest, over the query heads h of the kv head, of  sum_d max(q[h][d] lo[d], q[h][d] hi[d])
 * which no key of the page exceeds.  (For a negative scale of the attention, pass -q.)  tables_out names them, -1 behind the last of them; lens_out
 * is the number of their positions: all pages are full but the last one, which is the sequence's last.  Scores are
 * formed and compared in 64 bits; ties go to the page that comes first.  A page that does not exist, and one whose score is NaN, comes before all others,
 * so that it shows in the attention.  A length of 0 picks nothing; a negative length or one above max_len gives the
 * length -1.  workspace: nnc_page_pick_workspace bytes, on a multiple of 16.
 */
nnc_status nnc_page_pick_workspace(const nnc_pages *pages, const nnc_page_table *table, const nnc_pick *pick, size_t *bytes);
nnc_status nnc_page_pick(const nnc_pages *pages, uint32_t layer, const nnc_page_bounds *bounds, const nnc_page_table *table,
                         const nnc_pick *pick, void *workspace, size_t workspace_bytes, void *stream);

/*
 * nnc_page_attention where every kv head has a table and a length of its own: row i * n_kv_heads + h of the table (n_seqs: sequences
 * x kv heads), lens: device [n_seqs][n_kv_heads].  query->window must be 0.
 */
nnc_status nnc_page_attention_picked_workspace(const nnc_pages *pages, const nnc_page_table *table,
                                               const nnc_page_query *query, size_t *bytes);
nnc_status nnc_page_attention_picked(const nnc_pages *pages, uint32_t layer, const nnc_page_table *table,
                                     const nnc_page_query *query, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Beams take over the cache of the beams that they continue.  Sequences g * width .. + width - 1 of the table are
 * the beams of group g, all of one length lens[g * width] (device [n_seqs]); parents: device [n_seqs], each
 * 0 .. width - 1 (another value: the beam continues itself).  With f full pages and r more rows:
 *   after[b][i] = before[parent of b][i]  for i < f;
 *   if r > 0, rows 0 .. r - 1 of page before[parent][f] are copied to page after[b][f], in every layer;
 *   the other entries of after stay: from f on they name pages of the beam's own, which no other beam of `after` has.
 * after: device [n_seqs][max_pages], may be before->entries itself (then a beam's page may be another's
 * source, in any permutation).  Full pages are shared, nothing of them is copied.  A length that is negative or does not fit
 * the table changes nothing; a missing page is not copied.  width: up to 32; layers x kv heads x bytes of a head's page: up to 2^34.
 */
nnc_status nnc_page_reorder(const nnc_pages *pages, const nnc_page_table *before, int32_t *after,
                            const int32_t *lens, const int32_t *parents, uint32_t width, void *stream);

/* One step of a beam search over n_groups groups of `width` beams (row r = group * width + beam). */
typedef struct {
  const void *logits;      /* device, row r at logits + r * row_stride, vocab elements of dtype */
  uint32_t dtype;          /* NNC_F32, NNC_BF16 or NNC_F16 */
  int64_t row_stride;
  uint32_t n_groups, width, vocab;
  const float *scores;     /* device [rows]: log-probability so far; -infinity: the beam is not in use */
  const uint8_t *finished; /* device [rows]: not 0 where the beam has ended; NULL: none has */
  int32_t eos;             /* token that ends a beam, -1: none (then finished must be NULL) */
  int32_t *tokens_out, *parents_out; /* device [rows] */
  float *scores_out;       /* device [rows], may be scores */
  uint8_t *finished_out;   /* device [rows] or NULL, may be finished */
} nnc_beam;

/*
 * The `width` best continuations of every group, best first.  Beam w continued by token v has the score
 * scores[w] + logit[v] - log sum_u exp(logit[u]); an ended beam has one continuation, eos with its score unchanged; the
 * logits of ended and unused beams are not looked at (every continuation of an unused one is -infinity).
 * Ties go to the lower beam, then to the lower token; within a beam the larger logit always goes first.  The log-sums have the
 * error of fp32 exponentials and sums (below 2^-18; 40 to 600000 logits: 3.2e-7 at most), the same for equal rows; on top of them
 * scores are formed and compared in 64 bits, so that continuations of two beams closer than that error may stand in either order.  A logit of -infinity forbids its token (score -infinity: chosen only when
 * nothing else is left).  A beam with a NaN or a +infinity among its logits has NaN scores, but for the tokens that are
 * forbidden, whose score stays -infinity; NaN ranks first, so that such a failure shows, and its tokens rank by logit.  width: up to 32.
 * workspace: nnc_beam_select_workspace bytes, on a multiple of 16.
 */
nnc_status nnc_beam_select_workspace(const nnc_beam *beam, size_t *bytes);
nnc_status nnc_beam_select(const nnc_beam *beam, void *workspace, size_t workspace_bytes, void *stream);

/* Drafted tokens of n sequences, up to k of each, and what the target and the draft think of them. */
typedef struct {
  const void *logits;         /* device, of the target: row i * (k + 1) + j at logits + that * row_stride, vocab elements of dtype:
                                 the distribution of the token behind the first j drafts of sequence i */
  const void *draft_logits;   /* ... of the draft: row i * k + j, that draft j was drawn from; NULL: drafts that were not drawn */
  uint32_t dtype;             /* NNC_F32, NNC_BF16 or NNC_F16 */
  int64_t row_stride, draft_row_stride;
  uint32_t n, k, vocab;
  const int32_t *drafts;      /* device [n][k] */
  const int32_t *counts;      /* device [n]: drafts of each sequence, 0 .. k; NULL: k */
  const float *uniforms;      /* device [n][k + 1], random numbers of [0, 1): one for each draft, the last one for the token behind them */
  const float *temperatures;  /* device [n]; NULL: `temperature` for all.  0: the largest logit (the first of equals) has all the probability */
  float temperature;
  int32_t *tokens_out;        /* device [n][k + 1] */
  int32_t *accepted_out;      /* device [n] */
} nnc_drafts;

/*
 * Which drafts are kept, and the token behind them, so that the tokens are distributed as the target's would be:
 *   p_j = softmax(logits_j / T), q_j = softmax(draft_logits_j / T), without draft_logits q_j = 1 for the draft itself
 *   draft x_j is kept, as long as all before it are, if u_j q_j(x_j) < p_j(x_j)
 *   then one token more: the first v for which  sum_{w <= v} r(w) > u_k sum_w r(w),  where r = max(p_j - q_j, 0) behind a draft that
 *   was not kept (p_j itself if that is zero everywhere), and r = p_j of the row behind the last draft
 * tokens_out: the kept drafts, that token, and -1 behind it; accepted_out: how many were kept.  Sums, exponentials and comparisons are in
 * 64 bits (exponentials to 2^-42), and sums are taken in a fixed order: the same call gives the same tokens.  Rows behind a sequence's count are not looked at.
 * A logit that lies 693 T (a factor of 2^-1000) or more below the largest of its row has the probability 0 in u_j q_j(x_j) < p_j(x_j) and in max(p_j - q_j, 0); in r = p_j it
 * has next to none, which a u_k of exactly 0 does ask for: only -infinity forbids a token whatever the random numbers are.
 * A sequence whose count is none of 0 .. k or whose temperature is negative or not finite gives the token -1 and
 * keeps nothing; where a row that has to be looked at has no distribution (a NaN, a +infinity, only -infinities), a draft is
 * no token or a random number is NaN, the token there is -1, behind the drafts kept before.
 * n (2 k + 1): up to 65535; workspace: nnc_draft_verify_workspace bytes, on a multiple of 16.
 */
nnc_status nnc_draft_verify_workspace(const nnc_drafts *drafts, size_t *bytes);
nnc_status nnc_draft_verify(const nnc_drafts *drafts, void *workspace, size_t workspace_bytes, void *stream);

/*
 * A model on pages.  The calls below run on the model's stream like every other call on it; pages must have the
 * model's layers, kv heads and head_dim, any dtype.  They do not touch the lengths of the model's slots.
 *
 * Copy positions pos0 .. pos0 + n - 1 of a slot's cache, all layers, to the same positions of sequence `seq` of the
 * table: a prompt goes through nnc_prefill into a slot and from there into pages, and the slot is free again.
 */
nnc_status nnc_pages_store(nnc_model *m, const nnc_pages *pages, const nnc_page_table *table, uint32_t seq,
                           uint32_t slot, uint32_t pos0, uint32_t n);

/*
 * One decode step of the table's sequences (up to 21): token tokens[i] (device) becomes position lens[i] (device) of
 * sequence i, in pages that must be there already, and lens[i] grows by one.  max_len: no lens[i] is larger before
 * the call (0: only the table and max_seq bound them); NNC_E_KV_FULL if max_len + 1 positions fit neither the table
 * nor the rotary table (max_seq).  logits_out: device [n_seqs, vocab] floats or NULL, next_out: device [n_seqs] greedy
 * tokens or NULL.  A sequence whose token is outside the vocabulary, or whose length is outside 0 .. max_len, gets
 * NaN logits, caches nothing and keeps its length.
 * The arithmetic is that of nnc_decode_step, but for what the cache's type loses and the order of sums.
 */
nnc_status nnc_decode_step_paged(nnc_model *m, const nnc_pages *pages, const nnc_page_table *table, int32_t *lens,
                                 uint32_t max_len, const int32_t *tokens, float *logits_out, int32_t *next_out);

/*
 * One pass over a token of each of the table's sequences and up to k drafts behind it: tokens: device [n_seqs][k + 1], token j of
 * sequence i becomes position lens[i] + j, for j up to counts[i] (device, 0 .. k; NULL: k), in pages that must be there already; lens are
 * not changed.  logits_out: device [n_seqs * (k + 1), vocab], what nnc_draft_verify takes; next_out: device [n_seqs * (k + 1)] or NULL.  A
 * sequence of which a drafts are kept goes on with lens[i] + a + 1: what was cached behind that is overwritten and never looked at.
 * Tokens behind the count, outside the vocabulary or at positions outside 0 .. max_len + k are not cached and
 * have NaN logits; so has every token behind one that is not cached.  A pass reads a sequence's cache once for all of its tokens.  n_seqs * (k + 1): up to 21;
 * max_len: as for nnc_decode_step_paged (no lens[i] is larger); sequences must not name the same page behind lens[i].
 */
nnc_status nnc_decode_step_drafts(nnc_model *m, const nnc_pages *pages, const nnc_page_table *table, const int32_t *lens,
                                  uint32_t max_len, uint32_t k, const int32_t *tokens, const int32_t *counts,
                                  float *logits_out, int32_t *next_out);

/*
 * Beam search on the device: n_steps times a decode step of every beam, nnc_beam_select and nnc_page_reorder, without
 * host synchronisation.  tables: device [n_groups * width][max_pages], updated; the entries behind the full pages are
 * the beam's own.  With first_logits (device [n_groups][vocab], e.g. of nnc_prefill) the search begins: all beams of a
 * group stand at the same prompt, whose full pages every one of them names and whose last, not full page lies in beam
 * 0's own; scores and finished are set by the call, and its first step only selects and reorders.  Without, it
 * goes on from `tokens`, scores and finished as the call before left them (tokens: the last row of its tokens_out).
 * lens: device [n_groups * width], updated (a first step adds nothing); max_len as for nnc_decode_step_paged, before the call.
 * tokens_out, parents_out: device [n_steps][n_groups * width]; scores, finished: device [n_groups * width].
 * Beams that have ended keep their score and repeat eos; in a run that goes on without one (eos -1) those that
 * `finished` names stay ended too, and repeat their last token.  n_groups * width: up to 21.
 */
typedef struct {
  int32_t *tables;
  uint32_t max_pages, n_groups, width;
  int32_t *lens;
  uint32_t max_len;
  const float *first_logits; /* or NULL */
  const int32_t *tokens;     /* device [n_groups * width]; not read with first_logits */
  int32_t eos;               /* -1: none */
  uint32_t n_steps;
  int32_t *tokens_out, *parents_out;
  float *scores;
  uint8_t *finished;
} nnc_beam_run;
nnc_status nnc_decode_beam(nnc_model *m, const nnc_pages *pages, const nnc_beam_run *run);

/* Bytes of the canonical blob for a config (0 if the config is invalid).  (Paper silent: the blob
 * is this library's input format, the stand-in for the paper's pre-laid-out constants,
 * Section 3.3.1.) */
uint64_t nnc_blob_bytes(const nnc_config *cfg);

/* Message for the most recent failure on this thread (static storage).  (Paper silent.) */
const char *nnc_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* NNC_H_ */
