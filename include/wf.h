/*
 * wf.h -- C ABI of the GB300 (sm_103a) Whisper-Flash speculative decode step.
 *
 * One speculative decode step of a Whisper-shaped encoder-decoder (Whisper-Flash,
 * arXiv 2609.32869): a 2-layer parallel drafter proposes K=8 tokens in one
 * forward pass from the encoded audio and the target's accepted decoder states
 * (Sec. 3.2, Eq. 2, App. A.2); the frozen target decoder verifies the anchor
 * and the K proposals in one causal pass, keeps the longest agreeing prefix
 * plus its own correction or bonus token (greedy), or applies speculative
 * rejection sampling at temperature T (Sec. 3.1, App. A.4), and rolls back its
 * key/value cache to L+1+a positions (App. A.1).
 *
 * Conventions that hold for every entry point:
 *  - All pointers named d_* / device are DEVICE pointers; the library never
 *    copies them to the host unless an entry point says so.  Host pointers are
 *    named h_*.
 *  - Weights, the workspace and every output buffer are owned by the caller and
 *    borrowed by the handle; they must stay valid until wf_destroy.  Nothing is
 *    allocated by the library on the device: the caller passes one workspace
 *    of at least wf_workspace_bytes() bytes, 256-byte aligned.
 *  - Parameters are bfloat16, row-major; matrices are [out_features, in_features]
 *    (y = x W^T + b); every weight pointer is 16-byte aligned.  Token ids are
 *    int32.
 *  - Calls are asynchronous and ordered on the given stream unless stated.  The
 *    return value reports host-side validation and launch errors; conditions
 *    found on the device (capacity overflow, a bounded wait that gave up) are
 *    recorded in a device error word read by wf_get_state / wf_get_error.
 *  - A handle is not thread-safe.  No C++ exception crosses this boundary.
 *    There is no CPU fallback: without a usable sm_103a device every compute
 *    entry point returns WF_ERR_CUDA.
 */
#ifndef WF_H
#define WF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum wf_status {
  WF_OK = 0,
  WF_ERR_INVALID = 1,     /* a null pointer, a bad size, a misaligned buffer */
  WF_ERR_CAPACITY = 2,    /* max_batch / max_ctx / workspace too small for the call */
  WF_ERR_CUDA = 3,        /* a CUDA runtime or driver call failed */
  WF_ERR_UNSUPPORTED = 4, /* a shape the kernels do not support (see wf_config) */
  WF_ERR_DEVICE = 5       /* the device error word is set (see wf_get_error) */
} wf_status;

/* Device error word bits (wf_get_error). */
#define WF_DEV_ERR_TIMEOUT 0x1u  /* a bounded spin-wait gave up; results are invalid */
#define WF_DEV_ERR_CAPACITY 0x2u /* a sequence would pass max_ctx; it was frozen */
#define WF_DEV_ERR_TOKEN 0x4u    /* a token id outside [0, vocab) was clamped */
#define WF_DEV_ERR_LAUNCH 0x8u   /* a kernel found its launch inconsistent with its plan
                                    (grid, cluster or shared memory) and did nothing */
#define WF_DEV_ERR_PAGE 0x10u    /* a paged-cache call met a length, block id or slot out of
                                    bounds; what it names was skipped */

#define WF_MAX_TAPS 8
#define WF_MAX_LAYERS 64

/* Model shape.  Supported: head_dim = d_model / n_heads = 64; d_model a multiple
 * of 128 and at most 1536; d_ff a multiple of 64; block_k <= 8; max_pos <= 4096. */
typedef struct wf_config {
  int32_t d_model;        /* 1280 (Whisper large), 384 (tiny) */
  int32_t n_heads;        /* 20, 6 */
  int32_t d_ff;           /* 5120, 1536 */
  int32_t n_layers;       /* target decoder blocks: 32, 4 */
  int32_t vocab;          /* 51866, 51865 */
  int32_t max_pos;        /* learned text positions: 448 */
  int32_t enc_frames;     /* encoder frames per request: 1500 (30 s window) */
  int32_t n_draft_layers; /* drafter blocks: 2 (Sec. 3.2) */
  int32_t block_k;        /* proposals per round K: 8 (Eq. 2) */
  int32_t n_taps;         /* history taps: 5 (App. A.2) */
  int32_t taps[WF_MAX_TAPS]; /* zero-based target blocks tapped: 1,8,15,22,29 (App. A.2) */
  int32_t eos_id;         /* end-of-transcript id (App. A.1) */
  float rope_base;        /* drafter RoPE base: 10000 (App. A.2) */
  float ln_eps;           /* LayerNorm epsilon: 1e-5 */
} wf_config;

/* One Whisper decoder block (pre-LayerNorm).  qkv_w stacks the query, key and
 * value projections [3d, d] (bias [3d], key part zero); xkv_w stacks the
 * acoustic key and value projections [2d, d] (bias [2d], key part zero). */
typedef struct wf_layer_weights {
  const void *ln1_g, *ln1_b;    /* [d] */
  const void *qkv_w, *qkv_b;    /* [3d, d], [3d] */
  const void *out_w, *out_b;    /* [d, d], [d] */
  const void *ln2_g, *ln2_b;    /* [d] */
  const void *xq_w, *xq_b;      /* [d, d], [d] */
  const void *xkv_w, *xkv_b;    /* [2d, d], [2d] */
  const void *xout_w, *xout_b;  /* [d, d], [d] */
  const void *ln3_g, *ln3_b;    /* [d] */
  const void *fc1_w, *fc1_b;    /* [F, d], [F] */
  const void *fc2_w, *fc2_b;    /* [d, F], [d] */
} wf_layer_weights;

/* Frozen target decoder.  tok_emb is also the output head (tied). */
typedef struct wf_target_weights {
  const void *tok_emb;          /* [vocab, d] */
  const void *pos_emb;          /* [max_pos, d] */
  const void *lnf_g, *lnf_b;    /* [d] final LayerNorm, shared with the drafter */
  const wf_layer_weights *layers; /* HOST array of n_layers entries (copied at create) */
} wf_target_weights;

/* Drafter (Sec. 3.2, App. A.2).  Its blocks reuse wf_layer_weights: the key and
 * value rows of qkv_w also project the history memory.  It shares tok_emb, the
 * final LayerNorm and the head with the target. */
typedef struct wf_drafter_weights {
  const wf_layer_weights *layers; /* HOST array of n_draft_layers entries */
  const void *proj_w, *proj_b;  /* [d, n_taps*d], [d]: history projection */
  const void *hln_g, *hln_b;    /* [d]: LayerNorm after the projection */
  const void *mask_emb;         /* [d]: learned mask vector m (Eq. 2) */
} wf_drafter_weights;

/* Sampling parameters (App. A.4).  temperature == 0 selects greedy decoding.
 * d_suppress (nullable) is a device uint8 [vocab] mask; ids with a nonzero
 * entry get -inf logits in both the drafter and the target. */
typedef struct wf_sample_params {
  float temperature;
  uint32_t _pad;
  uint64_t seed;                /* Philox4x32-10 key */
  const uint8_t *d_suppress;
} wf_sample_params;

typedef struct wf_handle wf_handle;

/* Size of the workspace wf_create needs for these limits.  max_ctx <= max_pos. */
wf_status wf_workspace_bytes(const wf_config *cfg, int32_t max_batch, int32_t max_ctx,
                             size_t *out_bytes);

/* Build a handle over caller-owned weights and workspace.  Encodes the TMA
 * descriptors of every weight matrix and clears the per-sequence state on
 * `stream` (asynchronously).  d_workspace must be 256-byte aligned and every
 * weight pointer 16-byte aligned (else WF_ERR_INVALID). */
wf_status wf_create(const wf_config *cfg, const wf_target_weights *tw,
                    const wf_drafter_weights *dw, int32_t max_batch, int32_t max_ctx,
                    void *d_workspace, size_t workspace_bytes, void *stream,
                    wf_handle **out);

wf_status wf_destroy(wf_handle *h);

/* Admit n requests into batch slots (App. A.1, A.5): project the acoustic keys
 * and values of every target and drafter block from the encoder output (one
 * dense GEMM per block), run the prompt through the target in one causal pass
 * (filling its cache and the drafter's history memory), and emit the first
 * transcript token, which becomes the first anchor.
 *   d_slots   int32 [n]          distinct slots in [0, max_batch)
 *   d_enc     bf16  [n, enc_frames, d]   encoder output
 *   d_prompt  int32 [n, P]       prompt ids; P + 1 + block_k <= max_ctx
 *   d_budget  int32 [n]          output tokens allowed, >= 1
 *   d_first   int32 [n]          out: the first emitted token
 *   sp        nullable: greedy when null or temperature == 0
 * The admitted slots are appended to the active list. */
wf_status wf_prefill_cross_kv(wf_handle *h, int32_t n, const int32_t *d_slots,
                              const void *d_enc, const int32_t *d_prompt, int32_t P,
                              const int32_t *d_budget, int32_t *d_first,
                              const wf_sample_params *sp, void *stream);

/* Drafter forward for every active sequence (Sec. 3.2): one pass over
 * [Emb(anchor), m x K] per sequence, attending to its history memory and its
 * audio; writes K proposals per sequence into the handle (and, when sampling,
 * the draft logits). */
wf_status wf_draft(wf_handle *h, const wf_sample_params *sp, void *stream);

/* Verify [anchor, c_1..c_K] in one causal target pass, extend the drafter's
 * history with the block's states, and accept (Sec. 3.1, App. A.1):
 *   d_out_tokens int32 [max_batch, K+1] (per slot; entries past the count are -1)
 *   d_out_count  int32 [max_batch]      tokens emitted this step (0 if inactive)
 * d_forced (nullable) int32 [max_batch, K] replaces the drafter's proposals
 * (teacher forcing); the drafter's own pass is unaffected.
 * d_forced_q (nullable; needs d_forced) fp32 [max_batch, K, vocab]: the logits of
 * the distributions the forced proposals were drawn from, row j for proposal
 * c_{j+1}, in the units of the drafter's logits (they get the same temperature
 * and suppression).  When sampling, the rejection rule then uses
 * q = softmax(d_forced_q / T) in place of the drafter's distribution: the rule
 * preserves the target's distribution only if q is the distribution the
 * proposals actually came from (Sec. 3.1, App. A.4).  Ignored when greedy. */
wf_status wf_verify_accept(wf_handle *h, const wf_sample_params *sp,
                           const int32_t *d_forced, const float *d_forced_q,
                           int32_t *d_out_tokens, int32_t *d_out_count, void *stream);

/* wf_draft followed by wf_verify_accept. */
wf_status wf_step(wf_handle *h, const wf_sample_params *sp, const int32_t *d_forced,
                  const float *d_forced_q, int32_t *d_out_tokens, int32_t *d_out_count,
                  void *stream);

/* One plain autoregressive step of the target (Eq. 1; sampling when T > 0)
 * through the same kernels: the identity reference for the speculative path.
 * Outputs as wf_verify_accept (at most one token per slot). */
wf_status wf_greedy_step(wf_handle *h, const wf_sample_params *sp, int32_t *d_out_tokens,
                         int32_t *d_out_count, void *stream);

/* Rebuild the active list from the done flags (ascending slot order),
 * synchronise `stream`, and return the number of active sequences. */
wf_status wf_compact(wf_handle *h, void *stream, int32_t *h_n_active);

/* Rewind n slots to the state their prefill left (cache length, anchor,
 * budget, step counter) and re-activate them; the acoustic keys/values and
 * the prompt's cache rows are kept, so the same request decodes again. */
wf_status wf_reset_slots(wf_handle *h, int32_t n, const int32_t *d_slots, void *stream);

/* Copy per-slot state to HOST arrays (each [max_batch], any may be null) and
 * synchronise `stream`. */
wf_status wf_get_state(wf_handle *h, int32_t *h_len, int32_t *h_anchor, int32_t *h_remaining,
                       int32_t *h_done, void *stream);

/* Read (and optionally clear) the device error word; synchronises `stream`. */
wf_status wf_get_error(wf_handle *h, uint32_t *h_err, int32_t clear, void *stream);

/* Number of kernels the last call to a compute entry point launched. */
int32_t wf_last_launch_count(const wf_handle *h);

/* Inspection hooks for tests and profiling.  wf_set_option(WF_OPT_KEEP_LOGITS,
 * 1) makes every output-head pass also store raw fp32 logits (they are
 * stored anyway when sampling).  wf_debug_view returns the device address and
 * size of an internal buffer of the workspace (valid until wf_destroy; the
 * contents are those left by the last call that wrote them):
 *   WF_VIEW_TARGET_LOGITS  fp32 [rows][vocab]  rows of the last target head pass
 *   WF_VIEW_DRAFT_LOGITS   fp32 [rows][vocab]  rows of the last drafter pass
 *                          (row 9*i + j: sequence i of the active list, block row j)
 *   WF_VIEW_TAPS           bf16 [rows][n_taps*d] tapped residual streams (App. A.2)
 *   WF_VIEW_CANDIDATES     int32 [max_batch][K] proposals verified by the last step */
#define WF_OPT_KEEP_LOGITS 1
#define WF_OPT_PROFILE 2     /* 1: bracket every launch with CUDA events (serialises launches) */
#define WF_OPT_PDL 4         /* 1 (default): kernels use programmatic dependent launch */
#define WF_OPT_GRAPHS 3      /* 1 (default): wf_step / wf_greedy_step replay a CUDA graph
                                captured on first use per (active count, forcing, sampling
                                parameters); 0: launch kernel by kernel */
#define WF_OPT_PERSIST 5     /* 1: the blocks of every drafter, verify and greedy pass run
                                in one persistent cooperative launch (one CTA per SM, so
                                no other kernel may hold SMs meanwhile).  Off by default:
                                on GB300 it is slower than launch by launch.  Supported
                                when max_batch * (block_k + 1) <= 16, 64-wide heads,
                                d_model <= 1280, d_ff a multiple of 512 with
                                d_ff / 4 <= 1280, at most 2048 encoder frames and enough
                                SMs for at most five projection units per CTA; otherwise
                                setting it returns WF_ERR_UNSUPPORTED.  0: one launch per
                                projection and attention.  Both give results within the
                                tolerances of the method, not bit-identical ones. */
#define WF_OPT_SPIN_LIMIT 6  /* clock cycles a bounded wait in the projection kernels and the
                                persistent pass spins before it gives up (records
                                WF_DEV_ERR_TIMEOUT in the error word and returns; the kernel
                                still waits, with the default limit, for its own copies and
                                tensor-core work in flight before it exits).  0 (default)
                                restores about 1 s (projections) and 0.2 s (persistent pass).
                                Meant for tests of the failure path: a limit below a wait's
                                normal duration makes the results of that call invalid. */
#define WF_OPT_SKINNY 7      /* 1: passes of at most max_batch * (block_k + 1) <= 144 token
                                rows run their projections as low-latency kernels that hold
                                a CTA's whole weight slab in shared memory and reduce K in a
                                fixed order (up to 14 rows with the whole token operand
                                resident, more with it streamed by k-block); 0: the tcgen05
                                projections.  Default 1 when max_batch * (block_k + 1) <= 14
                                (single-sequence handles), else 0 (the streamed form is
                                slower than tcgen05 at 2-8 sequences and ties it at 16).
                                Setting 1 on a handle of more than 144 step rows returns
                                WF_ERR_UNSUPPORTED.
                                The two forms agree within the method's tolerances, not bit
                                for bit; a handle's speculative and plain greedy steps
                                always take the same form. */
#define WF_VIEW_TARGET_LOGITS 1
#define WF_VIEW_DRAFT_LOGITS 2
#define WF_VIEW_TAPS 3
#define WF_VIEW_CANDIDATES 4
wf_status wf_set_option(wf_handle *h, int32_t option, int32_t value);

/* Kernel families reported by wf_profile_read. */
#define WF_FAM_GEMM 0       /* tcgen05 projections (all but the output head) */
#define WF_FAM_HEAD 1       /* tcgen05 output head with its fused reduction records */
#define WF_FAM_ATTN_SELF 2  /* causal verify / prompt attention and the drafter's block attention */
#define WF_FAM_ATTN_CROSS 3 /* cross-attention over the encoder frames */
#define WF_FAM_LAYERNORM 4
#define WF_FAM_OTHER 5      /* embeddings, head reduction, accept, slot state */
#define WF_FAM_PERSIST 6    /* persistent small-batch pass: every block of a drafter,
                               verify or greedy pass in one launch (WF_OPT_PERSIST) */
#define WF_PROF_FAMILIES 7
/* With WF_OPT_PROFILE on: synchronise `stream`, then return per family the
 * summed kernel time (ms, CUDA events on the launching stream), the number of
 * launches and, for the GEMM and head families, the algorithmic bytes those
 * launches move (weights + token rows in + results out; split-K scratch is
 * not counted); for the persistent family the blocks' projection weights and
 * acoustic keys/values.  Each array has WF_PROF_FAMILIES entries; accumulators reset. */
wf_status wf_profile_read(wf_handle *h, void *stream, double *h_ms, int32_t *h_launches,
                          double *h_bytes);
wf_status wf_debug_view(wf_handle *h, int32_t which, void **d_ptr, size_t *bytes);

const char *wf_status_str(wf_status s);

/* ------------------------------------------------------------------------
 * Kernel-level entry points (device pointers, stream ordered).  They run one
 * kernel family of the step on caller buffers so each can be checked alone.
 * ---------------------------------------------------------------------- */

/* Y = X W^T (+ b): the skinny-M tcgen05 GEMM of every projection in the step.
 *   d_x bf16 [M, K], d_w bf16 [N, K], d_b bf16 [N] (nullable), d_y fp32 [M, N].
 *   K % 64 == 0, 1 <= M, 1 <= N.  Split-K partial sums are reduced on chip
 *   (thread-block cluster shared memory), so wf_gemm_scratch_bytes returns 0 and
 *   d_scratch may be null. */
wf_status wf_gemm_bf16(const void *d_x, const void *d_w, const void *d_b, float *d_y,
                       int32_t M, int32_t N, int32_t K, void *d_scratch,
                       size_t scratch_bytes, void *stream);
size_t wf_gemm_scratch_bytes(int32_t M, int32_t N, int32_t K);

/* Multi-head attention of RPS query rows per sequence against per-sequence
 * key/value caches laid out [slot][head][position][64] (bf16):
 *   d_q     bf16 [n_seq*RPS, n_heads*64]  queries, row r = seq*RPS + j
 *   d_kc/vc bf16 [n_slots, n_heads, ctx, 64]
 *   d_slot  int32 [n_seq]   cache slot of each sequence
 *   d_base  int32 [n_slots] position of query row 0 (the cache length L)
 *   mode 0: causal (query j sees keys [0, base+j]);  mode 1: all keys
 *   [0, base+RPS) (drafter block);  mode 2: all ctx keys (cross-attention)
 *   rope: nonzero applies RoPE (rope_base) to queries and keys by position
 *   d_out  bf16 [n_seq*RPS, n_heads*64] */
wf_status wf_attention(const void *d_q, const void *d_kc, const void *d_vc,
                       const int32_t *d_slot, const int32_t *d_base, int32_t n_seq,
                       int32_t RPS, int32_t n_heads, int32_t ctx, int32_t mode, int32_t rope,
                       float rope_base, void *d_out, void *d_scratch, size_t scratch_bytes,
                       void *stream);
size_t wf_attention_scratch_bytes(int32_t n_seq, int32_t RPS, int32_t n_heads, int32_t ctx);

/* wf_attention without a scratch argument, for callers that cannot allocate
 * device memory (a graph being captured in a mode that forbids cudaMalloc, a
 * plugin whose host framework owns every allocation, a latency-critical loop
 * that must not synchronise).  The paper has no counterpart: this is a
 * deployment convenience of this library.  Its scratch is one 8 MiB device
 * array inside the library, held by every GPU that loads it until exit;
 * calls needing more (wf_attention_scratch_bytes > 8 MiB) return
 * WF_ERR_CAPACITY.  The first call on a device looks the array up and may
 * load the library's module, so make it before any stream capture.  Every
 * call shares the array: calls that may overlap on the GPU race and must not
 * be issued.  Arguments and results are those of wf_attention. */
wf_status wf_attention_noalloc(const void *d_q, const void *d_kc, const void *d_vc,
                               const int32_t *d_slot, const int32_t *d_base, int32_t n_seq,
                               int32_t RPS, int32_t n_heads, int32_t ctx, int32_t mode,
                               int32_t rope, float rope_base, void *d_out, void *stream);

/* ------------------------------------------------------------------------
 * Beam decode over a paged key/value cache held in 4 bits.  The calls below
 * take no handle: every buffer is the caller's, every call is asynchronous on
 * its stream, and a step of beam search is
 *   wf_page_plan      blocks and slots for the step's new tokens,
 *   wf_kv4_store      the new keys and values of a layer,
 *   wf_kv4_attention  the layer's attention (self and cross),
 *   wf_beam_select    the next tokens and their parents,
 *   wf_beam_reorder   the block tables after the selection.
 * d_err (nullable) is a device uint32 that the call ORs WF_DEV_ERR_* bits
 * into; the caller clears it.
 * ---------------------------------------------------------------------- */

#define WF_BF16 0
#define WF_F16 1
#define WF_F32 2
#define WF_KV4_GROUP 64   /* values that share a scale and an offset */
#define WF_KV4_RECORD 1152 /* bytes of 16 positions of one group, keys and values */
#define WF_MAX_BEAMS 16

/* A paged cache in 4 bits.  A block holds block_size positions of every
 * key/value head; the same block id names that block in each of n_layers
 * layers, layer l starting at d_base + l * layer_stride bytes.  A row of a
 * head is cut into groups of 64 values (head_dim 64: one, 128: two).  A value
 * of a group is s (c - 8) + z: c a code of 4 bits, s and z the group's scale
 * and offset in `dtype` (WF_BF16 or WF_F16), which is also the type of the
 * rows stored and of the queries.  From a group's extremes,
 *   s = round((max - min) / 15), z = round(max - 7 s),
 *   c = clamp(rint((x - z) / s), -8, 7) + 8   (8 where s is 0),
 * in fp32, rounded to nearest even; a group with a value that is not finite
 * reads back as NaN.
 * Layout: [block][head][group][block_size / 16][1152 bytes].  A record of 16
 * positions holds 512 bytes of key codes (32 a position, low nibble first),
 * 512 of value codes in the order the attention's tensor instructions take
 * them, and 128 of (s, z) pairs: [position % 8][keys, values][position / 8]. */
typedef struct wf_kv4_pool {
  void *d_base;         /* 16-byte aligned */
  int64_t layer_stride; /* bytes, a multiple of 16; 0: n_blocks * wf_kv4_block_bytes() */
  int32_t n_layers;
  int32_t n_blocks;     /* block ids are 0 .. n_blocks - 1; n_blocks * block_size < 2^31 */
  int32_t block_size;   /* 16, 32 or 64 positions */
  int32_t n_kv_heads;
  int32_t head_dim;     /* 64 or 128 */
  int32_t dtype;        /* WF_BF16 or WF_F16 */
} wf_kv4_pool;

/* Bytes of one block in one layer; 0 for a shape that is not supported. */
size_t wf_kv4_block_bytes(int32_t block_size, int32_t n_kv_heads, int32_t head_dim);

/* Block tables and slot maps from request lengths.  Request i (0 <= i < n,
 * n <= 65536) grows from d_old_len[i] to d_new_len[i] positions.  Its table row,
 * d_table + i * table_stride, names the blocks of its first
 * ceil(old / block_size) columns; the columns up to ceil(new / block_size) are
 * filled from the free list, a stack of *d_n_free ids in d_free (capacity
 * n_blocks): request by request, column by column, from the top.
 *   d_offsets  int32 [n + 1]      out: request i's new tokens are
 *                                 [d_offsets[i], d_offsets[i + 1])
 *   d_slots    int32 [slots_cap]  out: of each new token, block * block_size +
 *                                 position % block_size; -1 after the last
 *                                 (slots_cap < 2^31 - 2^20)
 *   d_len      int32 [n]          out: new length if granted, else the old one
 *   d_n_free_out int32 [1]        out: ids left
 * Requests are granted in order; the first whose blocks or slots do not fit,
 * and all after it, are refused whole (WF_DEV_ERR_CAPACITY).  A request with
 * old < 0, new < old or more than table_stride columns is refused alone
 * (WF_DEV_ERR_PAGE).  d_len and d_n_free_out are buffers of their own, not
 * d_old_len, d_new_len or d_n_free: all of the grid reads those. */
wf_status wf_page_plan(const int32_t *d_old_len, const int32_t *d_new_len, int32_t n,
                       int32_t block_size, const int32_t *d_free, int32_t n_blocks,
                       const int32_t *d_n_free, int32_t *d_table, int32_t table_stride,
                       int32_t *d_offsets, int32_t *d_slots, int32_t slots_cap, int32_t *d_len,
                       int32_t *d_n_free_out, uint32_t *d_err, void *stream);

/* Quantise n rows of keys and values into one layer of the cache.
 *   d_k, d_v  dtype [n][n_kv_heads * head_dim], row strides in elements
 *             (multiples of 8; pointers 16-byte aligned)
 *   d_slots   int32 [n]: a negative slot skips its row.  The others are
 *             distinct: rows are written by many threads without order, so a
 *             slot named twice may hold one row's codes under another's scale
 *             (no other slot is touched)
 * wf_kv4_load reads the slots back into rows (zeros for a negative slot). */
wf_status wf_kv4_store(const wf_kv4_pool *pool, int32_t layer, const void *d_k, int64_t k_stride,
                       const void *d_v, int64_t v_stride, const int32_t *d_slots, int32_t n,
                       uint32_t *d_err, void *stream);
wf_status wf_kv4_load(const wf_kv4_pool *pool, int32_t layer, const int32_t *d_slots, int32_t n,
                      void *d_k, int64_t k_stride, void *d_v, int64_t v_stride, uint32_t *d_err,
                      void *stream);

/* Attention of rps query rows per sequence over one layer of the cache:
 * softmax(scale q K^T) V, n_heads query heads on n_kv_heads (n_heads a
 * multiple; query head h reads key/value head h / (n_heads / n_kv_heads)).
 *   d_q     dtype [n_seq * rps][n_heads * head_dim], row r = seq * rps + j
 *   d_table int32, sequence i's blocks at d_table + i * table_stride (the
 *           sequences may share blocks, and stride 0 shares one row)
 *   d_len   int32 [n_seq]  positions held; the rps rows are the last of them
 *           when causal: row j sees len - (rps - 1 - j) positions, else len
 *   max_len a bound on d_len, at most 2^31 - 1024; longer sequences are cut
 *           to it (WF_DEV_ERR_CAPACITY)
 *   d_out   dtype [n_seq * rps][n_heads * head_dim]
 * Strides are in elements, multiples of 8, pointers 16-byte aligned; d_out is
 * not d_q.  A row that sees nothing is zeros; a block id outside the pool is not read and its
 * positions are not seen (WF_DEV_ERR_PAGE).  Scores, softmax and sums are
 * fp32; a weight times its value's s is rounded for the second product, to bf16
 * for a bf16 cache and to at least 11 bits for an fp16 one (of weights down to
 * 2^-14 of a row's largest; of smaller ones at most 2^-25 of the s is lost).
 * Results do not depend on timing.  d_scratch (16-byte aligned) holds
 * wf_kv4_attention_scratch_bytes() bytes and belongs to the call until it is
 * done. */
wf_status wf_kv4_attention(const wf_kv4_pool *pool, int32_t layer, const void *d_q,
                           int64_t q_stride, const int32_t *d_table, int32_t table_stride,
                           const int32_t *d_len, int32_t n_seq, int32_t rps, int32_t n_heads,
                           int32_t causal, float scale, int32_t max_len, void *d_out,
                           int64_t out_stride, void *d_scratch, size_t scratch_bytes,
                           uint32_t *d_err, void *stream);
size_t wf_kv4_attention_scratch_bytes(int32_t n_seq, int32_t rps, int32_t n_heads,
                                      int32_t n_kv_heads, int32_t head_dim, int32_t max_len);

/* One selection of beam search.  Beam w of request i has the logits row
 * i * beams + w (`dtype` WF_F32, WF_BF16 or WF_F16, ld elements apart, at any
 * alignment of the type) and
 * the score d_scores[i * beams + w], the sum of its log-probabilities (-inf:
 * not in use).  A token's score is score + ((logit - max) - log(sum)) in fp32,
 * max the row's largest logit and sum that of exp(logit - max); ids with a nonzero d_suppress entry (nullable uint8
 * [vocab]) and NaN logits count as -inf; a row whose largest logit is +inf has
 * no scores and proposes nothing.  Each beam proposes its 2 beams best
 * tokens (ties: the lower id); of all proposals the 2 beams best are ranked
 * (ties: the lower beam, then its better token).  Then
 *   d_token, d_parent int32, d_score fp32 [n_req][beams]  the first `beams`
 *       that are not eos, best first; past the last one -1, the beam itself
 *       and -inf
 *   d_fin_parent int32, d_fin_score fp32 [n_req][beams]  hypotheses that end:
 *       eos among the first `beams` ranks; past the last one -1 and -inf
 * eos < 0: none ends.  2 beams <= vocab <= 2^22.  d_score may be d_scores. */
wf_status wf_beam_select(const void *d_logits, int32_t dtype, int64_t ld, const float *d_scores,
                         const uint8_t *d_suppress, int32_t n_req, int32_t beams, int32_t vocab,
                         int32_t eos, int32_t *d_token, int32_t *d_parent, float *d_score,
                         int32_t *d_fin_parent, float *d_fin_score, void *d_scratch,
                         size_t scratch_bytes, void *stream);
size_t wf_beam_select_scratch_bytes(int32_t n_req, int32_t beams, int32_t vocab);

/* The block tables of n_req requests' beams after a selection.  Beam w of
 * request i has the table row i * beams + w and d_len[i * beams] positions
 * (equal for the request's beams).  Beams of a request may share full blocks;
 * a last block that is partly filled belongs to one beam.  New beam w takes
 * beam d_parent[i * beams + w]'s full blocks; a parent's first child keeps its
 * last block, each other child gets the last block of a beam without children
 * and the parent's contents in it, in every layer (by 16 positions).  A parent
 * of -1 drops the beam's history: its row holds -1 but for a last block of its
 * own; if all of a request's parents are -1 the request is released.  Blocks
 * that no beam of the request holds any more are pushed on the free list
 * (d_free, capacity pool->n_blocks, *d_n_free ids before, *d_n_free_out
 * after; they may be one), by request, column and beam; an id outside the pool
 * is not pushed (WF_DEV_ERR_PAGE).  Columns past the length are not written.
 * d_table_out may be d_table_in. */
wf_status wf_beam_reorder(const wf_kv4_pool *pool, const int32_t *d_table_in, int32_t *d_table_out,
                          int32_t table_stride, const int32_t *d_len, const int32_t *d_parent,
                          int32_t n_req, int32_t beams, int32_t *d_free, const int32_t *d_n_free,
                          int32_t *d_n_free_out, void *d_scratch, size_t scratch_bytes,
                          uint32_t *d_err, void *stream);
size_t wf_beam_reorder_scratch_bytes(int32_t n_req, int32_t beams, int32_t table_stride);

#ifdef __cplusplus
}
#endif
#endif /* WF_H */
