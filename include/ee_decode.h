/*
 * ee_decode.h -- C ABI of the early-exit decode step for MI355X (gfx950).
 *
 * One call of ee_decode_iteration is one iteration of the paper's Algorithm 1
 * ("Iteration-level Batch Inference for Early-exit LLMs"): one new token for every
 * sequence of a batch, with the per-sequence sticky exit status of Section 3.1, the
 * whole-batch break at output_layer, and the KV-cache filling of Section 3.2.  The
 * other entry points expose the steps of that iteration one by one.
 *
 * Conventions
 *   - "dev" pointers are DEVICE pointers owned by the caller; the library borrows
 *     them for the duration of the enqueued work and never frees them.  "host"
 *     pointers are read before the call returns.
 *   - Every call only ENQUEUES work on `stream` (a hipStream_t passed as void*,
 *     NULL = the default stream) and returns without synchronising.  Outputs are
 *     valid once the caller has synchronised the stream.  No call allocates or
 *     frees device memory; scratch space comes in through `workspace`.
 *   - Layers are 1-based in every argument and output, as in Algorithm 1.
 *   - Return value: EE_OK, or a negative error code.  Arguments are validated on
 *     the host before anything is launched; on error nothing has been enqueued.
 *     ee_last_error() returns a thread-local message for the last failing call.
 *     Data errors that only the device can see (a block id outside 0..num_blocks-1,
 *     a position outside the block table, a row_table entry outside 0..B-1, a token
 *     id outside 0..vocab-1) are the
 *     caller's contract: the result for such a sequence is unspecified.  The kernels
 *     keep such an access inside the caller's buffers all the same (the id is read as
 *     0, the cache write is dropped), so bad data cannot fault the device.
 *   - dtype EE_FP32: weights, activations and KV cache are float; matrices are plain
 *     row-major [out_features][in_features].
 *     dtype EE_BF16: weights, embedding, gains and KV cache are bfloat16; matrices
 *     are in the MFMA tile order written by ee_pack_weight.  The residual stream,
 *     q, softmax statistics, logits and confidences are float in both cases.
 *   - Projections of more than 32 rows (EE_BF16) take up to 140 KiB of LDS per workgroup, of the 160 KiB that
 *     every compute unit of gfx950 has.  It is part of their code objects and not asked for, so no call checks
 *     for it.  (Two kernels ask for 128 KiB, the LM head's and gate/up's from 385 rows on and prompt attention's;
 *     where the runtime refuses that, others take their place.)
 */
#ifndef EE_DECODE_H
#define EE_DECODE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EE_OK 0
#define EE_ERR_INVALID_ARG (-1)  /* null pointer, non-positive size, bad enum          */
#define EE_ERR_SHAPE (-2)        /* sizes inconsistent with each other                 */
#define EE_ERR_UNSUPPORTED (-3)  /* a shape or mode this build has no kernel for       */
#define EE_ERR_WORKSPACE (-4)    /* workspace too small or misaligned                  */
#define EE_ERR_HIP (-5)          /* a HIP call failed (message in ee_last_error)       */

#define EE_FP32 0
#define EE_BF16 1

/* Row orders understood by ee_pack_weight. */
#define EE_PACK_PLAIN 0    /* w_o, w_down, w_lm                                           */
#define EE_PACK_QKV 1      /* w_qkv : rotary partners (j, j + head_dim/2) share a tile    */
#define EE_PACK_GATE_UP 2  /* w_gate_up : gate row f and up row f share a tile            */

#define EE_MAX_LAYERS 64

typedef struct ee_model_desc {
  int32_t n_layers, d_model, n_heads, head_dim, d_ffn, vocab; /* d_model == n_heads * head_dim */
  int32_t dtype;       /* EE_FP32 | EE_BF16                                                        */
  float rms_eps;       /* RMSNorm epsilon                                                          */
  float rope_theta;    /* rotary base; <= 0 disables the rotary embedding                         */
  int32_t exit_every;  /* exit head after layers i with i % exit_every == 0 and i < n_layers       */
  float logit_scale;   /* s: exit-head logits at layer i are multiplied by s * i                   */
  int32_t conf_mode;   /* confidence measure of the paper's Section 2.1.
                          0: largest softmax probability of the exit head;
                          1: top-1 minus top-2 probability (softmax response as the paper writes it);
                          2: hidden states similarity, cos(h_{i-1}, h_i) of the hidden states before and
                             after layer i (h_0 = the embedding), on the float residual stream;
                          3: dedicated classifier, 1 / (1 + exp(-(w_cls[i] . x_i + b_cls[i]))) with
                             x_i = h_i / sqrt(mean(h_i^2) + rms_eps), the hidden state at unit root mean square.
                          2 and 3 touch no LM head inside the layer loop (logit_scale is unused); the
                          tokens then come from one LM-head pass over the hidden state at output_layer */
} ee_model_desc;

/* Weights of one decoder layer (all dev).  Plain shapes: g_attn,g_ffn [d]; w_qkv [3d][d] (q rows, then
 * k rows, then v rows); w_o [d][d]; w_gate_up [2f][d] (gate rows, then up rows); w_down [d][f].
 * For EE_BF16 the matrices are the ee_pack_weight images of those plain matrices. */
typedef struct ee_layer_weights {
  const void *g_attn, *w_qkv, *w_o, *g_ffn, *w_gate_up, *w_down;
} ee_layer_weights;

typedef struct ee_model {
  ee_model_desc desc;
  const void* embed;              /* dev [vocab][d], plain row-major in the model dtype            */
  const void* g_final;            /* dev [d]; final RMSNorm gain, shared by every exit head        */
  const void* w_lm;               /* dev [vocab][d]; LM head (packed PLAIN for EE_BF16), shared by
                                     every exit head and by the final token selection              */
  const ee_layer_weights* layers; /* host array [n_layers]                                         */
  const float* w_cls;             /* dev [n_layers][d] float, row i-1 = classifier of layer i; may be
                                     NULL unless conf_mode == 3                                     */
  const float* b_cls;             /* dev [n_layers] float, its biases; may be NULL unless conf_mode == 3 */
} ee_model;

/* Paged KV cache (the block-virtualised cache the paper inherits, Section 2.2 / 3.2).
 * k_pool and v_pool: dev [n_layers][num_blocks][n_heads][block_size][head_dim] in the model dtype.
 * block_size must be 16.  Position p of sequence b lives in block block_tables[b][p / 16] at offset p % 16.
 * Slots that hold no position of a sequence (the rest of its last block, blocks nobody owns) may contain
 * anything, NaN included: the attention kernels never let them reach a result.  What one sequence has cached, Inf and
 * NaN included, reaches no other sequence's attention. */
typedef struct ee_kv_cache {
  void* k_pool;
  void* v_pool;
  int32_t num_blocks, block_size;
} ee_kv_cache;

/* One batch of sequences, one token each.  The block allocator is the caller's: the library only
 * dereferences block_tables, and writes position context_lens[b] of sequence b (whose block must exist). */
typedef struct ee_batch {
  int32_t batch;               /* B >= 0; B == 0 is a no-op that still returns EE_OK                     */
  const int32_t* tokens;       /* dev [B]: token each sequence consumes this iteration                   */
  const int32_t* context_lens; /* dev [B]: p_b = positions already cached; the new K/V go to position p_b */
  const int32_t* block_tables; /* dev [B][max_blocks]: physical block of each logical block (with row_table:
                                  one row per sequence, at least max(row_table) + 1 rows)                */
  int32_t max_blocks;          /* row pitch of block_tables                                              */
  int32_t max_context;         /* host-side upper bound of context_lens[b] + 1 (sizes the attention grid) */
  const int32_t* row_table;    /* dev [B] or NULL.  NULL: row b of the batch uses row b of block_tables.  Else
                                  row b uses row row_table[b]: several rows may then share one sequence's block
                                  table at consecutive positions p, p+1, .. (a chunk of a prompt pushed through
                                  in one call: every row caches its K/V before any row attends, and row b
                                  attends positions 0..context_lens[b], so the chunk is causal).  Only with
                                  EE_EXIT_NONE, and with ee_paged_attention_decode.                          */
} ee_batch;

const char* ee_last_error(void);

/* Number of bytes ee_pack_weight writes for an [n_out][n_in] matrix (EE_BF16 only). */
size_t ee_packed_weight_bytes(int32_t n_out, int32_t n_in);

/* Reorders a plain bf16 matrix w [n_out][n_in] (dev) into the tile order the MFMA kernels stream:
 * tiles of 32 output rows x 16 input columns, stored [row_tile][col_tile][lane 0..63][8 values], so that a
 * wavefront fetches one operand tile as 1 KiB of consecutive bytes.  `order` (EE_PACK_*) says which output
 * rows share a tile; pair_stride is head_dim/2 for EE_PACK_QKV, d_ffn for EE_PACK_GATE_UP, ignored for PLAIN.
 * n_out must be a multiple of 32, n_in of 16, pair_stride of 16.  A set-up step, not part of the decode step. */
int ee_pack_weight(const void* w /*dev*/, int32_t n_out, int32_t n_in, int32_t order, int32_t pair_stride,
                   void* packed /*dev*/, void* stream);

/* Scratch bytes the calls below need for batches up to max_batch and contexts up to max_context.
 * The workspace must be 256-byte aligned.  Its contents need no initialisation and are dead between calls. */
size_t ee_workspace_bytes(const ee_model_desc* desc, int32_t max_batch, int32_t max_context);

/* One decode iteration: Algorithm 1 of the paper.
 *   embed the batch's tokens; for layer i = 1..n run the layer over the whole batch (caching this position's
 *   K/V of layer i), evaluate the exit head on every sequence whose status is still false, OR the result into
 *   the status (sticky), and stop at the first layer where every status is true (output_layer); fill K/V of
 *   this position for layers output_layer+1..n from the hidden state at output_layer (Section 3.2); pick the
 *   greedy token of every sequence from that hidden state.
 * The layer loop is enqueued once: a device-side flag makes the kernels of the layers after output_layer
 * return at once, so there is no host round trip inside the iteration.
 *   thresholds        host [n_layers]: lambda_i; accepted means confidence > lambda_i (strict).
 *   forced_exit_layer dev [B] or NULL: synthetic confidence injection; the decision of sequence b at layer i
 *                     becomes (i >= forced_exit_layer[b]) while the exit-head arithmetic still runs.
 *   use_exit_heads    EE_EXIT_NONE (0): full-layer baseline, no exit check is made, output_layer = n.
 *                     EE_EXIT_BATCH (1): Algorithm 1 as above.
 *                     EE_EXIT_PER_SEQUENCE (2): an extension of Algorithm 1 in which each sequence leaves on its
 *                     own: once its status is true, later layers neither attend for it nor change its hidden
 *                     state; the loop still ends at the first layer after which every status is true
 *                     (output_layer = the largest exit layer); K/V of all layers above a sequence's OWN exit
 *                     layer are filled from its own exit hidden state (Section 3.2 applied per sequence), and
 *                     its token comes from that state.
 *   out_tokens        dev [B] int32: greedy token (lowest index on ties).
 *   out_exit_layer    dev [B] int32: first layer whose check accepted the sequence, n_layers if none.
 *   out_batch_exit_layer dev [1] int32: output_layer.
 *   out_conf          dev [n_layers][B] float or NULL: confidence evaluated at each layer; NaN where no check
 *                     was made (no head, sequence already accepted, layer not run).
 *   out_hidden        dev [B][d] float or NULL: hidden state at output_layer (what the tokens come from). */
#define EE_EXIT_NONE 0
#define EE_EXIT_BATCH 1
#define EE_EXIT_PER_SEQUENCE 2
int ee_decode_iteration(const ee_model* model, const ee_kv_cache* cache, const ee_batch* batch,
                        const float* thresholds, const int32_t* forced_exit_layer, int32_t use_exit_heads,
                        int32_t* out_tokens, int32_t* out_exit_layer, int32_t* out_batch_exit_layer,
                        float* out_conf, float* out_hidden, void* workspace, size_t workspace_bytes, void* stream);

/* The exit check of one layer (Section 3.1 status rule with the softmax-response confidence of Section 2.1;
 * conf_mode 0 or 1 only: EE_ERR_UNSUPPORTED for the measures without an exit head, which need the layer loop):
 * z = (logit_scale * layer) * (RMSNorm(hidden; g_final) . W_lm^T); confidence per conf_mode; a sequence whose
 * status is 0 and whose confidence exceeds `threshold` gets status 1 and exit_layer = layer; statuses never
 * revert.  n_exited counts the sequences with status 1; done_flag is set to 1 (and batch_exit_layer to `layer`)
 * when it reaches `batch`, and is left alone otherwise.
 *   hidden dev [B][d] float.  status, exit_layer dev [B] int32 in/out.  n_exited, done_flag, batch_exit_layer
 *   dev [1] int32 in/out.  argmax dev [B] int32 or NULL (arg max of the logits, every row).  conf dev [B] float
 *   or NULL (NaN for rows whose status was already 1).  forced_exit_layer as above. */
int ee_exit_check(const ee_model* model, int32_t layer, const float* hidden, int32_t batch, float threshold,
                  const int32_t* forced_exit_layer, int32_t* status, int32_t* exit_layer, int32_t* n_exited,
                  int32_t* done_flag, int32_t* batch_exit_layer, int32_t* argmax, float* conf, void* workspace,
                  size_t workspace_bytes, void* stream);

/* The same exit check for callers that cannot allocate device memory or hand over a workspace: code running
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, semantics and
 * results as ee_exit_check without the workspace: the scratch memory is a static device array of
 * EE_NOALLOC_SCRATCH_BYTES inside the library (each GPU the library runs on holds its own copy until the process
 * ends).  The call allocates and frees nothing.  A shape and batch that need more scratch than the array holds
 * (ee_exit_check_noalloc_bytes says how much: roughly batch * (vocab / 2 + 2 * d_model) bytes for EE_BF16, batch *
 * 4 * vocab for EE_FP32) are refused with EE_ERR_WORKSPACE before anything is enqueued.
 * Every call on one GPU uses that GPU's one array: calls that overlap on a GPU (two streams, two threads) race;
 * calls on one stream are ordered and each clears what it needs to start at zero.
 * ee_noalloc_init resolves the array's device address for the current device (one host-side query, no
 * allocation) and sets the function attributes of the projection and prompt-attention kernels; all of it is otherwise
 * done by the first call that needs it, so call it beforehand if that first call would fall inside a graph capture. */
#define EE_NOALLOC_SCRATCH_BYTES (8u << 20)
int ee_noalloc_init(void);
size_t ee_exit_check_noalloc_bytes(const ee_model_desc* desc, int32_t batch);
int ee_exit_check_noalloc(const ee_model* model, int32_t layer, const float* hidden, int32_t batch, float threshold,
                          const int32_t* forced_exit_layer, int32_t* status, int32_t* exit_layer, int32_t* n_exited,
                          int32_t* done_flag, int32_t* batch_exit_layer, int32_t* argmax, float* conf, void* stream);

/* KV-cache filling (Algorithm 1's second loop, Section 3.2): for every sequence b and every layer
 * i > fill_from_layer[b], K = RoPE(RMSNorm(hidden_b; g_attn_i) . Wk_i^T, p_b), V = RMSNorm(..) . Wv_i^T, written to
 * position p_b = context_lens[b] of layer i.  The paper's rule passes the same output_layer for every b.
 *   hidden dev [B][d] float; fill_from_layer dev [B] int32.  batch->tokens is not read. */
int ee_kv_fill(const ee_model* model, const ee_kv_cache* cache, const ee_batch* batch, const float* hidden,
               const int32_t* fill_from_layer, void* workspace, size_t workspace_bytes, void* stream);

/* Single-query attention over the paged cache of one layer (the attention inside Algorithm 1's M(i, ...)):
 * out[b][h] = softmax_j(q[b][h] . K[b][j][h] / sqrt(head_dim)) . V[b][j][h], j = 0..context_lens[b] INCLUSIVE: the new
 * token's K/V must already be in the cache.   q dev [B][H][dh] float, rotary embedding applied.
 * out dev [B][H][dh] float.  batch->tokens is not read.
 * workspace (dev, 16-byte aligned) may be NULL.  With B * H <= 64 and a block table at least 16 blocks wide, a
 * workspace of at least B * H * 8 * (head_dim + 2) * 4 bytes lets up to eight workgroups share one (sequence, head)
 * pair, each over a contiguous part of the context, merged in a fixed order by a second launch (single-stream decoding
 * over a long context would otherwise keep only B * H compute units busy); a smaller or missing one is not an error,
 * the call then runs one workgroup per pair.  ee_decode_iteration does the same out of its own workspace. */
int ee_paged_attention_decode(const ee_model_desc* desc, const ee_kv_cache* cache, int32_t layer, const float* q,
                              const ee_batch* batch, float* out, void* workspace, size_t workspace_bytes,
                              void* stream);

/* ---- An 8-bit paged cache, and the steps around it ------------------------------------------------------------
 * For programs that run a model's layers one call at a time: rotary positions, a cache of half (EE_BF16) or a quarter of
 * the bytes, the attention that reads it, and an eviction that bounds its length.  Same conventions as above: nothing
 * here allocates, synchronises or keeps anything between calls.
 *
 * Positions are counted twice.  `positions` of ee_rotary are the places in the text; context_lens of the other calls
 * are slots of the cache.  The two differ once a sequence has been through ee_kv_quant_evict. */

#define EE_ROTARY_HALF 0         /* pair j = channels j and j + rotary_dim/2                              */
#define EE_ROTARY_INTERLEAVED 1  /* pair j = channels 2j and 2j + 1                                       */

#define EE_ROTARY_PLAIN 0   /* f_j = theta^(-2j / rotary_dim)                                             */
#define EE_ROTARY_LINEAR 1  /* f_j / factor: positions squeezed into the context the model was trained on */
#define EE_ROTARY_TURNS 2   /* by how often pair j turns within original_context, t = original_context f_j / (2 pi):
                               f_j (w + (1 - w) / factor), w = (t - turns_low) / (turns_high - turns_low) within 0..1:
                               fast pairs keep their frequency, slow ones are squeezed                    */

typedef struct ee_rotary_desc {
  int32_t head_dim;    /* channels of a head, 2 .. 1024                                                   */
  int32_t rotary_dim;  /* even, 2 .. head_dim: the first rotary_dim channels are rotated, the others copied */
  int32_t layout;      /* EE_ROTARY_HALF | EE_ROTARY_INTERLEAVED                                          */
  int32_t scaling;     /* EE_ROTARY_PLAIN | _LINEAR | _TURNS                                              */
  int32_t original_context;     /* >= 1 (TURNS)                                                           */
  double theta;        /* > 0                                                                             */
  double factor;       /* > 0 (LINEAR, TURNS)                                                             */
  double turns_low, turns_high; /* low < high (TURNS)                                                     */
  double amplitude;    /* multiplies every rotated pair (1 = a rotation; finite as a float)               */
} ee_rotary_desc;

/* The rows of one tensor [rows][n_heads][head_dim]: heads and channels are consecutive, rows `stride` elements apart
 * (>= n_heads * head_dim).  in == out with equal strides works in place; otherwise the two must not overlap, nor may the
 * out of q overlap the in or out of k, or the out of k the in of q (rows of one buffer that lie between each other do not). */
typedef struct ee_rotary_rows {
  const void* in;      /* dev                                                                             */
  void* out;           /* dev                                                                             */
  int64_t in_stride, out_stride;
  int32_t n_heads;
} ee_rotary_rows;

/* Angular frequency per position of every pair, in double: freqs dev [rotary_dim/2].  A set-up step: the result serves
 * every later call with the same desc.  A caller with a scaling of its own fills freqs itself. */
int ee_rotary_frequencies(const ee_rotary_desc* desc, double* freqs, void* stream);

/* Rotary embedding of query and key rows in one launch: for every row m, head and pair j with channels (a, b)
 *   (a, b) -> amplitude * (a cos w - b sin w, a sin w + b cos w),   w = positions[m] * freqs[j],
 * the angle formed in double, the rest in float, rounded once to `dtype` (EE_FP32 | EE_BF16: the type of all four
 * tensors).  transpose = 1 multiplies by the transposed matrix instead (sin w -> -sin w): the gradient of `in` from
 * the gradient of `out`.
 *   positions dev [rows] int32 (any value).  q, k host; either may be NULL, not both. */
int ee_rotary(const ee_rotary_desc* desc, const double* freqs, const int32_t* positions, int32_t rows, int32_t dtype,
              const ee_rotary_rows* q, const ee_rotary_rows* k, int32_t transpose, void* stream);

#define EE_QUANT_INT8 0  /* a byte is a signed integer -127..127; the scale is a float                    */
#define EE_QUANT_E4M3 1  /* a byte is a float of 4 exponent and 3 mantissa bits (largest 448, no infinity); the scale
                            is a power of two                                                            */

/* Paged cache in 8 bits with one scale for each block of 16 positions and head, K and V apart.  A byte stands for the
 * float (byte's value) * scale.  Block tables as in ee_kv_cache.  Pools start on 16 bytes.
 * Slots that hold no position of a sequence may contain anything in bytes and scales.  The bytes of a cached position
 * are finite (ee_kv_quant_append writes no others). */
typedef struct ee_quant_cache {
  void* k_pool;        /* dev [n_layers][num_blocks][n_kv_heads][16][head_dim]                            */
  void* v_pool;        /* dev [n_layers][num_blocks][n_kv_heads][head_dim][16]                            */
  float* scales;       /* dev [n_layers][num_blocks][n_kv_heads][2]: of K, of V                           */
  int32_t n_layers, num_blocks, block_size; /* block_size must be 16                                      */
  int32_t n_kv_heads, head_dim;             /* head_dim: a multiple of 16, 16 .. 256                      */
  int32_t format;      /* EE_QUANT_INT8 | EE_QUANT_E4M3                                                   */
} ee_quant_cache;

/* Caches K and V of the batch's rows: row m goes to position context_lens[m] of its sequence.  With row_table several rows
 * may share a sequence; those that fall into one block stand next to each other in the batch, at consecutive ascending
 * positions.  A row with context_lens[m] < 0 is skipped (padding), and so is one whose row_table entry is none.
 * A block's scale is the smallest with which the largest magnitude ever appended to it fits,
 *   INT8: float(largest / 127), at least 2^-126;   E4M3: the smallest power of two with largest <= 448 * scale, at least
 *   2^-126,
 * (the largest float included: INT8 scales end at 0x1.020406p+121, 127 times which is a float, and with 2^120, E4M3's last one, bytes end at 240)
 * and the first position of a block starts anew, whatever the block held.  Where a call makes a block's scale grow, the
 * positions in front of the call's are rounded again, from the floats their bytes stood for.  Every rounding is to the
 * nearest, ties to even, of the exact quotient.  An infinity or NaN makes the block's scale NaN (every result that
 * depends on the block is then NaN, until the block starts anew).
 *   k, v dev, rows [n_kv_heads][head_dim] of `dtype` (EE_FP32 | EE_BF16), k_stride / v_stride elements apart (even, >=
 *   n_kv_heads * head_dim), starting on 8 (EE_FP32) or 4 bytes.  batch->tokens is not read. */
int ee_kv_quant_append(const ee_quant_cache* cache, int32_t layer, const void* k, int64_t k_stride, const void* v,
                       int64_t v_stride, int32_t dtype, const ee_batch* batch, void* stream);

/* The floats that the cache holds: row m reads position context_lens[m] of its sequence (row_table as above; any
 * order).  k, v dev [rows][n_kv_heads][head_dim] of `dtype`, starting on 8 (EE_FP32) or 4 bytes, not overlapping; zeros for
 * context_lens[m] < 0 or a row_table entry that is none. */
int ee_kv_quant_read(const ee_quant_cache* cache, int32_t layer, const ee_batch* batch, void* k, void* v, int32_t dtype,
                     void* stream);

/* Attention of single queries over the 8-bit cache:
 *   out[m][h] = softmax_j(q[m][h] . K[j][h / g] / sqrt(head_dim)) . V[j][h / g],  j = 0..context_lens[m] INCLUSIVE,
 * with g = n_heads / n_kv_heads query heads to a K/V head.  Rows that share a sequence (row_table) are a causal chunk of a
 * prompt, and quickest when they stand next to each other.  A row with context_lens[m] < 0 attends nothing: its
 * result is 0.  q and out dev [rows][n_heads][head_dim] float, 16-byte aligned, not overlapping.
 * Products and sums are float in effect; besides, a channel of q may be off by 2^-38 of the largest in its row and head, a probability times
 * the scale of its block of V by 2^-37 of the largest such product among the positions that the row attends.
 * batch->max_context sizes the launches: a bound near the longest context is quickest (up to 8192 where there are many rows and heads).
 * weights_out (dev [rows][n_kv_heads][weights_pitch] float, or NULL) receives the attention each cached position got, added
 * over the g heads that share it, for j <= p = context_lens[m]:
 *   weights_out[m][k][j] = weights_in[m][k][j] + sum_g probability   (j < p),   = sum_g probability   (j = p);
 * what lies behind is left as it was.  weights_in (same pitch) may be weights_out, or NULL for zeros.  Not with
 * row_table (EE_ERR_UNSUPPORTED).  weights_pitch >= max_context.
 * (weights_in and weights_out must not overlap in another way than being the same.)
 * A call has at most 65535 / ceil(g / 16) rows, with row_table 65535 * 32 / g.
 * workspace: ee_paged_attention_quant_bytes for the call's sizes or larger ones, 256-byte aligned; it needs no
 * initialisation and is dead between calls.  (Short contexts need none: NULL is refused only where something is needed.)
 * The bytes are 0 only for sizes that are refused (of rows: that the call refuses with row_table, or, with_weights, without). */
size_t ee_paged_attention_quant_bytes(const ee_quant_cache* cache, int32_t n_heads, int32_t max_batch, int32_t max_context,
                                      int32_t with_weights);
int ee_paged_attention_quant(const ee_quant_cache* cache, int32_t layer, int32_t n_heads, const float* q,
                             const ee_batch* batch, float* out, const float* weights_in, float* weights_out,
                             int32_t weights_pitch, void* workspace, size_t workspace_bytes, void* stream);

/* Shortens the cache of every sequence of the batch to `keep` (1 .. 262144, ceil(keep / 16) * n_kv_heads < 2^25) positions, for each K/V head by itself: the latest `recent`
 * (0 .. keep) positions stay, and of the others those with the largest weights_in (of equal ones the lowest position; NaN
 * counts as largest).  What stays moves together in its old order.  Here context_lens[b] is the NUMBER of cached
 * positions, at most max_context; row_table must be NULL; a sequence of `keep` positions or fewer keeps them all.
 * out_lens[b] = min(context_lens[b], keep) is the new number: the caller passes it on when every layer is done (it must not
 * be context_lens itself).
 *   dst_tables   dev [B][dst_max_blocks] or NULL.  NULL: the sequence's first blocks are written over (what lies behind
 *                out_lens[b] is free afterwards; no other sequence may share them).  Else the result goes to these blocks, which must not be among the
 *                blocks the batch's sequences are read from (for blocks that are shared, which must stay as they are).
 *   weights_in   dev [B][n_kv_heads][weights_pitch] float, weights_pitch >= max_context.
 *   weights_out  dev [B][n_kv_heads][weights_out_pitch] float or NULL, weights_out_pitch >= keep: the weights of what
 *                stays; may be weights_in (equal pitches; no other overlap).  Entries from out_lens[b] on are left as they were.
 *   kept         dev [B][n_kv_heads][keep] int32: the positions that stay, ascending, then -1.
 * A block that is written is built from its positions: its scale is the smallest that fits, and a position rounds
 * again (from the float its byte stood for) only where that scale differs from its old one.
 * workspace: ee_kv_quant_evict_bytes bytes, 256-byte aligned, without dst_tables; else unused. */
size_t ee_kv_quant_evict_bytes(const ee_quant_cache* cache, int32_t max_batch, int32_t keep);
int ee_kv_quant_evict(const ee_quant_cache* cache, int32_t layer, const ee_batch* batch, const int32_t* dst_tables,
                      int32_t dst_max_blocks, const float* weights_in, int32_t weights_pitch, float* weights_out,
                      int32_t weights_out_pitch, int32_t keep, int32_t recent, int32_t* kept, int32_t* out_lens,
                      void* workspace, size_t workspace_bytes, void* stream);

/* ---- Several continuations of a prompt ---------------------------------------------------------------------------
 * Beam search, parallel samples, many questions about one text: block tables whose sequences share blocks, kept by counts of
 * references on the device; the choice among beams; and an attention that reads what rows share once.  Same conventions as
 * above.  One step of a beam search over a cache:
 *   ee_beam_select -> ee_reorder_rows (what else belongs to a beam) -> ee_kv_pages_fork, releasing the old rows ->
 *   ee_kv_pages_grow -> ee_kv_copy -> ee_kv_pages_shared -> the layers, each with ee_paged_attention_shared.
 *
 * refs dev [num_blocks] int32: how many table entries name a block; 0 (or less) is a free block.  The tables of a call and its refs
 * belong together: an entry counts once for every row that names it within its length. */
typedef struct ee_page_tables {
  int32_t* block_tables; /* dev [rows][max_blocks]                                                        */
  int32_t* lens;         /* dev [rows]: cached positions (0 .. max_blocks * 16); the first ceil(lens / 16) entries of a row are
                            its blocks, what lies behind is never read                                     */
  int32_t rows, max_blocks; /* up to 2^20 and 2^23, together 2^30 entries                                    */
} ee_page_tables;

/* Scratch bytes of ee_kv_pages_grow and ee_kv_pages_compact for a pool of num_blocks (up to 2^23) and calls of up to max_rows rows.  256-byte
 * aligned, no initialisation, dead between calls; calls that may overlap need one each. */
size_t ee_kv_pages_bytes(int32_t num_blocks, int32_t max_rows);

/* Row m of dst becomes a copy of row parents[m] of src: its blocks (one more reference each) and its length.  parents dev [dst->rows]; where
 * it is no row of src, row m becomes empty.  What dst's rows held before is not given up (that is ee_kv_pages_release's).  Entries behind a row's blocks are left as they were.  release = 1: afterwards the rows of src give up theirs, as
 * by ee_kv_pages_release.  dst->max_blocks >= src->max_blocks; the tables must not overlap. */
int ee_kv_pages_fork(int32_t* refs, int32_t num_blocks, const ee_page_tables* src, const int32_t* parents, const ee_page_tables* dst,
                     int32_t release, void* stream);

/* Takes one reference from each block of every row, and sets the rows' lens to 0 (their entries stay as they are). */
int ee_kv_pages_release(int32_t* refs, int32_t num_blocks, const ee_page_tables* tables, void* stream);

/* Makes room for positions lens[m] .. new_lens[m] - 1 of every row (new_lens dev [rows], at most max_blocks * 16 count; a row with new_lens <= lens
 * wants nothing).  lens stay as they are: the caller sets them when the positions are cached.
 *   Blocks behind the row's are added.  A last block that is partly filled, and that other entries name too, is replaced by one of the row's own, and the
 *   row is given a move (old, new) for ee_kv_copy; where all its references are rows of this call that want to write it, the last of these rows keeps it.
 *   Free blocks are handed out in ascending order, to the rows in order and their entries in order.
 *   moves   dev [rows][2] int32: (old, new), or (-1, -1).
 *   missing dev [1] int32: 0, or how many blocks too few are free; then nothing has changed and every move is (-1, -1). */
int ee_kv_pages_grow(int32_t* refs, int32_t num_blocks, const ee_page_tables* tables, const int32_t* new_lens, int32_t* moves, int32_t* missing,
                     void* workspace, size_t workspace_bytes, void* stream);

/* Packs the n blocks in use into 0 .. n - 1: those from n on move, in ascending order, to the free ones below n, in ascending order.  refs and the tables
 * (NULL or rows == 0: none) follow.
 *   remap   dev [num_blocks] int32: the new place of every block in use, -1 for a free one (for tables that are kept elsewhere).
 *   moves   dev [num_blocks][2] int32: (old, new), then (-1, -1).     n_moves dev [1] int32.
 * The contents are the caller's to move: ee_kv_copy with these moves. */
int ee_kv_pages_compact(int32_t* refs, int32_t num_blocks, const ee_page_tables* tables, int32_t* remap, int32_t* moves, int32_t* n_moves,
                        void* workspace, size_t workspace_bytes, void* stream);

/* shared_blocks[g] = how many leading entries all rows first_row[g] .. first_row[g + 1] - 1 have in common, of those that every one of them has filled
 * (16 positions); 0 for a group without rows.  first_row dev [n_groups + 1] int32, shared_blocks dev [n_groups] int32. */
int ee_kv_pages_shared(const ee_page_tables* tables, const int32_t* first_row, int32_t n_groups, int32_t* shared_blocks, void* stream);

/* Copies blocks of every layer, K and V (and scales): moves dev [n][2] int32 (from, to), n up to 2^30; a pair with an entry outside 0 .. num_blocks - 1 is skipped.  count
 * dev [1] int32 or NULL: only the first *count of the n pairs.  No block may be written twice, or both read and written (but a pair of one block with itself
 * does nothing).  Pools start on 16 bytes. */
int ee_kv_copy(const ee_model_desc* desc, const ee_kv_cache* cache, const int32_t* moves, int32_t n, const int32_t* count, void* stream);
int ee_kv_quant_copy(const ee_quant_cache* cache, const int32_t* moves, int32_t n, const int32_t* count, void* stream);

/* One step of beam search.  Rows g * beams .. of the logits are group g's beams; candidate (row, t) has the score
 *   scores[row] + (logits[row][t] - log sum_t' exp(logits[row][t'])),
 * a row with finished[row] != 0 only the candidate (row, end_token) with scores[row] (its logits are not read).  A score that is not finite (a token masked by
 * -inf; any of a row with a NaN or +inf among its logits) counts as -inf.  For every group the n_out best, best first; of equal scores the lower
 * row, then the larger logit, then the lower token first.  Tokens and rows are given also where all that is left is -inf: by row and token alone, whatever the logits.  Scores are formed and compared in double, the sum's
 * exponentials in float; among one row's tokens the order is that of the logits.
 *   logits dev [groups * beams] rows of vocab values of `dtype` (EE_FP32 | EE_BF16), logits_stride (>= vocab) elements apart, any element alignment.
 *   scores dev [groups * beams] float.  finished dev [groups * beams] int32 or NULL (none).  end_token: 0 .. vocab - 1, or -1 (none; not with finished).
 *   tokens, parents (rows of the call), finished_out dev [groups][n_out] int32, scores_out float; finished_out (or NULL) is 1 where the row is finished or the token
 *   is end_token.  Results overlap neither each other nor the inputs.
 * beams and n_out are 1 .. 128, n_out <= beams * vocab.  workspace: 256-byte aligned, ee_beam_select_bytes for the call's
 * sizes or larger ones (0: refused sizes), no initialisation, dead between calls. */
size_t ee_beam_select_bytes(int32_t groups, int32_t beams, int32_t vocab, int32_t n_out);
int ee_beam_select(const void* logits, int64_t logits_stride, int32_t dtype, const float* scores, const int32_t* finished, int32_t groups, int32_t beams,
                   int32_t vocab, int32_t n_out, int32_t end_token, int32_t* tokens, int32_t* parents, float* scores_out, int32_t* finished_out,
                   void* workspace, size_t workspace_bytes, void* stream);

/* out[m] = in[parents[m]], rows of row_bytes bytes, in_stride and out_stride (>= row_bytes) bytes apart: whatever else belongs to a beam.  Where parents[m] is
 * none of 0 .. in_rows - 1 row m is left as it was.  in and out must not overlap. */
int ee_reorder_rows(const void* in, int64_t in_stride, int32_t in_rows, const int32_t* parents, int32_t rows, int64_t row_bytes, void* out,
                    int64_t out_stride, void* stream);

/* Rows whose sequences begin with the same blocks.  Groups are rows first_row[g] .. first_row[g + 1] - 1 of the batch (ascending); the first shared_blocks[g]
 * entries of their block tables are equal.  A group may have one row, or share nothing. */
typedef struct ee_prefix_groups {
  int32_t n_groups;             /* 0 .. 4096                                                                 */
  const int32_t* first_row;     /* dev [n_groups + 1] int32                                               */
  const int32_t* shared_blocks; /* dev [n_groups] int32                                                   */
  int32_t max_shared;           /* host-side upper bound of shared_blocks (more are not shared: read row by row) */
} ee_prefix_groups;

/* ee_paged_attention_decode for such rows, n_heads query heads over the desc->n_heads K/V heads of the cache (a multiple; g = n_heads / desc->n_heads):
 *   out[m][h] = softmax_j(q[m][h] . K[j][h / g] / sqrt(head_dim)) . V[j][h / g],   j = 0..context_lens[m] INCLUSIVE,
 * the same result as without groups; shared blocks are read once for up to 48 columns (a row and a query head; 32 of EE_FP32) instead of once a row.  A row shorter than its group's shared
 * blocks attends its own positions all the same; one with context_lens[m] < 0 attends nothing: its result is 0.  Rows of no group are left as they were.  row_table as in
 * ee_paged_attention_decode (shared blocks are then those of the rows' sequences).
 * q and out dev [rows][n_heads][head_dim] float, 16-byte aligned, not overlapping; pools start on 16 bytes.  Products and sums are float in effect; an infinite value
 * among the q, K or V that a row attends may make its result NaN.
 * workspace: 256-byte aligned, ee_paged_attention_shared_bytes for the call's sizes or larger ones, no initialisation, dead between calls. */
size_t ee_paged_attention_shared_bytes(const ee_model_desc* desc, int32_t n_heads, int32_t max_batch, int32_t max_groups, int32_t max_context);
int ee_paged_attention_shared(const ee_model_desc* desc, const ee_kv_cache* cache, int32_t layer, int32_t n_heads, const float* q, const ee_batch* batch,
                              const ee_prefix_groups* groups, float* out, void* workspace, size_t workspace_bytes, void* stream);

/* ---- Measurement helpers (not part of the decode path) ------------------------------------------------------
 * While enabled, every later ee_* call brackets the kernels it enqueues with pairs of HIP events on the call's
 * stream (the events add a few microseconds per kernel, so throughput is timed with profiling off).
 * ee_profile_read waits for the recorded events and returns, for up to max_records kernels in launch order,
 * the kernel class (EE_K_*), the 1-based layer it belongs to (0 = none) and its duration in milliseconds;
 * the records are then discarded.  Returns the number of records written, or a negative error code.
 * Launches that are made together have one record (attention with the merge of its parts, KV filling with its operand).
 * So has a launch that does the work of several kernels, under what it is named after: an exit decision or the start of an
 * iteration inside a QKV projection is part of EE_K_QKV; in small float models the exit head of a layer is part of the next
 * layer's EE_K_QKV, or of EE_K_KVFILL, and the exit decision and the output projection of EE_K_ATTN. */
#define EE_K_NORM 0     /* sum of squares + normalised projection input                         */
#define EE_K_QKV 1      /* QKV projection + rotary + cache write                                */
#define EE_K_ATTN 2     /* paged decode attention                                               */
#define EE_K_OPROJ 3    /* output projection + residual                                         */
#define EE_K_GATEUP 4   /* gate/up projection + SwiGLU                                          */
#define EE_K_DOWN 5     /* down projection + residual                                           */
#define EE_K_HEAD 6     /* exit head / LM head projection with softmax statistics               */
#define EE_K_COMBINE 7  /* exit decision, token selection and copy of the hidden states         */
#define EE_K_KVFILL 8   /* KV filling projection                                                */
#define EE_K_OTHER 9    /* state reset, embedding, rotary table, first normalisation            */
#define EE_K_CLASSES 10
/* Plain device copy of n_floats floats (dev to dev) with the library's own copy kernel: a kernel of known traffic
 * (4 * n_floats bytes read, as many written) against which hardware byte counters are calibrated. */
int ee_calibration_copy(const float* src, float* dst, size_t n_floats, void* stream);
/* Attainable-rate probes of the chip the benchmark runs on (what the fractions of the published peaks are set beside).
 * ee_calibration_read: a plain streaming read of `bytes` bytes (dev, 16-byte aligned) by `workgroups` workgroups of four
 *   wavefronts, each wavefront walking one contiguous piece with 16 KiB in flight; `sink` (dev, 16 bytes) is written only
 *   if the exclusive-or of a wavefront's words equals one fixed pattern.  Traffic: `bytes` read, nothing written.
 * ee_calibration_mfma: `workgroups` x 4 wavefronts each issue 4 * iterations 32x32x16 bf16 matrix instructions on
 *   registers (2 * 32 * 32 * 16 flop each), no memory traffic; `sink` (dev, 1 KiB) is never written.
 * ee_calibration_mfma_tile: the inner loop of a 128 x 128 wavefront tile alone: `workgroups` x 4 wavefronts (96 KiB of LDS
 *   each: one workgroup per compute unit) run `steps` (even, >= 2) contraction steps of 16 such instructions on 4 x 4
 *   accumulators; with `lds_fragment_reads` = 8 every step also reads the next step's 4 + 4 operand fragments (1 KiB
 *   each) from LDS, with 0 it reads none.  No global memory traffic in the loop; `sink` (dev, 1 KiB) is never written.
 *   Errors: EE_ERR_INVALID_ARG for a NULL sink, an odd or too small step count, another number of reads.
 * ee_calibration_intake: what a compute unit takes in when half of its loads come from beyond its L2: `workgroups` x 4
 *   wavefronts each read a piece of `own` (dev, own_bytes, read once: from HBM) in 1 KiB loads, alternating with 1 KiB
 *   loads from `common` (dev, a power of two >= 64 KiB of bytes that every workgroup walks alike, so its lines are in
 *   L2 after the first reader), `loads_in_flight` (8, 16, 32 or 48) per wavefront.  pairs = 0: every workgroup has a
 *   piece of `own` to itself; each workgroup takes in own_bytes / workgroups from `own` and as much from `common`.
 *   pairs = 1 (workgroups a multiple of 16): workgroups whose ids differ by 8 (one XCD, one L2) read the same piece, so
 *   every byte of `own` leaves HBM once and L2 twice: each takes in 2 * own_bytes / workgroups from `own` and as much from
 *   `common`.  `sink` (dev, 16 bytes) is practically never written. */
int ee_calibration_read(const void* src, size_t bytes, void* sink, int32_t workgroups, void* stream);
int ee_calibration_mfma(int32_t workgroups, int32_t iterations, float* sink, void* stream);
int ee_calibration_mfma_tile(int32_t workgroups, int32_t steps, int32_t lds_fragment_reads, float* sink, void* stream);
int ee_calibration_intake(const void* own, size_t own_bytes, const void* common, size_t common_bytes, int32_t workgroups,
                          int32_t loads_in_flight, int32_t pairs, void* sink, void* stream);
int ee_profile_enable(int32_t on);
int ee_profile_read(int32_t* kernel_class /*host*/, int32_t* layer /*host*/, float* ms /*host*/, int32_t max_records);

#ifdef __cplusplus
}
#endif
#endif /* EE_DECODE_H */
