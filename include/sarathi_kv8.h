/*
 * sarathi_kv8.h -- the KV cache in 8 bits: appending to it, attending over it
 * and reading it back, for hybrid and mixed batches (sarathi.h).
 *
 * The cache holds one byte per element and one fp32 scale for each `block`
 * consecutive positions of a slot, key/value head, and K or V; an element's
 * value is code * scale.  Half the bytes of a bf16 cache: twice the requests
 * fit (the decode batch of Sec. 4.3.1), and a decode's attention, which is
 * bound by reading the cache, has half as much to read.  Query heads may share
 * key/value heads, and the append normalises and rotates the heads of q and k
 * in the same pass.
 *
 * A batch is planned once (sarathi_kv8_plan_create) and its plan serves every
 * layer of the iteration.  Conventions of sarathi.h hold: pointers are
 * borrowed, device memory is the caller's, work is enqueued asynchronously on
 * the caller's stream (of the current device), errors are found on the host
 * before anything is enqueued, and the calls can be captured into HIP graphs.
 */
#ifndef SARATHI_KV8_H
#define SARATHI_KV8_H

#include "sarathi.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element formats. */
#define SARATHI_KV8_INT8  0   /* codes -127 .. 127; scale = largest magnitude / 127 */
#define SARATHI_KV8_E4M3  1   /* OCP e4m3 (4 exponent, 3 mantissa bits, largest 448); the scale is the
                                 smallest power of two not below largest magnitude / 448 */

/* Rotary pairs. */
#define SARATHI_ROPE_HALF         0   /* (i, i + rope_dim / 2) */
#define SARATHI_ROPE_INTERLEAVED  1   /* (2 i, 2 i + 1) */

/* Rotary frequencies theta_i = rope_base^(-2 i / rope_dim), scaled for contexts beyond the trained ones. */
#define SARATHI_ROPE_PLAIN   0   /* theta_i */
#define SARATHI_ROPE_LINEAR  1   /* theta_i / rope_factor */
#define SARATHI_ROPE_NTK     2   /* of the base rope_base * rope_factor^(r / (r - 2)), r = rope_dim */
#define SARATHI_ROPE_BANDS   3   /* theta_i (w + (1 - w) / rope_factor), w = clamp((n - rope_low) /
                                    (rope_high - rope_low), 0, 1), n = rope_orig_len * theta_i / (2 pi):
                                    pairs that turn often within the trained length are kept, slow ones divided */

/*
 * head_dim is 64 or 128, n_kv_heads divides n_heads (query head h attends to
 * key/value head h / (n_heads / n_kv_heads), at most 128 to one), block is 16,
 * 32, 64 or 128.  dtype is that of the rows (q, k, v in, q and o out).
 * softmax_scale 0 means 1 / sqrt(head_dim).  rope_dim (the leading dims that
 * are rotated; a multiple of 16, at most head_dim) 0 means no rotation, and
 * the other rope fields are then ignored; rope_factor is ignored by
 * ROPE_PLAIN, rope_low / rope_high / rope_orig_len by all but ROPE_BANDS.
 * cos and sin are multiplied by rope_mscale (0 means 1).
 */
typedef struct {
  int   n_heads;
  int   n_kv_heads;
  int   head_dim;
  int   n_layers;
  int   dtype;         /* SARATHI_F32 or SARATHI_BF16 */
  int   format;        /* SARATHI_KV8_* */
  int   block;         /* positions per scale */
  float softmax_scale;
  int   qk_norm;       /* 1: every q and k head x -> x / sqrt(mean(x^2) + qk_eps) * gain, before the rotation */
  float qk_eps;
  int   rope_dim;
  int   rope_layout;   /* SARATHI_ROPE_HALF or SARATHI_ROPE_INTERLEAVED */
  int   rope_scaling;  /* SARATHI_ROPE_PLAIN .. SARATHI_ROPE_BANDS */
  float rope_base;
  float rope_factor;
  float rope_low;
  float rope_high;
  int   rope_orig_len;
  float rope_mscale;
} sarathi_kv8_cfg;

/* ------------------------------------------------------------------ cache */
/*
 * Layout: codes [layer][slot][K=0 | V=1][kv head][pos][head_dim], one byte
 * each, pos < max_seq_len; then, at scale_offset bytes (a multiple of 256),
 * fp32 scales [layer][slot][K | V][kv head][block], ceil(max_seq_len / block)
 * blocks.
 */
typedef struct sarathi_kv8 sarathi_kv8;

size_t sarathi_kv8_bytes(const sarathi_kv8_cfg* cfg, int n_slots, int max_seq_len);
/* As sarathi_kv_alloc (same errors); the memory is not touched and needs no initial contents. */
int sarathi_kv8_alloc(const sarathi_kv8_cfg* cfg, int n_slots, int max_seq_len, void* dev_mem, size_t dev_bytes,
                      sarathi_kv8** out);
/* Free the host handle (plans made from it stay valid).  NULL is accepted. */
void sarathi_kv8_free(sarathi_kv8* kv);

/* Strides of the codes in bytes (layer, slot, K/V, head, pos), of the scales in floats (layer, slot, K/V,
 * head), and the byte offset of the scales. */
typedef struct {
  size_t layer, slot, kv, head, pos;
  size_t scale_layer, scale_slot, scale_kv, scale_head;
  size_t scale_offset;
} sarathi_kv8_layout;
int sarathi_kv8_get_layout(const sarathi_kv8* kv, sarathi_kv8_layout* out);

/* ------------------------------------------------------------------ batch plan */
/*
 * The plan of one batch: its metadata, rotary table and attention partials
 * live in the device memory `ws` (16-byte aligned, sarathi_kv8_plan_bytes or
 * more), which must stay in place and unshared while the plan is used: calls
 * with one plan, or with plans in the same memory, are ordered by their
 * stream, or race.  sarathi_kv8_plan_create checks the batch (errors as
 * sarathi_mixed_layer_forward) and enqueues the metadata's upload on
 * `hip_stream`; calls that use the plan come after it on that stream, or wait
 * for it.  sarathi_kv8_plan_free frees the host object at once (NULL is
 * accepted): enqueued or captured calls no longer need it, only the memory.
 */
typedef struct sarathi_kv8_plan sarathi_kv8_plan;

/* Enough for every batch of up to max_tokens rows in up to max_chunks prompt chunks. */
size_t sarathi_kv8_plan_bytes(const sarathi_kv8_cfg* cfg, int max_tokens, int max_chunks, int max_seq_len);
int sarathi_kv8_plan_create(const sarathi_kv8* kv, const sarathi_mixed_batch* batch, void* ws, size_t ws_bytes,
                            void* hip_stream, sarathi_kv8_plan** out);
void sarathi_kv8_plan_free(sarathi_kv8_plan* plan);

/* ------------------------------------------------------------------ operators */
/*
 * Append: rows qkv [T, ld_qkv] hold a token's n_heads query heads, then its
 * n_kv_heads key heads, then its value heads.  Every q and k head is
 * normalised (qk_norm; q_gain, k_gain: [head_dim] of dtype, shared by the
 * heads) and rotated by the row's position.  q goes to q_out [T, ld_q], which
 * may be qkv itself (ld_q == ld_qkv) and otherwise must not overlap it (here and
 * below, rows overlap where the memory from the first row's start to the last
 * one's end does: not even the rows' gaps are shared); k and
 * v go to the cache of `layer` at the row's (slot, position).  Strides are in
 * elements; rows must be 16-byte aligned.  Arithmetic in fp32; q is rounded
 * once to dtype, k and v once to their codes (nearest, ties to even).
 *
 * Scales: a block that the batch's rows reach gets the larger of its scale and
 * the one its new rows need; where that grows, the codes of its earlier
 * positions (those before the first new one) are rounded to the new scale,
 * exactly (save for the smallest) in e4m3, off by at most half a code in int8.
 * A block whose first position is written starts anew.  Scales below 2^-100
 * are zero, and so are the block's codes and values.  The cache holds finite
 * values: an infinity is stored as the largest code of its sign (zero where the
 * scale is zero), NaN as zero, and neither counts for the scale.  Nothing but
 * the new positions, those codes and the blocks' scales is written.
 * Errors: EINVAL (NULL, layer, alignment, gains missing, q_out overlapping),
 * EHIP.
 */
int sarathi_kv8_append(const sarathi_kv8_plan* plan, int layer, const void* qkv, size_t ld_qkv, const void* q_gain,
                       const void* k_gain, void* q_out, size_t ld_q, void* hip_stream);

/*
 * Attention: row r of q [T, ld_q] (n_heads heads), at (slot, position) of the
 * batch, attends to positions 0 .. its own of its slot in `layer`, all of which
 * must have been appended (its own included):
 *   out[r][h] = sum_j softmax_j(softmax_scale * q[r][h] . k_j) v_j.
 * Scores, softmax and sums in fp32; products on the matrix cores from the
 * codes, which are exact in bf16 and f16.  Chunks of bf16 rows multiply as they
 * are, with the probabilities (times the value scale) rounded to bf16; fp32 rows
 * and their probabilities go in as three bf16 terms each (24 bits).  Decodes of
 * bf16 rows multiply in f16: q by a power of two per head (its elements keep
 * their 8 bits down to 2^-28 of the head's largest), the probabilities (times
 * the value scale) with 11 bits, and dropped below 2^-32 of the largest.  Over
 * int8 codes a head of q with a magnitude beyond 2^111 gives NaN there, and sums
 * take the codes as code + 128, so their fp32 roundings are relative to 128
 * scales, not to the values; the 128 is taken out every 512 keys of a sum, which
 * bounds these roundings by 2^-10 of a code, whatever the number of keys.
 * The whole range of the cache's values is attended to: sums do not leave fp32's
 * range, and every key counts in the row sum whatever its value scale.  Value
 * scales below 2^-120 of the largest that a row sees count as that (or as zero).
 * out [T, ld_out] must not overlap q.
 * Errors: EINVAL (NULL, layer, alignment, overlap), EHIP.
 */
int sarathi_kv8_attention(const sarathi_kv8_plan* plan, int layer, const void* q, size_t ld_q, void* out,
                          size_t ld_out, void* hip_stream);

/*
 * Read: the values (code * scale, rounded to out_dtype) that `layer` holds at
 * the batch's rows' positions: k_out [T, ld_k] and v_out [T, ld_v], n_kv_heads
 * heads each (either may be NULL: not wanted).  A batch of one chunk (slot, 0,
 * n) reads a sequence's first n positions.
 * Errors: EINVAL (NULL plan, both outputs NULL, layer, alignment, overlap),
 * EUNSUPPORTED (out_dtype), EHIP.
 */
int sarathi_kv8_read(const sarathi_kv8_plan* plan, int layer, int out_dtype, void* k_out, size_t ld_k, void* v_out,
                     size_t ld_v, void* hip_stream);

/* ------------------------------------------------------------------ decoder layer */
/*
 * One decoder layer, and a stack of them, over a mixed batch with the 8-bit
 * cache: sarathi_mixed_layer_forward / sarathi_mixed_model_step (sarathi.h)
 * with its rotary embedding, append and attention replaced by the operators
 * above (the batch is planned once per call):
 *   a = norm_1(x); [q|k|v] = a W_qkv^T; append; o = attention;
 *   h = x + o W_o^T; m = act(norm_2(h) W_up^T); y = h + m W_down^T.
 * w_qkv is [(n_heads + 2 n_kv_heads) * head_dim, hidden]; q_gain, k_gain
 * [head_dim] are used with qk_norm.  cfg must agree with the cache's cfg in
 * n_heads, head_dim, n_layers, dtype, and in rope (rope_dim > 0) and rope_base.
 * Arguments, aliasing rules and errors otherwise as sarathi_mixed_layer_forward;
 * workspace: sarathi_kv8_workspace_bytes.  The intermediates that
 * sarathi_kv8_workspace_layout places hold the (last) layer's values after a
 * call (qkv: q normalised and rotated, k and v as projected).
 * sarathi_profile_begin / _end (sarathi.h) do not see these calls: they record
 * no stages of the 8-bit layer.
 */
typedef struct {
  sarathi_layer_weights base;
  const void* q_gain;
  const void* k_gain;
} sarathi_kv8_layer_weights;

size_t sarathi_kv8_workspace_bytes(const sarathi_model_cfg* cfg, const sarathi_kv8_cfg* kv_cfg, int max_tokens,
                                   int max_chunks, int max_seq_len);
int sarathi_kv8_workspace_layout(const sarathi_model_cfg* cfg, const sarathi_kv8_cfg* kv_cfg, int n_tokens,
                                 int n_chunks, int max_seq_len, sarathi_ws_layout* out);
int sarathi_kv8_layer_forward(const sarathi_model_cfg* cfg, const sarathi_kv8_layer_weights* w, const sarathi_kv8* kv,
                              int layer, const sarathi_mixed_batch* batch, const void* x_in, void* x_out, void* ws,
                              size_t ws_bytes, void* hip_stream);
int sarathi_kv8_model_step(const sarathi_model_cfg* cfg, const sarathi_kv8_layer_weights* w, const sarathi_kv8* kv,
                           const sarathi_mixed_batch* batch, const void* x_in, void* x_out, void* ws, size_t ws_bytes,
                           void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SARATHI_KV8_H */
