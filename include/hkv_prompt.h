/*
 * hkv_prompt.h — C-ABI of what a model does to queries, keys and values before
 * and beside the cache of hkv.h: rotary positions, the norms of queries and
 * keys, and attention of many queries (or one) over the states of an encoder
 * or over a prompt's own tokens. Same library (libheadkv.so), same conventions
 * as hkv.h: device pointers, caller-owned memory, asynchronous on `stream`,
 * statuses, error words, HKV_FAULT_INJECT. Of the config these calls use
 * n_seqs, n_heads (the query heads), head_dim and dtype.
 *
 * Rotary positions. The first rot_dim channels of a head form rot_dim / 2
 * pairs; pair i of a token at position p turns by the angle t = p f_i:
 *     (x, y) -> A (x cos t - y sin t, x sin t + y cos t),
 * the other channels stay. With several axes every pair belongs to one of
 * them and turns by the token's position on it (row and column of an image
 * grid). An angle is taken modulo one turn in integers, f_i / 2 pi in units of
 * 2^-64: it is off by 2^-32 turns, and by 2^-51 of itself at any position up to
 * 2^31 - 1 (the rounding of f_i in 64 bits).
 */
#ifndef HKV_PROMPT_H
#define HKV_PROMPT_H

#include "hkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* which channels form pair i */
enum {
  HKV_ROPE_HALF = 0,  /* i and i + rot_dim / 2 */
  HKV_ROPE_PAIRS = 1  /* 2i and 2i + 1 (interleaved) */
};

/* how the frequencies f_i = base^(-2i / d) change for contexts longer than
 * the `original` one by `factor` s >= 1 */
enum {
  HKV_ROPE_PLAIN = 0,
  HKV_ROPE_LINEAR = 1, /* f / s */
  HKV_ROPE_BASE = 2,   /* base s^(d / (d - 2)) instead of base (d > 2) */
  HKV_ROPE_PARTS = 3   /* f (g + (1 - g) / s), g = (r - low) / (high - low)
                        * within 0 .. 1, r = original f / 2 pi turns: a ramp
                        * over turns, not over the pairs' numbers */
};

/* flags of hkv_rope_rotate */
enum {
  HKV_ROPE_BACK = 1 /* by -t: the way back (with A = 1), and the gradient */
};

/* flags of hkv_cross_attention */
enum {
  HKV_ATTN_CAUSAL = 1 /* the queries are the last tokens of the keys: of q
                       * queries over n keys query i sees the first i + n - q + 1 */
};

enum { HKV_NORM_RMS = 1, HKV_NORM_LAYER = 2 };

/*
 * What a rotation is made of (host).
 *  rot_dim    rotated channels, even, 2 .. head_dim
 *  n_axes     1 .. 3; section[a]: the pairs of axis a, > 0, in the order of the
 *             pairs; their sum is rot_dim / 2
 *  joint      0: i counts from 0 in every section and d = 2 section[a]; 1: i
 *             runs through all pairs and d = rot_dim
 *  amplitude  A
 * factor, original, low and high are used where the scaling names them;
 * original > 0, 0 <= low < high.
 */
typedef struct {
  int32_t head_dim, rot_dim, layout, n_axes;
  int32_t section[3];
  int32_t joint;
  int32_t scaling;
  int32_t reserved; /* must be 0 */
  double base, factor, original, low, high, amplitude;
} hkv_rope_params;

/* A rotation, made by hkv_make_rope: plain host data that calls copy.
 * turns[i] = f_i / 2 pi in units of 2^-64, modulo 1; a caller whose model has
 * other frequencies (a ramp over the pairs' numbers, a factor for each pair) makes
 * a plain rotation and fills turns itself. */
typedef struct {
  int32_t head_dim, rot_dim, layout, n_axes;
  int32_t section[3];
  float amplitude;
  uint64_t turns[64];
} hkv_rope;

/*
 * Rows of head_dim elements for the tokens and heads of a batch; element
 * (s, t, h, d) sits at s * seq_stride + t * token_stride + h * head_stride + d.
 * data is 16-byte aligned; the strides (elements) are multiples of 16 bytes and
 * at least head_dim where the axis is longer than 1.
 */
typedef struct {
  void *data;
  int64_t seq_stride, token_stride, head_stride;
  int32_t n_heads;
  int32_t dtype; /* HKV_FP32 or HKV_BF16 */
} hkv_rows;

/*
 * The tokens of a batch: n_tokens places for each of the config's n_seqs
 * sequences.
 *  len   [n_seqs] int32 (device), 0 .. n_tokens, or NULL: n_tokens each. Rows
 *        of places from len on are neither read nor written.
 *  pos   int32 (device) positions, for rotations: of token t of sequence s on
 *        axis a at a * pos_axis_stride + s * pos_seq_stride + t (a
 *        pos_seq_stride of 0: one row for all sequences); of either sign; those
 *        of places from len on are read too, and do not matter
 *  err   error word (a cache's), or NULL: a len outside its range sets
 *        HKV_ERR_BOUNDS there, and that sequence's outputs are left as they are
 */
typedef struct {
  int32_t n_tokens;
  int32_t reserved; /* must be 0 */
  const int32_t *len;
  const int32_t *pos;
  int64_t pos_axis_stride, pos_seq_stride;
  uint32_t *err;
} hkv_tokens;

/*
 * Norms of queries and keys over the head_dim channels of each head:
 *     HKV_NORM_RMS    x / sqrt(mean(x^2) + eps) * weight
 *     HKV_NORM_LAYER  (x - mean(x)) / sqrt(var(x) + eps) * weight + bias
 * weights and biases in the config dtype, [head_dim] (head stride 0) or one
 * row for each head (head stride in elements, a multiple of 16 bytes); NULL:
 * ones and zeros. eps >= 0.
 */
typedef struct {
  int32_t kind;
  float eps;
  const void *q_weight, *q_bias, *k_weight, *k_bias;
  int64_t q_head_stride, k_head_stride;
} hkv_norm;

/*
 * Keys and values of the sequences' states, in the config dtype, for
 * hkv_cross_attention; element (s, h, j, d) sits at
 *     s * seq_stride + h * head_stride + j * token_stride + d.
 *  len      [n_seqs] int32 (device): states of each sequence, 0 .. max_len, or
 *           NULL: max_len each. What lies in rows from len on does not matter.
 *  n_heads  key heads, a divisor of the config's n_heads; query head h reads
 *           key head h / (n_heads of the config / n_heads)
 *  err      error word, or NULL: a len outside 0 .. max_len sets
 *           HKV_ERR_BOUNDS there; that sequence's queries get NaN
 * Alignment and strides as for hkv_rows.
 */
typedef struct {
  const void *k;
  const void *v;
  const int32_t *len;
  uint32_t *err;
  int64_t seq_stride, head_stride, token_stride;
  int32_t n_heads, max_len;
} hkv_states;

/* Fills *rope from *params (both host). Bad values -> HKV_ERR_INVALID_ARG;
 * sizes that do not fit together -> HKV_ERR_SHAPE. Host only. */
hkv_status hkv_make_rope(const hkv_rope_params *params, hkv_rope *rope);

/* Rotates the rows of x into out (config dtype, the same heads). out may be x
 * with the same strides; any other overlap is not allowed. Computed in fp32
 * from the angles' cosines and sines, rounded once. */
hkv_status hkv_rope_rotate(const hkv_config *cfg, const hkv_rope *rope, const hkv_tokens *tokens,
                           const hkv_rows *x, const hkv_rows *out, int flags, hkv_stream_t stream);

/* What stands between a model's projection and the cache, in one pass: q and
 * k normed for each head (norm; NULL: not), then rotated (rope; NULL: not) into
 * q_out and k_out, v copied to v_out. Of (q, q_out), (k, k_out) and (v, v_out)
 * any but all may be NULL pairs; q has the config's n_heads, k and v may have
 * others. The rows may be slices of one fused projection; for hkv_decode_step
 * the outs are [n_seqs][n_heads][head_dim], for hkv_prefill k_out and v_out
 * [n_seqs][n_heads][n_cond][head_dim]. Computed in fp32, rounded once at the
 * end. An out may be its input with the same strides; any other overlap is not
 * allowed. */
hkv_status hkv_qk_norm_rope(const hkv_config *cfg, const hkv_norm *norm, const hkv_rope *rope,
                            const hkv_tokens *tokens, const hkv_rows *q, const hkv_rows *k,
                            const hkv_rows *v, const hkv_rows *q_out, const hkv_rows *k_out,
                            const hkv_rows *v_out, hkv_stream_t stream);

/* Bytes of device workspace hkv_cross_attention needs (partial results; it may
 * hold anything). Calls that may overlap must not share it. Host only; 0 for
 * bad arguments. */
size_t hkv_cross_workspace_size(const hkv_config *cfg, const hkv_states *states,
                                const hkv_tokens *tokens);

/* Attention of the tokens' queries over their sequence's states (or, with
 * HKV_ATTN_CAUSAL, of a prompt's tokens over the tokens up to themselves):
 *     out = softmax(q k^T / sqrt(d)) v,  lse = log(sum(exp(q k^T / sqrt(d)))).
 * q in the config dtype; out in the config dtype or, with bf16 queries, in
 * fp32; lse fp32 [n_seqs][n_heads][n_tokens], or NULL. A query that sees no key
 * gets zeros and -inf. Rows of places from tokens->len on are left as they
 * are. With one query per sequence, out in fp32 and lse are a prior of
 * hkv_quant_attention and hkv_quant_step.
 * Scores and sums are fp32. The weights exp(score - a reference) are fp32 in
 * lse; their products with v take them in three bf16 parts for fp32 outs, and
 * for bf16 outs in two, or, where a key head has more than 128 query rows in the
 * call (n_tokens times the query heads that read it), rounded to bf16: outs of a
 * prompt as a whole and in pieces may differ by 2^-9 of the weights.
 * A key whose score is -inf (an infinite element against one of the other sign,
 * products below fp32's range) weighs nothing, and a query that has no other keys
 * gets zeros and -inf. Any other infinite or NaN element of a query or of a state
 * that counts shows in the outputs that its products enter as a number that is not
 * finite (NaN also where the definition gives an infinity); with HKV_ATTN_CAUSAL one
 * of v may show in earlier queries too, whose weight of zero it meets. A key whose
 * products of finite elements lie above fp32's range shows so too, or weighs nothing.
 * What lies in rows from a length on shows nowhere. A sequence whose number of
 * states is out of range gets NaN, and HKV_ERR_BOUNDS in the states' error word;
 * queries whose products did not finish within the kernel's limit of two seconds get
 * NaN, with HKV_ERR_TIMEOUT. out must not overlap q or the states. */
hkv_status hkv_cross_attention(const hkv_config *cfg, const hkv_states *states,
                               const hkv_tokens *tokens, const hkv_rows *q, const hkv_rows *out,
                               float *lse, void *workspace, size_t ws_bytes, int flags,
                               hkv_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* HKV_PROMPT_H */
