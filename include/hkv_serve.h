/*
 * hkv_serve.h — C-ABI of the serving cache: the ragged HeadKV cache of hkv.h
 * with its K/V rows held in 8 or 4 bits, and attention over a prompt that the
 * sequences of a batch share. Same library (libheadkv.so), same conventions
 * as hkv.h: device pointers, caller-owned memory, asynchronous on `stream`
 * (but hkv_quant_check), statuses, the error word, HKV_FAULT_INJECT.
 *
 * Row format. The D values of a K or V row are cut into groups of 32
 * neighbouring channels. With M = 127 (HKV_Q8) or 7 (HKV_Q4) and a the
 * largest magnitude of a group,
 *     s = bf16(a / M),   c_j = clamp(rint(x_j / s), -M, M),   x_j ~ s c_j,
 * a / M and x_j / s rounded to fp32 and rint to the nearest, ties to even; a
 * group of zeros (or one whose scale underflows) has s = 0, c = 0, and one
 * that holds an infinity or a NaN has s = NaN, c = 0 and reads back as NaN.
 * A code is stored biased: c + 128 in a byte (HKV_Q8); c + 8 in four bits,
 * channel 2j in the low and 2j + 1 in the high half of byte j (HKV_Q4).
 */
#ifndef HKV_SERVE_H
#define HKV_SERVE_H

#include "hkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* hkv_qcache.format: bits of a stored K/V value */
enum { HKV_Q8 = 8, HKV_Q4 = 4 };

/* the layer argument of hkv_quant_pack and hkv_quant_unpack for all layers */
enum { HKV_ALL_LAYERS = -1 };

/* flags of hkv_quant_pack */
enum {
  /* leave out the first n_cond rows of every head (the conditioning tokens,
   * which an hkv_cache keeps there) and count the positions of the others
   * from 0: for conditioning tokens that live in an hkv_prefix. The quantised
   * cache is then used with a config whose n_cond is 0. */
  HKV_PACK_SKIP_COND = 1
};

/*
 * A KV cache in 8 or 4 bits: an hkv_cache whose arena holds codes and scales.
 * All arrays but the following mean what they mean in hkv_cache.
 *  k, v      codes, [capacity_tokens][head_dim * format / 8] bytes
 *  ks, vs    scales, [capacity_tokens][head_dim / 32] bf16
 *  format    HKV_Q8 or HKV_Q4
 *  reserved  must be 0
 * Labels may be HKV_DENSE (an uncompressed cache), HKV_LOCAL or HKV_GLOBAL.
 * k, v, ks, vs and qbuf are 16-byte aligned.
 */
typedef struct {
  void *k;
  void *v;
  void *ks;
  void *vs;
  int32_t *pos;
  int64_t *off;
  int32_t *cap;
  int32_t *len;
  int32_t *nbuf;
  int32_t *ntok;
  uint8_t *label;
  void *qbuf;
  uint32_t *err;
  int64_t capacity_tokens;
  int32_t format;
  int32_t reserved;
} hkv_qcache;

/*
 * Prompts that sequences share, for one layer: n_groups prompts, the n_seqs
 * sequences of the config split into n_groups equal runs, run g attending
 * over prompt g. K/V in the config dtype; element (g, h, t, d) sits at
 *     g * group_stride + h * head_stride + t * token_stride + d.
 *  len       [n_groups] int32 (device): tokens of each prompt, 0 .. max_len
 *  max_len   host bound of len, > 0; rows up to max_len must be readable
 *  err       error word (a cache's), or NULL: a len outside 0 .. max_len sets
 *            HKV_ERR_BOUNDS there; the sequences of that prompt get NaN
 * k and v are 16-byte aligned and the strides (elements, positive, where the
 * axis is longer than 1) multiples of 16 bytes.
 */
typedef struct {
  const void *k;
  const void *v;
  const int32_t *len;
  uint32_t *err;
  int64_t group_stride, head_stride, token_stride;
  int32_t n_groups, max_len;
} hkv_prefix;

/* Quantises the live rows of every head of a layer (HKV_ALL_LAYERS: of all
 * layers) of a plain cache into the head's segment of the quantised one, in
 * storage order, and sets pos, len, nbuf and ntok there. off, cap and label
 * of dst are the caller's (they may be src's own arrays); dst->qbuf must be
 * src->qbuf. With HKV_PACK_SKIP_COND dst's pos and len must be other arrays
 * than src's (HKV_ERR_INVALID_ARG). A head that does not fit its segment, or
 * is longer than the config allows, sets HKV_ERR_CAPACITY, one outside an
 * arena HKV_ERR_BOUNDS, and with HKV_PACK_SKIP_COND one of fewer than n_cond
 * rows HKV_ERR_STATE in dst's error word; that head is left unchanged. */
hkv_status hkv_quant_pack(const hkv_config *cfg, const hkv_cache *src, const hkv_qcache *dst,
                          int layer, int flags, hkv_stream_t stream);

/* The way back: writes what every live row of src stands for, rounded to the
 * config dtype, into the head's segment of the plain cache dst (off, cap and
 * label the caller's), with pos, len, nbuf and ntok. dst->qbuf must be
 * src->qbuf. Errors as for hkv_quant_pack, in dst's error word. */
hkv_status hkv_quant_unpack(const hkv_config *cfg, const hkv_qcache *src, const hkv_cache *dst,
                            int layer, hkv_stream_t stream);

/* Bytes of device workspace hkv_quant_step and hkv_quant_attention need for
 * this config. Zero-fill it before the first use; every call leaves it ready
 * for the next. Calls that may overlap must not share it. Host only; 0 for a
 * bad config. */
size_t hkv_quant_workspace_size(const hkv_config *cfg);

/* Eq. 1 for one query per head of the layer over what the head's len live
 * rows stand for: out[s][h][:] = softmax(q k^T / sqrt(d)) V and lse[s][h] =
 * log(sum(exp(q k^T / sqrt(d)))), fp32, natural log; lse may be NULL.
 * prior_out, prior_lse: NULL, or the out and lse of the same queries over
 * other keys (hkv_prefix_attention); out and lse are then those over both
 * sets of keys. A head without keys yields zeros and -inf.
 * Nothing is rounded below fp32 but the products' operands, which are cut into
 * two fp16 parts over a power of two: q by groups of 32 channels, off by at
 * most 2^-22 of an element or 2^-50 of the group's largest, whichever is more;
 * the weights exp(x - the largest so far) times the rows' V scales by groups
 * and 32 rows, off by at most 2^-22 of a product or 2^-50 of the largest of
 * these scales. */
hkv_status hkv_quant_attention(const hkv_config *cfg, const hkv_qcache *cache, int layer,
                               const void *q, const float *prior_out, const float *prior_lse,
                               float *out, float *lse, void *workspace, size_t ws_bytes,
                               hkv_stream_t stream);

/* One decode step of one layer: k and v of the new token are quantised to the
 * row at len (pos = n_cond + ntok), q joins the Q_past ring, len and ntok
 * (and nbuf for compressed heads) advance by one, and out, lse are those of
 * hkv_quant_attention over the cache with that row. A compressed head whose
 * buffer already holds `period` tokens (hkv_quant_evict not run) sets
 * HKV_ERR_STATE, a full segment (or one longer than the config allows)
 * HKV_ERR_CAPACITY, one outside the arena HKV_ERR_BOUNDS in the error word;
 * that head's step is not taken and its outputs are not written.
 * flags: 0 or HKV_STEP_PREFETCH, with the meaning it has for hkv_decode_step
 * (true also when the previous kernel is hkv_prefix_attention). */
hkv_status hkv_quant_step(const hkv_config *cfg, const hkv_qcache *cache, int layer, const void *q,
                          const void *k, const void *v, const float *prior_out,
                          const float *prior_lse, float *out, float *lse, void *workspace,
                          size_t ws_bytes, int flags, hkv_stream_t stream);

/* The periodic head-aware update (hkv_evict) of a quantised cache, for one
 * layer or for every layer in one launch: the same rule, with Eq. 6's scores
 * taken from what the key rows stand for (s c in fp32, the sums in the same
 * fixed fp32 order); rows move with their scales. The i-th evicted row below
 * the new length, in storage order, takes the i-th surviving row above it.
 * The larger of period * head_dim * elem (elem of the config dtype) and 32 *
 * head_dim * format bytes, plus 16 bytes per token of the longest segment, 4 *
 * head_dim and 2544 bytes, must fit in 227 KB, else HKV_ERR_CAPACITY. */
hkv_status hkv_quant_evict(const hkv_config *cfg, const hkv_qcache *cache, int layer,
                           hkv_stream_t stream);
hkv_status hkv_quant_evict_all(const hkv_config *cfg, const hkv_qcache *cache, hkv_stream_t stream);

/* hkv_check for a quantised cache: synchronises the stream and returns the
 * status recorded in its error word. */
hkv_status hkv_quant_check(const hkv_qcache *cache, hkv_stream_t stream);

/* Bytes of device workspace hkv_prefix_attention needs (partial results; it
 * may hold anything). Calls that may overlap must not share it. Host only; 0
 * for bad arguments. */
size_t hkv_prefix_workspace_size(const hkv_config *cfg, const hkv_prefix *prefix);

/* Attention of one query per sequence and head over the sequence's shared
 * prompt, each prompt row read once for all its sequences: out[s][h][:] and
 * lse[s][h] as hkv_quant_attention defines them (both required), to be given
 * to hkv_quant_step or hkv_quant_attention as prior. A prompt of length 0
 * yields zeros and -inf. n_seqs not a multiple of n_groups, or strides that
 * are not multiples of 16 bytes -> HKV_ERR_SHAPE. An infinite or NaN element of
 * q, k or v shows in the outputs that its products enter, and in no others, as
 * a number that is not finite: NaN also where the definition gives an infinity
 * (the weights enter as parts, which may be zero). A group whose length is
 * negative or above max_len gets NaN, and HKV_ERR_BOUNDS in the error word;
 * so does one whose products did not finish within the kernel's limit of two
 * seconds, with HKV_ERR_TIMEOUT. */
hkv_status hkv_prefix_attention(const hkv_config *cfg, const hkv_prefix *prefix, const void *q,
                                float *out, float *lse, void *workspace, size_t ws_bytes,
                                hkv_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* HKV_SERVE_H */
