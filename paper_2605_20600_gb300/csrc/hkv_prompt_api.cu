// Host side of include/hkv_prompt.h: argument checks, plans and launches.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "hkv_host.h"
#include "hkv_heads.h"

namespace {

using namespace hkv;

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int elem_size(int dtype) { return dtype == HKV_BF16 ? 2 : 4; }

// strides (elements) of the axes longer than 1: whole pieces of 16 bytes, rows apart
struct Axis {
  int64_t stride;
  int n;
};
template <int N>
bool strides_ok(const Axis (&axes)[N], int head_dim, int dtype) {
  const int64_t unit = 16 / elem_size(dtype);
  for (const Axis &a : axes)
    if (a.n > 1 && (a.stride < head_dim || a.stride % unit != 0 || a.stride >= (1ll << 38)))
      return false;
  return true;
}

hkv_status check_rows(const hkv_config *cfg, const hkv_rows *r, int tokens) {
  if (!r || !r->data) return HKV_ERR_INVALID_ARG;
  if (r->dtype != HKV_FP32 && r->dtype != HKV_BF16) return HKV_ERR_INVALID_ARG;
  if (r->n_heads <= 0 || r->n_heads > (1 << 20)) return HKV_ERR_SHAPE;
  if (!aligned16(r->data)) return HKV_ERR_ALIGN;
  const Axis axes[] = {{r->seq_stride, cfg->n_seqs}, {r->token_stride, tokens},
                       {r->head_stride, r->n_heads}};
  return strides_ok(axes, cfg->head_dim, r->dtype) ? HKV_OK : HKV_ERR_SHAPE;
}

hkv_status check_tokens(const hkv_config *cfg, const hkv_tokens *t) {
  if (!t || t->reserved != 0) return HKV_ERR_INVALID_ARG;
  if (t->n_tokens <= 0 || t->n_tokens > (1 << 24) ||
      (long long)cfg->n_seqs * t->n_tokens > (1ll << 30))
    return HKV_ERR_SHAPE;
  if (!aligned4(t->len) || !aligned4(t->pos) || !aligned4(t->err)) return HKV_ERR_ALIGN;
  return HKV_OK;
}

hkv_status check_rope(const hkv_config *cfg, const hkv_rope *r, const hkv_tokens *t) {
  if (!r || !t->pos) return HKV_ERR_INVALID_ARG;
  if (r->layout != HKV_ROPE_HALF && r->layout != HKV_ROPE_PAIRS) return HKV_ERR_INVALID_ARG;
  if (r->head_dim != cfg->head_dim || r->rot_dim < 2 || r->rot_dim > r->head_dim ||
      r->rot_dim % 2 != 0 || r->n_axes < 1 || r->n_axes > 3)
    return HKV_ERR_SHAPE;
  int sum = 0;
  for (int i = 0; i < r->n_axes; ++i) {
    if (r->section[i] <= 0 || r->section[i] > r->rot_dim / 2) return HKV_ERR_SHAPE;
    sum += r->section[i];
  }
  if (sum != r->rot_dim / 2) return HKV_ERR_SHAPE;
  if (!(fabsf(r->amplitude) <= 3.0e38f)) return HKV_ERR_INVALID_ARG;
  if (t->pos_seq_stride < 0 || (r->n_axes > 1 && t->pos_axis_stride < 0)) return HKV_ERR_SHAPE;
  return HKV_OK;
}

// one set of rows and where they go
hkv_status add_set(const hkv_config *cfg, const hkv_rows *in, const hkv_rows *out, int tokens,
                   HeadsArgs *a) {
  HKV_TRY(check_rows(cfg, in, tokens));
  HKV_TRY(check_rows(cfg, out, tokens));
  if (in->dtype != cfg->dtype || out->dtype != cfg->dtype || in->n_heads != out->n_heads)
    return HKV_ERR_SHAPE;
  const Axis x[] = {{in->seq_stride, cfg->n_seqs}, {in->token_stride, tokens},
                    {in->head_stride, in->n_heads}};
  const Axis y[] = {{out->seq_stride, cfg->n_seqs}, {out->token_stride, tokens},
                    {out->head_stride, out->n_heads}};
  if (in->data == out->data)  // in place: the same rows
    for (int i = 0; i < 3; ++i)
      if (x[i].n > 1 && x[i].stride != y[i].stride) return HKV_ERR_INVALID_ARG;
  HeadSet &s = a->set[a->sets++];
  s = HeadSet{};
  s.in = in->data;
  s.out = out->data;
  s.is = in->seq_stride, s.it = in->token_stride, s.ih = in->head_stride;
  s.os = out->seq_stride, s.ot = out->token_stride, s.oh = out->head_stride;
  s.heads = in->n_heads;
  a->heads += s.heads;
  return HKV_OK;
}

HeadsArgs heads_args(const hkv_config *cfg, const hkv_tokens *t, const hkv_rope *rope, bool back) {
  HeadsArgs a = {};
  a.seqs = cfg->n_seqs;
  a.tokens = t->n_tokens;
  a.len = t->len;
  a.pos = t->pos;
  a.pa = t->pos_axis_stride;
  a.ps = t->pos_seq_stride;
  a.err = t->err;
  if (rope) {
    a.rope = *rope;
    for (int i = rope->n_axes; i < 3; ++i) a.rope.section[i] = rope->rot_dim / 2;  // no pair reaches it
    a.sign = back ? -rope->amplitude : rope->amplitude;
  }
  return a;
}

hkv_status check_states(const hkv_config *cfg, const hkv_states *s) {
  if (!s || !s->k || !s->v) return HKV_ERR_INVALID_ARG;
  if (s->n_heads <= 0 || cfg->n_heads % s->n_heads != 0 || s->max_len <= 0 ||
      s->max_len > (1 << 24))
    return HKV_ERR_SHAPE;
  if (!aligned16(s->k) || !aligned16(s->v) || !aligned4(s->len) || !aligned4(s->err))
    return HKV_ERR_ALIGN;
  const Axis axes[] = {{s->seq_stride, cfg->n_seqs}, {s->head_stride, s->n_heads},
                       {s->token_stride, s->max_len}};
  return strides_ok(axes, cfg->head_dim, cfg->dtype) ? HKV_OK : HKV_ERR_SHAPE;
}

// queries of all sequences and heads that partial results and lse count
hkv_status check_queries(const hkv_config *cfg, const hkv_tokens *t) {
  HKV_TRY(check_tokens(cfg, t));
  return (long long)cfg->n_seqs * cfg->n_heads * t->n_tokens > (1ll << 30) ? HKV_ERR_SHAPE
                                                                           : HKV_OK;
}

CrossPlan plan_of(const hkv_config *c, const hkv_states *s, const hkv_tokens *t, int out_dtype) {
  return cross_plan(c->n_seqs, c->n_heads, s->n_heads, t->n_tokens, s->max_len, c->head_dim,
                    c->dtype, out_dtype);
}

}  // namespace

extern "C" {

hkv_status hkv_make_rope(const hkv_rope_params *p, hkv_rope *rope) {
  HKV_TRY(injected("make_rope"));
  if (!p || !rope || p->reserved != 0) return HKV_ERR_INVALID_ARG;
  if (p->layout != HKV_ROPE_HALF && p->layout != HKV_ROPE_PAIRS) return HKV_ERR_INVALID_ARG;
  if (p->scaling < HKV_ROPE_PLAIN || p->scaling > HKV_ROPE_PARTS || p->joint < 0 || p->joint > 1)
    return HKV_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return HKV_ERR_SHAPE;
  if (p->rot_dim < 2 || p->rot_dim > p->head_dim || p->rot_dim % 2 != 0 || p->n_axes < 1 ||
      p->n_axes > 3)
    return HKV_ERR_SHAPE;
  long long sum = 0;
  for (int a = 0; a < p->n_axes; ++a) {
    if (p->section[a] <= 0) return HKV_ERR_SHAPE;
    sum += p->section[a];
  }
  if (sum != p->rot_dim / 2) return HKV_ERR_SHAPE;
  if (!(p->base > 0.0 && p->base < 1e30)) return HKV_ERR_INVALID_ARG;
  if (!(fabs(p->amplitude) < 1e30)) return HKV_ERR_INVALID_ARG;
  const bool scaled = p->scaling != HKV_ROPE_PLAIN;
  if (scaled && !(p->factor >= 1.0 && p->factor < 1e30)) return HKV_ERR_INVALID_ARG;
  if (p->scaling == HKV_ROPE_PARTS &&
      (!(p->original > 0.0 && p->original < 1e30) || !(p->low >= 0.0 && p->low < p->high) ||
       !(p->high < 1e30)))
    return HKV_ERR_INVALID_ARG;
  hkv_rope made = {};
  made.head_dim = p->head_dim;
  made.rot_dim = p->rot_dim;
  made.layout = p->layout;
  made.n_axes = p->n_axes;
  made.amplitude = (float)p->amplitude;
  int pair = 0;
  for (int a = 0; a < p->n_axes; ++a) {
    made.section[a] = p->section[a];
    for (int i = 0; i < p->section[a]; ++i, ++pair) {
      const double d = p->joint ? p->rot_dim : 2.0 * p->section[a];
      double base = p->base;
      if (p->scaling == HKV_ROPE_BASE && d > 2.0) base *= pow(p->factor, d / (d - 2.0));
      double turns = pow(base, -2.0 * (p->joint ? pair : i) / d) / 6.283185307179586476925;
      if (p->scaling == HKV_ROPE_LINEAR) turns /= p->factor;
      if (p->scaling == HKV_ROPE_PARTS) {
        double g = (p->original * turns - p->low) / (p->high - p->low);
        g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
        turns *= g + (1.0 - g) / p->factor;
      }
      if (!(turns < HUGE_VAL)) return HKV_ERR_INVALID_ARG;  // of a base next to zero
      // a fraction of a turn below 1 - 2^-54, so that 2^64 times it fits
      made.turns[pair] = (uint64_t)ldexp(turns - floor(turns), 64);
    }
  }
  *rope = made;
  return HKV_OK;
}

hkv_status hkv_rope_rotate(const hkv_config *cfg, const hkv_rope *rope, const hkv_tokens *tokens,
                           const hkv_rows *x, const hkv_rows *out, int flags,
                           hkv_stream_t stream) {
  HKV_TRY(injected("rope_rotate"));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_tokens(cfg, tokens));
  HKV_TRY(check_rope(cfg, rope, tokens));
  if (flags & ~HKV_ROPE_BACK) return HKV_ERR_INVALID_ARG;
  HeadsArgs a = heads_args(cfg, tokens, rope, flags & HKV_ROPE_BACK);
  HKV_TRY(add_set(cfg, x, out, tokens->n_tokens, &a));
  a.set[0].rotate = 1;
  return cuda_status(launch_heads(a, cfg->head_dim, cfg->dtype, 0, (cudaStream_t)stream));
}

hkv_status hkv_qk_norm_rope(const hkv_config *cfg, const hkv_norm *norm, const hkv_rope *rope,
                            const hkv_tokens *tokens, const hkv_rows *q, const hkv_rows *k,
                            const hkv_rows *v, const hkv_rows *q_out, const hkv_rows *k_out,
                            const hkv_rows *v_out, hkv_stream_t stream) {
  HKV_TRY(injected("qk_norm_rope"));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_tokens(cfg, tokens));
  if (rope) HKV_TRY(check_rope(cfg, rope, tokens));
  if (!q && !k && !v) return HKV_ERR_INVALID_ARG;
  if (!q != !q_out || !k != !k_out || !v != !v_out) return HKV_ERR_INVALID_ARG;
  if (q && q->n_heads != cfg->n_heads) return HKV_ERR_SHAPE;
  int kind = 0;
  if (norm) {
    kind = norm->kind;
    if (kind != HKV_NORM_RMS && kind != HKV_NORM_LAYER) return HKV_ERR_INVALID_ARG;
    if (!(norm->eps >= 0.f && norm->eps <= 3.0e38f)) return HKV_ERR_INVALID_ARG;
    if (kind == HKV_NORM_RMS && (norm->q_bias || norm->k_bias)) return HKV_ERR_INVALID_ARG;
    if (!aligned16(norm->q_weight) || !aligned16(norm->q_bias) || !aligned16(norm->k_weight) ||
        !aligned16(norm->k_bias))
      return HKV_ERR_ALIGN;
    const int64_t unit = 16 / elem_size(cfg->dtype);
    for (const int64_t st : {norm->q_head_stride, norm->k_head_stride})
      if (st != 0 && (st < cfg->head_dim || st % unit != 0)) return HKV_ERR_SHAPE;
  }
  HeadsArgs a = heads_args(cfg, tokens, rope, false);
  a.eps = norm ? norm->eps : 0.f;
  const struct {
    const hkv_rows *in, *out;
    const void *weight, *bias;
    int64_t stride;
  } given[3] = {{q, q_out, norm ? norm->q_weight : nullptr, norm ? norm->q_bias : nullptr,
                 norm ? norm->q_head_stride : 0},
                {k, k_out, norm ? norm->k_weight : nullptr, norm ? norm->k_bias : nullptr,
                 norm ? norm->k_head_stride : 0},
                {v, v_out, nullptr, nullptr, 0}};
  for (int i = 0; i < 3; ++i) {
    if (!given[i].in) continue;
    HKV_TRY(add_set(cfg, given[i].in, given[i].out, tokens->n_tokens, &a));
    HeadSet &s = a.set[a.sets - 1];
    s.weight = given[i].weight;
    s.bias = given[i].bias;
    s.wh = given[i].stride;
    s.norm = norm && i < 2;
    s.rotate = rope && i < 2;
  }
  return cuda_status(launch_heads(a, cfg->head_dim, cfg->dtype, kind, (cudaStream_t)stream));
}

size_t hkv_cross_workspace_size(const hkv_config *cfg, const hkv_states *states,
                                const hkv_tokens *tokens) {
  if (!cfg || hkv_validate_config(cfg) != HKV_OK || check_states(cfg, states) != HKV_OK ||
      check_queries(cfg, tokens) != HKV_OK)
    return 0;
  size_t most = 0;
  for (const int out_dtype : {HKV_FP32, HKV_BF16}) {
    const size_t n = plan_of(cfg, states, tokens, out_dtype).part_bytes;
    if (n > most) most = n;
  }
  return align256(most) + 256;
}

hkv_status hkv_cross_attention(const hkv_config *cfg, const hkv_states *states,
                               const hkv_tokens *tokens, const hkv_rows *q, const hkv_rows *out,
                               float *lse, void *workspace, size_t ws_bytes, int flags,
                               hkv_stream_t stream) {
  HKV_TRY(injected("cross_attention"));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_states(cfg, states));
  HKV_TRY(check_queries(cfg, tokens));
  HKV_TRY(check_rows(cfg, q, tokens->n_tokens));
  HKV_TRY(check_rows(cfg, out, tokens->n_tokens));
  if (flags & ~HKV_ATTN_CAUSAL) return HKV_ERR_INVALID_ARG;
  if (q->n_heads != cfg->n_heads || out->n_heads != cfg->n_heads || q->dtype != cfg->dtype)
    return HKV_ERR_SHAPE;
  if (cfg->dtype == HKV_FP32 && out->dtype != HKV_FP32) return HKV_ERR_SHAPE;
  if (!workspace || out->data == q->data) return HKV_ERR_INVALID_ARG;
  if (!aligned16(workspace) || !aligned4(lse)) return HKV_ERR_ALIGN;
  const CrossPlan pl = plan_of(cfg, states, tokens, out->dtype);
  if (ws_bytes < pl.part_bytes) return HKV_ERR_CAPACITY;
  CrossArgs a = {};
  a.q = q->data;
  a.k = states->k;
  a.v = states->v;
  a.out = out->data;
  a.lse = lse;
  a.qlen = tokens->len;
  a.klen = states->len;
  a.err = states->err;
  a.qerr = tokens->err;
  a.qs = q->seq_stride, a.qt = q->token_stride, a.qh = q->head_stride;
  a.os = out->seq_stride, a.ot = out->token_stride, a.oh = out->head_stride;
  a.ks = states->seq_stride, a.kh = states->head_stride, a.kt = states->token_stride;
  a.seqs = cfg->n_seqs;
  a.heads = cfg->n_heads;
  a.kv = states->n_heads;
  a.group = a.heads / a.kv;
  a.tokens = tokens->n_tokens;
  a.keys = states->max_len;
  a.causal = (flags & HKV_ATTN_CAUSAL) ? 1 : 0;
  a.splits = pl.splits;
  a.split_len = pl.split_len;
  a.tiles = pl.tiles;
  a.box_tokens = pl.box_tokens;
  a.box_heads = pl.box_heads;
  a.sorted = pl.sorted && (a.klen || a.qlen);
  a.part = static_cast<float *>(workspace);
  a.qscale = (float)(1.4426950408889634 / sqrt((double)cfg->head_dim));
  return cuda_status(
      launch_cross(a, pl, cfg->head_dim, cfg->dtype, out->dtype, (cudaStream_t)stream));
}

}  // extern "C"
