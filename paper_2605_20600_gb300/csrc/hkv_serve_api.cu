// Host side of the serving cache's C-ABI (include/hkv_serve.h): argument
// checks, workspace layouts and launches.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "hkv_host.h"
#include "hkv_quant.h"
#include "hkv_serve.h"

namespace {

using namespace hkv;

hkv_status check_qcache(const hkv_qcache *c) {
  if (!c || !c->k || !c->v || !c->ks || !c->vs || !c->pos || !c->off || !c->cap || !c->len ||
      !c->nbuf || !c->ntok || !c->label || !c->qbuf || !c->err)
    return HKV_ERR_INVALID_ARG;
  if ((c->format != HKV_Q8 && c->format != HKV_Q4) || c->reserved != 0) return HKV_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->ks) || !aligned16(c->vs) ||
      !aligned16(c->qbuf))
    return HKV_ERR_ALIGN;
  if (c->capacity_tokens <= 0) return HKV_ERR_CAPACITY;
  return HKV_OK;
}

QCacheArgs qcache_args(const hkv_qcache *c) {
  QCacheArgs a;
  a.c.K = c->k;
  a.c.V = c->v;
  a.c.pos = c->pos;
  a.c.off = c->off;
  a.c.cap = c->cap;
  a.c.len = c->len;
  a.c.nbuf = c->nbuf;
  a.c.ntok = c->ntok;
  a.c.label = c->label;
  a.c.qbuf = c->qbuf;
  a.c.err = c->err;
  a.c.arena_tokens = c->capacity_tokens;
  a.ks = c->ks;
  a.vs = c->vs;
  return a;
}

// heads [*first, *first + *count) of a layer, or of all layers
hkv_status layer_heads(const hkv_config *cfg, int layer, int *first, int *count) {
  const int hpl = heads_per_layer(cfg);
  if (layer == HKV_ALL_LAYERS) {
    *first = 0;
    *count = cfg->n_layers * hpl;  // at most 2^30 (hkv_validate_config)
    return HKV_OK;
  }
  if (layer < 0 || layer >= cfg->n_layers) return HKV_ERR_INVALID_ARG;
  *first = layer * hpl;
  *count = hpl;
  return HKV_OK;
}

// workspace of the attention: the heads' arrival counters, then partial results
size_t quant_counts_bytes(const hkv_config *c) {
  return align256((size_t)heads_per_layer(c) * sizeof(uint32_t));
}

size_t quant_ws_bytes(const hkv_config *c) {
  return quant_counts_bytes(c) +
         align256((size_t)kQuantMaxParts * (c->head_dim + 4) * sizeof(float));
}

// SMs of the current device, looked up once
hkv_status device_sms(int *sms) {
  static std::atomic<int> known[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return HKV_ERR_CUDA;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
      return HKV_ERR_CUDA;
    known[dev].store(n, std::memory_order_relaxed);
  }
  *sms = n;
  return HKV_OK;
}

hkv_status quant_attend(const char *name, const hkv_config *cfg, const hkv_qcache *cache,
                        int layer, const void *q, const void *k, const void *v, bool step,
                        const float *prior_out, const float *prior_lse, float *out, float *lse,
                        void *workspace, size_t ws_bytes, int flags, hkv_stream_t stream) {
  HKV_TRY(injected(name));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_qcache(cache));
  if (layer < 0 || layer >= cfg->n_layers) return HKV_ERR_INVALID_ARG;
  if (!q || !out || !workspace || (step && (!k || !v))) return HKV_ERR_INVALID_ARG;
  if ((prior_out == nullptr) != (prior_lse == nullptr)) return HKV_ERR_INVALID_ARG;
  if (flags & ~HKV_STEP_PREFETCH) return HKV_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) || !aligned16(prior_out) ||
      (step && (!aligned16(k) || !aligned16(v))))
    return HKV_ERR_ALIGN;
  if (ws_bytes < quant_ws_bytes(cfg)) return HKV_ERR_CAPACITY;
  QAttnArgs a = {};
  a.q8 = qcache_args(cache);
  a.nheads = heads_per_layer(cfg);
  a.base = layer * a.nheads;
  a.q = q;
  a.k_new = step ? k : nullptr;
  a.v_new = step ? v : nullptr;
  a.prior_out = prior_out;
  a.prior_lse = prior_lse;
  a.out = out;
  a.lse = lse;
  unsigned char *ws = static_cast<unsigned char *>(workspace);
  a.count = reinterpret_cast<uint32_t *>(ws);
  a.part = reinterpret_cast<float *>(ws + quant_counts_bytes(cfg));
  a.max_rows = max_segment(cfg);
  HKV_TRY(device_sms(&a.sms));
  a.P = cfg->period;
  a.C = cfg->n_cond;
  a.prefetch = (flags & HKV_STEP_PREFETCH) ? 1 : 0;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)cfg->head_dim));
  return cuda_status(
      launch_quant_attention(a, cfg->head_dim, cfg->dtype, cache->format, (cudaStream_t)stream));
}

// shared memory enabled for the update kernels, per device and kind
std::atomic<size_t> g_evict_smem[kMaxDevices][2][2][2];
std::mutex g_serve_mu;

hkv_status evict_ready(const hkv_config *cfg, int bits, size_t smem) {
  if (smem > kMaxUpdateSmem) return HKV_ERR_CAPACITY;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return HKV_ERR_CUDA;
  std::atomic<size_t> &have = g_evict_smem[dev][cfg->dtype == HKV_BF16][cfg->head_dim == 128]
                                          [bits == HKV_Q8];
  if (have.load(std::memory_order_acquire) < smem) {
    std::lock_guard<std::mutex> lk(g_serve_mu);
    if (have.load(std::memory_order_relaxed) < smem) {
      if (quant_evict_prepare(cfg->head_dim, cfg->dtype, bits, smem) != cudaSuccess)
        return HKV_ERR_CUDA;
      have.store(smem, std::memory_order_release);
    }
  }
  return HKV_OK;
}

hkv_status quant_evict(const char *name, const hkv_config *cfg, const hkv_qcache *cache, int layer,
                       hkv_stream_t stream) {
  HKV_TRY(injected(name));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_qcache(cache));
  int first, count;
  HKV_TRY(layer_heads(cfg, layer, &first, &count));
  const size_t smem = quant_evict_smem(max_segment(cfg), cfg->head_dim, cfg->period, cfg->dtype,
                                       cache->format);
  HKV_TRY(evict_ready(cfg, cache->format, smem));
  return cuda_status(launch_quant_evict(qcache_args(cache), method_args(cfg), first, count,
                                        cfg->head_dim, cfg->dtype, cache->format, smem,
                                        (cudaStream_t)stream));
}

hkv_status check_prefix(const hkv_config *cfg, const hkv_prefix *p) {
  if (!p || !p->k || !p->v || !p->len) return HKV_ERR_INVALID_ARG;
  if (p->n_groups <= 0 || p->max_len <= 0 || p->max_len > (1 << 24) ||
      cfg->n_seqs % p->n_groups != 0)
    return HKV_ERR_SHAPE;
  if (!aligned16(p->k) || !aligned16(p->v)) return HKV_ERR_ALIGN;
  const int64_t unit = cfg->dtype == HKV_BF16 ? 8 : 4;  // elements of 16 bytes
  const struct {
    int64_t stride;
    int n;
  } axes[3] = {{p->group_stride, p->n_groups}, {p->head_stride, cfg->n_heads},
               {p->token_stride, p->max_len}};
  for (const auto &a : axes)
    if (a.n > 1 && (a.stride <= 0 || a.stride % unit != 0)) return HKV_ERR_SHAPE;
  return HKV_OK;
}

PrefixPlan plan_of(const hkv_config *c, const hkv_prefix *p) {
  return prefix_plan(p->n_groups, c->n_seqs / p->n_groups, c->n_heads, p->max_len,
                     c->dtype);
}

size_t prefix_ws_bytes(const hkv_config *c, const PrefixPlan &pl) {
  const size_t parts = pl.splits > 1 ? (size_t)heads_per_layer(c) * pl.splits *
                                           (c->head_dim + 4) * sizeof(float)
                                     : 0;
  return align256(parts) + 256;
}

}  // namespace

extern "C" {

hkv_status hkv_quant_pack(const hkv_config *cfg, const hkv_cache *src, const hkv_qcache *dst,
                          int layer, int flags, hkv_stream_t stream) {
  HKV_TRY(injected("quant_pack"));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_cache(src));
  HKV_TRY(check_qcache(dst));
  if (flags & ~HKV_PACK_SKIP_COND) return HKV_ERR_INVALID_ARG;
  if (dst->qbuf != src->qbuf) return HKV_ERR_INVALID_ARG;
  int first, count;
  HKV_TRY(layer_heads(cfg, layer, &first, &count));
  const int skip = (flags & HKV_PACK_SKIP_COND) ? cfg->n_cond : 0;
  // a head's CTAs read src's while one of them writes dst's
  if (skip && (dst->len == src->len || dst->pos == src->pos)) return HKV_ERR_INVALID_ARG;
  return cuda_status(launch_quant_pack(cache_args(src), qcache_args(dst), first, count, skip,
                                       max_segment(cfg), cfg->head_dim, cfg->dtype, dst->format,
                                       (cudaStream_t)stream));
}

hkv_status hkv_quant_unpack(const hkv_config *cfg, const hkv_qcache *src, const hkv_cache *dst,
                            int layer, hkv_stream_t stream) {
  HKV_TRY(injected("quant_unpack"));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_qcache(src));
  HKV_TRY(check_cache(dst));
  if (dst->qbuf != src->qbuf) return HKV_ERR_INVALID_ARG;
  int first, count;
  HKV_TRY(layer_heads(cfg, layer, &first, &count));
  return cuda_status(launch_quant_unpack(qcache_args(src), cache_args(dst), first, count,
                                         max_segment(cfg), cfg->head_dim, cfg->dtype, src->format,
                                         (cudaStream_t)stream));
}

size_t hkv_quant_workspace_size(const hkv_config *cfg) {
  if (!cfg || hkv_validate_config(cfg) != HKV_OK) return 0;
  return quant_ws_bytes(cfg);
}

hkv_status hkv_quant_attention(const hkv_config *cfg, const hkv_qcache *cache, int layer,
                               const void *q, const float *prior_out, const float *prior_lse,
                               float *out, float *lse, void *workspace, size_t ws_bytes,
                               hkv_stream_t stream) {
  return quant_attend("quant_attention", cfg, cache, layer, q, nullptr, nullptr, false, prior_out,
                      prior_lse, out, lse, workspace, ws_bytes, 0, stream);
}

hkv_status hkv_quant_step(const hkv_config *cfg, const hkv_qcache *cache, int layer, const void *q,
                          const void *k, const void *v, const float *prior_out,
                          const float *prior_lse, float *out, float *lse, void *workspace,
                          size_t ws_bytes, int flags, hkv_stream_t stream) {
  return quant_attend("quant_step", cfg, cache, layer, q, k, v, true, prior_out, prior_lse, out,
                      lse, workspace, ws_bytes, flags, stream);
}

hkv_status hkv_quant_evict(const hkv_config *cfg, const hkv_qcache *cache, int layer,
                           hkv_stream_t stream) {
  if (layer == HKV_ALL_LAYERS) return HKV_ERR_INVALID_ARG;
  return quant_evict("quant_evict", cfg, cache, layer, stream);
}

hkv_status hkv_quant_evict_all(const hkv_config *cfg, const hkv_qcache *cache,
                               hkv_stream_t stream) {
  return quant_evict("quant_evict_all", cfg, cache, HKV_ALL_LAYERS, stream);
}

hkv_status hkv_quant_check(const hkv_qcache *cache, hkv_stream_t stream) {
  HKV_TRY(injected("quant_check"));
  if (!cache || !cache->err) return HKV_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  uint32_t word = 0;
  if (cudaMemcpyAsync(&word, cache->err, sizeof(word), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return HKV_ERR_CUDA;
  return (hkv_status)word;
}

size_t hkv_prefix_workspace_size(const hkv_config *cfg, const hkv_prefix *prefix) {
  if (!cfg || hkv_validate_config(cfg) != HKV_OK || check_prefix(cfg, prefix) != HKV_OK) return 0;
  return prefix_ws_bytes(cfg, plan_of(cfg, prefix));
}

hkv_status hkv_prefix_attention(const hkv_config *cfg, const hkv_prefix *prefix, const void *q,
                                float *out, float *lse, void *workspace, size_t ws_bytes,
                                hkv_stream_t stream) {
  HKV_TRY(injected("prefix_attention"));
  HKV_TRY(hkv_validate_config(cfg));
  HKV_TRY(check_prefix(cfg, prefix));
  if (!q || !out || !lse || !workspace) return HKV_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return HKV_ERR_ALIGN;
  const PrefixPlan pl = plan_of(cfg, prefix);
  if (ws_bytes < prefix_ws_bytes(cfg, pl)) return HKV_ERR_CAPACITY;
  PrefixArgs a = {};
  a.k = prefix->k;
  a.v = prefix->v;
  a.len = prefix->len;
  a.err = prefix->err;
  a.gs = prefix->n_groups > 1 ? prefix->group_stride : 0;
  a.hs = cfg->n_heads > 1 ? prefix->head_stride : 0;
  a.ts = prefix->max_len > 1 ? prefix->token_stride : 0;
  a.groups = prefix->n_groups;
  a.max_len = prefix->max_len;
  a.seqs = cfg->n_seqs / prefix->n_groups;
  a.heads = cfg->n_heads;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.part = static_cast<float *>(workspace);
  a.splits = pl.splits;
  a.tiles = pl.tiles;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)cfg->head_dim));
  return cuda_status(launch_prefix(a, pl, cfg->head_dim, cfg->dtype, (cudaStream_t)stream));
}

}  // extern "C"
