// Host-side pieces every C-ABI source shares: fault injection for tests,
// argument checks, and the launch arguments taken from the ABI's structs.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include "hkv.h"
#include "hkv_kernels.h"

namespace hkv {

constexpr int kMaxDevices = 64;
// dynamic shared memory of the update kernels: what a CTA may have, less theirs
constexpr size_t kMaxUpdateSmem = 227 * 1024 - kUpdateStatic;

inline hkv_status injected(const char *name) {
  const char *s = getenv("HKV_FAULT_INJECT");
  if (!s) return HKV_OK;
  const size_t n = strlen(name);
  if (strncmp(s, name, n) == 0 && s[n] == ':') return (hkv_status)atoi(s + n + 1);
  return HKV_OK;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline hkv_status cuda_status(cudaError_t e) { return e == cudaSuccess ? HKV_OK : HKV_ERR_CUDA; }

inline hkv_status check_cache(const hkv_cache *c) {
  if (!c || !c->k || !c->v || !c->pos || !c->off || !c->cap || !c->len || !c->nbuf || !c->ntok ||
      !c->label || !c->qbuf || !c->err)
    return HKV_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->qbuf)) return HKV_ERR_ALIGN;
  if (c->capacity_tokens <= 0) return HKV_ERR_CAPACITY;
  return HKV_OK;
}

inline CacheArgs cache_args(const hkv_cache *c) {
  CacheArgs a;
  a.K = c->k;
  a.V = c->v;
  a.pos = c->pos;
  a.off = c->off;
  a.cap = c->cap;
  a.len = c->len;
  a.nbuf = c->nbuf;
  a.ntok = c->ntok;
  a.label = c->label;
  a.qbuf = c->qbuf;
  a.err = c->err;
  a.arena_tokens = c->capacity_tokens;
  return a;
}

inline MethodArgs method_args(const hkv_config *cfg) {
  MethodArgs m;
  m.C = cfg->n_cond;
  m.w = cfg->recent_w;
  m.w_loc = cfg->local_w;
  m.P = cfg->period;
  m.r_s = cfg->r_s;
  m.tau = (float)cfg->tau;
  m.grid2d = cfg->distance_mode == HKV_DIST_GRID2D ? 1 : 0;
  m.row_len = cfg->row_len;
  return m;
}

inline int heads_per_layer(const hkv_config *c) { return c->n_seqs * c->n_heads; }

// the longest segment the config allows: the dense cache at grouping, or a
// global head's C + budget + P tokens (never more than C + N); a
// redistributed budget reaches B_g + (H - 1)(B_g - w) for a group of one
// global head
inline int max_segment(const hkv_config *c) {
  const int a = c->n_cond + c->group_at;
  long long bud = c->global_budget;
  if (c->budget_mode == HKV_BUDGET_REDISTRIBUTE)
    bud += (long long)(c->n_heads - 1) * (c->global_budget - c->recent_w);
  long long kept = bud + c->period;
  if (kept > c->n_image) kept = c->n_image;
  const int b = c->n_cond + (int)kept;
  return a > b ? a : b;
}

inline size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

#define HKV_TRY(x)                 \
  do {                             \
    hkv_status s_ = (x);           \
    if (s_ != HKV_OK) return s_;   \
  } while (0)

}  // namespace hkv
