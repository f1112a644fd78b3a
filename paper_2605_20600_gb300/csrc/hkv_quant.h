// Host-side launchers of the quantised-cache and shared-prompt kernels
// (internal to libheadkv.so).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "hkv_kernels.h"
#include "hkv_serve.h"

namespace hkv {

// a quantised cache: CacheArgs with code arenas in K and V, and the scales
struct QCacheArgs {
  CacheArgs c;
  void *ks, *vs;
};

// plain -> codes (pack) of heads [first, first + count): `skip` leading rows
// left out, segments of up to max_len rows
cudaError_t launch_quant_pack(const CacheArgs &src, const QCacheArgs &dst, int first, int count,
                              int skip, int max_len, int D, int dtype, int bits, cudaStream_t s);
cudaError_t launch_quant_unpack(const QCacheArgs &src, const CacheArgs &dst, int first, int count,
                                int max_len, int D, int dtype, int bits, cudaStream_t s);

// the periodic update; smem from quant_evict_smem (which, unlike that of a
// plain cache's update, goes by the rows' codes)
size_t quant_evict_smem(int max_len, int D, int P, int dtype, int bits);
cudaError_t quant_evict_prepare(int D, int dtype, int bits, size_t smem);
cudaError_t launch_quant_evict(const QCacheArgs &c, const MethodArgs &m, int first, int count,
                               int D, int dtype, int bits, size_t smem, cudaStream_t s);

// attention over the codes of one layer, with the append of the new token
// (k_new != nullptr) or without
struct QAttnArgs {
  QCacheArgs q8;               // full arrays
  int base, nheads;            // the layer's first flat head and its heads
  const void *q, *k_new, *v_new;          // [nheads][D]
  const float *prior_out, *prior_lse;     // [nheads][D], [nheads], or both null
  float *out, *lse;                       // [nheads][D], [nheads] or null
  uint32_t *count;             // [nheads] arrivals, zero between launches
  float *part;                 // [kQuantMaxParts][D + 4] partial results
  int max_rows;                // rows of the longest segment
  int sms, splits;             // of the device; CTAs of a head (the launcher's)
  int P, C, prefetch;
  float qscale;                // log2(e) / sqrt(D)
};

// most CTAs of the attention that share heads (the workspace holds a partial
// result of each)
constexpr int kQuantMaxParts = 2048;
cudaError_t launch_quant_attention(const QAttnArgs &a, int D, int dtype, int bits, cudaStream_t s);

// attention of a batch over shared prompts, one layer
struct PrefixArgs {
  const void *k, *v;
  const int32_t *len;          // [groups]
  uint32_t *err;
  long long gs, hs, ts;        // strides in elements
  int groups, max_len, seqs, heads;   // seqs per group
  const void *q;               // [groups * seqs][heads][D]
  float *out, *lse;
  float *part;                 // [groups * seqs * heads][splits][D + 4]
  int splits, tiles;           // key ranges, query tiles per (group, head)
  float qscale;
};

struct PrefixPlan {
  int mw;                        // queries of a CTA, over 16 (8: the tcgen05 kernel)
  int splits, tiles, split_len;  // key ranges, query tiles, keys of a range
};
PrefixPlan prefix_plan(int groups, int seqs, int heads, int max_len, int dtype);
cudaError_t launch_prefix(const PrefixArgs &a, const PrefixPlan &plan, int D, int dtype,
                          cudaStream_t s);

}  // namespace hkv
