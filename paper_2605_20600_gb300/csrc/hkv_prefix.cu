// Attention of a batch over prompts that its sequences share: every prompt
// row serves all sequences of its group.
//
// A CTA takes a tile of queries of one (group, head) and a range of the
// prompt's keys, one query per warp. Ranges of the same tile leave partial
// results in the workspace; the CTA that arrives last joins them in range
// order.
#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_select.cuh"

namespace hkv {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kThreads / 32;  // queries per CTA

constexpr float kLn2 = 0.6931471805599453f;

template <int D, typename T>
__global__ void __launch_bounds__(kThreads) prefix_kernel(const PrefixArgs p, int split_len) {
  constexpr int PF = D + 4, E = D / 32;
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int b = blockIdx.x;
  const int tile = b % p.tiles;
  b /= p.tiles;
  const int h = b % p.heads;
  b /= p.heads;
  const int g = b % p.groups, sp = b / p.groups;
  pdl_wait();
  pdl_launch_dependents();
  int len = p.len[g];
  const bool bad = len < 0 || len > p.max_len;
  if (bad) {
    if (p.err && tid == 0 && sp == 0) set_err(p.err, HKV_ERR_BOUNDS);
    len = 0;
  }
  const int sl = tile * kTile + warp;  // sequence within the group
  const bool on = sl < p.seqs;
  const size_t qi = ((size_t)g * p.seqs + sl) * p.heads + h;
  const int lo = sp * split_len, hi = min(len, lo + split_len);
  float q[E], acc[E];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  if (on) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      q[e] = (float)static_cast<const T *>(p.q)[qi * D + lane * E + e] * p.qscale;
    const T *K = static_cast<const T *>(p.k) + g * p.gs + h * p.hs + lane * E;
    const T *V = static_cast<const T *>(p.v) + g * p.gs + h * p.hs + lane * E;
    for (int t = lo; t < hi; ++t) {
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) x = fmaf(q[e], (float)K[t * p.ts + e], x);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
      const float mn = fmaxf(m, x);
      const float f = exp2f(m - mn), w = exp2f(x - mn);
      m = mn;
      l = l * f + w;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + w * (float)V[t * p.ts + e];
    }
  }
  if (p.splits > 1) {
    float *part = p.part + (qi * p.splits + sp) * PF;
    if (on) {
#pragma unroll
      for (int e = 0; e < E; ++e) part[lane * E + e] = acc[e];
      if (lane == 0) {
        part[D] = m;
        part[D + 1] = l;
      }
      __threadfence();
    }
    __syncthreads();
    uint32_t *count = p.count + ((size_t)g * p.heads + h) * p.tiles + tile;
    if (tid == 0) s_last = atomicAdd(count, 1u) == (uint32_t)p.splits - 1u;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    if (tid == 0) *count = 0u;
    if (on) {
      const float *first = p.part + qi * p.splits * PF;
      m = -INFINITY;
      for (int j = 0; j < p.splits; ++j) m = fmaxf(m, __ldcg(first + (size_t)j * PF + D));
      l = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = 0.f;
      for (int j = 0; j < p.splits; ++j) {
        const float lj = __ldcg(first + (size_t)j * PF + D + 1);
        if (lj == 0.f) continue;
        const float f = exp2f(__ldcg(first + (size_t)j * PF + D) - m);
        l += lj * f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += __ldcg(first + (size_t)j * PF + lane * E + e) * f;
      }
    }
  }
  if (!on) return;
#pragma unroll
  for (int e = 0; e < E; ++e)
    p.out[qi * D + lane * E + e] = bad ? NAN : l == 0.f ? 0.f : acc[e] / l;
  if (lane == 0) p.lse[qi] = bad ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

PrefixPlan prefix_plan(int groups, int seqs, int heads, int max_len, int D, int dtype) {
  (void)D;
  (void)dtype;
  PrefixPlan pl;
  pl.tiles = (seqs + kTile - 1) / kTile;
  const long long base = (long long)groups * heads * pl.tiles;
  long long want = (608 + base - 1) / base;  // about four CTAs an SM
  const long long most = (max_len + 63) / 64;
  if (want > most) want = most;
  if (want < 1) want = 1;
  pl.split_len = (int)((max_len + want - 1) / want);
  pl.splits = (max_len + pl.split_len - 1) / pl.split_len;
  return pl;
}

cudaError_t launch_prefix(const PrefixArgs &a, const PrefixPlan &pl, int D, int dtype,
                          cudaStream_t s) {
  const long long grid = (long long)a.groups * a.heads * pl.tiles * pl.splits;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  HKV_DISPATCH(D, dtype, return pdl_launch(prefix_kernel<kD, kT>, (int)grid, kThreads, 0, s, a,
                                           pl.split_len));
  return cudaErrorInvalidValue;
}

}  // namespace hkv
