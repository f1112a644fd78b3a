// What the kernels of attention over states share: which rows and keys a CTA
// works on, and how results are written.
#pragma once

#include "hkv_heads.h"
#include "hkv_mma.cuh"
#include "hkv_select.cuh"

namespace hkv {

constexpr float kLn2 = 0.6931471805599453f;

// Four neighbouring results to an output row.
__device__ __forceinline__ void store4(float *to, float4 v) { *reinterpret_cast<float4 *>(to) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *to, float4 v) {
  *reinterpret_cast<uint2 *>(to) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// what a CTA works on
struct Work {
  int s, kvh, tile, sp;   // sequence, key head, query tile, key range
  int qlen, klen;         // 0 where a length is out of range
  bool bad;               // the states' length is: NaN
};
__device__ __forceinline__ Work work_of(const CrossArgs &p, int b) {
  Work w;
  w.tile = p.tiles - 1 - b % p.tiles;  // causal: the longest rows of keys first
  b /= p.tiles;
  w.kvh = b % p.kv;
  b /= p.kv;
  w.s = b % p.seqs;
  w.sp = b / p.seqs;
  w.qlen = p.qlen ? p.qlen[w.s] : p.tokens;
  w.klen = p.klen ? p.klen[w.s] : p.keys;
  w.bad = w.klen < 0 || w.klen > p.keys;
  // (a lane of every warp: not all of them see every piece of work)
  const bool first = (threadIdx.x & 31) == 0 && w.tile == 0 && w.kvh == 0 && w.sp == 0;
  if (w.bad) {
    if (first) set_err(p.err, HKV_ERR_BOUNDS);
    w.klen = 0;
  }
  if (w.qlen < 0 || w.qlen > p.tokens) {
    if (first) set_err(p.qerr, HKV_ERR_BOUNDS);
    w.qlen = 0;
  }
  return w;
}
// a query row of a (sequence, key head): which head of the group, which token
struct Row {
  int head, token;
};
__device__ __forceinline__ Row row_of(const CrossArgs &p, int kvh, int r) {
  Row x;
  const int g = r / p.tokens;
  x.head = kvh * p.group + g;
  x.token = r - g * p.tokens;
  return x;
}
// keys that a query sees
__device__ __forceinline__ int keys_seen(const CrossArgs &p, const Work &w, int token) {
  if (token >= w.qlen) return 0;
  return p.causal ? max(0, min(w.klen, w.klen - w.qlen + token + 1)) : w.klen;
}
// keys that any of the rows [r0, r1) sees
__device__ __forceinline__ int keys_of_rows(const CrossArgs &p, const Work &w, int r0, int r1) {
  if (w.qlen == 0 || r0 >= r1) return 0;
  const int g0 = r0 / p.tokens, g1 = (r1 - 1) / p.tokens;
  const int first = r0 - g0 * p.tokens, last = g0 == g1 ? r1 - 1 - g1 * p.tokens : w.qlen - 1;
  if (g0 == g1 && first >= w.qlen) return 0;
  return keys_seen(p, w, min(last, w.qlen - 1));
}

// more than 16 query rows: bf16 in and out (plan.rows is 128 or 256), and fp32 outs
cudaError_t launch_cross_tc(const CrossArgs &a, const CrossPlan &plan, int D, cudaStream_t s);
cudaError_t launch_cross_parts(const CrossArgs &a, int D, int dtype, cudaStream_t s);

}  // namespace hkv
