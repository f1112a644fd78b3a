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

// ... NaN where one is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
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
  w.tile = p.tiles - 1 - b % p.tiles;  // causal: the longest rows of keys of a key head first
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
// The pieces of work (work_of's) of each range of keys in falling order of their
// sequence's states, so that those which end last are short, and without those that
// have no rows. A lane has a sequence.
struct Order {
  int first, tiles, all;  // of a range: its first piece; query tiles with rows; all pieces
};
// For the whole warp; tiles_of(n): query tiles that n tokens of a sequence reach.
template <typename F>
__device__ __forceinline__ Order order_of(const CrossArgs &p, F tiles_of) {
  Order o = {};
  if (!p.sorted) return o;
  const int lane = threadIdx.x & 31;
  const bool on = lane < p.seqs;
  int klen = !on ? 0 : p.klen ? p.klen[lane] : p.keys;
  int qlen = !on ? 0 : p.qlen ? p.qlen[lane] : p.tokens;
  const bool first = threadIdx.x < 32;  // of every CTA that is launched
  if (klen < 0 || klen > p.keys) {
    if (first) set_err(p.err, HKV_ERR_BOUNDS);
    klen = 0;
  }
  if (qlen < 0 || qlen > p.tokens) {
    if (first) set_err(p.qerr, HKV_ERR_BOUNDS);
    qlen = 0;
  }
  o.tiles = tiles_of(qlen);
#pragma unroll 4
  for (int i = 0; i < p.seqs; ++i) {
    const int other = __shfl_sync(0xFFFFFFFFu, klen, i), tiles = __shfl_sync(0xFFFFFFFFu, o.tiles, i);
    o.all += tiles;
    if (other > klen || (other == klen && i < lane)) o.first += tiles;
  }
  o.first *= p.kv;
  o.all *= p.kv;
  return o;
}
// work_of's number of piece i, or -1
__device__ __forceinline__ int piece_at(const CrossArgs &p, const Order &o, int i) {
  if (!p.sorted) return i;
  const int per = p.tiles * p.kv * p.seqs, range = i / per;
  i -= range * per;
  if (i >= o.all) return -1;
  const int at = i - o.first;
  const int s = __ffs(__ballot_sync(0xFFFFFFFFu, at >= 0 && at < o.tiles * p.kv)) - 1;
  const int n = __shfl_sync(0xFFFFFFFFu, o.tiles, s), in = __shfl_sync(0xFFFFFFFFu, at, s);
  return range * per + (s * p.kv + in / n) * p.tiles + p.tiles - n + in % n;
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
