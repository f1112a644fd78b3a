// Decode attention over a cache in 8 or 4 bits, with or without the append of
// the step's new token: one launch per layer.
//
// A CTA takes one chunk of one head's rows; its warps share the rows, each
// with its own running maximum, sum and accumulator, joined in shared memory.
// Heads of more than one chunk leave partial results (accumulator, maximum,
// sum) in the workspace; the CTA that arrives last at the head's counter joins
// them in chunk order (so the result does not depend on who is last), joins
// the prior, writes the outputs and, in a step, advances the head's counters.
// Every CTA of a head arrives, whether its chunk holds rows or not: each reads
// the head's length, which may change only after all have.
#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_select.cuh"

namespace hkv {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kChunk = 256;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// code c of channel d of a row, unbiased
template <int BITS>
__device__ __forceinline__ float code_at(const unsigned char *row, int d) {
  if (BITS == 8) return (float)((int)row[d] - 128);
  const int b = row[d >> 1];
  return (float)(((d & 1) ? b >> 4 : b & 15) - 8);
}

template <int D, typename T, int BITS, bool STEP>
__global__ void __launch_bounds__(kThreads) quant_attn_kernel(const QAttnArgs p) {
  using R = QRow<D, BITS>;
  constexpr int PF = D + 4;  // floats of a partial result
  __shared__ float s_acc[kWarps][D];
  __shared__ float s_m[kWarps], s_l[kWarps];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int hl = (int)(blockIdx.x % p.nheads), ch = (int)(blockIdx.x / p.nheads);
  const int i = p.base + hl;
  const CacheArgs &c = p.q8.c;
  if (!p.prefetch) pdl_wait();
  const int len = c.len[i], cap = c.cap[i];
  const long long off = c.off[i];
  const uint8_t lab = c.label[i];
  const int ntok = STEP ? c.ntok[i] : 0, nbuf = STEP ? c.nbuf[i] : 0;
  const int n = len + (STEP ? 1 : 0);
  uint32_t bad = 0;
  if (off < 0 || cap < 0 || off + cap > c.arena_tokens || len < 0 || len > cap)
    bad = HKV_ERR_BOUNDS;
  else if (STEP && lab != HKV_DENSE && nbuf >= p.P)
    bad = HKV_ERR_STATE;
  else if (n > cap || n > (long long)p.nchunks * kChunk)
    bad = HKV_ERR_CAPACITY;
  if (p.prefetch) pdl_wait();
  pdl_launch_dependents();
  if (bad) {  // the same for every CTA of the head
    if (ch == 0 && tid == 0) set_err(c.err, bad);
    return;
  }
  unsigned char *K = static_cast<unsigned char *>(c.K) + off * R::kBytes;
  unsigned char *V = static_cast<unsigned char *>(c.V) + off * R::kBytes;
  uint16_t *KS = static_cast<uint16_t *>(p.q8.ks) + off * R::kGroups;
  uint16_t *VS = static_cast<uint16_t *>(p.q8.vs) + off * R::kGroups;
  const int lo = ch * kChunk, hi = min(n, lo + kChunk);
  const bool active = ch == 0 || lo < n;

  if (STEP && active && len >= lo && len < hi) {  // this CTA holds the new row
    if (warp == 0 && lane < D / 4) {
      constexpr int TPR = D / 8;
      const int kv = lane / TPR, col = lane % TPR;
      float x[8];
      load8<T>(static_cast<const T *>(kv ? p.v_new : p.k_new) + (size_t)hl * D + col * 8, x);
      uint32_t a, b;
      const uint32_t sb = quant_group<BITS>(x, 0xFu << (lane & 28), a, b);
      unsigned char *row = (kv ? V : K) + (size_t)len * R::kBytes;
      if (BITS == 8) reinterpret_cast<uint2 *>(row)[col] = make_uint2(a, b);
      else reinterpret_cast<uint32_t *>(row)[col] = a;
      if ((col & 3) == 0) (kv ? VS : KS)[(size_t)len * R::kGroups + col / 4] = (uint16_t)sb;
    }
    for (int e = tid; e < D; e += kThreads)
      static_cast<T *>(c.qbuf)[((size_t)i * p.P + ntok % p.P) * D + e] =
          static_cast<const T *>(p.q)[(size_t)hl * D + e];
    if (tid == 0) c.pos[off + len] = p.C + ntok;
    __syncthreads();
  }

  if (active) {
    constexpr int E = D / 32;
    float q[E], acc[E];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[e] = (float)static_cast<const T *>(p.q)[(size_t)hl * D + lane * E + e] * p.qscale;
      acc[e] = 0.f;
    }
    const int g = lane * E / 32;
    for (int r = lo + warp; r < hi; r += kWarps) {
      const float sk = bf16_bits_to_float(KS[(size_t)r * R::kGroups + g]);
      const float sv = bf16_bits_to_float(VS[(size_t)r * R::kGroups + g]);
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e)
        x = fmaf(q[e], sk * code_at<BITS>(K + (size_t)r * R::kBytes, lane * E + e), x);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
      const float mn = fmaxf(m, x);
      const float f = exp2f(m - mn), w = exp2f(x - mn);
      m = mn;
      l = l * f + w;
#pragma unroll
      for (int e = 0; e < E; ++e)
        acc[e] = acc[e] * f + w * (sv * code_at<BITS>(V + (size_t)r * R::kBytes, lane * E + e));
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_acc[warp][lane * E + e] = acc[e];
    if (lane == 0) {
      s_m[warp] = m;
      s_l[warp] = l;
    }
  }
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc = 0.f;  // thread d < D: channel d
  if (active) {
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_m[w]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (s_l[w] == 0.f) continue;  // a warp without rows
      const float f = exp2f(s_m[w] - m);
      l += s_l[w] * f;
      if (tid < D) acc += s_acc[w][tid] * f;
    }
  }
  if (p.nchunks > 1) {
    float *part = p.part + ((size_t)hl * p.nchunks + ch) * PF;
    if (active) {
      if (tid < D) part[tid] = acc;
      if (tid == 0) {
        part[D] = m;
        part[D + 1] = l;
      }
      __threadfence();
    }
    __syncthreads();
    if (tid == 0) s_last = atomicAdd(p.count + hl, 1u) == (uint32_t)p.nchunks - 1u;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    const int np = n > 0 ? (n + kChunk - 1) / kChunk : 1;
    const float *first = p.part + (size_t)hl * p.nchunks * PF;
    m = -INFINITY;
    for (int j = 0; j < np; ++j) m = fmaxf(m, __ldcg(first + (size_t)j * PF + D));
    l = acc = 0.f;
    for (int j = 0; j < np; ++j) {
      const float lj = __ldcg(first + (size_t)j * PF + D + 1);
      if (lj == 0.f) continue;
      const float f = exp2f(__ldcg(first + (size_t)j * PF + D) - m);
      l += lj * f;
      if (tid < D) acc += __ldcg(first + (size_t)j * PF + tid) * f;
    }
    if (tid == 0) p.count[hl] = 0u;
  }
  // the prior: another set of keys with its own normalised output
  if (p.prior_lse) {
    const float pm = p.prior_lse[hl] * kLog2e;
    if (!(pm == -INFINITY)) {
      const float mn = fmaxf(m, pm);
      const float f = l == 0.f ? 0.f : exp2f(m - mn), w = exp2f(pm - mn);
      l = l * f + w;
      acc = acc * f;
      if (tid < D) acc += w * p.prior_out[(size_t)hl * D + tid];
      m = mn;
    }
  }
  if (tid < D) p.out[(size_t)hl * D + tid] = l == 0.f ? 0.f : acc / l;
  if (tid == 0) {
    if (p.lse) p.lse[hl] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    if (STEP) {
      c.len[i] = len + 1;
      c.ntok[i] = ntok + 1;
      if (lab != HKV_DENSE) c.nbuf[i] = nbuf + 1;
    }
  }
}

}  // namespace

int quant_chunks(int max_segment) { return (max_segment + kChunk - 1) / kChunk; }

cudaError_t launch_quant_attention(const QAttnArgs &a, int D, int dtype, int bits,
                                   cudaStream_t s) {
  const long long grid = (long long)a.nheads * a.nchunks;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
#define HKV_QATTN(BITS_, STEP_)                                                               \
  HKV_DISPATCH(D, dtype, return pdl_launch(quant_attn_kernel<kD, kT, BITS_, STEP_>, (int)grid, \
                                           kThreads, 0, s, a))
  if (bits == HKV_Q8) {
    if (a.k_new) HKV_QATTN(8, true);
    HKV_QATTN(8, false);
  }
  if (a.k_new) HKV_QATTN(4, true);
  HKV_QATTN(4, false);
#undef HKV_QATTN
  return cudaErrorInvalidValue;
}

}  // namespace hkv
