// The quantised cache outside its attention: rows written from a plain cache
// (pack), read back into one (unpack), and the periodic head-aware update.
#include <type_traits>

#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_select.cuh"

namespace hkv {
namespace {

// Pack and unpack: 8 values of K and V a thread, D / 8 threads a row; a group's
// maximum comes from its four lanes. DRAM bounds them: 512 heads of up to 1168
// rows of 128 bf16 channels go to 8 bits and back in 104 us (578 MB: 5.6 TB/s,
// 82 % of a copy). Pack computes more than half of the time, so it takes the
// threads of eight CTAs an SM over a second row in flight (five with two rows:
// 111 us), although bf16 rows then spill 20 bytes a thread at 32 registers;
// unpack waits more and keeps two. A CTA takes 64 rows, or 32 where the
// launch has few CTAs: 99 heads of up to 357 fp32 rows to 4 bits and back 13.7 us
// against 14.7 with 64 (the case above 115 with 32). fp32 rows, whose quotients
// are taken, keep the registers of five CTAs: 12.1 us for the 99 heads.
constexpr int kRowThreads = 256;
constexpr int kManyCtas = 1024;

int rows_of(int count, int max_len) {
  return (long long)count * ((max_len + 63) / 64) < kManyCtas ? 32 : 64;
}

__device__ __forceinline__ bool segment_ok(long long off, int cap, int len, long long arena) {
  return off >= 0 && cap >= 0 && off + cap <= arena && len >= 0 && len <= cap;
}

// One CTA: up to `rows` rows of one head. Block 0 of a head also sets
// its counters.
template <int D, typename T, int BITS>
__global__ void __launch_bounds__(kRowThreads, sizeof(T) == 2 ? 8 : 5)
    pack_kernel(const CacheArgs src, const QCacheArgs dst, int first, int blocks, int skip,
                int max_len, int rows) {
  using R = QRow<D, BITS>;
  constexpr int TPR = D / 8;  // threads per row
  // no early launch of the next kernel: a decode step that prefetches this
  // cache before its own wait must start after the rows are written
  pdl_wait();
  const int i = first + (int)(blockIdx.x / blocks), b = (int)(blockIdx.x % blocks);
  const int tid = threadIdx.x;
  const int len = src.len[i], scap = src.cap[i], dcap = dst.c.cap[i];
  const long long soff = src.off[i], doff = dst.c.off[i];
  const int n = len - skip;
  uint32_t bad = 0;
  if (!segment_ok(soff, scap, len, src.arena_tokens) ||
      !segment_ok(doff, dcap, 0, dst.c.arena_tokens))
    bad = HKV_ERR_BOUNDS;
  else if (n < 0)
    bad = HKV_ERR_STATE;
  else if (n > dcap || len > max_len)
    bad = HKV_ERR_CAPACITY;
  if (bad) {
    if (tid == 0 && b == 0) set_err(dst.c.err, bad);
    return;
  }
  if (b == 0 && tid == 0) {
    dst.c.len[i] = n;
    dst.c.nbuf[i] = src.nbuf[i];
    dst.c.ntok[i] = src.ntok[i];
  }
  const int r_end = min(n, (b + 1) * rows);
  const int col = tid % TPR;
  const uint32_t mask = 0xFu << (threadIdx.x & 28);  // the four lanes of a group
  constexpr int PCS = (int)sizeof(T) / 2;            // 16-byte pieces of 8 values
  for (int r = b * rows + tid / TPR; r < r_end; r += kRowThreads / TPR) {
    uint4 raw[2][PCS];
    const long long so = ((soff + skip + r) * (D / 8) + col) * PCS, dof = doff + r;
#pragma unroll
    for (int j = 0; j < PCS; ++j) {
      raw[0][j] = static_cast<const uint4 *>(src.K)[so + j];
      raw[1][j] = static_cast<const uint4 *>(src.V)[so + j];
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      float x[8];
#pragma unroll
      for (int j = 0; j < PCS; ++j) Elem<T>::unpack(raw[kv][j], x + j * Elem<T>::kPerPiece);
      uint32_t lo, hi;
      const uint32_t sb = quant_group<T, BITS>(x, mask, lo, hi);
      unsigned char *out = static_cast<unsigned char *>(kv ? dst.c.V : dst.c.K) + dof * R::kBytes;
      if (BITS == 8) reinterpret_cast<uint2 *>(out)[col] = make_uint2(lo, hi);
      else reinterpret_cast<uint32_t *>(out)[col] = lo;
      if ((col & 3) == 0)
        static_cast<uint16_t *>(kv ? dst.vs : dst.ks)[dof * R::kGroups + col / 4] = (uint16_t)sb;
    }
    if (col == 0) dst.c.pos[dof] = src.pos[soff + skip + r] - skip;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const float *x);
template <>
__device__ __forceinline__ void store8<float>(float *p, const float *x) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
template <>
__device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16 *p, const float *x) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
  *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(h);
}

template <int D, typename T, int BITS>
__global__ void __launch_bounds__(kRowThreads, 6)
    unpack_kernel(const QCacheArgs src, const CacheArgs dst, int first, int blocks, int max_len,
                  int rows) {
  using R = QRow<D, BITS>;
  constexpr int TPR = D / 8;
  pdl_wait();  // no early launch of the next kernel, as in pack_kernel
  const int i = first + (int)(blockIdx.x / blocks), b = (int)(blockIdx.x % blocks);
  const int tid = threadIdx.x;
  const int n = src.c.len[i], scap = src.c.cap[i], dcap = dst.cap[i];
  const long long soff = src.c.off[i], doff = dst.off[i];
  uint32_t bad = 0;
  if (!segment_ok(soff, scap, n, src.c.arena_tokens) ||
      !segment_ok(doff, dcap, 0, dst.arena_tokens))
    bad = HKV_ERR_BOUNDS;
  else if (n > dcap || n > max_len)
    bad = HKV_ERR_CAPACITY;
  if (bad) {
    if (tid == 0 && b == 0) set_err(dst.err, bad);
    return;
  }
  if (b == 0 && tid == 0) {
    dst.len[i] = n;
    dst.nbuf[i] = src.c.nbuf[i];
    dst.ntok[i] = src.c.ntok[i];
  }
  const int r_end = min(n, (b + 1) * rows);
  const int col = tid % TPR;
  constexpr int STEP = kRowThreads / TPR, U = 2;  // rows in flight a thread
  for (int r0 = b * rows + tid / TPR; r0 < r_end; r0 += U * STEP) {
    uint2 w[U][2];
    uint32_t sc[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + u * STEP < r_end) {
        const long long so = soff + r0 + u * STEP;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const unsigned char *row =
              static_cast<const unsigned char *>(kv ? src.c.V : src.c.K) + so * R::kBytes;
          w[u][kv].y = 0;
          if (BITS == 8) w[u][kv] = reinterpret_cast<const uint2 *>(row)[col];
          else w[u][kv].x = reinterpret_cast<const uint32_t *>(row)[col];
          sc[u][kv] = static_cast<const uint16_t *>(kv ? src.vs : src.ks)[so * R::kGroups + col / 4];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * STEP;
      if (r >= r_end) break;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const float s = bf16_bits_to_float(sc[u][kv]);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          x[j] = s * (lifted<BITS>(BITS == 4 || j < 4 ? w[u][kv].x : w[u][kv].y,
                                   BITS == 4 ? j : j & 3) - kLift<BITS>);
        store8<T>(static_cast<T *>(kv ? dst.V : dst.K) + (doff + r) * D + col * 8, x);
      }
      if (col == 0) dst.pos[doff + r] = src.c.pos[soff + r];
    }
  }
}

// Key rows as codes: the score of Eq. 6 takes what the row stands for, s c in
// fp32 (exact: 8 by 8 bits), in the channels' order with every product and
// sum rounded to fp32 by itself.
template <int D, int BITS>
struct CodeRows {
  static constexpr int kBytes = QRow<D, BITS>::kBytes, kStride = kBytes;
  static constexpr int G = QRow<D, BITS>::kGroups;
  const uint16_t *scale;  // the segment's first row
  // the row's scales, loaded while its codes are on their way
  using Ahead = typename std::conditional<G == 4, unsigned long long, uint32_t>::type;
  __device__ __forceinline__ Ahead ahead(int r) const {
    return reinterpret_cast<const Ahead *>(scale)[r];
  }
  __device__ __forceinline__ static int piece(int rr, int pc) { return piece_at<kBytes>(rr, pc); }
  // one group's part: HUGE where s 2^16 might overflow, else s c = s (2^15 + u) -
  // s (2^15 + bias) in one fma, exact: the second product has at most 21 bits
  template <bool HUGE>
  __device__ __forceinline__ float group(const unsigned char *stage, int rr, int g, const float *q,
                                         float sc, float s) const {
    const float minus = -sc * kLift<BITS>;
#pragma unroll
    for (int pc = 0; pc < BITS / 4; ++pc) {
      const uint4 u = *reinterpret_cast<const uint4 *>(stage + piece(rr, g * (BITS / 4) + pc));
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      constexpr int CPW = 32 / BITS;  // codes a word
#pragma unroll
      for (int j = 0; j < 4 * CPW; ++j) {
        const float f = lifted<BITS>(w[j / CPW], j % CPW);
        const float k = HUGE ? sc * (f - kLift<BITS>) : fmaf(sc, f, minus);
        s = __fadd_rn(s, __fmul_rn(q[pc * 4 * CPW + j], k));
      }
    }
    return s;
  }
  __device__ __forceinline__ float dot(const unsigned char *stage, int rr, const float *qbar,
                                       Ahead scales) const {
    float s = 0.f;
#pragma unroll 1
    for (int g = 0; g < G; ++g) {
      const float sc = bf16_bits_to_float((uint32_t)(scales >> (16 * g)) & 0xFFFFu);
      s = sc < 0x1p100f ? group<false>(stage, rr, g, qbar + g * 32, sc, s)
                        : group<true>(stage, rr, g, qbar + g * 32, sc, s);
    }
    return s;
  }
};

// The update: a CTA a head, the shared selection (select_evictions), then the
// moves. What bounds it is one head's chain: positions, the queries' sum, the
// scores (one lane a row, in a fixed order of 128 dependent sums), two radix
// selections, the moves, each with a trip to memory or a barrier in between.
// 1024 heads, half of them with 975 scored rows of 128 codes: 47 us, of which
// the bytes need 14; without the scored heads 19. So that as many chains as
// possible overlap, the work area is kept small: codes are staged as they are
// and without padding, which at up to 1233 rows leaves room for four CTAs an
// SM (three with padded rows: 3 us more).
constexpr int kQuantUpdCtasPerSm = 5;

template <int D, typename T, int BITS>
__global__ void __launch_bounds__(NT, kQuantUpdCtasPerSm)
    quant_evict_kernel(const QCacheArgs q, const MethodArgs m, int first, int max_len) {
  using R = QRow<D, BITS>;
  constexpr int KB = R::kBytes, SB = R::kScaleBytes, PPR = KB / 16;
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ UpdShared sh;
  // no early launch of the next kernel: a decode step that prefetches this
  // layer's cache before its own wait must start after the update is done
  pdl_wait();
  const CacheArgs &c = q.c;
  const int tid = threadIdx.x, i = first + blockIdx.x;
  const uint8_t lab = c.label[i];
  if (lab == HKV_DENSE || c.nbuf[i] < m.P) return;  // not due
  const int len = c.len[i], cp = c.cap[i], ntok = c.ntok[i];
  const long long off = c.off[i];
  if (!segment_ok(off, cp, len, c.arena_tokens)) {
    if (tid == 0) set_err(c.err, HKV_ERR_BOUNDS);
    return;
  }
  if (len > max_len) {
    if (tid == 0) set_err(c.err, HKV_ERR_CAPACITY);
    return;
  }
  unsigned char *K = static_cast<unsigned char *>(c.K) + off * KB;
  unsigned char *V = static_cast<unsigned char *>(c.V) + off * KB;
  unsigned char *KS = static_cast<unsigned char *>(q.ks) + off * SB;
  unsigned char *VS = static_cast<unsigned char *>(q.vs) + off * SB;
  int32_t *pos = c.pos + off;
  const unsigned char *ring =
      static_cast<const unsigned char *>(c.qbuf) + (size_t)i * m.P * D * sizeof(T);
  const UpdSmem u = carve(dyn, max_len, D, m.P, (int)sizeof(T), KB);
  SegRef sg{K, V, pos, K, V, pos, len, cp, true, c.err};
  const CodeRows<D, BITS> rows{reinterpret_cast<const uint16_t *>(KS)};
  const int M = select_evictions<D, T>(sg, lab, m, ring, ntok, u, sh, rows);
  if (M > 0) {
    int *hole, *fill;
    const int k = pair_holes(len, M, u, sh, &hole, &fill);
    // scales and positions ride with the first round of codes; every load of a
    // round is on its way before its first store (sources lie above the new
    // length, destinations below it)
    constexpr int B = 2, SW = SB / 4;
    uint32_t ks = 0, vs = 0;
    int ps = 0;
    if (tid < k * SW) {
      ks = *reinterpret_cast<const uint32_t *>(KS + (size_t)fill[tid / SW] * SB + tid % SW * 4);
      vs = *reinterpret_cast<const uint32_t *>(VS + (size_t)fill[tid / SW] * SB + tid % SW * 4);
    }
    if (tid < k) ps = u.ps[fill[tid]];
    for (int w0 = 0; w0 < k * PPR; w0 += NT * B) {
      uint4 kb[B], vb[B];
#pragma unroll
      for (int j = 0; j < B; ++j) {
        const int w = w0 + j * NT + tid;
        if (w < k * PPR) {
          const size_t src = (size_t)fill[w / PPR] * KB + (w % PPR) * 16;
          kb[j] = __ldcg(reinterpret_cast<const uint4 *>(K + src));
          vb[j] = __ldcg(reinterpret_cast<const uint4 *>(V + src));
        }
      }
#pragma unroll
      for (int j = 0; j < B; ++j) {
        const int w = w0 + j * NT + tid;
        if (w < k * PPR) {
          const size_t dst = (size_t)hole[w / PPR] * KB + (w % PPR) * 16;
          *reinterpret_cast<uint4 *>(K + dst) = kb[j];
          *reinterpret_cast<uint4 *>(V + dst) = vb[j];
        }
      }
    }
    if (tid < k * SW) {
      *reinterpret_cast<uint32_t *>(KS + (size_t)hole[tid / SW] * SB + tid % SW * 4) = ks;
      *reinterpret_cast<uint32_t *>(VS + (size_t)hole[tid / SW] * SB + tid % SW * 4) = vs;
    }
    if (tid < k) pos[hole[tid]] = ps;
    for (int w = tid + NT; w < k * SW; w += NT) {
      const size_t src = (size_t)fill[w / SW] * SB + w % SW * 4;
      const size_t dst = (size_t)hole[w / SW] * SB + w % SW * 4;
      *reinterpret_cast<uint32_t *>(KS + dst) = *reinterpret_cast<const uint32_t *>(KS + src);
      *reinterpret_cast<uint32_t *>(VS + dst) = *reinterpret_cast<const uint32_t *>(VS + src);
    }
    for (int j = tid + NT; j < k; j += NT) pos[hole[j]] = u.ps[fill[j]];
  }
  if (tid == 0 && M >= 0) {
    c.len[i] = len - M;
    c.nbuf[i] = 0;
  }
}

}  // namespace

#define HKV_QDISPATCH(D_, DT_, BITS_, ...)            \
  do {                                                \
    if ((BITS_) == HKV_Q8) {                          \
      constexpr int kBits = 8;                        \
      HKV_DISPATCH(D_, DT_, __VA_ARGS__);             \
    } else {                                          \
      constexpr int kBits = 4;                        \
      HKV_DISPATCH(D_, DT_, __VA_ARGS__);             \
    }                                                 \
  } while (0)

cudaError_t launch_quant_pack(const CacheArgs &src, const QCacheArgs &dst, int first, int count,
                              int skip, int max_len, int D, int dtype, int bits, cudaStream_t s) {
  const int rows = rows_of(count, max_len), blocks = (max_len + rows - 1) / rows;
  if ((long long)blocks * count > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  HKV_QDISPATCH(D, dtype, bits,
                return pdl_launch(pack_kernel<kD, kT, kBits>, blocks * count, kRowThreads, 0, s,
                                  src, dst, first, blocks, skip, max_len, rows));
  return cudaErrorInvalidValue;
}

cudaError_t launch_quant_unpack(const QCacheArgs &src, const CacheArgs &dst, int first, int count,
                                int max_len, int D, int dtype, int bits, cudaStream_t s) {
  const int rows = rows_of(count, max_len), blocks = (max_len + rows - 1) / rows;
  if ((long long)blocks * count > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  HKV_QDISPATCH(D, dtype, bits,
                return pdl_launch(unpack_kernel<kD, kT, kBits>, blocks * count, kRowThreads, 0, s,
                                  src, dst, first, blocks, max_len, rows));
  return cudaErrorInvalidValue;
}

size_t quant_evict_smem(int max_len, int D, int P, int dtype, int bits) {
  return update_smem_of(max_len, D, P, dtype == HKV_BF16 ? 2 : 4, D * bits / 8);
}

cudaError_t quant_evict_prepare(int D, int dtype, int bits, size_t smem) {
  HKV_QDISPATCH(D, dtype, bits, {
    cudaError_t e = cudaFuncSetAttribute(quant_evict_kernel<kD, kT, kBits>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(quant_evict_kernel<kD, kT, kBits>,
                               cudaFuncAttributePreferredSharedMemoryCarveout, 100);
    return e;
  });
  return cudaErrorInvalidValue;
}

cudaError_t launch_quant_evict(const QCacheArgs &c, const MethodArgs &m, int first, int count,
                               int D, int dtype, int bits, size_t smem, cudaStream_t s) {
  const int max_len = update_max_len(smem, D, m.P, dtype == HKV_BF16 ? 2 : 4, D * bits / 8);
  HKV_QDISPATCH(D, dtype, bits,
                return pdl_launch(quant_evict_kernel<kD, kT, kBits>, count, NT, smem, s, c, m,
                                  first, max_len));
  return cudaErrorInvalidValue;
}

}  // namespace hkv
