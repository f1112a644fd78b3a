// Decode attention over a cache in 8 or 4 bits, with or without the append of
// the step's new token: one launch per layer.
//
// A CTA takes one range of one head's rows; its warps share the range tile by
// tile (32 rows), each with its own running maximum, sum and accumulator,
// joined in shared memory at the end. Heads of more than one range leave
// partial results (accumulator, maximum, sum) in the workspace; the CTA that
// arrives last at the head's counter joins them in range order (so the result
// does not depend on who is last), joins the prior, writes the outputs and, in
// a step, advances the head's counters. Every CTA of a head arrives, whether
// its range holds rows or not: each reads the head's length, which may change
// only after all have.
//
// The products run on the tensor cores (mma.sync m16n8k16, fp16 operands, fp32
// sums), not because one query per head fills them (a sixteenth does) but
// because codes then need no conversion to fp32: a code is an exact fp16
// number two of which a bit operation and one packed subtraction make, and the
// eight columns carry what one query leaves empty:
//  * scores, 16 rows of K (M) x 16 channels (K): the columns hold the query cut
//    into two fp16 parts (hi, and the rest times 2^11: 22 bits), once per group
//    of 32 channels, zero outside the group. The sums of a row come out per
//    group, ready for the group's scale in fp32;
//  * output, 16 channels of V^T (M) x 16 rows (K): the columns hold the rows'
//    weights times the row's scale of each group, cut in two the same way,
//    after division by a power of two near the tile's largest scale of the
//    group; a channel uses its own group's two columns.
// Sums chain over at most 8 (scores) or 2 (output) products in the tensor core
// and are added in fp32 registers beyond that.
#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_select.cuh"

namespace hkv {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 32;    // rows a warp handles at a time

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLoScale = 2048.f, kLoUnscale = 1.f / 2048.f;  // second parts, 2^11

__device__ __forceinline__ uint32_t lop_and_or(uint32_t a, uint32_t m, uint32_t o) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(m), "r"(o));  // (a & m) | o
  return r;
}
__device__ __forceinline__ uint32_t h2_add(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}

// fp16 pairs from stored codes, exact. 0x64uu is the fp16 number 1024 + uu.
// codes8: bytes (0, 2) and (1, 3) of a word, less the bias of 128.
__device__ __forceinline__ void codes8(uint32_t w, uint32_t &even, uint32_t &odd) {
  constexpr uint32_t kOne = 0x64006400u, kSub = 0xE480E480u;  // 1024, -1152
  even = h2_add(lop_and_or(w, 0x00FF00FFu, kOne), kSub);
  odd = h2_add(__byte_perm(w, kOne | 0x00640064u, 0x4341), kSub);
}
// codes4: nibbles (0, 4), (1, 5), (2, 6), (3, 7) of a word, less the bias of
// 8; an odd nibble sits four bits up and reads as 1024 + 16 u
__device__ __forceinline__ void codes4(uint32_t w, uint32_t (&c)[4]) {
  constexpr uint32_t kOne = 0x64006400u, kSub = 0xE408E408u;       // -1032
  constexpr uint32_t kSix = 0x2C002C00u, kSubSix = 0xD480D480u;    // 1/16, -72
  const uint32_t v = w >> 8;
  c[0] = h2_add(lop_and_or(w, 0x000F000Fu, kOne), kSub);
  c[1] = h2_fma(lop_and_or(w, 0x00F000F0u, kOne), kSix, kSubSix);
  c[2] = h2_add(lop_and_or(v, 0x000F000Fu, kOne), kSub);
  c[3] = h2_fma(lop_and_or(v, 0x00F000F0u, kOne), kSix, kSubSix);
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int BYTES>
__device__ __forceinline__ void cp_async_small(void *dst, const void *src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(dst)), "l"(src), "n"(BYTES)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 2^e and 2^-e for the exponent e of a non-negative fp32 (its bits), e kept in
// [-126, 126]
__device__ __forceinline__ float pow2_of(uint32_t bits) {
  return __uint_as_float(min(max(bits & 0x7F800000u, 0x00800000u), 0x7E800000u));
}
__device__ __forceinline__ float inv_pow2(float p) {
  return __uint_as_float(0x7F000000u - __float_as_uint(p));
}

// Shared memory of a warp: STAGES tiles (codes of K and V, scales of K and
// V), the query's two parts, the weights' B operand.
template <int D, int BITS, int STAGES>
struct Smem {
  using R = QRow<D, BITS>;
  static constexpr int kCodes = kTile * R::kBytes, kScales = kTile * R::kScaleBytes;
  static constexpr int kStage = 2 * (kCodes + kScales);
  static constexpr int kQ = 2 * D * 2;        // fp16 [2][D]
  static constexpr int kW = 8 * kTile * 2;    // fp16 [8][kTile]
  static constexpr int kWarp = STAGES * kStage + kQ + kW;
  static constexpr int kTotal = kWarps * kWarp;
};

// Byte offset of the 16-byte piece `c` of row `r` in a tile: rows lie back to
// back, the pieces permuted so that the reads below spread over all banks.
template <int RB>
__device__ __forceinline__ int piece_at(int r, int c) {
  if (RB == 128) return r * 128 + ((c ^ (r & 7)) << 4);
  if (RB == 64) return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
  return r * 32 + ((c ^ ((r >> 2) & 1)) << 4);
}

// STAGES = 1: every warp has at most one tile (ranges of at most kThreads
// rows); more: it walks through its tiles, that many of them in flight.
template <int D, typename T, int BITS, bool STEP, int STAGES>
__global__ void __launch_bounds__(kThreads, STAGES == 1 ? 6 : 4)
    quant_attn_kernel(const QAttnArgs p) {
  using R = QRow<D, BITS>;
  using SM = Smem<D, BITS, STAGES>;
  constexpr int RB = R::kBytes, SB = R::kScaleBytes, G = R::kGroups;
  constexpr int PF = D + 4;          // floats of a partial result
  constexpr int KM = D / 16;         // products per 16 rows, scores and output alike
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ float s_acc[kWarps][D];
  __shared__ float s_m[kWarps], s_l[kWarps];
  __shared__ float s_factor[kThreads];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row8 = lane >> 2, quad = lane & 3;
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
  else if (n > cap || n > (long long)p.nchunks * p.chunk)
    bad = HKV_ERR_CAPACITY;
  if (bad) {  // the same for every CTA of the head
    pdl_wait();
    pdl_launch_dependents();
    if (ch == 0 && tid == 0) set_err(c.err, bad);
    return;
  }
  unsigned char *K = static_cast<unsigned char *>(c.K) + off * RB;
  unsigned char *V = static_cast<unsigned char *>(c.V) + off * RB;
  unsigned char *KS = static_cast<unsigned char *>(p.q8.ks) + off * SB;
  unsigned char *VS = static_cast<unsigned char *>(p.q8.vs) + off * SB;
  // the head's rows in equal ranges of whole tiles, one per CTA
  const int na = n > 0 ? (n + p.chunk - 1) / p.chunk : 1;
  const int per = n > 0 ? ((n + na - 1) / na + kTile - 1) / kTile * kTile : kTile;
  const int lo = ch * per, hi = min(n, lo + per);
  const bool active = ch == 0 || lo < n;
  unsigned char *ws = dyn + warp * SM::kWarp;

  // rows [r0, r0 + kTile) of the range into stage st: the old rows among them
  auto load_tile = [&](int r0, int st) {
    const int rows = min(kTile, min(hi, len) - r0);
    unsigned char *sk = ws + st * SM::kStage, *sv = sk + SM::kCodes;
    unsigned char *ss = sv + SM::kCodes;
#pragma unroll
    for (int e = lane; e < kTile * (RB / 16); e += 32) {
      const int r = e / (RB / 16), pc = e % (RB / 16);
      if (r < rows) {
        const size_t src = (size_t)(r0 + r) * RB + pc * 16;
        cp_async16(sk + piece_at<RB>(r, pc), K + src);
        cp_async16(sv + piece_at<RB>(r, pc), V + src);
      }
    }
    if (lane < rows) {
      cp_async_small<SB>(ss + lane * SB, KS + (size_t)(r0 + lane) * SB);
      cp_async_small<SB>(ss + SM::kScales + lane * SB, VS + (size_t)(r0 + lane) * SB);
    }
  };
  const int first = lo + warp * kTile;
#pragma unroll
  for (int st = 0; st < STAGES; ++st) {
    const int r0 = first + st * kWarps * kTile;
    if (r0 < hi) load_tile(r0, st);
    cp_async_commit();
  }
  if (p.prefetch) pdl_wait();  // the step's inputs are visible from here on
  pdl_launch_dependents();

  float m = -INFINITY, l = 0.f;
  float acc[KM][2];
#pragma unroll
  for (int x = 0; x < KM; ++x) acc[x][0] = acc[x][1] = 0.f;
  if (first < hi) {
    // the query over a power of two, in two fp16 parts, in the order in which
    // the codes of a word come out in pairs
    constexpr int E = D / 32;
    float qv[E];
    uint32_t qm = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      qv[e] = (float)static_cast<const T *>(p.q)[(size_t)hl * D + lane * E + e];
      qm = max(qm, __float_as_uint(qv[e]) & 0x7FFFFFFFu);
    }
    const float q2 = pow2_of(__reduce_max_sync(0xFFFFFFFFu, qm)), qi = inv_pow2(q2);
    const float xscale = q2 * p.qscale;
    __half *sq = reinterpret_cast<__half *>(ws + STAGES * SM::kStage);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int d = lane * E + e;
      const int at = BITS == 8 ? (d & ~3) + ((d & 1) << 1) + ((d >> 1) & 1)
                               : (d & ~7) + ((d & 3) << 1) + ((d >> 2) & 1);
      const float x = qv[e] * qi;
      const __half h = __float2half_rn(x);
      sq[at] = h;
      sq[D + at] = __float2half_rn((x - __half2float(h)) * kLoScale);
    }
    __syncwarp();
    // B operand of the scores: this lane's column is part (row8 & 1) of group
    // row8 / 2, its channels those of the lanes `quad` of the A operand
    uint32_t qf[KM][2];
    {
      const uint4 *src = reinterpret_cast<const uint4 *>(sq + (row8 & 1) * D + quad * (D / 4));
      const bool mine = (row8 >> 1) == quad * (D / 4) / 32;
#pragma unroll
      for (int x = 0; x < KM / 2; ++x) {
        const uint4 u = mine ? src[x] : make_uint4(0u, 0u, 0u, 0u);
        qf[2 * x][0] = u.x;
        qf[2 * x][1] = u.y;
        qf[2 * x + 1][0] = u.z;
        qf[2 * x + 1][1] = u.w;
      }
    }
    __half *sw = reinterpret_cast<__half *>(ws + STAGES * SM::kStage + SM::kQ);
    // where this lane's row (row8 + 8 quad) sits in the weights' columns
    const int own = row8 + 8 * quad;
    const int own_at = ((own >> 1) & 3) * 8 + (own >> 4) * 4 + ((own >> 3) & 1) * 2 + (own & 1);

    int st = 0;
    for (int r0 = first; r0 < hi; r0 += kWarps * kTile) {
      cp_async_wait<STAGES - 1>();
      __syncwarp();
      unsigned char *sk = ws + st * SM::kStage, *sv = sk + SM::kCodes;
      unsigned char *ss = sv + SM::kCodes;
      const int rows = min(kTile, hi - r0);
      if (STEP && len - r0 < kTile && len < hi && len >= r0) {
        // the new row: quantised into the arena and into the tile
        if (lane < D / 4) {
          constexpr int TPR = D / 8;
          const int kv = lane / TPR, col = lane % TPR, r = len - r0;
          float x[8];
          load8<T>(static_cast<const T *>(kv ? p.v_new : p.k_new) + (size_t)hl * D + col * 8, x);
          uint32_t a, b;
          const uint32_t sb = quant_group<BITS>(x, 0xFu << (lane & 28), a, b);
          unsigned char *row = (kv ? V : K) + (size_t)len * RB;
          unsigned char *tile = kv ? sv : sk;
          if (BITS == 8) {
            reinterpret_cast<uint2 *>(row)[col] = make_uint2(a, b);
            *reinterpret_cast<uint2 *>(tile + piece_at<RB>(r, col >> 1) + (col & 1) * 8) =
                make_uint2(a, b);
          } else {
            reinterpret_cast<uint32_t *>(row)[col] = a;
            *reinterpret_cast<uint32_t *>(tile + piece_at<RB>(r, col >> 2) + (col & 3) * 4) = a;
          }
          if ((col & 3) == 0) {
            reinterpret_cast<uint16_t *>((kv ? VS : KS) + (size_t)len * SB)[col / 4] = (uint16_t)sb;
            reinterpret_cast<uint16_t *>(ss + kv * SM::kScales + r * SB)[col / 4] = (uint16_t)sb;
          }
        }
        __syncwarp();
      }

      // scores: x[b2] is the sum of row row8 + 8 b2 over this lane's group
      float xs[4];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int ra = b * 16 + row8, rb = ra + 8;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t wa[RB / 16], wb[RB / 16];  // this lane's quarter of the two rows
        if (RB == 128) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 ua = *reinterpret_cast<const uint4 *>(sk + piece_at<RB>(ra, 2 * quad + h));
            const uint4 ub = *reinterpret_cast<const uint4 *>(sk + piece_at<RB>(rb, 2 * quad + h));
            wa[h * 4] = ua.x, wa[h * 4 + 1] = ua.y, wa[h * 4 + 2] = ua.z, wa[h * 4 + 3] = ua.w;
            wb[h * 4] = ub.x, wb[h * 4 + 1] = ub.y, wb[h * 4 + 2] = ub.z, wb[h * 4 + 3] = ub.w;
          }
        } else if (RB == 64) {
          const uint4 ua = *reinterpret_cast<const uint4 *>(sk + piece_at<RB>(ra, quad));
          const uint4 ub = *reinterpret_cast<const uint4 *>(sk + piece_at<RB>(rb, quad));
          wa[0] = ua.x, wa[1] = ua.y, wa[2] = ua.z, wa[3] = ua.w;
          wb[0] = ub.x, wb[1] = ub.y, wb[2] = ub.z, wb[3] = ub.w;
        } else {
          const uint2 ua = *reinterpret_cast<const uint2 *>(sk + piece_at<RB>(ra, quad >> 1) +
                                                            (quad & 1) * 8);
          const uint2 ub = *reinterpret_cast<const uint2 *>(sk + piece_at<RB>(rb, quad >> 1) +
                                                            (quad & 1) * 8);
          wa[0] = ua.x, wa[1] = ua.y;
          wb[0] = ub.x, wb[1] = ub.y;
        }
#pragma unroll
        for (int w = 0; w < RB / 16; ++w) {
          if (BITS == 8) {
            uint32_t a0, a1, a2, a3;
            codes8(wa[w], a0, a2);
            codes8(wb[w], a1, a3);
            mma_f16(s, a0, a1, a2, a3, qf[w][0], qf[w][1]);
          } else {
            uint32_t ca[4], cb[4];
            codes4(wa[w], ca);
            codes4(wb[w], cb);
            mma_f16(s, ca[0], cb[0], ca[1], cb[1], qf[2 * w][0], qf[2 * w][1]);
            mma_f16(s, ca[2], cb[2], ca[3], cb[3], qf[2 * w + 1][0], qf[2 * w + 1][1]);
          }
        }
        const uint16_t *sc = reinterpret_cast<const uint16_t *>(ss);
        const bool grp = quad < G;  // the columns beyond the groups are empty
        const float fa = grp ? bf16_bits_to_float(sc[ra * G + (grp ? quad : 0)]) : 0.f;
        const float fb = grp ? bf16_bits_to_float(sc[rb * G + (grp ? quad : 0)]) : 0.f;
        xs[2 * b] = fa * fmaf(s[1], kLoUnscale, s[0]);
        xs[2 * b + 1] = fb * fmaf(s[3], kLoUnscale, s[2]);
      }
      // sums over the groups: lane (row8, quad) ends up with row row8 + 8 quad
      const bool b0 = quad & 1, b1 = quad & 2;
      float k0 = (b0 ? xs[1] : xs[0]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? xs[0] : xs[1], 1);
      float k1 = (b0 ? xs[3] : xs[2]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? xs[2] : xs[3], 1);
      float x = (b1 ? k1 : k0) + __shfl_xor_sync(0xFFFFFFFFu, b1 ? k0 : k1, 2);
      const bool on = own < rows;
      x = on ? x * xscale : -INFINITY;

      float mt = x;
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xFFFFFFFFu, mt, o));
      if (STAGES == 1) {
        m = mt;
      } else if (mt > m) {  // the same for the whole warp
        const float f = ex2_approx(m - mt);
        m = mt;
        l *= f;
#pragma unroll
        for (int y = 0; y < KM; ++y) {
          acc[y][0] *= f;
          acc[y][1] *= f;
        }
      }
      const float w = on ? ex2_approx(x - m) : 0.f;
      l += w;

      // weights times scales, over the power of two of the tile's largest
      // scale of the group, in two parts
      float unit = 1.f;  // of group `quad`
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint32_t sb =
            on ? reinterpret_cast<const uint16_t *>(ss + SM::kScales)[own * G + g] : 0u;
        const float u = pow2_of(__reduce_max_sync(0xFFFFFFFFu, sb << 16));
        if (quad == g) unit = u;
        const float y = on ? w * (bf16_bits_to_float(sb) * inv_pow2(u)) : 0.f;
        const __half h = __float2half_rn(y);
        sw[(2 * g) * kTile + own_at] = h;
        sw[(2 * g + 1) * kTile + own_at] = __float2half_rn((y - __half2float(h)) * kLoScale);
      }
      __syncwarp();
      // B operand: this lane's column row8, rows 2 quad, + 1, + 8, + 9 of each half
      uint4 wf = make_uint4(0u, 0u, 0u, 0u);
      if (row8 < 2 * G) wf = *reinterpret_cast<const uint4 *>(sw + row8 * kTile + quad * 8);

      // output: this lane's channels [row8 D / 8, + D / 8), two per product
      constexpr int VW = D * BITS / 256;  // words of the lane's channels in a row
      float o[KM][4];
#pragma unroll
      for (int y = 0; y < KM; ++y) o[y][0] = o[y][1] = o[y][2] = o[y][3] = 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        uint32_t vw[4][VW];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = b * 16 + 2 * quad + (e & 1) + (e >> 1) * 8;
          if (VW == 4) {
            const uint4 u = *reinterpret_cast<const uint4 *>(sv + piece_at<RB>(r, row8));
            vw[e][0] = u.x, vw[e][1] = u.y, vw[e][2] = u.z, vw[e][3] = u.w;
          } else if (VW == 2) {
            const uint2 u = *reinterpret_cast<const uint2 *>(sv + piece_at<RB>(r, row8 >> 1) +
                                                             (row8 & 1) * 8);
            vw[e][0] = u.x, vw[e][1] = u.y;
          } else {
            vw[e][0] = *reinterpret_cast<const uint32_t *>(sv + piece_at<RB>(r, row8 >> 2) +
                                                           (row8 & 3) * 4);
          }
        }
        const uint32_t bw0 = b ? wf.z : wf.x, bw1 = b ? wf.w : wf.y;
#pragma unroll
        for (int w2 = 0; w2 < VW; ++w2) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t sel = h ? 0x7632 : 0x5410;
            const uint32_t v01 = __byte_perm(vw[0][w2], vw[1][w2], sel);
            const uint32_t v23 = __byte_perm(vw[2][w2], vw[3][w2], sel);
            if (BITS == 8) {
              uint32_t a0, a1, a2, a3;
              codes8(v01, a0, a1);
              codes8(v23, a2, a3);
              mma_f16(o[2 * w2 + h], a0, a1, a2, a3, bw0, bw1);
            } else {
              uint32_t ca[4], cb[4];
              codes4(v01, ca);
              codes4(v23, cb);
              mma_f16(o[4 * w2 + 2 * h], ca[0], ca[1], cb[0], cb[1], bw0, bw1);
              mma_f16(o[4 * w2 + 2 * h + 1], ca[2], ca[3], cb[2], cb[3], bw0, bw1);
            }
          }
        }
      }
#pragma unroll
      for (int y = 0; y < KM; ++y) {
        acc[y][0] = fmaf(fmaf(o[y][1], kLoUnscale, o[y][0]), unit, acc[y][0]);
        acc[y][1] = fmaf(fmaf(o[y][3], kLoUnscale, o[y][2]), unit, acc[y][1]);
      }
      if (STAGES == 1) break;
      __syncwarp();  // the stage and the weights are rewritten from here on
      const int next = r0 + STAGES * kWarps * kTile;
      if (next < hi) load_tile(next, st);
      cp_async_commit();
      st = st + 1 == STAGES ? 0 : st + 1;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    // the lanes whose columns are their channels' group hold the output
    if (quad == row8 * (D / 8) / 32) {
#pragma unroll
      for (int y = 0; y < KM; ++y) {
        s_acc[warp][row8 * (D / 8) + 2 * y] = acc[y][0];
        s_acc[warp][row8 * (D / 8) + 2 * y + 1] = acc[y][1];
      }
    }
  }
  if (STEP && active && len >= lo && len < hi) {  // this CTA holds the new row
    for (int e = tid; e < D; e += kThreads)
      static_cast<T *>(c.qbuf)[((size_t)i * p.P + ntok % p.P) * D + e] =
          static_cast<const T *>(p.q)[(size_t)hl * D + e];
    if (tid == 0) c.pos[off + len] = p.C + ntok;
  }
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  const int warps = active ? min(kWarps, (hi - lo + kTile - 1) / kTile) : 0;  // with rows
  __syncthreads();
  m = -INFINITY, l = 0.f;
  float out = 0.f;  // thread d < D: channel d
  for (int w = 0; w < warps; ++w) m = fmaxf(m, s_m[w]);
  for (int w = 0; w < warps; ++w) {
    const float f = ex2_approx(s_m[w] - m);
    l += s_l[w] * f;
    if (tid < D) out += s_acc[w][tid] * f;
  }
  if (p.nchunks > 1) {
    float *part = p.part + ((size_t)hl * p.nchunks + ch) * PF;
    if (active) {
      if (tid < D) part[tid] = out;
      if (tid == 0) *reinterpret_cast<float2 *>(part + D) = make_float2(m, l);
    }
    __syncthreads();
    if (tid == 0) {
      __threadfence();  // after the barrier it covers the whole CTA's writes
      s_last = atomicAdd(p.count + hl, 1u) == (uint32_t)p.nchunks - 1u;
      __threadfence();
    }
    __syncthreads();
    if (!s_last) return;
    // at most kThreads ranges (quant_chunk): one thread each for their factors
    const int np = n > 0 ? (n + per - 1) / per : 1;
    const float *first_part = p.part + (size_t)hl * p.nchunks * PF;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (tid < np) ml = __ldcg(reinterpret_cast<const float2 *>(first_part + (size_t)tid * PF + D));
    float mx = ml.x;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
    if (lane == 0) s_m[warp] = mx;
    __syncthreads();
    m = s_m[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s_m[w]);
    const float f = ml.y == 0.f ? 0.f : ex2_approx(ml.x - m);
    s_factor[tid] = f;
    l = ml.y * f;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    if (lane == 0) s_l[warp] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) l += s_l[w];
    out = 0.f;
    if (tid < D) {
#pragma unroll 8
      for (int j = 0; j < np; ++j) out += __ldcg(first_part + (size_t)j * PF + tid) * s_factor[j];
    }
    if (tid == 0) p.count[hl] = 0u;
  }
  // the prior: another set of keys with its own normalised output
  if (p.prior_lse) {
    const float pm = p.prior_lse[hl] * kLog2e;
    if (!(pm == -INFINITY)) {
      const float mn = fmaxf(m, pm);
      const float f = l == 0.f ? 0.f : ex2_approx(m - mn), w = ex2_approx(pm - mn);
      l = l * f + w;
      out = out * f;
      if (tid < D) out += w * p.prior_out[(size_t)hl * D + tid];
      m = mn;
    }
  }
  if (tid < D) p.out[(size_t)hl * D + tid] = l == 0.f ? 0.f : out / l;
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

// Rows of a CTA's range at most: one tile per warp, or, for segments of more
// than kMostRanges such ranges, as many as keep to that number (the CTA that
// joins a head's ranges handles one per thread).
constexpr int kMostRanges = 96;
int quant_chunk(int nheads, int max_segment) {
  (void)nheads;
  constexpr int one = kWarps * kTile;
  const int tiles = (max_segment + kMostRanges * one - 1) / (kMostRanges * one);
  return one * (tiles < 1 ? 1 : tiles);
}

namespace {

template <int D, typename T, int BITS, bool STEP, int STAGES>
cudaError_t launch(const QAttnArgs &a, int grid, cudaStream_t s) {
  constexpr int smem = Smem<D, BITS, STAGES>::kTotal;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem_of(quant_attn_kernel<D, T, BITS, STEP, STAGES>, smem, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(quant_attn_kernel<D, T, BITS, STEP, STAGES>, grid, kThreads, smem, s, a);
}

}  // namespace

cudaError_t launch_quant_attention(const QAttnArgs &a, int D, int dtype, int bits,
                                   cudaStream_t s) {
  const long long grid = (long long)a.nheads * a.nchunks;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
#define HKV_QATTN(BITS_, STEP_) \
  if (a.chunk == kWarps * kTile)                                              \
    HKV_DISPATCH(D, dtype, return launch<kD, kT, BITS_, STEP_, 1>(a, (int)grid, s)); \
  HKV_DISPATCH(D, dtype, return launch<kD, kT, BITS_, STEP_, 2>(a, (int)grid, s))
  if (bits == HKV_Q8) {
    if (a.k_new) {
      HKV_QATTN(8, true);
    }
    HKV_QATTN(8, false);
  }
  if (a.k_new) {
    HKV_QATTN(4, true);
  }
  HKV_QATTN(4, false);
#undef HKV_QATTN
  return cudaErrorInvalidValue;
}

}  // namespace hkv
