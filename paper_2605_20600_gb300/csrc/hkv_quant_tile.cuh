// Attention of one query over tiles of 32 quantised rows, one tile a warp.
//
// The products run on the tensor cores (mma.sync m16n8k16, fp16 operands, fp32
// sums), not because one query per head fills them (a sixteenth does) but
// because codes then need no conversion to fp32: a code is an exact fp16
// number two of which a bit operation and one packed subtraction make, and the
// eight columns carry what one query leaves empty:
//  * scores, 16 rows of K (M) x 16 channels (K): the columns hold the query's
//    channels of each group of 32, over a power of two by the group's largest,
//    cut into two fp16 parts (hi, and the rest times 2^11: 22 bits, down to 2^-50
//    of the largest), zero outside the group. The sums of a row come out per
//    group, ready for the group's scale and power of two in fp32;
//  * output, 16 channels of V^T (M) x 16 rows (K): the columns hold the rows'
//    weights times the row's scale of each group, cut in two the same way over
//    a power of two by the tile's largest scale of the group (the largest
//    product would be known only after the scores: 115 us instead of 112 for
//    eight layers of 256 heads); a channel uses its own group's two columns.
// Sums chain over at most 8 (scores) or 2 (output) products in the tensor core
// and are added in fp32 registers beyond that. A tile is 585 (4 bits) to 675
// instructions of a warp at D = 128; converting each code to fp32 for plain
// fused multiply-adds takes two a code, 512 a lane and tile before any product.
#pragma once

#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_select.cuh"

namespace hkv {

constexpr int kTile = 32;  // rows a warp handles at a time

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

// fp16 pairs of codes from stored ones, exact: 0x64uu is the fp16 number
// 1024 + uu, and 1024 + bias comes off. (The stored bits are fp16 numbers too,
// subnormal ones, and the bias could come off the sums: 64 operations a tile
// less for 1 % of the time, but the scores lose a factor of four in precision.)
// codes8: bytes (0, 2) and (1, 3) of a word.
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
// the first of a chain: c = a b
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                              uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// maximum over the warp
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
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

// The power of two over which numbers up to `bits` (a non-negative fp32's) are cut
// into two fp16 parts: they come out below 2^15, half of fp16's largest, so that
// parts are normal numbers down to 2^-28 of the largest. Kept in [2^-126, 2^113].
__device__ __forceinline__ float part_unit(uint32_t bits) {
  return __uint_as_float(min(max(bits & 0x7F800000u, 0x07800000u), 0x7F000000u) - 0x07000000u);
}
__device__ __forceinline__ float inv_pow2(float p) {
  return __uint_as_float(0x7F000000u - __float_as_uint(p));
}

// A tile in shared memory: codes of K and V, scales of K and V.
template <int D, int BITS>
struct TileOf {
  using R = QRow<D, BITS>;
  static constexpr int kCodes = kTile * R::kBytes, kScales = kTile * R::kScaleBytes;
  static constexpr int kBytes = 2 * (kCodes + kScales);
  // the query's two parts being made (fp16 [2][D])
  static constexpr int kOperand = 2 * D * 2;
};

// A head as its tiles see it.
struct HeadRef {
  long long off;
  int len, n, tiles;   // old rows, rows to attend over, tiles (at least one)
  uint16_t bad, dense; // status of a head that cannot be served; its label
};

// Tiles of a head of `len` rows: one at least, so that some warp reports,
// or writes the outputs of an empty head.
template <bool STEP>
__device__ __forceinline__ int head_tiles(int len, int max_rows) {
  const int n = len + (STEP ? 1 : 0);
  return n <= 0 || n > max_rows || len < 0 ? 1 : (n + kTile - 1) / kTile;
}

template <bool STEP>
__device__ __forceinline__ HeadRef head_ref(const QAttnArgs &p, int hl) {
  const CacheArgs &c = p.q8.c;
  const int i = p.base + hl;
  HeadRef r;
  r.off = c.off[i];
  r.len = c.len[i];
  const int cap = c.cap[i];
  r.n = r.len + (STEP ? 1 : 0);
  r.tiles = head_tiles<STEP>(r.len, p.max_rows);
  r.bad = 0;
  r.dense = STEP ? c.label[i] == HKV_DENSE : false;
  if (r.off < 0 || cap < 0 || r.off + cap > c.arena_tokens || r.len < 0 || r.len > cap)
    r.bad = HKV_ERR_BOUNDS;
  else if (STEP && !r.dense && c.nbuf[i] >= p.P)
    r.bad = HKV_ERR_STATE;
  else if (r.n > cap || r.n > p.max_rows)
    r.bad = HKV_ERR_CAPACITY;
  return r;
}

// Starts the copies of `rows` rows from arena row `row` on into a tile.
template <int D, int BITS>
__device__ __forceinline__ void load_tile(unsigned char *stage, const QCacheArgs &q, long long row,
                                          int rows) {
  using TL = TileOf<D, BITS>;
  constexpr int RB = QRow<D, BITS>::kBytes, SB = QRow<D, BITS>::kScaleBytes;
  const int lane = threadIdx.x & 31;
  unsigned char *sk = stage, *sv = sk + TL::kCodes, *ss = sv + TL::kCodes;
  const int my_at = piece_at<RB>(lane / (RB / 16), lane % (RB / 16));
  // the tile's codes are one stretch of the arena: lane e of each 512 bytes
  // takes piece e; its place in the tile moves by whole rows from one to
  // the next, which flips one swizzle bit at 128-byte rows
  const size_t src = (size_t)row * RB + lane * 16;
  const unsigned char *K = static_cast<const unsigned char *>(q.c.K) + src;
  const unsigned char *V = static_cast<const unsigned char *>(q.c.V) + src;
  const int pieces = rows * (RB / 16) - lane;
#pragma unroll
  for (int e = 0; e < RB / 16; ++e) {
    const int at = (RB == 128 && (e & 1) ? my_at ^ 64 : my_at) + e * 512;
    if (e * 32 < pieces) {
      cp_async16(sk + at, K + e * 512);
      cp_async16(sv + at, V + e * 512);
    }
  }
  if (lane < rows) {
    cp_async_small<SB>(ss + lane * SB, static_cast<const unsigned char *>(q.ks) +
                                           (row + lane) * SB);
    cp_async_small<SB>(ss + TL::kScales + lane * SB,
                       static_cast<const unsigned char *>(q.vs) + (row + lane) * SB);
  }
}

// The query as the scores' B operand, this lane's share.
template <int D, int BITS>
struct Query {
  uint32_t f[D / 16][2];
  float unit;              // power of two of group `quad`
};

// From the lane's channels lane * E ..; sq: the warp's operand area, free again
// on return. The whole warp calls.
template <int D, int BITS>
__device__ __forceinline__ Query<D, BITS> make_query(const float (&qv)[D / 32],
                                                     __half *sq) {
  // the query, each group over its power of two, in two fp16 parts, in the order
  // in which the codes of a word come out in pairs
  constexpr int E = D / 32, KM = D / 16, LPG = 32 / E;  // lanes of a group
  const int lane = threadIdx.x & 31, row8 = lane >> 2, quad = lane & 3;
  Query<D, BITS> r;
  uint32_t qm = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) qm = max(qm, __float_as_uint(qv[e]) & 0x7FFFFFFFu);
#pragma unroll
  for (int o = LPG / 2; o >= 1; o >>= 1) qm = max(qm, __shfl_xor_sync(0xFFFFFFFFu, qm, o));
  const float q2 = part_unit(qm), qi = inv_pow2(q2);
  r.unit = __shfl_sync(0xFFFFFFFFu, q2, quad * LPG & 31);  // (no group: any)
  __syncwarp();
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
  const uint4 *src = reinterpret_cast<const uint4 *>(sq + (row8 & 1) * D + quad * (D / 4));
  const bool in_group = (row8 >> 1) == quad * (D / 4) / 32;
#pragma unroll
  for (int x = 0; x < KM / 2; ++x) {
    const uint4 u = in_group ? src[x] : make_uint4(0u, 0u, 0u, 0u);
    r.f[2 * x][0] = u.x;
    r.f[2 * x][1] = u.y;
    r.f[2 * x + 1][0] = u.z;
    r.f[2 * x + 1][1] = u.w;
  }
  return r;
}

// The step's new token, as the warp that holds its tile loads it: 8 channels of
// K (the first D / 8 lanes) or V (the next), and the token's number.
struct NewRow {
  float x[8];
  int ntok;
};
template <int D, typename T>
__device__ __forceinline__ void load_new_row(const QAttnArgs &p, int hl, NewRow &nr) {
  const int lane = threadIdx.x & 31;
  if (lane < D / 4)
    load8<T>(static_cast<const T *>(lane < D / 8 ? p.k_new : p.v_new) + (size_t)hl * D +
                 lane % (D / 8) * 8,
             nr.x);
  nr.ntok = p.q8.c.ntok[p.base + hl];
}

// Quantises it to arena row hd.off + hd.len and to row r of the tile, and
// stores its query (qv) and position.
template <int D, typename T, int BITS>
__device__ __forceinline__ void append_row(const QAttnArgs &p, int hl, const HeadRef &hd,
                                           unsigned char *stage, int r, const NewRow &nr,
                                           const float (&qv)[D / 32]) {
  using R = QRow<D, BITS>;
  using TL = TileOf<D, BITS>;
  constexpr int RB = R::kBytes, SB = R::kScaleBytes, G = R::kGroups, E = D / 32;
  const CacheArgs &c = p.q8.c;
  const int lane = threadIdx.x & 31;
  if (lane < D / 4) {
    const int kv = lane / (D / 8), col = lane % (D / 8);
    uint32_t a, b;
    const uint32_t sb = quant_group<T, BITS>(nr.x, 0xFu << (lane & 28), a, b);
    const size_t at = (size_t)(hd.off + hd.len);
    unsigned char *row = static_cast<unsigned char *>(kv ? c.V : c.K) + at * RB;
    unsigned char *to = stage + kv * TL::kCodes;
    if (BITS == 8) {
      reinterpret_cast<uint2 *>(row)[col] = make_uint2(a, b);
      *reinterpret_cast<uint2 *>(to + piece_at<RB>(r, col >> 1) + (col & 1) * 8) =
          make_uint2(a, b);
    } else {
      reinterpret_cast<uint32_t *>(row)[col] = a;
      *reinterpret_cast<uint32_t *>(to + piece_at<RB>(r, col >> 2) + (col & 3) * 4) = a;
    }
    if ((col & 3) == 0) {
      static_cast<uint16_t *>(kv ? p.q8.vs : p.q8.ks)[at * G + col / 4] = (uint16_t)sb;
      reinterpret_cast<uint16_t *>(stage + 2 * TL::kCodes + kv * TL::kScales + r * SB)[col / 4] =
          (uint16_t)sb;
    }
  }
  T *ring = static_cast<T *>(c.qbuf) + ((size_t)(p.base + hl) * p.P + nr.ntok % p.P) * D;
#pragma unroll
  for (int e = 0; e < E; ++e) ring[lane * E + e] = (T)qv[e];
  if (lane == 0) c.pos[hd.off + hd.len] = p.C + nr.ntok;
  __syncwarp();
}

// The lane's channels of a head's query.
template <int D, typename T>
__device__ __forceinline__ void load_query(const QAttnArgs &p, int hl, float (&q)[D / 32]) {
  constexpr int E = D / 32;
  const T *from = static_cast<const T *>(p.q) + (size_t)hl * D + (threadIdx.x & 31) * E;
#pragma unroll
  for (int e = 0; e < E; ++e) q[e] = (float)from[e];
}

// One tile into the running maximum m, the lane's part of the sum l, and the
// accumulator: acc[y] are channels row8 D / 8 + 2 y, + 1, in the lanes whose
// `quad` is those channels' group.
template <int D, int BITS>
__device__ __forceinline__ void attend_tile(const unsigned char *stage, int rows,
                                            const Query<D, BITS> &q, float qscale, float &m,
                                            float &l, float (&acc)[D / 16][2]) {
  using R = QRow<D, BITS>;
  using TL = TileOf<D, BITS>;
  constexpr int RB = R::kBytes, G = R::kGroups, KM = D / 16;
  const int lane = threadIdx.x & 31, row8 = lane >> 2, quad = lane & 3;
  const unsigned char *sk = stage, *sv = sk + TL::kCodes, *ss = sv + TL::kCodes;
  const int own = row8 + 8 * quad;  // this lane's row
  // scores: x[b2] is the sum of row row8 + 8 b2 over this lane's group
  float xs[4];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int ra = b * 16 + row8, rb = ra + 8;
    float s[4];
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
        if (w == 0) mma_f16_first(s, a0, a1, a2, a3, q.f[0][0], q.f[0][1]);
        else mma_f16(s, a0, a1, a2, a3, q.f[w][0], q.f[w][1]);
      } else {
        uint32_t ca[4], cb[4];
        codes4(wa[w], ca);
        codes4(wb[w], cb);
        if (w == 0)
          mma_f16_first(s, ca[0], cb[0], ca[1], cb[1], q.f[0][0], q.f[0][1]);
        else
          mma_f16(s, ca[0], cb[0], ca[1], cb[1], q.f[2 * w][0], q.f[2 * w][1]);
        mma_f16(s, ca[2], cb[2], ca[3], cb[3], q.f[2 * w + 1][0], q.f[2 * w + 1][1]);
      }
    }
    const uint16_t *sc = reinterpret_cast<const uint16_t *>(ss);
    const bool grp = quad < G;  // the columns beyond the groups are empty
    const float fa = grp ? bf16_bits_to_float(sc[ra * G + (grp ? quad : 0)]) * q.unit : 0.f;
    const float fb = grp ? bf16_bits_to_float(sc[rb * G + (grp ? quad : 0)]) * q.unit : 0.f;
    xs[2 * b] = fa * fmaf(s[1], kLoUnscale, s[0]);
    xs[2 * b + 1] = fb * fmaf(s[3], kLoUnscale, s[2]);
  }
  // sums over the groups: lane (row8, quad) ends up with row row8 + 8 quad
  const bool b0 = quad & 1, b1 = quad & 2;
  float k0 = (b0 ? xs[1] : xs[0]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? xs[0] : xs[1], 1);
  float k1 = (b0 ? xs[3] : xs[2]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? xs[2] : xs[3], 1);
  float x = (b1 ? k1 : k0) + __shfl_xor_sync(0xFFFFFFFFu, b1 ? k0 : k1, 2);
  const bool on = own < rows;
  x = on ? x * qscale : -INFINITY;  // logits in powers of two

  const float mt = warp_max(x);
  if (mt > m) {  // the same for the whole warp
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

  // weights times scales of group `quad`, rows row8 + 8 b, over a power of two by
  // the tile's largest scale of the group, as two fp16 parts: the columns
  // 2 quad, 2 quad + 1 of an 8 x 8 block whose transpose is the B operand
  // (this lane: column row8, rows 2 quad, + 1 of the block)
  uint32_t sb[4], top = 0;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    sb[b] = 0;
    if (quad < G && row8 + 8 * b < rows)
      sb[b] = reinterpret_cast<const uint16_t *>(ss + TL::kScales)[(row8 + 8 * b) * G + quad];
    top = max(top, sb[b]);
  }
#pragma unroll
  for (int x2 = 4; x2 <= 16; x2 <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, x2));
  const float unit = part_unit(top << 16), inv = inv_pow2(unit);
  uint32_t wf[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const float y = __shfl_sync(0xFFFFFFFFu, w, (lane & ~3) | b) * (bf16_bits_to_float(sb[b]) * inv);
    const float lo = (y - __half2float(__float2half_rn(y))) * kLoScale;
    const __half2 pair = __floats2half2_rn(y, lo);
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;"
        : "=r"(wf[b])
        : "r"(*reinterpret_cast<const uint32_t *>(&pair)));
  }

  // output: this lane's channels [row8 D / 8, + D / 8), two per product
  constexpr int VW = D * BITS / 256;  // words of the lane's channels in a row
  float o[KM][4];
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
    const uint32_t bw0 = wf[2 * b], bw1 = wf[2 * b + 1];
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
          if (b == 0) mma_f16_first(o[2 * w2 + h], a0, a1, a2, a3, bw0, bw1);
          else mma_f16(o[2 * w2 + h], a0, a1, a2, a3, bw0, bw1);
        } else {
          uint32_t ca[4], cb[4];
          codes4(v01, ca);
          codes4(v23, cb);
          if (b == 0) {
            mma_f16_first(o[4 * w2 + 2 * h], ca[0], ca[1], cb[0], cb[1], bw0, bw1);
            mma_f16_first(o[4 * w2 + 2 * h + 1], ca[2], ca[3], cb[2], cb[3], bw0, bw1);
          } else {
            mma_f16(o[4 * w2 + 2 * h], ca[0], ca[1], cb[0], cb[1], bw0, bw1);
            mma_f16(o[4 * w2 + 2 * h + 1], ca[2], ca[3], cb[2], cb[3], bw0, bw1);
          }
        }
      }
    }
  }
#pragma unroll
  for (int y = 0; y < KM; ++y) {
    acc[y][0] = fmaf(fmaf(o[y][1], kLoUnscale, o[y][0]), unit, acc[y][0]);
    acc[y][1] = fmaf(fmaf(o[y][3], kLoUnscale, o[y][2]), unit, acc[y][1]);
  }
}

// The accumulator of attend_tile to `to` [D], from the lanes that hold it.
template <int D>
__device__ __forceinline__ void store_acc(float *to, const float (&acc)[D / 16][2]) {
  const int lane = threadIdx.x & 31, row8 = lane >> 2, quad = lane & 3;
  if (quad == row8 * (D / 8) / 32) {
#pragma unroll
    for (int y = 0; y < D / 16; ++y)
      *reinterpret_cast<float2 *>(to + row8 * (D / 8) + 2 * y) = make_float2(acc[y][0], acc[y][1]);
  }
}

template <int E>
__device__ __forceinline__ void store_row(float *to, const float (&o)[E]) {
  if (E == 4) *reinterpret_cast<float4 *>(to) = make_float4(o[0], o[1 % E], o[2 % E], o[3 % E]);
  else *reinterpret_cast<float2 *>(to) = make_float2(o[0], o[1 % E]);
}
// A head's result, channels lane * E .. of the unnormalised output: joined
// with the prior, normalised and written. The whole warp calls.
template <int D>
__device__ __forceinline__ void finish_head(const QAttnArgs &p, int hl, float m, float l,
                                            float (&o)[D / 32]) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  if (p.prior_lse) {
    const float pm = p.prior_lse[hl] * kLog2e;
    if (!(pm == -INFINITY)) {  // an empty prior's outputs are not looked at
      const float mn = fmaxf(m, pm);
      const float f = l == 0.f ? 0.f : ex2_approx(m - mn), w = ex2_approx(pm - mn);
      l = l * f + w;
#pragma unroll
      for (int e = 0; e < E; ++e)
        o[e] = o[e] * f + w * p.prior_out[(size_t)hl * D + lane * E + e];
      m = mn;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] *= inv;
  store_row<E>(p.out + (size_t)hl * D + lane * E, o);
  if (p.lse && lane == 0) p.lse[hl] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Adds a piece (maximum pm, sum pl, channels at src) to (m, l, o).
template <int E>
__device__ __forceinline__ void add_piece(float &m, float &l, float (&o)[E], float pm, float pl,
                                          const float *src) {
  const float mn = fmaxf(m, pm);
  const float f = l == 0.f ? 0.f : ex2_approx(m - mn), g = pl == 0.f ? 0.f : ex2_approx(pm - mn);
  m = mn;
  l = l * f + pl * g;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = o[e] * f + src[e] * g;
}

// A finished head's counters advance (a step).
__device__ __forceinline__ void advance_head(const QAttnArgs &p, int hl, bool dense) {
  const CacheArgs &c = p.q8.c;
  const int i = p.base + hl;
  atomicAdd(c.len + i, 1);
  atomicAdd(c.ntok + i, 1);
  if (!dense) atomicAdd(c.nbuf + i, 1);
}

}  // namespace hkv
