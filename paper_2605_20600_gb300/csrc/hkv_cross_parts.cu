// Attention of more than 16 query rows with fp32 outs on tcgen05, from fp32 or
// bf16 queries and states.
//
// An fp32 element is three bf16 parts of falling size (24 bits), a bf16 one is
// itself; the weights are three parts. Of the products of parts those that reach
// past 2^-24 are taken, the small ones first: six for fp32, for bf16 one (scores)
// and three (outs). A CTA takes 128 query rows of one (sequence, key head) and a
// range of keys in tiles of 64; its warps:
//   0-3    a thread per row: scores (TMEM) to weights, parts of weights to TMEM
//   4-7    a thread per row: O = O f + (W V of the tile), O in registers: chained
//          in the tensor core its sums would truncate once per 16 keys
//   8-11   loads of K (two warps) and of V, cut into parts in shared memory; those
//          of Q are the first eight warps', which have nothing else to do yet
//   12     issues the products; S of a tile is computed while the weights of the
//          one before are made (two buffers of S, of the last parts and of O)
//
// What bounds it: the chain of loads, parts and products around each tile of keys;
// the tensor pipe is busy for 0.42. Thirteen warps leave a thread 128 registers, too
// few for warps 4-7 with heads of 128 (a row of O and 32 columns more): 428 bytes are
// spilled (fp32; 52 with heads of 64). 1024 fp32 queries and states, 32 heads of 128:
// 118 us (145 TFLOP/s of the definition's products, 873 of bf16 ones; six products
// of parts on mma.sync took 915, Q loaded by the warps of K and V first 140); 257
// padded queries over up to 777 states, 5 x 8 heads of 64: 22.5 us (28).
#include "hkv_cross.cuh"
#include "hkv_quant.cuh"
#include "hkv_tcgen05.cuh"

namespace hkv {
namespace {

constexpr int kRows = 128, kKeys = 64, kThreads = 13 * 32;
// TMEM: two buffers of S (64 columns), which the weights' first two parts take
// over, two of the third part (32), two of O
constexpr int kS = 0, kThird = 128, kO = 192, kCols = 512;

template <int D, typename T>
struct PartsSmem {
  static constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
  static constexpr int kQPlane = kRows * D * 2, kPlane = kKeys * D * 2;
  static constexpr int kQ = kPlanes * kQPlane, kTile = kPlanes * kPlane;
  static constexpr int kOut = kRows * D * 4;   // the outs, where Q, K and V were
  static constexpr int kStages = kQ + 4 * kTile <= 220 * 1024 ? 2 : 1;  // of K and of V
  static constexpr int kUsed = kQ + 2 * kStages * kTile > kOut ? kQ + 2 * kStages * kTile : kOut;
  static constexpr int kBytes = 1024 + kUsed;
};

// A pair of fp32 as three bf16 parts of falling size; the remainders are exact.
// ANY: the first part stays finite where an element lies above the largest bf16
// number.
template <bool ANY>
__device__ __forceinline__ void split3(uint64_t x, uint32_t (&p)[3]) {
  const uint64_t minus = pair_of(-1.f, -1.f);
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    if (ANY && j == 0)
      asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(p[0]) : "f"(high(x)), "f"(low(x)));
    else
      p[j] = pack2(low(x), high(x));
    if (j < 2) x = fma2(pair_of(p[j] << 16, p[j] & 0xFFFF0000u), minus, x);
  }
}

// The 8 elements of a piece as they lie in global memory.
template <typename T>
struct RawPiece {
  uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ RawPiece<T> raw_piece(const T *from, bool on) {
  RawPiece<T> r;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i)
    r.u[i] = on ? reinterpret_cast<const uint4 *>(from)[i] : make_uint4(0, 0, 0, 0);
  return r;
}
// ... and its parts into the planes at dst (rows of 128 bytes by 64 channels,
// 128-byte swizzle)
__device__ __forceinline__ void put_piece(unsigned char *dst, int, const RawPiece<__nv_bfloat16> &r) {
  *reinterpret_cast<uint4 *>(dst) = r.u[0];
}
__device__ __forceinline__ void put_piece(unsigned char *dst, int plane, const RawPiece<float> &r) {
  const uint32_t x[8] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w, r.u[1].x, r.u[1].y, r.u[1].z, r.u[1].w};
  uint32_t p[4][3];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    split3<true>(pair_of(x[2 * j], x[2 * j + 1]), p[j]);
#pragma unroll
  for (int k = 0; k < 3; ++k)
    *reinterpret_cast<uint4 *>(dst + k * plane) = make_uint4(p[0][k], p[1][k], p[2][k], p[3][k]);
}
template <int ROWS>
__device__ __forceinline__ int piece_of(int r, int c) {
  return (c >> 3) * ROWS * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4);
}

// Scores that are NaN or +inf are computed once more from the elements: the parts of
// an infinite one have signs of their own, so that its products meet as inf - inf, and
// where a product of finite ones overflows, those of their small parts may have done so
// before it with the other sign. One thread's row and 64 keys, in TMEM at `at`, of
// which `left` count. (A function, so that its code costs the loop nothing: with it
// there 5 x 257 queries of 8 heads over 777 states take 28.7 us instead of 26.8.)
template <int D>
__device__ __noinline__ void plain_scores(const float *q, const float *k, long long kt, int left, uint32_t at) {
#pragma unroll 1
  for (int j = 0; j < kKeys; ++j) {
    uint32_t bits;
    tmem_ld1(bits, at + j);
    tmem_wait_ld();
    float sum = __uint_as_float(bits);
    if (j < left && !(sum < INFINITY)) {
      sum = 0.f;
#pragma unroll 1
      for (int c = 0; c < D; ++c) sum = fmaf(q[c], k[j * kt + c], sum);
    }
    tmem_st1(at + j, __float_as_uint(sum));
  }
  tmem_wait_st();
}

template <int D, typename T>
__global__ void __launch_bounds__(kThreads, 1) cross_parts_kernel(const __grid_constant__ CrossArgs p) {
  using SM = PartsSmem<D, T>;
  constexpr int NP = SM::kPlanes, ST = SM::kStages, PF = D + 4, PPR = D / 8;
  extern __shared__ unsigned char dyn_raw[];
  __shared__ uint64_t s_kvf[2][ST], s_kve[2][ST], s_q;   // K and V: filled, free again
  __shared__ uint64_t s_s[2], s_p[2], s_o[2], s_oe[2];   // S, W and O of a tile ready; O taken
  __shared__ uint64_t s_drain;
  __shared__ uint32_t s_tmem;
  __shared__ float s_f[2][kRows], s_ml[2][kRows];
  unsigned char *dyn = dyn_raw + ((1024u - (smem_u32(dyn_raw) & 1023u)) & 1023u);
  unsigned char *skv = dyn + SM::kQ;  // K's places, then V's
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
  if (tid == 0) {
    for (int j = 0; j < ST; ++j)
      for (int kv = 0; kv < 2; ++kv) {
        mbar_init(&s_kvf[kv][j], 2);
        mbar_init(&s_kve[kv][j], 1);
      }
    mbar_init(&s_q, 8);
    for (int b = 0; b < 2; ++b) {
      mbar_init(&s_s[b], 1);
      mbar_init(&s_p[b], 4);
      mbar_init(&s_o[b], 1);
      mbar_init(&s_oe[b], 4);
    }
    mbar_init(&s_drain, 1);
    fence_barrier_init();
  }
  // TMEM only after the wait, and the next kernel's CTAs only after TMEM (see
  // the shared prompts' kernel)
  pdl_wait();
  if (warp == 0) {
    tmem_alloc(&s_tmem, kCols);
    pdl_launch_dependents();
  }
  const Order order = order_of(p, [&](int tokens) {
    return tokens == 0 ? 0 : p.group == 1 ? (tokens + kRows - 1) / kRows : p.tiles;
  });
  const int piece = piece_at(p, order, blockIdx.x);
  Work w = {};
  if (piece >= 0) w = work_of(p, piece);
  const int all = p.group * p.tokens, r0 = w.tile * kRows;
  const int lo = w.sp * p.split_len;
  const int hi = min(keys_of_rows(p, w, r0, min(all, r0 + kRows)), lo + p.split_len);
  const int n = hi > lo ? (hi - lo + kKeys - 1) / kKeys : 0;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, s_tmem, 0);
  const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
  bool ok = true;
  float acc[D];  // warps 4-7
  if (n > 0 && warp < 8) {
    constexpr int E = kRows * PPR / 256;  // pieces a thread, all on their way at once
    RawPiece<T> raw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int r = (tid + e * 256) / PPR, c = (tid + e * 256) % PPR;
      const Row x = row_of(p, w.kvh, min(r0 + r, all - 1));
      const bool on = r0 + r < all && x.token < w.qlen;
      raw[e] = raw_piece<T>(static_cast<const T *>(p.q) + w.s * p.qs +
                                (on ? x.token * p.qt + x.head * p.qh : 0) + c * 8, on);
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      put_piece(dyn + piece_of<kRows>((tid + e * 256) / PPR, (tid + e * 256) % PPR), SM::kQPlane, raw[e]);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(&s_q);
  }
  if (n > 0 && warp >= 8 && warp < 12) {
    const int kv = (warp - 8) >> 1, lt = tid & 63;
    const T *from = static_cast<const T *>(kv ? p.v : p.k) + w.s * p.ks + w.kvh * p.kh + lo * p.kt;
    // a tile in chunks of eight pieces a thread; the next chunk is on its way
    // while a place for it is waited for
    constexpr int E = 8, CH = kKeys * PPR / 64 / E, ROWS = kKeys / CH;
    RawPiece<T> next[E];
    auto fetch = [&](int u) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int r = u * ROWS + (lt + e * 64) / PPR, c = (lt + e * 64) % PPR;
        const bool on = lo + r < hi;
        next[e] = raw_piece<T>(from + (on ? r * p.kt : 0) + c * 8, on);
      }
    };
    fetch(0);
    for (int u = 0; u < n * CH && ok; ++u) {
      const int i = u / CH, j = i % ST;
      if (u % CH == 0 && i >= ST)
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_kve[kv][j], (i / ST - 1) & 1));
      if (!ok) break;
      unsigned char *dst = skv + (kv * ST + j) * SM::kTile;
#pragma unroll
      for (int e = 0; e < E; ++e)
        put_piece(dst + piece_of<kKeys>(u % CH * ROWS + (lt + e * 64) / PPR, (lt + e * 64) % PPR),
                  SM::kPlane, next[e]);
      if (u % CH == CH - 1) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_kvf[kv][j]);
      }
      if (u + 1 < n * CH) fetch(u + 1);
    }
  } else if (n > 0 && warp == 12) {
    const uint32_t q_at = smem_u32(dyn);
    auto filled = [&](int kv, int i) {
      return __all_sync(0xFFFFFFFFu, mbar_wait(&s_kvf[kv][i % ST], (i / ST) & 1));
    };
    auto scores = [&](int i) {  // S of tile i
      if (elect_one()) {
        const uint32_t s = tmem + kS + (i & 1) * 64, k_at = smem_u32(skv) + i % ST * SM::kTile;
        bool add = false;
#pragma unroll
        for (int order = NP - 1; order >= 0; --order)
#pragma unroll
          for (int a = order; a >= 0; --a) {
            const uint64_t qd = tc_desc(q_at + a * SM::kQPlane, 16);
            const uint64_t kd = tc_desc(k_at + (order - a) * SM::kPlane, 16);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              tc_mma(s, qd + (((ks >> 2) * kRows * 128 + (ks & 3) * 32) >> 4),
                     kd + (((ks >> 2) * kKeys * 128 + (ks & 3) * 32) >> 4),
                     tc_instr(kRows, kKeys, false), add);
              add = true;
            }
          }
        tc_commit(&s_s[i & 1]);
        tc_commit(&s_kve[0][i % ST]);
      }
      __syncwarp();
    };
    ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_q, 0)) && filled(0, 0);
    tc_fence_after();
    if (ok) scores(0);
    for (int i = 0; i < n && ok; ++i) {
      const int b = i & 1;
      if (i + 1 < n) {
        ok = filled(0, i + 1);
        if (!ok) break;
        scores(i + 1);  // over the weights of tile i - 1, after the products that read them
      }
      // V, W and a place for O, asked for together
      uint64_t *vf = &s_kvf[1][i % ST], *wf = &s_p[b], *oe = &s_oe[b];
      const uint32_t vp = (i / ST) & 1, wp = (i >> 1) & 1, op = wp ^ 1;
      const bool v_here = mbar_try_wait(vf, vp), w_here = mbar_try_wait(wf, wp);
      if (!__all_sync(0xFFFFFFFFu, v_here && w_here && (i < 2 || mbar_try_wait(oe, op))))
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(vf, vp) && mbar_wait(wf, wp) && (i < 2 || mbar_wait(oe, op)));
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        const uint32_t v_at = smem_u32(skv) + (ST + i % ST) * SM::kTile;
        bool add = false;
#pragma unroll
        for (int order = 2; order >= 0; --order)
#pragma unroll
          for (int a = order; a >= 0; --a) {  // part a of W, plane order - a of V
            if (order - a >= NP) continue;
            const uint32_t wp = tmem + (a == 2 ? kThird + b * 32 : kS + b * 64 + a * 32);
            const uint64_t vd = tc_desc(v_at + (order - a) * SM::kPlane, kKeys * 128);
#pragma unroll
            for (int kk = 0; kk < kKeys / 16; ++kk) {
              tc_mma_ta(tmem + kO + b * D, wp + kk * 8, vd + kk * (16 * 128 >> 4),
                        tc_instr(kRows, D, true), add);
              add = true;
            }
          }
        tc_commit(&s_o[b]);
        tc_commit(&s_kve[1][i % ST]);
      }
      __syncwarp();
    }
  } else if (warp < 4) {
    const int r = r0 + tid;
    int seen = r < all ? keys_seen(p, w, row_of(p, w.kvh, r).token) : 0;
    seen = min(seen, lo + p.split_len);
    float m = kNoKey, l = 0.f;
    for (int i = 0; i < n; ++i) {
      const int b = i & 1;
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_s[b], (i >> 1) & 1));
      if (ok && i > 1) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_oe[b], ((i >> 1) - 1) & 1));
#ifdef HKV_CROSS_TEST_STALL  // one warp waits for a phase that nothing completes before its limit
      if (warp == (int)(blockIdx.x & 3) && i == 1) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_drain, 0));
#endif
      if (!ok) break;
      tc_fence_after();
      uint32_t s[2][32];
      const int left = seen - lo - i * kKeys;  // keys of the tile that count
      auto load_scores = [&] {
#pragma unroll
        for (int c = 0; c < 2; ++c) tmem_ld32(s[c], tmem + lanes + kS + b * 64 + c * 32);
        tmem_wait_ld();
      };
      load_scores();
      float mx;
      auto mask_and_max = [&] {
        if (left < kKeys) {
#pragma unroll
          for (int j = 0; j < kKeys; ++j)
            if (j >= left) s[j >> 5][j & 31] = 0xFF800000u;  // -inf
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < kKeys; j += 8)
#pragma unroll
          for (int u = 0; u < 4; ++u)
            top[u] = max3_nan(top[u], __uint_as_float(s[j >> 5][(j & 31) + 2 * u]),
                              __uint_as_float(s[j >> 5][(j & 31) + 2 * u + 1]));
        mx = max3_nan(max3_nan(top[0], top[1], top[2]), top[3], top[3]) * p.qscale;
      };
      mask_and_max();
      if (NP > 1 && __any_sync(0xFFFFFFFFu, !(mx < INFINITY))) {
        const Row x = row_of(p, w.kvh, min(r, all - 1));
        plain_scores<D>(static_cast<const float *>(p.q) + w.s * p.qs + x.token * p.qt + x.head * p.qh,
                        static_cast<const float *>(p.k) + w.s * p.ks + w.kvh * p.kh + (lo + i * kKeys) * p.kt,
                        p.kt, left, tmem + lanes + kS + b * 64);
        load_scores();
        mask_and_max();
      }
      // (the reference stays finite: scores of -inf weigh nothing against it)
      const float mn = fmaxf(m, mx), f = mn == m ? 1.f : ex2_approx(m - mn);
      m = mn;
      const uint64_t scale2 = pair_of(p.qscale, p.qscale), ref2 = pair_of(-m, -m);
      uint64_t sum[2] = {0, 0};
#pragma unroll
      for (int j0 = 0; j0 < kKeys; j0 += 16) {  // 8 columns of each part at a time
        uint32_t wp[3][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int a = j0 + 2 * j;
          const uint64_t e = fma2(pair_of(s[a >> 5][a & 31], s[a >> 5][(a & 31) + 1]), scale2, ref2);
          const uint64_t wj = pair_of(ex2_approx(low(e)), ex2_approx(high(e)));
          sum[j & 1] = add2(sum[j & 1], wj);
          uint32_t part[3];
          split3<false>(wj, part);
#pragma unroll
          for (int k = 0; k < 3; ++k) wp[k][j] = part[k];
        }
        tmem_st8(tmem + lanes + kS + b * 64 + j0 / 2, wp[0]);
        tmem_st8(tmem + lanes + kS + b * 64 + 32 + j0 / 2, wp[1]);
        tmem_st8(tmem + lanes + kThird + b * 32 + j0 / 2, wp[2]);
      }
      sum[0] = add2(sum[0], sum[1]);
      l = l * f + (low(sum[0]) + high(sum[0]));
      s_f[b][tid] = f;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_p[b]);
    }
    s_ml[0][tid] = m;
    s_ml[1][tid] = l;
  } else if (warp < 8) {
    const int row = tid - 128;
#pragma unroll
    for (int e = 0; e < D; ++e) acc[e] = 0.f;
    for (int i = 0; i < n; ++i) {
      const int b = i & 1;
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_p[b], (i >> 1) & 1));
      const float f = s_f[b][row];
      ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait(&s_o[b], (i >> 1) & 1));
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        tmem_ld32(o, tmem + lanes + kO + b * D + c);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; ++e) acc[c + e] = fmaf(acc[c + e], f, __uint_as_float(o[e]));
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_oe[b]);
    }
  }
  // one wait that ran out fails the whole CTA
  const bool failed = __syncthreads_or(!ok);
  if (failed) {
    // products that were issued may still run: they get the limit once more
    // before their place and the TMEM are used again
    if (warp == 12 && elect_one()) {
      set_err(p.err, HKV_ERR_TIMEOUT);
      tc_commit(&s_drain);
    }
    mbar_wait(&s_drain, 0);
    __syncthreads();
  }
  tc_fence_after();
  if (warp >= 4 && warp < 8) {
    // rows to shared memory, where Q, K and V were, then whole rows out
    const int r = tid - 128;
    Row x = {};
    if (r0 + r < all) x = row_of(p, w.kvh, r0 + r);
    const bool live = r0 + r < all && x.token < w.qlen, wrong = w.bad || failed;
    const float m = s_ml[0][r], l = s_ml[1][r];
    const size_t row = ((size_t)w.s * p.heads + x.head) * p.tokens + x.token;
    const float by = p.splits > 1 ? 1.f : wrong ? NAN : l == 0.f ? 0.f : 1.f / l;
    float *rows = reinterpret_cast<float *>(dyn) + (warp & 3) * 32 * D;
#pragma unroll
    for (int c = 0; c < D / 4; ++c)
      *reinterpret_cast<float4 *>(rows + lane * D + ((c ^ (lane & 7)) << 2)) = make_float4(
          acc[4 * c] * by, acc[4 * c + 1] * by, acc[4 * c + 2] * by, acc[4 * c + 3] * by);
    __syncwarp();
    float *part = p.part + (row * p.splits + w.sp) * PF;
    float *to = p.splits > 1 ? part
                             : static_cast<float *>(p.out) + w.s * p.os + x.token * p.ot + x.head * p.oh;
    constexpr int PR = D / 4, RPP = 32 / PR;  // pieces a row, rows a pass
#pragma unroll 4
    for (int i = 0; i < 32; i += RPP) {
      const int rr = i + lane / PR, c = lane % PR;
      const bool on = __shfl_sync(0xFFFFFFFFu, live, rr);
      float *at = reinterpret_cast<float *>(
          __shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(to), rr));
      if (on)
        *reinterpret_cast<float4 *>(at + c * 4) =
            *reinterpret_cast<const float4 *>(rows + rr * D + ((c ^ (rr & 7)) << 2));
    }
    if (live) {
      if (p.splits > 1)
        *reinterpret_cast<float2 *>(part + D) = make_float2(wrong ? NAN : m, wrong ? 0.f : l);
      else if (p.lse)
        p.lse[row] = wrong ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_free(tmem, kCols);
}

template <int D, typename T>
cudaError_t launch(const CrossArgs &a, int grid, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem_of(cross_parts_kernel<D, T>, PartsSmem<D, T>::kBytes, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(cross_parts_kernel<D, T>, grid, kThreads, PartsSmem<D, T>::kBytes, s, a);
}

}  // namespace

cudaError_t launch_cross_parts(const CrossArgs &a, int D, int dtype, cudaStream_t s) {
  const long long grid = (long long)a.seqs * a.kv * a.tiles * a.splits;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  cudaError_t e = cudaErrorInvalidValue;
  HKV_DISPATCH(D, dtype, e = (launch<kD, kT>(a, (int)grid, s)));
  return e;
}

}  // namespace hkv
