// Attention of the tokens' queries over their sequence's states, or of a
// prompt's tokens over the tokens up to themselves.
//
// cross_kernel (here) takes up to 16 bf16 query rows of a (sequence, key head), the
// heads of the group one after the other, and a range of keys on mma.sync
// m16n8k16, 16 keys of a tile a warp (32 for heads of 64: as many bytes on their way;
// single queries of 21 x 12 heads over up to 2861 states 30.4 -> 28.6 us);
// cross_few_kernel as many fp32 rows without the tensor core; the ranges of one query
// are joined by a second kernel. More rows are hkv_cross_tc.cu's and
// hkv_cross_parts.cu's.
//
// What bounds them: DRAM. One bf16 query of 64 x 32 heads over 300 states of 128:
// 59 us, 5.3 TB/s (tcgen05, with one of 128 rows in use, would take 64 keys a
// microsecond and CTA); 8 key heads over 2000 states: 86 us, 6.1 TB/s; fp32, 32
// heads over 300: 98 us, 6.4 TB/s (six products of parts on mma.sync: 400).
//
// Precision of cross_kernel: queries, keys and values (bf16) enter as they are, the weights as
// three bf16 parts for fp32 outs, which leaves nothing of them out, and as two,
// off by 2^-18 of a weight, for bf16 outs, whose own rounding is 2^-9. Sums are
// fp32; products chain in the tensor core within a tile.
#include "hkv_cross.cuh"
#include "hkv_quant.cuh"

namespace hkv {
namespace {

constexpr int kStages = 2;
using bf16 = __nv_bfloat16;

// the CTA's work. SORTED: by the sequences' lengths (kernels of their own, since
// the smallest wait for their instructions)
template <bool SORTED>
__device__ __forceinline__ Work few_work(const CrossArgs &p) {
  if (!SORTED) return work_of(p, blockIdx.x);
  const int piece = piece_at(p, order_of(p, [](int tokens) { return tokens > 0 ? 1 : 0; }), blockIdx.x);
  return piece < 0 ? Work{} : work_of(p, piece);
}

template <int D, int W>
struct CSmem {
  static constexpr int kStep = D == 64 ? 32 : 16;  // keys of a tile a warp
  static constexpr int kKeys = W * kStep;          // of a tile
  static constexpr int kPlane = kKeys * D * 2;     // K or V of one
  static constexpr int kTiles = kStages * 2 * kPlane;
  static constexpr int kTotal = kTiles + 16 * D * 2;
  static_assert(W * 16 * D * 4 <= kTiles, "the warps' outputs reuse the tiles");
};

template <int D, typename O, int W, bool SORTED>
__global__ void __launch_bounds__(W * 32, W == 8 ? 1 : 12 / W) cross_kernel(const __grid_constant__ CrossArgs p) {
  using SM = CSmem<D, W>;
  constexpr int kKeys = SM::kKeys, KW = SM::kStep, NB = KW / 16, kThreads = W * 32;
  constexpr int WP = sizeof(O) == 4 ? 3 : 2;  // parts of a weight
  constexpr int PF = D + 4, PPR = D / 8;
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ float s_m[W][16], s_l[W][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  const Work w = few_work<SORTED>(p);
  const int nq = p.group * p.tokens;  // query rows of the (sequence, key head)
  const int lo = w.sp * p.split_len;
  const int hi = min(keys_of_rows(p, w, 0, nq), lo + p.split_len);
  const bf16 *K = static_cast<const bf16 *>(p.k) + w.s * p.ks + w.kvh * p.kh;
  const bf16 *V = static_cast<const bf16 *>(p.v) + w.s * p.ks + w.kvh * p.kh;
  unsigned char *sq = dyn + SM::kTiles;

  // each warp loads the keys of a tile that it works on, and waits for no other
  auto load_tile = [&](int k0, int st) {
    unsigned char *s = dyn + st * 2 * SM::kPlane;
#pragma unroll
    for (int e = lane; e < KW * PPR; e += 32) {
      const int r = warp * KW + e / PPR, c = e % PPR;
      const bool on = k0 + r < hi;
      const long long at = (on ? (k0 + r) * p.kt : 0) + c * 8;
      cp_async16_zfill(s + at16<D>(r, c), K + at, on);
      cp_async16_zfill(s + SM::kPlane + at16<D>(r, c), V + at, on);
    }
  };

  float o[D / 8][4];
#pragma unroll
  for (int x = 0; x < D / 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
  float m[2] = {kNoKey, kNoKey}, l[2] = {0.f, 0.f};
  if (lo < hi) {
    for (int e = tid; e < 16 * PPR; e += kThreads) {
      const int r = e / PPR, c = e % PPR;
      const Row x = row_of(p, w.kvh, min(r, nq - 1));
      const bool on = r < nq && x.token < w.qlen;
      cp_async16_zfill(sq + at16<D>(r, c),
                       static_cast<const bf16 *>(p.q) + w.s * p.qs +
                           (on ? x.token * p.qt + x.head * p.qh : 0) + c * 8, on);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
    for (int st = 0; st < kStages; ++st) {
      if (lo + st * kKeys < hi) load_tile(lo + st * kKeys, st);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    int seen[2];  // keys that the thread's two rows see
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = (lane >> 2) + 8 * j;
      seen[j] = r < nq ? keys_seen(p, w, row_of(p, w.kvh, r).token) : 0;
    }
    // fragment addresses: which row and piece of a 16 x 16 block a lane names
    const int mi = lane >> 3, mr = lane & 7;
    const uint32_t q_base = smem_u32(sq), t_base = smem_u32(dyn);
    const int q_row = (mi & 1) * 8 + mr, q_pc = mi >> 1;
    const int k_row = warp * KW + (mi >> 1) * 8 + mr, k_pc = mi & 1;
    const int v_row = warp * KW + (mi & 1) * 8 + mr, v_pc = mi >> 1;
    int st = 0;
    for (int k0 = lo; k0 < hi; k0 += kKeys) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      if (k0 == lo) __syncthreads();  // the queries are everyone's
      else __syncwarp();
      const uint32_t kb = t_base + st * 2 * SM::kPlane, vb = kb + SM::kPlane;
      float s[2 * NB][4] = {};
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t qa[4];
        ldm4(qa, q_base + at16<D>(q_row, 2 * ks + q_pc));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          uint32_t f[4];
          ldm4(f, kb + at16<D>(k_row + nb * 16, 2 * ks + k_pc));
          mma_bf16(s[2 * nb], qa, f[0], f[1]);
          mma_bf16(s[2 * nb + 1], qa, f[2], f[3]);
        }
      }
      // weights of rows lane / 4 (j = 0) and lane / 4 + 8 (j = 1); keys of this
      // warp's part that count for either
      const int left[2] = {min(seen[0], hi) - k0 - warp * KW, min(seen[1], hi) - k0 - warp * KW};
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < 2 * NB; ++x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = x * 8 + (lane & 3) * 2 + (e & 1);
          s[x][e] = key < left[e >> 1] ? s[x][e] * p.qscale : -INFINITY;
          mx[e >> 1] = fmaxf(mx[e >> 1], s[x][e]);
        }
      }
      float f[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xFFFFFFFFu, mx[j], 1));
        mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xFFFFFFFFu, mx[j], 2));
        const float mn = fmaxf(m[j], mx[j]);
        f[j] = mn == m[j] ? 1.f : ex2_approx(m[j] - mn);
        m[j] = mn;
        l[j] *= f[j];
      }
      if (__any_sync(0xFFFFFFFFu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
        for (int x = 0; x < D / 8; ++x) {
          o[x][0] *= f[0];
          o[x][1] *= f[0];
          o[x][2] *= f[1];
          o[x][3] *= f[1];
        }
      }
      uint32_t pf[NB][WP][4];
#pragma unroll
      for (int x = 0; x < 2 * NB; ++x) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          // (a key that does not count has a score of -inf)
          const float w0 = ex2_approx(s[x][2 * j] - m[j]);
          const float w1 = ex2_approx(s[x][2 * j + 1] - m[j]);
          l[j] += w0 + w1;
          uint32_t pr[3];
          split2<false>(w0, w1, pr);
#pragma unroll
          for (int k = 0; k < WP; ++k) pf[x / 2][k][(x & 1) * 2 + j] = pr[k];
        }
      }
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {  // 16 channels at a time
        float t[2][4] = {};
        uint32_t vf[NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) ldm4t(vf[nb], vb + at16<D>(v_row + nb * 16, 2 * db + v_pc));
#pragma unroll
        for (int a = WP - 1; a >= 0; --a) {  // the small parts first
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma_bf16(t[0], pf[nb][a], vf[nb][0], vf[nb][1]);
            mma_bf16(t[1], pf[nb][a], vf[nb][2], vf[nb][3]);
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[2 * db + x][e] += t[x][e];
      }
      __syncwarp();  // the stage is rewritten
      const int next = k0 + kStages * kKeys;
      if (next < hi) load_tile(next, st);
      asm volatile("cp.async.commit_group;" ::: "memory");
      st = st + 1 == kStages ? 0 : st + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    l[j] += __shfl_xor_sync(0xFFFFFFFFu, l[j], 1);
    l[j] += __shfl_xor_sync(0xFFFFFFFFu, l[j], 2);
    if ((lane & 3) == 0) {
      s_m[warp][(lane >> 2) + 8 * j] = m[j];
      s_l[warp][(lane >> 2) + 8 * j] = l[j];
    }
  }
  __syncthreads();
  float *so = reinterpret_cast<float *>(dyn);  // [warp][16][D]
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = (lane >> 2) + 8 * j;
    if (r < nq) {
      float *to = so + (size_t)(warp * 16 + r) * D + (lane & 3) * 2;
#pragma unroll
      for (int x = 0; x < D / 8; ++x)
        *reinterpret_cast<float2 *>(to + x * 8) = make_float2(o[x][2 * j], o[x][2 * j + 1]);
    }
  }
  __syncthreads();
  // rows of D / 4 threads each: the warps joined
  for (int e = tid; e < nq * (D / 4); e += kThreads) {
    const int r = e / (D / 4), c = e % (D / 4);
    float mj = -INFINITY, lj = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) mj = fmaxf(mj, s_m[k][r]);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if (s_l[k][r] == 0.f) continue;
      const float fk = ex2_approx(s_m[k][r] - mj);
      const float4 u = *reinterpret_cast<const float4 *>(so + (size_t)(k * 16 + r) * D + c * 4);
      lj += s_l[k][r] * fk;
      v.x += u.x * fk, v.y += u.y * fk, v.z += u.z * fk, v.w += u.w * fk;
    }
    const Row x = row_of(p, w.kvh, r);
    if (x.token >= w.qlen) continue;
    const size_t row = ((size_t)w.s * p.heads + x.head) * p.tokens + x.token;
    if (p.splits > 1) {
      float *part = p.part + (row * p.splits + w.sp) * PF;
      *reinterpret_cast<float4 *>(part + c * 4) = v;
      if (c == 0) *reinterpret_cast<float2 *>(part + D) = make_float2(w.bad ? NAN : mj, lj);
    } else {
      const float inv = w.bad ? NAN : lj == 0.f ? 0.f : 1.f / lj;
      store4(static_cast<O *>(p.out) + w.s * p.os + x.token * p.ot + x.head * p.oh + c * 4,
             make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
      if (c == 0 && p.lse) p.lse[row] = w.bad ? NAN : lj == 0.f ? -INFINITY : (mj + log2f(lj)) * kLn2;
    }
  }
}

// fp32 queries and states, up to R query rows, without the tensor core: at 16
// rows the 4096 multiply-adds a key (32 cycles of an SM) still take less time
// than its 1024 bytes. A warp takes 32 keys at a time, a lane each: K and V rows
// go to shared memory (rows 16 bytes apart more, so that eight lanes' pieces
// spread over all banks); a lane makes its key's scores; then a lane has four
// channels (of 64: every second key) and all keys' weights.
template <int D, int R>
struct FSmem {
  static constexpr int kWarps = D == 128 ? 2 : 4;               // three CTAs an SM (R = 16: two)
  static constexpr int kRow = D * 4 + 16, kTile = 32 * kRow;   // bytes
  static constexpr int kWarp = 2 * kTile;                       // K, V
  static constexpr int kTotal = kWarps * kWarp + R * D * 4 + kWarps * R * 32 * 4;
  static_assert(R * D * 4 <= kWarp, "a warp's outputs reuse its tiles");
};
template <int D, int R, bool SORTED>
__global__ void __launch_bounds__(FSmem<D, R>::kWarps * 32) cross_few_kernel(const __grid_constant__ CrossArgs p) {
  using SM = FSmem<D, R>;
  constexpr int PF = D + 4, PPR = D / 4, kWarps = SM::kWarps, kThreads = kWarps * 32;
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ float s_m[kWarps][R], s_l[kWarps][R];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  const Work w = few_work<SORTED>(p);
  const int nq = p.group * p.tokens;
  const int lo = w.sp * p.split_len;
  const int hi = min(keys_of_rows(p, w, 0, nq), lo + p.split_len);
  const float *K = static_cast<const float *>(p.k) + w.s * p.ks + w.kvh * p.kh;
  const float *V = static_cast<const float *>(p.v) + w.s * p.ks + w.kvh * p.kh;
  unsigned char *sk = dyn + warp * SM::kWarp, *sv = sk + SM::kTile;
  float *sq = reinterpret_cast<float *>(dyn + kWarps * SM::kWarp);         // [R][D]
  float *sw = sq + R * D + warp * R * 32;                                  // [R][32] weights
  auto load_rows = [&](unsigned char *to, const float *from, int k0) {
#pragma unroll 8
    for (int e = lane; e < 32 * PPR; e += 32) {
      const int r = e / PPR, c = e % PPR;
      const bool on = k0 + r < hi;
      cp_async16_zfill(to + r * SM::kRow + c * 16, from + (on ? (k0 + r) * p.kt : 0) + c * 4, on);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float o[R][4], m[R], l[R];
  int seen[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    o[r][0] = o[r][1] = o[r][2] = o[r][3] = 0.f;
    m[r] = kNoKey;
    l[r] = 0.f;
    seen[r] = r < nq ? min(keys_seen(p, w, row_of(p, w.kvh, r).token), hi) : 0;
  }
  if (lo < hi) {
    int k0 = lo + warp * 32;
#pragma unroll
    for (int e = tid; e < R * PPR; e += kThreads) {
      const int r = e / PPR, c = e % PPR;
      const Row x = row_of(p, w.kvh, min(r, nq - 1));
      const bool on = r < nq && x.token < w.qlen;
      cp_async16_zfill(sq + e * 4, static_cast<const float *>(p.q) + w.s * p.qs +
                                       (on ? x.token * p.qt + x.head * p.qh : 0) + c * 4, on);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (k0 < hi) {
      load_rows(sk, K, k0);
      load_rows(sv, V, k0);
      asm volatile("cp.async.wait_group 2;" ::: "memory");
    } else {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncthreads();
    for (; k0 < hi; k0 += kWarps * 32) {
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      __syncwarp();
      float s[R];
#pragma unroll
      for (int r = 0; r < R; ++r) s[r] = 0.f;
      const float4 *row = reinterpret_cast<const float4 *>(sk + lane * SM::kRow);
#pragma unroll 4
      for (int c = 0; c < PPR; ++c) {
        const float4 kv = row[c];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float4 qv = reinterpret_cast<const float4 *>(sq + r * D)[c];
          s[r] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, s[r]))));
        }
      }
      __syncwarp();
      const int next = k0 + kWarps * 32;
      if (next < hi) load_rows(sk, K, next);
      else asm volatile("cp.async.commit_group;" ::: "memory");
#pragma unroll
      for (int r = 0; r < R; ++r) {
        s[r] = k0 + lane < seen[r] ? s[r] * p.qscale : -INFINITY;
        float mx = s[r];
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
        const float mn = fmaxf(m[r], mx), f = mn == m[r] ? 1.f : ex2_approx(m[r] - mn);
        m[r] = mn;
        const float e = ex2_approx(s[r] - mn);
        l[r] = l[r] * f + e;  // this lane's keys
        sw[r * 32 + lane] = e;
#pragma unroll
        for (int x = 0; x < 4; ++x) o[r][x] *= f;
      }
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      __syncwarp();
      // four channels a lane; heads of 64: lanes 16-31 take the odd keys
      constexpr int KS = 128 / D;
      const int first = lane / PPR, ch = lane % PPR;
      const int most = min(32, hi - k0);
#pragma unroll 4
      for (int j = first; j < most; j += KS) {
        const float4 vv = *reinterpret_cast<const float4 *>(sv + j * SM::kRow + ch * 16);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float wj = sw[r * 32 + j];
          o[r][0] = fmaf(wj, vv.x, o[r][0]);
          o[r][1] = fmaf(wj, vv.y, o[r][1]);
          o[r][2] = fmaf(wj, vv.z, o[r][2]);
          o[r][3] = fmaf(wj, vv.w, o[r][3]);
        }
      }
      __syncwarp();
      if (next < hi) load_rows(sv, V, next);
      else asm volatile("cp.async.commit_group;" ::: "memory");
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  }
  __syncwarp();
  // the warps joined through shared memory, each in its tiles' place
  float *so = reinterpret_cast<float *>(sk);  // [R][D]
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int x = 16; x >= 1; x >>= 1) l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], x);
    if (D == 64) {
#pragma unroll
      for (int x = 0; x < 4; ++x) o[r][x] += __shfl_xor_sync(0xFFFFFFFFu, o[r][x], 16);
    }
    if (lane == 0) s_m[warp][r] = m[r], s_l[warp][r] = l[r];
    if (lane < PPR)
      *reinterpret_cast<float4 *>(so + r * D + lane * 4) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
  }
  __syncthreads();
  for (int e = tid; e < nq * PPR; e += kThreads) {
    const int r = e / PPR, c = e % PPR;
    float mj = -INFINITY, lj = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) mj = fmaxf(mj, s_m[k][r]);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      if (s_l[k][r] == 0.f) continue;
      const float fk = ex2_approx(s_m[k][r] - mj);
      const float4 u = reinterpret_cast<const float4 *>(dyn + k * SM::kWarp)[r * PPR + c];
      lj += s_l[k][r] * fk;
      v.x += u.x * fk, v.y += u.y * fk, v.z += u.z * fk, v.w += u.w * fk;
    }
    const Row x = row_of(p, w.kvh, r);
    if (x.token >= w.qlen) continue;
    const size_t row = ((size_t)w.s * p.heads + x.head) * p.tokens + x.token;
    if (p.splits > 1) {
      float *part = p.part + (row * p.splits + w.sp) * PF;
      *reinterpret_cast<float4 *>(part + c * 4) = v;
      if (c == 0) *reinterpret_cast<float2 *>(part + D) = make_float2(w.bad ? NAN : mj, lj);
    } else {
      const float inv = w.bad ? NAN : lj == 0.f ? 0.f : 1.f / lj;
      store4(static_cast<float *>(p.out) + w.s * p.os + x.token * p.ot + x.head * p.oh + c * 4,
             make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
      if (c == 0 && p.lse) p.lse[row] = w.bad ? NAN : lj == 0.f ? -INFINITY : (mj + log2f(lj)) * kLn2;
    }
  }
}

// Joins a query's ranges: W warps a query, each a run of its ranges in order. What
// bounds it: its launch, and a read of what has just been written. 5 queries of 8
// heads in 147 ranges: the whole call takes 20.0 us, with eight warps a query that
// read maxima and sums before the rows 21.6, with one 31.
template <int D, typename O, int W>
__global__ void __launch_bounds__(W == 16 ? 512 : 256)
    cross_join_kernel(const CrossArgs p, long long rows) {
  constexpr int PF = D + 4, E = D / 32, ROWS = W == 16 ? 1 : 8 / W;
  __shared__ float s_acc[ROWS][W][D], s_ml[ROWS][W][2];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, w = warp % W, slot = warp / W;
  const long long row = (long long)blockIdx.x * ROWS + slot;
  const int token = (int)(row % p.tokens);
  const long long sh = row / p.tokens;
  const int h = (int)(sh % p.heads), s = (int)(sh / p.heads);
  const int qlen = row < rows ? p.qlen ? p.qlen[s] : p.tokens : 0;
  const bool live = token < qlen && qlen <= p.tokens;
  const int per = (p.splits + W - 1) / W, j0 = w * per, n = live ? min(per, p.splits - j0) : 0;
  const float *first = p.part + ((size_t)row * p.splits + j0) * PF;
  float m = -INFINITY, l = 0.f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  bool bad = false;
  // B ranges at a time: their rows, and their maxima and sums (a lane each)
  constexpr int B = W == 16 ? 16 : 8;
  for (int k0 = 0; k0 < n; k0 += B) {
    const int here = min(B, n - k0);
    float v[B][E];
#pragma unroll
    for (int u = 0; u < B; ++u)
      if (u < here) load_row<E>(first + (size_t)(k0 + u) * PF + lane * E, v[u]);
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < here) ml = *reinterpret_cast<const float2 *>(first + (size_t)(k0 + lane) * PF + D);
    bad |= __any_sync(0xFFFFFFFFu, ml.x != ml.x && ml.y == 0.f);
    float top = ml.y != 0.f ? ml.x : -INFINITY;
#pragma unroll
    for (int o = B / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    top = __shfl_sync(0xFFFFFFFFu, top, 0);
    const float mn = fmaxf(m, top), old = l == 0.f ? 0.f : ex2_approx(m - mn);
    const float f = ml.y == 0.f ? 0.f : ex2_approx(ml.x - mn);
    m = mn;
    float sum = ml.y * f;
#pragma unroll
    for (int o = B / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    l = l * old + __shfl_sync(0xFFFFFFFFu, sum, 0);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= old;
#pragma unroll
    for (int u = 0; u < B; ++u) {
      const float fu = __shfl_sync(0xFFFFFFFFu, f, u);
      if (u < here && fu != 0.f) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += v[u][e] * fu;
      }
    }
  }
  if (bad) l = NAN;
  if (W > 1) {  // the warps' parts, in order
#pragma unroll
    for (int e = 0; e < E; ++e) s_acc[slot][w][lane * E + e] = acc[e];
    if (lane == 0) s_ml[slot][w][0] = m, s_ml[slot][w][1] = l;
    __syncthreads();
    if (w > 0) return;
    float mn = -INFINITY;
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (s_ml[slot][i][1] != 0.f) mn = fmaxf(mn, s_ml[slot][i][0]);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float li = s_ml[slot][i][1], f = li == 0.f ? 0.f : ex2_approx(s_ml[slot][i][0] - mn);
      if (li == 0.f) continue;
      l += li * f;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += s_acc[slot][i][lane * E + e] * f;
    }
    m = mn;
  }
  if (!live) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  O *to = static_cast<O *>(p.out) + s * p.os + token * p.ot + h * p.oh + lane * E;
  if (E == 4)
    store4(to, make_float4(acc[0] * inv, acc[1] * inv, acc[2 % E] * inv, acc[3 % E] * inv));
  else if (sizeof(O) == 4)
    *reinterpret_cast<float2 *>(to) = make_float2(acc[0] * inv, acc[1] * inv);
  else
    *reinterpret_cast<uint32_t *>(to) = pack2(acc[0] * inv, acc[1] * inv);
  if (lane == 0 && p.lse) p.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int D, typename O, int W, bool SORTED>
cudaError_t launch_warps(const CrossArgs &a, int grid, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem_of(cross_kernel<D, O, W, SORTED>, CSmem<D, W>::kTotal, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(cross_kernel<D, O, W, SORTED>, grid, W * 32, CSmem<D, W>::kTotal, s, a);
}
// Twelve warps an SM as CTAs of two, whose starts and ends lie apart more, as
// soon as there are enough of them: one query of 64 x 32 heads over up to 300
// states takes 32 us, as CTAs of four 35, of one 37. Few CTAs of some length have
// eight: 32 heads over 300 states take 6.5 us, with four 6.7; over 1000 12.6 and 16.
template <int D, typename O>
cudaError_t launch_rows(const CrossArgs &a, int grid, cudaStream_t s) {
  if (grid >= 912)
    return a.sorted ? launch_warps<D, O, 2, true>(a, grid, s) : launch_warps<D, O, 2, false>(a, grid, s);
  if (grid <= 152 && a.split_len > 128) return launch_warps<D, O, 8, false>(a, grid, s);
  return a.sorted ? launch_warps<D, O, 4, true>(a, grid, s) : launch_warps<D, O, 4, false>(a, grid, s);
}
template <int D, int R, bool SORTED>
cudaError_t launch_few_of(const CrossArgs &a, int grid, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem_of(cross_few_kernel<D, R, SORTED>, FSmem<D, R>::kTotal, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(cross_few_kernel<D, R, SORTED>, grid, FSmem<D, R>::kWarps * 32, FSmem<D, R>::kTotal, s, a);
}
template <int D, int R>
cudaError_t launch_few(const CrossArgs &a, int grid, cudaStream_t s) {
  return a.sorted ? launch_few_of<D, R, true>(a, grid, s) : launch_few_of<D, R, false>(a, grid, s);
}

template <int D>
cudaError_t launch(const CrossArgs &a, const CrossPlan &pl, int dtype, int out_dtype, cudaStream_t s) {
  const long long grid = (long long)a.seqs * a.kv * a.tiles * a.splits;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  const int g = (int)grid, rows = a.group * a.tokens;
  cudaError_t e;
  if (pl.rows > 16) {
    e = out_dtype == HKV_BF16 ? launch_cross_tc(a, pl, D, s) : launch_cross_parts(a, D, dtype, s);
  } else if (dtype == HKV_BF16) {
    e = out_dtype == HKV_BF16 ? launch_rows<D, bf16>(a, g, s) : launch_rows<D, float>(a, g, s);
  } else {
    // (arithmetic for no more rows than twice those there: 7 rows of 12 x 9 key heads
    // of 64 over 253 states 14.2 -> 9.4 us, 6 of 17 x 8 of 128 over 333 37 -> 25.5)
    e = rows == 1   ? launch_few<D, 1>(a, g, s)
        : rows <= 4 ? launch_few<D, 4>(a, g, s)
        : rows <= 8 ? launch_few<D, 8>(a, g, s)
                    : launch_few<D, 16>(a, g, s);
  }
  if (e != cudaSuccess || a.splits == 1) return e;
  const long long queries = (long long)a.seqs * a.heads * a.tokens;
  const int warps = a.splits <= 8 ? 1 : a.splits <= 16 ? 2 : 16;  // a query
  const int blocks = (int)(warps == 16 ? queries : (queries * warps + 7) / 8);
  auto join = [&](auto *kernel) {
    return pdl_launch(kernel, blocks, warps == 16 ? 512 : 256, 0, s, a, queries);
  };
  if (out_dtype == HKV_BF16)
    return join(warps == 1 ? cross_join_kernel<D, bf16, 1>
                : warps == 2 ? cross_join_kernel<D, bf16, 2> : cross_join_kernel<D, bf16, 16>);
  return join(warps == 1 ? cross_join_kernel<D, float, 1>
              : warps == 2 ? cross_join_kernel<D, float, 2> : cross_join_kernel<D, float, 16>);
}

}  // namespace

// Key ranges for as many CTAs as the device holds at a time, once or several times
// over, each a multiple of 64 keys (with tiles of 96, a range's last one is partly
// empty). The 152 SMs are a constant here, so that the workspace a caller allocated
// does not depend on the device of the call.
CrossPlan cross_plan(int seqs, int heads, int kv, int tokens, int keys, int D, int dtype,
                     int out_dtype) {
  constexpr int kMostSplits = 456;
  CrossPlan pl;
  const long long all = (long long)(heads / kv) * tokens;
  const bool tc = all > 16 && out_dtype == HKV_BF16;
  pl.rows = all <= 16 ? 16 : tc && all > 128 ? 256 : 128;
  // CTAs that the device holds at a time, three, two or one an SM (9 to 16 fp32 rows: two,
  // counted as three here)
  const int ctas = pl.rows == 16 ? 456 : tc && pl.rows == 128 ? 304 : 152;
  // the tcgen05 kernel's query tiles: 128 tokens of a head, or all tokens of as
  // many heads of a group as fit 128 rows
  const int group = heads / kv;
  pl.box_tokens = tokens < 128 ? tokens : 128;
  pl.box_heads = 128 / pl.box_tokens < group ? 128 / pl.box_tokens : group;
  if (tc) {
    const long long units = (long long)((group + pl.box_heads - 1) / pl.box_heads) *
                            ((tokens + pl.box_tokens - 1) / pl.box_tokens);
    if (units == 1) pl.rows = 128;
    pl.tiles = (int)((units + pl.rows / 128 - 1) / (pl.rows / 128));
  } else {
    pl.tiles = (int)((all + pl.rows - 1) / pl.rows);
  }
  const long long base = (long long)seqs * kv * pl.tiles;
  // Rounds of CTAs, whose ranges are long enough that joining them pays. Few query
  // rows, whose partial results are small: one, or (ranges of 512 keys) four, so
  // that uneven ones even out. More: none, one or two, by the times below (in us):
  // two where the CTAs of one leave much of the device empty (fp32, 18 queries of 7 x
  // 77 heads on 11 over up to 6401 states, 77 CTAs: 140 -> 67 us; 1200 of 20 heads
  // over 8000, 100: 98 -> 87; four rounds 78 and 88).
  long long want = base < ctas ? ctas / base : 1;
  if (pl.rows == 16) {
    if (want > keys / 192) want = keys / 192;
    if (base < 4LL * ctas) {
      long long four = (4LL * ctas + base - 1) / base;
      if (four > keys / 512) four = keys / 512;
      if (want < four) want = four;
    }
  } else if (base < ctas) {
    const double start = tc ? 4 : 5;  // of a CTA; of 64 keys more:
    const double tile = !tc ? D / 64 * (dtype == HKV_FP32 ? 1.7 : 1.0) : pl.rows == 128 ? 0.5 : 0.8;
    const double part = (double)seqs * heads * tokens * (D + 4) * 8 / 4e6;  // written and read
    double least = start + keys / 64 * tile;
    want = 1;
    for (int rounds = 1; rounds <= 2; ++rounds) {
      long long n = rounds * (long long)ctas / base;
      if (n > keys / 256) n = keys / 256;
      if (n < 2) continue;
      const double us = rounds * (start + (double)keys / 64 / n * tile) + 2 + n * part;
      if (us < least) least = us, want = n;
    }
  }
  if (want > kMostSplits) want = kMostSplits;
  if (want < 1 || keys < 512) want = 1;
  pl.split_len = (int)(((keys + want - 1) / want + 63) / 64 * 64);
  pl.splits = (keys + pl.split_len - 1) / pl.split_len;
  // Where there are more CTAs than fit, by length: 16 x 577 padded queries of 20 heads
  // on 4 over up to 1025 states 35.6 -> 29.8 us; fp32, 16 x 257 over up to 777, 60 -> 49,
  // one query of 21 x 12 heads over up to 2861 in ranges 28.5 -> 23.6; but 0.3 more a
  // CTA (542 over up to 33: 56 -> 58.5).
  pl.sorted = seqs > 1 && seqs <= 32 && base * pl.splits > ctas &&
              (tc || keys >= (pl.rows == 16 ? 512 : 256));
  pl.part_bytes =
      pl.splits > 1 ? (size_t)seqs * heads * tokens * pl.splits * (D + 4) * sizeof(float) : 0;
  return pl;
}

cudaError_t launch_cross(const CrossArgs &a, const CrossPlan &pl, int D, int dtype, int out_dtype,
                         cudaStream_t s) {
  return D == 64 ? launch<64>(a, pl, dtype, out_dtype, s) : launch<128>(a, pl, dtype, out_dtype, s);
}

}  // namespace hkv
