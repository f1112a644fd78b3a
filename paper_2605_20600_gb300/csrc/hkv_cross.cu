// Attention of the tokens' queries over their sequence's states, or of a
// prompt's tokens over the tokens up to themselves.
//
// A CTA takes up to 16 MW queries of one (sequence, key head), the heads of the
// group one after the other, and a range of keys in tiles of 64; the ranges of
// one query are joined by a second kernel. cross_kernel (mma.sync m16n8k16): MW
// warps lie along the queries, 16 each, the others along the keys of a tile,
// joined in shared memory.
//
// Precision: bf16 queries, keys and values enter as they are; an fp32 element
// is three bf16 parts, and the six products of parts that reach past 2^-24 are
// taken, the small ones first. The weights are three parts for fp32 outs, which
// leaves nothing of them out, and two, off by 2^-18 of a weight, for bf16 outs,
// whose own rounding is 2^-9. Sums are fp32; products chain in the tensor core
// within a tile.
#include "hkv_cross.cuh"
#include "hkv_quant.cuh"

namespace hkv {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kKeys = 64;  // keys of a tile

template <typename T>
struct Planes {
  static constexpr int kN = 1, kStages = 2;
};
template <>
struct Planes<float> {
  static constexpr int kN = 3, kStages = 1;
};

template <int D, typename T, int MW>
struct CSmem {
  static constexpr int kRow = D * 2;                        // bytes of a bf16 row
  static constexpr int kPlane = kKeys * kRow;
  static constexpr int kStage = 2 * Planes<T>::kN * kPlane;  // K planes, V planes
  static constexpr int kQPlane = MW * 16 * kRow;
  static constexpr int kQ = Planes<T>::kN * kQPlane;
  static constexpr int kTiles = Planes<T>::kStages * kStage;
  static constexpr int kTotal = kTiles + kQ;
  static_assert(kWarps * 16 * D * 4 <= kTiles, "the warps' outputs reuse the tiles");
};

// A piece of 8 elements of a row (zeros where `on` is false) into the planes at
// dst. bf16: asynchronous.
template <typename T>
__device__ __forceinline__ void load_piece(unsigned char *dst, int plane, const T *from, bool on) {
  if (sizeof(T) == 2) {
    cp_async16_zfill(dst, from, on);
  } else {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (on) {
      Elem<float>::unpack(reinterpret_cast<const uint4 *>(from)[0], x);
      Elem<float>::unpack(reinterpret_cast<const uint4 *>(from)[1], x + 4);
    }
    uint32_t p[4][3];
#pragma unroll
    for (int j = 0; j < 4; ++j) split2<true>(x[2 * j], x[2 * j + 1], p[j]);
#pragma unroll
    for (int k = 0; k < 3; ++k)
      *reinterpret_cast<uint4 *>(dst + k * plane) = make_uint4(p[0][k], p[1][k], p[2][k], p[3][k]);
  }
}
// Rows [r0, r0 + rows) of a tile, those from `live` on as zeros, by the block
// or by each warp its own.
template <int D, typename T, int THREADS>
__device__ __forceinline__ void load_rows(unsigned char *dst, int plane, const T *src,
                                          long long stride, int r0, int rows, int live) {
  constexpr int PPR = D / 8;
  for (int e = threadIdx.x % THREADS; e < rows * PPR; e += THREADS) {
    const int r = r0 + e / PPR, c = e % PPR;
    const bool on = r < live;
    load_piece<T>(dst + at16<D>(r, c), plane, src + (on ? r * stride : 0) + c * 8, on);
  }
}

template <int D, typename T, typename O, int MW>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : MW == 1 ? 3 : 2)
    cross_kernel(const CrossArgs p) {
  using SM = CSmem<D, T, MW>;
  constexpr int NP = Planes<T>::kN, STAGES = Planes<T>::kStages;
  constexpr int WP = sizeof(O) == 4 ? 3 : 2;         // parts of a weight
  constexpr int KW = kWarps / MW, NKW = kKeys / KW;  // keys of a tile per warp
  constexpr int PF = D + 4;
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ float s_m[kWarps][16], s_l[kWarps][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int mw = warp % MW, kw = warp / MW;
  pdl_wait();
  pdl_launch_dependents();
  const Work w = work_of(p);
  const int all = p.group * p.tokens;                // query rows of the (sequence, key head)
  const int r0 = w.tile * MW * 16, nq = min(MW * 16, all - r0);
  const int lo = w.sp * p.split_len;
  const int hi = min(keys_of_rows(p, w, r0, r0 + nq), lo + p.split_len);
  const T *K = static_cast<const T *>(p.k) + w.s * p.ks + w.kvh * p.kh;
  const T *V = static_cast<const T *>(p.v) + w.s * p.ks + w.kvh * p.kh;
  unsigned char *sq = dyn + SM::kTiles;

  // a tile's rows: with one warp of queries each warp loads the keys that it
  // works on, and waits for no other
  constexpr bool ALONE = MW == 1 && STAGES > 1;
  auto load_tile = [&](int k0, int st) {
    unsigned char *s = dyn + st * SM::kStage;
    constexpr int FIRST = ALONE ? 32 : kThreads;
    const int r0 = ALONE ? kw * NKW : 0, n = ALONE ? NKW : kKeys;
    load_rows<D, T, FIRST>(s, SM::kPlane, K + k0 * p.kt, p.kt, r0, n, hi - k0);
    load_rows<D, T, FIRST>(s + NP * SM::kPlane, SM::kPlane, V + k0 * p.kt, p.kt, r0, n, hi - k0);
  };
  auto together = [&] {
    if (ALONE) __syncwarp();
    else __syncthreads();
  };

  float o[D / 8][4];
#pragma unroll
  for (int x = 0; x < D / 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
  float m[2] = {kNoKey, kNoKey}, l[2] = {0.f, 0.f};
  if (lo < hi) {
    for (int e = tid; e < MW * 16 * (D / 8); e += kThreads) {
      const int r = e / (D / 8), c = e % (D / 8);
      const Row x = row_of(p, w.kvh, r0 + min(r, nq - 1));
      const bool on = r < nq && x.token < w.qlen;
      load_piece<T>(sq + at16<D>(r, c), SM::kQPlane,
                    static_cast<const T *>(p.q) + w.s * p.qs +
                        (on ? x.token * p.qt + x.head * p.qh : 0) + c * 8, on);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (STAGES > 1) {
#pragma unroll
      for (int st = 0; st < STAGES; ++st) {
        if (lo + st * kKeys < hi) load_tile(lo + st * kKeys, st);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
    // fragment addresses: which row and piece of a 16 x 16 block a lane names
    int seen[2];  // keys that the thread's two rows see
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = r0 + mw * 16 + (lane >> 2) + 8 * j;
      seen[j] = r < r0 + nq ? keys_seen(p, w, row_of(p, w.kvh, r).token) : 0;
    }
    const int mi = lane >> 3, mr = lane & 7;
    const uint32_t q_base = smem_u32(sq), t_base = smem_u32(dyn);
    const int q_row = mw * 16 + (mi & 1) * 8 + mr, q_pc = mi >> 1;
    const int k_row = kw * NKW + (mi >> 1) * 8 + mr, k_pc = mi & 1;
    const int v_row = kw * NKW + (mi & 1) * 8 + mr, v_pc = mi >> 1;
    int st = 0;
    for (int k0 = lo; k0 < hi; k0 += kKeys) {
      if (STAGES == 1) {
        __syncthreads();  // the tile before this one has been read
        load_tile(k0, 0);
      } else {
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      }
      if (ALONE && k0 == lo) __syncthreads();  // the queries are everyone's
      else together();
      const uint32_t kb = t_base + st * SM::kStage, vb = kb + NP * SM::kPlane;
      float s[NKW / 8][4];
#pragma unroll
      for (int x = 0; x < NKW / 8; ++x) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.f;
      if (NP == 1) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t qa[4];
          ldm4(qa, q_base + at16<D>(q_row, 2 * ks + q_pc));
#pragma unroll
          for (int nb = 0; nb < NKW / 16; ++nb) {
            uint32_t f[4];
            ldm4(f, kb + at16<D>(k_row + nb * 16, 2 * ks + k_pc));
            mma_bf16(s[2 * nb], qa, f[0], f[1]);
            mma_bf16(s[2 * nb + 1], qa, f[2], f[3]);
          }
        }
      } else {
        // parts (2,0) (1,1) (0,2), then (1,0) (0,1), then (0,0)
#pragma unroll
        for (int order = 2; order >= 0; --order) {
#pragma unroll 1
          for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
            for (int a = order; a >= 0; --a) {
              uint32_t qa[4];
              ldm4(qa, q_base + a * SM::kQPlane + at16<D>(q_row, 2 * ks + q_pc));
#pragma unroll
              for (int nb = 0; nb < NKW / 16; ++nb) {
                uint32_t f[4];
                ldm4(f, kb + (order - a) * SM::kPlane + at16<D>(k_row + nb * 16, 2 * ks + k_pc));
                mma_bf16(s[2 * nb], qa, f[0], f[1]);
                mma_bf16(s[2 * nb + 1], qa, f[2], f[3]);
              }
            }
          }
        }
      }
      // weights of rows lane / 4 (j = 0) and lane / 4 + 8 (j = 1)
      // keys of this warp's part that count for either row
      const int left[2] = {min(seen[0], hi) - k0 - kw * NKW, min(seen[1], hi) - k0 - kw * NKW};
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < NKW / 8; ++x) {
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
      uint32_t pf[NKW / 16][WP][4];
#pragma unroll
      for (int x = 0; x < NKW / 8; ++x) {
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
      // 16 DBS channels at a time: 2 DBS chains of products side by side
      constexpr int DBS = 1;
#pragma unroll
      for (int db = 0; db < D / 16; db += DBS) {
        float t[2 * DBS][4] = {};
#pragma unroll
        for (int plane = NP - 1; plane >= 0; --plane) {  // parts of V, the small ones first
          uint32_t vf[DBS][NKW / 16][4];
#pragma unroll
          for (int x = 0; x < DBS; ++x)
#pragma unroll
            for (int kk = 0; kk < NKW / 16; ++kk)
              ldm4t(vf[x][kk],
                    vb + plane * SM::kPlane + at16<D>(v_row + kk * 16, 2 * (db + x) + v_pc));
#pragma unroll
          for (int a = WP - 1 - plane; a >= 0; --a) {  // parts of w
#pragma unroll
            for (int kk = 0; kk < NKW / 16; ++kk) {
#pragma unroll
              for (int x = 0; x < DBS; ++x) {
                mma_bf16(t[2 * x], pf[kk][a], vf[x][kk][0], vf[x][kk][1]);
                mma_bf16(t[2 * x + 1], pf[kk][a], vf[x][kk][2], vf[x][kk][3]);
              }
            }
          }
        }
#pragma unroll
        for (int x = 0; x < 2 * DBS; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[2 * db + x][e] += t[x][e];
      }
      if (STAGES > 1) {
        together();  // the stage is rewritten
        const int next = k0 + STAGES * kKeys;
        if (next < hi) load_tile(next, st);
        asm volatile("cp.async.commit_group;" ::: "memory");
        st = st + 1 == STAGES ? 0 : st + 1;
      }
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
    if (mw * 16 + r < nq) {
      float *to = so + (size_t)(warp * 16 + r) * D + (lane & 3) * 2;
#pragma unroll
      for (int x = 0; x < D / 8; ++x)
        *reinterpret_cast<float2 *>(to + x * 8) = make_float2(o[x][2 * j], o[x][2 * j + 1]);
    }
  }
  __syncthreads();
  // rows of D / 4 threads each: the warps along the keys joined
  for (int e = tid; e < nq * (D / 4); e += kThreads) {
    const int r = e / (D / 4), c = e % (D / 4), w0 = r >> 4, rr = r & 15;
    float mj = -INFINITY, lj = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) mj = fmaxf(mj, s_m[w0 + k * MW][rr]);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const int wk = w0 + k * MW;
      if (s_l[wk][rr] == 0.f) continue;
      const float fk = ex2_approx(s_m[wk][rr] - mj);
      const float4 u = *reinterpret_cast<const float4 *>(so + (size_t)(wk * 16 + rr) * D + c * 4);
      lj += s_l[wk][rr] * fk;
      v.x += u.x * fk, v.y += u.y * fk, v.z += u.z * fk, v.w += u.w * fk;
    }
    const Row x = row_of(p, w.kvh, r0 + r);
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

// Joins a query's ranges: W warps a query, each a run of its ranges in order.
constexpr int kJoinThreads = 256;
template <int D, typename O, int W>
__global__ void __launch_bounds__(kJoinThreads)
    cross_join_kernel(const CrossArgs p, long long rows) {
  constexpr int PF = D + 4, E = D / 32, ROWS = kJoinThreads / 32 / W;
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
  // the ranges' maxima and sums, a lane each, 32 at a time; then their rows, a
  // few on the way at a time
  for (int k0 = 0; k0 < n; k0 += 32) {
    const int here = min(32, n - k0);
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < here) ml = *reinterpret_cast<const float2 *>(first + (size_t)(k0 + lane) * PF + D);
    bad |= __any_sync(0xFFFFFFFFu, ml.x != ml.x && ml.y == 0.f);
    float top = ml.y != 0.f ? ml.x : -INFINITY;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float mn = fmaxf(m, top), old = l == 0.f ? 0.f : ex2_approx(m - mn);
    const float f = ml.y == 0.f ? 0.f : ex2_approx(ml.x - mn);
    m = mn;
    float sum = ml.y * f;
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    l = l * old + sum;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= old;
    constexpr int B = 8;
    for (int j = 0; j < here; j += B) {
      float v[B][E];
#pragma unroll
      for (int u = 0; u < B; ++u)
        if (j + u < here) load_row<E>(first + (size_t)(k0 + j + u) * PF + lane * E, v[u]);
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const float fj = __shfl_sync(0xFFFFFFFFu, f, (j + u) & 31);
        if (j + u < here && fj != 0.f) {
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] += v[u][e] * fj;
        }
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

template <int D, typename T, typename O, int MW>
cudaError_t launch_tiles(const CrossArgs &a, int grid, cudaStream_t s) {
  constexpr int smem = CSmem<D, T, MW>::kTotal;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem_of(cross_kernel<D, T, O, MW>, smem, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(cross_kernel<D, T, O, MW>, grid, kThreads, smem, s, a);
}

template <int D, typename T, typename O>
cudaError_t launch_rows(const CrossArgs &a, const CrossPlan &pl, cudaStream_t s) {
  const long long grid = (long long)a.seqs * a.kv * a.tiles * a.splits;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  cudaError_t e;
  if constexpr (sizeof(O) == 2) {  // (more than 16 rows are the tcgen05 kernel's)
    e = pl.rows >= 128 ? launch_cross_tc(a, pl, D, s) : launch_tiles<D, T, O, 1>(a, (int)grid, s);
  } else {
    if (pl.rows == 16) e = launch_tiles<D, T, O, 1>(a, (int)grid, s);
    else if (pl.rows == 32) e = launch_tiles<D, T, O, 2>(a, (int)grid, s);
    else e = launch_tiles<D, T, O, 4>(a, (int)grid, s);
  }
  if (e != cudaSuccess || a.splits == 1) return e;
  // a warp a query, or eight where there are many ranges
  const long long rows = (long long)a.seqs * a.heads * a.tokens;
  if (a.splits > 16)
    return pdl_launch(cross_join_kernel<D, O, 8>, (int)rows, kJoinThreads, 0, s, a, rows);
  return pdl_launch(cross_join_kernel<D, O, 1>, (int)((rows + 7) / 8), kJoinThreads, 0, s, a, rows);
}

}  // namespace

// As many key ranges as fill the device twice over (2 CTAs an SM), each a whole
// number of tiles. The 152 SMs are a constant here, so that the workspace a
// caller allocated does not depend on the device of the call.
CrossPlan cross_plan(int seqs, int heads, int kv, int tokens, int keys, int D, int dtype,
                     int out_dtype) {
  constexpr int kMostSplits = 456;
  CrossPlan pl;
  const long long all = (long long)(heads / kv) * tokens;
  const bool tc = dtype == HKV_BF16 && out_dtype == HKV_BF16 && all > 16;
#ifdef HKV_TC_ROWS
  if (tc) pl.rows = HKV_TC_ROWS;
#else
  if (tc) pl.rows = all > 128 ? 256 : 128;
#endif
  else pl.rows = all <= 16 ? 16 : all <= 32 ? 32 : 64;
  const int tile = tc ? 128 : kKeys;
  const int ctas = pl.rows == 256 ? 152 : pl.rows == 16 && dtype == HKV_BF16 ? 456 : dtype == HKV_BF16 ? 304 : 152;
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
  // several rounds of CTAs, or one, and no range that takes less time than its
  // partial result is worth
  constexpr int kLeast = 512;
  long long want = base < ctas ? ctas / base : 1;
  if (pl.rows == 16 && base >= ctas && base < 4LL * ctas) want = (4LL * ctas + base - 1) / base;
  if (want > kMostSplits) want = kMostSplits;
  if (want > keys / kLeast) want = keys / kLeast;
  if (want < 1) want = 1;
  pl.split_len = (int)(((keys + want - 1) / want + tile - 1) / tile * tile);
  pl.splits = (keys + pl.split_len - 1) / pl.split_len;
  pl.part_bytes =
      pl.splits > 1 ? (size_t)seqs * heads * tokens * pl.splits * (D + 4) * sizeof(float) : 0;
  return pl;
}

cudaError_t launch_cross(const CrossArgs &a, const CrossPlan &pl, int D, int dtype, int out_dtype,
                         cudaStream_t s) {
  if (dtype == HKV_BF16 && out_dtype == HKV_BF16)
    return D == 64 ? launch_rows<64, __nv_bfloat16, __nv_bfloat16>(a, pl, s)
                   : launch_rows<128, __nv_bfloat16, __nv_bfloat16>(a, pl, s);
  cudaError_t e = cudaErrorInvalidValue;
  HKV_DISPATCH(D, dtype, e = (launch_rows<kD, kT, float>(a, pl, s)));
  return e;
}

}  // namespace hkv
