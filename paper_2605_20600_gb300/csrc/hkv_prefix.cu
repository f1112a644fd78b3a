// Attention of a batch over prompts that its sequences share: every prompt
// row serves all sequences of its group.
//
// A CTA takes the queries of one (group, head) and a range of the prompt's
// keys, in tiles of 64 keys; the ranges of one prompt are joined by a second
// kernel. bf16 batches of more than 16 sequences a group and more than a few
// tiles go to tcgen05 (prefix_tc_kernel). Up to 16 queries, which fill an eighth
// of a tcgen05 product's rows, small batches, and fp32, whose six products of
// parts would not leave room in TMEM, are prefix_kernel's (mma.sync m16n8k16):
// MW warps lie along the queries, 16 each, the others along the keys of a tile,
// joined in shared memory.
//
// Precision: bf16 queries, keys and values enter as they are, and the weights
// as three bf16 parts (24 bits); an fp32 element is three parts as well, and
// the six products of parts that reach past 2^-24 are taken, the small ones
// first. Sums are fp32; products chain in the tensor core within a tile
// (prefix_kernel) or a range (O of prefix_tc_kernel).
//
// What bounds it: the chain of one tile (scores, weights, output, with a wait
// between any two), about 2 us a tile, and the start and the join around it.
// 32 heads x 4099 keys of 128 channels, 64 queries: 29 us, of which DRAM (67 MB)
// needs 10, and 128 queries 39; 20 heads, two prompts of 1000 and 667 keys of 64
// channels: 12 us; fp32, 8 heads x 777 keys, 5 queries: 10 us, and 32 heads x 4099
// keys of 128 channels, 64 queries: 259 us (100 TFLOP/s of bf16 products: its
// tiles are loaded and split between two barriers, with nothing in flight during
// the products, by one CTA an SM). One launch with the ranges of a
// prompt in a cluster, joined through distributed shared memory, took 18 us
// for the second, 15 for two launches then (a cluster waits for room for all its
// CTAs, and half of its warps wait while the others join).
#include "hkv_mma.cuh"
#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_select.cuh"
#include "hkv_tcgen05.cuh"

namespace hkv {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kKeys = 64;       // keys of a tile
constexpr int kMostSplits = 32; // key ranges of a prompt: a lane each in the join
constexpr float kLn2 = 0.6931471805599453f;

template <typename T>
struct Parts {
  static constexpr int kPlanes = 1, kStages = 2;
};
template <>
struct Parts<float> {
  static constexpr int kPlanes = 3, kStages = 1;
};

template <int D, typename T, int MW>
struct PSmem {
  static constexpr int kRow = D * 2;                            // bytes of a bf16 row
  static constexpr int kPlane = kKeys * kRow;
  static constexpr int kStage = 2 * Parts<T>::kPlanes * kPlane;  // K planes, V planes
  static constexpr int kQPlane = MW * 16 * kRow;
  static constexpr int kQ = Parts<T>::kPlanes * kQPlane;
  static constexpr int kTiles = Parts<T>::kStages * kStage;
  static constexpr int kTotal = kTiles + kQ;
  static_assert(kWarps * 16 * D * 4 <= kTiles, "the warps' outputs reuse the tiles");
};

// Copies `rows` rows of D elements into the planes at dst (row stride as
// at16), rows from `live` on as zeros. bf16: asynchronous.
template <int D, typename T, int THREADS>
__device__ __forceinline__ void load_rows(unsigned char *dst, int plane, const T *src,
                                          long long stride, int rows, int live) {
  constexpr int PPR = D / 8;
  for (int e = threadIdx.x; e < rows * PPR; e += THREADS) {
    const int r = e / PPR, c = e % PPR;
    const bool on = r < live;
    const T *from = src + (on ? r * stride : 0) + c * 8;
    if (sizeof(T) == 2) {
      cp_async16_zfill(dst + at16<D>(r, c), from, on);
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
        *reinterpret_cast<uint4 *>(dst + k * plane + at16<D>(r, c)) =
            make_uint4(p[0][k], p[1][k], p[2][k], p[3][k]);
    }
  }
}

template <int D, typename T, int MW>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1)
    prefix_kernel(const PrefixArgs p, int split_len) {
  using SM = PSmem<D, T, MW>;
  constexpr int NP = Parts<T>::kPlanes, STAGES = Parts<T>::kStages;
  constexpr int KW = kWarps / MW, NKW = kKeys / KW;  // keys of a tile per warp
  constexpr int PF = D + 4;
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ float s_m[kWarps][16], s_l[kWarps][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int mw = warp % MW, kw = warp / MW;
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
  const int q0 = tile * MW * 16;                 // first sequence within the group
  const int nq = min(MW * 16, p.seqs - q0);
  const size_t qrow = ((size_t)g * p.seqs + q0) * p.heads + h;  // row of query q0; next: + heads
  const int lo = sp * split_len, hi = min(len, lo + split_len);
  const T *K = static_cast<const T *>(p.k) + g * p.gs + h * p.hs;
  const T *V = static_cast<const T *>(p.v) + g * p.gs + h * p.hs;
  unsigned char *sq = dyn + SM::kTiles;

  auto load_tile = [&](int k0, int st) {
    unsigned char *s = dyn + st * SM::kStage;
    load_rows<D, T, kThreads>(s, SM::kPlane, K + k0 * p.ts, p.ts, kKeys, hi - k0);
    load_rows<D, T, kThreads>(s + NP * SM::kPlane, SM::kPlane, V + k0 * p.ts, p.ts, kKeys, hi - k0);
  };

  float o[D / 8][4];
#pragma unroll
  for (int x = 0; x < D / 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
  float m[2] = {kNoKey, kNoKey}, l[2] = {0.f, 0.f};
  if (lo < hi) {
    load_rows<D, T, kThreads>(sq, SM::kQPlane, static_cast<const T *>(p.q) + qrow * D,
                    (long long)p.heads * D, MW * 16, nq);
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (STAGES > 1) {
#pragma unroll
      for (int st = 0; st < STAGES; ++st) {
        if (lo + st * kKeys < hi) load_tile(lo + st * kKeys, st);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
    // fragment addresses: which row and piece of a 16 x 16 block a lane names
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
      __syncthreads();
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
      const int left = hi - k0 - kw * NKW;  // keys of this warp's part that count
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < NKW / 8; ++x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = x * 8 + (lane & 3) * 2 + (e & 1);
          s[x][e] = key < left ? s[x][e] * p.qscale : -INFINITY;
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
      uint32_t pf[NKW / 16][3][4];
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
          for (int k = 0; k < 3; ++k) pf[x / 2][k][(x & 1) * 2 + j] = pr[k];
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
          for (int a = 2 - plane; a >= 0; --a) {  // parts of w
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
        __syncthreads();  // the stage is rewritten
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
  for (int x = 0; x < D / 8; ++x) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      *reinterpret_cast<float2 *>(
          so + (size_t)(warp * 16 + (lane >> 2) + 8 * j) * D + x * 8 + (lane & 3) * 2) =
          make_float2(o[x][2 * j], o[x][2 * j + 1]);
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
      const int w = w0 + k * MW;
      if (s_l[w][rr] == 0.f) continue;
      const float fk = ex2_approx(s_m[w][rr] - mj);
      const float4 u = *reinterpret_cast<const float4 *>(so + (size_t)(w * 16 + rr) * D + c * 4);
      lj += s_l[w][rr] * fk;
      v.x += u.x * fk, v.y += u.y * fk, v.z += u.z * fk, v.w += u.w * fk;
    }
    const size_t row = qrow + (size_t)r * p.heads;
    if (p.splits > 1) {
      float *part = p.part + (row * p.splits + sp) * PF;
      *reinterpret_cast<float4 *>(part + c * 4) = v;
      if (c == 0) *reinterpret_cast<float2 *>(part + D) = make_float2(bad ? NAN : mj, lj);
    } else {
      const float inv = bad ? NAN : lj == 0.f ? 0.f : 1.f / lj;
      *reinterpret_cast<float4 *>(p.out + row * D + c * 4) =
          make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
      if (c == 0) p.lse[row] = bad ? NAN : lj == 0.f ? -INFINITY : (mj + log2f(lj)) * kLn2;
    }
  }
}

// Batches: up to 128 queries of one (group, head) a CTA, on tcgen05. Per tile of
// 64 keys: S = Q K^T into TMEM; a thread per query reads its row of S, makes the
// weights and writes them back as three bf16 parts, the A operand of O += W V.
// O stays in TMEM; a query's reference maximum moves (and O and its sum are
// rescaled) only when a tile's maximum is more than 2^8 above it, so that the
// weights stay below 2^8. The copies of the next tile run meanwhile, and two
// CTAs an SM fill each other's waits. Up to 64 queries (TWO): the rows hold them
// twice, and each copy takes half of a tile's keys (its weights of the other
// half are zero), so that all four warps have work; the copies are joined at the
// end.
constexpr int kTcQueries = 128, kTcThreads = 128;
constexpr int kTcCols = 256, kTcP = 0, kTcO = 128;  // TMEM: S and the parts of W, then O

template <int D>
struct TcSmem {
  static constexpr int kQ = kTcQueries * D * 2, kTile = kKeys * D * 2;
  static_assert(64 * (D + 4) * 4 <= 4 * kTile, "the second copies' results take the tiles' place");
  // 1024-byte aligned tiles; no less than 80 KB, so that at most two CTAs, and
  // with them their TMEM, fit an SM
  static constexpr int kUsed = kQ + 4 * kTile + 1024;
  static constexpr int kTotal = kUsed > 80 * 1024 ? kUsed : 80 * 1024;
};

// ROWS rows of D elements as column blocks of 128 bytes, 128-byte swizzle; the
// source's rows repeat after PERIOD, those from `live` on read as zero
template <int D, int ROWS, int PERIOD>
__device__ __forceinline__ void tc_load_rows(unsigned char *dst, const __nv_bfloat16 *src,
                                             long long stride, int live) {
  constexpr int PPR = D / 8, STEP = kTcThreads / PPR;  // pieces a row, rows a pass
  const int c = threadIdx.x % PPR, r0 = threadIdx.x / PPR;
  unsigned char *to = dst + (c >> 3) * ROWS * 128 + r0 * 128;
#pragma unroll 8
  for (int i = 0; i < ROWS / STEP; ++i) {
    const int r = r0 + i * STEP, from = r % PERIOD;
    const bool on = from < live;
    cp_async16_zfill(to + i * STEP * 128 + (((c & 7) ^ (r & 7)) << 4),
                     src + (on ? from * stride : 0) + c * 8, on);
  }
}

template <int D, bool TWO>
__global__ void __launch_bounds__(kTcThreads, 2)
    prefix_tc_kernel(const PrefixArgs p, int split_len) {
  using SM = TcSmem<D>;
  constexpr int PF = D + 4;
  extern __shared__ unsigned char dyn_raw[];
  __shared__ uint64_t s_bar[3];  // S ready, O ready; a failed CTA's products done
  __shared__ uint32_t s_tmem;
  unsigned char *dyn = dyn_raw + ((1024u - (smem_u32(dyn_raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, warp = tid >> 5;
  int b = blockIdx.x;
  const int tile = b % p.tiles;
  b /= p.tiles;
  const int h = b % p.heads;
  b /= p.heads;
  const int g = b % p.groups, sp = b / p.groups;
  if (tid == 0) {
    mbar_init(&s_bar[0], 1);
    mbar_init(&s_bar[1], 1);
    mbar_init(&s_bar[2], 1);
    fence_barrier_init();
  }
  // TMEM only after the wait, and the next kernel's CTAs only after TMEM: an
  // allocation waits for columns, so a CTA that held some while it waited for
  // the kernel before, or let a CTA of the kernel after take them first, could
  // wait for one that waits for it
  pdl_wait();
  if (warp == 0) {
    tmem_alloc(&s_tmem, kTcCols);
    pdl_launch_dependents();
  }
  int len = p.len[g];
  const bool bad = len < 0 || len > p.max_len;
  if (bad) {
    if (p.err && tid == 0 && sp == 0) set_err(p.err, HKV_ERR_BOUNDS);
    len = 0;
  }
  const int q0 = tile * kTcQueries, nq = min(kTcQueries, p.seqs - q0);
  const size_t qrow = ((size_t)g * p.seqs + q0) * p.heads + h;
  const int lo = sp * split_len, hi = min(len, lo + split_len);
  const __nv_bfloat16 *K = static_cast<const __nv_bfloat16 *>(p.k) + g * p.gs + h * p.hs;
  const __nv_bfloat16 *V = static_cast<const __nv_bfloat16 *>(p.v) + g * p.gs + h * p.hs;
  unsigned char *sq = dyn, *skv = dyn + SM::kQ;  // [stage][K, V]
  auto load_tile = [&](int k0, int st) {
    unsigned char *s = skv + st * 2 * SM::kTile;
    tc_load_rows<D, kKeys, kKeys>(s, K + k0 * p.ts, p.ts, hi - k0);
    tc_load_rows<D, kKeys, kKeys>(s + SM::kTile, V + k0 * p.ts, p.ts, hi - k0);
  };
  if (lo < hi) {
    tc_load_rows<D, kTcQueries, TWO ? 64 : kTcQueries>(
        sq, static_cast<const __nv_bfloat16 *>(p.q) + qrow * D, (long long)p.heads * D, nq);
    load_tile(lo, 0);
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem, mine = tmem + ((uint32_t)(warp * 32) << 16);
  const int first = TWO ? (warp & 1) * 32 : warp * 32;   // the warp's first query
  const bool works = first < nq;
  constexpr int CH = TWO ? 1 : 2;                       // 32 keys of a tile at a time
  const int key0 = TWO ? (warp >> 1) * 32 : 0;          // the row's keys of a tile
  float m = -INFINITY, l = 0.f;
  bool ok = true;
  uint32_t phase = 0;
  int st = 0;
  // a wait that runs out in one warp ends the loop for all, at one of its barriers
  for (int k0 = lo; k0 < hi; k0 += kKeys, phase ^= 1, st ^= 1) {
    // O holds the tiles before this one, and their stage is free
    if (k0 > lo) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_bar[1], phase ^ 1));
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    ok = !__syncthreads_or(!ok);
    if (!ok) break;
    const uint32_t kb = smem_u32(skv + st * 2 * SM::kTile), vb = kb + SM::kTile;
    if (tid == 0) {
      tc_fence_after();
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)  // 16 channels: 32 bytes of a column block
        tc_mma(tmem + kTcP,
               tc_desc(smem_u32(sq) + (ks >> 2) * kTcQueries * 128 + (ks & 3) * 32, 16),
               tc_desc(kb + (ks >> 2) * kKeys * 128 + (ks & 3) * 32, 16),
               tc_instr(kTcQueries, kKeys, false), ks > 0);
      tc_commit(&s_bar[0]);
    }
    if (k0 + kKeys < hi) load_tile(k0 + kKeys, st ^ 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_bar[0], phase));
#ifdef HKV_PREFIX_TEST_STALL  // one warp waits for a phase that nothing completes
    if (warp == (int)(blockIdx.x & 3) && k0 > lo)
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_bar[2], 0));
#endif
    tc_fence_after();
    if (works && ok) {
      uint32_t s[CH][32];
#pragma unroll
      for (int c = 0; c < CH; ++c) tmem_ld32(s[c], mine + kTcP + key0 + c * 32);
      tmem_wait_ld();
      const int left = hi - k0 - key0;  // keys that count, from the row's first on
      if (left < CH * 32) {
#pragma unroll
        for (int j = 0; j < CH * 32; ++j)
          if (j >= left) s[j >> 5][j & 31] = 0xFF800000u;  // -inf
      }
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < CH * 32; ++j) mx = fmaxf(mx, __uint_as_float(s[j >> 5][j & 31]));
      mx *= p.qscale;
      float f = 1.f;
      if (mx > m + 8.f) {
        f = ex2_approx(m - mx);  // (zero for the first keys)
        m = mx;
        l *= f;
      }
      const float ref = m == -INFINITY ? 0.f : m;  // no key yet: weights of zero
      if (k0 > lo && __any_sync(0xFFFFFFFFu, f != 1.f)) {
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          tmem_ld32(o, mine + kTcO + c);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
          tmem_st32(mine + kTcO + c, o);
        }
      }
      float l0 = 0.f, l1 = 0.f;
#pragma unroll
      for (int j0 = 0; j0 < CH * 32; j0 += 16) {  // 8 columns of each part at a time
        uint32_t w[3][8];
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const int a = j0 + j;
          const float w0 = ex2_approx(fmaf(__uint_as_float(s[a >> 5][a & 31]), p.qscale, -ref));
          const float w1 =
              ex2_approx(fmaf(__uint_as_float(s[a >> 5][(a & 31) + 1]), p.qscale, -ref));
          l0 += w0;
          l1 += w1;
          uint32_t part[3];
          split2<false>(w0, w1, part);
#pragma unroll
          for (int k = 0; k < 3; ++k) w[k][j / 2] = part[k];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) tmem_st8(mine + kTcP + k * 32 + (key0 + j0) / 2, w[k]);
      }
      l += l0 + l1;
      if (TWO) {
        const uint32_t zero[8] = {};
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int j0 = 0; j0 < 32; j0 += 16)
            tmem_st8(mine + kTcP + k * 32 + ((key0 ^ 32) + j0) / 2, zero);
      }
      tmem_wait_st();
    }
    tc_fence_before();
    ok = !__syncthreads_or(!ok);
    if (!ok) break;
    if (tid == 0) {
      tc_fence_after();
#pragma unroll
      for (int part = 2; part >= 0; --part)  // the small parts first
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
          tc_mma_ta(tmem + kTcO, tmem + kTcP + part * 32 + kk * 8,
                    tc_desc(vb + kk * 16 * 128, kKeys * 128), tc_instr(kTcQueries, D, true),
                    k0 > lo || part < 2 || kk > 0);
      tc_commit(&s_bar[1]);
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  // phase: that of the tile after the last
  if (ok && lo < hi) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&s_bar[1], phase ^ 1));
  ok = !__syncthreads_or(!ok);
  if (!ok) {
    // what was issued may still run: it gets the limit once more before its
    // operands' place and its TMEM are given back
    if (tid == 0) {
      set_err(p.err, HKV_ERR_TIMEOUT);
      tc_commit(&s_bar[2]);
    }
    mbar_wait(&s_bar[2], 0);
  }
  tc_fence_after();
  const bool wrong = bad || !ok, any = lo < hi && ok;
  // the two copies of a query joined: the second half of the rows hands its
  // result over (the tiles' place is free)
  float *so = reinterpret_cast<float *>(dyn + SM::kQ);  // [64][D + 4]
  float fa = 1.f, fb = 0.f;
  if (TWO) {
    if (warp >= 2 && works) {
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32] = {};
        if (any) {
          tmem_ld32(o, mine + kTcO + c);
          tmem_wait_ld();
        }
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          *reinterpret_cast<uint4 *>(so + (tid - 64) * PF + c + e) =
              make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
      *reinterpret_cast<float2 *>(so + (tid - 64) * PF + D) = make_float2(m, l);
    }
    __syncthreads();
    if (warp < 2 && works) {
      const float2 ml = *reinterpret_cast<const float2 *>(so + tid * PF + D);
      const float mn = fmaxf(m, ml.x);
      fa = l == 0.f ? 0.f : ex2_approx(m - mn);
      fb = ml.y == 0.f ? 0.f : ex2_approx(ml.x - mn);
      m = mn;
      l = l * fa + ml.y * fb;
    }
  }
  if (works && (!TWO || warp < 2)) {
    const float inv = p.splits > 1 ? 1.f : wrong ? NAN : l == 0.f ? 0.f : 1.f / l;
    const size_t row = qrow + (size_t)tid * p.heads;
    float *part = p.part + (row * p.splits + sp) * PF;
    float *to = p.splits > 1 ? part : p.out + row * D;
#pragma unroll 1
    for (int c = 0; c < D; c += 32) {
      uint32_t o[32] = {};
      if (any) {
        tmem_ld32(o, mine + kTcO + c);
        tmem_wait_ld();
      }
      if (tid < nq) {
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          float4 v = make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]),
                                 __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3]));
          if (TWO) {
            const float4 u = *reinterpret_cast<const float4 *>(so + tid * PF + c + e);
            v.x = v.x * fa + u.x * fb, v.y = v.y * fa + u.y * fb;
            v.z = v.z * fa + u.z * fb, v.w = v.w * fa + u.w * fb;
          }
          *reinterpret_cast<float4 *>(to + c + e) =
              make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        }
      }
    }
    if (tid < nq) {
      if (p.splits > 1)
        *reinterpret_cast<float2 *>(part + D) = make_float2(wrong ? NAN : m, wrong ? 0.f : l);
      else
        p.lse[row] = wrong ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_free(tmem, kTcCols);
}

// Joins a query's ranges in their order, a warp per query: lane j < splits
// holds range j's maximum and sum.
constexpr int kJoinThreads = 128;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) prefix_join_kernel(const PrefixArgs p, int rows) {
  constexpr int PF = D + 4, E = D / 32;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int row = blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5);
  if (row >= rows) return;
  const float *first = p.part + (size_t)row * p.splits * PF;
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < p.splits) ml = *reinterpret_cast<const float2 *>(first + (size_t)lane * PF + D);
  constexpr int B = 8;  // parts on their way at a time, the first before their weights
  float v[B][E];
  auto load = [&](int j0) {
#pragma unroll
    for (int j = 0; j < B; ++j)
      if (j0 + j < p.splits) load_row<E>(first + (size_t)(j0 + j) * PF + lane * E, v[j]);
  };
  load(0);
  const bool bad = __any_sync(0xFFFFFFFFu, ml.x != ml.x && ml.y == 0.f);
  float m = ml.x;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  const float f = ml.y == 0.f ? 0.f : ex2_approx(ml.x - m);
  float l = ml.y * f;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int j0 = 0; j0 < p.splits; j0 += B) {
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const float fj = __shfl_sync(0xFFFFFFFFu, f, (j0 + j) & 31);
      if (j0 + j < p.splits) {
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += v[j][e] * fj;
      }
    }
    load(j0 + B);
  }
  const float inv = bad ? NAN : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) p.out[(size_t)row * D + lane * E + e] = acc[e] * inv;
  if (lane == 0) p.lse[row] = bad ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <int D, bool TWO>
cudaError_t launch_tc(const PrefixArgs &a, int grid, int split_len, cudaStream_t s) {
  constexpr int smem = TcSmem<D>::kTotal;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem_of(prefix_tc_kernel<D, TWO>, smem, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(prefix_tc_kernel<D, TWO>, grid, kTcThreads, smem, s, a, split_len);
}

template <int D, typename T, int MW>
cudaError_t launch_tiles(const PrefixArgs &a, int grid, int split_len, cudaStream_t s) {
  constexpr int smem = PSmem<D, T, MW>::kTotal;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem_of(prefix_kernel<D, T, MW>, smem, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(prefix_kernel<D, T, MW>, grid, kThreads, smem, s, a, split_len);
}

}  // namespace

// As many key ranges as fill the device twice over (2 CTAs an SM), each a
// whole number of tiles. The 152 SMs are a constant here, so that the workspace
// a caller allocated does not depend on the device of the call. bf16 batches of more than 16 sequences go to tcgen05
// unless all their products of 16 queries and a tile are done in two rounds of
// CTAs: over 32 heads of 128 channels, 16 sequences and 4099 keys take 23 us
// with mma.sync and 27 with tcgen05; 32 take 29 and 28; 64 take 43 and 32, with
// 500 keys 14 and 14, with 64 keys 6 and 8.
PrefixPlan prefix_plan(int groups, int seqs, int heads, int max_len, int dtype) {
  constexpr int kCtas = 304;
  PrefixPlan pl;
  const long long key_tiles = (max_len + kKeys - 1) / kKeys;
  const long long products = (long long)groups * heads * ((seqs + 15) / 16) * key_tiles;
  if (dtype == HKV_BF16) pl.mw = seqs <= 16 || products <= 2 * kCtas ? 1 : 8;
  else pl.mw = seqs <= 16 ? 1 : seqs <= 32 ? 2 : 4;
  pl.tiles = (seqs + pl.mw * 16 - 1) / (pl.mw * 16);
  const long long base = (long long)groups * heads * pl.tiles;
  long long want = kCtas / base;
  if (want > kMostSplits) want = kMostSplits;
  if (want > key_tiles) want = key_tiles;
  if (want < 1) want = 1;
  pl.split_len = (int)(((max_len + want - 1) / want + kKeys - 1) / kKeys * kKeys);
  pl.splits = (max_len + pl.split_len - 1) / pl.split_len;
  return pl;
}

cudaError_t launch_prefix(const PrefixArgs &a, const PrefixPlan &pl, int D, int dtype,
                          cudaStream_t s) {
  const long long grid = (long long)a.groups * a.heads * pl.tiles * pl.splits;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  cudaError_t e = cudaErrorInvalidValue;
  HKV_DISPATCH(D, dtype, {
    if (pl.mw == 8 && a.seqs <= 64) e = launch_tc<kD, true>(a, (int)grid, pl.split_len, s);
    else if (pl.mw == 8) e = launch_tc<kD, false>(a, (int)grid, pl.split_len, s);
    else if (pl.mw == 1) e = launch_tiles<kD, kT, 1>(a, (int)grid, pl.split_len, s);
    else if (pl.mw == 2) e = launch_tiles<kD, float, 2>(a, (int)grid, pl.split_len, s);
    else e = launch_tiles<kD, float, 4>(a, (int)grid, pl.split_len, s);
  });
  if (e != cudaSuccess || a.splits == 1) return e;
  const int rows = a.groups * a.seqs * a.heads;
  const int blocks = (rows + kJoinThreads / 32 - 1) / (kJoinThreads / 32);
  if (D == 64) return pdl_launch(prefix_join_kernel<64>, blocks, kJoinThreads, 0, s, a, rows);
  return pdl_launch(prefix_join_kernel<128>, blocks, kJoinThreads, 0, s, a, rows);
}

}  // namespace hkv
