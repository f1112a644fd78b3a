// The choice of the rows a head-aware update evicts (Eqs. 2-6) and where the
// surviving rows move, shared by the updates of plain and of quantised caches:
// everything but the key rows' format and the copies. One CTA per head. Also
// the launch helpers of the per-head kernels.
#pragma once

#include <math.h>
#include <stdlib.h>

#include <atomic>

#include "hkv_device.cuh"
#include "hkv_kernels.h"

namespace hkv {

constexpr int NT = kCacheThreads;

// Phase timestamps per head of the update for latency studies; compiled out
// by default.
#ifdef HKV_UPD_TRACE
static __device__ unsigned long long *g_utrace = nullptr;  // [head of the layer][8], set by the tracer
#define HKV_UTRACE(slot)                                                   \
  do {                                                                     \
    if (g_utrace && threadIdx.x == 0)                                      \
      g_utrace[(size_t)blockIdx.x * 8 + (slot)] = globaltimer();           \
  } while (0)
#else
#define HKV_UTRACE(slot) \
  do {                   \
  } while (0)
#endif

__device__ __forceinline__ void pdl_wait() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void pdl_launch_dependents() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

struct SegRef {
  const unsigned char *sk, *sv;  // source rows, row 0 = segment start
  const int32_t *spos;
  unsigned char *dk, *dv;        // destination rows
  int32_t *dpos;
  int len;                       // live source rows
  int dst_cap;                   // destination capacity (rows)
  bool in_place;
  uint32_t *err;                 // the cache's error word
};

struct UpdShared {
  unsigned long long prefix[2];
  int rem[2];
  int iscan[33];
  long long lscan[33];
  uint64_t ring_bar;  // completion of the bulk copy of the query ring
};
static_assert(sizeof(UpdShared) == kUpdateStatic, "the host subtracts it from a CTA's 227 KB");

// Shared-memory work area of one update (dynamic).
struct UpdSmem {
  unsigned char *ring;       // [P][D] the buffered queries (<= 4 B each)
  unsigned long long *keys;  // [max_len]
  int *ps;                   // [max_len] positions of the source rows
  int *aux;                  // [max_len] class, then keep flag, then rank
  float *qbar;               // [D]
  int *hist;                 // [512]
  int stage_rows;            // rows a warp stages per pass of the score phase
};

// Rows a warp stages per pass of the score phase: 32, or fewer when every
// warp's share of the longest segment is smaller (short segments then leave
// room for more CTAs per SM).
__host__ __device__ constexpr int stage_rows(int max_len) {
  return max_len >= NT ? 32 : (max_len + NT / 32 - 1) / (NT / 32) < 1 ? 1 : (max_len + NT / 32 - 1) / (NT / 32);
}

// the query ring (P rows of es-byte elements); after q-bar it is the score
// stage: NT/32 warps x stage_rows rows of D * es + 16 bytes
// (or of kb bytes, key rows of codes); a multiple of 16
__host__ __device__ constexpr size_t ring_bytes(int P, int D, int es, int max_len, int kb = 0) {
  const size_t ring = (size_t)P * D * es;
  const size_t stage = (size_t)(NT / 32) * stage_rows(max_len) * (kb ? kb : D * es + 16);
  return ring > stage ? ring : stage;
}

__device__ __forceinline__ UpdSmem carve(unsigned char *dyn, int max_len, int D, int P, int es,
                                         int kb = 0) {
  UpdSmem u;
  u.ring = dyn;
  u.stage_rows = stage_rows(max_len);
  // rounding a multiple of 16 to 8 changes nothing but the compiler's schedule:
  // kernels over codes take 47.4 us with it and 48.3 without (1024 heads), plain
  // ones spill with it (hkv_evict_all of 8192 short heads: 156 us against 146)
  const size_t ring = ring_bytes(P, D, es, max_len, kb);
  u.keys = reinterpret_cast<unsigned long long *>(dyn + (kb ? (ring + 7) & ~(size_t)7 : ring));
  u.ps = reinterpret_cast<int *>(u.keys + max_len);
  u.aux = u.ps + max_len;
  u.qbar = reinterpret_cast<float *>(u.aux + max_len);
  u.hist = reinterpret_cast<int *>(u.qbar + D);
  return u;
}

// The k0-th smallest key among rows of class 0 and the k1-th among rows of
// class 1 (1-based; 0 = not needed; other classes ignored), by MSD radix
// select on bytes from `top_shift` down. Keys are unique within a class, so
// each result bounds exactly k keys of its class from above.
__device__ inline void radix_select2(const unsigned long long *keys, const int *cls, int n, int k0,
                              int k1, int top_shift, int *hist, UpdShared &sh) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    sh.prefix[0] = sh.prefix[1] = 0ull;
    sh.rem[0] = k0;
    sh.rem[1] = k1;
  }
  __syncthreads();
  for (int shift = top_shift; shift >= 0; shift -= 8) {
    for (int i = tid; i < 512; i += NT) hist[i] = 0;
    __syncthreads();
    const unsigned long long hi = shift >= 56 ? 0ull : (~0ull << (shift + 8));
    const unsigned long long p0 = sh.prefix[0], p1 = sh.prefix[1];
    const int r0 = sh.rem[0], r1 = sh.rem[1];
    for (int j = tid; j < n; j += NT) {
      const int s = cls[j];
      if (s != 0 && s != 1) continue;
      const unsigned long long key = keys[j];
      if ((s ? r1 : r0) > 0 && (key & hi) == (s ? p1 : p0))
        atomicAdd(&hist[s * 256 + (int)((key >> shift) & 255ull)], 1);
    }
    __syncthreads();
    if (warp < 2) {
      const int s = warp;
      const int target = sh.rem[s];
      if (target > 0) {  // warp-uniform
        int c[8], sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c[e] = hist[s * 256 + lane * 8 + e];
          sum += c[e];
        }
        const int incl = warp_incl_scan(sum);
        const int excl = incl - sum;
        if (excl < target && target <= incl) {
          int run = excl, digit = -1, rem = 0, in_bin = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (digit < 0 && run + c[e] >= target) {
              digit = lane * 8 + e;
              rem = target - run;
              in_bin = c[e];
            }
            run += c[e];
          }
          sh.prefix[s] |= (unsigned long long)digit << shift;
          if (rem == in_bin) {
            // every key of this bin is among the k: the bin's upper end
            // bounds exactly k keys (keys are unique), no further digit
            sh.prefix[s] |= shift > 0 ? (1ull << shift) - 1ull : 0ull;
            sh.rem[s] = 0;
          } else {
            sh.rem[s] = rem;
          }
        }
      }
    }
    __syncthreads();
    if (sh.rem[0] == 0 && sh.rem[1] == 0) break;
  }
}

__device__ __forceinline__ int block_sum(int x, UpdShared &sh) {
  int tot;
  block_excl_scan<int>(x, sh.iscan, &tot);
  return tot;
}

// Key rows in the config dtype: bytes of a row, and its product with q-bar in
// the order of the channels, every product and sum rounded to fp32 by itself
// (the order and rounding decide which rows go, so they are part of the rule).
template <int D, typename T>
struct PlainRows {
  static constexpr int kBytes = D * (int)sizeof(T);
  static constexpr int kStride = kBytes + 16;  // of a staged row
  struct Ahead {};
  __device__ __forceinline__ Ahead ahead(int) const { return {}; }
  // byte offset of piece pc of staged row rr: lanes that read one piece of
  // successive rows hit distinct banks
  __device__ __forceinline__ static int piece(int rr, int pc) { return rr * kStride + pc * 16; }
  __device__ __forceinline__ float dot(const unsigned char *stage, int rr, const float *qbar,
                                       Ahead) const {
    constexpr int EPL = Elem<T>::kPerPiece;
    const unsigned char *krow = stage + rr * kStride;
    float s = 0.f;
#pragma unroll 4
    for (int pc = 0; pc < kBytes / 16; ++pc) {
      float kf[EPL];
      Elem<T>::unpack(*reinterpret_cast<const uint4 *>(krow + pc * 16), kf);
#pragma unroll
      for (int e = 0; e < EPL; ++e) s = __fadd_rn(s, __fmul_rn(qbar[pc * EPL + e], kf[e]));
    }
    return s;
  }
};

// Decides which rows of a segment the update evicts (Eqs. 2-6). On return
// u.aux[r] is 1 for a kept row and 0 for an evicted one (r < len), u.ps
// holds the rows' positions, and the number of evicted rows is returned; or -1,
// with HKV_ERR_TIMEOUT in the error word, where the queries did not arrive in
// time: the head is then left as it is. Block-uniform. D, T: the queries' row; Rows: the format of the key rows.
template <int D, typename T, class Rows>
__device__ int select_evictions(const SegRef &sg, int label, const MethodArgs &m,
                                const unsigned char *qring, int ntok, const UpdSmem &u,
                                UpdShared &sh, const Rows &rows) {
  constexpr int RB = D * (int)sizeof(T);
  constexpr int KB = Rows::kBytes;
  constexpr int LPR = KB / 16;
  const int tid = threadIdx.x;
  const int C = m.C;
  const int recent_from = C + (ntok > m.w ? ntok - m.w : 0);   // newest w image tokens
  int nh = 0;
  for (int r = tid; r < sg.len; r += NT) {
    const int ps = sg.spos[r];
    u.ps[r] = ps;
    const bool hist = ps >= C && ps < recent_from;
    u.aux[r] = hist ? 0 : -1;   // class: history (0) or always kept (-1)
    nh += hist ? 1 : 0;
  }
  const int NH = block_sum(nh, sh);  // history candidates (Eq. 2)
  HKV_UTRACE(1);
  // the head's history budget, B_g - w with the paper's budgets, from the
  // capacity its segment was given (C + budget + P)
  const int hist_budget = sg.dst_cap - C - m.P - m.w > 0 ? sg.dst_cap - C - m.P - m.w : 0;
  int M = 0;
  if (label == HKV_LOCAL) M = NH;    // Eq. 3: no history
  else if (NH > hist_budget) M = NH - hist_budget;

  if (label == HKV_GLOBAL && M > 0) {
    // the query ring comes in with one bulk copy, behind the choice of the
    // subsets
    const int P = m.P;
    if (tid == 0) {
      mbar_init(&sh.ring_bar, 1);
      fence_barrier_init();
      const uint32_t bytes = (uint32_t)P * RB;
      mbar_arrive_expect_tx(&sh.ring_bar, bytes);
      bulk_g2s(u.ring, qring, bytes, &sh.ring_bar);
    }
    __syncthreads();
    // Eq. 5: the floor(NH r_s) oldest history tokens are long-range (or,
    // in the grid-distance variant, the farthest from the newest image
    // token, equal distances older first)
    const int n_long = (int)floor((double)NH * m.r_s);
    if (n_long > 0 && n_long < NH && m.grid2d) {
      const int ref = ntok - 1;
      for (int r = tid; r < sg.len; r += NT) {
        const int i = u.ps[r] - C;
        const long long dr = i / m.row_len - ref / m.row_len, dc = i % m.row_len - ref % m.row_len;
        const unsigned long long far = 0x7FFFFFFFull - (unsigned long long)(dr * dr + dc * dc);
        u.keys[r] = (far << 32) | (uint32_t)u.ps[r];
      }
      radix_select2(u.keys, u.aux, sg.len, n_long, 0, 56, u.hist, sh);
      const unsigned long long k_long = sh.prefix[0];
      for (int r = tid; r < sg.len; r += NT)
        if (u.aux[r] == 0) u.aux[r] = u.keys[r] <= k_long ? 0 : 1;
    } else if (n_long > 0 && n_long < NH) {
      for (int r = tid; r < sg.len; r += NT) u.keys[r] = (unsigned long long)(uint32_t)u.ps[r];
      const int maxp = C + ntok;  // positions are below it: start at its top byte
      const int top = maxp < (1 << 8) ? 0 : maxp < (1 << 16) ? 8 : maxp < (1 << 24) ? 16 : 24;
      radix_select2(u.keys, u.aux, sg.len, n_long, 0, top, u.hist, sh);
      const int p_long = (int)sh.prefix[0];
      for (int r = tid; r < sg.len; r += NT)
        if (u.aux[r] == 0) u.aux[r] = u.ps[r] <= p_long ? 0 : 1;
    } else {
      for (int r = tid; r < sg.len; r += NT)
        if (u.aux[r] == 0) u.aux[r] = n_long == NH ? 0 : 1;
    }
    HKV_UTRACE(2);
    // Eq. 6 scores: q-bar = the P buffered queries, oldest first; the sums keep
    // their order
    bool arrived = mbar_wait(&sh.ring_bar, 0);
#ifdef HKV_UPD_TEST_STALL  // one warp waits for a phase that nothing completes
    if (arrived && tid >> 5 == (int)(blockIdx.x & 7)) arrived = mbar_wait(&sh.ring_bar, 1);
#endif
    for (int d = tid; d < D; d += NT) {
      float acc = 0.f;
      int slot = (ntok - P) % P;
      if (slot < 0) slot += P;
#pragma unroll 4
      for (int pp = 0; pp < P; ++pp) {
        acc = __fadd_rn(acc, Elem<T>::load1(u.ring, (size_t)slot * D + d));
        slot = slot + 1 == P ? 0 : slot + 1;
      }
      u.qbar[d] = acc;
    }
    if (!__syncthreads_and(arrived)) {
      if (tid == 0) set_err(sg.err, HKV_ERR_TIMEOUT);
      mbar_wait(&sh.ring_bar, 0);  // the copy gets the limit once more to end in
      return -1;
    }
    HKV_UTRACE(3);
    // Each warp stages 32 rows at a time in the (now free) ring area with
    // coalesced 16-byte async copies, laid out so that lane l reading row l,
    // piece j, hits distinct banks; then lane l sums its row in the fixed
    // order.
    const int warp = tid >> 5, lane = tid & 31;
    const int SR = u.stage_rows;
    unsigned char *stage = u.ring + (size_t)warp * SR * Rows::kStride;
    for (int base = warp * SR; base < sg.len; base += (NT / 32) * SR) {
      const int nrows = sg.len - base < SR ? sg.len - base : SR;
      for (int w = lane; w < nrows * LPR; w += 32) {
        const int rr = w / LPR, pc = w % LPR;
        cp_async16(stage + Rows::piece(rr, pc), sg.sk + (size_t)(base + rr) * KB + pc * 16);
      }
      const int r = base + lane;
      const bool scored = lane < nrows && u.aux[r] >= 0;
      typename Rows::Ahead ah = {};
      if (scored) ah = rows.ahead(r);
      cp_async_wait_all();
      __syncwarp();
      if (scored) {
        float s = rows.dot(stage, lane, u.qbar, ah);
        s = __fadd_rn(s, 0.f);  // -0 reads as +0
        uint32_t bits = __float_as_uint(s);
        bits = (bits & 0x80000000u) ? ~bits : (bits | 0x80000000u);  // order-preserving
        u.keys[r] = ((unsigned long long)bits << 32) | (uint32_t)u.ps[r];
      }
      __syncwarp();  // the stage is rewritten next round
    }
    __syncthreads();
    HKV_UTRACE(4);
    // M/2 from each subset; a short subset hands its excess to the other
    int m_long = M / 2, m_near = M - M / 2;
    if (m_long > n_long) {
      m_near += m_long - n_long;
      m_long = n_long;
    }
    if (m_near > NH - n_long) {
      m_long += m_near - (NH - n_long);
      m_near = NH - n_long;
    }
    radix_select2(u.keys, u.aux, sg.len, m_long, m_near, 56, u.hist, sh);
    const unsigned long long thr0 = sh.prefix[0], thr1 = sh.prefix[1];
    for (int r = tid; r < sg.len; r += NT) {
      const int c = u.aux[r];
      const bool ev = c == 0 ? (m_long > 0 && u.keys[r] <= thr0)
                             : c == 1 ? (m_near > 0 && u.keys[r] <= thr1) : false;
      u.aux[r] = ev ? 0 : 1;
    }
    HKV_UTRACE(5);
  } else {
    for (int r = tid; r < sg.len; r += NT) u.aux[r] = (u.aux[r] == 0 && M > 0) ? 0 : 1;
  }
  __syncthreads();
  return M;
}

// In place: the new length is len - M; every evicted row below it takes a
// surviving row from above it (the i-th hole the i-th survivor). Sources
// are all >= new_len and destinations < new_len, so the moves are
// independent. Lists the rows to fill and the rows that fill them in the keys
// area (free after the selection): hole[i] takes fill[i], i < the number
// returned. Each thread ranks a contiguous run of rows (one block scan for
// holes and fills together). Block-uniform.
__device__ inline int pair_holes(int len, int M, const UpdSmem &u, UpdShared &sh, int **hole_out,
                                 int **fill_out) {
  const int tid = threadIdx.x, new_len = len - M;
  // the keys area is free now and holds the two index lists
  int *hole = reinterpret_cast<int *>(u.keys);  // [M]
  int *fill = hole + M;                          // [M]
  const int per = (len + NT - 1) / NT;
  const int r0 = tid * per < len ? tid * per : len;
  const int r1 = r0 + per < len ? r0 + per : len;
  long long nh = 0, nf = 0;
  for (int r = r0; r < r1; ++r) {
    const int keep = u.aux[r];
    nh += (r < new_len && !keep) ? 1 : 0;
    nf += (r >= new_len && keep) ? 1 : 0;
  }
  long long tot;
  const long long ex = block_excl_scan<long long>((nh << 32) | nf, sh.lscan, &tot);
  int hp = (int)(ex >> 32), fp = (int)(ex & 0xFFFFFFFFll);
  for (int r = r0; r < r1; ++r) {
    const int keep = u.aux[r];
    if (r < new_len && !keep) hole[hp++] = r;
    if (r >= new_len && keep) fill[fp++] = r;
  }
  __syncthreads();
  *hole_out = hole;
  *fill_out = fill;
  return (int)(tot >> 32);  // holes and fills pair up
}

#define HKV_DISPATCH(D_, DT_, ...)                  \
  do {                                              \
    if ((DT_) == HKV_BF16) {                        \
      if ((D_) == 64) {                             \
        constexpr int kD = 64;                      \
        using kT = __nv_bfloat16;                   \
        __VA_ARGS__;                                \
      } else {                                      \
        constexpr int kD = 128;                     \
        using kT = __nv_bfloat16;                   \
        __VA_ARGS__;                                \
      }                                             \
    } else {                                        \
      if ((D_) == 64) {                             \
        constexpr int kD = 64;                      \
        using kT = float;                           \
        __VA_ARGS__;                                \
      } else {                                      \
        constexpr int kD = 128;                     \
        using kT = float;                           \
        __VA_ARGS__;                                \
      }                                             \
    }                                               \
  } while (0)

// launch with programmatic stream serialisation (the kernels wait for their
// predecessor with griddepcontrol.wait before touching memory)
template <typename... KArgs, typename... Args>
inline cudaError_t pdl_launch(void (*kernel)(KArgs...), int grid, int block, size_t smem, cudaStream_t s,
                       Args... args) {
  static const bool pdl = getenv("HKV_NO_PDL") == nullptr;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Raises a kernel's limit of dynamic shared memory to `smem`, with all of an
// SM's L1 as shared memory, once per device and kernel.
template <typename... KArgs>
inline cudaError_t allow_smem_of(void (*kernel)(KArgs...), int smem, std::atomic<uint64_t> &ready) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (ready.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 100);
  if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_release);
  return e;
}

inline size_t update_smem_of(int max_len, int D, int P, int es, int kb = 0) {
  // the query ring / score stage; keys (8 B), positions (4 B), class/flag/
  // rank (4 B) per row; q-bar; two 256-bin histograms
  return ring_bytes(P, D, es, max_len, kb) + (size_t)max_len * 16 + (size_t)D * 4 + 512 * 4 + 64;
}

// the longest segment a launch with `smem` bytes takes (the inverse of
// update_smem_of, which grows with max_len)
inline int update_max_len(size_t smem, int D, int P, int es, int kb = 0) {
  int lo = 0, hi = 1 << 20;
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (update_smem_of(mid, D, P, es, kb) <= smem) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

}  // namespace hkv
