// Rotary positions of heads, and the norms of queries and keys with the
// rotation in the same pass.
//
// A row is one head of one token, D channels. Pair i turns by the angle p f_i;
// p (f_i / 2 pi) is taken modulo one turn as the low half of a product of
// integers, p times f_i / 2 pi in units of 2^-64, so that no position loses
// digits, and its high word, a signed fraction of a turn, goes to sincospif.
//
// heads_kernel: a thread holds two 16-byte pieces of a row, chosen so that both
// channels of each of its pairs are its own (half layout: a piece and the one
// rot_dim / 2 further; interleaved: two neighbours); rows are then rotated
// without an exchange, and in place. Norms sum over the G threads of a row with
// shuffles. A thread keeps the cosines and sines of its pairs for a few heads
// of the same token, so that the angles cost a fraction of the copies.
// heads_any_kernel takes half layouts whose pieces do not fall together
// (rot_dim / 2 not a multiple of a piece): a warp per row, through shared memory.
#include <cuda_bf16.h>

#include "hkv_device.cuh"
#include "hkv_heads.h"
#include "hkv_select.cuh"

namespace hkv {
namespace {

constexpr int kHeadThreads = 256;

// cosine and sine of one pair's angle, times the amplitude
__device__ __forceinline__ void turn(const HeadsArgs &a, int pair, const int (&pos)[3], float &c,
                                     float &s) {
  const int axis = pair >= a.rope.section[0] + a.rope.section[1] ? 2 : pair >= a.rope.section[0];
  const int p = axis == 0 ? pos[0] : axis == 1 ? pos[1] : pos[2];
  const uint64_t part = (uint64_t)(int64_t)p * a.rope.turns[pair];  // modulo one turn
  sincospif((float)(int32_t)(part >> 32) * 0x1p-31f, &s, &c);
  c *= a.rope.amplitude;
  s *= a.sign;  // (holds the amplitude)
}

__device__ __forceinline__ const HeadSet &set_of(const HeadsArgs &a, int &head) {
  int i = 0;
  if (i + 1 < a.sets && head >= a.set[0].heads) head -= a.set[i++].heads;
  if (i == 1 && a.sets > 2 && head >= a.set[1].heads) head -= a.set[i++].heads;
  return a.set[i];
}

template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int kN = 4;
  __device__ static __forceinline__ uint4 pack(const float *f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  }
  __device__ static __forceinline__ void store1(void *p, float f) { *static_cast<float *>(p) = f; }
};
template <>
struct Piece<__nv_bfloat16> {
  static constexpr int kN = 8;
  __device__ static __forceinline__ uint32_t two(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  __device__ static __forceinline__ uint4 pack(const float *f) {
    return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7]));
  }
  __device__ static __forceinline__ void store1(void *p, float f) {
    *static_cast<__nv_bfloat16 *>(p) = __float2bfloat16_rn(f);
  }
};

// the sequence's tokens; -1 (and the error word) where the length is out of range
__device__ __forceinline__ int tokens_of(const HeadsArgs &a, int s) {
  if (!a.len) return a.tokens;
  const int n = a.len[s];
  if (n >= 0 && n <= a.tokens) return n;
  set_err(a.err, HKV_ERR_BOUNDS);
  return -1;
}

// NORM: 0 none, else HKV_NORM_*. A block's threads are row slots of G: `per`
// slots for each of its tokens, which take heads first, first + per, ...
template <typename T, int D, int NORM>
__global__ void __launch_bounds__(kHeadThreads)
    heads_kernel(const __grid_constant__ HeadsArgs a, int per, int tokens_per_block, int chunks,
                 long long places) {
  constexpr int N = Piece<T>::kN, G = D / (2 * N), U = 2;
  pdl_wait();
  pdl_launch_dependents();
  const int g = threadIdx.x % G, slot = threadIdx.x / G;
  const int tok = slot / per, first = slot % per;
  const int chunk = blockIdx.x % chunks;
  const long long place = (long long)(blockIdx.x / chunks) * tokens_per_block + tok;
  bool on = tok < tokens_per_block && place < places;
  const int s = on ? (int)(place / a.tokens) : 0, t = on ? (int)(place % a.tokens) : 0;
  if (on) on = t < tokens_of(a, s);
  // (whole groups of G lanes, a power of two, are on or off together)
  const int R = a.rope.rot_dim;
  // the thread's two pieces
  const bool pairs = a.rope.layout == HKV_ROPE_PAIRS;
  const bool apart = !pairs && N * g < R / 2;  // the other channels two by two behind R
  const int ca = apart ? N * g : 2 * N * g, cb = apart ? ca + R / 2 : ca + N;
  const int heads_here = (a.heads + chunks - 1) / chunks;
  const int h1 = min(a.heads, (chunk + 1) * heads_here);
  float c[N], sn[N];
  bool have = false;
  for (int hb = chunk * heads_here; hb < h1; hb += U * per) {  // the same for all lanes
    const int h0 = hb + first;
    uint4 ra[U], rb[U];
    if (on) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        int h = h0 + u * per;
        if (h < h1) {
          const HeadSet &x = set_of(a, h);
          const T *row = static_cast<const T *>(x.in) + s * x.is + t * x.it + h * x.ih;
          ra[u] = *reinterpret_cast<const uint4 *>(row + ca);
          rb[u] = *reinterpret_cast<const uint4 *>(row + cb);
        }
      }
    }
    if (on && !have && R > 0) {
      have = true;
      int pos[3];
#pragma unroll
      for (int x = 0; x < 3; ++x)
        pos[x] = x < a.rope.n_axes ? a.pos[x * a.pa + s * a.ps + t] : 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        // half layout: pair of (a[i], b[i]); interleaved: of neighbours, a's then b's
        const int pair = pairs ? N * g + i : ca + i;
        c[i] = 1.f, sn[i] = 0.f;
        if (pair < R / 2) turn(a, pair, pos, c[i], sn[i]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int h = h0 + u * per;
      const bool live = on && h < h1;
      const HeadSet &x = set_of(a, h);
      float va[N], vb[N];
      if (live) {
        Elem<T>::unpack(ra[u], va);
        Elem<T>::unpack(rb[u], vb);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) va[i] = vb[i] = 0.f;
      }
      if (NORM != 0) {  // every lane takes part in the shuffles
        float mean = 0.f, sum = 0.f;
        if (NORM == HKV_NORM_LAYER) {
#pragma unroll
          for (int i = 0; i < N; ++i) mean += va[i] + vb[i];
#pragma unroll
          for (int o = G / 2; o >= 1; o >>= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);
          mean *= 1.f / D;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float da = va[i] - mean, db = vb[i] - mean;
          sum += da * da + db * db;
        }
#pragma unroll
        for (int o = G / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (live && x.norm) {
          const float inv = 1.f / sqrtf(sum * (1.f / D) + a.eps);
          float w[N], b[N];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float *v = half ? vb : va;
            const int at = half ? cb : ca;
            if (x.weight)
              Elem<T>::unpack(*reinterpret_cast<const uint4 *>(static_cast<const T *>(x.weight) +
                                                               h * x.wh + at), w);
            if (NORM == HKV_NORM_LAYER && x.bias)
              Elem<T>::unpack(*reinterpret_cast<const uint4 *>(static_cast<const T *>(x.bias) +
                                                               h * x.wh + at), b);
#pragma unroll
            for (int i = 0; i < N; ++i) {
              v[i] = (v[i] - mean) * inv;
              if (x.weight) v[i] *= w[i];
              if (NORM == HKV_NORM_LAYER && x.bias) v[i] += b[i];
            }
          }
        }
      }
      if (!live) continue;
      if (x.rotate) {
        if (pairs) {
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            const float x0 = va[2 * i], y0 = va[2 * i + 1], x1 = vb[2 * i], y1 = vb[2 * i + 1];
            va[2 * i] = x0 * c[i] - y0 * sn[i];
            va[2 * i + 1] = x0 * sn[i] + y0 * c[i];
            vb[2 * i] = x1 * c[N / 2 + i] - y1 * sn[N / 2 + i];
            vb[2 * i + 1] = x1 * sn[N / 2 + i] + y1 * c[N / 2 + i];
          }
        } else if (apart) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float x0 = va[i], y0 = vb[i];
            va[i] = x0 * c[i] - y0 * sn[i];
            vb[i] = x0 * sn[i] + y0 * c[i];
          }
        }
      }
      T *row = static_cast<T *>(x.out) + s * x.os + t * x.ot + h * x.oh;
      *reinterpret_cast<uint4 *>(row + ca) = Piece<T>::pack(va);
      *reinterpret_cast<uint4 *>(row + cb) = Piece<T>::pack(vb);
    }
  }
}

// a warp per row
template <typename T, int D, int NORM>
__global__ void __launch_bounds__(kHeadThreads)
    heads_any_kernel(const __grid_constant__ HeadsArgs a, long long rows) {
  constexpr int E = D / 32;
  __shared__ float s_row[kHeadThreads / 32][D];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long r = (long long)blockIdx.x * (kHeadThreads / 32) + warp;
  if (r >= rows) return;
  int h = (int)(r % a.heads);
  const long long place = r / a.heads;
  const int s = (int)(place / a.tokens), t = (int)(place % a.tokens);
  if (t >= tokens_of(a, s)) return;
  const HeadSet &x = set_of(a, h);
  const T *in = static_cast<const T *>(x.in) + s * x.is + t * x.it + h * x.ih;
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = Elem<T>::load1(in, lane + 32 * e);
  if (NORM != 0 && x.norm) {
    float mean = 0.f, sum = 0.f;
    if (NORM == HKV_NORM_LAYER) {
#pragma unroll
      for (int e = 0; e < E; ++e) mean += v[e];
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);
      mean *= 1.f / D;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sum += (v[e] - mean) * (v[e] - mean);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    const float inv = 1.f / sqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v[e] = (v[e] - mean) * inv;
      if (x.weight) v[e] *= Elem<T>::load1(x.weight, h * x.wh + lane + 32 * e);
      if (NORM == HKV_NORM_LAYER && x.bias) v[e] += Elem<T>::load1(x.bias, h * x.wh + lane + 32 * e);
    }
  }
  T *out = static_cast<T *>(x.out) + s * x.os + t * x.ot + h * x.oh;
  const int R = x.rotate ? a.rope.rot_dim : 0;
  int pos[3];
#pragma unroll
  for (int i = 0; i < 3; ++i)
    pos[i] = R > 0 && i < a.rope.n_axes ? a.pos[i * a.pa + s * a.ps + t] : 0;
#pragma unroll
  for (int e = 0; e < E; ++e) s_row[warp][lane + 32 * e] = v[e];
  __syncwarp();
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int ch = lane + 32 * e;
    if (ch < R) {
      const bool second = ch >= R / 2;
      float c, sn;
      turn(a, second ? ch - R / 2 : ch, pos, c, sn);
      const float other = s_row[warp][second ? ch - R / 2 : ch + R / 2];
      v[e] = second ? other * sn + v[e] * c : v[e] * c - other * sn;
    }
    Piece<T>::store1(out + ch, v[e]);
  }
}

template <typename T, int D, int NORM>
cudaError_t launch(const HeadsArgs &a, cudaStream_t s) {
  constexpr int N = Piece<T>::kN, kSlots = kHeadThreads / (D / (2 * N));
  const long long places = (long long)a.seqs * a.tokens;
  if (a.rope.layout == HKV_ROPE_HALF && a.rope.rot_dim / 2 % N != 0) {
    constexpr int kRows = kHeadThreads / 32;
    const long long rows = places * a.heads, grid = (rows + kRows - 1) / kRows;
    if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
    return pdl_launch(heads_any_kernel<T, D, NORM>, (int)grid, kHeadThreads, 0, s, a, rows);
  }
  int iters = 8;
  while (iters > 1 && places * a.heads < 608LL * kSlots * iters) iters >>= 1;
  int per = (a.heads + iters - 1) / iters;
  int chunks = 1;
  if (per > kSlots) {
    chunks = (a.heads + kSlots * iters - 1) / (kSlots * iters);
    per = kSlots;
  }
  const int tpb = kSlots / per;
  const long long grid = (places + tpb - 1) / tpb * chunks;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  return pdl_launch(heads_kernel<T, D, NORM>, (int)grid, kHeadThreads, 0, s, a, per, tpb, chunks,
                    places);
}

template <typename T, int D>
cudaError_t launch_norm(const HeadsArgs &a, int norm, cudaStream_t s) {
  if (norm == HKV_NORM_RMS) return launch<T, D, HKV_NORM_RMS>(a, s);
  if (norm == HKV_NORM_LAYER) return launch<T, D, HKV_NORM_LAYER>(a, s);
  return launch<T, D, 0>(a, s);
}

}  // namespace

cudaError_t launch_heads(const HeadsArgs &a, int D, int dtype, int norm, cudaStream_t s) {
  cudaError_t e = cudaErrorInvalidValue;
  HKV_DISPATCH(D, dtype, e = (launch_norm<kT, kD>(a, norm, s)));
  return e;
}

}  // namespace hkv
