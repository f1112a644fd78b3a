// Rotary positions of heads, and the norms of queries and keys with the
// rotation in the same pass.
//
// A row is one head of one token, D channels. Pair i turns by the angle p f_i;
// p (f_i / 2 pi) is taken modulo one turn as the low half of a product of
// integers, p times f_i / 2 pi in units of 2^-64, so that no position loses
// digits, and its high word, a signed fraction of a turn, goes to sincospif.
//
// heads_kernel: a block works on one of q, k and v; a thread holds two pieces of
// 4 channels of a row, chosen so that both channels of each of its pairs are its
// own (half layout: a piece and the one rot_dim / 2 further; interleaved: two
// neighbours); rows are then rotated without an exchange, and in place. Norms
// sum over the D / 8 threads of a row with shuffles. A thread keeps the cosines
// and sines of its pairs, and weights that all heads share, for several heads of
// the same token, so that the angles cost a fraction of the copies, and loads a
// few rows ahead of the first one's arithmetic.
// What bounds it: DRAM without norms (128 x 576 tokens of 20 heads of 64, bf16, two
// axes: 58 us, 6.5 TB/s, 0.97 of a copy); with them instruction issue too (8 x 4288
// tokens of 96 heads of 128, bf16, layer norms, q and k of three: 296 us, 5.7 TB/s;
// RMS norms 6.2), and the smallest calls the launch and three dependent reads (2.1
// us; a step of 8 sequences with norms 3.6). A thread with two 16-byte pieces of
// bf16 took 643 us for the second (127 registers, two reads on their way), the sums
// of four rows side by side 467 (spills).
// heads_any_kernel takes half layouts whose pieces do not fall together
// (rot_dim / 2 not a multiple of 4): a warp per row, through shared memory.
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

// a piece of 4 neighbouring channels as two pairs, and back
template <typename T>
struct Piece;
template <>
struct Piece<float> {
  using Raw = uint4;
  __device__ static __forceinline__ void unpack(const uint4 &u, uint64_t (&f)[2]) {
    f[0] = pair_of(u.x, u.y), f[1] = pair_of(u.z, u.w);
  }
  __device__ static __forceinline__ uint4 pack(const uint64_t (&f)[2]) {
    return make_uint4((uint32_t)f[0], (uint32_t)(f[0] >> 32), (uint32_t)f[1], (uint32_t)(f[1] >> 32));
  }
  __device__ static __forceinline__ void store1(void *p, float f) { *static_cast<float *>(p) = f; }
};
template <>
struct Piece<__nv_bfloat16> {
  using Raw = uint2;
  __device__ static __forceinline__ void unpack(const uint2 &u, uint64_t (&f)[2]) {
    f[0] = pair_of(u.x << 16, u.x & 0xFFFF0000u), f[1] = pair_of(u.y << 16, u.y & 0xFFFF0000u);
  }
  __device__ static __forceinline__ uint32_t two(uint64_t a) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(low(a), high(a));
    return *reinterpret_cast<const uint32_t *>(&h);
  }
  __device__ static __forceinline__ uint2 pack(const uint64_t (&f)[2]) {
    return make_uint2(two(f[0]), two(f[1]));
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
// slots for each of its tokens, which take heads first, first + per, ..., U of them
// at a time.
template <typename T, int D, int NORM, bool PAIRS, int U>
__global__ void __launch_bounds__(kHeadThreads, sizeof(T) == 4 ? 3 : 4)
    heads_kernel(const __grid_constant__ HeadsArgs a, uint32_t places) {
  constexpr int N = 4, G = D / (2 * N);
  // pairs that do not turn go out as they were read: a NaN's bits too
  constexpr bool kKeep = NORM == 0 && PAIRS && sizeof(T) == 2;
  using P = Piece<T>;
  using Raw = typename P::Raw;
  pdl_wait();
  pdl_launch_dependents();
  const int i = (a.sets > 1 && (int)blockIdx.x >= a.set[1].first_block) +
                (a.sets > 2 && (int)blockIdx.x >= a.set[2].first_block);
  const HeadSet &x = a.set[i];
  const uint32_t block = blockIdx.x - x.first_block;
  const uint32_t g = threadIdx.x % G, slot = threadIdx.x / G;
  const uint32_t tok = slot / (uint32_t)x.per, first = slot - tok * x.per;
  uint32_t group = block, chunk = 0;  // of tokens, of heads
  if (x.chunks > 1) group = block / (uint32_t)x.chunks, chunk = block - group * x.chunks;
  const uint32_t place = group * x.tokens + tok;
  bool on = (int)tok < x.tokens && place < places;
  const int s = on ? place / (uint32_t)a.tokens : 0, t = on ? place - (uint32_t)s * a.tokens : 0;
  // (the position is on its way while the length is)
  int pos[3];
#pragma unroll
  for (int k = 0; k < 3; ++k)
    pos[k] = on && x.rotate && k < a.rope.n_axes ? a.pos[k * a.pa + s * a.ps + t] : 0;
  if (on) on = t < tokens_of(a, s);
  // (whole groups of G lanes, a power of two, are on or off together)
  const int R = x.rotate ? a.rope.rot_dim : 0;
  // the thread's two pieces; the channels behind R of a half layout two by two
  const bool apart = !PAIRS && N * g < R / 2;
  const int ca = apart ? N * g : 2 * N * g, step = apart ? R / 2 : N;
  const int turning = PAIRS ? min(max(R / 2 - N * (int)g, 0), 4) : apart ? 4 : 0;  // of its 4 pairs
  const int hfirst = chunk * x.chunk + first, h1 = min(x.heads, (int)(chunk + 1) * x.chunk);
  const T *in = static_cast<const T *>(x.in) + s * x.is + t * x.it + hfirst * x.ih + ca;
  T *out = static_cast<T *>(x.out) + s * x.os + t * x.ot + hfirst * x.oh + ca;
  const long long in_step = x.per * x.ih, out_step = x.per * x.oh;
  // rows of this thread (x.most: of any in the block)
  const int rows = on && hfirst < h1 ? (int)((uint32_t)(h1 - hfirst + x.per - 1) / (uint32_t)x.per) : 0;
  const int most = x.most;
  // cosines and sines; half layout: of the pairs of channels 2 i, 2 i + 1 of the
  // two pieces; interleaved: of the pairs themselves, the first piece's first
  uint64_t c[2], sn[2], wa[2], wb[2], ba[2], bb[2];
  const bool shared = NORM != 0 && x.wh == 0;
  // The arithmetic below is a warp's, rows or none: 8 x 4288 padded tokens, on average
  // half of them there, 213 us, 168 without that of the padding. RMS norms ask behind
  // their first loads, and few rows not at all (5 x 1001 of 18 heads 6.3 us, 6.8 with
  // it); layer norms spill unless they ask here (8 x 4288 tokens 391 us against 296).
  if (NORM == HKV_NORM_LAYER && !__any_sync(0xFFFFFFFFu, on)) return;
  for (int r0 = 0; r0 < most; r0 += U) {
    Raw ra[U], rb[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r0 + u < rows) {
        ra[u] = *reinterpret_cast<const Raw *>(in + (r0 + u) * in_step);
        rb[u] = *reinterpret_cast<const Raw *>(in + (r0 + u) * in_step + step);
      }
    if (r0 == 0) {
      if (NORM == HKV_NORM_RMS && most >= 8 && !__any_sync(0xFFFFFFFFu, on)) return;
      if (shared && x.weight) {
        const T *w = static_cast<const T *>(x.weight) + ca;
        P::unpack(*reinterpret_cast<const Raw *>(w), wa);
        P::unpack(*reinterpret_cast<const Raw *>(w + step), wb);
      }
      if (shared && x.bias) {
        const T *b = static_cast<const T *>(x.bias) + ca;
        P::unpack(*reinterpret_cast<const Raw *>(b), ba);
        P::unpack(*reinterpret_cast<const Raw *>(b + step), bb);
      }
      if (rows > 0 && R > 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float cc[2] = {1.f, 1.f}, ss[2] = {0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int pair = PAIRS ? N * g + 2 * k + e : ca + 2 * k + e;
            if (pair < R / 2) turn(a, pair, pos, cc[e], ss[e]);
          }
          c[k] = pair_of(cc[0], cc[1]);
          sn[k] = pair_of(ss[0], ss[1]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + u >= most) break;
      const bool live = r0 + u < rows;
      if (NORM == 0 ? turning == 0 : !x.norm && R == 0) {  // a copy
        if (live) {
          *reinterpret_cast<Raw *>(out + (r0 + u) * out_step) = ra[u];
          *reinterpret_cast<Raw *>(out + (r0 + u) * out_step + step) = rb[u];
        }
        continue;
      }
      uint64_t va[2], vb[2];
      P::unpack(ra[u], va);
      P::unpack(rb[u], vb);
      if (NORM != 0 && x.norm) {  // every lane takes part in the shuffles
        if (NORM == HKV_NORM_LAYER) {
          const uint64_t both = add2(add2(va[0], va[1]), add2(vb[0], vb[1]));
          float mean = low(both) + high(both);
#pragma unroll
          for (int o = G / 2; o >= 1; o >>= 1) mean += __shfl_xor_sync(0xFFFFFFFFu, mean, o);
          mean *= -1.f / D;
          const uint64_t less = pair_of(mean, mean);
#pragma unroll
          for (int k = 0; k < 2; ++k) va[k] = add2(va[k], less), vb[k] = add2(vb[k], less);
        }
        const uint64_t squares =
            fma2(vb[1], vb[1], fma2(vb[0], vb[0], fma2(va[1], va[1], mul2(va[0], va[0]))));
        float sum = low(squares) + high(squares);
#pragma unroll
        for (int o = G / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const float inv = rsqrtf(sum * (1.f / D) + a.eps);
        const uint64_t by = pair_of(inv, inv);
        if (!shared && live) {  // the head's own
          const long long h = hfirst + (r0 + u) * x.per;
          if (x.weight) {
            const T *w = static_cast<const T *>(x.weight) + h * x.wh + ca;
            P::unpack(*reinterpret_cast<const Raw *>(w), wa);
            P::unpack(*reinterpret_cast<const Raw *>(w + step), wb);
          }
          if (NORM == HKV_NORM_LAYER && x.bias) {
            const T *b = static_cast<const T *>(x.bias) + h * x.wh + ca;
            P::unpack(*reinterpret_cast<const Raw *>(b), ba);
            P::unpack(*reinterpret_cast<const Raw *>(b + step), bb);
          }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          va[k] = mul2(va[k], by), vb[k] = mul2(vb[k], by);
          if (x.weight) va[k] = mul2(va[k], wa[k]), vb[k] = mul2(vb[k], wb[k]);
          if (NORM == HKV_NORM_LAYER && x.bias) va[k] = add2(va[k], ba[k]), vb[k] = add2(vb[k], bb[k]);
        }
      }
      if (!live) continue;
      if (PAIRS) {
        auto turned = [&](int k) {  // pair (x, y): c x - s y, s x + c y
          uint64_t &v = k < 2 ? va[k & 1] : vb[k & 1];
          const float cc = k & 1 ? high(c[k / 2]) : low(c[k / 2]);
          const float ss = k & 1 ? high(sn[k / 2]) : low(sn[k / 2]);
          v = pair_of(low(v) * cc - high(v) * ss, low(v) * ss + high(v) * cc);
        };
        if (kKeep || R == D) {
#pragma unroll
          for (int k = 0; k < 4; ++k) turned(k);
        } else {  // (the others not by a turn of zero: y may be infinite)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (k < turning) turned(k);
        }
      } else if (apart) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint64_t x0 = va[k], y0 = vb[k];
          va[k] = fma2(x0, c[k], mul2(y0, sn[k] ^ 0x8000000080000000ull));
          vb[k] = fma2(x0, sn[k], mul2(y0, c[k]));
        }
      }
      Raw pa = P::pack(va), pb = P::pack(vb);
      if constexpr (kKeep) {
        if (R < D) {
          if (turning < 2) pa.y = ra[u].y;
          if (turning < 3) pb.x = rb[u].x;
          if (turning < 4) pb.y = rb[u].y;
        }
      }
      *reinterpret_cast<Raw *>(out + (r0 + u) * out_step) = pa;
      *reinterpret_cast<Raw *>(out + (r0 + u) * out_step + step) = pb;
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
  const uint32_t place = (uint32_t)(r / a.heads);  // at most 2^30
  int h = (int)(r - (long long)place * a.heads);
  const int s = place / (uint32_t)a.tokens, t = place - (uint32_t)s * a.tokens;
  if (t >= tokens_of(a, s)) return;
  int i = 0;
  while (i + 1 < a.sets && h >= a.set[i].heads) h -= a.set[i++].heads;
  const HeadSet &x = a.set[i];
  const T *in = static_cast<const T *>(x.in) + s * x.is + t * x.it + h * x.ih;
  float v[E];
  T raw[E];
#pragma unroll
  for (int e = 0; e < E; ++e) raw[e] = in[lane + 32 * e], v[e] = Elem<T>::load1(raw, e);
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
    const float inv = rsqrtf(sum * (1.f / D) + a.eps);
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
    if (ch >= R && (NORM == 0 || !x.norm)) {  // as it was read: a NaN's bits too
      out[ch] = raw[e];
      continue;
    }
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
cudaError_t launch(HeadsArgs a, cudaStream_t s) {
  constexpr int kSlots = kHeadThreads / (D / 8);
  const long long places = (long long)a.seqs * a.tokens;
  if (a.rope.layout == HKV_ROPE_HALF && a.rope.rot_dim / 2 % 4 != 0) {
    constexpr int kRows = kHeadThreads / 32;
    const long long rows = places * a.heads, grid = (rows + kRows - 1) / kRows;
    if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
    return pdl_launch(heads_any_kernel<T, D, NORM>, (int)grid, kHeadThreads, 0, s, a, rows);
  }
  // several heads a thread as soon as the device is full (four blocks an SM): a
  // thread's start, the angles above all, takes as many instructions as ten rows.
  // 8 x 4288 tokens, 96 heads of 128, bf16, layer norms: 344 us with at most 8, 311
  // with 16, 296 with 32.
  const long long once = 608LL * kSlots, want = (places * a.heads + once - 1) / once;
  const int iters = (int)(want < 32 ? want : 32);
  long long grid = 0;
  for (int i = 0; i < a.sets; ++i) {
    HeadSet &x = a.set[i];
    x.per = (x.heads + iters - 1) / iters;
    x.chunks = 1;
    if (x.per > kSlots) {
      x.chunks = (x.heads + kSlots * iters - 1) / (kSlots * iters);
      x.per = kSlots;
    }
    x.tokens = kSlots / x.per;
    x.chunk = (x.heads + x.chunks - 1) / x.chunks;
    x.most = (x.chunk + x.per - 1) / x.per;
    x.first_block = (int)grid;
    grid += (places + x.tokens - 1) / x.tokens * x.chunks;
    if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  }
  // Rows on their way at a time. With two the code is shorter: the smallest calls
  // take 3.2 us instead of 3.4, 64 rows of 96 heads 4.9 instead of 5.5; the largest
  // 342 instead of 296.
  const bool pairs = a.rope.layout == HKV_ROPE_PAIRS;
  auto *kernel = iters > 2 ? pairs ? heads_kernel<T, D, NORM, true, 4> : heads_kernel<T, D, NORM, false, 4>
                 : pairs   ? heads_kernel<T, D, NORM, true, 2>
                           : heads_kernel<T, D, NORM, false, 2>;
  return pdl_launch(kernel, (int)grid, kHeadThreads, 0, s, a, (uint32_t)places);
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
