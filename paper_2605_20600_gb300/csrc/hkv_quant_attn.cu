// Decode attention over a cache in 8 or 4 bits, with or without the append of
// the step's new token: one launch per layer.
//
// A CTA of four warps takes a head, or, of heads that are long and few, one of
// several equal parts of each head's tiles of 32 rows. Its warps take the tiles
// in turn, each through its own ring of tiles in shared memory with its own
// running maximum, sum and accumulator, and are joined in shared memory. The
// parts of a head are left in the workspace and joined, in order, by the CTA
// that arrives last at the head's counter, so the result does not depend on who
// is last. No CTA waits for another.
//
// A step's CTAs all read a head's length to find their part, so its counters
// advance only when all of them have arrived, those without a part too.
//
// What bounds it: DRAM for rows of 128 bytes, 65537 x 32 of them take 96 us
// (5.9 TB/s), the issue of ~600 instructions a tile for rows of 32 bytes, 43 us
// (3.5 TB/s); and for short segments the launch, one round trip to memory and
// the join, 4 to 5 us a layer, some of which the next layer's CTAs hide: with
// HKV_STEP_PREFETCH they load their first tiles before they wait. A kernel that
// streamed equal runs of tiles, whatever heads they cross, through a grid of two
// CTAs an SM balances unequal heads but pays a scan of the lengths and two joins
// and leaves no room for the next layer's CTAs: 135 us for eight layers of 256
// heads of up to 1235 rows of 128 bytes (112 us here), 8 against 4.5 us a layer
// of short heads.
#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_quant_tile.cuh"
#include "hkv_select.cuh"

namespace hkv {
namespace {

constexpr int kWarps = 4;
constexpr int kSmSmem = 228 << 10;  // shared memory of an SM
// Least tiles of a part of a head, two a warp. Four layers of 8 heads of 38 tiles
// take 27 us (30 with 16); with 4, one head of 1563 tiles has 391 parts to join
// (35 us; 27 with 8, 18 with the 64 or so that cut_of finds).
constexpr int kPartTiles = 8;

// CTAs an SM has room for, with two tiles of a warp in flight
template <int D, int BITS>
constexpr int kMostResident = QRow<D, BITS>::kBytes == 128 ? 3 : 4;

// `SPLIT`: a head may be cut between CTAs. STAGES: tiles of a warp in flight.
template <int D, typename T, int BITS, bool STEP, int STAGES, bool SPLIT>
__global__ void __launch_bounds__(kWarps * 32, STAGES == 1   ? 7
                                               : STAGES == 3 ? 2
                                                             : kMostResident<D, BITS>)
    quant_attn_kernel(const QAttnArgs p) {
  using TL = TileOf<D, BITS>;
  constexpr int E = D / 32, PF = D + 4;  // PF: floats of a partial result
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ float s_acc[kWarps][D];
  __shared__ float s_m[kWarps], s_l[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = SPLIT ? blockIdx.x / p.nheads : 0;
  const int hl = SPLIT ? blockIdx.x - part * p.nheads : blockIdx.x;
  unsigned char *ws = dyn + warp * (STAGES * TL::kBytes + TL::kOperand);
  float qv[E];
  if (!p.prefetch) {
    pdl_wait();
    load_query<D, T>(p, hl, qv);
  }
  const HeadRef hd = head_ref<STEP>(p, hl);
  if (hd.bad) {
    pdl_wait();
    pdl_launch_dependents();
    if (threadIdx.x == 0 && part == 0) set_err(p.q8.c.err, hd.bad);
    return;
  }
  // this CTA's tiles of the head: [t0, t1), none beyond the head's parts
  const int parts = SPLIT ? max(1, min(p.splits, hd.tiles / kPartTiles)) : 1;
  int t0 = 0, t1 = hd.tiles;
  if (SPLIT) {
    t0 = part < parts ? (int)((long long)hd.tiles * part / parts) : hd.tiles;
    t1 = part < parts ? (int)((long long)hd.tiles * (part + 1) / parts) : hd.tiles;
    if (!STEP && part >= parts) return;
  }
  auto load = [&](int tile, int st) {
    const int r0 = tile * kTile;
    load_tile<D, BITS>(ws + st * TL::kBytes, p.q8, hd.off + r0, min(kTile, hd.len - r0));
  };
#pragma unroll
  for (int st = 0; st < STAGES; ++st) {
    if (t0 + warp + st * kWarps < t1) load(t0 + warp + st * kWarps, st);
    cp_async_commit();
  }
  if (p.prefetch) {
    pdl_wait();  // the step's inputs are visible from here on
    load_query<D, T>(p, hl, qv);
  }
  pdl_launch_dependents();
  NewRow nr;
  const int new_tile = hd.len / kTile;
  if (STEP && new_tile >= t0 && new_tile < t1 && (new_tile - t0) % kWarps == warp)
    load_new_row<D, T>(p, hl, nr);
  float m = kNoKey, l = 0.f;
  if (t0 + warp < t1 && hd.n > 0) {
    float acc[D / 16][2] = {};
    __half *operand = reinterpret_cast<__half *>(ws + STAGES * TL::kBytes);
    const Query<D, BITS> qr = make_query<D, BITS>(qv, operand);
    int st = 0;
    for (int tile = t0 + warp; tile < t1; tile += kWarps) {
      cp_async_wait<STAGES - 1>();
      __syncwarp();
      unsigned char *stage = ws + st * TL::kBytes;
      const int r0 = tile * kTile, rows = min(kTile, hd.n - r0);
      if (STEP && tile == new_tile)
        append_row<D, T, BITS>(p, hl, hd, stage, hd.len - r0, nr, qv);
      attend_tile<D, BITS>(stage, rows, qr, p.qscale, m, l, acc);
      if (STAGES == 1) break;  // no warp has a second tile
      __syncwarp();            // the stage is rewritten from here on
      if (tile + STAGES * kWarps < t1) load(tile + STAGES * kWarps, st);
      cp_async_commit();
      st = st + 1 == STAGES ? 0 : st + 1;
    }
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    store_acc<D>(s_acc[warp], acc);
  }
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  __syncthreads();
  if (warp != 0) return;
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  m = -INFINITY, l = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w)
    if (s_l[w] != 0.f) add_piece<E>(m, l, o, s_m[w], s_l[w], &s_acc[w][lane * E]);

  if (SPLIT) {
    const uint32_t all = (STEP ? p.splits : parts) - 1;  // the other CTAs that arrive
    if (parts == 1 && part == 0) finish_head<D>(p, hl, m, l, o);
    if (all == 0) return;
    float *mine = p.part + ((size_t)hl * p.splits + part) * PF;
    uint32_t seen = 0;
    if (lane == 0)
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];"
                   : "=r"(seen)
                   : "l"(p.count + hl)
                   : "memory");
    // where all others have been, this one has no need to leave its part
    if (__shfl_sync(0xFFFFFFFFu, seen, 0) != all) {
      if (parts > 1 && part < parts) {
        store_row<E>(mine + lane * E, o);
        if (lane == 0) *reinterpret_cast<float2 *>(mine + D) = make_float2(m, l);
      }
      __syncwarp();
      if (lane == 0)  // releases the warp's part, acquires the others'
        asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;"
                     : "=r"(seen)
                     : "l"(p.count + hl)
                     : "memory");
      if (__shfl_sync(0xFFFFFFFFu, seen, 0) != all) return;
    }
    __syncwarp();  // what lane 0 has acquired is every lane's
    if (parts > 1) {
      // all parts joined in order, this CTA's from its registers
      const float my_m = m, my_l = l;
      float my_o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) my_o[e] = o[e];
      m = -INFINITY, l = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
      for (int j0 = 0; j0 < parts; j0 += 32) {  // a lane per part, then all of it
        const int n = min(32, parts - j0);
        auto part_of = [&](int j) { return p.part + ((size_t)hl * p.splits + j0 + j) * PF; };
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < n) ml = __ldcg(reinterpret_cast<const float2 *>(part_of(lane) + D));
        if (j0 + lane == part) ml = make_float2(my_m, my_l);
        float v[4][E];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < n) load_row<E>(part_of(j) + lane * E, v[j]);
        const float mn = fmaxf(m, warp_max(ml.x));
        const float f = l == 0.f ? 0.f : ex2_approx(m - mn);
        const float g = ml.y == 0.f ? 0.f : ex2_approx(ml.x - mn);
        float lj = ml.y * g;
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) lj += __shfl_xor_sync(0xFFFFFFFFu, lj, x);
        m = mn;
        l = l * f + lj;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= f;
        for (int j1 = 0; j1 < n; j1 += 4) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float gj = __shfl_sync(0xFFFFFFFFu, g, (j1 + j) & 31);
            const bool own = j0 + j1 + j == part;
            if (j1 + j < n) {
#pragma unroll
              for (int e = 0; e < E; ++e) o[e] += (own ? my_o[e] : v[j][e]) * gj;
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (j1 + 4 + j < n) load_row<E>(part_of(j1 + 4 + j) + lane * E, v[j]);
        }
      }
      finish_head<D>(p, hl, m, l, o);
    }
    if (lane == 0) p.count[hl] = 0u;
  } else {
    finish_head<D>(p, hl, m, l, o);
  }
  if (STEP && lane == 0) advance_head(p, hl, hd.dense);
}

// Dynamic shared memory with which at most `n` CTAs are resident on an SM.
constexpr int smem_for(int n) { return (kSmSmem / (n + 1) + 1023) / 1024 * 1024; }

template <int D, typename T, int BITS, bool STEP, int STAGES, bool SPLIT>
cudaError_t launch_as(const QAttnArgs &a, int resident, cudaStream_t s) {
  using TL = TileOf<D, BITS>;
  constexpr int need = kWarps * (STAGES * TL::kBytes + TL::kOperand);
  static std::atomic<uint64_t> ready{0};
  cudaError_t e = allow_smem_of(quant_attn_kernel<D, T, BITS, STEP, STAGES, SPLIT>,
                                std::max(need, smem_for(1)), ready);
  if (e != cudaSuccess) return e;
  // warps that no head has a tile for need no shared memory (2048 heads of up to
  // 84 rows of 128 bytes, capacity 96: 16.9 us a layer with it, 14.0 without)
  const int tiles = (a.max_rows + kTile - 1) / kTile;
  const int smem = resident ? std::max(need, smem_for(resident))
                            : need / kWarps * std::min(kWarps, tiles);
  return pdl_launch(quant_attn_kernel<D, T, BITS, STEP, STAGES, SPLIT>, a.nheads * a.splits,
                    kWarps * 32, smem, s, a);
}

// CTAs of a head of `tiles` tiles, and how many of them an SM is to have: those
// of least estimated time, were all heads as long. The second matters because an
// SM that has room takes more than its share while others have fewer: 256 heads
// with room for three CTAs an SM take 142 us where two take 117 (and with three
// tiles in flight in the room gained, 112); 512 heads of 2300 rows 70 against
// 56.
struct Cut {
  int splits, resident;
};
template <int D, int BITS>
Cut cut_of(int nheads, int tiles, int sms) {
  // ns of an SM per tile with 1 to 4 resident CTAs, measured; joining costs
  // kJoin and kPart for each part
  constexpr bool kWide = QRow<D, BITS>::kBytes == 128;
  constexpr int kTileNs[4] = {kWide ? 180 : 125, kWide ? 130 : 80, kWide ? 125 : 67, 60};
  constexpr int kJoin = 2000, kPart = 85;
  Cut best = {1, 0};
  long long least = 0;
  const int most = std::min(tiles / kPartTiles, kQuantMaxParts / nheads);
  for (int s = 1; s <= std::max(1, most); ++s) {
    const int r = (int)(((long long)nheads * s + sms - 1) / sms);
    if (r > kMostResident<D, BITS>) break;
    const long long t = (long long)r * ((tiles + s - 1) / s) * kTileNs[r - 1] +
                        (s > 1 ? kJoin + s * kPart : 0);
    if (best.resident == 0 || t < least) best = {s, r}, least = t;
  }
  if (best.resident == 0) {  // more heads than there is room for: equal rounds
    const int rounds = (nheads - 1) / (sms * kMostResident<D, BITS>) + 1;
    best.resident = (nheads + sms * rounds - 1) / (sms * rounds);
  }
  return best;
}

template <int D, typename T, int BITS, bool STEP>
cudaError_t launch(QAttnArgs a, cudaStream_t s) {
  const int tiles = (a.max_rows + kTile - 1) / kTile;
  a.splits = 1;
  // short segments: all tiles of a head in flight at once
  if (tiles <= kWarps) return launch_as<D, T, BITS, STEP, 1, false>(a, 0, s);
  if (tiles <= 2 * kWarps) return launch_as<D, T, BITS, STEP, 2, false>(a, 0, s);
  const Cut cut = cut_of<D, BITS>(a.nheads, tiles, a.sms);
  a.splits = cut.splits;
  if (cut.splits > 1) return launch_as<D, T, BITS, STEP, 2, true>(a, cut.resident, s);
  if (cut.resident <= 2)
    return launch_as<D, T, BITS, STEP, 3, false>(a, cut.resident, s);
  return launch_as<D, T, BITS, STEP, 2, false>(a, cut.resident, s);
}

}  // namespace

cudaError_t launch_quant_attention(const QAttnArgs &a, int D, int dtype, int bits,
                                   cudaStream_t s) {
#define HKV_QATTN(BITS_, STEP_) HKV_DISPATCH(D, dtype, return launch<kD, kT, BITS_, STEP_>(a, s))
  if (bits == HKV_Q8) {
    if (a.k_new) HKV_QATTN(8, true);
    HKV_QATTN(8, false);
  }
  if (a.k_new) HKV_QATTN(4, true);
  HKV_QATTN(4, false);
#undef HKV_QATTN
  return cudaErrorInvalidValue;
}

}  // namespace hkv
