// Decode attention over a cache in 8 or 4 bits, with or without the append of
// the step's new token: one launch per layer.
//
// Two kernels, by the longest segment the config allows. Up to kHeadRows rows a
// CTA takes a whole head (quant_head_kernel). Else (quant_attn_kernel):
//
// The layer's rows, head after head in tiles of 32, are cut into equal runs of
// tiles, one per warp of a grid that fills the device once. A warp streams its
// run through its own ring of tiles in shared memory, whatever heads it
// crosses, with a running maximum, sum and accumulator per head. The part of a
// head that a warp holds (a piece) is written out at once if it is the whole
// head. Else the CTA joins its warps' pieces in shared memory, and a head that
// is cut between CTAs leaves partial results in the workspace: the CTA that
// arrives last at the head's counter joins them, in CTA order, so the result
// does not depend on who is last. No CTA waits for another.
//
// Every CTA reads the layer's lengths to find its run, so a step may advance a
// head's counters only when all have (advance_or_leave).
#include "hkv_quant.cuh"
#include "hkv_quant.h"
#include "hkv_quant_tile.cuh"
#include "hkv_select.cuh"

namespace hkv {
namespace {

// Short segments: a CTA per head, its warps taking the head's tiles in turn,
// the first STAGES of each in flight at once (all of them, as launched);
// nothing outlives the CTA.
constexpr int kHeadWarps = 4;

template <int D, typename T, int BITS, bool STEP, int STAGES>
__global__ void __launch_bounds__(kHeadWarps * 32, STAGES == 1 ? 6 : 4)
    quant_head_kernel(const QAttnArgs p) {
  using TL = TileOf<D, BITS>;
  constexpr int E = D / 32;
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ float s_acc[kHeadWarps][D];
  __shared__ float s_m[kHeadWarps], s_l[kHeadWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, hl = blockIdx.x;
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
    if (threadIdx.x == 0) set_err(p.q8.c.err, hd.bad);
    return;
  }
  auto load = [&](int tile, int st) {
    const int r0 = tile * kTile;
    load_tile<D, BITS>(ws + st * TL::kBytes, p.q8, hd.off + r0, min(kTile, hd.len - r0));
  };
#pragma unroll
  for (int st = 0; st < STAGES; ++st) {
    if (warp + st * kHeadWarps < hd.tiles) load(warp + st * kHeadWarps, st);
    cp_async_commit();
  }
  if (p.prefetch) {
    pdl_wait();  // the step's inputs are visible from here on
    load_query<D, T>(p, hl, qv);
  }
  pdl_launch_dependents();
  NewRow nr;
  const int new_tile = hd.len / kTile;  // its warp: the last with a tile
  if (STEP && new_tile % kHeadWarps == warp) load_new_row<D, T>(p, hl, nr);
  float m = -INFINITY, l = 0.f;
  if (warp < hd.tiles && hd.n > 0) {
    float acc[D / 16][2] = {};
    __half *operand = reinterpret_cast<__half *>(ws + STAGES * TL::kBytes);
    const Query<D, BITS> qr = make_query<D, BITS>(qv, p.qscale, operand);
    int st = 0;
    for (int tile = warp; tile < hd.tiles; tile += kHeadWarps) {
      cp_async_wait<STAGES - 1>();
      __syncwarp();
      unsigned char *stage = ws + st * TL::kBytes;
      const int r0 = tile * kTile, rows = min(kTile, hd.n - r0);
      if (STEP && tile == new_tile)
        append_row<D, T, BITS>(p, hl, hd, stage, hd.len - r0, nr, qv);
      attend_tile<D, BITS>(stage, rows, qr, m, l, acc);
      if (STAGES == 1) break;  // no warp has a second tile
      __syncwarp();            // the stage and the weights are rewritten from here on
      if (tile + STAGES * kHeadWarps < hd.tiles) load(tile + STAGES * kHeadWarps, st);
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
  for (int w = 0; w < kHeadWarps; ++w)
    if (s_l[w] != 0.f) add_piece<E>(m, l, o, s_m[w], s_l[w], &s_acc[w][lane * E]);
  finish_head<D>(p, hl, m, l, o);
  if (STEP && lane == 0) advance_head(p, hl, hd.dense);
}

// Warps of a CTA and tiles in flight of a warp, two CTAs an SM: as much of an
// SM's shared memory as goes into whole tiles, or as many warps as registers.
template <int RB>
struct Shape {
  static constexpr int kWarps = RB == 128 ? 6 : RB == 64 ? 7 : 8, kStages = 2;
};

// Shared memory of a warp: its tiles, the operand area, and the piece of the
// head its run starts inside.
template <int D, int BITS>
struct Smem {
  using R = QRow<D, BITS>;
  static constexpr int kWarps = Shape<R::kBytes>::kWarps, kStages = Shape<R::kBytes>::kStages;
  static constexpr int kStage = TileOf<D, BITS>::kBytes;
  static constexpr int kOperand = kStages * kStage;
  static constexpr int kPiece = kOperand + TileOf<D, BITS>::kOperand;  // fp32 [D]
  static constexpr int kWarp = kPiece + D * 4;
  static constexpr int kTotal = kWarps * kWarp;
  static_assert(kStage >= D * 4, "the last piece takes a tile's place");
};

// A finished head's counters may advance when every CTA has read the lengths.
// done[0] counts the CTAs that have (and wraps to zero at the last one, so that
// it reads zero from then on and at the next launch). Who finishes a head
// earlier than that leaves it: a mark in count[], counted in done[1]. The CTA
// that reads last takes the marks over; between the two, whoever takes the
// mark out advances the head.
constexpr uint32_t kLeft = 0x80000000u;

__device__ __forceinline__ void take_left(const QAttnArgs &p, int hl, bool dense) {
  if (atomicCAS(p.count + hl, kLeft, 0u) != kLeft) return;
  atomicSub(p.done + 1, 1u);
  advance_head(p, hl, dense);
}
// `reported`: whether this CTA has (zero also means that none has yet)
__device__ __forceinline__ bool all_read(const QAttnArgs &p, volatile int *reported) {
  if (!*reported) return false;
  uint32_t v;
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p.done) : "memory");
  return v == 0u;
}
__device__ __forceinline__ void advance_or_leave(const QAttnArgs &p, int hl, bool dense,
                                                 volatile int *reported, bool known = false) {
  if (known || all_read(p, reported)) {
    advance_head(p, hl, dense);
    return;
  }
  atomicAdd(p.done + 1, 1u);
  atomicExch(p.count + hl, kLeft);
  __threadfence();  // the mark, then the look back; the last reader the other way round
  if (all_read(p, reported)) take_left(p, hl, dense);
}

template <int D, typename T, int BITS, bool STEP>
__global__ void __launch_bounds__(Smem<D, BITS>::kWarps * 32, 2)
    quant_attn_kernel(const QAttnArgs p) {
  using SM = Smem<D, BITS>;
  constexpr int E = D / 32;
  constexpr int WARPS = SM::kWarps, STAGES = SM::kStages, THREADS = WARPS * 32;
  constexpr int PF = D + 4;          // floats of a partial result
  constexpr int KM = D / 16;         // products per 16 rows, scores and output alike
  extern __shared__ __align__(16) unsigned char dyn[];
  // the runs' first heads, and those heads' first tiles in the layer
  __shared__ int s_head[WARPS], s_base[WARPS], s_scan[33];
  __shared__ HeadRef s_ref[WARPS];
  __shared__ int s_reported;
  // pieces of heads that a warp does not hold whole: [0] its run starts inside
  // the head, [1] the head starts in its run
  __shared__ float s_m[WARPS][2], s_l[WARPS][2];
  __shared__ int s_piece[WARPS][2];  // head, -1 for none
  __shared__ int s_ends[WARPS][2];   // whether the head ends with the piece
  __shared__ int s_first[WARPS][2], s_tiles[WARPS][2];  // the head's first tile and tiles
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const CacheArgs &c = p.q8.c;
  if (!p.prefetch) pdl_wait();

  // the runs: an exclusive scan of the heads' tiles, a stretch of heads a
  // thread; each warp gets `share` tiles, the first `rest` warps one more
  const int hp = (p.nheads + THREADS - 1) / THREADS;
  const int h0 = min(tid * hp, p.nheads), h1 = min(h0 + hp, p.nheads);
  // (up to two heads a thread, with all that the runs' first heads need)
  HeadRef ref[2] = {};
  int mine = 0;
  if (hp <= 2) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (h0 + j < h1) {
        ref[j] = head_ref<STEP>(p, h0 + j);
        mine += ref[j].tiles;
      }
    }
  } else {
#pragma unroll 8
    for (int h = h0; h < h1; ++h) mine += head_tiles<STEP>(c.len[p.base + h], p.max_rows);
  }
  int total;
  const int before = block_excl_scan<int>(mine, s_scan, &total);
  const int ctas = min((int)gridDim.x, (total + WARPS - 1) / WARPS);
  const int share = total / (ctas * WARPS), rest = total - share * ctas * WARPS;
  const int cta = blockIdx.x;
  auto run_start = [&](int w) { return w * share + min(w, rest); };
  const int run0 = run_start(cta * WARPS + warp);
  int left = cta < ctas ? run_start(cta * WARPS + warp + 1) - run0 : 0;
  if (cta < ctas) {
    if (tid < WARPS * 2) s_piece[tid >> 1][tid & 1] = -1;
    if (tid == 0) s_reported = 0;
#pragma unroll 1
    for (int w = 0; w < WARPS; ++w) {
      const int t = run_start(cta * WARPS + w);
      if (t >= before && t < before + mine) {
        int at = before, h = h0;
        if (hp <= 2) {
          const bool second = t >= before + ref[0].tiles;
          h += second;
          at += second ? ref[0].tiles : 0;
          s_ref[w] = second ? ref[1] : ref[0];
        } else {
          for (; h < h1 - 1; ++h) {
            const int nt = head_tiles<STEP>(c.len[p.base + h], p.max_rows);
            if (t < at + nt) break;
            at += nt;
          }
          s_ref[w] = head_ref<STEP>(p, h);
        }
        s_head[w] = h;
        s_base[w] = at;
      }
    }
    __syncthreads();
  }
  unsigned char *ws = dyn + warp * SM::kWarp;

  // the ring: tiles of the run in order, old rows only
  int pl_left = left, pl_head = 0, pl_tile = 0, pl_st = 0;
  HeadRef pr = {};
  if (left > 0) {
    pl_head = s_head[warp];
    pl_tile = run0 - s_base[warp];
    pr = s_ref[warp];
  }
  HeadRef hd = pr;
  auto issue = [&]() {
    if (pl_left > 0) {
      const int r0 = pl_tile * kTile;
      const int rows = pr.bad ? 0 : min(kTile, pr.len - r0);
      load_tile<D, BITS>(ws + pl_st * SM::kStage, p.q8, pr.off + r0, rows);
      ++pl_tile;
      --pl_left;
      if (pl_tile == pr.tiles && pl_left > 0) {
        pl_tile = 0;
        pr = head_ref<STEP>(p, ++pl_head);
      }
    }
    cp_async_commit();
    pl_st = pl_st + 1 == STAGES ? 0 : pl_st + 1;
  };
#pragma unroll
  for (int st = 0; st < STAGES; ++st) issue();
  if (p.prefetch) pdl_wait();  // the step's inputs are visible from here on
  pdl_launch_dependents();
  if (STEP && warp == WARPS - 1) {
    // this CTA's runs are found (the barrier above): it has read the lengths
    uint32_t old = 0;
    if (lane == 0) {
      old = atomicInc(p.done, gridDim.x - 1u);
      *reinterpret_cast<volatile int *>(&s_reported) = 1;
    }
    if (__shfl_sync(0xFFFFFFFFu, old, 0) == gridDim.x - 1u) {  // the last to
      __threadfence();
      uint32_t marks = 0;
      if (lane == 0) marks = *reinterpret_cast<volatile uint32_t *>(p.done + 1);
      if (__shfl_sync(0xFFFFFFFFu, marks, 0) != 0u)
        for (int h = lane; h < p.nheads; h += 32)
          if (*reinterpret_cast<volatile uint32_t *>(p.count + h) == kLeft)
            take_left(p, h, c.label[p.base + h] == HKV_DENSE);
    }
  }

  if (left > 0) {
    int hl = s_head[warp], base = s_base[warp], tile = run0 - base, st = 0;
    HeadRef nx = hd;
    float qv[E], qn[E];  // this head's query, the next one's
    load_query<D, T>(p, hl, qn);
    __half *operand = reinterpret_cast<__half *>(ws + SM::kOperand);

    while (left > 0) {
      // a head: this warp's piece of it
      const int from = tile;
      const bool more = left > hd.tiles - tile;  // another head follows in the run
#pragma unroll
      for (int e = 0; e < E; ++e) qv[e] = qn[e];
      if (more) {
        nx = head_ref<STEP>(p, hl + 1);
        load_query<D, T>(p, hl + 1, qn);
      }
      if (hd.bad && tile == 0 && lane == 0) set_err(c.err, hd.bad);
      NewRow nr;
      const int new_tile = STEP && !hd.bad ? hd.len / kTile : -1;
      const bool appends = new_tile >= tile && new_tile - tile < left;
      if (appends) load_new_row<D, T>(p, hl, nr);
      const Query<D, BITS> qr = make_query<D, BITS>(qv, p.qscale, operand);
      float m = -INFINITY, l = 0.f;
      float acc[KM][2];
#pragma unroll
      for (int x = 0; x < KM; ++x) acc[x][0] = acc[x][1] = 0.f;

      for (; tile < hd.tiles && left > 0; ++tile, --left) {
        cp_async_wait<STAGES - 1>();
        __syncwarp();
        unsigned char *stage = ws + st * SM::kStage;
        const int r0 = tile * kTile;
        const int rows = hd.bad ? 0 : min(kTile, hd.n - r0);
        if (STEP && appends && tile == new_tile)
          append_row<D, T, BITS>(p, hl, hd, stage, hd.len - r0, nr, qv);
        if (rows > 0) attend_tile<D, BITS>(stage, rows, qr, m, l, acc);
        __syncwarp();  // the stage and the weights are rewritten from here on
        issue();
        st = st + 1 == STAGES ? 0 : st + 1;
      }
      // the piece: [from, tile) of the head's tiles
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
      if (!hd.bad) {
        const bool starts = from == 0, ends = tile == hd.tiles;
        // a piece that outlives the head is the run's last unless the run
        // started inside it: the ring has no tile in flight by then
        float *to = reinterpret_cast<float *>(starts ? ws : ws + SM::kPiece);
        if (starts && ends) to = reinterpret_cast<float *>(ws + SM::kOperand);
        store_acc<D>(to, acc);
        __syncwarp();
        if (starts && ends) {
          float o[E];
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = to[lane * E + e];
          finish_head<D>(p, hl, m, l, o);
          if (STEP && lane == 0) advance_or_leave(p, hl, hd.dense, &s_reported);
        } else if (lane == 0) {
          const int slot = starts ? 1 : 0;
          s_m[warp][slot] = m;
          s_l[warp][slot] = l;
          s_piece[warp][slot] = hl;
          s_ends[warp][slot] = ends;
          s_first[warp][slot] = base;
          s_tiles[warp][slot] = hd.tiles;
        }
        __syncwarp();
      }
      if (left > 0) {
        ++hl;
        base += hd.tiles;
        tile = 0;
        hd = nx;
      }
    }
  }
  const bool early = STEP && lane == 0 && all_read(p, &s_reported);  // (stays so)
  __syncthreads();

  // pieces joined: a warp those of the head that starts in its run, warp 0
  // (which has a run if any has) also those of the head the run starts inside
  if (cta < ctas) {
    auto piece = [&](int w, int slot) {
      return reinterpret_cast<const float *>(dyn + w * SM::kWarp + (slot ? 0 : SM::kPiece)) +
             lane * E;
    };
    // (the middle warp does the latter: its own run seldom starts a head too)
#pragma unroll 1
    for (int slot = 1; slot >= 0; --slot) {
      if (slot == 0 && warp != WARPS / 2) break;
      const int from = slot ? warp : 0;
      const int h = s_piece[from][slot];
      if (h < 0) continue;
      float m = s_m[from][slot], l = s_l[from][slot], o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = piece(from, slot)[e];
      bool ends = s_ends[from][slot];
      for (int w = from + 1; w < WARPS && !ends; ++w) {
        if (s_piece[w][0] != h) continue;  // a warp without a run
        add_piece<E>(m, l, o, s_m[w][0], s_l[w][0], piece(w, 0));
        ends = s_ends[w][0];
      }
      // (its label does not change; its length only once it is finished)
      const bool dense = STEP ? c.label[p.base + h] == HKV_DENSE : false;
      if (slot == 1 && ends) {
        finish_head<D>(p, h, m, l, o);
        if (STEP && lane == 0) advance_or_leave(p, h, dense, &s_reported, early);
        continue;
      }
      // cut between CTAs: those of the head's first and last tile, and between
      auto cta_of = [&](int t) {
        const int longer = rest * (share + 1);  // tiles of the warps with one more
        const int w = t < longer ? t / (share + 1) : rest + (t - longer) / share;
        return w / WARPS;
      };
      const int c0 = cta_of(s_first[from][slot]);
      const int c1 = cta_of(s_first[from][slot] + s_tiles[from][slot] - 1);
      // where all others have been, this one has no need to leave its part
      uint32_t seen = 0;
      if (lane == 0)
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];"
                     : "=r"(seen)
                     : "l"(p.count + h)
                     : "memory");
      const bool others = __shfl_sync(0xFFFFFFFFu, seen, 0) == (uint32_t)(c1 - c0);
      if (!others) {
        float *part = p.part + ((size_t)cta * 2 + slot) * PF;
        store_row<E>(part + lane * E, o);
        if (lane == 0) *reinterpret_cast<float2 *>(part + D) = make_float2(m, l);
        __syncwarp();
        if (lane == 0)  // releases the warp's part, acquires the others'
          asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;"
                       : "=r"(seen)
                       : "l"(p.count + h)
                       : "memory");
        if (__shfl_sync(0xFFFFFFFFu, seen, 0) != (uint32_t)(c1 - c0)) continue;
      }
      // joined in CTA order, this one's part from here
      const float my_m = m, my_l = l;
      float my_o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) my_o[e] = o[e];
      m = -INFINITY, l = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
      for (int j0 = c0; j0 <= c1; j0 += 32) {  // a lane per part, then all of it
        const int n = min(32, c1 - j0 + 1);
        auto part_of = [&](int j) {
          return p.part + ((size_t)(j0 + j) * 2 + (j0 + j == c0)) * PF;
        };
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < n) ml = __ldcg(reinterpret_cast<const float2 *>(part_of(lane) + D));
        if (j0 + lane == cta) ml = make_float2(my_m, my_l);
        float v[4][E];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < n) load_row<E>(part_of(j) + lane * E, v[j]);
        auto mine_at = [&](int j, float (&x)[E]) {
          if (j0 + j == cta) {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = my_o[e];
          }
        };
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
            mine_at(j1 + j, v[j]);
            if (j1 + j < n) {
#pragma unroll
              for (int e = 0; e < E; ++e) o[e] += v[j][e] * gj;
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (j1 + 4 + j < n) load_row<E>(part_of(j1 + 4 + j) + lane * E, v[j]);
        }
      }
      finish_head<D>(p, h, m, l, o);
      if (lane == 0) {
        p.count[h] = 0u;
        if (STEP) advance_or_leave(p, h, dense, &s_reported, early);
      }
    }
  }
}

// Rows up to which a CTA takes a head whole: every tile in flight at once.
constexpr int kHeadRows = 2 * kHeadWarps * kTile;

template <int D, typename T, int BITS, bool STEP, int STAGES>
cudaError_t launch_heads(const QAttnArgs &a, cudaStream_t s) {
  using TL = TileOf<D, BITS>;
  constexpr int smem = kHeadWarps * (STAGES * TL::kBytes + TL::kOperand);
  static std::atomic<uint64_t> ready{0};
  cudaError_t e = allow_smem_of(quant_head_kernel<D, T, BITS, STEP, STAGES>, smem, ready);
  if (e != cudaSuccess) return e;
  return pdl_launch(quant_head_kernel<D, T, BITS, STEP, STAGES>, a.nheads, kHeadWarps * 32, smem,
                    s, a);
}

template <int D, typename T, int BITS, bool STEP>
cudaError_t launch(const QAttnArgs &a, cudaStream_t s) {
  if (a.max_rows <= kHeadWarps * kTile) return launch_heads<D, T, BITS, STEP, 1>(a, s);
  if (a.max_rows <= kHeadRows) return launch_heads<D, T, BITS, STEP, 2>(a, s);
  using SM = Smem<D, BITS>;
  static std::atomic<uint64_t> ready{0};
  cudaError_t e = allow_smem_of(quant_attn_kernel<D, T, BITS, STEP>, SM::kTotal, ready);
  if (e != cudaSuccess) return e;
  // two CTAs an SM, or a warp for every tile there can be
  const long long tiles = (long long)a.nheads * ((a.max_rows + kTile - 1) / kTile);
  const long long want = (tiles + SM::kWarps - 1) / SM::kWarps;
  const int full = 2 * a.sms < kQuantMaxGrid ? 2 * a.sms : kQuantMaxGrid;
  const int grid = (int)(want < full ? want : full);
  return pdl_launch(quant_attn_kernel<D, T, BITS, STEP>, grid, SM::kWarps * 32, SM::kTotal, s, a);
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
