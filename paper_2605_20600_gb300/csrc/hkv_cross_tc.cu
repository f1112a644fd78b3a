// Attention of more than 16 bf16 query rows over their sequence's states, with
// bf16 outs, on tcgen05.
//
// A CTA works on TILES query tiles of one (sequence, key head) and a range of keys
// in tiles of 64 (96 for heads of 64, which the weights bound: longer tiles wait
// less often). A query tile is 128 tokens of a head, or all tokens of a few heads of
// the group, 128 rows at most. One warp loads Q, and K and V tiles into a ring of
// slots (TMA); four warps a query tile, a thread per row, turn scores into weights:
// S = Q K^T lies in TMEM in two buffers, a thread reads its row of S, writes the
// weights as bf16 over it, and they are the A operand of O += W V, which stays in
// TMEM; a warp a query tile issues its products. A CTA that has issued the loads of
// its work takes over that of a CTA which was not launched yet, so that loads and
// first scores run beside the outs of the work before.
//
// A row's reference maximum moves (and O and its sum are rescaled) only when a
// tile's maximum is more than 2^8 above it, so that weights stay below 2^8. The
// weights are rounded to bf16, off by at most 2^-9 each, as the outs are; their
// sum is that of the fp32 weights. One query tile a CTA (few queries, where the
// loads take longer than the products) takes them in two parts, off by 2^-18.
//
// Rows of V past the last state are set to zero in shared memory (a weight of
// zero times what lies there could be NaN); scores past it are masked.
//
// What bounds it, heads of 128: the products, which keep the tensor pipe busy for
// 0.77 of the cycles (2 x 32 heads of 4096 queries and keys: 321 us, 1713 TFLOP/s;
// causal over 4288: 0.70, 225 us: key heads come one after the other, so that the last
// one's long tiles start late and end at 1.15 of the mean work of a CTA). On the way: products issued from divergent code,
// each operand's descriptor moved to uniform registers, 470;
// from uniform code, K and V in one wait, 387; S in two buffers, so that products
// and weights of a tile overlap, 341; the scores after the next behind a tile's
// W V, one wait a tile, 322. Two threads a row: 365 (their agreement on a maximum
// costs more than half of the exponentials); one warp for both tiles' products in
// turn: 387; tiles of 128 keys leave no room in TMEM for a second S. Heads of 64
// have half of the products: 269 us (306 in tiles of 64 keys), bound by the weights
// (96 exponentials a row and tile, and the chain around them). Short states: a
// piece of work's chain, 8 x 4160 queries of 32 heads over 120: 111 us, 5 TB/s (145
// with every warp working out what the next piece is, and 16-byte stores of outs).
#include <cuda.h>
#include <type_traits>

#include "hkv_cross.cuh"
#include "hkv_tcgen05.cuh"

namespace hkv {
namespace {

constexpr int kTile = 128;  // queries of a tile

template <int D, int TILES>
struct TcPlan {
  static constexpr int kThreads = TILES * 160 + 32;
  static constexpr int kKeys = D == 64 ? 96 : 64;   // of a tile: two buffers of S fill TMEM beside O
  static constexpr int kQ = kTile * D * 2, kKV = kKeys * D * 2;  // bytes of a query tile, of a K or V tile
  // slots of the ring: slot p % kSlots holds K of key tile p and V of tile p - 1,
  // which the products need together
  static constexpr int kSlots = TILES * (D == 64 ? 3 : 2);
  // channels of a row that go out at a time, through a warp's piece of shared memory
  static constexpr int kOut = TILES == 2 ? 64 : 32;
  // the outs by bulk copies: 8 x 4160 queries of 32 heads over 120 states, heads of
  // 128, 119 -> 111 us; of 64, whose rows are one piece, 113.7 -> 114.5
  static constexpr bool kCopyOut = D == 128 && TILES == 2;
  static constexpr int kBytes = 1024 + TILES * kQ + kSlots * 2 * kKV + TILES * 4 * 32 * kOut * 2;
  static constexpr int kParts = TILES == 1 ? 2 : 1;  // bf16 parts of a weight
  static constexpr int kCols = TILES * 256;         // TMEM: two buffers of S of each tile, then O of each
  static constexpr int kO = TILES * 2 * kKeys;
};

__device__ __forceinline__ void tma_tile(void *dst, const CUtensorMap *map, int c, int row, int head,
                                         int seq, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(c), "r"(row), "r"(head), "r"(seq), "r"(smem_u32(bar))
      : "memory");
}

__device__ __forceinline__ void tma_store(const CUtensorMap *map, const void *from, int c, int row, int head,
                                          int seq) {
  asm volatile(
      "cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3, %4}], [%5];\n"
      "cp.async.bulk.commit_group;" ::"l"(map),
      "r"(c), "r"(row), "r"(head), "r"(seq), "r"(smem_u32(from))
      : "memory");
}

// the query tiles of a CTA's work
template <int TILES>
struct Item {
  Work w;
  int lo;                            // first key
  int head0[TILES], token0[TILES];   // heads within the group
  int n[TILES], most;                // key tiles
  bool any;                          // rows to write
  bool none;                         // no work at all
};
template <int D, int TILES>
__device__ __forceinline__ Item<TILES> item_of(const CrossArgs &p, int index) {
  constexpr int kKeys = TcPlan<D, TILES>::kKeys;
  Item<TILES> x;
  x = {};
  if (index < 0) return x;
  x.w = work_of(p, index);
  x.lo = x.w.sp * p.split_len;
  // the heads of a group side by side: query tiles of a CTA see the same keys, and
  // have rows or none together
  const int head_tiles = (p.group + p.box_heads - 1) / p.box_heads;
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int u = x.w.tile * TILES + t, token_tile = u / head_tiles;
    x.head0[t] = (u - token_tile * head_tiles) * p.box_heads;
    x.token0[t] = token_tile * p.box_tokens;
    int hi = 0;
    const bool live = x.token0[t] < x.w.qlen;
    x.any |= live;
    if (live)
      hi = min(keys_seen(p, x.w, min(x.token0[t] + p.box_tokens, x.w.qlen) - 1), x.lo + p.split_len);
    x.n[t] = hi > x.lo ? (hi - x.lo + kKeys - 1) / kKeys : 0;
    x.most = max(x.most, x.n[t]);
  }
  return x;
}

template <int D, int TILES>
__global__ void __launch_bounds__(TcPlan<D, TILES>::kThreads, TILES == 2 ? 1 : 2)
    cross_tc_kernel(const __grid_constant__ CrossArgs p, const __grid_constant__ CUtensorMap qmap,
                    const __grid_constant__ CUtensorMap kmap,
                    const __grid_constant__ CUtensorMap vmap,
                    const __grid_constant__ CUtensorMap omap) {
  using TP = TcPlan<D, TILES>;
  constexpr int PF = D + 4, SLOTS = TP::kSlots, kKeys = TP::kKeys;
  extern __shared__ unsigned char dyn_raw[];
  __shared__ __align__(16) uint4 s_answer;            // to the load warp: another CTA's work
  __shared__ uint64_t s_asked;
  __shared__ Item<TILES> s_item[2];                   // the CTA's items, and whether they are
  __shared__ uint64_t s_nf[2], s_ne[2];               // there, and read by the other warps
  __shared__ uint64_t s_full[SLOTS], s_empty[SLOTS];  // slots of the ring
  __shared__ uint64_t s_s[TILES][2], s_p[TILES][2];   // S and W of a key tile are ready
  __shared__ uint64_t s_v[TILES];                     // O holds a key tile's products
  __shared__ uint64_t s_q[TILES], s_qe[TILES];        // Q is there; its last product is done
  __shared__ uint64_t s_oe[TILES];                    // O has been read
  __shared__ int s_left[TILES * 4];                   // item that a warp did not wait for, or -1
  __shared__ uint64_t s_edge, s_drain;
  __shared__ uint32_t s_tmem;
  unsigned char *dyn = dyn_raw + ((1024u - (smem_u32(dyn_raw) & 1023u)) & 1023u);
  unsigned char *ring = dyn + TILES * TP::kQ, *stage = ring + SLOTS * 2 * TP::kKV;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_nf[i], 1);
      mbar_init(&s_ne[i], TILES * 5);
    }
    for (int i = 0; i < TILES * 4; ++i) s_left[i] = -1;
    mbar_init(&s_asked, 1);
    for (int i = 0; i < SLOTS; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_empty[i], TILES);
    }
    for (int t = 0; t < TILES; ++t) {
      for (int b = 0; b < 2; ++b) {
        mbar_init(&s_s[t][b], 1);
        mbar_init(&s_p[t][b], 4);
      }
      mbar_init(&s_v[t], 1);
      mbar_init(&s_q[t], 1);
      mbar_init(&s_qe[t], 1);
      mbar_init(&s_oe[t], 4);
    }
    mbar_init(&s_edge, 1);
    mbar_init(&s_drain, TILES);
    fence_barrier_init();
  }
  // TMEM only after the wait, and the next kernel's CTAs only after TMEM: an
  // allocation waits for columns, so a CTA that held some while it waited for
  // the kernel before, or let a CTA of the kernel after take them first, could
  // wait for one that waits for it
  pdl_wait();
  if (warp == 0) {
    tmem_alloc(&s_tmem, TP::kCols);
    pdl_launch_dependents();
  }
  const Order order = order_of(p, [&](int tokens) {
    const int token_tiles = (tokens + p.box_tokens - 1) / p.box_tokens;
    return (token_tiles * ((p.group + p.box_heads - 1) / p.box_heads) + TILES - 1) / TILES;
  });
  Item<TILES> x = item_of<D, TILES>(p, piece_at(p, order, blockIdx.x));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, s_tmem, 0);
  // A wait that runs out fails all that the CTA has still to do: its warps then
  // only go through the items, and write NaN.
  bool ok = true;
  auto wait = [&](uint64_t *bar, uint32_t parity) {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity));
  };
  // The load warp finds the CTA's items, the work of CTAs that were not launched
  // yet; the others read them, k = 0, 1, ... behind the first, until there is none.
  auto next_item = [&](int k) {
    if (!wait(&s_nf[k & 1], (k >> 1) & 1)) return ok = false;
    x = s_item[k & 1];
    __syncwarp();
    if (lane == 0) mbar_arrive(&s_ne[k & 1]);
    return !x.none;
  };
  if (warp == TILES * 4) {
    // loads: Q and the ring's slots, as far ahead as there is room, of the next
    // item too
    uint32_t slots = 0, queries[TILES] = {}, edges = 0;  // so far
    uint32_t asked = 0;
    bool ahead = false;  // the next item has been asked for
    for (int k = 0; !x.none; ++k) {
      for (int j = 0; x.most > 0 && j <= x.most && ok; ++j, ++slots) {
        const uint32_t slot = slots % SLOTS;
        const int k0 = x.lo + j * kKeys, past = k0 - x.w.klen;
        if (slots >= SLOTS) ok = wait(&s_empty[slot], (slots / SLOTS - 1) & 1);
        if (!ok) break;
        unsigned char *dst = ring + slot * 2 * TP::kKV;
        // V's tile ends behind the sequence (past the last one's states there are zeros)
        const bool edge = past > 0 && x.w.klen < p.keys;
        if (lane == 0) {
          uint64_t *bar = edge ? &s_edge : &s_full[slot];
          mbar_arrive_expect_tx(bar, ((j < x.most) + (j > 0)) * TP::kKV);
#pragma unroll
          for (int c = 0; c < D; c += 64) {
            if (j < x.most) tma_tile(dst + (c >> 6) * kKeys * 128, &kmap, c, k0, x.w.kvh, x.w.s, bar);
            if (j > 0)
              tma_tile(dst + TP::kKV + (c >> 6) * kKeys * 128, &vmap, c, k0 - kKeys, x.w.kvh, x.w.s, bar);
          }
        }
        if (j == 0) {
#pragma unroll
          for (int t = 0; t < TILES; ++t) {
            if (x.n[t] == 0) continue;
            if (queries[t] > 0) ok = ok && wait(&s_qe[t], (queries[t] - 1) & 1);
            if (!ok) break;
            ++queries[t];
            if (lane == 0) {
              mbar_arrive_expect_tx(&s_q[t], p.box_tokens * p.box_heads * D * 2);
#pragma unroll
              for (int c = 0; c < D; c += 64)
                tma_tile(dyn + t * TP::kQ + (c >> 6) * kTile * 128, &qmap, c, x.token0[t],
                         x.w.kvh * p.group + x.head0[t], x.w.s, &s_q[t]);
            }
          }
        }
        if (edge) {
          ahead = k < 2 || __all_sync(0xFFFFFFFFu, mbar_test_wait(&s_ne[k & 1], ((k >> 1) - 1) & 1));
          if (ahead && lane == 0) next_cta_ask(&s_answer, &s_asked);
          ok = ok && wait(&s_edge, edges++ & 1);
          if (!ok) break;
          for (int e = lane; e < past * (D / 8); e += 32) {
            const int r = kKeys - past + e / (D / 8), c = e % (D / 8);
            *reinterpret_cast<uint4 *>(dst + TP::kKV + (c >> 3) * kKeys * 128 + r * 128 + ((c & 7) << 4)) =
                make_uint4(0, 0, 0, 0);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(&s_full[slot]);
        }
      }
      // The next item that has rows to write; asked for only now, so that what is
      // left at the end goes to the CTA that is free first. What has been taken over
      // nobody else does, so it is asked for only when there is room to hand it on
      // (`ahead` has made sure). The other warps may take the limit before they read
      // on, so this wait may take several.
      bool room = ahead || k < 2;
      for (int i = 0; i < 4 && !room; ++i) {
        room = wait(&s_ne[k & 1], ((k >> 1) - 1) & 1);
        ok = ok && room;
      }
      if (!room) break;
      do {
        if (!ahead && lane == 0) next_cta_ask(&s_answer, &s_asked);
        ahead = false;
        int item = -1;
        if (wait(&s_asked, asked++ & 1)) item = next_cta(&s_answer);
        else ok = false;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (item >= 0) x = item_of<D, TILES>(p, piece_at(p, order, item));
        else x.none = true;
      } while (!x.any && !x.none);
      if (lane == 0) {
        s_item[k & 1] = x;
        mbar_arrive(&s_nf[k & 1]);
      }
    }
    if (!ok) {  // what was issued may still run: the limit once more
      for (uint32_t j = slots > SLOTS ? slots - SLOTS : 0; j < slots; ++j)
        mbar_wait(&s_full[j % SLOTS], (j / SLOTS) & 1);
#pragma unroll
      for (int t = 0; t < TILES; ++t)
        if (queries[t] > 0) mbar_wait(&s_q[t], (queries[t] - 1) & 1);
    }
  } else if (warp > TILES * 4) {
    // products of one query tile, issued by one lane; the whole warp waits. A warp
    // for each tile, so that one's products run while the other waits. With two
    // query tiles the scores of two key tiles are computed ahead; then a key tile's
    // weights take their V, and the scores of the tile after the next take the place
    // that they leave: one wait for 512 cycles of products. With one, whose ring is
    // shorter, the scores of the next tile only, before the weights are there.
    const int t = warp - TILES * 4 - 1;
    const uint32_t ring_at = smem_u32(ring), at_s = tmem + t * 2 * kKeys, at_o = tmem + TP::kO + t * D;
    const uint64_t qd = tc_desc(smem_u32(dyn) + t * TP::kQ, 16);
    uint32_t slots = 0, queries = 0, steps = 0;  // used so far: slots, items, key tiles
    auto here = [&](uint32_t j) { return wait(&s_full[j % SLOTS], (j / SLOTS) & 1); };
    auto scores = [&](uint32_t step, uint32_t j, bool last) {  // S with the K tile of slot j
      const uint64_t kd = tc_desc(ring_at + (j % SLOTS) * 2 * TP::kKV, 16);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)  // 16 channels: 32 bytes of a column block
        tc_mma(at_s + (step & 1) * kKeys, qd + (((ks >> 2) * kTile * 128 + (ks & 3) * 32) >> 4),
               kd + (((ks >> 2) * kKeys * 128 + (ks & 3) * 32) >> 4), tc_instr(kTile, kKeys, false),
               ks > 0);
      tc_commit(&s_s[t][step & 1]);
      if (last) tc_commit(&s_qe[t]);
    };
    int k = 0;
    do {
      const int n = TILES == 2 && t ? x.n[TILES - 1] : x.n[0];
      if (n > 0 && ok) {
        ok = here(slots) && wait(&s_q[t], queries++ & 1);
        if (ok) {
          tc_fence_after();
          if (elect_one()) {
            scores(steps, slots, n == 1);
            tc_commit(&s_empty[slots % SLOTS]);
          }
          __syncwarp();
          if (TILES == 2) ok = here(slots + 1);
          if (ok && TILES == 2 && n > 1) {
            tc_fence_after();
            if (elect_one()) scores(steps + 1, slots + 1, n == 2);
            __syncwarp();
          }
          if (ok && queries > 1) ok = wait(&s_oe[t], queries & 1);  // O of the item before has been read
        }
      }
      for (int i = 0; i < n && ok; ++i, ++steps) {
        const uint32_t j = slots + i + 1, b = steps & 1;  // the slot of V; of K after the next: j + 1
        uint64_t *weights = &s_p[t][b], *keys = &s_full[(j + 1) % SLOTS];
        const uint32_t wp = (steps >> 1) & 1, kp = ((j + 1) / SLOTS) & 1;
        if (TILES == 2) {
          const bool w_here = mbar_try_wait(weights, wp), k_here = i + 2 > n || mbar_try_wait(keys, kp);
          if (!__all_sync(0xFFFFFFFFu, w_here && k_here))
            ok = wait(weights, wp) && (i + 2 > n || wait(keys, kp));
        } else {
          ok = here(j);
          if (ok && i + 1 < n) {
            tc_fence_after();
            if (elect_one()) scores(steps + 1, j, i + 2 == n);
            __syncwarp();
          }
          ok = ok && wait(weights, wp);
        }
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t vd = tc_desc(ring_at + (j % SLOTS) * 2 * TP::kKV + TP::kKV, kKeys * 128);
#pragma unroll
          for (int part = TP::kParts - 1; part >= 0; --part)  // the small part first
#pragma unroll
            for (int kk = 0; kk < kKeys / 16; ++kk)
              tc_mma_ta(at_o, at_s + b * kKeys + part * (kKeys / 2) + kk * 8, vd + kk * (16 * 128 >> 4),
                        tc_instr(kTile, D, true), i > 0 || kk > 0 || part < TP::kParts - 1);
          tc_commit(&s_v[t]);
          if (TILES == 2 && i + 2 < n) scores(steps + 2, j + 1, i + 3 == n);
          tc_commit(&s_empty[j % SLOTS]);
        }
        __syncwarp();
      }
      // slots that only the other tile uses are given back as they come
      for (int j = n == 0 ? 0 : n + 1; x.most > 0 && j <= x.most && ok; ++j) {
        ok = here(slots + j);
        if (ok && lane == 0) mbar_arrive(&s_empty[(slots + j) % SLOTS]);
      }
      if (x.most > 0) slots += x.most + 1;
    } while (next_item(k++));
    if (!ok && elect_one()) {
      set_err(p.err, HKV_ERR_TIMEOUT);
      tc_commit(&s_drain);
    }
    if (ok && elect_one()) mbar_arrive(&s_drain);
    if (!ok) mbar_wait(&s_drain, 0);
  } else {
    const int t = warp >> 2, r = tid & 127, h = r / p.box_tokens, token_in = r - h * p.box_tokens;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t mine = tmem + t * 2 * kKeys + lanes, mine_o = tmem + TP::kO + t * D + lanes;
    unsigned char *rows = stage + warp * 32 * TP::kOut * 2;
    uint32_t steps = 0;                         // key tiles so far
    int k = 0;
    do {
      const int n = TILES == 2 && t ? x.n[TILES - 1] : x.n[0];
      const int first = TILES == 2 && t ? x.token0[TILES - 1] : x.token0[0];
      const int head0 = TILES == 2 && t ? x.head0[TILES - 1] : x.head0[0], token = first + token_in;
      const int seen = min(keys_seen(p, x.w, token) - x.lo, p.split_len);  // of the range
      const int head = x.w.kvh * p.group + head0 + h;
      const bool live = h < p.box_heads && head0 + h < p.group && token < x.w.qlen;
      float m = -INFINITY, l = 0.f;
      for (int i = 0; i < n && ok; ++i, ++steps) {
        const uint32_t b = steps & 1, mine_s = mine + b * kKeys;
        ok = wait(&s_s[t][b], (steps >> 1) & 1);
#ifdef HKV_CROSS_TEST_STALL  // one warp waits for a phase that nothing completes before its limit
        if (warp == (int)(blockIdx.x & 3) && i == 1) ok = wait(&s_drain, 0);
#endif
        if (!ok) break;
        tc_fence_after();
        uint32_t s[kKeys / 32][32];
#pragma unroll
        for (int c = 0; c < kKeys / 32; ++c) tmem_ld32(s[c], mine_s + c * 32);
        tmem_wait_ld();
        const int left = seen - i * kKeys;  // keys of the tile that count
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
            top[u] = max3(top[u], __uint_as_float(s[j >> 5][(j & 31) + 2 * u]),
                          __uint_as_float(s[j >> 5][(j & 31) + 2 * u + 1]));
        float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        mx *= p.qscale;
        float f = 1.f;
        if (mx > m + 8.f) {
          f = ex2_approx(m - mx);  // (zero for the first keys)
          m = mx;
          l *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;  // no key yet: weights of zero
        const bool rescale = __any_sync(0xFFFFFFFFu, f != 1.f);
        // O holds the tiles before this one. (A wait names a phase by its parity:
        // those two before have passed with S, and the one of the last tile but one
        // is waited for here, before the last one's can pass.)
        if (i > 0 && (rescale || i + 1 == n)) {
          ok = wait(&s_v[t], (steps - 1) & 1);
          if (!ok) break;
          tc_fence_after();
        }
        if (i > 0 && rescale) {
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            tmem_ld32(o, mine_o + c);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st32(mine_o + c, o);
          }
        }
        const uint64_t scale2 = pair_of(p.qscale, p.qscale), ref2 = pair_of(-ref, -ref);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < kKeys / 32; ++c) {
          uint32_t v[16], v2[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const uint64_t e = fma2(pair_of(s[c][2 * j], s[c][2 * j + 1]), scale2, ref2);
            const float w0 = ex2_approx(low(e)), w1 = ex2_approx(high(e));
            sum[j & 1] = add2(sum[j & 1], pair_of(w0, w1));
            v[j] = pack2(w0, w1);
            if (TP::kParts == 2)
              v2[j] = pack2(w0 - __uint_as_float(v[j] << 16), w1 - __uint_as_float(v[j] & 0xFFFF0000u));
          }
          tmem_st16(mine_s + c * 16, v);
          if (TP::kParts == 2) tmem_st16(mine_s + kKeys / 2 + c * 16, v2);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_p[t][b]);
        sum[0] = add2(sum[0], sum[1]);
        l += low(sum[0]) + high(sum[0]);
      }
      // O is complete
      if (ok && n > 0) ok = wait(&s_v[t], (steps - 1) & 1);
      tc_fence_after();
      const bool wrong = x.w.bad || !ok, any = n > 0 && ok;
      const size_t row = ((size_t)x.w.s * p.heads + head) * p.tokens + token;
      auto o_read = [&] {  // the next item's products may overwrite O
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_oe[t]);
      };
      if (p.splits > 1) {
        float *part = p.part + (row * p.splits + x.w.sp) * PF;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32] = {};
          if (any) {
            tmem_ld32(o, mine_o + c);
            tmem_wait_ld();
          }
          if (!live) continue;
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<uint4 *>(part + c + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
        if (any) o_read();
        if (live) *reinterpret_cast<float2 *>(part + D) = make_float2(wrong ? NAN : m, wrong ? 0.f : l);
      } else {
        const float inv = wrong ? NAN : l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat16 *to =
            static_cast<__nv_bfloat16 *>(p.out) + x.w.s * p.os + token * p.ot + head * p.oh;
        // kOut channels at a time to shared memory, then whole rows of them out
        constexpr int CH = TP::kOut, PPR = CH / 8;
        auto at = [](int rr, int c) {
          return rr * CH * 2 + ((c ^ (CH == 64 ? rr & 7 : (rr >> 1) & 3)) << 4);
        };
        auto piece = [&](int c, unsigned char *place, auto at_) {  // 32 channels of the thread's row
          uint32_t o[32] = {};
          if (any) {
            tmem_ld32(o, mine_o + c);
            tmem_wait_ld();
          }
          if (any && c + 32 == D) o_read();
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              v[i] = pack2(__uint_as_float(o[e * 8 + 2 * i]) * inv,
                           __uint_as_float(o[e * 8 + 2 * i + 1]) * inv);
            *reinterpret_cast<uint4 *>(place + at_(e)) = make_uint4(v[0], v[1], v[2], v[3]);
          }
        };
        auto copied = [&](auto left) {  // all but `left` of the warp's copies have left its place
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(decltype(left)::value) : "memory");
          __syncwarp();
        };
        // Copies of 32 channels of 32 rows where the warp's rows are of one head and
        // those without a token past the tensor's end, else row by row. The halves of
        // the warp's place take turns and all copies but the last are waited for, so
        // who writes a half copies it too: a warp without rows writes none (the last
        // copy of the work before may still read the second).
        if (!__any_sync(0xFFFFFFFFu, live)) {
          if (any) o_read();
        } else if (TP::kCopyOut && p.box_heads == 1 &&
                   __all_sync(0xFFFFFFFFu, live || h > 0 || token >= p.tokens)) {
          const int warp_token = __shfl_sync(0xFFFFFFFFu, token, 0);
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            unsigned char *half = rows + (c & 32) * 64;
            copied(std::integral_constant<int, 1>{});
            piece(c, half, [&](int e) { return lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4); });
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) tma_store(&omap, half, c, warp_token, head, x.w.s);
          }
        } else {
          if (TP::kCopyOut) copied(std::integral_constant<int, 0>{});
#pragma unroll 1
          for (int c = 0; c < D; c += CH) {
#pragma unroll
            for (int c1 = 0; c1 < CH; c1 += 32)
              piece(c + c1, rows, [&](int e) { return at(lane, c1 / 8 + e); });
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 32; i += 32 / PPR) {
              const int rr = i + lane / PPR, pc = lane % PPR;
              const bool on = __shfl_sync(0xFFFFFFFFu, live, rr);
              __nv_bfloat16 *row_at = reinterpret_cast<__nv_bfloat16 *>(
                  __shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(to), rr));
              if (on)
                *reinterpret_cast<uint4 *>(row_at + c + pc * 8) =
                    *reinterpret_cast<const uint4 *>(rows + at(rr, pc));
            }
            __syncwarp();
          }
        }
        if (live && p.lse) p.lse[row] = wrong ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      }
    } while (next_item(k++));
    if (TP::kCopyOut && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    if (!ok && lane == 0) {
      set_err(p.err, HKV_ERR_TIMEOUT);
      if (!x.none) s_left[warp] = k - 1;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_free(tmem, TP::kCols);
  // Items that were handed on after a warp's wait for the next one had run out (two
  // at most: there is no room for more until it reads them) get their NaN here, where
  // the code costs the loop above nothing (in it: 112 -> 114 us for 8 x 4160 queries of
  // 32 heads over 120 states).
  if (warp < TILES * 4 && s_left[warp] >= 0) {
    const int t = warp >> 2, r = tid & 127, h = r / p.box_tokens;
    for (int k = s_left[warp]; mbar_test_wait(&s_nf[k & 1], (k >> 1) & 1); ++k) {
      const Item<TILES> &y = s_item[k & 1];
      if (y.none) break;
      const int token = y.token0[t] + r - h * p.box_tokens, g = y.head0[t] + h, head = y.w.kvh * p.group + g;
      if (h >= p.box_heads || g >= p.group || token >= y.w.qlen) continue;
      const size_t row = ((size_t)y.w.s * p.heads + head) * p.tokens + token;
      if (p.splits > 1) {
        *reinterpret_cast<float2 *>(p.part + (row * p.splits + y.w.sp) * PF + D) = make_float2(NAN, 0.f);
        continue;
      }
      __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(p.out) + y.w.s * p.os + token * p.ot + head * p.oh;
#pragma unroll 1
      for (int c = 0; c < D; c += 8)
        *reinterpret_cast<uint4 *>(to + c) = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
      if (p.lse) p.lse[row] = NAN;
    }
  }
}

// Rows as a tensor of [sequences][heads][tokens][D], in boxes of 64 channels (128
// bytes, 128-byte swizzle) or 32; rows past the last are zero, and not written
cudaError_t encode(CUtensorMap *map, const void *base, int D, int tokens, long long token_stride,
                   int heads, long long head_stride, int seqs, long long seq_stride, int box_tokens,
                   int box_heads, int box_channels = 64) {
  using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                              const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
  static std::atomic<Encode> known{nullptr};
  Encode f = known.load(std::memory_order_acquire);
  if (!f) {
    void *at = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e =
        cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &at, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !at) return cudaErrorNotSupported;
    f = reinterpret_cast<Encode>(at);
    known.store(f, std::memory_order_release);
  }
  const auto stride = [&](long long s, int count) { return (cuuint64_t)(count > 1 ? s : D) * 2; };
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)tokens, (cuuint64_t)heads, (cuuint64_t)seqs};
  const cuuint64_t strides[3] = {stride(token_stride, tokens), stride(head_stride, heads),
                                 stride(seq_stride, seqs)};
  const cuuint32_t box[4] = {(cuuint32_t)box_channels, (cuuint32_t)box_tokens, (cuuint32_t)box_heads, 1};
  const cuuint32_t step[4] = {1, 1, 1, 1};
  const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides,
                       box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       box_channels == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int D, int TILES>
cudaError_t launch(const CrossArgs &a, int grid, cudaStream_t s) {
  using TP = TcPlan<D, TILES>;
  static std::atomic<uint64_t> ready{0};
  cudaError_t e = allow_smem_of(cross_tc_kernel<D, TILES>, TP::kBytes, ready);
  CUtensorMap q, k, v, o = {};
  if (e == cudaSuccess)
    e = encode(&q, a.q, D, a.tokens, a.qt, a.heads, a.qh, a.seqs, a.qs, a.box_tokens, a.box_heads);
  if (e == cudaSuccess) e = encode(&k, a.k, D, a.keys, a.kt, a.kv, a.kh, a.seqs, a.ks, TP::kKeys, 1);
  if (e == cudaSuccess) e = encode(&v, a.v, D, a.keys, a.kt, a.kv, a.kh, a.seqs, a.ks, TP::kKeys, 1);
  if (TP::kCopyOut && e == cudaSuccess)
    e = encode(&o, a.out, D, a.tokens, a.ot, a.heads, a.oh, a.seqs, a.os, 32, 1, 32);
  if (e != cudaSuccess) return e;
  return pdl_launch(cross_tc_kernel<D, TILES>, grid, TP::kThreads, TP::kBytes, s, a, q, k, v, o);
}

}  // namespace

cudaError_t launch_cross_tc(const CrossArgs &a, const CrossPlan &plan, int D, cudaStream_t s) {
  const long long grid = (long long)a.seqs * a.kv * a.tiles * a.splits;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  if (plan.rows == 256)
    return D == 64 ? launch<64, 2>(a, (int)grid, s) : launch<128, 2>(a, (int)grid, s);
  return D == 64 ? launch<64, 1>(a, (int)grid, s) : launch<128, 1>(a, (int)grid, s);
}

}  // namespace hkv
