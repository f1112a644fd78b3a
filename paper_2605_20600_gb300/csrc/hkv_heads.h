// Host-side launchers of the kernels around the cache: rotations and norms of
// heads, attention over other states (internal to libheadkv.so).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "hkv_prompt.h"
#include "hkv_kernels.h"

namespace hkv {

// rows of one input and where they go; strides in elements
struct HeadSet {
  const void *in;
  void *out;
  long long is, it, ih, os, ot, oh;   // sequence, token, head
  const void *weight, *bias;          // norm; NULL: ones, zeros
  long long wh;                       // head stride of weight and bias
  int heads;
  int norm, rotate;                   // whether the set is normed and rotated
  int first_block;                    // blocks of the set, and how they share its
  int per, tokens, chunks;            // rows (launch_heads fills these in):
  int chunk, most;                    // heads of a chunk, and rows of a thread
};

// The sets q, k, v of a call (those that it has).
struct HeadsArgs {
  HeadSet set[3];
  int sets, heads;                    // sets in use, heads of all of them
  int seqs, tokens;
  const int32_t *len, *pos;
  long long pa, ps;                   // strides of the positions: axis, sequence
  uint32_t *err;
  hkv_rope rope;                      // rot_dim 0: no rotation
  float sign;                         // of the sines
  float eps;
};

cudaError_t launch_heads(const HeadsArgs &a, int D, int dtype, int norm, cudaStream_t s);

// attention over states
struct CrossArgs {
  const void *q, *k, *v;
  void *out;
  float *lse;                         // [seqs][heads][tokens] or NULL
  const int32_t *qlen, *klen;         // or NULL
  uint32_t *err;                      // of the states
  uint32_t *qerr;                     // of the tokens
  long long qs, qt, qh, os, ot, oh;   // strides: sequence, token, head
  long long ks, kh, kt;               // of k and v
  int seqs, heads, kv, group;         // query heads, key heads, query heads a key head
  int tokens, keys;                   // most of a sequence
  int causal;
  int splits, split_len, tiles;       // key ranges; query tiles of a key head
  int box_tokens, box_heads;          // a query tile of the tcgen05 kernel
  int sorted;                         // work by the sequences' lengths (Order)
  float *part;                        // [rows of (sequence, head, token)][splits][D + 4]
  float qscale;                       // log2(e) / sqrt(D)
};

struct CrossPlan {
  int rows;                           // queries of a CTA (256, 128: the tcgen05 kernel)
  int splits, split_len, tiles;
  int box_tokens, box_heads, sorted;
  size_t part_bytes;
};
CrossPlan cross_plan(int seqs, int heads, int kv, int tokens, int keys, int D, int dtype,
                     int out_dtype);
cudaError_t launch_cross(const CrossArgs &a, const CrossPlan &plan, int D, int dtype,
                         int out_dtype, cudaStream_t s);

}  // namespace hkv
