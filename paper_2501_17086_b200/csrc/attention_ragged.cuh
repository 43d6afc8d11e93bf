// What the kernels of attention over ragged batches share: which block of rows a thread block has, and the rows of a sequence.
#pragma once
#include "hbp_internal.h"

namespace hbp {

// Blocks of `tile` rows over all heads and sequences, sequences slowest.
inline int64_t blocks_of(int longest, int tile, int heads, int sequences) {
  return (int64_t)((longest + tile - 1) / tile) * heads * sequences;
}
struct BlockOf {
  int blk, h, b;
};
// Heads are the fastest, so that blocks that run together read the same keys (the query heads of a group) and take equally long.
// last_first: the blocks of the last rows, which see the most keys of a causal batch, come before the others.
__device__ __forceinline__ BlockOf block_at(unsigned i, int longest, int tile, int heads, bool last_first) {
  const unsigned n = (unsigned)(longest + tile - 1) / tile;
  BlockOf w;
  w.h = (int)(i % heads);
  i /= heads;
  const unsigned blk = i % n;
  w.blk = (int)(last_first ? n - 1 - blk : blk);
  w.b = (int)(i / n);
  return w;
}
__device__ __forceinline__ BlockOf block_of(int longest, int tile, int heads, bool last_first) {
  return block_at(blockIdx.x, longest, tile, heads, last_first);
}

struct SeqPair {
  int64_t q0, k0;  // first rows
  int nq, nk;
};
// One side of a sequence; false where the offsets are not those of rows of the tensor.
__device__ __forceinline__ bool one_sequence(const int32_t* off, int b, int longest, int64_t rows, int64_t& beg, int& n) {
  if (!off) {
    beg = (int64_t)b * longest;
    n = longest;
    return true;
  }
  const int64_t lo = off[b], hi = off[b + 1];
  beg = lo;
  n = (int)(hi - lo);
  return lo >= 0 && hi >= lo && hi - lo <= longest && hi <= rows;
}
// A sequence with bad offsets is an empty one, and the status word says so.
__device__ __forceinline__ SeqPair sequence_pair(const hbp_attention& a, int b) {
  SeqPair s;
  const bool q = one_sequence(a.q_offsets, b, a.q_len, a.q_rows, s.q0, s.nq), k = one_sequence(a.kv_offsets, b, a.kv_len, a.kv_rows, s.k0, s.nk);
  if (!q || !k) {
    if (a.status && threadIdx.x == 0) atomicExch(a.status, (int)HBP_ERR_INVALID_ARG);
    s.q0 = s.k0 = 0;
    s.nq = s.nk = 0;
  }
  return s;
}

// bf16 on the tensor cores (attention_ragged_tc.cu); false if a tensor's strides or address are not such as tile copies take, in which case
// nothing was launched.
bool ragged_forward_tc(Launcher& lc, const RaggedAttn& r);
bool ragged_backward_tc(Launcher& lc, const RaggedAttn& r);

}  // namespace hbp
