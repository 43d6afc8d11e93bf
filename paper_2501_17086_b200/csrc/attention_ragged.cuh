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
__device__ __forceinline__ BlockOf block_at(unsigned i, const RaggedWalks& walks, bool last_first) {
  BlockOf w;
  const unsigned rest = walks.by_heads(i), b = walks.by_blocks(rest), blk = rest - b * walks.blocks;
  w.h = (int)(i - rest * walks.heads);
  w.blk = (int)(last_first ? walks.blocks - 1 - blk : blk);
  w.b = (int)b;
  return w;
}
// r with the walks of blocks of `tile` rows, `pack` query heads to a block.
inline RaggedAttn with_walks(RaggedAttn r, int tile, int pack = 1) {
  const auto walks = [&](int longest, int heads) {
    const uint32_t n = (uint32_t)((longest + (int64_t)tile - 1) / tile);
    return RaggedWalks{(uint32_t)heads, n, divider((uint32_t)heads), divider(n > 1 ? n : 1)};
  };
  r.q_walks = walks(r.a.q_len, r.a.q_heads / pack);
  r.kv_walks = walks(r.a.kv_len, r.a.kv_heads);
  r.group = r.a.q_heads / r.a.kv_heads;
  r.by_group = divider((uint32_t)r.group);
  return r;
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
// Ragged batches of up to a warp's lanes of sequences are taken longest walks first (over_keys: walks over the keys, else over the queries), so that
// no long walk begins when the others are nearly done: w.b, a place in that order, becomes the sequence.  12 sequences of up to 509 queries and 1301
// keys, 10 heads of 80, forward: 33 against 42 us in the batch's order.  (More sequences are taken in the batch's order; another one was not tried.)
__device__ __forceinline__ SeqPair sequence_pair(const hbp_attention& a, BlockOf& w, bool over_keys) {
  const int n = a.sequences;
  if ((a.q_offsets || a.kv_offsets) && n > 1 && n <= 32) {
    const int lane = threadIdx.x & 31;
    int len = 0, before = 0;
    if (lane < n) {
      const int32_t* off = over_keys ? a.kv_offsets : a.q_offsets;
      const int32_t* own = over_keys ? a.q_offsets : a.kv_offsets;
      len = off ? (int)((unsigned)off[lane + 1] - (unsigned)off[lane]) : 0;
      if (own && own[lane + 1] == own[lane]) len = -1;  // (none of its blocks does anything)
    }
    for (int i = 0; i < n; ++i) {
      const int other = __shfl_sync(0xffffffffu, len, i);
      before += other > len || (other == len && i < lane);
    }
    w.b = __ffs((int)__ballot_sync(0xffffffffu, lane < n && before == w.b)) - 1;
  }
  return sequence_pair(a, w.b);
}

// ---- outputs that are new memory: rows in no sequence, or in one that is skipped, become 0 (a log-sum-exp: -infinity).  kClearers more blocks of a
// launch that is there anyway do it, beside the others: no row of theirs is one that the pass writes.  (A launch of its own before the pass: 5 sequences of
// up to 77 rows, both passes, 18.7 -> 23.6 us a call instead of 19 to 19.7.)
constexpr int kClearers = 152;  // (whole clusters of up to eight)
// Can rows of a side be in no sequence, or in one that is skipped?  (Offsets of either side may be bad ones.)
inline bool rows_left_over(const hbp_attention& a, int64_t rows, int longest) {
  return a.q_offsets || a.kv_offsets || (int64_t)a.sequences * longest != rows;
}
// One side's rows, whole warps; this one is `part` of `parts`.  x, y: tensors of those rows, x.x and y.x may be NULL, as may be lse.
__device__ __forceinline__ void clear_side(const hbp_attention& a, bool keys, const hbp_heads& x, const hbp_heads& y, float* lse, int part, int parts) {
  const int lane = threadIdx.x & 31, n = a.sequences, longest = keys ? a.kv_len : a.q_len, heads = keys ? a.kv_heads : a.q_heads;
  const int es = a.dtype == HBP_F32 ? 4 : 2, units = a.head_dim * es / 16;
  const int64_t rows = keys ? a.kv_rows : a.q_rows;
  const int32_t* off = keys ? a.kv_offsets : a.q_offsets;
  auto clear = [&](int64_t row) {
    for (int i = lane; i < heads * units; i += 32) {
      const int h = i / units, u = i - h * units;
      if (x.x) *reinterpret_cast<uint4*>((char*)x.x + (row * x.row_stride + h * x.head_stride) * es + u * 16) = make_uint4(0, 0, 0, 0);
      if (y.x) *reinterpret_cast<uint4*>((char*)y.x + (row * y.row_stride + h * y.head_stride) * es + u * 16) = make_uint4(0, 0, 0, 0);
    }
    if (lse)
      for (int h = lane; h < heads; h += 32) lse[h * rows + row] = -INFINITY;
  };
  // is sequence b taken, and which rows of this side does it have?
  auto taken = [&](int b, int64_t& beg, int64_t& end) {
    int64_t other;
    int len;
    const bool q = one_sequence(a.q_offsets, b, a.q_len, a.q_rows, keys ? other : beg, len);
    if (!keys) end = beg + len;
    const bool k = one_sequence(a.kv_offsets, b, a.kv_len, a.kv_rows, keys ? beg : other, len);
    if (keys) end = beg + len;
    return q && k;
  };
  // is a row of from .. to - 1 in a sequence that is taken?
  auto overlap = [&](int64_t from, int64_t to) {
    bool any = false;
#pragma unroll 4
    for (int b = lane; b < n; b += 32) {
      int64_t beg, end;
      any = (taken(b, beg, end) && beg < to && end > from && beg < end) || any;
    }
    return __any_sync(0xffffffffu, any) != 0;
  };
  auto clear_range = [&](int64_t from, int64_t to, int at, int step) {
    from = from < 0 ? 0 : from;
    to = to > rows ? rows : to;
    if (from >= to) return;
    const bool some = overlap(from, to);  // (only where offsets decrease somewhere)
    for (int64_t row = from + at; row < to; row += step)
      if (!some || !overlap(row, row + 1)) clear(row);
  };
  // A row in no sequence that is taken lies before the first offset, behind the last, or between those of a sequence that is skipped.
  clear_range(0, off ? off[0] : 0, part, parts);
  clear_range(off ? off[n] : (int64_t)n * longest, rows, part, parts);
  for (int64_t b0 = (int64_t)part * 32; b0 < n; b0 += (int64_t)parts * 32) {
    int64_t beg, end;
    unsigned skipped = __ballot_sync(0xffffffffu, b0 + lane < n && !taken((int)b0 + lane, beg, end));
    for (; skipped; skipped &= skipped - 1) {
      const int b = (int)b0 + __ffs((int)skipped) - 1;
      clear_range(off ? off[b] : (int64_t)b * longest, off ? off[b + 1] : (int64_t)(b + 1) * longest, 0, 1);
    }
  }
}
// This block's share of a launch's clearing, `block` of kClearers (a call, so that the registers are those of the passes)
static __device__ __noinline__ void clear_block(const RaggedAttn& p, bool backward, int block, int threads) {
  const int part = block * (threads / 32) + threadIdx.x / 32, parts = kClearers * (threads / 32), fresh = p.a.fresh;
  const hbp_heads none = {};
  if (!backward) {
    if (fresh & (HBP_FRESH_O | HBP_FRESH_LSE)) clear_side(p.a, false, fresh & HBP_FRESH_O ? p.o : none, none, fresh & HBP_FRESH_LSE ? p.lse : nullptr, part, parts);
    return;
  }
  if (fresh & HBP_FRESH_DQ) clear_side(p.a, false, p.dq, none, nullptr, part, parts);
  if (fresh & (HBP_FRESH_DK | HBP_FRESH_DV)) clear_side(p.a, true, fresh & HBP_FRESH_DK ? p.dk : none, fresh & HBP_FRESH_DV ? p.dv : none, nullptr, part, parts);
}

// bf16 on the tensor cores (attention_ragged_tc.cu); false if a tensor's strides or address are not such as tile copies take, in which case
// nothing was launched.
bool ragged_forward_tc(Launcher& lc, const RaggedAttn& r);
bool ragged_backward_tc(Launcher& lc, const RaggedAttn& r);

}  // namespace hbp
