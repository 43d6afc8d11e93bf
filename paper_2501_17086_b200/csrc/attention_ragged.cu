// Attention over ragged batches with grouped heads (hbp_attention_forward / _backward): argument checks, and the CUDA-core
// kernels, which are those of float tensors.
//
// With s_ij = scale * q_i . k_j over the keys j that query i sees:
//   forward    o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - lse_i), lse_i = log sum_j exp(s_ij): one pass over the keys with a
//              running maximum and sum; what was summed before is scaled down when the maximum grows.
//   backward   p_ij again from q, k and lse; D_i = d_o_i . o_i; ds_ij = p_ij (d_o_i . v_j - D_i);
//              dv_j = sum_i p_ij d_o_i, dk_j = scale sum_i ds_ij q_i, dq_i = scale sum_j ds_ij k_j.
// Blocks own 64 queries (forward, dq) or 64 keys of a key head (dk, dv: all query heads of its group), so that every sum
// has one owner and one order.  Tiles of 64 rows lie in shared memory row by row, 16 bytes between rows more than they need, which
// keeps the 16-byte reads of neighbouring rows in different banks; a thread forms 4 x 4 products of a score tile, or 4 rows times
// every 16th vector of an output.  Bound by how few warps an SM has beside the registers of such tiles: 2048 rows of 8 heads of 64, forward 162 us
// (27 TFLOP/s of the 4 flops a pair and channel that are needed, tiles on the diagonal in full), backward 549 (20); the FFMA pipe is busy 38 %
// of the time.  (Two backward blocks an SM of 128 registers and one stage each: 2048 rows 561 us, six ragged sequences 234 instead of 164.)
#include <cooperative_groups.h>

#include <cmath>

#include "attention_ragged.cuh"
#include "float_pairs.cuh"

namespace hbp {

namespace cg = cooperative_groups;

namespace {

constexpr int TILE = 64, THREADS = 256;
constexpr int PS = TILE + 4;  // floats between rows of a score tile

template <int HD>
constexpr int kStride = HD + 4;

// Asks for `TILE` rows of a tensor from row r0 of a sequence of n rows on, into shared memory; zeros behind the sequence's end and
// behind channel `width`.  base: the sequence's first row of one head.
template <int HD>
__device__ __forceinline__ void ask_tile(float* __restrict__ dst, const float* __restrict__ base, int64_t row_stride, int r0, int n, int width) {
  constexpr int VECS = HD / 4;
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst);
#pragma unroll
  for (int i = threadIdx.x; i < TILE * VECS; i += THREADS) {
    const int r = i / VECS, c = (i % VECS) * 4;
    const bool there = r0 + r < n && c < width;
    const float* from = there ? base + (int64_t)(r0 + r) * row_stride + c : base;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (r * kStride<HD> + c) * 4), "l"(from), "r"(there ? 16 : 0) : "memory");
  }
}
__device__ __forceinline__ void asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until all that was asked for before the last `kLater` groups is there (and then, for all threads, a barrier)
template <int kLater>
__device__ __forceinline__ void wait_asked() { asm volatile("cp.async.wait_group %0;" ::"n"(kLater) : "memory"); }

// s[r][c] = sum over channels of A[ty * 4 + r] * B[tx + 16 * c], those of even and of odd channels side by side (two in an instruction)
template <int HD>
__device__ __forceinline__ void score_tile(const float* __restrict__ A, const float* __restrict__ B, int ty, int tx, float (&s)[4][4]) {
  constexpr int LD = kStride<HD>;
  f32x2 t[4][4];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) t[r][c] = both(0.0f);
#pragma unroll 4
  for (int k = 0; k < HD; k += 4) {
    ulonglong2 a[4], b[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) a[r] = *reinterpret_cast<const ulonglong2*>(A + (ty * 4 + r) * LD + k);
#pragma unroll
    for (int c = 0; c < 4; ++c) b[c] = *reinterpret_cast<const ulonglong2*>(B + (tx + 16 * c) * LD + k);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) t[r][c] = fma2(a[r].x, b[c].x, fma2(a[r].y, b[c].y, t[r][c]));
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float2 f = floats_of(t[r][c]);
      s[r][c] = f.x + f.y;
    }
}

// acc[r][4 v + e] += sum over rows j of W[j][ty * 4 + r] * X[j][(tx + 16 v) * 4 + e]; W has PS floats a row
template <int HD>
__device__ __forceinline__ void add_product(const float* __restrict__ W, const float* __restrict__ X, int ty, int tx, float (&acc)[4][HD / 16]) {
  constexpr int LD = kStride<HD>;
#pragma unroll 4
  for (int j = 0; j < TILE; ++j) {
    const float4 w = *reinterpret_cast<const float4*>(W + j * PS + ty * 4);
    const float wr[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int v = 0; v < HD / 64; ++v) {
      const float4 x = *reinterpret_cast<const float4*>(X + j * LD + (tx + 16 * v) * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        acc[r][4 * v] = fmaf(wr[r], x.x, acc[r][4 * v]);
        acc[r][4 * v + 1] = fmaf(wr[r], x.y, acc[r][4 * v + 1]);
        acc[r][4 * v + 2] = fmaf(wr[r], x.z, acc[r][4 * v + 2]);
        acc[r][4 * v + 3] = fmaf(wr[r], x.w, acc[r][4 * v + 3]);
      }
    }
  }
}

template <int HD>
__device__ __forceinline__ void store_rows(float* __restrict__ base, int64_t row_stride, int r0, int n, int width, int ty, int tx, float mul,
                                           const float (&acc)[4][HD / 16]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = r0 + ty * 4 + r;
    if (row >= n) continue;
#pragma unroll
    for (int v = 0; v < HD / 64; ++v) {
      const int c = (tx + 16 * v) * 4;
      if (c < width)
        *reinterpret_cast<float4*>(base + (int64_t)row * row_stride + c) =
            make_float4(mul * acc[r][4 * v], mul * acc[r][4 * v + 1], mul * acc[r][4 * v + 2], mul * acc[r][4 * v + 3]);
    }
  }
}

// Leaves a block's sums in its shared memory, rows LD floats apart.
template <int HD>
__device__ __forceinline__ void leave_rows(float* __restrict__ dst, int ty, int tx, const float (&acc)[4][HD / 16]) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int v = 0; v < HD / 64; ++v)
      *reinterpret_cast<float4*>(dst + (ty * 4 + r) * kStride<HD> + (tx + 16 * v) * 4) =
          make_float4(acc[r][4 * v], acc[r][4 * v + 1], acc[r][4 * v + 2], acc[r][4 * v + 3]);
}
// What all blocks of a cluster have left at `mine` (an address in this block's shared memory), added up in the blocks' order, each times
// weight(block).
template <typename W>
__device__ __forceinline__ float4 gather(cg::cluster_group& cluster, float* mine, int ranks, W weight) {
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int b = 0; b < ranks; ++b) {
    const float4 x = *reinterpret_cast<const float4*>(cluster.map_shared_rank(mine, b));
    const float w = weight(b);
    s.x = fmaf(w, x.x, s.x); s.y = fmaf(w, x.y, s.y); s.z = fmaf(w, x.z, s.z); s.w = fmaf(w, x.w, s.w);
  }
  return s;
}

// Few blocks with long walks leave most of the chip idle.  Then the tiles of a walk are dealt out to the `ranks` blocks of a cluster; each leaves its
// sums in its shared memory, and each puts together those of all for its share of the rows, in the blocks' order (ranks_of below).

// ------------------------------------------------------------------------------------------- forward
template <int HD>
__global__ void __launch_bounds__(THREADS) ragged_fwd_kernel(const __grid_constant__ RaggedAttn p, const int ranks) {
  extern __shared__ float4 smem4[];
  constexpr int LD = kStride<HD>;
  float* sQ = reinterpret_cast<float*>(smem4);
  float* sKV = sQ + TILE * LD;  // two stages of a key and a value tile: the next ones come while these are used
  float* sPt = sKV + 4 * TILE * LD;  // [key][query]
  chain_wait();
  if (blockIdx.x >= p.pass_blocks) return clear_block(p, false, (int)(blockIdx.x - p.pass_blocks), THREADS);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int rank = (int)(blockIdx.x % ranks);
  BlockOf w = block_at(blockIdx.x / ranks, p.q_walks, true);
  const SeqPair sq = sequence_pair(p.a, w, true);
  const int q0 = w.blk * TILE, kh = (int)p.by_group((uint32_t)w.h);
  if (q0 >= sq.nq) return;  // (all blocks of the cluster)
  const float* q = (const float*)p.q.x + sq.q0 * p.q.row_stride + w.h * p.q.head_stride;
  const float* k = (const float*)p.k.x + sq.k0 * p.k.row_stride + kh * p.k.head_stride;
  const float* v = (const float*)p.v.x + sq.k0 * p.v.row_stride + kh * p.v.head_stride;
  const int shift = p.a.causal ? sq.nk - sq.nq : sq.nk;  // query i sees keys 0 .. i + shift (capped by nk)
  const int seen = min(sq.nk, p.a.causal ? min(q0 + TILE, sq.nq) + shift : sq.nk);
  const int step = ranks * TILE;
  auto stage = [&](int k0) { return sKV + (k0 / step & 1) * 2 * TILE * LD; };
  auto ask = [&](int k0) {
    ask_tile<HD>(stage(k0), k, p.k.row_stride, k0, sq.nk, p.a.head_dim);
    ask_tile<HD>(stage(k0) + TILE * LD, v, p.v.row_stride, k0, sq.nk, p.a.head_dim);
  };
  if (rank * TILE < seen) {
    ask_tile<HD>(sQ, q, p.q.row_stride, q0, sq.nq, p.a.head_dim);
    ask(rank * TILE);
  }
  asked();
  float acc[4][HD / 16], m[4], l[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.0f;
#pragma unroll
    for (int e = 0; e < HD / 16; ++e) acc[r][e] = 0.0f;
  }
  for (int k0 = rank * TILE; k0 < seen; k0 += step) {
    if (k0 + step < seen) ask(k0 + step);
    asked();
    wait_asked<1>();
    __syncthreads();
    const float *sK = stage(k0), *sV = sK + TILE * LD;
    float s[4][4];
    score_tile<HD>(sQ, sK, ty, tx, s);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int last = min(sq.nk - 1, p.a.causal ? q0 + ty * 4 + r + shift : sq.nk - 1);  // the last key this query sees
      float top = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[r][c] = k0 + tx + 16 * c <= last ? s[r][c] * p.a.scale : -INFINITY;
        top = fmaxf(top, s[r][c]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float mn = fmaxf(m[r], top), ref = mn == -INFINITY ? 0.0f : mn;  // (a row that has seen nothing yet)
      const float keep = expf(m[r] - ref);
      m[r] = mn;
      float sum = 0.0f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[r][c] = expf(s[r][c] - ref);
        sum += s[r][c];
      }
      l[r] = l[r] * keep + sum;
#pragma unroll
      for (int e = 0; e < HD / 16; ++e) acc[r][e] *= keep;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<float4*>(sPt + (tx + 16 * c) * PS + ty * 4) = make_float4(s[0][c], s[1][c], s[2][c], s[3][c]);
    __syncthreads();
    add_product<HD>(sPt, sV, ty, tx, acc);
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
  float* lse = p.lse + w.h * p.a.q_rows + sq.q0 + q0;
  float* out = (float*)p.o.x + sq.q0 * p.o.row_stride + w.h * p.o.head_stride;
  // nothing seen: zeros and -infinity (a sum that is NaN stays NaN)
  auto inverse = [](float sum) { return sum > 0.0f ? 1.0f / sum : sum; };
  if (ranks == 1) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float inv = inverse(l[r]);
#pragma unroll
      for (int e = 0; e < HD / 16; ++e) acc[r][e] *= inv;
      if (tx == 0 && q0 + ty * 4 + r < sq.nq) lse[ty * 4 + r] = l[r] == 0.0f ? -INFINITY : m[r] + logf(l[r]);
    }
    store_rows<HD>(out, p.o.row_stride, q0, sq.nq, p.a.head_dim, ty, tx, 1.0f, acc);
    return;
  }
  leave_rows<HD>(sKV, ty, tx, acc);  // (the last tile has been used by all)
  float2* sML = reinterpret_cast<float2*>(sPt);
  if (tx == 0) {
#pragma unroll
    for (int r = 0; r < 4; ++r) sML[ty * 4 + r] = make_float2(m[r], l[r]);
  }
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  constexpr int VECS = HD / 4;
  for (int i = rank * THREADS + threadIdx.x; i < TILE * VECS; i += ranks * THREADS) {
    const int r = i / VECS, c = i % VECS * 4;
    if (q0 + r >= sq.nq || c >= p.a.head_dim) continue;
    float top = -INFINITY, sum = 0.0f;
    for (int b = 0; b < ranks; ++b) top = fmaxf(top, cluster.map_shared_rank(sML + r, b)->x);
    auto weight = [&](int b) { return top == -INFINITY ? 1.0f : expf(cluster.map_shared_rank(sML + r, b)->x - top); };
    for (int b = 0; b < ranks; ++b) sum = fmaf(weight(b), cluster.map_shared_rank(sML + r, b)->y, sum);
    const float4 o = gather(cluster, sKV + r * LD + c, ranks, weight);
    const float inv = inverse(sum);
    *reinterpret_cast<float4*>(out + (int64_t)(q0 + r) * p.o.row_stride + c) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (c == 0) lse[r] = sum == 0.0f ? -INFINITY : top + logf(sum);
  }
  cluster.sync();  // (no block ends while another reads its shared memory)
}

// ------------------------------------------------------------------------------------------- backward
// p and ds of one 64 x 64 tile; rows are queries.  lse, dd: those of this thread's four queries.
template <int HD>
__device__ __forceinline__ void probabilities(const float* sQ, const float* sK, const float* sG, const float* sV, int ty, int tx, int q0, int k0,
                                              const SeqPair& sq, const RaggedAttn& p, int shift, const float (&lse)[4], const float (&dd)[4],
                                              float (&pr)[4][4], float (&ds)[4][4]) {
  score_tile<HD>(sQ, sK, ty, tx, pr);
  score_tile<HD>(sG, sV, ty, tx, ds);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = q0 + ty * 4 + r, last = row < sq.nq ? min(sq.nk - 1, p.a.causal ? row + shift : sq.nk - 1) : -1;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool vis = k0 + tx + 16 * c <= last;
      pr[r][c] = vis ? expf(pr[r][c] * p.a.scale - lse[r]) : 0.0f;
      ds[r][c] = vis ? pr[r][c] * (ds[r][c] - dd[r]) : 0.0f;
    }
  }
}
__device__ __forceinline__ void row_statistics(const RaggedAttn& p, const SeqPair& sq, int h, int q0, int ty, float (&lse)[4], float (&dd)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = q0 + ty * 4 + r;
    const int64_t at = h * p.a.q_rows + sq.q0 + row;
    lse[r] = row < sq.nq ? p.lse[at] : 0.0f;
    dd[r] = row < sq.nq ? p.drow[at] : 0.0f;
  }
}

template <int HD>
__device__ __forceinline__ void ragged_dq(const RaggedAttn& p, BlockOf w) {
  extern __shared__ float4 smem4[];
  constexpr int LD = kStride<HD>;
  float* sQ = reinterpret_cast<float*>(smem4);
  float* sG = sQ + TILE * LD;
  float* sKV = sG + TILE * LD;
  float* sSt = sKV + 4 * TILE * LD;  // [key][query]
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const SeqPair sq = sequence_pair(p.a, w, true);
  const int q0 = w.blk * TILE, kh = (int)p.by_group((uint32_t)w.h);
  if (q0 >= sq.nq) return;
  const float* k = (const float*)p.k.x + sq.k0 * p.k.row_stride + kh * p.k.head_stride;
  const float* v = (const float*)p.v.x + sq.k0 * p.v.row_stride + kh * p.v.head_stride;
  const int shift = p.a.causal ? sq.nk - sq.nq : sq.nk;
  const int seen = min(sq.nk, p.a.causal ? min(q0 + TILE, sq.nq) + shift : sq.nk);
  auto stage = [&](int k0) { return sKV + (k0 / TILE & 1) * 2 * TILE * LD; };
  auto ask = [&](int k0) {
    ask_tile<HD>(stage(k0), k, p.k.row_stride, k0, sq.nk, p.a.head_dim);
    ask_tile<HD>(stage(k0) + TILE * LD, v, p.v.row_stride, k0, sq.nk, p.a.head_dim);
  };
  if (seen > 0) {
    ask_tile<HD>(sQ, (const float*)p.q.x + sq.q0 * p.q.row_stride + w.h * p.q.head_stride, p.q.row_stride, q0, sq.nq, p.a.head_dim);
    ask_tile<HD>(sG, (const float*)p.d_o.x + sq.q0 * p.d_o.row_stride + w.h * p.d_o.head_stride, p.d_o.row_stride, q0, sq.nq, p.a.head_dim);
    ask(0);
  }
  asked();
  float lse[4], dd[4], acc[4][HD / 16] = {};
  row_statistics(p, sq, w.h, q0, ty, lse, dd);
  for (int k0 = 0; k0 < seen; k0 += TILE) {
    if (k0 + TILE < seen) ask(k0 + TILE);
    asked();
    wait_asked<1>();
    __syncthreads();
    const float *sK = stage(k0), *sV = sK + TILE * LD;
    float pr[4][4], ds[4][4];
    probabilities<HD>(sQ, sK, sG, sV, ty, tx, q0, k0, sq, p, shift, lse, dd, pr, ds);
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<float4*>(sSt + (tx + 16 * c) * PS + ty * 4) = make_float4(ds[0][c], ds[1][c], ds[2][c], ds[3][c]);
    __syncthreads();
    add_product<HD>(sSt, sK, ty, tx, acc);
    __syncthreads();
  }
  store_rows<HD>((float*)p.dq.x + sq.q0 * p.dq.row_stride + w.h * p.dq.head_stride, p.dq.row_stride, q0, sq.nq, p.a.head_dim, ty, tx, p.a.scale, acc);
}

template <int HD>
__device__ __forceinline__ void ragged_dkv(const RaggedAttn& p, const BlockOf w, const int rank, const int ranks) {
  extern __shared__ float4 smem4[];
  constexpr int LD = kStride<HD>;
  float* sK = reinterpret_cast<float*>(smem4);
  float* sV = sK + TILE * LD;
  float* sQG = sV + TILE * LD;
  constexpr bool kOneTile = HD > 64;  // shared memory has room for the probabilities or for ds
  float* sP = sQG + 4 * TILE * LD;  // [query][key]
  float* sS = sP + (kOneTile ? 0 : TILE * PS);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  // (in the batch's order: with the longest first, the clusters of dK and dV and the blocks of dQ end less evenly, 128 against 122 us, 6 x 421 rows)
  const SeqPair sq = sequence_pair(p.a, w.b);
  const int k0 = w.blk * TILE, group = p.group;
  if (k0 >= sq.nk) return;  // (all blocks of the cluster)
  const int shift = p.a.causal ? sq.nk - sq.nq : sq.nk;
  const int first = p.a.causal ? max(0, k0 - shift) / TILE * TILE : 0;  // the first block of queries that sees key k0
  // the tiles of queries of all heads of the group, one head after the other
  const int tiles = max(0, (sq.nq + TILE - 1) / TILE - first / TILE), total = tiles * group;
  auto ask = [&](int it) {
    float* t = sQG + (it / ranks & 1) * 2 * TILE * LD;
    const int h = w.h * group + it / tiles, q0 = first + it % tiles * TILE;
    ask_tile<HD>(t, (const float*)p.q.x + sq.q0 * p.q.row_stride + h * p.q.head_stride, p.q.row_stride, q0, sq.nq, p.a.head_dim);
    ask_tile<HD>(t + TILE * LD, (const float*)p.d_o.x + sq.q0 * p.d_o.row_stride + h * p.d_o.head_stride, p.d_o.row_stride, q0, sq.nq, p.a.head_dim);
  };
  if (rank < total) {
    ask_tile<HD>(sK, (const float*)p.k.x + sq.k0 * p.k.row_stride + w.h * p.k.head_stride, p.k.row_stride, k0, sq.nk, p.a.head_dim);
    ask_tile<HD>(sV, (const float*)p.v.x + sq.k0 * p.v.row_stride + w.h * p.v.head_stride, p.v.row_stride, k0, sq.nk, p.a.head_dim);
    ask(rank);
  }
  asked();
  float dk[4][HD / 16] = {}, dv[4][HD / 16] = {};
  for (int it = rank; it < total; it += ranks) {
    if (it + ranks < total) ask(it + ranks);
    asked();
    const int h = w.h * group + it / tiles, q0 = first + it % tiles * TILE;
    float lse[4], dd[4];
    row_statistics(p, sq, h, q0, ty, lse, dd);
    wait_asked<1>();
    __syncthreads();
    const float *sQ = sQG + (it / ranks & 1) * 2 * TILE * LD, *sG = sQ + TILE * LD;
    float pr[4][4], ds[4][4];
    probabilities<HD>(sQ, sK, sG, sV, ty, tx, q0, k0, sq, p, shift, lse, dd, pr, ds);
    auto put = [&](float* dst, const float (&x)[4][4]) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) dst[(ty * 4 + r) * PS + tx + 16 * c] = x[r][c];
    };
    put(sP, pr);
    if (!kOneTile) put(sS, ds);
    __syncthreads();
    add_product<HD>(sP, sG, ty, tx, dv);
    if (kOneTile) {
      __syncthreads();
      put(sS, ds);
      __syncthreads();
    }
    add_product<HD>(sS, sQ, ty, tx, dk);
    __syncthreads();
  }
  float* dk_base = (float*)p.dk.x + sq.k0 * p.dk.row_stride + w.h * p.dk.head_stride;
  float* dv_base = (float*)p.dv.x + sq.k0 * p.dv.row_stride + w.h * p.dv.head_stride;
  if (ranks == 1) {
    store_rows<HD>(dk_base, p.dk.row_stride, k0, sq.nk, p.a.head_dim, ty, tx, p.a.scale, dk);
    store_rows<HD>(dv_base, p.dv.row_stride, k0, sq.nk, p.a.head_dim, ty, tx, 1.0f, dv);
    return;
  }
  __syncthreads();  // (a block without tiles of its own asked for nothing; the others' keys have been used by all)
  leave_rows<HD>(sK, ty, tx, dk);
  leave_rows<HD>(sV, ty, tx, dv);
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  constexpr int VECS = HD / 4;
  for (int i = rank * THREADS + threadIdx.x; i < 2 * TILE * VECS; i += ranks * THREADS) {
    const int which = i / (TILE * VECS), r = i / VECS % TILE, c = i % VECS * 4;
    if (k0 + r >= sq.nk || c >= p.a.head_dim) continue;
    const float mul = which ? 1.0f : p.a.scale;
    const float4 x = gather(cluster, (which ? sV : sK) + r * LD + c, ranks, [&](int) { return mul; });
    *reinterpret_cast<float4*>((which ? dv_base + (int64_t)(k0 + r) * p.dv.row_stride : dk_base + (int64_t)(k0 + r) * p.dk.row_stride) + c) = x;
  }
  cluster.sync();  // (no block ends while another reads its shared memory)
}

// dk, dv and dq in one launch: clusters of `ranks` blocks for the former; a block of dq's clusters works by itself.
template <int HD>
__global__ void __launch_bounds__(THREADS) ragged_bwd_kernel(const __grid_constant__ RaggedAttn p, const unsigned kv_walks, const unsigned q_walks, const int ranks) {
  chain_wait();  // (D comes from the launch before)
  const unsigned kv_blocks = kv_walks * ranks;
  if (blockIdx.x < kv_blocks) ragged_dkv<HD>(p, block_at(blockIdx.x / ranks, p.kv_walks, false), (int)(blockIdx.x % ranks), ranks);
  else if (blockIdx.x - kv_blocks < q_walks) ragged_dq<HD>(p, block_at(blockIdx.x - kv_blocks, p.q_walks, true));
}

// drow[h][row] = sum over channels of d_o * o, `lanes` (a power of two, 16 bytes each) to a row of a head; neighbouring lanes take neighbouring
// heads of a row.  (32 registers: at the 40 that clearing would take, 8 x 1024 rows of 12 heads cost a microsecond more.)
template <typename T>
__global__ void __launch_bounds__(256, 8) row_dot_kernel(const __grid_constant__ RaggedAttn p, int lanes) {
  constexpr int V = 16 / (int)sizeof(T);
  chain_next();  // (the backward kernels read the sums behind a chain_wait)
  if (blockIdx.x >= p.pass_blocks) return clear_block(p, true, (int)(blockIdx.x - p.pass_blocks), 256);
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / lanes;
  const int lane = threadIdx.x & (lanes - 1);
  const int64_t row = i / p.a.q_heads;
  const int h = (int)(i - row * p.a.q_heads);
  float s = 0.0f;
  if (row < p.a.q_rows && lane * V < p.a.head_dim) {
    const uint4 g4 = *reinterpret_cast<const uint4*>((const T*)p.d_o.x + row * p.d_o.row_stride + h * p.d_o.head_stride + lane * V);
    const uint4 o4 = *reinterpret_cast<const uint4*>((const T*)p.o.x + row * p.o.row_stride + h * p.o.head_stride + lane * V);
    const T *g = reinterpret_cast<const T*>(&g4), *o = reinterpret_cast<const T*>(&o4);
#pragma unroll
    for (int e = 0; e < V; ++e) s = fmaf(to_f(g[e]), to_f(o[e]), s);
  }
  for (int o = lanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (row < p.a.q_rows && lane == 0) p.drow[h * p.a.q_rows + row] = s;
}

// Where the pass itself has nothing to do
__global__ void __launch_bounds__(256) clear_kernel(const __grid_constant__ RaggedAttn p, bool backward) { clear_block(p, backward, blockIdx.x, 256); }
void clear_alone(Launcher& lc, const RaggedAttn& r, bool backward) {
  clear_kernel<<<kClearers, 256, 0, lc.stream>>>(r, backward);
  lc.count();
  lc.check();
}

template <int HD>
constexpr int smem_of(int tiles, int scores) {
  return (tiles * TILE * kStride<HD> + scores * TILE * PS) * 4;
}

template <typename K>
void allow_smem(Launcher& lc, K kernel, int smem, bool& done) {
  if (done) return;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  done = e == cudaSuccess;
  if (!done && lc.err == cudaSuccess) lc.err = e;
}

// Blocks that share each of `walks` walks of `tiles` tiles: twice as many for as long as blocks are fewer than the chip takes at a time and every
// block has a tile.  Shared against one block a walk: 3 x 421 rows, 6 query heads on 2 key heads of 64, 39 against 45 us forward and 116 against 226
// backward; 2 x 1024 rows, 8 on 2 of 128, backward 504 against 1044; 2048 rows, 8 heads of 64, forward 163 against 228; 5 x 77 rows, 4 heads of 64,
// 12.6 against 16.4 and 21 against 27.  Backward up to 296 blocks instead of 148: 3 x 421 rows 131 against 112, 4 x 512 rows of 8 heads 198 against 175.
int ranks_of(int64_t walks, int64_t at_a_time, int64_t tiles) {
  int r = 1;
  while (r < 8 && walks * r < at_a_time && 2 * r <= tiles) r *= 2;
  return r;
}

template <int HD>
void forward_f32(Launcher& lc, const RaggedAttn& given) {
  RaggedAttn r = with_walks(given, TILE);
  constexpr int kSmem = smem_of<HD>(5, 1);
  static PerDevice<bool> set;
  allow_smem(lc, ragged_fwd_kernel<HD>, kSmem, set.here());
  const int64_t blocks = blocks_of(r.a.q_len, TILE, r.a.q_heads, r.a.sequences);
  const int ranks = ranks_of(blocks, HD == 64 ? 2 * 148 : 148, (r.a.kv_len + TILE - 1) / TILE);
  r.pass_blocks = (uint32_t)(blocks * ranks);
  launch_chained(lc, ragged_fwd_kernel<HD>, dim3((unsigned)(blocks * ranks) + (r.a.fresh ? kClearers : 0)), THREADS, kSmem, ranks, r, ranks);
}
template <int HD>
void backward_f32(Launcher& lc, const RaggedAttn& given) {
  const RaggedAttn r = with_walks(given, TILE);
  constexpr int kSmem = smem_of<HD>(6, HD > 64 ? 1 : 2);
  static PerDevice<bool> set;
  allow_smem(lc, ragged_bwd_kernel<HD>, kSmem, set.here());
  const int64_t kv = blocks_of(r.a.kv_len, TILE, r.a.kv_heads, r.a.sequences), q = blocks_of(r.a.q_len, TILE, r.a.q_heads, r.a.sequences);
  const int ranks = ranks_of(kv, 148, (int64_t)(r.a.q_heads / r.a.kv_heads) * ((r.a.q_len + TILE - 1) / TILE));
  const int64_t blocks = (kv + (q + ranks - 1) / ranks) * ranks;
  if (blocks) launch_chained(lc, ragged_bwd_kernel<HD>, dim3((unsigned)blocks), THREADS, kSmem, ranks, r, (unsigned)kv, (unsigned)q, ranks);
}

void row_dots(Launcher& lc, RaggedAttn r) {
  const int v = r.a.dtype == HBP_F32 ? 4 : 8;
  int lanes = 1;
  while (lanes * v < r.a.head_dim) lanes *= 2;
  const int64_t blocks = (r.a.q_rows * r.a.q_heads * lanes + 255) / 256;
  r.pass_blocks = (uint32_t)blocks;
  const unsigned grid = (unsigned)blocks + (r.a.fresh ? kClearers : 0);
  if (r.a.dtype == HBP_F32) row_dot_kernel<float><<<grid, 256, 0, lc.stream>>>(r, lanes);
  else row_dot_kernel<bf16><<<grid, 256, 0, lc.stream>>>(r, lanes);
  lc.count();
  lc.check();
}

hbp_status check_attention(const hbp_attention* a) {
  if (!a) return HBP_ERR_INVALID_ARG;
  if (a->dtype != HBP_F32 && a->dtype != HBP_BF16) return HBP_ERR_DTYPE;
  if (a->sequences < 0 || a->q_heads <= 0 || a->kv_heads <= 0 || a->q_heads % a->kv_heads || a->q_heads > 65535) return HBP_ERR_SHAPE;
  if (a->head_dim <= 0 || a->head_dim > 128 || a->head_dim % (a->dtype == HBP_F32 ? 4 : 8)) return HBP_ERR_SHAPE;
  if (a->q_len < 0 || a->kv_len < 0 || a->q_rows < 0 || a->kv_rows < 0 || a->q_rows > INT32_MAX || a->kv_rows > INT32_MAX) return HBP_ERR_SHAPE;
  if (!a->q_offsets && (int64_t)a->sequences * a->q_len > a->q_rows) return HBP_ERR_SHAPE;
  if (!a->kv_offsets && (int64_t)a->sequences * a->kv_len > a->kv_rows) return HBP_ERR_SHAPE;
  if (a->q_len > a->q_rows || a->kv_len > a->kv_rows) return HBP_ERR_SHAPE;
  if (!std::isfinite(a->scale) || a->fresh & ~(HBP_FRESH_O | HBP_FRESH_LSE | HBP_FRESH_DQ | HBP_FRESH_DK | HBP_FRESH_DV)) return HBP_ERR_INVALID_ARG;
  if (((uintptr_t)a->q_offsets | (uintptr_t)a->kv_offsets | (uintptr_t)a->status) & 3u) return HBP_ERR_SHAPE;
  // (as many blocks of 64 rows as one grid holds)
  if (blocks_of(a->q_len, TILE, a->q_heads, a->sequences) > INT32_MAX / 2 || blocks_of(a->kv_len, TILE, a->kv_heads, a->sequences) > INT32_MAX / 2 ||
      a->q_rows * a->q_heads > (int64_t)INT32_MAX * 8)
    return HBP_ERR_SHAPE;
  return HBP_OK;
}

hbp_status check_heads(const hbp_attention& a, const hbp_heads* const* t, int n) {
  const int v = a.dtype == HBP_F32 ? 4 : 8;
  for (int i = 0; i < n; ++i) {
    if (!t[i] || !t[i]->x) return HBP_ERR_INVALID_ARG;
    if (((uintptr_t)t[i]->x & 15u) || t[i]->row_stride % v || t[i]->head_stride % v || t[i]->row_stride < 0 || t[i]->head_stride < 0) return HBP_ERR_SHAPE;
  }
  return HBP_OK;
}
// An output: no two of its elements in one place, rows of heads or heads of rows.
hbp_status check_output(const hbp_attention& a, const hbp_heads& t, int64_t rows, int heads) {
  const int64_t rs = t.row_stride, hs = t.head_stride, w = a.head_dim;
  const bool apart = (rows <= 1 || rs >= (heads - 1) * hs + w) && (heads <= 1 || hs >= w);
  const bool across = (heads <= 1 || hs >= (rows - 1) * rs + w) && (rows <= 1 || rs >= w);
  return apart || across ? HBP_OK : HBP_ERR_SHAPE;
}

}  // namespace

}  // namespace hbp

using namespace hbp;

extern "C" {

hbp_status hbp_attention_forward(const hbp_attention* a, const hbp_heads* q, const hbp_heads* k, const hbp_heads* v, const hbp_heads* o,
                                 float* lse, void* cuda_stream) {
  hbp_status st = check_attention(a);
  if (st != HBP_OK) return st;
  const bool nothing = a->sequences == 0 || a->q_len == 0;
  const int fresh = rows_left_over(*a, a->q_rows, a->q_len) && a->q_rows ? a->fresh & (HBP_FRESH_O | HBP_FRESH_LSE) : 0;
  if (nothing && !fresh) return HBP_OK;
  const hbp_heads* const qt[4] = {q, o, k, v};
  st = nothing ? check_heads(*a, qt + 1, 1) : check_heads(*a, qt, a->kv_len ? 4 : 2);  // (no keys at all: their tensors may be empty)
  if (st != HBP_OK || (st = check_output(*a, *o, a->q_rows, a->q_heads)) != HBP_OK) return st;
  if (!lse) return HBP_ERR_INVALID_ARG;
  if ((uintptr_t)lse & 3u) return HBP_ERR_SHAPE;
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  RaggedAttn r = {};
  r.a = *a;
  r.a.fresh = fresh;
  r.o = *o; r.lse = lse;
  if (nothing) {
    clear_alone(lc, r, false);
    return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
  }
  r.q = *q;
  if (a->kv_len) { r.k = *k; r.v = *v; }
  if (a->dtype == HBP_BF16) {
    if (!ragged_forward_tc(lc, r)) return lc.err == cudaSuccess ? HBP_ERR_UNSUPPORTED : HBP_ERR_CUDA;
  } else if (a->head_dim <= 64) {
    forward_f32<64>(lc, r);
  } else {
    forward_f32<128>(lc, r);
  }
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}

hbp_status hbp_attention_scratch_bytes(const hbp_attention* a, size_t* bytes) {
  if (!bytes) return HBP_ERR_INVALID_ARG;
  const hbp_status st = check_attention(a);
  if (st != HBP_OK) return st;
  *bytes = (size_t)a->q_heads * a->q_rows * sizeof(float);
  return HBP_OK;
}

hbp_status hbp_attention_backward(const hbp_attention* a, const hbp_heads* d_o, const hbp_heads* q, const hbp_heads* k, const hbp_heads* v,
                                  const hbp_heads* o, const float* lse, const hbp_heads* dq, const hbp_heads* dk, const hbp_heads* dv,
                                  void* scratch, size_t scratch_bytes, void* cuda_stream) {
  hbp_status st = check_attention(a);
  if (st != HBP_OK) return st;
  const bool nothing = a->sequences == 0 || (a->q_len == 0 && a->kv_len == 0);
  const int fresh = (rows_left_over(*a, a->q_rows, a->q_len) && a->q_rows ? a->fresh & HBP_FRESH_DQ : 0) |
                    (rows_left_over(*a, a->kv_rows, a->kv_len) && a->kv_rows ? a->fresh & (HBP_FRESH_DK | HBP_FRESH_DV) : 0);
  if (nothing && !fresh) return HBP_OK;
  const hbp_heads* const qt[4] = {d_o, q, o, dq};
  const hbp_heads* const kt[4] = {k, v, dk, dv};
  const bool queries = !nothing && a->q_len, keys = !nothing && a->kv_len;
  auto output = [&](const hbp_heads* t, int64_t rows, int heads) {
    const hbp_status bad = check_heads(*a, &t, 1);
    return bad != HBP_OK ? bad : check_output(*a, *t, rows, heads);
  };
  if (queries && (st = check_heads(*a, qt, 3)) != HBP_OK) return st;
  if (keys && (st = check_heads(*a, kt, 2)) != HBP_OK) return st;
  if ((queries || fresh & HBP_FRESH_DQ) && (st = output(dq, a->q_rows, a->q_heads)) != HBP_OK) return st;
  if ((keys || fresh & HBP_FRESH_DK) && (st = output(dk, a->kv_rows, a->kv_heads)) != HBP_OK) return st;
  if ((keys || fresh & HBP_FRESH_DV) && (st = output(dv, a->kv_rows, a->kv_heads)) != HBP_OK) return st;
  RaggedAttn r = {};
  r.a = *a;
  r.a.fresh = fresh;
  if (queries || fresh & HBP_FRESH_DQ) r.dq = *dq;
  if (keys || fresh & HBP_FRESH_DK) r.dk = *dk;
  if (keys || fresh & HBP_FRESH_DV) r.dv = *dv;
  if (queries) {
    if (!lse) return HBP_ERR_INVALID_ARG;
    if (!scratch || ((uintptr_t)scratch & 15u) || scratch_bytes < (size_t)a->q_heads * a->q_rows * sizeof(float)) return HBP_ERR_WORKSPACE;
    if ((uintptr_t)lse & 3u) return HBP_ERR_SHAPE;
    r.q = *q; r.o = *o; r.d_o = *d_o;
    r.lse = const_cast<float*>(lse);
    r.drow = (float*)scratch;
  }
  if (keys) { r.k = *k; r.v = *v; }
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  if (queries) row_dots(lc, r);
  else if (fresh) clear_alone(lc, r, true);
  if (nothing) return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
  if (a->dtype == HBP_BF16) {
    if (!ragged_backward_tc(lc, r)) return lc.err == cudaSuccess ? HBP_ERR_UNSUPPORTED : HBP_ERR_CUDA;
  } else if (a->head_dim <= 64) {
    backward_f32<64>(lc, r);
  } else {
    backward_f32<128>(lc, r);
  }
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}

}  // extern "C"
