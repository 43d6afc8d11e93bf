// Attention over ragged batches on the tensor cores (bf16, heads up to 128 wide): the formulas are those of attention_ragged.cu.
//
// Heads are padded to HD = 64 or 128 channels: a tensor map is head_dim channels wide and its boxes 64, so that the missing ones
// arrive as zeros.  Tiles are rows of 128 bytes (64 channels) under the 128-byte swizzle, 64 channels after the other; the same tile is a
// K-major operand (contraction over channels) and an MN-major one (contraction over its rows).  A tile that reaches past
// its sequence holds rows of the next one, which may be anything: where rows are contracted over, the copying warp waits for such a
// tile and overwrites those rows with zeros before it hands the tile on (0 * NaN is not 0).
//
// Scores come from shared memory into tensor memory; the softmax warps turn them into bf16 probabilities that go back into the columns
// the scores came from and are the A operand of the next product there: they never pass through shared memory, whose bandwidth
// the products need (M = 128, N = 64, K = 16 reads 6 KB in the 32 clocks that it takes at the tensor cores' rate).
//
// Forward: a block owns 128 queries and walks over tiles of 64 keys with a running maximum and sum, one row per thread of four
// warps.  Two buffers of scores, so that the next ones are formed under these exponentials.  The output stays in tensor memory; it is scaled
// down only when a row's maximum has grown by more than 2^8 since the last time, which is rare (sums are float: 2^8 costs no
// precision).  Two blocks share an SM.  2 x 4096 rows, causal: 16 heads of 128 127 us (1.08 PFLOP/s of the products that are needed), 16 of 64 111 us
// (0.62).  Bound, at 64 channels, by the exponentials (512 clocks a tile and SM for 128 x 64 at 16 a clock; measured 670 in the loop), at 128
// by what the products read from shared memory.  Tiles of 128 keys in one buffer: 150 and 132 us, the scores read twice from tensor memory 176
// and 161.
//
// Backward: two kinds of block in one launch, so that every output has one owner and one order of its sums:
//   dK, dV   128 keys of a key head; walks over tiles of 64 queries of all query heads of its group
//            S^T = K Q^T, dP^T = V dO^T;  P^T = exp(S^T - lse), dS^T = P^T (dP^T - D);  dV += P^T dO, dK += dS^T Q
//   dQ       128 queries; walks over tiles of 64 keys:  S = Q K^T, dP = dO V^T;  dQ += dS K
// That is seven products where five would do with sums in memory that blocks add to in no fixed order.  Probabilities and dS are rounded to
// bf16 as operands, and so is o, which D comes from: gradients are off by 2.4e-3 to 2.8e-3 in the norm, 1.7e-3 of it the output's own
// rounding.  HD = 128 takes all of tensor memory: two buffers of scores, two groups of softmax warps that take the tiles in turn; HD = 64 runs
// two blocks an SM, a buffer each, and overlaps the two halves of a tile (scores and probabilities, dP and dS) instead.  2 x 4096 rows, causal, of the
// five products that are needed: 16 heads of 128 440 us (0.78 PFLOP/s), 16 of 64 288 us (0.60).  At 128 channels the products and the
// copies read and write 1400 (dK, dV) and 1150 (dQ) clocks' worth of shared memory a tile, of 1670 and 1420 measured; at 64 a tile's chain of
// product, exponentials and product bounds it (2100 and 1630 clocks, two at a time).  HD = 64 with three buffers and one block an SM: 366 us; sixteen
// columns a warp instead of 32: 308.
// Few blocks with long walks are shared by clusters, in both passes (ranks_of below); the query heads of a key head share a block where queries are
// few (packed_heads): single queries are bound by the keys' and values' bytes (16 x 1 query, 4096 keys, 4 key heads of 128: 4.9 TB/s).
// All waits are bounded.
#include "attention_ragged.cuh"
#include "float_pairs.cuh"
#include "ring_drain.cuh"

namespace hbp {

using namespace tc;

namespace {

constexpr int BIG = 128;     // rows of a block
constexpr int SMALL = 64;    // rows of a tile that a block walks over, and of every copy
constexpr int SUB = 64;      // channels of a run of tile rows (128 bytes)
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float kGrowth = 8.0f;  // log2 of how far a row's maximum may grow before what was summed is scaled

struct RaggedMaps {
  CUtensorMap q, k, v, d_o;
};

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float ld_early(const float* p) {  // a load that is not moved down to its first use
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ bool elect_one() {
  uint32_t is_leader;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(is_leader));
  return is_leader != 0;
}
__device__ __forceinline__ uint64_t desc_add(uint64_t d, uint32_t bytes) { return d + (uint64_t)(bytes >> 4); }

// bf16 x bf16 -> float, M = 128, A K-major (or in tensor memory)
template <int N, int kBmn>
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)kBmn << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(BIG >> 4) << 24);
// A in tensor memory: 128 lanes, K = 16 in 8 columns
__device__ __forceinline__ void tc_mma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accum)
      : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t taddr, const float* v) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
  tc_st16(taddr, r);
  tc_st16(taddr + 16, r + 16);
}
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}

// 64 rows from row `row` of head `head` on, all HD channels, into a tile of `tile_rows` rows a run of channels
template <int HD>
__device__ __forceinline__ void copy_rows(uint32_t dst, int tile_rows, const CUtensorMap* tm, uint32_t bar, int head, int row) {
#pragma unroll
  for (int c = 0; c < HD / SUB; ++c) tma_load_3d(dst + c * tile_rows * 128, tm, bar, c * SUB, head, row);
}
// rows [from, rows) of a tile become zeros; the whole warp
template <int HD>
__device__ __forceinline__ void clear_rows(uint32_t tile, int rows, int from, int lane) {
#pragma unroll
  for (int c = 0; c < HD / SUB; ++c)
    for (int i = from * 8 + lane; i < rows * 8; i += 32) st_shared16(tile + c * rows * 128 + i * 16, make_uint4(0, 0, 0, 0));
}
// A bounded wait (mbar_wait) of the whole warp, where the status word may be missing: all lanes go on or none does.
__device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status) {
  bool ok = true;
  uint64_t t0 = 0;
  for (uint32_t spin = 0; !mbar_try_wait(bar, parity); ++spin) {
    if ((spin & 255u) != 255u) continue;
    const uint64_t now = global_ns();
    if (t0 == 0) t0 = now;
    if (*abort_flag || now - t0 > WAIT_LIMIT_NS) {
      if (!*abort_flag && status) atomicExch(status, (int)HBP_ERR_TIMEOUT);
      *abort_flag = 1;
      ok = false;
      break;
    }
  }
  return __all_sync(0xffffffffu, ok);
}
// Tensor memory is taken by warp 1, which gives up the permit for more at once: an SM's next block does not begin before.
__device__ __forceinline__ void take(uint32_t* slot, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
// A block that has nothing to do.
__device__ __forceinline__ void give_back(int warp, const uint32_t* slot, uint32_t columns) {
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*reinterpret_cast<const volatile uint32_t*>(slot)), "r"(columns) : "memory");
}
// The end of a block: after a wait that gave up, every copy and product is outlasted first.
__device__ __forceinline__ void leave(int warp, uint32_t tmem, uint32_t columns, volatile int* abort_flag) {
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) outlast_copies();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
  }
}
// Rows of a staged tile (this warp's 32 rows from `row0` on, kUnits 16-byte units from unit `unit0` on) to memory, neighbouring lanes
// along a row; rows behind the sequence and channels behind the head are left alone.
template <int kUnits>
__device__ __forceinline__ void store_staged(uint32_t tile, int row0, int unit0, bf16* base, int64_t row_stride, int rows_there, int head_dim, int lane) {
  constexpr int kRows = 32 / kUnits, kAtOnce = 4;
  const int u = unit0 + lane % kUnits, first = row0 + lane / kUnits;
  bf16* at = base + (int64_t)first * row_stride + u * 8;
#pragma unroll
  for (int i = 0; i < kUnits; i += kAtOnce) {  // (32 rows are kUnits steps of kRows)
    uint4 x[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) x[j] = ld_shared16(swz(tile + (u >> 3) * BIG * 128, first + (i + j) * kRows, u & 7));
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      if (first + (i + j) * kRows < rows_there && u * 8 < head_dim) *reinterpret_cast<uint4*>(at) = x[j];
      at += kRows * row_stride;
    }
  }
}

// ---- walks shared by a cluster: few blocks with long walks leave most of the chip idle.  The blocks of a cluster take the tiles of a walk in
// turn; each leaves its sums in its shared memory, and each puts together those of all for its share of the rows, in the blocks' order.
constexpr int MOST_RANKS = 8;
__device__ __forceinline__ int tiles_of(int tiles, int rank, int ranks) { return (tiles - rank + ranks - 1) >> (__ffs(ranks) - 1); }
// Rows of HD floats, their 16-byte units permuted among eight by the row: one row per lane is written without bank conflicts.
template <int HD>
__device__ __forceinline__ uint32_t sum_at(uint32_t base, int row, int unit) {
  return base + (row * (HD / 4) + (unit ^ (row & 7))) * 16;
}
// This thread's row of an accumulator in tensor memory (zeros if nothing was added up); `at` includes the warp's lanes.
template <int HD>
__device__ __forceinline__ void leave_sums(uint32_t base, bool any, uint32_t at, int row, int from = 0, int to = HD) {
#pragma unroll 1
  for (int c = from; c < to; c += 32) {
    float o[32];
    if (any) tc_ld32(at + c, o);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (any) x = *reinterpret_cast<const uint4*>(o + 4 * u);
      st_shared16(sum_at<HD>(base, row, c / 4 + u), x);
    }
  }
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// The rows' sums of all blocks of the cluster times factor(row of this block's share, block), added up: put(row, unit, sums) for each eight channels of
// the first `there` rows of this block's share.  Sixteen loads of a thread are under way at a time: one block's two at a time, two blocks' 128 rows of 80 channels took 5 us instead of 2.5.
template <int HD, int R, typename Factor, typename Put>
__device__ __forceinline__ void merge_sums(uint32_t base, int rank, int there, int t, int threads, Factor factor, Put put) {
  constexpr int NI = MOST_RANKS / R, units = HD / 8;
  const int n_units = min(BIG / R, there) * units;
  for (int i = t; i < n_units; i += NI * threads) {
    float4 x[NI][R][2];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int j = i + n * threads;
      if (j >= n_units) break;  // (every load's value is used: none is under way at the end)
#pragma unroll
      for (int b = 0; b < R; ++b) {
#pragma unroll
        for (int h = 0; h < 2; ++h) x[n][b][h] = ld_cluster4(sum_at<HD>(map_to_cta(base, b), rank * (BIG / R) + j / units, 2 * (j % units) + h));
      }
    }
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int j = i + n * threads;
      if (j >= n_units) break;
      float v[8] = {};
#pragma unroll
      for (int b = 0; b < R; ++b) {
        const float f = factor(j / units, b);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v[4 * h] = fmaf(f, x[n][b][h].x, v[4 * h]);
          v[4 * h + 1] = fmaf(f, x[n][b][h].y, v[4 * h + 1]);
          v[4 * h + 2] = fmaf(f, x[n][b][h].z, v[4 * h + 2]);
          v[4 * h + 3] = fmaf(f, x[n][b][h].w, v[4 * h + 3]);
        }
      }
      put(j / units, j % units, v);
    }
  }
}
template <int HD, typename Factor, typename Put>
__device__ __forceinline__ void merge_sums(int ranks, uint32_t base, int rank, int there, int t, int threads, Factor factor, Put put) {
  if (ranks == 1) merge_sums<HD, 1>(base, rank, there, t, threads, factor, put);
  else if (ranks == 2) merge_sums<HD, 2>(base, rank, there, t, threads, factor, put);
  else if (ranks == 4) merge_sums<HD, 4>(base, rank, there, t, threads, factor, put);
  else merge_sums<HD, 8>(base, rank, there, t, threads, factor, put);
}
// Nothing seen: sums of 0, outputs of 0 and a log-sum-exp of -infinity (a sum that is NaN stays NaN)
__device__ __forceinline__ float inverse(float total) { return total > 0.0f ? 1.0f / total : total; }
__device__ __forceinline__ float log_sum(float top, float total) { return total == 0.0f ? -INFINITY : (top + __log2f(total)) * LN2; }

// ------------------------------------------------------------------------------------------- forward
constexpr int FWD_THREADS = 192;  // warp 0 copies, warp 1 issues the products, warps 2..5 softmax (TMEM lane quarter = warp & 3)
template <int HD>
struct Fwd {
  static constexpr int kStages = HD == 64 ? 3 : 2;  // of keys, and of values (as many as two blocks an SM have room for)
  static constexpr int kBig = BIG * HD * 2, kSmall = SMALL * HD * 2;
  static constexpr int kSmem = kBig + 2 * kStages * kSmall + 256 + 1024;
};

// kShared: walks are shared by a cluster; kPacked, of those: `pack` query heads are a block's rows, query by query (a kernel of its own: in one, the others' took 119 us instead of 113, 2 x 4096 rows, 16 heads of 64).
// 128 registers (256 threads are told): at 132 a quarter of an SM holds three warps but not four, and when the second of two blocks ends first, a new one
// has to wait for the other too (ragged batch of cross attention 31 against 36 us, 16 heads of 128 126 against 131).
template <int HD, bool kShared, bool kPacked>
__global__ void __launch_bounds__(256, 2) ragged_fwd_tc_kernel(const __grid_constant__ RaggedMaps m, const __grid_constant__ RaggedAttn p,
                                                                       const int ranks_given, const int pack_given) {
  if (blockIdx.x >= p.pass_blocks) return clear_block(p, false, (int)(blockIdx.x - p.pass_blocks), FWD_THREADS);
  const int ranks = kShared ? ranks_given : 1, pack = kPacked ? pack_given : 1;
  using C = Fwd<HD>;
  constexpr int NS = C::kStages, NB = 2;
  const int rank = kShared ? (int)(blockIdx.x & (unsigned)(ranks - 1)) : 0;  // (a power of two of them)
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sQ = base, sK = base + C::kBig, sV = sK + NS * C::kSmall;
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(aligned + C::kBig + 2 * NS * C::kSmall);
  const uint32_t bars = smem_u32(bar_mem);
  const uint32_t bQ = bars, bDone = bars + 8, bTail = bars + 16;
  auto bProbs = [&](int b) { return bars + 24 + 8 * b; };
  auto bScores = [&](int b) { return bars + 24 + 8 * (NB + b); };
  auto bKFull = [&](int s) { return bars + 24 + 8 * (2 * NB + s); };
  auto bKFree = [&](int s) { return bars + 24 + 8 * (2 * NB + NS + s); };
  auto bVFull = [&](int s) { return bars + 24 + 8 * (2 * NB + 2 * NS + s); };
  auto bVFree = [&](int s) { return bars + 24 + 8 * (2 * NB + 3 * NS + s); };
  constexpr int kBars = 3 + 2 * NB + 4 * NS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_mem + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == 1) take(tmem_slot, 256);  // (first of all, so that the SM's second block begins 0.8 us earlier: 16 heads of 128, 126 against 127 us)

  BlockOf w = block_at(kShared ? blockIdx.x >> (__ffs(ranks) - 1) : blockIdx.x, p.q_walks, true);
  const SeqPair sq = sequence_pair(p.a, w, true);
  const int q0 = w.blk * BIG;
  if (q0 >= sq.nq) {  // (all blocks of the cluster)
    give_back(warp, tmem_slot, 256);
    return;
  }
  const int kh = kPacked ? w.h : (int)p.by_group((uint32_t)w.h);
  const int shift = sq.nk - sq.nq;  // causal: query i sees keys 0 .. i + shift
  const int seen = p.a.causal ? min(sq.nk, min(q0 + BIG, sq.nq) + shift) : sq.nk;
  // this block's tiles: rank, rank + ranks, ...
  const int tiles = seen > 0 ? (seen + SMALL - 1) / SMALL : 0, n_it = kShared ? tiles_of(tiles, rank, ranks) : tiles;


  if (threadIdx.x == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(bars + 8 * i, i >= 3 && i < 3 + NB ? 4 : 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (n_it > 0) {  // the first copies are under way while the others get ready
      if (kPacked) {  // (one box of heads and queries; the rows behind hold anything)
        mbar_expect_tx(bQ, HD * 2 * pack * p.a.q_len);
        copy_rows<HD>(sQ, BIG, &m.q, bQ, w.h * pack, (int)sq.q0);
      } else {
        mbar_expect_tx(bQ, C::kBig);
        for (int r = 0; r < BIG; r += SMALL) copy_rows<HD>(sQ + r * 128, BIG, &m.q, bQ, w.h, (int)sq.q0 + q0 + r);
      }
      mbar_expect_tx(bKFull(0), C::kSmall);
      copy_rows<HD>(sK, SMALL, &m.k, bKFull(0), kh, (int)sq.k0 + rank * SMALL);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, tO = tmem + 64 * NB;  // scores, and then probabilities, of buffer b: columns 64 b ..

  if (warp == 0) {
    bool ok = n_it > 0;
    for (int it = 0; it < n_it && ok; ++it) {
      const int s = it % NS;
      const uint32_t free_parity = ((uint32_t)(it / NS) & 1u) ^ 1u;
      const int tile = kShared ? rank + it * ranks : it, row = (int)sq.k0 + tile * SMALL;
      if (!wait_all(bKFree(s), free_parity, abort_flag, p.a.status)) { ok = false; break; }
      if (lane == 0 && it > 0) {
        mbar_expect_tx(bKFull(s), C::kSmall);
        copy_rows<HD>(sK + s * C::kSmall, SMALL, &m.k, bKFull(s), kh, row);
      }
      if (!wait_all(bVFree(s), free_parity, abort_flag, p.a.status)) { ok = false; break; }
      const int there = sq.nk - tile * SMALL;  // rows of the sequence in this tile
      const uint32_t bar = there < SMALL ? bTail : bVFull(s);
      if (lane == 0) {
        mbar_expect_tx(bar, C::kSmall);
        copy_rows<HD>(sV + s * C::kSmall, SMALL, &m.v, bar, kh, row);
      }
      if (there < SMALL) {  // the last tile: what is behind the sequence becomes zeros
        if (!wait_all(bTail, 0, abort_flag, p.a.status)) { ok = false; break; }
        clear_rows<HD>(sV + s * C::kSmall, SMALL, there, lane);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bVFull(s));
      }
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    const int steps = (p.a.head_dim + 15) / 16;  // of the contraction over channels (the channels behind are zeros)
    const uint64_t dQ = make_desc(sQ, 16, 1024), dK = make_desc(sK, 16, 1024), dV = make_desc(sV, SMALL * 128, 1024);
    auto scores = [&](int it) {
      const uint32_t off = (uint32_t)(it % NS) * C::kSmall, t = tmem + 64 * (it % NB);
      if (leader) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
          if (HD == 64 || k < steps) tc_mma(t, desc_add(dQ, (k / 4) * BIG * 128 + 32 * (k % 4)), desc_add(dK, off + (k / 4) * SMALL * 128 + 32 * (k % 4)), kIdesc<SMALL, 0>, k != 0);
        tc_commit(bScores(it % NB));
        tc_commit(bKFree(it % NS));
      }
    };
    bool ok = n_it == 0 || wait_all(bQ, 0, abort_flag, p.a.status);
    for (int it = 0; it < NB && it < n_it && ok; ++it) {
      ok = wait_all(bKFull(it % NS), 0, abort_flag, p.a.status);
      tc_fence_after();
      if (ok) scores(it);
    }
    for (int it = 0; it < n_it && ok; ++it) {
      const int s = it % NS;
      if (!wait_all(bVFull(s), (uint32_t)(it / NS) & 1u, abort_flag, p.a.status) ||
          !wait_all(bProbs(it % NB), (uint32_t)(it / NB) & 1u, abort_flag, p.a.status)) { ok = false; break; }
      tc_fence_after();
      if (leader) {
#pragma unroll
        for (int k = 0; k < SMALL / 16; ++k)
          tc_mma_ts(tO, tmem + 64 * (it % NB) + 8 * k, desc_add(dV, (uint32_t)s * C::kSmall + 2048 * k), kIdesc<HD, 1>, (it | k) != 0);
        tc_commit(bVFree(s));
      }
      if (it + NB < n_it) {  // into the buffer that these have read (products run in order)
        if (!wait_all(bKFull((it + NB) % NS), (uint32_t)((it + NB) / NS) & 1u, abort_flag, p.a.status)) { ok = false; break; }
        tc_fence_after();
        scores(it + NB);
      }
    }
    if (leader) tc_commit(bDone);
  } else {
    const int quarter = warp & 3, row = quarter * 32 + lane, qrow = q0 + (kPacked ? row / pack : row);
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const float scale2 = fabsf(p.a.scale) * LOG2E;
    float top = -INFINITY;  // the reference of the sums, in units of log2
    f32x2 sum0 = both(0.0f), sum1 = sum0;
    const int last = p.a.causal ? min(sq.nk - 1, qrow + shift) : sq.nk - 1;  // the last key this row sees
    bool ok = true;
    for (int it = 0; it < n_it; ++it) {
      if (!wait_all(bScores(it % NB), (uint32_t)(it / NB) & 1u, abort_flag, p.a.status)) { ok = false; break; }
      tc_fence_after();
      const int c0 = (kShared ? rank + it * ranks : it) * SMALL;
      const uint32_t t = tmem + lanes + 64 * (it % NB);
      const bool full = c0 + SMALL <= sq.nk && (!p.a.causal || c0 + SMALL - 1 <= q0 + shift);  // every row of the block sees the whole tile
      float sc[SMALL];  // this row's scores
      tc_ld32_async(t, sc);
      tc_ld32_async(t + 32, sc + 32);
      tc_ld_wait();
      if (p.a.scale < 0.0f) {
#pragma unroll
        for (int i = 0; i < SMALL; ++i) sc[i] = -sc[i];
      }
      if (!full) {
#pragma unroll
        for (int i = 0; i < SMALL; ++i) sc[i] = c0 + i <= last ? sc[i] : -INFINITY;
      }
      float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < SMALL; i += 8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) tops[e] = fmaxf(tops[e], fmaxf(sc[i + e], sc[i + 4 + e]));
      }
      float most = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      most = most == -INFINITY ? most : most * scale2;  // (a scale of 0 times nothing is not a maximum)
      if (it == 0) {
        top = most;
      } else {
        const bool grown = most > top + kGrowth;
        if (__any_sync(0xffffffffu, grown)) {  // scale what was summed down to the new reference
          const float keep = grown ? fast_exp2(top - most) : 1.0f;
          if (grown) top = most;
          sum0 = mul2(sum0, both(keep));
          sum1 = mul2(sum1, both(keep));
          if (!wait_all(bVFree((it - 1) % NS), (uint32_t)((it - 1) / NS) & 1u, abort_flag, p.a.status)) { ok = false; break; }
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            float o[32];
            tc_ld32(tO + lanes + c, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= keep;
            tc_st32(tO + lanes + c, o);
          }
        }
      }
      // (nothing seen so far: -infinity less 0; a scale of 0 times -infinity would not be -infinity)
      const f32x2 mul = both(scale2 > 0.0f ? scale2 : 1e-30f), ref = both(top == -INFINITY ? 0.0f : -top);
#pragma unroll
      for (int c = 0; c < SMALL; c += 32) {
        uint32_t packed[16];
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float2 x = floats_of(fma2(pair_of(sc[c + i], sc[c + i + 1]), mul, ref)), y = floats_of(fma2(pair_of(sc[c + i + 2], sc[c + i + 3]), mul, ref));
          const float e0 = fast_exp2(x.x), e1 = fast_exp2(x.y), e2 = fast_exp2(y.x), e3 = fast_exp2(y.y);
          sum0 = add2(sum0, pair_of(e0, e1));
          sum1 = add2(sum1, pair_of(e2, e3));
          packed[i / 2] = pack2(e0, e1);
          packed[i / 2 + 1] = pack2(e2, e3);
        }
        tc_st16(t + c / 2, packed);  // (columns whose scores this thread has read)
      }
      tc_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bProbs(it % NB));
    }
    ok = ok && wait_all(bDone, 0, abort_flag, p.a.status);
    if (ok && !kShared) {
      tc_fence_after();
      const float2 sums = floats_of(add2(sum0, sum1));
      const float total = sums.x + sums.y;
      const float inv = inverse(total);
#pragma unroll 1
      for (int c = 0; c < HD; c += 64) {
        float o[64];
        if (n_it > 0) {
          tc_ld32_async(tO + lanes + c, o);
          tc_ld32_async(tO + lanes + c + 32, o + 32);
          tc_ld_wait();
        }
#pragma unroll
        for (int i = 0; i < 64; ++i) o[i] = total == 0.0f ? 0.0f : o[i] * inv;
#pragma unroll
        for (int u = 0; u < 8; ++u) st_shared16(swz(sQ + (c / SUB) * BIG * 128, row, u), pack8(o + 8 * u));
      }
      __syncwarp();
      store_staged<HD / 8>(sQ, quarter * 32, 0, (bf16*)p.o.x + (sq.q0 + q0) * p.o.row_stride + w.h * p.o.head_stride, p.o.row_stride, sq.nq - q0, p.a.head_dim, lane);
      if (qrow < sq.nq) p.lse[w.h * p.a.q_rows + sq.q0 + qrow] = log_sum(top, total);
    } else if (ok) {  // for the other blocks of the cluster: this one's sums, in the place of keys and values, and its reference and total in the queries'
      tc_fence_after();
      const float2 sums = floats_of(add2(sum0, sum1));
      const float total = sums.x + sums.y;
      if (quarter * 32 < (sq.nq - q0) * pack) leave_sums<HD>(sK, n_it > 0, tO + lanes, row);
      asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(sQ + row * 8), "f"(top), "f"(total) : "memory");
    }
  }
  // (before the blocks of a cluster wait for one another: two clusters of two calls that each held tensor memory the other needs would wait for good)
  leave(warp, tmem, 256, abort_flag);
  if (kShared) {
    cluster_sync();
    const int rows = BIG / ranks, first = rank * rows, t = threadIdx.x;  // this block's share
    const int there = min(rows, (sq.nq - q0) * pack - first);
    float* factors = reinterpret_cast<float*>(aligned + BIG * 8);        // [row][16]: the blocks' factors; 1 / total (-1: nothing seen)
    if (t < there) {
      float most = -INFINITY, total = 0.0f;
      float2 st[MOST_RANKS];
#pragma unroll
      for (int b = 0; b < MOST_RANKS; ++b) st[b] = b < ranks ? ld_cluster2(map_to_cta(sQ + (first + t) * 8, b)) : make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int b = 0; b < MOST_RANKS; ++b) most = fmaxf(most, st[b].x);
#pragma unroll
      for (int b = 0; b < MOST_RANKS; ++b) {
        const float f = most == -INFINITY ? 1.0f : fast_exp2(st[b].x - most);
        total = fmaf(f, st[b].y, total);
        factors[t * 16 + b] = f;
      }
      factors[t * 16 + MOST_RANKS] = total == 0.0f ? -1.0f : inverse(total);
      p.lse[(w.h * pack + (first + t) % pack) * p.a.q_rows + sq.q0 + q0 + (first + t) / pack] = log_sum(most, total);
    }
    __syncthreads();
    bf16* out = (bf16*)p.o.x + (sq.q0 + q0) * p.o.row_stride + (int64_t)(w.h * pack) * p.o.head_stride;
    merge_sums<HD>(ranks, sK, rank, there, t, FWD_THREADS, [&](int r, int b) { return factors[r * 16 + b]; },
                   [&](int r, int u, float (&v)[8]) {
                     if (u * 8 >= p.a.head_dim) return;
                     const float inv = factors[r * 16 + MOST_RANKS];
#pragma unroll
                     for (int e = 0; e < 8; ++e) v[e] = inv < 0.0f ? 0.0f : v[e] * inv;
                     *reinterpret_cast<uint4*>(out + (int64_t)((first + r) / pack) * p.o.row_stride + (int64_t)((first + r) % pack) * p.o.head_stride + u * 8) = pack8(v);
                   });
    cluster_sync();  // (no block ends while another reads its shared memory)
  }
}

// ------------------------------------------------------------------------------------------- backward
template <int HD>
struct Bwd {
  static constexpr int kBuffers = HD == 64 ? 1 : 2;  // of scores
  // Groups of eight softmax warps, two to a lane quarter of tensor memory; they take the tiles in turn.
  static constexpr int kGroups = HD == 64 ? 1 : 2;
  static constexpr int kThreads = 64 + 256 * kGroups;  // warp 0 copies, warp 1 issues the products
  static constexpr int kStages = HD == 64 ? 3 : 4;
  static constexpr int kBig = BIG * HD * 2, kSmall = SMALL * HD * 2;
  static constexpr int kStats = 2 * SMALL * 4;  // minus log-sum-exp and minus D of a tile's queries (dK, dV)
  static constexpr int kStage = 2 * kSmall;
  static constexpr int kSmem = 2 * kBig + kStages * (kStage + kStats) + 256 + 1024;
  static constexpr uint32_t kColumns = HD == 64 ? 256 : 512;
  static constexpr int kBlocksAnSm = HD == 64 ? 2 : 1;
};

template <int HD, bool kDKV, bool kShared>
__device__ __forceinline__ void ragged_bwd_body(const RaggedMaps& m, const RaggedAttn& p, BlockOf w, const int rank, const int ranks_given) {
  const int ranks = kShared ? ranks_given : 1;
  using C = Bwd<HD>;
  constexpr int NB = C::kBuffers, NS = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* aligned = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sBig0 = base, sBig1 = base + C::kBig, sSmall = base + 2 * C::kBig;
  float* stats = reinterpret_cast<float*>(aligned + 2 * C::kBig + NS * C::kStage);  // [stage][log-sum-exp, D][64]
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(aligned + 2 * C::kBig + NS * (C::kStage + C::kStats));
  const uint32_t bars = smem_u32(bar_mem);
  const uint32_t bBig = bars, bDone = bars + 8, bTail = bars + 16;
  // of buffer b: the scores' columns may be taken over by the next ones (dK, dV: and hold probabilities); dS is there; scores; dP
  auto bProbs = [&](int b) { return bars + 24 + 8 * b; };
  auto bDS = [&](int b) { return bars + 24 + 8 * (NB + b); };
  auto bScores = [&](int b) { return bars + 24 + 8 * (2 * NB + b); };
  auto bDP = [&](int b) { return bars + 24 + 8 * (3 * NB + b); };
  auto bFull = [&](int s) { return bars + 24 + 8 * (4 * NB + s); };
  auto bFree = [&](int s) { return bars + 24 + 8 * (4 * NB + NS + s); };
  constexpr int kBars = 3 + 4 * NB + 2 * NS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_mem + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;


  const SeqPair sq = sequence_pair(p.a, w, !kDKV);
  const int big0 = w.blk * BIG, n_big = kDKV ? sq.nk : sq.nq, n_small = kDKV ? sq.nq : sq.nk;
  if (big0 >= n_big) {  // (all blocks of a cluster)
    chain_wait();
    return;
  }
  const int shift = p.a.causal ? sq.nk - sq.nq : sq.nk;  // query i sees keys 0 .. i + shift (capped by nk)
  // tiles of the other side: queries from the first that sees key big0 on; keys up to the last that the block's last query sees
  const int t_beg = kDKV && p.a.causal ? max(0, big0 - shift) / SMALL : 0;
  const int t_rows = kDKV ? n_small : p.a.causal ? min(n_small, min(big0 + BIG, n_big) + shift) : n_small;
  const int tiles = max(0, (max(t_rows, 0) + SMALL - 1) / SMALL - t_beg);
  // this block's tiles among those of all heads, one head after the other: rank, rank + ranks, ...
  const int n_all = kDKV ? tiles * p.group : tiles, n_it = kShared ? tiles_of(n_all, rank, ranks) : n_all;
  const int q_head0 = kDKV ? w.h * p.group : w.h, k_head = kDKV ? w.h : (int)p.by_group((uint32_t)w.h);

  if (threadIdx.x == 0) {
    // probabilities, dS: eight warps; full: the copies, and what the copying warp adds itself; scores of dK, dV: the products, and the warp that
    // issues them, which has seen the statistics there and passes them on
    for (int i = 0; i < kBars; ++i) {
      const bool warps = i >= 3 && i < 3 + 2 * NB, two = (kDKV && i >= 3 + 2 * NB && i < 3 + 3 * NB) || (i >= 3 + 4 * NB && i < 3 + 4 * NB + NS);
      mbar_init(bars + 8 * i, warps ? 8 : two ? 2 : 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (n_it > 0) {
      mbar_expect_tx(bBig, 2 * C::kBig);
      for (int r = 0; r < BIG; r += SMALL) {
        const int row = (int)(kDKV ? sq.k0 : sq.q0) + big0 + r;
        copy_rows<HD>(sBig0 + r * 128, BIG, kDKV ? &m.k : &m.q, bBig, w.h, row);
        copy_rows<HD>(sBig1 + r * 128, BIG, kDKV ? &m.v : &m.d_o, bBig, w.h, row);
      }
    }
  }
  if (warp == 1) take(tmem_slot, C::kColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // columns of buffer b: scores 128 b .., dP 128 b + 64 ..; probabilities of the first 32 rows of a tile in the first 16 of them, those of the
  // others 32 columns on (a warp writes only where it has read)
  const uint32_t tAcc0 = tmem + 128 * NB, tAcc1 = tAcc0 + HD;

  if (warp == 0) {
    bool ok = n_it > 0;
    int tails = 0, at_tile = 0, head = kDKV ? q_head0 : k_head;
    chain_wait();
    for (int it = 0; it < n_it && ok; ++it) {
      at_tile += it == 0 ? rank : ranks;
      for (; kDKV && at_tile >= tiles; at_tile -= tiles) ++head;
      const int s = it % NS, r0 = (t_beg + at_tile) * SMALL;
      const uint32_t tile = sSmall + s * C::kStage;
      if (!wait_all(bFree(s), ((uint32_t)(it / NS) & 1u) ^ 1u, abort_flag, p.a.status)) { ok = false; break; }
      const int there = n_small - r0;
      const bool tail = there < SMALL;
      const uint32_t bar = tail ? bTail : bFull(s);
      if (lane == 0) {
        const int row = (int)(kDKV ? sq.q0 : sq.k0) + r0;
        mbar_expect_tx(bar, 2 * C::kSmall);
        copy_rows<HD>(tile, SMALL, kDKV ? &m.q : &m.k, bar, head, row);
        copy_rows<HD>(tile + C::kSmall, SMALL, kDKV ? &m.d_o : &m.v, bar, head, row);
      }
      if (kDKV) {
        float* st = stats + s * 2 * SMALL;
        const int64_t at = (int64_t)head * p.a.q_rows + sq.q0 + r0;
        float v[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = i * 32 + lane;
          v[i] = r < there ? ld_early(p.lse + at + r) : -INFINITY;
          v[2 + i] = r < there ? ld_early(p.drow + at + r) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // a query that sees nothing, or is none, has probabilities of 0: exp2(s - infinity)
          st[i * 32 + lane] = v[i] == -INFINITY ? v[i] : v[i] * -LOG2E;
          st[SMALL + i * 32 + lane] = -v[2 + i];
        }
      }
      if (tail) {
        if (!wait_all(bTail, (uint32_t)tails & 1u, abort_flag, p.a.status)) { ok = false; break; }
        ++tails;
        clear_rows<HD>(tile, SMALL, there, lane);
        clear_rows<HD>(tile + C::kSmall, SMALL, there, lane);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bFull(s));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bFull(s));
    }
  } else if (warp == 1) {
    const bool leader = elect_one();
    const int steps = (p.a.head_dim + 15) / 16;  // of the contractions over channels (the channels behind are zeros)
    const uint64_t dB0 = make_desc(sBig0, 16, 1024), dB1 = make_desc(sBig1, 16, 1024);
    const uint64_t dS0 = make_desc(sSmall, 16, 1024), dS1 = make_desc(sSmall + C::kSmall, 16, 1024);
    const uint64_t dS0mn = make_desc(sSmall, SMALL * 128, 1024), dS1mn = make_desc(sSmall + C::kSmall, SMALL * 128, 1024);
    // Both contract over channels.
    auto scores = [&](int it) {
      const uint32_t off = (uint32_t)(it % NS) * C::kStage, t = tmem + 128 * (it % NB);
      if (leader) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
          if (HD == 64 || k < steps) tc_mma(t, desc_add(dB0, (k / 4) * BIG * 128 + 32 * (k % 4)), desc_add(dS0, off + (k / 4) * SMALL * 128 + 32 * (k % 4)), kIdesc<SMALL, 0>, k != 0);
        if (kDKV) mbar_arrive(bScores(it % NB));
        tc_commit(bScores(it % NB));
      }
    };
    auto dp_scores = [&](int it) {
      const uint32_t off = (uint32_t)(it % NS) * C::kStage, t = tmem + 128 * (it % NB) + 64;
      if (leader) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
          if (HD == 64 || k < steps) tc_mma(t, desc_add(dB1, (k / 4) * BIG * 128 + 32 * (k % 4)), desc_add(dS1, off + (k / 4) * SMALL * 128 + 32 * (k % 4)), kIdesc<SMALL, 0>, k != 0);
        tc_commit(bDP(it % NB));
      }
    };
    bool ok = n_it == 0 || wait_all(bBig, 0, abort_flag, p.a.status);
    for (int it = 0; it < NB && it < n_it && ok; ++it) {
      ok = wait_all(bFull(it % NS), 0, abort_flag, p.a.status);
      tc_fence_after();
      if (ok) {
        scores(it);
        dp_scores(it);
      }
    }
    // A tile's two halves follow one another: the product with the probabilities, and the scores that take over their columns, run while the
    // softmax warps form dS.  (Products run in order.)
    for (int it = 0; it < n_it && ok; ++it) {
      const uint32_t off = (uint32_t)(it % NS) * C::kStage, t = tmem + 128 * (it % NB), parity = (uint32_t)(it / NB) & 1u;
      if (!wait_all(bProbs(it % NB), parity, abort_flag, p.a.status)) { ok = false; break; }
      tc_fence_after();
      if (kDKV && leader) {
#pragma unroll
        for (int k = 0; k < SMALL / 16; ++k)  // dV += P^T dO: contraction over the tile's rows
          tc_mma_ts(tAcc1, t + (k / 2) * 32 + (k % 2) * 8, desc_add(dS1mn, off + 2048 * k), kIdesc<HD, 1>, (it | k) != 0);
      }
      if (NB == 1 && it + NB < n_it) {
        if (!wait_all(bFull((it + NB) % NS), (uint32_t)((it + NB) / NS) & 1u, abort_flag, p.a.status)) { ok = false; break; }
        tc_fence_after();
        scores(it + NB);
      }
      if (!wait_all(bDS(it % NB), parity, abort_flag, p.a.status)) { ok = false; break; }
      tc_fence_after();
      if (leader) {
#pragma unroll
        for (int k = 0; k < SMALL / 16; ++k)  // dK += dS^T Q, dQ += dS K
          tc_mma_ts(tAcc0, t + 64 + (k / 2) * 32 + (k % 2) * 8, desc_add(dS0mn, off + 2048 * k), kIdesc<HD, 1>, (it | k) != 0);
        tc_commit(bFree(it % NS));
      }
      if (it + NB < n_it) {
        if (NB > 1) {
          if (!wait_all(bFull((it + NB) % NS), (uint32_t)((it + NB) / NS) & 1u, abort_flag, p.a.status)) { ok = false; break; }
          tc_fence_after();
          scores(it + NB);
        }
        dp_scores(it + NB);
      }
    }
    if (leader) tc_commit(bDone);
  } else {
    const int group_id = (warp - 2) >> 3, ch = ((warp - 2) >> 2) & 1;  // which tiles, and which 32 of their rows (columns of the scores) this warp has
    const int quarter = warp & 3, row = quarter * 32 + lane, brow = big0 + row;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const float scale2 = p.a.scale * LOG2E;
    float my_lse = -INFINITY, my_d = 0.0f;  // dQ: minus log-sum-exp and minus D of this row
    chain_wait();
    if (!kDKV && brow < n_big) {
      const int64_t at = (int64_t)w.h * p.a.q_rows + sq.q0 + brow;
      my_lse = p.lse[at] == -INFINITY ? -INFINITY : p.lse[at] * -LOG2E;
      my_d = -p.drow[at];
    }
    bool ok = true;
    int at_tile = 0;
    for (int it = group_id; it < n_it; it += C::kGroups) {
      const uint32_t parity = (uint32_t)(it / NB) & 1u;
      if (!wait_all(bScores(it % NB), parity, abort_flag, p.a.status)) { ok = false; break; }
      tc_fence_after();
      at_tile += it == group_id ? rank + group_id * ranks : C::kGroups * ranks;
      while (kDKV && at_tile >= tiles) at_tile -= tiles;
      const int c0 = (t_beg + at_tile) * SMALL;
      const uint32_t t = tmem + lanes + 128 * (it % NB) + ch * 32;
      const ulonglong2* st = reinterpret_cast<const ulonglong2*>(stats + (it % NS) * 2 * SMALL + ch * 32);  // (dK, dV: of four columns each)
      // does every row of the block see (is every row of the block seen by) the whole tile?
      const bool full = kDKV ? (!p.a.causal || big0 + BIG - 1 <= c0 + shift) : (c0 + SMALL <= sq.nk && (!p.a.causal || c0 + SMALL - 1 <= big0 + shift));
      float sc[32];
      tc_ld32(t, sc);
      if (!kDKV) {  // the scores' columns are free
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bProbs(it % NB));
      }
#pragma unroll
      for (int c = 0; c < 32; c += 4) {
        const ulonglong2 l = kDKV ? st[c / 4] : make_ulonglong2(both(my_lse), both(my_lse));
        const float2 x = floats_of(fma2(pair_of(sc[c], sc[c + 1]), both(scale2), l.x)), y = floats_of(fma2(pair_of(sc[c + 2], sc[c + 3]), both(scale2), l.y));
        sc[c] = fast_exp2(x.x);
        sc[c + 1] = fast_exp2(x.y);
        sc[c + 2] = fast_exp2(y.x);
        sc[c + 3] = fast_exp2(y.y);
      }
      uint32_t seen = 0xffffffffu;  // of this row's 32 columns
      if (!full) {
        // dK, dV: a column is a query, the row a key, seen from query brow - shift on; dQ: a column is a key
        const int first = c0 + ch * 32, from = kDKV ? brow - shift - first : 0, to = kDKV ? 32 : min(brow + shift, sq.nk - 1) + 1 - first;
        seen = from >= 32 || to <= 0 ? 0u : (0xffffffffu << max(from, 0)) & (to >= 32 ? 0xffffffffu : (1u << to) - 1u);
#pragma unroll
        for (int c = 0; c < 32; ++c) sc[c] = (seen >> c) & 1u ? sc[c] : 0.0f;
      }
      uint32_t packed[16];
      if (kDKV) {
#pragma unroll
        for (int i = 0; i < 16; ++i) packed[i] = pack2(sc[2 * i], sc[2 * i + 1]);
        tc_st16(t, packed);
        tc_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bProbs(it % NB));
      }
      if (!wait_all(bDP(it % NB), parity, abort_flag, p.a.status)) { ok = false; break; }
      tc_fence_after();
      float dp[32];
      tc_ld32(t + 64, dp);
#pragma unroll
      for (int c = 0; c < 32; c += 4) {
        const ulonglong2 d = kDKV ? st[SMALL / 4 + c / 4] : make_ulonglong2(both(my_d), both(my_d));
        const float2 x = floats_of(mul2(add2(pair_of(dp[c], dp[c + 1]), d.x), pair_of(sc[c], sc[c + 1])));
        const float2 y = floats_of(mul2(add2(pair_of(dp[c + 2], dp[c + 3]), d.y), pair_of(sc[c + 2], sc[c + 3])));
        dp[c] = x.x;
        dp[c + 1] = x.y;
        dp[c + 2] = y.x;
        dp[c + 3] = y.y;
      }
      if (!full) {  // (a dP that is not finite times a probability of 0)
#pragma unroll
        for (int c = 0; c < 32; ++c) dp[c] = (seen >> c) & 1u ? dp[c] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) packed[i] = pack2(dp[2 * i], dp[2 * i + 1]);
      tc_st16(t + 64, packed);
      tc_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bDS(it % NB));
    }
    ok = ok && wait_all(bDone, 0, abort_flag, p.a.status);
    if (ok && !kShared) {  // accumulators -> bf16 -> shared memory (the block's own tiles are free) -> rows
      tc_fence_after();
      const int at = (2 * group_id + ch) * 32;  // the first of this warp's 32 channels
#pragma unroll 1
      for (int o = 0; o < (kDKV ? 2 : 1) && at < HD; ++o) {
        const uint32_t tile = o == 0 ? sBig0 : sBig1;
        const float mul = o == 0 ? p.a.scale : 1.0f;  // dK and dQ carry the scores' scale
        float v[32];
        if (n_it > 0) tc_ld32((o == 0 ? tAcc0 : tAcc1) + lanes + at, v);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = n_it > 0 ? v[i] * mul : 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u) st_shared16(swz(tile + (at / SUB) * BIG * 128, row, (at % SUB) / 8 + u), pack8(v + 8 * u));
        __syncwarp();
        const hbp_heads& out = kDKV ? (o == 0 ? p.dk : p.dv) : p.dq;
        store_staged<4>(tile, quarter * 32, at / 8, (bf16*)out.x + ((kDKV ? sq.k0 : sq.q0) + big0) * out.row_stride + w.h * out.head_stride,
                                out.row_stride, n_big - big0, p.a.head_dim, lane);
      }
    } else if (ok) {
      tc_fence_after();
      const int at = (2 * group_id + ch) * 32;
      if (at < HD) {
        leave_sums<HD>(sBig0, n_it > 0, tAcc0 + lanes, row, at, at + 32);
        if (kDKV) leave_sums<HD>(sSmall, n_it > 0, tAcc1 + lanes, row, at, at + 32);
      }
    }
  }
  // (before the blocks of a cluster wait for one another, as above)
  leave(warp, tmem, C::kColumns, abort_flag);
  if (kShared) {
    // the sums of dK and dQ in the place of the block's own tiles, those of dV in the place of the others
    cluster_sync();
    const int first = big0 + rank * (BIG / ranks);
    auto put = [&](const hbp_heads& out, float mul) {
      return [&, mul](int r, int u, float (&v)[8]) {
        if (u * 8 >= p.a.head_dim) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= mul;
        *reinterpret_cast<uint4*>((bf16*)out.x + ((kDKV ? sq.k0 : sq.q0) + first + r) * out.row_stride + w.h * out.head_stride + u * 8) = pack8(v);
      };
    };
    auto all = [](int, int) { return 1.0f; };
    merge_sums<HD>(ranks, sBig0, rank, n_big - first, (int)threadIdx.x, C::kThreads, all, put(kDKV ? p.dk : p.dq, p.a.scale));
    if (kDKV) merge_sums<HD>(ranks, sSmall, rank, n_big - first, (int)threadIdx.x, C::kThreads, all, put(p.dv, 1.0f));
    cluster_sync();  // (no block ends while another reads its shared memory)
  }
}

// kShared: walks are shared by clusters of `ranks` blocks.  The first `first` walks are those of one kind, the longer ones: 4 x 1 query, 4096 keys, 16 query
// heads on 4 of 128: dQ first 74 us, dK and dV first 94.
template <int HD, bool kShared>
__global__ void __launch_bounds__(Bwd<HD>::kThreads, Bwd<HD>::kBlocksAnSm)
ragged_bwd_tc_kernel(const __grid_constant__ RaggedMaps m, const __grid_constant__ RaggedAttn p, const unsigned first, const bool kv_first,
                     const int ranks) {
  // What the launch before leaves is D, waited for where it is read; that launch began when everything before it was over.  Without queries (the
  // longest sequence of them has none, whatever rows the tensors have) there is no such launch, and the offsets may still be on their way.
  if (p.a.q_len == 0) chain_wait();
  const unsigned i = kShared ? blockIdx.x >> (__ffs(ranks) - 1) : blockIdx.x;
  const int rank = kShared ? (int)(blockIdx.x & (unsigned)(ranks - 1)) : 0;  // (a power of two of them)
  const unsigned nth = i < first ? i : i - first;
  if ((i < first) == kv_first) ragged_bwd_body<HD, true, kShared>(m, p, block_at(nth, p.kv_walks, false), rank, ranks);
  else ragged_bwd_body<HD, false, kShared>(m, p, block_at(nth, p.q_walks, true), rank, ranks);
}

// Map {channel, head, row} of a [rows][heads][head_dim] tensor: boxes of 64 channels.
bool map_heads(CUtensorMap* tm, const hbp_heads& t, int64_t rows, int heads, int head_dim, int box_heads = 1, int box_rows = SMALL) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  // (the stride of a dimension of one element is never used, but is checked all the same)
  const int64_t hs = heads > 1 ? t.head_stride : head_dim, rs = rows > 1 ? t.row_stride : head_dim;
  cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)rows};
  cuuint64_t strides[2] = {(cuuint64_t)hs * 2, (cuuint64_t)rs * 2};
  cuuint32_t box[3] = {SUB, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, estr[3] = {1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, t.x, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Blocks that share each of `walks` walks of up to `tiles` tiles: twice as many for as long as blocks are fewer than the chip takes at a time
// and every block has kLeast tiles.  Shared against one block a walk: 4 x 1 query, 4096 keys, 16 heads of 128, forward 25 against 49 us; 128 queries, 4096 keys, 4 heads on one of
// 128, 19 against 47 and backward 31 against 58; 4096 queries, 77 keys, 4 heads of 64, backward 43 against 72; 2048 rows, 2 heads of 64, 15 against 27 and
// 25 against 39.  With four tiles a block instead of eight, 512 rows of 8 heads of 128 take 14.5 us forward instead of 12.4 and 18.2 instead of 16.5 backward; 1024 rows
// of 4 heads 14.5 instead of 18.6.
constexpr int kLeast = 8;
int ranks_of(int64_t walks, int64_t at_a_time, int64_t tiles) {
  int r = 1;
  while (r < MOST_RANKS && 2 * walks * r <= at_a_time && 2 * r * kLeast <= tiles) r *= 2;
  return r;
}
// Forward: the query heads of a key head whose rows, of all its queries, are one tile's at most become the rows of one block, which reads the keys
// and values once for all, where that makes the launch fit the chip at once or lets more blocks share a walk.  Packed against a block a head: 32 x 1 query, 1000 keys,
// 32 heads on 4 of 128, 18.6 against 76 us; 16 x 1, 4096 keys, 16 on 4 of 128, 27 (4.9 TB/s) against 66; 8 x 4, 2048 keys, 12 on 4 of 64, 12 against 19.5; where neither
// holds, 1 x 1, 300 keys, 4 on one of 64, 8.1 against 7.0.
int packed_heads(const hbp_attention& a) {
  const int group = a.q_heads / a.kv_heads;
  if ((int64_t)a.q_len * group > SMALL) return 1;
  const int64_t alone = blocks_of(a.q_len, BIG, a.q_heads, a.sequences), tiles = (a.kv_len + SMALL - 1) / SMALL;
  return alone > 2 * 148 || ranks_of(alone / group, 2 * 148, tiles) > ranks_of(alone, 2 * 148, tiles) ? group : 1;
}
template <typename... P, typename... A>
void launch_clusters(Launcher& lc, void (*kernel)(P...), int64_t blocks, int threads, size_t smem, int ranks, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = lc.stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = ranks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = ranks > 1 ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
  if (e != cudaSuccess && lc.err == cudaSuccess) lc.err = e;
  lc.count();
  lc.check();
}

template <typename K>
bool allow_smem(K kernel, int bytes, bool& done) {
  if (!done) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
      cudaGetLastError();
      return false;
    }
    done = true;
  }
  return true;
}

template <int HD>
bool forward(Launcher& lc, const RaggedAttn& given, const RaggedMaps& m) {
  static PerDevice<bool> set, set_shared, set_packed;
  if (!allow_smem(ragged_fwd_tc_kernel<HD, false, false>, Fwd<HD>::kSmem, set.here()) ||
      !allow_smem(ragged_fwd_tc_kernel<HD, true, false>, Fwd<HD>::kSmem, set_shared.here()) ||
      !allow_smem(ragged_fwd_tc_kernel<HD, true, true>, Fwd<HD>::kSmem, set_packed.here()))
    return false;
  const int pack = packed_heads(given.a);
  RaggedAttn r = with_walks(given, BIG, pack);
  const int64_t walks = blocks_of(r.a.q_len, BIG, r.a.q_heads / pack, r.a.sequences);
  const int ranks = ranks_of(walks, 2 * 148, (r.a.kv_len + SMALL - 1) / SMALL);
  const auto kernel = pack > 1 ? ragged_fwd_tc_kernel<HD, true, true> : ranks > 1 ? ragged_fwd_tc_kernel<HD, true, false> : ragged_fwd_tc_kernel<HD, false, false>;
  r.pass_blocks = (uint32_t)(walks * ranks);
  launch_clusters(lc, kernel, walks * ranks + (r.a.fresh ? kClearers : 0), FWD_THREADS, Fwd<HD>::kSmem, ranks, m, r, ranks, pack);
  return true;
}

template <int HD>
bool backward(Launcher& lc, const RaggedAttn& given, const RaggedMaps& m) {
  using C = Bwd<HD>;
  const RaggedAttn r = with_walks(given, BIG);
  static PerDevice<bool> set, set_shared;
  if (!allow_smem(ragged_bwd_tc_kernel<HD, false>, C::kSmem, set.here()) || !allow_smem(ragged_bwd_tc_kernel<HD, true>, C::kSmem, set_shared.here())) return false;
  const int64_t kv = blocks_of(r.a.kv_len, BIG, r.a.kv_heads, r.a.sequences), q = blocks_of(r.a.q_len, BIG, r.a.q_heads, r.a.sequences);
  const int64_t q_tiles = (r.a.q_len + SMALL - 1) / SMALL * (int64_t)(r.a.q_heads / r.a.kv_heads), kv_tiles = (r.a.kv_len + SMALL - 1) / SMALL;
  const int ranks = ranks_of(kv + q, C::kBlocksAnSm * 148, q_tiles > kv_tiles ? q_tiles : kv_tiles);
  const bool kv_first = q_tiles >= kv_tiles;  // the long walks before the short ones
  launch_chained(lc, ranks > 1 ? ragged_bwd_tc_kernel<HD, true> : ragged_bwd_tc_kernel<HD, false>, dim3((unsigned)((kv + q) * ranks)), C::kThreads, C::kSmem, ranks,
                 m, r, (unsigned)(kv_first ? kv : q), kv_first, ranks);
  return true;
}

// A side without rows has no tensors: its maps are never used.
bool maps(const RaggedAttn& r, bool back, RaggedMaps& m) {
  const hbp_attention& a = r.a;
  const int pack = back ? 1 : packed_heads(a);
  if (a.q_len && !map_heads(&m.q, r.q, a.q_rows, a.q_heads, a.head_dim, pack, pack > 1 ? a.q_len : SMALL)) return false;
  if (a.q_len && back && !map_heads(&m.d_o, r.d_o, a.q_rows, a.q_heads, a.head_dim)) return false;
  return !a.kv_len || (map_heads(&m.k, r.k, a.kv_rows, a.kv_heads, a.head_dim) && map_heads(&m.v, r.v, a.kv_rows, a.kv_heads, a.head_dim));
}

}  // namespace

bool ragged_forward_tc(Launcher& lc, const RaggedAttn& r) {
  RaggedMaps m = {};
  if (!maps(r, false, m)) return false;
  return r.a.head_dim <= 64 ? forward<64>(lc, r, m) : forward<128>(lc, r, m);
}

bool ragged_backward_tc(Launcher& lc, const RaggedAttn& r) {
  RaggedMaps m = {};
  if (!maps(r, true, m)) return false;
  return r.a.head_dim <= 64 ? backward<64>(lc, r, m) : backward<128>(lc, r, m);
}

}  // namespace hbp
