// Softmax cross entropy of hidden states x [rows][d] against a vocabulary matrix w [vocab][d] (hbp_cross_entropy), and with its
// gradients (hbp_cross_entropy_gradients).  z = x w^T is not in memory with bf16 data, whose gradients keep a number of 2 bytes a logit instead; float logits are, of a
// piece of the rows.
//
// With t a row's target and r a number near its largest logit, e_j = exp(z_j - r):
//   S' = sum over j != t of e_j,   S = S' + e_t,   loss = log(S) - (z_t - r),   dz_j = g e_j / S (j != t),   dz_t = -g S' / S
// so that neither a small loss nor its gradient is a difference of like numbers.  Taking r = z_t, which a dot product a row gives
// beforehand, makes e_t = 1 and loss = log1p(S').
//
// bf16, three products of 2 rows vocab d flop instead of the four of a backward pass that forms the logits again:
//   1. target_kernel   z_t by a warp a row
//   2. gemm_tc, EPI_EXP: e rounded to bf16 into E [rows][vocab] (0 at the target), in float each row's sums and its largest logit
//   3. finish_kernel   S', loss, the row's factor s = g / S; E at the target becomes -S'; s x, rounded to bf16
//   4. gemm_tc, EPI_ROWS: dx = s (E w)          5. gemm_tc: dw = E^T (s x)
// s is a number a row, which is why E needs no second pass: it comes out of the sum over the vocabulary in 4, and goes into the other
// operand in 5.  E and s x are rounded to bf16, the operands' type: 2^-8 of each of their values at most, as a rounding of dz would be.  A row whose largest logit is more than
// kFar above the target's (a loss of 40) would leave the range that bf16 and float sums of e have: finish_kernel then takes r = the largest logit,
// and 2 and 3 run again; their launches return at once where no row asked for that.
// The forward pass alone has no E: the product sums exp(z - its largest) without z_t, and loss_kernel joins what its tiles have.
//
// float: products of operands in three bf16 parts (gemm_parts.cu); the logits of a piece of the rows lie in scratch, and
// one pass over them forms dz, in parts.  Few rows take w as it is, in float: what bounds them is its bytes, and in parts it is 16 a value to write and read instead of 4.
//
// E has a piece of the rows at a time where it would be more than kPieceBytes, or than the scratch that the caller has.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "float_pairs.cuh"
#include "float_parts.cuh"
#include "tc_common.cuh"

namespace hbp {

namespace {

constexpr float kFar = 40.0f;
constexpr size_t kPieceBytes = (size_t)4 << 30;
constexpr int kPairs = 74;  // of CTAs, that a B200 runs at a time

struct Targets {
  const void* t;
  int bytes;
  __device__ __forceinline__ int64_t operator[](int64_t i) const { return bytes == 8 ? ((const int64_t*)t)[i] : (int64_t)((const int32_t*)t)[i]; }
  // the column, -1 for a row that is ignored
  __device__ __forceinline__ int column(int64_t i, int vocab, int* status) const {
    const int64_t v = (*this)[i];
    if (v >= vocab && status) *status = (int)HBP_ERR_INVALID_ARG;
    return v < 0 || v >= vocab ? -1 : (int)v;
  }
};

// ------------------------------------------------------------------------------------------- bf16
struct RowData {
  int64_t rows;
  int vocab, d;
  const bf16* x;
  int64_t ldx;
  const bf16* w;
  int64_t ldw;
  Targets targets;
  int* status;
  int* target;  // [rows]
  float *zt, *ref, *factor;
  float2* parts;  // [slots][rows]
  int slots;
  int* redo;
  bool again;  // the second time, for rows whose reference was too low
  const float* d_loss;
  int64_t d_loss_stride;
  float* loss;
  bf16* E;
  int64_t ldE;
  bf16* xs;
};

// A row's logit of its target t >= 0, by a warp: a float dot product.  (The tensor core's sum is truncated, and would take ten times the error to a loss.)
__device__ __forceinline__ float target_logit(const RowData& p, int64_t row, int t) {
  const int lane = threadIdx.x & 31;
  const bf16 *x = p.x + row * p.ldx, *w = p.w + (int64_t)t * p.ldw;
  float z = 0.0f;
#pragma unroll 4
  for (int c = lane * 8; c < p.d; c += 256) {
    float a[8], b[8];
    tc::unpack8(*reinterpret_cast<const uint4*>(x + c), a);
    tc::unpack8(*reinterpret_cast<const uint4*>(w + c), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) z = fmaf(a[e], b[e], z);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
  return z;
}

__global__ void __launch_bounds__(256) target_kernel(const RowData p) {
  chain_next();
  chain_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.redo = 0;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  const int t = p.targets.column(row, p.vocab, p.status);
  const float z = t >= 0 ? target_logit(p, row, t) : 0.0f;
  if (lane == 0) {
    p.target[row] = t;
    p.zt[row] = z;
    p.ref[row] = isfinite(z) ? z : 0.0f;
  }
}

constexpr int kFinishWarps = 16;
// Rows a block: a quarter of a warp has a slot of all of them at a time.  (With 32 the 16 rows of a short call are one block's, 10 us instead of 4; 8192 rows take 29 us and 31.)
constexpr int kFinishRows = 8, kSlotStep = kFinishWarps * 32 / kFinishRows;

__global__ void __launch_bounds__(32 * kFinishWarps) finish_kernel(const RowData p) {
  __shared__ float sums[kFinishWarps][kFinishRows], mosts[kFinishWarps][kFinishRows], factors[kFinishRows];
  chain_next();
  chain_wait();
  if (p.again && *(const volatile int*)p.redo == 0) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_block = lane % kFinishRows;
  const int64_t row0 = (int64_t)blockIdx.x * kFinishRows, row = row0 + in_block;
  float sum = 0.0f, most = -INFINITY;
  if (row < p.rows) {
#pragma unroll 8
    for (int k = threadIdx.x / kFinishRows; k < p.slots; k += kSlotStep) {
      const float2 v = p.parts[(int64_t)k * p.rows + row];
      sum += v.x;
      most = fmaxf(most, v.y);
    }
  }
#pragma unroll
  for (int o = kFinishRows; o < 32; o <<= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  }
  if (lane < kFinishRows) {
    sums[warp][lane] = sum;
    mosts[warp][lane] = most;
  }
  __syncthreads();
  if (threadIdx.x < kFinishRows) {
#pragma unroll
    for (int k = 1; k < kFinishWarps; ++k) {
      sum += sums[k][lane];
      most = fmaxf(most, mosts[k][lane]);
    }
    float factor = 0.0f;
    if (row < p.rows) {
      const int t = p.target[row];
      const float zt = p.zt[row], ref = p.ref[row];
      float loss = 0.0f;
      if (t >= 0) {
        if (!p.again && most - ref > kFar) {
          p.ref[row] = most;
          *p.redo = 1;
        }
        const bool at_target = zt == ref;
        const float total = sum + (at_target ? 1.0f : expf(zt - ref));
        loss = at_target ? log1pf(sum) : logf(total) - (zt - ref);
        factor = (p.d_loss ? p.d_loss[row * p.d_loss_stride] : 1.0f) / total;
        const bf16 e = __float2bfloat16_rn(-sum);
        p.E[row * p.ldE + t] = e;
        // the largest term of most rows' gradients, with its rounding taken out again: the others share it, as large as their own
        const float kept = __bfloat162float(e);
        if (sum > 0.0f && isfinite(kept)) factor *= sum / -kept;
      }
      p.loss[row] = loss;
      p.factor[row] = factor;
    }
    factors[lane] = factor;
  }
  if (!p.xs) return;
  __syncthreads();
  const int per_row = p.d / 8;
  const int64_t left = p.rows - row0;
  const int n = (int)(left < kFinishRows ? left : kFinishRows) * per_row;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 32 * kFinishWarps) {
    const int r = i / per_row, c = (i - r * per_row) * 8;
    float f[8];
    tc::unpack8(*reinterpret_cast<const uint4*>(p.x + (row0 + r) * p.ldx + c), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = factors[r] != 0.0f ? f[e] * factors[r] : 0.0f;  // (a row that is ignored may hold anything)
    *reinterpret_cast<uint4*>(p.xs + (row0 + r) * p.d + c) = tc::pack8(f);
  }
}

// The forward pass alone: sums of exp(z - largest) of the tiles, joined the same way.
__global__ void __launch_bounds__(32 * kFinishWarps) loss_kernel(const RowData p) {
  __shared__ float2 joined[kFinishWarps][kFinishRows];
  __shared__ float logits[kFinishRows];
  chain_next();
  chain_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row0 = (int64_t)blockIdx.x * kFinishRows, row = row0 + lane % kFinishRows;
  if (warp < kFinishRows) {
    const int t = row0 + warp < p.rows ? p.targets.column(row0 + warp, p.vocab, p.status) : -1;
    const float z = t >= 0 ? target_logit(p, row0 + warp, t) : 0.0f;
    if (lane == 0) logits[warp] = z;
  }
  float2 s = make_float2(0.0f, -INFINITY);
  // several sums at a time: their exponentials wait for one maximum, not for each other
  auto join = [&](auto& v, auto count) {
    constexpr int n = decltype(count)::value;
    float top = s.y;
#pragma unroll
    for (int i = 0; i < n; ++i) top = fmaxf(top, v[i].y);
    const float ref = top == -INFINITY ? 0.0f : top;
    s.x *= __expf(s.y - ref);
#pragma unroll
    for (int i = 0; i < n; ++i) s.x = fmaf(v[i].x, __expf(v[i].y - ref), s.x);
    s.y = top;
  };
  const float2 empty = make_float2(0.0f, -INFINITY);
  for (int k = threadIdx.x / kFinishRows; k < p.slots; k += 8 * kSlotStep) {
    float2 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int slot = k + i * kSlotStep;
      v[i] = row < p.rows && slot < p.slots ? p.parts[(int64_t)slot * p.rows + row] : empty;
    }
    join(v, std::integral_constant<int, 8>());
  }
#pragma unroll
  for (int o = kFinishRows; o < 32; o <<= 1) {
    const float2 v[1] = {make_float2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o))};
    join(v, std::integral_constant<int, 1>());
  }
  if (lane < kFinishRows) joined[warp][lane] = s;
  __syncthreads();
  if (threadIdx.x >= kFinishRows || row >= p.rows) return;
  s = empty;
  float2 v[kFinishWarps];
#pragma unroll
  for (int k = 0; k < kFinishWarps; ++k) v[k] = joined[k][lane];
  join(v, std::integral_constant<int, kFinishWarps>());
  float loss = 0.0f;
  if (p.targets.column(row, p.vocab, nullptr) >= 0) {
    const float zt = logits[lane], above = s.y - zt;
    if (zt == INFINITY) loss = NAN;
    else if (above <= kFar) loss = log1pf(s.x * expf(above));
    else loss = logf(s.x + expf(-above)) + above;
  }
  p.loss[row] = loss;
}

// out (rows ld apart, bf16) = factor[row] * the sum of `splits` [rows][d], in their order; eight channels a thread
__global__ void __launch_bounds__(256) narrow_kernel(const float* in, int splits, const float* factor, bf16* out, int64_t ld, int64_t rows, int d) {
  chain_next();
  chain_wait();
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, n = rows * d;
  if (i >= n) return;
  float f[8] = {};
#pragma unroll 8
  for (int k = 0; k < splits; ++k) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(in + k * n + i)), b = __ldcs(reinterpret_cast<const float4*>(in + k * n + i + 4));
    f[0] += a.x; f[1] += a.y; f[2] += a.z; f[3] += a.w;
    f[4] += b.x; f[5] += b.y; f[6] += b.z; f[7] += b.w;
  }
  const int64_t row = i / d;
  if (factor) {
    const float s = factor[row];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = s != 0.0f ? f[e] * s : 0.0f;
  }
  *reinterpret_cast<uint4*>(out + row * ld + (i - row * d)) = tc::pack8(f);
}

// ------------------------------------------------------------------------------------------- float
// rows of src, ld apart -> planes; zeros for those behind the last, and for rows without a target (they may hold anything), where targets are given
__global__ void __launch_bounds__(256) split_rows_kernel(const float* src, int64_t ld, Planes dst, int64_t rows, int64_t all, int d, Targets targets, int vocab) {
  chain_next();
  chain_wait();
  const int per_row = d / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
  if (row >= all) return;
  const int c = (int)(i - row * per_row) * 4;
  const bool there = row < rows && (!targets.t || targets.column(row, vocab, nullptr) >= 0);
  store_parts4(dst.p + row * dst.ld + c, dst.plane, there ? *reinterpret_cast<const float4*>(src + row * ld + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f));
}

// out (rows ld apart) = the sum of `splits` [rows][d], in their order; four channels a thread
__global__ void __launch_bounds__(256) sum_splits_kernel(const float* in, int splits, float* out, int64_t ld, int64_t rows, int d) {
  chain_next();
  chain_wait();
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, n = rows * d;
  if (i >= n) return;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int k = 0; k < splits; ++k) {
    const float4 v = __ldcs(reinterpret_cast<const float4*>(in + k * n + i));
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  const int64_t row = i / d;
  *reinterpret_cast<float4*>(out + row * ld + (i - row * d)) = s;
}

__device__ __forceinline__ int cluster_blocks() {
  uint32_t n;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return (int)n;
}
__device__ __forceinline__ int cluster_block() {
  uint32_t n;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(n));
  return (int)n;
}
__device__ __forceinline__ float2 cluster_load(const float2* p, int block) {
  const uint32_t at = tc::map_to_cta((uint32_t)__cvta_generic_to_shared(p), block);
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}

struct LogitsData {
  const float* z;  // [rows][ldz], ldz a multiple of 4
  int64_t ldz;
  int vocab, columns;  // of dz: zeros behind the vocabulary
  Targets targets;
  int* status;
  const float* d_loss;
  int64_t d_loss_stride;
  float* loss;
  Planes dz;         // not of the forward pass alone: in parts,
  float* dz_f;       // or as floats in the logits' place
};

constexpr int kRowThreads = 512;

// A block a row, or a cluster of up to eight where there are few rows; each reads its columns once for the sum (twice where the target is far from the largest logit),
// and once more for dz.  Instructions bound it, expf half of them; a row's exponentials held in registers in between took as long (1901 rows of 8111: 44 us, 49; 94
// where a thread holds 64).
template <bool kClusters>
__global__ void __launch_bounds__(kRowThreads) logits_kernel(const LogitsData p) {
  __shared__ float sums[kRowThreads / 32], mosts[kRowThreads / 32];
  __shared__ float2 blocks[2];
  chain_next();
  chain_wait();
  const int shares = kClusters ? cluster_blocks() : 1, share = kClusters ? cluster_block() : 0;
  const int64_t row = blockIdx.x / shares;
  const float* z = p.z + row * p.ldz;
  const bool first = threadIdx.x == 0 && share == 0;
  const int t = p.targets.column(row, p.vocab, first ? p.status : nullptr), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int from = (share * kRowThreads + (int)threadIdx.x) * 4, step = shares * kRowThreads * 4;
  const float zt = t >= 0 ? z[t] : 0.0f;
  float ref = isfinite(zt) ? zt : 0.0f, sum = 0.0f, most = -INFINITY;
  if (t >= 0) {
    for (int again = 0; again < 2; ++again) {
      sum = 0.0f;
#pragma unroll 4
      for (int c = from; c < p.vocab; c += step) {
        const float4 q = *reinterpret_cast<const float4*>(z + c);
        const float v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < p.vocab && c + e != t) {
            most = fmaxf(most, v[e]);
            sum += expf(v[e] - ref);
          }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      }
      __syncthreads();
      if (lane == 0) {
        sums[warp] = sum;
        mosts[warp] = most;
      }
      __syncthreads();
      sum = 0.0f;
      for (int k = 0; k < kRowThreads / 32; ++k) {
        sum += sums[k];
        most = fmaxf(most, mosts[k]);
      }
      if (kClusters) {  // (a place a turn: nobody waits for the others to have read)
        if (threadIdx.x == 0) blocks[again] = make_float2(sum, most);
        tc::cluster_sync();
        sum = 0.0f;
        for (int k = 0; k < shares; ++k) {
          const float2 q = cluster_load(&blocks[again], k);
          sum += q.x;
          most = fmaxf(most, q.y);
        }
      }
      if (!(most - ref > kFar)) break;
      ref = most;
    }
    if (kClusters) tc::cluster_sync();  // (the others read this block's; and the target's logit may be written over)
  }
  const bool at_target = zt == ref;
  const float total = sum + (at_target ? 1.0f : expf(zt - ref));
  if (first) p.loss[row] = t < 0 ? 0.0f : at_target ? log1pf(sum) : logf(total) - (zt - ref);
  if (!p.dz.p && !p.dz_f) return;
  const float factor = t < 0 ? 0.0f : (p.d_loss ? p.d_loss[row * p.d_loss_stride] : 1.0f) / total;
  for (int c = from; c < p.columns; c += step) {
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (factor != 0.0f && c < p.vocab) {
      const float4 q = *reinterpret_cast<const float4*>(z + c);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = c + e >= p.vocab ? 0.0f : factor * (c + e == t ? -sum : expf(v[e] - ref));
    }
    const float4 dz = make_float4(v[0], v[1], v[2], v[3]);
    if (p.dz_f) *reinterpret_cast<float4*>(p.dz_f + row * p.ldz + c) = dz;
    else store_parts4(p.dz.p + row * p.dz.ld + c, p.dz.plane, dz);
  }
}

// How many blocks a row, so that few rows fill the GPU: two an SM, of one turn of its threads at least.
int logit_shares(int64_t rows, int vocab) {
  int n = 1;
  while (n < 8 && rows * 2 * n <= 4 * kPairs && (int64_t)2 * n * kRowThreads * 4 <= vocab) n *= 2;
  return n;
}

// ------------------------------------------------------------------------------------------- float, few rows
constexpr int kFewAtOnce = 16, kFewTile = 64;  // rows of x, rows of w
constexpr int kFewSteps = 32, kFewPitch = kFewSteps + 4, kFewStages = 3, kFewThreads = 256;

__device__ __forceinline__ void copy_or_zero(float* to, const float* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_made() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
struct alignas(16) Pairs2 {
  f32x2 a, b;
};

// z [rows][ldz]: 16 x 64 of it a block of two warps, 4 x 4 a thread, the sums of even and odd channels and of each 32 apart (8 + d / 64 units of 2^-23 at most); 32 channels at a time by asynchronous copies, two steps
// ahead.  Rows of shared memory are 36 floats apart: the eight rows of w that a warp reads at once lie in different banks.  (16 rows of 131072 x 2048: 259 us with
// all of the loss, of 163 for w's bytes; w straight into registers, a row a warp, 696.)
__global__ void __launch_bounds__(64) few_logits_kernel(const float* x, int64_t ldx, int rows, const float* w, int64_t ldw, int vocab, int d, float* z, int64_t ldz) {
  constexpr int kRows = kFewTile + kFewAtOnce;
  __shared__ __align__(16) float shared[kFewStages][kRows * kFewPitch];
  chain_next();
  chain_wait();
  const int tid = threadIdx.x, i0 = blockIdx.y * kFewAtOnce, piece = tid % 8 * 4;
  const int64_t j0 = (int64_t)blockIdx.x * kFewTile;
  const int steps = (d + kFewSteps - 1) / kFewSteps;
  const float* from[kRows / 8];
  uint32_t there = 0;
#pragma unroll
  for (int q = 0; q < kRows / 8; ++q) {
    const int row = q * 8 + tid / 8;
    const bool of_w = q < kFewTile / 8, in = of_w ? j0 + row < vocab : i0 + row - kFewTile < rows;
    from[q] = !in ? w : of_w ? w + (j0 + row) * ldw : x + (int64_t)(i0 + row - kFewTile) * ldx;
    there |= (uint32_t)in << q;
  }
  auto copy = [&](int step) {
    float* to = shared[step % kFewStages] + tid / 8 * kFewPitch + piece;
    const int k = step * kFewSteps + piece;
#pragma unroll
    for (int q = 0; q < kRows / 8; ++q) copy_or_zero(to + q * 8 * kFewPitch, from[q] + (k < d ? k : 0), (there >> q & 1) && k < d);
  };
#pragma unroll
  for (int i = 0; i < kFewStages - 1; ++i) {
    if (i < steps) copy(i);
    copies_made();
  }
  const int column = tid % 8 + tid / 32 * 32, row = tid / 8 % 4;
  f32x2 all[4][4];
#pragma unroll
  for (int i = 0; i < 16; ++i) all[i / 4][i % 4] = both(0.0f);
  for (int step = 0; step < steps; ++step) {
    copies_wait<kFewStages - 2>();
    __syncthreads();
    if (step + kFewStages - 1 < steps) copy(step + kFewStages - 1);
    copies_made();
    const float* at = shared[step % kFewStages];
    f32x2 v[4][4];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i / 4][i % 4] = both(0.0f);
#pragma unroll
    for (int k = 0; k < kFewSteps; k += 4) {
      Pairs2 a[4], b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = *reinterpret_cast<const Pairs2*>(at + (column + e * 8) * kFewPitch + k);
        b[e] = *reinterpret_cast<const Pairs2*>(at + (kFewTile + row + e * 4) * kFewPitch + k);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = fma2(b[i].b, a[j].b, fma2(b[i].a, a[j].a, v[i][j]));
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) all[i / 4][i % 4] = add2(all[i / 4][i % 4], v[i / 4][i % 4]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = floats_of(all[i][j]);
      if (i0 + row + i * 4 < rows && j0 + column + j * 8 < vocab) z[(int64_t)(i0 + row + i * 4) * ldz + j0 + column + j * 8] = f.x + f.y;
    }
}

// The two gradients' blocks: `width` threads of four channels each, the rows of w among the 256 / width groups of them; as many blocks as there are to be of columns and
// stretches of the vocabulary.
struct FewSplit {
  int width, columns, per, splits;
  FewSplit(int vocab, int d, int blocks) {
    const int vectors = d / 4;
    for (width = 4; width < 64 && width < vectors;) width *= 2;
    columns = (vectors + width - 1) / width;
    const int wanted = std::max(1, blocks / columns);
    per = (int)((((int64_t)vocab + wanted - 1) / wanted + kFewTile - 1) / kFewTile) * kFewTile;
    splits = (vocab + per - 1) / per;
  }
};

// dz of 64 columns and 16 rows: [column][row], each twice, as the factor of a pair of channels.  Asked for a tile ahead.
struct FewTiles {
  static constexpr int kEach = kFewTile * kFewAtOnce / kFewThreads;
  float next[kEach];
  __device__ __forceinline__ void ask(const float* dz, int64_t ldz, int rows, int64_t j0, int end) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int i = e * (kFewThreads / kFewTile) + threadIdx.x / kFewTile;
      const int64_t j = j0 + threadIdx.x % kFewTile;
      next[e] = i < rows && j < end ? dz[i * ldz + j] : 0.0f;
    }
  }
  __device__ __forceinline__ void put(f32x2 (&tile)[kFewTile][kFewAtOnce + 2]) const {
#pragma unroll
    for (int e = 0; e < kEach; ++e) tile[threadIdx.x % kFewTile][e * (kFewThreads / kFewTile) + threadIdx.x / kFewTile] = both(next[e]);
  }
};

// partial [splits][rows][d] of dx = dz w: a thread has four channels of 16 rows, all there are; the groups' sums are joined in shared memory.  (16 rows of
// 131072 x 2048: 385 us, of 163 for w's bytes; 16 rows of 32003 x 1024 75, of 20.  Sums of whole blocks, without the groups, were 4 times the bytes to join.)
__global__ void __launch_bounds__(kFewThreads, 2) few_dx_kernel(const float* dz, int64_t ldz, int rows, const float* w, int64_t ldw, int vocab, int d, int width, int per, float* partial) {
  __shared__ __align__(16) f32x2 tile[kFewTile][kFewAtOnce + 2];
  __shared__ float4 groups_sums[4][kFewThreads];
  chain_next();
  chain_wait();
  const int groups = kFewThreads / width, group = threadIdx.x / width, at = threadIdx.x % width, c0 = blockIdx.x * width * 4, c = c0 + at * 4;
  const int64_t lo = (int64_t)blockIdx.y * per;
  const int end = (int)(lo + per < vocab ? lo + per : vocab);
  f32x2 acc[kFewAtOnce][2];
#pragma unroll
  for (int i = 0; i < kFewAtOnce; ++i) acc[i][0] = acc[i][1] = both(0.0f);
  FewTiles tiles;
  tiles.ask(dz, ldz, rows, lo, end);
  for (int64_t j0 = lo; j0 < end; j0 += kFewTile) {
    __syncthreads();
    tiles.put(tile);
    __syncthreads();
    if (j0 + kFewTile < end) tiles.ask(dz, ldz, rows, j0 + kFewTile, end);
    if (c >= d) continue;
    const int n = (int)(end - j0 < kFewTile ? end - j0 : kFewTile);
    const float* from = w + j0 * ldw + c;
#pragma unroll 8
    for (int j = group; j < n; j += groups) {
      const float4 f = __ldcs(reinterpret_cast<const float4*>(from + (int64_t)j * ldw));
      const f32x2 b[2] = {pair_of(f.x, f.y), pair_of(f.z, f.w)};
#pragma unroll
      for (int i = 0; i < kFewAtOnce; i += 2) {
        const Pairs2 g = *reinterpret_cast<const Pairs2*>(&tile[j][i]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          acc[i][h] = fma2(g.a, b[h], acc[i][h]);
          acc[i + 1][h] = fma2(g.b, b[h], acc[i + 1][h]);
        }
      }
    }
  }
#pragma unroll
  for (int q = 0; q < kFewAtOnce; q += 4) {
    if (q) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = floats_of(acc[q + i][0]), b = floats_of(acc[q + i][1]);
      groups_sums[i][threadIdx.x] = make_float4(a.x, a.y, b.x, b.y);
    }
    __syncthreads();
    const int i = threadIdx.x / width;  // (its row of the four)
    if (i < 4 && q + i < rows && c < d) {
      float4 s = groups_sums[i][at];
      for (int k = 1; k < groups; ++k) {
        const float4 v = groups_sums[i][k * width + at];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      *reinterpret_cast<float4*>(partial + ((int64_t)blockIdx.y * rows + q + i) * d + c) = s;
    }
  }
}

// dw = dz^T x: a thread has four channels of the rows of x and writes those of one row of dw after the other (16 rows of 131072 x 2048: 297 us, of 163; as a product
// in parts 245, and dz and x to write in parts.  32 rows, the second 16 added to what the first wrote: 941, which is why 16 are the most).
__global__ void __launch_bounds__(kFewThreads, 2) few_dw_kernel(const float* dz, int64_t ldz, int rows, const float* x, int64_t ldx, Targets targets, int vocab, int d, int width, int per,
                                                                 float* dw, int64_t lddw) {
  __shared__ __align__(16) f32x2 tile[kFewTile][kFewAtOnce + 2];
  chain_next();
  chain_wait();
  const int groups = kFewThreads / width, group = threadIdx.x / width, c = (blockIdx.x * width + threadIdx.x % width) * 4;
  const int64_t lo = (int64_t)blockIdx.y * per;
  const int end = (int)(lo + per < vocab ? lo + per : vocab);
  f32x2 v[kFewAtOnce][2];
#pragma unroll
  for (int i = 0; i < kFewAtOnce; ++i) {
    float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    // (a row that is ignored may hold anything)
    if (i < rows && c < d && targets.column(i, vocab, nullptr) >= 0) f = *reinterpret_cast<const float4*>(x + i * ldx + c);
    v[i][0] = pair_of(f.x, f.y);
    v[i][1] = pair_of(f.z, f.w);
  }
  FewTiles tiles;
  tiles.ask(dz, ldz, rows, lo, end);
  for (int64_t j0 = lo; j0 < end; j0 += kFewTile) {
    __syncthreads();
    tiles.put(tile);
    __syncthreads();
    if (j0 + kFewTile < end) tiles.ask(dz, ldz, rows, j0 + kFewTile, end);
    if (c >= d) continue;
    const int n = (int)(end - j0 < kFewTile ? end - j0 : kFewTile);
    for (int j = group; j < n; j += groups) {
      f32x2 s[2] = {both(0.0f), both(0.0f)};
#pragma unroll
      for (int i = 0; i < kFewAtOnce; i += 2) {
        const Pairs2 g = *reinterpret_cast<const Pairs2*>(&tile[j][i]);
#pragma unroll
        for (int h = 0; h < 2; ++h) s[h] = fma2(g.b, v[i + 1][h], fma2(g.a, v[i][h], s[h]));
      }
      const float2 a = floats_of(s[0]), b = floats_of(s[1]);
      __stcs(reinterpret_cast<float4*>(dw + (j0 + j) * lddw + c), make_float4(a.x, a.y, b.x, b.y));
    }
  }
}

// out (rows ld apart) = the sum of many splits of few elements: 32 x 4 channels a block, its eight warps an eighth of the splits each
__global__ void __launch_bounds__(256) sum_many_kernel(const float* in, int splits, float* out, int64_t ld, int rows, int d) {
  __shared__ float4 part[8][32];
  chain_next();
  chain_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (splits + 7) / 8, end = min(splits, (warp + 1) * per);
  const int64_t n = (int64_t)rows * d, i = ((int64_t)blockIdx.x * 32 + lane) * 4;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (i < n)
#pragma unroll 8
    for (int k = warp * per; k < end; ++k) {
      const float4 v = __ldcs(reinterpret_cast<const float4*>(in + k * n + i));
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  part[warp][lane] = s;
  __syncthreads();
  if (warp || i >= n) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) {
    const float4 v = part[k][lane];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  const int64_t row = i / d;
  *reinterpret_cast<float4*>(out + row * ld + (i - row * d)) = s;
}

// ------------------------------------------------------------------------------------------- host
size_t up(size_t n) { return (n + 255) & ~(size_t)255; }
int64_t plane_ld(int64_t cols) { return cols < 256 ? (cols + 15) / 16 * 16 : (cols + 63) / 64 * 64; }

constexpr int kMostSplits = 32;  // of dx's contraction

// How many ways dx's contraction over the vocabulary is split, so that its few tiles fill the waves of CTA pairs: 8192 rows of 768 channels are 96 tiles,
// 1.3 waves that take the time of 2, and split in three 3.9 of 4.  In blocks of 64: a tile's own, 8 for its beginning and end, and the partial
// sums, which cost what 8 bytes an element do (512 clocks a block; 3.4 bytes a clock and pair from memory).
int dx_splits(int64_t rows, int vocab, int d) {
  const bool pair = rows > 128;
  const int64_t tile = pair ? 256 : 128, tiles = (rows + tile - 1) / tile * ((d + 255) / 256), at_once = pair ? kPairs : 2 * kPairs, blocks = (vocab + 63) / 64;
  const double sums = 8.0 * (double)rows * d / (at_once * (pair ? 44.0 : 22.0) * 512);
  int best = 1;
  double least = 0;
  for (int n = 1; n <= kMostSplits && (n == 1 || blocks / n >= 8); ++n) {
    const double cost = (double)((tiles * n + at_once - 1) / at_once) * ((blocks + n - 1) / n + 8) + (n > 1 ? n * sums + 10 : 0);
    if (n == 1 || cost < 0.97 * least) {
      best = n;
      least = cost;
    }
  }
  return best;
}

// The same for float: 12 instructions a block of 32, of n_tile / 2 clocks each and 40 at least, tiles of 256 x 32 to 192 (gemm_parts.cu), and what is
// read for a tile, of which the pairs get 50 bytes a clock: for 1901 rows of 520 channels 72 tiles of 64 columns read the probabilities nine times over and took 1.5
// times as long as the product of the logits, of as many operations; split in three they take as long.
int dx_splits_f32(int64_t rows, int vocab, int d) {
  const int64_t m_tiles = (rows + 255) / 256, blocks = (vocab + 31) / 32;
  int best = 1;
  double least = 0;
  for (int n = 1; n <= kMostSplits && (n == 1 || blocks / n >= 16); ++n) {
    double cost = 0;
    for (int w = 32; w <= 192; w += 32) {
      const int64_t tiles = m_tiles * ((d + w - 1) / w) * n;
      const int issue = 12 * (w / 2 > 40 ? w / 2 : 40), read = (256 + w) * 32 * 6 / 50, block = issue > read ? issue : read;
      const double c = (double)((tiles + kPairs - 1) / kPairs) * ((double)((blocks + n - 1) / n) * block + 1500 + 12 * w);
      if (cost == 0 || c < cost) cost = c;
    }
    if (n > 1) cost += n * 8.0 * (double)rows * d / (kPairs * 44.0) + 5000;
    if (n == 1 || cost < 0.97 * least) {
      best = n;
      least = cost;
    }
  }
  return best;
}

// float, up to so many rows: products of w as it is.  Before and now, 16 rows of 32003 x 1024: the loss 157 and 59 us, gradients 293 and 150; of 131072 x 2048 960 and
// 259, 1909 and 881; of 5003 x 512 37 and 27, 72 and 73.  32 rows take w twice, by way of L2: the loss 138 and 76, 930 and 485 us; gradients would be 260 and 290.
bool few_rows(int64_t rows, bool grads) { return rows <= (grads ? 1 : 2) * kFewAtOnce; }
constexpr int kFewBlocks = 4 * kPairs;  // of the gradients: two an SM

// The scratch of pieces of `piece` rows.  Without dx's partial sums it grows with the rows; with them it need not, as fewer rows have more splits.
struct Plan {
  int64_t piece;
  bool few = false;
  int splits = 1;   // of dx's contraction; float: in chunks of so many columns
  int chunk = 0;
  int64_t ldE = 0;  // bf16: of E; float: of the logits
  size_t target, zt, ref, factor, words, parts = 0, E = 0, xs = 0, partial = 0, dwf = 0, xp = 0, wp = 0, ep = 0;
  size_t bytes = 0;
  Planes x, w, e;  // float: strides alone
  // n: rows of a piece; most: of dx's splits
  Plan(int dtype, int64_t rows, int vocab, int d, bool grads, bool dx, bool dw_bf16, int64_t n, int most) : piece(n) {
    auto take = [&](size_t b) {
      const size_t at = bytes;
      bytes += up(b);
      return at;
    };
    words = take(256);
    target = take(n * 4);
    zt = take(n * 4);
    ref = take(n * 4);
    factor = take(n * 4);
    if (dtype == HBP_BF16) {
      ldE = ((int64_t)vocab + 63) / 64 * 64;
      parts = take(((size_t)(vocab + 63) / 64 + 3) * n * 8);  // (slots of 64 columns, of whole tiles of up to 256)
      if (grads) {
        E = take((size_t)n * ldE * 2);
        xs = take((size_t)n * d * 2);
        if (dx && most > 1) splits = std::min(most, dx_splits(n, vocab, d));
        if (splits > 1) partial = take((size_t)splits * n * d * 4);
        if (dw_bf16 && n < rows) dwf = take((size_t)vocab * d * 4);
      }
      return;
    }
    ldE = ((int64_t)vocab + 3) / 4 * 4;
    few = few_rows(rows, grads);
    if (few) {  // (its one piece)
      E = take((size_t)n * ldE * 4);
      if (grads && dx) partial = take((size_t)FewSplit(vocab, d, kFewBlocks).splits * n * d * 4);
      return;
    }
    if (grads && dx && most > 1) splits = std::min(most, dx_splits_f32(n, vocab, d));
    chunk = splits > 1 ? ((vocab + splits - 1) / splits + 63) / 64 * 64 : vocab;
    x.ld = w.ld = plane_ld(d);
    e.ld = splits > 1 ? (int64_t)splits * chunk : plane_ld(vocab);
    x.plane = n * x.ld;
    w.plane = (int64_t)splits * chunk * w.ld;
    e.plane = n * e.ld;
    e.sb = chunk;
    w.sb = (int64_t)chunk * w.ld;
    xp = take((size_t)3 * x.plane * 2);
    wp = take((size_t)3 * w.plane * 2);
    E = take((size_t)n * ldE * 4);
    if (grads) ep = take((size_t)3 * e.plane * 2);
    if (splits > 1) partial = take((size_t)splits * n * d * 4);
  }
};
constexpr int64_t kLeastPiece = 256;
// what grows with rows times vocab: bytes a row
size_t row_bytes(int dtype, int vocab, bool grads) { return dtype == HBP_BF16 ? (grads ? (size_t)vocab * 2 : ((size_t)(vocab + 63) / 64 + 3) * 8) : (size_t)vocab * (grads ? 10 : 4); }

int64_t wanted_piece(int dtype, int64_t rows, int vocab, bool grads) {
  const size_t b = row_bytes(dtype, vocab, grads);
  int64_t n = (int64_t)(kPieceBytes / b) / kLeastPiece * kLeastPiece;
  if (n < kLeastPiece) n = kLeastPiece;
  if (n >= rows) return rows;
  const int64_t pieces = (rows + n - 1) / n;  // of like size
  n = ((rows + pieces - 1) / pieces + kLeastPiece - 1) / kLeastPiece * kLeastPiece;
  return n < rows ? n : rows;
}

struct Call {
  const hbp_vocabulary* v;
  const float* d_loss = nullptr;
  int64_t d_loss_stride = 0;
  float* loss = nullptr;
  void* dx = nullptr;
  int64_t lddx = 0;
  void* dw = nullptr;
  int dw_dtype = 0;
  int64_t lddw = 0;
  bool grads = false;
  uint8_t* scratch = nullptr;
  bool dw_bf16() const { return dw && dw_dtype == HBP_BF16; }
};

bool run_bf16(Launcher& lc, const Call& c, const Plan& plan, int* status) {
  const hbp_vocabulary& v = *c.v;
  uint8_t* s = c.scratch;
  const bool pieces = plan.piece < v.rows;
  for (int64_t lo = 0; lo < v.rows; lo += plan.piece) {
    const int64_t n = v.rows - lo < plan.piece ? v.rows - lo : plan.piece;
    RowData p = {};
    p.rows = n;
    p.vocab = v.vocab; p.d = v.d;
    p.x = (const bf16*)v.x + lo * v.ldx; p.ldx = v.ldx;
    p.w = (const bf16*)v.w; p.ldw = v.ldw;
    p.targets = {(const uint8_t*)v.targets + lo * v.target_bytes, v.target_bytes};
    p.status = v.status;
    p.target = (int*)(s + plan.target);
    p.zt = (float*)(s + plan.zt);
    p.ref = (float*)(s + plan.ref);
    p.factor = (float*)(s + plan.factor);
    p.parts = (float2*)(s + plan.parts);
    p.redo = (int*)(s + plan.words);
    p.d_loss = c.d_loss ? c.d_loss + lo * c.d_loss_stride : nullptr;
    p.d_loss_stride = c.d_loss_stride;
    p.loss = c.loss + lo;
    if (c.grads) {
      p.E = (bf16*)(s + plan.E);
      p.ldE = plan.ldE;
      if (c.dw) p.xs = (bf16*)(s + plan.xs);
    }
    const dim3 blocks((unsigned)((n + kFinishRows - 1) / kFinishRows));
    GemmArgs g;
    g.M = (int)n; g.N = v.vocab; g.K = v.d;
    g.in_dtype = HBP_BF16;
    g.A = p.x; g.a_sm = v.ldx; g.a_sk = 1;
    g.B = p.w; g.b_sn = v.ldw; g.b_sk = 1;
    g.epi = EPI_EXP;
    g.row_parts = p.parts; g.slots_out = &p.slots;
    if (!c.grads) {
      g.target = (const int*)p.targets.t; g.target_bytes = v.target_bytes;
      if (!gemm_tc(lc, g, status)) return false;
      launch_chained(lc, loss_kernel, blocks, 32 * kFinishWarps, 0, 1, p);
      continue;
    }
    launch_chained(lc, target_kernel, dim3((unsigned)((n + 7) / 8)), 256, 0, 1, p);
    g.D = p.E; g.ldd = p.ldE;
    g.row_f = p.ref; g.target = p.target;
    for (int again = 0; again < 2; ++again) {
      p.again = again != 0;
      g.redo = again ? p.redo : nullptr;
      if (!gemm_tc(lc, g, status)) return false;
      launch_chained(lc, finish_kernel, blocks, 32 * kFinishWarps, 0, 1, p);
    }
    if (c.dx) {
      GemmArgs b;
      b.M = (int)n; b.N = v.d; b.K = v.vocab;
      b.in_dtype = HBP_BF16;
      b.A = p.E; b.a_sm = p.ldE; b.a_sk = 1;
      b.B = p.w; b.b_sn = 1; b.b_sk = v.ldw;
      bf16* dx = (bf16*)c.dx + lo * c.lddx;
      const int splits = std::min(plan.splits, dx_splits(n, v.vocab, v.d));  // (the last piece is smaller, and its memory the others')
      if (splits > 1) {
        b.splitk = splits;
        b.wide = true;
        b.partial = (float*)(s + plan.partial);
        b.d_f32 = true;
        b.D = b.partial; b.ldd = v.d;
        int made = 1;
        b.splits_out = &made;
        if (!gemm_tc(lc, b, status)) return false;
        launch_chained(lc, narrow_kernel, dim3((unsigned)((n * v.d / 8 + 255) / 256)), 256, 0, 1, (const float*)b.partial, made, p.factor, dx, c.lddx, n, v.d);
      } else {
        b.epi = EPI_ROWS;
        b.row_f = p.factor;
        b.D = dx; b.ldd = c.lddx;
        if (!gemm_tc(lc, b, status)) return false;
      }
    }
    if (c.dw) {
      GemmArgs b;
      b.M = v.vocab; b.N = v.d; b.K = (int)n;
      b.in_dtype = HBP_BF16;
      b.A = p.E; b.a_sm = 1; b.a_sk = p.ldE;
      b.B = p.xs; b.b_sn = 1; b.b_sk = v.d;
      const bool narrow_after = pieces && c.dw_bf16();
      b.d_f32 = narrow_after || !c.dw_bf16();
      b.D = narrow_after ? (void*)(s + plan.dwf) : c.dw;
      b.ldd = narrow_after ? v.d : c.lddw;
      if (lo) b.epi = EPI_ACCUM;
      if (!gemm_tc(lc, b, status)) return false;
      if (narrow_after && lo + n == v.rows)
        launch_chained(lc, narrow_kernel, dim3((unsigned)(((int64_t)v.vocab * v.d / 8 + 255) / 256)), 256, 0, 1, (const float*)b.D, 1, (const float*)nullptr, (bf16*)c.dw,
                       c.lddw, (int64_t)v.vocab, v.d);
    }
  }
  return true;
}

void run_few(Launcher& lc, const Call& c, const Plan& plan) {
  const hbp_vocabulary& v = *c.v;
  const int n = (int)v.rows;
  const Targets targets = {v.targets, v.target_bytes};
  float* z = (float*)(c.scratch + plan.E);
  const int64_t ldz = plan.ldE;
  launch_chained(lc, few_logits_kernel, dim3((unsigned)((v.vocab + kFewTile - 1) / kFewTile), (unsigned)((n + kFewAtOnce - 1) / kFewAtOnce)), 64, 0, 1,
                 (const float*)v.x, v.ldx, n, (const float*)v.w, v.ldw, v.vocab, v.d, z, ldz);
  LogitsData p = {};
  p.z = z; p.ldz = ldz;
  p.vocab = p.columns = v.vocab;
  p.targets = targets;
  p.status = v.status;
  p.d_loss = c.d_loss;
  p.d_loss_stride = c.d_loss_stride;
  p.loss = c.loss;
  if (c.grads) p.dz_f = z;
  const int shares = logit_shares(n, v.vocab);
  launch_chained(lc, shares > 1 ? logits_kernel<true> : logits_kernel<false>, dim3((unsigned)(n * shares)), kRowThreads, 0, shares, p);
  const FewSplit f(v.vocab, v.d, kFewBlocks);
  if (c.dx) {
    float* partial = (float*)(c.scratch + plan.partial);
    launch_chained(lc, few_dx_kernel, dim3(f.columns, f.splits), kFewThreads, 0, 1, (const float*)z, ldz, n, (const float*)v.w, v.ldw, v.vocab, v.d, f.width, f.per, partial);
    launch_chained(lc, sum_many_kernel, dim3((unsigned)(((int64_t)n * v.d / 4 + 31) / 32)), 256, 0, 1, (const float*)partial, f.splits, (float*)c.dx, c.lddx, n, v.d);
  }
  if (c.dw)
    launch_chained(lc, few_dw_kernel, dim3(f.columns, f.splits), kFewThreads, 0, 1, (const float*)z, ldz, n, (const float*)v.x, v.ldx, targets, v.vocab, v.d, f.width, f.per,
                   (float*)c.dw, c.lddw);
}

bool run_f32(Launcher& lc, const Call& c, const Plan& plan, int* status) {
  const hbp_vocabulary& v = *c.v;
  uint8_t* s = c.scratch;
  Planes x = plan.x, w = plan.w, e = plan.e;
  x.p = (bf16*)(s + plan.xp);
  w.p = (bf16*)(s + plan.wp);
  auto split = [&](const float* src, int64_t ld, const Planes& P, int64_t rows, int64_t all, const Targets& targets) {
    launch_chained(lc, split_rows_kernel, dim3((unsigned)((all * (v.d / 4) + 255) / 256)), 256, 0, 1, src, ld, P, rows, all, v.d, targets, v.vocab);
  };
  if (plan.few) {
    run_few(lc, c, plan);
    return true;
  }
  const int64_t columns = (int64_t)plan.splits * plan.chunk;
  split((const float*)v.w, v.ldw, w, v.vocab, columns, Targets{nullptr, 8});
  for (int64_t lo = 0; lo < v.rows; lo += plan.piece) {
    const int64_t n = v.rows - lo < plan.piece ? v.rows - lo : plan.piece;
    const Targets targets = {(const uint8_t*)v.targets + lo * v.target_bytes, v.target_bytes};
    split((const float*)v.x + lo * v.ldx, v.ldx, x, n, n, targets);
    PartsGemm g;
    g.M = (int)n; g.N = v.vocab; g.K = v.d;
    g.A = x; g.B = w;
    g.D = (float*)(s + plan.E); g.ldd = plan.ldE;
    if (!gemm_parts(lc, g, status)) return false;
    LogitsData p = {};
    p.z = g.D; p.ldz = plan.ldE;
    p.vocab = v.vocab; p.columns = (int)columns;
    p.targets = targets;
    p.status = v.status;
    p.d_loss = c.d_loss ? c.d_loss + lo * c.d_loss_stride : nullptr;
    p.d_loss_stride = c.d_loss_stride;
    p.loss = c.loss + lo;
    if (c.grads) {
      e.p = (bf16*)(s + plan.ep);
      p.dz = e;
    }
    const int shares = logit_shares(n, v.vocab);
    launch_chained(lc, shares > 1 ? logits_kernel<true> : logits_kernel<false>, dim3((unsigned)(n * shares)), kRowThreads, 0, shares, p);
    if (c.dx) {
      PartsGemm b;
      b.M = (int)n; b.N = v.d; b.K = plan.chunk;
      b.batch = plan.splits;  // (chunks of the contraction; behind the vocabulary there are zeros)
      b.A = e; b.B = w;
      b.b_mn = true;
      float* dx = (float*)c.dx + lo * c.lddx;
      b.D = plan.splits > 1 ? (float*)(s + plan.partial) : dx;
      b.ldd = plan.splits > 1 ? v.d : c.lddx;
      b.d_sb = n * v.d;
      if (!gemm_parts(lc, b, status)) return false;
      if (plan.splits > 1)
        launch_chained(lc, sum_splits_kernel, dim3((unsigned)((n * v.d / 4 + 255) / 256)), 256, 0, 1, (const float*)b.D, plan.splits, dx, c.lddx, n, v.d);
    }
    if (c.dw) {
      PartsGemm b;
      b.M = v.vocab; b.N = v.d; b.K = (int)n;
      b.A = e; b.B = x;
      b.a_mn = b.b_mn = true;
      b.D = (float*)c.dw; b.ldd = c.lddw;
      if (lo) {
        b.epi = EPI_RESID;
        b.E = (const float*)c.dw; b.lde = c.lddw;
      }
      if (!gemm_parts(lc, b, status)) return false;
    }
  }
  return true;
}

hbp_status check(const hbp_vocabulary* v) {
  if (!v) return HBP_ERR_INVALID_ARG;
  if (v->dtype != HBP_F32 && v->dtype != HBP_BF16) return HBP_ERR_DTYPE;
  const int k = v->dtype == HBP_F32 ? 4 : 8;
  // (columns and rows of tiles are 32-bit numbers, a little beyond the last ones too)
  if (v->rows < 0 || v->rows > (1 << 30) || v->vocab <= 0 || v->vocab > (1 << 30) || v->d <= 0 || v->d % k || v->d > (1 << 24)) return HBP_ERR_SHAPE;
  if (v->target_bytes != 4 && v->target_bytes != 8) return HBP_ERR_INVALID_ARG;
  if (((uintptr_t)v->targets % v->target_bytes) || ((uintptr_t)v->status & 3u)) return HBP_ERR_SHAPE;
  return HBP_OK;
}
bool bad_rows(const void* t, int64_t ld, int d, int v) { return ((uintptr_t)t & 15u) || ld % v || ld < d; }

hbp_status call(Call& c, void* scratch, size_t bytes, void* stream) {
  const hbp_vocabulary& v = *c.v;
  const int k = v.dtype == HBP_F32 ? 4 : 8;
  if (!v.w || (v.rows && (!v.x || !v.targets || !c.loss))) return HBP_ERR_INVALID_ARG;
  if (bad_rows(v.w, v.ldw, v.d, k) || (v.rows && bad_rows(v.x, v.ldx, v.d, k)) || ((uintptr_t)c.loss & 3u)) return HBP_ERR_SHAPE;
  Launcher lc;
  lc.stream = (cudaStream_t)stream;
  if (v.rows == 0) {
    if (!c.dw) return HBP_OK;
    const size_t es = c.dw_bf16() ? 2 : 4;
    return cudaMemset2DAsync(c.dw, c.lddw * es, 0, v.d * es, v.vocab, lc.stream) == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
  }
  int64_t n = wanted_piece(v.dtype, v.rows, v.vocab, c.grads);
  auto plan_of = [&](int64_t piece, int most) { return Plan(v.dtype, v.rows, v.vocab, v.d, c.grads, c.dx != nullptr, c.dw_bf16(), piece, most); };
  if (!scratch || ((uintptr_t)scratch & 255u)) return HBP_ERR_WORKSPACE;
  Plan plan = plan_of(n, kMostSplits);
  while (plan.bytes > bytes) {  // fewer splits for less memory (what is enough for more rows is then enough), then smaller pieces
    if (plan.splits > 1) {
      plan = plan_of(n, plan.splits - 1);
      continue;
    }
    if (n <= kLeastPiece) return HBP_ERR_WORKSPACE;
    n = (n / 2 + kLeastPiece - 1) / kLeastPiece * kLeastPiece;
    plan = plan_of(n, kMostSplits);
  }
  c.scratch = (uint8_t*)scratch;
  int* status = v.status ? v.status : (int*)(c.scratch + plan.words) + 1;
  const bool ok = v.dtype == HBP_BF16 ? run_bf16(lc, c, plan, status) : run_f32(lc, c, plan, status);
  return ok && lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}

}  // namespace

}  // namespace hbp

using namespace hbp;

extern "C" hbp_status hbp_cross_entropy_scratch_bytes(const hbp_vocabulary* v, int32_t gradients, size_t* bytes) {
  if (!bytes) return HBP_ERR_INVALID_ARG;
  const hbp_status st = check(v);
  if (st != HBP_OK) return st;
  const bool grads = gradients != 0;
  *bytes = v->rows ? Plan(v->dtype, v->rows, v->vocab, v->d, grads, true, true, wanted_piece(v->dtype, v->rows, v->vocab, grads), kMostSplits).bytes : 0;
  return HBP_OK;
}

extern "C" hbp_status hbp_cross_entropy(const hbp_vocabulary* v, float* loss, void* scratch, size_t scratch_bytes, void* cuda_stream) {
  const hbp_status st = check(v);
  if (st != HBP_OK) return st;
  Call c;
  c.v = v;
  c.loss = loss;
  return call(c, scratch, scratch_bytes, cuda_stream);
}

extern "C" hbp_status hbp_cross_entropy_gradients(const hbp_vocabulary* v, const float* d_loss, int64_t d_loss_stride, float* loss, void* dx, int64_t lddx,
                                                  void* dw, int32_t dw_dtype, int64_t lddw, void* scratch, size_t scratch_bytes, void* cuda_stream) {
  const hbp_status st = check(v);
  if (st != HBP_OK) return st;
  const int k = v->dtype == HBP_F32 ? 4 : 8;
  if (!dx && !dw) return HBP_ERR_INVALID_ARG;
  if (dw && dw_dtype != HBP_F32 && !(dw_dtype == HBP_BF16 && v->dtype == HBP_BF16)) return HBP_ERR_DTYPE;
  if (d_loss_stride < 0 || ((uintptr_t)d_loss & 3u) || (dx && v->rows && bad_rows(dx, lddx, v->d, k)) || (dw && bad_rows(dw, lddw, v->d, dw_dtype == HBP_F32 ? 4 : 8)))
    return HBP_ERR_SHAPE;
  Call c;
  c.v = v;
  c.d_loss = d_loss;
  c.d_loss_stride = d_loss_stride;
  c.loss = loss;
  c.dx = dx; c.lddx = lddx;
  c.dw = dw; c.dw_dtype = dw_dtype; c.lddw = lddw;
  c.grads = true;
  return call(c, scratch, scratch_bytes, cuda_stream);
}
