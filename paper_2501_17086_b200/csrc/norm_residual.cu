// A residual update with its gate and scale, the norm of the block's output before it and the norm of the new stream after it, in one
// pass over the rows (hbp_norm_residual), and its gradients (hbp_norm_residual_backward).
//
//   h = norm(f) * w_post (or f),   x' = gate * x + scale * h, rounded to dtype,   y = norm(x') * w_pre
//   norm: (v - mean) / sqrt(mean((v - mean)^2) + eps), or without the mean (RMS)
//
// A row is held in the registers of 32 to 512 threads, 16 bytes of consecutive channels a vector: each tensor is read once and written
// once, and the sum of squares is taken around the mean itself.  The backward pass forms the statistics again from the rows that it reads
// anyway (nothing is kept by the forward pass) and merges its row sums: with a = dy * w_pre, of which the norm's gradient is
// r (a - mean(a) - xhat mean(a xhat)), sum(a) and sum(a (v - mean)) come with the sum of squares.  Gradients of the [d] weights are added
// up in registers over the rows of a group of threads, over a block's groups in shared memory, and over blocks by a second launch, all in
// fixed order.
#include <type_traits>

#include "hbp_internal.h"
#include "tc_common.cuh"

namespace hbp {

namespace {

struct Rows {
  const void* x;
  int64_t ld;
};

struct NormParams {
  int64_t rows;
  int d, per_row, threads;  // vectors a row; threads that hold one
  float eps, scale, inv_d;
  const void *w_post, *gate, *w_pre;
  Rows x, f, x_new, y;                 // forward: x_new and y are written
  Rows d_y, d_new, dx, df;             // backward
  float* partial;                      // [blocks][3][d]: of dw_pre, dw_post, da
  bool want_pre, want_post, want_gate;
};

template <typename T>
struct Vec {
  static constexpr int V = 16 / (int)sizeof(T);
  static __device__ __forceinline__ void widen(const uint4& r, float* f) {
    if constexpr (sizeof(T) == 2) {
      tc::unpack8(r, f);
    } else {
      f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
    }
  }
  static __device__ __forceinline__ uint4 narrow(const float* f) {
    if constexpr (sizeof(T) == 2) return tc::pack8(f);
    else return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};

constexpr int kMaxWarps = 16;  // of a block

// Sums of K values over the threads of a row, in every one of them.  Rows of more than a warp use a barrier of their own; two buffers in
// turn, so that one barrier a sum is enough.
template <int K>
__device__ __forceinline__ void row_sum(float (&v)[K], int threads, int group, float (*buf)[kMaxWarps][4], int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (threads == 32) return;
  const int warp = threadIdx.x >> 5, warps = threads >> 5;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) buf[turn][warp][k] = v[k];
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.0f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += buf[turn][group * warps + w][k];
  turn ^= 1;
}

template <typename T>
__device__ __forceinline__ uint4 load(const Rows& r, int64_t row, int c) {
  return *reinterpret_cast<const uint4*>((const T*)r.x + row * r.ld + c);
}
template <typename T>
__device__ __forceinline__ void store(const Rows& r, int64_t row, int c, const float* f) {
  *reinterpret_cast<uint4*>((T*)r.x + row * r.ld + c) = Vec<T>::narrow(f);
}
// weights of one vector of channels, or ones
template <typename T>
__device__ __forceinline__ void weights(const void* w, int c, float* f) {
  constexpr int V = Vec<T>::V;
  if (w) {
    Vec<T>::widen(*reinterpret_cast<const uint4*>((const T*)w + c), f);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 1.0f;
  }
}

// Mean (0 without kLayer) and 1 / sqrt(mean square + eps) of a row's values.  Channels beyond d hold zeros.
template <int NV, int V, bool kLayer>
__device__ __forceinline__ float2 statistics(const float (&v)[NV][V], const bool (&in)[NV], const NormParams& p, int group, float (*buf)[kMaxWarps][4],
                                             int& turn) {
  float m[1] = {0.0f};
  if (kLayer) {
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) m[0] += v[u][e];
    row_sum(m, p.threads, group, buf, turn);
    m[0] *= p.inv_d;
  }
  float q[1] = {0.0f};
#pragma unroll
  for (int u = 0; u < NV; ++u)
    if (in[u])
#pragma unroll
      for (int e = 0; e < V; ++e) q[0] = fmaf(v[u][e] - m[0], v[u][e] - m[0], q[0]);
  row_sum(q, p.threads, group, buf, turn);
  return make_float2(m[0], 1.0f / sqrtf(fmaf(q[0], p.inv_d, p.eps)));
}

// ------------------------------------------------------------------------------------------- forward
// kBlock: the block's output and the update, else only the norm of the stream.
template <typename T, int NV, bool kLayer, bool kBlock, bool kPost>
__global__ void __launch_bounds__(512) norm_forward_kernel(const NormParams p) {
  constexpr int V = Vec<T>::V;
  __shared__ float buf[2][kMaxWarps][4];
  chain_next();
  chain_wait();
  int turn = 0;
  const int group = threadIdx.x / p.threads, t = threadIdx.x - group * p.threads;
  const int64_t row = (int64_t)blockIdx.x * (blockDim.x / p.threads) + group;
  if (row >= p.rows) return;
  float v[NV][V];
  bool in[NV];
  uint4 x[NV], f[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int c = (t + u * p.threads) * V;
    in[u] = c < p.d;
    x[u] = f[u] = make_uint4(0, 0, 0, 0);
    if (in[u]) {
      x[u] = load<T>(p.x, row, c);
      if (kBlock) f[u] = load<T>(p.f, row, c);
    }
  }
  if (kBlock) {
    float2 s = make_float2(0.0f, 1.0f);
#pragma unroll
    for (int u = 0; u < NV; ++u) Vec<T>::widen(f[u], v[u]);
    if (kPost) s = statistics<NV, V, kLayer>(v, in, p, group, buf, turn);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * p.threads) * V;
      if (!in[u]) continue;
      float w[V], g[V], xf[V];
      weights<T>(kPost ? p.w_post : nullptr, c, w);
      weights<T>(p.gate, c, g);
      Vec<T>::widen(x[u], xf);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = kPost ? (v[u][e] - s.x) * s.y * w[e] : v[u][e];
        v[u][e] = fmaf(p.scale, h, g[e] * xf[e]);
      }
      x[u] = Vec<T>::narrow(v[u]);
      *reinterpret_cast<uint4*>((T*)p.x_new.x + row * p.x_new.ld + c) = x[u];
    }
    if (!p.y.x) return;
  }
#pragma unroll
  for (int u = 0; u < NV; ++u) Vec<T>::widen(x[u], v[u]);  // the stream as it is stored
  const float2 s = statistics<NV, V, kLayer>(v, in, p, group, buf, turn);
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int c = (t + u * p.threads) * V;
    if (!in[u]) continue;
    float w[V];
    weights<T>(p.w_pre, c, w);
#pragma unroll
    for (int e = 0; e < V; ++e) v[u][e] = (v[u][e] - s.x) * s.y * w[e];
    store<T>(p.y, row, c, v[u]);
  }
}

// ------------------------------------------------------------------------------------------- backward
template <typename T, int NV, bool kLayer, bool kPost>
__global__ void __launch_bounds__(512) norm_backward_kernel(const NormParams p) {
  constexpr int V = Vec<T>::V;
  __shared__ float buf[2][kMaxWarps][4];
  extern __shared__ float sums[];  // [3][d]: of a block's groups
  chain_next();
  chain_wait();
  int turn = 0;
  const int groups = blockDim.x / p.threads, group = threadIdx.x / p.threads, t = threadIdx.x - group * p.threads;
  float dw_pre[NV][V], dw_post[NV][V], da[NV][V];
  bool in[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    in[u] = (t + u * p.threads) * V < p.d;
#pragma unroll
    for (int e = 0; e < V; ++e) dw_pre[u][e] = dw_post[u][e] = da[u][e] = 0.0f;
  }
  for (int64_t row = (int64_t)blockIdx.x * groups + group; row < p.rows; row += (int64_t)gridDim.x * groups) {
    uint4 dy[NV], dn[NV], xn[NV], f[NV], x[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * p.threads) * V;
      dy[u] = dn[u] = xn[u] = f[u] = x[u] = make_uint4(0, 0, 0, 0);
      if (!in[u]) continue;
      if (p.d_y.x) {
        dy[u] = load<T>(p.d_y, row, c);
        xn[u] = load<T>(p.x_new, row, c);
      }
      if (p.d_new.x) dn[u] = load<T>(p.d_new, row, c);
      if (kPost) f[u] = load<T>(p.f, row, c);
      if (p.want_gate) x[u] = load<T>(p.x, row, c);
    }
    // means of the stream and the block's output
    float mean[2] = {0.0f, 0.0f};
    if (kLayer) {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float a[V], b[V];
        Vec<T>::widen(xn[u], a);
        Vec<T>::widen(f[u], b);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          mean[0] += a[e];
          if (kPost) mean[1] += b[e];
        }
      }
      row_sum(mean, p.threads, group, buf, turn);
      mean[0] *= p.inv_d;
      mean[1] *= p.inv_d;
    }
    // sums of squares around them, and of a = dy * w_pre and a times the centred stream
    float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!in[u]) continue;
      float a[V], v[V], w[V];
      Vec<T>::widen(dy[u], a);
      Vec<T>::widen(xn[u], v);
      weights<T>(p.w_pre, (t + u * p.threads) * V, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float cx = v[e] - mean[0], g = a[e] * w[e];
        q[0] = fmaf(cx, cx, q[0]);
        q[1] = fmaf(g, cx, q[1]);
        q[2] += g;
      }
      if (kPost) {
        Vec<T>::widen(f[u], v);
#pragma unroll
        for (int e = 0; e < V; ++e) q[3] = fmaf(v[e] - mean[1], v[e] - mean[1], q[3]);
      }
    }
    row_sum(q, p.threads, group, buf, turn);
    const float r = 1.0f / sqrtf(fmaf(q[0], p.inv_d, p.eps)), along = q[1] * r * p.inv_d, flat = kLayer ? q[2] * p.inv_d : 0.0f;
    const float rf = kPost ? 1.0f / sqrtf(fmaf(q[3], p.inv_d, p.eps)) : 1.0f;
    // the gradient of the new stream; what it gives
    float g[NV][V], b[2] = {0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * p.threads) * V;
      if (!in[u]) continue;
      float a[V], v[V], w[V], fv[V], wp[V];
      Vec<T>::widen(dn[u], g[u]);
      if (p.d_y.x) {
        Vec<T>::widen(dy[u], a);
        Vec<T>::widen(xn[u], v);
        weights<T>(p.w_pre, c, w);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float xhat = (v[e] - mean[0]) * r;
          dw_pre[u][e] = fmaf(a[e], xhat, dw_pre[u][e]);
          g[u][e] = fmaf(fmaf(-xhat, along, fmaf(a[e], w[e], -flat)), r, g[u][e]);
        }
      }
      if (p.want_gate) {
        Vec<T>::widen(x[u], v);
#pragma unroll
        for (int e = 0; e < V; ++e) da[u][e] = fmaf(g[u][e], v[e], da[u][e]);
      }
      if (kPost) {
        Vec<T>::widen(f[u], fv);
        weights<T>(p.w_post, c, wp);
      }
      if (p.dx.x) {
        weights<T>(p.gate, c, w);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = g[u][e] * w[e];
        store<T>(p.dx, row, c, v);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) g[u][e] *= p.scale;  // of h
      if (kPost) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float fhat = (fv[e] - mean[1]) * rf;
          dw_post[u][e] = fmaf(g[u][e], fhat, dw_post[u][e]);
          g[u][e] *= wp[e];
          b[0] = fmaf(g[u][e], fhat, b[0]);
          b[1] += g[u][e];
        }
      }
    }
    if (!p.df.x) continue;
    if (kPost) row_sum(b, p.threads, group, buf, turn);
    const float along_f = b[0] * p.inv_d, flat_f = kLayer ? b[1] * p.inv_d : 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!in[u]) continue;
      if (kPost) {
        float fv[V];
        Vec<T>::widen(f[u], fv);
#pragma unroll
        for (int e = 0; e < V; ++e) g[u][e] = (g[u][e] - flat_f - (fv[e] - mean[1]) * rf * along_f) * rf;
      }
      store<T>(p.df, row, (t + u * p.threads) * V, g[u]);
    }
  }
  if (!p.partial) return;
  for (int k = 0; k < groups; ++k) {  // the groups' sums, one after the other
    if (k == group) {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int c = (t + u * p.threads) * V;
        if (!in[u]) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          sums[c + e] = k ? sums[c + e] + dw_pre[u][e] : dw_pre[u][e];
          sums[p.d + c + e] = k ? sums[p.d + c + e] + dw_post[u][e] : dw_post[u][e];
          sums[2 * p.d + c + e] = k ? sums[2 * p.d + c + e] + da[u][e] : da[u][e];
        }
      }
    }
    __syncthreads();
  }
  float* to = p.partial + (int64_t)blockIdx.x * 3 * p.d;
  for (int i = threadIdx.x * 4; i < 3 * p.d; i += blockDim.x * 4) {
    const int k = i / p.d;
    if (k == 0 ? p.want_pre : k == 1 ? p.want_post : p.want_gate) *reinterpret_cast<float4*>(to + i) = *reinterpret_cast<const float4*>(sums + i);
  }
}

// out[k][c] = sum over the blocks: 32 x 4 channels a block, its eight warps an eighth of them each
struct WeightSums {
  const float* partial;
  int blocks, d;
  float* out[3];
};
__global__ void __launch_bounds__(256) weight_sums_kernel(const WeightSums p) {
  __shared__ float4 part[8][32];
  chain_next();
  chain_wait();
  float* out = p.out[blockIdx.y];
  if (!out) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (blockIdx.x * 32 + lane) * 4;
  const int per = (p.blocks + 7) / 8, end = min(p.blocks, (warp + 1) * per);
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (c < p.d)
#pragma unroll 8
    for (int b = warp * per; b < end; ++b) {
      const float4 v = *reinterpret_cast<const float4*>(p.partial + ((int64_t)b * 3 + blockIdx.y) * p.d + c);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < p.d) {
#pragma unroll
    for (int w = 1; w < 8; ++w) {
      const float4 v = part[w][lane];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    *reinterpret_cast<float4*>(out + c) = s;
  }
}

// ------------------------------------------------------------------------------------------- host
constexpr int kMaxWidth = 8192;

// Vectors a thread holds, and threads a row (whole warps).  Rows of up to 128 vectors (forward; 32 backward, whose threads hold the weights' sums
// too) are a warp's: no barriers.
void split_of(int per_row, bool backward, int* nv, int* threads) {
  if (per_row <= 32) *nv = 1;
  else if (!backward && per_row <= 64) *nv = 2;
  else if (!backward && per_row <= 128) *nv = 4;
  else if (backward && per_row <= 256) *nv = 1;
  else *nv = per_row <= 1024 ? 2 : 4;
  *threads = ((per_row + *nv - 1) / *nv + 31) / 32 * 32;
}

// Blocks of `threads` threads and `smem` bytes that an SM runs at once, by the kernel's registers (looked up once, as its leave for the
// widest rows' shared memory is asked for); 0: an error.
int blocks_at_once(const void* kernel, int& registers, int threads, size_t smem) {
  if (registers == 0) {
    cudaFuncAttributes a;
    if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kMaxWidth * 4) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    registers = (a.numRegs + 7) / 8 * 8;
  }
  const int by_regs = 65536 / registers / threads, by_threads = 2048 / threads, by_smem = (int)((227 << 10) / (smem + 2048));
  const int n = by_regs < by_threads ? by_regs : by_threads, m = n < by_smem ? n : by_smem;
  return m > 0 ? m : 1;
}

template <typename T, int NV, bool kLayer>
void forward(Launcher& lc, const NormParams& p, bool post) {
  const int groups = p.threads >= 256 ? 1 : 256 / p.threads;
  auto kernel = !p.f.x ? norm_forward_kernel<T, NV, kLayer, false, false>
                       : post ? norm_forward_kernel<T, NV, kLayer, true, true> : norm_forward_kernel<T, NV, kLayer, true, false>;
  launch_chained(lc, kernel, dim3((unsigned)((p.rows + groups - 1) / groups)), groups * p.threads, 0, 1, p);
}

constexpr int kMostBlocks = 4;     // an SM, backward: each leaves 12 d bytes for the second launch
constexpr int kMostPartials = 640;  // and all of them together

template <typename T, int NV, bool kLayer>
int backward(Launcher& lc, NormParams& p, bool post) {
  const int groups = p.threads >= 256 ? 1 : 256 / p.threads;
  auto kernel = post ? norm_backward_kernel<T, NV, kLayer, true> : norm_backward_kernel<T, NV, kLayer, false>;
  const size_t smem = p.partial ? (size_t)3 * p.d * 4 : 0;
  static PerDevice<int> registers[2];
  int per_sm = blocks_at_once((const void*)kernel, registers[post].here(), groups * p.threads, smem);
  if (per_sm == 0) {
    lc.err = cudaErrorInvalidValue;
    return 0;
  }
  if (per_sm > kMostBlocks) per_sm = kMostBlocks;
  const int64_t wanted = (p.rows + groups - 1) / groups, at_once = (int64_t)per_sm * tc::sm_count(), most = at_once < kMostPartials ? at_once : kMostPartials;
  const int blocks = (int)(wanted < most ? wanted : most);
  launch_chained(lc, kernel, dim3(blocks), groups * p.threads, smem, 1, p);
  return blocks;
}

hbp_status check(const hbp_norm* n) {
  if (!n) return HBP_ERR_INVALID_ARG;
  if (n->dtype != HBP_F32 && n->dtype != HBP_BF16) return HBP_ERR_DTYPE;
  if (n->kind != HBP_NORM_LAYER && n->kind != HBP_NORM_RMS) return HBP_ERR_UNSUPPORTED;
  if (n->rows < 0 || n->rows > INT32_MAX || n->d <= 0 || n->d % (n->dtype == HBP_F32 ? 4 : 8) || n->d > kMaxWidth) return HBP_ERR_SHAPE;
  if (!(n->eps >= 0.0f) || !(n->eps - n->eps == 0.0f) || !(n->scale - n->scale == 0.0f)) return HBP_ERR_INVALID_ARG;
  for (const void* w : {n->w_post, n->gate, n->w_pre})
    if ((uintptr_t)w & 15u) return HBP_ERR_SHAPE;
  return HBP_OK;
}
// a tensor's rows, none if it is not given
bool rows_of(const hbp_norm& n, const hbp_rows* t, bool input, Rows* r) {
  *r = {nullptr, 0};
  if (!t || !t->x) return true;
  const int v = n.dtype == HBP_F32 ? 4 : 8;
  if (((uintptr_t)t->x & 15u) || t->stride % v || (t->stride < n.d && !(input && t->stride == 0) && n.rows > 1)) return false;
  *r = {t->x, t->stride};
  return true;
}
// an output that lies on an input has to lie on it row by row
bool on_itself(const Rows& out, const Rows& in) { return !out.x || out.x != in.x || out.ld == in.ld; }

NormParams params_of(const hbp_norm& n, bool backward, int* nv) {
  NormParams p = {};
  p.rows = n.rows;
  p.d = n.d;
  p.per_row = n.d / (n.dtype == HBP_F32 ? 4 : 8);
  split_of(p.per_row, backward, nv, &p.threads);
  p.eps = n.eps;
  p.scale = n.scale;
  p.inv_d = (float)(1.0 / n.d);
  p.w_post = n.w_post; p.gate = n.gate; p.w_pre = n.w_pre;
  return p;
}

size_t partial_bytes(int64_t rows, int d) { return (size_t)(rows < kMostPartials ? rows : kMostPartials) * 3 * d * 4; }

template <typename F>
auto by_variant(const hbp_norm& n, int nv, F&& f) {
  const bool layer = n.kind == HBP_NORM_LAYER;
  if (n.dtype == HBP_F32) {
    if (nv == 1) return layer ? f(float(), std::integral_constant<int, 1>(), std::true_type()) : f(float(), std::integral_constant<int, 1>(), std::false_type());
    if (nv == 2) return layer ? f(float(), std::integral_constant<int, 2>(), std::true_type()) : f(float(), std::integral_constant<int, 2>(), std::false_type());
    return layer ? f(float(), std::integral_constant<int, 4>(), std::true_type()) : f(float(), std::integral_constant<int, 4>(), std::false_type());
  }
  if (nv == 1) return layer ? f(bf16(), std::integral_constant<int, 1>(), std::true_type()) : f(bf16(), std::integral_constant<int, 1>(), std::false_type());
  if (nv == 2) return layer ? f(bf16(), std::integral_constant<int, 2>(), std::true_type()) : f(bf16(), std::integral_constant<int, 2>(), std::false_type());
  return layer ? f(bf16(), std::integral_constant<int, 4>(), std::true_type()) : f(bf16(), std::integral_constant<int, 4>(), std::false_type());
}

}  // namespace

}  // namespace hbp

using namespace hbp;

extern "C" hbp_status hbp_norm_residual(const hbp_norm* n, const hbp_rows* x, const hbp_rows* f, const hbp_rows* x_new, const hbp_rows* y, void* cuda_stream) {
  const hbp_status st = check(n);
  if (st != HBP_OK) return st;
  if (n->rows == 0) return HBP_OK;
  int nv = 1;
  NormParams p = params_of(*n, false, &nv);
  if (!rows_of(*n, x, true, &p.x) || !rows_of(*n, f, true, &p.f) || !rows_of(*n, x_new, false, &p.x_new) || !rows_of(*n, y, false, &p.y)) return HBP_ERR_SHAPE;
  // without a block's output there is no update: the norm of the stream is left
  if (!p.x.x || (!p.f.x && (p.x_new.x || !p.y.x || n->post || n->gate)) || (p.f.x && !p.x_new.x)) return HBP_ERR_INVALID_ARG;
  if (p.y.x && p.y.x == p.x_new.x) return HBP_ERR_INVALID_ARG;
  for (const Rows& out : {p.x_new, p.y})
    if (!on_itself(out, p.x) || !on_itself(out, p.f)) return HBP_ERR_INVALID_ARG;
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  by_variant(*n, nv, [&](auto t, auto v, auto layer) {
    forward<decltype(t), decltype(v)::value, decltype(layer)::value>(lc, p, n->post != 0);
    return 0;
  });
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}

extern "C" hbp_status hbp_norm_residual_scratch_bytes(int64_t rows, int32_t d, size_t* bytes) {
  if (!bytes) return HBP_ERR_INVALID_ARG;
  if (rows < 0 || d <= 0 || d > kMaxWidth) return HBP_ERR_SHAPE;
  *bytes = partial_bytes(rows, d);
  return HBP_OK;
}

extern "C" hbp_status hbp_norm_residual_backward(const hbp_norm* n, const hbp_rows* d_y, const hbp_rows* d_new, const hbp_rows* x_new, const hbp_rows* f,
                                                 const hbp_rows* x, const hbp_rows* dx, const hbp_rows* df, float* dw_pre, float* dw_post, float* da,
                                                 void* scratch, size_t scratch_bytes, void* cuda_stream) {
  const hbp_status st = check(n);
  if (st != HBP_OK) return st;
  int nv = 1;
  NormParams p = params_of(*n, true, &nv);
  if (!rows_of(*n, d_y, true, &p.d_y) || !rows_of(*n, d_new, true, &p.d_new) || !rows_of(*n, x_new, true, &p.x_new) || !rows_of(*n, f, true, &p.f) ||
      !rows_of(*n, x, true, &p.x) || !rows_of(*n, dx, false, &p.dx) || !rows_of(*n, df, false, &p.df))
    return HBP_ERR_SHAPE;
  p.want_pre = dw_pre != nullptr;
  p.want_post = dw_post != nullptr;
  p.want_gate = da != nullptr;
  const bool post = n->post != 0;
  if ((p.want_post && !post) || (n->rows && ((!p.d_y.x && !p.d_new.x) || (p.d_y.x && !p.x_new.x) || (post && !p.f.x) || (p.want_gate && !p.x.x) ||
                                            (p.want_pre && !p.d_y.x) || (!p.dx.x && !p.df.x && !p.want_pre && !p.want_post && !p.want_gate))))
    return HBP_ERR_INVALID_ARG;
  if (p.dx.x && p.dx.x == p.df.x) return HBP_ERR_INVALID_ARG;
  for (const Rows& out : {p.dx, p.df})
    for (const Rows& in : {p.d_y, p.d_new, p.x_new, p.f, p.x})
      if (!on_itself(out, in)) return HBP_ERR_INVALID_ARG;
  const bool sums = p.want_pre || p.want_post || p.want_gate;
  for (const float* w : {dw_pre, dw_post, da})
    if ((uintptr_t)w & 15u) return HBP_ERR_SHAPE;
  if (sums && n->rows && (!scratch || ((uintptr_t)scratch & 15u) || scratch_bytes < partial_bytes(n->rows, n->d))) return HBP_ERR_WORKSPACE;
  if (!sums && n->rows == 0) return HBP_OK;
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  p.partial = sums ? (float*)scratch : nullptr;
  WeightSums w = {(const float*)scratch, 0, n->d, {dw_pre, dw_post, da}};
  if (n->rows)
    w.blocks = by_variant(*n, nv, [&](auto t, auto v, auto layer) { return backward<decltype(t), decltype(v)::value, decltype(layer)::value>(lc, p, post); });
  if (sums) launch_chained(lc, weight_sums_kernel, dim3((n->d + 127) / 128, 3), 256, 0, 1, w);
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}
