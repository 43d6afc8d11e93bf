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

#include "float_pairs.cuh"
#include "hbp_internal.h"
#include "tc_common.cuh"

namespace hbp {

namespace {

struct Rows {
  const void* x;
  int64_t ld;
  int64_t step;  // from a group's row to its next, in elements
};

struct NormParams {
  int64_t rows;
  int d, per_row, threads;  // vectors a row; threads that hold one
  int stages;  // rows of a group under way
  float eps, scale, inv_d;
  const void *w_post, *gate, *w_pre;
  Rows x, f, x_new, y;                 // forward: x_new and y are written
  Rows d_y, d_new, dx, df;             // backward
  float* partial;                      // [blocks][3][d]: of dw_pre, dw_post, da
  bool want_pre, want_post, want_gate;
};

template <typename T>
struct Channels {
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
// What the warps of a row exchange: two buffers in turn, so that one barrier a sum is enough.
struct Exchange {
  float part[2][kMaxWarps][4];
};

// Sums of K values over the threads of a row, in every one of them.  Rows of more than a warp use a barrier of their own.
template <int K>
__device__ __forceinline__ void row_sum(float (&v)[K], int threads, int group, Exchange& x, int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (threads == 32) return;
  const int warp = threadIdx.x >> 5, warps = threads >> 5;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) x.part[turn][warp][k] = v[k];
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(threads) : "memory");
  // a lane takes a warp's: adding up eight warps' is three times the instructions for every thread
  const int lane = threadIdx.x & 31;
  const float4 q = lane < warps ? *reinterpret_cast<const float4*>(x.part[turn][group * warps + lane]) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const float part[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = part[k];
#pragma unroll
  for (int o = kMaxWarps / 2; o > 0; o >>= 1)
    if (o < warps) {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    }
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = __shfl_sync(0xffffffffu, v[k], 0);
  turn ^= 1;
}

// Vectors of rows on their way: a thread copies its own into its own place of shared memory, so that it waits for nobody to have them and registers
// hold none of them.
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_made() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// A vector of 16 bytes as pairs of floats
template <typename T>
__device__ __forceinline__ void pairs_of(const uint4& r, f32x2 (&p)[8 / sizeof(T)]) {
#pragma unroll
  for (int e = 0; e < (int)(8 / sizeof(T)); ++e) p[e] = widen2(reinterpret_cast<const T*>(&r) + 2 * e);
}
template <typename T>
__device__ __forceinline__ uint4 vector_of(const f32x2 (&p)[8 / sizeof(T)]) {
  uint4 r;
#pragma unroll
  for (int e = 0; e < (int)(8 / sizeof(T)); ++e) narrow2(p[e], reinterpret_cast<T*>(&r) + 2 * e);
  return r;
}
__device__ __forceinline__ float total(f32x2 v) {
  const float2 f = floats_of(v);
  return f.x + f.y;
}

__device__ __forceinline__ void copies_wait_but(int left) {
  if (left >= 3) copies_wait<3>();
  else if (left == 2) copies_wait<2>();
  else if (left == 1) copies_wait<1>();
  else copies_wait<0>();
}

constexpr int kMostStages = 4;  // rows of a group under way

// a weight's vector of channels, or ones
template <typename T>
__device__ __forceinline__ void weights(const void* w, int c, f32x2 (&p)[8 / sizeof(T)]) {
  if (w) {
    pairs_of<T>(*reinterpret_cast<const uint4*>((const T*)w + c), p);
  } else {
#pragma unroll
    for (int e = 0; e < (int)(8 / sizeof(T)); ++e) p[e] = both(1.0f);
  }
}

// Less the mean (0 without kLayer) and 1 / sqrt(mean square + eps) of a row's values.
template <int NV, int H, bool kLayer>
__device__ __forceinline__ float2 statistics(const f32x2 (&v)[NV][H], const bool (&in)[NV], const NormParams& p, int group, Exchange& buf, int& turn) {
  float m[1] = {0.0f};
  if (kLayer) {
    f32x2 s = both(0.0f);
#pragma unroll
    for (int u = 0; u < NV; ++u)
      if (in[u])
#pragma unroll
        for (int e = 0; e < H; ++e) s = add2(s, v[u][e]);
    m[0] = total(s);
    row_sum(m, p.threads, group, buf, turn);
    m[0] *= -p.inv_d;
  }
  f32x2 s = both(0.0f);
  const f32x2 less = both(m[0]);
#pragma unroll
  for (int u = 0; u < NV; ++u)
    if (in[u])
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const f32x2 c = kLayer ? add2(v[u][e], less) : v[u][e];
        s = fma2(c, c, s);
      }
  float q[1] = {total(s)};
  row_sum(q, p.threads, group, buf, turn);
  return make_float2(m[0], 1.0f / sqrtf(fmaf(q[0], p.inv_d, p.eps)));
}

// ------------------------------------------------------------------------------------------- forward
// float: a group of threads a row, loaded as it comes, near a copy's rate (16384 x 2048, both norms 92 us of 82 for the bytes; copied ahead by groups that walk over
// the rows, and in pairs of floats, as bf16 below, 107).
__device__ __forceinline__ uint4 row_vector(const Rows& r, int64_t row, int c) { return *reinterpret_cast<const uint4*>((const float*)r.x + row * r.ld + c); }
// weights of one vector of channels, or ones
__device__ __forceinline__ void row_weights(const void* w, int c, float* f) {
  constexpr int V = Channels<float>::V;
  if (w) {
    Channels<float>::widen(*reinterpret_cast<const uint4*>((const float*)w + c), f);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = 1.0f;
  }
}

// Mean (0 without kLayer) and 1 / sqrt(mean square + eps) of a row's values.  Channels beyond d hold zeros.
template <int NV, int V, bool kLayer>
__device__ __forceinline__ float2 row_statistics(const float (&v)[NV][V], const bool (&in)[NV], const NormParams& p, int group, Exchange& buf, int& turn) {
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

// kBlock: the block's output and the update, else only the norm of the stream.
template <int NV, bool kLayer, bool kBlock, bool kPost>
__global__ void __launch_bounds__(512) norm_row_kernel(const NormParams p) {
  constexpr int V = Channels<float>::V;
  __shared__ __align__(16) Exchange buf;
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
      x[u] = row_vector(p.x, row, c);
      if (kBlock) f[u] = row_vector(p.f, row, c);
    }
  }
  if (kBlock) {
    float2 s = make_float2(0.0f, 1.0f);
#pragma unroll
    for (int u = 0; u < NV; ++u) Channels<float>::widen(f[u], v[u]);
    if (kPost) s = row_statistics<NV, V, kLayer>(v, in, p, group, buf, turn);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * p.threads) * V;
      if (!in[u]) continue;
      float w[V], g[V], xf[V];
      row_weights(kPost ? p.w_post : nullptr, c, w);
      row_weights(p.gate, c, g);
      Channels<float>::widen(x[u], xf);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = kPost ? (v[u][e] - s.x) * s.y * w[e] : v[u][e];
        v[u][e] = fmaf(p.scale, h, g[e] * xf[e]);
      }
      x[u] = Channels<float>::narrow(v[u]);
      *reinterpret_cast<uint4*>((float*)p.x_new.x + row * p.x_new.ld + c) = x[u];
    }
    if (!p.y.x) return;
  }
#pragma unroll
  for (int u = 0; u < NV; ++u) Channels<float>::widen(x[u], v[u]);  // the stream as it is stored
  const float2 s = row_statistics<NV, V, kLayer>(v, in, p, group, buf, turn);
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int c = (t + u * p.threads) * V;
    if (!in[u]) continue;
    float w[V];
    row_weights(p.w_pre, c, w);
#pragma unroll
    for (int e = 0; e < V; ++e) v[u][e] = (v[u][e] - s.x) * s.y * w[e];
    *reinterpret_cast<uint4*>((float*)p.y.x + row * p.y.ld + c) = Channels<float>::narrow(v[u]);
  }
}

// bf16: groups of 32 to 512 threads walk over the rows, a grid apart.  (A block for every eight rows of 768 channels, which read them when it
// came, had both norms' 16384 rows in 31 us, so 25; for every four, in 39: blocks cost that much to come and go.)
template <int NV, bool kLayer, bool kBlock, bool kPost>
__global__ void __launch_bounds__(512) norm_forward_kernel(const NormParams p) {
  typedef bf16 T;
  constexpr int V = Channels<T>::V, H = V / 2;
  __shared__ __align__(16) Exchange buf;
  extern __shared__ float4 dynamic[];  // [stages][x, f][NV][threads of the block]
  chain_next();
  chain_wait();
  int turn = 0;
  const int groups = blockDim.x / p.threads, group = threadIdx.x / p.threads, t = threadIdx.x - group * p.threads;
  const uint32_t slab = NV * blockDim.x * 16, row_bytes = (kBlock ? 2 : 1) * slab, mine = tc::smem_u32(dynamic) + threadIdx.x * 16;
  const uint32_t end = mine + p.stages * row_bytes;
  bool in[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) in[u] = (t + u * p.threads) * V < p.d;
  const int64_t step = (int64_t)gridDim.x * groups, first = (int64_t)blockIdx.x * groups + group;
  auto at = [&](const Rows& r) { return (const T*)r.x + first * r.ld + t * V; };
  const T *a_x = at(p.x), *a_f = at(p.f);
  T *o_new = (T*)at(p.x_new), *o_y = (T*)at(p.y);
  int64_t asked = first;
  uint32_t to = mine, from = mine;
  auto ask = [&]() {
    if (asked < p.rows) {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        if (!in[u]) continue;
        const uint32_t place = to + u * blockDim.x * 16;
        copy16(place, a_x + u * p.threads * V);
        if (kBlock) copy16(place + slab, a_f + u * p.threads * V);
      }
      a_x += p.x.step;
      a_f += p.f.step;
      asked += step;
    }
    to = to + row_bytes == end ? mine : to + row_bytes;
    copies_made();
  };
  for (int s = 0; s < p.stages - 1; ++s) ask();
  for (int64_t row = first; row < p.rows; row += step) {
    ask();  // into the place of the row before, which this thread is done with
    copies_wait_but(p.stages - 1);
    const uint32_t here = from;
    from = from + row_bytes == end ? mine : from + row_bytes;
    f32x2 v[NV][H];
    if (kBlock) {
      float2 s = make_float2(0.0f, 1.0f);
#pragma unroll
      for (int u = 0; u < NV; ++u)
        if (in[u]) pairs_of<T>(tc::ld_shared16(here + slab + u * blockDim.x * 16), v[u]);
      if (kPost) s = statistics<NV, H, kLayer>(v, in, p, group, buf, turn);
      const f32x2 less = both(s.x), r = both(s.y), scale = both(p.scale);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        if (!in[u]) continue;
        const int c = (t + u * p.threads) * V;
        f32x2 x[H], w[H];
        if (kPost) {
          weights<T>(p.w_post, c, w);
#pragma unroll
          for (int e = 0; e < H; ++e) v[u][e] = mul2(mul2(kLayer ? add2(v[u][e], less) : v[u][e], r), w[e]);
        }
        pairs_of<T>(tc::ld_shared16(here + u * blockDim.x * 16), x);
        if (p.gate) {
          weights<T>(p.gate, c, w);
#pragma unroll
          for (int e = 0; e < H; ++e) x[e] = mul2(x[e], w[e]);
        }
#pragma unroll
        for (int e = 0; e < H; ++e) v[u][e] = fma2(v[u][e], scale, x[e]);
        const uint4 stored = vector_of<T>(v[u]);
        *reinterpret_cast<uint4*>(o_new + u * p.threads * V) = stored;
        pairs_of<T>(stored, v[u]);  // the stream as it is stored
      }
      o_new += p.x_new.step;
      if (!p.y.x) continue;
    } else {
#pragma unroll
      for (int u = 0; u < NV; ++u)
        if (in[u]) pairs_of<T>(tc::ld_shared16(here + u * blockDim.x * 16), v[u]);
    }
    const float2 s = statistics<NV, H, kLayer>(v, in, p, group, buf, turn);
    const f32x2 less = both(s.x), r = both(s.y);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!in[u]) continue;
      f32x2 w[H];
      weights<T>(p.w_pre, (t + u * p.threads) * V, w);
#pragma unroll
      for (int e = 0; e < H; ++e) v[u][e] = mul2(mul2(kLayer ? add2(v[u][e], less) : v[u][e], r), w[e]);
      *reinterpret_cast<uint4*>(o_y + u * p.threads * V) = vector_of<T>(v[u]);
    }
    o_y += p.y.step;
  }
}

// ------------------------------------------------------------------------------------------- backward
// Whether threads of few registers keep the weights in shared memory (five floats of 8192 channels leave no room there)
template <typename T>
constexpr bool kShares = sizeof(T) == 2;

// A vector that is used more than once: as floats, or as it came where registers are short (two vectors a thread and more).
template <typename T, bool kFloats>
struct Kept {
  static constexpr int H = 8 / sizeof(T);
  f32x2 v[kFloats ? H : 1];
  uint4 r;
  __device__ __forceinline__ void set(const uint4& raw) {
    if constexpr (kFloats) pairs_of<T>(raw, v);
    else r = raw;
  }
  __device__ __forceinline__ void get(f32x2 (&p)[H]) const {
    if constexpr (kFloats) {
#pragma unroll
      for (int e = 0; e < H; ++e) p[e] = v[e];
    } else {
      pairs_of<T>(r, p);
    }
  }
};

// Rows are on their way up to three before they are used, as in the forward pass (16384 x 2048 bf16, both norms and a gate: loaded when they are used 171 us, ahead 118,
// where the bytes take 72).  Then it is the instructions, 76 a channel then and 59 now, and the way of a row through its sums, two or three that wait for all of its warps: 16
// channels a thread instead of 8 halve what a row costs beside its channels, pointers walk along with the rows, lanes share the warps' sums; and four rows are
// under way an SM where weights of bf16 rows are read from shared memory again instead of holding registers (208 of these: 122 us): 103 us.  float: values that are
// used again stay in registers, 6.2 TB/s.  Groups walk over the rows, a grid apart.
// kFew: 128 registers a thread, for rows of more than 256 threads, or twice the rows under way.  kAll: both gradients arrive and both are wanted.
template <typename T, int NV, bool kLayer, bool kPost, bool kFew, bool kAll>
__global__ void __launch_bounds__(kFew ? 512 : 256) norm_backward_kernel(const NormParams p) {
  constexpr int V = Channels<T>::V, H = V / 2;
  constexpr bool kFloats = !kFew, kShared = kShares<T> && kFew;
  typedef Kept<T, kFloats> Vector;
  __shared__ __align__(16) Exchange buf;
  extern __shared__ float4 dynamic[];  // [stages][tensors][NV][threads of the block]; at the end [3][d], the sums of the block's groups
  chain_next();
  chain_wait();
  int turn = 0;
  const int groups = blockDim.x / p.threads, group = threadIdx.x / p.threads, t = threadIdx.x - group * p.threads;
  const bool has_y = kAll || p.d_y.x, has_new = kAll || p.d_new.x;
  // the tensors' places in a stage
  const int at_new = has_y ? 2 : 0, at_f = at_new + has_new, at_x = at_f + kPost, tensors = at_x + p.want_gate;
  const uint32_t slab = NV * blockDim.x * 16, row_bytes = tensors * slab, mine = tc::smem_u32(dynamic) + threadIdx.x * 16;
  f32x2 dw_pre[NV][H], dw_post[NV][H], da[NV][H];
  Vector w_pre[NV], w_post[NV], gate[NV];  // (kShared: in shared memory)
  const uint32_t weights_at = mine + p.stages * row_bytes;
  bool in[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int c = (t + u * p.threads) * V;
    in[u] = c < p.d;
#pragma unroll
    for (int e = 0; e < H; ++e) dw_pre[u][e] = dw_post[u][e] = da[u][e] = both(0.0f);
    float ones[V];
#pragma unroll
    for (int e = 0; e < V; ++e) ones[e] = 1.0f;
    auto keep = [&](Vector& v, const void* w, int which) {
      const uint4 raw = in[u] && w ? *reinterpret_cast<const uint4*>((const T*)w + c) : Channels<T>::narrow(ones);
      if constexpr (!kShared) v.set(raw);
      else tc::st_shared16(weights_at + (which * NV + u) * blockDim.x * 16, raw);
    };
    keep(w_pre[u], p.w_pre, 0);
    if (kPost) keep(w_post[u], p.w_post, 1);
    keep(gate[u], p.gate, 2);
  }
  auto weight = [&](const Vector& v, int which, int u, f32x2 (&w)[H]) {
    if constexpr (!kShared) v.get(w);
    else pairs_of<T>(tc::ld_shared16(weights_at + (which * NV + u) * blockDim.x * 16), w);
  };
  const int64_t step = (int64_t)gridDim.x * groups, first = (int64_t)blockIdx.x * groups + group;
  // where this thread's first vector is: of the row to ask for next, and of the outputs' row
  auto at = [&](const Rows& r) { return (const T*)r.x + first * r.ld + t * V; };
  const T *a_dy = at(p.d_y), *a_xn = at(p.x_new), *a_dn = at(p.d_new), *a_f = at(p.f), *a_x = at(p.x);
  T *o_dx = (T*)at(p.dx), *o_df = (T*)at(p.df);
  int64_t asked = first;
  uint32_t to = mine;
  const uint32_t end = mine + p.stages * row_bytes;
  auto ask = [&]() {
    if (asked < p.rows) {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        if (!in[u]) continue;
        const int c = u * p.threads * V;
        uint32_t place = to + u * blockDim.x * 16;
        auto one = [&](const T* from) {
          copy16(place, from + c);
          place += slab;
        };
        if (has_y) {
          one(a_dy);
          one(a_xn);
        }
        if (has_new) one(a_dn);
        if (kPost) one(a_f);
        if (p.want_gate) one(a_x);
      }
      a_dy += p.d_y.step;
      a_xn += p.x_new.step;
      a_dn += p.d_new.step;
      a_f += p.f.step;
      a_x += p.x.step;
      asked += step;
    }
    to = to + row_bytes == end ? mine : to + row_bytes;
    copies_made();
  };
  for (int s = 0; s < p.stages - 1; ++s) ask();
  uint32_t from = mine;
  for (int64_t row = first; row < p.rows; row += step) {
    ask();  // into the place of the row before, which this thread is done with
    copies_wait_but(p.stages - 1);
    const uint32_t here = from;
    from = from + row_bytes == end ? mine : from + row_bytes;
    auto held = [&](int i, int u) { return tc::ld_shared16(here + i * slab + u * blockDim.x * 16); };
    Vector xn[NV], f[NV], a[NV];  // a = dy * w_pre
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!in[u]) continue;
      if (has_y) xn[u].set(held(1, u));
      if (kPost) f[u].set(held(at_f, u));
    }
    // means of the stream and the block's output
    float mean[2] = {0.0f, 0.0f};
    if (kLayer) {
      f32x2 m0 = both(0.0f), m1 = both(0.0f), v[H];
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        if (!in[u]) continue;
        if (has_y) {
          xn[u].get(v);
#pragma unroll
          for (int e = 0; e < H; ++e) m0 = add2(m0, v[e]);
        }
        if (kPost) {
          f[u].get(v);
#pragma unroll
          for (int e = 0; e < H; ++e) m1 = add2(m1, v[e]);
        }
      }
      mean[0] = total(m0);
      mean[1] = total(m1);
      row_sum(mean, p.threads, group, buf, turn);
      mean[0] *= p.inv_d;
      mean[1] *= p.inv_d;
    }
    const f32x2 less = both(-mean[0]), less_f = both(-mean[1]);
    // sums of squares around them, of a times the centred stream, and of a
    constexpr int Q = kLayer ? 4 : kPost ? 3 : 2;
    float q[4];
    {
      f32x2 s[4] = {both(0.0f), both(0.0f), both(0.0f), both(0.0f)};
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        f32x2 v[H], w[H], g[H];
        if (!in[u]) continue;
        if (has_y) {
          pairs_of<T>(held(0, u), g);
          xn[u].get(v);
          weight(w_pre[u], 0, u, w);
#pragma unroll
          for (int e = 0; e < H; ++e) {
            const f32x2 cx = kLayer ? add2(v[e], less) : v[e], aw = mul2(g[e], w[e]);
            if constexpr (kFloats) a[u].v[e] = aw;
            s[0] = fma2(cx, cx, s[0]);
            s[1] = fma2(aw, cx, s[1]);
            if (kLayer) s[3] = add2(s[3], aw);
          }
        }
        if (kPost) {
          f[u].get(v);
#pragma unroll
          for (int e = 0; e < H; ++e) {
            const f32x2 cf = kLayer ? add2(v[e], less_f) : v[e];
            s[2] = fma2(cf, cf, s[2]);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) q[k] = total(s[k]);
    }
    row_sum(*reinterpret_cast<float(*)[Q]>(q), p.threads, group, buf, turn);
    const float r = 1.0f / sqrtf(fmaf(q[0], p.inv_d, p.eps)), along = q[1] * r * p.inv_d, flat = kLayer ? q[3] * p.inv_d : 0.0f;
    const float rf = kPost ? 1.0f / sqrtf(fmaf(q[2], p.inv_d, p.eps)) : 1.0f;
    const f32x2 r2 = both(r), rf2 = both(rf), along2 = both(-along), flat2 = both(-flat), scale = both(p.scale);
    // the gradient of the new stream; what it gives
    f32x2 g[NV][H], b0 = both(0.0f), b1 = both(0.0f);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!in[u]) continue;
      f32x2 v[H], w[H], y[H];
      if (has_new) {
        pairs_of<T>(held(at_new, u), g[u]);
      } else {
#pragma unroll
        for (int e = 0; e < H; ++e) g[u][e] = both(0.0f);
      }
      if (has_y) {
        pairs_of<T>(held(0, u), y);
        xn[u].get(v);
        if constexpr (!kFloats) weight(w_pre[u], 0, u, w);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          const f32x2 xhat = mul2(kLayer ? add2(v[e], less) : v[e], r2);
          dw_pre[u][e] = fma2(y[e], xhat, dw_pre[u][e]);
          f32x2 aw;
          if constexpr (kFloats) aw = a[u].v[e];
          else aw = mul2(y[e], w[e]);
          if (kLayer) aw = add2(aw, flat2);
          g[u][e] = fma2(fma2(xhat, along2, aw), r2, g[u][e]);
        }
      }
      if (p.want_gate) {
        pairs_of<T>(held(at_x, u), v);
#pragma unroll
        for (int e = 0; e < H; ++e) da[u][e] = fma2(g[u][e], v[e], da[u][e]);
      }
      if (kAll || p.dx.x) {
        weight(gate[u], 2, u, w);
#pragma unroll
        for (int e = 0; e < H; ++e) v[e] = mul2(g[u][e], w[e]);
        *reinterpret_cast<uint4*>(o_dx + u * p.threads * V) = vector_of<T>(v);
      }
#pragma unroll
      for (int e = 0; e < H; ++e) g[u][e] = mul2(g[u][e], scale);  // of h
      if (kPost) {
        f[u].get(v);
        weight(w_post[u], 1, u, w);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          const f32x2 fhat = mul2(kLayer ? add2(v[e], less_f) : v[e], rf2);
          dw_post[u][e] = fma2(g[u][e], fhat, dw_post[u][e]);
          g[u][e] = mul2(g[u][e], w[e]);
          b0 = fma2(g[u][e], fhat, b0);
          if (kLayer) b1 = add2(b1, g[u][e]);
        }
      }
    }
    o_dx += p.dx.step;
    if (!kAll && !p.df.x) continue;
    float b[2] = {total(b0), total(b1)};
    if (kPost) row_sum(*reinterpret_cast<float(*)[kLayer ? 2 : 1]>(b), p.threads, group, buf, turn);
    const f32x2 along_f = both(-b[0] * p.inv_d), flat_f = both(kLayer ? -b[1] * p.inv_d : 0.0f);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!in[u]) continue;
      if (kPost) {
        f32x2 v[H];
        f[u].get(v);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          const f32x2 fhat = mul2(kLayer ? add2(v[e], less_f) : v[e], rf2);
          g[u][e] = mul2(fma2(fhat, along_f, kLayer ? add2(g[u][e], flat_f) : g[u][e]), rf2);
        }
      }
      *reinterpret_cast<uint4*>(o_df + u * p.threads * V) = vector_of<T>(g[u]);
    }
    o_df += p.df.step;
  }
  if (!p.partial) return;
  copies_wait<0>();
  __syncthreads();  // the stages are done with
  float* sums = reinterpret_cast<float*>(dynamic);
  for (int k = 0; k < groups; ++k) {  // the groups' sums, one after the other
    if (k == group) {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int c = (t + u * p.threads) * V;
        if (!in[u]) continue;
#pragma unroll
        for (int e = 0; e < H; ++e) {
          auto put = [&](int which, f32x2 v) {
            f32x2* to = reinterpret_cast<f32x2*>(sums + which * p.d + c + 2 * e);
            *to = k ? add2(*to, v) : v;
          };
          put(0, dw_pre[u][e]);
          put(1, dw_post[u][e]);
          put(2, da[u][e]);
        }
      }
    }
    __syncthreads();
  }
  float* out = p.partial + (int64_t)blockIdx.x * 3 * p.d;
  for (int i = threadIdx.x * 4; i < 3 * p.d; i += blockDim.x * 4) {
    const int k = i / p.d;
    if (k == 0 ? p.want_pre : k == 1 ? p.want_post : p.want_gate) *reinterpret_cast<float4*>(out + i) = *reinterpret_cast<const float4*>(sums + i);
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
constexpr int kMostShared = 224 << 10;

// Vectors a thread holds, and threads a row (whole warps).  Forward: rows of up to 128 vectors are a warp's: no barriers.  Backward: 8 to 16
// channels, as threads hold three sums a channel too.
void split_of(int per_row, bool backward, bool f32, int* nv, int* threads) {
  if (backward) *nv = per_row <= 32 ? 1 : f32 ? (per_row <= 512 ? 2 : 4) : 2;
  else *nv = per_row <= 32 ? 1 : per_row <= 64 ? 2 : per_row <= 128 ? 4 : per_row <= 1024 ? 2 : 4;
  *threads = ((per_row + *nv - 1) / *nv + 31) / 32 * 32;
}

// Blocks of `threads` threads that an SM runs at once, by the kernel's registers (looked up once, as its leave for the widest rows' shared
// memory is asked for); 0: an error.
int blocks_at_once(const void* kernel, int& registers, int threads) {
  if (registers == 0) {
    cudaFuncAttributes a;
    if (cudaFuncGetAttributes(&a, kernel) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared) != cudaSuccess) {
      cudaGetLastError();
      return 0;
    }
    registers = (a.numRegs + 7) / 8 * 8;
  }
  const int by_regs = 65536 / registers / threads, by_threads = 2048 / threads, n = by_regs < by_threads ? by_regs : by_threads;
  return n > 0 ? n : 1;
}

// Dynamic shared memory of each of so many blocks on an SM
size_t room(int blocks) { return (size_t)(226 << 10) / blocks - 2048; }

template <typename T, int NV, bool kLayer>
void forward(Launcher& lc, NormParams& p, bool post) {
  const int groups = p.threads >= 256 ? 1 : 256 / p.threads, kind = !p.f.x ? 0 : post ? 2 : 1;
  const int64_t wanted = (p.rows + groups - 1) / groups;
  if constexpr (sizeof(T) == 4) {
    auto kernel = kind == 0 ? norm_row_kernel<NV, kLayer, false, false> : kind == 2 ? norm_row_kernel<NV, kLayer, true, true> : norm_row_kernel<NV, kLayer, true, false>;
    launch_chained(lc, kernel, dim3((unsigned)wanted), groups * p.threads, 0, 1, p);
  } else {
    auto kernel = kind == 0 ? norm_forward_kernel<NV, kLayer, false, false>
                            : kind == 2 ? norm_forward_kernel<NV, kLayer, true, true> : norm_forward_kernel<NV, kLayer, true, false>;
    static PerDevice<int> registers[3];
    int per_sm = blocks_at_once((const void*)kernel, registers[kind].here(), groups * p.threads);
    if (per_sm == 0) {
      lc.err = cudaErrorInvalidValue;
      return;
    }
    if (per_sm > 4) per_sm = 4;  // (65536 x 256: 22 us, five 25)
    // two rows under way a group, if need be with fewer blocks
    const size_t stage = (size_t)(p.f.x ? 2 : 1) * NV * groups * p.threads * 16;
    while (per_sm > 1 && room(per_sm) < 2 * stage) --per_sm;
    const size_t fits = room(per_sm) / stage;  // (32 KB are the most that a row takes)
    p.stages = (int)(fits < kMostStages ? fits : kMostStages);
    const int64_t most = (int64_t)per_sm * tc::sm_count(), blocks = wanted < most ? wanted : most;
    for (Rows* r : {&p.x, &p.f, &p.x_new, &p.y}) r->step = r->ld * blocks * groups;
    launch_chained(lc, kernel, dim3((unsigned)blocks), groups * p.threads, p.stages * stage, 1, p);
  }
}

constexpr int kMostBlocks = 4;     // an SM, backward: each leaves 12 d bytes for the second launch
constexpr int kMostPartials = 640;  // and all of them together

template <typename T, int NV, bool kLayer>
int backward(Launcher& lc, NormParams& p, bool post) {
  const int groups = p.threads >= 256 ? 1 : 256 / p.threads;
  const bool few = sizeof(T) == 2 ? NV == 2 : p.threads > 256, all = p.d_y.x && p.d_new.x && p.dx.x && p.df.x;
  auto pick = [&](auto of_few) {
    constexpr bool kFew = decltype(of_few)::value;
    return post ? (all ? norm_backward_kernel<T, NV, kLayer, true, kFew, true> : norm_backward_kernel<T, NV, kLayer, true, kFew, false>)
                : (all ? norm_backward_kernel<T, NV, kLayer, false, kFew, true> : norm_backward_kernel<T, NV, kLayer, false, kFew, false>);
  };
  void (*kernel)(NormParams);
  if constexpr (sizeof(T) == 4 && NV == 4) kernel = few ? pick(std::true_type()) : pick(std::false_type());
  else kernel = pick(std::integral_constant<bool, sizeof(T) == 2 && NV == 2>());
  static PerDevice<int> registers[8];
  int per_sm = blocks_at_once((const void*)kernel, registers[4 * all + 2 * few + post].here(), groups * p.threads);
  if (per_sm == 0) {
    lc.err = cudaErrorInvalidValue;
    return 0;
  }
  if (per_sm > kMostBlocks) per_sm = kMostBlocks;
  // as many rows under way as the blocks of an SM have shared memory for; fewer blocks where not even one fits
  const int tensors = (p.d_y.x ? 2 : 0) + (p.d_new.x != nullptr) + post + p.want_gate;
  const size_t stage = (size_t)tensors * NV * groups * p.threads * 16, sums = p.partial ? (size_t)3 * p.d * 4 : 0;
  const size_t weights = few && kShares<T> ? (size_t)3 * NV * groups * p.threads * 16 : 0;
  while (per_sm > 1 && (room(per_sm) < stage + weights || room(per_sm) < sums)) --per_sm;
  const size_t fits = (room(per_sm) - weights) / stage;
  p.stages = (int)(fits < kMostStages ? fits : kMostStages);
  if (p.stages < 1) {  // (5 * 32 KB are the most that a row takes)
    lc.err = cudaErrorInvalidValue;
    return 0;
  }
  const size_t rows = p.stages * stage + weights, smem = rows > sums ? rows : sums;
  const int64_t wanted = (p.rows + groups - 1) / groups, at_once = (int64_t)per_sm * tc::sm_count(), most = at_once < kMostPartials ? at_once : kMostPartials;
  const int blocks = (int)(wanted < most ? wanted : most);
  for (Rows* r : {&p.x, &p.f, &p.x_new, &p.d_y, &p.d_new, &p.dx, &p.df}) r->step = r->ld * blocks * groups;
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
  *r = {nullptr, 0, 0};
  if (!t || !t->x) return true;
  const int v = n.dtype == HBP_F32 ? 4 : 8;
  if (((uintptr_t)t->x & 15u) || t->stride % v || (t->stride < n.d && !(input && t->stride == 0) && n.rows > 1)) return false;
  *r = {t->x, t->stride, 0};
  return true;
}
// an output that lies on an input has to lie on it row by row
bool on_itself(const Rows& out, const Rows& in) { return !out.x || out.x != in.x || out.ld == in.ld; }

NormParams params_of(const hbp_norm& n, bool backward, int* nv) {
  NormParams p = {};
  p.rows = n.rows;
  p.d = n.d;
  p.per_row = n.d / (n.dtype == HBP_F32 ? 4 : 8);
  split_of(p.per_row, backward, n.dtype == HBP_F32, nv, &p.threads);
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
    w.blocks = by_variant(*n, nv, [&](auto t, auto v, auto layer) {
      if constexpr (sizeof(t) == 2 && decltype(v)::value == 4) return 0;  // (rows of bf16 have 1024 vectors at most)
      else return backward<decltype(t), decltype(v)::value, decltype(layer)::value>(lc, p, post);
    });
  if (sums) launch_chained(lc, weight_sums_kernel, dim3((n->d + 127) / 128, 3), 256, 0, 1, w);
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}
