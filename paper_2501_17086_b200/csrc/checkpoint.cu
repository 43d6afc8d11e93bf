// Activations in 8 bits and GELU's backward pass from them (hbp_checkpoint_*).
//
// A group of 32 channels shares a power of two, the smallest 2^e with max |x| <= 127 * 2^e, found from the bits of the
// largest magnitude (the maximum is taken over bit patterns, so that infinities and NaN come out on top of it).  Powers of two
// make both directions exact but for the one rounding to a whole number, and every stored value a bf16 number.
//
// HBM-bound: a thread moves kBatch vectors of 16 bytes, all loads before the first use.  A group is 4 (bf16) or 8 (float)
// neighbouring lanes, its maximum 2 or 3 shuffles.  bf16 values leave 27 instruction slots a value before GELU costs more than
// its bytes, and erff alone takes that many: there erfc is formed by formula 7.1.26 of Abramowitz and Stegun, "Handbook of
// Mathematical Functions" (absolute error 1.5e-7; half a step of bf16 is 2^-9 of the value), whose exponential is GELU's
// density as well: one ex2, one reciprocal and some 14 other instructions for gelu and gelu' together.
#include "hbp_internal.h"

namespace hbp {

namespace {

constexpr int kThreads = 256, kBatch = 4;
constexpr int kGroup = 32;

enum Work { kStore = 0, kLoad = 1, kGelu = 2, kGeluBackward = 3 };

struct CheckpointParams {
  int64_t rows;
  int d, groups;
  int64_t chunks;  // vectors of all rows, those of a row padded to whole groups
  int per_row;     // of them in a row
  const void* x;   // x, z or d_act
  void* y;         // x (load), act (gelu), dz
  void* act;       // gelu(z8) of the backward pass, or nullptr
  int64_t ldx, ldy, lda;
  int8_t* codes;
  uint8_t* scales;
};

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// gelu(z) and gelu'(z); every rounding is written out, so that no call's other outputs change them
__device__ __forceinline__ void gelu_both(float z, float& act, float& slope, float) {
  const float phi = fmaf(0.5f, erff(__fmul_rn(z, 0.70710678118654752440f)), 0.5f);
  act = __fmul_rn(z, phi);
  slope = fmaf(__fmul_rn(z, expf(__fmul_rn(__fmul_rn(-0.5f, z), z))), 0.39894228040143267794f, phi);
}
__device__ __forceinline__ void gelu_both(float z, float& act, float& slope, bf16) {
  const float a = fabsf(z);
  float e, t;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(__fmul_rn(z, z), -0.72134752044448170368f)));      // e^(-z^2 / 2)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(a, 0.23164188f, 1.0f)));            // 1 / (1 + p |z| / sqrt 2)
  // the formula's coefficients over two: half of erfc(|z| / sqrt 2)
  float q = fmaf(t, 0.5307027145f, -0.7265760135f);
  q = fmaf(q, t, 0.7107068705f);
  q = fmaf(q, t, -0.142248368f);
  q = fmaf(q, t, 0.127414796f);
  const float tail = __fmul_rn(__fmul_rn(q, t), e);
  const float phi = z < 0.0f ? tail : __fsub_rn(1.0f, tail);
  act = __fmul_rn(z, phi);
  slope = fmaf(__fmul_rn(z, e), 0.39894228040143267794f, phi);
}

// e + 127 of a group whose largest magnitude has these bits; 255 where it is not finite
__device__ __forceinline__ uint32_t scale_of(uint32_t amax) {
  if (amax >= 0x7f800000u) return 255u;
  // 1.f * 2^(E - 127) <= 127 * 2^e: e = E - 133, one more where 1.f > 127 / 64
  const int s = (int)(amax >> 23) - 6 + ((amax & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return s < 1 ? 1u : (uint32_t)s;
}
constexpr uint32_t kLargestScale = 249;  // steps of 2^122, of which 64 are 2^128 and no float
// 2^e; a code times this is the stored value (a group that was not finite: NaN)
__device__ __forceinline__ float step_of(uint32_t s) { return s == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(s << 23); }
// 2^-e
__device__ __forceinline__ float inverse_of(uint32_t s) { return __uint_as_float((254u - s) << 23); }

// kFlat: rows are whole groups without gaps: one run of chunks
template <typename T, int W, bool kFlat>
__global__ void __launch_bounds__(kThreads) checkpoint_kernel(const CheckpointParams p) {
  constexpr int V = 16 / (int)sizeof(T), kLanes = kGroup / V;
  using VT = Vec<T, V>;
  using VC = Vec<int8_t, V>;
  VT x[kBatch];
  VC code[kBatch];
  uint32_t scale[kBatch];
  int64_t row[kBatch];
  int col[kBatch];
  bool in[kBatch];
  const int64_t base = (int64_t)blockIdx.x * (kThreads * kBatch) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const int64_t i = base + u * kThreads;
    if (kFlat) {
      row[u] = 0;
      in[u] = i < p.chunks;
    } else {
      row[u] = i / p.per_row;
      col[u] = (int)(i - row[u] * p.per_row) * V;
      in[u] = i < p.chunks && col[u] < p.d;
    }
    if (in[u]) {
      if (W != kLoad) x[u] = *reinterpret_cast<const VT*>((const T*)p.x + (kFlat ? i * V : row[u] * p.ldx + col[u]));
      if (W == kLoad || W == kGeluBackward) {
        code[u] = *reinterpret_cast<const VC*>(p.codes + (kFlat ? i * V : row[u] * p.d + col[u]));
        scale[u] = p.scales[kFlat ? i / kLanes : row[u] * p.groups + col[u] / kGroup];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const int64_t i = base + u * kThreads;
    const int64_t at_y = kFlat ? i * V : row[u] * p.ldy + col[u];
    if (W == kStore || W == kGelu) {
      uint32_t amax = 0;
      if (in[u]) {
#pragma unroll
        for (int e = 0; e < V; ++e) amax = max(amax, __float_as_uint(to_f(x[u].v[e])) & 0x7fffffffu);
      }
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      if (!in[u]) continue;
      const uint32_t s = scale_of(amax);
      const float inv = s == 255u ? 0.0f : inverse_of(s);
#pragma unroll
      for (int e = 0; e < V; ++e) code[u].v[e] = (int8_t)(s == 255u ? 0 : __float2int_rn(to_f(x[u].v[e]) * inv));
      if (s == kLargestScale) {
#pragma unroll
        for (int e = 0; e < V; ++e) code[u].v[e] = max(-63, min(63, (int)code[u].v[e]));
      }
      *reinterpret_cast<VC*>(p.codes + (kFlat ? i * V : row[u] * p.d + col[u])) = code[u];
      if (i % kLanes == 0) p.scales[kFlat ? i / kLanes : row[u] * p.groups + col[u] / kGroup] = (uint8_t)s;
      if (W == kGelu) {
        VT y;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float act, slope;
          gelu_both(to_f(x[u].v[e]), act, slope, T());
          y.v[e] = from_f<T>(act);
        }
        *reinterpret_cast<VT*>((T*)p.y + at_y) = y;
      }
    } else if (in[u]) {
      const float step = step_of(scale[u]);
      VT y, a;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float z = (float)code[u].v[e] * step;
        if (W == kLoad) {
          y.v[e] = from_f<T>(z);
        } else {
          float act, slope;
          gelu_both(z, act, slope, T());
          y.v[e] = from_f<T>(to_f(x[u].v[e]) * slope);
          a.v[e] = from_f<T>(act);
        }
      }
      *reinterpret_cast<VT*>((T*)p.y + at_y) = y;
      if (W == kGeluBackward && p.act) *reinterpret_cast<VT*>((T*)p.act + (kFlat ? i * V : row[u] * p.lda + col[u])) = a;
    }
  }
}

template <typename T, int W>
void launch(Launcher& lc, CheckpointParams& p) {
  constexpr int V = 16 / (int)sizeof(T);
  p.groups = (p.d + kGroup - 1) / kGroup;
  p.per_row = p.groups * (kGroup / V);
  p.chunks = p.rows * p.per_row;
  const bool flat = p.d % kGroup == 0 && (W == kLoad || p.ldx == p.d) && (W == kStore || p.ldy == p.d) && (!p.act || p.lda == p.d);
  const int64_t blocks = (p.chunks + kThreads * kBatch - 1) / (kThreads * kBatch);
  if (flat) checkpoint_kernel<T, W, true><<<(unsigned)blocks, kThreads, 0, lc.stream>>>(p);
  else checkpoint_kernel<T, W, false><<<(unsigned)blocks, kThreads, 0, lc.stream>>>(p);
  lc.count();
  lc.check();
}

template <int W>
hbp_status call(int dtype, int64_t rows, int d, const void* x, int64_t ldx, void* y, int64_t ldy, void* act, int64_t lda, int8_t* codes,
                uint8_t* scales, void* stream) {
  if (dtype != HBP_F32 && dtype != HBP_BF16) return HBP_ERR_DTYPE;
  const int v = dtype == HBP_F32 ? 4 : 8;
  if (rows < 0 || d <= 0 || d % v) return HBP_ERR_SHAPE;
  const int64_t per_row = (d + kGroup - 1) / kGroup * (kGroup / v);
  if (rows > (int64_t)INT32_MAX * kThreads / per_row) return HBP_ERR_SHAPE;
  if (rows == 0) return HBP_OK;
  if (!codes || !scales || (W != kLoad && !x) || (W != kStore && !y)) return HBP_ERR_INVALID_ARG;
  auto bad = [&](const void* t, int64_t ld) { return ((uintptr_t)t & 15u) || ld < d || ld % v; };
  if (((uintptr_t)codes & 15u) || (W != kLoad && bad(x, ldx)) || (W != kStore && bad(y, ldy)) || (act && bad(act, lda))) return HBP_ERR_SHAPE;
  if (x && x == y && ldx != ldy) return HBP_ERR_INVALID_ARG;  // in place, but rows elsewhere
  Launcher lc;
  lc.stream = (cudaStream_t)stream;
  CheckpointParams p = {};
  p.rows = rows; p.d = d;
  p.x = x; p.y = y; p.act = act;
  p.ldx = ldx; p.ldy = ldy; p.lda = lda;
  p.codes = codes; p.scales = scales;
  if (dtype == HBP_F32) launch<float, W>(lc, p);
  else launch<bf16, W>(lc, p);
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}

}  // namespace

}  // namespace hbp

using namespace hbp;

extern "C" {

hbp_status hbp_checkpoint_store(int32_t dtype, int64_t rows, int32_t d, const void* x, int64_t ldx, int8_t* codes, uint8_t* scales,
                                void* cuda_stream) {
  return call<kStore>(dtype, rows, d, x, ldx, nullptr, 0, nullptr, 0, codes, scales, cuda_stream);
}
hbp_status hbp_checkpoint_load(int32_t dtype, int64_t rows, int32_t d, const int8_t* codes, const uint8_t* scales, void* x, int64_t ldx,
                               void* cuda_stream) {
  return call<kLoad>(dtype, rows, d, nullptr, 0, x, ldx, nullptr, 0, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales), cuda_stream);
}
hbp_status hbp_checkpoint_gelu(int32_t dtype, int64_t rows, int32_t d, const void* z, int64_t ldz, void* act, int64_t lda, int8_t* codes,
                               uint8_t* scales, void* cuda_stream) {
  return call<kGelu>(dtype, rows, d, z, ldz, act, lda, nullptr, 0, codes, scales, cuda_stream);
}
hbp_status hbp_checkpoint_gelu_backward(int32_t dtype, int64_t rows, int32_t d, const int8_t* codes, const uint8_t* scales, const void* d_act,
                                        int64_t ldd, void* dz, int64_t ldz, void* act, int64_t lda, void* cuda_stream) {
  return call<kGeluBackward>(dtype, rows, d, d_act, ldd, dz, ldz, act, lda, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales), cuda_stream);
}

}  // extern "C"
