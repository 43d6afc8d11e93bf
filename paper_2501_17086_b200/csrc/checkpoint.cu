// Activations in 8 bits and GELU's backward pass from them (hbp_checkpoint_*).
//
// A group of 32 channels shares a power of two, the smallest 2^e with max |x| <= 127 * 2^e, found from the bits of the
// largest magnitude (the maximum is taken over bit patterns, so that infinities and NaN come out on top of it).  Powers of two
// make both directions exact but for the one rounding to a whole number, and every stored value a bf16 number.
//
// HBM-bound, if the arithmetic stays out of the way: at 6.5 TB/s an SM has 27 instruction slots for each bf16 value of GELU's forward
// pass.  So whole numbers are rounded and widened by adding 1.5 * 2^23 (conversions run at an eighth of the rate),
// magnitudes of bf16 pairs are compared two at a time, float arithmetic is done on pairs (one instruction for two values), and
// erfc(x) is e^(-x^2) times a polynomial in t = 1 / (1 + p x) without a constant term, the form of 7.1.26 in Abramowitz and Stegun, "Handbook of
// Mathematical Functions" (erff alone takes some 25 instructions); its exponential is GELU's density as well: one ex2 and one reciprocal serve gelu and
// gelu' together.  7.1.26 itself is off by up to 1.5e-7, which is 0.2 % of erfc at z = -5 and 1 % at -8; half a step of bf16 is 0.4 %.  So for bf16 p and
// the coefficients, one more than there, are those for which the larger of (error of erfc / 2) / 6e-8 and (error relative to erfc) / 1e-4 is least over
// 0 <= x <= 9.4 (a linear programme for each p): 0.88.  Float takes ten coefficients and accurate exponentials and reciprocals.
// 8192 x 4096, us (of what a copy of the same bytes takes): bf16 store 18.4 (0.84), load 18.5 (0.84), GELU 28.9 (0.89), its backward pass with gelu 38.9
// (0.93); float 28.7 (0.90), 28.9 (0.89), 55.4 (0.83), 68.9 (0.97; with erfcf 71.7 and 90.8).  bf16 with erff, conversions and one value at a time:
// 24.6, 24.8, 40.6, 57.4.
// A thread moves kBatch vectors of 16 bytes, all loads before the first use.  A group is 4 (bf16) or 8 (float) neighbouring lanes, its
// maximum 2 or 3 shuffles.  (kBatch 1, 2, 4: store 22.6, 18.5, 18.7; GELU 32.7, 28.9, 30.0; float 8192 x 1024 stored 12.6, 10.3, 10.3.)
#include "float_pairs.cuh"

namespace hbp {

namespace {

constexpr int kThreads = 256, kBatch = 2;
constexpr int kGroup = 32;

enum Work { kStore = 0, kLoad = 1, kGelu = 2, kGeluBackward = 3, kGeluAgain = 4 };  // the last: gelu(z8) alone

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

// gelu(z) and gelu'(z) of two values; every rounding is written out, so that no call's other outputs change them.  `tail` is the normal
// distribution's beyond |z|, half of erfc(|z| / sqrt 2): taken as it is below zero, where 1/2 less what erf gives would cancel (4 % of gelu at -5).
__device__ __forceinline__ float one_from_zero_on(float z) {
  float b;
  asm("set.ge.f32.f32 %0, %1, 0f00000000;" : "=f"(b) : "f"(z));
  return b;
}
// From the tail and e = e^(-z^2 / 2).  Both are of |z| and b - tail, b = 1 from 0 on and else 0: gelu as it is, the slope but for its sign.
__device__ __forceinline__ void gelu_from(float2 zf, f32x2 size, f32x2 tail, f32x2 e, float2& act, float2& slope) {
  const f32x2 b = pair_of(one_from_zero_on(zf.x), one_from_zero_on(zf.y)), phi = fma2(tail, both(-1.0f), b);
  act = floats_of(mul2(size, phi));
  slope = floats_of(mul2(fma2(mul2(size, e), both(0.39894228040143267794f), phi), fma2(b, both(2.0f), both(-1.0f))));
}
__device__ __forceinline__ void gelu_pair(float2 zf, float2& act, float2& slope, float) {
  const f32x2 size = pair_of(fabsf(zf.x), fabsf(zf.y));
  const float2 arg = floats_of(mul2(mul2(size, both(-0.5f)), size)), den = floats_of(fma2(size, both(0.3889087439f), both(1.0f)));
  const f32x2 e = pair_of(expf(arg.x), expf(arg.y)), t = pair_of(__frcp_rn(den.x), __frcp_rn(den.y));  // t = 1 / (1 + 0.55 |z| / sqrt 2)
  // tail / e, to 9e-9 of itself up to |z| = 13.5 (interpolated at the Chebyshev nodes of t, relative to its values)
  f32x2 q = fma2(t, both(0.02973128855f), both(-0.172106415f));
  q = fma2(q, t, both(0.3993062079f));
  q = fma2(q, t, both(-0.437952131f));
  q = fma2(q, t, both(0.19097054f));
  q = fma2(q, t, both(-0.05208843574f));
  q = fma2(q, t, both(0.1025155559f));
  q = fma2(q, t, both(0.1291147918f));
  q = fma2(q, t, both(0.1553640366f));
  q = fma2(q, t, both(0.1551445723f));
  gelu_from(zf, size, mul2(mul2(q, t), e), e, act, slope);
}
__device__ __forceinline__ void gelu_pair(float2 zf, float2& act, float2& slope, bf16) {
  const f32x2 size = pair_of(fabsf(zf.x), fabsf(zf.y));
  const float2 arg = floats_of(mul2(mul2(size, size), both(-0.72134752044448170368f))), den = floats_of(fma2(size, both(0.28991378f), both(1.0f)));
  float2 ef, tf;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ef.x) : "f"(arg.x));  // e^(-z^2 / 2)
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ef.y) : "f"(arg.y));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(tf.x) : "f"(den.x));  // t = 1 / (1 + 0.41 |z| / sqrt 2)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(tf.y) : "f"(den.y));
  const f32x2 e = pair_of(ef.x, ef.y), t = pair_of(tf.x, tf.y);
  // tail / e^(-z^2 / 2), to 9e-5 of itself up to |z| = 13.3 and 6e-8 e^(z^2 / 2)
  f32x2 q = fma2(t, both(-0.0895100138f), both(0.2877123734f));
  q = fma2(q, t, both(-0.0970873242f));
  q = fma2(q, t, both(0.1820728296f));
  q = fma2(q, t, both(0.0998823909f));
  q = fma2(q, t, both(0.1169299858f));
  gelu_from(zf, size, mul2(mul2(q, t), e), e, act, slope);
}

// Bits of the largest magnitude of a vector, as a float's
__device__ __forceinline__ uint32_t largest(const float* v) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ uint32_t largest(const bf16* v) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) m = __vmaxu2(m, w[e] & 0x7fff7fffu);
  return max(m << 16, m & 0xffff0000u);
}
constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: what is added to it is rounded to a whole number, in its low bits
// four codes of four values
__device__ __forceinline__ uint32_t codes_of(const float* f, float inv) {
  uint32_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(fmaf(f[e], inv, kMagic));
  return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}
// and back
__device__ __forceinline__ void values_of(uint32_t c, float step, float* f) {
  c ^= 0x80808080u;  // codes + 128
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = __fmul_rn(__fsub_rn(__uint_as_float(__byte_perm(c, 0x4b000000u, 0x7440 + e)), 8388736.0f), step);
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
__device__ __forceinline__ float inverse_of(uint32_t s) { return __uint_as_float((254u - min(s, 253u)) << 23); }

// kFlat: rows are whole groups without gaps: one run of chunks
template <typename T, int W, bool kFlat>
__global__ void __launch_bounds__(kThreads) checkpoint_kernel(const CheckpointParams p) {
  constexpr int V = 16 / (int)sizeof(T), kLanes = kGroup / V;
  using VT = Vec<T, V>;
  using VC = Vec<uint32_t, V / 4>;  // four codes a word
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
      if (W != kLoad && W != kGeluAgain) x[u] = *reinterpret_cast<const VT*>((const T*)p.x + (kFlat ? i * V : row[u] * p.ldx + col[u]));
      if (W == kLoad || W == kGeluBackward || W == kGeluAgain) {
        code[u] = *reinterpret_cast<const VC*>(p.codes + (kFlat ? i * V : row[u] * p.d + col[u]));
        scale[u] = p.scales[kFlat ? i / kLanes : row[u] * p.groups + col[u] / kGroup];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const int64_t i = base + u * kThreads;
    const int64_t at_y = kFlat ? i * V : row[u] * p.ldy + col[u];
    float f[V];
    if (W == kStore || W == kGelu) {
      uint32_t amax = in[u] ? largest(x[u].v) : 0u;
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      if (!in[u]) continue;
      const uint32_t s = scale_of(amax);
      const float inv = inverse_of(s);
      widen<V>(x[u].v, f);
#pragma unroll
      for (int e = 0; e < V; e += 4) code[u].v[e / 4] = codes_of(f + e, inv);
      if (s >= kLargestScale) {
        int8_t* c = reinterpret_cast<int8_t*>(code[u].v);
#pragma unroll
        for (int e = 0; e < V; ++e) c[e] = (int8_t)(s == 255u ? 0 : fabsf(f[e]) >= 63.5f * 0x1p122f ? (f[e] < 0.0f ? -63 : 63) : c[e]);
      }
      *reinterpret_cast<VC*>(p.codes + (kFlat ? i * V : row[u] * p.d + col[u])) = code[u];
      if (i % kLanes == 0) p.scales[kFlat ? i / kLanes : row[u] * p.groups + col[u] / kGroup] = (uint8_t)s;
      if (W == kGelu) {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          float2 act, slope;
          gelu_pair(make_float2(f[e], f[e + 1]), act, slope, T());
          f[e] = act.x;
          f[e + 1] = act.y;
        }
        VT y;
        narrow<V>(f, y.v);
        *reinterpret_cast<VT*>((T*)p.y + at_y) = y;
      }
    } else if (in[u]) {
      const float step = step_of(scale[u]);
      VT y, a;
#pragma unroll
      for (int e = 0; e < V; e += 4) values_of(code[u].v[e / 4], step, f + e);
      if (W == kGeluBackward) {
        float g[V], af[V];
        widen<V>(x[u].v, g);
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          float2 act, slope;
          gelu_pair(make_float2(f[e], f[e + 1]), act, slope, T());
          f[e] = __fmul_rn(g[e], slope.x);
          f[e + 1] = __fmul_rn(g[e + 1], slope.y);
          af[e] = act.x;
          af[e + 1] = act.y;
        }
        if (p.act) {
          narrow<V>(af, a.v);
          *reinterpret_cast<VT*>((T*)p.act + (kFlat ? i * V : row[u] * p.lda + col[u])) = a;
        }
      }
      if (W == kGeluAgain) {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          float2 act, slope;
          gelu_pair(make_float2(f[e], f[e + 1]), act, slope, T());
          f[e] = act.x;
          f[e + 1] = act.y;
        }
      }
      narrow<V>(f, y.v);
      *reinterpret_cast<VT*>((T*)p.y + at_y) = y;
    }
  }
}

template <typename T, int W>
void launch(Launcher& lc, CheckpointParams& p) {
  constexpr int V = 16 / (int)sizeof(T);
  p.groups = (p.d + kGroup - 1) / kGroup;
  p.per_row = p.groups * (kGroup / V);
  p.chunks = p.rows * p.per_row;
  const bool flat = p.d % kGroup == 0 && (W == kLoad || W == kGeluAgain || p.ldx == p.d) && (W == kStore || p.ldy == p.d) && (!p.act || p.lda == p.d);
  const int64_t blocks = (p.chunks + kThreads * kBatch - 1) / (kThreads * kBatch);
  if (flat) checkpoint_kernel<T, W, true><<<(unsigned)blocks, kThreads, 0, lc.stream>>>(p);
  else checkpoint_kernel<T, W, false><<<(unsigned)blocks, kThreads, 0, lc.stream>>>(p);
  lc.count();
  lc.check();
}

template <int W>
void run(Launcher& lc, int dtype, int64_t rows, int d, const void* x, int64_t ldx, void* y, int64_t ldy, void* act, int64_t lda, int8_t* codes,
         uint8_t* scales) {
  CheckpointParams p = {};
  p.rows = rows; p.d = d;
  p.x = x; p.y = y; p.act = act;
  p.ldx = ldx; p.ldy = ldy; p.lda = lda;
  p.codes = codes; p.scales = scales;
  if (dtype == HBP_F32) launch<float, W>(lc, p);
  else launch<bf16, W>(lc, p);
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
  constexpr bool kIn = W != kLoad && W != kGeluAgain;
  if (!codes || !scales || (kIn && !x) || (W != kStore && !y)) return HBP_ERR_INVALID_ARG;
  auto bad = [&](const void* t, int64_t ld) { return ((uintptr_t)t & 15u) || ld < d || ld % v; };
  if (((uintptr_t)codes & 15u) || (kIn && bad(x, ldx)) || (W != kStore && bad(y, ldy)) || (act && bad(act, lda))) return HBP_ERR_SHAPE;
  if (x && x == y && ldx != ldy) return HBP_ERR_INVALID_ARG;  // in place, but rows elsewhere
  Launcher lc;
  lc.stream = (cudaStream_t)stream;
  run<W>(lc, dtype, rows, d, x, ldx, y, ldy, act, lda, codes, scales);
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}

}  // namespace

void checkpoint_gelu(Launcher& lc, int dtype, int64_t rows, int d, void* z, int8_t* codes, uint8_t* scales) {
  run<kGelu>(lc, dtype, rows, d, z, d, z, d, nullptr, 0, codes, scales);
}
void checkpoint_gelu_backward(Launcher& lc, int dtype, int64_t rows, int d, const int8_t* codes, const uint8_t* scales, void* dz) {
  run<kGeluBackward>(lc, dtype, rows, d, dz, d, dz, d, nullptr, 0, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales));
}
void checkpoint_gelu_again(Launcher& lc, int dtype, int64_t rows, int d, const int8_t* codes, const uint8_t* scales, void* act) {
  run<kGeluAgain>(lc, dtype, rows, d, nullptr, 0, act, d, nullptr, 0, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales));
}

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
  if (!d_act && !dz && act)
    return call<kGeluAgain>(dtype, rows, d, nullptr, 0, act, lda, nullptr, 0, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales), cuda_stream);
  return call<kGeluBackward>(dtype, rows, d, d_act, ldd, dz, ldz, act, lda, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales), cuda_stream);
}

}  // extern "C"
