// Rotary positions on the queries and keys of an attention step (hbp_rotary).
//
// HBM-bound: every element is read and written once, and a pair costs 6 flops.  What costs more is everything around them, so
//  - angles are whole-number fractions of a turn: position times f_i / 2 pi * 2^64, modulo 2^64.  That needs no reduction, is off by 2^-64 turns a
//    position and 2^-33 turns (a float product pos * f loses all of its fraction at 2^17; a float fraction alone would be off by 2^-26), and takes a
//    few integer instructions where doubles took a conversion, a product, a rounding and a difference;
//  - they are shared by all heads of a row: a block forms cosines and sines of its rows once, in shared memory, rows fastest, since the lanes of a
//    warp that read different frequencies from the constant bank would be served one after the other;
//  - a thread keeps CV pairs of a row (two vectors of up to 16 bytes) and walks over heads: its cosines and sines stay in registers
//    and a head costs two loads, the rotation and two stores.
// bf16, 16384 rows, 12 + 12 heads of 64 (101 MB): 22.2 us (4.5 TB/s; 15.4 at the rate of a copy), 8192 rows, 32 + 8 heads of 128 (168 MB): 32.9.
// With the angles in double and every thread forming its own: 34.8 and 49.6; the pairs of a block dealt out one by one
// (280 instructions a unit): 26.6 and 36.9.  Blocks of 256 threads and 16 rows, which all start at once and wait at once: 24.6 and 48.0.
// What is left are the instructions of a unit and the first wait of a block, for its positions.
#include <cmath>

#include "float_pairs.cuh"

namespace hbp {

namespace {

constexpr int kMaxPairs = 128, kUnroll = 2, kThreads = 128, kMaxRows = 8;

struct RotaryParams {
  uint64_t turns[kMaxPairs];  // f_i / 2 pi * 2^64
  float amplitude, sign;
  int64_t rows, first, period;
  const void* positions;
  int position_bytes;
  int q_heads, heads;       // heads of q; of q and k
  int turn_chunks, chunks;  // units of a head that turn; with those that are copied
  int rotary_dim, head_dim;
  hbp_heads q, qo, k, ko;
};

// A unit is, of every head, in the half layout CV pairs: two vectors of CV channels rotary_dim / 2 apart; in the interleaved one
// CV / 2 pairs: one vector.  (Two neighbouring vectors there: 49.3 us where this takes 36.9, 8192 rows, 32 + 8 heads of 128.)
// A unit that is copied has as many vectors, side by side.
template <typename T, int CV, bool kHalf>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  using V = Vec<T, CV>;
  constexpr int kPairs = kHalf ? CV : CV / 2, kVectors = kHalf ? 2 : 1;
  // {cosine, sine} of pair i of unit c in row r at [r][i][c]: neighbouring threads, which have neighbouring units, read neighbouring words
  extern __shared__ float2 table[];
  const int c = threadIdx.x, slot = threadIdx.y, r = threadIdx.z, slots = blockDim.y, half = p.rotary_dim / 2;
  const int64_t row = (int64_t)blockIdx.x * blockDim.z + r;
  const bool turning = c < p.turn_chunks;
  if (row < p.rows && turning) {
    int64_t pos;
    if (p.position_bytes == 4) pos = ((const int32_t*)p.positions)[row];
    else if (p.position_bytes == 8) pos = ((const int64_t*)p.positions)[row];
    else pos = p.first + (p.period ? row % p.period : row);
    for (int i = slot; i < kPairs; i += slots) {
      const int32_t t = (int32_t)(((uint64_t)pos * p.turns[c * kPairs + i] + 0x80000000u) >> 32);  // of a turn, from -1/2 on
      const float f = (float)t;
      float sn, cs;
      sincospif(f * 0x1p-31f, &sn, &cs);
      // what the float has lost of it, up to 2^-26 turns: an angle so small that it is its own sine
      const float rest = (float)(t - (int32_t)f) * (3.14159265358979323846f * 0x1p-31f), s0 = sn;
      sn = fmaf(rest, cs, sn);
      cs = fmaf(-rest, s0, cs);
      table[(r * kPairs + i) * p.turn_chunks + c] = make_float2(p.amplitude * cs, p.amplitude * p.sign * sn);
    }
  }
  __syncthreads();
  if (row >= p.rows) return;
  const int c0 = turning ? c * CV : p.rotary_dim + (c - p.turn_chunks) * kVectors * CV;  // first channels of the vectors
  const int c1 = turning ? c0 + half : c0 + CV;
  const bool two = kHalf && c1 < p.head_dim;
  // half layout: cosines, and sines, of two neighbouring pairs at a time; interleaved: (cos, cos) and (-sin, sin) of a pair
  constexpr int kTwos = kHalf ? (CV + 1) / 2 : kPairs;
  f32x2 cs[kTwos], sn[kTwos];
  if (turning) {
#pragma unroll
    for (int i = 0; i < kTwos; ++i) {
      if (kHalf) {
        const float2 e = table[(r * kPairs + 2 * i) * p.turn_chunks + c], f = table[(r * kPairs + (2 * i + 1) % CV) * p.turn_chunks + c];
        cs[i] = pair_of(e.x, f.x);
        sn[i] = pair_of(e.y, f.y);
      } else {
        const float2 e = table[(r * kPairs + i) * p.turn_chunks + c];
        cs[i] = pair_of(e.x, e.x);
        sn[i] = pair_of(-e.y, e.y);
      }
    }
  }
  auto heads = [&](const hbp_heads& in, const hbp_heads& out, int h, int count) {
    const T* x = (const T*)in.x + row * in.row_stride + h * in.head_stride + c0;
    T* y = (T*)out.x + row * out.row_stride + h * out.head_stride + c0;
    const int64_t dx = slots * in.head_stride, dy = slots * out.head_stride;
    for (; h < count; h += kUnroll * slots) {
      V a[kUnroll], b[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (h + u * slots < count) {
          a[u] = *reinterpret_cast<const V*>(x + u * dx);
          if (two) b[u] = *reinterpret_cast<const V*>(x + u * dx + (c1 - c0));
        }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (h + u * slots < count) {
          if (turning) {
            if (kHalf && CV == 1) {
              const float2 k = floats_of(cs[0]), l = floats_of(sn[0]);
              const float m = to_f(a[u].v[0]), n = to_f(b[u].v[0]);
              a[u].v[0] = from_f<T>(fmaf(m, k.x, -__fmul_rn(n, l.x)));
              b[u].v[0] = from_f<T>(fmaf(n, k.x, __fmul_rn(m, l.x)));
            } else {
#pragma unroll
              for (int i = 0; i + 1 < CV; i += 2) {
                const f32x2 m = widen2(a[u].v + i);
                if (kHalf) {
                  const f32x2 n = widen2(b[u].v + i);
                  const float2 t = floats_of(mul2(n, sn[i / 2]));
                  narrow2(fma2(m, cs[i / 2], pair_of(-t.x, -t.y)), a[u].v + i);
                  narrow2(fma2(n, cs[i / 2], mul2(m, sn[i / 2])), b[u].v + i);
                } else {
                  const float2 t = floats_of(m);
                  narrow2(fma2(m, cs[i / 2], mul2(pair_of(t.y, t.x), sn[i / 2])), a[u].v + i);
                }
              }
            }
          }
          *reinterpret_cast<V*>(y + u * dy) = a[u];
          if (two) *reinterpret_cast<V*>(y + u * dy + (c1 - c0)) = b[u];
        }
      x += kUnroll * dx;
      y += kUnroll * dy;
    }
  };
  heads(p.q, p.qo, slot, p.q_heads);
  // (the threads that had one head of q fewer begin)
  heads(p.k, p.ko, (slot + slots - p.q_heads % slots) % slots, p.heads - p.q_heads);
}

template <typename T, int CV, bool kHalf>
void launch(Launcher& lc, RotaryParams& p, bool copies) {
  constexpr int kUnit = kHalf ? 2 * CV : CV;  // channels
  p.turn_chunks = p.rotary_dim / kUnit;
  p.chunks = p.turn_chunks + (copies ? (p.head_dim - p.rotary_dim + kUnit - 1) / kUnit : 0);
  // as many rows to a block as leave four blocks an SM, up to kMaxRows; then as many threads to a unit as it still has
  const int64_t want = p.rows / (4 * 148);
  int rows = want < 1 ? 1 : want > kMaxRows ? kMaxRows : (int)want;
  if (rows > kThreads / p.chunks) rows = kThreads / p.chunks;
  int slots = kThreads / (p.chunks * rows);
  if (slots > p.heads) slots = p.heads;
  const int64_t blocks = (p.rows + rows - 1) / rows;
  const size_t smem = (size_t)rows * (p.rotary_dim / 2) * sizeof(float2);
  rotary_kernel<T, CV, kHalf><<<(unsigned)blocks, dim3(p.chunks, slots, rows), smem, lc.stream>>>(p);
  lc.count();
  lc.check();
}

}  // namespace

hbp_status check_rotary_spec(const hbp_rotary_spec* s, int head_dim) {
  if (!s) return HBP_ERR_INVALID_ARG;
  if (s->layout != HBP_ROTARY_HALF && s->layout != HBP_ROTARY_INTERLEAVED) return HBP_ERR_UNSUPPORTED;
  if (s->scaling < HBP_ROTARY_NONE || s->scaling > HBP_ROTARY_BY_PARTS) return HBP_ERR_UNSUPPORTED;
  if (s->rotary_dim < 2 || s->rotary_dim % 2 || s->rotary_dim > head_dim || head_dim > 2 * kMaxPairs) return HBP_ERR_SHAPE;
  if (!(s->base > 1.0f) || std::isinf(s->base) || !std::isfinite(s->amplitude)) return HBP_ERR_INVALID_ARG;
  if (s->scaling != HBP_ROTARY_NONE && (!(s->factor >= 1.0f) || std::isinf(s->factor))) return HBP_ERR_INVALID_ARG;
  if (s->scaling == HBP_ROTARY_BY_PARTS && (!(s->trained_length > 0.0f) || std::isinf(s->trained_length) || !(s->fast > s->slow) || !std::isfinite(s->fast) || !std::isfinite(s->slow)))
    return HBP_ERR_INVALID_ARG;
  return HBP_OK;
}

void rotary(Launcher& lc, const hbp_rotary_spec& s, bool inverse, int dtype, int64_t rows, int q_heads, int kv_heads, int head_dim,
            const void* positions, int position_bytes, int64_t first, int64_t period, const hbp_heads& q, const hbp_heads& qo,
            const hbp_heads& k, const hbp_heads& ko) {
  RotaryParams p;
  const int pairs = s.rotary_dim / 2;
  // In 64 binary digits (a double's 53 would be off by 2^-57 turns a position): base^(-2i/r) = 2^(i c), whose exponent is off by 2 |i c| 2^-64, which
  // is less than 2^-64 of a turn whatever the base, since 2^-x x is below 0.54.  Eight at a time from one: a power takes as long as pow in double did.
  typedef long double wide;
  const wide pi2 = 6.283185307179586476925286766559L, c = -2.0L / s.rotary_dim * std::log2((wide)s.base);
  wide low[8], high = 1.0L;
  for (int i = 0; i < 8 && i < pairs; ++i) low[i] = std::exp2(c * i);
  for (int i = 0; i < pairs; ++i) {
    if (i && i % 8 == 0) high = std::exp2(c * i);
    wide f = high * low[i % 8];
    if (s.scaling == HBP_ROTARY_LINEAR) f /= s.factor;
    if (s.scaling == HBP_ROTARY_BY_PARTS) {
      wide w = ((wide)s.trained_length * f / pi2 - s.slow) / ((wide)s.fast - s.slow);
      w = w < 0.0L ? 0.0L : w > 1.0L ? 1.0L : w;
      f *= w + (1.0L - w) / s.factor;
    }
    p.turns[i] = (uint64_t)(int64_t)(f * (18446744073709551616.0L / pi2) + 0.5L);  // (below 1/6 of 2^64)
  }
  p.amplitude = s.amplitude;
  p.sign = inverse ? -1.0f : 1.0f;
  p.rows = rows; p.first = first; p.period = period;
  p.positions = positions; p.position_bytes = positions ? position_bytes : 0;
  p.q_heads = q_heads; p.heads = q_heads + kv_heads;
  p.rotary_dim = s.rotary_dim; p.head_dim = head_dim;
  p.q = q; p.qo = qo; p.k = k; p.ko = ko;
  const bool half = s.layout == HBP_ROTARY_HALF;
  auto in_place = [](const hbp_heads& a, const hbp_heads& b) { return a.x == b.x; };
  const bool copies = head_dim > s.rotary_dim && !(in_place(q, qo) && (kv_heads == 0 || in_place(k, ko)));
  // The widest vectors that the turning channels (half layout: each half of them) and the others come in whole numbers of; rows and heads start
  // on 16 bytes.
  const int run = half ? pairs : s.rotary_dim, rest = head_dim - s.rotary_dim;
  auto fits = [&](int cv) { return run % cv == 0 && rest % cv == 0; };
  if (dtype == HBP_F32) {
    if (fits(4)) half ? launch<float, 4, true>(lc, p, copies) : launch<float, 4, false>(lc, p, copies);
    else half ? launch<float, 1, true>(lc, p, copies) : launch<float, 2, false>(lc, p, copies);
  } else if (fits(8)) {
    half ? launch<bf16, 8, true>(lc, p, copies) : launch<bf16, 8, false>(lc, p, copies);
  } else if (fits(4)) {
    half ? launch<bf16, 4, true>(lc, p, copies) : launch<bf16, 4, false>(lc, p, copies);
  } else {
    half ? launch<bf16, 1, true>(lc, p, copies) : launch<bf16, 2, false>(lc, p, copies);
  }
}

}  // namespace hbp

using namespace hbp;

extern "C" hbp_status hbp_rotary(const hbp_rotary_spec* spec, int32_t inverse, int32_t dtype, int64_t rows, int32_t q_heads, int32_t kv_heads,
                                 int32_t head_dim, const void* positions, int32_t position_bytes, int64_t first, int64_t period,
                                 const hbp_heads* q, const hbp_heads* q_out, const hbp_heads* k, const hbp_heads* k_out, void* cuda_stream) {
  if (dtype != HBP_F32 && dtype != HBP_BF16) return HBP_ERR_DTYPE;
  const int v = dtype == HBP_F32 ? 4 : 8;
  if (rows < 0 || q_heads <= 0 || kv_heads < 0 || (int64_t)q_heads + kv_heads > 65535 || head_dim <= 0 || head_dim % v) return HBP_ERR_SHAPE;
  const hbp_status st = check_rotary_spec(spec, head_dim);
  if (st != HBP_OK) return st;
  if (rows > INT32_MAX) return HBP_ERR_SHAPE;
  if (period < 0 || (positions && position_bytes != 4 && position_bytes != 8)) return HBP_ERR_INVALID_ARG;
  if (positions && ((uintptr_t)positions % position_bytes)) return HBP_ERR_SHAPE;
  if (!q || !q_out || (kv_heads && (!k || !k_out))) return HBP_ERR_INVALID_ARG;
  if (rows == 0) return HBP_OK;
  const hbp_heads none = {};
  const hbp_heads t[4] = {*q, *q_out, kv_heads ? *k : none, kv_heads ? *k_out : none};
  for (int i = 0; i < (kv_heads ? 4 : 2); ++i) {
    if (!t[i].x) return HBP_ERR_INVALID_ARG;
    if (((uintptr_t)t[i].x & 15u) || t[i].row_stride % v || t[i].head_stride % v || t[i].row_stride < 0 || t[i].head_stride < 0) return HBP_ERR_SHAPE;
  }
  for (int i = 0; i < 4; i += 2)
    if (t[i].x && t[i].x == t[i + 1].x && (t[i].row_stride != t[i + 1].row_stride || t[i].head_stride != t[i + 1].head_stride))
      return HBP_ERR_INVALID_ARG;  // in place, but rows or heads elsewhere
  for (int i = 1; i < (kv_heads ? 4 : 2); i += 2) {  // outputs: no two elements in one place, rows of heads or heads of rows
    const int64_t rs = t[i].row_stride, hs = t[i].head_stride, heads = i == 1 ? q_heads : kv_heads;
    const bool apart = (rows <= 1 || rs >= (heads - 1) * hs + head_dim) && (heads <= 1 || hs >= head_dim);
    const bool across = (heads <= 1 || hs >= (rows - 1) * rs + head_dim) && (rows <= 1 || rs >= head_dim);
    if (!apart && !across) return HBP_ERR_SHAPE;
  }
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  rotary(lc, *spec, inverse != 0, dtype, rows, q_heads, kv_heads, head_dim, positions, position_bytes, first, period, t[0], t[1], t[2], t[3]);
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}
