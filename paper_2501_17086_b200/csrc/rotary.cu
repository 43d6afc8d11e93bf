// Rotary positions on the queries and keys of an attention step (hbp_rotary).
//
// HBM-bound: every element is read and written once, and a pair costs 6 flops.  What could cost more are the angles: formed in double,
// since a float product pos * f loses all of its fraction at positions of 2^17, and shared by all heads of a row.  So a thread
// owns CV pairs of a row for a run of heads: it forms their cosines and sines once, as fractions of a turn (one product and one
// rounding in double, then sincospif, which needs no reduction), keeps them in registers and streams the heads through,
// kHeads at a time so that 2 * kHeads 16-byte loads are in flight.  Heads are split over threads only as far as
// the rows do not fill the chip.
// bf16, 16384 rows, 12 + 12 heads of 64 (101 MB): FILL
#include <cmath>

#include "hbp_internal.h"

namespace hbp {

namespace {

constexpr int kMaxPairs = 128, kHeads = 4, kThreads = 128;

struct RotaryParams {
  double turns[kMaxPairs];  // f_i / 2 pi
  float amplitude, sign;
  int64_t rows, first, period;
  const void* positions;
  int position_bytes;
  int q_heads, heads;      // heads of q; of q and k
  int heads_each;          // heads of one thread
  int turn_chunks, chunks; // chunks of CV pairs that turn; with those that are copied
  int rotary_dim, head_dim;
  hbp_heads q, qo, k, ko;
};

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// kHalf: the two members of a pair lie rotary_dim / 2 apart.  CV: pairs of a thread; a Vec<T, CV> is at most 16 bytes.
template <typename T, int CV, bool kHalf>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  using V = Vec<T, CV>;
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x, row = idx / p.chunks;
  if (row >= p.rows) return;
  const int c = (int)(idx - row * p.chunks);
  const bool turning = c < p.turn_chunks;
  // first channels of the two vectors of this chunk; a copied chunk is two vectors, the second of which may lie past the head
  const int c0 = !turning ? p.rotary_dim + (c - p.turn_chunks) * 2 * CV : kHalf ? c * CV : 2 * c * CV;
  const int c1 = turning && kHalf ? c0 + p.rotary_dim / 2 : c0 + CV;
  const bool both = c1 < p.head_dim;
  float cs[CV], sn[CV];
  if (turning) {
    int64_t pos;
    if (!p.positions) pos = p.first + (p.period ? row % p.period : row);
    else if (p.position_bytes == 8) pos = ((const int64_t*)p.positions)[row];
    else pos = ((const int32_t*)p.positions)[row];
#pragma unroll
    for (int i = 0; i < CV; ++i) {
      double t = (double)pos * p.turns[c * CV + i];
      t -= rint(t);
      float s, co;
      sincospif(2.0f * (float)t, &s, &co);
      cs[i] = p.amplitude * co;
      sn[i] = p.amplitude * p.sign * s;
    }
  }
  const int h_end = min(p.heads, (int)(blockIdx.y + 1) * p.heads_each);
  for (int h0 = blockIdx.y * p.heads_each; h0 < h_end; h0 += kHeads) {
    V a[kHeads], b[kHeads];
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = h0 + u;
      if (h < h_end) {
        const bool key = h >= p.q_heads;
        const T* x = key ? (const T*)p.k.x + row * p.k.row_stride + (h - p.q_heads) * p.k.head_stride
                         : (const T*)p.q.x + row * p.q.row_stride + h * p.q.head_stride;
        a[u] = *reinterpret_cast<const V*>(x + c0);
        if (both) b[u] = *reinterpret_cast<const V*>(x + c1);
      }
    }
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = h0 + u;
      if (h < h_end) {
        if (turning) {
          if (kHalf) {
#pragma unroll
            for (int i = 0; i < CV; ++i) {
              const float x0 = to_f(a[u].v[i]), x1 = to_f(b[u].v[i]);
              a[u].v[i] = from_f<T>(x0 * cs[i] - x1 * sn[i]);
              b[u].v[i] = from_f<T>(x1 * cs[i] + x0 * sn[i]);
            }
          } else if (CV == 1) {
            const float x0 = to_f(a[u].v[0]), x1 = to_f(b[u].v[0]);
            a[u].v[0] = from_f<T>(x0 * cs[0] - x1 * sn[0]);
            b[u].v[0] = from_f<T>(x1 * cs[0] + x0 * sn[0]);
          } else {
#pragma unroll
            for (int i = 0; i < CV; i += 2) {
              const float x0 = to_f(a[u].v[i]), x1 = to_f(a[u].v[i + 1]), y0 = to_f(b[u].v[i]), y1 = to_f(b[u].v[i + 1]);
              a[u].v[i] = from_f<T>(x0 * cs[i / 2] - x1 * sn[i / 2]);
              a[u].v[i + 1] = from_f<T>(x1 * cs[i / 2] + x0 * sn[i / 2]);
              b[u].v[i] = from_f<T>(y0 * cs[(CV + i) / 2] - y1 * sn[(CV + i) / 2]);
              b[u].v[i + 1] = from_f<T>(y1 * cs[(CV + i) / 2] + y0 * sn[(CV + i) / 2]);
            }
          }
        }
        const bool key = h >= p.q_heads;
        T* y = key ? (T*)p.ko.x + row * p.ko.row_stride + (h - p.q_heads) * p.ko.head_stride
                   : (T*)p.qo.x + row * p.qo.row_stride + h * p.qo.head_stride;
        *reinterpret_cast<V*>(y + c0) = a[u];
        if (both) *reinterpret_cast<V*>(y + c1) = b[u];
      }
    }
  }
}

template <typename T, int CV>
void launch(Launcher& lc, RotaryParams& p, bool half, bool copies) {
  p.turn_chunks = p.rotary_dim / (2 * CV);
  p.chunks = p.turn_chunks + (copies ? (p.head_dim - p.rotary_dim + 2 * CV - 1) / (2 * CV) : 0);
  const int64_t blocks = (p.rows * p.chunks + kThreads - 1) / kThreads;
  // heads over threads until there are eight blocks an SM, in whole batches of loads
  const int most = (p.heads + kHeads - 1) / kHeads;
  int64_t parts = (8 * 148 + blocks - 1) / blocks;
  if (parts > most) parts = most;
  p.heads_each = (int)((most + parts - 1) / parts) * kHeads;
  const dim3 grid((unsigned)blocks, (unsigned)((p.heads + p.heads_each - 1) / p.heads_each));
  if (half) rotary_kernel<T, CV, true><<<grid, kThreads, 0, lc.stream>>>(p);
  else rotary_kernel<T, CV, false><<<grid, kThreads, 0, lc.stream>>>(p);
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
  const double pi2 = 6.283185307179586476925;
  for (int i = 0; i < pairs; ++i) {
    double f = std::pow((double)s.base, -2.0 * i / s.rotary_dim);
    if (s.scaling == HBP_ROTARY_LINEAR) f /= s.factor;
    if (s.scaling == HBP_ROTARY_BY_PARTS) {
      double w = ((double)s.trained_length * f / pi2 - s.slow) / ((double)s.fast - s.slow);
      w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
      f *= w + (1.0 - w) / s.factor;
    }
    p.turns[i] = f / pi2;
  }
  p.amplitude = s.amplitude;
  p.sign = inverse ? -1.0f : 1.0f;
  p.rows = rows; p.first = first; p.period = period;
  p.positions = positions; p.position_bytes = position_bytes;
  p.q_heads = q_heads; p.heads = q_heads + kv_heads;
  p.rotary_dim = s.rotary_dim; p.head_dim = head_dim;
  p.q = q; p.qo = qo; p.k = k; p.ko = ko;
  const bool half = s.layout == HBP_ROTARY_HALF;
  auto in_place = [](const hbp_heads& a, const hbp_heads& b) { return a.x == b.x; };
  const bool copies = head_dim > s.rotary_dim && !(in_place(q, qo) && (kv_heads == 0 || in_place(k, ko)));
  // The widest vectors that pairs and copied channels come in whole numbers of (rows and heads start on 16 bytes): half layout,
  // vectors of rotary_dim / 2 channels; interleaved, two vectors side by side.
  auto fits = [&](int cv) { return pairs % cv == 0 && (head_dim - s.rotary_dim) % cv == 0; };
  if (dtype == HBP_F32) {
    if (fits(4)) launch<float, 4>(lc, p, half, copies);
    else launch<float, 1>(lc, p, half, copies);
  } else {
    if (fits(8)) launch<bf16, 8>(lc, p, half, copies);
    else if (fits(4)) launch<bf16, 4>(lc, p, half, copies);
    else launch<bf16, 1>(lc, p, half, copies);
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
  if (rows > (int64_t)INT32_MAX * kThreads / kMaxPairs) return HBP_ERR_SHAPE;
  if (period < 0 || (positions && position_bytes != 4 && position_bytes != 8)) return HBP_ERR_INVALID_ARG;
  if (positions && ((uintptr_t)positions % position_bytes)) return HBP_ERR_SHAPE;
  if (!q || !q_out || (kv_heads && (!k || !k_out))) return HBP_ERR_INVALID_ARG;
  if (rows == 0) return HBP_OK;
  const hbp_heads none = {};
  const hbp_heads t[4] = {*q, *q_out, kv_heads ? *k : none, kv_heads ? *k_out : none};
  for (int i = 0; i < (kv_heads ? 4 : 2); ++i) {
    if (!t[i].x) return HBP_ERR_INVALID_ARG;
    if (((uintptr_t)t[i].x & 15u) || t[i].row_stride % v || t[i].head_stride % v) return HBP_ERR_SHAPE;
  }
  for (int i = 0; i < 4; i += 2)
    if (t[i].x && t[i].x == t[i + 1].x && (t[i].row_stride != t[i + 1].row_stride || t[i].head_stride != t[i + 1].head_stride))
      return HBP_ERR_INVALID_ARG;  // in place, but rows or heads elsewhere
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  rotary(lc, *spec, inverse != 0, dtype, rows, q_heads, kv_heads, head_dim, positions, position_bytes, first, period, t[0], t[1], t[2], t[3]);
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}
