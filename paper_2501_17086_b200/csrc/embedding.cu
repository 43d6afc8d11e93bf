// Rows of a table by tokens, scaled, and the table's gradient (hbp_embedding, hbp_embedding_gradient).
//
// Gradient: d_table[v] = add[v] + scale * sum of d_out[i] over the rows i whose token is v, in three launches.
//  1. One cluster of eight blocks sorts the tokens with their rows (stable, by digits of up to 9 bits, least first: 18 bits, which most
//     vocabularies need, are two passes); the other blocks of the launch meanwhile clear the table, or copy `add`: with 16384
//     tokens of 50021 that is what takes the time.  Eight blocks of 1024 threads rank and move 16384 tokens in some microseconds; their
//     exchange is a cluster's barrier and 512 counts a block.
//  2. Blocks add up the rows of 32 sorted tokens each, whole runs of one token straight to the table.  The share of a run that began in an
//     earlier tile, or goes on in the next, is a partial sum in scratch.
//  3. Those runs' partial sums are added in the order of the tiles, eight stretches of them at a time.
// Every sum has a fixed order: runs agree bit for bit.  A token that is every second one of a text costs no more than others.
#include "hbp_internal.h"
#include "tc_common.cuh"

namespace hbp {

namespace {

constexpr int kThreads = 256, kBatch = 4;  // lookup: vectors of 16 bytes a block, and how many of them a thread

struct Tokens {
  const void* t;
  int bytes;
  __device__ __forceinline__ int64_t operator[](int64_t i) const { return bytes == 8 ? ((const int64_t*)t)[i] : (int64_t)((const int32_t*)t)[i]; }
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

// ------------------------------------------------------------------------------------------- lookup
struct LookupParams {
  Tokens tokens;
  int64_t rows, ldt, ldo;
  const void* table;
  void* out;
  int vocab, per_row;  // vectors a row
  Divider by_row;
  float scale;
  int* status;
};

// Bound by bytes, and for few rows by its two waits (a token, then its row).  A thread's four vectors are asked for together.
template <typename T>
__global__ void __launch_bounds__(kThreads) lookup_kernel(const LookupParams p) {
  chain_next();
  chain_wait();
  constexpr int V = Vec<T>::V;
  const int64_t base = (int64_t)blockIdx.x * (kThreads * kBatch), row0 = base / p.per_row;
  const uint32_t rest = (uint32_t)(base - row0 * p.per_row);
  int64_t row[kBatch], token[kBatch];
  int col[kBatch];
  uint4 v[kBatch];
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const uint32_t i = rest + u * kThreads + threadIdx.x, r = p.by_row(i);
    row[u] = row0 + r;
    col[u] = (int)(i - r * p.per_row) * V;
    token[u] = row[u] < p.rows ? p.tokens[row[u]] : -1;
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    v[u] = make_uint4(0, 0, 0, 0);
    if (token[u] >= 0 && token[u] < p.vocab) v[u] = *reinterpret_cast<const uint4*>((const T*)p.table + token[u] * p.ldt + col[u]);
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    if (row[u] >= p.rows) continue;
    if (token[u] >= p.vocab && col[u] == 0 && p.status) *p.status = (int)HBP_ERR_INVALID_ARG;
    if (token[u] >= 0 && token[u] < p.vocab) {  // (no token: zeros, whatever the scale)
      float f[V];
      Vec<T>::widen(v[u], f);
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] *= p.scale;
      v[u] = Vec<T>::narrow(f);
    }
    *reinterpret_cast<uint4*>((T*)p.out + row[u] * p.ldo + col[u]) = v[u];
  }
}

// ------------------------------------------------------------------------------------------- tokens in order
constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kMaxDigit = 9, kMaxBins = 1 << kMaxDigit;
constexpr int kTile = 32;  // sorted tokens a block adds up

struct SortParams {
  Tokens tokens;
  int64_t rows;
  int vocab, passes, digit;  // digit: bits a pass
  uint32_t *keys[2], *from[2];
  int* status;
  float4* table;  // to be cleared, or filled from add, by the blocks behind the first eight
  const float4* add;
  int64_t vectors;
};

struct SortShared {
  uint32_t counts[kSortWarps][kMaxBins];  // of a warp's tokens, then where the next one of a digit goes
  uint32_t totals[kMaxBins];              // of a block's, read by the others
  uint32_t base[kMaxBins];
  uint32_t warp_sums[kSortWarps];
};

__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_fill_kernel(const SortParams p) {
  extern __shared__ uint8_t raw[];
  SortShared& s = *reinterpret_cast<SortShared*>(raw);
  chain_next();
  chain_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (blockIdx.x >= kSortCtas) {
    const int64_t step = (int64_t)(gridDim.x - kSortCtas) * kSortThreads;
    const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int64_t i = (int64_t)(blockIdx.x - kSortCtas) * kSortThreads + tid; i < p.vectors; i += 4 * step) {
      float4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = p.add && i + u * step < p.vectors ? p.add[i + u * step] : zero;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + u * step < p.vectors) p.table[i + u * step] = v[u];
    }
    return;
  }
  const uint32_t rank = blockIdx.x;  // (the first cluster of the grid)
  const uint32_t bins = 1u << p.digit;
  // each warp of the cluster has a stretch of its own, in whole rounds of 32
  const int64_t stretch = (p.rows + kSortCtas * kSortWarps * 32 - 1) / (kSortCtas * kSortWarps * 32) * 32;
  const int64_t lo = (int64_t)(rank * kSortWarps + warp) * stretch, hi = lo + stretch < p.rows ? lo + stretch : p.rows;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.digit;
    const uint32_t* keys_in = p.keys[(pass + 1) & 1];
    const uint32_t* from_in = p.from[(pass + 1) & 1];
    uint32_t* keys_out = p.keys[pass & 1];
    uint32_t* from_out = p.from[pass & 1];
    auto key_at = [&](int64_t i) {
      if (pass) return __ldcg(keys_in + i);
      const int64_t t = p.tokens[i];
      if (t >= p.vocab && p.status) *p.status = (int)HBP_ERR_INVALID_ARG;
      return t < 0 || t >= p.vocab ? (uint32_t)p.vocab : (uint32_t)t;  // no token: behind all others
    };
    for (uint32_t b = lane; b < bins; b += 32) s.counts[warp][b] = 0;
    __syncwarp();
    for (int64_t i = lo + lane; i < hi; i += 32) atomicAdd(&s.counts[warp][(key_at(i) >> shift) & (bins - 1)], 1u);
    __syncthreads();
    uint32_t total = 0;
    if (tid < (int)bins) {
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = s.counts[w][tid];
        s.counts[w][tid] = total;
        total += c;
      }
      s.totals[tid] = total;
    }
    tc::cluster_sync_whole_warps();
    uint32_t all = 0, before = 0;
    if (tid < (int)bins) {
      const uint32_t at = tc::smem_u32(&s.totals[tid]);
#pragma unroll
      for (uint32_t r = 0; r < kSortCtas; ++r) {
        const uint32_t c = ld_cluster(tc::map_to_cta(at, r));
        all += c;
        before += r < rank ? c : 0;
      }
    }
    uint32_t upto = all;  // of the warp's digits, this one's included
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) s.warp_sums[warp] = upto;
    __syncthreads();
    if (tid < (int)bins) {
      uint32_t first = 0;
      for (int w = 0; w < warp; ++w) first += s.warp_sums[w];
      s.base[tid] = first + upto - all + before;
    }
    __syncthreads();
    for (int64_t i0 = lo; i0 < hi; i0 += 32) {
      const int64_t i = i0 + lane;
      const bool in = i < hi;
      const uint32_t key = in ? key_at(i) : 0u, digit = in ? (key >> shift) & (bins - 1) : bins;
      const uint32_t row = in ? (pass ? __ldcg(from_in + i) : (uint32_t)i) : 0u;
      const uint32_t alike = __match_any_sync(0xffffffffu, digit), below = __popc(alike & ((1u << lane) - 1u));
      const uint32_t at = in ? s.base[digit] + s.counts[warp][digit] + below : 0u;
      __syncwarp();
      if (in && below == 0) s.counts[warp][digit] += __popc(alike);
      __syncwarp();
      if (in) {
        keys_out[at] = key;
        from_out[at] = row;
      }
    }
    tc::cluster_sync_whole_warps();  // what is written is seen by all; the totals have been read
  }
}

// ------------------------------------------------------------------------------------------- sums
struct SumParams {
  const uint32_t *keys, *from;  // tokens in order, and the rows that they are of
  int64_t rows, ldd, tiles;
  const void* d_out;
  int vocab, d;
  float scale;
  const float* add;
  float* table;
  float *head, *tail;  // [tiles][d]: of a run that began in an earlier tile; of one that began here and goes on
};

constexpr int kSumThreads = 128;
constexpr uint32_t kNoKey = 0xffffffffu;

template <typename T>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const SumParams p) {
  constexpr int V = Vec<T>::V, kAhead = 8;
  __shared__ uint32_t key[kTile + 2], from[kTile];
  chain_next();
  chain_wait();
  const int64_t first = (int64_t)blockIdx.x * kTile;
  const int n = p.rows - first < kTile ? (int)(p.rows - first) : kTile, tid = threadIdx.x;
  if (tid < kTile + 2) {  // (one before, one behind)
    const int64_t i = first + tid - 1;
    key[tid] = i >= 0 && i < p.rows ? p.keys[i] : kNoKey;
    if (tid >= 1 && tid <= n) from[tid - 1] = p.from[i];
  }
  __syncthreads();
  const int c = (int)(blockIdx.y * kSumThreads + tid) * V;
  if (c >= p.d) return;
  float acc[V];
#pragma unroll
  for (int e = 0; e < V; ++e) acc[e] = 0.0f;
  for (int j0 = 0; j0 < n; j0 += kAhead) {
    uint4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (j0 + u < n && key[j0 + u + 1] < (uint32_t)p.vocab)
        v[u] = *reinterpret_cast<const uint4*>((const T*)p.d_out + (int64_t)from[j0 + u] * p.ldd + c);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u;
      const uint32_t k = j < n ? key[j + 1] : kNoKey;
      if (k >= (uint32_t)p.vocab) return;  // the end, or rows without a token
      float f[V];
      Vec<T>::widen(v[u], f);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += f[e];
      const bool goes_on = key[j + 2] == k;
      if (goes_on && j + 1 < n) continue;
      float* to;
      float scale = 1.0f;
      const bool began_before = key[0] == k;  // (sorted: then the tile's first is k too)
      if (began_before) to = p.head + (int64_t)blockIdx.x * p.d + c;
      else if (goes_on) to = p.tail + (int64_t)blockIdx.x * p.d + c;
      else {
        to = p.table + (int64_t)k * p.d + c;
        scale = p.scale;
      }
      const bool add = p.add && !began_before && !goes_on;
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        float4 o = add ? *reinterpret_cast<const float4*>(p.add + (int64_t)k * p.d + c + e) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        o.x = fmaf(scale, acc[e], o.x);
        o.y = fmaf(scale, acc[e + 1], o.y);
        o.z = fmaf(scale, acc[e + 2], o.z);
        o.w = fmaf(scale, acc[e + 3], o.w);
        *reinterpret_cast<float4*>(to + e) = o;
        acc[e] = acc[e + 1] = acc[e + 2] = acc[e + 3] = 0.0f;
      }
    }
  }
}

constexpr int kJoinTiles = 8;  // a block looks at, a warp each; then eight stretches of a run's tiles, a warp each

__global__ void __launch_bounds__(32 * kJoinTiles) join_kernel(const SumParams p) {
  __shared__ int64_t last[kJoinTiles];  // tile of the run that begins in a tile and goes on
  __shared__ uint32_t token[kJoinTiles];
  __shared__ float4 part[kJoinTiles][32];
  chain_next();
  chain_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) {
    const int64_t tile = (int64_t)blockIdx.x * kJoinTiles + warp, at = tile * kTile, next = at + kTile;
    int64_t end = -1;
    if (next < p.rows) {
      const uint32_t k = p.keys[next];
      if (k < (uint32_t)p.vocab && p.keys[next - 1] == k && !(at > 0 && p.keys[at - 1] == k)) {
        int64_t lo = next, hi = p.rows;  // keys[lo] is k; hi is behind the run
        while (hi - lo > 1) {
          const int64_t mid = lo + (hi - lo) / 2;
          if (p.keys[mid] == k) lo = mid;
          else hi = mid;
        }
        end = lo / kTile;
        token[warp] = k;
      }
    }
    last[warp] = end;
  }
  __syncthreads();
  const int c = (int)(blockIdx.y * 32 + lane) * 4;
  for (int w = 0; w < kJoinTiles; ++w) {
    if (last[w] < 0) continue;
    const int64_t tile = (int64_t)blockIdx.x * kJoinTiles + w, count = last[w] - tile, per = (count + kJoinTiles - 1) / kJoinTiles;
    const int64_t lo = tile + 1 + warp * per, hi = lo + per < last[w] + 1 ? lo + per : last[w] + 1;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < p.d) {
      if (warp == 0) sum = *reinterpret_cast<const float4*>(p.tail + tile * p.d + c);
#pragma unroll 8
      for (int64_t i = lo; i < hi; ++i) {
        const float4 v = *reinterpret_cast<const float4*>(p.head + i * p.d + c);
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
      }
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && c < p.d) {
#pragma unroll
      for (int g = 1; g < kJoinTiles; ++g) {
        const float4 v = part[g][lane];
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
      }
      const int64_t at = (int64_t)token[w] * p.d + c;
      float4 o = p.add ? *reinterpret_cast<const float4*>(p.add + at) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      o.x = fmaf(p.scale, sum.x, o.x);
      o.y = fmaf(p.scale, sum.y, o.y);
      o.z = fmaf(p.scale, sum.z, o.z);
      o.w = fmaf(p.scale, sum.w, o.w);
      *reinterpret_cast<float4*>(p.table + at) = o;
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------- host
constexpr int64_t kMostRows = 1ll << 30;

hbp_status check_sizes(int dtype, int64_t rows, int vocab, int d) {
  if (dtype != HBP_F32 && dtype != HBP_BF16) return HBP_ERR_DTYPE;
  const int v = dtype == HBP_F32 ? 4 : 8;
  if (rows < 0 || rows > kMostRows || vocab <= 0 || vocab > kMostRows || d <= 0 || d % v || d > 65535 * kSumThreads) return HBP_ERR_SHAPE;
  return HBP_OK;
}
hbp_status check_tokens(const void* tokens, int bytes, const int* status) {
  if (bytes != 4 && bytes != 8) return HBP_ERR_INVALID_ARG;
  if (((uintptr_t)tokens % bytes) || ((uintptr_t)status & 3u)) return HBP_ERR_SHAPE;
  return HBP_OK;
}
// rows `ld` elements apart; inputs may be one row for all
bool bad_rows(const void* t, int64_t ld, int d, int v, bool input) { return ((uintptr_t)t & 15u) || ld % v || (ld < d && !(input && ld == 0)); }

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }
struct Scratch {
  size_t list, sums, bytes;  // of a list of the sorted tokens; of a list of partial sums; of all
  int64_t tiles;
  Scratch(int64_t rows, int d) {
    tiles = (rows + kTile - 1) / kTile;
    list = up((size_t)rows * 4);
    sums = up((size_t)tiles * d * 4);
    bytes = 4 * list + 2 * sums;
  }
};

}  // namespace

}  // namespace hbp

using namespace hbp;

extern "C" hbp_status hbp_embedding(int32_t dtype, int64_t rows, int32_t vocab, int32_t d, const void* tokens, int32_t token_bytes, const void* table,
                                    int64_t ldt, float scale, void* out, int64_t ldo, int32_t* status, void* cuda_stream) {
  hbp_status st = check_sizes(dtype, rows, vocab, d);
  if (st != HBP_OK) return st;
  if ((st = check_tokens(tokens, token_bytes, status)) != HBP_OK) return st;
  if (!(scale - scale == 0.0f)) return HBP_ERR_INVALID_ARG;
  if (rows == 0) return HBP_OK;
  if (!tokens || !table || !out) return HBP_ERR_INVALID_ARG;
  const int v = dtype == HBP_F32 ? 4 : 8;
  if (bad_rows(table, ldt, d, v, true) || bad_rows(out, ldo, d, v, false)) return HBP_ERR_SHAPE;
  LookupParams p;
  p.tokens = {tokens, token_bytes};
  p.rows = rows; p.ldt = ldt; p.ldo = ldo;
  p.table = table; p.out = out;
  p.vocab = vocab;
  p.per_row = d / v;
  p.by_row = divider((uint32_t)p.per_row);
  p.scale = scale;
  p.status = status;
  const int64_t blocks = (rows * p.per_row + kThreads * kBatch - 1) / (kThreads * kBatch);
  if (blocks > INT32_MAX) return HBP_ERR_SHAPE;
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  launch_chained(lc, dtype == HBP_F32 ? lookup_kernel<float> : lookup_kernel<bf16>, dim3((unsigned)blocks), kThreads, 0, 1, p);
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}

extern "C" hbp_status hbp_embedding_gradient_scratch_bytes(int64_t rows, int32_t d, size_t* bytes) {
  if (!bytes) return HBP_ERR_INVALID_ARG;
  if (rows < 0 || rows > kMostRows || d <= 0) return HBP_ERR_SHAPE;
  *bytes = Scratch(rows, d).bytes;
  return HBP_OK;
}

extern "C" hbp_status hbp_embedding_gradient(int32_t dtype, int64_t rows, int32_t vocab, int32_t d, const void* tokens, int32_t token_bytes,
                                             const void* d_out, int64_t ldd, float scale, const float* add, float* d_table, void* scratch,
                                             size_t scratch_bytes, int32_t* status, void* cuda_stream) {
  hbp_status st = check_sizes(dtype, rows, vocab, d);
  if (st != HBP_OK) return st;
  if ((st = check_tokens(tokens, token_bytes, status)) != HBP_OK) return st;
  if (!(scale - scale == 0.0f)) return HBP_ERR_INVALID_ARG;
  if (!d_table || (rows && (!tokens || !d_out))) return HBP_ERR_INVALID_ARG;
  if (((uintptr_t)d_table & 15u) || ((uintptr_t)add & 15u) || (rows && bad_rows(d_out, ldd, d, dtype == HBP_F32 ? 4 : 8, true))) return HBP_ERR_SHAPE;
  const Scratch need(rows, d);
  if (rows && (!scratch || ((uintptr_t)scratch & 15u) || scratch_bytes < need.bytes)) return HBP_ERR_WORKSPACE;
  if (need.tiles > INT32_MAX) return HBP_ERR_SHAPE;
  const bool in_place = add == d_table;
  if (rows == 0 && in_place) return HBP_OK;
  static PerDevice<bool> attr_done;
  if (!attr_done.here()) {
    if (cudaFuncSetAttribute(sort_fill_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared)) != cudaSuccess) {
      cudaGetLastError();
      return HBP_ERR_CUDA;
    }
    attr_done.here() = true;
  }
  uint8_t* at = (uint8_t*)scratch;
  SortParams s = {};
  s.tokens = {tokens, token_bytes};
  s.rows = rows;
  s.vocab = vocab;
  int bits = 1;
  while (((uint32_t)vocab >> bits) != 0) ++bits;  // keys go up to vocab itself
  s.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  s.digit = (bits + s.passes - 1) / s.passes;
  if (rows == 0) s.passes = 0;
  for (int i = 0; i < 2 && rows; ++i) {
    s.keys[i] = (uint32_t*)(at + 2 * i * need.list);
    s.from[i] = (uint32_t*)(at + (2 * i + 1) * need.list);
  }
  s.status = status;
  s.table = (float4*)d_table;
  s.add = (const float4*)add;
  s.vectors = in_place ? 0 : (int64_t)vocab * d / 4;
  // clusters of eight that fill a GPU with one block an SM, and no more than have a quarter of a block's round each
  const int64_t wanted = (s.vectors + kSortThreads * kSortCtas - 1) / (kSortThreads * kSortCtas), most = tc::sm_count() / kSortCtas - 1;
  const int fill = (int)(wanted < most ? wanted : most > 0 ? most : 1);
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  launch_chained(lc, sort_fill_kernel, dim3(kSortCtas * (1 + fill)), kSortThreads, sizeof(SortShared), kSortCtas, s);
  if (rows) {
    SumParams p;
    const int last = (s.passes - 1) & 1;
    p.keys = s.keys[last]; p.from = s.from[last];
    p.rows = rows; p.ldd = ldd; p.tiles = need.tiles;
    p.d_out = d_out;
    p.vocab = vocab; p.d = d;
    p.scale = scale;
    p.add = add;
    p.table = d_table;
    p.head = (float*)(at + 4 * need.list);
    p.tail = (float*)(at + 4 * need.list + need.sums);
    const int per_row = d / (dtype == HBP_F32 ? 4 : 8);
    const dim3 grid((unsigned)p.tiles, (per_row + kSumThreads - 1) / kSumThreads);
    launch_chained(lc, dtype == HBP_F32 ? sum_kernel<float> : sum_kernel<bf16>, grid, kSumThreads, 0, 1, p);
    if (p.tiles > 1)
      launch_chained(lc, join_kernel, dim3((unsigned)((p.tiles + kJoinTiles - 1) / kJoinTiles), (d + 127) / 128), 32 * kJoinTiles, 0, 1, p);
  }
  return lc.err == cudaSuccess ? HBP_OK : HBP_ERR_CUDA;
}
