// Rows of a table by tokens, scaled, and the table's gradient (hbp_embedding, hbp_embedding_gradient).
//
// Gradient: d_table[v] = add[v] + scale * sum of d_out[i] over the rows i whose token is v, in three launches.
//  1. One cluster of eight blocks (a block alone up to 2048 tokens) sorts the tokens with their rows: stable, by digits of up to 9 bits, least first, 18
//     bits, which most vocabularies need, in two passes; 16384 tokens 22 us, 262144 150, of one block 14 for 1000.  Meanwhile the other blocks of the
//     launch clear the table, or copy `add`: 50021 x 768 floats 24 us, which is what bounds such a step.
//  2. Blocks add up the rows of 16 to 128 sorted tokens each, whole runs of one token straight to the table.  The share of a run that began in an
//     earlier tile, or goes on in the next, is a partial sum in scratch.  Bound by bytes and by the wait for tokens, then rows: 16384 tokens of 768
//     bf16 channels 13 us.
//  3. Those runs' partial sums are added in the order of the tiles, eight stretches of them at a time (7 us).
// Every sum has a fixed order: runs agree bit for bit.  The longest chain of float additions is a tile, an eighth of a run's tiles, and eight.  A run's partial sums are
// one block's for 128 channels, so that a token that is every second one costs: of 16384 tokens of 50021 x 768 bf16 channels 55 us (52 where all are equally
// frequent), of 65536 159 (121, of which joins 12; then 71), of 2^20 911 (886).
// All of it, with the lookup (8 us): 16384 tokens of 50021 x 768, 57 us of 35 for the bytes; 5003 of 10007 x 1492 floats added to another gradient 47 of 32.
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
// Up to so many tokens one block sorts, in shared memory: no exchange.
constexpr int kAlone = 2048;
// Sorted tokens a block adds up: 16, and more of more than 65536, whose longest runs would have too many parts to join.
constexpr int kLeastTile = 16, kMostTile = 128;
constexpr int64_t kTilesBefore = 4096;  // tiles there are before they grow

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
  uint32_t counts[kSortWarps][kMaxBins + 1];  // of a warp's tokens, then where the next one of a digit goes (a digit's column has 32 banks)
  uint32_t totals[kMaxBins];                  // of a block's, read by the others
  uint32_t base[kMaxBins];
  uint32_t warp_sums[kSortWarps];
  uint32_t keys[2][kAlone], from[2][kAlone];
};

__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// kAdd: filled from add
template <bool kAdd>
__device__ __forceinline__ void fill(const SortParams& p, int block, int blocks) {
  // 64 KB at a time, each block's own: 154 MB 24 us (38 with every thread's four vectors as far apart as the blocks together are wide)
  for (int64_t i = ((int64_t)block * 4) * kSortThreads + threadIdx.x; i < p.vectors; i += (int64_t)blocks * 4 * kSortThreads) {
    float4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = kAdd && i + u * kSortThreads < p.vectors ? __ldcs(p.add + i + u * kSortThreads) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * kSortThreads < p.vectors) p.table[i + u * kSortThreads] = v[u];
  }
}

__global__ void __launch_bounds__(kSortThreads, 1) sort_fill_kernel(const SortParams p) {
  extern __shared__ uint8_t raw[];
  SortShared& s = *reinterpret_cast<SortShared*>(raw);
  chain_next();
  chain_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (blockIdx.x >= kSortCtas) {
    if (p.add) fill<true>(p, blockIdx.x - kSortCtas, gridDim.x - kSortCtas);
    else fill<false>(p, blockIdx.x - kSortCtas, gridDim.x - kSortCtas);
    return;
  }
  const uint32_t rank = blockIdx.x;  // (the first cluster of the grid)
  const bool alone = p.rows <= kAlone;
  if (alone && rank) return;
  const uint32_t bins = 1u << p.digit;
  // each warp has a stretch of its own, in whole rounds of 32
  const int64_t warps = (alone ? 1 : kSortCtas) * kSortWarps, stretch = (p.rows + warps * 32 - 1) / (warps * 32) * 32;
  const int64_t lo = (int64_t)(rank * kSortWarps + warp) * stretch, hi = lo + stretch < p.rows ? lo + stretch : p.rows;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.digit;
    const bool last = pass == p.passes - 1;
    const uint32_t* keys_in = p.keys[(pass + 1) & 1];
    const uint32_t* from_in = p.from[(pass + 1) & 1];
    uint32_t* keys_out = alone && !last ? s.keys[pass & 1] : p.keys[pass & 1];
    uint32_t* from_out = alone && !last ? s.from[pass & 1] : p.from[pass & 1];
    bool beyond = false;
    auto key_at = [&](int64_t i) {
      if (pass) return alone ? s.keys[(pass + 1) & 1][i] : __ldcg(keys_in + i);
      const int64_t t = p.tokens[i];
      beyond = beyond || t >= p.vocab;
      return t < 0 || t >= p.vocab ? (uint32_t)p.vocab : (uint32_t)t;  // no token: behind all others
    };
    auto row_at = [&](int64_t i) { return pass ? (alone ? s.from[(pass + 1) & 1][i] : __ldcg(from_in + i)) : (uint32_t)i; };
    for (uint32_t b = lane; b < bins; b += 32) s.counts[warp][b] = 0;
    __syncwarp();
    constexpr int kAhead = 8;  // rounds asked for at once
    for (int64_t i0 = lo + lane; i0 < hi; i0 += 32 * kAhead) {
      uint32_t key[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) key[k] = i0 + 32 * k < hi ? key_at(i0 + 32 * k) : 0u;
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + 32 * k < hi) atomicAdd(&s.counts[warp][(key[k] >> shift) & (bins - 1)], 1u);
    }
    if (beyond && p.status) *p.status = (int)HBP_ERR_INVALID_ARG;
    __syncthreads();
    // a warp takes every 32nd digit: its lanes the warps' counts, in their order
    for (uint32_t b = warp; b < bins; b += kSortWarps) {
      const uint32_t c = s.counts[lane][b];
      uint32_t upto = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      s.counts[lane][b] = upto - c;
      if (lane == 31) s.totals[b] = upto;
    }
    if (alone) __syncthreads();
    else tc::cluster_sync_whole_warps();
    uint32_t all = 0, before = 0;
    if (tid < (int)bins) {
      if (alone) {
        all = s.totals[tid];
      } else {
        const uint32_t at = tc::smem_u32(&s.totals[tid]);
#pragma unroll
        for (uint32_t r = 0; r < kSortCtas; ++r) {
          const uint32_t c = ld_cluster(tc::map_to_cta(at, r));
          all += c;
          before += r < rank ? c : 0;
        }
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
#pragma unroll
      for (int w = 0; w < kMaxBins / 32; ++w) first += w < warp ? s.warp_sums[w] : 0;
      s.base[tid] = first + upto - all + before;
    }
    __syncthreads();
    auto place = [&](bool in, uint32_t key) {
      // the lanes that have the same digit, bit by bit (__match_any_sync takes a turn for each value among them: 1 us for 32 of them in all warps)
      const uint32_t digit = (key >> shift) & (bins - 1);
      uint32_t alike = __ballot_sync(0xffffffffu, in);
      for (int b = 0; b < p.digit; ++b) {
        const uint32_t set = __ballot_sync(0xffffffffu, (digit >> b) & 1u);
        alike &= (digit >> b) & 1u ? set : ~set;
      }
      const uint32_t below = __popc(alike & ((1u << lane) - 1u));
      const uint32_t at = in ? s.base[digit] + s.counts[warp][digit] + below : 0u;
      __syncwarp();
      if (in && below == 0) s.counts[warp][digit] += __popc(alike);
      __syncwarp();
      return at;
    };
    for (int64_t i0 = lo; i0 < hi; i0 += 32 * kAhead) {
      uint32_t key[kAhead], row[kAhead], at[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int64_t i = i0 + 32 * k + lane;
        key[k] = i < hi ? key_at(i) : 0u;
        row[k] = i < hi ? row_at(i) : 0u;
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + 32 * k < hi) at[k] = place(i0 + 32 * k + lane < hi, key[k]);
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + 32 * k + lane < hi) {
          keys_out[at[k]] = key[k];
          from_out[at[k]] = row[k];
        }
    }
    if (alone) {
      __syncthreads();
      continue;
    }
    tc::cluster_sync_whole_warps();  // what is written is seen by all; the totals have been read
  }
}

// ------------------------------------------------------------------------------------------- sums
struct SumParams {
  const uint32_t *keys, *from;  // tokens in order, and the rows that they are of
  int64_t rows, ldd, tiles;
  int tile;
  const void* d_out;
  int vocab, d;
  float scale;
  bool add;
  float* table;
  float *head, *tail;  // [tiles][d]: of a run that began in an earlier tile; of one that began here and goes on
};

// Four floats added to what the table has (`add`: it has been copied there, or is the table).  Each element is added to once a call, so the order of
// these is no matter; nothing waits for what was there: a thread that read it lost a memory's latency at the end of each run, 65536 tokens, of
// which 36 thousand differ, 88 us.
__device__ __forceinline__ void add4(float* to, const float4& v) {
  asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(to), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

constexpr int kSumThreads = 128;
constexpr uint32_t kNoKey = 0xffffffffu;

template <typename T>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const SumParams p) {
  constexpr int V = Vec<T>::V, kAhead = 8;
  __shared__ uint32_t key[kMostTile + 2], from[kMostTile];
  chain_next();
  chain_wait();
  const int64_t first = (int64_t)blockIdx.x * p.tile;
  const int n = p.rows - first < p.tile ? (int)(p.rows - first) : p.tile, tid = threadIdx.x;
  for (int k = tid; k < p.tile + 2; k += kSumThreads) {  // (one before, one behind)
    const int64_t i = first + k - 1;
    key[k] = i >= 0 && i < p.rows ? p.keys[i] : kNoKey;
    if (k >= 1 && k <= n) from[k - 1] = p.from[i];
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
        const float4 o = make_float4(scale * acc[e], scale * acc[e + 1], scale * acc[e + 2], scale * acc[e + 3]);
        if (add) add4(to + e, o);
        else *reinterpret_cast<float4*>(to + e) = o;
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
  {
    const int64_t tile = (int64_t)blockIdx.x * kJoinTiles + warp, at = tile * p.tile, next = at + p.tile;
    int64_t end = -1;
    if (next < p.rows) {
      const uint32_t k = p.keys[next], in = p.keys[next - 1], before = at > 0 ? p.keys[at - 1] : kNoKey;
      if (k < (uint32_t)p.vocab && in == k && before != k) {
        // the last tile whose first token is k: of 32 at a time, then of those between two of them
        int64_t lo = tile + 1, hi = p.tiles - 1;  // lo is one, none is behind hi
        for (int64_t step = 1; lo < hi;) {
          const int64_t i = lo + step * (lane + 1);
          const uint32_t same = __ballot_sync(0xffffffffu, i <= hi && p.keys[i * p.tile] == k);
          const int n = __ffs(~same) - 1;  // (sorted: the first n; -1 for all)
          lo += step * (n < 0 ? 32 : n);
          if (n >= 0) {
            hi = min(hi, lo + step - 1);
            step = (hi - lo + 31) / 32;
          } else {
            step *= 32;
          }
        }
        end = lo;
        if (lane == 0) token[warp] = k;
      }
    }
    if (lane == 0) last[warp] = end;
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
#pragma unroll 16
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
      float* to = p.table + (int64_t)token[w] * p.d + c;
      const float4 o = make_float4(p.scale * sum.x, p.scale * sum.y, p.scale * sum.z, p.scale * sum.w);
      if (p.add) add4(to, o);
      else *reinterpret_cast<float4*>(to) = o;
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
  size_t asked;              // of all, and as much as fewer rows take
  int tile;
  int64_t tiles;
  Scratch(int64_t rows, int d) {
    for (tile = kLeastTile; tile < kMostTile && rows > kTilesBefore * tile; tile *= 2) {
    }
    tiles = (rows + tile - 1) / tile;
    list = up((size_t)rows * 4);
    sums = up((size_t)tiles * d * 4);
    bytes = 4 * list + 2 * sums;
    // (65537 rows have half the tiles that 65536 have: the most are those of the last number of rows that the smaller tiles are for)
    const int64_t most = tile > kLeastTile && tiles < kTilesBefore ? kTilesBefore : tiles;
    asked = 4 * list + 2 * up((size_t)most * d * 4);
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
  *bytes = Scratch(rows, d).asked;
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
  // as many clusters beside the first as run at a time (15 in all: 18 took two turns, 154 MB 40 us), and no more than have 64 KB a block
  const int64_t wanted = (s.vectors + 4 * kSortThreads * kSortCtas - 1) / (4 * kSortThreads * kSortCtas);
  const int fill = (int)(wanted < 14 ? wanted : 14);
  Launcher lc;
  lc.stream = (cudaStream_t)cuda_stream;
  launch_chained(lc, sort_fill_kernel, dim3(kSortCtas * (1 + fill)), kSortThreads, sizeof(SortShared), kSortCtas, s);
  if (rows) {
    SumParams p;
    const int last = (s.passes - 1) & 1;
    p.keys = s.keys[last]; p.from = s.from[last];
    p.rows = rows; p.ldd = ldd; p.tiles = need.tiles; p.tile = need.tile;
    p.d_out = d_out;
    p.vocab = vocab; p.d = d;
    p.scale = scale;
    p.add = add != nullptr;
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
