// Embedding lookup with scaling, and its weight gradient from sorted tokens.
//
//   out[t] = scale table[ids[t]];     dW[v] = scale sum_{t : ids[t] = v} dOut[t]
//
// The gradient adds whole rows of dOut that share an id.  Atomics would add them in any order; here the tokens are sorted
// by id first (a stable radix sort of (id, t), so that equal ids keep the order of t), and runs of equal ids are summed
// front to back: the same bits from call to call.  The sorted tokens are cut into chunks of equal length, whatever the ids,
// so that one frequent id does not keep a single CTA busy: a run inside a chunk goes to dW at once, the pieces of a run
// that crosses chunks meet in a last launch, in order.
//
// What bounds it: dOut read once and dW written once (overwriting: all of it, rows without tokens as zeros).
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "asi_internal.h"

namespace asi {

namespace {

constexpr int kEmbThreads = 256;

template <typename T>
__device__ __forceinline__ float as_float(T v);
template <>
__device__ __forceinline__ float as_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float& o, float v) { o = v; }
__device__ __forceinline__ void from_float(__nv_bfloat16& o, float v) { o = __float2bfloat16_rn(v); }

template <typename T, int N>
struct __align__(sizeof(T) * N) Pack {
  T v[N];
};

// n consecutive values as floats; loads of up to 16 bytes
template <typename T, int N>
__device__ __forceinline__ void load_values(const T* p, float* f) {
  constexpr int kEach = sizeof(T) * N > 16 ? 16 / (int)sizeof(T) : N;
#pragma unroll
  for (int i = 0; i < N; i += kEach) {
    const Pack<T, kEach> a = *reinterpret_cast<const Pack<T, kEach>*>(p + i);
#pragma unroll
    for (int e = 0; e < kEach; ++e) f[i + e] = as_float<T>(a.v[e]);
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_values(T* p, const float* f) {
  constexpr int kEach = sizeof(T) * N > 16 ? 16 / (int)sizeof(T) : N;
#pragma unroll
  for (int i = 0; i < N; i += kEach) {
    Pack<T, kEach> a;
#pragma unroll
    for (int e = 0; e < kEach; ++e) from_float(a.v[e], f[i + e]);
    *reinterpret_cast<Pack<T, kEach>*>(p + i) = a;
  }
}

// ---- lookup: one thread for VEC values of a row
struct LookupArgs {
  const void* table;
  const int64_t* ids;
  void* out;
  int64_t V, D, items;      // items = tokens * ceil(D / VEC)
  int per_row;
  float scale;
};

template <typename TT, typename TO, int VEC>
__global__ void __launch_bounds__(kEmbThreads) k_embed(const __grid_constant__ LookupArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  for (int64_t i = (int64_t)blockIdx.x * kEmbThreads + threadIdx.x; i < p.items; i += (int64_t)gridDim.x * kEmbThreads) {
    const int64_t t = i / p.per_row;
    const int64_t col = (i - t * p.per_row) * VEC;
    const int64_t id = p.ids[t];
    float f[VEC];
    if (id >= 0 && id < p.V) {
      load_values<TT, VEC>(static_cast<const TT*>(p.table) + id * p.D + col, f);
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] *= p.scale;
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) f[e] = NAN;
    }
    store_values<TO, VEC>(static_cast<TO*>(p.out) + t * p.D + col, f);
  }
}

// ---- stable radix sort of (id, t): tiles of kTile tokens, digits of up to ten bits
constexpr int kSortItems = 8;
constexpr int kTile = kEmbThreads * kSortItems;
constexpr int kSortWarps = kEmbThreads / 32;
constexpr int kMaxBins = 1024;

struct SortArgs {
  const int64_t* ids;       // first pass; else null
  const uint32_t *key_in, *pos_in;
  uint32_t *key_out, *pos_out;
  uint32_t* hist;           // [tiles][bins]
  int64_t V, padding;
  int T, tiles, shift, bits;
};

// The token's key: its id, or V (sorted behind all ids) where it contributes nothing.
__device__ __forceinline__ uint32_t token_key(const SortArgs& p, int i) {
  if (!p.ids) return p.key_in[i];
  const int64_t id = p.ids[i];
  return id >= 0 && id < p.V && id != p.padding ? (uint32_t)id : (uint32_t)p.V;
}

__global__ void __launch_bounds__(kEmbThreads) k_sort_hist(const __grid_constant__ SortArgs p) {
  __shared__ uint32_t h[kMaxBins];
  const int bins = 1 << p.bits;
  for (int b = threadIdx.x; b < bins; b += kEmbThreads) h[b] = 0;
  pdl_wait();
  pdl_launch_dependents();
  __syncthreads();
  for (int i = threadIdx.x; i < kTile; i += kEmbThreads) {
    const int at = blockIdx.x * kTile + i;
    if (at < p.T) atomicAdd(&h[(token_key(p, at) >> p.shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kEmbThreads) p.hist[(int64_t)blockIdx.x * bins + b] = h[b];
}

// exclusive sum over the CTA's threads
__device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t* warp_sum, int warps) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(~0u, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sum[warp] = x;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < warp; ++w) before += warp_sum[w];
  __syncthreads();
  return before + x - v;
}

__global__ void __launch_bounds__(kEmbThreads) k_sort_scatter(const __grid_constant__ SortArgs p) {
  __shared__ uint16_t wh[kSortWarps][kMaxBins];      // per warp: tokens of each digit so far, then those of earlier warps
  __shared__ uint32_t start[kMaxBins];
  __shared__ uint32_t warp_sum[kSortWarps];
  const int bins = 1 << p.bits, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  for (int b = tid; b < kSortWarps * kMaxBins; b += kEmbThreads) (&wh[0][0])[b] = 0;
  pdl_wait();
  pdl_launch_dependents();
  // where each digit's tokens of this tile start
  const int each = (bins + kEmbThreads - 1) / kEmbThreads;
  uint32_t sum = 0, mine[kMaxBins / kEmbThreads], total[kMaxBins / kEmbThreads];
#pragma unroll
  for (int e = 0; e < kMaxBins / kEmbThreads; ++e) {
    mine[e] = total[e] = 0;
    const int b = tid * each + e;
    if (e >= each || b >= bins) continue;
    for (int t = 0; t < p.tiles; ++t) {
      const uint32_t c = p.hist[(int64_t)t * bins + b];
      if (t < (int)blockIdx.x) mine[e] += c;
      total[e] += c;
    }
    sum += total[e];
  }
  uint32_t run = block_exclusive(sum, warp_sum, kSortWarps);
#pragma unroll
  for (int e = 0; e < kMaxBins / kEmbThreads; ++e) {
    const int b = tid * each + e;
    if (e >= each || b >= bins) continue;
    start[b] = run + mine[e];
    run += total[e];
  }
  __syncthreads();
  uint32_t key[kSortItems], pos[kSortItems];
  uint16_t rank[kSortItems];
  const int base = blockIdx.x * kTile + warp * 32 * kSortItems + lane;
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int at = base + i * 32;
    if (at < p.T) key[i] = token_key(p, at), pos[i] = p.ids ? at : p.pos_in[at];
  }
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const bool on = base + i * 32 < p.T;
    const uint32_t active = __ballot_sync(~0u, on);
    if (on) {
      const uint32_t d = (key[i] >> p.shift) & (bins - 1);
      const uint32_t peers = __match_any_sync(active, d);
      const uint16_t before = wh[warp][d];
      __syncwarp(active);
      if (lane == __ffs(peers) - 1) wh[warp][d] = before + __popc(peers);
      rank[i] = before + __popc(peers & ((1u << lane) - 1));
    }
    __syncwarp();
  }
  __syncthreads();
  for (int b = tid; b < bins; b += kEmbThreads) {
    uint16_t so_far = 0;
    for (int w = 0; w < kSortWarps; ++w) {
      const uint16_t c = wh[w][b];
      wh[w][b] = so_far;
      so_far += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i)
    if (base + i * 32 < p.T) {
      const uint32_t d = (key[i] >> p.shift) & (bins - 1);
      const uint32_t to = start[d] + wh[warp][d] + rank[i];
      p.key_out[to] = key[i];
      p.pos_out[to] = pos[i];
    }
}

// ---- sums of runs
constexpr int kMaxChunk = 64;
constexpr int kZeroRows = 16;

struct SumArgs {
  const void* dout;
  const uint32_t *key, *pos;
  float* dW;
  float *head, *tail;       // [chunks][D]: the chunk's piece of a run that starts earlier / here and goes on
  int64_t D;
  uint32_t V;
  int T, C, chunks, accumulate;
  float scale;
};

template <int VEC>
__device__ __forceinline__ void put_row(const SumArgs& p, uint32_t v, int64_t col, const float* acc) {
  float* o = p.dW + (int64_t)v * p.D + col;
  float f[VEC];
  if (p.accumulate) load_values<float, VEC>(o, f);
#pragma unroll
  for (int e = 0; e < VEC; ++e) f[e] = p.accumulate ? fmaf(p.scale, acc[e], f[e]) : p.scale * acc[e];
  store_values<float, VEC>(o, f);
}

// first place whose key is not below v
__device__ __forceinline__ int lower_bound(const uint32_t* key, int n, uint32_t v) {
  int lo = 0;
  while (n > 0) {
    const int half = n >> 1;
    if (key[lo + half] < v) lo += half + 1, n -= half + 1;
    else n = half;
  }
  return lo;
}

// CTAs [0, chunks): sums.  CTAs behind them (overwriting): rows of dW without tokens.
template <typename T, int VEC>
__global__ void __launch_bounds__(kEmbThreads) k_embed_sum(const __grid_constant__ SumArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  const int64_t col = ((int64_t)blockIdx.y * kEmbThreads + threadIdx.x) * VEC;
  if ((int)blockIdx.x >= p.chunks) {
    __shared__ int empty[kZeroRows];
    const int64_t v0 = (int64_t)(blockIdx.x - p.chunks) * kZeroRows;
    if (threadIdx.x < kZeroRows) {
      const uint32_t v = (uint32_t)(v0 + threadIdx.x);
      const int at = lower_bound(p.key, p.T, v);
      empty[threadIdx.x] = v < p.V && (at == p.T || p.key[at] != v);
    }
    __syncthreads();
    if (col >= p.D) return;
    float f[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = 0.f;
    for (int r = 0; r < kZeroRows; ++r)
      if (empty[r]) store_values<float, VEC>(p.dW + (v0 + r) * p.D + col, f);
    return;
  }
  __shared__ uint32_t sk[kMaxChunk + 2], sp[kMaxChunk];
  const int c = blockIdx.x, c0 = c * p.C, m = min(p.C, p.T - c0);
  // sk[0] is the key before the chunk, sk[m + 1] the one behind it; V where there is none
  for (int i = threadIdx.x; i < m + 2; i += kEmbThreads) {
    const int at = c0 + i - 1;
    sk[i] = at < 0 || at >= p.T ? p.V : p.key[at];
    if (i >= 1 && i <= m) sp[i - 1] = p.pos[at];
  }
  __syncthreads();
  if (col >= p.D) return;
  constexpr int U = 4;
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  bool from_before = sk[0] == sk[1];
  const T* src = static_cast<const T*>(p.dout) + col;
  for (int i0 = 0; i0 < m && sk[i0 + 1] != p.V; i0 += U) {
    float f[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u < m && sk[i0 + u + 1] != p.V) load_values<T, VEC>(src + (int64_t)sp[i0 + u] * p.D, f[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u;
      if (i >= m || sk[i + 1] == p.V) break;
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += f[u][e];
      const bool ends = sk[i + 2] != sk[i + 1];
      if (!ends && i + 1 < m) continue;
      if (from_before) store_values<float, VEC>(p.head + (int64_t)c * p.D + col, acc);
      else if (!ends) store_values<float, VEC>(p.tail + (int64_t)c * p.D + col, acc);
      else put_row<VEC>(p, sk[i + 1], col, acc);
      from_before = false;
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    }
  }
}

// The runs that cross chunks: chunk c's CTA joins the pieces of the run that starts in c and goes on behind it.
template <int VEC>
__global__ void __launch_bounds__(kEmbThreads) k_embed_join(const __grid_constant__ SumArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  const int c = blockIdx.x, c0 = c * p.C, c1 = c0 + p.C;
  if (c1 >= p.T) return;
  const uint32_t v = p.key[c1];
  if (v == p.V || p.key[c1 - 1] != v) return;                        // nothing goes on
  if (p.key[c0] == v && c0 > 0 && p.key[c0 - 1] == v) return;        // it started earlier
  const int64_t col = ((int64_t)blockIdx.y * kEmbThreads + threadIdx.x) * VEC;
  if (col >= p.D) return;
  const int last = (lower_bound(p.key + c1, p.T - c1, v + 1) + c1 - 1) / p.C;   // the chunk that holds its last token
  float acc[VEC], f[VEC];
  load_values<float, VEC>(p.tail + (int64_t)c * p.D + col, acc);
  for (int q = c + 1; q <= last; ++q) {
    load_values<float, VEC>(p.head + (int64_t)q * p.D + col, f);
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] += f[e];
  }
  put_row<VEC>(p, v, col, acc);
}

// ---- host side
struct Layout {
  int T, C, chunks, tiles, passes, bits;
  size_t key[2], pos[2], hist, head, tail, bytes;
};

Layout layout_of(const asi_embedding_desc_t* d) {
  Layout l = {};
  l.T = (int)d->tokens;
  // chunks of 8 to 64 tokens, four CTAs an SM where there are tokens enough
  constexpr int kMost = 148 * 4;
  l.C = 8;
  while (l.C < kMaxChunk && l.T > l.C * kMost) l.C *= 2;
  l.chunks = (l.T + l.C - 1) / l.C;
  // the most chunks of any shorter batch: a workspace serves fewer tokens too
  const size_t most = std::max(std::min((l.T + 7) / 8, kMost), (l.T + kMaxChunk - 1) / kMaxChunk);
  l.tiles = (l.T + kTile - 1) / kTile;
  int bits = 1;
  while ((d->vocab >> bits) != 0) ++bits;             // keys up to vocab itself
  l.passes = bits <= 8 ? 1 : bits <= 20 ? 2 : (bits + 9) / 10;
  l.bits = (bits + l.passes - 1) / l.passes;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes, 256);
    return here;
  };
  for (int i = 0; i < 2; ++i) {
    l.key[i] = take((size_t)l.T * 4);
    l.pos[i] = take((size_t)l.T * 4);
  }
  l.hist = take(((size_t)l.tiles << l.bits) * 4);
  l.head = take(most * d->dim * 4);
  l.tail = take(most * d->dim * 4);
  l.bytes = std::max<size_t>(at, 256);
  return l;
}

asi_status_t check_desc(const asi_embedding_desc_t* d) {
  if (!d || (d->in_dtype != ASI_F32 && d->in_dtype != ASI_BF16)) return ASI_ERR_INVALID_ARG;
  if (d->vocab < 1 || d->dim < 1 || d->tokens < 0 || !std::isfinite(d->scale)) return ASI_ERR_INVALID_ARG;
  if (d->padding_idx < -1 || d->padding_idx >= d->vocab) return ASI_ERR_INVALID_ARG;
  if (d->vocab > 1 << 30 || d->dim > 1 << 22 || d->tokens > 1 << 24) return ASI_ERR_UNSUPPORTED;
  return ASI_OK;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t size_of(int32_t dtype) { return dtype == ASI_BF16 ? 2 : 4; }
bool apart(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x + na <= y || y + nb <= x;
}

template <typename TT, typename TO>
cudaError_t launch_lookup(LookupArgs a, int64_t tokens, int vec, cudaStream_t st) {
  a.per_row = (int)(a.D / vec);
  a.items = tokens * a.per_row;
  const dim3 grid((unsigned)std::min<int64_t>((a.items + kEmbThreads - 1) / kEmbThreads, 148 * 64)), block(kEmbThreads);
  switch (vec) {
    case 8: return launch_pdl(k_embed<TT, TO, 8>, grid, block, 0, st, a);
    case 4: return launch_pdl(k_embed<TT, TO, 4>, grid, block, 0, st, a);
    case 2: return launch_pdl(k_embed<TT, TO, 2>, grid, block, 0, st, a);
    default: return launch_pdl(k_embed<TT, TO, 1>, grid, block, 0, st, a);
  }
}

template <typename T, int VEC>
cudaError_t launch_sums(const SumArgs& a, cudaStream_t st) {
  const unsigned slabs = (unsigned)((a.D + (int64_t)kEmbThreads * VEC - 1) / ((int64_t)kEmbThreads * VEC));
  const unsigned zero = a.accumulate ? 0 : (unsigned)((a.V + kZeroRows - 1) / kZeroRows);
  if (a.chunks + zero == 0) return cudaSuccess;
  cudaError_t e = launch_pdl(k_embed_sum<T, VEC>, dim3(a.chunks + zero, slabs), dim3(kEmbThreads), 0, st, a);
  if (e != cudaSuccess || a.chunks < 2) return e;
  return launch_pdl(k_embed_join<VEC>, dim3(a.chunks, slabs), dim3(kEmbThreads), 0, st, a);
}

}  // namespace

}  // namespace asi

using namespace asi;

extern "C" {

asi_status_t asi_embedding_forward(const asi_embedding_desc_t* desc, const void* table, const int64_t* ids, void* out, void* stream) {
  const asi_status_t s = check_desc(desc);
  if (s != ASI_OK) return s;
  if (desc->table_dtype != ASI_F32 && desc->table_dtype != ASI_BF16) return ASI_ERR_INVALID_ARG;
  if (desc->tokens == 0) return ASI_OK;
  const size_t et = size_of(desc->table_dtype), eo = size_of(desc->in_dtype);
  if (!table || !ids || !out || !aligned(table, et) || !aligned(out, eo)) return ASI_ERR_INVALID_ARG;
  if (!apart(table, et * desc->vocab * desc->dim, out, eo * desc->tokens * desc->dim)) return ASI_ERR_INVALID_ARG;
  LookupArgs a = {};
  a.table = table;
  a.ids = ids;
  a.out = out;
  a.V = desc->vocab;
  a.D = desc->dim;
  a.scale = desc->scale;
  int vec = 8;            // values a thread moves: the most that the row length and both addresses allow (16 bytes at a time)
  while (vec > 1 && (desc->dim % vec || !aligned(table, std::min<size_t>(16, vec * et)) || !aligned(out, std::min<size_t>(16, vec * eo)))) vec /= 2;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (desc->table_dtype == ASI_BF16)
    e = desc->in_dtype == ASI_BF16 ? launch_lookup<__nv_bfloat16, __nv_bfloat16>(a, desc->tokens, vec, st)
                                   : launch_lookup<__nv_bfloat16, float>(a, desc->tokens, vec, st);
  else
    e = desc->in_dtype == ASI_BF16 ? launch_lookup<float, __nv_bfloat16>(a, desc->tokens, vec, st)
                                   : launch_lookup<float, float>(a, desc->tokens, vec, st);
  return cuda_status(e, "embedding");
}

size_t asi_embedding_wgrad_ws_bytes(const asi_embedding_desc_t* desc) { return check_desc(desc) == ASI_OK ? layout_of(desc).bytes : 0; }

asi_status_t asi_embedding_wgrad(const asi_embedding_desc_t* desc, const int64_t* ids, const void* dOut, float* dW, int32_t accumulate,
                                 void* ws, size_t ws_bytes, void* stream) {
  const asi_status_t s = check_desc(desc);
  if (s != ASI_OK) return s;
  const size_t eo = size_of(desc->in_dtype), dw_bytes = (size_t)desc->vocab * desc->dim * 4;
  if (!dW || !aligned(dW, 4) || !ws || (desc->tokens && (!ids || !dOut || !aligned(dOut, eo)))) return ASI_ERR_INVALID_ARG;
  const Layout l = layout_of(desc);
  if (ws_bytes < l.bytes || !aligned(ws, 256)) return ASI_ERR_WORKSPACE;
  if (!apart(dW, dw_bytes, ws, l.bytes)) return ASI_ERR_INVALID_ARG;
  if (desc->tokens && (!apart(dW, dw_bytes, dOut, eo * desc->tokens * desc->dim) || !apart(dW, dw_bytes, ids, 8 * desc->tokens) ||
                       !apart(ws, l.bytes, dOut, eo * desc->tokens * desc->dim) || !apart(ws, l.bytes, ids, 8 * desc->tokens)))
    return ASI_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* w = static_cast<char*>(ws);
  int cur = 0;
  for (int pass = 0; pass < l.passes && l.T > 0; ++pass, cur ^= 1) {
    SortArgs a = {};
    a.ids = pass ? nullptr : ids;
    a.key_in = reinterpret_cast<const uint32_t*>(w + l.key[cur ^ 1]);
    a.pos_in = reinterpret_cast<const uint32_t*>(w + l.pos[cur ^ 1]);
    a.key_out = reinterpret_cast<uint32_t*>(w + l.key[cur]);
    a.pos_out = reinterpret_cast<uint32_t*>(w + l.pos[cur]);
    a.hist = reinterpret_cast<uint32_t*>(w + l.hist);
    a.V = desc->vocab;
    a.padding = desc->padding_idx;
    a.T = l.T;
    a.tiles = l.tiles;
    a.shift = pass * l.bits;
    a.bits = l.bits;
    cudaError_t e = launch_pdl(k_sort_hist, dim3(l.tiles), dim3(kEmbThreads), 0, st, a);
    if (e == cudaSuccess) e = launch_pdl(k_sort_scatter, dim3(l.tiles), dim3(kEmbThreads), 0, st, a);
    if (e != cudaSuccess) return cuda_status(e, "sort of tokens");
  }
  cur ^= 1;               // what the last pass wrote
  SumArgs a = {};
  a.dout = dOut;
  a.key = reinterpret_cast<const uint32_t*>(w + l.key[cur]);
  a.pos = reinterpret_cast<const uint32_t*>(w + l.pos[cur]);
  a.dW = dW;
  a.head = reinterpret_cast<float*>(w + l.head);
  a.tail = reinterpret_cast<float*>(w + l.tail);
  a.D = desc->dim;
  a.V = (uint32_t)desc->vocab;
  a.T = l.T;
  a.C = l.C;
  a.chunks = l.chunks;
  a.accumulate = accumulate != 0;
  a.scale = desc->scale;
  const bool wide = aligned(dW, 16) && desc->dim % 4 == 0;
  cudaError_t e;
  if (desc->in_dtype == ASI_BF16)
    e = wide && desc->dim % 8 == 0 && aligned(dOut, 16) ? launch_sums<__nv_bfloat16, 8>(a, st) : launch_sums<__nv_bfloat16, 1>(a, st);
  else
    e = wide && aligned(dOut, 16) ? launch_sums<float, 4>(a, st) : launch_sums<float, 1>(a, st);
  return cuda_status(e, "embedding weight gradient");
}

}  // extern "C"
