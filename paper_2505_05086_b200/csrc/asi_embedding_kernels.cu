// Embedding lookup with scaling, and its weight gradient from sorted tokens.
//
//   out[t] = scale table[ids[t]];     dW[v] = scale sum_{t : ids[t] = v} dOut[t]
//
// The gradient adds whole rows of dOut that share an id.  Atomics would add them in any order; here the tokens are sorted
// by id first (a stable radix sort of (id, t), so that equal ids keep the order of t), and runs of equal ids are summed
// front to back: the same bits from call to call.  The sorted tokens are cut into chunks of equal length, whatever the ids,
// so that one frequent id does not keep a single CTA busy: a run inside a chunk goes to dW at once, the pieces of a run
// that crosses chunks are added in order by the CTA that leaves the last of them.
//
// What bounds it: dOut read once and dW written once (overwriting: all of it, rows without tokens as zeros, by a kernel that
// runs beside sort and sums).
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "asi_internal.h"

namespace asi {

namespace cg = cooperative_groups;

namespace {

constexpr int kEmbThreads = 256;

// N consecutive values as one word of N sizeof(T) bytes (at most 16), unpacked to and packed from floats
template <int kBytes>
struct WordOf;
template <>
struct WordOf<16> { using type = uint4; };
template <>
struct WordOf<8> { using type = uint2; };
template <>
struct WordOf<4> { using type = uint32_t; };
template <>
struct WordOf<2> { using type = uint16_t; };

template <typename T, int N>
struct Word {
  typename WordOf<sizeof(T) * N>::type w;
  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const decltype(w)*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<decltype(w)*>(p) = w; }
  __device__ __forceinline__ uint32_t part(int i) const {
    if constexpr (sizeof(w) == 16) return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    else if constexpr (sizeof(w) == 8) return i == 0 ? w.x : w.y;
    else return w;
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(part(i));
    else return __uint_as_float(i & 1 ? part(i >> 1) & 0xffff0000u : part(i >> 1) << 16);
  }
  __device__ __forceinline__ void set(const float* f) {
    uint32_t u[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4) u[i] = __float_as_uint(f[i]);
      else u[i >> 1] |= (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(f[i])) << (16 * (i & 1));
    }
    if constexpr (sizeof(w) == 16) w = make_uint4(u[0], u[1], u[2], u[3]);
    else if constexpr (sizeof(w) == 8) w = make_uint2(u[0], u[1]);
    else w = u[0];
  }
};

// N consecutive values as floats, in words of up to 16 bytes
template <typename T, int N>
__device__ __forceinline__ void load_values(const T* p, float* f) {
  constexpr int kEach = sizeof(T) * N > 16 ? 16 / (int)sizeof(T) : N;
#pragma unroll
  for (int i = 0; i < N; i += kEach) {
    Word<T, kEach> a;
    a.load(p + i);
#pragma unroll
    for (int e = 0; e < kEach; ++e) f[i + e] = a.value(e);
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_values(T* p, const float* f) {
  constexpr int kEach = sizeof(T) * N > 16 ? 16 / (int)sizeof(T) : N;
#pragma unroll
  for (int i = 0; i < N; i += kEach) {
    Word<T, kEach> a;
    a.set(f + i);
    a.store(p + i);
  }
}

// the same from another CTA's results: past L1, which knows nothing of them
template <int N>
__device__ __forceinline__ void load_shared_values(const float* p, float* f) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(p + i));
      f[i] = v.x, f[i + 1] = v.y, f[i + 2] = v.z, f[i + 3] = v.w;
    }
  } else if constexpr (N == 2) {
    const float2 v = __ldcg(reinterpret_cast<const float2*>(p));
    f[0] = v.x, f[1] = v.y;
  } else {
    f[0] = __ldcg(p);
  }
}
// ---- lookup: blocks of tx x ty threads, ty rows side by side; kRows rows of a thread on their way at once, by loads that no
// condition holds up (beyond the row's end they read its last word again).  Where rows lie off 16 bytes words are narrow, and a
// thread takes several, a block apart.  (16384 x 2048 bf16: 25 us, 5.3 TB/s.  8192 x 2048, 1878 and 1877 bf16: 11.5, 13.4 and
// 17.4 us; with a word each and conditions 13.2, 16.1 and 23.5.)
constexpr int words_of(int vec) { return vec >= 4 ? 1 : 4 / vec; }
struct LookupArgs {
  const void* table;
  const int64_t* ids;
  void* out;
  int64_t V, D, T;
  int per_row;              // D / VEC
  float scale;
};
constexpr int kRows = 4;

template <typename TT, typename TO, int VEC, int W>
__global__ void __launch_bounds__(kEmbThreads) k_embed(const __grid_constant__ LookupArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  const int64_t t0 = (int64_t)blockIdx.x * blockDim.y * kRows + threadIdx.y;
  const TT* row[kRows];
  float scale[kRows];                      // NaN for an id outside the vocabulary, whose row is read as row 0
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int64_t t = t0 + r * blockDim.y, id = t < p.T ? p.ids[t] : 0;
    const bool there = id >= 0 && id < p.V;
    row[r] = static_cast<const TT*>(p.table) + (there ? id * p.D : 0);
    scale[r] = there ? p.scale : NAN;
  }
  constexpr int kTake = sizeof(TT) * VEC > 16 ? 16 / (int)sizeof(TT) : VEC;   // (a word has 16 bytes at most)
  for (int c0 = threadIdx.x; c0 < p.per_row; c0 += W * blockDim.x) {
    Word<TT, kTake> f[kRows][W][VEC / kTake];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int i = 0; i < VEC / kTake; ++i) f[r][w][i].load(row[r] + (int64_t)min(c0 + w * (int)blockDim.x, p.per_row - 1) * VEC + i * kTake);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      const int64_t t = t0 + r * blockDim.y;
      if (t >= p.T) break;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const int c = c0 + w * blockDim.x;
        if (c >= p.per_row) break;
        float o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = f[r][w][e / kTake].value(e % kTake) * scale[r];
        store_values<TO, VEC>(static_cast<TO*>(p.out) + t * p.D + (int64_t)c * VEC, o);
      }
    }
  }
}

// ---- stable radix sort of (id, t), digits of eight bits
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kBins = 256, kDigit = 8;
constexpr int kItems = 8;                   // a thread's tokens
constexpr int kTile = kSortThreads * kItems;
constexpr int kSortCluster = 8;             // CTAs that sort in one launch
constexpr int kFewTokens = 1024;            // sorted by one
constexpr int kOneTokens = kSortCluster * kTile;

struct SortArgs {
  const int64_t* ids;       // null behind the first pass
  const uint32_t *key_in, *pos_in;
  uint32_t *key_out, *pos_out;
  uint32_t* hist;           // [tiles][bins]
  int* count;               // the sums' counters, cleared here
  float* dW;                // k_clear_rows
  int64_t V, D, padding;
  int T, tiles, shift, passes, counters;
  int seg;                  // k_sort_one: tokens of a CTA (its logarithm)
  int rows;                 // k_clear_rows: rows of a CTA
};

// The token's key: its id, or V (sorted behind all ids) where it contributes nothing.
__device__ __forceinline__ uint32_t id_key(const SortArgs& p, int64_t id) {
  return id >= 0 && id < p.V && id != p.padding ? (uint32_t)id : (uint32_t)p.V;
}

// exclusive sum over the CTA's 1024 threads
__device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t* warp_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(~0u, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sum[warp] = x;
  __syncthreads();
  const uint32_t before = __reduce_add_sync(~0u, lane < warp ? warp_sum[lane] : 0u);
  __syncthreads();
  return before + x - v;
}

// Ranks of a tile's tokens among those of the same digit, in order: a thread's item i is token warp 32 items + 32 i + lane, the
// first `here` of its items are there.  Leaves in wh[w][b] how many tokens of digit b earlier warps have, and returns how
// many the tile has of digit threadIdx.x.
__device__ __forceinline__ uint32_t digit_ranks(const uint32_t (&key)[kItems], int here, int items, int shift, uint16_t (*wh)[kBins],
                                                uint16_t (&rank)[kItems]) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t* clear = reinterpret_cast<uint32_t*>(wh[warp]);
#pragma unroll
  for (int b = 0; b < kBins / 2; b += 32) clear[b + lane] = 0;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    if (i >= items) break;
    const bool on = i < here;
    const uint32_t active = __ballot_sync(~0u, on);
    if (on) {
      const uint32_t d = (key[i] >> shift) & (kBins - 1);
      uint32_t peers = active;               // the lanes with this digit (a ballot a bit: the match instruction is slower)
#pragma unroll
      for (int bit = 1; bit < kBins; bit <<= 1) {
        const uint32_t have = __ballot_sync(active, d & bit);
        peers &= d & bit ? have : ~have;
      }
      const uint16_t before = wh[warp][d];
      __syncwarp(active);
      if (lane == __ffs(peers) - 1) wh[warp][d] = before + __popc(peers);
      rank[i] = before + __popc(peers & ((1u << lane) - 1));
    }
    __syncwarp();
  }
  __syncthreads();
  uint32_t total = 0;
  if (tid < kBins) {
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) {
      const uint16_t c = wh[w][tid];
      wh[w][tid] = (uint16_t)total;
      total += c;
    }
  }
  return total;
}

__global__ void __launch_bounds__(kSortThreads) k_sort_hist(const __grid_constant__ SortArgs p) {
  __shared__ uint32_t h[kBins];
  if (threadIdx.x < kBins) h[threadIdx.x] = 0;
  pdl_wait();
  pdl_launch_dependents();
  if (p.ids)
    for (int i = blockIdx.x * kSortThreads + threadIdx.x; i < p.counters; i += gridDim.x * kSortThreads) p.count[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int at = blockIdx.x * kTile + i * kSortThreads + threadIdx.x;
    if (at < p.T) atomicAdd(&h[((p.ids ? id_key(p, p.ids[at]) : p.key_in[at]) >> p.shift) & (kBins - 1)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kBins) p.hist[(int64_t)blockIdx.x * kBins + threadIdx.x] = h[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(const __grid_constant__ SortArgs p) {
  __shared__ __align__(4) uint16_t wh[kSortWarps][kBins];
  __shared__ uint32_t start[kBins], warp_sum[kSortWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  pdl_launch_dependents();
  // where each digit's tokens of this tile start
  uint32_t earlier = 0, total = 0;
  if (tid < kBins) {
#pragma unroll 8
    for (int t = 0; t < p.tiles; ++t) {
      const uint32_t c = p.hist[(int64_t)t * kBins + tid];
      if (t < (int)blockIdx.x) earlier += c;
      total += c;
    }
  }
  const uint32_t before = block_exclusive(total, warp_sum);
  if (tid < kBins) start[tid] = before + earlier;
  uint32_t key[kItems], pos[kItems];
  uint16_t rank[kItems];
  const int base = blockIdx.x * kTile + warp * 32 * kItems + lane;
  int here = 0;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int at = base + i * 32;
    if (at < p.T) {
      key[i] = p.ids ? id_key(p, p.ids[at]) : p.key_in[at];
      pos[i] = p.ids ? at : p.pos_in[at];
      here = i + 1;
    }
  }
  digit_ranks(key, here, kItems, p.shift, wh, rank);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kItems; ++i)
    if (i < here) {
      const uint32_t d = (key[i] >> p.shift) & (kBins - 1);
      const uint32_t to = start[d] + wh[warp][d] + rank[i];
      p.key_out[to] = key[i];
      p.pos_out[to] = pos[i];
    }
}

// Up to 65536 tokens: a cluster of CL CTAs sorts them in one launch, each a segment of 2^seg of them in its shared memory;
// counts and tokens travel through distributed shared memory.  (32000 ids: 10000 tokens take one CTA 29 us and eight 10.  Below
// kFewTokens one CTA does it without the cluster's barriers; a whole accumulating call over 50257 x 768 with 8 tokens takes 7.5
// us where eight CTAs take 9.9, with 1000 11.0 and 12.5, with 2000 as much either way.)
// SMALL, up to three passes: a token travels as one word, sixteen bits of its key and its place.  Of a key with three digits
// the lowest is dropped once the tokens are sorted by it, and read again at the end.  The scattered words are what the cluster
// waits for (calls over 50257 x 770 with 9973 tokens 25.2 us with a store for the key and one for the place, 23.0 with the
// word; 128256 x 770 29.6 and 28.1; 65536 tokens 126 and 115).
template <int CL, bool SMALL>
__global__ void __launch_bounds__(kSortThreads) k_sort_one(const __grid_constant__ SortArgs p) {
  extern __shared__ uint32_t sort_mem[];
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  __shared__ __align__(4) uint16_t wh[kSortWarps][kBins];
  __shared__ uint32_t start[kBins], count[CL][kBins], warp_sum[kSortWarps];
  cg::cluster_group cluster = cg::this_cluster();
  auto together = [&] {
    if constexpr (CL > 1) cluster.sync();
    else __syncthreads();
  };
  auto of = [&](auto* here, int q) { return CL > 1 ? cluster.map_shared_rank(here, q) : here; };
  if constexpr (CL > 1) cluster.barrier_arrive();                    // (shared memory of CTAs that run can be written)
  const int warp = tid >> 5, lane = tid & 31, rank0 = blockIdx.x, seg = 1 << p.seg;
  const int items = (seg + kSortThreads - 1) / kSortThreads;         // of a thread
  uint32_t* skey = sort_mem;
  uint16_t* spos = reinterpret_cast<uint16_t*>(skey + seg);
  for (int i = rank0 * kSortThreads + tid; i < p.counters; i += CL * kSortThreads) p.count[i] = 0;
  uint32_t key[kItems];
  uint16_t pos[kItems], rank[kItems];
  const int base = warp * 32 * items + lane;                         // of the segment
  const int mine = min(max(p.T - rank0 * seg, 0), seg);              // tokens of it
  int here = 0;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int at = base + i * 32;
    if (i < items && at < mine) {
      key[i] = id_key(p, p.ids[rank0 * seg + at]);
      pos[i] = (uint16_t)(rank0 * seg + at);
      here = i + 1;
    }
  }
  const int drop = SMALL && p.passes == 3 ? kDigit : 0;              // of the key, once the tokens are sorted by them
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * kDigit - (pass ? drop : 0);
    const uint32_t own = digit_ranks(key, here, items, shift, wh, rank);
    if constexpr (CL > 1) {
      if (pass == 0) cluster.barrier_wait();
    }
    if (tid < kBins) {                                               // to everybody
#pragma unroll
      for (int q = 0; q < CL; ++q) *of(&count[rank0][tid], q) = own;
    }
    together();                                                      // (every segment is in registers, every count is there)
    uint32_t earlier = 0, total = 0;
    if (tid < kBins) {
#pragma unroll
      for (int q = 0; q < CL; ++q) {
        const uint32_t c = count[q][tid];
        if (q < rank0) earlier += c;
        total += c;
      }
    }
    const uint32_t before = block_exclusive(total, warp_sum);
    if (tid < kBins) start[tid] = before + earlier;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (i < here) {
        const uint32_t d = (key[i] >> shift) & (kBins - 1);
        const uint32_t to = start[d] + wh[warp][d] + rank[i];
        *of(&skey[to & (seg - 1)], to >> p.seg) = SMALL ? key[i] >> (pass ? 0 : drop) << 16 | pos[i] : key[i];
        if (!SMALL) *of(&spos[to & (seg - 1)], to >> p.seg) = pos[i];
      }
    together();
    if (pass + 1 < p.passes) {
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        if (i < here) {
          const uint32_t w = skey[base + i * 32];
          key[i] = SMALL ? w >> 16 : w;
          pos[i] = SMALL ? (uint16_t)w : spos[base + i * 32];
        }
    }
  }
  for (int i = tid; i < mine; i += kSortThreads) {
    const uint32_t w = skey[i], from = SMALL ? w & 0xffffu : spos[i];
    p.key_out[rank0 * seg + i] = !SMALL ? w : drop ? id_key(p, p.ids[from]) : w >> 16;
    p.pos_out[rank0 * seg + i] = from;
  }
}

// The rows of dW that no token has, as zeros: most of the work of a large table (32000 x 2048: 43 us of 51).  Needs nothing of
// the sort and the sums before it on the stream and runs beside them (each CTA marks the ids of its own rows first); it ends
// when they have ended.
constexpr int kClearThreads = 512;
__global__ void __launch_bounds__(kClearThreads) k_clear_rows(const __grid_constant__ SortArgs p) {
  extern __shared__ uint32_t seen[];                                 // a bit for each row
  const int tid = threadIdx.x;
  const int64_t v0 = (int64_t)blockIdx.x * p.rows, rows = min((int64_t)p.rows, p.V - v0);
  for (int i = tid; i < (p.rows + 31) / 32; i += kClearThreads) seen[i] = 0;
  __syncthreads();
#pragma unroll 4
  for (int i = tid; i < p.T; i += kClearThreads) {
    const int64_t r = (int64_t)id_key(p, p.ids[i]) - v0;
    if (r >= 0 && r < rows) atomicOr(&seen[r >> 5], 1u << (r & 31));
  }
  __syncthreads();
  float* row0 = p.dW + v0 * p.D;
  auto each = [&](int units, auto put) {                             // (row, unit) without a division for each
    const int down = kClearThreads / units, along = kClearThreads % units;
    int64_t r = tid / units;
    int u = tid % units;
    while (r < rows) {
      if (!((seen[r >> 5] >> (r & 31)) & 1u)) put(row0 + r * p.D, u);
      r += down;
      u += along;
      if (u >= units) u -= units, ++r;
    }
  };
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  if (p.D % 4 == 0 && (reinterpret_cast<uintptr_t>(p.dW) & 15) == 0) {
    each((int)(p.D / 4), [&](float* row, int u) { reinterpret_cast<float4*>(row)[u] = zero; });
  } else {
    // aligned words of 16 bytes that a row reaches: whole but for its first and last
    each((int)((p.D + 6) / 4), [&](float* row, int u) {
      const int64_t j = 4 * (int64_t)u - ((reinterpret_cast<uintptr_t>(row) >> 2) & 3);
      if (j >= 0 && j + 4 <= p.D) {
        *reinterpret_cast<float4*>(row + j) = zero;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e >= 0 && j + e < p.D) row[j + e] = 0.f;
      }
    });
  }
  pdl_wait();
}

// ---- sums of runs
constexpr int kMaxChunk = 64;
constexpr int kZeroRows = 64;
constexpr int kSumCtas = 3;                 // CTAs of an SM (tied table of 50257 x 770: 25 us, with two 32, with four 25 to 27)
constexpr int kInFlight = 16;              // registers of a thread for the rows in hand, and as many for those on their way

struct SumArgs {
  const void* dout;
  const uint32_t *key, *pos;
  float* dW;
  float *head, *tail;       // [chunks][D]: the chunk's piece of a run that starts earlier / here and goes on
  int* count;               // [chunks][slabs]: pieces of the run that starts in a chunk and goes on
  int64_t D;
  uint32_t V;
  int T, C, chunks, accumulate;
  float scale;
};

// The sum of a run to its row: the one thread that has it writes it, or lets L2 add it (one addition an element: no order
// to depend on, and nobody waits for the old value).
template <int VEC>
__device__ __forceinline__ void put_row(const SumArgs& p, uint32_t v, int64_t col, const float* acc) {
  float* o = p.dW + (int64_t)v * p.D + col;
  float f[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) f[e] = p.scale * acc[e];
  if (!p.accumulate) {
    store_values<float, VEC>(o, f);
  } else if constexpr (VEC >= 4) {
#pragma unroll
    for (int e = 0; e < VEC; e += 4)
      asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(o + e), "f"(f[e]), "f"(f[e + 1]), "f"(f[e + 2]), "f"(f[e + 3])
                   : "memory");
  } else if constexpr (VEC == 2) {
    asm volatile("red.global.add.v2.f32 [%0], {%1, %2};" ::"l"(o), "f"(f[0]), "f"(f[1]) : "memory");
  } else {
    asm volatile("red.global.add.f32 [%0], %1;" ::"l"(o), "f"(f[0]) : "memory");
  }
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

// first of the chunks [lo, lo + n) that does not begin with a key below v, for a whole warp: 32 of them a step.  (Chunk by chunk, or 32
// in a row, each chunk of a long run would walk through all the others: 2^20 tokens of one id, 512 columns, 7.4 ms; so
// 2.3, most of it the pieces added in order.)
__device__ __forceinline__ int heads_below(const SumArgs& p, int lo, int n, uint32_t v) {
  const int lane = threadIdx.x & 31;
  while (n > 0) {
    const int step = (n + 31) / 32, at = lane * step;
    const int below = __popc(__ballot_sync(~0u, at < n && p.key[(lo + at) * p.C] < v));
    if (below == 0) break;
    const int past = (below - 1) * step + 1;
    lo += past;
    n = min(step - 1, n - past);
  }
  return lo;
}

// Bound by latency where tokens are few (keys, rows, fence and count, join one after another: 12 to 15 us for 4096 to 10000
// tokens), by DRAM where they are many (65536 x 2048 bf16: 90 us, 5 TB/s with the rows of dW read and written).
// CTAs [0, chunks): sums, with one warp more that looks for the ends of the runs that cross chunks.  CTAs behind them (many
// tokens, overwriting): rows of dW without tokens.
template <typename T, int VEC>
__global__ void __launch_bounds__(kEmbThreads + 32, kSumCtas) k_embed_sum(const __grid_constant__ SumArgs p) {
  pdl_launch_dependents();                                           // (what comes next waits for this kernel, or needs nothing of it)
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, workers = blockDim.x - 32;
  const int64_t col = tid < workers ? ((int64_t)blockIdx.y * workers + tid) * VEC : p.D;
  if ((int)blockIdx.x >= p.chunks) {
    __shared__ int empty[kZeroRows];
    const int64_t v0 = (int64_t)(blockIdx.x - p.chunks) * kZeroRows;
    for (int r = tid; r < kZeroRows; r += blockDim.x) {
      const uint32_t v = (uint32_t)(v0 + r);
      const int at = lower_bound(p.key, p.T, v);
      empty[r] = v < p.V && (at == p.T || p.key[at] != v);
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
  __shared__ uint32_t sk[kMaxChunk + 2], sp[kMaxChunk], end_bits[2];
  __shared__ int from[2], to[2], done[2];                            // chunks of the run that comes in, and that goes out
  const int c = blockIdx.x, c0 = c * p.C, m = min(p.C, p.T - c0);
  // sk[0] is the key before the chunk, sk[m + 1] the one behind it; V where there is none
  for (int i = tid; i < m + 2; i += blockDim.x) {
    const int at = c0 + i - 1;
    sk[i] = at < 0 || at >= p.T ? p.V : p.key[at];
    if (i >= 1 && i <= m) sp[i - 1] = p.pos[at];
  }
  // a bit for each token that ends a run, or the chunk
  if (tid < 64) {
    const int at = c0 + tid;
    const bool end = tid < m && (tid + 1 == m || p.key[at + 1] != p.key[at]);
    const uint32_t bits = __ballot_sync(~0u, end);
    if (lane == 0) end_bits[tid >> 5] = bits;
  }
  const int live = __syncthreads_count(tid < m && p.key[c0 + tid] != p.V);   // tokens behind them contribute nothing
  if (live == 0) return;
  const bool comes = sk[0] == sk[1], through = comes && sk[m + 1] == sk[m] && sk[1] == sk[m];
  const bool goes = !through && sk[m] != p.V && sk[m + 1] == sk[m];
  if (tid >= workers) {
    // a look at the 32 chunks on either side, then a search
    int first = c;
    if (comes) {                                                     // chunks before this one that begin with its key, and one more
      const int q = c - 1 - lane;
      const uint32_t other = __ballot_sync(~0u, q < 0 || p.key[q * p.C] != sk[1]);
      first = other ? c + 1 - __ffs(other) : heads_below(p, 0, c - 32, sk[1]);
      if (first > 0 && p.key[first * p.C - 1] == sk[1]) --first;
    }
    int last = c;
    if (through || goes) {
      const int q = c + 1 + lane;
      const uint32_t other = __ballot_sync(~0u, q >= p.chunks || p.key[q * p.C] != sk[m]);
      last = other ? c - 1 + __ffs(other) : heads_below(p, c + 33, p.chunks - (c + 33), sk[m] + 1) - 1;
    }
    if (lane == 0) from[0] = first, to[0] = through ? last : c, from[1] = c, to[1] = last;
  } else if (col < p.D) {
    // U rows in hand and the next U on their way, without a condition for each: behind the last row it is read and added again,
    // to a sum that nobody takes (14376 x 1877 bf16: 70 us with conditions, 58; 9973 x 770 fp32: 27 and 25)
    constexpr int kWordRegs = VEC * (int)sizeof(T) / 4, U = kWordRegs > kInFlight / 8 ? kInFlight / kWordRegs : 8;
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
    const uint64_t ends = ((uint64_t)end_bits[1] << 32 | end_bits[0]) & (~0ull >> (64 - live));
    bool first_run = true;
    const T* src = static_cast<const T*>(p.dout) + col;
    Word<T, VEC> f[2][U];
    auto bring = [&](int i0, Word<T, VEC>* w) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        w[u].load(src + (int64_t)sp[min(i0 + u, live - 1)] * p.D);
    };
    bring(0, f[0]);
#pragma unroll 1
    for (int j0 = 0; j0 < live; j0 += 2 * U) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i0 = j0 + h * U;
        if (i0 >= live) break;
        if (i0 + U < live) bring(i0 + U, f[h ^ 1]);
        const uint32_t here = (uint32_t)(ends >> i0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + u;
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] += f[h][u].value(e);
          if (!(here & (1u << u))) continue;
          if (first_run && comes) store_values<float, VEC>(p.head + (int64_t)c * p.D + col, acc);
          else if (goes && i + 1 == m) store_values<float, VEC>(p.tail + (int64_t)c * p.D + col, acc);
          else put_row<VEC>(p, sk[i + 1], col, acc);
          first_run = false;
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
        }
      }
    }
  }
  if (!comes && !goes) return;
  // Runs that cross chunks: the CTA that leaves the last piece of a run joins them, in order.
  __syncthreads();
  if (tid < 2) {
    __threadfence();                                                 // the CTA's pieces before the count, the others' behind it
    done[tid] = (tid ? goes : comes) && atomicAdd(&p.count[(int64_t)from[tid] * gridDim.y + blockIdx.y], 1) == to[tid] - from[tid];
    __threadfence();
  }
  __syncthreads();
  if (col >= p.D) return;
#pragma unroll 1
  for (int side = 0; side < 2; ++side) {
    if (!done[side]) continue;
    float acc[VEC];
    load_shared_values<VEC>(p.tail + (int64_t)from[side] * p.D + col, acc);
    constexpr int P = VEC == 1 ? 16 : 32 / VEC;                      // pieces on their way at once
    const int end = to[side];
    for (int q = from[side] + 1; q <= end; q += P) {
      float f[P][VEC];
#pragma unroll
      for (int u = 0; u < P; ++u)
        if (q + u <= end) load_shared_values<VEC>(p.head + (int64_t)(q + u) * p.D + col, f[u]);
#pragma unroll
      for (int u = 0; u < P; ++u)
        if (q + u <= end) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] += f[u][e];
        }
    }
    put_row<VEC>(p, side ? sk[m] : sk[1], col, acc);
  }
}

// ---- host side
struct Layout {
  int T, tiles, passes;
  bool one;                 // a single launch sorts
  size_t key[2], pos[2], hist, count, head, tail, bytes;
};

constexpr int kMinChunk = 8, kMostChunks = 148 * 4;
// Tokens of a chunk: as many chunks as run at once, of 8 to 64 tokens
int chunk_of(int64_t T, int slabs, int ctas) {
  return (int)std::min<int64_t>(std::max<int64_t>((T * slabs + 148 * ctas - 1) / (148 * ctas), kMinChunk), kMaxChunk);
}

Layout layout_of(const asi_embedding_desc_t* d) {
  Layout l = {};
  l.T = (int)d->tokens;
  // the most chunks of this and any shorter batch: a workspace serves fewer tokens too
  const size_t most = std::max(std::min((l.T + kMinChunk - 1) / kMinChunk, kMostChunks), (l.T + kMaxChunk - 1) / kMaxChunk);
  l.one = l.T <= kOneTokens;
  l.tiles = (l.T + kTile - 1) / kTile;
  l.passes = 1;
  while ((d->vocab >> (l.passes * kDigit)) != 0) ++l.passes;          // keys up to vocab itself
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
  l.hist = take((size_t)l.tiles * kBins * 4);
  l.count = take(most * ((d->dim + kEmbThreads - 1) / kEmbThreads) * 4);
  l.head = take(most * d->dim * 4);
  l.tail = take(most * d->dim * 4);
  l.bytes = std::max<size_t>(at, 256);
  return l;
}

asi_status_t check_desc(const asi_embedding_desc_t* d) {
  if (!d || (d->in_dtype != ASI_F32 && d->in_dtype != ASI_BF16)) return ASI_ERR_INVALID_ARG;
  if (d->vocab < 1 || d->dim < 1 || d->tokens < 0 || !std::isfinite(d->scale)) return ASI_ERR_INVALID_ARG;
  if (d->padding_idx < -1 || d->padding_idx >= d->vocab) return ASI_ERR_INVALID_ARG;
  if (d->vocab > 1 << 30 || d->dim > 1 << 22 || d->tokens > 1 << 24 || d->dim * d->tokens > (int64_t)1 << 38) return ASI_ERR_UNSUPPORTED;
  return ASI_OK;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
size_t size_of(int32_t dtype) { return dtype == ASI_BF16 ? 2 : 4; }
bool apart(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x + na <= y || y + nb <= x;
}

template <typename TT, typename TO>
cudaError_t launch_lookup(LookupArgs a, int vec, cudaStream_t st) {
  a.per_row = (int)(a.D / vec);
  unsigned tx = 32;
  while (tx < (unsigned)kEmbThreads && (int)tx * words_of(vec) < a.per_row) tx *= 2;
  const unsigned ty = kEmbThreads / tx;
  const dim3 grid((unsigned)((a.T + (int64_t)ty * kRows - 1) / ((int64_t)ty * kRows))), block(tx, ty);
  switch (vec) {
    case 8: return launch_pdl(k_embed<TT, TO, 8, words_of(8)>, grid, block, 0, st, a);
    case 4: return launch_pdl(k_embed<TT, TO, 4, words_of(4)>, grid, block, 0, st, a);
    case 2: return launch_pdl(k_embed<TT, TO, 2, words_of(2)>, grid, block, 0, st, a);
    default: return launch_pdl(k_embed<TT, TO, 1, words_of(1)>, grid, block, 0, st, a);
  }
}

// Sorted keys and positions into the layout's buffers *out; clears the sums' counters.
cudaError_t sort_tokens(SortArgs a, const Layout& l, int counters, char* w, int* out, cudaStream_t st) {
  a.hist = reinterpret_cast<uint32_t*>(w + l.hist);
  a.count = reinterpret_cast<int*>(w + l.count);
  a.counters = counters;
  a.tiles = l.tiles;
  a.passes = l.passes;
  if (l.one) {
    a.key_out = reinterpret_cast<uint32_t*>(w + l.key[0]);
    a.pos_out = reinterpret_cast<uint32_t*>(w + l.pos[0]);
    const bool few = l.T <= kFewTokens;
    while (l.T > (few ? 1 : kSortCluster) << a.seg) ++a.seg;
    const size_t smem = (size_t)6 << a.seg;
    *out = 0;
    const bool small = l.passes <= 3;
    if (few) return launch_pdl(k_sort_one<1, false>, dim3(1), dim3(kSortThreads), smem, st, a);
    const auto kernel = small ? k_sort_one<kSortCluster, true> : k_sort_one<kSortCluster, false>;
    cudaError_t e = smem > 16 << 10 ? opt_in_smem(reinterpret_cast<const void*>(kernel), smem) : cudaSuccess;
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kSortCluster);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = kSortCluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
  }
  cudaError_t e = cudaSuccess;
  for (int pass = 0; pass < l.passes && e == cudaSuccess; ++pass) {
    const int to = pass & 1;
    if (pass) a.ids = nullptr;
    a.key_in = reinterpret_cast<const uint32_t*>(w + l.key[to ^ 1]);
    a.pos_in = reinterpret_cast<const uint32_t*>(w + l.pos[to ^ 1]);
    a.key_out = reinterpret_cast<uint32_t*>(w + l.key[to]);
    a.pos_out = reinterpret_cast<uint32_t*>(w + l.pos[to]);
    a.shift = pass * kDigit;
    e = launch_pdl(k_sort_hist, dim3(l.tiles), dim3(kSortThreads), 0, st, a);
    if (e == cudaSuccess) e = launch_pdl(k_sort_scatter, dim3(l.tiles), dim3(kSortThreads), 0, st, a);
    *out = to;
  }
  return e;
}

cudaError_t clear_rows(SortArgs a, cudaStream_t st) {
  constexpr int kClear = 148 * 4;
  a.rows = (int)std::min<int64_t>((a.V + kClear - 1) / kClear, 65536);
  return launch_pdl(k_clear_rows, dim3((unsigned)((a.V + a.rows - 1) / a.rows)), dim3(kClearThreads), (size_t)(a.rows + 31) / 32 * 4, st, a);
}

// CTAs that share a row of dW, and their threads
unsigned slabs_of(int64_t D, int vec) { return (unsigned)((D / vec + kEmbThreads - 1) / kEmbThreads); }

template <typename T, int VEC>
cudaError_t launch_sums(const SumArgs& a, bool clear, cudaStream_t st) {
  const unsigned slabs = slabs_of(a.D, VEC), zero = clear ? (unsigned)((a.V + kZeroRows - 1) / kZeroRows) : 0;
  const unsigned threads = (unsigned)(((a.D / VEC + slabs - 1) / slabs + 31) / 32 * 32);
  return a.chunks + zero ? launch_pdl(k_embed_sum<T, VEC>, dim3(a.chunks + zero, slabs), dim3(threads + 32), 0, st, a) : cudaSuccess;
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
  if (!table || !ids || !out || !aligned(table, et) || !aligned(out, eo) || !aligned(ids, 8)) return ASI_ERR_INVALID_ARG;
  const size_t out_bytes = eo * desc->tokens * desc->dim;
  if (!apart(table, et * desc->vocab * desc->dim, out, out_bytes) || !apart(ids, 8 * desc->tokens, out, out_bytes)) return ASI_ERR_INVALID_ARG;
  LookupArgs a = {};
  a.table = table;
  a.ids = ids;
  a.out = out;
  a.V = desc->vocab;
  a.D = desc->dim;
  a.T = desc->tokens;
  a.scale = desc->scale;
  int vec = 8;            // values a thread moves: the most that the row length and both addresses allow (16 bytes at a time)
  while (vec > 1 && (desc->dim % vec || !aligned(table, std::min<size_t>(16, vec * et)) || !aligned(out, std::min<size_t>(16, vec * eo)))) vec /= 2;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (desc->table_dtype == ASI_BF16)
    e = desc->in_dtype == ASI_BF16 ? launch_lookup<__nv_bfloat16, __nv_bfloat16>(a, vec, st) : launch_lookup<__nv_bfloat16, float>(a, vec, st);
  else
    e = desc->in_dtype == ASI_BF16 ? launch_lookup<float, __nv_bfloat16>(a, vec, st) : launch_lookup<float, float>(a, vec, st);
  return cuda_status(e, "embedding");
}

size_t asi_embedding_wgrad_ws_bytes(const asi_embedding_desc_t* desc) { return check_desc(desc) == ASI_OK ? layout_of(desc).bytes : 0; }

asi_status_t asi_embedding_wgrad(const asi_embedding_desc_t* desc, const int64_t* ids, const void* dOut, float* dW, int32_t accumulate,
                                 void* ws, size_t ws_bytes, void* stream) {
  const asi_status_t s = check_desc(desc);
  if (s != ASI_OK) return s;
  const size_t eo = size_of(desc->in_dtype), dw_bytes = (size_t)desc->vocab * desc->dim * 4;
  if (!dW || !aligned(dW, 4) || !ws || (desc->tokens && (!ids || !dOut || !aligned(dOut, eo) || !aligned(ids, 8)))) return ASI_ERR_INVALID_ARG;
  const Layout l = layout_of(desc);
  if (ws_bytes < l.bytes || !aligned(ws, 256)) return ASI_ERR_WORKSPACE;
  if (!apart(dW, dw_bytes, ws, l.bytes)) return ASI_ERR_INVALID_ARG;
  if (desc->tokens && (!apart(dW, dw_bytes, dOut, eo * desc->tokens * desc->dim) || !apart(dW, dw_bytes, ids, 8 * desc->tokens) ||
                       !apart(ws, l.bytes, dOut, eo * desc->tokens * desc->dim) || !apart(ws, l.bytes, ids, 8 * desc->tokens)))
    return ASI_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* w = static_cast<char*>(ws);
  // columns of a thread: the most that the row length and the addresses allow, 16 bytes of dW at a time
  int vec = 4;
  while (vec > 1 && (desc->dim % vec || !aligned(dOut, vec * eo) || !aligned(dW, vec * 4))) vec /= 2;
  try {
    // (beside the clearing kernel the sums have two CTAs an SM, so that both fit)
    const bool clear = !accumulate, beside = clear && l.one;
    const int slabs = (int)slabs_of(desc->dim, vec), C = chunk_of(l.T, slabs, beside ? 2 : kSumCtas), chunks = (l.T + C - 1) / C;
    SortArgs sort = {};
    sort.ids = ids;
    sort.dW = dW;
    sort.V = desc->vocab;
    sort.D = desc->dim;
    sort.padding = desc->padding_idx;
    sort.T = l.T;
    int at = 0;
    cudaError_t e = cudaSuccess;
    if (l.T || clear) e = sort_tokens(sort, l, chunks * slabs, w, &at, st);
    if (e != cudaSuccess) return cuda_status(e, "sort of tokens");
    SumArgs a = {};
    a.dout = dOut;
    a.key = reinterpret_cast<const uint32_t*>(w + l.key[at]);
    a.pos = reinterpret_cast<const uint32_t*>(w + l.pos[at]);
    a.dW = dW;
    a.head = reinterpret_cast<float*>(w + l.head);
    a.tail = reinterpret_cast<float*>(w + l.tail);
    a.count = reinterpret_cast<int*>(w + l.count);
    a.D = desc->dim;
    a.V = (uint32_t)desc->vocab;
    a.T = l.T;
    a.C = C;
    a.chunks = chunks;
    a.accumulate = accumulate != 0;
    a.scale = desc->scale;
    if (desc->in_dtype == ASI_BF16)
      e = vec == 4 ? launch_sums<__nv_bfloat16, 4>(a, clear && !beside, st) : vec == 2 ? launch_sums<__nv_bfloat16, 2>(a, clear && !beside, st) : launch_sums<__nv_bfloat16, 1>(a, clear && !beside, st);
    else
      e = vec == 4 ? launch_sums<float, 4>(a, clear && !beside, st) : vec == 2 ? launch_sums<float, 2>(a, clear && !beside, st) : launch_sums<float, 1>(a, clear && !beside, st);
    if (e == cudaSuccess && beside) e = clear_rows(sort, st);
    return cuda_status(e, "embedding weight gradient");
  } catch (...) {
    return no_host_memory();
  }
}

}  // extern "C"
