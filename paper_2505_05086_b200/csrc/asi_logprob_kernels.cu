// Log probabilities of given tokens, with entropy and top alternatives, and their gradient: the loss over the vocabulary
// whose gradient is the dY of a model's output layer.
//
// With x_j = scale * logit_j, M the largest logit, a_j = (logit_j - M) scale log2(e) and e_j = 2^a_j:
//   S = sum e_j,  W = sum e_j a_j;   lse = scale M + ln S;   entropy = ln S - ln2 W / S;   logp_j = ln2 a_j - ln S
//   dlogits_j = scale (alpha ([j = y] - p_j) - beta p_j (log p_j + entropy)) = e_j (A + B a_j) + [j = y] scale alpha
// with A = -scale (alpha + beta (entropy - ln S)) / S and B = -scale beta ln2 / S.
//
// What bounds it: the logits, read once (and the gradient, written once).  A row stays in shared memory between the maximum,
// the sums and the gradient, split over a cluster of up to eight CTAs where it is long or where there are few rows; the
// cluster's shares (M, S, W and the leading entries) meet through distributed shared memory, in rank order.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "asi_internal.h"

namespace asi {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kCand = 512;                 // candidates of a CTA's top entries
constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;

struct LogprobArgs {
  const void* x;
  const int64_t* y;
  float *logp, *entropy, *lse, *top_logp;
  int64_t* top_ids;
  const float *dlogp, *dent;
  void* dx;
  int64_t ld, ldg, ignore;
  int V, k, cl;
  float scale;
};

struct LogprobGradArgs {
  const void* x;
  const int64_t* y;
  const float *lse, *ent, *dlogp, *dent;
  void* dx;
  int64_t ld, ldg, ignore, blocks;
  int V, splits;
  float scale;
};

__device__ __forceinline__ float nan_max(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t nan_max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float exp2_approx(float a) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t smem_at(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ float remote_f(const float* p, int rank) {       // the same address in another CTA of the cluster
  uint32_t at;
  float v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_at(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long remote_u64(const unsigned long long* p, int rank) {
  uint32_t at;
  unsigned long long v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_at(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Sixteen bytes of a row: 8 bf16 or 4 fp32 values.
template <typename T>
struct Granule;
template <>
struct Granule<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void floats(const uint4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float largest(const uint4& v) {
    const uint32_t m = nan_max2(nan_max2(v.x, v.y), nan_max2(v.z, v.w));
    return nan_max(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ __nv_bfloat16 one(float f) { return __float2bfloat16_rn(f); }
  static __device__ __forceinline__ float read(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};
template <>
struct Granule<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void floats(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float largest(const uint4& v) {
    return nan_max(nan_max(__uint_as_float(v.x), __uint_as_float(v.y)), nan_max(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float one(float f) { return f; }
  static __device__ __forceinline__ float read(const float* p) { return *p; }
};

// A row as granules that start on 16 bytes: granule g holds the elements [g n - mis, g n - mis + n), those outside
// [0, V) are not the row's (the first and the last granule).
template <typename T>
struct RowView {
  const T* x;
  int mis, V;
  __device__ RowView(const T* at, int v) : x(at), mis((int)((reinterpret_cast<uintptr_t>(at) & 15) / sizeof(T))), V(v) {}
  __device__ __forceinline__ int first(int g) const { return g * Granule<T>::n - mis; }
  __device__ __forceinline__ int granules() const { return (int)(((int64_t)mis + V + Granule<T>::n - 1) / Granule<T>::n); }
  __device__ __forceinline__ bool whole(int g) const {
    const int j = first(g);
    return j >= 0 && (int64_t)j + Granule<T>::n <= V;
  }
  __device__ __forceinline__ uint4 edge(int g) const {            // element by element, -inf outside the row
    float f[Granule<T>::n];
    const int j = first(g);
#pragma unroll
    for (int i = 0; i < Granule<T>::n; ++i)
      f[i] = j + i >= 0 && j + i < V ? Granule<T>::read(x + j + i) : -INFINITY;
    return Granule<T>::pack(f);
  }
  __device__ __forceinline__ uint4 load(int g) const {
    if (whole(g)) return *reinterpret_cast<const uint4*>(x + first(g));
    return edge(g);
  }
};

// writes the row's elements of granule g; `wide`: dx starts on the same offset within 16 bytes as x
template <typename T>
__device__ __forceinline__ void store_granule(T* dx, const RowView<T>& row, int g, const float* f, bool wide) {
  const int j = row.first(g);
  if (wide && row.whole(g)) {
    *reinterpret_cast<uint4*>(dx + j) = Granule<T>::pack(f);
  } else {
#pragma unroll
    for (int i = 0; i < Granule<T>::n; ++i)
      if (j + i >= 0 && j + i < row.V) dx[j + i] = Granule<T>::one(f[i]);
  }
}

// Orders entries by value, then by lower index; never 0.
__device__ __forceinline__ unsigned long long order_key(float v, int j) {
  const uint32_t b = __float_as_uint(v + 0.f);                     // -0 counts as 0
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return ((unsigned long long)o << 32) | (0xffffffffu - (uint32_t)j);
}
__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_index(unsigned long long key) { return (int)(0xffffffffu - (uint32_t)key); }

struct TopShared {
  unsigned long long cand[kCand];
  unsigned long long list[ASI_TOP_MAX];    // this CTA's leading entries, largest first; 0: none
  float group[32];
  float tau;
  int count;
};

// GRAD: the gradient in the same pass.  TOP: leading entries.  RES: the CTA's share of the row stays in shared memory
// (else it is read again for each sweep: rows of more than 1.6 MB).
template <typename T, bool GRAD, bool TOP, bool RES>
__global__ void __launch_bounds__(kThreads) k_logprob(const __grid_constant__ LogprobArgs p) {
  constexpr int n = Granule<T>::n;
  extern __shared__ uint4 buf[];
  __shared__ float red[3][kWarps];
  __shared__ float mine[3];                // M, S, W of this CTA's share
  __shared__ float parts[3][kMaxCluster];
  __shared__ TopShared top;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cl = p.cl, t = blockIdx.x / cl, rank = blockIdx.x - t * cl;
  const RowView<T> row(static_cast<const T*>(p.x) + (int64_t)t * p.ld, p.V);
  const int G = row.granules(), per = (G + cl - 1) / cl;
  const int g0 = min(G, rank * per), cnt = min(G - g0, per);

  pdl_wait();
  pdl_launch_dependents();
  const int64_t y = p.y[t];
  const bool given = y >= 0 && y < p.V, skip = y == p.ignore;
  float xy = 0.f;
  if (given && tid == 0 && rank == 0) xy = Granule<T>::read(row.x + y);

  if (RES) {
    for (int i = tid; i < cnt; i += kThreads) {
      if (row.whole(g0 + i))
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_at(buf + i)), "l"(row.x + row.first(g0 + i)) : "memory");
      else
        buf[i] = row.edge(g0 + i);
    }
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
  }
  // every thread reads back what it brought itself: no barrier
  auto at = [&](int i) -> uint4 { return RES ? buf[i] : row.load(g0 + i); };

  float M = -INFINITY;
  for (int i = tid; i < cnt; i += kThreads) M = nan_max(M, Granule<T>::largest(at(i)));
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    if (TOP && o == 8 && (lane & 7) == 0) top.group[tid >> 3] = M;
    M = nan_max(M, __shfl_xor_sync(~0u, M, o));
  }
  if (lane == 0) red[0][warp] = M;
  if (TOP && tid == 0) top.count = 0;
  __syncthreads();
  M = red[0][0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) M = nan_max(M, red[0][i]);
  // The k-th largest of the maxima of 32 groups of threads: at least k entries reach it, and few more.
  float tau = 0.f;
  if (TOP) {
    if (warp == 0) {
      const float v = top.group[lane];
      int above = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float o = __shfl_sync(~0u, v, i);
        above += o > v || (o == v && i < lane);
      }
      if (above == p.k - 1) top.tau = v;                         // one lane, unless there are NaNs (then no matter)
    }
    __syncthreads();
    tau = top.tau;
  }

  const float c2 = p.scale * kLog2e, Mz = M == -INFINITY ? 0.f : M;
  float S = 0.f, W = 0.f;
  for (int i = tid; i < cnt; i += kThreads) {
    const uint4 v = at(i);
    float f[n];
    Granule<T>::floats(v, f);
    if (TOP && Granule<T>::largest(v) >= tau) {
      const int j = row.first(g0 + i);
#pragma unroll
      for (int e = 0; e < n; ++e)
        if (f[e] >= tau && j + e >= 0 && j + e < p.V) {
          const int slot = atomicAdd(&top.count, 1);
          if (slot < kCand) top.cand[slot] = order_key(f[e], j + e);
        }
    }
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const float a = (f[e] - Mz) * c2, ex = exp2_approx(a);
      S += ex;
      W = fmaf(ex, fmaxf(a, -1e4f), W);                             // 0 * -inf would be NaN
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    S += __shfl_xor_sync(~0u, S, o);
    W += __shfl_xor_sync(~0u, W, o);
  }
  if (lane == 0) red[1][warp] = S, red[2][warp] = W;
  __syncthreads();
  S = red[1][0], W = red[2][0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) S += red[1][i], W += red[2][i];

  if (TOP) {                                // this CTA's leading entries, in order
    const int found = top.count;
    if (tid < ASI_TOP_MAX) top.list[tid] = 0;
    __syncthreads();
    if (found <= kCand) {
      for (int i = tid; i < found; i += kThreads) {
        const unsigned long long key = top.cand[i];
        int above = 0;
        for (int q = 0; q < found; ++q) above += top.cand[q] > key;
        if (above < p.k) top.list[above] = key;
      }
    } else {                                // many equal values: one sweep for each entry
      unsigned long long prev = ~0ull;
      for (int r = 0; r < p.k; ++r) {
        unsigned long long best = 0;
        for (int i = tid; i < cnt; i += kThreads) {
          float f[n];
          Granule<T>::floats(at(i), f);
          const int j = row.first(g0 + i);
#pragma unroll
          for (int e = 0; e < n; ++e)
            if (j + e >= 0 && j + e < p.V) {
              const unsigned long long key = order_key(f[e], j + e);
              if (key < prev && key > best) best = key;
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
          const unsigned long long other = __shfl_xor_sync(~0u, best, o);
          if (other > best) best = other;
        }
        __syncthreads();                    // cand[] is free: the warps' best
        if (lane == 0) top.cand[warp] = best;
        __syncthreads();
        best = top.cand[0];
#pragma unroll
        for (int i = 1; i < kWarps; ++i)
          if (top.cand[i] > best) best = top.cand[i];
        if (tid == 0) top.list[r] = best;
        prev = best;
      }
    }
  }

  if (cl > 1) {
    if (tid == 0) mine[0] = M, mine[1] = S, mine[2] = W;
    cluster_arrive();                       // (every thread's writes above, the lists among them)
    cluster_wait();
    if (tid < 3 * cl) parts[tid % 3][tid / 3] = remote_f(&mine[tid % 3], tid / 3);
    if (TOP && rank == 0)
      for (int i = tid; i < cl * p.k; i += kThreads) top.cand[i] = remote_u64(&top.list[i % p.k], i / p.k);
    __syncthreads();
    cluster_arrive();                       // the others' shared memory is read no more; waited for at the end
    float Mt = parts[0][0];
    for (int q = 1; q < cl; ++q) Mt = nan_max(Mt, parts[0][q]);
    S = W = 0.f;
    for (int q = 0; q < cl; ++q) {
      if (parts[0][q] == -INFINITY) continue;                       // nothing there
      const float a = (parts[0][q] - Mt) * c2, f = exp2_approx(a);
      S = fmaf(f, parts[1][q], S);
      W = fmaf(f, fmaf(fmaxf(a, -1e4f), parts[1][q], parts[2][q]), W);
    }
    M = Mt;
    if (TOP && rank == 0) {
      for (int i = tid; i < cl * p.k; i += kThreads) {
        const unsigned long long key = top.cand[i];
        int above = 0;
        for (int q = 0; q < cl * p.k; ++q) above += top.cand[q] > key;
        if (key && above < p.k) top.list[above] = key;           // (no CTA reads this list any more)
      }
    }
  }
  if (TOP) __syncthreads();

  const bool dead = M == -INFINITY;
  const float lnS = logf(S);
  const float H = dead ? 0.f : lnS - kLn2 * W / S;
  if (rank == 0) {
    if (tid == 0) {
      p.lse[t] = dead ? -INFINITY : fmaf(M, p.scale, lnS);
      if (p.entropy) p.entropy[t] = H;
      p.logp[t] = skip ? 0.f : !given ? NAN : dead ? -INFINITY : (xy - M) * p.scale - lnS;
    }
    if (TOP && tid < p.k) {
      const bool fine = !isnan(lnS);
      const unsigned long long key = fine ? top.list[tid] : 0;
      p.top_ids[(int64_t)t * p.k + tid] = fine ? key_index(key) : tid;
      p.top_logp[(int64_t)t * p.k + tid] = !fine ? NAN : dead ? -INFINITY : (key_value(key) - M) * p.scale - lnS;
    }
  }

  if (GRAD) {
    T* dx = static_cast<T*>(p.dx) + (int64_t)t * p.ldg;
    const bool wide = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(row.x)) & 15) == 0;
    const float alpha = p.dlogp[t], beta = p.dent ? p.dent[t] : 0.f, inv = 1.f / S;
    const bool zero = skip || dead;
    const float A = given ? -p.scale * (alpha + beta * (H - lnS)) * inv : NAN, B = -p.scale * beta * kLn2 * inv;
    for (int i = tid; i < cnt; i += kThreads) {
      float f[n];
      Granule<T>::floats(at(i), f);
      const int j = row.first(g0 + i);
#pragma unroll
      for (int e = 0; e < n; ++e) {
        const float a = (f[e] - M) * c2;
        f[e] = zero ? 0.f : exp2_approx(a) * fmaf(B, fmaxf(a, -1e4f), A);
      }
      if (given && !zero && y >= j && y < j + n) {
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (j + e == y) f[e] += p.scale * alpha;
      }
      store_granule(dx, row, g0 + i, f, wide);
    }
  }
  if (cl > 1) cluster_wait();
}

// The gradient alone, from lse and entropy: a stream of 1024 granules a CTA.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_logprob_grad(const __grid_constant__ LogprobGradArgs p) {
  constexpr int n = Granule<T>::n, kEach = 4;
  pdl_wait();
  pdl_launch_dependents();
  for (int64_t b = blockIdx.x; b < p.blocks; b += gridDim.x) {
    const int64_t t = b / p.splits;
    const int g0 = (int)(b - t * p.splits) * kThreads * kEach + threadIdx.x;
    const RowView<T> row(static_cast<const T*>(p.x) + t * p.ld, p.V);
    const int G = row.granules();
    T* dx = static_cast<T*>(p.dx) + t * p.ldg;
    const bool wide = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(row.x)) & 15) == 0;
    const int64_t y = p.y[t];
    const float lse = p.lse[t], alpha = p.dlogp[t], beta = p.dent ? p.dent[t] : 0.f, H = p.dent ? p.ent[t] : 0.f;
    const bool given = y >= 0 && y < p.V, zero = y == p.ignore || lse == -INFINITY;
    const float A = given ? -p.scale * (alpha + beta * H) : NAN, B = -p.scale * beta;
    uint4 v[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int g = g0 + q * kThreads;
      v[q] = make_uint4(0, 0, 0, 0);
      if (g < G && !zero) v[q] = row.load(g);
    }
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int g = g0 + q * kThreads;
      if (g >= G) break;
      float f[n];
      Granule<T>::floats(v[q], f);
      const int j = row.first(g);
#pragma unroll
      for (int e = 0; e < n; ++e) {
        const float lp = fmaf(f[e], p.scale, -lse);
        f[e] = zero ? 0.f : exp2_approx(lp * kLog2e) * fmaf(B, fmaxf(lp, -1e4f), A);
      }
      if (given && !zero && y >= j && y < j + n) {
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (j + e == y) f[e] += p.scale * alpha;
      }
      store_granule(dx, row, g, f, wide);
    }
  }
}

// CTAs of a row: few enough that a share of 72 KB at most lets three CTAs run on an SM, more where the rows alone do not
// fill the machine and a share keeps two granules a thread.
int cluster_of(int64_t rows, int64_t granules) {
  int cl = 1;
  while (cl < kMaxCluster && granules * 16 > (int64_t)cl * (72 << 10)) cl *= 2;
  while (cl < kMaxCluster && rows * cl < 148 && granules >= 4 * cl * kThreads) cl *= 2;
  return cl;
}

template <typename T, bool GRAD, bool TOP, bool RES>
cudaError_t launch_one(const LogprobArgs& a, int64_t rows, size_t smem, cudaStream_t st) {
  auto kernel = k_logprob<T, GRAD, TOP, RES>;
  if (smem > 32 << 10) {
    const cudaError_t e = opt_in_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * a.cl));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)a.cl;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = a.cl > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T>
cudaError_t launch_logprob(LogprobArgs a, int64_t rows, bool grad, cudaStream_t st) {
  const int64_t granules = ((int64_t)a.V + 2 * Granule<T>::n - 2) / Granule<T>::n;   // of a row at the worst offset
  a.cl = cluster_of(rows, granules);
  const size_t share = (size_t)((granules + a.cl - 1) / a.cl) * 16;
  const bool res = share <= 200 << 10;
  const size_t smem = res ? share : 0;
  if (grad) return res ? launch_one<T, true, false, true>(a, rows, smem, st) : launch_one<T, true, false, false>(a, rows, smem, st);
  if (a.k) return res ? launch_one<T, false, true, true>(a, rows, smem, st) : launch_one<T, false, true, false>(a, rows, smem, st);
  return res ? launch_one<T, false, false, true>(a, rows, smem, st) : launch_one<T, false, false, false>(a, rows, smem, st);
}

asi_status_t check_desc(const asi_logprob_desc_t* d) {
  if (!d || (d->in_dtype != ASI_F32 && d->in_dtype != ASI_BF16)) return ASI_ERR_INVALID_ARG;
  if (d->rows < 0 || d->vocab < 1 || d->ld < d->vocab) return ASI_ERR_INVALID_ARG;
  if (!(d->scale > 0.f) || !std::isfinite(d->scale)) return ASI_ERR_INVALID_ARG;
  if (d->rows > ASI_LOGPROB_MAX_ROWS || d->vocab > ASI_LOGPROB_MAX_VOCAB) return ASI_ERR_UNSUPPORTED;
  if (d->ld > INT64_MAX / 8 / std::max<int64_t>(d->rows, 1)) return ASI_ERR_INVALID_ARG;
  return ASI_OK;
}

size_t logit_bytes(const asi_logprob_desc_t* d) { return d->in_dtype == ASI_BF16 ? 2 : 4; }

bool off_element(const asi_logprob_desc_t* d, const void* p) { return (reinterpret_cast<uintptr_t>(p) & (logit_bytes(d) - 1)) != 0; }

// dlogits is logits itself, row for row, or lies apart from it
asi_status_t check_grad(const asi_logprob_desc_t* d, const void* x, const void* dx) {
  if (!dx || off_element(d, dx) || d->ld_grad < d->vocab) return ASI_ERR_INVALID_ARG;
  if (d->ld_grad > INT64_MAX / 8 / std::max<int64_t>(d->rows, 1)) return ASI_ERR_INVALID_ARG;
  const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(dx);
  if (a == b) return d->ld_grad == d->ld || d->rows == 1 ? ASI_OK : ASI_ERR_INVALID_ARG;
  const uintptr_t na = ((d->rows - 1) * d->ld + d->vocab) * logit_bytes(d), nb = ((d->rows - 1) * d->ld_grad + d->vocab) * logit_bytes(d);
  return a < b + nb && b < a + na ? ASI_ERR_INVALID_ARG : ASI_OK;
}

LogprobArgs base_args(const asi_logprob_desc_t* d, const void* logits, const int64_t* targets) {
  LogprobArgs a = {};
  a.x = logits;
  a.y = targets;
  a.ld = d->ld;
  a.ldg = d->ld_grad;
  a.ignore = d->ignore_index;
  a.V = (int)d->vocab;
  a.scale = d->scale;
  return a;
}

asi_status_t run_logprob(const asi_logprob_desc_t* d, const LogprobArgs& a, bool grad, void* stream) {
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cuda_status(d->in_dtype == ASI_BF16 ? launch_logprob<__nv_bfloat16>(a, d->rows, grad, st) : launch_logprob<float>(a, d->rows, grad, st),
                     "log probabilities");
}

}  // namespace

}  // namespace asi

using namespace asi;

extern "C" {

asi_status_t asi_token_logprobs(const asi_logprob_desc_t* desc, const void* logits, const int64_t* targets, float* logp,
                                float* entropy, float* lse, float* top_logp, int64_t* top_ids, void* stream) {
  const asi_status_t s = check_desc(desc);
  if (s != ASI_OK) return s;
  if (desc->top_k < 0 || desc->top_k > ASI_TOP_MAX || desc->top_k > desc->vocab) return ASI_ERR_INVALID_ARG;
  if (desc->rows == 0) return ASI_OK;
  if (!logits || !targets || !logp || !lse || off_element(desc, logits)) return ASI_ERR_INVALID_ARG;
  if ((desc->top_k > 0) != (top_logp != nullptr) || (desc->top_k > 0) != (top_ids != nullptr)) return ASI_ERR_INVALID_ARG;
  LogprobArgs a = base_args(desc, logits, targets);
  a.logp = logp;
  a.entropy = entropy;
  a.lse = lse;
  a.top_logp = top_logp;
  a.top_ids = top_ids;
  a.k = desc->top_k;
  try {
    return run_logprob(desc, a, false, stream);
  } catch (...) {
    return no_host_memory();
  }
}

asi_status_t asi_token_loss(const asi_logprob_desc_t* desc, const void* logits, const int64_t* targets, const float* dlogp,
                            const float* dentropy, float* logp, float* entropy, float* lse, void* dlogits, void* stream) {
  const asi_status_t s = check_desc(desc);
  if (s != ASI_OK) return s;
  if (desc->rows == 0) return ASI_OK;
  if (!logits || !targets || !dlogp || !logp || !lse || off_element(desc, logits)) return ASI_ERR_INVALID_ARG;
  const asi_status_t g = check_grad(desc, logits, dlogits);
  if (g != ASI_OK) return g;
  LogprobArgs a = base_args(desc, logits, targets);
  a.logp = logp;
  a.entropy = entropy;
  a.lse = lse;
  a.dlogp = dlogp;
  a.dent = dentropy;
  a.dx = dlogits;
  try {
    return run_logprob(desc, a, true, stream);
  } catch (...) {
    return no_host_memory();
  }
}

asi_status_t asi_token_logprobs_grad(const asi_logprob_desc_t* desc, const void* logits, const int64_t* targets, const float* lse,
                                     const float* entropy, const float* dlogp, const float* dentropy, void* dlogits, void* stream) {
  const asi_status_t s = check_desc(desc);
  if (s != ASI_OK) return s;
  if (desc->rows == 0) return ASI_OK;
  if (!logits || !targets || !lse || !dlogp || (dentropy && !entropy) || off_element(desc, logits)) return ASI_ERR_INVALID_ARG;
  const asi_status_t g = check_grad(desc, logits, dlogits);
  if (g != ASI_OK) return g;
  LogprobGradArgs a = {};
  a.x = logits;
  a.y = targets;
  a.lse = lse;
  a.ent = entropy;
  a.dlogp = dlogp;
  a.dent = dentropy;
  a.dx = dlogits;
  a.ld = desc->ld;
  a.ldg = desc->ld_grad;
  a.ignore = desc->ignore_index;
  a.V = (int)desc->vocab;
  a.scale = desc->scale;
  const int64_t n = desc->in_dtype == ASI_BF16 ? 8 : 4, granules = (desc->vocab + 2 * n - 2) / n;
  a.splits = (int)((granules + kThreads * 4 - 1) / (kThreads * 4));
  a.blocks = desc->rows * a.splits;
  const dim3 grid((unsigned)std::min<int64_t>(a.blocks, INT32_MAX));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cuda_status(desc->in_dtype == ASI_BF16 ? launch_pdl(k_logprob_grad<__nv_bfloat16>, grid, dim3(kThreads), 0, st, a)
                                                : launch_pdl(k_logprob_grad<float>, grid, dim3(kThreads), 0, st, a),
                     "gradient of log probabilities");
}

}  // extern "C"
