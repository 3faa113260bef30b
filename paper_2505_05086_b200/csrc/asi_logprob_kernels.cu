// Log probabilities of given tokens, with entropy and top alternatives, and their gradient: the loss over the vocabulary
// whose gradient is the dY of a model's output layer.
//
// With x_j = scale * logit_j, M the largest logit, a_j = (logit_j - M) scale log2(e) and e_j = 2^a_j:
//   S = sum e_j,  W = sum e_j a_j;   lse = scale M + ln S;   entropy = ln S - ln2 W / S;   logp_j = ln2 a_j - ln S
//   dlogits_j = scale (alpha ([j = y] - p_j) - beta p_j (log p_j + entropy)) = e_j (A + B a_j) + [j = y] scale alpha
// with A = -scale (alpha + beta (entropy - ln S)) / S and B = -scale beta ln2 / S.
//
// What bounds it: the logits, read once (and the gradient, written once).  Each thread keeps a running maximum with its sums
// in packed fp32 (two values an instruction), so that one pass in registers is all that the forward direction needs; for
// the gradient the row waits in shared memory meanwhile.  Rows are split over a cluster of up to eight CTAs where they are
// long or few; the cluster's shares (M, S, W and the leading entries) meet through distributed shared memory, in rank order.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "asi_internal.h"

namespace asi {

namespace {

// Threads of a CTA and CTAs of an SM, as registers and shared memory allow: forward (one more with leading entries: their
// search waits a lot), loss, both for rows of a few granules, gradient alone
constexpr int kFwd = 128, kFwdCtas = 8, kLoss = 384, kLoss4 = 256, kLoss8 = 128, kShort = 32, kMid = 64;
constexpr int ctas_of(int threads, int large) { return threads == kShort ? 32 : threads == kMid ? 1024 / kMid : large; }
constexpr int kThreads = 128, kEach = 8;    // granules of a thread in the gradient alone (4096 x 32000 bf16, in bursts: 79 us, with 4 of them 87)
constexpr int kMaxCluster = 8;
constexpr int kShare4 = 55 << 10;           // ... with which four CTAs share an SM
constexpr int kShare = 72 << 10;            // bytes of a row that a CTA of the loss keeps, where a cluster allows it
// granules of a row for CTAs of one warp, of two, and (loss) of four
constexpr int kLittle = 160, kFew = 512, kSome = 2100;
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
// two fp32 values as one operand of the packed instructions
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum2(f2 v) {
  float a, b;
  unpair(v, a, b);
  return a + b;
}
__device__ __forceinline__ f2 exp2_both(f2 v) {
  float a, b;
  unpair(v, a, b);
  return pair(exp2_approx(a), exp2_approx(b));
}
// -inf (of a masked entry, times whose 0 it would be NaN) as a finite exponent whose power is 0 just as well
__device__ __forceinline__ f2 finite2(f2 v) {
  float a, b;
  unpair(v, a, b);
  return pair(fmaxf(a, -1e4f), fmaxf(b, -1e4f));
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
__device__ __forceinline__ int remote_int(const int* p, int rank) { return __float_as_int(remote_f(reinterpret_cast<const float*>(p), rank)); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// Sixteen bytes of a row: 8 bf16 or 4 fp32 values.
template <typename T>
struct Granule;
template <>
struct Granule<__nv_bfloat16> {
  static constexpr int n = 8;
  static constexpr uint32_t kNone = 0xff80ff80u;                    // -inf
  static constexpr uint32_t kUnit = 1u << 16;                       // the last place, of the same value in fp32
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
  static __device__ __forceinline__ void pairs(const uint4& v, f2* p) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  template <int N>
  static __device__ __forceinline__ float largest_of(const uint4* v) {
    uint32_t m = nan_max2(nan_max2(v[0].x, v[0].y), nan_max2(v[0].z, v[0].w));
#pragma unroll
    for (int q = 1; q < N; ++q) m = nan_max2(m, nan_max2(nan_max2(v[q].x, v[q].y), nan_max2(v[q].z, v[q].w)));
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
  static constexpr uint32_t kNone = 0xff800000u;
  static constexpr uint32_t kUnit = 1u;
  static __device__ __forceinline__ void floats(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float largest(const uint4& v) {
    return nan_max(nan_max(__uint_as_float(v.x), __uint_as_float(v.y)), nan_max(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ void pairs(const uint4& v, f2* p) {
    p[0] = pair(__uint_as_float(v.x), __uint_as_float(v.y));
    p[1] = pair(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  template <int N>
  static __device__ __forceinline__ float largest_of(const uint4* v) {
    float m = largest(v[0]);
#pragma unroll
    for (int q = 1; q < N; ++q) m = nan_max(m, largest(v[q]));
    return m;
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float one(float f) { return f; }
  static __device__ __forceinline__ float read(const float* p) { return *p; }
};

// Elements j .. j + n - 1 of a row one by one, -inf outside it.
template <typename T>
__device__ __forceinline__ uint4 edge_granule(const T* x, int V, int j) {
  float f[Granule<T>::n];
#pragma unroll
  for (int i = 0; i < Granule<T>::n; ++i) f[i] = j + i >= 0 && j + i < V ? Granule<T>::read(x + j + i) : -INFINITY;
  return Granule<T>::pack(f);
}

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
  // granules [first_whole(), end_whole()) are whole: all but perhaps the first and the last
  __device__ __forceinline__ int first_whole() const { return mis != 0; }
  __device__ __forceinline__ int end_whole() const { return (int)(((int64_t)mis + V) / Granule<T>::n); }
  __device__ __forceinline__ const uint4* granule(int g) const { return reinterpret_cast<const uint4*>(x - mis) + g; }
  __device__ __forceinline__ uint4 edge(int g) const { return edge_granule<T>(x, V, first(g)); }
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
__device__ __forceinline__ uint32_t order_bits(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);                     // -0 counts as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ unsigned long long order_key(float v, int j) {
  return ((unsigned long long)order_bits(v) << 32) | (0xffffffffu - (uint32_t)j);
}
__device__ __forceinline__ float key_value(unsigned long long key) { return order_value((uint32_t)(key >> 32)); }
__device__ __forceinline__ int key_index(unsigned long long key) { return (int)(0xffffffffu - (uint32_t)key); }

// S and W relative to the maximum M, from shares relative to their own; M >= each, a share of nothing has -inf
__device__ __forceinline__ void rebase(float& S, float& W, float from, float M, float c2) {
  if (from == -INFINITY) {
    S = W = 0.f;
  } else {
    const float a = (from - M) * c2, f = exp2_approx(a);
    W = f * fmaf(fmaxf(a, -1e4f), S, W);
    S *= f;
  }
}

template <int kWarps>
struct RowShared {
  float red[3][kWarps];
  float mine[3];                           // M, S, W of this CTA's share
  float parts[3][kMaxCluster];
};

// M over the CTA
template <int kWarps>
__device__ __forceinline__ float block_max(float M, float* red) {
#pragma unroll
  for (int o = 16; o; o >>= 1) M = nan_max(M, __shfl_xor_sync(~0u, M, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = M;
  __syncthreads();
  M = red[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) M = nan_max(M, red[i]);
  return M;
}
template <int kWarps>
__device__ __forceinline__ void block_sums(float& S, float& W, float (*red)[kWarps]) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    S += __shfl_xor_sync(~0u, S, o);
    W += __shfl_xor_sync(~0u, W, o);
  }
  if ((threadIdx.x & 31) == 0) red[1][threadIdx.x >> 5] = S, red[2][threadIdx.x >> 5] = W;
  __syncthreads();
  S = red[1][0], W = red[2][0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) S += red[1][i], W += red[2][i];
}
// M, S and W of the row from the shares of its cluster, in rank order, which the caller has read into sh.parts.
template <int kWarps>
__device__ __forceinline__ void cluster_sums(float& M, float& S, float& W, float c2, int cl, RowShared<kWarps>& sh) {
  float Mt = sh.parts[0][0];
  for (int q = 1; q < cl; ++q) Mt = nan_max(Mt, sh.parts[0][q]);
  S = W = 0.f;
  for (int q = 0; q < cl; ++q) {
    float s = sh.parts[1][q], w = sh.parts[2][q];
    rebase(s, w, sh.parts[0][q], Mt, c2);
    S += s;
    W += w;
  }
  M = Mt;
}

__device__ __forceinline__ void write_row(const LogprobArgs& p, int t, float M, float S, float W, float xy, bool given, bool skip) {
  const bool dead = M == -INFINITY;
  const float lnS = logf(S);
  p.lse[t] = dead ? -INFINITY : fmaf(M, p.scale, lnS);
  if (p.entropy) p.entropy[t] = dead ? 0.f : lnS - kLn2 * W / S;
  p.logp[t] = skip ? 0.f : !given ? NAN : dead ? -INFINITY : (xy - M) * p.scale - lnS;
}

// ---- forward: one pass over the row in registers, each thread with a running maximum (two passes over a copy in shared
// memory: 86 us at 4096 x 32000 bf16; this one 49, 5.4 TB/s, and in short bursts 62 with five alternatives, under sustained load
// 64).  Bound by issue slots (70 %).
constexpr int kBatch = 4;                  // granules a thread has in hand
constexpr int kSlots = 16;                 // maxima a thread remembers of what it has read
constexpr int kHits = 512;

template <int kN>
struct TopShared {
  unsigned long long cand[kCand];
  unsigned long long pool[kCand];          // and of a cluster's
  unsigned long long list[ASI_TOP_MAX];    // the leading entries, largest first
  unsigned long long best[kN / 32];
  float slot[kSlots][kN];
  uint16_t hit[kHits];                     // slot * kN + thread: granules that may hold candidates
  float most[kN];                        // each thread's maximum
  float tau;
  uint32_t least;
  int count, hits, pooled;
};

// About the k-th largest of a warp's keys: what at least k and hardly more than k + 4 of them reach.  Found bit by bit below the
// bits that all of them share.  `unit`: the last place that differs; keys of 0 are none.
template <int N>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&key)[N], int k, uint32_t unit) {
  uint32_t high = 0, low = ~0u;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    high = max(high, key[i]);
    low = min(low, key[i]);
  }
  high = __reduce_max_sync(~0u, high);
  low = __reduce_min_sync(~0u, low);
  uint32_t bit = high == low ? 0u : 1u << (31 - __clz(high ^ low)), t = bit ? high & ~(2 * bit - 1) : low;
  for (; bit >= unit; bit >>= 1) {
    uint32_t reach = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) reach += key[i] >= (t | bit);
    reach = __reduce_add_sync(~0u, reach);
    if ((int)reach >= k) t |= bit;
    if ((int)reach >= k && (int)reach <= k + 4) break;
  }
  return max(t, low);
}

// The largest key below prev among those that `each` offers, over the CTA
template <int kN, typename F>
__device__ __forceinline__ unsigned long long block_best(unsigned long long prev, unsigned long long* warps, F each) {
  unsigned long long best = 0;
  each([&](unsigned long long key) {
    if (key < prev && key > best) best = key;
  });
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const unsigned long long other = __shfl_xor_sync(~0u, best, o);
    if (other > best) best = other;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = best;
  __syncthreads();
  best = warps[0];
#pragma unroll
  for (int i = 1; i < kN / 32; ++i)
    if (warps[i] > best) best = warps[i];
  return best;
}

// S and W of some granules relative to M
template <typename T>
__device__ __forceinline__ void add_terms(const uint4& v, f2 minus, f2 k2, f2& S2, f2& W2) {
  constexpr int n = Granule<T>::n;
  f2 x[n / 2];
  Granule<T>::pairs(v, x);
#pragma unroll
  for (int e = 0; e < n / 2; ++e) {
    const f2 a = mul2(add2(x[e], minus), k2), ex = exp2_both(a);
    S2 = add2(S2, ex);
    W2 = fma2(ex, finite2(a), W2);
  }
}

// A CTA's share of a row: granules [g0, g0 + cnt), those in [lo, hi) of it whole.
template <typename T>
struct Share {
  RowView<T> row;
  int g0, cnt, lo, hi;
  __device__ __forceinline__ Share(const LogprobArgs& p, int t, int rank) : row(static_cast<const T*>(p.x) + (int64_t)t * p.ld, p.V) {
    const int G = row.granules(), per = (G + p.cl - 1) / p.cl;
    g0 = min(G, rank * per);
    cnt = min(G - g0, per);
    lo = max(row.first_whole() - g0, 0);
    hi = min(row.end_whole() - g0, cnt);
  }
  __device__ __forceinline__ explicit Share(const RowView<T>& all)
      : row(all), g0(0), cnt(all.granules()), lo(all.first_whole()), hi(all.end_whole()) {}
};

// Batch b of a share: granules b kBatch kN + q kN + tid, -inf where it runs past the share (an entry counted twice would
// spoil tau).
template <typename T, int kN>
__device__ __forceinline__ void bring(const Share<T>& s, int b, uint4* v) {
  const int i0 = b * kBatch * kN;
  const uint4* src = s.row.granule(s.g0 + i0) + threadIdx.x;
  if (i0 >= s.lo && i0 + kBatch * kN <= s.hi) {
#pragma unroll
    for (int q = 0; q < kBatch; ++q) v[q] = src[q * kN];
  } else {
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = i0 + q * kN + threadIdx.x;
      v[q] = make_uint4(Granule<T>::kNone, Granule<T>::kNone, Granule<T>::kNone, Granule<T>::kNone);
      if (i >= s.lo && i < s.hi) v[q] = src[q * kN];
      else if (i < s.cnt) v[q] = s.row.edge(s.g0 + i);
    }
  }
}

// M, S and W with a batch of granules, the largest of them `most`
template <typename T>
__device__ __forceinline__ void add_batch(const uint4* v, float most, float c2, float& M, float& S, float& W) {
  if (!(most <= M)) {
    const float to = nan_max(M, most);
    rebase(S, W, M, to, c2);
    M = to;
  }
  if (M != -INFINITY) {
    const f2 minus = pair(-M, -M), k2 = pair(c2, c2);
    f2 S2 = 0, W2 = 0;
#pragma unroll
    for (int q = 0; q < kBatch; ++q) add_terms<T>(v[q], minus, k2, S2, W2);
    S += sum2(S2);
    W += sum2(W2);
  }
}

// One pass over the share: M, S and W of this thread's granules, four of them in hand and the next four on their way.
// seen(b, most) gets each batch's maximum.
template <typename T, int kN, typename F>
__device__ __forceinline__ void stream_share(const Share<T>& s, float c2, float& M, float& S, float& W, F seen) {
  const int batches = (s.cnt + kBatch * kN - 1) / (kBatch * kN);
  M = -INFINITY, S = 0.f, W = 0.f;
  uint4 v[2][kBatch];
  if (batches) bring<T, kN>(s, 0, v[0]);
#pragma unroll 1
  for (int b0 = 0; b0 < batches; b0 += 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = b0 + h;
      if (b >= batches) break;
      if (b + 1 < batches) bring<T, kN>(s, b + 1, v[h ^ 1]);
      const float most = Granule<T>::template largest_of<kBatch>(v[h]);
      seen(b, most);
      add_batch<T>(v[h], most, c2, M, S, W);
    }
  }
}

// all but the `pending` youngest groups of copies of this thread have arrived
__device__ __forceinline__ void wait_copies(int pending) {
  if (pending >= 4) asm volatile("cp.async.wait_group 4;" ::: "memory");
  else if (pending == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
  else if (pending == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (pending == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// The same with the share left in shared memory: all of it is on its way at once, a group of copies a batch.  Every thread reads
// what it copied itself, here and later: no barrier.
template <typename T, int kN>
__device__ __forceinline__ void keep_share(const Share<T>& s, uint4* buf, float c2, float& M, float& S, float& W) {
  const int tid = threadIdx.x, batches = (s.cnt + kBatch * kN - 1) / (kBatch * kN);
  const uint4* src = s.row.granule(s.g0);
  if (tid < s.lo && s.cnt > 0) buf[0] = s.row.edge(s.g0);
  if (s.hi >= s.lo && s.hi < s.cnt && tid == s.hi % kN) buf[s.hi] = s.row.edge(s.g0 + s.hi);
#pragma unroll 1
  for (int b = 0; b < batches; ++b) {
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = (b * kBatch + q) * kN + tid;
      if (i >= s.lo && i < s.hi) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_at(buf + i)), "l"(src + i) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  M = -INFINITY, S = 0.f, W = 0.f;
#pragma unroll 1
  for (int b = 0; b < batches; ++b) {
    wait_copies(batches - 1 - b);
    uint4 v[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int i = (b * kBatch + q) * kN + tid;
      v[q] = make_uint4(Granule<T>::kNone, Granule<T>::kNone, Granule<T>::kNone, Granule<T>::kNone);
      if (i < s.cnt) v[q] = buf[i];
    }
    add_batch<T>(v, Granule<T>::template largest_of<kBatch>(v), c2, M, S, W);
  }
}

template <typename T, bool TOP, int kN>
__global__ void __launch_bounds__(kN, ctas_of(kN, kFwdCtas + TOP)) k_logprob(const __grid_constant__ LogprobArgs p) {
  constexpr int n = Granule<T>::n, kWarps = kN / 32;
  __shared__ RowShared<kWarps> sh;
  __shared__ TopShared<kN> top;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cl = p.cl, t = blockIdx.x / cl, rank = blockIdx.x - t * cl;
  const Share<T> s(p, t, rank);
  const RowView<T>& row = s.row;
  const int g0 = s.g0, cnt = s.cnt;
  const int batches = (cnt + kBatch * kN - 1) / (kBatch * kN);
  const int span = (batches + kSlots - 1) / kSlots;                 // batches that share a slot
  const float c2 = p.scale * kLog2e;

  pdl_wait();
  pdl_launch_dependents();
  const int64_t y = p.y[t];
  const bool given = y >= 0 && y < p.V, skip = y == p.ignore;
  float xy = 0.f;
  if (given && tid == 0 && rank == 0) xy = Granule<T>::read(row.x + y);

  float M, S, W, slot = -INFINITY;
  int in_slot = 0, slots = 0;
  stream_share<T, kN>(s, c2, M, S, W, [&](int b, float most) {
    if (TOP) {
      slot = nan_max(slot, most);
      if (++in_slot == span || b == batches - 1) {
        top.slot[slots++][tid] = slot;
        slot = -INFINITY;
        in_slot = 0;
      }
    }
  });

  const float own = M;
  if (TOP) {
    top.most[tid] = M;
    if (tid == 0) top.count = top.hits = 0;
  }
  M = block_max<kWarps>(M, sh.red[0]);
  rebase(S, W, own, M, c2);
  if (TOP) {
    // tau, about the k-th largest of the threads' maxima: at least k entries reach it, and few more
    if (warp == 0) {
      uint32_t key[kN / 32];
#pragma unroll
      for (int i = 0; i < kN / 32; ++i) key[i] = order_bits(top.most[i * 32 + lane]);
      const uint32_t t = reached_by(key, p.k, Granule<T>::kUnit);
      if (lane == 0) top.tau = order_value(t);
    }
  }
  block_sums<kWarps>(S, W, sh.red);

  if (TOP) {
    const float tau = top.tau;
    // The slots that reach it are listed, and each gets a warp that reads its entries once more, one a lane.
    if (own >= tau)
      for (int k = 0; k < slots; ++k)
        if (top.slot[k][tid] >= tau) {
          const int place = atomicAdd(&top.hits, 1);
          if (place < kHits) top.hit[place] = (uint16_t)(k * kN + tid);
        }
    __syncthreads();
    const int hits = top.hits;
    if (hits > kHits && tid == 0) top.count = kCand + 1;             // too many: the sweeps below
    constexpr int kEntries = kBatch * n, kAtOnce = 4;
    const int pieces = min(hits, kHits) * span;                      // (hit, batch of its slot), four of them in flight
    for (int h0 = warp; h0 < pieces; h0 += kWarps * kAtOnce) {
      float f[kAtOnce];
      int j[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int h = h0 + u * kWarps;
        j[u] = -1;
        if (h < pieces && lane < kEntries) {
          const int at = span == 1 ? h : h / span, which = top.hit[at];
          const int b = which / kN * span + (h - at * span), i = (b * kBatch + lane / n) * kN + which % kN;
          if (i < cnt) j[u] = row.first(g0 + i) + lane % n;
          if (j[u] >= p.V) j[u] = -1;
        }
        f[u] = j[u] >= 0 ? Granule<T>::read(row.x + j[u]) : -INFINITY;
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (j[u] >= 0 && f[u] >= tau) {
          const int place = atomicAdd(&top.count, 1);
          if (place < kCand) top.cand[place] = order_key(f[u], j[u]);
        }
    }
    __syncthreads();
    if (top.count > kCand) {                // many equal values: one sweep for each entry
      unsigned long long prev = ~0ull;
      for (int r = 0; r < p.k; ++r) {
        prev = block_best<kN>(prev, top.best, [&](auto offer) {
          for (int i = tid; i < cnt; i += kN) {
            float f[n];
            Granule<T>::floats(row.load(g0 + i), f);
            const int j = row.first(g0 + i);
#pragma unroll
            for (int e = 0; e < n; ++e)
              if (j + e >= 0 && j + e < p.V) offer(order_key(f[e], j + e));
          }
        });
        if (tid == 0) top.cand[r] = prev;
      }
      if (tid == 0) top.count = p.k;
    }
    if (tid == 0) top.pooled = 0;
    __syncthreads();
  }

  if (cl > 1) {
    if (tid == 0) sh.mine[0] = M, sh.mine[1] = S, sh.mine[2] = W;
    cluster_arrive();                       // (every thread's writes above, the candidates among them)
    cluster_wait();
    if (rank == 0) {
      if (tid < 3 * cl) sh.parts[tid % 3][tid / 3] = remote_f(&sh.mine[tid % 3], tid / 3);
      if (TOP) {
        // every CTA's tau is reached by k entries: the cluster's k largest reach the largest tau
        const float of_lane = remote_f(&top.tau, lane % cl);
        const int found = remote_int(&top.count, lane % cl);
        float tau = of_lane;
#pragma unroll
        for (int o = 1; o < kMaxCluster; o <<= 1) tau = fmaxf(tau, __shfl_xor_sync(~0u, tau, o));
        for (int q = warp; q < cl; q += kWarps) {
          const int of_q = __shfl_sync(~0u, found, q);
          for (int i = lane; i < of_q; i += 32) {
            const unsigned long long key = remote_u64(&top.cand[i], q);
            if (key_value(key) >= tau) {
              const int place = atomicAdd(&top.pooled, 1);
              if (place < kCand) top.pool[place] = key;
            }
          }
        }
        __syncthreads();
        if (top.pooled <= kCand) {          // up to eight times as many as wanted: tau once more, over them
          const int pooled = top.pooled;
          if (warp == 0) {
            uint32_t key[kCand / 32];
#pragma unroll
            for (int i = 0; i < kCand / 32; ++i) key[i] = i * 32 + lane < pooled ? (uint32_t)(top.pool[i * 32 + lane] >> 32) : 0u;
            const uint32_t t = reached_by(key, p.k, Granule<T>::kUnit);
            if (lane == 0) top.least = t;
          }
          __syncthreads();
          unsigned long long keep[kCand / kN];
#pragma unroll
          for (int i = 0; i < kCand / kN; ++i) keep[i] = i * kN + tid < pooled ? top.pool[i * kN + tid] : 0;
          if (tid == 0) top.pooled = 0;
          __syncthreads();
#pragma unroll
          for (int i = 0; i < kCand / kN; ++i)
            if (keep[i] && (uint32_t)(keep[i] >> 32) >= top.least) top.pool[atomicAdd(&top.pooled, 1)] = keep[i];
        } else {                            // many equal values again
          unsigned long long prev = ~0ull;
          for (int r = 0; r < p.k; ++r) {
            prev = block_best<kN>(prev, top.best, [&](auto offer) {
              for (int q = 0; q < cl; ++q) {
                const int of_q = __shfl_sync(~0u, found, q);
                for (int i = tid; i < of_q; i += kN) offer(remote_u64(&top.cand[i], q));
              }
            });
            if (tid == 0) top.pool[r] = prev;
          }
          if (tid == 0) top.pooled = p.k;
        }
      }
      __syncthreads();
    }
    cluster_arrive();                       // the others' shared memory is read no more
    cluster_wait();
    if (rank) return;
    cluster_sums<kWarps>(M, S, W, c2, cl, sh);
  }
  if (TOP) {
    const unsigned long long* from = cl > 1 ? top.pool : top.cand;
    const int found = min(cl > 1 ? top.pooled : top.count, kCand);
    for (int i = tid; i < found; i += kN) {
      const unsigned long long key = from[i];
      int above = 0;
#pragma unroll 4
      for (int q = 0; q < found; ++q) above += from[q] > key;
      if (above < p.k) top.list[above] = key;
    }
    __syncthreads();
  }
  if (tid == 0) write_row(p, t, M, S, W, xy, given, skip);
  if (TOP && tid < p.k) {
    const float lnS = logf(S);
    const bool fine = !isnan(lnS), dead = M == -INFINITY;
    const unsigned long long key = fine ? top.list[tid] : 0;
    p.top_ids[(int64_t)t * p.k + tid] = fine ? key_index(key) : tid;
    p.top_logp[(int64_t)t * p.k + tid] = !fine ? NAN : dead ? -INFINITY : (key_value(key) - M) * p.scale - lnS;
  }
}

// ---- forward and gradient.  Bound by the exponentials, two an element (4096 x 32000 bf16: in short bursts 100 us, 67 % of their
// unit, 5.2 TB/s, under sustained load 108; 1001 x 50257 fp32: 82 and 87 us).  RES: the CTA's share of the row stays in shared
// memory between the sums and the gradient (else it is read again: rows of more than 1.6 MB).  Every thread reads back what it left
// there itself: no barrier.
template <typename T, bool RES, int kN>
__global__ void __launch_bounds__(kN, ctas_of(kN, kN == kLoss8 ? 8 : kN == kLoss4 ? 4 : 3)) k_loss(const __grid_constant__ LogprobArgs p) {
  constexpr int n = Granule<T>::n, kWarps = kN / 32;
  extern __shared__ uint4 buf[];
  __shared__ RowShared<kWarps> sh;
  const int tid = threadIdx.x, cl = p.cl, t = blockIdx.x / cl, rank = blockIdx.x - t * cl;
  const float c2 = p.scale * kLog2e;
  const Share<T> s(p, t, rank);
  pdl_wait();
  pdl_launch_dependents();
  const int64_t y = p.y[t];
  const bool given = y >= 0 && y < p.V, skip = y == p.ignore;
  // the given entry: read by the thread that reports logp and by the one that writes its gradient (dx may be x)
  const int yg = given ? (int)((s.row.mis + y) / n) - s.g0 : -1;
  const bool mine = yg >= 0 && yg < s.cnt && yg % kN == tid;
  float xy = 0.f;
  if (mine || (given && tid == 0 && rank == 0)) xy = Granule<T>::read(s.row.x + y);
  const float alpha = p.dlogp[t], beta = p.dent ? p.dent[t] : 0.f;

  float M, S, W;
  if (RES) keep_share<T, kN>(s, buf, c2, M, S, W);
  else stream_share<T, kN>(s, c2, M, S, W, [](int, float) {});
  const float own = M;
  M = block_max<kWarps>(M, sh.red[0]);
  rebase(S, W, own, M, c2);
  block_sums<kWarps>(S, W, sh.red);
  if (cl > 1) {
    if (tid == 0) sh.mine[0] = M, sh.mine[1] = S, sh.mine[2] = W;
    cluster_arrive();
    cluster_wait();
    if (tid < 3 * cl) sh.parts[tid % 3][tid / 3] = remote_f(&sh.mine[tid % 3], tid / 3);
    __syncthreads();
    cluster_arrive();                       // the others' shared memory is read no more; waited for at the end
    cluster_sums<kWarps>(M, S, W, c2, cl, sh);
  }
  if (rank == 0 && tid == 0) write_row(p, t, M, S, W, xy, given, skip);

  T* dx = static_cast<T*>(p.dx) + (int64_t)t * p.ldg;
  // granules stored whole: where dx starts on the same offset within 16 bytes as x
  const bool wide = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(s.row.x)) & 15) == 0;
  const int wlo = wide ? s.lo : s.cnt, whi = wide ? s.hi : 0;
  uint4* to = reinterpret_cast<uint4*>(dx - s.row.mis) + s.g0;
  auto put = [&](int i, const float (&f)[n]) {
    if (i >= wlo && i < whi) {
      to[i] = Granule<T>::pack(f);
    } else {
      const int j = s.row.first(s.g0 + i);
#pragma unroll
      for (int e = 0; e < n; ++e)
        if (j + e >= 0 && j + e < s.row.V) dx[j + e] = Granule<T>::one(f[e]);
    }
  };
  if (skip || M == -INFINITY) {
    float f[n];
#pragma unroll
    for (int e = 0; e < n; ++e) f[e] = 0.f;
    for (int i = tid; i < s.cnt; i += kN) put(i, f);
  } else {
    const float inv = 1.f / S, lnS = logf(S), H = lnS - kLn2 * W * inv;
    const float A = given ? -p.scale * (alpha + beta * (H - lnS)) * inv : NAN, B = -p.scale * beta * kLn2 * inv;
    const f2 minus = pair(-M, -M), k2 = pair(c2, c2), A2 = pair(A, A), B2 = pair(B, B);
    const uint4* src = s.row.granule(s.g0);
    auto gradient = [&](auto with_entropy) {
#pragma unroll 2
      for (int i = tid; i < s.cnt; i += kN) {
        f2 x[n / 2];
        Granule<T>::pairs(RES ? buf[i] : i >= s.lo && i < s.hi ? src[i] : s.row.edge(s.g0 + i), x);
        float f[n];
#pragma unroll
        for (int e = 0; e < n / 2; ++e) {
          const f2 a = mul2(add2(x[e], minus), k2);
          unpair(mul2(exp2_both(a), decltype(with_entropy)::value ? fma2(B2, finite2(a), A2) : A2), f[2 * e], f[2 * e + 1]);
        }
        put(i, f);
      }
    };
    if (beta != 0.f) gradient(std::true_type());
    else gradient(std::false_type());
    if (mine) {
      const float a = (xy - M) * c2;
      dx[y] = Granule<T>::one(fmaf(p.scale, alpha, exp2_approx(a) * fmaf(B, fmaxf(a, -1e4f), A)));
    }
  }
  if (cl > 1) cluster_wait();
}

// ---- the gradient alone, from lse and entropy: a stream of 1024 granules a CTA (4096 x 32000 bf16: 78 us in short bursts, 83 under
// sustained load, floor 81).
// p = exp(x - lse) is off by 2^-24 |lse|: rows where that would show in the type (2^-17 in fp32, 2^-12 beside the 2^-9 of a
// rounding to bf16; logits that share an offset, or lie at a type's lowest value) sum up for themselves, in one CTA (dx may be
// x, so nobody else of the row may have begun to write).  fp32, all logits around 1000: 1001 x 50257 takes 111 us instead of 61, 4 x
// 131073 takes 72 instead of 8, and the median error of an entry is 2.6e-7 of it instead of 1.5e-5.
template <typename T>
constexpr float kFarLse = sizeof(T) == 4 ? 128.f : 4096.f;

template <typename T>
__device__ __forceinline__ void far_row(const LogprobGradArgs& p, const RowView<T>& row, T* dx, int64_t t, bool wide) {
  constexpr int n = Granule<T>::n, kWarps = kThreads / 32;
  __shared__ RowShared<kWarps> sh;
  const Share<T> s(row);
  const int tid = threadIdx.x;
  const int64_t y = p.y[t];
  const bool given = y >= 0 && y < p.V;
  const float c2 = p.scale * kLog2e, alpha = p.dlogp[t], beta = p.dent ? p.dent[t] : 0.f;
  float M = -INFINITY, S = 0.f, W = 0.f;
#pragma unroll 1
  for (int b = 0; b * kBatch * kThreads < s.cnt; ++b) {
    uint4 v[kBatch];
    bring<T, kThreads>(s, b, v);
    add_batch<T>(v, Granule<T>::template largest_of<kBatch>(v), c2, M, S, W);
  }
  const float own = M;
  M = block_max<kWarps>(M, sh.red[0]);
  rebase(S, W, own, M, c2);
  block_sums<kWarps>(S, W, sh.red);
  const bool zero = y == p.ignore || M == -INFINITY;
  const float inv = 1.f / S, lnS = logf(S), H = lnS - kLn2 * W * inv;
  const float A = given ? -p.scale * (alpha + beta * (H - lnS)) * inv : NAN, B = -p.scale * beta * kLn2 * inv;
  const f2 minus = pair(-M, -M), k2 = pair(c2, c2), A2 = pair(A, A), B2 = pair(B, B);
#pragma unroll 1
  for (int b = 0; b * kBatch * kThreads < s.cnt; ++b) {
    uint4 v[kBatch];
    bring<T, kThreads>(s, b, v);
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int g = (b * kBatch + q) * kThreads + tid;
      if (g >= s.cnt) break;
      f2 x[n / 2];
      Granule<T>::pairs(v[q], x);
      const int j = row.first(g);
      float f[n];
#pragma unroll
      for (int e = 0; e < n / 2; ++e) {
        const f2 a = mul2(add2(x[e], minus), k2);
        unpair(mul2(exp2_both(a), fma2(B2, finite2(a), A2)), f[2 * e], f[2 * e + 1]);
      }
#pragma unroll
      for (int e = 0; e < n; ++e) f[e] = zero ? 0.f : j + e == y ? fmaf(p.scale, alpha, f[e]) : f[e];
      store_granule(dx, row, g, f, wide);
    }
  }
  __syncthreads();                           // sh is free
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_logprob_grad(const __grid_constant__ LogprobGradArgs p) {
  constexpr int n = Granule<T>::n;
  pdl_wait();
  pdl_launch_dependents();
  for (int64_t b = blockIdx.x; b < p.blocks; b += gridDim.x) {
    const int64_t t = b / p.splits;
    const int split = (int)(b - t * p.splits), g0 = split * kThreads * kEach + threadIdx.x;
    const RowView<T> row(static_cast<const T*>(p.x) + t * p.ld, p.V);
    const int G = row.granules();
    T* dx = static_cast<T*>(p.dx) + t * p.ldg;
    const bool wide = ((reinterpret_cast<uintptr_t>(dx) ^ reinterpret_cast<uintptr_t>(row.x)) & 15) == 0;
    const int64_t y = p.y[t];
    const float lse = p.lse[t], alpha = p.dlogp[t], beta = p.dent ? p.dent[t] : 0.f, H = p.dent ? p.ent[t] : 0.f;
    if (fabsf(lse) >= kFarLse<T>) {
      if (split == 0) far_row(p, row, dx, t, wide);
      continue;
    }
    const bool given = y >= 0 && y < p.V, zero = y == p.ignore;
    const float A = given ? -p.scale * (alpha + beta * H) : NAN, B = -p.scale * beta;
    uint4 v[kEach];
#pragma unroll
    for (int q = 0; q < kEach; ++q) {
      const int g = g0 + q * kThreads;
      v[q] = make_uint4(0, 0, 0, 0);
      if (g < G && !zero) v[q] = row.load(g);
    }
    const f2 scale2 = pair(p.scale, p.scale), minus = pair(-lse, -lse), e2 = pair(kLog2e, kLog2e), A2 = pair(A, A), B2 = pair(B, B);
    const int yj = given && !zero ? (int)y : -1;
    auto gradient = [&](auto with_entropy) {
#pragma unroll
      for (int q = 0; q < kEach; ++q) {
        const int g = g0 + q * kThreads;
        if (g >= G) break;
        f2 x[n / 2];
        Granule<T>::pairs(v[q], x);
        float f[n];
#pragma unroll
        for (int e = 0; e < n / 2; ++e) {
          const f2 lp = fma2(x[e], scale2, minus);
          unpair(mul2(exp2_both(mul2(lp, e2)), decltype(with_entropy)::value ? fma2(B2, finite2(lp), A2) : A2), f[2 * e], f[2 * e + 1]);
        }
        const int j = row.first(g);
        if (yj >= j && yj < j + n) {
#pragma unroll
          for (int e = 0; e < n; ++e) f[e] += j + e == yj ? p.scale * alpha : 0.f;
        }
        store_granule(dx, row, g, f, wide);
      }
    };
    if (zero) {
      float f[n];
#pragma unroll
      for (int e = 0; e < n; ++e) f[e] = 0.f;
      for (int q = 0; q < kEach; ++q)
        if (g0 + q * kThreads < G) store_granule(dx, row, g0 + q * kThreads, f, wide);
    } else if (beta != 0.f) {
      gradient(std::true_type());
    } else {
      gradient(std::false_type());
    }
  }
}

template <typename K>
cudaError_t launch_rows(K kernel, int threads, const LogprobArgs& a, int64_t rows, size_t smem, cudaStream_t st) {
  if (smem > 32 << 10) {
    const cudaError_t e = opt_in_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * a.cl));
  cfg.blockDim = dim3((unsigned)threads);
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

// CTAs of a row: more where the rows alone do not give every SM `each` CTAs, while a share keeps `least` granules
int spread_rows(int64_t rows, int64_t granules, int cl, int each, int least) {
  while (cl < kMaxCluster && rows * cl < 148 * each && granules >= (int64_t)2 * cl * least) cl *= 2;
  return cl;
}

template <typename T>
cudaError_t launch_logprob(LogprobArgs a, int64_t rows, bool grad, cudaStream_t st) {
  const int64_t granules = ((int64_t)a.V + 2 * Granule<T>::n - 2) / Granule<T>::n;   // of a row at the worst offset
  // Rows of a few granules leave most threads of a large CTA without work and wait for its barriers: where there are many of
  // them, smaller CTAs (loss of 8192 x 300 bf16: 13 us with 32 threads, 54 with 256; of 4096 x 16000: 56 with 128, 64 with
  // 256; of 4096 x 24000: 91 and 86.  Forward, 4096 x 3000 and 5 alternatives: 18 us with 64, 21 with 128).
  const bool many = rows >= 148 * 4, little = many && granules <= kLittle, few = many && granules <= kFew, some = many && granules <= kSome;
  if (!grad) {
    a.cl = few ? 1 : spread_rows(rows, granules, 1, 5, 2 * kFwd);
    if (little) return a.k ? launch_rows(k_logprob<T, true, kShort>, kShort, a, rows, 0, st) : launch_rows(k_logprob<T, false, kShort>, kShort, a, rows, 0, st);
    if (few) return a.k ? launch_rows(k_logprob<T, true, kMid>, kMid, a, rows, 0, st) : launch_rows(k_logprob<T, false, kMid>, kMid, a, rows, 0, st);
    return a.k ? launch_rows(k_logprob<T, true, kFwd>, kFwd, a, rows, 0, st) : launch_rows(k_logprob<T, false, kFwd>, kFwd, a, rows, 0, st);
  }
  // shares of 72 KB at most let three CTAs run on an SM
  a.cl = 1;
  while (a.cl < kMaxCluster && granules * 16 > (int64_t)a.cl * kShare) a.cl *= 2;
  if (!some) a.cl = spread_rows(rows, granules, a.cl, 1, kLoss);
  const size_t share = (size_t)((granules + a.cl - 1) / a.cl) * 16;
  if (little) return launch_rows(k_loss<T, true, kShort>, kShort, a, rows, share, st);
  if (few) return launch_rows(k_loss<T, true, kMid>, kMid, a, rows, share, st);
  if (some) return launch_rows(k_loss<T, true, kLoss8>, kLoss8, a, rows, share, st);
  if (share <= kShare4) return launch_rows(k_loss<T, true, kLoss4>, kLoss4, a, rows, share, st);
  return share <= 200 << 10 ? launch_rows(k_loss<T, true, kLoss>, kLoss, a, rows, share, st)
                            : launch_rows(k_loss<T, false, kLoss>, kLoss, a, rows, 0, st);
}

asi_status_t check_desc(const asi_logprob_desc_t* d) {
  if (!d || (d->in_dtype != ASI_F32 && d->in_dtype != ASI_BF16)) return ASI_ERR_INVALID_ARG;
  if (d->rows < 0 || d->vocab < 1 || d->ld < d->vocab) return ASI_ERR_INVALID_ARG;
  if (!(d->scale >= 1e-8f && d->scale <= 1e8f)) return ASI_ERR_INVALID_ARG;
  if (d->rows > ASI_LOGPROB_MAX_ROWS || d->vocab > ASI_LOGPROB_MAX_VOCAB) return ASI_ERR_UNSUPPORTED;
  if (d->ld > INT64_MAX / 8 / std::max<int64_t>(d->rows, 1)) return ASI_ERR_INVALID_ARG;
  return ASI_OK;
}

size_t logit_bytes(const asi_logprob_desc_t* d) { return d->in_dtype == ASI_BF16 ? 2 : 4; }

bool off_element(const asi_logprob_desc_t* d, const void* p) { return asi::off_element(p, logit_bytes(d)); }

bool off_float(std::initializer_list<const float*> buffers) {
  for (const float* p : buffers)
    if (asi::off_element(p, 4)) return true;
  return false;
}

// dlogits is logits itself, row for row, or lies apart from it (between its rows, perhaps, where both have the same stride)
asi_status_t check_grad(const asi_logprob_desc_t* d, const void* x, const void* dx) {
  if (!dx || off_element(d, dx) || d->ld_grad < d->vocab) return ASI_ERR_INVALID_ARG;
  if (d->ld_grad > INT64_MAX / 8 / std::max<int64_t>(d->rows, 1)) return ASI_ERR_INVALID_ARG;
  const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(dx);
  if (a == b) return d->ld_grad == d->ld || d->rows == 1 ? ASI_OK : ASI_ERR_INVALID_ARG;
  const uintptr_t row = d->vocab * logit_bytes(d), stride = d->ld * logit_bytes(d), shift = (a < b ? b - a : a - b) % stride;
  if (d->ld == d->ld_grad && shift >= row && stride - shift >= row) return ASI_OK;
  const uintptr_t na = ((d->rows - 1) * d->ld + d->vocab) * logit_bytes(d), nb = ((d->rows - 1) * d->ld_grad + d->vocab) * logit_bytes(d);
  return a < b + nb && b < a + na ? ASI_ERR_INVALID_ARG : ASI_OK;
}

// A contiguous buffer of a call; null where the call has none
struct Span {
  const void* p;
  size_t bytes;
  bool meets(const Span& o) const {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
    return p && o.p && a < b + o.bytes && b < a + bytes;
  }
};

// The span meets a row of logits or dlogits, `ld` elements apart (it may lie between two of them).
bool meets_rows(const asi_logprob_desc_t* d, const Span& s, const void* rows, int64_t ld) {
  if (!s.p || !rows) return false;
  const uintptr_t at = reinterpret_cast<uintptr_t>(rows), a = reinterpret_cast<uintptr_t>(s.p);
  const uintptr_t row = d->vocab * logit_bytes(d), stride = ld * logit_bytes(d), end = at + (d->rows - 1) * stride + row;
  if (a + s.bytes <= at || a >= end) return false;
  return a < at || (a - at) % stride < row || (a - at) % stride + s.bytes > stride;
}

// What a call writes (`out`, and dlogits if any) meets nothing that it reads or writes beside.  dlogits over logits is check_grad's.
bool written_apart(const asi_logprob_desc_t* d, const void* logits, const void* dlogits, std::initializer_list<Span> out,
                   std::initializer_list<Span> in) {
  for (const Span* o = out.begin(); o != out.end(); ++o) {
    if (meets_rows(d, *o, logits, d->ld) || meets_rows(d, *o, dlogits, d->ld_grad)) return false;
    for (const Span* q = out.begin(); q != o; ++q)
      if (o->meets(*q)) return false;
    for (const Span& i : in)
      if (o->meets(i)) return false;
  }
  for (const Span& i : in)
    if (meets_rows(d, i, dlogits, d->ld_grad)) return false;
  return true;
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
  if (off_element(targets, 8) || off_element(top_ids, 8) || off_float({logp, entropy, lse, top_logp})) return ASI_ERR_INVALID_ARG;
  const size_t n = (size_t)desc->rows, top = n * desc->top_k;
  if (!written_apart(desc, logits, nullptr, {{logp, 4 * n}, {entropy, 4 * n}, {lse, 4 * n}, {top_logp, 4 * top}, {top_ids, 8 * top}},
                     {{targets, 8 * n}}))
    return ASI_ERR_INVALID_ARG;
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
  if (off_element(targets, 8) || off_float({dlogp, dentropy, logp, entropy, lse})) return ASI_ERR_INVALID_ARG;
  const size_t n = (size_t)desc->rows;
  if (!written_apart(desc, logits, dlogits, {{logp, 4 * n}, {entropy, 4 * n}, {lse, 4 * n}},
                     {{targets, 8 * n}, {dlogp, 4 * n}, {dentropy, 4 * n}}))
    return ASI_ERR_INVALID_ARG;
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
  if (off_element(targets, 8) || off_float({lse, dlogp, dentropy, dentropy ? entropy : nullptr})) return ASI_ERR_INVALID_ARG;
  const size_t rows = (size_t)desc->rows;
  if (!written_apart(desc, logits, dlogits, {},
                     {{targets, 8 * rows}, {lse, 4 * rows}, {dlogp, 4 * rows}, {dentropy, 4 * rows}, {dentropy ? entropy : nullptr, 4 * rows}}))
    return ASI_ERR_INVALID_ARG;
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
  a.splits = (int)((granules + kThreads * kEach - 1) / (kThreads * kEach));
  a.blocks = desc->rows * a.splits;
  const dim3 grid((unsigned)std::min<int64_t>(a.blocks, INT32_MAX));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return cuda_status(desc->in_dtype == ASI_BF16 ? launch_pdl(k_logprob_grad<__nv_bfloat16>, grid, dim3(kThreads), 0, st, a)
                                                : launch_pdl(k_logprob_grad<float>, grid, dim3(kThreads), 0, st, a),
                     "gradient of log probabilities");
}

}  // extern "C"
