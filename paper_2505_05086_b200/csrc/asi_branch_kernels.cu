// A block's end: dropout by a counter-based generator, and what joins a branch to the residual stream, with its gradient.
//
//   out = keep(e) x / (1 - p) [+ residual]
//   z = norm(y);  h' = r h + b drop(gate z);  x = norm(h')
//
// and backwards, with hats for what a norm made of its input before weight and bias, D values a row:
//   a = dx w_n;  d = dh' + s_n (a - h^ mean(a h^) - mean a);   dh = r d;   u = drop(b d);   v = gate u w_a
//   dy = s_a (v - y^ mean(v y^) - mean v);   dgate = sum u z,  dw_a = sum gate u y^,  db_a = sum gate u,  dw_n = sum dx h^,  db_n = sum dx
// (mean a and mean v are layer norm's alone).  With S1 = sum u y^ and S0 = sum u over the rows of a gate's row:
//   dgate = w_a S1 + b_a S0,  dw_a = sum over the gate's rows of gate S1,  db_a = sum of gate S0.
//
// What bounds them: bytes.  A thread keeps eight values of its row in registers, a row's sums meet in shared memory, and what the
// backward pass sums over rows stays in the threads' registers from row to row: each worker (the threads of a row) takes
// neighbouring rows and leaves one partial sum a column, which k_branch_sums adds up in order.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "asi_internal.h"
#include "asi_philox.h"

namespace asi {

namespace {

constexpr int kEach = 8;                   // values of a thread: a group of the generator
constexpr int kDropThreads = 256;

struct Drop {
  uint64_t seed;
  const int64_t* step_dev;
  uint32_t stream, step, below;            // dropped where sixteen bits are below `below`; 0: nothing is
  float more;                              // 65536 / (65536 - below)
};

__device__ __forceinline__ uint32_t step_of(const Drop& d) { return d.step_dev ? (uint32_t)*d.step_dev : d.step; }
__device__ __forceinline__ Words words_of(const Drop& d, uint32_t step, uint64_t group) {
  return philox4x32_10((uint32_t)group, (uint32_t)(group >> 32), d.stream, step, (uint32_t)d.seed, (uint32_t)(d.seed >> 32));
}
__device__ __forceinline__ bool kept(const Drop& d, const Words& w, int j) {
  const uint32_t x = w.w[j >> 1];
  return (j & 1 ? x >> 16 : x & 0xffffu) >= d.below;
}
__device__ __forceinline__ bool kept_alone(const Drop& d, uint32_t step, uint64_t e) {
  const Words w = words_of(d, step, e >> 3);
  const int j = (int)(e & 7);
  const uint32_t x = j < 4 ? (j < 2 ? w.w[0] : w.w[1]) : (j < 6 ? w.w[2] : w.w[3]);
  return (j & 1 ? x >> 16 : x & 0xffffu) >= d.below;
}

// eight neighbouring values, aligned to as many bytes as they have.  (32 bytes of fp32 in one piece: two of 16 would each touch every sector of
// the warp's kilobyte and write half of it)
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&f)[kEach]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(u[i] << 16), f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
}
__device__ __forceinline__ void load8(const float* p, float (&f)[kEach]) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&f)[kEach]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&f)[kEach]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]),
               "f"(f[6]), "f"(f[7])
               : "memory");
}
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
template <typename T>
__device__ __forceinline__ float stored(float x) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(__float2bfloat16_rn(x));
  else return x;
}

// Eight values at a time, two an instruction
__device__ __forceinline__ void fma2(float* d, const float* a, const float* b, const float* c) {
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]), "f"(c[0]), "f"(c[1]));
}
__device__ __forceinline__ void mul2(float* d, const float* a, const float* b) {
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]));
}
__device__ __forceinline__ void add2(float* d, const float* a, const float* b) {
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]));
}
using Eight = float[kEach];
__device__ __forceinline__ void fma8(Eight& d, const Eight& a, const Eight& b, const Eight& c) {
#pragma unroll
  for (int i = 0; i < kEach; i += 2) fma2(d + i, a + i, b + i, c + i);
}
__device__ __forceinline__ void fma8(Eight& d, const Eight& a, float b, const Eight& c) {
  const float q[2] = {b, b};
#pragma unroll
  for (int i = 0; i < kEach; i += 2) fma2(d + i, a + i, q, c + i);
}
__device__ __forceinline__ void fma8(Eight& d, const Eight& a, float b, float c) {
  const float q[2] = {b, b}, r[2] = {c, c};
#pragma unroll
  for (int i = 0; i < kEach; i += 2) fma2(d + i, a + i, q, r);
}
__device__ __forceinline__ void mul8(Eight& d, const Eight& a, const Eight& b) {
#pragma unroll
  for (int i = 0; i < kEach; i += 2) mul2(d + i, a + i, b + i);
}
__device__ __forceinline__ void mul8(Eight& d, const Eight& a, float b) {
  const float q[2] = {b, b};
#pragma unroll
  for (int i = 0; i < kEach; i += 2) mul2(d + i, a + i, q);
}
__device__ __forceinline__ void add8(Eight& d, const Eight& a, const Eight& b) {
#pragma unroll
  for (int i = 0; i < kEach; i += 2) add2(d + i, a + i, b + i);
}
__device__ __forceinline__ void add8(Eight& d, const Eight& a, float b) {
  const float q[2] = {b, b};
#pragma unroll
  for (int i = 0; i < kEach; i += 2) add2(d + i, a + i, q);
}
__device__ __forceinline__ float dot8(const Eight& a, const Eight& b) {
  float x[2], y[2];
  mul2(x, a, b), mul2(y, a + 2, b + 2);
  fma2(x, a + 4, b + 4, x), fma2(y, a + 6, b + 6, y);
  add2(x, x, y);
  return x[0] + x[1];
}
__device__ __forceinline__ float sum8(const Eight& a) {
  float x[2], y[2];
  add2(x, a, a + 2), add2(y, a + 4, a + 6);
  add2(x, x, y);
  return x[0] + x[1];
}

struct DropoutArgs {
  const void *x, *res;
  void* out;
  int64_t n;
  Drop drop;
};

// A group of eight a thread.  (The words need nothing that the kernel before has written, but for a step number on the device.)
template <typename T, bool kVec>
__global__ void __launch_bounds__(kDropThreads) k_dropout(const __grid_constant__ DropoutArgs p) {
  const int64_t g = (int64_t)blockIdx.x * kDropThreads + threadIdx.x, at = g * kEach;
  if (p.drop.step_dev) pdl_wait();
  const Words w = words_of(p.drop, step_of(p.drop), (uint64_t)g);
  if (!p.drop.step_dev) pdl_wait();
  pdl_launch_dependents();
  if (at >= p.n) return;
  const T *x = static_cast<const T*>(p.x) + at, *res = p.res ? static_cast<const T*>(p.res) + at : nullptr;
  T* out = static_cast<T*>(p.out) + at;
  if (kVec && at + kEach <= p.n) {
    float f[kEach], r[kEach];
    load8(x, f);
    if (res) load8(res, r);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      f[i] = kept(p.drop, w, i) ? f[i] * p.drop.more : 0.f;
      if (res) f[i] += r[i];
    }
    store8(out, f);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (at + i < p.n) {
        const float f = kept(p.drop, w, i) ? value(x[i]) * p.drop.more : 0.f;
        put(out + i, res ? f + value(res[i]) : f);
      }
  }
}

struct BranchArgs {
  const void *y, *h;
  const float *gate, *aw, *ab, *nw, *nb;
  void *h_out, *x;
  float* stats;
  const void *dx, *dh_out;
  void *dy, *dh;
  float *dgate, *daw, *dab, *dnw, *dnb;
  float* part;             // [kParts][workers][dim]
  int64_t rows, per;       // rows of a gate's row
  int64_t run;             // rows of a worker
  int workers, dim, norm_after, accumulate;
  int zero_sums;           // S0 is wanted (a bias behind the norm after: of dgate, or its own gradient)
  int stages;              // rows on their way at once
  float eps, rs, bs, inv_dim;
  Drop drop;
};
// partial sums of a worker: over the first of its gate's rows, over the last one, over all
enum Part { kHead1 = 0, kTail1 = 1, kNext1 = 2, kAfter1 = 3, kHead0 = 4, kTail0 = 5, kNext0 = 6, kAfter0 = 7, kParts = 8 };

// Sums of up to three values over the threads of a CTA, for all of them (a multiple of 32, kMax at most)
template <int kMax>
struct RowSum {
  static constexpr int kWarps = kMax / 32, kMost = 3;
  float* sh;               // [2][kMost][kWarps], 0 where no warp writes
  uint32_t phase = 0;
  __device__ __forceinline__ RowSum(float* s) : sh(s) {
    for (int i = threadIdx.x; i < 2 * kMost * kWarps; i += blockDim.x) s[i] = 0.f;
    __syncthreads();
  }
  template <int kN>
  __device__ __forceinline__ void get(float (&v)[kN]) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += __shfl_xor_sync(~0u, v[i], o);
    if (blockDim.x == 32) return;
    float* s = sh + phase;
    phase ^= kMost * kWarps;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int i = 0; i < kN; ++i) s[i * kWarps + (threadIdx.x >> 5)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float x[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kWarps; k += 4) {
        const float4 q = *reinterpret_cast<const float4*>(s + i * kWarps + k);
        const float lo[2] = {q.x, q.y}, hi[2] = {q.z, q.w};
        add2(x, x, lo), add2(x, x, hi);
      }
      v[i] = x[0] + x[1];
    }
  }
  __device__ __forceinline__ float one(float a) {
    float v[1] = {a};
    get(v);
    return v[0];
  }
};

// A thread's columns: eight neighbours, or (rows off 16 bytes) eight a row's threads apart.
template <bool kVec>
struct Columns {
  int first, step, dim;
  __device__ __forceinline__ Columns(int d) : first(kVec ? threadIdx.x * kEach : threadIdx.x), step(kVec ? 1 : blockDim.x), dim(d) {}
  __device__ __forceinline__ int at(int i) const { return first + i * step; }
  __device__ __forceinline__ bool there(int i) const { return kVec ? first < dim : at(i) < dim; }
  template <typename T>
  __device__ __forceinline__ void load(const T* row, float (&f)[kEach], bool any = true) const {
    if constexpr (kVec) {
      if (any && first < dim) {
        load8(row + first, f);
      } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) f[i] = 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) f[i] = any && at(i) < dim ? value(row[at(i)]) : 0.f;
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (&f)[kEach]) const {
    if constexpr (kVec) {
      if (first < dim) store8(row + first, f);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (at(i) < dim) put(row + at(i), f[i]);
    }
  }
  // fp32 parameters, `none` where there are none, 0 where there is no column; they start at any float
  __device__ __forceinline__ void param(const float* p, float (&f)[kEach], float none, bool wide) const {
    if (!p) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) f[i] = there(i) ? none : 0.f;
    } else if (kVec && wide) {
      load(p, f);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) f[i] = there(i) ? __ldg(p + at(i)) : 0.f;
    }
  }
  // which of this thread's values of row t stay, a bit each
  __device__ __forceinline__ uint32_t kept_bits(const Drop& d, uint32_t step_no, int64_t t) const {
    const uint64_t e = (uint64_t)t * dim + first;
    uint32_t bits = 0;
    if constexpr (kVec) {
      const Words w = words_of(d, step_no, e >> 3);         // (dim is a multiple of eight)
#pragma unroll
      for (int i = 0; i < kEach; ++i) bits |= kept(d, w, i) ? 1u << i : 0u;
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (at(i) < dim) bits |= kept_alone(d, step_no, e + (uint64_t)i * step) ? 1u << i : 0u;
    }
    return bits;
  }
  static __device__ __forceinline__ void drop(const Drop& d, uint32_t bits, Eight& f) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) f[i] = bits >> i & 1 ? f[i] * d.more : 0.f;
  }
};

// Rows on their way: a warp copies its values of the next rows to shared memory and reads them there itself, so that no warp waits for
// another (rows on 16 bytes, of fp32 on 32, alone).  A thread brings 16 bytes at a time, neighbours side by side: of fp32 half of its own
// eight values or another's (its own two halves would read every sector twice, past L1: 6304 x 768 34.1 us instead of 33.4).  A stage is a row: kTensors slots of kPieces times 16 bytes a thread, 0 where
// nothing is fetched (columns beyond the row's end, tensors that a call has not).
constexpr int kMaxStages = 4;
template <int kTensors, int kPieces>
struct Ring {
  uint32_t mine, piece, stage_bytes, at;                   // (at: of the row that is next)
  int stages, left;
  __device__ __forceinline__ Ring(void* smem, int n) {
    mine = at = (uint32_t)__cvta_generic_to_shared(smem) + threadIdx.x * 16;
    piece = blockDim.x * 16;
    stage_bytes = kTensors * kPieces * piece;
    stages = left = n;
  }
  __device__ __forceinline__ void clear() const {
    for (int i = 0; i < stages * kTensors * kPieces; ++i)
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(mine + i * piece), "r"(0) : "memory");
  }
  // the warp's part of a row into stage `to`; first: this thread's first column
  template <int kTensor, typename T>
  __device__ __forceinline__ void fetch(uint32_t to, const T* row, int first, int dim) const {
    if constexpr (sizeof(T) == 2) {
      if (first < dim) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + kTensor * kPieces * piece), "l"(row + first) : "memory");
    } else {
      const int lane = threadIdx.x & 31;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = i * 32 + lane, col = first - lane * kEach + c * 4;
        const uint32_t at_ = to + (uint32_t)(((c >> 1) - lane) * 16) + (kTensor * kPieces + (c & 1)) * piece;
        if (col < dim) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at_), "l"(row + col) : "memory");
      }
    }
  }
  __device__ __forceinline__ void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
  __device__ __forceinline__ void wait() const {            // the oldest row is there
    if (stages == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
  }
  template <int kTensor, typename T>
  __device__ __forceinline__ void take(const T*, Eight& f) const {
    uint32_t u[4], v[4];
    const uint32_t from = at + kTensor * kPieces * piece;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(from) : "memory");
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(u[i] << 16), f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    } else {
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(from + piece) : "memory");
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(u[i]), f[4 + i] = __uint_as_float(v[i]);
    }
  }
  __device__ __forceinline__ void advance() {
    at += stage_bytes;
    if (--left == 0) left = stages, at = mine;
  }
};

__device__ __forceinline__ void clear8(float (&f)[kEach]) {
#pragma unroll
  for (int i = 0; i < kEach; ++i) f[i] = 0.f;
}

__device__ __forceinline__ bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
__device__ __forceinline__ bool on32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }

// Mean (layer norm) and reciprocal deviation of a row; f is what the norm makes of it on return (rubbish in columns that are not there).
template <bool kLayer, bool kVec, int kMax>
__device__ __forceinline__ float2 normalise(Eight& f, const Columns<kVec>& c, const BranchArgs& p, RowSum<kMax>& sum) {
  float m = 0.f;
  if constexpr (kLayer) {
    m = sum.one(sum8(f)) * p.inv_dim;   // (0 where there is no column)
    add8(f, f, -m);
    if (!kVec) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) f[i] = c.there(i) ? f[i] : 0.f;
    }
  }
  float q = dot8(f, f);
  if (kLayer && kVec) q = c.there(0) ? q : 0.f;
  const float r = rsqrtf(fmaf(sum.one(q), p.inv_dim, p.eps));   // (off by 2^-22 at most)
  mul8(f, f, r);
  return make_float2(m, r);
}

constexpr int ctas_of(int most, int small) { return most == 256 ? small : 1; }

// A thread's columns of a parameter: in registers from row to row (kHeld), or read again for each (from L1; rows of 1024 threads,
// which have 64 registers each)
template <bool kVec, bool kHeld>
struct Param {
  const float* p;
  float none;
  float v[kHeld ? kEach : 1];
  __device__ __forceinline__ Param(const float* q, float n, const Columns<kVec>& c) : p(q), none(n) {
    if constexpr (kHeld) c.param(q, v, n, on32(q));
  }
  __device__ __forceinline__ void get(float (&f)[kEach], const Columns<kVec>& c) const {
    if constexpr (kHeld) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) f[i] = v[i];
    } else {
      c.param(p, f, none, on32(p));
    }
  }
};

// The branch's factor and offset: drop(f W + B) with W = b gate w_a, B = b gate b_a in a row of the gate
template <bool kVec>
__device__ __forceinline__ void branch_factor(float (&w)[kEach], const float* a, float none, float scale, const float* gate, const Columns<kVec>& c) {
  c.param(a, w, none, on32(a));
  float g[kEach];
  c.param(gate, g, 1.f, on32(gate));
#pragma unroll
  for (int i = 0; i < kEach; ++i) w[i] *= scale * g[i];
}

template <typename TI, typename TR, bool kVec, bool kLayer, int kMax>
__global__ void __launch_bounds__(kMax, ctas_of(kMax, 3)) k_branch_forward(const __grid_constant__ BranchArgs p) {
  extern __shared__ __align__(16) uint8_t ring_smem[];
  __shared__ __align__(16) float sh[6 * kMax / 32];
  constexpr bool kHeld = kMax <= 512;
  pdl_wait();
  pdl_launch_dependents();
  RowSum<kMax> sum(sh);
  const Columns<kVec> c(p.dim);
  const int worker = blockIdx.x;
  const int64_t t0 = worker * p.run, t1 = t0 + p.run < p.rows ? t0 + p.run : p.rows;
  const uint32_t step = p.drop.below ? step_of(p.drop) : 0;
  Ring<2, sizeof(TR) / 2> ring(ring_smem, p.stages);
  const bool mine = c.there(0), res = p.h != nullptr, groups = p.gate && p.per < p.rows;
  const TI* y = static_cast<const TI*>(p.y);
  const TR* h_in = static_cast<const TR*>(p.h);
  const int rows = t1 > t0 ? (int)(t1 - t0) : 0;           // (of this worker)
  int64_t ahead = t0 * p.dim;                              // the row to be fetched next
  int fetched = 0;
  auto fetch = [&](uint32_t to) {
    if (fetched++ < rows) {
      ring.template fetch<0>(to, y + ahead, c.first, p.dim);
      if (res) ring.template fetch<1>(to, h_in + ahead, c.first, p.dim);
    }
    ahead += p.dim;
    ring.commit();
  };
  if (kVec) {
    if (!mine || !res) ring.clear();
    __syncwarp();
    for (int i = 0; i < p.stages; ++i) fetch(ring.mine + i * ring.stage_bytes);
  }
  int64_t next_group = groups ? t0 : INT64_MAX;            // row from which on another of the gate's rows holds
  const float* gate = p.gate;
  float w[kEach], b[kEach];
  if (kHeld && !groups) {
    branch_factor(w, p.aw, 1.f, p.bs, gate, c);
    if (kLayer) branch_factor(b, p.ab, 0.f, p.bs, gate, c);
  }
  const Param<kVec, kHeld> nw(p.nw, 1.f, c), nb(kLayer ? p.nb : nullptr, 0.f, c);
  int64_t at = t0 * p.dim;
#pragma unroll 1
  for (int k = 0; k < rows; ++k, at += p.dim) {
    const int64_t t = t0 + k;
    float f[kEach], h[kEach], x[kEach];
    if constexpr (kVec) {
      ring.wait();
      ring.template take<0>(y, f);
      ring.template take<1>(h_in, h);
      __syncwarp();
      fetch(ring.at);
      ring.advance();
    } else {
      c.load(y + at, f);
      c.load(h_in + at, h, res);
    }
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p.norm_after) {
      const float2 s = normalise<kLayer>(f, c, p, sum);
      st.x = s.x, st.y = s.y;
    }
    if (!kHeld || t >= next_group) {
      if (groups && t >= next_group) {
        const int64_t group = t / p.per;
        gate = p.gate + group * p.dim;
        next_group = (group + 1) * p.per;
      }
      branch_factor(w, p.aw, 1.f, p.bs, gate, c);
      if (kLayer) branch_factor(b, p.ab, 0.f, p.bs, gate, c);
    }
    if (kLayer) fma8(f, f, w, b);
    else mul8(f, f, w);
    if (p.drop.below) c.drop(p.drop, c.kept_bits(p.drop, step, t), f);
    fma8(f, h, p.rs, f);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      f[i] = stored<TR>(f[i]);
      if (!kVec) f[i] = c.there(i) ? f[i] : 0.f;
    }
    c.store(static_cast<TR*>(p.h_out) + at, f);
    if (p.x) {
      const float2 s = normalise<kLayer>(f, c, p, sum);
      st.z = s.x, st.w = s.y;
      nw.get(x, c);
      if (kLayer) {
        nb.get(h, c);
        fma8(f, f, x, h);
      } else {
        mul8(f, f, x);
      }
      c.store(static_cast<TI*>(p.x) + at, f);
    }
    if (threadIdx.x == 0) {
      float* s = p.stats + 4 * t;
      if (on16(s)) *reinterpret_cast<float4*>(s) = st;
      else s[0] = st.x, s[1] = st.y, s[2] = st.z, s[3] = st.w;
    }
  }
}

// dgate of a gate's row from its sums
template <bool kVec>
__device__ __forceinline__ void put_gate(const BranchArgs& p, const Columns<kVec>& c, int64_t s, const float (&s1)[kEach], const float (&s0)[kEach]) {
  float w[kEach], b[kEach];
  c.param(p.aw, w, 1.f, on32(p.aw));
  c.param(p.ab, b, 0.f, on32(p.ab));
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (c.there(i)) {
      float* g = p.dgate + s * p.dim + c.at(i);
      const float v = fmaf(w[i], s1[i], b[i] * s0[i]);
      *g = p.accumulate ? *g + v : v;
    }
}

// kGroups: the gate has several rows
template <typename TI, typename TR, bool kVec, bool kLayer, bool kGroups, int kMax>
__global__ void __launch_bounds__(kMax, ctas_of(kMax, 2)) k_branch_backward(const __grid_constant__ BranchArgs p) {
  extern __shared__ __align__(16) uint8_t ring_smem[];
  __shared__ __align__(16) float sh[6 * kMax / 32];
  constexpr bool kHeld = kMax <= 512;
  pdl_wait();
  pdl_launch_dependents();
  RowSum<kMax> sum(sh);
  const Columns<kVec> c(p.dim);
  const int worker = blockIdx.x;
  const int64_t t0 = worker * p.run, t1 = t0 + p.run < p.rows ? t0 + p.run : p.rows;
  const uint32_t step = p.drop.below ? step_of(p.drop) : 0;
  Ring<4, sizeof(TR) / 2> ring(ring_smem, p.stages);
  const bool mine = c.there(0), next = p.dx != nullptr, more = p.dh_out != nullptr;
  const TI *dx = static_cast<const TI*>(p.dx), *y = static_cast<const TI*>(p.y);
  const TR *h_out = static_cast<const TR*>(p.h_out), *dh_out = static_cast<const TR*>(p.dh_out);
  const int rows = t1 > t0 ? (int)(t1 - t0) : 0;           // (of this worker)
  int64_t ahead = t0 * p.dim;                              // the row to be fetched next
  int fetched = 0;
  auto fetch = [&](uint32_t to) {
    if (fetched++ < rows) {
      if (next) {
        ring.template fetch<0>(to, dx + ahead, c.first, p.dim);
        ring.template fetch<1>(to, h_out + ahead, c.first, p.dim);
      }
      if (more) ring.template fetch<2>(to, dh_out + ahead, c.first, p.dim);
      ring.template fetch<3>(to, y + ahead, c.first, p.dim);
    }
    ahead += p.dim;
    ring.commit();
  };
  if (kVec) {
    if (!mine || !next || !more) ring.clear();
    __syncwarp();
    for (int i = 0; i < p.stages; ++i) fetch(ring.mine + i * ring.stage_bytes);
  }
  float s1[kEach] = {}, s0[kEach] = {}, n1[kEach] = {}, n0[kEach] = {};
  bool again = false;                                      // (kGroups) the sums over all of the gate's rows have been begun
  const int64_t first = kGroups ? t0 / p.per : 0;
  int64_t group = first, next_group = kGroups ? (first + 1) * p.per : INT64_MAX;
  const float* gate = p.gate ? p.gate + (kGroups && t0 < p.rows ? group * p.dim : 0) : nullptr;
  float w[kEach];                                          // b gate w_a
  if (kHeld) branch_factor(w, p.aw, 1.f, p.bs, gate, c);
  const Param<kVec, kHeld> nw(p.nw, 1.f, c);
  auto stats_of = [&](int64_t t) {
    const float* q = p.stats + 4 * t;
    return on16(q) ? *reinterpret_cast<const float4*>(q) : make_float4(q[0], q[1], q[2], q[3]);
  };
  float4 ahead_st = stats_of(t0);                          // (t0 < rows: there are no more workers than rows)
  auto part = [&](int which) { return p.part + ((int64_t)which * p.workers + worker) * p.dim; };
  // the sums over the worker's rows of one of the gate's
  auto flush = [&](bool whole) {
    mul8(s1, s1, p.bs);
    if (kLayer && p.zero_sums) mul8(s0, s0, p.bs);
    float g[kEach];
    c.param(gate, g, 1.f, on32(gate));
    if (p.dgate) {
      if (whole) {
        put_gate(p, c, group, s1, s0);
      } else {
        float *q1 = part(group == first ? kHead1 : kTail1), *q0 = part(group == first ? kHead0 : kTail0);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
          if (c.there(i)) {
            q1[c.at(i)] = s1[i];
            if (kLayer && p.zero_sums) q0[c.at(i)] = s0[i];
          }
      }
    }
    // gate S1 and gate S0 add up in the worker's own partial sums (rarely: registers for them would cost every row)
    auto add = [&](int which, Eight& v) {
      Eight sum;
      clear8(sum);
      if (again) c.load(part(which), sum);
      fma8(sum, g, v, sum);
      c.store(part(which), sum);
    };
    if (p.daw) add(kAfter1, s1);
    if (kLayer && p.dab) add(kAfter0, s0);
    again = true;
    clear8(s1);
    if (kLayer) clear8(s0);
  };
  int64_t at = t0 * p.dim;
#pragma unroll 1
  for (int k = 0; k < rows; ++k, at += p.dim) {
    const int64_t t = t0 + k;
    float d[kEach], f[kEach];
    const float4 st = ahead_st;
    if (k + 1 < rows) ahead_st = stats_of(t + 1);          // (waited for here it cost a fifth of a row's time)
    const uint32_t bits = p.drop.below ? c.kept_bits(p.drop, step, t) : 0u;
    float x[kEach], y_[kEach];
    if constexpr (kVec) {
      ring.wait();
      ring.template take<0>(dx, x);
      ring.template take<1>(h_out, f);
      ring.template take<2>(dh_out, d);
      ring.template take<3>(y, y_);
      __syncwarp();
      fetch(ring.at);
      ring.advance();
    } else {
      c.load(dh_out + at, d, more);
      c.load(dx + at, x, next);
      c.load(h_out + at, f, next);
      c.load(y + at, y_);
    }
    if (kGroups && t >= next_group) {
      flush(group != first || first * p.per >= t0);
      group = t / p.per;
      next_group = (group + 1) * p.per;
      gate = p.gate + group * p.dim;
      if (kHeld) branch_factor(w, p.aw, 1.f, p.bs, gate, c);
    }
    if (!kHeld) branch_factor(w, p.aw, 1.f, p.bs, gate, c);
    float v[kEach];
    nw.get(v, c);
    if (p.norm_after) {                                    // y^
      if (kLayer) fma8(y_, y_, st.y, -st.x * st.y);
      else mul8(y_, y_, st.y);
    }
    // (x and w are 0 where there is no column, and so are their products)
    if (kLayer) fma8(f, f, st.w, -st.z * st.w);            // h^
    else mul8(f, f, st.w);
    fma8(n1, x, f, n1);
    if (kLayer) add8(n0, n0, x);
    mul8(x, x, v);                                         // a
    float m1 = 0.f;                                        // mean(v y^)
    if constexpr (!kLayer) {
      // All sums of a row at once: with e = d' + s_n a and q = b keep gate w_a y^ the second mean is that of q e - s_n mean(a h^) q h^, so that a
      // row meets one barrier instead of two (4096 x 2048 bf16: 28.5 us instead of 29.2)
      float sums[3] = {dot8(x, f), 0.f, 0.f};
      fma8(d, x, st.w, d);                                 // e
      if (p.norm_after) {
        mul8(x, y_, w);
        if (p.drop.below) c.drop(p.drop, bits, x);
        sums[1] = dot8(x, d), sums[2] = dot8(x, f);
      }
      sum.get(sums);
      const float m = -sums[0] * p.inv_dim * st.w;
      fma8(d, f, m, d);
      m1 = fmaf(m, sums[2], sums[1]) * p.inv_dim;
    } else if (next) {
      float sums[2] = {dot8(x, f), sum8(x)};
      sum.get(sums);
      // d' + s (a - m0 - h^ m1)
      fma8(x, f, -sums[0] * p.inv_dim, x);
      add8(x, x, -sums[1] * p.inv_dim);
      fma8(d, x, st.w, d);
    }
    if (p.dh) {
      mul8(x, d, p.rs);
      c.store(static_cast<TR*>(p.dh) + at, x);
    }
    if (p.drop.below) c.drop(p.drop, bits, d);             // u / b
    fma8(s1, d, y_, s1);
    if (kLayer && p.zero_sums) add8(s0, s0, d);
    mul8(d, d, w);                                         // v
    if (p.norm_after) {
      if constexpr (kLayer) {
        float sums[2] = {dot8(d, y_), sum8(d)};
        sum.get(sums);
        m1 = sums[0] * p.inv_dim;
        add8(d, d, -sums[1] * p.inv_dim);
      }
      fma8(d, y_, -m1, d);
      mul8(d, d, st.y);
    }
    c.store(static_cast<TI*>(p.dy) + at, d);
  }
  if (t0 >= p.rows) return;
  if (kGroups) {
    const int64_t end = (group + 1) * p.per < p.rows ? (group + 1) * p.per : p.rows;
    flush((group != first || first * p.per >= t0) && end <= t1);
  }
  if (!p.part) return;
  auto keep = [&](int which, const float (&v)[kEach]) { c.store(part(which), v); };
  if (!kGroups) {
    mul8(s1, s1, p.bs);
    if (kLayer && p.zero_sums) mul8(s0, s0, p.bs);
  }
  if (!kGroups && (p.dgate || p.daw)) keep(kHead1, s1);
  if (!kGroups && kLayer && p.zero_sums) keep(kHead0, s0);
  if (p.dnw) keep(kNext1, n1);
  if (kLayer && p.dnb) keep(kNext0, n0);
}

// The workers' sums joined in order: 32 columns a cluster of up to eight CTAs, eight shares of the workers side by side in each, joined in
// shared memory and then across the cluster (one CTA with 44 of 701 workers a thread took 15 us, loads waiting for one another).
// blockIdx.y 0: of the next norm, 1: of the norm after and of a gate of one row; 2 ..: rows of a gate that workers share
constexpr int kSlices = 8, kSumCtas = 8;
struct SumsArgs {
  BranchArgs b;
  int layer, groups;
  int each;                // warps that share a row of the gate
};
__global__ void __launch_bounds__(32 * kSlices) k_branch_sums(const __grid_constant__ SumsArgs a) {
  __shared__ float sh[2][kSlices][33];
  __shared__ float2 joined[32];
  namespace cg = cooperative_groups;
  const BranchArgs& p = a.b;
  pdl_wait();
  pdl_launch_dependents();
  cg::cluster_group cluster = cg::this_cluster();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, rank = (int)cluster.block_rank(), ctas = (int)gridDim.z;
  // of partial sums `one` and `two` (or none) over the workers; for the first warp of the first CTA
  auto total = [&](int one, int two) {
    const int64_t share = (p.workers + ctas - 1) / ctas, w0 = rank * share, w1 = w0 + share < p.workers ? w0 + share : p.workers;
    float x = 0.f, y = 0.f;
    if (col < p.dim)
#pragma unroll 8
      for (int64_t w = w0 + slice; w < w1; w += kSlices) {
        x += p.part[((int64_t)one * p.workers + w) * p.dim + col];
        if (two >= 0) y += p.part[((int64_t)two * p.workers + w) * p.dim + col];
      }
    sh[0][slice][lane] = x, sh[1][slice][lane] = y;
    __syncthreads();
    if (slice == 0) {
      float2 r = make_float2(0.f, 0.f);
      for (int i = 0; i < kSlices; ++i) r.x += sh[0][i][lane], r.y += sh[1][i][lane];
      joined[lane] = r;
    }
    cluster.sync();
    float2 r = make_float2(0.f, 0.f);
    if (rank == 0 && slice == 0)
      for (int i = 0; i < ctas; ++i) {
        const float2 v = cluster.map_shared_rank(joined, i)[lane];
        r.x += v.x, r.y += v.y;
      }
    cluster.sync();                                       // (all have been read)
    return r;
  };
  auto write = [&](float* out, float v) {
    if (out && rank == 0 && slice == 0 && col < p.dim) out[col] = p.accumulate ? out[col] + v : v;
  };
  if (blockIdx.y == 0) {
    if (!p.dnw && !p.dnb) return;
    const bool one = p.dnw != nullptr, two = p.dnb && a.layer;
    const float2 r = total(one ? kNext1 : kNext0, one && two ? kNext0 : -1);
    if (one) write(p.dnw, r.x);
    if (two) write(p.dnb, one ? r.y : r.x);
  } else if (blockIdx.y == 1) {
    if (a.groups) {
      if (p.daw) write(p.daw, total(kAfter1, -1).x);
      if (p.dab) write(p.dab, total(kAfter0, -1).x);
      return;
    }
    if (!p.dgate && !p.daw && !p.dab) return;
    const bool one = p.dgate || p.daw, two = p.zero_sums != 0;
    float2 r = total(one ? kHead1 : kHead0, one && two ? kHead0 : -1);
    if (!one) r.y = r.x;
    if (rank || slice || col >= p.dim) return;
    const float w = p.aw ? p.aw[col] : 1.f, b = p.ab ? p.ab[col] : 0.f, g = p.gate ? p.gate[col] : 1.f;
    write(p.dgate, fmaf(w, r.x, b * r.y));
    write(p.daw, g * r.x);
    write(p.dab, g * r.y);
  } else {
    // `each` warps a row of the gate
    const int sub = slice % a.each, rows = kSlices / a.each;
    for (int64_t s0 = ((int64_t)(blockIdx.y - 2) * ctas + rank) * rows; s0 * p.per < p.rows; s0 += (int64_t)(gridDim.y - 2) * ctas * rows) {
      const int64_t s = s0 + slice / a.each;
      float x = 0.f, y = 0.f;
      bool shared = false;
      if (s * p.per < p.rows) {
        const int64_t end = (s + 1) * p.per < p.rows ? (s + 1) * p.per : p.rows, w0 = s * p.per / p.run, w1 = (end - 1) / p.run;
        shared = w0 != w1;                                // (else its worker wrote it)
        const bool head = w0 * p.run / p.per == s;        // the first worker's first row is the gate row's too
        if (shared && col < p.dim)
#pragma unroll 8
          for (int64_t w = w0 + sub; w <= w1; w += a.each) {
            const bool tail = w == w0 && !head;
            x += p.part[((int64_t)(tail ? kTail1 : kHead1) * p.workers + w) * p.dim + col];
            if (p.zero_sums) y += p.part[((int64_t)(tail ? kTail0 : kHead0) * p.workers + w) * p.dim + col];
          }
      }
      __syncthreads();
      sh[0][slice][lane] = x, sh[1][slice][lane] = y;
      __syncthreads();
      if (sub == 0 && shared && col < p.dim) {
        x = y = 0.f;
        for (int i = 0; i < a.each; ++i) x += sh[0][slice + i][lane], y += sh[1][slice + i][lane];
        float* g = p.dgate + s * p.dim + col;
        const float v = fmaf(p.aw ? p.aw[col] : 1.f, x, (p.ab ? p.ab[col] : 0.f) * y);
        *g = p.accumulate ? *g + v : v;
      }
    }
  }
}

// ---- host side -----------------------------------------------------------------------------------------

size_t size_of(int dtype) { return dtype == ASI_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool make_drop(const asi_dropout_t& d, Drop* out) {
  if (!(d.p >= 0.0 && d.p < 1.0) || d.step < 0 || off_element(d.step_dev, 8)) return false;
  const double k = std::floor(d.p * 65536.0 + 0.5);
  if (k >= 65536.0) return false;
  out->seed = d.seed;
  out->step_dev = d.step_dev;
  out->stream = d.stream_id;
  out->step = (uint32_t)d.step;
  out->below = (uint32_t)k;
  out->more = (float)(65536.0 / (65536.0 - k));
  return true;
}

// A contiguous buffer of a call; null where the call has none
struct Span {
  const void* p;
  size_t bytes, element;
  const void* same = nullptr;   // the buffer that it may be
  bool meets(const Span& o) const {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
    return p && o.p && a < b + o.bytes && b < a + bytes;
  }
};

// every buffer on an element, what is written apart from what else there is (but for the buffer that it may be, from its start)
bool fine(std::initializer_list<Span> in, std::initializer_list<Span> out) {
  for (const auto* list : {&in, &out})
    for (const Span& s : *list)
      if (s.p && off_element(s.p, s.element)) return false;
  for (const Span* o = out.begin(); o != out.end(); ++o) {
    for (const Span* q = out.begin(); q != o; ++q)
      if (o->meets(*q)) return false;
    for (const Span& i : in)
      if (o->meets(i) && !(o->p == i.p && o->same == i.p && o->bytes == i.bytes)) return false;
  }
  return true;
}

asi_status_t check_desc(const asi_branch_desc_t* d, Drop* drop) {
  if (!d || (d->in_dtype != ASI_F32 && d->in_dtype != ASI_BF16) || (d->res_dtype != ASI_F32 && d->res_dtype != d->in_dtype)) return ASI_ERR_INVALID_ARG;
  if ((d->norm != ASI_NORM_RMS && d->norm != ASI_NORM_LAYER) || d->rows < 0 || d->dim < 1 || d->rows_per_gate < 0) return ASI_ERR_INVALID_ARG;
  if (!(d->eps >= 1e-30f) || !std::isfinite(d->eps) || !std::isfinite(d->res_scale) || !std::isfinite(d->branch_scale)) return ASI_ERR_INVALID_ARG;
  if (!make_drop(d->drop, drop)) return ASI_ERR_INVALID_ARG;
  if (d->rows > ASI_BRANCH_MAX_ROWS || d->dim > ASI_BRANCH_MAX_DIM) return ASI_ERR_UNSUPPORTED;
  return ASI_OK;
}

// A CTA a row at a time: its threads
int threads_of(int64_t dim) { return (int)align_up((size_t)ceil_div(dim, kEach), 32); }
// Rows of a worker (a CTA) and workers: as many as registers leave room for, `threads` an SM
struct Work {
  int64_t run;
  int workers;
};
constexpr int kForwardThreads = 768, kBackwardThreads = 512;
int ctas_of_sm(int64_t dim, int threads) { return std::min(24, std::max(1, threads / threads_of(dim))); }
Work work_of(int64_t rows, int64_t dim, int threads) {
  const int64_t run = std::max<int64_t>(1, ceil_div(rows, 148 * ctas_of_sm(dim, threads)));
  return {run, (int)std::max<int64_t>(1, ceil_div(rows, run))};
}
size_t part_bytes(int64_t rows, int64_t dim) {
  return align_up((size_t)kParts * std::max<int64_t>(1, std::min<int64_t>(rows, 148 * ctas_of_sm(dim, kBackwardThreads))) * dim * 4, 256);
}
// shared memory of the rows on their way: as many stages as a CTA's share of 200 KB holds
size_t stages_of(BranchArgs* a, bool vec, int tensors, int pieces, int threads) {
  const size_t each = (size_t)tensors * pieces * 16 * threads_of(a->dim), room = (200 << 10) / ctas_of_sm(a->dim, threads);
  a->stages = vec ? (int)std::max<size_t>(1, std::min<size_t>(kMaxStages, room / each)) : 0;
  return a->stages * each;
}

BranchArgs args_of(const asi_branch_desc_t* d, const asi_branch_t* t, const Drop& drop) {
  BranchArgs a = {};
  a.y = t->y, a.gate = d->rows_per_gate ? t->gate : nullptr;
  a.aw = t->after_weight, a.ab = t->after_bias, a.nw = t->next_weight, a.nb = t->next_bias;
  a.stats = t->stats;
  a.rows = d->rows, a.per = d->rows_per_gate, a.dim = (int)d->dim, a.norm_after = d->norm_after != 0;
  a.eps = d->eps, a.rs = d->res_scale, a.bs = d->branch_scale, a.inv_dim = 1.f / (float)d->dim;
  a.drop = drop;
  return a;
}

template <typename... P>
cudaError_t launch_ring(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const BranchArgs& a) {
  if (smem > 40 << 10) {
    const cudaError_t e = opt_in_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kernel, grid, block, smem, st, a);
}

template <typename TI, typename TR, bool kVec, int kMax>
cudaError_t launch_forward_as(BranchArgs& a, bool layer, cudaStream_t st) {
  const Work k = work_of(a.rows, a.dim, kForwardThreads);
  a.run = k.run;
  a.workers = k.workers;
  const size_t smem = stages_of(&a, kVec, 2, sizeof(TR) == 4 ? 2 : 1, kForwardThreads);
  const dim3 grid((unsigned)k.workers), block(threads_of(a.dim));
  return layer ? launch_ring(k_branch_forward<TI, TR, kVec, true, kMax>, grid, block, smem, st, a) : launch_ring(k_branch_forward<TI, TR, kVec, false, kMax>, grid, block, smem, st, a);
}
template <typename TI, typename TR, bool kVec>
cudaError_t launch_forward(BranchArgs& a, bool layer, cudaStream_t st) {
  const int tpr = threads_of(a.dim);
  if (tpr <= 256) return launch_forward_as<TI, TR, kVec, 256>(a, layer, st);
  return tpr <= 512 ? launch_forward_as<TI, TR, kVec, 512>(a, layer, st) : launch_forward_as<TI, TR, kVec, 1024>(a, layer, st);
}

template <typename TI, typename TR, bool kVec, int kMax>
cudaError_t launch_backward_as(BranchArgs& a, bool layer, cudaStream_t st) {
  const Work k = work_of(a.rows, a.dim, kBackwardThreads);
  a.run = k.run;
  a.workers = k.workers;
  const bool groups = a.gate && a.per < a.rows;
  const size_t smem = stages_of(&a, kVec, 4, sizeof(TR) == 4 ? 2 : 1, kBackwardThreads);
  const dim3 grid((unsigned)k.workers), block(threads_of(a.dim));
  cudaError_t e;
  if (layer) e = groups ? launch_ring(k_branch_backward<TI, TR, kVec, true, true, kMax>, grid, block, smem, st, a) : launch_ring(k_branch_backward<TI, TR, kVec, true, false, kMax>, grid, block, smem, st, a);
  else e = groups ? launch_ring(k_branch_backward<TI, TR, kVec, false, true, kMax>, grid, block, smem, st, a) : launch_ring(k_branch_backward<TI, TR, kVec, false, false, kMax>, grid, block, smem, st, a);
  if (e != cudaSuccess || !a.part) return e;
  SumsArgs q = {a, layer, groups, 1};
  while (q.each < kSlices && q.each * 8 * a.run < a.per) q.each *= 2;      // (about eight workers a warp)
  const int64_t shared = groups && a.dgate && a.per > 1 ? std::min<int64_t>(ceil_div(ceil_div(a.rows, a.per), kSumCtas * kSlices / q.each), 1024) : 0;
  // CTAs of a cluster: as many as stay well within a wave (4096 x 2048, 293 workers: 29.0 us for the whole gradient with four, 32.7 with eight;
  // 6304 x 768, 701 workers: 36.6 and 33.7)
  const int64_t columns = ceil_div(a.dim, 32);
  int ctas = kSumCtas;
  while (ctas > 1 && columns * (2 + shared) * ctas > 800) ctas /= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)columns, (unsigned)(2 + shared), (unsigned)ctas);
  cfg.blockDim = dim3(32 * kSlices);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = (unsigned)ctas;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_branch_sums, q);
}
template <typename TI, typename TR, bool kVec>
cudaError_t launch_backward(BranchArgs& a, bool layer, cudaStream_t st) {
  const int tpr = threads_of(a.dim);
  if (tpr <= 256) return launch_backward_as<TI, TR, kVec, 256>(a, layer, st);
  return tpr <= 512 ? launch_backward_as<TI, TR, kVec, 512>(a, layer, st) : launch_backward_as<TI, TR, kVec, 1024>(a, layer, st);
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" {

asi_status_t asi_dropout(const asi_dropout_t* drop, int32_t dtype, int64_t n, const void* x, const void* residual, void* out, void* stream) {
  DropoutArgs a = {};
  if (!drop || (dtype != ASI_F32 && dtype != ASI_BF16) || n < 0 || !make_drop(*drop, &a.drop)) return ASI_ERR_INVALID_ARG;
  if (n > (int64_t)1 << 40) return ASI_ERR_UNSUPPORTED;
  if (n == 0) return ASI_OK;
  const size_t e = size_of(dtype), bytes = (size_t)n * e;
  if (!x || !out) return ASI_ERR_INVALID_ARG;
  if (!fine({{x, bytes, e}, {residual == x ? nullptr : residual, bytes, e}, {drop->step_dev, 8, 8}}, {{out, bytes, e, residual && out == residual ? residual : x}}))
    return ASI_ERR_INVALID_ARG;
  a.x = x, a.res = residual, a.out = out, a.n = n;
  const bool vec = aligned(x, 8 * e) && aligned(out, 8 * e) && (!residual || aligned(residual, 8 * e));
  const dim3 grid((unsigned)ceil_div(ceil_div(n, kEach), kDropThreads)), block(kDropThreads);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t r;
  if (dtype == ASI_BF16) r = vec ? launch_pdl(k_dropout<__nv_bfloat16, true>, grid, block, 0, st, a) : launch_pdl(k_dropout<__nv_bfloat16, false>, grid, block, 0, st, a);
  else r = vec ? launch_pdl(k_dropout<float, true>, grid, block, 0, st, a) : launch_pdl(k_dropout<float, false>, grid, block, 0, st, a);
  return cuda_status(r, "dropout");
}

asi_status_t asi_branch_forward(const asi_branch_desc_t* desc, const asi_branch_t* t, void* stream) try {
  Drop drop = {};
  const asi_status_t s = check_desc(desc, &drop);
  if (s != ASI_OK) return s;
  if (!t) return ASI_ERR_INVALID_ARG;
  if (desc->rows == 0) return ASI_OK;
  if (!t->y || !t->h_out || !t->stats || (desc->rows_per_gate && !t->gate) || (!desc->norm_after && (t->after_weight || t->after_bias)) || (desc->norm == ASI_NORM_RMS && (t->after_bias || t->next_bias))) return ASI_ERR_INVALID_ARG;
  const size_t ei = size_of(desc->in_dtype), er = size_of(desc->res_dtype), n = (size_t)desc->rows * desc->dim, w = (size_t)desc->dim * 4;
  const size_t gates = desc->rows_per_gate ? (size_t)((desc->rows - 1) / desc->rows_per_gate + 1) * w : 0;   // (rows > 0, any int64 of them a gate)
  const float* gate = desc->rows_per_gate ? t->gate : nullptr;
  if (!fine({{t->y, n * ei, ei}, {t->h, n * er, er}, {gate, gates, 4}, {t->after_weight, w, 4}, {t->after_bias, w, 4}, {t->next_weight, w, 4},
             {t->next_bias, w, 4}, {desc->drop.step_dev, 8, 8}},
            {{t->h_out, n * er, er, t->h}, {t->x, n * ei, ei}, {t->stats, (size_t)desc->rows * 16, 4}}))
    return ASI_ERR_INVALID_ARG;
  BranchArgs a = args_of(desc, t, drop);
  a.h = t->h, a.h_out = t->h_out, a.x = t->x;
  const bool vec = desc->dim % kEach == 0 && aligned(a.y, 8 * ei) && aligned(a.h, 8 * er) && aligned(a.h_out, 8 * er) && aligned(a.x, 8 * ei);
  const bool layer = desc->norm == ASI_NORM_LAYER;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  using B = __nv_bfloat16;
  cudaError_t e;
  if (desc->in_dtype == ASI_F32) e = vec ? launch_forward<float, float, true>(a, layer, st) : launch_forward<float, float, false>(a, layer, st);
  else if (desc->res_dtype == ASI_F32) e = vec ? launch_forward<B, float, true>(a, layer, st) : launch_forward<B, float, false>(a, layer, st);
  else e = vec ? launch_forward<B, B, true>(a, layer, st) : launch_forward<B, B, false>(a, layer, st);
  return cuda_status(e, "branch and residual stream");
} catch (...) {
  return no_host_memory();
}

size_t asi_branch_backward_ws_bytes(const asi_branch_desc_t* desc) {
  Drop drop = {};
  return check_desc(desc, &drop) == ASI_OK ? part_bytes(desc->rows, desc->dim) : 0;
}

asi_status_t asi_branch_backward(const asi_branch_desc_t* desc, const asi_branch_t* t, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) try {
  Drop drop = {};
  const asi_status_t s = check_desc(desc, &drop);
  if (s != ASI_OK) return s;
  if (!t) return ASI_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const size_t ei = size_of(desc->in_dtype), er = size_of(desc->res_dtype), n = (size_t)desc->rows * desc->dim, w = (size_t)desc->dim * 4;
  const bool layer = desc->norm == ASI_NORM_LAYER;
  if ((t->dgate && !desc->rows_per_gate) || (!desc->norm_after && (t->dafter_weight || t->dafter_bias || t->after_weight || t->after_bias))) return ASI_ERR_INVALID_ARG;
  if (!layer && (t->after_bias || t->next_bias || t->dafter_bias || t->dnext_bias)) return ASI_ERR_INVALID_ARG;
  if (desc->rows == 0) {                                   // sums of nothing (a gate has no rows then)
    if (accumulate) return ASI_OK;
    for (float* p : {t->dafter_weight, t->dafter_bias, t->dnext_weight, t->dnext_bias}) {
      if (p && off_element(p, 4)) return ASI_ERR_INVALID_ARG;
      const cudaError_t e = p ? cudaMemsetAsync(p, 0, w, st) : cudaSuccess;
      if (e != cudaSuccess) return cuda_status(e, "sums of no rows");
    }
    return ASI_OK;
  }
  if (!t->y || !t->stats || !t->dy || (!t->dx && !t->dh_out) || (t->dx && !t->h_out) || (desc->rows_per_gate && !t->gate)) return ASI_ERR_INVALID_ARG;
  if (!t->dx && (t->dnext_weight || t->dnext_bias)) return ASI_ERR_INVALID_ARG;
  const size_t gates = desc->rows_per_gate ? (size_t)((desc->rows - 1) / desc->rows_per_gate + 1) * w : 0;   // (rows > 0, any int64 of them a gate)
  const float* gate = desc->rows_per_gate ? t->gate : nullptr;
  const size_t need = part_bytes(desc->rows, desc->dim);
  const bool sums = t->dgate || t->dafter_weight || t->dafter_bias || t->dnext_weight || t->dnext_bias;
  if (!ws) return ASI_ERR_INVALID_ARG;
  if (ws_bytes < need || !aligned(ws, 256)) return ASI_ERR_WORKSPACE;
  if (!fine({{t->y, n * ei, ei}, {t->dx ? t->h_out : nullptr, n * er, er}, {t->stats, (size_t)desc->rows * 16, 4}, {gate, gates, 4}, {t->after_weight, w, 4},
             {t->after_bias, w, 4}, {t->dx ? t->next_weight : nullptr, w, 4}, {t->dx, n * ei, ei}, {t->dh_out, n * er, er}, {desc->drop.step_dev, 8, 8}},
            {{t->dy, n * ei, ei, t->dx}, {t->dh, n * er, er, t->dh_out}, {t->dgate, gates, 4}, {t->dafter_weight, w, 4}, {t->dafter_bias, w, 4},
             {t->dnext_weight, w, 4}, {t->dnext_bias, w, 4}, {ws, need, 256}}))
    return ASI_ERR_INVALID_ARG;
  BranchArgs a = args_of(desc, t, drop);
  a.h_out = t->h_out;
  a.dx = t->dx, a.dh_out = t->dh_out, a.dy = t->dy, a.dh = t->dh;
  a.dgate = t->dgate, a.daw = t->dafter_weight, a.dab = t->dafter_bias, a.dnw = t->dnext_weight, a.dnb = t->dnext_bias;
  a.accumulate = accumulate != 0;
  a.zero_sums = a.dab || (a.dgate && a.ab);
  a.part = sums ? static_cast<float*>(ws) : nullptr;
  const bool vec = desc->dim % kEach == 0 && aligned(a.y, 8 * ei) && aligned(t->dx ? a.h_out : nullptr, 8 * er) && aligned(a.dx, 8 * ei) && aligned(a.dh_out, 8 * er) &&
                   aligned(a.dy, 8 * ei) && aligned(a.dh, 8 * er);
  using B = __nv_bfloat16;
  cudaError_t e;
  if (desc->in_dtype == ASI_F32) e = vec ? launch_backward<float, float, true>(a, layer, st) : launch_backward<float, float, false>(a, layer, st);
  else if (desc->res_dtype == ASI_F32) e = vec ? launch_backward<B, float, true>(a, layer, st) : launch_backward<B, float, false>(a, layer, st);
  else e = vec ? launch_backward<B, B, true>(a, layer, st) : launch_backward<B, B, false>(a, layer, st);
  return cuda_status(e, "gradient of branch and residual stream");
} catch (...) {
  return no_host_memory();
}

}  // extern "C"
