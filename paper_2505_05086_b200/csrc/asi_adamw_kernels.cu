// One AdamW step over many tensors, states in 32 or 8 bits.
//
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  w = (1 - lr wd) w - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// m and v are computed in separately rounded fp32 operations in the order written (no contraction that another build or a plain
// restatement would do otherwise); the square root and the reciprocal are the hardware's, off by a unit or two in the last place,
// and the root of a subnormal v is 0.
//
// What bounds it: weights and states read and written once, gradients read once (27 million weights: 125 us with fp32 states,
// the copy rate; 51 us with 8-bit states and bf16 weights, where issue slots are 77 % taken).  A warp takes blocks of 256 elements,
// eight a lane: with 8-bit states the block's largest magnitude is one warp reduction away and codes are quantised where
// they were computed.  The tensors of a call share a launch: a table of them travels with the kernel's arguments.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>
#include <vector>

#include "asi_internal.h"

namespace asi {

namespace {

constexpr int kAwThreads = 128;
constexpr int kAwWarps = kAwThreads / 32;
constexpr int kBlock = ASI_ADAMW_BLOCK;
constexpr int kLane = kBlock / 32;            // elements of a lane
constexpr int kSpan = 8;                     // blocks of a CTA

struct AwTensor {
  void* w;
  const void* g;
  void *m, *v;
  uint8_t *ms, *vs;
  __nv_bfloat16* copy;
  int64_t n;
};
struct AwHyper {
  float b1, b2, c1, c2;                       // betas and 1 - beta
  float decay, step, root, eps;               // 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  float lr, wd, log_b1, log_b2;               // for lr and t in device memory
  float one;                                  // a sum x 1 + y: the assembler contracts packed products and sums, but not this
  const float *lr_dev, *scale;
  const int64_t* step_dev;
};
// kCap tensors a launch: a few, or as many as the argument space (32 KB) takes
template <int kCap>
struct AwArgs {
  AwHyper h;
  AwTensor t[kCap];
  uint32_t first[kCap + 1];                   // first CTA of each tensor
  uint8_t wide[kCap];                         // every buffer starts on 16 bytes
  int count;
};

// two fp32 values as one operand of the packed instructions (each rounded as the scalar ones round)
typedef unsigned long long f2;
__device__ __forceinline__ f2 pair(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 both(f2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
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
__device__ __forceinline__ f2 twice(float a) { return pair(a, a); }
__device__ __forceinline__ float root_approx(float v) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float inverse_approx(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// Eight consecutive values of a lane as they lie in memory.  `whole`: all eight are there, 16-byte aligned (8 for codes);
// else `left` of them, one by one, the others 0.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  uint4 a, b;
  __device__ __forceinline__ void load(const void* from, int64_t at, int64_t left, bool whole) {
    const float* p = static_cast<const float*>(from) + at;
    if (whole) {
      a = *reinterpret_cast<const uint4*>(p);
      b = *reinterpret_cast<const uint4*>(p + 4);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = i < left ? __float_as_uint(p[i]) : 0u;
      a = make_uint4(w[0], w[1], w[2], w[3]);
      b = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
  __device__ __forceinline__ void values(f2* f) const {
    f[0] = pair(__uint_as_float(a.x), __uint_as_float(a.y)), f[1] = pair(__uint_as_float(a.z), __uint_as_float(a.w));
    f[2] = pair(__uint_as_float(b.x), __uint_as_float(b.y)), f[3] = pair(__uint_as_float(b.z), __uint_as_float(b.w));
  }
};
template <>
struct Raw<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const void* from, int64_t at, int64_t left, bool whole) {
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(from) + at;
    if (whole) {
      a = *reinterpret_cast<const uint4*>(p);
    } else {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) w[i >> 1] |= (uint32_t)__bfloat16_as_ushort(p[i]) << (16 * (i & 1));
      a = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  __device__ __forceinline__ void values(f2* f) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
};
struct Codes {
  uint2 a;
  __device__ __forceinline__ void load(const void* from, int64_t at, int64_t left, bool whole) {
    const uint8_t* p = static_cast<const uint8_t*>(from) + at;
    if (whole) {
      a = *reinterpret_cast<const uint2*>(p);
    } else {
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
      a = make_uint2(w[0], w[1]);
    }
  }
  __device__ __forceinline__ void store(void* to, int64_t at, int64_t left, bool whole) const {
    uint8_t* p = static_cast<uint8_t*>(to) + at;
    if (whole) {
      *reinterpret_cast<uint2*>(p) = a;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = (uint8_t)((i < 4 ? a.x : a.y) >> (8 * (i & 3)));
    }
  }
  __device__ __forceinline__ void values(float scale, f2* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t two = (uint16_t)((i < 2 ? a.x : a.y) >> (16 * (i & 1)));
      const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3)));
      f[i] = mul2(pair(v.x, v.y), twice(scale));
    }
  }
};

__device__ __forceinline__ void store_values(float* base, int64_t at, int64_t left, bool whole, const f2* f) {
  float* p = base + at;
  const float2 v[4] = {both(f[0]), both(f[1]), both(f[2]), both(f[3])};
  if (whole) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = i & 1 ? v[i >> 1].y : v[i >> 1].x;
  }
}
__device__ __forceinline__ void store_values(__nv_bfloat16* base, int64_t at, int64_t left, bool whole, const f2* f) {
  __nv_bfloat16* p = base + at;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = both(f[i]);
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  if (whole) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = __ushort_as_bfloat16((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
  }
}

// 2^(byte - 127)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }

// The block's scale byte from the lanes' eight values each: the smallest 2^k with max <= 448 2^k = 1.75 2^(k + 8), over
// the finite values.  `finite` tells whether there are others than those (or NaN, which a maximum passes over).
__device__ __forceinline__ uint32_t block_scale(const f2* f, bool& finite) {
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = both(f[i]);
    most = fmaxf(fmaxf(most, fabsf(v.x)), fabsf(v.y));
  }
  uint32_t top = __reduce_max_sync(~0u, __float_as_uint(most));   // magnitudes order as their bits do
  finite = top < 0x7f800000u;
  if (!finite) {
    top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = both(f[i]);
      const uint32_t x = __float_as_uint(fabsf(v.x)), y = __float_as_uint(fabsf(v.y));
      top = max(top, max(x < 0x7f800000u ? x : 0u, y < 0x7f800000u ? y : 0u));
    }
    top = __reduce_max_sync(~0u, top);
  }
  if (top == 0) return 127;
  const int k = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
  return (uint32_t)(max(k, -126) + 127);
}

// kRoot: values above 0 whose code is 0 get the smallest code, 1
template <bool kRoot>
__device__ __forceinline__ Codes encode(const f2* f, uint32_t byte, bool finite) {
  const f2 inv = twice(__uint_as_float((254u - byte) << 23));      // 2^-k; byte is 1 .. 247
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = both(mul2(f[i], inv));
    uint32_t two = __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
    if (!finite) {                                                 // infinities (saturated above) are held as NaN
      if (isinf(v.x)) two |= 0x7fu;
      if (isinf(v.y)) two |= 0x7f00u;
    }
    w[i >> 1] |= two << (16 * (i & 1));
  }
  if (kRoot) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if ((w[h] - 0x01010101u) & 0x80808080u & ~w[h]) {            // a code of 0 among the four
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 v = both(f[2 * h + (i >> 1)]);
          if (!((w[h] >> (8 * i)) & 0xffu) && (i & 1 ? v.y : v.x) > 0.f) w[h] |= 1u << (8 * i);
        }
      }
  }
  Codes c;
  c.a = make_uint2(w[0], w[1]);
  return c;
}

template <typename TW, typename TG, bool BITS8>
struct Block {                              // eight values a lane of everything
  Raw<TW> w;
  Raw<TG> g;
  std::conditional_t<BITS8, Codes, Raw<float>> m, v;
  uint32_t ms, vs;
  __device__ __forceinline__ void load(const AwTensor& t, int64_t b, int64_t at, int64_t left, bool whole) {
    w.load(t.w, at, left, whole);
    g.load(t.g, at, left, whole);
    m.load(t.m, at, left, whole);
    v.load(t.v, at, left, whole);
    if (BITS8) ms = t.ms[b], vs = t.vs[b];
  }
};
struct Rates {
  float decay, step, root, gs;
  bool scaled;
};

template <typename TW, typename TG, bool BITS8>
__device__ __forceinline__ void step_block(const Block<TW, TG, BITS8>& in, const AwTensor& t, const AwHyper& h, const Rates& r,
                                           int64_t b, int64_t at, int64_t left, bool whole) {
  f2 w[4], g[4], m[4], v[4], root[4];
  in.w.values(w);
  in.g.values(g);
  if constexpr (BITS8) {
    in.m.values(scale_of(in.ms), m);
    in.v.values(scale_of(in.vs), v);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], v[i]);
  } else {
    in.m.values(m);
    in.v.values(v);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (r.scaled) g[i] = mul2(g[i], twice(r.gs));
    m[i] = fma2(mul2(m[i], twice(h.b1)), twice(h.one), mul2(g[i], twice(h.c1)));
    v[i] = fma2(mul2(v[i], twice(h.b2)), twice(h.one), mul2(mul2(g[i], g[i]), twice(h.c2)));
    const float2 x = both(v[i]);
    root[i] = pair(root_approx(x.x), root_approx(x.y));
    const float2 d = both(fma2(root[i], twice(r.root), twice(h.eps)));
    const f2 u = mul2(m[i], pair(inverse_approx(d.x), inverse_approx(d.y)));
    w[i] = fma2(u, twice(-r.step), mul2(w[i], twice(r.decay)));
  }
  store_values(static_cast<TW*>(t.w), at, left, whole, w);
  if (t.copy) store_values(t.copy, at, left, whole, w);
  if constexpr (BITS8) {
    bool fm, fv;
    const uint32_t sm = block_scale(m, fm), sv = block_scale(root, fv);
    encode<false>(m, sm, fm).store(t.m, at, left, whole);
    encode<true>(root, sv, fv).store(t.v, at, left, whole);
    if ((threadIdx.x & 31) == 0) t.ms[b] = (uint8_t)sm, t.vs[b] = (uint8_t)sv;
  } else {
    store_values(static_cast<float*>(t.m), at, left, whole, m);
    store_values(static_cast<float*>(t.v), at, left, whole, v);
  }
}

template <typename TW, typename TG, bool BITS8, int kCap>
__global__ void __launch_bounds__(kAwThreads) k_adamw(const __grid_constant__ AwArgs<kCap> p) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int lo = 0, n = p.count;                                  // the tensor of this CTA: the last that starts at or before it
  while (n > 1) {
    const int half = n >> 1;
    if (p.first[lo + half] <= blockIdx.x) lo += half, n -= half;
    else n = half;
  }
  const AwTensor& t = p.t[lo];
  const int64_t blocks = (t.n + kBlock - 1) / kBlock, b0 = (int64_t)(blockIdx.x - p.first[lo]) * kSpan + warp;
  pdl_wait();
  pdl_launch_dependents();
  const AwHyper& h = p.h;
  Rates r = {h.decay, h.step, h.root, 1.f, h.scale != nullptr};
  if (h.lr_dev || h.step_dev) {
    const float lr = h.lr_dev ? *h.lr_dev : h.lr;
    r.decay = 1.f - lr * h.wd;
    float c = h.step;                                       // 1 / (1 - b1^t) where lr is apart
    if (h.step_dev) {
      const float s = (float)*h.step_dev;
      c = -1.f / expm1f(s * h.log_b1);
      r.root = rsqrtf(-expm1f(s * h.log_b2));
    }
    r.step = lr * c;
  }
  if (r.scaled) r.gs = *h.scale;
  constexpr int kEach = kSpan / kAwWarps;                   // blocks of a warp, all on their way before the first is worked on
  if (p.wide[lo] && (b0 - warp + kSpan) * kBlock <= t.n) {
    Block<TW, TG, BITS8> in[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) in[i].load(t, b0 + i * kAwWarps, (b0 + i * kAwWarps) * kBlock + lane * kLane, 8, true);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      step_block(in[i], t, h, r, b0 + i * kAwWarps, (b0 + i * kAwWarps) * kBlock + lane * kLane, 8, true);
  } else {
    for (int64_t b = b0; b < min(b0 - warp + kSpan, blocks); b += kAwWarps) {
      const int64_t at = b * kBlock + lane * kLane, left = t.n - at;
      const bool whole = p.wide[lo] && left >= 8;
      Block<TW, TG, BITS8> in;
      in.load(t, b, at, left, whole);
      step_block(in, t, h, r, b, at, left, whole);
    }
  }
}

template <int kCap>
cudaError_t launch_adamw(const AwArgs<kCap>& a, bool w16, bool g16, bool bits8, cudaStream_t st) {
  using B = __nv_bfloat16;
  const dim3 grid(a.first[a.count]), block(kAwThreads);
  if (bits8) {
    if (w16) return g16 ? launch_pdl(k_adamw<B, B, true, kCap>, grid, block, 0, st, a) : launch_pdl(k_adamw<B, float, true, kCap>, grid, block, 0, st, a);
    return g16 ? launch_pdl(k_adamw<float, B, true, kCap>, grid, block, 0, st, a) : launch_pdl(k_adamw<float, float, true, kCap>, grid, block, 0, st, a);
  }
  if (w16) return g16 ? launch_pdl(k_adamw<B, B, false, kCap>, grid, block, 0, st, a) : launch_pdl(k_adamw<B, float, false, kCap>, grid, block, 0, st, a);
  return g16 ? launch_pdl(k_adamw<float, B, false, kCap>, grid, block, 0, st, a) : launch_pdl(k_adamw<float, float, false, kCap>, grid, block, 0, st, a);
}

// tensors [from, count) as launches of up to kCap
template <int kCap>
cudaError_t step_tensors(const AwHyper& h, const asi_adamw_desc_t* d, const asi_adamw_tensor_t* tensors, int32_t count, cudaStream_t st) {
  AwArgs<kCap> a;
  a.h = h;
  a.count = 0;
  uint32_t ctas = 0;
  for (int32_t i = 0; i <= count; ++i) {
    const int64_t more = i < count ? (tensors[i].n + (int64_t)kBlock * kSpan - 1) / ((int64_t)kBlock * kSpan) : 0;
    if (a.count && (i == count || a.count == kCap || ctas + more > INT32_MAX)) {
      a.first[a.count] = ctas;
      const cudaError_t e = launch_adamw<kCap>(a, d->weight_dtype == ASI_BF16, d->grad_dtype == ASI_BF16, d->state_bits == 8, st);
      if (e != cudaSuccess) return e;
      a.count = 0;
      ctas = 0;
    }
    if (!more) continue;
    const asi_adamw_tensor_t& t = tensors[i];
    a.t[a.count] = AwTensor{t.weight, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale,
                            static_cast<__nv_bfloat16*>(t.copy), t.n};
    a.wide[a.count] = ((reinterpret_cast<uintptr_t>(t.weight) | reinterpret_cast<uintptr_t>(t.grad) | reinterpret_cast<uintptr_t>(t.exp_avg) |
                        reinterpret_cast<uintptr_t>(t.exp_avg_sq) | reinterpret_cast<uintptr_t>(t.copy)) & 15u) == 0;
    a.first[a.count++] = ctas;
    ctas += (uint32_t)more;
  }
  return cudaSuccess;
}

struct Range {
  uintptr_t from, to;
  bool written;
  bool operator<(const Range& o) const { return from < o.from; }
};

// no written range meets another: swept by start, with the furthest ends seen so far
bool written_apart(std::vector<Range>& r) {
  std::sort(r.begin(), r.end());
  uintptr_t any = 0, written = 0;
  for (const Range& x : r) {
    if (x.from < written || (x.written && x.from < any)) return false;
    any = std::max(any, x.to);
    if (x.written) written = std::max(written, x.to);
  }
  return true;
}

}  // namespace

}  // namespace asi

using namespace asi;

extern "C" asi_status_t asi_adamw_step(const asi_adamw_desc_t* d, const asi_adamw_tensor_t* tensors, int32_t count, void* stream) {
  if (!d || count < 0 || (count > 0 && !tensors)) return ASI_ERR_INVALID_ARG;
  if ((d->weight_dtype != ASI_F32 && d->weight_dtype != ASI_BF16) || (d->grad_dtype != ASI_F32 && d->grad_dtype != ASI_BF16) ||
      (d->state_bits != 32 && d->state_bits != 8))
    return ASI_ERR_INVALID_ARG;
  const bool betas = d->beta1 >= 0 && d->beta1 < 1 && d->beta2 >= 0 && d->beta2 < 1;
  const bool rates = d->weight_decay >= 0 && std::isfinite((float)d->weight_decay) && d->eps >= 1e-16 && std::isfinite((float)d->eps) &&
                     (d->lr_dev || (d->lr >= 0 && std::isfinite((float)d->lr)));
  if (!betas || !rates || (!d->step_dev && d->step < 1)) return ASI_ERR_INVALID_ARG;
  const size_t ew = d->weight_dtype == ASI_BF16 ? 2 : 4, eg = d->grad_dtype == ASI_BF16 ? 2 : 4, es = d->state_bits / 8;
  try {
    std::vector<Range> ranges;
    ranges.reserve((size_t)count * 7 + 3);
    bool fine = true;
    auto add = [&](const void* p, size_t bytes, size_t element, bool written) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(p);
      fine = fine && p && at % element == 0;
      ranges.push_back(Range{at, at + bytes, written});
    };
    for (int32_t i = 0; i < count && fine; ++i) {
      const asi_adamw_tensor_t& t = tensors[i];
      if (t.n < 0 || t.n > (int64_t)1 << 38) return ASI_ERR_INVALID_ARG;
      if (t.n == 0) continue;
      const size_t n = (size_t)t.n, blocks = (n + kBlock - 1) / kBlock;
      add(t.weight, n * ew, ew, true);
      add(t.grad, n * eg, eg, false);
      add(t.exp_avg, n * es, es, true);
      add(t.exp_avg_sq, n * es, es, true);
      if (d->state_bits == 8) {
        add(t.exp_avg_scale, blocks, 1, true);
        add(t.exp_avg_sq_scale, blocks, 1, true);
      }
      if (t.copy) add(t.copy, n * 2, 2, true);
    }
    if (d->lr_dev) add(d->lr_dev, 4, 4, false);
    if (d->step_dev) add(d->step_dev, 8, 8, false);
    if (d->grad_scale) add(d->grad_scale, 4, 4, false);
    if (!fine || !written_apart(ranges)) return ASI_ERR_INVALID_ARG;
    AwHyper h = {};
    h.b1 = (float)d->beta1, h.b2 = (float)d->beta2, h.c1 = (float)(1 - d->beta1), h.c2 = (float)(1 - d->beta2);
    h.one = 1.f;
    h.eps = (float)d->eps, h.lr = (float)d->lr, h.wd = (float)d->weight_decay;
    h.log_b1 = (float)std::log(d->beta1), h.log_b2 = (float)std::log(d->beta2);
    h.lr_dev = d->lr_dev, h.step_dev = d->step_dev, h.scale = d->grad_scale;
    if (!d->step_dev) {
      const double c = 1 / (1 - std::pow(d->beta1, (double)d->step));
      h.step = (float)(d->lr_dev ? c : d->lr * c);
      h.root = (float)(1 / std::sqrt(1 - std::pow(d->beta2, (double)d->step)));
    }
    h.decay = (float)(1 - d->lr * d->weight_decay);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(count <= 16   ? step_tensors<16>(h, d, tensors, count, st)
                       : count <= 64 ? step_tensors<64>(h, d, tensors, count, st)
                                     : step_tensors<400>(h, d, tensors, count, st),
                       "AdamW step");
  } catch (...) {
    return no_host_memory();
  }
}
