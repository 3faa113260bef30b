// One AdamW step over many tensors, states in 32 or 8 bits.
//
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;  w = (1 - lr wd) w - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// m, v and sqrt(v) are computed in separately rounded fp32 operations in the order written, so that the 8-bit codes are a
// function of the inputs alone (no contraction that another build or a plain restatement would do otherwise).
//
// What bounds it: weights and states read and written once, gradients read once.  A warp takes blocks of 256 elements,
// eight a lane: with 8-bit states the block's largest magnitude is one warp reduction away and codes are quantised where
// they were computed.  The tensors of a call share a launch: a table of them travels with the kernel's arguments.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <utility>
#include <vector>

#include "asi_internal.h"

namespace asi {

namespace {

constexpr int kAwThreads = 256;
constexpr int kAwWarps = kAwThreads / 32;
constexpr int kBlock = ASI_ADAMW_BLOCK;
constexpr int kLane = kBlock / 32;            // elements of a lane
constexpr int kSpan = 16;                     // blocks of a CTA

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

template <typename T>
__device__ __forceinline__ void read8(const T* p, int64_t left, bool wide, float* f);
template <>
__device__ __forceinline__ void read8<float>(const float* p, int64_t left, bool wide, float* f) {
  if (wide && left >= 8) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < left ? p[i] : 0.f;
  }
}
template <>
__device__ __forceinline__ void read8<__nv_bfloat16>(const __nv_bfloat16* p, int64_t left, bool wide, float* f) {
  if (wide && left >= 8) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < left ? __bfloat162float(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void write8(float* p, int64_t left, bool wide, const float* f) {
  if (wide && left >= 8) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = f[i];
  }
}
__device__ __forceinline__ void write8(__nv_bfloat16* p, int64_t left, bool wide, const float* f) {
  if (wide && left >= 8) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = __float2bfloat16_rn(f[i]);
  }
}

// 2^(byte - 127)
__device__ __forceinline__ float scale_of(uint8_t byte) { return __uint_as_float(byte ? (uint32_t)byte << 23 : 0x00400000u); }

__device__ __forceinline__ void decode8(const uint8_t* p, int64_t left, bool wide, float scale, float* f) {
  uint32_t w[2] = {0, 0};
  if (wide && left >= 8) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    w[0] = a.x, w[1] = a.y;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint16_t two = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(two, __NV_E4M3);
    const float2 v = __half22float2(__half2(h));
    f[2 * i] = v.x * scale, f[2 * i + 1] = v.y * scale;
  }
}

// The block's scale byte from the lanes' eight values each: the smallest 2^k with max <= 448 2^k = 1.75 2^(k + 8)
__device__ __forceinline__ uint32_t block_scale(const float* f) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(f[i]) & 0x7fffffffu;
    if (b < 0x7f800000u) top = max(top, b);                 // finite: magnitudes order as their bits do
  }
  top = __reduce_max_sync(~0u, top);
  if (top == 0) return 127;
  const int k = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
  return (uint32_t)(max(k, -126) + 127);
}

__device__ __forceinline__ void encode8(uint8_t* p, int64_t left, bool wide, uint32_t byte, bool above_zero, const float* f) {
  const float inv = __uint_as_float((254u - byte) << 23);   // 2^-k; byte is 1 .. 247
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = f[2 * i] * inv, b = f[2 * i + 1] * inv;
    if (above_zero) {
      if (a > 0.f) a = fmaxf(a, 0.001953125f);              // 2^-9, the smallest code
      if (b > 0.f) b = fmaxf(b, 0.001953125f);
    }
    uint32_t two = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    // infinities (saturated above) are held as NaN
    if (isinf(a)) two |= 0x7fu;
    if (isinf(b)) two |= 0x7f00u;
    w[i >> 1] |= two << (16 * (i & 1));
  }
  if (wide && left >= 8) {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
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
  const bool wide = p.wide[lo];
  const int64_t b0 = (int64_t)(blockIdx.x - p.first[lo]) * kSpan, blocks = (t.n + kBlock - 1) / kBlock;
  pdl_wait();
  pdl_launch_dependents();
  const AwHyper& h = p.h;
  float decay = h.decay, step = h.step, root = h.root;
  if (h.lr_dev || h.step_dev) {
    const float lr = h.lr_dev ? *h.lr_dev : h.lr;
    decay = 1.f - lr * h.wd;
    float c = h.step;                                       // 1 / (1 - b1^t) where lr is apart
    if (h.step_dev) {
      const float s = (float)*h.step_dev;
      c = -1.f / expm1f(s * h.log_b1);
      root = rsqrtf(-expm1f(s * h.log_b2));
    }
    step = lr * c;
  }
  const float gs = h.scale ? *h.scale : 1.f;
  for (int64_t b = b0 + warp; b < min(b0 + kSpan, blocks); b += kAwWarps) {
    const int64_t at = b * kBlock + lane * kLane, left = t.n - at;
    float w[8], g[8], m[8], v[8];
    read8<TW>(static_cast<const TW*>(t.w) + at, left, wide, w);
    read8<TG>(static_cast<const TG*>(t.g) + at, left, wide, g);
    if (BITS8) {
      decode8(static_cast<const uint8_t*>(t.m) + at, left, wide, scale_of(t.ms[b]), m);
      decode8(static_cast<const uint8_t*>(t.v) + at, left, wide, scale_of(t.vs[b]), v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], v[i]);
    } else {
      read8<float>(static_cast<const float*>(t.m) + at, left, wide, m);
      read8<float>(static_cast<const float*>(t.v) + at, left, wide, v);
    }
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float gi = h.scale ? __fmul_rn(g[i], gs) : g[i];
      m[i] = __fadd_rn(__fmul_rn(m[i], h.b1), __fmul_rn(gi, h.c1));
      v[i] = __fadd_rn(__fmul_rn(v[i], h.b2), __fmul_rn(__fmul_rn(gi, gi), h.c2));
      r[i] = __fsqrt_rn(v[i]);
      w[i] = fmaf(w[i], decay, -step * __fdividef(m[i], fmaf(r[i], root, h.eps)));
    }
    write8(static_cast<TW*>(t.w) + at, left, wide, w);
    if (t.copy) write8(t.copy + at, left, wide, w);
    if (BITS8) {
      const uint32_t sm = block_scale(m), sv = block_scale(r);
      encode8(static_cast<uint8_t*>(t.m) + at, left, wide, sm, false, m);
      encode8(static_cast<uint8_t*>(t.v) + at, left, wide, sv, true, r);
      if (lane == 0) t.ms[b] = (uint8_t)sm, t.vs[b] = (uint8_t)sv;
    } else {
      write8(static_cast<float*>(t.m) + at, left, wide, m);
      write8(static_cast<float*>(t.v) + at, left, wide, v);
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
  const bool rates = d->weight_decay >= 0 && std::isfinite(d->weight_decay) && d->eps >= 1e-30 && std::isfinite((float)d->eps) &&
                     (d->lr_dev || (d->lr >= 0 && std::isfinite(d->lr)));
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
    return cuda_status(count <= 32 ? step_tensors<32>(h, d, tensors, count, st) : step_tensors<400>(h, d, tensors, count, st), "AdamW step");
  } catch (...) {
    return no_host_memory();
  }
}
