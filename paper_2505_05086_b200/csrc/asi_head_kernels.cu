// Output layer and loss in one: log probabilities of given tokens from the last hidden states x [T][D] and the output layer's weight
// w [V][D], and their gradients, without logits that outlive a tile.
//
//   X_j = scale x_t . w_j;   lse = log sum_j exp X_j;   logp = X_y - lse;   entropy = lse - sum_j p_j X_j
//   G[t][j] = scale (dlogp ([j = y] - p_j) - dentropy p_j (log p_j + entropy));   dx = G w;   dw = G^T x
//
// Four matrix products, all by k_head_gemm: the logits' tiles leave nothing but a maximum and two sums a row (and the target's logit)
// behind, k_head_rows joins these, and then for a piece of the vocabulary at a time the logits are computed again, this time
// leaving G (in the workspace), from which one launch makes the piece's share of dx and its rows of dw.  Few rows keep their logits (in
// fp32, in the workspace) where these take no more than a piece of G would.
//
// What bounds it: the tensor cores, 2 T V D operations a product (for a few rows the bytes of w, read twice, and of dw).  4096 x 32000 x 2048
// bf16 in bursts: logits and their sums 356 us (1508 TFLOP/s), G of 16128 columns 182 (1487), both products of G 336 (1611); in long loops the
// power cap takes 15 % of that.
//
// Operands are bf16.  fp32 ones are split into three terms each (hi, mid, lo: 24 bits) by k_head_split, and a product takes the
// six pairs of terms down to 2^-16 of the first (what is left out is 2^-24).  G is split likewise where its product goes to
// fp32.  Rows of bf16 off 16 bytes, which tensor copies cannot fetch, go through the same kernel as one term.
// G for results in bf16 is rounded to bf16.  One entry of its row, the target's, is as large as all others together, and its rounding no less: that comes
// back as rank-one terms, off[t] w[y] in dx, off[t] x[t] in row y of dw (struct Back); few rows have two terms of G for dw instead (kFewRows).
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "asi_internal.h"
#include "asi_tc_ptx.h"

namespace asi {

namespace {

constexpr int kWorkers = 8;                               // epilogue warps
constexpr int kThreads = (kWorkers + 4) * 32;             // + the issuer's, the producer's and two that make these a group of four
// Registers of a thread: 168 at launch (65536 / 384); the second group hands on what it does not need
constexpr int kWorkerRegs = 216, kOtherRegs = 72;
static_assert(kWorkers * 32 * kWorkerRegs + 128 * kOtherRegs <= kThreads * 168, "the groups' shares have to fit what the CTA was launched with");
constexpr int kTile = 256;                                // rows and columns of a pair's tile
constexpr int kK = 64;                                    // k of a box: 64 bf16 = one 128-byte swizzle row
constexpr int kMaxStages = 3;
constexpr uint32_t kHalf = 128 * kK * 2;                  // a CTA's half of an operand's box
constexpr uint32_t kStaged = 32 * 128;                    // a warp's staged results: 32 rows of 128 bytes
// Pairs of boxes that a product's segments in TMEM aim at where results are held to fp32 (kWhole need no segments), before they are rounded up to
// whole chunks: 8 with one term of either operand (512 k), 12 with six pairs of terms a chunk (128 k of the operands), 9 with three (192).  What truncation
// takes from a logit is in proportion to them: lse of 40 x 11324 x 761 fp32 5.4e-7 too small with 18, 2.9e-7 with 12 (entropy 1.0e-6 and 5.4e-7 too
// large); of 4096 x 32000 x 2048 bf16 5.9e-6 with 16, 2.9e-6 with 8 (lse around 13; entropy 5.5e-6 and 2.3e-6).  Aiming at 16 instead would spare operands in
// three terms 0 to 4 % (1001 x 30011 x 771 794 us -> 760), single terms 4 % (scoring 4096 x 32000 x 2048 373 us -> 357).
constexpr int kSeg = 8, kWhole = 12;
// The same where results are rounded to bf16 (by 2^-8 of them at most): truncation takes 1.6e-3 of a sum of 4096 pairs (dw of 262144 rows), always towards zero, so
// that sums of more than 512 (2e-4) go in segments of about 64.
constexpr int kSegB16 = 64, kWholeB16 = 512;
constexpr float kLog2e = 1.44269504088896341f, kLog2eLow = 1.925963033500e-8f, kLn2 = 0.69314718055994531f;

enum Epi { kStats = 0, kGrad = 1, kOut = 2 };
enum Kind { kNone = 0, kF32 = 1, kB16 = 2 };

// One product C[m][n] = sum over k and pairs of terms of A(m, k) B(n, k).  An operand lies with its k together (mn = 0: boxes of 64 k
// x 128 rows) or with its rows together (mn = 1: boxes of 64 rows x all k of the chunk, two of them); terms are the map's third axis.
struct HeadProb {
  CUtensorMap a, b;
  int a_mn, b_mn;
  int a_off, a_k, b_off, b_k;   // where the product's first row and first k lie in the operand
  int M, N, mt, nt, splits;     // tiles; `splits` shares of k one after another
  int kc, per;                  // chunks of k, and of a share
  // A chunk of `sub` times 64 k shares a stage: A's terms, then B's, `sub` times 16 KB each
  int sub, a_terms, b_terms;
  int pairs;                    // pairs of parts (64 k of a term) that are multiplied
  uint32_t a_part, b_part;      // of each pair, two bits
  int seg_pairs, whole;         // pairs of boxes that its segments aim at, and that need none (kSeg, kWhole)
  int seg;                      // chunks that add up in TMEM (kSegmented), or all
  int n_first;                  // tiles of a row follow one another (else tiles of a column)
  const void* add;              // added to the result, laid out like it; null: nothing
  void* out;
  int add_kind, out_kind;
  int64_t ld, split_stride;     // elements
  CUtensorMap o;                // the result in boxes of 32 rows of 128 bytes
  int how;                      // Store: how results leave
  int correct;                  // Correct: where what rounding took from G at the targets is added
};
// not at all, to rows of x's gradient (off[t] w[y]), or to those of w's (off[t] x[t] for the rows t of that target)
enum Correct { kNowhere = 0, kToDx = 1, kToDw = 2 };
// by coalesced words (any alignment, `add` of any kind), by tensor copies, or added to fp32 by tensor copies (add is out)
enum Store { kWords = 0, kCopy = 1, kAdd = 2 };
struct HeadArgs {
  HeadProb p[2];
  int np, tiles0, tiles;        // tiles of the first product, of all
  int few, each_few, more_few, each_rest, more_rest;   // of the second product: how many a pair takes (see Mine)
  int nst, stage;               // stages, and bytes of one
  int place;
  int* status;
  int stall;                    // test hook: no copies, short waits
  // kStats, kGrad:
  const int64_t* y;
  int64_t ignore, V;
  int64_t v0;                   // first column of the piece
  int T;
  float c, scale;               // c = scale log2(e)
  float *pm, *ps, *pw, *xy;     // [2 nt][T]: maximum (base 2), sum, weighted sum; [T]: the target's logit
  const float2* row;            // maximum (base 2) and log2 of the sum of each row
  const float* lse;             // null, or what a row goes by where it is below `far`.  Then kStats sums the others alone (see kFarLse)
  float far;
  const float *entropy, *dlogp, *dent;
  float* off;                   // [T]: what rounding took from G at the target (bf16 operands), or null; w and its row stride beside it
  const __nv_bfloat16 *w, *x;   // (x has it too)
  int64_t ld_w;
  const int *first, *next;      // [V], [T]: rows of a target, one after another in any order; each is its number + 1, 0 ends them
  CUtensorMap g;                // G: boxes of 32 rows of 64 columns (one term) or 32
  int terms;                    // of G
};

__device__ __forceinline__ void add_scaled(float* v, float a, const uint4& x) {   // v += a x, eight values, two an instruction
  const uint32_t h[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %4};\n\tmov.b64 z, {%0, %1};\n\tfma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "+f"(v[2 * i]), "+f"(v[2 * i + 1]) : "f"(__uint_as_float(h[i] << 16)), "f"(__uint_as_float(h[i] & 0xffff0000u)), "f"(a));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// The rows of a target, for what rounding took from G there.  Of up to kWalk rows the first kBack in order have theirs given back, from more none: a thread walks the
// list of its row of dw and reads rows of x for it, which many would hold up.  A tile's epilogue waits for its own instructions, so that warps without
// such rows skip all of it (300 x 32000 x 2048 bf16 220 us instead of 234; 208 without the lists, 251 with four rows given back).
constexpr int kBack = 2, kWalk = 4, kNoRow = 1 << 30;
struct Back {
  bool some = false, more = false;   // any lane of the warp has one, or two
  int row[kBack];
  float off[kBack];
  uint4 x[kBack][4];               // 32 columns of theirs
  // t: the first of this lane's list
  __device__ __forceinline__ void find(const HeadArgs& g, int t) {
    some = __any_sync(~0u, t != 0);
    if (!some) return;
    int n = 0;
#pragma unroll
    for (int i = 0; i < kBack; ++i) row[i] = kNoRow;
#pragma unroll 1
    for (; t && n <= kWalk; t = g.next[t - 1], ++n) {
      int r = t - 1;
#pragma unroll
      for (int i = 0; i < kBack; ++i) {
        const int low = min(row[i], r);
        r = max(row[i], r);
        row[i] = low;
      }
    }
    if (n > kWalk) row[0] = row[1] = kNoRow;
#pragma unroll
    for (int i = 0; i < kBack; ++i) off[i] = row[i] != kNoRow ? g.off[row[i]] : 0.f;
    more = __any_sync(~0u, row[1] != kNoRow);
  }
  // columns from n of N on (rows of x, or of its terms, go on to a multiple of 8)
  __device__ __forceinline__ void bring(const HeadArgs& g, int n, int N) {
    if (!some) return;
    bring_of(g, 0, n, N);
    if (more) bring_of(g, 1, n, N);
  }
  __device__ __forceinline__ void give(float (&v)[32], int n, int N) const {
    if (!some) return;
    give_of(0, v, n, N);
    if (more) give_of(1, v, n, N);
  }
  __device__ __forceinline__ void bring_of(const HeadArgs& g, int i, int n, int N) {
    if (row[i] == kNoRow) return;
    const uint4* at = reinterpret_cast<const uint4*>(g.x + row[i] * g.ld_w + n);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (n + 8 * u < N) x[i][u] = __ldg(at + u);
  }
  __device__ __forceinline__ void give_of(int i, float (&v)[32], int n, int N) const {
    if (row[i] == kNoRow) return;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (n + 8 * u < N) add_scaled(v + 8 * u, off[i], x[i][u]);
  }
};
static_assert(kBack == 2, "some and more stand for the two");

// maximum, sum and weighted sum (of e_j = 2^a_j: sum e_j, sum e_j a_j) of what a thread has seen of its row
struct RowStats {
  float top = -INFINITY, m = 0.f, s = 0.f, w = 0.f;      // top: largest logit; m = c top, what exponents are relative to
  __device__ __forceinline__ void add(const float (&v)[32], float c) {
    float t = v[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) t = fmaxf(t, v[i]);
    if (t > top) {
      const float m2 = t * c;
      if (top != -INFINITY) {                            // (else the sums are 0, or NaN for good)
        const float d = m - m2, r = ex2(d);
        w = r * fmaf(d, s, w);
        s *= r;
      }
      top = t, m = m2;
    }
    float s2 = 0.f, w2 = 0.f;
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float a = fmaf(v[i], c, -m), b = fmaf(v[i + 1], c, -m), ea = ex2(a), eb = ex2(b);
      s += ea, s2 += eb;
      w = fmaf(ea, fmaxf(a, -200.f), w), w2 = fmaf(eb, fmaxf(b, -200.f), w2);   // (2^-200 is 0 here; 0 * -inf would not be)
    }
    s += s2, w += w2;
  }
};

// What a gradient without its forward pass takes lse for: p = exp(x - lse) is off by 2^-24 |lse|, 2^-17 of it from 128 on where G goes out in terms, 2^-12 from
// 4096 on beside the 2^-9 of a rounding to bf16.  Rows beyond that are summed again: the forward direction's kernels are launched in any case and have
// nothing to do where their rows are near (9 x 32000 x 2048 bf16 133 us instead of 126).
constexpr float kFarLseTerms = 128.f, kFarLse = 4096.f;
__device__ __forceinline__ bool is_far(const float* lse, const int64_t* y, int64_t ignore, int64_t row, float far) { return fabsf(lse[row]) >= far && y[row] != ignore; }

// what G of a row needs
struct RowGrad {
  float hi, lo, alpha, beta, h;
  int y;                       // its target's column in the vocabulary, -1: none
  bool live;
  float* off;                  // where what rounding takes from G there goes, or null
};

__device__ __forceinline__ RowGrad row_grad(const HeadArgs& g, int row) {
  RowGrad r = {0.f, 0.f, 0.f, 0.f, 0.f, -1, false, nullptr};
  if (row >= g.T) return r;
  const int64_t y = g.y[row];
  r.live = y != g.ignore;
  const bool in = y >= 0 && y < g.V;
  r.y = in ? (int)y : -1;
  r.off = g.off ? g.off + row : nullptr;
  r.alpha = in ? g.dlogp[row] : NAN;
  if (g.dent) r.beta = g.dent[row], r.h = g.entropy[row];
  const float l = g.lse ? g.lse[row] : 0.f;
  if (!g.lse || fabsf(l) >= g.far) {
    const float2 q = g.row[row];
    r.hi = q.x, r.lo = q.y;
  } else {
    r.hi = l * kLog2e;
    r.lo = fmaf(l, kLog2e, -r.hi) + l * kLog2eLow;
  }
  if (r.hi == -INFINITY) r.hi = INFINITY, r.lo = 0.f;      // a row of nothing but -inf: every p is 0
  return r;
}

// kN logits of a row, the first in column j0 of the vocabulary, become their gradients (by a whole warp)
template <int kN>
__device__ __forceinline__ void to_gradient(float (&v)[kN], const RowGrad& r, const HeadArgs& g, int64_t j0) {
  const float a = -g.scale * r.alpha;
  if (__any_sync(~0u, r.beta != 0.f)) {
    const float b = g.scale * r.beta;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float x = fmaf(v[i], g.c, -r.hi) - r.lo, p = ex2(x);
      v[i] = p * fmaf(-b, fmaf(fmaxf(x, -200.f), kLn2, r.h), a);
    }
  } else {
    // (hi and lo apart: their sum is off by 2^-24 of it, which logits of 10^4 and more would show in bf16 too)
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = ex2(fmaf(v[i], g.c, -r.hi) - r.lo) * a;
  }
  const int hot = r.y - (int)j0;                           // (V <= 2^24)
  if (hot >= 0 && hot < kN) {
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (i == hot) {
        v[i] -= a;
        if (r.off) *r.off = v[i] - __bfloat162float(__float2bfloat16_rn(v[i]));
      }
  }
  if (!r.live) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = 0.f;
  }
  if (g.V - j0 < kN) {
    const int left = (int)(g.V - j0);
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (i >= left) v[i] = 0.f;
  }
}

// Waits of a whole warp that end (mbar_wait's limit); one answer for all lanes, so that what follows stays in uniform registers
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int stall) {
  bool ok = __all_sync(~0u, mbar_try_wait(bar, parity));
  if (!ok) ok = __all_sync(~0u, mbar_wait(bar, parity, stall));
  return ok;
}

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// Column `lane` of staged results (32 x 32, column i of row r at i ^ r), up to 32 rows, added to another's and stored.  What is added is on its
// way for sixteen rows at once.
template <typename TO, typename TA>
__device__ __forceinline__ void put_words(const float* s, int lane, TO* to, const TA* add, int64_t ld, int rows) {
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += 16, to += 16 * ld, add += add ? 16 * ld : 0) {
    float f[16];
    const TA* from = add;
#pragma unroll
    for (int r = 0; r < 16; ++r, from += ld) f[r] = add && r0 + r < rows ? as_float(*from) : 0.f;
    TO* at = to;
#pragma unroll
    for (int r = 0; r < 16; ++r, at += ld)
      if (r0 + r < rows) *at = (TO)(f[r] + s[(r0 + r) * 32 + (lane ^ (r0 + r))]);
  }
}

// A pair of CTAs owns a tile of 256 x 256: each brings half of either operand's chunk (128 rows) to its shared memory, products are
// issued for both by the first one (tcgen05, cta_group 2: each tensor core reads its own half of A and both halves of B), and each
// has the 128 x 256 accumulators of its rows in its TMEM, twice, so that the next tile's products run under this one's epilogue.
// (A CTA by itself would read twice the bytes of B for the same products.)  Roles: a producer warp, an issuer warp, eight epilogue warps (a
// thread a row and half of the columns).
// kSegmented: long sums.  The unit's own sums truncate, so they go to registers on the way (HeadProb::seg).
// kLists: rows of dw get back what rounding took from G (Correct).
template <int kEpi, bool kSegmented, bool kLists>
__global__ void __launch_bounds__(kThreads, 1) k_head_gemm(const __grid_constant__ HeadArgs g) {
  extern __shared__ __align__(1024) uint8_t head_smem[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(head_smem) + 1023) & ~(uintptr_t)1023);
  __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], done[2], acc_free[2], drained[1];
  __shared__ uint32_t tmem_slot[1];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = (int)cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  if (tid == 0) {
    for (int i = 0; i < kMaxStages; ++i) mbar_init(full + i, 1), mbar_init(empty + i, 1);
    for (int i = 0; i < 2; ++i) mbar_init(done + i, 1), mbar_init(acc_free + i, 2 * kWorkers);
    mbar_init(drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_sync_all();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  struct Tile { int q, m, n, s, chunks, k0; };
  // The tiles of a pair: every `pairs`-th of the first product, and of the second one every so many of a stretch for pairs that had as many
  // of the first (pairs below `few` had one more; the stretches' lengths make up for that).  Pairs side by side work on tiles side by side, which
  // share a row of G (a stretch a pair read 1.19 GB instead of 0.43 for 4096 x 16128 x 2048, in 371 us instead of 340)
  int mine0 = (g.tiles0 - pair + pairs - 1) / pairs;
  if constexpr (kEpi == kStats) {
    if (g.lse) {                                         // (tiles of a column: a tile's rows come again after mt of them at most)
      const int mt = g.p[0].mt, some = mine0 < mt ? mine0 : mt;
      bool any = false;
#pragma unroll 4
      for (int i = 0; i < some; ++i) {
        const int64_t row = (int64_t)((pair + (int64_t)i * pairs) % mt) * kTile + tid;
        any |= tid < kTile && row < g.T && is_far(g.lse, g.y, g.ignore, row, g.far);
      }
      if (!__syncthreads_or(any)) mine0 = 0;
    }
  }
  const bool late = pair >= g.few;
  const int q1 = late ? pair - g.few : pair, each1 = late ? g.each_rest : g.each_few, more1 = late ? g.more_rest : g.more_few;
  const int from1 = (late ? g.few * g.each_few + g.more_few : 0) + q1, step1 = late ? pairs - g.few : g.few;
  const int mine = mine0 + (g.np > 1 ? each1 + (q1 < more1 ? 1 : 0) : 0);
  auto tile_of = [&](int i) {
    Tile x;
    x.q = i >= mine0 ? 1 : 0;
    const HeadProb& p = g.p[x.q];
    int t = x.q ? from1 + (i - mine0) * step1 : pair + i * pairs;
    const int each = p.mt * p.nt;
    x.s = t / each;
    t -= x.s * each;
    x.m = p.n_first ? t / p.nt : t % p.mt;
    x.n = p.n_first ? t % p.nt : t / p.mt;
    x.k0 = x.s * p.per;
    x.chunks = p.kc - x.k0 < p.per ? p.kc - x.k0 : p.per;
    if (x.chunks < 0) x.chunks = 0;
    return x;
  };
  const int nst = g.nst, stall = g.stall, stage = g.stage;
  bool ok = true;
  int loads = 0;
  if (warp >= kWorkers) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  if (warp == kWorkers) {
    // ---- issuer: the warp as a whole goes through the loop, so that addresses and descriptors stay in uniform registers (by one
    // lane alone a chunk's issue took 600 cycles, its products 512), and one lane issues
    if (rank == 0) {
      const uint32_t at = smem_u32(base);
      int st = 0, seg = 0;
      uint32_t ph = 0;
      bool ready = false;
      const uint32_t empty0 = smem_u32(empty), done0 = smem_u32(done);
#pragma unroll 1
      for (int t = 0; t < mine && ok; ++t) {
        const Tile x = tile_of(t);
        const HeadProb& p = g.p[x.q];
        const uint32_t idesc = instr_desc_bf16(kTile, kTile, p.a_mn != 0, p.b_mn != 0);
        // a k-step is 16 bf16: 32 bytes inside the swizzle row of a K-major tile, 16 rows (2048 bytes) of an MN-major one
        const uint64_t a_step = p.a_mn ? 128 : 2, b_step = p.b_mn ? 128 : 2;
        const uint64_t da0 = smem_desc_sw128(at, p.a_mn ? p.sub * kHalf / 2 : 16), db0 = smem_desc_sw128(at + p.a_terms * p.sub * kHalf, p.b_mn ? p.sub * kHalf / 2 : 16);
        // the second 64 k of a chunk: the next box, or the next rows of the same ones
        const uint32_t a_next = (p.a_mn && p.sub > 1 ? kHalf / 2 : kHalf) >> 4, b_next = (p.b_mn && p.sub > 1 ? kHalf / 2 : kHalf) >> 4;
        const int per_seg = p.seg, pairs_of = p.pairs;
        const uint32_t a_part = p.a_part, b_part = p.b_part;
#pragma unroll 1
        for (int c0 = 0; c0 < x.chunks && ok; c0 += per_seg, ++seg) {
          const int buf = seg & 1, turn = seg >> 1;
          if (turn > 0) {
            ok = warp_wait(acc_free + buf, (uint32_t)(turn + 1) & 1u, stall);
            if (!ok) break;
            // (TMEM is ordered by tcgen05's own fences; one of the cluster's memory took 2400 cycles here)
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          }
          const int c1 = x.chunks - c0 < per_seg ? x.chunks : c0 + per_seg;
          const uint32_t acc = tmem + (uint32_t)(buf * kTile);
#pragma unroll 1
          for (int c = c0; c < c1; ++c) {
            ok = __all_sync(~0u, ready);
            if (!ok) ok = warp_wait(full + st, ph, stall);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t da1 = da0 + (uint64_t)(st * (stage >> 4)), db1 = db0 + (uint64_t)(st * (stage >> 4));
            const uint32_t used = empty0 + st * 8;
            if (++st == nst) st = 0, ph ^= 1u;
            ready = mbar_test(full + st, ph);              // (the answer comes while products are issued)
#pragma unroll 1
            for (int e = 0; e < pairs_of; ++e) {
              const uint64_t da = da1 + ((a_part >> (2 * e)) & 3) * a_next, db = db1 + ((b_part >> (2 * e)) & 3) * b_next;
#pragma unroll
              for (int ks = 0; ks < kK / 16; ++ks)
                umma_pair_bf16_one(acc, da + ks * a_step, db + ks * b_step, idesc, ((c - c0) | e | ks) ? 1u : 0u);
            }
            umma_pair_commit_one(used);
            if (c + 1 == c1) umma_pair_commit_one(done0 + buf * 8);
          }
        }
      }
    }
  } else if (warp == kWorkers + 1) {
    // ---- producer: this CTA's half of each chunk, counted by the first CTA's barrier
    {
      const uint32_t full0 = in_cta(full, 0);
      int st = 0;
      uint32_t ph = 1;
#pragma unroll 1
      for (int t = 0; t < mine && ok; ++t) {
        const Tile x = tile_of(t);
        const HeadProb& p = g.p[x.q];
        const int am = p.a_off + x.m * kTile + rank * 128, bn = p.b_off + x.n * kTile + rank * 128;
        const CUtensorMap *ma = &p.a, *mb = &p.b;
        const bool a_mn = p.a_mn != 0, b_mn = p.b_mn != 0;
        const int a_terms = p.a_terms, b_terms = p.b_terms, sub = p.sub;
        int ka = p.a_k + x.k0 * sub * kK, kb = p.b_k + x.k0 * sub * kK;
#pragma unroll 1
        for (int c = 0; c < x.chunks; ++c, ++loads) {
          if (loads >= nst) {
            ok = warp_wait(empty + st, ph, stall);
            if (!ok) break;
          }
          if (rank == 0) mbar_expect_tx_one(smem_u32(full) + st * 8, 2 * (a_terms + b_terms) * sub * kHalf);
          if (!stall) {
            uint32_t to = smem_u32(base) + st * stage;
            const uint32_t bar = full0 + st * 8;
            auto fetch = [&](const CUtensorMap* map, bool mn, int row, int k, int terms) {
#pragma unroll 1
              for (int e = 0; e < terms; ++e, to += sub * kHalf) {
                tma_pair_load_3d_one(to, map, mn ? row : k, mn ? k : row, e, bar);
                if (mn) tma_pair_load_3d_one(to + sub * kHalf / 2, map, row + 64, k, e, bar);
                else if (sub > 1) tma_pair_load_3d_one(to + kHalf, map, k + kK, row, e, bar);
              }
            };
            fetch(ma, a_mn, am, ka, a_terms);
            fetch(mb, b_mn, bn, kb, b_terms);
          }
          ka += sub * kK, kb += sub * kK;
          if (++st == nst) st = 0, ph ^= 1u;
        }
      }
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWorkerRegs));
    // ---- epilogue: warp w has the lanes 32 (w mod 4) .. of TMEM, warps 0-3 the columns [0, 128) of the tile, warps 4-7 the others
    const int quad = warp & 3, col0 = (warp >> 2) * 128;
    const uint32_t lanes = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)col0;
    const uint32_t free0 = in_cta(acc_free, 0), free1 = in_cta(acc_free + 1, 0);
    const int place = g.place;                           // results on their way out have two places in turn, `place` bytes apart, or (0) one
    uint8_t* staged = base + nst * stage + warp * (kStaged + (kEpi == kGrad && g.terms > 1 ? 0 : place));
    int seg = 0, flip = 0;
    auto next_place = [&]() {                            // its last contents have left
      if (lane == 0) {
        if (place) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      }
      __syncwarp();
      flip ^= 1;
      return staged + flip * place;
    };
    uint8_t* out = staged;
    // the first in the list of a row of dw
    auto first_of = [&](const HeadProb& p, int row) { return p.correct == kToDw && row < p.M ? g.first[g.v0 + row] : 0; };
    constexpr bool kAheadOf = kLists && !kSegmented;     // (segments' sums leave no registers: there lists are walked for every 32 columns)
    int first = 0;                                       // in the next tile
    auto next_first = [&](int t) {
      if (t >= mine) return;
      const Tile x = tile_of(t);
      first = first_of(g.p[x.q], x.m * kTile + rank * 128 + quad * 32 + lane);
    };
    if (kAheadOf) next_first(0);
#pragma unroll 1
    for (int t = 0; t < mine && ok; ++t) {
      const Tile x = tile_of(t);
      const HeadProb& p = g.p[x.q];
      const int row0 = x.m * kTile + rank * 128 + quad * 32, row = row0 + lane;
      const int n0 = x.n * kTile + col0;
      Back back;
      if constexpr (kAheadOf) {
        back.find(g, first);
        back.bring(g, n0, p.N);
        next_first(t + 1);
      }
      float acc[kSegmented ? 128 : 1];
      if constexpr (kSegmented) {
#pragma unroll
        for (int i = 0; i < 128; ++i) acc[i] = 0.f;
#pragma unroll 1
        for (int c0 = 0; c0 < x.chunks; c0 += p.seg, ++seg) {
          const int buf = seg & 1;
          ok = mbar_wait(done + buf, (uint32_t)(seg >> 1) & 1u, stall);
          if (__any_sync(0xffffffffu, !ok)) ok = false;
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
          for (int cc = 0; cc < 4; ++cc) {
            uint32_t u[32];
            tmem_ld32(lanes + (uint32_t)(buf * kTile + cc * 32), u);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[cc * 32 + i] += __uint_as_float(u[i]);
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive_in(buf ? free1 : free0);
        }
        if (!ok) break;
      } else if (x.chunks > 0) {
        ok = mbar_wait(done + (seg & 1), (uint32_t)(seg >> 1) & 1u, stall);
        if (__any_sync(0xffffffffu, !ok)) ok = false;
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      // 32 columns of results on their way by copies: rows of 128 bytes, 32 columns of fp32 or 64 of bf16, 16-byte units swizzled by the row
      auto by_copy = [&](const float (&v)[32], int cc, int n) {
        const bool wide = p.out_kind == kF32;
        if (wide || (cc & 1) == 0) out = next_place();
        uint8_t* r = out + lane * 128;
        if (wide) {
#pragma unroll
          for (int u = 0; u < 8; ++u) *reinterpret_cast<float4*>(r + ((u ^ (lane & 7)) * 16)) = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            *reinterpret_cast<uint4*>(r + ((((cc & 1) * 4 + u) ^ (lane & 7)) * 16)) =
                make_uint4(pack2(v[8 * u], v[8 * u + 1]), pack2(v[8 * u + 2], v[8 * u + 3]), pack2(v[8 * u + 4], v[8 * u + 5]), pack2(v[8 * u + 6], v[8 * u + 7]));
        }
        if (wide || (cc & 1)) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            const int col = wide ? n : n - 32;
            if (col < p.N && row0 < p.M) {
              if (p.how == kAdd) tma_add_3d(&p.o, out, col, row0, x.s);
              else tma_store_3d(&p.o, out, col, row0, x.s);
            }
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        }
      };
      const bool live = row0 < p.M;                      // (a warp without rows only hands its accumulators on)
      RowStats stats;
      RowGrad rg;
      if constexpr (kEpi == kGrad) rg = row_grad(g, row);
      const int64_t y = (kEpi == kStats || (kEpi == kOut && p.correct == kToDx)) && row < g.T ? g.y[row] : -1;
      const bool corrected = kEpi == kOut && p.correct == kToDx && y >= 0 && y < g.V && y != g.ignore;
      const float off = corrected ? g.off[row] : 0.f;
      const __nv_bfloat16* hot_row = g.w + (corrected ? y * g.ld_w : 0);
#pragma unroll
      for (int cc = 0; cc < 4; ++cc) {
        float v[32];
        if constexpr (kSegmented) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = acc[cc * 32 + i];
        } else if (x.chunks > 0) {
          tmem_ld32(lanes + (uint32_t)((seg & 1) * kTile + cc * 32), reinterpret_cast<uint32_t*>(v));
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (cc == 3) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_in(seg & 1 ? free1 : free0);
            ++seg;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = 0.f;
        }
        const int n = n0 + cc * 32;
        if (!live) continue;
        if constexpr (kEpi == kOut) {
          if (p.correct == kToDx && off != 0.f) {
#pragma unroll
            for (int u = 0; u < 4; ++u)                    // (rows of w, or of its terms, go on to a multiple of 8)
              if (n + 8 * u < p.N) add_scaled(v + 8 * u, off, __ldg(reinterpret_cast<const uint4*>(hot_row + n + 8 * u)));
          }
          if constexpr (kLists) {
            if (kSegmented) back.find(g, first_of(p, row)), back.bring(g, n, p.N);
            back.give(v, n, p.N);
            if (kAheadOf && cc < 3) back.bring(g, n + 32, p.N);
          }
        }
        if constexpr (kEpi == kStats) {
          if (p.how == kCopy) by_copy(v, cc, n);
          const int64_t left = g.V - n;
          if (left < 32)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (i >= left) v[i] = -INFINITY;
          stats.add(v, g.c);
          const int64_t hot = y - n;
          if (hot >= 0 && hot < 32 && y < g.V) {
            float h = v[0];
#pragma unroll
            for (int i = 1; i < 32; ++i) h = hot == i ? v[i] : h;
            g.xy[row] = h;
          }
        } else if constexpr (kEpi == kGrad) {
          if (g.terms == 1) {
            // rows of 128 bytes (64 columns), 16-byte units swizzled by the row as the tensor copy expects them
            if ((cc & 1) == 0) out = next_place();
            to_gradient<32>(v, rg, g, g.v0 + n);
#pragma unroll
            for (int u = 0; u < 4; ++u)
              *reinterpret_cast<uint4*>(out + lane * 128 + ((((cc & 1) * 4 + u) ^ (lane & 7)) * 16)) =
                  make_uint4(pack2(v[8 * u], v[8 * u + 1]), pack2(v[8 * u + 2], v[8 * u + 3]), pack2(v[8 * u + 4], v[8 * u + 5]), pack2(v[8 * u + 6], v[8 * u + 7]));
            if (cc & 1) {
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) {
                tma_store_3d(&g.g, out, n - 32, row0, 0);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
              }
            }
          } else {
            // a term after the other, rows of 64 bytes (32 columns)
            to_gradient<32>(v, rg, g, g.v0 + n);
#pragma unroll 1
            for (int e = 0; e < g.terms; ++e) {
              out = next_place();
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                uint32_t q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  q[i] = pack2(v[8 * u + 2 * i], v[8 * u + 2 * i + 1]);
                  v[8 * u + 2 * i] -= __uint_as_float(q[i] << 16);
                  v[8 * u + 2 * i + 1] -= __uint_as_float(q[i] & 0xffff0000u);
                }
                *reinterpret_cast<uint4*>(out + lane * 64 + ((u ^ ((lane >> 1) & 3)) * 16)) = make_uint4(q[0], q[1], q[2], q[3]);
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) {
                tma_store_3d(&g.g, out, n, row0, e);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
              }
            }
          }
        } else {
          if (p.how != kWords) {
            by_copy(v, cc, n);
          } else {
            // through shared memory, so that a warp's lanes are neighbouring columns
            float* s = reinterpret_cast<float*>(staged);
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");   // (of a tile of the other product)
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 32; ++i) s[lane * 32 + (i ^ lane)] = v[i];
            __syncwarp();
            const int rows = p.M - row0 < 32 ? p.M - row0 : 32;
            if (n + lane < p.N && rows > 0) {
              const int64_t at = x.s * p.split_stride + (int64_t)row0 * p.ld + n + lane;
              if (p.out_kind == kF32) {
                float* to = static_cast<float*>(p.out) + at;
                if (p.add_kind == kF32) put_words<float, float>(s, lane, to, static_cast<const float*>(p.add) + at, p.ld, rows);
                else put_words<float, float>(s, lane, to, nullptr, p.ld, rows);
              } else {
                __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.out) + at;
                if (p.add_kind == kF32) put_words<__nv_bfloat16, float>(s, lane, to, static_cast<const float*>(p.add) + at, p.ld, rows);
                else put_words<__nv_bfloat16, __nv_bfloat16>(s, lane, to, p.add_kind == kB16 ? static_cast<const __nv_bfloat16*>(p.add) + at : nullptr, p.ld, rows);
              }
            }
          }
        }
      }
      if constexpr (kEpi == kStats) {
        if (row < g.T) {
          const int64_t at = (int64_t)(2 * x.n + (warp >> 2)) * g.T + row;
          g.pm[at] = stats.top == -INFINITY ? -INFINITY : stats.m;
          g.ps[at] = stats.s;
          g.pw[at] = stats.w;
        }
      }
    }
    {
      if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // all is there before the next kernel reads it
      __syncwarp();
    }
  }
  const bool fail = __syncthreads_or(ok ? 0 : 1) != 0;
  if (fail) {                                           // what is in flight gets the limit once more
    if (tid == 0) atomicMax(g.status, (int)ASI_ERR_TIMEOUT);
    if (warp == kWorkers && rank == 0) {
      umma_pair_commit_one(smem_u32(drained));
      mbar_wait(drained, 0, g.stall);
    } else if (warp == kWorkers + 1 && lane == 0 && rank == 0) {
      for (int i = 0; i < nst; ++i)
        if (loads > i) mbar_wait(full + i, (uint32_t)((loads - 1 - i) / nst) & 1u, g.stall);
    }
    __syncwarp();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  cluster_sync_all();                                          // the other CTA's products read this one's memory
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// The rows' shares joined: 32 rows a CTA, 32 shares side by side
struct RowsArgs {
  const float *pm, *ps, *pw, *xy;
  const int64_t* y;
  int64_t ignore, V;
  float *logp, *entropy, *lse;
  float2* row;
  int T, parts;
  float c;
  const float* given;          // null, or an earlier call's lse: rows below `far` are left out
  float far;
  int *first, *next;           // as in HeadArgs, to be made (from 0s), or null
};
constexpr int kAhead = 8;
__global__ void __launch_bounds__(1024) k_head_rows(const __grid_constant__ RowsArgs p) {
  __shared__ float sm[32][33], ss[32][33], sw[32][33];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  int row = blockIdx.x * 32 + lane;
  if (p.first && slice == 0 && row < p.T) {
    const int64_t y = p.y[row];
    if (y >= 0 && y < p.V && y != p.ignore) p.next[row] = atomicExch(p.first + y, row + 1);
  }
  if (p.given && !__syncthreads_or(row < p.T && is_far(p.given, p.y, p.ignore, row, p.far))) return;
  row = blockIdx.x * 32 + slice;                         // (the row that this warp's first lane writes)
  const int64_t y = row < p.T ? p.y[row] : 0;
  const float xy = row < p.T && p.logp && y >= 0 && y < p.V ? p.xy[row] : 0.f;
  row = blockIdx.x * 32 + lane;
  float m = -INFINITY, s = 0.f, w = 0.f;
  auto join = [&](float m2, float s2, float w2) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) {                              // the sums are 0 or NaN
      s += s2;
      return;
    }
    const float d = m - top, d2 = m2 - top, r = ex2(d), r2 = ex2(d2);
    w = (m == -INFINITY ? 0.f : r * fmaf(d, s, w)) + (m2 == -INFINITY ? 0.f : r2 * fmaf(d2, s2, w2));
    s = r * s + r2 * s2;                                 // (a NaN stays)
    m = top;
  };
  if (row < p.T) {
    for (int i0 = slice; i0 < p.parts; i0 += 32 * kAhead) {
      float m2[kAhead], s2[kAhead], w2[kAhead];            // (all on their way at once)
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const bool there = i0 + 32 * k < p.parts;
        const int64_t at = (int64_t)(there ? i0 + 32 * k : i0) * p.T + row;
        m2[k] = p.pm[at], s2[k] = p.ps[at], w2[k] = p.pw[at];
        if (!there) m2[k] = -INFINITY, s2[k] = w2[k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) join(m2[k], s2[k], w2[k]);
    }
  }
  sm[slice][lane] = m, ss[slice][lane] = s, sw[slice][lane] = w;
  __syncthreads();
  // a warp a row, a lane a share
  row = blockIdx.x * 32 + slice;
  m = sm[lane][slice], s = ss[lane][slice], w = sw[lane][slice];
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const float m2 = __shfl_down_sync(~0u, m, o), s2 = __shfl_down_sync(~0u, s, o), w2 = __shfl_down_sync(~0u, w, o);
    join(m2, s2, w2);                                    // (lane 0 meets all shares in their order)
  }
  if (lane == 0 && row < p.T) {
    const bool nothing = m == -INFINITY && s == 0.f;
    const float l2 = log2f(s), y2 = nothing ? -INFINITY : l2;
    if (p.lse) p.lse[row] = nothing ? -INFINITY : (m + l2) * kLn2;
    if (p.entropy) p.entropy[row] = nothing ? 0.f : kLn2 * (l2 - w / s);
    if (p.logp) {
      float l = 0.f;
      if (y < 0 || y >= p.V) l = NAN;
      else if (nothing) l = -INFINITY;
      else l = (fmaf(xy, p.c, -m) - l2) * kLn2;
      p.logp[row] = y == p.ignore ? 0.f : l;
    }
    if (p.row) p.row[row] = make_float2(m, nothing ? 0.f : y2);
  }
}

// G of a piece from logits that were kept: 1024 columns of a row a CTA
struct KeptArgs {
  HeadArgs h;
  const float* x;              // [T][ld_x], from the piece's first column on
  __nv_bfloat16* out;          // [terms][T][ld]
  int64_t ld_x, ld, n;         // n: columns that are there, a multiple of 256 (whole warps)
};
__global__ void __launch_bounds__(256) k_head_kept(const __grid_constant__ KeptArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  const int row = blockIdx.x;
  const int64_t j0 = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
  if (j0 >= p.n) return;
  const RowGrad r = row_grad(p.h, row);
  const float4 in = *reinterpret_cast<const float4*>(p.x + row * p.ld_x + j0);
  float v[4] = {in.x, in.y, in.z, in.w};
  to_gradient<4>(v, r, p.h, p.h.v0 + j0);
  for (int e = 0; e < p.h.terms; ++e) {
    const uint2 w = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    *reinterpret_cast<uint2*>(p.out + ((int64_t)e * p.h.T + row) * p.ld + j0) = w;
    v[0] -= __uint_as_float(w.x << 16), v[1] -= __uint_as_float(w.x & 0xffff0000u);
    v[2] -= __uint_as_float(w.y << 16), v[3] -= __uint_as_float(w.y & 0xffff0000u);
  }
}

// bf16 terms of a matrix, in rows on 16 bytes
struct SplitArgs {
  const void* in;
  __nv_bfloat16* out;          // [terms][rows][ld]
  int64_t rows, D, ld;
  int terms;
};
// (eight neighbours a thread: 30011 x 771 fp32 41 us, a value a thread 94)
template <typename T>
__global__ void __launch_bounds__(256) k_head_split(const __grid_constant__ SplitArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  const int groups = (int)(p.ld / 8);
  const int64_t n = p.rows * groups;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / groups;
    const int c = (int)(i - r * groups) * 8;
    const T* in = static_cast<const T*>(p.in) + r * p.D + c;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < p.D ? (float)in[k] : 0.f;
    for (int e = 0; e < p.terms; ++e) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[k] = pack2(v[2 * k], v[2 * k + 1]);
        v[2 * k] -= __uint_as_float(w[k] << 16);
        v[2 * k + 1] -= __uint_as_float(w[k] & 0xffff0000u);
      }
      *reinterpret_cast<uint4*>(p.out + (e * p.rows + r) * p.ld + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// dx from its shares of k, in order
struct JoinArgs {
  const float* in;             // [splits][n]
  void* out;
  int64_t n, D;
  int splits, out_kind;
  const float* off;            // as in HeadArgs
  const int64_t* y;
  int64_t ignore, V, ld_w;
  const __nv_bfloat16* w;
};
__global__ void __launch_bounds__(256) k_head_join(const __grid_constant__ JoinArgs p) {
  pdl_wait();
  pdl_launch_dependents();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.n; i += (int64_t)gridDim.x * 256) {
    float s = 0.f;
#pragma unroll 16
    for (int e = 0; e < p.splits; ++e) s += p.in[e * p.n + i];
    if (p.off) {
      const int64_t t = i / p.D, y = p.y[t];
      if (y >= 0 && y < p.V && y != p.ignore) s = fmaf(p.off[t], __bfloat162float(p.w[y * p.ld_w + i - t * p.D]), s);
    }
    if (p.out_kind == kF32) static_cast<float*>(p.out)[i] = s;
    else static_cast<__nv_bfloat16*>(p.out)[i] = __float2bfloat16_rn(s);
  }
}

// ---- host side -----------------------------------------------------------------------------------------

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
size_t size_of(int dtype) { return dtype == ASI_BF16 ? 2 : 4; }

asi_status_t check_desc(const asi_head_desc_t* d) {
  if (!d || (d->in_dtype != ASI_F32 && d->in_dtype != ASI_BF16) || (d->dw_dtype != ASI_F32 && d->dw_dtype != d->in_dtype)) return ASI_ERR_INVALID_ARG;
  if (d->rows < 0 || d->vocab < 1 || d->dim < 1 || d->vocab_chunk < 0) return ASI_ERR_INVALID_ARG;
  if (!(d->scale >= 1e-8f && d->scale <= 1e8f) || (d->flags & ~ASI_FLAG_TEST_EXPIRE_WAIT)) return ASI_ERR_INVALID_ARG;
  if (d->rows > ASI_HEAD_MAX_ROWS || d->vocab > ASI_HEAD_MAX_VOCAB || d->dim > ASI_HEAD_MAX_DIM) return ASI_ERR_UNSUPPORTED;
  return ASI_OK;
}

constexpr int64_t kPieceBytes = 128 << 20;               // of G in the workspace, where 1024 columns take no more
constexpr int64_t kJoinRows = 4096;                      // rows of shares of dx beyond dx itself
// Rows (one tile) up to which G goes into a bf16 dw as two terms (17 bits) instead of one.  The roundings of few rows do not average out (9 x 50257 x 768: dw
// 0.0026 off with one, 0.0017 with two, which is its own rounding), and the second product mostly hides behind dw's way out (9 x 50257 x 768 97 us with both;
// 256 x 32000 x 2048 162 -> 169, 256 x 60000 x 1000 185 -> 194; 384 rows 216 -> 240).
constexpr int64_t kFewRows = 256;

struct Layout {
  size_t first, next, part, xy, row, off, xs, ws, g, acc, kept, least, bytes;   // least: without logits that are kept (kept 0: never)
  int64_t ld;                                            // of split operands
  int64_t cols;                                          // of a piece
  int in_terms;
  bool lists;                                            // of each target's rows
  bool split;                                            // operands go through k_head_split
  int64_t acc_rows;
};

Layout layout_of(const asi_head_desc_t* d, bool grad) {
  Layout l = {};
  const int64_t T = d->rows, V = d->vocab, nt = ceil_div(V, kTile), all = nt * kTile;
  l.in_terms = d->in_dtype == ASI_F32 ? 3 : 1;
  l.split = d->in_dtype == ASI_F32 || d->dim % 8 != 0;
  l.ld = (d->dim + 63) / 64 * 64;                        // (rows on 128 bytes: on 16 alone a row of a copy meets two lines, and 1001 x 30011 x 771 fp32 took 794 us instead of 768)
  size_t at = 256;                                       // status word
  auto take = [&](size_t bytes) {
    const size_t a = at;
    at = align_up(at + bytes, 256);
    return a;
  };
  l.lists = grad && T > kFewRows && d->dw_dtype == ASI_BF16;
  if (l.lists) {
    l.first = take((size_t)V * 4);                       // (right behind the status word: cleared with it)
    l.next = take((size_t)T * 4);
  }
  l.part = take((size_t)2 * nt * T * 12);
  l.xy = take((size_t)T * 4);
  l.row = take((size_t)T * 8);
  l.off = take((size_t)T * 4);
  if (l.split) {
    l.xs = take((size_t)l.in_terms * T * l.ld * 2);
    l.ws = take((size_t)l.in_terms * V * l.ld * 2);
  }
  if (grad && T) {
    // bytes of a column of G (dx of fp32 operands comes with dw in fp32; never less than fewer rows take)
    const int64_t col = d->dw_dtype == ASI_F32 ? 6 * T : std::max(2 * T, 4 * std::min(T, kFewRows));
    int64_t most = d->vocab_chunk ? ceil_div(std::min(d->vocab_chunk, V), kTile) * kTile * col : std::max(kPieceBytes, 1024 * col);
    most = std::min(most, all * col);
    l.cols = most / col / kTile * kTile;
    l.cols = ceil_div(nt, ceil_div(all, l.cols)) * kTile;   // pieces of about the same size
    l.g = take((size_t)most);
    l.acc_rows = std::max(T, std::min(64 * T, kJoinRows));
    l.acc = take((size_t)l.acc_rows * d->dim * 4);
  }
  l.least = l.bytes = at;
  // Logits of few rows take no more than a piece of G may: where the workspace has room for them they stay, in fp32, and the third of the
  // four products is spared (the same bits, but for G in bf16 where sums of more than 768 k are not segmented).  9 x 50257 x 768 bf16:
  // 136 us instead of 168; 1001 x 30011 x 771 fp32: 768 instead of 939.
  if (grad && T && !d->vocab_chunk && all * T * 4 <= kPieceBytes) {
    l.kept = take((size_t)(all * T * 4));
    l.bytes = at;
  }
  return l;
}

bool operand_map(CUtensorMap* map, const void* base, int64_t inner, int64_t rows, int64_t ld, int terms, int64_t term_stride, int box_inner, int box_rows,
                 CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
  const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)terms};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)term_stride * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows, 1};
  return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, 3, dims, strides, box, swizzle);
}

// The chunks of a product over K: of one term of either operand 128 k a stage, of more 64 with the pairs of
// terms that matter, small ones first
void set_chunks(HeadProb* p, int64_t K, int a_terms, int b_terms) {
  p->pairs = 0;
  p->a_part = p->b_part = 0;
  auto pair = [&](int a, int b) {
    p->a_part |= (uint32_t)a << (2 * p->pairs);
    p->b_part |= (uint32_t)b << (2 * p->pairs);
    ++p->pairs;
  };
  p->sub = a_terms == 1 && b_terms == 1 ? 2 : 1;
  p->a_terms = a_terms, p->b_terms = b_terms;
  if (p->sub == 2) {
    pair(0, 0), pair(1, 1);
  } else {
    for (int sum = 2; sum >= 0; --sum)
      for (int a = 0; a < a_terms; ++a)
        if (sum - a >= 0 && sum - a < b_terms) pair(a, sum - a);
  }
  p->kc = (int)ceil_div(K, kK * p->sub);
  p->per = p->kc;
  p->splits = 1;
  p->seg_pairs = kSeg, p->whole = kWhole;
}
bool too_long(const HeadProb& p) { return p.per * p.pairs > p.whole; }

template <int kEpi, bool kSegmented, bool kLists>
cudaError_t launch_gemm_as(HeadArgs& g, cudaStream_t st) {
  const size_t smem = 1024 + (size_t)g.nst * g.stage + kWorkers * (kStaged + (kEpi == kGrad && g.terms > 1 ? 0 : g.place));
  const cudaError_t e = opt_in_smem(reinterpret_cast<const void*>(k_head_gemm<kEpi, kSegmented, kLists>), smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * std::min(g.tiles, 74)));    // a pair on each pair of SMs
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_head_gemm<kEpi, kSegmented, kLists>, g);
}

// cycles of a tile's results on their way out, as measured.  (With few tokens a tile of dw is hardly anything else: 5 x 25417 x 366 bf16 took
// 146 us when tiles were shared out by their products alone, 91 so.  128 columns a row at a time, by words that start at sectors, took 117.)
constexpr double kCopiesOut = 6e3, kWordsOut = 24e3;
// Cycles that a tile keeps its pair busy: its products, or its results' way out where that takes longer (it runs under the next one's products)
double tile_cost(const HeadProb& p, bool words) { return std::max(512.0 * p.per * p.pairs, words ? kWordsOut : kCopiesOut); }

// Shares out the tiles of the second product so that all pairs end at about the same time: `few` pairs have had one tile more of the
// first (each worth `ratio` of the second's).
void share_tiles(HeadArgs* g, int pairs) {
  const int tiles1 = g->tiles - g->tiles0, base = g->tiles0 / pairs;
  g->few = g->tiles0 - base * pairs;
  const int rest = pairs - g->few;
  const double ratio = tile_cost(g->p[0], g->p[0].how == kWords) / tile_cost(g->p[1], g->p[1].how == kWords);
  // each_few x few + (each_few + ratio) x rest = tiles1
  const double share = (tiles1 - ratio * rest) / pairs;
  int to_few = share > 0 ? (int)std::lround(share * g->few) : 0;
  if (g->few == 0) to_few = 0;
  to_few = std::min(to_few, tiles1);
  if (rest == 0) to_few = tiles1;
  g->each_few = g->few ? to_few / g->few : 0;
  g->more_few = g->few ? to_few - g->each_few * g->few : 0;
  const int to_rest = tiles1 - to_few;
  g->each_rest = rest ? to_rest / rest : 0;
  g->more_rest = rest ? to_rest - g->each_rest * rest : 0;
}

template <int kEpi, bool kLists = false>
cudaError_t launch_gemm(HeadArgs& g, bool segmented, cudaStream_t st) {
  // Stages of what the larger chunk takes (64 KB for one term of either operand, 96 for three), as many as 192 KB hold, beside a place for
  // each warp's results on their way out.  Chunks of 128 k and not 64 for the issuer's sake: one of 64 took it 560 cycles (waiting 120, four products
  // 270, commit 170) for 512 of products.
  int parts = 0;
  for (int q = 0; q < g.np; ++q) {
    HeadProb& p = g.p[q];
    parts = std::max(parts, (p.a_terms + p.b_terms) * p.sub);
    p.seg = 1 << 30;
    if (segmented && too_long(p)) {
      const int n = std::max(2, (int)ceil_div(p.per * p.pairs, p.seg_pairs));
      p.seg = (int)ceil_div(p.per, n);
    }
  }
  g.stage = parts * kHalf;
  g.nst = std::min<int>(kMaxStages, (192 << 10) / g.stage);   // (two terms by one, alone: 48 KB)
  g.place = kEpi == kGrad && g.terms > 1 ? kStaged / 2 : 0;
  g.tiles0 = g.p[0].mt * g.p[0].nt * g.p[0].splits;
  g.tiles = g.tiles0 + (g.np > 1 ? g.p[1].mt * g.p[1].nt * g.p[1].splits : 0);
  g.few = 0;
  g.each_few = g.more_few = g.each_rest = g.more_rest = 0;
  if (g.np > 1) share_tiles(&g, std::min(g.tiles, 74));
  return segmented ? launch_gemm_as<kEpi, true, kLists>(g, st) : launch_gemm_as<kEpi, false, kLists>(g, st);
}

cudaError_t launch_split(const asi_head_desc_t* d, const Layout& l, const void* in, int64_t rows, void* out, cudaStream_t st) {
  SplitArgs a = {in, static_cast<__nv_bfloat16*>(out), rows, d->dim, l.ld, l.in_terms};
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(rows * (l.ld / 8), 256), 148 * 16));
  return d->in_dtype == ASI_BF16 ? launch_pdl(k_head_split<__nv_bfloat16>, grid, dim3(256), 0, st, a) : launch_pdl(k_head_split<float>, grid, dim3(256), 0, st, a);
}

// How a product's results leave: by copies where their rows lie on 16 bytes and what is added is what is there, in fp32
void set_store(HeadProb* p, int64_t rows, int64_t N) {
  const size_t e = p->out_kind == kF32 ? 4 : 2;
  p->how = kWords;
  if ((p->ld * e) % 16 != 0 || !aligned(p->out, 16) || (p->add && (p->out_kind != kF32 || p->add != p->out))) return;
  const cuuint64_t dims[3] = {(cuuint64_t)N, (cuuint64_t)rows, (cuuint64_t)p->splits};
  const cuuint64_t strides[2] = {(cuuint64_t)p->ld * e, (cuuint64_t)std::max(p->split_stride, p->ld) * e};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / e), 32, 1};
  if (!encode_map(&p->o, e == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, p->out, 3, dims, strides, box)) return;
  p->how = p->add ? kAdd : kCopy;
}

// A call's buffers
struct Call {
  const void *x, *w;
  const int64_t* y;
  float *logp, *entropy, *lse;               // written by the forward direction
  const float *lse_in, *entropy_in, *dlogp, *dent;
  void *dx, *dw;
  bool accumulate, forward, grad;
};

void size_product(HeadProb* p, int64_t M, int64_t N) {
  p->M = (int)M;
  p->N = (int)N;
  p->mt = (int)ceil_div(M, kTile);
  p->nt = (int)ceil_div(N, kTile);
}

asi_status_t run(const asi_head_desc_t* d, const Call& c, char* ws, size_t ws_bytes, cudaStream_t st) {
  const Layout l = layout_of(d, c.grad);
  const int64_t T = d->rows, V = d->vocab, D = d->dim;
  const bool fine = d->in_dtype == ASI_F32;              // logits and dx are held to fp32
  int* status = reinterpret_cast<int*>(ws);
  const bool lists = l.lists && c.dw;
  cudaError_t e = cudaMemsetAsync(status, 0, lists ? l.first + (size_t)V * 4 : 4, st);
  if (e != cudaSuccess) return cuda_status(e, "output layer's status");
  const void *x = c.x, *w = c.w;
  int64_t ld = D;
  if (l.split) {
    e = launch_split(d, l, c.x, T, ws + l.xs, st);
    if (e == cudaSuccess) e = launch_split(d, l, c.w, V, ws + l.ws, st);
    if (e != cudaSuccess) return cuda_status(e, "terms of the output layer's operands");
    x = ws + l.xs, w = ws + l.ws, ld = l.ld;
  }
  HeadArgs g = {};
  g.status = status;
  g.stall = (d->flags & ASI_FLAG_TEST_EXPIRE_WAIT) != 0;
  g.y = c.y;
  g.ignore = d->ignore_index;
  g.V = V;
  g.T = (int)T;
  g.scale = d->scale;
  g.c = (float)(d->scale * 1.4426950408889634);
  const int64_t nt = ceil_div(V, kTile);
  g.pm = reinterpret_cast<float*>(ws + l.part);
  g.ps = g.pm + 2 * nt * T;
  g.pw = g.ps + 2 * nt * T;
  g.xy = reinterpret_cast<float*>(ws + l.xy);
  float2* row = reinterpret_cast<float2*>(ws + l.row);
  // the logits' product: whole, then in pieces
  HeadProb logits = {};
  size_product(&logits, T, V);
  set_chunks(&logits, D, l.in_terms, l.in_terms);
  if (!operand_map(&logits.a, x, D, T, ld, l.in_terms, T * ld, kK, 128) || !operand_map(&logits.b, w, D, V, ld, l.in_terms, V * ld, kK, 128))
    return cuda_status(cudaErrorNotSupported, "tensor map");
  const bool keep = c.forward && c.grad && l.kept && ws_bytes >= l.bytes;
  // of G (bf16 operands: what dw wants)
  const int terms = fine || (c.dw && d->dw_dtype == ASI_F32) ? 3 : c.dw && T <= kFewRows ? 2 : 1;
  if (!c.forward) {
    g.lse = c.lse_in;
    g.far = terms > 1 ? kFarLseTerms : kFarLse;
  }
  g.p[0] = logits;
  g.np = 1;
  if (keep) {
    g.p[0].out = ws + l.kept;
    g.p[0].out_kind = kF32;
    g.p[0].ld = nt * kTile;
    set_store(&g.p[0], T, nt * kTile);
    if (g.p[0].how != kCopy) return cuda_status(cudaErrorNotSupported, "tensor map");
  }
  e = launch_gemm<kStats>(g, too_long(logits), st);
  if (e != cudaSuccess) return cuda_status(e, "logits of the output layer");
  const RowsArgs r = {g.pm, g.ps, g.pw, g.xy, c.y, d->ignore_index, V, c.logp, c.entropy, c.lse, row, (int)T, (int)(2 * nt), g.c, g.lse, g.far,
                      lists ? reinterpret_cast<int*>(ws + l.first) : nullptr, reinterpret_cast<int*>(ws + l.next)};
  e = launch_pdl(k_head_rows, dim3((unsigned)ceil_div(T, 32)), dim3(1024), 0, st, r);
  if (e != cudaSuccess) return cuda_status(e, "rows of the output layer");
  if (!c.grad) return ASI_OK;
  g.row = row;
  g.entropy = c.entropy_in;
  g.dlogp = c.dlogp;
  g.dent = c.dent;
  g.terms = terms;
  g.off = (!fine && c.dx) || lists ? reinterpret_cast<float*>(ws + l.off) : nullptr;
  g.first = reinterpret_cast<const int*>(ws + l.first);
  g.next = reinterpret_cast<const int*>(ws + l.next);
  g.w = static_cast<const __nv_bfloat16*>(w);
  g.x = static_cast<const __nv_bfloat16*>(x);
  g.ld_w = ld;
  void* G = ws + l.g;
  HeadProb px = {}, pw = {};
  if (!operand_map(&g.g, G, l.cols, T, l.cols, terms, T * l.cols, terms == 1 ? 64 : 32, 32, terms == 1 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B))
    return cuda_status(cudaErrorNotSupported, "tensor map");
  const int64_t pieces = ceil_div(V, l.cols);
  const int dx_kind = d->in_dtype == ASI_BF16 ? kB16 : kF32, dw_kind = d->dw_dtype == ASI_BF16 ? kB16 : kF32;
  float* acc = reinterpret_cast<float*>(ws + l.acc);
  int splits = 1;
  for (int64_t i = 0; i < pieces; ++i) {
    const int64_t v0 = i * l.cols, nv = std::min(V - v0, l.cols);
    g.p[0] = logits;
    g.p[0].N = (int)nv;
    g.p[0].nt = (int)ceil_div(nv, kTile);
    g.p[0].b_off = (int)v0;
    g.np = 1;
    g.v0 = v0;
    if (keep) {
      const int64_t n = ceil_div(nv, kTile) * kTile;
      const KeptArgs k = {g, reinterpret_cast<const float*>(ws + l.kept) + v0, static_cast<__nv_bfloat16*>(G), nt * kTile, l.cols, n};
      e = launch_pdl(k_head_kept, dim3((unsigned)T, (unsigned)ceil_div(n, 1024)), dim3(256), 0, st, k);
    } else {
      // G in terms (24 bits) wants logits summed as those behind lse.  To G in bf16, whose step is 2^-9, what truncation takes from a logit
      // (about 1e-5 at D = 2048) is nothing, and summing them in segments costs 4096 x 32000 x 2048 2 % (1451 us -> 1483)
      e = launch_gemm<kGrad>(g, terms > 1 && too_long(logits), st);
    }
    if (e != cudaSuccess) return cuda_status(e, "gradient of the logits");
    // (the first operand lies with k together for dx, with its rows together for dw; x and w with their rows together)
    size_product(&px, T, D);
    set_chunks(&px, nv, fine ? 3 : 1, fine ? 3 : 1);
    if (!fine) px.seg_pairs = kSegB16, px.whole = kWholeB16;
    px.a_mn = 0, px.b_mn = 1, px.b_k = (int)v0, px.n_first = 1;
    size_product(&pw, nv, D);
    set_chunks(&pw, T, terms, l.in_terms);
    if (dw_kind == kB16) pw.seg_pairs = kSegB16, pw.whole = kWholeB16;
    pw.a_mn = 1, pw.b_mn = 1, pw.n_first = 1;
    if (i == 0) {
      bool maps = operand_map(&px.a, G, l.cols, T, l.cols, terms, T * l.cols, kK, 128) && operand_map(&px.b, w, D, V, ld, l.in_terms, V * ld, 64, kK * px.sub);
      maps = maps && operand_map(&pw.a, G, l.cols, T, l.cols, terms, T * l.cols, 64, kK * pw.sub) && operand_map(&pw.b, x, D, T, ld, l.in_terms, T * ld, 64, kK * pw.sub);
      if (!maps) return cuda_status(cudaErrorNotSupported, "tensor map");
    }
    pw.ld = D;
    pw.out = static_cast<char*>(c.dw) + v0 * D * size_of(d->dw_dtype);
    pw.out_kind = dw_kind;
    pw.add = c.accumulate ? pw.out : nullptr;
    pw.add_kind = c.accumulate ? dw_kind : kNone;
    if (i == 0) {
      // few tiles of dx: shares of k, about half of what a pair has to do in all (eight chunks at least)
      const double each = 512.0 * px.pairs, tw = c.dw ? (double)pw.mt * pw.nt * tile_cost(pw, D * size_of(d->dw_dtype) % 16 != 0) : 0.0;
      const double load = ((double)px.mt * px.nt * px.kc * each + tw) / 74;
      const int64_t share = std::max<int64_t>((int64_t)(load / 2 / each), 8);
      splits = (int)std::max<int64_t>(1, std::min({ceil_div(px.kc, share), l.acc_rows / T, (int64_t)64}));
    }
    px.per = (int)ceil_div(px.kc, splits);
    px.splits = splits;
    px.split_stride = T * D;
    px.ld = D;
    const bool last = i + 1 == pieces && splits == 1;
    px.add = i ? acc : nullptr;
    px.add_kind = i ? kF32 : kNone;
    px.out = last ? c.dx : static_cast<void*>(acc);
    px.out_kind = last ? dx_kind : kF32;
    px.correct = last && !fine ? kToDx : kNowhere;
    pw.correct = lists ? kToDw : kNowhere;
    g.np = 0;
    if (c.dx) g.p[g.np++] = px;
    if (c.dw) g.p[g.np++] = pw;
    for (int q = 0; q < g.np; ++q) set_store(&g.p[q], g.p[q].M, D);
    // (sums that leave TMEM on the way)
    const bool segmented = (c.dw && too_long(pw)) || (c.dx && too_long(px));
    e = lists ? launch_gemm<kOut, true>(g, segmented, st) : launch_gemm<kOut>(g, segmented, st);
    if (e != cudaSuccess) return cuda_status(e, "gradients of the output layer");
  }
  if (c.dx && splits > 1) {
    const JoinArgs j = {acc, c.dx, T * D, D, splits, dx_kind, fine ? nullptr : g.off, c.y, d->ignore_index, V, ld, g.w};
    e = launch_pdl(k_head_join, dim3((unsigned)std::min<int64_t>(ceil_div(T * D, 256), 148 * 8)), dim3(256), 0, st, j);
    if (e != cudaSuccess) return cuda_status(e, "shares of dx");
  }
  return ASI_OK;
}

// A contiguous buffer of a call; null where the call has none
struct Span {
  const void* p;
  size_t bytes;
  size_t element;
  bool meets(const Span& o) const {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
    return p && o.p && a < b + o.bytes && b < a + bytes;
  }
};

asi_status_t check_buffers(std::initializer_list<Span> in, std::initializer_list<Span> out) {
  for (const auto* list : {&in, &out})
    for (const Span& s : *list)
      if (s.p && off_element(s.p, s.element)) return ASI_ERR_INVALID_ARG;
  for (const Span* o = out.begin(); o != out.end(); ++o) {
    for (const Span* q = out.begin(); q != o; ++q)
      if (o->meets(*q)) return ASI_ERR_INVALID_ARG;
    for (const Span& i : in)
      if (o->meets(i)) return ASI_ERR_INVALID_ARG;
  }
  return ASI_OK;
}

asi_status_t check_call(const asi_head_desc_t* d, const Call& c, void* ws, size_t ws_bytes) {
  if (!c.x || !c.w || !c.y || !ws) return ASI_ERR_INVALID_ARG;
  if (c.forward && (!c.logp || !c.lse)) return ASI_ERR_INVALID_ARG;
  if (c.grad && (!c.dlogp || (!c.dx && !c.dw) || (!c.forward && !c.lse_in) || (c.dent && !c.entropy_in))) return ASI_ERR_INVALID_ARG;
  const Layout l = layout_of(d, c.grad);
  if (ws_bytes < l.least || !aligned(ws, 256)) return ASI_ERR_WORKSPACE;
  if (!l.split && (!aligned(c.x, 16) || !aligned(c.w, 16))) return ASI_ERR_INVALID_ARG;
  const size_t T = (size_t)d->rows, e = size_of(d->in_dtype), n = T * 4;
  const bool in_rows = c.grad && !c.forward;
  return check_buffers({{c.x, T * d->dim * e, e}, {c.w, (size_t)d->vocab * d->dim * e, e}, {c.y, T * 8, 8}, {c.dlogp, n, 4}, {c.dent, n, 4},
                        {in_rows ? c.lse_in : nullptr, n, 4}, {in_rows ? c.entropy_in : nullptr, n, 4}},
                       {{c.logp, n, 4}, {c.entropy, n, 4}, {c.lse, n, 4}, {c.dx, T * d->dim * e, e},
                        {c.dw, (size_t)d->vocab * d->dim * size_of(d->dw_dtype), size_of(d->dw_dtype)}, {ws, std::min(ws_bytes, l.bytes), 256}});
}

asi_status_t call(const asi_head_desc_t* d, const Call& c, void* ws, size_t ws_bytes, void* stream) {
  asi_status_t s = check_desc(d);
  if (s != ASI_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (d->rows == 0) {
    if (c.grad && c.dw && !c.accumulate && off_element(c.dw, size_of(d->dw_dtype))) return ASI_ERR_INVALID_ARG;
    if (ws && ws_bytes >= 4 && aligned(ws, 4)) {           // (a workspace may be missing here)
      const cudaError_t e = cudaMemsetAsync(ws, 0, 4, st);
      if (e != cudaSuccess) return cuda_status(e, "output layer's status");
    }
    if (!c.grad || !c.dw || c.accumulate) return ASI_OK;   // no rows: their gradient of w is 0
    return cuda_status(cudaMemsetAsync(c.dw, 0, (size_t)d->vocab * d->dim * size_of(d->dw_dtype), st), "gradient of no rows");
  }
  s = check_call(d, c, ws, ws_bytes);
  if (s != ASI_OK) return s;
  try {
    return run(d, c, static_cast<char*>(ws), ws_bytes, st);
  } catch (...) {
    return no_host_memory();
  }
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" {

size_t asi_head_ws_bytes(const asi_head_desc_t* desc, int32_t grad) { return check_desc(desc) == ASI_OK ? layout_of(desc, grad != 0).bytes : 0; }

asi_status_t asi_head_logprobs(const asi_head_desc_t* desc, const void* x, const void* w, const int64_t* targets, float* logp,
                               float* entropy, float* lse, void* ws, size_t ws_bytes, void* stream) {
  Call c = {};
  c.x = x, c.w = w, c.y = targets, c.logp = logp, c.entropy = entropy, c.lse = lse, c.forward = true;
  return call(desc, c, ws, ws_bytes, stream);
}

asi_status_t asi_head_grad(const asi_head_desc_t* desc, const void* x, const void* w, const int64_t* targets, const float* lse,
                           const float* entropy, const float* dlogp, const float* dentropy, void* dx, void* dw, int32_t accumulate,
                           void* ws, size_t ws_bytes, void* stream) {
  Call c = {};
  c.x = x, c.w = w, c.y = targets, c.lse_in = lse, c.entropy_in = entropy, c.dlogp = dlogp, c.dent = dentropy;
  c.dx = dx, c.dw = dw, c.accumulate = accumulate != 0, c.grad = true;
  return call(desc, c, ws, ws_bytes, stream);
}

asi_status_t asi_head_loss(const asi_head_desc_t* desc, const void* x, const void* w, const int64_t* targets, const float* dlogp,
                           const float* dentropy, float* logp, float* entropy, float* lse, void* dx, void* dw, int32_t accumulate,
                           void* ws, size_t ws_bytes, void* stream) {
  Call c = {};
  c.x = x, c.w = w, c.y = targets, c.logp = logp, c.entropy = entropy, c.lse = lse, c.dlogp = dlogp, c.dent = dentropy;
  c.entropy_in = entropy, c.dx = dx, c.dw = dw, c.accumulate = accumulate != 0, c.forward = c.grad = true;
  return call(desc, c, ws, ws_bytes, stream);
}

asi_status_t asi_head_status(const void* ws, void* stream, asi_status_t* device_status) {
  if (!ws || !device_status) return ASI_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int v = 0;
  cudaError_t e = cudaMemcpyAsync(&v, ws, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return cuda_status(e, "status of the output layer");
  *device_status = static_cast<asi_status_t>(v);
  return ASI_OK;
}

}  // extern "C"
