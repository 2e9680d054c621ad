// What stands between the layers: the residual's addition with the root-mean-square norm in front of a layer, the gated
// activation in front of a down projection, and the reading back of MXINT activations.  (The paper's Section 2.1 leaves the
// activations between the layers quantised in the w&a setting; Section 4.1: MXINT, blocks [1, 16].)
//
// All three are one pass over their tensors: a lane holds eight consecutive elements (16 bytes of bf16), a 16-block is two
// neighbouring lanes, and nothing but the result goes back to memory.
//
// MXINT outputs are those of 64-bit arithmetic, bit for bit.  The values are computed in fp32 with a known bound on their relative
// error; a block whose exponent or one of whose mantissas could fall on the other side of a border within that bound is decided
// again from fp64 values.  About one warp in thirty goes that way, so fp64 throughput does not matter.
// What it costs beside that is instructions, so two elements share one where they can.
//
// Measured, and what bounds them.  Norm with residual, 2048 x 4096 bf16 to MXINT8: 12.8 us, 4.6 TB/s (to bf16 12.7); 59 % of the issue slots are
// taken, memory a third: its 24 warps an SM wait for fixed latencies and for the barrier of each row, and 2048 rows are five turns of 444 CTAs
// for 4.6.  4096 x 5120 to bf16: 27.7 us, 6.1 TB/s.  Gate, 2048 x 11008 bf16 to MXINT8: SiLU 26.2 us, 4.4 TB/s, 64 % of the issue slots
// (the exponential, the borders), GELU 32.5; of fp32 34.5 and 36.4, 5.9 TB/s; bf16 to bf16 23.8 us with either, 5.7 TB/s; fp32 2048 x 13824 to
// fp32 55 us, 6.2 TB/s.  MXINT8 to bf16, 2048 x 11008: 12.0 us, 5.7 TB/s, memory.  One row of the first two: 2.2 and 1.4 us, a launch and a trip to memory.
#include "lqer_tc_ptx.cuh"

namespace lqer {
namespace bd {

// Eight consecutive elements of an fp32 or bf16 tensor as they lie in memory, and as values.
template <bool BF16>
struct Raw {
  uint4 a, b;               // bf16: a only
  __device__ __forceinline__ void load(const void* p, size_t idx) {
    if (BF16) {
      a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + idx);
    } else {
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + idx);
      a = q[0];
      b = q[1];
    }
  }
  __device__ __forceinline__ void clear() { a = b = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < (BF16 ? 4 : 8); ++i) {
      if (BF16) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        v[i] = __uint_as_float(w[i]);
      }
    }
  }
};
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, size_t idx, float (&v)[8]) {
  Raw<BF16> r;
  r.load(p, idx);
  r.values(v);
}
// Two fp32 values rounded to nearest even bf16 (low half: the first).
__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
template <bool BF16>
__device__ __forceinline__ void store8(void* p, size_t idx, const float (&v)[8]) {
  if (BF16) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + idx) =
        make_uint4(round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]), round_bf16x2(v[4], v[5]), round_bf16x2(v[6], v[7]));
  } else {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + idx);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}
// 32 bytes, a whole sector, in one access.
__device__ __forceinline__ void store32(void* p, const uint32_t (&u)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]) : "memory");
}
// Two fp32 operations in one instruction.
struct F2 { unsigned long long w; };
__device__ __forceinline__ F2 f2(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.w) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unf2(F2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v.w)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.w) : "l"(a.w), "l"(b.w), "l"(c.w)); return r; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w)); return r; }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

// One of eight registers by a running index, without an array in memory.
__device__ __forceinline__ float pick8(const float (&v)[8], int i) {
  float r = v[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) r = i == k ? v[k] : r;
  return r;
}

// Quantises the eight values of a lane; lanes 2 i and 2 i + 1 share a block.  Every lane of the warp takes part.
// rel: bound on the relative error of the lane's values; wide(i): the same value in fp64.  A mantissa is in doubt where the scaled value
// lies within its error of a half; it is then decided from wide(i).  Where the block's maximum lies within its error of a
// power of two, or a value is NaN or infinite, the whole octet is.  That way is rolled up: it is rare, and the ordinary one
// should keep its registers.
template <class Wide>
__device__ __forceinline__ void quantise8(const float (&v)[8], const QuantConsts& c, float rel, Wide wide, uint2& m8, int& e) {
  float amax = 0.f;                                  // fmaxf drops a NaN operand: NaN counts as zero
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
  amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
  const uint32_t top = __float_as_uint(fmaf(amax, rel, amax)), low = __float_as_uint(fmaf(amax, -rel, amax));
  e = min(max((int)(top >> 23) - 127, c.emin), c.emax);
  bool hard = (top ^ low) >= 0x00800000u;            // another exponent
  const float inv_step = pow2f(c.shift - e), kRound = 12582912.0f;       // 1.5 * 2^23, see quantize_quad
  const float largest = amax * inv_step;
  const float sure = fmaf(largest, -rel, 0.4999995f);                    // a scaled value up to this far from an integer rounds to it
  const F2 inv2 = f2(inv_step, inv_step), round2 = f2(kRound, kRound), minus2 = f2(-1.f, -1.f);
  float s[8], d[8], far = 0.f;                       // far: the largest distance to the chosen integer
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const F2 v2 = f2(v[i], v[i + 1]);
    const F2 s2 = fma2(v2, inv2, round2);            // exact scaling, one rounding: to the integer
    const F2 d2 = fma2(v2, inv2, fma2(s2, minus2, round2));
    unf2(s2, s[i], s[i + 1]);
    unf2(d2, d[i], d[i + 1]);
    far = max_nan(far, max_nan(fabsf(d[i]), fabsf(d[i + 1])));
  }
  const bool doubt = !(far <= sure);
  if (largest >= c.qlim) {                           // may round past the symmetric range, or lie far beyond it
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = fminf(fmaxf(s[i], kRound - c.qmax), kRound + c.qmax);
    hard = hard || !(largest < 4194304.f);           // the rounding trick has a limit
  }
  m8.x = __byte_perm(__byte_perm(__float_as_uint(s[0]), __float_as_uint(s[1]), 0x0040),
                     __byte_perm(__float_as_uint(s[2]), __float_as_uint(s[3]), 0x0040), 0x5410);
  m8.y = __byte_perm(__byte_perm(__float_as_uint(s[4]), __float_as_uint(s[5]), 0x0040),
                     __byte_perm(__float_as_uint(s[6]), __float_as_uint(s[7]), 0x0040), 0x5410);
  if (!__any_sync(0xFFFFFFFFu, hard || doubt)) return;
  unsigned long long m = (unsigned long long)m8.y << 32 | m8.x;
  unsigned mine = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) mine |= !(fabsf(d[i]) <= sure) ? 1u << i : 0u;
  if (__any_sync(0xFFFFFFFFu, hard || far != far)) {
    double big = 0.0;
#pragma unroll 1
    for (int i = 0; i < 8; ++i) big = fmax(big, fabs(wide(i)));
    big = fmax(big, __shfl_xor_sync(0xFFFFFFFFu, big, 1));
    e = block_exponent(big, c.emin, c.emax);
    mine = 0xFFu;
  }
#pragma unroll 1
  for (unsigned left = __reduce_or_sync(0xFFFFFFFFu, mine); left != 0; left &= left - 1) {
    const int i = __ffs(left) - 1;
    if ((mine >> i) & 1u) m = (m & ~(0xFFull << (8 * i))) | (unsigned long long)((uint32_t)quant_mantissa(wide(i), e, c.shift + 2) & 0xFFu) << (8 * i);
  }
  m8 = make_uint2((uint32_t)m, (uint32_t)(m >> 32));
}

// The lane's octet at idx (K is a multiple of 16: a block's exponent lies at its first element's place / 16).
__device__ __forceinline__ void store_mxint8(void* Ym, uint8_t* Ye, size_t idx, const uint2& m8, int e) {
  *reinterpret_cast<uint2*>(static_cast<int8_t*>(Ym) + idx) = m8;
  if ((idx & 8) == 0) Ye[idx >> 4] = (uint8_t)(e + 127);
}

struct Format { int bits, emin, emax; };

// ---------------------------------------------------------------------------- norm
struct NormParams {
  const void* X;
  const void* res;          // may be null
  void* res_out;            // may be null; may be res, or X if the types agree
  const void* w;
  void* Y;
  uint8_t* Ye;              // an MXINT8 result's exponents
  double eps, inv_k;        // inv_k: 1 / K
  int M, K;
  int w_bf16;
  Format f;
};
template <bool XB, bool RB>
struct RawRow {              // a lane's octet of X and of the residual
  Raw<XB> x;
  Raw<RB> r;
  __device__ __forceinline__ void load(const NormParams& p, size_t idx) {
    x.load(p.X, idx);
    if (p.res != nullptr) r.load(p.res, idx);
  }
  // the residual stream's value h: x + res in fp32, rounded to the stream's type (what a later reader of it sees)
  // (two bf16 values add up exactly in fp32, or differ by more than bf16 can show: one rounding to bf16 is the same)
  __device__ __forceinline__ void sum(const NormParams& p, float (&h)[8]) const {
    if constexpr (XB && RB) {
      Raw<true> t = x;
      if (p.res != nullptr) {
        uint32_t* w[4] = {&t.a.x, &t.a.y, &t.a.z, &t.a.w};
        const uint32_t o[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(*w[i]) : "r"(*w[i]), "r"(o[i]));
      }
      t.values(h);
    } else {
      x.values(h);
      if (p.res != nullptr) {
        float v[8];
        r.values(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += v[i];
      }
      if (RB) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const uint32_t u = round_bf16x2(h[i], h[i + 1]);
          h[i] = __uint_as_float(u << 16);
          h[i + 1] = __uint_as_float(u & 0xFFFF0000u);
        }
      }
    }
  }
};
// h * inv * w in fp64, rounded to 48 bits.  Borders have nine, so a value that lies on one exactly (rows of one magnitude, eps 0) gets back on it,
// from which the inverse root, a unit or two off, and the products have taken it; none gets across.
__device__ __forceinline__ double norm_wide(float h, double inv, float w) {
  return __longlong_as_double((__double_as_longlong((double)h * inv * (double)w) + 16) & ~31LL);
}
// One row's octet of Y.  Bound on the fp32 values' error: the inverse root, its product with h and the product with w are
// rounded once each, 3 * 2^-24 < 2^-22; an inverse root near the end of fp32's range has no such bound.
template <int YT>
__device__ __forceinline__ void finish8(const NormParams& p, size_t idx, bool in, const float (&h)[8], const float (&w)[8], float inv,
                                        double inv64, const QuantConsts& qc) {
  float v[8];
  const F2 inv2 = f2(inv, inv);
#pragma unroll
  for (int i = 0; i < 8; i += 2) unf2(mul2(mul2(f2(h[i], h[i + 1]), inv2), f2(w[i], w[i + 1])), v[i], v[i + 1]);
  if (YT == kYMXINT8) {
    uint2 m8;
    int e;
    quantise8(v, qc, inv > 1e-30f ? 2.3841858e-7f : 1.0f, [&](int i) { return norm_wide(pick8(h, i), inv64, pick8(w, i)); }, m8, e);
    if (in) store_mxint8(p.Y, p.Ye, idx, m8, e);
  } else {
    if (!(inv > 1e-37f && inv < 1e37f)) {             // the whole row's; not a normal fp32 number
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)((double)h[i] * inv64 * (double)w[i]);
    }
    if (in) store8<YT == kYBF16>(p.Y, idx, v);
  }
}
// The sum over the CTA, in every thread: warps first, then one value a warp.  Two calls in a row need two sets of slots.
__device__ __forceinline__ double cta_sum(double s, double* slots) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (warps == 1) return s;
  if (lane == 0) slots[threadIdx.x >> 5] = s;
  __syncthreads();
  s = lane < warps ? slots[lane] : 0.0;
  if (warps > 8) {
    s += __shfl_xor_sync(0xFFFFFFFFu, s, 16);
    s += __shfl_xor_sync(0xFFFFFFFFu, s, 8);
  } else {
    s = __shfl_sync(0xFFFFFFFFu, s, lane & 7);
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return s;
}
// 1 / sqrt(a), good to fp64: the reciprocal root of fp32 and two Newton steps, or, outside fp32's range, the library's.
__device__ __forceinline__ double inverse_root(double a) {
  if (!(a > 1e-30 && a < 1e30)) return 1.0 / sqrt(a);
  double y = (double)rsqrtf((float)a);
  y = fma(y, fma(-0.5 * a * y, y, 0.5), y);
  return fma(y, fma(-0.5 * a * y, y, 0.5), y);
}
__device__ __forceinline__ void load_w(const NormParams& p, int col, float (&w)[8]) {
  if (p.w_bf16) load8<true>(p.w, col, w);
  else load8<false>(p.w, col, w);
}
__device__ __forceinline__ void zero8(float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
}
// A CTA takes a row at a time, in registers: OPT octets a thread.  Up to 8192 columns (16384 of bf16) the next row's elements are on their
// way while this row's sum is formed and its results are written (AHEAD); a thread then holds two octets and their weights (bf16) or
// one.  The sum of squares is kept in fp64: it makes the row's factor good to fp64 (the MXINT borders need that) and holds
// squares that fp32 cannot.
// CTAs that are to fit an SM: two octets a thread, their weights and what comes next take 80 registers, four octets and what comes next
// 128, the other forms 64.
__host__ __device__ constexpr int norm_ctas(int threads, int opt, bool ahead) {
  return !ahead || opt == 1 ? 1024 / threads : opt == 2 ? 768 / threads : 1;
}
template <bool XB, bool RB, int YT, int OPT, bool AHEAD, int THREADS>
__global__ void __launch_bounds__(THREADS, norm_ctas(THREADS, OPT, AHEAD)) add_rms_norm_kernel(const NormParams p) {
  __shared__ double slots[2][THREADS / 32];
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const QuantConsts qc = quant_consts(p.f.bits, p.f.emin, p.f.emax);
  const int step = blockDim.x * 8, col0 = threadIdx.x * 8;
  bool in[OPT];
#pragma unroll
  for (int o = 0; o < OPT; ++o) in[o] = col0 + o * step < p.K;
  RawRow<XB, RB> raw[AHEAD ? OPT : 1];
  size_t idx = (size_t)blockIdx.x * p.K + col0;
  const size_t hop = (size_t)gridDim.x * p.K;
  constexpr bool KEEP = AHEAD && OPT == 2;            // the weights stay in registers
  float w[KEEP ? OPT : 1][8];
  if (AHEAD) {
#pragma unroll
    for (int o = 0; o < OPT; ++o) {
      raw[o].x.clear();
      raw[o].r.clear();
      if (in[o]) raw[o].load(p, idx + o * step);
      if (KEEP) load_w(p, in[o] ? col0 + o * step : 0, w[o]);
    }
  }
  int turn = 0;
  for (int row = blockIdx.x; row < p.M; row += gridDim.x, idx += hop, turn ^= 1) {
    float h[OPT][8];
    double sum = 0.0;
    const bool more = row + (int)gridDim.x < p.M;
#pragma unroll
    for (int o = 0; o < OPT; ++o) {
      RawRow<XB, RB>& r = raw[AHEAD ? o : 0];
      if (!AHEAD) {
        r.x.clear();
        r.r.clear();
        if (in[o]) r.load(p, idx + o * step);
      }
      r.sum(p, h[o]);
      if (AHEAD && in[o] && more) r.load(p, idx + hop + o * step);
    }
#pragma unroll
    for (int o = 0; o < OPT; ++o) {
      if (p.res_out != nullptr && in[o]) store8<RB>(p.res_out, idx + o * step, h[o]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)h[o][i], (double)h[o][i], sum);
    }
    sum = cta_sum(sum, slots[turn]);
    const double inv64 = inverse_root(fma(sum, p.inv_k, p.eps));
    const float inv = (float)inv64;
#pragma unroll
    for (int o = 0; o < OPT; ++o) {
      if (!KEEP) load_w(p, in[o] ? col0 + o * step : 0, w[0]);              // again for every row: from L1
      finish8<YT>(p, idx + o * step, in[o], h[o], w[KEEP ? o : 0], inv, inv64, qc);
    }
  }
}
// Rows too long for the registers: h is formed twice, the second time from the residual stream where that was written (it may have
// replaced one of the summands; a thread reads what it wrote itself).
template <bool XB, bool RB, int YT>
__global__ void __launch_bounds__(1024) add_rms_norm_long_kernel(const NormParams p) {
  __shared__ double slots[32];
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const size_t row = blockIdx.x;
  double sum = 0.0;
  for (int col = threadIdx.x * 8; col < p.K; col += blockDim.x * 8) {
    RawRow<XB, RB> raw;
    float h[8];
    raw.load(p, row * p.K + col);
    raw.sum(p, h);
    if (p.res_out != nullptr) store8<RB>(p.res_out, row * p.K + col, h);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma((double)h[i], (double)h[i], sum);
  }
  sum = cta_sum(sum, slots);
  const double inv64 = inverse_root(fma(sum, p.inv_k, p.eps));
  const float inv = (float)inv64;
  const QuantConsts qc = quant_consts(p.f.bits, p.f.emin, p.f.emax);
  for (int at = 0; at < p.K; at += blockDim.x * 8) {            // whole warps, for the blocks' maxima
    const int col = at + threadIdx.x * 8;
    const bool in = col < p.K;
    float h[8], w[8];
    zero8(h);
    zero8(w);
    if (in) {
      if (p.res_out != nullptr) {
        load8<RB>(p.res_out, row * p.K + col, h);
      } else {
        RawRow<XB, RB> raw;
        raw.load(p, row * p.K + col);
        raw.sum(p, h);
      }
      load_w(p, col, w);
    }
    finish8<YT>(p, row * p.K + col, in, h, w, inv, inv64, qc);
  }
}

// Launches with the programmatic attribute: the kernels wait for their predecessor before they touch memory.
template <class... P, class... A>
static cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <bool XB, bool RB, int YT>
static cudaError_t launch_norm(const NormParams& p, cudaStream_t s) {
  const int octets = p.K / 8;
  LaunchScope scope(kFamQuantize, s);
  if (octets > 4096) return launch_after(add_rms_norm_long_kernel<XB, RB, YT>, dim3(p.M), 1024, s, p);
  constexpr int AHEAD_OPT = XB && RB ? 2 : 1, LONG = 4;
  const bool ahead = octets <= 1024, ahead_long = !ahead && XB && RB && octets <= 2048;
  const int opt = ahead ? AHEAD_OPT : LONG;
  const int threads = ((octets + opt - 1) / opt + 31) / 32 * 32;
  // as many CTAs as are resident
  const int room = ahead && opt == 2 ? 768 : ahead_long ? 512 : 1024, per = threads <= 64 ? 12 : threads > room ? 1 : room / threads;
  const int resident = sm_count() * per, grid = p.M < resident ? p.M : resident;
  if constexpr (XB && RB)
    if (ahead_long) return launch_after(add_rms_norm_kernel<XB, RB, YT, LONG, true, 512>, dim3(grid), threads, s, p);
  if (!ahead) return launch_after(add_rms_norm_kernel<XB, RB, YT, LONG, false, 1024>, dim3(grid), threads, s, p);
  constexpr int MOST = AHEAD_OPT == 2 ? 512 : 1024, MIDDLE = AHEAD_OPT == 2 ? 384 : 512;
  return threads <= 256      ? launch_after(add_rms_norm_kernel<XB, RB, YT, AHEAD_OPT, true, 256>, dim3(grid), threads, s, p)
         : threads <= MIDDLE ? launch_after(add_rms_norm_kernel<XB, RB, YT, AHEAD_OPT, true, MIDDLE>, dim3(grid), threads, s, p)
                             : launch_after(add_rms_norm_kernel<XB, RB, YT, AHEAD_OPT, true, MOST>, dim3(grid), threads, s, p);
}
template <bool XB, bool RB>
static cudaError_t launch_norm_y(const NormParams& p, int y_type, cudaStream_t s) {
  return y_type == kYF32    ? launch_norm<XB, RB, kYF32>(p, s)
         : y_type == kYBF16 ? launch_norm<XB, RB, kYBF16>(p, s)
                            : launch_norm<XB, RB, kYMXINT8>(p, s);
}

// ---------------------------------------------------------------------------- gated activation
struct GateParams {
  const void* gate;
  const void* up;
  void* Y;
  uint8_t* Ye;              // an MXINT8 result's exponents
  size_t ld;                // elements from one row of gate (and of up) to the next
  int M, N;
  Format f;
};
// act(g) = g / (1 + exp(-z)) with z = g (SiLU) or z = 2 sqrt(2 / pi) (g + 0.044715 g^3) (the tanh form of GELU, 1 + tanh(z / 2)
// being 2 / (1 + exp(-z)): no cancellation where z is far below zero).
template <int ACT, class T>
__device__ __forceinline__ T act_argument(T g) {
  return ACT == LQER_SILU ? g : (T)1.5957691216057307117597842397375 * (g + (T)0.044715 * g * g * g);
}
// Eight values of the result, and a bound on their relative error.  fp32 results take expf and the quick quotient, two units in
// the last place off (bf16 to fp32, 2048 x 11008: 30.1 us, with an exactly rounded one 44.0).  Narrower ones take the special
// function unit's 2^x of -z log2(e): beside the units of 2^-23 of ex2 (2), of the reciprocal (1), of the sum and of two products (1/2
// each) an error of z counts |z| times where exp(-z) rules the denominator, z < 0: one rounding and that of the constant for
// SiLU (2^-23 |z|), five more for GELU (2^-21 |z|); the bound allows twice that, and 6 units for the rest, that of z > 0
// (|z| exp(-z) < 0.37) included.  y: the largest -z log2(e).
template <int ACT, bool FULL>
__device__ __forceinline__ void gate8(const float (&g)[8], const float (&u)[8], float (&v)[8], float& rel) {
  if (FULL) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fdividef(g[i], 1.0f + expf(-act_argument<ACT>(g[i]))) * u[i];
    return;
  }
  constexpr float kLog2e = 1.4426950408889634f;
  const F2 one2 = f2(1.f, 1.f);
  float y = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const F2 g2 = f2(g[i], g[i + 1]);
    F2 t2;
    if (ACT == LQER_SILU) {
      t2 = mul2(g2, f2(-kLog2e, -kLog2e));
    } else {
      constexpr float k1 = -1.5957691216057308f * kLog2e, k3 = k1 * 0.044715f;
      t2 = mul2(g2, fma2(mul2(g2, g2), f2(k3, k3), f2(k1, k1)));
    }
    float t[2], r[2];
    unf2(t2, t[0], t[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) y = fmaxf(y, ACT == LQER_SILU || t[k] < 128.f ? t[k] : 0.f);         // 2^y beyond fp32: the value is zero, surely
#pragma unroll
    for (int k = 0; k < 2; ++k) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t[k]) : "f"(t[k]));
    const F2 d2 = add2(f2(t[0], t[1]), one2);
    unf2(d2, r[0], r[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r[k]) : "f"(r[k]));
    const F2 v2 = mul2(mul2(g2, f2(r[0], r[1])), f2(u[i], u[i + 1]));
    unf2(v2, v[i], v[i + 1]);
  }
  if (ACT == LQER_SILU && !(y < 128.f)) {             // rare (a mask of the type's lowest value): the same without those that are zero
    y = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y = fmaxf(y, g[i] * -kLog2e < 128.f ? g[i] * -kLog2e : 0.f);
  }
  rel = fmaf(y, ACT == LQER_SILU ? 2.3841858e-7f : 9.5367432e-7f, 7.1525574e-7f);
}
// act(gate[at]) * up[at] in fp64: for values in doubt, from memory again, so that nothing has to be kept for them.
template <bool XB, int ACT>
__device__ __noinline__ double gate_wide(const void* gate, const void* up, size_t at) {
  double g, u;
  if (XB) {
    g = __uint_as_float((uint32_t)static_cast<const uint16_t*>(gate)[at] << 16);
    u = __uint_as_float((uint32_t)static_cast<const uint16_t*>(up)[at] << 16);
  } else {
    g = static_cast<const float*>(gate)[at];
    u = static_cast<const float*>(up)[at];
  }
  return g / (1.0 + exp(-act_argument<ACT>(g))) * u;
}
// Thread t of a CTA's row of threads holds columns 8 t .. 8 t + 7 of the CTA's stretch, of every gridDim.y-th row; the next row's are on
// their way while this one's are worked on.  Eight CTAs of 64 registers fit an SM: the values in doubt come from memory again, since with all
// inputs kept for them registers were spilled (2048 x 11008 to MXINT8, SiLU of fp32 39.9 us against 34.4, GELU of bf16 58 against 32.5).
template <bool XB, int YT, int ACT>
__global__ void __launch_bounds__(128, 8) gated_activation_kernel(const GateParams p) {
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const int col = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
  const bool in = col < p.N;
  const QuantConsts qc = quant_consts(p.f.bits, p.f.emin, p.f.emax);
  Raw<XB> rg, ru;
  rg.clear();
  ru.clear();
  size_t at = blockIdx.y * p.ld + col, idx = (size_t)blockIdx.y * p.N + col;
  const size_t hop = gridDim.y * p.ld, out_hop = (size_t)gridDim.y * p.N;
  if (in) {
    rg.load(p.gate, at);
    ru.load(p.up, at);
  }
  for (int row = blockIdx.y; row < p.M; row += gridDim.y, idx += out_hop) {
    float g[8], u[8], v[8], rel = 0.f;
    rg.values(g);
    ru.values(u);
    const size_t now = at;
    at += hop;
    if (in && row + (int)gridDim.y < p.M) {
      rg.load(p.gate, at);
      ru.load(p.up, at);
    }
    gate8<ACT, YT == kYF32>(g, u, v, rel);
    if (YT == kYMXINT8) {
      uint2 m8;
      int e;
      quantise8(v, qc, rel, [&](int i) { return in ? gate_wide<XB, ACT>(p.gate, p.up, now + i) : 0.0; }, m8, e);
      if (in) store_mxint8(p.Y, p.Ye, idx, m8, e);
    } else if (in) {
      store8<YT == kYBF16>(p.Y, idx, v);
    }
  }
}
template <bool XB, int YT>
static cudaError_t launch_gate(const GateParams& p, int act, cudaStream_t s) {
  const int threads = 128, across = (p.N / 8 + threads - 1) / threads;
  int down = sm_count() * 8 / across;                 // eight CTAs an SM
  if (down > p.M) down = p.M;
  if (down > 65535) down = 65535;
  if (down < 1) down = 1;
  LaunchScope scope(kFamQuantize, s);
  return act == LQER_SILU ? launch_after(gated_activation_kernel<XB, YT, LQER_SILU>, dim3(across, down), threads, s, p)
                          : launch_after(gated_activation_kernel<XB, YT, LQER_GELU_TANH>, dim3(across, down), threads, s, p);
}
template <bool XB>
static cudaError_t launch_gate_y(const GateParams& p, int act, int y_type, cudaStream_t s) {
  return y_type == kYF32 ? launch_gate<XB, kYF32>(p, act, s) : y_type == kYBF16 ? launch_gate<XB, kYBF16>(p, act, s) : launch_gate<XB, kYMXINT8>(p, act, s);
}

// ---------------------------------------------------------------------------- MXINT activations as values
// A thread takes whole blocks: 16 bytes of mantissas and an exponent.  wide: the values are aligned to 32 bytes.
template <int YT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* __restrict__ Xq, void* Y, size_t blocks, bool wide, Format f) {
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const uint8_t* exps = Xq + blocks * 16;
  for (size_t o = (size_t)blockIdx.x * blockDim.x + threadIdx.x; o < blocks; o += (size_t)gridDim.x * blockDim.x) {
    const uint4 m = reinterpret_cast<const uint4*>(Xq)[o];
    const uint32_t eb = exps[o];
    float v[2][8];
    const uint32_t w[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 q = mxint_quad_values(w[i], eb, f.bits, f.emin, f.emax);
      v[i >> 1][4 * (i & 1)] = q.x; v[i >> 1][4 * (i & 1) + 1] = q.y; v[i >> 1][4 * (i & 1) + 2] = q.z; v[i >> 1][4 * (i & 1) + 3] = q.w;
    }
    if (!wide) {
      store8<YT == kYBF16>(Y, o * 16, v[0]);
      store8<YT == kYBF16>(Y, o * 16 + 8, v[1]);
    } else if (YT == kYBF16) {
      uint32_t u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = round_bf16x2(v[i >> 2][2 * (i & 3)], v[i >> 2][2 * (i & 3) + 1]);
      store32(static_cast<uint16_t*>(Y) + o * 16, u);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(v[h][i]);
        store32(static_cast<float*>(Y) + o * 16 + h * 8, u);
      }
    }
  }
}

}  // namespace bd

cudaError_t launch_add_rms_norm(const void* X, int x_type, const void* res, void* res_out, int r_type, const void* w, int w_type, double eps,
                                int M, int K, int bits, int emin, int emax, void* Y, int y_type, cudaStream_t s) {
  const bd::NormParams p{X, res, res_out, w, Y, static_cast<uint8_t*>(Y) + (size_t)M * K, eps, 1.0 / K, M, K, w_type == kXBF16, {bits, emin, emax}};
  return x_type == kXBF16 ? (r_type == kXBF16 ? bd::launch_norm_y<true, true>(p, y_type, s) : bd::launch_norm_y<true, false>(p, y_type, s))
                          : (r_type == kXBF16 ? bd::launch_norm_y<false, true>(p, y_type, s) : bd::launch_norm_y<false, false>(p, y_type, s));
}
cudaError_t launch_gated_activation(const void* gate, const void* up, int x_type, size_t ld, int M, int N, int act, int bits, int emin,
                                    int emax, void* Y, int y_type, cudaStream_t s) {
  const bd::GateParams p{gate, up, Y, static_cast<uint8_t*>(Y) + (size_t)M * N, ld, M, N, {bits, emin, emax}};
  return x_type == kXBF16 ? bd::launch_gate_y<true>(p, act, y_type, s) : bd::launch_gate_y<false>(p, act, y_type, s);
}
cudaError_t launch_dequantize(const void* Xq, int M, int K, int bits, int emin, int emax, void* Y, int y_type, cudaStream_t s) {
  const size_t blocks = (size_t)M * K / 16, want = (blocks + 255) / 256, most = (size_t)sm_count() * 32;
  const bool wide = reinterpret_cast<uintptr_t>(Y) % 32 == 0;
  const bd::Format f{bits, emin, emax};
  const dim3 grid((unsigned)(want < most ? want : most));
  LaunchScope scope(kFamQuantize, s);
  return y_type == kYBF16 ? bd::launch_after(bd::dequantize_kernel<kYBF16>, grid, 256, s, static_cast<const uint8_t*>(Xq), Y, blocks, wide, f)
                          : bd::launch_after(bd::dequantize_kernel<kYF32>, grid, 256, s, static_cast<const uint8_t*>(Xq), Y, blocks, wide, f);
}

}  // namespace lqer
