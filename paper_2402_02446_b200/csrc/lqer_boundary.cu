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
#include "lqer_tc_ptx.cuh"

namespace lqer {
namespace bd {

// Eight consecutive elements from index idx (a multiple of 8) of an fp32 or bf16 tensor.
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, size_t idx, float (&v)[8]) {
  if (BF16) {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + idx);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + idx);
    const float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
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

// Quantises the eight values of a lane; lanes 2 i and 2 i + 1 share a block.  Every lane of the warp takes part.
// rel(i): bound on the relative error of v[i]; wide(i): the same value in fp64.  A mantissa is in doubt where the scaled value
// lies within its error of a half, the exponent where the block's maximum does of a power of two.
template <class Rel, class Wide>
__device__ __forceinline__ void quantise8(const float (&v)[8], const QuantConsts& c, Rel rel, Wide wide, uint2& m8, int& e) {
  float hi = 0.f, lo = 0.f;                          // fmaxf drops a NaN operand: NaN counts as zero
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(v[i]);
    hi = fmaxf(hi, fmaf(a, rel(i), a));
    lo = fmaxf(lo, fmaf(a, -rel(i), a));
  }
  hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, 1));
  lo = fmaxf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, 1));
  e = block_exponent(hi, c.emin, c.emax);
  bool doubt = e != block_exponent(lo, c.emin, c.emax);
  const float inv_step = pow2f(c.shift - e), kRound = 12582912.0f;       // 1.5 * 2^23, see quantize_quad
  uint32_t rb[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = (v[i] == v[i]) ? v[i] : 0.0f;                        // NaN -> 0
    const float t = fminf(fmaxf(x * inv_step, -c.qmax), c.qmax);         // exact scaling; +-inf saturate
    const float s = t + kRound;
    const float d = fabsf(t - (s - kRound));                             // exact: distance to the chosen integer
    doubt = doubt || fmaf(fabsf(t), rel(i), d) > 0.49999f;
    rb[i] = __float_as_uint(s);
  }
  m8.x = __byte_perm(__byte_perm(rb[0], rb[1], 0x0040), __byte_perm(rb[2], rb[3], 0x0040), 0x5410);
  m8.y = __byte_perm(__byte_perm(rb[4], rb[5], 0x0040), __byte_perm(rb[6], rb[7], 0x0040), 0x5410);
  if (__any_sync(0xFFFFFFFFu, doubt)) {
    double amax = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmax(amax, fabs(wide(i)));
    amax = fmax(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
    e = block_exponent(amax, c.emin, c.emax);
    uint32_t m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = (uint32_t)quant_mantissa(wide(i), e, c.shift + 2) & 0xFFu;
    m8.x = m[0] | m[1] << 8 | m[2] << 16 | m[3] << 24;
    m8.y = m[4] | m[5] << 8 | m[6] << 16 | m[7] << 24;
  }
}

struct Format { int bits, emin, emax; };

// ---------------------------------------------------------------------------- norm
struct NormParams {
  const void* X;
  const void* res;          // may be null
  void* res_out;            // may be null; may be res, or X if the types agree
  const void* w;
  void* Y;
  double eps;
  int M, K;
  int w_bf16;
  Format f;
};
// v -> the residual stream's value h: x + res in fp32, rounded to the stream's type (what a later reader of it sees).
template <bool XB, bool RB>
__device__ __forceinline__ void form_h(const NormParams& p, size_t idx, float (&h)[8]) {
  load8<XB>(p.X, idx, h);
  if (p.res != nullptr) {
    float r[8];
    load8<RB>(p.res, idx, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] += r[i];
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
// One row's octet of Y.  Bound on the fp32 values' error: the inverse root, its product with h and the product with w are
// rounded once each, 3 * 2^-24 < 2^-22; an inverse root near the end of fp32's range has no such bound.
template <int YT>
__device__ __forceinline__ void finish8(const NormParams& p, size_t row, int col, bool in, const float (&h)[8], const float (&w)[8],
                                        float inv, double inv64, const QuantConsts& qc) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = h[i] * inv * w[i];
  const size_t idx = row * p.K + col;
  if (YT == kYMXINT8) {
    uint2 m8;
    int e;
    const float rel = inv > 1e-30f ? 2.3841858e-7f : 1.0f;
    quantise8(v, qc, [=](int) { return rel; }, [&](int i) { return (double)h[i] * inv64 * (double)w[i]; }, m8, e);
    if (in) {
      int8_t* Ym = static_cast<int8_t*>(p.Y);
      *reinterpret_cast<uint2*>(Ym + idx) = m8;
      if ((col & 8) == 0) reinterpret_cast<uint8_t*>(Ym + (size_t)p.M * p.K)[row * (p.K / 16) + (col >> 4)] = (uint8_t)(e + 127);
    }
  } else if (in) {
    store8<YT == kYBF16>(p.Y, idx, v);
  }
}
// The sum over the CTA, in every thread: warps first, then one value a warp.
__device__ __forceinline__ double cta_sum(double s, double* slots) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) slots[threadIdx.x >> 5] = s;
  __syncthreads();
  s = lane < warps ? slots[lane] : 0.0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return s;
}
__device__ __forceinline__ void load_w(const NormParams& p, int col, float (&w)[8]) {
  if (p.w_bf16) load8<true>(p.w, col, w);
  else load8<false>(p.w, col, w);
}

// One CTA a row, the row in registers: OPT octets a thread.  The sum of squares is kept in fp64: it makes the row's factor good
// to fp64 (the MXINT borders need that) and holds squares that fp32 cannot.
template <bool XB, bool RB, int YT, int OPT>
__global__ void __launch_bounds__(1024) add_rms_norm_kernel(const NormParams p) {
  __shared__ double slots[32];
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const size_t row = blockIdx.x;
  float h[OPT][8], w[OPT][8];
  double sum = 0.0;
#pragma unroll
  for (int o = 0; o < OPT; ++o) {
    const int col = (o * blockDim.x + threadIdx.x) * 8;
    if (col < p.K) {
      form_h<XB, RB>(p, row * p.K + col, h[o]);
      load_w(p, col, w[o]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[o][i] = w[o][i] = 0.f;
    }
  }
#pragma unroll
  for (int o = 0; o < OPT; ++o) {
    const int col = (o * blockDim.x + threadIdx.x) * 8;
    if (p.res_out != nullptr && col < p.K) store8<RB>(p.res_out, row * p.K + col, h[o]);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma((double)h[o][i], (double)h[o][i], sum);
  }
  sum = cta_sum(sum, slots);
  const double inv64 = 1.0 / sqrt(sum / p.K + p.eps);
  const float inv = (float)inv64;
  const QuantConsts qc = quant_consts(p.f.bits, p.f.emin, p.f.emax);
#pragma unroll
  for (int o = 0; o < OPT; ++o) {
    const int col = (o * blockDim.x + threadIdx.x) * 8;
    finish8<YT>(p, row, col, col < p.K, h[o], w[o], inv, inv64, qc);
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
    float h[8];
    form_h<XB, RB>(p, row * p.K + col, h);
    if (p.res_out != nullptr) store8<RB>(p.res_out, row * p.K + col, h);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fma((double)h[i], (double)h[i], sum);
  }
  sum = cta_sum(sum, slots);
  const double inv64 = 1.0 / sqrt(sum / p.K + p.eps);
  const float inv = (float)inv64;
  const QuantConsts qc = quant_consts(p.f.bits, p.f.emin, p.f.emax);
  for (int at = 0; at < p.K; at += blockDim.x * 8) {            // whole warps, for the blocks' maxima
    const int col = at + threadIdx.x * 8;
    const bool in = col < p.K;
    float h[8] = {}, w[8] = {};
    if (in) {
      if (p.res_out != nullptr) load8<RB>(p.res_out, row * p.K + col, h);
      else form_h<XB, RB>(p, row * p.K + col, h);
      load_w(p, col, w);
    }
    finish8<YT>(p, row, col, in, h, w, inv, inv64, qc);
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
  const int opt = octets <= 1024 ? 1 : octets <= 2048 ? 2 : 4;
  const int threads = ((octets + opt - 1) / opt + 31) / 32 * 32;
  LaunchScope scope(kFamQuantize, s);
  if (threads > 1024) return launch_after(add_rms_norm_long_kernel<XB, RB, YT>, dim3(p.M), 1024, s, p);
  return opt == 1   ? launch_after(add_rms_norm_kernel<XB, RB, YT, 1>, dim3(p.M), threads, s, p)
         : opt == 2 ? launch_after(add_rms_norm_kernel<XB, RB, YT, 2>, dim3(p.M), threads, s, p)
                    : launch_after(add_rms_norm_kernel<XB, RB, YT, 4>, dim3(p.M), threads, s, p);
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
// Thread t of a CTA's row of threads holds columns 8 t .. 8 t + 7 of the CTA's stretch, of every gridDim.y-th row.
template <bool XB, int YT, int ACT>
__global__ void __launch_bounds__(128) gated_activation_kernel(const GateParams p) {
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const int col = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
  const bool in = col < p.N;
  const QuantConsts qc = quant_consts(p.f.bits, p.f.emin, p.f.emax);
  for (size_t row = blockIdx.y; row < (size_t)p.M; row += gridDim.y) {
    float g[8] = {}, u[8] = {}, v[8], z[8];
    if (in) {
      load8<XB>(p.gate, row * p.ld + col, g);
      load8<XB>(p.up, row * p.ld + col, u);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      z[i] = act_argument<ACT>(g[i]);
      v[i] = __fdividef(g[i], 1.0f + expf(-z[i])) * u[i];
    }
    const size_t idx = row * p.N + col;
    if (YT == kYMXINT8) {
      uint2 m8;
      int e;
      // error of v: expf 2 units of 2^-23 at most, the sum and the products half a unit each, the quotient 2; an error of z
      // (GELU: seven roundings) counts |z| times
      quantise8(
          v, qc, [&](int i) { return ACT == LQER_SILU ? 9.5367432e-7f : fmaf(fabsf(z[i]), 9.5367432e-7f, 9.5367432e-7f); },
          [&](int i) {
            const double gd = g[i];
            return gd / (1.0 + exp(-act_argument<ACT>(gd))) * (double)u[i];
          },
          m8, e);
      if (in) {
        int8_t* Ym = static_cast<int8_t*>(p.Y);
        *reinterpret_cast<uint2*>(Ym + idx) = m8;
        if ((col & 8) == 0) reinterpret_cast<uint8_t*>(Ym + (size_t)p.M * p.N)[row * (p.N / 16) + (col >> 4)] = (uint8_t)(e + 127);
      }
    } else if (in) {
      store8<YT == kYBF16>(p.Y, idx, v);
    }
  }
}
template <bool XB, int YT>
static cudaError_t launch_gate(const GateParams& p, int act, cudaStream_t s) {
  const int threads = 128, across = (p.N / 8 + threads - 1) / threads;
  int down = 16 * sm_count() * 4 / across;
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
template <int YT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* __restrict__ Xq, void* Y, size_t octets, Format f) {
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const uint8_t* exps = Xq + octets * 8;
  for (size_t o = (size_t)blockIdx.x * blockDim.x + threadIdx.x; o < octets; o += (size_t)gridDim.x * blockDim.x) {
    const uint2 m = *reinterpret_cast<const uint2*>(Xq + o * 8);
    const uint32_t eb = exps[o >> 1];
    const float4 a = mxint_quad_values(m.x, eb, f.bits, f.emin, f.emax), b = mxint_quad_values(m.y, eb, f.bits, f.emin, f.emax);
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    store8<YT == kYBF16>(Y, o * 8, v);
  }
}

}  // namespace bd

cudaError_t launch_add_rms_norm(const void* X, int x_type, const void* res, void* res_out, int r_type, const void* w, int w_type, double eps,
                                int M, int K, int bits, int emin, int emax, void* Y, int y_type, cudaStream_t s) {
  const bd::NormParams p{X, res, res_out, w, Y, eps, M, K, w_type == kXBF16, {bits, emin, emax}};
  return x_type == kXBF16 ? (r_type == kXBF16 ? bd::launch_norm_y<true, true>(p, y_type, s) : bd::launch_norm_y<true, false>(p, y_type, s))
                          : (r_type == kXBF16 ? bd::launch_norm_y<false, true>(p, y_type, s) : bd::launch_norm_y<false, false>(p, y_type, s));
}
cudaError_t launch_gated_activation(const void* gate, const void* up, int x_type, size_t ld, int M, int N, int act, int bits, int emin,
                                    int emax, void* Y, int y_type, cudaStream_t s) {
  const bd::GateParams p{gate, up, Y, ld, M, N, {bits, emin, emax}};
  return x_type == kXBF16 ? bd::launch_gate_y<true>(p, act, y_type, s) : bd::launch_gate_y<false>(p, act, y_type, s);
}
cudaError_t launch_dequantize(const void* Xq, int M, int K, int bits, int emin, int emax, void* Y, int y_type, cudaStream_t s) {
  const size_t octets = (size_t)M * K / 8, want = (octets + 255) / 256, most = (size_t)sm_count() * 32;
  const bd::Format f{bits, emin, emax};
  const dim3 grid((unsigned)(want < most ? want : most));
  LaunchScope scope(kFamQuantize, s);
  return y_type == kYBF16 ? bd::launch_after(bd::dequantize_kernel<kYBF16>, grid, 256, s, static_cast<const uint8_t*>(Xq), Y, octets, f)
                          : bd::launch_after(bd::dequantize_kernel<kYF32>, grid, 256, s, static_cast<const uint8_t*>(Xq), Y, octets, f);
}

}  // namespace lqer
