// Keys and values of past tokens: the layout of a step's plan and of the cache, and what the kernels that read them share
// (lqer_cache.cu: tables and appending; lqer_attention.cu, lqer_attention_tiles.cu: the attention).
//
// A cache holds pages of `page` tokens: keys and values [n_pages, kv_heads, page, head_dim] each, bf16 or MXINT8 (int8 mantissas in that
// order, then an exponent byte for every 16 of them).  Row r of a table lists the pages of request r in the order of its tokens.  A slot is
// page * tokens a page + place in the page.  A step's plan says which rows of the step's tensors belong to which request and how long that is then.
#pragma once

#include "lqer_tc_ptx.cuh"

namespace lqer {
namespace kv {

constexpr uint32_t kStepMagic = 0x50455453u;

struct StepHead {              // first 256 bytes of a step's plan
  DeviceStatus status;
  uint32_t magic;
  int R, M, page, max_pages, n_pages, max_added;
};
struct StepRequest {           // one per request, behind the head
  int row0, n, len, reserved;  // first row, rows (0: none, or refused), tokens that it holds once they are in
};
constexpr size_t kStepHeadBytes = 256;
// Behind the requests: lengths and ring as they are after the step, for whoever keeps the step when the tables' own go on.
__host__ __device__ constexpr size_t step_lengths_at(int R) { return kStepHeadBytes + (size_t)R * sizeof(StepRequest); }
__host__ __device__ constexpr size_t step_ring_at(int R) { return step_lengths_at(R) + ((size_t)R * sizeof(int) + 15) / 16 * 16; }
inline size_t step_bytes(int R) { return step_ring_at(R) + 2 * sizeof(long long); }

// What the attention kernels read.
struct Attention {
  const void* Q;
  void* Y;
  const void* keys;            // MXINT8: the mantissas
  const void* values;
  const uint8_t* key_exps;     // MXINT8
  const uint8_t* value_exps;
  const int* tables;
  StepHead* step;
  size_t q_stride;             // elements from one row of Q to the next
  int M, R, max_pages, n_pages, page, page_shift, max_added;
  int hq, hkv, group;
  int window, sinks;           // window 0: none
  float scale_log2;            // of the scores, times log2(e)
  int bits;                    // of the mantissas of an MXINT8 cache
};
__device__ __forceinline__ const StepRequest* requests_of(const StepHead* h) {
  return reinterpret_cast<const StepRequest*>(reinterpret_cast<const uint8_t*>(h) + kStepHeadBytes);
}
// Whether the plan is one of this batch and of tables like these; if not, one thread says so.
__device__ __forceinline__ bool step_fits(const Attention& p, bool first) {
  const StepHead& h = *p.step;
  if (h.magic == kStepMagic && h.R == p.R && h.M == p.M && h.page == p.page && h.max_pages == p.max_pages && h.n_pages == p.n_pages &&
      h.max_added <= p.max_added)
    return true;
  if (first) report_error(&p.step->status, LQER_ERR_BAD_PACKED, 1);
  return false;
}
// A table entry as a page: one that is none is reported and stands for page 0.
__device__ __forceinline__ int checked_page(const Attention& p, int id, int r) {
  if ((unsigned)id < (unsigned)p.n_pages) return id;
  report_error(&p.step->status, LQER_ERR_BOUNDS, 2, r, id);
  return 0;
}

// Two int8 mantissas m (in the low bytes of the halves of `b`) as bf16 values m s, exact.  With the sign bit turned over the byte is u = m + 128, and 0x4300 + u
// the bf16 number y = 128 + u up to u = 127 and 2 u from there on: z = (y - 256) s is m s below zero and 2 m s above, and half of
// what is positive of it too much.  All but the first step are multiply-adds: the integer units are what bounds the kernels that do this.
struct MantissaScale { uint32_t s, c; };       // bf16 pairs: s, and -256 s
__device__ __forceinline__ uint32_t mantissas_bf16x2(uint32_t b, const MantissaScale& k) {
  const uint32_t y = (b & 0x00FF00FFu) ^ 0x43804380u;
  uint32_t z, t;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(z) : "r"(y), "r"(k.s), "r"(k.c));
  asm("fma.rn.relu.bf16x2 %0, %1, %2, %3;" : "=r"(t) : "r"(y), "r"(k.s), "r"(k.c));
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(z) : "r"(t), "r"(0xBF00BF00u), "r"(z));
  return z;
}
// The scale 2^(e - (bits - 2)) of two blocks from their exponent bytes (in the low bytes of the halves of `e`; within the format's window), or of one; shift = bits - 2.
__device__ __forceinline__ MantissaScale mantissa_scales(uint32_t e, int shift) {
  return {e * 128u - (uint32_t)shift * 0x00800080u, e * 128u + (0x80008000u + (uint32_t)(8 - shift) * 0x00800080u)};
}
__device__ __forceinline__ MantissaScale mantissa_scale(uint32_t e, int shift) {
  return {e * 0x00800080u - (uint32_t)shift * 0x00800080u, e * 0x00800080u + (0x80008000u + (uint32_t)(8 - shift) * 0x00800080u)};
}
// A word right by a byte (as a multiplication, where there is room, it takes longer: 40 heads, MXINT8, 171 -> 185 us).
__device__ __forceinline__ uint32_t byte_down(uint32_t w) { return w >> 8; }
// Eight mantissas as four pairs in order.
__device__ __forceinline__ uint4 mantissas8(uint2 m, const MantissaScale& k) {
  return make_uint4(mantissas_bf16x2(__byte_perm(m.x, 0u, 0x4140), k), mantissas_bf16x2(__byte_perm(m.x, 0u, 0x4342), k),
                    mantissas_bf16x2(__byte_perm(m.y, 0u, 0x4140), k), mantissas_bf16x2(__byte_perm(m.y, 0u, 0x4342), k));
}
__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Requests of more than `few` rows (tokens times heads that share a key head) on tcgen05 (lqer_attention_tiles.cu).
cudaError_t launch_tiles(const Attention& a, int few, size_t y_extent, const lqer_kv_cache_t& c, void* scratch, cudaStream_t s);
size_t tiles_scratch_bytes(const Attention& a, int head_dim);

// Launches with the programmatic attribute: the kernels wait for their predecessor before they touch memory.  What it may have written while they were
// there already (plan, tables, slots, queries, keys, values) is read by ordinary loads: those that are marked read-only promise that nobody writes during the
// kernel's whole life, and could find what a kernel before the predecessor left in the SM's cache.
template <class... P, class... A>
static cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace kv
}  // namespace lqer
