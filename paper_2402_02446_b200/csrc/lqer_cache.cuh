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
constexpr int kMaxRequests = 16384;

struct StepHead {              // first 256 bytes of a step's plan
  DeviceStatus status;
  uint32_t magic;
  int R, M, page, max_pages, n_pages, max_added, rows;     // rows: of all requests together
};
struct StepRequest {           // one per request, behind the head
  int row0, n, len, reserved;  // first row, rows (0: none, or refused), tokens that it holds once they are in
};
constexpr size_t kStepHeadBytes = 256;
inline size_t step_bytes(int R) { return kStepHeadBytes + (size_t)R * sizeof(StepRequest); }

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
  int bits, emin, emax;        // format of an MXINT8 cache
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

// Two int8 mantissas (in the low bytes of the halves of `b`, the rest zero) as bf16, times s (a power of two, twice): exact.
// 0x4300 | low seven bits is 128 + them; taken from it are 128, or 256 where the sign bit is set.
__device__ __forceinline__ uint32_t mantissas_bf16x2(uint32_t b, uint32_t s) {
  uint32_t d;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"((b & 0x007F007Fu) | 0x43004300u), "r"((b & 0x00800080u) | 0x43004300u));
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(d), "r"(s));
  return d;
}
// The bf16 pair of 2^(e - (bits - 2)) for an exponent byte; lo, hi: the window's ends as bytes.
__device__ __forceinline__ uint32_t mantissa_scale(uint32_t byte, int lo, int hi, int shift) {
  const uint32_t s = (uint32_t)(min(max((int)byte, lo), hi) - shift) << 7;
  return s | (s << 16);
}
// Eight mantissas as four pairs.
__device__ __forceinline__ uint4 mantissas8(uint2 m, uint32_t s) {
  return make_uint4(mantissas_bf16x2(__byte_perm(m.x, 0u, 0x4140), s), mantissas_bf16x2(__byte_perm(m.x, 0u, 0x4342), s),
                    mantissas_bf16x2(__byte_perm(m.y, 0u, 0x4140), s), mantissas_bf16x2(__byte_perm(m.y, 0u, 0x4342), s));
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
cudaError_t launch_tiles(const Attention& a, int few, size_t y_extent, const lqer_kv_cache_t& c, cudaStream_t s);

// Launches with the programmatic attribute: the kernels wait for their predecessor before they touch memory.
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
