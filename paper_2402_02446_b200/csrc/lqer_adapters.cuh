// Adapters of many requests: the layouts of pool and plan, and what the kernels for few and for many rows share (lqer_adapters.cu,
// lqer_adapters_many.cu; the layouts are described in the former).
#pragma once

#include "lqer_tc_ptx.cuh"

namespace lqer {
namespace ad {

constexpr uint32_t kPoolMagic = 0x4C4F5242u, kPlanMagic = 0x4E414C50u;
constexpr int kFewRows = 8, kManyRows = 128; // rows of a tile of the kernels for few and for many rows

struct SlotHead {            // first 32 bytes of a slot
  uint32_t magic;
  int K, N, max_rank;
  int rank;                  // 0: empty
  float scale;
  int reserved[2];
};
struct PlanHead {            // first 256 bytes of a plan
  DeviceStatus status;
  uint32_t magic;
  int M, n_slots, reserved;
  struct { int n_tiles, n_adapted; } of[2];    // of the list for few and of that for many rows: tiles; those in front that name a slot
};
struct Tile { int slot, rows; };

// Bytes of a row of B's image (also the span of its swizzle).
__host__ __device__ inline int b_pitch(int max_rank) { return max_rank <= 16 ? 32 : max_rank <= 32 ? 64 : 128; }
__host__ __device__ inline int rank16(int rank) { return (rank + 15) / 16; }
__host__ __device__ inline size_t a_bytes(int K, int rank) { return (size_t)((K + 63) / 64) * rank16(rank) * 2048; }
__host__ __device__ inline size_t b_bytes(int N, int rank, int pitch) { return (size_t)((N + 127) / 128) * ((rank + 63) / 64) * 128 * pitch; }
// Place of 16-byte piece c of row r in an image of that pitch.
__host__ __device__ inline uint32_t swizzled(uint32_t r, uint32_t c, uint32_t pitch) {
  const uint32_t at = r * pitch + c * 16;
  return at ^ (((at >> 7) & (pitch / 16 - 1)) << 4);
}

// Row of B's image, among 128, of a column.
__host__ __device__ inline int image_row(int n) { return (n & ~31) + 8 * ((n & 7) >> 1) + 2 * ((n & 31) >> 3) + (n & 1); }

// ---------------------------------------------------------------------------- what both kinds of kernels share
struct Params {
  const void* X;
  const uint8_t* pool;
  PlanHead* plan;
  const Tile* tiles;
  const int* rows;
  const void* Y0;
  void* Y;
  size_t slot_bytes;
  int M, K, N, max_rank, plan_slots;
  int y0_bf16, y_bf16;
  bool x_wide, y_wide;       // X; Y0 and Y: aligned to 32 bytes
  int bits, emin, emax;      // format of an MXINT8 X
  size_t y_extent;
};

__device__ __forceinline__ uint4 ld16(const void* p) { return __ldg(static_cast<const uint4*>(p)); }
__device__ __forceinline__ uint4 ld16_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// 32 bytes in one access (a whole sector), or in two where the tensor is not aligned to 32.
__device__ __forceinline__ void ld32(const void* p, bool aligned, uint4& a, uint4& b) {
  if (aligned) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p) : "memory");
  } else {
    a = static_cast<const uint4*>(p)[0];
    b = static_cast<const uint4*>(p)[1];
  }
}
__device__ __forceinline__ void st32(void* p, bool aligned, const uint4& a, const uint4& b) {
  if (aligned) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
  } else {
    static_cast<uint4*>(p)[0] = a;
    static_cast<uint4*>(p)[1] = b;
  }
}
// The upper halves of two fp32 values (their leading bf16 parts, cut off) in one word.
__device__ __forceinline__ uint32_t top_halves(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
__device__ __forceinline__ float top_half(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t round_bf16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// P bf16 parts of fp32 values.  Three parts are cut off one after the other and hold all 24 bits.  Two are rounded to nearest: what is left of
// the first is at most 2^-8 of the value, of the second 2^-17, either way alike (cut off, it would be up to 2^-15, always towards
// zero).  Either takes as many instructions.  kBf16Max: beyond the largest bf16 a value would be rounded to infinity.
constexpr float kBf16Max = 3.3895313892515354759e38f;
// The first part of a pair, and what is left of it.
template <int P>
__device__ __forceinline__ uint32_t first_part(float& a, float& b) {
  const uint32_t w = P == 2 ? round_bf16x2(a, b) : top_halves(a, b);
  a -= P == 2 ? __uint_as_float(w << 16) : top_half(a);                    // exact
  b -= P == 2 ? __uint_as_float(w & 0xFFFF0000u) : top_half(b);
  return w;
}
// Any pair: word p holds part p of both.  The first part of a value beyond kBf16Max is cut off; what is left of an infinity is nothing (it is
// all in its first part); NaN stays.
template <int P>
__device__ __forceinline__ void split(float a, float b, uint32_t (&w)[P]) {
  const float inf = __uint_as_float(0x7F800000u);
  w[0] = top_halves(fabsf(a) > kBf16Max || P != 2 ? a : __uint_as_float(round_bf16x2(a, a) & 0xFFFF0000u),
                    fabsf(b) > kBf16Max || P != 2 ? b : __uint_as_float(round_bf16x2(b, b) & 0xFFFF0000u));
  a = fabsf(a) == inf ? 0.f : a - __uint_as_float(w[0] << 16);
  b = fabsf(b) == inf ? 0.f : b - __uint_as_float(w[0] & 0xFFFF0000u);
#pragma unroll
  for (int p = 1; p + 1 < P; ++p) w[p] = first_part<P>(a, b);
  if (P > 1) w[P - 1] = P == 2 ? round_bf16x2(a, b) : top_halves(a, b);
}
// Eight values, of which one beyond kBf16Max is rare: one test for all.
template <int P>
__device__ __forceinline__ void split8(const float (&v)[8], uint32_t (&w)[4][P]) {
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(v[i]));
  if (big > kBf16Max) {
#pragma unroll
    for (int i = 0; i < 4; ++i) split<P>(v[2 * i], v[2 * i + 1], w[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
    for (int p = 0; p + 1 < P; ++p) w[i][p] = first_part<P>(a, b);
    w[i][P - 1] = P == 2 ? round_bf16x2(a, b) : top_halves(a, b);
  }
}

// Eight consecutive activations of a row as raw bits, and as P words of bf16 pairs for each of the four pairs.
template <int XT>
struct XOct {
  uint4 a, b;                // fp32: both; bf16: a; MXINT8: a.x, a.y mantissas, a.z exponent byte
  struct Place {
    const uint8_t* x;
    const uint8_t* e;        // MXINT8: of the exponent byte
    __device__ __forceinline__ void set(const Params& p, int row, int col) {
      const size_t idx = (size_t)row * p.K + col;
      x = static_cast<const uint8_t*>(p.X) + idx * (XT == kXF32 ? 4 : XT == kXBF16 ? 2 : 1);
      if (XT == kXMXINT8) e = static_cast<const uint8_t*>(p.X) + (size_t)p.M * p.K + (idx >> 4);      // K is a multiple of 16
    }
    __device__ __forceinline__ void next_slab() {
      x += 64 * (XT == kXF32 ? 4 : XT == kXBF16 ? 2 : 1);
      if (XT == kXMXINT8) e += 4;
    }
  };
  __device__ __forceinline__ void load(const Params& p, const Place& at, bool in) {
    if (!in) {
      a = b = make_uint4(0u, 0u, 0u, 0u);
      if (XT == kXMXINT8) a.z = 127u;
    } else if (XT == kXF32) {
      ld32(at.x, p.x_wide, a, b);
    } else if (XT == kXBF16) {
      a = ld16_once(at.x);
    } else {
      const uint2 m = __ldg(reinterpret_cast<const uint2*>(at.x));
      a = make_uint4(m.x, m.y, __ldg(at.e), 0u);
    }
  }
  __device__ __forceinline__ void load(const Params& p, int row, int col, bool in) {
    Place at;
    at.set(p, row, col);
    load(p, at, in);
  }
  template <int P>
  __device__ __forceinline__ void pairs(const Params& p, uint32_t (&w)[4][P]) const {
    if (XT == kXF32) {
      const float v[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                          __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
      split8<P>(v, w);
    } else if (XT == kXBF16) {
      w[0][0] = a.x; w[1][0] = a.y; w[2][0] = a.z; w[3][0] = a.w;
    } else {
      const float4 u = mxint_quad_values(a.x, a.z, p.bits, p.emin, p.emax), v = mxint_quad_values(a.y, a.z, p.bits, p.emin, p.emax);
      w[0][0] = top_halves(u.x, u.y); w[1][0] = top_halves(u.z, u.w);
      w[2][0] = top_halves(v.x, v.y); w[3][0] = top_halves(v.z, v.w);
    }
  }
};

struct Y0Quad {
  uint4 a;                   // four values of Y0: fp32, or bf16 in a.x and a.y
  __device__ __forceinline__ void load(const Params& p, size_t idx) {
    if (p.y0_bf16) {
      const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.Y0) + idx);
      a.x = u.x;
      a.y = u.y;
    } else {
      a = *reinterpret_cast<const uint4*>(static_cast<const float*>(p.Y0) + idx);
    }
  }
  __device__ __forceinline__ float4 values(const Params& p) const {
    if (p.y0_bf16)
      return make_float4(__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xFFFF0000u), __uint_as_float(a.y << 16), __uint_as_float(a.y & 0xFFFF0000u));
    return make_float4(__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w));
  }
};
__device__ __forceinline__ void store_y(const Params& p, size_t idx, const float4& v) {
  if (!LQER_IN_BOUNDS(&p.plan->status, idx * (p.y_bf16 ? 2 : 4), p.y_bf16 ? 8 : 16, p.y_extent, 802)) return;
  if (p.y_bf16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.Y) + idx) = make_uint2(round_bf16x2(v.x, v.y), round_bf16x2(v.z, v.w));
  else *reinterpret_cast<float4*>(static_cast<float*>(p.Y) + idx) = v;
}
// What a kernel needs of a plan's head.
struct ListHead {
  uint32_t magic;
  int M, n_slots, n_tiles, n_adapted;
};
__device__ __forceinline__ ListHead load_head(const PlanHead* h, int list) {
  const uint4 a = *reinterpret_cast<const uint4*>(&h->magic);
  const int2 b = *reinterpret_cast<const int2*>(&h->of[list]);
  return ListHead{a.x, (int)a.y, (int)a.z, b.x, b.y};
}
// Whether the plan is one of this batch.  (A plan of another batch, or none, has other sizes in its head: nothing is done then, and its
// status says so.)
__device__ __forceinline__ bool plan_fits(const Params& p, const ListHead& h) {
  if (h.magic == kPlanMagic && h.M == p.M && h.n_slots == p.plan_slots) return true;
  if (blockIdx.x == 0 && threadIdx.x == 0) report_error(&p.plan->status, LQER_ERR_BAD_PACKED, 803);
  return false;
}
// The rank of a tile's adapter, 0 where the rows take none.
__device__ __forceinline__ int rank_of(const Params& p, int slot, const SlotHead& hd, bool tell) {
  if (slot < 0) return 0;
  if (hd.magic == kPoolMagic && hd.K == p.K && hd.N == p.N && hd.max_rank == p.max_rank && hd.rank >= 0 && hd.rank <= p.max_rank) return hd.rank;
  if (tell) report_error(&p.plan->status, LQER_ERR_BAD_PACKED, 804, slot);
  return 0;
}
__device__ __forceinline__ SlotHead load_slot(const uint8_t* slot) {
  const uint4 a = *reinterpret_cast<const uint4*>(slot);
  const uint2 b = *reinterpret_cast<const uint2*>(slot + 16);
  return SlotHead{a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, __uint_as_float(b.y), {0, 0}};
}

// ---------------------------------------------------------------------------- host
inline size_t slot_bytes(int K, int N, int max_rank) {
  return (256 + a_bytes(K, max_rank) + b_bytes(N, max_rank, b_pitch(max_rank)) + 255) & ~(size_t)255;
}
// A plan holds the rows in tiles of 8 for up to kFewMost of them, and in tiles of 128 for more than kManyLeast: in between the call
// chooses, by its work.  Both measured in bf16, few / many, us.  1024 rows: of 1264 x 1968 rank 32 9.6 / 14.7, of 4096 x 4096 rank 16
// 15.9 / 19.5, of 5120 x 5120 rank 32 21.2 / 22.3 (fp32: 29 / 34), of 4096 x 4096 rank 64 22.7 / 21.7, of 5120 x 5120 rank 128 43 / 29, of
// 4096 x 11008 rank 64 44 / 29.  513 rows: of 4096 x 4096 rank 64 14.3 / 18.5, of 4096 x 11008 rank 64 24.3 / 22.7, of 5120 x 5120 rank 128
// 24.9 / 22.5.
constexpr int kFewMost = 1024, kManyLeast = 512;
constexpr long long kFewWork = 350LL * 1000 * 1000;
inline bool takes_few(int M, int K, int N, int max_rank) {
  return M <= kManyLeast || (M <= kFewMost && (long long)M * (K + N) * max_rank <= kFewWork);
}
// No batch has more tiles than this: one that is not full per slot (and one of rows without), the rest are full.
inline int max_tiles(int M, int n_slots, int tile_rows) {
  const long long partial = n_slots + 1 < M ? n_slots + 1 : M, t = partial + M / tile_rows;
  return (int)(t < M ? t : M);
}
// Where a plan's lists lie: tiles and their rows, for few and for many rows.
struct PlanLayout {
  int tiles[2];
  size_t tiles_at[2], rows_at[2], bytes;
};
inline PlanLayout plan_layout(int M, int n_slots) {
  auto up = [](size_t v) { return (v + 255) & ~(size_t)255; };
  PlanLayout l;
  l.bytes = 256;
  for (int i = 0; i < 2; ++i) {
    const int rows = i == 0 ? kFewRows : kManyRows;
    l.tiles[i] = (i == 0 ? M <= kFewMost : M > kManyLeast) ? max_tiles(M, n_slots, rows) : 0;
    l.tiles_at[i] = l.bytes;
    l.rows_at[i] = l.tiles_at[i] + up((size_t)l.tiles[i] * sizeof(Tile));
    l.bytes = l.rows_at[i] + up((size_t)l.tiles[i] * rows * 4);
  }
  return l;
}

// The kernels for many rows: three launches, T in between in `scratch`.
size_t many_scratch_bytes(int tiles, int max_rank);
cudaError_t launch_many(const Params& p, int x_type, int tiles, void* scratch, cudaStream_t s);

}  // namespace ad
}  // namespace lqer
