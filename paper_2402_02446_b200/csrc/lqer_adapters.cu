// Low-rank adapters of many requests beside a shared projection:
//   Y[m] = Y0[m] + scale_a (X[m] A_a) B_a,   a = the slot of row m (none: Y[m] = Y0[m]).
// The same kind of term as the layer's own (X A_k) B_k (paper Section 3.1), with factors that differ from row to row.
//
// Pool: n_slots places of one size for adapters of a [K, N] projection up to max_rank, bf16 in the order in which mma.sync takes
// its B fragments, so that a lane reads 16 bytes per fragment pair and a warp 512 consecutive bytes:
//   A: [K / 32][rank / 8][lane][8]      lane (g, t) = (lane / 4, lane % 4): element i is A[32 kb + 8 t + i][8 n + g]
//   B: [N / 32][rank / 16][2][lane][8]  element 4 jj + i of half h is B[16 s + 4 t + i][32 nb + 8 (g / 2) + 2 (2 h + jj) + g % 2]
// The contraction index may be dealt to the MMA's K positions in any order as long as both operands agree, and the
// output columns to its N positions: dealt like this a lane's activations are 8 consecutive elements of a row, and its
// outputs 8 consecutive columns, so that X, Y0 and Y go between memory and registers in 16-byte pieces without shared memory.
//
// Plan: the rows sorted by slot (stable) and cut into tiles of at most tile_rows rows of one slot.  It belongs to a batch, not to a
// layer: a step of a model makes it once and uses it for every projection.
//
// A cluster of CTAs takes one tile.  First the CTAs share the contraction over K (each warp 16 rows), then they add up their
// partial T through distributed shared memory, and then they share the columns of Y.  X, A, B, Y0 and Y are touched once by a
// tile; T never leaves the chip.  The sums are taken in a fixed order.
//
// Precision: A, B and MXINT8 or bf16 X are exact in bf16.  fp32 X and T enter the tensor cores as sums of bf16 parts, cut off
// rather than rounded (no part can overflow): three parts hold all 24 bits, two parts 16 bits (2^-16, against 2^-9 for the
// bf16 result they are used for).
#include "lqer_tc_ptx.cuh"

namespace lqer {
namespace ad {

constexpr int kThreads = 256, kWarps = 8;
constexpr uint32_t kPoolMagic = 0x4C4F5241u, kPlanMagic = 0x4E414C50u;
constexpr int kMaxCluster = 8;

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
  int M, n_slots, tile_rows, n_tiles;
};
struct Tile { int slot, first, rows, reserved; };

__host__ __device__ inline size_t a_bytes(int K, int rank) { return (size_t)((K + 31) / 32) * ((rank + 7) / 8) * 512; }
__host__ __device__ inline size_t b_bytes(int N, int rank) { return (size_t)((N + 31) / 32) * ((rank + 15) / 16) * 1024; }

// ---------------------------------------------------------------------------- pool
__global__ void pool_init_kernel(uint8_t* pool, size_t slot_bytes, int n_slots, int K, int N, int max_rank) {
  const int s = blockIdx.x * blockDim.x + threadIdx.x;
  if (s < n_slots) *reinterpret_cast<SlotHead*>(pool + s * slot_bytes) = SlotHead{kPoolMagic, K, N, max_rank, 0, 0.f, {0, 0}};
}
__device__ __forceinline__ uint16_t to_bf16(const void* p, bool bf16, size_t i) {
  if (bf16) return static_cast<const uint16_t*>(p)[i];
  uint32_t d;
  const float v = static_cast<const float*>(p)[i];
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(0.f), "f"(v));
  return (uint16_t)d;
}
__global__ void adapter_load_kernel(uint8_t* slot, const void* A, const void* B, bool bf16, int K, int N, int max_rank, int rank, float scale) {
  const size_t stride = (size_t)gridDim.x * blockDim.x, first = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (first == 0) *reinterpret_cast<SlotHead*>(slot) = SlotHead{kPoolMagic, K, N, max_rank, rank, scale, {0, 0}};
  uint16_t* pa = reinterpret_cast<uint16_t*>(slot + 256);
  uint16_t* pb = reinterpret_cast<uint16_t*>(slot + 256 + a_bytes(K, max_rank));
  const int r8 = (rank + 7) / 8, r16 = (rank + 15) / 16;
  for (size_t e = first; e < a_bytes(K, rank) / 2; e += stride) {
    const int i = e & 7, lane = (e >> 3) & 31;
    const size_t blk = e >> 8;
    const int k = (int)(blk / r8) * 32 + (lane & 3) * 8 + i, r = (int)(blk % r8) * 8 + (lane >> 2);
    pa[e] = k < K && r < rank ? to_bf16(A, bf16, (size_t)k * rank + r) : (uint16_t)0;
  }
  for (size_t e = first; e < b_bytes(N, rank) / 2; e += stride) {
    const int i = e & 3, jj = (e >> 2) & 1, lane = (e >> 3) & 31, h = (e >> 8) & 1, g = lane >> 2;
    const size_t blk = e >> 9;
    const int r = (int)(blk % r16) * 16 + (lane & 3) * 4 + i, n = (int)(blk / r16) * 32 + (g >> 1) * 8 + 2 * (2 * h + jj) + (g & 1);
    pb[e] = n < N && r < rank ? to_bf16(B, bf16, (size_t)r * N + n) : (uint16_t)0;
  }
}

// ---------------------------------------------------------------------------- plan
// One CTA: a stable counting sort of the rows by slot (key n_slots: no adapter), then the tiles.  Each warp counts and places
// a stretch of rows of its own, with cursors of its own, so that only the prefix sums in between go over the whole CTA.
constexpr int kPlanThreads = 1024, kPlanWarps = 32;
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const int* __restrict__ slots, int M, int n_slots, int tile_rows, PlanHead* head,
                                                            Tile* tiles, int* order) {
  extern __shared__ int cursors[];                     // [bins][32 warps], then [bins + 1] tiles before a bin
  const int bins = n_slots + 1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int* tile_at = cursors + bins * kPlanWarps;
  __shared__ int bad, sums[kPlanWarps];
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  if (tid == 0) bad = 0;
  for (int i = tid; i < bins * kPlanWarps; i += kPlanThreads) cursors[i] = 0;
  __syncthreads();
  const int per = ((M + kPlanWarps - 1) / kPlanWarps + 31) / 32 * 32, lo = min(warp * per, M), hi = min(lo + per, M);
  auto key_of = [&](int row) {
    const int s = slots[row];
    if (s < -1 || s >= n_slots) bad = 1;
    return s < 0 || s >= n_slots ? n_slots : s;
  };
  for (int at = lo; at < hi; at += 32) {
    const int row = at + lane, key = row < hi ? key_of(row) : -1;
    const unsigned same = __match_any_sync(0xFFFFFFFFu, key);
    if (key >= 0 && lane == __ffs(same) - 1) cursors[key * kPlanWarps + warp] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  // exclusive sums over [bin][warp]: first within a thread's run of entries, then over the threads
  const int n = bins * kPlanWarps, run = (n + kPlanThreads - 1) / kPlanThreads, from = min(tid * run, n), to = min(from + run, n);
  auto scan = [&](int mine) {                          // exclusive prefix of `mine` over the CTA
    int x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xFFFFFFFFu, x, o); if (lane >= o) x += y; }
    __syncthreads();
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
      int v = sums[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xFFFFFFFFu, v, o); if (lane >= o) v += y; }
      sums[lane] = v;
    }
    __syncthreads();
    return x - mine + (warp > 0 ? sums[warp - 1] : 0);
  };
  int mine = 0;
  for (int i = from; i < to; ++i) mine += cursors[i];
  int before = scan(mine);
  for (int i = from; i < to; ++i) { const int c = cursors[i]; cursors[i] = before; before += c; }
  __syncthreads();
  // tiles: bin b holds rows [cursors[b][0], cursors[b + 1][0]) of the order
  const int brun = (bins + kPlanThreads - 1) / kPlanThreads, bfrom = min(tid * brun, bins), bto = min(bfrom + brun, bins);
  auto rows_of = [&](int b) { return (b + 1 < bins ? cursors[(b + 1) * kPlanWarps] : M) - cursors[b * kPlanWarps]; };
  int mine_t = 0;
  for (int b = bfrom; b < bto; ++b) mine_t += (rows_of(b) + tile_rows - 1) / tile_rows;
  int t0 = scan(mine_t);
  for (int b = bfrom; b < bto; ++b) {
    tile_at[b] = t0;
    const int rows = rows_of(b), first = cursors[b * kPlanWarps];
    for (int r = 0; r < rows; r += tile_rows) tiles[t0++] = Tile{b < n_slots ? b : -1, first + r, min(tile_rows, rows - r), 0};
  }
  if (bto == bins && bfrom < bins) tile_at[bins] = t0;
  __syncthreads();
  if (tid == 0) *head = PlanHead{DeviceStatus{bad ? (int)LQER_ERR_BOUNDS : 0, 801, 0, 0}, kPlanMagic, M, n_slots, tile_rows, tile_at[bins]};
  for (int at = lo; at < hi; at += 32) {
    const int row = at + lane, key = row < hi ? key_of(row) : -1;
    const unsigned same = __match_any_sync(0xFFFFFFFFu, key);
    if (key >= 0) order[cursors[key * kPlanWarps + warp] + __popc(same & ((1u << lane) - 1u))] = row;
    __syncwarp();
    if (key >= 0 && lane == __ffs(same) - 1) cursors[key * kPlanWarps + warp] += __popc(same);
    __syncwarp();
  }
}

// ---------------------------------------------------------------------------- the operator
struct Params {
  const void* X;
  const uint8_t* pool;
  PlanHead* plan;
  const Tile* tiles;
  const int* order;
  const void* Y0;
  void* Y;
  size_t slot_bytes;
  int M, K, N, max_rank, plan_slots, tile_rows;
  int y0_bf16, y_bf16;
  int bits, emin, emax;      // format of an MXINT8 X
  size_t y_extent;
};

// Floats from one row of partial sums to the next: the rows g of a fragment's stores lie 8 banks apart.
__host__ __device__ inline int part_stride(int max_rank) { return ((max_rank + 15) & ~15) + 8; }

__device__ __forceinline__ uint4 ld16(const void* p) { return __ldg(static_cast<const uint4*>(p)); }
__device__ __forceinline__ uint4 ld16_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The upper halves of two fp32 values (their leading bf16 parts, cut off) in one word.
__device__ __forceinline__ uint32_t top_halves(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
__device__ __forceinline__ float without_top(float v) {
  const float r = v - __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);      // exact
  return fabsf(v) == __uint_as_float(0x7F800000u) ? 0.f : r;                   // an infinity is all in its first part; NaN stays NaN
}
// P parts of two values: word p holds part p of both.
template <int P>
__device__ __forceinline__ void split(float a, float b, uint32_t (&w)[P]) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    w[p] = top_halves(a, b);
    if (p + 1 < P) { a = without_top(a); b = without_top(b); }
  }
}

// Eight consecutive activations of a row as raw bits, and as P words of bf16 pairs for each of the four pairs.
template <int XT>
struct XOct {
  uint4 a, b;                // fp32: both; bf16: a; MXINT8: a.x, a.y mantissas, a.z exponent byte
};
template <int XT>
__device__ __forceinline__ void load_x(XOct<XT>& o, const Params& p, int row, int col, bool in) {
  if (!in) {
    o.a = o.b = make_uint4(0u, 0u, 0u, 0u);
    if (XT == kXMXINT8) o.a.z = 127u;
    return;
  }
  const size_t idx = (size_t)row * p.K + col;
  if (XT == kXF32) {
    const float* x = static_cast<const float*>(p.X) + idx;
    o.a = ld16_once(x);
    o.b = ld16_once(x + 4);
  } else if (XT == kXBF16) {
    o.a = ld16_once(static_cast<const uint16_t*>(p.X) + idx);
  } else {
    const uint8_t* x = static_cast<const uint8_t*>(p.X);
    const uint2 m = __ldg(reinterpret_cast<const uint2*>(x + idx));
    o.a = make_uint4(m.x, m.y, __ldg(x + (size_t)p.M * p.K + (size_t)row * (p.K / 16) + (col >> 4)), 0u);
  }
}
template <int XT, int P>
__device__ __forceinline__ void pairs_of(const XOct<XT>& o, const Params& p, uint32_t (&w)[4][P]) {
  if (XT == kXF32) {
    split<P>(__uint_as_float(o.a.x), __uint_as_float(o.a.y), w[0]);
    split<P>(__uint_as_float(o.a.z), __uint_as_float(o.a.w), w[1]);
    split<P>(__uint_as_float(o.b.x), __uint_as_float(o.b.y), w[2]);
    split<P>(__uint_as_float(o.b.z), __uint_as_float(o.b.w), w[3]);
  } else if (XT == kXBF16) {
    w[0][0] = o.a.x; w[1][0] = o.a.y; w[2][0] = o.a.z; w[3][0] = o.a.w;
  } else {
    const float4 u = mxint_quad_values(o.a.x, o.a.z, p.bits, p.emin, p.emax), v = mxint_quad_values(o.a.y, o.a.z, p.bits, p.emin, p.emax);
    w[0][0] = top_halves(u.x, u.y); w[1][0] = top_halves(u.z, u.w);
    w[2][0] = top_halves(v.x, v.y); w[3][0] = top_halves(v.z, v.w);
  }
}

__device__ __forceinline__ void load_y0(const Params& p, int row, int col, float (&v)[8]) {
  const size_t idx = (size_t)row * p.N + col;
  if (p.y0_bf16) {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Y0) + idx);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  } else {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p.Y0) + idx);
    const float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}
__device__ __forceinline__ void store_y(const Params& p, int row, int col, const float (&v)[8]) {
  const size_t idx = (size_t)row * p.N + col;
  if (!LQER_IN_BOUNDS(&p.plan->status, idx * (p.y_bf16 ? 2 : 4), p.y_bf16 ? 16 : 32, p.y_extent, 802)) return;
  if (p.y_bf16) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.Y) + idx) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p.Y) + idx);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}
__device__ __forceinline__ float4 ld_dsmem_f4(const float* p, uint32_t cta) {
  float4 v;
  asm volatile("{\n .reg .b32 ra;\n mapa.shared::cluster.u32 ra, %4, %5;\n ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [ra];\n}\n"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(tc::smem_u32(p)), "r"(cta) : "memory");
  return v;
}

// XP, TP: bf16 parts of X and of T.  WR: warps along the rows (16 each); the other kWarps / WR share the contraction over K, and
// later the columns.  RC8: octets of the rank that a pass over X takes.
template <int XT, int XP, int TP, int WR, int RC8>
__global__ void __launch_bounds__(kThreads, 2) adapters_kernel(const Params p) {
  constexpr int WK = kWarps / WR, ROWS = 16 * WR;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int rows[ROWS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int wr = warp % WR, wk = warp / WR;
  uint32_t c;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(c));
  const uint32_t q = tc::cluster_rank();
  const int tile_id = blockIdx.x / c;
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  // A plan of another batch (or none) has other sizes in its head: nothing is done then, and its status says so.
  if (p.plan->magic != kPlanMagic || p.plan->M != p.M || p.plan->n_slots != p.plan_slots || p.plan->tile_rows != ROWS) {
    if (blockIdx.x == 0 && tid == 0) report_error(&p.plan->status, LQER_ERR_BAD_PACKED, 803);
    return;
  }
  if (tile_id >= p.plan->n_tiles) return;               // the whole cluster
  const Tile tile = p.tiles[tile_id];
  const uint8_t* slot = p.pool + (size_t)max(tile.slot, 0) * p.slot_bytes;
  const SlotHead hd = *reinterpret_cast<const SlotHead*>(slot);
  const bool known = hd.magic == kPoolMagic && hd.K == p.K && hd.N == p.N && hd.max_rank == p.max_rank && hd.rank >= 0 && hd.rank <= p.max_rank;
  if (tile.slot >= 0 && !known && q == 0 && tid == 0) report_error(&p.plan->status, LQER_ERR_BAD_PACKED, 804, tile.slot);
  const int rank = tile.slot >= 0 && known ? hd.rank : 0;
  if (tid < ROWS) rows[tid] = p.order[tile.first + min(tid, tile.rows - 1)];
  __syncthreads();
  const int NB = (p.N + 31) / 32, nb_lo = NB * q / c, nb_hi = NB * (q + 1) / c;
  if (rank == 0) {                                      // no adapter: the rows as they are
    if (p.Y0 == p.Y) return;
    const int octets = min(nb_hi * 4, p.N / 8) - nb_lo * 4;
    for (int i = warp; i < tile.rows; i += kWarps)
      for (int o = lane; o < octets; o += 32) {
        float v[8];
        load_y0(p, rows[i], (nb_lo * 4 + o) * 8, v);
        store_y(p, rows[i], (nb_lo * 4 + o) * 8, v);
      }
    return;
  }
  const int r8 = (rank + 7) / 8, r16 = (rank + 15) / 16, ld = part_stride(p.max_rank);
  float* part = reinterpret_cast<float*>(smem);                        // [WK][ROWS][ld]; the first becomes the CTA's sum,
  uint4* frags = reinterpret_cast<uint4*>(part + (size_t)ROWS * ld);   // the others make room for [WR][rank / 16][TP][lane]
  const int row_a = rows[wr * 16 + g], row_b = rows[wr * 16 + g + 8];

  // ---- T's share of this CTA: K blocks of 32, dealt to the warps in turn
  const int KB = (p.K + 31) / 32, kb_lo = KB * q / c, kb_hi = KB * (q + 1) / c;
  const uint8_t* A = slot + 256;
  for (int n0 = 0; n0 < r8; n0 += RC8) {
    const int nn = min(RC8, r8 - n0);
    float acc[RC8][4];
#pragma unroll
    for (int j = 0; j < RC8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    XOct<XT> xa, xb;
    int kb = kb_lo + wk;
    bool in = kb < kb_hi && kb * 32 + 8 * t < p.K;
    load_x<XT>(xa, p, row_a, kb * 32 + 8 * t, in);
    load_x<XT>(xb, p, row_b, kb * 32 + 8 * t, in);
    for (; kb < kb_hi; kb += WK) {
      uint4 f[RC8];
#pragma unroll
      for (int j = 0; j < RC8; ++j)
        if (j < nn) f[j] = ld16(A + ((size_t)kb * r8 + n0 + j) * 512 + lane * 16);
      uint32_t wa[4][XP], wb[4][XP];
      pairs_of<XT, XP>(xa, p, wa);
      pairs_of<XT, XP>(xb, p, wb);
      const int next = kb + WK;
      in = next < kb_hi && next * 32 + 8 * t < p.K;
      load_x<XT>(xa, p, row_a, next * 32 + 8 * t, in);
      load_x<XT>(xb, p, row_b, next * 32 + 8 * t, in);
#pragma unroll
      for (int j = 0; j < RC8; ++j)
        if (j < nn) {
#pragma unroll
          for (int x = 0; x < XP; ++x) {
            const uint32_t a0[4] = {wa[0][x], wb[0][x], wa[1][x], wb[1][x]}, a1[4] = {wa[2][x], wb[2][x], wa[3][x], wb[3][x]};
            mma(acc[j], a0, f[j].x, f[j].y);
            mma(acc[j], a1, f[j].z, f[j].w);
          }
        }
    }
    float* mine = part + ((size_t)wk * ROWS + wr * 16) * ld + n0 * 8;
#pragma unroll
    for (int j = 0; j < RC8; ++j)
      if (j < nn) {
        *reinterpret_cast<float2*>(mine + (size_t)g * ld + j * 8 + 2 * t) = make_float2(acc[j][0], acc[j][1]);
        *reinterpret_cast<float2*>(mine + (size_t)(g + 8) * ld + j * 8 + 2 * t) = make_float2(acc[j][2], acc[j][3]);
      }
  }
  __syncthreads();
  // ---- the CTA's sum, then the cluster's: every CTA reads all of them, in order
  const int quads = r8 * 2;
  if (WK > 1) {
    for (int i = tid; i < ROWS * quads; i += kThreads) {
      float4* at = reinterpret_cast<float4*>(part + (size_t)(i / quads) * ld) + i % quads;
      float4 s = *at;
      for (int w = 1; w < WK; ++w) {
        const float4 v = *reinterpret_cast<float4*>(reinterpret_cast<float*>(at) + (size_t)w * ROWS * ld);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      *at = s;
    }
  }
  tc::cluster_barrier();
  // T's element (row, 16 s + 4 t + i) belongs to lane (row % 8, t) of the row's warp: registers row / 8 and 2 + row / 8
  for (int i = tid; i < ROWS * r16 * 4; i += kThreads) {
    const int row = i / (r16 * 4), quad = i % (r16 * 4);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (quad < quads)
      for (uint32_t k = 0; k < c; ++k) {
        const float4 v = ld_dsmem_f4(part + (size_t)row * ld + quad * 4, k);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
    // beyond the rank the packed A holds zeros, and an infinite activation times zero is no zero
    const int past = quad * 4 + 4 - rank;
    if (past > 0) { s.w = 0.f; if (past > 1) s.z = 0.f; if (past > 2) s.y = 0.f; if (past > 3) s.x = 0.f; }
    uint32_t lo[TP], hi[TP];
    split<TP>(s.x * hd.scale, s.y * hd.scale, lo);
    split<TP>(s.z * hd.scale, s.w * hd.scale, hi);
    uint32_t* f = reinterpret_cast<uint32_t*>(frags + ((size_t)(row / 16) * r16 + quad / 4) * TP * 32 + (row % 8) * 4 + quad % 4) + (row / 8) % 2;
#pragma unroll
    for (int x = 0; x < TP; ++x) { f[x * 128] = lo[x]; f[x * 128 + 2] = hi[x]; }
  }
  // no CTA leaves while its sums may still be read
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  __syncthreads();
  // ---- the CTA's columns of Y: blocks of 32, dealt to the warps in turn
  const uint8_t* B = slot + 256 + a_bytes(p.K, p.max_rank);
  const uint4* fr = frags + (size_t)wr * r16 * TP * 32 + lane;
  const bool has_a = wr * 16 + g < tile.rows, has_b = wr * 16 + g + 8 < tile.rows;
  for (int nb = nb_lo + wk; nb < nb_hi; nb += WK) {
    const int col = nb * 32 + 8 * t;
    const bool in = col < p.N;
    float ya[8], yb[8];
    if (in && has_a) load_y0(p, row_a, col, ya);
    if (in && has_b) load_y0(p, row_b, col, yb);
    float acc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    const uint8_t* b = B + (size_t)nb * r16 * 1024 + lane * 16;
    for (int s = 0; s < r16; ++s) {
      const uint4 b0 = ld16(b + s * 1024), b1 = ld16(b + s * 1024 + 512);
#pragma unroll
      for (int x = 0; x < TP; ++x) {
        const uint4 v = fr[(s * TP + x) * 32];
        const uint32_t a[4] = {v.x, v.y, v.z, v.w};
        mma(acc[0], a, b0.x, b0.y);
        mma(acc[1], a, b0.z, b0.w);
        mma(acc[2], a, b1.x, b1.y);
        mma(acc[3], a, b1.z, b1.w);
      }
    }
    if (in && has_a) {
#pragma unroll
      for (int j = 0; j < 4; ++j) { ya[2 * j] += acc[j][0]; ya[2 * j + 1] += acc[j][1]; }
      store_y(p, row_a, col, ya);
    }
    if (in && has_b) {
#pragma unroll
      for (int j = 0; j < 4; ++j) { yb[2 * j] += acc[j][2]; yb[2 * j + 1] += acc[j][3]; }
      store_y(p, row_b, col, yb);
    }
  }
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------- host
inline size_t slot_bytes(int K, int N, int max_rank) { return (256 + a_bytes(K, max_rank) + b_bytes(N, max_rank) + 255) & ~(size_t)255; }
inline int tile_rows_of(int M) { return M <= 512 ? 16 : 64; }
// No batch has more tiles than this: one that is not full per slot (and one of rows without), the rest are full.
inline int max_tiles(int M, int n_slots) {
  const int rows = tile_rows_of(M), partial = n_slots + 1 < M ? n_slots + 1 : M;
  const long long t = (long long)partial + M / rows;
  return (int)(t < M ? t : M);
}

template <int XT, int XP, int TP, int WR, int RC8>
static cudaError_t launch(const Params& p, int clusters, int c, cudaStream_t s) {
  constexpr int WK = kWarps / WR, ROWS = 16 * WR;
  const size_t sums = (size_t)ROWS * part_stride(p.max_rank) * 4, frags = (size_t)WR * ((p.max_rank + 15) / 16) * TP * 512;
  const size_t smem = sums + ((WK - 1) * sums > frags ? (WK - 1) * sums : frags);
  static OncePerDevice once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(adapters_kernel<XT, XP, TP, WR, RC8>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(clusters * c));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = c; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  LaunchScope scope(kFamDecode, s);
  return cudaLaunchKernelEx(&cfg, adapters_kernel<XT, XP, TP, WR, RC8>, p);
}
template <int XT, int XP, int TP>
static cudaError_t launch_rows(const Params& p, int clusters, int c, cudaStream_t s) {
  if (p.tile_rows == 16) return p.max_rank <= 16 ? launch<XT, XP, TP, 1, 2>(p, clusters, c, s) : launch<XT, XP, TP, 1, 8>(p, clusters, c, s);
  return p.max_rank <= 16 ? launch<XT, XP, TP, 4, 2>(p, clusters, c, s) : launch<XT, XP, TP, 4, 8>(p, clusters, c, s);
}

}  // namespace ad

size_t adapter_slot_bytes(int K, int N, int max_rank) { return ad::slot_bytes(K, N, max_rank); }
size_t adapter_plan_bytes(int M, int n_slots) {
  return 256 + (((size_t)ad::max_tiles(M, n_slots) * sizeof(ad::Tile) + 255) & ~(size_t)255) + (((size_t)M * 4 + 255) & ~(size_t)255);
}
cudaError_t launch_adapter_pool_init(void* pool, int K, int N, int max_rank, int n_slots, cudaStream_t s) {
  LaunchScope scope(kFamPack, s);
  ad::pool_init_kernel<<<(n_slots + 255) / 256, 256, 0, s>>>(static_cast<uint8_t*>(pool), ad::slot_bytes(K, N, max_rank), n_slots, K, N, max_rank);
  return cudaGetLastError();
}
cudaError_t launch_adapter_load(void* pool, int K, int N, int max_rank, int slot, const void* A, const void* B, bool bf16, int rank, float scale,
                                cudaStream_t s) {
  LaunchScope scope(kFamPack, s);
  ad::adapter_load_kernel<<<rank > 0 ? 2 * sm_count() : 1, 256, 0, s>>>(static_cast<uint8_t*>(pool) + (size_t)slot * ad::slot_bytes(K, N, max_rank), A, B,
                                                                       bf16, K, N, max_rank, rank, scale);
  return cudaGetLastError();
}
cudaError_t launch_adapter_plan(const int* slots, int M, int n_slots, void* plan, cudaStream_t s) {
  uint8_t* at = static_cast<uint8_t*>(plan);
  ad::Tile* tiles = reinterpret_cast<ad::Tile*>(at + 256);
  int* order = reinterpret_cast<int*>(at + 256 + (((size_t)ad::max_tiles(M, n_slots) * sizeof(ad::Tile) + 255) & ~(size_t)255));
  const size_t smem = (size_t)(n_slots + 1) * ad::kPlanWarps * 4 + (size_t)(n_slots + 2) * 4;
  static OncePerDevice once;
  cudaError_t e = once.run([] { return cudaFuncSetAttribute(ad::plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1);
  cfg.blockDim = dim3(ad::kPlanThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  LaunchScope scope(kFamDecode, s);
  return cudaLaunchKernelEx(&cfg, ad::plan_kernel, slots, M, n_slots, ad::tile_rows_of(M), reinterpret_cast<ad::PlanHead*>(at), tiles, order);
}
cudaError_t launch_adapters(const void* X, int x_type, int M, const void* pool, int K, int N, int max_rank, void* plan, int plan_slots,
                            const void* Y0, int y0_type, void* Y, int y_type, int bits, int emin, int emax, cudaStream_t s) {
  uint8_t* at = static_cast<uint8_t*>(plan);
  const int most = ad::max_tiles(M, plan_slots);
  ad::Params p;
  p.X = X; p.pool = static_cast<const uint8_t*>(pool);
  p.plan = reinterpret_cast<ad::PlanHead*>(at);
  p.tiles = reinterpret_cast<const ad::Tile*>(at + 256);
  p.order = reinterpret_cast<const int*>(at + 256 + (((size_t)most * sizeof(ad::Tile) + 255) & ~(size_t)255));
  p.Y0 = Y0; p.Y = Y;
  p.slot_bytes = ad::slot_bytes(K, N, max_rank);
  p.M = M; p.K = K; p.N = N; p.max_rank = max_rank; p.plan_slots = plan_slots; p.tile_rows = ad::tile_rows_of(M);
  p.y0_bf16 = y0_type == kYBF16; p.y_bf16 = y_type == kYBF16;
  p.bits = bits; p.emin = emin; p.emax = emax;
  const size_t whole = y_bytes(y_type, M, N), less = debug_y_shrink();
  p.y_extent = whole > less ? whole - less : 0;
  // CTAs to a tile: as many as give every SM two, but no fewer than one K block and one column block to a warp of each.
  const int wk = p.tile_rows == 16 ? 8 : 2, full = (M + p.tile_rows - 1) / p.tile_rows;
  int c = ad::kMaxCluster;
  while (c > 1 && (p.tile_rows > 16 && full * c > 2 * sm_count())) c /= 2;
  while (c > 1 && (K + 31) / 32 < c * wk && (N + 31) / 32 < c * wk) c /= 2;
  if (x_type == kXF32)
    return p.y_bf16 ? ad::launch_rows<kXF32, 2, 2>(p, most, c, s) : ad::launch_rows<kXF32, 3, 3>(p, most, c, s);
  if (x_type == kXBF16)
    return p.y_bf16 ? ad::launch_rows<kXBF16, 1, 2>(p, most, c, s) : ad::launch_rows<kXBF16, 1, 3>(p, most, c, s);
  return p.y_bf16 ? ad::launch_rows<kXMXINT8, 1, 2>(p, most, c, s) : ad::launch_rows<kXMXINT8, 1, 3>(p, most, c, s);
}

}  // namespace lqer
