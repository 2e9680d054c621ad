// Low-rank adapters of many requests beside a shared projection:
//   Y[m] = Y0[m] + scale_a (X[m] A_a) B_a,   a = the slot of row m (none: Y[m] = Y0[m]).
// The same kind of term as the layer's own (X A_k) B_k (paper Section 3.1), with factors that differ from row to row.
//
// Pool: n_slots places of one size for adapters of a [K, N] projection up to max_rank, bf16, both factors with the contraction index
// innermost, in the images that the tensor cores read from shared memory (128-byte swizzle: the 16-byte pieces of a row change
// places by the row's index):
//   A: [K / 64][rank, padded to 16] rows of 64 K
//   B: [N / 128][rank / 64][128 columns] rows of 64 ranks (32 or 16 where max_rank is no more: rows of 64 or 32 bytes); column
//      8 t + 2 j + i of 32 is row 8 j + 2 t + i: of an accumulator's columns, which a lane holds in pairs, it then has 8 neighbours
// They are read as they lie: by bulk copies for the tcgen05 kernels, and for mma.sync in 16-byte pieces, a lane's eight consecutive
// elements being its share of two MMA steps (the contraction index may be dealt to the MMA's K positions in any order as long as
// both operands agree).
//
// Plan: the rows sorted by slot (stable) and cut into tiles of at most tile_rows rows of one slot.  It belongs to a batch, not to a
// layer: a step of a model makes it once and uses it for every projection.
//
// Few rows (up to 512, and up to 1024 of small products; few_rows_kernel): a cluster of CTAs takes a tile of up to 8 rows.  The factors are the MMA's 16-row operand, the tokens its 8
// columns.  First the CTAs share the contraction over K, then each sends its part of T to all (distributed shared memory),
// and then they share the columns of Y.  T never leaves the chip, and everything is summed in a fixed order.
// Measured: one row of 4096 x 4096 rank 16 5.1 us, 64 rows of 24 adapters of 5120 x 5120 rank 16 in bf16 7.5 us, 16 rows of as many
// adapters of 4096 x 11008 rank 64 (MXINT8 to fp32) 12.1 us, 1.3 TB/s.  What bounds them is the chain of a tile: plan, slot, A and
// X, the exchange of T, B - some seven trips to memory one after the other - and not bytes (2.5 us of the 12.1) or instructions (a fifth of
// the issue slots).  With more tiles than fit the device at once it is the tiles of eight rows, each of which reads its adapter whole:
// 256 rows of 4 adapters of 4096 x 11008 rank 64 in bf16 21.6 us, 512 rows 31.7.  The plan, one CTA: 3.7 us for 64 rows, 7.5 us for 4096.
// Many rows: lqer_adapters_many.cu.
//
// Precision: A, B and MXINT8 or bf16 X are exact in bf16.  fp32 X and T (summed in fp32) enter the tensor cores as sums of bf16 parts:
// for fp32 Y three, which hold all 24 bits, for bf16 Y two, rounded to nearest (2^-17 of each value, against 2^-8 for the bf16 result;
// three there as well: 2048 rows of 4096 x 11008 rank 64 in bf16 38.0 -> 40.8 us, rank 128 47.7 -> 58.3, 201 rows of 4112 x 10992 rank 20
// fp32 to bf16 12.6 -> 14.2).  The tensor cores cut a running sum off where it does not fit, so their chains are kept
// short, lower parts first, and added up by ordinary fp32 additions.  A chain is, for few rows: 32 of K and the parts of X (then fp32 additions),
// all ranks and parts of T; for many rows: up to 2048 of K and one part of X - all three parts of an fp32 X where the rank is beyond 160,
// for which tensor memory has no room apart - and all ranks and parts of T.
#include "lqer_adapters.cuh"

namespace lqer {
namespace ad {

constexpr int kThreads = 256, kWarps = 8;

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
// (A thread writes two bytes at a time, wherever they belong: loading is not on a step's path.  Rank 16 of 4096 x 4096 3 us, rank 64 of
// 4096 x 11008 11.8 us, rank 256 of 5120 x 13824 45 us.)
__global__ void adapter_load_kernel(uint8_t* slot, const void* A, const void* B, bool bf16, int K, int N, int max_rank, int rank, float scale) {
  const size_t stride = (size_t)gridDim.x * blockDim.x, first = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (first == 0) *reinterpret_cast<SlotHead*>(slot) = SlotHead{kPoolMagic, K, N, max_rank, rank, scale, {0, 0}};
  uint8_t* pa = slot + 256;
  uint8_t* pb = slot + 256 + a_bytes(K, max_rank);
  const int rows = rank16(rank) * 16, pitch = b_pitch(max_rank), wide = pitch / 2, slabs = (rank + 63) / 64;
  // a thread writes one element; consecutive threads read consecutive ones of A's and B's rows
  const size_t na = (size_t)((K + 63) / 64) * 64 * rows;
  for (size_t e = first; e < na; e += stride) {
    const int r = (int)(e % rows), k = (int)(e / rows);
    const uint16_t v = k < K && r < rank ? to_bf16(A, bf16, (size_t)k * rank + r) : (uint16_t)0;
    *reinterpret_cast<uint16_t*>(pa + (size_t)(k / 64) * rows * 128 + swizzled(r, (k % 64) / 8, 128) + (k % 8) * 2) = v;
  }
  const size_t cols = (size_t)((N + 127) / 128) * 128, nb = cols * slabs * wide;
  for (size_t e = first; e < nb; e += stride) {
    const int n = (int)(e % cols), r = (int)(e / cols);
    const uint16_t v = n < N && r < rank ? to_bf16(B, bf16, (size_t)r * N + n) : (uint16_t)0;
    *reinterpret_cast<uint16_t*>(pb + ((size_t)(n / 128) * slabs + r / wide) * 128 * pitch + swizzled(image_row(n % 128), (r % wide) / 8, pitch) + (r % 8) * 2) = v;
  }
}

// ---------------------------------------------------------------------------- plan
// One CTA: a stable counting sort of the rows by slot (key n_slots: no adapter), cut into tiles twice: of 8 rows and of 128 (either list
// may be left out).  Each warp counts and places a stretch of rows of its own, with cursors of its own, so that only the prefix
// sums in between go over the whole CTA.
struct PlanList {
  Tile* tiles;
  int* rows;                 // an entry for each row of each tile; places behind a tile's last row name that row again
  int tile_rows;             // 0: no such list
};
constexpr int kPlanThreads = 1024, kPlanWarps = 32;
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const int* __restrict__ slots, int M, int n_slots, PlanHead* head, const PlanList few,
                                                            const PlanList many) {
  extern __shared__ int cursors[];                     // [bins][32 warps], then [bins] rows before a bin and, for both lists, [bins + 1] tiles before it
  const int bins = n_slots + 1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int* first_of = cursors + bins * kPlanWarps;
  int* tile_at[2] = {first_of + bins, first_of + 2 * bins + 1};
  const PlanList lists[2] = {few, many};
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
  for (int b = bfrom; b < bto; ++b) first_of[b] = cursors[b * kPlanWarps];
#pragma unroll
  for (int l = 0; l < 2; ++l) {
    const int per = lists[l].tile_rows;
    if (per == 0) continue;
    int mine_t = 0;
    for (int b = bfrom; b < bto; ++b) mine_t += (rows_of(b) + per - 1) / per;
    int t0 = scan(mine_t);
    for (int b = bfrom; b < bto; ++b) {
      tile_at[l][b] = t0;
      const int n_rows = rows_of(b);
      for (int r = 0; r < n_rows; r += per) lists[l].tiles[t0++] = Tile{b < n_slots ? b : -1, min(per, n_rows - r)};
    }
    if (bto == bins && bfrom < bins) tile_at[l][bins] = t0;
  }
  __syncthreads();
  if (tid == 0) {
    head->status = DeviceStatus{bad ? (int)LQER_ERR_BOUNDS : 0, 801, 0, 0};
    head->magic = kPlanMagic;
    head->M = M;
    head->n_slots = n_slots;
#pragma unroll
    for (int l = 0; l < 2; ++l) {
      head->of[l].n_tiles = lists[l].tile_rows > 0 ? tile_at[l][bins] : 0;
      head->of[l].n_adapted = lists[l].tile_rows > 0 ? tile_at[l][n_slots] : 0;
    }
  }
  for (int at = lo; at < hi; at += 32) {
    const int row = at + lane, key = row < hi ? key_of(row) : -1;
    const unsigned same = __match_any_sync(0xFFFFFFFFu, key);
    if (key >= 0) {
      const int place = cursors[key * kPlanWarps + warp] + __popc(same & ((1u << lane) - 1u)) - first_of[key];
      const int end = (key + 1 < bins ? first_of[key + 1] : M) - first_of[key];
#pragma unroll
      for (int l = 0; l < 2; ++l) {
        const int per = lists[l].tile_rows;
        if (per == 0) continue;
        int* at_tile = lists[l].rows + ((size_t)tile_at[l][key] + place / per) * per;
        at_tile[place % per] = row;
        if (place + 1 == end)
          for (int i = place % per + 1; i < per; ++i) at_tile[i] = row;
      }
    }
    __syncwarp();
    if (key >= 0 && lane == __ffs(same) - 1) cursors[key * kPlanWarps + warp] += __popc(same);
    __syncwarp();
  }
}

// ---------------------------------------------------------------------------- few rows
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void st_dsmem_f4(float* p, uint32_t cta, const float4& v) {
  asm volatile("{\n .reg .b32 ra;\n mapa.shared::cluster.u32 ra, %0, %1;\n st.shared::cluster.v4.f32 [ra], {%2, %3, %4, %5};\n}\n"
               ::"r"(tc::smem_u32(p)), "r"(cta), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// XP, TP: bf16 parts of X and of T.  PITCH: bytes of a row of B's image.  The MMA's eight columns are tokens;
// where the tile has so few that the parts fit side by side (two tokens of three parts, four of two) they are tokens and parts, and
// one MMA takes the place of two or three: column = token + part * 2 (or 4).
__host__ __device__ constexpr int side_by_side(int parts) { return parts == 1 ? 8 : parts == 2 ? 4 : 2; }
// Floats from one column of partial sums to the next: a fragment's stores then go to 32 different banks.
__host__ __device__ inline int part_stride(int max_rank) { return rank16(max_rank) * 16 + 4; }

// A warp's ring of the factors' pieces: at rank 128 and eight CTAs to a tile two CTAs still fit an SM.
__host__ __device__ constexpr int ring_sets(int pitch) { return pitch == 32 ? 4 : 3; }
__host__ __device__ constexpr int ring_set_bytes(int pitch) { return pitch == 32 ? 1024 : 2048; }

template <int XT, int XP, int TP, int PITCH>
__global__ void __launch_bounds__(kThreads, 2) few_rows_kernel(const Params p) {
  constexpr int RB = PITCH == 32 ? 16 : 32;             // ranks of a step of B
  constexpr int XS = side_by_side(XP), TS = side_by_side(TP);
  constexpr int RC = PITCH == 32 ? 1 : PITCH == 64 ? 2 : 4;                  // sixteens of the rank that one pass over X takes
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  uint32_t c;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(c));
  const uint32_t q = tc::cluster_rank();
  const int tile_id = blockIdx.x / c;
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  // the head first: the lists of another batch's plan may be shorter than this grid (0.1 us of a call, against loads side by side)
  const ListHead head = load_head(p.plan, 0);
  if (!plan_fits(p, head) || tile_id >= head.n_tiles) return;            // the whole cluster
  const Tile tile = p.tiles[tile_id];
  const int row_g = p.rows[tile_id * kFewRows + g];
  const int row_0 = p.rows[tile_id * kFewRows + 2 * t], row_1 = p.rows[tile_id * kFewRows + 2 * t + 1];
  const uint8_t* slot = p.pool + (size_t)max(tile.slot, 0) * p.slot_bytes;
  const SlotHead hd = load_slot(slot);
  const int rank = rank_of(p, tile.slot, hd, q == 0 && tid == 0);
  const int NB = (p.N + 31) / 32, nb_lo = NB * q / c, nb_hi = NB * (q + 1) / c;
  if (rank == 0) {                                      // no adapter: the rows as they are
    if (p.Y0 == p.Y) return;
    const int quads = min(nb_hi * 8, p.N / 4) - nb_lo * 8;
    const size_t at = (size_t)p.rows[tile_id * kFewRows + warp % kFewRows] * p.N + nb_lo * 32;
    if (warp % kFewRows < tile.rows)
      for (int o = lane + warp / kFewRows * 32; o < quads; o += kWarps / kFewRows * 32) {
        Y0Quad y;
        y.load(p, at + o * 4);
        store_y(p, at + o * 4, y.values(p));
      }
    return;
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");    // waited for before the first remote store
  const int r16 = rank16(rank), ld = part_stride(p.max_rank);
  float* part = reinterpret_cast<float*>(smem);         // [two warps][column][ld], and then [lane][...] the fragments of T
  float* sums = part + kWarps / 2 * 8 * ld;              // [CTA of the cluster][token][ld]
  const uint8_t* A = slot + 256;
  const uint8_t* B = slot + 256 + a_bytes(p.K, p.max_rank);

  // ---- The factors' pieces, first of A and then of B, come through a ring of the warp's own in shared memory, AHEAD sets ahead of their
  // use; a lane reads what it copied itself.  So the first of B are on their way while T is being exchanged.
  // A set is a step of B's 32 columns, or two sixteens of A's ranks.
  constexpr int AHEAD = ring_sets(PITCH), SET = ring_set_bytes(PITCH);
  const int KB = (p.K + 31) / 32, kb_lo = KB * q / c, kb_hi = KB * (q + 1) / c;
  const int slabs = (rank + 63) / 64, steps = (rank + RB - 1) / RB;
  const uint8_t* ring = reinterpret_cast<const uint8_t*>(sums + c * 8 * ld) + warp * AHEAD * SET;
  const uint8_t* a_lane = A + g * 128;                  // ranks g and, 1024 bytes on, g + 8; the swizzle's share is the row's index, g
  const uint32_t piece0 = (t ^ (g & 3)) << 4, flip = (g & 4) << 4;
  int s_n0 = kb_lo + warp < kb_hi ? 0 : r16, s_j = 0, s_kb = kb_lo + warp, s_nb = nb_lo + warp, s_step = 0, s_set = 0, set = 0;
  auto send = [&]() {
    const uint32_t to = tc::smem_u32(ring + s_set * SET);
    if (s_n0 < r16) {
      const uint8_t* a = a_lane + ((size_t)(s_kb >> 1) * r16 + s_n0 + s_j) * 2048 + (piece0 | (flip ^ (s_kb & 1) << 6));
#pragma unroll
      for (int j = 0; j < (RC > 1 ? 2 : 1); ++j)
        if (s_n0 + s_j + j < r16) {
          copy_async<16>(to + (2 * j * 32 + lane) * 16, a + j * 2048);
          copy_async<16>(to + ((2 * j + 1) * 32 + lane) * 16, a + j * 2048 + 1024);
        }
      s_j += 2;
      if (s_j >= RC || s_n0 + s_j >= r16) {
        s_j = 0;
        s_kb += kWarps;
        if (s_kb >= kb_hi) { s_kb = kb_lo + warp; s_n0 += RC; }
      }
    } else if (s_nb < nb_hi) {
      // column 4 g + i of 32 of the block; the swizzle goes by the image's row modulo 8
      const int half = PITCH == 128 ? s_step & 1 : 0;
      const uint8_t* b = B + ((size_t)(s_nb >> 2) * slabs + (PITCH == 128 ? s_step >> 1 : 0)) * 128 * PITCH +
                         ((s_nb & 3) * 32 + 16 * (g & 1) + 2 * (g >> 1)) * PITCH;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t row = 2 * (g >> 1) + (i & 1), at = (8 * (i >> 1) + (i & 1)) * PITCH;
        if (PITCH > 32) copy_async<16>(to + (i * 32 + lane) * 16, b + at + (((half * 4 + t) ^ (PITCH == 128 ? row : row >> 1)) << 4));
        else copy_async<8>(to + (i * 32 + lane) * 8, b + at + (((t >> 1) ^ (row >> 2)) << 4) + (t & 1) * 8);
      }
      if (++s_step == steps) { s_step = 0; s_nb += kWarps; }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    s_set = s_set + 1 == AHEAD ? 0 : s_set + 1;
  };
  auto arrived = [&]() {                                // the oldest set under way
    asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
    const uint8_t* at = ring + set * SET;
    set = set + 1 == AHEAD ? 0 : set + 1;
    return at;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) send();

  // ---- T's share of this CTA: K blocks of 32, dealt to the warps in turn.  Factor rows (ranks) g and g + 8 of each sixteen, tokens g.
  const bool xpack = XP > 1 && tile.rows <= XS;
  const int x_row = xpack ? __shfl_sync(0xFFFFFFFFu, row_g, (g % XS) * 4) : row_g, x_part = g / XS;
  for (int n0 = 0; n0 < r16; n0 += RC) {
    const int nn = min(RC, r16 - n0);
    float acc[RC][4];
#pragma unroll
    for (int j = 0; j < RC; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    XOct<XT> x;
    int kb = kb_lo + warp;
    x.load(p, x_row, kb * 32 + 8 * t, kb < kb_hi && kb * 32 + 8 * t < p.K);
    for (; kb < kb_hi; kb += kWarps) {
      uint32_t w[4][XP];
      x.template pairs<XP>(p, w);
      const int next = kb + kWarps;
      x.load(p, x_row, next * 32 + 8 * t, next < kb_hi && next * 32 + 8 * t < p.K);
      if (xpack) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t m = 0;
#pragma unroll
          for (int k = 0; k < XP; ++k) m = x_part == k ? w[i][k] : m;
          w[i][0] = m;
        }
      }
#pragma unroll
      for (int j0 = 0; j0 < RC; j0 += 2)
        if (j0 < nn) {
          const uint4* f = reinterpret_cast<const uint4*>(arrived()) + lane;
#pragma unroll
          for (int j = j0; j < j0 + (RC > 1 ? 2 : 1); ++j)
            if (j < nn) {
              const uint4 f0 = f[2 * (j - j0) * 32], f1 = f[(2 * (j - j0) + 1) * 32];
              float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int k = XP - 1; k >= 0; --k)
                if (k == 0 || !xpack) {
                  mma(d, f0.x, f1.x, f0.y, f1.y, w[0][k], w[1][k]);
                  mma(d, f0.z, f1.z, f0.w, f1.w, w[2][k], w[3][k]);
                }
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[j][i] += d[i];
            }
          send();
        }
    }
    // four places of partial sums: the upper four warps add theirs to the lower four's
    float* mine = part + ((warp & 3) * 8 + 2 * t) * ld + n0 * 16 + g;
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
      if (warp >> 2 == turn) {
#pragma unroll
        for (int j = 0; j < RC; ++j)
          if (j < nn) {
            mine[j * 16] = turn ? mine[j * 16] + acc[j][0] : acc[j][0];
            mine[ld + j * 16] = turn ? mine[ld + j * 16] + acc[j][1] : acc[j][1];
            mine[j * 16 + 8] = turn ? mine[j * 16 + 8] + acc[j][2] : acc[j][2];
            mine[ld + j * 16 + 8] = turn ? mine[ld + j * 16 + 8] + acc[j][3] : acc[j][3];
          }
      }
      if (turn == 0) __syncthreads();
    }
  }
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // every CTA of the cluster is there to be written to
  __syncthreads();
  // ---- the CTA's sum, warps in order (and parts, lower first, where they lie side by side), to every CTA
  for (int i = tid; i < tile.rows * r16 * 4; i += kThreads) {
    const int row = i / (r16 * 4), quad = i % (r16 * 4);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = XP - 1; k >= 0; --k)
      if (k == 0 || xpack) {
#pragma unroll
        for (int w = 0; w < kWarps / 2; ++w) {
          const float4 v = *reinterpret_cast<const float4*>(part + (w * 8 + row + k * XS) * ld + quad * 4);
          s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
      }
    for (uint32_t k = 0; k < c; ++k) st_dsmem_f4(sums + (q * 8 + row) * ld + quad * 4, k, s);
  }
  // ---- what the last phase reads first is on its way while the sums travel
  const bool tpack = tile.rows <= TS;
  const int ra = tpack ? (TS == 8 || t * 2 < TS ? 2 * t : 8) : 2 * t;      // this lane's tokens are ra and ra + 1
  const bool has_a = ra < tile.rows, has_b = ra + 1 < tile.rows;
  Y0Quad ya, yb;
  int nb = nb_lo + warp, col = nb * 32 + 4 * g;
  const size_t at_a = (size_t)row_0 * p.N, at_b = (size_t)row_1 * p.N;
  if (nb < nb_hi && col < p.N) {
    if (has_a) ya.load(p, at_a + col);
    if (has_b) yb.load(p, at_b + col);
  }
  __syncwarp();
  tc::cluster_barrier();
  // ---- fragments of T: column g, ranks RB / 4 * t ... of a step; one set for each part, or one for all side by side
  constexpr int RL = RB / 4;                            // ranks of a lane in a step: 8 or 4
  uint32_t* frags = reinterpret_cast<uint32_t*>(part);  // [step][part][lane][RL / 2]
  for (int i = tid; i < steps * 32; i += kThreads) {
    const int col = (i >> 2) & 7, first = (i >> 5) * RB + (i & 3) * RL, token = tpack ? col % TS : col;
    float v[RL];
#pragma unroll
    for (int k = 0; k < RL; ++k) v[k] = 0.f;
    if (token < tile.rows && first < r16 * 16) {
      for (uint32_t k = 0; k < c; ++k)
#pragma unroll
        for (int h = 0; h < RL; h += 4) {
          const float4 u = *reinterpret_cast<const float4*>(sums + (k * 8 + token) * ld + first + h);
          v[h] += u.x; v[h + 1] += u.y; v[h + 2] += u.z; v[h + 3] += u.w;
        }
    }
    uint32_t w[RL / 2][TP];
#pragma unroll
    for (int k = 0; k < RL; k += 2) {
      // beyond the rank the packed A holds zeros, and an infinite activation times zero is no zero
      const float lo = first + k < rank ? v[k] * hd.scale : 0.f, hi = first + k + 1 < rank ? v[k + 1] * hd.scale : 0.f;
      split<TP>(lo, hi, w[k / 2]);
    }
    uint32_t* at = frags + ((size_t)(i >> 5) * TP * 32 + (i & 31)) * (RL / 2);
#pragma unroll
    for (int k = 0; k < RL / 2; ++k) {
      if (tpack) {
        uint32_t m = 0;
#pragma unroll
        for (int x = 0; x < TP; ++x) m = col / TS == x ? w[k][x] : m;
        at[k] = m;
      } else {
#pragma unroll
        for (int x = 0; x < TP; ++x) at[x * 32 * (RL / 2) + k] = w[k][x];
      }
    }
  }
  __syncthreads();
  // ---- the CTA's columns of Y: blocks of 32, dealt to the warps in turn; a lane's four columns 4 g .. 4 g + 3 are rows g and g + 8
  // of two MMAs
  const uint32_t* fr = frags + lane * (RL / 2);
  for (; nb < nb_hi; nb += kWarps, col += kWarps * 32) {
    float acc[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    for (int s = 0; s < steps; ++s) {
      const uint8_t* at = arrived();
      uint32_t f[4][RL / 2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (PITCH > 32) {
          const uint4 u = reinterpret_cast<const uint4*>(at)[i * 32 + lane];
          f[i][0] = u.x; f[i][1] = u.y; f[i][RL / 2 - 2] = u.z; f[i][RL / 2 - 1] = u.w;
        } else {
          const uint2 u = reinterpret_cast<const uint2*>(at)[i * 32 + lane];
          f[i][0] = u.x; f[i][1] = u.y;
        }
      }
#pragma unroll
      for (int x = TP - 1; x >= 0; --x)
        if (x == 0 || !tpack) {
          uint32_t w[RL / 2];
#pragma unroll
          for (int k = 0; k < RL / 2; ++k) w[k] = fr[(s * TP + x) * 32 * (RL / 2) + k];
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k = 0; k < RL / 2; k += 2) mma(acc[j], f[2 * j][k], f[2 * j + 1][k], f[2 * j][k + 1], f[2 * j + 1][k + 1], w[k], w[k + 1]);
        }
      send();
    }
    float4 va = ya.values(p), vb = yb.values(p);
    const int next = col + kWarps * 32;
    if (nb + kWarps < nb_hi && next < p.N) {            // the next block's Y0
      if (has_a) ya.load(p, at_a + next);
      if (has_b) yb.load(p, at_b + next);
    }
    if (tpack && TP > 1) {                              // the parts of a token are in the neighbouring lanes
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (TS == 2) acc[j][i] += __shfl_xor_sync(0xFFFFFFFFu, acc[j][i], 1);
          acc[j][i] += __shfl_xor_sync(0xFFFFFFFFu, acc[j][i], 2);
        }
    }
    if (col < p.N) {
      va.x += acc[0][0]; va.y += acc[0][2]; va.z += acc[1][0]; va.w += acc[1][2];
      vb.x += acc[0][1]; vb.y += acc[0][3]; vb.z += acc[1][1]; vb.w += acc[1][3];
      if (has_a) store_y(p, at_a + col, va);
      if (has_b) store_y(p, at_b + col, vb);
    }
  }
}

// ---------------------------------------------------------------------------- host
template <int XT, int XP, int TP, int PITCH>
static cudaError_t launch_few(const Params& p, int tiles, int c, cudaStream_t s) {
  const size_t part = (size_t)kWarps / 2 * 8 * part_stride(p.max_rank) * 4;      // the fragments of T fit in the same place
  const size_t smem = part + (size_t)c * 8 * part_stride(p.max_rank) * 4 + (size_t)kWarps * ring_sets(PITCH) * ring_set_bytes(PITCH);
  static OncePerDevice once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(few_rows_kernel<XT, XP, TP, PITCH>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * c));
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
  return cudaLaunchKernelEx(&cfg, few_rows_kernel<XT, XP, TP, PITCH>, p);
}
template <int XT, int XP, int TP>
static cudaError_t launch_few_rank(const Params& p, int tiles, int c, cudaStream_t s) {
  const int pitch = b_pitch(p.max_rank);
  return pitch == 32   ? launch_few<XT, XP, TP, 32>(p, tiles, c, s)
         : pitch == 64 ? launch_few<XT, XP, TP, 64>(p, tiles, c, s)
                       : launch_few<XT, XP, TP, 128>(p, tiles, c, s);
}

}  // namespace ad

size_t adapter_slot_bytes(int K, int N, int max_rank) { return ad::slot_bytes(K, N, max_rank); }
size_t adapter_plan_bytes(int M, int n_slots) { return ad::plan_layout(M, n_slots).bytes; }
cudaError_t launch_adapter_pool_init(void* pool, int K, int N, int max_rank, int n_slots, cudaStream_t s) {
  LaunchScope scope(kFamPack, s);
  ad::pool_init_kernel<<<(n_slots + 255) / 256, 256, 0, s>>>(static_cast<uint8_t*>(pool), ad::slot_bytes(K, N, max_rank), n_slots, K, N, max_rank);
  return cudaGetLastError();
}
cudaError_t launch_adapter_load(void* pool, int K, int N, int max_rank, int slot, const void* A, const void* B, bool bf16, int rank, float scale,
                                cudaStream_t s) {
  LaunchScope scope(kFamPack, s);
  ad::adapter_load_kernel<<<rank > 0 ? 4 * sm_count() : 1, 256, 0, s>>>(static_cast<uint8_t*>(pool) + (size_t)slot * ad::slot_bytes(K, N, max_rank), A, B,
                                                                       bf16, K, N, max_rank, rank, scale);
  return cudaGetLastError();
}
cudaError_t launch_adapter_plan(const int* slots, int M, int n_slots, void* plan, cudaStream_t s) {
  uint8_t* at = static_cast<uint8_t*>(plan);
  const ad::PlanLayout l = ad::plan_layout(M, n_slots);
  auto list = [&](int i) {
    return ad::PlanList{reinterpret_cast<ad::Tile*>(at + l.tiles_at[i]), reinterpret_cast<int*>(at + l.rows_at[i]),
                        l.tiles[i] == 0 ? 0 : i == 0 ? ad::kFewRows : ad::kManyRows};
  };
  const size_t smem = (size_t)(n_slots + 1) * (ad::kPlanWarps + 3) * 4 + 8;
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
  return cudaLaunchKernelEx(&cfg, ad::plan_kernel, slots, M, n_slots, reinterpret_cast<ad::PlanHead*>(at), list(0), list(1));
}
size_t adapter_scratch_bytes(int M, int plan_slots, int K, int N, int max_rank) {
  return ad::takes_few(M, K, N, max_rank) ? 0 : ad::many_scratch_bytes(ad::plan_layout(M, plan_slots).tiles[1], max_rank);
}
cudaError_t launch_adapters(const void* X, int x_type, int M, const void* pool, int K, int N, int max_rank, void* plan, int plan_slots,
                            const void* Y0, int y0_type, void* Y, int y_type, int bits, int emin, int emax, void* scratch, cudaStream_t s) {
  uint8_t* at = static_cast<uint8_t*>(plan);
  const bool few = ad::takes_few(M, K, N, max_rank);
  const ad::PlanLayout l = ad::plan_layout(M, plan_slots);
  const int most = l.tiles[few ? 0 : 1];
  ad::Params p;
  p.X = X; p.pool = static_cast<const uint8_t*>(pool);
  p.plan = reinterpret_cast<ad::PlanHead*>(at);
  p.tiles = reinterpret_cast<const ad::Tile*>(at + l.tiles_at[few ? 0 : 1]);
  p.rows = reinterpret_cast<const int*>(at + l.rows_at[few ? 0 : 1]);
  p.Y0 = Y0; p.Y = Y;
  p.slot_bytes = ad::slot_bytes(K, N, max_rank);
  p.M = M; p.K = K; p.N = N; p.max_rank = max_rank; p.plan_slots = plan_slots;
  p.y0_bf16 = y0_type == kYBF16; p.y_bf16 = y_type == kYBF16;
  p.x_wide = reinterpret_cast<uintptr_t>(X) % 32 == 0;
  p.y_wide = reinterpret_cast<uintptr_t>(Y0) % 32 == 0 && reinterpret_cast<uintptr_t>(Y) % 32 == 0;
  p.bits = bits; p.emin = emin; p.emax = emax;
  const size_t whole = y_bytes(y_type, M, N), less = debug_y_shrink();
  p.y_extent = whole > less ? whole - less : 0;
  if (!few) return ad::launch_many(p, x_type, most, scratch, s);
  // CTAs to a tile: as many, up to eight, as fit two to an SM (of whole clusters fewer do: 33 of eight, 71 of four), for a number of
  // tiles between the fewest and the most that the batch can have; but no more than there are blocks of K or of columns for.
  const int tiles = (M / ad::kFewRows + most + 1) / 2;
  int c = 8;
  while (c > 1 && tiles * c > 2 * sm_count() - 4 * c) c /= 2;
  while (c > 1 && (K + 31) / 32 < c * ad::kWarps && (N + 31) / 32 < c * ad::kWarps) c /= 2;
  if (x_type == kXF32)
    return p.y_bf16 ? ad::launch_few_rank<kXF32, 2, 2>(p, most, c, s) : ad::launch_few_rank<kXF32, 3, 3>(p, most, c, s);
  if (x_type == kXBF16)
    return p.y_bf16 ? ad::launch_few_rank<kXBF16, 1, 2>(p, most, c, s) : ad::launch_few_rank<kXBF16, 1, 3>(p, most, c, s);
  return p.y_bf16 ? ad::launch_few_rank<kXMXINT8, 1, 2>(p, most, c, s) : ad::launch_few_rank<kXMXINT8, 1, 3>(p, most, c, s);
}

}  // namespace lqer
