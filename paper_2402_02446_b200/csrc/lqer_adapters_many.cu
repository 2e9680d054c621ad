// Adapters of many requests, more than 512 rows (see lqer_adapters.cu for the term, its precision and the layouts of pool and plan):
// two launches on the tcgen05 tensor cores, tiles of 128 rows of one adapter.
//
// project_kernel: T = X A_a.  The MMA's 128 rows are tokens, its columns the ranks.  Eight warps bring X from its rows, wherever they lie,
// through registers into the swizzled image (fp32 as bf16 parts, MXINT8 as its values), A's slabs of 64 K come by bulk copies, and
// the accumulators - one for each part, so that the small ones are not cut off against the large - stay in tensor memory.
// expand_kernel: Y = Y0 + scale T B_a.  T is the 128-row operand, in parts, written once a tile; B's images come by bulk copies; each
// block of 128 columns is one accumulator, and two of them take turns, so that the tensor cores work ahead of the warps that
// add Y0, which is on its way from memory a block ahead.
//
// Both are bound by memory: X is read once, Y0 read and Y written once; A and B come from L2 after a tile's first use.  The tiles'
// number is known on the device only, so the work (tile by tile, its slabs of K or blocks of columns in turn) is cut into equal
// stretches, one for each CTA of a grid as large as the device.  A stretch of the projection ends where it ends, in the middle of a
// tile if need be: it leaves its partial sums of T in place (tile + CTA) of the scratch, which no other stretch has, and the
// expansion adds up a tile's stretches in order.
#include "lqer_adapters.cuh"

namespace lqer {
namespace ad {

constexpr int kWorkWarps = 8, kCopyWarp = 8, kMmaWarp = 9, kManyThreads = 320;
constexpr int kXImage = 128 * 128;           // bytes of 128 rows of 64 bf16
constexpr int kMaxStages = 4;
constexpr int kMaxChain = 32;                // slabs of K that an accumulator takes before it is added to the partial sums

struct ManyParams {
  Params p;
  float4* scratch;           // [tile + CTA][rank / 4][128 rows]
  int project_ctas, stages;
  int stall;                 // test hook: the first copy never comes
  long long wait_limit;
};
__host__ __device__ inline size_t partial_floats(int max_rank) { return (size_t)rank16(max_rank) * 16 * 128; }
// CTAs that have work, first unit of CTA i's stretch of `units`, and the CTA whose stretch holds a unit.
__device__ __forceinline__ int busy(long long units, int ctas) { return (int)min(units, (long long)ctas); }
__device__ __forceinline__ long long stretch(long long units, int i, int ctas) { return units * i / ctas; }
__device__ __forceinline__ int holder(long long units, long long u, int ctas) {
  int i = (int)(u * ctas / units);
  while (i + 1 < ctas && stretch(units, i + 1, ctas) <= u) ++i;
  while (stretch(units, i, ctas) > u) --i;
  return i;
}
__device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// Shared-memory descriptor of a K-major image whose rows are `pitch` bytes (and so is its swizzle), 8-row groups 8 rows apart.
__device__ __forceinline__ uint64_t image_desc(uint32_t saddr, int pitch) {
  const uint64_t layout = pitch == 128 ? 2 : pitch == 64 ? 4 : 6;
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(pitch >> 1) << 32 | (uint64_t)1 << 46 | layout << 61;
}
// 16 rows x 32 columns of an accumulator in the fragment layout: register 4 j + 2 h + i is row lane / 4 + 8 h, column 8 j + 2 (lane % 4) + i.
__device__ __forceinline__ void tmem_ld_16x32(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ uint32_t columns_pow2(int n) {
  uint32_t c = 32;
  while ((int)c < n) c *= 2;
  return c;
}
// Barriers of a CTA, set up by its first thread.
struct Barriers {
  unsigned long long full[kMaxStages], copied[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], ready;
};
__device__ __forceinline__ uint32_t bar_of(unsigned long long& b) { return tc::smem_u32(&b); }
__device__ __forceinline__ void init_barriers(Barriers& b) {
  for (int i = 0; i < kMaxStages; ++i) {
    tc::mbar_init(bar_of(b.full[i]), kWorkWarps);
    tc::mbar_init(bar_of(b.copied[i]), 1);
    tc::mbar_init(bar_of(b.empty[i]), 1);
  }
  for (int i = 0; i < 2; ++i) {
    tc::mbar_init(bar_of(b.acc_full[i]), 1);
    tc::mbar_init(bar_of(b.acc_empty[i]), kWorkWarps);
  }
  tc::mbar_init(bar_of(b.ready), kWorkWarps);
  tc::fence_barrier_init();
}

// ---------------------------------------------------------------------------- T = X A
// A CTA's stretch is walked by all roles alike: runs of slabs of one tile, at most kMaxChain each; tiles without a rank are passed over.
struct Run {
  int tile, slab, slabs, rank;
  bool first;                // the first of its tile in this stretch
};
struct RunWalk {
  long long u, end, begin;
  int KS;
  __device__ bool next(const Params& p, Run& r) {
    while (u < end) {
      r.tile = (int)(u / KS);
      r.slab = (int)(u % KS);
      r.first = u == begin || r.slab == 0;
      r.slabs = (int)min((long long)min(KS - r.slab, kMaxChain), end - u);
      const int slot = p.tiles[r.tile].slot;
      r.rank = rank_of(p, slot, load_slot(p.pool + (size_t)max(slot, 0) * p.slot_bytes), false);
      u += r.slabs;
      if (r.rank > 0) return true;
    }
    return false;
  }
};

template <int XT, int XP>
__global__ void __launch_bounds__(kManyThreads, 1) project_kernel(const __grid_constant__ ManyParams mp) {
  constexpr int AHEAD = XT == kXF32 ? 2 : 4;            // slabs whose X is on its way
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_at;
  __shared__ tc::WaitState ws;
  const Params& p = mp.p;
  uint8_t* smem = smem_raw + ((1024u - (tc::smem_u32(smem_raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int stage_bytes = XP * kXImage + rank16(p.max_rank) * 2048;
  const bool apart = XP * rank16(p.max_rank) * 16 <= 512;                  // an accumulator for each part
  const uint32_t tmem_cols = columns_pow2((apart ? XP : 1) * rank16(p.max_rank) * 16);
  if (tid == 0) {
    init_barriers(bars);
    ws.abort = 0;
    ws.limit = mp.wait_limit;
  }
  if (warp == kMmaWarp) tc::tmem_alloc(tc::smem_u32(&tmem_at), tmem_cols);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_at;
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const PlanHead head = load_head(p.plan);
  RunWalk walk;
  walk.KS = (p.K + 63) / 64;
  const long long units = plan_fits(p, head) ? (long long)head.n_adapted * walk.KS : 0;
  const int ctas = busy(units, gridDim.x), cta = min((int)blockIdx.x, ctas);
  walk.begin = walk.u = ctas > 0 ? stretch(units, cta, ctas) : 0;
  walk.end = ctas > 0 ? stretch(units, min(cta + 1, ctas), ctas) : 0;
  Run r;
  bool ok = true;
  if (warp < kWorkWarps) {
    // ---- X into its images; then, at a run's end, the accumulators into the partial sums
    int it = 0, runs = 0;
    const uint32_t piece = lane & 7;
    while (ok && walk.next(p, r)) {
      int row[4];
      uint32_t at[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = warp * 16 + i * 4 + (lane >> 3);
        row[i] = p.rows[(size_t)r.tile * kManyRows + m];
        at[i] = swizzled(m, piece, 128);
      }
      XOct<XT> x[AHEAD][4];
      auto load = [&](XOct<XT> (&o)[4], int s) {
        const int col = (r.slab + s) * 64 + piece * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i].load(p, row[i], col, s < r.slabs && col < p.K);
      };
#pragma unroll
      for (int a = 0; a < AHEAD; ++a) load(x[a], a);
      for (int s0 = 0; s0 < r.slabs && ok; s0 += AHEAD) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
          if (s0 + a < r.slabs && ok) {
            const int st = it % mp.stages, turn = it / mp.stages;
            ++it;
            ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.empty[st]), (turn & 1) ^ 1, &ws)) != 0;
            if (ok) {
              uint8_t* img = smem + (size_t)st * stage_bytes;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t w[4][XP];
                x[a][i].template pairs<XP>(p, w);
#pragma unroll
                for (int k = 0; k < XP; ++k) *reinterpret_cast<uint4*>(img + k * kXImage + at[i]) = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
              }
              load(x[a], s0 + a + AHEAD);
              tc::fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) tc::mbar_arrive(bar_of(bars.full[st]));
            }
          }
        }
      }
      if (ok) ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.acc_full[0]), runs & 1, &ws)) != 0;
      ++runs;
      if (!ok) break;
      tc::tc_fence_after();
      const int r16 = rank16(r.rank), m = (warp & 3) * 32 + lane;
      float4* out = mp.scratch + (size_t)(r.tile + blockIdx.x) * (partial_floats(p.max_rank) / 4) + m;
      for (int b = warp >> 2; b < r16; b += 2) {
        float v[16];
#pragma unroll
        for (int k = XP - 1; k >= 0; --k) {
          if (k > 0 && !apart) continue;
          uint32_t u[16];
          tc::tmem_ld16(tmem + ((uint32_t)((warp & 3) * 32) << 16) + k * r16 * 16 + b * 16, u);
          tc::tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = k == XP - 1 || !apart ? __uint_as_float(u[i]) : v[i] + __uint_as_float(u[i]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float4 s = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          float4* to = out + (b * 4 + q) * 128;
          if (!r.first) {                               // what this stretch has of the tile already; the same thread wrote it
            const float4 o = *to;
            s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
          }
          *to = s;
        }
      }
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar_of(bars.acc_empty[0]));
    }
  } else if (warp == kCopyWarp) {
    // ---- slabs of A
    if (lane == 0) {
      int it = 0;
      while (ok && walk.next(p, r)) {
        const uint32_t bytes = rank16(r.rank) * 2048;
        const uint8_t* A = p.pool + (size_t)p.tiles[r.tile].slot * p.slot_bytes + 256 + (size_t)r.slab * bytes;
        for (int s = 0; s < r.slabs && ok; ++s, ++it) {
          const int st = it % mp.stages, turn = it / mp.stages;
          ok = tc::mbar_wait(bar_of(bars.empty[st]), (turn & 1) ^ 1, &ws);
          if (!ok) break;
          if (mp.stall != 0 && it == 0 && blockIdx.x == 0) continue;
          tc::mbar_expect_tx(bar_of(bars.copied[st]), bytes);
          tc::bulk_load(tc::smem_u32(smem + (size_t)st * stage_bytes + XP * kXImage), A + (size_t)s * bytes, bytes, bar_of(bars.copied[st]));
        }
      }
      // on the way out after a wait that ran out: no copy of this CTA is left in flight
      for (int k = 0; k < mp.stages && !ok && k < it; ++k) {
        const int last = it - 1 - k, st = last % mp.stages, turn = last / mp.stages;
        if (mp.stall != 0 && last == 0 && blockIdx.x == 0) continue;
        const long long t0 = clock64();
        while (!tc::mbar_try_wait(bar_of(bars.copied[st]), turn & 1) && clock64() - t0 < mp.wait_limit) {}
      }
    }
  } else {
    // ---- MMAs
    if (lane == 0) {
      int it = 0, runs = 0;
      while (ok && walk.next(p, r)) {
        const int cols = rank16(r.rank) * 16;
        const uint32_t idesc = tc::make_idesc(128, cols);
        ok = tc::mbar_wait(bar_of(bars.acc_empty[0]), (runs & 1) ^ 1, &ws);
        ++runs;
        tc::tc_fence_after();
        for (int s = 0; s < r.slabs && ok; ++s, ++it) {
          const int st = it % mp.stages, turn = it / mp.stages;
          ok = tc::mbar_wait(bar_of(bars.full[st]), turn & 1, &ws) && tc::mbar_wait(bar_of(bars.copied[st]), turn & 1, &ws);
          if (!ok) break;
          tc::tc_fence_after();
          const uint32_t base = tc::smem_u32(smem + (size_t)st * stage_bytes);
          const uint64_t b = image_desc(base + XP * kXImage, 128);
#pragma unroll
          for (int k = XP - 1; k >= 0; --k) {
            const uint64_t a = image_desc(base + k * kXImage, 128);
#pragma unroll
            for (int h = 0; h < 4; ++h)
              umma(tmem + (apart ? k * cols : 0), a + 2 * h, b + 2 * h, idesc, s > 0 || h > 0 || (!apart && k < XP - 1) ? 1u : 0u);
          }
          tc::umma_commit(bar_of(bars.empty[st]));
        }
        if (ok) tc::umma_commit(bar_of(bars.acc_full[0]));
      }
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (tid == 0 && ws.abort != 0) report_error(&p.plan->status, LQER_ERR_TIMEOUT, 810);
  if (warp == kMmaWarp) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, tmem_cols);
  }
}

// ---------------------------------------------------------------------------- Y = Y0 + T B
template <bool BF16>
struct Oct {
  uint4 a, b;                // eight values: fp32 both, bf16 a
  __device__ __forceinline__ void load(const void* p, size_t idx) {
    if (BF16) {
      a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + idx);
    } else {
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + idx);
      a = q[0];
      b = q[1];
    }
  }
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
__device__ __forceinline__ void store_oct(const Params& p, size_t idx, const float (&v)[8]) {
  if (!LQER_IN_BOUNDS(&p.plan->status, idx * (BF16 ? 2 : 4), BF16 ? 16 : 32, p.y_extent, 812)) return;
  if (BF16) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.Y) + idx) =
        make_uint4(round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]), round_bf16x2(v[4], v[5]), round_bf16x2(v[6], v[7]));
  } else {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p.Y) + idx);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

template <bool Y0B, bool YB>
__global__ void __launch_bounds__(kManyThreads, 1) expand_kernel(const __grid_constant__ ManyParams mp) {
  constexpr int TP = YB ? 2 : 3;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_at;
  __shared__ tc::WaitState ws;
  const Params& p = mp.p;
  uint8_t* smem = smem_raw + ((1024u - (tc::smem_u32(smem_raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int max_slabs = (p.max_rank + 63) / 64, pitch = b_pitch(p.max_rank), image = 128 * pitch;
  uint8_t* ring = smem + (size_t)TP * max_slabs * kXImage;
  if (tid == 0) {
    init_barriers(bars);
    ws.abort = 0;
    ws.limit = mp.wait_limit;
  }
  if (warp == kMmaWarp) tc::tmem_alloc(tc::smem_u32(&tmem_at), 256);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_at;
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const PlanHead head = load_head(p.plan);
  const bool fits = plan_fits(p, head);
  const int NC = (p.N + 127) / 128;
  const long long items = fits ? (long long)(p.Y0 == p.Y ? head.n_adapted : head.n_tiles) * NC : 0;
  const long long begin = stretch(items, blockIdx.x, gridDim.x), end = stretch(items, blockIdx.x + 1, gridDim.x);
  bool ok = true;
  int tile_id = -1, rank = 0;
  Tile tile{-1, 0};
  SlotHead hd;
  // the tile of item v, if it is another one than that of the item before
  auto enter = [&](long long v) {
    const int t = (int)(v / NC);
    if (t == tile_id) return false;
    tile_id = t;
    tile = p.tiles[t];
    hd = load_slot(p.pool + (size_t)max(tile.slot, 0) * p.slot_bytes);
    rank = rank_of(p, tile.slot, hd, tid == 0);
    return true;
  };
  if (warp < kWorkWarps) {
    const int quarter = (warp & 3) * 32, half = (warp >> 2) * 64, t = lane & 3;
    int n = 0;                                          // blocks with an accumulator so far
    size_t at[4];                                       // this lane's rows, quarter + lane / 4 + 8 i, in Y0 and Y
    bool has[4];
    Oct<Y0B> y[4][2];
    auto load_y0 = [&](int i, int c, long long v) {     // rows i, columns 32 c + 8 t of the warp's 64
      const int col = (int)(v % NC) * 128 + half + c * 32 + 8 * t;
      if (has[i] && col < p.N) y[i][c].load(p.Y0, at[i] + col);
    };
    for (long long v = begin; v < end && ok; ++v) {
      if (enter(v)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int m = quarter + (lane >> 2) + 8 * i;
          has[i] = m < tile.rows;
          at[i] = (size_t)p.rows[(size_t)tile_id * kManyRows + m] * p.N;
#pragma unroll
          for (int c = 0; c < 2; ++c) load_y0(i, c, v);
        }
        if (rank > 0) {
          // T, summed over the stretches that have a part of this tile, into its images.  The last tile's MMAs are done: its last
          // accumulator was waited for.
          const int KS = (p.K + 63) / 64, r16 = rank16(rank), m = tid & 127, slabs = (rank + 63) / 64;
          const long long units = (long long)head.n_adapted * KS;
          const int ctas = busy(units, mp.project_ctas), from = holder(units, (long long)tile_id * KS, ctas),
                    to = holder(units, (long long)(tile_id + 1) * KS - 1, ctas);
          const size_t per = partial_floats(p.max_rank) / 4;
          const float4* src = mp.scratch + (size_t)(tile_id + from) * per + m;
          for (int e = tid >> 7; e < slabs * 8; e += 2) {                   // eight ranks
            float v8[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (e < r16 * 2)
              for (int k = 0; k <= to - from; ++k) {
                const float4 lo = src[k * per + e * 256], hi = src[k * per + e * 256 + 128];
                v8[0] += lo.x; v8[1] += lo.y; v8[2] += lo.z; v8[3] += lo.w;
                v8[4] += hi.x; v8[5] += hi.y; v8[6] += hi.z; v8[7] += hi.w;
              }
            uint32_t w[4][TP];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              // beyond the rank the packed A holds zeros, and an infinite activation times zero is no zero
              const float lo = e * 8 + 2 * i < rank ? v8[2 * i] * hd.scale : 0.f, hi = e * 8 + 2 * i + 1 < rank ? v8[2 * i + 1] * hd.scale : 0.f;
              split<TP>(lo, hi, w[i]);
            }
            uint8_t* img = smem + (size_t)(e >> 3) * kXImage + swizzled(m, e & 7, 128);
#pragma unroll
            for (int k = 0; k < TP; ++k)
              *reinterpret_cast<uint4*>(img + (size_t)k * max_slabs * kXImage) = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
          }
          tc::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(bar_of(bars.ready));
        }
      }
      const bool more = v + 1 < end && (int)((v + 1) / NC) == tile_id;
      const int buf = n & 1;
      if (rank > 0) {
        ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.acc_full[buf]), (n >> 1) & 1, &ws)) != 0;
        ++n;
        if (!ok) break;
        tc::tc_fence_after();
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t u[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) u[i] = 0u;
          if (rank > 0) {
            tmem_ld_16x32(tmem + ((uint32_t)(quarter + h * 16) << 16) + buf * 128 + half + c * 32, u);
            tc::tmem_ld_wait();
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {                 // rows lane / 4 and lane / 4 + 8 of the sixteen
            const int k = 2 * h + i, col = (int)(v % NC) * 128 + half + c * 32 + 8 * t;
            float o[8];
            y[k][c].values(o);
            if (more) load_y0(k, c, v + 1);
            if (rank > 0) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                o[2 * j] += __uint_as_float(u[4 * j + 2 * i]);
                o[2 * j + 1] += __uint_as_float(u[4 * j + 2 * i + 1]);
              }
            }
            if (has[k] && col < p.N) store_oct<YB>(p, at[k] + col, o);
          }
        }
      }
      if (rank > 0) {
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar_of(bars.acc_empty[buf]));
      }
    }
  } else if (warp == kCopyWarp) {
    // ---- images of B: a stage is 128 columns of up to 64 ranks
    if (lane == 0) {
      int it = 0;
      for (long long v = begin; v < end && ok; ++v) {
        enter(v);
        const int slabs = (rank + 63) / 64;
        const uint8_t* B = p.pool + (size_t)max(tile.slot, 0) * p.slot_bytes + 256 + a_bytes(p.K, p.max_rank) + (size_t)(v % NC) * slabs * image;
        for (int s = 0; s < slabs && ok; ++s, ++it) {
          const int st = it % mp.stages, turn = it / mp.stages;
          ok = tc::mbar_wait(bar_of(bars.empty[st]), (turn & 1) ^ 1, &ws);
          if (!ok) break;
          tc::mbar_expect_tx(bar_of(bars.copied[st]), image);
          tc::bulk_load(tc::smem_u32(ring + (size_t)st * image), B + (size_t)s * image, image, bar_of(bars.copied[st]));
        }
      }
      for (int k = 0; k < mp.stages && !ok && k < it; ++k) {                // after a wait that ran out: no copy is left in flight
        const int last = it - 1 - k, st = last % mp.stages, turn = last / mp.stages;
        const long long t0 = clock64();
        while (!tc::mbar_try_wait(bar_of(bars.copied[st]), turn & 1) && clock64() - t0 < mp.wait_limit) {}
      }
    }
  } else {
    // ---- MMAs
    if (lane == 0) {
      const uint32_t idesc = tc::make_idesc(128, 128);
      int it = 0, n = 0, tiles = 0;
      for (long long v = begin; v < end && ok; ++v) {
        if (enter(v) && rank > 0) ok = tc::mbar_wait(bar_of(bars.ready), tiles++ & 1, &ws);
        if (rank == 0) continue;
        if (ok) ok = tc::mbar_wait(bar_of(bars.acc_empty[n & 1]), ((n >> 1) & 1) ^ 1, &ws);
        tc::tc_fence_after();
        const int slabs = (rank + 63) / 64, r16 = rank16(rank);
        for (int s = 0; s < slabs && ok; ++s, ++it) {
          const int st = it % mp.stages, turn = it / mp.stages;
          ok = tc::mbar_wait(bar_of(bars.copied[st]), turn & 1, &ws);
          if (!ok) break;
          tc::tc_fence_after();
          const uint64_t b = image_desc(tc::smem_u32(ring + (size_t)st * image), pitch);
          const int steps = min(4, r16 - s * 4);
#pragma unroll
          for (int k = TP - 1; k >= 0; --k) {
            const uint64_t a = image_desc(tc::smem_u32(smem + (size_t)(k * max_slabs + s) * kXImage), 128);
            for (int h = 0; h < steps; ++h) umma(tmem + (n & 1) * 128, a + 2 * h, b + 2 * h, idesc, s > 0 || h > 0 || k < TP - 1 ? 1u : 0u);
          }
          tc::umma_commit(bar_of(bars.empty[st]));
        }
        if (ok) tc::umma_commit(bar_of(bars.acc_full[n & 1]));
        ++n;
      }
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (tid == 0 && ws.abort != 0) report_error(&p.plan->status, LQER_ERR_TIMEOUT, 811);
  if (warp == kMmaWarp) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, 256);
  }
}

// ---------------------------------------------------------------------------- host
constexpr size_t kSmemMost = 226 * 1024;
size_t many_scratch_bytes(int M, int plan_slots, int max_rank) {
  // the grids are no larger than this many CTAs (launch_many takes fewer where the device has fewer SMs)
  return ((size_t)max_tiles(M, plan_slots) + kPrologueMaxCtas) * partial_floats(max_rank) * 4;
}
template <class Kernel>
static cudaError_t launch(Kernel kernel, OncePerDevice& once, const ManyParams& mp, int ctas, size_t smem, cudaStream_t s) {
  cudaError_t e = once.run([=] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kManyThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, mp);
}
template <int XT, int XP>
static cudaError_t launch_project(ManyParams mp, cudaStream_t s) {
  static OncePerDevice once;
  const size_t stage = (size_t)XP * kXImage + rank16(mp.p.max_rank) * 2048;
  mp.stages = (int)((kSmemMost - 1024) / stage);
  if (mp.stages > kMaxStages) mp.stages = kMaxStages;
  return launch(project_kernel<XT, XP>, once, mp, mp.project_ctas, mp.stages * stage + 1024, s);
}
template <bool Y0B, bool YB>
static cudaError_t launch_expand(ManyParams mp, int ctas, cudaStream_t s) {
  static OncePerDevice once;
  const size_t t = (size_t)(YB ? 2 : 3) * ((mp.p.max_rank + 63) / 64) * kXImage, image = (size_t)128 * b_pitch(mp.p.max_rank);
  mp.stages = (int)((kSmemMost - 1024 - t) / image);
  if (mp.stages > kMaxStages) mp.stages = kMaxStages;
  return launch(expand_kernel<Y0B, YB>, once, mp, ctas, t + mp.stages * image + 1024, s);
}
cudaError_t launch_many(const Params& p, int x_type, int tiles, void* scratch, cudaStream_t s) {
  (void)tiles;
  const int sms = sm_count(), ctas = sms < kPrologueMaxCtas ? sms : kPrologueMaxCtas;
  ManyParams mp{p, static_cast<float4*>(scratch), ctas, 0, take_stall(kFamDecode) ? 1 : 0, wait_limit_cycles()};
  LaunchScope scope(kFamDecode, s, 2);
  cudaError_t e = x_type == kXF32    ? (p.y_bf16 ? launch_project<kXF32, 2>(mp, s) : launch_project<kXF32, 3>(mp, s))
                  : x_type == kXBF16 ? launch_project<kXBF16, 1>(mp, s)
                                     : launch_project<kXMXINT8, 1>(mp, s);
  if (e != cudaSuccess) return e;
  return p.y0_bf16 ? (p.y_bf16 ? launch_expand<true, true>(mp, ctas, s) : launch_expand<true, false>(mp, ctas, s))
                   : (p.y_bf16 ? launch_expand<false, true>(mp, ctas, s) : launch_expand<false, false>(mp, ctas, s));
}

}  // namespace ad
}  // namespace lqer
