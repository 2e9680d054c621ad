// Adapters of many requests, many rows (see lqer_adapters.cu for the term, its precision and the layouts of pool and plan):
// three launches, tiles of 128 rows of one adapter, the products on the tcgen05 tensor cores.
//
// project_kernel: T = X A_a.  The MMA's 128 rows are tokens, its columns the ranks.  Sixteen warps bring X from its rows, wherever they lie,
// through registers into the swizzled image (fp32 as bf16 parts, MXINT8 as its values), A's slabs of 64 K come by bulk copies, and
// the accumulators - one for each part, so that the small ones are not cut off against the large - stay in tensor memory.
// finish_kernel: T from its partial sums, scaled, in bf16 parts, in the swizzled images that the next kernel copies.
// expand_kernel: Y = Y0 + T B_a.  T is the 128-row operand, copied once a tile, as B's images are; each block of 128 columns is one
// accumulator, and two of them take turns, so that the tensor cores work ahead of the sixteen warps that add Y0, of which two blocks
// are on their way from memory (64 KB a CTA in bf16, 128 KB in fp32).
//
// They are bound by memory: X is read once, Y0 read and Y written once; A and B come from L2 after a tile's first use.  The tiles'
// number is known on the device only.  The projection's work (tile by tile, its slabs of K in turn) is cut into equal stretches, one
// for each CTA of a grid as large as the device; a stretch ends where it ends, in the middle of a tile if need be: it leaves its
// partial sums of T in place (tile + CTA) of the scratch, which no other stretch has, and finish_kernel adds up a tile's
// stretches in order.  The expansion's CTAs draw groups of columns from a counter.
//
// Measured, all three: 4096 rows of 5120 x 13824 rank 64 in fp32 106 us, 5.1 TB/s: 28 us project, of which 13 would do for X's bytes (the
// rest goes into the instructions that cut fp32 into three parts), 4 finish, 72 expand at 6.3 TB/s, 4 in between.  2048 rows of
// 4096 x 11008 rank 64 in bf16 38 us: the bytes would take 17, but about 15 us pass before the first Y can be written.
#include "lqer_adapters.cuh"

namespace lqer {
namespace ad {

constexpr int kWorkWarps = 16, kCopyWarp = 16, kMmaWarp = 17, kManyThreads = 576;
constexpr int kXImage = 128 * 128;           // bytes of 128 rows of 64 bf16
constexpr int kMaxStages = 4;
constexpr int kMaxChain = 32;                // slabs of K that an accumulator takes before it is added to the partial sums

struct ManyParams {
  Params p;
  float4* scratch;           // [tile + CTA][rank / 4][128 rows]
  uint8_t* images;           // T: [tile][part][rank / 64][128 rows x 128 bytes]
  int* drawn;                // groups that expand_kernel's CTAs took beside their first
  int project_ctas, stages, t_sets;      // t_sets: tiles' T that fit side by side, 1 or 2
  int stall;                 // test hook: the first copy never comes
  long long wait_limit;
};
__host__ __device__ inline size_t partial_floats(int max_rank) { return (size_t)rank16(max_rank) * 16 * 128; }
// The projection's work, KS slabs of each of `tiles` tiles, cut into stretches for up to `most` CTAs.  Either every tile is cut alike
// (`parts` CTAs, `each` slabs a stretch), or the whole of it is (parts == 0), with stretches that may reach into the next tile.  To
// change tiles costs a CTA about as much as four slabs, so tiles are cut alike where that makes the longest stretch no more than four
// slabs longer (2048 rows of 4096 x 11008 rank 64 in bf16, the whole call: 40.6 -> 39.6 us).
struct Cut {
  unsigned KS, each, rest;              // tiles * KS stays below 2^32: no more than 2^24 rows in 2^17 + 1025 tiles, and 2^20 columns
  int ctas, parts;                      // ctas: those that have work; parts == 0: units = each * ctas + rest
  __device__ Cut(int tiles, int slabs, int most) : KS(slabs) {
    const unsigned units = (unsigned)max(tiles, 0) * KS;
    parts = tiles > 0 ? min(most / tiles, slabs) : 0;
    ctas = (int)min(units, (unsigned)most);
    each = ctas > 0 ? units / (unsigned)ctas : 0;
    rest = units - each * (unsigned)ctas;
    if (parts > 0) {
      const unsigned alike = (KS + parts - 1) / parts;
      if (alike <= each + (rest > 0 ? 1 : 0) + 4) {
        each = alike;
        parts = (KS + each - 1) / each;
        ctas = tiles * parts;
        return;
      }
    }
    parts = 0;
  }
  // first unit (tile * KS + slab) of CTA i's stretch; i may be ctas
  __device__ unsigned first(int i) const {
    if (parts > 0) return (unsigned)i / (unsigned)parts * KS + (unsigned)i % (unsigned)parts * each;
    return each * (unsigned)i + (ctas > 0 ? rest * (unsigned)i / (unsigned)ctas : 0u);
  }
  // the first of the CTAs that have a share of a tile, and how many they are
  __device__ int first_of(int tile, int& count) const {
    if (ctas == 0) return count = 0;
    if (parts > 0) {
      count = parts;
      return tile * parts;
    }
    const int a = holder((unsigned)tile * KS);
    count = holder((unsigned)(tile + 1) * KS - 1) - a + 1;
    return a;
  }
  // (parts == 0) the CTA whose stretch holds a unit
  __device__ int holder(unsigned u) const {
    int i = min(max((int)((float)u / ((float)each + (float)rest / (float)ctas)), 0), ctas - 1);
    while (i + 1 < ctas && first(i + 1) <= u) ++i;
    while (first(i) > u) --i;
    return i;
  }
};
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
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16_or_zeros(uint32_t dst, const void* src, int bytes) {      // bytes: 16, or 0 for zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t columns_pow2(int n) {
  uint32_t c = 32;
  while ((int)c < n) c *= 2;
  return c;
}
// Barriers of a CTA, set up by its first thread.
struct Barriers {
  unsigned long long full[kMaxStages], copied[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], t_full[2], t_empty[2], drawn[4], taken[4], drained;
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
    tc::mbar_init(bar_of(b.t_full[i]), 1);
    tc::mbar_init(bar_of(b.t_empty[i]), 1);
  }
  for (int i = 0; i < 4; ++i) {
    tc::mbar_init(bar_of(b.drawn[i]), 1);
    tc::mbar_init(bar_of(b.taken[i]), kWorkWarps + 1);
  }
  tc::mbar_init(bar_of(b.drained), 1);
  tc::fence_barrier_init();
}
// On the way out after a wait ran out in any role: what this CTA has under way may still write its shared and tensor memory, which other
// CTAs own once it has gone.  The threads that sent it wait for it, with a bound of their own (about a millisecond) whatever that of the waits is.
constexpr long long kDrainCycles = 2000000;
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
  const long long t0 = clock64();
  while (!tc::mbar_try_wait(bar, parity) && clock64() - t0 < kDrainCycles) {}
}
// (the thread that issued the MMAs)
__device__ __forceinline__ void drain_mmas(Barriers& b) {
  tc::umma_commit(bar_of(b.drained));
  drain(bar_of(b.drained), 0);
}
// (the thread that issued the copies: `copies` of them, in turn into `stages` places)
__device__ __forceinline__ void drain_copies(unsigned long long* bars, int copies, int stages) {
  for (int k = 0; k < stages && k < copies; ++k) {
    const int last = copies - 1 - k;
    drain(bar_of(bars[last % stages]), last / stages & 1);
  }
}

// ---------------------------------------------------------------------------- T = X A
// A CTA's stretch is walked by all roles alike: runs of slabs of one tile, at most kMaxChain each.  (An empty slot's rank counts as 16
// here, so that nobody has to know it before X is on its way; finish_kernel knows.)
struct Run {
  int tile, slab, slabs;
  bool first;                // the first of its tile in this stretch
};
struct RunWalk {
  unsigned u, end, begin, KS;
  __device__ bool next(Run& r) {
    if (u >= end) return false;
    r.tile = (int)(u / KS);
    r.slab = (int)(u % KS);
    r.first = u == begin || r.slab == 0;
    r.slabs = (int)min(min(KS - r.slab, (unsigned)kMaxChain), end - u);
    u += r.slabs;
    return true;
  }
};
__device__ __forceinline__ int project_rank16(const Params& p, int tile, int& slot) {
  slot = max(p.tiles[tile].slot, 0);
  return max(rank16(rank_of(p, slot, load_slot(p.pool + (size_t)slot * p.slot_bytes), false)), 1);
}

// AHEAD: slabs whose X is on its way, 32 KB (fp32) or 16 KB each: fp32 by copies into shared memory, the others into registers.
template <int XT, int XP, int AHEAD>
__global__ void __launch_bounds__(kManyThreads, 1) project_kernel(const __grid_constant__ ManyParams mp) {
  constexpr bool STAGED = XT == kXF32;
  constexpr int RW = 128 / kWorkWarps / 4;              // rows of a lane: eight lanes a row
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
  tc::pdl_wait();
  tc::pdl_launch_dependents();                          // in this order: see expand_kernel
  const ListHead head = load_head(p.plan, 1);
  RunWalk walk;
  walk.KS = (p.K + 63) / 64;
  const Cut cut(plan_fits(p, head) ? head.n_adapted : 0, walk.KS, gridDim.x);
  walk.begin = walk.u = cut.first(min((int)blockIdx.x, cut.ctas));
  walk.end = cut.first(min((int)blockIdx.x + 1, cut.ctas));
  Run r;
  bool ok = true;
  int it = 0;                // slabs so far
  if (warp < kWorkWarps) {
    // ---- X into its images; then, at a run's end, the accumulators into the partial sums
    int runs = 0;
    const uint32_t piece = lane & 7;
    while (ok && walk.next(r)) {
      uint32_t at[RW];
#pragma unroll
      for (int i = 0; i < RW; ++i) at[i] = swizzled((warp * RW + i) * 4 + (lane >> 3), piece, 128);
      const int stop = min((r.slab + r.slabs) * 64, p.K);
      int slot, r16;
      // one slab's octets into a stage, once it is free; sent: what has to be done as soon as they are in registers
      auto put = [&](const XOct<XT> (&x)[RW], auto&& sent) {
        const int st = it % mp.stages, turn = it / mp.stages;
        ++it;
        ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.empty[st]), (turn & 1) ^ 1, &ws)) != 0;
        if (!ok) return;
        uint8_t* img = smem + (size_t)st * stage_bytes;
#pragma unroll
        for (int i = 0; i < RW; ++i) {
          uint32_t w[4][XP];
          x[i].template pairs<XP>(p, w);
#pragma unroll
          for (int k = 0; k < XP; ++k) *reinterpret_cast<uint4*>(img + k * kXImage + at[i]) = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
        }
        sent();
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar_of(bars.full[st]));
      };
      if constexpr (STAGED) {
        // A warp's eight rows of 256 bytes, in 16-byte pieces: sixteen lanes send for a row.  A lane reads two neighbouring pieces of a row;
        // pieces of a row's second half change places with their neighbours, so that eight lanes meet no bank twice.
        const uint8_t* from[4];
        const int c = lane & 15;
        const uint32_t ring = tc::smem_u32(smem + (size_t)mp.stages * stage_bytes) + warp * 2048;
        const uint32_t to = (lane >> 4) * 256 + ((c ^ (c >> 3)) << 4), get = (lane >> 3) * 256 + ((2 * piece ^ (piece >> 2)) << 4);
        int col = r.slab * 64 + c * 4, sent_for = 0, here = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          from[j] = static_cast<const uint8_t*>(p.X) + ((size_t)p.rows[(size_t)r.tile * kManyRows + warp * 8 + 2 * j + (lane >> 4)] * p.K + col) * 4;
        auto send = [&] {                               // for the next slab
          if (sent_for < r.slabs) {
            const int bytes = col < stop ? 16 : 0;      // beyond K: zeros
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              cp_async16_or_zeros(ring + (uint32_t)(sent_for % AHEAD) * (kWorkWarps * 2048) + j * 512 + to, bytes ? from[j] : static_cast<const uint8_t*>(p.X), bytes);
              from[j] += 256;
            }
          }
          cp_async_commit();
          ++sent_for;
          col += 64;
        };
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) send();
        r16 = project_rank16(p, r.tile, slot);
        for (int s = 0; s < r.slabs && ok; ++s) {
          cp_async_wait<AHEAD - 1>();
          __syncwarp();
          XOct<XT> x[RW];
          const uint32_t src = ring + (uint32_t)here * (kWorkWarps * 2048) + get;
#pragma unroll
          for (int i = 0; i < RW; ++i) {
            x[i].a = lds16(src + i * 1024);
            x[i].b = lds16((src + i * 1024) ^ 16);
          }
          here = here + 1 == AHEAD ? 0 : here + 1;
          __syncwarp();
          send();
          put(x, [] {});
        }
        cp_async_wait<0>();
        __syncwarp();
      } else {
        typename XOct<XT>::Place from[RW];              // of the octet that is sent for next
        int col = r.slab * 64 + piece * 8;
#pragma unroll
        for (int i = 0; i < RW; ++i) from[i].set(p, p.rows[(size_t)r.tile * kManyRows + (warp * RW + i) * 4 + (lane >> 3)], col);
        XOct<XT> x[AHEAD][RW];
        auto load = [&](XOct<XT> (&o)[RW]) {            // the next slab's
#pragma unroll
          for (int i = 0; i < RW; ++i) {
            o[i].load(p, from[i], col < stop);
            from[i].next_slab();
          }
          col += 64;
        };
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) load(x[a]);
        r16 = project_rank16(p, r.tile, slot);
        for (int s0 = 0; s0 < r.slabs && ok; s0 += AHEAD) {
#pragma unroll
          for (int a = 0; a < AHEAD; ++a)
            if (s0 + a < r.slabs && ok) put(x[a], [&] { load(x[a]); });
        }
      }
      if (ok) ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.acc_full[0]), runs & 1, &ws)) != 0;
      ++runs;
      if (!ok) break;
      tc::tc_fence_after();
      const int m = (warp & 3) * 32 + lane;
      float4* out = mp.scratch + (size_t)(r.tile + blockIdx.x) * (partial_floats(p.max_rank) / 4) + m;
      for (int b = warp >> 2; b < r16; b += kWorkWarps / 4) {
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
      while (ok && walk.next(r)) {
        int slot;
        const uint32_t bytes = project_rank16(p, r.tile, slot) * 2048;
        const uint8_t* A = p.pool + (size_t)slot * p.slot_bytes + 256 + (size_t)r.slab * bytes;
        for (int s = 0; s < r.slabs && ok; ++s, ++it) {
          const int st = it % mp.stages, turn = it / mp.stages;
          ok = tc::mbar_wait(bar_of(bars.empty[st]), (turn & 1) ^ 1, &ws);
          if (!ok) break;
          if (mp.stall != 0 && it == 0 && blockIdx.x == 0) continue;
          tc::mbar_expect_tx(bar_of(bars.copied[st]), bytes);
          tc::bulk_load(tc::smem_u32(smem + (size_t)st * stage_bytes + XP * kXImage), A + (size_t)s * bytes, bytes, bar_of(bars.copied[st]));
        }
      }
    }
  } else {
    // ---- MMAs
    if (lane == 0) {
      int runs = 0;
      while (ok && walk.next(r)) {
        int slot;
        const int cols = project_rank16(p, r.tile, slot) * 16;
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
  if (ws.abort != 0) {
    if (tid == 0) report_error(&p.plan->status, LQER_ERR_TIMEOUT, 810);
    if (warp == kCopyWarp && lane == 0) {
      // the copy that the test hook withholds has the first place to itself: nothing comes there, and only the others are waited for
      if (mp.stall != 0 && blockIdx.x == 0 && it <= mp.stages) {
        for (int k = 1; k < it; ++k) drain(bar_of(bars.copied[k]), 0);
      } else {
        drain_copies(bars.copied, it, mp.stages);
      }
    }
    if (warp == kMmaWarp && lane == 0) drain_mmas(bars);
    __syncthreads();
  }
  if (warp == kMmaWarp) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, tmem_cols);
  }
}

// ---------------------------------------------------------------------------- T from its partial sums
// An item is sixteen ranks of a tile, a thread's share eight of one row: half as many CTAs as with four, each with twice the loads on
// their way (4096 rows of 5120 x 13824 rank 64 in fp32, the whole call: 108.1 -> 105.8 us).  No more CTAs than SMs.
template <int TP>
__global__ void __launch_bounds__(256) finish_kernel(const __grid_constant__ ManyParams mp) {
  const Params& p = mp.p;
  // plan and pool were there before project_kernel (see expand_kernel); its partial sums have to be waited for
  const int slabs = (p.max_rank + 63) / 64, m = threadIdx.x & 127, h = threadIdx.x >> 7;
  const ListHead head = load_head(p.plan, 1);
  const int tiles = plan_fits(p, head) ? head.n_adapted : 0;
  const Cut cut(tiles, (p.K + 63) / 64, mp.project_ctas);
  const size_t per = partial_floats(p.max_rank) / 4;
  bool waited = false;
  auto wait = [&] {
    if (waited) return;
    waited = true;
    tc::pdl_wait();
    tc::pdl_launch_dependents();                        // not before: expand_kernel's CTAs would take the places of this kernel's last ones
    if (blockIdx.x == 0 && threadIdx.x == 0) *mp.drawn = 0;
  };
  for (int item = blockIdx.x; item < tiles * slabs * 4; item += gridDim.x) {
    const int tile = item / (slabs * 4), e = item % (slabs * 4), first = e * 16 + h * 8;
    const int slot = p.tiles[tile].slot;
    const SlotHead hd = load_slot(p.pool + (size_t)max(slot, 0) * p.slot_bytes);
    const int rank = rank_of(p, slot, hd, threadIdx.x == 0 && e == 0);
    int count;
    const float4* src = mp.scratch + (size_t)(tile + cut.first_of(tile, count)) * per + (e * 4 + h * 2) * 128 + m;
    if (first >= rank) count = 0;
    wait();
    if (e * 16 >= (rank + 63) / 64 * 64) continue;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    constexpr int TOGETHER = 6;                         // stretches whose sums are on their way together
    for (int k0 = 0; k0 < count; k0 += TOGETHER) {
      float4 u[TOGETHER][2];
#pragma unroll
      for (int k = 0; k < TOGETHER; ++k) {
        u[k][0] = u[k][1] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + k < count) {
          u[k][0] = src[(k0 + k) * per];
          u[k][1] = src[(k0 + k) * per + 128];
        }
      }
#pragma unroll
      for (int k = 0; k < TOGETHER; ++k) {
        v[0] += u[k][0].x; v[1] += u[k][0].y; v[2] += u[k][0].z; v[3] += u[k][0].w;
        v[4] += u[k][1].x; v[5] += u[k][1].y; v[6] += u[k][1].z; v[7] += u[k][1].w;
      }
    }
    // beyond the rank the packed A holds zeros, and an infinite activation times zero is no zero
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = first + i < rank ? v[i] * hd.scale : 0.f;
    uint32_t w[4][TP];
#pragma unroll
    for (int i = 0; i < 4; ++i) split<TP>(v[2 * i], v[2 * i + 1], w[i]);
    uint8_t* img = mp.images + ((size_t)tile * TP * slabs + (e >> 2)) * kXImage + swizzled(m, (e & 3) * 2 + h, 128);
#pragma unroll
    for (int k = 0; k < TP; ++k) *reinterpret_cast<uint4*>(img + (size_t)k * slabs * kXImage) = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
  }
  wait();
}

// ---------------------------------------------------------------------------- Y = Y0 + T B
template <bool BF16>
struct Oct {
  uint4 a, b;                // eight values: fp32 both, bf16 a
  __device__ __forceinline__ void load(const Params& p, size_t idx) {
    if (BF16) a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Y0) + idx);
    else ld32(static_cast<const float*>(p.Y0) + idx, p.y_wide, a, b);
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
__device__ __forceinline__ void store_oct(const Params& p, size_t at, const float (&v)[8]) {
  if (!LQER_IN_BOUNDS(&p.plan->status, at * (BF16 ? 2 : 4), BF16 ? 16 : 32, p.y_extent, 812)) return;
  uint8_t* to = static_cast<uint8_t*>(p.Y) + at * (BF16 ? 2 : 4);
  if (BF16) {
    *reinterpret_cast<uint4*>(to) =
        make_uint4(round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]), round_bf16x2(v[4], v[5]), round_bf16x2(v[6], v[7]));
  } else {
    uint4 a, b;
    a.x = __float_as_uint(v[0]); a.y = __float_as_uint(v[1]); a.z = __float_as_uint(v[2]); a.w = __float_as_uint(v[3]);
    b.x = __float_as_uint(v[4]); b.y = __float_as_uint(v[5]); b.z = __float_as_uint(v[6]); b.w = __float_as_uint(v[7]);
    st32(to, p.y_wide, a, b);
  }
}

// The groups - 256 columns of a tile - are taken in order, each by the next CTA that is free: some SMs get at memory faster than others,
// and CTAs that work side by side on neighbouring columns are kind to the memory's pages (4096 rows of 5120 x 13824 rank 64 in fp32, the
// whole call, before later steps: 108 us; 112 with every 148th group for a CTA, 114 with a stretch of its own for each).  The copying warp draws them, from
// a counter in the scratch; whose work a group is changes nothing in the results.  What the other warps see of it:
struct Group { int g, rank, tile, part; };       // part: which 256 columns of the tile
struct Groups {
  uint32_t list;             // four places in shared memory
  Barriers* bars;
  int k = 0;
  // the next group (all lanes of a warp, or one thread alone); g is negative if a wait ran out
  template <bool WARP>
  __device__ __forceinline__ Group next(volatile tc::WaitState* ws) {
    const uint32_t place = k & 3;
    bool ok = tc::mbar_wait(bar_of(bars->drawn[place]), (k >> 2) & 1, ws);
    if (WARP) ok = __all_sync(0xFFFFFFFFu, ok) != 0;
    const uint4 v = lds16(list + place * 16);
    if (WARP) __syncwarp();
    if (!WARP || (threadIdx.x & 31) == 0) tc::mbar_arrive(bar_of(bars->taken[place]));
    ++k;
    return Group{ok ? (int)v.x : -1, (int)v.y, (int)v.z, (int)v.w};
  }
};

// STAGED: an fp32 Y0 is on its way a group ahead, 128 KB a CTA, by copies into shared memory.  Otherwise - rank beyond 64 (bf16 Y: 128), whose
// T leaves no room, or bf16 Y0 - it comes into registers, 64 KB a CTA.  4096 rows of 5120 x 13824 rank 64, us: fp32 108 staged, 138 not, to
// bf16 81 and 118; bf16 needs no more than 64 KB: 2048 rows of 4096 x 11008 39.5 staged, 38.5 not, rank 128 52.7 and 48.8.
template <bool Y0B, bool YB, bool STAGED>
__global__ void __launch_bounds__(kManyThreads, 1) expand_kernel(const __grid_constant__ ManyParams mp) {
  constexpr int TP = YB ? 2 : 3;
  static_assert(!STAGED || !Y0B, "fp32 Y0 only");
  constexpr int FIXED = 2;                              // groups of a CTA that need no drawing
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_at;
  __shared__ tc::WaitState ws;
  __shared__ int4 list[4];
  const Params& p = mp.p;
  uint8_t* smem = smem_raw + ((1024u - (tc::smem_u32(smem_raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int max_slabs = (p.max_rank + 63) / 64, pitch = b_pitch(p.max_rank), image = 128 * pitch;
  const uint32_t t_bytes = TP * max_slabs * kXImage;
  uint8_t* ring = smem + mp.t_sets * t_bytes;
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
  // project_kernel lets the kernels behind it start only once it has waited for all that came before the call, so plan, pool and Y0
  // may be read here at once; only what finish_kernel writes - the images of T, the counter - has to be waited for, which the
  // copying warp does.
  const ListHead head = load_head(p.plan, 1);
  const bool fits = plan_fits(p, head);
  const int NG = (p.N + 255) / 256, NC = (p.N + 127) / 128;
  const int groups = fits ? (p.Y0 == p.Y ? head.n_adapted : head.n_tiles) * NG : 0;
  // a CTA's first groups: neighbours where all CTAs get as many, so that one T serves them
  const bool side_by_side = groups >= FIXED * (int)gridDim.x;
  const int g0 = blockIdx.x * (side_by_side ? FIXED : 1), g_step = side_by_side ? 1 : gridDim.x;
  bool ok = true;
  int it = 0, tiles = 0;     // (copying and MMA warps) stages of B and tiles' T so far
  Groups mine{tc::smem_u32(list), &bars};
  if (warp < kWorkWarps) {
    // ---- accumulators and Y0 into Y: a warp has 32 rows and 32 columns of a block, a lane rows lane / 4 + 8 i and columns 8 (lane % 4) ...
    const int quarter = (warp & 3) * 32, first = (warp >> 2) * 32 + 8 * (lane & 3);
    int n = 0;                                          // turns with accumulators so far
    // Of a group: the places of the lane's first eight columns in its four rows, and which of the rows there are.
    struct Place { size_t at[4]; int col; uint32_t there; };
    auto place = [&](int tile, int part, Place& q) {
      const int rows = p.tiles[tile].rows;
      q.col = part * 256 + first;
      q.there = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = quarter + (lane >> 2) + 8 * i;
        q.at[i] = (size_t)p.rows[(size_t)tile * kManyRows + m] * p.N + q.col;
        if (m < rows) q.there |= 1u << i;
      }
    };
    // eight columns of two rows of an accumulator and of Y0, added up
    auto put = [&](const Oct<Y0B>& y, const uint32_t (&u)[16], int k, size_t at) {
      float o[8];
      y.values(o);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o[2 * j] += __uint_as_float(u[4 * j + 2 * k]);
        o[2 * j + 1] += __uint_as_float(u[4 * j + 2 * k + 1]);
      }
      store_oct<YB>(p, at, o);
    };
    // sixteen rows of an accumulator
    auto take = [&](int rank, int buf, int h, uint32_t (&u)[16]) {
      if (rank > 0) {
        tmem_ld_16x32(tmem + ((uint32_t)(quarter + 16 * h) << 16) + buf * 128 + (warp >> 2) * 32, u);
        tc::tmem_ld_wait();
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) u[i] = 0u;
      }
    };
    Place q;
    Group now, then;
    if constexpr (STAGED) {
      // Eight lanes send for the 128 bytes of a row; pairs of rows swap their 16-byte pieces, so that the lanes that read them meet no bank twice.
      const uint32_t here = tc::smem_u32(ring + (size_t)mp.stages * image) + warp * 8192;      // two blocks' shares of 32 rows
      const int piece = lane & 7, send_row = lane >> 3;
      const uint32_t to = send_row * 128 + ((piece ^ (send_row & 1)) << 4), get = (lane >> 2) * 128 + ((2 * (lane & 3) ^ (lane >> 2 & 1)) << 4);
      const uint8_t* from[8];                           // of the group that is sent for
      uint32_t from_there = 0;
      int from_col = 0;
      auto sources = [&](int tile, int part) {
        const int rows = p.tiles[tile].rows;
        from_col = part * 256 + (warp >> 2) * 32 + piece * 4;
        from_there = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int m = quarter + 4 * j + send_row;
          from[j] = static_cast<const uint8_t*>(p.Y0) + ((size_t)p.rows[(size_t)tile * kManyRows + m] * p.N + from_col) * 4;
          if (m < rows) from_there |= 1u << j;
        }
      };
      auto send = [&](int turn, bool any) {
        const uint32_t there = any && from_col + turn * 128 < p.N ? from_there : 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (there & 1u << j) cp_async16(here + turn * 4096 + j * 512 + to, from[j] + turn * 512);
        cp_async_commit();
      };
      if (g0 < groups) sources(g0 / NG, g0 % NG);
      send(0, g0 < groups);
      send(1, g0 < groups);
      now = mine.next<true>(&ws);
      while (now.g >= 0 && now.g < groups && ok) {
        then = mine.next<true>(&ws);
        if (then.g < 0) break;
        const bool more = then.g < groups;
        place(now.tile, now.part, q);
#pragma unroll
        for (int turn = 0; turn < 2; ++turn) {
          if (!ok) break;
          const int buf = n & 1;
          if (now.rank > 0) {
            ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.acc_full[buf]), (n >> 1) & 1, &ws)) != 0;
            ++n;
            tc::tc_fence_after();
          }
          cp_async_wait<1>();
          __syncwarp();
          if (!ok) break;
          const uint32_t there = q.col + turn * 128 < p.N ? q.there : 0u;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t u[16];
            take(now.rank, buf, h, u);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int i = 2 * h + k;
              const uint32_t src = here + turn * 4096 + i * 1024 + get;
              Oct<Y0B> y;
              y.a = lds16(src);
              y.b = lds16(src ^ 16);
              if (there & 1u << i) put(y, u, k, q.at[i] + turn * 128);
            }
          }
          if (now.rank > 0) tc::tc_fence_before();
          __syncwarp();
          if (now.rank > 0 && lane == 0) tc::mbar_arrive(bar_of(bars.acc_empty[buf]));
          if (turn == 0 && more) sources(then.tile, then.part);
          send(turn, more);
        }
        now = then;
      }
      cp_async_wait<0>();
    } else {
      constexpr int AHEAD = Y0B ? 2 : 1;                // blocks of 128 columns whose Y0 is on its way
      Place next;
      Oct<Y0B> y[AHEAD][4];
      if (g0 < groups) {
        place(g0 / NG, g0 % NG, next);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (next.there & 1u << i && next.col + a * 128 < p.N) y[a][i].load(p, next.at[i] + a * 128);
      }
      now = mine.next<true>(&ws);
      while (now.g >= 0 && now.g < groups && ok) {
        q = next;
        then = mine.next<true>(&ws);
        const bool more = then.g >= 0 && then.g < groups;
        if (more) place(then.tile, then.part, next);
#pragma unroll
        for (int turn = 0; turn < 2; ++turn) {
          if (!ok) break;
          const int buf = n & 1;
          if (now.rank > 0) {
            ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.acc_full[buf]), (n >> 1) & 1, &ws)) != 0;
            ++n;
            tc::tc_fence_after();
          }
          if (!ok) break;
          const uint32_t there = q.col + turn * 128 < p.N ? q.there : 0u;
          // what comes into the same registers: this group's second block, or the next group's
          const bool own = AHEAD == 1 && turn == 0;
          const int next_at = AHEAD == 2 || own ? turn * 128 + (own ? 128 : 0) : 0;
          const uint32_t coming = own ? (q.col + 128 < p.N ? q.there : 0u) : more && next.col + next_at < p.N ? next.there : 0u;
          Oct<Y0B>(&yt)[4] = y[AHEAD == 2 ? turn : 0];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t u[16];
            take(now.rank, buf, h, u);
#pragma unroll
            for (int i = 2 * h; i < 2 * h + 2; ++i)
              if (there & 1u << i) put(yt[i], u, i & 1, q.at[i] + turn * 128);
#pragma unroll
            for (int i = 2 * h; i < 2 * h + 2; ++i)
              if (coming & 1u << i) yt[i].load(p, (own ? q.at[i] : next.at[i]) + next_at);
          }
          if (now.rank > 0) {
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar_of(bars.acc_empty[buf]));
          }
        }
        now = then;
      }
    }
  } else if (warp == kCopyWarp) {
    // ---- draws the groups; copies a tile's images of T, and images of B: a stage is 128 columns of up to 64 ranks
    if (lane == 0) {
      struct Item { int g, slot, rank; };
      int at = -1, told = 0, left = 0;
      Item then{-1, -1, 0};              // the last that was told
      auto tell = [&](int g) {                          // the next group, to all warps
        const int before = then.g;
        then.g = g;
        if (g < groups && (before < 0 || before / NG != g / NG)) {
          then.slot = p.tiles[g / NG].slot;
          then.rank = rank_of(p, then.slot, load_slot(p.pool + (size_t)max(then.slot, 0) * p.slot_bytes), true);
        }
        const int slot = told & 3;
        ok = tc::mbar_wait(bar_of(bars.taken[slot]), ((told >> 2) & 1) ^ 1, &ws);
        ++told;
        if (!ok) return;
        list[slot] = make_int4(g, then.rank, g / NG, g % NG);
        tc::mbar_arrive(bar_of(bars.drawn[slot]));
      };
      // The first groups need no drawing, so that their Y0 comes while T is still being made.
      Item items[FIXED];
#pragma unroll
      for (int k = 0; k < FIXED; ++k) {
        if (k == 0 || then.g < groups) tell(g0 + k * g_step);
        items[k] = then;
      }
      tc::pdl_wait();                                   // for the counter and T
      while (items[0].g < groups && ok) {
        const int g = items[0].g, rank = items[0].rank, slot = items[0].slot;
        int draw = groups;
        if (left > 0) {
          draw = then.g + 1;
        } else if (then.g < groups) {
          // several neighbours at a time (one T for all) as long as there is much left
          const int take = then.g + 16 * (int)gridDim.x < groups ? 4 : then.g + 6 * (int)gridDim.x < groups ? 2 : 1;
          draw = FIXED * (int)gridDim.x + atomicAdd(mp.drawn, take);
          left = take;
        }
        --left;
        const int slabs = (rank + 63) / 64;
        if (g / NG != at && rank > 0) {
          at = g / NG;
          const int set = tiles % mp.t_sets, use = tiles / mp.t_sets;
          if (use > 0) ok = tc::mbar_wait(bar_of(bars.t_empty[set]), (use - 1) & 1, &ws);
          if (!ok) break;
          ++tiles;
          tc::mbar_expect_tx(bar_of(bars.t_full[set]), TP * slabs * kXImage);
          for (int x = 0; x < TP; ++x)
            for (int s = 0; s < slabs; ++s)
              tc::bulk_load(tc::smem_u32(smem + set * t_bytes + (size_t)(x * max_slabs + s) * kXImage),
                            mp.images + ((size_t)(at * TP + x) * max_slabs + s) * kXImage, kXImage, bar_of(bars.t_full[set]));
        }
        const int c0 = (g % NG) * 2, stages = (min(c0 + 2, NC) - c0) * slabs;
        const uint8_t* B = p.pool + (size_t)max(slot, 0) * p.slot_bytes + 256 + a_bytes(p.K, p.max_rank) + (size_t)c0 * slabs * image;
        for (int s = 0; s < stages && ok; ++s, ++it) {
          const int st = it % mp.stages, turn = it / mp.stages;
          ok = tc::mbar_wait(bar_of(bars.empty[st]), (turn & 1) ^ 1, &ws);
          if (!ok) break;
          tc::mbar_expect_tx(bar_of(bars.copied[st]), image);
          tc::bulk_load(tc::smem_u32(ring + (size_t)st * image), B + (size_t)s * image, image, bar_of(bars.copied[st]));
        }
#pragma unroll
        for (int k = 0; k + 1 < FIXED; ++k) items[k] = items[k + 1];
        if (ok && then.g < groups) tell(draw);
        items[FIXED - 1] = then;
      }
    }
  } else {
    // ---- MMAs
    if (lane == 0) {
      const uint32_t idesc = tc::make_idesc(128, 128);
      int n = 0, at = -1;
      for (Group now = mine.next<false>(&ws); now.g >= 0 && now.g < groups && ok; now = mine.next<false>(&ws)) {
        const int rank = now.rank, t = now.tile, slabs = (rank + 63) / 64, r16 = rank16(rank);
        if (rank == 0) continue;
        if (t != at) {
          at = t;
          if (tiles > 0) tc::umma_commit(bar_of(bars.t_empty[(tiles - 1) % mp.t_sets]));         // once what was issued so far is done
          ok = tc::mbar_wait(bar_of(bars.t_full[tiles % mp.t_sets]), tiles / mp.t_sets & 1, &ws);
          ++tiles;
        }
        const uint8_t* T = smem + (tiles - 1) % mp.t_sets * t_bytes;
        for (int turn = 0; turn < 2 && ok; ++turn, ++n) {
          ok = tc::mbar_wait(bar_of(bars.acc_empty[n & 1]), ((n >> 1) & 1) ^ 1, &ws);
          tc::tc_fence_after();
          const int stages = now.part * 2 + turn < NC ? slabs : 0;
          for (int s = 0; s < stages && ok; ++s, ++it) {
            const int st = it % mp.stages, round = it / mp.stages;
            ok = tc::mbar_wait(bar_of(bars.copied[st]), round & 1, &ws);
            if (!ok) break;
            tc::tc_fence_after();
            const uint64_t b = image_desc(tc::smem_u32(ring + (size_t)st * image), pitch);
            const int steps = min(4, r16 - s * 4);
#pragma unroll
            for (int x = TP - 1; x >= 0; --x) {
              const uint64_t a = image_desc(tc::smem_u32(T + (size_t)(x * max_slabs + s) * kXImage), 128);
              for (int h = 0; h < steps; ++h) umma(tmem + (n & 1) * 128, a + 2 * h, b + 2 * h, idesc, s > 0 || h > 0 || x < TP - 1 ? 1u : 0u);
            }
            tc::umma_commit(bar_of(bars.empty[st]));
          }
          if (ok) tc::umma_commit(bar_of(bars.acc_full[n & 1]));
        }
      }
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (ws.abort != 0) {
    if (tid == 0) report_error(&p.plan->status, LQER_ERR_TIMEOUT, 811);
    if (warp == kCopyWarp && lane == 0) {
      drain_copies(bars.t_full, tiles, mp.t_sets);
      drain_copies(bars.copied, it, mp.stages);
    }
    if (warp == kMmaWarp && lane == 0) drain_mmas(bars);
    __syncthreads();
  }
  if (warp == kMmaWarp) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, 256);
  }
}

// ---------------------------------------------------------------------------- host
constexpr size_t kSmemMost = 226 * 1024;
// The grids are no larger than kPrologueMaxCtas (launch_many takes fewer CTAs where the device has fewer SMs).
static size_t partial_bytes(int tiles, int max_rank) { return ((size_t)tiles + kPrologueMaxCtas) * partial_floats(max_rank) * 4; }
static size_t image_bytes(int tiles, int max_rank) { return (size_t)tiles * 3 * ((max_rank + 63) / 64) * kXImage; }
size_t many_scratch_bytes(int tiles, int max_rank) {
  return partial_bytes(tiles, max_rank) + image_bytes(tiles, max_rank) + 256;
}
template <class Kernel>
static cudaError_t launch(Kernel kernel, OncePerDevice& once, const ManyParams& mp, int ctas, int threads, size_t smem, cudaStream_t s) {
  cudaError_t e = once.run([=] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost); });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, mp);
}
template <int XT, int XP, int AHEAD>
static cudaError_t launch_project(ManyParams mp, cudaStream_t s) {
  static OncePerDevice once;
  const size_t stage = (size_t)XP * kXImage + rank16(mp.p.max_rank) * 2048, ring = XT == kXF32 ? (size_t)AHEAD * 2 * kXImage : 0;
  mp.stages = (int)((kSmemMost - 1024 - ring) / stage);
  if (mp.stages > kMaxStages) mp.stages = kMaxStages;
  return launch(project_kernel<XT, XP, AHEAD>, once, mp, mp.project_ctas, kManyThreads, mp.stages * stage + ring + 1024, s);
}
template <bool Y0B, bool YB>
static cudaError_t launch_expand(ManyParams mp, int ctas, cudaStream_t s) {
  static OncePerDevice once[2];
  const size_t t = (size_t)(YB ? 2 : 3) * ((mp.p.max_rank + 63) / 64) * kXImage, image = (size_t)128 * b_pitch(mp.p.max_rank);
  const size_t ring = 128 * 1024, most = kSmemMost - 1024;
  const bool staged = !Y0B && t + 2 * image + ring <= most;
  const size_t room = staged ? most - ring : most;
  mp.t_sets = 2 * t + 2 * image <= room ? 2 : 1;
  mp.stages = (int)((room - mp.t_sets * t) / image);
  if (mp.stages > kMaxStages) mp.stages = kMaxStages;
  const size_t smem = mp.t_sets * t + mp.stages * image + (staged ? ring : 0) + 1024;
  if constexpr (!Y0B)
    if (staged) return launch(expand_kernel<false, YB, true>, once[0], mp, ctas, kManyThreads, smem, s);
  return launch(expand_kernel<Y0B, YB, false>, once[1], mp, ctas, kManyThreads, smem, s);
}
cudaError_t launch_many(const Params& p, int x_type, int tiles, void* scratch, cudaStream_t s) {
  const int sms = sm_count(), ctas = sms < kPrologueMaxCtas ? sms : kPrologueMaxCtas;
  uint8_t* images = static_cast<uint8_t*>(scratch) + partial_bytes(tiles, p.max_rank);
  ManyParams mp{p, static_cast<float4*>(scratch), images, reinterpret_cast<int*>(images + image_bytes(tiles, p.max_rank)), ctas, 0, 1,
                take_stall(kFamDecode) ? 1 : 0, wait_limit_cycles()};
  LaunchScope scope(kFamDecode, s, 3);
  // fp32: three slabs on their way; two where no more fit beside two stages
  cudaError_t e = x_type == kXF32    ? (p.y_bf16           ? launch_project<kXF32, 2, 3>(mp, s)
                                        : p.max_rank <= 128 ? launch_project<kXF32, 3, 3>(mp, s)
                                                            : launch_project<kXF32, 3, 2>(mp, s))
                  : x_type == kXBF16 ? launch_project<kXBF16, 1, 6>(mp, s)
                                     : launch_project<kXMXINT8, 1, 6>(mp, s);
  if (e != cudaSuccess) return e;
  static OncePerDevice once[2];
  const int items = tiles * ((p.max_rank + 63) / 64) * 4, finish_ctas = items < ctas ? items : ctas;
  e = p.y_bf16 ? launch(finish_kernel<2>, once[0], mp, finish_ctas, 256, 0, s) : launch(finish_kernel<3>, once[1], mp, finish_ctas, 256, 0, s);
  if (e != cudaSuccess) return e;
  return p.y0_bf16 ? (p.y_bf16 ? launch_expand<true, true>(mp, ctas, s) : launch_expand<true, false>(mp, ctas, s))
                   : (p.y_bf16 ? launch_expand<false, true>(mp, ctas, s) : launch_expand<false, false>(mp, ctas, s));
}

}  // namespace ad
}  // namespace lqer
