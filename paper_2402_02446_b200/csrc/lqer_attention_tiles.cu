// Attention of prompts over the paged cache: tiles of 128 rows against tiles of 128 keys on tcgen05.
//
// The formulas are those of lqer_attention.cu.  The rows of a key head are its query heads' rows, token by token (row i * group + g), and a CTA takes
// 256 neighbours of them as two tiles, A and B: S = Q K^T (128 x 128, fp32, tensor memory), weights P (bf16, over S in tensor memory), O += P V.
// While one tile's weights are formed, the tensor cores work for the other.  Bound: the products are 4 D flops a pair at the tensor cores' rate,
// an exponential a pair at 16 a clock and SM; for heads of 128 both take the same time, so either is the limit.
//
//   warps 0-3, 4-7   tile A, tile B: a thread owns a row: scores from tensor memory, maximum, weights back to tensor memory; no exchange
//                    between threads.  The row's maximum is let lag by up to 2^8 before what is summed up is scaled anew (the sum
//                    and the values carry the same factor, so nothing is lost), which after the first tiles is rare.
//   copies           bf16: one warp, a lane a page: TMA brings pages into swizzled tiles.  MXINT8: one warp copies pages as they lie, four form the exact bf16
//                    values and store them into the same tiles.
//   issuer           one lane: per key tile and row tile, O += P V of the last key tile, in two halves as the weights come, then S of the next.
// Keys and values share a ring of tiles.  Every wait is bounded.
//
// Measured, 32/8 heads of 128, GPU time in bursts: a prompt of 8192 tokens 465 us (1.18 PFLOP/s of what a causal row sees, 0.71 of a long GEMM's burst rate; 530 us when
// it runs without a pause and the power cap lowers the clock), from MXINT8 536, heads of 64 408; windows of 1024, 32/32 heads, 7682 tokens 189, from MXINT8 219.  A key
// tile takes a CTA 3100 clocks: 16 MMAs for each row tile at some 85 clocks (64 by the rate; S reads both operands from shared memory, 128 bytes a
// clock), 2100 from S to the last weights, and the issuer's way between.  Beside its key tiles an item takes 16000: 3500 until it is known, 5000 for the queries
// (where all CTAs ask for theirs at once; 1900 by itself), 2200 until the first scores, 2500 for the results, 1300 until the next CTA, and at the end
// the second row tile is alone with its last key tile.  Tried, and not faster under a full load: CTAs that stay and take items by turns, with the next
// queries under way (460 -> 470 us); the next item's queries into L2 ahead; the first keys ahead of all others; weights by the old maximum with the new one beside
// them, which takes 800 of the 2100 clocks away but not the total; two threads a row; an issuer for each row tile (574); short loops over 32 columns (480 to 515).
//
// Where the items of 256 rows leave a last turn of CTAs half empty or more (few requests, short pieces of long prompts), that turn's items are divided over
// their keys, up to 16 CTAs to one, and a second kernel joins the parts.  Whole / divided, us: 2048 tokens behind 10240, 40/8 heads (320 items) 483 / 397, MXINT8
// 594 / 486; 512 behind 15488, 32/8 heads 212 / 123; 300 of 4000, two requests 67 / 49.  It is a kernel of its own: what it needs beside costs registers
// that those without it miss (8192 tokens 455 -> 490 us, MXINT8 520 -> 610).
#include "lqer_cache.cuh"

namespace lqer {
namespace kv {

constexpr int kRows = 128, kKeys = 128;      // of a tile
constexpr float kNear = 512.f;               // largest exponent of a row's maximum that is rounded by itself: half of its last place is 2^-16, 1.1e-5 of a weight

template <int D, bool MX>
struct Shape {
  static constexpr int TILE = 128 * D * 2, HALF = 128 * 128;               // bytes: a tile, and its part of 64 columns
  static constexpr int BLOCKS = D / 16;                                     // of 16 elements of a row
  static constexpr int STAGES = MX ? (D == 128 ? 3 : 6) : (D == 128 ? 5 : 8);
  static constexpr int RAW_STAGES = MX ? (D == 128 ? 3 : 6) : 0, RAW_EXPS = 128 * D, RAW = 128 * D + 128 * BLOCKS;   // an MXINT8 tile as it lies in the cache
  static constexpr int SMEM = 1024 + (2 + STAGES) * TILE + RAW_STAGES * RAW;
  static constexpr int COPY_WARPS = MX ? 4 : 1, COPY0 = 8, ISSUER = COPY0 + COPY_WARPS, RAW_WARP = MX ? ISSUER + 1 : -1;
  static constexpr int THREADS = MX ? 512 : 384;
  static constexpr int S_COL = 0, O_COL = 256;                              // tensor memory: S of A and B, O of A and B
};
struct Tiles {
  Attention a;
  int few;                     // requests of more rows than this are taken
  int negate;                  // the scale is negative: S = -Q K^T, and a.scale_log2 is its absolute value
  uint32_t group_inv;          // 2^32 / group rounded up (a group of 1: 0), for quotients of rows below 2^20 / group
  int stall;
  long long wait_limit;
  size_t y_extent;
  bool y_wide;                 // Y: aligned to 32 bytes
  int sms;                     // items beyond whole turns of so many CTAs may be divided over their keys; 0: none is
  struct Divided* divided;     // [1 + sms / 2]: their number (request of the first entry), and what they are
  size_t divided_extent, parts_extent;
  float* parts;                // [sms][256][D + 2]: rows' sums, then maxima and sums of weights
};
struct Barriers {
  unsigned long long full[8], empty[8], raw_full[6], raw_empty[6], s_full[2], p_half[2], p_full[2], o_done[2], q_full[2], drained;
};
__device__ __forceinline__ uint32_t bar_of(unsigned long long& b) { return tc::smem_u32(&b); }

// On the way out after a wait ran out: what the CTA has under way may still write its memory.
constexpr long long kDrainCycles = 2000000;
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
  const long long t0 = clock64();
  while (!tc::mbar_try_wait(bar, parity) && clock64() - t0 < kDrainCycles) {}
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// Descriptors in halves: of an MMA's operands only the low words, with the addresses, change from MMA to MMA.  Queries and keys: rows along the
// contraction, 128 bytes of it swizzled, 8 rows 1024 bytes apart.  Values as the second operand: their columns along memory, 64 to a swizzled row; 8 keys
// are 1024 bytes, and the next 64 columns lie a half tile on.
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t rows_desc(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | 1u << 16; }
__device__ __forceinline__ uint32_t values_desc(uint32_t saddr, int half) { return ((saddr & 0x3FFFFu) >> 4) | (uint32_t)(half >> 4) << 16; }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %5, 0;\n mov.b64 a, {%1, %3};\n mov.b64 b, {%2, %3};\n"
               " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n}\n" ::"r"(d), "r"(a), "r"(b), "r"(kDescHigh), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.b32 p, %5, 0;\n mov.b64 b, {%2, %3};\n"
               " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n}\n" ::"r"(d), "r"(a), "r"(b), "r"(kDescHigh), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// 32 bytes in one access (a whole sector), or in two where the tensor is not aligned to 32.
__device__ __forceinline__ void store32(void* p, bool aligned, const uint32_t* u) {
  if (aligned) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]) : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(u[0], u[1], u[2], u[3]);
    static_cast<uint4*>(p)[1] = make_uint4(u[4], u[5], u[6], u[7]);
  }
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {     // NaN if one is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Two fp32 operations in one instruction.
struct F2 { unsigned long long w; };
__device__ __forceinline__ F2 f2(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.w) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unf2(F2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v.w)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.w) : "l"(a.w), "l"(b.w), "l"(c.w)); return r; }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w)); return r; }
// 2^x of two values on the arithmetic units, which have time to spare where the exponential unit has not: x = n + f, n the nearest integer, and a
// polynomial of third degree in f that is nowhere in [-1/2, 1/2] more than 7.5e-5 of 2^f off (the minimax one, by Remez' exchange).
// Below 2^-125 it stays 2^-125: no more beside a row's largest weight, which is 2^-8 or more of the sums' scale, than nothing.
__device__ __forceinline__ void exp2_poly(F2 x, float& a, float& b) {
  float lo, hi;
  unf2(x, lo, hi);
  x = f2(fmaxf(lo, -125.f), fmaxf(hi, -125.f));                           // (NaN gets lost here: the row's other weights are NaN then, too)
  const F2 round = f2(12582912.f, 12582912.f), minus = f2(-1.f, -1.f);      // 1.5 * 2^23: the sum's low bits are n
  const F2 r = add2(x, round), n = add2(r, f2(-12582912.f, -12582912.f)), f = fma2(n, minus, x);
  F2 q = fma2(f, f2(0.05517166853f, 0.05517166853f), f2(0.24261112511f, 0.24261112511f));
  q = fma2(q, f, f2(0.69326096773f, 0.69326096773f));
  q = fma2(q, f, f2(0.99992805719f, 0.99992805719f));
  float ra, rb, qa, qb;
  unf2(r, ra, rb);
  unf2(q, qa, qb);
  a = __uint_as_float((__float_as_uint(ra) << 23) + __float_as_uint(qa));
  b = __uint_as_float((__float_as_uint(rb) << 23) + __float_as_uint(qb));
  // what -125 gives: what is hidden, or as good as, weighs nothing, whatever its value
  const float least = -0.99992805719f * 0x1p-125f;
  unf2(add2(f2(a, b), f2(least, least)), a, b);
}

template <int N> struct Every { static constexpr int value = N; };
// Pairs between two that take the polynomial, bf16 (8192 tokens, heads of 128 / 64, us: none 478 / 423, every eighth 472 / 411, fourth 465 / 405, third 478 / 405, second
// 506 / 440).  Beside the conversion of MXINT8, which takes the same units, there are none (530 against 542).
constexpr int kPolyEvery = 4;

// What a CTA works on: 256 rows of a request's key head from `base` on, the first of them head `head0` of the group of token `token0`; of its key tiles
// part `part` of `parts`, the `slot`-th item that is divided at all.
struct Item { int request, head, row0, n, len, base, rows, token0, head0, slot, part, parts; };      // rows: n * group
struct Divided { int request, head, row0, rows, token0, head0, base, parts; };
constexpr int kMostParts = 16, kAtOnce = 8;
// Row z of an item: its token, and its head within the group.
__device__ __forceinline__ void row_of(const Tiles& s, const Item& it, int z, int& token, int& head) {
  const uint32_t x = (uint32_t)(z + it.head0), q = s.a.group == 1 ? x : __umulhi(x, s.group_inv);
  token = it.token0 + (int)q;
  head = (int)(x - q * s.a.group);
}
// The key tiles that its two row tiles see: sink tiles, then [start, ..), `count` together; a row tile sees those of them in [from, end) and the sinks'.
template <bool DIVIDED>
struct Plan {
  int sinks, sink_tiles, start, count, skip;         // skip: turns of the parts before (DIVIDED)
  int from[2], end[2], first_pos[2], last_pos[2];
  __device__ __forceinline__ int tile(int j) const {
    if (DIVIDED) j += skip;
    return j < sinks ? j : start + j - sinks;
  }
  __device__ __forceinline__ bool sees(int t, int kv) const { return kv < (t ? end[1] : end[0]) && (kv >= (t ? from[1] : from[0]) || kv < sink_tiles); }
};
template <bool DIVIDED>
__device__ __forceinline__ Plan<DIVIDED> plan_of(const Tiles& s, const Item& it) {
  const Attention& p = s.a;
  Plan<DIVIDED> q;
  const int first = it.len - it.n;
  q.sink_tiles = p.window > 0 ? (min(p.sinks, it.len) + kKeys - 1) / kKeys : 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int lo = t * kRows, hi = min(lo + kRows, it.rows - it.base);
    const bool live = lo < hi;
    int a, b, h;
    row_of(s, it, lo, a, h);
    row_of(s, it, max(hi - 1, 0), b, h);
    q.first_pos[t] = live ? first + a : 0;
    q.last_pos[t] = live ? first + b : -1;
    q.end[t] = live ? q.last_pos[t] / kKeys + 1 : 0;
    q.from[t] = p.window > 0 ? max(0, q.first_pos[t] - p.window + 1) / kKeys : 0;
  }
  q.start = q.from[0];
  q.sinks = min(q.sink_tiles, q.start);
  q.count = q.sinks + max(q.end[0], q.end[1]) - q.start;
  q.skip = 0;
  return q;
}
// The CTA's item, to where all threads find it; heavy ones (a request's last) first.  False: there is none.  Of up to 32 requests every warp
// knows the sums by itself.
template <bool DIVIDED>
__device__ __forceinline__ bool find_item(const Tiles& s, Item& found) {
  const Attention& p = s.a;
  const StepRequest* reqs = requests_of(p.step);
  __shared__ int sums[16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const bool one = p.R <= 32;
  const int per = one ? 1 : (p.R + blockDim.x - 1) / blockDim.x, from = min((one ? lane : tid) * per, p.R), to = min(from + per, p.R);
  auto items_of = [&](const int4& w) {
    const int rows = w.y * p.group;
    return w.y > 0 && rows > s.few ? (rows + 2 * kRows - 1) / (2 * kRows) : 0;
  };
  int4 w = make_int4(0, 0, 0, 0);
  int mine = 0;
  for (int r = from; r < to; ++r) {
    w = *reinterpret_cast<const int4*>(reqs + r);
    mine += items_of(w);
  }
  int x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xFFFFFFFFu, x, o); if (lane >= o) x += y; }
  int before = x - mine, total = __shfl_sync(0xFFFFFFFFu, x, 31);
  if (!one) {
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    total = 0;
    for (int k = 0; k < warps; ++k) { if (k < warp) before += sums[k]; total += sums[k]; }
  }
  // All but the last turn of CTAs take an item each; what is left, if it would keep no more than half of them busy, is divided.
  const uint32_t all = (uint32_t)(total * p.hkv);                  // (the host has seen to it that this fits)
  const uint32_t left = DIVIDED ? all % (uint32_t)s.sms : 0u, parts = left > 0 ? min((uint32_t)s.sms / left, (uint32_t)kMostParts) : 1u;
  const uint32_t undivided = parts > 1 ? all - left : all;
  if (DIVIDED && blockIdx.x == 0 && tid == 0) s.divided[0].request = parts > 1 ? (int)left : 0;
  const bool whole = blockIdx.x < undivided;
  const uint32_t beyond = whole ? 0u : blockIdx.x - undivided, slot = DIVIDED ? beyond / parts : beyond, number = whole ? blockIdx.x : undivided + slot;
  if (number >= all) return false;
  const uint32_t back = number / (uint32_t)p.hkv, head = number - back * p.hkv;
  const int index = total - 1 - (int)back;
  if (index >= before && index < before + mine && (!one || warp == 0)) {
    for (int r = from;; ++r) {
      if (per > 1) w = *reinterpret_cast<const int4*>(reqs + r);
      const int c = items_of(w);
      if (index < before + c) {
        const int base = (index - before) * 2 * kRows, token = base / p.group;
        found = Item{r, (int)head, w.x, w.y, w.z, base, w.y * p.group, token, base - token * p.group, whole ? -1 : (int)slot,
                     whole ? 0 : (int)(beyond - slot * parts), whole ? 1 : (int)parts};
        break;
      }
      before += c;
    }
  }
  __syncthreads();
  return true;
}
// The columns of a key tile from key0 on that the row at `pos` sees, 32 to a word.
__device__ __forceinline__ uint32_t upto(int n) { return n < 0 ? 0u : n >= 31 ? 0xFFFFFFFFu : (2u << n) - 1u; }       // bits 0 .. n
__device__ __forceinline__ uint32_t seen_columns(const Attention& p, int pos, int key0, int k) {
  uint32_t w = upto(pos - key0 - 32 * k);
  if (p.window > 0) w &= ~upto(pos - p.window - key0 - 32 * k) | upto(p.sinks - 1 - key0 - 32 * k);
  return w;
}

template <int D, bool MX, bool DIVIDED>
__global__ void __launch_bounds__(Shape<D, MX>::THREADS, 1)
tiles_kernel(const Tiles s, const __grid_constant__ CUtensorMap key_map, const __grid_constant__ CUtensorMap value_map) {
  using SH = Shape<D, MX>;
  extern __shared__ uint8_t dynamic[];
  __shared__ Barriers bars;
  __shared__ uint32_t tmem_at;
  __shared__ tc::WaitState ws;
  const Attention& p = s.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t q_at = (tc::smem_u32(dynamic) + 1023u) & ~1023u, ring_at = q_at + 2 * SH::TILE, raw_at = ring_at + SH::STAGES * SH::TILE;
  uint8_t* const q_mem = dynamic + (q_at - tc::smem_u32(dynamic));
  uint8_t* const ring_mem = q_mem + 2 * SH::TILE;
  if (tid == 0) {
    for (int i = 0; i < SH::STAGES; ++i) {
      tc::mbar_init(bar_of(bars.full[i]), SH::COPY_WARPS);
      tc::mbar_init(bar_of(bars.empty[i]), 1);
    }
    for (int i = 0; i < SH::RAW_STAGES; ++i) {
      tc::mbar_init(bar_of(bars.raw_full[i]), 1);
      tc::mbar_init(bar_of(bars.raw_empty[i]), SH::COPY_WARPS);
    }
    for (int t = 0; t < 2; ++t) {
      tc::mbar_init(bar_of(bars.s_full[t]), 1);
      tc::mbar_init(bar_of(bars.p_half[t]), 4);
      tc::mbar_init(bar_of(bars.p_full[t]), 4);
      tc::mbar_init(bar_of(bars.o_done[t]), 1);
      tc::mbar_init(bar_of(bars.q_full[t]), 4 + (s.stall && blockIdx.x == 0 ? 1 : 0));
    }
    tc::mbar_init(bar_of(bars.drained), 1);
    tc::fence_barrier_init();
    ws.abort = 0;
    ws.limit = s.wait_limit;
    if (!MX) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&key_map)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&value_map)) : "memory");
    }
  }
  tc::pdl_wait();
  if (!step_fits(p, blockIdx.x == 0 && tid == 0)) {
    if (DIVIDED && blockIdx.x == 0 && tid == 0) s.divided[0].request = 0;
    return;
  }
  __shared__ Item item;
  if (!find_item<DIVIDED>(s, item)) return;
  const Item it = item;
  Plan<DIVIDED> plan = plan_of<DIVIDED>(s, it);
  int parts = 1;
  if constexpr (DIVIDED) {
    if (it.slot >= 0) {
      // a part has two key tiles or so (of an odd count one has a single one); an item with few has fewer parts
      parts = min(it.parts, max((plan.count + 1) / 2, 1));
      if (it.part == 0 && tid == 0 && LQER_IN_BOUNDS(&p.step->status, (size_t)(1 + it.slot) * sizeof(Divided), sizeof(Divided), s.divided_extent, 67))
        s.divided[1 + it.slot] = Divided{it.request, it.head, it.row0, it.rows, it.token0, it.head0, it.base, parts};
      if (it.part >= parts) return;
      plan.skip = (int)((long long)plan.count * it.part / parts);
      plan.count = (int)((long long)plan.count * (it.part + 1) / parts) - plan.skip;
    }
  }
  if (warp == SH::ISSUER) tc::tmem_alloc(tc::smem_u32(&tmem_at), 512);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  tc::pdl_launch_dependents();         // not before: a CTA of the next kernel could take tensor memory on this SM first, and then wait for this kernel to end
  const uint32_t tmem = tmem_at;
  const int* table = p.tables + (size_t)it.request * p.max_pages;
  // keys that no row of the step sees: from the end on, and between the first tokens and the window
  const int seen_from = p.window > 0 ? max(0, it.len - it.n - p.window + 1) : 0;
  auto unseen = [&](int key) { return key >= it.len || (key < seen_from && key >= p.sinks); };
  auto has_unseen = [&](int key0) { return key0 + kKeys > it.len || (key0 < seen_from && key0 + kKeys > p.sinks); };
  int copies = 0;
  bool ok = true;

  if (warp < 8) {
    // ---- a row tile
    // registers: what the launch gave, 128 x 512 or 168 x 384, shared out anew: 2 x 192 + 96 + 32 = 4 x 128, 2 x 216 + 72 = 3 x 168
    // (what the warps take together is what the block was launched with: 4 warpgroups of 128)
    if constexpr (MX && DIVIDED) asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    else if constexpr (MX) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int t = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;
    const uint32_t s_at = tmem + lanes + SH::S_COL + t * 128, o_at = tmem + lanes + SH::O_COL + t * D;
    const int left = it.rows - it.base - t * kRows;               // rows from the tile's first on
    {
      // queries, as the MMA reads them; 16 bytes a thread, the tile's rows in turn
      constexpr int PER = D / 8, STEP = 128 / PER;
      uint8_t* const to = q_mem + t * SH::TILE;
      const int c = row % PER, r0 = row / PER;
      const uint16_t* from = static_cast<const uint16_t*>(p.Q) + (size_t)it.row0 * p.q_stride + (size_t)(it.head * p.group) * D + 8 * c;
      uint4 v[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int r = r0 + i * STEP;
        int token, head;
        row_of(s, it, t * kRows + r, token, head);
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < left) v[i] = *reinterpret_cast<const uint4*>(from + (size_t)token * p.q_stride + head * D);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int r = r0 + i * STEP;
        *reinterpret_cast<uint4*>(to + (c >> 3) * SH::HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[i];
      }
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar_of(bars.q_full[t]));
    }
    const int first_pos = t ? plan.first_pos[1] : plan.first_pos[0], last_pos = t ? plan.last_pos[1] : plan.last_pos[0];
    int token, head;
    row_of(s, it, t * kRows + max(min(row, left - 1), 0), token, head);
    const int pos = it.len - it.n + token;
    const float c = p.scale_log2;
    const F2 c2 = f2(c, c);
    // Of the key tiles that have something that no row sees the first row tile clears the values of those that it sees, the second those beyond, which are behind the
    // window: so nobody writes what is being read (products are issued for the first row tile first, and not before its weights are there).
    const int clear_end = max(it.len - kKeys + 1, t ? plan.end[0] * kKeys : 0), clear_seen = t ? 0 : seen_from;
    // Exponents are s c - m c in one operation, with m c rounded once.  That is off by 2^-24 of m c, the same for the whole row, and no more than the
    // polynomial is up to kNear.  Of larger ones, in any row of the warp, the difference is taken first: from 2^30 on the rounding alone would leave the range
    // of an exponent.  There a maximum that is infinite or NaN makes all weights NaN, too; the polynomial alone would hide it.
    float m = -INFINITY, base = 0.f;
    bool far = false;
    F2 la = f2(0.f, 0.f), lb = f2(0.f, 0.f);                       // sums of weights, four to a row
    int n = 0;                                                     // key tiles so far
    for (int j = 0; j < plan.count && ok; ++j) {
      const int kv = plan.tile(j), key0 = kv * kKeys;
      if (!plan.sees(t, kv)) continue;
      ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.s_full[t]), n & 1, &ws)) != 0;
      if (!ok) break;
      tc::tc_fence_after();
      float v[128];
#pragma unroll
      for (int k = 0; k < 2; ++k) tc::tmem_ld32(s_at + 32 * k, *reinterpret_cast<uint32_t(*)[32]>(&v[32 * k]));
      if constexpr (!MX) {
        if (key0 >= clear_end || (key0 < clear_seen && key0 + kKeys > p.sinks)) {
          // values that no row sees may be anything: 0 times that has to be 0
          const int at = 2 * j + 1;
          ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.full[at % SH::STAGES]), at / SH::STAGES & 1, &ws)) != 0;
          if (!ok) break;
          if (unseen(key0 + row)) {
            uint4* to = reinterpret_cast<uint4*>(ring_mem + (at % SH::STAGES) * SH::TILE + row * 128);
#pragma unroll
            for (int h = 0; h < D / 64; ++h)
#pragma unroll
              for (int i = 0; i < 8; ++i) to[h * (SH::HALF / 16) + i] = make_uint4(0u, 0u, 0u, 0u);
          }
          tc::fence_proxy_async_smem();
        }
      }
      const bool masked = key0 + kKeys - 1 > first_pos || (p.window > 0 && key0 <= last_pos - p.window);
      // the second half of the scores is on its way while the first half's maximum is taken
      float bigs[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        tc::tmem_ld_wait();
        if (h == 0) {
#pragma unroll
          for (int k = 2; k < 4; ++k) tc::tmem_ld32(s_at + 32 * k, *reinterpret_cast<uint32_t(*)[32]>(&v[32 * k]));
        }
        if (masked) {
#pragma unroll
          for (int k = 2 * h; k < 2 * h + 2; ++k) {
            const uint32_t seen = seen_columns(p, pos, key0, k);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[32 * k + i] = seen & (1u << i) ? v[32 * k + i] : -INFINITY;
          }
        }
        float* const x = v + 64 * h;
#pragma unroll
        for (int k = 0; k < 8; ++k) bigs[k] = h == 0 ? max3(x[k], x[k + 8], x[k + 16]) : max3(bigs[k], x[k], x[k + 8]);
#pragma unroll
        for (int i = 24 - 8 * h; i < 56; i += 16)
#pragma unroll
          for (int k = 0; k < 8; ++k) bigs[k] = max3(bigs[k], x[i + k], x[i + k + 8]);
        if (h == 0) {
#pragma unroll
          for (int k = 0; k < 8; ++k) bigs[k] = max3(bigs[k], x[56 + k], x[56 + k]);
        }
      }
      const float big = max3(max3(bigs[0], bigs[1], bigs[2]), max3(bigs[3], bigs[4], bigs[5]), max3(bigs[6], bigs[7], bigs[7]));
      const bool up = !((big - m) * c <= 8.f) && big != -INFINITY;     // (from nothing, and for NaN, too)
      if (__any_sync(0xFFFFFFFFu, up)) {
        const float f = up ? exp2_fast((m - big) * c) : 1.f;
        if (up) m = big;
        if (n > 0) {
          la = fma2(la, f2(f, f), f2(0.f, 0.f));
          lb = fma2(lb, f2(f, f), f2(0.f, 0.f));
          ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.o_done[t]), (n - 1) & 1, &ws)) != 0;
          if (!ok) break;
          tc::tc_fence_after();
#pragma unroll 1
          for (int k = 0; k < D / 16; ++k) {
            uint32_t o[16];
            tc::tmem_ld16(o_at + 16 * k, o);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st16(o_at + 16 * k, o);
          }
        }
        base = m == -INFINITY ? 0.f : -m * c;
        far = __any_sync(0xFFFFFFFFu, !(fabsf(base) <= kNear));
        if (far) base = 0.f;
      }
      if (far) {
        const float top = m == -INFINITY ? 0.f : m, less = (top - top) - top;
        const F2 less2 = f2(less, less);
#pragma unroll
        for (int i = 0; i < 128; i += 2) unf2(add2(f2(v[i], v[i + 1]), less2), v[i], v[i + 1]);
      }
      const F2 base2 = f2(base, base);
      // the weights, and word to the issuer, which may begin with the first half; POLY: every POLY-th pair by the polynomial
      auto weights = [&](auto every) {
        constexpr int POLY = decltype(every)::value;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const F2 x = fma2(f2(v[32 * k + 2 * i], v[32 * k + 2 * i + 1]), c2, base2);
            float a, b;
            if (POLY > 0 && i % (POLY > 0 ? POLY : 1) == POLY - 1) {
              exp2_poly(x, a, b);
            } else {
              unf2(x, a, b);
              a = exp2_fast(a);
              b = exp2_fast(b);
            }
            if (i % 2) lb = add2(lb, f2(a, b));
            else la = add2(la, f2(a, b));
            w[i] = round_bf16x2(a, b);                            // as in lqer_attention.cu: the weights are rounded, their sum is not
          }
          if (k == 2) {                                           // (by now the first half has arrived, so this waits for nothing)
            tmem_st_wait();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar_of(bars.p_half[t]));
          }
          tmem_st16(s_at + 16 * k, w);
        }
        tmem_st_wait();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar_of(bars.p_full[t]));
      };
      // (one for all tiles: without one of their own for tiles in which something is hidden, 8192 tokens 459 -> 454 us, the window's 217 -> 213)
      weights(Every<MX ? 0 : kPolyEvery>{});
      ++n;
    }
    if (ok && n > 0) {
      ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.o_done[t]), (n - 1) & 1, &ws)) != 0;
      tc::tc_fence_after();
    }
    float l[4];
    unf2(la, l[0], l[1]);
    unf2(lb, l[2], l[3]);
    const float all = (l[0] + l[1]) + (l[2] + l[3]);
    if (DIVIDED && parts > 1) {
      // a part's sums as they are; where it saw nothing, only that it did not
      const size_t part_at = (size_t)(it.slot * it.parts + it.part) * 2 * kRows * (D + 2);
      float* const part = s.parts + part_at + (size_t)(t * kRows + row) * D;
      float* const marks = s.parts + part_at + (size_t)2 * kRows * D + t * kRows + row;
      const bool fits = LQER_IN_BOUNDS(&p.step->status, part_at * 4, (size_t)2 * kRows * (D + 2) * 4, s.parts_extent, 68);
      if (ok && left > 0 && fits) {
        marks[0] = n > 0 ? m : -INFINITY;                          // (of the scores as they are: the join scales differences, too)
        marks[2 * kRows] = all;
      }
#pragma unroll 1
      for (int k = 0; k < D / 32 && ok && n > 0; ++k) {
        uint32_t o[32];
        tc::tmem_ld32(o_at + 32 * k, o);
        tc::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (fits) store32(part + 32 * k + 8 * i, true, o + 8 * i);
      }
    } else if (ok && n > 0) {
      const float inv = 1.f / all;
      const size_t at = ((size_t)(it.row0 + token) * p.hq + it.head * p.group + head) * D;
      const bool mine = row < left && LQER_IN_BOUNDS(&p.step->status, at * 2, D * 2, s.y_extent, 62);
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        uint32_t o[32], w[16];
        tc::tmem_ld32(o_at + 32 * k, o);
        tc::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = round_bf16x2(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
        if (mine) {
          uint16_t* const to = static_cast<uint16_t*>(p.Y) + at + 32 * k;
          store32(to, s.y_wide, w);
          store32(to + 16, s.y_wide, w + 8);
        }
      }
    }
  } else if (warp < SH::ISSUER) {
    if constexpr (!MX) {
      // ---- copies: a lane a page
      asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
      const int pages = kKeys >> p.page_shift;
      for (int j = 0; j < plan.count && ok; ++j) {
        const int key0 = plan.tile(j) * kKeys, key = key0 + (lane << p.page_shift);
        const bool mine = lane < pages && key < it.len;
        const int id = mine ? checked_page(p, table[key >> p.page_shift], it.request) : 0;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, mine)) * (uint32_t)(p.page * D * 2);
        for (int which = 0; which < 2; ++which, ++copies) {
          const int at = copies % SH::STAGES;
          if (copies >= SH::STAGES) ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.empty[at]), (copies / SH::STAGES - 1) & 1, &ws)) != 0;
          if (!ok) break;
          if (lane == 0) tc::mbar_expect_tx(bar_of(bars.full[at]), bytes);
          __syncwarp();
          if (mine) {
            const uint32_t to = ring_at + at * SH::TILE + (uint32_t)(lane << p.page_shift) * 128;
#pragma unroll
            for (int h = 0; h < D / 64; ++h)
              tma_load_4d(to + h * SH::HALF, which ? &value_map : &key_map, 64 * h, 0, it.head, id, bar_of(bars.full[at]));
          }
        }
      }
    } else {
      // ---- mantissas, as they lie in the cache, into swizzled bf16 values; a lane a block of 16, its row's other blocks beside it
      if constexpr (DIVIDED) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
      else asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
      constexpr int B = SH::BLOCKS, N = B, STEP = 128 / B;         // a thread's blocks of a tile, and the rows between them
      const int k = tid - 256, b = k % B, r0 = k / B, shift = p.bits - 2;
      const uint8_t* const raw_mem = ring_mem + SH::STAGES * SH::TILE;
      // the two halves' columns lie on the same banks: their lanes store their chunks in opposite order
      const int turn = D == 128 ? b >> 2 : 0, c = 2 * (b & 3);
      const uint32_t to0 = (b >> 2) * SH::HALF + r0 * 128 + (((c + turn) ^ (r0 & 7)) << 4), to1 = (b >> 2) * SH::HALF + r0 * 128 + (((c + 1 - turn) ^ (r0 & 7)) << 4);
      for (int x = 0; x < 2 * plan.count && ok; ++x) {
        const int at = x % SH::STAGES, raw = x % SH::RAW_STAGES, key0 = plan.tile(x >> 1) * kKeys;
        ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.raw_full[raw]), x / SH::RAW_STAGES & 1, &ws)) != 0;
        if (!ok) break;
        const uint8_t* const from = raw_mem + raw * SH::RAW;
        uint4 m[N];
        uint32_t e[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          m[i] = *reinterpret_cast<const uint4*>(from + (r0 + i * STEP) * D + b * 16);
          e[i] = from[SH::RAW_EXPS + (r0 + i * STEP) * B + b];
        }
        if (has_unseen(key0)) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (unseen(key0 + r0 + i * STEP)) { m[i] = make_uint4(0u, 0u, 0u, 0u); e[i] = 127; }
        }
        if (x >= SH::STAGES) ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.empty[at]), (x / SH::STAGES - 1) & 1, &ws)) != 0;
        if (!ok) break;
        uint8_t* const to = ring_mem + at * SH::TILE;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const MantissaScale sc = mantissa_scale(e[i], shift);
          const uint4 w0 = mantissas8(make_uint2(m[i].x, m[i].y), sc), w1 = mantissas8(make_uint2(m[i].z, m[i].w), sc);
          *reinterpret_cast<uint4*>(to + to0 + i * STEP * 128) = turn ? w1 : w0;          // (STEP is a multiple of 8: the swizzle stays)
          *reinterpret_cast<uint4*>(to + to1 + i * STEP * 128) = turn ? w0 : w1;
        }
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tc::mbar_arrive(bar_of(bars.full[at]));
          tc::mbar_arrive(bar_of(bars.raw_empty[raw]));
        }
      }
    }
  } else if (warp == SH::ISSUER) {
    if constexpr (MX && DIVIDED) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    else if constexpr (MX) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    // The whole warp walks along, so that addresses stay in uniform registers; one lane issues.
    const bool leader = tc::elect_one();
    const uint32_t s_idesc = tc::make_idesc(128, 128) | (s.negate ? 1u << 13 : 0u), o_idesc = tc::make_idesc(128, D) | 1u << 16;
    const uint32_t base = __shfl_sync(0xFFFFFFFFu, tmem, 0);
    auto all = [&](bool got) { ok = __all_sync(0xFFFFFFFFu, got) != 0; return ok; };
    auto scores = [&](int t, int k_at) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t off = (k >> 2) * (SH::HALF >> 4) + (k & 3) * 2;
        mma_ss(base + SH::S_COL + t * 128, rows_desc(q_at + t * SH::TILE) + off, rows_desc(ring_at + k_at * SH::TILE) + off, s_idesc, k > 0 ? 1u : 0u);
      }
      tc::umma_commit(bar_of(bars.s_full[t]));
    };
    int n[2] = {0, 0};                                             // key tiles whose O is under way
    int at = 0;                                                    // place in the ring, and how often it has been round
    uint32_t phase = 0;
    // the first scores, of each row tile as soon as its queries are there
    if (all(tc::mbar_wait(bar_of(bars.full[0]), 0, &ws))) {
#pragma unroll 1
      for (int t = 0; t < 2 && all(tc::mbar_wait(bar_of(bars.q_full[t]), 0, &ws)); ++t) {
        tc::tc_fence_after();
        if (plan.sees(t, plan.tile(0)) && leader) scores(t, 0);
      }
      if (leader) tc::umma_commit(bar_of(bars.empty[0]));
      at = 1;
    }
    for (int j = 1; j <= plan.count && ok; ++j) {                  // values of tile j - 1, keys of tile j
      const int v_at = at;
      if (!all(tc::mbar_wait(bar_of(bars.full[v_at]), phase, &ws))) break;
      if (++at == SH::STAGES) { at = 0; phase ^= 1; }
      const int k_at = at;
      const uint32_t k_phase = phase;
      bool keys_there = false;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (plan.sees(t, plan.tile(j - 1))) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (!all(tc::mbar_wait(bar_of(half ? bars.p_full[t] : bars.p_half[t]), n[t] & 1, &ws))) break;
            tc::tc_fence_after();
            if (leader) {
#pragma unroll
              for (int k = 4 * half; k < 4 * half + 4; ++k)
                mma_ts(base + SH::O_COL + t * D, base + SH::S_COL + t * 128 + 8 * k, values_desc(ring_at + v_at * SH::TILE, SH::HALF) + k * 128, o_idesc,
                       k > 0 ? 1u : n[t] > 0 ? 1u : 0u);
              if (half) tc::umma_commit(bar_of(bars.o_done[t]));
            }
          }
          if (!ok) break;
          ++n[t];
        }
        if (j < plan.count) {
          if (!keys_there) {
            if (!all(tc::mbar_wait(bar_of(bars.full[k_at]), k_phase, &ws))) break;
            tc::tc_fence_after();
            keys_there = true;
          }
          if (plan.sees(t, plan.tile(j)) && leader) scores(t, k_at);
        }
      }
      if (!ok) break;
      if (leader) {
        tc::umma_commit(bar_of(bars.empty[v_at]));
        if (j < plan.count) tc::umma_commit(bar_of(bars.empty[k_at]));
      }
      if (++at == SH::STAGES) { at = 0; phase ^= 1; }
    }
  } else {
    if constexpr (MX && DIVIDED) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    else if constexpr (MX) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == SH::RAW_WARP) {
      // ---- copies of an MXINT8 cache: a lane a page
      const int pages = kKeys >> p.page_shift;
      for (int j = 0; j < plan.count && ok; ++j) {
        const int key0 = plan.tile(j) * kKeys, key = key0 + (lane << p.page_shift);
        const bool mine = lane < pages && key < it.len;
        const int id = mine ? checked_page(p, table[key >> p.page_shift], it.request) : 0;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, mine)) * (uint32_t)(p.page * (D + D / 16));
        const size_t block = ((((size_t)id * p.hkv + it.head) << p.page_shift)) * SH::BLOCKS;      // of 16 elements
        for (int which = 0; which < 2; ++which, ++copies) {
          const int at = copies % SH::RAW_STAGES;
          if (copies >= SH::RAW_STAGES) ok = __all_sync(0xFFFFFFFFu, tc::mbar_wait(bar_of(bars.raw_empty[at]), (copies / SH::RAW_STAGES - 1) & 1, &ws)) != 0;
          if (!ok) break;
          if (lane == 0) tc::mbar_expect_tx(bar_of(bars.raw_full[at]), bytes);
          __syncwarp();
          if (mine) {
            const uint32_t to = raw_at + at * SH::RAW, place = lane << p.page_shift;
            tc::bulk_load(to + place * D, static_cast<const uint8_t*>(which ? p.values : p.keys) + block * 16, p.page * D, bar_of(bars.raw_full[at]));
            tc::bulk_load(to + SH::RAW_EXPS + place * SH::BLOCKS, (which ? p.value_exps : p.key_exps) + block, p.page * SH::BLOCKS, bar_of(bars.raw_full[at]));
          }
        }
      }
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  if (ws.abort != 0) {
    if (tid == 0) report_error(&p.step->status, LQER_ERR_TIMEOUT, 820);
    if (warp == (MX ? SH::RAW_WARP : SH::COPY0) && lane == 0) {
      constexpr int PLACES = MX ? SH::RAW_STAGES : SH::STAGES;
      for (int k = 0; k < PLACES && k < copies; ++k) {
        const int last = copies - 1 - k;
        drain(bar_of(MX ? bars.raw_full[last % PLACES] : bars.full[last % PLACES]), last / PLACES & 1);
      }
    }
    if (warp == SH::ISSUER && tc::elect_one()) {
      tc::umma_commit(bar_of(bars.drained));
      drain(bar_of(bars.drained), 0);
    }
    __syncthreads();
  }
  if (warp == SH::ISSUER) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, 512);
  }
}

// Joins the parts of the items that were divided, in the order of the keys: blockIdx.x is an item, blockIdx.y 1024 / D of its rows, a thread four columns of one.
// (32 rows to a CTA, and the parts one behind the other, made 64 rows behind 4000 31 us instead of 23; all 16 at once 512 behind 15488 141 instead of 137.)
template <int D>
__global__ void __launch_bounds__(256, 4) join_tiles_kernel(const Tiles s) {
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const Attention& p = s.a;
  if ((int)blockIdx.x >= s.divided[0].request) return;
  const Divided q = s.divided[1 + blockIdx.x];
  if (q.parts < 2) return;
  // places of the parts go by how many the items were to have
  const int planned = min(s.sms / s.divided[0].request, kMostParts);
  const float* const first = s.parts + (size_t)blockIdx.x * planned * 2 * kRows * (D + 2);
  const int row = blockIdx.y * (1024 / D) + threadIdx.x / (D / 4), d = 4 * (threadIdx.x % (D / 4));
  if (row >= q.rows - q.base) return;
  float big = -INFINITY, all = 0.f;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int at = 0; at < q.parts; at += kAtOnce) {                  // what so many parts say is all asked for before any of it is used
    float m[kAtOnce], l[kAtOnce];
    float4 x[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float* const part = first + (size_t)(at + k) * 2 * kRows * (D + 2);
      m[k] = -INFINITY;
      l[k] = 0.f;
      if (at + k < q.parts) {
        m[k] = part[(size_t)2 * kRows * D + row];
        l[k] = part[(size_t)2 * kRows * D + 2 * kRows + row];
        x[k] = *reinterpret_cast<const float4*>(part + (size_t)row * D + d);
      }
    }
    float top = big;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) top = fmaxf(top, m[k]);
    const float base = top == -INFINITY ? 0.f : top, f0 = exp2_fast((big - base) * p.scale_log2);
    sum.x *= f0; sum.y *= f0; sum.z *= f0; sum.w *= f0;
    all *= f0;
    big = top;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (l[k] == 0.f) continue;                                   // nothing was put there, or nothing of weight
      const float f = exp2_fast((m[k] - base) * p.scale_log2);
      sum.x += f * x[k].x; sum.y += f * x[k].y; sum.z += f * x[k].z; sum.w += f * x[k].w;
      all += f * l[k];
    }
  }
  const float inv = 1.f / all;
  const uint32_t z = (uint32_t)(row + q.head0), token = p.group == 1 ? z : __umulhi(z, s.group_inv), head = z - token * p.group;
  const size_t at = ((size_t)(q.row0 + q.token0 + token) * p.hq + q.head * p.group + head) * D + d;
  if (LQER_IN_BOUNDS(&p.step->status, at * 2, 8, s.y_extent, 64))
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.Y) + at) = make_uint2(round_bf16x2(sum.x * inv, sum.y * inv), round_bf16x2(sum.z * inv, sum.w * inv));
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<EncodeTiledFn>(f);
  }();
  return fn;
}
// 64 columns of a page of one head; x is 0 or 64, so a copy starts on a 128-byte boundary.
static bool page_map(CUtensorMap* map, const void* base, const lqer_kv_cache_t& c) {
  const EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return false;
  const cuuint64_t row = (cuuint64_t)c.head_dim * 2;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page, (cuuint64_t)c.kv_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t strides[3] = {row, row * c.page, row * c.page * c.kv_heads};
  const cuuint32_t box[4] = {64, (cuuint32_t)c.page, 1, 1}, ones[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool MX, bool DIVIDED>
static cudaError_t launch_shape(const Tiles& k, int ctas, const lqer_kv_cache_t& c, cudaStream_t s) {
  using SH = Shape<D, MX>;
  static OncePerDevice once;
  cudaError_t e = once.run([] { return cudaFuncSetAttribute(tiles_kernel<D, MX, DIVIDED>, cudaFuncAttributeMaxDynamicSharedMemorySize, SH::SMEM); });
  if (e != cudaSuccess) return e;
  CUtensorMap maps[2] = {};
  if (!MX && (!page_map(&maps[0], c.keys, c) || !page_map(&maps[1], c.values, c))) return cudaErrorInvalidValue;
  LaunchScope scope(kFamDecode, s, DIVIDED ? 2 : 1);
  e = launch_after(tiles_kernel<D, MX, DIVIDED>, dim3(ctas), SH::THREADS, SH::SMEM, s, k, maps[0], maps[1]);
  if (e != cudaSuccess || !DIVIDED) return e;
  return launch_after(join_tiles_kernel<D>, dim3(k.sms / 2, 2 * kRows * D / 1024), 256, 0, s, k);
}
// Whether items may be divided: a division costs a launch and the way of the parts through memory, some 5 us, and gains what the last turn of CTAs leaves of it, if the
// rows are where they can be, and the keys as many (some 1.8 us for 128).  Not divided / divided, us: 300 tokens, 32/8 heads: 15 / 20, of 600: 19 / 25, of 1000: 23 / 22,
// of 4000, 1100 tokens, 32/32 heads, MXINT8: 120 / 98, of 16000, 512 tokens: 212 / 123.  Where the rows begin is not known here: the last turn's items of a whole prompt are its
// first rows, which see few keys, so that nothing gets divided and the variant is taken for nothing (4096 tokens, 32/8 heads: 138 / 154, MXINT8 161 / 175; 7680: 414 / 436).
static bool may_divide(const Attention& a) {
  const int sms = sm_count();
  if (sms < 2) return false;
  const long long rows = (long long)a.M * a.group, items = (rows + 2 * kRows - 1) / (2 * kRows) * a.hkv, left = items % sms;
  if (left == 0 || left > sms / 2) return false;
  const long long room = (long long)a.max_pages * a.page, keys = a.window > 0 && a.window + 2 * kRows < room ? a.window + 2 * kRows : room;
  const double turn = 1.8 * (double)((keys + kKeys - 1) / kKeys), parts = (double)(sms / left < kMostParts ? sms / left : kMostParts);
  return turn * (1.0 - 1.0 / parts) > 10.0;
}
static size_t divided_bytes() { return ((size_t)(1 + sm_count() / 2) * sizeof(Divided) + 255) & ~(size_t)255; }
size_t tiles_scratch_bytes(const Attention& a, int head_dim) {
  return may_divide(a) ? divided_bytes() + (size_t)sm_count() * 2 * kRows * (head_dim + 2) * sizeof(float) : 0;
}
cudaError_t launch_tiles(const Attention& a, int few, size_t y_extent, const lqer_kv_cache_t& c, void* scratch, cudaStream_t s) {
  Tiles k = {};
  if (may_divide(a)) {
    k.sms = sm_count();
    k.divided_extent = divided_bytes();
    k.parts_extent = (size_t)k.sms * 2 * kRows * (c.head_dim + 2) * sizeof(float);
    k.divided = static_cast<Divided*>(scratch);
    k.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + divided_bytes());
  }
  k.a = a;
  k.few = few;
  k.negate = a.scale_log2 < 0.f;
  if (k.negate) k.a.scale_log2 = -a.scale_log2;
  // what is hidden is minus infinity before the scale comes in, and has to stay that: a scale of 0 is the least number that there is, 2^-149, which makes 2^-20 of the
  // largest difference of two scores
  if (k.a.scale_log2 == 0.f) k.a.scale_log2 = 0x1p-149f;
  k.group_inv = a.group == 1 ? 0u : (uint32_t)(((1ull << 32) + a.group - 1) / a.group);
  k.stall = take_stall(kFamDecode) ? 1 : 0;
  k.wait_limit = wait_limit_cycles();
  k.y_extent = y_extent;
  k.y_wide = reinterpret_cast<uintptr_t>(a.Y) % 32 == 0;
  // no more items than this: whole ones, and one that is not for every request that has enough rows to be taken
  const long long rows = (long long)a.M * a.group, most = rows / (few + 1);
  const long long items = rows / (2 * kRows) + (most < a.R ? most : a.R);
  if (items * a.hkv + k.sms > 0x7FFFFFFF) return cudaErrorInvalidValue;
  const int ctas = (int)(items * a.hkv) + k.sms;                  // (parts are never more than the SMs)
  auto launch = [&](auto dim, auto mx) {
    constexpr int D = decltype(dim)::value;
    constexpr bool MX = decltype(mx)::value != 0;
    return k.sms > 0 ? launch_shape<D, MX, true>(k, ctas, c, s) : launch_shape<D, MX, false>(k, ctas, c, s);
  };
  if (c.dtype == LQER_MXINT8) return c.head_dim == 128 ? launch(Every<128>{}, Every<1>{}) : launch(Every<64>{}, Every<1>{});
  return c.head_dim == 128 ? launch(Every<128>{}, Every<0>{}) : launch(Every<64>{}, Every<0>{});
}

}  // namespace kv
}  // namespace lqer
