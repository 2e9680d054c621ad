// Attention of a few new tokens of each request over the paged cache, split over its length and joined.
//
// Row i of head h of a request sees key j <= position, and under a window only the last `window` of them and the first `sinks`:
//   y = sum_j p_j v_j / sum_j p_j,  p_j = exp2(s_j - m),  s_j = scale log2(e) q . k_j,  m = the largest s_j so far.
// (m, sum p, sum p v) of two sets of keys join to that of their union: with M = max(m1, m2), each side counts 2^(m_i - M).
// A row sees itself at least, so its sum is 0 only where all of its scores are minus infinity: 0 / 0, NaN, as the formula says.
//
// The rows of the query heads that share a key head, of all of a request's new tokens, go together (a row tile of 8 NT): the keys
// and values are read once for them.  Bound: those bytes.  The products are far from any limit, so they are mma.sync m16n8k16 with the keys (and
// the values' columns) on the 16-row side and the row tile on the 8-column side, which wastes least of it.  Within a dot product the order of the
// elements is free, so a lane takes 16 consecutive bytes of a key (8 of an MXINT8 one), and of four keys' values, and both sides use the order that this gives.
// Each warp has a ring of its own in shared memory, which asynchronous copies fill ahead of it: no barrier between the keys, and what is on its way
// takes no registers.  Of MXINT8 the mantissas become bf16 on their way from there (exact), two at a time.
//
// Work is counted in chunks of 64 keys of a (request, key head, row tile), all in one row; each CTA takes an equal run of them, wherever that begins
// and ends, so lengths may differ as they like.  The four warps take 16 keys of every chunk and join at the end of a run's part; what is not a
// whole row's part goes to the workspace, and a second kernel joins those parts, in the order of the keys.
//
// Measured (GPU time): 64 requests of up to 8191 tokens, 40/8 heads of 128, bf16: 209 us, 6.4 TB/s, what a copy reaches; 24 of up to 4099, 40/40 heads, MXINT8: 168 us,
// 4.1 TB/s, bound by instructions (some 600 for a warp's 16 keys, more than half of them for the mantissas); eight long ones, four drafted tokens, 32/8 heads under a
// window of 4096: 34 us, 3.9 TB/s (of it 5 before the first keys are there and 3 for the joining); 64 requests of up to 8191, 32/8 heads of 64: 110, from MXINT8 111; one of 1021 tokens 9.5 us, of 16000 16, of
// 100000 73: launches and a chain of trips to memory, then the bytes.  Tried: the CTA that brings a row's last part joins them (a launch less, 2 us on the host,
// but 1 to 3 us more on the GPU where parts are many); mantissas' low bytes by multiplication (slower); more or deeper stages (none).
#include "lqer_cache.cuh"

namespace lqer {
namespace kv {

constexpr int kChunk = 64, kWarps = 4, kSplitThreads = 32 * kWarps;
// Requests of up to this many rows of a key head (tokens times heads that share it) are taken here, of more by lqer_attention_tiles.cu.  There a tile of
// keys costs what it costs for 256 rows, and where few requests leave SMs without work a request's keys are divided among them, for some 5 us; here
// the time is shared by all SMs from the start, but grows with the rows, 16 at a time (some 12 ns a key and head, over the SMs).  So long tables, which
// are what the host knows of the lengths, leave less to it.  Both sides measured, here / there, 32/8 heads, us: one request, 64 rows behind 1000: 12 / 16,
// behind 4000: 19 / 17, behind 16000: 44 / 27 (MXINT8 56 / 30); two, 64 rows: 16 / 20, 24 / 24, 54 / 44; four, 32 rows: 16 / 21, 24 / 31, 59 / 74, 64 rows:
// 18 / 21, 31 / 31, 81 / 75; 8, 80 rows behind 2000: 36 / 36; 64, 32 rows: 418 / 318, 80: 200 / 106.  The constants below are where the two sides cross in these
// cases.  Tables that are much wider than the requests are long take the other side sooner than they should: 64 rows behind 1000, tables for 32768: 14.6 instead of 13.0.
constexpr int kLeast = 16;
inline int few_rows(const Attention& p) {
  const long long heads = (long long)(p.R < p.M ? p.R : p.M) * p.hkv, few = 2900 / heads, most = (long long)p.max_pages * p.page > 4096 ? 48 : 96;
  return few < kLeast ? kLeast : (int)(few < most ? few : most);
}
// The most rows of a key head that a request can have; a step may be told of more tokens than the batch has rows.
inline long long most_rows(const Attention& p) { return (long long)(p.max_added < p.M ? p.max_added : p.M) * p.group; }
constexpr int kMinChunks = 2;                // of a CTA's run

// What a CTA leaves for the join: the (request, key head, row tile) that begins in its run and goes on behind it, if any.
struct Span { int row0, rows, head, tile, parts, unused[3]; };   // row0: the request's first row
struct Split {
  Attention a;
  Span* spans;                               // [CTAs]
  float* parts;                              // [CTAs][2][8 NT][D + 2]: part 0 continues a row, part 1 begins one; sums, then m and l
  int few;                                   // requests of more rows than this are left alone
  size_t y_extent, spans_extent, parts_extent;
};

struct Visible { int sink_chunks, first_chunk, chunks; };     // chunks [0, sink_chunks) and [first_chunk, ..), as many as chunks together
__device__ __forceinline__ Visible visible(const Attention& p, int n, int len) {
  Visible v = {0, 0, (len + kChunk - 1) / kChunk};
  if (p.window > 0) {
    v.first_chunk = max(0, len - n - p.window + 1) / kChunk;
    v.sink_chunks = min((min(p.sinks, len) + kChunk - 1) / kChunk, v.first_chunk);
    v.chunks += v.sink_chunks - v.first_chunk;
  }
  return v;
}
__device__ __forceinline__ int row_tiles(const Attention& p, int n, int few, int per) {
  const long long rows = (long long)n * p.group;
  return n > 0 && rows <= few ? (int)((rows + per - 1) / per) : 0;
}
// Where a CTA's run lies: chunks of all requests, chunks a CTA, the request in which the run begins and the chunks before that request.
struct Run { long long total, per, before; int request; };
__device__ __forceinline__ Run find_run(const Split& s, int per_tile, Run* shared) {
  const Attention& p = s.a;
  const StepRequest* reqs = requests_of(p.step);
  __shared__ long long sums[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int q = (p.R + kSplitThreads - 1) / kSplitThreads, from = min(tid * q, p.R), to = min(from + q, p.R);
  auto chunks_of = [&](int r) {
    const int4 w = *reinterpret_cast<const int4*>(reqs + r);
    const int t = row_tiles(p, w.y, s.few, per_tile);
    return t == 0 ? 0LL : (long long)t * p.hkv * visible(p, w.y, w.z).chunks;
  };
  long long mine = 0;
  for (int r = from; r < to; ++r) mine += chunks_of(r);
  long long x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o); if (lane >= o) x += y; }
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) { if (w < warp) before += sums[w]; total += sums[w]; }
  before += x - mine;
  const long long per = max((total + gridDim.x - 1) / gridDim.x, (long long)kMinChunks), u0 = per * blockIdx.x;
  if (tid == 0) *shared = Run{total, per, 0, -1};
  __syncthreads();
  if (u0 >= before && u0 < before + mine) {          // one thread
    int r = from;
    for (;; ++r) {
      const long long c = chunks_of(r);
      if (u0 < before + c) break;
      before += c;
    }
    shared->request = r;
    shared->before = before;
  }
  __syncthreads();
  return *shared;
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t w) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(w));
  return d;
}
__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// CTAs to an SM: more warps hide more of one another's latency, fewer divide the work less and leave a warp its registers.  Heads of 128, three / two to an SM,
// us: 64 requests of up to 8191 tokens, 40/8 heads, bf16 209 / 204, 256 of up to 120, 32/32 heads, 71 / 80, one of 16000 16.4 / 17.6; 24 requests, 40/40 heads,
// MXINT8 169 / 183; 16 rows a tile, 16 requests of 4 tokens 74 / 65.
__host__ __device__ constexpr int ctas_per_sm(int D, int NT) { return D == 64 ? 4 : NT == 1 ? 3 : 2; }
template <bool MX> struct OctOf { using type = uint4; };
template <> struct OctOf<true> { using type = uint2; };
// A warp's ring: stages of 16 keys and their values as they lie in the cache (and their exponents behind each), their 16-byte pieces moved within a row so
// that no two lanes that read together meet on a bank.
template <int D, bool MX, int NT>
struct Ring {
  static constexpr int ROWS = 8 * NT, ROW = MX ? D : 2 * D, PIECES = ROW / 16, SET = 16 * ROW, EXPS = MX ? D : 0, STAGE = 2 * (SET + EXPS);
  static constexpr int STAGES = MX ? 4 : 2, WARP = STAGES * STAGE;
  static constexpr int OUT = ROWS * (D + 4);                          // floats of a warp's sums, then its maxima and sums of weights: over its ring at the end
  static constexpr int CTAS = ctas_per_sm(D, NT);
  static_assert((OUT + 2 * ROWS) * 4 <= WARP, "a warp's sums fit its ring");
  __device__ static __forceinline__ int key_swizzle(int row) { return MX ? (D == 128 ? (row & 3) << 1 : ((row >> 1) & 1) << 1) : (row & 1) << 2 | ((row >> 1) & 3); }
  __device__ static __forceinline__ int value_swizzle(int row) { return MX && D == 64 ? ((row >> 1) & 1) << 1 : ((row >> 1) & 3) << 1; }
  // Where a lane's pieces of a stage go: those of copy i lie 32 / PIECES rows behind those of copy i - 1, and the swizzles repeat after (at most) four.
  static constexpr int COPIES = SET / 512, OFFSETS = COPIES < 4 ? COPIES : 4, STEP = 32 / PIECES;
  static_assert(4 * STEP % 8 == 0 || COPIES <= 4, "the swizzles repeat");
  uint32_t key_to[OFFSETS], value_to[OFFSETS];
  __device__ __forceinline__ explicit Ring(int lane) {
#pragma unroll
    for (int i = 0; i < OFFSETS; ++i) {
      const int r = lane / PIECES + i * STEP, c = lane % PIECES;
      key_to[i] = r * ROW + ((c ^ key_swizzle(r)) << 4);
      value_to[i] = SET + EXPS + r * ROW + ((c ^ value_swizzle(r)) << 4);
    }
  }
  // Sends a stage on its way: 16 rows from `row` on of the [.., D] tensors, which lie one after the other.
  __device__ __forceinline__ void fill(const Attention& p, uint32_t at, size_t row, int lane) const {
    const uint8_t* k = static_cast<const uint8_t*>(p.keys) + row * ROW + 16 * lane;
    const uint8_t* v = static_cast<const uint8_t*>(p.values) + row * ROW + 16 * lane;
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      copy16(at + key_to[i % OFFSETS] + i / OFFSETS * OFFSETS * STEP * ROW, k + 512 * i);
      copy16(at + value_to[i % OFFSETS] + i / OFFSETS * OFFSETS * STEP * ROW, v + 512 * i);
    }
    if (MX && lane < 2 * EXPS / 16) {
      const int which = lane >= EXPS / 16, x = lane - which * (EXPS / 16);
      copy16(at + SET + which * (SET + EXPS) + 16 * x, (which ? p.value_exps : p.key_exps) + row * (D / 16) + 16 * x);
    }
  }
};
// The eight elements of a key's octet j of a lane as pairs; MXINT8: pairs (0, 2), (1, 3), (4, 6), (5, 7), the other way without permutes.
template <int D, bool MX>
__device__ __forceinline__ uint4 key_octet(const uint8_t* keys, int row, int j, int lane, int swizzle, uint2 exps, int shift) {
  const int c = lane & 3;
  if constexpr (MX) {
    const uint2 w = *reinterpret_cast<const uint2*>(keys + row * D + (((2 * j + (c >> 1)) ^ swizzle) << 4) + 8 * (c & 1));
    const MantissaScale s = mantissa_scale(((j & 2 ? exps.y : exps.x) >> (16 * (j & 1) + 8 * (c >> 1))) & 0xFFu, shift);
    return make_uint4(mantissas_bf16x2(w.x, s), mantissas_bf16x2(byte_down(w.x), s), mantissas_bf16x2(w.y, s), mantissas_bf16x2(byte_down(w.y), s));
  } else {
    return *reinterpret_cast<const uint4*>(keys + row * 2 * D + (((4 * j + c) ^ swizzle) << 4));
  }
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ uint32_t word_of(const uint2& v, int i) { return i == 0 ? v.x : v.y; }

template <int D, bool MX, int NT>
__global__ void __launch_bounds__(kSplitThreads, Ring<D, MX, NT>::CTAS) split_kernel(const Split s) {
  using R = Ring<D, MX, NT>;
  constexpr int ROWS = 8 * NT, T = D / 16, H = D / 64;   // T: tiles of 16 columns of the output; H: octets of values a lane takes of a key
  extern __shared__ __align__(128) uint8_t rings[];
  __shared__ Run sm_run;
  const Attention& p = s.a;
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const bool span_fits = LQER_IN_BOUNDS(&p.step->status, blockIdx.x * sizeof(Span), sizeof(Span), s.spans_extent, 65);
  if (tid == 0 && span_fits) s.spans[blockIdx.x].parts = 0;
  if (!step_fits(p, blockIdx.x == 0 && tid == 0)) return;
  const Run run = find_run(s, ROWS, &sm_run);
  long long u = run.per * blockIdx.x;
  const long long end = min(u + run.per, run.total);
  if (u >= end) return;
  uint8_t* const ring = rings + warp * R::WARP;
  const uint32_t ring_at = tc::smem_u32(ring);
  const R copier(lane);
  const StepRequest* reqs = requests_of(p.step);
  const int shift = p.bits - 2;
  int r = run.request, turn = 0;
  long long before = run.before;
  while (u < end) {
    const int4 req = *reinterpret_cast<const int4*>(reqs + r);
    const int row0 = req.x, n = req.y, len = req.z;
    const int tiles = row_tiles(p, n, s.few, ROWS);
    const Visible vis = visible(p, n, len);
    const long long mine = tiles == 0 ? 0 : (long long)tiles * p.hkv * vis.chunks;
    if (u >= before + mine) { before += mine; ++r; continue; }
    const long long local = u - before, which = local / vis.chunks;
    const int h = (int)(which / tiles), tile = (int)(which % tiles), c0 = (int)(local - which * vis.chunks);
    const int c1 = (int)min((long long)vis.chunks, c0 + (end - u));
    const int rows = min(ROWS, n * p.group - tile * ROWS), first_pos = len - n;
    const bool whole = c0 == 0 && c1 == vis.chunks;
    // Where a run holds many short rows, a warp takes a whole one, and nobody waits for anybody (256 requests of up to 120 tokens, 32/32 heads: 103 -> 74 us).
    const bool alone = whole && run.per >= 12 * vis.chunks;
    const long long next = u + (c1 - c0);
    if (alone && (turn++ & 3) != warp) { u = next; continue; }
    // A warp's steps, of 16 keys: of every chunk its own, or of a row of its own all; behind the first tokens' they go on at the window's.
    const int x0 = alone ? 0 : c0, x1 = alone ? 4 * vis.chunks : c1, hop = alone ? 16 : kChunk, mine_at = alone ? 0 : warp * 16;
    const int jump_at = alone ? 4 * vis.sink_chunks : vis.sink_chunks, jump_to = vis.first_chunk * kChunk + mine_at;
    int key0 = x0 < jump_at ? x0 * hop + mine_at : jump_to + (x0 - jump_at) * hop;     // first key of the step
    auto next_key = [&](int key, int x) { return x + 1 == jump_at ? jump_to : key + hop; };
    const int* table = p.tables + (size_t)r * p.max_pages;
    int sent = x0, sent_key = key0, place = 0, sent_place = 0;      // the step that is sent next, its first key and its page
    auto entry_of = [&]() { return sent < x1 && sent_key < len ? table[sent_key >> p.page_shift] : 0; };
    int entry = entry_of();
    auto send = [&]() {
      if (sent < x1 && sent_key < len)
        copier.fill(p, ring_at + sent_place, (((size_t)checked_page(p, entry, r) * p.hkv + h) << p.page_shift) + (sent_key & (p.page - 1)), lane);
      copies_sent();
      sent_place = sent_place == (R::STAGES - 1) * R::STAGE ? 0 : sent_place + R::STAGE;
      sent_key = next_key(sent_key, sent);
      ++sent;
      entry = entry_of();
    };
#pragma unroll
    for (int i = 0; i < R::STAGES - 1; ++i) send();
    // the row tile's queries, in the order in which a lane holds a key
    uint4 q[NT][D / 32];
    int pos[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int x = tile * ROWS + 8 * t + g;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        q[t][j] = make_uint4(0u, 0u, 0u, 0u);
        if (8 * t + g < rows)
          q[t][j] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.Q) + (size_t)(row0 + x / p.group) * p.q_stride +
                                                     (size_t)(h * p.group + x % p.group) * D + 8 * c + 32 * j);
        if (MX) {
          const uint4 w = q[t][j];
          q[t][j] = make_uint4(__byte_perm(w.x, w.y, 0x5410), __byte_perm(w.x, w.y, 0x7632), __byte_perm(w.z, w.w, 0x5410), __byte_perm(w.z, w.w, 0x7632));
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) pos[t][i] = first_pos + (tile * ROWS + 8 * t + 2 * c + i) / p.group;
    }
    const int last_pos = len - 1, seen_from = p.window > 0 ? max(0, first_pos - p.window + 1) : 0;
    float o[NT][T][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int i = 0; i < T; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
      m[t][0] = m[t][1] = -INFINITY;
      l[t][0] = l[t][1] = 0.f;
    }
    for (int x = x0; x < x1 && key0 < len; key0 = next_key(key0, x), ++x) {      // (the last chunk may end before its warps' keys)
      send();
      copies_wait<R::STAGES - 1>();
      __syncwarp();
      const uint8_t* const keys = ring + place;
      const uint8_t* const values = keys + R::SET + R::EXPS;
      float sc[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
      uint2 ke[2] = {make_uint2(0u, 0u), make_uint2(0u, 0u)};
      if constexpr (MX) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint8_t* x = keys + R::SET + (g + 8 * i) * (D / 16);
          if (D == 128) ke[i] = *reinterpret_cast<const uint2*>(x);
          else ke[i].x = *reinterpret_cast<const uint32_t*>(x);
        }
      }
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const uint4 a = key_octet<D, MX>(keys, g, j, lane, R::key_swizzle(g), ke[0], shift);
        const uint4 b = key_octet<D, MX>(keys, g + 8, j, lane, R::key_swizzle(g + 8), ke[1], shift);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma(sc[t], a.x, b.x, a.y, b.y, q[t][j].x, q[t][j].y);
          mma(sc[t], a.z, b.z, a.w, b.w, q[t][j].z, q[t][j].w);
        }
      }
      const bool masked = key0 + 15 > first_pos || (p.window > 0 && key0 <= last_pos - p.window);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[t][i] *= p.scale_log2;
        if (masked) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = key0 + g + 8 * (i >> 1), at = pos[t][i & 1];
            if (key > at || (p.window > 0 && key <= at - p.window && key >= p.sinks)) sc[t][i] = -INFINITY;
          }
        }
      }
      uint32_t pb[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float big[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          big[i] = fmaxf(sc[t][i], sc[t][i + 2]);
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) big[i] = fmaxf(big[i], __shfl_xor_sync(0xFFFFFFFFu, big[i], x));
        }
        if (__any_sync(0xFFFFFFFFu, big[0] > m[t][0] || big[1] > m[t][1])) {
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float to = fmaxf(m[t][i], big[i]);
            f[i] = m[t][i] == to ? 1.f : exp2_fast(m[t][i] - to);
            m[t][i] = to;
            l[t][i] *= f[i];
          }
#pragma unroll
          for (int i = 0; i < T; ++i) {
            o[t][i][0] *= f[0]; o[t][i][1] *= f[1];
            o[t][i][2] *= f[0]; o[t][i][3] *= f[1];
          }
        }
        const float base[2] = {m[t][0] == -INFINITY ? 0.f : m[t][0], m[t][1] == -INFINITY ? 0.f : m[t][1]};
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = exp2_fast(sc[t][i] - base[i & 1]);
        l[t][0] += e[0] + e[2];
        l[t][1] += e[1] + e[3];
        // the weights enter the product rounded to bf16, 2^-8 of each at most, as the values do that they weigh; their sum does not
        pb[t][0] = transposed(round_bf16x2(e[0], e[1]));
        pb[t][1] = transposed(round_bf16x2(e[2], e[3]));
      }
      // of keys 2 c + {0, 1, 8, 9} the values of columns 8 g .. + 7, and of those 64 further on
      using Oct = typename OctOf<MX>::type;
      Oct v[4][H];
      uint2 ve[4] = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 2 * c + (i & 1) + 8 * (i >> 1);
#pragma unroll
        for (int k = 0; k < H; ++k) {
          const int piece = MX ? (g >> 1) + 4 * k : g + 8 * k;
          v[i][k] = *reinterpret_cast<const Oct*>(values + row * R::ROW + ((piece ^ R::value_swizzle(row)) << 4) + (MX ? 8 * (g & 1) : 0));
        }
        if constexpr (MX) {
          const uint8_t* x = values + R::SET + row * (D / 16);
          if (D == 128) ve[i] = *reinterpret_cast<const uint2*>(x);
          else ve[i].x = *reinterpret_cast<const uint32_t*>(x);
        }
        if (masked) {
          // values that no row sees may be anything: 0 times that has to be 0
          const int key = key0 + row;
          if (key >= len || (key < seen_from && key >= p.sinks)) {
#pragma unroll
            for (int k = 0; k < H; ++k) v[i][k] = Oct{};
            ve[i] = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
          }
        }
      }
      MantissaScale vs[2][H];                             // MXINT8: the scales of a pair of keys
      if constexpr (MX) {
        const uint32_t pick = (uint32_t)(g >> 1) * 0x1111u + 0x4400u;
#pragma unroll
        for (int k = 0; k < H; ++k)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            vs[i][k] = mantissa_scales(__byte_perm(word_of(ve[2 * i], k), word_of(ve[2 * i + 1], k), pick) & 0x00FF00FFu, shift);
      }
      // column x (of the eight of octet k) of keys 2 c + 8 i and the next one
      auto pair_of = [&](int i, int k, int x) {
        if constexpr (MX) {
          const uint32_t two = __byte_perm(word_of(v[2 * i][k], x >> 2), word_of(v[2 * i + 1][k], x >> 2), x & 2 ? 0x7632 : 0x5410);
          return mantissas_bf16x2(x & 1 ? byte_down(two) : two, vs[i][k]);
        } else {
          return __byte_perm(word_of(v[2 * i][k], x >> 1), word_of(v[2 * i + 1][k], x >> 1), x & 1 ? 0x7632 : 0x5410);
        }
      };
#pragma unroll
      for (int i = 0; i < T; ++i) {
        // column i of both halves; heads of 64: i and i + 4
        const int hi = D == 128 ? i : i + 4;
        const uint32_t a0 = pair_of(0, 0, i), a1 = pair_of(0, H - 1, hi), a2 = pair_of(1, 0, i), a3 = pair_of(1, H - 1, hi);
#pragma unroll
        for (int t = 0; t < NT; ++t) mma(o[t][i], a0, a1, a2, a3, pb[t][0], pb[t][1]);
      }
      __syncwarp();                                       // the stage may be filled again
      place = place == (R::STAGES - 1) * R::STAGE ? 0 : place + R::STAGE;
    }
    copies_wait<0>();
    __syncwarp();
    u = next;
    if (alone) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) l[t][i] += __shfl_xor_sync(0xFFFFFFFFu, l[t][i], x);
          const int row = 8 * t + 2 * c + i;
          if (row >= rows) continue;
          const float inv = 1.f / l[t][i];
          const int x = tile * ROWS + row;
          const size_t at = ((size_t)(row0 + x / p.group) * p.hq + h * p.group + x % p.group) * D + 8 * g;
          auto two = [&](int k, int half) { return round_bf16x2(o[t][k][i + 2 * half] * inv, o[t][k + 1][i + 2 * half] * inv); };
          uint16_t* const y = static_cast<uint16_t*>(p.Y) + at;
          if (!LQER_IN_BOUNDS(&p.step->status, at * 2, D == 128 ? 144 : 16, s.y_extent, 63)) continue;
          if constexpr (D == 128) {
            *reinterpret_cast<uint4*>(y) = make_uint4(two(0, 0), two(2, 0), two(4, 0), two(6, 0));
            *reinterpret_cast<uint4*>(y + 64) = make_uint4(two(0, 1), two(2, 1), two(4, 1), two(6, 1));
          } else {
            *reinterpret_cast<uint4*>(y) = make_uint4(two(0, 0), two(2, 0), two(0, 1), two(2, 1));
          }
        }
      }
      continue;
    }
    // the four warps' parts
    float* const out = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[t][i] += __shfl_xor_sync(0xFFFFFFFFu, l[t][i], x);
        const int row = 8 * t + 2 * c + i;
        if (g == 0) { out[R::OUT + row] = m[t][i]; out[R::OUT + ROWS + row] = l[t][i]; }
        float* to = out + row * (D + 4) + 8 * g;
        float4* a = reinterpret_cast<float4*>(to);
        if constexpr (D == 128) {
          float4* b = reinterpret_cast<float4*>(to + 64);
          a[0] = make_float4(o[t][0][i], o[t][1][i], o[t][2][i], o[t][3][i]);
          a[1] = make_float4(o[t][4][i], o[t][5][i], o[t][6][i], o[t][7][i]);
          b[0] = make_float4(o[t][0][i + 2], o[t][1][i + 2], o[t][2][i + 2], o[t][3][i + 2]);
          b[1] = make_float4(o[t][4][i + 2], o[t][5][i + 2], o[t][6][i + 2], o[t][7][i + 2]);
        } else {
          a[0] = make_float4(o[t][0][i], o[t][1][i], o[t][2][i], o[t][3][i]);
          a[1] = make_float4(o[t][0][i + 2], o[t][1][i + 2], o[t][2][i + 2], o[t][3][i + 2]);
        }
      }
    }
    __syncthreads();
    float* part = s.parts + (size_t)(2 * blockIdx.x + (c0 > 0 ? 0 : 1)) * ROWS * (D + 2);
    auto of_warp = [&](int w) { return reinterpret_cast<const float*>(rings + w * R::WARP); };
    for (int i = tid; i < rows * (D / 4); i += kSplitThreads) {
      const int row = i / (D / 4), d = 4 * (i % (D / 4));
      float big = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) big = fmaxf(big, of_warp(w)[R::OUT + row]);
      const float base = big == -INFINITY ? 0.f : big;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      float all = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_fast(of_warp(w)[R::OUT + row] - base);
        const float4 x = *reinterpret_cast<const float4*>(of_warp(w) + row * (D + 4) + d);
        sum.x += f * x.x; sum.y += f * x.y; sum.z += f * x.z; sum.w += f * x.w;
        all += f * of_warp(w)[R::OUT + ROWS + row];
      }
      if (whole) {
        const float inv = 1.f / all;
        const int x = tile * ROWS + row;
        const size_t at = ((size_t)(row0 + x / p.group) * p.hq + h * p.group + x % p.group) * D + d;
        if (LQER_IN_BOUNDS(&p.step->status, at * 2, 8, s.y_extent, 60))
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.Y) + at) = make_uint2(round_bf16x2(sum.x * inv, sum.y * inv), round_bf16x2(sum.z * inv, sum.w * inv));
      } else if (LQER_IN_BOUNDS(&p.step->status, (size_t)(part - s.parts) * 4, (size_t)ROWS * (D + 2) * 4, s.parts_extent, 66)) {
        *reinterpret_cast<float4*>(part + row * D + d) = sum;
        if (d == 0) { part[ROWS * D + row] = big; part[ROWS * D + ROWS + row] = all; }
      }
    }
    if (!whole && c0 == 0 && tid == 0 && span_fits) {
      const long long stop = before + (which + 1) * vis.chunks;      // where the row tile ends
      s.spans[blockIdx.x] = Span{row0, rows, h, tile, (int)((stop - 1) / run.per) - (int)blockIdx.x + 1, {}};
    }
    __syncthreads();
  }
}

// Joins the parts of the row tile that begins in a CTA's run.  A thread takes four columns of a row, and where the rows leave threads over, several take a
// share of the parts each, in order; few CTAs with much to do each, for most have nothing.
constexpr int kJoinThreads = 512;
template <int D, int NT>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const Split s) {
  constexpr int ROWS = 8 * NT, QUADS = D / 4;
  __shared__ float4 sums[kJoinThreads];
  __shared__ float2 tops[kJoinThreads];                  // a thread's maximum, and its sum of weights
  const Attention& p = s.a;
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const Span span = s.spans[blockIdx.x];
  if (span.parts == 0) return;
  const int rows = span.rows, items = rows * QUADS, shares = kJoinThreads / items;
  const int tid = threadIdx.x, share = tid / items, item = tid - share * items, row = item / QUADS, d = 4 * (item - row * QUADS);
  const int per = (span.parts + shares - 1) / shares, from = share * per, to = share < shares ? min(from + per, span.parts) : from;
  auto part = [&](int i) { return s.parts + (size_t)(2 * (blockIdx.x + i) + (i == 0 ? 1 : 0)) * ROWS * (D + 2); };
  float big = -INFINITY, all = 0.f;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int at = from; at < to; at += 4) {                // four parts on their way
    float m[4], l[4];
    float4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
      x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (at + i < to) {
        const float* a = part(at + i);
        m[i] = a[ROWS * D + row];
        l[i] = a[ROWS * D + ROWS + row];
        x[i] = *reinterpret_cast<const float4*>(a + row * D + d);
      }
    }
    const float top = fmaxf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), big), base = top == -INFINITY ? 0.f : top;
    const float f0 = exp2_fast(big - base);
    sum.x *= f0; sum.y *= f0; sum.z *= f0; sum.w *= f0;
    all *= f0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = exp2_fast(m[i] - base);
      sum.x += f * x[i].x; sum.y += f * x[i].y; sum.z += f * x[i].z; sum.w += f * x[i].w;
      all += f * l[i];
    }
    big = top;
  }
  if (shares > 1) {
    sums[tid] = sum;
    tops[tid] = make_float2(big, all);
    __syncthreads();
    if (share == 0) {
      for (int k = 1; k < shares; ++k) {
        const float2 t = tops[item + k * items];
        const float4 x = sums[item + k * items];
        const float top = fmaxf(big, t.x), base = top == -INFINITY ? 0.f : top, f = exp2_fast(big - base), g = exp2_fast(t.x - base);
        sum.x = f * sum.x + g * x.x; sum.y = f * sum.y + g * x.y; sum.z = f * sum.z + g * x.z; sum.w = f * sum.w + g * x.w;
        all = f * all + g * t.y;
        big = top;
      }
    }
  }
  if (share > 0) return;
  const float inv = 1.f / all;
  const int x = span.tile * ROWS + row;
  const size_t at = ((size_t)(span.row0 + x / p.group) * p.hq + span.head * p.group + x % p.group) * D + d;
  if (LQER_IN_BOUNDS(&p.step->status, at * 2, 8, s.y_extent, 61))
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.Y) + at) = make_uint2(round_bf16x2(sum.x * inv, sum.y * inv), round_bf16x2(sum.z * inv, sum.w * inv));
}

static int split_grid(const Attention& p, int few, int rows_per, int dim) {
  const long long most_rows = (long long)(few < p.M * (long long)p.group ? few : p.M * (long long)p.group);
  const long long tiles = (most_rows + rows_per - 1) / rows_per, chunks = ((long long)p.max_pages * p.page + kChunk - 1) / kChunk;
  const long long units = (long long)(p.R < p.M ? p.R : p.M) * tiles * p.hkv * chunks;
  const long long most = (long long)sm_count() * ctas_per_sm(dim, rows_per / 8);
  const long long want = (units + kMinChunks - 1) / kMinChunks;
  return (int)(want < most ? want : most);
}
static int rows_per_tile(const Attention& p) { return most_rows(p) <= 8 ? 8 : 16; }

template <int D, bool MX, int NT>
static cudaError_t launch_split(const Split& s, int grid, cudaStream_t stream) {
  constexpr int SMEM = kWarps * Ring<D, MX, NT>::WARP;
  static OncePerDevice once;
  cudaError_t e = once.run([] { return cudaFuncSetAttribute(split_kernel<D, MX, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); });
  if (e != cudaSuccess) return e;
  LaunchScope scope(kFamDecode, stream, 2);
  e = launch_after(split_kernel<D, MX, NT>, dim3(grid), kSplitThreads, SMEM, stream, s);
  if (e != cudaSuccess) return e;
  return launch_after(join_kernel<D, NT>, dim3(grid), kJoinThreads, 0, stream, s);
}

}  // namespace kv

static kv::Attention attention_params(const lqer_kv_cache_t& c, const lqer_page_table_t& t, int M, int hq, int max_added) {
  kv::Attention p = {};
  p.M = M; p.R = t.n_requests; p.max_pages = t.max_pages; p.n_pages = t.n_pages; p.page = t.page;
  p.page_shift = 0;
  while ((1 << p.page_shift) < t.page) ++p.page_shift;
  p.max_added = max_added;
  p.hq = hq; p.hkv = c.kv_heads; p.group = hq / c.kv_heads;
  const size_t elements = (size_t)c.n_pages * c.kv_heads * c.page * c.head_dim;
  p.keys = c.keys; p.values = c.values;
  p.key_exps = static_cast<const uint8_t*>(c.keys) + elements;
  p.value_exps = static_cast<const uint8_t*>(c.values) + elements;
  return p;
}
static size_t spans_bytes() { return ((size_t)4 * sm_count() * sizeof(kv::Span) + 255) & ~(size_t)255; }

// Parts of few rows, and behind them those of tiles.
static size_t few_parts_bytes(const kv::Attention& p, int head_dim) {
  const int rows = kv::rows_per_tile(p);
  return (size_t)kv::split_grid(p, kv::few_rows(p), rows, head_dim) * 2 * rows * (head_dim + 2) * sizeof(float);
}
static size_t few_bytes(const kv::Attention& p, int head_dim) { return (spans_bytes() + few_parts_bytes(p, head_dim) + 255) & ~(size_t)255; }
// A window as long as the tables hides nothing; and positions are below 2^30, so that no difference of one with either overflows.
static void set_window(kv::Attention& p, int window, int sinks) {
  p.window = window < (long long)p.max_pages * p.page ? window : 0;
  p.sinks = p.window == 0 ? 0 : sinks < (1 << 30) ? sinks : 1 << 30;
}
// The most that a call takes, whatever its window.
size_t attention_scratch_bytes(const lqer_kv_cache_t& c, const lqer_page_table_t& t, int M, int hq, int max_added) {
  const kv::Attention p = attention_params(c, t, M, hq, max_added);
  return few_bytes(p, c.head_dim) + (kv::most_rows(p) > kv::few_rows(p) ? kv::tiles_scratch_bytes(p, c.head_dim) : 0);
}
cudaError_t launch_paged_attention(const void* Q, size_t q_stride, int M, int hq, const lqer_kv_cache_t& c, const lqer_page_table_t& t, void* step,
                                   int max_added, int window, int sinks, double scale, int bits, void* Y, void* scratch,
                                   cudaStream_t s) {
  kv::Split k = {};
  k.a = attention_params(c, t, M, hq, max_added);
  k.a.Q = Q; k.a.Y = Y; k.a.q_stride = q_stride;
  k.a.tables = t.tables; k.a.step = static_cast<kv::StepHead*>(step);
  set_window(k.a, window, sinks);
  k.a.scale_log2 = (float)(scale * 1.4426950408889634);
  k.a.bits = bits;
  k.few = kv::few_rows(k.a);
  k.spans = static_cast<kv::Span*>(scratch);
  k.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(scratch) + spans_bytes());
  const size_t whole = (size_t)M * hq * c.head_dim * 2, less = debug_y_shrink();
  k.y_extent = whole > less ? whole - less : 0;
  if (kDebugBounds) { k.spans_extent = spans_bytes(); k.parts_extent = few_parts_bytes(k.a, c.head_dim); }
  if (kv::most_rows(k.a) > k.few) {                                // (then there are items of more than kLeast rows, or a single request's)
    // A single request goes there whatever it turns out to bring; beside one that has to, only those of few rows stay (three prompts of 42 to 97 tokens,
    // 16/4 heads: 18.4 us where the smaller ones stayed, 11.7).
    k.few = t.n_requests == 1 ? 0 : kv::kLeast;
    const cudaError_t e = kv::launch_tiles(k.a, k.few, k.y_extent, c, static_cast<uint8_t*>(scratch) + few_bytes(k.a, c.head_dim), s);
    if (e != cudaSuccess || t.n_requests == 1) return e;
  }
  const bool mx = c.dtype == LQER_MXINT8;
  const int rows = kv::rows_per_tile(k.a), grid = kv::split_grid(k.a, k.few, rows, c.head_dim);
  if (c.head_dim == 128)
    return rows == 8 ? (mx ? kv::launch_split<128, true, 1>(k, grid, s) : kv::launch_split<128, false, 1>(k, grid, s))
                     : (mx ? kv::launch_split<128, true, 2>(k, grid, s) : kv::launch_split<128, false, 2>(k, grid, s));
  return rows == 8 ? (mx ? kv::launch_split<64, true, 1>(k, grid, s) : kv::launch_split<64, false, 1>(k, grid, s))
                   : (mx ? kv::launch_split<64, true, 2>(k, grid, s) : kv::launch_split<64, false, 2>(k, grid, s));
}

}  // namespace lqer
