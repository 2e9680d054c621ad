// Tables of a paged cache from one step of a batch to the next, and the new tokens' keys and values into their slots.
#include "lqer_cache.cuh"

namespace lqer {
namespace kv {

// ---------------------------------------------------------------------------- tables
// The step is a chain of sums over the requests (rows before a request, pages wanted before it, pages given back before it) and then lists that
// are as long as what moves.  One CTA does it: the sums need all requests, everything it reads of what it replaces (lengths, ring) is
// read before, so they may be replaced in place, and a list's entry finds its request by bisection in shared memory.  What bounds it is latency: about a
// dozen trips to L2 and barriers.  Beyond kRowsInside rows, where a thread would have several behind one another, the slots take a launch of their own over
// all SMs.  Measured: 64 requests of a token each 7 us, 512 that bring 13000 rows, end and lose drafts 14 (7000 pages move, two launches).
constexpr int kStepThreads = 1024, kRowsInside = 4096;

struct StepParams {
  const int* lengths;
  const int* added;
  int* tables;
  int* free_pages;
  const long long* ring;
  int* lengths_out;
  long long* ring_out;
  int* slots;
  int* positions;
  StepHead* head;
  int R, M, max_pages, n_pages, page, page_shift, max_added;
  size_t rows_extent;        // bytes of slots, and of positions
};
struct Request {
  int len, next;             // tokens before and after
  int have, want;            // pages before and after
  long long rows;            // rows of the step's tensors
  bool bad;
};
__device__ __forceinline__ Request request_at(const StepParams& p, int r) {
  Request q = {0, 0, 0, 0, 0, false};
  if (r >= p.R) return q;
  const long long cap = (long long)p.max_pages << p.page_shift;
  const int len = p.lengths[r], add = p.added[r];
  q.rows = add > 0 ? min(add, p.M + 1) : 0;
  const long long next = max(0LL, (long long)len + add);
  q.bad = len < 0 || len > cap || next > cap || add > p.max_added;
  q.len = len;
  if (q.bad) return q;
  q.next = (int)next;
  q.have = (len + p.page - 1) >> p.page_shift;
  q.want = (q.next + p.page - 1) >> p.page_shift;
  return q;
}
// Exclusive prefix over the CTA, and the total.
template <class T>
__device__ __forceinline__ T scan(T mine, T* sums, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const T y = __shfl_up_sync(0xFFFFFFFFu, x, o); if (lane >= o) x += y; }
  __syncthreads();
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  T v = sums[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const T y = __shfl_up_sync(0xFFFFFFFFu, v, o); if (lane >= o) v += y; }
  total = __shfl_sync(0xFFFFFFFFu, v, 31);
  const T before = __shfl_sync(0xFFFFFFFFu, v, max(warp - 1, 0));
  return x - mine + (warp > 0 ? before : T(0));
}
// The last of the CTA's ascending entries that is not above `at` (the first one is not): ten steps without a branch, so that several searches run side by side.
__device__ __forceinline__ int last_not_above(const int* first, int at) {
  int lo = 0;
#pragma unroll
  for (int step = kStepThreads / 2; step > 0; step >>= 1) lo += first[lo + step] <= at ? step : 0;
  return lo;
}
// Slot and position of row i of request r; fail: told of a table entry that is no page.
template <class Fail>
__device__ __forceinline__ void slot_of(const StepParams& p, int r, int i, int n, int len, Fail fail, int& slot, int& pos) {
  slot = pos = -1;
  if (i >= n) return;
  const int at = len - n + i, id = p.tables[(size_t)r * p.max_pages + (at >> p.page_shift)];
  if ((unsigned)id < (unsigned)p.n_pages) {
    slot = (id << p.page_shift) + (at & (p.page - 1));
    pos = at;
  } else {
    fail(LQER_ERR_BOUNDS);
  }
}
// The checked build's view of the step's stores: entry i of a list of n, and of the rows' slots and positions.
__device__ __forceinline__ bool entry_fits(DeviceStatus* st, size_t i, size_t n, int site) { return LQER_IN_BOUNDS(st, i * sizeof(int), sizeof(int), n * sizeof(int), site); }
__device__ __forceinline__ bool row_fits(const StepParams& p, DeviceStatus* st, int row) {
  return LQER_IN_BOUNDS(st, (size_t)row * sizeof(int), sizeof(int), p.rows_extent, 11);
}
// Place i of a ring of n entries from `start` on (i below n).
__device__ __forceinline__ int around(int start, int i, int n) { return i < n - start ? start + i : i - (n - start); }
constexpr int kBatch = 4;    // list entries that a thread has on their way
__global__ void __launch_bounds__(kStepThreads) step_kernel(const StepParams p, const int rows_inside) {
  __shared__ int first[kStepThreads], from[kStepThreads], row0s[kStepThreads], ns[kStepThreads], lens[kStepThreads];
  __shared__ int sums32[32];
  __shared__ long long sums64[32];
  __shared__ int taken;
  __shared__ DeviceStatus status;
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const int tid = threadIdx.x;
  const long long head = p.ring[0], tail = p.ring[1];
  if (tid == 0) { taken = 0; status = DeviceStatus{LQER_OK, 0, 0, 0}; }
  __syncthreads();
  auto fail = [&](int code) { report_error(&status, code, 10); };
  const Request q0 = request_at(p, tid);
  auto request = [&](int base) { return base == 0 ? q0 : request_at(p, base + tid); };
  // pages that come back
  int given = 0, total = 0;
  for (int base = 0; base < p.R; base += kStepThreads) {
    const Request q = request(base);
    given += max(q.have - q.want, 0);
  }
  scan(given, sums32, total);
  const int all_given = total;
  const bool ring_ok = head >= 0 && tail >= head && tail < (1LL << 62) && tail - head + all_given <= p.n_pages;     // (so that no sum overflows)
  if (!ring_ok && tid == 0) fail(LQER_ERR_BOUNDS);
  if (ring_ok && all_given > 0) {
    int before = 0;
    for (int base = 0; base < p.R; base += kStepThreads) {
      const Request q = request(base);
      first[tid] = scan(max(q.have - q.want, 0), sums32, total);
      from[tid] = q.want;
      __syncthreads();
      const int start = (int)((tail + before) % p.n_pages);        // (no more than n_pages come back: the ring has room for them)
      for (int at = tid; at < total; at += kBatch * kStepThreads) {
        int id[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int i = at + u * kStepThreads, k = last_not_above(first, i);
          if (i < total) id[u] = p.tables[(size_t)(base + k) * p.max_pages + from[k] + i - first[k]];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int i = at + u * kStepThreads;
          if (i >= total) continue;
          const int at = around(start, i, p.n_pages);
          if (entry_fits(&status, at, p.n_pages, 12)) p.free_pages[at] = id[u];
          if ((unsigned)id[u] >= (unsigned)p.n_pages) fail(LQER_ERR_BOUNDS);
        }
      }
      before += total;
      __syncthreads();
    }
  }
  __syncthreads();
  // rows, and pages that are wanted; those that came back may go out again
  const long long avail = ring_ok ? tail + all_given - head : 0;
  long long rows_before = 0;
  int wanted_before = 0;
  uint8_t* const plan = reinterpret_cast<uint8_t*>(p.head);
  StepRequest* out = reinterpret_cast<StepRequest*>(plan + kStepHeadBytes);
  int* const lengths = reinterpret_cast<int*>(plan + step_lengths_at(p.R));
  for (int base = 0; base < p.R; base += kStepThreads) {
    const int r = base + tid;
    const Request q = request(base);
    long long all_rows;
    const long long row0 = rows_before + scan(q.rows, sums64, all_rows);
    const bool fits = row0 + q.rows <= p.M || q.rows == 0;
    bool ok = !q.bad && fits && (ring_ok || q.have == q.want);
    if (!ok && r < p.R) fail(LQER_ERR_BOUNDS);
    const int want = ok ? max(q.want - q.have, 0) : 0;
    const int at = wanted_before + scan(want, sums32, total);
    if (want > 0 && at + want > avail) {
      ok = false;
      fail(LQER_ERR_BUFFER_TOO_SMALL);
    }
    if (want > 0 && ok) atomicMax(&taken, at + want);
    first[tid] = at - wanted_before;
    from[tid] = ok ? q.have : -1;
    row0s[tid] = (int)min(row0, (long long)p.M);
    ns[tid] = ok ? (int)q.rows : 0;
    lens[tid] = ok ? q.next : q.bad ? 0 : q.len;
    if (r < p.R) {
      if (entry_fits(&status, r, p.R, 13)) {
        out[r] = StepRequest{row0s[tid], ns[tid], lens[tid], 0};
        p.lengths_out[r] = lengths[r] = ok ? q.next : q.len;
      }
    }
    __syncthreads();
    // (whoever is not refused takes pages that are there: fewer than n_pages before them)
    const int start = ring_ok ? (int)((head + min((long long)wanted_before, avail)) % p.n_pages) : 0;
    for (int at = tid; at < total; at += kBatch * kStepThreads) {
      int id[kBatch], entry[kBatch], of[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int i = at + u * kStepThreads, k = last_not_above(first, i);
        of[u] = i < total && from[k] >= 0 ? base + k : -1;
        entry[u] = from[k] + i - first[k];
        if (of[u] >= 0) id[u] = p.free_pages[around(start, i, p.n_pages)];
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (of[u] >= 0 && entry_fits(&status, (size_t)of[u] * p.max_pages + entry[u], (size_t)p.R * p.max_pages, 14))
          p.tables[(size_t)of[u] * p.max_pages + entry[u]] = id[u];
    }
    wanted_before += total;
    __syncthreads();
    if (rows_inside) {
      const int lo = (int)min(rows_before, (long long)p.M), hi = (int)min(rows_before + all_rows, (long long)p.M);
      for (int at = lo + tid; at < hi; at += kBatch * kStepThreads) {
        int slot[kBatch], pos[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int row = at + u * kStepThreads, k = last_not_above(row0s, row);
          if (row < hi) slot_of(p, base + k, row - row0s[k], ns[k], lens[k], fail, slot[u], pos[u]);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int row = at + u * kStepThreads;
          if (row < hi && row_fits(p, &status, row)) { p.slots[row] = slot[u]; p.positions[row] = pos[u]; }
        }
      }
      __syncthreads();
    }
    rows_before += all_rows;
  }
  const int rows = (int)min(rows_before, (long long)p.M);
  if (rows_inside)
    for (int row = rows + tid; row < p.M; row += kStepThreads)
      if (row_fits(p, &status, row)) p.slots[row] = p.positions[row] = -1;
  if (kDebugBounds) __syncthreads();
  if (tid == 0) {
    long long* const ring = reinterpret_cast<long long*>(plan + step_ring_at(p.R));
    p.ring_out[0] = ring[0] = head + taken;
    p.ring_out[1] = ring[1] = ring_ok ? tail + all_given : tail;
    StepHead h = {};
    h.magic = kStepMagic;
    h.R = p.R; h.M = p.M; h.page = p.page; h.max_pages = p.max_pages; h.n_pages = p.n_pages; h.max_added = p.max_added;
    h.status = status;
    *p.head = h;
  }
}
// Slots of many rows: a thread a row, its request by bisection in the plan.
__global__ void __launch_bounds__(256) rows_kernel(const StepParams p) {
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const StepRequest* reqs = requests_of(p.head);
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row >= p.M) return;
  int lo = 0, hi = p.R;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (reqs[mid].row0 <= row) lo = mid; else hi = mid;
  }
  const StepRequest q = reqs[lo];
  int slot, pos;
  slot_of(p, lo, row - q.row0, q.n, q.len, [&](int code) { report_error(&p.head->status, code, 10, lo, row); }, slot, pos);
  if (row_fits(p, &p.head->status, row)) { p.slots[row] = slot; p.positions[row] = pos; }
}

// ---------------------------------------------------------------------------- appending
// A thread takes 16 consecutive elements of a head, of keys or of values: 32 or 64 bytes in, 32 (bf16) or 16 and an exponent byte
// (MXINT8) out, in one pass.  Bound: memory from some hundred rows on, a launch below: 64 rows of 8 heads of 128 1.8 us, 4096 in a row 5.1 (4.6 TB/s, much of it
// L2's), in any order 6.7, to MXINT8 6.6, from fp32 8.0 and 7.5.
struct AppendParams {
  const void* K;
  const void* V;
  size_t k_stride, v_stride;
  const int* slots;
  void* keys;
  void* values;
  int M, hkv, page, page_shift, blocks;      // blocks: of 16 elements of a head
  size_t exps;                               // MXINT8: bytes of mantissas in front of the exponents
  long long capacity;
  int bits, emin, emax;
};
template <bool XB, bool MX>
__global__ void __launch_bounds__(256) append_kernel(const AppendParams p) {
  tc::pdl_launch_dependents();
  tc::pdl_wait();
  const int per_row = 2 * p.hkv * p.blocks;
  const size_t items = (size_t)p.M * per_row;
  for (size_t i = blockIdx.x * (size_t)256 + threadIdx.x; i < items; i += (size_t)gridDim.x * 256) {
    const int row = (int)(i / per_row), rest = (int)(i - (size_t)row * per_row);
    const int which = rest >= p.hkv * p.blocks, at = rest - which * p.hkv * p.blocks, h = at / p.blocks, b = at - h * p.blocks;
    const int slot = p.slots[row];
    if (slot < 0 || slot >= p.capacity) continue;
    const size_t x = (size_t)row * (which ? p.v_stride : p.k_stride) + (size_t)at * 16;
    const size_t y = ((((size_t)(slot >> p.page_shift) * p.hkv + h) << p.page_shift) + (slot & (p.page - 1))) * (size_t)p.blocks + b;   // in blocks
    const void* X = which ? p.V : p.K;
    void* C = which ? p.values : p.keys;
    uint4 raw[4];
    if (XB) {
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(X) + x);
      raw[0] = src[0];
      raw[1] = src[1];
    } else {
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const float*>(X) + x);
#pragma unroll
      for (int k = 0; k < 4; ++k) raw[k] = src[k];
    }
    if (XB && !MX) {
      uint4* dst = static_cast<uint4*>(C) + 2 * y;
      dst[0] = raw[0];
      dst[1] = raw[1];
      continue;
    }
    float v[16];
    const uint32_t* w = reinterpret_cast<const uint32_t*>(raw);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (XB) v[k] = __uint_as_float(k % 2 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
      else v[k] = __uint_as_float(w[k]);
    }
    if (MX) {
      int e;
      uint4 m, bf0, bf1;
      quantize_block16(v, quant_consts(p.bits, p.emin, p.emax), e, m, bf0, bf1);
      static_cast<uint4*>(C)[y] = m;
      static_cast<uint8_t*>(C)[p.exps + y] = (uint8_t)(e + 127);
    } else {
      uint4* dst = static_cast<uint4*>(C) + 2 * y;
      dst[0] = make_uint4(round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]), round_bf16x2(v[4], v[5]), round_bf16x2(v[6], v[7]));
      dst[1] = make_uint4(round_bf16x2(v[8], v[9]), round_bf16x2(v[10], v[11]), round_bf16x2(v[12], v[13]), round_bf16x2(v[14], v[15]));
    }
  }
}

}  // namespace kv

static int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

size_t cache_step_bytes(int R) { return kv::step_bytes(R); }
cudaError_t launch_cache_step(const lqer_page_table_t& t, const int* lengths, const int* added, const long long* ring, int M, int max_added,
                              int* lengths_out, long long* ring_out, int* slots, int* positions, void* step, cudaStream_t s) {
  kv::StepParams p = {lengths, added, t.tables, t.free_pages, ring, lengths_out, ring_out, slots, positions, static_cast<kv::StepHead*>(step),
                      t.n_requests, M, t.max_pages, t.n_pages, t.page, log2_of(t.page), max_added, 0};
  const size_t rows = (size_t)M * sizeof(int), less = debug_y_shrink();
  p.rows_extent = rows > less ? rows - less : 0;
  const bool inside = M <= kv::kRowsInside;
  LaunchScope scope(kFamDecode, s, inside ? 1 : 2);
  cudaError_t e = kv::launch_after(kv::step_kernel, dim3(1), kv::kStepThreads, 0, s, p, inside ? 1 : 0);
  if (e != cudaSuccess || inside) return e;
  return kv::launch_after(kv::rows_kernel, dim3((M + 255) / 256), 256, 0, s, p);
}
cudaError_t launch_append_kv(const void* K, const void* V, int x_type, size_t k_stride, size_t v_stride, int M, const int* slots,
                             const lqer_kv_cache_t& c, int bits, int emin, int emax, cudaStream_t s) {
  kv::AppendParams p = {};
  p.K = K; p.V = V; p.k_stride = k_stride; p.v_stride = v_stride; p.slots = slots;
  p.keys = c.keys; p.values = c.values;
  p.M = M; p.hkv = c.kv_heads; p.page = c.page; p.page_shift = log2_of(c.page); p.blocks = c.head_dim / 16;
  p.exps = (size_t)c.n_pages * c.kv_heads * c.page * c.head_dim;
  p.capacity = (long long)c.n_pages * c.page;
  p.bits = bits; p.emin = emin; p.emax = emax;
  const size_t items = (size_t)M * 2 * c.kv_heads * p.blocks, ctas = (items + 255) / 256, most = (size_t)sm_count() * 64;
  const dim3 grid((unsigned)(ctas < most ? ctas : most));
  LaunchScope scope(kFamQuantize, s);
  const bool xb = x_type == kXBF16, mx = c.dtype == LQER_MXINT8;
  return xb ? (mx ? kv::launch_after(kv::append_kernel<true, true>, grid, 256, 0, s, p) : kv::launch_after(kv::append_kernel<true, false>, grid, 256, 0, s, p))
            : (mx ? kv::launch_after(kv::append_kernel<false, true>, grid, 256, 0, s, p) : kv::launch_after(kv::append_kernel<false, false>, grid, 256, 0, s, p));
}

}  // namespace lqer
