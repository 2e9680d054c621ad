// Host side of the C ABI, continued: argument checks of the cache of keys and values and of the attention over it.
#include "lqer_common.cuh"

using namespace lqer;

namespace {

bool misaligned(const void* p, size_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
bool page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128; }
lqer_status_t of(cudaError_t e) { return e == cudaSuccess ? LQER_OK : LQER_ERR_CUDA; }

lqer_status_t cache_shape(const lqer_kv_cache_t* c) {
  if (c == nullptr) return LQER_ERR_NULL;
  if (c->dtype != LQER_BF16 && c->dtype != LQER_MXINT8) return LQER_ERR_CONFIG;
  if (!page_ok(c->page) || (c->head_dim != 64 && c->head_dim != 128) || c->kv_heads < 1 || c->kv_heads > kKvMaxHeads) return LQER_ERR_SHAPE;
  if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFF / c->page) return LQER_ERR_SHAPE;
  return LQER_OK;
}
lqer_status_t cache_ready(const lqer_kv_cache_t* c) {
  lqer_status_t st = cache_shape(c);
  if (st != LQER_OK) return st;
  if (c->keys == nullptr || c->values == nullptr) return LQER_ERR_NULL;
  if (misaligned(c->keys) || misaligned(c->values)) return LQER_ERR_ALIGN;
  return c->keys == c->values ? LQER_ERR_CONFIG : LQER_OK;
}
lqer_status_t table_shape(const lqer_page_table_t* t) {
  if (t == nullptr) return LQER_ERR_NULL;
  if (t->n_requests < 1 || t->n_requests > kKvMaxRequests || !page_ok(t->page) || t->max_pages < 1 || t->n_pages < 1) return LQER_ERR_SHAPE;
  if (t->max_pages > (1 << 30) / t->page || (long long)t->n_requests * t->max_pages > 0x7FFFFFFFLL || t->n_pages > 0x7FFFFFFF / t->page) return LQER_ERR_SHAPE;
  return LQER_OK;
}
lqer_status_t table_ready(const lqer_page_table_t* t, bool all) {
  lqer_status_t st = table_shape(t);
  if (st != LQER_OK) return st;
  if (t->tables == nullptr || (all && t->free_pages == nullptr)) return LQER_ERR_NULL;
  return misaligned(t->tables, 4) || misaligned(t->free_pages, 4) ? LQER_ERR_ALIGN : LQER_OK;
}
bool rows_ok(int M) { return M > 0 && M <= (1 << 24); }
lqer_status_t activation_format(const lqer_config_t* cfg, lqer_config_t* out) {
  if (cfg == nullptr) return lqer_default_config(out);
  *out = *cfg;
  return check_config(cfg);
}
lqer_status_t attention_shape(int M, int q_heads, const lqer_kv_cache_t* c, const lqer_page_table_t* t, int max_added) {
  if (!rows_ok(M) || max_added < 1 || q_heads < 1 || q_heads > kKvMaxHeads || q_heads % c->kv_heads != 0) return LQER_ERR_SHAPE;
  if ((long long)M * q_heads > 0x7FFFFFFF) return LQER_ERR_SHAPE;
  return t->page == c->page && t->n_pages == c->n_pages ? LQER_OK : LQER_ERR_SHAPE;
}

}  // namespace

extern "C" {

lqer_status_t lqer_kv_cache_bytes(const lqer_kv_cache_t* cache, size_t* bytes) {
  if (bytes == nullptr) return LQER_ERR_NULL;
  lqer_status_t st = cache_shape(cache);
  if (st != LQER_OK) return st;
  const size_t n = (size_t)cache->n_pages * cache->kv_heads * cache->page * cache->head_dim;
  *bytes = cache->dtype == LQER_MXINT8 ? n + n / 16 : 2 * n;
  return LQER_OK;
}

lqer_status_t lqer_cache_step_bytes(int n_requests, size_t* bytes) {
  if (bytes == nullptr) return LQER_ERR_NULL;
  if (n_requests < 1 || n_requests > kKvMaxRequests) return LQER_ERR_SHAPE;
  *bytes = cache_step_bytes(n_requests);
  return LQER_OK;
}

lqer_status_t lqer_cache_step(const lqer_page_table_t* table, const int* lengths, const int* added, const long long* ring, int M, int max_added,
                              int* lengths_out, long long* ring_out, int* slots, int* positions, void* step, size_t step_bytes, void* stream) {
  const bool empty = M == 0 && slots == nullptr && positions == nullptr;       // a step without rows has no lists of them
  if (lengths == nullptr || added == nullptr || ring == nullptr || lengths_out == nullptr || ring_out == nullptr || step == nullptr ||
      (!empty && (slots == nullptr || positions == nullptr)))
    return LQER_ERR_NULL;
  lqer_status_t st = table_ready(table, true);
  if (st != LQER_OK) return st;
  if ((!empty && !rows_ok(M)) || max_added < 1) return LQER_ERR_SHAPE;
  if (misaligned(lengths, 4) || misaligned(added, 4) || misaligned(ring, 8) || misaligned(lengths_out, 4) || misaligned(ring_out, 8) || misaligned(slots, 4) ||
      misaligned(positions, 4) || misaligned(step, 256))
    return LQER_ERR_ALIGN;
  if (step_bytes < cache_step_bytes(table->n_requests)) return LQER_ERR_BUFFER_TOO_SMALL;
  if (lengths_out == added || (!empty && slots == positions) || table->tables == table->free_pages) return LQER_ERR_CONFIG;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_cache_step(*table, lengths, added, ring, M, max_added, lengths_out, ring_out, slots, positions, step, static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_append_kv(const void* K, const void* V, lqer_dtype_t x_dtype, long long k_stride, long long v_stride, int M, const int* slots,
                             const lqer_kv_cache_t* cache, const lqer_config_t* cfg, void* stream) {
  if (K == nullptr || V == nullptr || slots == nullptr) return LQER_ERR_NULL;
  lqer_status_t st = cache_ready(cache);
  if (st != LQER_OK) return st;
  lqer_config_t f;
  if ((st = activation_format(cfg, &f)) != LQER_OK) return st;
  if (x_dtype != LQER_F32 && x_dtype != LQER_BF16) return LQER_ERR_CONFIG;
  const long long width = (long long)cache->kv_heads * cache->head_dim;
  if (!rows_ok(M) || k_stride < width || v_stride < width || k_stride % 8 != 0 || v_stride % 8 != 0 || k_stride > (1LL << 32) || v_stride > (1LL << 32))
    return LQER_ERR_SHAPE;
  if (misaligned(K) || misaligned(V) || misaligned(slots, 4)) return LQER_ERR_ALIGN;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_append_kv(K, V, x_dtype, (size_t)k_stride, (size_t)v_stride, M, slots, *cache, f.a_bits, f.exp_min, f.exp_max,
                             static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_attention_workspace_bytes(int M, int q_heads, const lqer_kv_cache_t* cache, const lqer_page_table_t* table, int max_added,
                                             size_t* bytes) {
  if (bytes == nullptr) return LQER_ERR_NULL;
  lqer_status_t st = cache_shape(cache);
  if (st == LQER_OK) st = table_shape(table);
  if (st == LQER_OK) st = attention_shape(M, q_heads, cache, table, max_added);
  if (st == LQER_OK) *bytes = attention_scratch_bytes(*cache, *table, M, q_heads, max_added);
  return st;
}

lqer_status_t lqer_paged_attention(const void* Q, long long q_stride, int M, int q_heads, const lqer_kv_cache_t* cache, const lqer_page_table_t* table,
                                   void* step, int max_added, int window, int sinks, double scale, const lqer_config_t* cfg, void* Y, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  if (Q == nullptr || Y == nullptr || step == nullptr) return LQER_ERR_NULL;
  lqer_status_t st = cache_ready(cache);
  if (st == LQER_OK) st = table_ready(table, false);
  if (st != LQER_OK) return st;
  lqer_config_t f;
  if ((st = activation_format(cfg, &f)) != LQER_OK) return st;
  if (!(scale < 1e30 && scale > -1e30)) return LQER_ERR_CONFIG;
  if ((st = attention_shape(M, q_heads, cache, table, max_added)) != LQER_OK) return st;
  if (q_stride < (long long)q_heads * cache->head_dim || q_stride % 8 != 0 || q_stride > (1LL << 32) || window < 0 || sinks < 0) return LQER_ERR_SHAPE;
  if (misaligned(Q) || misaligned(Y) || misaligned(step, 256) || misaligned(workspace, 256)) return LQER_ERR_ALIGN;
  if (Y == Q || Y == cache->keys || Y == cache->values) return LQER_ERR_CONFIG;
  if (workspace == nullptr) return LQER_ERR_NULL;
  if (workspace_bytes < attention_scratch_bytes(*cache, *table, M, q_heads, max_added)) return LQER_ERR_BUFFER_TOO_SMALL;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_paged_attention(Q, (size_t)q_stride, M, q_heads, *cache, *table, step, max_added, window, sinks, scale, f.a_bits, Y, workspace,
                                   static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
