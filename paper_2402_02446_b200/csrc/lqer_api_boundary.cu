// Host side of the C ABI, continued: argument checks of what stands between the layers (norm, gated activation, adapters).
#include "lqer_common.cuh"

using namespace lqer;

namespace {

bool misaligned(const void* p, size_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
bool plain_type(lqer_dtype_t t) { return t == LQER_F32 || t == LQER_BF16; }
bool any_type(lqer_dtype_t t) { return plain_type(t) || t == LQER_MXINT8; }
bool rows_ok(int M) { return M > 0 && M <= (1 << 24); }
// kX* and kY* number the types as lqer_dtype_t does
static_assert(kXF32 == LQER_F32 && kXBF16 == LQER_BF16 && kXMXINT8 == LQER_MXINT8 && kYF32 == LQER_F32 && kYBF16 == LQER_BF16 && kYMXINT8 == LQER_MXINT8, "types");

// The activation format of *cfg, or the default one.
lqer_status_t activation_format(const lqer_config_t* cfg, lqer_config_t* out) {
  if (cfg == nullptr) return lqer_default_config(out);
  *out = *cfg;
  return check_config(cfg);
}
lqer_status_t pool_shape(const lqer_adapter_pool_t* pool) {
  if (pool == nullptr) return LQER_ERR_NULL;
  if (pool->K <= 0 || pool->K % 16 != 0 || pool->K > (1 << 20) || pool->N <= 0 || pool->N % 8 != 0 || pool->N > (1 << 22)) return LQER_ERR_SHAPE;
  if (pool->max_rank < 1 || pool->max_rank > kAdapterMaxRank || pool->n_slots < 1 || pool->n_slots > kAdapterMaxSlots) return LQER_ERR_SHAPE;
  return LQER_OK;
}
lqer_status_t pool_ready(const lqer_adapter_pool_t* pool) {
  lqer_status_t st = pool_shape(pool);
  if (st != LQER_OK) return st;
  if (pool->data == nullptr) return LQER_ERR_NULL;
  return misaligned(pool->data, 256) ? LQER_ERR_ALIGN : LQER_OK;
}
size_t pool_size(const lqer_adapter_pool_t* pool) { return (size_t)pool->n_slots * adapter_slot_bytes(pool->K, pool->N, pool->max_rank); }
lqer_status_t of(cudaError_t e) { return e == cudaSuccess ? LQER_OK : LQER_ERR_CUDA; }

}  // namespace

extern "C" {

lqer_status_t lqer_add_rms_norm(const void* X, lqer_dtype_t x_dtype, const void* residual, void* residual_out, lqer_dtype_t r_dtype,
                                const void* weight, lqer_dtype_t w_dtype, double eps, int M, int K, const lqer_config_t* cfg,
                                void* Y, lqer_dtype_t y_dtype, void* stream) {
  if (X == nullptr || weight == nullptr || Y == nullptr) return LQER_ERR_NULL;
  lqer_config_t f;
  lqer_status_t st = activation_format(cfg, &f);
  if (st != LQER_OK) return st;
  if (!plain_type(x_dtype) || !plain_type(r_dtype) || !plain_type(w_dtype) || !any_type(y_dtype) || !(eps >= 0.0)) return LQER_ERR_CONFIG;
  if (!rows_ok(M) || K <= 0 || K > (1 << 20) || K % (y_dtype == LQER_MXINT8 ? 16 : 8) != 0) return LQER_ERR_SHAPE;
  if (misaligned(X) || misaligned(weight) || misaligned(Y) || misaligned(residual) || misaligned(residual_out)) return LQER_ERR_ALIGN;
  if ((residual_out == X && r_dtype != x_dtype) || Y == X || Y == residual || Y == residual_out) return LQER_ERR_CONFIG;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_add_rms_norm(X, x_dtype, residual, residual_out, r_dtype, weight, w_dtype, eps, M, K, f.a_bits, f.exp_min, f.exp_max, Y,
                                y_dtype, static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_gated_activation(const void* gate, const void* up, lqer_dtype_t x_dtype, long long row_stride, int M, int N,
                                    lqer_activation_t act, const lqer_config_t* cfg, void* Y, lqer_dtype_t y_dtype, void* stream) {
  if (gate == nullptr || up == nullptr || Y == nullptr) return LQER_ERR_NULL;
  lqer_config_t f;
  lqer_status_t st = activation_format(cfg, &f);
  if (st != LQER_OK) return st;
  if (!plain_type(x_dtype) || !any_type(y_dtype) || (act != LQER_SILU && act != LQER_GELU_TANH)) return LQER_ERR_CONFIG;
  if (!rows_ok(M) || N <= 0 || N > (1 << 22) || N % (y_dtype == LQER_MXINT8 ? 16 : 8) != 0) return LQER_ERR_SHAPE;
  if (row_stride < N || row_stride % 8 != 0 || row_stride > (1LL << 32)) return LQER_ERR_SHAPE;
  if (misaligned(gate) || misaligned(up) || misaligned(Y)) return LQER_ERR_ALIGN;
  if (Y == gate || Y == up) return LQER_ERR_CONFIG;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_gated_activation(gate, up, x_dtype, (size_t)row_stride, M, N, act, f.a_bits, f.exp_min, f.exp_max, Y, y_dtype,
                                    static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_dequantize_activations(const void* Xq, int M, int K, const lqer_config_t* cfg, void* Y, lqer_dtype_t y_dtype,
                                          void* stream) {
  if (Xq == nullptr || Y == nullptr) return LQER_ERR_NULL;
  lqer_config_t f;
  lqer_status_t st = activation_format(cfg, &f);
  if (st != LQER_OK) return st;
  if (!plain_type(y_dtype)) return LQER_ERR_CONFIG;
  if (!rows_ok(M) || K <= 0 || K % 16 != 0 || K > (1 << 20)) return LQER_ERR_SHAPE;
  if (misaligned(Xq) || misaligned(Y)) return LQER_ERR_ALIGN;
  if (Y == Xq) return LQER_ERR_CONFIG;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_dequantize(Xq, M, K, f.a_bits, f.exp_min, f.exp_max, Y, y_dtype, static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_adapter_pool_bytes(const lqer_adapter_pool_t* pool, size_t* bytes) {
  if (bytes == nullptr) return LQER_ERR_NULL;
  lqer_status_t st = pool_shape(pool);
  if (st == LQER_OK) *bytes = pool_size(pool);
  return st;
}

lqer_status_t lqer_adapter_pool_init(const lqer_adapter_pool_t* pool, size_t pool_bytes, void* stream) {
  lqer_status_t st = pool_ready(pool);
  if (st != LQER_OK) return st;
  if (pool_bytes < pool_size(pool)) return LQER_ERR_BUFFER_TOO_SMALL;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_adapter_pool_init(pool->data, pool->K, pool->N, pool->max_rank, pool->n_slots, static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_adapter_load(const lqer_adapter_pool_t* pool, int slot, const void* A, const void* B, lqer_dtype_t dtype, int rank,
                                float scale, void* stream) {
  lqer_status_t st = pool_ready(pool);
  if (st != LQER_OK) return st;
  if (!plain_type(dtype)) return LQER_ERR_CONFIG;
  if (slot < 0 || slot >= pool->n_slots || rank < 0 || rank > pool->max_rank) return LQER_ERR_SHAPE;
  if (rank > 0 && (A == nullptr || B == nullptr)) return LQER_ERR_NULL;
  if (rank > 0 && (misaligned(A) || misaligned(B))) return LQER_ERR_ALIGN;
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_adapter_load(pool->data, pool->K, pool->N, pool->max_rank, slot, A, B, dtype == LQER_BF16, rank, scale,
                                static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_adapter_plan_bytes(int M, int n_slots, size_t* bytes) {
  if (bytes == nullptr) return LQER_ERR_NULL;
  if (!rows_ok(M) || n_slots < 1 || n_slots > kAdapterMaxSlots) return LQER_ERR_SHAPE;
  *bytes = adapter_plan_bytes(M, n_slots);
  return LQER_OK;
}

lqer_status_t lqer_adapter_plan(const int* slots, int M, int n_slots, void* plan, size_t plan_bytes, void* stream) {
  if (slots == nullptr || plan == nullptr) return LQER_ERR_NULL;
  if (!rows_ok(M) || n_slots < 1 || n_slots > kAdapterMaxSlots) return LQER_ERR_SHAPE;
  if (misaligned(slots, 4) || misaligned(plan, 256)) return LQER_ERR_ALIGN;
  if (plan_bytes < adapter_plan_bytes(M, n_slots)) return LQER_ERR_BUFFER_TOO_SMALL;
  lqer_status_t st = check_arch();
  if (st != LQER_OK) return st;
  return of(launch_adapter_plan(slots, M, n_slots, plan, static_cast<cudaStream_t>(stream)));
}

lqer_status_t lqer_adapters_workspace_bytes(int M, const lqer_adapter_pool_t* pool, int plan_slots, size_t* bytes) {
  if (bytes == nullptr) return LQER_ERR_NULL;
  lqer_status_t st = pool_shape(pool);
  if (st != LQER_OK) return st;
  if (!rows_ok(M) || plan_slots < 1 || plan_slots > pool->n_slots) return LQER_ERR_SHAPE;
  *bytes = adapter_scratch_bytes(M, plan_slots, pool->K, pool->N, pool->max_rank);
  return LQER_OK;
}

lqer_status_t lqer_adapters(const void* X, lqer_dtype_t x_dtype, int M, const lqer_adapter_pool_t* pool, void* plan, int plan_slots,
                            const void* Y0, lqer_dtype_t y0_dtype, void* Y, lqer_dtype_t y_dtype, const lqer_config_t* cfg, void* workspace,
                            size_t workspace_bytes, void* stream) {
  if (X == nullptr || plan == nullptr || Y0 == nullptr || Y == nullptr) return LQER_ERR_NULL;
  lqer_status_t st = pool_ready(pool);
  if (st != LQER_OK) return st;
  lqer_config_t f;
  if ((st = activation_format(cfg, &f)) != LQER_OK) return st;
  if (!any_type(x_dtype) || !plain_type(y0_dtype) || !plain_type(y_dtype)) return LQER_ERR_CONFIG;
  if (!rows_ok(M) || plan_slots < 1 || plan_slots > pool->n_slots) return LQER_ERR_SHAPE;
  if (misaligned(X) || misaligned(Y0) || misaligned(Y) || misaligned(plan, 256)) return LQER_ERR_ALIGN;
  if (Y == X || (Y == Y0 && y0_dtype != y_dtype)) return LQER_ERR_CONFIG;
  const size_t need = adapter_scratch_bytes(M, plan_slots, pool->K, pool->N, pool->max_rank);
  if (need > 0) {
    if (workspace == nullptr) return LQER_ERR_NULL;
    if (misaligned(workspace, 256)) return LQER_ERR_ALIGN;
    if (workspace_bytes < need) return LQER_ERR_BUFFER_TOO_SMALL;
  }
  if ((st = check_arch()) != LQER_OK) return st;
  return of(launch_adapters(X, x_dtype, M, pool->data, pool->K, pool->N, pool->max_rank, plan, plan_slots, Y0, y0_dtype, Y,
                            y_dtype, f.a_bits, f.exp_min, f.exp_max, workspace, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
