// C-ABI entry points of libtaot: argument validation, workspace checks and
// kernel launches.  See include/taot.h for the contract of each call.
#include <math.h>

#include "common.h"

using namespace taot;

namespace {

bool bad_dims(int32_t B, int32_t R) { return B < 0 || R <= 0; }

bool bad_type(int32_t dtype) { return dtype != TAOT_BF16 && dtype != TAOT_F16 && dtype != TAOT_F32; }

bool bad_weight_type(int32_t dtype, int32_t weight_dtype) {
  return bad_type(dtype) || (weight_dtype != dtype && weight_dtype != TAOT_F32);
}

// A gate's rows: `gates` of them divide the T rows.
bool bad_gates(const void* gate, int64_t gates, int64_t T) { return gate && (gates < 1 || T % gates); }

// A workspace that is missing, too small, or begins where the kernels' atomics and scalar loads of its words may not.
bool bad_room(const void* ws, size_t bytes, size_t needed) {
  return !ws || bytes < needed || reinterpret_cast<uintptr_t>(ws) % 8;
}

constexpr int64_t kMaxGrid = 0x7fffffffLL;  // rows that one launch can number
constexpr int32_t kMaxWide = 1 << 30;       // columns whose steps 32 bits can count

// Rows, tokens and choices of the calls that move rows; `copies` gets tokens * k.
taot_status check_rows(int64_t rows, int64_t tokens, int32_t k, int64_t* copies) {
  if (rows < 0 || tokens < 0 || k < 1) return TAOT_ERR_INVALID_ARG;
  if (k > TAOT_MAX_TOP_K || tokens > kMaxGrid / k || (tokens > 0 && rows > kMaxGrid / tokens))
    return TAOT_ERR_UNSUPPORTED;
  *copies = tokens * k;
  return TAOT_OK;
}

}  // namespace

extern "C" {

const char* taot_status_string(taot_status s) {
  switch (s) {
    case TAOT_OK: return "ok";
    case TAOT_ERR_INVALID_ARG: return "invalid argument";
    case TAOT_ERR_UNSUPPORTED: return "unsupported shape";
    case TAOT_ERR_WORKSPACE: return "workspace missing or too small";
    case TAOT_ERR_LAUNCH: return "kernel launch failed";
    case TAOT_ERR_SCRATCH: return "needs more than the fixed scratch of the allocation-free entry point";
  }
  return "unknown status";
}

size_t taot_plan_loads_workspace_size(int32_t B, int32_t R, int32_t E) {
  if (bad_dims(B, R) || E <= 0) return 0;
  return plan_loads_ws(B, R, E);
}

taot_status taot_plan_loads(const int32_t* ids, int32_t B, int32_t R, int64_t N, int32_t E,
                            const int32_t* home, int32_t* n, int64_t* load_e, int64_t* load_r,
                            int64_t* excess, int64_t* spare, int64_t* spill, float* supply,
                            float* demand, double* rho, double* alpha, int64_t* bad_ids,
                            int32_t* hot_idx, int32_t* cold_idx, int32_t* hot_cnt, int32_t* cold_cnt,
                            uint32_t* status, void* ws, size_t ws_bytes, void* stream) {
  if (bad_dims(B, R) || E <= 0 || N < 0) return TAOT_ERR_INVALID_ARG;
  if (R > TAOT_MAX_RANKS || E > TAOT_MAX_EXPERTS) return TAOT_ERR_UNSUPPORTED;
  if (B == 0) return TAOT_OK;
  if ((N > 0 && !ids) || !home || !n || !load_e || !load_r || !excess || !spare || !spill || !alpha)
    return TAOT_ERR_INVALID_ARG;
  if ((int64_t)B * R > 0x7fffffffLL || N > 0x7fffffffLL) return TAOT_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < plan_loads_ws(B, R, E)) return TAOT_ERR_WORKSPACE;
  return launch_plan_loads(ids, B, R, N, E, home, n, load_e, load_r, excess, spare, spill, supply,
                           demand, rho, alpha, bad_ids, hot_idx, cold_idx, hot_cnt, cold_cnt, status, ws,
                           static_cast<hipStream_t>(stream));
}

taot_status taot_plan_loads_noalloc(const int32_t* ids, int32_t B, int32_t R, int64_t N, int32_t E,
                                    const int32_t* home, int32_t* n, int64_t* load_e, int64_t* load_r,
                                    int64_t* excess, int64_t* spare, int64_t* spill, float* supply,
                                    float* demand, double* rho, double* alpha, int64_t* bad_ids,
                                    int32_t* hot_idx, int32_t* cold_idx, int32_t* hot_cnt, int32_t* cold_cnt,
                                    uint32_t* status, void* stream) {
  if (bad_dims(B, R) || E <= 0 || N < 0) return TAOT_ERR_INVALID_ARG;
  if (R > TAOT_MAX_RANKS || E > TAOT_MAX_EXPERTS) return TAOT_ERR_UNSUPPORTED;
  if (B == 0) return TAOT_OK;
  if ((N > 0 && !ids) || !home || !n || !load_e || !load_r || !excess || !spare || !spill || !alpha)
    return TAOT_ERR_INVALID_ARG;
  if ((int64_t)B * R > 0x7fffffffLL || N > 0x7fffffffLL) return TAOT_ERR_UNSUPPORTED;
  if (plan_loads_ws(B, R, E) > plan_loads_scratch_limit()) return TAOT_ERR_SCRATCH;
  void* ws = plan_loads_scratch();
  if (!ws) return TAOT_ERR_LAUNCH;
  return launch_plan_loads(ids, B, R, N, E, home, n, load_e, load_r, excess, spare, spill, supply,
                           demand, rho, alpha, bad_ids, hot_idx, cold_idx, hot_cnt, cold_cnt, status, ws,
                           static_cast<hipStream_t>(stream));
}

size_t taot_plan_loads_noalloc_max_problems(int32_t R, int32_t E) {
  if (R <= 0 || E <= 0 || R > TAOT_MAX_RANKS || E > TAOT_MAX_EXPERTS) return 0;
  size_t lo = 0, hi = (size_t)1 << 31;  // largest B whose workspace fits the scratch
  while (lo + 1 < hi) {
    const size_t mid = (lo + hi) / 2;
    if (plan_loads_ws((int32_t)(mid > 0x7fffffff ? 0x7fffffff : mid), R, E) <= plan_loads_scratch_limit()) lo = mid;
    else hi = mid;
  }
  return lo;
}

size_t taot_sinkhorn_workspace_size(int32_t B, int32_t R) {
  if (bad_dims(B, R)) return 0;
  return sinkhorn_ws(B, R);
}

taot_status taot_sinkhorn_batched(const float* a, const float* b, int32_t B, int32_t R,
                                  const float* C, int64_t C_batch_stride, float eps,
                                  int32_t iters, uint32_t flags, float* T, float* f, float* g,
                                  uint32_t* status, void* ws, size_t ws_bytes, void* stream) {
  if (bad_dims(B, R) || !(eps > 0.f) || !isfinite(eps) || iters < 1 ||
      (C_batch_stride != 0 && C_batch_stride != (int64_t)R * R) ||
      (flags & ~(TAOT_SK_NO_COLCAP | TAOT_SK_FORCE_STREAM | TAOT_SK_NO_REGISTER | TAOT_SK_WAVES_1 |
                 TAOT_SK_DENSE | TAOT_SK_LINEAR)))
    return TAOT_ERR_INVALID_ARG;
  if (R > TAOT_MAX_RANKS) return TAOT_ERR_UNSUPPORTED;
  if (B == 0) return TAOT_OK;
  if (!a || !b || !C) return TAOT_ERR_INVALID_ARG;
  if (!ws || ws_bytes < sinkhorn_ws(B, R)) return TAOT_ERR_WORKSPACE;
  return launch_sinkhorn(a, b, B, R, C, C_batch_stride, eps, iters, flags, T, f, g, status, ws,
                         static_cast<hipStream_t>(stream));
}

size_t taot_round_schedule_workspace_size(int32_t B, int32_t R, int32_t E, int32_t K) {
  if (bad_dims(B, R) || E <= 0 || K < 0) return 0;
  return schedule_ws(B, R, E, K);
}

taot_status taot_round_schedule(const int32_t* n, const int64_t* spill, const int64_t* spare,
                                const int64_t* excess, const double* alpha, const int32_t* home,
                                const float* T, const double* Bpref, const double* Bauct,
                                int32_t B, int32_t R, int32_t E, int32_t K, double price_step,
                                int64_t t_max, uint32_t flags, int32_t* slot_expert, int64_t* slot_amount,
                                int32_t* X, int64_t* unfilled, int32_t* rounds_used,
                                uint32_t* status, void* ws, size_t ws_bytes, void* stream) {
  if (bad_dims(B, R) || E <= 0 || K < 0 || !isfinite(price_step)) return TAOT_ERR_INVALID_ARG;
  if (flags & ~(TAOT_SCH_NO_TOPO | TAOT_SCH_NO_FLOW | TAOT_SCH_ROW_PRIORITY)) return TAOT_ERR_INVALID_ARG;
  if (R > TAOT_MAX_RANKS || E > TAOT_MAX_EXPERTS || K > TAOT_MAX_SLOTS_PER_RANK)
    return TAOT_ERR_UNSUPPORTED;
  if (B == 0) return TAOT_OK;
  if (!n || !spill || !spare || !excess || !alpha || !home || !T || !Bpref || !Bauct ||
      (K > 0 && (!slot_expert || !slot_amount || !X)) || !unfilled)
    return TAOT_ERR_INVALID_ARG;
  if ((int64_t)R * K * R > 0x7fffffffLL * 8) return TAOT_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < schedule_ws(B, R, E, K)) return TAOT_ERR_WORKSPACE;
  return launch_schedule(n, spill, spare, excess, alpha, home, T, Bpref, Bauct, B, R, E, K,
                         price_step, t_max, flags, slot_expert, slot_amount, X, unfilled, rounds_used,
                         status, ws, static_cast<hipStream_t>(stream));
}

taot_status taot_add_rms_norm(const void* x, const void* residual, const void* weight, int64_t T, int32_t H,
                              int32_t dtype, int32_t weight_dtype, float eps, int32_t group, void* h, void* y,
                              void* q, float* scale, float* rstd, void* stream) {
  if (T < 0 || H <= 0 || bad_weight_type(dtype, weight_dtype) || !(eps >= 0.f) || !isfinite(eps) || !q != !scale)
    return TAOT_ERR_INVALID_ARG;
  if (group != 0 && (group < 8 || group > 512 || (group & (group - 1)))) return TAOT_ERR_INVALID_ARG;
  if (H > TAOT_MAX_WIDTH || T > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (T == 0) return TAOT_OK;
  if (!x || !weight) return TAOT_ERR_INVALID_ARG;
  return launch_add_rms_norm(x, residual, weight, T, H, dtype, weight_dtype, eps, group, h, y,
                             static_cast<uint8_t*>(q), scale, rstd, static_cast<hipStream_t>(stream));
}

size_t taot_add_rms_norm_backward_workspace_size(int64_t T, int32_t H) {
  if (T < 0 || H <= 0) return 0;
  return add_rms_norm_backward_ws(T, H);
}

taot_status taot_add_rms_norm_backward(const void* dy, const void* dh, const void* h, const float* rstd,
                                       const void* weight, int64_t T, int32_t H, int32_t dtype,
                                       int32_t weight_dtype, void* dx, float* dweight, void* ws, size_t ws_bytes,
                                       void* stream) {
  if (T < 0 || H <= 0 || bad_weight_type(dtype, weight_dtype)) return TAOT_ERR_INVALID_ARG;
  if (H > TAOT_MAX_WIDTH || T > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (!weight || !dweight || (T > 0 && (!dy || !h || !rstd || !dx))) return TAOT_ERR_INVALID_ARG;
  if (T > 0 && (!ws || ws_bytes < add_rms_norm_backward_ws(T, H))) return TAOT_ERR_WORKSPACE;
  return launch_add_rms_norm_backward(dy, dh, h, rstd, weight, T, H, dtype, weight_dtype, dx, dweight, ws,
                                      static_cast<hipStream_t>(stream));
}

taot_status taot_route(const void* logits, const float* bias, int64_t T, int32_t E, int32_t k, int32_t groups,
                       int32_t top_groups, float scale, uint32_t flags, int32_t dtype, int32_t* ids, float* weights,
                       void* stream) {
  if (T < 0 || E <= 0 || k < 1 || k > E || groups < 1 || top_groups < 1 || top_groups > groups || bad_type(dtype) ||
      !isfinite(scale) || (flags & ~(TAOT_ROUTE_SIGMOID | TAOT_ROUTE_RENORM | TAOT_ROUTE_GROUP_TWO)))
    return TAOT_ERR_INVALID_ARG;
  if (E % groups || (int64_t)(E / groups) * top_groups < k) return TAOT_ERR_INVALID_ARG;
  if (E > TAOT_MAX_EXPERTS || k > TAOT_MAX_TOP_K || groups > TAOT_MAX_ROUTE_GROUPS || T > kMaxGrid)
    return TAOT_ERR_UNSUPPORTED;
  if (T == 0) return TAOT_OK;
  if (!logits || !ids || !weights) return TAOT_ERR_INVALID_ARG;
  return launch_route(logits, bias, T, E, k, groups, top_groups, scale, flags, dtype, ids, weights,
                      static_cast<hipStream_t>(stream));
}

taot_status taot_route_backward(const float* dweights, const void* logits, const int32_t* ids, int64_t T, int32_t E,
                                int32_t k, float scale, uint32_t flags, int32_t dtype, void* dlogits, void* stream) {
  if (T < 0 || E <= 0 || k < 1 || k > E || bad_type(dtype) || !isfinite(scale) ||
      (flags & ~(TAOT_ROUTE_SIGMOID | TAOT_ROUTE_RENORM | TAOT_ROUTE_GROUP_TWO)))
    return TAOT_ERR_INVALID_ARG;
  if (E > TAOT_MAX_EXPERTS || k > TAOT_MAX_TOP_K || T > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (T == 0) return TAOT_OK;
  if (!dweights || !logits || !ids || !dlogits) return TAOT_ERR_INVALID_ARG;
  return launch_route_backward(dweights, logits, ids, T, E, k, scale, flags, dtype, dlogits,
                               static_cast<hipStream_t>(stream));
}

size_t taot_dispatch_map_workspace_size(int32_t B, int32_t rows, int64_t N, int32_t R, int32_t E, int32_t K) {
  if (bad_dims(B, R) || rows <= 0 || N < 0 || E <= 0 || K < 0) return 0;
  return dispatch_map_ws(B, rows, N, R, E, K);
}

taot_status taot_dispatch_map(const int32_t* ids, int32_t B, int32_t rows, int32_t rank0, int64_t N,
                              const int32_t* home, int32_t R, int32_t E, int32_t K, const int32_t* slot_expert,
                              const int32_t* X, int32_t* pos, int32_t* offsets, int32_t* sends, uint32_t* status,
                              void* ws, size_t ws_bytes, void* stream) {
  if (bad_dims(B, R) || rows <= 0 || rank0 < 0 || rank0 > R - rows || N < 0 || E <= 0 || K < 0)
    return TAOT_ERR_INVALID_ARG;
  if (R > TAOT_MAX_RANKS || E > TAOT_MAX_EXPERTS || K > TAOT_MAX_SLOTS_PER_RANK) return TAOT_ERR_UNSUPPORTED;
  if ((int64_t)B * rows > kMaxGrid / 4 || N > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (B == 0) return TAOT_OK;
  if ((N > 0 && (!ids || !pos)) || !home || (K > 0 && (!slot_expert || !X)) || !offsets || !sends)
    return TAOT_ERR_INVALID_ARG;
  if (!ws || ws_bytes < dispatch_map_ws(B, rows, N, R, E, K)) return TAOT_ERR_WORKSPACE;
  return launch_dispatch_map(ids, B, rows, rank0, N, home, R, E, K, slot_expert, X, pos, offsets, sends, status, ws,
                             static_cast<hipStream_t>(stream));
}

taot_status taot_dispatch_rows(const void* x, int64_t row_bytes, const void* x_more, int64_t more_bytes,
                               int64_t rows, int64_t tokens, int32_t k, const int32_t* pos, void* out,
                               void* out_more, void* stream) {
  int64_t n = 0;
  if (row_bytes <= 0 || more_bytes < 0 || (more_bytes > 0) != (x_more != nullptr) ||
      (more_bytes > 0) != (out_more != nullptr))
    return TAOT_ERR_INVALID_ARG;
  if (taot_status s = check_rows(rows, tokens, k, &n)) return s;
  if (row_bytes > kMaxGrid || more_bytes > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (rows == 0 || n == 0) return TAOT_OK;
  if (!x || !pos || !out) return TAOT_ERR_INVALID_ARG;
  return launch_dispatch_rows(x, row_bytes, x_more, more_bytes, rows, tokens, k, pos, out, out_more,
                              static_cast<hipStream_t>(stream));
}

taot_status taot_combine_rows(const void* y, const int32_t* pos, const float* weights, int64_t rows, int64_t tokens,
                              int32_t k, int32_t H, int32_t dtype, void* out, void* stream) {
  int64_t n = 0;
  if (H <= 0 || bad_type(dtype)) return TAOT_ERR_INVALID_ARG;
  if (taot_status s = check_rows(rows, tokens, k, &n)) return s;
  if (H > kMaxWide) return TAOT_ERR_UNSUPPORTED;
  if (rows == 0 || n == 0) return TAOT_OK;
  if (!y || !pos || !out) return TAOT_ERR_INVALID_ARG;
  return launch_combine_rows(y, pos, weights, rows, tokens, k, H, dtype, out, static_cast<hipStream_t>(stream));
}

taot_status taot_combine_rows_backward(const void* dout, const void* y, const int32_t* pos, const float* weights,
                                       int64_t rows, int64_t tokens, int32_t k, int32_t H, int32_t dtype, void* dy,
                                       float* dweights, void* stream) {
  int64_t n = 0;
  if (H <= 0 || bad_type(dtype)) return TAOT_ERR_INVALID_ARG;
  if (taot_status s = check_rows(rows, tokens, k, &n)) return s;
  if (H > kMaxWide) return TAOT_ERR_UNSUPPORTED;
  if (rows == 0 || n == 0) return TAOT_OK;
  if (!dout || !y || !pos || !weights || !dy || !dweights) return TAOT_ERR_INVALID_ARG;
  return launch_combine_rows_backward(dout, y, pos, weights, rows, tokens, k, H, dtype, dy, dweights,
                                      static_cast<hipStream_t>(stream));
}

taot_status taot_block_norm(const void* x, const void* residual, const void* post, const void* gate, int64_t gates,
                            const void* weight, int64_t T, int32_t H, int32_t dtype, int32_t weight_dtype,
                            int32_t gate_dtype, float eps, float alpha, void* h, void* y, float* rstd_x, float* rstd_h,
                            void* stream) {
  if (T < 0 || H <= 0 || bad_weight_type(dtype, weight_dtype) || bad_weight_type(dtype, gate_dtype) || !(eps >= 0.f) ||
      !isfinite(eps) || !isfinite(alpha) || bad_gates(gate, gates, T) || (y && !weight))
    return TAOT_ERR_INVALID_ARG;
  if (H > TAOT_MAX_WIDTH || T > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (T == 0) return TAOT_OK;
  if (!x || !residual) return TAOT_ERR_INVALID_ARG;
  return launch_block_norm(BlockNormArgs{x, residual, post, gate, weight, T, gate ? gates : 1, H, weight_dtype == TAOT_F32,
                                         gate_dtype == TAOT_F32, eps, alpha, h, y, rstd_x, rstd_h},
                           dtype, static_cast<hipStream_t>(stream));
}

size_t taot_block_norm_backward_workspace_size(int64_t T, int32_t H, int64_t gates) {
  if (T <= 0 || H <= 0 || gates < 0 || (gates > 0 && T % gates)) return 0;
  return block_norm_backward_ws(T, H, gates > 0 ? gates : 1);
}

taot_status taot_block_norm_backward(const void* dy, const void* dh, const void* x, const void* h, const float* rstd_x,
                                     const float* rstd_h, const void* post, const void* gate, int64_t gates,
                                     const void* weight, int64_t T, int32_t H, int32_t dtype, int32_t weight_dtype,
                                     int32_t gate_dtype, float alpha, void* dx, void* dresidual, float* dweight,
                                     float* dpost, float* dgate, void* ws, size_t ws_bytes, void* stream) {
  if (T < 0 || H <= 0 || bad_weight_type(dtype, weight_dtype) || bad_weight_type(dtype, gate_dtype) || !isfinite(alpha) ||
      bad_gates(gate, gates, T) || (dweight && !weight) || (dpost && !post) || (dgate && !gate))
    return TAOT_ERR_INVALID_ARG;
  if (H > TAOT_MAX_WIDTH || T > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (T > 0 && (!x || !dx || !dresidual || (weight && (!dy || !h || !rstd_h)) || (!weight && !dh) || (post && !rstd_x)))
    return TAOT_ERR_INVALID_ARG;
  const int64_t sets = gate ? gates : 1;
  if (T > 0 && bad_room(ws, ws_bytes, block_norm_backward_ws(T, H, sets))) return TAOT_ERR_WORKSPACE;
  return launch_block_norm_backward(
      BlockNormGradArgs{dy, dh, x, h, rstd_x, rstd_h, post, gate, weight, T, sets, H, weight_dtype == TAOT_F32,
                        gate_dtype == TAOT_F32, alpha, dx, dresidual, dweight, dpost, dgate},
      dtype, ws, static_cast<hipStream_t>(stream));
}

size_t taot_balance_loss_workspace_size(int64_t rows, int64_t tokens, int32_t E) {
  if (rows <= 0 || tokens < 0 || E <= 0) return 0;
  return balance_loss_ws(rows, tokens, E);
}

taot_status taot_balance_loss(const void* logits, const int32_t* ids, const uint8_t* mask, int64_t rows, int64_t tokens,
                              int32_t E, int32_t k, uint32_t flags, int32_t dtype, float* loss, float* z,
                              int32_t* counts, float* prob, int32_t* counted, void* ws, size_t ws_bytes, void* stream) {
  int64_t n = 0;
  if (E <= 0 || bad_type(dtype) || (flags & ~TAOT_ROUTE_SIGMOID) || (z && (flags & TAOT_ROUTE_SIGMOID)))
    return TAOT_ERR_INVALID_ARG;
  if (taot_status s = check_rows(rows, tokens, k, &n)) return s;
  if (E > TAOT_MAX_EXPERTS || rows > kMaxGrid || (n > 0 && rows > kMaxGrid / n)) return TAOT_ERR_UNSUPPORTED;
  if (rows == 0) return TAOT_OK;
  if ((tokens > 0 && (!logits || !ids)) || !loss || !counts || !prob) return TAOT_ERR_INVALID_ARG;
  if (bad_room(ws, ws_bytes, balance_loss_ws(rows, tokens, E))) return TAOT_ERR_WORKSPACE;
  return launch_balance_loss(logits, ids, mask, rows, tokens, E, k, flags, dtype, loss, z, counts, prob, counted, ws,
                             static_cast<hipStream_t>(stream));
}

taot_status taot_balance_loss_backward(const float* dloss, const float* dz, const void* logits, const int32_t* counts,
                                       const int32_t* counted, const uint8_t* mask, const void* add, int64_t rows,
                                       int64_t tokens, int32_t E, uint32_t flags, int32_t dtype, void* dlogits,
                                       void* stream) {
  int64_t n = 0;
  if (E <= 0 || bad_type(dtype) || (flags & ~TAOT_ROUTE_SIGMOID) || (dz && (flags & TAOT_ROUTE_SIGMOID)))
    return TAOT_ERR_INVALID_ARG;
  if (taot_status s = check_rows(rows, tokens, 1, &n)) return s;
  if (E > TAOT_MAX_EXPERTS) return TAOT_ERR_UNSUPPORTED;
  if (rows == 0 || tokens == 0) return TAOT_OK;
  if (!dloss || !logits || !counts || !counted || !dlogits) return TAOT_ERR_INVALID_ARG;
  return launch_balance_loss_backward(dloss, dz, logits, counts, counted, mask, add, rows, tokens, E, flags, dtype, dlogits,
                                      static_cast<hipStream_t>(stream));
}

taot_status taot_quantize_rows(const void* x, int64_t T, int32_t H, int32_t gated, int32_t dtype, int8_t* q,
                               float* scale, void* stream) {
  if (T < 0 || H <= 0 || bad_type(dtype) || (gated != 0 && gated != 1)) return TAOT_ERR_INVALID_ARG;
  if (H > TAOT_MAX_WIDTH || T > kMaxGrid) return TAOT_ERR_UNSUPPORTED;
  if (T == 0) return TAOT_OK;
  if (!x || !q || !scale) return TAOT_ERR_INVALID_ARG;
  return launch_quantize_rows(x, T, H, gated != 0, dtype, q, scale, static_cast<hipStream_t>(stream));
}

size_t taot_matmul_i8_workspace_size(int64_t M, int32_t runs) {
  if (M < 0 || runs < 0 || M > kMaxWide || runs > kMaxWide) return 0;
  return matmul_i8_ws(M, runs);
}

taot_status taot_matmul_i8(const int8_t* x, const float* scale, const int8_t* weight, const float* weight_scale,
                           const int32_t* offsets, const int32_t* experts, int64_t M, int32_t N, int32_t K, int32_t runs,
                           int32_t G, int32_t dtype, void* out, void* ws, size_t ws_bytes, void* stream) {
  if (M < 0 || N <= 0 || K <= 0 || runs < 0 || G <= 0 || bad_type(dtype) || (!offsets && (runs != 0 || G != 1 || experts)))
    return TAOT_ERR_INVALID_ARG;
  if (K > TAOT_MAX_INNER || M > kMaxWide || N > kMaxWide || runs > kMaxWide) return TAOT_ERR_UNSUPPORTED;
  if (M == 0) return TAOT_OK;
  if (!x || !scale || !weight || !weight_scale || !out) return TAOT_ERR_INVALID_ARG;
  if (offsets && bad_room(ws, ws_bytes, matmul_i8_ws(M, runs))) return TAOT_ERR_WORKSPACE;
  return launch_matmul_i8(ProductArgs{x, scale, weight, weight_scale, offsets, experts, M, N, K, runs, G, out}, dtype, ws,
                          static_cast<hipStream_t>(stream));
}

taot_status taot_topology_pref(const float* C_host, int32_t R, double* Bpref_host,
                               double* Bauct_host) {
  if (!C_host || !Bpref_host || !Bauct_host || R <= 0) return TAOT_ERR_INVALID_ARG;
  double cmin = INFINITY;
  for (int64_t i = 0; i < R; ++i)
    for (int64_t j = 0; j < R; ++j) {
      if (i == j) continue;
      const double c = (double)C_host[i * R + j];
      if (!isfinite(c) || !(c > 0.0)) return TAOT_ERR_INVALID_ARG;
      cmin = c < cmin ? c : cmin;
    }
  if (R == 1) cmin = 1.0;
  for (int64_t i = 0; i < R; ++i)
    for (int64_t j = 0; j < R; ++j) {
      const int64_t q = i * R + j;
      if (i == j) {
        Bpref_host[q] = 0.0;
        Bauct_host[q] = 1.0;
      } else {
        Bpref_host[q] = cmin / (double)C_host[q];
        Bauct_host[q] = Bpref_host[q];
      }
    }
  return TAOT_OK;
}

}  // extern "C"
