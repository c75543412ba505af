// gs_softmax_loss, gs_scores: argument checks and the choice of the storage format (kernels: softmax.h).
#include "softmax.h"

#include <cmath>

namespace gs {
namespace {

bool dtype_known(int32_t dtype) { return dtype == GS_F32 || dtype == GS_BF16 || dtype == GS_F16; }

SoftmaxPlan plan_any(void* ws, int64_t num_pairs, int64_t num_nodes, int32_t dim, int32_t dtype, bool loss, bool grad) {
  if (dtype == GS_F32) return plan_softmax<F32>(ws, num_pairs, num_nodes, dim, loss, grad);
  if (dtype == GS_BF16) return plan_softmax<BF16>(ws, num_pairs, num_nodes, dim, loss, grad);
  return plan_softmax<F16>(ws, num_pairs, num_nodes, dim, loss, grad);
}

int32_t run_any(const SoftmaxCall& q, const SoftmaxPlan& p, int32_t dtype, hipStream_t stream) {
  if (dtype == GS_F32) return run_softmax<F32>(q, p, stream);
  if (dtype == GS_BF16) return run_softmax<BF16>(q, p, stream);
  return run_softmax<F16>(q, p, stream);
}

bool shape_ok(int64_t num_pairs, int64_t num_nodes, int32_t dim, int32_t dtype) {
  return dtype_known(dtype) && num_pairs >= 0 && num_pairs <= (int64_t)INT32_MAX && num_nodes >= 1 &&
         num_nodes <= (int64_t)INT32_MAX && dim >= 1 && dim <= 256 && dim % (dtype == GS_F32 ? 4 : 8) == 0;
}

int32_t check_call(const SoftmaxCall& q, int32_t dtype, const void* ws) {
  if (!shape_ok(q.num_pairs, q.num_nodes, q.dim, dtype) || q.num_in < 1 || q.num_in > (int64_t)INT32_MAX) return GS_EINVAL;
  if (!q.w_in || !q.w_out || !aligned(q.w_in, 16) || !aligned(q.w_out, 16)) return GS_EINVAL;
  if (!(q.scale > 0.0f) || !std::isfinite(q.scale)) return GS_EINVAL;
  if (!ws || !aligned(ws, 256)) return GS_EINVAL;
  return GS_OK;
}

}  // namespace
}  // namespace gs

using namespace gs;

extern "C" size_t gs_softmax_loss_workspace_bytes(int64_t num_pairs, int64_t num_nodes, int32_t dim, int32_t dtype,
                                                  int32_t want_grad) {
  if (!shape_ok(num_pairs, num_nodes, dim, dtype)) return 0;
  return plan_any(nullptr, num_pairs, num_nodes, dim, dtype, true, want_grad != 0).bytes;
}

extern "C" int32_t gs_softmax_loss(const void* w_in, int64_t num_in, const void* w_out, int64_t num_nodes, int32_t dim,
                                   int32_t dtype, const int32_t* centers, const int32_t* contexts, int64_t num_pairs,
                                   const float* bias, float scale, float* loss_out, void* g_in, void* g_out,
                                   float grad_scale, void* ws, size_t ws_bytes, void* stream) {
  SoftmaxCall q{w_in, w_out, num_in, num_nodes, num_pairs, dim, centers, contexts, bias, scale, grad_scale, loss_out, g_in, g_out, nullptr};
  const int32_t rc = check_call(q, dtype, ws);
  if (rc != GS_OK) return rc;
  if (num_pairs > 0 && (!centers || !contexts || !loss_out)) return GS_EINVAL;
  if (!aligned(g_in, 16) || !aligned(g_out, 16) || !std::isfinite(grad_scale)) return GS_EINVAL;
  if ((g_in && (g_in == w_in || g_in == w_out)) || (g_out && (g_out == w_in || g_out == w_out || g_out == g_in))) return GS_EINVAL;
  const SoftmaxPlan p = plan_any(ws, num_pairs, num_nodes, dim, dtype, true, g_in || g_out);
  if (ws_bytes < p.bytes) return GS_EWORKSPACE;
  return run_any(q, p, dtype, (hipStream_t)stream);
}

extern "C" size_t gs_scores_workspace_bytes(int64_t num_pairs, int64_t num_nodes, int32_t dim, int32_t dtype) {
  if (!shape_ok(num_pairs, num_nodes, dim, dtype)) return 0;
  return plan_any(nullptr, num_pairs, num_nodes, dim, dtype, false, false).bytes;
}

extern "C" int32_t gs_scores(const void* w_in, int64_t num_in, const void* w_out, int64_t num_nodes, int32_t dim,
                             int32_t dtype, const int32_t* centers, int64_t num_centers, const float* bias, float scale,
                             float* scores_out, void* ws, size_t ws_bytes, void* stream) {
  SoftmaxCall q{w_in, w_out, num_in, num_nodes, num_centers, dim, centers, nullptr, bias, scale, 0.0f, nullptr, nullptr, nullptr, scores_out};
  const int32_t rc = check_call(q, dtype, ws);
  if (rc != GS_OK) return rc;
  if (num_centers > 0 && (!centers || !scores_out)) return GS_EINVAL;
  const SoftmaxPlan p = plan_any(ws, num_centers, num_nodes, dim, dtype, false, false);
  if (ws_bytes < p.bytes) return GS_EWORKSPACE;
  if (num_centers == 0) return GS_OK;
  return run_any(q, p, dtype, (hipStream_t)stream);
}
