// The kernels of gs_softmax_loss and gs_scores for one storage format (the formats compile side by side).
#define GS_SOFTMAX_KERNELS
#include "softmax.h"

namespace gs {
template SoftmaxPlan plan_softmax<F16>(void*, int64_t, int64_t, int32_t, bool, bool);
template int32_t run_softmax<F16>(const SoftmaxCall&, const SoftmaxPlan&, hipStream_t);
}  // namespace gs
