// Group norm of bf16 maps.
#include "group_norm.h"

namespace qrm {

hipError_t launch_norm_forward_bf16(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s) { return norm_forward<bf16_t>(c, p, ws, s); }
hipError_t launch_norm_backward_bf16(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s) { return norm_backward<bf16_t>(c, p, ws, s); }

} // namespace qrm
