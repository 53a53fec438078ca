// Group norm of f16 maps.
#include "group_norm.h"

namespace qrm {

hipError_t launch_norm_forward_f16(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s) { return norm_forward<f16_t>(c, p, ws, s); }
hipError_t launch_norm_backward_f16(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s) { return norm_backward<f16_t>(c, p, ws, s); }

} // namespace qrm
