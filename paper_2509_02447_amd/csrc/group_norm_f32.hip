// Group norm of f32 maps.
#include "group_norm.h"

namespace qrm {

hipError_t launch_norm_forward_f32(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s) { return norm_forward<float>(c, p, ws, s); }
hipError_t launch_norm_backward_f32(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s) { return norm_backward<float>(c, p, ws, s); }

} // namespace qrm
