// Attention of f32 rows.
#include "attention.h"

namespace qrm {

hipError_t launch_attention_f32(int kind, const AttnArgs &a, hipStream_t s) { return attention_forward<float>(kind, a, s); }
hipError_t launch_attention_backward_f32(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s) { return attention_backward<float>(by_q, by_k, s); }

} // namespace qrm
