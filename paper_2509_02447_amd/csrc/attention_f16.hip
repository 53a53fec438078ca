// Attention of f16 rows.
#include "attention.h"

namespace qrm {

hipError_t launch_attention_f16(int kind, const AttnArgs &a, hipStream_t s) { return attention_forward<f16_t>(kind, a, s); }
hipError_t launch_attention_backward_f16(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s) { return attention_backward<f16_t>(by_q, by_k, s); }

} // namespace qrm
