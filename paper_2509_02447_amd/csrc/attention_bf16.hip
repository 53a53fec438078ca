// Attention of bf16 rows.
#include "attention.h"

namespace qrm {

hipError_t launch_attention_bf16(int kind, const AttnArgs &a, hipStream_t s) { return attention_forward<bf16_t>(kind, a, s); }
hipError_t launch_attention_backward_bf16(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s) { return attention_backward<bf16_t>(by_q, by_k, s); }

} // namespace qrm
