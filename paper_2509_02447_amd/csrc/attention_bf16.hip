// Attention of bf16 rows.
#include "attention.h"

namespace qrm {

hipError_t launch_attention_bf16(int kind, const AttnArgs &a, hipStream_t s) { return attention_launch<bf16_t>(kind, a, s); }

} // namespace qrm
