// Attention of f16 rows.
#include "attention.h"

namespace qrm {

hipError_t launch_attention_f16(int kind, const AttnArgs &a, hipStream_t s) { return attention_launch<f16_t>(kind, a, s); }

} // namespace qrm
