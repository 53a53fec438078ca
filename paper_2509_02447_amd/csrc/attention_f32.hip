// Attention of f32 rows.
#include "attention.h"

namespace qrm {

hipError_t launch_attention_f32(int kind, const AttnArgs &a, hipStream_t s) { return attention_launch<float>(kind, a, s); }

} // namespace qrm
