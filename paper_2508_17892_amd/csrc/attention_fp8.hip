// Attention over a cache of 8-bit codes.
#include "attend.h"

namespace ilre {

hipError_t launch_attention_fp8(const AttnPlan &p, const AttnArgs &a, hipStream_t s) { return launch_kernels<true, ILRE_KV_FP8, false>(p, a, s); }

}  // namespace ilre
