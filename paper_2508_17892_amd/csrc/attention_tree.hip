// Attention of a tree of drafted tokens over a cache of the states' own element type.
#include "attend.h"

namespace ilre {

hipError_t launch_attention_tree(const AttnPlan &p, const AttnArgs &a, hipStream_t s) { return launch_kernels<true, kPlain, true>(p, a, s); }

}  // namespace ilre
