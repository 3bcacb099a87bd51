// Attention of each sequence's newest tokens over the keys behind those that its
// group shares (attention_kernels.h, kOwn), joined with the parts of those.
#include "attention_kernels.h"

namespace neo {

size_t attention_own_floats(const AttnArgs& a) { return parts_floats<kOwn>(a); }

hipError_t launch_attention_own(int dtype, const AttnArgs& a, float* ws, hipStream_t st) { return by_type<kOwn>(dtype, a, ws, st); }

}  // namespace neo
