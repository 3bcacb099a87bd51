// Causal attention of the newest tokens of each sequence over all of its paged
// int8 cache: the kernels of attention_kernels.h.
#include "attention_kernels.h"

namespace neo {

size_t attention_workspace(const AttnArgs& a) { return parts_floats<kAll>(a) * sizeof(float); }

hipError_t launch_attention(int dtype, const AttnArgs& a, float* ws, hipStream_t st) { return by_type<kAll>(dtype, a, ws, st); }

}  // namespace neo
