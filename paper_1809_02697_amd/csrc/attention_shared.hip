// Attention of the tokens of each group of sequences over the keys that the group
// shares (attention_kernels.h, kShared): every row's part, for attention_own.hip.
#include "attention_kernels.h"

namespace neo {

size_t attention_shared_floats(const AttnArgs& a) { return parts_floats<kShared>(a); }

hipError_t launch_attention_shared(int dtype, const AttnArgs& a, float* ws, hipStream_t st) { return by_type<kShared>(dtype, a, ws, st); }

}  // namespace neo
