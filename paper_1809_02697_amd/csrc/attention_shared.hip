// Attention of the tokens of each group of sequences over the keys that the group
// shares (attention_kernels.h, kShared): every row's part, for attention_own.hip.
#include "attention_kernels.h"

namespace neo {

// By the bytes of the cache that sharing saves at most.  Its second launch, and the
// parts that its first leaves and joins, take as long as some 250 MB of reading.
// Shared, and each sequence reading all of its own (us, 32 heads on 8 of 128):
// one token of each of 2 sequences on 32,000 (68 MB) 34 and 32, 16 on 4000 (127 MB)
// 47 and 33, 32 on 4000 (262 MB) 47 and 49, 256 on 32,000 (17 GB) 217 and 1777;
// float16 chunks of up to 128 tokens, 16 on 4 prefixes of 8000 (203 MB) 216 and 184,
// 16 on one (253 MB) 318 and 341; of up to 16, 64 on 4 of 2000 (253 MB) 85 and 77.
bool attention_worth_sharing(const AttnArgs& shared, const AttnArgs& own, int prefix) {
    const double each = (double)own.c.kv_heads * (2 * own.c.head_dim + 8);
    return (double)(own.seqs - shared.seqs) * prefix * each >= 250e6;
}

size_t attention_shared_floats(const AttnArgs& a) { return parts_floats<kShared>(a); }

hipError_t launch_attention_shared(int dtype, const AttnArgs& a, float* ws, hipStream_t st) { return by_type<kShared>(dtype, a, ws, st); }

}  // namespace neo
