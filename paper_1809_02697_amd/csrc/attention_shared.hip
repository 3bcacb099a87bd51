// Attention of the tokens of each group of sequences over the keys that the group
// shares (attention_kernels.h, kShared): every row's part, for attention_own.hip.
#include "attention_kernels.h"

namespace neo {

// By the bytes of the cache that sharing saves at most.  Against each sequence
// reading all of its own (one token a sequence, 32 heads on 8 of 128, bfloat16): a
// second launch and the join of its parts take some 10 us, as long as 64 MB of
// reading (8 sequences on 4000 tokens, 59 MB: 28.7 us shared and 27.6 apart; 2 on
// 32,000, 68 MB: 34 and 40), and more where the groups' rows go to the kernel of
// tiles (16 on 4000, 127 MB: 47 and 37; 32 on 4000, 262 MB: 47 and 53; 16 chunks of
// up to 128 on 8000, 253 MB: 315 and 355).
bool attention_worth_sharing(const AttnArgs& shared, const AttnArgs& own, int prefix) {
    const double each = (double)own.c.kv_heads * (2 * own.c.head_dim + 8);
    return (double)(own.seqs - shared.seqs) * prefix * each >= (tile_rows(shared) == 16 ? 64e6 : 200e6);
}

size_t attention_shared_floats(const AttnArgs& a) { return parts_floats<kShared>(a); }

hipError_t launch_attention_shared(int dtype, const AttnArgs& a, float* ws, hipStream_t st) { return by_type<kShared>(dtype, a, ws, st); }

}  // namespace neo
