// Whether attention reads the tokens that groups of sequences share once a group:
// numbers alone, so that a program on the host can ask it.
#pragma once
#include <algorithm>
#include <cstdint>

namespace neo {

// By how many cached tokens sharing lessens the reading, from the bounds of a call
// that does not say: as if every sequence were as long as the longest one, which has
// max_own (0: not known, none) tokens behind its prefix, and the groups alike.
//
// A window lessens what sequences read apart to `seen` of the prefix; together all rows
// (`rows` a key/value head: tokens times query heads of one) are multiplied with all of
// it.  32 rows' products with a key that is hidden from them count as reading it.  One
// token of each of 256 sequences on 32,000, bfloat16, shared and apart (us): window 500
// 140 and 59, 1000 155 and 96, 2000 180 and 141, 4000 231 and 249 (apart by this), 8000 226
// and 459 (shared); float32 4000 332 and 290; 16 sequences 8000 76 and 50, 16,000 72 and
// 86 (shared); one query head a key head 1000 122 and 92, 2000 123 and 138 (shared); in 16
// groups on 8000 the rule is wrong at 2000 (shared: 169 and 145).
inline double saved_by_bounds(int64_t seqs, int64_t groups, int64_t rows, int64_t max_chunk, int64_t max_context, int64_t max_own, int64_t window) {
    const int64_t prefix = max_context - std::min(max_own, max_context);
    const int64_t seen = window ? std::min(prefix, window + max_chunk - 1) : prefix;
    return (double)seqs * (double)seen - (double)groups * (double)prefix - (double)rows * (double)(prefix - seen) / 32;
}

// The second launch, and the parts that the first leaves and joins, take as long as some
// 250 MB of reading.  Shared, and each sequence reading all of its own (us, 32 heads on 8 of
// 128): one token of each of 2 sequences on 32,000 (68 MB) 34 and 32, 16 on 4000 (127 MB)
// 47 and 33, 32 on 4000 (262 MB) 47 and 49, 256 on 32,000 (17 GB) 217 and 1777;
// float16 chunks of up to 128 tokens, 16 on 4 prefixes of 8000 (203 MB) 216 and 184,
// 16 on one (253 MB) 318 and 341; of up to 16, 64 on 4 of 2000 (253 MB) 85 and 77.
inline bool worth_sharing(double saved, int kv_heads, int head_dim) {
    return saved * kv_heads * (2.0 * head_dim + 8) >= 250e6;
}

}  // namespace neo
