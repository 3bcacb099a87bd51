// Which keys a token of a chunk sees: integers alone, so that a program on the
// host can go through their whole range.
#pragma once

#if defined(__HIPCC__)
#define NEO_KEYS_FN __host__ __device__ inline
#else
#define NEO_KEYS_FN inline
#endif

namespace neo {

// The first key that the token at `pos` sees under `window` (0: no limit); 0 for
// a token that sees nothing (pos < 0).  No intermediate leaves 32 bits.
NEO_KEYS_FN int first_seen(int pos, int window) {
    const int first = pos < 0 || window == 0 ? 0 : pos - (window - 1);
    return first < 0 ? 0 : first;
}

// The keys [lo, hi) that the tokens t0 .. t1 of a sequence's `all` new ones see
// among the first `end` of its `ctx` cached ones: 0 <= lo <= hi <= end, empty
// where they see none of those (a window that lies past `end`, say).
NEO_KEYS_FN void seen_keys(int ctx, int all, int end, int t0, int t1, int window, int& lo, int& hi) {
    const int first = first_seen(ctx - all + t0, window), past = ctx - all + t1 + 1;
    hi = past < 0 ? 0 : past < end ? past : end;
    lo = first < hi ? first : hi;
}

}  // namespace neo
