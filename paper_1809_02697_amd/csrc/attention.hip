// Causal attention of the newest tokens of each sequence over its paged int8
// cache:
//
//   out[i] = sum_j w_ij v_j / sum_j p_ij,   p_ij = exp(scale q_i.k_j - m_i)
//   k_j = ks_j K_j,  v_j = vs_j V_j  (K, V int8),  w_ij = p_ij vs_j
//
// in one pass over the cache with the running maximum m_i and sum of each row.
//
// The rows of a unit (a sequence and a key/value head) are its new tokens times
// the query heads that share the head: row = token * G + head.  Products run on
// fp16 MFMA with float32 sums.  int8 values are exact in fp16.  A query row is
// scaled by a power of two that puts its largest value in [2^14, 2^15), so
// float16 and bfloat16 queries are exact too (values 2^-28 of the largest and
// less lose bits); a float32 query is the sum of two fp16 terms.  A query with an
// infinity or a NaN gives NaN where it sees a key, and no other row.  The weights
// w_ij are scaled by 2^(14 - E), E the exponent of the largest vs that the row
// has seen so far, and rounded to fp16 (float16 and float32: two terms; Weights below).
//
// S^T = K Q^T and O^T = V^T P^T: the accumulator's layout of S^T (a lane holds
// four neighbouring keys of one row) is the layout of the second product's
// operand, so weights go from one product to the other in registers.
#include <atomic>
#include <type_traits>

#include "attention_keys.h"
#include "token_types.h"

namespace neo {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr float kLift = 14.f;  // weights are at most 2^15: the top of fp16's range
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMinusInf = -__builtin_inff();

constexpr int kLowestE = -64;

// Four rows' values of this lane's column: in each 16 lanes, lane i points at
// four neighbouring columns of row i / 4, and gets the four rows of column i.
__device__ inline h4 read_transposed(const _Float16* p) {
    return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p));
}

// ---- int8 to fp16 ------------------------------------------------------------------------
// A byte v + 128 (the sign bit flipped) under a zero byte is the fp16 number
// (v + 128) 2^-24; times 2^15, minus 2^-2, it is v 2^-9, exactly.
constexpr float kInt8Unit = 1.f / 512;
__device__ inline uint32_t biased(uint32_t w) { return w ^ 0x80808080u; }
__device__ inline h2 from_biased(uint32_t halves) {
    const h2 up = {(_Float16)32768.f, (_Float16)32768.f}, bias = {(_Float16)-0.25f, (_Float16)-0.25f};
    return __builtin_elementwise_fma(__builtin_bit_cast(h2, halves), up, bias);
}
// Four neighbouring bytes of one dword; one byte of each of two dwords.
__device__ inline void unpack4(uint32_t w, h2& lo, h2& hi) {
    lo = from_biased(__builtin_amdgcn_perm(0, w, 0x0c010c00u));
    hi = from_biased(__builtin_amdgcn_perm(0, w, 0x0c030c02u));
}
__device__ inline h2 pair(uint32_t a, uint32_t b, int t) {
    return from_biased(__builtin_amdgcn_perm(b, a, 0x0c000c00u | (uint32_t)(4 + t) << 16 | (uint32_t)t));
}
__device__ inline h8 join(h2 a, h2 b, h2 c, h2 d) {
    return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ inline int exponent(uint32_t bits) { return (int)(bits >> 23) - 127; }
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// How many fp16 terms a type's queries and weights are taken as.  float16 queries
// are exact in one, but one rounding of the weights would be as large as the
// output's own (error against 64 bits 1.4 times as much); bfloat16's is eight
// times larger.
//
// A term holds 11 bits from fp16's least normal number 2^-14 up, two terms 22
// from 2^-3 up (and at least 11 from 2^-14).  Smaller weights (of keys whose
// scores lie far below the row's largest) are taken apart and multiplied in
// bf16, which has float32's range, as two terms of 8 bits (float32: three), so
// that every weight keeps its bits: a position at which the largest keys'
// values are 0 is the sum of the small ones.
template <typename T>
struct Weights {
    static constexpr bool F32 = std::is_same<T, float>::value;
    static constexpr int QTERMS = F32 ? 2 : 1, TERMS = std::is_same<T, __bf16>::value ? 1 : 2, SMALL = F32 ? 3 : 2;
    static constexpr float least = F32 ? 0x1p-3f : 0x1p-14f;
    __device__ static void terms(const f32x8& v, h8 (&w)[TERMS]) {
        w[0] = __builtin_convertvector(v, h8);
        if constexpr (TERMS == 2) w[1] = __builtin_convertvector(v - __builtin_convertvector(w[0], f32x8), h8);
    }
    // The small ones among v as bf16 terms; v keeps the others.
    __device__ static void take_small(f32x8& v, b8 (&w)[SMALL]) {
        f32x8 rest;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool later = v[i] < least;  // (a NaN stays)
            rest[i] = later ? v[i] : 0.f;
            v[i] = later ? 0.f : v[i];
        }
#pragma unroll
        for (int t = 0; t < SMALL; ++t) {
            w[t] = __builtin_convertvector(rest, b8);
            rest -= __builtin_convertvector(w[t], f32x8);
        }
    }
};
__device__ inline b8 to_bf16(h8 v) { return __builtin_convertvector(__builtin_convertvector(v, f32x8), b8); }

// ---- a unit's tokens -----------------------------------------------------------------
struct Unit {
    int first, n, all, ctx, end;  // first row of q; new tokens computed, all of them; cached tokens, those read
};
__device__ inline Unit unit_of(const AttnArgs& a, int b) {
    Unit u;
    u.first = min(max(a.starts[b], 0), a.tokens);
    u.all = min(max(a.starts[b + 1], u.first), a.tokens) - u.first;
    u.n = min(u.all, a.max_chunk);
    u.ctx = max(a.contexts[b], 0);
    u.end = min(u.ctx, a.max_context);
    return u;
}

// ---- shares ---------------------------------------------------------------------------
// A unit of work is a row tile of a sequence's key/value head; its keys are
// counted in blocks of BLK from the first it sees, rounded down to 32.  The
// blocks of all units, in the order sequence, head, tile, are cut into equal
// shares, one a workgroup, however the lengths differ.  A unit that lies in
// one share is written at once; of one that is cut, each share leaves its part
// in the workspace (a share has at most two such: where it starts in the
// middle of a unit, and where it ends in one) and attention_join adds them.
struct Shares {
    int groups;  // workgroups; 0: one for each unit
    // key / page_size = key * page_mul >> page_shift for keys below 2^31
    uint32_t page_mul;
    int page_shift;
    __device__ int page(int key) const { return (int)((uint64_t)(uint32_t)key * page_mul >> page_shift); }
    // of W blocks: shares of two blocks at least, a multiple of the chip's 8 dies
    __device__ int used(int64_t W) const {
        const int64_t n = min((int64_t)groups, max((int64_t)1, W / 2));
        return (int)(n >= 8 ? n & ~7 : n);
    }
};
// A value that all lanes hold, in scalar registers.
__device__ inline int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ inline int64_t share_start(int64_t W, int used, int i) { return W * i / used; }

// Parts in the workspace: part 2 i of share i is the unit it starts in, 2 i + 1
// the one it ends in; o[part][row of the tile][head_dim] in true units relative
// to the part's maximum, ml[part][row] (maximum, sum).  starts[i]: where share i
// starts, for the join (W = 0: no such share).
struct Start {
    int64_t W;
    int b, h, tile, skip, blocks, unused;
};
struct Parts {
    float* o;
    float2* ml;
    Start* starts;
};

// Setting a unit up and joining its waves takes a workgroup about as long as
// this many blocks: they are counted as blocks in front of each unit's own.
constexpr int kUnitCost = 4;

template <int ROWS, int BLK>
struct Cursor {
    Unit u;
    int b, h, tile, rows, tiles;  // rows and tiles of sequence b
    int lo, hi, blocks;           // of the unit: its keys from lo (rounded) to hi
    int skip;                     // blocks of the unit that lie before the share

    __device__ static int tile_blocks(const AttnArgs& a, const Unit& u, int rows, int G, int tile, int& lo, int& hi) {
        seen_keys(u.ctx, u.all, u.end, tile * ROWS / G, (min(tile * ROWS + ROWS, rows) - 1) / G, a.window, lo, hi);
        lo &= ~31;
        return kUnitCost + max(1, (hi - lo + BLK - 1) / BLK);
    }
    // blocks of one head of sequence b
    __device__ static int64_t head_blocks(const AttnArgs& a, int G, int b) {
        const Unit u = unit_of(a, b);
        const int rows = u.n * G;
        int64_t n = 0;
        int lo, hi;
        for (int t = 0; t * ROWS < rows; ++t) n += tile_blocks(a, u, rows, G, t, lo, hi);
        return n;
    }
    __device__ void sequence(const AttnArgs& a, int G) {
        u = unit_of(a, b);
        rows = u.n * G;
        tiles = (rows + ROWS - 1) / ROWS;
    }
    __device__ void unit(const AttnArgs& a, int G) { blocks = tile_blocks(a, u, rows, G, tile, lo, hi); }
    __device__ void next(const AttnArgs& a, int G) {  // (there is a next one: the share goes on)
        skip = 0;
        if (++tile == tiles) {
            tile = 0;
            if (++h == a.c.kv_heads) {
                h = 0;
                do {
                    ++b;
                    sequence(a, G);
                } while (rows == 0 && b + 1 < a.seqs);
            }
        }
        unit(a, G);
    }

    // All threads of the workgroup: the sum W of all blocks, and with `find` the
    // unit that holds block find(W) (none if that is not below W).
    struct Scratch {
        int64_t wave[16], off;
        int b;
    };
    template <int THREADS, typename F>
    __device__ int64_t locate(const AttnArgs& a, int G, Scratch& lds, F&& find) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        auto scan = [&](int64_t n, int64_t& total) {  // exclusive, over the workgroup
            int64_t in = n;
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) {
                const int64_t v = __shfl_up(in, x, 64);
                if (lane >= x) in += v;
            }
            __syncthreads();
            if (lane == 63) lds.wave[wave] = in;
            __syncthreads();
            int64_t before = 0;
            total = 0;
            for (int w = 0; w < THREADS / 64; ++w) {
                if (w < wave) before += lds.wave[w];
                total += lds.wave[w];
            }
            total = uniform(total);
            return before + in - n;
        };
        const int H = a.c.kv_heads;
        int64_t W = 0, x = -1;
        for (int pass = 0; pass < 2; ++pass) {
            int64_t at = 0;
            for (int b0 = 0; b0 < a.seqs; b0 += THREADS) {
                const int64_t n = b0 + tid < a.seqs ? head_blocks(a, G, b0 + tid) * H : 0;
                int64_t total;
                const int64_t off = at + scan(n, total);
                at += total;
                if (a.seqs <= THREADS) W = at, x = find(W);  // (one round does both)
                if (x >= off && x < off + n) {
                    lds.b = b0 + tid;
                    lds.off = off;
                }
            }
            if (a.seqs <= THREADS) break;
            W = at;
            x = find(W);
        }
        __syncthreads();
        if (x < 0 || x >= W) return W;
        b = __builtin_amdgcn_readfirstlane(lds.b);
        sequence(a, G);
        int64_t rest = x - uniform(lds.off), each = 0;
        int l, e;
        for (int t = 0; t < tiles; ++t) each += tile_blocks(a, u, rows, G, t, l, e);
        each = uniform(each);
        h = __builtin_amdgcn_readfirstlane((int)(rest / each));
        rest -= (int64_t)h * each;
        for (tile = 0;; ++tile) {
            unit(a, G);
            if (rest < blocks) break;
            rest -= blocks;
        }
        tile = __builtin_amdgcn_readfirstlane(tile);
        unit(a, G);
        skip = __builtin_amdgcn_readfirstlane((int)rest);
        return W;
    }
};

// The workgroup's share: x of `end` blocks done, the cursor at the next unit.
template <int ROWS, int BLK, int THREADS>
struct Walk {
    Cursor<ROWS, BLK> c;
    int64_t x, end;
    int share;
    // The keys [first, last) of the unit that the share takes, as `take` blocks.
    int take, first, last;
    bool head, whole;  // it starts in the middle of the unit; it holds all of it
    __device__ void unit_keys() {
        take = (int)min((int64_t)(c.blocks - c.skip), end - x);
        head = c.skip > 0;
        whole = !head && take == c.blocks;
        first = c.lo + max(c.skip - kUnitCost, 0) * BLK;
        last = (int)min((int64_t)c.hi, c.lo + (int64_t)max(c.skip + take - kUnitCost, 0) * BLK);
    }
    __device__ bool next(const AttnArgs& a, int G) {
        x += take;
        if (x >= end) return false;
        c.next(a, G);
        return true;
    }
    __device__ bool begin(const AttnArgs& a, const Shares& sh, int G, const Parts& ws, typename Cursor<ROWS, BLK>::Scratch& lds) {
        c.skip = 0;
        if (sh.groups == 0) {
            // tiles from the last, which sees the most keys; heads fastest
            const int units = a.seqs * a.c.kv_heads, at = blockIdx.x / units, unit = blockIdx.x - at * units;
            c.b = unit / a.c.kv_heads;
            c.h = unit - c.b * a.c.kv_heads;
            c.sequence(a, G);
            c.tile = c.tiles - 1 - at;
            if (c.tile < 0) return false;
            c.unit(a, G);
            share = 0, x = 0, end = c.blocks;
            return true;
        }
        int used = 0;
        const int64_t W = c.template locate<THREADS>(a, G, lds, [&](int64_t W) {
            used = sh.used(W);
            if ((int)blockIdx.x >= used) return W;
            // neighbouring shares on one die, whose cache they share
            share = used >= 8 ? (int)(blockIdx.x % 8) * (used / 8) + (int)blockIdx.x / 8 : (int)blockIdx.x;
            return share_start(W, used, share);
        });
        if ((int)blockIdx.x >= used || W == 0) {
            if (threadIdx.x == 0) ws.starts[blockIdx.x].W = 0;
            return false;
        }
        x = uniform(share_start(W, used, share));
        end = uniform(share_start(W, used, share + 1));
        if (threadIdx.x == 0) ws.starts[share] = Start{W, c.b, c.h, c.tile, c.skip, c.blocks, 0};
        return x < end;
    }
};

template <typename T>
__device__ inline void store_row(const AttnArgs& a, const Unit& u, int h, int G, int row, int d, float v) {
    const int t = row / G, hq = h * G + row - t * G;
    static_cast<T*>(a.out)[(int64_t)(u.first + t) * a.ots + (int64_t)hq * a.ohs + d] = (T)v;
}

// ---- 16 rows a workgroup ------------------------------------------------------------
// Four waves take turns at blocks of 32 keys; the key and value bytes go from
// memory straight into registers (every byte is used once), the next block's
// while this one's are used, and the waves' results are joined in LDS.
// TILED: pages of whole 16 tokens, so a page is looked up once per 16 keys for
// the whole wave; other pages are looked up key by key.
//
// The cache, read once, bounds it: one token each of 32 sequences, 32 query
// heads on 8 of 128, contexts up to 32,000 (650 MB) 124 us, 5.2 TB/s, and 8 us
// to join.
constexpr int kRowsWaves = 4;

template <int DP>
struct KeyBlock {
    static constexpr int KB = DP / 4, VB = DP / 16;  // bytes of a key, of a value a lane holds
    u4 k[2][KB / 16];              // keys 16 t + li: bytes g * KB ...
    uint32_t v[2][4][VB / 4];      // values 16 t + 4 g + r: bytes li * VB ...
    v4f ks[2], vs[2];              // their scales
    uint32_t there;                // bit 4 t + r: the key's page exists
};

// The pages of a block's keys, looked up a block earlier than the bytes that
// they lead to.
template <bool TILED>
struct KeyPages {
    int k[2], v[2][TILED ? 1 : 4];
};
template <bool TILED>
__device__ inline void look_up(const Shares& sp, const int32_t* table, int kb, int hi, int li, int g, KeyPages<TILED>& to) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        to.k[t] = table[sp.page(min(kb + 16 * t + (TILED ? 0 : li), TILED ? (hi - 1) & ~15 : hi - 1))];
        if constexpr (!TILED)
#pragma unroll
            for (int r = 0; r < 4; ++r) to.v[t][r] = table[sp.page(min(kb + 16 * t + 4 * g + r, hi - 1))];
    }
}

// Every lane loads, and blocks past the last key load that key's: the number of
// loads under way is then known, and a block's use waits for its own loads
// only.  (Pieces past head_dim read the row's start: the query is 0 there, and
// such values are not stored.)
template <int DP, bool TILED>
__device__ inline void load_block(const AttnArgs& a, const Shares& sp, const KeyPages<TILED>& pages, int h, int kb, int hi,
                                  int li, int g, KeyBlock<DP>& to) {
    constexpr int KB = DP / 4, VB = DP / 16;
    const int H = a.c.kv_heads, D = a.c.head_dim, ps = a.c.page_size;
    int koff[KB / 16];
#pragma unroll
    for (int c = 0; c < KB / 16; ++c) koff[c] = g * KB + c * 16 < D ? g * KB + c * 16 : 0;
    const int voff = li * VB < D ? li * VB : 0;
    typedef float loose4 __attribute__((ext_vector_type(4), aligned(4)));
    to.there = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if constexpr (TILED) {
            // (entries past the last key lie in its page)
            const int key = min(kb + 16 * t, (hi - 1) & ~15), pg = sp.page(key), page = pages.k[t];
            const bool there = (uint32_t)page < (uint32_t)a.c.pages;
            to.there |= there ? 0xfu << (4 * t) : 0u;
            const uint64_t e = (uint64_t)(uint32_t)(there ? page : 0) * (uint32_t)(H * ps) + (uint32_t)(h * ps + key - pg * ps);
            const int8_t *k = a.c.k + e * D, *v = a.c.v + e * D;
            to.ks[t] = *reinterpret_cast<const loose4*>(a.c.k_scale + e + 4 * g);
            to.vs[t] = *reinterpret_cast<const loose4*>(a.c.v_scale + e + 4 * g);
#pragma unroll
            for (int c = 0; c < KB / 16; ++c) to.k[t][c] = *reinterpret_cast<const u4*>(k + li * D + koff[c]);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < VB / 4; ++c) to.v[t][r][c] = reinterpret_cast<const uint32_t*>(v + (4 * g + r) * D + voff)[c];
        } else {
            auto entry = [&](int j, int page, bool& there) {
                const int key = min(j, hi - 1), pg = sp.page(key);
                there = (uint32_t)page < (uint32_t)a.c.pages;
                return (uint64_t)(uint32_t)(there ? page : 0) * (uint32_t)(H * ps) + (uint32_t)(h * ps + key - pg * ps);
            };
            bool there;
            const int8_t* k = a.c.k + entry(kb + 16 * t + li, pages.k[t], there) * D;
#pragma unroll
            for (int c = 0; c < KB / 16; ++c) to.k[t][c] = *reinterpret_cast<const u4*>(k + koff[c]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint64_t e = entry(kb + 16 * t + 4 * g + r, pages.v[t][r], there);
                to.there |= there ? 1u << (4 * t + r) : 0u;
                to.ks[t][r] = a.c.k_scale[e];
                to.vs[t][r] = a.c.v_scale[e];
#pragma unroll
                for (int c = 0; c < VB / 4; ++c) to.v[t][r][c] = reinterpret_cast<const uint32_t*>(a.c.v + e * D + voff)[c];
            }
        }
    }
}

constexpr int kRowsBlock = kRowsWaves * 32;  // keys the workgroup takes at a time

template <typename T, int DP, bool TILED>
__global__ __launch_bounds__(kRowsWaves * 64, DP == 256 ? 1 : DP == 64 ? 3 : 2) void attention_rows(AttnArgs a, Shares sp, Parts ws) {
    typedef Weights<T> W;
    constexpr int KB = DP / 4, STEPS = DP / 32, VB = DP / 16;
    __shared__ float red_m[kRowsWaves][16], red_l[kRowsWaves][16], red_o[kRowsWaves][16][DP + 4];
    __shared__ typename Cursor<16, kRowsBlock>::Scratch scratch;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, g = lane >> 4;
    const int H = a.c.kv_heads, G = a.q_heads / H, D = a.c.head_dim;
    Walk<16, kRowsBlock, kRowsWaves * 64> walk;
    if (!walk.begin(a, sp, G, ws, scratch)) return;
    for (;;) {
        const Unit u = walk.c.u;
        const int h = walk.c.h, rows = walk.c.rows, row0 = walk.c.tile * 16, hi = walk.c.hi;
        walk.unit_keys();
        const int first = walk.first, last = walk.last;
        const int32_t* table = a.table + walk.c.b * a.table_stride;

        KeyBlock<DP> kv;
        int kb = first + wave * 32;
        KeyPages<TILED> pages;
        if (hi > 0) {
            look_up<TILED>(sp, table, kb, hi, li, g, pages);
            load_block<DP, TILED>(a, sp, pages, h, kb, hi, li, g, kv);
            look_up<TILED>(sp, table, kb + kRowsBlock, hi, li, g, pages);
        }

        // this lane's row of queries: values d = g * KB + ...
        const int row = min(row0 + li, rows - 1), tok = row / G, pos = u.ctx - u.all + tok;
        const int pos_lo = u.ctx - u.all + row0 / G, pos_hi = u.ctx - u.all + (min(row0 + 16, rows) - 1) / G;
        const int from_hi = first_seen(pos_hi, a.window);
        h8 q[W::QTERMS][STEPS];
        float fq;  // what a score is multiplied with
        {
            const T* src = static_cast<const T*>(a.q) + (int64_t)(u.first + tok) * a.qts + (int64_t)(h * G + row - tok * G) * a.qhs + g * KB;
            f32x8 v[STEPS];
            uint32_t top = 0;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const bool in = g * KB + s * 8 < D;
                v[s] = load8(in ? src + s * 8 : src - g * KB);
                if (!in) v[s] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, magnitude(v[s][i]));
            }
            top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
            top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
            const int e = top >= kInfBits ? 0 : min(14 - exponent(top), 126);
            const float up = ldexpf(1.f, e);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                v[s] *= up;
                q[0][s] = __builtin_convertvector(v[s], h8);
                if constexpr (W::QTERMS == 2) q[1][s] = __builtin_convertvector(v[s] - __builtin_convertvector(q[0][s], f32x8), h8);
            }
            fq = ldexpf(a.scale * kLog2e / kInt8Unit, -e);
            // (no score of a query with an infinity is finite: its softmax is undefined)
            if (top >= kInfBits) fq = __uint_as_float(0x7fc00000u);
        }

        v4f o[VB];
#pragma unroll
        for (int t = 0; t < VB; ++t) o[t] = v4f{0, 0, 0, 0};
        float m = kMinusInf, l = 0.f;
        int E = -127;  // exponent of the largest value scale seen so far

        while (kb < last) {
            const int kn = kb + kRowsBlock;
            KeyBlock<DP> next;
            load_block<DP, TILED>(a, sp, pages, h, kn, hi, li, g, next);
            look_up<TILED>(sp, table, kn + kRowsBlock, hi, li, g, pages);

            v4f s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < STEPS; ++c) {
                    h2 x[4];
                    unpack4(biased(kv.k[t][c / 2][c % 2 * 2]), x[0], x[1]);
                    unpack4(biased(kv.k[t][c / 2][c % 2 * 2 + 1]), x[2], x[3]);
                    const h8 k = join(x[0], x[1], x[2], x[3]);
#pragma unroll
                    for (int i = 0; i < W::QTERMS; ++i) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[i][c], s[t], 0, 0, 0);
                }
            }

            // (from_hi is 0 without a window; asked all the same, single tokens over up to
            // 32,000 take 128 us, and 139 else: the compiler orders the loop otherwise)
            const bool all = kb + 32 <= last && kb + 31 <= pos_lo && (!a.window || kb >= from_hi) &&
                             __all(kv.there == 0xff);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[t][r] *= kv.ks[t][r] * fq;
            if (!all) {
                // this lane's keys j0 + x: seen from x = from_x up to to_x (after
                // the scales, which may be NaN)
                const int j0 = kb + 4 * g, to_x = min(pos, last - 1) - j0, from_x = first_seen(pos, a.window) - j0;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int x = 16 * t + r;
                        const bool see = x <= to_x && x >= from_x && (kv.there >> (4 * t + r) & 1);
                        s[t][r] = see ? s[t][r] : kMinusInf;
                        kv.vs[t][r] = see ? kv.vs[t][r] : 0.f;
                    }
            }
            float top = kMinusInf;
            uint32_t vtop = 0;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    top = fmaxf(top, s[t][r]);
                    vtop = max(vtop, magnitude(kv.vs[t][r]));
                }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            vtop = max(vtop, (uint32_t)__shfl_xor((int)vtop, 16, 64));
            vtop = max(vtop, (uint32_t)__shfl_xor((int)vtop, 32, 64));
            const float mn = fmaxf(m, top), m0 = mn == kMinusInf ? 0.f : mn;
            const float lift = m0 - kLift;  // weights (and l) are 2^14 times p
            const int En = max(E, min(exponent(vtop), 126));
            if (__any(mn > m || En > E)) {
                const float f = exp2_fast(m - m0), fo = ldexpf(f, E - En);
                l *= f;
#pragma unroll
                for (int t = 0; t < VB; ++t) o[t] *= fo;
                m = mn;
                E = En;
            }
            f32x8 pv;
            bool small = false;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = exp2_fast(s[t][r] - lift);
                    l += p;
                    pv[4 * t + r] = p * ldexpf(kv.vs[t][r], -E);
                    small |= pv[4 * t + r] != 0.f && pv[4 * t + r] < W::least;
                }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int c = 0; c < VB / 4; ++c) kv.v[t][r][c] = biased(kv.v[t][r][c]);
            auto values = [&](int t) {
                const int c = t / 4, y = t % 4;
                return join(pair(kv.v[0][0][c], kv.v[0][1][c], y), pair(kv.v[0][2][c], kv.v[0][3][c], y),
                            pair(kv.v[1][0][c], kv.v[1][1][c], y), pair(kv.v[1][2][c], kv.v[1][3][c], y));
            };
            h8 w[W::TERMS];
            if (__any(small)) {
                b8 ws[W::SMALL];
                W::take_small(pv, ws);
#pragma unroll
                for (int t = 0; t < VB; ++t) {
                    const b8 v = to_bf16(values(t));
#pragma unroll
                    for (int i = 0; i < W::SMALL; ++i) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, ws[i], o[t], 0, 0, 0);
                }
                // (converted anew below: kept, the values would take registers from the common case)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int c = 0; c < VB / 4; ++c) asm volatile("" : "+v"(kv.v[i / 4][i % 4][c]));
            }
            W::terms(pv, w);
#pragma unroll
            for (int t = 0; t < VB; ++t) {
                const h8 v = values(t);
#pragma unroll
                for (int i = 0; i < W::TERMS; ++i) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[i], o[t], 0, 0, 0);
            }
            kv = next;
            kb = kn;
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        l *= 0x1p-14f;

        // the waves' parts: o[t][r] is value d = (4 g + r) * VB + t of row li
        if (g == 0) {
            red_m[wave][li] = m;
            red_l[wave][li] = l;
        }
        __syncthreads();
        if (row0 + li < rows) {
            float M = kMinusInf;
#pragma unroll
            for (int w = 0; w < kRowsWaves; ++w) M = fmaxf(M, red_m[w][li]);
            const float f = m == kMinusInf ? 0.f : ldexpf(exp2_fast(m - M), E - 14 + 9);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int t = 0; t < VB; t += 4)
                    *reinterpret_cast<v4f*>(&red_o[wave][li][(4 * g + r) * VB + t]) = v4f{o[t][r], o[t + 1][r], o[t + 2][r], o[t + 3][r]} * f;
        }
        __syncthreads();
        const int live = min(16, rows - row0);
        for (int x = threadIdx.x; x < live * DP; x += kRowsWaves * 64) {
            const int rr = x / DP, d = x - rr * DP, rw = row0 + rr;
            if (d >= D) continue;
            float M = kMinusInf, L = 0.f, v = 0.f;
#pragma unroll
            for (int w = 0; w < kRowsWaves; ++w) M = fmaxf(M, red_m[w][rr]);
#pragma unroll
            for (int w = 0; w < kRowsWaves; ++w) {
                L += red_m[w][rr] == kMinusInf ? red_l[w][rr] : red_l[w][rr] * exp2_fast(red_m[w][rr] - M);
                v += red_o[w][rr][d];
            }
            if (walk.whole) {
                store_row<T>(a, u, h, G, rw, d, L == 0.f ? 0.f : v / L);
            } else {
                const int64_t part = ((int64_t)walk.share * 2 + !walk.head) * 16 + rr;
                ws.o[part * D + d] = v;
                if (d == 0) ws.ml[part] = make_float2(M, L);
            }
        }
        if (!walk.next(a, G)) break;
        __syncthreads();  // (the parts in LDS are read)
    }
}

// ---- 32 rows a wave -------------------------------------------------------------------
// NW waves share tiles of KT keys: keys and values are converted to fp16 once
// per workgroup on their way into LDS (the next tile's bytes travel meanwhile),
// and each wave multiplies its 32 rows with them on 32x32x16 products.  Values
// lie in LDS as they came and are read transposed.
//
// The softmax's arithmetic and the products bound it, one after the other more
// than side by side: of the cycles the vector unit works 58 %, the matrix unit
// 37 % and LDS 38 %.  2048 tokens at 32,768, 32 query heads on 8 of 128 in
// bfloat16 take 1.29 ms, 823 TFLOP/s (float16, whose weights are two terms, 28 %
// more; float32, whose queries are too, 57 %).  Scores ten times as far apart, so
// that most tiles hold small weights, take 2.24 ms.  32 rows a wave rather than
// 16 halve the reads of keys and values (16 rows: 1.63 ms); eight waves share a
// tile because each then converts an eighth of it (two workgroups of four
// waves a CU: 1.54 ms).
template <int DP, int NW>
struct TileShape {
    static constexpr int KT = DP == 256 ? 32 : 64, THREADS = NW * 64, ROWS = NW * 32;
    static constexpr int CH = DP / 16, CHUNKS = KT * CH, LOADS = (CHUNKS + THREADS - 1) / THREADS;
    static constexpr int KSTRIDE = DP, VSTRIDE = DP + 32;  // halves; the value rows' 64 spare bytes spread their banks
    struct alignas(512) Buffer {  // (a key row's pieces are exchanged within 256 bytes by xor)
        _Float16 k[KT * KSTRIDE], v[KT * VSTRIDE];
        float ks[KT], vs[KT];
        unsigned long long hidden;  // tokens in pages outside the cache
        int top;                    // exponent of the largest value scale
    };
    static constexpr int BYTES = 2 * sizeof(Buffer);
    // A key row's 16-byte pieces are exchanged by xor with turn(key), so that 16
    // keys, which LDS reads at once, lie in all banks (rows of 128 bytes: two a turn).
    __device__ static int turn(int key) { return CH * 2 < 16 ? key >> 1 & 7 : key & 15; }
};

template <typename T, int DP, int NW>
__global__ __launch_bounds__(NW * 64) void attention_tile(AttnArgs a, Shares sp, Parts ws) {
    typedef TileShape<DP, NW> C;
    typedef Weights<T> W;
    constexpr int KT = C::KT, SUB = KT / 32, STEPS = DP / 16, DT = DP / 32;
    typedef typename C::Buffer Buffer;
    extern __shared__ __align__(512) char lds[];
    Buffer* buf = reinterpret_cast<Buffer*>(lds);

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 31, half = lane >> 5;
    const int H = a.c.kv_heads, G = a.q_heads / H, D = a.c.head_dim, ps = a.c.page_size;
    Walk<C::ROWS, KT, C::THREADS> walk;
    if (!walk.begin(a, sp, G, ws, *reinterpret_cast<typename Cursor<C::ROWS, KT>::Scratch*>(lds))) return;
    __syncthreads();  // (the scratch lies where the tiles will)
    for (;;) {
        const Unit u = walk.c.u;
        const int h = walk.c.h, rows = walk.c.rows, row0 = walk.c.tile * C::ROWS, hi = walk.c.hi;
        walk.unit_keys();
        const int first = walk.first, last = walk.last;

        // this lane's row of queries; the positions of its wave's rows
        const int wrow = row0 + wave * 32, row = wrow + li;
        const bool live = row < rows;
        const int tok = min(row, rows - 1) / G, pos = u.ctx - u.all + tok;
        const int pos_lo = u.ctx - u.all + min(wrow, rows - 1) / G, pos_hi = u.ctx - u.all + min(wrow + 31, rows - 1) / G;
        const int from_lo = first_seen(pos_lo, a.window), from_hi = first_seen(pos_hi, a.window);
        h8 q[W::QTERMS][STEPS];
        float fq;
        bool undefined;  // (a query with an infinity has no finite score)
        {
            const int hq = h * G + min(row, rows - 1) - tok * G;
            const T* src = static_cast<const T*>(a.q) + (int64_t)(u.first + tok) * a.qts + (int64_t)hq * a.qhs + half * 8;
            uint32_t top = 0;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                if (s * 16 >= D) continue;
                const f32x8 v = load8(src + s * 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, magnitude(v[i]));
            }
            top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
            const int e = top >= kInfBits ? 0 : min(14 - exponent(top), 126);
            const float up = ldexpf(1.f, e);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                // (a query with an infinity is taken as zeros, and its sum made NaN at the end:
                // no score of it is the minus infinity of a masked key)
                const f32x8 v = (s * 16 < D && top < kInfBits ? load8(src + s * 16) : f32x8{0, 0, 0, 0, 0, 0, 0, 0}) * up;
                q[0][s] = __builtin_convertvector(v, h8);
                if constexpr (W::QTERMS == 2) q[1][s] = __builtin_convertvector(v - __builtin_convertvector(q[0][s], f32x8), h8);
            }
            // (positive, so that minus infinity stays that)
            fq = fmaxf(ldexpf(a.scale * kLog2e / kInt8Unit, -e), 0x1p-126f);
            undefined = top >= kInfBits;
        }

        // the tiles' way into LDS: 16 bytes of a key and of a value a thread and load
        const int32_t* table = a.table + walk.c.b * a.table_stride;
        int pg[C::LOADS], spg = 0;
        u4 kr[C::LOADS], vr[C::LOADS];
        float ksr = 0.f, vsr = 0.f;
        bool hid = false;
        // (every thread loads, tiles past the last key load that key's, and pieces
        // past head_dim the row's start: see load_block)
        auto lookup = [&](int k0) {
#pragma unroll
            for (int i = 0; i < C::LOADS; ++i) pg[i] = table[sp.page(min(k0 + (tid + i * C::THREADS) / C::CH, hi - 1))];
            spg = table[sp.page(min(k0 + tid % KT, hi - 1))];
        };
        auto fetch = [&](int k0) {
#pragma unroll
            for (int i = 0; i < C::LOADS; ++i) {
                const int x = tid + i * C::THREADS, c = x % C::CH, key = min(k0 + x / C::CH, hi - 1);
                const int page = (uint32_t)pg[i] < (uint32_t)a.c.pages ? pg[i] : 0;
                const uint64_t e = (uint64_t)(uint32_t)page * (uint32_t)(H * ps * D) +
                                   (uint32_t)((h * ps + key - sp.page(key) * ps) * D + (c * 16 < D ? c * 16 : 0));
                kr[i] = *reinterpret_cast<const u4*>(a.c.k + e);
                vr[i] = *reinterpret_cast<const u4*>(a.c.v + e);
            }
            const int key = min(k0 + tid % KT, hi - 1);
            hid = (uint32_t)spg >= (uint32_t)a.c.pages;
            const uint64_t e = (uint64_t)(uint32_t)(hid ? 0 : spg) * (uint32_t)(H * ps) + (uint32_t)(h * ps + key - sp.page(key) * ps);
            ksr = a.c.k_scale[e];
            vsr = a.c.v_scale[e];
        };
        auto store = [&](Buffer& to) {
#pragma unroll
            for (int i = 0; i < C::LOADS; ++i) {
                const int x = tid + i * C::THREADS, c = x % C::CH, key = x / C::CH;
                if (C::CHUNKS % C::THREADS && x >= C::CHUNKS) break;
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    h2 x0, x1, x2, x3;
                    unpack4(biased(kr[i][2 * o]), x0, x1);
                    unpack4(biased(kr[i][2 * o + 1]), x2, x3);
                    *reinterpret_cast<h8*>(to.k + key * C::KSTRIDE + ((2 * c + o) ^ C::turn(key)) * 8) = join(x0, x1, x2, x3);
                }
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    h2 x0, x1, x2, x3;
                    unpack4(biased(vr[i][2 * o]), x0, x1);
                    unpack4(biased(vr[i][2 * o + 1]), x2, x3);
                    *reinterpret_cast<h8*>(to.v + key * C::VSTRIDE + (2 * c + o) * 8) = join(x0, x1, x2, x3);
                }
            }
            if (wave == 0) {  // (the KT scales lie in its lanes)
                const uint32_t top = lanes_max(lane < KT && !hid ? magnitude(vsr) : 0u);
                const unsigned long long bad = __ballot(lane < KT && hid);
                if (lane < KT) {
                    to.ks[lane] = ksr;
                    to.vs[lane] = vsr;
                }
                if (lane == 0) {
                    to.hidden = bad;
                    to.top = exponent(top);
                }
            }
        };

        f32x16 o[DT];
#pragma unroll
        for (int t = 0; t < DT; ++t) o[t] = f32x16{0};
        float m = kMinusInf, l = 0.f;  // the running maximum is of scores / fq
        int E = kLowestE;

        auto compute = [&](const Buffer& from, int k0) {
            f32x16 s[SUB];
            // byte address of this lane's piece 0 of key li; piece c is that xor 32 c
            uint32_t kaddr = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)reinterpret_cast<const char*>(from.k) +
                             li * (2 * C::KSTRIDE) + ((half ^ C::turn(li)) * 16);
            asm volatile("" : "+v"(kaddr));  // (kept in one register, not in one for every c)
#pragma unroll
            for (int t = 0; t < SUB; ++t) s[t] = f32x16{0};
            h8 kf[3][SUB];  // keys are read two steps ahead of their products
            auto read = [&](int c) {
#pragma unroll
                for (int t = 0; t < SUB; ++t) kf[c % 3][t] = *(__attribute__((address_space(3))) const h8*)(uintptr_t)((kaddr ^ (c * 32)) + t * 32 * (2 * C::KSTRIDE));
            };
            read(0);
            read(1);
#pragma unroll
            for (int c = 0; c < STEPS; ++c) {
                if (c + 2 < STEPS) read(c + 2);
                __builtin_amdgcn_sched_barrier(0);  // (left alone, the compiler puts each read right before its use)
#pragma unroll
                for (int t = 0; t < SUB; ++t)
#pragma unroll
                    for (int i = 0; i < W::QTERMS; ++i) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[c % 3][t], q[i][c], s[t], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_sched_barrier(0);
            const uint64_t hidden = (uint64_t)uniform((int64_t)from.hidden);
            const bool all = k0 + KT - 1 <= pos_lo && k0 + KT <= last && hidden == 0 && k0 >= from_hi;
            auto scales = [&](const float* p, int t, int g) { return *reinterpret_cast<const v4f*>(p + 32 * t + 8 * g + 4 * half); };
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const v4f ks = scales(from.ks, t, g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[t][4 * g + i] *= ks[i];
                }
            int En = max(E, __builtin_amdgcn_readfirstlane(min(from.top, 126)));
            if (!all) {
                // this lane's keys k0 + 4 half + x: seen from x = from_x up to to_x
                const int j0 = k0 + 4 * half, to_x = live ? min(pos, last - 1) - j0 : -1;
                const int from_x = first_seen(pos, a.window) - j0;
                uint32_t vtop = 0;
#pragma unroll
                for (int t = 0; t < SUB; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const v4f vs = scales(from.vs, t, g);
                        const uint32_t hid8 = (uint32_t)(hidden >> (32 * t + 8 * g)) >> (4 * half);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int x = 32 * t + 8 * g + i;
                            const bool see = x <= to_x && x >= from_x && !(hid8 >> i & 1);
                            s[t][4 * g + i] = see ? s[t][4 * g + i] : kMinusInf;
                            vtop = max(vtop, see ? magnitude(vs[i]) : 0u);
                        }
                    }
                vtop = max(vtop, (uint32_t)__shfl_xor((int)vtop, 32, 64));
                En = max(E, min(exponent(vtop), 126));
            }
            float top = kMinusInf;
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float mn = fmaxf(m, top), m0 = mn == kMinusInf ? 0.f : mn;
            if (__any(mn > m || En > E)) {
                const float f = ldexpf(exp2_fast((m - m0) * fq), E - En);
                l *= f;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] *= f;
                m = mn;
                E = En;
            }
            const float lift = m0 * fq - kLift + (float)E;  // weights and l are 2^(14 - E) times p
            float least = 1.f;
            auto weigh = [&](auto whole) {
#pragma unroll
                for (int t = 0; t < SUB; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const v4f vs = scales(from.vs, t, g);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = s[t][4 * g + i];
                            const float p = exp2_fast(x * fq - lift);
                            l += p;
                            // (the scale of an entry that is not seen may be a NaN)
                            s[t][4 * g + i] = p * (whole.value || x != kMinusInf ? vs[i] : 0.f);
                            least = fminf(least, s[t][4 * g + i]);
                        }
                    }
            };
            if (all)
                weigh(std::true_type{});
            else
                weigh(std::false_type{});
            auto values = [&](int t, int x, int d) {
                // rows 32 t + 16 x + 8 {0, 1} + 4 half + 0..3, columns 32 d + 0..31, transposed
                const _Float16* p = from.v + (32 * t + 16 * x + 4 * half + (lane & 15) / 4) * C::VSTRIDE + 32 * d + (lane & 16) + (lane & 3) * 4;
                const h4 y0 = read_transposed(p), y1 = read_transposed(p + 8 * C::VSTRIDE);
                return h8{y0[0], y0[1], y0[2], y0[3], y1[0], y1[1], y1[2], y1[3]};
            };
            if (__any(least < W::least)) {
#pragma unroll
                for (int t = 0; t < SUB; ++t)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        f32x8 pv;
#pragma unroll
                        for (int i = 0; i < 8; ++i) pv[i] = s[t][8 * x + i];
                        b8 w[W::SMALL];
                        W::take_small(pv, w);
#pragma unroll
                        for (int i = 0; i < 8; ++i) s[t][8 * x + i] = pv[i];
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            const b8 v = to_bf16(values(t, x, d));
#pragma unroll
                            for (int i = 0; i < W::SMALL; ++i) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[i], o[d], 0, 0, 0);
                            asm volatile("" ::: "memory");  // (the values are read again below: kept, they would take its registers)
                        }
                    }
            }
            h8 vf[3];  // values, two products ahead
            vf[0] = values(0, 0, 0);
            vf[1] = values(0, 0, 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    f32x8 pv;
#pragma unroll
                    for (int i = 0; i < 8; ++i) pv[i] = s[t][8 * x + i];
                    h8 w[W::TERMS];
                    W::terms(pv, w);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const int n = (t * 2 + x) * DT + d, n2 = n + 2;
                        if (n2 < SUB * 2 * DT) vf[n2 % 3] = values(n2 / DT / 2, n2 / DT % 2, n2 % DT);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int i = 0; i < W::TERMS; ++i) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[n % 3], w[i], o[d], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
        };

        if (first < last) {
            lookup(first);
            fetch(first);
            lookup(first + KT);
            store(buf[0]);
            fetch(first + KT);
            __syncthreads();
            int at_buf = 0;
            for (int k0 = first; k0 < last; k0 += KT) {
                lookup(k0 + 2 * KT);
                if (wrow < rows && k0 <= pos_hi && k0 + KT > from_lo) compute(buf[at_buf], k0);
                store(buf[at_buf ^ 1]);
                fetch(k0 + 2 * KT);
                __syncthreads();
                at_buf ^= 1;
            }
        }
        l += __shfl_xor(l, 32, 64);
        if (undefined && l != 0.f) l = __uint_as_float(0x7fc00000u);  // (it saw a key)
        if (live && walk.whole) {
            const float f = l == 0.f ? 0.f : 512.f / l;
            const int hq = h * G + row - tok * G;
            T* out = static_cast<T*>(a.out) + (int64_t)(u.first + tok) * a.ots + (int64_t)hq * a.ohs + 4 * half;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (32 * d + 8 * g >= D) continue;
                    store4(out + 32 * d + 8 * g, v4f{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]} * f);
                }
        } else if (live) {
            const int64_t part = ((int64_t)walk.share * 2 + !walk.head) * C::ROWS + wave * 32 + li;
            float* out = ws.o + part * D + 4 * half;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (32 * d + 8 * g >= D) continue;
                    v4f v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = ldexpf(o[d][4 * g + i], E - 14 + 9);
                    *reinterpret_cast<v4f*>(out + 32 * d + 8 * g) = v;
                }
            if (half == 0) ws.ml[part] = make_float2(m == kMinusInf ? kMinusInf : m * fq, ldexpf(l, E - 14));
        }
        if (!walk.next(a, G)) break;
    }  // (the tiles' last barrier lies behind every read of LDS)
}

// The parts of the unit in which share j starts, if it is the first to start in
// it: workgroup (j - 1, y) joins ROUNDS times four rows of the tile, a wave a
// row, or with WAVES = 4 row y, its waves taking the parts in turn.
template <typename T, int ROWS, int WAVES, int ROUNDS>
__global__ __launch_bounds__(256) void attention_join(AttnArgs a, Shares sh, Parts ws) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, turn = wave % WAVES;
    const int G = a.q_heads / a.c.kv_heads, D = a.c.head_dim, j = blockIdx.x + 1;
    const Start at = ws.starts[j];
    if (at.W == 0 || at.skip == 0) return;
    const int64_t W = at.W;
    const int used = sh.used(W);
    const int64_t x0 = share_start(W, used, j) - at.skip;
    if (x0 < share_start(W, used, j - 1)) return;
    // parts: the end of share j - 1, the starts of shares j .. j + count - 2
    int count = 2;
    while (j + count - 1 < used && share_start(W, used, j + count - 1) < x0 + at.blocks) ++count;
    const Unit u = unit_of(a, at.b);
    static_assert(WAVES == 1 || ROUNDS == 1, "");
#pragma unroll 1
    for (int round = 0; round < ROUNDS; ++round) {
        const int rr = (blockIdx.y * ROUNDS + round) * (4 / WAVES) + wave / WAVES, row = at.tile * ROWS + rr;
        if (row >= u.n * G) return;  // (with four waves a row: all of them)
        auto part = [&](int i) { return ((int64_t)(j - 1 + i) * 2 + (i == 0)) * ROWS + rr; };
        float M = kMinusInf, L = 0.f;
        for (int i = lane; i < count; i += 64) M = fmaxf(M, ws.ml[part(i)].x);
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor(M, x, 64));
        auto factor = [&](float m) { return m == kMinusInf ? 1.f : exp2_fast(m - M); };  // (a part that saw nothing, or a NaN)
        for (int i = lane; i < count; i += 64) L += ws.ml[part(i)].y * factor(ws.ml[part(i)].x);
        L = lanes_sum(L);
        float v[4] = {0, 0, 0, 0};
        for (int i0 = 0; i0 < count; i0 += 64 * WAVES) {
            const int mine = i0 + lane * WAVES + turn;  // this lane's part
            const float f = mine < count ? factor(ws.ml[part(mine)].x) : 0.f;
            const int parts = min(64, (count - i0 - turn + WAVES - 1) / WAVES);
            for (int i = 0; i < parts; i += 4) {  // (past the last: the last, not added)
                float w[4][4];
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        w[y][x] = ws.o[part(i0 + min(i + y, parts - 1) * WAVES + turn) * D + min(lane + 64 * x, D - 1)];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float fi = __shfl(f, min(i + y, 63), 64);
#pragma unroll
                    for (int x = 0; x < 4; ++x) v[x] += i + y < parts ? w[y][x] * fi : 0.f;
                }
            }
        }
        if constexpr (WAVES > 1) {
            __shared__ float red[WAVES][256];
#pragma unroll
            for (int x = 0; x < 4; ++x) red[turn][lane + 64 * x] = v[x];
            __syncthreads();
            if (turn) return;
#pragma unroll
            for (int w = 1; w < WAVES; ++w)
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] += red[w][lane + 64 * x];
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (lane + 64 * x < D) store_row<T>(a, u, at.h, G, row, lane + 64 * x, L == 0.f ? 0.f : v[x] / L);
    }
}

// Rows a workgroup takes.  Up to two tiles of 16 go to the kernel for few rows
// (8 tokens of 4 heads a unit, 8 sequences of 8192: 61 us against 79 in tiles of
// 64); the tiles grow with the rows that the longest chunk has.  (A sequence of one
// token beside a chunk takes a whole such tile: 512 tokens and 31 single ones over
// 8192 take 407 us in one call, 125 and 112 in two.)
int tile_rows(const AttnArgs& a) {
    const int64_t rows = (int64_t)a.max_chunk * (a.q_heads / a.c.kv_heads);
    if (rows <= 32) return 16;
    if (rows <= 64) return 64;
    if (rows <= 128 || a.c.head_dim > 128) return 128;
    return 256;
}

// As many shares as the chip holds workgroups at a time.  Short units are not
// worth cutting, as a join is a launch of its own: seven float32 tokens of 3
// heads a unit over 700 tokens take 14 us whole and 20 us cut; one token of one
// head over 300 keys 12 and 17, over 1000 (eight blocks in one workgroup) 16.0 and
// 16.8; 4 tokens of 8 heads over 1000 16.1 and 15.9, 32 of them 20 and 29; 40
// tokens over 600 in the tile kernel 29 us cut and 42 whole.
Shares choose_shares(const AttnArgs& a) {
    const int tile = tile_rows(a), G = a.q_heads / a.c.kv_heads;
    int64_t range = a.max_context;
    if (a.window) range = std::min<int64_t>(range, (int64_t)a.window + (tile + G - 1) / G + 33);
    const int64_t units = ((int64_t)a.max_chunk * G + tile - 1) / tile * a.seqs * a.c.kv_heads;
    Shares sh;
    if (range <= (tile == 16 ? 1024 : 256) && units <= 1 << 22)  // (2^32 threads a launch)
        sh.groups = 0;
    else if (tile == 16)
        sh.groups = a.c.head_dim <= 64 ? 768 : a.c.head_dim <= 128 ? 512 : 256;
    else
        sh.groups = tile == 64 ? 512 : 256;
    const int log = ilog2(a.c.page_size);
    sh.page_mul = (uint32_t)((1ull << (31 + log)) / (uint32_t)a.c.page_size + 1);
    sh.page_shift = 31 + log;
    return sh;
}

int64_t part_rows(const AttnArgs& a, const Shares& sh) { return (int64_t)sh.groups * 2 * tile_rows(a); }

template <typename T, int DP, int NW>
hipError_t launch_tile(const AttnArgs& a, const Shares& sh, const Parts& p, unsigned blocks, hipStream_t st) {
    typedef TileShape<DP, NW> C;
    // (more LDS than a kernel gets unasked; set once per device)
    static std::atomic<uint64_t> asked{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !(asked.load() >> dev & 1)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&attention_tile<T, DP, NW>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
        if (e != hipSuccess) return e;
        if (dev >= 0 && dev < 64) asked.fetch_or(1ull << dev);
    }
    hipLaunchKernelGGL((attention_tile<T, DP, NW>), dim3(blocks), dim3(NW * 64), C::BYTES, st, a, sh, p);
    e = hipGetLastError();
    if (e != hipSuccess || sh.groups < 2) return e;
    hipLaunchKernelGGL((attention_join<T, C::ROWS, 1, 4>), dim3(sh.groups - 1, C::ROWS / 16), dim3(256), 0, st, a, sh, p);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_d(const AttnArgs& a, float* ws, hipStream_t st) {
    const Shares sh = choose_shares(a);
    const int G = a.q_heads / a.c.kv_heads, tile = tile_rows(a);
    const int64_t n = part_rows(a, sh);
    const Parts p{ws, reinterpret_cast<float2*>(ws + n * a.c.head_dim), reinterpret_cast<Start*>(ws + n * (a.c.head_dim + 2))};
    const int64_t units = (((int64_t)a.max_chunk * G + tile - 1) / tile) * a.seqs * a.c.kv_heads;
    const unsigned blocks = (unsigned)(sh.groups ? sh.groups : units);
    if (tile == 64) return launch_tile<T, DP, 2>(a, sh, p, blocks, st);
    if (tile == 128) return launch_tile<T, DP, 4>(a, sh, p, blocks, st);
    if constexpr (DP <= 128)
        if (tile == 256) return launch_tile<T, DP, 8>(a, sh, p, blocks, st);
    if (a.c.page_size % 16 == 0)
        hipLaunchKernelGGL((attention_rows<T, DP, true>), dim3(blocks), dim3(kRowsWaves * 64), 0, st, a, sh, p);
    else
        hipLaunchKernelGGL((attention_rows<T, DP, false>), dim3(blocks), dim3(kRowsWaves * 64), 0, st, a, sh, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || sh.groups < 2) return e;
    hipLaunchKernelGGL((attention_join<T, 16, 4, 1>), dim3(sh.groups - 1, std::min(16, a.max_chunk * G)), dim3(256), 0, st, a, sh, p);
    return hipGetLastError();
}

template <typename T>
hipError_t by_dim(const AttnArgs& a, float* ws, hipStream_t st) {
    if (a.c.head_dim <= 64) return launch_d<T, 64>(a, ws, st);
    if (a.c.head_dim <= 128) return launch_d<T, 128>(a, ws, st);
    return launch_d<T, 256>(a, ws, st);
}

}  // namespace

size_t attention_workspace(int, const AttnArgs& a) {
    const Shares sh = choose_shares(a);
    return part_rows(a, sh) * (a.c.head_dim + 2) * sizeof(float) + sh.groups * sizeof(Start);
}

hipError_t launch_attention(int dtype, const AttnArgs& a, float* ws, hipStream_t st) {
    if (dtype == NEO_F32) return by_dim<float>(a, ws, st);
    if (dtype == NEO_F16) return by_dim<_Float16>(a, ws, st);
    return by_dim<__bf16>(a, ws, st);
}

}  // namespace neo
