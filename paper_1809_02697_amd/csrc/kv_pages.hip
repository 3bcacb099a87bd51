// Pages of the paged int8 cache, in every layer's cache at once: copied (a
// sequence forks, or pages move together), and closed up (tokens of a sequence
// are dropped).  Both move each byte once, bytes and scales as they are.
#include "token_types.h"

namespace neo {
namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// ---- copies -----------------------------------------------------------------------------
// A page's keys (or values) in one layer are kv_heads stretches of page_size
// entries, of which the first `n` are copied; whole pages are one stretch.  Pieces of
// 16 bytes, four a thread, all loaded before the first is stored.  Nothing is read
// again soon, so the stores (and where whole pages move, the loads) pass the caches
// by: 256 pages of 64 tokens, 8 heads of 128, 16 layers (1.1 GB) 211 us (5.2 TB/s; 222
// without); 256 pairs' first entries of pages of 64 79 (84 without, and 136 with
// loads that do so too).
constexpr int kDepth = 4, kChunk = 256 * kDepth;

template <bool WHOLE>
__global__ __launch_bounds__(256) void kv_copy(CopyArgs a, int chunks, int64_t work) {
    const neo_kv_cache& c = a.c;
    const uint32_t each = (uint32_t)c.head_dim / 16, page = (uint32_t)(c.kv_heads * c.page_size);
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int64_t q = w / chunks;
        const int chunk = (int)(w - q * chunks), of = (int)(q % (2 * a.layers)), pair = (int)(q / (2 * a.layers));
        const int src = a.src[pair], dst = a.dst[pair];
        if ((uint32_t)src >= (uint32_t)c.pages || (uint32_t)dst >= (uint32_t)c.pages || src == dst) continue;
        const int64_t layer = (of >> 1) * a.layer_stride, from = layer + (int64_t)src * page, to = layer + (int64_t)dst * page;
        int8_t* data = of & 1 ? c.v : c.k;
        float* scales = of & 1 ? c.v_scale : c.k_scale;
        const uint32_t start = (uint32_t)chunk * kChunk;
        u4 v[kDepth];
        if constexpr (WHOLE) {
            const uint32_t pieces = page * each, end = min(start + kChunk, pieces);
            const u4* x = reinterpret_cast<const u4*>(data + from * c.head_dim);
            u4* y = reinterpret_cast<u4*>(data + to * c.head_dim);
#pragma unroll
            for (int i = 0; i < kDepth; ++i)
                if (start + i * 256 + threadIdx.x < end) v[i] = __builtin_nontemporal_load(x + start + i * 256 + threadIdx.x);
            // (the scales of the entries that start in the chunk)
            for (uint32_t e = (start + each - 1) / each + threadIdx.x; e < (end + each - 1) / each; e += 256) scales[to + e] = scales[from + e];
#pragma unroll
            for (int i = 0; i < kDepth; ++i)
                if (start + i * 256 + threadIdx.x < end) __builtin_nontemporal_store(v[i], y + start + i * 256 + threadIdx.x);
        } else {
            const uint32_t row = (uint32_t)min(max(a.entries[pair], 0), c.page_size) * each, pieces = row * (uint32_t)c.kv_heads;
            if (start >= pieces) continue;
            float s[kDepth];
            uint32_t entry[kDepth], piece[kDepth];
#pragma unroll
            for (int i = 0; i < kDepth; ++i) {
                const uint32_t x = start + i * 256 + threadIdx.x, h = x / row, y = x - h * row, o = y / each;
                entry[i] = x < pieces ? h * (uint32_t)c.page_size + o : 0xffffffffu;
                piece[i] = y - o * each;
                if (x >= pieces) continue;
                v[i] = *reinterpret_cast<const u4*>(data + (from + entry[i]) * c.head_dim + piece[i] * 16);
                if (piece[i] == 0) s[i] = scales[from + entry[i]];
            }
#pragma unroll
            for (int i = 0; i < kDepth; ++i) {
                if (entry[i] == 0xffffffffu) continue;
                __builtin_nontemporal_store(v[i], reinterpret_cast<u4*>(data + (to + entry[i]) * c.head_dim + piece[i] * 16));
                if (piece[i] == 0) scales[to + entry[i]] = s[i];
            }
        }
    }
}

// ---- closing up --------------------------------------------------------------------------
// Token base + i of a sequence becomes what token keep[i] >= base + i was.  A
// workgroup takes a head (or a part of its entries) of a sequence's keys (or
// values) in one layer, and its tokens in order, a chunk at a time: what later chunks
// read lies behind what this one writes, so only a chunk's own loads have to be
// back, in every wave, before the first of its stores.  Four waves move bytes, the
// next chunk's on their way while one is stored; a fifth looks up where the
// tokens of the chunk after that lie.
// (4 sequences of 6000 kept tokens of up to 12,064, 8 layers of 8 heads of 128: the
// call 157 to 172 us, the kernel 159 under the profiler, 5.1 TB/s; the call 178 with stores
// that stay in the caches, 370 with a chunk's loads waited for before the next one's.)
constexpr int kMovers = 256, kTokensMax = 256;

struct Lines {  // entries of head 0, of a chunk's tokens; to < 0: nothing moves
    int64_t from[kTokensMax], to[kTokensMax];
};
struct Moved {
    u4 v[kDepth];
    float s[kDepth];
    int64_t to[kDepth];
};

// Sequences that keep no more tokens than a chunk holds: every lane looks its own up
// (32 sequences of up to 8 proposed tokens, 16 layers: 7.0 us, 12 in chunks).
__global__ __launch_bounds__(kMovers) void kv_close_up_few(CompactArgs a, int heads, int tokens, int64_t work) {
    const neo_kv_cache& c = a.c;
    const int parts = (c.kv_heads + heads - 1) / heads;
    const uint32_t each = (uint32_t)c.head_dim / 16;
    const int64_t limit = a.table_pages * c.page_size;
    for (int64_t at = blockIdx.x; at < work; at += gridDim.x) {
        const int64_t q = at / parts;
        const int part = (int)(at - q * parts), of = (int)(q % (2 * a.layers)), b = (int)(q / (2 * a.layers));
        const int64_t layer = (of >> 1) * a.layer_stride;
        int8_t* data = (of & 1 ? c.v : c.k) + layer * c.head_dim;
        float* scales = (of & 1 ? c.v_scale : c.k_scale) + layer;
        const int first = min(max(a.starts[b], 0), a.kept), count = min(min(max(a.starts[b + 1], first), a.kept) - first, a.max_keep);
        const int base = a.bases[b];
        const int32_t* table = a.table + (int64_t)b * a.table_stride;
        u4 v[kDepth];
        float s[kDepth];
        int64_t to[kDepth];
        uint32_t byte[kDepth];
#pragma unroll
        for (int x = 0; x < kDepth; ++x) {
            const uint32_t idx = x * kMovers + threadIdx.x, row = idx / each, hh = row / (uint32_t)tokens;
            const int i = (int)(row - hh * (uint32_t)tokens), h = part * heads + (int)hh;
            byte[x] = (idx - row * each) * 16;
            to[x] = -1;
            if ((int)hh >= heads || h >= c.kv_heads || i >= count || base < 0) continue;
            const int64_t kept = a.keep[first + i], t = (int64_t)base + i;
            if (kept <= t || kept >= limit) continue;
            const int p0 = (int)kept / c.page_size, p1 = (int)t / c.page_size, page0 = table[p0], page1 = table[p1];
            if ((uint32_t)page0 >= (uint32_t)c.pages || (uint32_t)page1 >= (uint32_t)c.pages) continue;
            const int64_t e = ((int64_t)page0 * c.kv_heads + h) * c.page_size + ((int)kept - p0 * c.page_size);
            to[x] = ((int64_t)page1 * c.kv_heads + h) * c.page_size + ((int)t - p1 * c.page_size);
            v[x] = *reinterpret_cast<const u4*>(data + e * c.head_dim + byte[x]);
            s[x] = scales[e];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the loads are back, in every wave)
        __syncthreads();
#pragma unroll
        for (int x = 0; x < kDepth; ++x) {
            if (to[x] < 0) continue;
            *reinterpret_cast<u4*>(data + to[x] * c.head_dim + byte[x]) = v[x];
            if (byte[x] == 0) scales[to[x]] = s[x];
        }
    }
}

__global__ __launch_bounds__(kMovers + 64) void kv_close_up(CompactArgs a, int tokens, int splits, int64_t work) {
    __shared__ Lines lines[3];
    const neo_kv_cache& c = a.c;
    const int parts = c.kv_heads * splits;
    const uint32_t each = (uint32_t)c.head_dim / 16 / (uint32_t)splits;
    const int64_t limit = a.table_pages * c.page_size;  // tokens that a sequence's table has
    const bool mover = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) < kMovers / 64;
    for (int64_t at = blockIdx.x; at < work; at += gridDim.x) {
        const int64_t q = at / parts;
        const int part = (int)(at - q * parts), of = (int)(q % (2 * a.layers)), b = (int)(q / (2 * a.layers));
        const int64_t layer = (of >> 1) * a.layer_stride;
        const int first = min(max(a.starts[b], 0), a.kept), count = min(min(max(a.starts[b + 1], first), a.kept) - first, a.max_keep);
        const int base = a.bases[b];
        if (base < 0) continue;
        const int chunks = (count + tokens - 1) / tokens;
        const int32_t* table = a.table + (int64_t)b * a.table_stride;
        auto look_up = [&](int chunk) {
            Lines& l = lines[chunk % 3];
            for (int x = threadIdx.x & 63; x < tokens; x += 64) {
                const int i = chunk * tokens + x;
                int64_t from = 0, to = -1;
                const int64_t t = (int64_t)base + i, kept = i < count ? a.keep[first + i] : 0;
                if (kept > t && kept < limit) {
                    const int p0 = (int)kept / c.page_size, p1 = (int)t / c.page_size, page0 = table[p0], page1 = table[p1];
                    if ((uint32_t)page0 < (uint32_t)c.pages && (uint32_t)page1 < (uint32_t)c.pages) {
                        from = (int64_t)page0 * c.kv_heads * c.page_size + ((int)kept - p0 * c.page_size);
                        to = (int64_t)page1 * c.kv_heads * c.page_size + ((int)t - p1 * c.page_size);
                    }
                }
                l.from[x] = from;
                l.to[x] = to;
            }
        };
        // this thread's pieces of 16 bytes: of which token of a chunk, and their place
        int8_t* data = (of & 1 ? c.v : c.k) + layer * c.head_dim;
        float* scales = (of & 1 ? c.v_scale : c.k_scale) + layer;
        const int shift = part / splits * c.page_size;
        int line[kDepth];
        uint32_t byte[kDepth];
#pragma unroll
        for (int x = 0; x < kDepth; ++x) {
            const uint32_t idx = x * kMovers + threadIdx.x, row = idx / each;
            line[x] = row < (uint32_t)tokens ? (int)row : -1;
            byte[x] = (idx - row * each + (uint32_t)(part % splits) * each) * 16;
        }
        // (every thread loads, past the last chunk too, so that the number of loads under way is known
        // and a chunk's use waits for its own only; those that move nothing load the cache's start)
        auto load = [&](int chunk, Moved& m) {
            const Lines& l = lines[chunk % 3];
#pragma unroll
            for (int x = 0; x < kDepth; ++x) {
                const int64_t to = l.to[max(line[x], 0)];
                const bool moves = line[x] >= 0 && to >= 0;
                m.to[x] = moves ? to + shift : -1;
                const int64_t e = moves ? l.from[line[x]] + shift : 0;
                m.v[x] = *reinterpret_cast<const u4*>(data + e * c.head_dim + byte[x]);
                m.s[x] = scales[e];
            }
        };
        auto step = [&](int chunk, Moved& m, Moved& next) {
            load(chunk + 1, next);
#pragma unroll
            for (int x = 0; x < kDepth; ++x) asm volatile("" : "+v"(m.v[x]), "+v"(m.s[x])::"memory");  // (these loads are back)
            __syncthreads();
#pragma unroll
            for (int x = 0; x < kDepth; ++x) {
                if (m.to[x] < 0) continue;
                __builtin_nontemporal_store(m.v[x], reinterpret_cast<u4*>(data + m.to[x] * c.head_dim + byte[x]));
                if (byte[x] == 0) scales[m.to[x]] = m.s[x];
            }
        };
        if (chunks == 0) continue;
        // (whole waves take either way, with as many barriers: on one way the waits between loads
        // and stores count the movers' loads alone)
        if (mover) {
            __syncthreads();
            Moved m, next;
            load(0, m);
            for (int chunk = 0; chunk < chunks; chunk += 2) {
                step(chunk, m, next);
                if (chunk + 1 == chunks) break;
                step(chunk + 1, next, m);
            }
        } else {
            look_up(0);
            look_up(1);
            __syncthreads();
            for (int chunk = 0; chunk < chunks; ++chunk) {
                look_up(chunk + 2);
                __syncthreads();
            }
        }
    }
}

}  // namespace

// (a launch has fewer than 2^32 threads)
constexpr int64_t kBlocksMax = 1 << 22;

hipError_t launch_kv_copy(const CopyArgs& a, hipStream_t st) {
    const int64_t pieces = (int64_t)a.c.kv_heads * a.c.page_size * (a.c.head_dim / 16);
    const int chunks = (int)((pieces + kChunk - 1) / kChunk);
    const int64_t work = (int64_t)a.pairs * 2 * a.layers * chunks;
    const dim3 blocks((unsigned)std::min(work, kBlocksMax));
    if (a.entries)
        hipLaunchKernelGGL(kv_copy<false>, blocks, dim3(256), 0, st, a, chunks, work);
    else
        hipLaunchKernelGGL(kv_copy<true>, blocks, dim3(256), 0, st, a, chunks, work);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const CompactArgs& a, hipStream_t st) {
    constexpr int kPieces = kMovers * kDepth;
    int each = a.c.head_dim / 16, splits = 1;
    if ((int64_t)a.max_keep * each <= kPieces) {  // as many heads as a chunk holds of all entries
        const int heads = std::min(a.c.kv_heads, kPieces / (each * a.max_keep));
        const int64_t work = (int64_t)a.seqs * 2 * a.layers * cdiv(a.c.kv_heads, heads);
        hipLaunchKernelGGL(kv_close_up_few, dim3((unsigned)std::min(work, kBlocksMax)), dim3(kMovers), 0, st, a, heads, a.max_keep, work);
        return hipGetLastError();
    }
    // where that makes few workgroups, an entry's bytes are split, down to 64
    int64_t work = (int64_t)a.seqs * 2 * a.layers * a.c.kv_heads;
    while (each % 2 == 0 && each > 4 && work < 512) each /= 2, splits *= 2, work *= 2;
    const int tokens = std::min(kPieces / each, kTokensMax);
    hipLaunchKernelGGL(kv_close_up, dim3((unsigned)std::min(work, kBlocksMax)), dim3(kMovers + 64), 0, st, a, tokens, splits, work);
    return hipGetLastError();
}

}  // namespace neo
