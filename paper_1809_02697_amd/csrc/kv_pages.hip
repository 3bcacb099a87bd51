// Pages of the paged int8 cache, in every layer's cache at once: copied (a
// sequence forks, or pages move together), and closed up (tokens of a sequence
// are dropped).  Both move each byte once, bytes and scales as they are.
#include "token_types.h"

namespace neo {
namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// ---- copies -----------------------------------------------------------------------------
// A page's keys (or values) in one layer are kv_heads stretches of page_size
// entries, of which the first `n` are copied: pieces of 16 bytes, an entry's
// scale with its first piece.  A workgroup takes kChunk pieces, four a thread,
// all loaded before the first is stored.
constexpr int kDepth = 4, kChunk = 256 * kDepth;

__global__ __launch_bounds__(256) void kv_copy(CopyArgs a, int chunks, int64_t work) {
    const neo_kv_cache& c = a.c;
    const uint32_t each = (uint32_t)c.head_dim / 16, page = (uint32_t)(c.kv_heads * c.page_size);
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int64_t q = w / chunks;
        const int chunk = (int)(w - q * chunks), of = (int)(q % (2 * a.layers)), pair = (int)(q / (2 * a.layers));
        const int src = a.src[pair], dst = a.dst[pair], n = a.entries ? min(max(a.entries[pair], 0), c.page_size) : c.page_size;
        if ((uint32_t)src >= (uint32_t)c.pages || (uint32_t)dst >= (uint32_t)c.pages || src == dst) continue;
        const int64_t layer = (of >> 1) * a.layer_stride;
        int8_t* data = (of & 1 ? c.v : c.k) + layer * c.head_dim;
        float* scales = (of & 1 ? c.v_scale : c.k_scale) + layer;
        const uint32_t row = (uint32_t)n * each, pieces = row * (uint32_t)c.kv_heads;
        const int64_t from = (int64_t)src * page, to = (int64_t)dst * page;
        u4 v[kDepth];
        float s[kDepth];
        uint32_t entry[kDepth], piece[kDepth];
#pragma unroll
        for (int i = 0; i < kDepth; ++i) {
            const uint32_t x = (uint32_t)chunk * kChunk + i * 256 + threadIdx.x, h = n == c.page_size ? 0 : x / max(row, 1u), y = x - h * row;
            const uint32_t o = y / each;
            entry[i] = x < pieces ? h * (uint32_t)c.page_size + o : 0xffffffffu;
            piece[i] = y - o * each;
            if (x >= pieces) continue;
            v[i] = *reinterpret_cast<const u4*>(data + (from + entry[i]) * c.head_dim + piece[i] * 16);
            if (piece[i] == 0) s[i] = scales[from + entry[i]];
        }
#pragma unroll
        for (int i = 0; i < kDepth; ++i) {
            if (entry[i] == 0xffffffffu) continue;
            *reinterpret_cast<u4*>(data + (to + entry[i]) * c.head_dim + piece[i] * 16) = v[i];
            if (piece[i] == 0) scales[to + entry[i]] = s[i];
        }
    }
}

// ---- closing up --------------------------------------------------------------------------
// Token base + i of a sequence becomes what token keep[i] >= base + i was.  A
// workgroup takes some heads of a sequence's keys (or values) in one layer, and
// its tokens in order, a chunk of `tokens` at a time: what later chunks read lies
// behind what this one writes, so only a chunk's own loads have to be back before
// the first of its stores.
__global__ __launch_bounds__(256) void kv_close_up(CompactArgs a, int heads, int tokens, int64_t work) {
    const neo_kv_cache& c = a.c;
    const int parts = (c.kv_heads + heads - 1) / heads;
    const uint32_t each = (uint32_t)c.head_dim / 16;
    const int64_t limit = a.table_stride * c.page_size;  // tokens that a sequence's table has
    for (int64_t at = blockIdx.x; at < work; at += gridDim.x) {
        const int64_t q = at / parts;
        const int part = (int)(at - q * parts), of = (int)(q % (2 * a.layers)), b = (int)(q / (2 * a.layers));
        const int64_t layer = (of >> 1) * a.layer_stride;
        int8_t* data = (of & 1 ? c.v : c.k) + layer * c.head_dim;
        float* scales = (of & 1 ? c.v_scale : c.k_scale) + layer;
        const int first = min(max(a.starts[b], 0), a.kept), count = min(min(max(a.starts[b + 1], first), a.kept) - first, a.max_keep);
        const int base = a.bases[b];
        if (base < 0) continue;
        const int32_t* table = a.table + (int64_t)b * a.table_stride;
        auto entry = [&](int token, int h) {  // -1: not in the cache
            const int p = token / c.page_size, page = table[p];
            if ((uint32_t)page >= (uint32_t)c.pages) return (int64_t)-1;
            return ((int64_t)page * c.kv_heads + h) * c.page_size + (token - p * c.page_size);
        };
        for (int i0 = 0; i0 < count; i0 += tokens) {
            u4 v[kDepth];
            float s[kDepth];
            int64_t to[kDepth];
            uint32_t piece[kDepth];
#pragma unroll
            for (int x = 0; x < kDepth; ++x) {
                const uint32_t idx = x * 256 + threadIdx.x, row = idx / each, hh = row / (uint32_t)tokens;
                const int i = i0 + (int)(row - hh * (uint32_t)tokens), h = part * heads + (int)hh;
                piece[x] = idx - row * each;
                to[x] = -1;
                if ((int)hh >= heads || h >= c.kv_heads || i >= count) continue;
                const int64_t kept = a.keep[first + i], t = (int64_t)base + i;
                if (kept <= t || kept >= limit) continue;
                const int64_t e = entry((int)kept, h);
                to[x] = e < 0 ? -1 : entry((int)t, h);
                if (to[x] < 0) continue;
                v[x] = *reinterpret_cast<const u4*>(data + e * c.head_dim + piece[x] * 16);
                if (piece[x] == 0) s[x] = scales[e];
            }
            // every wave's loads are back
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
#pragma unroll
            for (int x = 0; x < kDepth; ++x) {
                if (to[x] < 0) continue;
                *reinterpret_cast<u4*>(data + to[x] * c.head_dim + piece[x] * 16) = v[x];
                if (piece[x] == 0) scales[to[x]] = s[x];
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
    hipLaunchKernelGGL(kv_copy, dim3((unsigned)std::min(work, kBlocksMax)), dim3(256), 0, st, a, chunks, work);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const CompactArgs& a, hipStream_t st) {
    const int each = a.c.head_dim / 16;
    const int heads = std::max(1, std::min<int>(a.c.kv_heads, kChunk / (each * std::min(a.max_keep, kChunk))));
    const int tokens = std::max(1, std::min(a.max_keep, kChunk / (each * heads)));
    const int64_t work = (int64_t)a.seqs * 2 * a.layers * cdiv(a.c.kv_heads, heads);
    hipLaunchKernelGGL(kv_close_up, dim3((unsigned)std::min(work, kBlocksMax)), dim3(256), 0, st, a, heads, tokens, work);
    return hipGetLastError();
}

}  // namespace neo
