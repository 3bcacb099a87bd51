// The paged int8 key/value cache: tokens quantized as they are written, one
// scale per token and head, and read back.
//
// A row is one token's head: head_dim values, s = max|v| / 127.  LANES lanes
// take a row, eight values each, so a wave holds 64 / LANES rows and a row's
// maximum is a few lane exchanges.  Both directions move each value once, and
// memory bounds them: 16,000 tokens x 8 heads of 128 written from float16 in
// 29 us (3.4 TB/s: a launch of some 10 us at the front and end of its loads),
// 60,000 read back in 75 us (4.9 TB/s); 32 tokens 4 us either way, the launch
// and the trips slot -> value -> entry.
#include "token_types.h"

namespace neo {
namespace {

// A group takes a token's key and value of a head: one lookup of the slot, and
// two rows' loads under way at once (16,000 tokens x 8 heads of 128 in float16
// 32 us, 41 with a row a group and a division a value).
template <typename T, int LANES>
__global__ __launch_bounds__(256) void kv_write(KvArgs a) {
    const int D = a.c.head_dim, H = a.c.kv_heads;
    const int64_t rows = (int64_t)a.tokens * H;
    const int j = (threadIdx.x % LANES) * 8;
    for (int64_t r = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; r < rows;
         r += (int64_t)gridDim.x * (256 / LANES)) {
        const int64_t t = rows <= 0x7fffffff ? (int64_t)((uint32_t)r / (uint32_t)H) : r / H;
        const int h = (int)(r - t * H), jj = j < D ? j : 0;
        f32x8 v[2] = {load8(static_cast<const T*>(a.k) + t * a.kts + h * a.khs + jj),
                      load8(static_cast<const T*>(a.v) + t * a.vts + h * a.vhs + jj)};
        const int64_t e = entry_of(a.c, a.slots[t], h);
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, j < D ? magnitude(v[o][i]) : 0u);
            top = lanes_max<LANES>(top);  // (the lanes of a row leave the loop together)
            const float s = row_scale(top);
            if (e < 0 || j >= D) continue;
            if (j == 0) (o ? a.c.v_scale : a.c.k_scale)[e] = s;
            *reinterpret_cast<uint2*>((o ? a.c.v : a.c.k) + e * D + j) = quantized8(v[o], s);
        }
    }
}

template <typename T, int LANES>
__global__ __launch_bounds__(256) void kv_read(KvArgs a) {
    const int D = a.c.head_dim, H = a.c.kv_heads;
    const int64_t rows = (int64_t)a.tokens * H;
    const int j = (threadIdx.x % LANES) * 8;
    if (j >= D) return;
    for (int64_t r = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; r < rows;
         r += (int64_t)gridDim.x * (256 / LANES)) {
        const int64_t t = rows <= 0x7fffffff ? (int64_t)((uint32_t)r / (uint32_t)H) : r / H;
        const int64_t e = entry_of(a.c, a.slots[t], (int)(r - t * H));
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            T* out = static_cast<T*>(o ? a.vo : a.ko);
            if (!out) continue;
            f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
            if (e >= 0)
                v = dequantized8(*reinterpret_cast<const uint2*>((o ? a.c.v : a.c.k) + e * D + j),
                                 (o ? a.c.v_scale : a.c.k_scale)[e]);
            store8(out + r * D + j, v);
        }
    }
}

template <typename T, int LANES>
hipError_t launch(const KvArgs& a, bool write, hipStream_t st) {
    const int64_t rows = (int64_t)a.tokens * a.c.kv_heads;
    const unsigned blocks = (unsigned)std::min<int64_t>((rows + 256 / LANES - 1) / (256 / LANES), 16384);
    if (write)
        hipLaunchKernelGGL((kv_write<T, LANES>), dim3(blocks), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((kv_read<T, LANES>), dim3(blocks), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <typename T>
hipError_t by_dim(const KvArgs& a, bool write, hipStream_t st) {
    if (a.c.head_dim <= 64) return launch<T, 8>(a, write, st);
    if (a.c.head_dim <= 128) return launch<T, 16>(a, write, st);
    return launch<T, 32>(a, write, st);
}

hipError_t by_type(int dtype, const KvArgs& a, bool write, hipStream_t st) {
    if (dtype == NEO_F32) return by_dim<float>(a, write, st);
    if (dtype == NEO_F16) return by_dim<_Float16>(a, write, st);
    return by_dim<__bf16>(a, write, st);
}

}  // namespace

hipError_t launch_kv_write(int dtype, const KvArgs& a, hipStream_t st) { return by_type(dtype, a, true, st); }
hipError_t launch_kv_read(int dtype, const KvArgs& a, hipStream_t st) { return by_type(dtype, a, false, st); }

}  // namespace neo
