// Rotary positions: pairs of a head's values turned by an angle that grows with
// the token's position,
//
//   (a, b) -> A (a cos t - b sin t, b cos t + a sin t),  t = position * frequency_i
//
// out of place or in it, and with the keys' and values' way into the paged int8
// cache in the same launch: a key goes from the product that wrote it to the
// cache's bytes without a rounding between.
//
// t is one product in 64 bits, taken to the quarter turn next to it in two parts
// of pi / 2, so that positions of 2^30 keep their angle; sine and cosine are
// polynomials in 64 bits, rounded once.  A lane has eight pairs and takes their
// angles once for several heads.
#include "token_types.h"

namespace neo {
namespace {

// A cos t and A sin t.  |rest| <= pi / 4: the series end at rest^13 / 13! < 7e-12
// and rest^12 / 12! < 2e-10.
__device__ inline void angle(double t, float amplitude, float& c, float& s) {
    const double n = rint(t * 0.6366197723675814);
    const double x = fma(-n, 6.123233995736766e-17, fma(-n, 1.5707963267948966, t)), z = x * x;
    const double sine = fma(x * z, fma(z, fma(z, fma(z, fma(z, -1. / 39916800, 1. / 362880), -1. / 5040), 1. / 120), -1. / 6), x);
    const double cosine = fma(z, fma(z, fma(z, fma(z, fma(z, -1. / 3628800, 1. / 40320), -1. / 720), 1. / 24), -0.5), 1.);
    const int quarter = (int)(n - 4. * floor(n * 0.25));  // 0 .. 3
    const double cc = quarter & 1 ? sine : cosine, ss = quarter & 1 ? cosine : sine;
    c = (float)((quarter + 1) & 2 ? -cc : cc) * amplitude;
    s = (float)(quarter & 2 ? -ss : ss) * amplitude;
}

// A row's pieces: of eight pairs (the first `turned`), then of 16 values that stay.
struct Pieces {
    int turned, all;
};
__host__ __device__ inline Pieces pieces_of(int dim, int rot) {
    const int turned = (rot + 15) / 16;
    return Pieces{turned, turned + (dim - rot + 15) / 16};
}
// Where the two halves of eight values of piece p lie, and how many each has.
struct Place {
    int at[2], n[2];
    bool turns;
};
template <int LAYOUT>
__device__ inline Place place_of(int p, const Pieces& ps, int dim, int rot) {
    Place w;
    w.turns = p < ps.turned;
    if (w.turns) {
        const int n = min(8, rot / 2 - p * 8);
        if (LAYOUT == NEO_ROTARY_HALF) {
            w.at[0] = p * 8, w.at[1] = rot / 2 + p * 8;
            w.n[0] = w.n[1] = n;
        } else {
            w.at[0] = p * 16, w.at[1] = p * 16 + 8;
            w.n[0] = min(8, 2 * n), w.n[1] = max(0, 2 * n - 8);
        }
    } else {
        w.at[0] = rot + (p - ps.turned) * 16, w.at[1] = w.at[0] + 8;
        w.n[0] = min(8, max(0, dim - w.at[0])), w.n[1] = min(8, max(0, dim - w.at[1]));
    }
    return w;
}

struct Angles {
    f32x8 c, s;
};
__device__ inline Angles angles(const RotaryArgs& a, int64_t token, int p, bool turns) {
    Angles g;
    if (!turns) return g;
    const double at = (double)a.positions[token];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float c, s;
        angle(at * a.freqs[min(p * 8 + i, a.rot / 2 - 1)], a.amplitude, c, s);
        g.c[i] = c, g.s[i] = s;
    }
    return g;
}
template <int LAYOUT>
__device__ inline void turn(f32x8 (&v)[2], const Angles& g) {
    if (LAYOUT == NEO_ROTARY_HALF) {
        const f32x8 x = v[0] * g.c - v[1] * g.s;
        v[1] = v[1] * g.c + v[0] * g.s;
        v[0] = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = v[i / 4][i % 4 * 2], y = v[i / 4][i % 4 * 2 + 1];
            v[i / 4][i % 4 * 2] = x * g.c[i] - y * g.s[i];
            v[i / 4][i % 4 * 2 + 1] = y * g.c[i] + x * g.s[i];
        }
    }
}

// Thread = (token, part of the heads, piece), piece fastest: HEADS heads, `parts` apart.
template <typename T, int LAYOUT, int HEADS>
__device__ void turn_rows(const RotaryArgs& a, uint32_t thread, int parts, int pieces) {
    const Pieces ps = pieces_of(a.dim, a.rot);
    const uint32_t rest = thread / (uint32_t)pieces, t = rest / (uint32_t)parts;
    const int p = (int)(thread - rest * (uint32_t)pieces), part = (int)(rest - t * (uint32_t)parts);
    if (t >= (uint32_t)a.tokens) return;
    const Place w = place_of<LAYOUT>(p, ps, a.dim, a.rot);
    const T* x = static_cast<const T*>(a.x) + (int64_t)t * a.xts;
    T* y = static_cast<T*>(a.y) + (int64_t)t * a.yts;
    f32x8 v[HEADS][2];
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
#pragma unroll
        for (int o = 0; o < 2; ++o)  // (past the last head: that one again)
            v[i][o] = load8(x + (int64_t)min(part + i * parts, a.heads - 1) * a.xhs + w.at[o], w.n[o]);
    const Angles g = angles(a, t, p, w.turns);
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int h = part + i * parts;
        if (h >= a.heads) continue;
        if (w.turns) turn<LAYOUT>(v[i], g);
#pragma unroll
        for (int o = 0; o < 2; ++o) store8(y + (int64_t)h * a.yhs + w.at[o], v[i][o], w.n[o]);
    }
}

template <typename T, int LAYOUT, int HEADS>
__global__ __launch_bounds__(256) void rotary(RotaryArgs a, int parts, int pieces) {
    turn_rows<T, LAYOUT, HEADS>(a, blockIdx.x * 256u + threadIdx.x, parts, pieces);
}

__device__ inline void store_int8(int8_t* to, uint2 w, int n) {
    typedef uint32_t loose __attribute__((ext_vector_type(2), aligned(1)));
    if (n >= 8) {
        *reinterpret_cast<loose*>(to) = loose{w.x, w.y};
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) to[i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}

// The first `q_blocks` workgroups turn the queries, the others take the keys and
// values: LANES lanes (a piece each) a token's head.
template <typename T, int LAYOUT, int HEADS, int LANES>
__global__ __launch_bounds__(256) void rotary_kv_write(RotaryArgs a, int parts, int pieces, uint32_t q_blocks) {
    if (blockIdx.x < q_blocks) {
        turn_rows<T, LAYOUT, HEADS>(a, blockIdx.x * 256u + threadIdx.x, parts, pieces);
        return;
    }
    const neo_kv_cache& c = a.kv.c;
    const int D = c.head_dim, H = c.kv_heads, p = threadIdx.x % LANES;
    const uint32_t row = (blockIdx.x - q_blocks) * (256u / LANES) + threadIdx.x / LANES, t = row / (uint32_t)H;
    if (t >= (uint32_t)a.tokens) return;  // (all lanes of the row)
    const int h = (int)(row - t * (uint32_t)H);
    const Pieces ps = pieces_of(D, a.rot);
    Place w[2] = {place_of<LAYOUT>(p, ps, D, a.rot), {{p * 16, p * 16 + 8}, {0, 0}, false}};
    if (p >= ps.all) w[0].n[0] = w[0].n[1] = 0;
    if (p * 16 < D) w[1].n[0] = w[1].n[1] = 8;
    const T* x[2] = {static_cast<const T*>(a.kv.k) + (int64_t)t * a.kv.kts + (int64_t)h * a.kv.khs,
                     static_cast<const T*>(a.kv.v) + (int64_t)t * a.kv.vts + (int64_t)h * a.kv.vhs};
    f32x8 v[2][2];
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int i = 0; i < 2; ++i) v[o][i] = load8(x[o] + w[o].at[i], w[o].n[i]);
    const int64_t e = entry_of(c, a.kv.slots[t], h);
    if (w[0].turns) turn<LAYOUT>(v[0], angles(a, t, p, true));
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, j < w[o].n[i] ? magnitude(v[o][i][j]) : 0u);
        top = lanes_max<LANES>(top);
        const float s = row_scale(top);
        if (e < 0) continue;
        if (p == 0) (o ? c.v_scale : c.k_scale)[e] = s;
#pragma unroll
        for (int i = 0; i < 2; ++i) store_int8((o ? c.v : c.k) + e * D + w[o].at[i], quantized8(v[o][i], s), w[o].n[i]);
    }
}

// Heads a lane takes: several once there are threads enough without.
constexpr int kHeads = 4;

template <typename T, int LAYOUT, int HEADS>
hipError_t launch_part(const RotaryArgs& a, bool write, hipStream_t st) {
    const Pieces ps = pieces_of(a.dim, a.rot);
    const int parts = cdiv(a.heads, HEADS), pieces = a.x == a.y ? ps.turned : ps.all;
    const uint32_t q_blocks = (uint32_t)(((int64_t)a.tokens * parts * pieces + 255) / 256);
    if (!write) {
        if (q_blocks) hipLaunchKernelGGL((rotary<T, LAYOUT, HEADS>), dim3(q_blocks), dim3(256), 0, st, a, parts, pieces);
        return hipGetLastError();
    }
    const int lanes = ps.all <= 4 ? 4 : ps.all <= 8 ? 8 : ps.all <= 16 ? 16 : 32;
    const uint32_t blocks = q_blocks + (uint32_t)(((int64_t)a.tokens * a.kv.c.kv_heads * lanes + 255) / 256);
#define NEO_LANES(n) \
    case n: hipLaunchKernelGGL((rotary_kv_write<T, LAYOUT, HEADS, n>), dim3(blocks), dim3(256), 0, st, a, parts, pieces, q_blocks); break
    switch (lanes) {
        NEO_LANES(4);
        NEO_LANES(8);
        NEO_LANES(16);
        NEO_LANES(32);
    }
#undef NEO_LANES
    return hipGetLastError();
}

// Tokens in slices that have fewer than 2^30 threads.
template <typename T>
hipError_t by_layout(const RotaryArgs& a, bool write, hipStream_t st) {
    const int64_t row = (int64_t)pieces_of(a.dim, a.rot).all * a.heads + (write ? 32ll * a.kv.c.kv_heads : 0);
    const int most = (int)std::max<int64_t>(1, (1ll << 30) / row);
    for (int64_t t = 0; t < a.tokens; t += most) {
        RotaryArgs b = a;
        b.tokens = (int)std::min<int64_t>(most, a.tokens - t);
        b.x = static_cast<const T*>(a.x) + t * a.xts;
        b.y = static_cast<T*>(a.y) + t * a.yts;
        b.positions += t;
        if (write) {
            b.kv.k = static_cast<const T*>(a.kv.k) + t * a.kv.kts;
            b.kv.v = static_cast<const T*>(a.kv.v) + t * a.kv.vts;
            b.kv.slots += t;
        }
        const bool many = (int64_t)b.tokens * row >= 1 << 18;
        hipError_t e;
        if (a.layout == NEO_ROTARY_HALF)
            e = many ? launch_part<T, NEO_ROTARY_HALF, kHeads>(b, write, st) : launch_part<T, NEO_ROTARY_HALF, 1>(b, write, st);
        else
            e = many ? launch_part<T, NEO_ROTARY_INTERLEAVED, kHeads>(b, write, st) : launch_part<T, NEO_ROTARY_INTERLEAVED, 1>(b, write, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(int dtype, const RotaryArgs& a, bool write, hipStream_t st) {
    if (dtype == NEO_F32) return by_layout<float>(a, write, st);
    if (dtype == NEO_F16) return by_layout<_Float16>(a, write, st);
    return by_layout<__bf16>(a, write, st);
}

}  // namespace neo
