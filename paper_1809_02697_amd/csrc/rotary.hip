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
// polynomials in 64 bits, rounded once, with the amplitude in them.  A workgroup
// works its tokens' angles out once, into LDS, while the values are on their way; a
// lane takes two vectors of 16 bytes, neighbouring lanes neighbouring ones.
#include "token_types.h"

namespace neo {
namespace {

// A cos t and A sin t, each rounded once.  |x| <= pi / 4: the series end at
// x^13 / 13! < 7e-12 and x^12 / 12! < 2e-10.
__device__ inline void angle(double t, double amplitude, float& c, float& s) {
    const double n = rint(t * 0.6366197723675814);
    const double x = fma(-n, 6.123233995736766e-17, fma(-n, 1.5707963267948966, t)), z = x * x;
    const double sine = fma(x * z, fma(z, fma(z, fma(z, fma(z, -1. / 39916800, 1. / 362880), -1. / 5040), 1. / 120), -1. / 6), x);
    const double cosine = fma(z, fma(z, fma(z, fma(z, fma(z, -1. / 3628800, 1. / 40320), -1. / 720), 1. / 24), -0.5), 1.);
    const int quarter = (int)(n - 4. * floor(n * 0.25));  // 0 .. 3
    const double cc = quarter & 1 ? sine : cosine, ss = quarter & 1 ? cosine : sine;
    c = (float)(((quarter + 1) & 2 ? -cc : cc) * amplitude);
    s = (float)((quarter & 2 ? -ss : ss) * amplitude);
}

// ---- vectors of a row ----------------------------------------------------------------
// 16 bytes, at an element's alignment.
template <typename T>
struct Vec {
    static constexpr int N = 16 / sizeof(T);
    typedef float floats __attribute__((ext_vector_type(N)));
    typedef T raw __attribute__((ext_vector_type(N)));
    typedef T loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    // the first n of them; the rest read as zero, are not touched
    __device__ static floats load(const T* p, int n) {
        if (n >= N) {
            const raw v = *reinterpret_cast<const loose*>(p);
            return __builtin_convertvector(v, floats);
        }
        floats v = 0.f;
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (i < n) v[i] = (float)p[i];
        return v;
    }
    __device__ static void store(T* p, floats v, int n) {
        const raw w = __builtin_convertvector(v, raw);
        if (n >= N) {
            *reinterpret_cast<loose*>(p) = w;
            return;
        }
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (i < n) p[i] = w[i];
    }
};

// A row's pieces, of two vectors each.  HALF: those that hold a pair's one value in
// the first and its other in the second vector (`turned`), then those of values
// that stay.  INTERLEAVED: vector p and the one as far behind as there are pieces.
struct Pieces {
    int turned, all;
};
__host__ __device__ inline Pieces pieces_of(int layout, int dim, int rot, int n) {
    if (layout == NEO_ROTARY_INTERLEAVED) {
        const int all = ((dim + n - 1) / n + 1) / 2;
        return Pieces{all, all};
    }
    const int turned = (rot / 2 + n - 1) / n;
    return Pieces{turned, turned + (dim - rot + 2 * n - 1) / (2 * n)};
}
struct Place {
    int at[2], n[2];  // where its vectors start, how many values they have
    bool turns;
};
template <int LAYOUT, int N>
__device__ inline Place place_of(int p, const Pieces& ps, int dim, int rot) {
    Place w;
    w.turns = LAYOUT == NEO_ROTARY_INTERLEAVED || p < ps.turned;
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        if (LAYOUT == NEO_ROTARY_INTERLEAVED) {
            w.at[o] = (p + o * ps.all) * N;
            w.n[o] = min(max(dim - w.at[o], 0), N);
        } else if (w.turns) {
            w.at[o] = p * N + o * (rot / 2);
            w.n[o] = min(rot / 2 - p * N, N);
        } else {
            w.at[o] = rot + (2 * (p - ps.turned) + o) * N;
            w.n[o] = min(max(dim - w.at[o], 0), N);
        }
    }
    return w;
}

// ---- angles --------------------------------------------------------------------------
// Of the tokens first .. first + count - 1, in LDS: cosines of all, then sines,
// a token's from a multiple of 8.
struct Angles {
    float *c, *s;
    int row;
};
__host__ __device__ inline int angle_row(int rot) { return (rot / 2 + 7) / 8 * 8; }
__device__ inline Angles work_out(const RotaryArgs& a, int64_t first, int count, int most, float* lds) {
    Angles g;
    g.row = angle_row(a.rot);
    g.c = lds, g.s = lds + most * g.row;
    const int half = a.rot / 2;
    for (int x = threadIdx.x; x < count * half; x += 256) {
        const int t = x / half, i = x - t * half;
        angle((double)a.positions[first + t] * a.freqs[i], a.amplitude, g.c[t * g.row + i], g.s[t * g.row + i]);
    }
    return g;
}
template <int LAYOUT, int N, typename F>
__device__ inline void turn(F (&v)[2], const Place& w, const Angles& g, int token, int rot) {
    const float *c = g.c + token * g.row, *s = g.s + token * g.row;
    if (LAYOUT == NEO_ROTARY_HALF) {
        const F cc = *reinterpret_cast<const F*>(c + w.at[0]), ss = *reinterpret_cast<const F*>(s + w.at[0]);
        const F x = v[0] * cc - v[1] * ss;
        v[1] = v[1] * cc + v[0] * ss;
        v[0] = x;
    } else {
        typedef float pairs __attribute__((ext_vector_type(N / 2)));
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            if (w.at[o] >= rot) continue;
            const pairs cc = *reinterpret_cast<const pairs*>(c + w.at[o] / 2), ss = *reinterpret_cast<const pairs*>(s + w.at[o] / 2);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float x = v[o][2 * i], y = v[o][2 * i + 1];
                const bool turns = w.at[o] + 2 * i < rot;  // (a vector may hold both kinds)
                v[o][2 * i] = turns ? x * cc[i] - y * ss[i] : x;
                v[o][2 * i + 1] = turns ? y * cc[i] + x * ss[i] : y;
            }
        }
    }
}

// ---- rows that are turned and stored --------------------------------------------------
// A thread an item (token, head, piece), piece fastest.  Memory bounds it: 16,384
// tokens of 40 heads of 128 in bfloat16 64 us, 5.2 TB/s, where a copy of them takes
// 61 (two items a thread 66; angles worked out by each lane for itself 95, for four
// heads of one piece 76).
template <typename T, int LAYOUT>
__device__ void turn_rows(const RotaryArgs& a, uint32_t block, int pieces, int most, float* lds) {
    typedef Vec<T> V;
    const uint32_t each = (uint32_t)pieces * (uint32_t)a.heads, start = block * 256u, item = start + threadIdx.x;
    const uint32_t first = start / each, last = min((start + 255u) / each, (uint32_t)a.tokens - 1);
    const uint32_t row = item / (uint32_t)pieces, t = row / (uint32_t)a.heads, h = row - t * (uint32_t)a.heads;
    const bool live = t <= last;
    const Place w = place_of<LAYOUT, V::N>((int)(item - row * (uint32_t)pieces), pieces_of(LAYOUT, a.dim, a.rot, V::N), a.dim, a.rot);
    typename V::floats v[2];
    if (live) {
        const T* x = static_cast<const T*>(a.x) + (int64_t)t * a.xts + (int64_t)h * a.xhs;
#pragma unroll
        for (int o = 0; o < 2; ++o) v[o] = V::load(x + w.at[o], w.n[o]);
    }
    const Angles g = work_out(a, first, (int)(last - first) + 1, most, lds);
    __syncthreads();
    if (!live) return;
    if (w.turns) turn<LAYOUT, V::N>(v, w, g, (int)(t - first), a.rot);
    T* y = static_cast<T*>(a.y) + (int64_t)t * a.yts + (int64_t)h * a.yhs;
#pragma unroll
    for (int o = 0; o < 2; ++o) V::store(y + w.at[o], v[o], w.n[o]);
}

template <typename T, int LAYOUT>
__global__ __launch_bounds__(256) void rotary(RotaryArgs a, int pieces, int most) {
    extern __shared__ __align__(16) float lds[];
    turn_rows<T, LAYOUT>(a, blockIdx.x, pieces, most, lds);
}

// ---- with the cache's write -----------------------------------------------------------
template <int N>
__device__ inline void store_int8(int8_t* to, uint2 w, int n) {
    typedef uint32_t loose2 __attribute__((ext_vector_type(2), aligned(1)));
    typedef uint32_t loose1 __attribute__((aligned(1)));
    if (n >= N) {
        if constexpr (N == 8)
            *reinterpret_cast<loose2*>(to) = loose2{w.x, w.y};
        else
            *reinterpret_cast<loose1*>(to) = w.x;
        return;
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
        if (i < n) to[i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}

// The first `q_blocks` workgroups turn the queries, the others take the keys and
// values: LANES lanes (a piece each) a token's head, its key and its value.  Memory
// bounds it: 16,000 tokens of 32 query heads and 8 of keys and values of 128 in
// float16 81 us, 4.45 TB/s; 64 tokens 6.3 us, a launch and its trips.
template <typename T, int LAYOUT, int LANES>
__global__ __launch_bounds__(256) void rotary_kv_write(RotaryArgs a, int pieces, int most, uint32_t q_blocks) {
    extern __shared__ __align__(16) float lds[];
    if (blockIdx.x < q_blocks) {
        turn_rows<T, LAYOUT>(a, blockIdx.x, pieces, most, lds);
        return;
    }
    typedef Vec<T> V;
    constexpr int N = V::N, ROWS = 256 / LANES;
    const neo_kv_cache& c = a.kv.c;
    const int D = c.head_dim, H = c.kv_heads, p = threadIdx.x % LANES;
    const uint32_t row0 = (blockIdx.x - q_blocks) * (uint32_t)ROWS, row = row0 + threadIdx.x / LANES, t = row / (uint32_t)H;
    const uint32_t first = row0 / (uint32_t)H, last = min((row0 + ROWS - 1) / (uint32_t)H, (uint32_t)a.tokens - 1);
    const int h = (int)(row - t * (uint32_t)H);
    const bool live = t <= last;  // (all lanes of the row)
    const Pieces ps = pieces_of(LAYOUT, D, a.rot, N);
    Place w[2] = {place_of<LAYOUT, N>(p, ps, D, a.rot), {{p * N, p * N + D / 2}, {0, 0}, false}};
    if (p >= ps.all) w[0].n[0] = w[0].n[1] = 0;
    if (p * N < D / 2) w[1].n[0] = w[1].n[1] = N;  // (half a head is whole vectors)
    typename V::floats v[2][2];
    int64_t e = -1;
    if (live) {
        const T* x[2] = {static_cast<const T*>(a.kv.k) + (int64_t)t * a.kv.kts + (int64_t)h * a.kv.khs,
                         static_cast<const T*>(a.kv.v) + (int64_t)t * a.kv.vts + (int64_t)h * a.kv.vhs};
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int i = 0; i < 2; ++i) v[o][i] = V::load(x[o] + w[o].at[i], w[o].n[i]);
        e = entry_of(c, a.kv.slots[t], h);
    }
    const Angles g = work_out(a, first, (int)(last - first) + 1, most, lds);
    __syncthreads();
    if (!live) return;
    if (w[0].turns && p < ps.all) turn<LAYOUT, N>(v[0], w[0], g, (int)(t - first), a.rot);
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) top = max(top, j < w[o].n[i] ? magnitude(v[o][i][j]) : 0u);
        top = lanes_max<LANES>(top);
        const float s = row_scale(top);
        if (e < 0) continue;
        if (p == 0) (o ? c.v_scale : c.k_scale)[e] = s;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x8 eight = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < N; ++j) eight[j] = v[o][i][j];
            store_int8<N>((o ? c.v : c.k) + e * D + w[o].at[i], quantized8(eight, s), w[o].n[i]);
        }
    }
}

// Tokens that `n` neighbouring rows of `each` a token touch at most.
int tokens_of(int64_t n, int64_t each) { return (int)((n - 2 + each) / each + 1); }

template <typename T, int LAYOUT>
hipError_t launch_part(const RotaryArgs& a, bool write, hipStream_t st) {
    const Pieces ps = pieces_of(LAYOUT, a.dim, a.rot, Vec<T>::N);
    const int pieces = a.x == a.y && LAYOUT == NEO_ROTARY_HALF ? ps.turned : ps.all;  // (in place the others stay where they are)
    const uint32_t q_blocks = (uint32_t)(((int64_t)a.tokens * a.heads * pieces + 255) / 256);
    // tokens of a workgroup: at most 24 KB of angles, as heads have up to 1024 values
    int most = tokens_of(256, (int64_t)a.heads * pieces);
    const size_t row = 2 * sizeof(float) * angle_row(a.rot);
    if (!write) {
        hipLaunchKernelGGL((rotary<T, LAYOUT>), dim3(q_blocks), dim3(256), most * row, st, a, pieces, most);
        return hipGetLastError();
    }
    int lanes = 4;
    while (lanes < ps.all) lanes *= 2;
    most = std::max(most, tokens_of(256 / lanes, a.kv.c.kv_heads));
    const uint32_t blocks = q_blocks + (uint32_t)(((int64_t)a.tokens * a.kv.c.kv_heads * lanes + 255) / 256);
#define NEO_LANES(n) \
    case n: hipLaunchKernelGGL((rotary_kv_write<T, LAYOUT, n>), dim3(blocks), dim3(256), most * row, st, a, pieces, most, q_blocks); break
    switch (lanes) {
        NEO_LANES(4);
        NEO_LANES(8);
        NEO_LANES(16);
        NEO_LANES(32);
        NEO_LANES(64);
    }
#undef NEO_LANES
    return hipGetLastError();
}

// Tokens in slices that have fewer than 2^30 threads.
template <typename T>
hipError_t by_layout(const RotaryArgs& a, bool write, hipStream_t st) {
    const int64_t row = (int64_t)pieces_of(a.layout, a.dim, a.rot, Vec<T>::N).all * a.heads + (write ? 64ll * a.kv.c.kv_heads : 0);
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
        const hipError_t e = a.layout == NEO_ROTARY_HALF ? launch_part<T, NEO_ROTARY_HALF>(b, write, st) : launch_part<T, NEO_ROTARY_INTERLEAVED>(b, write, st);
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
