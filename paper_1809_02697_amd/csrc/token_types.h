// Element types and small device helpers shared by the token operators
// (tokens.hip, matmul_int8.hip, kv_cache.hip, attention.hip).
#pragma once

#include "neo_internal.h"

namespace neo {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));

inline int dtype_size(int dtype) { return dtype == NEO_F32 ? 4 : 2; }
inline bool dtype_valid(int dtype) { return dtype == NEO_F32 || dtype == NEO_F16 || dtype == NEO_BF16; }

// Eight neighbouring elements, loaded and stored at their element's alignment:
// rows of odd widths and slices start anywhere, and the hardware takes global
// accesses at any address.
template <typename T>
struct Vec8 {
    typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};
typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T>
__device__ inline f32x8 load8(const T* p) {
    typename Vec8<T>::type v = *reinterpret_cast<const typename Vec8<T>::type*>(p);
    return __builtin_convertvector(v, f32x8);
}
template <typename T>
__device__ inline void store8(T* p, f32x8 v) {
    typedef T raw __attribute__((ext_vector_type(8)));
    *reinterpret_cast<typename Vec8<T>::type*>(p) = __builtin_convertvector(v, raw);
}
template <typename T>
__device__ inline void store4(T* p, v4f v) {
    typedef T raw __attribute__((ext_vector_type(4)));
    typedef T loose __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    *reinterpret_cast<loose*>(p) = __builtin_convertvector(v, raw);
}
// The first n (0 .. 8) of them; the rest read as zero, are not touched.
template <typename T>
__device__ inline f32x8 load8(const T* p, int n) {
    if (n >= 8) return load8(p);
    f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) v[i] = (float)p[i];
    return v;
}
template <typename T>
__device__ inline void store8(T* p, f32x8 v, int n) {
    if (n >= 8) return store8(p, v);
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) p[i] = (T)v[i];
}

// Magnitudes compared as integers: the order of the finite ones, with
// infinity above them and NaN above infinity, so a maximum keeps both.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t kInfBits = 0x7f800000u;

// The scale of a row whose largest magnitude is `top`: top / 127, 1 for zero,
// NaN where the row holds an infinity or a NaN.
__device__ inline float row_scale(uint32_t top) {
    if (top >= kInfBits) return __uint_as_float(0x7fc00000u);
    if (top == 0) return 1.f;
    return fmaxf(__uint_as_float(top) / 127.f, 1.17549435e-38f);
}

// round_half_even(v / s) of a row of scale s: |v / s| is at most 127 by the
// choice of s up to a rounding, which the clamp takes back.  0 in a row whose
// scale is NaN.
__device__ inline int quantized(float v, float s) {
    const float q = rintf(v / s);
    return s == s ? (int)fminf(fmaxf(q, -127.f), 127.f) : 0;
}
// Eight of a row.  v times the scale's reciprocal lies within 3e-5 of v / s, so
// it rounds to the same integer but near the middle of two, and only there the
// quotient itself is taken (one value in 10^4; a quotient is 11 instructions).
__device__ inline uint2 quantized8(f32x8 v, float s) {
    const float inv = 1.f / s;
    f32x8 q;
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = v[i] * inv;
        q[i] = rintf(t);
        far = fmaxf(far, fabsf(t - q[i]));
    }
    uint32_t w[2] = {0, 0};
    if (far < 0.49995f && s == s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)((int)q[i] & 0xff) << (8 * (i & 3));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)(quantized(v[i], s) & 0xff) << (8 * (i & 3));
    }
    return make_uint2(w[0], w[1]);
}
__device__ inline f32x8 dequantized8(uint2 w, float s) {
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3))) * s;
    return v;
}

// One value to `y[at]` of the type that `dtype` names.
__device__ inline void store1(void* y, int64_t at, float v, int dtype) {
    if (dtype == NEO_F32)
        static_cast<float*>(y)[at] = v;
    else if (dtype == NEO_F16)
        static_cast<_Float16*>(y)[at] = (_Float16)v;
    else
        static_cast<__bf16*>(y)[at] = (__bf16)v;
}

// max and sum over groups of W neighbouring lanes (a power of two).
template <int W = 64>
__device__ inline uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    return v;
}
template <int W = 64>
__device__ inline float lanes_sum(float v) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// ---- launchers: arguments are valid (token_api.cpp checks them) ------------------------

struct RowsArgs {
    const void *x, *r;  // rows; residual (norm) or gate
    const float* gamma;
    void *h, *y;
    int8_t* q;
    float* scale;
    int64_t xs, rs, hs, ys, qs;  // strides in elements
    float eps;
    int rows, cols;
};
constexpr int kRowsMaxCols = 65536;
hipError_t launch_rmsnorm(int dtype, const RowsArgs& a, hipStream_t st);
hipError_t launch_quantize_tokens(int dtype, const RowsArgs& a, hipStream_t st);
hipError_t launch_dequantize_tokens(int dtype, const int8_t* q, int64_t qs, const float* scale, int rows,
                                    int cols, void* y, int64_t ys, hipStream_t st);

struct MatmulArgs {
    const int8_t *x, *w;
    const float *xscale, *wscale, *bias;
    void* y;
    int64_t xs, ys;  // row strides of x (bytes) and y (elements)
    int M, N, Kp;    // Kp: padded row length, a multiple of 16
    int act, dtype;
};
size_t matmul_int8_workspace(const MatmulArgs& a);
hipError_t launch_matmul_int8(const MatmulArgs& a, float* ws, hipStream_t st);

struct KvArgs {
    neo_kv_cache c;
    const void *k, *v;  // new tokens
    void *ko, *vo;      // tokens read back
    int64_t kts, khs, vts, vhs;
    const int64_t* slots;
    int tokens;
};
hipError_t launch_kv_write(int dtype, const KvArgs& a, hipStream_t st);
hipError_t launch_kv_read(int dtype, const KvArgs& a, hipStream_t st);

struct AttnArgs {
    neo_kv_cache c;
    const void* q;
    void* out;
    int64_t qts, qhs, ots, ohs, table_stride;
    const int32_t *table, *contexts, *starts;
    int tokens, q_heads, seqs, max_chunk, max_context, window;
    float scale;
};
size_t attention_workspace(int dtype, const AttnArgs& a);
hipError_t launch_attention(int dtype, const AttnArgs& a, float* ws, hipStream_t st);

}  // namespace neo
