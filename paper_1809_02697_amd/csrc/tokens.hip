// Rows of tokens: residual addition + root-mean-square norm, and quantization
// of rows to int8 with a scale of their own.
//
//   h = x + r,  y = h / sqrt(mean(h^2) + eps) * gamma      (norm)
//   y = x,  or  y = x * g / (1 + exp(-g))                  (quantization)
//   s = max|y| / 127,  q = round_half_even(y / s)
//
// A row is read once: it stays in registers, eight neighbouring elements a
// lane and chunk, between the load, the sum of squares, the maximum and the
// quantization.  Memory bounds it: 8192 rows of 8192 in bfloat16 with residual,
// h and int8 rows 105 us, 4.5 TB/s of the 4.8 that a copy reaches; quantized 36 us
// (5.6 TB/s), with a gate 65 us (5.2 TB/s); one row of 4096 3.6 us, a launch and
// three trips to memory; the gate of 96 rows of 16,384 in float16 7.5 us, on 96 of
// 256 CUs.
#include "token_types.h"

namespace neo {
namespace {

enum { kNorm, kPlain, kGate };

// g / (1 + exp(-g)) within 4 u.  exp2 of the product with log2(e) carried in two
// parts (its rounding alone would be |g| u), and the reciprocal instruction: 12
// instructions instead of the 40 of expf and a division, which bound the rows
// of few tokens.
__device__ inline float silu(float g) {
    constexpr float kLog2eHi = 1.44269502f, kLog2eLo = 1.92596299e-8f, kLn2 = 0.693147181f;
    const float hi = -g * kLog2eHi, lo = fmaf(-g, kLog2eHi, -hi) - g * kLog2eLo;
    if (hi >= 125.f) {
        // The reciprocal of such a sum lies below the normal numbers, which the
        // instruction makes 0: g exp(g), 2^64 times as large until it is rounded.
        // (Far past float32's range lo is noise, and the result -0.)
        const float e = __builtin_amdgcn_exp2f(64.f - hi);
        return g * (hi < 256.f ? fmaf(e, lo * -kLn2, e) : e) * 0x1p-64f;
    }
    float e = __builtin_amdgcn_exp2f(hi);
    if (hi > -126.f) e = fmaf(e, lo * kLn2, e);
    return g * __builtin_amdgcn_rcpf(1.f + e);
}

// One row per group of WAVES waves; a workgroup holds several groups where a
// group is one wave.  The sum of squares is added in float32 in the lane, then
// across lanes and waves: one order, whatever the rows.
template <typename T, int MODE, int WAVES, int CH>
__global__ __launch_bounds__((WAVES > 4 ? WAVES : 4) * 64) void row_int8(RowsArgs a) {
    constexpr int THREADS = WAVES * 64, GROUPS = WAVES >= 4 ? 1 : 4 / WAVES;
    const int lane = threadIdx.x & 63;
    const int tid = WAVES >= 4 ? threadIdx.x : threadIdx.x % THREADS;
    const int wave = tid >> 6;
    const int64_t row = (int64_t)blockIdx.x * GROUPS + (WAVES >= 4 ? 0 : threadIdx.x / THREADS);
    if (WAVES == 1 && row >= a.rows) return;  // whole wave; no barrier below

    const T* x = static_cast<const T*>(a.x) + row * a.xs;
    const T* r = a.r ? static_cast<const T*>(a.r) + row * a.rs : nullptr;
    f32x8 v[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j = (c * THREADS + tid) * 8, n = a.cols - j;
        v[c] = n > 0 ? load8(x + j, n) : f32x8{0, 0, 0, 0, 0, 0, 0, 0};
    }
    if constexpr (MODE != kPlain) {
        if (r) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int j = (c * THREADS + tid) * 8, n = a.cols - j;
                if (n <= 0) continue;
                const f32x8 g = load8(r + j, n);
                if constexpr (MODE == kNorm) {
                    v[c] += g;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c][i] *= silu(g[i]);
                }
            }
        }
    }

    __shared__ float part[2][WAVES > 1 ? WAVES : 1];
    if constexpr (MODE == kNorm) {
        if (a.h) {
            T* h = static_cast<T*>(a.h) + row * a.hs;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int j = (c * THREADS + tid) * 8, n = a.cols - j;
                if (n > 0) store8(h + j, v[c], n);
            }
        }
        auto sum_squares = [&](int turn) {
            float ss = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += v[c][i] * v[c][i];
            ss = lanes_sum(ss);
            if constexpr (WAVES > 1) {
                if (turn) __syncthreads();
                if (lane == 0) part[0][wave] = ss;
                __syncthreads();
                ss = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) ss += part[0][w];
            }
            return ss;
        };
        float ss = sum_squares(0), eps = a.eps;
        const bool over = !(ss < __uint_as_float(kInfBits)), under = ss / (float)a.cols + eps < 0x1p-100f;
        if (over || under) {
            // Squares past float32's range (or an infinity, a NaN), or so small that
            // they lose bits below it: the same norm of the row times 2^-80, or 2^100,
            // whose squares stay in range.
            const float by = over ? 0x1p-80f : 0x1p100f;
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c] *= by;
            eps *= by;
            eps *= by;
            ss = sum_squares(1);
        }
        const float mean = ss / (float)a.cols + eps;
        const float inv = mean == 0.f ? 0.f : 1.f / sqrtf(mean);  // (a row of zeros with eps 0 is zeros)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j = (c * THREADS + tid) * 8, n = a.cols - j;
            if (n <= 0) continue;
            v[c] *= inv;
            if (a.gamma) v[c] *= load8(a.gamma + j, n);
        }
        if (a.y) {
            T* y = static_cast<T*>(a.y) + row * a.ys;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int j = (c * THREADS + tid) * 8, n = a.cols - j;
                if (n > 0) store8(y + j, v[c], n);
            }
        }
        if (!a.q) return;
    }

    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude(v[c][i]));
    top = lanes_max(top);
    if constexpr (WAVES > 1) {
        if (lane == 0) part[1][wave] = __uint_as_float(top);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = max(top, __float_as_uint(part[1][w]));
    }
    const float s = row_scale(top);
    if (tid == 0) a.scale[row] = s;
    int8_t* q = a.q + row * a.qs;
    const int padded = (a.cols + 15) / 16 * 16;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j = (c * THREADS + tid) * 8;
        if (j >= padded) continue;
        *reinterpret_cast<uint2*>(q + j) = quantized8(v[c], s);
    }
}

template <typename T, int MODE, int WAVES, int CH>
hipError_t launch(const RowsArgs& a, hipStream_t st) {
    constexpr int GROUPS = WAVES >= 4 ? 1 : 4 / WAVES;
    // (a launch has fewer than 2^32 threads)
    constexpr int kMost = ((1 << 22) - 1) * GROUPS;
    for (int64_t r0 = 0; r0 < a.rows; r0 += kMost) {
        RowsArgs b = a;
        b.rows = (int)std::min<int64_t>(a.rows - r0, kMost);
        b.x = static_cast<const T*>(a.x) + r0 * a.xs;
        if (a.r) b.r = static_cast<const T*>(a.r) + r0 * a.rs;
        if (a.h) b.h = static_cast<T*>(a.h) + r0 * a.hs;
        if (a.y) b.y = static_cast<T*>(a.y) + r0 * a.ys;
        if (a.q) b.q = a.q + r0 * a.qs, b.scale = a.scale + r0;
        hipLaunchKernelGGL((row_int8<T, MODE, WAVES, CH>), dim3((b.rows + GROUPS - 1) / GROUPS),
                           dim3((WAVES > 4 ? WAVES : 4) * 64), 0, st, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int MODE>
hipError_t dispatch(const RowsArgs& a, hipStream_t st) {
    if (a.cols <= 512) return launch<T, MODE, 1, 1>(a, st);
    if (a.cols <= 2048) return launch<T, MODE, 1, 4>(a, st);
    if (a.rows <= 512) {  // few rows: more waves on each
        if (a.cols <= 8192) return launch<T, MODE, 16, 1>(a, st);
        if (a.cols <= 16384) return launch<T, MODE, 16, 2>(a, st);
    }
    if (a.cols <= 4096) return launch<T, MODE, 4, 2>(a, st);
    if (a.cols <= 8192) return launch<T, MODE, 4, 4>(a, st);
    if (a.cols <= 16384) return launch<T, MODE, 4, 8>(a, st);
    if (a.cols <= 32768) return launch<T, MODE, 16, 4>(a, st);
    return launch<T, MODE, 16, 8>(a, st);
}

template <int MODE>
hipError_t by_type(int dtype, const RowsArgs& a, hipStream_t st) {
    if (dtype == NEO_F32) return dispatch<float, MODE>(a, st);
    if (dtype == NEO_F16) return dispatch<_Float16, MODE>(a, st);
    return dispatch<__bf16, MODE>(a, st);
}

// int8 rows times their scales, each product rounded once: eight elements a
// thread, the rows' groups of eight in one sequence, so that no width leaves
// threads idle.  Memory bounds it: 8192 x 8192 into bfloat16 34 us.
template <typename T>
__global__ __launch_bounds__(256) void dequantize_rows(const int8_t* q, int64_t qs, const float* scale, int rows,
                                                       int cols, T* y, int64_t ys) {
    const int groups = (cols + 7) / 8;
    const int64_t total = (int64_t)rows * groups;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / groups;
        const int j = (int)(t - row * groups) * 8;
        // (eight bytes of a row padded to 16 are all there)
        const uint2 w = *reinterpret_cast<const uint2*>(q + row * qs + j);
        const f32x8 v = dequantized8(w, scale[row]);
        store8(y + row * ys + j, v, cols - j);
    }
}

template <typename T>
hipError_t launch_dequantize(const int8_t* q, int64_t qs, const float* scale, int rows, int cols, void* y, int64_t ys,
                             hipStream_t st) {
    const int64_t threads = (int64_t)rows * ((cols + 7) / 8);
    const unsigned blocks = (unsigned)std::min<int64_t>((threads + 255) / 256, 8192);
    hipLaunchKernelGGL(dequantize_rows<T>, dim3(blocks), dim3(256), 0, st, q, qs, scale, rows, cols, static_cast<T*>(y), ys);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(int dtype, const RowsArgs& a, hipStream_t st) { return by_type<kNorm>(dtype, a, st); }

hipError_t launch_quantize_tokens(int dtype, const RowsArgs& a, hipStream_t st) {
    return a.r ? by_type<kGate>(dtype, a, st) : by_type<kPlain>(dtype, a, st);
}

hipError_t launch_dequantize_tokens(int dtype, const int8_t* q, int64_t qs, const float* scale, int rows, int cols,
                                    void* y, int64_t ys, hipStream_t st) {
    if (dtype == NEO_F32) return launch_dequantize<float>(q, qs, scale, rows, cols, y, ys, st);
    if (dtype == NEO_F16) return launch_dequantize<_Float16>(q, qs, scale, rows, cols, y, ys, st);
    return launch_dequantize<__bf16>(q, qs, scale, rows, cols, y, ys, st);
}

}  // namespace neo
