// Products of int8 rows and int8 weight rows with a scale per token and per
// channel, on v_mfma_i32_16x16x64_i8:
//
//   y[m][n] = act( (float(sum_k x[m][k] w[n][k]) * xscale[m]) * wscale[n] + bias[n] )
//
// Rows are padded with zeros to a multiple of 16 bytes, so every 16-byte piece
// of a row is whole.  The sums are exact integers: no split of the reduction
// and no order changes a bit.
#include "token_types.h"

namespace neo {
namespace {

__device__ inline float epilogue(int acc, float xs, float ws, const float* bias, int n, int act) {
#pragma clang fp contract(off)
    float v = (float)acc * xs * ws;
    if (bias) v += bias[n];
    return act == NEO_ACT_RELU ? fmaxf(v, 0.f) : v;
}

// A tile of 16 channels x 16 FM tokens per workgroup; its waves take turns at
// the 128-byte pieces of the rows and add their sums in LDS.
constexpr int kRowWaves = 8;
template <int FM>
__global__ __launch_bounds__(kRowWaves * 64) void matmul_rows(MatmulArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * FM;
    const int8_t* w = a.w + (int64_t)min(n0 + li, a.N - 1) * a.Kp + g * 16;
    const int8_t* x[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) x[f] = a.x + (int64_t)min(m0 + 16 * f + li, a.M - 1) * a.xs + g * 16;

    v4i acc[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) acc[f] = v4i{0, 0, 0, 0};
    const v4i zero = {0, 0, 0, 0};
    for (int k = wave * 128; k < a.Kp; k += kRowWaves * 128) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = k + h * 64;
            const bool in = at + g * 16 < a.Kp;  // (past the row: its start, times zero)
            v4i wv = *reinterpret_cast<const v4i*>(w + (in ? at : 0));
            if (!in) wv = zero;
#pragma unroll
            for (int f = 0; f < FM; ++f) {
                const v4i xv = *reinterpret_cast<const v4i*>(x[f] + (in ? at : 0));
                acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, acc[f], 0, 0, 0);
            }
        }
    }

    __shared__ int part[kRowWaves][FM][4][64];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][f][r][lane] = acc[f][r];
    __syncthreads();
    for (int t = threadIdx.x; t < FM * 256; t += kRowWaves * 64) {
        // consecutive threads: the 16 channels of a token
        const int f = t >> 8, nn = t & 15, mm = (t >> 4) & 15;
        const int n = n0 + nn, m = m0 + f * 16 + mm;
        if (n >= a.N || m >= a.M) continue;
        int s = 0;
#pragma unroll
        for (int v = 0; v < kRowWaves; ++v) s += part[v][f][nn & 3][(nn >> 2) * 16 + mm];
        store1(a.y, m * a.ys + n, epilogue(s, a.xscale[m], a.wscale[n], a.bias, n, a.act), a.dtype);
    }
}

template <int FM>
hipError_t launch_rows(const MatmulArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(matmul_rows<FM>, dim3(cdiv(a.N, 16), cdiv(a.M, 16 * FM)), dim3(kRowWaves * 64), 0, st, a);
    return hipGetLastError();
}

}  // namespace

size_t matmul_int8_workspace(const MatmulArgs&) { return 0; }

hipError_t launch_matmul_int8(const MatmulArgs& a, float*, hipStream_t st) {
    if (a.M <= 16) return launch_rows<1>(a, st);
    if (a.M <= 32) return launch_rows<2>(a, st);
    return launch_rows<4>(a, st);
}

}  // namespace neo
