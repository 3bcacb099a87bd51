// Products of int8 rows and int8 weight rows with a scale per token and per
// channel, on v_mfma_i32_16x16x64_i8:
//
//   y[m][n] = act( (float(sum_k x[m][k] w[n][k]) * xscale[m]) * wscale[n] + bias[n] )
//
// Rows are padded with zeros to a multiple of 16 bytes, so every 16-byte piece
// of a row is whole.  The sums are exact integers: no split of the reduction
// and no order changes a bit.
#include <atomic>
#include <cmath>
#include <type_traits>

#include "token_types.h"

namespace neo {
namespace {

__device__ inline int cdiv_d(int a, int b) { return (a + b - 1) / b; }

__device__ inline float epilogue(int acc, float xs, float ws, const float* bias, int n, int act) {
#pragma clang fp contract(off)
    float v = (float)acc * xs * ws;
    if (bias) v += bias[n];
    return act == NEO_ACT_RELU && v < 0.f ? 0.f : v;  // (a NaN stays one)
}

// Four neighbouring channels of a token, n < N the first; the callers' branch on
// the type lies outside their loops.
template <typename T>
__device__ inline void finish4(const MatmulArgs& a, int m, int n, v4i acc, float xs) {
    typedef float loose4 __attribute__((ext_vector_type(4), aligned(4)));
    T* y = static_cast<T*>(a.y) + m * a.ys + n;
    if (n + 4 <= a.N) {
        const v4f ws = *reinterpret_cast<const loose4*>(a.wscale + n);
        v4f v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = epilogue(acc[r], xs, ws[r], a.bias ? a.bias + n : nullptr, r, a.act);
        store4(y, v);
    } else {
        for (int r = 0; n + r < a.N; ++r)
            y[r] = (T)epilogue(r == 0 ? acc[0] : r == 1 ? acc[1] : acc[2], xs, a.wscale[n + r], a.bias, n + r, a.act);
    }
}
template <typename F>
__device__ inline void by_dtype(int dtype, F&& f) {
    if (dtype == NEO_F32)
        f(0.f);
    else if (dtype == NEO_F16)
        f((_Float16)0);
    else
        f((__bf16)0.f);
}

// ---- few tokens ------------------------------------------------------------------------
// A tile of 16 channels x 16 FM tokens per workgroup; its waves take turns at
// the 128-byte pieces of the rows, U pieces' loads under way at once, and add
// their sums in LDS.  The weights, each read once, bound it: they go straight
// into registers, as no wave shares them, and 16 channels a workgroup with
// eight waves along the reduction put 512 workgroups on 8192 channels.  A token
// times 4096 -> 8192 7.7 us (4.4 TB/s, a launch's 3 us included).
constexpr int kRowWaves = 8;
template <int FM, int U>
__global__ __launch_bounds__(kRowWaves * 64) void matmul_rows(MatmulArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * FM;
    const int8_t* w = a.w + (int64_t)min(n0 + li, a.N - 1) * a.Kp;
    const int8_t* x[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) x[f] = a.x + (int64_t)min(m0 + 16 * f + li, a.M - 1) * a.xs;

    v4i acc[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) acc[f] = v4i{0, 0, 0, 0};
    for (int k = wave * 128; k < a.Kp; k += U * kRowWaves * 128) {
        v4i wv[U][2], xv[U][2][FM];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = k + u * kRowWaves * 128 + h * 64 + g * 16, in = at < a.Kp ? at : 0;  // (past the row: its start, times zero)
                wv[u][h] = *reinterpret_cast<const v4i*>(w + in);
#pragma unroll
                for (int f = 0; f < FM; ++f) xv[u][h][f] = *reinterpret_cast<const v4i*>(x[f] + in);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (k + u * kRowWaves * 128 + h * 64 + g * 16 >= a.Kp) wv[u][h] = v4i{0, 0, 0, 0};
#pragma unroll
                for (int f = 0; f < FM; ++f) acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][h], xv[u][h][f], acc[f], 0, 0, 0);
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

template <int FM, int U>
hipError_t launch_rows(const MatmulArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((matmul_rows<FM, U>), dim3(cdiv(a.N, 16), cdiv(a.M, 16 * FM)), dim3(kRowWaves * 64), 0, st, a);
    return hipGetLastError();
}

// ---- tiles -----------------------------------------------------------------------------
// A workgroup of WM x WN waves computes BM tokens x BN channels in steps of 128
// bytes of the rows.  Both operands' pieces go from memory straight into LDS,
// STAGES - 1 steps ahead; a step is one barrier.  A row's eight 16-byte pieces
// are exchanged by xor with half its number, so that 16 rows, which LDS reads at
// once, lie in all banks; the exchange is made in the global
// address, since a load writes LDS in lane order.  Large products are bound by
// the matrix unit and its clock under that load: 8192^3 in tiles of 256 x 256
// 513 us, 2.14 POP/s (a large library product of int8 1.95 at that size).  Few
// tokens are bound by the weights, and their reduction is split until the chip
// is full: 96 tokens x 16,384 -> 4096 21 us and 4 us to join, 67 MB of weights
// at 3.2 TB/s.
typedef int v16i __attribute__((ext_vector_type(16)));
static __device__ const v4i kZeros = {0, 0, 0, 0};

__device__ inline void load_to_lds(const int8_t* from, char* to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                     (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// All but the N newest loads of this wave are done.
template <int N>
__device__ inline void wait_loads() {
    static_assert(N < 64, "");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
}

template <int BM, int BN, int WM, int WN, int STAGES>
struct Tile {
    static constexpr int WAVES = WM * WN, THREADS = WAVES * 64;
    static constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES, LOADS = LA + LB;  // a wave's loads a step, 8 rows each
    static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;
    static constexpr int STAGE = (BM + BN) * 128, BYTES = STAGE * STAGES;
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "");
};

// steps [k0, k1) of the reduction into acc
template <int BM, int BN, int WM, int WN, int STAGES>
__device__ inline void tile_sums(const MatmulArgs& a, int m0, int n0, int k0, int k1, char* lds,
                                 v16i (&acc)[Tile<BM, BN, WM, WN, STAGES>::MT][Tile<BM, BN, WM, WN, STAGES>::NT]) {
    typedef Tile<BM, BN, WM, WN, STAGES> C;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // A load takes eight rows, 8 j ..; this lane's is lane / 8 of them and its
    // piece of that row (lane & 7) ^ (row / 2 & 7), j's parity deciding bit 2.
    const int piece = (lane & 7) ^ (lane >> 4);
    // this lane's offsets from the tile's first rows (rows past the last: the last)
    const int8_t *xb = a.x + (int64_t)m0 * a.xs, *wb = a.w + (int64_t)n0 * a.Kp;
    uint32_t ao[C::LA], bo[C::LB];
#pragma unroll
    for (int i = 0; i < C::LA; ++i) {
        const int j = wave * C::LA + i;
        ao[i] = (uint32_t)min(j * 8 + (lane >> 3), a.M - 1 - m0) * (uint32_t)a.xs + (piece ^ (j & 1) * 4) * 16;
    }
#pragma unroll
    for (int i = 0; i < C::LB; ++i) {
        const int j = wave * C::LB + i;
        bo[i] = (uint32_t)min(j * 8 + (lane >> 3), a.N - 1 - n0) * (uint32_t)a.Kp + (piece ^ (j & 1) * 4) * 16;
    }

    auto issue = [&](int k, char* stage) {
        char* to = stage + wave * C::LA * 1024;
        const int8_t *xk = xb + (int64_t)k * 128, *wk = wb + (int64_t)k * 128;
        if (k * 128 + 128 <= a.Kp) {
#pragma unroll
            for (int i = 0; i < C::LA; ++i) load_to_lds(xk + ao[i], to + i * 1024);
            to = stage + BM * 128 + wave * C::LB * 1024;
#pragma unroll
            for (int i = 0; i < C::LB; ++i) load_to_lds(wk + bo[i], to + i * 1024);
        } else {
            // the last, shorter step: pieces past the row's end are zeros
            const int8_t* z = reinterpret_cast<const int8_t*>(&kZeros);
            const int end = a.Kp - k * 128;
#pragma unroll
            for (int i = 0; i < C::LA; ++i)
                load_to_lds((piece ^ ((wave * C::LA + i) & 1) * 4) * 16 < end ? xk + ao[i] : z, to + i * 1024);
            to = stage + BM * 128 + wave * C::LB * 1024;
#pragma unroll
            for (int i = 0; i < C::LB; ++i)
                load_to_lds((piece ^ ((wave * C::LB + i) & 1) * 4) * 16 < end ? wk + bo[i] : z, to + i * 1024);
        }
    };
    const int wm = wave / WN, wn = wave % WN, li = lane & 31, half = lane >> 5;
    // byte address of piece 0 of this lane's rows; piece p is that xor 16 p
    const uint32_t ra = (wm * C::MT * 32 + li) * 128 + ((half ^ (li >> 1 & 7)) * 16);
    const uint32_t rb = BM * 128 + (wn * C::NT * 32 + li) * 128 + ((half ^ (li >> 1 & 7)) * 16);

#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s)
        if (k0 + s < k1) issue(k0 + s, lds + s * C::STAGE);
    int at = 0;  // k's stage
    for (int k = k0; k < k1; ++k) {
        if (k + STAGES - 2 < k1)
            wait_loads<(STAGES - 2) * C::LOADS>();
        else
            wait_loads<0>();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();  // step k lies in LDS, and no wave reads step k - 1 any more
        asm volatile("" ::: "memory");
        const int into = at == 0 ? STAGES - 1 : at - 1;
        if (k + STAGES - 1 < k1) issue(k + STAGES - 1, lds + into * C::STAGE);
        const char* stage = lds + at * C::STAGE;
        v4i av[2][C::MT], bv[2][C::NT];
        auto read = [&](int s) {
#pragma unroll
            for (int i = 0; i < C::MT; ++i) av[s & 1][i] = *reinterpret_cast<const v4i*>(stage + (ra ^ (s * 32)) + i * 4096);
#pragma unroll
            for (int j = 0; j < C::NT; ++j) bv[s & 1][j] = *reinterpret_cast<const v4i*>(stage + (rb ^ (s * 32)) + j * 4096);
        };
        read(0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s < 3) read(s + 1);
#pragma unroll
            for (int i = 0; i < C::MT; ++i)
#pragma unroll
                for (int j = 0; j < C::NT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bv[s & 1][j], av[s & 1][i], acc[i][j], 0, 0, 0);
        }
        // the next quarter's reads between this one's products
        __builtin_amdgcn_sched_group_barrier(0x100, C::MT + C::NT, 0);
#pragma unroll
        for (int s = 0; s < 3; ++s) {
#pragma unroll
            for (int i = 0; i < C::MT + C::NT; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            if constexpr (C::MT * C::NT > C::MT + C::NT) __builtin_amdgcn_sched_group_barrier(0x008, C::MT * C::NT - C::MT - C::NT, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, C::MT * C::NT, 0);
        at = at == STAGES - 1 ? 0 : at + 1;
    }
}

template <int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM * WN * 64) void matmul_tile(MatmulArgs a, int splits, int* ws) {
    typedef Tile<BM, BN, WM, WN, STAGES> C;
    extern __shared__ __align__(256) char lds[];
    const int tiles_n = cdiv_d(a.N, BN), tiles_m = cdiv_d(a.M, BM), tiles = tiles_n * tiles_m;
    // neighbouring tiles on one die (workgroups go to the 8 dies in turn), in
    // bands of 8 tiles of tokens, channel by channel
    const int total = tiles * splits, per = total / 8, rest = total % 8, die = blockIdx.x % 8;
    const int at = die * per + min(die, rest) + blockIdx.x / 8;
    const int split = at / tiles, t = at - split * tiles;
    const int band = t / (8 * tiles_n), height = min(8, tiles_m - band * 8), in = t - band * 8 * tiles_n;
    const int m0 = (band * 8 + in % height) * BM, n0 = in / height * BN;
    const int steps = cdiv_d(a.Kp, 128), k0 = (int)((int64_t)steps * split / splits), k1 = (int)((int64_t)steps * (split + 1) / splits);

    v16i acc[C::MT][C::NT];
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
        for (int j = 0; j < C::NT; ++j) acc[i][j] = v16i{0};
    tile_sums<BM, BN, WM, WN, STAGES>(a, m0, n0, k0, k1, lds, acc);

    // acc[i][j][4 q + r]: token 32 i + li, channel 32 j + 8 q + 4 half + r of the
    // wave's part.  Each wave turns 32 tokens at a time in its own piece of LDS,
    // so that neighbouring lanes store neighbouring channels.
    constexpr int CN = C::NT * 32, ROW = CN + 4, LANES = CN / 4;
    static_assert(C::WAVES * 32 * ROW * 4 <= C::BYTES, "");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN, li = lane & 31, half = lane >> 5;
    int* turn = reinterpret_cast<int*>(lds) + wave * 32 * ROW;
    __syncthreads();
    const int nn = lane % LANES * 4, n = n0 + wn * CN + nn;
    auto finish = [&](auto zero) {
#pragma unroll
        for (int i = 0; i < C::MT; ++i) {
#pragma unroll
            for (int j = 0; j < C::NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<v4i*>(turn + li * ROW + 32 * j + 8 * q + 4 * half) =
                        v4i{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            // (a wave's LDS operations are done in order)
            asm volatile("" ::: "memory");
#pragma unroll
            for (int p = 0; p < 32; p += 64 / LANES) {
                const int mm = p + lane / LANES, m = m0 + (wm * C::MT + i) * 32 + mm;
                const v4i s = *reinterpret_cast<const v4i*>(turn + mm * ROW + nn);
                if (m < a.M && n < a.N) {
                    if constexpr (std::is_same<decltype(zero), int>::value)
                        *reinterpret_cast<v4i*>(ws + ((int64_t)split * a.M + m) * ((a.N + 3) & ~3) + n) = s;
                    else
                        finish4<decltype(zero)>(a, m, n, s, a.xscale[m]);
                }
            }
            asm volatile("" ::: "memory");
        }
    };
    if (splits > 1)
        finish(0);
    else
        by_dtype(a.dtype, finish);
}

// The splits' sums, added, and the epilogue: four channels a thread.  Sums of
// integers: the same bits as in one piece.  (96 x 4096 of four splits 3.9 us.)
__global__ __launch_bounds__(256) void matmul_join(MatmulArgs a, int splits, const int* ws) {
    const int quads = (a.N + 3) / 4;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, m = t / quads;
    if (m >= a.M) return;
    const int n = (int)(t - m * quads) * 4;
    const int* p = ws + m * (quads * 4) + n;
    v4i s = {0, 0, 0, 0};
    for (int i = 0; i < splits; ++i) s += *reinterpret_cast<const v4i*>(p + (int64_t)i * a.M * (quads * 4));
    by_dtype(a.dtype, [&](auto zero) { finish4<decltype(zero)>(a, (int)m, n, s, a.xscale[m]); });
}

template <int BM, int BN, int WM, int WN, int STAGES>
hipError_t launch_tile(const MatmulArgs& a, int splits, float* ws, hipStream_t st) {
    typedef Tile<BM, BN, WM, WN, STAGES> C;
    // (more LDS than a kernel gets unasked; set once per device)
    static std::atomic<uint64_t> asked{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !(asked.load() >> dev & 1)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&matmul_tile<BM, BN, WM, WN, STAGES>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
        if (e != hipSuccess) return e;
        if (dev >= 0 && dev < 64) asked.fetch_or(1ull << dev);
    }
    const unsigned blocks = (unsigned)cdiv(a.M, BM) * cdiv(a.N, BN) * splits;
    hipLaunchKernelGGL((matmul_tile<BM, BN, WM, WN, STAGES>), dim3(blocks), dim3(C::THREADS), C::BYTES, st, a, splits, reinterpret_cast<int*>(ws));
    e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    const int64_t threads = (int64_t)a.M * ((a.N + 3) / 4);
    hipLaunchKernelGGL(matmul_join, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a, splits, reinterpret_cast<const int*>(ws));
    return hipGetLastError();
}

// The time in us of each way, from what the tiles measured on the chip, and the
// least of them.
struct Choice {
    int kind, splits;  // kind 0: matmul_rows
};
enum { kRows, k256x256, k128x128, k64x128, k64x64, k32x128 };
struct Cost {
    int kind, bm, bn;
    int resident;      // workgroups a CU holds
    float step[2];     // us a step of 128 with one workgroup a CU, with all
};
// (256 x 256: 2.3 us a step is 1.87 POP/s; 8192^3 at the same clock 587 us against 648 in tiles of
// 128 x 128; 1003 x 2049 -> 1001 12.2 us in 64 x 64 and 12.5 in 32 x 128, which the
// costs prefer by half a microsecond, against 17.4 in 64 x 128 and 24.7 in 128 x 128;
// 32 x 16,384 -> 4096 17.6 us in 32 x 128 against 18.3 in 64 x 64;
// 96 x 16,384 -> 4096 24.5 us in 64 x 128 and four splits, 68.9 by matmul_rows)
constexpr Cost kCosts[] = {{k256x256, 256, 256, 1, {2.3f, 2.3f}}, {k128x128, 128, 128, 2, {0.9f, 1.27f}},
                           {k64x128, 64, 128, 1, {0.56f, 0.56f}}, {k64x64, 64, 64, 2, {0.48f, 0.58f}},
                           {k32x128, 32, 128, 2, {0.45f, 0.7f}}};

Choice choose(const MatmulArgs& a) {
    // (the tiles' row offsets are 32-bit)
    if (a.M <= 16 || a.xs > (1 << 23)) return Choice{kRows, 1};
    const int steps = cdiv(a.Kp, 128);
    Choice best{kRows, 1};
    // matmul_rows: 1024 bytes of the rows a turn; its tiles of 32 or 64 tokens
    // load their operands through the L1 (24 x 1000 -> 300 3.5 us against 6.0 in tiles)
    const float turn = (float)cdiv(a.N, 16) * cdiv(a.M, a.M <= 32 ? 32 : 64) / 256 * (a.M <= 32 ? 1.4f : 2.4f);
    float least = 2.f + (float)cdiv(a.Kp, 1024) * std::max(1.2f, turn);
    if (a.M > 64 * 65535) least = INFINITY;  // (past the grid's y)
    for (const Cost& c : kCosts) {
        const int64_t tiles = (int64_t)cdiv(a.M, c.bm) * cdiv(a.N, c.bn);
        for (int splits = 1; splits <= 16 && splits <= steps; splits *= 2) {
            const int64_t groups = tiles * splits;
            if (groups > 1 << 22 || (splits > 1 && groups > 4096)) break;  // (2^32 threads a launch)
            const int64_t full = 256 * c.resident;
            const float step = groups <= 256 ? c.step[0] : c.step[1];
            float us = 3.5f + (float)((groups + full - 1) / full) * cdiv(steps, splits) * step;
            // the partial sums are written and read, by a launch of its own
            if (splits > 1) us += 2.5f + (float)((int64_t)splits * a.M * a.N * 8) / 3.5e6f;
            if (us < least) least = us, best = Choice{c.kind, splits};
        }
    }
    return best;
}

}  // namespace

size_t matmul_int8_workspace(const MatmulArgs& a) {
    const Choice c = choose(a);
    return c.splits > 1 ? (size_t)c.splits * a.M * ((a.N + 3) & ~3) * sizeof(int) : 0;
}

hipError_t launch_matmul_int8(const MatmulArgs& a, float* ws, hipStream_t st) {
    const Choice c = choose(a);
    switch (c.kind) {
        case k256x256: return launch_tile<256, 256, 2, 4, 2>(a, c.splits, ws, st);
        case k128x128: return launch_tile<128, 128, 2, 2, 2>(a, c.splits, ws, st);
        case k64x128: return launch_tile<64, 128, 1, 4, 4>(a, c.splits, ws, st);
        case k64x64: return launch_tile<64, 64, 2, 2, 4>(a, c.splits, ws, st);
        case k32x128: return launch_tile<32, 128, 1, 4, 4>(a, c.splits, ws, st);
    }
    if (a.M <= 16) return launch_rows<1, 4>(a, st);
    if (a.M <= 32) return launch_rows<2, 2>(a, st);
    return launch_rows<4, 1>(a, st);
}

}  // namespace neo
