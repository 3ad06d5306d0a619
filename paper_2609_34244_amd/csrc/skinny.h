// Products with few rows of X (single tokens): Y[m][n] = sum over k of X[m][k] W[n][k].
//
// Bound by reading W once. A workgroup of WAVES wavefronts takes 16 rows of W
// (gated: 16 gate and 16 up rows) and every row of X, 16 MB at a time; each
// wavefront takes its part of k. W goes from memory straight to the registers that the
// matrix instruction reads (16 rows x 32 k, lane = row, 16 bytes of k), U pieces of W in
// flight per lane, and X, which the caches hold, beside it. The wavefronts' sums meet in LDS in a
// fixed order. Loads need only the alignment of a value, so no operand is copied. One row of
// 4096 x 4096: 10.4 us, 3.2 TB/s of W from memory (8.4 us from the memory-side cache); of
// 2 x 10816 x 4096, gated: 34.5 us, 5.1 TB/s (a large copy moves 4.8).
//
// Groups: a workgroup takes the j-th group that has rows; there are at most as many as rows.
#pragma once

#include <type_traits>

#include "gemm.h"

namespace heddle {
namespace mm {

// group j of those with rows; false past the last one
__device__ inline bool find_group(const int32_t *offsets, int groups, int total, int j, int &g, int &lo, int &hi)
{
    int carry = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
        int a, b;
        group_ranges(offsets, groups, total, g0, carry, a, b);
        uint64_t has = __ballot(b > a);
        const int n = __popcll(has);
        if (j < n) {
            for (; j > 0; j--) has &= has - 1;
            const int l = __builtin_ctzll(has);
            g = __builtin_amdgcn_readfirstlane(g0 + l);
            lo = __builtin_amdgcn_readfirstlane(__shfl(a, l));
            hi = __builtin_amdgcn_readfirstlane(__shfl(b, l));
            return true;
        }
        j -= n;
        carry = __builtin_amdgcn_readlane(b, 63);
    }
    return false;
}

// 8 H values at any address that values may have. H = 2: by whole words, as loads of 16 bytes
// at odd multiples of 2 run at half the rate (20000 x 4096, one row: 73 us; 59 by words for
// each eight, 53 for sixteen; 42 at multiples of 4); no word without one of the values is read.
template <int H, typename T> __device__ inline void load_any(const T *p, typename pack8<T>::type *v)
{
    if (H == 1) {
        __builtin_memcpy(v, p, 16);
        return;
    }
    const uint32_t *words = (const uint32_t *)((uintptr_t)p & ~(uintptr_t)3), skew = (uint32_t)((uintptr_t)p & 2);
    uint32_t w[4 * H + 1];
    __builtin_memcpy(w, words, 16 * H);
    w[4 * H] = words[4 * H - 1 + skew / 2];
#pragma unroll
    for (int i = 0; i < 4 * H; i++) w[i] = __builtin_amdgcn_alignbyte(w[i + 1], w[i], skew);
    __builtin_memcpy(v, w, 16 * H);
}
// the values with index below count; the others are zero and not read
template <typename T> __device__ inline typename pack8<T>::type load_some(const T *p, int count)
{
    typename pack8<T>::type v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < count ? p[i] : (T)0.0f;
    return v;
}

template <int MB, int WAVES, bool ODD, typename T, typename Epi>
__global__ void __launch_bounds__(WAVES * 64) skinny_kernel(Args x, Epi epi)
{
    constexpr bool PAIR = Epi::gated;
    constexpr int P = PAIR ? 2 : 1, H = ODD ? 2 : 1, U = (MB * P > 1 ? 4 : 8) / H;   // H eights of k a lane and step
    typedef typename pack8<T>::type frag;
    __shared__ float part[WAVES][P * MB * 256], sum[P * MB * 256];
    const int lane = threadIdx.x & 63, i = lane & 15, kg = (lane >> 4) * 8 * H;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int g = 0, lo = 0, hi = x.M;
    if (x.offsets && !find_group(x.offsets, x.groups, x.M, blockIdx.y, g, lo, hi)) return;
    const int n0 = blockIdx.x * 16;
    const T *w = (const T *)x.b + (int64_t)g * x.stride_b + (int64_t)min(n0 + i, x.N - 1) * x.ldb;
    const int64_t up = PAIR ? (int64_t)x.F * x.ldb : 0;
    // whole steps (32 k, 64 for ODD) of this wavefront, and the last, partial one
    const int steps = x.K / (32 * H), each = (steps + WAVES - 1) / WAVES;
    const int first = min(wave * each, steps), last = min(first + each, steps);
    for (int m0 = lo; m0 < hi; m0 += 16 * MB) {
        const T *xr[MB];
#pragma unroll
        for (int b = 0; b < MB; b++) xr[b] = (const T *)x.a + (int64_t)min(m0 + b * 16 + i, hi - 1) * x.lda;
        f32x4 acc[P][MB];
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int b = 0; b < MB; b++) acc[p][b] = f32x4{0, 0, 0, 0};
        int s = first;
        // n steps: all their loads, then their products
        auto batch = [&](auto n) {
            constexpr int N = decltype(n)::value;
            frag fw[P][N][H], fx[MB][N][H];
#pragma unroll
            for (int u = 0; u < N; u++) {
                const int k = (s + u) * 32 * H + kg;
#pragma unroll
                for (int p = 0; p < P; p++) load_any<H>(w + p * up + k, fw[p][u]);
#pragma unroll
                for (int b = 0; b < MB; b++) load_any<H>(xr[b] + k, fx[b][u]);
            }
#pragma unroll
            for (int u = 0; u < N * H; u++)
#pragma unroll
                for (int p = 0; p < P; p++)
#pragma unroll
                    for (int b = 0; b < MB; b++) acc[p][b] = mfma(fw[p][u / H][u % H], fx[b][u / H][u % H], acc[p][b]);
            s += N;
        };
        while (s + U <= last) batch(std::integral_constant<int, U>());
        if (U > 4 && s + 4 <= last) batch(std::integral_constant<int, 4>());
        if (U > 2 && s + 2 <= last) batch(std::integral_constant<int, 2>());
        if (s < last) batch(std::integral_constant<int, 1>());
        if (wave == WAVES - 1 && x.K % (32 * H)) {
#pragma unroll
            for (int h = 0; h < H; h++) {
                const int k = steps * 32 * H + kg + h * 8, count = x.K - k;
                frag fx[MB];
#pragma unroll
                for (int b = 0; b < MB; b++) fx[b] = load_some(xr[b] + k, count);
#pragma unroll
                for (int p = 0; p < P; p++) {
                    const frag fw = load_some(w + p * up + k, count);
#pragma unroll
                    for (int b = 0; b < MB; b++) acc[p][b] = mfma(fw, fx[b], acc[p][b]);
                }
            }
        }
        // a lane holds row i of X and rows 4 (lane / 16) .. + 3 of W: [p][b][row of X][row of W]
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int b = 0; b < MB; b++) *(f32x4 *)&part[wave][((p * MB + b) * 16 + i) * 16 + (lane >> 4) * 4] = acc[p][b];
        __syncthreads();
        for (int c = threadIdx.x; c < P * MB * 256; c += WAVES * 64) {
            float v = 0;
#pragma unroll
            for (int q = 0; q < WAVES; q++) v += part[q][c];
            sum[c] = v;
        }
        __syncthreads();
        if (threadIdx.x < MB * 32) {
            const int r = threadIdx.x >> 1, n = n0 + (threadIdx.x & 1) * 8, m = m0 + r;
            if (m < hi && n < x.N) {
                const float *at = sum + r * 16 + (threadIdx.x & 1) * 8;
                float v[8], u[8];
#pragma unroll
                for (int q = 0; q < 8; q++) {
                    v[q] = at[q];
                    if (PAIR) u[q] = at[MB * 256 + q];
                }
                if constexpr (PAIR) epi(m, n, g, v, u);
                else epi(m, n, g, v);
            }
        }
    }
}

// Whether it is the faster way. A row costs it what X's loads add to those of W, which tiles of
// 64 rows do not have; they need a second launch, that joins parts of k, and where an operand's
// rows are not on 4-byte boundaries a copy of it. us with it / with tiles:
//   4096 x 4096: 1 row 10.7 / 15.1, 32 rows 14.0 / 14.2;  8192 x 8192: 1 row 30.4 / 30.7, 8 rows
//   35.9 / 31.1;  4096 x 10816: 4 rows 23.0 / 21.2;  20000 x 4096 with odd rows: 8 rows 63 / about
//   105, 32 rows 119 / about 107;  at the bound on m n k, 24032 x 8192: 1 row 80.6 / 93.2;  past it,
//   48064 x 8192: 1 row 157 / 170, 128000 x 8192: 391 / 375, 24032 x 8192: 4 rows 89 / 95.
// Groups, forward pass of the block: 64 of 4096 x 1632: 2 rows each 349 / 379, 4: 435 / 427, 8:
//   595 / 460;  8 of 4096 x 816: 2: 33 / 49, 4: 56 / 52;  32 of 4096 x 204: 2: 37 / 48, 6: 71 / 60.
inline bool is_skinny(int64_t m, int64_t n, int64_t k, int groups, bool copied)
{
    if (groups) return m <= (copied ? 10 : 3) * (int64_t)groups;
    return copied ? m <= 16 : m <= 32 && m * n * k <= 1 << 28;
}

template <int MB, int WAVES, typename T, typename Epi>
inline void launch_skinny_cfg(const Args &x, const Epi &epi, unsigned groups, hipStream_t stream)
{
    const bool odd = (((uintptr_t)x.a | (uintptr_t)x.b) & 2) || ((x.lda | x.ldb | x.stride_b) & 1);
    const dim3 grid((unsigned)((x.N + 15) / 16), groups);
    if (odd) hipLaunchKernelGGL((skinny_kernel<MB, WAVES, true, T, Epi>), grid, dim3(WAVES * 64), 0, stream, x, epi);
    else hipLaunchKernelGGL((skinny_kernel<MB, WAVES, false, T, Epi>), grid, dim3(WAVES * 64), 0, stream, x, epi);
}

template <typename T, typename Epi> inline int launch_skinny(const Args &x, const Epi &epi, hipStream_t stream)
{
    const unsigned blocks = (unsigned)((x.N + 15) / 16);
    const unsigned groups = x.offsets ? (unsigned)(x.groups < x.M ? x.groups : x.M) : 1;
    // k is divided among 16 wavefronts where each has eight pieces of W to load at once, twice
    // over (4096 x 10816, one row: 17.0 us, 20.4 with 8), else among 8, or 4 where there are
    // workgroups enough for the chip without (experts of 4096 x 1632: 66 us, 83 with 8). A gated
    // workgroup has as much in flight with 8 and half the pieces (2 x 10816 x 4096: 35 us, 37
    // with 16 wavefronts, 44 with twice the pieces and half the workgroups on a CU).
    const bool one = x.offsets || x.M <= 16;
    const int waves = Epi::gated ? 8 : x.K >= 16 * 8 * 32 ? 16 : blocks * groups >= 4 * 256 ? 4 : 8;
    auto run = [&](auto w) {
        constexpr int WAVES = decltype(w)::value;
        if (one) launch_skinny_cfg<1, WAVES, T>(x, epi, groups, stream);
        else launch_skinny_cfg<2, WAVES, T>(x, epi, groups, stream);
    };
    if (waves == 8) run(std::integral_constant<int, 8>());
    if constexpr (!Epi::gated) {
        if (waves == 16) run(std::integral_constant<int, 16>());
        if (waves == 4) run(std::integral_constant<int, 4>());
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "skinny_kernel");
}

}  // namespace mm
}  // namespace heddle
