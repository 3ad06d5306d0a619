// Layer normalisation and its gradients on gfx950.
//
// mean = sum x / n, rstd = 1 / sqrt(sum (x - mean)^2 / n + eps), xh = (x - mean) rstd, y = xh w + b;
// g = dy w, dx = rstd (g - mean(g) - xh mean(g xh)) + r, dw = sum over rows of dy xh, db of dy.
// Memory is read and written once: a row is read once and stays in registers, TPR lanes to a row, K pieces of 16
// bytes a lane; the variance is summed from the differences to the mean, so that a mean far from
// zero costs no digits. All sums are fp32.
// The backward pass takes a row at a time in each of its workgroups (several where a row needs
// less than one), so that a lane keeps its columns' sums of dy xh and dy in registers; a second
// kernel adds up the workgroups' sums, in one order. The next row's loads are in flight while a
// row's two sums are formed. 4096 rows of 4096, bf16: forward 20 us (3.4 TB/s), backward with a residual 34 + 4.4 us (3.9 TB/s
// without the sums), wavefronts waiting 62 and 55% of the time: forward, each workgroup has one row, and reads the weights and
// shifts for it from the caches, as many requests to the L2 as for the row. Rows of more than 512 kLongest values are read again instead.
#include <algorithm>
#include <cmath>

#include "linear.h"

namespace heddle {
namespace norm {

using mm::Region;
using mm::Scratch;

struct Args {
    const void *x, *w, *bias, *dy, *residual;
    void *y, *dx, *dw, *db;
    float *stats;                             // [m][2]: mean, rstd
    float *partial;                           // [blocks][2][n]: sums of dy xh, of dy
    int64_t ldx, ldy, lddy, ldr, lddx, m;
    int32_t n, wide;                          // wide: w, bias, dw and db are fp32
    float eps, inv_n;
};

template <typename T> struct Piece {
    static constexpr int V = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef T loose __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));   // at any address its values may have
};

// The values from column c on, those past the row's end 0. WHOLE: rows end with a piece, and no load
// waits for a test of the end (4096 rows of 4096 in bf16, forward: 19.8 us, 20.4 with the tests).
template <typename T, bool WHOLE = false> __device__ inline typename Piece<T>::type load(const T *row, int c, int n)
{
    typename Piece<T>::type v = {};
    if (c + Piece<T>::V <= n) return *(const typename Piece<T>::loose *)(row + c);
    if (WHOLE || c >= n) return v;
    // a row's end: loads of which none waits for a test
#pragma unroll
    for (int i = 0; i < Piece<T>::V; i++) v[i] = row[min(c + i, n - 1)];
#pragma unroll
    for (int i = 1; i < Piece<T>::V; i++) v[i] = c + i < n ? v[i] : (T)0.0f;
    return v;
}
template <typename T> __device__ inline void store(T *row, int c, int n, typename Piece<T>::type v)
{
    if (c + Piece<T>::V <= n) {
        *(typename Piece<T>::loose *)(row + c) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < Piece<T>::V; i++)
        if (c + i < n) row[c + i] = v[i];
}
// V weights from column c on: of the rows' type or fp32
template <typename T, bool WHOLE> __device__ inline void load_weights(const void *w, int wide, int c, int n, float other, float v[Piece<T>::V])
{
    constexpr int V = Piece<T>::V;
    if (!w) {
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = other;
    } else if (wide) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const auto p = load<float, WHOLE>((const float *)w, c + i, n);
#pragma unroll
            for (int j = 0; j < 4; j++) v[i + j] = p[j];
        }
    } else {
        const auto p = load<T, WHOLE>((const T *)w, c, n);
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = (float)p[i];
    }
}

// Sums over a row's TPR lanes, in every one of them, in a fixed order. `lds`: one float2 a wavefront, two sets
// used in turn, so that one barrier is enough.
template <int TPR> __device__ inline float2 row_sum(float2 s, float2 (*lds)[16], int turn)
{
#pragma unroll
    for (int d = (TPR < 64 ? TPR : 64) / 2; d; d /= 2) s.x += __shfl_xor(s.x, d), s.y += __shfl_xor(s.y, d);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = s;
        __syncthreads();
        s = lds[turn][0];
#pragma unroll
        for (int i = 1; i < TPR / 64; i++) s.x += lds[turn][i].x, s.y += lds[turn][i].y;
    }
    return s;
}

constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

template <typename T, int TPR, int K, bool WHOLE> __device__ __attribute__((always_inline)) inline void forward_rows(const Args &a, float2 (*lds)[16])
{
    constexpr int V = Piece<T>::V, kRows = block_of(TPR) / TPR;
    const int lane = threadIdx.x % TPR;
    float w[K][V], b[K][V];
#pragma unroll
    for (int k = 0; k < K; k++) {
        load_weights<T, WHOLE>(a.w, a.wide, (k * TPR + lane) * V, a.n, 1.0f, w[k]);
        load_weights<T, WHOLE>(a.bias, a.wide, (k * TPR + lane) * V, a.n, 0.0f, b[k]);
    }
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.m; first += (int64_t)gridDim.x * kRows) {
        const int64_t r = first + threadIdx.x / TPR;
        const bool any = r < a.m;                           // (all lanes' where TPR > 64)
        const T *row = (const T *)a.x + (any ? r : a.m - 1) * a.ldx;
        typename Piece<T>::type x[K];
#pragma unroll
        for (int k = 0; k < K; k++) x[k] = load<T, WHOLE>(row, (k * TPR + lane) * V, a.n);
        float2 s = {0, 0};
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int i = 0; i < V; i++) s.x += (float)x[k][i];
        const float mean = row_sum<TPR>(s, lds, 0).x * a.inv_n;
        s = {0, 0};
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int i = 0; i < V; i++) {
                const float d = (k * TPR + lane) * V + i < a.n ? (float)x[k][i] - mean : 0.0f;
                s.x += d * d;
            }
        const float rstd = rsqrtf(row_sum<TPR>(s, lds, 1).x * a.inv_n + a.eps);
        if (!any) continue;
        if (a.stats && lane == 0) *(float2 *)(a.stats + 2 * r) = {mean, rstd};
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int c = (k * TPR + lane) * V;
            if (c >= a.n) break;
            typename Piece<T>::type y;
#pragma unroll
            for (int i = 0; i < V; i++) y[i] = (T)(((float)x[k][i] - mean) * rstd * w[k][i] + b[k][i]);
            store<T>((T *)a.y + r * a.ldy, c, a.n, y);
        }
    }
}

template <typename T, int TPR, int K> __global__ void __launch_bounds__(block_of(TPR)) forward_kernel(Args a)
{
    __shared__ float2 lds[2][16];
    if (a.n % Piece<T>::V == 0) forward_rows<T, TPR, K, true>(a, lds);
    else forward_rows<T, TPR, K, false>(a, lds);
}

// rows that do not fit in registers: three readings, the later two from the caches
template <typename T> __global__ void __launch_bounds__(1024) forward_long_kernel(Args a)
{
    constexpr int V = Piece<T>::V;
    __shared__ float2 lds[2][16];
    for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x) {
        const T *row = (const T *)a.x + r * a.ldx;
        float2 s = {0, 0};
        for (int c = threadIdx.x * V; c < a.n; c += 1024 * V) {
            const auto x = load<T>(row, c, a.n);
#pragma unroll
            for (int i = 0; i < V; i++) s.x += (float)x[i];
        }
        const float mean = row_sum<1024>(s, lds, 0).x * a.inv_n;
        s = {0, 0};
        for (int c = threadIdx.x * V; c < a.n; c += 1024 * V) {
            const auto x = load<T>(row, c, a.n);
#pragma unroll
            for (int i = 0; i < V; i++) {
                const float d = c + i < a.n ? (float)x[i] - mean : 0.0f;
                s.x += d * d;
            }
        }
        const float rstd = rsqrtf(row_sum<1024>(s, lds, 1).x * a.inv_n + a.eps);
        if (a.stats && threadIdx.x == 0) *(float2 *)(a.stats + 2 * r) = {mean, rstd};
        for (int c = threadIdx.x * V; c < a.n; c += 1024 * V) {
            const auto x = load<T>(row, c, a.n);
            float w[V], b[V];
            load_weights<T, false>(a.w, a.wide, c, a.n, 1.0f, w);
            load_weights<T, false>(a.bias, a.wide, c, a.n, 0.0f, b);
            typename Piece<T>::type y;
#pragma unroll
            for (int i = 0; i < V; i++) y[i] = (T)(((float)x[i] - mean) * rstd * w[i] + b[i]);
            store<T>((T *)a.y + r * a.ldy, c, a.n, y);
        }
    }
}

// SUMS: the sums for dw and db too
template <typename T, int TPR, int K, bool SUMS, bool WHOLE> __device__ __attribute__((always_inline)) inline void backward_rows(const Args &a, float2 (*lds)[16], float *part)
{
    constexpr int V = Piece<T>::V, kRows = block_of(TPR) / TPR;
    typedef typename Piece<T>::type piece;
    const int lane = threadIdx.x % TPR;
    const int64_t step = (int64_t)gridDim.x * kRows;
    float w[K][V], sw[K][V], sb[K][V];
#pragma unroll
    for (int k = 0; k < K; k++) {
        load_weights<T, WHOLE>(a.w, a.wide, (k * TPR + lane) * V, a.n, 1.0f, w[k]);
#pragma unroll
        for (int i = 0; i < V; i++) sw[k][i] = sb[k][i] = 0;
    }
    piece x[K], g[K], nx[K], ng[K];
    float2 st, nst;
    // a workgroup's rows end together: lanes without a row take part with dy = 0
    auto fetch = [&](int64_t first) {
        const int64_t r = first + threadIdx.x / TPR;
        const bool any = r < a.m;
        const int64_t at = any ? r : a.m - 1;
        nst = *(const float2 *)(a.stats + 2 * at);
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int c = (k * TPR + lane) * V;
            nx[k] = load<T, WHOLE>((const T *)a.x + at * a.ldx, c, a.n);
            ng[k] = load<T, WHOLE>((const T *)a.dy + at * a.lddy, c, any ? a.n : 0);
        }
    };
    int64_t first = (int64_t)blockIdx.x * kRows;
    if (first < a.m) fetch(first);
    for (int turn = 0; first < a.m; first += step, turn ^= 1) {
        st = nst;
#pragma unroll
        for (int k = 0; k < K; k++) x[k] = nx[k], g[k] = ng[k];
        if (first + step < a.m) fetch(first + step);
        const int64_t r = first + threadIdx.x / TPR;
        const bool any = r < a.m;
        piece res[K];
        const bool add = a.dx && a.residual && any;
#pragma unroll
        for (int k = 0; k < K; k++)
            if (add) res[k] = load<T, WHOLE>((const T *)a.residual + r * a.ldr, (k * TPR + lane) * V, a.n);
        float2 s = {0, 0};
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int i = 0; i < V; i++) {
                const bool in = any && (k * TPR + lane) * V + i < a.n;
                const float dy = (float)g[k][i], xh = in ? ((float)x[k][i] - st.x) * st.y : 0.0f;
                if constexpr (SUMS) sw[k][i] += dy * xh, sb[k][i] += dy;
                s.x += dy * w[k][i];
                s.y += dy * w[k][i] * xh;
            }
        if (!a.dx) continue;
        s = row_sum<TPR>(s, lds, turn);
        const float mg = s.x * a.inv_n, mgx = s.y * a.inv_n;
        if (!any) continue;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int c = (k * TPR + lane) * V;
            if (c >= a.n) break;
            piece d;
#pragma unroll
            for (int i = 0; i < V; i++) {
                const float xh = ((float)x[k][i] - st.x) * st.y;
                float v = st.y * ((float)g[k][i] * w[k][i] - mg - xh * mgx);
                if (add) v += (float)res[k][i];
                d[i] = (T)v;
            }
            store<T>((T *)a.dx + r * a.lddx, c, a.n, d);
        }
    }
    if constexpr (SUMS) {
        if constexpr (kRows > 1) {
            // the workgroup's rows of lanes share columns
            constexpr int kLine = TPR * K * V + 1;
            for (int which = 0; which < 2; which++) {
                __syncthreads();
#pragma unroll
                for (int k = 0; k < K; k++)
#pragma unroll
                    for (int i = 0; i < V; i++) part[threadIdx.x / TPR * kLine + (k * TPR + lane) * V + i] = which ? sb[k][i] : sw[k][i];
                __syncthreads();
                for (int c = threadIdx.x; c < a.n; c += block_of(TPR)) {
                    float t = 0;
#pragma unroll
                    for (int q = 0; q < kRows; q++) t += part[q * kLine + c];
                    a.partial[((int64_t)blockIdx.x * 2 + which) * a.n + c] = t;
                }
            }
        } else {
            float *p = a.partial + (int64_t)blockIdx.x * 2 * a.n;
#pragma unroll
            for (int k = 0; k < K; k++)
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const int c = (k * TPR + lane) * V + i;
                    if (c < a.n) p[c] = sw[k][i], p[(int64_t)a.n + c] = sb[k][i];
                }
        }
    }
}

template <typename T, int TPR, int K, bool SUMS> __global__ void __launch_bounds__(block_of(TPR)) backward_kernel(Args a)
{
    __shared__ float2 lds[2][16];
    __shared__ float part[SUMS && TPR < 256 ? 256 / TPR * (TPR * K * Piece<T>::V + 1) : 1];   // sums of the workgroup's rows of lanes
    if (a.n % Piece<T>::V == 0) backward_rows<T, TPR, K, SUMS, true>(a, lds, part);
    else backward_rows<T, TPR, K, SUMS, false>(a, lds, part);
}

// long rows: dx alone
template <typename T> __global__ void __launch_bounds__(1024) backward_long_kernel(Args a)
{
    constexpr int V = Piece<T>::V;
    __shared__ float2 lds[2][16];
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.m; r += gridDim.x, turn ^= 1) {
        const T *px = (const T *)a.x + r * a.ldx, *pg = (const T *)a.dy + r * a.lddy;
        const float2 st = *(const float2 *)(a.stats + 2 * r);
        float2 s = {0, 0};
        for (int c = threadIdx.x * V; c < a.n; c += 1024 * V) {
            const auto x = load<T>(px, c, a.n), g = load<T>(pg, c, a.n);
            float w[V];
            load_weights<T, false>(a.w, a.wide, c, a.n, 1.0f, w);
#pragma unroll
            for (int i = 0; i < V; i++) {
                if (c + i >= a.n) break;
                s.x += (float)g[i] * w[i];
                s.y += (float)g[i] * w[i] * (((float)x[i] - st.x) * st.y);
            }
        }
        s = row_sum<1024>(s, lds, turn);
        const float mg = s.x * a.inv_n, mgx = s.y * a.inv_n;
        for (int c = threadIdx.x * V; c < a.n; c += 1024 * V) {
            const auto x = load<T>(px, c, a.n), g = load<T>(pg, c, a.n);
            float w[V];
            load_weights<T, false>(a.w, a.wide, c, a.n, 1.0f, w);
            typename Piece<T>::type d, res;
            if (a.residual) res = load<T>((const T *)a.residual + r * a.ldr, c, a.n);
#pragma unroll
            for (int i = 0; i < V; i++) {
                float v = st.y * ((float)g[i] * w[i] - mg - ((float)x[i] - st.x) * st.y * mgx);
                if (a.residual) v += (float)res[i];
                d[i] = (T)v;
            }
            store<T>((T *)a.dx + r * a.lddx, c, a.n, d);
        }
    }
}
// long rows: a workgroup's columns' sums over its part of the rows
template <typename T> __global__ void __launch_bounds__(256) sums_long_kernel(Args a)
{
    constexpr int V = Piece<T>::V;
    const int c = (blockIdx.x * 256 + threadIdx.x) * V;
    if (c >= a.n) return;
    float sw[V], sb[V];
#pragma unroll
    for (int i = 0; i < V; i++) sw[i] = sb[i] = 0;
    for (int64_t r = blockIdx.y; r < a.m; r += gridDim.y) {
        const float2 st = *(const float2 *)(a.stats + 2 * r);
        const auto x = load<T>((const T *)a.x + r * a.ldx, c, a.n), g = load<T>((const T *)a.dy + r * a.lddy, c, a.n);
#pragma unroll
        for (int i = 0; i < V; i++) sw[i] += (float)g[i] * (((float)x[i] - st.x) * st.y), sb[i] += (float)g[i];
    }
    float *p = a.partial + (int64_t)blockIdx.y * 2 * a.n;
#pragma unroll
    for (int i = 0; i < V; i++)
        if (c + i < a.n) p[c + i] = sw[i], p[(int64_t)a.n + c + i] = sb[i];
}

// dw and db from the workgroups' sums: 32 columns by 32 lanes' shares of the sums
template <typename T> __global__ void __launch_bounds__(1024) sums_kernel(Args a, int blocks)
{
    __shared__ float part[32][33];
    const int which = blockIdx.y, col = threadIdx.x & 31, share = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
    void *out = which ? a.db : a.dw;
    if (!out) return;
    float s = 0;
    if (c < a.n) {
        const float *p = a.partial + (int64_t)which * a.n + c;
#pragma unroll 4
        for (int b = share; b < blocks; b += 32) s += p[(int64_t)b * 2 * a.n];
    }
    part[share][col] = s;
    __syncthreads();
    if (threadIdx.x >= 32 || c >= a.n) return;
    s = 0;
#pragma unroll
    for (int i = 0; i < 32; i++) s += part[i][col];
    if (a.wide) ((float *)out)[c] = s;
    else ((T *)out)[c] = (T)s;
}

template <typename T> __global__ void __launch_bounds__(256) no_sums_kernel(Args a)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    void *out = blockIdx.y ? a.db : a.dw;
    if (!out || c >= a.n) return;
    if (a.wide) ((float *)out)[c] = 0;
    else ((T *)out)[c] = (T)0.0f;
}

// lanes to a row and pieces a lane for n columns: the fewest lanes, up to a workgroup of 512, that hold
// a row in one piece each; more pieces only beyond that, up to what 256 registers hold beside the sums
struct Shape { int tpr, k; };              // tpr 0: rows are read again
constexpr int kLongest = 16;               // values a lane
template <typename T> static Shape shape_of(int64_t n)
{
    const int64_t pieces = (n + Piece<T>::V - 1) / Piece<T>::V;
    for (int tpr : {8, 16, 32, 64, 256})
        if (pieces <= tpr) return {tpr, 1};
    for (int k = 1; k * Piece<T>::V <= kLongest; k *= 2)
        if (pieces <= 512 * k) return {512, k};
    return {0, 0};
}

// f(TPR, K) as constants
template <typename T, typename F> static void with_shape(Shape s, F f)
{
#define HEDDLE_NORM_SHAPE(TPR, K) \
    if (s.tpr == TPR && s.k == K) return f(std::integral_constant<int, TPR>(), std::integral_constant<int, K>())
    HEDDLE_NORM_SHAPE(8, 1);
    HEDDLE_NORM_SHAPE(16, 1);
    HEDDLE_NORM_SHAPE(32, 1);
    HEDDLE_NORM_SHAPE(64, 1);
    HEDDLE_NORM_SHAPE(256, 1);
    HEDDLE_NORM_SHAPE(512, 1);
    HEDDLE_NORM_SHAPE(512, 2);
    if constexpr (sizeof(T) == 4) HEDDLE_NORM_SHAPE(512, 4);
#undef HEDDLE_NORM_SHAPE
}

static int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, what);
}

template <typename T> static int forward(const Args &a, hipStream_t stream)
{
    if (a.m == 0) return HEDDLE_OK;
    const Shape s = shape_of<T>(a.n);
    constexpr int64_t kBlocks = 1 << 20;                    // a launch of 1024 lanes each stays below 2^32
    if (s.tpr == 0) {
        hipLaunchKernelGGL((forward_long_kernel<T>), dim3((unsigned)std::min(a.m, kBlocks)), dim3(1024), 0, stream, a);
    } else {
        with_shape<T>(s, [&](auto tpr, auto k) {
            constexpr int rows = block_of(tpr) / tpr;
            hipLaunchKernelGGL((forward_kernel<T, tpr, k>), dim3((unsigned)std::min((a.m + rows - 1) / rows, kBlocks)), dim3(block_of(tpr)), 0, stream, a);
        });
    }
    return launched("layer norm");
}

// Workgroups of the backward pass, each with sums of its own: as many as the CUs hold (4096 rows of 4096: 33 us with 512,
// 36 with 256, 45 with 1024; 8192 rows of 1024: 20 us with 1024, 26 with 512), but with four turns each where there are
// few rows, as every one adds a row of sums (1001 rows of 1027: 14 + 6 us with a workgroup each, 10.5 + 4 so).
static int64_t blocks_of(Shape s, int64_t m)
{
    const int64_t rows = s.tpr ? block_of(s.tpr) / s.tpr : 1, want = (m + rows - 1) / rows, most = s.tpr == 0 ? 32 : s.tpr <= 256 ? 1024 : s.k == 1 ? 512 : 256;
    return std::min({want, most, std::max<int64_t>(256, want / 4)});
}

template <typename T> static int backward(Args a, Scratch &ws, bool run, hipStream_t stream)
{
    const Shape s = shape_of<T>(a.n);
    const int64_t blocks = blocks_of(s, a.m);
    const bool sums = a.dw || a.db;
    if (sums) a.partial = (float *)ws.take((size_t)blocks * 2 * a.n * 4);
    if (!run) return HEDDLE_OK;
    if (a.m == 0) {
        if (!sums) return HEDDLE_OK;
        hipLaunchKernelGGL((no_sums_kernel<T>), dim3((unsigned)((a.n + 255) / 256), 2), dim3(256), 0, stream, a);
        return launched("layer norm's gradients");
    }
    if (s.tpr == 0) {
        // the sums first: dx may lie on dy
        if (sums) {
            const int64_t cols = (a.n + 256 * Piece<T>::V - 1) / (256 * Piece<T>::V);
            hipLaunchKernelGGL((sums_long_kernel<T>), dim3((unsigned)cols, (unsigned)blocks), dim3(256), 0, stream, a);
        }
        if (a.dx) hipLaunchKernelGGL((backward_long_kernel<T>), dim3((unsigned)std::min(a.m, int64_t(1) << 20)), dim3(1024), 0, stream, a);
    } else if (sums || a.dx) {
        with_shape<T>(s, [&](auto tpr, auto k) {
            if (sums) hipLaunchKernelGGL((backward_kernel<T, tpr, k, true>), dim3((unsigned)blocks), dim3(block_of(tpr)), 0, stream, a);
            else hipLaunchKernelGGL((backward_kernel<T, tpr, k, false>), dim3((unsigned)blocks), dim3(block_of(tpr)), 0, stream, a);
        });
    }
    if (sums) hipLaunchKernelGGL((sums_kernel<T>), dim3((unsigned)((a.n + 31) / 32), 2), dim3(1024), 0, stream, a, (int)blocks);
    return launched("layer norm's gradients");
}

static int check(const heddle_layer_norm_desc *d, bool backward)
{
    if (!d) return fail(HEDDLE_E_INVAL, "descriptor is NULL");
    if (d->dtype < HEDDLE_T_BF16 || d->dtype > HEDDLE_T_F32) return fail(HEDDLE_E_INVAL, "unknown dtype");
    if (d->wtype != d->dtype && d->wtype != HEDDLE_T_F32) return fail(HEDDLE_E_INVAL, "wtype is neither dtype nor F32");
    if (d->m < 0 || d->n < 1 || d->m > HEDDLE_MAX_ROWS || d->n > HEDDLE_MAX_LD) return fail(HEDDLE_E_INVAL, "m or n out of range");
    if (!backward && !(std::isfinite(d->eps) && d->eps >= 0)) return fail(HEDDLE_E_INVAL, "eps is not finite and >= 0");
    const uintptr_t mask = d->dtype == HEDDLE_T_F32 ? 3 : 1, wmask = d->wtype == HEDDLE_T_F32 ? 3 : 1;
    int rc = HEDDLE_OK;
    auto matrix = [&](const char *name, const void *p, int64_t ld) {
        if (rc || d->m == 0) return;
        rc = mm::check_matrix(name, p, ld, d->n);
        if (rc == HEDDLE_OK && ((uintptr_t)p & mask)) rc = fail(HEDDLE_E_INVAL, std::string(name) + " is not aligned to its values");
    };
    auto vector = [&](const char *name, const void *p) {
        if (rc == HEDDLE_OK && ((uintptr_t)p & wmask)) rc = fail(HEDDLE_E_INVAL, std::string(name) + " is not aligned to its values");
    };
    matrix("x", d->x, d->ldx);
    vector("w", d->w);
    if (rc == HEDDLE_OK && (((uintptr_t)d->stats & 7) || (backward && !d->stats && d->m > 0))) rc = fail(HEDDLE_E_INVAL, "stats is NULL or misaligned");
    if (!backward) {
        vector("bias", d->bias);
        matrix("y", d->y, d->ldy);
    } else {
        matrix("dy", d->dy, d->lddy);
        if (d->dx) matrix("dx", d->dx, d->lddx);
        if (d->dx && d->residual) matrix("residual", d->residual, d->ldr);
        vector("dw", d->dw);
        vector("db", d->db);
    }
    return rc;
}

// Regions count in values of 16 bits.
static int check_overlaps(const heddle_layer_norm_desc *d, bool backward)
{
    const int64_t u = d->dtype == HEDDLE_T_F32 ? 2 : 1, wu = d->wtype == HEDDLE_T_F32 ? 2 : 1;
    auto rows = [&](const char *name, const void *p, int64_t ld) { return Region{name, p, d->m, d->n * u, ld * u}; };
    auto vector = [&](const char *name, const void *p) { return Region{name, p, 1, d->n * wu, d->n * wu}; };
    auto same = [&](const Region &a, const Region &b) { return a.p == b.p && (a.ld == b.ld || d->m == 1); };
    const Region x = rows("x", d->x, d->ldx), w = vector("w", d->w), stats = {"stats", d->stats, 1, d->m * 4, d->m * 4};
    if (!backward) {
        const Region y = rows("y", d->y, d->ldy), bias = vector("bias", d->bias);
        const int rc = mm::check_apart(y, {same(x, y) ? nullptr : &x, &w, &bias, d->m > 0 ? &stats : nullptr});
        return rc || d->m == 0 ? rc : mm::check_apart(stats, {&x, &w, &bias});
    }
    const Region dy = rows("dy", d->dy, d->lddy), dx = rows("dx", d->dx, d->lddx), r = rows("residual", d->dx ? d->residual : nullptr, d->ldr);
    const Region dw = vector("dw", d->dw), db = vector("db", d->db);
    // dx may be dy or the residual itself: a lane has read what it overwrites
    int rc = mm::check_apart(dx, {&x, &w, same(dy, dx) ? nullptr : &dy, same(r, dx) ? nullptr : &r, &stats, &dw, &db});
    // dw and db are written when all else has been done
    return rc ? rc : mm::check_apart(dw, {&db});
}

static int run_norm(const heddle_layer_norm_desc *d, bool back, void *ws, int64_t bytes, bool run, hipStream_t stream, int64_t *need)
{
    int rc = check(d, back);
    if (rc) return rc;
    Args a = {};
    a.x = d->x, a.ldx = d->ldx, a.w = d->w, a.stats = d->stats, a.m = d->m, a.n = (int32_t)d->n;
    a.wide = d->wtype == HEDDLE_T_F32, a.eps = d->eps, a.inv_n = (float)(1.0 / (double)d->n);
    if (back) {
        a.dy = d->dy, a.lddy = d->lddy, a.residual = d->residual, a.ldr = d->ldr, a.dx = d->dx, a.lddx = d->lddx;
        a.dw = d->dw, a.db = d->db;
    } else {
        a.bias = d->bias, a.y = d->y, a.ldy = d->ldy;
    }
    for (int pass = 0; pass < 2; pass++) {
        Scratch s = {pass ? (char *)ws : nullptr, 0};
        const bool go = pass == 1;
        auto call = [&](auto t) {
            typedef decltype(t) T;
            return back ? backward<T>(a, s, go, stream) : go ? forward<T>(a, stream) : HEDDLE_OK;
        };
        rc = d->dtype == HEDDLE_T_BF16 ? call((__bf16)0.0f) : d->dtype == HEDDLE_T_F16 ? call((_Float16)0.0f) : call(0.0f);
        if (rc) return rc;
        if (pass == 0) {
            if (need) *need = (int64_t)s.used;
            if (!run) return HEDDLE_OK;
            rc = mm::check_scratch(s.used, ws, bytes);
            if (rc == HEDDLE_OK) rc = check_overlaps(d, back);
            if (rc) return rc;
        }
    }
    return HEDDLE_OK;
}

}  // namespace norm
}  // namespace heddle

using namespace heddle;

extern "C" int heddle_layer_norm(const heddle_layer_norm_desc *d, hipStream_t stream)
{
    return norm::run_norm(d, false, nullptr, 0, true, stream, nullptr);
}

extern "C" int heddle_layer_norm_backward(const heddle_layer_norm_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return norm::run_norm(d, true, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_layer_norm_workspace(const heddle_layer_norm_desc *d, int64_t *h_bytes)
{
    if (!h_bytes) return fail(HEDDLE_E_INVAL, "h_bytes is NULL");
    return norm::run_norm(d, true, nullptr, 0, false, nullptr, h_bytes);
}
