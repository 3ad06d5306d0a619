// A router's balance: how often each expert was picked, and a loss that grows as picks and
// probabilities gather on few experts, with its gradient.
//
// p = softmax(logits) of a row, c_e = picks of expert e, C = sum c, N = rows with a pick,
// P_e = sum of p_e over those rows / N, loss = scale E sum_e (c_e / C) P_e;
// dlogits = dloss scale E / (C N) p (c_e - sum_j p_j c_j) + r.
// The logits are read once, and once more for the gradient (p is formed again
// rather than kept). G lanes to a row, K neighbouring values a lane, so that a wavefront reads 64 / G
// rows side by side, kAhead of them before the first is used. A workgroup counts picks in LDS with integer atomics, whose order changes nothing;
// probabilities are summed in fp32 registers, then over workgroups, in one order. 131072 rows of 64 in bf16, top 2: 16 + 6.5 us,
// the gradient with a residual 21 us: 1.2 and 2.4 TB/s, wavefronts waiting 62 and 66% of the time (forward, a CU has
// eight wavefronts, and the next rows are loaded when the last are used up).
#include <algorithm>
#include <cmath>

#include "linear.h"

namespace heddle {
namespace balance {

using mm::Region;
using mm::Scratch;

struct Args {
    const void *logits, *residual, *picked;
    void *dlogits;
    const float *dloss;
    float *loss, *mean, *sums;                // sums: [blocks][experts] of probabilities
    int32_t *counts, *offsets, *rows, *parts; // parts: [blocks][experts + 1] picks, and rows with one
    int64_t ldl, ldr, ldd, ldp;
    int64_t t;
    int32_t experts, picks, wide_picks;       // wide_picks: 8 bytes each
    float scale;
};

__device__ inline int64_t pick_at(const Args &a, int64_t r, int i)
{
    return a.wide_picks ? ((const int64_t *)a.picked)[r * a.ldp + i] : (int64_t)((const int32_t *)a.picked)[r * a.ldp + i];
}

// K neighbouring values of a row; past its end other
template <typename T, int K> struct Some {
    typedef T loose __attribute__((ext_vector_type(K), aligned(sizeof(T))));   // at any address its values may have
};
template <typename T, int K> __device__ inline void load_row(const T *row, int e, int experts, float other, float z[K])
{
    if (e + K <= experts) {
        const typename Some<T, K>::loose v = *(const typename Some<T, K>::loose *)(row + e);
#pragma unroll
        for (int k = 0; k < K; k++) z[k] = (float)v[k];
        return;
    }
    if (e >= experts) {
#pragma unroll
        for (int k = 0; k < K; k++) z[k] = other;
        return;
    }
#pragma unroll
    for (int k = 0; k < K; k++) z[k] = (float)row[min(e + k, experts - 1)];
#pragma unroll
    for (int k = 1; k < K; k++) z[k] = e + k < experts ? z[k] : other;
}

// op over G neighbouring lanes, in all of them: within 16 by moves of the vector units (the cross-lane
// exchange through LDS is as slow as a read of it, and a row takes three such sums)
template <int CTRL> __device__ inline float moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int G, typename Op> __device__ inline float over(float v, Op op)
{
    v = op(v, moved<0xb1>(v));                              // the neighbour of a pair
    v = op(v, moved<0x4e>(v));                              // the other pair of four
    v = op(v, moved<0x141>(v));                             // eight in reverse
    if constexpr (G >= 16) v = op(v, moved<0x140>(v));      // sixteen in reverse
    if constexpr (G >= 32) v = op(v, __shfl_xor(v, 16));
    if constexpr (G >= 64) v = op(v, __shfl_xor(v, 32));
    return v;
}
template <int G> __device__ inline float sum_over(float v) { return over<G>(v, [](float a, float b) { return a + b; }); }

// softmax over G lanes' K values; a row of -infinity alone has no probabilities: zeros
template <int G, int K> __device__ inline void softmax(float z[K])
{
    float top = z[0], sum = 0;
#pragma unroll
    for (int k = 1; k < K; k++) top = fmaxf(top, z[k]);
    top = over<G>(top, [](float a, float b) { return fmaxf(a, b); });
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int k = 0; k < K; k++) z[k] = __expf(z[k] - base), sum += z[k];
    sum = sum_over<G>(sum);
    const float inv = sum == 0 ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int k = 0; k < K; k++) z[k] *= inv;
}

// whether a row has a pick at all
__device__ inline bool has_pick(const Args &a, int64_t r)
{
    bool some = false;
    for (int i = 0; i < a.picks; i++) {
        const int64_t e = pick_at(a, r, i);
        some |= e >= 0 && e < a.experts;
    }
    return some;
}

template <typename T, int G, int K> __global__ void __launch_bounds__(256) forward_kernel(Args a)
{
    constexpr int kRows = 256 / G, kAhead = K <= 4 ? 4 : K <= 8 ? 2 : 1;
    __shared__ int count[G * K + 1];
    __shared__ float part[kRows > 1 ? kRows : 1][G * K];
    for (int i = threadIdx.x; i <= G * K; i += 256) count[i] = 0;
    __syncthreads();
    const int lane = threadIdx.x % G;
    float sum[K];
#pragma unroll
    for (int k = 0; k < K; k++) sum[k] = 0;
    int with = 0;
    const int64_t step = (int64_t)gridDim.x * kRows;
    // whole rows of lanes: every lane of a row takes the same turns
    for (int64_t r0 = (int64_t)blockIdx.x * kRows + threadIdx.x / G; r0 < a.t; r0 += step * kAhead) {
        float z[kAhead][K];
        int64_t pick[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; n++) {
            const int64_t r = min(r0 + n * step, a.t - 1);
            load_row<T, K>((const T *)a.logits + r * a.ldl, lane * K, a.experts, -INFINITY, z[n]);
            pick[n] = pick_at(a, r, min(lane, a.picks - 1));
        }
#pragma unroll
        for (int n = 0; n < kAhead; n++) {
            const int64_t r = r0 + n * step;
            if (r >= a.t) break;
            int has = 0;
            for (int i = lane; i < a.picks; i += G) {
                const int64_t e = i < G ? pick[n] : pick_at(a, r, i);
                if (e >= 0 && e < a.experts) {
                    atomicAdd(&count[e], 1);
                    has = 1;
                }
            }
            // a row's lanes: any of them with a pick
            has = (__ballot(has) >> ((threadIdx.x & 63) / G * G) & (G == 64 ? ~0ull : (1ull << (G & 63)) - 1)) != 0;
            softmax<G, K>(z[n]);
            if (has) {
                with += lane == 0;
#pragma unroll
                for (int k = 0; k < K; k++) sum[k] += z[n][k];
            }
        }
    }
    if (with) atomicAdd(&count[G * K], with);
#pragma unroll
    for (int k = 0; k < K; k++) part[threadIdx.x / G][lane * K + k] = sum[k];
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += 256) {
        float s = 0;
#pragma unroll
        for (int q = 0; q < kRows; q++) s += part[q][e];
        a.sums[(int64_t)blockIdx.x * a.experts + e] = s;
        a.parts[(int64_t)blockIdx.x * (a.experts + 1) + e] = count[e];
    }
    if (threadIdx.x == 0) a.parts[(int64_t)blockIdx.x * (a.experts + 1) + a.experts] = count[G * K];
}

// the workgroups' sums become one row: 32 columns by 32 shares
__global__ void __launch_bounds__(1024) fold_kernel(Args a, int blocks, float *sums, int32_t *parts)
{
    __shared__ float fs[32][33];
    __shared__ int fc[32][33];
    const int col = threadIdx.x & 31, share = threadIdx.x >> 5, e = blockIdx.x * 32 + col;
    float s = 0;
    int c = 0;
    if (e <= a.experts)
#pragma unroll 4
        for (int b = share; b < blocks; b += 32) {
            if (e < a.experts) s += a.sums[(int64_t)b * a.experts + e];
            c += a.parts[(int64_t)b * (a.experts + 1) + e];
        }
    fs[share][col] = s, fc[share][col] = c;
    __syncthreads();
    if (share || e > a.experts) return;
    s = 0, c = 0;
#pragma unroll
    for (int i = 0; i < 32; i++) s += fs[i][col], c += fc[i][col];
    if (e < a.experts) sums[e] = s;
    parts[e] = c;
}

// One workgroup: the counts, their running sums, the mean probabilities and the loss. W columns by 1024 / W shares of
// the workgroups' sums at a time.
template <int W> __global__ void __launch_bounds__(1024) finish_kernel(Args a, int blocks)
{
    constexpr int kShares = 1024 / W;
    __shared__ float fs[kShares > 1 ? kShares : 1][W];
    __shared__ int fc[kShares > 1 ? kShares : 1][W], fr[16], scan[16], carry_of;
    __shared__ double weight[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = threadIdx.x % W, share = threadIdx.x / W;
    int rows = 0;
    for (int b = threadIdx.x; b < blocks; b += 1024) rows += a.parts[(int64_t)b * (a.experts + 1) + a.experts];
#pragma unroll
    for (int d = 32; d; d /= 2) rows += __shfl_xor(rows, d);
    if (lane == 0) fr[wave] = rows;
    int carry = 0;
    double dot = 0;
    for (int e0 = 0; e0 < a.experts; e0 += W) {
        const int e = e0 + col;
        int c = 0;
        float s = 0;
        if (e < a.experts)
#pragma unroll 8
            for (int b = share; b < blocks; b += kShares) {
                c += a.parts[(int64_t)b * (a.experts + 1) + e];
                s += a.sums[(int64_t)b * a.experts + e];
            }
        fs[share][col] = s, fc[share][col] = c;
        __syncthreads();
        s = 0, c = 0, rows = 0;
#pragma unroll
        for (int i = 0; i < 16; i++) rows += fr[i];
        if (share == 0) {
#pragma unroll
            for (int i = 0; i < kShares; i++) s += fs[i][col], c += fc[i][col];
        }
        int run = c;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(run, d);
            if (lane >= d) run += o;
        }
        if (lane == 63) scan[wave] = run;
        __syncthreads();
        int before = carry;
        for (int i = 0; i < wave; i++) before += scan[i];
        if (threadIdx.x == W - 1) carry_of = before + run;
        if (share == 0 && e < a.experts) {
            a.counts[e] = c;
            const float mean = rows ? s / (float)rows : 0.0f;
            if (a.mean) a.mean[e] = mean;
            if (a.offsets) a.offsets[e + 1] = before + run;
            dot += (double)c * (double)mean;
        }
        __syncthreads();
        carry = carry_of;
    }
#pragma unroll
    for (int d = 32; d; d /= 2) dot += __shfl_xor(dot, d);
    if (lane == 0) weight[wave] = dot;
    __syncthreads();
    if (threadIdx.x) return;
    dot = 0;
    for (int i = 0; i < 16; i++) dot += weight[i];
    if (a.offsets) a.offsets[0] = 0;
    if (a.rows) *a.rows = rows;
    if (a.loss) *a.loss = carry ? (float)((double)a.scale * a.experts * dot / (double)carry) : 0.0f;
}

// Every workgroup forms C from the counts by itself.
template <typename T, int G, int K> __global__ void __launch_bounds__(256) backward_kernel(Args a)
{
    constexpr int kRows = 256 / G, kAhead = K <= 4 ? 4 : K <= 8 ? 2 : 1;
    __shared__ double all[4];
    const int lane = threadIdx.x % G;
    double total = 0;
    for (int e = threadIdx.x; e < a.experts; e += 256) total += (double)a.counts[e];
#pragma unroll
    for (int d = 32; d; d /= 2) total += __shfl_xor(total, d);
    if ((threadIdx.x & 63) == 0) all[threadIdx.x >> 6] = total;
    __syncthreads();
    total = (all[0] + all[1]) + (all[2] + all[3]);
    const double rows = (double)*a.rows;
    const float factor = total > 0 && rows > 0 ? (float)((double)a.scale * (a.dloss ? (double)*a.dloss : 1.0) * a.experts / (total * rows)) : 0.0f;
    float c[K];
#pragma unroll
    for (int k = 0; k < K; k++) c[k] = lane * K + k < a.experts ? (float)a.counts[lane * K + k] : 0.0f;
    const int64_t step = (int64_t)gridDim.x * kRows;
    for (int64_t r0 = (int64_t)blockIdx.x * kRows + threadIdx.x / G; r0 < a.t; r0 += step * kAhead) {
        float z[kAhead][K], add[kAhead][K];
        bool some[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; n++) {
            const int64_t r = min(r0 + n * step, a.t - 1);
            load_row<T, K>((const T *)a.logits + r * a.ldl, lane * K, a.experts, -INFINITY, z[n]);
#pragma unroll
            for (int k = 0; k < K; k++) add[n][k] = 0;
            if (a.residual) load_row<T, K>((const T *)a.residual + r * a.ldr, lane * K, a.experts, 0.0f, add[n]);
            some[n] = has_pick(a, r);
        }
#pragma unroll
        for (int n = 0; n < kAhead; n++) {
            const int64_t r = r0 + n * step;
            if (r >= a.t) break;
            softmax<G, K>(z[n]);
            float dot = 0;
#pragma unroll
            for (int k = 0; k < K; k++) dot += z[n][k] * c[k];
            dot = sum_over<G>(dot);
            T *out = (T *)a.dlogits + r * a.ldd + lane * K;
            typename Some<T, K>::loose v;
#pragma unroll
            for (int k = 0; k < K; k++) v[k] = (T)((some[n] ? factor * z[n][k] * (c[k] - dot) : 0.0f) + add[n][k]);
            if (lane * K + K <= a.experts) {
                *(typename Some<T, K>::loose *)out = v;
            } else {
#pragma unroll
                for (int k = 0; k < K; k++)
                    if (lane * K + k < a.experts) out[k] = v[k];
            }
        }
    }
}

// lanes of a row and values of a lane
template <typename F> static void with_shape(int experts, F f)
{
#define HEDDLE_BALANCE_SHAPE(G, K) \
    if (experts <= G * K) return f(std::integral_constant<int, G>(), std::integral_constant<int, K>())
    HEDDLE_BALANCE_SHAPE(8, 1);
    HEDDLE_BALANCE_SHAPE(16, 1);
    HEDDLE_BALANCE_SHAPE(16, 2);
    HEDDLE_BALANCE_SHAPE(16, 4);
    HEDDLE_BALANCE_SHAPE(32, 4);
    HEDDLE_BALANCE_SHAPE(64, 4);
    HEDDLE_BALANCE_SHAPE(64, 8);
    HEDDLE_BALANCE_SHAPE(64, 16);
    HEDDLE_BALANCE_SHAPE(64, 32);
#undef HEDDLE_BALANCE_SHAPE
}

static int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, what);
}

// Experts up to which the last kernel adds up the workgroups' sums itself, 16 shares a column: past that
// one workgroup would read for longer than another launch takes.
constexpr int kNarrow = 64;

static int64_t blocks_of(int experts, int64_t t)
{
    int64_t rows = 1;
    with_shape(experts, [&](auto g, auto) { rows = 256 / g; });
    return std::max<int64_t>(1, std::min<int64_t>((t + rows - 1) / rows, 512));
}

template <typename T> static int forward(Args a, Scratch &s, bool run, hipStream_t stream)
{
    const int64_t blocks = blocks_of(a.experts, a.t);
    a.sums = (float *)s.take((size_t)blocks * a.experts * 4);
    a.parts = (int32_t *)s.take((size_t)blocks * (a.experts + 1) * 4);
    const bool fold = a.experts > kNarrow && blocks > 1;
    float *sums = nullptr;
    int32_t *parts = nullptr;
    if (fold) {
        sums = (float *)s.take((size_t)a.experts * 4);
        parts = (int32_t *)s.take((size_t)(a.experts + 1) * 4);
    }
    if (!run) return HEDDLE_OK;
    with_shape(a.experts, [&](auto g, auto k) {
        hipLaunchKernelGGL((forward_kernel<T, g, k>), dim3((unsigned)blocks), dim3(256), 0, stream, a);
    });
    if (fold) {
        hipLaunchKernelGGL(fold_kernel, dim3((unsigned)(a.experts / 32 + 1)), dim3(1024), 0, stream, a, (int)blocks, sums, parts);
        a.sums = sums, a.parts = parts;
    }
    if (a.experts <= kNarrow) hipLaunchKernelGGL(finish_kernel<kNarrow>, dim3(1), dim3(1024), 0, stream, a, (int)blocks);
    else hipLaunchKernelGGL(finish_kernel<1024>, dim3(1), dim3(1024), 0, stream, a, 1);
    return launched("expert balance");
}

template <typename T> static int backward(const Args &a, hipStream_t stream)
{
    if (a.t == 0) return HEDDLE_OK;
    with_shape(a.experts, [&](auto g, auto k) {
        constexpr int rows = 256 / g;
        hipLaunchKernelGGL((backward_kernel<T, g, k>), dim3((unsigned)std::min<int64_t>((a.t + rows - 1) / rows, 2048)), dim3(256), 0, stream, a);
    });
    return launched("expert balance's gradient");
}

static int check(const heddle_expert_balance_desc *d, bool backward)
{
    if (!d) return fail(HEDDLE_E_INVAL, "descriptor is NULL");
    if (d->dtype < HEDDLE_T_BF16 || d->dtype > HEDDLE_T_F32) return fail(HEDDLE_E_INVAL, "unknown dtype");
    if (d->pick_bytes != 4 && d->pick_bytes != 8) return fail(HEDDLE_E_INVAL, "pick_bytes is neither 4 nor 8");
    if (d->experts < 1 || d->experts > HEDDLE_MAX_EXPERTS) return fail(HEDDLE_E_INVAL, "experts out of range");
    if (d->picks < 1 || d->picks > d->experts) return fail(HEDDLE_E_INVAL, "picks out of range");
    if (d->t < 0 || d->t > HEDDLE_MAX_ROWS || d->t * d->picks > INT32_MAX) return fail(HEDDLE_E_INVAL, "t out of range: picks are counted in 32 bits");
    if (!std::isfinite(d->scale)) return fail(HEDDLE_E_INVAL, "scale is not finite");
    const uintptr_t mask = d->dtype == HEDDLE_T_F32 ? 3 : 1;
    int rc = HEDDLE_OK;
    auto matrix = [&](const char *name, const void *p, int64_t ld, int64_t cols, uintptr_t m) {
        if (rc || d->t == 0) return;
        rc = mm::check_matrix(name, p, ld, cols);
        if (rc == HEDDLE_OK && ((uintptr_t)p & m)) rc = fail(HEDDLE_E_INVAL, std::string(name) + " is not aligned to its values");
    };
    auto word = [&](const char *name, const void *p, bool must) {
        if (rc == HEDDLE_OK && (((uintptr_t)p & 3) || (must && !p))) rc = fail(HEDDLE_E_INVAL, std::string(name) + " is NULL or misaligned");
    };
    matrix("logits", d->logits, d->ldl, d->experts, mask);
    matrix("d_picked", d->d_picked, d->ldp, d->picks, (uintptr_t)d->pick_bytes - 1);
    word("d_counts", d->d_counts, true);
    word("d_rows", d->d_rows, backward);
    if (!backward) {
        word("d_loss", d->d_loss, false);
        word("d_mean", d->d_mean, false);
        word("d_offsets", d->d_offsets, false);
    } else {
        word("d_dloss", d->d_dloss, false);
        if (d->residual) matrix("residual", d->residual, d->ldr, d->experts, mask);
        matrix("dlogits", d->dlogits, d->ldd, d->experts, mask);
    }
    return rc;
}

// Regions count in values of 16 bits.
static int check_overlaps(const heddle_expert_balance_desc *d, bool backward)
{
    const int64_t u = d->dtype == HEDDLE_T_F32 ? 2 : 1, pu = d->pick_bytes / 2, e = d->experts;
    auto words = [](const char *name, const void *p, int64_t n) { return Region{name, p, 1, 2 * n, 2 * n}; };
    auto rows = [&](const char *name, const void *p, int64_t ld) { return Region{name, d->t ? p : nullptr, d->t, e * u, ld * u}; };
    const Region logits = rows("logits", d->logits, d->ldl), picked = {"d_picked", d->t ? d->d_picked : nullptr, d->t, d->picks * pu, d->ldp * pu};
    const Region counts = words("d_counts", d->d_counts, e), n = words("d_rows", d->d_rows, 1);
    if (!backward) {
        // written when logits and picks have been read
        const Region offsets = words("d_offsets", d->d_offsets, e + 1), mean = words("d_mean", d->d_mean, e), loss = words("d_loss", d->d_loss, 1);
        int rc = mm::check_apart(counts, {&offsets, &mean, &loss, &n});
        if (rc == HEDDLE_OK) rc = mm::check_apart(offsets, {&mean, &loss, &n});
        if (rc == HEDDLE_OK) rc = mm::check_apart(mean, {&loss, &n});
        return rc ? rc : mm::check_apart(loss, {&n});
    }
    const Region out = rows("dlogits", d->dlogits, d->ldd), r = rows("residual", d->residual, d->ldr), dloss = words("d_dloss", d->d_dloss, 1);
    // dlogits may be the logits or the residual itself: a lane has read what it overwrites
    auto same = [&](const Region &a) { return a.p == out.p && (a.ld == out.ld || d->t == 1); };
    return mm::check_apart(out, {&picked, &counts, &n, &dloss, same(logits) ? nullptr : &logits, same(r) ? nullptr : &r});
}

static int run_balance(const heddle_expert_balance_desc *d, bool back, void *ws, int64_t bytes, bool run, hipStream_t stream, int64_t *need)
{
    int rc = check(d, back);
    if (rc) return rc;
    Args a = {};
    a.logits = d->logits, a.ldl = d->ldl, a.picked = d->d_picked, a.ldp = d->ldp, a.wide_picks = d->pick_bytes == 8;
    a.t = d->t, a.experts = d->experts, a.picks = d->picks, a.scale = d->scale, a.counts = d->d_counts, a.rows = d->d_rows;
    if (back) {
        a.dloss = d->d_dloss, a.residual = d->residual, a.ldr = d->ldr, a.dlogits = d->dlogits, a.ldd = d->ldd;
    } else {
        a.loss = d->d_loss, a.mean = d->d_mean, a.offsets = d->d_offsets;
    }
    for (int pass = 0; pass < 2; pass++) {
        Scratch s = {pass ? (char *)ws : nullptr, 0};
        auto call = [&](auto t) {
            typedef decltype(t) T;
            return back ? pass == 1 ? backward<T>(a, stream) : HEDDLE_OK : forward<T>(a, s, pass == 1, stream);
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

}  // namespace balance
}  // namespace heddle

using namespace heddle;

extern "C" int heddle_expert_balance(const heddle_expert_balance_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return balance::run_balance(d, false, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_expert_balance_backward(const heddle_expert_balance_desc *d, hipStream_t stream)
{
    return balance::run_balance(d, true, nullptr, 0, true, stream, nullptr);
}

extern "C" int heddle_expert_balance_workspace(const heddle_expert_balance_desc *d, int64_t *h_bytes)
{
    if (!h_bytes) return fail(HEDDLE_E_INVAL, "h_bytes is NULL");
    return balance::run_balance(d, false, nullptr, 0, false, nullptr, h_bytes);
}
