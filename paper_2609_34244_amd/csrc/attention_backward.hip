// The gradients of attention on gfx950's matrix cores, from the kept lse.
//
// P = exp(s - lse), delta = sum dy y, dP = dY V^T, dS = P (dP - delta), with a cap dS (1 - tanh^2);
// dq = scale dS K, dk = scale dS^T Q, dv = P^T dY. P is formed again in both kernels, so that each
// sum stays in registers and is added up in one order, without atomics: 7 products instead of 5.
// rows_kernel (dq): 128 query rows a workgroup, tiles of 64 keys, like the forward pass; it also
// leaves lse log2(e) and delta of its rows for the other one. keys_kernel (dk, dv): 128 keys a
// workgroup, 32 a wavefront, over tiles of query rows of each head of the group in turn, whose sum
// the shared heads' gradient is. P and dS are rounded to the operands' type, as the products' operands.
#include <algorithm>
#include <cmath>

#include "attention.h"

namespace heddle {
namespace attn {

// P and dS of 32 x 32 scores. at: distance from register 0's key or row (the sign does not matter);
// seen(r): whether register r's pair is visible; lse2 and delta by register.
template <bool MOD, typename Seen, typename Lse, typename Delta>
__device__ inline void weigh(const Args &a, f32x16 &s, f32x16 &dp, float slope2, int at, bool masked, Seen seen, Lse lse2, Delta delta)
{
    f32x16 t;
    modify<MOD>(a, s, slope2, at, &t);
#pragma unroll
    for (int r = 0; r < 16; r++) s[r] = __builtin_amdgcn_exp2f(s[r] - lse2(r));
    if (masked) {
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] = seen(r) ? s[r] : 0.0f;
    }
#pragma unroll
    for (int r = 0; r < 16; r++) dp[r] = s[r] * (dp[r] - delta(r));
    if constexpr (MOD) {
        if (a.cap > 0) {
#pragma unroll
            for (int r = 0; r < 16; r++) dp[r] *= 1.0f - t[r] * t[r];
        }
    }
}

template <typename T, int DP, bool MOD> __global__ void __launch_bounds__(256, 2) rows_kernel(Args a, int64_t tiles)
{
    typedef Tile<DP, 64, 4> Tk;
    typedef typename mm::pack8<T>::type frag;
    __shared__ __align__(1024) char smem[2][2 * Tk::kBytes];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int hk = blockIdx.x % a.kv_heads;
    const int64_t slot = gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads;
    int s;
    int64_t tile;
    if (a.packed) {
        if (!find_slot(a.d_q, a.q_rows, 1, a.sequences, a.group, 128, tiles, slot, s, tile)) return;
    } else {
        s = (int)(slot % a.sequences), tile = slot / a.sequences;
    }
    const Sequence q = sequence_of(a, s);
    if (tile * 128 >= (int64_t)q.lq * a.group) return;
    const int rows = q.lq * a.group, r = (int)tile * 128 + wave * 32 + col;
    const bool any = r < rows;
    const int i = r / a.group, head = hk * a.group + (any ? r - i * a.group : 0), shift = q.lk - q.lq;
    auto limit_at = [&](int x) { return x >= rows ? 0 : max(min(q.lk, a.causal ? max(x / a.group + shift + 1, q.prefix) : q.lk), 0); };
    const int limit = limit_at(r), r0 = (int)tile * 128 + wave * 32;
    const int end = __builtin_amdgcn_readfirstlane(limit_at(min((int)tile * 128 + 127, rows - 1)));
    const int mine = r0 < rows ? __builtin_amdgcn_readfirstlane(limit_at(min(r0 + 31, rows - 1))) : 0;
    const int whole = r0 + 31 < rows ? __builtin_amdgcn_readfirstlane(limit_at(r0)) : 0;
    const int count = (a.grads & 1) ? (end + 63) / 64 : 0;

    const T *pk = (const T *)a.k.p + s * a.k.seq + q.k0 * a.k.row + hk * a.k.head;
    const T *pv = (const T *)a.v.p + s * a.v.seq + q.k0 * a.v.row + hk * a.v.head;
    int ok[Tk::kLoads], ov[Tk::kLoads];
#pragma unroll
    for (int n = 0; n < Tk::kLoads; n++) ok[n] = Tk::offset(n, wave, a.k.row, a.dim, 64), ov[n] = Tk::offset(n, wave, a.v.row, a.dim, 64);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&smem[0][0];
    auto load = [&](int t) {
        const int valid = q.lk - t * 64;
        const i32x4 bk = buffer_at(pk + (int64_t)t * 64 * a.k.row), bv = buffer_at(pv + (int64_t)t * 64 * a.v.row);
        const uint32_t to = lds + (t & 1) * 2 * Tk::kBytes + wave * 1024;
#pragma unroll
        for (int n = 0; n < Tk::kLoads; n++) {
            mm::load_to_lds(bk, valid >= 64 ? ok[n] : Tk::offset(n, wave, a.k.row, a.dim, valid), to + n * 4096);
            mm::load_to_lds(bv, valid >= 64 ? ov[n] : Tk::offset(n, wave, a.v.row, a.dim, valid), to + Tk::kBytes + n * 4096);
        }
    };
    if (count) load(0);

    const int64_t at = (a.packed ? q.q0 : (int64_t)s * a.q_len) + i;
    frag qf[DP / 16], gf[DP / 16];
    const T *pq = (const T *)a.q.p + s * a.q.seq + (q.q0 + i) * a.q.row + head * a.q.head;
    const T *pg = (const T *)a.dy.p + s * a.dy.seq + (q.q0 + i) * a.dy.row + head * a.dy.head;
    const T *py = (const T *)a.y.p + s * a.y.seq + (q.q0 + i) * a.y.row + head * a.y.head;
    float delta = 0;
#pragma unroll
    for (int k = 0; k < DP / 16; k++) {
        qf[k] = global_fragment<T>(pq, k * 16 + 8 * h, a.dim, any);
        gf[k] = global_fragment<T>(pg, k * 16 + 8 * h, a.dim, any);
        const frag yf = global_fragment<T>(py, k * 16 + 8 * h, a.dim, any);
#pragma unroll
        for (int n = 0; n < 8; n++) delta = __builtin_fmaf((float)gf[k][n], (float)yf[n], delta);
    }
    delta += other_half(delta);
    float lse2 = INFINITY;                                  // of a row that sees nothing: P = 0
    if (any) {
        const float v = a.lse[at * a.heads + head];
        lse2 = v == -INFINITY ? INFINITY : v * kLog2e;
        if (h == 0) a.rows[(int64_t)head * a.q_rows + at] = {lse2, delta};
    }
    if (!(a.grads & 1)) return;
    const float slope2 = MOD && a.d_slopes ? a.d_slopes[head] * kLog2e : 0.0f;

    f32x16 dq[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) dq[d] = f32x16{};
    for (int t = 0; t < count; t++) {
        mm::arrive();
        if (t + 1 < count) load(t + 1);
        const char *tk = smem[t & 1], *tv = tk + Tk::kBytes;
#pragma unroll
        for (int c = 0; c < 2; c++) {
            const int j0 = t * 64 + c * 32;
            if (j0 >= mine) break;
            f32x16 p = {}, ds = {};
#pragma unroll
            for (int k = 0; k < DP / 16; k++) p = mfma(row_fragment<DP, T>(tk, c * 32 + col, k, h), qf[k], p);
#pragma unroll
            for (int k = 0; k < DP / 16; k++) ds = mfma(row_fragment<DP, T>(tv, c * 32 + col, k, h), gf[k], ds);
            const int first = j0 + 4 * h;
            weigh<MOD>(a, p, ds, slope2, i + shift - first, j0 + 32 > whole, [&](int n) { return first + mfma_row(n, 0) < limit; },
                       [&](int) { return lse2; }, [&](int) { return delta; });
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const frag b = pack<T>(ds, 8 * k);
#pragma unroll
                for (int d = 0; d < DP / 32; d++) dq[d] = mfma(column_fragment<DP, T>(tk, c * 32 + 16 * k, d), b, dq[d]);
            }
        }
    }
    if (!any) return;
    T *out = (T *)a.dq.p + s * a.dq.seq + (q.q0 + i) * a.dq.row + head * a.dq.head;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int n = 0; n < 16; n += 4)
            store4<T>(out, d * 32 + mfma_row(n, h), a.dim, a.out_vec, dq[d][n] * a.scale, dq[d][n + 1] * a.scale, dq[d][n + 2] * a.scale, dq[d][n + 3] * a.scale);
}

template <typename T, int DP, bool MOD> __global__ void __launch_bounds__(256) keys_kernel(Args a, int64_t tiles)
{
    constexpr int kRows = 64;
    typedef Tile<DP, kRows, 4> Tk;
    typedef typename mm::pack8<T>::type frag;
    __shared__ __align__(1024) char smem[2][2 * Tk::kBytes];
    __shared__ __align__(16) float stats[2][2][kRows];      // lse log2(e), delta
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int hk = blockIdx.x % a.kv_heads;
    const int64_t slot = blockIdx.x / a.kv_heads;           // the first tiles, which the most rows see, first
    int s;
    int64_t tile;
    if (a.packed) {
        if (!find_slot(a.d_k, a.k_rows, 1, a.sequences, 1, 128, tiles, slot, s, tile)) return;
    } else {
        s = (int)(slot % a.sequences), tile = slot / a.sequences;
    }
    const Sequence q = sequence_of(a, s);
    if (tile * 128 >= q.lk) return;
    const int j0 = (int)tile * 128, j = j0 + wave * 32 + col, shift = q.lk - q.lq;
    const bool any = j < q.lk;
    // the first row of a head that sees a key
    auto first_of = [&](int key) { return a.causal && key >= q.prefix ? max(key - shift, 0) : 0; };
    const int from = first_of(j), start = first_of(j0) / kRows * kRows;
    const int w0 = j0 + wave * 32;                          // the wavefront's keys: all seen from row `whole` on
    const int whole = __builtin_amdgcn_readfirstlane(first_of(w0 + 31)), mine = w0 < q.lk ? __builtin_amdgcn_readfirstlane(first_of(w0)) : INT32_MAX;
    const int per = q.lq > start ? (q.lq - start + kRows - 1) / kRows : 0, count = per * a.group;

    const T *pk = (const T *)a.k.p + s * a.k.seq + (q.k0 + j) * a.k.row + hk * a.k.head;
    const T *pv = (const T *)a.v.p + s * a.v.seq + (q.k0 + j) * a.v.row + hk * a.v.head;
    frag kf[DP / 16], vf[DP / 16];
#pragma unroll
    for (int k = 0; k < DP / 16; k++) {
        kf[k] = global_fragment<T>(pk, k * 16 + 8 * h, a.dim, any);
        vf[k] = global_fragment<T>(pv, k * 16 + 8 * h, a.dim, any);
    }
    int oq[Tk::kLoads], og[Tk::kLoads];
#pragma unroll
    for (int n = 0; n < Tk::kLoads; n++) oq[n] = Tk::offset(n, wave, a.q.row, a.dim, kRows), og[n] = Tk::offset(n, wave, a.dy.row, a.dim, kRows);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&smem[0][0];
    const T *pq = (const T *)a.q.p + s * a.q.seq + q.q0 * a.q.row, *pg = (const T *)a.dy.p + s * a.dy.seq + q.q0 * a.dy.row;
    const int64_t row0 = a.packed ? q.q0 : (int64_t)s * a.q_len;
    float2 stat;
    auto load = [&](int n, int g, int i0) {
        const int head = hk * a.group + g, valid = q.lq - i0;
        const i32x4 bq = buffer_at(pq + (int64_t)i0 * a.q.row + head * a.q.head), bg = buffer_at(pg + (int64_t)i0 * a.dy.row + head * a.dy.head);
        const uint32_t to = lds + (n & 1) * 2 * Tk::kBytes + wave * 1024;
        stat = {INFINITY, 0};                               // past the last row: P = 0
        if ((int)threadIdx.x < min(valid, kRows)) stat = a.rows[(int64_t)head * a.q_rows + row0 + i0 + threadIdx.x];
#pragma unroll
        for (int m = 0; m < Tk::kLoads; m++) {
            mm::load_to_lds(bq, valid >= kRows ? oq[m] : Tk::offset(m, wave, a.q.row, a.dim, valid), to + m * 4096);
            mm::load_to_lds(bg, valid >= kRows ? og[m] : Tk::offset(m, wave, a.dy.row, a.dim, valid), to + Tk::kBytes + m * 4096);
        }
    };
    auto keep = [&](int n) {
        if (threadIdx.x < kRows) stats[n & 1][0][threadIdx.x] = stat.x, stats[n & 1][1][threadIdx.x] = stat.y;
    };
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) dk[d] = f32x16{}, dv[d] = f32x16{};
    if (count) load(0, 0, start), keep(0);
    int g = 0, i0 = start;
    for (int n = 0; n < count; n++) {
        const int head = hk * a.group + g, i = i0;
        i0 += kRows;
        if (i0 >= q.lq) i0 = start, g++;
        mm::arrive();
        if (n + 1 < count) load(n + 1, g, i0);
        const char *tq = smem[n & 1], *tg = tq + Tk::kBytes;
        const float slope2 = MOD && a.d_slopes ? a.d_slopes[head] * kLog2e : 0.0f;
#pragma unroll
        for (int u = 0; u < kRows / 32; u++) {
            const int b = i + u * 32;
            if (b + 31 < mine || b >= q.lq) continue;
            f32x16 p = {}, ds = {};
#pragma unroll
            for (int k = 0; k < DP / 16; k++) p = mfma(row_fragment<DP, T>(tq, u * 32 + col, k, h), kf[k], p);
#pragma unroll
            for (int k = 0; k < DP / 16; k++) ds = mfma(row_fragment<DP, T>(tg, u * 32 + col, k, h), vf[k], ds);
            float ls[16], de[16];
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const mm::f32x4 x = *(const mm::f32x4 *)&stats[n & 1][0][u * 32 + mfma_row(r, h)], y = *(const mm::f32x4 *)&stats[n & 1][1][u * 32 + mfma_row(r, h)];
#pragma unroll
                for (int m = 0; m < 4; m++) ls[r + m] = x[m], de[r + m] = y[m];
            }
            const int first = b + 4 * h;
            weigh<MOD>(a, p, ds, slope2, j - shift - first, b < whole, [&](int r) { return first + mfma_row(r, 0) >= from; },
                       [&](int r) { return ls[r]; }, [&](int r) { return de[r]; });
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const frag bp = pack<T>(p, 8 * k), bs = pack<T>(ds, 8 * k);
#pragma unroll
                for (int d = 0; d < DP / 32; d++) {
                    dv[d] = mfma(column_fragment<DP, T>(tg, u * 32 + 16 * k, d), bp, dv[d]);
                    dk[d] = mfma(column_fragment<DP, T>(tq, u * 32 + 16 * k, d), bs, dk[d]);
                }
            }
        }
        if (n + 1 < count) keep(n + 1);
    }
    if (!any) return;
    T *ok = (T *)a.dk.p + s * a.dk.seq + (q.k0 + j) * a.dk.row + hk * a.dk.head;
    T *ov = (T *)a.dv.p + s * a.dv.seq + (q.k0 + j) * a.dv.row + hk * a.dv.head;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            store4<T>(ok, d * 32 + mfma_row(r, h), a.dim, a.out_vec, dk[d][r] * a.scale, dk[d][r + 1] * a.scale, dk[d][r + 2] * a.scale, dk[d][r + 3] * a.scale);
            store4<T>(ov, d * 32 + mfma_row(r, h), a.dim, a.out_vec, dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]);
        }
}

template <typename T, int DP, bool MOD> static void launch(const Args &a, int64_t blocks, int64_t tiles, int64_t kblocks, int64_t ktiles, hipStream_t stream)
{
    if (blocks) hipLaunchKernelGGL((rows_kernel<T, DP, MOD>), dim3((unsigned)blocks), dim3(256), 0, stream, a, tiles);
    if (kblocks) hipLaunchKernelGGL((keys_kernel<T, DP, MOD>), dim3((unsigned)kblocks), dim3(256), 0, stream, a, ktiles);
}

int backward(const heddle_attention_desc *d, mm::Scratch &s, bool run, hipStream_t stream)
{
    Args a = base_args(d);
    a.grads = (d->dq ? 1 : 0) | (d->dk ? 2 : 0);
    if (d->sequences == 0 || !a.grads) return HEDDLE_OK;
    Copies c;
    if (a.q_rows) c.add(d, a.q, false, s);
    if (a.q_rows) c.add(d, a.y, false, s);
    if (a.q_rows) c.add(d, a.dy, false, s);
    if (a.k_rows) c.add(d, a.k, true, s);
    if (a.k_rows) c.add(d, a.v, true, s);
    a.rows = (float2 *)s.take((size_t)a.q_rows * d->heads * 8);
    auto aligned = [&](const void *p, const View &v) { return !((uintptr_t)p & 7) && !((v.seq | v.row | v.head | d->dim) & 3); };
    a.out_vec = (!d->dq || aligned(d->dq, a.dq)) && (!d->dk || (aligned(d->dk, a.dk) && aligned(d->dv, a.dv)));
    const int64_t blocks = a.q_rows ? slots_of(d->packed, d->sequences, d->q_len, d->q_len, a.group, 128) * d->kv_heads : 0;
    const int64_t tiles = (d->q_len * a.group + 127) / 128, ktiles = (d->k_len + 127) / 128;
    const int64_t kblocks = d->dk && a.k_rows ? slots_of(d->packed, d->sequences, d->k_len, d->k_len, 1, 128) * d->kv_heads : 0;
    if (std::max(blocks, kblocks) > (int64_t(1) << 24) - 1) return fail(HEDDLE_E_RANGE, "more tiles than a launch holds");
    if (!run) return HEDDLE_OK;
    if (const int rc = c.launch(stream)) return rc;
    const bool mod = modified(d), narrow = d->dim <= 64;
    auto call = [&](auto t) {
        typedef decltype(t) T;
        if (narrow) mod ? launch<T, 64, true>(a, blocks, tiles, kblocks, ktiles, stream) : launch<T, 64, false>(a, blocks, tiles, kblocks, ktiles, stream);
        else mod ? launch<T, 128, true>(a, blocks, tiles, kblocks, ktiles, stream) : launch<T, 128, false>(a, blocks, tiles, kblocks, ktiles, stream);
    };
    if (d->dtype == HEDDLE_T_BF16) call((__bf16)0.0f);
    else call((_Float16)0.0f);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "attention's gradients");
}

}  // namespace attn
}  // namespace heddle
