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

// sixteen floats of a 32 x 32 product's rows: by fours, eight apart
HEDDLE_INLINE f32x16 four(const float *p)
{
    const mm::f32x4 a = *(const mm::f32x4 *)p, b = *(const mm::f32x4 *)(p + 8), c = *(const mm::f32x4 *)(p + 16), d = *(const mm::f32x4 *)(p + 24);
    const auto x = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), y = __builtin_shufflevector(c, d, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15);
}

// P and dS of 32 x 32 scores. INIT: the products' sums started from -delta and, without a cap or slopes, from
// -lse / scale. at: distance from register 0's key or row (the sign does not matter); seen(r): whether register r's
// pair is visible; start of four registers: cap log2(e) - lse log2(e); delta by register.
// The cap's derivative is 1 - tanh^2 = 4 (r - r^2), r = 1 / (1 + e^u); kLift of the 4 is taken here, the rest by scale_of().
template <typename T> constexpr float kLift = sizeof(T) == 2 && __is_same(T, _Float16) ? 4.0f : 1.0f;   // float16 has no range to spare
template <typename T, int MODE> __device__ inline float scale_of(const Args &a) { return MODE & kCap ? a.scale * (4.0f / kLift<T>) : a.scale; }

template <typename T, int MODE, bool INIT, bool MASKED, typename Seen, typename Start, typename Delta>
HEDDLE_INLINE void weigh(const Args &a, f32x16 &s, f32x16 &dp, float slope2, int at, Seen seen, Start start, Delta delta)
{
    if constexpr (!INIT) each<16>([&](int r) { dp[r] -= delta(r); });
    if constexpr (MODE == kPlain) {
        each<4>([&](int q) {
            mm::f32x4 l = {};
            if constexpr (!INIT) l = start(q);
            each<4>([&](int n) { s[4 * q + n] = __builtin_amdgcn_exp2f(INIT ? s[4 * q + n] * a.scale2 : __builtin_fmaf(s[4 * q + n], a.scale2, l[n])); });
        });
    } else {
        if constexpr (MODE & kCap) {
            each<4>([&](int q) {
                const mm::f32x4 l = start(q);
                each<4>([&](int n) {
                    const float x = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[4 * q + n] * a.scale2));
                    s[4 * q + n] = __builtin_fmaf(-2.0f * a.cap2, x, l[n]);
                    dp[4 * q + n] *= kLift<T> * __builtin_fmaf(-x, x, x);
                });
            });
        } else {
            each<4>([&](int q) {
                const mm::f32x4 l = start(q);
                each<4>([&](int n) { s[4 * q + n] = __builtin_fmaf(s[4 * q + n], a.scale2, l[n]); });
            });
        }
        if constexpr (MODE & kSlopes) {
            const float from = (float)at;
            each<16>([&](int r) { s[r] = __builtin_fmaf(-slope2, fabsf(from - (float)(8 * (r >> 2) + (r & 3))), s[r]); });
        }
        each<16>([&](int r) { s[r] = __builtin_amdgcn_exp2f(s[r]); });
    }
    if constexpr (MASKED) each<16>([&](int r) { s[r] = seen(r) ? s[r] : 0.0f; });
    each<16>([&](int r) { dp[r] *= s[r]; });
}

template <typename T, int DP, int MODE> __global__ void __launch_bounds__(256, 2) rows_kernel(Args a, int64_t tiles)
{
    typedef Tile<DP, 64, 4> Tk;
    typedef typename mm::pack8<T>::type frag;
    __shared__ __align__(1024) char smem[2][2 * Tk::kBytes];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int hk = blockIdx.x % (uint32_t)a.kv_heads;
    const int64_t slot = gridDim.x / (uint32_t)a.kv_heads - 1 - blockIdx.x / (uint32_t)a.kv_heads;
    int s;
    int64_t tile;
    if (a.packed) {
        if (!find_slot(a.d_q, a.q_rows, 1, a.sequences, a.group, 128, tiles, slot, s, tile)) return;
    } else {
        s = (int)((uint32_t)slot % (uint32_t)a.sequences), tile = (uint32_t)slot / (uint32_t)a.sequences;
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
    const float slope2 = MODE & kSlopes ? a.d_slopes[head] * kLog2e : 0.0f, base = a.cap2 - lse2;

    Places places;
    places.set<DP>();
    f32x16 dq[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) dq[d] = f32x16{};
    auto next = [&](int t) __attribute__((always_inline)) {
        mm::arrive();
        if (t + 1 < count) load(t + 1);
    };
    auto add = [&](int t, auto masked) __attribute__((always_inline)) {
        const char *tk = smem[t & 1], *tv = tk + Tk::kBytes;
#pragma unroll
        for (int c = 0; c < 2; c++) {
            f32x16 p = {}, ds = {};
#pragma unroll
            for (int k = 0; k < DP / 16; k++) p = mfma(row_fragment<DP, T>(tk, places, c * 32, k), qf[k], p);
#pragma unroll
            for (int k = 0; k < DP / 16; k++) ds = mfma(row_fragment<DP, T>(tv, places, c * 32, k), gf[k], ds);
            const int first = t * 64 + c * 32 + 4 * h;
            weigh<T, MODE, false, decltype(masked)::value>(a, p, ds, slope2, i + shift - first, [&](int n) { return first + mfma_row(n, 0) < limit; },
                                                          [&](int) { return mm::f32x4{base, base, base, base}; }, [&](int) { return delta; });
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const frag b = pack<T>(ds, 8 * k);
#pragma unroll
                for (int d = 0; d < DP / 32; d++) dq[d] = mfma(column_fragment<DP, T>(tk, places, c * 32 + 16 * k, d), b, dq[d]);
            }
        }
    };
    // tiles seen whole, in part, and by other wavefronts alone: see the forward pass
    const int open = min(whole / 64, count), some = min((mine + 63) / 64, count);
    int t = 0;
    for (; t < open; t++) {
        next(t);
        add(t, std::false_type());
    }
    for (; t < some; t++) {
        next(t);
        add(t, std::true_type());
    }
    for (; t < count; t++) next(t);
    if (!any) return;
    const float sc = scale_of<T, MODE>(a);
    T *out = (T *)a.dq.p + s * a.dq.seq + (q.q0 + i) * a.dq.row + head * a.dq.head;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int n = 0; n < 16; n += 4)
            store4<T>(out, d * 32 + mfma_row(n, h), a.dim, a.out_vec, dq[d][n] * sc, dq[d][n + 1] * sc, dq[d][n + 2] * sc, dq[d][n + 3] * sc);
}

template <typename T, int DP, int MODE> __global__ void __launch_bounds__(256, 2) keys_kernel(Args a, int64_t tiles)
{
    constexpr int kRows = 32;
    typedef Tile<DP, kRows, 4> Tk;
    typedef typename mm::pack8<T>::type frag;
    __shared__ __align__(1024) char smem[2][2 * Tk::kBytes];
    typedef Tile<DP, 128, 4> Tv;
    __shared__ __align__(1024) char values[Tv::kBytes];
    __shared__ __align__(16) float stats[2][2][kRows];      // what the exponents, or the scores' sums, start from; -delta
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int hk = blockIdx.x % (uint32_t)a.kv_heads;
    // The first tiles, which the most rows see, first. Where all workgroups find a place at once, two a CU, the second
    // half in reverse: a CU's two then have as much to do as another's (4 sequences of 2048, 64 heads on 8: 1118 us without).
    int64_t slot = blockIdx.x / (uint32_t)a.kv_heads;
    const int64_t slots = gridDim.x / (uint32_t)a.kv_heads, half = 256 / (uint32_t)a.kv_heads;
    if (slots <= 2 * half && slot >= half) slot = half + (slots - 1 - slot);
    int s;
    int64_t tile;
    if (a.packed) {
        if (!find_slot(a.d_k, a.k_rows, 1, a.sequences, 1, 128, tiles, slot, s, tile)) return;
    } else {
        s = (int)((uint32_t)slot % (uint32_t)a.sequences), tile = (uint32_t)slot / (uint32_t)a.sequences;
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
    const T *pv = (const T *)a.v.p + s * a.v.seq + (q.k0 + j0) * a.v.row + hk * a.v.head;
    frag kf[DP / 16];
#pragma unroll
    for (int k = 0; k < DP / 16; k++) kf[k] = global_fragment<T>(pk, k * 16 + 8 * h, a.dim, any);
    if (count) {
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&values[0] + wave * 1024;
        const i32x4 bv = buffer_at(pv);
#pragma unroll
        for (int n = 0; n < Tv::kLoads; n++) mm::load_to_lds(bv, Tv::offset(n, wave, a.v.row, a.dim, q.lk - j0), to + n * 4096);
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
        if (threadIdx.x < kRows) stats[n & 1][0][threadIdx.x] = MODE != kPlain ? a.cap2 - stat.x : stat.x * a.unscale, stats[n & 1][1][threadIdx.x] = -stat.y;
    };
    Places places;
    places.set<DP>();
    const char *mine_values = values + wave * (32 * DP * 2);
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) dk[d] = f32x16{}, dv[d] = f32x16{};
    if (count) load(0, 0, start), keep(0);
    int n = 0, slot_of = 0;                                 // tiles so far; the current one's buffer
    // the tile at row i of head g has arrived, the one after it is on its way
    auto next = [&](int g, int i) __attribute__((always_inline)) {
        mm::arrive();
        const bool last = i + kRows >= q.lq;
        if (n + 1 < count) load(n + 1, last ? g + 1 : g, last ? start : i + kRows);
        slot_of = n & 1;
    };
    auto leave = [&]() __attribute__((always_inline)) {
        n++;
        if (n < count) keep(n);
    };
    auto add = [&](int i, float slope2, auto masked) __attribute__((always_inline)) {
        const char *tq = smem[slot_of], *tg = tq + Tk::kBytes;
        const float *ls = &stats[slot_of][0][4 * h], *de = &stats[slot_of][1][4 * h];
        f32x16 p = {}, ds = four(de);
        if constexpr (MODE == kPlain) p = four(ls);
#pragma unroll
        for (int k = 0; k < DP / 16; k++) p = mfma(row_fragment<DP, T>(tq, places, 0, k), kf[k], p);
#pragma unroll
        for (int k = 0; k < DP / 16; k++) ds = mfma(row_fragment<DP, T>(tg, places, 0, k), row_fragment<DP, T>(mine_values, places, 0, k), ds);
        const int first = i + 4 * h;
        weigh<T, MODE, true, decltype(masked)::value>(a, p, ds, slope2, j - shift - first, [&](int r) { return first + mfma_row(r, 0) >= from; },
                                                     [&](int q) { return *(const mm::f32x4 *)(ls + 8 * q); }, [](int) { return 0.0f; });
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const frag bp = pack<T>(p, 8 * k), bs = pack<T>(ds, 8 * k);
#pragma unroll
            for (int d = 0; d < DP / 32; d++) {
                dv[d] = mfma(column_fragment<DP, T>(tg, places, 16 * k, d), bp, dv[d]);
                dk[d] = mfma(column_fragment<DP, T>(tq, places, 16 * k, d), bs, dk[d]);
            }
        }
    };
    if (count) {
        for (int g = 0; g < a.group; g++) {
            const float slope2 = MODE & kSlopes ? a.d_slopes[hk * a.group + g] * kLog2e : 0.0f;
            int i = start;
            // rows that see none of the wavefront's keys, some, all
            for (; i < q.lq && i + kRows <= mine; i += kRows) next(g, i), leave();
            for (; i < q.lq && i < whole; i += kRows) {
                next(g, i);
                add(i, slope2, std::true_type());
                leave();
            }
            for (; i < q.lq; i += kRows) {
                next(g, i);
                add(i, slope2, std::false_type());
                leave();
            }
        }
    }
    if (!any) return;
    const float sc = scale_of<T, MODE>(a);
    T *ok = (T *)a.dk.p + s * a.dk.seq + (q.k0 + j) * a.dk.row + hk * a.dk.head;
    T *ov = (T *)a.dv.p + s * a.dv.seq + (q.k0 + j) * a.dv.row + hk * a.dv.head;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            store4<T>(ok, d * 32 + mfma_row(r, h), a.dim, a.out_vec, dk[d][r] * sc, dk[d][r + 1] * sc, dk[d][r + 2] * sc, dk[d][r + 3] * sc);
            store4<T>(ov, d * 32 + mfma_row(r, h), a.dim, a.out_vec, dv[d][r], dv[d][r + 1], dv[d][r + 2], dv[d][r + 3]);
        }
}

void launch_rows(const heddle_attention_desc *d, const Args &a, int64_t blocks, int64_t tiles, hipStream_t stream)
{
    with_kind(d, [&](auto t, auto dp, auto mode) {
        hipLaunchKernelGGL((rows_kernel<decltype(t), dp, mode>), dim3((unsigned)blocks), dim3(256), 0, stream, a, tiles);
    });
}
void launch_keys(const heddle_attention_desc *d, const Args &a, int64_t blocks, int64_t tiles, hipStream_t stream)
{
    with_kind(d, [&](auto t, auto dp, auto mode) {
        hipLaunchKernelGGL((keys_kernel<decltype(t), dp, mode>), dim3((unsigned)blocks), dim3(256), 0, stream, a, tiles);
    });
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
    if (blocks) launch_rows(d, a, blocks, tiles, stream);
    if (kblocks) launch_keys(d, a, kblocks, ktiles, stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "attention's gradients");
}

}  // namespace attn
}  // namespace heddle
