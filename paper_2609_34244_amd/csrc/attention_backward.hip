// The gradients of attention on gfx950's matrix cores, from the kept lse.
//
// P = exp(s - lse), delta = sum dy y, dP = dY V^T, dS = P (dP - delta), with a cap dS (1 - tanh^2);
// dq = scale dS K, dk = scale dS^T Q, dv = P^T dY. P is formed again in both kernels, so that each
// sum stays in registers and is added up in one order, without atomics: 7 products instead of 5.
// rows_kernel (dq): 128 query rows a workgroup, tiles of 64 keys, like the forward pass; it also
// leaves lse log2(e) and delta of its rows for the other one. keys_kernel (dk, dv): 128 keys or two times 128 a
// workgroup, 32 a wavefront, over tiles of query rows of each head of the group in turn, whose sum
// the shared heads' gradient is; the values' operands are read from LDS, as with keys, values and both sums in registers a SIMD
// would hold one wavefront.
// P and dS are rounded to the operands' type, and D is formed from the y of that type that the caller keeps: in bf16 dq and dk are off by
// 0.25%, dv by 0.23%, where fp32 throughout is off by the 0.17% of its last rounding. A second operand of what dS's rounding leaves
// brings dq and dk to 0.18 to 0.19%, and the layer below with its forward pass from 1534 us to 1750, 11 documents of 4092 rows from 194 to 212.
// Bound as the forward pass is: 4 sequences of 2048, 64 heads on 8: dq 452 us, dk and dv 562 us (912 and 977 TFLOP/s of products), with a
// cap 509 and 646.
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

// The cap's derivative is 1 - tanh^2 = 4 (x - x^2), x = 1 / (1 + e^u); kLift of the 4 is taken here, the rest by scale_of().
template <typename T> constexpr float kLift = __is_same(T, _Float16) ? 4.0f : 1.0f;   // float16 has no range to spare
template <typename T, int MODE> __device__ inline float scale_of(const Args &a) { return MODE & kCap ? a.scale * (4.0f / kLift<T>) : a.scale; }

// A probability from a score, and P times the cap's derivative where there is one. start: what
// the exponent starts from, cap log2(e) - lse log2(e) (READY: the score's sum started from -lse / scale instead).
// distance: from register 0's key or row (the sign does not matter).
template <typename T, int MODE, bool READY> HEDDLE_INLINE float2 weigh(const Args &a, float s, int r, float start, float slope2, float distance, bool seen)
{
    float w = 1;
    if constexpr (MODE == kPlain) {
        s = READY ? s * a.scale2 : __builtin_fmaf(s, a.scale2, start);
    } else if constexpr (MODE & kCap) {
        const float x = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s * a.scale2));
        s = __builtin_fmaf(-2.0f * a.cap2, x, start);
        w = __builtin_fmaf(-x, x, x);
    } else {
        s = __builtin_fmaf(s, a.scale2, start);
    }
    if constexpr (MODE & kSlopes) s = __builtin_fmaf(-slope2, fabsf(distance - (float)(8 * (r >> 2) + (r & 3))), s);
    float p = __builtin_amdgcn_exp2f(s);
    p = seen ? p : 0.0f;
    float pw = MODE & kCap ? p * (kLift<T> * w) : p;
    here(pw);
    return {p, pw};
}

template <typename T, int DP, int MODE> __global__ void __launch_bounds__(256, 2) rows_kernel(Args a)
{
    typedef Tile<DP, 64, 4> Tk;
    constexpr int kRows = 128;
    typedef typename mm::pack8<T>::type frag;
    __shared__ __align__(1024) char smem[2][2 * Tk::kBytes];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    if (__builtin_expect(blockIdx.x >= a.blocks, false)) return clear_rows(a, a.dq, false, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    const uint32_t slot = blockIdx.x / (uint32_t)a.kv_heads;
    const int hk = blockIdx.x - slot * a.kv_heads;
    Sequence q;
    int64_t tile;
    if (!find_tile(a, false, kRows, slot, a.blocks / (uint32_t)a.kv_heads, q, tile)) return;
    const int s = q.s;
    if (tile * kRows >= (int64_t)q.lq * a.group) return;
    const int rows = q.lq * a.group, r = (int)tile * kRows + wave * 32 + col;
    const bool any = r < rows;
    const int i = r / a.group, head = hk * a.group + (any ? r - i * a.group : 0), shift = q.lk - q.lq;
    auto limit_at = [&](int x) { return x >= rows ? 0 : max(min(q.lk, a.causal ? max(x / a.group + shift + 1, q.prefix) : q.lk), 0); };
    const int limit = limit_at(r), r0 = (int)tile * kRows + wave * 32;
    const int end = __builtin_amdgcn_readfirstlane(limit_at(min((int)tile * kRows + kRows - 1, rows - 1)));
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
    // Products of 32 keys, in this order: scores, dP, dq. Probabilities are formed between dP's; operands are read ahead.
    auto add = [&](int t, auto masked) __attribute__((always_inline)) {
        const char *tk = smem[t & 1], *tv = tk + Tk::kBytes;
        constexpr int N = DP / 16, kAhead = 4, M = 16 / N;      // N products each; M scores to a product
        each<2>([&](int c) __attribute__((always_inline)) {
            const int first = t * 64 + c * 32 + 4 * h;
            const float distance = (float)(i + shift - first);
            f32x16 p = {}, ds = {};
            Words<T> w;
            frag f[kAhead];
            auto fetch = [&](int n) __attribute__((always_inline)) {
                f[n % kAhead] = n < N ? row_fragment<DP, T>(tk, places, c * 32, n) : n < 2 * N ? row_fragment<DP, T>(tv, places, c * 32, n - N) :
                                column_fragment<DP, T>(tk, places, c * 32 + 16 * ((n - 2 * N) / (DP / 32)), (n - 2 * N) % (DP / 32));
            };
            each<kAhead - 1>([&](int n) __attribute__((always_inline)) { fetch(n); });
            each<3 * N>([&](int n) __attribute__((always_inline)) {
                if (n + kAhead - 1 < 3 * N) fetch(n + kAhead - 1);
                if (n < N) p = mfma(f[n % kAhead], qf[n], p);
                else if (n < 2 * N) {
                    ds = mfma(f[n % kAhead], gf[n - N], ds);
                    each<M>([&](int m) __attribute__((always_inline)) {
                        const int r = (n - N) * M + m;
                        p[r] = weigh<T, MODE, false>(a, p[r], r, base, slope2, distance, !decltype(masked)::value || first + mfma_row(r, 0) < limit).y;
                    });
                } else {
                    if (n == 2 * N) each<8>([&](int m) __attribute__((always_inline)) { w.set(m, p[2 * m] * (ds[2 * m] - delta), p[2 * m + 1] * (ds[2 * m + 1] - delta)); });
                    dq[(n - 2 * N) % (DP / 32)] = mfma(f[n % kAhead], w.half((n - 2 * N) / (DP / 32)), dq[(n - 2 * N) % (DP / 32)]);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
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
    store_row<T, DP>(out, dq, sc, a.dim, a.out_vec);
}

// Adds 32 rows of a tile (from its row `sub` on) to the gradients of 32 keys and values. Products in this order: scores,
// dP, dv, dk. Probabilities are formed between dP's, dS between dv's; operands are read ahead. ls, de: what the
// exponents or the scores' sums start from, and -delta, of the lane's rows; first: its first row; from: the first row that sees its key.
template <typename T, int DP, int MODE, bool MASKED, typename Value>
HEDDLE_INLINE void gather(const Args &a, f32x16 *dk, f32x16 *dv, const char *tq, const char *tg, int sub, const float *ls, const float *de,
                          const typename mm::pack8<T>::type *kf, Value value, const Places &places, int first, int from, int place, float slope2)
{
    constexpr int N = DP / 16, kAhead = 3, M = 16 / N;          // N products each; M scores to a product
    typedef typename mm::pack8<T>::type frag;
    const float distance = (float)(place - first);
    f32x16 p = {}, ds;
    if constexpr (MODE == kPlain) p = four(ls);
    mm::f32x4 l = {};
    Words<T> wp, ws;
    frag f[kAhead], v[kAhead];
    auto fetch = [&](int n) __attribute__((always_inline)) {
        const int k = (n - 2 * N) % N / (DP / 32) * 16, d = (n - 2 * N) % (DP / 32);
        f[n % kAhead] = n < N ? row_fragment<DP, T>(tq, places, sub, n) : n < 2 * N ? row_fragment<DP, T>(tg, places, sub, n - N) :
                        column_fragment<DP, T>(n < 3 * N ? tg : tq, places, sub + k, d);
        if (n >= N && n < 2 * N) v[n % kAhead] = value(n - N);
    };
    each<kAhead - 1>([&](int n) __attribute__((always_inline)) { fetch(n); });
    each<4 * N>([&](int n) __attribute__((always_inline)) {
        if (n + kAhead - 1 < 4 * N) fetch(n + kAhead - 1);
        const int k = (n - 2 * N) % N / (DP / 32), d = (n - 2 * N) % (DP / 32);
        if (n < N) {
            p = mfma(f[n % kAhead], kf[n], p);
            if (n == N - 1) ds = four(de);
        } else if (n < 2 * N) {
            ds = mfma(f[n % kAhead], v[n % kAhead], ds);
            each<M / 2>([&](int m) __attribute__((always_inline)) {
                const int r = (n - N) * M + 2 * m;
                if (MODE != kPlain && (r & 3) == 0) l = *(const mm::f32x4 *)(ls + 2 * r);
                const float2 x = weigh<T, MODE, true>(a, p[r], r, l[r & 3], slope2, distance, !MASKED || first + mfma_row(r, 0) >= from);
                const float2 y = weigh<T, MODE, true>(a, p[r + 1], r + 1, l[(r + 1) & 3], slope2, distance, !MASKED || first + mfma_row(r + 1, 0) >= from);
                wp.set(r / 2, x.x, y.x);
                p[r] = x.y, p[r + 1] = y.y;
            });
        } else if (n < 3 * N) {
            dv[d] = mfma(f[n % kAhead], wp.half(k), dv[d]);
            each<M / 2>([&](int m) __attribute__((always_inline)) {
                const int r = (n - 2 * N) * M + 2 * m;
                ws.set(r / 2, p[r] * ds[r], p[r + 1] * ds[r + 1]);
            });
        } else {
            dk[d] = mfma(f[n % kAhead], ws.half(k), dk[d]);
        }
        __builtin_amdgcn_sched_barrier(0);
    });
}

HEDDLE_INLINE void clear_keys(const Args &a, uint32_t b, uint32_t n)
{
    if (a.grads & 4) clear_rows(a, a.dk, true, b, n);
    if (a.grads & 8) clear_rows(a, a.dv, true, b, n);
}

// NW 8: two tiles of 128 keys a workgroup, the sequence's p-th and p-th from the end, which together see as many rows as
// any other such pair, and share the rows' tiles.
template <typename T, int DP, int MODE, int NW> __global__ void __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) keys_kernel(Args a)
{
    constexpr int kRows = DP == 64 && NW == 8 ? 64 : 32;
    typedef Tile<DP, kRows, NW> Tk;
    typedef typename mm::pack8<T>::type frag;
    __shared__ __align__(1024) char smem[2][2 * Tk::kBytes];
    typedef Tile<DP, 128, 4> Tv;
    __shared__ __align__(1024) char values[NW / 4][Tv::kBytes];
    __shared__ __align__(16) float stats[2][2][kRows];      // what the exponents, or the scores' sums, start from; -delta
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    if (__builtin_expect(blockIdx.x >= a.blocks, false)) return clear_keys(a, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    const uint32_t slot = blockIdx.x / (uint32_t)a.kv_heads;
    const int hk = blockIdx.x - slot * a.kv_heads;
    Sequence q;
    int64_t tile;
    if (!find_tile(a, true, 32 * NW, slot, a.blocks / (uint32_t)a.kv_heads, q, tile)) return;
    const int s = q.s;
    if (tile * (32 * NW) >= q.lk) return;
    const int team = wave >> 2, last_tile = (q.lk + 127) / 128 - 1, own = team ? last_tile - (int)tile : (int)tile;
    const int j0 = own * 128, w0 = j0 + (wave & 3) * 32, j = w0 + col, shift = q.lk - q.lq;   // the wavefront's keys: w0 on
    const bool busy = w0 < q.lk && (team == 0 || own > (int)tile), any = busy && j < q.lk;
    // the first row of a head that sees a key
    auto first_of = [&](int key) { return a.causal && key >= q.prefix ? max(key - shift, 0) : 0; };
    const int from = first_of(j), start = first_of((int)tile * 128) / kRows * kRows;
    const int whole = __builtin_amdgcn_readfirstlane(first_of(w0 + 31)), mine = busy ? __builtin_amdgcn_readfirstlane(first_of(w0)) : INT32_MAX;
    const int per = q.lq > start ? (q.lq - start + kRows - 1) / kRows : 0, count = per * a.group;

    const T *pk = (const T *)a.k.p + s * a.k.seq + (q.k0 + j) * a.k.row + hk * a.k.head;
    const T *pv = (const T *)a.v.p + s * a.v.seq + (q.k0 + j0) * a.v.row + hk * a.v.head;
    frag kf[DP / 16];
#pragma unroll
    for (int k = 0; k < DP / 16; k++) kf[k] = global_fragment<T>(pk, k * 16 + 8 * h, a.dim, any);
    if (count) {
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&values[team][0] + (wave & 3) * 1024;
        const i32x4 bv = buffer_at(pv);
#pragma unroll
        for (int n = 0; n < Tv::kLoads; n++) mm::load_to_lds(bv, Tv::offset(n, wave & 3, a.v.row, a.dim, q.lk - j0), to + n * 4096);
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
            mm::load_to_lds(bq, valid >= kRows ? oq[m] : Tk::offset(m, wave, a.q.row, a.dim, valid), to + m * (NW * 1024));
            mm::load_to_lds(bg, valid >= kRows ? og[m] : Tk::offset(m, wave, a.dy.row, a.dim, valid), to + Tk::kBytes + m * (NW * 1024));
        }
    };
    auto keep = [&](int n) {
        if (threadIdx.x < kRows) stats[n & 1][0][threadIdx.x] = MODE != kPlain ? a.cap2 - stat.x : stat.x * a.unscale, stats[n & 1][1][threadIdx.x] = -stat.y;
    };
    Places places;
    places.set<DP>();
    const char *mine_values = values[team] + (wave & 3) * (32 * DP * 2);
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
        each<kRows / 32>([&](int c) __attribute__((always_inline)) {
            gather<T, DP, MODE, decltype(masked)::value>(a, dk, dv, tq, tg, c * 32, &stats[slot_of][0][c * 32 + 4 * h], &stats[slot_of][1][c * 32 + 4 * h], kf,
                                                         [&](int n) __attribute__((always_inline)) { return row_fragment<DP, T>(mine_values, places, 0, n); }, places,
                                                         i + c * 32 + 4 * h, from, j - shift, slope2);
        });
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
    store_row<T, DP>(ok, dk, sc, a.dim, a.out_vec);
    store_row<T, DP>(ov, dv, 1.0f, a.dim, a.out_vec);
}

// Few keys: 32 a workgroup, whose eight wavefronts take tiles of 32 rows in turn, each with a tile and sums of its own; the
// sums are added up at the end. One tile a wavefront: while it waits for the next, the other wavefront of its SIMD has
// its products (3 sequences of 333, 12 heads on 4: 41 us with 128 keys a workgroup, which leaves most CUs without one,
// 30 with four wavefronts of two tiles).
template <typename T, int DP, int MODE> __global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) few_keys_kernel(Args a, int64_t tiles)
{
    typedef Tile<DP, 32, 1> Tk;
    typedef typename mm::pack8<T>::type frag;
    constexpr int kStage = 2 * Tk::kBytes, kLine = DP + 4;
    static_assert(4 * 32 * kLine * 4 <= 8 * kStage && 4 * 2 * DP / 2 * 64 * 4 <= 8 * kStage, "the wavefronts' sums fit where the tiles were");
    __shared__ __align__(1024) char smem[8][kStage], values[Tk::kBytes];
    __shared__ __align__(16) float stats[8][2][32];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    if (__builtin_expect(blockIdx.x >= a.blocks, false)) return clear_keys(a, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    const uint32_t slot = blockIdx.x / (uint32_t)a.kv_heads;
    const int hk = blockIdx.x - slot * a.kv_heads;
    int s;
    int64_t tile;
    if (!find_slot(a.d_k, a.k_rows, a.packed, a.sequences, 1, 32, tiles, slot, s, tile)) return;
    const Sequence q = sequence_of(a, s);
    if (tile * 32 >= q.lk) return;
    const int j0 = (int)tile * 32, j = j0 + col, shift = q.lk - q.lq;
    const bool any = j < q.lk;
    auto first_of = [&](int key) { return a.causal && key >= q.prefix ? max(key - shift, 0) : 0; };
    const int from = first_of(j), start = first_of(j0) / 32 * 32;
    const int per = q.lq > start ? (q.lq - start + 31) / 32 : 0, count = per * a.group;

    const T *pk = (const T *)a.k.p + s * a.k.seq + (q.k0 + j) * a.k.row + hk * a.k.head;
    const T *pv = (const T *)a.v.p + s * a.v.seq + (q.k0 + j0) * a.v.row + hk * a.v.head;
    frag kf[DP / 16];
#pragma unroll
    for (int k = 0; k < DP / 16; k++) kf[k] = global_fragment<T>(pk, k * 16 + 8 * h, a.dim, any);
    if (wave < Tk::kLoads)                                  // (one instruction a wavefront)
        mm::load_to_lds(buffer_at(pv), Tk::offset(wave, 0, a.v.row, a.dim, q.lk - j0), (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&values[0] + wave * 1024);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&smem[wave][0];
    const T *pq = (const T *)a.q.p + s * a.q.seq + q.q0 * a.q.row, *pg = (const T *)a.dy.p + s * a.dy.seq + q.q0 * a.dy.row;
    const int64_t row0 = a.packed ? q.q0 : (int64_t)s * a.q_len;
    auto load = [&](int n) __attribute__((always_inline)) {
        const int g = n / per, i0 = start + (n - g * per) * 32, head = hk * a.group + g, valid = q.lq - i0;
        const i32x4 bq = buffer_at(pq + (int64_t)i0 * a.q.row + head * a.q.head), bg = buffer_at(pg + (int64_t)i0 * a.dy.row + head * a.dy.head);
        float2 stat = {INFINITY, 0};                        // past the last row: P = 0
        if (lane < min(valid, 32)) stat = a.rows[(int64_t)head * a.q_rows + row0 + i0 + lane];
#pragma unroll
        for (int m = 0; m < Tk::kLoads; m++) {
            mm::load_to_lds(bq, Tk::offset(m, 0, a.q.row, a.dim, valid), lds + m * 1024);
            mm::load_to_lds(bg, Tk::offset(m, 0, a.dy.row, a.dim, valid), lds + Tk::kBytes + m * 1024);
        }
        if (lane < 32) stats[wave][0][lane] = MODE != kPlain ? a.cap2 - stat.x : stat.x * a.unscale, stats[wave][1][lane] = -stat.y;
    };
    Places places;
    places.set<DP>();
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) dk[d] = f32x16{}, dv[d] = f32x16{};
    if (wave < count) load(wave);
    mm::arrive();                                           // the values
    for (int n = wave; n < count; n += 8) {
        const int g = n / per, i = start + (n - g * per) * 32;
        const float slope2 = MODE & kSlopes ? a.d_slopes[hk * a.group + g] * kLog2e : 0.0f;
        const char *tq = smem[wave];
        gather<T, DP, MODE, true>(a, dk, dv, tq, tq + Tk::kBytes, 0, &stats[wave][0][4 * h], &stats[wave][1][4 * h], kf,
                                  [&](int k) __attribute__((always_inline)) { return row_fragment<DP, T>(values, places, 0, k); }, places, i + 4 * h, from, j - shift, slope2);
        if (n + 8 >= count) break;
        // a wavefront's tile is its own: it waits for its reads of it before it is filled again, and for its loads
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load(n + 8);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }
    // the upper four wavefronts' sums to the lower four
    float *sums = (float *)&smem[0][0];
    __syncthreads();
    if (wave >= 4) {
#pragma unroll
        for (int d = 0; d < DP / 32; d++)
#pragma unroll
            for (int r = 0; r < 16; r++) {
                sums[((wave & 3) * DP + d * 16 + r) * 64 + lane] = dk[d][r];
                sums[((wave & 3) * DP + DP / 2 + d * 16 + r) * 64 + lane] = dv[d][r];
            }
    }
    __syncthreads();
    if (wave < 4) {
#pragma unroll
        for (int d = 0; d < DP / 32; d++)
#pragma unroll
            for (int r = 0; r < 16; r++) {
                dk[d][r] += sums[(wave * DP + d * 16 + r) * 64 + lane];
                dv[d][r] += sums[(wave * DP + DP / 2 + d * 16 + r) * 64 + lane];
            }
    }
    // those four's sums, of keys, then of values
    const int mine = threadIdx.x >> 3, sub = threadIdx.x & 7;
    const float sc = scale_of<T, MODE>(a);
    each<2>([&](int which) __attribute__((always_inline)) {
        __syncthreads();
        if (wave < 4)
#pragma unroll
        for (int d = 0; d < DP / 32; d++)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x16 &x = which ? dv[d] : dk[d];
                *(mm::f32x4 *)(sums + (wave * 32 + col) * kLine + d * 32 + mfma_row(r, h)) = mm::f32x4{x[r], x[r + 1], x[r + 2], x[r + 3]};
            }
        __syncthreads();
        if (wave >= 4 || j0 + mine >= q.lk) return;
        const View &o = which ? a.dv : a.dk;
        T *out = (T *)o.p + s * o.seq + (q.k0 + j0 + mine) * o.row + hk * o.head;
        const float f = which ? 1.0f : sc;
#pragma unroll
        for (int c = 0; c < DP / 32; c++) {
            const int d = c * 32 + sub * 4;
            mm::f32x4 v = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; w++) v += *(const mm::f32x4 *)(sums + (w * 32 + mine) * kLine + d);
            store4<T>(out, d, a.dim, a.out_vec, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
        }
    });
}

static void launch_rows(const heddle_attention_desc *d, Args a, int64_t blocks, hipStream_t stream)
{
    a.blocks = (uint32_t)blocks;
    const dim3 grid(a.blocks + (d->dq ? clearing(d, 1, false, 256) : 0));
    with_kind(d, [&](auto t, auto dp, auto mode) {
        hipLaunchKernelGGL((rows_kernel<decltype(t), dp, mode>), grid, dim3(256), 0, stream, a);
    });
}
static void launch_keys(const heddle_attention_desc *d, Args a, int span, int64_t blocks, int64_t tiles, hipStream_t stream)
{
    a.blocks = (uint32_t)blocks;
    const dim3 grid(a.blocks + clearing(d, 6, true, 256));
    with_kind(d, [&](auto t, auto dp, auto mode) {
        if (span == 32) hipLaunchKernelGGL((few_keys_kernel<decltype(t), dp, mode>), grid, dim3(512), 0, stream, a, tiles);
        else if (span == 256) hipLaunchKernelGGL((keys_kernel<decltype(t), dp, mode, 8>), grid, dim3(512), 0, stream, a);
        else hipLaunchKernelGGL((keys_kernel<decltype(t), dp, mode, 4>), grid, dim3(256), 0, stream, a);
    });
}

int backward(const heddle_attention_desc *d, mm::Scratch &s, bool run, hipStream_t stream)
{
    Args a = base_args(d);
    if (!d->dq && !d->dk) return HEDDLE_OK;
    a.grads = (d->dq ? 1 : 0) | (d->clear & 6) * 2;
    auto aligned = [&](const void *p, const View &v) { return !((uintptr_t)p & 15) && !((v.seq | v.row | v.head | d->dim) & 7); };
    a.out_vec = (!d->dq || aligned(d->dq, a.dq)) && (!d->dk || (aligned(d->dk, a.dk) && aligned(d->dv, a.dv)));
    if (d->sequences == 0) return run ? clear_all(d, a, true, stream) : HEDDLE_OK;
    Copies c;
    if (a.q_rows) c.add(d, a.q, false, s);
    if (a.q_rows) c.add(d, a.y, false, s);
    if (a.q_rows) c.add(d, a.dy, false, s);
    if (a.k_rows) c.add(d, a.k, true, s);
    if (a.k_rows) c.add(d, a.v, true, s);
    a.rows = (float2 *)s.take((size_t)a.q_rows * d->heads * 8);
    const int64_t blocks = a.q_rows ? slots_of(d->packed, d->sequences, d->q_len, d->q_len, a.group, 128) * d->kv_heads : 0;
    const int64_t span = plan_keys({d->sequences, a.q_rows, a.k_rows, d->heads, d->kv_heads});
    const int64_t ktiles = (d->k_len + span - 1) / span;
    const int64_t kblocks = d->dk && a.k_rows ? slots_of(d->packed, d->sequences, d->k_len, d->k_len, 1, span) * d->kv_heads : 0;
    if (std::max(blocks, kblocks) > kMostBlocks) return fail(HEDDLE_E_RANGE, "more tiles than a launch holds");
    if (!run) return HEDDLE_OK;
    if (const int rc = c.launch(stream)) return rc;
    if (blocks) launch_rows(d, a, blocks, stream);
    if (kblocks) launch_keys(d, a, (int)span, kblocks, ktiles, stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "attention's gradients");
}

}  // namespace attn
}  // namespace heddle
