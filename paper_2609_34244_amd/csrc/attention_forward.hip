// Attention's forward pass over many query rows.
//
// A workgroup of four or eight wavefronts takes 32 rows each over tiles of 64 keys; keys and values are in LDS twice. Bound by the
// matrix cores and the vector units, which overlap little: a step of 32 keys is 16 products of 32 cycles and
// vector instructions of about 610 cycles with slopes, 900 with a cap. 8192 queries, 32 heads on 8, slopes: 564 us (975
// TFLOP/s; 659 with addresses formed at each read, masks in every tile, keys from first to last, and products and exponentials apart); 4
// sequences of 2048, 64 heads on 8: 330 us (832 TFLOP/s), with a cap 387.
#include "attention.h"

namespace heddle {
namespace attn {

// soften() in sixteen parts, to be done between products: 0 to 3 four scores each, 4 the maximum, 5 to 12 two
// probabilities each.
template <typename T, int MODE, bool MASKED> struct Softening {
    const Args &a;
    f32x16 &s;
    float &m;
    int first, limit;
    float distance, slope, top, was, base, sum = 0;
    bool follow;
    Words<T> words;
    HEDDLE_INLINE void part(int u)
    {
        const float unit = unit_of<MODE>(a);
        if (u < 4) {
            each<4>([&](int n) {
                const int r = 4 * u + n;
                s[r] = modify<MODE>(a, s[r], r, slope, distance);
                if constexpr (MASKED) s[r] = first + mfma_row(r, 0) >= limit ? -INFINITY : s[r];
                top = r ? fmaxf(top, s[r]) : s[r];
            });
        } else if (u == 4) {
            top = max_halves(top);
            follow = __any((top - m) * unit > 8.0f);
            was = m;
            m = follow ? fmaxf(m, top) : m;
            here(m);
            base = m == -INFINITY ? 0.0f : m * unit;
        } else if (u < 13) {
            const int r = 2 * (u - 5);
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], unit, -base)), y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], unit, -base));
            sum += x + y;
            words.set(r >> 1, x, y);
            here(sum);
        }
    }
    // all of them from the differences to the maximum (see is_far())
    HEDDLE_INLINE void again()
    {
        const float unit = unit_of<MODE>(a), at = m == -INFINITY ? 0.0f : m;
        sum = 0;
        each<8>([&](int i) {
            const float x = __builtin_amdgcn_exp2f((s[2 * i] - at) * unit), y = __builtin_amdgcn_exp2f((s[2 * i + 1] - at) * unit);
            sum += x + y;
            words.set(i, x, y);
        });
    }
};

template <typename T, int DP, int MODE, int NW> __global__ void __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) forward_kernel(Args a)
{
    typedef Tile<DP, 64, NW> Tk;
    constexpr int kRows = NW * 32;
    typedef typename mm::pack8<T>::type frag;
    __shared__ __align__(1024) char smem[2][2][Tk::kBytes]; // keys, values
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
    if (__builtin_expect(blockIdx.x >= a.blocks, false)) return clear_rows(a, a.y, false, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    // key heads fastest: 8 of them lie on one XCD each, whose L2 then holds its head's keys
    const uint32_t slot = blockIdx.x / (uint32_t)a.kv_heads;
    const int hk = blockIdx.x - slot * a.kv_heads;
    Sequence q;
    int64_t tile;
    if (!find_tile(a, false, kRows, slot, a.blocks / (uint32_t)a.kv_heads, q, tile)) return;
    const int s = q.s;
    if (tile * kRows >= (int64_t)q.lq * a.group) return;
    const int r0 = (int)tile * kRows, rows = q.lq * a.group;
    const Row row = row_of(a, q, hk, r0 + wave * 32 + (lane & 31));
    const int end = limit_of(a, q, min(r0 + kRows - 1, rows - 1)), mine = limit_of(a, q, min(r0 + wave * 32 + 31, max(rows - 1, r0 + wave * 32)));
    const int whole = r0 + wave * 32 + 31 < rows ? limit_of(a, q, r0 + wave * 32) : 0;   // keys that all of the wavefront's rows see
    const int count = (end + 63) / 64;

    const T *pk = (const T *)a.k.p + s * a.k.seq + q.k0 * a.k.row + hk * a.k.head;
    const T *pv = (const T *)a.v.p + s * a.v.seq + q.k0 * a.v.row + hk * a.v.head;
    int ok[Tk::kLoads], ov[Tk::kLoads];
#pragma unroll
    for (int i = 0; i < Tk::kLoads; i++) ok[i] = Tk::offset(i, wave, a.k.row, a.dim, 64), ov[i] = Tk::offset(i, wave, a.v.row, a.dim, 64);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&smem[0][0][0];
    // one half of a tile of 64 rows each: keys and values go their own ways
    auto load = [&](int t, const T *p, int64_t ld, const int *offsets, uint32_t to) __attribute__((always_inline)) {
        if (t >= count) return;
        const int row = (count - 1 - t) * 64, valid = q.lk - row;
        const i32x4 b = buffer_at(p + row * ld);
        to += (t & 1) * Tk::kBytes + wave * 1024;
        if (valid >= 64) {
#pragma unroll
            for (int i = 0; i < Tk::kLoads; i++) mm::load_to_lds(b, offsets[i], to + i * (NW * 1024));
        } else {
#pragma unroll
            for (int i = 0; i < Tk::kLoads; i++) mm::load_to_lds(b, Tk::offset(i, wave, ld, a.dim, valid), to + i * (NW * 1024));
        }
    };
    auto load_keys = [&](int t) __attribute__((always_inline)) { load(t, pk, a.k.row, ok, lds); };
    auto load_values = [&](int t) __attribute__((always_inline)) { load(t, pv, a.v.row, ov, lds + 2 * Tk::kBytes); };
    State<DP> st;
    st.init();
    Places at;
    at.set<DP>();
    load_keys(0);
    load_values(0);
    load_keys(1);
    frag qf[DP / 16];
    load_query<T, DP>(a, a.q, q, row, qf);
    const float slope = slope_of<MODE>(a, row.any ? row.head : 0);

    // Steps of 32 keys, from the last ones to the first: a bias by distance then has each row's maximum first, and
    // the sums are hardly scaled again. A step's probabilities are formed while the products of the next step's keys and
    // of the previous step's values run: the two are independent, and a wavefront's instructions of both kinds alternate.
    // Tile t's keys are used by the steps 2 t - 1 and 2 t, its values by 2 t + 1 and 2 t + 2, so that one barrier a tile,
    // between its two steps, frees a buffer of each.
    const int open = whole / 64, some = (mine + 63) / 64;   // tiles that all of the wavefront's rows see whole; that some see
    f32x16 now, then;
    frag was_p[2] = {};                                     // (of no keys before the first ones)
    auto turn = [&](int t) __attribute__((always_inline)) {
        mm::arrive();
        load_keys(t + 2);
        load_values(t + 1);
    };
    auto step = [&](f32x16 &s, f32x16 &next, const char *keys, int from, const char *values, int back, int j0, auto masked) __attribute__((always_inline)) {
        // even products: the next step's scores; odd ones: the previous step's values. Their operands are read kAhead ahead.
        constexpr int N = DP / 8, kAhead = 5;
        const int first = j0 + 4 * h;
        Softening<T, MODE, decltype(masked)::value> v = {a, s, st.m, first, row.limit, (float)(row.pos - first), slope};
        frag f[kAhead];
        auto fetch = [&](int i) __attribute__((always_inline)) {
            const int n = i >> 1;
            f[i % kAhead] = i & 1 ? column_fragment<DP, T>(values, at, back + n / (DP / 32) * 16, n % (DP / 32)) : row_fragment<DP, T>(keys, at, from, n);
        };
        next = f32x16{};
        each<kAhead - 1>([&](int i) __attribute__((always_inline)) { fetch(i); });
        each<N>([&](int i) __attribute__((always_inline)) {
            each<16 / N>([&](int n) __attribute__((always_inline)) { v.part(i * (16 / N) + n); });
            if (i + kAhead - 1 < N) fetch(i + kAhead - 1);
            const int n = i >> 1;
            if (i & 1) st.o[n % (DP / 32)] = mfma(f[i % kAhead], was_p[n / (DP / 32)], st.o[n % (DP / 32)]);
            else next = mfma(f[i % kAhead], qf[n], next);
            __builtin_amdgcn_sched_barrier(0);
        });
        // (Far rows' probabilities are formed twice: 8192 queries, 32 heads on 8, slopes take 577 us and 575 without all this, 571
        // and 560 on another card with the test between maximum and exponentials, where soften() has it.)
        if (__builtin_expect(v.follow || st.far, false)) {
            rescale<MODE>(a, st, v.was);
            st.far = is_far<MODE>(v.base);
            if (st.far) v.again();
        }
        st.l += v.sum;
        was_p[0] = v.words.half(0), was_p[1] = v.words.half(1);
    };
    auto tile_of = [&](int t, auto masked) __attribute__((always_inline)) {
        const int j0 = (count - 1 - t) * 64;
        const char *values = smem[1][t & 1];
        step(now, then, smem[0][t & 1], 0, t ? smem[1][~t & 1] : values, 0, j0 + 32, masked);
        turn(t);
        step(then, now, smem[0][~t & 1], 32, values, 32, j0, masked);
    };
    mm::arrive();
    int t = 0;
    for (; t < count - some; t++) turn(t);
    if (some) now = score<T, DP>(smem[0][t & 1], at, 32, qf);
    for (; t < count - open; t++) tile_of(t, std::true_type());
    for (; t < count; t++) tile_of(t, std::false_type());
    if (some) collect<T, DP>(st, smem[1][(count - 1) & 1], at, 0, was_p);
    const float l = st.l + other_half(st.l), inv = l == 0 ? 0.0f : 1.0f / l;
    T *y = (T *)a.y.p + s * a.y.seq + (q.q0 + row.i) * a.y.row + row.head * a.y.head;
    if (!row.any) return;                                   // (both of a row's lanes)
    store_row<T, DP>(y, st.o, inv, a.dim, a.out_vec);
    if (a.lse && h == 0)
        a.lse[row.at * a.heads + row.head] = l == 0 ? -INFINITY : (st.m * unit_of<MODE>(a) + offset_of<MODE>(a) + __log2f(l)) * kLn2;
}

void launch_forward(const heddle_attention_desc *d, Args a, int rows, int64_t blocks, hipStream_t stream)
{
    a.blocks = (uint32_t)blocks;
    const dim3 grid(a.blocks + clearing(d, 1, false, 2 * rows));
    with_kind(d, [&](auto t, auto dp, auto mode) {
        if (rows == 128) hipLaunchKernelGGL((forward_kernel<decltype(t), dp, mode, 4>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((forward_kernel<decltype(t), dp, mode, 8>), grid, dim3(512), 0, stream, a);
    });
}

}  // namespace attn
}  // namespace heddle
