// What the attention kernels on gfx950 share: tiles of keys (or of query rows) in LDS, fragments
// for the matrix cores, the scores' cap, bias and mask, and where a workgroup's rows lie.
//
// Products are of 32 x 32 x 16. Scores are formed as S^T = K Q^T (A: keys, B: query rows): a lane
// then holds 16 keys of ONE query row, so that a row's running maximum, sum and factors are one
// register of a lane (with the lane 32 on holding the other keys). P^T in this layout is
// the next product's B operand as it is, if that product's 16 terms are taken in the order in which
// the lanes hold them: 4 h + 0..3, 8 + 4 h + 0..3 for a lane of half h. The transposing LDS read
// brings the other operand (V^T, K^T, Q^T, dY^T) in that order.
//
// Tiles lie in LDS by blocks of 16 rows, in a block by 16-byte pieces of the rows: piece p of row r at
// 256 p + 16 (r ^ 4 (p % 4)) bytes. 16 lanes that read the same piece of 16 rows, and 32 lanes of a transposing
// read (4 rows, 64 bytes of each), touch every bank once, and all of a lane's addresses are two
// registers plus constants (with the pieces of a row side by side, exchanged by bits of the row, a sixth of the
// forward pass's vector instructions formed addresses).
// They are filled straight from global memory through a buffer resource, 64 bytes of 16 rows an instruction; rows
// past a sequence's end and columns past the head's width arrive as zeros.
#pragma once

#include <utility>

#include "attention_plan.h"
#include "linear.h"

namespace heddle {
namespace attn {

// a call would pass the sums through memory
#define HEDDLE_INLINE __device__ __attribute__((always_inline)) inline

// f(0) .. f(N - 1), each index a constant from the start: vectors that are passed by reference and indexed
// in loops stayed in memory where many of them were unrolled late
template <typename F, int... I> HEDDLE_INLINE void each_of(F f, std::integer_sequence<int, I...>) { (f(I), ...); }
template <int N, typename F> HEDDLE_INLINE void each(F f) { each_of(f, std::make_integer_sequence<int, N>()); }

// A value that is formed here, between the products before and after, and not where it is used: the compiler would
// gather what the vector units can do beside products behind them.
template <typename V> HEDDLE_INLINE void here(V &v)
{
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("" : "+v"(v));
#endif
}
template <typename T> struct Pair;
template <> struct Pair<__bf16> { typedef __bf16 type __attribute__((ext_vector_type(2))); };
template <> struct Pair<_Float16> { typedef _Float16 type __attribute__((ext_vector_type(2))); };

using mm::i32x4;
using mm::s16x4;
using mm::s16x8;
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ inline f32x16 mfma(mm::bf16x8 a, mm::bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma(mm::f16x8 a, mm::f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

constexpr int kClearing = 256;                // the most workgroups that clear rows
constexpr int64_t kMostBlocks = (int64_t(1) << 23) - 1 - kClearing;   // of 512 lanes: a launch has fewer than 2^32
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// a tensor of rows by heads: elements between sequences (0 where packed), rows and heads
struct View {
    const void *p;
    int64_t seq, row, head;
};

struct Args {
    View q, k, v, y, dy, dq, dk, dv;
    float *lse;                               // [query rows][heads], or NULL
    const int32_t *d_q, *d_k, *d_prefix;
    const float *d_slopes;
    float2 *rows;                             // [heads][query rows]: backward's lse log2(e) and delta
    float *partial;                           // few queries: [slot][key head][32 rows][parts][DP + 2]
    int64_t q_rows, k_rows;                   // of all sequences (batched: sequences * length)
    int32_t sequences, q_len, k_len, packed;
    int32_t heads, kv_heads, group, dim;
    int32_t causal, parts;
    uint32_t blocks;                          // the launch's workgroups for tiles; those past them clear rows
    int32_t out_vec, grads;                   // outputs on 16-byte addresses, their strides and dim whole eights; 1: dq wanted, 4, 8: dk, dv to be cleared
    float scale, scale2, cap2, unscale;       // scale2 = scale log2(e); with a cap: 2 scale log2(e) / cap and cap log2(e); -1 / scale2
};

// A sequence's rows: first row of its queries and of its keys, counted over all sequences where packed, else in the sequence.
struct Sequence {
    int64_t q0, k0;
    int32_t s, lq, lk, prefix;                // prefix: keys that every query sees
};

__device__ inline int clamp_row(int v, int64_t rows) { return (int)(v < 0 ? 0 : v > rows ? rows : v); }

__device__ inline Sequence sequence_of(const Args &a, int s)
{
    Sequence r;
    r.s = s;
    r.q0 = r.k0 = 0;
    r.lq = a.q_len, r.lk = a.k_len;
    if (a.packed) {
        const int q0 = clamp_row(a.d_q[s], a.q_rows), q1 = clamp_row(a.d_q[s + 1], a.q_rows);
        const int k0 = clamp_row(a.d_k[s], a.k_rows), k1 = clamp_row(a.d_k[s + 1], a.k_rows);
        r.q0 = q0, r.k0 = k0, r.lq = max(q1 - q0, 0), r.lk = max(k1 - k0, 0);
    } else {
        if (a.d_q) r.lq = clamp_row(a.d_q[s], a.q_len);
        if (a.d_k) r.lk = clamp_row(a.d_k[s], a.k_len);
    }
    r.prefix = a.d_prefix ? a.d_prefix[s] : 0;
    return r;
}

// The sequence and the tile in it of slot `slot`. Batched: `tiles` slots a sequence. Packed: sequence s has slots
// floor(off[s] mul / T) + s onwards, at least as many as its tiles and none that another one has, so that a
// slot's sequence is found by search alone: 64 of them looked at a step. Whatever the offsets hold, s and the rows
// stay inside.
__device__ inline bool find_slot(const int32_t *offsets, int64_t rows, int packed, int sequences, int mul, int T, int64_t tiles, int64_t slot,
                                 int &s, int64_t &tile)
{
    if (!packed) {
        s = (int)((uint32_t)slot / (uint32_t)tiles);        // (slots of a launch stay below 2^24)
        tile = slot - s * tiles;
        return s < sequences;
    }
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = sequences;
    for (;;) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const bool in = at < hi && (int64_t)clamp_row(offsets[min(at, sequences)], rows) * mul / T + at <= slot;
        const int count = __builtin_popcountll(__ballot(in));
        if (count == 0) return false;
        lo += (count - 1) * step;
        hi = min(hi, lo + step);
        if (step == 1) break;
    }
    s = __builtin_amdgcn_readfirstlane(lo);
    tile = slot - ((int64_t)clamp_row(offsets[s], rows) * mul / T + s);
    return tile >= 0;
}
// The sum over a wavefront, in a scalar register: within 16 lanes by moves of the vector units.
__device__ inline int wave_sum(int v)
{
#ifdef __HIP_DEVICE_COMPILE__
    v += __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);
    return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48);
#else
    return v;
#endif
}

// Tiles of up to 64 packed sequences by their number in their sequence, the highest first: slot `slot` of this order. The
// last tiles of the longest documents see the most keys, and begun last they would run on alone (11 documents of 4092
// rows, 32 heads: forward, dq, dk with dv 69, 80, 79 us in the documents' order, 62, 76, 70 so). F(t) tiles have a number of at least t.
__device__ inline bool find_ordered(const Args &a, bool keys, int T, int slot, Sequence &q, int64_t &tile, int &tiles)
{
    const int lane = threadIdx.x & 63, at0 = min(lane, a.sequences), at1 = min(lane + 1, a.sequences), mul = keys ? 1 : a.group;
    const int q0 = clamp_row(a.d_q[at0], a.q_rows), q1 = clamp_row(a.d_q[at1], a.q_rows);
    const int k0 = clamp_row(a.d_k[at0], a.k_rows), k1 = clamp_row(a.d_k[at1], a.k_rows);
    const int prefixes = a.d_prefix && a.sequences ? a.d_prefix[min(lane, a.sequences - 1)] : 0;
    const int from = keys ? k0 : q0, to = keys ? k1 : q1, sequences = a.sequences;
    const int mine = lane < sequences && to > from ? (int)(((int64_t)(to - from) * mul + T - 1) / T) : 0;
    auto f = [&](int t) { return wave_sum(max(mine - t, 0)); };
    const int all = f(0);
    if (slot >= all) return false;
    int lo = 0, hi = all, above = 0;                        // F(lo) > slot >= F(hi) = above
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2, n = f(mid);
        if (n > slot) lo = mid;
        else hi = mid, above = n;
    }
    const uint64_t with = __ballot(mine > lo);
    const uint64_t at = __ballot(mine > lo && __builtin_popcountll(with & ((1ull << lane) - 1)) == slot - above);
    if (at == 0) return false;                              // (not with offsets in order)
    q.s = __builtin_ctzll(at);
    q.q0 = __builtin_amdgcn_readlane(q0, q.s), q.k0 = __builtin_amdgcn_readlane(k0, q.s);
    q.lq = max(__builtin_amdgcn_readlane(q1, q.s) - (int)q.q0, 0), q.lk = max(__builtin_amdgcn_readlane(k1, q.s) - (int)q.k0, 0);
    q.prefix = __builtin_amdgcn_readlane(prefixes, q.s);
    tile = lo;
    tiles = __builtin_amdgcn_readlane(mine, q.s);
    return true;
}
// A workgroup's sequence and its tile of T query rows of a key head, or of T keys, those with the most work first; slots: how
// many there may be.
__device__ inline bool find_tile(const Args &a, bool keys, int T, uint32_t slot, uint32_t slots, Sequence &q, int64_t &tile)
{
    int s, tiles;
    if (!a.packed) {
        // the last tiles of queries see the most keys, the first tiles of keys are seen by the most queries
        const uint32_t at = keys ? slot : slots - 1 - slot;
        s = (int)(at % (uint32_t)a.sequences), tile = at / (uint32_t)a.sequences;
    } else if (a.sequences <= 64) {
        if (!find_ordered(a, keys, T, (int)slot, q, tile, tiles)) return false;
        if (keys) tile = tiles - 1 - tile;
        return true;
    } else if (!find_slot(keys ? a.d_k : a.d_q, keys ? a.k_rows : a.q_rows, 1, a.sequences, keys ? 1 : a.group, T, 0, keys ? slot : slots - 1 - slot, s, tile)) {
        return false;
    }
    q = sequence_of(a, s);
    return true;
}
inline int64_t slots_of(int packed, int64_t sequences, int64_t rows, int64_t length, int64_t mul, int64_t T)
{
    return packed ? rows * mul / T + sequences : sequences * ((length * mul + T - 1) / T);
}

// ---- tiles in LDS ----
constexpr int kNowhere = -16;                 // past any buffer's end: arrives as zeros

// ROWS x DP values by NW wavefronts, 1 KB of LDS an instruction
template <int DP, int ROWS, int NW> struct Tile {
    static constexpr int kBytes = ROWS * DP * 2, kLoads = kBytes / (1024 * NW), kGroups = DP / 32;   // groups of four pieces in a row
    static_assert(kLoads * NW * 1024 == kBytes && ROWS % 16 == 0, "whole instructions");
    // byte offset of a lane's piece of instruction i, from the tile's first row; valid: rows that the sequence has from there
    static __device__ inline int offset(int i, int wave, int64_t ld, int dim, int valid)
    {
        const int lane = threadIdx.x & 63, block = i * NW + wave, p = lane >> 4;
        const int row = block / kGroups * 16 + ((lane & 15) ^ p << 2), col = (block % kGroups * 4 + p) * 8;
        return row < valid && col < dim ? (row * (int)ld + col) * 2 : kNowhere;
    }
};

// a buffer from p on; every offset that is used lies in the tensor, or is kNowhere
__device__ inline i32x4 buffer_at(const void *p)
{
    const uint64_t v = (uint64_t)p;
    return i32x4{__builtin_amdgcn_readfirstlane((int)v), __builtin_amdgcn_readfirstlane((int)(v >> 32) & 0xffff), 0x7fffffff, 0x00020000};
}

// A lane's places in a tile (bytes): for reads of its row lane % 32, even and odd steps; for transposing reads.
struct Places {
    int row[2], column[2];
    template <int DP> __device__ inline void set()
    {
        const int lane = threadIdx.x & 63, h = lane >> 5, r = lane & 31, i = lane & 15, p = (lane >> 4 & 1) * 2 + (i >> 1 & 1);
        for (int k = 0; k < 2; k++) {
            row[k] = r / 16 * (DP * 32) + h * 256 + ((r & 15) ^ (2 * k + h) << 2) * 16;
            column[k] = p * 256 + ((4 * h + 8 * k + (i >> 2)) ^ p << 2) * 16 + (i & 1) * 8;
        }
    }
};

// 16 bytes of columns 16 step + 8 h of row from + lane % 32; from a multiple of 32
template <int DP, typename T> HEDDLE_INLINE typename mm::pack8<T>::type row_fragment(const char *tile, const Places &at, int from, int step)
{
    return *(const typename mm::pack8<T>::type *)(tile + at.row[step & 1] + (from / 16 * (DP * 32) + step * 512));
}

// Column 32 dt + lane % 32 of rows base + 4 h + 0..3 and base + 8 + 4 h + 0..3; base a multiple of 16.
template <int DP, typename T> HEDDLE_INLINE typename mm::pack8<T>::type column_fragment(const char *tile, const Places &at, int base, int dt)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef __attribute__((address_space(3))) s16x4 *rd;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((rd)(tile + at.column[0] + (base / 16 * (DP * 32) + dt * 1024)));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((rd)(tile + at.column[1] + (base / 16 * (DP * 32) + dt * 1024)));
    return __builtin_bit_cast(typename mm::pack8<T>::type, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#else
    return {};
#endif
}

// a lane's 8 values of a row in global memory, columns 16 step + 8 h, zeros past the head's width
template <typename T> __device__ inline typename mm::pack8<T>::type global_fragment(const T *row, int col, int dim, bool any)
{
    typename mm::pack8<T>::type x = {};
    if (any && col < dim) x = *(const typename mm::pack8<T>::type *)(row + col);
    return x;
}

// Zeros for an output's rows of no sequence: workgroup b of n that share them. They are workgroups of the kernel that writes the
// output's other rows; a launch of their own takes 2 us, and 3 of the host (11 documents of 4092 rows, 32 heads, training: 196.8 us without clearing, 198.3 so, 2% more
// with launches).
HEDDLE_INLINE void clear_rows(const Args &a, const View &v, bool keys, uint32_t b, uint32_t n)
{
    const int32_t *at = keys ? a.d_k : a.d_q;
    const int rows = keys ? a.k_len : a.q_len, heads = keys ? a.kv_heads : a.heads, per = (a.dim + 7) / 8, line = heads * per;
    const uint32_t sequences = a.packed ? 1 : a.sequences, chunks = max(1u, n / sequences);
    for (uint32_t x = b; x < sequences * chunks; x += n) {
        const uint32_t s = x % sequences, chunk = x / sequences;
        int first = 0, last = rows;                         // rows before the first and from the last on
        if (!a.packed) last = at ? clamp_row(at[s], rows) : rows;
        else if (a.sequences) first = clamp_row(at[0], rows), last = max(first, clamp_row(at[a.sequences], rows));
        else last = 0;
        const int64_t all = (int64_t)(first + rows - last) * line, step = (int64_t)chunks * blockDim.x;
        for (int64_t i = (int64_t)chunk * blockDim.x + threadIdx.x; i < all; i += step) {
            const int64_t u = i / line, row = u < first ? u : u - first + last;
            const int rest = (int)(i - u * line), head = rest / per, col = (rest - head * per) * 8;
            uint16_t *p = (uint16_t *)v.p + s * v.seq + row * v.row + head * v.head + col;
            if (a.out_vec) {
                *(s16x8 *)p = s16x8{};
            } else {
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (col + k < a.dim) p[k] = 0;
            }
        }
    }
}

// eight probabilities as the next product's operand, rounded to the type that the matrix cores read at full rate: in bf16 y is
// off by 0.19 to 0.22% where fp32 throughout is off by the 0.17% of its last rounding. A second operand of what the rounding
// leaves would be half as many products again; in split_kernel, bound by reading, 134 us for 131 (32 sequences of up to 8192 keys).
template <typename T> __device__ inline typename mm::pack8<T>::type pack(const f32x16 &p, int from)
{
    typename mm::pack8<T>::type x;
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = (T)p[from + i];
    return x;
}

// sixteen values as the next product's operands, two a word, each formed where it is set
template <typename T> struct Words {
    unsigned word[8];
    HEDDLE_INLINE void set(int i, float x, float y)
    {
        const typename Pair<T>::type v = {(T)x, (T)y};
        word[i] = __builtin_bit_cast(unsigned, v);
        here(word[i]);
    }
    HEDDLE_INLINE typename mm::pack8<T>::type half(int k) const
    {
        typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
        return __builtin_bit_cast(typename mm::pack8<T>::type, u32x4{word[4 * k], word[4 * k + 1], word[4 * k + 2], word[4 * k + 3]});
    }
};

// row of a 32 x 32 product's register r
__device__ inline int mfma_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

__device__ inline float other_half(float v) { return __shfl_xor(v, 32); }
// the greater of a lane's value and the other half's
__device__ inline float max_halves(float v)
{
#ifdef __HIP_DEVICE_COMPILE__
    // (written out: of the builtin's two results with one operand twice the compiler keeps one)
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return fmaxf(a, b);
#else
    return v;
#endif
}

// What is done to the scores, fixed for a kernel: a test in the loop would keep its products and exponentials apart.
enum Mode { kPlain = 0, kCap = 1, kSlopes = 2 };

// Scores in the units of the running maximum, which unit_of() turns into powers of two. With a cap:
// -1 / (1 + e^u), u = 2 scale q k / cap, as tanh(u / 2) = 1 - 2 / (1 + e^u) and a row's constants
// cancel (offset_of() has them for lse). slope: in these units. distance: from register 0's key to the row's place.
template <int MODE> HEDDLE_INLINE float unit_of(const Args &a) { return MODE & kCap ? 2 * a.cap2 : a.scale2; }
template <int MODE> HEDDLE_INLINE float offset_of(const Args &a) { return MODE & kCap ? a.cap2 : 0.0f; }
// the same where the mode is not a constant
__device__ inline float unit_of(const Args &a) { return a.cap2 > 0 ? 2 * a.cap2 : a.scale2; }
template <int MODE> HEDDLE_INLINE float slope_of(const Args &a, int head) { return MODE & kSlopes ? a.d_slopes[head] * kLog2e / unit_of<MODE>(a) : 0.0f; }
template <int MODE> HEDDLE_INLINE float modify(const Args &a, float s, int r, float slope, float distance)
{
    if constexpr (MODE & kCap) s = __builtin_amdgcn_rcpf(-1.0f - __builtin_amdgcn_exp2f(s * a.scale2));
    if constexpr (MODE & kSlopes) s = __builtin_fmaf(-slope, fabsf(distance - (float)(8 * (r >> 2) + (r & 3))), s);
    return s;
}

// ---- the forward pass's steps ----
// A lane's query row and what it sees: keys 0 .. limit - 1.
struct Row {
    int64_t at;                               // counted over all rows of q
    int32_t i, head, limit, pos;
    bool any;
};
__device__ inline Row row_of(const Args &a, const Sequence &q, int hk, int r)
{
    Row x;
    x.any = r < q.lq * a.group;
    x.i = r / a.group;
    x.head = hk * a.group + (r - x.i * a.group);
    x.at = (a.packed ? q.q0 : (int64_t)q.s * a.q_len) + x.i;
    x.pos = x.i + (q.lk - q.lq);
    x.limit = x.any ? max(min(q.lk, a.causal ? max(x.pos + 1, q.prefix) : q.lk), 0) : 0;
    return x;
}
__device__ inline int limit_of(const Args &a, const Sequence &q, int r)
{
    if (r >= q.lq * a.group) return 0;
    const int pos = r / a.group + (q.lk - q.lq);
    return __builtin_amdgcn_readfirstlane(max(min(q.lk, a.causal ? max(pos + 1, q.prefix) : q.lk), 0));
}

// The running state of 32 rows: m in modify()'s units.
template <int DP> struct State {
    f32x16 o[DP / 32];
    float m, l;
    bool far;                                 // (of forward_kernel)
    __device__ inline void init()
    {
        m = -INFINITY, l = 0, far = false;
#pragma unroll
        for (int d = 0; d < DP / 32; d++) o[d] = f32x16{};
    }
};

// a tile's 32 keys from row `from` on against the query rows
template <typename T, int DP> HEDDLE_INLINE f32x16 score(const char *tk, const Places &at, int from, const typename mm::pack8<T>::type *q)
{
    f32x16 s = {};
#pragma unroll
    for (int k = 0; k < DP / 16; k++) s = mfma(row_fragment<DP, T>(tk, at, from, k), q[k], s);
    return s;
}

// The maximum times the unit is what exponents start from. Its rounding is common to a row's probabilities, but from
// kFar on past 2^-4 of an exponent, and for scores near 2^28 past float16's range: there the maximum is taken off
// the scores first, exactly near it. far: whether it is so far for one of the wavefront's rows.
constexpr float kFar = 1 << 20;
template <int MODE> HEDDLE_INLINE bool is_far(float base)
{
    if constexpr (MODE == kCap) return false;               // (scores to 2 cap log2(e))
    return __any(fabsf(base) > kFar);
}

// Probabilities of 32 keys, key `first` the lane's register 0. The maximum follows only when it is 2^8 behind: p then
// stays below 2^8, and the sums are scaled again seldom; true: they have to be, from the maximum `was` on, before p is added.
template <typename T, int MODE, bool MASKED>
HEDDLE_INLINE bool soften(const Args &a, f32x16 &s, float &m, float &was, float &sum, int first, const Row &row, float slope, typename mm::pack8<T>::type p[2])
{
    each<16>([&](int r) { s[r] = modify<MODE>(a, s[r], r, slope, (float)(row.pos - first)); });
    if constexpr (MASKED) each<16>([&](int r) { s[r] = first + mfma_row(r, 0) >= row.limit ? -INFINITY : s[r]; });
    float top = s[0];
    each<15>([&](int r) { top = fmaxf(top, s[r + 1]); });
    top = max_halves(top);
    const float unit = unit_of<MODE>(a);
    const bool follow = __any((top - m) * unit > 8.0f);     // (NaN where both are -infinity)
    was = m;
    m = follow ? fmaxf(m, top) : m;
    here(m);
    float base = m == -INFINITY ? 0.0f : m * unit;
    if (is_far<MODE>(base)) {
        each<16>([&](int r) { s[r] -= m == -INFINITY ? 0.0f : m; });
        base = 0;
    }
    sum = 0;
    each<16>([&](int r) {
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], unit, -base));
        sum += s[r];
    });
    p[0] = pack<T>(s, 0), p[1] = pack<T>(s, 8);
    return follow;
}

template <int MODE, int DP> HEDDLE_INLINE void rescale(const Args &a, State<DP> &st, float was)
{
    const float f = st.m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((was - st.m) * unit_of<MODE>(a));
    st.l *= f;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int r = 0; r < 16; r++) st.o[d][r] *= f;
}

// adds the products of 32 probabilities with a tile's values from row `from` on
template <typename T, int DP> HEDDLE_INLINE void collect(State<DP> &st, const char *tv, const Places &at, int from, const typename mm::pack8<T>::type p[2])
{
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
        for (int d = 0; d < DP / 32; d++) st.o[d] = mfma(column_fragment<DP, T>(tv, at, from + 16 * k, d), p[k], st.o[d]);
}

// a lane's query row as the products' operand
template <typename T, int DP> HEDDLE_INLINE void load_query(const Args &a, const View &v, const Sequence &q, const Row &row, typename mm::pack8<T>::type *f)
{
    const int h = (threadIdx.x & 63) >> 5;
    const T *p = (const T *)v.p + q.s * v.seq + (q.q0 + row.i) * v.row + row.head * v.head;
#pragma unroll
    for (int k = 0; k < DP / 16; k++) f[k] = global_fragment<T>(p, k * 16 + 8 * h, a.dim, row.any);
}

// four neighbouring values of an output row
template <typename T> __device__ inline void store4(T *p, int col, int dim, int vec, float a, float b, float c, float d)
{
    const T v[4] = {(T)a, (T)b, (T)c, (T)d};
    if (vec) {
        if (col < dim) __builtin_memcpy(__builtin_assume_aligned(p + col, 8), v, 8);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (col + i < dim) p[col + i] = v[i];
}

// A row of 32 x 32 products, factor times the lane's sums: lane l and l + 32 hold fours of the row's values in turn; they
// exchange half of them, so that each has eight side by side.
template <typename T, int DP> HEDDLE_INLINE void store_row(T *p, const f32x16 *o, float factor, int dim, int vec)
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            unsigned w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const typename Pair<T>::type v = {(T)(o[d][4 * q + 2 * i] * factor), (T)(o[d][4 * q + 2 * i + 1] * factor)};
                w[i] = __builtin_bit_cast(unsigned, v);
            }
#ifdef __HIP_DEVICE_COMPILE__
            asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\tv_permlane32_swap_b32 %2, %3" : "+v"(w[0]), "+v"(w[2]), "+v"(w[1]), "+v"(w[3]));
#endif
            const int col = d * 32 + q * 8 + 8 * h;
            if (vec) {
                if (col < dim) __builtin_memcpy(__builtin_assume_aligned(p + col, 16), w, 16);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (col + i < dim) p[col + i] = __builtin_bit_cast(T, (uint16_t)(w[i >> 1] >> (i & 1) * 16));
            }
        }
}

Args base_args(const heddle_attention_desc *d);
int mode_of(const heddle_attention_desc *d);
int backward(const heddle_attention_desc *d, mm::Scratch &s, bool run, hipStream_t stream);
// the launches
// workgroups of `threads` that clear rows: 0 unless one of `bits` of the descriptor's `clear` is set
unsigned clearing(const heddle_attention_desc *d, int bits, bool keys, int threads);
int clear_all(const heddle_attention_desc *d, const Args &a, bool backward, hipStream_t stream);
void launch_forward(const heddle_attention_desc *d, Args a, int rows, int64_t blocks, hipStream_t stream);

// f(type, padded head width, mode) as constants
template <typename F> void with_kind(const heddle_attention_desc *d, F f)
{
    auto mode = [&](auto t, auto dp) {
        switch (mode_of(d)) {
        case kPlain: return f(t, dp, std::integral_constant<int, kPlain>());
        case kCap: return f(t, dp, std::integral_constant<int, kCap>());
        case kSlopes: return f(t, dp, std::integral_constant<int, kSlopes>());
        default: return f(t, dp, std::integral_constant<int, kCap | kSlopes>());
        }
    };
    auto wide = [&](auto t) { return d->dim <= 64 ? mode(t, std::integral_constant<int, 64>()) : mode(t, std::integral_constant<int, 128>()); };
    d->dtype == HEDDLE_T_BF16 ? wide((__bf16)0.0f) : wide((_Float16)0.0f);
}

// operands that do not lie on 16-byte boundaries are copied to scratch
struct Copy {
    const uint16_t *src;
    uint16_t *dst;
    int64_t seq, row, head, per, rows;        // per: rows of a sequence
    int32_t heads, dim, pad;                  // pad: the copies' head width
};
struct Copies {
    Copy one[5];
    int count = 0;
    void add(const heddle_attention_desc *d, View &v, bool keys, mm::Scratch &s);
    int launch(hipStream_t stream) const;
};

}  // namespace attn
}  // namespace heddle
