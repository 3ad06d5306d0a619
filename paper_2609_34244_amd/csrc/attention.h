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
// Tiles lie in LDS as [row][DP] of 16-bit values, DP = 64 or 128, the 16-byte pieces of a row
// exchanged by 4 bits of the row (3 and its parity for DP = 64): 16 lanes that read the same
// piece of 16 rows, and 32 lanes of a transposing read (4 rows, 64 bytes), touch every bank once.
// They are filled straight from global memory through a buffer resource; rows past a sequence's
// end and columns past the head's width arrive as zeros.
#pragma once

#include "linear.h"

namespace heddle {
namespace attn {

using mm::i32x4;
using mm::s16x4;
using mm::s16x8;
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ inline f32x16 mfma(mm::bf16x8 a, mm::bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma(mm::f16x8 a, mm::f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

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
    float *partial;                           // few queries: [parts][slot rows][DP + 2]
    int64_t q_rows, k_rows;                   // of all sequences (batched: sequences * length)
    int32_t sequences, q_len, k_len, packed;
    int32_t heads, kv_heads, group, dim;
    int32_t causal, parts;
    int32_t q_vec, out_vec, grads;            // 16-byte rows of q, k, v (dy); 8-byte rows of outputs; which gradients
    float scale, scale2, cap, cap2;           // scale2 = scale log2(e); with a cap: 2 scale log2(e) / cap and cap log2(e)
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
        s = (int)(slot / tiles);
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
inline int64_t slots_of(int packed, int64_t sequences, int64_t rows, int64_t length, int64_t mul, int64_t T)
{
    return packed ? rows * mul / T + sequences : sequences * ((length * mul + T - 1) / T);
}

// ---- tiles in LDS ----
template <int DP> __device__ inline int swz(int row)
{
    return DP == 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
}

constexpr int kNowhere = -16;                 // past any buffer's end: arrives as zeros

// ROWS x DP values by NW wavefronts, 1 KB of LDS an instruction
template <int DP, int ROWS, int NW> struct Tile {
    static constexpr int kRowBytes = DP * 2, kBytes = ROWS * kRowBytes, kPer = 1024 / kRowBytes;   // rows of an instruction
    static constexpr int kLoads = ROWS / (kPer * NW);
    static_assert(kLoads * kPer * NW == ROWS, "whole instructions");
    // byte offset of a lane's piece of instruction i, from the tile's first row; valid: rows that the sequence has from there
    static __device__ inline int offset(int i, int wave, int64_t ld, int dim, int valid)
    {
        const int lane = threadIdx.x & 63, row = (i * NW + wave) * kPer + lane / (DP / 8);
        const int col = ((lane % (DP / 8)) ^ swz<DP>(row)) * 8;
        return row < valid && col < dim ? (int)(row * ld * 2) + col * 2 : kNowhere;
    }
};

// a buffer from p on; every offset that is used lies in the tensor, or is kNowhere
__device__ inline i32x4 buffer_at(const void *p)
{
    const uint64_t v = (uint64_t)p;
    return i32x4{__builtin_amdgcn_readfirstlane((int)v), __builtin_amdgcn_readfirstlane((int)(v >> 32) & 0xffff), 0x7fffffff, 0x00020000};
}

// 16 bytes of columns 16 step + 8 h of row `row`
template <int DP, typename T> __device__ inline typename mm::pack8<T>::type row_fragment(const char *tile, int row, int step, int h)
{
    return *(const typename mm::pack8<T>::type *)(tile + row * (DP * 2) + (((step * 2 + h) ^ swz<DP>(row)) << 4));
}

// Column 32 dt + lane % 32 of rows base + 4 h + 0..3 and base + 8 + 4 h + 0..3; base a multiple of 16.
template <int DP, typename T> __device__ inline typename mm::pack8<T>::type column_fragment(const char *tile, int base, int dt)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int lane = threadIdx.x & 63, i = lane & 15, h = lane >> 5;
    const int row = base + 4 * h + (i >> 2), piece = dt * 4 + (lane >> 4 & 1) * 2 + (i >> 1 & 1);
    typedef __attribute__((address_space(3))) s16x4 *rd;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((rd)(tile + row * (DP * 2) + ((piece ^ swz<DP>(row)) << 4) + (i & 1) * 8));
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((rd)(tile + (row + 8) * (DP * 2) + ((piece ^ swz<DP>(row + 8)) << 4) + (i & 1) * 8));
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

// eight probabilities as the next product's operand
template <typename T> __device__ inline typename mm::pack8<T>::type pack(const f32x16 &p, int from)
{
    typename mm::pack8<T>::type x;
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = (T)p[from + i];
    return x;
}

// row of a 32 x 32 product's register r
__device__ inline int mfma_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

__device__ inline float other_half(float v) { return __shfl_xor(v, 32); }

// tanh(u / 2) for u log2(e) = z: 1 - 2 / (1 + e^u); the ends are exact
__device__ inline float tanh_half(float z) { return 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z)); }

// Scores times log2(e), capped and biased; pos: the row's place among the keys, j: the key of register 0.
// MOD: a cap or slopes. t receives the tanh where a cap is given.
template <bool MOD> __device__ inline void modify(const Args &a, f32x16 &s, float slope2, int distance, f32x16 *t)
{
    if constexpr (!MOD) {
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] *= a.scale2;
        return;
    }
    if (a.cap > 0) {
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const float u = tanh_half(s[r] * a.scale2);
            if (t) (*t)[r] = u;
            s[r] = a.cap2 * u;
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] *= a.scale2;
    }
    if (a.d_slopes) {
        const float at = (float)distance;
#pragma unroll
        for (int r = 0; r < 16; r++) s[r] -= slope2 * fabsf(at - (float)(8 * (r >> 2) + (r & 3)));
    }
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

int check(const heddle_attention_desc *d, bool backward);
int check_overlaps(const heddle_attention_desc *d, bool backward);
Args base_args(const heddle_attention_desc *d);
bool modified(const heddle_attention_desc *d);

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
