// Tiled matrix products on gfx950's matrix cores (16-bit operands, fp32 sums):
// C[i][j] = sum over k of A(i, k) B(j, k), with the operand's memory order as
// a template parameter, expert groups, a split reduction and a fused epilogue.
//
// Operands. An operand is "rows" (row i holds its k contiguous: X and W of a
// forward product) or "columns" (row k holds its i contiguous: W in dX = dZ W,
// both operands of dW = dZ^T X). Tiles of 64 k go from global memory straight
// to LDS, 16 bytes a lane, through a buffer resource whose size is the
// operand's remaining bytes: what lies past the end arrives as zero, so no
// address needs a test. Rows tiles are [row][64] with the 16-byte pieces of a
// row exchanged by 3 bits of the row; a lane reads its 8 k with one 16-byte read.
// Columns tiles are [64][column] with the 32-byte pieces exchanged by 3 bits of
// k; the transposing LDS read hands each lane 4 k of its column. Either way a
// quarter-wave's reads touch every bank once.
//
// Groups. With offsets, rows offsets[g] .. offsets[g+1] of the "row" dimension
// (kGroupRows) or of the reduction (kGroupSum) belong to group g. The offsets
// are device data: every workgroup finds its group by itself, clamps what it
// reads to the tensors, and a group without rows costs no product.
#pragma once

#include "heddle_internal.h"

namespace heddle {
namespace mm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct pack8;
template <> struct pack8<__bf16> { typedef bf16x8 type; };
template <> struct pack8<_Float16> { typedef f16x8 type; };

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

constexpr int kBK = 64;                       // k of a tile

// what the offsets split: rows of the output, or the reduction (one output per group)
enum Grouping { kGroupRows = 1, kGroupSum = 2 };

struct Args {
    const void *a, *b;
    int64_t lda, ldb;                         // elements between rows in memory, even, at most HEDDLE_MAX_LD:
                                              // 256 rows stay below 2^31 bytes
    int64_t stride_b;                         // elements from a group's B to the next one's
    int32_t M, N, K;                          // K: the reduction (kGroupSum: of all groups together)
    int32_t F;                                // gated: rows of B from a gate row to its up row (N = F)
    const int32_t *offsets;                   // device [groups + 1], or NULL
    int32_t groups;                           // 1 without offsets
    int32_t tiles_m, tiles_n;                 // (kGroupRows: an upper bound over all groups)
    int32_t splits, split_tiles;              // parts of the reduction and k-tiles of each
    float *partial;                           // [splits][M][columns()]: sums of each part (splits > 1)
};
// columns of a partial sum's row: whole eights; gated: the up columns after the gate ones
__host__ __device__ inline int64_t partial_cols(int n, bool gated) { return (int64_t)((n + 7) & ~7) * (gated ? 2 : 1); }

// ---- activations (fp32) ----
// the reciprocal of one instruction, off by 1 ulp: a division is ten, and the activations bound
// the pass that forms dZ (4096 x 10816, gelu_tanh: 79 us with a division, 75 without)
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
// The normal distribution's Phi(z); e: exp(-z^2 / 2). Phi(-t) = e P(1 / (1 + 0.3 t)) for t >= 0, the
// form of Hastings's approximations (1955), P fitted to the least relative error over t = 0 .. 14.5:
// 1.6e-7, in fp32 arithmetic (t^2 + 8) 2^-24. (1 + erf(z / sqrt 2) cancels for z < 0: 4% off at -5,
// and 0 below -5.5.)
__device__ inline float normal_cdf(float z, float &e)
{
    const float t = fabsf(z), w = __builtin_amdgcn_rcpf(1.0f + 0.3f * t);
    e = __expf(-0.5f * t * t);
    float p = 0.035423696f;
    p = p * w - 0.15615829f;
    p = p * w + 0.20455651f;
    p = p * w - 0.052033775f;
    p = p * w + 0.12769164f;
    p = p * w + 0.1001759842f;
    p = p * w + 0.12071213f;
    p = p * w + 0.119632006f;
    p *= w * e;
    return z > 0 ? 1.0f - p : p;
}
__device__ inline float act_of(int act, float z)
{
    switch (act) {
    case HEDDLE_A_RELU: return z > 0 ? z : (z != z ? z : 0.0f);
    case HEDDLE_A_SILU: return z * sigmoid(z);
    case HEDDLE_A_GELU: {
        float e;
        return z * normal_cdf(z, e);
    }
    case HEDDLE_A_GELU_TANH: {
        // 0.5 (1 + tanh u) = sigmoid(2 u)
        const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
        return z * sigmoid(2.0f * u);
    }
    default: return z;
    }
}
// Value and derivative of a kept z. The derivative is that at +-88 beyond, where it is 0 or 1 to
// fp32 but its factors leave the type's range; the value that at -88 below, where it is 0: a z below
// float16's range was kept as -infinity, and the forward pass had 0 there.
__device__ inline void act_both(int act, float z, float &v, float &d)
{
    const float y = z > 88.0f ? 88.0f : z < -88.0f ? -88.0f : z;
    switch (act) {
    case HEDDLE_A_RELU:
        v = z > 0 ? z : (z != z ? z : 0.0f);
        d = z > 0 ? 1.0f : (z != z ? z : 0.0f);
        break;
    case HEDDLE_A_SILU: {
        const float s = sigmoid(z);
        v = fmaxf(z, y) * s;
        d = s * (1.0f + y * (1.0f - s));
        break;
    }
    case HEDDLE_A_GELU: {
        float e;
        const float c = normal_cdf(z, e);
        v = fmaxf(z, y) * c;
        d = c + y * 0.39894228040143268f * e;
        break;
    }
    case HEDDLE_A_GELU_TANH: {
        const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
        const float s = sigmoid(2.0f * u);
        v = fmaxf(z, y) * s;
        d = s + 2.0f * y * s * (1.0f - s) * 0.79788456080286536f * (1.0f + 0.134145f * y * y);
        break;
    }
    default:
        v = z;
        d = 1.0f;
    }
}

// ---- eight neighbouring values of a row: one access of 16 bytes at any address that its
// values may have, single values at the row's end ----
template <typename T> __device__ inline void load8(const T *p, int count, float v[8])
{
    typename pack8<T>::type x;
    if (count >= 8) {
        __builtin_memcpy(&x, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = i < count ? p[i] : (T)0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)x[i];
}
// Past the caches: a kernel's outputs are many times what its L2 slices hold, and there they
// would take the operands' place (64 experts of 64 rows, 2 x 1632 columns of 4096: 399 us, 460
// with ordinary stores; the block's training step on 4096 rows of 4096 x 10816: 1% less).
template <typename T> __device__ inline void store8(T *p, int count, const float v[8])
{
    typedef short piece __attribute__((ext_vector_type(8), aligned(2)));
    typename pack8<T>::type x;
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = (T)v[i];
    if (count >= 8) {
        __builtin_nontemporal_store(__builtin_bit_cast(s16x8, x), (piece *)p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < count) p[i] = x[i];
    }
}

// ---- epilogues: one call finishes eight columns n .. n+7 of row m; unroll: of the loop of calls ----
// y = act(z + bias) + residual, z rounded once where it is kept for the
// backward pass (`pre`), the outputs once.
template <typename T> struct EpiLinear {
    static constexpr bool gated = false;
    static constexpr int unroll = 1;
    T *y, *pre;
    const T *bias, *residual;
    int64_t ldy, ldp, ldr;
    int32_t act, N;
    __device__ inline void operator()(int64_t m, int n, int g, float v[8]) const
    {
        const int count = N - n;
        if (bias) {
            float b[8];
            load8(bias + (int64_t)g * N + n, count, b);
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] += b[i];
        }
        if (pre) store8(pre + m * ldp + n, count, v);
        if (act) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act_of(act, v[i]);
        }
        if (residual) {
            float r[8];
            load8(residual + m * ldr + n, count, r);
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] += r[i];
        }
        store8(y + m * ldy + n, count, v);
    }
};

// A gradient: the sums, rounded once. Apart from EpiLinear, whose tests and registers show where
// little is summed for each output (64 experts of 64 rows, both weights' gradients: the training
// step 2.11 ms, 2.18 with it).
template <typename T> struct EpiPlain {
    static constexpr bool gated = false;
    static constexpr int unroll = 8;          // short enough for its LDS reads and stores to overlap
    T *y;
    int64_t ldy, stride_y;
    int32_t N;
    __device__ inline void operator()(int64_t m, int n, int g, const float v[8]) const
    {
        store8(y + (int64_t)g * stride_y + m * ldy + n, N - n, v);
    }
};

// h = act(gate) * up, with both kept for the backward pass where `pre` is given
template <typename T> struct EpiGated {
    static constexpr bool gated = true;
    static constexpr int unroll = 1;
    T *h, *pre;
    int64_t ldh, ldp;
    int32_t act, N;                           // N = F
    __device__ inline void operator()(int64_t m, int n, int, float gate[8], const float up[8]) const
    {
        const int count = N - n;
        if (pre) {
            store8(pre + m * ldp + n, count, gate);
            store8(pre + m * ldp + N + n, count, up);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) gate[i] = act_of(act, gate[i]) * up[i];
        store8(h + m * ldh + n, count, gate);
    }
};

// From dh (the product) and the kept gate and up values: the gradients of
// both, and h again for the output weights' gradient. dp and h are rounded to
// the operands' type here because the next products read them as operands.
template <typename T> struct EpiGatedGrad {
    static constexpr bool gated = false;
    static constexpr int unroll = 1;
    T *dp, *h;
    const T *pre;
    int64_t ldd, ldh, ldp;
    int32_t act, N;
    __device__ inline void operator()(int64_t m, int n, int, float v[8]) const
    {
        const int count = N - n;
        float g[8], u[8], dg[8], hh[8];
        load8(pre + m * ldp + n, count, g);
        load8(pre + m * ldp + N + n, count, u);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float a, d;
            act_both(act, g[i], a, d);
            dg[i] = v[i] * u[i] * d;
            hh[i] = a * u[i];
            v[i] *= a;
        }
        store8(dp + m * ldd + n, count, dg);
        store8(dp + m * ldd + N + n, count, v);
        store8(h + m * ldh + n, count, hh);
    }
};

// ---- groups ----
// Group g's rows are c[g] .. c[g + 1] - 1, c[i] the largest of offsets[0 .. i], inside 0 .. total:
// the offsets themselves where they are in order, and whatever they hold no row is in two groups,
// so that a grid sized for the rows and groups has a workgroup for every tile. Offsets in order,
// which a ballot shows, cost no scan. All lanes of a wavefront call these.

// the first 64 offsets, one a lane: a kernel asks for them before it knows its group
__device__ inline int first_offsets(const int32_t *offsets, int groups) { return offsets[min((int)(threadIdx.x & 63), groups)]; }

// rows of group g; head: first_offsets()
__device__ inline void group_range(const int32_t *offsets, int head, int g, int total, int &lo, int &hi)
{
    const int lane = threadIdx.x & 63;
    int before = lane < g ? head : 0, next;
    if (g < 63) {
        lo = __builtin_amdgcn_readlane(head, g);
        next = __builtin_amdgcn_readlane(head, g + 1);
    } else {
#pragma unroll 4
        for (int i = 64 + lane; i < g; i += 64) before = max(before, offsets[i]);
        lo = offsets[g];
        next = offsets[g + 1];
    }
    lo = min(max(lo, 0), total);
    if (__ballot(before > lo)) {
#pragma unroll
        for (int d = 32; d; d /= 2) before = max(before, __shfl_xor(before, d));
        lo = min(max(lo, __builtin_amdgcn_readfirstlane(before)), total);
    }
    hi = min(max(next, lo), total);
}

// rows of group g0 + lane, none past the last group; carry: c[g0]
__device__ inline void group_ranges(const int32_t *offsets, int groups, int total, int g0, int carry, int &lo, int &hi)
{
    const int lane = threadIdx.x & 63;
    const bool any = g0 + lane < groups;
    lo = hi = 0;
    if (any) {
        lo = min(max(offsets[g0 + lane], 0), total);
        hi = min(max(offsets[g0 + lane + 1], 0), total);
    }
    if (!__ballot(any && (lo < carry || hi < lo))) return;
    lo = max(lo, carry);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) lo = max(lo, __shfl_up(lo, d));   // (a lane without one d below has its own)
    hi = max(hi, lo);
}

// tiles of bm rows of all groups together
__device__ inline int count_tiles(const int32_t *offsets, int groups, int total, int bm)
{
    int sum = 0, carry = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
        int lo, hi;
        group_ranges(offsets, groups, total, g0, carry, lo, hi);
        sum += (hi - lo + bm - 1) / bm;
        carry = __builtin_amdgcn_readlane(hi, 63);
    }
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    return __builtin_amdgcn_readfirstlane(sum);
}

// the group and first row of tile t of BM rows; false past the last tile
__device__ inline bool find_tile(const int32_t *offsets, int groups, int total, int bm, int t, int &g, int &row, int &end)
{
    const int lane = threadIdx.x & 63;
    int before = 0, carry = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
        int lo, hi;
        group_ranges(offsets, groups, total, g0, carry, lo, hi);
        const int mine = (hi - lo + bm - 1) / bm;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        const uint64_t past = __ballot(before + sum > t);
        if (past) {
            const int l = __builtin_ctzll(past);
            g = g0 + l;
            const int first = before + __shfl(sum - mine, l);
            row = __shfl(lo, l) + (t - first) * bm;
            end = __shfl(hi, l);
            g = __builtin_amdgcn_readfirstlane(g);
            row = __builtin_amdgcn_readfirstlane(row);
            end = __builtin_amdgcn_readfirstlane(end);
            return true;
        }
        before += __shfl(sum, 63);
        carry = __builtin_amdgcn_readlane(hi, 63);
    }
    return false;
}

// ---- tile loads ----
typedef int i32x4 __attribute__((ext_vector_type(4)));

// What is left of an operand from a tile's first value on: a raw buffer in whole 4-byte
// words (the word of the last value never crosses a page); what lies past it reads as zero.
// Kept as a pointer and a 64-bit count, advanced by whole tiles in scalar arithmetic.
struct Rest {
    const char *p;
    int64_t bytes;
    __device__ inline void set(const char *base, int64_t n)
    {
        p = base;
        bytes = n <= 0 ? 0 : (n + 3) & ~int64_t(3);
    }
    __device__ inline i32x4 buffer() const
    {
        const int high = (int)(bytes >> 32), low = (int)bytes;
        return i32x4{(int)(uintptr_t)p, (int)((uintptr_t)p >> 32), high > 0 ? -4 : high < 0 ? 0 : low, 0x00020000};
    }
    __device__ inline void advance(int64_t step) { p += step, bytes -= step; }
};

// 16 bytes a lane from the buffer to LDS, at lds + 16 lane; two of them. Written out, because
// after the builtin the compiler waits for the load before the next transposing LDS read,
// whichever buffer that reads; arrive() has the wait. No register receives anything. The
// no-ops cover the wait states after a write of m0, and after one of the buffer's registers by
// a vector instruction.
__device__ inline void load_to_lds(i32x4 buffer, int offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 : : "s"(lds), "v"(offset), "s"(buffer) : "memory", "m0");
}
__device__ inline void load_to_lds(i32x4 buffer, int offset0, uint32_t lds0, int offset1, uint32_t lds1)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\t"
                 "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds"
                 : : "s"(lds0), "s"(lds1), "v"(offset0), "v"(offset1), "s"(buffer) : "memory", "m0");
}

// the exchange of a rows tile's 16-byte and of a columns tile's 32-byte pieces
__device__ inline int row_swz(int r) { return (r >> 1) & 7; }
template <int ROWS> __device__ inline int col_swz(int k) { return ((k & 3) | ((k >> 3 & 1) << 2)) & (ROWS / 16 - 1); }

// One operand's tile of ROWS x 64, loaded by NW wavefronts. COLS: the operand
// is "columns". PAIR: 16-row blocks alternate between gate and up rows.
template <int ROWS, int NW, bool COLS, bool PAIR> struct Loader {
    static constexpr int kLoads = ROWS * 8 / (NW * 64);   // 16-byte pieces of a lane
    static constexpr int kBytes = ROWS * kBK * 2;
    int voff[kLoads];
    __device__ inline void init(int64_t ld, int wave)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int c = (i * NW + wave) * 64 + lane;
            if (COLS) {
                const int k = c / (ROWS / 8), pos = c % (ROWS / 8);
                voff[i] = (int)(k * ld * 2) + (pos ^ (col_swz<ROWS>(k) << 1)) * 16;
            } else {
                const int r = c / 8, pos = c % 8;
                const int src = PAIR ? (r / 32) * 16 + r % 16 : r;
                voff[i] = (int)(src * ld * 2) + (pos ^ row_swz(r)) * 16;
            }
        }
    }
    // a wavefront's 8 rows lie in one 16-row block, every kLoads piece in one of the same kind
    static __device__ inline bool takes_up(int wave) { return PAIR && (wave / 2) % 2; }
    // piece i of the tile: 1024 bytes a wavefront, 8 rows of a rows tile
    __device__ inline void load(int i, i32x4 buffer, uint32_t lds, int wave) const
    {
        load_to_lds(buffer, voff[i], lds + (i * NW + wave) * 1024);
    }
    __device__ inline void load_all(i32x4 buffer, uint32_t lds, int wave) const
    {
        static_assert(kLoads % 2 == 0 && NW % 4 == 0, "pieces in pairs");
#pragma unroll
        for (int i = 0; i < kLoads; i += 2)
            load_to_lds(buffer, voff[i], lds + (i * NW + wave) * 1024, voff[i + 1], lds + ((i + 1) * NW + wave) * 1024);
    }
    // a rows tile's values with k >= valid hold the next row's: make them zero
    __device__ static inline void clear_tail(char *lds, int valid)
    {
        for (int c = threadIdx.x; c < ROWS * kBK; c += NW * 64) {
            const int r = c / kBK, k = c % kBK;
            if (k >= valid) *(short *)(lds + r * 128 + (((k / 8) ^ row_swz(r)) * 16) + (k % 8) * 2) = 0;
        }
    }
};

// fragment of 16 rows (block `rb` of the tile), k-step s, for one lane
template <int ROWS, bool COLS, typename T>
__device__ inline typename pack8<T>::type fragment(const char *lds, int rb, int s)
{
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    if (COLS) {
        const int q = i >> 2, f = col_swz<ROWS>(g * 8 + q);
        const char *p = lds + (s * 32 + g * 8 + q) * (ROWS * 2) + ((rb ^ f) << 5) + (i & 3) * 8;
        typedef __attribute__((address_space(3))) s16x4 *rd;
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((rd)p);
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((rd)(p + 4 * ROWS * 2));
        const s16x8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(typename pack8<T>::type, z);
    }
    return *(const typename pack8<T>::type *)(lds + (rb * 16 + i) * 128 + (((s * 4 + g) ^ row_swz(i)) << 4));
}

// every wavefront's loads to LDS have landed and its reads of LDS are done
__device__ inline void arrive()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// the same, but for each wavefront's `later` newest loads
template <int later> __device__ inline void arrive_but()
{
    static_assert(later < 64, "vmcnt");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((later & 15) | 7 << 4 | (later >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// the order of a half step's instructions: one LDS read to every other product, so that the
// reads of the next fragments run beside the products of these
template <int READS, int PRODUCTS, bool COLS> __device__ inline void interleave()
{
#pragma unroll
    for (int i = 0; i < READS; i++) {
        __builtin_amdgcn_sched_group_barrier(0x100, COLS ? 2 : 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS / READS, 0);
    }
}

// Workgroup order: consecutive workgroups go to the 8 XCDs in turn, so each
// XCD is given a contiguous range of tiles, walked 8 row-tiles wide, and its
// L2 holds the operands that neighbouring tiles share.
__device__ inline int xcd_order(int id, int total)
{
    const int per = total / 8, extra = total % 8, x = id % 8;
    return x * per + min(x, extra) + id / 8;
}
__device__ inline void tile_of(int t, int tiles_m, int tiles_n, int &tm, int &tn)
{
    constexpr int kWide = 8;
    const int band = t / (kWide * tiles_n), first = band * kWide, width = min(kWide, tiles_m - first);
    const int in = t - band * kWide * tiles_n;
    tm = first + in % width;
    tn = in / width;
}

template <int BM, int BN, int WM, int WN, int STAGES, bool ACOL, bool BCOL, Grouping GR, typename T, typename Epi>
__global__ void __launch_bounds__(WM * WN * 64) gemm_kernel(Args x, Epi epi)
{
#ifdef __HIP_DEVICE_COMPILE__   // the host pass knows no LDS loads
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, kOut = BN / WN;
    constexpr bool PAIR = Epi::gated, PIPED = STAGES == 2 && BM * BN >= 256 * 256;   // one workgroup on a CU
    typedef Loader<BM, NW, ACOL, false> LA;
    typedef Loader<BN, NW, BCOL, PAIR> LB;
    constexpr int kStage = LA::kBytes + LB::kBytes;
    static_assert(TM % 4 == 0 && (!PAIR || TN % 2 == 0), "a wavefront's part");
    constexpr int kFit = STAGES * kStage / (NW * kOut * 4), kRows = kFit >= 64 ? 64 : kFit >= 32 ? 32 : 16;   // of the epilogue at a time
    static_assert(NW * kRows * kOut * 4 <= STAGES * kStage, "the epilogue's part of LDS");
    __shared__ __align__(1024) char smem[STAGES * kStage];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const bool grouped_sum = GR == kGroupSum && x.offsets;
    const int head = grouped_sum ? first_offsets(x.offsets, x.groups) : 0;
    // The grid of grouped rows holds the most tiles that the groups may have. Those that they do
    // have are shared out among the XCDs (shared out by the grid, the last XCDs had none).
    int tiles_m = x.tiles_m, ids = gridDim.x;
    if (GR == kGroupRows && x.offsets) {
        tiles_m = count_tiles(x.offsets, x.groups, x.M, BM);
        ids = tiles_m * x.tiles_n;
        if ((int)blockIdx.x >= ids) return;
    }
    const int per = tiles_m * x.tiles_n;
    int t = xcd_order(blockIdx.x, ids);
    const int outer = t / per;                              // split, or group of kGroupSum
    t -= outer * per;
    int tm, tn;
    tile_of(t, tiles_m, x.tiles_n, tm, tn);

    int g = 0, m0 = tm * BM, m_end = x.M, k_lo = 0, k_hi = x.K;
    if (GR == kGroupRows && x.offsets && !find_tile(x.offsets, x.groups, x.M, BM, tm, g, m0, m_end)) return;
    if (grouped_sum) {
        g = __builtin_amdgcn_readfirstlane(outer);
        group_range(x.offsets, head, g, x.K, k_lo, k_hi);
    }
    const int split = grouped_sum ? 0 : outer;              // a grouped product is not split
    const int k_first = k_lo + split * x.split_tiles * kBK;
    const int k_last = grouped_sum ? k_hi : min(k_hi, k_first + x.split_tiles * kBK);
    const int tiles = k_last > k_first ? (k_last - k_first + kBK - 1) / kBK : 0;
    const int n0 = PAIR ? tn * (BN / 2) : tn * BN;          // PAIR: first gate row

    // the tiles' first values, and the bytes from there to the operand's end
    const int64_t eb = 2;
    const char *pa = (const char *)x.a, *pb = (const char *)x.b + (GR == kGroupRows ? g * x.stride_b * eb : 0);
    int64_t na, nb;
    if (ACOL) {
        pa += ((int64_t)k_first * x.lda + m0) * eb;
        na = ((int64_t)(k_hi - k_first - 1) * x.lda + (x.M - m0)) * eb;
    } else {
        pa += ((int64_t)m0 * x.lda + k_first) * eb;
        na = ((int64_t)(m_end - m0 - 1) * x.lda + (k_hi - k_first)) * eb;
    }
    const int brows = PAIR ? x.F + x.N : x.N;
    if (BCOL) {
        pb += ((int64_t)k_first * x.ldb + n0) * eb;
        nb = ((int64_t)(k_hi - k_first - 1) * x.ldb + (x.N - n0)) * eb;
    } else {
        pb += ((int64_t)n0 * x.ldb + k_first) * eb;
        nb = ((int64_t)(brows - n0 - 1) * x.ldb + (k_hi - k_first)) * eb;
    }
    const int64_t step_a = (ACOL ? x.lda * kBK : kBK) * eb, step_b = (BCOL ? x.ldb * kBK : kBK) * eb;
    // a wavefront loads either gate or up rows
    const int64_t up = LB::takes_up(wave) ? (int64_t)x.F * x.ldb * eb : 0;
    Rest rest_a, rest_b;
    rest_a.set(pa, na);
    rest_b.set(pb + up, nb - up);

    LA la;
    LB lb;
    la.init(x.lda, wave);
    lb.init(x.ldb, wave);
    const int wm = wave / WN, wn = wave % WN;

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = f32x4{0, 0, 0, 0};

    typedef typename pack8<T>::type frag;
    frag fa[2][TM], fb[2][TN];
    auto read = [&](const char *tile, int s, frag *a, frag *b) {
#pragma unroll
        for (int j = 0; j < TN; j++) b[j] = fragment<BN, BCOL, T>(tile + LA::kBytes, wn * TN + j, s);
#pragma unroll
        for (int i = 0; i < TM; i++) a[i] = fragment<BM, ACOL, T>(tile, wm * TM + i, s);
    };
    auto multiply = [&](const frag *a, const frag *b) {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) acc[i][j] = mfma(b[j], a[i], acc[i][j]);
    };
    constexpr int kLoads = LA::kLoads + LB::kLoads;
    int asked = 0;                                          // k-tiles asked for
    auto load = [&](uint32_t tile) {
        if (asked++ >= tiles) return;
        la.load_all(rest_a.buffer(), tile, wave);
        lb.load_all(rest_b.buffer(), tile + LA::kBytes, wave);
        rest_a.advance(step_a);
        rest_b.advance(step_b);
    };
    // the same, where a wait counts loads: past the last tile from empty buffers
    auto load_counted = [&](uint32_t tile) {
        const bool any = asked++ < tiles;
        i32x4 ra = rest_a.buffer(), rb = rest_b.buffer();
        ra[2] = any ? ra[2] : 0, rb[2] = any ? rb[2] : 0;
        la.load_all(ra, tile, wave);
        lb.load_all(rb, tile + LA::kBytes, wave);
        rest_a.advance(step_a);
        rest_b.advance(step_b);
    };
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    const int valid = (k_last - k_first) % kBK;             // k of a last, partial tile
    auto landed = [&](char *tile, int kt) {
        if constexpr (STAGES > 2) arrive_but<(STAGES - 2) * kLoads>();
        else arrive();
        if ((!ACOL || !BCOL) && valid && kt == tiles - 1 && k_last == k_hi) {
            if (!ACOL) LA::clear_tail(tile, valid);
            if (!BCOL) LB::clear_tail(tile + LA::kBytes, valid);
            __syncthreads();
        }
    };
    if (PIPED && tiles) {
        // Half a k-tile's fragments are read while the other half's are multiplied. A tile's
        // buffer is free, and the next tile must be there, at the middle of the tile. The loads
        // of the one after it go out at once where the wait for them shows (a rows operand:
        // 1225 against 1200 TFLOP/s at 2048 x 8192 x 24032), else between the products of the
        // second half (columns of both: 1335 against 1432).
        load(lds);
        landed(smem, 0);
        load(lds + kStage);
        read(smem, 0, fa[0], fb[0]);
        for (int kt = 0; kt < tiles; kt++) {
            char *cur = smem + (kt & 1) * kStage, *nxt = smem + (~kt & 1) * kStage;
            read(cur, 1, fa[1], fb[1]);
            multiply(fa[0], fb[0]);
            interleave<TM + TN, TM * TN, ACOL || BCOL>();
            landed(nxt, kt + 1);
            if constexpr (!ACOL) {
                load(lds + (kt & 1) * kStage);
                read(nxt, 0, fa[0], fb[0]);
                multiply(fa[1], fb[1]);
                interleave<TM + TN, TM * TN, ACOL || BCOL>();
            } else {
                const bool any = asked++ < tiles;           // past the last tile: empty buffers
                i32x4 ra = rest_a.buffer(), rb = rest_b.buffer();
                ra[2] = any ? ra[2] : 0, rb[2] = any ? rb[2] : 0;
                rest_a.advance(step_a);
                rest_b.advance(step_b);
#pragma unroll
                for (int i = 0; i < kLoads; i++) {
                    if (i < LA::kLoads) la.load(i, ra, lds + (kt & 1) * kStage, wave);
                    else lb.load(i - LA::kLoads, rb, lds + (kt & 1) * kStage + LA::kBytes, wave);
#pragma unroll
                    for (int f = i * (TM + TN) / kLoads; f < (i + 1) * (TM + TN) / kLoads; f++) {
                        if (f < TN) fb[0][f] = fragment<BN, BCOL, T>(nxt + LA::kBytes, wn * TN + f, 0);
                        else fa[0][f - TN] = fragment<BM, ACOL, T>(nxt, wm * TM + f - TN, 0);
                    }
#pragma unroll
                    for (int q = i * TM * TN / kLoads; q < (i + 1) * TM * TN / kLoads; q++)
                        acc[q / TN][q % TN] = mfma(fb[1][q % TN], fa[1][q / TN], acc[q / TN][q % TN]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    } else if (STAGES == 1 && tiles) {
        for (int kt = 0; kt < tiles; kt++) {
            if (kt) __syncthreads();
            load(lds);
            landed(smem, kt);
#pragma unroll
            for (int s = 0; s < kBK / 32; s++) {
                read(smem, s, fa[0], fb[0]);
                multiply(fa[0], fb[0]);
            }
        }
    } else if (STAGES > 2 && tiles) {
        // STAGES - 1 tiles on their way; the wait is for the oldest one's loads
#pragma unroll
        for (int i = 0; i < STAGES - 1; i++) load_counted(lds + i * kStage);
        for (int kt = 0, at = 0; kt < tiles; kt++) {
            char *cur = smem + at * kStage;
            landed(cur, kt);
            load_counted(lds + (at ? at - 1 : STAGES - 1) * kStage);
            at = at + 1 == STAGES ? 0 : at + 1;
#pragma unroll
            for (int s = 0; s < kBK / 32; s++) {
                read(cur, s, fa[0], fb[0]);
                multiply(fa[0], fb[0]);
            }
        }
    } else if (tiles) {
        // several workgroups on a CU hide each other's reads
        load(lds);
        for (int kt = 0; kt < tiles; kt++) {
            char *cur = smem + (kt & 1) * kStage;
            landed(cur, kt);
            load(lds + (~kt & 1) * kStage);
#pragma unroll
            for (int s = 0; s < kBK / 32; s++) {
                read(cur, s, fa[0], fb[0]);
                multiply(fa[0], fb[0]);
            }
        }
    }
    arrive();                                               // also the loads of empty buffers

    // Epilogue: a wavefront takes kRows of its rows at a time through its own part
    // of LDS, so that a lane finishes eight neighbouring columns. The product
    // was formed transposed: a lane holds row lane % 16, columns 4 (lane / 16)
    // .. + 3 of a block. 16-byte pieces of a row are exchanged by row & (pieces - 1).
    constexpr int kPieces = kOut / 4;
    float *own = (float *)smem + wave * kRows * kOut;
    const int nw = n0 + (PAIR ? wn * kOut / 2 : wn * kOut);
#pragma unroll
    for (int h = 0; h < TM * 16 / kRows; h++) {
#pragma unroll
        for (int i = 0; i < kRows / 16; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) {
                const int r = i * 16 + (lane & 15), p = j * 4 + (lane >> 4);
                *(f32x4 *)(own + r * kOut + ((p ^ (r & (kPieces - 1))) << 2)) = acc[h * (kRows / 16) + i][j];
            }
        __builtin_amdgcn_wave_barrier();
        constexpr int kUnits = (PAIR ? kOut / 2 : kOut) / 8;    // eights of a row
#pragma unroll Epi::unroll
        for (int c = lane; c < kRows * kUnits; c += 64) {
            const int r = c / kUnits, q = c % kUnits;
            const int m = m0 + wm * (TM * 16) + h * kRows + r;
            const int n = nw + q * 8;
            auto piece = [&](int p) { return *(const f32x4 *)(own + r * kOut + ((p ^ (r & (kPieces - 1))) << 2)); };
            // PAIR: gate columns 16 b .. + 15 are pieces 8 b .. + 3, the up columns the four after
            const int p0 = PAIR ? (q / 2) * 8 + (q % 2) * 2 : q * 2;
            const f32x4 v0 = piece(p0), v1 = piece(p0 + 1);
            float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            if (m >= m_end || n >= x.N) continue;
            if constexpr (PAIR) {
                const f32x4 u0 = piece(p0 + 4), u1 = piece(p0 + 5);
                float u[8] = {u0[0], u0[1], u0[2], u0[3], u1[0], u1[1], u1[2], u1[3]};
                if (x.splits > 1) {
                    float *to = x.partial + ((int64_t)split * x.M + m) * partial_cols(x.N, true) + n;
                    float *tu = to + partial_cols(x.N, false);
                    *(f32x4 *)to = v0, *(f32x4 *)(to + 4) = v1, *(f32x4 *)tu = u0, *(f32x4 *)(tu + 4) = u1;
                } else {
                    epi(m, n, g, v, u);
                }
            } else {
                if (x.splits > 1) {
                    float *to = x.partial + ((int64_t)split * x.M + m) * partial_cols(x.N, false) + n;
                    *(f32x4 *)to = v0, *(f32x4 *)(to + 4) = v1;
                } else {
                    epi(m, n, g, v);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
#endif
}

// Joins the parts of a split reduction, in their order, and finishes them.
template <typename Epi> __global__ void __launch_bounds__(256) join_kernel(Args x, Epi epi)
{
    const int eights = (x.N + 7) / 8;
    const int64_t total = (int64_t)x.M * eights, cols = partial_cols(x.N, Epi::gated);
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < total; c += (int64_t)gridDim.x * 256) {
        const int m = (int)(c / eights), n = (int)(c - (int64_t)m * eights) * 8;
        f32x4 v0 = {0, 0, 0, 0}, v1 = v0, u0 = v0, u1 = v0;
        for (int s = 0; s < x.splits; s++) {
            const float *from = x.partial + ((int64_t)s * x.M + m) * cols + n;
            v0 += *(const f32x4 *)from, v1 += *(const f32x4 *)(from + 4);
            if (Epi::gated) from += cols / 2, u0 += *(const f32x4 *)from, u1 += *(const f32x4 *)(from + 4);
        }
        float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
        if constexpr (Epi::gated) {
            float u[8] = {u0[0], u0[1], u0[2], u0[3], u1[0], u1[1], u1[2], u1[3]};
            epi(m, n, 0, v, u);
        } else {
            epi(m, n, 0, v);
        }
    }
}

// ---- host side ----
// A tile shape and the parts of the reduction.
struct Shape { int cfg, splits, split_tiles; };
enum Order { kRowsRows = 0, kRowsCols = 1, kColsCols = 2 };   // of the operands in memory
Shape shape_of(int64_t M, int64_t N, int64_t K, int groups, bool gated, Order order);   // groups: 0 without offsets
bool third_buffer(int64_t M, int64_t N, int groups, bool gated, bool sums, int splits);       // of 64 x 128 tiles
inline size_t partial_bytes(const Shape &s, int64_t M, int64_t N, bool gated)
{
    return s.splits > 1 ? (size_t)s.splits * M * partial_cols((int)N, gated) * 4 : 0;
}

template <int BM, int BN, int WM, int WN, int STAGES, bool ACOL, bool BCOL, Grouping GR, typename T, typename Epi>
inline int launch_cfg(Args x, const Shape &s, const Epi &epi, hipStream_t stream)
{
    const int64_t cols = Epi::gated ? 2 * (int64_t)x.N : x.N;
    const bool grouped = x.offsets != nullptr;
    x.tiles_m = (int)((x.M + BM - 1) / BM) + (GR == kGroupRows && grouped ? x.groups : 0);
    x.tiles_n = (int)((cols + BN - 1) / BN);
    x.splits = s.splits;
    x.split_tiles = s.split_tiles;
    const int64_t blocks = (int64_t)x.tiles_m * x.tiles_n * (GR == kGroupSum && grouped ? x.groups : s.splits);
    if (blocks > 0xFFFFFFFF / (WM * WN * 64)) return fail(HEDDLE_E_RANGE, "more tiles than a launch holds");   // below 2^32 lanes
    hipLaunchKernelGGL((gemm_kernel<BM, BN, WM, WN, STAGES, ACOL, BCOL, GR, T, Epi>), dim3((unsigned)blocks), dim3(WM * WN * 64), 0,
                       stream, x, epi);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "gemm_kernel");
    if (s.splits > 1) {
        const int64_t want = ((int64_t)x.M * ((x.N + 7) / 8) + 255) / 256;
        hipLaunchKernelGGL((join_kernel<Epi>), dim3((unsigned)(want < 4096 ? want : 4096)), dim3(256), 0, stream, x, epi);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "join_kernel");
    }
    return HEDDLE_OK;
}

template <bool ACOL, bool BCOL, Grouping GR, typename T, typename Epi>
inline int launch_gemm(const Args &x, const Shape &s, const Epi &epi, hipStream_t stream)
{
    switch (s.cfg) {
    case 0: return launch_cfg<256, 256, 2, 4, 2, ACOL, BCOL, GR, T>(x, s, epi, stream);
    case 1: return launch_cfg<128, 128, 2, 2, 1, ACOL, BCOL, GR, T>(x, s, epi, stream);
    case 2:
        if (third_buffer(x.M, x.N, x.offsets ? x.groups : 0, Epi::gated, GR == kGroupSum, s.splits))
            return launch_cfg<64, 128, 1, 4, 3, ACOL, BCOL, GR, T>(x, s, epi, stream);
        return launch_cfg<64, 128, 1, 4, 2, ACOL, BCOL, GR, T>(x, s, epi, stream);
    default:   // groups of few rows only
        if constexpr (GR == kGroupRows) return launch_cfg<64, 256, 1, 4, 2, ACOL, BCOL, GR, T>(x, s, epi, stream);
        else return fail(HEDDLE_E_INVAL, "no such tile");
    }
}

}  // namespace mm
}  // namespace heddle
