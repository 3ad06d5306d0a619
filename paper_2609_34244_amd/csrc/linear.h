// Internal host side of the feed-forward operators: operands as the products
// want them, scratch layout, and the launches the entry points are made of.
#pragma once

#include <initializer_list>

#include "gemm.h"
#include "skinny.h"

namespace heddle {
namespace mm {

constexpr int64_t kMaxRows = HEDDLE_MAX_ROWS;   // sums of a row and a few tiles or chunks stay 32-bit

// Distance between rows of a scratch matrix: whole 128-byte lines, an odd number of them, so
// that the 128 bytes a tile reads of a row are one line and neighbouring rows lie in
// different memory channels (2048 x 8192 x 24576: 1327 TFLOP/s from a distance of 384 lines,
// 1453 from 386).
inline int64_t scratch_ld(int64_t n) { return (((n + 63) / 64) | 1) * 64; }

// Caller's scratch, handed out in 256-byte steps. With base NULL it only measures.
struct Scratch {
    char *base;
    size_t used;
    void *take(size_t bytes)
    {
        void *p = base ? base + used : nullptr;
        used += (bytes + 255) & ~size_t(255);
        return p;
    }
};

// An operand of a product: rows of ld elements, groups stride apart.
struct Operand { const void *p; int64_t ld, stride; };

// Rows that do not start on 4-byte boundaries are copied to scratch, in
// rows of whole 16 bytes: one pass over the operand at memory speed, against
// products whose loads would otherwise be single values.
inline bool needs_copy(const Operand &o, int groups)
{
    return ((uintptr_t)o.p & 3) || (o.ld & 1) || (groups > 1 && (o.stride & 1));
}
class Copies {
public:
    // takes scratch for the copy of o, if it needs one, and lets o name it
    void add(Operand &o, int64_t rows, int64_t cols, int groups, Scratch &s);
    int launch(hipStream_t stream) const;     // one launch for all that were added
    static constexpr int kMost = 4;
    struct One {
        const uint16_t *src;
        uint16_t *dst;
        int64_t ld, stride, rows, cols, ldd, first;   // first: its first eight of the launch
    } one[kMost];
    int count = 0;
    int64_t eights = 0;
};

// dZ = dY act'(Z) (written where dz is given) and its column sums per group
struct BiasGrad {
    const void *dy, *pre;
    int64_t lddy, ldp, lddz;
    void *dz, *db;
    const int32_t *offsets;
    int32_t groups, act, m, n;
    int32_t chunks, chunk_rows;               // parts of the rows (1 with offsets)
    float *partial;                           // [chunks][n] (chunks > 1)
};
int64_t bias_grad_bytes(int64_t m, int64_t n, bool grouped);
int launch_bias_grad(int dtype, BiasGrad b, hipStream_t stream);

int check_matrix(const char *name, const void *p, int64_t ld, int64_t cols);

// What a descriptor's pointer stands for: rows of cols values, ld apart, groups stride apart.
struct Region {
    const char *name;
    const void *p;                            // NULL: not given
    int64_t rows, cols, ld;
    int groups = 1;
    int64_t stride = 0;
};
// An output and what must not lie in it (NULL: nothing). Exact where both have one distance between rows or one
// of them is a single run of values; else an overlap is seen if the first value of one is in the other.
int check_apart(const Region &out, std::initializer_list<const Region *> others);

// C = A B^T with EpiLinear, all in rows (skinny: by is_skinny, with operands as they are); cols:
// B in columns (dX = dZ W); sum: C = A^T B over rows
template <typename T>
int product(bool skinny, const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int groups,
            const int32_t *offsets, EpiLinear<T> epi, Scratch &s, bool run, hipStream_t stream);
template <typename T>
int product_cols(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int groups, const int32_t *offsets,
                 EpiPlain<T> epi, Scratch &s, bool run, hipStream_t stream);
template <typename T>
int product_sum(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int groups, const int32_t *offsets,
                EpiPlain<T> epi, Scratch &s, bool run, hipStream_t stream);

template <typename T> inline EpiPlain<T> plain_output(void *y, int64_t ld, int64_t n, int64_t stride = 0)
{
    return {(T *)y, ld, stride, (int32_t)n};
}
template <typename T> inline EpiLinear<T> linear_output(void *y, int64_t ld, int64_t n)
{
    EpiLinear<T> e = {};
    e.y = (T *)y;
    e.ldy = ld;
    e.N = (int32_t)n;
    return e;
}

inline int check_scratch(size_t need, const void *ws, int64_t bytes)
{
    if (need == 0) return HEDDLE_OK;
    if (!ws || bytes < 0 || (size_t)bytes < need) return fail(HEDDLE_E_INVAL, "workspace smaller than the call needs");
    if ((uintptr_t)ws & 255) return fail(HEDDLE_E_INVAL, "workspace is not 256-byte aligned");
    return HEDDLE_OK;
}

}  // namespace mm
}  // namespace heddle
