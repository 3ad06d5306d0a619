// Y = act(X W^T + b) + R and its gradients on gfx950's matrix cores.
//
// Forward: 2 m n k flops over m k + n k + m n values, one launch: bias,
// activation and residual are applied to the sums before they are rounded.
// Backward: dZ = dY act'(Z) is formed once, in the pass that sums db (without
// an activation dZ is dY itself), then dX = dZ W and dW = dZ^T X.
// Bound by the matrix cores from some 500 rows on: 4096 rows of 4096 x 10816 with bias and
// gelu_tanh 366 us forward (990 TFLOP/s), dZ and db 76 us (266 MB, 3.5 TB/s), dX 295 us and dW
// 328 us (1232 and 1107 TFLOP/s); 8192^3 alone 795 us (1383 TFLOP/s). Bound by latency for small
// odd sizes: 1001 x 1027 x 513 in 80 to 144 workgroups that walk 9 to 17 k-tiles, 10 to 18 us each.
#include "linear.h"

namespace heddle {
namespace mm {

// The tile shape and the split of the reduction with the least estimated time. Constants in
// us, from times of every shape and split on 270 products of 33 .. 8192 rows, 128 .. 20000
// columns and k of the three memory orders, before stores went past the caches, gradients had
// an epilogue of their own and 64 x 128 a third buffer. On the kernels as they are, over 270
// other such products: the choice is the best one for half of them, costs 1.3% over it on
// average, 9% for one in twenty and 18% at worst (59 x 976 x 3456, 16 parts for 8). step: a k-tile on a CU whose workgroup slots are taken; least: the same for
// workgroups alone on their CU; fixed: start and epilogue of a round of workgroups.
//   256 x 256: one workgroup a CU, the highest rate; 128 x 128: four a CU, each with one buffer
//   (what fills the chip with 2000 x 2000 outputs, and what writes most while little is
//   summed); 64 x 128: three a CU, for few rows.
// (Of 64 x 128, a third buffer where a workgroup has a CU to itself is not in the estimate.)
Shape shape_of(int64_t M, int64_t N, int64_t K, int groups, bool gated, Order order)
{
    static const struct { int bm, bn, per_cu; double step[3], least, fixed; } cfg[3] = {
        {256, 256, 1, {1.53, 1.50, 1.64}, 1.20, 7.2},
        {128, 128, 4, {2.45, 2.36, 2.29}, 0.93, 5.3},
        {64, 128, 3, {1.13, 1.09, 1.16}, 0.52, 3.3},
    };
    const int cus = 256;
    const bool sums = order == kColsCols;
    const int64_t cols = gated ? 2 * N : N, kt = K > 0 ? (K + kBK - 1) / kBK : 1;
    // groups: every one of the average size; with offsets, also of one group, a reduction is not split
    const bool grouped = groups > 0;
    const int64_t rows = grouped && !sums ? (M + groups - 1) / groups : M, outer = grouped ? groups : 1;
    const int64_t steps = grouped && sums ? (kt + groups - 1) / groups : kt;
    Shape best = {0, 1, (int)kt};
    // Experts of few rows: the weights' reading bounds, and tiles of 64 x 256 read 512 bytes of
    // a row of theirs (training step over 64 experts of 4096 x 1632, 24 rows each: 1.68 ms, 1.71
    // with 64 x 128), where they fill the chip (16 of 2048 x 408, 24 rows each, forward: 52 us,
    // 33 with 64 x 128).
    if (grouped && !sums && rows <= 96 && (cols + 255) / 256 * groups > 2 * cus) return {3, 1, (int)kt};
    double least = 0;
    for (int c = 0; c < 3; c++)
        for (int s = 1, log2 = 0; s == 1 || (s <= 16 && !grouped && (kt + s - 1) / s >= 4); s *= 2, log2++) {
            const double part = (double)((steps + s - 1) / s);
            const int64_t tiles = (rows + cfg[c].bm - 1) / cfg[c].bm * ((cols + cfg[c].bn - 1) / cfg[c].bn) * outer * s;
            const int64_t full = tiles / (cus * cfg[c].per_cu), rest = tiles - full * cus * cfg[c].per_cu;
            const double step = cfg[c].step[order];
            double t = (double)full * (part * step + cfg[c].fixed);
            if (rest) {
                const double share = (double)((rest + cus - 1) / cus) / cfg[c].per_cu;
                const double alone = step * share > cfg[c].least ? step * share : cfg[c].least;
                t += part * alone + cfg[c].fixed * (0.5 + 0.5 * share);
            }
            if (s > 1) t += 2.9 + 0.3 * log2 + 1.2e-6 * (double)s * (double)M * (double)cols;
            if (least == 0 || t < least) {
                least = t;
                best = {c, s, (int)((kt + s - 1) / s)};
            }
        }
    return best;
}

// A workgroup alone on its CU keeps two tiles on their way, not one (64 x 10816 x 4096:
// 27.5 -> 23.1 us); where there are more, a third workgroup does more than a third buffer
// (64 x 4096 x 10816: 24.7 us, 26.6 with three). Groups: about half have a tile that is
// not full.
bool third_buffer(int64_t M, int64_t N, int groups, bool gated, bool sums, int splits)
{
    const int64_t rows = (M + 63) / 64 + (sums ? 0 : groups / 2), cols = (gated ? 2 * N : N) + 127;
    return rows * (cols / 128) * (sums && groups ? groups : splits) <= 256;
}

int check_matrix(const char *name, const void *p, int64_t ld, int64_t cols)
{
    if (!p) return fail(HEDDLE_E_INVAL, std::string(name) + " is NULL");
    if ((uintptr_t)p & 1) return fail(HEDDLE_E_INVAL, std::string(name) + " is not aligned to its values");
    if (ld < cols || ld > HEDDLE_MAX_LD) return fail(HEDDLE_E_INVAL, std::string(name) + ": ld out of range");
    return HEDDLE_OK;
}

// values from a's first to b's
static int64_t between(const Region &a, const Region &b) { return ((intptr_t)b.p - (intptr_t)a.p) / 2; }

static bool holds_first_of(const Region &a, const Region &b)
{
    int64_t at = between(a, b);
    if (at < 0) return false;
    if (a.groups > 1) {
        const int64_t g = at / a.stride < a.groups ? at / a.stride : a.groups - 1;
        at -= g * a.stride;
    }
    return at / a.ld < a.rows && at % a.ld < a.cols;
}

static bool overlap(const Region &x, const Region &y)
{
    // (in fp64: exact below 2^53 values, and no product of sizes overflows)
    auto length = [](const Region &r) { return (double)(r.groups - 1) * (double)r.stride + (double)(r.rows - 1) * (double)r.ld + (double)r.cols; };
    const int64_t d = between(x, y);
    if (d >= 0 ? (double)d >= length(x) : (double)-d >= length(y)) return false;
    Region a = x, b = y;
    for (Region *r : {&a, &b}) {
        if (r->groups > 1 && r->stride == r->rows * r->ld) r->rows *= r->groups, r->groups = 1;
        if (r->groups == 1 && (r->ld == r->cols || r->rows == 1)) r->cols += (r->rows - 1) * r->ld, r->rows = 1;
    }
    if (a.groups > 1 || b.groups > 1 || (a.rows > 1 && b.rows > 1 && a.ld != b.ld)) return holds_first_of(a, b) || holds_first_of(b, a);
    // rows i of a and j of b meet where -b.cols < d + q ld < a.cols, q = j - i
    const int64_t ld = a.rows > 1 ? a.ld : b.ld, least = -b.cols - d;
    int64_t q = least / ld - (least % ld < 0) + 1;
    if (q < 1 - a.rows) q = 1 - a.rows;
    return q <= b.rows - 1 && d + q * ld < a.cols;
}

int check_apart(const Region &out, std::initializer_list<const Region *> others)
{
    if (!out.p || out.rows == 0) return HEDDLE_OK;
    for (const Region *r : others)
        if (r && r->p && r->rows > 0 && overlap(out, *r)) return fail(HEDDLE_E_INVAL, std::string(out.name) + " overlaps " + r->name);
    return HEDDLE_OK;
}

__global__ void __launch_bounds__(256) copy_rows_kernel(Copies c)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < c.eights; i += (int64_t)gridDim.x * 256) {
        int n = 0;
        while (n + 1 < c.count && i >= c.one[n + 1].first) n++;
        const Copies::One &o = c.one[n];
        const int64_t at = i - o.first, per = o.ldd / 8, r = at / per, j = (at - r * per) * 8, g = r / o.rows;
        const uint16_t *from = o.src + g * o.stride + (r - g * o.rows) * o.ld + j;
        s16x8 v;
        if (j + 8 <= o.cols) {
            __builtin_memcpy(&v, from, 16);   // at any address its values may have
        } else {
#pragma unroll
            for (int q = 0; q < 8; q++) v[q] = j + q < o.cols ? (short)from[q] : (short)0;
        }
        *(s16x8 *)(o.dst + r * o.ldd + j) = v;
    }
}

void Copies::add(Operand &o, int64_t rows, int64_t cols, int groups, Scratch &s)
{
    if (rows == 0 || !needs_copy(o, groups)) return;
    const int64_t ldd = scratch_ld(cols);
    uint16_t *to = (uint16_t *)s.take((size_t)(rows * groups) * ldd * 2);
    one[count++] = {(const uint16_t *)o.p, to, o.ld, o.stride, rows, cols, ldd, eights};
    eights += rows * groups * (ldd / 8);
    o = {to, ldd, rows * ldd};
}

int Copies::launch(hipStream_t stream) const
{
    if (count == 0) return HEDDLE_OK;
    const int64_t want = (eights + 255) / 256;
    hipLaunchKernelGGL(copy_rows_kernel, dim3((unsigned)(want < 16384 ? want : 16384)), dim3(256), 0, stream, *this);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "copy_rows_kernel");
}

// A workgroup takes 256 columns (32 lanes of eight) and its chunk of rows, 8
// rows at a time; its lanes' sums are joined in LDS in a fixed order.
template <typename T> __global__ void __launch_bounds__(256) bias_grad_kernel(BiasGrad b)
{
    __shared__ float part[8][256 + 8];
    const int col = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int n = blockIdx.x * 256 + col * 8, count = b.n - n;
    const int g = blockIdx.y / b.chunks, chunk = blockIdx.y - g * b.chunks;
    int lo = 0, hi = b.m;
    if (b.offsets) group_range(b.offsets, first_offsets(b.offsets, b.groups), g, b.m, lo, hi);
    const int first = lo + chunk * b.chunk_rows;
    const int last = b.offsets ? hi : min(hi, first + b.chunk_rows);
    float sum[8] = {};
    if (count > 0) {
#pragma unroll 4
        for (int m = first + row; m < last; m += 8) {
            float v[8];
            load8((const T *)b.dy + m * b.lddy + n, count, v);
            if (b.act) {
                float z[8];
                load8((const T *)b.pre + m * b.ldp + n, count, z);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    float a, d;
                    act_both(b.act, z[i], a, d);
                    v[i] *= d;
                }
            }
            if (b.dz) store8((T *)b.dz + m * b.lddz + n, count, v);
#pragma unroll
            for (int i = 0; i < 8; i++) sum[i] += v[i];
        }
    }
    if (!b.db) return;
#pragma unroll
    for (int i = 0; i < 8; i++) part[row][col * 8 + i] = sum[i];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= b.n) return;
    float v = 0;
#pragma unroll
    for (int r = 0; r < 8; r++) v += part[r][threadIdx.x];
    if (b.chunks > 1) b.partial[(int64_t)chunk * b.n + c] = v;
    else ((T *)b.db)[(int64_t)g * b.n + c] = (T)v;
}

// 32 columns, 8 parts of the chunks
template <typename T> __global__ void __launch_bounds__(256) bias_join_kernel(BiasGrad b)
{
    __shared__ float part[8][32];
    const int col = threadIdx.x & 31, row = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
    float v = 0;
    if (c < b.n) {
#pragma unroll 8
        for (int i = row; i < b.chunks; i += 8) v += b.partial[(int64_t)i * b.n + c];
    }
    part[row][col] = v;
    __syncthreads();
    if (row || c >= b.n) return;
#pragma unroll
    for (int r = 1; r < 8; r++) v += part[r][col];
    ((T *)b.db)[c] = (T)v;
}

// enough chunks of rows to fill the chip, at least 32 rows in each
static void bias_chunks(int64_t m, int64_t n, bool grouped, int &chunks, int &rows)
{
    const int64_t blocks = (n + 255) / 256, want = grouped ? 1 : (2048 + blocks - 1) / blocks, most = (m + 31) / 32;
    chunks = (int)(want < most ? want : most);
    if (chunks < 1) chunks = 1;
    rows = (int)((m + chunks - 1) / chunks);
}

int64_t bias_grad_bytes(int64_t m, int64_t n, bool grouped)
{
    int chunks, rows;
    bias_chunks(m, n, grouped, chunks, rows);
    return chunks > 1 ? (int64_t)chunks * n * 4 : 0;
}

template <typename T> static int run_bias_grad(BiasGrad b, hipStream_t stream)
{
    bias_chunks(b.m, b.n, b.offsets != nullptr, b.chunks, b.chunk_rows);
    const int groups = b.offsets ? b.groups : 1;
    const dim3 grid((unsigned)((b.n + 255) / 256), (unsigned)(groups * b.chunks));
    hipLaunchKernelGGL((bias_grad_kernel<T>), grid, dim3(256), 0, stream, b);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "bias_grad_kernel");
    if (b.db && b.chunks > 1) {
        hipLaunchKernelGGL((bias_join_kernel<T>), dim3((unsigned)((b.n + 31) / 32)), dim3(256), 0, stream, b);
        e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "bias_join_kernel");
    }
    return HEDDLE_OK;
}

int launch_bias_grad(int dtype, BiasGrad b, hipStream_t stream)
{
    return dtype == HEDDLE_T_BF16 ? run_bias_grad<__bf16>(b, stream) : run_bias_grad<_Float16>(b, stream);
}

static Args rows_args(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int groups, const int32_t *offsets)
{
    Args x = {};
    x.a = a.p, x.lda = a.ld;
    x.b = b.p, x.ldb = b.ld, x.stride_b = b.stride;
    x.M = (int)m, x.N = (int)n, x.K = (int)k;
    x.offsets = offsets;
    x.groups = offsets ? groups : 1;
    return x;
}

template <typename T>
int product(bool skinny, const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int groups,
            const int32_t *offsets, EpiLinear<T> epi, Scratch &s, bool run, hipStream_t stream)
{
    const Shape sh = shape_of(m, n, k, offsets ? groups : 0, false, kRowsRows);
    Args x = rows_args(a, b, m, n, k, groups, offsets);
    if (!skinny) x.partial = (float *)s.take(partial_bytes(sh, m, n, false));
    if (!run || m == 0) return HEDDLE_OK;
    if (skinny) return launch_skinny<T>(x, epi, stream);
    return launch_gemm<false, false, kGroupRows, T>(x, sh, epi, stream);
}

template <typename T>
int product_cols(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int groups, const int32_t *offsets,
                 EpiPlain<T> epi, Scratch &s, bool run, hipStream_t stream)
{
    const Shape sh = shape_of(m, n, k, offsets ? groups : 0, false, kRowsCols);
    Args x = rows_args(a, b, m, n, k, groups, offsets);
    x.partial = (float *)s.take(partial_bytes(sh, m, n, false));
    if (!run || m == 0) return HEDDLE_OK;
    return launch_gemm<false, true, kGroupRows, T>(x, sh, epi, stream);
}

template <typename T>
int product_sum(const Operand &a, const Operand &b, int64_t m, int64_t n, int64_t k, int groups, const int32_t *offsets,
                EpiPlain<T> epi, Scratch &s, bool run, hipStream_t stream)
{
    const Shape sh = shape_of(m, n, k, offsets ? groups : 0, false, kColsCols);
    Args x = rows_args(a, b, m, n, k, groups, offsets);
    x.partial = (float *)s.take(partial_bytes(sh, m, n, false));
    if (!run) return HEDDLE_OK;
    return launch_gemm<true, true, kGroupSum, T>(x, sh, epi, stream);
}

#define HEDDLE_PRODUCTS(T)                                                                                             \
    template int product<T>(bool, const Operand &, const Operand &, int64_t, int64_t, int64_t, int, const int32_t *,   \
                            EpiLinear<T>, Scratch &, bool, hipStream_t);                                               \
    template int product_cols<T>(const Operand &, const Operand &, int64_t, int64_t, int64_t, int, const int32_t *,    \
                                 EpiPlain<T>, Scratch &, bool, hipStream_t);                                           \
    template int product_sum<T>(const Operand &, const Operand &, int64_t, int64_t, int64_t, int, const int32_t *,     \
                                EpiPlain<T>, Scratch &, bool, hipStream_t);
HEDDLE_PRODUCTS(__bf16)
HEDDLE_PRODUCTS(_Float16)

static int check_linear(const heddle_linear_desc *d, bool backward)
{
    if (!d) return fail(HEDDLE_E_INVAL, "descriptor is NULL");
    if (d->dtype != HEDDLE_T_BF16 && d->dtype != HEDDLE_T_F16) return fail(HEDDLE_E_INVAL, "dtype is neither BF16 nor F16");
    if (d->act < HEDDLE_A_NONE || d->act > HEDDLE_A_SILU) return fail(HEDDLE_E_INVAL, "unknown activation");
    if (d->m < 0 || d->n < 1 || d->k < 1 || d->m > kMaxRows || d->n > HEDDLE_MAX_LD || d->k > HEDDLE_MAX_LD)
        return fail(HEDDLE_E_INVAL, "m, n or k out of range");
    if (d->d_offsets && (d->groups < 1 || d->groups > HEDDLE_MAX_GROUPS)) return fail(HEDDLE_E_INVAL, "groups out of range");
    if (((uintptr_t)d->d_offsets & 3)) return fail(HEDDLE_E_INVAL, "d_offsets is misaligned");
    const bool grouped = d->d_offsets != nullptr;
    int rc = HEDDLE_OK;
    auto matrix = [&](const char *name, const void *p, int64_t ld, int64_t cols) {
        if (rc == HEDDLE_OK && d->m > 0) rc = check_matrix(name, p, ld, cols);
    };
    auto weights = [&](const char *name, const void *p, int64_t ld, int64_t stride) {
        if (rc == HEDDLE_OK) rc = check_matrix(name, p, ld, d->k);
        if (rc == HEDDLE_OK && grouped && d->groups > 1 && stride < (d->n - 1) * ld + d->k)
            rc = fail(HEDDLE_E_INVAL, std::string(name) + ": the groups overlap");
    };
    if (!backward) {
        matrix("x", d->x, d->ldx, d->k);
        weights("w", d->w, d->ldw, d->stride_w);
        if (d->residual) matrix("residual", d->residual, d->ldr, d->n);
        if (d->preact) matrix("preact", d->preact, d->ldp, d->n);
        matrix("y", d->y, d->ldy, d->n);
        if (rc == HEDDLE_OK && ((uintptr_t)d->bias & 1)) rc = fail(HEDDLE_E_INVAL, "bias is not aligned to its values");
    } else {
        matrix("dy", d->dy, d->lddy, d->n);
        if (d->act != HEDDLE_A_NONE) matrix("preact", d->preact, d->ldp, d->n);
        if (d->dx) {
            weights("w", d->w, d->ldw, d->stride_w);
            matrix("dx", d->dx, d->lddx, d->k);
        }
        if (d->dw) {
            matrix("x", d->x, d->ldx, d->k);
            weights("dw", d->dw, d->lddw, d->stride_dw);
        }
        if (rc == HEDDLE_OK && ((uintptr_t)d->db & 1)) rc = fail(HEDDLE_E_INVAL, "db is not aligned to its values");
    }
    return rc;
}

// Whether an output lies on what the call reads when it writes it, or later.
static int check_overlaps(const heddle_linear_desc *d, bool backward)
{
    const int groups = d->d_offsets ? d->groups : 1;
    const Region x = {"x", d->x, d->m, d->k, d->ldx}, w = {"w", d->w, d->n, d->k, d->ldw, groups, d->stride_w};
    const Region pre = {"preact", d->preact, d->m, d->n, d->ldp};
    int rc;
    if (!backward) {
        const Region y = {"y", d->y, d->m, d->n, d->ldy}, bias = {"bias", d->bias, 1, groups * d->n, groups * d->n};
        const Region r = {"residual", d->residual, d->m, d->n, d->ldr};
        const bool own = r.p == y.p && (r.ld == y.ld || d->m == 1);       // y may be the residual itself
        rc = check_apart(y, {&x, &w, &bias, &pre, own ? nullptr : &r});
        return rc ? rc : check_apart(pre, {&x, &w, &bias, &r});
    }
    const Region dy = {"dy", d->dy, d->m, d->n, d->lddy};
    const Region dx = {"dx", d->dx, d->m, d->k, d->lddx}, dw = {"dw", d->dw, d->n, d->k, d->lddw, groups, d->stride_dw};
    const Region db = {"db", d->db, 1, groups * d->n, groups * d->n};
    // with an activation, dy and preact are read by the first pass alone, which leaves dZ and db
    const bool act = d->act != HEDDLE_A_NONE;
    rc = check_apart(db, {&dy, act ? &pre : nullptr, &dx, &dw, d->dx ? &w : nullptr, d->dw ? &x : nullptr});
    if (rc == HEDDLE_OK) rc = check_apart(dx, {act ? nullptr : &dy, &w, &dw, d->dw ? &x : nullptr});
    return rc ? rc : check_apart(dw, {act ? nullptr : &dy, &x});
}

template <typename T> static int forward(const heddle_linear_desc *d, Scratch &s, bool run, hipStream_t stream)
{
    const int groups = d->d_offsets ? d->groups : 1;
    Operand x = {d->x, d->ldx, 0}, w = {d->w, d->ldw, d->stride_w};
    const bool skinny = is_skinny(d->m, d->n, d->k, d->d_offsets ? groups : 0, needs_copy(x, 1) || needs_copy(w, groups));
    if (!skinny) {
        Copies c;
        c.add(x, d->m, d->k, 1, s);
        c.add(w, d->n, d->k, groups, s);
        if (const int rc = run ? c.launch(stream) : HEDDLE_OK) return rc;
    }
    EpiLinear<T> e = linear_output<T>(d->y, d->ldy, d->n);
    e.pre = (T *)d->preact, e.ldp = d->ldp;
    e.bias = (const T *)d->bias;
    e.residual = (const T *)d->residual, e.ldr = d->ldr;
    e.act = d->act;
    return product<T>(skinny, x, w, d->m, d->n, d->k, groups, d->d_offsets, e, s, run, stream);
}

template <typename T> static int backward(const heddle_linear_desc *d, Scratch &s, bool run, hipStream_t stream)
{
    const int groups = d->d_offsets ? d->groups : 1;
    int rc = HEDDLE_OK;
    Operand dz = {d->dy, d->lddy, 0};
    const bool act = d->act != HEDDLE_A_NONE, products = d->dx || d->dw;
    BiasGrad b = {};
    b.dy = d->dy, b.lddy = d->lddy, b.pre = d->preact, b.ldp = d->ldp, b.db = d->db, b.act = d->act;
    b.m = (int)d->m, b.n = (int)d->n, b.offsets = d->d_offsets, b.groups = groups;
    if (products && (act || needs_copy(dz, 1))) {
        // dZ, or dY in rows that the products can read
        b.lddz = scratch_ld(d->n);
        b.dz = s.take((size_t)d->m * b.lddz * 2);
        dz = {b.dz, b.lddz, 0};
    }
    if (b.db) b.partial = (float *)s.take(bias_grad_bytes(d->m, d->n, d->d_offsets != nullptr));
    if (run && (b.db || (b.dz && d->m > 0))) rc = launch_bias_grad(d->dtype, b, stream);
    Operand w = {d->w, d->ldw, d->stride_w}, x = {d->x, d->ldx, 0};
    Copies c;
    if (d->dx && d->m > 0) c.add(w, d->n, d->k, groups, s);
    if (d->dw) c.add(x, d->m, d->k, 1, s);
    if (rc == HEDDLE_OK && run) rc = c.launch(stream);
    if (rc == HEDDLE_OK && d->dx)
        rc = product_cols<T>(dz, w, d->m, d->k, d->n, groups, d->d_offsets, plain_output<T>(d->dx, d->lddx, d->k), s, run,
                             stream);
    if (rc == HEDDLE_OK && d->dw)
        rc = product_sum<T>(dz, x, d->n, d->k, d->m, groups, d->d_offsets,
                            plain_output<T>(d->dw, d->lddw, d->k, groups > 1 ? d->stride_dw : 0), s, run, stream);
    return rc;
}

static int linear(const heddle_linear_desc *d, bool back, void *ws, int64_t bytes, bool run, hipStream_t stream, int64_t *need)
{
    int rc = check_linear(d, back);
    if (rc) return rc;
    for (int pass = 0; pass < 2; pass++) {
        Scratch s = {pass ? (char *)ws : nullptr, 0};
        const bool go = pass == 1;
        rc = d->dtype == HEDDLE_T_BF16 ? (back ? backward<__bf16>(d, s, go, stream) : forward<__bf16>(d, s, go, stream))
                                       : (back ? backward<_Float16>(d, s, go, stream) : forward<_Float16>(d, s, go, stream));
        if (rc) return rc;
        if (pass == 0) {
            if (need) *need = (int64_t)s.used;
            if (!run) return HEDDLE_OK;
            rc = check_scratch(s.used, ws, bytes);
            if (rc == HEDDLE_OK) rc = check_overlaps(d, back);
            if (rc) return rc;
        }
    }
    return HEDDLE_OK;
}

}  // namespace mm
}  // namespace heddle

using namespace heddle;

extern "C" int heddle_linear(const heddle_linear_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return mm::linear(d, false, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_linear_backward(const heddle_linear_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return mm::linear(d, true, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_linear_workspace(const heddle_linear_desc *d, int32_t backward, int64_t *h_bytes)
{
    if (!h_bytes) return fail(HEDDLE_E_INVAL, "h_bytes is NULL");
    return mm::linear(d, backward != 0, nullptr, 0, false, nullptr, h_bytes);
}
