// The gated feed-forward block and its gradients on gfx950's matrix cores.
//
// Forward, 6 t d f flops: one product over [gate | up] rows whose tiles
// alternate 16 gate and 16 up rows of Win, so that a lane holds a unit's gate
// and up sums side by side and writes H = act(gate) up; then H Wout^T.
// Backward, 12 t d f flops: dY Wout forms dP and H again in its epilogue
// (P is what the forward pass kept; H costs t f values less to keep), then the
// three products over them.
// Bound by the matrix cores for many rows: 4096 rows of 4096 x 10816, forward 657 + 289 us (1104
// and 1258 TFLOP/s), backward 417 us with dP and H in the epilogue (871), then 558, 610 and 309 us
// (1301, 1191, 1174). Bound by the weights for few rows a group: 64 rows for each of 64 experts
// of 4096 x 1632, forward 398 + 250 us (4.3 and 3.4 TB/s), backward 236 + 355 us (3.6 and 4.8),
// the weights' gradients 552 + 323 us (3.1 and 2.6 TB/s written).
#include "linear.h"

namespace heddle {
namespace mm {

static int check_ffn(const heddle_gated_ffn_desc *d, bool backward)
{
    if (!d) return fail(HEDDLE_E_INVAL, "descriptor is NULL");
    if (d->dtype != HEDDLE_T_BF16 && d->dtype != HEDDLE_T_F16) return fail(HEDDLE_E_INVAL, "dtype is neither BF16 nor F16");
    if (d->act < HEDDLE_A_NONE || d->act > HEDDLE_A_SILU) return fail(HEDDLE_E_INVAL, "unknown activation");
    if (d->t < 0 || d->d < 1 || d->f < 1 || d->t > kMaxRows || d->d > HEDDLE_MAX_LD || 2 * d->f > HEDDLE_MAX_LD)
        return fail(HEDDLE_E_INVAL, "t, d or f out of range");
    if (d->d_offsets && (d->groups < 1 || d->groups > HEDDLE_MAX_GROUPS)) return fail(HEDDLE_E_INVAL, "groups out of range");
    if (((uintptr_t)d->d_offsets & 3)) return fail(HEDDLE_E_INVAL, "d_offsets is misaligned");
    const bool grouped = d->d_offsets != nullptr;
    int rc = HEDDLE_OK;
    auto matrix = [&](const char *name, const void *p, int64_t ld, int64_t cols) {
        if (rc == HEDDLE_OK && d->t > 0) rc = check_matrix(name, p, ld, cols);
    };
    auto weights = [&](const char *name, const void *p, int64_t ld, int64_t stride, int64_t rows, int64_t cols) {
        if (rc == HEDDLE_OK) rc = check_matrix(name, p, ld, cols);
        if (rc == HEDDLE_OK && grouped && d->groups > 1 && stride < (rows - 1) * ld + cols)
            rc = fail(HEDDLE_E_INVAL, std::string(name) + ": the groups overlap");
    };
    if (!backward) {
        matrix("x", d->x, d->ldx, d->d);
        weights("w_in", d->w_in, d->ldw_in, d->stride_in, 2 * d->f, d->d);
        weights("w_out", d->w_out, d->ldw_out, d->stride_out, d->d, d->f);
        if (d->residual) matrix("residual", d->residual, d->ldr, d->d);
        if (d->preact) matrix("preact", d->preact, d->ldp, 2 * d->f);
        matrix("y", d->y, d->ldy, d->d);
    } else {
        matrix("dy", d->dy, d->lddy, d->d);
        matrix("preact", d->preact, d->ldp, 2 * d->f);
        weights("w_out", d->w_out, d->ldw_out, d->stride_out, d->d, d->f);
        if (d->dx) {
            weights("w_in", d->w_in, d->ldw_in, d->stride_in, 2 * d->f, d->d);
            matrix("dx", d->dx, d->lddx, d->d);
        }
        if (d->dw_in) {
            matrix("x", d->x, d->ldx, d->d);
            weights("dw_in", d->dw_in, d->lddw_in, d->stride_dw_in, 2 * d->f, d->d);
        }
        if (d->dw_out) weights("dw_out", d->dw_out, d->lddw_out, d->stride_dw_out, d->d, d->f);
    }
    return rc;
}

// Whether an output lies on what the call reads when it writes it, or later, or on another output.
static int check_overlaps(const heddle_gated_ffn_desc *d, bool backward)
{
    const int groups = d->d_offsets ? d->groups : 1;
    const Region x = {"x", d->x, d->t, d->d, d->ldx}, wi = {"w_in", d->w_in, 2 * d->f, d->d, d->ldw_in, groups, d->stride_in};
    const Region wo = {"w_out", d->w_out, d->d, d->f, d->ldw_out, groups, d->stride_out}, pre = {"preact", d->preact, d->t, 2 * d->f, d->ldp};
    int rc;
    if (!backward) {
        // the first product has read x when the second one writes y
        const Region y = {"y", d->y, d->t, d->d, d->ldy}, r = {"residual", d->residual, d->t, d->d, d->ldr};
        const bool own = r.p == y.p && (r.ld == y.ld || d->t == 1);       // y may be the residual itself
        rc = check_apart(y, {&wo, &pre, own ? nullptr : &r});
        return rc ? rc : check_apart(pre, {&x, &wi, &wo, &r});
    }
    const Region dy = {"dy", d->dy, d->t, d->d, d->lddy}, dx = {"dx", d->dx, d->t, d->d, d->lddx};
    const Region di = {"dw_in", d->dw_in, 2 * d->f, d->d, d->lddw_in, groups, d->stride_dw_in};
    const Region dout = {"dw_out", d->dw_out, d->d, d->f, d->lddw_out, groups, d->stride_dw_out};
    // in this order, after dP and H, which are the last to read preact and w_out
    rc = check_apart(dx, {&wi, &di, &dout, d->dw_in ? &x : nullptr, d->dw_out ? &dy : nullptr});
    if (rc == HEDDLE_OK) rc = check_apart(di, {&x, &dout, d->dw_out ? &dy : nullptr});
    return rc ? rc : check_apart(dout, {&dy});
}

template <typename T, typename Epi, bool BCOL>
static int hidden(bool skinny, const Operand &a, const Operand &b, int64_t t, int64_t f, int64_t k, int groups, const int32_t *offsets,
                  const Epi &epi, Scratch &s, bool run, hipStream_t stream)
{
    const Shape sh = shape_of(t, f, k, offsets ? groups : 0, Epi::gated, BCOL ? kRowsCols : kRowsRows);
    Args x = {};
    if (!skinny) x.partial = (float *)s.take(partial_bytes(sh, t, f, Epi::gated));
    if (!run || t == 0) return HEDDLE_OK;
    x.a = a.p, x.lda = a.ld;
    x.b = b.p, x.ldb = b.ld, x.stride_b = b.stride;
    x.M = (int)t, x.N = (int)f, x.K = (int)k, x.F = (int)f;
    x.offsets = offsets;
    x.groups = offsets ? groups : 1;
    if constexpr (!BCOL)
        if (skinny) return launch_skinny<T>(x, epi, stream);
    return launch_gemm<false, BCOL, kGroupRows, T>(x, sh, epi, stream);
}

template <typename T> static int forward(const heddle_gated_ffn_desc *d, Scratch &s, bool run, hipStream_t stream)
{
    const int groups = d->d_offsets ? d->groups : 1;
    if (d->t == 0) return HEDDLE_OK;
    Operand x = {d->x, d->ldx, 0}, wi = {d->w_in, d->ldw_in, d->stride_in}, wo = {d->w_out, d->ldw_out, d->stride_out};
    const int used = d->d_offsets ? groups : 0;
    const bool skinny_in = is_skinny(d->t, 2 * d->f, d->d, used, needs_copy(x, 1) || needs_copy(wi, groups));
    const bool skinny_out = is_skinny(d->t, d->d, d->f, used, needs_copy(wo, groups));
    Copies c;
    if (!skinny_in) {
        c.add(x, d->t, d->d, 1, s);
        c.add(wi, 2 * d->f, d->d, groups, s);
    }
    if (!skinny_out) c.add(wo, d->d, d->f, groups, s);
    if (const int rc = run ? c.launch(stream) : HEDDLE_OK) return rc;
    EpiGated<T> e = {};
    e.ldh = scratch_ld(d->f), e.h = (T *)s.take((size_t)d->t * e.ldh * 2);
    e.pre = (T *)d->preact, e.ldp = d->ldp;
    e.act = d->act, e.N = (int)d->f;
    int rc = hidden<T, EpiGated<T>, false>(skinny_in, x, wi, d->t, d->f, d->d, groups, d->d_offsets, e, s, run, stream);
    if (rc) return rc;
    EpiLinear<T> o = linear_output<T>(d->y, d->ldy, d->d);
    o.residual = (const T *)d->residual, o.ldr = d->ldr;
    return product<T>(skinny_out, {e.h, e.ldh, 0}, wo, d->t, d->d, d->f, groups, d->d_offsets, o, s, run, stream);
}

template <typename T> static int backward(const heddle_gated_ffn_desc *d, Scratch &s, bool run, hipStream_t stream)
{
    const int groups = d->d_offsets ? d->groups : 1;
    Operand dy = {d->dy, d->lddy, 0}, x = {d->x, d->ldx, 0}, wi = {d->w_in, d->ldw_in, d->stride_in},
            wo = {d->w_out, d->ldw_out, d->stride_out};
    int rc = HEDDLE_OK;
    if (!d->dx && !d->dw_in && !d->dw_out) return rc;
    if (d->t > 0) {
        Copies c;
        c.add(dy, d->t, d->d, 1, s);
        c.add(wo, d->d, d->f, groups, s);
        if (d->dx) c.add(wi, 2 * d->f, d->d, groups, s);
        if (d->dw_in) c.add(x, d->t, d->d, 1, s);
        if (run) rc = c.launch(stream);
        if (rc) return rc;
    }
    EpiGatedGrad<T> e = {};
    e.ldd = scratch_ld(2 * d->f), e.ldh = scratch_ld(d->f);
    e.dp = (T *)s.take((size_t)d->t * e.ldd * 2);
    e.h = (T *)s.take((size_t)d->t * e.ldh * 2);
    e.pre = (const T *)d->preact, e.ldp = d->ldp;
    e.act = d->act, e.N = (int)d->f;
    rc = hidden<T, EpiGatedGrad<T>, true>(false, dy, wo, d->t, d->f, d->d, groups, d->d_offsets, e, s, run, stream);
    if (rc) return rc;
    const Operand dp = {e.dp, e.ldd, 0}, h = {e.h, e.ldh, 0};
    if (d->dx)
        rc = product_cols<T>(dp, wi, d->t, d->d, 2 * d->f, groups, d->d_offsets, plain_output<T>(d->dx, d->lddx, d->d), s,
                             run, stream);
    if (rc == HEDDLE_OK && d->dw_in)
        rc = product_sum<T>(dp, x, 2 * d->f, d->d, d->t, groups, d->d_offsets,
                            plain_output<T>(d->dw_in, d->lddw_in, d->d, groups > 1 ? d->stride_dw_in : 0), s, run, stream);
    if (rc == HEDDLE_OK && d->dw_out)
        rc = product_sum<T>(dy, h, d->d, d->f, d->t, groups, d->d_offsets,
                            plain_output<T>(d->dw_out, d->lddw_out, d->f, groups > 1 ? d->stride_dw_out : 0), s, run, stream);
    return rc;
}

static int gated_ffn(const heddle_gated_ffn_desc *d, bool back, void *ws, int64_t bytes, bool run, hipStream_t stream,
                     int64_t *need)
{
    int rc = check_ffn(d, back);
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

extern "C" int heddle_gated_ffn(const heddle_gated_ffn_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return mm::gated_ffn(d, false, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_gated_ffn_backward(const heddle_gated_ffn_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return mm::gated_ffn(d, true, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_gated_ffn_workspace(const heddle_gated_ffn_desc *d, int32_t backward, int64_t *h_bytes)
{
    if (!h_bytes) return fail(HEDDLE_E_INVAL, "h_bytes is NULL");
    return mm::gated_ffn(d, backward != 0, nullptr, 0, false, nullptr, h_bytes);
}
