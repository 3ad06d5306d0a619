// Attention on gfx950's matrix cores: y = softmax(mask(cap tanh(scale q k / cap) - slope |distance|)) v.
//
// One pass over the keys with a running maximum and sum. Query rows of a key head, (query, head of its
// group) pairs in that order, are taken 32 a wavefront, so that heads that share keys share their tiles.
// forward_kernel (attention_forward.hip): 128 or 256 rows a workgroup over tiles of 64 keys.
// split_kernel: 32 rows a workgroup (few queries over long caches), each wavefront with tiles of its own, the
// keys of a row tile divided over `parts` workgroups; combine_kernel joins them. Bound by reading keys and values: 32
// sequences of up to 8192 keys, 8 key heads, 129 us (4.1 TB/s); one of 2048, 32 heads, 13 + 3.6 us (a wavefront has two tiles, and
// its start, its wait for both and the sums' exchange follow one another).
#include <algorithm>
#include <cmath>

#include "attention.h"

namespace heddle {
namespace attn {

// 32 rows a workgroup. The sums of a part, where there are several: DP values, the maximum (in modify()'s units, whose differences are exact where they count) and the sum.
template <typename T, int DP, int MODE> __global__ void __launch_bounds__(256) split_kernel(Args a, int64_t tiles)
{
    typedef Tile<DP, 32, 1> Tk;
    constexpr int kStage = 2 * Tk::kBytes, kLine = DP + 4;
    static_assert(4 * 32 * kLine * 4 + 4 * 64 * 4 <= 8 * kStage, "the wavefronts' sums fit where the tiles were");
    __shared__ __align__(1024) char smem[4][2][kStage];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const uint32_t rest = blockIdx.x / (uint32_t)a.kv_heads;
    const int hk = blockIdx.x - rest * a.kv_heads;
    const int64_t slot = rest / (uint32_t)a.parts;
    const int part = (int)(rest - (uint32_t)slot * a.parts);
    int s;
    int64_t tile;
    if (!find_slot(a.d_q, a.q_rows, a.packed, a.sequences, a.group, 32, tiles, slot, s, tile)) return;
    const Sequence q = sequence_of(a, s);
    if (tile * 32 >= (int64_t)q.lq * a.group) return;
    const int r0 = (int)tile * 32, rows = q.lq * a.group;
    const Row row = row_of(a, q, hk, r0 + col);
    const int end = limit_of(a, q, min(r0 + 31, rows - 1)), whole = limit_of(a, q, r0);   // (no row: what is summed is not written)
    const int all = (end + 31) / 32, per = (all + a.parts - 1) / a.parts;
    const int first = part * per, last = min(first + per, all);

    const T *pk = (const T *)a.k.p + s * a.k.seq + q.k0 * a.k.row + hk * a.k.head;
    const T *pv = (const T *)a.v.p + s * a.v.seq + q.k0 * a.v.row + hk * a.v.head;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&smem[wave][0][0];
    int ok[Tk::kLoads], ov[Tk::kLoads];
#pragma unroll
    for (int i = 0; i < Tk::kLoads; i++) ok[i] = Tk::offset(i, 0, a.k.row, a.dim, 32), ov[i] = Tk::offset(i, 0, a.v.row, a.dim, 32);
    auto load = [&](int t, int stage) {
        const int valid = q.lk - t * 32;
        const i32x4 bk = buffer_at(pk + (int64_t)t * 32 * a.k.row), bv = buffer_at(pv + (int64_t)t * 32 * a.v.row);
        const uint32_t to = lds + stage * kStage;
#pragma unroll
        for (int i = 0; i < Tk::kLoads; i++) mm::load_to_lds(bk, valid >= 32 ? ok[i] : Tk::offset(i, 0, a.k.row, a.dim, valid), to + i * 1024);
#pragma unroll
        for (int i = 0; i < Tk::kLoads; i++) mm::load_to_lds(bv, valid >= 32 ? ov[i] : Tk::offset(i, 0, a.v.row, a.dim, valid), to + Tk::kBytes + i * 1024);
    };
    State<DP> st;
    st.init();
    Places at;
    at.set<DP>();
    typename mm::pack8<T>::type qf[DP / 16];
    load_query<T, DP>(a, a.q, q, row, qf);
    const float slope = slope_of<MODE>(a, row.any ? row.head : 0);
    int stage = 0, t = first + wave;
    if (t < last) load(t, 0);
    // a wavefront's tiles are its own: it waits for its loads, and for its reads of the buffer that is filled next
    auto next = [&]() __attribute__((always_inline)) {
        constexpr int later = 2 * Tk::kLoads;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (t + 4 < last) {
            load(t + 4, stage ^ 1);
            asm volatile("s_waitcnt vmcnt(%0)" :: "n"(later) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
    };
    auto attend = [&](auto masked) __attribute__((always_inline)) {
        const char *tk = smem[wave][stage];
        f32x16 x = score<T, DP>(tk, at, 0, qf);
        typename mm::pack8<T>::type p[2];
        float was, sum;
        if (soften<T, MODE, decltype(masked)::value>(a, x, st.m, was, sum, t * 32 + 4 * h, row, slope, p)) rescale<MODE>(a, st, was);
        st.l += sum;
        collect<T, DP>(st, tk + Tk::kBytes, at, 0, p);
    };
    const int open = min(whole / 32, last);
    for (; t < open; t += 4, stage ^= 1) {
        next();
        attend(std::false_type());
    }
    for (; t < last; t += 4, stage ^= 1) {
        next();
        attend(std::true_type());
    }
    // the four wavefronts' sums
    const float m = st.m, l = st.l + other_half(st.l), unit = unit_of<MODE>(a);
    float *sums = (float *)&smem[0][0][0], *ms = sums + 4 * 32 * kLine;   // [wave][row][kLine], [wave][row] of m, then of l
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            *(mm::f32x4 *)(sums + (wave * 32 + col) * kLine + d * 32 + mfma_row(r, h)) = mm::f32x4{st.o[d][r], st.o[d][r + 1], st.o[d][r + 2], st.o[d][r + 3]};
    if (h == 0) ms[wave * 32 + col] = m, ms[128 + wave * 32 + col] = l;
    __syncthreads();
    const int mine = threadIdx.x >> 3, sub = threadIdx.x & 7;
    const Row out = row_of(a, q, hk, r0 + mine);
    if (!out.any) return;
    float top = ms[mine];
#pragma unroll
    for (int w = 1; w < 4; w++) top = fmaxf(top, ms[w * 32 + mine]);
    float f[4], sum = 0;
#pragma unroll
    for (int w = 0; w < 4; w++) {
        f[w] = ms[w * 32 + mine] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ms[w * 32 + mine] - top) * unit);
        sum += f[w] * ms[128 + w * 32 + mine];
    }
    const float inv = a.parts > 1 ? 1.0f : sum == 0 ? 0.0f : 1.0f / sum;
    float *p = a.partial + (((slot * a.kv_heads + hk) * 32 + mine) * a.parts + part) * (DP + 2);
    T *y = (T *)a.y.p + s * a.y.seq + (q.q0 + out.i) * a.y.row + out.head * a.y.head;
#pragma unroll
    for (int c = 0; c < DP / 32; c++) {
        const int d = c * 32 + sub * 4;
        mm::f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; w++) v += f[w] * *(const mm::f32x4 *)(sums + (w * 32 + mine) * kLine + d);
        if (a.parts > 1) {
#pragma unroll
            for (int i = 0; i < 4; i++) p[d + i] = v[i];
        } else {
            store4<T>(y, d, a.dim, a.out_vec, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        }
    }
    if (sub) return;
    if (a.parts > 1) p[DP] = top, p[DP + 1] = sum;
    else if (a.lse) a.lse[out.at * a.heads + out.head] = sum == 0 ? -INFINITY : (top * unit + offset_of<MODE>(a) + __log2f(sum)) * kLn2;
}

// Joins the parts of a row, one wavefront a row: a lane has a part's maximum and sum (parts <= 64), then DP / 64
// of the row's values, whose loads do not wait for each other (64 parts: 30 us when eight lanes took them in turn).
template <typename T, int DP> __global__ void __launch_bounds__(256) combine_kernel(Args a, int64_t tiles)
{
    constexpr int kValues = DP / 64;
    typedef float vec __attribute__((ext_vector_type(kValues)));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t tile_id = blockIdx.x >> 3, slot = tile_id / (uint32_t)a.kv_heads;      // eight workgroups for 32 rows
    const int mine = (blockIdx.x & 7) * 4 + wave, hk = tile_id - slot * a.kv_heads;
    int s;
    int64_t tile;
    if (!find_slot(a.d_q, a.q_rows, a.packed, a.sequences, a.group, 32, tiles, slot, s, tile)) return;
    const Sequence q = sequence_of(a, s);
    if (tile * 32 + mine >= (int64_t)q.lq * a.group) return;
    const Row out = row_of(a, q, hk, (int)tile * 32 + mine);
    const float *p = a.partial + (((int64_t)slot * a.kv_heads + hk) * 32 + mine) * a.parts * (DP + 2);
    const bool any = lane < a.parts;
    const float m = any ? p[lane * (DP + 2) + DP] : -INFINITY, l = any ? p[lane * (DP + 2) + DP + 1] : 0.0f;
    constexpr int kAhead = 8;
    vec x[kAhead], v = {};
    auto fetch = [&](int from) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kAhead; i++) x[i] = *(const vec *)(p + min(from + i, a.parts - 1) * (DP + 2) + lane * kValues);
    };
    fetch(0);
    float top = m;
#pragma unroll
    for (int d = 32; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float unit = unit_of(a), f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * unit);
    float sum = f * l;
#pragma unroll
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    for (int from = 0; from < a.parts; from += kAhead) {
        if (from) fetch(from);
#pragma unroll
        for (int i = 0; i < kAhead; i++)                    // (past the last part: a factor of zero; a part of no keys: zeros)
            v += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), min(from + i, 63))) * (from + i < a.parts ? x[i] : vec{});
    }
    const float inv = sum == 0 ? 0.0f : 1.0f / sum;
    T *y = (T *)a.y.p + s * a.y.seq + (q.q0 + out.i) * a.y.row + out.head * a.y.head;
#pragma unroll
    for (int i = 0; i < kValues; i++)
        if (lane * kValues + i < a.dim) y[lane * kValues + i] = (T)(v[i] * inv);
    if (a.lse && lane == 0) a.lse[out.at * a.heads + out.head] = sum == 0 ? -INFINITY : (top * unit + a.cap2 + __log2f(sum)) * kLn2;
}

// ---- operands that do not lie on 16-byte boundaries ----
__global__ void __launch_bounds__(256) copy_kernel(Copies c)
{
    const Copy &o = c.one[blockIdx.y];
    const int64_t per = o.pad / 8, all = o.rows * o.heads * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t line = i / per, row = line / o.heads, seq = row / o.per;
        const int col = (int)(i - line * per) * 8, head = (int)(line - row * o.heads);
        const uint16_t *from = o.src + seq * o.seq + (row - seq * o.per) * o.row + head * o.head + col;
        s16x8 v;
        if (col + 8 <= o.dim) {
            __builtin_memcpy(&v, from, 16);   // at any address its values may have
        } else {
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = col + k < o.dim ? (short)from[k] : (short)0;
        }
        *(s16x8 *)(o.dst + line * o.pad + col) = v;
    }
}

void Copies::add(const heddle_attention_desc *d, View &v, bool keys, mm::Scratch &s)
{
    if (!((uintptr_t)v.p & 15) && !((v.seq | v.row | v.head | d->dim) & 7)) return;
    const int64_t length = keys ? d->k_len : d->q_len, rows = d->packed ? length : length * d->sequences;
    const int32_t heads = keys ? d->kv_heads : d->heads, pad = (d->dim + 7) & ~7;
    if (rows == 0) return;
    uint16_t *to = (uint16_t *)s.take((size_t)(rows * heads) * pad * 2);
    one[count++] = {(const uint16_t *)v.p, to, d->packed ? 0 : v.seq, v.row, v.head, length, rows, heads, d->dim, pad};
    v = {to, d->packed ? 0 : length * heads * pad, (int64_t)heads * pad, pad};
}

int Copies::launch(hipStream_t stream) const
{
    if (count == 0) return HEDDLE_OK;
    int64_t most = 1;
    for (int i = 0; i < count; i++) most = std::max(most, (one[i].rows * one[i].heads * (one[i].pad / 8) + 255) / 256);
    hipLaunchKernelGGL(copy_kernel, dim3((unsigned)std::min<int64_t>(most, 4096), (unsigned)count), dim3(256), 0, stream, *this);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "attention's copies");
}

// ---- rows of no sequence, with few queries and where there is no sequence ----
__global__ void __launch_bounds__(256) clear_kernel(Args a, View v, int keys) { clear_rows(a, v, keys, blockIdx.x, gridDim.x); }

unsigned clearing(const heddle_attention_desc *d, int bits, bool keys, int threads)
{
    if (!(d->clear & bits)) return 0;
    const int64_t rows = (keys ? d->k_len : d->q_len) * (d->packed ? 1 : d->sequences), all = rows * (keys ? d->kv_heads : d->heads) * ((d->dim + 7) / 8);
    return (unsigned)std::min<int64_t>((all + threads - 1) / threads, kClearing);
}

int clear_all(const heddle_attention_desc *d, const Args &a, bool backward, hipStream_t stream)
{
    auto clear = [&](int bit, const View &v, bool keys) {
        const unsigned n = clearing(d, bit, keys, 256);
        if (v.p && n) hipLaunchKernelGGL(clear_kernel, dim3(n), dim3(256), 0, stream, a, v, (int)keys);
    };
    clear(1, backward ? a.dq : a.y, false);
    if (backward) clear(2, a.dk, true), clear(4, a.dv, true);
    if (!d->clear) return HEDDLE_OK;
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "attention's empty rows");
}

// ---- host ----
int mode_of(const heddle_attention_desc *d) { return (d->cap > 0 ? kCap : 0) | (d->d_slopes ? kSlopes : 0); }

Args base_args(const heddle_attention_desc *d)
{
    Args a = {};
    auto view = [&](const void *p, const int64_t *st, bool keys) {
        return View{p, d->packed || d->sequences <= 1 ? 0 : st[0], (keys ? d->k_len : d->q_len) <= 1 ? 0 : st[1], (keys ? d->kv_heads : d->heads) == 1 ? 0 : st[2]};
    };
    a.q = view(d->q, d->q_strides, false), a.k = view(d->k, d->k_strides, true), a.v = view(d->v, d->v_strides, true);
    a.y = view(d->y, d->y_strides, false), a.dy = view(d->dy, d->dy_strides, false), a.dq = view(d->dq, d->dq_strides, false);
    a.dk = view(d->dk, d->dk_strides, true), a.dv = view(d->dv, d->dv_strides, true);
    a.lse = d->lse, a.d_q = d->d_q, a.d_k = d->d_k, a.d_prefix = d->d_prefix, a.d_slopes = d->d_slopes;
    a.q_rows = d->packed ? d->q_len : d->q_len * d->sequences, a.k_rows = d->packed ? d->k_len : d->k_len * d->sequences;
    a.sequences = d->sequences, a.q_len = (int32_t)d->q_len, a.k_len = (int32_t)d->k_len, a.packed = d->packed;
    a.heads = d->heads, a.kv_heads = d->kv_heads, a.group = d->heads / d->kv_heads, a.dim = d->dim, a.causal = d->causal;
    a.scale = d->scale;
    a.scale2 = d->cap > 0 ? 2 * d->scale * kLog2e / d->cap : d->scale * kLog2e;
    a.cap2 = d->cap * kLog2e;
    a.unscale = -1.0f / a.scale2;
    return a;
}

// A tensor as runs of `cols` values at up to three distances, the smallest first. Dimensions that go on a run, or its
// repetition, are part of it.
typedef __int128 Wide;                        // (distances between sequences have no bound)
struct Runs {
    const char *name;
    const void *p;                            // NULL: not given, or of no values
    int64_t cols;
    int levels;
    int64_t size[3], step[3];
    // values from the first to the last, of the first n levels
    Wide extent(int n) const
    {
        Wide e = cols;
        for (int i = 0; i < n; i++) e += (Wide)(size[i] - 1) * step[i];
        return e;
    }
    // (distances that each step over all that is smaller; others may do without an overlap, but nothing lays tensors so)
    bool over_itself() const
    {
        for (int i = 0; i < levels; i++)
            if (step[i] < extent(i)) return true;
        return false;
    }
};
static Runs runs_of(const heddle_attention_desc *d, const char *name, const void *p, const int64_t *st, bool keys)
{
    const int64_t n[3] = {keys ? d->kv_heads : d->heads, keys ? d->k_len : d->q_len, d->packed ? 1 : d->sequences}, step[3] = {st[2], st[1], st[0]};
    Runs r = {name, n[0] * n[1] * n[2] ? p : nullptr, d->dim, 0, {}, {}};
    int order[3], count = 0;
    for (int i = 0; i < 3; i++) {
        if (n[i] <= 1) continue;
        int at = count++;
        for (; at > 0 && step[order[at - 1]] > step[i]; at--) order[at] = order[at - 1];
        order[at] = i;
    }
    for (int o = 0; o < count; o++) {
        const int i = order[o];
        if (!r.levels && step[i] == r.cols) r.cols *= n[i];
        else if (r.levels && step[i] == (Wide)r.size[r.levels - 1] * r.step[r.levels - 1]) r.size[r.levels - 1] *= n[i];
        else r.size[r.levels] = n[i], r.step[r.levels++] = step[i];
    }
    return r;
}

static int check(const heddle_attention_desc *d, bool backward)
{
    if (!d) return fail(HEDDLE_E_INVAL, "descriptor is NULL");
    if (d->dtype != HEDDLE_T_BF16 && d->dtype != HEDDLE_T_F16) return fail(HEDDLE_E_INVAL, "dtype is neither BF16 nor F16");
    if (d->heads < 1 || d->kv_heads < 1 || d->heads > HEDDLE_MAX_HEADS || d->heads % d->kv_heads)
        return fail(HEDDLE_E_INVAL, "heads out of range, or not a multiple of kv_heads");
    if (d->dim < 1 || d->dim > HEDDLE_MAX_HEAD_DIM) return fail(HEDDLE_E_INVAL, "dim out of range");
    if (d->sequences < 0 || d->sequences > HEDDLE_MAX_GROUPS) return fail(HEDDLE_E_INVAL, "sequences out of range");
    if (d->q_len < 0 || d->k_len < 0 || d->q_len > HEDDLE_MAX_ROWS / d->heads || d->k_len > HEDDLE_MAX_ROWS)
        return fail(HEDDLE_E_INVAL, "q_len or k_len out of range");
    if (!(d->scale >= 1e-20f && d->scale <= 1e20f)) return fail(HEDDLE_E_INVAL, "scale out of range");
    // the tanh is off by a few 2^-24 of 1: by 2^-11 of a score of any size at the largest cap
    if (!(d->cap == 0 || (d->cap >= 1e-3f && d->cap <= 4096))) return fail(HEDDLE_E_INVAL, "cap out of range");
    if (d->clear & ~7) return fail(HEDDLE_E_INVAL, "clear is no sum of 1, 2 and 4");
    if (d->packed && d->sequences > 0 && (!d->d_q || !d->d_k)) return fail(HEDDLE_E_INVAL, "packed sequences without offsets");
    if (((uintptr_t)d->d_q | (uintptr_t)d->d_k | (uintptr_t)d->d_prefix | (uintptr_t)d->d_slopes | (uintptr_t)d->lse) & 3)
        return fail(HEDDLE_E_INVAL, "d_q, d_k, d_prefix, d_slopes or lse is misaligned");
    const int64_t n = d->packed ? 1 : d->sequences, q_all = n * d->q_len, k_all = n * d->k_len;
    int rc = HEDDLE_OK;
    auto tensor = [&](const char *name, const void *p, const int64_t *st, bool keys, bool out = false) {
        if (rc || (keys ? k_all : q_all) == 0) return;
        const int64_t heads = keys ? d->kv_heads : d->heads;
        if (!p || ((uintptr_t)p & 1)) rc = fail(HEDDLE_E_INVAL, std::string(name) + " is NULL or not aligned to its values");
        else if ((heads > 1 && st[2] < d->dim) || ((keys ? d->k_len : d->q_len) > 1 && (st[1] < d->dim || st[1] > HEDDLE_MAX_LD)) ||
                 (!d->packed && d->sequences > 1 && st[0] < d->dim))
            rc = fail(HEDDLE_E_INVAL, std::string(name) + ": strides out of range");
        else if (out && runs_of(d, name, p, st, keys).over_itself()) rc = fail(HEDDLE_E_INVAL, std::string(name) + ": strides let its values overlap");
    };
    tensor("q", d->q, d->q_strides, false);
    tensor("k", d->k, d->k_strides, true);
    tensor("v", d->v, d->v_strides, true);
    tensor("y", d->y, d->y_strides, false, !backward);
    if (backward) {
        tensor("dy", d->dy, d->dy_strides, false);
        if (rc == HEDDLE_OK && !d->lse && q_all > 0) rc = fail(HEDDLE_E_INVAL, "lse is NULL");
        if (rc == HEDDLE_OK && !d->dk != !d->dv) rc = fail(HEDDLE_E_INVAL, "dk without dv, or dv without dk");
        if (d->dq) tensor("dq", d->dq, d->dq_strides, false, true);
        if (d->dk) tensor("dk", d->dk, d->dk_strides, true, true);
        if (d->dv) tensor("dv", d->dv, d->dv_strides, true, true);
    }
    return rc;
}

// Whether a value of b (its first n levels), which lies d values after a, is one of a's (its first m levels). Levels
// of one distance are taken apart together, by the difference of their indices: few come into question. Of others the
// larger one is, index by index: at most kLooks of them, past which tensors count as apart.
constexpr int kLooks = 4096;
static bool meet(const Runs &a, int m, const Runs &b, int n, Wide d, int &looks)
{
    if (d >= a.extent(m) || -d >= b.extent(n)) return false;
    if (m == 0 && n == 0) return true;
    const bool of_a = m && (!n || a.step[m - 1] >= b.step[n - 1]), of_b = n && (!m || b.step[n - 1] >= a.step[m - 1]);
    if (of_a) m--;
    if (of_b) n--;
    // d + q step, q = index in b - index in a, from the first that lies less than b's extent before a
    const Wide step = of_a ? a.step[m] : b.step[n], end = a.extent(m), least = 1 - b.extent(n) - d;
    Wide q = least / step + (least % step > 0);
    if (q < (of_a ? 1 - a.size[m] : 0)) q = of_a ? 1 - a.size[m] : 0;
    for (; q <= (of_b ? b.size[n] - 1 : 0) && d + q * step < end && looks > 0; q++) {
        looks--;
        if (meet(a, m, b, n, d + q * step, looks)) return true;
    }
    return false;
}

static int check_apart(const Runs &out, std::initializer_list<const Runs *> others)
{
    if (!out.p) return HEDDLE_OK;
    for (const Runs *r : others) {
        int looks = kLooks;
        if (r->p && meet(out, out.levels, *r, r->levels, ((intptr_t)r->p - (intptr_t)out.p) / 2, looks))
            return fail(HEDDLE_E_INVAL, std::string(out.name) + " overlaps " + r->name);
    }
    return HEDDLE_OK;
}

static int check_overlaps(const heddle_attention_desc *d, bool backward)
{
    const Runs q = runs_of(d, "q", d->q, d->q_strides, false), k = runs_of(d, "k", d->k, d->k_strides, true), v = runs_of(d, "v", d->v, d->v_strides, true);
    const Runs y = runs_of(d, "y", d->y, d->y_strides, false);
    const int64_t n = d->packed ? 1 : d->sequences, words = n * d->q_len * d->heads;
    const Runs lse = {"lse", words ? d->lse : nullptr, 2 * words, 0, {}, {}};
    int rc;
    if (!backward) {
        rc = check_apart(y, {&q, &k, &v, &lse});
        return rc ? rc : check_apart(lse, {&q, &k, &v});
    }
    const Runs dy = runs_of(d, "dy", d->dy, d->dy_strides, false), dq = runs_of(d, "dq", d->dq, d->dq_strides, false);
    const Runs dk = runs_of(d, "dk", d->dk, d->dk_strides, true), dv = runs_of(d, "dv", d->dv, d->dv_strides, true);
    rc = check_apart(dq, {&q, &k, &v, &y, &dy, &lse, &dk, &dv});
    if (rc == HEDDLE_OK) rc = check_apart(dk, {&q, &k, &v, &y, &dy, &lse, &dv});
    return rc ? rc : check_apart(dv, {&q, &k, &v, &y, &dy, &lse});
}

static int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, what);
}

// (the partial sums' rows lie on 8-byte boundaries: DP + 2 is even)
static void launch_combine(const heddle_attention_desc *d, const Args &a, int64_t blocks, int64_t tiles, hipStream_t stream)
{
    auto go = [&](auto t) {
        typedef decltype(t) T;
        if (d->dim <= 64) hipLaunchKernelGGL((combine_kernel<T, 64>), dim3((unsigned)(blocks * 8)), dim3(256), 0, stream, a, tiles);
        else hipLaunchKernelGGL((combine_kernel<T, 128>), dim3((unsigned)(blocks * 8)), dim3(256), 0, stream, a, tiles);
    };
    d->dtype == HEDDLE_T_BF16 ? go((__bf16)0.0f) : go((_Float16)0.0f);
}

static int forward(const heddle_attention_desc *d, mm::Scratch &s, bool run, hipStream_t stream)
{
    Args a = base_args(d);
    if (a.q_rows == 0) return HEDDLE_OK;
    a.out_vec = !((uintptr_t)d->y & 15) && !((a.y.seq | a.y.row | a.y.head | d->dim) & 7);
    if (d->sequences == 0) return run ? clear_all(d, a, false, stream) : HEDDLE_OK;
    Copies c;
    c.add(d, a.q, false, s);
    c.add(d, a.k, true, s);
    c.add(d, a.v, true, s);
    const ForwardPlan plan = plan_forward({d->sequences, a.q_rows, a.k_rows, d->heads, d->kv_heads});
    const int T = plan.rows;
    const int64_t slots = slots_of(d->packed, d->sequences, d->q_len, d->q_len, a.group, T), tiles = (d->q_len * a.group + T - 1) / T;
    const int64_t blocks = slots * d->kv_heads;
    a.parts = plan.parts;
    if (a.parts > 1) a.partial = (float *)s.take((size_t)blocks * 32 * a.parts * ((d->dim <= 64 ? 64 : 128) + 2) * 4);
    if (blocks * (a.parts > 1 ? std::max(a.parts, 8) : 1) > kMostBlocks) return fail(HEDDLE_E_RANGE, "more tiles than a launch holds");
    if (!run) return HEDDLE_OK;
    if (const int rc = c.launch(stream)) return rc;
    if (!plan.split) {
        launch_forward(d, a, T, blocks, stream);
    } else {
        // (in a launch of its own: with its code in split_kernel too, 32 sequences of up to 8192 keys took 130.2 us instead of 128.9)
        if (const int rc = clear_all(d, a, false, stream)) return rc;
        with_kind(d, [&](auto t, auto dp, auto mode) {
            typedef decltype(t) T;
            hipLaunchKernelGGL((split_kernel<T, dp, mode>), dim3((unsigned)(blocks * a.parts)), dim3(256), 0, stream, a, tiles);
        });
        if (a.parts > 1) launch_combine(d, a, blocks, tiles, stream);
    }
    return launched("attention");
}

static int run_attention(const heddle_attention_desc *d, bool back, void *ws, int64_t bytes, bool run, hipStream_t stream, int64_t *need)
{
    int rc = check(d, back);
    if (rc) return rc;
    for (int pass = 0; pass < 2; pass++) {
        mm::Scratch s = {pass ? (char *)ws : nullptr, 0};
        rc = back ? backward(d, s, pass == 1, stream) : forward(d, s, pass == 1, stream);
        if (rc) return rc;
        if (pass == 0) {
            if (need) *need = (int64_t)s.used;
            if (!run) return HEDDLE_OK;
            rc = mm::check_scratch(s.used, ws, bytes);
            if (rc == HEDDLE_OK) rc = check_overlaps(d, back);
            if (rc) return rc;
        }
    }
    return HEDDLE_OK;
}

}  // namespace attn
}  // namespace heddle

using namespace heddle;

extern "C" int heddle_attention(const heddle_attention_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return attn::run_attention(d, false, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_attention_backward(const heddle_attention_desc *d, void *ws, int64_t bytes, hipStream_t stream)
{
    return attn::run_attention(d, true, ws, bytes, true, stream, nullptr);
}

extern "C" int heddle_attention_workspace(const heddle_attention_desc *d, int32_t backward, int64_t *h_bytes)
{
    if (!h_bytes) return fail(HEDDLE_E_INVAL, "h_bytes is NULL");
    return attn::run_attention(d, backward != 0, nullptr, 0, false, nullptr, h_bytes);
}
