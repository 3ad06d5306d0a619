// Global gradient norm over many tensors, and clipping by it, on gfx950.
//
// norm = sqrt(sum over tensors of sum g^2); out = g min(1, max_norm / (norm + 1e-6)).
// Bound by memory: every value is read for the norm and read again, and
// written, for the clipping. The tensors' table goes to the kernels as an
// argument (kTensors a launch), so no copy to the device precedes them.
// A tensor is cut into chunks at 16-byte addresses; workgroup
// b of G takes chunks b, b + G, ... and leaves one fp64 sum. Squares are
// summed in fp64 throughout: fp32 squares overflow from 1.9e19, and at two
// fp64 operations a value the sums stay far below the vector units' rate. The
// clipping's workgroups each add up the at most kParts sums by themselves, in
// one order, which saves a launch between the two passes. 2e8 bf16 values: 74 + 137 us (5.4 and
// 5.9 TB/s); 1.6e9 values of 320 tensors: 1.96 ms (4.9 TB/s); 1e6 fp32 values: 4.3 + 6.2 us.
#include <cmath>

#include "heddle_internal.h"

namespace heddle {

constexpr int kTensors = 120, kParts = 2048;
// 16-byte pieces of a lane in a chunk: many to have their loads in flight, few where a call's
// tensors are too small to give every CU a large chunk (9 tensors of 1e6 fp32 values in all:
// both kernels 14.6 us with 8, 10.4 us with 2)
constexpr int kMany = 8, kFew = 2;
constexpr int64_t kSmallBytes = int64_t(32) << 20;
constexpr int64_t chunk_bytes(int pieces) { return (int64_t)pieces * 16 * 256; }

// one entry is half a cache line: the argument lies in host memory
struct GradEntry {
    const void *g;
    void *out;
    int64_t n;
    int32_t first, dtype;                     // first: the tensor's first chunk in the launch
};
struct GradTable {
    int32_t count, chunks;
    GradEntry t[kTensors];
};

// the tensor that holds chunk c
__device__ inline int tensor_of(const GradTable &t, int c)
{
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.t[mid].first <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Chunk c of a tensor, one 16-byte piece a lane at a time. A whole chunk's loads
// precede the first use, f(values, index of the first); at a tensor's ends
// the values come one by one, g(value, index). LAST: nothing reads the values again.
template <int kPieces, bool LAST, typename T, typename F, typename G> __device__ inline void each_of_chunk(const void *g, int64_t n, int64_t c, F f, G one)
{
    constexpr int V = 16 / sizeof(T);
    constexpr int64_t kChunk = chunk_bytes(kPieces);
    typedef T piece __attribute__((ext_vector_type(V)));
    const uintptr_t p = (uintptr_t)g;
    const int64_t skew = (int64_t)(p & 15) / (int64_t)sizeof(T);        // values before g in its first piece
    const T *base = (const T *)(p & ~(uintptr_t)15);
    const int64_t end = skew + n, v0 = c * (kChunk / (int64_t)sizeof(T)) + threadIdx.x * V;
    if ((c > 0 || skew == 0) && (c + 1) * (kChunk / (int64_t)sizeof(T)) <= end) {
        piece x[kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
            const piece *at = (const piece *)(base + v0 + i * 256 * V);
            x[i] = LAST ? __builtin_nontemporal_load(at) : *at;
        }
#pragma unroll
        for (int i = 0; i < kPieces; i++) f(x[i], v0 + i * 256 * V - skew);
        return;
    }
    for (int i = 0; i < kPieces; i++)
        for (int64_t v = v0 + i * 256 * V, j = 0; j < V; j++)
            if (v + j >= skew && v + j < end) one(base[v + j], v + j - skew);
}

template <int PIECES, typename T> __device__ inline double chunk_squares(const void *g, int64_t n, int64_t c)
{
    double s = 0;
    auto add = [&](float v) { s = fma((double)v, (double)v, s); };
    each_of_chunk<PIECES, false, T>(g, n, c, [&](auto x, int64_t) {
#pragma unroll
        for (int i = 0; i < 16 / (int)sizeof(T); i++) add((float)x[i]);
    }, [&](T x, int64_t) { add((float)x); });
    return s;
}

// sum over the workgroup's 256 lanes, in a fixed order, in every lane
__device__ inline double block_sum(double s, double *lds)
{
#pragma unroll
    for (int d = 32; d; d /= 2) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    __syncthreads();
    return s;
}

// held: sums that earlier launches left
template <int PIECES> __global__ void __launch_bounds__(256) grad_squares_kernel(GradTable t, double *parts, int held)
{
    __shared__ double lds[4];
    double s = 0;
    int k = -1;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        if (k < 0) k = tensor_of(t, c);
        while (k + 1 < t.count && c >= t.t[k + 1].first) k++;
        const GradEntry &e = t.t[k];
        const int64_t local = c - e.first;
        if (e.dtype == HEDDLE_T_BF16) s += chunk_squares<PIECES, __bf16>(e.g, e.n, local);
        else if (e.dtype == HEDDLE_T_F16) s += chunk_squares<PIECES, _Float16>(e.g, e.n, local);
        else s += chunk_squares<PIECES, float>(e.g, e.n, local);
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) parts[blockIdx.x] = (int)blockIdx.x < held ? parts[blockIdx.x] + s : s;
}

__device__ inline float norm_of(const double *parts, int count, double *lds)
{
    double s = 0;
    for (int i = threadIdx.x; i < count; i += 256) s += parts[i];
    return (float)sqrt(block_sum(s, lds));
}

__global__ void __launch_bounds__(256) grad_norm_kernel(const double *parts, int count, float *norm)
{
    __shared__ double lds[4];
    const float v = norm_of(parts, count, lds);
    if (threadIdx.x == 0) *norm = v;
}

template <int PIECES, typename T>
__device__ inline void clip_chunk(const void *g, void *out, int64_t n, int64_t c, float factor)
{
    typedef T aligned __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));   // out may start anywhere its values may
    each_of_chunk<PIECES, true, T>(g, n, c, [&](auto x, int64_t at) {
#pragma unroll
        for (int i = 0; i < 16 / (int)sizeof(T); i++) x[i] = (T)((float)x[i] * factor);
        __builtin_nontemporal_store(x, (aligned *)((T *)out + at));
    }, [&](T x, int64_t at) { ((T *)out)[at] = (T)((float)x * factor); });
}

// The factor from d_norm, or from the parts (then the first workgroup of the
// first launch writes the norm).
template <int PIECES>
__global__ void __launch_bounds__(256) clip_kernel(GradTable t, const double *parts, int count, float *norm, int write, float max_norm)
{
    __shared__ double lds[4];
    float v;
    if (parts) {
        v = norm_of(parts, count, lds);
        if (write && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
    } else {
        v = *norm;
    }
    float factor = max_norm / (v + 1e-6f);
    if (factor >= 1.0f) factor = 1.0f;                                  // a NaN stays
    // The table runs from the last tensor to the first, and so do a tensor's chunks here: what
    // the norm read last is still in the 256 MB memory-side cache. It keeps what is still to be
    // read, as this pass reads and writes past the caches (2e8 bf16 values, both passes: 249 us
    // without, 210 us; 1.6e9: 2003 and 1970 us).
    int k = -1;
    for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        if (k < 0) k = tensor_of(t, c);
        while (k + 1 < t.count && c >= t.t[k + 1].first) k++;
        const GradEntry &e = t.t[k];
        if (factor == 1.0f && e.out == e.g) continue;
        const int64_t local = (k + 1 < t.count ? t.t[k + 1].first : t.chunks) - 1 - c;
        if (e.dtype == HEDDLE_T_BF16) clip_chunk<PIECES, __bf16>(e.g, e.out, e.n, local, factor);
        else if (e.dtype == HEDDLE_T_F16) clip_chunk<PIECES, _Float16>(e.g, e.out, e.n, local, factor);
        else clip_chunk<PIECES, float>(e.g, e.out, e.n, local, factor);
    }
}

static int64_t bytes_of(const heddle_grad_desc &g) { return g.n * (g.dtype == HEDDLE_T_F32 ? 4 : 2); }

static int check_grads(const heddle_grad_desc *g, int32_t count)
{
    if (count < 0) return fail(HEDDLE_E_INVAL, "count < 0");
    if (count > 0 && !g) return fail(HEDDLE_E_INVAL, "grads is NULL");
    for (int32_t i = 0; i < count; i++) {
        if (g[i].dtype != HEDDLE_T_BF16 && g[i].dtype != HEDDLE_T_F16 && g[i].dtype != HEDDLE_T_F32)
            return fail(HEDDLE_E_INVAL, "unknown dtype of a gradient tensor");
        const uintptr_t mask = g[i].dtype == HEDDLE_T_F32 ? 3 : 1;
        if (g[i].n < 0 || g[i].n > (int64_t(1) << 40)) return fail(HEDDLE_E_INVAL, "size of a gradient tensor out of range");
        if (g[i].n > 0 && !g[i].g) return fail(HEDDLE_E_INVAL, "a gradient tensor is NULL");
        if (((uintptr_t)g[i].g | (uintptr_t)g[i].out) & mask)
            return fail(HEDDLE_E_INVAL, "a gradient tensor is not aligned to its values");
        const uintptr_t from = (uintptr_t)g[i].g, to = (uintptr_t)g[i].out, bytes = (uintptr_t)bytes_of(g[i]);
        if (to && to != from && (to > from ? to - from : from - to) < bytes)
            return fail(HEDDLE_E_INVAL, "a gradient tensor's output overlaps it");
    }
    return HEDDLE_OK;
}

static bool is_small(const heddle_grad_desc *g, int32_t count)
{
    int64_t all = 0;
    for (int32_t i = 0; i < count; i++) all += bytes_of(g[i]);
    return all < kSmallBytes;
}

// tables of up to kTensors tensors (and 2^30 chunks) each, from the first tensor or from
// the last; f(table) launches
template <typename F> static int each_table(const heddle_grad_desc *g, int32_t count, bool small, bool backward, F f)
{
    const int64_t chunk = chunk_bytes(small ? kFew : kMany);
    int32_t done = 0;
    do {
        GradTable t;
        t.count = t.chunks = 0;
        for (; done < count && t.count < kTensors; done++) {
            const heddle_grad_desc &d = g[backward ? count - 1 - done : done];
            if (d.n == 0) continue;
            const int64_t c = ((int64_t)((uintptr_t)d.g & 15) + bytes_of(d) + chunk - 1) / chunk;
            if (t.chunks + c > (int64_t(1) << 30)) break;
            t.t[t.count++] = {d.g, d.out ? d.out : const_cast<void *>(d.g), d.n, t.chunks, d.dtype};
            t.chunks += (int32_t)c;
        }
        const int rc = f(t);
        if (rc) return rc;
    } while (done < count);
    return HEDDLE_OK;
}

static int check_parts(const void *ws, int64_t bytes)
{
    if (!ws || ((uintptr_t)ws & 255)) return fail(HEDDLE_E_INVAL, "workspace is NULL or not 256-byte aligned");
    if (bytes < (int64_t)kParts * 8) return fail(HEDDLE_E_INVAL, "workspace smaller than the call needs");
    return HEDDLE_OK;
}

// the sums of squares; *parts: how many
static int launch_squares(const heddle_grad_desc *g, int32_t count, double *ws, int *parts, hipStream_t stream)
{
    const bool small = is_small(g, count);
    *parts = 0;
    return each_table(g, count, small, false, [&](const GradTable &t) {
        const int blocks = t.chunks < 1 ? 1 : t.chunks < kParts ? t.chunks : kParts;
        auto kernel = small ? grad_squares_kernel<kFew> : grad_squares_kernel<kMany>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, t, ws, *parts);
        if (blocks > *parts) *parts = blocks;
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "grad_squares_kernel");
    });
}

static int launch_clip(const heddle_grad_desc *g, int32_t count, const double *parts, int n_parts, float *norm, float max_norm,
                       hipStream_t stream)
{
    const bool small = is_small(g, count);
    int write = 1;
    return each_table(g, count, small, true, [&](const GradTable &t) {
        const int blocks = t.chunks < 1 ? 1 : t.chunks < kParts ? t.chunks : kParts;
        auto kernel = small ? clip_kernel<kFew> : clip_kernel<kMany>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, t, parts, n_parts, norm, write, max_norm);
        write = 0;
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "clip_kernel");
    });
}

static int check_max_norm(float max_norm)
{
    return std::isfinite(max_norm) && max_norm > 0 ? HEDDLE_OK : fail(HEDDLE_E_INVAL, "max_norm is not finite and > 0");
}

}  // namespace heddle

using namespace heddle;

extern "C" int heddle_grad_norm_workspace(const heddle_grad_desc *grads, int32_t count, int64_t *h_bytes)
{
    if (!h_bytes) return fail(HEDDLE_E_INVAL, "h_bytes is NULL");
    const int rc = check_grads(grads, count);
    if (rc) return rc;
    *h_bytes = (int64_t)kParts * 8;
    return HEDDLE_OK;
}

extern "C" int heddle_grad_norm(const heddle_grad_desc *grads, int32_t count, float *d_norm, void *ws, int64_t bytes,
                                hipStream_t stream)
{
    int rc = check_grads(grads, count);
    if (rc) return rc;
    if (!d_norm || ((uintptr_t)d_norm & 3)) return fail(HEDDLE_E_INVAL, "d_norm is NULL or misaligned");
    rc = check_parts(ws, bytes);
    if (rc) return rc;
    int parts = 0;
    rc = launch_squares(grads, count, (double *)ws, &parts, stream);
    if (rc) return rc;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, stream, (const double *)ws, parts, d_norm);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HEDDLE_OK : hip_fail(e, "grad_norm_kernel");
}

extern "C" int heddle_clip_grads(const heddle_grad_desc *grads, int32_t count, const float *d_norm, float max_norm,
                                 hipStream_t stream)
{
    int rc = check_grads(grads, count);
    if (rc) return rc;
    if (!d_norm || ((uintptr_t)d_norm & 3)) return fail(HEDDLE_E_INVAL, "d_norm is NULL or misaligned");
    rc = check_max_norm(max_norm);
    if (rc) return rc;
    return launch_clip(grads, count, nullptr, 0, const_cast<float *>(d_norm), max_norm, stream);
}

extern "C" int heddle_clip_grad_norm(const heddle_grad_desc *grads, int32_t count, float max_norm, float *d_norm, void *ws,
                                     int64_t bytes, hipStream_t stream)
{
    int rc = check_grads(grads, count);
    if (rc) return rc;
    if (!d_norm || ((uintptr_t)d_norm & 3)) return fail(HEDDLE_E_INVAL, "d_norm is NULL or misaligned");
    rc = check_max_norm(max_norm);
    if (rc) return rc;
    rc = check_parts(ws, bytes);
    if (rc) return rc;
    int parts = 0;
    rc = launch_squares(grads, count, (double *)ws, &parts, stream);
    if (rc) return rc;
    return launch_clip(grads, count, (const double *)ws, parts, d_norm, max_norm, stream);
}
