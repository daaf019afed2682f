// grace_grad_norm, grace_clip_grads, grace_clip_grad_norm: the global 2-norm of many gradients, and their scaling by it.
//
// norm = sqrt(sum over all tensors of x^2); scale = 1 where norm <= max_norm, else max_norm / norm.
// Squares and sums are in 64 bits: bf16 and fp32 squares are exact there, do not overflow and do not vanish, and the conversions hide behind HBM.
// The tensors are cut into chunks, chunk c goes to workgroup c mod the grid, each of which leaves one sum; they are added up in a fixed order, so
// the norm is the same in every run.  The tensors' addresses travel as kernel arguments: nothing is copied to the device, and a captured
// launch keeps them.
#include <cmath>
#include <memory>
#include <new>

#include "bf16.h"
#include "common.h"

namespace grace {
namespace norm {

constexpr int MAX_TENSORS = 112;     // of one launch: 32 bytes each in 4 KB of kernel arguments
constexpr int FEW_TENSORS = 32;      // a launch copies its arguments: clipping of 30 tensors, 1 KB of them, 10.6 us a call; 3.6 KB 10.9
constexpr int MAX_GROUPS = 2048;     // workgroups of a launch, so partial sums it leaves
constexpr int THREADS = 256;

struct Tensor {
    const void *in;
    void *out;                 // scaled values (clipping)
    int64_t numel;
    int32_t first_chunk, bf16;
};
template <int MOST>
struct Tensors {
    Tensor t[MOST];
    int32_t n, chunks, chunk;  // chunk: elements of one, a multiple of 2048
};
static_assert(sizeof(Tensors<MAX_TENSORS>) + 64 <= 4096, "kernel arguments");

// Tensor that holds chunk c: as many as begin at or before it, less one.  A lane looks at two of them: one round of loads.
template <int MOST>
__device__ __forceinline__ int tensor_of(const Tensors<MOST> &a, int c) {
    static_assert(MOST <= 128, "two of a lane");
    const int lane = (int)threadIdx.x & 63;
    const bool low = lane < a.n && a.t[lane].first_chunk <= c, high = MOST > 64 && lane + 64 < a.n && a.t[lane + 64].first_chunk <= c;
    return __popcll(__ballot(low)) + __popcll(__ballot(high)) - 1;
}

// Elements of T ahead of the first 16-byte boundary.
template <typename T>
__device__ __forceinline__ int64_t elements_to_boundary(const T *p) { return (int64_t)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T)); }

__device__ __forceinline__ float to_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ uint16_t from_f32(float v, uint16_t) { return (uint16_t)f32_to_bf16_bits(v); }
__device__ __forceinline__ float from_f32(float v, float) { return v; }
template <typename T>
__device__ __forceinline__ void unpack(const uint4 &v, float *f) {
    if constexpr (sizeof(T) == 2) unpack_bf16x8(v, f); else unpack_f32x4(v, f);
}

// Sum over the workgroup, in every thread.
__device__ __forceinline__ double block_sum(double v, double *lds) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
    return s;
}

constexpr int AHEAD = 4;   // 16-byte loads of a thread in flight

template <typename T>
__device__ __forceinline__ double square_sum(const T *p, int64_t n) {
    constexpr int NV = 16 / sizeof(T);
    double sum[2] = {0.0, 0.0};
    const int64_t head = min(n, elements_to_boundary(p)), vecs = (n - head) / NV;
    const uint4 *v = (const uint4 *)(p + head);
    int64_t i = threadIdx.x;
    for (; i + (AHEAD - 1) * THREADS < vecs; i += AHEAD * THREADS) {
        uint4 x[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) x[q] = v[i + q * THREADS];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            float f[NV];
            unpack<T>(x[q], f);
#pragma unroll
            for (int e = 0; e < NV; ++e) sum[e & 1] = fma((double)f[e], (double)f[e], sum[e & 1]);
        }
    }
    for (; i < vecs; i += THREADS) {
        float f[NV];
        unpack<T>(v[i], f);
#pragma unroll
        for (int e = 0; e < NV; ++e) sum[e & 1] = fma((double)f[e], (double)f[e], sum[e & 1]);
    }
    // (fewer than a vector on either side)
    const int64_t tail = head + vecs * NV;
    if ((int64_t)threadIdx.x < head) { const double x = to_f32(p[threadIdx.x]); sum[0] = fma(x, x, sum[0]); }
    if (tail + (int64_t)threadIdx.x < n) { const double x = to_f32(p[tail + threadIdx.x]); sum[1] = fma(x, x, sum[1]); }
    return sum[0] + sum[1];
}

template <int MOST>
__global__ __launch_bounds__(THREADS) void square_sum_kernel(const Tensors<MOST> a, double *__restrict__ partial) {
    __shared__ double lds[THREADS / 64];
    double sum = 0.0;
    for (int c = (int)blockIdx.x; c < a.chunks; c += (int)gridDim.x) {
        const Tensor t = a.t[tensor_of(a, c)];
        const int64_t e0 = (int64_t)(c - t.first_chunk) * a.chunk, n = min((int64_t)a.chunk, t.numel - e0);
        sum += t.bf16 ? square_sum((const uint16_t *)t.in + e0, n) : square_sum((const float *)t.in + e0, n);
    }
    sum = block_sum(sum, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// The norm from the partial sums, in every thread of the workgroup.
__device__ __forceinline__ float norm_of(const double *__restrict__ partial, int n, double *lds) {
    double sum = 0.0;
    for (int i = (int)threadIdx.x; i < n; i += THREADS) sum += partial[i];
    return (float)sqrt(block_sum(sum, lds));
}

__global__ __launch_bounds__(THREADS) void norm_kernel(const double *__restrict__ partial, int n, float *__restrict__ norm) {
    __shared__ double lds[THREADS / 64];
    const float v = norm_of(partial, n, lds);
    if (threadIdx.x == 0) *norm = v;
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const T *p, T *out, int64_t n, float scale) {
    constexpr int NV = 16 / sizeof(T);
    if (((uintptr_t)p ^ (uintptr_t)out) & 15) {   // no vectors that are whole on both sides
        for (int64_t i = threadIdx.x; i < n; i += THREADS) out[i] = from_f32(to_f32(p[i]) * scale, T());
        return;
    }
    const int64_t head = min(n, elements_to_boundary(p)), vecs = (n - head) / NV;
    const uint4 *v = (const uint4 *)(p + head);
    uint4 *o = (uint4 *)(out + head);
    auto scaled = [&](const uint4 &x) {
        float f[NV];
        unpack<T>(x, f);
#pragma unroll
        for (int e = 0; e < NV; ++e) f[e] *= scale;
        if constexpr (sizeof(T) == 2) return pack_bf16x8(f); else return pack_f32x4(f);
    };
    int64_t i = threadIdx.x;
    for (; i + (AHEAD - 1) * THREADS < vecs; i += AHEAD * THREADS) {
        uint4 x[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) x[q] = v[i + q * THREADS];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) nt_store16(scaled(x[q]), o + i + q * THREADS);
    }
    for (; i < vecs; i += THREADS) nt_store16(scaled(v[i]), o + i);
    const int64_t tail = head + vecs * NV;
    if ((int64_t)threadIdx.x < head) out[threadIdx.x] = from_f32(to_f32(p[threadIdx.x]) * scale, T());
    if (tail + (int64_t)threadIdx.x < n) out[tail + threadIdx.x] = from_f32(to_f32(p[tail + threadIdx.x]) * scale, T());
}

// norm: of all gradients; or null, then it is made of n_partial sums here and kept in norm_out.
template <int MOST>
__global__ __launch_bounds__(THREADS) void clip_kernel(const Tensors<MOST> a, const float *norm, const double *__restrict__ partial, int n_partial,
                                                       float max_norm, float *norm_out) {
    __shared__ double lds[THREADS / 64];
    const float v = norm ? *norm : norm_of(partial, n_partial, lds);
    if (!norm && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = v;
    const float scale = v <= max_norm ? 1.0f : max_norm / v;   // (a norm that is NaN scales by NaN)
    // from the last chunk to the first: the ones read last for the norm are in the caches still (403 M elements in 20 tensors, both kernels 473 ->
    // 457 us, 438 with stores that bypass the caches; the bytes at the rate of a large copy 480)
    for (int b = (int)blockIdx.x; b < a.chunks; b += (int)gridDim.x) {
        const int c = a.chunks - 1 - b;
        const Tensor t = a.t[tensor_of(a, c)];
        if (scale == 1.0f && t.in == t.out) continue;          // nothing to change in place
        const int64_t e0 = (int64_t)(c - t.first_chunk) * a.chunk, n = min((int64_t)a.chunk, t.numel - e0);
        if (t.bf16) scale_chunk((const uint16_t *)t.in + e0, (uint16_t *)t.out + e0, n, scale);
        else scale_chunk((const float *)t.in + e0, (float *)t.out + e0, n, scale);
    }
}

// Elements of a chunk: 2048 (one round of a workgroup in bf16), more where there would be many times as many chunks as workgroups.
static int chunk_elements(const int64_t *numel, int32_t n) {
    int64_t total = 0;
    for (int i = 0; i < n; ++i) total += numel[i];
    int64_t chunk = 2048;
    while (chunk < 32768 && total / chunk > 4 * MAX_GROUPS) chunk *= 2;
    while (total / chunk > (int64_t)INT32_MAX / 4) chunk *= 2;   // chunk numbers in 32 bits
    return chunk > INT32_MAX / 2 ? 0 : (int)chunk;
}

static int check(const char *who, const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n) {
    if (n < 0) return fail(GRACE_EINVAL, "%s: n=%d invalid", who, n);
    if (n > 0 && (!grads || !numel || !dtypes)) return fail(GRACE_EINVAL, "%s: null host pointer", who);
    for (int i = 0; i < n; ++i) {
        if (numel[i] < 0 || numel[i] > ((int64_t)1 << 40)) return fail(GRACE_EINVAL, "%s: gradient %d: %lld elements", who, i, (long long)numel[i]);
        if (dtypes[i] != GRACE_F32 && dtypes[i] != GRACE_BF16) return fail(GRACE_EINVAL, "%s: gradient %d: unknown dtype %d", who, i, dtypes[i]);
        if (numel[i] > 0 && !grads[i]) return fail(GRACE_EINVAL, "%s: gradient %d: null device pointer", who, i);
        if ((uintptr_t)grads[i] % (dtypes[i] == GRACE_F32 ? 4 : 2))
            return fail(GRACE_EINVAL, "%s: gradient %d is not aligned to its elements", who, i);
    }
    return GRACE_OK;
}

// Memory of a call: what is written has to be apart from everything else, or workgroups would read and scale the same values in any order.
struct Range {
    uintptr_t begin, end;
    int32_t index;             // of the gradient or output, -1: norm or workspace
    bool written;
};

// No written range may meet another.  In order of their beginnings a range meets one ahead of it where the latter's end is past its beginning.
static int check_apart(const char *who, Range *r, size_t n) {
    std::sort(r, r + n, [](const Range &a, const Range &b) { return a.begin < b.begin; });
    uintptr_t any_end = 0, written_end = 0;
    for (size_t i = 0; i < n; ++i) {
        if (r[i].begin < (r[i].written ? any_end : written_end))
            return r[i].index < 0 ? fail(GRACE_EINVAL, "%s: norm or workspace overlaps a gradient or output", who)
                                  : fail(GRACE_EINVAL, "%s: %s %d overlaps other memory of the call", who, r[i].written ? "output" : "gradient", r[i].index);
        any_end = std::max(any_end, r[i].end);
        if (r[i].written) written_end = std::max(written_end, r[i].end);
    }
    return GRACE_OK;
}

// ws: null where the call has none and reads the norm, else the norm is written.
static int check_outputs(const char *who, const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n, void *const *out,
                         float max_norm, const float *norm, const void *ws) {
    if (!(max_norm >= 0.0f) || std::isinf(max_norm)) return fail(GRACE_EINVAL, "%s: max_norm=%g invalid", who, (double)max_norm);
    if (n > 0 && !out) return fail(GRACE_EINVAL, "%s: null host pointer", who);
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const uintptr_t el = dtypes[i] == GRACE_F32 ? 4 : 2, a = (uintptr_t)grads[i], b = (uintptr_t)out[i], bytes = (uintptr_t)numel[i] * el;
        if (!out[i]) return fail(GRACE_EINVAL, "%s: output %d: null device pointer", who, i);
        if (b % el) return fail(GRACE_EINVAL, "%s: output %d is not aligned to its elements", who, i);
        if (a != b && a < b + bytes && b < a + bytes) return fail(GRACE_EINVAL, "%s: output %d overlaps its gradient in part", who, i);
    }
    Range few[2 * FEW_TENSORS + 2];
    std::unique_ptr<Range[]> many;
    if (n > FEW_TENSORS) many.reset(new (std::nothrow) Range[2 * (size_t)n + 2]);
    Range *const r = n > FEW_TENSORS ? many.get() : few;
    if (!r) return fail(GRACE_ENOMEM, "%s: no host memory for %d gradients", who, n);
    size_t count = 0;
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const uintptr_t a = (uintptr_t)grads[i], b = (uintptr_t)out[i], bytes = (uintptr_t)numel[i] * (dtypes[i] == GRACE_F32 ? 4 : 2);
        r[count++] = Range{b, b + bytes, i, true};
        if (a != b) r[count++] = Range{a, a + bytes, i, false};
    }
    r[count++] = Range{(uintptr_t)norm, (uintptr_t)norm + sizeof(float), -1, ws != nullptr};
    if (ws) r[count++] = Range{(uintptr_t)ws, (uintptr_t)ws + grace_grad_norm_workspace_bytes(n), -1, true};
    return check_apart(who, r, count);
}

template <typename F>
static int sized(const Tensors<MAX_TENSORS> &a, int launch, F take) {
    if (a.n > FEW_TENSORS) return take(a, launch);
    Tensors<FEW_TENSORS> few;
    std::copy(a.t, a.t + a.n, few.t);
    few.n = a.n;
    few.chunks = a.chunks;
    few.chunk = a.chunk;
    return take(few, launch);
}

// Calls take(tensors, launch number) for every MAX_TENSORS of the tensors that hold anything (at least once: the sums of none are zero).
template <typename F>
static int for_launches(const void *const *grads, void *const *out, const int64_t *numel, const int32_t *dtypes, int32_t n, int chunk, F take) {
    Tensors<MAX_TENSORS> a;
    a.n = 0;
    a.chunks = 0;
    a.chunk = chunk;
    int launches = 0;
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const int64_t chunks = ceil_div(numel[i], chunk);
        a.t[a.n++] = Tensor{grads[i], out ? out[i] : nullptr, numel[i], a.chunks, dtypes[i] == GRACE_BF16};
        a.chunks += (int32_t)chunks;
        if (a.n == MAX_TENSORS) {
            const int rc = sized(a, launches++, take);
            if (rc != GRACE_OK) return rc;
            a.n = 0;
            a.chunks = 0;
        }
    }
    return a.n > 0 || launches == 0 ? sized(a, launches, take) : GRACE_OK;
}

template <int MOST>
static unsigned groups_of(const Tensors<MOST> &a) { return (unsigned)std::max(1, std::min(a.chunks, MAX_GROUPS)); }

// Partial sums of all tensors -> how many there are.
static int square_sums(const char *who, const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n, int chunk, double *partial,
                       hipStream_t st, int &n_partial) {
    n_partial = 0;
    return for_launches(grads, nullptr, numel, dtypes, n, chunk, [&](const auto &a, int) {
        const unsigned groups = groups_of(a);
        square_sum_kernel<<<groups, THREADS, 0, st>>>(a, partial + n_partial);
        n_partial += (int)groups;
        GRACE_LAUNCH_CHECK(who);
        return (int)GRACE_OK;
    });
}

}  // namespace norm
}  // namespace grace

using namespace grace;

extern "C" size_t grace_grad_norm_workspace_bytes(int32_t n) {
    if (n < 0) return 0;
    return (size_t)std::max<int64_t>(1, ceil_div(n, norm::MAX_TENSORS)) * norm::MAX_GROUPS * sizeof(double);
}

extern "C" int grace_grad_norm(const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n, float *norm_out, void *ws,
                               void *stream) {
    int rc = norm::check("grad_norm", grads, numel, dtypes, n);
    if (rc != GRACE_OK) return rc;
    if (!norm_out || !ws || ((uintptr_t)ws & 7) || ((uintptr_t)norm_out & 3)) return fail(GRACE_EINVAL, "grad_norm: null or unaligned device pointer");
    const int chunk = norm::chunk_elements(numel, n);
    if (chunk == 0) return fail(GRACE_ESHAPE, "grad_norm: too many elements");
    int n_partial;
    rc = norm::square_sums("grad_norm", grads, numel, dtypes, n, chunk, (double *)ws, (hipStream_t)stream, n_partial);
    if (rc != GRACE_OK) return rc;
    norm::norm_kernel<<<1, norm::THREADS, 0, (hipStream_t)stream>>>((const double *)ws, n_partial, norm_out);
    GRACE_LAUNCH_CHECK("grad_norm");
    return GRACE_OK;
}

extern "C" int grace_clip_grads(const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n, const float *norm_in,
                                float max_norm, void *const *out, void *stream) {
    int rc = norm::check("clip_grads", grads, numel, dtypes, n);
    if (rc != GRACE_OK) return rc;
    if (!norm_in || ((uintptr_t)norm_in & 3)) return fail(GRACE_EINVAL, "clip_grads: null or unaligned device pointer");
    rc = norm::check_outputs("clip_grads", grads, numel, dtypes, n, out, max_norm, norm_in, nullptr);
    if (rc != GRACE_OK) return rc;
    const int chunk = norm::chunk_elements(numel, n);
    if (chunk == 0) return fail(GRACE_ESHAPE, "clip_grads: too many elements");
    return norm::for_launches(grads, out, numel, dtypes, n, chunk, [&](const auto &a, int) {
        if (a.chunks == 0) return (int)GRACE_OK;
        norm::clip_kernel<<<norm::groups_of(a), norm::THREADS, 0, (hipStream_t)stream>>>(a, norm_in, nullptr, 0, max_norm, nullptr);
        GRACE_LAUNCH_CHECK("clip_grads");
        return (int)GRACE_OK;
    });
}

extern "C" int grace_clip_grad_norm(const void *const *grads, const int64_t *numel, const int32_t *dtypes, int32_t n, float max_norm,
                                    void *const *out, float *norm_out, void *ws, void *stream) {
    int rc = norm::check("clip_grad_norm", grads, numel, dtypes, n);
    if (rc != GRACE_OK) return rc;
    if (!norm_out || !ws || ((uintptr_t)ws & 7) || ((uintptr_t)norm_out & 3))
        return fail(GRACE_EINVAL, "clip_grad_norm: null or unaligned device pointer");
    rc = norm::check_outputs("clip_grad_norm", grads, numel, dtypes, n, out, max_norm, norm_out, ws);
    if (rc != GRACE_OK) return rc;
    const int chunk = norm::chunk_elements(numel, n);
    if (chunk == 0) return fail(GRACE_ESHAPE, "clip_grad_norm: too many elements");
    hipStream_t st = (hipStream_t)stream;
    int n_partial;
    rc = norm::square_sums("clip_grad_norm", grads, numel, dtypes, n, chunk, (double *)ws, st, n_partial);
    if (rc != GRACE_OK) return rc;
    // the norm is made by every workgroup of the first scaling launch; further launches read it
    return norm::for_launches(grads, out, numel, dtypes, n, chunk, [&](const auto &a, int launch) {
        norm::clip_kernel<<<norm::groups_of(a), norm::THREADS, 0, st>>>(a, launch == 0 ? nullptr : norm_out, (const double *)ws, n_partial, max_norm,
                                                                       norm_out);
        GRACE_LAUNCH_CHECK("clip_grad_norm");
        return (int)GRACE_OK;
    });
}
