// grace_combine_backward, grace_permute_backward: gradients of the rows' two ways, from the experts back to the tokens (the weighted
// aggregation, Section 1) and from the tokens to the experts (the dispatch, Section 5).
#include "bf16.h"
#include "common.h"
#include "gemm_common.h"

namespace grace {

// Rows [lo, hi) of the buffer of n rows that a call is about: all, or those of one rank.
__device__ __forceinline__ void row_range(const int32_t *__restrict__ rank_off, int rank, int64_t n, int &lo, int &hi) {
    lo = 0;
    hi = (int)n;
    if (rank_off) {
        lo = max(0, rank_off[rank]);
        hi = min(hi, rank_off[rank + 1]);
    }
}

// out[t] = sum_j w[t,j] y[p(t,j)]:  dy[p(t,j)] = w[t,j] dout[t],  dw[t,j] = <dout[t], y[p(t,j)]>.
// A wavefront takes the choices part, part + parts, ... of a token: the token's k positions lie in its lanes, a ballot gives the choices whose row is
// in range, and the token's gradient stays in registers (VPL 16-byte vectors a lane) while its rows pass; of rows wider than that it is read again for every
// row (from the caches).  The sum over a row is each lane's in ascending order, then a tree over the lanes: the same in every run.
// dy may be y: a row's vectors are all read ahead of the stores to them, an order that the compiler keeps because neither pointer is __restrict__.
// Bound by HBM, each row read and written once: 16384 tokens, 8 choices, rows of 4 KB 216 us, 5.3 TB/s (a large copy reaches 5.0); 64 tokens 3.7 us.
template <bool BF16, int VPL>
__global__ __launch_bounds__(256) void combine_backward_kernel(const uint4 *__restrict__ dout, const uint4 *y,
                                                               const int32_t *__restrict__ perm_pos, const float *__restrict__ weight, int64_t T,
                                                               int k, int row_vec, const int32_t *__restrict__ rank_off, int rank, int parts,
                                                               uint4 *dy, float *__restrict__ dweight) {
    constexpr int NV = BF16 ? 8 : 4;   // values per vector
    const int lane = (int)threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t t = unit / parts;
    const int part = (int)(unit - t * parts);
    if (t >= T) return;
    int lo, hi;
    row_range(rank_off, rank, T * k, lo, hi);
    const int chunks = (row_vec + 64 * VPL - 1) / (64 * VPL);
    uint4 g[VPL];
    auto load_gradient = [&](int c0) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int c = c0 + i * 64 + lane;
            g[i] = c < row_vec ? dout[t * row_vec + c] : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    if (chunks == 1) load_gradient(0);
    for (int j0 = 0; j0 < k; j0 += 64) {   // 64 choices at a time
        const int j = j0 + lane;
        const bool mine = j < k && j % parts == part;
        const int64_t a = t * k + min(j, k - 1);
        const int32_t p_lane = perm_pos[a];
        const float w_lane = weight[a];
        uint64_t todo = __ballot(mine && p_lane >= lo && p_lane < hi);
        float dw_lane = 0.0f;
        while (todo) {
            const int src = __builtin_ctzll(todo);
            todo &= todo - 1;
            const int64_t row = (int64_t)__builtin_amdgcn_readlane(p_lane, src) * row_vec;
            const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w_lane), src));
            float dot = 0.0f;
            for (int c0 = 0; c0 < row_vec; c0 += 64 * VPL) {
                if (chunks > 1) load_gradient(c0);
                uint4 v[VPL];
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    const int c = c0 + i * 64 + lane;
                    v[i] = c < row_vec ? nt_load16(y + row + c) : make_uint4(0u, 0u, 0u, 0u);
                }
#pragma unroll
                for (int i = 0; i < VPL; ++i) {
                    const int c = c0 + i * 64 + lane;
                    float fg[NV], fy[NV];
                    if constexpr (BF16) { unpack_bf16x8(g[i], fg); unpack_bf16x8(v[i], fy); } else { unpack_f32x4(g[i], fg); unpack_f32x4(v[i], fy); }
#pragma unroll
                    for (int e = 0; e < NV; ++e) {
                        dot = fmaf(fg[e], fy[e], dot);
                        fg[e] *= w;
                    }
                    if (c < row_vec) {
                        if constexpr (BF16) nt_store16(pack_bf16x8(fg), dy + row + c); else nt_store16(pack_f32x4(fg), dy + row + c);
                    }
                }
            }
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) dot += __shfl_xor(dot, o, 64);
            if (lane == src) dw_lane = dot;
        }
        if (mine) dweight[t * k + j] = dw_lane;
    }
}

// xp[p(t,j)] = x[t]:  dx[t] = sum_j dxp[p(t,j)] (+ dx_shared[t]), in fp32 in ascending j, rounded once.
// A wavefront takes 64 vectors of a token's row (consecutive wavefronts consecutive parts of it); positions and ballot as above, two
// rows in flight (16384 tokens, one choice 25.3 us, 29.2 with four in flight; 8 choices the same).  A surplus load has a descriptor without records,
// reads nothing and gives zeros.  Bound by HBM: 16384 tokens, 8 choices, rows of 4 KB 104 us, 5.8 TB/s; 64 tokens 3.6 us.
// dx may be dx_shared, so neither is __restrict__.
template <bool BF16>
__global__ __launch_bounds__(256) void permute_backward_kernel(const char *__restrict__ dxp, const int32_t *__restrict__ perm_pos, int64_t T, int k,
                                                               int row_vec, int pieces, const int32_t *__restrict__ rank_off, int rank,
                                                               const uint4 *dx_shared, uint4 *dx) {
    constexpr int NV = BF16 ? 8 : 4, BATCH = 2;
    const int lane = (int)threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t t = unit / pieces;
    if (t >= T) return;
    const int c = (int)(unit - t * pieces) * 64 + lane, cc = min(c, row_vec - 1);   // whole wavefronts stay for the ballots
    const int64_t row_bytes = (int64_t)row_vec * 16;
    int lo, hi;
    row_range(rank_off, rank, T * k, lo, hi);
    uint4 vs = make_uint4(0u, 0u, 0u, 0u);
    if (dx_shared) vs = nt_load16(dx_shared + t * row_vec + cc);
    float acc[NV];
#pragma unroll
    for (int e = 0; e < NV; ++e) acc[e] = 0.0f;
    for (int j0 = 0; j0 < k; j0 += 64) {
        const int32_t p_lane = perm_pos[t * k + min(j0 + lane, k - 1)];
        uint64_t todo = __ballot(j0 + lane < k && p_lane >= lo && p_lane < hi);
        while (todo) {
            u32x4_t v[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int32_t p = __builtin_amdgcn_readlane(p_lane, todo ? __builtin_ctzll(todo) : 0);
                const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(dxp + (int64_t)p * row_bytes), 0, todo ? (int)row_bytes : 0, 0x00020000);
                v[b] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, cc * 16, 0, 2 /* nt */);
                todo &= todo - 1;
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const uint4 q = make_uint4(v[b][0], v[b][1], v[b][2], v[b][3]);
                float f[NV];
                if constexpr (BF16) unpack_bf16x8(q, f); else unpack_f32x4(q, f);
#pragma unroll
                for (int e = 0; e < NV; ++e) acc[e] += f[e];
            }
        }
    }
    if (c >= row_vec) return;
    if (dx_shared) {
        float f[NV];
        if constexpr (BF16) unpack_bf16x8(vs, f); else unpack_f32x4(vs, f);
#pragma unroll
        for (int e = 0; e < NV; ++e) acc[e] += f[e];
    }
    if constexpr (BF16) nt_store16(pack_bf16x8(acc), dx + t * row_vec + c); else nt_store16(pack_f32x4(acc), dx + t * row_vec + c);
}

}  // namespace grace

using namespace grace;

// Row bytes that a buffer descriptor spans.
constexpr int64_t MAX_ROW_BYTES = INT32_MAX;

static int check_rows(const char *who, int32_t T, int32_t k, int32_t d, grace_dtype dt, const int32_t *rank_off, int32_t rank) {
    if (T < 0 || k < 1 || d < 1) return fail(GRACE_EINVAL, "%s: T=%d, k=%d, d=%d invalid", who, T, k, d);
    if (dt != GRACE_F32 && dt != GRACE_BF16) return fail(GRACE_EINVAL, "%s: unknown dtype %d", who, (int)dt);
    const int64_t row_bytes = (int64_t)d * (dt == GRACE_F32 ? 4 : 2);
    if (row_bytes % 16 != 0) return fail(GRACE_ESHAPE, "%s: row of %lld bytes is not a multiple of 16", who, (long long)row_bytes);
    if (row_bytes > MAX_ROW_BYTES) return fail(GRACE_ESHAPE, "%s: row of %lld bytes is too long", who, (long long)row_bytes);
    if ((int64_t)T * k > INT32_MAX) return fail(GRACE_ESHAPE, "%s: T*k exceeds 2^31-1", who);
    if (rank_off && (rank < 0 || rank >= GRACE_MAX_RANKS)) return fail(GRACE_EINVAL, "%s: rank=%d invalid", who, rank);
    return GRACE_OK;
}

// Workgroups of four wavefronts for `units` of them; launches take at most 2^32 work-items.
static int grid_of(const char *who, int64_t units, unsigned &groups) {
    const int64_t n = ceil_div(units, 4);
    if (n * 256 > 0xFFFFFFFFll) return fail(GRACE_ESHAPE, "%s: too many rows", who);
    groups = (unsigned)n;
    return GRACE_OK;
}

extern "C" int grace_combine_backward(const void *dout, const void *y, const int32_t *perm_pos, const float *topk_weight, int32_t T, int32_t k,
                                      int32_t d, grace_dtype dt, const int32_t *rank_off, int32_t rank, void *dy, float *dtopk_weight,
                                      void *stream) {
    int rc = check_rows("combine_backward", T, k, d, dt, rank_off, rank);
    if (rc != GRACE_OK || T == 0) return rc;
    if (!dout || !y || !perm_pos || !topk_weight || !dy || !dtopk_weight) return fail(GRACE_EINVAL, "combine_backward: null device pointer");
    if ((((uintptr_t)dout) | ((uintptr_t)y) | ((uintptr_t)dy)) & 15)
        return fail(GRACE_EINVAL, "combine_backward: dout, y and dy must be 16-byte aligned");
    const int row_vec = (int)((int64_t)d * (dt == GRACE_F32 ? 4 : 2) / 16);
    // A token's choices over several wavefronts up to 65536 of them, k = 8: 64 tokens of 4 KB 8.9 -> 3.7 us, 512 15.6 -> 8.7; 8192 tokens 110.3 ->
    // 107.9; 8192 of 20 KB, k = 6 466 -> 433.  More of them read the gradient more often: 32768 tokens of 1 KB 109 us, with 8 parts 126.
    int parts = 1;
    while (parts < k && (int64_t)T * parts < 65536) parts *= 2;
    parts = std::min(parts, k);
    unsigned groups;
    rc = grid_of("combine_backward", (int64_t)T * parts, groups);
    if (rc != GRACE_OK) return rc;
    auto launch = [&](auto kernel) {
        kernel<<<groups, 256, 0, (hipStream_t)stream>>>((const uint4 *)dout, (const uint4 *)y, perm_pos, topk_weight, T, k, row_vec, rank_off, rank,
                                                        parts, (uint4 *)dy, dtopk_weight);
    };
    // rows of one vector a lane: 32768 tokens of 1 KB 111 us, 124 with four; longer rows, four: 512 tokens of 4 KB 8.7 us, 9.4 with one, 10.1 with eight
    if (dt == GRACE_BF16) launch(row_vec <= 64 ? combine_backward_kernel<true, 1> : combine_backward_kernel<true, 4>);
    else launch(row_vec <= 64 ? combine_backward_kernel<false, 1> : combine_backward_kernel<false, 4>);
    GRACE_LAUNCH_CHECK("combine_backward_kernel");
    return GRACE_OK;
}

extern "C" int grace_permute_backward(const void *dxp, const int32_t *perm_pos, int32_t T, int32_t k, int32_t d, grace_dtype dt,
                                      const int32_t *rank_off, int32_t rank, const void *dx_shared, void *dx, void *stream) {
    int rc = check_rows("permute_backward", T, k, d, dt, rank_off, rank);
    if (rc != GRACE_OK || T == 0) return rc;
    if (!dxp || !perm_pos || !dx) return fail(GRACE_EINVAL, "permute_backward: null device pointer");
    if ((((uintptr_t)dxp) | ((uintptr_t)dx_shared) | ((uintptr_t)dx)) & 15)
        return fail(GRACE_EINVAL, "permute_backward: dxp, dx_shared and dx must be 16-byte aligned");
    const int row_vec = (int)((int64_t)d * (dt == GRACE_F32 ? 4 : 2) / 16), pieces = (row_vec + 63) / 64;
    unsigned groups;
    rc = grid_of("permute_backward", (int64_t)T * pieces, groups);
    if (rc != GRACE_OK) return rc;
    auto launch = [&](auto kernel) {
        kernel<<<groups, 256, 0, (hipStream_t)stream>>>((const char *)dxp, perm_pos, T, k, row_vec, pieces, rank_off, rank,
                                                        (const uint4 *)dx_shared, (uint4 *)dx);
    };
    if (dt == GRACE_BF16) launch(permute_backward_kernel<true>);
    else launch(permute_backward_kernel<false>);
    GRACE_LAUNCH_CHECK("permute_backward_kernel");
    return GRACE_OK;
}
