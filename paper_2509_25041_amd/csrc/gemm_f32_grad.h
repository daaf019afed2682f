// fp32 kernel of the FFN's backward products (ffn_grad.h) on v_mfma_f32_16x16x4_f32: products and sums in 32 bits.  64 x 64 tiles, sums in
// steps of 32, four wavefronts (2 x 2) of 32 x 32 results.  Both operands lie in LDS as [32 positions of the sum axis][64], whichever way they
// lie in memory; the next AHEAD steps' values are loaded to registers meanwhile.
// Bound by the matrix cores and how well tiles fill: 4000 rows of 4 experts, d = 2048, f = 1408 1505 us, 122 of the 147 TFLOP/s that a large product
// reaches; 1000 rows of 8, d = 1024, f = 2816 487 us, 95 (tiles of 64 of their rows hold 78 % of what they could).  Figures below: the latter's whole pass.
#pragma once
#include <type_traits>

#include "ffn_grad.h"

namespace grace {
namespace grad {
namespace f32 {

constexpr int TILE = 64, BK = 32, THREADS = 256;
constexpr int AHEAD = 2;   // steps whose values are in registers or on their way there (three: a workgroup less on a compute unit; 504 -> 523 us)
typedef float Staged[BK * TILE];
// Where a position's column (row) lies.  A matrix instruction takes positions k, k + 8, k + 16, k + 24 (of a sum any four do): 64 lanes that read 16
// columns of these touch every bank once, and a lane's reads are at constant distances (rows of LDS 16 bytes apart in the banks instead: 504 -> 512 us).
__device__ __forceinline__ int staged(int k, int r) { return (k % 8) * (4 * TILE) + k / 8 * TILE + (r ^ (k / 8 * 16)); }

// One operand's 64 x 32 values of a step, as vectors of four along memory's contiguous axis.  Buffer loads without branches: what is not there has
// an offset past the descriptor's range and is zero.  VEC: rows in memory are whole 16-byte vectors (d and f multiples of 4), so a vector is there
// or is not; else its values are loaded one by one.
template <bool SLOW, bool VEC>
struct Source {
    static constexpr int N = TILE * BK / 4 / THREADS, E = VEC ? 1 : 4;   // vectors of a thread; loads of one
    const char *p0, *p1;    // the next step's first element; of a second matrix that rows TILE / 2 .. come from (gate and up weights)
    const char *half;       // the second half's first element
    int64_t step;
    uint32_t off[N][E];     // NO_DATA past the tile's extent
    int at[N];              // first position of a vector in a step
    int K, left;

    static __device__ __forceinline__ int place(int idx, int &k) {   // a vector's first row (column) and position
        k = SLOW ? idx / (TILE / 4) : idx % (BK / 4) * 4;
        return SLOW ? idx % (TILE / 4) * 4 : idx / (BK / 4);
    }
    __device__ __forceinline__ void set(const void *base, const void *base1, int64_t ld, int extent, int k_all, bool pair, int tid) {
        p0 = (const char *)base;
        p1 = pair ? (const char *)base1 : p0;
        half = (const char *)base1;
        step = SLOW ? (int64_t)BK * ld * 4 : BK * 4;
        K = left = k_all;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = place(tid + i * THREADS, at[i]), rr = pair ? r % (TILE / 2) : r;
#pragma unroll
            for (int e = 0; e < E; ++e)
                off[i][e] = rr + (SLOW ? e : 0) < extent ? ((uint32_t)(SLOW ? at[i] : rr) * (uint32_t)ld + (uint32_t)(SLOW ? rr : at[i]) + e) * 4u : NO_DATA;
        }
    }
    template <bool HALVES>
    __device__ __forceinline__ void load(f32x4_t (&v)[N]) {
        const auto r0 = rsrc_of(p0), r1 = rsrc_of(p1);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const auto r = !SLOW && i >= N / 2 ? r1 : r0;   // (rows TILE / 2 .. are the second half of a thread's vectors)
            if constexpr (VEC) {
                v[i] = __builtin_bit_cast(f32x4_t, load16(r, at[i] < left ? off[i][0] : NO_DATA, 0));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[i][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (int)(at[i] + (SLOW ? 0 : e) < left ? off[i][e] : NO_DATA), 0, 0));
            }
        }
        left -= BK;
        if (HALVES && left <= 0 && half) {
            p0 = p1 = half;
            half = nullptr;
            left = K;
        } else {
            p0 += step;
            p1 += step;
        }
    }
    static __device__ __forceinline__ void store(Staged &lds, const f32x4_t (&v)[N], int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int k;
            const int r = place(tid + i * THREADS, k);
            if constexpr (SLOW) {
                *(f32x4_t *)&lds[staged(k, r)] = v[i];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) lds[staged(k, r) + e * (4 * TILE)] = v[i][e];   // (k is a multiple of 4)
            }
        }
    }
};
static_assert(THREADS / (BK / 4) == TILE / 2, "a thread's first vector is of the first half of the rows, its second of the second");

constexpr int F = TILE / 32;   // fragments of a wavefront along each side

// A sum is made of parts of PART steps (256 terms), which are added up: a running sum of 8192 terms was off by 1.6e-6 of its norm, this is by 3.8e-7.  A part is
// added while the next step's values are on their way to LDS (4000 rows of 4 experts, d = 2048, f = 1408 1495 -> 1520 us, behind the step's products 1533,
// with the sums in LDS 1550).
constexpr int PART = 8;
static_assert(PART % AHEAD == 0, "a part begins with a round of steps");

// One step's products.
template <Product P>
__device__ __forceinline__ void products(const Staged &sa, const Staged &sb, int wm, int wn, int lane, f32x4_t (&acc)[F][F]) {
    // (a ds_read2 serves two groups of positions; the four of the next two groups are read a group of products ahead of their own)
    float fa[BK / 4][F], fb[BK / 4][F];
#pragma unroll
    for (int kk = 0; kk < BK / 4; ++kk) {
        const int k = kk + (lane >> 4) * 8;
#pragma unroll
        for (int i = 0; i < F; ++i) fa[kk][i] = sa[staged(k, wm * (TILE / 2) + i * 16 + (lane & 15))];
#pragma unroll
        for (int j = 0; j < F; ++j)
            fb[kk][j] = sb[staged(k, (P == GATES ? j / (F / 2) * (TILE / 2) + wn * (TILE / 4) + j % (F / 2) * 16 : wn * (TILE / 2) + j * 16) + (lane & 15))];
    }
#pragma unroll
    for (int kk = 0; kk < BK / 4; ++kk)
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[kk][j], fa[kk][i], acc[i][j], 0, 0, 0);
    constexpr int DS_READ = 0x100, MFMA = 0x008;
    __builtin_amdgcn_sched_group_barrier(DS_READ, 2 * F, 0);
#pragma unroll
    for (int kk = 0; kk < BK / 4; ++kk) {
        __builtin_amdgcn_sched_group_barrier(MFMA, F * F, 0);
        if (kk % 2 == 0 && kk + 2 < BK / 4) __builtin_amdgcn_sched_group_barrier(DS_READ, 2 * F, 0);
    }
}

template <Product P, int SPL, bool VEC>
__device__ __forceinline__ void tile(const FfnGrad &g, int block, Staged &sa, Staged &sb) {
    using A = Source<A_SLOW<P>, VEC>;
    using B = Source<B_SLOW<P>, VEC>;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
    TileOf<float> t;
    if (!locate<P, TILE, TILE, SPL>(g, block, t)) return;
    A a;
    B b;
    a.set(t.a0, t.a1, t.lda, t.m, t.K, false, tid);
    b.set(t.b0, t.b1, t.ldb, t.n, t.K, P == GATES, tid);
    const int steps = (t.K + BK - 1) / BK * t.halves;
    f32x4_t va[AHEAD][A::N], vb[AHEAD][B::N];
    auto load = [&](int slot) {   // (past the last step nothing is left: zeros that nobody uses)
        a.template load<P == INPUT>(va[slot]);
        b.template load<P == INPUT>(vb[slot]);
    };
    f32x4_t acc[F][F], sum[F][F];   // of the part, of the parts before it
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = sum[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    auto end_part = [&] {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) {
                sum[i][j] += acc[i][j];
                acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            }
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) load(s);
    // A wavefront whose rows or columns are not there stages and keeps step, and leaves the matrix cores to the others (504 -> 493 us).
    const bool idle = wm * (TILE / 2) >= t.m || (P == GATES ? wn * (TILE / 4) : wn * (TILE / 2)) >= t.n;   // uniform
    auto all_steps = [&](auto works) {
        // (two buffers and one barrier a step took the same time)
        auto step = [&](int slot, bool begins_part) {
            A::store(sa, va[slot], tid);
            B::store(sb, vb[slot], tid);
            if constexpr (works.value)
                if (begins_part) end_part();   // (the first one: of zeros)
            __syncthreads();
            load(slot);
            if constexpr (works.value) products<P>(sa, sb, wm, wn, lane, acc);
            __syncthreads();
        };
        int s = 0;
        for (; s + AHEAD <= steps; s += AHEAD) {
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) step(q, q == 0 && s % PART == 0);   // (a register array is indexed by constants)
        }
#pragma unroll
        for (int q = 0; q < AHEAD - 1; ++q)
            if (s + q < steps) step(q, false);
        end_part();
    };
    if (idle) all_steps(std::false_type{});
    else all_steps(std::true_type{});

    // value v of sum[i][j]: row 16 i + lane % 16, column 16 j + 4 (lane / 16) + v
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const int row = wm * (TILE / 2) + i * 16 + (lane & 15);
        if (row >= t.m) continue;
#pragma unroll
        for (int j = 0; j < (P == GATES ? F / 2 : F); ++j) {
            const int col = (P == GATES ? wn * (TILE / 4) : wn * (TILE / 2)) + j * 16 + (lane >> 4) * 4;
            if constexpr (P == GATES) {
                const int64_t at = t.hid + (int64_t)row * t.ldo + col;
                float *to[3] = {(float *)g.hid + at, (float *)g.dg + at, (float *)g.du + at};
                f32x4_t out[3], dh;
                if (VEC && col < t.n) dh = *(const f32x4_t *)to[0];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    if (!VEC) dh[v] = col + v < t.n ? to[0][v] : 0.0f;
                    float h, dg, du;
                    swiglu_grad<false>(sum[i][j][v], sum[i][j + F / 2][v], dh[v], h, dg, du);
                    out[0][v] = h; out[1][v] = dg; out[2][v] = du;
                }
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    if (VEC) {
                        if (col < t.n) *(f32x4_t *)to[q] = out[q];
                    } else {
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (col + v < t.n) to[q][v] = out[q][v];
                    }
                }
            } else {
                float *to = t.out + (int64_t)row * t.ldo + col;
                if (VEC) {
                    if (col < t.n) *(f32x4_t *)to = sum[i][j];
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (col + v < t.n) to[v] = sum[i][j][v];
                }
            }
        }
    }
}

// HIDDEN, GATES
template <Product P, int SPL, bool VEC>
__global__ __launch_bounds__(THREADS, VEC ? 4 : 2) void kernel(const FfnGrad g) {
    __shared__ __attribute__((aligned(16))) Staged sa, sb;
    tile<P, SPL, VEC>(g, (int)blockIdx.x, sa, sb);
}

// INPUT and WEIGHTS, as in bf16
template <int SPL, bool VEC>
__global__ __launch_bounds__(THREADS, VEC ? 4 : 2) void input_weights_kernel(const FfnGrad g, int input_grid, int weights_first) {
    __shared__ __attribute__((aligned(16))) Staged sa, sb;
    const int block = (int)blockIdx.x, weights = (int)gridDim.x - input_grid;
    const int input = weights_first ? block - weights : block;
    if (input >= 0 && input < input_grid) tile<INPUT, SPL, VEC>(g, input, sa, sb);
    else tile<WEIGHTS, SPL, VEC>(g, weights_first ? block : block - input_grid, sa, sb);
}

}  // namespace f32
}  // namespace grad
}  // namespace grace
