// bf16 matrix-core kernel of the FFN's backward products (ffn_grad.h).
//
// An operand whose sum axis is contiguous in memory lies in LDS as [rows][BK], its 16-byte chunks exchanged by row; a
// fragment of v_mfma_f32_16x16x32_bf16 (16 rows x 32, eight consecutive values of the sum axis per lane) is one 16-byte read.  One whose
// sum axis is the slow one (weights in dh and dx, everything in the weights' gradients) lies as [BK][columns], and a fragment is two
// transposing reads (ds_read_b64_tr_b16: sixteen lanes read a block of 4 x 16 values and each gets a column), so no operand is ever
// transposed in memory.  Its 32-byte units are exchanged by row so that the rows that one read touches are spread over all banks alike.
// Both are copied HBM -> LDS by 16-byte buffer loads that write LDS directly, into a ring of a few steps; what is past a matrix' edge, a segment's last
// row or the end of the sum axis has an offset past the descriptor's range and arrives as zeros.
#pragma once
#include "ffn_grad.h"

namespace grace {
namespace grad {

typedef __attribute__((ext_vector_type(4))) short s16x4_t;

// Tile BM x BN, sums in steps of BK, SA and SB >= SA steps of the operands in LDS, WM x WN wavefronts.
template <int BM_, int BN_, int BK_, int SA_, int SB_, int WM_, int WN_>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, BK = BK_, SA = SA_, SB = SB_, WM = WM_, WN = WN_;
    static constexpr int WAVES = WM * WN, THREADS = WAVES * 64;
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, B_BASE = SA * A_BYTES, LDS_BYTES = B_BASE + SB * B_BYTES;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;                                        // fragments of a wavefront
    static constexpr int LOADS_A = A_BYTES / 1024 / WAVES, LOADS_B = B_BYTES / 1024 / WAVES;          // of a wavefront per step
    // Loads that may be in flight when a step begins, of the step's own loads the last ones apart (they land in order of issue, a step's A before B)
    static constexpr int IN_FLIGHT = (SA - 2) * (LOADS_A + LOADS_B) + (SB > SA ? LOADS_B : 0);
    static_assert(SB == SA || SB == SA + 1, "the order of issue that IN_FLIGHT counts");
    static constexpr bool PIPELINED = BN == 256;                      // sum_pipelined, else a plain loop
};

// 16 bytes per lane from the descriptor's base + voff to lds_wave_base + 16 * lane.  Inline assembly, so that the compiler does not hold
// back the fragment reads around it until the load has landed; the kernel waits for it.  s_nop 0: the wait state between the write of M0
// and its use.  The compiler does not keep wait states for what is inside either: that no vector instruction writes the descriptor or the
// address too shortly before is checked on the compiled code (asm_hazards.py).
__device__ __forceinline__ void load16_to_lds(u32x4_t rsrc, uint32_t voff, char *lds_wave_base) {
    const uint32_t lds = (uint32_t)(size_t)(__attribute__((address_space(3))) char *)lds_wave_base;
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %0, 0 offen lds" ::"s"(rsrc), "v"(voff), "s"(lds) : "memory");
}
__device__ __forceinline__ u32x4_t descriptor(const void *base) {
    const uint64_t b = (uint64_t)base;
    return u32x4_t{(uint32_t)b, (uint32_t)(b >> 32) & 0xFFFFu, NO_DATA, 0x00020000u};
}

// Where a row's chunks (contiguous sum axis) and a position's units (slow) go: xor of their number with this.  256 bytes of LDS hold all
// banks once; a fragment read takes 16 rows at one chunk, a transposing one 16 positions (0-3, 8-11, 16-19, 24-27 of 32, or those + 4) at one unit.
template <int BK>
__device__ __forceinline__ int chunk_key(int row) { return BK == 64 ? (row >> 1) & 7 : (0 - (row >> 2)) & 3; }
template <int COLS>
__device__ __forceinline__ int unit_key(int k) {
    return COLS == 256 ? (k & 3) | ((k >> 3) & 3) << 2 : COLS == 128 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
}

// One operand of a tile: R rows (SLOW: columns) by the sum axis.
template <bool SLOW, int R, int BK, int WAVES>
struct Source {
    static constexpr int LOADS = R * BK * 2 / 1024 / WAVES;
    static constexpr int PER_ROW = SLOW ? R / 8 : BK / 8;    // lanes of a row in LDS
    static constexpr int ROWS = 64 / PER_ROW;                // rows that a wavefront's load fills
    static_assert(LOADS >= 1, "every wavefront loads");
    const char *p0, *p1;      // the next step's first element; of a second matrix that rows R / 2 .. come from (gate and up weights)
    const char *half;         // the second half's first element
    int64_t step;             // bytes from step to step
    uint32_t off[LOADS];      // of the lane's loads; NO_DATA past the tile's extent
    int at;                   // lane's place on the sum axis: its first element of a step (SLOW: of load 0)
    int K, left;              // positions of a half of the sum axis; of them not yet loaded
    int buf;                  // where the next step goes

    // rows (or columns) beyond `extent` are not there; pair: rows R / 2 .. are rows 0 .. of the second matrix, base1
    __device__ __forceinline__ void set(const void *base, const void *base1, int64_t ld, int extent, int k, bool pair, int wave, int lane) {
        p0 = (const char *)base;
        p1 = pair ? (const char *)base1 : p0;
        half = (const char *)base1;
        step = SLOW ? (int64_t)BK * ld * 2 : BK * 2;
        K = left = k;
        buf = 0;
        const int pos = lane % PER_ROW;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = (i * WAVES + wave) * ROWS + lane / PER_ROW;
            if constexpr (SLOW) {
                const int col = ((pos >> 1) ^ unit_key<R>(row)) * 16 + (pos & 1) * 8;
                off[i] = col < extent ? (uint32_t)row * (uint32_t)(ld * 2) + (uint32_t)col * 2u : NO_DATA;
                if (i == 0) at = row;
            } else {
                const int chunk = pos ^ chunk_key<BK>(row), r = pair ? row % (R / 2) : row;
                off[i] = r < extent ? (uint32_t)r * (uint32_t)(ld * 2) + (uint32_t)chunk * 16u : NO_DATA;
                if (i == 0) at = chunk * 8;   // the same for all: their rows are a multiple of 16 apart
            }
        }
    }
    // Load i of the next step into one of the buffers from lds on.  Past the last step nothing is left: the loads bring zeros that nobody
    // reads, so that every step issues as many.
    __device__ __forceinline__ void load_one(int i, char *lds, int wave) const {
        const bool here = SLOW ? at + i * WAVES * ROWS < left : at < left;
        const bool second = !SLOW && (i * WAVES + wave) * ROWS >= R / 2;   // uniform
        load16_to_lds(descriptor(second ? p1 : p0), here ? off[i] : NO_DATA, lds + buf * (R * BK * 2) + (i * WAVES + wave) * 1024);
    }
    template <bool HALVES, int STAGES>
    __device__ __forceinline__ void advance() {
        buf = buf + 1 == STAGES ? 0 : buf + 1;
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
    template <bool HALVES, int STAGES>
    __device__ __forceinline__ void load(char *lds, int wave) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_one(i, lds, wave);
        advance<HALVES, STAGES>();
    }
};

// Fragment of 16 rows (or columns) from `first` on, positions 32 gk .. of the step.
template <bool SLOW, int R, int BK>
__device__ __forceinline__ bf16x8_t fragment(const char *buf, int first, int gk, int lane) {
    if constexpr (SLOW) {
        const int k = (lane >> 4) * 8 + ((lane >> 2) & 3), key = unit_key<R>(k);   // (the same for k + 4 and k + 32)
        const char *p = buf + (gk * 32 + k) * (R * 2) + (((first >> 4) ^ key) * 32) + (lane & 3) * 8;
        typedef __attribute__((address_space(3))) s16x4_t lds_t;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)p);
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p + 4 * R * 2));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        const int r = first + (lane & 15), chunk = (gk * 4 + (lane >> 4)) ^ chunk_key<BK>(lane & 15);
        return *(const bf16x8_t *)(buf + r * (BK * 2) + chunk * 16);
    }
}

// First column of a wavefront's fragment j in the column operand's tile.
template <Product P, typename SH>
__device__ __forceinline__ int fragment_column(int wn, int j) {
    return P == GATES ? (j / (SH::FN / 2)) * (SH::BN / 2) + wn * (SH::BN / 2 / SH::WN) + (j % (SH::FN / 2)) * 16 : wn * (SH::BN / SH::WN) + j * 16;
}

// One step's products.  The scheduler is told the order: what the first products need, then after every row fragment's FN products the reads
// of the row fragment two further on and a part of the next 32 positions' column fragments, so that a read has the time of
// FN or more products to come back (left to itself the compiler reads two fragments and waits for them).  Small launches are bound by the weights: 128
// rows of 16 experts, d = 2048, f = 1024 dx and weights 62 us, 134 MB of weights read and 201 MB of gradients written, 5.4 TB/s.
template <Product P, typename SH>
__device__ __forceinline__ void compute_step(const char *sa, const char *sb, int wm, int wn, int lane, f32x4_t (&acc)[SH::FM][SH::FN]) {
    constexpr int FM = SH::FM, FN = SH::FN, G = SH::BK / 32, RA = A_SLOW<P> ? 2 : 1, RB = B_SLOW<P> ? 2 : 1, N = G * FM;
    bf16x8_t fa[N], fb[G][FN];
#pragma unroll
    for (int gk = 0; gk < G; ++gk) {
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[gk][j] = fragment<B_SLOW<P>, SH::BN, SH::BK>(sb, fragment_column<P, SH>(wn, j), gk, lane);
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[gk * FM + i] = fragment<A_SLOW<P>, SH::BM, SH::BK>(sa, wm * (SH::BM / SH::WM) + i * 16, gk, lane);
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int j = 0; j < FN; ++j)
            acc[n % FM][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[n / FM][j], fa[n], acc[n % FM][j], 0, 0, 0);
    constexpr int DS_READ = 0x100, MFMA = 0x008, SPREAD = FM > 1 ? FM / 2 : 1;
    __builtin_amdgcn_sched_group_barrier(DS_READ, FN * RB + 2 * RA, 0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        __builtin_amdgcn_sched_group_barrier(MFMA, FN, 0);
        if (n + 2 < N) __builtin_amdgcn_sched_group_barrier(DS_READ, RA, 0);
        if (n / FM + 1 < G && n % FM < SPREAD) __builtin_amdgcn_sched_group_barrier(DS_READ, FN * RB / SPREAD, 0);
    }
}

template <int N>
__device__ __forceinline__ void wait_loads_and_sync() {
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The large tiles' sum: steps of two groups of 32 positions, with the fragments of a group read while the group before it is multiplied, across
// steps too.  A step's one barrier is between its groups: by then every wavefront has read all that it needs of the step's buffers, and has seen
// its own loads of the next step land.  The row operand has two buffers and the column operand three, all of LDS; during a step's first group the columns
// of the step after next are loaded (their buffer was read in the step before), during its second group the rows (theirs is this step's).
// 4096 rows of 2 experts, d = 4096, f = 14336: dx and the weights' gradients 1963 us, 1.23 PFLOP/s (a step read, then multiplied, as in compute_step: 2166).
// Counters of that launch: matrix cores busy 69 % at a clock of 1.7 GHz (the power limit; 2.4 nominal), LDS 29 %, of which 2 % bank conflicts.  What the
// matrix cores wait for was not counted.  The 64 KB to LDS per step and compute unit are near what loads bring with all units asking: 1.5 us at 44
// GB/s, and a step takes 1.6 to 1.7.
template <Product P, typename SH, typename A, typename B>
__device__ __forceinline__ void sum_pipelined(A &a, B &b, int steps, int wm, int wn, int wave, int lane, bool idle, char *smem,
                                              f32x4_t (&acc)[SH::FM][SH::FN]) {
    constexpr int FM = SH::FM, FN = SH::FN, BK = SH::BK, RA = A_SLOW<P> ? 2 : 1, RB = B_SLOW<P> ? 2 : 1;
    static_assert(SH::SA == 2 && SH::SB == 3 && BK == 64 && SH::LOADS_A <= 4 && SH::LOADS_B == 4 && FM >= 4, "the order of loads below");
    char *const lds_b = smem + SH::B_BASE;
    a.template load<P == INPUT, 2>(smem, wave);
    b.template load<P == INPUT, 3>(lds_b, wave);
    a.template load<P == INPUT, 2>(smem, wave);
    b.template load<P == INPUT, 3>(lds_b, wave);
    wait_loads_and_sync<SH::LOADS_A + SH::LOADS_B>();   // the first step has landed
    int buf_a = 0, buf_b = 0;
    bf16x8_t fa[2][FM], fb[2][FN];
    // fragment r of a group: the columns' first, then the rows'
    auto fetch = [&](int set, const char *sa, const char *sb, int gk, int r) {
        if (r < FN) fb[set][r] = fragment<B_SLOW<P>, SH::BN, BK>(sb, fragment_column<P, SH>(wn, r), gk, lane);
        else fa[set][r - FN] = fragment<A_SLOW<P>, SH::BM, BK>(sa, wm * (SH::BM / SH::WM) + (r - FN) * 16, gk, lane);
    };
    // products of one set of fragments; the other set is read, and four loads are issued, meanwhile
    auto group = [&](int set, const char *sa, const char *sb, int gk, int loads, auto load_one) {
        constexpr int N = FN + FM, PER = (N + FM - 2) / (FM - 1);   // fragments read per row fragment's products, none during the last one's
#pragma unroll
        for (int i = 0; i < FM; ++i) {
#pragma unroll
            for (int r = i * PER; r < (i + 1) * PER && r < N; ++r) fetch(set ^ 1, sa, sb, gk, r);
#pragma unroll
            for (int l = 0; l < loads; ++l)   // spread over the row fragments
                if (l * FM / 4 == i) load_one(l);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[set][j], fa[set][i], acc[i][j], 0, 0, 0);
        }
        constexpr int DS_READ = 0x100, MFMA = 0x008;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            int reads = 0;
            for (int r = i * PER; r < (i + 1) * PER && r < N; ++r) reads += r < FN ? RB : RA;
            // a read or two after each product
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
                const int some = reads * (j + 1) / FN - reads * j / FN;
                if (some == 1) __builtin_amdgcn_sched_group_barrier(DS_READ, 1, 0);
                if (some == 2) __builtin_amdgcn_sched_group_barrier(DS_READ, 2, 0);
            }
        }
    };
    if (idle) {   // no rows or columns of the tile are this wavefront's: it loads and keeps step
        for (int s = 0; s < steps; ++s) {
            b.template load<P == INPUT, 3>(lds_b, wave);
            wait_loads_and_sync<SH::LOADS_B>();
            a.template load<P == INPUT, 2>(smem, wave);
        }
    } else {
#pragma unroll
        for (int r = 0; r < FN + FM; ++r) fetch(0, smem, lds_b, 0, r);
        for (int s = 0; s < steps; ++s) {
            const char *sa = smem + buf_a * SH::A_BYTES, *sb = lds_b + buf_b * SH::B_BYTES;
            buf_a ^= 1;
            buf_b = buf_b == 2 ? 0 : buf_b + 1;
            group(0, sa, sb, 1, SH::LOADS_B, [&](int i) { b.load_one(i, lds_b, wave); });
            b.template advance<P == INPUT, 3>();
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(SH::LOADS_B) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            // (behind the last step: what is in the next buffers, which nobody uses)
            group(1, smem + buf_a * SH::A_BYTES, lds_b + buf_b * SH::B_BYTES, 0, SH::LOADS_A, [&](int i) { a.load_one(i, smem, wave); });
            a.template advance<P == INPUT, 2>();
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Results to memory.  The columns' fragment is an instruction's first operand, so value v of acc[i][j] is row 16 i + lane % 16, column 16 j +
// 4 (lane / 16) + v.  Written from there, a store would touch 32 bytes of each of 16 rows; instead every wavefront turns 16 rows at a
// time through LDS (16-byte chunks exchanged by row: no bank conflicts) and stores them as whole runs of 16-byte vectors (8192 rows of 16
// experts, d = 2048, f = 1024, us: dh 66 -> 60, gates 139 -> 128, dx 129 -> 115, weights 168 -> 133).  d and f are multiples of 8, so a vector is there or is not.
template <Product P, typename SH>
__device__ __forceinline__ void write_tile(const FfnGrad &g, const TileOf<uint16_t> &t, int wm, int wn, int wave, int lane, char *smem,
                                           const f32x4_t (&acc)[SH::FM][SH::FN]) {
    constexpr int FM = SH::FM, FN = SH::FN, ROWS = SH::BM / SH::WM;
    const int r16 = lane & 15, quad = lane >> 4;
    if constexpr (P == GATES) {
        constexpr int CW = SH::BN / 2 / SH::WN, CHUNKS = CW / 4, PER = CW / 8, AT_ONCE = 64 / PER;   // columns; fp32 chunks of a row; lanes of a row; rows
        static_assert(SH::WAVES * 16 * CW * 8 <= SH::LDS_BYTES, "staging space");
        char *sg = smem + wave * (16 * CW * 8), *su = sg + 16 * CW * 4;
        const int rr = lane / PER, cc = lane % PER, col = wn * CW + cc * 8;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int row0 = wm * ROWS + i * 16;
            if (row0 >= t.m) break;   // uniform
            f32x4_t dh[16 / AT_ONCE][2];
            bool here[16 / AT_ONCE];
            int64_t at[16 / AT_ONCE];
#pragma unroll
            for (int q = 0; q < 16 / AT_ONCE; ++q) {
                const int row = row0 + q * AT_ONCE + rr;
                here[q] = row < t.m && col < t.n;
                at[q] = t.hid + (int64_t)row * t.ldo + col;
#pragma unroll
                for (int e = 0; e < 2; ++e) dh[q][e] = here[q] ? *(const f32x4_t *)(g.dh + at[q] + e * 4) : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll
            for (int j = 0; j < FN / 2; ++j) {
                const int at16 = r16 * (CW * 4) + (((j * 4 + quad) ^ r16) % CHUNKS) * 16;
                *(f32x4_t *)(sg + at16) = acc[i][j];
                *(f32x4_t *)(su + at16) = acc[i][j + FN / 2];
            }
#pragma unroll
            for (int q = 0; q < 16 / AT_ONCE; ++q) {
                const int r = q * AT_ONCE + rr, c0 = r * (CW * 4) + (((cc * 2) ^ r) % CHUNKS) * 16, c1 = r * (CW * 4) + (((cc * 2 + 1) ^ r) % CHUNKS) * 16;
                const f32x4_t g0 = *(const f32x4_t *)(sg + c0), g1 = *(const f32x4_t *)(sg + c1);
                const f32x4_t u0 = *(const f32x4_t *)(su + c0), u1 = *(const f32x4_t *)(su + c1);
                float h[8], dg[8], du[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    swiglu_grad<true>(e < 4 ? g0[e & 3] : g1[e & 3], e < 4 ? u0[e & 3] : u1[e & 3], dh[q][e >> 2][e & 3], h[e], dg[e], du[e]);
                if (here[q]) {
                    *(uint4 *)((uint16_t *)g.hid + at[q]) = pack_bf16x8(h);
                    *(uint4 *)((uint16_t *)g.dg + at[q]) = pack_bf16x8(dg);
                    *(uint4 *)((uint16_t *)g.du + at[q]) = pack_bf16x8(du);
                }
            }
        }
    } else if constexpr (P == HIDDEN) {
        constexpr int CW = SH::BN / SH::WN, CHUNKS = CW / 4, AT_ONCE = 64 / CHUNKS;   // fp32: as the gates' staging
        static_assert(SH::WAVES * 16 * CW * 4 <= SH::LDS_BYTES, "staging space");
        char *stage = smem + wave * (16 * CW * 4);
        const int rr = lane / CHUNKS, cc = lane % CHUNKS, col = wn * CW + cc * 4;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int row0 = wm * ROWS + i * 16;
            if (row0 >= t.m) break;   // uniform
#pragma unroll
            for (int j = 0; j < FN; ++j) *(f32x4_t *)(stage + r16 * (CW * 4) + (((j * 4 + quad) ^ r16) % CHUNKS) * 16) = acc[i][j];
#pragma unroll
            for (int q = 0; q < 16 / AT_ONCE; ++q) {
                const int r = q * AT_ONCE + rr, row = row0 + r;
                const f32x4_t v = *(const f32x4_t *)(stage + r * (CW * 4) + ((cc ^ r) % CHUNKS) * 16);
                if (row < t.m && col < t.n) *(f32x4_t *)(g.dh + t.hid + (int64_t)row * t.ldo + col) = v;
            }
        }
    } else {
        constexpr int CW = SH::BN / SH::WN, CHUNKS = CW / 8, AT_ONCE = 64 / CHUNKS, KEY = CW >= 128 ? 0 : CW == 64 ? 1 : 2;
        static_assert(SH::WAVES * 16 * CW * 2 <= SH::LDS_BYTES, "staging space");
        char *stage = smem + wave * (16 * CW * 2);
        const int rr = lane / CHUNKS, cc = lane % CHUNKS, col = wn * CW + cc * 8;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int row0 = wm * ROWS + i * 16;
            if (row0 >= t.m) break;   // uniform
#pragma unroll
            for (int j = 0; j < FN; ++j)
                *(uint2 *)(stage + r16 * (CW * 2) + (((j * 2 + (quad >> 1)) ^ (r16 >> KEY)) % CHUNKS) * 16 + (quad & 1) * 8) =
                    make_uint2(pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3]));
#pragma unroll
            for (int q = 0; q < 16 / AT_ONCE; ++q) {
                const int r = q * AT_ONCE + rr, row = row0 + r;
                const uint4 v = *(const uint4 *)(stage + r * (CW * 2) + ((cc ^ (r >> KEY)) % CHUNKS) * 16);
                // (dx and the weights' gradients are not read again by this pass and would push operands out of the caches)
                if (row < t.m && col < t.n) nt_store16(v, (uint4 *)(t.out + (int64_t)row * t.ldo + col));
            }
        }
    }
}

template <Product P, int SPL, typename SH>
__device__ __forceinline__ bool bf16_tile(const FfnGrad &g, int block, char *smem) {
    constexpr int BM = SH::BM, BN = SH::BN, BK = SH::BK, FM = SH::FM, FN = SH::FN;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / SH::WN, wn = wave % SH::WN;
    TileOf<uint16_t> t;
    if (!locate<P, BM, BN, SPL>(g, block, t)) return false;

    Source<A_SLOW<P>, BM, BK, SH::WAVES> a;
    Source<B_SLOW<P>, BN, BK, SH::WAVES> b;
    a.set(t.a0, t.a1, t.lda, t.m, t.K, false, wave, lane);
    b.set(t.b0, t.b1, t.ldb, t.n, t.K, P == GATES, wave, lane);
    auto load_a = [&]() { a.template load<P == INPUT, SH::SA>(smem, wave); };
    auto load_b = [&]() { b.template load<P == INPUT, SH::SB>(smem + SH::B_BASE, wave); };
    const int steps = (t.K + BK - 1) / BK * t.halves;

    f32x4_t acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if (steps > 0 && SH::PIPELINED) {
        if constexpr (SH::PIPELINED) {
            const bool idle = wm * (BM / SH::WM) >= t.m || fragment_column<P, SH>(wn, 0) >= t.n;   // uniform
            sum_pipelined<P, SH>(a, b, steps, wm, wn, wave, lane, idle, smem, acc);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    } else if (steps > 0) {
#pragma unroll
        for (int s = 0; s < SH::SB - SH::SA; ++s) load_b();
#pragma unroll
        for (int s = 0; s < SH::SA - 1; ++s) { load_a(); load_b(); }
        int buf_a = 0, buf_b = 0;
        for (int s = 0; s < steps; ++s) {
            // this step's loads have landed for every wavefront, and every wavefront has read the buffers of the step before, which are filled again
            wait_loads_and_sync<SH::IN_FLIGHT>();
            load_a();
            load_b();
            compute_step<P, SH>(smem + buf_a * SH::A_BYTES, smem + SH::B_BASE + buf_b * SH::B_BYTES, wm, wn, lane, acc);
            buf_a = buf_a + 1 == SH::SA ? 0 : buf_a + 1;
            buf_b = buf_b + 1 == SH::SB ? 0 : buf_b + 1;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // these buffers are read before the barrier that hands them over
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // no load may be on its way to LDS when its bytes are used otherwise
    }

    // every wavefront is done with the ring: its bytes are staging space now
    asm volatile("s_barrier" ::: "memory");
    write_tile<P, SH>(g, t, wm, wn, wave, lane, smem, acc);
    return true;
}

// Tiles first, first + stride, ... of `blocks` numbers: one each, unless there could be many more of them than there are expected to be.
template <Product P, int SPL, typename SH>
__device__ __forceinline__ void bf16_tiles(const FfnGrad &g, int first, int stride, int blocks, char *smem) {
    while (bf16_tile<P, SPL, SH>(g, first, smem)) {
        if (first >= blocks - stride) break;
        first += stride;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the staging space is the ring again
    }
}

// HIDDEN, GATES
template <Product P, int SPL, typename SH>
__global__ __launch_bounds__(SH::THREADS, 2) void bf16_kernel(const FfnGrad g, int blocks) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    bf16_tiles<P, SPL, SH>(g, (int)blockIdx.x, (int)gridDim.x, blocks, smem);
}

// INPUT and WEIGHTS need nothing of each other: in one launch the second's tiles fill the compute units that the first's last round leaves idle.  The
// one whose tiles take longer comes first.
template <int SPL, typename SH_INPUT, typename SH_WEIGHTS>
__global__ __launch_bounds__(SH_INPUT::THREADS, 2) void bf16_input_weights_kernel(const FfnGrad g, int input_grid, int input_blocks, int weights_first) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int block = (int)blockIdx.x, weights = (int)gridDim.x - input_grid;
    const int input = weights_first ? block - weights : block;
    if (input >= 0 && input < input_grid) bf16_tiles<INPUT, SPL, SH_INPUT>(g, input, input_grid, input_blocks, smem);
    else bf16_tile<WEIGHTS, SPL, SH_WEIGHTS>(g, weights_first ? block : block - input_grid, smem);
}

}  // namespace grad
}  // namespace grace
