// grace_expert_ffn_backward, grace_shared_ffn_backward: gradients of the grouped SwiGLU FFN (Section 1's expert computation) for the rows
// and the weights, as four products (ffn_grad.h).
#include <atomic>
#include <initializer_list>

#include "common.h"
#include "gemm_bf16_grad.h"
#include "gemm_f32_grad.h"

namespace grace {
namespace grad {

constexpr int MAX_WIDTH = 1 << 20;   // of d and of all hidden columns: offsets inside a tile fit 31 bits

// LDS past 64 KB has to be allowed for a kernel, once on each device.
template <typename K>
static int allow_lds(K kernel, int bytes, std::atomic<uint64_t> &done, const char *what) {
    int dev = 0;
    GRACE_HIP(hipGetDevice(&dev));
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (done.load(std::memory_order_acquire) & bit) return GRACE_OK;
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return fail(GRACE_EHIP, "%s: cannot reserve LDS: %s", what, hipGetErrorString(e));
    done.fetch_or(bit, std::memory_order_release);
    return GRACE_OK;
}

// Shapes of the bf16 kernel's tiles.  LARGE fills a compute unit's matrix cores best; LOWER fills the last row tiles and the last round better; two
// workgroups of MEDIUM or SMALL share a compute unit, so that one works while the other waits, and there are four and sixteen times as many tiles for
// launches that would leave compute units idle.
using LARGE = Shape<256, 256, 64, 2, 3, 2, 4>;
using LOWER = Shape<192, 256, 64, 2, 3, 2, 4>;
using MEDIUM = Shape<128, 128, 64, 2, 3, 2, 2>;
using SMALL = Shape<64, 64, 64, 4, 4, 4, 1>;
enum class Tiles { LARGE, LOWER, MEDIUM, SMALL };

// dh and gates: time of a launch by its rounds of tiles.  Measured for sums of 2048 (32 steps), us a round: LARGE 62, LOWER 52; MEDIUM 47 with two workgroups on
// every compute unit, 30 with one; SMALL 24 and 17.  Only the ratios matter, and they are taken to be the same for other widths d; where d is so small that
// a tile is mostly start and epilogue that was not measured.  Whole pass, us, with these tiles for one launch and the rules' for the other two, and
// which are chosen; 16 experts, d = 2048, f = 1024 unless said:
//                                             dh LARGE  LOWER MEDIUM SMALL          gates LARGE  LOWER MEDIUM SMALL
//     16 rows of 8, d = 1024, f = 512            33.0   30.5   28.7   24.4  S              32.9   31.2   28.9   24.4  S
//     128 rows                                    108    104    102     94  S               101     98     95     94  S
//     512                                         123    124    115    113  S               114    115    107    113  S
//     2048                                        164    154    146    149  M               152    144    145    153  M
//     4096                                        205    191    191    200  M               197    190    202    222  LOWER
//     8192                                        337    322    338    361  LOWER           338    321    331    382  LOWER
//     16000 of 4, d = 1024, f = 512               162    157    156    172  M               155    167    162    191  L
//     4096 of 2, d = 4096, f = 14336             3223   3215   3287   3688  L              3224   3204   3339   4111  L
//     2000 of two shared, d = 1024, f = 1408      124    119    116    123  M               118    116    120    136  LOWER
//     8001 of two shared, f = 1408                656    647    662    718  LOWER           654    660    667    791  L
static double rounds_cost(Tiles shape, int64_t tiles, int n_cu) {
    if (shape == Tiles::LARGE || shape == Tiles::LOWER) return (shape == Tiles::LARGE ? 62.0 : 52.0) * (double)ceil_div(tiles, n_cu);
    const double both = shape == Tiles::MEDIUM ? 47.0 : 24.0, one = shape == Tiles::MEDIUM ? 30.0 : 17.0;
    const int64_t rest = tiles % (2 * n_cu);
    return both * (double)(tiles / (2 * n_cu)) + (rest == 0 ? 0.0 : rest <= n_cu ? one : both);
}

// dx and the weights' gradients, in one launch: time by the steps (64 positions of a sum) of its tiles; storing a weights' tile takes two steps' time.
// SMALL tiles are for dx only, beside MEDIUM ones for the weights, and LARGE ones for the weights only, beside LOWER ones for dx; the fit is older than that and
// still counts dx's tiles as 256 x 256 then.  Fitted to 16 measured sizes.  Whole pass, us, with LARGE tiles for both, LOWER and LARGE, MEDIUM for both, SMALL and
// MEDIUM, the other launches by their rule, and which of the last three is chosen (LARGE: the first
// of them); 16 experts, d = 2048, f = 1024 unless said:
//     16 rows of 8, d = 1024, f = 512            33.0   30.9   28.0   24.5  SMALL
//     100 rows of 4, d = 512, f = 2048           62.1   56.4   53.0   35.3  SMALL
//     128 rows                                     99     98     94     96  MEDIUM
//     512                                         115    116    113    115  MEDIUM
//     2048                                        144    147    144    156  LARGE
//     4096                                        194    190    202    233  LARGE
//     8192                                        325    320    342    409  LARGE
//     16000 of 4, d = 1024, f = 512               193    194    158    188  MEDIUM
//     4096 of 2, d = 4096, f = 14336             3245   3223   3811   5096  LARGE
//     2000 of two shared, d = 1024, f = 1408      158    134    118    137  MEDIUM
//     8001 of two shared, f = 1408                687    652    753    852  LARGE
static double joined_cost(Tiles shape, const FfnGrad &g, int n_cu) {
    struct Fit { int side, at_once; double start, step, step_full, tail; };   // us: of a launch, a step alone, a step on every unit, the last tiles' steps
    constexpr Fit large{256, 1, 5.0, 1.0, 1.9, 0.5}, medium{128, 2, 3.0, 0.65, 1.2, 0.25}, small{64, 2, 5.0, 0.3, 0.55, 0.0};
    const Fit &fi = shape == Tiles::LARGE ? large : shape == Tiles::MEDIUM ? medium : small, &fw = shape == Tiles::LARGE ? large : medium;
    const double in_slots = (double)n_cu * fi.at_once, w_slots = (double)n_cu * fw.at_once;
    const double in = (double)expected_tiles<INPUT>(g, fi.side, fi.side), w = (double)expected_tiles<WEIGHTS>(g, fw.side, fw.side);
    const double in_steps = (double)steps_of<INPUT>(g), w_steps = (double)steps_of<WEIGHTS>(g);
    const double longest = g.seg_off ? 1.75 * w_steps : w_steps;   // (experts with more rows than the mean: an assumption about skew, not a measurement)
    return fi.start + std::max({fi.step * in_steps, fw.step * longest, fi.step_full * in * in_steps / in_slots + fw.step_full * w * (w_steps + 2.0) / w_slots}) +
           fi.tail * std::min(w_steps, w_steps * w / w_slots);
}

template <typename F>
static Tiles cheapest(std::initializer_list<Tiles> among, F cost) {
    Tiles best = Tiles::LARGE;
    for (Tiles shape : among)
        if (cost(shape) < cost(best)) best = shape;
    return best;
}

static int compute_units() {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return -1;
    return n;
}

// Workgroups for tiles over rows.  A rank's share may be any part of the rows; far more workgroups than its tiles are expected to be would cost more to
// start than the tiles that some might have to take besides their own.
template <Product P, typename SH>
static int64_t row_grid(const FfnGrad &g, int n_cu, int64_t blocks) {
    return std::min(blocks, 8 * ceil_div(std::max<int64_t>(2 * expected_tiles<P>(g, SH::BM, SH::BN), 8 * n_cu), 8));
}

template <Product P, int SPL, typename SH>
static int launch_rows(const FfnGrad &g, int n_cu, hipStream_t st, const char *what) {
    static std::atomic<uint64_t> done{0};
    const int64_t blocks = workgroups<P, SH::BM, SH::BN>(g);
    const int rc = allow_lds(bf16_kernel<P, SPL, SH>, SH::LDS_BYTES, done, what);
    if (rc != GRACE_OK) return rc;
    bf16_kernel<P, SPL, SH><<<(unsigned)row_grid<P, SH>(g, n_cu, blocks), SH::THREADS, SH::LDS_BYTES, st>>>(g, (int)blocks);
    GRACE_LAUNCH_CHECK(what);
    return GRACE_OK;
}
template <Product P, int SPL>
static int launch_rows(const FfnGrad &g, int n_cu, hipStream_t st, const char *what) {
    const Tiles shape = cheapest({Tiles::LOWER, Tiles::MEDIUM, Tiles::SMALL}, [&](Tiles t) {
        const int bn = t == Tiles::LARGE || t == Tiles::LOWER ? 256 : t == Tiles::MEDIUM ? 128 : 64, bm = t == Tiles::LOWER ? 192 : bn;
        return rounds_cost(t, expected_tiles<P>(g, bm, bn), n_cu);
    });
    return shape == Tiles::LARGE    ? launch_rows<P, SPL, LARGE>(g, n_cu, st, what)
           : shape == Tiles::LOWER  ? launch_rows<P, SPL, LOWER>(g, n_cu, st, what)
           : shape == Tiles::MEDIUM ? launch_rows<P, SPL, MEDIUM>(g, n_cu, st, what)
                                    : launch_rows<P, SPL, SMALL>(g, n_cu, st, what);
}

// (without rows: the weights' gradients alone, which are zeros)
template <int SPL, typename SH, typename SH_WEIGHTS = SH>
static int launch_input_weights(const FfnGrad &g, int n_cu, hipStream_t st) {
    static std::atomic<uint64_t> done{0};
    static_assert(SH::THREADS == SH_WEIGHTS::THREADS, "one launch");
    constexpr int lds = std::max(SH::LDS_BYTES, SH_WEIGHTS::LDS_BYTES);
    const char *what = "ffn_backward dx and weights";
    const int rc = allow_lds(bf16_input_weights_kernel<SPL, SH, SH_WEIGHTS>, lds, done, what);
    if (rc != GRACE_OK) return rc;
    const int64_t input = g.rows > 0 ? workgroups<INPUT, SH::BM, SH::BN>(g) : 0, weights = workgroups<WEIGHTS, SH_WEIGHTS::BM, SH_WEIGHTS::BN>(g);
    const int64_t grid = row_grid<INPUT, SH>(g, n_cu, input);
    bf16_input_weights_kernel<SPL, SH, SH_WEIGHTS><<<(unsigned)(grid + weights), SH::THREADS, lds, st>>>(g, (int)grid, (int)input,
                                                                                                      steps_of<WEIGHTS>(g) > steps_of<INPUT>(g));
    GRACE_LAUNCH_CHECK(what);
    return GRACE_OK;
}

template <int SPL>
static int backward_bf16(const FfnGrad &g, hipStream_t st) {
    const int n_cu = compute_units();
    if (n_cu <= 0) return fail(GRACE_EHIP, "ffn_backward: cannot query the device");
    int rc = GRACE_OK;
    if (g.rows > 0) {
        rc = launch_rows<HIDDEN, SPL>(g, n_cu, st, "ffn_backward dh");
        if (rc == GRACE_OK) rc = launch_rows<GATES, SPL>(g, n_cu, st, "ffn_backward gates");
    }
    if (rc != GRACE_OK) return rc;
    const Tiles shape = cheapest({Tiles::MEDIUM, Tiles::SMALL}, [&](Tiles t) { return joined_cost(t, g, n_cu); });
    return shape == Tiles::LARGE    ? launch_input_weights<SPL, LOWER, LARGE>(g, n_cu, st)
           : shape == Tiles::MEDIUM ? launch_input_weights<SPL, MEDIUM>(g, n_cu, st)
                                    : launch_input_weights<SPL, SMALL, MEDIUM>(g, n_cu, st);
}

template <Product P, int SPL>
static int launch_rows_f32(const FfnGrad &g, hipStream_t st, const char *what) {
    const auto kernel = g.d % 4 == 0 && g.f % 4 == 0 ? f32::kernel<P, SPL, true> : f32::kernel<P, SPL, false>;
    kernel<<<(unsigned)workgroups<P, f32::TILE, f32::TILE>(g), f32::THREADS, 0, st>>>(g);
    GRACE_LAUNCH_CHECK(what);
    return GRACE_OK;
}

template <int SPL>
static int backward_f32(const FfnGrad &g, hipStream_t st) {
    int rc = GRACE_OK;
    if (g.rows > 0) {
        rc = launch_rows_f32<HIDDEN, SPL>(g, st, "ffn_backward dh");
        if (rc == GRACE_OK) rc = launch_rows_f32<GATES, SPL>(g, st, "ffn_backward gates");
    }
    if (rc != GRACE_OK) return rc;
    // (1000 rows of 8 experts, d = 1024, f = 2816: dx and the weights' gradients as two launches 451 us, as one 369)
    const int64_t input = g.rows > 0 ? workgroups<INPUT, f32::TILE, f32::TILE>(g) : 0, weights = workgroups<WEIGHTS, f32::TILE, f32::TILE>(g);
    const auto kernel = g.d % 4 == 0 && g.f % 4 == 0 ? f32::input_weights_kernel<SPL, true> : f32::input_weights_kernel<SPL, false>;
    kernel<<<(unsigned)(input + weights), f32::THREADS, 0, st>>>(g, (int)input, steps_of<WEIGHTS>(g) > steps_of<INPUT>(g));
    GRACE_LAUNCH_CHECK("ffn_backward dx and weights");
    return GRACE_OK;
}

// Launches take at most 2^32 work-items; tile numbers stay below 2^31.
static bool fits(const FfnGrad &g) {
    static_assert(SMALL::BM == f32::TILE && SMALL::THREADS == f32::THREADS, "the smallest tiles, so the most workgroups");
    constexpr int SIDE = f32::TILE;
    const int64_t most = std::max({workgroups<HIDDEN, SIDE, SIDE>(g), workgroups<GATES, SIDE, SIDE>(g), workgroups<INPUT, SIDE, SIDE>(g)});
    return most * f32::THREADS <= 0x7FFFFFFFll && workgroups<WEIGHTS, SIDE, SIDE>(g) * f32::THREADS <= 0x7FFFFFFFll;
}

// Workspace: h, dg and du of the rows' type and, in bf16, dh.
static size_t hidden_bytes(int64_t rows, int64_t hcols, grace_dtype dt) {
    return align_up((size_t)rows * (size_t)hcols * (dt == GRACE_F32 ? 4 : 2), 256);
}
static size_t workspace_bytes(int64_t rows, int64_t hcols, grace_dtype dt) {
    return 3 * hidden_bytes(rows, hcols, dt) + (dt == GRACE_BF16 ? hidden_bytes(rows, hcols, GRACE_F32) : 0) + 256;
}

static int check_shapes(const char *who, int32_t d, int32_t f, int64_t hcols, grace_dtype dt) {
    if (dt != GRACE_F32 && dt != GRACE_BF16) return fail(GRACE_EINVAL, "%s: unknown dtype %d", who, (int)dt);
    if (d < 1 || f < 1) return fail(GRACE_EINVAL, "%s: d=%d, f=%d invalid", who, d, f);
    if (dt == GRACE_BF16 && ((d % 8) || (f % 8)))
        return fail(GRACE_ESHAPE, "%s: bf16 needs d and f to be multiples of 8 (d=%d, f=%d)", who, d, f);
    if (d > MAX_WIDTH || hcols > MAX_WIDTH)
        return fail(GRACE_ESHAPE, "%s: d=%d or %lld hidden columns exceed %d", who, d, (long long)hcols, MAX_WIDTH);
    return GRACE_OK;
}

static int backward(const char *who, FfnGrad &g, grace_dtype dt, void *ws, void *stream) {
    if (!g.w_gate || !g.w_up || !g.w_down || !g.dw_gate || !g.dw_up || !g.dw_down) return fail(GRACE_EINVAL, "%s: null device pointer", who);
    if (g.rows > 0 && (!g.x || !g.dy || !g.dx || !ws)) return fail(GRACE_EINVAL, "%s: null device pointer", who);
    const void *all[] = {g.x, g.dy, g.dx, g.w_gate, g.w_up, g.w_down, g.dw_gate, g.dw_up, g.dw_down, ws};
    for (const void *p : all)
        if ((uintptr_t)p & 15) return fail(GRACE_EINVAL, "%s: device pointers must be 16-byte aligned", who);
    if (!fits(g))
        return fail(GRACE_ESHAPE, "%s: more tiles than a launch takes (%d rows, d=%d, %lld hidden columns)", who, g.rows, g.d, (long long)g.hcols);
    const size_t bytes = hidden_bytes(g.rows, g.hcols, dt);
    g.hid = ws;
    g.dg = (char *)ws + bytes;
    g.du = (char *)ws + 2 * bytes;
    g.dh = dt == GRACE_BF16 ? (float *)((char *)ws + 3 * bytes) : (float *)ws;
    hipStream_t st = (hipStream_t)stream;
    if (dt == GRACE_BF16) return g.S <= 64 ? backward_bf16<1>(g, st) : backward_bf16<4>(g, st);
    return g.S <= 64 ? backward_f32<1>(g, st) : backward_f32<4>(g, st);
}

}  // namespace grad
}  // namespace grace

using namespace grace;

extern "C" size_t grace_ffn_backward_workspace_bytes(int32_t rows, int32_t d, int32_t f, int32_t n_shared, grace_dtype dt) {
    if (rows < 0 || d < 1 || f < 1 || n_shared < 0 || (dt != GRACE_F32 && dt != GRACE_BF16)) return 0;
    return grad::workspace_bytes(rows, (int64_t)f * (n_shared ? n_shared : 1), dt);
}

extern "C" int grace_expert_ffn_backward(const grace_table *table, int32_t rank, const void *xp, const void *dy, const int32_t *inst_off,
                                         int32_t T, int32_t k, int32_t d, int32_t f, grace_dtype dt, const void *w_gate, const void *w_up,
                                         const void *w_down, void *dxp, void *dw_gate, void *dw_up, void *dw_down, void *ws, void *stream) {
    if (!table) return fail(GRACE_EINVAL, "expert_ffn_backward: table is null");
    if (rank < 0 || rank >= table->R) return fail(GRACE_EINVAL, "expert_ffn_backward: rank=%d outside [0,%d)", rank, table->R);
    if (T < 0 || k < 1) return fail(GRACE_EINVAL, "expert_ffn_backward: T=%d, k=%d invalid", T, k);
    if ((int64_t)T * k > INT32_MAX) return fail(GRACE_ESHAPE, "expert_ffn_backward: T*k exceeds 2^31-1");
    const int rc = grad::check_shapes("expert_ffn_backward", d, f, f, dt);
    if (rc != GRACE_OK) return rc;
    const int g0 = table->rank_ptr[rank], S = table->rank_ptr[rank + 1] - g0;
    if (S == 0) return GRACE_OK;
    if (!inst_off) return fail(GRACE_EINVAL, "expert_ffn_backward: null device pointer");
    grad::FfnGrad g{};
    g.x = xp; g.dy = dy; g.w_gate = w_gate; g.w_up = w_up; g.w_down = w_down;
    g.dx = dxp; g.dw_gate = dw_gate; g.dw_up = dw_up; g.dw_down = dw_down;
    g.expected = (int)ceil_div((int64_t)T * k * S, table->I);
    g.seg_off = inst_off + g0; g.S = S; g.rows = T * k; g.d = d; g.f = f; g.hcols = f;
    return grad::backward("expert_ffn_backward", g, dt, ws, stream);
}

extern "C" int grace_shared_ffn_backward(const void *x, const void *dy, int32_t T, int32_t d, int32_t f, int32_t n_shared, grace_dtype dt,
                                         const void *w_gate, const void *w_up, const void *w_down, void *dx, void *dw_gate, void *dw_up,
                                         void *dw_down, void *ws, void *stream) {
    if (T < 0 || n_shared < 1) return fail(GRACE_EINVAL, "shared_ffn_backward: T=%d, n_shared=%d invalid", T, n_shared);
    const int rc = grad::check_shapes("shared_ffn_backward", d, f, (int64_t)n_shared * f, dt);
    if (rc != GRACE_OK) return rc;
    grad::FfnGrad g{};
    g.x = x; g.dy = dy; g.w_gate = w_gate; g.w_up = w_up; g.w_down = w_down;
    g.dx = dx; g.dw_gate = dw_gate; g.dw_up = dw_up; g.dw_down = dw_down;
    g.expected = T;
    g.seg_off = nullptr; g.S = n_shared; g.rows = T; g.d = d; g.f = f; g.hcols = (int64_t)n_shared * f;
    return grad::backward("shared_ffn_backward", g, dt, ws, stream);
}
