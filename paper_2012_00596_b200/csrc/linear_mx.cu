// Entry points of the GEMM with microscaled 4-bit weights: argument checks, workspace, the choice of a kernel.
#include "internal_api.h"
#include "mx_tc.cuh"

namespace npas {

namespace {

npas_status check_args(const npas_mx_linear_desc *d)
{
    if (!d) return NPAS_ERR_NULL;
    const npas_mx_desc w = {d->O, d->I, NPAS_BF16}, x = {d->M, d->I, NPAS_BF16};
    npas_status s = check_mx_desc(&w);
    if (s == NPAS_OK) s = check_mx_desc(&x);
    if (s != NPAS_OK) return s;
    if (d->M > 0x7FFFFF00 || d->O > 0x7FFFFF00) return NPAS_ERR_SHAPE;         // (rounded up to a tile of 256 they are ints)
    if (d->x_dtype != NPAS_BF16 && d->x_dtype != NPAS_MX4) return NPAS_ERR_DTYPE;
    if (d->quantize_x && d->x_dtype != NPAS_BF16) return NPAS_ERR_DTYPE;
    if (d->y_dtype != NPAS_F32 && d->y_dtype != NPAS_BF16) return NPAS_ERR_DTYPE;
    return NPAS_OK;
}

// Up to 16 rows the kernel for few rows quantises the input itself: every CTA its share, again for every 128 outputs.  One launch less
// (1x2048 -> 1000 6.0 -> 4.2 us of host time); from 32 rows on its CTAs take longer than the launch (32x2048 -> 2048 6.8 us, 6.3 in two).
// The GPU by itself takes longer that way where the columns are many, since each stage waits for its part of X: 16x4096 -> 8192 14.7 us, 1.8 and 7.2 in two
// launches; 1x8192 -> 8192 15.7, the product of a blob 9.9.
bool quantizes_itself(const npas_mx_linear_desc &d) { return d.quantize_x && d.M <= 16; }

npas_mx_linear_desc behind_quantize(npas_mx_linear_desc d)
{
    if (d.quantize_x) { d.x_dtype = NPAS_MX4; d.quantize_x = 0; }
    return d;
}

// Kernel (1: CUDA cores, 3: few rows, 4: persistent tiles, 5: the same on CTA pairs, 6: a 16-bit input of up to 16 rows; 0: none) and variant.
struct Choice { int kernel, variant; };

// The automatic choice: the kernel, tile or split that a model puts lowest.  Fitted by least squares to 14700 random layers per kind of input
// (M 17 to 60000, I and O 16 to 8192, a third with residuals, half of odd widths), each timed on every kernel that takes it: standard
// error 7 to 15 %, the kernel it picks takes 1.0 % (4-bit) and 1.3 % (16-bit) more than the best one on average, a fifth more in one layer of 100.  Microseconds of a launch,
// and per round of tiles of a stage of 256 columns (of a step of 64 with a 16-bit input; where the weights stay), of the epilogue, of
// residuals in slabs, of bf16 outputs that do not leave by TMA, of those with residuals, of fp32 residuals.
struct Cost { double launch, k, k_stay, round, res, direct, direct_res, f32_res; };
constexpr Cost kCosts[2][3] = {
    {{3.29, 0.405, 0.331, 0.90, 0.36, 0.00, 0.58, 0.04}, {2.25, 0.474, 0.598, 2.36, 0.47, 0.00, 0.65, 0.00}, {1.78, 0.344, 0.344, 3.46, 0.52, 0.00, 0.79, 0.14}},
    {{3.52, 0.245, 0.164, 1.43, 0.25, 0.11, 0.79, 0.13}, {0.87, 0.351, 0.352, 4.61, 0.62, 0.00, 0.90, 0.00}, {}}};

Choice choose(const npas_mx_linear_desc &d)
{
    const npas_mx_linear_desc in = behind_quantize(d);
    const bool mx = in.x_dtype == NPAS_MX4;
    const int sms = sm_count();
    const auto div = [](long long a, long long b) { return (a + b - 1) / b; };
    const long long stages = div(d.I, 256), steps = div(d.I, 64);
    Choice best = {0, 0};
    double least = 0.;
    auto consider = [&](int kernel, int variant, double us) {
        npas_mx_linear_desc t = in;
        t.variant = variant;
        if (best.kernel && us >= least) return;
        if (kernel == 3 ? !linear_mx_sw_supported(t) : kernel == 4 ? !linear_mx_ps_supported(t) : !linear_mx_d2_supported(t)) return;
        best = {kernel, variant}; least = us;
    };
    // (a few rows more than eight of few columns are left to the tensor cores: 14x48 -> 1042 4.2 us against 3.7.  Path 2 asks for
    // the kernels of tcgen05 MMAs; this one's are warp-wide)
    if (d.path != 2 && linear_mx_gv_supported(in) && (d.M <= 8 || d.I > 128)) return {6, 0};
    // few rows: a CTA, or a cluster that splits the columns, per 128 outputs and up to 128 rows
    if (d.M <= 1024) {
        const long long tiles = div(d.M, 128) * div(d.O, 128);
        const double rows = d.M < 128 ? (double)div(d.M, 16) * 16. : 128.;
        for (int ks = 1; ks <= 8; ks *= 2) {
            // (a split is one wave; clusters do not straddle groups of SMs, so larger ones fill less of the chip: 34 of four took two waves)
            if (ks > 1 && (ks > stages || tiles * ks > (ks == 8 ? sms / 2 : ks == 4 ? sms - sms / 9 : sms))) break;
            const double per_row = ks == 1 ? (mx ? 0.027 : 0.022) + (d.has_residual ? 0.006 : 0.) : (mx ? 0.042 : 0.032) + (d.has_residual ? 0.004 : 0.);
            const double us = (ks == 1 ? 2.49 : mx ? 2.81 : 3.49) + (double)div(tiles * ks, sms) * ((mx ? 0.308 : 0.88) * (double)div(stages, ks) + per_row * rows);
            consider(3, ks, us);
        }
        if (quantizes_itself(d)) return best;
    }
    // persistent tiles of 128 or 256 rows, and of 256 on CTA pairs
    const bool f32 = d.y_dtype == NPAS_F32, direct = !f32 && d.O % 8 != 0;
    for (int i = 0; i < (mx && d.O > 128 ? 3 : 2); ++i) {
        const Cost &c = kCosts[mx ? 0 : 1][i];
        const bool pair = i == 2;
        const long long across = div(d.O, pair ? 256 : 128), tiles = div(d.M, i == 0 ? 128 : 256) * across, units = pair ? sms / 2 : sms;
        const bool stay = !pair && tiles > sms && sms / across * across * 8 >= sms * 7 && (mx ? stages <= 4 : steps <= 8);
        const double rounds = (double)div(tiles, stay ? units / across * across : units), k = (double)(mx ? stages : steps);
        consider(pair ? 5 : 4, pair ? 0 : i == 0 ? 128 : 256,
                 c.launch + rounds * (k * (stay ? c.k_stay : c.k) + c.round + (direct ? c.direct : 0.) +
                                      (d.has_residual ? direct ? c.direct_res : f32 ? c.f32_res : c.res : 0.)));
    }
    return best;
}

Choice choice_for(const npas_mx_linear_desc &d)
{
    const npas_mx_linear_desc in = behind_quantize(d);
    switch (d.path) {
        case 1: return {d.variant ? 0 : 1, 0};
        case 3: return {linear_mx_sw_supported(in) ? 3 : 0, d.variant};
        case 4: return {linear_mx_ps_supported(in) ? 4 : 0, d.variant};
        case 5: return {linear_mx_d2_supported(in) ? 5 : 0, d.variant};
        case 6: return {linear_mx_gv_supported(in) ? 6 : 0, d.variant};
        case 0: case 2: break;
        default: return {0, 0};
    }
    if (d.variant) return {0, 0};
    Choice c = {0, 0};
    const int32_t none = 0;
    cached_plan(d, none, 0, c, [&](Choice &q) { q = choose(d); return true; });
    if (!c.kernel && d.path == 0) c.kernel = 1;
    return c;
}

// Rows of a 16-bit input that do not start on 16-byte boundaries are copied to a pitch that does: the tensor cores' kernels load by TMA.
bool needs_pitch(const npas_mx_linear_desc &d, int kernel) { return kernel != 1 && d.x_dtype == NPAS_BF16 && !d.quantize_x && d.I % 8 != 0; }
int64_t pitch_of(const npas_mx_linear_desc &d) { return ((int64_t)d.I + 7) / 8 * 8; }

// scratch behind the status words: the quantised input, or the copied one
size_t scratch_bytes(const npas_mx_linear_desc &d)
{
    const int kernel = choice_for(d).kernel;
    if (d.quantize_x) return kernel == 3 && quantizes_itself(d) ? 0 : mx_layout(d.M, d.I).total;
    return needs_pitch(d, kernel) ? (size_t)d.M * pitch_of(d) * 2 : 0;
}

constexpr int kPitchThreads = 256;

// `lanes` neighbouring threads have a row and write 16 bytes each at a time, four on their way together; columns past the end are zeros.
__global__ void __launch_bounds__(kPitchThreads) mx_pitch_kernel(int64_t M, int I, int pieces, int lanes, const uint16_t *x, uint4 *out)
{
    tc::pdl_trigger();
    tc::pdl_wait();
    x = tc::behind_wait(x);
    constexpr int kAhead = 4;
    const int rows = kPitchThreads / lanes, lane = threadIdx.x % lanes;
    for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; row < M; row += (int64_t)gridDim.x * rows)
        for (int p0 = lane; p0 < pieces; p0 += kAhead * lanes) {
            tc::MxRaw<4> raw[kAhead];
            const uint16_t *from = x + row * I + 8 * p0;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) tc::mx_load_raw(raw[k], from + 8 * k * lanes, min(I - 8 * (p0 + k * lanes), 8), x + M * I);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int p = p0 + k * lanes;
                uint32_t v[4];
                tc::mx_align(v, raw[k], from + 8 * k * lanes, min(I - 8 * p, 8));
                if (p < pieces) out[row * pieces + p] = make_uint4(v[0], v[1], v[2], v[3]);
            }
        }
}

npas_status pitch_launch(const npas_mx_linear_desc &d, const void *x, void *out, cudaStream_t st)
{
    const int pieces = (int)(pitch_of(d) / 8);
    int lanes = 1;
    while (lanes < 32 && lanes < pieces) lanes *= 2;
    const int64_t rows = kPitchThreads / lanes, blocks = ((int64_t)d.M + rows - 1) / rows, most = (int64_t)sm_count() * 32;
    const cudaError_t e = tc::launch_pdl(Launch(), mx_pitch_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kPitchThreads), 0, st, (int64_t)d.M,
                                         (int)d.I, pieces, lanes, static_cast<const uint16_t *>(x), static_cast<uint4 *>(out));
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace

}  // namespace npas

using namespace npas;

extern "C" {

npas_status npas_linear_mx_workspace(const npas_mx_linear_desc *d, size_t *ws_bytes)
{
    if (!ws_bytes) return NPAS_ERR_NULL;
    npas_status s = check_args(d);
    if (s != NPAS_OK) return s;
    *ws_bytes = NPAS_WORKSPACE_BYTES + scratch_bytes(*d);
    return NPAS_OK;
}

npas_status npas_linear_mx_kernel(const npas_mx_linear_desc *d, int32_t *kernel_id)
{
    if (!kernel_id) return NPAS_ERR_NULL;
    npas_status s = check_args(d);
    if (s != NPAS_OK) return s;
    *kernel_id = choice_for(*d).kernel;
    return *kernel_id ? NPAS_OK : NPAS_ERR_UNSUPPORTED;
}

npas_status npas_linear_mx(const npas_mx_linear_desc *d, const void *x, const void *w, const float *bias, const void *res, void *y, void *ws,
                           size_t ws_bytes, void *stream)
{
    if (ws && ws_bytes < NPAS_WORKSPACE_BYTES) return NPAS_ERR_BUFFER_TOO_SMALL;
    return npas_internal_linear_mx(d, x, w, bias, res, y, ws, ws ? static_cast<uint8_t *>(ws) + NPAS_WORKSPACE_BYTES : nullptr,
                                   ws_bytes - NPAS_WORKSPACE_BYTES, stream);
}

npas_status npas_internal_linear_mx(const npas_mx_linear_desc *d, const void *x, const void *w, const float *bias, const void *res, void *y, void *ws,
                                    void *scratch, size_t scratch_size, void *stream)
{
    npas_status s = check_args(d);
    if (s != NPAS_OK) return s;
    if (!x || !w || !y || !ws || (d->has_bias && !bias) || (d->has_residual && !res)) return NPAS_ERR_NULL;
    if (!d->has_bias) bias = nullptr;
    if (!d->has_residual) res = nullptr;
    for (const void *q : {x, w, static_cast<const void *>(y), static_cast<const void *>(ws), res, static_cast<const void *>(bias)})
        if (q && !aligned16(q)) return NPAS_ERR_ALIGNMENT;
    if (x == y || w == y || res == y) return NPAS_ERR_UNSUPPORTED;
    const Choice choice = choice_for(*d);
    const int kernel = choice.kernel;
    if (!kernel) return NPAS_ERR_UNSUPPORTED;
    if (scratch_size < scratch_bytes(*d)) return NPAS_ERR_BUFFER_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    npas_mx_linear_desc in = *d;
    in.variant = choice.variant;
    if (d->quantize_x && !(kernel == 3 && quantizes_itself(*d))) {
        const npas_mx_desc q = {d->M, d->I, NPAS_BF16};
        s = quantize_mx_launch(q, x, scratch, st);
        if (s != NPAS_OK) return s;
        x = scratch;
        in = behind_quantize(in);
    }
    int64_t pitch = d->I;
    if (needs_pitch(*d, kernel)) {
        s = pitch_launch(*d, x, scratch, st);
        if (s != NPAS_OK) return s;
        x = scratch;
        pitch = pitch_of(*d);
    }
    switch (kernel) {
        case 1: return linear_mx_simt_launch(in, x, w, bias, res, y, st);
        case 3: return linear_mx_sw_launch(in, x, pitch, w, bias, res, y, static_cast<uint32_t *>(ws), st);
        case 6: return linear_mx_gv_launch(in, x, pitch, w, bias, res, y, st);
        case 5: return linear_mx_d2_launch(in, x, w, bias, res, y, static_cast<uint32_t *>(ws), st);
        case 4: return linear_mx_ps_launch(in, x, pitch, w, bias, res, y, static_cast<uint32_t *>(ws), st);
    }
    return NPAS_ERR_UNSUPPORTED;
}

}  // extern "C"
