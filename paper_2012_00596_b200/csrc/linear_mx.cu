// Entry points of the GEMM with microscaled 4-bit weights: argument checks, workspace, the choice of a kernel.
#include "internal_api.h"
#include "mx.cuh"
#include "tc_common.cuh"

namespace npas {

namespace {

npas_status check_args(const npas_mx_linear_desc *d)
{
    if (!d) return NPAS_ERR_NULL;
    const npas_mx_desc w = {d->O, d->I, NPAS_BF16}, x = {d->M, d->I, NPAS_BF16};
    npas_status s = check_mx_desc(&w);
    if (s == NPAS_OK) s = check_mx_desc(&x);
    if (s != NPAS_OK) return s;
    if (d->x_dtype != NPAS_BF16 && d->x_dtype != NPAS_MX4) return NPAS_ERR_DTYPE;
    if (d->quantize_x && d->x_dtype != NPAS_BF16) return NPAS_ERR_DTYPE;
    if (d->y_dtype != NPAS_F32 && d->y_dtype != NPAS_BF16) return NPAS_ERR_DTYPE;
    return NPAS_OK;
}

// 1: CUDA cores, 3: few rows, 4: persistent tiles, 5: the same on CTA pairs, 6: a 16-bit input of up to 16 rows.  0: the requested path does not take the geometry.
// Up to 16 rows the kernel for few rows quantises the input itself: every CTA its share, again for every 128 outputs.  (FIXME)
bool quantizes_itself(const npas_mx_linear_desc &d) { return d.quantize_x && d.M <= 16; }

npas_mx_linear_desc behind_quantize(npas_mx_linear_desc d)
{
    if (d.quantize_x) { d.x_dtype = NPAS_MX4; d.quantize_x = 0; }
    return d;
}

int kernel_for(const npas_mx_linear_desc &d)
{
    const npas_mx_linear_desc in = behind_quantize(d);
    switch (d.path) {
        case 1: return d.variant ? 0 : 1;
        case 3: return linear_mx_sw_supported(in) ? 3 : 0;
        case 4: return linear_mx_ps_supported(in) ? 4 : 0;
        case 5: return linear_mx_d2_supported(in) ? 5 : 0;
        case 6: return linear_mx_gv_supported(in) ? 6 : 0;
        case 0: case 2: break;
        default: return 0;
    }
    if (linear_mx_gv_supported(in)) return 6;
    if (d.M > 128 && d.O > 128 && d.I >= 2048 && linear_mx_d2_supported(in)) return 5;
    if (d.M > 128 && linear_mx_ps_supported(in)) return 4;
    if (linear_mx_sw_supported(in)) return 3;
    return d.path == 2 ? 0 : 1;
}

// Rows of a 16-bit input that do not start on 16-byte boundaries are copied to a pitch that does: the tensor cores' kernels load by TMA.
bool needs_pitch(const npas_mx_linear_desc &d, int kernel) { return kernel != 1 && d.x_dtype == NPAS_BF16 && !d.quantize_x && d.I % 8 != 0; }
int64_t pitch_of(const npas_mx_linear_desc &d) { return ((int64_t)d.I + 7) / 8 * 8; }

// scratch behind the status words: the quantised input, or the copied one
size_t scratch_bytes(const npas_mx_linear_desc &d)
{
    const int kernel = kernel_for(d);
    if (d.quantize_x) return kernel == 3 && quantizes_itself(d) ? 0 : mx_layout(d.M, d.I).total;
    return needs_pitch(d, kernel) ? (size_t)d.M * pitch_of(d) * 2 : 0;
}

constexpr int kPitchThreads = 256;

// A thread writes 16 bytes of a row; columns past the end are zeros.
__global__ void __launch_bounds__(kPitchThreads) mx_pitch_kernel(int64_t M, int I, int64_t pieces, const uint16_t *x, uint4 *out)
{
    tc::pdl_trigger();
    tc::pdl_wait();
    x = tc::behind_wait(x);
    for (int64_t i = (int64_t)blockIdx.x * kPitchThreads + threadIdx.x; i < M * pieces; i += (int64_t)gridDim.x * kPitchThreads) {
        const int64_t row = i / pieces;
        const int c = (int)(i - row * pieces) * 8;
        uint32_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < I ? x[row * I + c + j] : 0u;
        out[i] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
    }
}

npas_status pitch_launch(const npas_mx_linear_desc &d, const void *x, void *out, cudaStream_t st)
{
    const int64_t pieces = pitch_of(d) / 8, blocks = (d.M * pieces + kPitchThreads - 1) / kPitchThreads, most = (int64_t)sm_count() * 16;
    const cudaError_t e = tc::launch_pdl(Launch(), mx_pitch_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kPitchThreads), 0, st, (int64_t)d.M,
                                         (int)d.I, pieces, static_cast<const uint16_t *>(x), static_cast<uint4 *>(out));
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
    *kernel_id = kernel_for(*d);
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
    const int kernel = kernel_for(*d);
    if (!kernel) return NPAS_ERR_UNSUPPORTED;
    if (scratch_size < scratch_bytes(*d)) return NPAS_ERR_BUFFER_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    npas_mx_linear_desc in = *d;
    if (d->quantize_x && !(kernel == 3 && quantizes_itself(*d))) {
        const npas_mx_desc q = {d->M, d->I, NPAS_BF16};
        s = quantize_mx_launch(q, x, scratch, st, Launch());
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
