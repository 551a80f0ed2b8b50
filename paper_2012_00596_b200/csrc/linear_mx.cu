// Entry points of the GEMM with microscaled 4-bit weights: argument checks, workspace, the choice of a kernel.
#include "internal_api.h"
#include "mx.cuh"

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

// 1: CUDA cores.  0: the requested path does not take the geometry.
int kernel_for(const npas_mx_linear_desc &d)
{
    switch (d.path) {
        case 0: case 1: return 1;
    }
    return 0;
}

// scratch behind the status words: the quantised input
size_t scratch_bytes(const npas_mx_linear_desc &d)
{
    return d.quantize_x ? mx_layout(d.M, d.I).total : 0;
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
    if (d->quantize_x) {
        const npas_mx_desc q = {d->M, d->I, NPAS_BF16};
        s = quantize_mx_launch(q, x, scratch, st, Launch());
        if (s != NPAS_OK) return s;
        x = scratch;
        in.x_dtype = NPAS_MX4;
        in.quantize_x = 0;
    }
    return linear_mx_simt_launch(in, x, w, bias, res, y, st);
}

}  // extern "C"
