// GEMM with microscaled 4-bit weights on CUDA cores, fp32: every geometry, the kernel the others are checked against.
//
// Y[m,o] = act(bias[o] + sum_i X[m,i] W[o,i] + residual[m,o]).  A block of threads takes 64 rows x 64 outputs and walks the columns
// a scale block (32) at a time: elements are widened to their fp32 values on the way into shared memory, a thread multiplies
// a 4 x 4 corner.  Bound by the FMA pipe (128 a cycle and SM).
#include "mx.cuh"
#include "tc_common.cuh"

namespace npas {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;

// Eight columns of a row of a blob as floats (zeros for rows past the end).
__device__ __forceinline__ void mx_load8(float (&v)[8], const uint8_t *blob, const MxLayout &L, int64_t row, int64_t rows, int c)
{
    const bool in = row < rows && (uint32_t)c < 2 * L.pitch;
    const uint32_t word = in ? *reinterpret_cast<const uint32_t *>(blob + L.off_values + (uint64_t)row * L.pitch + c / 2) : 0u;
    const uint32_t code = in ? blob[L.off_scales + ((uint64_t)(row / kMxTileRows) * L.nKT + c / kMxTileCols) * kMxScaleTile +
                                    mx_scale_at((uint32_t)(row % kMxTileRows), (uint32_t)c / kMxBlock)] : 0u;
    const float s = mx_scale_value(code);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = mx_element_value(mx_nibble(word, i)) * s;
}

template <bool kMx>
__global__ void __launch_bounds__(kThreads)
linear_mx_simt_kernel(int M, int I, int O, int relu, int y_bf16, const void *x, const uint8_t *w, const float *bias, const void *res, void *y)
{
    __shared__ float xs[kMxBlock][kTile + 4], wsm[kMxBlock][kTile + 4];
    tc::pdl_trigger();
    tc::pdl_wait();
    x = tc::behind_wait(x); w = tc::behind_wait(w); bias = tc::behind_wait(bias); res = tc::behind_wait(res);
    const int nNT = (O + kTile - 1) / kTile, mt = blockIdx.x / nNT, nt = blockIdx.x - mt * nNT;
    const int r = threadIdx.x >> 2, c8 = (threadIdx.x & 3) * 8, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t row = (int64_t)mt * kTile + r;
    const MxLayout LW = mx_layout(O, I), LX = mx_layout(M, I);
    float acc[4][4] = {};
    for (int c0 = 0; c0 < I; c0 += kMxBlock) {
        float v[8];
        if (kMx) mx_load8(v, static_cast<const uint8_t *>(x), LX, row, M, c0 + c8);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = row < M && c0 + c8 + i < I ? bf16_bits_to_f32(static_cast<const uint16_t *>(x)[row * I + c0 + c8 + i]) : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) xs[c8 + i][r] = v[i];
        mx_load8(v, w, LW, (int64_t)nt * kTile + r, O, c0 + c8);
#pragma unroll
        for (int i = 0; i < 8; ++i) wsm[c8 + i][r] = v[i];
        __syncthreads();
        const int n = min(kMxBlock, I - c0);
        for (int k = 0; k < n; ++k) {
            const float4 a = *reinterpret_cast<const float4 *>(&xs[k][ty * 4]), b = *reinterpret_cast<const float4 *>(&wsm[k][tx * 4]);
            const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t m = (int64_t)mt * kTile + ty * 4 + i;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int o = nt * kTile + tx * 4 + j;
            if (m >= M || o >= O) continue;
            const int64_t at = m * O + o;
            float v = acc[i][j];
            if (bias) v += bias[o];
            if (res) v += y_bf16 ? bf16_bits_to_f32(static_cast<const uint16_t *>(res)[at]) : static_cast<const float *>(res)[at];
            if (relu) v = fmaxf(v, 0.f);
            if (y_bf16) static_cast<uint16_t *>(y)[at] = (uint16_t)tc::cvt_bf16x2(v, 0.f);
            else static_cast<float *>(y)[at] = v;
        }
    }
}

}  // namespace

npas_status linear_mx_simt_launch(const npas_mx_linear_desc &d, const void *x, const void *w, const float *bias, const void *res, void *y,
                                  cudaStream_t st)
{
    const int64_t tiles = ((int64_t)d.M + kTile - 1) / kTile * ((d.O + kTile - 1) / kTile);
    if (tiles > 0x7FFFFFFF) return NPAS_ERR_SHAPE;
    const cudaError_t e = tc::launch_pdl(Launch(), d.x_dtype == NPAS_MX4 ? linear_mx_simt_kernel<true> : linear_mx_simt_kernel<false>, dim3((unsigned)tiles),
                                         dim3(kThreads), 0, st, d.M, d.I, d.O, (int)d.relu, (int)(d.y_dtype == NPAS_BF16), x, static_cast<const uint8_t *>(w),
                                         bias, res, y);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
