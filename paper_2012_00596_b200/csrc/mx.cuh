// Microscaled 4-bit floating point: the blob's layout, the arithmetic of elements and scales, the launchers of its
// kernels.  An element is e2m1 (sign, two exponent bits, one mantissa bit: 0, 1/2, 1, 3/2, 2, 3, 4, 6), a scale is e8m0
// (a power of two 2^(code - 127), 255 = NaN) shared by 32 consecutive columns of a row.
#pragma once

#include "common.cuh"

namespace npas {

constexpr uint32_t kMagicMX = 0x584D504Eu;  // 'NPMX'
constexpr uint32_t kVersionMX = 1;
constexpr int kMxBlock = 32;                // columns that share a scale
constexpr int kMxTileRows = 128;            // a tile of scales: 128 rows x 4 blocks, 512 bytes
constexpr int kMxTileCols = 4 * kMxBlock;
constexpr uint32_t kMxScaleTile = 512;

enum MxHdr { MX_MAGIC, MX_VERSION, MX_ROWS, MX_COLS, MX_PITCH, MX_OFF_SCALES, MX_OFF_VALUES_LO, MX_OFF_VALUES_HI, MX_TOTAL_LO,
             MX_TOTAL_HI };

// Where things lie in a blob; everything follows from rows and columns.
struct MxLayout {
    uint32_t nRT, nKT;                      // tiles of scales down and across
    uint32_t pitch;                         // bytes of a row of values: whole blocks
    uint64_t off_scales, off_values, total;
};

__host__ __device__ inline MxLayout mx_layout(int rows, int cols)
{
    MxLayout L;
    L.nRT = ((uint32_t)rows + kMxTileRows - 1) / kMxTileRows;
    L.nKT = ((uint32_t)cols + kMxTileCols - 1) / kMxTileCols;
    L.pitch = ((uint32_t)cols + kMxBlock - 1) / kMxBlock * (kMxBlock / 2);
    L.off_scales = 128;
    L.off_values = L.off_scales + (uint64_t)L.nRT * L.nKT * kMxScaleTile;       // multiples of 128
    L.total = L.off_values + ((uint64_t)rows * L.pitch + 127) / 128 * 128;
    return L;
}

// byte of the scale of (row, block) inside its tile
__host__ __device__ inline uint32_t mx_scale_at(uint32_t row, uint32_t block)
{
    return (row % 32) * 16 + (row % 128) / 32 * 4 + block % 4;
}

inline npas_status check_mx_desc(const npas_mx_desc *d)
{
    if (!d) return NPAS_ERR_NULL;
    if (d->rows <= 0 || d->cols <= 0 || d->cols > (1 << 20)) return NPAS_ERR_SHAPE;
    const MxLayout L = mx_layout(d->rows, d->cols);
    if ((uint64_t)L.nRT * L.nKT > 0x7FFFFFFFull) return NPAS_ERR_SHAPE;         // a block of threads per tile of scales
    if (d->src_dtype != NPAS_F32 && d->src_dtype != NPAS_BF16) return NPAS_ERR_DTYPE;
    return NPAS_OK;
}

// 2^(code - 127) as a float; 255 is NaN.  (Code 0 is 2^-127, a subnormal.)
__device__ __forceinline__ float mx_scale_value(uint32_t code)
{
    return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7FC00000u : code << 23);
}

// Element `i` of a word's eight.  Nibble n holds element 2n for n < 4 and 2n - 7 for n >= 4, so that (word >> 4i) & 0x000F000F
// is the pair (2i, 2i + 1): both halves of a pair move together when they are widened to 16 bits.
__device__ __forceinline__ uint32_t mx_nibble(uint32_t word, int i) { return (word >> (4 * (i / 2) + 16 * (i & 1))) & 15u; }

// The element's value: its three magnitude bits are exponent and mantissa of a float 2^126 times smaller, subnormals included
// (both products are exact).
__device__ __forceinline__ float mx_element_value(uint32_t nibble)
{
    return __uint_as_float((nibble & 8u) << 28 | (nibble & 7u) << 22) * 0x1p126f;
}

npas_status quantize_mx_launch(const npas_mx_desc &d, const void *src, void *blob, cudaStream_t st);
// (x_pitch: elements from row to row of a 16-bit input, a multiple of 8; a blob has its own)
bool linear_mx_sw_supported(const npas_mx_linear_desc &d);
npas_status linear_mx_sw_launch(const npas_mx_linear_desc &d, const void *x, int64_t x_pitch, const void *w, const float *bias, const void *res, void *y,
                                uint32_t *ws, cudaStream_t st);
bool linear_mx_ps_supported(const npas_mx_linear_desc &d);
npas_status linear_mx_ps_launch(const npas_mx_linear_desc &d, const void *x, int64_t x_pitch, const void *w, const float *bias, const void *res, void *y,
                                uint32_t *ws, cudaStream_t st);
bool linear_mx_d2_supported(const npas_mx_linear_desc &d);
npas_status linear_mx_d2_launch(const npas_mx_linear_desc &d, const void *x, const void *w, const float *bias, const void *res, void *y, uint32_t *ws,
                                cudaStream_t st);
bool linear_mx_gv_supported(const npas_mx_linear_desc &d);
npas_status linear_mx_gv_launch(const npas_mx_linear_desc &d, const void *x, int64_t x_pitch, const void *w, const float *bias, const void *res, void *y,
                                cudaStream_t st);
npas_status linear_mx_simt_launch(const npas_mx_linear_desc &d, const void *x, const void *w, const float *bias, const void *res, void *y,
                                  cudaStream_t st);

}  // namespace npas
