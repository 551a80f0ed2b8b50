// Quantisation to microscaled 4-bit floating point and back.
//
// A block of 32 columns of a row with largest magnitude a gets the scale 2^s, s = max(floor(log2 a) - 2, -127): a / 2^s lies in
// [4, 8) and 6 is the largest element.  Every element is divided by 2^s (exact) and rounded to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6,
// ties to the even mantissa, what is past 6 to 6.  A block that holds an infinity or a NaN gets the NaN scale.  s comes from the
// exponent bits of a, so there is no rounding before the one to four bits, and equal inputs give equal blobs on every GPU.
//
// What bounds both directions: bytes (2.53 per bf16 element, 4.53 per fp32 one).  A block of threads takes 128 rows x 128 columns,
// which is one 512-byte tile of scales: 16 lanes share a row with eight columns each (one 16-byte load of bf16, one word of
// nibbles stored), a block's maximum crosses four lanes, eight rows' loads of a thread are in flight together, and the tile of scales
// is put together in shared memory and leaves in whole sectors.
#include "mx.cuh"
#include "tc_common.cuh"

namespace npas {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerPass = kThreads / 16;
constexpr int kPasses = kMxTileRows / kRowsPerPass;

// Eight floats -> a word of e2m1 elements in the order of mx_nibble: to nearest even, past 6 to 6.
__device__ __forceinline__ uint32_t cvt_e2m1x8(const float (&v)[8])
{
    uint32_t d;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %3, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %7, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %4, %2;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %6;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(d) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return d;
}

// Eight columns of a row as floats, zeros past the end.  `whole`: rows start on 16-byte boundaries and 8 divides the columns.
template <typename T>
__device__ __forceinline__ void load8(float (&v)[8], const T *row, int c, int cols, bool whole)
{
    if (whole) {
        if constexpr (sizeof(T) == 2) {
            uint4 u = make_uint4(0, 0, 0, 0);
            if (c < cols) u = *reinterpret_cast<const uint4 *>(row + c);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
        } else {
            float4 a = make_float4(0, 0, 0, 0), b = a;
            if (c < cols) { a = *reinterpret_cast<const float4 *>(row + c); b = *reinterpret_cast<const float4 *>(row + c + 4); }
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 2) v[i] = c + i < cols ? bf16_bits_to_f32(row[c + i]) : 0.f;
        else v[i] = c + i < cols ? row[c + i] : 0.f;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) quantize_mx_kernel(int rows, int cols, int whole, const T *src, uint8_t *blob)
{
    __shared__ uint32_t scales[kMxTileRows];            // word (r % 32) * 4 + r / 32: the four codes of row r
    const MxLayout L = mx_layout(rows, cols);
    const uint32_t rt = blockIdx.x / L.nKT, kt = blockIdx.x - rt * L.nKT;
    const int lane16 = threadIdx.x & 15, r0 = threadIdx.x >> 4, c = (int)(kt * kMxTileCols) + lane16 * 8;
    tc::pdl_trigger();
    tc::pdl_wait();
    src = tc::behind_wait(src);
    blob = tc::behind_wait(blob);
    uint8_t *values = blob + L.off_values;
    const bool stored = (uint32_t)c < 2 * L.pitch;
    float v[kPasses][8];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int64_t row = (int64_t)rt * kMxTileRows + p * kRowsPerPass + r0;
        if (row < rows) load8(v[p], src + row * cols, c, cols, whole);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[p][i] = 0.f;
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int r = p * kRowsPerPass + r0;
        const int64_t row = (int64_t)rt * kMxTileRows + r;
        // largest magnitude as a bit pattern: infinities and NaN come out above every number
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[p][i]) & 0x7FFFFFFFu);
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t e = top >> 23, code = e == 255 ? 255u : e > 2 ? e - 2 : 0u;
        const float inv = __uint_as_float((254u - min(code, 253u)) << 23);       // 2^(127 - code); the NaN block's elements mean nothing
#pragma unroll
        for (int i = 0; i < 8; ++i) v[p][i] *= inv;
        const uint32_t word = code == 255 ? 0u : cvt_e2m1x8(v[p]);
        if (row < rows && stored) *reinterpret_cast<uint32_t *>(values + (uint64_t)row * L.pitch + c / 2) = word;
        uint32_t codes = row < rows && c < cols ? code << (8 * (lane16 >> 2)) : 0u;
        // (a short last block has lanes past the end that must not hide its code)
        codes |= __shfl_xor_sync(0xFFFFFFFFu, codes, 1); codes |= __shfl_xor_sync(0xFFFFFFFFu, codes, 2);
        codes |= __shfl_xor_sync(0xFFFFFFFFu, codes, 4); codes |= __shfl_xor_sync(0xFFFFFFFFu, codes, 8);
        if (lane16 == 0) scales[(r & 31) * 4 + (r >> 5)] = codes;
    }
    __syncthreads();
    if (threadIdx.x < kMxTileRows)
        reinterpret_cast<uint32_t *>(blob + L.off_scales + (uint64_t)blockIdx.x * kMxScaleTile)[threadIdx.x] = scales[threadIdx.x];
    // header, and the padding behind the last row
    if (blockIdx.x == 0 && threadIdx.x < 32) {
        uint32_t h = 0;
        switch (threadIdx.x) {
            case MX_MAGIC: h = kMagicMX; break;
            case MX_VERSION: h = kVersionMX; break;
            case MX_ROWS: h = (uint32_t)rows; break;
            case MX_COLS: h = (uint32_t)cols; break;
            case MX_PITCH: h = L.pitch; break;
            case MX_OFF_SCALES: h = (uint32_t)L.off_scales; break;
            case MX_OFF_VALUES_LO: h = (uint32_t)L.off_values; break;
            case MX_OFF_VALUES_HI: h = (uint32_t)(L.off_values >> 32); break;
            case MX_TOTAL_LO: h = (uint32_t)L.total; break;
            case MX_TOTAL_HI: h = (uint32_t)(L.total >> 32); break;
        }
        reinterpret_cast<uint32_t *>(blob)[threadIdx.x] = h;
        const uint64_t end = (uint64_t)rows * L.pitch;
        for (uint64_t at = end + threadIdx.x * 4; at < L.total - L.off_values; at += 128) *reinterpret_cast<uint32_t *>(values + at) = 0u;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *row, int c, int cols, bool whole, const float (&v)[8])
{
    if (whole) {
        if (c >= cols) return;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(row + c) = make_uint4(tc::cvt_bf16x2(v[0], v[1]), tc::cvt_bf16x2(v[2], v[3]), tc::cvt_bf16x2(v[4], v[5]),
                                                             tc::cvt_bf16x2(v[6], v[7]));
        } else {
            *reinterpret_cast<float4 *>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < cols) {
            if constexpr (sizeof(T) == 2) row[c + i] = (uint16_t)tc::cvt_bf16x2(v[i], 0.f);
            else row[c + i] = v[i];
        }
}

// (element times 2^126, then times the scale: both exact; every value is a bf16 number too, subnormals included)
template <typename T>
__global__ void __launch_bounds__(kThreads) dequantize_mx_kernel(int rows, int cols, int whole, const uint8_t *blob, T *out)
{
    const MxLayout L = mx_layout(rows, cols);
    const uint32_t rt = blockIdx.x / L.nKT, kt = blockIdx.x - rt * L.nKT;
    const int lane16 = threadIdx.x & 15, r0 = threadIdx.x >> 4, c = (int)(kt * kMxTileCols) + lane16 * 8;
    tc::pdl_trigger();
    tc::pdl_wait();
    blob = tc::behind_wait(blob);
    out = tc::behind_wait(out);
    if (c >= cols) return;
    const uint8_t *scales = blob + L.off_scales + (uint64_t)blockIdx.x * kMxScaleTile, *values = blob + L.off_values;
    uint32_t word[kPasses], code[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int r = p * kRowsPerPass + r0;
        const int64_t row = (int64_t)rt * kMxTileRows + r;
        word[p] = row < rows ? *reinterpret_cast<const uint32_t *>(values + (uint64_t)row * L.pitch + c / 2) : 0u;
        code[p] = row < rows ? scales[mx_scale_at((uint32_t)r, (uint32_t)lane16 >> 2)] : 0u;
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int64_t row = (int64_t)rt * kMxTileRows + p * kRowsPerPass + r0;
        if (row >= rows) break;
        const float s = mx_scale_value(code[p]);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = mx_element_value(mx_nibble(word[p], i)) * s;
        store8(out + row * cols, c, cols, whole, v);
    }
}

}  // namespace

npas_status quantize_mx_launch(const npas_mx_desc &d, const void *src, void *blob, cudaStream_t st, Launch how)
{
    const MxLayout L = mx_layout(d.rows, d.cols);
    const dim3 grid(L.nRT * L.nKT), block(kThreads);
    const int whole = d.cols % 8 == 0;
    cudaError_t e;
    if (d.src_dtype == NPAS_BF16)
        e = tc::launch_pdl(how, quantize_mx_kernel<uint16_t>, grid, block, 0, st, d.rows, d.cols, whole, static_cast<const uint16_t *>(src),
                           static_cast<uint8_t *>(blob));
    else
        e = tc::launch_pdl(how, quantize_mx_kernel<float>, grid, block, 0, st, d.rows, d.cols, whole, static_cast<const float *>(src),
                           static_cast<uint8_t *>(blob));
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas

using namespace npas;

extern "C" {

npas_status npas_quantize_mx_size(const npas_mx_desc *d, size_t *blob_bytes)
{
    if (!blob_bytes) return NPAS_ERR_NULL;
    npas_status s = check_mx_desc(d);
    if (s != NPAS_OK) return s;
    *blob_bytes = mx_layout(d->rows, d->cols).total;
    return NPAS_OK;
}

npas_status npas_quantize_mx(const npas_mx_desc *d, const void *src, void *blob, size_t blob_bytes, void *stream)
{
    npas_status s = check_mx_desc(d);
    if (s != NPAS_OK) return s;
    if (!src || !blob) return NPAS_ERR_NULL;
    if (!aligned16(src) || !aligned16(blob)) return NPAS_ERR_ALIGNMENT;
    if (blob_bytes < mx_layout(d->rows, d->cols).total) return NPAS_ERR_BUFFER_TOO_SMALL;
    if (src == blob) return NPAS_ERR_UNSUPPORTED;
    return quantize_mx_launch(*d, src, blob, static_cast<cudaStream_t>(stream), Launch());
}

npas_status npas_dequantize_mx(const npas_mx_desc *d, const void *blob, size_t blob_bytes, int32_t out_dtype, void *out, void *stream)
{
    npas_status s = check_mx_desc(d);
    if (s != NPAS_OK) return s;
    if (!blob || !out) return NPAS_ERR_NULL;
    if (out_dtype != NPAS_F32 && out_dtype != NPAS_BF16) return NPAS_ERR_DTYPE;
    if (!aligned16(blob) || !aligned16(out)) return NPAS_ERR_ALIGNMENT;
    const MxLayout L = mx_layout(d->rows, d->cols);
    if (blob_bytes < L.total) return NPAS_ERR_BUFFER_TOO_SMALL;
    if (blob == out) return NPAS_ERR_UNSUPPORTED;
    const dim3 grid(L.nRT * L.nKT), block(kThreads);
    const int whole = d->cols % 8 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (out_dtype == NPAS_BF16)
        e = tc::launch_pdl(Launch(), dequantize_mx_kernel<uint16_t>, grid, block, 0, st, d->rows, d->cols, whole, static_cast<const uint8_t *>(blob),
                           static_cast<uint16_t *>(out));
    else
        e = tc::launch_pdl(Launch(), dequantize_mx_kernel<float>, grid, block, 0, st, d->rows, d->cols, whole, static_cast<const uint8_t *>(blob),
                           static_cast<float *>(out));
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

npas_status npas_mx_blob_check(const npas_mx_desc *d, const void *blob, size_t blob_bytes, void *stream)
{
    npas_status s = check_mx_desc(d);
    if (s != NPAS_OK) return s;
    if (!blob) return NPAS_ERR_NULL;
    const MxLayout L = mx_layout(d->rows, d->cols);
    if (blob_bytes < L.total) return NPAS_ERR_BUFFER_TOO_SMALL;
    uint32_t h[32];
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(h, blob, sizeof(h), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) return NPAS_ERR_CUDA;
    const bool ok = h[MX_MAGIC] == kMagicMX && h[MX_VERSION] == kVersionMX && h[MX_ROWS] == (uint32_t)d->rows && h[MX_COLS] == (uint32_t)d->cols &&
                    h[MX_PITCH] == L.pitch && h[MX_OFF_SCALES] == L.off_scales && h[MX_OFF_VALUES_LO] == (uint32_t)L.off_values &&
                    h[MX_OFF_VALUES_HI] == (uint32_t)(L.off_values >> 32) && h[MX_TOTAL_LO] == (uint32_t)L.total &&
                    h[MX_TOTAL_HI] == (uint32_t)(L.total >> 32);
    return ok ? NPAS_OK : NPAS_ERR_BLOB;
}

}  // extern "C"
