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
// is put together in shared memory and leaves in whole sectors.  Maxima and scaling on pairs of bf16: with every element as a float
// 125 instructions for eight of them bound it (200704x256 57 us, now 21.2 to 22.5: 89 to 94 % of the copy rate; fp32 37, 97 %; back 22.3, 89 %, and
// 38.7, 92 %).  Rows off 16-byte boundaries: 2.4 times the instructions, which bound both ways (100000x1003 bf16 issues in 73 % of the cycles, back in 92 %).
#include <type_traits>

#include "mx_tc.cuh"

namespace npas {

namespace {

constexpr int kThreads = 256;

// kWhole: mx_load_whole can be used; else a block has half a tile at most (its loads take more registers)
template <typename T, bool kParts, int kLanes, bool kWhole>
__global__ void __launch_bounds__(kThreads) quantize_mx_kernel(int rows, int cols, int n_parts, const T *src, uint8_t *blob)
{
    __shared__ __align__(16) uint8_t scales[kMxScaleTile];
    const MxLayout L = mx_layout(rows, cols);
    constexpr int kRowsPerPass = kThreads / kLanes, kTilePasses = kMxTileRows / kRowsPerPass, kPasses = kWhole ? kTilePasses : 4;
    const int parts = kParts ? n_parts : 1;
    const uint32_t tile = blockIdx.x / parts, part = blockIdx.x - tile * parts, rt = tile / L.nKT, kt = tile - rt * L.nKT;
    const int rows_part = kMxTileRows / parts, row_lo = (int)part * rows_part;   // this block's rows of the tile
    const int lane = threadIdx.x % kLanes, r0 = row_lo + threadIdx.x / kLanes, c = (int)(kt * kMxTileCols) + lane * 8;
    const int rows_here = min(rows - (int)(rt * kMxTileRows) - row_lo, rows_part), left = rows_here + row_lo - r0;   // pass p has a row where p * kRowsPerPass < left
    tc::pdl_trigger();
    tc::pdl_wait();
    src = tc::behind_wait(src);
    blob = tc::behind_wait(blob);
    uint8_t *values = blob + L.off_values;
    // passes that have rows (a tile of few rows is latency: one row of 2048 columns took 2.2 us with all eight)
    const int passes = (max(rows_here, 0) + kRowsPerPass - 1) / kRowsPerPass;
    if (kLanes < 16 || passes < kTilePasses) {
        if (threadIdx.x < kMxTileRows) reinterpret_cast<uint32_t *>(scales)[threadIdx.x] = 0u;
        __syncthreads();
    }
    constexpr int W = sizeof(T) == 2 ? 4 : 8;
    typename std::conditional<kWhole, uint32_t[W], tc::MxRaw<W>>::type raw[kPasses];
    const int64_t row0 = (int64_t)rt * kMxTileRows + r0;
    const T *from = src + row0 * cols + c, *end = src + (int64_t)rows * cols;
    const int n = max(0, min(cols - c, 8));
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        if (p >= passes) break;
        const bool there = p * kRowsPerPass < left && n > 0;
        if constexpr (kWhole) tc::mx_load_whole(raw[p], from + (int64_t)p * kRowsPerPass * cols, there);
        else tc::mx_load_raw(raw[p], from + (int64_t)p * kRowsPerPass * cols, there ? n : 0, end);
    }
    uint8_t *to = values + (uint64_t)row0 * L.pitch + c / 2;
    const bool stored = (uint32_t)c < 2 * L.pitch;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        if (p >= passes) break;
        const int r = p * kRowsPerPass + r0;
        uint32_t v[W];
        if constexpr (kWhole) {
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = raw[p][i];
        } else {
            tc::mx_align(v, raw[p], from + (int64_t)p * kRowsPerPass * cols, p * kRowsPerPass < left ? n : 0);
        }
        uint32_t top = tc::mx_top8(v);
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t code = tc::mx_code(top);
        float f[8];
        tc::mx_scaled8(f, v, code);
        const uint32_t word = tc::mx_cvt_e2m1x8(f);
        if (p * kRowsPerPass < left && stored) *reinterpret_cast<uint32_t *>(to) = code == 255 ? 0u : word;
        to += (uint64_t)kRowsPerPass * L.pitch;
        if ((lane & 3) == 0) scales[mx_scale_at((uint32_t)r, (uint32_t)lane >> 2)] = (uint8_t)code;   // (rows and blocks past the end: 0)
    }
    __syncthreads();
    if ((int)threadIdx.x < rows_part) {
        // the whole tile in order, or the words of this block's rows
        const int r = row_lo + (int)threadIdx.x, word = parts == 1 ? (int)threadIdx.x : (r & 31) * 4 + (r >> 5);
        reinterpret_cast<uint32_t *>(blob + L.off_scales + (uint64_t)tile * kMxScaleTile)[word] = reinterpret_cast<const uint32_t *>(scales)[word];
    }
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
__device__ __forceinline__ void store8(T *row, int c, const float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4 *>(row + c) = make_uint4(tc::cvt_bf16x2(v[0], v[1]), tc::cvt_bf16x2(v[2], v[3]), tc::cvt_bf16x2(v[4], v[5]),
                                                         tc::cvt_bf16x2(v[6], v[7]));
    } else {
        uint32_t o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(v[i]);
        tc::st_sector(row + c, o);
    }
}

// Eight bf16 values a lane of rows that start anywhere: the lanes of a row put its aligned 16-byte pieces together from their own words and
// the next lane's, what lies before the first and behind the last piece leaves in 8, 4 and 2 bytes.  `bytes`: of the row's part in this tile, zero
// where there is no row.  (With a store per value 100000x1003 took 109 us, 72 so.  fp32 values leave one by one, neighbouring lanes neighbouring
// columns: 60000x1003 78 us, in pieces 88.)
template <int kLanes>
__device__ __forceinline__ void store_pieces(void *row, int lane, int bytes, const uint32_t (&own)[4])
{
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = own[i];
        w[4 + i] = __shfl_down_sync(0xFFFFFFFFu, own[i], 1, kLanes);
    }
    const uint32_t s = (16u - (uint32_t)reinterpret_cast<uintptr_t>(row)) & 15u;          // bytes before the first piece
    char *base = static_cast<char *>(row);
    if (lane == 0 && s && bytes) {
        if (bytes >= (int)s) {
            char *to = base;
            uint32_t a = own[0], b = own[1], c = own[2];
            if (s & 2u) {
                *reinterpret_cast<uint16_t *>(to) = (uint16_t)a;
                to += 2;
                a = __funnelshift_r(a, b, 16); b = __funnelshift_r(b, c, 16); c = __funnelshift_r(c, own[3], 16);
            }
            if (s & 4u) { *reinterpret_cast<uint32_t *>(to) = a; to += 4; a = b; b = c; }
            if (s & 8u) *reinterpret_cast<uint2 *>(to) = make_uint2(a, b);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (4 * i < bytes) reinterpret_cast<uint16_t *>(base)[2 * i] = (uint16_t)own[i];
                if (4 * i + 2 < bytes) reinterpret_cast<uint16_t *>(base)[2 * i + 1] = (uint16_t)(own[i] >> 16);
            }
        }
    }
    if (s & 8u) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (s & 4u) {
#pragma unroll
        for (int i = 0; i < 7; ++i) w[i] = w[i + 1];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 8 * (s & 2u));
    const int at = (int)s + 16 * lane, left = bytes - at;
    if (left >= 16) *reinterpret_cast<uint4 *>(base + at) = make_uint4(w[0], w[1], w[2], w[3]);
    else if (left > 0) {
        char *to = base + at;
        uint32_t a = w[0], b = w[1];
        if (left & 8) { *reinterpret_cast<uint2 *>(to) = make_uint2(a, b); to += 8; a = w[2]; b = w[3]; }
        if (left & 4) { *reinterpret_cast<uint32_t *>(to) = a; to += 4; a = b; }
        if (left & 2) *reinterpret_cast<uint16_t *>(to) = (uint16_t)a;
    }
}

// (element times 2^126, then times the scale: both exact; every value is a bf16 number too, subnormals included)
template <typename T, bool kParts, int kLanes>
__global__ void __launch_bounds__(kThreads) dequantize_mx_kernel(int rows, int cols, int whole, int n_parts, const uint8_t *blob, T *out)
{
    const MxLayout L = mx_layout(rows, cols);
    constexpr int kRowsPerPass = kThreads / kLanes, kPasses = kMxTileRows / kRowsPerPass;
    const int parts = kParts ? n_parts : 1;
    const uint32_t tile = blockIdx.x / parts, part = blockIdx.x - tile * parts, rt = tile / L.nKT, kt = tile - rt * L.nKT;
    const int rows_part = kMxTileRows / parts, row_lo = (int)part * rows_part;
    const int lane = threadIdx.x % kLanes, r0 = row_lo + threadIdx.x / kLanes;
    tc::pdl_trigger();
    tc::pdl_wait();
    blob = tc::behind_wait(blob);
    out = tc::behind_wait(out);
    const uint8_t *scales = blob + L.off_scales + (uint64_t)tile * kMxScaleTile;
    const int64_t row0 = (int64_t)rt * kMxTileRows + r0;
    const uint8_t *from = blob + L.off_values + (uint64_t)row0 * L.pitch + kt * (kMxTileCols / 2);
    T *to = out + row0 * cols + kt * kMxTileCols;
    const int left = min(rows - (int)(rt * kMxTileRows), row_lo + rows_part) - r0, width = cols - (int)(kt * kMxTileCols);
    if (sizeof(T) == 4 && !whole) {
        for (int p = 0; p * kRowsPerPass < left; ++p) {
            const uint32_t codes = *reinterpret_cast<const uint32_t *>(scales + mx_scale_at((uint32_t)(p * kRowsPerPass + r0), 0));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = i * kLanes + lane;
                if (c < width)
                    to[c] = mx_element_value(mx_nibble(reinterpret_cast<const uint32_t *>(from)[c >> 3], c & 7)) * mx_scale_value(codes >> (8 * (c >> 5)) & 255u);
            }
            from += (uint64_t)kRowsPerPass * L.pitch;
            to += (int64_t)kRowsPerPass * cols;
        }
        return;
    }
    uint32_t word[kPasses], code[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const bool in = p * kRowsPerPass < left && lane * 8 < width;
        word[p] = in ? reinterpret_cast<const uint32_t *>(from)[lane] : 0u;
        code[p] = in ? scales[mx_scale_at((uint32_t)(p * kRowsPerPass + r0), (uint32_t)lane >> 2)] : 0u;
        from += (uint64_t)kRowsPerPass * L.pitch;
    }
    auto values = [&](float (&v)[8], int p) {
        const float s = mx_scale_value(code[p]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = mx_element_value(mx_nibble(word[p], i)) * s;
    };
    if (whole) {
        if (lane * 8 >= width) return;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            if (p * kRowsPerPass >= left) break;
            float v[8];
            values(v, p);
            store8(to, lane * 8, v);
            to += (int64_t)kRowsPerPass * cols;
        }
        return;
    }
    if constexpr (sizeof(T) == 2) {
        // (the lanes of a warp stay together: they take words from one another)
        const int bytes = min(width, kLanes * 8) * 2, rows_here = min(rows - (int)(rt * kMxTileRows), row_lo + rows_part) - row_lo;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            if (p * kRowsPerPass >= rows_here) break;
            float v[8];
            values(v, p);
            const uint32_t own[4] = {tc::cvt_bf16x2(v[0], v[1]), tc::cvt_bf16x2(v[2], v[3]), tc::cvt_bf16x2(v[4], v[5]), tc::cvt_bf16x2(v[6], v[7])};
            store_pieces<kLanes>(to, lane, p * kRowsPerPass < left ? bytes : 0, own);
            to += (int64_t)kRowsPerPass * cols;
        }
    }
}

// The launch of either kernel.  Up to 64 columns: eight lanes a row instead of sixteen (the rest of the tile is not there).  Small matrices: a
// tile in parts of 64, 32 or 16 rows, so that more SMs have work and a thread has fewer passes.
struct Shape { int narrow, parts, whole; dim3 grid; };
Shape shape_of(const npas_mx_desc &d, const MxLayout &L, bool quantize)
{
    Shape s;
    s.narrow = d.cols <= 64;
    s.whole = d.cols % 8 == 0;
    s.parts = !quantize || s.whole || s.narrow ? 1 : 2;
    const uint64_t tiles = (uint64_t)L.nRT * L.nKT;
    while (s.parts < (s.narrow ? 4 : 8) && tiles * s.parts * 2 <= 6ull * sm_count()) s.parts *= 2;
    s.grid = dim3((unsigned)(tiles * s.parts));
    return s;
}
template <typename T>
cudaError_t quantize_any(const npas_mx_desc &d, const Shape &s, const void *src, void *blob, cudaStream_t st)
{
    const auto kernel = !s.whole ? (s.narrow ? quantize_mx_kernel<T, true, 8, false> : quantize_mx_kernel<T, true, 16, false>)
                      : s.narrow ? (s.parts > 1 ? quantize_mx_kernel<T, true, 8, true> : quantize_mx_kernel<T, false, 8, true>)
                                 : (s.parts > 1 ? quantize_mx_kernel<T, true, 16, true> : quantize_mx_kernel<T, false, 16, true>);
    return tc::launch_pdl(Launch(), kernel, s.grid, dim3(kThreads), 0, st, (int)d.rows, (int)d.cols, s.parts, static_cast<const T *>(src),
                          static_cast<uint8_t *>(blob));
}
template <typename T>
cudaError_t dequantize_any(const npas_mx_desc &d, const Shape &s, const void *blob, void *out, cudaStream_t st)
{
    const auto kernel = s.narrow ? (s.parts > 1 ? dequantize_mx_kernel<T, true, 8> : dequantize_mx_kernel<T, false, 8>)
                                 : (s.parts > 1 ? dequantize_mx_kernel<T, true, 16> : dequantize_mx_kernel<T, false, 16>);
    return tc::launch_pdl(Launch(), kernel, s.grid, dim3(kThreads), 0, st, (int)d.rows, (int)d.cols, s.whole, s.parts, static_cast<const uint8_t *>(blob),
                          static_cast<T *>(out));
}

}  // namespace

npas_status quantize_mx_launch(const npas_mx_desc &d, const void *src, void *blob, cudaStream_t st)
{
    const Shape s = shape_of(d, mx_layout(d.rows, d.cols), true);
    const cudaError_t e = d.src_dtype == NPAS_BF16 ? quantize_any<uint16_t>(d, s, src, blob, st) : quantize_any<float>(d, s, src, blob, st);
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
    return quantize_mx_launch(*d, src, blob, static_cast<cudaStream_t>(stream));
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
    const Shape f = shape_of(*d, L, false);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = out_dtype == NPAS_BF16 ? dequantize_any<uint16_t>(*d, f, blob, out, st) : dequantize_any<float>(*d, f, blob, out, st);
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
