// tcgen05 wrappers of the kernels on microscaled 4-bit operands: the block-scaled MMA, the copy of scales into tensor memory, the MMA
// whose first operand lies in tensor memory, stores into it.
#pragma once

#include "mx.cuh"
#include "tc_common.cuh"

namespace npas {
namespace tc {

constexpr uint32_t kMxDescHiSw128 = (1024u >> 4) | (1u << 14) | (2u << 29);      // SBO 1024 bytes, version bit, 128-byte swizzle
constexpr uint32_t kMxDescLboOne = 1u << 16;                                     // (LBO is not used by swizzled K-major layouts)
__device__ __forceinline__ uint64_t mx_desc64(uint32_t lo) { return ((uint64_t)kMxDescHiSw128 << 32) | lo; }

// Instruction descriptor: e2m1 x e2m1 -> fp32 with e8m0 scales, both operands K-major, tile M x N, K = 64.  `half`: which two of the
// four scales in a row's 32-bit word belong to this K step.
__host__ __device__ constexpr uint32_t idesc_mxf4(uint32_t M, uint32_t N, uint32_t half)
{
    return (2u * half << 4) | (1u << 7) | (1u << 10) | ((N >> 3) << 17) | (1u << 23) | ((M >> 4) << 24) | (2u * half << 29);
}

// D[tmem] (+)= (A[smem] * scales) (B[smem] * scales); issued by ONE thread.
__device__ __forceinline__ void mma_mxf4_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem, uint32_t sb_tmem,
                                            uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa_tmem), "r"(sb_tmem), "r"(accumulate) : "memory");
}

// The same shared by the two CTAs of a cluster: A 128 rows per CTA, B N/2 rows per CTA, scales of A per CTA, of B in both; ONE thread of the leader.
__device__ __forceinline__ void mma_mxf4_ss_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa_tmem, uint32_t sb_tmem,
                                                 uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa_tmem), "r"(sb_tmem), "r"(accumulate) : "memory");
}

// D[tmem] (+)= A[tmem: bf16 pairs, 128 lanes x 8 columns] * B[smem]; issued by ONE thread.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// A tile of scales (512 bytes: 32 rows of 16 bytes) -> four columns of tensor memory, the same in all four lane quarters.  In
// order with the MMAs that the same thread issues behind it.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t saddr)
{
    const uint64_t desc = smem_desc_kmajor(saddr, 16, 128);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

// eight columns of the warp's lane quarter
__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint4 &a, const uint4 &b)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}

// 32 consecutive 32-bit columns of the warp's lane quarter (thread i writes TMEM lane base + i).
__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 16 lanes x 32 consecutive 32-bit columns: thread t gets, for k = 0..3, columns 8k + 2 (t % 4) and the next of lane t / 4 (r[4k], r[4k + 1])
// and of lane t / 4 + 8 (r[4k + 2], r[4k + 3]): the layout of 8 x 8 matrices that stmatrix takes.
__device__ __forceinline__ void tmem_ld_16x32(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
// four 8 x 8 matrices of 16-bit values, transposed: lane l gives the address of row l % 8 of matrix l / 8
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t saddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(saddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t saddr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr) : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *m, const void *src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(src)), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// A word of eight elements -> four pairs of bf16 values (columns 2i, 2i + 1), times `factor` (mx_factor).  A pair's two nibbles lie 16 bits
// apart: times 2^12 + 2^6 their signs and, once more, their magnitudes come to where a bf16 number has its sign and the last two exponent
// bits and first mantissa bit (elements 2^-126 times their size, subnormals included).  The multiplications take the place of shifts, of
// which an SM does half as many a cycle.
__device__ __forceinline__ void mx_widen_word(uint32_t (&p)[4], uint32_t w, uint32_t factor)
{
    const uint32_t v = w >> 8;
    p[0] = mul_bf16x2(((w & 0x000F000Fu) * 0x1040u) & 0x81C081C0u, factor);
    p[1] = mul_bf16x2(((w & 0x00F000F0u) * 0x0104u) & 0x81C081C0u, factor);
    p[2] = mul_bf16x2(((v & 0x000F000Fu) * 0x1040u) & 0x81C081C0u, factor);
    p[3] = mul_bf16x2(((v & 0x00F000F0u) * 0x0104u) & 0x81C081C0u, factor);
}

// What a block's elements, 2^-126 times their size, are multiplied by to become bf16 values: 2^126 times the scale, in two factors
// where it is past bf16's range (scales above 2).  Both products are exact.
struct MxFactor { uint32_t first, second; };
__device__ __forceinline__ MxFactor mx_factor(uint32_t code)
{
    MxFactor f;
    f.first = (min(code, 128u) + 126u) * 0x00800080u;              // (code 0 to 128: exponents 126 to 254)
    f.second = code == 255u ? 0x7FC07FC0u : code > 128u ? (code - 1u) * 0x00800080u : 0x3F803F80u;
    return f;
}

// 64 columns of a row: two 16-byte pieces of elements, two scale codes -> 32 pairs of bf16 values
__device__ __forceinline__ void mx_widen(uint32_t (&r)[32], const uint4 &a, const uint4 &b, uint32_t code0, uint32_t code1)
{
    const MxFactor f0 = mx_factor(code0), f1 = mx_factor(code1);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t p[4];
        mx_widen_word(p, w[j], j < 4 ? f0.first : f1.first);
        r[4 * j] = p[0]; r[4 * j + 1] = p[1]; r[4 * j + 2] = p[2]; r[4 * j + 3] = p[3];
    }
    if (__any_sync(0xFFFFFFFFu, code0 > 128u || code1 > 128u)) {
#pragma unroll
        for (int j = 0; j < 32; ++j) r[j] = mul_bf16x2(r[j], j < 16 ? f0.second : f1.second);
    }
}

// ---- quantising: eight columns of a row ----------------------------------------------------------------
// Eight floats -> a word of e2m1 elements in the order of mx_nibble: to nearest even, past 6 to 6.
__device__ __forceinline__ uint32_t mx_cvt_e2m1x8(const float (&v)[8])
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

// Eight columns of a row as they are, zeros past the end: bf16 in pairs (four words), fp32 (eight).  `whole`: rows start on 16-byte
// boundaries and 8 divides the columns; else in two halves, the loads and what waits for them: the aligned 16-byte pieces that hold a column
// of them (never one past `end`, where the matrix ends), then the words moved to their places.
template <int W> struct MxRaw {
    uint32_t w[W == 4 ? 8 : 12];
};
template <int W>
__device__ __forceinline__ void mx_load_whole(uint32_t (&v)[W], const void *at, bool there)
{
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = 0u;
    if (!there) return;
    if constexpr (W == 4) {
        const uint4 u = *static_cast<const uint4 *>(at);
        v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    } else {
        ld_sector(v, at);
    }
}
template <int W>
__device__ __forceinline__ void mx_load_raw(MxRaw<W> &r, const void *at, int n, const void *end)
{
    constexpr int kPieces = W == 4 ? 2 : 3, kSize = W == 4 ? 2 : 4;
    const uintptr_t first = reinterpret_cast<uintptr_t>(at), stop = first + (uintptr_t)(n * kSize), last = reinterpret_cast<uintptr_t>(end);
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const uintptr_t a = (first & ~(uintptr_t)15) + 16 * j;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (n > 0 && a < stop) {
            if (a + 16 <= last) u = *reinterpret_cast<const uint4 *>(a);
            else {
                // the matrix ends inside the piece
                uint32_t t[4] = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (a + 4 * i + 4 <= last) t[i] = *reinterpret_cast<const uint32_t *>(a + 4 * i);
                    else if (kSize == 2 && a + 4 * i + 2 <= last) t[i] = *reinterpret_cast<const uint16_t *>(a + 4 * i);
                }
                u = make_uint4(t[0], t[1], t[2], t[3]);
            }
        }
        r.w[4 * j] = u.x; r.w[4 * j + 1] = u.y; r.w[4 * j + 2] = u.z; r.w[4 * j + 3] = u.w;
    }
}
template <int W>
__device__ __forceinline__ void mx_align(uint32_t (&v)[W], const MxRaw<W> &r, const void *at, int n)
{
    constexpr int kN = W == 4 ? 8 : 12;
    const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(at) & 15u;
    uint32_t w[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) w[i] = r.w[i];
    if (off & 8u) {
#pragma unroll
        for (int i = 0; i + 2 < kN; ++i) w[i] = w[i + 2];
    }
    if (off & 4u) {
#pragma unroll
        for (int i = 0; i + 1 < kN; ++i) w[i] = w[i + 1];
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if constexpr (W == 4) {
            v[i] = __funnelshift_r(w[i], w[i + 1], 8 * (off & 3u));
            if (2 * i + 1 >= n) v[i] = 2 * i < n ? v[i] & 0xFFFFu : 0u;
        } else {
            v[i] = i < n ? w[i] : 0u;
        }
    }
}

// largest magnitude of the eight, the upper half of its bits (infinities and NaN come out above every number)
template <int W>
__device__ __forceinline__ uint32_t mx_top8(const uint32_t (&v)[W])
{
    if constexpr (W == 4) {
        uint32_t m = __vmaxu2(__vmaxu2(v[0] & 0x7FFF7FFFu, v[1] & 0x7FFF7FFFu), __vmaxu2(v[2] & 0x7FFF7FFFu, v[3] & 0x7FFF7FFFu));
        return max(m & 0xFFFFu, m >> 16);
    } else {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, v[i] & 0x7FFFFFFFu);
        return m >> 16;
    }
}

// the eight times 2^(127 - code), as floats.  (In pairs of bf16 where they are: what falls below bf16's smallest number is far below 1/4.)
template <int W>
__device__ __forceinline__ void mx_scaled8(float (&f)[8], const uint32_t (&v)[W], uint32_t code)
{
    const uint32_t e = 254u - min(code, 253u);                 // (the NaN block's elements mean nothing)
    if constexpr (W == 4) {
        const uint32_t inv = e * 0x00800080u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = mul_bf16x2(v[i], inv);
            f[2 * i] = __uint_as_float(u << 16);
            f[2 * i + 1] = __uint_as_float(u & 0xFFFF0000u);
        }
    } else {
        const float inv = __uint_as_float(e << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[i]) * inv;
    }
}

// The scale code of a block from the upper half of its largest magnitude: its exponent less two, 255 for infinities and NaN.
__device__ __forceinline__ uint32_t mx_code(uint32_t top)
{
    const uint32_t e = top >> 7;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}

// ---- host: tensor maps ------------------------------------------------------------------------
// values of a blob: bytes, boxes of 128 bytes (256 columns) x rows, 128-byte swizzled, past the end zeros
inline bool mx_encode_values(CUtensorMap *map, const void *blob, const MxLayout &L, int rows, uint32_t box_rows)
{
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {L.pitch, (cuuint64_t)rows}, strides[1] = {L.pitch};
    const cuuint32_t box[2] = {128, box_rows}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(static_cast<const uint8_t *>(blob)) + L.off_values, dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// a bf16 matrix with rows of `pitch` elements (a multiple of 8; inputs, outputs, residuals): boxes of 64 columns x rows, 128-byte swizzled, past the end zeros
inline bool mx_encode_bf16(CUtensorMap *map, const void *base, uint64_t cols, uint64_t pitch, uint64_t rows, uint32_t box_rows)
{
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch * 2};
    const cuuint32_t box[2] = {64, box_rows}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace tc
}  // namespace npas
