// GEMM of a 16-bit input of up to 16 rows with microscaled 4-bit weights: single tokens, where the weights' bytes are the work.
//
// Y[m,o] = act(bias[o] + sum_i X[m,i] W[o,i] + residual[m,o]).  With so few rows nothing is read twice, so the weights go from memory
// to registers, are widened there and multiplied by warp-wide MMAs (m16n8k16, fp32 sums): no stage, barrier or tensor-memory hand-over between
// the load and the product (linear_mx_sw.cu, whose tensor-core MMAs take the weights from tensor memory, is held up by those: 1x8192 -> 8192
// 20.7 us, 11.9 here).  The order of the columns in an MMA is free as long as both operands agree: a thread takes a whole block of 32
// columns of a row (16 bytes) and one scale, and of X the same 32 columns (64 bytes) of one row, each exactly as it lies in memory.
// A block of threads has 32 outputs (8a + g, + 32, + 64, + 96 of a tile of scales, whose 16 bytes hold those four rows), a warp every
// sixteenth tile of 128 columns of them; the warps' sums meet in shared memory and are added in order.  What it takes is no unit's rate: 1x8192 -> 8192 (11.9 us, 5.5 at
// the copy rate) issues in 57 % of the cycles, the logic pipe (nine of the 17 instructions that widen eight weights) is busy 41 %, memory 30 %; the rest are waits for
// loads and the two microseconds that a launch, its first loads and its last sums take.  With 16 rows waits for loads come first (16x4096 -> 8192
// 10.8 us, issue 39 %): every block of 32 outputs reads all of X from L2, 34 MB for 18 MB of weights, and not ahead.  Copies of the weights into a ring in
// shared memory, three shares ahead, cost more instructions than the wait that they save (1x8192 -> 8192 17.2 us).
#include "mx_tc.cuh"
#include "tc_pair.cuh"

namespace npas {

using namespace tc;

namespace {

constexpr int kMaxWarps = 16;
constexpr int kOutputs = 32;                               // of a block of threads

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// A thread's share of a tile of 128 columns: a block of 32 of four rows of W and their scales; and the same columns of NT rows of X.
struct Share {
    uint4 e[4], codes;
};
template <int NT> struct ShareX {
    uint4 x[NT][4];
};

// kSplit: a cluster of KS blocks shares the outputs and splits the columns
template <int NT, bool kSplit>
__global__ void __launch_bounds__(kMaxWarps * 32)
linear_mx_gv_kernel(int KS, int M, int I, int O, int relu, int y_bf16, int nKT, uint32_t pitch, uint64_t off_scales, uint64_t off_values, int64_t x_pitch,
                    const uint16_t *x, const uint8_t *w, const float *bias, const void *res, void *y)
{
    __shared__ float sums[kMaxWarps][kOutputs][NT * 8 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, warps = blockDim.x >> 5;
    const int rank = kSplit ? (int)cluster_ctarank() : 0, block = kSplit ? blockIdx.x / KS : blockIdx.x, stride = kSplit ? warps * KS : warps;
    const int ot = block >> 2, a8 = (block & 3) * 8;
    pdl_trigger();
    pdl_wait();
    x = behind_wait(x); w = behind_wait(w); bias = behind_wait(bias); res = behind_wait(res);
    float c[2][NT][4] = {};
    // Rows past the end are the last one again: what they give is not stored.  Offsets from the tile's first byte, and from X, fit in 32 bits.
    const uint8_t *wt = w + off_values + (uint64_t)ot * kMxTileRows * pitch;
    const uint8_t *st = w + off_scales + (uint64_t)ot * nKT * kMxScaleTile;
    const uint8_t *xb = reinterpret_cast<const uint8_t *>(x);
    uint32_t row[4], x_row[NT];
#pragma unroll
    for (int j = 0; j < 4; ++j) row[j] = (uint32_t)min(32 * j + a8 + g, O - 1 - ot * kMxTileRows) * pitch + q * (kMxBlock / 2);
#pragma unroll
    for (int t = 0; t < NT; ++t) x_row[t] = (uint32_t)min(t * 8 + g, M - 1) * (uint32_t)x_pitch * 2u + q * (kMxBlock * 2);
    const uint32_t code_row = (uint32_t)(a8 + g) * 16u, pick = 0x4440u | (uint32_t)q;
    const int nW = I / kMxTileCols;                            // tiles without an end inside
    auto load = [&](Share &v, int kt) {
        v.codes = __ldg(reinterpret_cast<const uint4 *>(st + (uint32_t)kt * kMxScaleTile + code_row));
        const bool in = kt < nW || I - (kt * kMxTileCols + q * kMxBlock) > 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v.e[j] = make_uint4(0, 0, 0, 0);
            if (in) v.e[j] = __ldg(reinterpret_cast<const uint4 *>(wt + (row[j] + (uint32_t)kt * (kMxTileCols / 2))));
        }
    };
    auto load_x = [&](ShareX<NT> &v, int kt) {
        const int left = I - (kt * kMxTileCols + q * kMxBlock);            // columns there are from this thread's first one on
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint4 *from = reinterpret_cast<const uint4 *>(xb + (x_row[t] + (uint32_t)kt * (kMxTileCols * 2)));
            if (kt < nW) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v.x[t][i] = __ldg(from + i);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v.x[t][i] = 8 * i < left ? __ldg(from + i) : make_uint4(0, 0, 0, 0);
            }
        }
    };
    auto multiply = [&](const Share &v, const ShareX<NT> &vx) {
        uint32_t code[4], f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            code[j] = __byte_perm(j == 0 ? v.codes.x : j == 1 ? v.codes.y : j == 2 ? v.codes.z : v.codes.w, 0, pick);
            f[j] = mx_factor(code[j]).first;
        }
        const bool large = __any_sync(0xFFFFFFFFu, max(max(code[0], code[1]), max(code[2], code[3])) > 128u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t p[4][4];                                  // of the rows: four pairs of columns
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t word = i == 0 ? v.e[j].x : i == 1 ? v.e[j].y : i == 2 ? v.e[j].z : v.e[j].w;
                mx_widen_word(p[j], word, f[j]);
            }
            if (large) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) p[j][k] = mul_bf16x2(p[j][k], mx_factor(code[j]).second);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    mma_16816(c[h][t], p[2 * h][0], p[2 * h + 1][0], p[2 * h][1], p[2 * h + 1][1], vx.x[t][i].x, vx.x[t][i].y);
                    mma_16816(c[h][t], p[2 * h][2], p[2 * h + 1][2], p[2 * h][3], p[2 * h + 1][3], vx.x[t][i].z, vx.x[t][i].w);
                }
        }
    };
    // the next share is on its way while one is multiplied (of X only where the registers are there for it: it comes from L2)
    constexpr bool kAheadX = NT == 1;
    Share a, b;
    ShareX<NT> ax, bx;
    int kt = rank * warps + warp;
    if (kt < nKT) { load(a, kt); if (kAheadX) load_x(ax, kt); }
    while (kt < nKT) {
        const int next = kt + stride, third = next + stride;
        if (!kAheadX) load_x(ax, kt);
        if (next < nKT) { load(b, next); if (kAheadX) load_x(bx, next); }
        multiply(a, ax);
        if (next >= nKT) break;
        if (!kAheadX) load_x(bx, next);
        if (third < nKT) { load(a, third); if (kAheadX) load_x(ax, third); }
        multiply(b, bx);
        kt = third;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][(2 * h + (i >> 1)) * 8 + g][t * 8 + 2 * q + (i & 1)] = c[h][t][i];
    __syncthreads();
    if (kSplit) {
        // the block's sums in the place of its first warp's, from where the first block takes them
        for (int i = threadIdx.x; i < kOutputs * M; i += blockDim.x) {
            const int m = i / kOutputs, r = i & (kOutputs - 1);
            float v = 0.f;
            for (int k = 0; k < warps; ++k) v += sums[k][r][m];
            sums[0][r][m] = v;
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    for (int i = threadIdx.x; i < kOutputs * M && rank == 0; i += blockDim.x) {
        const int m = i / kOutputs, r = i & (kOutputs - 1), o = ot * kMxTileRows + 32 * (r >> 3) + a8 + (r & 7);
        if (o >= O) continue;
        const int64_t at = (int64_t)m * O + o;
        float v = 0.f;
        if (kSplit) {
            for (int k = 0; k < KS; ++k) v += ld_cluster_f32(map_to_cta(smem_u32(&sums[0][r][m]), (uint32_t)k));
        } else {
            for (int k = 0; k < warps; ++k) v += sums[k][r][m];
        }
        if (bias) v += __ldg(bias + o);
        if (res) v += y_bf16 ? bf16_bits_to_f32(__ldg(static_cast<const uint16_t *>(res) + at)) : __ldg(static_cast<const float *>(res) + at);
        if (relu) v = fmaxf(v, 0.f);
        if (y_bf16) static_cast<uint16_t *>(y)[at] = (uint16_t)cvt_bf16x2(v, 0.f);
        else static_cast<float *>(y)[at] = v;
    }
    if (kSplit) { __syncwarp(); cluster_arrive(); cluster_wait(); }          // no block leaves while its sums are read
}

}  // namespace

bool linear_mx_gv_supported(const npas_mx_linear_desc &d)
{
    return d.x_dtype == NPAS_BF16 && !d.quantize_x && d.M <= 16 && !d.variant;
}

npas_status linear_mx_gv_launch(const npas_mx_linear_desc &d, const void *x, int64_t x_pitch, const void *w, const float *bias, const void *res, void *y,
                                cudaStream_t st)
{
    if (!linear_mx_gv_supported(d)) return NPAS_ERR_UNSUPPORTED;
    const MxLayout L = mx_layout(d.O, d.I);
    // sixteen warps where a block has an SM to itself, else eight, of which two blocks fit on one
    const int blocks = (int)L.nRT * 4, sms = sm_count(), most = blocks <= sms ? kMaxWarps : kMaxWarps / 2;
    // Few outputs and more columns than one tile a warp: a cluster splits the columns, as long as there are eight warps with a tile in each block
    // and all clusters run at once (those of four do not get every SM).  1x8192 -> 1024 7.3 -> 5.0 us, 1x8192 -> 2048 7.4 -> 6.0, 5x6000 -> 500
    // 6.1 -> 4.4; with one tile a warp it costs more than it saves (1x2048 -> 1000 3.2 -> 3.6).
    constexpr int kLeast = 8;
    int ks = 1;
    while ((int)L.nKT > kMaxWarps && ks < 4 && blocks * ks * 2 <= (ks == 2 ? sms - sms / 9 : sms) && (int)L.nKT >= 2 * ks * kLeast) ks *= 2;
    const int share = ((int)L.nKT + ks - 1) / ks, warps = share < most ? share : most;
    const dim3 grid((unsigned)(blocks * ks)), block((unsigned)(warps * 32));
    auto launch = [&](auto kernel) {
        return ks > 1 ? launch_pdl_cluster(Launch(), kernel, grid, block, ks, 0, st, ks, (int)d.M, (int)d.I, (int)d.O, (int)d.relu, (int)(d.y_dtype == NPAS_BF16),
                                           (int)L.nKT, L.pitch, L.off_scales, L.off_values, x_pitch, static_cast<const uint16_t *>(x),
                                           static_cast<const uint8_t *>(w), bias, res, y)
                      : launch_pdl(Launch(), kernel, grid, block, 0, st, ks, (int)d.M, (int)d.I, (int)d.O, (int)d.relu, (int)(d.y_dtype == NPAS_BF16), (int)L.nKT,
                                   L.pitch, L.off_scales, L.off_values, x_pitch, static_cast<const uint16_t *>(x), static_cast<const uint8_t *>(w), bias, res, y);
    };
    const cudaError_t e = d.M <= 8 ? ks > 1 ? launch(linear_mx_gv_kernel<1, true>) : launch(linear_mx_gv_kernel<1, false>)
                                   : ks > 1 ? launch(linear_mx_gv_kernel<2, true>) : launch(linear_mx_gv_kernel<2, false>);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
