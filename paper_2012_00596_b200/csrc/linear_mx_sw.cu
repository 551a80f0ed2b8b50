// GEMM with microscaled 4-bit weights for few rows: the weights are the tensor core's 128-row operand, the input's rows its columns.
//
// Y^T[o, m] = sum_i W[o,i] X[m,i]: an MMA takes 128 outputs x N input rows (N = 16 to 128), so a single row of X costs a sixteenth of what it
// would as the 128-row operand, and the weights, which are all the bytes there are with few rows, stream through shared memory
// once.  A tile is shared by a cluster of KS CTAs that split the input columns in steps of 256 (a row of a 128-byte swizzled
// box); partial sums go through distributed shared memory to the CTA that owns the input rows and are added in rank order, so
// results do not depend on timing.  Tensor memory lane = output, column = input row: the epilogue's stores are 32 consecutive outputs a warp.
//   4-bit input: both operands by TMA as they lie in the blobs, scales copied from shared into tensor memory ahead of the MMAs of a
//     step (a set of columns per ring stage, so that no copy meets an MMA that still reads), MMAs of kind::mxf4 over 64 columns.
//   16-bit input: eight warps widen the weights, a thread a row: 32 bytes -> 64 bf16 values in 32 columns of tensor memory, from where the
//     MMAs of kind::f16 take their first operand.  Four such slots; weights and inputs have rings of their own (256 and 64 columns a
//     stage).  Widening costs 2.4 instructions a weight, at the issue rate about what HBM delivers.
// Every wait is bounded.
#include "mx_tc.cuh"
#include "tc_pair.cuh"

namespace npas {

using namespace tc;

namespace {

constexpr int kEpiWarps = 8;                               // widening, then the epilogue
constexpr int kXWarp = 2 + kEpiWarps;                      // copies of a 16-bit input
constexpr int kThreads = (kXWarp + 1) * 32;                // warp 0: copies, warp 1: MMAs
constexpr int kRows = 128;
constexpr int kStepCols = 256;                             // columns of a weight stage
constexpr int kMaxStages = 6, kMaxXStages = 8, kSlots = 4;
constexpr int kMaxSplit = 8;                               // portable cluster size
constexpr uint32_t kSmemLimit = 232448;
constexpr uint32_t kWBytes = kRows * 128;
constexpr uint32_t kScaleBytes = 2 * kMxScaleTile;         // of 128 rows and a stage

struct MxSwParams {
    int M, I, O, N, KS, nS, spr, nMT, nOT, nKT, S, SX, cpr;   // spr: steps per CTA; SX: stages of the input (16 bits); cpr: input rows a CTA owns
    int relu, y_bf16;
    uint32_t x_bytes, stage_bytes, off_x, off_red, off_bar, smem_bytes, tmem_cols, tmem_scales;
    uint64_t w_scales, x_scales;                           // offsets of the scales in the blobs
};

struct MxSwBars {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t x_full[kMaxXStages], x_empty[kMaxXStages];
    uint64_t slot_full[kSlots], slot_empty[kSlots];
    uint64_t acc_full;
    uint32_t tmem_base;
    uint32_t abort_flag;
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ float load_res(const void *res, int64_t at, int y_bf16)
{
    return y_bf16 ? bf16_bits_to_f32(__ldg(static_cast<const uint16_t *>(res) + at)) : __ldg(static_cast<const float *>(res) + at);
}
__device__ __forceinline__ void store_y(void *y, int64_t at, float v, int relu, int y_bf16)
{
    if (relu) v = fmaxf(v, 0.f);
    if (y_bf16) static_cast<uint16_t *>(y)[at] = (uint16_t)cvt_bf16x2(v, 0.f);
    else static_cast<float *>(y)[at] = v;
}

template <bool kMx>
__global__ void __launch_bounds__(kThreads, 1)
linear_mx_sw_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w, const MxSwParams p, const uint8_t *xblob,
                    const uint8_t *wblob, const float *bias, const void *res, void *y, uint32_t *ws)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    MxSwBars *bars = reinterpret_cast<MxSwBars *>(smem + p.off_bar);
    volatile uint32_t *abort_flag = &bars->abort_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = p.KS > 1 ? (int)cluster_ctarank() : 0, tile = blockIdx.x / p.KS;
    const int mt = tile / p.nOT, ot = tile - mt * p.nOT;
    const int s_lo = rank * p.spr, s_n = max(0, min(p.nS - s_lo, p.spr));
    const int live = (p.nS + p.spr - 1) / p.spr;               // CTAs that have steps
    // K steps of 64 columns: of this CTA, the last stage's what is left of the input
    const int k_n = max(0, min((p.I + 63) / 64 - s_lo * 4, s_n * 4));

    if (tid == 0) {
        for (int s = 0; s < p.S; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], kMx ? 1 : kEpiWarps); }
        for (int s = 0; s < p.SX; ++s) { mbar_init(&bars->x_full[s], 1); mbar_init(&bars->x_empty[s], 1); }
        for (int s = 0; s < kSlots; ++s) { mbar_init(&bars->slot_full[s], kEpiWarps / 2); mbar_init(&bars->slot_empty[s], 1); }
        mbar_init(&bars->acc_full, 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmap_x);
        prefetch_tensormap(&tmap_w);
    }
    if (warp == 1) tmem_alloc(&bars->tmem_base, p.tmem_cols);
    pdl_trigger();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
    if (p.KS > 1) cluster_arrive();    // this CTA is running: its shared memory may be written by the others
    pdl_wait();
    const int z = zero_behind_wait();

    // bytes of scales of stage `step`: the last tile of columns may stand alone
    auto scale_bytes = [&](int step) { return (uint32_t)min(2, p.nKT - 2 * step) * kMxScaleTile; };

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, lap = 0;
            for (int i = 0; i < s_n; ++i) {
                if (lap >= 1 && !mbar_wait(&bars->empty[s], (lap & 1u) ^ 1u, abort_flag, ws, 0xA100)) break;
                uint8_t *st = smem + (size_t)s * p.stage_bytes;
                const int step = s_lo + i;
                const uint32_t sb = scale_bytes(step);
                mbar_arrive_expect_tx(&bars->full[s], kWBytes + sb + (kMx ? p.x_bytes + sb : 0u));
                tma_load_2d(st, &tmap_w, &bars->full[s], step * 128, ot * kRows);
                bulk_load_1d(st + kWBytes, wblob + p.w_scales + ((uint64_t)ot * p.nKT + 2 * step) * kMxScaleTile, sb, &bars->full[s]);
                if (kMx) {
                    tma_load_2d(st + kWBytes + 2 * kScaleBytes, &tmap_x, &bars->full[s], step * 128, mt * kRows);
                    bulk_load_1d(st + kWBytes + kScaleBytes, xblob + p.x_scales + ((uint64_t)mt * p.nKT + 2 * step) * kMxScaleTile, sb, &bars->full[s]);
                }
                if (++s == (uint32_t)p.S) { s = 0; ++lap; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) {
            // (18 address bits: in the CTAs of a cluster a shared-memory address carries the CTA's rank above them)
            const uint32_t base = smem_u32(smem) & 0x3FFFFu;
            bool go = true;
            if (kMx) {
                uint32_t s = 0, ph = 0;
                for (int i = 0; i < s_n && go; ++i) {
                    if (!mbar_wait(&bars->full[s], ph, abort_flag, ws, 0xA300)) { go = false; break; }
                    tc_fence_after_sync();
                    const uint32_t st = base + s * p.stage_bytes, a_lo = (st >> 4) | kMxDescLboOne, b_lo = ((st + kWBytes + 2 * kScaleBytes) >> 4) | kMxDescLboOne;
                    const uint32_t sf = tmem_base + p.tmem_scales + s * 16u;         // two tiles of W's scales, two of X's
                    const int n = min(4, k_n - 4 * i);
                    for (int t = 0; t < (n + 1) / 2; ++t) {
                        copy_scales(sf + 4 * t, st + kWBytes + t * kMxScaleTile);
                        copy_scales(sf + 8 + 4 * t, st + kWBytes + kScaleBytes + t * kMxScaleTile);
                    }
                    for (int j = 0; j < n; ++j)                                      // 64 columns = 32 bytes inside the swizzled row
                        mma_mxf4_ss(tmem_base, mx_desc64(a_lo + 2 * j), mx_desc64(b_lo + 2 * j), idesc_mxf4(128, (uint32_t)p.N, j & 1),
                                    sf + 4 * (j / 2), sf + 8 + 4 * (j / 2), i > 0 || j > 0);
                    mma_commit(&bars->empty[s]);
                    if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
                }
            } else {
                uint32_t sx = 0, phx = 0;
                const uint32_t idesc = idesc_bf16_f32(128, (uint32_t)p.N), xb = base + p.off_x;
                for (int k = 0; k < k_n; ++k) {
                    const uint32_t slot = k % kSlots;
                    if (!mbar_wait(&bars->x_full[sx], phx, abort_flag, ws, 0xA310) ||
                        !mbar_wait(&bars->slot_full[slot], (k / kSlots) & 1u, abort_flag, ws, 0xA320)) { go = false; break; }
                    tc_fence_after_sync();
                    const uint32_t b_lo = ((xb + sx * p.x_bytes) >> 4) | kMxDescLboOne, a_t = tmem_base + p.tmem_scales + slot * 32u;
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j)
                        mma_bf16_ts(tmem_base, a_t + 8 * j, mx_desc64(b_lo + 2 * j), idesc, (k > 0 || j > 0) ? 1u : 0u);
                    mma_commit(&bars->slot_empty[slot]);
                    mma_commit(&bars->x_empty[sx]);
                    if (++sx == (uint32_t)p.SX) { sx = 0; phx ^= 1u; }
                }
            }
            if (go) mma_commit(&bars->acc_full);
        }
        __syncwarp();
    } else if (warp == kXWarp) {
        if (!kMx && lane == 0) {
            uint32_t sx = 0, lap = 0;
            for (int k = 0; k < k_n; ++k) {
                if (lap >= 1 && !mbar_wait(&bars->x_empty[sx], (lap & 1u) ^ 1u, abort_flag, ws, 0xA110)) break;
                mbar_arrive_expect_tx(&bars->x_full[sx], p.x_bytes);
                tma_load_2d(smem + p.off_x + (size_t)sx * p.x_bytes, &tmap_x, &bars->x_full[sx], (4 * s_lo + k) * 64, mt * p.N);
                if (++sx == (uint32_t)p.SX) { sx = 0; ++lap; }
            }
        }
        __syncwarp();
    } else if (!kMx) {
        // ---- widening: group g of four warps takes every second K step, a thread one row of the weights -----------------
        const int group = (warp - 2) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        bool ok = true;
        uint32_t s = 0, ph = 0;
        for (int i = 0; i < s_n && ok; ++i) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->full[s], ph, abort_flag, ws, 0xA400));
            if (!ok) break;
            const uint8_t *st = smem + (size_t)s * p.stage_bytes;
            for (int q = group; q < 4 && 4 * i + q < k_n; q += 2) {
                const int k = 4 * i + q;
                const uint32_t slot = k % kSlots;
                const uint4 a = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q) ^ (r & 7)) * 16);
                const uint4 b = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q + 1) ^ (r & 7)) * 16);
                const uint32_t codes = *reinterpret_cast<const uint32_t *>(st + kWBytes + (q >> 1) * kMxScaleTile + lane * 16 + quarter * 4) >> (16 * (q & 1));
                uint32_t v[32];
                mx_widen(v, a, b, codes & 255u, (codes >> 8) & 255u);
                if (k >= kSlots) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->slot_empty[slot], ((k / kSlots) & 1u) ^ 1u, abort_flag, ws, 0xA410));
                if (!ok) break;
                tc_fence_after_sync();
                tmem_st_x32(tmem_base + ((uint32_t)(quarter * 32) << 16) + p.tmem_scales + slot * 32u, v);
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->slot_full[slot]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->empty[s]);
            if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
        }
    }

    const int rows = min(p.N, p.M - mt * p.N);                 // rows of X in this tile (with a 4-bit input several tiles are of 128)
    if (p.KS > 1) cluster_wait();      // every CTA of the cluster is running
    if (warp >= 2 && warp < kXWarp && s_n > 0) {
        const int quarter = warp & 3, part = (warp - 2) >> 2, o = ot * kRows + quarter * 32 + lane;
        if (__all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full, 0, abort_flag, ws, 0xA500))) {
            tc_fence_after_sync();
            const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
            const float b = p.KS == 1 && bias && o < p.O ? __ldg(bias + o + z) : 0.f;
            for (int c0 = part * 16; c0 < rows; c0 += 16 * (kEpiWarps / 4)) {
                uint32_t v[16];
                __syncwarp();
                tmem_ld_x16(t_addr + c0, v);
                if (p.KS == 1) {
                    float add[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        add[i] = res && o < p.O && c0 + i < rows ? load_res(res, (int64_t)(mt * p.N + c0 + i) * p.O + o + z, p.y_bf16) : 0.f;
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (o < p.O && c0 + i < rows) store_y(y, (int64_t)(mt * p.N + c0 + i) * p.O + o, __uint_as_float(v[i]) + b + add[i], p.relu, p.y_bf16);
                } else {
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int m = c0 + i, owner = m / p.cpr;
                        if (m < rows)
                            st_remote_u32(map_to_cta(smem_u32(smem + p.off_red), (uint32_t)owner) +
                                              (uint32_t)((rank * p.cpr + m - owner * p.cpr) * kRows + quarter * 32 + lane) * 4u, v[i]);
                    }
                }
            }
        }
    }
    tc_fence_before_sync();
    if (p.KS > 1) { cluster_arrive(); cluster_wait(); }        // all partial sums are in place; no CTA touches another's memory after this
    else __syncthreads();
    tc_fence_after_sync();
    if (warp == 1) tmem_dealloc(tmem_base, p.tmem_cols);
    if (*abort_flag) {
        // a role gave up: leave time for copies still in flight to land before the CTA retires
        const long long t0 = clock64();
        while (clock64() - t0 < 400000ll) { }
        return;
    }
    if (p.KS == 1) return;
    const int own = max(0, min(p.cpr, rows - rank * p.cpr));
    for (int i = tid; i < own * kRows; i += kThreads) {
        const int m = i / kRows, ol = i - m * kRows, o = ot * kRows + ol;
        if (o >= p.O) continue;
        const int64_t at = (int64_t)(mt * p.N + rank * p.cpr + m) * p.O + o + z;
        const float add = res ? load_res(res, at, p.y_bf16) : 0.f;
        float v = 0.f;
        for (int s = 0; s < live; ++s) v += *reinterpret_cast<const float *>(smem + p.off_red + (uint32_t)((s * p.cpr + m) * kRows + ol) * 4u);
        if (bias) v += __ldg(bias + o + z);
        store_y(y, at, v + add, p.relu, p.y_bf16);
    }
}

bool plan(const npas_mx_linear_desc &d, MxSwParams &p, int sms)
{
    const bool mx = d.x_dtype == NPAS_MX4;
    const MxLayout LW = mx_layout(d.O, d.I), LX = mx_layout(d.M, d.I);
    p = MxSwParams{};
    p.M = d.M; p.I = d.I; p.O = d.O;
    p.relu = d.relu; p.y_bf16 = d.y_dtype == NPAS_BF16;
    p.nS = (d.I + kStepCols - 1) / kStepCols;
    p.nKT = (int)LW.nKT;
    p.nOT = (d.O + kRows - 1) / kRows;
    p.nMT = (d.M + kRows - 1) / kRows;
    // Input rows of a tile: all of them, or equal shares in multiples of 16 (4-bit: a tile starts where a tile of scales does)
    p.N = mx && p.nMT > 1 ? kRows : ((d.M + p.nMT - 1) / p.nMT + 15) / 16 * 16;
    p.w_scales = LW.off_scales; p.x_scales = LX.off_scales;
    // Split of the columns: as many CTAs as one wave holds
    const long long tiles = (long long)p.nMT * p.nOT;
    if (tiles > 0x7FFFFFFF / kMaxSplit) return false;
    p.KS = 1;
    while (p.KS < kMaxSplit && 2 * p.KS <= p.nS && tiles * 2 * p.KS <= sms) p.KS *= 2;
    if (d.variant) {
        p.KS = d.variant;
        if (p.KS < 1 || p.KS > kMaxSplit || p.KS & (p.KS - 1)) return false;
    }
    p.spr = (p.nS + p.KS - 1) / p.KS;
    p.cpr = (p.N + p.KS - 1) / p.KS;
    const uint32_t red = p.KS > 1 ? (uint32_t)p.KS * p.cpr * kRows * 4u : 0u;
    const uint32_t fixed = red + (uint32_t)sizeof(MxSwBars) + 128u + 1024u;
    p.x_bytes = (uint32_t)p.N * 128u;
    p.stage_bytes = round_up(kWBytes + (mx ? 2 * kScaleBytes + p.x_bytes : kScaleBytes), 1024);
    const uint32_t budget = kSmemLimit - fixed;
    if (mx) {
        p.S = (int)(budget / p.stage_bytes);
        p.SX = 0;
    } else {
        // the input's ring (of 64 columns a stage)
        p.SX = kMaxXStages;
        while (p.SX > 3 && (uint32_t)p.SX * p.x_bytes + 3 * p.stage_bytes > budget) --p.SX;
        p.S = (int)((budget - (uint32_t)p.SX * p.x_bytes) / p.stage_bytes);
    }
    if (p.S > kMaxStages) p.S = kMaxStages;
    if (p.S > p.spr) p.S = p.spr;
    if (p.S < 1 || (p.S < 2 && p.spr > 1)) return false;
    p.off_x = (uint32_t)p.S * p.stage_bytes;
    p.off_red = p.off_x + (uint32_t)p.SX * p.x_bytes;
    p.off_bar = round_up(p.off_red + red, 128);
    p.smem_bytes = p.off_bar + (uint32_t)sizeof(MxSwBars) + 1024u;
    if (p.smem_bytes > kSmemLimit) return false;
    // columns of tensor memory: the sums, then scales of every stage (4-bit) or the widened weights
    p.tmem_scales = round_up((uint32_t)p.N, 32);
    const uint32_t cols = p.tmem_scales + (mx ? 16u * p.S : 32u * kSlots);
    p.tmem_cols = 32;
    while (p.tmem_cols < cols) p.tmem_cols *= 2;
    return p.tmem_cols <= 512;
}

bool planned(const npas_mx_linear_desc &d, MxSwParams &p)
{
    const int32_t none = 0;
    return cached_plan(d, none, 0, p, [&](MxSwParams &q) { return plan(d, q, sm_count()); });
}

}  // namespace

bool linear_mx_sw_supported(const npas_mx_linear_desc &d)
{
    MxSwParams p;
    return planned(d, p);
}

npas_status linear_mx_sw_launch(const npas_mx_linear_desc &d, const void *x, int64_t x_pitch, const void *w, const float *bias, const void *res, void *y,
                                uint32_t *ws, cudaStream_t st)
{
    MxSwParams p;
    if (!planned(d, p)) return NPAS_ERR_UNSUPPORTED;
    const bool mx = d.x_dtype == NPAS_MX4;
    CUtensorMap tmx, tmw;
    if (!mx_encode_values(&tmw, w, mx_layout(d.O, d.I), d.O, kRows)) return NPAS_ERR_CUDA;
    if (!(mx ? mx_encode_values(&tmx, x, mx_layout(d.M, d.I), d.M, (uint32_t)p.N)
             : mx_encode_bf16(&tmx, x, (uint64_t)d.I, (uint64_t)x_pitch, (uint64_t)d.M, (uint32_t)p.N)))
        return NPAS_ERR_CUDA;
    const auto kernel = mx ? linear_mx_sw_kernel<true> : linear_mx_sw_kernel<false>;
    if (allow_dynamic_smem(reinterpret_cast<const void *>(kernel), (int)kSmemLimit) != NPAS_OK) return NPAS_ERR_CUDA;
    const dim3 grid((unsigned)(p.nMT * p.nOT * p.KS)), block(kThreads);
    const uint8_t *xb = static_cast<const uint8_t *>(x), *wb = static_cast<const uint8_t *>(w);
    const cudaError_t e = p.KS > 1 ? launch_pdl_cluster(Launch(), kernel, grid, block, p.KS, p.smem_bytes, st, tmx, tmw, p, xb, wb, bias, res, y, ws)
                                   : launch_pdl(Launch(), kernel, grid, block, p.smem_bytes, st, tmx, tmw, p, xb, wb, bias, res, y, ws);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
