// GEMM with microscaled 4-bit weights, persistent tiles: 128 outputs x N input rows (N = 128 or 256) per MMA, weights as the
// 128-row operand like in linear_mx_sw.cu.
//
// A CTA per SM walks tiles (outputs fastest, so that the rows of X of a tile are read from L2 by its neighbours).  Copies, MMAs, with a
// 16-bit input the widening of the weights into tensor memory, and the epilogue are roles of their own that hand stages, slots and
// accumulators on through barriers, so the next tile is loaded and multiplied while one is written out.  Two accumulators of 128 columns,
// or one of 256 (with 256 rows of X a weight is fetched half as often, which long inputs need).
// Where the tiles of a CTA all have the same outputs (the grid is a multiple of the tiles across) and their weights fit, the weights stay: a
// 4-bit input's in shared memory (their copies were half of a small tile's), a 16-bit input's widened in tensor memory.
// Outputs leave by mx_epi.cuh.  Every wait is bounded.
#include <type_traits>

#include "mx_epi.cuh"

namespace npas {

using namespace tc;

namespace {

constexpr int kRows = 128;
constexpr int kStepCols = 256;                             // columns of a weight stage
constexpr int kMaxStages = 6, kMaxXStages = 8, kSlots = 4;
constexpr uint32_t kSlotCols = 64;                         // tensor memory of a slot: 128 widened columns of the weights
constexpr uint32_t kSmemLimit = 232448;
constexpr uint32_t kWBytes = kRows * 128;
constexpr uint32_t kScaleBytes = 2 * kMxScaleTile;         // of 128 rows and a stage
constexpr uint32_t kWStage = kWBytes + kScaleBytes;

// warps: 0 copies, 1 MMAs, then a 16-bit input's own copies and the widening warps, then the epilogue, one of them for the slabs' copies
template <bool kMx> struct Roles {
    static constexpr int kXWarp = 2, kWideWarps = kMx ? 0 : 8, kFirstWide = 3;
    static constexpr int kFirstEpi = kMx ? 2 : kFirstWide + kWideWarps + 1;
    static constexpr int kEpiWarps = kMx ? 16 : 8;
    static constexpr int kStoreWarp = kMx ? kFirstEpi + kEpiWarps : kFirstWide + kWideWarps;
    static constexpr int kThreads = (kFirstEpi + kEpiWarps + (kMx ? 1 : 0)) * 32;
};

struct MxPsParams {
    MxTiles t;
    int I, nS, nKT, S, SX, x_steps, slots, resident;           // SX: stages of a 16-bit input, of x_steps K steps; slots: of widened weights; resident: weights stay
    uint32_t x_bytes, xs_bytes, stage_bytes, x_in_stage, off_stages, off_x, off_bar, smem_bytes, tmem_cols, tmem_scales, scale_cols;
    uint64_t w_scales, x_scales;                           // offsets of the scales in the blobs
    int y_bf16;
};

struct MxPsBars {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t x_full[kMaxXStages], x_empty[kMaxXStages];
    uint64_t slot_full[kSlots], slot_empty[kSlots];
    uint64_t w_full;                                       // resident weights of a 4-bit input
    MxEpiBars epi;
    uint32_t tmem_base;
    uint32_t abort_flag;
};

template <bool kMx, bool kBf16>
__global__ void __launch_bounds__(Roles<kMx>::kThreads, 1)
linear_mx_ps_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_y,
                    const __grid_constant__ CUtensorMap tmap_r, const MxPsParams p, const uint8_t *xblob,
                    const uint8_t *wblob, const float *bias, const void *res, void *y, uint32_t *ws)
{
    using R = Roles<kMx>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    MxPsBars *bars = reinterpret_cast<MxPsBars *>(smem + p.off_bar);
    volatile uint32_t *abort_flag = &bars->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int nK = (p.I + 63) / 64;                        // K steps of 64 columns
    // Outputs leave from registers and the widening is over after the first tile: its warps are the epilogue's second group (50000x64 -> 333 18.8 ->
    // 16.4 us, 200704x256 -> 250 with residual 87 -> 78; outputs that leave by TMA gain nothing by it, 200704x64 -> 256 33.1 -> 35.0)
    const bool helped = !kMx && p.resident && !p.t.NS;

    if (tid == 0) {
        for (int s = 0; s < p.S; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], kMx ? 1 : R::kWideWarps); }
        for (int s = 0; s < p.SX; ++s) { mbar_init(&bars->x_full[s], 1); mbar_init(&bars->x_empty[s], 1); }
        for (int s = 0; s < p.slots; ++s) { mbar_init(&bars->slot_full[s], 4); mbar_init(&bars->slot_empty[s], 1); }
        mbar_init(&bars->w_full, 1);
        mx_epi_init(&bars->epi, p.t, p.t.acc == 2 || !(kMx || helped) ? 8 : 16);
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmap_x);
        prefetch_tensormap(&tmap_w);
        if (p.t.NS) { prefetch_tensormap(&tmap_y); if (res) prefetch_tensormap(&tmap_r); }
    }
    if (warp == 1) tmem_alloc(&bars->tmem_base, p.tmem_cols);
    pdl_trigger();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
    pdl_wait();
    bias = behind_wait(bias); res = behind_wait(res);

    auto release = [&](uint32_t acc) {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->epi.acc_empty[acc]);
    };
    // warp e of the epilogue's, where outputs leave from registers
    auto rows = [&](auto groups, int e) {
        mx_epilogue_rows<decltype(groups)::value, kBf16>(p.t, blockIdx.x, 0, e, lane, warp & 3, tmem_base, &bars->epi, bias, res, y, abort_flag, ws, release);
    };
    const std::integral_constant<int, 2> two;

    if (warp == 0) {
        if (lane == 0) {
            auto scale_bytes = [&](int step) { return (uint32_t)min(2, p.nKT - 2 * step) * kMxScaleTile; };      // (the last tile of columns may stand alone)
            auto weights = [&](uint8_t *st, uint64_t *bar, int ot, int step) {
                tma_load_2d(st, &tmap_w, bar, step * 128, ot * kRows);
                bulk_load_1d(st + kWBytes, wblob + p.w_scales + ((uint64_t)ot * p.nKT + 2 * step) * kMxScaleTile, scale_bytes(step), bar);
            };
            MxWalk w(p.t, blockIdx.x, 0);
            if (kMx && p.resident) {
                uint32_t bytes = 0;
                for (int step = 0; step < p.nS; ++step) bytes += kWBytes + scale_bytes(step);
                mbar_arrive_expect_tx(&bars->w_full, bytes);
                for (int step = 0; step < p.nS; ++step) weights(smem + (size_t)step * kWStage, &bars->w_full, w.ot, step);
            }
            uint32_t s = 0, lap = 0;
            bool ok = true;
            // (resident weights of a 16-bit input: the first tile's are all there is to load)
            for (; w.in(p.t) && ok && (kMx || !p.resident || w.tile == (int)blockIdx.x); w.next(p.t)) {
                for (int step = 0; step < p.nS; ++step) {
                    if (lap >= 1 && !mbar_wait(&bars->empty[s], (lap & 1u) ^ 1u, abort_flag, ws, 0xB100)) { ok = false; break; }
                    uint8_t *st = smem + p.off_stages + (size_t)s * p.stage_bytes;
                    const uint32_t sb = scale_bytes(step);
                    // row tiles of X's scales: those that exist
                    const int xt = kMx ? min(p.t.N / kRows, (p.t.M + kRows - 1) / kRows - w.mt * (p.t.N / kRows)) : 0;
                    mbar_arrive_expect_tx(&bars->full[s], (kMx && p.resident ? 0u : kWBytes + sb) + (kMx ? p.x_bytes + xt * sb : 0u));
                    if (!(kMx && p.resident)) weights(st, &bars->full[s], w.ot, step);
                    if (kMx) {
                        tma_load_2d(st + p.x_in_stage + p.xs_bytes, &tmap_x, &bars->full[s], step * 128, w.m0(p.t));
                        for (int t = 0; t < xt; ++t)
                            bulk_load_1d(st + p.x_in_stage + t * kScaleBytes,
                                         xblob + p.x_scales + ((uint64_t)(w.mt * (p.t.N / kRows) + t) * p.nKT + 2 * step) * kMxScaleTile, sb, &bars->full[s]);
                    }
                    if (++s == (uint32_t)p.S) { s = 0; ++lap; }
                }
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t base = smem_u32(smem) & 0x3FFFFu;
            uint32_t s = 0, ph = 0, it = 0, slot = 0, slot_ph = 0;
            bool ok = true;
            // tensor memory of scales: two tiles of W's a stage (a step where they stay), then X's, a K tile's row tiles side by side
            const uint32_t idesc0 = idesc_mxf4(128, (uint32_t)p.t.N, 0), idesc1 = idesc_mxf4(128, (uint32_t)p.t.N, 1);
            const uint32_t xc = (uint32_t)p.t.N / 32, w_cols = kMx && p.resident ? 8u * p.nS : 0u;
            if (kMx && p.resident) {
                ok = mbar_wait(&bars->w_full, 0, abort_flag, ws, 0xB330);
                for (int step = 0; step < p.nS && ok; ++step)
                    for (int t = 0; t < 2 && 2 * step + t < p.nKT; ++t)
                        copy_scales(tmem_base + p.tmem_scales + 8 * step + 4 * t, base + step * kWStage + kWBytes + t * kMxScaleTile);
            }
            for (int tile = blockIdx.x; tile < p.t.n_tiles && ok; tile += p.t.grid, ++it) {
                const uint32_t acc = p.t.acc == 2 ? it & 1u : 0u, lap_acc = p.t.acc == 2 ? it >> 1 : it;
                if (lap_acc >= 1 && !mbar_wait(&bars->epi.acc_empty[acc], (lap_acc & 1u) ^ 1u, abort_flag, ws, 0xB200)) break;
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + acc * p.t.N;
                if (kMx) {
                    for (int step = 0; step < p.nS; ++step) {
                        if (!mbar_wait(&bars->full[s], ph, abort_flag, ws, 0xB300)) { ok = false; break; }
                        tc_fence_after_sync();
                        const uint32_t st = base + p.off_stages + s * p.stage_bytes, wst = p.resident ? base + step * kWStage : st, xs = st + p.x_in_stage;
                        const uint32_t a_lo = (wst >> 4) | kMxDescLboOne, b_lo = ((xs + p.xs_bytes) >> 4) | kMxDescLboOne;
                        const uint32_t sx = tmem_base + p.tmem_scales + w_cols + s * p.scale_cols + (p.resident ? 0u : 8u);
                        const uint32_t sw = p.resident ? tmem_base + p.tmem_scales + 8 * step : sx - 8u;
                        const int n = min(4, nK - 4 * step);
                        const uint32_t ws_at = wst + kWBytes, wide = (uint32_t)p.t.N / kRows - 1u;
                        uint32_t more = step > 0;
                        // 128 columns: their scales, two MMAs of 64 columns (32 bytes inside the swizzled row); no branch between the MMAs of a
                        // whole stage
                        auto scales = [&](uint32_t t) {
                            if (!p.resident) copy_scales(sw + 4 * t, ws_at + t * kMxScaleTile);
                            copy_scales(sx + xc * t, xs + t * kMxScaleTile);
                            if (wide) copy_scales(sx + xc * t + 4, xs + kScaleBytes + t * kMxScaleTile);
                        };
                        auto mma = [&](uint32_t j) {
                            mma_mxf4_ss(d_tmem, mx_desc64(a_lo + 2 * j), mx_desc64(b_lo + 2 * j), j & 1 ? idesc1 : idesc0, sw + 4 * (j / 2), sx + xc * (j / 2), more);
                            more = 1;
                        };
                        scales(0);
                        if (n > 2) scales(1);
                        if (n == 4) { mma(0); mma(1); mma(2); mma(3); }
                        else {
                            mma(0);
                            if (n > 1) mma(1);
                            if (n > 2) mma(2);
                        }
                        mma_commit(&bars->empty[s]);
                        if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
                    }
                } else {
                    // The issuing thread's own instructions are on the critical path.  With 128 rows of X, waits and commits for every K step took it
                    // 455 cycles a step while the MMAs take 256: there a slot's two steps are one stage of X, eight MMAs without a branch
                    // between them (8192x4096 -> 4096 264 -> 225 us).  With 256 rows the MMAs take 512, and stages of one step keep more
                    // of X on its way.
                    const uint32_t idesc = idesc_bf16_f32(128, (uint32_t)p.t.N), x16 = p.x_bytes >> 4, xb = ((base + p.off_x) >> 4) | kMxDescLboOne;
                    const bool wait_w = !(p.resident && it > 0);                 // (weights that stay are waited for once)
                    uint32_t more = 0;                                           // whether the sums are added to
                    auto step = [&](uint32_t b_lo, uint32_t a_t) {
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j) { mma_bf16_ts(d_tmem, a_t + 8 * j, mx_desc64(b_lo + 2 * j), idesc, more); more = 1; }
                    };
                    auto next_slot = [&]() {
                        if (!p.resident) mma_commit(&bars->slot_empty[slot]);
                        if (++slot == (uint32_t)p.slots) { slot = 0; slot_ph ^= 1u; }
                    };
                    auto next_x = [&]() {
                        mma_commit(&bars->x_empty[s]);
                        if (++s == (uint32_t)p.SX) { s = 0; ph ^= 1u; }
                    };
                    if (p.x_steps == 2) {
                        for (int k = 0; k < nK; k += 2) {
                            if (!mbar_wait(&bars->x_full[s], ph, abort_flag, ws, 0xB310) ||
                                (wait_w && !mbar_wait(&bars->slot_full[slot], slot_ph, abort_flag, ws, 0xB320))) { ok = false; break; }
                            tc_fence_after_sync();
                            const uint32_t b_lo = xb + s * 2u * x16, a_t = tmem_base + p.tmem_scales + slot * kSlotCols;
                            if (k + 1 < nK) { step(b_lo, a_t); step(b_lo + x16, a_t + 32u); }
                            else step(b_lo, a_t);
                            next_slot();
                            next_x();
                        }
                    } else {
                        for (int k = 0; k < nK; k += 2) {
                            if ((wait_w && !mbar_wait(&bars->slot_full[slot], slot_ph, abort_flag, ws, 0xB321)) ||
                                !mbar_wait(&bars->x_full[s], ph, abort_flag, ws, 0xB311)) { ok = false; break; }
                            tc_fence_after_sync();
                            const uint32_t a_t = tmem_base + p.tmem_scales + slot * kSlotCols;
                            step(xb + s * x16, a_t);
                            next_x();
                            if (k + 1 < nK) {
                                if (!mbar_wait(&bars->x_full[s], ph, abort_flag, ws, 0xB312)) { ok = false; break; }
                                tc_fence_after_sync();
                                step(xb + s * x16, a_t + 32u);
                                next_x();
                            }
                            next_slot();
                        }
                    }
                }
                if (ok) mma_commit(&bars->epi.acc_full[acc]);
            }
        }
    } else if (!kMx && warp == R::kXWarp) {
        if (lane == 0) {
            uint32_t s = 0, lap = 0;
            bool ok = true;
            for (MxWalk w(p.t, blockIdx.x, 0); w.in(p.t) && ok; w.next(p.t)) {
                for (int k = 0; k < nK; k += p.x_steps) {
                    if (lap >= 1 && !mbar_wait(&bars->x_empty[s], (lap & 1u) ^ 1u, abort_flag, ws, 0xB110)) { ok = false; break; }
                    uint8_t *st = smem + p.off_x + (size_t)s * p.x_steps * p.x_bytes;
                    const int n = min(p.x_steps, nK - k);
                    mbar_arrive_expect_tx(&bars->x_full[s], n * p.x_bytes);
                    for (int h = 0; h < n; ++h) tma_load_2d(st + h * p.x_bytes, &tmap_x, &bars->x_full[s], (k + h) * 64, w.mt * p.t.N);
                    if (++s == (uint32_t)p.SX) { s = 0; ++lap; }
                }
            }
        }
    } else if (!kMx && warp < R::kFirstWide + R::kWideWarps) {
        // ---- widening: a group of four warps takes every second slot (128 columns, two K steps), a thread one row of the weights ------------
        const int group = (warp - R::kFirstWide) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        bool ok = true;
        uint32_t s = 0, ph = 0, u0 = 0;                        // u0: slots before this stage
        for (int tile = blockIdx.x; tile < p.t.n_tiles && ok && !(p.resident && tile != (int)blockIdx.x); tile += p.t.grid) {
            for (int step = 0; step < p.nS && ok; ++step) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->full[s], ph, abort_flag, ws, 0xB400));
                if (!ok) break;
                const uint8_t *st = smem + (size_t)s * p.stage_bytes;
                const int n = min(4, nK - 4 * step);
                for (int t = (int)((group ^ u0) & 1u); 2 * t < n; t += 2) {
                    const uint32_t u = u0 + t, slot = u % kSlots;               // (weights that stay have at most kSlots)
                    // scale codes of the tile of 128 columns: four blocks of this row
                    const uint32_t codes = *reinterpret_cast<const uint32_t *>(st + kWBytes + t * kMxScaleTile + lane * 16 + quarter * 4);
                    const uint32_t to = tmem_base + ((uint32_t)(quarter * 32) << 16) + p.tmem_scales + slot * kSlotCols;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (2 * t + h >= n) break;
                        const int q = 2 * t + h;
                        const uint4 a = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q) ^ (r & 7)) * 16);
                        const uint4 b = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q + 1) ^ (r & 7)) * 16);
                        uint32_t v[32];
                        mx_widen(v, a, b, codes >> (16 * h) & 255u, codes >> (16 * h + 8) & 255u);
                        if (h == 0) {
                            if (u >= kSlots) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->slot_empty[slot], ((u / kSlots) & 1u) ^ 1u, abort_flag, ws, 0xB410));
                            if (!ok) break;
                            tc_fence_after_sync();
                        }
                        tmem_st_x32(to + 32 * h, v);
                    }
                    if (!ok) break;
                    tmem_st_wait();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars->slot_full[slot]);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->empty[s]);
                u0 += (n + 1) / 2;
                if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
            }
        }
        if (helped) rows(two, 8 + warp - R::kFirstWide);
    } else if (warp == R::kStoreWarp) {
        if (lane == 0 && p.t.NS) mx_slab_copies(p.t, blockIdx.x, 0, smem, &bars->epi, &tmap_y, &tmap_r, res != nullptr, abort_flag, ws);
    } else if (warp >= R::kFirstEpi) {
        const std::integral_constant<int, R::kEpiWarps / 8> groups;
        const int e = warp - R::kFirstEpi;
        if (kBf16 && p.t.NS)
            mx_epilogue_slabs<decltype(groups)::value, false>(p.t, blockIdx.x, 0, e, lane, warp & 3, smem_u32(smem), tmem_base, &bars->epi, bias, res != nullptr, abort_flag, ws,
                                                              release);
        else if (helped) rows(two, e);
        else rows(groups, e);
    }
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        // a role gave up: leave time for copies still in flight to land before the CTA retires
        const long long t0 = clock64();
        while (clock64() - t0 < 400000ll) { }
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, p.tmem_cols);
    }
}

bool plan(const npas_mx_linear_desc &d, MxPsParams &p, int sms)
{
    const bool mx = d.x_dtype == NPAS_MX4;
    const MxLayout LW = mx_layout(d.O, d.I), LX = mx_layout(d.M, d.I);
    p = MxPsParams{};
    p.I = d.I;
    p.y_bf16 = d.y_dtype == NPAS_BF16;
    p.nS = (d.I + kStepCols - 1) / kStepCols;
    p.nKT = (int)LW.nKT;
    const int N = d.variant & 0xFFFF ? d.variant & 0xFFFF : 128;              // (the automatic choice names a width)
    if ((N != 128 && N != 256) || d.variant >> 17) return false;
    mx_tiles_plan(p.t, d, N, kRows, N == 128 ? 2 : 1, sms);
    if (!p.t.n_tiles) return false;
    // Weights that stay: with more than a round of tiles, and few SMs idle for a grid that is a multiple of the tiles across
    const int same = sms / p.t.n_ot * p.t.n_ot, nK = (d.I + 63) / 64;
    p.resident = !(d.variant >> 16) && p.t.n_tiles > sms && same * 8 >= sms * 7 && (mx ? p.nS <= 4 : nK <= 2 * kSlots);
    if (p.resident) mx_tiles_plan(p.t, d, N, kRows, p.t.acc, same);
    p.w_scales = LW.off_scales; p.x_scales = LX.off_scales;
    p.x_bytes = (uint32_t)N * 128u;
    p.xs_bytes = mx ? (uint32_t)N / kRows * kScaleBytes : 0u;
    p.x_in_stage = mx && p.resident ? 0u : kWStage;
    p.off_stages = mx && p.resident ? (uint32_t)p.nS * kWStage : 0u;
    p.stage_bytes = p.x_in_stage + (mx ? p.xs_bytes + p.x_bytes : 0u);
    const uint32_t budget = kSmemLimit - (uint32_t)sizeof(MxPsBars) - 128u - 1024u;
    // Slabs for bf16 outputs with rows on 16-byte boundaries: two where the loads need the room (256 rows of X in 16 bits, or without residuals), else four, eight where
    // residuals are ahead of little else (200704x64 -> 256 with residual, 16-bit input 43.0 us with four, 39.9); and the input's ring
    p.t.NS = !p.y_bf16 || d.O % 8 ? 0 : N == 256 && (!mx || (p.nS > 2 && !d.has_residual)) ? 2 : (mx ? d.has_residual && p.nS <= 2 : p.resident && nK <= 2) && N == 128 ? 8 : 4;
    while ((1 << p.t.ns_log) < p.t.NS) ++p.t.ns_log;
    p.slots = mx ? 0 : p.resident ? (nK + 1) / 2 : kSlots;
    p.x_steps = N == 256 || (p.resident && nK == 1) ? 1 : 2;
    const uint32_t slabs = (uint32_t)p.t.NS * kMxSlabBytes;
    if (!mx) {
        // (weights that stay need their stages once: the room is the input's)
        p.SX = N == 256 ? 4 : 3;
        if (p.resident) p.SX = min(kMaxXStages, (int)((budget - slabs - (uint32_t)p.nS * p.stage_bytes) / ((uint32_t)p.x_steps * p.x_bytes)));
    }
    const uint32_t fixed = p.off_stages + (uint32_t)(p.SX * p.x_steps) * p.x_bytes + slabs;
    if (fixed >= budget) return false;
    p.S = (int)((budget - fixed) / p.stage_bytes);
    if (p.S > kMaxStages) p.S = kMaxStages;
    if (p.S < (p.resident ? 1 : 2)) return false;
    p.off_x = p.off_stages + (uint32_t)p.S * p.stage_bytes;
    p.t.off_slabs = p.off_x + (uint32_t)(p.SX * p.x_steps) * p.x_bytes;
    p.off_bar = round_up(p.t.off_slabs + (uint32_t)p.t.NS * kMxSlabBytes, 128);
    p.smem_bytes = p.off_bar + (uint32_t)sizeof(MxPsBars) + 1024u;
    if (p.smem_bytes > kSmemLimit) return false;
    p.tmem_scales = 256;
    p.scale_cols = (p.resident ? 0 : 8) + 2 * (uint32_t)N / 32;
    const uint32_t cols = p.tmem_scales + (mx ? (p.resident ? 8u * p.nS : 0u) + p.scale_cols * p.S : kSlotCols * p.slots);
    p.tmem_cols = 32;
    while (p.tmem_cols < cols) p.tmem_cols *= 2;
    return p.tmem_cols <= 512;
}

bool planned(const npas_mx_linear_desc &d, MxPsParams &p)
{
    const int32_t none = 0;
    return cached_plan(d, none, 0, p, [&](MxPsParams &q) { return plan(d, q, sm_count()); });
}

}  // namespace

bool linear_mx_ps_supported(const npas_mx_linear_desc &d)
{
    MxPsParams p;
    return planned(d, p);
}

npas_status linear_mx_ps_launch(const npas_mx_linear_desc &d, const void *x, int64_t x_pitch, const void *w, const float *bias, const void *res, void *y,
                                uint32_t *ws, cudaStream_t st)
{
    MxPsParams p;
    if (!planned(d, p)) return NPAS_ERR_UNSUPPORTED;
    const bool mx = d.x_dtype == NPAS_MX4;
    CUtensorMap tmx, tmw;
    if (!mx_encode_values(&tmw, w, mx_layout(d.O, d.I), d.O, kRows)) return NPAS_ERR_CUDA;
    if (!(mx ? mx_encode_values(&tmx, x, mx_layout(d.M, d.I), d.M, (uint32_t)p.t.N)
             : mx_encode_bf16(&tmx, x, (uint64_t)d.I, (uint64_t)x_pitch, (uint64_t)d.M, (uint32_t)p.t.N)))
        return NPAS_ERR_CUDA;
    CUtensorMap tmy = tmx, tmr = tmx;
    if (p.t.NS && (!mx_encode_bf16(&tmy, y, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows) ||
                 (res && !mx_encode_bf16(&tmr, res, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows))))
        return NPAS_ERR_CUDA;
    const auto kernel = mx ? (p.y_bf16 ? linear_mx_ps_kernel<true, true> : linear_mx_ps_kernel<true, false>)
                           : (p.y_bf16 ? linear_mx_ps_kernel<false, true> : linear_mx_ps_kernel<false, false>);
    if (allow_dynamic_smem(reinterpret_cast<const void *>(kernel), (int)kSmemLimit) != NPAS_OK) return NPAS_ERR_CUDA;
    const cudaError_t e = launch_pdl(Launch(), kernel, dim3((unsigned)p.t.grid), dim3(mx ? Roles<true>::kThreads : Roles<false>::kThreads),
                                     p.smem_bytes, st, tmx, tmw, tmy, tmr, p, static_cast<const uint8_t *>(x), static_cast<const uint8_t *>(w), bias, res, y, ws);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
