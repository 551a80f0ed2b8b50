// GEMM of 4-bit inputs with 4-bit weights on CTA pairs (tcgen05 cta_group::2): 256 outputs x 256 input rows per MMA.
//
// The kernel of linear_mx_ps.cu for inputs that are blobs, with every MMA shared by the two CTAs of a cluster: each CTA has the weights
// of its own 128 outputs and one half of the input's rows.  A stage of 256 columns is 32 KB per SM instead of 48 with 256 rows: by
// themselves the loads of 8192^3 take 230 us on single CTAs (what the SMs take in from L2), the MMAs 120.  Scales go to tensor memory through
// the registers of four warps per CTA, a lane quarter each, in groups of five stages: tcgen05.cp on a pair takes 130 cycles for 512
// bytes and holds up the MMAs behind it (8192^3 261 us with six a stage, 177 with none), and a hand-over between the CTAs per stage
// takes longer than the stage (620).  Copies of both CTAs complete on the leader's barriers, the leader's warp 1 issues the
// MMAs for both and frees stages and hands over accumulators with multicast commits; both CTAs' epilogues
// (mx_epi.cuh) read their own 128 lanes; the peer's hand the accumulator back through one arrival with release semantics at cluster
// scope by its warp 1, as in linear_d2.cu.  Every wait is bounded.  A role that waits for the other CTA raises the abort flag of both when it gives
// up; the others (epilogue, slabs, copies of scales, the relay) raise their own CTA's, and the other one runs into its own limit.
#include "mx_epi.cuh"
#include "tc_pair.cuh"

namespace npas {

using namespace tc;

namespace {

constexpr int kRows = 128;
constexpr int kStepCols = 256;                             // columns of a stage
constexpr int kMaxStages = 8;
// warps: 0 copies, 1 MMAs, 2 the slabs' copies, 3 copies of scales, 4 to 7 scales into tensor memory, then the epilogue
constexpr int kStoreWarp = 2, kScaleCopyWarp = 3, kFirstScale = 4, kFirstEpi = 8, kEpiWarps = 8, kThreads = (kFirstEpi + kEpiWarps) * 32;
constexpr uint32_t kSmemLimit = 232448;
constexpr uint32_t kWBytes = kRows * 128;
constexpr int kGroup = 5;                                  // stages whose scales are handed over together
constexpr uint32_t kGroupScales = kGroup * 2 * kMxScaleTile; // bytes of them for 128 rows
constexpr int kN = 256;                                    // rows of X in a tile
constexpr uint32_t kXBytes = kN / 2 * 128, kStageBytes = kXBytes + kWBytes;
constexpr uint32_t kGroupBytes = (1 + kN / kRows) * kGroupScales;
// columns of tensor memory: sums, then scales of every stage of two groups (two tiles of W's, then X's, a K tile's row tiles side by side)
constexpr uint32_t kTmemScales = kN, kScaleCols = 8 + 2 * kN / 32, kTmemCols = 512;
static_assert(kTmemScales + 2 * kGroup * kScaleCols <= kTmemCols, "tensor memory");

struct MxD2Params {
    MxTiles t;
    int I, nS, nKT, S;
    uint32_t off_scales, off_bar, smem_bytes;
    uint64_t w_scales, x_scales;                           // offsets of the scales in the blobs
    int w_tiles, x_tiles;                                  // tiles of scales down the blobs
    int y_bf16;
};

struct MxD2Bars {
    uint64_t full[kMaxStages], empty[kMaxStages];          // full: the leader's only
    uint64_t group_full[2], group_empty[2];                // a group's scales are in this CTA's shared memory / have been read
    uint64_t scales_full[2], scales_empty[2];              // they are in this CTA's tensor memory (leader: both CTAs') / the MMAs have read them
    uint64_t acc_done;                                     // peer: its epilogue warps have the accumulator
    MxEpiBars epi;
    uint32_t tmem_base;
    uint32_t abort_flag;
};

template <bool kBf16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_mx_d2_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_y,
                    const __grid_constant__ CUtensorMap tmap_r, const MxD2Params p, const uint8_t *xblob, const uint8_t *wblob, const float *bias, const void *res, void *y, uint32_t *ws)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    MxD2Bars *bars = reinterpret_cast<MxD2Bars *>(smem + p.off_bar);
    volatile uint32_t *abort_flag = &bars->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();                  // 0: leader (issues the MMAs), 1: its peer
    const int pair = blockIdx.x >> 1, nK = (p.I + 63) / 64;
    const uint32_t peer_abort = map_to_cta(smem_u32(&bars->abort_flag), rank ^ 1u);

    if (tid == 0) {
        for (int s = 0; s < p.S; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], 1); }
        for (int g = 0; g < 2; ++g) {
            mbar_init(&bars->group_full[g], 1); mbar_init(&bars->group_empty[g], 4);
            mbar_init(&bars->scales_full[g], rank == 0 ? 5 : 4); mbar_init(&bars->scales_empty[g], 1);   // four warps; the leader's: and the peer's relay
        }
        mbar_init(&bars->acc_done, kEpiWarps);
        mx_epi_init(&bars->epi, p.t, kEpiWarps + 1);        // (the leader's: its own warps and the peer's relay)
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmap_x); prefetch_tensormap(&tmap_w);
        if (p.t.NS) { prefetch_tensormap(&tmap_y); if (res) prefetch_tensormap(&tmap_r); }
    }
    if (warp == 1) tmem_alloc_pair(&bars->tmem_base, kTmemCols);
    pdl_trigger();
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_relaxed();             // barriers of both CTAs exist before anything arrives on them
    tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
    pdl_wait();
    bias = behind_wait(bias); res = behind_wait(res); xblob = behind_wait(xblob); wblob = behind_wait(wblob);

    if (warp == 0) {
        // ---- TMA producer: this CTA's outputs, its half of the rows of X -----------------------------------------------------------
        if (lane == 0) {
            const uint32_t full0 = map_to_cta(smem_u32(&bars->full[0]), 0u);     // the leader's barriers
            uint32_t s = 0, lap = 0;
            bool ok = true;
            for (MxWalk w(p.t, pair, (int)rank); w.in(p.t) && ok; w.next(p.t)) {
                for (int step = 0; step < p.nS; ++step) {
                    if (lap >= 1 && !pair_wait(&bars->empty[s], (lap & 1u) ^ 1u, abort_flag, peer_abort, ws, 0xC100)) { ok = false; break; }
                    uint8_t *st = smem + (size_t)s * kStageBytes;
                    const uint32_t bar = full0 + s * 8u;
                    if (rank == 0) mbar_arrive_expect_tx(&bars->full[s], 2u * kStageBytes);
                    tma_load_2d_pair(st, &tmap_x, bar, step * 128, w.m0(p.t) + (int)rank * (kN / 2));
                    tma_load_2d_pair(st + kXBytes, &tmap_w, bar, step * 128, w.o0(p.t));
                    if (++s == (uint32_t)p.S) { s = 0; ++lap; }
                }
            }
            // do not leave while the leader's commits may still arrive on this CTA's barriers
            for (int e = 0; e < p.S && ok; ++e) {
                if (lap >= 1 && !pair_wait(&bars->empty[s], (lap & 1u) ^ 1u, abort_flag, peer_abort, ws, 0xC110)) break;
                if (++s == (uint32_t)p.S) { s = 0; ++lap; }
            }
        }
    } else if (warp == 1) {
        if (!elect_one()) {
            // one thread per CTA acts in this role
        } else if (rank == 1) {
            // ---- peer: relay "this CTA's epilogue has the accumulator" to the leader (only where the leader waits for it: an arrival
            // nobody waits for could outlive the leader) ------------------------------------------------------------------------
            const uint32_t acc_empty0 = map_to_cta(smem_u32(&bars->epi.acc_empty[0]), 0u);
            uint32_t it = 0;
            for (int tile = pair; tile + p.t.grid < p.t.n_tiles; tile += p.t.grid, ++it) {
                if (!mbar_wait(&bars->acc_done, it & 1u, abort_flag, ws, 0xC700)) break;
                tc_fence_after_sync();
                tc_fence_before_sync();
                mbar_arrive_remote_release(acc_empty0);
            }
        } else {
            // ---- leader: MMAs for the pair -----------------------------------------------------------------
            const uint32_t base = smem_u32(smem) & 0x3FFFFu, idesc0 = idesc_mxf4(256, kN, 0), idesc1 = idesc_mxf4(256, kN, 1);
            uint32_t s = 0, ph = 0, it = 0, g = 0;             // g: groups of scales so far
            bool ok = true;
            for (int tile = pair; tile < p.t.n_tiles && ok; tile += p.t.grid, ++it) {
                if (it >= 1 && !pair_wait<true>(&bars->epi.acc_empty[0], (it & 1u) ^ 1u, abort_flag, peer_abort, ws, 0xC200)) break;
                tc_fence_after_sync();
                for (int step = 0; step < p.nS; ++step) {
                    const int in_group = step % kGroup;
                    if ((in_group == 0 && !pair_wait<true>(&bars->scales_full[g & 1], (g >> 1) & 1u, abort_flag, peer_abort, ws, 0xC320)) ||
                        !pair_wait(&bars->full[s], ph, abort_flag, peer_abort, ws, 0xC300)) { ok = false; break; }
                    tc_fence_after_sync();
                    const uint32_t st = base + s * kStageBytes, a_lo = ((st + kXBytes) >> 4) | kMxDescLboOne, b_lo = (st >> 4) | kMxDescLboOne;
                    const uint32_t sf = tmem_base + kTmemScales + ((g & 1) * kGroup + in_group) * kScaleCols;
                    const int n = min(4, nK - 4 * step);
                    uint32_t more = step > 0;
                    auto mma = [&](uint32_t j) {                                     // 64 columns = 32 bytes inside the swizzled row
                        mma_mxf4_ss_pair(tmem_base, mx_desc64(a_lo + 2 * j), mx_desc64(b_lo + 2 * j), j & 1 ? idesc1 : idesc0, sf + 4 * (j / 2), sf + 8 + 8 * (j / 2), more);
                        more = 1;
                    };
                    if (n == 4) { mma(0); mma(1); mma(2); mma(3); }                  // (no branch between the MMAs of a whole stage)
                    else {
                        mma(0);
                        if (n > 1) mma(1);
                        if (n > 2) mma(2);
                    }
                    mma_commit_pair(&bars->empty[s]);
                    if (in_group == kGroup - 1 || step + 1 == p.nS) { mma_commit_pair(&bars->scales_empty[g & 1]); ++g; }
                    if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
                }
                if (ok) mma_commit_pair(&bars->epi.acc_full[0]);
            }
        }
    } else if (warp == kStoreWarp) {
        if (lane == 0 && p.t.NS) mx_slab_copies(p.t, pair, (int)rank, smem, &bars->epi, &tmap_y, &tmap_r, res != nullptr, abort_flag, ws);
    } else if (warp == kScaleCopyWarp) {
        // ---- scales of a group of stages into shared memory: W's tiles, then X's row tile by row tile, those that exist; two groups ahead
        // of the one whose arrival in the peer's tensor memory the peer's thread tells the leader (a release at cluster scope takes
        // several hundred cycles, which the warps that write the scales do not have) -----------------------------------------------
        if (lane == 0) {
            constexpr int x_tiles = kN / kRows;
            MxWalk w(p.t, pair, (int)rank);
            int k = 0;
            uint32_t asked = 0;
            auto ask = [&]() {
                if (!w.in(p.t)) return;
                uint64_t *bar = &bars->group_full[asked & 1];
                uint8_t *to = smem + p.off_scales + (asked & 1) * kGroupBytes;
                const uint32_t bytes = (uint32_t)min(2 * kGroup, p.nKT - k) * kMxScaleTile;
                const int wt = w.ot * 2 + (int)rank, xt = w.mt * x_tiles, nx = min(x_tiles, p.x_tiles - xt);
                mbar_arrive_expect_tx(bar, bytes * (uint32_t)((wt < p.w_tiles ? 1 : 0) + nx));
                if (wt < p.w_tiles) bulk_load_1d(to, wblob + p.w_scales + ((uint64_t)wt * p.nKT + k) * kMxScaleTile, bytes, bar);
                for (int t = 0; t < nx; ++t)
                    bulk_load_1d(to + (1 + t) * kGroupScales, xblob + p.x_scales + ((uint64_t)(xt + t) * p.nKT + k) * kMxScaleTile, bytes, bar);
                ++asked;
                if ((k += 2 * kGroup) >= p.nKT) { k = 0; w.next(p.t); }
            };
            ask(); ask();
            const uint32_t scales_full0 = map_to_cta(smem_u32(&bars->scales_full[0]), 0u);
            for (uint32_t g = 0; g < asked; ++g) {
                if (rank == 1) {
                    if (!mbar_wait(&bars->scales_full[g & 1], (g >> 1) & 1u, abort_flag, ws, 0xC710)) break;
                    tc_fence_after_sync();
                    tc_fence_before_sync();
                    mbar_arrive_remote_release(scales_full0 + (g & 1) * 8u);
                }
                if (w.in(p.t) && !mbar_wait(&bars->group_empty[g & 1], (g >> 1) & 1u, abort_flag, ws, 0xC120)) break;
                ask();
            }
        }
    } else if (warp >= kFirstScale && warp < kFirstEpi) {
        // ---- scales from shared memory into this warp's lane quarter of tensor memory.  A tile of scales is 32 x 16 bytes, lane l's are words
        // (rows l, l + 32, l + 64, l + 96), a column each ----------------------------------------------------------------------------
        const int quarter = warp & 3;
        const uint32_t tmem = tmem_base + ((uint32_t)(quarter * 32) << 16) + kTmemScales;
        uint32_t g = 0;
        bool ok = true;
        for (int tile = pair; tile < p.t.n_tiles && ok; tile += p.t.grid)
            for (int step0 = 0; step0 < p.nS; step0 += kGroup, ++g) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->group_full[g & 1], (g >> 1) & 1u, abort_flag, ws, 0xC400) &&
                                                 (g < 2 || pair_wait(&bars->scales_empty[g & 1], ((g >> 1) & 1u) ^ 1u, abort_flag, peer_abort, ws, 0xC410)));
                if (!ok) break;
                tc_fence_after_sync();
                const uint4 *from = reinterpret_cast<const uint4 *>(smem + p.off_scales + (g & 1) * kGroupBytes) + lane;
                const int n = min(kGroup, p.nS - step0);
                for (int i = 0; i < n; ++i) {
                    const uint32_t sf = tmem + ((g & 1) * kGroup + i) * kScaleCols;
                    auto at = [&](int t, int k) { return from[(t * (int)kGroupScales + (2 * i + k) * (int)kMxScaleTile) / 16]; };
                    // two tiles of W's scales, then X's, a K tile's row tiles side by side
                    tmem_st_x8(sf, at(0, 0), at(0, 1));
                    tmem_st_x8(sf + 8, at(1, 0), at(2, 0));
                    tmem_st_x8(sf + 16, at(1, 1), at(2, 1));
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bars->group_empty[g & 1]);
                    mbar_arrive(&bars->scales_full[g & 1]);
                }
                __syncwarp();
            }
        // do not leave while the leader's commits may still arrive on this CTA's barriers
        for (uint32_t e = 1; e <= 2 && e <= g && ok; ++e)
            ok = __all_sync(0xFFFFFFFFu, pair_wait(&bars->scales_empty[(g - e) & 1], ((g - e) >> 1) & 1u, abort_flag, peer_abort, ws, 0xC420));
    } else if (warp >= kFirstEpi) {
        auto release = [&](uint32_t acc) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(rank == 0 ? &bars->epi.acc_empty[acc] : &bars->acc_done);
        };
        if (kBf16 && p.t.NS)
            mx_epilogue_slabs<1, true>(p.t, pair, (int)rank, warp - kFirstEpi, lane, warp & 3, smem_u32(smem), tmem_base, &bars->epi, bias, res != nullptr, abort_flag, ws, release);
        else
            mx_epilogue_rows<1, kBf16>(p.t, pair, (int)rank, warp - kFirstEpi, lane, warp & 3, tmem_base, &bars->epi, bias, res, y, abort_flag, ws, release);
    }
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        // a role gave up: leave time for copies still in flight to land before the CTA retires
        const long long t0 = clock64();
        while (clock64() - t0 < 400000ll) { }
    }
    cluster_sync_relaxed();             // neither CTA retires (or frees tensor memory) while the other may still use it
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

bool plan(const npas_mx_linear_desc &d, MxD2Params &p, int sms)
{
    if (d.x_dtype != NPAS_MX4 || d.variant) return false;
    const MxLayout LW = mx_layout(d.O, d.I), LX = mx_layout(d.M, d.I);
    p = MxD2Params{};
    p.I = d.I;
    p.y_bf16 = d.y_dtype == NPAS_BF16;
    p.nS = (d.I + kStepCols - 1) / kStepCols;
    p.nKT = (int)LW.nKT;
    mx_tiles_plan(p.t, d, kN, 2 * kRows, 1, sms / 2);
    if (!p.t.n_tiles) return false;
    p.w_scales = LW.off_scales; p.x_scales = LX.off_scales; p.w_tiles = (int)LW.nRT; p.x_tiles = (int)LX.nRT;
    p.t.NS = !p.y_bf16 || d.O % 8 ? 0 : d.has_residual ? 4 : 2;
    p.t.ns_log = p.t.NS == 4 ? 2 : 1;
    const uint32_t fixed = (uint32_t)p.t.NS * kMxSlabBytes + 2 * kGroupBytes + (uint32_t)sizeof(MxD2Bars) + 1024u;
    p.S = (int)((kSmemLimit - fixed) / kStageBytes);
    if (p.S > kMaxStages) p.S = kMaxStages;
    p.t.off_slabs = (uint32_t)p.S * kStageBytes;
    p.off_scales = p.t.off_slabs + (uint32_t)p.t.NS * kMxSlabBytes;
    p.off_bar = p.off_scales + 2 * kGroupBytes;
    p.smem_bytes = p.off_bar + (uint32_t)sizeof(MxD2Bars) + 1024u;
    return p.S >= 2;
}

bool planned(const npas_mx_linear_desc &d, MxD2Params &p)
{
    const int32_t none = 0;
    return cached_plan(d, none, 0, p, [&](MxD2Params &q) { return plan(d, q, sm_count()); });
}

}  // namespace

bool linear_mx_d2_supported(const npas_mx_linear_desc &d)
{
    MxD2Params p;
    return planned(d, p);
}

npas_status linear_mx_d2_launch(const npas_mx_linear_desc &d, const void *x, const void *w, const float *bias, const void *res, void *y, uint32_t *ws,
                                cudaStream_t st)
{
    MxD2Params p;
    if (!planned(d, p)) return NPAS_ERR_UNSUPPORTED;
    const MxLayout LW = mx_layout(d.O, d.I), LX = mx_layout(d.M, d.I);
    CUtensorMap tmx, tmw;
    if (!mx_encode_values(&tmx, x, LX, d.M, kN / 2) || !mx_encode_values(&tmw, w, LW, d.O, kRows))
        return NPAS_ERR_CUDA;
    CUtensorMap tmy = tmx, tmr = tmx;
    if (p.t.NS && (!mx_encode_bf16(&tmy, y, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows) ||
                   (res && !mx_encode_bf16(&tmr, res, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows))))
        return NPAS_ERR_CUDA;
    const auto kernel = p.y_bf16 ? linear_mx_d2_kernel<true> : linear_mx_d2_kernel<false>;
    if (allow_dynamic_smem(reinterpret_cast<const void *>(kernel), (int)kSmemLimit) != NPAS_OK) return NPAS_ERR_CUDA;
    const cudaError_t e = launch_pdl(Launch(), kernel, dim3((unsigned)p.t.grid * 2), dim3(kThreads), p.smem_bytes, st, tmx, tmw, tmy, tmr, p, static_cast<const uint8_t *>(x),
                                     static_cast<const uint8_t *>(w), bias, res, y, ws);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
