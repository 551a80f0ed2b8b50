// GEMM of 4-bit inputs with 4-bit weights on CTA pairs (tcgen05 cta_group::2): 256 outputs x N input rows (128 or 256) per MMA.
//
// The kernel of linear_mx_ps.cu for inputs that are blobs, with every MMA shared by the two CTAs of a cluster: each CTA has the weights
// (and their scales) of its own 128 outputs and one half of the input's rows, and the scales of all of them.  A stage of 256 columns is
// 35 KB per SM instead of 51 with 256 rows: by themselves the loads of 8192^3 take 230 us on single CTAs (what the SMs take in from L2),
// the MMAs 120.  Where the weights of a tile fit and a pair's tiles all have the same outputs (the number of pairs is a multiple of the
// tiles across), they are loaded once and stay.  Copies of both CTAs complete on the leader's barriers, the leader's warp 1 issues the
// MMAs and the copies of scales for both and frees stages and hands over accumulators with multicast commits; both CTAs' epilogues
// (mx_epi.cuh) read their own 128 lanes; the peer's hand the accumulator back through one arrival with release semantics at cluster
// scope by its warp 1, as in linear_d2.cu.  Every wait is bounded; a role that gives up raises the abort flag of both CTAs.
#include "mx_epi.cuh"
#include "tc_pair.cuh"

namespace npas {

using namespace tc;

namespace {

constexpr int kRows = 128;
constexpr int kStepCols = 256;                             // columns of a stage
constexpr int kMaxStages = 8;
constexpr int kEpiWarps = 16, kFirstEpi = 2, kStoreWarp = kFirstEpi + kEpiWarps, kThreads = (kStoreWarp + 1) * 32;
constexpr uint32_t kSmemLimit = 232448;
constexpr uint32_t kScaleBytes = 2 * kMxScaleTile;         // of 128 rows and a stage
constexpr uint32_t kWBytes = kRows * 128, kWStage = kWBytes + kScaleBytes;

struct MxD2Params {
    MxTiles t;
    int I, nS, nKT, S, resident;                           // resident: the weights of all stages stay in shared memory
    uint32_t x_bytes, xs_bytes, stage_bytes, off_stages, off_bar, smem_bytes, tmem_scales, scale_cols;
    int y_bf16;
};

struct MxD2Bars {
    uint64_t full[kMaxStages], empty[kMaxStages];          // full: the leader's only
    uint64_t w_full;                                       // leader: resident weights
    uint64_t acc_done[2];                                  // peer: its epilogue warps have the accumulator
    MxEpiBars epi;
    uint32_t tmem_base;
    uint32_t abort_flag;
};

template <bool kBf16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_mx_d2_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_xs,
                    const __grid_constant__ CUtensorMap tmap_ws, const __grid_constant__ CUtensorMap tmap_y, const __grid_constant__ CUtensorMap tmap_r,
                    const MxD2Params p, const float *bias, const void *res, void *y, uint32_t *ws)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    MxD2Bars *bars = reinterpret_cast<MxD2Bars *>(smem + p.off_bar);
    volatile uint32_t *abort_flag = &bars->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();                  // 0: leader (issues the MMAs), 1: its peer
    const int pair = blockIdx.x >> 1, nK = (p.I + 63) / 64;
    const uint32_t peer_abort = map_to_cta(smem_u32(&bars->abort_flag), rank ^ 1u);
    const int groups_warps = p.t.acc == 2 ? 8 : kEpiWarps;     // epilogue warps that hand an accumulator back

    if (tid == 0) {
        for (int s = 0; s < p.S; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], 1); }
        mbar_init(&bars->w_full, 1);
        for (int a = 0; a < 2; ++a) mbar_init(&bars->acc_done[a], groups_warps);
        mx_epi_init(&bars->epi, p.t, groups_warps + 1);        // (the leader's: its own warps and the peer's relay)
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmap_x); prefetch_tensormap(&tmap_w); prefetch_tensormap(&tmap_xs); prefetch_tensormap(&tmap_ws);
        if (p.t.NS) { prefetch_tensormap(&tmap_y); if (res) prefetch_tensormap(&tmap_r); }
    }
    if (warp == 1) tmem_alloc_pair(&bars->tmem_base, 512);
    pdl_trigger();
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_relaxed();             // barriers of both CTAs exist before anything arrives on them
    tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
    pdl_wait();
    bias = behind_wait(bias); res = behind_wait(res);

    if (warp == 0) {
        // ---- TMA producer: this CTA's outputs, its half of the rows of X, the scales of its outputs and of all the rows ------------
        if (lane == 0) {
            const uint32_t full0 = map_to_cta(smem_u32(&bars->full[0]), 0u), w_full = map_to_cta(smem_u32(&bars->w_full), 0u);     // the leader's barriers
            const int half = p.t.N / 2, x_tiles = p.t.N / kRows;
            auto weights = [&](uint8_t *st, uint32_t bar, int ot, int step) {
                tma_load_2d_pair(st, &tmap_w, bar, step * 128, (ot * 2 + (int)rank) * kRows);
                tma_load_2d_pair(st + kWBytes, &tmap_ws, bar, 0, (ot * 2 + (int)rank) * p.nKT + 2 * step);
            };
            MxWalk w(p.t, pair, (int)rank);
            if (p.resident && w.in(p.t)) {
                if (rank == 0) mbar_arrive_expect_tx(&bars->w_full, 2u * p.nS * kWStage);
                for (int step = 0; step < p.nS; ++step) weights(smem + (size_t)step * kWStage, w_full, w.ot, step);
            }
            const uint32_t bytes = 2u * (p.x_bytes + p.xs_bytes + (p.resident ? 0u : kWStage));
            uint32_t s = 0, lap = 0;
            bool ok = true;
            for (; w.in(p.t) && ok; w.next(p.t)) {
                for (int step = 0; step < p.nS; ++step) {
                    if (lap >= 1 && !pair_wait(&bars->empty[s], (lap & 1u) ^ 1u, abort_flag, peer_abort, ws, 0xC100)) { ok = false; break; }
                    uint8_t *st = smem + p.off_stages + (size_t)s * p.stage_bytes;
                    const uint32_t bar = full0 + s * 8u;
                    if (rank == 0) mbar_arrive_expect_tx(&bars->full[s], bytes);
                    tma_load_2d_pair(st, &tmap_x, bar, step * 128, w.m0(p.t) + (int)rank * half);
                    for (int t = 0; t < x_tiles; ++t)
                        tma_load_2d_pair(st + p.x_bytes + t * kScaleBytes, &tmap_xs, bar, 0, (w.mt * x_tiles + t) * p.nKT + 2 * step);
                    if (!p.resident) weights(st + p.x_bytes + p.xs_bytes, bar, w.ot, step);
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
            for (int tile = pair; tile + p.t.acc * p.t.grid < p.t.n_tiles; tile += p.t.grid, ++it) {
                const uint32_t acc = p.t.acc == 2 ? it & 1u : 0u, lap = p.t.acc == 2 ? it >> 1 : it;
                if (!mbar_wait(&bars->acc_done[acc], lap & 1u, abort_flag, ws, 0xC700)) break;
                tc_fence_after_sync();
                tc_fence_before_sync();
                mbar_arrive_remote_release(acc_empty0 + acc * 8u);
            }
        } else {
            // ---- leader: MMAs and copies of scales for the pair -----------------------------------------------------------------
            const uint32_t base = smem_u32(smem) & 0x3FFFFu, xc = (uint32_t)p.t.N / 32;
            uint32_t s = 0, ph = 0, it = 0;
            bool ok = true;
            if (p.resident && pair < p.t.n_tiles) ok = pair_wait(&bars->w_full, 0, abort_flag, peer_abort, ws, 0xC310);
            for (int tile = pair; tile < p.t.n_tiles && ok; tile += p.t.grid, ++it) {
                const uint32_t acc = p.t.acc == 2 ? it & 1u : 0u, lap_acc = p.t.acc == 2 ? it >> 1 : it;
                if (lap_acc >= 1 && !pair_wait<true>(&bars->epi.acc_empty[acc], (lap_acc & 1u) ^ 1u, abort_flag, peer_abort, ws, 0xC200)) break;
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + acc * p.t.N, idesc0 = idesc_mxf4(256, (uint32_t)p.t.N, 0), idesc1 = idesc_mxf4(256, (uint32_t)p.t.N, 1);
                for (int step = 0; step < p.nS; ++step) {
                    if (!pair_wait(&bars->full[s], ph, abort_flag, peer_abort, ws, 0xC300)) { ok = false; break; }
                    tc_fence_after_sync();
                    const uint32_t xs = base + p.off_stages + s * p.stage_bytes, wst = p.resident ? base + step * kWStage : xs + p.x_bytes + p.xs_bytes;
                    const uint32_t a_lo = (wst >> 4) | kMxDescLboOne, b_lo = (xs >> 4) | kMxDescLboOne;
                    // tensor memory of this stage's scales: two tiles of W's, then X's, a K tile's row tiles side by side
                    const uint32_t sf = tmem_base + p.tmem_scales + s * p.scale_cols;
                    const int n = min(4, nK - 4 * step);
                    for (int t = 0; t < (n + 1) / 2; ++t) {
                        copy_scales_pair(sf + 4 * t, wst + kWBytes + t * kMxScaleTile);
                        for (int r = 0; r < p.t.N / kRows; ++r)
                            copy_scales_pair(sf + 8 + xc * t + 4 * r, xs + p.x_bytes + r * kScaleBytes + t * kMxScaleTile);
                    }
                    for (int j = 0; j < n; ++j)                                      // 64 columns = 32 bytes inside the swizzled row
                        mma_mxf4_ss_pair(d_tmem, mx_desc64(a_lo + 2 * j), mx_desc64(b_lo + 2 * j), j & 1 ? idesc1 : idesc0, sf + 4 * (j / 2), sf + 8 + xc * (j / 2),
                                         step > 0 || j > 0);
                    mma_commit_pair(&bars->empty[s]);
                    if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
                }
                if (ok) mma_commit_pair(&bars->epi.acc_full[acc]);
            }
        }
    } else if (warp == kStoreWarp) {
        if (lane == 0 && p.t.NS) mx_slab_copies(p.t, pair, (int)rank, smem, &bars->epi, &tmap_y, &tmap_r, res != nullptr, abort_flag, ws);
    } else {
        auto release = [&](uint32_t acc) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(rank == 0 ? &bars->epi.acc_empty[acc] : &bars->acc_done[acc]);
        };
        if (kBf16 && p.t.NS)
            mx_epilogue_slabs<2>(p.t, pair, (int)rank, warp - kFirstEpi, lane, warp & 3, smem_u32(smem), tmem_base, &bars->epi, bias, res != nullptr, abort_flag, ws, release);
        else
            mx_epilogue_rows<2, kBf16>(p.t, pair, (int)rank, warp - kFirstEpi, lane, warp & 3, tmem_base, &bars->epi, bias, res, y, abort_flag, ws, release);
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
        tmem_dealloc_pair(tmem_base, 512);
    }
}

// `variant`: rows of X in a tile (0: the choice), + (1 << 16): weights are loaded for every tile
bool plan(const npas_mx_linear_desc &d, MxD2Params &p, int sms)
{
    if (d.x_dtype != NPAS_MX4) return false;
    const MxLayout LW = mx_layout(d.O, d.I);
    p = MxD2Params{};
    p.I = d.I;
    p.y_bf16 = d.y_dtype == NPAS_BF16;
    p.nS = (d.I + kStepCols - 1) / kStepCols;
    p.nKT = (int)LW.nKT;
    const int pairs = sms / 2;
    const int N = d.variant & 0xFFFF ? d.variant & 0xFFFF : 256;
    if ((N != 128 && N != 256) || d.variant >> 17) return false;
    mx_tiles_plan(p.t, d, N, 2 * kRows, N == 128 ? 2 : 1, pairs);
    if (!p.t.n_tiles) return false;
    p.x_bytes = (uint32_t)N * 64u;
    p.xs_bytes = (uint32_t)N / kRows * kScaleBytes;
    const uint32_t budget = kSmemLimit - (uint32_t)sizeof(MxD2Bars) - 128u - 1024u;
    // Weights stay where four stages of the input and the slabs fit beside them and few pairs are idle for it
    const int same = pairs / p.t.n_ot * p.t.n_ot;              // pairs whose tiles all have the same outputs
    p.t.NS = !p.y_bf16 || d.O % 8 ? 0 : p.nS > 2 ? 2 : 4;
    p.resident = !(d.variant >> 16) && p.t.n_tiles > pairs && same * 8 >= pairs * 7 && p.nS * kWStage + 4 * (p.x_bytes + p.xs_bytes) + 4 * kMxSlabBytes <= budget;
    if (p.resident) mx_tiles_plan(p.t, d, N, 2 * kRows, p.t.acc, same);
    p.stage_bytes = p.x_bytes + p.xs_bytes + (p.resident ? 0u : kWStage);
    p.off_stages = p.resident ? (uint32_t)p.nS * kWStage : 0u;
    if (p.resident && p.t.NS) {
        p.t.NS = 4;
        if (d.has_residual && p.off_stages + 8 * kMxSlabBytes + 3 * p.stage_bytes <= budget) p.t.NS = 8;
    }
    p.t.ns_log = p.t.NS == 8 ? 3 : p.t.NS == 4 ? 2 : 1;
    // columns of tensor memory: sums, then scales of every stage
    p.tmem_scales = 256;
    p.scale_cols = 8 + 2 * (uint32_t)N / 32;
    p.S = (int)((budget - p.off_stages - (uint32_t)p.t.NS * kMxSlabBytes) / p.stage_bytes);
    if (p.S > kMaxStages) p.S = kMaxStages;
    if (p.S * p.scale_cols > 256) p.S = 256 / p.scale_cols;
    if (p.S < 2) return false;
    p.t.off_slabs = p.off_stages + (uint32_t)p.S * p.stage_bytes;
    p.off_bar = round_up(p.t.off_slabs + (uint32_t)p.t.NS * kMxSlabBytes, 128);
    p.smem_bytes = p.off_bar + (uint32_t)sizeof(MxD2Bars) + 1024u;
    return p.smem_bytes <= kSmemLimit;
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
    CUtensorMap tmx, tmw, tmxs, tmws;
    if (!mx_encode_values(&tmx, x, LX, d.M, (uint32_t)p.t.N / 2) || !mx_encode_values(&tmw, w, LW, d.O, kRows) || !mx_encode_scales(&tmxs, x, LX) ||
        !mx_encode_scales(&tmws, w, LW))
        return NPAS_ERR_CUDA;
    CUtensorMap tmy = tmx, tmr = tmx;
    if (p.t.NS && (!mx_encode_bf16(&tmy, y, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows) ||
                   (res && !mx_encode_bf16(&tmr, res, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows))))
        return NPAS_ERR_CUDA;
    const auto kernel = p.y_bf16 ? linear_mx_d2_kernel<true> : linear_mx_d2_kernel<false>;
    if (allow_dynamic_smem(reinterpret_cast<const void *>(kernel), (int)kSmemLimit) != NPAS_OK) return NPAS_ERR_CUDA;
    const cudaError_t e = launch_pdl(Launch(), kernel, dim3((unsigned)p.t.grid * 2), dim3(kThreads), p.smem_bytes, st, tmx, tmw, tmxs, tmws, tmy, tmr, p, bias, res, y, ws);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
