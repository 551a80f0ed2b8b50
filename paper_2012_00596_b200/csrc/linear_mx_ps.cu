// GEMM with microscaled 4-bit weights, persistent tiles: 128 outputs x N input rows (N = 128 or 256) per MMA, weights as the
// 128-row operand like in linear_mx_sw.cu.
//
// A CTA per SM walks tiles (outputs fastest, so that the rows of X of a tile are read from L2 by its neighbours).  Copies, MMAs, with a
// 16-bit input the widening of the weights into tensor memory, and the epilogue are roles of their own that hand stages, slots and
// accumulators on through barriers, so the next tile is loaded and multiplied while one is written out.  Two accumulators of 128 columns,
// or one of 256 (with 256 rows of X a weight is fetched half as often, which long inputs need).
//
// Tensor memory lane = output, column = row of X, while a row of Y has its outputs side by side.  bf16 outputs whose rows start on 16-byte
// boundaries go through shared memory: a warp takes 32 outputs x 32 rows out of tensor memory as 8 x 8 matrices, rounds pairs of rows
// and stores them transposed (stmatrix) into a slab of 128 rows x 64 outputs, 128-byte swizzled, which leaves by TMA; residuals arrive
// in the slab by TMA before and are read the same way, requested a ring of slots ahead.  2.3 instructions an output (4.3 with a
// residual).  Other outputs (fp32, odd widths) are written from registers: 32 consecutive outputs of a row a warp, whatever the alignment,
// residuals requested before the wait for the accumulator.
// Every wait is bounded.
#include <type_traits>

#include "mx_tc.cuh"

namespace npas {

using namespace tc;

namespace {

constexpr int kRows = 128;
constexpr int kStepCols = 256;                             // columns of a weight stage
constexpr int kMaxStages = 6, kMaxXStages = 8, kSlots = 4;
constexpr uint32_t kSmemLimit = 232448;
constexpr int kMaxSlots = 8;
constexpr uint32_t kWBytes = kRows * 128;
constexpr uint32_t kSlabBytes = kRows * 128;               // 128 rows x 64 outputs
constexpr uint32_t kScaleBytes = 2 * kMxScaleTile;         // of 128 rows and a stage

// warps: 0 copies, 1 MMAs, then a 16-bit input's own copies and the widening warps, then the epilogue, one of them for the slabs' copies
template <bool kMx> struct Roles {
    static constexpr int kXWarp = 2, kWideWarps = kMx ? 0 : 8, kFirstWide = 3;
    static constexpr int kFirstEpi = kMx ? 2 : kFirstWide + kWideWarps + 1;
    static constexpr int kEpiWarps = kMx ? 16 : 8, kGroups = kEpiWarps / 8;
    static constexpr int kStoreWarp = kMx ? kFirstEpi + kEpiWarps : kFirstWide + kWideWarps;
    static constexpr int kThreads = (kFirstEpi + kEpiWarps + (kMx ? 1 : 0)) * 32;
};

struct MxPsParams {
    int M, I, O, N, acc, nS, nMT, nOT, n_tiles, nKT, S, SX, NS, ns_log;
    // acc: accumulators; SX: stages of the input (16 bits); NS = 2^ns_log: slabs (0: none)
    int grid, step_mt, step_ot;                                  // a CTA's way from tile to tile
    int relu, y_bf16;
    uint32_t x_bytes, xs_bytes, stage_bytes, off_x, off_slabs, off_bar, smem_bytes, tmem_cols, tmem_scales, scale_cols;
    uint64_t w_scales, x_scales;                           // offsets of the scales in the blobs
};

struct MxPsBars {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t x_full[kMaxXStages], x_empty[kMaxXStages];
    uint64_t slot_full[kSlots], slot_empty[kSlots];
    uint64_t acc_full[2], acc_empty[2];
    uint64_t slab_ready[kMaxSlots], slab_done[kMaxSlots];  // free (or its residuals have landed) / every epilogue warp has finished its part
    uint32_t tmem_base;
    uint32_t abort_flag;
};

// 32 rows of one output: bias + residuals, then sums + those, ReLU, one rounding.  `at`: element of the first row; `n`: rows there are
// (none where the output lies past the end).
// (The pointer walks from row to row: 32 addresses at once would not fit beside the sums.)
template <bool kBf16>
__device__ __forceinline__ void load_residuals(float (&add)[32], float b, const void *res, int64_t at, int64_t O, int n)
{
    using T = typename std::conditional<kBf16, uint16_t, float>::type;
    const T *q = static_cast<const T *>(res) + at;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        add[i] = 0.f;
        if (i < n) {
            if constexpr (kBf16) add[i] = __uint_as_float((uint32_t)__ldg(q) << 16);
            else add[i] = __ldg(q);
        }
        q += O;
        asm volatile("" : "+l"(q));
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) add[i] += b;
}
template <bool kBf16>
__device__ __forceinline__ void store_rows(const uint32_t (&v)[32], const float (&add)[32], void *y, int64_t at, int64_t O, int n, int relu)
{
    using T = typename std::conditional<kBf16, uint16_t, float>::type;
    T *q = static_cast<T *>(y) + at;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        float u = __uint_as_float(v[i]) + add[i];
        if (relu) u = fmaxf(u, 0.f);
        if (i < n) {
            if constexpr (kBf16) *q = (uint16_t)cvt_bf16x2(u, 0.f);
            else *q = u;
        }
        q += O;
        asm volatile("" : "+l"(q));
    }
}

// the tiles of a CTA (the coordinates are carried along: two divisions a tile take longer than some roles' work on it)
struct TileWalk {
    int tile, mt, ot;
    __device__ __forceinline__ explicit TileWalk(const MxPsParams &p) : tile(blockIdx.x), mt(blockIdx.x / p.nOT), ot(blockIdx.x - mt * p.nOT) {}
    __device__ __forceinline__ bool in(const MxPsParams &p) const { return tile < p.n_tiles; }
    __device__ __forceinline__ void next(const MxPsParams &p)
    {
        tile += gridDim.x; mt += p.step_mt; ot += p.step_ot;
        if (ot >= p.nOT) { ot -= p.nOT; ++mt; }
    }
    // blocks of 128 rows and halves of 64 outputs that exist
    __device__ __forceinline__ int blocks(const MxPsParams &p) const { return min(p.N / kRows, (p.M - mt * p.N + kRows - 1) / kRows); }
    __device__ __forceinline__ int halves(const MxPsParams &p) const { return ot * kRows + 64 < p.O ? 2 : 1; }
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

    if (tid == 0) {
        for (int s = 0; s < p.S; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], kMx ? 1 : R::kWideWarps); }
        for (int s = 0; s < p.SX; ++s) { mbar_init(&bars->x_full[s], 1); mbar_init(&bars->x_empty[s], 1); }
        for (int s = 0; s < kSlots; ++s) { mbar_init(&bars->slot_full[s], 4); mbar_init(&bars->slot_empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&bars->acc_full[a], 1); mbar_init(&bars->acc_empty[a], p.acc == 2 ? 8 : R::kEpiWarps); }
        for (int n = 0; n < p.NS; ++n) { mbar_init(&bars->slab_ready[n], 1); mbar_init(&bars->slab_done[n], 4); }
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tensormap(&tmap_x);
        prefetch_tensormap(&tmap_w);
        if (p.NS) { prefetch_tensormap(&tmap_y); if (res) prefetch_tensormap(&tmap_r); }
    }
    if (warp == 1) tmem_alloc(&bars->tmem_base, p.tmem_cols);
    pdl_trigger();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
    pdl_wait();
    const int z = zero_behind_wait();

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, lap = 0;
            bool ok = true;
            for (TileWalk w(p); w.in(p) && ok; w.next(p)) {
                const int mt = w.mt, ot = w.ot;
                for (int step = 0; step < p.nS; ++step) {
                    if (lap >= 1 && !mbar_wait(&bars->empty[s], (lap & 1u) ^ 1u, abort_flag, ws, 0xB100)) { ok = false; break; }
                    uint8_t *st = smem + (size_t)s * p.stage_bytes;
                    const uint32_t sb = (uint32_t)min(2, p.nKT - 2 * step) * kMxScaleTile;   // (the last tile of columns may stand alone)
                    // row tiles of X's scales: those that exist
                    const int xt = kMx ? min(p.N / kRows, (p.M + kRows - 1) / kRows - mt * (p.N / kRows)) : 0;
                    mbar_arrive_expect_tx(&bars->full[s], kWBytes + sb + (kMx ? p.x_bytes + xt * sb : 0u));
                    tma_load_2d(st, &tmap_w, &bars->full[s], step * 128, ot * kRows);
                    bulk_load_1d(st + kWBytes, wblob + p.w_scales + ((uint64_t)ot * p.nKT + 2 * step) * kMxScaleTile, sb, &bars->full[s]);
                    if (kMx) {
                        tma_load_2d(st + kWBytes + kScaleBytes + p.xs_bytes, &tmap_x, &bars->full[s], step * 128, mt * p.N);
                        for (int t = 0; t < xt; ++t)
                            bulk_load_1d(st + kWBytes + kScaleBytes + t * kScaleBytes,
                                         xblob + p.x_scales + ((uint64_t)(mt * (p.N / kRows) + t) * p.nKT + 2 * step) * kMxScaleTile, sb, &bars->full[s]);
                    }
                    if (++s == (uint32_t)p.S) { s = 0; ++lap; }
                }
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t base = smem_u32(smem) & 0x3FFFFu;
            uint32_t s = 0, ph = 0, it = 0, k_all = 0;
            bool ok = true;
            for (int tile = blockIdx.x; tile < p.n_tiles && ok; tile += gridDim.x, ++it) {
                const uint32_t acc = p.acc == 2 ? it & 1u : 0u, lap_acc = p.acc == 2 ? it >> 1 : it;
                if (lap_acc >= 1 && !mbar_wait(&bars->acc_empty[acc], (lap_acc & 1u) ^ 1u, abort_flag, ws, 0xB200)) break;
                tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + acc * p.N;
                if (kMx) {
                    for (int step = 0; step < p.nS; ++step) {
                        if (!mbar_wait(&bars->full[s], ph, abort_flag, ws, 0xB300)) { ok = false; break; }
                        tc_fence_after_sync();
                        const uint32_t st = base + s * p.stage_bytes, a_lo = (st >> 4) | kMxDescLboOne;
                        const uint32_t b_lo = ((st + kWBytes + kScaleBytes + p.xs_bytes) >> 4) | kMxDescLboOne;
                        // tensor memory of this stage's scales: two tiles of W's, then X's, a K tile's row tiles side by side
                        const uint32_t sf = tmem_base + p.tmem_scales + s * p.scale_cols, xc = (uint32_t)p.N / 32;
                        const int n = min(4, nK - 4 * step);
                        for (int t = 0; t < (n + 1) / 2; ++t) {
                            copy_scales(sf + 4 * t, st + kWBytes + t * kMxScaleTile);
                            for (int r = 0; r < p.N / kRows; ++r)
                                copy_scales(sf + 8 + xc * t + 4 * r, st + kWBytes + kScaleBytes + r * kScaleBytes + t * kMxScaleTile);
                        }
                        for (int j = 0; j < n; ++j)                                  // 64 columns = 32 bytes inside the swizzled row
                            mma_mxf4_ss(d_tmem, mx_desc64(a_lo + 2 * j), mx_desc64(b_lo + 2 * j), idesc_mxf4(128, (uint32_t)p.N, j & 1),
                                        sf + 4 * (j / 2), sf + 8 + xc * (j / 2), step > 0 || j > 0);
                        mma_commit(&bars->empty[s]);
                        if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
                    }
                } else {
                    const uint32_t idesc = idesc_bf16_f32(128, (uint32_t)p.N), xb = base + p.off_x;
                    for (int k = 0; k < nK; ++k, ++k_all) {
                        const uint32_t slot = k_all % kSlots;
                        if (!mbar_wait(&bars->x_full[s], ph, abort_flag, ws, 0xB310) ||
                            !mbar_wait(&bars->slot_full[slot], (k_all / kSlots) & 1u, abort_flag, ws, 0xB320)) { ok = false; break; }
                        tc_fence_after_sync();
                        const uint32_t b_lo = ((xb + s * p.x_bytes) >> 4) | kMxDescLboOne, a_t = tmem_base + p.tmem_scales + slot * 32u;
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j)
                            mma_bf16_ts(d_tmem, a_t + 8 * j, mx_desc64(b_lo + 2 * j), idesc, (k > 0 || j > 0) ? 1u : 0u);
                        mma_commit(&bars->slot_empty[slot]);
                        mma_commit(&bars->x_empty[s]);
                        if (++s == (uint32_t)p.SX) { s = 0; ph ^= 1u; }
                    }
                }
                if (ok) mma_commit(&bars->acc_full[acc]);
            }
        }
    } else if (!kMx && warp == R::kXWarp) {
        if (lane == 0) {
            uint32_t s = 0, lap = 0;
            bool ok = true;
            for (TileWalk w(p); w.in(p) && ok; w.next(p)) {
                for (int k = 0; k < nK; ++k) {
                    if (lap >= 1 && !mbar_wait(&bars->x_empty[s], (lap & 1u) ^ 1u, abort_flag, ws, 0xB110)) { ok = false; break; }
                    mbar_arrive_expect_tx(&bars->x_full[s], p.x_bytes);
                    tma_load_2d(smem + p.off_x + (size_t)s * p.x_bytes, &tmap_x, &bars->x_full[s], k * 64, w.mt * p.N);
                    if (++s == (uint32_t)p.SX) { s = 0; ++lap; }
                }
            }
        }
    } else if (!kMx && warp < R::kFirstWide + R::kWideWarps) {
        // ---- widening: group g of four warps takes every second K step, a thread one row of the weights -----------------
        const int group = (warp - R::kFirstWide) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
        bool ok = true;
        uint32_t s = 0, ph = 0, k0 = 0;                        // k0: K steps before this stage
        for (int tile = blockIdx.x; tile < p.n_tiles && ok; tile += gridDim.x) {
            for (int step = 0; step < p.nS && ok; ++step) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->full[s], ph, abort_flag, ws, 0xB400));
                if (!ok) break;
                const uint8_t *st = smem + (size_t)s * p.stage_bytes;
                const int n = min(4, nK - 4 * step);
                for (int q = (int)((group ^ k0) & 1u); q < n; q += 2) {
                    const uint32_t k = k0 + q, slot = k % kSlots;
                    const uint4 a = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q) ^ (r & 7)) * 16);
                    const uint4 b = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q + 1) ^ (r & 7)) * 16);
                    const uint32_t codes = *reinterpret_cast<const uint32_t *>(st + kWBytes + (q >> 1) * kMxScaleTile + lane * 16 + quarter * 4) >> (16 * (q & 1));
                    uint32_t v[32];
                    mx_widen(v, a, b, codes & 255u, (codes >> 8) & 255u);
                    if (k >= kSlots) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->slot_empty[slot], ((k / kSlots) & 1u) ^ 1u, abort_flag, ws, 0xB410));
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
                k0 += n;
                if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
            }
        }
    } else if (warp == R::kStoreWarp) {
        // ---- slabs: one leaves by TMA as soon as every epilogue warp has finished its part; when the store before it has been read,
        // that slab is free again, or takes the residuals of the slab a ring further on ----------------------------------------
        if (lane == 0 && p.NS) {
            // the slabs of this CTA's tiles in order: (tile, 128 rows, 64 outputs), those that exist
            struct Walk {
                TileWalk t;
                int r, h, blocks, halves;
                bool more;
                __device__ explicit Walk(const MxPsParams &p) : t(p), r(0), h(0), blocks(t.blocks(p)), halves(t.halves(p)), more(t.in(p)) {}
                __device__ void next(const MxPsParams &p)
                {
                    if (++h < halves) return;
                    h = 0;
                    if (++r < blocks) return;
                    r = 0;
                    t.next(p);
                    more = t.in(p); blocks = t.blocks(p); halves = t.halves(p);
                }
                __device__ int row(const MxPsParams &p) const { return t.mt * p.N + r * kRows; }
                __device__ int col(const MxPsParams &) const { return t.ot * kRows + h * 64; }
            };
            const uint32_t mask = (uint32_t)p.NS - 1;
            auto request = [&](const Walk &w, uint32_t n) {
                uint64_t *bar = &bars->slab_ready[n & mask];
                mbar_arrive_expect_tx(bar, kSlabBytes);
                tma_load_2d(smem + p.off_slabs + (size_t)(n & mask) * kSlabBytes, &tmap_r, bar, w.col(p), w.row(p));
            };
            Walk ahead(p);
            uint32_t n = 0, asked = 0;
            for (; res && asked < (uint32_t)p.NS && ahead.more; ++asked) { request(ahead, asked); ahead.next(p); }
            for (Walk w(p); w.more; w.next(p), ++n) {
                if (!mbar_wait(&bars->slab_done[n & mask], (n >> p.ns_log) & 1u, abort_flag, ws, 0xB600)) break;
                tma_store_2d(&tmap_y, smem + p.off_slabs + (size_t)(n & mask) * kSlabBytes, w.col(p), w.row(p));
                bulk_commit();
                if (n) {
                    bulk_wait_read<1>();
                    if (!res) mbar_arrive(&bars->slab_ready[(n - 1) & mask]);
                    else if (ahead.more) { request(ahead, asked++); ahead.next(p); }     // (slab n - 1 + NS)
                }
            }
            bulk_wait_read<0>();                               // the slabs stay valid until the last store has read them
        }
    } else if (warp >= R::kFirstEpi && p.NS) {
        // ---- epilogue through slabs.  Groups of eight warps: with two accumulators a group has every other tile (while one waits for
        // tensor memory or a barrier the other one computes), with one accumulator a block of 128 rows of every tile.  Warp -> lane
        // quarter and 64 of a block's 128 rows -----------------------------------------------------------------------------
        const int e = warp - R::kFirstEpi, group = e >> 3, quarter = warp & 3, part = (e >> 2) & 1, half = quarter >> 1;
        // this lane's row and 16-byte piece in the slab: row (lane % 8) of 8 x 8 matrix (lane / 8)
        const uint32_t lane_at = smem_u32(smem) + p.off_slabs + (uint32_t)((part * 64 + (lane & 7)) * 128 + ((((quarter & 1) * 4 + (lane >> 3)) ^ (lane & 7)) * 16));
        uint32_t it = 0, n = 0;                                // n: slabs of the tiles before
        bool ok = true;
        for (TileWalk w(p); w.in(p) && ok; w.next(p), ++it) {
            const int halves = w.halves(p), blocks = w.blocks(p);
            const uint32_t n_tile = n;
            n += (uint32_t)(halves * blocks);
            if (p.acc == 2 && R::kGroups == 2 && (it & 1u) != (uint32_t)group) continue;
            const int o0 = w.ot * kRows + quarter * 32 + (lane >> 2);
            const uint32_t acc = p.acc == 2 ? it & 1u : 0u, lap = p.acc == 2 ? it >> 1 : it;
            float b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = bias && o0 + 8 * i < p.O ? __ldg(bias + o0 + 8 * i + z) : 0.f;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full[acc], lap & 1u, abort_flag, ws, 0xB500));
            if (!ok) break;
            tc_fence_after_sync();
            const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * p.N + (uint32_t)(part * 64);
            for (int r = p.acc == 1 && R::kGroups == 2 ? group : 0; r < blocks && half < halves && ok; r += p.acc == 1 ? R::kGroups : 1) {
                const uint32_t at = n_tile + (uint32_t)(r * halves + half), slot = at & (p.NS - 1), slab = lane_at + slot * kSlabBytes, use = at >> p.ns_log;
                // with residuals: they have landed; without: the store that last used the slab has read it (from its second use on)
                if (res || use) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->slab_ready[slot], (res ? use : use - 1) & 1u, abort_flag, ws, 0xB510));
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < 64; c += 32) {
                    uint32_t u[16], v[16];                     // outputs 0 to 15 and 16 to 31 of the quarter
                    tmem_ld_16x32(t_addr + r * kRows + c, u);
                    tmem_ld_16x32(t_addr + r * kRows + c + (16u << 16), v);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 4; ++k) {              // eight rows of Y
                        float f[8] = {__uint_as_float(u[4 * k]) + b[0], __uint_as_float(u[4 * k + 1]) + b[0], __uint_as_float(u[4 * k + 2]) + b[1],
                                      __uint_as_float(u[4 * k + 3]) + b[1], __uint_as_float(v[4 * k]) + b[2], __uint_as_float(v[4 * k + 1]) + b[2],
                                      __uint_as_float(v[4 * k + 2]) + b[3], __uint_as_float(v[4 * k + 3]) + b[3]};
                        const uint32_t sa = slab + (uint32_t)(c + 8 * k) * 128u;
                        if (res) {
                            uint32_t q[4];
                            ldmatrix_x4_trans(sa, q);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                f[2 * i] += __uint_as_float(q[i] << 16);
                                f[2 * i + 1] += __uint_as_float(q[i] & 0xFFFF0000u);
                            }
                        }
                        // one rounding, then ReLU on the rounded pairs (max with +0 is exact on them)
                        uint32_t h[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            h[i] = cvt_bf16x2(f[2 * i], f[2 * i + 1]);
                            if (p.relu) h[i] = relu_bf16x2(h[i]);
                        }
                        if (res) __syncwarp();                 // (every lane has read these rows' residuals)
                        stmatrix_x4_trans(sa, h[0], h[1], h[2], h[3]);
                    }
                }
                fence_proxy_async_smem();                      // the TMA store reads what this thread wrote
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->slab_done[slot]);
            }
            if (!ok) break;
            // this warp has read its part of the accumulator: the MMA warp may overwrite it
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->acc_empty[acc]);
        }
    } else if (warp >= R::kFirstEpi) {
        // ---- epilogue from registers, by the same groups; a lane writes one output of 64 rows of a block ----------------------
        const int e = warp - R::kFirstEpi, group = e >> 3, quarter = warp & 3, part = (e >> 2) & 1;
        uint32_t it = 0;
        bool ok = true;
        for (TileWalk w(p); w.in(p) && ok; w.next(p), ++it) {
            if (p.acc == 2 && R::kGroups == 2 && (it & 1u) != (uint32_t)group) continue;
            const int o = w.ot * kRows + quarter * 32 + lane, blocks = w.blocks(p);
            const uint32_t acc = p.acc == 2 ? it & 1u : 0u, lap = p.acc == 2 ? it >> 1 : it;
            const float b = bias && o < p.O ? __ldg(bias + o + z) : 0.f;
            bool waited = false;
            for (int r = p.acc == 1 && R::kGroups == 2 ? group : 0; r < blocks && ok; r += p.acc == 1 ? R::kGroups : 1)
                for (int c = 0; c < 64 && ok; c += 32) {
                    const int m0 = w.mt * p.N + r * kRows + part * 64 + c, n = o < p.O ? p.M - m0 : 0;       // rows from m0 on (may be none)
                    const int64_t at = (int64_t)m0 * p.O + o + z;
                    float add[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) add[i] = b;
                    if (res) load_residuals<kBf16>(add, b, res, at, p.O, n);
                    if (!waited) {
                        ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full[acc], lap & 1u, abort_flag, ws, 0xB520));
                        if (!ok) break;
                        tc_fence_after_sync();
                        waited = true;
                    }
                    uint32_t v[32];
                    tmem_ld_x32(tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * p.N + (uint32_t)(r * kRows + part * 64 + c), v);
                    tmem_ld_wait();
                    store_rows<kBf16>(v, add, y, at, p.O, n, p.relu);
                }
            if (ok && !waited) {                               // (no block of this tile is the group's: it hands the accumulator on all the same)
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full[acc], lap & 1u, abort_flag, ws, 0xB530));
                tc_fence_after_sync();
            }
            if (!ok) break;
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->acc_empty[acc]);
        }
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
    p.M = d.M; p.I = d.I; p.O = d.O;
    p.relu = d.relu; p.y_bf16 = d.y_dtype == NPAS_BF16;
    p.nS = (d.I + kStepCols - 1) / kStepCols;
    p.nKT = (int)LW.nKT;
    p.nOT = (d.O + kRows - 1) / kRows;
    p.N = d.variant ? d.variant : (d.I >= 2048 && (long long)((d.M + 255) / 256) * p.nOT >= sms ? 256 : 128);
    if (p.N != 128 && p.N != 256) return false;
    p.acc = p.N == 128 ? 2 : 1;
    p.nMT = (d.M + p.N - 1) / p.N;
    const long long tiles = (long long)p.nMT * p.nOT;
    if (tiles > 0x7FFFFFFF) return false;
    p.n_tiles = (int)tiles;
    const int grid = p.n_tiles < sms ? p.n_tiles : sms;
    p.grid = grid; p.step_mt = grid / p.nOT; p.step_ot = grid % p.nOT;
    p.w_scales = LW.off_scales; p.x_scales = LX.off_scales;
    p.x_bytes = (uint32_t)p.N * 128u;
    p.xs_bytes = mx ? (uint32_t)p.N / kRows * kScaleBytes : 0u;
    p.stage_bytes = round_up(kWBytes + kScaleBytes + (mx ? p.xs_bytes + p.x_bytes : 0u), 1024);
    const uint32_t budget = kSmemLimit - (uint32_t)sizeof(MxPsBars) - 128u - 1024u;
    // Slabs for bf16 outputs with rows on 16-byte boundaries: four, eight where residuals are ahead of little else; and the input's ring
    p.NS = p.y_bf16 && d.O % 8 == 0 ? (mx && d.has_residual && p.nS <= 2 && p.N == 128 ? 8 : 4) : 0;
    p.ns_log = p.NS == 8 ? 3 : 2;
    if (!mx) p.SX = p.N == 256 ? 3 : 6;
    const uint32_t fixed = (uint32_t)p.SX * p.x_bytes + (uint32_t)p.NS * kSlabBytes;
    p.S = (int)((budget - fixed) / p.stage_bytes);
    if (p.S > kMaxStages) p.S = kMaxStages;
    if (p.S < 2) return false;
    p.off_x = (uint32_t)p.S * p.stage_bytes;
    p.off_slabs = p.off_x + (uint32_t)p.SX * p.x_bytes;
    p.off_bar = round_up(p.off_slabs + (uint32_t)p.NS * kSlabBytes, 128);
    p.smem_bytes = p.off_bar + (uint32_t)sizeof(MxPsBars) + 1024u;
    if (p.smem_bytes > kSmemLimit) return false;
    p.tmem_scales = 256;
    p.scale_cols = 8 + 2 * (uint32_t)p.N / 32;
    const uint32_t cols = p.tmem_scales + (mx ? p.scale_cols * p.S : 32u * kSlots);
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
    if (!(mx ? mx_encode_values(&tmx, x, mx_layout(d.M, d.I), d.M, (uint32_t)p.N)
             : mx_encode_bf16(&tmx, x, (uint64_t)d.I, (uint64_t)x_pitch, (uint64_t)d.M, (uint32_t)p.N)))
        return NPAS_ERR_CUDA;
    CUtensorMap tmy = tmx, tmr = tmx;
    if (p.NS && (!mx_encode_bf16(&tmy, y, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows) ||
                 (res && !mx_encode_bf16(&tmr, res, (uint64_t)d.O, (uint64_t)d.O, (uint64_t)d.M, kRows))))
        return NPAS_ERR_CUDA;
    const auto kernel = mx ? (p.y_bf16 ? linear_mx_ps_kernel<true, true> : linear_mx_ps_kernel<true, false>)
                           : (p.y_bf16 ? linear_mx_ps_kernel<false, true> : linear_mx_ps_kernel<false, false>);
    if (allow_dynamic_smem(reinterpret_cast<const void *>(kernel), (int)kSmemLimit) != NPAS_OK) return NPAS_ERR_CUDA;
    const cudaError_t e = launch_pdl(Launch(), kernel, dim3((unsigned)p.grid), dim3(mx ? Roles<true>::kThreads : Roles<false>::kThreads),
                                     p.smem_bytes, st, tmx, tmw, tmy, tmr, p, static_cast<const uint8_t *>(x), static_cast<const uint8_t *>(w), bias, res, y, ws);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
