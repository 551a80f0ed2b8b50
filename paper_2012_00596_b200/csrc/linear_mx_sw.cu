// GEMM with microscaled 4-bit weights for few rows: the weights are the tensor core's 128-row operand, the input's rows its columns.
//
// Y^T[o, m] = sum_i W[o,i] X[m,i]: an MMA takes 128 outputs x N input rows (N = 16 to 128), so a single row of X costs a sixteenth of what it
// would as the 128-row operand, and the weights, which are all the bytes there are with few rows, stream through shared memory
// once.  A tile is shared by a cluster of KS CTAs that split the input columns in steps of 256 (a row of a 128-byte swizzled
// box); partial sums go through distributed shared memory to the CTA that owns the input rows and are added in rank order, so
// results do not depend on timing.  Tensor memory lane = output, column = input row: the epilogue's stores are 32 consecutive outputs a warp.
//   4-bit input: both operands by TMA as they lie in the blobs, scales copied from shared into tensor memory ahead of the MMAs of a
//     step (a set of columns per ring stage, so that no copy meets an MMA that still reads), MMAs of kind::mxf4 over 64 columns.
//   16-bit input to be quantised: the eight warps that have nothing to do before the epilogue quantise the CTA's share of X into the stage, a row
//     of 256 columns a warp, instead of a launch of its own ahead of this one (a call of one row 6.0 -> 4.2 us of host time).
//   16-bit input: sixteen warps widen the weights, a thread a row: 32 bytes -> 64 bf16 values in 32 columns of tensor memory, from where the
//     MMAs of kind::f16 take their first operand.  Slots of two steps; weights and inputs have rings of their own (256 and 128 columns a
//     stage).  Widening costs 2.4 instructions a weight (17 for eight of them; scales, loads and stores), 0.32 us a stage of 128 x 256 at the issue rate; a
//     stage takes 0.88 (64x4096 -> 4096 9.9 us): each group of four warps has one slot, and widens again when the MMAs of its last one are done.
// Every wait is bounded.
#include <type_traits>

#include "mx_tc.cuh"
#include "tc_pair.cuh"

namespace npas {

using namespace tc;

namespace {

constexpr int kRows = 128;
constexpr int kStepCols = 256;                             // columns of a weight stage
constexpr int kMaxStages = 6, kMaxXStages = 4, kSlots = 4;
constexpr uint32_t kSlotCols = 64;                         // tensor memory of a slot: 128 widened columns of the weights
constexpr int kMaxSplit = 8;                               // portable cluster size
constexpr uint32_t kSmemLimit = 232448, kSmemHalf = 115712;   // of a CTA alone on its SM, of one of two (1 KB each is the system's)
constexpr uint32_t kWBytes = kRows * 128;
constexpr uint32_t kScaleBytes = 2 * kMxScaleTile;         // of 128 rows and a stage

struct MxSwParams {
    int M, I, O, N, KS, nS, spr, nMT, nOT, nKT, S, SX, slots, cpr;   // spr: steps per CTA; SX: stages of two K steps of the input (16 bits); cpr: input rows a CTA owns
    int relu, y_bf16;
    uint32_t x_bytes, stage_bytes, off_x, off_red, red_pitch, off_bar, smem_bytes, tmem_cols, tmem_scales;
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

__device__ __forceinline__ void st_cluster_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
template <bool kBf16> __device__ __forceinline__ float load_res(const void *res, int64_t at)
{
    if constexpr (kBf16) return bf16_bits_to_f32(__ldg(static_cast<const uint16_t *>(res) + at));
    else return __ldg(static_cast<const float *>(res) + at);
}
template <bool kBf16> __device__ __forceinline__ void store_y(void *y, int64_t at, float v, int relu)
{
    if (relu) v = fmaxf(v, 0.f);
    if constexpr (kBf16) static_cast<uint16_t *>(y)[at] = (uint16_t)cvt_bf16x2(v, 0.f);
    else static_cast<float *>(y)[at] = v;
}

// what the input is: a blob, 16 bits to be quantised, 16 bits
enum MxIn { kBlob, kQuantize, kWide };

// warps: 0 copies, 1 MMAs, then those that widen or quantise and make the epilogue, last the copies of a 16-bit input.  Sixteen widen: eight
// took 500 cycles for two K steps each, the MMAs of a step 50 to 250
template <MxIn kIn> struct SwRoles {
    static constexpr int kEpiWarps = kIn == kWide ? 16 : 8, kXWarp = 2 + kEpiWarps, kThreads = (kXWarp + 1) * 32, kPerSm = kIn == kWide ? 1 : 2;
};

template <MxIn kIn, bool kBf16>
__global__ void __launch_bounds__(SwRoles<kIn>::kThreads, SwRoles<kIn>::kPerSm)
linear_mx_sw_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w, const MxSwParams p, const uint8_t *xin,
                    const uint8_t *wblob, const float *bias, const void *res, void *y, uint32_t *ws)
{
    constexpr bool kMx = kIn != kWide;
    constexpr int kEpiWarps = SwRoles<kIn>::kEpiWarps, kXWarp = SwRoles<kIn>::kXWarp, kThreads = SwRoles<kIn>::kThreads;
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
        for (int s = 0; s < p.S; ++s) { mbar_init(&bars->full[s], kIn == kQuantize ? 1 + kEpiWarps : 1); mbar_init(&bars->empty[s], kMx ? 1 : kEpiWarps); }
        for (int s = 0; s < p.SX; ++s) { mbar_init(&bars->x_full[s], 1); mbar_init(&bars->x_empty[s], 1); }
        for (int s = 0; s < p.slots; ++s) { mbar_init(&bars->slot_full[s], 4); mbar_init(&bars->slot_empty[s], 1); }
        mbar_init(&bars->acc_full, 1);
        bars->abort_flag = 0;
        fence_barrier_init();
        if (kIn != kQuantize) prefetch_tensormap(&tmap_x);
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
    xin = behind_wait(xin); wblob = behind_wait(wblob);

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
                mbar_arrive_expect_tx(&bars->full[s], kWBytes + sb + (kIn == kBlob ? p.x_bytes + sb : 0u));
                tma_load_2d(st, &tmap_w, &bars->full[s], step * 128, ot * kRows);
                bulk_load_1d(st + kWBytes, wblob + p.w_scales + ((uint64_t)ot * p.nKT + 2 * step) * kMxScaleTile, sb, &bars->full[s]);
                if (kIn == kBlob) {
                    tma_load_2d(st + kWBytes + 2 * kScaleBytes, &tmap_x, &bars->full[s], step * 128, mt * kRows);
                    bulk_load_1d(st + kWBytes + kScaleBytes, xin + p.x_scales + ((uint64_t)mt * p.nKT + 2 * step) * kMxScaleTile, sb, &bars->full[s]);
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
                // a slot and a stage of X are two K steps: eight MMAs without a branch between them
                uint32_t sx = 0, phx = 0, slot = 0, slot_ph = 0, more = 0;
                const uint32_t idesc = idesc_bf16_f32(128, (uint32_t)p.N), x16 = p.x_bytes >> 4, xb = ((base + p.off_x) >> 4) | kMxDescLboOne;
                auto step = [&](uint32_t b_lo, uint32_t a_t) {
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) { mma_bf16_ts(tmem_base, a_t + 8 * j, mx_desc64(b_lo + 2 * j), idesc, more); more = 1; }
                };
                for (int k = 0; k < k_n; k += 2) {
                    if (!mbar_wait(&bars->x_full[sx], phx, abort_flag, ws, 0xA310) ||
                        !mbar_wait(&bars->slot_full[slot], slot_ph, abort_flag, ws, 0xA320)) { go = false; break; }
                    tc_fence_after_sync();
                    const uint32_t b_lo = xb + sx * 2u * x16, a_t = tmem_base + p.tmem_scales + slot * kSlotCols;
                    if (k + 1 < k_n) { step(b_lo, a_t); step(b_lo + x16, a_t + 32u); }
                    else step(b_lo, a_t);
                    mma_commit(&bars->slot_empty[slot]);
                    mma_commit(&bars->x_empty[sx]);
                    if (++slot == (uint32_t)p.slots) { slot = 0; slot_ph ^= 1u; }
                    if (++sx == (uint32_t)p.SX) { sx = 0; phx ^= 1u; }
                }
            }
            if (go) mma_commit(&bars->acc_full);
        }
        __syncwarp();
    } else if (warp == kXWarp) {
        if (!kMx && lane == 0) {
            uint32_t sx = 0, lap = 0;
            for (int k = 0; k < k_n; k += 2) {
                if (lap >= 1 && !mbar_wait(&bars->x_empty[sx], (lap & 1u) ^ 1u, abort_flag, ws, 0xA110)) break;
                uint8_t *st = smem + p.off_x + (size_t)sx * 2 * p.x_bytes;
                const int n = min(2, k_n - k);
                mbar_arrive_expect_tx(&bars->x_full[sx], n * p.x_bytes);
                for (int h = 0; h < n; ++h) tma_load_2d(st + h * p.x_bytes, &tmap_x, &bars->x_full[sx], (4 * s_lo + k + h) * 64, mt * p.N);
                if (++sx == (uint32_t)p.SX) { sx = 0; ++lap; }
            }
        }
        __syncwarp();
    } else if (kIn == kQuantize) {
        // ---- quantising: a warp takes 256 columns of a row, eight a lane, and writes them as the TMA would (16-byte pieces XOR-ed with the
        // row number) and their scales as they lie in a blob; rows past the last are left as they are (their sums are nobody's) -----------
        const uint16_t *x = reinterpret_cast<const uint16_t *>(xin);
        const int rows = min(p.N, p.M - mt * p.N);
        const bool whole = p.I % 8 == 0;
        uint32_t s = 0, lap = 0;
        for (int i = 0; i < s_n; ++i) {
            if (lap >= 1 && !__all_sync(0xFFFFFFFFu, mbar_wait(&bars->empty[s], (lap & 1u) ^ 1u, abort_flag, ws, 0xA120))) break;
            uint8_t *st = smem + (size_t)s * p.stage_bytes;
            const int c = (s_lo + i) * kStepCols + lane * 8;
            for (int r = warp - 2; r < rows; r += kEpiWarps) {
                uint32_t v[4];
                const uint16_t *from = x + (int64_t)(mt * p.N + r) * p.I + c;
                const int n = max(0, min(p.I - c, 8));
                if (whole) mx_load_whole(v, from, n > 0);
                else {
                    MxRaw<4> raw;
                    mx_load_raw(raw, from, n, x + (int64_t)p.M * p.I);
                    mx_align(v, raw, from, n);
                }
                uint32_t top = mx_top8(v);
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const uint32_t code = mx_code(top);
                float f[8];
                mx_scaled8(f, v, code);
                const uint32_t word = mx_cvt_e2m1x8(f);
                *reinterpret_cast<uint32_t *>(st + kWBytes + 2 * kScaleBytes + r * 128 + (((lane >> 2) ^ (r & 7)) * 16) + (lane & 3) * 4) = code == 255 ? 0u : word;
                if ((lane & 3) == 0) st[kWBytes + kScaleBytes + (lane >> 4) * kMxScaleTile + mx_scale_at((uint32_t)r, (uint32_t)lane >> 2)] = (uint8_t)code;
            }
            fence_proxy_async_smem();                          // the tensor core reads what this thread wrote
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->full[s]);
            if (++s == (uint32_t)p.S) { s = 0; ++lap; }
        }
    } else if (kIn == kWide) {
        // ---- widening: a group of four warps takes every fourth slot (128 columns, two K steps), a thread one row of the weights ------------
        const int group = (warp - 2) >> 2, quarter = warp & 3, r = quarter * 32 + lane, t = group & 1;       // t: which slot of a stage
        bool ok = true;
        uint32_t s = 0, ph = 0;
        for (int i = 0; i < s_n && ok; ++i) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->full[s], ph, abort_flag, ws, 0xA400));
            if (!ok) break;
            const uint8_t *st = smem + (size_t)s * p.stage_bytes;
            const int u = 2 * i + t, n = (i & 1) == (group >> 1) ? min(2, k_n - 2 * u) : 0;    // this group's slot of the stage, K steps in it
            if (n > 0) {
                const uint32_t lap = (uint32_t)u / (uint32_t)p.slots, slot = (uint32_t)u - lap * (uint32_t)p.slots;
                const uint32_t codes = *reinterpret_cast<const uint32_t *>(st + kWBytes + t * kMxScaleTile + lane * 16 + quarter * 4);
                const uint32_t to = tmem_base + ((uint32_t)(quarter * 32) << 16) + p.tmem_scales + slot * kSlotCols;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h >= n) break;
                    const int q = 2 * t + h;
                    const uint4 a = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q) ^ (r & 7)) * 16);
                    const uint4 b = *reinterpret_cast<const uint4 *>(st + r * 128 + ((2 * q + 1) ^ (r & 7)) * 16);
                    uint32_t v[32];
                    mx_widen(v, a, b, codes >> (16 * h) & 255u, codes >> (16 * h + 8) & 255u);
                    if (h == 0) {
                        if (lap) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&bars->slot_empty[slot], (lap & 1u) ^ 1u, abort_flag, ws, 0xA410));
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
            if (++s == (uint32_t)p.S) { s = 0; ph ^= 1u; }
        }
    }

    const int rows = min(p.N, p.M - mt * p.N);                 // rows of X in this tile (with a 4-bit input several tiles are of 128)
    if (p.KS > 1) cluster_wait();      // every CTA of the cluster is running
    if (warp >= 2 && warp < kXWarp && s_n > 0) {
        constexpr int kStride = 16 * (kEpiWarps / 4);
        const int quarter = warp & 3, part = (warp - 2) >> 2, o = ot * kRows + quarter * 32 + lane;
        const bool direct = p.KS == 1;
        // Residuals of 16 rows, asked for before the sums are there and, from the second 16 on, while the ones before are written.  Loads without
        // conditions (rows past the last are the last one), converted when they are used: else each waits for the one before
        typename std::conditional<kBf16, uint16_t, float>::type ahead[16];
        auto load_ahead = [&](int c0) {
            const int n = o < p.O ? rows - c0 : 0;
            if (!direct || !res || n <= 0) return;
            const auto *from = static_cast<const std::remove_reference_t<decltype(ahead[0])> *>(res) + ((int64_t)(mt * p.N + c0) * p.O + o + z);
#pragma unroll
            for (int i = 0; i < 16; ++i) ahead[i] = __ldg(from + (int64_t)min(i, n - 1) * p.O);
        };
        load_ahead(part * 16);
        if (__all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full, 0, abort_flag, ws, 0xA500))) {
            tc_fence_after_sync();
            const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
            const float b = direct && bias && o < p.O ? __ldg(bias + o + z) : 0.f;
            for (int c0 = part * 16; c0 < rows; c0 += kStride) {
                uint32_t v[16];
                __syncwarp();
                tmem_ld_x16(t_addr + c0, v);
                if (direct) {
                    const int64_t at = (int64_t)(mt * p.N + c0) * p.O + o + z;
                    const int n = o < p.O ? rows - c0 : 0;
                    float add[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if constexpr (kBf16) add[i] = res ? bf16_bits_to_f32(ahead[i]) : 0.f;
                        else add[i] = res ? ahead[i] : 0.f;
                    }
                    load_ahead(c0 + kStride);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (i < n) store_y<kBf16>(y, at + (int64_t)i * p.O, __uint_as_float(v[i]) + b + add[i], p.relu);
                } else {
                    // four rows of X at a time to the CTA that owns them: [rank][output][its rows] floats, an output's padded by 16 bytes
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int m = c0 + i, owner = m / p.cpr;
                        if (m < rows)
                            st_cluster_v4(map_to_cta(smem_u32(smem + p.off_red), (uint32_t)owner) + (uint32_t)(rank * kRows + quarter * 32 + lane) * p.red_pitch +
                                              (uint32_t)(m - owner * p.cpr) * 4u, v[i], v[i + 1], v[i + 2], v[i + 3]);
                    }
                }
            }
        }
    }
    tc_fence_before_sync();
    if (p.KS > 1) { cluster_arrive(); cluster_wait(); }        // all partial sums are in place; no CTA touches another's memory after this
    else __syncthreads();
    tc_fence_after_sync();
    const bool gave_up = *abort_flag;
    if (gave_up) {
        // a role gave up: leave time for copies and MMAs still in flight to land before tensor memory goes back and the CTA retires
        const long long t0 = clock64();
        while (clock64() - t0 < 400000ll) { }
        __syncwarp();
    }
    if (warp == 1) tmem_dealloc(tmem_base, p.tmem_cols);
    if (gave_up) return;
    if (p.KS == 1) return;
    const int own = max(0, min(p.cpr, rows - rank * p.cpr));
    for (int i = tid; i < (own + 3) / 4 * kRows; i += kThreads) {
        const int m0 = i / kRows * 4, ol = i & (kRows - 1), o = ot * kRows + ol;
        if (o >= p.O) continue;
        const int64_t at = (int64_t)(mt * p.N + rank * p.cpr + m0) * p.O + o + z;
        float add[4], v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) add[j] = res && m0 + j < own ? load_res<kBf16>(res, at + (int64_t)j * p.O) : 0.f;
        const uint8_t *src = smem + p.off_red + (uint32_t)ol * p.red_pitch + (uint32_t)m0 * 4u;
        for (int s = 0; s < live; ++s, src += kRows * p.red_pitch) {
            const float4 u = *reinterpret_cast<const float4 *>(src);
            v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
        }
        const float b = bias ? __ldg(bias + o + z) : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (m0 + j < own) store_y<kBf16>(y, at + (int64_t)j * p.O, v[j] + b + add[j], p.relu);
    }
}

// the rest of the plan for a split into `ks`; false where shared or tensor memory does not hold it
bool shape(MxSwParams &p, bool mx, int ks, int sms)
{
    p.KS = ks;
    p.spr = (p.nS + ks - 1) / ks;
    p.cpr = ((p.N + ks - 1) / ks + 3) / 4 * 4;
    p.red_pitch = (uint32_t)p.cpr * 4u + 16u;
    const uint32_t red = ks > 1 ? (uint32_t)ks * kRows * p.red_pitch : 0u;
    const uint32_t fixed = red + (uint32_t)sizeof(MxSwBars) + 128u + 1024u;
    p.x_bytes = (uint32_t)p.N * 128u;
    p.stage_bytes = round_up(kWBytes + (mx ? 2 * kScaleBytes + p.x_bytes : kScaleBytes), 1024);
    // (two CTAs on an SM where there are more CTAs than SMs; those that widen have too many warps for that)
    const uint32_t limit = mx && (long long)p.nMT * p.nOT * ks > sms ? kSmemHalf : kSmemLimit;
    if (fixed >= limit) return false;
    const uint32_t budget = limit - fixed;
    p.SX = 0;
    if (!mx) {
        // the input's ring (of 128 columns a stage)
        p.SX = kMaxXStages;
        while (p.SX > 1 && (uint32_t)p.SX * 2 * p.x_bytes + 3 * p.stage_bytes > budget) --p.SX;
        if ((uint32_t)p.SX * 2 * p.x_bytes >= budget) return false;
    }
    p.S = (int)((budget - (uint32_t)p.SX * 2 * p.x_bytes) / p.stage_bytes);
    if (p.S > kMaxStages) p.S = kMaxStages;
    if (p.S > p.spr) p.S = p.spr;
    if (p.S < 1 || (p.S < 2 && p.spr > 1)) return false;
    p.off_x = (uint32_t)p.S * p.stage_bytes;
    p.off_red = p.off_x + (uint32_t)p.SX * 2 * p.x_bytes;
    p.off_bar = round_up(p.off_red + red, 128);
    p.smem_bytes = p.off_bar + (uint32_t)sizeof(MxSwBars) + 1024u;
    if (p.smem_bytes > kSmemLimit) return false;
    // columns of tensor memory: the sums, then scales of every stage (4-bit) or the widened weights
    p.tmem_scales = round_up((uint32_t)p.N, 32);
    p.slots = kSlots;
    const uint32_t cols = p.tmem_scales + (mx ? 16u * p.S : kSlotCols * p.slots);
    p.tmem_cols = 32;
    while (p.tmem_cols < cols) p.tmem_cols *= 2;
    return p.tmem_cols <= 512;
}

bool plan(const npas_mx_linear_desc &d, MxSwParams &p, int sms)
{
    const bool mx = d.x_dtype == NPAS_MX4 || d.quantize_x;
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
    const long long tiles = (long long)p.nMT * p.nOT;
    if (tiles > 0x7FFFFFFF / kMaxSplit) return false;
    if (d.variant) return d.variant >= 1 && d.variant <= kMaxSplit && !(d.variant & (d.variant - 1)) && shape(p, mx, d.variant, sms);
    return shape(p, mx, 1, sms);                               // (the automatic choice names a split)
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
    const bool blob = d.x_dtype == NPAS_MX4;
    CUtensorMap tmx, tmw;
    if (!mx_encode_values(&tmw, w, mx_layout(d.O, d.I), d.O, kRows)) return NPAS_ERR_CUDA;
    if (d.quantize_x) tmx = tmw;
    else if (!(blob ? mx_encode_values(&tmx, x, mx_layout(d.M, d.I), d.M, (uint32_t)p.N)
                    : mx_encode_bf16(&tmx, x, (uint64_t)d.I, (uint64_t)x_pitch, (uint64_t)d.M, (uint32_t)p.N)))
        return NPAS_ERR_CUDA;
    const auto kernel = blob ? (p.y_bf16 ? linear_mx_sw_kernel<kBlob, true> : linear_mx_sw_kernel<kBlob, false>)
                      : d.quantize_x ? (p.y_bf16 ? linear_mx_sw_kernel<kQuantize, true> : linear_mx_sw_kernel<kQuantize, false>)
                                     : (p.y_bf16 ? linear_mx_sw_kernel<kWide, true> : linear_mx_sw_kernel<kWide, false>);
    if (allow_dynamic_smem(reinterpret_cast<const void *>(kernel), (int)kSmemLimit) != NPAS_OK) return NPAS_ERR_CUDA;
    const dim3 grid((unsigned)(p.nMT * p.nOT * p.KS)), block(blob || d.quantize_x ? SwRoles<kBlob>::kThreads : SwRoles<kWide>::kThreads);
    const uint8_t *xb = static_cast<const uint8_t *>(x), *wb = static_cast<const uint8_t *>(w);
    const cudaError_t e = p.KS > 1 ? launch_pdl_cluster(Launch(), kernel, grid, block, p.KS, p.smem_bytes, st, tmx, tmw, p, xb, wb, bias, res, y, ws)
                                   : launch_pdl(Launch(), kernel, grid, block, p.smem_bytes, st, tmx, tmw, p, xb, wb, bias, res, y, ws);
    count_launch();
    return e == cudaSuccess ? launch_status() : NPAS_ERR_CUDA;
}

}  // namespace npas
