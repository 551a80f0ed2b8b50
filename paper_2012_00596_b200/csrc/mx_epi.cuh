// Epilogue of the persistent kernels on 4-bit weights (linear_mx_ps.cu, linear_mx_d2.cu): the walk over tiles, the slabs, the stores.
//
// Tensor memory lane = output, column = row of X, while a row of Y has its outputs side by side.  bf16 outputs whose rows start on 16-byte
// boundaries go through shared memory: a warp takes 32 outputs x 64 rows out of tensor memory as 8 x 8 matrices, rounds pairs of rows
// and stores them transposed (stmatrix) into a slab of 128 rows x 64 outputs, 128-byte swizzled, which leaves by TMA; residuals arrive
// in the slab by TMA before and are read the same way, requested a ring of slabs ahead.  2.3 instructions an output, 4.3 with a
// residual (with a store per output from registers 200704x64 -> 256 with residual took 110 us, 46 so).  Other outputs (fp32, odd widths) are
// written from registers: 32 consecutive outputs of a row a warp, whatever the alignment, residuals requested before the wait for the
// accumulator.
// The warps work in groups of eight: with two accumulators a group has every other tile (while one waits for tensor memory or a barrier
// the other one computes), with one accumulator of 256 columns a block of 128 rows of every tile.  A warp has one quarter of the lanes
// and 64 of a block's 128 rows.  When the accumulator is free: through slabs, a warp with one block of a tile hands it back as soon as
// the sums are in registers; one with both (a 16-bit input and 256 rows; pairs with residuals) has written the first block's slab before it takes the
// second block's sums; kBoth takes both first.  From registers it is handed back behind the tile's last store.
// A slab counts as gone when the store of the one after it has been issued, so with NS slabs NS - 1 are being filled: with two, one half of 64
// outputs after the other.
#pragma once

#include <type_traits>

#include "mx_tc.cuh"

namespace npas {
namespace tc {

constexpr int kMxMaxSlabs = 8;
constexpr uint32_t kMxSlabBytes = 128 * 128;               // 128 rows x 64 bf16 outputs

// Tiles of `o_step` outputs x N rows of X, outputs fastest; unit u of `grid` (a CTA or a pair) has tiles u, u + grid, ...
struct MxTiles {
    int M, O, N, n_ot, n_tiles, o_step, grid, step_mt, step_ot;
    int acc, NS, ns_log, relu;                             // accumulators; NS = 2^ns_log slabs (0: outputs from registers)
    uint32_t off_slabs;
};

// (the coordinates are carried along: two divisions a tile take longer than some roles' work on it)
struct MxWalk {
    int tile, mt, ot, rank;
    __device__ __forceinline__ MxWalk(const MxTiles &p, int unit, int r) : tile(unit), mt(unit / p.n_ot), ot(unit - mt * p.n_ot), rank(r) {}
    __device__ __forceinline__ bool in(const MxTiles &p) const { return tile < p.n_tiles; }
    __device__ __forceinline__ void next(const MxTiles &p)
    {
        tile += p.grid; mt += p.step_mt; ot += p.step_ot;
        if (ot >= p.n_ot) { ot -= p.n_ot; ++mt; }
    }
    __device__ __forceinline__ int m0(const MxTiles &p) const { return mt * p.N; }
    __device__ __forceinline__ int o0(const MxTiles &p) const { return ot * p.o_step + rank * 128; }
    // blocks of 128 rows and halves of 64 outputs of this CTA that exist
    __device__ __forceinline__ int blocks(const MxTiles &p) const { return min(p.N >> 7, (p.M - m0(p) + 127) >> 7); }
    __device__ __forceinline__ int halves(const MxTiles &p) const { const int o = o0(p); return (o < p.O ? 1 : 0) + (o + 64 < p.O ? 1 : 0); }
};

struct MxEpiBars {
    uint64_t acc_full[2], acc_empty[2];
    uint64_t landed[kMxMaxSlabs], slab_done[kMxMaxSlabs];      // a slab's residuals have landed / its epilogue warps have finished their parts
    uint32_t freed;                                            // slabs, in their order, that have left: number n may be written when n - NS has
};

// Bounded wait for the count of slabs that have left.  (A count and not a barrier's parity: a warp has a part in some uses of a slab only, and
// could find the parity of the use before last.)
__device__ __forceinline__ bool mx_wait_freed(const MxEpiBars *bars, uint32_t n, volatile uint32_t *abort_flag, uint32_t *ws, uint32_t where)
{
    auto ready = [&]() {
        uint32_t v;
        asm volatile("ld.acquire.cta.shared::cta.u32 %0, [%1];" : "=r"(v) : "r"(smem_u32(&bars->freed)) : "memory");
        return (int32_t)(v - n) >= 0;
    };
    if (ready()) return true;
    long long t0 = 0;
    uint32_t spins = 0;
    while (!ready()) {
        __nanosleep(32);
        ++spins;
        if (spins == 256u) t0 = clock64();
        else if ((spins & 255u) == 0u) {
            if (*abort_flag) return false;
            if (clock64() - t0 > kWaitLimitCycles) {
                *abort_flag = 1;
                if (atomicCAS(ws, 0u, 10u /* NPAS_ERR_TIMEOUT */) == 0u) ws[1] = where;
                return false;
            }
        }
    }
    return true;
}
__device__ __forceinline__ void mx_set_freed(MxEpiBars *bars, uint32_t n)
{
    asm volatile("st.release.cta.shared::cta.u32 [%0], %1;" ::"r"(smem_u32(&bars->freed)), "r"(n) : "memory");
}

__device__ __forceinline__ void mx_epi_init(MxEpiBars *bars, const MxTiles &p, int releases)
{
    for (int a = 0; a < 2; ++a) { mbar_init(&bars->acc_full[a], 1); mbar_init(&bars->acc_empty[a], releases); }
    for (int n = 0; n < p.NS; ++n) { mbar_init(&bars->landed[n], 1); mbar_init(&bars->slab_done[n], 4); }
    bars->freed = 0;
}

// ---- the slabs' copies, one thread: a slab leaves by TMA as soon as every epilogue warp has finished its part; when the store before it has
// been read, that slab is free again, or takes the residuals of the slab a ring further on ------------------------------------------
struct MxSlabWalk {
    MxWalk t;
    int r, h, blocks, halves;
    __device__ MxSlabWalk(const MxTiles &p, int unit, int rank) : t(p, unit, rank), r(0), h(0) { settle(p); }
    __device__ void settle(const MxTiles &p)
    {
        while (t.in(p) && t.halves(p) == 0) t.next(p);
        blocks = t.blocks(p); halves = t.halves(p);
    }
    __device__ bool in(const MxTiles &p) const { return t.in(p); }
    __device__ void next(const MxTiles &p)
    {
        if (++h < halves) return;
        h = 0;
        if (++r < blocks) return;
        r = 0;
        t.next(p);
        settle(p);
    }
};

__device__ __forceinline__ void mx_slab_copies(const MxTiles &p, int unit, int rank, uint8_t *smem, MxEpiBars *bars, const CUtensorMap *tmap_y, const CUtensorMap *tmap_r,
                                               bool res, volatile uint32_t *abort_flag, uint32_t *ws)
{
    const uint32_t mask = (uint32_t)p.NS - 1;
    auto request = [&](const MxSlabWalk &w, uint32_t n) {
        uint64_t *bar = &bars->landed[n & mask];
        mbar_arrive_expect_tx(bar, kMxSlabBytes);
        tma_load_2d(smem + p.off_slabs + (size_t)(n & mask) * kMxSlabBytes, tmap_r, bar, w.t.o0(p) + w.h * 64, w.t.m0(p) + w.r * 128);
    };
    MxSlabWalk ahead(p, unit, rank);
    uint32_t n = 0, asked = 0;
    for (; res && asked < (uint32_t)p.NS && ahead.in(p); ++asked) { request(ahead, asked); ahead.next(p); }
    for (MxSlabWalk w(p, unit, rank); w.in(p); w.next(p), ++n) {
        if (!mbar_wait(&bars->slab_done[n & mask], (n >> p.ns_log) & 1u, abort_flag, ws, 0xC600)) break;
        tma_store_2d(tmap_y, smem + p.off_slabs + (size_t)(n & mask) * kMxSlabBytes, w.t.o0(p) + w.h * 64, w.t.m0(p) + w.r * 128);
        bulk_commit();
        if (n) {
            bulk_wait_read<1>();
            mx_set_freed(bars, n);
            if (res && ahead.in(p)) { request(ahead, asked++); ahead.next(p); }           // (slab n - 1 + NS)
        }
    }
    bulk_wait_read<0>();                                       // the slabs stay valid until the last store has read them
}

// ---- epilogue through slabs; e: number of the warp among the epilogue's, `release(acc)`: this warp has the sums in registers.  kBoth: a warp
// with both blocks of a tile of 256 rows rounds the first one's sums, takes the second one's and hands the accumulator back before it waits
// for a slab (without residuals; 32 more registers) -------------------------------------------------------------------------------
template <int kGroups, bool kBoth, typename F>
__device__ __forceinline__ void mx_epilogue_slabs(const MxTiles &p, int unit, int rank, int e, int lane, int quarter, uint32_t smem, uint32_t tmem_base, MxEpiBars *bars,
                                                  const float *bias, bool res, volatile uint32_t *abort_flag, uint32_t *ws, F release)
{
    const int group = e >> 3, part = (e >> 2) & 1, half = quarter >> 1;
    // this lane's row and 16-byte piece in the slab: row (lane % 8) of 8 x 8 matrix (lane / 8)
    const uint32_t lane_at = smem + p.off_slabs + (uint32_t)((part * 64 + (lane & 7)) * 128 + ((((quarter & 1) * 4 + (lane >> 3)) ^ (lane & 7)) * 16));
    const int step = p.acc == 1 ? kGroups : 1;
    uint32_t it = 0, n = 0;                                    // n: slabs of the tiles before
    for (MxWalk w(p, unit, rank); w.in(p); w.next(p), ++it) {
        const int halves = w.halves(p), blocks = w.blocks(p);
        const uint32_t n_tile = n;
        n += (uint32_t)(halves * blocks);
        if (p.acc == 2 && kGroups == 2 && (it & 1u) != (uint32_t)group) continue;
        const int o = w.o0(p) + quarter * 32 + (lane >> 2);
        const uint32_t acc = p.acc == 2 ? it & 1u : 0u, lap = p.acc == 2 ? it >> 1 : it;
        float b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = bias && o + 8 * i < p.O ? __ldg(bias + o + 8 * i) : 0.f;
        if (!__all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full[acc], lap & 1u, abort_flag, ws, 0xC500))) return;
        tc_fence_after_sync();
        const uint32_t t_addr = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * p.N + (uint32_t)(part * 64);
        // outputs 0 to 15 and 16 to 31 of the quarter, twice 32 rows of block r
        auto take = [&](int r, uint32_t (&u)[2][16], uint32_t (&v)[2][16]) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                tmem_ld_16x32(t_addr + r * 128 + c * 32, u[c]);
                tmem_ld_16x32(t_addr + r * 128 + c * 32 + (16u << 16), v[c]);
            }
            tmem_ld_wait();
        };
        // eight rows of Y, k of 32: + bias (+ residuals q), one rounding, then ReLU on the rounded pairs (max with +0 is exact on them)
        auto rounded = [&](const uint32_t (&u)[16], const uint32_t (&v)[16], int k, const uint32_t (&q)[4], uint32_t (&h)[4]) {
            float f[8] = {__uint_as_float(u[4 * k]) + b[0], __uint_as_float(u[4 * k + 1]) + b[0], __uint_as_float(u[4 * k + 2]) + b[1],
                          __uint_as_float(u[4 * k + 3]) + b[1], __uint_as_float(v[4 * k]) + b[2], __uint_as_float(v[4 * k + 1]) + b[2],
                          __uint_as_float(v[4 * k + 2]) + b[3], __uint_as_float(v[4 * k + 3]) + b[3]};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (res) {
                    f[2 * i] += __uint_as_float(q[i] << 16);
                    f[2 * i + 1] += __uint_as_float(q[i] & 0xFFFF0000u);
                }
                h[i] = cvt_bf16x2(f[2 * i], f[2 * i + 1]);
                if (p.relu) h[i] = relu_bf16x2(h[i]);
            }
        };
        // the slab of block r: what last lay in it has left, and with residuals, they have landed
        auto slab_of = [&](int r, uint32_t &slot) {
            const uint32_t at = n_tile + (uint32_t)(r * halves + half);
            slot = at & (p.NS - 1);
            return __all_sync(0xFFFFFFFFu, (at < (uint32_t)p.NS || mx_wait_freed(bars, at - p.NS + 1, abort_flag, ws, 0xC510)) &&
                                               (!res || mbar_wait(&bars->landed[slot], (at >> p.ns_log) & 1u, abort_flag, ws, 0xC511)));
        };
        auto hand_over = [&](uint32_t slot) {
            fence_proxy_async_smem();                          // the TMA store reads what this thread wrote
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->slab_done[slot]);
        };
        constexpr uint32_t kNone[4] = {0, 0, 0, 0};
        uint32_t slot;
        if (kBoth && !res && blocks == 2 && half < halves) {
            uint32_t h[8][4];
            {
                uint32_t u[2][16], v[2][16];
                take(0, u, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) rounded(u[k >> 2], v[k >> 2], k & 3, kNone, h[k]);
            }
            uint32_t u[2][16], v[2][16];
            take(1, u, v);
            release(acc);
            if (!slab_of(0, slot)) return;
#pragma unroll
            for (int k = 0; k < 8; ++k) stmatrix_x4_trans(lane_at + slot * kMxSlabBytes + (uint32_t)k * 1024u, h[k][0], h[k][1], h[k][2], h[k][3]);
            hand_over(slot);
            if (!slab_of(1, slot)) return;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                rounded(u[k >> 2], v[k >> 2], k & 3, kNone, h[0]);
                stmatrix_x4_trans(lane_at + slot * kMxSlabBytes + (uint32_t)k * 1024u, h[0][0], h[0][1], h[0][2], h[0][3]);
            }
            hand_over(slot);
            continue;
        }
        bool held = true;
        for (int r = p.acc == 1 && kGroups == 2 ? group : 0; r < blocks && half < halves; r += step) {
            uint32_t u[2][16], v[2][16];
            take(r, u, v);
            if (r + step >= blocks) { release(acc); held = false; }
            if (!slab_of(r, slot)) return;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t sa = lane_at + slot * kMxSlabBytes + (uint32_t)k * 1024u;
                uint32_t q[4] = {0, 0, 0, 0}, h[4];
                if (res) ldmatrix_x4_trans(sa, q);
                rounded(u[k >> 2], v[k >> 2], k & 3, q, h);
                if (res) __syncwarp();                         // (every lane has read these rows' residuals)
                stmatrix_x4_trans(sa, h[0], h[1], h[2], h[3]);
            }
            hand_over(slot);
        }
        if (held) release(acc);                                // (nothing of this tile is this warp's)
    }
}

// ---- epilogue from registers: a lane writes one output of 64 rows of a block -----------------------------------------------------
// 32 rows of one output: bias + residuals, then sums + those, ReLU, one rounding.  `at`: element of the first row; `n`: rows there are
// (none where the output lies past the end).  The pointer walks from row to row: 32 addresses at once would not fit beside the sums.
// The loads of 32 whole rows have no conditions between them and are converted behind the last one (with a condition and a conversion at
// each 200704x64 -> 250 with residual took 87 us, 68 so, with a 16-bit input 143 and 82).
template <bool kBf16>
__device__ __forceinline__ void mx_load_residuals(float (&add)[32], float b, const void *res, int64_t at, int64_t O, int n)
{
    using T = typename std::conditional<kBf16, uint16_t, float>::type;
    const T *q = static_cast<const T *>(res) + at;
    T raw[32];
    if (n >= 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            raw[i] = __ldg(q);
            q += O;
            asm volatile("" : "+l"(q));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            raw[i] = 0;
            if (i < n) raw[i] = __ldg(q);
            q += O;
            asm volatile("" : "+l"(q));
        }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        if constexpr (kBf16) {
            asm volatile("" : "+h"(raw[i]));
            add[i] = b + __uint_as_float((uint32_t)raw[i] << 16);
        } else {
            add[i] = b + raw[i];
        }
    }
}
template <bool kBf16>
__device__ __forceinline__ void mx_store_rows(const uint32_t (&v)[32], const float (&add)[32], void *y, int64_t at, int64_t O, int n, int relu)
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
__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

template <int kGroups, bool kBf16, typename F>
__device__ __forceinline__ void mx_epilogue_rows(const MxTiles &p, int unit, int rank, int e, int lane, int quarter, uint32_t tmem_base, MxEpiBars *bars, const float *bias,
                                                 const void *res, void *y, volatile uint32_t *abort_flag, uint32_t *ws, F release)
{
    const int group = e >> 3, part = (e >> 2) & 1, step = p.acc == 1 ? kGroups : 1;
    uint32_t it = 0;
    for (MxWalk w(p, unit, rank); w.in(p); w.next(p), ++it) {
        if (p.acc == 2 && kGroups == 2 && (it & 1u) != (uint32_t)group) continue;
        const int o = w.o0(p) + quarter * 32 + lane, blocks = w.blocks(p);
        const uint32_t acc = p.acc == 2 ? it & 1u : 0u, lap = p.acc == 2 ? it >> 1 : it;
        const float b = bias && o < p.O ? __ldg(bias + o) : 0.f;
        if (res) {
            // the residuals of this warp's next tile on their way to L2 (fetched when they are needed they held the tile up twice)
            MxWalk next = w;
            next.next(p);
            if (p.acc == 2 && kGroups == 2) next.next(p);
            const int no = next.o0(p) + quarter * 32;
            if (next.in(p) && no < p.O)
                for (int r = p.acc == 1 && kGroups == 2 ? group : 0; r < next.blocks(p); r += step)
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        const int m = next.m0(p) + r * 128 + part * 64 + c + lane;
                        if (m >= p.M) continue;
                        constexpr int kSize = kBf16 ? 2 : 4;
                        const char *q = static_cast<const char *>(res) + ((int64_t)m * p.O + no) * kSize, *last = q + (min(32, p.O - no) * kSize - 1);
#pragma unroll
                        for (int i = 0; i < 32 * kSize; i += 32) prefetch_l2(q + i < last ? q + i : last);
                        prefetch_l2(last);
                    }
        }
        bool waited = false;
        for (int r = p.acc == 1 && kGroups == 2 ? group : 0; r < blocks; r += step)
            for (int c = 0; c < 64; c += 32) {
                const int m = w.m0(p) + r * 128 + part * 64 + c, n = o < p.O ? p.M - m : 0;       // rows from m on (may be none)
                const int64_t at = (int64_t)m * p.O + o;
                float add[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) add[i] = b;
                if (res) mx_load_residuals<kBf16>(add, b, res, at, p.O, n);
                if (!waited) {
                    if (!__all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full[acc], lap & 1u, abort_flag, ws, 0xC520))) return;
                    tc_fence_after_sync();
                    waited = true;
                }
                uint32_t v[32];
                tmem_ld_x32(tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * p.N + (uint32_t)(r * 128 + part * 64 + c), v);
                tmem_ld_wait();
                mx_store_rows<kBf16>(v, add, y, at, p.O, n, p.relu);
            }
        if (!waited) {                                         // (no block of this tile is the group's: it hands the accumulator on all the same)
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(&bars->acc_full[acc], lap & 1u, abort_flag, ws, 0xC530))) return;
            tc_fence_after_sync();
        }
        release(acc);
    }
}

// ---- host ---------------------------------------------------------------------------------------
inline void mx_tiles_plan(MxTiles &t, const npas_mx_linear_desc &d, int N, int o_step, int acc, int units)
{
    t.M = d.M; t.O = d.O; t.N = N; t.o_step = o_step; t.acc = acc; t.relu = d.relu;
    t.n_ot = (d.O + o_step - 1) / o_step;
    const long long tiles = (long long)t.n_ot * ((d.M + N - 1) / N);
    t.n_tiles = tiles > 0x3FFFFFFF ? 0 : (int)tiles;           // (0: too many)
    t.grid = t.n_tiles < units ? t.n_tiles : units;
    if (t.grid) { t.step_mt = t.grid / t.n_ot; t.step_ot = t.grid % t.n_ot; }
}

}  // namespace tc
}  // namespace npas
