// Softmax cross entropy of H W^T over a large vocabulary and its gradients, the logits never stored:
//   l = H W^T,  lse_t = log sum_v exp l_tv,  loss_t = lse_t - l_{t,y_t},
//   dl_tv = g_t (exp(l_tv - lse_t) - [v = y_t]),   dH = dl W,   dW = dl^T H.
// All four products run on one tensor-core kernel (TMA + tcgen05 kind::f16, binary32 accumulators in TMEM); they differ
// in which dimension of each stored matrix is contiguous and in what the epilogue does with a finished tile:
//   STATS   l = H W^T       both K-major       per row and tile: maximum and sum of exponentials (one pass, running
//                                              maximum), and the label's logit; joined per row by a small kernel
//   DLOGIT  l again         both K-major       dl of one piece of the vocabulary, rounded to 16 bits: T x Vp
//   DW      dW = dl^T H     both MN-major      rows of this piece, final
//   DH      dH += dl W      K-major, MN-major  summed over the pieces in a binary32 buffer, in their order
// The backward pass recomputes the logits of a piece (2 T Vp D operations) rather than keep them: what is kept between the
// two passes is lse, one float per row.  A piece's dl has 64 MB at most, and so stays in L2 between the product that writes it and
// the two that read it, up to 16384 rows; a piece has 2048 words at least, so that with more rows dl grows, 4096 bytes a row, and goes
// through HBM.
//
// The label's entry of dl is -g_t sum_{v != y_t} exp(l_tv - lse_t) where g_t (exp(l_ty - lse_t) - 1) would cancel: lse is a
// binary32 number of the logits' size, so the difference from 1 is only good to 2^-24 |lse| (a loss of 1e-4 among logits of
// 25: 0.5 % off, of 300: 10 %).  With one piece, DLOGIT adds up the other probabilities of its columns and loss_label_kernel puts
// the entry into dl before it is read (2 to 6 us: 16 x 3027 x 1958 40.7 -> 43.2, 777 x 32003 x 1000 222 -> 226, 79 x 61013 x 182 69 ->
// 74).  With several, dl of the first piece is consumed before the last is known: the rows whose label has a probability close to
// 1 (loss_confident_kernel) are put together, and their other words' sums taken by STATS before the first piece (where there is
// no such row 6 to 17 us, 1024 x 100000 x 64 214 -> 227; the backward pass of 4096 x 32000 x 1024 602 us: 608 without, 627 with 40, 660
// with 1023, 780 with all 4096); the other rows' entries are good to 2^-10 as the difference.
//
// Tiles: 256 x 256 per CTA pair (cta_group::2), 64 reduced entries (128 bytes) per stage, six stages; two accumulators
// in TMEM let the epilogue of a tile run beside the products of the next.  Where pairs would leave half of the device idle
// (few rows, a small vocabulary) the statistics take 128-row tiles of one CTA, narrower ones if need be.  The backward pass
// mixes the products that read one piece's dl with the product that writes the next one's in one launch, whose units are
// spread over the pairs by their lengths: one ragged end per piece instead of three (4096 x 50176 x 2048, forward and backward: 2.85 ->
// 2.28 ms together with a stage loop of its own for each kind of operands; 2.6 to 2.7 under the power cap).
// What bounds it: the tensor cores, 520 cycles a stage of 512 forward (92.5 % of their cycles, 1.66 PFLOP/s) and 608 backward
// (86 %); below about 400 reduced entries the exponentials of the epilogue, 3300 cycles a tile (a special-function unit
// takes eight per instruction and scheduler: 2112).  Rows that do not start on 128 bytes cost 725 cycles a stage.
// Every wait is bounded.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_softmax.cuh"
#include "cdl_tc.cuh"
#include "cdl_wait.cuh"

namespace cdl {
namespace {

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

enum LossMode { STATS = 0, DLOGIT = 1, DW = 2, DH = 3 };

constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kBK = 64;                                // reduced entries of a stage (128 bytes)
constexpr int kBlockBytes = 128 * 128;                 // operand block of 128 rows
constexpr int kOutWarpBytes = 32 * 128;
constexpr int kStagesMax = 6;
constexpr int kSmemBytes = 1024 + kStagesMax * 2 * kBlockBytes + kEpiWarps * kOutWarpBytes;
constexpr unsigned long long kWaitNs = 2000000000ull;
// An epilogue's wait is for all stages of a tile, which take up to 0.6 us each (rows that do not start on 128 bytes, under the power
// cap): 2^24 of them, a reduced dimension of 2^30, are five to ten seconds of valid work.
constexpr unsigned long long kWaitStageNs = 2000ull;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr size_t kStatusBytes = 256;

constexpr int kMaxSlots = 160;                         // CTAs, or pairs of them, of a backward launch (148 or 74 on a B200)

// One product of a launch: output I x J, reduced over R, cut into `splits` parts of the reduced dimension.
struct LossJob {
    int mode;
    int I, J, R;
    int tn;                         // columns of a tile: 256, or fewer where there are few tiles (STATS, DLOGIT)
    int tiles_i, tiles_j, splits;
    // Backward: its units (tile, split) on the launch's slots: slot s takes units i * slots + s for i < rounds, then extra[s] .. extra[s + 1] - 1.
    int rounds;
    int extra[kMaxSlots + 1];
};
struct LossMaps {
    CUtensorMap a[3], b[3], o[3];
};

struct LossParams {
    LossJob job[3];
    int jobs, slots;
    const long long *labels;        // STATS, DLOGIT
    int V;                          // words of the vocabulary
    int v0;                         // DLOGIT: first word of the piece
    float2 *part;                   // STATS: (maximum in units of log 2, sum of exponentials relative to it) per row and half tile
    int parts;                      // ... entries per row
    float *target;                  // STATS: the label's logit
    // STATS of the backward pass: the number of rows, on the device, and the label's own logit left out
    const int *count;
    int others_only;
    const float *lse, *dloss;       // DLOGIT
    float *others;                  // DLOGIT, nullable: per row and half tile, the sum of exponentials without the label's
    int others_ld;
    const float *entry;             // DLOGIT, nullable: per row, the label's entry over dloss where it is 0 or less
    const float *scale;             // backward: {S, 1/S}, what dl is stored with
    int first, last;                // DH: first / last piece (last: the output itself is written, unless the job is split)
    float *acc;                     // DH: binary32 sums of the pieces so far, row pitch acc_ld, acc_rows rows per split
    long long acc_ld;
    int acc_rows;
    void *out_w, *out_h;            // DW, DH: outputs, row pitches
    long long ldw, ldh;
    int out_cols;                   // ... of which TMA stores these columns, the threads the few behind them
    int *status;
};

// The units of a slot, in order.
struct LossWalk {
    int j, i;
};
struct LossUnit {
    int j, ti, tj, split, rb0, rb1;     // j < 0: no more
};
template <bool GRAD>
__device__ __forceinline__ LossUnit next_unit(LossWalk &w, const LossParams &P, int slot, int stats_tiles_i)
{
    LossUnit u;
    u.j = -1;
    if constexpr (!GRAD) {                                      // one job of whole tiles, taken in turn
        const LossJob &J = P.job[0];
        const int n = w.i * P.slots + slot;
        if (n >= stats_tiles_i * J.tiles_j) return u;
        ++w.i;
        u.j = 0;
        u.split = 0;
        tile_at(n, stats_tiles_i, J.tiles_j, u.ti, u.tj);
        u.rb0 = 0;
        u.rb1 = (J.R + kBK - 1) / kBK;
        return u;
    } else {
        while (w.j < P.jobs) {
            const LossJob &J = P.job[w.j];
            int n = w.i * P.slots + slot;
            if (w.i >= J.rounds) n = J.extra[slot] + (w.i - J.rounds);
            if (w.i < J.rounds || n < J.extra[slot + 1]) {
                ++w.i;
                u.j = w.j;
                const int t = J.splits == 1 ? n : n / J.splits;
                u.split = n - t * J.splits;
                tile_at(t, J.tiles_i, J.tiles_j, u.ti, u.tj);
                const int rblocks = (J.R + kBK - 1) / kBK;
                u.rb0 = J.splits == 1 ? 0 : (int)((long long)rblocks * u.split / J.splits);
                u.rb1 = J.splits == 1 ? rblocks : (int)((long long)rblocks * (u.split + 1) / J.splits);
                return u;
            }
            ++w.j;
            w.i = 0;
        }
        return u;
    }
}

// GRAD: a launch of the backward pass (jobs DLOGIT, DW and DH in any mixture); otherwise STATS alone.
template <bool PAIR, bool GRAD, typename T>
__global__ void __launch_bounds__(kThreads, 1)
loss_gemm_kernel(const __grid_constant__ LossMaps maps, const __grid_constant__ LossParams P)
{
    extern __shared__ unsigned char smem_dyn[];
    __shared__ __align__(8) unsigned long long bars[2 * kStagesMax + 4];
    __shared__ uint32_t tmem_base_s, asked_s;
    __shared__ int abort_s;

    constexpr int kBRows = PAIR ? 128 : 256;           // most columns of a tile that this CTA stages
    constexpr uint32_t kStageBytes = (uint32_t)kBlockBytes + (uint32_t)kBRows * 128u;
    constexpr int kStages = PAIR ? 6 : 4;
    static_assert(kStages * kStageBytes <= kStagesMax * 2 * kBlockBytes, "shared memory");
    const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &abort_s;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const int slot = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;

    if (!GRAD && P.count != nullptr) {                 // mostly there is no such row
        follow_previous();
        if (*P.count == 0) return;
    }
    const uint32_t bar0 = smem_u32(&bars[0]);
    constexpr uint32_t kEmptyOff = 8u * kStagesMax;
    const uint32_t tfull0 = bar0 + 16u * kStagesMax, tempty0 = tfull0 + 16u;
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar0 + 8u * s, 1);
            mbar_init(bar0 + kEmptyOff + 8u * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull0 + 8u * b, 1);
            mbar_init(tempty0 + 8u * b, PAIR ? 2 * kEpiWarps : kEpiWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_all<PAIR>(smem_u32(&tmem_base_s));
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_s;
    follow_previous();
    bool failed = false;
    const int stats_rows = GRAD ? 0 : (P.count != nullptr ? *P.count : P.job[0].I);
    const int stats_tiles_i = GRAD ? 0 : (stats_rows + (PAIR ? 255 : 127)) / (PAIR ? 256 : 128);

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (one lane)
        if (lane == 0) {
            uint32_t st = 0u, par = 1u, asked = 0u;
            auto load = [&](uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t fb) {
                if (PAIR) tma_load_2d_pair(dst, map, c0, c1, fb);
                else tma_load_2d(dst, map, c0, c1, fb);
            };
            // The stages of a unit, one loop per kind of operands (the stage loop tests nothing but its barrier: with the
            // kind looked up in every stage, 612 cycles a stage became 770).  K-major: one box of 64 reduced entries x the
            // block's rows.  MN-major: boxes of 64 rows x 64 reduced entries, the stored matrix's rows being the reduced
            // dimension.
            // With one CTA per tile (few rows of H: bound by reading W) each tile begins at another place of the reduced
            // dimension: a row pitch that is a power of two would have all CTAs read the same few memory channels at a time.
            auto stages_of = [&](auto a_mn, auto b_mn, const CUtensorMap *map_a, const CUtensorMap *map_b, int arow, int brow, uint32_t bytes,
                                 int r0, int r1) {
                const int count = (r1 - r0) / kBK;
                int r = PAIR || count == 0 ? r0 : r0 + brow / 64 * 5 % count * kBK;
                for (int left = count; left > 0; --left) {
                    const uint32_t fb = bar0 + 8u * st;
                    if (!mbar_try_wait_now(fb + kEmptyOff, par) && !mbar_wait(fb + kEmptyOff, par, abort_flag, kWaitNs)) {
                        failed = true;
                        return;
                    }
                    const uint32_t sa = smem_base + st * kStageBytes, sb = sa + kBlockBytes;
                    if (!PAIR || rank == 0) mbar_expect_tx(fb, bytes);
                    if (decltype(a_mn)::value) {
                        load(sa, map_a, arow, r, fb);
                        load(sa + 8192u, map_a, arow + 64, r, fb);
                    } else load(sa, map_a, r, arow, fb);
                    if (decltype(b_mn)::value) {
#pragma unroll
                        for (int b = 0; b < kBRows / 64; ++b) load(sb + (uint32_t)b * 8192u, map_b, brow + b * 64, r, fb);
                    } else load(sb, map_b, r, brow, fb);
                    ++asked;
                    r += kBK;
                    if (!PAIR && r == r1) r = r0;
                    if (++st == (uint32_t)kStages) {
                        st = 0u;
                        par ^= 1u;
                    }
                }
            };
            LossWalk walk{0, 0};
            while (!failed) {
                const LossUnit u = next_unit<GRAD>(walk, P, slot, stats_tiles_i);
                if (u.j < 0) break;
                const int mode = GRAD ? P.job[u.j].mode : STATS;
                const CUtensorMap *map_a = &maps.a[u.j], *map_b = &maps.b[u.j];
                const int arow = u.ti * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0);
                const int brows = PAIR ? P.job[u.j].tn / 2 : P.job[u.j].tn, brow = u.tj * P.job[u.j].tn + (PAIR ? (int)rank * brows : 0);
                const uint32_t bytes = (PAIR ? 2u : 1u) * ((uint32_t)kBlockBytes + (uint32_t)brows * 128u);      // of a stage, of both CTAs of a pair
                if (GRAD && mode == DW) stages_of(Yes(), Yes(), map_a, map_b, arow, brow, bytes, u.rb0 * kBK, u.rb1 * kBK);
                else if (GRAD && mode == DH) stages_of(No(), Yes(), map_a, map_b, arow, brow, bytes, u.rb0 * kBK, u.rb1 * kBK);
                else stages_of(No(), No(), map_a, map_b, arow, brow, bytes, u.rb0 * kBK, u.rb1 * kBK);
            }
            asked_s = asked;
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (one lane; CTA 0 of a pair)
        if (lane == 0 && (!PAIR || rank == 0)) {
            // K-major: 128-byte rows, groups of eight 1024 bytes apart, 32 bytes per MMA.  MN-major: one reduced entry per
            // 128-byte line, eight lines 1024 bytes apart, 64-row blocks 8192 bytes apart, 16 lines per MMA.
            const uint64_t k_d = make_desc(smem_base, 16, 1024), mn_d = make_desc(smem_base, 8192, 1024);
            const uint32_t d_hi = (uint32_t)(k_d >> 32), k_lo = (uint32_t)k_d, mn_lo = (uint32_t)mn_d;      // (the upper words agree)
            constexpr uint32_t kFmt = __is_same(T, __nv_bfloat16) ? 1u : 0u;
            const uint32_t idesc0 = (1u << 4) | (kFmt << 7) | (kFmt << 10) | ((uint32_t)((PAIR ? 256 : 128) >> 4) << 24);
            uint32_t st = 0u, par = 0u, buf = 0u, tpar = 1u;
            auto stages_of = [&](auto a_mn, auto b_mn, int tn, int count) {
                constexpr bool kA = decltype(a_mn)::value, kB = decltype(b_mn)::value;
                const uint32_t a_lo0 = kA ? mn_lo : k_lo, b_lo0 = (kB ? mn_lo : k_lo) + (uint32_t)(kBlockBytes >> 4);
                const uint32_t idesc = idesc0 | ((kA ? 1u : 0u) << 15) | ((kB ? 1u : 0u) << 16) | ((uint32_t)(tn >> 3) << 17);
                uint32_t accumulate = 0u;
                for (int i = 0; i < count; ++i) {
                    const uint32_t fb = bar0 + 8u * st;
                    if (!mbar_try_wait_now(fb, par) && !mbar_wait(fb, par, abort_flag, kWaitNs)) {
                        failed = true;
                        return;
                    }
                    tc_fence_after();
                    const uint32_t off = st * (kStageBytes >> 4);
                    tc_mma4<PAIR, KIND_F16>(tmem_base + buf * 256u, a_lo0 + off, d_hi, kA ? 2048u >> 4 : 2u, b_lo0 + off, d_hi, kB ? 2048u >> 4 : 2u, idesc,
                                            accumulate);
                    accumulate = 1u;
                    if (PAIR) tc_commit_pair(fb + kEmptyOff);
                    else tc_commit(fb + kEmptyOff);
                    if (++st == (uint32_t)kStages) {
                        st = 0u;
                        par ^= 1u;
                    }
                }
            };
            LossWalk walk{0, 0};
            while (!failed) {
                const LossUnit u = next_unit<GRAD>(walk, P, slot, stats_tiles_i);
                if (u.j < 0) break;
                const int mode = GRAD ? P.job[u.j].mode : STATS;
                if (!mbar_try_wait_now(tempty0 + 8u * buf, tpar) && !mbar_wait(tempty0 + 8u * buf, tpar, abort_flag, kWaitNs)) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                if (GRAD && mode == DW) stages_of(Yes(), Yes(), 256, u.rb1 - u.rb0);
                else if (GRAD && mode == DH) stages_of(No(), Yes(), 256, u.rb1 - u.rb0);
                else stages_of(No(), No(), P.job[u.j].tn, u.rb1 - u.rb0);
                if (!failed) {
                    if (PAIR) tc_commit_pair(tfull0 + 8u * buf);
                    else tc_commit(tfull0 + 8u * buf);
                }
                buf ^= 1u;
                if (buf == 0u) tpar ^= 1u;
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue warps: 32 rows x half of the tile's columns each
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t wbuf = smem_base + (uint32_t)kStagesMax * 2u * kBlockBytes + (uint32_t)((warp - 2) * kOutWarpBytes);
        const float unscale = GRAD ? P.scale[1] : 1.0f;
        uint32_t buf = 0u, tpar = 0u;
        // 128 bytes of each of the warp's rows -> staging block -> TMA box at (col, row0)
        auto send = [&](const uint32_t (&w)[32], const CUtensorMap *map, bool add, int col, int row0) {
            if (lane == 0) bulk_wait_read<0>();
            __syncwarp();
            const uint32_t dst = wbuf + (uint32_t)lane * 128u;
#pragma unroll
            for (int c4 = 0; c4 < 8; ++c4)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)((c4 ^ (lane & 7)) << 4)),
                             "r"(w[4 * c4]), "r"(w[4 * c4 + 1]), "r"(w[4 * c4 + 2]), "r"(w[4 * c4 + 3])
                             : "memory");
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                if (add) tma_reduce_add_2d(map, col, row0, wbuf);
                else tma_store_2d(map, col, row0, wbuf);
                bulk_commit();
            }
        };
        LossWalk walk{0, 0};
        while (!failed) {
            const LossUnit u = next_unit<GRAD>(walk, P, slot, stats_tiles_i);
            if (u.j < 0) break;
            const int mode = GRAD ? P.job[u.j].mode : STATS;
            const int I = GRAD ? P.job[u.j].I : stats_rows, J = P.job[u.j].J;
            const CUtensorMap *map_o = &maps.o[u.j];
            const int row0 = u.ti * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0) + quarter * 32;
            const int wcols = P.job[u.j].tn / 2;         // columns of this warp
            const int col0 = u.tj * 2 * wcols + half * wcols;
            const int row = row0 + lane;
            // what the epilogue needs of its row, fetched while the products run
            int label = -1;                              // column of the row's label in this tile's matrix, or outside it
            float lse2 = 0.0f, g = 0.0f, entry = 1.0f;
            if ((!GRAD || mode == DLOGIT) && row < I) {
                const long long y = P.labels[row];
                const long long c = y - (GRAD ? P.v0 : 0);
                label = c >= 0 && y < P.V ? (int)c : -1;
                if (GRAD) {
                    // (exponentials are taken times 2^24, which dloss gives back: a probability below the smallest normal number
                    // is not flushed to 0)
                    lse2 = fmaf(P.lse[row], kLog2e, -24.0f);
                    // (a label outside the vocabulary: no gradient)
                    g = y >= 0 && y < P.V ? P.dloss[row] * P.scale[0] * 5.9604644775390625e-8f : 0.0f;
                    if (!(y >= 0 && y < P.V)) label = -2;
                    if (P.entry != nullptr) entry = P.entry[row];
                }
            }
            if (!__all_sync(0xffffffffu, mbar_try_wait_now(tfull0 + 8u * buf, tpar) ||
                                             mbar_wait(tfull0 + 8u * buf, tpar, abort_flag, kWaitNs + kWaitStageNs * (unsigned)(u.rb1 - u.rb0)))) {
                failed = true;
                break;
            }
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * 256u + (uint32_t)(half * wcols);
            const bool live = row0 < I && col0 < J;          // uniform over the warp
            if (live) {
                if (!GRAD) {
                    float m = -INFINITY, s = 0.0f, tgt = 0.0f;         // running maximum, in units of log 2
                    bool hit = false;
#pragma unroll 1
                    for (int ch = 0; ch < wcols / 32; ++ch) {
                        const int c0 = col0 + ch * 32;
                        if (c0 >= J) break;
                        uint32_t v[32];
                        tc_ld32(taddr + (uint32_t)(ch * 32), v);
                        tc_wait_ld_pin(v);
                        if (c0 + 32 > J) {
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (c0 + c >= J) v[c] = 0xff800000u;       // a column that does not exist: -infinity
                        }
                        if (__any_sync(0xffffffffu, (unsigned)(label - c0) < 32u)) {
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (label == c0 + c) {
                                    if (P.others_only) v[c] = 0xff800000u;
                                    else {
                                        tgt = __uint_as_float(v[c]);
                                        hit = true;
                                    }
                                }
                        }
                        float cm = __uint_as_float(v[0]);
#pragma unroll
                        for (int c = 1; c < 32; ++c) cm = fmaxf(cm, __uint_as_float(v[c]));
                        const float mn = fmaxf(m, cm * kLog2e);
                        const float base = mn == -INFINITY ? 0.0f : mn;     // (all logits -infinity: exponentials are 0)
                        float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
                        for (int c = 0; c < 32; c += 4) {
                            s0 += exp2_fast(fmaf(__uint_as_float(v[c]), kLog2e, -base));
                            s1 += exp2_fast(fmaf(__uint_as_float(v[c + 1]), kLog2e, -base));
                            s2 += exp2_fast(fmaf(__uint_as_float(v[c + 2]), kLog2e, -base));
                            s3 += exp2_fast(fmaf(__uint_as_float(v[c + 3]), kLog2e, -base));
                        }
                        s = s * (m == -INFINITY ? 0.0f : exp2_fast(m - base)) + ((s0 + s1) + (s2 + s3));
                        m = mn;
                    }
                    if (row < I) {
                        P.part[(long long)row * P.parts + 2 * u.tj + half] = make_float2(m, s);
                        if (hit) P.target[row] = tgt;
                    }
                } else if (mode == DLOGIT) {
                    float others = 0.0f;
#pragma unroll 1
                    for (int ch = 0; ch < wcols / 64; ++ch) {
                        const int c0 = col0 + ch * 64;
                        if (c0 >= J) break;
                        uint32_t w[32];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t v[32];
                            tc_ld32(taddr + (uint32_t)(ch * 64 + h * 32), v);
                            tc_wait_ld_pin(v);
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                v[c] = __float_as_uint(exp2_fast(fmaf(__uint_as_float(v[c]), kLog2e, -lse2)));
                            if (P.others != nullptr && c0 + 32 * h + 32 > J) {
#pragma unroll
                                for (int c = 0; c < 32; ++c)
                                    if (c0 + 32 * h + c >= J) v[c] = 0u;           // a column that does not exist
                            }
                            const bool here = __any_sync(0xffffffffu, (unsigned)(label - (c0 + 32 * h)) < 32u);
                            float own = 0.0f;
                            if (here) {
#pragma unroll
                                for (int c = 0; c < 32; ++c)
                                    if (label == c0 + 32 * h + c) {
                                        own = __uint_as_float(v[c]);
                                        v[c] = 0u;
                                    }
                            }
                            if (P.others != nullptr) {
                                float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
                                for (int c = 0; c < 32; c += 4) {
                                    s0 += __uint_as_float(v[c]);
                                    s1 += __uint_as_float(v[c + 1]);
                                    s2 += __uint_as_float(v[c + 2]);
                                    s3 += __uint_as_float(v[c + 3]);
                                }
                                others += (s0 + s1) + (s2 + s3);
                            }
                            if (here) {
                                own = entry <= 0.0f ? entry * 16777216.0f : own - 16777216.0f;
#pragma unroll
                                for (int c = 0; c < 32; ++c)
                                    if (label == c0 + 32 * h + c) v[c] = __float_as_uint(own);
                            }
#pragma unroll
                            for (int c = 0; c < 16; ++c) {
                                const float d0 = label != -2 ? __uint_as_float(v[2 * c]) * g : 0.0f;
                                const float d1 = label != -2 ? __uint_as_float(v[2 * c + 1]) * g : 0.0f;
                                w[16 * h + c] = pack2<T>(d0, d1);
                            }
                        }
                        send(w, map_o, false, c0, row0);
                    }
                    if (P.others != nullptr && row < I) P.others[(long long)row * P.others_ld + 2 * u.tj + half] = others;
                } else if (mode == DW || (P.last && P.job[u.j].splits == 1)) {
#pragma unroll 1
                    for (int ch = 0; ch < 2; ++ch) {
                        const int c0 = col0 + ch * 64;
                        if (c0 >= J) break;
                        uint32_t w[32];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t v[32];
                            tc_ld32(taddr + (uint32_t)(ch * 64 + h * 32), v);
                            tc_wait_ld_pin(v);
                            if (mode == DH && !P.first && row < I) {       // what the earlier pieces have summed
                                const float4 *q = reinterpret_cast<const float4 *>(P.acc + (long long)row * P.acc_ld + c0 + 32 * h);
#pragma unroll
                                for (int c = 0; c < 8; ++c) {
                                    const float4 a = q[c];
                                    v[4 * c] = __float_as_uint(__uint_as_float(v[4 * c]) + a.x);
                                    v[4 * c + 1] = __float_as_uint(__uint_as_float(v[4 * c + 1]) + a.y);
                                    v[4 * c + 2] = __float_as_uint(__uint_as_float(v[4 * c + 2]) + a.z);
                                    v[4 * c + 3] = __float_as_uint(__uint_as_float(v[4 * c + 3]) + a.w);
                                }
                            }
#pragma unroll
                            for (int c = 0; c < 16; ++c)
                                w[16 * h + c] = pack2<T>(__uint_as_float(v[2 * c]) * unscale, __uint_as_float(v[2 * c + 1]) * unscale);
                        }
                        if (c0 < P.out_cols) send(w, map_o, false, c0, row0);
                        if (P.out_cols < J && c0 + 64 > P.out_cols && row < I) {
                            T *o = static_cast<T *>(mode == DW ? P.out_w : P.out_h) + (long long)row * (mode == DW ? P.ldw : P.ldh) + c0;
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                if (c0 + 8 * c == P.out_cols) {
#pragma unroll
                                    for (int j = 0; j < 8; ++j)
                                        if (c0 + 8 * c + j < J) reinterpret_cast<unsigned short *>(o)[8 * c + j] = (unsigned short)(w[4 * c + (j >> 1)] >> (16 * (j & 1)));
                                }
                        }
                    }
                } else {
#pragma unroll 1
                    for (int ch = 0; ch < 4; ++ch) {
                        const int c0 = col0 + ch * 32;
                        if (c0 >= J) break;
                        uint32_t v[32];
                        tc_ld32(taddr + (uint32_t)(ch * 32), v);
                        tc_wait_ld_pin(v);
                        if (u.rb0 == u.rb1) {            // a last piece too short for all splits: nothing was multiplied
#pragma unroll
                            for (int c = 0; c < 32; ++c) v[c] = 0u;
                        }
                        send(v, map_o, !P.first, c0, u.split * P.acc_rows + row0);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_remote(tempty0 + 8u * buf, 0u);
                else mbar_arrive(tempty0 + 8u * buf);
            }
            buf ^= 1u;
            if (buf == 0u) tpar ^= 1u;
        }
        if (lane == 0) bulk_wait_all();
    }
    if (failed) {
        abort_s = 1;
        if (lane == 0) record_timeout(P.status);
    }
    tc_fence_before();
    __syncthreads();
    // after an abandoned wait: loads that are still under way land (or a limit runs out) before the CTA ends
    if (abort_s != 0 && threadIdx.x == 0 && rank == 0) drain_stages(bar0, asked_s, (uint32_t)kStages);
    __syncwarp();
    if (PAIR) cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        tmem_free_all<PAIR>(tmem_base);
    }
}

// One row per block: joins the tiles' maxima and sums, in a fixed order.
__global__ void __launch_bounds__(128)
loss_join_kernel(const float2 *part, int parts, const float *target, const long long *labels, int V, float *loss, float *lse)
{
    __shared__ float2 sh[4];
    follow_previous();
    const long long row = blockIdx.x;
    const float2 *p = part + row * parts;
    float m = -INFINITY, s = 0.0f;
    for (int i = threadIdx.x; i < parts; i += 128) join_stats(m, s, p[i].x, p[i].y);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        join_stats(m, s, m2, s2);
    }
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 1; k < 4; ++k) join_stats(m, s, sh[k].x, sh[k].y);
        const long long y = labels[row];
        lse[row] = fmaf(m, kLn2, logf(s));
        // (from the logit's distance to the maximum, in the units of the sum: the difference of two rounded numbers of the logits'
        // size would leave a small loss few right digits)
        loss[row] = y >= 0 && y < V ? kLn2 * (log2f(s) - fmaf(target[row], kLog2e, -m)) : 0.0f;
    }
}

// The scale that dl is stored with, {S, 1/S}: S = top / max |dloss| over the counted positions (1 where there is none, or none
// that is finite).  A mean has the same dloss everywhere: the label's entry, p - 1 with a small p, then is a number of few
// bits, where dloss itself would be rounded the same way in every row and the error would add up instead of averaging out
// (measured on 777 x 32003 x 1000 in binary16: 3.9e-4 of dH's norm without it).  binary16 takes top = 2^14, so that
// probabilities down to 2^-28 are normal numbers.
__global__ void __launch_bounds__(1024)
loss_scale_kernel(const float *dloss, const long long *labels, int T, int V, float top, float *out, int *count)
{
    __shared__ float sh[32];
    follow_previous();
    float m = 0.0f;
    for (int t = threadIdx.x; t < T; t += 1024) {
        const long long y = labels[t];
        if (y >= 0 && y < V) m = fmaxf(m, fabsf(dloss[t]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x < 32) {
        m = sh[threadIdx.x];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (threadIdx.x == 0) {
            // (magnitudes beyond 2^+-100 keep a scale whose reciprocal is a normal number)
            const bool use = m > 7.9e-31f && m < 1.2e30f;
            out[0] = use ? top / m : 1.0f;
            out[1] = use ? m / top : 1.0f;
            *count = 0;                              // of loss_confident_kernel
        }
    }
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The labels' entries of dl, one piece, where the label has more than half of the probability: minus the sum of the other words' entries,
// a warp per row.  (Where it has less, the difference from 1 that DLOGIT has written is the better one: probabilities are good to
// lse's 2^-24 |lse|, which the sum has in proportion to the other words' share and the difference to the label's.)
template <typename T>
__global__ void __launch_bounds__(128)
loss_label_kernel(const float *others, int parts, const long long *labels, const float *dloss, const float *scale, int rows, int V, T *dl, long long ld)
{
    follow_previous();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= rows) return;
    const long long y = labels[row];
    if (y < 0 || y >= V) return;
    const float g = dloss[row] * scale[0] * 5.9604644775390625e-8f;      // (as DLOGIT has it)
    float s = 0.0f;
    for (int i = lane; i < parts; i += 32) s += others[row * parts + i];
    s = warp_sum(s);
    if (lane == 0 && s < 8388608.0f) dl[row * ld + y] = from_f32<T>(-s * g);     // (sums are in units of 2^-24)
}

// Several pieces: the rows whose label's probability is so close to 1 that its distance, taken from lse, is not good to 2^-10: where
// the loss is below 2^-12 max(|lse|, 8).  A warp per row multiplies the label's logit out; a row that is one of them is copied
// behind the others (in any order: no result depends on a row's place).
template <typename T>
__global__ void __launch_bounds__(128)
loss_confident_kernel(const T *H, long long ldh, const T *W, long long ldw, const long long *labels, const float *lse, int rows, int V, int D,
                      float *entry, int *count, int *index, long long *label, T *copy, long long ldc)
{
    follow_previous();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= rows) return;
    if (lane == 0) entry[row] = 1.0f;
    const long long y = labels[row];
    if (y < 0 || y >= V) return;
    const T *h = H + row * ldh, *w = W + y * ldw;
    float l = 0.0f;
    for (int d = lane * 8; d < D; d += 256) {
        float a[8], b[8];
        load8(h + d, a);
        load8(w + d, b);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < D) l = fmaf(a[i], b[i], l);
    }
    l = warp_sum(l);
    const float z = lse[row];
    if (!(z - l < fmaxf(fabsf(z), 8.0f) * 2.44140625e-4f)) return;
    int at = 0;
    if (lane == 0) {
        at = atomicAdd(count, 1);
        index[at] = (int)row;
        label[at] = y;
    }
    at = __shfl_sync(0xffffffffu, at, 0);
    for (int d = lane * 8; d < D; d += 256) *reinterpret_cast<uint4 *>(copy + at * ldc + d) = *reinterpret_cast<const uint4 *>(h + d);
}

// ... and their entries, from the statistics of the other words: a warp per row, the tiles' sums joined in a fixed order.
__global__ void __launch_bounds__(128)
loss_entry_kernel(const float2 *part, int parts, const int *count, const int *index, const float *lse, float *entry)
{
    follow_previous();
    const int lane = threadIdx.x & 31, rows = *count;
    for (long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 5); i < rows; i += (long long)gridDim.x * 4) {
        const int row = index[i];
        const float z = lse[row];
        float s = 0.0f;
        for (int k = lane; k < parts; k += 32) {
            const float2 p = part[i * parts + k];
            s += p.y * exp2_fast(fmaf(-z, kLog2e, p.x));
        }
        s = warp_sum(s);
        if (lane == 0) entry[row] = -s;
    }
}

// dH from the binary32 sums of the splits, added in their order
template <typename T>
__global__ void __launch_bounds__(128)
loss_sum_kernel(const float *acc, long long acc_ld, long long split_elems, int splits, int rows, int cols, const float *scale, T *out, long long ldo)
{
    follow_previous();
    const float unscale = scale[1];
    const int per_row = (cols + 7) / 8;
    for (long long i = (long long)blockIdx.x * 128 + threadIdx.x; i < (long long)rows * per_row; i += (long long)gridDim.x * 128) {
        const long long r = i / per_row;
        const int c = (int)(i - r * per_row) * 8;
        const float *p = acc + r * acc_ld + c;
        float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        for (int s0 = 0; s0 < splits; s0 += 4) {         // four splits' loads at a time: with few rows this kernel is their latency
            float w[4][8];
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (s0 + s < splits) load8(p + (s0 + s) * split_elems, w[s]);
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (s0 + s < splits)
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] += w[s][k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= unscale;
        T *o = out + r * ldo + c;
        if (c + 8 <= cols) store8(o, v);
        else
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < cols) o[k] = from_f32<T>(v[k]);
    }
}

template <typename T>
const void *variant(bool pair, bool grad)
{
    if (grad) return pair ? reinterpret_cast<const void *>(&loss_gemm_kernel<true, true, T>) : reinterpret_cast<const void *>(&loss_gemm_kernel<false, true, T>);
    return pair ? reinterpret_cast<const void *>(&loss_gemm_kernel<true, false, T>) : reinterpret_cast<const void *>(&loss_gemm_kernel<false, false, T>);
}
const void *variant(bool pair, bool grad, int type) { return type == CDL_BF16 ? variant<__nv_bfloat16>(pair, grad) : variant<__half>(pair, grad); }

inline size_t up256(size_t n) { return (n + 255u) & ~(size_t)255u; }
inline int tiles256(long long n) { return (int)((n + 255) / 256); }

// Layout of the workspace.  The forward part (partial statistics) and the backward part share the space after the status
// block and the scale.
struct LossPlan {
    int parts;              // partial statistics per row
    bool stats_pair;        // STATS: CTA pairs on 256 rows, or single CTAs on 128
    int stats_tn, dlogit_tn;
    int pieces, Vp;         // vocabulary pieces of the backward pass and their width (a multiple of 256)
    bool grad_pair;         // backward: CTA pairs on 256 rows, or single CTAs on 128 where H has no more
    int splits;             // parts of the vocabulary piece that dH's product is cut into
    size_t off_target;      // forward
    // backward, the labels' entries.  One piece: the sums over the other words, dead before dH's sums, whose place they take.
    // Several: the entries, ahead of dl, and in dl's place, before the first piece is written, the confident rows: their
    // indexes, labels, copies and statistics.
    int others_ld, entry_parts;
    size_t off_entry, off_index, off_label, off_copy, off_part;
    long long copy_ld;
    size_t off_dl;
    size_t dl_bytes;        // dl of one piece (two of them when there are several pieces)
    size_t off_acc;         // backward: binary32 sums of dH, [splits][acc_rows][acc_ld]
    long long acc_ld;
    int acc_rows;
    size_t fwd_bytes, bwd_bytes;
};
constexpr size_t kOffScale = kStatusBytes, kOffData = kStatusBytes + 256;
constexpr long long kPieceBytes = 64ll << 20;          // dl of one piece, where that is 2048 words or more
constexpr long long kAccBytes = 64ll << 20;            // most that the splits of dH's product may add up to
constexpr int kPlanSlots = 74;                         // B200: planned for this count so that workspace sizes are fixed

LossPlan make_plan(int T, int V, int D)
{
    LossPlan p;
    // Forward: pairs where their tiles fill half of the device, otherwise single CTAs.  Narrower tiles where there are few: a
    // stage of a CTA that reads W mostly for itself takes as long as its bytes (450, 300, 250 ns for 256, 128, 64 columns;
    // 16 x 3027 x 1958: 20.9 us in 12 tiles of 256, 14.7 in 48 of 64).
    const long long ti = tiles256(T), words = tiles256(V);
    p.stats_pair = T > 128 && ti * words >= kPlanSlots / 2;
    p.stats_tn = 256;
    if (!p.stats_pair) {
        long long best = -1;
        for (int tn = 256; tn >= 64; tn /= 2) {
            const long long tiles = (((long long)T + 127) / 128) * (((long long)V + tn - 1) / tn);
            const long long ns = (tiles + 2 * kPlanSlots - 1) / (2 * kPlanSlots) * (tn == 256 ? 450 : (tn == 128 ? 300 : 250));
            if (best < 0 || ns < best) {
                best = ns;
                p.stats_tn = tn;
            }
        }
    }
    // With at most 128 rows a pair's second CTA would have nothing of dl or dH to do (16 x 3027 x 1958: 36 us of backward pass in pairs,
    // 28 in single CTAs; 64 x 5000 x 1500 40 and 32; 79 x 61013 x 182, all outputs and no reduction, 51 and 55).
    p.grad_pair = T > 128;
    const long long slots = p.grad_pair ? kPlanSlots : 2 * kPlanSlots, edge = p.grad_pair ? 256 : 128;
    const long long gi = ((long long)T + edge - 1) / edge;
    p.dlogit_tn = gi * words * 2 <= slots ? 128 : 256;
    p.parts = T <= kFewRowsLoss ? loss_rows_parts(V) : (int)(((long long)V + p.stats_tn / 2 - 1) / (p.stats_tn / 2));
    p.off_target = kOffData + up256((size_t)T * (size_t)p.parts * sizeof(float2));
    p.fwd_bytes = p.off_target + up256((size_t)T * sizeof(float));
    long long most = kPieceBytes / (512ll * (T > 0 ? T : 1));
    if (most < 8) most = 8;
    p.pieces = (int)((words + most - 1) / most);
    p.Vp = (int)((words + p.pieces - 1) / p.pieces) * 256;
    p.pieces = (int)((V + (long long)p.Vp - 1) / p.Vp);
    p.acc_ld = (long long)tiles256(D) * 256;
    p.acc_rows = tiles256(T > 0 ? T : 1) * 256;
    // dH has few tiles, each as long as the piece: cut so that a part is at most half of a slot's share of the launch
    const long long td = tiles256(D), wp = p.Vp / edge;
    const long long len_h = p.Vp / kBK, len_w = (T + kBK - 1) / kBK;
    const long long share = (gi * td * len_h + wp * td * len_w) / slots + 1;
    long long s = (2 * len_h + share - 1) / share;
    if (s > len_h / 8) s = len_h / 8;
    const long long acc_bytes = 4ll * p.acc_rows * p.acc_ld;
    if (s > kAccBytes / acc_bytes) s = kAccBytes / acc_bytes;
    if (s > 16) s = 16;
    p.splits = s > 1 ? (int)s : 1;
    p.dl_bytes = up256((size_t)T * (size_t)p.Vp * 2);
    p.others_ld = (int)(((long long)V + p.dlogit_tn / 2 - 1) / (p.dlogit_tn / 2));
    p.entry_parts = (int)(((long long)V + p.stats_tn / 2 - 1) / (p.stats_tn / 2));
    p.copy_ld = ((long long)D + 7) / 8 * 8;
    p.off_entry = kOffData;
    p.off_dl = kOffData + (p.pieces > 1 ? up256((size_t)T * sizeof(float)) : 0);
    p.off_index = p.off_dl;
    p.off_label = p.off_index + up256((size_t)T * sizeof(int));
    p.off_copy = p.off_label + up256((size_t)T * sizeof(long long));
    p.off_part = p.off_copy + up256((size_t)T * (size_t)p.copy_ld * 2);
    p.off_acc = p.off_dl + p.dl_bytes * (p.pieces > 1 ? 2 : 1);
    p.bwd_bytes = p.off_acc + (p.pieces > 1 || p.splits > 1 ? up256((size_t)p.splits * (size_t)p.acc_rows * (size_t)p.acc_ld * sizeof(float)) : 0);
    const size_t before = p.pieces > 1 ? p.off_part + up256((size_t)T * (size_t)p.entry_parts * sizeof(float2))
                                       : p.off_acc + up256((size_t)T * (size_t)p.others_ld * sizeof(float));
    if (p.bwd_bytes < before) p.bwd_bytes = before;
    return p;
}

// Spreads the units of the launch's jobs over the slots: longest units first, each job's counts chosen so that the slots'
// loads (in pipeline stages, and two for a unit's epilogue) fill to one level.
void spread_units(LossParams &P)
{
    int order[3] = {0, 1, 2};
    long long len[3], load[kMaxSlots];
    for (int j = 0; j < P.jobs; ++j) len[j] = ((P.job[j].R + kBK - 1) / kBK + P.job[j].splits - 1) / P.job[j].splits + 2;
    for (int a = 0; a < P.jobs; ++a)                     // longest first
        for (int b = a + 1; b < P.jobs; ++b)
            if (len[order[b]] > len[order[a]]) {
                const int t = order[a];
                order[a] = order[b];
                order[b] = t;
            }
    for (int s = 0; s < P.slots; ++s) load[s] = 0;
    for (int a = 0; a < P.jobs; ++a) {
        LossJob &J = P.job[order[a]];
        const long long n = (long long)J.tiles_i * J.tiles_j * J.splits, L = len[order[a]];
        long long lo = 0, hi = 0;
        for (int s = 0; s < P.slots; ++s) hi = load[s] > hi ? load[s] : hi;
        hi += (n / P.slots + 2) * L;
        auto count = [&](long long level, int s) { return level > load[s] ? (level - load[s]) / L : 0; };
        while (lo < hi) {                               // the lowest level that holds all n units
            const long long mid = (lo + hi) / 2;
            long long have = 0;
            for (int s = 0; s < P.slots; ++s) have += count(mid, s);
            if (have >= n) hi = mid;
            else lo = mid + 1;
        }
        long long c[kMaxSlots], over = -n, least;
        for (int s = 0; s < P.slots; ++s) over += c[s] = count(lo, s);
        for (int s = 0; s < P.slots && over > 0; ++s)
            if (c[s] > 0 && load[s] + c[s] * L == lo) {  // (those that reach the level exactly came in with it)
                --c[s];
                --over;
            }
        least = c[0];
        for (int s = 1; s < P.slots; ++s) least = c[s] < least ? c[s] : least;
        J.rounds = (int)least;
        J.extra[0] = (int)least * P.slots;
        for (int s = 0; s < P.slots; ++s) {
            J.extra[s + 1] = J.extra[s] + (int)(c[s] - least);
            load[s] += c[s] * L;
        }
    }
}

// Adds a product to a launch.  Operands whose rows are the reduced dimension (MN-major) are stored [R][I] / [R][J].
bool add_job(LossParams &P, LossMaps &maps, int type, bool pair, int mode, int tn, int I, int J, int R, int splits, const void *A, long long lda,
             const void *B, long long ldb)
{
    LossJob &job = P.job[P.jobs];
    job.mode = mode;
    job.I = I;
    job.J = J;
    job.R = R;
    job.tiles_i = pair ? tiles256(I) : (int)(((long long)I + 127) / 128);
    job.tn = tn;
    job.tiles_j = (int)(((long long)J + tn - 1) / tn);
    job.splits = splits;
    const CUtensorMapDataType dt = type == CDL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    const bool a_mn = mode == DW, b_mn = mode == DW || mode == DH;
    const int k = P.jobs++;
    return (a_mn ? encode_map_2d(&maps.a[k], dt, 2, A, (uint64_t)I, (uint64_t)R, (uint64_t)lda * 2, 64)
                 : encode_map_2d(&maps.a[k], dt, 2, A, (uint64_t)R, (uint64_t)I, (uint64_t)lda * 2, 128)) &&
           (b_mn ? encode_map_2d(&maps.b[k], dt, 2, B, (uint64_t)J, (uint64_t)R, (uint64_t)ldb * 2, 64)
                 : encode_map_2d(&maps.b[k], dt, 2, B, (uint64_t)R, (uint64_t)J, (uint64_t)ldb * 2, (uint32_t)(pair ? tn / 2 : tn)));
}
bool set_output(LossMaps &maps, int k, int type, const void *out, uint64_t cols, uint64_t rows, long long ld)
{
    const CUtensorMapDataType dt = type == CDL_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                                   : (type == CDL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16);
    return encode_map_2d(&maps.o[k], dt, type_bytes(type), out, cols, rows, (uint64_t)ld * (uint64_t)type_bytes(type), 32);
}

int launch_jobs(bool pair, bool grad, int type, LossMaps &maps, LossParams &P, cudaStream_t stream)
{
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    static bool attr_set[64];
    static int pair_slots[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.attrs = at + 1;
    if (!attr_set[dev]) {
        for (int v = 0; v < 8; ++v)
            if (cudaFuncSetAttribute(variant((v & 1) != 0, (v & 2) != 0, (v & 4) != 0 ? CDL_BF16 : CDL_F16), cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) {
                (void)cudaGetLastError();
                return CDL_ERR_LAUNCH;
            }
        cfg.gridDim = dim3(2u * (unsigned)(sms / 2));
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, variant(true, true, CDL_BF16), &cfg) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();
            n = sms / 2;
        }
        n = n < sms / 2 ? n : sms / 2;
        pair_slots[dev] = n < kMaxSlots ? n : kMaxSlots;
        attr_set[dev] = true;
    }
    long long units = 0;
    for (int j = 0; j < P.jobs; ++j) units += (long long)P.job[j].tiles_i * P.job[j].tiles_j * P.job[j].splits;
    if (units > 0x3fffffff) return CDL_ERR_ARG;
    const int most = pair ? pair_slots[dev] : (sms < kMaxSlots ? sms : kMaxSlots);
    P.slots = (int)(units < most ? units : most);
    if (grad) spread_units(P);
    cfg.gridDim = dim3((pair ? 2u : 1u) * (unsigned)P.slots);
    cfg.stream = stream;
    cfg.attrs = at;
    cfg.numAttrs = pair ? 2 : 1;
    void *args[2] = {&maps, &P};
    if (cudaLaunchKernelExC(&cfg, variant(pair, grad, type), args) != cudaSuccess) {
        (void)cudaGetLastError();
        return CDL_ERR_LAUNCH;
    }
    return CDL_OK;
}

int launch_join(const float2 *part, int parts, const float *target, const long long *labels, int T, int V, float *loss, float *lse, cudaStream_t stream)
{
    return launch_following(&loss_join_kernel, dim3((unsigned)T), dim3(128), 0, stream, part, parts, target, labels, V, loss, lse);
}

// Several pieces: the labels' entries of the rows that need them, before the first piece.
template <typename E>
int confident_rows(const LossPlan &p, const void *H, long long ldh, const void *W, long long ldw, const long long *labels, const float *lse, int T, int V, int D,
                   char *base, int *count, cudaStream_t st)
{
    return launch_following(&loss_confident_kernel<E>, dim3((unsigned)(((long long)T + 3) / 4)), dim3(128), 0, st, static_cast<const E *>(H), ldh,
                            static_cast<const E *>(W), ldw, labels, lse, T, V, D, reinterpret_cast<float *>(base + p.off_entry), count,
                            reinterpret_cast<int *>(base + p.off_index), reinterpret_cast<long long *>(base + p.off_label), reinterpret_cast<E *>(base + p.off_copy),
                            p.copy_ld);
}
int label_entries(const LossPlan &p, const void *H, long long ldh, const void *W, long long ldw, int type, const long long *labels, const float *lse, int T, int V,
                  int D, char *base, int *count, cudaStream_t st)
{
    int rc = type == CDL_BF16 ? confident_rows<__nv_bfloat16>(p, H, ldh, W, ldw, labels, lse, T, V, D, base, count, st)
                              : confident_rows<__half>(p, H, ldh, W, ldw, labels, lse, T, V, D, base, count, st);
    if (rc != CDL_OK) return rc;
    LossParams P;
    LossMaps maps;
    memset(&P, 0, sizeof P);
    memset(&maps, 0, sizeof maps);
    P.labels = reinterpret_cast<const long long *>(base + p.off_label);
    P.V = V;
    P.count = count;
    P.others_only = 1;
    P.part = reinterpret_cast<float2 *>(base + p.off_part);
    P.parts = p.entry_parts;
    P.status = reinterpret_cast<int *>(base);
    if (!add_job(P, maps, type, p.stats_pair, STATS, p.stats_tn, T, V, D, 1, base + p.off_copy, p.copy_ld, W, ldw)) return CDL_ERR_LAUNCH;
    if ((rc = launch_jobs(p.stats_pair, false, type, maps, P, st)) != CDL_OK) return rc;
    const int blocks = T < 4 * 148 ? (T + 3) / 4 : 148;
    return launch_following(&loss_entry_kernel, dim3((unsigned)blocks), dim3(128), 0, st, (const float2 *)P.part, P.parts, (const int *)count,
                            reinterpret_cast<const int *>(base + p.off_index), lse, reinterpret_cast<float *>(base + p.off_entry));
}

int check_common(const void *H, int64_t ldh, const void *W, int64_t ldw, int32_t type, const int64_t *labels, int32_t T, int32_t V, int32_t D)
{
    if (T < 0 || V < 1 || D < 1 || T > kMostExtent || V > kMostExtent || D > kMostExtent || (type != CDL_BF16 && type != CDL_F16)) return CDL_ERR_ARG;
    if (W == nullptr || ldw < D) return CDL_ERR_ARG;
    if (T > 0 && (H == nullptr || labels == nullptr || ldh < D)) return CDL_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(H) & 15u) || (reinterpret_cast<uintptr_t>(W) & 15u) || (ldw & 7) || (T > 0 && (ldh & 7)) ||
        (reinterpret_cast<uintptr_t>(labels) & 7u))
        return CDL_ERR_ALIGN;
    return CDL_OK;
}

}  // namespace
}  // namespace cdl

extern "C" size_t cdl_vocab_loss_workspace_bytes(int32_t T, int32_t V, int32_t D, int32_t with_gradient)
{
    using namespace cdl;
    if (T < 0 || V < 1 || D < 1 || T > kMostExtent || V > kMostExtent || D > kMostExtent) return 0;
    const LossPlan p = make_plan(T, V, D);
    return with_gradient && p.bwd_bytes > p.fwd_bytes ? p.bwd_bytes : p.fwd_bytes;
}

extern "C" int cdl_vocab_loss_fwd(const void *H, int64_t ldh, const void *W, int64_t ldw, int32_t type, const int64_t *labels,
                                  int32_t T, int32_t V, int32_t D, float *loss, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    using namespace cdl;
    int rc = check_common(H, ldh, W, ldw, type, labels, T, V, D);
    if (rc != CDL_OK) return rc;
    if (T == 0) return CDL_OK;
    if (loss == nullptr || lse == nullptr) return CDL_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(loss) & 3u) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return CDL_ERR_ALIGN;
    const LossPlan p = make_plan(T, V, D);
    if (ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < p.fwd_bytes) return CDL_ERR_WORKSPACE;
    if ((rc = check_device()) != CDL_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char *base = static_cast<char *>(ws);
    if (T <= kFewRowsLoss) {
        float2 *part = reinterpret_cast<float2 *>(base + kOffData);
        float *target = reinterpret_cast<float *>(base + p.off_target);
        const long long *y = reinterpret_cast<const long long *>(labels);
        if ((rc = launch_loss_rows(H, ldh, W, ldw, type, y, T, V, D, part, p.parts, target, static_cast<int *>(ws), st)) != CDL_OK) return rc;
        return launch_join(part, p.parts, target, y, T, V, loss, lse, st);
    }
    LossParams P;
    LossMaps maps;
    memset(&P, 0, sizeof P);
    memset(&maps, 0, sizeof maps);
    P.labels = reinterpret_cast<const long long *>(labels);
    P.V = V;
    P.part = reinterpret_cast<float2 *>(base + kOffData);
    P.parts = p.parts;
    P.target = reinterpret_cast<float *>(base + p.off_target);
    P.status = static_cast<int *>(ws);
    const bool pair = p.stats_pair;
    if (!add_job(P, maps, type, pair, STATS, p.stats_tn, T, V, D, 1, H, ldh, W, ldw)) return CDL_ERR_LAUNCH;
    if ((rc = launch_jobs(pair, false, type, maps, P, st)) != CDL_OK) return rc;
    return launch_join(P.part, p.parts, P.target, P.labels, T, V, loss, lse, st);
}

extern "C" int cdl_vocab_loss_bwd(const void *H, int64_t ldh, const void *W, int64_t ldw, int32_t type, const int64_t *labels,
                                  const float *lse, const float *dloss, int32_t T, int32_t V, int32_t D, void *dH, int64_t lddh,
                                  void *dW, int64_t lddw, void *ws, size_t ws_bytes, void *stream)
{
    using namespace cdl;
    int rc = check_common(H, ldh, W, ldw, type, labels, T, V, D);
    if (rc != CDL_OK) return rc;
    if (T > 0 && (lse == nullptr || dloss == nullptr)) return CDL_ERR_ARG;
    if ((dH != nullptr && T > 0 && lddh < D) || (dW != nullptr && lddw < D)) return CDL_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(dH) & 15u) || (reinterpret_cast<uintptr_t>(dW) & 15u) || (dH != nullptr && (lddh & 7)) ||
        (dW != nullptr && (lddw & 7)) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(dloss) & 3u))
        return CDL_ERR_ALIGN;
    const LossPlan p = make_plan(T, V, D);
    if (T > 0 && (ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < p.bwd_bytes)) return CDL_ERR_WORKSPACE;
    if ((rc = check_device()) != CDL_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        if (dW != nullptr && cudaMemset2DAsync(dW, (size_t)lddw * 2, 0, (size_t)D * 2, (size_t)V, st) != cudaSuccess) {
            (void)cudaGetLastError();
            return CDL_ERR_LAUNCH;
        }
        return CDL_OK;
    }
    if (dH == nullptr && dW == nullptr) return CDL_OK;
    char *base = static_cast<char *>(ws);
    float *scale = reinterpret_cast<float *>(base + kOffScale), *acc = reinterpret_cast<float *>(base + p.off_acc);
    const long long *y = reinterpret_cast<const long long *>(labels);
    int *count = reinterpret_cast<int *>(base + kOffScale) + 2;
    if ((rc = launch_following(&loss_scale_kernel, dim3(1), dim3(1024), 0, st, dloss, y, (int)T, (int)V, type == CDL_F16 ? 16384.0f : 1.0f, scale, count)) != CDL_OK)
        return rc;
    LossParams P;
    LossMaps maps;
    if (p.pieces > 1 && (rc = label_entries(p, H, ldh, W, ldw, type, y, lse, T, V, D, base, count, st)) != CDL_OK) return rc;
    // Launch k works on two pieces at a time: the products that read dl of piece k, and dl of piece k + 1 (into the other
    // buffer).  One launch of mixed units has one ragged end where three would have three.
    for (int k = -1; k < p.pieces; ++k) {
        memset(&P, 0, sizeof P);
        memset(&maps, 0, sizeof maps);
        P.labels = y;
        P.V = V;
        P.entry = p.pieces > 1 ? reinterpret_cast<const float *>(base + p.off_entry) : nullptr;
        P.others = p.pieces > 1 ? nullptr : acc;
        P.others_ld = p.others_ld;
        P.lse = lse;
        P.dloss = dloss;
        P.scale = scale;
        P.status = static_cast<int *>(ws);
        P.acc = acc;
        P.acc_ld = p.acc_ld;
        P.acc_rows = p.acc_rows;
        P.first = k == 0;
        P.last = k == p.pieces - 1;
        // (a TMA store fills the last 16-byte unit of a row with zeros beyond the output's columns, which are not this call's: what a
        // row has in a last, partial unit is stored by the threads.  All of it by them: 5 x 58057 x 1326
        // 221 us instead of 176.)
        P.out_cols = D / 8 * 8;
        bool ok = true;
        if (k >= 0) {
            const int v0 = k * p.Vp, words = V - v0 < p.Vp ? V - v0 : p.Vp;
            const void *dl = base + p.off_dl + (size_t)(k & 1) * p.dl_bytes;
            if (dH != nullptr) {
                const bool direct = P.last && p.splits == 1;
                P.out_h = dH;
                P.ldh = lddh;
                ok = ok && add_job(P, maps, type, p.grad_pair, DH, 256, T, D, words, p.splits, dl, p.Vp, static_cast<const char *>(W) + (size_t)v0 * (size_t)ldw * 2, ldw);
                ok = ok && (direct ? P.out_cols == 0 || set_output(maps, P.jobs - 1, type, dH, (uint64_t)P.out_cols, (uint64_t)T, lddh)
                                   : set_output(maps, P.jobs - 1, CDL_F32, acc, (uint64_t)p.acc_ld, (uint64_t)p.splits * (uint64_t)p.acc_rows, p.acc_ld));
            }
            if (dW != nullptr) {
                char *out = static_cast<char *>(dW) + (size_t)v0 * (size_t)lddw * 2;
                P.out_w = out;
                P.ldw = lddw;
                ok = ok && add_job(P, maps, type, p.grad_pair, DW, 256, words, D, T, 1, dl, p.Vp, H, ldh);
                ok = ok && (P.out_cols == 0 || set_output(maps, P.jobs - 1, type, out, (uint64_t)P.out_cols, (uint64_t)words, lddw));
            }
        }
        if (k + 1 < p.pieces) {
            const int v0 = (k + 1) * p.Vp, words = V - v0 < p.Vp ? V - v0 : p.Vp;
            P.v0 = v0;
            ok = ok && add_job(P, maps, type, p.grad_pair, DLOGIT, p.dlogit_tn, T, words, D, 1, H, ldh, static_cast<const char *>(W) + (size_t)v0 * (size_t)ldw * 2, ldw);
            ok = ok && set_output(maps, P.jobs - 1, type, base + p.off_dl + (size_t)((k + 1) & 1) * p.dl_bytes, (uint64_t)words, (uint64_t)T, p.Vp);
        }
        if (!ok) return CDL_ERR_LAUNCH;
        if ((rc = launch_jobs(p.grad_pair, true, type, maps, P, st)) != CDL_OK) return rc;
        if (k < 0 && p.pieces == 1) {
            const dim3 grid((unsigned)(((long long)T + 3) / 4));
            rc = type == CDL_BF16 ? launch_following(&loss_label_kernel<__nv_bfloat16>, grid, dim3(128), 0, st, (const float *)acc, p.others_ld, y, dloss, (const float *)scale,
                                                     (int)T, (int)V, reinterpret_cast<__nv_bfloat16 *>(base + p.off_dl), (long long)p.Vp)
                                  : launch_following(&loss_label_kernel<__half>, grid, dim3(128), 0, st, (const float *)acc, p.others_ld, y, dloss, (const float *)scale,
                                                     (int)T, (int)V, reinterpret_cast<__half *>(base + p.off_dl), (long long)p.Vp);
            if (rc != CDL_OK) return rc;
        }
    }
    if (dH != nullptr && p.splits > 1) {
        const long long units = (long long)T * ((D + 7) / 8);
        const int blocks = (int)(units / 128 + 1 < 4096 ? units / 128 + 1 : 4096);
        const long long step = (long long)p.acc_rows * p.acc_ld;
        if (type == CDL_BF16)
            return launch_following(&loss_sum_kernel<__nv_bfloat16>, dim3((unsigned)blocks), dim3(128), 0, st, (const float *)acc, p.acc_ld, step, p.splits,
                                    (int)T, (int)D, (const float *)scale, static_cast<__nv_bfloat16 *>(dH), (long long)lddh);
        return launch_following(&loss_sum_kernel<__half>, dim3((unsigned)blocks), dim3(128), 0, st, (const float *)acc, p.acc_ld, step, p.splits, (int)T, (int)D,
                                (const float *)scale, static_cast<__half *>(dH), (long long)lddh);
    }
    return CDL_OK;
}
