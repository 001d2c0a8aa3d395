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
// two passes is lse, one float per row, and the piece's dl is small enough to stay in L2 between the product that
// writes it and the two that read it.
//
// Tiles: 256 x 256 per CTA pair (cta_group::2), 64 reduced entries (128 bytes) per stage, six stages; two accumulators
// in TMEM let the epilogue of a tile run beside the products of the next.  With at most 128 rows (scoring, decoding) a CTA
// takes 128 x 256 by itself: rows beyond T are zero-filled by TMA, and the launch is bound by reading W once.
// Every wait is bounded.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_tc.cuh"
#include "cdl_wait.cuh"

namespace cdl {
namespace {

enum LossMode { STATS = 0, DLOGIT = 1, DW = 2, DH = 3 };

constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kBK = 64;                                // reduced entries of a stage (128 bytes)
constexpr int kBlockBytes = 128 * 128;                 // operand block of 128 rows
constexpr int kOutWarpBytes = 32 * 128;
constexpr int kStagesMax = 6;
constexpr int kSmemBytes = 1024 + kStagesMax * 2 * kBlockBytes + kEpiWarps * kOutWarpBytes;
constexpr unsigned long long kWaitNs = 2000000000ull;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr size_t kStatusBytes = 256;

struct LossParams {
    int I, J, R;                    // output rows, output columns, reduced entries
    int tiles_i, tiles_j, slots;
    const long long *labels;        // STATS, DLOGIT
    int v0;                         // word of column 0 (DLOGIT: first word of the piece)
    float2 *part;                   // STATS: (maximum, sum) per row and half tile
    int parts;                      // ... entries per row
    int V;                          // DLOGIT: words of the whole vocabulary
    float *target;                  // STATS: the label's logit
    const float *lse, *dloss;       // DLOGIT
    const float *scale;             // backward: {S, 1/S}, what dl is stored with
    int first, last;                // DH: first / last piece
    void *out;                      // DW, last DH: output, row pitch ldo, stored directly unless out_tma
    long long ldo;
    int out_tma;
    float *acc;                     // DH: binary32 sums, row pitch acc_ld
    long long acc_ld;
    int *status;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void tile_at(int u, int tiles_i, int tiles_j, int &ti, int &tj)
{
    const int band = 8 * tiles_j;
    const int b = u / band, first = b * 8, rows = min(8, tiles_i - first), in = u - b * band;
    tj = in / rows;
    ti = first + in - tj * rows;
}

template <bool PAIR, int MODE, typename T>
__global__ void __launch_bounds__(kThreads, 1)
loss_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                 const __grid_constant__ CUtensorMap map_o, const __grid_constant__ CUtensorMap map_f, const LossParams P)
{
    extern __shared__ unsigned char smem_dyn[];
    __shared__ __align__(8) unsigned long long bars[2 * kStagesMax + 4];
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;

    constexpr bool kAMn = MODE == DW, kBMn = MODE == DW || MODE == DH;
    constexpr int kBRows = PAIR ? 128 : 256;           // columns of the tile that this CTA stages
    constexpr uint32_t kBBytes = (uint32_t)kBRows * 128u;
    constexpr uint32_t kStageBytes = (uint32_t)kBlockBytes + kBBytes;
    constexpr int kStages = PAIR ? 6 : 4;
    static_assert(kStages * kStageBytes <= kStagesMax * 2 * kBlockBytes, "shared memory");
    const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &abort_s;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const int slot = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
    const int units = P.tiles_i * P.tiles_j, rblocks = (P.R + kBK - 1) / kBK;

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
    bool failed = false;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (one lane)
        if (lane == 0) {
            uint32_t st = 0u, par = 1u;
            auto load = [&](uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t fb) {
                if (PAIR) tma_load_2d_pair(dst, map, c0, c1, fb);
                else tma_load_2d(dst, map, c0, c1, fb);
            };
            for (int u = slot; u < units && !failed; u += P.slots) {
                int ti, tj;
                tile_at(u, P.tiles_i, P.tiles_j, ti, tj);
                const int arow = ti * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0);
                const int brow = tj * 256 + (PAIR ? (int)rank * 128 : 0);
                for (int rb = 0; rb < rblocks; ++rb) {
                    const uint32_t fb = bar0 + 8u * st;
                    if (!mbar_try_wait_now(fb + kEmptyOff, par) && !mbar_wait(fb + kEmptyOff, par, abort_flag, kWaitNs)) {
                        failed = true;
                        break;
                    }
                    const uint32_t sa = smem_base + st * kStageBytes, sb = sa + kBlockBytes;
                    const int r = rb * kBK;
                    if (!PAIR || rank == 0) mbar_expect_tx(fb, (PAIR ? 2u : 1u) * kStageBytes);
                    // K-major: one box of 64 reduced entries x the block's rows.  MN-major: boxes of 64 rows x 64
                    // reduced entries, the stored matrix's rows being the reduced dimension.
                    if (kAMn) {
                        load(sa, &map_a, arow, r, fb);
                        load(sa + 8192u, &map_a, arow + 64, r, fb);
                    } else load(sa, &map_a, r, arow, fb);
                    if (kBMn) {
#pragma unroll
                        for (int b = 0; b < kBRows / 64; ++b) load(sb + (uint32_t)b * 8192u, &map_b, brow + b * 64, r, fb);
                    } else load(sb, &map_b, r, brow, fb);
                    if (++st == (uint32_t)kStages) {
                        st = 0u;
                        par ^= 1u;
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (one lane; CTA 0 of a pair)
        if (lane == 0 && (!PAIR || rank == 0)) {
            // K-major: 128-byte rows, groups of eight 1024 bytes apart, 32 bytes per MMA.  MN-major: one reduced entry per
            // 128-byte line, eight lines 1024 bytes apart, 64-row blocks 8192 bytes apart, 16 lines per MMA.
            const uint64_t a_d = kAMn ? make_desc(smem_base, 8192, 1024) : make_desc(smem_base, 16, 1024);
            const uint64_t b_d = kBMn ? make_desc(smem_base + kBlockBytes, 8192, 1024) : make_desc(smem_base + kBlockBytes, 16, 1024);
            const uint32_t a_hi = (uint32_t)(a_d >> 32), b_hi = (uint32_t)(b_d >> 32), a_lo0 = (uint32_t)a_d, b_lo0 = (uint32_t)b_d;
            constexpr uint32_t a_step = kAMn ? 2048u >> 4 : 2u, b_step = kBMn ? 2048u >> 4 : 2u;
            constexpr uint32_t kFmt = sizeof(T) == 2 && __is_same(T, __nv_bfloat16) ? 1u : 0u;
            const uint32_t idesc = (1u << 4) | (kFmt << 7) | (kFmt << 10) | ((kAMn ? 1u : 0u) << 15) | ((kBMn ? 1u : 0u) << 16) |
                                   ((256u >> 3) << 17) | ((uint32_t)((PAIR ? 256 : 128) >> 4) << 24);
            uint32_t st = 0u, par = 0u, buf = 0u, tpar = 1u;
            for (int u = slot; u < units && !failed; u += P.slots) {
                if (!mbar_try_wait_now(tempty0 + 8u * buf, tpar) && !mbar_wait(tempty0 + 8u * buf, tpar, abort_flag, kWaitNs)) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                uint32_t accumulate = 0u;
                for (int rb = 0; rb < rblocks; ++rb) {
                    const uint32_t fb = bar0 + 8u * st;
                    if (!mbar_try_wait_now(fb, par) && !mbar_wait(fb, par, abort_flag, kWaitNs)) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t off = st * (kStageBytes >> 4);
                    tc_mma4<PAIR, KIND_F16>(tmem_base + buf * 256u, a_lo0 + off, a_hi, a_step, b_lo0 + off, b_hi, b_step, idesc, accumulate);
                    accumulate = 1u;
                    if (PAIR) tc_commit_pair(fb + kEmptyOff);
                    else tc_commit(fb + kEmptyOff);
                    if (++st == (uint32_t)kStages) {
                        st = 0u;
                        par ^= 1u;
                    }
                }
                if (!failed) {
                    if (PAIR) tc_commit_pair(tfull0 + 8u * buf);
                    else tc_commit(tfull0 + 8u * buf);
                }
                buf ^= 1u;
                if (buf == 0u) tpar ^= 1u;
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue warps: 32 rows x 128 columns each
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t wbuf = smem_base + (uint32_t)kStagesMax * 2u * kBlockBytes + (uint32_t)((warp - 2) * kOutWarpBytes);
        const float unscale = MODE == DW || MODE == DH ? P.scale[1] : 1.0f;
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
        for (int u = slot; u < units && !failed; u += P.slots) {
            int ti, tj;
            tile_at(u, P.tiles_i, P.tiles_j, ti, tj);
            const int row0 = ti * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0) + quarter * 32;
            const int col0 = tj * 256 + half * 128;
            const int row = row0 + lane;
            // what the epilogue needs of its row, fetched while the products run
            int label = -1;                              // column of the row's label in this tile's matrix, or outside it
            float lse2 = 0.0f, g = 0.0f;
            if ((MODE == STATS || MODE == DLOGIT) && row < P.I) {
                const long long y = P.labels[row];
                const long long words = MODE == STATS ? (long long)P.J : 0x7fffffffll;
                const long long c = y - P.v0;
                label = y >= 0 && c >= 0 && c < words ? (int)c : -1;
                if (MODE == DLOGIT) {
                    lse2 = P.lse[row] * kLog2e;
                    // (a label outside the vocabulary: no gradient)
                    g = y >= 0 && y < P.V ? P.dloss[row] * P.scale[0] : 0.0f;
                    if (!(y >= 0 && y < P.V)) label = -2;
                }
            }
            if (!__all_sync(0xffffffffu, mbar_try_wait_now(tfull0 + 8u * buf, tpar) || mbar_wait(tfull0 + 8u * buf, tpar, abort_flag, kWaitNs))) {
                failed = true;
                break;
            }
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * 256u + (uint32_t)(half * 128);
            const bool live = row0 < P.I && col0 < P.J;          // uniform over the warp
            if (live) {
                if (MODE == STATS) {
                    float m = -INFINITY, s = 0.0f, tgt = 0.0f;
                    bool hit = false;
#pragma unroll 1
                    for (int ch = 0; ch < 4; ++ch) {
                        const int c0 = col0 + ch * 32;
                        if (c0 >= P.J) break;
                        uint32_t v[32];
                        tc_ld32(taddr + (uint32_t)(ch * 32), v);
                        tc_wait_ld_pin(v);
                        if (c0 + 32 > P.J) {
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (c0 + c >= P.J) v[c] = 0xff800000u;       // a column that does not exist: -infinity
                        }
                        if (__any_sync(0xffffffffu, (unsigned)(label - c0) < 32u)) {
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (label == c0 + c) {
                                    tgt = __uint_as_float(v[c]);
                                    hit = true;
                                }
                        }
                        float cm = __uint_as_float(v[0]);
#pragma unroll
                        for (int c = 1; c < 32; ++c) cm = fmaxf(cm, __uint_as_float(v[c]));
                        const float mn = fmaxf(m, cm);
                        const float base = mn == -INFINITY ? 0.0f : mn * kLog2e;     // (all logits -infinity: exponentials are 0)
                        float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
                        for (int c = 0; c < 32; c += 4) {
                            s0 += exp2_fast(fmaf(__uint_as_float(v[c]), kLog2e, -base));
                            s1 += exp2_fast(fmaf(__uint_as_float(v[c + 1]), kLog2e, -base));
                            s2 += exp2_fast(fmaf(__uint_as_float(v[c + 2]), kLog2e, -base));
                            s3 += exp2_fast(fmaf(__uint_as_float(v[c + 3]), kLog2e, -base));
                        }
                        s = s * (m == -INFINITY ? 0.0f : exp2_fast(fmaf(m, kLog2e, -base))) + ((s0 + s1) + (s2 + s3));
                        m = mn;
                    }
                    if (row < P.I) {
                        P.part[(long long)row * P.parts + 2 * tj + half] = make_float2(m, s);
                        if (hit) P.target[row] = tgt;
                    }
                } else if (MODE == DLOGIT) {
#pragma unroll 1
                    for (int ch = 0; ch < 2; ++ch) {
                        const int c0 = col0 + ch * 64;
                        if (c0 >= P.J) break;
                        uint32_t w[32];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t v[32];
                            tc_ld32(taddr + (uint32_t)(ch * 64 + h * 32), v);
                            tc_wait_ld_pin(v);
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                v[c] = __float_as_uint(exp2_fast(fmaf(__uint_as_float(v[c]), kLog2e, -lse2)));
                            if (__any_sync(0xffffffffu, (unsigned)(label - (c0 + 32 * h)) < 32u)) {
#pragma unroll
                                for (int c = 0; c < 32; ++c)
                                    if (label == c0 + 32 * h + c) v[c] = __float_as_uint(__uint_as_float(v[c]) - 1.0f);
                            }
#pragma unroll
                            for (int c = 0; c < 16; ++c) {
                                const float d0 = label != -2 ? __uint_as_float(v[2 * c]) * g : 0.0f;
                                const float d1 = label != -2 ? __uint_as_float(v[2 * c + 1]) * g : 0.0f;
                                w[16 * h + c] = pack2<T>(d0, d1);
                            }
                        }
                        send(w, &map_o, false, c0, row0);
                    }
                } else if (MODE == DW || (MODE == DH && P.last)) {
#pragma unroll 1
                    for (int ch = 0; ch < 2; ++ch) {
                        const int c0 = col0 + ch * 64;
                        if (c0 >= P.J) break;
                        uint32_t w[32];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t v[32];
                            tc_ld32(taddr + (uint32_t)(ch * 64 + h * 32), v);
                            tc_wait_ld_pin(v);
                            if (MODE == DH && !P.first && row < P.I) {       // what the earlier pieces have summed
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
                        if (P.out_tma) send(w, &map_o, false, c0, row0);
                        else if (row < P.I) {
                            T *o = static_cast<T *>(P.out) + (long long)row * P.ldo + c0;
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                if (c0 + 8 * c + 8 <= P.J) *reinterpret_cast<uint4 *>(o + 8 * c) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
                                else
#pragma unroll
                                    for (int j = 0; j < 8; ++j)
                                        if (c0 + 8 * c + j < P.J)
                                            reinterpret_cast<unsigned short *>(o)[8 * c + j] = (unsigned short)(w[4 * c + (j >> 1)] >> (16 * (j & 1)));
                            }
                        }
                    }
                } else {
#pragma unroll 1
                    for (int ch = 0; ch < 4; ++ch) {
                        const int c0 = col0 + ch * 32;
                        if (c0 >= P.J) break;
                        uint32_t v[32];
                        tc_ld32(taddr + (uint32_t)(ch * 32), v);
                        tc_wait_ld_pin(v);
                        send(v, &map_f, !P.first, c0, row0);
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
    if (PAIR) cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        tmem_free_all<PAIR>(tmem_base);
    }
}

// One row per block: joins the tiles' maxima and sums, in a fixed order.
__global__ void __launch_bounds__(128)
loss_join_kernel(const float2 *__restrict__ part, int parts, const float *__restrict__ target, const long long *__restrict__ labels, int V,
                 float *__restrict__ loss, float *__restrict__ lse)
{
    __shared__ float2 sh[4];
    const long long row = blockIdx.x;
    const float2 *p = part + row * parts;
    float m = -INFINITY, s = 0.0f;
    auto join = [&](float m2, float s2) {
        const float mn = fmaxf(m, m2);
        if (mn != -INFINITY) s = s * exp2_fast((m - mn) * kLog2e) + s2 * exp2_fast((m2 - mn) * kLog2e);
        else s += s2;                                // (no maximum: 0, or NaN where a logit is NaN)
        m = mn;
    };
    for (int i = threadIdx.x; i < parts; i += 128) join(p[i].x, p[i].y);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o);
        join(m2, s2);
    }
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 1; k < 4; ++k) join(sh[k].x, sh[k].y);
        const float l = m + logf(s);
        const long long y = labels[row];
        lse[row] = l;
        loss[row] = y >= 0 && y < V ? l - target[row] : 0.0f;
    }
}

// The scale that dl is stored with, {S, 1/S}: S = top / max |dloss| over the counted positions (1 where there is none, or none
// that is finite).  A mean has the same dloss everywhere: the label's entry, p - 1 with a small p, then is a number of few
// bits, where dloss itself would be rounded the same way in every row and the error would add up instead of averaging out
// (measured on 777 x 32003 x 1000 in binary16: 3.9e-4 of dH's norm without it).  binary16 takes top = 2^14, so that
// probabilities down to 2^-28 are normal numbers.
__global__ void __launch_bounds__(1024)
loss_scale_kernel(const float *__restrict__ dloss, const long long *__restrict__ labels, int T, int V, float top, float *__restrict__ out)
{
    __shared__ float sh[32];
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
        }
    }
}

template <typename T>
const void *variant(int mode, bool pair)
{
    switch (mode) {
    case STATS: return pair ? reinterpret_cast<const void *>(&loss_gemm_kernel<true, STATS, T>) : reinterpret_cast<const void *>(&loss_gemm_kernel<false, STATS, T>);
    case DLOGIT: return pair ? reinterpret_cast<const void *>(&loss_gemm_kernel<true, DLOGIT, T>) : reinterpret_cast<const void *>(&loss_gemm_kernel<false, DLOGIT, T>);
    case DW: return pair ? reinterpret_cast<const void *>(&loss_gemm_kernel<true, DW, T>) : reinterpret_cast<const void *>(&loss_gemm_kernel<false, DW, T>);
    default: return pair ? reinterpret_cast<const void *>(&loss_gemm_kernel<true, DH, T>) : reinterpret_cast<const void *>(&loss_gemm_kernel<false, DH, T>);
    }
}
const void *variant(int mode, bool pair, int type) { return type == CDL_BF16 ? variant<__nv_bfloat16>(mode, pair) : variant<__half>(mode, pair); }

inline size_t up256(size_t n) { return (n + 255u) & ~(size_t)255u; }

// Layout of the workspace.  The forward part (partial statistics) and the backward part share the space after the status
// block and the scale.
struct LossPlan {
    int parts;              // partial statistics per row
    int pieces, Vp;         // vocabulary pieces of the backward pass and their width (a multiple of 256)
    size_t off_target;      // forward
    size_t off_acc;         // backward: binary32 sums of dH
    long long acc_ld;
    size_t fwd_bytes, bwd_bytes;
};
constexpr size_t kOffScale = kStatusBytes, kOffData = kStatusBytes + 256;
constexpr long long kPieceBytes = 64ll << 20;          // dl of one piece: half of L2

LossPlan make_plan(int T, int V, int D)
{
    LossPlan p;
    p.parts = (int)(((long long)V + 127) / 128);
    p.off_target = kOffData + up256((size_t)T * (size_t)p.parts * sizeof(float2));
    p.fwd_bytes = p.off_target + up256((size_t)T * sizeof(float));
    const long long words = ((long long)V + 255) / 256;                 // in units of 256
    long long most = kPieceBytes / (512ll * (T > 0 ? T : 1));
    if (most < 8) most = 8;
    p.pieces = (int)((words + most - 1) / most);
    p.Vp = (int)((words + p.pieces - 1) / p.pieces) * 256;
    p.pieces = (int)((V + (long long)p.Vp - 1) / p.Vp);
    p.acc_ld = ((long long)D + 255) / 256 * 256;
    p.off_acc = kOffData + up256((size_t)T * (size_t)p.Vp * 2);
    p.bwd_bytes = p.off_acc + (p.pieces > 1 ? up256((size_t)T * (size_t)p.acc_ld * sizeof(float)) : 0);
    return p;
}

// One product: output I x J, reduced over R.  a_mn / b_mn operands are stored [R][I] / [R][J].
int launch_product(int mode, int type, const void *A, long long lda, const void *B, long long ldb, const void *out, long long ldo,
                   const void *facc, long long ldf, LossParams &P, cudaStream_t stream)
{
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    const bool pair = P.I > 128;
    const bool a_mn = mode == DW, b_mn = mode == DW || mode == DH;
    const CUtensorMapDataType dt = type == CDL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap map_a, map_b, map_o, map_f;
    bool ok = a_mn ? encode_map_2d(&map_a, dt, 2, A, (uint64_t)P.I, (uint64_t)P.R, (uint64_t)lda * 2, 64)
                   : encode_map_2d(&map_a, dt, 2, A, (uint64_t)P.R, (uint64_t)P.I, (uint64_t)lda * 2, 128);
    ok = ok && (b_mn ? encode_map_2d(&map_b, dt, 2, B, (uint64_t)P.J, (uint64_t)P.R, (uint64_t)ldb * 2, 64)
                     : encode_map_2d(&map_b, dt, 2, B, (uint64_t)P.R, (uint64_t)P.J, (uint64_t)ldb * 2, pair ? 128 : 256));
    map_o = map_a;
    map_f = map_a;
    if (out != nullptr) ok = ok && encode_map_2d(&map_o, dt, 2, out, (uint64_t)P.J, (uint64_t)P.I, (uint64_t)ldo * 2, 32);
    if (facc != nullptr) ok = ok && encode_map_2d(&map_f, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, facc, (uint64_t)P.J, (uint64_t)P.I, (uint64_t)ldf * 4, 32);
    if (!ok) return CDL_ERR_LAUNCH;
    // (a TMA store fills the last 16-byte unit of a row with zeros beyond the output's columns: rows of a caller's matrix
    // that do not end on one are stored by the threads)
    P.out = const_cast<void *>(out);
    P.ldo = ldo;
    P.out_tma = P.J % 8 == 0;
    P.tiles_i = pair ? (P.I + 255) / 256 : (P.I + 127) / 128;
    P.tiles_j = (P.J + 255) / 256;
    static bool attr_set[64];
    static int pair_slots[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.attrs = at;
    if (!attr_set[dev]) {
        for (int m = 0; m < 4; ++m)
            for (int v = 0; v < 4; ++v)
                if (cudaFuncSetAttribute(variant(m, (v & 1) != 0, (v & 2) != 0 ? CDL_BF16 : CDL_F16), cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) {
                    (void)cudaGetLastError();
                    return CDL_ERR_LAUNCH;
                }
        cfg.gridDim = dim3(2u * (unsigned)(sms / 2));
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, variant(STATS, true, CDL_BF16), &cfg) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();
            n = sms / 2;
        }
        pair_slots[dev] = n < sms / 2 ? n : sms / 2;
        attr_set[dev] = true;
    }
    const long long units = (long long)P.tiles_i * P.tiles_j;
    if (units > 0x7fffffff) return CDL_ERR_ARG;
    const int most = pair ? pair_slots[dev] : sms;
    P.slots = (int)(units < most ? units : most);
    cfg.gridDim = dim3((pair ? 2u : 1u) * (unsigned)P.slots);
    cfg.stream = stream;
    cfg.numAttrs = pair ? 1 : 0;
    void *args[5] = {&map_a, &map_b, &map_o, &map_f, &P};
    if (cudaLaunchKernelExC(&cfg, variant(mode, pair, type), args) != cudaSuccess) {
        (void)cudaGetLastError();
        return CDL_ERR_LAUNCH;
    }
    return CDL_OK;
}

int check_common(const void *H, int64_t ldh, const void *W, int64_t ldw, int32_t type, const int64_t *labels, int32_t T, int32_t V, int32_t D)
{
    if (T < 0 || V < 1 || D < 1 || (type != CDL_BF16 && type != CDL_F16)) return CDL_ERR_ARG;
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
    if (T < 0 || V < 1 || D < 1) return 0;
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
    LossParams P;
    memset(&P, 0, sizeof P);
    P.I = T;
    P.J = V;
    P.R = D;
    P.labels = reinterpret_cast<const long long *>(labels);
    P.part = reinterpret_cast<float2 *>(base + kOffData);
    P.parts = p.parts;
    P.target = reinterpret_cast<float *>(base + p.off_target);
    P.status = static_cast<int *>(ws);
    if ((rc = launch_product(STATS, type, H, ldh, W, ldw, nullptr, 0, nullptr, 0, P, st)) != CDL_OK) return rc;
    loss_join_kernel<<<(unsigned)T, 128, 0, st>>>(P.part, p.parts, P.target, P.labels, V, loss, lse);
    return cudaGetLastError() == cudaSuccess ? CDL_OK : CDL_ERR_LAUNCH;
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
    LossParams P;
    memset(&P, 0, sizeof P);
    P.labels = reinterpret_cast<const long long *>(labels);
    P.lse = lse;
    P.dloss = dloss;
    P.V = V;
    P.status = static_cast<int *>(ws);
    float *scale = reinterpret_cast<float *>(base + kOffScale);
    loss_scale_kernel<<<1, 1024, 0, st>>>(dloss, P.labels, T, V, type == CDL_F16 ? 16384.0f : 1.0f, scale);
    if (cudaGetLastError() != cudaSuccess) return CDL_ERR_LAUNCH;
    P.scale = scale;
    void *dl = base + kOffData;
    P.acc = reinterpret_cast<float *>(base + p.off_acc);
    P.acc_ld = p.acc_ld;
    for (int k = 0; k < p.pieces; ++k) {
        const int v0 = k * p.Vp, words = V - v0 < p.Vp ? V - v0 : p.Vp;
        const char *Wk = static_cast<const char *>(W) + (size_t)v0 * (size_t)ldw * 2;
        P.v0 = v0;
        P.I = T;
        P.J = words;
        P.R = D;
        if ((rc = launch_product(DLOGIT, type, H, ldh, Wk, ldw, dl, p.Vp, nullptr, 0, P, st)) != CDL_OK) return rc;
        if (dW != nullptr) {
            P.I = words;
            P.J = D;
            P.R = T;
            if ((rc = launch_product(DW, type, dl, p.Vp, H, ldh, static_cast<char *>(dW) + (size_t)v0 * (size_t)lddw * 2, lddw, nullptr, 0, P, st)) != CDL_OK)
                return rc;
        }
        if (dH != nullptr) {
            P.I = T;
            P.J = D;
            P.R = words;
            P.first = k == 0;
            P.last = k == p.pieces - 1;
            if ((rc = launch_product(DH, type, dl, p.Vp, Wk, ldw, P.last ? dH : nullptr, lddh, P.last ? nullptr : P.acc, p.acc_ld, P, st)) != CDL_OK)
                return rc;
        }
    }
    return CDL_OK;
}
