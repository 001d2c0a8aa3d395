// Block-scaled product of 8-bit floating-point operands on the tensor cores of sm_100a:
//   out[m,n] = sum_kb sa[kb][m] * sb[kb][n or n / 128] * ( sum_{k in block kb of 128} A[m,k] B[n,k] )  (+ bias[n])
// A [M][K] and B [N][K] are e4m3 codes with the reduced dimension contiguous; the inner sum is one 128-byte pipeline
// stage: four tcgen05.mma (kind::f8f6f4, K = 32 each) into TMEM in binary32.
//
// The scales change with every stage, so an accumulator cannot stay in TMEM over the whole reduction: each stage's partial
// tile goes into the next of the TMEM buffers, the epilogue warps read it back while the following stages' products run,
// and add it, scaled, to the tile they keep in registers (one fused multiply-add per entry and stage; one more product
// where B's scales change from column to column).  For a 256 x 256 tile of a CTA pair a stage takes 930 cycles (1306 with column
// scales).  Measured one by one: the same loop without the hand-over 750 (the products are 510 of them, the delivery of the operands
// probably the rest), TMEM read-back and additions alone 320 (580: two packed instructions per two entries, two cycles each).  A
// partial tile is complete 800 cycles after its products are issued, drained 400 (750) later, and its buffer's release reaches the
// issuing thread another 200 later; over two buffers that makes 700 (875) a stage, so 180 (430) are not accounted for by these parts.
// 8192 x 8192 x 4096: 267 us, 2060 TFLOP/s; 315 to 320 under the power cap.  Between 5 and 128 rows a tile is mostly empty rows and
// the time is latency: 4096 x 4096 8.9 us for 8 rows, 10.1 for 128 (5.6 for 4 rows in their own form).
//
// Tiles: 256 x 256 per CTA pair (cta_group::2, as in the index products), or 128 x 128 per CTA where that is estimated to be
// faster (make_plan).  With few tiles (a short prompt) the reduced dimension is also cut over the CTAs of a cluster, whose
// partial tiles are added in a fixed order through distributed shared memory: no scratch in global memory, no atomics, one
// launch.  A last round that would fill the device partly is one sequence of stages, cut into as many runs as there are CTAs
// (pairs); tiles that runs share are added from the workspace by a second kernel (398 x 2507 x 23585, 20 pair tiles: 43 us
// against 82 in 80 single tiles; 2304 x 2304 x 4608, 81: 34 against 43; 48 x 139 x 34086: 13.2 against 18.5 over clusters).  Rows beyond
// M are zero-filled by TMA and cost no memory traffic.
// Warp roles: warp 0 issues TMA, warp 1 owns TMEM and issues the MMAs, warp 2 fetches scales (four stages at a time, with
// asynchronous 4-byte copies: handed over stage by stage they cost another barrier per stage, 1062 cycles instead of 930),
// warps 4..11 are the epilogue.  Every wait is bounded.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <string.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_tc.cuh"
#include "cdl_wait.cuh"

namespace cdl {
namespace {

constexpr int kEpiWarps = 8;
constexpr int kThreads = 128 + 32 * kEpiWarps;         // a warpgroup whose first three warps feed the others, two of epilogue warps
// Registers: a pair's epilogue thread holds 128 sums besides the 32 partial ones it has just read, more than an even share
// of the register file (168 for 384 threads).  The first warpgroup gives up what it does not need:
// 128 * 88 + 256 * 208 = 384 * 168.
constexpr int kRegsLaunch = 168, kRegsDrive = 88, kRegsEpilogue = 208;
static_assert(128 * kRegsDrive + 32 * kEpiWarps * kRegsEpilogue <= kThreads * kRegsLaunch, "register shares");
constexpr int kBlockBytes = 128 * 128;                 // one operand block of a stage: 128 rows x 128 bytes
constexpr int kStageBytes = 2 * kBlockBytes;
constexpr int kOutBytes = 32 * 64;                     // output staging block of a warp: 32 rows x 64 bytes
constexpr int kOutBlocks = 2;                          // ... of which a warp has as many stores in flight
constexpr int kOutWarpBytes = kOutBlocks * kOutBytes;
constexpr int kStages = 5;
constexpr int kGroup = 4;                              // stages whose scales are handed over together
constexpr int kScaleSlots = 4;                         // groups on their way or in use
__host__ __device__ constexpr int slot_floats(bool bvec) { return bvec ? 128 + 256 : 128 + 4; }      // scales of a stage: rows, then columns
__host__ __device__ constexpr int smem_bytes(bool bvec)
{
    return 1024 + kStages * kStageBytes + kEpiWarps * kOutWarpBytes + kScaleSlots * kGroup * slot_floats(bvec) * 4;
}
constexpr unsigned long long kWaitNs = 2000000000ull;

struct Fp8Params {
    int M, N, KB;                   // KB: blocks of 128 along the reduced dimension
    int tiles_i, tiles_j, slots;
    int splits;                     // CTAs of a cluster that share a tile (single-CTA tiles only)
    // The first `whole` tiles are taken as they are.  The stages of the tiles behind them, too few to fill the device once more,
    // are one sequence, cut into `ranges` runs of `run` stages wherever that falls; a tile that several runs share goes through
    // `part`, one piece per run r and tile t (counted from `whole`) at r + t.
    int whole, ranges, run;
    float *part;                    // [r + t][columns / 4 of a tile][rows of a tile][4]
    int nb;                         // scales of a k-block of B: N, or ceil(N / 128)
    const float *sa, *sb, *bias;
    void *out;
    long long ldo;
    int out_tma;                    // the output goes through shared memory and TMA
    int *status;
};

// four bytes from global to shared memory, asynchronously; zero where `live` is not set (nothing is read then)
__device__ __forceinline__ void copy4_async(uint32_t dst, const float *src, bool live)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(live ? 4 : 0) : "memory");
}
__device__ __forceinline__ float lds32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 lds128(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void store32_if(bool live, char *at, uint32_t v)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p st.global.b32 [%0], %1;\n\t}" ::"l"(at), "r"(v), "r"((uint32_t)live) : "memory");
}
__device__ __forceinline__ void store16_if(bool live, char *at, uint32_t v)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p st.global.b16 [%0], %1;\n\t}" ::"l"(at), "h"((unsigned short)v), "r"((uint32_t)live) : "memory");
}

// A staged piece, 32 rows of 64 bytes, to an output whose rows start anywhere: 16 lanes to a row, four bytes each, and no branch in
// between (with one per row, which waits for each row's limits, 8207 x 4234 x 223 took 47 us; now 40; entry by entry 74; a row per
// lane is slower still).  Rows of 16-bit entries that start between two words are staged one entry late: their first word ends
// with the piece's first entry and begins with the one before it, which the piece on the left has left over (`inner`: there is one).
template <typename T>
__device__ __forceinline__ void copy_rows(const Fp8Params &P, uint32_t src, int row0, int c0, bool inner, int lane)
{
    const int j = lane & 15, half = lane >> 4, rows = P.M - row0 - half;
    const int left = P.N - c0 - j * (4 / (int)sizeof(T));                // columns from this lane's entries on
    char *o = static_cast<char *>(P.out) + ((long long)(row0 + half) * P.ldo + c0) * (long long)sizeof(T) + j * 4;
    const long long step = 2 * P.ldo * (long long)sizeof(T);             // (a multiple of four bytes: `between` holds for all of a lane's rows)
    const bool between = sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(o) & 2u) != 0;
    const bool word = sizeof(T) == 4 ? left >= 1 : (between ? left >= 1 && (inner || j > 0) : left >= 2);
    const bool single = sizeof(T) == 2 && !between && left == 1;         // an odd last entry
    if (between) o -= 2;
#pragma unroll
    for (int b = 0; b < 2; ++b, o += 8 * step) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = __float_as_uint(lds32(src + (uint32_t)((b * 16 + i * 2 + half) * 64) + ((((uint32_t)j >> 2) ^ ((uint32_t)i & 3u)) << 4) + ((uint32_t)j & 3u) * 4u));
#pragma unroll
        for (int i = 0; i < 8; ++i) store32_if(word && b * 16 + i * 2 < rows, o + i * step, w[i]);
        if (sizeof(T) == 2 && (P.N & 1) != 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) store16_if(single && b * 16 + i * 2 < rows, o + i * step, w[i]);
        }
    }
}

// RUNS: some tiles are cut into runs of stages (in one kernel with the others, a product of 2048 x 2048 x 256 took 7.1 us, not 6.2).
template <bool PAIR, bool BVEC, bool RUNS, typename T>
__global__ void __launch_bounds__(kThreads, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_o, const Fp8Params P)
{
    extern __shared__ unsigned char smem_dyn[];
    __shared__ __align__(8) unsigned long long bars[2 * kStages + 8 + 2 * kScaleSlots];
    __shared__ uint32_t tmem_base_s, asked_s;
    __shared__ int abort_s, span_s[4];

    constexpr int kTN = PAIR ? 256 : 128;
    constexpr int kBufs = 512 / kTN;                   // TMEM buffers of a partial tile
    constexpr int kCols = kTN / 2;                     // columns of an epilogue warp
    const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &abort_s;
    const uint32_t rank = PAIR || P.splits > 1 ? cluster_ctarank() : 0u;
    const int slot = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x / P.splits;
    const int split = PAIR ? 0 : (int)rank;
    // The tiles of a CTA (a pair): slot, slot + slots and so on below `whole`, then those its run of stages touches (kept in
    // shared memory: the epilogue has no registers to spare).
    volatile int *span = span_s;                        // the run's stages, its tiles
    if (RUNS && threadIdx.x == 0) {
        int lo = 0, hi = 0, tail_first = P.whole, tail_end = P.whole;
        if (slot < P.ranges) {
            lo = slot * P.run;
            hi = min(lo + P.run, (P.tiles_i * P.tiles_j - P.whole) * P.KB);
            tail_first = P.whole + lo / P.KB;
            tail_end = P.whole + (hi - 1) / P.KB + 1;
        }
        span[0] = lo;
        span[1] = hi;
        span[2] = tail_first;
        span[3] = tail_end;
    }
    auto first_tile = [&] { return !RUNS || slot < P.whole ? slot : span[2]; };
    auto next_tile = [&](int u) { return !RUNS || u + P.slots < P.whole ? u + P.slots : (u < P.whole ? span[2] : u + 1); };
    auto end_tile = [&] { return RUNS ? span[3] : P.whole; };
    // its place, its k-blocks, and where the sums go: a piece, or (-1) the output
    auto tile_of = [&](int u, int &ti, int &tj, int &kb0, int &kb1, int &piece) {
        tile_at(u, P.tiles_i, P.tiles_j, ti, tj);
        const int parts = PAIR || RUNS ? 1 : P.splits;
        kb0 = parts == 1 ? 0 : (int)((long long)P.KB * split / parts);
        kb1 = parts == 1 ? P.KB : (int)((long long)P.KB * (split + 1) / parts);
        piece = -1;
        if (RUNS && u >= P.whole) {
            const int first = (u - P.whole) * P.KB;
            kb0 = max(span[0] - first, 0);
            kb1 = min(span[1] - first, P.KB);
            if (kb1 - kb0 < P.KB) piece = slot + u - P.whole;
        }
    };

    const uint32_t bar0 = smem_u32(&bars[0]);
    constexpr uint32_t kEmptyOff = 8u * kStages;
    const uint32_t tfull0 = bar0 + 16u * kStages, tempty0 = tfull0 + 32u;
    const uint32_t sfull0 = tempty0 + 32u;              // scales of a stage are there; taken: + 8 kScaleSlots
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar0 + 8u * s, 1);
            mbar_init(bar0 + kEmptyOff + 8u * s, 1);
        }
        for (int b = 0; b < kBufs; ++b) {
            mbar_init(tfull0 + 8u * b, 1);
            mbar_init(tempty0 + 8u * b, (PAIR ? 2 : 1) * kEpiWarps);
        }
        for (int s = 0; s < kScaleSlots; ++s) {
            mbar_init(sfull0 + 8u * s, 32);
            mbar_init(sfull0 + 8u * (kScaleSlots + s), kEpiWarps);
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
    const uint32_t scale_base = smem_base + (uint32_t)(kStages * kStageBytes + kEpiWarps * kOutWarpBytes);

    if (warp < 4) {
        if (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsDrive));
        if (warp == 0) {
            // ------------------------------------------------------------ TMA producer (one lane)
            if (lane == 0) {
                uint32_t st = 0u, par = 1u, asked = 0u;
                for (int u = first_tile(); u < end_tile() && !failed; u = next_tile(u)) {
                    int ti, tj, kb0, kb1, piece;
                    tile_of(u, ti, tj, kb0, kb1, piece);
                    const int arow = ti * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0);
                    const int brow = tj * kTN + (PAIR ? (int)rank * 128 : 0);
                    for (int kb = kb0; kb < kb1; ++kb) {
                        const uint32_t fb = bar0 + 8u * st;
                        if (!mbar_try_wait_now(fb + kEmptyOff, par) && !mbar_wait(fb + kEmptyOff, par, abort_flag, kWaitNs)) {
                            failed = true;
                            break;
                        }
                        const uint32_t sa = smem_base + st * (uint32_t)kStageBytes, sb = sa + kBlockBytes;
                        if (!PAIR || rank == 0) mbar_expect_tx(fb, (PAIR ? 2u : 1u) * (uint32_t)kStageBytes);
                        if (PAIR) {
                            tma_load_2d_pair(sa, &map_a, kb * 128, arow, fb);
                            tma_load_2d_pair(sb, &map_b, kb * 128, brow, fb);
                        } else {
                            tma_load_2d(sa, &map_a, kb * 128, arow, fb);
                            tma_load_2d(sb, &map_b, kb * 128, brow, fb);
                        }
                        ++asked;
                        if (++st == (uint32_t)kStages) {
                            st = 0u;
                            par ^= 1u;
                        }
                    }
                }
                asked_s = asked;
            }
        } else if (warp == 1) {
            // ------------------------------------------------------------ MMA issuer (one lane; CTA 0 of a pair)
            if (lane == 0 && (!PAIR || rank == 0)) {
                const uint64_t a_d = make_desc(smem_base, 16, 1024), b_d = make_desc(smem_base + kBlockBytes, 16, 1024);
                const uint32_t a_hi = (uint32_t)(a_d >> 32), b_hi = (uint32_t)(b_d >> 32), a_lo0 = (uint32_t)a_d, b_lo0 = (uint32_t)b_d;
                // D binary32, A and B e4m3, both K-major
                const uint32_t idesc = (1u << 4) | ((uint32_t)(kTN >> 3) << 17) | ((uint32_t)((PAIR ? 256 : 128) >> 4) << 24);
                uint32_t st = 0u, par = 0u, buf = 0u, tpar = 1u;
                for (int u = first_tile(); u < end_tile() && !failed; u = next_tile(u)) {
                    int ti, tj, kb0, kb1, piece;
                    tile_of(u, ti, tj, kb0, kb1, piece);
                    for (int kb = kb0; kb < kb1; ++kb) {
                        const uint32_t fb = bar0 + 8u * st, tf = tfull0 + 8u * buf, te = tempty0 + 8u * buf;
                        if ((!mbar_try_wait_now(fb, par) && !mbar_wait(fb, par, abort_flag, kWaitNs)) ||
                            (!mbar_try_wait_now(te, tpar) && !mbar_wait(te, tpar, abort_flag, kWaitNs))) {
                            failed = true;
                            break;
                        }
                        tc_fence_after();
                        const uint32_t off = st * (uint32_t)(kStageBytes >> 4);
                        tc_mma4<PAIR, KIND_F8F6F4>(tmem_base + buf * (uint32_t)kTN, a_lo0 + off, a_hi, 2u, b_lo0 + off, b_hi, 2u, idesc, 0u);
                        if (PAIR) {
                            tc_commit_pair(tf);
                            tc_commit_pair(fb + kEmptyOff);
                        } else {
                            tc_commit(tf);
                            tc_commit(fb + kEmptyOff);
                        }
                        if (++st == (uint32_t)kStages) {
                            st = 0u;
                            par ^= 1u;
                        }
                        if (++buf == (uint32_t)kBufs) {
                            buf = 0u;
                            tpar ^= 1u;
                        }
                    }
                }
            }
        } else if (warp == 2) {
            // ------------------------------------------------------------ scales: a stage's row and column scales by
            // asynchronous 4-byte copies (their addresses have no alignment to rely on), several stages ahead
            uint32_t q = 0u, par = 1u;
            for (int u = first_tile(); u < end_tile() && !failed; u = next_tile(u)) {
                int ti, tj, kb0, kb1, piece;
                tile_of(u, ti, tj, kb0, kb1, piece);
                const int arow = ti * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0), col = tj * kTN;
                for (int kg = kb0; kg < kb1; kg += kGroup) {
                    const uint32_t sf = sfull0 + 8u * q;
                    if (!__all_sync(0xffffffffu, mbar_try_wait_now(sf + 8u * kScaleSlots, par) || mbar_wait(sf + 8u * kScaleSlots, par, abort_flag, kWaitNs))) {
                        failed = true;
                        break;
                    }
                    for (int kb = kg; kb < min(kg + kGroup, kb1); ++kb) {
                        const uint32_t dst = scale_base + (q * (uint32_t)kGroup + (uint32_t)(kb - kg)) * (uint32_t)(slot_floats(BVEC) * 4);
                        const float *pa = P.sa + (long long)kb * P.M, *pb = P.sb + (long long)kb * P.nb;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int r = arow + j * 32 + lane;
                            copy4_async(dst + (uint32_t)(j * 32 + lane) * 4u, r < P.M ? pa + r : P.sa, r < P.M);
                        }
                        if (BVEC) {
#pragma unroll
                            for (int j = 0; j < kTN / 32; ++j) {
                                const int c = col + j * 32 + lane;
                                copy4_async(dst + (uint32_t)(128 + j * 32 + lane) * 4u, c < P.N ? pb + c : P.sb, c < P.N);
                            }
                        } else if (lane < kTN / 128) {
                            const int c = (col >> 7) + lane;
                            copy4_async(dst + (uint32_t)(128 + lane) * 4u, c < P.nb ? pb + c : P.sb, c < P.nb);
                        }
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(sf) : "memory");
                    if (++q == (uint32_t)kScaleSlots) {
                        q = 0u;
                        par ^= 1u;
                    }
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
    } else {
        if (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpilogue));
        // ------------------------------------------------------------ epilogue warps: 32 rows x kCols columns each
        float2 acc[kCols / 2];
        const int quarter = warp & 3, group = (warp - 4) >> 2;
        auto tile_col = [&](int ch) { return group * kCols + ch * 32; };      // of chunk ch of 32 columns
        const uint32_t wbuf = smem_base + (uint32_t)(kStages * kStageBytes) + (uint32_t)((warp - 4) * kOutWarpBytes);
        uint32_t buf = 0u, tpar = 0u, q = 0u, spar = 0u, oblk = 0u;
        for (int u = first_tile(); u < end_tile() && !failed; u = next_tile(u)) {
            int ti, tj, kb0, kb1, piece;
            tile_of(u, ti, tj, kb0, kb1, piece);
#pragma unroll
            for (int j = 0; j < kCols / 2; ++j) acc[j] = make_float2(0.0f, 0.0f);
            int in = 0;                                  // stage of the group
            for (int kb = kb0; kb < kb1; ++kb) {
                const uint32_t blk = buf, tf = tfull0 + 8u * blk;
                if (in == 0) {
                    const uint32_t sf = sfull0 + 8u * q;
                    if (!__all_sync(0xffffffffu, mbar_try_wait_now(sf, spar) || mbar_wait(sf, spar, abort_flag, kWaitNs))) {
                        failed = true;
                        break;
                    }
                }
                const uint32_t sc = scale_base + (q * (uint32_t)kGroup + (uint32_t)in) * (uint32_t)(slot_floats(BVEC) * 4);
                float s_row = lds32(sc + (uint32_t)(quarter * 32 + lane) * 4u);
                if (!BVEC) s_row *= lds32(sc + (uint32_t)(128 + (PAIR ? group : 0)) * 4u);
                if (!__all_sync(0xffffffffu, mbar_try_wait_now(tf, tpar) || mbar_wait(tf, tpar, abort_flag, kWaitNs))) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + blk * (uint32_t)kTN;
                // 16 columns at a time, the next ones on their way while these are added
                uint32_t va[16], vb[16];
                float4 f[BVEC ? 4 : 1];                  // column scales of the 16 columns
                auto fetch = [&](int c16) {
                    if (BVEC) {
                        const uint32_t sv = sc + (uint32_t)(128 + tile_col(c16 >> 1) + (c16 & 1) * 16) * 4u;
#pragma unroll
                        for (int j = 0; j < 4; ++j) f[BVEC ? j : 0] = lds128(sv + (uint32_t)j * 16u);
                    }
                };
                auto add = [&](const uint32_t (&v)[16], int c16) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float2 f0 = make_float2(s_row, s_row), f1 = f0;
                        if (BVEC) {
                            f0 = mul2(f0, make_float2(f[BVEC ? j : 0].x, f[BVEC ? j : 0].y));
                            f1 = mul2(f1, make_float2(f[BVEC ? j : 0].z, f[BVEC ? j : 0].w));
                        }
                        fma2(acc[c16 * 8 + 2 * j], v[4 * j], v[4 * j + 1], f0);
                        fma2(acc[c16 * 8 + 2 * j + 1], v[4 * j + 2], v[4 * j + 3], f1);
                    }
                };
                tc_ld16(taddr + (uint32_t)tile_col(0), va);
                fetch(0);
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    tc_wait_ld_pin(va);
                    tc_ld16(taddr + (uint32_t)tile_col(c) + 16u, vb);
                    add(va, 2 * c);
                    fetch(2 * c + 1);
                    tc_wait_ld_pin(vb);
                    if (c < kCols / 32 - 1) {
                        tc_ld16(taddr + (uint32_t)tile_col(c + 1), va);
                        add(vb, 2 * c + 1);
                        fetch(2 * c + 2);
                    } else {                             // the partial tile is in registers: its buffer is free
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if (PAIR) mbar_arrive_remote(tempty0 + 8u * blk, 0u);
                            else mbar_arrive(tempty0 + 8u * blk);
                        }
                        if (++buf == (uint32_t)kBufs) {
                            buf = 0u;
                            tpar ^= 1u;
                        }
                        add(vb, 2 * c + 1);
                        if (++in == kGroup || kb + 1 == kb1) {       // the group's scales have been read
                            __syncwarp();
                            if (lane == 0) mbar_arrive(sfull0 + 8u * (kScaleSlots + q));
                            in = 0;
                            if (++q == (uint32_t)kScaleSlots) {
                                q = 0u;
                                spar ^= 1u;
                            }
                        }
                    }
                }
            }
            if (failed) break;
            if (RUNS) {                                  // its place is worked out anew instead of being held over the stages
                asm("" : "+r"(u));
                tile_of(u, ti, tj, kb0, kb1, piece);
            }
            const int row0 = ti * (PAIR ? 256 : 128) + (PAIR ? (int)rank * 128 : 0) + quarter * 32;
            const int row = row0 + lane;
            if (!PAIR && P.splits > 1) {
                // The partial tile, [rows][128] binary32, takes the place of the pipeline's stages: this warp has seen the
                // last of the CTA's products, so all loads have landed and been read.  16-byte units of a row are
                // exclusive-ored with the row number: eight rows at a time hit all banks.
                float *part = reinterpret_cast<float *>(smem_dyn + (smem_base - smem_u32(smem_dyn)));
                const int r = quarter * 32 + lane;
                if (row < P.M) {
#pragma unroll
                    for (int j = 0; j < kCols / 4; ++j) {
                        const int unit = (group * kCols >> 2) + j;
                        *reinterpret_cast<float4 *>(part + r * 128 + ((unit ^ (r & 7)) << 2)) =
                            make_float4(acc[2 * j].x, acc[2 * j].y, acc[2 * j + 1].x, acc[2 * j + 1].y);
                    }
                }
                break;
            }
            if (row0 >= P.M) continue;
            if (RUNS && piece >= 0) {
                // a part of a tile: its sums as they are, four columns of 32 consecutive rows per instruction
                constexpr int kRows = PAIR ? 256 : 128;
                float4 *q = reinterpret_cast<float4 *>(P.part) + ((long long)piece * (kTN / 4) + group * (kCols / 4)) * kRows + (PAIR ? (int)rank * 128 : 0) + quarter * 32 + lane;
#pragma unroll
                for (int j = 0; j < kCols / 4; ++j) q[j * kRows] = make_float4(acc[2 * j].x, acc[2 * j].y, acc[2 * j + 1].x, acc[2 * j + 1].y);
                continue;
            }
            T *row_out = static_cast<T *>(P.out) + (long long)row * P.ldo;
            const bool late = sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(row_out) & 2u) != 0;       // (see copy_rows)
            uint32_t before = 0u;
#pragma unroll
            for (int ch = 0; ch < kCols / 32; ++ch) {
                const int col0 = tj * kTN + tile_col(ch);
                if (col0 >= P.N) continue;
                float2 *a = acc + ch * 16;
                if (P.bias != nullptr) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (col0 + 2 * j < P.N) a[j].x += P.bias[col0 + 2 * j];
                        if (col0 + 2 * j + 1 < P.N) a[j].y += P.bias[col0 + 2 * j + 1];
                    }
                }
                // 64-byte pieces of the warp's 32 rows through its staging block (64-byte swizzle), then by TMA (which clips at the
                // edges), or, where rows do not start and end on 16 bytes, copied out row by row
                constexpr int kPiece = 64 / (int)sizeof(T);
#pragma unroll
                for (int pc = 0; pc < 32 / kPiece; ++pc) {
                    const int c0 = col0 + pc * kPiece;
                    if (c0 >= P.N) break;
                    if (lane == 0) bulk_wait_read<kOutBlocks - 1>();     // the store that last used this block has read it
                    __syncwarp();
                    const uint32_t src = wbuf + oblk, dst = src + (uint32_t)lane * 64u;
#pragma unroll
                    for (int c4 = 0; c4 < 4; ++c4) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if constexpr (sizeof(T) == 4) w[j] = __float_as_uint((j & 1) ? a[pc * 8 + c4 * 2 + (j >> 1)].y : a[pc * 8 + c4 * 2 + (j >> 1)].x);
                            else {
                                const uint32_t two = pack2<T>(a[c4 * 4 + j].x, a[c4 * 4 + j].y);
                                w[j] = late ? __funnelshift_r(before, two, 16) : two;
                                if (c4 == 0 && j == 0 && ch == 0) store16_if(late && row < P.M, reinterpret_cast<char *>(row_out + c0), two);
                                before = two;
                            }
                        }
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)((c4 ^ ((lane >> 1) & 3)) << 4)),
                                     "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                                     : "memory");
                    }
                    if (P.out_tma) {
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(&map_o, c0, row0, src);
                            bulk_commit();
                        }
                    } else {
                        __syncwarp();
                        copy_rows<T>(P, src, row0, c0, ch > 0, lane);
                        if constexpr (sizeof(T) == 2) {                  // what the last piece of a late row has left over
                            const int cols = min(kPiece, P.N - c0);
                            if (late && row < P.M && (cols & 1) == 0 && (ch == kCols / 32 - 1 || c0 + kPiece >= P.N)) {
                                uint32_t v = before >> 16;
                                if (cols < kPiece) v = __float_as_uint(lds32(src + (uint32_t)lane * 64u + ((((uint32_t)cols >> 3) ^ (((uint32_t)lane >> 1) & 3u)) << 4) + (((uint32_t)cols >> 1) & 3u) * 4u));
                                store16_if(true, reinterpret_cast<char *>(row_out + c0 + cols - 1), v);
                            }
                        }
                        __syncwarp();
                    }
                    oblk = oblk + (uint32_t)kOutBytes == (uint32_t)kOutWarpBytes ? 0u : oblk + (uint32_t)kOutBytes;
                }
            }
        }
        if (lane == 0) bulk_wait_all();
    }
    if (failed) {
        abort_s = 1;
        if (lane == 0) record_timeout(P.status);
    }

    if (!PAIR && P.splits > 1) {
        // each CTA adds its share of the tile's entries over the cluster's partial tiles, in the order of the splits
        int ti, tj;
        tile_at(slot, P.tiles_i, P.tiles_j, ti, tj);
        const int rows = min(128, P.M - ti * 128), cols = min(128, P.N - tj * 128);
        __syncthreads();
        cluster_sync_all();
        const int n4 = rows * 32;
        for (int i = (int)rank * kThreads + (int)threadIdx.x; i < n4; i += P.splits * kThreads) {
            const int r = i >> 5, unit = i & 31, c = unit * 4;
            if (c >= cols) continue;
            const uint32_t local = smem_base + (uint32_t)(r * 128 + ((unit ^ (r & 7)) << 2)) * 4u;
            float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int s = 0; s < P.splits; ++s) {
                float4 v;
                asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\t"
                             "ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
                             : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                             : "r"(local), "r"(s));
                sum.x += v.x;
                sum.y += v.y;
                sum.z += v.z;
                sum.w += v.w;
            }
            const float o4[4] = {sum.x, sum.y, sum.z, sum.w};
            T *o = static_cast<T *>(P.out) + (long long)(ti * 128 + r) * P.ldo + tj * 128 + c;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < cols) o[j] = from_f32<T>(o4[j] + (P.bias != nullptr ? P.bias[tj * 128 + c + j] : 0.0f));
        }
    }

    tc_fence_before();
    __syncthreads();
    // after an abandoned wait: loads that are still under way land (or a limit runs out) before the CTA ends
    if (abort_s != 0 && threadIdx.x == 0 && (!PAIR || rank == 0)) drain_stages(bar0, asked_s, (uint32_t)kStages);
    __syncwarp();
    if (PAIR || P.splits > 1) cluster_sync_all();       // no CTA leaves while another may touch its shared memory or TMEM
    if (warp == 1) {
        tc_fence_after();
        tmem_free_all<PAIR>(tmem_base);
    }
}

template <bool PAIR, bool BVEC, bool RUNS>
const void *variant(int type)
{
    if (type == CDL_F32) return reinterpret_cast<const void *>(&fp8_gemm_kernel<PAIR, BVEC, RUNS, float>);
    if (type == CDL_BF16) return reinterpret_cast<const void *>(&fp8_gemm_kernel<PAIR, BVEC, RUNS, __nv_bfloat16>);
    return reinterpret_cast<const void *>(&fp8_gemm_kernel<PAIR, BVEC, RUNS, __half>);
}
template <bool PAIR, bool BVEC>
const void *variant(int type, bool runs) { return runs ? variant<PAIR, BVEC, true>(type) : variant<PAIR, BVEC, false>(type); }
const void *variant(int type, bool pair, bool bvec, bool runs)
{
    if (pair) return bvec ? variant<true, true>(type, runs) : variant<true, false>(type, runs);
    return bvec ? variant<false, true>(type, runs) : variant<false, false>(type, runs);
}

// The tiles that runs share: their pieces in the order of the runs, the bias, the output type.  A block takes 64 rows x 16 columns:
// read as the pieces are stored (consecutive threads on consecutive rows), written along rows through shared memory.
constexpr int kSumRows = 64, kSumCols = 16;
template <int EDGE, typename T>
__global__ void __launch_bounds__(kSumRows * kSumCols / 4)
fp8_sum_kernel(const float *part, int run, int KB, int first, int tiles_i, int tiles_j, int M, int N, const float *bias, T *out, long long ldo)
{
    __shared__ float tile[kSumRows][kSumCols + 1];
    follow_previous();                                  // (also where nothing is left to do: what follows relies on it)
    const int t = (int)blockIdx.x, r0 = t * KB / run, r1 = ((t + 1) * KB - 1) / run;
    if (r0 == r1) return;                               // one run had all of it
    int ti, tj;
    tile_at(first + t, tiles_i, tiles_j, ti, tj);
    constexpr int kAcross = EDGE / kSumCols;
    const int rb = (int)blockIdx.y / kAcross * kSumRows, cb = (int)blockIdx.y % kAcross * kSumCols;
    const long long row0 = (long long)ti * EDGE + rb;
    const int col0 = tj * EDGE + cb, r = (int)threadIdx.x % kSumRows, c4 = (int)threadIdx.x / kSumRows;
    if (row0 >= M || col0 >= N) return;
    if (row0 + r < M) {                                 // (rows beyond M were not stored)
        const float4 *q = reinterpret_cast<const float4 *>(part) + ((long long)(r0 + t) * (EDGE / 4) + cb / 4 + c4) * EDGE + rb + r;
        float4 v = q[0];
#pragma unroll 8
        for (int k = 1; k <= r1 - r0; ++k) {
            const float4 w = q[(long long)k * (EDGE / 4) * EDGE];
            v.x += w.x;
            v.y += w.y;
            v.z += w.z;
            v.w += w.w;
        }
        tile[r][c4 * 4] = v.x;
        tile[r][c4 * 4 + 1] = v.y;
        tile[r][c4 * 4 + 2] = v.z;
        tile[r][c4 * 4 + 3] = v.w;
    }
    __syncthreads();
    const int c = (int)threadIdx.x % kSumCols;
    if (col0 + c >= N) return;
    const float b = bias != nullptr ? bias[col0 + c] : 0.0f;
#pragma unroll
    for (int k = (int)threadIdx.x / kSumCols; k < kSumRows; k += kSumRows / 4)
        if (row0 + k < M) out[(row0 + k) * ldo + col0 + c] = from_f32<T>(tile[k][c] + b);
}

template <typename T>
int launch_sum(bool pair, const Fp8Params &P, cudaStream_t st)
{
    const int edge = pair ? 256 : 128;
    const dim3 grid((unsigned)(P.tiles_i * P.tiles_j - P.whole), (unsigned)((edge / kSumRows) * (edge / kSumCols)));
    return launch_following(pair ? &fp8_sum_kernel<256, T> : &fp8_sum_kernel<128, T>, grid, dim3(kSumRows * kSumCols / 4), 0, st,
                            static_cast<const float *>(P.part), P.run, P.KB, P.whole, P.tiles_i, P.tiles_j, P.M, P.N, P.bias, static_cast<T *>(P.out), P.ldo);
}

// out = bias (or 0) where the reduced dimension is empty
template <typename T>
__global__ void fill_bias_kernel(T *out, long long ldo, long long M, int N, const float *bias)
{
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < M * N; i += (long long)gridDim.x * blockDim.x)
        out[i / N * ldo + i % N] = from_f32<T>(bias != nullptr ? bias[i % N] : 0.0f);
}

}  // namespace
}  // namespace cdl

namespace {
// What a product of these sizes runs as.  Planned for a B200's 148 SMs so that workspace sizes are fixed.
struct Fp8Plan {
    bool rows;                  // few rows of A: the form of its own
    bool pair;
    int tiles_i, tiles_j;
    int splits;                 // CTAs of a cluster per tile (single-CTA tiles)
    int whole, ranges, run;     // see Fp8Params
    size_t part_bytes;
};
constexpr int kPlanSms = 148;
constexpr int64_t kL2Bytes = 126000000;
constexpr size_t kStatusBytes = 256;

bool make_plan(int32_t M, int32_t N, int32_t K, Fp8Plan *p)
{
    const int64_t KB = ((int64_t)K + 127) / 128, pairs = kPlanSms / 2;
    const int64_t pair_tiles = (((int64_t)M + 255) / 256) * (((int64_t)N + 255) / 256), tiles = (((int64_t)M + 127) / 128) * (((int64_t)N + 127) / 128);
    if (tiles > 0x3fffffff) return false;
    // Three forms, each with its estimate in nanoseconds: tiles as they are; with the last, partly filled round cut into runs
    // that fill the device, which costs the pieces' way through memory and another launch; and, for few tiles of a single CTA,
    // cut over the CTAs of a cluster.  (Clusters of four and eight do not fit everywhere: the device runs 32 and 14 of them at
    // once for certain.)
    struct Form { int64_t ns, whole, ranges, run, splits, piece_bytes; bool pair; } best = {INT64_MAX, 0, 0, 0, 1, 0, false};
    auto consider = [&](const Form &f) {
        if (f.ns < best.ns) best = f;
    };
    for (int pair = 0; pair < 2; ++pair) {
        const int64_t slots = pair ? pairs : kPlanSms, n = pair ? pair_tiles : tiles, tail = n % slots, stage = pair ? 550 : 420;
        const int64_t start = pair ? 5000 : 4000, tile = (pair ? 1200 : 800) + stage * KB, edge = pair ? 256 : 128;
        consider(Form{start + (n + slots - 1) / slots * tile, n, 0, 0, 1, 0, pair != 0});
        if (tail > 0) {
            const int64_t stages = tail * KB, most = stages / 4 < slots ? stages / 4 : slots;        // four stages at least
            if (most > 1) {
                const int64_t run = (stages + most - 1) / most, ranges = (stages + run - 1) / run, bytes = (ranges + tail) * edge * edge * 4;
                // (tiles that run side by side no longer read the same k-blocks at one time: 582 x 5164 x 34907 in pairs 156 us, 147 whole)
                const int64_t apart = ((int64_t)M + N) * K > kL2Bytes ? stage * run / 10 : 0;
                consider(Form{start + n / slots * tile + stage * run + apart + (pair ? 3000 : 1000) + 3500 + bytes / 6000 + 30 * (ranges / tail), n - tail, ranges, run, 1, bytes, pair != 0});
            }
        }
    }
    int64_t splits = 1;
    const int64_t clusters[4] = {kPlanSms, pairs, 32, 14};
    for (int i = 1; i < 4 && tiles <= clusters[i] && (2ll << i) <= KB; ++i) splits = 1ll << i;
    if (splits > 1) consider(Form{4000 + 800 + 420 * ((KB + splits - 1) / splits) + 2000, tiles, 0, 0, splits, 0, false});
    // A few rows take the form that streams B past them, unless this one is clearly faster (rows of B too short for it: 1 x 100000 x
    // 128 16.0 us there, 11.1 here; 30000 x 500 6.6 and 8.8).
    p->rows = M <= cdl::kFewRowsFp8 && cdl::plan_fp8_rows(N, K).ns * 85 / 100 <= best.ns;
    const int edge = best.pair ? 256 : 128;
    p->pair = best.pair;
    p->tiles_i = (int)(((int64_t)M + edge - 1) / edge);
    p->tiles_j = (int)(((int64_t)N + edge - 1) / edge);
    p->splits = (int)best.splits;
    p->whole = (int)best.whole;
    p->ranges = (int)best.ranges;
    p->run = (int)best.run;
    p->part_bytes = p->rows ? 0 : (size_t)best.piece_bytes;
    return true;
}
}  // namespace

extern "C" size_t cdl_fp8_matmul_workspace_bytes(int32_t M, int32_t N, int32_t K)
{
    Fp8Plan p;
    if (M < 0 || N < 0 || K < 0 || M > cdl::kMostExtent || N > cdl::kMostExtent || K > cdl::kMostExtent) return 0;
    return make_plan(M, N, K, &p) ? kStatusBytes + p.part_bytes : kStatusBytes;      // the status block, the parts of cut tiles
}

extern "C" int cdl_fp8_matmul(const void *A, int64_t lda, const float *a_scale, const void *B, int64_t ldb, const float *b_scale,
                              int32_t b_mode, int32_t M, int32_t N, int32_t K, void *out, int64_t ldo, int32_t out_type,
                              const float *bias, void *ws, size_t ws_bytes, void *stream)
{
    using namespace cdl;
    if (M < 0 || N < 0 || K < 0 || M > kMostExtent || N > kMostExtent || K > kMostExtent || !valid_type(out_type) || (b_mode != CDL_FP8_ROWS && b_mode != CDL_FP8_BLOCKS)) return CDL_ERR_ARG;
    if (M == 0 || N == 0) return CDL_OK;
    if (out == nullptr || ldo < N) return CDL_ERR_ARG;
    if (K > 0 && (A == nullptr || B == nullptr || a_scale == nullptr || b_scale == nullptr || lda < K || ldb < K)) return CDL_ERR_ARG;
    if (misaligned(out, out_type) || (reinterpret_cast<uintptr_t>(bias) & 3u)) return CDL_ERR_ALIGN;
    if (K > 0 && ((reinterpret_cast<uintptr_t>(A) & 15u) || (reinterpret_cast<uintptr_t>(B) & 15u) || (lda & 15) || (ldb & 15) ||
                  (reinterpret_cast<uintptr_t>(a_scale) & 3u) || (reinterpret_cast<uintptr_t>(b_scale) & 3u)))
        return CDL_ERR_ALIGN;
    if (ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < cdl_fp8_matmul_workspace_bytes(M, N, K)) return CDL_ERR_WORKSPACE;
    int rc = check_device();
    if (rc != CDL_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    if (K == 0) {
        if (out_type == CDL_F32) fill_bias_kernel<<<sms * 4, 256, 0, st>>>(static_cast<float *>(out), ldo, M, N, bias);
        else if (out_type == CDL_BF16) fill_bias_kernel<<<sms * 4, 256, 0, st>>>(static_cast<__nv_bfloat16 *>(out), ldo, M, N, bias);
        else fill_bias_kernel<<<sms * 4, 256, 0, st>>>(static_cast<__half *>(out), ldo, M, N, bias);
        return cudaGetLastError() == cudaSuccess ? CDL_OK : CDL_ERR_LAUNCH;
    }
    Fp8Plan plan;
    if (!make_plan(M, N, K, &plan)) return CDL_ERR_ARG;
    if (plan.rows)
        return launch_fp8_rows(A, lda, a_scale, B, ldb, b_scale, b_mode == CDL_FP8_ROWS, M, N, K, out, ldo, out_type, bias, st);
    Fp8Params P;
    memset(&P, 0, sizeof P);
    P.M = M;
    P.N = N;
    P.KB = (int)(((int64_t)K + 127) / 128);
    const bool bvec = b_mode == CDL_FP8_ROWS;
    P.nb = bvec ? N : (int)(((int64_t)N + 127) / 128);
    P.sa = a_scale;
    P.sb = b_scale;
    P.bias = bias;
    P.out = out;
    P.ldo = ldo;
    P.status = static_cast<int *>(ws);
    const bool pair = plan.pair;
    P.tiles_i = plan.tiles_i;
    P.tiles_j = plan.tiles_j;
    P.splits = plan.splits;
    P.whole = plan.whole;
    P.ranges = plan.ranges;
    P.run = plan.run;
    P.part = reinterpret_cast<float *>(static_cast<char *>(ws) + kStatusBytes);
    const int esz = type_bytes(out_type);
    // (a TMA store fills the last 16-byte unit of a row with zeros beyond N: rows that do not end on one are stored directly)
    P.out_tma = P.splits == 1 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0 && (ldo * esz) % 16 == 0 && ((int64_t)N * esz) % 16 == 0;
    CUtensorMap map_a, map_b, map_o;
    bool ok = encode_map_2d(&map_a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, A, (uint64_t)K, (uint64_t)M, (uint64_t)lda, 128) &&
              encode_map_2d(&map_b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, B, (uint64_t)K, (uint64_t)N, (uint64_t)ldb, 128);
    map_o = map_a;
    if (P.out_tma)
        ok = ok && encode_map_2d(&map_o, out_type == CDL_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                                             : (out_type == CDL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16),
                                 esz, out, (uint64_t)N, (uint64_t)M, (uint64_t)(ldo * esz), 32, 64);
    if (!ok) return CDL_ERR_LAUNCH;
    static bool attr_set[64];
    static int pair_slots[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.attrs = at;
    if (!attr_set[dev]) {
        for (int t = 0; t < 3; ++t)
            for (int v = 0; v < 8; ++v)
                if (cudaFuncSetAttribute(variant(t, (v & 1) != 0, (v & 2) != 0, (v & 4) != 0), cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes((v & 2) != 0)) != cudaSuccess) {
                    (void)cudaGetLastError();
                    return CDL_ERR_LAUNCH;
                }
        // the pair kernels' shares must fit what a block is launched with, or an epilogue warpgroup would wait for good
        for (int t = 0; t < 3; ++t)
            for (int v = 0; v < 4; ++v) {
                cudaFuncAttributes fa;
                if (cudaFuncGetAttributes(&fa, variant(t, true, (v & 1) != 0, (v & 2) != 0)) != cudaSuccess || fa.numRegs < kRegsLaunch) {
                    (void)cudaGetLastError();
                    return CDL_ERR_LAUNCH;
                }
            }
        at[1].val.clusterDim.x = 2;
        cfg.gridDim = dim3(2u * (unsigned)(sms / 2));
        cfg.dynamicSmemBytes = smem_bytes(false);
        cfg.attrs = at + 1;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, variant(CDL_BF16, true, false, false), &cfg) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();
            n = sms / 2;
        }
        pair_slots[dev] = n < sms / 2 ? n : sms / 2;
        attr_set[dev] = true;
    }
    // (a CTA has one run at most: as many are started as there are runs, should the device have fewer places)
    const int64_t places = pair ? pair_slots[dev] : (P.splits > 1 ? P.whole : sms);
    P.slots = (int)(P.whole < places ? P.whole : places);
    if (P.slots < P.ranges) P.slots = P.ranges;
    at[1].val.clusterDim.x = pair ? 2u : (unsigned)P.splits;
    cfg.attrs = at;
    cfg.gridDim = dim3((pair ? 2u : (unsigned)P.splits) * (unsigned)P.slots);
    cfg.dynamicSmemBytes = smem_bytes(bvec);
    cfg.stream = st;
    cfg.numAttrs = pair || P.splits > 1 ? 2 : 1;
    void *args[4] = {&map_a, &map_b, &map_o, &P};
    if (cudaLaunchKernelExC(&cfg, variant(out_type, pair, bvec, P.ranges > 0), args) != cudaSuccess) {
        (void)cudaGetLastError();
        return CDL_ERR_LAUNCH;
    }
    if (P.ranges > 0) {
        if (out_type == CDL_F32) return launch_sum<float>(pair, P, st);
        return out_type == CDL_BF16 ? launch_sum<__nv_bfloat16>(pair, P, st) : launch_sum<__half>(pair, P, st);
    }
    return CDL_OK;
}
