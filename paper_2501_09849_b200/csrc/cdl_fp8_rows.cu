// Block-scaled 8-bit product for one to four rows of A (single tokens): out[m,n] = sum_kb sa sb sum_k A[m,k] B[n,k].
//
// Bound by reading B once.  The tensor-core form for many rows hands over every 128 reduced entries between four kinds of warps,
// which for one tile row is all latency (4096 x 4096, four rows: 9.5 us for 16.8 MB; here 5.6).  Here a warp takes eight rows of
// B and multiplies a block of 128 entries by two m16n8k32 matrix instructions: rows 0..7 of their first operand are the eight
// rows' first 64 entries, rows 8..15 their other 64, and the columns of the second operand are the rows of A, once for either half.
// (Any order of the reduced entries will do as long as both operands have the same, so a lane's part is 16 consecutive codes.)
// Unpacking the codes and multiplying in binary32 instead took 13.5 codes per cycle and SM: 48828 x 4096 53 us, now 38.5, one row.
// Sums are binary32; the two scales multiply a block's sum.
//
// B comes through shared memory by 16-byte asynchronous copies, two steps of 512 entries ahead, 128 KB per SM on their way.  A lane
// fetches what it reads itself: no barrier, and any length.  (Bulk copies of 1 KB per row cost 70 cycles each and ended at 3.8 TB/s.)
// The warps of a CTA share the reduced dimension when there are few rows of B, and are added in their order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_wait.cuh"

namespace cdl {
namespace {

constexpr int kRowsPerWarp = 8;
constexpr int kWarps = 16;              // most warps of a CTA
constexpr int kStep = 512;              // entries of the reduced dimension that a warp fetches together: four blocks
constexpr int kSlots = 3;               // ... of which as many are on their way or in use
constexpr int kSlotBytes = kRowsPerWarp * kStep;
constexpr int kWarpSmem = kSlots * kSlotBytes;

struct RowsParams {
    const unsigned char *A, *B;
    long long lda, ldb;
    const float *sa, *sb, *bias;
    int b_rows;                 // scales of B per k-block change from row to row
    int nb;                     // scales of a k-block of B
    int M, N, K;
    int slices;                 // warps of a CTA that share the reduced dimension (a power of two)
    int passes;                 // groups of rows a warp takes in turn
    void *out;
    long long ldo;
};

// D += A B, 16 x 32 times 32 x 8 codes, binary32 sums
__device__ __forceinline__ void mma_codes(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the first `live` of sixteen codes, zeros behind them
__device__ __forceinline__ uint4 keep_codes(uint4 q, int live)
{
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = live - 4 * i;
        w[i] = n >= 4 ? w[i] : (n <= 0 ? 0u : w[i] & ((1u << (8 * n)) - 1u));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// sixteen bytes from global to shared memory, asynchronously, of which `live` exist; zeros behind them
__device__ __forceinline__ void copy16_async(uint32_t dst, const unsigned char *src, int live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(max(0, min(16, live))) : "memory");
}
template <int M, typename T>
__global__ void __launch_bounds__(32 * kWarps, 1)
fp8_rows_kernel(RowsParams P)
{
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ float sums[kWarps][2][32];
    constexpr int kPad = M <= 2 ? 2 : 4;               // columns of the product for each half of a block
    constexpr int kBlocks = kStep / 128;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    follow_previous();
    const int warps = (int)(blockDim.x >> 5), groups = warps / P.slices, slice = warp % P.slices, group = warp / P.slices;
    const int steps = (P.K + kStep - 1) / kStep;
    const int j0 = (int)((long long)steps * slice / P.slices), count = (int)((long long)steps * (slice + 1) / P.slices) - j0;
    const long long first = ((long long)blockIdx.x * groups + group) * kRowsPerWarp, step = (long long)gridDim.x * groups * kRowsPerWarp;
    const int passes = first < P.N ? (int)((P.N - 1 - first) / step) + 1 : 0;
    // Each warp begins at another step of its slice: with a row pitch that is a power of two all warps would otherwise read the same
    // few memory channels at the same time.
    const int turn = count > 0 ? ((int)blockIdx.x * warps + warp) % count : 0;
    // This lane's part of a product: row g of B in both halves of A's operand, entries 16 t .. 16 t + 15 of either half; and, as
    // the other operand's column g, row g % kPad of A and the half g / kPad.  Of the sums, {row g, columns 2 t and 2 t + 1} of
    // the half that the columns belong to.
    const int g = lane >> 2, t = lane & 3;
    const int m_in = g % kPad, k_in = g / kPad * 64 + t * 16;
    const bool has_row = g < 2 * kPad && m_in < M;
    const unsigned char *x_in = P.A + (long long)(has_row ? m_in : 0) * P.lda;
    const int m0 = 2 * (t % (kPad / 2)), m_own = m0 < M ? m0 : M - 1;
    const bool second = t / (kPad / 2) != 0;
    auto row_of = [&](int pass) {
        const long long n = first + pass * step + g;
        return n < P.N ? n : P.N - 1;
    };
    // A lane fetches what it will read itself, so that nothing is waited for but its own copies.
    const uint32_t mine = smem_u32(ring) + (uint32_t)(warp * kWarpSmem + lane * 16);
    int ask_pass = 0, ask_j = 0, ask_slot = 0;
    auto ask = [&] {
        if (count > 0 && ask_pass < passes) {
            const int k = (j0 + (ask_j + turn < count ? ask_j + turn : ask_j + turn - count)) * kStep + t * 16;
            const unsigned char *src = P.B + row_of(ask_pass) * P.ldb + k;
#pragma unroll
            for (int i = 0; i < 2 * kBlocks; ++i)
                copy16_async(mine + (uint32_t)(ask_slot * kSlotBytes + i * 512), k + i * 64 < P.K ? src + i * 64 : P.B, P.K - k - i * 64);
            ask_slot = ask_slot + 1 == kSlots ? 0 : ask_slot + 1;
            if (++ask_j == count) {
                ask_j = 0;
                ++ask_pass;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int s = 0; s < kSlots - 1; ++s) ask();
    int slot = 0;
    for (int pass = 0; pass < P.passes; ++pass) {
        const float *sb = P.sb + (P.b_rows ? row_of(pass) : row_of(pass) >> 7);
        float acc0 = 0.0f, acc1 = 0.0f;
        for (int j = 0; j < (pass < passes ? count : 0); ++j) {
            const int k0 = (j0 + (j + turn < count ? j + turn : j + turn - count)) * kStep;
            ask();
            // what the blocks need of A and of the scales is on its way while the codes are waited for (behind the end: the last
            // block's again, so that no load waits for a branch)
            uint4 x[kBlocks];
            float s[kBlocks], s0[kBlocks], s1[kBlocks];
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const int kb = min(k0 + i * 128, P.K - 1) >> 7;
                x[i] = *reinterpret_cast<const uint4 *>(x_in + min(k0 + i * 128 + k_in, (P.K - 1) & ~15));
                s[i] = sb[(long long)kb * P.nb];
                s0[i] = P.sa[(long long)kb * M + m_own];
                s1[i] = P.sa[(long long)kb * M + (m0 + 1 < M ? m0 + 1 : m_own)];
            }
            asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 1) : "memory");
            const uint32_t at = mine + (uint32_t)(slot * kSlotBytes);
            slot = slot + 1 == kSlots ? 0 : slot + 1;
            if (k0 + kStep > P.K) {                      // nothing behind the row's end counts (of B there are zeros)
#pragma unroll
                for (int i = 0; i < kBlocks; ++i) {
                    x[i] = keep_codes(x[i], P.K - k0 - i * 128 - k_in);
                    if (k0 + i * 128 >= P.K) s[i] = s0[i] = s1[i] = 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const uint4 q0 = lds_u128(at + (uint32_t)(i * 1024)), q1 = lds_u128(at + (uint32_t)(i * 1024 + 512));
                if (!has_row) x[i] = make_uint4(0u, 0u, 0u, 0u);
                float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                mma_codes(c, q0.x, q1.x, q0.y, q1.y, x[i].x, x[i].y);
                mma_codes(c, q0.z, q1.z, q0.w, q1.w, x[i].z, x[i].w);
                acc0 = fmaf(second ? c[2] : c[0], s[i] * s0[i], acc0);
                acc1 = fmaf(second ? c[3] : c[1], s[i] * s1[i], acc1);
            }
        }
        acc0 += __shfl_xor_sync(0xffffffffu, acc0, kPad / 2);        // the two halves
        acc1 += __shfl_xor_sync(0xffffffffu, acc1, kPad / 2);
        if (P.slices > 1) {
            sums[warp][0][lane] = acc0;
            sums[warp][1][lane] = acc1;
            __syncthreads();
            if (slice == 0)
                for (int i = 1; i < P.slices; ++i) {
                    acc0 += sums[warp + i][0][lane];
                    acc1 += sums[warp + i][1][lane];
                }
            __syncthreads();
        }
        const long long n = first + pass * step + g;
        if (slice == 0 && !second && t < kPad / 2 && n < P.N) {
            T *o = static_cast<T *>(P.out) + n;
            const float b = P.bias != nullptr ? P.bias[n] : 0.0f;
            if (m0 < M) o[(long long)m0 * P.ldo] = from_f32<T>(acc0 + b);
            if (m0 + 1 < M) o[(long long)(m0 + 1) * P.ldo] = from_f32<T>(acc1 + b);
        }
    }
}

typedef void (*RowsKernel)(RowsParams);
template <typename T>
RowsKernel variant(int M)
{
    return M == 1 ? &fp8_rows_kernel<1, T> : (M == 2 ? &fp8_rows_kernel<2, T> : (M == 3 ? &fp8_rows_kernel<3, T> : &fp8_rows_kernel<4, T>));
}
RowsKernel variant(int M, int type)
{
    return type == CDL_F32 ? variant<float>(M) : (type == CDL_BF16 ? variant<__nv_bfloat16>(M) : variant<__half>(M));
}

}  // namespace

// Warps of a CTA, and how many of them share the reduced dimension: what takes the shortest time.  In cycles: the 4 KB steps of w
// warps take 140 w + 1320 (measured with 8 and 16 of them; few warps wait for memory), a pass 1500 besides for the sums over
// lanes and slices.  Planned for a B200's 148 SMs.
Fp8RowsPlan plan_fp8_rows(int N, int K)
{
    constexpr long long kPlanSms = 148;
    const long long units = ((long long)N + kRowsPerWarp - 1) / kRowsPerWarp, steps = ((long long)K + kStep - 1) / kStep;
    Fp8RowsPlan best{0, 0, 0, 0};
    long long least = 0;
    for (int w = 2; w <= kWarps; w *= 2)
        for (int slices = 1; slices <= w && (slices == 1 || slices <= steps); slices *= 2) {
            const long long n = (units + w / slices - 1) / (w / slices);
            const long long time = (n + kPlanSms - 1) / kPlanSms * ((steps + slices - 1) / slices * (140 * w + 1320) + 1500);
            if (best.warps == 0 || time < least) {
                least = time;
                best = Fp8RowsPlan{w, slices, n, 2500 + time * 10 / 19};
            }
        }
    return best;
}

int launch_fp8_rows(const void *A, long long lda, const float *sa, const void *B, long long ldb, const float *sb, bool b_rows, int M, int N,
                    int K, void *out, long long ldo, int out_type, const float *bias, cudaStream_t stream)
{
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    RowsParams P{static_cast<const unsigned char *>(A), static_cast<const unsigned char *>(B), lda, ldb, sa, sb, bias,
                 b_rows ? 1 : 0, b_rows ? N : (int)(((long long)N + 127) / 128), M, N, K, 1, 1, out, ldo};
    const Fp8RowsPlan plan = plan_fp8_rows(N, K);
    P.slices = plan.slices;
    const int warps = plan.warps;
    const long long blocks = plan.blocks;
    const int grid = (int)(blocks < sms ? blocks : sms);
    P.passes = (int)((blocks + grid - 1) / grid);
    static bool attr_set[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    if (!attr_set[dev]) {
        for (int m = 1; m <= kFewRowsFp8; ++m)
            for (int t = 0; t < 3; ++t)
                if (cudaFuncSetAttribute(variant(m, t), cudaFuncAttributeMaxDynamicSharedMemorySize, kWarps * kWarpSmem) != cudaSuccess) {
                    (void)cudaGetLastError();
                    return CDL_ERR_LAUNCH;
                }
        attr_set[dev] = true;
    }
    return launch_following(variant(M, out_type), dim3((unsigned)grid), dim3(32u * (unsigned)warps), (size_t)(warps * kWarpSmem), stream, P);
}

}  // namespace cdl
