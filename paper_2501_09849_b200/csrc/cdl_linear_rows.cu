// 16-bit product for one to eight rows of A (single tokens): z[m,n] = sum_k A[m,k] W[n,k], and the layer's epilogue.
//
// Bound by reading W once.  A warp takes sixteen rows of W and multiplies 32 reduced entries by two m16n8k16 matrix instructions whose
// first operand is W and whose eight columns are the rows of A: a lane's part of either is eight consecutive entries of a row (any order
// of the reduced entries will do as long as both operands have the same).  The instructions' binary32 sums are cut off, not rounded, so they
// are added up after 512 entries (in one go 8 x 4655 x 60000 was off by 8e-6 of the norm).
// W comes through shared memory by 16-byte asynchronous copies, kSlots - 1 steps of 128 entries ahead; a lane fetches what it reads
// itself: no barrier, and any length.  The warps of a CTA share the reduced dimension when there are few rows of W, and are added in
// their order.
// 1 x 4096 x 4096 7.0 us (4.8 TB/s out of L2 and memory), with bias and residual 7.4; 8 rows 7.9, the tiles' form 10.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cdl_internal.h"
#include "cdl_linear.cuh"
#include "cdl_lowp.cuh"
#include "cdl_wait.cuh"

namespace cdl {
namespace {

constexpr int kRowsPerWarp = 16;
constexpr int kWarps = 16;              // most warps of a CTA
constexpr int kStep = 128;              // entries of the reduced dimension that a warp fetches together
constexpr int kPieces = kStep / 32;     // ... in pieces of 32: four lanes of eight entries
constexpr int kSegment = 4;             // steps that the matrix instructions sum
constexpr int kSlots = 3;               // steps on their way or in use
constexpr int kSlotBytes = kRowsPerWarp * kStep * 2;
constexpr int kWarpSmem = kSlots * kSlotBytes;

struct RowsParams {
    const unsigned short *A, *W;
    long long lda, ldw;
    int M, N, K;
    int slices;                 // warps of a CTA that share the reduced dimension (a power of two)
    int passes;                 // groups of rows a warp takes in turn
    float *part;
    LinearOut out;
};

template <typename T>
__device__ __forceinline__ void mma_16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (__is_same(T, __nv_bfloat16))
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the first `live` of eight entries, zeros behind them
__device__ __forceinline__ uint4 keep_entries(uint4 q, int live)
{
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = live - 2 * i;
        w[i] = n >= 2 ? w[i] : (n <= 0 ? 0u : w[i] & 0xffffu);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// sixteen bytes from global to shared memory, asynchronously, of which `live` exist; zeros behind them
__device__ __forceinline__ void copy16_async(uint32_t dst, const void *src, int live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(max(0, min(16, live))) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(32 * kWarps, 1)
linear_rows_kernel(RowsParams P)
{
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ float sums[kWarps][4][32];
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
    // This lane's part of a product: rows g and g + 8 of W, entries 8 t .. 8 t + 7 of a piece; as the other operand's column g, row g
    // of A.  Of the sums, {row g, row g + 8 of W} x {rows 2 t, 2 t + 1 of A}.
    const int g = lane >> 2, t = lane & 3;
    const bool has_row = g < P.M;
    const unsigned short *x_in = P.A + (long long)(has_row ? g : 0) * P.lda;
    auto row_of = [&](int pass, int h) {
        const long long n = first + pass * step + g + 8 * h;
        return n < P.N ? n : P.N - 1;
    };
    const uint32_t mine = smem_u32(ring) + (uint32_t)(warp * kWarpSmem + lane * 16);
    int ask_pass = 0, ask_j = 0, ask_slot = 0;
    auto ask = [&] {
        if (count > 0 && ask_pass < passes) {
            const int k = (j0 + (ask_j + turn < count ? ask_j + turn : ask_j + turn - count)) * kStep + t * 8;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned short *src = P.W + row_of(ask_pass, h) * P.ldw + k;
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
                    copy16_async(mine + (uint32_t)(ask_slot * kSlotBytes + (h * kPieces + i) * 512), k + i * 32 < P.K ? src + i * 32 : P.W, 2 * (P.K - k - i * 32));
            }
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
        float c[4] = {0.0f, 0.0f, 0.0f, 0.0f}, part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        // what the epilogue reads is on its way before the first entries of W are
        LinearIn<1> in[4];
        float bias[4];
        const bool ends = slice == 0 && P.part == nullptr;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long n = first + pass * step + g + 8 * (i >> 1);
            const int m = 2 * t + (i & 1);
            bias[i] = 0.0f;
            if (ends && n < P.N && m < P.M) {
                linear_fetch<1>(P.out, m, (int)n, 1, in[i]);
                if (P.out.bias != nullptr) bias[i] = P.out.bias[n];
            }
        }
        for (int j = 0; j < (pass < passes ? count : 0); ++j) {
            const int k0 = (j0 + (j + turn < count ? j + turn : j + turn - count)) * kStep;
            ask();
            // A's entries are on their way while W's are waited for (behind the end: a unit that exists, cleared below)
            uint4 x[kPieces];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) x[i] = *reinterpret_cast<const uint4 *>(x_in + min(k0 + i * 32 + t * 8, (P.K - 1) & ~7));
            asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 1) : "memory");
            const uint32_t at = mine + (uint32_t)(slot * kSlotBytes);
            slot = slot + 1 == kSlots ? 0 : slot + 1;
            if (k0 + kStep > P.K)
#pragma unroll
                for (int i = 0; i < kPieces; ++i) x[i] = keep_entries(x[i], P.K - k0 - i * 32 - t * 8);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint4 q0 = lds_u128(at + (uint32_t)(i * 512)), q1 = lds_u128(at + (uint32_t)((kPieces + i) * 512));
                if (!has_row) x[i] = make_uint4(0u, 0u, 0u, 0u);
                mma_16<T>(part, q0.x, q1.x, q0.y, q1.y, x[i].x, x[i].y);
                mma_16<T>(part, q0.z, q1.z, q0.w, q1.w, x[i].z, x[i].w);
            }
            if (j % kSegment == kSegment - 1 || j == count - 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    c[i] += part[i];
                    part[i] = 0.0f;
                }
        }
        if (P.slices > 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[warp][i][lane] = c[i];
            __syncthreads();
            if (slice == 0)
                for (int s = 1; s < P.slices; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) c[i] += sums[warp + s][i][lane];
            __syncthreads();
        }
        if (slice == 0)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const long long n = first + pass * step + g + 8 * (i >> 1);
                const int m = 2 * t + (i & 1);
                if (n >= P.N || m >= P.M) continue;
                if (P.part != nullptr) {
                    P.part[((n >> 8) * 8 + m) * 256 + (n & 255)] = c[i];
                    continue;
                }
                float v[1] = {c[i] + bias[i]};
                linear_store<1>(P.out, m, (int)n, 1, in[i], v);
            }
    }
}

}  // namespace

// Warps of a CTA, and how many of them share the reduced dimension: what takes the shortest time.  In cycles: the 4 KB steps of w
// warps take 140 w + 1320, a pass 1500 besides for the sums over slices and the epilogue.  Planned for a B200's 148 SMs.
LinearRowsPlan plan_linear_rows(int N, int K)
{
    constexpr long long kPlanSms = 148;
    const long long units = ((long long)N + kRowsPerWarp - 1) / kRowsPerWarp, steps = ((long long)K + kStep - 1) / kStep;
    LinearRowsPlan best{0, 0, 0, 0};
    long long least = 0;
    for (int w = 2; w <= kWarps; w *= 2)
        for (int slices = 1; slices <= w && (slices == 1 || slices <= steps); slices *= 2) {
            const long long n = (units + w / slices - 1) / (w / slices);
            const long long time = (n + kPlanSms - 1) / kPlanSms * ((steps + slices - 1) / slices * (140 * w + 1320) + 1500);
            if (best.warps == 0 || time < least) {
                least = time;
                best = LinearRowsPlan{w, slices, n, 2500 + time * 10 / 19};
            }
        }
    return best;
}

int launch_linear_rows(const void *A, long long lda, const void *W, long long ldw, int type, int M, int N, int K, const LinearOut &out, float *part,
                       cudaStream_t stream)
{
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    RowsParams P{static_cast<const unsigned short *>(A), static_cast<const unsigned short *>(W), lda, ldw, M, N, K, 1, 1, part, out};
    const LinearRowsPlan plan = plan_linear_rows(N, K);
    P.slices = plan.slices;
    const int grid = (int)(plan.blocks < sms ? plan.blocks : sms);
    P.passes = (int)((plan.blocks + grid - 1) / grid);
    void (*const kernel)(RowsParams) = type == CDL_BF16 ? &linear_rows_kernel<__nv_bfloat16> : &linear_rows_kernel<__half>;
    static bool attr_set[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    if (!attr_set[dev]) {
        if (cudaFuncSetAttribute(&linear_rows_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWarps * kWarpSmem) != cudaSuccess ||
            cudaFuncSetAttribute(&linear_rows_kernel<__half>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWarps * kWarpSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return CDL_ERR_LAUNCH;
        }
        attr_set[dev] = true;
    }
    return launch_following(kernel, dim3((unsigned)grid), dim3(32u * (unsigned)plan.warps), (size_t)(plan.warps * kWarpSmem), stream, P);
}

}  // namespace cdl
