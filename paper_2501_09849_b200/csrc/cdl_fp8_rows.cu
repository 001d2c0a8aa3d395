// Block-scaled 8-bit product for one or two rows of A (single tokens): out[m,n] = sum_kb sa sb sum_k A[m,k] B[n,k].
//
// Bound by reading B once.  The tensor-core form hands over every 128 reduced entries between four kinds of warps, which for
// one tile row is all latency (4096 x 4096, one row: 9.6 us for 16.8 MB); here a warp streams four rows of B through its
// ring in shared memory, 16 codes per lane at a time, and multiplies in binary32.  The entries of A that a lane meets are
// the same for its four rows and converted once.  Codes become binary32 through binary16 pairs (exact); a lane's 16
// entries lie in one block of 128, so the two scales multiply its partial sum once.  The warps of a CTA share the reduced
// dimension when there are few rows of B, and are added in their order.  From three rows on the conversions and products
// of this form take longer than the hand-overs of the other (three rows: 16.3 us against 9.6).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_row_ring.cuh"

namespace cdl {
namespace {

constexpr int kRowsPerWarp = kRingRows;
constexpr int kWarps = 16;
using Ring = RowRing<kWarps, 1024>;
constexpr int kRingBytes = Ring::kRingBytes;

struct RowsParams {
    const unsigned char *A, *B;
    long long lda, ldb;
    const float *sa, *sb, *bias;
    int b_rows;                 // scales of B per k-block change from row to row
    int nb;                     // scales of a k-block of B
    int M, N, K;
    int slices;                 // warps of a CTA that share the reduced dimension (a power of two)
    int passes;                 // groups of rows a warp takes in turn
    int *status;
    void *out;
    long long ldo;
};

// sixteen codes -> binary32
__device__ __forceinline__ void codes16(uint4 q, float (&v)[16])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t lo, hi;
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
            "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
            : "=r"(lo), "=r"(hi)
            : "r"(w[i]));
        unpack2(lo, v[4 * i], v[4 * i + 1], __half());
        unpack2(hi, v[4 * i + 2], v[4 * i + 3], __half());
    }
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

template <int M, typename T>
__global__ void __launch_bounds__(32 * kWarps, 1)
fp8_rows_kernel(RowsParams P)
{
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) unsigned long long bars[kWarps * kRingSlots];
    __shared__ float sums[kWarps][kRowsPerWarp * M];
    __shared__ int abort_s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int i = 0; i < kWarps * kRingSlots; ++i) mbar_init(smem_u32(&bars[i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    follow_previous();
    const int groups = kWarps / P.slices, slice = warp % P.slices, group = warp / P.slices;
    // a slice is a run of whole steps of 512 entries (16 per lane)
    const int steps = (P.K + 511) / 512;
    const int k0 = (int)((long long)steps * slice / P.slices) * 512, k1 = min(P.K, (int)((long long)steps * (slice + 1) / P.slices) * 512);
    Ring R;
    R.base = P.B;
    R.pitch = P.ldb;
    R.first = ((long long)blockIdx.x * groups + group) * kRowsPerWarp;
    R.step = (long long)gridDim.x * groups * kRowsPerWarp;
    R.rows = P.N;
    R.groups = R.first < P.N ? (int)((P.N - 1 - R.first) / R.step) + 1 : 0;
    R.from = k0;
    R.to = k1;
    R.smem = smem_u32(ring) + (uint32_t)(warp * kRingSlots * kRingRows * kRingBytes);
    R.bar = smem_u32(&bars[warp * kRingSlots]);
    R.abort_flag = &abort_s;
    R.lane = lane;
    R.turn = (int)blockIdx.x * kWarps + warp;
    R.start();
    bool failed = false;
    for (int pass = 0; pass < P.passes; ++pass) {
        const long long n0 = R.first + pass * R.step;
        float acc[M][kRowsPerWarp];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < kRowsPerWarp; ++r) acc[m][r] = 0.0f;
        for (int kp = k0 + R.turn, left = pass < R.groups ? k1 - k0 : 0; left > 0 && !failed; left -= kRingBytes, kp = R.after(kp)) {
            uint32_t piece;
            if (!R.take(piece)) {
                failed = true;
                break;
            }
            for (int k = kp + lane * 16; k < min(kp + kRingBytes, k1); k += 512) {
                const int kb = k >> 7, live = P.K - k;
                float s[kRowsPerWarp];
#pragma unroll
                for (int r = 0; r < kRowsPerWarp; ++r) {
                    const long long n = n0 + r < P.N ? n0 + r : P.N - 1;
                    s[r] = __ldg(P.sb + (long long)kb * P.nb + (P.b_rows ? n : n >> 7));
                }
                float a[M][16], sa[M];
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    uint4 c = __ldg(reinterpret_cast<const uint4 *>(P.A + (long long)m * P.lda + k));
                    if (live < 16) c = keep_codes(c, live);
                    codes16(c, a[m]);
                    sa[m] = __ldg(P.sa + (long long)kb * M + m);
                }
#pragma unroll
                for (int r = 0; r < kRowsPerWarp; ++r) {
                    uint4 q = lds_u128(piece + (uint32_t)(r * kRingBytes + (k - kp)));
                    if (live < 16) q = keep_codes(q, live);
                    float v[16];
                    codes16(q, v);
#pragma unroll
                    for (int m = 0; m < M; ++m) {
                        float p0 = 0.0f, p1 = 0.0f;
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            p0 = fmaf(a[m][i], v[i], p0);
                            p1 = fmaf(a[m][i + 1], v[i + 1], p1);
                        }
                        acc[m][r] = fmaf(p0 + p1, sa[m] * s[r], acc[m][r]);
                    }
                }
            }
            R.done();
        }
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < kRowsPerWarp; ++r) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) acc[m][r] += __shfl_xor_sync(0xffffffffu, acc[m][r], o);
            }
        if (P.slices > 1) {
            if (lane == 0)
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int r = 0; r < kRowsPerWarp; ++r) sums[warp][m * kRowsPerWarp + r] = acc[m][r];
            __syncthreads();
            if (slice == 0 && lane == 0)
                for (int s = 1; s < P.slices; ++s)
#pragma unroll
                    for (int m = 0; m < M; ++m)
#pragma unroll
                        for (int r = 0; r < kRowsPerWarp; ++r) acc[m][r] += sums[warp + s][m * kRowsPerWarp + r];
            __syncthreads();
        }
        if (slice == 0 && lane == 0)
#pragma unroll
            for (int r = 0; r < kRowsPerWarp; ++r)
                if (n0 + r < P.N)
#pragma unroll
                    for (int m = 0; m < M; ++m)
                        static_cast<T *>(P.out)[(long long)m * P.ldo + n0 + r] = from_f32<T>(acc[m][r] + (P.bias != nullptr ? __ldg(P.bias + n0 + r) : 0.0f));
    }
    if (failed) {
        abort_s = 1;
        if (lane == 0) record_timeout(P.status);
        R.drain();
    }
}

typedef void (*RowsKernel)(RowsParams);
template <typename T>
RowsKernel variant(int M) { return M == 1 ? &fp8_rows_kernel<1, T> : &fp8_rows_kernel<2, T>; }
RowsKernel variant(int M, int type)
{
    return type == CDL_F32 ? variant<float>(M) : (type == CDL_BF16 ? variant<__nv_bfloat16>(M) : variant<__half>(M));
}

}  // namespace

int launch_fp8_rows(const void *A, long long lda, const float *sa, const void *B, long long ldb, const float *sb, bool b_rows, int M, int N,
                    int K, void *out, long long ldo, int out_type, const float *bias, int *status, cudaStream_t stream)
{
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    RowsParams P{static_cast<const unsigned char *>(A), static_cast<const unsigned char *>(B), lda, ldb, sa, sb, bias,
                 b_rows ? 1 : 0, b_rows ? N : (int)(((long long)N + 127) / 128), M, N, K, 1, 1, status, out, ldo};
    const long long units = ((long long)N + kRowsPerWarp - 1) / kRowsPerWarp;
    // the warps of the device share out what there is: groups of four rows first, then steps of the reduced dimension
    while (P.slices < kWarps && (long long)P.slices * 512 < K && units * P.slices * 2 <= (long long)sms * kWarps) P.slices *= 2;
    const long long per_block = kWarps / P.slices, blocks = (units + per_block - 1) / per_block;
    const int grid = (int)(blocks < sms ? blocks : sms);
    P.passes = (int)((blocks + grid - 1) / grid);
    static bool attr_set[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    if (!attr_set[dev]) {
        for (int m = 1; m <= 2; ++m)
            for (int t = 0; t < 3; ++t)
                if (cudaFuncSetAttribute(variant(m, t), cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem) != cudaSuccess) {
                    (void)cudaGetLastError();
                    return CDL_ERR_LAUNCH;
                }
        attr_set[dev] = true;
    }
    return launch_following(variant(M, out_type), dim3((unsigned)grid), dim3(32 * kWarps), kRingSmem, stream, P);
}

}  // namespace cdl
