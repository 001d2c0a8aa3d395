// Statistics of the logits H W^T for one or two rows of H (scoring and decoding): per row and CTA the maximum and the sum of
// exponentials over the words that the CTA has seen, and the label's logit.
//
// Bound by reading W once (32000 x 4096 bf16: 262 MB).  Tiles of the tensor-core form spread 125 tiles over 148 SMs; here the
// warps of one CTA per SM take four words at a time in turn, streamed through their rings in shared memory, and multiply in
// binary32 (a 16-bit entry is unpacked once for all rows).  Logits exist in registers only; a warp keeps its running
// maximum and sum, a CTA joins its warps', and the same small kernel as for the tensor-core form joins the CTAs'.  One row:
// 44 us (tensor-core form 55); two rows 53, where the products begin to count; from three rows on the other form is taken.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_row_ring.cuh"
#include "cdl_softmax.cuh"

namespace cdl {
namespace {

constexpr int kWords = kRingRows;      // words a warp works on at a time
constexpr int kWarps = 8;
using Ring = RowRing<kWarps, 2048>;
constexpr unsigned kRingBytes = Ring::kRingBytes;
constexpr int kPieceEntries = (int)kRingBytes / 2;

template <int R, typename T>
__global__ void __launch_bounds__(32 * kWarps, 1)
loss_rows_kernel(const T *H, long long ldh, const T *W, long long ldw, const long long *labels,
                 int rows, int V, int D, float2 *part, int parts, float *target, int *status)
{
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) unsigned long long bars[kWarps * kRingSlots];
    __shared__ float2 sh[kWarps][R];
    __shared__ int abort_s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int i = 0; i < kWarps * kRingSlots; ++i) mbar_init(smem_u32(&bars[i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    follow_previous();
    Ring ringw;
    ringw.base = reinterpret_cast<const unsigned char *>(W);
    ringw.pitch = ldw * 2;
    ringw.first = ((long long)blockIdx.x * kWarps + warp) * kWords;
    ringw.step = (long long)gridDim.x * kWarps * kWords;
    ringw.rows = V;
    ringw.groups = ringw.first < V ? (int)((V - 1 - ringw.first) / ringw.step) + 1 : 0;
    ringw.bytes = (unsigned)D * 2u;
    ringw.smem = smem_u32(ring) + (uint32_t)(warp * kRingSlots * kRingRows) * kRingBytes;
    ringw.bar = smem_u32(&bars[warp * kRingSlots]);
    ringw.abort_flag = &abort_s;
    ringw.lane = lane;
    ringw.turn = blockIdx.x * kWarps + (unsigned)warp;
    ringw.start();
    bool failed = false;
    float m[R], s[R];
    long long label[R];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        m[t] = -INFINITY;
        s[t] = 0.0f;
        label[t] = t < rows ? labels[t] : -1;
    }
    for (int pass = 0; pass < ringw.groups && !failed; ++pass) {
        const long long v0 = ringw.first + pass * ringw.step;
        float acc[R][kWords];
#pragma unroll
        for (int t = 0; t < R; ++t)
#pragma unroll
            for (int w = 0; w < kWords; ++w) acc[t][w] = 0.0f;
        unsigned at = ringw.turn;
        for (unsigned left = ringw.pieces(); left > 0; --left, at = ringw.after(at)) {
            const int dp = (int)(at / 2u);
            uint32_t piece;
            if (!ringw.take(piece)) {
                failed = true;
                break;
            }
            for (int d = dp + lane * 8; d < min(dp + kPieceEntries, D); d += 256) {
                const int live = D - d;                  // (what lies behind a row's end is not part of it)
                float x[kWords][8];
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    const uint4 u = lds_u128(piece + (uint32_t)w * kRingBytes + (uint32_t)(d - dp) * 2u);
                    unpack2(u.x, x[w][0], x[w][1], T());
                    unpack2(u.y, x[w][2], x[w][3], T());
                    unpack2(u.z, x[w][4], x[w][5], T());
                    unpack2(u.w, x[w][6], x[w][7], T());
                    if (live < 8)
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[w][i] = i < live ? x[w][i] : 0.0f;
                }
#pragma unroll
                for (int t = 0; t < R; ++t) {
                    float h[8];
                    const uint4 u = *reinterpret_cast<const uint4 *>(H + (long long)(t < rows ? t : 0) * ldh + d);
                    unpack2(u.x, h[0], h[1], T());
                    unpack2(u.y, h[2], h[3], T());
                    unpack2(u.z, h[4], h[5], T());
                    unpack2(u.w, h[6], h[7], T());
                    if (live < 8)
#pragma unroll
                        for (int i = 0; i < 8; ++i) h[i] = i < live ? h[i] : 0.0f;
#pragma unroll
                    for (int w = 0; w < kWords; ++w)
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[t][w] = fmaf(h[i], x[w][i], acc[t][w]);
                }
            }
            ringw.done();
        }
#pragma unroll
        for (int t = 0; t < R; ++t) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) acc[t][w] += __shfl_xor_sync(0xffffffffu, acc[t][w], o);
                if (lane == 0 && t < rows && label[t] == v0 + w && v0 + w < V) target[t] = acc[t][w];
                if (v0 + w >= V) acc[t][w] = -INFINITY;
            }
            float mn = m[t];                             // (in units of log 2)
#pragma unroll
            for (int w = 0; w < kWords; ++w) mn = fmaxf(mn, acc[t][w] * kLog2e);
            const float base = mn == -INFINITY ? 0.0f : mn;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWords; ++w) sum += exp2_fast(fmaf(acc[t][w], kLog2e, -base));
            s[t] = s[t] * (m[t] == -INFINITY ? 0.0f : exp2_fast(m[t] - base)) + sum;
            m[t] = mn;
        }
    }
    if (failed) {
        abort_s = 1;
        if (lane == 0) record_timeout(status);
        ringw.drain();
    }
    if (lane == 0)
#pragma unroll
        for (int t = 0; t < R; ++t) sh[warp][t] = make_float2(m[t], s[t]);
    __syncthreads();
    if (threadIdx.x < R && (int)threadIdx.x < rows) {
        float mm = sh[0][threadIdx.x].x, ss = sh[0][threadIdx.x].y;
#pragma unroll
        for (int k = 1; k < kWarps; ++k) join_stats(mm, ss, sh[k][threadIdx.x].x, sh[k][threadIdx.x].y);
        part[(long long)threadIdx.x * parts + blockIdx.x] = make_float2(mm, ss);
    }
}

}  // namespace

// Partial statistics per row: one CTA on each of a B200's SMs (a fixed number, so that workspaces have a fixed size), fewer where
// the vocabulary is small.
int loss_rows_parts(int V)
{
    const long long n = ((long long)V + kWarps * kWords - 1) / (kWarps * kWords);
    return (int)(n < 148 ? n : 148);
}

namespace {
template <typename T>
int launch_typed(const void *H, long long ldh, const void *W, long long ldw, const long long *labels, int rows, int V, int D, float2 *part,
                 int parts, float *target, int *status, cudaStream_t stream)
{
    const int blocks = loss_rows_parts(V);
    const auto kernel = rows == 1 ? &loss_rows_kernel<1, T> : &loss_rows_kernel<2, T>;
    static bool attr_set[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    if (!attr_set[dev]) {
        if (cudaFuncSetAttribute(&loss_rows_kernel<1, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem) != cudaSuccess ||
            cudaFuncSetAttribute(&loss_rows_kernel<2, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return CDL_ERR_LAUNCH;
        }
        attr_set[dev] = true;
    }
    return launch_following(kernel, dim3((unsigned)blocks), dim3(32 * kWarps), kRingSmem, stream, static_cast<const T *>(H), ldh,
                            static_cast<const T *>(W), ldw, labels, rows, V, D, part, parts, target, status);
}
}  // namespace

int launch_loss_rows(const void *H, long long ldh, const void *W, long long ldw, int type, const long long *labels, int rows, int V, int D,
                     float2 *part, int parts, float *target, int *status, cudaStream_t stream)
{
    if (type == CDL_BF16) return launch_typed<__nv_bfloat16>(H, ldh, W, ldw, labels, rows, V, D, part, parts, target, status, stream);
    return launch_typed<__half>(H, ldh, W, ldw, labels, rows, V, D, part, parts, target, status, stream);
}

}  // namespace cdl
