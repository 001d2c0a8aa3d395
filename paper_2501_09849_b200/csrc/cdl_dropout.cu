// Counter-based dropout, the mask never stored:  y_i = [u_i >= p] x_i / (1 - p)  (+ residual_i),  u_i the uniform
// number of element e = first_index + i in the counter space of the sampling quantizer (one Philox4x32-10 block per
// four elements).  The backward pass is the same map applied to the gradient, so nothing is kept in between.
//
// What bounds it: 4 to 12 bytes of HBM per element, and close behind them the integer pipes: a Philox block is 20 wide
// multiplies and 20 three-input logic operations for four elements.  One thread therefore handles eight consecutive
// elements (two blocks, one or two 16-byte accesses per tensor), the comparison with p is one unsigned comparison of the
// raw word, and the kept value, the scale and the residual are one fused multiply-add.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_philox.cuh"

namespace cdl {
namespace {

struct DropoutDev {
    float scale;               // RN(1 / (1 - p))
    unsigned int threshold;    // a word w keeps its element when w >= threshold: (w >> 8) 2^-24 >= p
    int drop_all;              // p = 1: the threshold does not fit 32 bits
    unsigned long long seed, first_index;
};

template <bool RES>
__device__ __forceinline__ float drop1(float x, float r, unsigned int w, const DropoutDev &d)
{
    // the element is selected before the product: a dropped infinity or NaN is gone
    const float kept = (w >= d.threshold && !d.drop_all) ? x : 0.0f;
    return RES ? fmaf(kept, d.scale, r) : kept * d.scale;
}

// Eight elements per thread and step.  Every row starts at a multiple of 4 in the counter space and at a 16-byte
// boundary of each tensor; cols is a multiple of 8 except for a single row, whose tail one more thread handles.
template <typename T, bool RES>
__global__ void __launch_bounds__(256)
dropout_vec_kernel(const T *x, long long ldx, const T *res, long long ldr, T *y, long long ldy, long long rows, long long cols, DropoutDev d)
{
    const long long octs = (cols + 7) >> 3;
    const long long stride = (long long)gridDim.x * blockDim.x;
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        const unsigned long long e_row = d.first_index + (unsigned long long)(r * cols);
        for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < octs; i += stride) {
            const long long c = i << 3;
            const unsigned long long blk = (e_row + (unsigned long long)c) >> 2;
            float v[8], q[8];
            const bool whole = c + 8 <= cols;
            if (whole) {
                load8(x + r * ldx + c, v);
                if (RES) load8(res + r * ldr + c, q);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = c + k < cols ? to_f32(x[r * ldx + c + k]) : 0.0f;
                    if (RES) q[k] = c + k < cols ? to_f32(res[r * ldr + c + k]) : 0.0f;
                }
            }
            const uint4 a = philox4x32_10(blk, d.seed), b = philox4x32_10(blk + 1, d.seed);
            const unsigned int w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = drop1<RES>(v[k], RES ? q[k] : 0.0f, w[k], d);
            if (whole) store8(y + r * ldy + c, v);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < cols) y[r * ldy + c + k] = from_f32<T>(v[k]);
        }
    }
}

// Any alignment, pitch and first index: a thread takes the (up to four) elements of a row that share a Philox block.
template <typename T, bool RES>
__global__ void __launch_bounds__(256)
dropout_any_kernel(const T *x, long long ldx, const T *res, long long ldr, T *y, long long ldy, long long rows, long long cols, DropoutDev d)
{
    const long long stride = (long long)gridDim.x * blockDim.x;
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        const unsigned long long e_row = d.first_index + (unsigned long long)(r * cols);
        const int lead = (int)(e_row & 3u);
        const long long groups = (cols + lead + 3) >> 2;
        for (long long g = (long long)blockIdx.x * blockDim.x + threadIdx.x; g < groups; g += stride) {
            const uint4 a = philox4x32_10((e_row >> 2) + (unsigned long long)g, d.seed);
            const unsigned int w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const long long c = 4 * g + k - lead;
                if (c >= 0 && c < cols)
                    y[r * ldy + c] = from_f32<T>(drop1<RES>(to_f32(x[r * ldx + c]), RES ? to_f32(res[r * ldr + c]) : 0.0f, w[k], d));
            }
        }
    }
}

template <typename T>
int launch_typed(const void *xv, long long ldx, const void *rv, long long ldr, void *yv, long long ldy, long long rows, long long cols,
                 const DropoutDev &d, cudaStream_t stream)
{
    const T *x = static_cast<const T *>(xv), *res = static_cast<const T *>(rv);
    T *y = static_cast<T *>(yv);
    // an unpadded tensor is one row
    if (ldx == cols && ldy == cols && (res == nullptr || ldr == cols)) {
        cols *= rows;
        rows = 1;
    }
    auto aligned = [&](const void *p, long long ld) {
        return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows == 1 || (ld * (long long)sizeof(T)) % 16 == 0);
    };
    const bool vec = (d.first_index & 3u) == 0 && (rows == 1 || cols % 8 == 0) && aligned(x, ldx) && aligned(y, ldy) &&
                     (res == nullptr || aligned(res, ldr));
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    const long long per_row = vec ? (cols + 7) / 8 : (cols + 6) / 4;
    const int threads = 256;
    const long long cap = (long long)sms * 8 * 4;
    long long bx = (per_row + threads - 1) / threads;
    if (bx > cap) bx = cap;
    long long by = cap / bx;
    if (by > rows) by = rows;
    if (by > 65535) by = 65535;
    if (by < 1) by = 1;
    const dim3 grid((unsigned)bx, (unsigned)by);
    if (vec) {
        if (res != nullptr) dropout_vec_kernel<T, true><<<grid, threads, 0, stream>>>(x, ldx, res, ldr, y, ldy, rows, cols, d);
        else dropout_vec_kernel<T, false><<<grid, threads, 0, stream>>>(x, ldx, res, ldr, y, ldy, rows, cols, d);
    } else {
        if (res != nullptr) dropout_any_kernel<T, true><<<grid, threads, 0, stream>>>(x, ldx, res, ldr, y, ldy, rows, cols, d);
        else dropout_any_kernel<T, false><<<grid, threads, 0, stream>>>(x, ldx, res, ldr, y, ldy, rows, cols, d);
    }
    if (cudaGetLastError() != cudaSuccess) return CDL_ERR_LAUNCH;
    return CDL_OK;
}

}  // namespace
}  // namespace cdl

extern "C" int cdl_dropout(const void *x, int64_t ldx, const void *residual, int64_t ldr, void *y, int64_t ldy, int32_t type,
                           int64_t rows, int64_t cols, float p, uint64_t seed, uint64_t first_index, void *stream)
{
    using namespace cdl;
    if (rows < 0 || cols < 0 || !valid_type(type)) return CDL_ERR_ARG;
    if (!(p >= 0.0f && p <= 1.0f)) return CDL_ERR_RANGE;
    if (rows == 0 || cols == 0) return CDL_OK;
    if (x == nullptr || y == nullptr) return CDL_ERR_ARG;
    if (rows > INT64_MAX / cols) return CDL_ERR_ARG;
    if (rows > 1 && (ldx < cols || ldy < cols || (residual != nullptr && ldr < cols))) return CDL_ERR_ARG;
    if (misaligned(x, type) || misaligned(y, type) || misaligned(residual, type)) return CDL_ERR_ALIGN;
    if (rows == 1) ldx = ldy = ldr = cols;
    int rc = check_device();
    if (rc != CDL_OK) return rc;
    DropoutDev d;
    d.drop_all = p == 1.0f;
    d.scale = d.drop_all ? 0.0f : (float)(1.0 / (1.0 - (double)p));
    d.threshold = d.drop_all ? 0xffffffffu : (unsigned int)ceil((double)p * 16777216.0) << 8;
    // (the largest p below 1 is 1 - 2^-24, whose threshold (2^24 - 1) << 8 fits)
    d.seed = seed;
    d.first_index = first_index;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (type) {
    case CDL_F32: return launch_typed<float>(x, ldx, residual, ldr, y, ldy, rows, cols, d, st);
    case CDL_BF16: return launch_typed<__nv_bfloat16>(x, ldx, residual, ldr, y, ldy, rows, cols, d, st);
    default: return launch_typed<__half>(x, ldx, residual, ldr, y, ldy, rows, cols, d, st);
    }
}
