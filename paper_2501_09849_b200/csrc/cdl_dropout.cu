// Counter-based dropout, the mask never stored:  y_i = [u_i >= p] x_i / (1 - p)  (+ residual_i),  u_i the uniform
// number of element e = first_index + i in the counter space of the sampling quantizer (one Philox4x32-10 block per
// four elements).  The backward pass is the same map applied to the gradient, so nothing is kept in between.
//
// What bounds it: 4 to 12 bytes of HBM per element, and close behind them the generator: a Philox block is 18 wide multiplies
// of four to five cycles each per scheduler and 18 three-input logic operations for four elements.  One thread handles
// eight consecutive elements (two blocks, one or two 16-byte accesses per tensor) and fetches the next eight while it draws
// these; the comparison with p is one unsigned comparison of the raw word, the kept value, the scale and the residual are one
// fused multiply-add under its predicate, and the round keys are kernel parameters.  32749 x 2304: bf16 with residual 78 to 89 us
// (5.1 to 5.8 TB/s), without 79 to 86 us (3.5 to 3.8 TB/s, the multiplies), f32 with residual 147 us (6.2 TB/s); four CTAs of 256
// threads per SM (five: 92, 80, 165 us, with the same loop before the keys were parameters).  A padded tensor has rows of their own,
// which do not fill the blocks evenly: 2304 columns of pitch 2312 218 us.
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
    PhiloxKeys keys;
    unsigned long long first_index;
};

template <bool RES>
__device__ __forceinline__ float drop1(float x, float r, unsigned int w, const DropoutDev &d)
{
    // (a dropped infinity or NaN is gone: the product is not taken)
    float y = RES ? r : 0.0f;
    if (w >= d.threshold && !d.drop_all) y = RES ? fmaf(x, d.scale, r) : x * d.scale;
    return y;
}

// Eight elements as they lie in memory: two or one 16-byte words.
template <typename T>
struct Oct {
    uint4 q[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
    }
    // elements 4 h .. 4 h + 3
    __device__ __forceinline__ void half(int h, float (&v)[4]) const
    {
        if constexpr (sizeof(T) == 4) {
            v[0] = __uint_as_float(q[h].x);
            v[1] = __uint_as_float(q[h].y);
            v[2] = __uint_as_float(q[h].z);
            v[3] = __uint_as_float(q[h].w);
        } else {
            unpack2(h ? q[0].z : q[0].x, v[0], v[1], T());
            unpack2(h ? q[0].w : q[0].y, v[2], v[3], T());
        }
    }
};

// Eight elements per thread and step, the next step's loads on their way while this one's words are drawn.  Every row starts
// at a multiple of 4 in the counter space and at a 16-byte boundary of each tensor; cols is a multiple of 8 except for a
// single row, whose tail further threads handle.  A row is shorter than 2^28 elements: offsets are 32 bits.
template <typename T, bool RES>
__global__ void __launch_bounds__(256, 4)
dropout_vec_kernel(const T *x, long long ldx, const T *res, long long ldr, T *y, long long ldy, long long rows, unsigned int cols,
                   const __grid_constant__ DropoutDev d)
{
    follow_previous();
    const unsigned int octs = cols >> 3, stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + threadIdx.x;
    constexpr unsigned int kOct = 8u * sizeof(T);            // bytes
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        const unsigned long long e_row = d.first_index + (unsigned long long)r * cols;
        const char *xr = reinterpret_cast<const char *>(x + r * ldx), *qr = RES ? reinterpret_cast<const char *>(res + r * ldr) : nullptr;
        char *yr = reinterpret_cast<char *>(y + r * ldy);
        const unsigned long long blk0 = e_row >> 2;
        unsigned int hi = (unsigned int)(blk0 >> 32);
        unsigned long long head = philox_head(hi, d.keys);
        Oct<T> xn, qn;
        if (first < octs) {
            xn.load(reinterpret_cast<const T *>(xr + first * kOct));
            if (RES) qn.load(reinterpret_cast<const T *>(qr + first * kOct));
        }
        for (unsigned int i = first; i < octs; i += stride) {
            const Oct<T> xc = xn, qc = qn;
            if (i + stride < octs) {                         // (below 2^26: no wrap)
                xn.load(reinterpret_cast<const T *>(xr + (i + stride) * kOct));
                if (RES) qn.load(reinterpret_cast<const T *>(qr + (i + stride) * kOct));
            }
            const unsigned long long blk = blk0 + 2u * i;
            if ((unsigned int)(blk >> 32) != hi) {
                hi = (unsigned int)(blk >> 32);
                head = philox_head(hi, d.keys);
            }
            uint4 out[sizeof(T) / 2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h == 1 && (unsigned int)blk == 0xffffffffu) head = philox_head(++hi, d.keys);
                const uint4 a = philox4x32_10((unsigned int)blk + h, head, d.keys);
                float v[4], q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                xc.half(h, v);
                if (RES) qc.half(h, q);
                v[0] = drop1<RES>(v[0], q[0], a.x, d);
                v[1] = drop1<RES>(v[1], q[1], a.y, d);
                v[2] = drop1<RES>(v[2], q[2], a.z, d);
                v[3] = drop1<RES>(v[3], q[3], a.w, d);
                if constexpr (sizeof(T) == 4) out[h] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
                else if (h == 0) {
                    out[0].x = pack2<T>(v[0], v[1]);
                    out[0].y = pack2<T>(v[2], v[3]);
                } else {
                    out[0].z = pack2<T>(v[0], v[1]);
                    out[0].w = pack2<T>(v[2], v[3]);
                }
            }
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) __stcs(reinterpret_cast<uint4 *>(yr + i * kOct) + k, out[k]);
        }
        if ((cols & 7u) != 0 && first < (cols & 7u)) {       // (a single row)
            const unsigned int c = octs * 8u + first;
            const unsigned long long e = e_row + c;
            const uint4 a = philox4x32_10(e >> 2, d.keys);
            const unsigned int k = (unsigned int)e & 3u, w = k == 0 ? a.x : (k == 1 ? a.y : (k == 2 ? a.z : a.w));
            const T *xe = reinterpret_cast<const T *>(xr) + c, *qe = reinterpret_cast<const T *>(qr) + c;
            reinterpret_cast<T *>(yr)[c] = from_f32<T>(drop1<RES>(to_f32(*xe), RES ? to_f32(*qe) : 0.0f, w, d));
        }
    }
}

// Any alignment, pitch and first index: a thread takes the (up to four) elements of a row that share a Philox block, one at a time
// and none ahead.  32749 x 2304 bf16: first index 2 118 us, a pointer between 16-byte units 119, pitch 2305 158; f32, first index 1, 178.
template <typename T, bool RES>
__global__ void __launch_bounds__(256)
dropout_any_kernel(const T *x, long long ldx, const T *res, long long ldr, T *y, long long ldy, long long rows, long long cols,
                   const __grid_constant__ DropoutDev d)
{
    follow_previous();
    const long long stride = (long long)gridDim.x * blockDim.x;
    for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
        const unsigned long long e_row = d.first_index + (unsigned long long)(r * cols);
        const int lead = (int)(e_row & 3u);
        const long long groups = (cols + lead + 3) >> 2;
        for (long long g = (long long)blockIdx.x * blockDim.x + threadIdx.x; g < groups; g += stride) {
            const uint4 a = philox4x32_10((e_row >> 2) + (unsigned long long)g, d.keys);
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
                 DropoutDev d, cudaStream_t stream)
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
    constexpr long long kMostCols = 1ll << 28;           // of a row of the vector form
    const bool vec = (d.first_index & 3u) == 0 && (rows == 1 || (cols % 8 == 0 && cols < kMostCols)) && aligned(x, ldx) && aligned(y, ldy) &&
                     (res == nullptr || aligned(res, ldr));
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    const int threads = 256;
    // (vector form: a grid that is resident at once, so that a thread has several steps to fetch ahead)
    auto grid_for = [&](long long per_row, long long cap) {
        long long bx = (per_row + threads - 1) / threads;
        if (bx > cap) bx = cap;
        if (bx < 1) bx = 1;
        long long by = cap / bx;
        if (by > rows) by = rows;
        if (by > 65535) by = 65535;
        return dim3((unsigned)bx, (unsigned)by);
    };
    if (!vec) {
        const dim3 grid = grid_for((cols + 6) / 4, (long long)sms * 32);
        return launch_following(res != nullptr ? &dropout_any_kernel<T, true> : &dropout_any_kernel<T, false>, grid, dim3(threads), 0, stream, x, ldx, res,
                                ldr, y, ldy, rows, cols, (const DropoutDev)d);
    }
    // a longer single row goes in several launches
    const long long piece = rows == 1 ? kMostCols - 8 : cols;
    for (long long c = 0; c < cols; c += piece) {
        const long long n = cols - c < piece ? cols - c : piece;
        const dim3 grid = grid_for((n + 7) / 8, (long long)sms * 4);
        const int rc = launch_following(res != nullptr ? &dropout_vec_kernel<T, true> : &dropout_vec_kernel<T, false>, grid, dim3(threads), 0, stream,
                                        x + c, ldx, res != nullptr ? res + c : res, ldr, y + c, ldy, rows, (unsigned)n, (const DropoutDev)d);
        if (rc != CDL_OK) return rc;
        d.first_index += (unsigned long long)n;
    }
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
    d.keys = philox_keys(seed);
    d.first_index = first_index;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (type) {
    case CDL_F32: return launch_typed<float>(x, ldx, residual, ldr, y, ldy, rows, cols, d, st);
    case CDL_BF16: return launch_typed<__nv_bfloat16>(x, ldx, residual, ldr, y, ldy, rows, cols, d, st);
    default: return launch_typed<__half>(x, ldx, residual, ldr, y, ldy, rows, cols, d, st);
    }
}
