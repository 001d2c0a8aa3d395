// Block-scaled 8-bit floating-point quantizer: e4m3 codes with one binary32 scale per group of 128 consecutive entries
// of a row (CDL_FP8_ROWS) or per 128 x 128 block (CDL_FP8_BLOCKS):
//   s = max(RN(amax * RN(1/448)), 2^-126),   r = RN(1/s),   code = e4m3(sat(RN(x * r)))   (nearest even, saturated at 448)
// and, from the same read of x, the codes and scales of the transposed matrix (row mode: with the transposed matrix's own
// groups, 128 rows of a column).
//
// One CTA takes a 128 x 128 tile: every group of either orientation lies in one tile, so the tile is read once and kept in
// registers between its maxima and its codes.  A thread holds 8 rows x 8 columns; the sixteen threads of a row own
// 128 consecutive columns, so loads and code stores are whole lines, and a row's maximum is four shuffles.  The transposed
// codes go through 16 KB of shared memory in units of 8 rows, the unit number exclusive-ored with the column's, which
// keeps both the stores (a thread has eight rows of one column) and the loads (a warp writes two columns) free of bank
// conflicts.  HBM is the bound: 4 (bf16, both orientations) to 6 (f32) bytes per element: 8192 x 4096 bf16 both ways 26 us
// (5.2 TB/s), 5001 x 4608 f32 blocks 26 us; 16-bit pieces unpacked into floats, at half the CTAs per SM, took 56 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cdl_internal.h"
#include "cdl_lowp.cuh"

namespace cdl {
namespace {

constexpr int kThreads = 256;
constexpr float kInvMax = 1.0f / 448.0f;
constexpr float kTiny = 1.17549435e-38f;      // 2^-126

struct QuantFp8 {
    const void *x;
    long long ldx;
    int rows, cols;
    int tiles_i, tiles_j;      // 128 x 128 tiles along the rows and the columns; one CTA each, columns fastest
    unsigned char *codes, *codes_t;
    long long ldc, ldt;
    float *scales, *scales_t;
};

__device__ __forceinline__ void scale_of(float amax, float &s, float &r)
{
    s = fmaxf(__fmul_rn(amax, kInvMax), kTiny);
    r = __frcp_rn(s);
}

// codes of two values, the first in the low byte (saturating; NaN becomes the NaN code)
__device__ __forceinline__ uint32_t code2(float a, float b)
{
    uint16_t w;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(w) : "f"(b), "f"(a));
    return w;
}

// Four words (eight 16-bit entries) from an address that is only aligned to its elements: the two 16-byte units they lie in,
// shifted (3001 x 3003 bf16 both ways: 10.6 to 12.4 us, with loads of single entries 19.1; for f32 single entries are the faster
// form, 15.5 against 18.2).  The units may reach up to 14 bytes before and behind the words; the caller has seen that they
// are inside the matrix.
__device__ __forceinline__ void load_shifted(const void *p, uint32_t (&out)[4])
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint4 *q = reinterpret_cast<const uint4 *>(at & ~(uintptr_t)15);
    const uint4 a = __ldcs(q);
    const uint4 b = (at & 15) ? __ldcs(q + 1) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = (at & 8) ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = (at & 4) ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = (at & 2) ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
}

// A thread's 8 x 8 piece of the tile: 64 floats, or 32 words of two 16-bit values, whose magnitudes are compared two at a
// time.  Maxima drop a NaN: it does not enter a group's scale.
template <typename T>
struct Piece {
    uint32_t w[8][4];
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
    {
        uint32_t m;
        if (__is_same(T, __nv_bfloat16)) asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
        else asm("max.f16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
        return m;
    }
    static __device__ __forceinline__ float max_of(uint32_t m)
    {
        float lo, hi;
        unpack2(m, lo, hi, T());
        return fmaxf(lo, hi);
    }
    __device__ __forceinline__ void load(int i, const T *p)
    {
        const uint4 q = __ldcs(reinterpret_cast<const uint4 *>(p));
        w[i][0] = q.x;
        w[i][1] = q.y;
        w[i][2] = q.z;
        w[i][3] = q.w;
    }
    __device__ __forceinline__ void load_unaligned(int i, const T *p) { load_shifted(p, w[i]); }
    __device__ __forceinline__ void load_some(int i, const T *p, int live)
    {
        const unsigned short *h = reinterpret_cast<const unsigned short *>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[i][j] = (2 * j < live ? (uint32_t)h[2 * j] : 0u) | (2 * j + 1 < live ? (uint32_t)h[2 * j + 1] << 16 : 0u);
    }
    __device__ __forceinline__ float row_max(int i) const
    {
        const uint32_t k = 0x7fff7fffu;
        return max_of(max2(max2(w[i][0] & k, w[i][1] & k), max2(w[i][2] & k, w[i][3] & k)));
    }
    // maxima of the 8 columns over the warp's 16 rows -> part (floats)
    __device__ __forceinline__ void column_max(float *part, int lane) const
    {
        const uint32_t k = 0x7fff7fffu;
        float c[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t m = w[0][j] & k;
#pragma unroll
            for (int i = 1; i < 8; ++i) m = max2(m, w[i][j] & k);
            m = max2(m, __shfl_xor_sync(0xffffffffu, m, 16));
            unpack2(m, c[2 * j], c[2 * j + 1], T());
            c[2 * j] = fmaxf(c[2 * j], 0.0f);            // (both NaN: no magnitude)
            c[2 * j + 1] = fmaxf(c[2 * j + 1], 0.0f);
        }
        if (lane < 16) {
            *reinterpret_cast<float4 *>(part) = make_float4(c[0], c[1], c[2], c[3]);
            *reinterpret_cast<float4 *>(part + 4) = make_float4(c[4], c[5], c[6], c[7]);
        }
    }
    __device__ __forceinline__ float value(int i, int j) const
    {
        float lo, hi;
        unpack2(w[i][j >> 1], lo, hi, T());
        return (j & 1) ? hi : lo;
    }
};
template <>
struct Piece<float> {
    float v[8][8];
    __device__ __forceinline__ void load(int i, const float *p) { load8(p, v[i]); }
    __device__ __forceinline__ void load_unaligned(int i, const float *p) { load_some(i, p, 8); }
    __device__ __forceinline__ void load_some(int i, const float *p, int live)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = j < live ? p[j] : 0.0f;
    }
    __device__ __forceinline__ float row_max(int i) const
    {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[i][j]));
        return m;
    }
    __device__ __forceinline__ void column_max(float *part, int lane) const
    {
        float c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) c[j] = fmaxf(c[j], fabsf(v[i][j]));
            c[j] = fmaxf(c[j], __shfl_xor_sync(0xffffffffu, c[j], 16));
        }
        if (lane < 16) {
            *reinterpret_cast<float4 *>(part) = make_float4(c[0], c[1], c[2], c[3]);
            *reinterpret_cast<float4 *>(part + 4) = make_float4(c[4], c[5], c[6], c[7]);
        }
    }
    __device__ __forceinline__ float value(int i, int j) const { return v[i][j]; }
};

// BLOCKS: one scale for the tile; otherwise one per row of the tile and, with BOTH, one per column.  VEC: rows of x can be
// read 16 bytes at a time.
template <typename T, bool BLOCKS, bool BOTH, bool VEC>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : 4)
quantize_fp8_kernel(const QuantFp8 Q)
{
    __shared__ __align__(16) float part[8][128];                // per warp: column maxima, or one tile maximum
    __shared__ __align__(16) unsigned char tile_t[BOTH ? 128 * 128 : 16];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ti = (int)(blockIdx.x / (unsigned)Q.tiles_j), tj = (int)(blockIdx.x - (unsigned)ti * (unsigned)Q.tiles_j);
    const int r0 = ti * 128, c0 = tj * 128;
    const int row = r0 + ty * 8, col = c0 + tx * 8;             // this thread's 8 x 8 piece
    const T *x = static_cast<const T *>(Q.x);
    follow_previous();

    Piece<T> v;
    if (VEC && row + 8 <= Q.rows && col + 8 <= Q.cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.load(i, x + (long long)(row + i) * Q.ldx + col);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const T *p = x + (long long)(row + i) * Q.ldx + col;
            const bool whole = row + i < Q.rows && col + 8 <= Q.cols;
            // (unaligned: not at the matrix' first and last entries, where a 16-byte unit may begin before it or end behind it)
            const uintptr_t lo = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15, hi = (reinterpret_cast<uintptr_t>(p + 8) + 15) & ~(uintptr_t)15;
            if (VEC && whole) v.load(i, p);
            else if (sizeof(T) == 2 && !VEC && whole && lo >= reinterpret_cast<uintptr_t>(x) && hi <= reinterpret_cast<uintptr_t>(x + (long long)(Q.rows - 1) * Q.ldx + Q.cols))
                v.load_unaligned(i, p);
            else v.load_some(i, p, row + i < Q.rows ? Q.cols - col : 0);
        }
    }
    float rrec[8], crec[8];
    if (BLOCKS) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, v.row_max(i));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) part[warp][0] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, part[k][0]);
        float s, r;
        scale_of(m, s, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) rrec[i] = crec[i] = r;
        if (threadIdx.x == 0) {
            Q.scales[(long long)tj * Q.tiles_i + ti] = s;
            if (BOTH) Q.scales_t[(long long)ti * Q.tiles_j + tj] = s;
        }
    } else {
        if (BOTH) v.column_max(&part[warp][tx * 8], lane);
        // Row maxima over sixteen lanes: each exchange halves the number of rows a lane is left with (8 shuffles instead of
        // 32), so that a lane ends with one row, whose scale it computes once and hands back.
        float m[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = v.row_max(i);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float keep = (tx & 8) ? m[i + 4] : m[i], send = (tx & 8) ? m[i] : m[i + 4];
            m[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, send, 8));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float keep = (tx & 4) ? m[i + 2] : m[i], send = (tx & 4) ? m[i] : m[i + 2];
            m[i] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, send, 4));
        }
        const float keep = (tx & 2) ? m[1] : m[0], send = (tx & 2) ? m[0] : m[1];
        m[0] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, send, 2));
        m[0] = fmaxf(m[0], __shfl_xor_sync(0xffffffffu, m[0], 1));
        float s, r;
        scale_of(fmaxf(m[0], 0.0f), s, r);
        const int mine = tx >> 1;                                // the row this lane was left with
        if ((tx & 1) == 0 && row + mine < Q.rows) Q.scales[(long long)tj * Q.rows + row + mine] = s;
#pragma unroll
        for (int i = 0; i < 8; ++i) rrec[i] = __shfl_sync(0xffffffffu, r, (lane & 16) | (i << 1));
        if (BOTH) {
            __syncthreads();
            if (threadIdx.x < 128) {        // one column each; the reciprocal goes back through part[0]
                float mc = part[0][threadIdx.x];
#pragma unroll
                for (int k = 1; k < 8; ++k) mc = fmaxf(mc, part[k][threadIdx.x]);
                scale_of(mc, s, r);
                part[0][threadIdx.x] = r;
                if (c0 + (int)threadIdx.x < Q.cols) Q.scales_t[(long long)ti * Q.cols + c0 + threadIdx.x] = s;
            }
        }
    }
    if (col < Q.cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (row + i >= Q.rows) break;
            uint32_t h[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = code2(__fmul_rn(v.value(i, 2 * j), rrec[i]), __fmul_rn(v.value(i, 2 * j + 1), rrec[i]));
            unsigned char *p = Q.codes + (long long)(row + i) * Q.ldc + col;
            if (col + 8 <= Q.cols) *reinterpret_cast<uint2 *>(p) = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j < Q.cols) p[j] = (unsigned char)(h[j >> 1] >> (8 * (j & 1)));
        }
    }
    if (BOTH) {
        if (!BLOCKS) {
            __syncthreads();
            const float4 a = *reinterpret_cast<const float4 *>(&part[0][tx * 8]), b = *reinterpret_cast<const float4 *>(&part[0][tx * 8 + 4]);
            crec[0] = a.x; crec[1] = a.y; crec[2] = a.z; crec[3] = a.w;
            crec[4] = b.x; crec[5] = b.y; crec[6] = b.z; crec[7] = b.w;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = code2(__fmul_rn(v.value(2 * i, j), crec[j]), __fmul_rn(v.value(2 * i + 1, j), crec[j]));
            *reinterpret_cast<uint2 *>(&tile_t[(tx * 8 + j) * 128 + ((ty ^ tx) << 3)]) = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = k * 16 + ty, unit = tx;                // sixteen threads write the 128 rows of one column
            if (c0 + c >= Q.cols) continue;
            const uint2 w = *reinterpret_cast<const uint2 *>(&tile_t[c * 128 + ((unit ^ (c >> 3)) << 3)]);
            const int rr = r0 + unit * 8;
            unsigned char *p = Q.codes_t + (long long)(c0 + c) * Q.ldt + rr;
            if (rr + 8 <= Q.rows) *reinterpret_cast<uint2 *>(p) = w;
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (rr + j < Q.rows) p[j] = (unsigned char)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
        }
    }
}

template <typename T>
int launch_typed(const QuantFp8 &Q, bool blocks, cudaStream_t stream)
{
    const bool vec = (reinterpret_cast<uintptr_t>(Q.x) & 15u) == 0 && (Q.rows == 1 || (Q.ldx * (long long)sizeof(T)) % 16 == 0);
    const unsigned grid = (unsigned)Q.tiles_i * (unsigned)Q.tiles_j;
    const bool both = Q.codes_t != nullptr;
#define CDL_GO(BL, BO, VE) return launch_following(&quantize_fp8_kernel<T, BL, BO, VE>, dim3(grid), dim3(kThreads), 0, stream, Q)
    if (vec) {
        if (blocks) { if (both) CDL_GO(true, true, true); else CDL_GO(true, false, true); }
        else { if (both) CDL_GO(false, true, true); else CDL_GO(false, false, true); }
    } else {
        if (blocks) { if (both) CDL_GO(true, true, false); else CDL_GO(true, false, false); }
        else { if (both) CDL_GO(false, true, false); else CDL_GO(false, false, false); }
    }
#undef CDL_GO
}

}  // namespace
}  // namespace cdl

extern "C" int cdl_fp8_quantize(const void *x, int64_t ldx, int32_t type, int32_t rows, int32_t cols, int32_t mode, void *codes,
                                int64_t ldc, float *scales, void *codes_t, int64_t ldt, float *scales_t, void *stream)
{
    using namespace cdl;
    if (rows < 0 || cols < 0 || rows > kMostExtent || cols > kMostExtent || !valid_type(type) || (mode != CDL_FP8_ROWS && mode != CDL_FP8_BLOCKS)) return CDL_ERR_ARG;
    if (rows == 0 || cols == 0) return CDL_OK;
    if (x == nullptr || codes == nullptr || scales == nullptr || (codes_t == nullptr) != (scales_t == nullptr)) return CDL_ERR_ARG;
    if ((rows > 1 && ldx < cols) || ldc < cols || (codes_t != nullptr && ldt < rows)) return CDL_ERR_ARG;
    const int64_t tiles_i = ((int64_t)rows + 127) / 128, tiles_j = ((int64_t)cols + 127) / 128;
    if (tiles_i * tiles_j > 0x7fffffff) return CDL_ERR_ARG;
    if (misaligned(x, type) || (reinterpret_cast<uintptr_t>(scales) & 3u) || (reinterpret_cast<uintptr_t>(scales_t) & 3u)) return CDL_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(codes) & 15u) || (ldc & 15) || (reinterpret_cast<uintptr_t>(codes_t) & 15u) || (codes_t != nullptr && (ldt & 15)))
        return CDL_ERR_ALIGN;
    int rc = check_device();
    if (rc != CDL_OK) return rc;
    const QuantFp8 Q{x, ldx, rows, cols, (int)tiles_i, (int)tiles_j, static_cast<unsigned char *>(codes), static_cast<unsigned char *>(codes_t), ldc, ldt, scales, scales_t};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool blocks = mode == CDL_FP8_BLOCKS;
    switch (type) {
    case CDL_F32: return launch_typed<float>(Q, blocks, st);
    case CDL_BF16: return launch_typed<__nv_bfloat16>(Q, blocks, st);
    default: return launch_typed<__half>(Q, blocks, st);
    }
}
