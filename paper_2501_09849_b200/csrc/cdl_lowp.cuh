// Element types of the operators that take 32- and 16-bit floats (CDL_F32, CDL_BF16, CDL_F16): conversions, 16-byte and eight-element
// accesses, and the argument checks they have in common.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "cdl_internal.h"

namespace cdl {

inline bool valid_type(int type) { return type == CDL_F32 || type == CDL_BF16 || type == CDL_F16; }
// Most rows, columns or reduced entries of an operand: tile corners and stage coordinates are 32-bit numbers.
constexpr int kMostExtent = 1 << 30;
inline int type_bytes(int type) { return type == CDL_F32 ? 4 : 2; }
inline bool misaligned(const void *p, int type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type_bytes(type) - 1)) != 0; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// two floats -> the packed word of two 16-bit values, `lo` at the lower address
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    uint32_t w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

__device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi, __nv_bfloat16)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi, __half)
{
    const __half2 h = *reinterpret_cast<const __half2 *>(&w);
    const float2 f = __half22float2(h);
    lo = f.x;
    hi = f.y;
}

__device__ __forceinline__ uint4 lds_u128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// Eight consecutive elements at a 16-byte boundary.  The loads are evict-first: the operators read each input once.
__device__ __forceinline__ void load8(const float *p, float (&v)[8])
{
    const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8])
{
    const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(p));
    unpack2(w.x, v[0], v[1], T());
    unpack2(w.y, v[2], v[3], T());
    unpack2(w.z, v[4], v[5], T());
    unpack2(w.w, v[6], v[7], T());
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}

}  // namespace cdl
