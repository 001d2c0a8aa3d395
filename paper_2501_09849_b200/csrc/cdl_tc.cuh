// What the tensor-core kernels of this library share: thin wrappers of the TMA, mbarrier-cluster, tcgen05 and TMEM
// instructions, the shared-memory operand descriptor, and the driver's tensor-map encoder.
#pragma once
#include <cuda.h>
#include <stdint.h>

#include "cdl_internal.h"

namespace cdl {

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
}

// Load issued by either CTA of a pair into its own shared memory; the bytes are counted on the barrier at offset
// `bar` of CTA 0 (no multicast: each CTA fetches its own box).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t bar)
{
    asm volatile(
        "{\n\t.reg .b32 rb;\n\t"
        "mapa.shared::cluster.u32 rb, %4, 0;\n\t"
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [rb];\n\t}"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, int c0, int c1, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(map), "r"(c0), "r"(c1), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_reduce_add_2d(const CUtensorMap *map, int c0, int c1, uint32_t src)
{
    asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(map), "r"(c0), "r"(c1), "r"(src) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// ---- CTA-pair helpers (cluster of two CTAs, cta_group::2)
__device__ __forceinline__ uint32_t cluster_ctarank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// arrive on the barrier at the same shared-memory offset in CTA `rank` of the cluster
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar, uint32_t rank)
{
    asm volatile(
        "{\n\t.reg .b32 ra;\n\t"
        "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
        "mbarrier.arrive.shared::cluster.b64 _, [ra];\n\t}"
        ::"r"(bar), "r"(rank)
        : "memory");
}
// both CTAs of the pair get the arrival (same barrier offset in each)
__device__ __forceinline__ void tc_commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}
// Wait for the TMEM loads in flight and tie the loaded registers to the wait, so that no use of them is scheduled
// ahead of it.
__device__ __forceinline__ void tc_wait_ld_pin(uint32_t (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
    asm volatile(""
                 : "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                   "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :
                 : "memory");
}

__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tc_wait_ld_pin(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

// Shared-memory operand descriptor (sm_100 format): start address, leading / stride byte offsets in 16-byte
// units, version 1, 128-byte swizzle.
__device__ __forceinline__ uint64_t make_desc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3fffu);
    d |= (uint64_t)((lbo_bytes >> 4) & 0x3fffu) << 16;
    d |= (uint64_t)((sbo_bytes >> 4) & 0x3fffu) << 32;
    d |= (uint64_t)1 << 46;   // descriptor version for sm_100
    d |= (uint64_t)2 << 61;   // SWIZZLE_128B
    return d;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn get_encode()
{
    static EncodeTiledFn fn = nullptr;
    if (fn == nullptr) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
            qres != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            return nullptr;
        }
        fn = reinterpret_cast<EncodeTiledFn>(p);
    }
    return fn;
}

// The four MMAs of one 128-byte stage (K = 32 eight-bit or 16 sixteen-bit entries each) in one go: descriptor k is
// (lo + k * step, hi); the first one accumulates only when `accumulate` is set, the others always.
#define CDL_TC_MMA4(GROUP, KIND, MASK)                                                                                          \
    asm volatile(                                                                                                             \
        "{\n\t.reg .pred p, t;\n\t.reg .b64 da, db;\n\t.reg .b32 al, bl;\n\t"                                                   \
        "setp.ne.b32 p, %8, 0;\n\t"                                                                                           \
        "setp.eq.b32 t, 0, 0;\n\t"                                                                                            \
        "mov.b64 da, {%1, %2};\n\tmov.b64 db, {%4, %5};\n\t"                                                                  \
        "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], da, db, %7, {" MASK "}, p;\n\t"                                \
        "add.u32 al, %1, %3;\n\tadd.u32 bl, %4, %6;\n\t"                                                                      \
        "mov.b64 da, {al, %2};\n\tmov.b64 db, {bl, %5};\n\t"                                                                  \
        "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], da, db, %7, {" MASK "}, t;\n\t"                                \
        "add.u32 al, al, %3;\n\tadd.u32 bl, bl, %6;\n\t"                                                                      \
        "mov.b64 da, {al, %2};\n\tmov.b64 db, {bl, %5};\n\t"                                                                  \
        "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], da, db, %7, {" MASK "}, t;\n\t"                                \
        "add.u32 al, al, %3;\n\tadd.u32 bl, bl, %6;\n\t"                                                                      \
        "mov.b64 da, {al, %2};\n\tmov.b64 db, {bl, %5};\n\t"                                                                  \
        "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], da, db, %7, {" MASK "}, t;\n\t}"                               \
        ::"r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(a_step), "r"(b_lo), "r"(b_hi), "r"(b_step), "r"(idesc), "r"(accumulate), "r"(0u) \
        : "memory")

enum TcKind { KIND_F8F6F4 = 0, KIND_F16 = 1 };

template <bool PAIR, int KIND>
__device__ __forceinline__ void tc_mma4(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t a_step, uint32_t b_lo, uint32_t b_hi,
                                        uint32_t b_step, uint32_t idesc, uint32_t accumulate)
{
    if (PAIR) {
        if (KIND == KIND_F16) CDL_TC_MMA4("2", "f16", "%9, %9, %9, %9, %9, %9, %9, %9");
        else CDL_TC_MMA4("2", "f8f6f4", "%9, %9, %9, %9, %9, %9, %9, %9");
    } else {
        if (KIND == KIND_F16) CDL_TC_MMA4("1", "f16", "%9, %9, %9, %9");
        else CDL_TC_MMA4("1", "f8f6f4", "%9, %9, %9, %9");
    }
}
#undef CDL_TC_MMA4

template <bool PAIR>
__device__ __forceinline__ void tmem_alloc_all(uint32_t slot_addr)      // all 512 columns; one warp, converged
{
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot_addr), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot_addr), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free_all(uint32_t base)
{
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(512u) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(512u) : "memory");
}

// Tiles in bands of eight tile rows, columns outer, so that what runs at one time shares operand blocks in L2.
__device__ __forceinline__ void tile_at(int u, int tiles_i, int tiles_j, int &ti, int &tj)
{
    const int band = 8 * tiles_j;
    const int b = u / band, first = b * 8, rows = min(8, tiles_i - first), in = u - b * band;
    tj = in / rows;
    ti = first + in - tj * rows;
}

// acc.{x,y} += v.{x,y} * s.{x,y}, two binary32 fused multiply-adds in one instruction
__device__ __forceinline__ void fma2(float2 &acc, uint32_t v0, uint32_t v1, float2 s)
{
    asm("{\n\t.reg .b64 a, v, f;\n\t"
        "mov.b64 a, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\tmov.b64 f, {%4, %5};\n\t"
        "fma.rn.f32x2 a, v, f, a;\n\t"
        "mov.b64 {%0, %1}, a;\n\t}"
        : "+f"(acc.x), "+f"(acc.y)
        : "r"(v0), "r"(v1), "f"(s.x), "f"(s.y));
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 c;
    asm("{\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 a, a, b;\n\t"
        "mov.b64 {%0, %1}, a;\n\t}"
        : "=f"(c.x), "=f"(c.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return c;
}

// Two-dimensional tensor map of `cols` x `rows` elements (cols contiguous, row pitch in bytes) with boxes of 128 (or 64)
// bytes under the swizzle of that width; reads outside are zero, writes outside are dropped in units of 16 bytes.
inline bool encode_map_2d(CUtensorMap *map, CUtensorMapDataType type, int elem_bytes, const void *base, uint64_t cols, uint64_t rows,
                          uint64_t pitch_bytes, uint32_t box_rows, uint32_t box_bytes = 128)
{
    EncodeTiledFn fn = get_encode();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {cols, rows};
    const cuuint64_t strides[1] = {pitch_bytes};
    const cuuint32_t box[2] = {box_bytes / (uint32_t)elem_bytes, box_rows};
    const cuuint32_t estr[2] = {1u, 1u};
    return fn(map, type, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace cdl
