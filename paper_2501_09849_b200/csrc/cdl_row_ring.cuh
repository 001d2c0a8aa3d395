// Streaming rows of a matrix through shared memory, one ring per warp: lane 0 asks for the next pieces of kRingRows rows with
// untiled bulk copies while the warp works on the ones that have arrived; the warps of a CTA never wait for one another.
// What it buys over loads into registers is bytes in flight: 192 KB per SM, where eight
// 16-byte loads per lane keep 4 KB of a warp's under way (reading 262 MB once: 59 us with loads, see the kernels).
#pragma once
#include <stdint.h>

#include "cdl_wait.cuh"

namespace cdl {

constexpr int kRingRows = 4;                 // rows of a piece
constexpr int kRingSlots = 3;
constexpr int kRingSmem = 192 * 1024;        // rings of a CTA: WARPS x kRingSlots x kRingRows x BYTES
constexpr unsigned long long kRingWaitNs = 2000000000ull;

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// The pieces of a group are taken from a different one on in every warp (`turn`): with a row pitch that is a power of two all
// warps would otherwise read the same few memory channels at the same time.
// The groups of rows of one warp: rows first + i * step .. + kRingRows - 1 for i < groups, the first `bytes` of each (the last
// 16-byte unit is fetched whole).  Positions in a row are unsigned: a row of 2^30 16-bit entries has 2^31 bytes.
// BYTES: of each row of a piece (eight warps with 2 KB read longer runs than sixteen with 1 KB: 32000 x 4096 bf16 43.9 us and 48.0).
template <int WARPS, int BYTES>
struct RowRing {
    static constexpr unsigned kRingBytes = BYTES;
    static_assert(WARPS * kRingSlots * kRingRows * BYTES == kRingSmem, "shared memory");
    const unsigned char *base;
    long long pitch, first, step, rows;
    int groups;
    unsigned bytes, turn;                    // turn: byte offset of a group's first piece, a multiple of kRingBytes below `bytes`
    uint32_t smem, bar;                      // this warp's slots and barriers
    volatile int *abort_flag;
    int lane;
    int next_group, used, got;               // what is asked for next; slots used so far; pieces taken so far
    unsigned next_at;

    __device__ __forceinline__ unsigned pieces() const { return (bytes + kRingBytes - 1u) / kRingBytes; }            // of a row
    __device__ __forceinline__ unsigned after(unsigned at) const { return at + kRingBytes < bytes ? at + kRingBytes : 0u; }     // the piece behind one
    __device__ __forceinline__ void ask()    // lane 0: the next piece, if there is one
    {
        if (next_group >= groups) return;
        const unsigned left = bytes - next_at, len = ((left < kRingBytes ? left : kRingBytes) + 15u) & ~15u;
        const uint32_t slot = (uint32_t)(used % kRingSlots);
        const uint32_t dst = smem + slot * (kRingRows * kRingBytes), b = bar + 8u * slot;
        mbar_expect_tx(b, kRingRows * len);
        const long long r0 = first + next_group * step;
#pragma unroll
        for (int r = 0; r < kRingRows; ++r)
            bulk_load(dst + (uint32_t)r * kRingBytes, base + (r0 + r < rows ? r0 + r : rows - 1) * pitch + next_at, len, b);
        ++used;
        next_at = after(next_at);
        if (next_at == turn) ++next_group;
    }
    __device__ __forceinline__ void start()
    {
        next_group = used = got = 0;
        turn = turn % pieces() * kRingBytes;         // (given as a number of pieces)
        next_at = turn;
        if (lane == 0)
            for (int s = 0; s < kRingSlots; ++s) ask();
    }
    // shared address of the next piece (false: gave up waiting)
    __device__ __forceinline__ bool take(uint32_t &addr)
    {
        const uint32_t slot = (uint32_t)(got % kRingSlots), parity = (uint32_t)(got / kRingSlots) & 1u;
        ++got;
        addr = smem + slot * (kRingRows * kRingBytes);
        return __all_sync(0xffffffffu, mbar_try_wait_now(bar + 8u * slot, parity) || mbar_wait(bar + 8u * slot, parity, abort_flag, kRingWaitNs));
    }
    __device__ __forceinline__ void done()   // the piece has been read
    {
        __syncwarp();
        if (lane == 0) ask();
    }
    // Before the CTA ends after an abandoned wait: bulk copies of this warp that are still under way have landed (or a limit has
    // run out for each; the flag that ends the other waits is set by now and does not count here).
    __device__ __forceinline__ void drain()
    {
        __syncwarp();
        drain_stages(bar, (uint32_t)__shfl_sync(0xffffffffu, used, 0), (uint32_t)kRingSlots);
    }
};

}  // namespace cdl
