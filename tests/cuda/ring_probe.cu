// Test-only kernel (built by tests/test_gpu_ring_drain.py, never linked into libcdl.so): warp 0 leaves a ring after an abandoned
// wait while a piece of it is still under way.  The piece is played by warp 1, which completes the slot's barrier `late_ns` after
// the start (or never, late_ns = 0); out[0] is 1 where the barrier was complete when drain() returned, out[1] the time it took.
#include "cdl_row_ring.cuh"

using Ring = cdl::RowRing<8, 2048>;

__global__ void ring_probe_kernel(unsigned long long late_ns, unsigned long long *out)
{
    __shared__ __align__(8) unsigned long long bars[cdl::kRingSlots];
    __shared__ int abort_s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        abort_s = 1;                     // a wait of this CTA was abandoned
        for (int s = 0; s < cdl::kRingSlots; ++s) cdl::mbar_init(cdl::smem_u32(&bars[s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const unsigned long long t0 = cdl::global_ns();
    if (warp == 0) {
        Ring ring;
        ring.bar = cdl::smem_u32(&bars[0]);
        ring.abort_flag = &abort_s;
        ring.lane = lane;
        ring.used = 1;                   // one piece asked for
        ring.got = 0;
        ring.drain();
        if (lane == 0) {
            out[1] = cdl::global_ns() - t0;
            out[0] = cdl::mbar_try_wait_now(ring.bar, 0u) ? 1ull : 0ull;
        }
    } else if (lane == 0 && late_ns != 0) {
        while (cdl::global_ns() - t0 < late_ns) __nanosleep(1000);
        cdl::mbar_arrive(cdl::smem_u32(&bars[0]));
    }
    __syncthreads();
}

extern "C" int ring_probe(unsigned long long late_ns, void *out, void *stream)
{
    if (late_ns > 8000000ull) return -1;
    ring_probe_kernel<<<1, 64, 0, static_cast<cudaStream_t>(stream)>>>(late_ns, static_cast<unsigned long long *>(out));
    return cudaGetLastError() == cudaSuccess ? 0 : -6;
}
