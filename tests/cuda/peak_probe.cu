// Test-only kernel (built by tests/test_gpu_peak_exchange.py, never linked into libcdl.so): two warps exchange their lanes' numbers `rounds` times.
// Warp `quitter` (0, 1, or -1 for neither) gives up before its exchange number `quit`, setting the abort flag or not; the other one comes `late_ns`
// after the start.  met[w]: exchanges that returned true in warp w; wrong[w]: those whose result was not the larger number.
#include "cdl_wait.cuh"

__global__ void peak_probe_kernel(int rounds, int quitter, int quit, int flag, unsigned long long late_ns, unsigned long long limit_ns, int *met, int *wrong)
{
    __shared__ __align__(8) unsigned char meet[cdl::PeakExchange::kBytes];
    __shared__ float peaks[2 * 32];
    __shared__ int abort_s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bars = cdl::smem_u32(meet);
    if (threadIdx.x == 0) {
        abort_s = 0;
        cdl::PeakExchange::init(bars);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const unsigned long long t0 = cdl::global_ns();
    if (warp != quitter)
        while (cdl::global_ns() - t0 < late_ns) __nanosleep(1000);
    cdl::PeakExchange exchange{bars, 0u};
    int done = 0, bad = 0;
    for (; done < rounds; ++done) {
        if (warp == quitter && done == quit) {
            if (flag && lane == 0) *(volatile int *)&abort_s = 1;
            break;
        }
        float m = (float)((done * 7 + lane * (warp + 3)) % 61);
        const float mine = m, other = (float)((done * 7 + lane * ((warp ^ 1) + 3)) % 61);
        if (!exchange(&peaks[warp * 32 + lane], &peaks[(warp ^ 1) * 32 + lane], lane, m, &abort_s, limit_ns)) break;
        if (m != fmaxf(mine, other)) ++bad;
    }
    __syncthreads();
    if (lane == 0) met[warp] = done;
    atomicAdd(&wrong[warp], bad);
}

extern "C" int peak_probe(int rounds, int quitter, int quit, int flag, unsigned long long late_ns, unsigned long long limit_ns, void *met, void *wrong, void *stream)
{
    if (rounds < 0 || rounds > 10000 || late_ns > 8000000ull || limit_ns > 50000000ull) return -1;
    peak_probe_kernel<<<1, 64, 0, static_cast<cudaStream_t>(stream)>>>(rounds, quitter, quit, flag, late_ns, limit_ns, static_cast<int *>(met), static_cast<int *>(wrong));
    return cudaGetLastError() == cudaSuccess ? 0 : -6;
}
