// Layer norm of the rows of a matrix and its gradients:
//   m = mean x,  v = mean (x - m)^2,  r = 1 / sqrt(v + eps),  n = (x - m) r,  y = n gamma + beta
//   a = dy gamma,  dx = r (a - mean a - n mean(a n)) (+ residual),  dgamma = sum over rows of dy n,  dbeta = sum over rows of dy
//
// HBM is the bound: x and y forward, dy, x (the residual) and dx backward.  A row is read once and stays in registers: the mean comes first,
// then the deviations from it, whose own mean (what the mean's rounding left) is taken out again: the statistics are as good as two
// passes over memory, whatever the offset of the row.  A row belongs to a warp (up to 512 columns) or to a block; the grid is what
// the device holds at once, a block goes from row to row, and its threads keep their columns: gamma and beta, and backward the
// columns' sums, stay in registers.  The sums of all blocks are added by a second, small kernel in a fixed order.  A longer row is
// shared by the blocks of a cluster, which exchange their sums (2000 x 16384 backward, read again from L2 instead, took 149 us); one that is
// too long for that as well (forward 131072, backward 65536 columns) is read again.
// The next rows are on their way to shared memory in 16-byte asynchronous copies, three of them (one in binary32): with one row ahead in
// registers 8192 x 4096 took 87 us backward (spilled) and 33 forward.  A thread fetches what it reads itself; where rows do not start
// on 16 bytes the row's units are copied as they lie, and the threads take every G-th entry of it behind a barrier.
// 8192 x 4096 bf16: forward 29 us (4.6 TB/s), backward 43 (4.7), with a residual 50 (5.4); 4095 columns 44 and 62.  5000 x 4096 binary32:
// 28 (5.8) and with a residual 54 (6.1).  Beyond 8192 columns a block takes four units a thread forward, half of which a row of 8200 does not have, and two
// blocks share a row backward, with half of their threads: 2500 rows of 8192 columns 21 and 31 us, of 8200 33 and 77, of 8193 (unaligned) 44 and 101.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

#include "cdl_act.cuh"
#include "cdl_internal.h"
#include "cdl_lowp.cuh"
#include "cdl_tc.cuh"
#include "cdl_wait.cuh"

namespace cdl {
namespace {

struct NormDev {
    const void *x, *dy, *res;
    long long ldx, lddy, ldr;
    void *y;                        // backward: dx
    long long ldy;
    const float *gamma, *beta;
    float *mean, *rstd;
    int rows, cols;
    float eps, inv;                 // inv: 1 / cols
    float *part_g, *part_b;         // sums of a block, [blocks][cols] each; with one block the results, nullable
    int weight;                     // dgamma and dbeta are wanted
    int split, share;               // blocks of a cluster that share a row, columns of each
};

// The G threads of a row, in a block of several rows or of one.
template <int G, int BLOCK>
__device__ __forceinline__ void group_sync()
{
    if (G == 32) __syncwarp();
    else if (G == BLOCK) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / G), "n"(G) : "memory");
}

// Sums over the G threads of a row.  One barrier: the warps' sums go to two places in turn.
template <int G, int N, int BLOCK>
struct RowSum {
    float (*buf)[N][32];            // [2][N][warps of the block]
    int turn;
    __device__ __forceinline__ void operator()(float (&s)[N])
    {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
        if (G == 32) return;
        const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, first = (int)threadIdx.x / G * (G / 32);
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) buf[turn][k][warp] = s[k];
        group_sync<G, BLOCK>();
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] = buf[turn][k][first + (lane & (G / 32 - 1))];
#pragma unroll
        for (int o = G / 64; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] += __shfl_xor_sync(0xffffffffu, s[k], o);
        turn ^= 1;
    }
};

// Threads of a block, blocks that an SM is to hold, and rows that are taken together (what the registers hold without spilling).
__host__ __device__ constexpr int fwd_threads(int G) { return G == 32 ? 256 : G; }
constexpr int kBwdThreads = 512;        // a block an SM, and so 148 sums of a column at most
__host__ __device__ constexpr int fwd_blocks(int G, int UNITS) { return G == 32 ? 2 : (G == 128 ? (UNITS == 1 ? 6 : 4) : (G == 256 ? 2 : 1)); }
__host__ __device__ constexpr int fwd_rows(int bytes) { return bytes == 4 ? 1 : 2; }
__host__ __device__ constexpr int bwd_rows(int bytes, int UNITS) { return bytes == 4 || UNITS > 1 ? 1 : 2; }
// Steps of as many rows on their way or in use (a power of two; what shared memory holds).
__host__ __device__ constexpr int fwd_steps(int bytes, int UNITS) { return bytes == 4 && UNITS <= 2 ? 4 : 2; }
__host__ __device__ constexpr int bwd_steps(int bytes, int UNITS) { return bytes == 2 && UNITS > 1 ? 4 : 2; }

// The blocks of a cluster that share a row: their sums to all of them, added in the order of the blocks.  The places are used in turn, as
// above: a block writes to one again after a barrier that all have passed since they read it.
template <int N>
struct ClusterSum {
    float (*buf)[8][N];             // [2][blocks][N], in every block's shared memory
    int turn, rank, blocks;
    __device__ __forceinline__ void send(const float (&s)[N])
    {
        if ((int)threadIdx.x < blocks) {
            const uint32_t mine = smem_u32(&buf[turn][rank][0]);
#pragma unroll
            for (int k = 0; k < N; ++k)
                asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f32 [a], %2;\n\t}" ::"r"(mine + 4u * k), "r"((int)threadIdx.x), "f"(s[k]) : "memory");
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    __device__ __forceinline__ void receive(float (&s)[N])
    {
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
        for (int k = 0; k < N; ++k) {
            s[k] = buf[turn][0][k];
            for (int i = 1; i < blocks; ++i) s[k] += buf[turn][i][k];
        }
        turn ^= 1;
    }
    __device__ __forceinline__ void operator()(float (&s)[N])
    {
        send(s);
        receive(s);
    }
};

// The rows of up to three matrices on their way through shared memory to the G threads of a group: 16 bytes a thread and its neighbours
// behind one another (VEC), or every G-th entry.  UNITS * 8 entries a thread.  (Binary32 with 32 consecutive bytes a thread wrote and read half
// sectors: 2500 x 8192 forward 50 us instead of 29.)
template <typename T, bool VEC, int UNITS, int G, int ROWS, int STEPS, int BLOCK>
struct Feed {
    static constexpr int kRows = ROWS;                                     // taken together: one chain of exchanges and barriers for them
    static constexpr int kBlock = BLOCK;
    static constexpr int kSteps = STEPS;     // on their way or in use
    static constexpr int kDepth = kSteps * kRows;                          // ... in rows
    static constexpr int kUnitBytes = 8 * (int)sizeof(T);
    static constexpr int kTensorBytes = VEC ? UNITS * kBlock * kUnitBytes : (kBlock / G) * (UNITS * G * kUnitBytes + 32);     // a row of each group
    uint32_t base;                  // shared memory
    int tensors, cols, t;           // of a slot; of a row; this thread in its group
    int asked, taken;               // steps of kRows rows
    // The eight entries of a unit are in kParts parts of kPart; how many of a part's exist (of all of them: kPart or more).
    static constexpr int kPart = VEC ? 16 / (int)sizeof(T) : 8, kParts = 8 / kPart;
    static __device__ __forceinline__ int column(int u, int j, int t) { return VEC ? ((u * kParts + j / kPart) * G + t) * kPart + j % kPart : (u * 8 + j) * G + t; }
    static __device__ __forceinline__ int live(int u, int h, int cols, int t) { return VEC ? cols - column(u, h * kPart, t) : (cols - t + G - 1) / G - u * 8; }
    static __device__ __forceinline__ void copy16(uint32_t dst, const void *src, int live)
    {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(max(0, min(16, live))) : "memory");
    }
    __device__ __forceinline__ uint32_t slot(int step, int k, int tensor) const { return base + (uint32_t)(((step & (kSteps - 1)) * kRows + k) * tensors + tensor) * (uint32_t)kTensorBytes; }
    __device__ __forceinline__ uint32_t group_row(int step, int k, int tensor) const { return slot(step, k, tensor) + (uint32_t)((int)threadIdx.x / G * (UNITS * G * kUnitBytes + 32)); }
    // p: the k-th row of the step; [lo, hi): the matrix it is of
    __device__ __forceinline__ void ask(int k, int tensor, const T *p, const T *lo, const T *hi)
    {
        if constexpr (VEC) {
            const uint32_t dst = slot(asked, k, tensor) + threadIdx.x * 16u;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
#pragma unroll
                for (int h = 0; h < kParts; ++h) {
                    const int at = column(u, h * kPart, t), live = (cols - at) * (int)sizeof(T);
                    copy16(dst + (uint32_t)(u * kParts + h) * (uint32_t)(kBlock * 16), live > 0 ? p + at : lo, live);
                }
            }
        } else {
            // the 16-byte units that the row lies in, as they lie; at the ends of the matrix what does not belong to it is not read
            const uintptr_t first = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15, end = reinterpret_cast<uintptr_t>(p + cols);
            const uint32_t dst = group_row(asked, k, tensor);
            const int units = (int)((end - first + 15) >> 4);
            for (int i = t; i < units; i += G) {
                const uintptr_t at = first + (uintptr_t)i * 16;
                if (at >= reinterpret_cast<uintptr_t>(lo) && at + 16 <= reinterpret_cast<uintptr_t>(hi)) copy16(dst + (uint32_t)i * 16u, reinterpret_cast<const void *>(at), 16);
                else
#pragma unroll
                    for (int j = 0; j < 16; j += (int)sizeof(T)) {
                        const uintptr_t e = at + (uintptr_t)j;
                        if (e < reinterpret_cast<uintptr_t>(p) || e >= end) continue;
                        if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + (uint32_t)(i * 16 + j)), "r"(*reinterpret_cast<const uint32_t *>(e)) : "memory");
                        else asm volatile("st.shared.b16 [%0], %1;" ::"r"(dst + (uint32_t)(i * 16 + j)), "h"(*reinterpret_cast<const unsigned short *>(e)) : "memory");
                    }
            }
        }
    }
    __device__ __forceinline__ void asked_step()
    {
        asm volatile("cp.async.commit_group;" ::: "memory");
        ++asked;
    }
    // A thread's own copies of the next step have landed, and everyone's where entries are shared: then the slots of the step before are free.
    __device__ __forceinline__ void take()
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(kSteps - 2) : "memory");
        if (!VEC) group_sync<G, BLOCK>();
    }
    // Entries behind the row's end are `none`, or 0 where the rows start on 16 bytes (the copies put it there).
    __device__ __forceinline__ void floats(int step, int k, int tensor, const T *p, int u, float2 (&f)[4], float none = 0.0f) const
    {
        if constexpr (VEC) {
            const uint32_t src = slot(step, k, tensor) + threadIdx.x * 16u + (uint32_t)(u * kParts) * (uint32_t)(kBlock * 16);
            const uint4 a = lds_u128(src);
            if constexpr (sizeof(T) == 4) {
                const uint4 b = lds_u128(src + (uint32_t)(kBlock * 16));
                f[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
                f[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
                f[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
                f[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
            } else {
                unpack2(a.x, f[0].x, f[0].y, T());
                unpack2(a.y, f[1].x, f[1].y, T());
                unpack2(a.z, f[2].x, f[2].y, T());
                unpack2(a.w, f[3].x, f[3].y, T());
            }
        } else {
            // (what lies behind the row is read as well, and dropped)
            const uint32_t src = group_row(step, k, tensor) + (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) + (uint32_t)t * (uint32_t)sizeof(T);
            const int n = live(u, 0, cols, t);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (sizeof(T) == 4) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[j]) : "r"(src + (uint32_t)((u * 8 + j) * G * 4)));
                else {
                    unsigned short h;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(src + (uint32_t)((u * 8 + j) * G * 2)));
                    v[j] = to_f32(*reinterpret_cast<T *>(&h));
                }
                if (j >= n) v[j] = none;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = make_float2(v[2 * j], v[2 * j + 1]);
        }
    }
    static __device__ __forceinline__ void store(T *p, int u, int cols, int t, const float2 (&f)[4])
    {
        const float v[8] = {f[0].x, f[0].y, f[1].x, f[1].y, f[2].x, f[2].y, f[3].x, f[3].y};
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
            const int n = live(u, h, cols, t);
            T *o = p + column(u, h * kPart, t);
            if (VEC && n >= kPart) {
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(o) = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
                else store8(o, v);
            } else
#pragma unroll
                for (int j = 0; j < kPart; ++j)
                    if (j < n) o[VEC ? j : j * G] = from_f32<T>(v[h * kPart + j]);
        }
    }
    // The sum of a n without what a row does not have.
    __device__ __forceinline__ float2 existing(int u, const float2 (&n)[4], const float2 (&a)[4], float2 s) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = live(u, 2 * j / kPart, cols, t), i = 2 * j % kPart;
            if (i < e) s.x = fmaf(a[j].x, n[j].x, s.x);
            if (i + 1 < e) s.y = fmaf(a[j].y, n[j].y, s.y);
        }
        return s;
    }
    // Whether unit u has columns for this thread: what has none is left out, which is up to half of a row's units (the first never).
    __device__ __forceinline__ bool used(int u) const { return u == 0 || live(u, 0, cols, t) > 0; }
    // Weights of unit u's columns, `none` where there are none.
    static __device__ __forceinline__ void load_weight(const float *w, float none, int u, int cols, int t, float2 (&f)[4])
    {
        float v[8];
#pragma unroll
        for (int h = 0; h < 8; h += 4) {
            const int c = column(u, h, t);
            if (VEC && w != nullptr && c + 4 <= cols && (reinterpret_cast<uintptr_t>(w) & 15u) == 0) {
                const float4 a = *reinterpret_cast<const float4 *>(w + c);
                v[h] = a.x;
                v[h + 1] = a.y;
                v[h + 2] = a.z;
                v[h + 3] = a.w;
            } else
#pragma unroll
                for (int j = h; j < h + 4; ++j) v[j] = w != nullptr && column(u, j, t) < cols ? w[column(u, j, t)] : none;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = make_float2(v[2 * j], v[2 * j + 1]);
    }
};

// 1 / sqrt(v + eps) from the mean of the deviations and that of their squares; a NaN stays one.
__device__ __forceinline__ float rstd_of(float left, float square, float eps) { return 1.0f / sqrtf(max_nan(fmaf(-left, left, square), 0.0f) + eps); }

// SHARED: a row is shared by the blocks of a cluster.
template <typename T, bool VEC, int UNITS, int G, bool SHARED>
__global__ void __launch_bounds__(fwd_threads(G), fwd_blocks(G, UNITS))
norm_fwd_kernel(const NormDev P)
{
    static_assert(!SHARED || G == fwd_threads(G), "a block's own row");
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float buf1[2][Feed<T, VEC, UNITS, G, fwd_rows(sizeof(T)), fwd_steps(sizeof(T), UNITS), fwd_threads(G)>::kRows][32], buf2[2][2 * Feed<T, VEC, UNITS, G, fwd_rows(sizeof(T)), fwd_steps(sizeof(T), UNITS), fwd_threads(G)>::kRows][32];
    __shared__ float shared1[2][8][fwd_rows(sizeof(T))], shared2[2][8][2 * fwd_rows(sizeof(T))];
    typedef Feed<T, VEC, UNITS, G, fwd_rows(sizeof(T)), fwd_steps(sizeof(T), UNITS), fwd_threads(G)> F;
    const int t = (int)threadIdx.x % G, per = fwd_threads(G) / G;
    const int rank = SHARED ? (int)cluster_ctarank() : 0, from = SHARED ? rank * P.share : 0, cols = SHARED ? max(0, min(P.share, P.cols - from)) : P.cols;
    const int blocks = SHARED ? (int)gridDim.x / P.split : (int)gridDim.x, block = SHARED ? (int)blockIdx.x / P.split : (int)blockIdx.x;
    if (SHARED) cluster_sync_all();                     // (the others' shared memory is there)
    follow_previous();
    constexpr int kRows = F::kRows;
    RowSum<G, kRows, fwd_threads(G)> sum1{buf1, 0};
    RowSum<G, 2 * kRows, fwd_threads(G)> sum2{buf2, 0};
    ClusterSum<kRows> all1{shared1, 0, rank, P.split};
    ClusterSum<2 * kRows> all2{shared2, 0, rank, P.split};
    constexpr bool kKeep = UNITS <= 2;                  // gamma and beta stay in registers
    float2 gamma[kKeep ? UNITS : 1][4], beta[kKeep ? UNITS : 1][4];
    const float *gamma_in = P.gamma == nullptr ? nullptr : P.gamma + from, *beta_in = P.beta == nullptr ? nullptr : P.beta + from;
    const long long first = (long long)block * per + (int)threadIdx.x / G, step = (long long)blocks * per;
    const T *x = static_cast<const T *>(P.x) + from, *x_end = x + (P.rows - 1) * P.ldx + cols;
    F feed{smem_u32(ring), 1, cols, t, 0, 0};
    long long ahead = first;
    auto ask = [&] {
#pragma unroll
        for (int k = 0; k < kRows; ++k, ahead += step)
            if (ahead < P.rows) feed.ask(k, 0, x + ahead * P.ldx, x, x_end);
        feed.asked_step();
    };
    for (int i = 0; i < F::kSteps - 1; ++i) ask();
    if (kKeep)
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            F::load_weight(gamma_in, 1.0f, u, cols, t, gamma[kKeep ? u : 0]);
            F::load_weight(beta_in, 0.0f, u, cols, t, beta[kKeep ? u : 0]);
        }
    // (a step's second row may be behind the last: what lies in its slot is worked through and goes nowhere)
    for (long long row = first; row < P.rows; row += kRows * step) {
        feed.take();
        ask();
        float2 v[kRows][UNITS][4];
        float s[kRows], d2[2 * kRows], r[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            float2 a = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                if (!feed.used(u)) continue;
                feed.floats(feed.taken, k, 0, x + (row + k * step) * P.ldx, u, v[k][u]);
                a = add_2(a, add_2(add_2(v[k][u][0], v[k][u][1]), add_2(v[k][u][2], v[k][u][3])));
            }
            s[k] = a.x + a.y;
        }
        ++feed.taken;
        sum1(s);
        if (SHARED) all1(s);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const float m0 = s[k] * P.inv;
            float2 a = make_float2(0.0f, 0.0f), b = a;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                if (!feed.used(u)) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = F::live(u, 2 * j / F::kPart, cols, t), i = 2 * j % F::kPart;
                    float2 d = add_2(v[k][u][j], both(-m0));
                    if (i >= n) d.x = 0.0f;
                    if (i + 1 >= n) d.y = 0.0f;
                    v[k][u][j] = d;
                    a = add_2(a, d);
                    b = fma_2(d, d, b);
                }
            }
            d2[2 * k] = a.x + a.y;
            d2[2 * k + 1] = b.x + b.y;
            s[k] = m0;
        }
        sum2(d2);
        if (SHARED) all2(d2);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const float left = d2[2 * k] * P.inv;           // what the mean's rounding left
            r[k] = rstd_of(left, d2[2 * k + 1] * P.inv, P.eps);
            d2[2 * k] = left;
            if (t == 0 && rank == 0 && row + k * step < P.rows) {
                if (P.mean != nullptr) P.mean[row + k * step] = s[k] + left;
                if (P.rstd != nullptr) P.rstd[row + k * step] = r[k];
            }
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (!feed.used(u)) continue;
            if (!kKeep) {
                F::load_weight(gamma_in, 1.0f, u, cols, t, gamma[0]);
                F::load_weight(beta_in, 0.0f, u, cols, t, beta[0]);
            }
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[k][u][j] = fma_2(mul_2(add_2(v[k][u][j], both(-d2[2 * k])), both(r[k])), gamma[kKeep ? u : 0][j], beta[kKeep ? u : 0][j]);
                if (row + k * step < P.rows) F::store(static_cast<T *>(P.y) + from + (row + k * step) * P.ldy, u, cols, t, v[k][u]);
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// A row of any length by a block, read three times (the last two from L2): N entries a thread and step, kAhead steps on their way.
constexpr int kLong = 512;
template <typename T, bool VEC>
struct Strip {
    static constexpr int kN = VEC ? 8 : 1, kAhead = VEC ? 4 : 16, kSpan = kLong * kN * kAhead;
    float v[kAhead][kN];
    __device__ __forceinline__ void load(const T *p, int c0, int cols, float none)
    {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + (i * kLong + (int)threadIdx.x) * kN;
            if constexpr (VEC) {
                if (c + 8 <= cols) load8(p + c, v[i]);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] = c + j < cols ? to_f32(p[c + j]) : none;
            } else v[i][0] = c < cols ? to_f32(p[c]) : none;
        }
    }
    __device__ __forceinline__ void store(T *p, int c0, int cols) const
    {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + (i * kLong + (int)threadIdx.x) * kN;
            if constexpr (VEC) {
                if (c + 8 <= cols) store8(p + c, v[i]);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < cols) p[c + j] = from_f32<T>(v[i][j]);
            } else if (c < cols) p[c] = from_f32<T>(v[i][0]);
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(int c0, F f)      // f(entry, its column)
    {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j) f(v[i][j], c0 + (i * kLong + (int)threadIdx.x) * kN + j, i, j);
    }
};
// Weights of a strip's columns: 1 or 0 where there are none.
template <bool VEC>
__device__ __forceinline__ void load_strip(Strip<float, VEC> &s, const float *w, int c0, int cols, float none)
{
    if (w != nullptr && (!VEC || (reinterpret_cast<uintptr_t>(w) & 15u) == 0)) s.load(w, c0, cols, none);
    else s.each(c0, [&](float &v, int c, int, int) { v = w != nullptr && c < cols ? w[c] : none; });
}
template <typename T, bool VEC>
__global__ void __launch_bounds__(kLong)
norm_fwd_long_kernel(const NormDev P)
{
    __shared__ float buf1[2][1][32], buf2[2][2][32];
    typedef Strip<T, VEC> S;
    follow_previous();
    RowSum<kLong, 1, kLong> sum1{buf1, 0};
    RowSum<kLong, 2, kLong> sum2{buf2, 0};
    for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(P.x) + row * P.ldx;
        T *y = static_cast<T *>(P.y) + row * P.ldy;
        float s[1] = {0.0f}, d2[2] = {0.0f, 0.0f};
        S a;
        for (int c0 = 0; c0 < P.cols; c0 += S::kSpan) {
            a.load(x, c0, P.cols, 0.0f);
            a.each(c0, [&](float v, int, int, int) { s[0] += v; });
        }
        sum1(s);
        const float m0 = s[0] * P.inv;
        for (int c0 = 0; c0 < P.cols; c0 += S::kSpan) {
            a.load(x, c0, P.cols, m0);
            a.each(c0, [&](float v, int, int, int) {
                const float d = v - m0;
                d2[0] += d;
                d2[1] = fmaf(d, d, d2[1]);
            });
        }
        sum2(d2);
        const float left = d2[0] * P.inv;
        const float r = rstd_of(left, d2[1] * P.inv, P.eps);
        if (threadIdx.x == 0) {
            if (P.mean != nullptr) P.mean[row] = m0 + left;
            if (P.rstd != nullptr) P.rstd[row] = r;
        }
        for (int c0 = 0; c0 < P.cols; c0 += S::kSpan) {
            Strip<float, VEC> g, b;
            a.load(x, c0, P.cols, 0.0f);
            load_strip<VEC>(g, P.gamma, c0, P.cols, 1.0f);
            load_strip<VEC>(b, P.beta, c0, P.cols, 0.0f);
            a.each(c0, [&](float &v, int, int i, int j) { v = fmaf((v - m0 - left) * r, g.v[i][j], b.v[i][j]); });
            a.store(y, c0, P.cols);
        }
    }
}

// Whether n of a 0 behind the row's end is infinite.  It meets an a of 0 there, and the sum of a n has to be taken again without it.  (8192 x 4096 with
// this test once a row 43.3 us, without 42.3, with n of such entries made 0 in every row 43.9.)
__device__ __forceinline__ bool far_off(float mean, float r) { return fabsf(mean * r) > FLT_MAX; }

template <typename T, bool VEC, int UNITS, int G, bool SHARED>
__global__ void __launch_bounds__(kBwdThreads, 1)
norm_bwd_kernel(const NormDev P)
{
    static_assert(!SHARED || G == kBwdThreads, "a block's own row");
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float buf[2][2 * Feed<T, VEC, UNITS, G, bwd_rows(sizeof(T), UNITS), bwd_steps(sizeof(T), UNITS), kBwdThreads>::kRows][32];
    __shared__ float shared[2][8][2 * bwd_rows(sizeof(T), UNITS)];
    typedef Feed<T, VEC, UNITS, G, bwd_rows(sizeof(T), UNITS), bwd_steps(sizeof(T), UNITS), kBwdThreads> F;
    constexpr int per = kBwdThreads / G;
    const int t = (int)threadIdx.x % G, sub = (int)threadIdx.x / G;
    const int rank = SHARED ? (int)cluster_ctarank() : 0, from = SHARED ? rank * P.share : 0, cols = SHARED ? max(0, min(P.share, P.cols - from)) : P.cols;
    const int blocks = SHARED ? (int)gridDim.x / P.split : (int)gridDim.x, block = SHARED ? (int)blockIdx.x / P.split : (int)blockIdx.x;
    if (SHARED) cluster_sync_all();                     // (the others' shared memory is there)
    follow_previous();
    constexpr int kRows = F::kRows;
    RowSum<G, 2 * kRows, kBwdThreads> sum{buf, 0};
    ClusterSum<2 * kRows> all{shared, 0, rank, P.split};
    float2 gamma[UNITS][4], dg[UNITS][4], db[UNITS][4];
    const long long first = (long long)block * per + sub, step = (long long)blocks * per;
    const T *x = static_cast<const T *>(P.x) + from, *dy = static_cast<const T *>(P.dy) + from, *res = P.res != nullptr ? static_cast<const T *>(P.res) + from : nullptr;
    const bool dx_wanted = P.y != nullptr;
    const T *x_end = x + (P.rows - 1) * P.ldx + cols, *dy_end = dy + (P.rows - 1) * P.lddy + cols, *res_end = res + (P.rows - 1) * P.ldr + cols;
    F feed{smem_u32(ring), res != nullptr ? 3 : 2, cols, t, 0, 0};
    long long ahead = first;
    float next_mean[kRows], next_r[kRows];
    auto ask = [&] {
#pragma unroll
        for (int k = 0; k < kRows; ++k, ahead += step) {
            if (ahead < P.rows) {
                feed.ask(k, 0, x + ahead * P.ldx, x, x_end);
                feed.ask(k, 1, dy + ahead * P.lddy, dy, dy_end);
                if (res != nullptr) feed.ask(k, 2, res + ahead * P.ldr, res, res_end);
            }
        }
        feed.asked_step();
    };
    for (int i = 0; i < F::kSteps - 1; ++i) ask();
    auto statistics = [&](long long row) {
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const long long at = row + k * step;
            next_mean[k] = at < P.rows ? P.mean[at] : 0.0f;
            next_r[k] = at < P.rows ? P.rstd[at] : 0.0f;
        }
    };
    statistics(first);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        F::load_weight(P.gamma == nullptr ? nullptr : P.gamma + from, 1.0f, u, cols, t, gamma[u]);
#pragma unroll
        for (int j = 0; j < 4; ++j) dg[u][j] = db[u][j] = make_float2(0.0f, 0.0f);
    }
    constexpr bool kLate = SHARED && F::kSteps > 2;
    if constexpr (kLate) {
        // While a row's sums go round, the next row's are taken; the first is read from shared memory once more for dx, so two slots are in use.
        // (Waited for in place: 1220 x 16800 bf16 with a residual 114 us, so 96.
        // Binary32 has shared memory for two slots only, and waits.)
        static_assert(kRows == 1, "a row at a time");
        float mean0 = 0.0f, r0 = 0.0f;                  // of the row before
        auto entries = [&](int at, long long row, float mean, float r, int u, float2 (&n)[4], float2 (&a)[4]) {
            feed.floats(at, 0, 0, x + row * P.ldx, u, n, mean);
            feed.floats(at, 0, 1, dy + row * P.lddy, u, a);
#pragma unroll
            for (int j = 0; j < 4; ++j) n[j] = mul_2(add_2(n[j], both(-mean)), both(r));
        };
        for (long long row = first;; row += step) {
            const bool live = row < P.rows;
            const float mean = next_mean[0], r = next_r[0];
            float s[2];
            if (live) {
                feed.take();
                statistics(row + step);
                float2 s0 = make_float2(0.0f, 0.0f), s1 = s0;
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    if (!feed.used(u)) continue;
                    float2 n[4], a[4];
                    entries(feed.taken, row, mean, r, u, n, a);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        dg[u][j] = fma_2(a[j], n[j], dg[u][j]);
                        db[u][j] = add_2(db[u][j], a[j]);
                        a[j] = mul_2(a[j], gamma[u][j]);
                        s0 = add_2(s0, a[j]);
                        s1 = fma_2(a[j], n[j], s1);
                    }
                }
                if (VEC && far_off(mean, r)) {
                    s1 = make_float2(0.0f, 0.0f);
#pragma unroll 1
                    for (int u = 0; u < UNITS; ++u) {
                        if (!feed.used(u)) continue;
                        float2 n[4], a[4], g[4];
                        entries(feed.taken, row, mean, r, u, n, a);
                        F::load_weight(P.gamma == nullptr ? nullptr : P.gamma + from, 1.0f, u, cols, t, g);
#pragma unroll
                        for (int j = 0; j < 4; ++j) a[j] = mul_2(a[j], g[j]);
                        s1 = feed.existing(u, n, a, s1);
                    }
                }
                s[0] = s0.x + s0.y;
                s[1] = s1.x + s1.y;
                if (dx_wanted) sum(s);
            }
            if (dx_wanted && row != first) {
                float all_s[2];
                all.receive(all_s);
                const float ma = all_s[0] * P.inv, man = all_s[1] * P.inv;
                T *dx = static_cast<T *>(P.y) + from + (row - step) * P.ldy;
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    if (!feed.used(u)) continue;
                    float2 n[4], a[4], f[4];
                    entries(feed.taken - 1, row - step, mean0, r0, u, n, a);
                    if (res != nullptr) feed.floats(feed.taken - 1, 0, 2, res + (row - step) * P.ldr, u, f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        a[j] = mul_2(fma_2(n[j], both(-man), fma_2(a[j], gamma[u][j], both(-ma))), both(r0));
                        if (res != nullptr) a[j] = add_2(a[j], f[j]);
                    }
                    F::store(dx, u, cols, t, a);
                }
            }
            if (!live) break;
            if (dx_wanted) all.send(s);
            mean0 = mean;
            r0 = r;
            if (!VEC) group_sync<G, kBwdThreads>();     // (the others have read what is overwritten now)
            ask();
            ++feed.taken;
        }
    }
    for (long long row = first; !kLate && row < P.rows; row += kRows * step) {
        feed.take();
        float mean[kRows], r[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            mean[k] = next_mean[k];
            r[k] = next_r[k];
        }
        ask();
        statistics(row + kRows * step);
        float2 n[kRows][UNITS][4], a[kRows][UNITS][4];
        float s[2 * kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            float2 s0 = make_float2(0.0f, 0.0f), s1 = s0;
            if (row + k * step < P.rows) {
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    if (!feed.used(u)) continue;
                    feed.floats(feed.taken, k, 0, x + (row + k * step) * P.ldx, u, n[k][u], mean[k]);
                    feed.floats(feed.taken, k, 1, dy + (row + k * step) * P.lddy, u, a[k][u]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // (beyond the row dy is 0, and with it every sum's term)
                        n[k][u][j] = mul_2(add_2(n[k][u][j], both(-mean[k])), both(r[k]));
                        dg[u][j] = fma_2(a[k][u][j], n[k][u][j], dg[u][j]);
                        db[u][j] = add_2(db[u][j], a[k][u][j]);
                        a[k][u][j] = mul_2(a[k][u][j], gamma[u][j]);
                        s0 = add_2(s0, a[k][u][j]);
                        s1 = fma_2(a[k][u][j], n[k][u][j], s1);
                    }
                }
            }
            if (VEC && far_off(mean[k], r[k])) {
                s1 = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int u = 0; u < UNITS; ++u)
                    if (feed.used(u)) s1 = feed.existing(u, n[k][u], a[k][u], s1);
            }
            s[2 * k] = s0.x + s0.y;
            s[2 * k + 1] = s1.x + s1.y;
        }
        if (dx_wanted) {
            sum(s);
            if (SHARED) all(s);
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                if (row + k * step >= P.rows) break;
                const float ma = s[2 * k] * P.inv, man = s[2 * k + 1] * P.inv;
                T *dx = static_cast<T *>(P.y) + from + (row + k * step) * P.ldy;
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    if (!feed.used(u)) continue;
                    float2 f[4];
                    if (res != nullptr) feed.floats(feed.taken, k, 2, res + (row + k * step) * P.ldr, u, f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        a[k][u][j] = mul_2(fma_2(n[k][u][j], both(-man), add_2(a[k][u][j], both(-ma))), both(r[k]));
                        if (res != nullptr) a[k][u][j] = add_2(a[k][u][j], f[j]);
                    }
                    F::store(dx, u, cols, t, a[k][u]);
                }
            }
        }
        ++feed.taken;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!P.weight) return;
    // the block's sums of its columns (one block: the result), over its groups where the rows came through
    float *pg = P.part_g == nullptr ? nullptr : P.part_g + (long long)block * P.cols + from, *pb = P.part_b == nullptr ? nullptr : P.part_b + (long long)block * P.cols + from;
    constexpr int kCols = UNITS * 8 * G;
    static_assert(per * kCols * sizeof(float) <= 2 * F::kDepth * F::kTensorBytes, "shared memory");
    float *sums = reinterpret_cast<float *>(ring);
    for (int pass = 0; pass < 2; ++pass) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 v = pass ? db[u][j] : dg[u][j];
                sums[sub * kCols + F::column(u, 2 * j, t)] = v.x;
                sums[sub * kCols + F::column(u, 2 * j + 1, t)] = v.y;
            }
        __syncthreads();
        float *o = pass ? pb : pg;
        if (o != nullptr)
            for (int c = (int)threadIdx.x; c < cols; c += kBwdThreads) {
                float s = sums[c];
#pragma unroll
                for (int k = 1; k < per; ++k) s += sums[k * kCols + c];
                o[c] = s;
            }
    }
}

// A row of any length by a block, dx only; read twice.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kLong)
norm_bwd_long_kernel(const NormDev P)
{
    __shared__ float buf[2][2][32];
    typedef Strip<T, VEC> S;
    follow_previous();
    RowSum<kLong, 2, kLong> sum{buf, 0};
    for (long long row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(P.x) + row * P.ldx, *dy = static_cast<const T *>(P.dy) + row * P.lddy;
        const T *res = P.res != nullptr ? static_cast<const T *>(P.res) + row * P.ldr : nullptr;
        T *dx = static_cast<T *>(P.y) + row * P.ldy;
        const float mean = P.mean[row], r = P.rstd[row];
        float s[2] = {0.0f, 0.0f};
        S n, a;
        Strip<float, VEC> g;
        for (int c0 = 0; c0 < P.cols; c0 += S::kSpan) {
            n.load(x, c0, P.cols, mean);
            a.load(dy, c0, P.cols, 0.0f);
            load_strip<VEC>(g, P.gamma, c0, P.cols, 1.0f);
            a.each(c0, [&](float v, int, int i, int j) {
                s[0] = fmaf(v, g.v[i][j], s[0]);
                s[1] = fmaf(v * g.v[i][j], (n.v[i][j] - mean) * r, s[1]);
            });
        }
        sum(s);
        const float ma = s[0] * P.inv, man = s[1] * P.inv;
        for (int c0 = 0; c0 < P.cols; c0 += S::kSpan) {
            n.load(x, c0, P.cols, 0.0f);
            a.load(dy, c0, P.cols, 0.0f);
            load_strip<VEC>(g, P.gamma, c0, P.cols, 1.0f);
            a.each(c0, [&](float &v, int, int i, int j) { v = r * (v * g.v[i][j] - ma - (n.v[i][j] - mean) * r * man); });
            if (res != nullptr) {
                n.load(res, c0, P.cols, 0.0f);
                a.each(c0, [&](float &v, int, int i, int j) { v += n.v[i][j]; });
            }
            a.store(dx, c0, P.cols);
        }
    }
}

// Columns' sums of dy n and dy over a chunk of rows, for rows that are too long to be kept: a thread eight columns, or one.  Runs before the
// kernel above, which may write dx over dy.
constexpr int kColThreads = 128, kColRows = 4;
template <typename T, bool VEC>
__global__ void __launch_bounds__(kColThreads)
norm_columns_kernel(const NormDev P, int chunk)
{
    constexpr int kN = VEC ? 8 : 1, kAhead = VEC ? kColRows : 16;
    follow_previous();
    const int c = ((int)blockIdx.x * kColThreads + (int)threadIdx.x) * kN;
    const long long r0 = (long long)blockIdx.y * chunk, r1 = r0 + chunk < P.rows ? r0 + chunk : P.rows;
    if (c >= P.cols) return;
    const T *x = static_cast<const T *>(P.x) + c, *dy = static_cast<const T *>(P.dy) + c;
    float g[kN], b[kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) g[j] = b[j] = 0.0f;
    auto load = [&](const T *p, float (&v)[kN]) {
        if constexpr (VEC) {
            if (c + 8 <= P.cols) load8(p, v);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = c + j < P.cols ? to_f32(p[j]) : 0.0f;
        } else v[0] = to_f32(*p);
    };
    for (long long row = r0; row < r1; row += kAhead) {
        float xv[kAhead][kN], dv[kAhead][kN], m[kAhead], r[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const bool live = row + i < r1;
            const long long at = live ? row + i : r1 - 1;
            load(x + at * P.ldx, xv[i]);
            load(dy + at * P.lddy, dv[i]);
            m[i] = P.mean[at];
            r[i] = P.rstd[at];
            if (!live)
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    dv[i][j] = 0.0f;
                    xv[i][j] = m[i];
                }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                if (row + i < r1) g[j] = fmaf(dv[i][j], (xv[i][j] - m[i]) * r[i], g[j]);
                b[j] += dv[i][j];
            }
    }
    float *pg = P.part_g == nullptr ? nullptr : P.part_g + (long long)blockIdx.y * P.cols, *pb = P.part_b == nullptr ? nullptr : P.part_b + (long long)blockIdx.y * P.cols;
#pragma unroll
    for (int j = 0; j < kN; ++j)
        if (c + j < P.cols) {
            if (pg != nullptr) pg[c + j] = g[j];
            if (pb != nullptr) pb[c + j] = b[j];
        }
}

// The blocks' sums, in a fixed order: 32 columns a block, 32 threads a column.  (With eight it took 13 us for 444 blocks' sums.)
constexpr int kSumLanes = 32;
__global__ void __launch_bounds__(32 * kSumLanes)
norm_sum_kernel(const float *part_g, const float *part_b, int parts, int cols, float *dgamma, float *dbeta)
{
    __shared__ float sums[2][kSumLanes][33];
    follow_previous();
    const int lane = (int)threadIdx.x & 31, k = (int)threadIdx.x >> 5, c = (int)blockIdx.x * 32 + lane;
    float g = 0.0f, b = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int p = k; p < parts; p += kSumLanes) {
            g += part_g[(long long)p * cols + c];
            b += part_b[(long long)p * cols + c];
        }
    sums[0][k][lane] = g;
    sums[1][k][lane] = b;
    __syncthreads();
    if (k < 2 && c < cols) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kSumLanes; ++i) s += sums[k][i][lane];
        float *o = k == 0 ? dgamma : dbeta;
        if (o != nullptr) o[c] = s;
    }
}

constexpr int kPlanSms = 148;                   // sizes of workspaces and the order of sums are planned for a B200
constexpr size_t kHeadBytes = 256;
// Columns of a block's row; a cluster of two, four or eight blocks has as many times more.  (So many clusters the device runs at once for
// certain: with more, 1000 x 32000 forward took 112 us.)
constexpr int kFwdMost = 16384, kBwdMost = 8192;
int blocks_of_row(int cols, int most) { return cols <= most ? 1 : (cols <= 2 * most ? 2 : (cols <= 4 * most ? 4 : 8)); }
long long rows_at_once(int split) { return split == 1 ? kPlanSms : (split == 2 ? kPlanSms / 2 : (split == 4 ? 32 : 14)); }
constexpr int kFewSteps = 4;

// Blocks of the backward pass, which is how many sums there are of a column.
int bwd_parts(int rows, int cols, int *chunk = nullptr)
{
    if (cols > 8 * kBwdMost) {
        const long long across = ((long long)cols + kColThreads * 8 - 1) / (kColThreads * 8);      // (of the form with eight columns a thread)
        long long chunks = 8 * kPlanSms / across;
        const long long most = ((long long)rows + 15) / 16;
        if (chunks > most) chunks = most;
        if (chunks < 1) chunks = 1;
        const long long per = (rows + chunks - 1) / chunks;
        if (chunk != nullptr) *chunk = (int)per;
        return (int)((rows + per - 1) / per);
    }
    // (few rows: a block that takes them one after the other is through before a second kernel has added the sums of several)
    const int G = cols <= 512 ? 32 : (cols <= 2048 ? 128 : (cols <= 4096 ? 256 : 512));
    const long long per = kBwdThreads / G, blocks = (rows + per - 1) / per, most = rows_at_once(blocks_of_row(cols, kBwdMost));
    if (blocks <= kFewSteps) return 1;
    return (int)(blocks < most ? blocks : most);
}

// Shared memory of a block beyond what every kernel has is asked for once per device.
int allow_smem(const void *kernel, size_t bytes, bool (&done)[64])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
    if (done[dev]) return CDL_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return CDL_ERR_LAUNCH;
    }
    done[dev] = true;
    return CDL_OK;
}
// `groups` blocks, or clusters of as many blocks as share a row.
template <bool SHARED>
int go(void (*kernel)(const NormDev), NormDev P, int split, long long groups, int threads, size_t bytes, cudaStream_t st)
{
    if (!SHARED) return launch_following(kernel, dim3((unsigned)groups), dim3((unsigned)threads), bytes, st, (const NormDev)P);
    P.split = split;
    P.share = ((P.cols + P.split - 1) / P.split + 7) / 8 * 8;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)P.split;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(groups * P.split));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, (const NormDev)P) != cudaSuccess) {
        (void)cudaGetLastError();
        return CDL_ERR_LAUNCH;
    }
    return CDL_OK;
}
template <typename T, bool VEC, int UNITS, int G, bool SHARED>
int go_fwd(const NormDev &P, cudaStream_t st)
{
    typedef Feed<T, VEC, UNITS, G, fwd_rows(sizeof(T)), fwd_steps(sizeof(T), UNITS), fwd_threads(G)> F;
    const long long per = fwd_threads(G) / G, blocks = (P.rows + per - 1) / per;
    const int split = SHARED ? blocks_of_row(P.cols, kFwdMost) : 1;
    const long long most = SHARED ? rows_at_once(split) : (long long)kPlanSms * fwd_blocks(G, UNITS);
    constexpr size_t kBytes = (size_t)F::kDepth * F::kTensorBytes;
    static bool done[64];
    const int rc = allow_smem(reinterpret_cast<const void *>(&norm_fwd_kernel<T, VEC, UNITS, G, SHARED>), kBytes, done);
    if (rc != CDL_OK) return rc;
    return go<SHARED>(&norm_fwd_kernel<T, VEC, UNITS, G, SHARED>, P, split, blocks < most ? blocks : most, fwd_threads(G), kBytes, st);
}
template <typename T, bool VEC>
int launch_fwd(const NormDev &P, cudaStream_t st)
{
    if (P.cols <= 256) return go_fwd<T, VEC, 1, 32, false>(P, st);
    if (P.cols <= 512) return go_fwd<T, VEC, 2, 32, false>(P, st);
    if (P.cols <= 1024) return go_fwd<T, VEC, 1, 128, false>(P, st);
    if (P.cols <= 2048) return go_fwd<T, VEC, 2, 128, false>(P, st);
    if (P.cols <= 4096) return go_fwd<T, VEC, 2, 256, false>(P, st);
    if (P.cols <= 8192) return go_fwd<T, VEC, 2, 512, false>(P, st);
    if (P.cols <= kFwdMost) return go_fwd<T, VEC, 4, 512, false>(P, st);
    if (P.cols <= 8 * kFwdMost) return go_fwd<T, VEC, 4, 512, true>(P, st);
    const int most = kPlanSms * 4;
    return launch_following(&norm_fwd_long_kernel<T, VEC>, dim3((unsigned)(P.rows < most ? P.rows : most)), dim3(kLong), 0, st, P);
}
template <typename T, bool VEC, int UNITS, int G, bool SHARED>
int go_bwd(const NormDev &P, cudaStream_t st)
{
    typedef Feed<T, VEC, UNITS, G, bwd_rows(sizeof(T), UNITS), bwd_steps(sizeof(T), UNITS), kBwdThreads> F;
    constexpr size_t kBytes = (size_t)F::kDepth * F::kTensorBytes;      // a tensor
    static bool done[64];
    const int rc = allow_smem(reinterpret_cast<const void *>(&norm_bwd_kernel<T, VEC, UNITS, G, SHARED>), 3 * kBytes, done);
    if (rc != CDL_OK) return rc;
    return go<SHARED>(&norm_bwd_kernel<T, VEC, UNITS, G, SHARED>, P, blocks_of_row(P.cols, kBwdMost), bwd_parts(P.rows, P.cols), kBwdThreads, (P.res != nullptr ? 3 : 2) * kBytes, st);
}
template <typename T, bool VEC>
int launch_bwd(const NormDev &P, cudaStream_t st)
{
    if (P.cols <= 256) return go_bwd<T, VEC, 1, 32, false>(P, st);
    if (P.cols <= 512) return go_bwd<T, VEC, 2, 32, false>(P, st);
    if (P.cols <= 1024) return go_bwd<T, VEC, 1, 128, false>(P, st);
    if (P.cols <= 2048) return go_bwd<T, VEC, 2, 128, false>(P, st);
    if (P.cols <= 4096) return go_bwd<T, VEC, 2, 256, false>(P, st);
    if (P.cols <= kBwdMost) return go_bwd<T, VEC, 2, 512, false>(P, st);
    if (P.cols <= 8 * kBwdMost) return go_bwd<T, VEC, 2, 512, true>(P, st);
    if (P.weight) {
        int chunk = 1;
        const int parts = bwd_parts(P.rows, P.cols, &chunk);
        const int rc = launch_following(&norm_columns_kernel<T, VEC>, dim3((unsigned)((P.cols + kColThreads * (VEC ? 8 : 1) - 1) / (kColThreads * (VEC ? 8 : 1))), (unsigned)parts), dim3(kColThreads), 0, st, P, chunk);
        if (rc != CDL_OK) return rc;
    }
    if (P.y == nullptr) return CDL_OK;
    const int most = kPlanSms * 4;
    return launch_following(&norm_bwd_long_kernel<T, VEC>, dim3((unsigned)(P.rows < most ? P.rows : most)), dim3(kLong), 0, st, P);
}

template <typename T>
int launch_typed(const NormDev &P, bool backward, cudaStream_t st)
{
    auto aligned = [&](const void *p, long long ld) {
        return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (P.rows == 1 || (ld * (long long)sizeof(T)) % 16 == 0));
    };
    const bool vec = aligned(P.x, P.ldx) && aligned(P.y, P.ldy) && aligned(P.dy, P.lddy) && aligned(P.res, P.ldr);
    if (backward) return vec ? launch_bwd<T, true>(P, st) : launch_bwd<T, false>(P, st);
    return vec ? launch_fwd<T, true>(P, st) : launch_fwd<T, false>(P, st);
}
int launch_norm(const NormDev &P, int type, bool backward, cudaStream_t st)
{
    switch (type) {
    case CDL_F32: return launch_typed<float>(P, backward, st);
    case CDL_BF16: return launch_typed<__nv_bfloat16>(P, backward, st);
    default: return launch_typed<__half>(P, backward, st);
    }
}

bool bad_extents(int32_t rows, int32_t cols) { return rows < 0 || cols < 0 || rows > kMostExtent || cols > kMostExtent; }
bool odd4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

}  // namespace
}  // namespace cdl

extern "C" size_t cdl_layernorm_workspace_bytes(int32_t rows, int32_t cols)
{
    using namespace cdl;
    if (bad_extents(rows, cols)) return 0;
    if (rows == 0 || cols == 0) return kHeadBytes;
    return kHeadBytes + 2 * sizeof(float) * (size_t)bwd_parts(rows, cols) * (size_t)cols;
}

extern "C" int cdl_layernorm_fwd(const void *x, int64_t ldx, int32_t type, const float *gamma, const float *beta, int32_t rows, int32_t cols,
                                 float eps, void *y, int64_t ldy, float *mean, float *rstd, void *stream)
{
    using namespace cdl;
    if (bad_extents(rows, cols) || !valid_type(type)) return CDL_ERR_ARG;
    if (!(eps >= 0.0f) || !isfinite(eps)) return CDL_ERR_RANGE;
    if (rows == 0 || cols == 0) return CDL_OK;
    if (x == nullptr || y == nullptr || (rows > 1 && (ldx < cols || ldy < cols))) return CDL_ERR_ARG;
    if (misaligned(x, type) || misaligned(y, type) || odd4(gamma) || odd4(beta) || odd4(mean) || odd4(rstd)) return CDL_ERR_ALIGN;
    const int rc = check_device();
    if (rc != CDL_OK) return rc;
    NormDev P = {};
    P.x = x;
    P.ldx = ldx;
    P.y = y;
    P.ldy = ldy;
    P.gamma = gamma;
    P.beta = beta;
    P.mean = mean;
    P.rstd = rstd;
    P.rows = rows;
    P.cols = cols;
    P.eps = eps;
    P.inv = (float)(1.0 / (double)cols);
    return launch_norm(P, type, false, static_cast<cudaStream_t>(stream));
}

extern "C" int cdl_layernorm_bwd(const void *dy, int64_t lddy, const void *x, int64_t ldx, int32_t type, const float *gamma, const float *mean,
                                 const float *rstd, int32_t rows, int32_t cols, const void *residual, int64_t ldr, void *dx, int64_t lddx,
                                 float *dgamma, float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    using namespace cdl;
    if (bad_extents(rows, cols) || !valid_type(type)) return CDL_ERR_ARG;
    if (cols == 0) return CDL_OK;
    const bool weight = dgamma != nullptr || dbeta != nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (odd4(dgamma) || odd4(dbeta)) return CDL_ERR_ALIGN;
    if (rows > 0) {
        if (dy == nullptr || x == nullptr || mean == nullptr || rstd == nullptr || (dx == nullptr && !weight)) return CDL_ERR_ARG;
        if (rows > 1 && (lddy < cols || ldx < cols || (dx != nullptr && (lddx < cols || (residual != nullptr && ldr < cols))))) return CDL_ERR_ARG;
        if (misaligned(dy, type) || misaligned(x, type) || misaligned(dx, type) || misaligned(residual, type) || odd4(gamma) || odd4(mean) || odd4(rstd)) return CDL_ERR_ALIGN;
        if (weight && (ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < cdl_layernorm_workspace_bytes(rows, cols))) return CDL_ERR_WORKSPACE;
    } else if (!weight) return CDL_OK;
    int rc = check_device();
    if (rc != CDL_OK) return rc;
    const int parts = rows > 0 ? bwd_parts(rows, cols) : 0;
    NormDev P = {};
    P.weight = weight ? 1 : 0;
    P.part_g = ws != nullptr ? reinterpret_cast<float *>(static_cast<char *>(ws) + kHeadBytes) : nullptr;
    P.part_b = ws != nullptr ? P.part_g + (size_t)parts * (size_t)cols : nullptr;
    if (parts == 1) {
        P.part_g = dgamma;
        P.part_b = dbeta;
    }
    if (rows > 0) {
        P.x = x;
        P.ldx = ldx;
        P.dy = dy;
        P.lddy = lddy;
        P.res = dx != nullptr ? residual : nullptr;
        P.ldr = ldr;
        P.y = dx;
        P.ldy = lddx;
        P.gamma = gamma;
        P.mean = const_cast<float *>(mean);
        P.rstd = const_cast<float *>(rstd);
        P.rows = rows;
        P.cols = cols;
        P.inv = (float)(1.0 / (double)cols);
        rc = launch_norm(P, type, true, st);
        if (rc != CDL_OK || !weight || parts == 1) return rc;
    }
    return launch_following(&norm_sum_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(32 * kSumLanes), 0, st, (const float *)P.part_g, (const float *)P.part_b, parts, (int)cols,
                            dgamma, dbeta);
}
