// Linear layers on 16-bit operands, forward and backward, with everything that belongs to an output entry in the product's epilogue:
//   forward   out = act(A W^T + bias) + residual, optionally z = A W^T + bias kept in 8 bits      A, W K-major
//   data      dA = (dY W) act'(z8) + residual                                                     dY K-major, W MN-major
//   weight    dW = dY^T A (+ dW), dbias = sum over rows of dY                                     both MN-major
// One tensor-core kernel (TMA + tcgen05 kind::f16, binary32 accumulators in TMEM) for the three: they differ in which dimension of a
// stored matrix is contiguous.
//
// The tensor cores' sums are cut off, not rounded, so an accumulator loses up to 2^-24 of itself with every instruction: over a
// reduction of 8192 that is 1e-5, and without a limit where the reduction has none.  So a tile is summed in segments, which the
// epilogue warps take out of TMEM into registers (128 a thread) while the next segment's products run in the other half of TMEM: 8
// stages where the result is binary32, off by 4.8e-7 of the norm (12 by 7e-7; a binary32 product by 3e-7 to 1e-6), 16 where it has 16
// bits, by 9e-7, with a checkpoint or without, so that the result is the same.  A segment's hand-over costs some 1200 cycles of the
// products' 520 a stage, and the last one holds its half of TMEM during the epilogue: 8192 x 8192 x 2048 to 16 bits 212 us, with GELU and
// checkpoint 262, to binary32 254; 16-bit results in one segment 205 and 241 to 253, binary32 ones in segments of 12 stages 243.
// A finished tile leaves TMEM a row a lane, 32 columns at a time, and goes out by TMA; where the output's rows do not start on 16 bytes it is
// turned through shared memory and stored with neighbouring lanes on neighbouring columns.
// Tiles: 256 x 256 per CTA pair (cta_group::2), or 128 x 128 per CTA where there are few; 64 reduced entries (128 bytes) a stage.
// The stages of a last, partly filled round are one sequence, cut into as many runs as there are CTAs (pairs); tiles that runs share
// are added in the order of the runs, and finished, by a second kernel.  One to eight rows of A have a form of their own.
// Bound by the tensor cores, and under load by the power cap (8192 x 8192 x 2048 212 us, 1300 TFLOP/s; 8192^3 797 to 814 us); with much epilogue
// and few reduced entries by its instructions (64 reduced entries: 42 us, with GELU 82).  Every wait is bounded.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <string.h>

#include "cdl_act.cuh"
#include "cdl_internal.h"
#include "cdl_linear.cuh"
#include "cdl_lowp.cuh"
#include "cdl_tc.cuh"
#include "cdl_wait.cuh"

namespace cdl {
namespace {

enum LinearMode { FORWARD = 0, DATA = 1, WEIGHT = 2 };
struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

constexpr int kEpiWarps = 8;
constexpr int kThreads = 128 + 32 * kEpiWarps;         // a warpgroup that feeds the others, two of epilogue warps
// Registers: an epilogue thread holds 128 sums, more than an even share of the register file (168 for 384 threads) leaves room for.
// The first warpgroup gives up what it does not need: 128 * 88 + 256 * 208 = 384 * 168.
constexpr int kRegsLaunch = 168, kRegsDrive = 88, kRegsEpilogue = 208;
static_assert(128 * kRegsDrive + 32 * kEpiWarps * kRegsEpilogue <= kThreads * kRegsLaunch, "register shares");
constexpr int kBK = 64;                                // reduced entries of a stage (128 bytes)
// Stages that are summed in TMEM, for binary32 and for 16-bit results.
constexpr int kSegment32 = 8, kSegment16 = 16;
constexpr int kSlope = 8;                              // + CDL_ACT_*: the derivative instead of the activation
constexpr int kBlockBytes = 128 * 128;                 // operand block of 128 rows
constexpr int kOutWarpBytes = 32 * 128;
constexpr int kStages = 6;
constexpr uint32_t kStageBytes = 2u * (uint32_t)kBlockBytes;
constexpr int kRingBytes = kStages * (int)kStageBytes;
constexpr int kSmemBytes = 1024 + kRingBytes + kEpiWarps * kOutWarpBytes;
static_assert(kSmemBytes + 1024 + 512 <= 227 * 1024, "shared memory, with what is declared in the kernel");
constexpr unsigned long long kWaitNs = 2000000000ull;
// An epilogue's wait is for all stages of a tile, which take up to 0.6 us each: 2^24 of them are five to ten seconds of valid work.
constexpr unsigned long long kWaitStageNs = 2000ull;

struct LinearParams {
    int mode;
    int R;                          // reduced extent
    int KB;                         // ... in stages
    int tiles_i, tiles_j, slots;
    uint32_t fmt;                   // of the operands: 0 binary16, 1 bfloat16
    int a_rows, b_rows;             // rows of a K-major box
    // The first `whole` tiles are taken as they are; the stages of those behind them are cut into `ranges` runs of `run` stages,
    // the pieces of run r and tile t (counted from `whole`) at r + t.
    int whole, ranges, run;
    int splits;                     // CTAs of a cluster that share a tile
    float *part;                    // [r + t][rows of a tile][256]
    int *status;
    LinearOut out;
    int out_tma, out_cols;          // the output leaves by TMA: these columns of it (whole units of 16 bytes), the threads store the others
};
struct LinearMaps {
    CUtensorMap a, b, o;
};

// The epilogue goes through a row's 128 columns in pieces of 32, a row a lane: the entries' chains of dependent instructions run side
// by side, and what depends on the call is looked up once a piece.  (Four columns a lane, looked up in every step, took 30000 cycles
// for a 256 x 256 tile, four times as long as the products of a reduction of 1024; sixteen columns a piece 12000.)
constexpr int kPiece = 32;
template <int ACT>
__device__ __forceinline__ void slope_piece(float (&v)[kPiece], const uint32_t (&w)[kPiece / 4], float zscale)
{
#pragma unroll
    for (int j = 0; j < kPiece; j += 2) {
        const float2 d = mul_2(make_float2(v[j], v[j + 1]), act_pair<ACT, false, true>(mul_2(fp8_value2(w[j >> 2] >> (8 * (j & 2))), both(zscale))).slope);
        v[j] = d.x;
        v[j + 1] = d.y;
    }
}
__device__ __forceinline__ void put_unit(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// A piece's results by TMA, 64 bytes of the warp's rows at a time through two buffers in turn; the residual is added on the way.
template <typename T>
__device__ __forceinline__ void send_piece(const LinearParams &P, const CUtensorMap *map_o, float (&v)[kPiece], uint32_t wbuf, uint32_t &turn, int lane, int row0, int c0)
{
    constexpr int kBox = 64 / (int)sizeof(T), kUnit = 16 / (int)sizeof(T);      // columns of a box, of 16 bytes
    const LinearOut &E = P.out;
    const int row = row0 + lane;
    const bool live = row < E.I;
    if (E.res != nullptr) {
        const T *res = static_cast<const T *>(E.res) + (long long)row * E.ldr + c0;
        uint4 q[kPiece / kUnit];
#pragma unroll
        for (int i = 0; i < kPiece / kUnit; ++i) q[i] = live && c0 + (i + 1) * kUnit <= P.out_cols ? *reinterpret_cast<const uint4 *>(res + i * kUnit) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < kPiece / kUnit; ++i) {
            const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (sizeof(T) == 4) v[4 * i + k] += __uint_as_float(w[k]);
                else {
                    float lo, hi;
                    unpack2(w[k], lo, hi, T());
                    v[8 * i + 2 * k] += lo;
                    v[8 * i + 2 * k + 1] += hi;
                }
            }
        }
    }
#pragma unroll
    for (int b = 0; b < kPiece / kBox; ++b) {
        const int cb = c0 + b * kBox;
        if (cb >= P.out_cols) break;
        if (lane == 0) bulk_wait_read<1>();                // the store that last used this buffer has read it
        __syncwarp();
        const uint32_t src = wbuf + turn, dst = src + (uint32_t)lane * 64u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = dst + (uint32_t)((i ^ ((lane >> 1) & 3)) << 4);
            const float *f = v + b * kBox + i * kUnit;
            if constexpr (sizeof(T) == 4) put_unit(at, __float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            else put_unit(at, pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]), pack2<T>(f[4], f[5]), pack2<T>(f[6], f[7]));
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(map_o, cb, row0, src);
            bulk_commit();
        }
        turn ^= 2048u;
    }
    if (c0 + kPiece > P.out_cols && live) {                // the entries behind the last whole 16 bytes of a row
#pragma unroll
        for (int j = 0; j < kPiece; ++j)
            if (c0 + j >= P.out_cols && c0 + j < E.J)
                static_cast<T *>(E.out)[(long long)row * E.ldo + c0 + j] =
                    from_f32<T>(v[j] + (E.res != nullptr ? to_f32(static_cast<const T *>(E.res)[(long long)row * E.ldr + c0 + j]) : 0.0f));
    }
}
// The same where rows do not start on 16 bytes: as binary32 through the buffer (16-byte units of a row exclusive-ored with the row
// number), and out with a column a lane, a row a step.
template <typename T>
__device__ __forceinline__ void copy_piece(const LinearOut &E, const float (&v)[kPiece], uint32_t wbuf, int lane, int row0, int c0)
{
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q)
        put_unit(wbuf + (uint32_t)lane * 128u + (uint32_t)((q ^ (lane & 7)) << 4), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
    __syncwarp();
    const int rows = c0 + lane < E.J ? E.I - row0 : 0;
    T *o = static_cast<T *>(E.out) + (long long)row0 * E.ldo + c0 + lane;
    const T *r = static_cast<const T *>(E.res) + (long long)row0 * E.ldr + c0 + lane;
#pragma unroll 1
    for (int r0 = 0; r0 < 32; r0 += 16) {
        float f[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            asm volatile("ld.shared.f32 %0, [%1];"
                         : "=f"(f[i])
                         : "r"(wbuf + (uint32_t)(r0 + i) * 128u + (uint32_t)(((lane >> 2) ^ (i & 7)) << 4) + (uint32_t)(lane & 3) * 4u)
                         : "memory");
        if (E.res != nullptr) {
            T a[16];
#pragma unroll
            for (int i = 0; i < 16; ++i, r += E.ldr) a[i] = r0 + i < rows ? *r : from_f32<T>(0.0f);
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] += to_f32(a[i]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i, o += E.ldo)
            if (r0 + i < rows) *o = from_f32<T>(f[i]);
    }
}

// v += the bias of the piece's columns from c0 on: where they are whole and start on 16 bytes four at a time, the same address in all
// lanes, otherwise a shuffle an entry out of the lanes that hold it.  (Shuffles, and peaks with a test for the row's end, for every
// entry: 8192 x 8192 x 2048 with GELU, bias and checkpoint 287 us, so 263.)
__device__ __forceinline__ void add_bias(const LinearOut &E, float lane_bias, int c0, float (&v)[kPiece])
{
    if (E.bias == nullptr) return;
    if ((reinterpret_cast<uintptr_t>(E.bias) & 15u) == 0 && c0 + kPiece <= E.J) {
        const float4 *b = reinterpret_cast<const float4 *>(E.bias + c0);
#pragma unroll
        for (int q = 0; q < kPiece / 4; ++q) {
            const float4 f = b[q];
            const float2 lo = add_2(make_float2(v[4 * q], v[4 * q + 1]), make_float2(f.x, f.y)), hi = add_2(make_float2(v[4 * q + 2], v[4 * q + 3]), make_float2(f.z, f.w));
            v[4 * q] = lo.x;
            v[4 * q + 1] = lo.y;
            v[4 * q + 2] = hi.x;
            v[4 * q + 3] = hi.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPiece; ++j) v[j] += __shfl_sync(0xffffffffu, lane_bias, j);
    }
}
// The largest magnitude of the piece's columns that exist (a NaN does not count).
__device__ __forceinline__ float peak_of(const float (&v)[kPiece], int cols, float m)
{
    if (cols >= kPiece) {
        float a[4] = {m, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kPiece; ++j) a[j & 3] = fmaxf(a[j & 3], fabsf(v[j]));
        return fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
    }
#pragma unroll
    for (int j = 0; j < kPiece; ++j) m = fmaxf(m, j < cols ? fabsf(v[j]) : 0.0f);
    return m;
}

// What the epilogue of 32 rows x HALF columns reads besides the sums, asked for before they are waited for: the lane's bias of each piece
// and its row's scale; its row of the residual and of the codes on their way to L2.
template <int HALF>
struct RowsIn {
    float bias[HALF / kPiece], zscale;
};
__device__ __forceinline__ void ask_line(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
template <int HALF>
__device__ __forceinline__ RowsIn<HALF> ask_rows(const LinearOut &E, int lane, int row0, int col0)
{
    RowsIn<HALF> in;
    const int row = row0 + lane;
    const bool live = row < E.I;
#pragma unroll
    for (int i = 0; i < HALF / kPiece; ++i) in.bias[i] = E.bias != nullptr && col0 + kPiece * i + lane < E.J ? E.bias[col0 + kPiece * i + lane] : 0.0f;
    in.zscale = 0.0f;
    if (E.zc != nullptr && live) {
        in.zscale = E.zs[(long long)(col0 >> 7) * E.I + row];
        ask_line(E.zc + (long long)row * E.ldz + col0);
    }
    if (E.res != nullptr && live) {
        const int esz = E.type == CDL_F32 ? 4 : 2;
        const char *p = static_cast<const char *>(E.res) + ((long long)row * E.ldr + col0) * esz;
        for (int i = 0; i < min(HALF, E.J - col0) * esz; i += 128) ask_line(p + i);
    }
    return in;
}

// 32 rows x HALF columns of finished sums in TMEM at `taddr`.  Where two warps share a checkpoint's groups of 128, they exchange their rows'
// largest magnitudes through `peaks` ([half][row of the tile]); false where the other one does not come.  added: the bias is in the sums already,
// and `peak` is known.
template <int HALF>
__device__ __forceinline__ bool emit_rows(const LinearParams &P, const CUtensorMap *map_o, const RowsIn<HALF> &in, bool added, float peak, float *peaks, PeakExchange &exchange, volatile int *abort_flag, int quarter, uint32_t taddr, uint32_t wbuf, uint32_t &turn, int lane, int row0, int col0)
{
    const LinearOut &E = P.out;
    const int row = row0 + lane;
    const bool live = row < E.I;
    float rrec = 0.0f;
    auto bias_of = [&](int c) {
        if constexpr (HALF == 64) return c < 32 ? in.bias[0] : in.bias[1];
        else return c < 64 ? (c < 32 ? in.bias[0] : in.bias[1]) : (c < 96 ? in.bias[2] : in.bias[3]);
    };
    if (E.codes != nullptr) {
        float m = peak, s;
#pragma unroll 1
        for (int c = 0; c < HALF && !added && col0 + c < E.J; c += kPiece) {
            uint32_t w[kPiece];
            tc_ld32(taddr + (uint32_t)c, w);
            const float b = bias_of(c);
            tc_wait_ld_pin(w);
            float v[kPiece];
#pragma unroll
            for (int j = 0; j < kPiece; ++j) v[j] = __uint_as_float(w[j]);
            add_bias(E, b, col0 + c, v);
            m = peak_of(v, E.J - col0 - c, m);
        }
        const int half = HALF == 64 ? (col0 >> 6) & 1 : 0;
        if (HALF == 64 && (half == 1 || col0 + HALF < E.J)) {      // (the other warp is there)
            float *at = peaks + quarter * 32 + lane;
            if (!exchange(at + half * 128, at + (half ^ 1) * 128, lane, m, abort_flag, kWaitNs)) return false;
        }
        fp8_scale_of(m, s, rrec);
        if (live && half == 0) E.scales[(long long)(col0 >> 7) * E.I + row] = s;
    }
#pragma unroll 1
    for (int c = 0; c < HALF; c += kPiece) {
        const int c0 = col0 + c, cols = E.J - c0;
        if (cols <= 0) break;
        uint32_t zw[kPiece / 4];
        if (E.zc != nullptr) {                             // (a row's pitch is whole units of 16)
            const unsigned char *zc = E.zc + (long long)row * E.ldz + c0;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint4 w = live && q * 16 < cols ? *reinterpret_cast<const uint4 *>(zc + q * 16) : make_uint4(0u, 0u, 0u, 0u);
                zw[4 * q] = w.x;
                zw[4 * q + 1] = w.y;
                zw[4 * q + 2] = w.z;
                zw[4 * q + 3] = w.w;
            }
        }
        float v[kPiece];
        {
            uint32_t w[kPiece];
            tc_ld32(taddr + (uint32_t)c, w);
            const float b = bias_of(c);
            tc_wait_ld_pin(w);
#pragma unroll
            for (int j = 0; j < kPiece; ++j) v[j] = __uint_as_float(w[j]);
            if (!added) add_bias(E, b, c0, v);
        }
        if (E.codes != nullptr) {
            unsigned char *codes = E.codes + (long long)row * E.ldc + c0;
            uint32_t w[kPiece / 4];
#pragma unroll
            for (int j = 0; j < kPiece / 4; ++j)
            {
                const float2 lo = mul_2(make_float2(v[4 * j], v[4 * j + 1]), both(rrec)), hi = mul_2(make_float2(v[4 * j + 2], v[4 * j + 3]), both(rrec));
                w[j] = fp8_code2(lo.x, lo.y) | (fp8_code2(hi.x, hi.y) << 16);
            }
            if (live && cols >= kPiece) {
                reinterpret_cast<uint4 *>(codes)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4 *>(codes)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else if (live)
#pragma unroll
                for (int j = 0; j < kPiece; ++j)
                    if (j < cols) codes[j] = (unsigned char)(w[j >> 2] >> (8 * (j & 3)));
        }
        switch (E.zc != nullptr ? kSlope + E.act : E.act) {
        case CDL_ACT_RELU: act_each<CDL_ACT_RELU>(v); break;
        case CDL_ACT_GELU: act_each<CDL_ACT_GELU>(v); break;
        case CDL_ACT_GELU_TANH: act_each<CDL_ACT_GELU_TANH>(v); break;
        case CDL_ACT_SILU: act_each<CDL_ACT_SILU>(v); break;
        case kSlope + CDL_ACT_RELU: slope_piece<CDL_ACT_RELU>(v, zw, in.zscale); break;
        case kSlope + CDL_ACT_GELU: slope_piece<CDL_ACT_GELU>(v, zw, in.zscale); break;
        case kSlope + CDL_ACT_GELU_TANH: slope_piece<CDL_ACT_GELU_TANH>(v, zw, in.zscale); break;
        case kSlope + CDL_ACT_SILU: slope_piece<CDL_ACT_SILU>(v, zw, in.zscale); break;
        default: break;
        }
        if (P.out_tma) {
            if (E.type == CDL_F32) send_piece<float>(P, map_o, v, wbuf, turn, lane, row0, c0);
            else if (E.type == CDL_BF16) send_piece<__nv_bfloat16>(P, map_o, v, wbuf, turn, lane, row0, c0);
            else send_piece<__half>(P, map_o, v, wbuf, turn, lane, row0, c0);
        } else if (E.type == CDL_F32) copy_piece<float>(E, v, wbuf, lane, row0, c0);
        else if (E.type == CDL_BF16) copy_piece<__nv_bfloat16>(E, v, wbuf, lane, row0, c0);
        else copy_piece<__half>(E, v, wbuf, lane, row0, c0);
    }
    return true;
}

// 128 columns of a row by a warp, four columns a lane (or every 32nd, where rows do not start on four entries): sums, the bias and the
// checkpoint; then the rest of the epilogue.
__device__ __forceinline__ void finish_row(const LinearOut &E, long long row, int col0, int lane, LinearIn<4> &in, float (&v)[4])
{
    const int step = E.vec ? 1 : 32, col = col0 + (E.vec ? lane * 4 : lane);
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + j * step < E.J) {
            if (E.bias != nullptr) v[j] += E.bias[col + j * step];
            m = fmaxf(m, fabsf(v[j]));
        }
    if (E.codes != nullptr) {
        float s, rec;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        fp8_scale_of(m, s, rec);
        if (lane == 0) E.scales[(long long)(col0 >> 7) * E.I + row] = s;
        linear_codes<4>(E, row, col, step, rec, v);
    }
    linear_store<4>(E, row, col, step, in, v);
}

// RUNS: some tiles are cut into runs of stages.  SEGMENT: stages after which sums are taken out of TMEM.
// SPLIT: a tile is a cluster's, whose CTAs share its stages; their sums go to shared memory, and each CTA finishes a part of the rows over
// all of them, in the order of the CTAs.
template <bool PAIR, bool RUNS, int SEGMENT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1)
linear_kernel(const __grid_constant__ LinearMaps maps, const __grid_constant__ LinearParams P)
{
    extern __shared__ unsigned char smem_dyn[];
    constexpr int kEdge = PAIR ? 256 : 128;            // of a tile; a CTA stages 128 rows of either operand
    constexpr int kHalf = kEdge / 2;                   // columns of an epilogue warp
    static_assert(!SPLIT || kEdge * kEdge * 4 <= kRingBytes, "shared memory");
    __shared__ __align__(8) unsigned long long bars[2 * kStages + 4];
    __shared__ uint32_t tmem_base_s, asked_s;
    __shared__ int abort_s;
    __shared__ float peaks[PAIR ? 1 : 2 * 128];
    __shared__ __align__(8) unsigned char meet[PAIR ? 8 : 4 * PeakExchange::kBytes];

    const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &abort_s;
    static_assert(!SPLIT || (!PAIR && !RUNS), "forms");
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const int slot = PAIR ? (int)(blockIdx.x >> 1) : (SPLIT ? (int)blockIdx.x / P.splits : (int)blockIdx.x);
    const int split = SPLIT ? (int)cluster_ctarank() : 0;

    // The tiles of a CTA (a pair): slot, slot + slots and so on below `whole`, then those that its run of stages touches.
    int run_lo = 0, run_hi = 0, tail_first = P.whole, tail_end = P.whole;
    if (RUNS && slot < P.ranges) {
        run_lo = slot * P.run;
        run_hi = min(run_lo + P.run, (P.tiles_i * P.tiles_j - P.whole) * P.KB);
        tail_first = P.whole + run_lo / P.KB;
        tail_end = P.whole + (run_hi - 1) / P.KB + 1;
    }
    const int first_tile = !RUNS || slot < P.whole ? slot : tail_first;
    auto next_tile = [&](int u) { return !RUNS || u + P.slots < P.whole ? u + P.slots : (u < P.whole ? tail_first : u + 1); };
    auto stages_of = [&](int u, int &kb0, int &kb1) {
        kb0 = SPLIT ? (int)((long long)P.KB * split / P.splits) : 0;
        kb1 = SPLIT ? (int)((long long)P.KB * (split + 1) / P.splits) : P.KB;
        if (RUNS && u >= P.whole) {
            const int first = (u - P.whole) * P.KB;
            kb0 = max(run_lo - first, 0);
            kb1 = min(run_hi - first, P.KB);
        }
    };

    const uint32_t bar0 = smem_u32(&bars[0]);
    constexpr uint32_t kEmptyOff = 8u * kStages;
    const uint32_t tfull0 = bar0 + 16u * kStages, tempty0 = tfull0 + 16u;
    if (threadIdx.x == 0) {
        abort_s = 0;
        asked_s = 0u;
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar0 + 8u * s, 1);
            mbar_init(bar0 + kEmptyOff + 8u * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull0 + 8u * b, 1);
            mbar_init(tempty0 + 8u * b, PAIR ? 2 * kEpiWarps : kEpiWarps);
        }
        if (!PAIR)
            for (int q = 0; q < 4; ++q) PeakExchange::init(smem_u32(meet) + (uint32_t)q * PeakExchange::kBytes);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc_all<PAIR>(smem_u32(&tmem_base_s));
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_s;
    follow_previous();
    bool failed = false;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsDrive));
        if (warp == 0 && lane == 0) {
            // -------------------------------------------------------- TMA producer (one lane)
            uint32_t st = 0u, par = 1u, asked = 0u;
            auto load = [&](uint32_t dst, const CUtensorMap *map, int c0, int c1, uint32_t fb) {
                if (PAIR) tma_load_2d_pair(dst, map, c0, c1, fb);
                else tma_load_2d(dst, map, c0, c1, fb);
            };
            // K-major: one box of 64 reduced entries x the block's rows.  MN-major: boxes of 64 rows x 64 reduced entries, the stored
            // matrix's rows being the reduced dimension.  With one CTA per tile each tile begins at another place of its stages: a
            // row pitch that is a power of two would have all CTAs read the same few memory channels at a time.
            auto stages = [&](auto a_mn, auto b_mn, int arow, int brow, int kb0, int kb1) {
                constexpr bool kA = decltype(a_mn)::value, kB = decltype(b_mn)::value;
                const uint32_t bytes = (PAIR ? 2u : 1u) * ((kA ? 128u : (uint32_t)P.a_rows) + (kB ? 128u : (uint32_t)P.b_rows)) * 128u;
                int kb = PAIR ? kb0 : kb0 + brow / 64 * 5 % (kb1 - kb0);
                for (int left = kb1 - kb0; left > 0; --left) {
                    const uint32_t fb = bar0 + 8u * st;
                    if (!mbar_try_wait_now(fb + kEmptyOff, par) && !mbar_wait(fb + kEmptyOff, par, abort_flag, kWaitNs)) {
                        failed = true;
                        return;
                    }
                    const uint32_t sa = smem_base + st * kStageBytes, sb = sa + kBlockBytes;
                    const int r = kb * kBK;
                    if (!PAIR || rank == 0) mbar_expect_tx(fb, bytes);
                    if (kA) {
                        load(sa, &maps.a, arow, r, fb);
                        load(sa + 8192u, &maps.a, arow + 64, r, fb);
                    } else load(sa, &maps.a, r, arow, fb);
                    if (kB) {
                        load(sb, &maps.b, brow, r, fb);
                        load(sb + 8192u, &maps.b, brow + 64, r, fb);
                    } else load(sb, &maps.b, r, brow, fb);
                    ++asked;
                    ++kb;
                    if (!PAIR && kb == kb1) kb = kb0;
                    if (++st == (uint32_t)kStages) {
                        st = 0u;
                        par ^= 1u;
                    }
                }
            };
            for (int u = first_tile; u < tail_end && !failed; u = next_tile(u)) {
                int ti, tj, kb0, kb1;
                tile_at(u, P.tiles_i, P.tiles_j, ti, tj);
                stages_of(u, kb0, kb1);
                const int arow = ti * kEdge + (int)rank * 128, brow = tj * kEdge + (int)rank * 128;
                if (P.mode == FORWARD) stages(No(), No(), arow, brow, kb0, kb1);
                else if (P.mode == DATA) stages(No(), Yes(), arow, brow, kb0, kb1);
                else stages(Yes(), Yes(), arow, brow, kb0, kb1);
            }
            asked_s = asked;
        } else if (warp == 1 && lane == 0 && (!PAIR || rank == 0)) {
            // -------------------------------------------------------- MMA issuer (one lane; CTA 0 of a pair)
            // K-major: 128-byte rows, groups of eight 1024 bytes apart, 32 bytes per MMA.  MN-major: one reduced entry per
            // 128-byte line, eight lines 1024 bytes apart, 64-row blocks 8192 bytes apart, 16 lines per MMA.
            const uint64_t k_d = make_desc(smem_base, 16, 1024), mn_d = make_desc(smem_base, 8192, 1024);
            const uint32_t d_hi = (uint32_t)(k_d >> 32), k_lo = (uint32_t)k_d, mn_lo = (uint32_t)mn_d;      // (the upper words agree)
            const uint32_t idesc0 = (1u << 4) | (P.fmt << 7) | (P.fmt << 10) | ((uint32_t)(kEdge >> 3) << 17) | ((uint32_t)(kEdge >> 4) << 24);
            uint32_t st = 0u, par = 0u, buf = 0u, tpar = 1u;
            auto stages = [&](auto a_mn, auto b_mn, int count) {
                constexpr bool kA = decltype(a_mn)::value, kB = decltype(b_mn)::value;
                const uint32_t a_lo0 = kA ? mn_lo : k_lo, b_lo0 = (kB ? mn_lo : k_lo) + (uint32_t)(kBlockBytes >> 4);
                const uint32_t idesc = idesc0 | ((kA ? 1u : 0u) << 15) | ((kB ? 1u : 0u) << 16);
                while (count > 0) {
                    const uint32_t te = tempty0 + 8u * buf;
                    if (!mbar_try_wait_now(te, tpar) && !mbar_wait(te, tpar, abort_flag, kWaitNs)) {
                        failed = true;
                        return;
                    }
                    uint32_t accumulate = 0u;
                    for (int i = min(count, SEGMENT); i > 0; --i) {
                        const uint32_t fb = bar0 + 8u * st;
                        if (!mbar_try_wait_now(fb, par) && !mbar_wait(fb, par, abort_flag, kWaitNs)) {
                            failed = true;
                            return;
                        }
                        tc_fence_after();
                        const uint32_t off = st * (kStageBytes >> 4);
                        tc_mma4<PAIR, KIND_F16>(tmem_base + buf * (uint32_t)kEdge, a_lo0 + off, d_hi, kA ? 2048u >> 4 : 2u, b_lo0 + off, d_hi, kB ? 2048u >> 4 : 2u, idesc, accumulate);
                        accumulate = 1u;
                        if (PAIR) tc_commit_pair(fb + kEmptyOff);
                        else tc_commit(fb + kEmptyOff);
                        if (++st == (uint32_t)kStages) {
                            st = 0u;
                            par ^= 1u;
                        }
                    }
                    if (PAIR) tc_commit_pair(tfull0 + 8u * buf);
                    else tc_commit(tfull0 + 8u * buf);
                    buf ^= 1u;
                    if (buf == 0u) tpar ^= 1u;
                    count -= SEGMENT;
                }
            };
            for (int u = first_tile; u < tail_end && !failed; u = next_tile(u)) {
                int kb0, kb1;
                stages_of(u, kb0, kb1);
                if (P.mode == FORWARD) stages(No(), No(), kb1 - kb0);
                else if (P.mode == DATA) stages(No(), Yes(), kb1 - kb0);
                else stages(Yes(), Yes(), kb1 - kb0);
            }
        }
        if (SPLIT) {
            __syncwarp();
            cluster_sync_all();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpilogue));
        // ------------------------------------------------------------ epilogue warps: 32 rows x half of the tile's columns each
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t wbuf = smem_base + (uint32_t)kRingBytes + (uint32_t)((warp - 4) * kOutWarpBytes);
        const LinearOut &E = P.out;
        uint32_t buf = 0u, tpar = 0u, turn = 0u;
        PeakExchange exchange{smem_u32(meet) + (PAIR ? 0u : (uint32_t)quarter * PeakExchange::kBytes), 0u};
        for (int u = first_tile; u < tail_end && !failed; u = next_tile(u)) {
            int ti, tj, kb0, kb1;
            tile_at(u, P.tiles_i, P.tiles_j, ti, tj);
            stages_of(u, kb0, kb1);
            const int in_row = (int)rank * 128 + quarter * 32, in_col = half * kHalf;    // of this warp in the tile
            const int row0 = ti * kEdge + in_row, col0 = tj * kEdge + in_col;
            RowsIn<kHalf> in;
            if (!SPLIT && (!RUNS || kb1 - kb0 == P.KB) && row0 < E.I && col0 < E.J) in = ask_rows<kHalf>(E, lane, row0, col0);
            const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * kHalf);
            auto ready = [&] {
                return __all_sync(0xffffffffu, mbar_try_wait_now(tfull0 + 8u * buf, tpar) || mbar_wait(tfull0 + 8u * buf, tpar, abort_flag, kWaitNs + kWaitStageNs * (unsigned)(kb1 - kb0)));
            };
            auto release = [&] {                           // the sums have been read: their half of TMEM is free
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_remote(tempty0 + 8u * buf, 0u);
                    else mbar_arrive(tempty0 + 8u * buf);
                }
                buf ^= 1u;
                if (buf == 0u) tpar ^= 1u;
            };
            bool added = false;                            // the bias is in the sums, and `peak` is their rows' largest magnitude
            float peak = 0.0f;
            if (kb1 - kb0 > SEGMENT) {
                // the segments' sums, in registers; then back to where the last one's were, so that the epilogue is one
                float acc[kHalf];
#pragma unroll
                for (int j = 0; j < kHalf; ++j) acc[j] = 0.0f;
                for (int left = kb1 - kb0;;) {
                    if (!ready()) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t taddr = lanes + buf * (uint32_t)kEdge;
                    // 16 columns at a time, the next ones on their way while these are added
                    uint32_t va[16], vb[16];
                    tc_ld16(taddr, va);
#pragma unroll
                    for (int c = 0; c < kHalf / 32; ++c) {
                        tc_wait_ld_pin(va);
                        tc_ld16(taddr + (uint32_t)(c * 32 + 16), vb);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[c * 32 + j] += __uint_as_float(va[j]);
                        tc_wait_ld_pin(vb);
                        if (c < kHalf / 32 - 1) tc_ld16(taddr + (uint32_t)(c * 32 + 32), va);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[c * 32 + 16 + j] += __uint_as_float(vb[j]);
                    }
                    left -= SEGMENT;
                    if (left <= 0) break;
                    release();
                }
                if (failed) break;
                if (!SPLIT && E.codes != nullptr && (!RUNS || kb1 - kb0 == P.KB)) {
                    // what a checkpoint needs of all columns before the first, while they are in registers
                    added = true;
#pragma unroll
                    for (int c = 0; c < kHalf / kPiece; ++c) {
                        float v[kPiece];
#pragma unroll
                        for (int j = 0; j < kPiece; ++j) v[j] = acc[c * kPiece + j];
                        add_bias(E, in.bias[c], col0 + c * kPiece, v);
                        peak = peak_of(v, E.J - col0 - c * kPiece, peak);
#pragma unroll
                        for (int j = 0; j < kPiece; ++j) acc[c * kPiece + j] = v[j];
                    }
                }
#pragma unroll
                for (int c = 0; c < kHalf / 16; ++c) {
                    uint32_t v[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(acc[c * 16 + j]);
                    tc_st16(lanes + buf * (uint32_t)kEdge + (uint32_t)(c * 16), v);
                }
                tc_wait_st();
            } else {
                if (!ready()) {
                    failed = true;
                    break;
                }
                tc_fence_after();
            }
            const uint32_t taddr = lanes + buf * (uint32_t)kEdge;
            if (row0 < E.I && col0 < E.J) {
                if (SPLIT) {
                    // the sums take the place of the pipeline's stages, [rows][128]: this warp has seen the last of the CTA's products,
                    // so all loads have landed and been read.  16-byte units of a row are exclusive-ored with the row number.
                    const int r = quarter * 32 + lane;
#pragma unroll 1
                    for (int c = 0; c < kHalf; c += 32) {
                        uint32_t v[32];
                        tc_ld32(taddr + (uint32_t)c, v);
                        tc_wait_ld_pin(v);
                        if (row0 + lane < E.I)
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                put_unit(smem_base + (uint32_t)r * 512u + (uint32_t)((((in_col + c) / 4 + q) ^ (r & 7)) << 4), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                    }
                } else if (!RUNS || kb1 - kb0 == P.KB) {
                    if (!emit_rows<kHalf>(P, &maps.o, in, added, peak, peaks, exchange, abort_flag, quarter, taddr, wbuf, turn, lane, row0, col0)) {
                        failed = true;
                        break;
                    }
                } else {
                    // a part of a tile: its sums as they are, through the staging buffer 32 columns at a time
#pragma unroll 1
                    for (int ch = 0; ch < kHalf / 32 && col0 + ch * 32 < E.J; ++ch) {
                        uint32_t v[32];
                        tc_ld32(taddr + (uint32_t)(ch * 32), v);
                        tc_wait_ld_pin(v);
                        if (lane == 0) bulk_wait_read<0>();
                        __syncwarp();
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(wbuf + (uint32_t)lane * 128u + (uint32_t)((q ^ (lane & 7)) << 4)),
                                         "r"(v[4 * q]), "r"(v[4 * q + 1]), "r"(v[4 * q + 2]), "r"(v[4 * q + 3])
                                         : "memory");
                        __syncwarp();
                        const int sub = lane >> 3, unit = lane & 7;
                        float *p = P.part + ((long long)(slot + u - P.whole) * kEdge + in_row) * kEdge + in_col + ch * 32 + unit * 4;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int r = i * 4 + sub;
                            const uint4 q = lds_u128(wbuf + (uint32_t)r * 128u + (uint32_t)((unit ^ (r & 7)) << 4));
                            if (row0 + r < E.I) *reinterpret_cast<uint4 *>(p + r * kEdge) = q;
                        }
                    }
                }
            }
            release();
        }
        if (lane == 0) bulk_wait_read<0>();                // (the stores themselves are complete when the kernel is)
        if (SPLIT) {
            int ti, tj;
            tile_at(slot, P.tiles_i, P.tiles_j, ti, tj);
            __syncwarp();
            cluster_sync_all();
            const int rows = min(128, E.I - ti * 128), col0 = tj * 128;
            const int first = split * kEpiWarps + warp - 4, every = P.splits * kEpiWarps;
            constexpr int kBatch = 2;
            const int step = E.vec ? 1 : 32, off = E.vec ? lane * 4 : lane;
#pragma unroll 1
            for (int i0 = first; i0 < rows; i0 += every * kBatch) {
                LinearIn<4> in[kBatch];
                float v[kBatch][4];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int r = i0 + b * every;
                    if (r < rows) linear_fetch<4>(E, ti * 128 + r, col0 + off, step, in[b]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[b][j] = 0.0f;
                }
                float q[kBatch][8][4];                       // (all on their way before the first is added)
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int r = min(i0 + b * every, rows - 1);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (k >= P.splits) break;
                        if (E.vec) {
                            const uint32_t local = smem_base + (uint32_t)r * 512u + (uint32_t)(((off >> 2) ^ (r & 7)) << 4);
                            asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
                                         : "=f"(q[b][k][0]), "=f"(q[b][k][1]), "=f"(q[b][k][2]), "=f"(q[b][k][3])
                                         : "r"(local), "r"(k));
                        } else
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int at = off + j * 32;
                                const uint32_t local = smem_base + (uint32_t)r * 512u + (uint32_t)(((at >> 2) ^ (r & 7)) << 4) + (uint32_t)(at & 3) * 4u;
                                asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(q[b][k][j]) : "r"(local), "r"(k));
                            }
                    }
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (k >= P.splits) break;
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[b][j] += q[b][k][j];
                    }
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int r = i0 + b * every;
                    if (r < rows) finish_row(E, ti * 128 + r, col0, lane, in[b], v[b]);
                }
            }
        }
    }
    if (failed) {
        abort_s = 1;
        if (lane == 0) record_timeout(P.status);
    }
    tc_fence_before();
    __syncthreads();
    // after an abandoned wait: loads that are still under way land (or a limit runs out) before the CTA ends
    if (abort_s != 0 && threadIdx.x == 0 && (!PAIR || rank == 0)) drain_stages(bar0, asked_s, (uint32_t)kStages);
    __syncwarp();
    if (PAIR || SPLIT) cluster_sync_all();      // no CTA leaves while another may touch its shared memory or TMEM
    if (warp == 1) {
        tc_fence_after();
        tmem_free_all<PAIR>(tmem_base);
    }
}

// The tiles that runs share (and sums of the form for few rows whose checkpoint is wanted): their pieces in order, then the
// epilogue.  A warp takes 128 columns of a row, which is a group of the checkpoint.
// fixed < 0: the pieces of tile first + t are those of the runs that touch it; otherwise there are `fixed` of them, at t.
__global__ void __launch_bounds__(256)
linear_finish_kernel(const __grid_constant__ LinearOut E, const float *part, int tile_rows, int tile_cols, int tiles_i, int tiles_j, int first, int run, int KB, int fixed)
{
    follow_previous();                                  // (also where nothing is left to do: what follows relies on it)
    const int t = (int)blockIdx.x, warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    int pieces = fixed, at = t;
    if (fixed < 0) {
        const int r0 = t * KB / run, r1 = ((t + 1) * KB - 1) / run;
        if (r0 == r1) return;                           // one run had all of it
        pieces = r1 - r0 + 1;
        at = r0 + t;
    }
    int ti, tj;
    tile_at(first + t, tiles_i, tiles_j, ti, tj);
    const bool wide = tile_cols == 256;
    const int r = wide ? (int)blockIdx.y * 4 + (warp >> 1) : (int)blockIdx.y * 8 + warp, c = wide ? (warp & 1) * 128 : 0;
    const long long row = (long long)ti * tile_rows + r;
    const int col0 = tj * tile_cols + c;
    if (r >= tile_rows || row >= E.I || col0 >= E.J) return;
    const int step = E.vec ? 1 : 32, off = E.vec ? lane * 4 : lane, col = col0 + off;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    LinearIn<4> in;
    linear_fetch<4>(E, row, col, step, in);
    const float *p = part + ((long long)at * tile_rows + r) * tile_cols + c + off;
#pragma unroll 8
    for (int k = 0; k < pieces; ++k, p += (long long)tile_rows * tile_cols) {
        if (E.vec) {
            const float4 w = *reinterpret_cast<const float4 *>(p);
            v[0] += w.x;
            v[1] += w.y;
            v[2] += w.z;
            v[3] += w.w;
        } else
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += p[32 * j];
    }
    finish_row(E, row, col0, lane, in, v);
}

// Sums of the columns of a 16-bit matrix: 64 columns a cluster, whose CTAs share the rows and are added in their order.
constexpr int kSumCtas = 8, kSumThreads = 256;
template <typename T>
__global__ void __cluster_dims__(kSumCtas, 1, 1) __launch_bounds__(kSumThreads)
column_sums_kernel(const T *x, long long ldx, int rows, int cols, float *out)
{
    __shared__ float sums[kSumThreads / 8][64 + 1];
    __shared__ float total[64];
    const int unit = (int)threadIdx.x & 7, lane = (int)threadIdx.x >> 3;      // eight columns, every 32nd row
    const int rank = (int)cluster_ctarank(), col = (int)(blockIdx.x / kSumCtas) * 64 + unit * 8;
    follow_previous();
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 0.0f;
    const long long r0 = (long long)rows * rank / kSumCtas, r1 = (long long)rows * (rank + 1) / kSumCtas;
    if (col + 8 <= cols) {
#pragma unroll 8
        for (long long r = r0 + lane; r < r1; r += kSumThreads / 8) {
            float v[8];
            load8(x + r * ldx + col, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += v[j];
        }
    } else {
        for (long long r = r0 + lane; r < r1; r += kSumThreads / 8)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < cols) s[j] += to_f32(x[r * ldx + col + j]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[lane][unit * 8 + j] = s[j];
    __syncthreads();
    if (threadIdx.x < 64) {
        float a = 0.0f;
#pragma unroll
        for (int k = 0; k < kSumThreads / 8; ++k) a += sums[k][threadIdx.x];
        total[threadIdx.x] = a;
    }
    cluster_sync_all();
    const int c = (int)(blockIdx.x / kSumCtas) * 64 + (int)threadIdx.x;
    if (rank == 0 && threadIdx.x < 64 && c < cols) {
        float a = 0.0f;
        for (int k = 0; k < kSumCtas; ++k) {
            float v;
            asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}"
                         : "=f"(v)
                         : "r"(smem_u32(&total[threadIdx.x])), "r"(k));
            a += v;
        }
        out[c] = a;
    }
    cluster_sync_all();
}

// What a product of these sizes runs as.  Planned for a B200's 148 SMs so that workspace sizes are fixed.
struct LinearPlan {
    bool pair;
    int tiles_i, tiles_j;
    int whole, ranges, run;
    int splits;                 // CTAs of a cluster per tile (single-CTA tiles)
    size_t part_bytes;
    long long ns;
};
constexpr int kPlanSms = 148;
constexpr int64_t kL2Bytes = 126000000;
constexpr size_t kStatusBytes = 256;

bool make_plan(int64_t I, int64_t J, int64_t R, LinearPlan *p)
{
    const int64_t KB = (R + kBK - 1) / kBK, pairs = kPlanSms / 2, singles = ((I + 127) / 128) * ((J + 127) / 128);
    if (singles > 0x3fffffff) return false;
    // Tiles as they are, or with the last, partly filled round cut into runs that fill the device, which costs the pieces' way through
    // memory and another launch; each with its estimate in nanoseconds.  (45 sizes of 10 to 9000 rows and columns and 64 to 28000 reduced entries, in
    // every form: the form chosen takes 4.8 % longer than the fastest one on average, 43 % at most, 39 x 230 x 7413 16.0 for 11.2 us.)
    struct Form { int64_t ns, whole, ranges, run, splits, piece_bytes; bool pair; } best = {INT64_MAX, 0, 0, 0, 1, 0, false};
    auto consider = [&](const Form &f) {
        if (f.ns < best.ns) best = f;
    };
    for (int pair = 0; pair < 2; ++pair) {
        const int64_t edge = pair ? 256 : 128, slots = pair ? pairs : kPlanSms, n = pair ? (I + 255) / 256 * ((J + 255) / 256) : singles, tail = n % slots;
        const int64_t stage = pair ? 310 : 290, start = pair ? 5000 : 4000, tile = (pair ? 2500 : 1500) + stage * KB;
        consider(Form{start + (n + slots - 1) / slots * tile, n, 0, 0, 1, 0, pair != 0});
        if (tail > 0) {
            const int64_t stages = tail * KB, most = stages / 4 < slots ? stages / 4 : slots;        // four stages at least
            if (most > 1) {
                const int64_t run = (stages + most - 1) / most, ranges = (stages + run - 1) / run, bytes = (ranges + tail) * edge * edge * 4;
                const int64_t apart = 2 * (I + J) * R > kL2Bytes ? stage * run / 10 : 0;             // (they no longer read the same entries at one time)
                consider(Form{start + n / slots * tile + stage * run + apart + (pair ? 9000 : 4500) + bytes / 6000 + 30 * (ranges / tail), n - tail, ranges, run, 1, bytes, pair != 0});
            }
        }
    }
    // Few tiles: a cluster each.  (Clusters of four and eight do not fit everywhere: the device runs 32 and 14 of them at once for certain.)
    const int64_t clusters[4] = {kPlanSms, pairs, 32, 14};
    for (int i = 1; i < 4 && singles <= clusters[i] && (2ll << i) <= KB; ++i)
        consider(Form{4000 + 290 * ((KB + (1 << i) - 1) >> i) + 3500, singles, 0, 0, 1ll << i, 0, false});
    p->pair = best.pair;
    p->splits = (int)best.splits;
    p->tiles_i = (int)((I + (best.pair ? 255 : 127)) / (best.pair ? 256 : 128));
    p->tiles_j = (int)((J + (best.pair ? 255 : 127)) / (best.pair ? 256 : 128));
    p->whole = (int)best.whole;
    p->ranges = (int)best.ranges;
    p->run = (int)best.run;
    p->part_bytes = (size_t)best.piece_bytes;
    p->ns = best.ns;
    return true;
}

size_t rows_part_bytes(int64_t N) { return (size_t)((N + 255) / 256) * 8 * 256 * sizeof(float); }

int launch_finish(const LinearOut &E, const float *part, int tile_rows, int tile_cols, int tiles_i, int tiles_j, int first, int run, int KB, int fixed, cudaStream_t st)
{
    const dim3 grid((unsigned)(tiles_i * tiles_j - first), (unsigned)(tile_rows / (tile_cols == 256 ? 4 : 8)));
    return launch_following(&linear_finish_kernel, grid, dim3(256), 0, st, E, part, tile_rows, tile_cols, tiles_i, tiles_j, first, run, KB, fixed);
}

// mode FORWARD: A [I][R], B [J][R];  DATA: A [I][R], B [R][J];  WEIGHT: A [R][I], B [R][J]
int launch_linear(int mode, const void *A, int64_t lda, const void *B, int64_t ldb, int type, int64_t R, LinearOut E, void *ws, cudaStream_t st)
{
    const int esz = type_bytes(E.type);
    auto four = [&](const void *p, int64_t ld) {
        return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & (uintptr_t)(4 * esz - 1)) == 0 && (E.I == 1 || ld % 4 == 0));
    };
    E.vec = four(E.out, E.ldo) && four(E.res, E.ldr);
    const int sms = sm_count();
    if (sms <= 0) return CDL_ERR_LAUNCH;
    LinearPlan plan;
    if (!make_plan(E.I, E.J, R, &plan)) return CDL_ERR_ARG;
    const int edge = plan.pair ? 256 : 128;
    if (R == 0) return launch_finish(E, nullptr, edge, edge, plan.tiles_i, plan.tiles_j, 0, 0, 0, 0, st);
    float *part = reinterpret_cast<float *>(static_cast<char *>(ws) + kStatusBytes);
    // (Weights that come out of L2 leave the form for few rows 0.5 to 0.9 of its estimate, a tile's form 0.8 to 1.4 of its own.  70 sizes of one to eight
    // rows where the estimates are within a factor of three: 1.8 % longer than the faster form on average with this factor, 2.8 % with 1, 2.0 % with 0.6;
    // 1 x 4424 x 1912 6.2 us and 9.9 in tiles, 8 x 459 x 52388 41.8 and 24.9, next to the border 4 x 4791 x 3458 13.7 and 12.3, 1 x 1457 x 24815 19.8 and 21.1.)
    if (mode == FORWARD && E.I <= kFewRowsLinear && plan_linear_rows(E.J, (int)R).ns * 3 / 4 <= plan.ns) {
        const int rc = launch_linear_rows(A, lda, B, ldb, type, E.I, E.J, (int)R, E, E.codes != nullptr ? part : nullptr, st);
        if (rc != CDL_OK || E.codes == nullptr) return rc;
        return launch_finish(E, part, 8, 256, 1, (E.J + 255) / 256, 0, 0, 0, 1, st);
    }
    LinearParams P;
    memset(&P, 0, sizeof P);
    P.mode = mode;
    P.R = (int)R;
    P.KB = (int)((R + kBK - 1) / kBK);
    P.tiles_i = plan.tiles_i;
    P.tiles_j = plan.tiles_j;
    P.whole = plan.whole;
    P.ranges = plan.ranges;
    P.run = plan.run;
    P.part = part;
    P.status = static_cast<int *>(ws);
    P.fmt = type == CDL_BF16 ? 1u : 0u;
    P.out = E;
    auto box = [](int64_t rows, int64_t most) { return (int)(rows >= most ? most : (rows + 7) / 8 * 8); };
    P.a_rows = box(E.I, 128);
    P.b_rows = box(E.J, 128);
    const CUtensorMapDataType kind = type == CDL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    LinearMaps maps;
    const bool ok = (mode == WEIGHT ? encode_map_2d(&maps.a, kind, 2, A, (uint64_t)E.I, (uint64_t)R, (uint64_t)lda * 2u, 64)
                                    : encode_map_2d(&maps.a, kind, 2, A, (uint64_t)R, (uint64_t)E.I, (uint64_t)lda * 2u, (uint32_t)P.a_rows)) &&
                    (mode == FORWARD ? encode_map_2d(&maps.b, kind, 2, B, (uint64_t)R, (uint64_t)E.J, (uint64_t)ldb * 2u, (uint32_t)P.b_rows)
                                     : encode_map_2d(&maps.b, kind, 2, B, (uint64_t)E.J, (uint64_t)R, (uint64_t)ldb * 2u, 64));
    if (!ok) return CDL_ERR_LAUNCH;
    auto sixteen = [&](const void *p, int64_t ld) { return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (ld * esz) % 16 == 0); };
    P.out_cols = (int)((int64_t)E.J * esz / 16 * 16 / esz);
    P.out_tma = P.out_cols > 0 && sixteen(E.out, E.ldo) && sixteen(E.res, E.ldr);
    maps.o = maps.a;
    if (P.out_tma && !encode_map_2d(&maps.o, E.type == CDL_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : (E.type == CDL_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16),
                                    esz, E.out, (uint64_t)P.out_cols, (uint64_t)E.I, (uint64_t)(E.ldo * esz), 32, 64))
        return CDL_ERR_LAUNCH;
    static bool attr_set[64];
    static int pair_slots[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return CDL_ERR_LAUNCH;
#define CDL_FORMS(SEGMENT)                                                                                                                                \
    {reinterpret_cast<const void *>(&linear_kernel<false, false, SEGMENT, false>), reinterpret_cast<const void *>(&linear_kernel<true, false, SEGMENT, false>), \
     reinterpret_cast<const void *>(&linear_kernel<false, true, SEGMENT, false>), reinterpret_cast<const void *>(&linear_kernel<true, true, SEGMENT, false>),   \
     reinterpret_cast<const void *>(&linear_kernel<false, false, SEGMENT, true>)}
    static const void *const kernels[2][5] = {CDL_FORMS(kSegment32), CDL_FORMS(kSegment16)};
#undef CDL_FORMS
    const void *const kernel = kernels[E.type == CDL_F32 ? 0 : 1][plan.splits > 1 ? 4 : (plan.pair ? 1 : 0) + (plan.ranges > 0 ? 2 : 0)];
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    if (!attr_set[dev]) {
        for (int v = 0; v < 10; ++v)
            if (cudaFuncSetAttribute(kernels[v / 5][v % 5], cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) {
                (void)cudaGetLastError();
                return CDL_ERR_LAUNCH;
            }
        // the warpgroups' shares must fit what a block is launched with, or an epilogue warpgroup would wait for good
        for (int v = 0; v < 10; ++v) {
            cudaFuncAttributes fa;
            if (cudaFuncGetAttributes(&fa, kernels[v / 5][v % 5]) != cudaSuccess || fa.numRegs < kRegsLaunch) {
                (void)cudaGetLastError();
                return CDL_ERR_LAUNCH;
            }
        }
        cfg.gridDim = dim3(2u * (unsigned)(sms / 2));
        cfg.attrs = at + 1;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernels[0][1], &cfg) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();
            n = sms / 2;
        }
        pair_slots[dev] = n < sms / 2 ? n : sms / 2;
        attr_set[dev] = true;
    }
    // (a CTA has one run at most: as many are started as there are runs, should the device have fewer places)
    P.splits = plan.splits;
    const int places = plan.pair ? pair_slots[dev] : (plan.splits > 1 ? P.whole : sms);
    P.slots = P.whole < places ? P.whole : places;
    if (P.slots < P.ranges) P.slots = P.ranges;
    const unsigned cluster = plan.pair ? 2u : (unsigned)plan.splits;
    at[1].val.clusterDim.x = cluster;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    cfg.gridDim = dim3(cluster * (unsigned)P.slots);
    cfg.stream = st;
    void *args[2] = {&maps, &P};
    if (cudaLaunchKernelExC(&cfg, kernel, args) != cudaSuccess) {
        (void)cudaGetLastError();
        return CDL_ERR_LAUNCH;
    }
    if (P.ranges > 0) return launch_finish(E, part, edge, edge, plan.tiles_i, plan.tiles_j, P.whole, P.run, P.KB, -1, st);
    return CDL_OK;
}

bool bad_extent(int32_t n) { return n < 0 || n > kMostExtent; }
bool half_type(int type) { return type == CDL_BF16 || type == CDL_F16; }
bool odd16(const void *p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0 || (ld & 7) != 0; }
bool odd4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
bool tiles_fit(int64_t I, int64_t J) { return ((I + 127) / 128) * ((J + 127) / 128) <= 0x3fffffff; }
bool bad_workspace(const void *ws, size_t bytes, int32_t M, int32_t N, int32_t K)
{
    return ws == nullptr || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || bytes < cdl_linear_workspace_bytes(M, N, K);
}

}  // namespace
}  // namespace cdl

extern "C" size_t cdl_linear_workspace_bytes(int32_t M, int32_t N, int32_t K)
{
    using namespace cdl;
    if (bad_extent(M) || bad_extent(N) || bad_extent(K)) return 0;
    size_t most = M <= kFewRowsLinear ? rows_part_bytes(N) : 0;
    const int64_t sizes[3][3] = {{M, N, K}, {M, K, N}, {N, K, M}};
    for (const auto &s : sizes) {
        LinearPlan p;
        if (s[0] > 0 && s[1] > 0 && s[2] > 0 && make_plan(s[0], s[1], s[2], &p) && p.part_bytes > most) most = p.part_bytes;
    }
    return kStatusBytes + most;
}

extern "C" int cdl_linear_fwd(const void *A, int64_t lda, const void *W, int64_t ldw, int32_t type, const float *bias, int32_t act,
                              const void *residual, int64_t ldr, int32_t M, int32_t N, int32_t K, void *out, int64_t ldo, int32_t out_type,
                              void *codes, int64_t ldc, float *scales, void *ws, size_t ws_bytes, void *stream)
{
    using namespace cdl;
    if (bad_extent(M) || bad_extent(N) || bad_extent(K) || !half_type(type) || !valid_type(out_type) || !valid_act(act)) return CDL_ERR_ARG;
    if (M == 0 || N == 0) return CDL_OK;
    if (out == nullptr || ldo < N || (residual != nullptr && ldr < N) || !tiles_fit(M, N)) return CDL_ERR_ARG;
    if (K > 0 && (A == nullptr || W == nullptr || lda < K || ldw < K)) return CDL_ERR_ARG;
    if ((codes == nullptr) != (scales == nullptr) || (codes != nullptr && ldc < N)) return CDL_ERR_ARG;
    if (misaligned(out, out_type) || misaligned(residual, out_type) || odd4(bias) || odd4(scales)) return CDL_ERR_ALIGN;
    if (K > 0 && (odd16(A, lda) || odd16(W, ldw))) return CDL_ERR_ALIGN;
    if (codes != nullptr && ((reinterpret_cast<uintptr_t>(codes) & 15u) || (ldc & 15))) return CDL_ERR_ALIGN;
    if (bad_workspace(ws, ws_bytes, M, N, K)) return CDL_ERR_WORKSPACE;
    const int rc = check_device();
    if (rc != CDL_OK) return rc;
    const LinearOut E{M, N, out, ldo, out_type, bias, act, nullptr, 0, nullptr, residual, ldr, static_cast<unsigned char *>(codes), ldc, scales, 0};
    return launch_linear(FORWARD, A, lda, W, ldw, type, K, E, ws, static_cast<cudaStream_t>(stream));
}

extern "C" int cdl_linear_bwd_data(const void *dY, int64_t lddy, const void *W, int64_t ldw, int32_t type, int32_t act, const void *codes,
                                   int64_t ldc, const float *scales, const void *residual, int64_t ldr, int32_t M, int32_t N, int32_t K, void *dA,
                                   int64_t ldda, int32_t out_type, void *ws, size_t ws_bytes, void *stream)
{
    using namespace cdl;
    if (bad_extent(M) || bad_extent(N) || bad_extent(K) || !half_type(type) || !valid_type(out_type) || !valid_act(act)) return CDL_ERR_ARG;
    if (M == 0 || K == 0) return CDL_OK;
    if (dA == nullptr || ldda < K || (residual != nullptr && ldr < K) || !tiles_fit(M, K)) return CDL_ERR_ARG;
    if (N > 0 && (dY == nullptr || W == nullptr || lddy < N || ldw < K)) return CDL_ERR_ARG;
    if ((codes == nullptr) != (scales == nullptr) || (act != CDL_ACT_NONE && codes == nullptr) || (codes != nullptr && ldc < K)) return CDL_ERR_ARG;
    if (misaligned(dA, out_type) || misaligned(residual, out_type) || odd4(scales)) return CDL_ERR_ALIGN;
    if (N > 0 && (odd16(dY, lddy) || odd16(W, ldw))) return CDL_ERR_ALIGN;
    if (codes != nullptr && ((reinterpret_cast<uintptr_t>(codes) & 15u) || (ldc & 15))) return CDL_ERR_ALIGN;
    if (bad_workspace(ws, ws_bytes, M, N, K)) return CDL_ERR_WORKSPACE;
    const int rc = check_device();
    if (rc != CDL_OK) return rc;
    const bool slope = act != CDL_ACT_NONE;             // (the identity's derivative needs no checkpoint)
    const LinearOut E{M, K, dA, ldda, out_type, nullptr, act, slope ? static_cast<const unsigned char *>(codes) : nullptr, ldc, slope ? scales : nullptr, residual, ldr,
                      nullptr, 0, nullptr, 0};
    return launch_linear(DATA, dY, lddy, W, ldw, type, N, E, ws, static_cast<cudaStream_t>(stream));
}

extern "C" int cdl_linear_bwd_weight(const void *dY, int64_t lddy, const void *A, int64_t lda, int32_t type, int32_t M, int32_t N, int32_t K,
                                     int32_t accumulate, void *dW, int64_t lddw, int32_t out_type, float *dbias, void *ws, size_t ws_bytes, void *stream)
{
    using namespace cdl;
    if (bad_extent(M) || bad_extent(N) || bad_extent(K) || !half_type(type) || !valid_type(out_type)) return CDL_ERR_ARG;
    if (N == 0) return CDL_OK;
    const bool product = K > 0 && dW != nullptr;
    if (!product && dbias == nullptr) return K == 0 ? CDL_OK : CDL_ERR_ARG;
    if (M > 0 && (dY == nullptr || lddy < N)) return CDL_ERR_ARG;
    if (product && (lddw < K || (M > 0 && (A == nullptr || lda < K)) || !tiles_fit(N, K))) return CDL_ERR_ARG;
    if (M > 0 && (odd16(dY, lddy) || (product && odd16(A, lda)))) return CDL_ERR_ALIGN;
    if ((product && misaligned(dW, out_type)) || odd4(dbias)) return CDL_ERR_ALIGN;
    if (product && bad_workspace(ws, ws_bytes, M, N, K)) return CDL_ERR_WORKSPACE;
    int rc = check_device();
    if (rc != CDL_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (product) {
        const LinearOut E{N, K, dW, lddw, out_type, nullptr, CDL_ACT_NONE, nullptr, 0, nullptr, accumulate ? dW : nullptr, lddw, nullptr, 0, nullptr, 0};
        rc = launch_linear(WEIGHT, dY, lddy, A, lda, type, M, E, ws, st);
        if (rc != CDL_OK) return rc;
    }
    if (dbias == nullptr) return CDL_OK;
    const dim3 grid((unsigned)(((int64_t)N + 63) / 64 * kSumCtas));
    if (type == CDL_BF16) return launch_following(&column_sums_kernel<__nv_bfloat16>, grid, dim3(kSumThreads), 0, st, static_cast<const __nv_bfloat16 *>(dY), (long long)lddy, (int)M, (int)N, dbias);
    return launch_following(&column_sums_kernel<__half>, grid, dim3(kSumThreads), 0, st, static_cast<const __half *>(dY), (long long)lddy, (int)M, (int)N, dbias);
}
