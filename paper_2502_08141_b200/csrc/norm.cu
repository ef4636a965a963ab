// lowra_norm_forward / lowra_norm_backward: the norm before a layer's projections, with the residual stream's addition on the way,
//     h = bf16(X + residual);   Y = (h - mu) rstd weight + bias,   rstd = 1 / sqrt(mean (h - mu)^2 + eps)          (root mean square: mu = 0, no bias)
// and its gradient, with g = dY weight and xh = (h - mu) rstd,
//     dX = rstd (g - mean g - xh mean(g xh)) + dsum;    dweight = sum over the rows of dY xh;    dbias = sum over the rows of dY
// Bound by memory.  A row is taken by one group of threads, eight neighbouring channels (16 bytes) to a thread or two or four times as many, and stays in their
// registers, or in shared memory, between its statistics and its output: every array is read or written once.  The statistics are sums in fp32 over the registers; the variance is that of the
// differences from the mean, a second sum, so that a mean far from zero costs no digits.
// Measured, us, in brackets at the copy rate: kernels one behind the other on inputs from memory: forward with a residual, layer norm 333 x 5120 5.5 (2.1), 4096 x 4096 25.3 (20.8; root mean square 24.6), one token of 4096 2.0;
// without one, layer norm 3039 x 3968 15.1 (7.5), 1673 x 10024 25.5 (10.4: one row at work on an SM, two barriers to it); backward with the weight's gradient, root mean square 4096 x 4096, residual, 31.5 to 32.6
// (20.8: the rows 26, their CTAs' sums 5), layer norm 1001 x 1024 5.4 (1.0: a chain of loads, two sums over a row, and a thousand rows for every column), 256 x 4096 4.1 (1.0), 2048 x 13824 54.4 (26.3).
#include <algorithm>
#include <tuple>
#include <type_traits>

#include "lowra_common.cuh"
#include "ptx.cuh"

namespace lowra {

namespace {

constexpr int kMostThreads = 1024, kMostCols = 16384, kMostRows = 1 << 30;
constexpr int kManyRows = 2;                      // of a group, from which on the forward pass asks for its rows ahead
constexpr int kBackwardThreads = 512;               // of a CTA of the backward pass: 128 registers to each
constexpr int kForwardThreads = 512;              // of a CTA, where rows are short enough for several groups

struct NormParams {
    const uint16_t *X, *residual, *dY;            // backward: residual holds dsum
    const void *weight, *bias;
    uint16_t *sum, *Y;                            // backward: Y holds dX
    float *mean, *rstd;                           // written forward, read backward
    float* parts;                                 // backward: [CTAs][weight's, then bias's sums][N], or the gradients themselves
    int M, N, group, fp32;                        // threads to a row; parameters in fp32
    float eps, over_n;
};

// Not as read-only memory: an output may be one of the inputs.
__device__ __forceinline__ uint4 load8(const uint16_t* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void unpack8(uint4 v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ void load_params(const void* p, int fp32, int n, float (&x)[8]) {
    if (fp32) {
        const float4 a = __ldg(static_cast<const float4*>(p) + n / 4), b = __ldg(static_cast<const float4*>(p) + n / 4 + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        unpack8(__ldg(static_cast<const uint4*>(p) + n / 8), x);
    }
}

// 16 bytes into shared memory, not waited for.
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// Sums over the threads of a group (whole warps, all of one CTA), the same in every thread.  Two places in shared memory in turn, so that one barrier does: a warp
// that is a sum ahead writes into the other one.
template <int COUNT>
struct GroupSum {
    float (*shared)[kMostThreads / 32][COUNT];
    int first, warps, barrier, turn;
    __device__ __forceinline__ void operator()(float (&v)[COUNT]) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
        if (warps == 1) return;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) shared[turn][warp][i] = v[i];
        ptx::named_barrier_sync((uint32_t)barrier, (uint32_t)warps * 32u);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] = lane < warps ? shared[turn][first + lane][i] : 0.0f;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
        }
        turn ^= 1;
    }
};

// The same for the kernels that keep many rows going, with fewer instructions: behind the barrier every thread adds up the warps' sums itself, four to a read.
constexpr int kSumPlaces = 2 * kMostThreads / 32 + 64;        // of all groups' warps, those of each filled up to four
template <int COUNT>
struct RowSum {
    float* mine;              // [turn][sum][place]
    int warps, barrier, turn;
    __device__ __forceinline__ RowSum(float* shared, int group, int number) : warps(group / 32), barrier(number + 1), turn(0) {
        const int places = (warps + 3) / 4 * 4;
        mine = shared + number * places;
        if (warps == 1) return;
        const int in_group = (int)threadIdx.x - number * group;
        if (in_group < places)                        // (what no warp writes stays zero)
            for (int i = 0; i < 2 * COUNT; ++i) mine[i * kSumPlaces + in_group] = 0.0f;
        ptx::named_barrier_sync((uint32_t)barrier, (uint32_t)warps * 32u);
    }
    __device__ __forceinline__ void operator()(float (&v)[COUNT]) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
        if (warps == 1) return;
        float* at = mine + turn * COUNT * kSumPlaces;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) at[i * kSumPlaces + ((int)threadIdx.x >> 5) - (barrier - 1) * warps] = v[i];
        ptx::named_barrier_sync((uint32_t)barrier, (uint32_t)warps * 32u);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = 0.0f;
        for (int w = 0; w < warps; w += 4)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const float4 p = *reinterpret_cast<const float4*>(at + i * kSumPlaces + w);
                v[i] += (p.x + p.y) + (p.z + p.w);
            }
        turn ^= 1;
    }
};

// VECTORS of eight channels to a thread: group, group + threads, ...
template <int VECTORS, bool LAYER, bool RESIDUAL>
__global__ void __launch_bounds__(kMostThreads) forward_kernel(const NormParams P) {
    __shared__ float shared[2][kMostThreads / 32][1];
    pdl_enter();
    const int mine = (int)threadIdx.x / P.group, t = (int)threadIdx.x % P.group;
    GroupSum<1> add = {shared, mine * P.group / 32, P.group / 32, mine + 1, 0};
    const long long m = (long long)blockIdx.x * (int)(blockDim.x / P.group) + mine;
    if (m >= P.M) return;                             // (a whole group)
    float x[VECTORS][8], w[8], b[8];
    uint4 in[VECTORS], beside[VECTORS];
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        const int n = (t + v * P.group) * 8;
        if (n >= P.N) continue;
        in[v] = load8(P.X + m * P.N + n);
        if (RESIDUAL) beside[v] = load8(P.residual + m * P.N + n);
    }
    if (VECTORS == 1 && t * 8 < P.N) {                // under way with the row
        load_params(P.weight, P.fp32, t * 8, w);
        if (LAYER) load_params(P.bias, P.fp32, t * 8, b);
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        const int n = (t + v * P.group) * 8;
        if (n >= P.N) continue;
        unpack8(in[v], x[v]);
        if (RESIDUAL) {
            float r[8];
            unpack8(beside[v], r);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] += r[i];
            const uint4 h = pack8(x[v]);
            *reinterpret_cast<uint4*>(P.sum + m * P.N + n) = h;
            unpack8(h, x[v]);                         // the statistics are those of the stored sum, which the backward pass reads
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += LAYER ? x[v][i] : x[v][i] * x[v][i];
    }
    add(s);
    float mean = 0.0f;
    if (LAYER) {
        mean = s[0] * P.over_n;
        s[0] = 0.0f;
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) {
            if ((t + v * P.group) * 8 >= P.N) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[v][i] -= mean;
                s[0] += x[v][i] * x[v][i];
            }
        }
        add(s);
    }
    const float rstd = 1.0f / sqrtf(s[0] * P.over_n + P.eps);
    if (t == 0) {
        if (P.rstd != nullptr) P.rstd[m] = rstd;
        if (LAYER && P.mean != nullptr) P.mean[m] = mean;
    }
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        const int n = (t + v * P.group) * 8;
        if (n >= P.N) continue;
        if (VECTORS > 1) {
            load_params(P.weight, P.fp32, n, w);
            if (LAYER) load_params(P.bias, P.fp32, n, b);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[v][i] = LAYER ? x[v][i] * rstd * w[i] + b[i] : x[v][i] * rstd * w[i];
        *reinterpret_cast<uint4*>(P.Y + m * P.N + n) = pack8(x[v]);
    }
}

// Rows that a thread has asked for ahead (cp.async: no registers), in places in shared memory that are its own, so that no barrier is needed: [slot][vector][array][thread].
// DEPTH rows are under way, of which ROWS are worked on together, one barrier for their sums.
template <int VECTORS, int ARRAYS, int ROWS, int DEPTH>
struct Ring {
    static constexpr int kRows = ROWS, kDepth = DEPTH;
    uint4* base;
    __device__ __forceinline__ uint4* place(int slot, int v, int array) const { return base + ((slot * VECTORS + v) * ARRAYS + array) * (int)blockDim.x + (int)threadIdx.x; }
    // one row (or nothing) into a slot: a group of copies each, so that they can be counted
    __device__ __forceinline__ void ask(const NormParams& P, const uint16_t* const (&from)[ARRAYS], long long m, int t, int slot) const {
        if (m < P.M) {
#pragma unroll
            for (int v = 0; v < VECTORS; ++v) {
                const int n = (t + v * P.group) * 8;
                if (n >= P.N) continue;
                const long long at = m * P.N + n;
#pragma unroll
                for (int a = 0; a < ARRAYS; ++a) copy16(ptx::smem_u32(place(slot, v, a)), from[a] + at);
            }
        }
        ptx::cp_async_commit();
    }
    static __device__ __forceinline__ void wait() { ptx::cp_async_wait<kDepth - kRows>(); }     // the oldest kRows are there
    static size_t bytes(int threads) { return (size_t)kDepth * VECTORS * ARRAYS * threads * 16; }
};
// Forward: a row's values are read again for its output, from shared memory; of two rows under way (four of short rows) half are worked on together.
template <int VECTORS, bool RESIDUAL>
using ForwardRing = Ring<VECTORS, RESIDUAL ? 2 : 1, VECTORS == 1 ? 2 : 1, VECTORS == 1 ? 4 : 2>;
// Backward: with up to sixteen channels to a thread they are kept in registers, with 32 read again.
template <int VECTORS, bool BESIDE>
using BackwardRing = Ring<VECTORS, BESIDE ? 3 : 2, 1, VECTORS <= 2 ? 4 : 2>;

// Eight bf16 as four pairs.
__device__ __forceinline__ void unpack4(uint4 v, float2 (&x)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack4(const float2 (&x)[4]) {
    return make_uint4(pack_bf16x2(x[0].x, x[0].y), pack_bf16x2(x[1].x, x[1].y), pack_bf16x2(x[2].x, x[2].y), pack_bf16x2(x[3].x, x[3].y));
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// The parameters, read again for every row (volatile: kept over the rows, they would cost registers that the sums need).
template <bool FP32>
__device__ __forceinline__ void load_params4(const void* p, int n, float2 (&x)[4]) {
    auto get = [](const char* from) {
        uint4 v;
        asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(from));
        return v;
    };
    const char* from = static_cast<const char*>(p) + (size_t)n * (FP32 ? 4 : 2);
    const uint4 a = get(from);
    if constexpr (FP32) {
        const uint4 b = get(from + 16);
        x[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
        x[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
        x[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
        x[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
    } else {
        unpack4(a, x);
    }
}

// The forward pass over many rows: a CTA to an SM, its groups walk over the rows.
template <int VECTORS, bool LAYER, bool RESIDUAL, bool FP32>
__global__ void __launch_bounds__(kMostThreads, 1) forward_rows_kernel(const NormParams P) {
    using Rows = ForwardRing<VECTORS, RESIDUAL>;
    constexpr int R = Rows::kRows;
    __shared__ __align__(16) float shared[2 * R * kSumPlaces];
    extern __shared__ uint4 under_way[];
    pdl_enter();
    const int groups = (int)blockDim.x / P.group, mine = (int)threadIdx.x / P.group, t = (int)threadIdx.x % P.group, step = (int)gridDim.x * groups;
    RowSum<R> add(shared, P.group, mine);
    const Rows ring = {under_way};
    const uint16_t* from[RESIDUAL ? 2 : 1];
    from[0] = P.X;
    if constexpr (RESIDUAL) from[1] = P.residual;
    const long long first = (long long)blockIdx.x * groups + mine;
    for (int k = 0; k < Rows::kDepth; ++k) ring.ask(P, from, first + (long long)k * step, t, k);
    int slot0 = 0;
    for (long long m0 = first; m0 < P.M; m0 += (long long)R * step, slot0 ^= R) {
        Rows::wait();
        float s[R], mean[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long m = m0 + (long long)r * step;
            float2 part = both(0.0f);
            mean[r] = 0.0f;
            if (m < P.M)
#pragma unroll
                for (int v = 0; v < VECTORS; ++v) {
                    const int n = (t + v * P.group) * 8;
                    if (n >= P.N) continue;
                    float2 x[4];
                    uint4 h = *ring.place(slot0 + r, v, 0);
                    unpack4(h, x);
                    if constexpr (RESIDUAL) {
                        float2 y[4];
                        unpack4(*ring.place(slot0 + r, v, 1), y);
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = add2(x[i], y[i]);
                        h = pack4(x);
                        *ring.place(slot0 + r, v, 0) = h;
                        *reinterpret_cast<uint4*>(P.sum + m * P.N + n) = h;
                        unpack4(h, x);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) part = LAYER ? add2(part, x[i]) : fma2(x[i], x[i], part);
                }
            s[r] = part.x + part.y;
        }
        add(s);
        if constexpr (LAYER) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                mean[r] = s[r] * P.over_n;
                float2 part = both(0.0f);
                if (m0 + (long long)r * step < P.M)
#pragma unroll
                    for (int v = 0; v < VECTORS; ++v) {
                        if ((t + v * P.group) * 8 >= P.N) continue;
                        float2 x[4];
                        unpack4(*ring.place(slot0 + r, v, 0), x);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x[i] = add2(x[i], both(-mean[r]));
                            part = fma2(x[i], x[i], part);
                        }
                    }
                s[r] = part.x + part.y;
            }
            add(s);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long m = m0 + (long long)r * step;
            const float rstd = 1.0f / sqrtf(s[r] * P.over_n + P.eps);
            if (m < P.M) {
                if (t == 0) {
                    if (P.rstd != nullptr) P.rstd[m] = rstd;
                    if (LAYER && P.mean != nullptr) P.mean[m] = mean[r];
                }
#pragma unroll
                for (int v = 0; v < VECTORS; ++v) {
                    const int n = (t + v * P.group) * 8;
                    if (n >= P.N) continue;
                    float2 x[4], w[4], b[4];
                    load_params4<FP32>(P.weight, n, w);
                    if constexpr (LAYER) load_params4<FP32>(P.bias, n, b);
                    unpack4(*ring.place(slot0 + r, v, 0), x);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (LAYER) x[i] = fma2(mul2(add2(x[i], both(-mean[r])), both(rstd)), w[i], b[i]);
                        else x[i] = mul2(mul2(x[i], both(rstd)), w[i]);
                    }
                    *reinterpret_cast<uint4*>(P.Y + m * P.N + n) = pack4(x);
                }
            }
            ring.ask(P, from, m + (long long)Rows::kDepth * step, t, slot0 + r);
        }
    }
}

// A CTA to an SM, its groups walk over the rows.  The parameters' gradients are summed up by the threads over their rows, in registers, then over the groups of the CTA in their order, and, by another
// kernel, over the CTAs in theirs: no atomics, so repeated calls agree bit for bit.
template <int VECTORS, bool LAYER, bool BESIDE, bool SUMS, bool FP32>
__global__ void __launch_bounds__(kBackwardThreads, 1) backward_kernel(const NormParams P) {
    constexpr int kSums = LAYER ? 2 : 1;
    constexpr bool kHold = VECTORS <= 2;              // dY weight and xh, over the row's sums
    using Rows = BackwardRing<VECTORS, BESIDE>;
    __shared__ __align__(16) float shared[2 * kSums * kSumPlaces];
    extern __shared__ uint4 under_way[];
    const int groups = (int)blockDim.x / P.group, mine = (int)threadIdx.x / P.group, t = (int)threadIdx.x % P.group, step = (int)gridDim.x * groups;
    RowSum<kSums> add(shared, P.group, mine);
    float2 dw[VECTORS][4], db[VECTORS][4];
#pragma unroll
    for (int v = 0; v < VECTORS; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[v][i] = db[v][i] = both(0.0f);
    const Rows ring = {under_way};
    const uint16_t* from[BESIDE ? 3 : 2];
    from[0] = P.dY;
    from[1] = P.X;
    if constexpr (BESIDE) from[2] = P.residual;
    pdl_enter();
    const long long first = (long long)blockIdx.x * groups + mine;
    for (int k = 0; k < Rows::kDepth; ++k) ring.ask(P, from, first + (long long)k * step, t, k);
    float rstd = 0.0f, mean = 0.0f;
    auto statistics = [&](long long m) {              // of the next row, asked for before this one's sums
        if (m >= P.M) return;
        rstd = P.rstd[m];
        if (LAYER) mean = P.mean[m];
    };
    statistics(first);
    int slot = 0;
    for (long long m = first; m < P.M; m += step) {
        Rows::wait();
        constexpr int kKept = kHold ? VECTORS : 1;
        float2 along = both(0.0f), same = both(0.0f), kept_g[kKept][4], kept_xh[kKept][4];
        uint4 kept_beside[kKept];
        const float scale = rstd, level = -mean;
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) {
            const int n = (t + v * P.group) * 8;
            if (n >= P.N) continue;
            float2 w[4];
            float2(&g)[4] = kept_g[kHold ? v : 0], (&xh)[4] = kept_xh[kHold ? v : 0];
            load_params4<FP32>(P.weight, n, w);
            unpack4(*ring.place(slot, v, 0), g);
            unpack4(*ring.place(slot, v, 1), xh);
            if (kHold && BESIDE) kept_beside[kHold ? v : 0] = *ring.place(slot, v, 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                xh[i] = mul2(LAYER ? add2(xh[i], both(level)) : xh[i], both(scale));
                if (SUMS) {
                    dw[v][i] = fma2(g[i], xh[i], dw[v][i]);
                    if (LAYER) db[v][i] = add2(db[v][i], g[i]);
                }
                g[i] = mul2(g[i], w[i]);
                along = fma2(g[i], xh[i], along);
                if (LAYER) same = add2(g[i], same);
            }
        }
        if (kHold) ring.ask(P, from, m + (long long)Rows::kDepth * step, t, slot);
        statistics(m + step);
        float s[kSums];
        s[0] = along.x + along.y;
        if (LAYER) s[kSums - 1] = same.x + same.y;
        add(s);
        // dX = scale (g - same - xh along) + dsum
        const float by = -s[0] * P.over_n, less = LAYER ? -s[kSums - 1] * P.over_n : 0.0f;
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) {
            const int n = (t + v * P.group) * 8;
            if (n >= P.N) continue;
            float2 d[4];
            float2(&g)[4] = kept_g[kHold ? v : 0], (&xh)[4] = kept_xh[kHold ? v : 0];
            if constexpr (!kHold) {
                float2 w[4];
                load_params4<FP32>(P.weight, n, w);
                unpack4(*ring.place(slot, v, 0), g);
                unpack4(*ring.place(slot, v, 1), xh);
                if (BESIDE) kept_beside[0] = *ring.place(slot, v, 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    xh[i] = mul2(LAYER ? add2(xh[i], both(level)) : xh[i], both(scale));
                    g[i] = mul2(g[i], w[i]);
                }
            }
            if (BESIDE) unpack4(kept_beside[kHold ? v : 0], d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 dx = fma2(xh[i], both(by), LAYER ? add2(g[i], both(less)) : g[i]);
                g[i] = BESIDE ? fma2(dx, both(scale), d[i]) : mul2(dx, both(scale));
            }
            *reinterpret_cast<uint4*>(P.Y + m * P.N + n) = pack4(g);
        }
        if (!kHold) ring.ask(P, from, m + (long long)Rows::kDepth * step, t, slot);
        if (++slot == Rows::kDepth) slot = 0;
    }
    if (!SUMS) return;
    // all groups' sums side by side, then added up in the order of the groups
    ptx::cp_async_wait<0>();
    __syncthreads();
    float4* kept = reinterpret_cast<float4*>(under_way);
#pragma unroll
    for (int v = 0; v < VECTORS; ++v)
#pragma unroll
        for (int k = 0; k < kSums * 2; ++k) {
            const float2 a = k < 2 ? dw[v][2 * (k & 1)] : db[v][2 * (k & 1)], b = k < 2 ? dw[v][2 * (k & 1) + 1] : db[v][2 * (k & 1) + 1];
            kept[((mine * VECTORS + v) * kSums * 2 + k) * P.group + t] = make_float4(a.x, a.y, b.x, b.y);
        }
    __syncthreads();
    float* out = P.parts + (size_t)blockIdx.x * kSums * P.N;
    const int each = VECTORS * kSums * 2 * P.group;   // of a group
    for (int i = threadIdx.x; i < each; i += (int)blockDim.x) {
        const int k = i / P.group % (kSums * 2), n = (i % P.group + i / P.group / (kSums * 2) * P.group) * 8;
        if (n >= P.N) continue;
        float4 a = kept[i];
        for (int other = 1; other < groups; ++other) {
            const float4 b = kept[other * each + i];
            a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
        }
        *reinterpret_cast<float4*>(out + (size_t)(k / 2) * P.N + n + 4 * (k & 1)) = a;
    }
}

// The gradients of the parameters from the CTAs' sums, in a fixed order: 32 channels to a CTA, an eighth of the sums to each of its warps.
constexpr int kMostParts = (kNumSMs + 7) / 8;
__global__ void __launch_bounds__(256) add_parts_kernel(const float* parts, int count, int N, int sums, float* dweight, float* dbias) {
    __shared__ float shared[8][32];
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (int)blockIdx.x * 32 + lane, which = (int)blockIdx.y;
    float total = 0.0f, v[kMostParts];                // all of a warp's under way at once
#pragma unroll
    for (int i = 0; i < kMostParts; ++i) v[i] = n < N && warp + 8 * i < count ? parts[((size_t)(warp + 8 * i) * sums + which) * N + n] : 0.0f;
#pragma unroll
    for (int i = 0; i < kMostParts; ++i) total += v[i];
    shared[warp][lane] = total;
    __syncthreads();
    if (warp != 0 || n >= N) return;
    for (int w = 1; w < 8; ++w) total += shared[w][lane];
    float* out = which == 0 ? dweight : dbias;
    if (out != nullptr) out[n] = total;
}

// Few rows, where the CTAs' sums would be more than the rows themselves: the parameters' gradients are formed by CTAs of their own, beside those of the rows, from the same inputs (from L2, as a
// rule: the rows' CTAs read them at the same time).  One launch; where dX takes the place of dY or X, the columns' CTAs go ahead in a launch of their own.
// Columns: 16, 32 or 64 channels to a CTA, LANES lanes to a row's part of them, a warp 32 / LANES rows at a time, joined by shuffles, then over the warps in their order; two rows to a lane under way (four: 600 x 4096 7.8 -> 8.2 us).
struct BackwardFew {
    int first, columns;                               // CTA that the launch begins with; CTAs of the columns, before those of the rows
    float *dweight, *dbias;
};
template <bool LAYER, int LANES>
__device__ __forceinline__ void columns_of(const NormParams& P, const BackwardFew& C, int strip) {
    constexpr int kSums = LAYER ? 2 : 1, kUnder = 2;
    constexpr int kCols = 8 * LANES, kRowsOfWarp = 32 / LANES;
    __shared__ __align__(8) float shared[kMostThreads / 32][kSums][kCols];      // (written in pairs)
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, warps = (int)blockDim.x >> 5, n = strip * kCols + lane % LANES * 8;
    float2 dw[4], db[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[i] = db[i] = both(0.0f);
    const int step = warps * kRowsOfWarp;
    if (n < P.N)
        for (int m0 = warp * kRowsOfWarp + lane / LANES; m0 < P.M; m0 += kUnder * step) {
            uint4 y[kUnder], x[kUnder];
            float rstd[kUnder], mean[kUnder];
#pragma unroll
            for (int k = 0; k < kUnder; ++k) {
                const int m = m0 + k * step;
                y[k] = x[k] = make_uint4(0u, 0u, 0u, 0u);
                rstd[k] = mean[k] = 0.0f;
                if (m >= P.M) continue;
                y[k] = *reinterpret_cast<const uint4*>(P.dY + (size_t)m * P.N + n);
                x[k] = *reinterpret_cast<const uint4*>(P.X + (size_t)m * P.N + n);
                rstd[k] = P.rstd[m];
                if (LAYER) mean[k] = P.mean[m];
            }
#pragma unroll
            for (int k = 0; k < kUnder; ++k) {
                if (m0 + k * step >= P.M) continue;
                float2 g[4], xh[4];
                unpack4(y[k], g);
                unpack4(x[k], xh);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    xh[i] = mul2(LAYER ? add2(xh[i], both(-mean[k])) : xh[i], both(rstd[k]));
                    dw[i] = fma2(g[i], xh[i], dw[i]);
                    if (LAYER) db[i] = add2(db[i], g[i]);
                }
            }
        }
#pragma unroll
    for (int d = LANES; d < 32; d *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dw[i] = add2(dw[i], make_float2(__shfl_xor_sync(0xffffffffu, dw[i].x, d), __shfl_xor_sync(0xffffffffu, dw[i].y, d)));
            if (LAYER) db[i] = add2(db[i], make_float2(__shfl_xor_sync(0xffffffffu, db[i].x, d), __shfl_xor_sync(0xffffffffu, db[i].y, d)));
        }
    if (lane < LANES)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<float2*>(&shared[warp][0][lane * 8 + 2 * i]) = dw[i];
            if (LAYER) *reinterpret_cast<float2*>(&shared[warp][kSums - 1][lane * 8 + 2 * i]) = db[i];
        }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < kSums * kCols; i += (int)blockDim.x) {
        const int which = i / kCols, at = i % kCols;
        float total = 0.0f;
        for (int w = 0; w < warps; ++w) total += shared[w][which][at];
        float* out = which == 0 ? C.dweight : C.dbias;
        if (out != nullptr && strip * kCols + at < P.N) out[strip * kCols + at] = total;
    }
}

template <int VECTORS, bool LAYER, bool BESIDE, int LANES>
__global__ void __launch_bounds__(kMostThreads) backward_few_kernel(const NormParams P, const BackwardFew C) {
    constexpr int kSums = LAYER ? 2 : 1;
    __shared__ float shared[2][kMostThreads / 32][kSums];
    pdl_enter();
    const int cta = C.first + (int)blockIdx.x;
    if (cta < C.columns) {
        columns_of<LAYER, LANES>(P, C, cta);
        return;
    }
    const int mine = (int)threadIdx.x / P.group, t = (int)threadIdx.x % P.group;
    GroupSum<kSums> add = {shared, mine * P.group / 32, P.group / 32, mine + 1, 0};
    const long long m = (long long)(cta - C.columns) * (int)(blockDim.x / P.group) + mine;
    if (m >= P.M) return;                             // (a whole group)
    uint4 y[VECTORS], x[VECTORS], beside[VECTORS];
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        const int n = (t + v * P.group) * 8;
        if (n >= P.N) continue;
        y[v] = load8(P.dY + m * P.N + n);
        x[v] = load8(P.X + m * P.N + n);
        if (BESIDE) beside[v] = load8(P.residual + m * P.N + n);
    }
    const float scale = P.rstd[m], level = LAYER ? -P.mean[m] : 0.0f;
    float2 along = both(0.0f), same = both(0.0f), g[VECTORS][4], xh[VECTORS][4];
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        const int n = (t + v * P.group) * 8;
        if (n >= P.N) continue;
        float w[8];
        load_params(P.weight, P.fp32, n, w);
        unpack4(y[v], g[v]);
        unpack4(x[v], xh[v]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xh[v][i] = mul2(LAYER ? add2(xh[v][i], both(level)) : xh[v][i], both(scale));
            g[v][i] = mul2(g[v][i], make_float2(w[2 * i], w[2 * i + 1]));
            along = fma2(g[v][i], xh[v][i], along);
            if (LAYER) same = add2(g[v][i], same);
        }
    }
    float s[kSums];
    s[0] = along.x + along.y;
    if (LAYER) s[kSums - 1] = same.x + same.y;
    add(s);
    const float by = -s[0] * P.over_n, less = LAYER ? -s[kSums - 1] * P.over_n : 0.0f;
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        const int n = (t + v * P.group) * 8;
        if (n >= P.N) continue;
        float2 d[4];
        if (BESIDE) unpack4(beside[v], d);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 dx = fma2(xh[v][i], both(by), LAYER ? add2(g[v][i], both(less)) : g[v][i]);
            d[i] = BESIDE ? fma2(dx, both(scale), d[i]) : mul2(dx, both(scale));
        }
        *reinterpret_cast<uint4*>(P.Y + m * P.N + n) = pack4(d);
    }
}

struct NormShape {
    int vectors, group, threads;     // vectors to a thread, threads to a row and to a CTA
};
// Rows of up to `longest` channels by eight to a thread, longer ones by sixteen; as many rows side by side in a CTA as `most` threads have room for (a named barrier to a group of
// several warps: fifteen at most).
NormShape shape_of(int N, int most, int longest) {
    const int vectors = N <= longest ? 1 : N <= 16 * most ? 2 : 4;
    const int group = (N / 8 + 32 * vectors - 1) / (32 * vectors) * 32;
    int groups = most / group;
    if (groups < 1) groups = 1;
    if (group > 32 && groups > 15) groups = 15;
    return {vectors, group, group * groups};
}
// Many rows: what a row costs beside its elements - its reduction, its addresses - is a third less with sixteen channels to a thread.  Few rows: the shorter way.
NormShape shape_of_many(int N) { return shape_of(N, kMostThreads, 256); }
// Backward, us with eight channels to a thread and with sixteen: root mean square 8192 x 1024 18.1, 20.6; layer norm, twice the sums, 1001 x 1024 9.7, 7.3, 4096 x 4096 40.4, 34.9.
NormShape shape_of_backward(int N, bool layer) { return shape_of(N, kBackwardThreads, layer ? 256 : 2048); }
// A CTA of so many threads, or of one row.
NormShape with_threads(NormShape S, int threads) {
    const int groups = std::max(threads / S.group, 1);
    S.threads = S.group * (S.group > 32 ? std::min(groups, 15) : groups);
    return S;
}
// Up to one for each SM: a CTA to each.  Layer norm over more than two for each: sixteen channels to a thread, and so more rows at once on an SM (333 x 5120 6.8 -> 5.0 us, 149 x 4096 3.3 -> 4.1;
// root mean square 600 x 4096 6.3 -> 7.1).
NormShape shape_of_few(int M, int N, bool layer) {
    NormShape S = shape_of(N, kMostThreads, layer && M > 2 * kNumSMs ? 2048 : 8 * kMostThreads);
    return with_threads(S, M > kNumSMs ? kForwardThreads : 32);
}
// Backward, rows up to which their CTAs and those of the columns are one launch (us with two launches, a CTA to an SM, and so; layer norm / root mean square: 1 x 4096 5.1 / 3.9, 2.0 / 1.8;
// 256 x 4096 10.5 / 9.4, 4.6 / 4.6; 800 x 264 4.5 / 3.8, 3.4 / 3.3, 1500 x 264 4.9 / 5.0, 4.8 / 4.5, 2000 x 392 6.3 / 5.8, 7.9 / 7.2; 1001 x 1024 7.3 / 6.0, 5.6 / 5.0, 2000 x 1024 11.6 / 8.2, 8.3 / 7.7;
// 2048 x 2056 17.3 / 15.8, 12.4 / 11.3; 3000 x 4096 29.3 / 26.8, 28.6 / 27.9; 1500 x 13824 55.6 / 49.3, 51.7 / 49.9, 2048 x 13824 67.5 / 60.2, 70.2 / 67.5.  What three arrays take at the copy rate: 256 x 4096 1.0, 1500 x 264 0.4, 2000 x 392 0.7, 1001 x 1024 1.0, 2000 x 1024 1.9, 2048 x 2056 3.9,
// 3000 x 4096 11.4, 1500 x 13824 19.3, 2048 x 13824 26.3: about the border both ways are two to three times that, as large sums or as inputs read twice).
int few_rows_of(int N) { return N <= 8192 ? std::min(1024 + N, 2048) : 1536; }
// Sixteen channels to a thread above 4096, for two CTAs to an SM (600 x 8192 19.1 -> 11.2); few warps would go over the columns' rows for long (128 x 256 with one warp 4.0 us, with eight 1.7;
// 2048 x 2056 with nine 16.1, with eighteen 12.4; 2048 x 2552, of ten warps a row, twenty 18.6, ten 14.3).
NormShape shape_of_few_backward(int M, int N) { return with_threads(shape_of(N, kMostThreads, 4096), M > kNumSMs ? kForwardThreads + kForwardThreads / 8 : 256); }
// Lanes to a row of the columns (8 channels each): as few as leave the SMs room for the columns' CTAs beside the rows' (four and eight: 256 x 4096 5.2 -> 4.6 us, 128 x 8192 5.6 -> 4.2, 1001 x 5120, 160 CTAs of
// ten warps, 11.9 -> 15.8; four and two, which takes hold with more than a few
// rows to a lane: 1001 x 1024 6.2 -> 5.6, 1500 x 1288 8.0 -> 7.4, 300 x 1024 3.0 -> 3.3).
int lanes_of_columns(int M, int N, const NormShape& S) {
    for (int lanes = M > 512 ? 2 : 4; lanes < 8; lanes *= 2)
        if ((N + 8 * lanes - 1) / (8 * lanes) * S.threads <= 360 * kNumSMs) return lanes;
    return 8;
}

cudaLaunchConfig_t config_of(unsigned grid, int threads, size_t bytes, cudaStream_t stream, cudaLaunchAttribute* attr) {
    cudaLaunchConfig_t cfg = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

bool good_shape(int M, int N) { return M >= 1 && M <= kMostRows && N >= 8 && N <= kMostCols && N % 8 == 0; }

// Of outputs and inputs of one extent: the same array, or none of its bytes.
bool in_the_way(const Span* out, int outs, const Span* in, int ins, bool same_may) {
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < ins; ++j)
            if (!(same_may && out[i].at == in[j].at) && overlap(out[i], in[j])) return true;
        for (int j = i + 1; j < outs; ++j)
            if (overlap(out[i], out[j])) return true;
    }
    return false;
}

template <int VECTORS, bool LAYER, bool BESIDE, bool SUMS, bool FP32>
lowra_status launch_backward(const NormParams& P, const NormShape& S, int ctas, cudaStream_t stream) {
    static SmemLimit limit = {};
    const size_t bytes = BackwardRing<VECTORS, BESIDE>::bytes(S.threads);        // (room for the sums too: 32 or 64 bytes for eight channels, where the rows take 64 or more)
    const auto kernel = backward_kernel<VECTORS, LAYER, BESIDE, SUMS, FP32>;
    if (ensure_smem_limit(reinterpret_cast<const void*>(kernel), bytes, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = config_of((unsigned)ctas, S.threads, bytes, stream, attr);
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}
// Truth values as types: launch(std::true_type or std::false_type, ...), one for each of them.
template <typename F, typename... Types>
lowra_status choose(F launch, std::tuple<Types...>) { return launch(Types()...); }
template <typename F, typename... Types, typename... More>
lowra_status choose(F launch, std::tuple<Types...>, bool value, More... more) {
    return value ? choose(launch, std::tuple<Types..., std::true_type>(), more...) : choose(launch, std::tuple<Types..., std::false_type>(), more...);
}

int backward_ctas(int M, int N, const NormShape& S) {
    const int groups = S.threads / S.group, wanted = (M + groups - 1) / groups;
    return wanted < kNumSMs ? wanted : kNumSMs;
}

}  // namespace
}  // namespace lowra

extern "C" size_t lowra_norm_workspace_bytes(int32_t M, int32_t N) {
    using namespace lowra;
    if (!good_shape(M, N)) return 0;
    const size_t layer = (size_t)backward_ctas(M, N, shape_of_backward(N, true)) * 2, rms = (size_t)backward_ctas(M, N, shape_of_backward(N, false));
    return ((layer > rms ? layer : rms) * (size_t)N * 4 + 255) / 256 * 256;
}

extern "C" lowra_status lowra_norm_forward(const uint16_t* X_dev, const uint16_t* residual_dev, const void* weight_dev, const void* bias_dev, int32_t params_fp32,
                                           int32_t M, int32_t N, int32_t kind, float eps, uint16_t* sum_dev, uint16_t* Y_dev, float* mean_dev, float* rstd_dev,
                                           void* stream_v) {
    using namespace lowra;
    const bool layer = kind == LOWRA_NORM_LAYER;
    if (!X_dev || !weight_dev || !Y_dev || (residual_dev == nullptr) != (sum_dev == nullptr) || (layer && !bias_dev)) return LOWRA_ERR_NULL;
    if (!good_shape(M, N) || (kind != LOWRA_NORM_LAYER && kind != LOWRA_NORM_RMS) || (!layer && (bias_dev || mean_dev)) || !(eps >= 0.0f)) return LOWRA_ERR_SHAPE;
    if (!aligned16(X_dev) || !aligned16(residual_dev) || !aligned16(weight_dev) || !aligned16(bias_dev) || !aligned16(sum_dev) || !aligned16(Y_dev) ||
        !aligned16(mean_dev) || !aligned16(rstd_dev))
        return LOWRA_ERR_ALIGN;
    const size_t rows = (size_t)M * (size_t)N * 2, params = (size_t)N * (params_fp32 ? 4 : 2);
    const Span big[2] = {{X_dev, rows}, {residual_dev, rows}}, small[2] = {{weight_dev, params}, {bias_dev, params}};
    const Span out[4] = {{sum_dev, rows}, {Y_dev, rows}, {mean_dev, (size_t)M * 4}, {rstd_dev, (size_t)M * 4}};
    if (in_the_way(out, 2, big, 2, true) || in_the_way(out, 4, small, 2, false) || in_the_way(out + 2, 2, big, 2, false)) return LOWRA_ERR_SHAPE;
    const lowra_status st = check_device();
    if (st != LOWRA_OK) return st;
    NormParams P = {X_dev, residual_dev, nullptr, weight_dev, bias_dev, sum_dev, Y_dev, mean_dev, rstd_dev, nullptr, M, N, 0, params_fp32 != 0, eps, 1.0f / (float)N};
    cudaStream_t stream = (cudaStream_t)stream_v;
    const NormShape many = shape_of_many(N);
    if (M >= kManyRows * kNumSMs * (many.threads / many.group)) {
        P.group = many.group;
        return choose([&](auto two, auto is_layer, auto with_residual, auto fp32) {
            static SmemLimit limit = {};
            const auto kernel = forward_rows_kernel<two ? 2 : 1, is_layer, with_residual, fp32>;
            const size_t bytes = ForwardRing<two ? 2 : 1, with_residual>::bytes(many.threads);
            if (ensure_smem_limit(reinterpret_cast<const void*>(kernel), bytes, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
            cudaLaunchAttribute attr[1];
            const cudaLaunchConfig_t cfg = config_of((unsigned)kNumSMs, many.threads, bytes, stream, attr);
            return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
        }, std::tuple<>(), many.vectors == 2, layer, residual_dev != nullptr, params_fp32 != 0);
    }
    const NormShape S = shape_of_few(M, N, layer);
    const int groups = S.threads / S.group;
    P.group = S.group;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = config_of((unsigned)((M + groups - 1) / groups), S.threads, 0, stream, attr);
    auto pick = [&](auto vectors) {
        constexpr int V = decltype(vectors)::value;
        if (layer) return residual_dev ? forward_kernel<V, true, true> : forward_kernel<V, true, false>;
        return residual_dev ? forward_kernel<V, false, true> : forward_kernel<V, false, false>;
    };
    const auto kernel = S.vectors == 1 ? pick(std::integral_constant<int, 1>()) : pick(std::integral_constant<int, 2>());
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}

extern "C" lowra_status lowra_norm_backward(const uint16_t* dY_dev, const uint16_t* X_dev, const void* weight_dev, int32_t params_fp32, const float* mean_dev,
                                            const float* rstd_dev, const uint16_t* dsum_dev, int32_t M, int32_t N, uint16_t* dX_dev, float* dweight_dev,
                                            float* dbias_dev, void* workspace_dev, size_t workspace_bytes, void* stream_v) {
    using namespace lowra;
    if (!dY_dev || !X_dev || !weight_dev || !rstd_dev || !dX_dev) return LOWRA_ERR_NULL;
    const bool layer = mean_dev != nullptr, sums = dweight_dev || dbias_dev;
    if (!good_shape(M, N) || (dbias_dev && !layer)) return LOWRA_ERR_SHAPE;
    if (!aligned16(dY_dev) || !aligned16(X_dev) || !aligned16(weight_dev) || !aligned16(mean_dev) || !aligned16(rstd_dev) || !aligned16(dsum_dev) ||
        !aligned16(dX_dev) || !aligned16(dweight_dev) || !aligned16(dbias_dev))
        return LOWRA_ERR_ALIGN;
    if (sums && (!workspace_dev || workspace_bytes < lowra_norm_workspace_bytes(M, N) || (reinterpret_cast<uintptr_t>(workspace_dev) & 255u) != 0)) return LOWRA_ERR_WORKSPACE;
    const size_t rows = (size_t)M * (size_t)N * 2;
    const Span big[3] = {{dY_dev, rows}, {X_dev, rows}, {dsum_dev, rows}};
    const Span small[3] = {{weight_dev, (size_t)N * (params_fp32 ? 4 : 2)}, {mean_dev, (size_t)M * 4}, {rstd_dev, (size_t)M * 4}};
    const Span out[3] = {{dX_dev, rows}, {dweight_dev, (size_t)N * 4}, {dbias_dev, (size_t)N * 4}};
    const Span scratch[1] = {{sums ? workspace_dev : nullptr, sums ? lowra_norm_workspace_bytes(M, N) : 0}};
    if (in_the_way(out, 1, big, 3, true) || in_the_way(out, 3, small, 3, false) || in_the_way(out + 1, 2, big, 3, false) || in_the_way(out, 3, scratch, 1, false) ||
        in_the_way(scratch, 1, big, 3, false) || in_the_way(scratch, 1, small, 3, false))
        return LOWRA_ERR_SHAPE;
    lowra_status st = check_device();
    if (st != LOWRA_OK) return st;
    const bool in_place = sums && (dX_dev == dY_dev || dX_dev == X_dev);      // (two launches either way: 600 x 1024 6.3 us as columns and rows, 5.3 a CTA to an SM)
    const bool few = M <= (in_place ? few_rows_of(N) / 4 : few_rows_of(N));
    const NormShape S = few ? shape_of_few_backward(M, N) : shape_of_backward(N, layer);
    const int ctas = backward_ctas(M, N, S);
    NormParams P = {X_dev, dsum_dev, dY_dev, weight_dev, nullptr, nullptr, dX_dev, const_cast<float*>(mean_dev), const_cast<float*>(rstd_dev),
                    static_cast<float*>(workspace_dev), M, N, S.group, params_fp32 != 0, 0.0f, 1.0f / (float)N};
    cudaStream_t stream = (cudaStream_t)stream_v;
    if (few) {
        const int lanes = lanes_of_columns(M, N, S);
        const int columns = sums ? (N + 8 * lanes - 1) / (8 * lanes) : 0, groups = S.threads / S.group, rows_ctas = (M + groups - 1) / groups;
        auto launch = [&](int first, int count) {
            return choose([&](auto two, auto is_layer, auto beside, auto two_lanes, auto four_lanes) {
                cudaLaunchAttribute attr[1];
                const cudaLaunchConfig_t cfg = config_of((unsigned)count, S.threads, 0, stream, attr);
                return cudaLaunchKernelEx(&cfg, backward_few_kernel<two ? 2 : 1, is_layer, beside, two_lanes ? 2 : four_lanes ? 4 : 8>, P, BackwardFew{first, columns, dweight_dev, dbias_dev}) == cudaSuccess ? LOWRA_OK
                                                                                                                                                                           : LOWRA_ERR_CUDA;
            }, std::tuple<>(), S.vectors == 2, layer, dsum_dev != nullptr, lanes == 2, lanes == 4);
        };
        if (in_place) st = launch(0, columns);
        return st != LOWRA_OK ? st : in_place ? launch(columns, rows_ctas) : launch(0, columns + rows_ctas);
    }
    st = choose([&](auto four, auto two, auto is_layer, auto beside, auto with_sums, auto fp32) {
        return launch_backward<four ? 4 : two ? 2 : 1, is_layer, beside, with_sums, fp32>(P, S, ctas, stream);
    }, std::tuple<>(), S.vectors == 4, S.vectors == 2, layer, dsum_dev != nullptr, sums, params_fp32 != 0);
    if (st != LOWRA_OK || !sums) return st;
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config_of((unsigned)((N + 31) / 32), 256, 0, stream, attr);
    cfg.gridDim.y = layer ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, add_parts_kernel, (const float*)P.parts, ctas, (int)N, layer ? 2 : 1, dweight_dev, dbias_dev) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}
