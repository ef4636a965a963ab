// lowra_norm_forward / lowra_norm_backward: the norm before a layer's projections, with the residual stream's addition on the way,
//     h = bf16(X + residual);   Y = (h - mu) rstd weight + bias,   rstd = 1 / sqrt(mean (h - mu)^2 + eps)          (root mean square: mu = 0, no bias)
// and its gradient, with g = dY weight and xh = (h - mu) rstd,
//     dX = rstd (g - mean g - xh mean(g xh)) + dsum;    dweight = sum over the rows of dY xh;    dbias = sum over the rows of dY
// Bound by memory.  A row is taken by one group of threads, eight neighbouring channels (16 bytes) to a thread, sixteen above 8192 channels, and stays in their
// registers between its statistics and its output: every array is read or written once.  The statistics are sums in fp32 over the registers; the variance is that of the
// differences from the mean, a second sum, so that a mean far from zero costs no digits.
#include "lowra_common.cuh"
#include "ptx.cuh"

namespace lowra {

namespace {

constexpr int kMostThreads = 1024, kMostCols = 16384, kMostRows = 1 << 30;
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

// The same, read again for every row (volatile: kept over the rows, they would cost registers that the sums need).
__device__ __forceinline__ void load_params_again(const void* p, int fp32, int n, float (&x)[8]) {
    auto get = [](const char* from) {
        uint4 v;
        asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(from));
        return v;
    };
    const char* from = static_cast<const char*>(p) + (size_t)n * (fp32 ? 4 : 2);
    const uint4 a = get(from);
    if (fp32) {
        const uint4 b = get(from + 16);
        x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
        x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
    } else {
        unpack8(a, x);
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

// A CTA to an SM, its groups walk over the rows.  What a thread reads of a row it has asked for some rows ahead, into places in shared memory that are its own (cp.async: no barrier,
// no registers; 4096 rows of 4096 with dsum 40.0 us with one row ahead in registers).  The parameters' gradients are summed up by the threads over their rows, in registers (in shared memory where
// a thread has sixteen channels), then over the groups of the CTA in their order, and, by another kernel, over the CTAs in theirs: no atomics, so repeated calls agree bit for bit.
template <int VECTORS, bool LAYER, bool BESIDE, bool SUMS>
__global__ void __launch_bounds__(kMostThreads, 1) backward_kernel(const NormParams P, const int depth) {
    constexpr int kSums = LAYER ? 2 : 1, kArrays = BESIDE ? 3 : 2;
    __shared__ float shared[2][kMostThreads / 32][kSums];
    extern __shared__ float4 kept[];                  // VECTORS > 1: [vector][weight's, bias's][half][thread]; else, at the end, one row of sums;  behind them the rows under way
    const int groups = (int)blockDim.x / P.group, mine = (int)threadIdx.x / P.group, t = (int)threadIdx.x % P.group, threads = (int)blockDim.x;
    GroupSum<kSums> add = {shared, mine * P.group / 32, P.group / 32, mine + 1, 0};
    const int step = (int)gridDim.x * groups;
    float dw[8], db[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[i] = db[i] = 0.0f;
    if (SUMS && VECTORS > 1)
        for (int k = 0; k < VECTORS * kSums * 2; ++k) kept[k * threads + (int)threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
    const uint4* ring = reinterpret_cast<const uint4*>(kept + (!SUMS ? 0 : VECTORS > 1 ? VECTORS * kSums * 2 * threads : kSums * 2 * P.group)) + threadIdx.x;   // [slot][vector][array][thread]
    pdl_enter();
    auto ask = [&](long long m, int slot) {
        if (m < P.M) {
#pragma unroll
            for (int v = 0; v < VECTORS; ++v) {
                const int n = (t + v * P.group) * 8;
                if (n >= P.N) continue;
                const uint32_t to = ptx::smem_u32(ring + (slot * VECTORS + v) * kArrays * threads);
                const long long at = m * P.N + n;
                copy16(to, P.dY + at);
                copy16(to + 16u * threads, P.X + at);
                if (BESIDE) copy16(to + 32u * threads, P.residual + at);
            }
        }
        ptx::cp_async_commit();
    };
    long long m = (long long)blockIdx.x * groups + mine, ahead = m;
    for (int k = 0; k < depth; ++k, ahead += step) ask(ahead, k);
    float rstd = 0.0f, mean = 0.0f;
    auto statistics = [&](long long of) {
        if (of >= P.M) return;
        rstd = P.rstd[of];
        if (LAYER) mean = P.mean[of];
    };
    statistics(m);
    int slot = 0;
    for (; m < P.M; m += step) {
        if (depth == 1) ptx::cp_async_wait<0>();
        else if (depth == 2) ptx::cp_async_wait<1>();
        else ptx::cp_async_wait<3>();
        float s[kSums];
#pragma unroll
        for (int i = 0; i < kSums; ++i) s[i] = 0.0f;
        float g[VECTORS][8], xh[VECTORS][8];
        uint4 beside[VECTORS];
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) {
            const int n = (t + v * P.group) * 8;
            if (n >= P.N) continue;
            float wf[8];
            load_params_again(P.weight, P.fp32, n, wf);
            const uint4* row = ring + (slot * VECTORS + v) * kArrays * threads;
            unpack8(row[0], g[v]);
            unpack8(row[threads], xh[v]);
            if (BESIDE) beside[v] = row[2 * threads];
            float pw[8], pb[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (LAYER) xh[v][i] -= mean;
                xh[v][i] *= rstd;
                pw[i] = g[v][i] * xh[v][i];
                pb[i] = g[v][i];
                g[v][i] *= wf[i];
                s[0] += g[v][i] * xh[v][i];
                if (LAYER) s[kSums - 1] += g[v][i];
            }
            if (SUMS && VECTORS == 1) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dw[i] += pw[i];
                    if (LAYER) db[i] += pb[i];
                }
            } else if (SUMS) {
                float4* at = kept + (size_t)v * kSums * 2 * threads + threadIdx.x;
#pragma unroll
                for (int k = 0; k < kSums * 2; ++k) {
                    float4 a = at[k * threads];
                    const float* p = k < 2 ? pw + 4 * k : pb + 4 * (k - 2);
                    a.x += p[0]; a.y += p[1]; a.z += p[2]; a.w += p[3];
                    at[k * threads] = a;
                }
            }
        }
        ask(ahead, slot);                             // into the place that has just been read
        ahead += step;
        if (++slot == depth) slot = 0;
        const float scale = rstd;
        statistics(m + step);
        add(s);
        const float along = s[0] * P.over_n, level = LAYER ? s[kSums - 1] * P.over_n : 0.0f;
#pragma unroll
        for (int v = 0; v < VECTORS; ++v) {
            const int n = (t + v * P.group) * 8;
            if (n >= P.N) continue;
            float d[8];
            if (BESIDE) unpack8(beside[v], d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float dx = g[v][i] - xh[v][i] * along;
                if (LAYER) dx -= level;
                dx *= scale;
                g[v][i] = BESIDE ? dx + d[i] : dx;
            }
            *reinterpret_cast<uint4*>(P.Y + m * P.N + n) = pack8(g[v]);
        }
    }
    if (!SUMS) return;
    float* out = P.parts + (size_t)blockIdx.x * kSums * P.N;
    if constexpr (VECTORS > 1) {                      // one group
        for (int v = 0; v < VECTORS; ++v) {
            const int n = (t + v * P.group) * 8;
            if (n >= P.N) continue;
            for (int k = 0; k < kSums * 2; ++k)
                *reinterpret_cast<float4*>(out + (size_t)(k / 2) * P.N + n + 4 * (k & 1)) = kept[(size_t)(v * kSums * 2 + k) * blockDim.x + threadIdx.x];
        }
    } else for (int turn = 0; turn < groups; ++turn) {       // group after group adds its sums to those of the ones before
        if (mine == turn && t * 8 < P.N) {
            float4* at = kept + t;
#pragma unroll
            for (int k = 0; k < kSums * 2; ++k) {
                const float* p = k < 2 ? dw + 4 * k : db + 4 * (k - 2);
                float4 a = make_float4(p[0], p[1], p[2], p[3]);
                if (turn > 0) {
                    const float4 b = at[k * P.group];
                    a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
                }
                if (turn + 1 < groups) at[k * P.group] = a;
                else *reinterpret_cast<float4*>(out + (size_t)(k / 2) * P.N + t * 8 + 4 * (k & 1)) = a;
            }
        }
        __syncthreads();
    }
}

// The gradients of the parameters from the CTAs' sums, in the order of the CTAs: 32 channels to a CTA, an eighth of the sums to each of its warps.
__global__ void __launch_bounds__(256) add_parts_kernel(const float* parts, int count, int N, int sums, float* dweight, float* dbias) {
    __shared__ float shared[8][32];
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (int)blockIdx.x * 32 + lane, which = (int)blockIdx.y;
    const int first = count * warp / 8, end = count * (warp + 1) / 8;
    float total = 0.0f;
    if (n < N) {
#pragma unroll 8
        for (int i = first; i < end; ++i) total += parts[((size_t)i * sums + which) * N + n];
    }
    shared[warp][lane] = total;
    __syncthreads();
    if (warp != 0 || n >= N) return;
    for (int w = 1; w < 8; ++w) total += shared[w][lane];
    float* out = which == 0 ? dweight : dbias;
    if (out != nullptr) out[n] = total;
}

struct NormShape {
    int vectors, group, threads;     // vectors to a thread, threads to a row and to a CTA
};
// Rows of up to 8192 channels by eight to a thread, longer ones by sixteen; as many rows side by side in a CTA as `most` threads have room for (a named barrier to a group
// of several warps: fifteen at most).
NormShape shape_of(int N, int most) {
    const int vectors = N <= 8 * kMostThreads ? 1 : 2;
    const int group = (N / 8 + 32 * vectors - 1) / (32 * vectors) * 32;
    int groups = most / group;
    if (groups < 1) groups = 1;
    if (group > 32 && groups > 15) groups = 15;
    return {vectors, group, group * groups};
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

template <int VECTORS, bool LAYER, bool BESIDE, bool SUMS>
lowra_status launch_backward(const NormParams& P, const NormShape& S, int ctas, cudaStream_t stream) {
    static SmemLimit limit = {};
    constexpr size_t kMost = 225 * 1024;
    const size_t sums = !SUMS ? 0 : VECTORS > 1 ? (size_t)VECTORS * (LAYER ? 2 : 1) * 2 * S.threads * 16 : (size_t)(LAYER ? 2 : 1) * 2 * S.group * 16;
    const size_t row = (size_t)VECTORS * (BESIDE ? 3 : 2) * S.threads * 16;
    const int depth = sums + 4 * row <= kMost ? 4 : sums + 2 * row <= kMost ? 2 : 1;        // rows ahead
    const auto kernel = backward_kernel<VECTORS, LAYER, BESIDE, SUMS>;
    if (ensure_smem_limit(reinterpret_cast<const void*>(kernel), sums + (size_t)depth * row, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = config_of((unsigned)ctas, S.threads, sums + (size_t)depth * row, stream, attr);
    return cudaLaunchKernelEx(&cfg, kernel, P, depth) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}
template <int VECTORS>
lowra_status launch_backward(const NormParams& P, const NormShape& S, int ctas, bool layer, bool beside, bool sums, cudaStream_t stream) {
    if (layer) {
        if (beside) return sums ? launch_backward<VECTORS, true, true, true>(P, S, ctas, stream) : launch_backward<VECTORS, true, true, false>(P, S, ctas, stream);
        return sums ? launch_backward<VECTORS, true, false, true>(P, S, ctas, stream) : launch_backward<VECTORS, true, false, false>(P, S, ctas, stream);
    }
    if (beside) return sums ? launch_backward<VECTORS, false, true, true>(P, S, ctas, stream) : launch_backward<VECTORS, false, true, false>(P, S, ctas, stream);
    return sums ? launch_backward<VECTORS, false, false, true>(P, S, ctas, stream) : launch_backward<VECTORS, false, false, false>(P, S, ctas, stream);
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
    return ((size_t)backward_ctas(M, N, shape_of(N, kMostThreads)) * 2 * (size_t)N * 4 + 255) / 256 * 256;
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
    const NormShape S = shape_of(N, M > kNumSMs ? kForwardThreads : 0);      // (few rows: a CTA to each)
    const int groups = S.threads / S.group;
    const NormParams P = {X_dev, residual_dev, nullptr, weight_dev, bias_dev, sum_dev, Y_dev, mean_dev, rstd_dev, nullptr, M, N, S.group, params_fp32 != 0, eps,
                          1.0f / (float)N};
    cudaLaunchAttribute attr[1];
    const cudaLaunchConfig_t cfg = config_of((unsigned)((M + groups - 1) / groups), S.threads, 0, (cudaStream_t)stream_v, attr);
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
    const NormShape S = shape_of(N, kMostThreads);
    const int ctas = backward_ctas(M, N, S);
    NormParams P = {X_dev, dsum_dev, dY_dev, weight_dev, nullptr, nullptr, dX_dev, const_cast<float*>(mean_dev), const_cast<float*>(rstd_dev),
                    static_cast<float*>(workspace_dev), M, N, S.group, params_fp32 != 0, 0.0f, 1.0f / (float)N};
    cudaStream_t stream = (cudaStream_t)stream_v;
    st = S.vectors == 1 ? launch_backward<1>(P, S, ctas, layer, dsum_dev != nullptr, sums, stream) : launch_backward<2>(P, S, ctas, layer, dsum_dev != nullptr, sums, stream);
    if (st != LOWRA_OK || !sums) return st;
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config_of((unsigned)((N + 31) / 32), 256, 0, stream, attr);
    cfg.gridDim.y = layer ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, add_parts_kernel, (const float*)P.parts, ctas, (int)N, layer ? 2 : 1, dweight_dev, dbias_dev) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}
