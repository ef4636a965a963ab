// lowra_epilogue_backward: the gradient through what stands behind a product,
//     dZ = dY * multiply * act'(Z),   dmultiply = dY * act(Z),   dbias[n] = sum over the tokens of dZ[m, n]
// Bound by memory: 2 bytes for every element of every array, each read or written once (4096 x 11008: gated, five arrays, 72 us = 6.2 TB/s; GELU, three, 46 us = 5.8, with the
// bias's sums 51).  A thread takes eight neighbouring channels (16 bytes) of a row;
// without a bias the elements are dealt out flat, with one a CTA takes 256 channels of a run of rows, sums them up in registers (fp32, before dZ is rounded),
// its eight warps' sums through shared memory, and writes them down for a second kernel that adds up the runs in their order: no atomics, so repeated calls
// agree bit for bit.  The second launch is left out where one run holds all rows, as with up to 128 rows, which narrower CTAs take whole.  (Up to eight runs as a cluster that adds up through distributed shared memory:
// no second launch, but 333 x 4096 with GELU 6.7 -> 7.1 us, 1001 x 13824 20.2 -> 27.2, whose clusters do not all find room at once.)
#include "epilogue.cuh"

namespace lowra {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kCols = 32 * 8;
constexpr int kNarrowThreads = 512, kNarrowCols = 8 * 8, kNarrowRows = 128;
constexpr int kResident = 3;              // CTAs to an SM
constexpr int kLeastRows = 16;            // of a run

struct BackwardParams {
    const uint16_t *dY, *pre, *multiply;
    uint16_t *dZ, *dmultiply;
    float* sums;                          // [runs][N], or dbias itself
    int M, N, activation, rows;           // rows of a run
};

struct Vec8 {
    uint4 dY, z, m;
};

// Read once, and not as read-only memory (ld_stream_v4): an output may be one of the inputs, and while a thread writes only what it has read itself, its
// neighbours' values lie in the same sectors.  (Nothing comes before a load: what a thread reads it has not written.)
__device__ __forceinline__ uint4 ld_once_v4(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <bool MULTIPLY>
__device__ __forceinline__ void load(const BackwardParams& P, size_t at, Vec8& v) {
    v.dY = ld_once_v4(P.dY + at);
    if (P.pre != nullptr) v.z = ld_once_v4(P.pre + at);
    if (MULTIPLY) v.m = ld_once_v4(P.multiply + at);
}

// Eight elements: dZ, returned in fp32 too, and dmultiply.
template <bool MULTIPLY>
__device__ __forceinline__ void differentiate(const BackwardParams& P, size_t at, const Vec8& v, float (&dz)[8]) {
    float dh[8], z[8], h[8];
    unpack8(v.dY, dz);
    if (P.pre != nullptr) unpack8(v.z, z);
#pragma unroll
    for (int i = 0; i < 8; ++i) dh[i] = dz[i];
    if (MULTIPLY) {
        float m[8];
        unpack8(v.m, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) dz[i] *= m[i];
    }
    auto all = [&](auto act) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float2 a, slope;
            activate_and_slope<decltype(act)::value>(make_float2(z[i], z[i + 1]), &a, &slope);
            dz[i] *= slope.x;
            dz[i + 1] *= slope.y;
            h[i] = a.x;
            h[i + 1] = a.y;
        }
    };
    if (P.activation == LOWRA_ACT_RELU) all(std::integral_constant<int, LOWRA_ACT_RELU>());
    else if (P.activation == LOWRA_ACT_GELU) all(std::integral_constant<int, LOWRA_ACT_GELU>());
    else if (P.activation == LOWRA_ACT_GELU_TANH) all(std::integral_constant<int, LOWRA_ACT_GELU_TANH>());
    else if (P.activation == LOWRA_ACT_SILU) all(std::integral_constant<int, LOWRA_ACT_SILU>());
    else if (P.pre != nullptr) all(std::integral_constant<int, LOWRA_ACT_NONE>());
    if (P.dZ != nullptr) *reinterpret_cast<uint4*>(P.dZ + at) = pack8(dz);
    if (MULTIPLY && P.dmultiply != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] *= dh[i];
        *reinterpret_cast<uint4*>(P.dmultiply + at) = pack8(h);
    }
}

template <bool MULTIPLY>
__global__ void __launch_bounds__(kThreads, kResident) flat_kernel(const __grid_constant__ BackwardParams P) {
    constexpr int kRowsAtOnce = MULTIPLY ? 2 : 4;         // whose loads are under way together
    pdl_enter();
    const size_t vectors = (size_t)P.M * (size_t)(P.N / 8), step = (size_t)gridDim.x * kThreads;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < vectors; i += kRowsAtOnce * step) {
        Vec8 v[kRowsAtOnce];
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u)
            if (i + u * step < vectors) load<MULTIPLY>(P, (i + u * step) * 8, v[u]);
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u) {
            float dz[8];
            if (i + u * step < vectors) differentiate<MULTIPLY>(P, (i + u * step) * 8, v[u], dz);
        }
    }
}

template <bool MULTIPLY, int THREADS, int COLS>
__global__ void __launch_bounds__(THREADS, THREADS == kThreads ? kResident : 1) rows_kernel(const __grid_constant__ BackwardParams P) {
    constexpr int kRowsAtOnce = MULTIPLY ? 2 : 4;         // whose loads are under way together
    constexpr int kLanes = COLS / 8, kStep = THREADS / kLanes;      // lanes to a row, rows side by side
    __shared__ float shared[THREADS / 32][COLS];
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x % kLanes, n = (int)blockIdx.x * COLS + lane * 8;
    const int m_first = (int)blockIdx.y * P.rows, m_end = min(P.M, m_first + P.rows);
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    for (int m = m_first + (int)threadIdx.x / kLanes; n < P.N && m < m_end; m += kRowsAtOnce * kStep) {
        Vec8 v[kRowsAtOnce];
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u)
            if (m + u * kStep < m_end) load<MULTIPLY>(P, (size_t)(m + u * kStep) * P.N + n, v[u]);
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u) {
            if (m + u * kStep >= m_end) break;
            float dz[8];
            differentiate<MULTIPLY>(P, (size_t)(m + u * kStep) * P.N + n, v[u], dz);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += dz[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int other = kLanes; other < 32; other *= 2) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], other);
        if ((threadIdx.x & 31) < kLanes) shared[warp][lane * 8 + i] = sum[i];
    }
    __syncthreads();
    const int col = (int)blockIdx.x * COLS + (int)threadIdx.x;
    if (threadIdx.x >= COLS || col >= P.N) return;
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) total += shared[w][threadIdx.x];
    P.sums[(size_t)blockIdx.y * P.N + col] = total;
}

// A CTA takes 32 channels, each of its eight warps an eighth of the runs.
__global__ void __launch_bounds__(kThreads) sum_runs_kernel(const float* sums, int runs, int N, float* out) {
    __shared__ float shared[kWarps][32];
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = (int)blockIdx.x * 32 + lane;
    const int first = runs * warp / kWarps, end = runs * (warp + 1) / kWarps;
    float total = 0.0f;
    if (n < N) {
#pragma unroll 4
        for (int i = first; i < end; ++i) total += sums[(size_t)i * N + n];
    }
    shared[warp][lane] = total;
    __syncthreads();
    if (warp != 0 || n >= N) return;
    for (int w = 1; w < kWarps; ++w) total += shared[w][lane];
    out[n] = total;
}

constexpr int kMostRows = 1 << 30, kMostCols = 1 << 24;       // (rows and their steps are counted in 32 bits)
// Few rows: CTAs of 64 channels (eight lanes to a row, 64 rows side by side) that hold all rows each, and one launch, as long as all of them fit at once.
// 512, 4096 and 9472 channels with GELU: 24 rows 1.6, 1.6, 1.7 us against 2.9, 3.1, 3.6 in runs, 128 rows 2.5, 2.7, 3.2 against 3.1, 4.2, 4.7; past either bound
// it loses sooner or later (10240 channels, 128 rows 5.2 against 4.8; 512 channels gated, 200 rows 3.9 against 3.6; 4096, 333 rows 7.1 against 6.1).
bool takes_narrow(int M, int N) { return M <= kNarrowRows && N <= kNumSMs * kNarrowCols; }

// So many that their CTAs are all resident at once (one more wave of a few cost a third of the time: 4096 x 11008 gated 72 -> 100 us).
int runs_of(int M, int N) {
    if (takes_narrow(M, N)) return 1;
    const int tiles = (N + kCols - 1) / kCols, wanted = kNumSMs * kResident / tiles, most = (M + kLeastRows - 1) / kLeastRows;
    return wanted < 1 ? 1 : wanted < most ? wanted : most;
}

}  // namespace
}  // namespace lowra

extern "C" size_t lowra_epilogue_workspace_bytes(int32_t M, int32_t N) {
    if (M < 1 || M > lowra::kMostRows || N < 8 || N > lowra::kMostCols || N % 8 != 0) return 0;
    return ((size_t)lowra::runs_of(M, N) * (size_t)N * 4 + 255) / 256 * 256;
}

extern "C" lowra_status lowra_epilogue_backward(const uint16_t* dY_dev, const uint16_t* pre_dev, const uint16_t* multiply_dev, int32_t M, int32_t N,
                                                int32_t activation, uint16_t* dZ_dev, uint16_t* dmultiply_dev, float* dbias_dev, void* workspace_dev,
                                                size_t workspace_bytes, void* stream_v) {
    using namespace lowra;
    if (!dY_dev || (!dZ_dev && !dmultiply_dev && !dbias_dev) || (!pre_dev && (activation != LOWRA_ACT_NONE || dmultiply_dev)) || (dmultiply_dev && !multiply_dev))
        return LOWRA_ERR_NULL;
    if (M < 1 || M > kMostRows || N < 8 || N > kMostCols || N % 8 != 0 || activation < LOWRA_ACT_NONE || activation > LOWRA_ACT_SILU || (dZ_dev && dZ_dev == dmultiply_dev)) return LOWRA_ERR_SHAPE;
    if (!aligned16(dY_dev) || !aligned16(pre_dev) || !aligned16(multiply_dev) || !aligned16(dZ_dev) || !aligned16(dmultiply_dev) || !aligned16(dbias_dev))
        return LOWRA_ERR_ALIGN;
    int runs = dbias_dev ? runs_of(M, N) : 0;
    if (runs > 0 && (!workspace_dev || workspace_bytes < lowra_epilogue_workspace_bytes(M, N) || (reinterpret_cast<uintptr_t>(workspace_dev) & 255u) != 0))
        return LOWRA_ERR_WORKSPACE;
    // An output may be an input, element for element; else it shares memory with nothing.
    const size_t rows = (size_t)M * (size_t)N * 2;
    const Span read[3] = {{dY_dev, rows}, {pre_dev, rows}, {multiply_dev, rows}}, written[2] = {{dZ_dev, rows}, {dmultiply_dev, rows}}, dbias = {dbias_dev, (size_t)N * 4};
    for (const Span& w : written) {
        for (const Span& x : read)
            if (w.at != x.at && overlap(w, x)) return LOWRA_ERR_SHAPE;
        if (overlap(w, dbias)) return LOWRA_ERR_SHAPE;
    }
    for (const Span& x : read)
        if (overlap(x, dbias)) return LOWRA_ERR_SHAPE;
    if (overlap(written[0], written[1])) return LOWRA_ERR_SHAPE;
    lowra_status st = check_device();
    if (st != LOWRA_OK) return st;
    cudaStream_t stream = (cudaStream_t)stream_v;
    BackwardParams P = {dY_dev, pre_dev, multiply_dev, dZ_dev, dmultiply_dev, nullptr, M, N, activation, M};
    if (!dbias_dev) {
        const size_t ctas = ((size_t)M * (size_t)(N / 8) + kThreads - 1) / kThreads, most = (size_t)kNumSMs * kResident;
        return launch_pdl(multiply_dev ? flat_kernel<true> : flat_kernel<false>, (unsigned)(ctas < most ? ctas : most), kThreads, stream, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
    }
    P.rows = (M + runs - 1) / runs;
    runs = (M + P.rows - 1) / P.rows;
    P.sums = runs > 1 ? static_cast<float*>(workspace_dev) : dbias_dev;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    const bool narrow = takes_narrow(M, N);
    const int cols = narrow ? kNarrowCols : kCols;
    cfg.gridDim = dim3((unsigned)((N + cols - 1) / cols), (unsigned)runs, 1);
    cfg.blockDim = dim3(narrow ? kNarrowThreads : kThreads, 1, 1);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const auto gated = narrow ? rows_kernel<true, kNarrowThreads, kNarrowCols> : rows_kernel<true, kThreads, kCols>;
    const auto plain = narrow ? rows_kernel<false, kNarrowThreads, kNarrowCols> : rows_kernel<false, kThreads, kCols>;
    if (cudaLaunchKernelEx(&cfg, multiply_dev ? gated : plain, P) != cudaSuccess) return LOWRA_ERR_CUDA;
    if (runs > 1 && launch_pdl(sum_runs_kernel, (unsigned)((N + 31) / 32), kThreads, stream, (const float*)P.sums, runs, N, dbias_dev) != cudaSuccess) return LOWRA_ERR_CUDA;
    return LOWRA_OK;
}
