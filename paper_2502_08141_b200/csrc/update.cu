// lowra_update_factors: momentum and an orthogonalised update for many low-rank factors in one call.
//     m' = mu m + g;   u = g + mu m' (Nesterov) or m';   X_0 = u / (|u| + eps);   X_{k+1} = a X_k + X_k (b G_k + c G_k^2), G_k = X_k^T X_k;
//     w' = (1 - lr wd) w - lr scale X_n
// A factor is L x r (A, "tall") or r x L (B): the short side is the rank, and every product above is one of r x r matrices with u.  All of them are
// polynomials in S = u^T u (over the long side), which commute, so X_n = u Q with an r x r matrix Q: with alpha = 1 / (|u| + eps)^2, G_0 = alpha S,
//     P_k = a + b G_k + c G_k^2,   G_{k+1} = G_k P_k^2,   Q = P_0 P_1 ... / (|u| + eps),   |u|^2 = trace S.
// Three kernels: gram_kernel reads g and m, writes m', and forms parts of S; iterate_kernel adds them up and forms Q; apply_kernel forms u Q and writes
// the weights.  u is read twice whatever the number of steps (the second time mostly from L2).
// S holds the squares of u's singular values, so a value of 1e-3 |u|, which the iteration lifts to 0.5, is 1e-6 of S: in fp32 it would be off by a
// percent.  S and everything of size r x r are therefore fp64, on the fp64 tensor instructions (m8n8k4, measured 36 TFLOP/s); u and u Q are fp32.
#include <string.h>

#include "epilogue.cuh"
#include "ptx.cuh"

namespace lowra {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;     // of the two kernels that walk over u
constexpr int kTileElements = 4096;                       // of u at a time: 32 to a thread
constexpr int kQuads = kTileElements / 4 / kThreads;      // four neighbouring elements each, to a thread
constexpr int kWalkers = 2 * kNumSMs;                     // CTAs that share the tiles of all factors out, in gram_kernel
constexpr int kApplyResident = 2;                         // CTAs of apply_kernel to an SM
constexpr int kMaxFactors = LOWRA_MAX_FACTORS;

struct Factor {
    const void* grad;              // bf16 or fp32
    const float* momentum;         // null: none
    float* momentum_out;
    const float* master;           // null: none
    float* master_out;
    uint16_t* weight;
    float* update;
    int L;
    float rate;                    // lr * scale
    int tile0;                     // tiles of the factors before this one
    uint8_t tall, grad_fp32;
};
struct UpdateParams {
    double* sums;                  // [walker + factor][tiles of S][64]: the part of S that a walker has formed
    float* Q;                      // [factor][r][r]
    int count, tiles;
    float mu, decay;               // decay: 1 - lr wd
    int nesterov, steps;
    double a, b, c, eps;
    Factor f[kMaxFactors];
};

// r = 16 NB.  Blocks of 8 x 8 of S: 2 NB to a side, those on and above the diagonal are kept, row by row.
template <int NB>
struct Shape {
    static constexpr int r = 16 * NB, blocks = 2 * NB, tri = blocks * (blocks + 1) / 2;
    static constexpr int TL = kTileElements / r / 16 * 16 < 48 ? kTileElements / r / 8 * 8 : kTileElements / r / 16 * 16;    // u at a time: so many of the long side
    // shared memory of a tile of u, element (l, c) at l * sl + c * sc: without bank conflicts for the stores of four neighbours in memory and for the
    // fragments (eight c, four l)
    static constexpr int tall_pitch = r + 8, wide_pitch = (TL + 31) / 32 * 32 + 4;
    static constexpr int floats = TL * tall_pitch > r * wide_pitch ? TL * tall_pitch : r * wide_pitch;
};
__host__ __device__ constexpr int tri_index(int blocks, int i, int j) { return i * blocks - i * (i - 1) / 2 + (j - i); }

__device__ __forceinline__ void dmma(double (&c)[2], double a, double b) {
    asm("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};" : "+d"(c[0]), "+d"(c[1]) : "d"(a), "d"(b));
}

// How a tile's quads (four neighbours in memory) go to the threads: rows of them in passes, the threads of a pass side by side in memory.  A row is one of the
// long side (tall: its r values) or of the rank (wide: TL values).
template <int NB, bool TALL>
struct Deal {
    using S = Shape<NB>;
    static constexpr int per_row = (TALL ? S::r : S::TL) / 4, rows = TALL ? S::TL : S::r, at_once = kThreads / per_row, passes = rows / at_once;
    static_assert(at_once * passes == rows && passes <= kQuads, "whole passes");
    bool in;                      // this thread has quads (wide: that lie inside; the length is a multiple of 8, so a quad is in or out as a whole)
    int row, col;                 // of its first one
    size_t at;                    // in the factor's arrays
    size_t step;
    int left;                     // tall: rows of the tile inside the factor
    __device__ __forceinline__ Deal(const Factor& F, int l0) {
        row = (int)threadIdx.x / per_row;
        col = (int)threadIdx.x % per_row * 4;
        in = row < at_once && (TALL || l0 + col < F.L);
        at = TALL ? (size_t)(l0 + row) * S::r + col : (size_t)row * F.L + (l0 + col);
        step = TALL ? (size_t)(at_once * S::r) : (size_t)at_once * F.L;
        left = F.L - l0;
    }
    template <typename Body>      // body(pass, place in memory, inside)
    __device__ __forceinline__ void each(Body body) const {
        size_t p = at;
#pragma unroll
        for (int i = 0; i < passes; ++i, p += step) body(i, p, in && (!TALL || row + i * at_once < left));
    }
};

// What a thread holds of a tile: its quads of the gradient (bf16 or fp32) and of the momentum.
struct Held {
    uint4 g[kQuads];
    float4 m[kQuads];
};

__device__ __forceinline__ float4 grad_quad(const Factor& F, uint4 g) {
    if (F.grad_fp32) return make_float4(__uint_as_float(g.x), __uint_as_float(g.y), __uint_as_float(g.z), __uint_as_float(g.w));
    return make_float4(__uint_as_float(g.x << 16), __uint_as_float(g.x & 0xffff0000u), __uint_as_float(g.y << 16), __uint_as_float(g.y & 0xffff0000u));
}
__device__ __forceinline__ float4 axpy(float a, float4 x, float4 y) { return make_float4(fmaf(a, x.x, y.x), fmaf(a, x.y, y.y), fmaf(a, x.z, y.z), fmaf(a, x.w, y.w)); }

__device__ __forceinline__ float4 axpy2(float a, float4 x, float4 y) {       // two products to an instruction
    const float2 aa = make_float2(a, a), lo = fma2(aa, make_float2(x.x, x.y), make_float2(y.x, y.y)), hi = fma2(aa, make_float2(x.z, x.w), make_float2(y.z, y.w));
    return make_float4(lo.x, lo.y, hi.x, hi.y);
}
__device__ __forceinline__ float4 zero4() { return make_float4(0.0f, 0.0f, 0.0f, 0.0f); }

// The tile's gradient, and its old momentum (OLD) or the new one where u needs it.
template <int NB, bool TALL, bool OLD>
__device__ __forceinline__ void fetch(const UpdateParams& P, const Factor& F, int l0, Held& held) {
    const Deal<NB, TALL> deal(F, l0);
    const float* m = OLD ? F.momentum : F.momentum_out;
    if (OLD || m == nullptr || P.nesterov) {
        if (F.grad_fp32) deal.each([&](int i, size_t at, bool in) { held.g[i] = in ? *reinterpret_cast<const uint4*>(static_cast<const float*>(F.grad) + at) : make_uint4(0u, 0u, 0u, 0u); });
        else deal.each([&](int i, size_t at, bool in) {
            const uint2 p = in ? *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(F.grad) + at) : make_uint2(0u, 0u);
            held.g[i].x = p.x;
            held.g[i].y = p.y;
        });
    }
    if (m != nullptr) deal.each([&](int i, size_t at, bool in) { held.m[i] = in ? __ldcg(reinterpret_cast<const float4*>(m + at)) : zero4(); });
}

// The walkers' shares of the tiles; the factor of a tile.
__device__ __forceinline__ int share(const UpdateParams& P, int walker) { return (int)((long long)P.tiles * walker / gridDim.x); }
__device__ __forceinline__ int factor_of(const UpdateParams& P, int tile) {
    int lo = 0, hi = P.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (P.f[mid].tile0 <= tile) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// ------------------------------------------------------------------------------------------------ parts of S
// A walker takes neighbouring tiles; what it forms of a factor's S goes to slot walker + factor (both only ever go up, so a slot is one walker's and one
// factor's).  Up to r = 64 every warp takes a quarter of the tile's long side and all blocks of S (36 at r = 64: 144 registers); above that each warp takes
// all of it and a quarter of the blocks: the triangles of the two halves of the rank, and two halves of the square between them.
template <int NB>
__global__ void __launch_bounds__(kThreads, 2) gram_kernel(const __grid_constant__ UpdateParams P) {
    using S = Shape<NB>;
    constexpr bool kSplit = NB > 4;
    constexpr int kSide = kSplit ? NB : 2 * NB, kHalf = (NB + 1) / 2;       // blocks of a triangle's side; columns of a part of the square
    constexpr int kAcc = kSplit && NB * kHalf > kSide * (kSide + 1) / 2 ? NB * kHalf : kSide * (kSide + 1) / 2;
    extern __shared__ __align__(16) unsigned char update_smem[];
    float* tiles[2] = {reinterpret_cast<float*>(update_smem), reinterpret_cast<float*>(update_smem) + S::floats};
    double2* joined = reinterpret_cast<double2*>(update_smem);              // (after the last tile)
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int first = share(P, blockIdx.x), end = share(P, blockIdx.x + 1);
    if (first >= end) return;
    int f = factor_of(P, first);
    Held held;
    auto fetch_tile = [&](int tile, int factor) {
        const Factor& F = P.f[factor];
        const int l0 = (tile - F.tile0) * S::TL;
        if (F.tall) fetch<NB, true, true>(P, F, l0, held);
        else fetch<NB, false, true>(P, F, l0, held);
    };
    fetch_tile(first, f);
    double acc[kAcc][2];
#pragma unroll
    for (int i = 0; i < kAcc; ++i) acc[i][0] = acc[i][1] = 0.0;
    // u of the tile into shared memory, the new momentum into its own
    auto put = [&](auto tall, const Factor& F, int l0, float* u) {
        constexpr bool TALL = decltype(tall)::value;
        using D = Deal<NB, TALL>;
        constexpr int pitch = TALL ? S::tall_pitch : S::wide_pitch;
        const D deal(F, l0);
        float* to = u + deal.row * pitch + deal.col;
        const bool has = deal.row < D::at_once;
        deal.each([&](int i, size_t at, bool in) {
            const float4 grad = grad_quad(F, held.g[i]);
            float4 x = grad;
            if (F.momentum != nullptr) {
                const float4 m = axpy(P.mu, held.m[i], grad);
                if (in) *reinterpret_cast<float4*>(F.momentum_out + at) = m;
                x = P.nesterov ? axpy(P.mu, m, grad) : m;
            }
            if (has) *reinterpret_cast<float4*>(to + i * D::at_once * pitch) = x;
        });
    };
    auto multiply = [&](auto tall, const float* u) {
        constexpr bool TALL = decltype(tall)::value;
        constexpr int sl = TALL ? S::tall_pitch : 1, sc = TALL ? 1 : S::wide_pitch;
        constexpr int steps = (kSplit ? S::TL : S::TL / kWarps) / 4;
        const float* at = u + g * sc + t4 * sl + (kSplit ? 0 : warp * (S::TL / kWarps) * sl);
        if (!kSplit || warp < 2) {
            at += kSplit ? warp * (8 * NB) * sc : 0;
            float next[kSide];
#pragma unroll
            for (int i = 0; i < kSide; ++i) next[i] = at[i * 8 * sc];
#pragma unroll 1
            for (int k = 0; k < steps; ++k) {
                double x[kSide];
#pragma unroll
                for (int i = 0; i < kSide; ++i) x[i] = (double)next[i];
                if (k + 1 < steps) {
                    at += 4 * sl;
#pragma unroll
                    for (int i = 0; i < kSide; ++i) next[i] = at[i * 8 * sc];
                }
                int n = 0;
#pragma unroll
                for (int i = 0; i < kSide; ++i) {
#pragma unroll
                    for (int j = i; j < kSide; ++j) dmma(acc[n++], x[i], x[j]);
                }
            }
        } else {
            const int j0 = (warp - 2) * kHalf;
            const float* bt = at + (NB + j0) * 8 * sc;
#pragma unroll 1
            for (int k = 0; k < steps; ++k, at += 4 * sl, bt += 4 * sl) {
                double x[NB], y[kHalf];
#pragma unroll
                for (int i = 0; i < NB; ++i) x[i] = (double)at[i * 8 * sc];
#pragma unroll
                for (int j = 0; j < kHalf; ++j) y[j] = j0 + j < NB ? (double)bt[j * 8 * sc] : 0.0;
#pragma unroll
                for (int i = 0; i < NB; ++i) {
#pragma unroll
                    for (int j = 0; j < kHalf; ++j) dmma(acc[i * kHalf + j], x[i], y[j]);
                }
            }
        }
    };
    for (int tile = first; tile < end; ++tile) {
        const Factor& F = P.f[f];
        const int l0 = (tile - F.tile0) * S::TL;
        const bool last_of_factor = l0 + S::TL >= F.L;
        float* u = tiles[(tile - first) & 1];
        if (F.tall) put(std::true_type(), F, l0, u);
        else put(std::false_type(), F, l0, u);
        if (tile + 1 < end) fetch_tile(tile + 1, last_of_factor ? f + 1 : f);
        __syncthreads();                                                     // the tile is there (and the one before it has been read)
        if (F.tall) multiply(std::true_type(), u);
        else multiply(std::false_type(), u);
        if (tile + 1 < end && !last_of_factor) continue;
        double2* out = reinterpret_cast<double2*>(P.sums) + (size_t)(blockIdx.x + f) * S::tri * 32;
        if (kSplit) {
            if (warp < 2) {
                int n = 0;
#pragma unroll
                for (int i = 0; i < kSide; ++i) {
#pragma unroll
                    for (int j = i; j < kSide; ++j, ++n) out[tri_index(S::blocks, warp * NB + i, warp * NB + j) * 32 + lane] = make_double2(acc[n][0], acc[n][1]);
                }
            } else {
                const int j0 = (warp - 2) * kHalf;
#pragma unroll
                for (int i = 0; i < NB; ++i) {
#pragma unroll
                    for (int j = 0; j < kHalf; ++j)
                        if (j0 + j < NB) out[tri_index(S::blocks, i, NB + j0 + j) * 32 + lane] = make_double2(acc[i * kHalf + j][0], acc[i * kHalf + j][1]);
                }
            }
        } else {
            // the warps' sums, through shared memory, in the warps' order
            __syncthreads();
#pragma unroll
            for (int n = 0; n < S::tri; ++n) joined[(n * kWarps + warp) * 32 + lane] = make_double2(acc[n][0], acc[n][1]);
            __syncthreads();
            for (int n = warp; n < S::tri; n += kWarps) {
                double2 v = joined[n * kWarps * 32 + lane];
#pragma unroll
                for (int w = 1; w < kWarps; ++w) {
                    const double2 x = joined[(n * kWarps + w) * 32 + lane];
                    v.x += x.x;
                    v.y += x.y;
                }
                out[n * 32 + lane] = v;
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kAcc; ++i) acc[i][0] = acc[i][1] = 0.0;
        ++f;
    }
}

// ------------------------------------------------------------------------------------------------ the iteration on r x r matrices
// A cluster takes a factor, a warp one block of the upper triangle of every product, which it writes into the shared memory of all CTAs.  Blocks below the
// diagonal are read as the transposes of those above it: the products of commuting symmetric matrices are symmetric.
// A block is 8 x 8 doubles, row by row, the halves of rows 2, 3, 6 and 7 changed over (both ways of reading fragments are then without bank conflicts).
__device__ __forceinline__ int in_block(int row, int col) { return row * 8 + (col ^ ((row & 2) << 1)); }
__device__ __forceinline__ void st_cluster_f64x2(uint32_t at, double x, double y) {
    asm volatile("st.shared::cluster.v2.f64 [%0], {%1, %2};" ::"r"(at), "d"(x), "d"(y) : "memory");
}
__device__ __forceinline__ void st_cluster_f64(uint32_t at, double x) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(x) : "memory"); }

template <int NB>
__global__ void __launch_bounds__(1024) iterate_kernel(const __grid_constant__ UpdateParams P, const int ctas) {
    using S = Shape<NB>;
    constexpr int B = S::blocks;
    constexpr bool kThree = 4 * S::tri * 512 > 220 * 1024;       // the product that follows G takes G's place (one barrier more a step)
    extern __shared__ __align__(16) unsigned char update_smem[];
    double* G = reinterpret_cast<double*>(update_smem);
    double* Pk = G + S::tri * 64;
    double* Q = Pk + S::tri * 64;
    double* M = kThree ? G : Q + S::tri * 64;
    double* trace = Q + (kThree ? 1 : 2) * S::tri * 64;          // [B], of the diagonal blocks
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (behind the wait: apply_kernel reads what gram_kernel wrote before its own)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int f = (int)blockIdx.x / ctas, rank = (int)blockIdx.x % ctas;
    const Factor& F = P.f[f];
    const int block = rank * (int)(blockDim.x >> 5) + warp;
    const bool mine = block < S::tri;
    int bi = 0;
    while (mine && tri_index(B, bi + 1, bi + 1) <= block) ++bi;
    const int bj = mine ? bi + block - tri_index(B, bi, bi) : 0;
    const int own = block * 64 + in_block(g, 2 * t4);            // this lane's two values of its block
    auto store = [&](double* X, const double (&v)[2]) {
        const uint32_t at = ptx::smem_u32(X + own);
        for (int i = 0; i < ctas; ++i) st_cluster_f64x2(ptx::map_to_cta(at, (uint32_t)i), v[0], v[1]);
    };
    // Blocks (bi, k) of X times blocks (k, bj) of Y, for one or two X.  Those left of the diagonal in X's row and below it in Y's column are read as transposes:
    // three ranges of k, in each of which the places of the blocks follow by simple steps.
    const int straight = in_block(g, t4), across = in_block(t4, g), straight4 = in_block(g, 4 + t4) - straight;      // (across: 32 further)
    auto products = [&](auto two, const double* X, const double* X2, const double* Y, double (&v)[2], double (&v2)[2]) {
        constexpr bool TWO = decltype(two)::value;
        double odd[2] = {0.0, 0.0}, odd2[2] = {0.0, 0.0};
        v[0] = v[1] = 0.0;
        if (TWO) v2[0] = v2[1] = 0.0;
        int xo = bi * 64, yo = bj * 64;                          // block (0, bi), block (0, bj)
        auto step = [&](int xl, int x4, int yl, int y4) {
            const double y0 = Y[yo + yl], y1 = Y[yo + yl + y4];
            dmma(v, X[xo + xl], y0);
            dmma(odd, X[xo + xl + x4], y1);
            if (TWO) {
                dmma(v2, X2[xo + xl], y0);
                dmma(odd2, X2[xo + xl + x4], y1);
            }
        };
        int k = 0;
#pragma unroll 2
        for (; k < bi; ++k) {
            step(across, 32, across, 32);
            xo += (B - 1 - k) * 64;
            yo += (B - 1 - k) * 64;
        }
#pragma unroll 2
        for (; k <= bj; ++k) {
            step(straight, straight4, across, 32);
            xo += 64;
            yo += (k < bj ? B - 1 - k : 1) * 64;                 // (the block behind (bj, bj) is (bj, bj + 1))
        }
#pragma unroll 2
        for (; k < B; ++k) {
            step(straight, straight4, straight, straight4);
            xo += 64;
            yo += 64;
        }
        v[0] += odd[0];
        v[1] += odd[1];
        if (TWO) {
            v2[0] += odd2[0];
            v2[1] += odd2[1];
        }
    };
    double unused[2];
    auto product = [&](const double* X, const double* Y, double (&v)[2]) { products(std::false_type(), X, X, Y, v, unused); };
    ptx::cluster_sync();                                          // (every CTA of the cluster runs: its shared memory may be written)
    // ---- S, from its parts in the walkers' order
    if (mine) {
        const int walkers = (int)min(kWalkers, P.tiles), tiles = (F.L + S::TL - 1) / S::TL;
        auto walker_of = [&](int tile) {                          // the one whose share holds the tile
            int w = (int)((long long)tile * walkers / P.tiles);
            while ((int)((long long)P.tiles * (w + 1) / walkers) <= tile) ++w;
            while ((int)((long long)P.tiles * w / walkers) > tile) --w;
            return w;
        };
        const int w0 = walker_of(F.tile0), w1 = walker_of(F.tile0 + tiles - 1);
        const double2* from = reinterpret_cast<const double2*>(P.sums) + (size_t)block * 32 + lane;
        double v[2] = {0.0, 0.0};
#pragma unroll 8
        for (int w = w0; w <= w1; ++w) {
            const double2 x = __ldcg(from + (size_t)(w + f) * S::tri * 32);
            v[0] += x.x;
            v[1] += x.y;
        }
        if (bi == bj) {
            double d = g == 2 * t4 ? v[0] : g == 2 * t4 + 1 ? v[1] : 0.0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
            if (lane < ctas) st_cluster_f64(ptx::map_to_cta(ptx::smem_u32(trace + bi), (uint32_t)lane), d);
        }
        store(G, v);
    }
    ptx::cluster_sync();
    double norm = 0.0;
    for (int i = 0; i < B; ++i) norm += trace[i];
    norm = sqrt(norm) + P.eps;
    double alpha = 1.0 / (norm * norm);                           // (G_0 is alpha times what G holds; the later ones are held as they are)
    double q[2] = {0.0, 0.0};
    for (int step = 0; step < P.steps; ++step) {
        double v[2], p[2] = {0.0, 0.0};
        if (mine) {
            product(G, G, v);
#pragma unroll
            for (int i = 0; i < 2; ++i) p[i] = (bi == bj && g == 2 * t4 + i ? P.a : 0.0) + P.b * (alpha * G[own + i]) + P.c * (alpha * alpha * v[i]);
            store(Pk, p);
        }
        ptx::cluster_sync();
        const bool more = step + 1 < P.steps;
        if (mine) {
            if (step == 0) {
                q[0] = p[0];
                q[1] = p[1];
                if (more) product(G, Pk, v);
            } else if (more) {
                products(std::true_type(), G, Q, Pk, v, q);
            } else {
                product(Q, Pk, q);
            }
            v[0] *= alpha;
            v[1] *= alpha;
        }
        if (!more) break;
        if (kThree) ptx::cluster_sync();                          // everybody has read G
        if (mine) store(M, v);
        ptx::cluster_sync();
        if (mine) {
            product(M, Pk, v);
            store(Q, q);                                          // (read by all before the barrier)
        }
        if (kThree) ptx::cluster_sync();                          // everybody has read M
        if (mine) store(G, v);
        ptx::cluster_sync();
        alpha = 1.0;
    }
    if (mine) {
        float* out = P.Q + (size_t)f * S::r * S::r;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = bi * 8 + g, col = bj * 8 + 2 * t4 + i;
            const float v = (float)(q[i] / norm);
            out[row * S::r + col] = v;
            if (bi != bj) out[col * S::r + row] = v;
        }
    }
}

// ------------------------------------------------------------------------------------------------ u Q, and the weights
// A thread forms eight of the long side times four ranks, from the tile of u and Q in shared memory, fp32.  What the tile after this one needs of the gradient
// and the momentum, and this one's master weights, are under way meanwhile.
template <int NB>
__global__ void __launch_bounds__(kThreads, kApplyResident) apply_kernel(const __grid_constant__ UpdateParams P) {
    using S = Shape<NB>;
    constexpr int kPitch = S::r + 4;                              // u, tall: [l][c]
    extern __shared__ __align__(16) unsigned char update_smem[];
    float* Q = reinterpret_cast<float*>(update_smem);             // [r][r]
    float* u = Q + S::r * S::r;                                   // tall: [TL][kPitch]; wide: [r][TL]
    const int first = share(P, blockIdx.x), end = share(P, blockIdx.x + 1);
    if (first >= end) return;
    int f = factor_of(P, first), loaded = -1;
    Held held;
    auto fetch_tile = [&](int tile, int factor) {
        const Factor& F = P.f[factor];
        const int l0 = (tile - F.tile0) * S::TL;
        if (F.tall) fetch<NB, true, false>(P, F, l0, held);
        else fetch<NB, false, false>(P, F, l0, held);
    };
    auto put = [&](auto tall, const Factor& F, int l0) {
        constexpr bool TALL = decltype(tall)::value;
        using D = Deal<NB, TALL>;
        constexpr int pitch = TALL ? kPitch : S::TL;
        const D deal(F, l0);
        float* to = u + deal.row * pitch + deal.col;
        if (deal.row >= D::at_once) return;
        deal.each([&](int i, size_t, bool) {
            float4 x = F.momentum != nullptr ? held.m[i] : grad_quad(F, held.g[i]);
            if (F.momentum != nullptr && P.nesterov) x = axpy(P.mu, x, grad_quad(F, held.g[i]));
            *reinterpret_cast<float4*>(to + i * D::at_once * pitch) = x;
        });
    };
    // thread's outputs, quads of four neighbours in memory: number i of eight at place + (i / 4) * far + (i % 4) * near
    auto work = [&](auto tall, const Factor& F, int l0, auto next) {
        constexpr bool TALL = decltype(tall)::value;
        constexpr int groups = S::TL / 8;
        // tall: ranks c .. c + 3, rows lg, lg + TL / 8, ...: a warp's lanes lie side by side along the rank
        // wide: ranks c .. c + 3, and two runs of four of the long side: the lanes lie side by side along it
        const int cg = TALL ? (int)threadIdx.x % (S::r / 4) : (int)threadIdx.x / groups, lg = TALL ? (int)threadIdx.x / (S::r / 4) : (int)threadIdx.x % groups;
        const bool has = TALL ? lg < groups : cg < S::r / 4;
        const size_t place = TALL ? (size_t)(l0 + lg) * S::r + cg * 4 : (size_t)(cg * 4) * F.L + (l0 + lg * 4);
        const size_t near_by = TALL ? (size_t)(groups * S::r) : (size_t)F.L, far = TALL ? 4 * near_by : (size_t)(S::TL / 2);
        auto inside = [&](int i) { return has && (TALL ? l0 + lg + i * groups < F.L : l0 + lg * 4 + (i / 4) * (S::TL / 2) < F.L); };
        float4 w[8];
        if (F.master != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = inside(i) ? *reinterpret_cast<const float4*>(F.master + place + (i / 4) * far + (i % 4) * near_by) : zero4();
        }
        next();
        float4 acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = zero4();
        if (has) {
            if (TALL) {
                const float *x_at = u + lg * kPitch, *q_at = Q + cg * 4;
#pragma unroll 1
                for (int j = 0; j < S::r; j += 4, x_at += 4, q_at += 4 * S::r) {
                    float4 q[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) q[k] = *reinterpret_cast<const float4*>(q_at + k * S::r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float4 x = *reinterpret_cast<const float4*>(x_at + i * groups * kPitch);
                        acc[i] = axpy2(x.x, q[0], acc[i]);
                        acc[i] = axpy2(x.y, q[1], acc[i]);
                        acc[i] = axpy2(x.z, q[2], acc[i]);
                        acc[i] = axpy2(x.w, q[3], acc[i]);
                    }
                }
            } else {
                const float *x_at = u + lg * 4, *q_at = Q + cg * 4;
#pragma unroll 4
                for (int j = 0; j < S::r; ++j, x_at += S::TL, q_at += S::r) {
                    const float4 q = *reinterpret_cast<const float4*>(q_at);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 x = *reinterpret_cast<const float4*>(x_at + h * (S::TL / 2));
                        acc[4 * h] = axpy2(q.x, x, acc[4 * h]);
                        acc[4 * h + 1] = axpy2(q.y, x, acc[4 * h + 1]);
                        acc[4 * h + 2] = axpy2(q.z, x, acc[4 * h + 2]);
                        acc[4 * h + 3] = axpy2(q.w, x, acc[4 * h + 3]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!inside(i)) continue;
            const size_t at = place + (i / 4) * far + (i % 4) * near_by;
            if (F.update != nullptr) *reinterpret_cast<float4*>(F.update + at) = acc[i];
            if (F.master != nullptr) {
                const float4 n = make_float4(fmaf(-F.rate, acc[i].x, P.decay * w[i].x), fmaf(-F.rate, acc[i].y, P.decay * w[i].y),
                                             fmaf(-F.rate, acc[i].z, P.decay * w[i].z), fmaf(-F.rate, acc[i].w, P.decay * w[i].w));
                *reinterpret_cast<float4*>(F.master_out + at) = n;
                if (F.weight != nullptr) *reinterpret_cast<uint2*>(F.weight + at) = make_uint2(pack_bf16x2(n.x, n.y), pack_bf16x2(n.z, n.w));
            }
        }
    };
    // (iterate_kernel lets this kernel start when gram_kernel is through: u may be read before the wait for Q)
    fetch_tile(first, f);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int tile = first; tile < end; ++tile) {
        const Factor& F = P.f[f];
        const int l0 = (tile - F.tile0) * S::TL;
        const bool last_of_factor = l0 + S::TL >= F.L;
        if (F.tall) put(std::true_type(), F, l0);
        else put(std::false_type(), F, l0);
        if (loaded != f) {
            if (loaded < 0) asm volatile("griddepcontrol.wait;" ::: "memory");
            for (int i = threadIdx.x; i < S::r * S::r / 4; i += kThreads)
                reinterpret_cast<float4*>(Q)[i] = __ldcg(reinterpret_cast<const float4*>(P.Q + (size_t)f * S::r * S::r) + i);
            loaded = f;
        }
        __syncthreads();
        auto next = [&]() {
            if (tile + 1 < end) fetch_tile(tile + 1, last_of_factor ? f + 1 : f);
        };
        if (F.tall) work(std::true_type(), F, l0, next);
        else work(std::false_type(), F, l0, next);
        __syncthreads();                                          // u and Q have been read
        if (last_of_factor) ++f;
    }
}

// ------------------------------------------------------------------------------------------------ host
template <int NB>
int tiles_of(int L) { return (L + Shape<NB>::TL - 1) / Shape<NB>::TL; }

template <int NB>
size_t sums_bytes(int tiles, int count) { return (size_t)((tiles < kWalkers ? tiles : kWalkers) + count) * Shape<NB>::tri * 512; }

// CTAs of a factor's cluster in iterate_kernel
int iterate_ctas(int tri) { return tri <= 10 ? 1 : tri <= 21 ? 2 : tri <= 55 ? 4 : 8; }

template <int NB>
lowra_status launch_update(UpdateParams& P, void* workspace, cudaStream_t stream) {
    using S = Shape<NB>;
    P.tiles = 0;
    for (int i = 0; i < P.count; ++i) {
        P.f[i].tile0 = P.tiles;
        P.tiles += tiles_of<NB>(P.f[i].L);
    }
    P.sums = static_cast<double*>(workspace);
    P.Q = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + sums_bytes<NB>(P.tiles, P.count));
    const unsigned walkers = (unsigned)(P.tiles < kWalkers ? P.tiles : kWalkers);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(walkers, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    {
        static SmemLimit limit = {};
        const size_t tiles = 2 * S::floats * 4, joined = NB > 4 ? 0 : (size_t)S::tri * 512 * kWarps;
        cfg.dynamicSmemBytes = tiles > joined ? tiles : joined;
        if (ensure_smem_limit(reinterpret_cast<const void*>(gram_kernel<NB>), cfg.dynamicSmemBytes, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
        if (cudaLaunchKernelEx(&cfg, gram_kernel<NB>, P) != cudaSuccess) return LOWRA_ERR_CUDA;
    }
    {
        static SmemLimit limit = {};
        const int ctas = iterate_ctas(S::tri);
        constexpr bool three = 4 * S::tri * 512 > 220 * 1024;
        cfg.dynamicSmemBytes = (size_t)(three ? 3 : 4) * S::tri * 512 + S::blocks * 8;
        cfg.gridDim = dim3((unsigned)(P.count * ctas), 1, 1);
        cfg.blockDim = dim3(32u * (unsigned)((S::tri + ctas - 1) / ctas), 1, 1);
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)ctas;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
        if (ensure_smem_limit(reinterpret_cast<const void*>(iterate_kernel<NB>), cfg.dynamicSmemBytes, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
        if (cudaLaunchKernelEx(&cfg, iterate_kernel<NB>, P, ctas) != cudaSuccess) return LOWRA_ERR_CUDA;
        cfg.numAttrs = 1;
    }
    static SmemLimit limit = {};
    const size_t tall = (size_t)S::TL * (S::r + 4), wide = (size_t)S::TL * S::r;
    cfg.dynamicSmemBytes = ((size_t)S::r * S::r + (tall > wide ? tall : wide)) * 4;
    cfg.gridDim = dim3((unsigned)(P.tiles < kApplyResident * kNumSMs ? P.tiles : kApplyResident * kNumSMs), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    if (ensure_smem_limit(reinterpret_cast<const void*>(apply_kernel<NB>), cfg.dynamicSmemBytes, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
    return cudaLaunchKernelEx(&cfg, apply_kernel<NB>, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}

template <int NB>
size_t workspace_bytes_of(const lowra_factor* m, int count) {
    long long tiles = 0;
    for (int i = 0; i < count; ++i) tiles += tiles_of<NB>(m[i].rows == Shape<NB>::r ? m[i].cols : m[i].rows);
    const int walkers = tiles < kWalkers ? (int)tiles : kWalkers;
    return (sums_bytes<NB>(walkers, count) + (size_t)count * Shape<NB>::r * Shape<NB>::r * 4 + 255) / 256 * 256;
}

// Shapes and number of the factors.
lowra_status check_shapes(const lowra_factor* m, int32_t count, int32_t r) {
    if (!m) return LOWRA_ERR_NULL;
    if (count < 1 || count > kMaxFactors || r < 16 || r > 128 || r % 16 != 0) return LOWRA_ERR_SHAPE;
    long long elements = 0;
    for (int i = 0; i < count; ++i) {
        if (m[i].rows != r && m[i].cols != r) return LOWRA_ERR_SHAPE;
        const int32_t L = m[i].rows == r ? m[i].cols : m[i].rows;
        if (L < 8 || L % 8 != 0) return LOWRA_ERR_SHAPE;
        elements += (long long)L * r;
    }
    return elements < (1ll << 40) ? LOWRA_OK : LOWRA_ERR_SHAPE;
}

}  // namespace
}  // namespace lowra

extern "C" size_t lowra_update_workspace_bytes(const lowra_factor* members_host, int32_t count, int32_t r) {
    using namespace lowra;
    if (check_shapes(members_host, count, r) != LOWRA_OK) return 0;
    switch (r / 16) {
        case 1: return workspace_bytes_of<1>(members_host, count);
        case 2: return workspace_bytes_of<2>(members_host, count);
        case 3: return workspace_bytes_of<3>(members_host, count);
        case 4: return workspace_bytes_of<4>(members_host, count);
        case 5: return workspace_bytes_of<5>(members_host, count);
        case 6: return workspace_bytes_of<6>(members_host, count);
        case 7: return workspace_bytes_of<7>(members_host, count);
        default: return workspace_bytes_of<8>(members_host, count);
    }
}

extern "C" lowra_status lowra_update_factors(const lowra_factor* members_host, int32_t count, int32_t r, const lowra_update_step* step_host,
                                             void* workspace_dev, size_t workspace_bytes, void* stream_v) {
    using namespace lowra;
    lowra_status st = check_shapes(members_host, count, r);
    if (st != LOWRA_OK) return st;
    if (!step_host || !workspace_dev) return LOWRA_ERR_NULL;
    if (step_host->steps < 1 || step_host->steps > 32) return LOWRA_ERR_SHAPE;
    UpdateParams P;
    memset(&P, 0, sizeof(P));
    P.count = count;
    P.mu = (float)step_host->momentum;
    P.decay = (float)(1.0 - step_host->lr * step_host->weight_decay);
    P.nesterov = step_host->nesterov != 0;
    P.steps = step_host->steps;
    P.a = step_host->coefficients[0];
    P.b = step_host->coefficients[1];
    P.c = step_host->coefficients[2];
    P.eps = step_host->eps;
    for (int i = 0; i < count; ++i) {
        const lowra_factor& m = members_host[i];
        if (!m.grad_dev || (m.momentum_dev == nullptr) != (m.momentum_out_dev == nullptr) || (m.master_dev == nullptr) != (m.master_out_dev == nullptr) ||
            (m.weight_dev && !m.master_dev) || (!m.master_dev && !m.update_dev))
            return LOWRA_ERR_NULL;
        if (!aligned16(m.grad_dev) || !aligned16(m.momentum_dev) || !aligned16(m.momentum_out_dev) || !aligned16(m.master_dev) || !aligned16(m.master_out_dev) ||
            !aligned16(m.weight_dev) || !aligned16(m.update_dev))
            return LOWRA_ERR_ALIGN;
        const bool tall = m.rows != r;
        P.f[i] = Factor{m.grad_dev, m.momentum_dev, m.momentum_out_dev, m.master_dev, m.master_out_dev, m.weight_dev, m.update_dev, tall ? m.rows : m.cols,
                        (float)(step_host->lr * m.scale), 0, (uint8_t)tall, (uint8_t)(m.grad_fp32 != 0)};
    }
    if (workspace_bytes < lowra_update_workspace_bytes(members_host, count, r) || (reinterpret_cast<uintptr_t>(workspace_dev) & 255u) != 0) return LOWRA_ERR_WORKSPACE;
    if ((st = check_device()) != LOWRA_OK) return st;
    cudaStream_t stream = (cudaStream_t)stream_v;
    switch (r / 16) {
        case 1: return launch_update<1>(P, workspace_dev, stream);
        case 2: return launch_update<2>(P, workspace_dev, stream);
        case 3: return launch_update<3>(P, workspace_dev, stream);
        case 4: return launch_update<4>(P, workspace_dev, stream);
        case 5: return launch_update<5>(P, workspace_dev, stream);
        case 6: return launch_update<6>(P, workspace_dev, stream);
        case 7: return launch_update<7>(P, workspace_dev, stream);
        default: return launch_update<8>(P, workspace_dev, stream);
    }
}
