// lowra_update_factors: momentum and an orthogonalised update for many low-rank factors in one call.
//     m' = mu m + g;   u = g + mu m' (Nesterov) or m';   X_0 = u / (|u| + eps);   X_{k+1} = a X_k + X_k (b G_k + c G_k^2), G_k = X_k^T X_k;
//     w' = (1 - lr wd) w - lr scale X_n
// A factor is L x r (A, "tall") or r x L (B): the short side is the rank, and every product above is one of r x r matrices with u.  All of them are
// polynomials in S = u^T u (over the long side), which commute, so X_n = u Q with an r x r matrix Q: with alpha = 1 / (|u| + eps)^2, G_0 = alpha S,
//     P_k = a + b G_k + c G_k^2,   G_{k+1} = G_k P_k^2,   Q = P_0 P_1 ... / (|u| + eps),   |u|^2 = trace S.
// One kernel for a few short factors of small rank (one_kernel); else three: gram_kernel reads g and m, writes m', and forms parts of S; iterate_kernel adds them up and forms Q; apply_kernel forms u Q and writes
// the weights.  u is read twice whatever the number of steps (the second time mostly from L2).
// S holds the squares of u's singular values, so a value of 1e-3 |u|, which the iteration lifts to 0.5, is 1e-6 of S: in fp32 it would be off by a
// percent.  S and everything of size r x r are therefore fp64, on the fp64 tensor instructions (m8n8k4; 24 TFLOP/s in gram_kernel); u and u Q are fp32.
#include <string.h>

#include <algorithm>

#include "epilogue.cuh"
#include "ptx.cuh"

namespace lowra {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;     // that share a tile of u
constexpr int kTileElements = 4096;                       // of u at a time: 32 to a thread
constexpr int kQuads = kTileElements / 4 / kThreads;      // four neighbouring elements each, to a thread
constexpr int kWalkers = kNumSMs;                         // CTAs that share the tiles of all factors out, in gram_kernel
constexpr int kStages = 4, kFillers = 2;                  // tiles in its shared memory; groups of kThreads that fill them
constexpr int kGramThreads = (1 + kFillers) * kThreads;
constexpr int kMaxFactors = LOWRA_MAX_FACTORS, kLongest = 1 << 24;

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

// The most rows up to `most` that `rows` is a multiple of.
__host__ __device__ constexpr int whole_rows(int rows, int most) { return rows % most == 0 ? most : whole_rows(rows, most - 1); }

// How a tile's quads (four neighbours in memory) go to the threads: rows of them in passes, the threads of a pass side by side in memory.  A row is one of the
// long side (tall: its r values) or of the rank (wide: TL values).
template <int NB, bool TALL>
struct Deal {
    using S = Shape<NB>;
    static constexpr int per_row = (TALL ? S::r : S::TL) / 4, rows = TALL ? S::TL : S::r, at_once = whole_rows(rows, kThreads / per_row), passes = rows / at_once;
    static_assert(at_once * passes == rows && passes <= kQuads, "whole passes");
    bool in;                      // this thread has quads (wide: that lie inside; the length is a multiple of 8, so a quad is in or out as a whole)
    int row, col;                 // of its first one
    size_t at;                    // in the factor's arrays
    size_t step;
    int left;                     // tall: rows of the tile inside the factor
    __device__ __forceinline__ Deal(const Factor& F, int l0, int thread) {      // (of kThreads: several groups of them may take a tile each)
        row = thread / per_row;
        col = thread % per_row * 4;
        in = row < at_once && (TALL || l0 + col < F.L);
        at = TALL ? (size_t)(l0 + row) * S::r + col : (size_t)row * F.L + (l0 + col);
        step = TALL ? (size_t)(at_once * S::r) : (size_t)at_once * F.L;
        left = F.L - l0;
    }
    template <int FROM = 0, int N = kQuads, typename Body>      // body(pass, place in memory, inside), for passes FROM .. FROM + N - 1
    __device__ __forceinline__ void each(Body body) const {
        size_t p = at + FROM * step;
#pragma unroll
        for (int i = FROM; i < FROM + N && i < passes; ++i, p += step) body(i, p, in && (!TALL || row + i * at_once < left));
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
__device__ __forceinline__ float4 axpy2(float a, float4 x, float4 y) {       // two products to an instruction
    const float2 aa = make_float2(a, a), lo = fma2(aa, make_float2(x.x, x.y), make_float2(y.x, y.y)), hi = fma2(aa, make_float2(x.z, x.w), make_float2(y.z, y.w));
    return make_float4(lo.x, lo.y, hi.x, hi.y);
}
__device__ __forceinline__ float4 zero4() { return make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
// Four neighbours' weights: x of the update, w before it.
__device__ __forceinline__ void step_weights(const UpdateParams& P, const Factor& F, size_t at, float4 x, float4 w) {
    const float4 n = make_float4(fmaf(-F.rate, x.x, P.decay * w.x), fmaf(-F.rate, x.y, P.decay * w.y), fmaf(-F.rate, x.z, P.decay * w.z), fmaf(-F.rate, x.w, P.decay * w.w));
    *reinterpret_cast<float4*>(F.master_out + at) = n;
    if (F.weight != nullptr) *reinterpret_cast<uint2*>(F.weight + at) = make_uint2(pack_bf16x2(n.x, n.y), pack_bf16x2(n.z, n.w));
}

// A tile's gradient and momentum.
template <typename D>
__device__ __forceinline__ void fetch(const Factor& F, const D& deal, Held& held) {
    if (F.grad_fp32) deal.each([&](int i, size_t at, bool in) { held.g[i] = in ? *reinterpret_cast<const uint4*>(static_cast<const float*>(F.grad) + at) : make_uint4(0u, 0u, 0u, 0u); });
    else deal.each([&](int i, size_t at, bool in) {
        const uint2 p = in ? *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(F.grad) + at) : make_uint2(0u, 0u);
        held.g[i].x = p.x;
        held.g[i].y = p.y;
    });
    if (F.momentum != nullptr) deal.each([&](int i, size_t at, bool in) { held.m[i] = in ? *reinterpret_cast<const float4*>(F.momentum + at) : zero4(); });
}

// The thread's number, as if it were another one every time: what follows from it is then worked out where it is needed.  (Kept from tile to tile, the places of
// both orientations' quads and outputs took 400 bytes of local memory a thread, more traffic than u.)
__device__ __forceinline__ int thread_here() {
    int t;
    asm volatile("mov.u32 %0, %%tid.x;" : "=r"(t));
    return t;
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
// A walker (one CTA to an SM) takes neighbouring tiles; what it forms of a factor's S goes to slot walker + factor (both only ever go up, so a slot is one
// walker's and one factor's).  Two groups of four warps take the tiles in turn: gradient and momentum into registers, the new momentum to memory, u to shared
// memory.  The four warps of a third group feed the tensor instructions, which is what bounds it: of the 22 us for a layer's fourteen factors of rank 64, 17 remain without the
// filling, and 18 without the products.  (All warps doing both in turn, two CTAs to an SM: 26 us.  m16n8k4 on pairs of blocks, which runs at twice the rate in isolation but has
// a tenth more to do: the same.  Three groups that fill: the same.)
// Up to r = 64 every warp takes a quarter of the tile's long side and all blocks of S (36 at r = 64: 144 registers); above that each warp takes
// all of it and a quarter of the blocks: the triangles of the two halves of the rank, and two halves of the square between them.
constexpr int kFull = 1, kEmpty = kFull + kStages, kJoin = kEmpty + kStages;       // named barriers

template <int NB>
struct GramMemory {
    static constexpr size_t tiles = (size_t)kStages * Shape<NB>::floats * 4, joined = NB > 4 ? 0 : (size_t)Shape<NB>::tri * 512 * kWarps, bytes = tiles + joined;
};

template <int NB>
__global__ void __launch_bounds__(kGramThreads, 1) gram_kernel(const __grid_constant__ UpdateParams P) {
    using S = Shape<NB>;
    constexpr bool kSplit = NB > 4;
    constexpr int kSide = kSplit ? NB : 2 * NB, kHalf = (NB + 1) / 2;       // blocks of a triangle's side; columns of a part of the square
    constexpr int kAcc = kSplit && NB * kHalf > kSide * (kSide + 1) / 2 ? NB * kHalf : kSide * (kSide + 1) / 2;
    extern __shared__ __align__(16) unsigned char update_smem[];
    float* tiles = reinterpret_cast<float*>(update_smem);
    pdl_enter();
    const int group = (int)threadIdx.x / kThreads;
    const int first = share(P, blockIdx.x), count = share(P, blockIdx.x + 1) - first;
    int f = factor_of(P, first);
    if (group > 0) {
        // ================================================================== fillers: tiles group - 1, group - 1 + kFillers, ...
        asm volatile("setmaxnreg.dec.sync.aligned.u32 136;");
        Held held;
        for (int n = group - 1; n < count; n += kFillers) {
            while (f + 1 < P.count && P.f[f + 1].tile0 <= first + n) ++f;
            const Factor& F = P.f[f];
            const int l0 = (first + n - F.tile0) * S::TL, stage = n % kStages;
            float* u = tiles + stage * S::floats;
            auto fill = [&](auto tall) {
                constexpr bool TALL = decltype(tall)::value;
                using D = Deal<NB, TALL>;
                constexpr int pitch = TALL ? S::tall_pitch : S::wide_pitch;
                const D deal(F, l0, thread_here() % kThreads);
                fetch(F, deal, held);
                float* to = u + deal.row * pitch + deal.col;
                const bool has = deal.row < D::at_once;
                if (n >= kStages) ptx::named_barrier_sync(kEmpty + stage, 2 * kThreads);      // the tile there before has been read
                deal.each([&](int i, size_t at, bool in) {
                    const float4 grad = grad_quad(F, held.g[i]);
                    float4 x = grad;
                    if (F.momentum != nullptr) {
                        const float4 m = axpy2(P.mu, held.m[i], grad);
                        if (in) *reinterpret_cast<float4*>(F.momentum_out + at) = m;
                        x = P.nesterov ? axpy2(P.mu, m, grad) : m;
                    }
                    if (has) *reinterpret_cast<float4*>(to + i * D::at_once * pitch) = x;
                });
            };
            if (F.tall) fill(std::true_type());
            else fill(std::false_type());
            ptx::named_barrier_arrive(kFull + stage, 2 * kThreads);
        }
        return;
    }
    // ====================================================================== the products
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    double2* joined = reinterpret_cast<double2*>(update_smem + GramMemory<NB>::tiles);
    double acc[kAcc][2];
#pragma unroll
    for (int i = 0; i < kAcc; ++i) acc[i][0] = acc[i][1] = 0.0;
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
            float nx[NB], ny[kHalf];
            auto ask = [&]() {
#pragma unroll
                for (int i = 0; i < NB; ++i) nx[i] = at[i * 8 * sc];
#pragma unroll
                for (int j = 0; j < kHalf; ++j) ny[j] = j0 + j < NB ? bt[j * 8 * sc] : 0.0f;
            };
            ask();
#pragma unroll 1
            for (int k = 0; k < steps; ++k) {
                double x[NB], y[kHalf];
#pragma unroll
                for (int i = 0; i < NB; ++i) x[i] = (double)nx[i];
#pragma unroll
                for (int j = 0; j < kHalf; ++j) y[j] = (double)ny[j];
                at += 4 * sl;
                bt += 4 * sl;
                if (k + 1 < steps) ask();
#pragma unroll
                for (int i = 0; i < NB; ++i) {
#pragma unroll
                    for (int j = 0; j < kHalf; ++j) dmma(acc[i * kHalf + j], x[i], y[j]);
                }
            }
        }
    };
    for (int n = 0; n < count; ++n) {
        const Factor& F = P.f[f];
        const int stage = n % kStages;
        ptx::named_barrier_sync(kFull + stage, 2 * kThreads);
        const float* u = tiles + stage * S::floats;
        if (F.tall) multiply(std::true_type(), u);
        else multiply(std::false_type(), u);
        if (n + kStages < count) ptx::named_barrier_arrive(kEmpty + stage, 2 * kThreads);
        const bool last_of_factor = (first + n - F.tile0 + 1) * S::TL >= F.L;
        if (n + 1 < count && !last_of_factor) continue;
        double2* out = reinterpret_cast<double2*>(P.sums) + (size_t)(blockIdx.x + f) * S::tri * 32;
        if (kSplit) {
            if (warp < 2) {
                int b = 0;
#pragma unroll
                for (int i = 0; i < kSide; ++i) {
#pragma unroll
                    for (int j = i; j < kSide; ++j, ++b) out[tri_index(S::blocks, warp * NB + i, warp * NB + j) * 32 + lane] = make_double2(acc[b][0], acc[b][1]);
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
#pragma unroll
            for (int b = 0; b < S::tri; ++b) joined[(b * kWarps + warp) * 32 + lane] = make_double2(acc[b][0], acc[b][1]);
            ptx::named_barrier_sync(kJoin, kThreads);
            for (int b = warp; b < S::tri; b += kWarps) {
                double2 v = joined[b * kWarps * 32 + lane];
#pragma unroll
                for (int w = 1; w < kWarps; ++w) {
                    const double2 x = joined[(b * kWarps + w) * 32 + lane];
                    v.x += x.x;
                    v.y += x.y;
                }
                out[b * 32 + lane] = v;
            }
            ptx::named_barrier_sync(kJoin, kThreads);
        }
#pragma unroll
        for (int i = 0; i < kAcc; ++i) acc[i][0] = acc[i][1] = 0.0;
        ++f;
    }
}

// ------------------------------------------------------------------------------------------------ the iteration on r x r matrices
// A cluster takes a factor, a warp one block of 8 x 8 of the upper triangle of every product.  The products of commuting symmetric matrices are symmetric, so
// a block below the diagonal is the transpose of one above it, and the second operand's block (k, j) is the first operand's block (j, k): both are read along
// rows.  In the result of m8n8k4 a lane holds two neighbours of a row, and as the contraction may run in any order these two are just what it needs of that
// block as an operand (contraction indices 2 t and 2 t + 1, one for each of two instructions): blocks are stored as 32 pairs in the lanes' order, written and read
// without conflicts, 16 bytes at a time.  The whole matrix, both triangles, up to rank 48, where one CTA does a factor; above that, where every block is written
// into the shared memory of all CTAs of the cluster, the upper triangle, whose transposes are read as two single values.
// (Stores counted on mbarriers, st.async, in place of the cluster's barriers: rank 64 4.1 -> 4.4 us a step, 128 15.0 -> 15.7; bulk copies 4.4 and 17.5.)
__device__ __forceinline__ void st_cluster_f64x2(uint32_t at, double x, double y) {
    asm volatile("st.shared::cluster.v2.f64 [%0], {%1, %2};" ::"r"(at), "d"(x), "d"(y) : "memory");
}
__device__ __forceinline__ void st_cluster_f64(uint32_t at, double x) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(x) : "memory"); }

// `few` factors, whose clusters all find room at once: more CTAs to each (64 factors of rank 64 at 4 / 2 CTAs: 8.9 / 5.1 us a step, 14 of them 4.1 / 4.9).
template <int NB, bool FEW>
struct IterateShape {
    static constexpr int B = 2 * NB, tri = B * (B + 1) / 2;
    static constexpr bool whole = NB <= 3;                        // (in clusters the transposes' single stores cost more than they save)
    static constexpr int blocks = whole ? B * B : tri, bytes = blocks * 512;         // of a matrix
    static constexpr bool three = 4 * bytes > 220 * 1024;        // three matrices: the product that follows G takes G's place (two barriers more a step)
    // CTAs of a cluster: one warp to a block
    static constexpr int ctas = tri <= 21 ? 1 : tri <= 55 ? (FEW ? 4 : 2) : tri <= 105 ? (FEW ? 8 : 4) : 8, warps = (tri + ctas - 1) / ctas;
    static constexpr size_t smem = (size_t)(three ? 3 : 4) * bytes + B * 8;
    static_assert(!whole || ctas == 1, "in a cluster a block goes to the other CTAs without its transpose");
};

// For one factor: sums(block, s) gives this lane's two values of a block of S, out(row, column, value) takes Q.  memory: I::smem bytes; rank: of the CTA in its cluster.
template <typename I, typename Sums, typename Out>
__device__ __forceinline__ void iterate(const UpdateParams& P, unsigned char* memory, int rank, Sums sums, Out out) {
    constexpr int B = I::B, ctas = I::ctas;
    unsigned char* const G = memory;
    unsigned char* const Pk = G + I::bytes;
    unsigned char* const Q = Pk + I::bytes;
    unsigned char* const M = I::three ? G : Q + I::bytes;
    double* trace = reinterpret_cast<double*>(Q + (I::three ? 1 : 2) * I::bytes);      // [B], of the diagonal blocks
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int block = rank * I::warps + warp;
    const bool mine = block < I::tri;
    int bi = 0;
    while (mine && tri_index(B, bi + 1, bi + 1) <= block) ++bi;
    const int bj = mine ? bi + block - tri_index(B, bi, bi) : 0;
    auto meet = [&]() {
        if (ctas > 1) ptx::cluster_sync();
        else __syncthreads();
    };
    // Place of a lane's pair in its block (triangle: changed over so that the transposes are read without conflicts), and of its transposes' two values.
    const auto place_of = [](int l) { return I::whole ? l * 16 : (l ^ (l >> 3) ^ ((l >> 3 & 1) << 2)) * 16; };
    const int straight = place_of(lane), across0 = place_of(8 * t4 + (g >> 1)) + 8 * (g & 1), across1 = place_of(8 * t4 + 4 + (g >> 1)) + 8 * (g & 1);
    const int own = (I::whole ? bi * B + bj : block) * 512 + straight, other = (bj * B + bi) * 512;
    auto store = [&](unsigned char* X, const double (&v)[2]) {
        if (ctas == 1) {
            *reinterpret_cast<double2*>(X + own) = make_double2(v[0], v[1]);
            if (I::whole && bi != bj) {
                *reinterpret_cast<double*>(X + other + across0) = v[0];
                *reinterpret_cast<double*>(X + other + across1) = v[1];
            }
            return;
        }
        const uint32_t at = ptx::smem_u32(X);
#pragma unroll
        for (int i = 0; i < ctas; ++i) st_cluster_f64x2(ptx::map_to_cta(at, (uint32_t)i) + own, v[0], v[1]);      // (own added to each: added to `at`, rank 128 took 2 % longer)
    };
    // Block (bi, bj) of X Y, and of X2 Y.
    auto products = [&](auto two, const unsigned char* X, const unsigned char* X2, const unsigned char* Y, double (&v)[2], double (&v2)[2]) {
        constexpr bool TWO = decltype(two)::value;
        double odd[2] = {0.0, 0.0}, odd2[2] = {0.0, 0.0};
        v[0] = v[1] = 0.0;
        if (TWO) v2[0] = v2[1] = 0.0;
        auto step = [&](double2 x, double2 x2, double2 y) {
            dmma(v, x.x, y.x);
            dmma(odd, x.y, y.y);
            if (TWO) {
                dmma(v2, x2.x, y.x);
                dmma(odd2, x2.y, y.y);
            }
        };
        auto along = [&](const unsigned char* Z, int at) { return *reinterpret_cast<const double2*>(Z + at + straight); };
        if (I::whole) {
            const int x_at = bi * B * 512, y_at = bj * B * 512;
#pragma unroll
            for (int k = 0; k < B; ++k) step(along(X, x_at + k * 512), along(X2, x_at + k * 512), along(Y, y_at + k * 512));
        } else {
            // Blocks (i, k) left of the diagonal are read as transposes of (k, i): three ranges of k, in each of which the blocks follow by simple steps.
            auto across = [&](const unsigned char* Z, int at) {
                return make_double2(*reinterpret_cast<const double*>(Z + at + across0), *reinterpret_cast<const double*>(Z + at + across1));
            };
            int x_at = bi * 512, y_at = bj * 512, k = 0;         // blocks (0, bi), (0, bj)
#pragma unroll 2
            for (; k < bi; ++k, x_at += (B - k) * 512, y_at += (B - k) * 512) step(across(X, x_at), across(X2, x_at), across(Y, y_at));
#pragma unroll 2
            for (; k < bj; ++k, x_at += 512, y_at += (B - k) * 512) step(along(X, x_at), along(X2, x_at), across(Y, y_at));
#pragma unroll 2
            for (; k < B; ++k, x_at += 512, y_at += 512) step(along(X, x_at), along(X2, x_at), along(Y, y_at));
        }
        v[0] += odd[0];
        v[1] += odd[1];
        if (TWO) {
            v2[0] += odd2[0];
            v2[1] += odd2[1];
        }
    };
    double unused[2];
    auto product = [&](const unsigned char* X, const unsigned char* Y, double (&v)[2]) { products(std::false_type(), X, X, Y, v, unused); };
    if (ctas > 1) ptx::cluster_sync();                            // (every CTA of the cluster runs: its shared memory may be written)
    double s[2] = {0.0, 0.0};                                     // this lane's values of G
    if (mine) {
        sums(block, s);
        if (bi == bj) {
            double d = g == 2 * t4 ? s[0] : g == 2 * t4 + 1 ? s[1] : 0.0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
            if (ctas == 1 && lane == 0) trace[bi] = d;
            if (ctas > 1 && lane < ctas) st_cluster_f64(ptx::map_to_cta(ptx::smem_u32(trace + bi), (uint32_t)lane), d);
        }
        store(G, s);
    }
    meet();
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
            for (int i = 0; i < 2; ++i) p[i] = (bi == bj && g == 2 * t4 + i ? P.a : 0.0) + P.b * (alpha * s[i]) + P.c * (alpha * alpha * v[i]);
            store(Pk, p);
        }
        meet();
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
        if (I::three) meet();                                     // everybody has read G
        if (mine) store(M, v);
        meet();
        if (mine) {
            product(M, Pk, s);
            store(Q, q);                                          // (read by all before the barrier)
        }
        if (I::three) meet();                                     // everybody has read M
        if (mine) store(G, s);
        meet();
        alpha = 1.0;
    }
    if (mine) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = bi * 8 + g, col = bj * 8 + 2 * t4 + i;
            const float v = (float)(q[i] / norm);
            out(row, col, v);
            if (bi != bj) out(col, row, v);
        }
    }
}

template <int NB, bool FEW>
__global__ void __launch_bounds__(32 * IterateShape<NB, FEW>::warps) iterate_kernel(const __grid_constant__ UpdateParams P) {
    using S = Shape<NB>;
    using I = IterateShape<NB, FEW>;
    extern __shared__ __align__(16) unsigned char update_smem[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (behind the wait: apply_kernel reads what gram_kernel wrote before its own)
    const int f = (int)blockIdx.x / I::ctas, lane = threadIdx.x & 31;
    const Factor& F = P.f[f];
    // S, from its parts in the walkers' order
    auto sums = [&](int block, double (&s)[2]) {
        const int walkers = (int)min(kWalkers, P.tiles), tiles = (F.L + S::TL - 1) / S::TL;
        auto walker_of = [&](int tile) {                          // the one whose share holds the tile
            int w = (int)((long long)tile * walkers / P.tiles);
            while ((int)((long long)P.tiles * (w + 1) / walkers) <= tile) ++w;
            while ((int)((long long)P.tiles * w / walkers) > tile) --w;
            return w;
        };
        const int w0 = walker_of(F.tile0), w1 = walker_of(F.tile0 + tiles - 1);
        const double2* from = reinterpret_cast<const double2*>(P.sums) + (size_t)block * 32 + lane;
#pragma unroll 8
        for (int w = w0; w <= w1; ++w) {
            const double2 x = __ldcg(from + (size_t)(w + f) * S::tri * 32);
            s[0] += x.x;
            s[1] += x.y;
        }
    };
    float* const Q = P.Q + (size_t)f * S::r * S::r;
    iterate<I>(P, update_smem, (int)blockIdx.x % I::ctas, sums, [&](int row, int col, float v) { Q[row * S::r + col] = v; });
}

// ------------------------------------------------------------------------------------------------ u Q, and the weights
// On the fp32 pipe: a thread forms eight of the long side times four ranks, from a tile of u and Q in shared memory.  (In two or three tf32 parts on the tensor
// instructions it was no faster, and its errors, 2e-5 of the update, were ten times those of fp32.)  One CTA to an SM: two groups of four warps fill tiles of u in turn, two others
// multiply them by Q, each with a copy of its own.  Loads, products and stores then go on side by side; CTAs that did one after the
// other, three to an SM, took 50 us for fourteen factors of 11008 x 64 where these take 44 (and 150 where these take 131 at rank 128).  What bounds it is shared memory, three reads of 16 bytes for
// 32 products (eight by eight values a thread: fewer reads, but tiles too large to be dealt out evenly).
// u, four neighbours in memory, from the gradient and the new momentum.
struct Raw {
    uint4 g;
    float4 m;
};
__device__ __forceinline__ Raw load_raw(const UpdateParams& P, const Factor& F, size_t at, bool in) {
    Raw r;
    r.g = make_uint4(0u, 0u, 0u, 0u);
    r.m = zero4();
    if (in && F.momentum_out != nullptr) r.m = __ldcg(reinterpret_cast<const float4*>(F.momentum_out + at));
    if (in && (F.momentum_out == nullptr || P.nesterov)) {
        if (F.grad_fp32) r.g = __ldg(reinterpret_cast<const uint4*>(static_cast<const float*>(F.grad) + at));
        else {
            const uint2 p = __ldg(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(F.grad) + at));
            r.g.x = p.x;
            r.g.y = p.y;
        }
    }
    return r;
}
__device__ __forceinline__ float4 u_of(const UpdateParams& P, const Factor& F, const Raw& r) {
    if (F.momentum_out == nullptr) return grad_quad(F, r.g);
    return P.nesterov ? axpy2(P.mu, r.m, grad_quad(F, r.g)) : r.m;
}

constexpr int kApplyThreads = 4 * kThreads;
constexpr int kMultiply = kEmpty + kStages;                       // named barriers of the two groups that multiply (gram_kernel has one there)
template <int NB>
struct ApplyShape {
    using S = Shape<NB>;
    static constexpr int pitch = S::r + 4;                        // u, tall: [l][c]; wide: [c][l]
    static constexpr int floats = S::TL * pitch > S::r * S::TL ? S::TL * pitch : S::r * S::TL;
    static constexpr size_t bytes = (size_t)(2 * S::r * S::r + kStages * floats) * 4;
};
template <int NB>
__global__ void __launch_bounds__(kApplyThreads, 1) apply_kernel(const __grid_constant__ UpdateParams P) {
    using S = Shape<NB>;
    using A = ApplyShape<NB>;
    constexpr int TL = S::TL, groups = TL / 8;
    extern __shared__ __align__(16) unsigned char update_smem[];
    float* const Qs = reinterpret_cast<float*>(update_smem);      // [2][r][r]
    float* const tiles = Qs + 2 * S::r * S::r;
    const int group = (int)threadIdx.x / kThreads, half = group & 1;
    const int first = share(P, blockIdx.x), count = share(P, blockIdx.x + 1) - first;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int f = factor_of(P, first);
    if (group >= 2) {
        // ================================================================== fillers: tiles half, half + 2, ...
        // (iterate_kernel lets this kernel start when gram_kernel is through: u may be read before the wait for Q)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        for (int n = half; n < count; n += 2) {
            while (f + 1 < P.count && P.f[f + 1].tile0 <= first + n) ++f;
            const Factor& F = P.f[f];
            const int l0 = (first + n - F.tile0) * TL, stage = n % kStages;
            float* u = tiles + stage * A::floats;
            auto fill = [&](auto tall) {
                constexpr bool TALL = decltype(tall)::value;
                using D = Deal<NB, TALL>;
                constexpr int pitch = TALL ? A::pitch : TL;
                const D deal(F, l0, thread_here() % kThreads);
                float* to = u + deal.row * pitch + deal.col;
                const bool has = deal.row < D::at_once;
                auto part = [&](auto from) {                      // (half of the quads at a time: registers)
                    constexpr int FROM = decltype(from)::value, N = kQuads / 2;
                    Raw raw[N];
                    deal.template each<FROM, N>([&](int i, size_t at, bool in) { raw[i - FROM] = load_raw(P, F, at, in); });
                    if (FROM == 0 && n >= kStages) ptx::named_barrier_sync(kEmpty + stage, 2 * kThreads);     // the tile there before has been read
                    deal.template each<FROM, N>([&](int i, size_t, bool) {
                        if (has) *reinterpret_cast<float4*>(to + i * D::at_once * pitch) = u_of(P, F, raw[i - FROM]);
                    });
                };
                part(std::integral_constant<int, 0>());
                part(std::integral_constant<int, kQuads / 2>());
            };
            if (F.tall) fill(std::true_type());
            else fill(std::false_type());
            ptx::named_barrier_arrive(kFull + stage, 2 * kThreads);
        }
        return;
    }
    // ====================================================================== u Q: tiles half, half + 2, ...
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    float* const Q = Qs + half * S::r * S::r;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int loaded = -1;
    // A thread's outputs, quads of four neighbours in memory: number i of eight at place + (i / 4) * far + (i % 4) * near_by
    auto work = [&](auto tall, const Factor& F, int l0, const float* u, auto done) {
        constexpr bool TALL = decltype(tall)::value;
        // tall: ranks c .. c + 3, rows lg, lg + TL / 8, ...: a warp's lanes lie side by side along the rank
        // wide: ranks c .. c + 3, and two runs of four of the long side: the lanes lie side by side along it
        const int thread = thread_here() % kThreads, cg = TALL ? thread % (S::r / 4) : thread / groups, lg = TALL ? thread / (S::r / 4) : thread % groups;
        const bool has = TALL ? lg < groups : cg < S::r / 4;
        const size_t place = TALL ? (size_t)(l0 + lg) * S::r + cg * 4 : (size_t)(cg * 4) * F.L + (l0 + lg * 4);
        const size_t near_by = TALL ? (size_t)(groups * S::r) : (size_t)F.L, far = TALL ? 4 * near_by : (size_t)(TL / 2);
        auto inside = [&](int i) { return has && (TALL ? l0 + lg + i * groups < F.L : l0 + lg * 4 + (i / 4) * (TL / 2) < F.L); };
        float4 w[8];
        if (F.master != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = inside(i) ? *reinterpret_cast<const float4*>(F.master + place + (i / 4) * far + (i % 4) * near_by) : zero4();
        }
        float4 acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = zero4();
        if (TALL) {
            const float *x_at = u + (has ? lg : 0) * A::pitch, *q_at = Q + cg * 4;
#pragma unroll 1
            for (int j = 0; j < S::r; j += 4, x_at += 4, q_at += 4 * S::r) {
                float4 q[4], x[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) q[k] = *reinterpret_cast<const float4*>(q_at + k * S::r);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const float4*>(x_at + i * groups * A::pitch);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] = axpy2(k == 0 ? x[i].x : k == 1 ? x[i].y : k == 2 ? x[i].z : x[i].w, q[k], acc[i]);
                }
            }
        } else {
            const float *x_at = u + lg * 4, *q_at = Q + (has ? cg : 0) * 4;
#pragma unroll 4
            for (int j = 0; j < S::r; ++j, x_at += TL, q_at += S::r) {
                const float4 q = *reinterpret_cast<const float4*>(q_at);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 x = *reinterpret_cast<const float4*>(x_at + h * (TL / 2));
                    acc[4 * h] = axpy2(q.x, x, acc[4 * h]);
                    acc[4 * h + 1] = axpy2(q.y, x, acc[4 * h + 1]);
                    acc[4 * h + 2] = axpy2(q.z, x, acc[4 * h + 2]);
                    acc[4 * h + 3] = axpy2(q.w, x, acc[4 * h + 3]);
                }
            }
        }
        done();
        if (F.update != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (inside(i)) *reinterpret_cast<float4*>(F.update + place + (i / 4) * far + (i % 4) * near_by) = acc[i];
        }
        if (F.master == nullptr) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (inside(i)) step_weights(P, F, place + (i / 4) * far + (i % 4) * near_by, acc[i], w[i]);
        }
    };
    for (int n = half; n < count; n += 2) {
        while (f + 1 < P.count && P.f[f + 1].tile0 <= first + n) ++f;
        const Factor& F = P.f[f];
        const int l0 = (first + n - F.tile0) * TL, stage = n % kStages;
        if (loaded != f) {
            ptx::named_barrier_sync(kMultiply + half, kThreads);  // the group has read the Q before
            for (int i = (int)threadIdx.x % kThreads; i < S::r * S::r / 4; i += kThreads)
                reinterpret_cast<float4*>(Q)[i] = __ldcg(reinterpret_cast<const float4*>(P.Q + (size_t)f * S::r * S::r) + i);
            ptx::named_barrier_sync(kMultiply + half, kThreads);
            loaded = f;
        }
        ptx::named_barrier_sync(kFull + stage, 2 * kThreads);
        const float* u = tiles + stage * A::floats;
        auto done = [&]() {
            if (n + kStages < count) ptx::named_barrier_arrive(kEmpty + stage, 2 * kThreads);
        };
        if (F.tall) work(std::true_type(), F, l0, u, done);
        else work(std::false_type(), F, l0, u, done);
    }
}

// ------------------------------------------------------------------------------------------------ all of it in one launch
// For up to 14 short factors of rank 16 or 32: a cluster of eight CTAs takes a factor, a CTA an eighth of the long side, whose u stays in its shared memory.  Each forms its
// part of S, sends it to all others, adds the eight up in their order, and goes through the iteration by itself (all get the same Q), then forms its part of u Q.
// What bounds it is the chain of dependent steps.  Five steps, 1 / 2 / 3 / 4 / 6 / 14 factors in a captured graph, against the three kernels, us:
//     2048 x 16   7.4 /  7.5 /  7.4 /  7.4 /  7.6 /  7.5   against   9.8 / 10.8 / 10.9 / 10.6 / 10.9 / 11.4
//     4096 x 16   9.1 /  9.2 /  9.2 /  9.3 /  9.5 /  9.4   against  10.6 / 11.5 / 11.3 / 11.5 / 11.9 / 15.5
//     5632 x 16  11.4 / 11.4 / 11.5 / 11.4 / 11.4 / 11.6   against  12.3 / 13.0 / 12.9 / 13.2 / 13.6 / 18.3
//     6144 x 16  11.6 / 11.6 / 11.7 / 11.6 / 11.7 / 11.8   against  10.9 / 11.9 / 12.1 / 12.2 / 13.5 / 18.6
//     7680 x 16  12.9 / 12.9 / 13.0 / 13.0 / 13.0 / 13.1   against  12.5 / 13.3 / 14.0 / 14.0 / 15.7 / 18.8
//     8192 x 16  13.2 / 13.3 / 13.4 / 13.3 / 13.4 / 13.4   against  11.8 / 12.7 / 12.9 / 13.4 / 15.5 / 19.7
//     1024 x 32  13.0 / 13.1 / 13.1 / 13.1 / 13.3 / 13.4   against  14.7 / 15.5 / 15.6 / 15.7 / 15.7 / 16.1
//     2048 x 32  15.4 / 15.5 / 15.5 / 15.6 / 15.7 / 15.9   against  15.4 / 15.9 / 16.1 / 16.2 / 16.4 / 20.6
// and a call costs the host 5.5 us instead of 11.5.  Longer ones lose.  More factors: 16 clusters do not find room at once (64 x 16: 10.6 against 9.8).
constexpr int kOneCtas = 8, kOneFactors = 14, kMostOne = 2;             // CTAs to a factor; factors; rank / 16
constexpr int kOneRows = 1024;                                          // of the long side to a CTA, times (rank / 16)^2: what its shared memory is sized for
template <int NB>
constexpr int rows_that_pay(int count) { return NB > 1 || count > 3 ? kOneRows : count > 1 ? 960 : 704; }      // up to which it is the faster way
template <int NB>
struct OneShape {
    using I = IterateShape<NB, true>;
    static constexpr int r = 16 * NB, tri = I::tri, warps = 16, threads = 32 * warps;
    static constexpr int tall_pitch = r + 8;                      // u as in gram_kernel: tall [l][c], wide [c][l]
    static constexpr size_t part = (size_t)tri * 512, joined = warps * part, first = joined > (I::smem + 15) / 16 * 16 ? joined : (I::smem + 15) / 16 * 16;
    static constexpr size_t fixed = first + kOneCtas * part + r * r * 4;       // the warps' sums, then the iteration's matrices; parts of S; Q; u follows
    static int wide_pitch(int rows) { return (rows + 31) / 32 * 32 + 4; }
    static size_t bytes(int rows) { return fixed + (size_t)(rows * tall_pitch > r * wide_pitch(rows) ? rows * tall_pitch : r * wide_pitch(rows)) * 4; }
    static_assert(I::ctas == 1, "a CTA goes through the iteration by itself");
};
__host__ __device__ inline int one_rows(int L) { return (L / 8 + kOneCtas - 1) / kOneCtas * 8; }      // of a CTA

template <int NB>
__global__ void __launch_bounds__(OneShape<NB>::threads, 1) one_kernel(const __grid_constant__ UpdateParams P) {
    using O = OneShape<NB>;
    constexpr int r = O::r, blocks = 2 * NB, kAtOnce = 4;
    extern __shared__ __align__(16) unsigned char update_smem[];
    double2* const joined = reinterpret_cast<double2*>(update_smem);
    double2* const parts = reinterpret_cast<double2*>(update_smem + O::first);
    float* const Q = reinterpret_cast<float*>(update_smem + O::first + kOneCtas * O::part);
    float* const u = Q + r * r;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int f = (int)blockIdx.x / kOneCtas, rank = (int)blockIdx.x % kOneCtas;
    const Factor& F = P.f[f];
    const int most = one_rows(F.L), l0 = rank * most, rows = max(0, min(most, F.L - l0)), wide_pitch = (most + 31) / 32 * 32 + 4;
    const int quads = rows * r / 4, wide_quads = max(rows / 4, 1);         // quads of four neighbours in memory; of a rank's row
    // ---- u, into shared memory
    for (int first = (int)threadIdx.x; first < quads; first += kAtOnce * O::threads) {
        Raw raw[kAtOnce];
        size_t at[kAtOnce];
        int to[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int q = first + i * O::threads;
            if (F.tall) {
                at[i] = (size_t)l0 * r + (size_t)q * 4;
                to[i] = q / (r / 4) * O::tall_pitch + q % (r / 4) * 4;
            } else {
                const int c = q / wide_quads, l = (q - c * wide_quads) * 4;
                at[i] = (size_t)c * F.L + (l0 + l);
                to[i] = c * wide_pitch + l;
            }
            raw[i].g = make_uint4(0u, 0u, 0u, 0u);
            raw[i].m = zero4();
            if (q >= quads) continue;
            if (F.grad_fp32) raw[i].g = *reinterpret_cast<const uint4*>(static_cast<const float*>(F.grad) + at[i]);
            else {
                const uint2 two = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(F.grad) + at[i]);
                raw[i].g.x = two.x;
                raw[i].g.y = two.y;
            }
            if (F.momentum != nullptr) raw[i].m = *reinterpret_cast<const float4*>(F.momentum + at[i]);
            if (F.master != nullptr) asm volatile("prefetch.global.L2 [%0];" ::"l"(F.master + at[i]));
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (first + i * O::threads >= quads) break;
            const float4 grad = grad_quad(F, raw[i].g);
            float4 x = grad;
            if (F.momentum != nullptr) {
                const float4 m = axpy2(P.mu, raw[i].m, grad);
                *reinterpret_cast<float4*>(F.momentum_out + at[i]) = m;
                x = P.nesterov ? axpy2(P.mu, m, grad) : m;
            }
            *reinterpret_cast<float4*>(u + to[i]) = x;
        }
    }
    __syncthreads();
    // ---- a warp's part of S, the CTA's, and everybody's
    {
        double acc[O::tri][2];
#pragma unroll
        for (int b = 0; b < O::tri; ++b) acc[b][0] = acc[b][1] = 0.0;
        const int sl = F.tall ? O::tall_pitch : 1, sc = F.tall ? 1 : wide_pitch;
        const float* at = u + t4 * sl + g * sc;
#pragma unroll 2
        for (int l = warp * 4; l < rows; l += 4 * O::warps) {
            double x[blocks];
#pragma unroll
            for (int i = 0; i < blocks; ++i) x[i] = (double)at[l * sl + i * 8 * sc];
            int b = 0;
#pragma unroll
            for (int i = 0; i < blocks; ++i) {
#pragma unroll
                for (int j = i; j < blocks; ++j) dmma(acc[b++], x[i], x[j]);
            }
        }
#pragma unroll
        for (int b = 0; b < O::tri; ++b) joined[(b * O::warps + warp) * 32 + lane] = make_double2(acc[b][0], acc[b][1]);
    }
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");           // (every CTA of the cluster runs: its shared memory may be written)
    for (int b = warp; b < O::tri; b += O::warps) {
        double2 v = joined[b * O::warps * 32 + lane];
#pragma unroll
        for (int w = 1; w < O::warps; ++w) {
            const double2 x = joined[(b * O::warps + w) * 32 + lane];
            v.x += x.x;
            v.y += x.y;
        }
        const uint32_t to = ptx::smem_u32(parts + (rank * O::tri + b) * 32 + lane);
#pragma unroll
        for (int i = 0; i < kOneCtas; ++i) st_cluster_f64x2(ptx::map_to_cta(to, (uint32_t)i), v.x, v.y);
    }
    ptx::cluster_sync();
    auto sums = [&](int block, double (&s)[2]) {
#pragma unroll
        for (int i = 0; i < kOneCtas; ++i) {
            const double2 x = parts[(i * O::tri + block) * 32 + lane];
            s[0] += x.x;
            s[1] += x.y;
        }
    };
    // ---- u Q: a thread forms four ranks of four of the long side (tall: a quarter of the rows apart, wide: neighbours); its first weights are asked for before the iteration
    const int runs = rows / 4, items = runs * (r / 4);
    const size_t step = F.tall ? (size_t)runs * r : (size_t)F.L;
    int cg = 0, lg = 0;
    size_t place = 0;
    float4 w[4];
    auto ask = [&](int item) {
        cg = F.tall ? item % (r / 4) : item / wide_quads;
        lg = F.tall ? item / (r / 4) : item - cg * wide_quads;
        place = F.tall ? (size_t)(l0 + lg) * r + cg * 4 : (size_t)(cg * 4) * F.L + (l0 + lg * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = F.master != nullptr && item < items ? *reinterpret_cast<const float4*>(F.master + place + i * step) : zero4();
    };
    ask((int)threadIdx.x);
    iterate<typename O::I>(P, update_smem, 0, sums, [&](int row, int col, float v) { Q[row * r + col] = v; });
    __syncthreads();
    for (int item = (int)threadIdx.x; item < items; item += O::threads) {
        if (item >= O::threads) ask(item);
        float4 acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = zero4();
        if (F.tall) {
#pragma unroll 2
            for (int j = 0; j < r; j += 4) {
                float4 q[4], x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) q[k] = *reinterpret_cast<const float4*>(Q + (j + k) * r + cg * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(u + (lg + i * runs) * O::tall_pitch + j);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i] = axpy2(k == 0 ? x[i].x : k == 1 ? x[i].y : k == 2 ? x[i].z : x[i].w, q[k], acc[i]);
                }
            }
        } else {
#pragma unroll 4
            for (int j = 0; j < r; ++j) {
                const float4 q = *reinterpret_cast<const float4*>(Q + j * r + cg * 4), x = *reinterpret_cast<const float4*>(u + j * wide_pitch + lg * 4);
                acc[0] = axpy2(q.x, x, acc[0]);
                acc[1] = axpy2(q.y, x, acc[1]);
                acc[2] = axpy2(q.z, x, acc[2]);
                acc[3] = axpy2(q.w, x, acc[3]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const size_t at = place + i * step;
            if (F.update != nullptr) *reinterpret_cast<float4*>(F.update + at) = acc[i];
            if (F.master != nullptr) step_weights(P, F, at, acc[i], w[i]);
        }
    }
}

// ------------------------------------------------------------------------------------------------ host
template <int NB>
int tiles_of(int L) { return (L + Shape<NB>::TL - 1) / Shape<NB>::TL; }

template <int NB>
size_t sums_bytes(int tiles, int count) { return (size_t)((tiles < kWalkers ? tiles : kWalkers) + count) * Shape<NB>::tri * 512; }

template <int NB>
bool takes_one(const UpdateParams& P, int* rows) {
    if (P.count > kOneFactors) return false;
    *rows = 0;
    for (int i = 0; i < P.count; ++i) *rows = max(*rows, one_rows(P.f[i].L));
    return *rows * NB * NB <= rows_that_pay<NB>(P.count);
}

template <int NB>
lowra_status launch_one(const UpdateParams& P, int rows, cudaStream_t stream) {
    static SmemLimit limit = {};
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kOneCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cfg.gridDim = dim3((unsigned)(P.count * kOneCtas), 1, 1);
    cfg.blockDim = dim3(OneShape<NB>::threads, 1, 1);
    cfg.dynamicSmemBytes = OneShape<NB>::bytes(rows);
    if (ensure_smem_limit(reinterpret_cast<const void*>(one_kernel<NB>), OneShape<NB>::bytes(kOneRows / NB / NB), &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
    return cudaLaunchKernelEx(&cfg, one_kernel<NB>, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}

template <int NB>
lowra_status launch_update(UpdateParams& P, void* workspace, cudaStream_t stream) {
    if constexpr (NB <= kMostOne) {
        int rows = 0;
        if (takes_one<NB>(P, &rows)) return launch_one<NB>(P, rows, stream);
    }
    using S = Shape<NB>;
    using A = ApplyShape<NB>;
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
    cfg.blockDim = dim3(kGramThreads, 1, 1);
    {
        static SmemLimit limit = {};
        cfg.dynamicSmemBytes = GramMemory<NB>::bytes;
        if (ensure_smem_limit(reinterpret_cast<const void*>(gram_kernel<NB>), cfg.dynamicSmemBytes, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
        if (cudaLaunchKernelEx(&cfg, gram_kernel<NB>, P) != cudaSuccess) return LOWRA_ERR_CUDA;
    }
    auto iterate = [&](auto few) -> bool {
        constexpr bool FEW = decltype(few)::value;
        using I = IterateShape<NB, FEW>;
        static SmemLimit limit = {};
        cfg.dynamicSmemBytes = I::smem;
        // one to an SM where there are SMs enough (several clusters on the same ones, as they come in one after the other: 8.8 us a step instead of 4.5)
        if (P.count * I::ctas <= kNumSMs && cfg.dynamicSmemBytes < 120 * 1024) cfg.dynamicSmemBytes = 120 * 1024;
        cfg.gridDim = dim3((unsigned)(P.count * I::ctas), 1, 1);
        cfg.blockDim = dim3(32u * I::warps, 1, 1);
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)I::ctas;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = I::ctas > 1 ? 2 : 1;
        if (ensure_smem_limit(reinterpret_cast<const void*>(iterate_kernel<NB, FEW>), cfg.dynamicSmemBytes, &limit) != LOWRA_OK) return false;
        return cudaLaunchKernelEx(&cfg, iterate_kernel<NB, FEW>, P) == cudaSuccess;
    };
    bool launched = false;
    if constexpr (IterateShape<NB, true>::ctas == IterateShape<NB, false>::ctas) launched = iterate(std::true_type());      // (the two forms are one)
    else launched = P.count * IterateShape<NB, true>::ctas <= kNumSMs ? iterate(std::true_type()) : iterate(std::false_type());
    if (!launched) return LOWRA_ERR_CUDA;
    cfg.numAttrs = 1;
    static SmemLimit limit = {};
    cfg.dynamicSmemBytes = A::bytes;
    cfg.gridDim = dim3(walkers, 1, 1);
    cfg.blockDim = dim3(kApplyThreads, 1, 1);
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
    for (int i = 0; i < count; ++i) {
        if (m[i].rows != r && m[i].cols != r) return LOWRA_ERR_SHAPE;
        const int32_t L = m[i].rows == r ? m[i].cols : m[i].rows;
        if (L < 8 || L > kLongest || L % 8 != 0) return LOWRA_ERR_SHAPE;      // (their tiles, and those of all, then are numbers of 32 bits)
    }
    return LOWRA_OK;
}

// Arrays in each other's way: something written that shares memory with anything else that the call reads or writes, of another member or of the same one.  (Momentum
// and master may be updated in place, element for element.)  In the order of their places, an array is in the way of one before it if it is in that of the one that
// reaches furthest, among all if it is written, among the written if it is read.
enum Clash { kNone, kWithin, kBetween };
Clash find_clash(const UpdateParams& P, size_t r) {
    struct Array {
        uintptr_t at, end;
        int member;
        bool written;
    } arrays[7 * kMaxFactors];
    int n = 0;
    for (int i = 0; i < P.count; ++i) {
        const Factor& F = P.f[i];
        const size_t elements = (size_t)F.L * r;
        auto add = [&](const void* p, size_t bytes, bool written) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(p);
            if (p != nullptr) arrays[n++] = Array{at, at + elements * bytes, i, written};
        };
        add(F.grad, F.grad_fp32 ? 4 : 2, false);
        if (F.momentum != F.momentum_out) add(F.momentum, 4, false);
        if (F.master != F.master_out) add(F.master, 4, false);
        add(F.momentum_out, 4, true);
        add(F.master_out, 4, true);
        add(F.weight, 2, true);
        add(F.update, 4, true);
    }
    std::sort(arrays, arrays + n, [](const Array& a, const Array& b) { return a.at < b.at; });
    Clash found = kNone;
    const Array *any = nullptr, *written = nullptr;             // of those before, the one that reaches furthest
    for (int i = 0; i < n; ++i) {
        const Array &a = arrays[i], *before = a.written ? any : written;
        if (before != nullptr && a.at < before->end) {
            if (a.member != before->member) return kBetween;
            found = kWithin;
        }
        if (any == nullptr || a.end > any->end) any = &a;
        if (a.written && (written == nullptr || a.end > written->end)) written = &a;
    }
    return found;
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
    const Clash clash = find_clash(P, (size_t)r);
    if (clash == kBetween) return LOWRA_ERR_SHAPE;
    if (workspace_bytes < lowra_update_workspace_bytes(members_host, count, r) || (reinterpret_cast<uintptr_t>(workspace_dev) & 255u) != 0) return LOWRA_ERR_WORKSPACE;
    if (clash != kNone) return LOWRA_ERR_SHAPE;
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
