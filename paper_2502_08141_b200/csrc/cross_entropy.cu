// lowra_cross_entropy: cross entropy over a vocabulary of V words from hidden states X [M, K] and the head's weights W [V, K], in pieces of the vocabulary, and the gradient of X:
//     l = X W^T;   loss = log sum_v exp(l_v) - l_y;   dX = c (softmax(l) - onehot(y)) W,   c = scale * weights[m]
// The logits are never kept.  Without the gradient a tile of them leaves, of every token, its largest and the sum of the exponentials under it.  With the gradient a piece of the
// vocabulary at a time goes through two products: e = exp(l - lift) of the piece, in bf16, into scratch; O += e W_piece in fp32.  The lift of a token is a whole number of octaves,
// zero as long as the largest logits of all its tiles are within 64 octaves of zero.  Where a tile's are not, its exponentials are taken under a lift of its own, and between the two products
// what the token has so far (its exponentials in the piece, sums and O) is brought to the largest lift: by a power of two, exactly, and hardly ever.
// The label's own word is left out of e and of the sum S, and comes back at the end:
//     p_y = E / (S + E);   dX = c (O - S W_y) / (S + E);   loss = log(1 + S / E)          E = exp(l_y - lift)
// so that 1 - p_y = S / (S + E) and a small loss have no cancellation (with e_y among the others, a token known to 0.99 got its gradient to 2^-9 / 0.01).
// That is two products of 2 M V K operations, where forming the sums first and the exponentials again would be three.
// The tensor core adds up in fp32 without rounding to nearest, which over 256 additions takes some 2^-18 off a logit; so a logit's sum is formed in segments of 1024 features, which the epilogue
// adds (losses over 4096 features: error against fp64 2.0e-6 -> 5e-7).  The second product is not cut: over 16000 words that leaves some 4e-6 of dX, which is rounded to bf16 in the end.
// The exponentials are bf16 in the second product because its operands are of one type and W is bf16 (as two such numbers each they would double that product): 1.4e-4 to 1.5e-4 of the gradient's norm
// over a vocabulary of 32000 to 50265 words, beside 1.66e-3 for the rounding of dX itself; 2^-9 at most, where one word has all that the label has not.  S is the sum of the unrounded ones.
//
// The products: CTA pairs (clusters of two) walk over tiles of 256 tokens x up to 256 words (features), tcgen05.mma with cta_group::2, both operands by TMA, 64 contraction indices
// (32 KB a CTA) to a stage, six stages; two accumulators in turn, so the epilogue's eight warps work on one tile while the next is formed.
// Up to 64 tokens and no gradient, bound by reading W: the other way round, 256 words by 32 or 64 tokens, ten stages; a pair's MMAs then take an eighth or a quarter of the time that its words do.
// Measured: 4096 tokens, 32000 words, 4096 features with the gradient 1400 us at full clock and 1650 under the power cap (at the rate of two library products 1262 and 1509), the tensor pipe 88 to 91 %
// busy; 777 tokens, 50265 words, 1024 features 189 to 193 us (94: nine tokens are all that the fourth tile of them holds, and the pipe is 75 % busy); 16 tokens, 32000 words, 4096 features, loss alone 46 to 48 us (W
// once: 40.6).
// warp 0 = TMA, 1 = MMA (of the CTA of rank 0) and TMEM, 4-11 = epilogue.  The 128 columns that an epilogue's thread holds, and 32 more on their way, do not fit into the 168 registers that
// twelve warps get: the first four give some to the others.  All waits are bounded (lowra_set_wait_limit); no CTA waits for another cluster.
#include <atomic>

#include "gemm_params.cuh"
#include "lowra_diag.h"
#include "ptx.cuh"

namespace lowra {

namespace {

constexpr int kTile = 256;                        // tokens, and at most so many words or features, of a pair's tile
constexpr int kDepth = 64;                        // contraction indices of a stage
constexpr uint32_t kHalfBytes = 128 * kDepth * 2;
constexpr int kFewTokens = 64;                    // up to so many, the words are the tile's rows and the tokens its columns
constexpr int kThreads = 384, kEpilogue = 8, kFirstEpilogue = 4;      // threads; epilogue warps, behind four others
constexpr int kLaunchRegisters = 168, kFewRegisters = 40, kManyRegisters = 232;   // a thread: at the launch, of the first four warps, of the others
static_assert(128 * kFewRegisters + 256 * kManyRegisters <= kThreads * kLaunchRegisters, "what the others take, the first four have given (a larger share would be waited for without end)");
constexpr uint64_t kGrace = 50ull * 1000ull;      // after a failure: time for copies and MMAs still in flight to land
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kHeadroom = 64.0f;                // octaves that the largest exponentials may be from one
constexpr int kSegment = 16;                      // contraction blocks of a logit that are added up in the tensor memory
constexpr int kSums = 0, kExponentials = 1, kGradient = 2, kFew = 3;
// Stages of the ring: 128 rows of either operand, or, for few tokens, 128 words and 32 tokens.
template <int KIND>
constexpr uint32_t kStageBytes = kHalfBytes + (KIND == kFew ? kHalfBytes / 4 : kHalfBytes);
template <int KIND>
constexpr int kStages = KIND == kFew ? 10 : 6;
constexpr int kMostStages = 10;
template <int KIND>
constexpr uint32_t kSmem = kStages<KIND> * kStageBytes<KIND> + 1024 + (KIND == kFew ? 8 * 32 * 8 : 0);

struct CeBarriers {
    uint64_t full[kMostStages], empty[kMostStages];
    uint64_t tmem_full[2], tmem_empty[2];
    uint32_t tmem_base, abort;
};
static_assert(sizeof(CeBarriers) <= 1024, "barrier block");

// Of a token: the label's logit, lift and sum so far, 2^-(lift added by the last piece).
struct CeRows {
    float *logit, *lift, *sum, *scale;
};

// What the end of a token's gradient takes: dX = c (O - S W_y) / (S + E).
struct CeEnd {
    CeRows rows;
    const uint16_t* W;
    const long long* labels;
    const float* weights;
    uint16_t* dX;
    long long ignore;
    int V, K;
    float scale;
};

struct CeParams {
    CUtensorMap a, b;                             // X, or the exponentials [M, piece];  W as [V, K], in boxes of words or of 64 words x 64 features  (few tokens: W; X)
    int M, N, V;                                  // tokens; words of the piece or features; words in all
    int v0;                                       // the piece's first word
    int width, tiles_m, tiles_n;                  // columns of a tile; tiles  (few tokens: words of a tile, its rows; tiles_m 1)
    int columns;                                  // (few tokens) of a tile: the tokens, filled up to a multiple of 32
    int a_rows, a_halves;                         // (not of few tokens) rows that a CTA loads of its half of a tile's tokens, and CTAs of a pair that do
    int whole, splits;                            // the first tiles are whole, the contraction of the others is cut into so many parts (all whole: splits 1)
    int blocks;                                   // contraction blocks in all
    int first, last;                              // the first piece: lift and O have no value yet; (gradient) the last one: whole tiles are finished
    const long long* labels;
    const float* lift;                            // (exponentials) a token's lift so far, in octaves
    float* label_logit;                           // l_y (out)
    float2* stats;                                // [2 tiles_n][M]: of half a tile (few tokens: [CTAs][M]), (largest in octaves, or lift; sum)
    uint16_t* e;                                  // [M, ld_e]
    long long ld_e;
    const float* scale;                           // (gradient) 2^-(lift added by the piece)
    float *out, *parts;                           // (gradient) O [M, N] of whole tiles; of the others' parts, [part][tile][256 tokens][256 features]
    CeEnd end;                                    // (gradient)
    uint32_t* status;
    unsigned long long wait_ns;
    int clear_status;
    int withheld;                                 // diagnostic (lowra_diag_drop_tiles): nothing is loaded behind a pair's first block, so the waits run out
};

// The factors of a token's O and of its label's row of W in dX.  S and O are brought to S in [1/2, 1) first: the label may be so far above the lift that its own exponential under it is no fp32 number,
// while the others are as far above it too.
struct Factors {
    float o, w, scale;        // of O scale, a power of two, with it; of W
    const uint16_t* row;      // null: the token does not count, or has no word (and o, w are NaN)
};
__device__ __forceinline__ Factors factors_of(const CeEnd& E, int m) {
    const long long y = E.labels[m];
    if (y < 0 || y >= E.V) {
        const float none = y == E.ignore ? 0.0f : NAN;
        return {none, none, 1.0f, nullptr};
    }
    if (y == E.ignore) return {0.0f, 0.0f, 1.0f, nullptr};
    const float logit = E.rows.logit[m], sum = E.rows.sum[m], c = E.weights != nullptr ? E.scale * E.weights[m] : E.scale;
    int octaves = 0;
    const float others = frexpf(sum, &octaves);               // sum = others 2^octaves, others in [1/2, 1), or both zero
    const float own = logit < INFINITY ? exp2f(fmaf(logit, kLog2e, -(E.rows.lift[m] + (float)octaves))) : NAN;
    const float a = c / (others + own);
    return {a, -a * others, exp2f((float)-octaves), E.W + (size_t)y * E.K};
}
// Eight features of dX from those of O, at feature k.
__device__ __forceinline__ uint4 end_of(const Factors& f, const float (&o)[8], int k) {
    if (f.row == nullptr) {
        const uint32_t v = pack_bf16x2(f.o, f.o);     // (zero or NaN, whatever O holds)
        return make_uint4(v, v, v, v);
    }
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(f.row + k));
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        r[j] = pack_bf16x2(fmaf(f.w, __uint_as_float(x[j] << 16), f.o * (f.scale * o[2 * j])), fmaf(f.w, __uint_as_float(x[j] & 0xffff0000u), f.o * (f.scale * o[2 * j + 1])));
    return make_uint4(r[0], r[1], r[2], r[3]);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Of 32 values a lane, each joined over the lanes: lane l gets the one numbered l.  Halves of the values change places, so that it takes 31 shuffles in all.
template <typename F>
__device__ __forceinline__ float over_lanes(float (&v)[32], F join) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const bool upper = (lane & d) != 0;
            const float keep = upper ? v[i + d] : v[i], give = upper ? v[i] : v[i + d];
            v[i] = join(keep, __shfl_xor_sync(0xffffffffu, give, d));
        }
    return v[0];
}

template <int KIND>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ CeParams P) {
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int kRing = kStages<KIND>;
    constexpr uint32_t kStage = kStageBytes<KIND>;
    CeBarriers* bars = reinterpret_cast<CeBarriers*>(smem + kRing * kStage);
    [[maybe_unused]] float2* const parts = reinterpret_cast<float2*>(smem + kRing * kStage + 1024);      // (few tokens) [half of the tokens][quarter of the words][token]
    volatile uint32_t* abort_flag = &bars->abort;
    if ((ptx::smem_u32(smem) & 1023u) != 0u) {      // never seen; without it the operand descriptors would be wrong
        if (threadIdx.x == 0) atomicExch(P.status, (uint32_t)LOWRA_ERR_CUDA);
        return;
    }
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t crank = blockIdx.x & 1u;
    const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
    const int rest = P.tiles_m * P.tiles_n - P.whole, units = P.whole + rest * P.splits;
    const bool mn = KIND == kGradient;              // W's features are the contiguous ones of its tiles

    if (threadIdx.x == 0) {
        for (int s = 0; s < kRing; ++s) { ptx::mbar_init(&bars->full[s], 1); ptx::mbar_init(&bars->empty[s], 1); }
        for (int a = 0; a < 2; ++a) { ptx::mbar_init(&bars->tmem_full[a], 1); ptx::mbar_init(&bars->tmem_empty[a], 2 * kEpilogue); }
        bars->abort = 0u;
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&P.a);
        ptx::prefetch_tensormap(&P.b);
    }
    if (warp == 1) ptx::tmem_alloc_pair(&bars->tmem_base, 512);
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync();
    ptx::tc_fence_after();
    pdl_enter();
    const uint32_t tmem_base = bars->tmem_base;
    if (P.clear_status && blockIdx.x == 0 && threadIdx.x == 0) *P.status = 0u;
    bool failed = false;

    // Unit u: its tile (tokens fastest, so that the pairs at work share the words or features of their tiles), and which of its parts (none: the whole contraction).
    auto tile_of = [&](int u) { return u < P.whole ? u : P.whole + (u - P.whole) % rest; };
    auto blocks_of = [&](int u, int* kb0) {
        *kb0 = 0;
        if (u < P.whole) return P.blocks;
        const int s = (u - P.whole) / rest;
        *kb0 = (int)((long long)P.blocks * s / P.splits);
        return (int)((long long)P.blocks * (s + 1) / P.splits) - *kb0;
    };
    auto segments_of = [&](int n) { return KIND == kGradient ? (n > 0 ? 1 : 0) : (n + kSegment - 1) / kSegment; };
    if (warp < kFirstEpilogue) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
        if (warp == 0) {
            const bool leader = ptx::elect_one();
            ptx::fence_proxy_async_all();               // (the exponentials were written by ordinary stores)
            const uint32_t full0 = ptx::map_to_cta(ptx::smem_u32(&bars->full[0]), 0u);
            // of the pair: rows and columns x 64 x 2 bytes
            const uint32_t a_bytes = KIND == kFew ? (uint32_t)P.width * (kDepth * 2) : (uint32_t)(P.a_rows * P.a_halves) * (kDepth * 2);
            const uint32_t bytes = a_bytes + (uint32_t)(KIND == kFew ? P.columns : P.width) * (kDepth * 2);
            const bool has_a = KIND == kFew || (int)crank < P.a_halves;
            int s = 0;
            uint32_t ph = 0;
            const int loaded = P.withheld ? pair + 1 : units;
            for (int u = pair; u < loaded && !failed; u += pairs) {
                const int t = tile_of(u);
                const int m0 = KIND == kFew ? P.v0 + t * P.width + (int)crank * (P.width / 2) : t % P.tiles_m * kTile + (int)crank * 128;
                const int n0 = KIND == kFew ? (int)crank * (P.columns / 2) : t / P.tiles_m * P.width + (int)crank * (P.width / 2);
                int kb0;
                int n = blocks_of(u, &kb0);
                if (P.withheld && n > 1) n = 1;
                for (int kb = kb0; kb < kb0 + n; ++kb) {
                    if (!ptx::mbar_wait_lanes(&bars->empty[s], ph ^ 1u, abort_flag, P.wait_ns)) { failed = true; break; }
                    unsigned char* a_s = smem + s * kStage;
                    const uint32_t bar = full0 + (uint32_t)s * 8u;
                    if (leader) {
                        if (crank == 0u) ptx::mbar_arrive_expect_tx(&bars->full[s], bytes);
                        if (has_a) ptx::tma_load_2d_pair(a_s, &P.a, kb * kDepth, m0, bar);
                        if (mn) {
                            ptx::tma_load_2d_pair(a_s + kHalfBytes, &P.b, n0, P.v0 + kb * kDepth, bar);
                            ptx::tma_load_2d_pair(a_s + kHalfBytes + 8192, &P.b, n0 + 64, P.v0 + kb * kDepth, bar);
                        } else {
                            ptx::tma_load_2d_pair(a_s + kHalfBytes, &P.b, kb * kDepth, KIND == kFew ? n0 : P.v0 + n0, bar);
                        }
                    }
                    __syncwarp();
                    if (++s == kRing) { s = 0; ph ^= 1u; }
                }
            }
            if (failed) bars->abort = 1u;
        } else if (warp == 1) {
            if (crank == 0u) {
                const bool leader = ptx::elect_one();
                const uint32_t idesc = ptx::umma_idesc_bf16(kTile, KIND == kFew ? P.columns : P.width) | (mn ? 1u << 16 : 0u), b_step = mn ? 128u : 2u;
                const uint64_t a0 = ptx::umma_desc_k_sw128(ptx::smem_u32(smem));
                const uint64_t b0 = mn ? ptx::umma_desc_mn_sw128(ptx::smem_u32(smem) + kHalfBytes, 8192u) : ptx::umma_desc_k_sw128(ptx::smem_u32(smem) + kHalfBytes);
                int s = 0, i = 0;
                uint32_t ph = 0;
                bool ready = false;
                for (int u = pair; u < units && !failed; u += pairs) {
                    int kb0;
                    const int n = blocks_of(u, &kb0), segments = segments_of(n);      // (none in a part without blocks: a short last piece)
                    for (int g = 0; g < segments && !failed; ++g, ++i) {
                        const uint32_t acc = (uint32_t)i & 1u, d = tmem_base + acc * kTile;
                        if (!ptx::mbar_wait_lanes(&bars->tmem_empty[acc], (((uint32_t)i >> 1) & 1u) ^ 1u, abort_flag, P.wait_ns)) { failed = true; break; }
                        ptx::tc_fence_after();
                        const int first = n * g / segments, last = n * (g + 1) / segments - 1;
                        for (int kb = first; kb <= last; ++kb) {
                            if (!ready && !ptx::mbar_wait_lanes(&bars->full[s], ph, abort_flag, P.wait_ns)) { failed = true; break; }
                            ptx::tc_fence_after();
                            const uint64_t a = a0 + (uint64_t)s * (kStage >> 4), b = b0 + (uint64_t)s * (kStage >> 4);
                            const int here = s;
                            if (++s == kRing) { s = 0; ph ^= 1u; }
                            ready = __all_sync(0xffffffffu, ptx::mbar_test_wait(&bars->full[s], ph));      // (asked for ahead of its use)
                            if (leader) {
#pragma unroll
                                for (uint32_t k = 0; k < kDepth / 16; ++k) ptx::umma_bf16_pair(d, a + 2u * k, b + b_step * k, idesc, (kb != first || k != 0) ? 1u : 0u);
                                ptx::umma_commit_pair(&bars->empty[here]);
                                if (kb == last) ptx::umma_commit_pair(&bars->tmem_full[acc]);
                            }
                            __syncwarp();
                        }
                    }
                }
                if (failed) bars->abort = 1u;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
        // ------------------------------------------------------------------ epilogue: a lane is a token, a warp takes half of the tile's columns, 32 at a time
        const int q = warp & 3, ch = (warp - kFirstEpilogue) >> 2;
        const int chunks = P.width / 32, c_first = ch == 0 ? 0 : (chunks + 1) / 2, c_count = ch == 0 ? (chunks + 1) / 2 : chunks / 2;
        const uint32_t empty0 = ptx::map_to_cta(ptx::smem_u32(&bars->tmem_empty[0]), 0u);
        int i = 0;
        // an accumulator's columns from `first` on: `take` reads them, then it is free
        auto drain = [&](int first, auto take) {
            const uint32_t acc = (uint32_t)i & 1u;
            if (!ptx::mbar_wait_warp(&bars->tmem_full[acc], ((uint32_t)i >> 1) & 1u, abort_flag, P.wait_ns)) { failed = true; return; }
            ptx::tc_fence_after();
            take(tmem_base + acc * kTile + ((uint32_t)(q * 32) << 16) + (uint32_t)first);
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (crank == 0u) ptx::mbar_arrive(&bars->tmem_empty[acc]);
                else ptx::mbar_arrive_cluster(empty0 + acc * 8u);
            }
            ++i;
        };
        if constexpr (KIND == kFew) {
            // A lane is a word, a column a token, half of the tokens to a warp.  Lane l keeps the largest and the sum of its token l, over all of the CTA's tiles.
            const int first = ch * 32, place = q * 32 + lane, half = P.width / 2, token = first + lane;
            long long label = -1;
            if (token < P.M) label = P.labels[token];
            float top = -INFINITY, total = 0.0f;
            for (int u = pair; u < units && !failed; u += pairs) {
                const int word0 = P.v0 + u * P.width + (int)crank * half + q * 32, segments = segments_of(P.blocks);
                const bool is_word = place < half && word0 + lane < P.V;
                float v[32], e[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = 0.0f;
                for (int g = 0; g < segments && !failed; ++g)
                    drain(first, [&](uint32_t from) {
                        if (first >= P.columns) return;
                        uint32_t w[32];
                        ptx::tmem_ld_32x32(from, w);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += __uint_as_float(w[j]);
                    });
                if (failed) break;
                // the labels' own words do not take part, nor do lanes without one
                const uint32_t near = __ballot_sync(0xffffffffu, label >= word0 && label < word0 + 32 && label < P.V);
                if (near != 0u) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const long long l = __shfl_sync(0xffffffffu, label, j);
                        if ((near >> j & 1u) != 0u && l == word0 + lane && is_word) {
                            P.label_logit[first + j] = v[j];
                            v[j] = -INFINITY;
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    if (!is_word) v[j] = -INFINITY;
                    e[j] = v[j];
                }
                const float most = over_lanes(e, [](float a, float b) { return fmaxf(a, b); });
                const float under = most == -INFINITY ? 0.0f : most * kLog2e;
#pragma unroll
                for (int j = 0; j < 32; ++j) e[j] = exp2_fast(fmaf(v[j], kLog2e, -__shfl_sync(0xffffffffu, under, j)));
                const float sum = over_lanes(e, [](float a, float b) { return a + b; });
                if (most != -INFINITY) {
                    const float more = fmaxf(top, under);
                    total = total * exp2_fast(top - more) + sum * exp2_fast(under - more);
                    top = more;
                } else {
                    total += sum;                     // (zero, or NaN)
                }
            }
            parts[(ch * 4 + q) * 32 + lane] = make_float2(top, total);
        } else {
            for (int u = pair; u < units && !failed; u += pairs) {
                const int t = tile_of(u), tn = t / P.tiles_m, row = t % P.tiles_m * kTile + (int)crank * 128 + q * 32 + lane;
                const bool mine = row < P.M;
                int kb0;
                const int segments = segments_of(blocks_of(u, &kb0));
                __syncwarp();
                // what belongs to the token is asked for ahead of the tile
                float lift = -INFINITY, scale = 1.0f;
                int label = -1;
                if (mine) {
                    if (KIND == kExponentials && !P.first) lift = P.lift[row];
                    if (KIND != kGradient) {
                        const long long y = P.labels[row];
                        label = y >= 0 && y < P.V ? (int)y : -1;
                    }
                    if (KIND == kGradient && !P.first) scale = P.scale[row];
                }
                uint32_t v[4][32];
                if (KIND != kGradient || segments > 0) {
                    drain(c_first * 32, [&](uint32_t from) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) ptx::tmem_ld_32x32(from + (uint32_t)c * 32u, v[c]);
                        ptx::tmem_ld_wait();
                    });
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[c][j] = 0u;
                }
                if constexpr (KIND != kGradient)
                    for (int g = 1; g < segments && !failed; ++g)
                        drain(c_first * 32, [&](uint32_t from) {
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                uint32_t w[32];
                                ptx::tmem_ld_32x32(from + (uint32_t)c * 32u, w);
                                ptx::tmem_ld_wait();
#pragma unroll
                                for (int j = 0; j < 32; ++j) v[c][j] = __float_as_uint(__uint_as_float(v[c][j]) + __uint_as_float(w[j]));
                            }
                        });
                if (failed) break;
                const int n0 = tn * P.width + c_first * 32;      // the first column, in the piece
                if constexpr (KIND == kGradient) {
                    const bool is_whole = u < P.whole, ends = is_whole && P.last != 0;
                    float* out = is_whole ? P.out + (size_t)row * P.N + n0
                                          : P.parts + (size_t)(u - P.whole) * (kTile * kTile) + ((int)crank * 128 + q * 32 + lane) * kTile + c_first * 32;
                    Factors f = {0.0f, 0.0f, 1.0f, nullptr};
                    if (ends && mine) f = factors_of(P.end, row);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (!mine || n0 + c * 32 + j * 8 >= P.N) continue;
                            float* at = out + c * 32 + j * 8;
                            uint32_t* w = &v[c][j * 8];
                            if (!P.first) {
                                const float4 a = reinterpret_cast<const float4*>(at)[0], b = reinterpret_cast<const float4*>(at)[1];
                                const float old[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                                for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(fmaf(old[k], scale, __uint_as_float(w[k])));
                            }
                            if (ends) {
                                float o[8];
#pragma unroll
                                for (int k = 0; k < 8; ++k) o[k] = __uint_as_float(w[k]);
                                const int k0 = n0 + c * 32 + j * 8;
                                *reinterpret_cast<uint4*>(P.end.dX + (size_t)row * P.N + k0) = end_of(f, o, k0);
                            } else {
                                ptx::st_global_v8(at, w);
                            }
                        }
                    }
                } else {
                    // The label's word and those past the last do not take part, nor do columns that a narrower tile does not have.  Looked for 32 columns at a time: a column by itself takes three
                    // instructions, for a warp's 128 as many as all the rest (every tile but full ones, and a tenth of those: 1664 tokens, 38593 words, 512 features 115 -> 56 us).
                    const int at = label - (P.v0 + n0), last = P.V - (P.v0 + n0);
                    float most = -INFINITY, own = 0.0f, sum = 0.0f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (c >= c_count) continue;
                        if (__any_sync(0xffffffffu, (uint32_t)(at - c * 32) < 32u || last < c * 32 + 32)) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                if (c * 32 + j == at) own = __uint_as_float(v[c][j]);
                                if (c * 32 + j == at || c * 32 + j >= last) v[c][j] = 0xff800000u;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) most = fmaxf(most, __uint_as_float(v[c][j]));
                    }
                    if (at >= 0 && at < c_count * 32) P.label_logit[row] = own;
                    // under which the exponentials are taken, in octaves: the largest, or the token's lift
                    const float octaves = most * kLog2e;
                    float under = 0.0f;
                    if (KIND == kSums) {
                        if (most != -INFINITY) under = octaves;
                    } else {
                        if (lift != -INFINITY) under = lift;
                        if (octaves - under > kHeadroom || (lift == -INFINITY && octaves - under < -kHeadroom)) under = most == -INFINITY ? under : ceilf(octaves);
                    }
                    float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (c >= c_count) continue;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const float y = exp2_fast(fmaf(__uint_as_float(v[c][j]), kLog2e, -under));
                            v[c][j] = __float_as_uint(y);
                            part[j & 3] += y;
                        }
                    }
                    sum = (part[0] + part[1]) + (part[2] + part[3]);
                    if (mine) {
                        P.stats[(size_t)(tn * 2 + ch) * P.M + row] = make_float2(most == -INFINITY ? -INFINITY : under, sum);
                        if constexpr (KIND == kExponentials) {
                            uint16_t* e = P.e + (size_t)row * P.ld_e + n0;
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                if (c >= c_count) continue;
                                uint32_t w[16];
#pragma unroll
                                for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(__uint_as_float(v[c][2 * j]), __uint_as_float(v[c][2 * j + 1]));
                                ptx::st_global_v8(e + c * 32, w);
                                ptx::st_global_v8(e + c * 32 + 16, w + 8);
                            }
                        }
                    }
                }
            }
        }
        if (failed) bars->abort = 1u;
    }

    if (failed) {
        atomicExch(P.status, (uint32_t)LOWRA_ERR_TIMEOUT);
        ptx::st_relaxed_cluster(ptx::map_to_cta(ptx::smem_u32(&bars->abort), crank ^ 1u), 1u);
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
    if constexpr (KIND == kFew) {
        const int token = threadIdx.x;
        if (token < P.M) {                            // (up to 64; after a failure the numbers mean nothing, and the status says so)
            float2 all = parts[token / 32 * 128 + token % 32];
            for (int w = 1; w < 4; ++w) {
                const float2 part = parts[token / 32 * 128 + w * 32 + token % 32];
                if (part.x != -INFINITY) {
                    const float more = fmaxf(all.x, part.x);
                    all = make_float2(more, all.y * exp2_fast(all.x - more) + part.y * exp2_fast(part.x - more));
                } else {
                    all.y += part.y;
                }
            }
            P.stats[(size_t)blockIdx.x * P.M + token] = all;
        }
    }
    ptx::cluster_sync();   // the peer's copies, arrivals and MMAs no longer touch this CTA
    if (*abort_flag != 0u) {
        // somebody gave up, and roles that did not wait may have left copies or MMAs in flight (the same answer in both CTAs)
        if (threadIdx.x == 0) {
            const uint64_t t0 = ptx::globaltimer_ns();
            while (ptx::globaltimer_ns() - t0 < kGrace) __nanosleep(1000);
        }
        __syncthreads();
        ptx::cluster_sync();
    }
    if (warp == 1) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc_pair(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------------ the tokens' own numbers
// A token's halves of tiles, or of a CTA's words, (octaves that the exponentials were taken under, sum of them) each, joined: eight tokens to a CTA, 32 threads to a token, eight of their loads under way at once.
// (Halves without a word: minus infinity and zero.)  Empty in the end where no half had one.
constexpr int kTokens = 8, kLanes = 32;
struct Joined {
    float top, sum, low;      // the largest of the octaves, the sum under it, the least
    __device__ __forceinline__ void add(float2 s) {
        if (s.x != -INFINITY && s.x != top) {
            const float more = fmaxf(top, s.x);
            sum *= exp2f(top - more);
            s.y *= exp2f(s.x - more);
            top = more;
        }
        if (s.x != -INFINITY) low = fminf(low, s.x);
        sum += s.y;
    }
    // the token's, in the threads of the first warp (all of which are there)
    __device__ __forceinline__ void collect(const float2* stats, int count, int M, int m, float (*shared)[kTokens][3]) {
        const int lane = (int)threadIdx.x / kTokens;
        if (m < M)
            for (int i0 = lane; i0 < count; i0 += 8 * kLanes) {
                float2 s[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) s[k] = i0 + k * kLanes < count ? stats[(size_t)(i0 + k * kLanes) * M + m] : make_float2(-INFINITY, 0.0f);
#pragma unroll
                for (int k = 0; k < 8; ++k) add(s[k]);
            }
        auto join = [&](float other_top, float other_sum, float other_low) {
            low = fminf(low, other_low);
            add(make_float2(other_top, other_sum));
        };
#pragma unroll
        for (int d = 8; d < 32; d *= 2) {
            const float a = __shfl_xor_sync(0xffffffffu, top, d), b = __shfl_xor_sync(0xffffffffu, sum, d), c = __shfl_xor_sync(0xffffffffu, low, d);
            join(a, b, c);
        }
        const int warp = (int)threadIdx.x >> 5, token = (int)threadIdx.x % kTokens;
        if ((threadIdx.x & 31) < kTokens) {
            shared[warp][token][0] = top;
            shared[warp][token][1] = sum;
            shared[warp][token][2] = low;
        }
        __syncthreads();
        if (warp == 0)
            for (int w = 1; w < kTokens * kLanes / 32; ++w) join(shared[w][token][0], shared[w][token][1], shared[w][token][2]);
    }
};

// -log of the label's share, from its logit and the sum of the others' exponentials, taken under `top` octaves (minus infinity: none has one).  `top` is the largest of the others' or, with a gradient, the
// token's lift, from which both may be far: so the label is set against the others' sum, and not against `top`, whose octaves cancel in fp64.  Neither way has a difference of large numbers: with the
// larger share of the two the loss is log(1 + their ratio), else both of its terms are positive.
__device__ __forceinline__ float loss_of(float logit, float top, float sum) {
    if (!(logit < INFINITY) || (top == -INFINITY && logit == -INFINITY)) return NAN;
    if (top == -INFINITY) return sum;                         // (zero, or NaN)
    int octaves = 0;
    const float others = 2.0f * frexpf(sum, &octaves);        // sum = others 2^(octaves - 1), others in [1, 2)
    const float over = (float)((double)logit * (double)kLog2e - ((double)top + (double)(octaves - 1)));
    return over >= 0.0f ? log1pf(others * exp2f(-over)) : logf(others + exp2f(over)) - over * kLn2;
}

// Loss without a gradient.
__global__ void __launch_bounds__(kTokens * kLanes) loss_kernel(const float2* stats, int count, const float* logit, const long long* labels, int M, int V, long long ignore, float* loss) {
    __shared__ float shared[kTokens * kLanes / 32][kTokens][3];
    pdl_enter();
    const int m = (int)blockIdx.x * kTokens + (int)threadIdx.x % kTokens;
    Joined all = {-INFINITY, 0.0f, INFINITY};
    all.collect(stats, count, M, m, shared);
    if (threadIdx.x >= kTokens || m >= M) return;
    const long long y = labels[m];
    if (y == ignore || y < 0 || y >= V) {
        loss[m] = y == ignore ? 0.0f : NAN;
        return;
    }
    loss[m] = loss_of(logit[m], all.top, all.sum);
}

// Between a piece's two products: the largest lift of each token, its sum, the factor for O; exponentials that were formed under a smaller lift are brought to it.
__global__ void __launch_bounds__(kTokens * kLanes) lift_kernel(const float2* stats, int count, int M, int width, int first, uint16_t* e, long long ld_e, CeRows R) {
    __shared__ float shared[kTokens * kLanes / 32][kTokens][3];
    __shared__ float common[kTokens];
    __shared__ int some;
    pdl_enter();
    const int m0 = (int)blockIdx.x * kTokens, m = m0 + (int)threadIdx.x % kTokens;
    const float before = m < M && !first ? R.lift[m] : -INFINITY;
    Joined all = {before, 0.0f, INFINITY};
    all.collect(stats, count, M, m, shared);
    if (threadIdx.x < 32) {
        if (threadIdx.x < kTokens && m < M) {
            const float scale = before == -INFINITY ? 0.0f : exp2f(before - all.top);
            R.sum[m] = first ? all.sum : R.sum[m] * scale + all.sum;
            R.scale[m] = scale;
            R.lift[m] = all.top;
        }
        if (threadIdx.x < kTokens) common[threadIdx.x] = all.top;
        const bool unequal = __any_sync(0xffffffffu, threadIdx.x < kTokens && all.low < all.top);
        if (threadIdx.x == 0) some = unequal;
    }
    __syncthreads();
    if (some == 0) return;
    const int chunks = width / 32, wide = (chunks + 1) / 2 * 32, narrow = chunks / 2 * 32, lane = threadIdx.x & 31;
    for (int r = 0; r < kTokens && m0 + r < M; ++r) {
        const int row = m0 + r;
        for (int i = (int)threadIdx.x >> 5; i < count; i += kTokens * kLanes / 32) {
            const float under = stats[(size_t)i * M + row].x;
            if (under == -INFINITY || under == common[r]) continue;
            const float by = exp2f(under - common[r]);
            uint16_t* at = e + (size_t)row * ld_e + (size_t)(i >> 1) * width + (i & 1 ? wide : 0);
            for (int j = lane; j < (i & 1 ? narrow : wide); j += 32) at[j] = (uint16_t)pack_bf16x2(__uint_as_float((uint32_t)at[j] << 16) * by, 0.0f);
        }
    }
}

// The losses, and dX where the contraction was cut: the parts in their order, eight features to a thread.
__global__ void __launch_bounds__(256) finish_kernel(const CeEnd E, const float* parts, int whole, int rest, int splits, int tiles_m, int M, float* loss) {
    pdl_enter();
    const long long step = (long long)gridDim.x * 256, vectors = (long long)rest * kTile * (kTile / 8);
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < vectors; i += step) {
        const int r = (int)(i / (kTile * kTile / 8)), in = (int)(i % (kTile * kTile / 8)), t = whole + r;
        const int m = t % tiles_m * kTile + in / (kTile / 8), k = t / tiles_m * kTile + in % (kTile / 8) * 8;
        if (m >= M || k >= E.K) continue;
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) {
            const float4* from = reinterpret_cast<const float4*>(parts + ((size_t)s * rest + r) * (kTile * kTile) + (size_t)in * 8);
            const float4 p = __ldcs(from), q = __ldcs(from + 1);
            o[0] += p.x; o[1] += p.y; o[2] += p.z; o[3] += p.w; o[4] += q.x; o[5] += q.y; o[6] += q.z; o[7] += q.w;
        }
        *reinterpret_cast<uint4*>(E.dX + (size_t)m * E.K + k) = end_of(factors_of(E, m), o, k);
    }
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < M; i += step) {
        const int m = (int)i;
        const long long y = E.labels[m];
        loss[m] = y == E.ignore ? 0.0f : y >= 0 && y < E.V ? loss_of(E.rows.logit[m], E.rows.lift[m], E.rows.sum[m]) : NAN;
    }
}

// ------------------------------------------------------------------------------------------------ host
constexpr int kMostTokens = 4096;                          // of a pass; more go in several passes
constexpr size_t kPieceBytes = (size_t)128 << 20;          // of a piece's exponentials
constexpr int kMostV = 1 << 24, kMostK = 1 << 16, kMostM = 1 << 30, kMostSplits = 64;
constexpr int kPairs = kNumSMs / 2;

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// How a call is cut: by rules on its sizes alone, so that the scratch can be asked for beforehand.
struct CePlan {
    int passes, tokens;                 // passes over the tokens, tokens of one
    int width, tiles;                   // columns of a tile of logits (few tokens: rows), and tiles of a piece
    int few;                            // few tokens, no gradient: columns of the tile
    int pieces, piece;                  // pieces of the vocabulary, their words (the last may have fewer)
    size_t off_rows, off_stats, off_e, off_out, off_parts, total;
};
// The gradient's tiles: as many whole ones as fill all pairs, the contraction of the rest cut into parts that do.
struct CeCut {
    int whole, rest, splits;
};
CeCut cut_of(int tokens, int K, int blocks) {
    const int tiles = ((tokens + kTile - 1) / kTile) * ((K + kTile - 1) / kTile), rest = tiles % kPairs;
    CeCut c = {tiles - rest, rest, 1};
    // rounds of blocks, six more for filling and draining, and what a part costs in memory and at the end (1.5 blocks' time for each of a round)
    double least = -1.0;
    for (int s = 1; rest > 0 && s <= kMostSplits && s <= blocks && (s == 1 || rest * s <= 2 * kPairs); ++s) {
        const double cost = (double)((rest * s + kPairs - 1) / kPairs) * ((blocks + s - 1) / s + 6) + 1.5 * s * rest / kPairs;
        if (least < 0.0 || cost < least) { least = cost; c.splits = s; }
    }
    if (c.splits == 1) c = {tiles, 0, 1};
    return c;
}
int blocks_of_piece(int words) { return (words + kDepth - 1) / kDepth; }
CePlan plan_of(int M, int V, int K, bool grad) {
    CePlan p;
    p.passes = (M + kMostTokens - 1) / kMostTokens;
    p.tokens = (M + p.passes - 1) / p.passes;
    p.tokens = p.passes > 1 ? (p.tokens + kTile - 1) / kTile * kTile : p.tokens;
    const int tiles_m = (p.tokens + kTile - 1) / kTile;
    // pieces as few as the scratch allows, of equal length
    long long most = grad ? (long long)(kPieceBytes / 2 / (size_t)p.tokens) / kTile * kTile : V;
    p.pieces = (int)((V + most - 1) / most);
    const int words = (V + p.pieces - 1) / p.pieces;
    // the width that the pairs' last round wastes the least with (a round costs its tiles' columns and, for filling and draining, some 16 more)
    long best = -1;
    p.width = kTile;
    for (int width = kTile; width >= 128; width -= 32) {
        const long tiles = (words + width - 1) / width, rounds = (tiles * tiles_m + kPairs - 1) / kPairs, cost = rounds * (width + 16);
        if (best < 0 || cost < best) { best = cost; p.width = width; }
    }
    p.tiles = (words + p.width - 1) / p.width;
    p.piece = p.pieces > 1 ? p.tiles * p.width : V;
    p.pieces = (V + p.piece - 1) / p.piece;
    p.few = !grad && M <= kFewTokens ? (M + 31) / 32 * 32 : 0;
    p.off_rows = 256;
    p.off_stats = p.off_rows + 4 * up256((size_t)p.tokens * 4);
    p.off_e = p.off_stats + up256((size_t)(p.few ? 2 * kPairs : 2 * p.tiles) * p.tokens * 8);
    p.off_out = p.off_e + (grad ? up256((size_t)p.tokens * p.tiles * p.width * 2) : 0);
    p.off_parts = p.off_out + (grad && p.pieces > 1 ? up256((size_t)p.tokens * K * 4) : 0);
    size_t parts = 0;
    auto room = [&](int m) {
        const CeCut c = cut_of(m, K, blocks_of_piece(p.piece));
        const size_t bytes = (size_t)c.rest * c.splits * kTile * kTile * 4;
        if (bytes > parts) parts = bytes;
    };
    if (grad) room(p.tokens);
    const int left = M - (p.passes - 1) * p.tokens;      // (the last pass may have fewer tokens)
    if (grad && left > 0) room(left);
    p.total = p.off_parts + parts;
    return p;
}

std::atomic<int> g_dropping{0};     // diagnostic: calls to come, times four, and which of their products (1: the logits', 2: the gradient's) load no more than a first block

bool good_sizes(int M, int V, int K) { return M >= 1 && M <= kMostM && V >= 1 && V <= kMostV && K >= 64 && K <= kMostK && K % 8 == 0; }

// Pairs that a launch has: a unit each at least.
int pairs_of(const CeParams& P) {
    const int units = P.whole + (P.tiles_m * P.tiles_n - P.whole) * P.splits, sms = device_sm_count();
    return units < sms / 2 ? units : sms / 2;
}
template <int KIND>
lowra_status launch_product(CeParams& P, cudaStream_t stream) {
    static SmemLimit limit = {};
    if (ensure_smem_limit(reinterpret_cast<const void*>(product_kernel<KIND>), kSmem<KIND>, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
    // (the warps' shares of the registers were added up for a kernel of this size)
    static std::atomic<int> registers{0};
    if (registers.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes of;
        if (cudaFuncGetAttributes(&of, product_kernel<KIND>) != cudaSuccess) return LOWRA_ERR_CUDA;
        registers.store(of.numRegs, std::memory_order_relaxed);
    }
    const int pairs = pairs_of(P);
    if (pairs < 1 || registers.load(std::memory_order_relaxed) != kLaunchRegisters) return LOWRA_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)pairs * 2, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = kSmem<KIND>;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, product_kernel<KIND>, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}

}  // namespace
}  // namespace lowra

extern "C" lowra_status lowra_diag_drop_tiles(int32_t calls, int32_t products) {
    if (calls < 0 || calls > 1000 || products < 1 || products > 3) return LOWRA_ERR_SHAPE;
    lowra::g_dropping.store(calls > 0 ? calls * 4 + products : 0, std::memory_order_relaxed);
    return LOWRA_OK;
}

extern "C" size_t lowra_cross_entropy_workspace_bytes(int32_t M, int32_t V, int32_t K, int32_t grad) {
    using namespace lowra;
    return good_sizes(M, V, K) ? plan_of(M, V, K, grad != 0).total : 0;
}

extern "C" lowra_status lowra_cross_entropy(const uint16_t* X_dev, const uint16_t* W_dev, const int64_t* labels_dev, const float* weights_dev, int32_t M, int32_t V, int32_t K,
                                            int64_t ignore_index, float scale, float* loss_dev, uint16_t* dX_dev, void* workspace_dev, size_t workspace_bytes, void* stream_v) {
    using namespace lowra;
    if (!X_dev || !W_dev || !labels_dev || !loss_dev || !workspace_dev) return LOWRA_ERR_NULL;
    if (!good_sizes(M, V, K)) return LOWRA_ERR_SHAPE;
    if (!aligned16(X_dev) || !aligned16(W_dev) || !aligned16(labels_dev) || !aligned16(weights_dev) || !aligned16(loss_dev) || !aligned16(dX_dev)) return LOWRA_ERR_ALIGN;
    const CePlan p = plan_of(M, V, K, dX_dev != nullptr);
    if (workspace_bytes < p.total || (reinterpret_cast<uintptr_t>(workspace_dev) & 255u) != 0) return LOWRA_ERR_WORKSPACE;
    const Span read[4] = {{X_dev, (size_t)M * K * 2}, {W_dev, (size_t)V * K * 2}, {labels_dev, (size_t)M * 8}, {weights_dev, (size_t)M * 4}};
    const Span written[3] = {{loss_dev, (size_t)M * 4}, {dX_dev, (size_t)M * K * 2}, {workspace_dev, p.total}};
    for (int i = 0; i < 3; ++i) {
        for (const Span& r : read)
            if (overlap(written[i], r)) return LOWRA_ERR_SHAPE;
        for (int j = i + 1; j < 3; ++j)
            if (overlap(written[i], written[j])) return LOWRA_ERR_SHAPE;
    }
    lowra_status st = check_device();
    if (st != LOWRA_OK) return st;
    int dropping = g_dropping.load(std::memory_order_relaxed);
    while (dropping >= 4 && !g_dropping.compare_exchange_weak(dropping, dropping - 4, std::memory_order_relaxed)) {}
    if (dropping < 4) dropping = 0;
    cudaStream_t stream = (cudaStream_t)stream_v;
    unsigned char* ws = static_cast<unsigned char*>(workspace_dev);
    uint32_t* status = reinterpret_cast<uint32_t*>(ws);
    const size_t row = up256((size_t)p.tokens * 4) / 4;
    float* rows = reinterpret_cast<float*>(ws + p.off_rows);
    const CeRows R = {rows, rows + row, rows + 2 * row, rows + 3 * row};
    float2* stats = reinterpret_cast<float2*>(ws + p.off_stats);
    uint16_t* e = reinterpret_cast<uint16_t*>(ws + p.off_e);
    float *O = reinterpret_cast<float*>(ws + p.off_out), *parts = reinterpret_cast<float*>(ws + p.off_parts);
    const long long ld_e = (long long)p.tiles * p.width;
    for (int pass = 0; pass < p.passes; ++pass) {
        const long long m0 = (long long)pass * p.tokens;
        const int m = (int)(M - m0 < p.tokens ? M - m0 : p.tokens);
        if (m < 1) break;
        const uint16_t* X = X_dev + m0 * K;
        const long long* labels = reinterpret_cast<const long long*>(labels_dev) + m0;
        const float* weights = weights_dev ? weights_dev + m0 : nullptr;
        CeParams P = {};
        P.M = m;
        P.V = V;
        P.width = p.width;
        P.tiles_m = (m + kTile - 1) / kTile;
        P.splits = 1;
        P.blocks = (K + kDepth - 1) / kDepth;
        P.labels = labels;
        P.lift = R.lift;
        P.label_logit = R.logit;
        P.stats = stats;
        P.e = e;
        P.ld_e = ld_e;
        P.status = status;
        P.wait_ns = wait_limit_ns();
        P.withheld = dropping & 1;
        // Up to 128 tokens: the second CTA of a pair has none, and the first loads its own only.  What the tile's other rows hold of earlier kernels comes out in rows that are not looked at.
        // (35006 words, 3672 features, us with all 128 rows of either CTA, past the end filled with zeros, and so: 157, 117 for 12 tokens)
        P.a_halves = m <= 128 ? 1 : 2;
        P.a_rows = m < 128 ? (m + 7) / 8 * 8 : 128;
        if (!make_map(&P.a, X, (uint64_t)m, (uint64_t)K, (uint64_t)K, (uint32_t)P.a_rows) || !make_map(&P.b, W_dev, (uint64_t)V, (uint64_t)K, (uint64_t)K, (uint32_t)p.width / 2)) return LOWRA_ERR_CUDA;
        if (!dX_dev) {
            P.N = V;
            P.tiles_n = p.tiles;
            P.whole = P.tiles_m * P.tiles_n;
            P.clear_status = pass == 0;
            if (p.few) {
                P.columns = p.few;
                if (!make_map(&P.a, W_dev, (uint64_t)V, (uint64_t)K, (uint64_t)K, (uint32_t)p.width / 2) || !make_map(&P.b, X, (uint64_t)m, (uint64_t)K, (uint64_t)K, (uint32_t)p.few / 2))
                    return LOWRA_ERR_CUDA;
            }
            if ((st = p.few ? launch_product<kFew>(P, stream) : launch_product<kSums>(P, stream)) != LOWRA_OK) return st;
            if (launch_pdl(loss_kernel, (unsigned)((m + kTokens - 1) / kTokens), kTokens * kLanes, stream, (const float2*)stats, p.few ? 2 * pairs_of(P) : 2 * p.tiles, (const float*)R.logit, labels, m, (int)V, (long long)ignore_index,
                           loss_dev + m0) != cudaSuccess)
                return LOWRA_ERR_CUDA;
            continue;
        }
        CeParams G = P;
        G.N = K;
        G.width = kTile;
        G.withheld = dropping >> 1 & 1;
        G.tiles_n = (K + kTile - 1) / kTile;
        const CeCut cut = cut_of(m, K, blocks_of_piece(p.piece));
        G.whole = cut.whole;
        G.splits = cut.splits;
        G.scale = R.scale;
        G.out = O;
        G.parts = parts;
        G.end = CeEnd{R, W_dev, labels, weights, dX_dev + m0 * K, (long long)ignore_index, (int)V, (int)K, scale};
        if (!make_map(&G.b, W_dev, (uint64_t)V, (uint64_t)K, (uint64_t)K, 64)) return LOWRA_ERR_CUDA;
        for (int c = 0; c < p.pieces; ++c) {
            P.v0 = G.v0 = c * p.piece;
            P.N = V - P.v0 < p.piece ? V - P.v0 : p.piece;
            P.tiles_n = (P.N + p.width - 1) / p.width;
            P.whole = P.tiles_m * P.tiles_n;
            G.blocks = blocks_of_piece(P.N);
            G.last = c + 1 == p.pieces;
            P.first = G.first = c == 0;
            P.clear_status = pass == 0 && c == 0;
            // (columns that the first product does not write, in a last block that is not full, are past the end)
            if (!make_map(&G.a, e, (uint64_t)m, (uint64_t)P.tiles_n * p.width, (uint64_t)ld_e, (uint32_t)P.a_rows)) return LOWRA_ERR_CUDA;
            if ((st = launch_product<kExponentials>(P, stream)) != LOWRA_OK) return st;
            if (launch_pdl(lift_kernel, (unsigned)((m + kTokens - 1) / kTokens), kTokens * kLanes, stream, (const float2*)stats, 2 * P.tiles_n, m, p.width, P.first, e, ld_e, R) != cudaSuccess) return LOWRA_ERR_CUDA;
            if ((st = launch_product<kGradient>(G, stream)) != LOWRA_OK) return st;
        }
        long long ctas = ((long long)cut.rest * (kTile * kTile / 8) + 255) / 256;
        if (ctas < (m + 255) / 256) ctas = (m + 255) / 256;
        if (launch_pdl(finish_kernel, (unsigned)(ctas < 8 * kNumSMs ? ctas : 8 * kNumSMs), 256, stream, G.end, (const float*)parts, cut.whole, cut.rest, cut.splits, P.tiles_m, m, loss_dev + m0) !=
            cudaSuccess)
            return LOWRA_ERR_CUDA;
    }
    return LOWRA_OK;
}
