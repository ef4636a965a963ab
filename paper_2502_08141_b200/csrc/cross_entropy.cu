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
// adds (losses over 4096 features: error against fp64 2.0e-6 -> 5e-7).
//
// The products: CTA pairs (clusters of two) walk over tiles of 256 tokens x up to 256 words (features), tcgen05.mma with cta_group::2, both operands by TMA, 64 contraction indices
// (32 KB a CTA) to a stage, six stages; two accumulators in turn, so the epilogue's eight warps work on one tile while the next is formed.
// warp 0 = TMA, 1 = MMA (of the CTA of rank 0) and TMEM, 4-11 = epilogue.  The 128 columns that an epilogue's thread holds, and 32 more on their way, do not fit into the 168 registers that
// twelve warps get: the first four give some to the others.  All waits are bounded (lowra_set_wait_limit); no CTA waits for another cluster.
#include <atomic>

#include "gemm_params.cuh"
#include "ptx.cuh"

namespace lowra {

namespace {

constexpr int kTile = 256;                        // tokens, and at most so many words or features, of a pair's tile
constexpr int kStages = 6, kDepth = 64;           // contraction indices of a stage
constexpr uint32_t kHalfBytes = 128 * kDepth * 2, kStageBytes = 2 * kHalfBytes;
constexpr int kThreads = 384, kEpilogue = 8, kFirstEpilogue = 4;      // threads; epilogue warps, behind four others
constexpr int kLaunchRegisters = 168, kFewRegisters = 40, kManyRegisters = 232;   // a thread: at the launch, of the first four warps, of the others
static_assert(128 * kFewRegisters + 256 * kManyRegisters <= kThreads * kLaunchRegisters, "what the others take, the first four have given (a larger share would be waited for without end)");
constexpr uint32_t kSmem = kStages * kStageBytes + 1024;
constexpr uint64_t kGrace = 50ull * 1000ull;      // after a failure: time for copies and MMAs still in flight to land
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kHeadroom = 64.0f;                // octaves that the largest exponentials may be from one
constexpr int kSegment = 16;                      // contraction blocks of a logit that are added up in the tensor memory
constexpr int kSums = 0, kExponentials = 1, kGradient = 2;

struct CeBarriers {
    uint64_t full[kStages], empty[kStages];
    uint64_t tmem_full[2], tmem_empty[2];
    uint32_t tmem_base, abort;
};
static_assert(sizeof(CeBarriers) <= 1024, "barrier block");

struct CeParams {
    CUtensorMap a, b;                             // X, or the exponentials [M, piece];  W as [V, K], in boxes of words or of 64 words x 64 features
    int M, N, V;                                  // tokens; words of the piece or features; words in all
    int v0;                                       // the piece's first word
    int width, tiles_m, tiles_n, splits;          // columns of a tile; tiles; (gradient) parts of the contraction
    int blocks;                                   // contraction blocks in all
    int first;                                    // the first piece: lift and O have no value yet
    const long long* labels;
    const float* lift;                            // (exponentials) a token's lift so far, in octaves
    float* label_logit;                           // l_y (out)
    float2* stats;                                // [2 tiles_n][M]: of half a tile, (largest in octaves, or lift; sum)
    uint16_t* e;                                  // [M, ld_e]
    long long ld_e;
    const float* scale;                           // (gradient) 2^-(lift added by the piece)
    float* out;                                   // (gradient) O [splits][M, N]
    uint32_t* status;
    unsigned long long wait_ns;
    int clear_status;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int KIND>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ CeParams P) {
    extern __shared__ __align__(1024) unsigned char smem[];
    CeBarriers* bars = reinterpret_cast<CeBarriers*>(smem + kStages * kStageBytes);
    volatile uint32_t* abort_flag = &bars->abort;
    if ((ptx::smem_u32(smem) & 1023u) != 0u) {      // never seen; without it the operand descriptors would be wrong
        if (threadIdx.x == 0) atomicExch(P.status, (uint32_t)LOWRA_ERR_CUDA);
        return;
    }
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t crank = blockIdx.x & 1u;
    const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
    const int tiles = P.tiles_m * P.tiles_n, units = tiles * P.splits;
    const bool mn = KIND == kGradient;              // W's features are the contiguous ones of its tiles

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { ptx::mbar_init(&bars->full[s], 1); ptx::mbar_init(&bars->empty[s], 1); }
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

    // Unit u: tokens fastest, so that the pairs at work share the words or features of their tiles; a part of the contraction after the other.
    auto blocks_of = [&](int u, int* kb0) {
        const int s = u / tiles;
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
        const uint32_t b_bytes = (uint32_t)P.width * kDepth;      // half the tile's columns x 64 x 2 bytes
        int s = 0;
        uint32_t ph = 0;
        for (int u = pair; u < units && !failed; u += pairs) {
            const int t = u % tiles, m0 = t % P.tiles_m * kTile + (int)crank * 128, n0 = t / P.tiles_m * P.width + (int)crank * (P.width / 2);
            int kb0;
            const int n = blocks_of(u, &kb0);
            for (int kb = kb0; kb < kb0 + n; ++kb) {
                if (!ptx::mbar_wait_lanes(&bars->empty[s], ph ^ 1u, abort_flag, P.wait_ns)) { failed = true; break; }
                unsigned char* a_s = smem + s * kStageBytes;
                const uint32_t bar = full0 + (uint32_t)s * 8u;
                if (leader) {
                    if (crank == 0u) ptx::mbar_arrive_expect_tx(&bars->full[s], 2u * (kHalfBytes + b_bytes));
                    ptx::tma_load_2d_pair(a_s, &P.a, kb * kDepth, m0, bar);
                    if (mn) {
                        ptx::tma_load_2d_pair(a_s + kHalfBytes, &P.b, n0, P.v0 + kb * kDepth, bar);
                        ptx::tma_load_2d_pair(a_s + kHalfBytes + 8192, &P.b, n0 + 64, P.v0 + kb * kDepth, bar);
                    } else {
                        ptx::tma_load_2d_pair(a_s + kHalfBytes, &P.b, kb * kDepth, P.v0 + n0, bar);
                    }
                }
                __syncwarp();
                if (++s == kStages) { s = 0; ph ^= 1u; }
            }
        }
        if (failed) bars->abort = 1u;
    } else if (warp == 1) {
        if (crank == 0u) {
            const bool leader = ptx::elect_one();
            const uint32_t idesc = ptx::umma_idesc_bf16(kTile, P.width) | (mn ? 1u << 16 : 0u), b_step = mn ? 128u : 2u;
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
                        const uint64_t a = a0 + (uint64_t)s * (kStageBytes >> 4), b = b0 + (uint64_t)s * (kStageBytes >> 4);
                        const int here = s;
                        if (++s == kStages) { s = 0; ph ^= 1u; }
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
        for (int u = pair; u < units && !failed; u += pairs) {
            const int t = u % tiles, tn = t / P.tiles_m, row = t % P.tiles_m * kTile + (int)crank * 128 + q * 32 + lane;
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
            // the next accumulator's columns: `take` reads them, then it is free
            auto drain = [&](auto take) {
                const uint32_t acc = (uint32_t)i & 1u;
                if (!ptx::mbar_wait_warp(&bars->tmem_full[acc], ((uint32_t)i >> 1) & 1u, abort_flag, P.wait_ns)) { failed = true; return; }
                ptx::tc_fence_after();
                take(tmem_base + acc * kTile + ((uint32_t)(q * 32) << 16) + (uint32_t)c_first * 32u);
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (crank == 0u) ptx::mbar_arrive(&bars->tmem_empty[acc]);
                    else ptx::mbar_arrive_cluster(empty0 + acc * 8u);
                }
                ++i;
            };
            if (KIND != kGradient || segments > 0) {
                drain([&](uint32_t from) {
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
                    drain([&](uint32_t from) {
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
                float* out = P.out + (size_t)(u / tiles) * P.M * P.N + (size_t)row * P.N + n0;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (!mine || c >= c_count || n0 + c * 32 + j * 8 >= P.N) continue;
                        float* at = out + c * 32 + j * 8;
                        uint32_t* w = &v[c][j * 8];
                        if (!P.first) {
                            const float4 a = reinterpret_cast<const float4*>(at)[0], b = reinterpret_cast<const float4*>(at)[1];
                            const float old[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                            for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(fmaf(old[k], scale, __uint_as_float(w[k])));
                        }
                        ptx::st_global_v8(at, w);
                    }
                }
            } else {
                // the label's word and those past the last do not take part, nor do columns that a narrower tile does not have
                const int at = label - (P.v0 + n0), last = min(P.V - (P.v0 + n0), c_count * 32);
                if (__any_sync(0xffffffffu, (at >= 0 && at < last) || last < 128)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            if (c * 32 + j == at && at < last) P.label_logit[row] = __uint_as_float(v[c][j]);
                            if (c * 32 + j == at || c * 32 + j >= last) v[c][j] = 0xff800000u;
                        }
                }
                float most = -INFINITY, sum = 0.0f;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int j = 0; j < 32; ++j) most = fmaxf(most, __uint_as_float(v[c][j]));
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
        if (failed) bars->abort = 1u;
    }

    if (failed) {
        atomicExch(P.status, (uint32_t)LOWRA_ERR_TIMEOUT);
        ptx::st_relaxed_cluster(ptx::map_to_cta(ptx::smem_u32(&bars->abort), crank ^ 1u), 1u);
    }
    __syncwarp();
    ptx::tc_fence_before();
    __syncthreads();
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
// Of a token: the label's logit, lift and sum so far, 2^-(lift added by the last piece).
struct CeRows {
    float *logit, *lift, *sum, *scale;
};

// A token's halves of tiles, (octaves that the exponentials were taken under, sum of them) each, joined: eight tokens to a CTA, 32 threads to a token, eight of their loads under way at once.
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
    const float over = fmaf(logit[m], kLog2e, -all.top);      // the label's logit above the largest of the others, octaves
    loss[m] = all.top == -INFINITY ? all.sum : over >= 0.0f ? log1pf(all.sum * exp2f(-over)) : logf(all.sum + exp2f(over)) - over * kLn2;
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

// dX = c (O - S W_y) / (S + E), and the loss; eight features to a thread.
__global__ void __launch_bounds__(256) finish_kernel(const float* O, int splits, const uint16_t* W, const long long* labels, const float* weights, int M, int V, int K, long long ignore,
                                                     float scale, CeRows R, uint16_t* dX, float* loss) {
    pdl_enter();
    const long long vectors = (long long)M * (K / 8), step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < vectors; i += step) {
        const int m = (int)(i / (K / 8)), k = (int)(i - (long long)m * (K / 8)) * 8;
        const long long y = labels[m];
        uint4 out = make_uint4(0u, 0u, 0u, 0u);
        if (y != ignore) {
            const bool word = y >= 0 && y < V;
            const float sum = word ? R.sum[m] : NAN, over = word ? fmaf(R.logit[m], kLog2e, -R.lift[m]) : 0.0f;      // (over: the label's logit above the lift, octaves)
            const float own = exp2f(over), total = sum + own;
            if (k == 0) loss[m] = sum == 0.0f ? 0.0f : over >= 0.0f ? log1pf(sum * exp2f(-over)) : logf(total) - over * kLn2;
            const float c = weights != nullptr ? scale * weights[m] : scale, a = c / total, b = a * sum;
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int s = 0; s < splits; ++s) {
                const float4* o = reinterpret_cast<const float4*>(O + ((size_t)s * M + m) * K + k);
                const float4 p = __ldcs(o), q = __ldcs(o + 1);
                x[0] += p.x; x[1] += p.y; x[2] += p.z; x[3] += p.w; x[4] += q.x; x[5] += q.y; x[6] += q.z; x[7] += q.w;
            }
            const uint4 w = word ? __ldg(reinterpret_cast<const uint4*>(W + (size_t)y * K + k)) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t wv[4] = {w.x, w.y, w.z, w.w};
            uint32_t r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float lo = a * x[2 * j] - b * __uint_as_float(wv[j] << 16), hi = a * x[2 * j + 1] - b * __uint_as_float(wv[j] & 0xffff0000u);
                r[j] = pack_bf16x2(lo, hi);
            }
            out = make_uint4(r[0], r[1], r[2], r[3]);
        } else if (k == 0) {
            loss[m] = 0.0f;
        }
        *reinterpret_cast<uint4*>(dX + (size_t)m * K + k) = out;
    }
}

// ------------------------------------------------------------------------------------------------ host
constexpr int kMostTokens = 4096;                          // of a pass; more go in several passes
constexpr size_t kPieceBytes = (size_t)128 << 20;          // of a piece's exponentials
constexpr int kMostV = 1 << 24, kMostK = 1 << 16, kMostM = 1 << 30, kMostSplits = 16;
constexpr int kPairs = kNumSMs / 2;

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// How a call is cut: by rules on its sizes alone, so that the scratch can be asked for beforehand.
struct CePlan {
    int passes, tokens;                 // passes over the tokens, tokens of one
    int width, tiles;                   // columns of a tile of logits, and tiles of a piece
    int pieces, piece;                  // pieces of the vocabulary, their words (the last may have fewer)
    int splits;                         // parts of the gradient's contraction
    size_t off_rows, off_stats, off_e, off_out, total;
};
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
    p.splits = 1;
    if (grad) {
        // parts of the contraction: rounds of blocks, six more for filling and draining, and what O costs in memory (in blocks' time, 0.3 us)
        const long units = (long)tiles_m * ((K + kTile - 1) / kTile), blocks = (p.tiles * p.width + kDepth - 1) / kDepth;
        double least = -1.0;
        for (int s = 1; s <= kMostSplits && s <= blocks; ++s) {
            const double cost = (double)((units * s + kPairs - 1) / kPairs) * ((blocks + s - 1) / s + 6) * p.pieces + s * ((double)p.tokens * K * 8.0 / 6.4e12 / 0.3e-6);
            if (least < 0.0 || cost < least) { least = cost; p.splits = s; }
        }
    }
    p.off_rows = 256;
    p.off_stats = p.off_rows + 4 * up256((size_t)p.tokens * 4);
    p.off_e = p.off_stats + up256((size_t)p.tiles * 2 * p.tokens * 8);
    p.off_out = p.off_e + (grad ? up256((size_t)p.tokens * p.tiles * p.width * 2) : 0);
    p.total = p.off_out + (grad ? up256((size_t)p.splits * p.tokens * K * 4) : 0);
    return p;
}

bool good_sizes(int M, int V, int K) { return M >= 1 && M <= kMostM && V >= 1 && V <= kMostV && K >= 64 && K <= kMostK && K % 8 == 0; }

template <int KIND>
lowra_status launch_product(CeParams& P, cudaStream_t stream) {
    static SmemLimit limit = {};
    if (ensure_smem_limit(reinterpret_cast<const void*>(product_kernel<KIND>), kSmem, &limit) != LOWRA_OK) return LOWRA_ERR_CUDA;
    // (the warps' shares of the registers were added up for a kernel of this size)
    static std::atomic<int> registers{0};
    if (registers.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes of;
        if (cudaFuncGetAttributes(&of, product_kernel<KIND>) != cudaSuccess) return LOWRA_ERR_CUDA;
        registers.store(of.numRegs, std::memory_order_relaxed);
    }
    const int sms = device_sm_count();
    if (sms < 2 || registers.load(std::memory_order_relaxed) != kLaunchRegisters) return LOWRA_ERR_CUDA;
    const int units = P.tiles_m * P.tiles_n * P.splits, pairs = units < sms / 2 ? units : sms / 2;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)pairs * 2, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, product_kernel<KIND>, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}

}  // namespace
}  // namespace lowra

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
    cudaStream_t stream = (cudaStream_t)stream_v;
    unsigned char* ws = static_cast<unsigned char*>(workspace_dev);
    uint32_t* status = reinterpret_cast<uint32_t*>(ws);
    const size_t row = up256((size_t)p.tokens * 4) / 4;
    float* rows = reinterpret_cast<float*>(ws + p.off_rows);
    const CeRows R = {rows, rows + row, rows + 2 * row, rows + 3 * row};
    float2* stats = reinterpret_cast<float2*>(ws + p.off_stats);
    uint16_t* e = reinterpret_cast<uint16_t*>(ws + p.off_e);
    float* O = reinterpret_cast<float*>(ws + p.off_out);
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
        if (!make_map(&P.a, X, (uint64_t)m, (uint64_t)K, (uint64_t)K, 128) || !make_map(&P.b, W_dev, (uint64_t)V, (uint64_t)K, (uint64_t)K, (uint32_t)p.width / 2)) return LOWRA_ERR_CUDA;
        if (!dX_dev) {
            P.N = V;
            P.tiles_n = p.tiles;
            P.clear_status = pass == 0;
            if ((st = launch_product<kSums>(P, stream)) != LOWRA_OK) return st;
            if (launch_pdl(loss_kernel, (unsigned)((m + kTokens - 1) / kTokens), kTokens * kLanes, stream, (const float2*)stats, 2 * p.tiles, (const float*)R.logit, labels, m, (int)V, (long long)ignore_index,
                           loss_dev + m0) != cudaSuccess)
                return LOWRA_ERR_CUDA;
            continue;
        }
        CeParams G = P;
        G.N = K;
        G.width = kTile;
        G.tiles_n = (K + kTile - 1) / kTile;
        G.splits = p.splits;
        G.scale = R.scale;
        G.out = O;
        if (!make_map(&G.b, W_dev, (uint64_t)V, (uint64_t)K, (uint64_t)K, 64)) return LOWRA_ERR_CUDA;
        for (int c = 0; c < p.pieces; ++c) {
            P.v0 = G.v0 = c * p.piece;
            P.N = V - P.v0 < p.piece ? V - P.v0 : p.piece;
            P.tiles_n = (P.N + p.width - 1) / p.width;
            G.blocks = (P.N + kDepth - 1) / kDepth;
            P.first = G.first = c == 0;
            P.clear_status = pass == 0 && c == 0;
            // (columns that the first product does not write, in a last block that is not full, are past the end)
            if (!make_map(&G.a, e, (uint64_t)m, (uint64_t)P.tiles_n * p.width, (uint64_t)ld_e, 128)) return LOWRA_ERR_CUDA;
            if ((st = launch_product<kExponentials>(P, stream)) != LOWRA_OK) return st;
            if (launch_pdl(lift_kernel, (unsigned)((m + kTokens - 1) / kTokens), kTokens * kLanes, stream, (const float2*)stats, 2 * P.tiles_n, m, p.width, P.first, e, ld_e, R) != cudaSuccess) return LOWRA_ERR_CUDA;
            if ((st = launch_product<kGradient>(G, stream)) != LOWRA_OK) return st;
        }
        const long long ctas = ((long long)m * (K / 8) + 255) / 256;
        if (launch_pdl(finish_kernel, (unsigned)(ctas < 8 * kNumSMs ? ctas : 8 * kNumSMs), 256, stream, (const float*)O, p.splits, W_dev, labels, weights, m, (int)V, (int)K,
                       (long long)ignore_index, scale, R, dX_dev + m0 * K, loss_dev + m0) != cudaSuccess)
            return LOWRA_ERR_CUDA;
    }
    return LOWRA_OK;
}
