// lowra_adamw: the optimiser's step over the factors of a model together, decoupled weight decay, states in fp32 or in 8 bits:
//     m' = b1 m + (1 - b1) g;   v' = b2 v + (1 - b2) g^2;   w' = w (1 - lr wd) - lr (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps)
// In 8 bits, of every 256 values one behind the other in a factor, are kept s = (their largest magnitude) / 448 in fp32 and the values over s as e4m3 (three bits behind the leading one, down
// to 2^-9 of 448); of the second moment its root is kept that way, whose range is half as many octaves, and a root that is not zero is kept off zero, so that no step is divided by
// eps for it.  m' and v' go into w' before they are rounded.
// To nearest, a step that changes a kept value by less than half a step of e4m3 (3 to 6 %) leaves it where it was: with b2 = 0.999 a root does not fall at all, and grows only where the gradient is some ten times
// as large.  Dithered, a value goes up or down with the chance that its place between two codes gives it, by a sequence of its own that is spread evenly over the steps (multiples of the golden ratio from a hash
// of the place), so that over the steps nothing is lost: gradients of 0.1, 0.5 and 0.01 for 4000, 4000 and 8000 steps, kept root over that of fp32: to nearest 0.98, 0.20, 7.3; dithered 0.99, 1.01, 0.87
// (fourteen factors of rank 64 18.5 -> 20.0 us).
// The states' arithmetic is fp32 with every operation rounded by itself, in the order above ((1 - b2) g first, then times g): what is rounded to 8 bits does not depend on
// how a compiler joins operations.
// Bound by memory: gradient, weights and states each read once and written once, 28 bytes a weight (bf16 gradient, fp32 states) or 16 (8 bits).  A warp takes 256 values at a
// time, eight to a lane, so that a scale is a warp reduction and all accesses are 16 bytes wide (8 for codes); the factors' descriptions are kernel parameters: a warp looks for
// the one of its first block by bisection and then goes on from one to the next.
// Measured: 448 factors of rank 64 (160 M weights, fp32 states) 720 us, one reading and writing 693 at the copy rate; fourteen of them in 8 bits 17.8 us (12.4), of which a launch with nothing to do is 2;
// two of 1024 x 16 and 16 x 4096 3.1 us.
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "lowra_common.cuh"

namespace lowra {

namespace {

// CTAs to an SM that the registers are shared out for, and that a launch has: with fp32 states the memory is bound by the number of streams that it serves (448 factors: 738 us with three, 815 with
// four, 926 with six; with fp32 gradients, one stream more in wider pieces, the other way: 8 layers 218 us with four, 241 with three); with 8-bit ones loads have to hide more work (8 layers 118 us with five, 124 with four; with fp32
// gradients 137, 125).
template <bool EIGHT>
constexpr int kAdamResident = EIGHT ? 5 : 4;
int resident_of(bool eight, bool grad_fp32) { return eight ? (grad_fp32 ? 4 : 5) : grad_fp32 ? 4 : 3; }
// Blocks from which on a launch waits for the one before to have ended, as launches do: CTAs that come in as the others leave crowd on the SMs that are done first (448 factors, two
// launches a step, step after step: 840 us when they may come in from the start, 777 when this launch is nearly done, 716 so; a layer's fourteen, 8 bits: 19.7, 17.8, 19.8).
constexpr uint32_t kAdamMany = 1 << 16;
constexpr int kAdamThreads = 256, kAdamBlock = LOWRA_ADAMW_BLOCK;
constexpr int kFewMembers = 16, kManyMembers = 224;       // members of a launch that its parameters have room for (24 KB of them take a launch 2 us more than 2 KB)
static_assert(kAdamBlock == 32 * 8, "a warp's values");

struct AdamMember {
    const void* grad;
    const float* master;
    float* master_out;
    uint16_t* weight;
    const void *m, *v;
    void *m_out, *v_out;
    const float *m_scale, *v_scale;
    float *m_scale_out, *v_scale_out;
    long long n;
};
template <int MEMBERS>
struct AdamParams {
    AdamMember f[MEMBERS];
    uint32_t first[MEMBERS + 1];                    // blocks before each factor's, and of all
    uint16_t count, grad_fp32;
    float b1, c1, b2, c2, decay, rate, root_scale, eps;
    uint32_t before, number;                        // (dithered) blocks in earlier launches of the call; the step.  (They fill what the others leave: eight bytes more take the host 0.3 us.)
    // on the device, or null: the gradient's factor, the step and the learning rate
    const float *grad_scale, *lr;
    const int32_t* step;
    double log_b1, log_b2, wd;
};

template <typename T>
__device__ __forceinline__ T load(const void* p) {  // (not as read-only memory: states and weights are written in place)
    T v;
    static_assert(sizeof(T) == 16 || sizeof(T) == 8, "");
    if constexpr (sizeof(T) == 16)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    else
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}

__device__ __forceinline__ float2 mul2(float2 a, float b) { return lowra::mul2(a, make_float2(b, b)); }
// Sums of two products each, every operation rounded by itself (an add.rn.f32x2 behind a mul.rn.f32x2 came out as one operation, rounded once; single additions do not).
__device__ __forceinline__ float2 add_products(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }

// Eight values of a lane: `left` of them exist (eight but at a factor's end).
__device__ __forceinline__ void load_floats(const float* p, int left, float (&x)[8]) {
    if (left >= 8) {
        const uint4 a = load<uint4>(p), b = load<uint4>(p + 4);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < left ? *reinterpret_cast<const volatile float*>(p + i) : 0.0f;
    }
}
__device__ __forceinline__ void store_floats(float* p, int left, const float (&x)[8]) {
    if (left >= 8) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(x[0], x[1], x[2], x[3]));      // (not read again soon: 736 -> 720 us)
        __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(x[4], x[5], x[6], x[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = x[i];
    }
}
__device__ __forceinline__ void load_bf16(const uint16_t* p, int left, float (&x)[8]) {
    if (left >= 8) {
        const uint4 a = load<uint4>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < left ? __uint_as_float((uint32_t)p[i] << 16) : 0.0f;
    }
}
// codes (e4m3) times their block's scale
__device__ __forceinline__ void load_codes(const uint8_t* p, int left, float scale, float (&x)[8]) {
    uint32_t w[2] = {0u, 0u};
    if (left >= 8) {
        const uint2 a = load<uint2>(p);
        w[0] = a.x;
        w[1] = a.y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) w[i >> 2] |= (uint32_t)*reinterpret_cast<const volatile uint8_t*>(p + i) << (8 * (i & 3));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3)));
        const float2 v = mul2(f, scale);
        x[2 * i] = v.x;
        x[2 * i + 1] = v.y;
    }
}
// The larger magnitude; a NaN is above all.
__device__ __forceinline__ float larger(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(fabsf(b)));
    return m;
}
// One of the two e4m3 numbers about f, the upper with the chance that f's place between them gives it; u even over 32 bits.  (What is above 448, or a NaN, stays for the conversion.)
__device__ __forceinline__ float dithered(float f, uint32_t u) {
    const float a = fabsf(f);
    // steps of 2^-9 below the normal numbers; else the twenty bits of the fraction that e4m3 has not, added and cut off
    float r = a < 0x1p-6f ? floorf(fmaf(a, 512.0f, (float)(u >> 8) * 0x1p-24f)) * 0x1p-9f : __uint_as_float((__float_as_uint(a) + (u >> 12)) & 0xfff00000u);
    if (!(a <= 448.0f)) r = a;
    return copysignf(r, f);
}
// Fractions of 2^32: the golden ratio less 1, half the root of 2, the root of 2 less 1.
constexpr uint32_t kGolden = 0x9e3779b9u, kNext = 0xb504f333u, kFirstMoment = 0x6a09e667u;
// A permutation of 32 bits after which neighbours are nowhere near one another, nor a fixed multiple of anything apart.
__device__ __forceinline__ uint32_t mixed(uint32_t x) {
    x *= kGolden;
    x = (x ^ x >> 16) * kNext;
    return (x ^ x >> 15) * kGolden;
}

// The block's scale and the lane's codes.  Over the lanes magnitudes are compared as integers: a NaN is above all there too, and its scale is NaN.
template <bool ROOT, bool DITHER>
__device__ __forceinline__ float store_codes(uint8_t* p, int left, const float (&x)[8], [[maybe_unused]] uint32_t u) {
    float most = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) most = larger(most, x[i]);
    float scale = __fmul_rn(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most))), 1.0f / 448.0f);
    if (scale < 0x1p-126f) scale = 0.0f;             // its reciprocal would be out of range: the block is zero
    const float over = scale > 0.0f ? __frcp_rn(scale) : 0.0f;
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 f = mul2(make_float2(x[2 * i], x[2 * i + 1]), over);
        if (ROOT) {
            if (f.x > 0.0f) f.x = fmaxf(f.x, 0x1p-9f);
            if (f.y > 0.0f) f.y = fmaxf(f.y, 0x1p-9f);
        }
        if (DITHER) f = make_float2(dithered(f.x, u + 2u * i * kNext), dithered(f.y, u + (2u * i + 1u) * kNext));
        w[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3) << (16 * (i & 1));
    }
    if (left >= 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
    return scale;
}

template <bool EIGHT, int MEMBERS, bool DITHER>
__global__ void __launch_bounds__(kAdamThreads, kAdamResident<EIGHT>) adamw_kernel(const __grid_constant__ AdamParams<MEMBERS> P) {
    __shared__ float shared[3];
    if (gridDim.x <= kNumSMs) pdl_release();          // (few blocks: there is room for the next launch's)
    pdl_wait();
    float decay = P.decay, rate = P.rate, root_scale = P.root_scale;
    if (P.step != nullptr || P.lr != nullptr) {      // a captured step reads them when it runs
        if (threadIdx.x == 0) {                      // (fp64, a chain of its own for each of the two powers: a captured step of two factors 3.9 -> 3.6 us, with the host's step 3.2)
            const float lr = P.lr != nullptr ? *P.lr : 1.0f;
            // rate: lr / (1 - b1^t) as far as the host knows it, else lr, 1 / (1 - b1^t) or 1
            const double one = P.step != nullptr ? -expm1((double)*P.step * P.log_b1) : 1.0;
            shared[0] = P.lr != nullptr ? (float)(1.0 - (double)lr * P.wd) : decay;
            shared[1] = (float)((double)rate * (double)lr / one);
        }
        if (threadIdx.x == 32) shared[2] = P.step != nullptr ? (float)(1.0 / sqrt(-expm1((double)*P.step * P.log_b2))) : root_scale;
        __syncthreads();
        decay = shared[0];
        rate = shared[1];
        root_scale = shared[2];
    }
    const float grad_scale = P.grad_scale != nullptr ? *P.grad_scale : 1.0f;
    [[maybe_unused]] uint32_t turn = 0;
    if constexpr (DITHER) turn = (P.step != nullptr ? (uint32_t)*P.step : P.number) * kGolden;
    const int lane = threadIdx.x & 31;
    // The CTAs go through the blocks side by side (448 factors 736 us; each through a run of its own 764); the factor of the first one is searched for, the next ones follow.
    const uint32_t blocks = P.first[P.count], step = gridDim.x * (kAdamThreads / 32);
    uint32_t block = blockIdx.x * (kAdamThreads / 32) + (threadIdx.x >> 5);
    int lo = 0;
    for (int hi = P.count; hi - lo > 1;) {           // first[lo] <= block < first[hi]
        const int mid = (lo + hi) >> 1;
        if (P.first[mid] <= block) lo = mid;
        else hi = mid;
    }
    for (; block < blocks; block += step) {
        while (P.first[lo + 1] <= block) ++lo;
        const AdamMember& F = P.f[lo];
        const uint32_t in = block - P.first[lo];
        const long long at = (long long)in * kAdamBlock + lane * 8;
        const int left = (int)min((long long)8, F.n - at);             // (none or fewer: lanes past the end)
        float g[8], w[8], m[8], v[8];
        if (P.grad_fp32) load_floats(static_cast<const float*>(F.grad) + at, left, g);
        else load_bf16(static_cast<const uint16_t*>(F.grad) + at, left, g);
        load_floats(F.master + at, left, w);
        if (EIGHT) {
            load_codes(static_cast<const uint8_t*>(F.m) + at, left, F.m_scale[in], m);
            load_codes(static_cast<const uint8_t*>(F.v) + at, left, F.v_scale[in], v);
        } else {
            load_floats(static_cast<const float*>(F.m) + at, left, m);
            load_floats(static_cast<const float*>(F.v) + at, left, v);
        }
        float root[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float2 gg = make_float2(g[i], g[i + 1]), vv = make_float2(v[i], v[i + 1]);
            if (P.grad_scale != nullptr) gg = mul2(gg, grad_scale);
            if (EIGHT) vv = lowra::mul2(vv, vv);        // (what is kept is the root)
            const float2 mm = add_products(mul2(make_float2(m[i], m[i + 1]), P.b1), mul2(gg, P.c1));
            vv = add_products(mul2(vv, P.b2), lowra::mul2(mul2(gg, P.c2), gg));
            m[i] = mm.x;
            m[i + 1] = mm.y;
            v[i] = vv.x;
            v[i + 1] = vv.y;
            root[i] = __fsqrt_rn(vv.x);
            root[i + 1] = __fsqrt_rn(vv.y);
            const float2 under = fma2(make_float2(root[i], root[i + 1]), make_float2(root_scale, root_scale), make_float2(P.eps, P.eps));
            const float2 step2 = make_float2(__fdividef(mm.x, under.x), __fdividef(mm.y, under.y));
            const float2 ww = fma2(step2, make_float2(-rate, -rate), mul2(make_float2(w[i], w[i + 1]), decay));
            w[i] = ww.x;
            w[i + 1] = ww.y;
        }
        store_floats(F.master_out + at, left, w);
        if (F.weight != nullptr) {
            if (left >= 8) {
                __stcs(reinterpret_cast<uint4*>(F.weight + at), make_uint4(pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left) F.weight[at + i] = (uint16_t)pack_bf16x2(w[i], 0.0f);
            }
        }
        if (EIGHT) {
            [[maybe_unused]] uint32_t u = 0;
            if constexpr (DITHER) u = mixed((P.before + block) * 32u + (uint32_t)lane) + turn;
            const float a = store_codes<false, DITHER>(static_cast<uint8_t*>(F.m_out) + at, left, m, u + kFirstMoment), b = store_codes<true, DITHER>(static_cast<uint8_t*>(F.v_out) + at, left, root, u);
            if (lane == 0) {
                F.m_scale_out[in] = a;
                F.v_scale_out[in] = b;
            }
        } else {
            store_floats(static_cast<float*>(F.m_out) + at, left, m);
            store_floats(static_cast<float*>(F.v_out) + at, left, v);
        }
    }
    pdl_release();
}

template <bool EIGHT, int MEMBERS, bool DITHER>
lowra_status launch_adamw(const lowra_adamw_member* members, int count, const lowra_adamw_step& S, cudaStream_t stream) {
    AdamParams<MEMBERS> P;
    P.grad_fp32 = S.grad_fp32 != 0;
    P.b1 = (float)S.beta1;
    P.c1 = (float)(1.0 - S.beta1);
    P.b2 = (float)S.beta2;
    P.c2 = (float)(1.0 - S.beta2);
    P.eps = (float)S.eps;
    P.wd = S.weight_decay;
    P.decay = (float)(1.0 - S.lr * S.weight_decay);
    P.log_b1 = std::log(S.beta1);
    P.log_b2 = std::log(S.beta2);
    const double one = S.step_dev ? 1.0 : 1.0 - std::pow(S.beta1, (double)S.step);
    P.rate = (float)((S.lr_dev ? 1.0 : S.lr) / one);
    P.root_scale = S.step_dev ? 1.0f : (float)(1.0 / std::sqrt(1.0 - std::pow(S.beta2, (double)S.step)));
    P.grad_scale = S.grad_scale_dev;
    P.lr = S.lr_dev;
    P.step = S.step_dev;
    P.number = (uint32_t)S.step;
    P.before = 0;
    for (int i0 = 0; i0 < count; i0 += MEMBERS) {
        P.count = (uint16_t)std::min(count - i0, MEMBERS);
        P.first[0] = 0;
        for (int i = 0; i < P.count; ++i) {
            const lowra_adamw_member& m = members[i0 + i];
            P.f[i] = AdamMember{m.grad_dev, m.master_dev, m.master_out_dev, m.weight_dev, m.m_dev, m.v_dev, m.m_out_dev, m.v_out_dev,
                                m.m_scale_dev, m.v_scale_dev, m.m_scale_out_dev, m.v_scale_out_dev, m.n};
            P.first[i + 1] = P.first[i] + (uint32_t)((m.n + kAdamBlock - 1) / kAdamBlock);
        }
        const uint32_t wanted = (P.first[P.count] + kAdamThreads / 32 - 1) / (kAdamThreads / 32), most = (uint32_t)(kNumSMs * resident_of(EIGHT, P.grad_fp32 != 0));
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3(std::min(wanted, most), 1, 1);
        cfg.blockDim = dim3(kAdamThreads, 1, 1);
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = P.first[P.count] < kAdamMany ? 1 : 0;
        if (cudaLaunchKernelEx(&cfg, adamw_kernel<EIGHT, MEMBERS, DITHER>, P) != cudaSuccess) return LOWRA_ERR_CUDA;
        P.before += P.first[P.count];
    }
    return LOWRA_OK;
}

// Something written that shares memory with anything else of the call.  In the order of their places, an array is in the way of one before it if it is in that of the one that reaches
// furthest, among all if it is written, among the written if it is read.
struct Place {
    uintptr_t at, end;
    bool written;
};
// Sorted by merging the runs that are in order already: the arrays come kind by kind, and those of a kind mostly as they were allocated (448 factors, 3584 arrays: 30 us, 150 by std::sort).
void sort_runs(Place* p, Place* room, size_t n, size_t* starts) {
    const auto before = [](const Place& a, const Place& b) { return a.at < b.at; };
    size_t runs = 0;
    for (size_t i = 0; i < n; ++i)
        if (i == 0 || p[i].at < p[i - 1].at) starts[runs++] = i;
    Place *from = p, *to = room;
    while (runs > 1) {
        size_t left = 0;
        for (size_t r = 0; r < runs; r += 2) {
            const size_t a = starts[r], b = r + 1 < runs ? starts[r + 1] : n, c = r + 2 < runs ? starts[r + 2] : n;
            std::merge(from + a, from + b, from + b, from + c, to + a, before);
            starts[left++] = a;
        }
        runs = left;
        std::swap(from, to);
    }
    if (from != p) std::copy(from, from + n, p);
}
bool any_clash(const Place* p, size_t n) {
    uintptr_t any = 0, written = 0;
    for (size_t i = 0; i < n; ++i) {
        if (p[i].at < (p[i].written ? any : written)) return true;
        any = std::max(any, p[i].end);
        if (p[i].written) written = std::max(written, p[i].end);
    }
    return false;
}

}  // namespace
}  // namespace lowra

extern "C" lowra_status lowra_adamw(const lowra_adamw_member* members_host, int32_t count, const lowra_adamw_step* step_host, void* stream_v) {
    using namespace lowra;
    if (!members_host || !step_host) return LOWRA_ERR_NULL;
    const lowra_adamw_step& S = *step_host;
    if (count < 1 || count > LOWRA_MAX_ADAMW || (S.bits != 8 && S.bits != 32 && S.bits != (8 | LOWRA_ADAMW_DITHER)) || (!S.step_dev && S.step < 1) || !(S.beta1 >= 0.0 && S.beta1 < 1.0) ||
        !(S.beta2 >= 0.0 && S.beta2 < 1.0) || !(S.eps >= 0.0))
        return LOWRA_ERR_SHAPE;
    const bool eight = S.bits != 32, dither = eight && S.bits != 8;
    const size_t wide = eight ? 1 : 4;
    constexpr int kKinds = 12;
    const size_t most = (size_t)count * kKinds + 3;
    std::unique_ptr<Place[]> places(new (std::nothrow) Place[2 * most]);
    std::unique_ptr<size_t[]> starts(new (std::nothrow) size_t[most]);
    if (!places || !starts) return LOWRA_ERR_CUDA;
    size_t n_places = 0;
    auto add = [&](const void* p, size_t bytes, bool written) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        if (p != nullptr) places[n_places++] = Place{at, at + bytes, written};
    };
    unsigned long long blocks = 0;
    for (int i = 0; i < count; ++i) {
        const lowra_adamw_member& m = members_host[i];
        if (!m.grad_dev || !m.master_dev || !m.master_out_dev || !m.m_dev || !m.m_out_dev || !m.v_dev || !m.v_out_dev) return LOWRA_ERR_NULL;
        if (eight && (!m.m_scale_dev || !m.m_scale_out_dev || !m.v_scale_dev || !m.v_scale_out_dev)) return LOWRA_ERR_NULL;
        if (m.n < 1 || m.n > (1ll << 36)) return LOWRA_ERR_SHAPE;
        const void* all[12] = {m.grad_dev, m.master_dev, m.master_out_dev, m.weight_dev, m.m_dev, m.m_out_dev, m.v_dev, m.v_out_dev,
                               eight ? m.m_scale_dev : nullptr, eight ? m.m_scale_out_dev : nullptr, eight ? m.v_scale_dev : nullptr, eight ? m.v_scale_out_dev : nullptr};
        for (int k = 0; k < 8; ++k)
            if (!aligned16(all[k])) return LOWRA_ERR_ALIGN;
        for (int k = 8; k < 12; ++k)
            if ((reinterpret_cast<uintptr_t>(all[k]) & 3u) != 0) return LOWRA_ERR_ALIGN;
        blocks += ((unsigned long long)m.n + kAdamBlock - 1) / kAdamBlock;
    }
    // kind by kind; an input that is its own output counts once
    using M = lowra_adamw_member;
    auto add_all = [&](auto array, size_t bytes, size_t per, bool written, auto unless) {
        for (int i = 0; i < count; ++i) {
            const M& m = members_host[i];
            const void *p = array(m), *same = unless(m);
            if (p != same) add(p, ((size_t)m.n + per - 1) / per * bytes, written);
        }
    };
    const auto never = [](const M&) -> const void* { return nullptr; };
    add_all([](const M& m) { return m.grad_dev; }, S.grad_fp32 ? 4 : 2, 1, false, never);
    add_all([](const M& m) { return (const void*)m.weight_dev; }, 2, 1, true, never);
    add_all([](const M& m) { return (const void*)m.master_out_dev; }, 4, 1, true, never);
    add_all([](const M& m) { return (const void*)m.m_out_dev; }, wide, 1, true, never);
    add_all([](const M& m) { return (const void*)m.v_out_dev; }, wide, 1, true, never);
    add_all([](const M& m) { return (const void*)m.master_dev; }, 4, 1, false, [](const M& m) { return (const void*)m.master_out_dev; });
    add_all([](const M& m) { return m.m_dev; }, wide, 1, false, [](const M& m) { return (const void*)m.m_out_dev; });
    add_all([](const M& m) { return m.v_dev; }, wide, 1, false, [](const M& m) { return (const void*)m.v_out_dev; });
    if (eight) {
        add_all([](const M& m) { return (const void*)m.m_scale_out_dev; }, 4, kAdamBlock, true, never);
        add_all([](const M& m) { return (const void*)m.v_scale_out_dev; }, 4, kAdamBlock, true, never);
        add_all([](const M& m) { return (const void*)m.m_scale_dev; }, 4, kAdamBlock, false, [](const M& m) { return (const void*)m.m_scale_out_dev; });
        add_all([](const M& m) { return (const void*)m.v_scale_dev; }, 4, kAdamBlock, false, [](const M& m) { return (const void*)m.v_scale_out_dev; });
    }
    add(S.grad_scale_dev, 4, false);
    add(S.lr_dev, 4, false);
    add(S.step_dev, 4, false);
    if (((reinterpret_cast<uintptr_t>(S.grad_scale_dev) | reinterpret_cast<uintptr_t>(S.lr_dev) | reinterpret_cast<uintptr_t>(S.step_dev)) & 3u) != 0) return LOWRA_ERR_ALIGN;
    if (blocks > 0x7fffffffull) return LOWRA_ERR_SHAPE;
    sort_runs(places.get(), places.get() + most, n_places, starts.get());
    if (any_clash(places.get(), n_places)) return LOWRA_ERR_SHAPE;
    const lowra_status st = check_device();
    if (st != LOWRA_OK) return st;
    const bool few = count <= kFewMembers;
    cudaStream_t stream = (cudaStream_t)stream_v;
    if (dither) return few ? launch_adamw<true, kFewMembers, true>(members_host, count, S, stream) : launch_adamw<true, kManyMembers, true>(members_host, count, S, stream);
    if (eight) return few ? launch_adamw<true, kFewMembers, false>(members_host, count, S, stream) : launch_adamw<true, kManyMembers, false>(members_host, count, S, stream);
    return few ? launch_adamw<false, kFewMembers, false>(members_host, count, S, stream) : launch_adamw<false, kManyMembers, false>(members_host, count, S, stream);
}
