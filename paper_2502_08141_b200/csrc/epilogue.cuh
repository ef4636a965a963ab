// What stands behind a product in a model, on the fp32 sums: Z = product + bias, H = act(Z), Y = H multiply + residual.  Everything is computed in 32 bits
// and rounded once, to bf16 (Y, and the copy of Z that the backward pass reads).  Shared by the tensor-core kernel, the kernels for few tokens and the backward
// pass.
#pragma once

#include "lowra_common.cuh"

namespace lowra {

struct Epilogue {
    const void* bias;             // [N] bf16 or fp32, or null
    const uint16_t* multiply;     // [M, N] bf16, or null
    const uint16_t* residual;     // [M, N] bf16, or null; may be the output itself (an element is read by the thread that writes it, before it does)
    uint16_t* pre;                // [M, N] bf16 (out), or null
    int32_t activation;           // lowra_activation
    int32_t bias_bf16;
};

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint16_t bf16_bits(float v) { return (uint16_t)pack_bf16x2(v, 0.0f); }

// The activations, on the hardware's 2^x and 1 / x (each within 2^-22 of itself; subnormal results are zero): far below the rounding to bf16 that follows, and with
// errors of either sign, so that sums of many (a bias's gradient, fp32) are as good as in full precision.  Where the divisor overflows they give the limit, a
// zero.  The tails are computed without cancellation: gelu by the normal distribution's own tail, the tanh form as z sigmoid(2 t), so that no value is
// the difference of two near ones.  NaN passes everywhere, through relu too (which a maximum would not let through).
constexpr float kTanhScale = 0.79788456080286536f, kTanhCubic = 0.044715f, kNormPeak = 0.39894228040143268f, kLog2E = 1.4426950408889634f;
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid(float z) { return reciprocal_fast(1.0f + exp2_fast(-kLog2E * z)); }
__device__ __forceinline__ float tanh_argument(float z) { return 2.0f * kTanhScale * (z + kTanhCubic * z * z * z); }

// Phi(z), and exp(-z^2 / 2) for its derivative.  Phi(-|z|) = exp(-z^2 / 2) R(|z|), where R falls off like 1 / |z|: a polynomial in t = 1 / (1 + 0.425 |z| / sqrt 2)
// without a constant term, whose coefficients make the largest relative error on 0 <= |z| <= 13.4 least (iteratively reweighted least squares on 500 Chebyshev
// points: 1.2e-7; 4.6e-7 with fp32's roundings).  The exponential serves the derivative too; erfcf takes three times the instructions, and one call of it
// per element took the backward pass's arithmetic beyond its memory traffic.
__device__ __forceinline__ float normal_cdf(float z, float* bell) {
    const float t = reciprocal_fast(1.0f + 0.300520382f * fabsf(z));
    const float e = exp2_fast((-0.5f * kLog2E) * (z * z));
    float p = 0.0360919518f;
    p = p * t - 0.158048567f;
    p = p * t + 0.206342268f;
    p = p * t - 0.0539579815f;
    p = p * t + 0.12877795f;
    p = p * t + 0.0999785458f;
    p = p * t + 0.120980384f;
    p = p * t + 0.11983539f;
    const float q = p * t * e;
    *bell = e;
    return z < 0.0f ? q : 1.0f - q;
}

template <int ACT>
__device__ __forceinline__ float activate_as(float z) {
    float bell;
    if (ACT == LOWRA_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == LOWRA_ACT_GELU) return z * normal_cdf(z, &bell);
    if (ACT == LOWRA_ACT_GELU_TANH) return z * sigmoid(tanh_argument(z));
    if (ACT == LOWRA_ACT_SILU) return z * sigmoid(z);
    return z;
}
// act(z) and act'(z).  (relu at zero: slope 0.)
template <int ACT>
__device__ __forceinline__ float2 activate_and_slope(float z) {
    if (ACT == LOWRA_ACT_RELU) return make_float2(z < 0.0f ? 0.0f : z, z <= 0.0f ? 0.0f : 1.0f);
    if (ACT == LOWRA_ACT_GELU) {
        float bell;
        const float cdf = normal_cdf(z, &bell);
        return make_float2(z * cdf, cdf + z * (kNormPeak * bell));
    }
    if (ACT == LOWRA_ACT_GELU_TANH || ACT == LOWRA_ACT_SILU) {
        // p = sigmoid(t) and p (1 - p) from exp(-|t|), which neither overflows nor is a difference of near values
        const float t = ACT == LOWRA_ACT_SILU ? z : tanh_argument(z);
        const float e = exp2_fast(-kLog2E * fabsf(t)), r = reciprocal_fast(1.0f + e), p = t >= 0.0f ? r : e * r, w = e * r * r;
        if (ACT == LOWRA_ACT_SILU) return make_float2(z * p, p + z * w);
        const float c = fminf(fmaxf(z, -16.0f), 16.0f);           // (w is zero further out, and its factor may be infinite)
        return make_float2(z * p, p + c * w * (2.0f * kTanhScale) * (1.0f + 3.0f * kTanhCubic * c * c));
    }
    return make_float2(z, 1.0f);
}
// Phi of two values and their exp(-z^2 / 2), with two products to an instruction: value by value what normal_cdf gives.
__device__ __forceinline__ float2 normal_cdf(float2 z, float2* bell) {
    auto both = [](float c) { return make_float2(c, c); };
    const float2 d = fma2(both(0.300520382f), make_float2(fabsf(z.x), fabsf(z.y)), both(1.0f)), t = make_float2(reciprocal_fast(d.x), reciprocal_fast(d.y));
    const float2 x = mul2(mul2(z, z), both(-0.5f * kLog2E)), e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
    float2 p = fma2(both(0.0360919518f), t, both(-0.158048567f));
    p = fma2(p, t, both(0.206342268f));
    p = fma2(p, t, both(-0.0539579815f));
    p = fma2(p, t, both(0.12877795f));
    p = fma2(p, t, both(0.0999785458f));
    p = fma2(p, t, both(0.120980384f));
    p = fma2(p, t, both(0.11983539f));
    const float2 q = mul2(mul2(p, t), e);
    *bell = e;
    return make_float2(z.x < 0.0f ? q.x : 1.0f - q.x, z.y < 0.0f ? q.y : 1.0f - q.y);
}
// Two values; gelu with two products to an instruction (the backward pass is as much bound by its instructions as by memory there: 4096 x 11008 with a bias 53.3 -> 51.2 us).
template <int ACT>
__device__ __forceinline__ void activate_and_slope(float2 z, float2* act, float2* slope) {
    if (ACT != LOWRA_ACT_GELU) {
        const float2 a = activate_and_slope<ACT>(z.x), b = activate_and_slope<ACT>(z.y);
        *act = make_float2(a.x, b.x);
        *slope = make_float2(a.y, b.y);
        return;
    }
    float2 e;
    const float2 cdf = normal_cdf(z, &e);
    *act = mul2(z, cdf);
    *slope = fma2(z, mul2(make_float2(kNormPeak, kNormPeak), e), cdf);
}
// One activation for a few values: the choice is made once for all of them (it is the same in the whole launch).
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int activation) {
    auto all = [&](auto act) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = activate_as<decltype(act)::value>(z[i]);
    };
    if (activation == LOWRA_ACT_RELU) all(std::integral_constant<int, LOWRA_ACT_RELU>());
    else if (activation == LOWRA_ACT_GELU) all(std::integral_constant<int, LOWRA_ACT_GELU>());
    else if (activation == LOWRA_ACT_GELU_TANH) all(std::integral_constant<int, LOWRA_ACT_GELU_TANH>());
    else if (activation == LOWRA_ACT_SILU) all(std::integral_constant<int, LOWRA_ACT_SILU>());
}

__device__ __forceinline__ void unpack8(uint4 p, float (&v)[8]) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// Thirty-two neighbouring channels of one token, `groups` (1 .. 4) of eight of them, whose element there is number `at` of the [M, N] arrays (a multiple of 8).
// What is read first of those arrays is asked for ahead of time.
struct Behind {
    uint4 v[4];                   // of multiply, or of the residual where there is none
};
__device__ __forceinline__ void load_behind(const Epilogue& E, size_t at, int groups, Behind& x) {
    const uint16_t* from = E.multiply != nullptr ? E.multiply : E.residual;
    if (from == nullptr) return;
#pragma unroll
    for (int g = 0; g < 4; ++g)
        if (g < groups) x.v[g] = *reinterpret_cast<const uint4*>(from + at + 8 * g);
}
__device__ __forceinline__ void pack16(const float (&v)[16], uint32_t (&o)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
}
// Sixteen of them, numbers 16 H ..: the sums z become outputs; before() is called with Z itself.
template <int H, typename Before>
__device__ __forceinline__ void finish16(const Epilogue& E, const float* bias /* shared memory, 16 */, const Behind& x, size_t at, int groups, float (&z)[16], Before before) {
    if (E.bias != nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 b = reinterpret_cast<const float4*>(bias)[i];
            z[4 * i] += b.x; z[4 * i + 1] += b.y; z[4 * i + 2] += b.z; z[4 * i + 3] += b.w;
        }
    }
    if (E.pre != nullptr) before();
    if (E.activation == LOWRA_ACT_GELU) {
        // (Two values at a time, by the one form that all paths have, good to fp32: a residual may cancel what stands before it.  A polynomial good to 4e-4 alone, without the
        // division, was 1 % faster, and 4 % on short contractions: 11008 x 4096, 4096 tokens with the copy of Z 318 against 320 us, under the power cap 364 against 368;
        // 4096 x 512 46 against 48.)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 v = make_float2(z[2 * i], z[2 * i + 1]);
            float2 bell;
            const float2 h = mul2(v, normal_cdf(v, &bell));
            z[2 * i] = h.x;
            z[2 * i + 1] = h.y;
        }
    } else {
        activate(z, E.activation);
    }
    if (E.multiply != nullptr) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float m[8];
            unpack8(x.v[2 * H + g], m);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[8 * g + i] *= m[i];
        }
    }
    if (E.residual != nullptr) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            uint4 p = x.v[2 * H + g];
            if (E.multiply != nullptr && 2 * H + g < groups) p = *reinterpret_cast<const uint4*>(E.residual + at + 16 * H + 8 * g);
            float d[8];
            unpack8(p, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[8 * g + i] += d[i];
        }
    }
}

// One channel of one token: what is read for it, and the output.
struct Behind1 {
    float bias, multiply, residual;
};
__device__ __forceinline__ float load_bias(const Epilogue& E, int n) {
    if (E.bias == nullptr) return 0.0f;
    return E.bias_bf16 ? bf16_value(__ldg(static_cast<const uint16_t*>(E.bias) + n)) : __ldg(static_cast<const float*>(E.bias) + n);
}
__device__ __forceinline__ Behind1 load_behind1(const Epilogue& E, int n, size_t at) {
    Behind1 x = {load_bias(E, n), 1.0f, 0.0f};
    if (E.multiply != nullptr) x.multiply = bf16_value(E.multiply[at]);
    if (E.residual != nullptr) x.residual = bf16_value(E.residual[at]);
    return x;
}
__device__ __forceinline__ uint16_t finish1(const Epilogue& E, const Behind1& x, size_t at, float sum) {
    float z[1] = {sum};
    if (E.bias != nullptr) z[0] += x.bias;
    if (E.pre != nullptr) E.pre[at] = bf16_bits(z[0]);
    activate(z, E.activation);
    if (E.multiply != nullptr) z[0] *= x.multiply;
    if (E.residual != nullptr) z[0] += x.residual;
    return bf16_bits(z[0]);
}

}  // namespace lowra
