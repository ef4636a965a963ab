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

// The activations.  __expf and __fdividef (a few units of 2^-22) are far below the rounding to bf16 that follows; where the divisor overflows they give
// the limit, a zero.  The tails are computed without cancellation: gelu by the normal distribution's own tail, the tanh form as z sigmoid(2 t), so that no
// value is the difference of two near ones.  NaN passes everywhere, through relu too (which a maximum would not let through).
constexpr float kTanhScale = 0.79788456080286536f, kTanhCubic = 0.044715f, kNormPeak = 0.39894228040143268f;
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }
__device__ __forceinline__ float tanh_argument(float z) { return 2.0f * kTanhScale * (z + kTanhCubic * z * z * z); }

// Phi(z), and exp(-z^2 / 2) for its derivative.  Phi(-|z|) = exp(-z^2 / 2) R(|z|), where R falls off like 1 / |z|: a polynomial in t = 1 / (1 + 0.44 |z| / sqrt 2)
// without a constant term, whose coefficients make the largest relative error on 0 <= |z| <= 13.4 least (a linear programme over 800 points: 5.2e-6).  Sixteen
// instructions, and the exponential serves the derivative too; erfcf takes three times as many, and one call of it per element took the backward
// pass's arithmetic beyond its memory traffic.
__device__ __forceinline__ float normal_cdf(float z, float* bell) {
    const float t = __fdividef(1.0f, 1.0f + 0.311126984f * fabsf(z));
    const float e = __expf(-0.5f * z * z);
    float p = -0.146105705f;
    p = p * t + 0.350652419f;
    p = p * t + 0.0407313712f;
    p = p * t + 0.263586132f;
    p = p * t + 0.242569605f;
    p = p * t + 0.248561012f;
    const float q = 0.5f * p * t * e;
    *bell = e;
    return z < 0.0f ? q : 1.0f - q;
}

template <int ACT>
__device__ __forceinline__ float activate_as(float z) {
    float bell;
    if (ACT == LOWRA_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == LOWRA_ACT_GELU) return z * normal_cdf(z, &bell);
    if (ACT == LOWRA_ACT_GELU_TANH) return __fdividef(z, 1.0f + __expf(-tanh_argument(z)));
    if (ACT == LOWRA_ACT_SILU) return __fdividef(z, 1.0f + __expf(-z));
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
    if (ACT == LOWRA_ACT_GELU_TANH) {
        const float p = sigmoid(tanh_argument(z));
        return make_float2(z * p, p + z * p * (1.0f - p) * (2.0f * kTanhScale) * (1.0f + 3.0f * kTanhCubic * z * z));
    }
    if (ACT == LOWRA_ACT_SILU) {
        const float p = sigmoid(z);
        return make_float2(z * p, p * (1.0f + z * (1.0f - p)));
    }
    return make_float2(z, 1.0f);
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

// Eight neighbouring channels from n on of one token, whose element there is number `at` of the [M, N] arrays (a multiple of 8, as n is): the sums z -> packed
// outputs; the copy of Z is written.
__device__ __forceinline__ uint4 finish8(const Epilogue& E, int n, size_t at, float (&z)[8]) {
    if (E.bias != nullptr) {
        float b[8];
        if (E.bias_bf16) {
            unpack8(__ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(E.bias) + n)), b);
        } else {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(E.bias) + n);
            const float4 lo = __ldg(p), hi = __ldg(p + 1);
            b[0] = lo.x; b[1] = lo.y; b[2] = lo.z; b[3] = lo.w; b[4] = hi.x; b[5] = hi.y; b[6] = hi.z; b[7] = hi.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += b[i];
    }
    if (E.pre != nullptr) *reinterpret_cast<uint4*>(E.pre + at) = pack8(z);
    activate(z, E.activation);
    if (E.multiply != nullptr) {
        float m[8];
        unpack8(*reinterpret_cast<const uint4*>(E.multiply + at), m);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= m[i];
    }
    if (E.residual != nullptr) {
        float d[8];
        unpack8(*reinterpret_cast<const uint4*>(E.residual + at), d);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += d[i];
    }
    return pack8(z);
}

// One channel of one token.
__device__ __forceinline__ uint16_t finish1(const Epilogue& E, int n, size_t at, float sum) {
    float z[1] = {sum};
    if (E.bias != nullptr) z[0] += E.bias_bf16 ? bf16_value(__ldg(static_cast<const uint16_t*>(E.bias) + n)) : __ldg(static_cast<const float*>(E.bias) + n);
    if (E.pre != nullptr) E.pre[at] = bf16_bits(z[0]);
    activate(z, E.activation);
    if (E.multiply != nullptr) z[0] *= bf16_value(E.multiply[at]);
    if (E.residual != nullptr) z[0] += bf16_value(E.residual[at]);
    return bf16_bits(z[0]);
}

}  // namespace lowra
