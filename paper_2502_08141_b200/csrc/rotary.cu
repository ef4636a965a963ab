// lowra_rotary: positions turned into the heads of queries and keys.  A pair (a, b) of a head's first R values at position p becomes
//     scale * (a cos t - b sin t, b cos t + a sin t),   t = p * frequency of the pair;   the gradient turns the other way.
// Pairs lie side by side (interleaved) or half of the R values apart.  The frequencies come in turns (of 2 pi), as fractions of 2^64: the product with a position is taken modulo
// 2^64, which is modulo one turn, so that at any 32-bit position what is left of a turn is right to 2^-33 of one, without a wide multiplication or a
// reduction.  As an fp32 number, half turns from -1 to 1, it is right to 2^-26 of a turn, 9e-8 radians: cosines and sines are off by 2e-7 at most, absolutely (an output's rounding to bf16 is 2^-9 of it).
// Bound by memory, 4 bytes for every value.  A CTA takes the heads of a few tokens: its threads first work out the tokens' cosines and sines into shared memory, one pair each,
// with their first loads already under way, then go over the heads, sixteen values (eight pairs) of a head at a time.
// Measured: 4096 tokens, 32 + 32 heads of 128 25.4 us (20.8 at the copy rate; at 134 MB filling and draining the memory takes some 3 us), 16 tokens 2.4, one head of 64 for 1346 tokens 3.6.
#include <math.h>

#include "lowra_common.cuh"

namespace lowra {

namespace {

constexpr int kRotaryThreads = 256;
constexpr int kMostPairs = 512;                     // R / 2
constexpr int kTablePairs = 2048;                   // tokens x pairs of a run (or one token's)
constexpr int kRotaryResident = 4;                  // CTAs to an SM

struct RotaryPart {
    const uint16_t* x;
    uint16_t* out;
    long long x_token, x_head, out_token, out_head; // in elements
    int heads, copies;                              // whether the values past the turned ones have to be copied
};
struct RotaryParams {
    RotaryPart part[2];
    const int32_t* positions;
    const unsigned long long* turns;
    int M, D, R, tokens, heads, splits, ranges;     // tokens of a run; heads of both parts; CTAs that share a token's heads; ranges of tokens
    float scale;
    int interleaved, inverse;
};

__device__ __forceinline__ uint4 load8(const uint16_t* p) {       // (not as read-only memory: in place it is written)
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// A head's work in pieces of sixteen values: eight pairs each, then values to copy.  A thread keeps its place in the head and goes from head to head, so that it reads the cosines and sines of a token once
// and divides nothing on the way.
struct Piece {
    uint4 a, b;
    uint16_t* to;                                   // null: nothing to do
    int token;
};

template <bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryThreads, kRotaryResident) rotary_kernel(const __grid_constant__ RotaryParams P) {
    __shared__ __align__(16) float4 table[kTablePairs / 2];     // [token][pair of the piece / 2][piece]: (cosine, sine) of two pairs
    pdl_enter();
    const int range = (int)blockIdx.x / P.splits, split = (int)blockIdx.x - range * P.splits;
    const int begin = (int)((long long)P.M * range / P.ranges), end = (int)((long long)P.M * (range + 1) / P.ranges);
    const int head0 = P.heads * split / P.splits, heads = P.heads * (split + 1) / P.splits - head0;
    const int turned = P.R / 16, per_head = turned + (P.D - P.R + 15) / 16, pairs = P.R / 2;
    const int lanes = kRotaryThreads / per_head;       // heads side by side (a head has 256 pieces at most)
    const int lane = (int)threadIdx.x / per_head, u = (int)threadIdx.x % per_head;     // a thread's head and piece
    const int first = lane / heads, tokens_on = lanes / heads, heads_on = lanes - tokens_on * heads;      // from a thread's piece to its next
    constexpr int kAhead = 2;
    Piece q[kAhead];
    for (int token0 = begin; token0 < end; token0 += P.tokens) {
        const int tokens = min(P.tokens, end - token0);
        if (token0 > begin) __syncthreads();            // the table has been read
        const bool turns = u < turned;
        const int at = turns ? (INTERLEAVED ? u * 16 : u * 8) : P.R + (u - turned) * 16, other = INTERLEAVED || !turns ? 8 : P.R / 2;
        const bool both = turns || at + 8 < P.D;     // (the last piece to copy may have eight values)
        int token = first, head = lane - first * heads;                 // of the next piece to load
        auto load = [&](Piece& p) {
            p.to = nullptr;
            p.token = token;
            if (token < tokens && lane < lanes) {
                const bool second = head0 + head >= P.part[0].heads;
                const RotaryPart& part = P.part[second ? 1 : 0];
                const int h = head0 + head - (second ? P.part[0].heads : 0);
                if (turns || part.copies) {
                    const uint16_t* x = part.x + (long long)(token0 + token) * part.x_token + (long long)h * part.x_head + at;
                    p.a = load8(x);
                    if (both) p.b = load8(x + other);
                    p.to = part.out + (long long)(token0 + token) * part.out_token + (long long)h * part.out_head + at;
                }
            }
            token += tokens_on;
            head += heads_on;
            if (head >= heads) { head -= heads; ++token; }
        };
#pragma unroll
        for (int k = 0; k < kAhead; ++k) load(q[k]);
        for (int i = threadIdx.x; i < tokens * pairs; i += kRotaryThreads) {
            const int m = i / pairs, pair = i - m * pairs;
            // the turn's fraction, to the nearest 2^-32, as half turns from -1 to 1
            const unsigned long long turn = (unsigned long long)(long long)P.positions[token0 + m] * P.turns[pair] + 0x80000000ull;
            float s, c;
            sincospif((float)(int32_t)(uint32_t)(turn >> 32) * 0x1p-31f, &s, &c);
            reinterpret_cast<float2*>(table + (m * 4 + (pair & 7) / 2) * turned + pair / 8)[pair & 1] = make_float2(c * P.scale, (P.inverse ? -s : s) * P.scale);
        }
        __syncthreads();
        int have = -1;                              // the token whose cosines and sines are at hand
        float4 cs[4];
        auto finish = [&](Piece& p) {
            if (p.to == nullptr) return;
            if (turns) {
                if (p.token != have) {
                    have = p.token;
#pragma unroll
                    for (int i = 0; i < 4; ++i) cs[i] = table[(have * 4 + i) * turned + u];
                }
                const uint32_t a[4] = {p.a.x, p.a.y, p.a.z, p.a.w}, b[4] = {p.b.x, p.b.y, p.b.z, p.b.w};
                uint32_t ra[4], rb[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 c = cs[i];         // two pairs
                    if (INTERLEAVED) {
                        const uint32_t v0 = i < 2 ? a[2 * i] : b[2 * i - 4], v1 = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
                        const uint32_t r0 = pack_bf16x2(low(v0) * c.x - high(v0) * c.y, high(v0) * c.x + low(v0) * c.y);
                        const uint32_t r1 = pack_bf16x2(low(v1) * c.z - high(v1) * c.w, high(v1) * c.z + low(v1) * c.w);
                        if (i < 2) { ra[2 * i] = r0; ra[2 * i + 1] = r1; }
                        else { rb[2 * i - 4] = r0; rb[2 * i - 3] = r1; }
                    } else {
                        ra[i] = pack_bf16x2(low(a[i]) * c.x - low(b[i]) * c.y, high(a[i]) * c.z - high(b[i]) * c.w);
                        rb[i] = pack_bf16x2(low(b[i]) * c.x + low(a[i]) * c.y, high(b[i]) * c.z + high(a[i]) * c.w);
                    }
                }
                p.a = make_uint4(ra[0], ra[1], ra[2], ra[3]);
                p.b = make_uint4(rb[0], rb[1], rb[2], rb[3]);
            }
            *reinterpret_cast<uint4*>(p.to) = p.a;
            if (both) *reinterpret_cast<uint4*>(p.to + other) = p.b;
        };
        while (q[0].token < tokens) {               // (pieces come in order: where the first is past the end, so is the other)
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                finish(q[k]);
                load(q[k]);
            }
        }
    }
}

// A part's values in memory: rows of `extent` bytes, `step` bytes from one to the next.
struct Rows {
    uintptr_t at;
    unsigned long long extent, step, count;
};
// The larger stride counts the rows; false where rows, or heads inside a row, run into each other.
bool rows_of(const void* p, long long token, long long head, long long M, long long heads, long long D, Rows* r) {
    if (M == 1) token = head * heads + D;
    if (heads == 1) head = D;
    const bool by_token = token >= head;
    const long long outer = by_token ? token : head, inner = by_token ? head : token, n_outer = by_token ? M : heads, n_inner = by_token ? heads : M;
    const long long extent = (n_inner - 1) * inner + D;
    if (inner < D || (n_outer > 1 && outer < extent)) return false;
    *r = {reinterpret_cast<uintptr_t>(p), (unsigned long long)extent * 2, (unsigned long long)(n_outer > 1 ? outer : extent) * 2, (unsigned long long)n_outer};
    return true;
}
// Whether two of them may share a byte (rows a fixed step apart: by their places inside the step).
bool meet(const Rows& a, const Rows& b) {
    if (!overlap(Span{reinterpret_cast<const void*>(a.at), (a.count - 1) * a.step + a.extent}, Span{reinterpret_cast<const void*>(b.at), (b.count - 1) * b.step + b.extent}))
        return false;
    if (a.step != b.step || a.count < 2 || b.count < 2) {
        // one row of one of them against the gaps of the other
        const Rows &one = a.count == 1 ? a : b, &many = a.count == 1 ? b : a;
        if (one.count != 1) return true;
        if (one.at < many.at) return one.at + one.extent > many.at;
        const unsigned long long in = (one.at - many.at) % many.step;
        return in < many.extent || in + one.extent > many.step;
    }
    const unsigned long long apart = a.at <= b.at ? (b.at - a.at) % a.step : (a.step - (a.at - b.at) % a.step) % a.step;   // from a row of a to the next of b
    return apart < a.extent || a.step - apart < b.extent;
}

bool multiple_of_8(long long v) { return v >= 0 && v % 8 == 0 && v < (1ll << 40); }

}  // namespace
}  // namespace lowra

extern "C" lowra_status lowra_rotary_turns(int32_t dim, double base, const lowra_rotary_scaling* scaling_host, uint64_t* turns_host, float* scale_host) {
    using namespace lowra;
    if (!scaling_host || !turns_host || !scale_host) return LOWRA_ERR_NULL;
    const lowra_rotary_scaling& S = *scaling_host;
    const int pairs = dim / 2;
    if (dim < 2 || dim % 2 != 0 || dim > 2 * kMostPairs || !(base > 1.0) || !(base < 1e30) || S.kind < LOWRA_ROTARY_NONE || S.kind > LOWRA_ROTARY_BANDS) return LOWRA_ERR_SHAPE;
    if (S.kind != LOWRA_ROTARY_NONE && (!(S.factor >= 1.0) || !(S.factor < 1e9))) return LOWRA_ERR_SHAPE;
    if (S.kind >= LOWRA_ROTARY_YARN && (!(S.original >= 1.0) || !(S.original < 1e12) || !(S.low > 0.0) || !(S.high > S.low) || !(S.high < 1e9))) return LOWRA_ERR_SHAPE;
    const long double two_pi = 2.0L * acosl(-1.0L);
    long double b = base;
    if (S.kind == LOWRA_ROTARY_NTK && dim > 2) b *= powl(S.factor, (long double)dim / (dim - 2));
    long double first = 0.0L, last = 1.0L;                // yarn: pairs up to `first` keep their frequency, from `last` on they are divided
    if (S.kind == LOWRA_ROTARY_YARN) {
        auto place = [&](long double turns) { return dim * logl(S.original / (turns * two_pi)) / (2.0L * logl(b)); };
        first = fmaxl(floorl(place(S.high)), 0.0L);
        last = fminl(ceill(place(S.low)), dim - 1.0L);
        if (last - first < 0.001L) last = first + 0.001L;
    }
    for (int i = 0; i < pairs; ++i) {
        long double f = powl(b, -2.0L * i / dim);
        if (S.kind == LOWRA_ROTARY_LINEAR) f /= S.factor;
        if (S.kind >= LOWRA_ROTARY_YARN) {
            // the share of the frequency that is divided
            const long double t = S.kind == LOWRA_ROTARY_YARN ? (i - first) / (last - first) : 1.0L - (S.original * f / two_pi - S.low) / ((long double)S.high - S.low);
            const long double share = fminl(fmaxl(t, 0.0L), 1.0L);
            f = f * (1.0L - share) + f / S.factor * share;
        }
        long double turn = f / two_pi;
        turn -= floorl(turn);
        const long double scaled = roundl(turn * 18446744073709551616.0L);
        turns_host[i] = scaled >= 18446744073709551616.0L ? 0ull : (uint64_t)scaled;
    }
    *scale_host = S.kind == LOWRA_ROTARY_YARN && S.factor > 1.0 ? (float)(0.1 * log(S.factor) + 1.0) : 1.0f;
    return LOWRA_OK;
}

extern "C" lowra_status lowra_rotary(const lowra_rotary_part* parts_host, int32_t count, int32_t M, int32_t D, int32_t dim, const int32_t* positions_dev,
                                     const uint64_t* turns_dev, float scale, int32_t interleaved, int32_t inverse, void* stream_v) {
    using namespace lowra;
    if (!parts_host || !positions_dev || !turns_dev) return LOWRA_ERR_NULL;
    if (count < 1 || count > LOWRA_MAX_ROTARY_PARTS || M < 1 || M > (1 << 30) || D < 16 || D % 8 != 0 || D > 4096 || dim < 16 || dim % 16 != 0 || dim > D || dim > 2 * kMostPairs)
        return LOWRA_ERR_SHAPE;
    RotaryParams P = {};
    Rows out[LOWRA_MAX_ROTARY_PARTS];
    lowra_rotary_part parts[LOWRA_MAX_ROTARY_PARTS];
    for (int i = 0; i < count; ++i) {
        lowra_rotary_part& p = parts[i] = parts_host[i];
        if (!p.x_dev || !p.out_dev) return LOWRA_ERR_NULL;
        if (M == 1) p.x_token_stride = p.out_token_stride = 0;          // (strides that no step takes)
        if (p.heads == 1) p.x_head_stride = p.out_head_stride = 0;
        if (p.heads < 1 || p.heads > 65536 || !multiple_of_8(p.x_token_stride) || !multiple_of_8(p.x_head_stride) || !multiple_of_8(p.out_token_stride) ||
            !multiple_of_8(p.out_head_stride) || !rows_of(p.out_dev, p.out_token_stride, p.out_head_stride, M, p.heads, D, &out[i]))
            return LOWRA_ERR_SHAPE;
        if (!aligned16(p.x_dev) || !aligned16(p.out_dev)) return LOWRA_ERR_ALIGN;
        const bool same = p.x_dev == p.out_dev && p.x_token_stride == p.out_token_stride && p.x_head_stride == p.out_head_stride;
        P.part[i] = RotaryPart{p.x_dev, p.out_dev, p.x_token_stride, p.x_head_stride, p.out_token_stride, p.out_head_stride, p.heads, same ? 0 : 1};
        P.heads += p.heads;
    }
    if ((reinterpret_cast<uintptr_t>(positions_dev) & 3u) != 0 || !aligned16(turns_dev)) return LOWRA_ERR_ALIGN;
    // An output may be its own input, value for value; else it shares memory with nothing.
    for (int i = 0; i < count; ++i) {
        const Span whole = {parts[i].out_dev, (size_t)((out[i].count - 1) * out[i].step + out[i].extent)};
        if (overlap(whole, Span{positions_dev, (size_t)M * 4}) || overlap(whole, Span{turns_dev, (size_t)dim * 4})) return LOWRA_ERR_SHAPE;
        for (int j = 0; j < count; ++j) {
            if (j != i && j > i && meet(out[i], out[j])) return LOWRA_ERR_SHAPE;
            if (j == i && !P.part[i].copies) continue;
            const lowra_rotary_part& p = parts[j];
            Rows in;
            if (!rows_of(p.x_dev, p.x_token_stride, p.x_head_stride, M, p.heads, D, &in)) {       // (rows read more than once: the whole of them)
                const unsigned long long bytes = 2ull * ((unsigned long long)(M - 1) * p.x_token_stride + (unsigned long long)(p.heads - 1) * p.x_head_stride + D);
                in = Rows{reinterpret_cast<uintptr_t>(p.x_dev), bytes, bytes, 1};
            }
            if (meet(out[i], in)) return LOWRA_ERR_SHAPE;
        }
    }
    const lowra_status st = check_device();
    if (st != LOWRA_OK) return st;
    P.positions = positions_dev;
    P.turns = reinterpret_cast<const unsigned long long*>(turns_dev);
    P.M = M;
    P.D = D;
    P.R = dim;
    P.scale = scale;
    P.interleaved = interleaved != 0;
    P.inverse = inverse != 0;
    const int most = kTablePairs / (dim / 2), ctas = kNumSMs * kRotaryResident;
    P.ranges = M < ctas ? M : ctas;
    P.tokens = (M + P.ranges - 1) / P.ranges;
    if (P.tokens > most) P.tokens = most;
    // fewer tokens than CTAs: several share a token's heads, as long as each has a piece for every other thread
    const long long pieces = (long long)P.heads * (dim / 16 + (D - dim + 15) / 16);
    P.splits = 1;
    while (P.ranges * P.splits * 2 <= ctas && P.splits * 2 <= P.heads && pieces > (long long)P.splits * kRotaryThreads / 2) P.splits *= 2;
    const auto kernel = P.interleaved ? rotary_kernel<true> : rotary_kernel<false>;
    return launch_pdl(kernel, (unsigned)(P.ranges * P.splits), kRotaryThreads, (cudaStream_t)stream_v, P) == cudaSuccess ? LOWRA_OK : LOWRA_ERR_CUDA;
}
