// What the 8-bit operators' kernel files share.  Nothing here is part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bcq.h"

namespace bcq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// One 8-bit product, plain (one matrix) or gated (gate and up), forward or backward.
struct Int8Args {
    const int8_t *q;                // [tokens][n]
    const float *token_scales;      // [tokens]
    const int8_t *w[2];             // [m][n]: the matrix, or gate and up
    const float *channel_scales[2]; // [m]
    int matrices;                   // 1 or 2
    int activation;                 // bcq_activation (gated)
    bool bf16;                      // 16-bit values are bfloat16, else binary16
    uint16_t *y;                    // forward: [tokens][m]
    int64_t m, n, tokens;
    // backward
    const uint16_t *dy;             // [tokens][m]
    uint16_t *dx;                   // [tokens][n]
    float *dscales[2];              // [m]
    void *workspace;
};

constexpr float kGeluTwoK = 1.5957691216057308f;        // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

__device__ __forceinline__ float from_16(uint32_t bits, bool bf16)
{
    return bf16 ? __builtin_bit_cast(float, bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// Rounded to nearest even; a NaN stays one.
__device__ __forceinline__ uint32_t to_16(float v, bool bf16)
{
    if (bf16) return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v);
    return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v);
}

// 1 / (1 + exp(-z)): both of the hardware's approximations are good to about an ulp, and what they make is rounded to 16 bits or
// summed with errors of that size.
__device__ __forceinline__ float sigmoid(float z)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
}

// act(g) and, with SLOPE, act'(g).  Both activations are g sig(z), z = g (silu) or 2 sqrt(2 / pi) (g + 0.044715 g^3) (gelu).
template <bool SLOPE>
__device__ __forceinline__ float activate(float g, int activation, float &slope)
{
    // (the square is held where its products with a sigmoid that is 0 or 1 stay numbers)
    const float g2 = fminf(g * g, 1e30f);
    const bool gelu = activation == BCQ_ACT_GELU;
    const float s = sigmoid(gelu ? kGeluTwoK * (g + kGeluCubic * g2 * g) : g);
    if constexpr (SLOPE) slope = s + g * (s * (1.f - s)) * (gelu ? kGeluTwoK + 3.f * kGeluTwoK * kGeluCubic * g2 : 1.f);
    return g * s;
}

// The backward passes hold the projections' gradients times their channels' scales, G, in binary16 between their two products, times a power of two for
// each token: what lies above 2^-14 has 11 bits then, what lies below is off by up to 2^-25.
// One matrix: G = dy c, and the power brings a token's largest to 2^14.
// Two: dg c_gate and du c_up are both at most 1.13 dh c_gate c_up |s| |sum q w|, of which |sum q w| <= |q| 128 sqrt(n) (|act(g)| <= |g|, |act'| <= 1.13).  The
// power brings the largest such product of the token to between 2^13 and 2^15, so that nothing overflows that has a number for its
// gradient.  What the token's largest really is depends on the weights' codes and on the activation: 2^5 and more where
// those are as usual.  Where it ends below 1 (gates that are all shut, say), the token's gradients are made a second time, with the power that fits.  So
// a gradient is off by up to 2^-11 of itself or 2^-25 of its token's largest.
constexpr int kTop = 14, kGatedTop = 13;                // exponents
constexpr int kMostPower = 126;                         // of a power, either way
constexpr float kFitsFrom = 1.f, kFitsTo = 65000.f;
// Whether a token's first power fits, by its largest G: `some`, there is one between kFitsFrom and kFitsTo; `other`, the largest that is not, as fp32's
// bits.  (Above kFitsTo: only where the scales' product leaves fp32 and a power is 1 at first.)
struct TokenFit {
    uint32_t *some, *other;
};
__device__ __forceinline__ bool power_fits(const TokenFit &fit, int64_t token)
{
    const uint32_t some = fit.some[token];              // (both loads at once)
    const float other = __builtin_bit_cast(float, fit.other[token]);
    return (other == 0.f) | (other == __builtin_inff()) | ((some != 0) & (other <= kFitsTo));
}
__device__ __forceinline__ float token_power(const float *first, const TokenFit &fit, int64_t token)
{
    if (power_fits(fit, token)) return first[token];
    const int e = ilogbf(first[token]) + kTop - ilogbf(__builtin_bit_cast(float, fit.other[token]));
    return ldexpf(1.f, min(max(e, -kMostPower), kMostPower));
}

// The gradients of the channels' scales: a channel's partial sums in order, eight under way at a time.  parts: [count][channels]
__device__ __forceinline__ float sum_of_parts(const float *parts, int64_t count, int64_t channels, int64_t channel)
{
    float sum = 0.f;
    int64_t p = 0;
    for (; p + 8 <= count; p += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = parts[(p + k) * channels + channel];
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += v[k];
    }
    for (; p < count; ++p) sum += parts[p * channels + channel];
    return sum;
}

hipError_t int8_quantize_launch(const uint16_t *x, bool bf16, int8_t *q, float *scales, int64_t rows, int64_t n, hipStream_t stream);

// What a workgroup of the products takes and keeps, as bcq_int8_layout has it
struct Int8Layout {
    int rows, tokens, step, teams, ring, rounds, lds_bytes;
};

// Few tokens: every wave streams rows of weights through LDS of its own.
bool int8_rows_supports(const Int8Args &a);
hipError_t int8_rows_launch(const Int8Args &a, hipStream_t stream);
Int8Layout int8_rows_layout(const Int8Args &a);

// Any number of tokens: tiles of both operands in LDS.
hipError_t int8_tile_launch(const Int8Args &a, hipStream_t stream);
Int8Layout int8_tile_layout(const Int8Args &a, bool backward, bool &mixed);

// The backward passes' workspace, in this order.
struct Int8Workspace {
    int64_t grad_stride;            // halves between tokens: matrices * m rounded up to 64
    int splits;                     // runs of channels whose contributions to dx are summed apart
    int second_shape;               // ... and the tiles that they are taken in
    int64_t grad, powers, some, other, parts, split_sums, bytes;    // offsets in bytes, and the whole
    int64_t part_count;             // room for so many partial sums of a channel
};
Int8Workspace int8_workspace(int matrices, int64_t m, int64_t n, int64_t tokens);
// The gradients of the projections and partial sums of the channel scales' gradients.  again (two matrices): the gradients of the tokens whose power did not
// fit, and with add_up the partial sums' sums.
hipError_t int8_tile_backward_launch(const Int8Args &a, const Int8Workspace &ws, bool again, bool add_up, hipStream_t stream, int64_t &part_count);
hipError_t int8_backward_launch(const Int8Args &a, hipStream_t stream);
// of the second product (rows: columns)
Int8Layout int8_second_layout(const Int8Args &a, int &runs);

}  // namespace bcq
