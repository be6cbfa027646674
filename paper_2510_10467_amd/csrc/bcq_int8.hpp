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

// The backward passes hold a projection's gradients G in binary16, scaled so that a token's are of the order of 1 whatever dy, the token's scale and
// the channels' are: times `norm`, the power of two that brings the token's largest |dy| to kPlainTop (one matrix: G = dy c) or kGatedTop, and over
// the power of two next to what the other projection is typically made of, |token_scale| top 73 73 sqrt(n) (codes spread evenly have a mean
// square of 73^2).  It is at most 128 128 n / (73 73 sqrt(n)) = 1113 times that, so with slopes of at most 1.13 a scaled G stays below
// 2 kGatedTop 2 1113 1.13 = 40300: nothing overflows that has a number for its gradient.
constexpr int kPlainTop = 9, kGatedTop = 3;             // exponents
__device__ __forceinline__ float gradient_power(float norm, float token_scale, float top, float typical)
{
    const float size = fabsf(token_scale) * top * typical;              // (typical: 73 73 sqrt(n), or 0 for one matrix)
    if (!(size > 0.f && size < __builtin_inff())) return norm;
    return ldexpf(1.f, min(max(ilogbf(norm) - ilogbf(size), -120), 120));
}

hipError_t int8_quantize_launch(const uint16_t *x, bool bf16, int8_t *q, float *scales, int64_t rows, int64_t n, hipStream_t stream);

// Few tokens: every wave streams rows of weights through LDS of its own.
bool int8_rows_supports(const Int8Args &a);
hipError_t int8_rows_launch(const Int8Args &a, hipStream_t stream);

// Any number of tokens: tiles of both operands in LDS.
hipError_t int8_tile_launch(const Int8Args &a, hipStream_t stream);

// The backward passes' workspace, in this order.
struct Int8Workspace {
    int64_t grad_stride;            // halves between tokens: matrices * m rounded up to 64
    int splits;                     // runs of channels whose contributions to dx are summed apart
    int second_shape;               // ... and the tiles that they are taken in
    int64_t grad, norms, scale_top, parts, split_sums, bytes;       // offsets in bytes, and the whole
    int64_t part_count;             // room for so many partial sums of a channel
    float typical;                  // what gradient_power counts with
};
Int8Workspace int8_workspace(int matrices, int64_t m, int64_t n, int64_t tokens);
// the gradients of the projections, scaled as int8_backward_* explains, and partial sums of the channel scales' gradients
hipError_t int8_tile_backward_launch(const Int8Args &a, const Int8Workspace &ws, hipStream_t stream, int64_t &part_count);
hipError_t int8_backward_launch(const Int8Args &a, hipStream_t stream);

}  // namespace bcq
