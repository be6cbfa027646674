// 8-bit products on tiles in LDS, plain and gated, forward and the first half of the backward pass.
//
//   forward    y = s_t c_r sum q w;   gated: act(g) u of two such products, which one wave holds lane by lane
//   backward   the sums again (they are cheaper to make than to keep), and with dy the gradients of the projections,
//              dg = dh u act'(g), du = dh act(g), which the second half multiplies by the weights, and the sums over tokens
//              dc_r = sum_t dg s_t (sum_j q w)
//
// v_mfma_i32_32x32x32_i8, weights as rows and tokens as columns, so that a lane holds four neighbouring channels of one token.  A
// workgroup's tile is ROWS weight rows by TOKS tokens; a step of 128 columns of both (8 and 8 KiB per 64 rows) goes from memory
// into LDS by loads that write there, into one of two buffers while the other is multiplied.  The eight 16-byte parts of an LDS row sit
// XOR-permuted by half the row's number, so that sixteen rows' operand reads use all banks.  A gated tile holds as many rows of gate as of up, by
// turns of half a wave's rows.  Results go through LDS, to be stored in whole rows.
//
// Neighbouring workgroups' numbers go to different XCDs, each with a cache of its own: they are renumbered so that one XCD works on
// the token tiles of the same weights.
#include "bcq_int8.hpp"
#include "bcq_internal.hpp"

namespace bcq {
namespace {

struct TileParams {
    const int8_t *q, *w[2];
    const float *token_scales, *channel_scales[2];
    uint16_t *y;
    uint32_t m, n, tokens;
    uint32_t row_tiles, token_tiles;
    int activation;
    bool bf16, whole;               // whole: rows of y and dy are in pieces of 16 bytes
    // backward
    const uint16_t *dy;
    const float *norms, *scale_top;
    _Float16 *grad;                 // [tokens][grad_stride]: matrix k from k * m_padded on
    uint32_t grad_stride, m_padded;
    float *parts;                   // [token_tiles * WT][matrices][m]
};

// FR x FT tiles of 32 x 32 in a wave, WR x WT waves
template <int WR_, int WT_, int FR_, int FT_>
struct TileShape {
    static constexpr int WR = WR_, WT = WT_, FR = FR_, FT = FT_;
    static constexpr int ROWS = WR * FR * 32, TOKS = WT * FT * 32, WAVES = WR * WT;
};

constexpr int kStep = 128;          // columns, and bytes of an LDS row

template <typename S, int MATS, bool BACKWARD>
struct TileLds {
    static constexpr int STAGE = (S::ROWS + S::TOKS) * kStep;
    static constexpr int CHANNELS = S::ROWS / MATS;
    static constexpr int OUT_ROW = CHANNELS * 2 + 16;
    static constexpr int OUT = S::TOKS * OUT_ROW;           // one 16-bit result tile
    static constexpr int OUTS = BACKWARD ? MATS : 1;
    static constexpr int SCALES = OUTS * OUT;               // the channels' scales behind them
    static constexpr int TOKEN_SCALES = SCALES + MATS * CHANNELS * 4;       // the tokens' scales, and their powers of two
    static constexpr int EPILOGUE = TOKEN_SCALES + 2 * S::TOKS * 4;
    static constexpr int BYTES = 2 * STAGE > EPILOGUE ? 2 * STAGE : EPILOGUE;
};

// Sums over a half wave's 32 lanes of 32 values each: lane l ends with the sum of value l (31 exchanges instead of 160).
__device__ __forceinline__ float sums_of_32(float (&v)[32], int lane)
{
#pragma unroll
    for (int d = 16; d >= 1; d /= 2) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const float keep = upper ? v[i + d] : v[i], give = upper ? v[i] : v[i + d];
            v[i] = keep + __shfl_xor(give, d, 64);
        }
    }
    return v[0];
}

template <typename S, int MATS, bool BACKWARD>
__global__ __launch_bounds__(S::WAVES * 64) void int8_tile_kernel(const TileParams a)
{
    using L = TileLds<S, MATS, BACKWARD>;
    constexpr int FRC = S::FR / MATS;                       // tiles of 32 channels in a wave
    constexpr int CHANNELS = L::CHANNELS;
    static_assert(!BACKWARD || CHANNELS % 64 == 0, "the last tile writes the gradients' rows to their end");
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wr = wave / S::WT, wt = wave % S::WT;
    const int r32 = lane & 31, half = lane >> 5;

    // the tile: first by XCD, then in groups of up to eight token tiles, the tokens of a group running fastest
    const uint32_t total = gridDim.x, xcd = blockIdx.x & 7;
    const uint32_t id = xcd * (total >> 3) + min(xcd, total & 7) + (blockIdx.x >> 3);
    const uint32_t group = id / (8 * a.row_tiles);
    const uint32_t in_group = min(8u, a.token_tiles - group * 8);
    const uint32_t rest = id - group * 8 * a.row_tiles;
    const uint32_t row_tile = rest / in_group, token_tile = group * 8 + rest % in_group;
    const uint32_t ch0 = row_tile * CHANNELS, t0 = token_tile * S::TOKS;

    const uint32_t chs = min((uint32_t)CHANNELS, a.m - ch0), toks = min((uint32_t)S::TOKS, a.tokens - t0);
    const int8_t *const q_base = a.q + (int64_t)t0 * a.n;
    const int8_t *const w_base = a.w[0] + (int64_t)ch0 * a.n, *const u_base = a.w[MATS - 1] + (int64_t)ch0 * a.n;

    // Load k of a stage brings 1 KiB: LDS rows 8k .. 8k+7; lane l delivers the part that belongs at place l % 8 of row 8k + l / 8.
    // Rows and tokens past the end repeat the last one (their results are not stored).
    constexpr int W_LOADS = S::ROWS / 8 / S::WAVES, Q_LOADS = S::TOKS / 8 / S::WAVES;
    static_assert(W_LOADS * 8 * S::WAVES == S::ROWS && Q_LOADS * 8 * S::WAVES == S::TOKS, "whole loads per wave");
    uint32_t w_src[W_LOADS], q_src[Q_LOADS], w_part[W_LOADS], q_part[Q_LOADS];
#pragma unroll
    for (int k = 0; k < W_LOADS; ++k) {
        const uint32_t row = 8 * (wave * W_LOADS + k) + (lane >> 3);
        w_part[k] = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
        const uint32_t in_wave = row % (S::FR * 32);
        const uint32_t ch = MATS == 1 ? row : row / (S::FR * 32) * (FRC * 32) + in_wave % (FRC * 32);
        w_src[k] = min(ch, chs - 1) * a.n;
    }
#pragma unroll
    for (int k = 0; k < Q_LOADS; ++k) {
        const uint32_t tok = 8 * (wave * Q_LOADS + k) + (lane >> 3);
        q_part[k] = ((lane & 7) ^ ((tok >> 1) & 7)) * 16;
        q_src[k] = min(tok, toks - 1) * a.n;
    }
    // Columns k0 .. k0+127 into a buffer.  In the last step parts past the row's end bring the row's first part instead: what is
    // multiplied with them is set to zero.
    auto stage = [&](int buffer, uint32_t k0) {
        unsigned char *to = lds + buffer * L::STAGE;
        const bool last = k0 + kStep > a.n;
        const auto q_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(q_base), 0, (int)(toks * a.n), 0x00020000);
        auto column = [&](uint32_t part) { return last && k0 + part >= a.n ? 0u : k0 + part; };
#pragma unroll
        for (int k = 0; k < W_LOADS; ++k) {
            const int unit = wave * W_LOADS + k;
            const bool up = MATS == 2 && (unit * 8) % (S::FR * 32) >= FRC * 32;
            const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(up ? u_base : w_base), 0, (int)(chs * a.n), 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (__attribute__((address_space(3))) void *)(to + unit * 1024), 16,
                                                     (int)(w_src[k] + column(w_part[k])), 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < Q_LOADS; ++k) {
            const int unit = wave * Q_LOADS + k;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(q_rsrc, (__attribute__((address_space(3))) void *)(to + S::ROWS * kStep + unit * 1024), 16,
                                                     (int)(q_src[k] + column(q_part[k])), 0, 0, 0);
        }
    };

    v16i acc[S::FR][S::FT];
#pragma unroll
    for (int r = 0; r < S::FR; ++r)
#pragma unroll
        for (int t = 0; t < S::FT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[r][t][i] = 0;

    const uint32_t swz = (r32 >> 1) & 7;
    auto multiply = [&](int buffer, int kk, bool there) {
        const unsigned char *from = lds + buffer * L::STAGE + r32 * kStep + (((2 * kk + half) ^ swz) << 4);
        v4i w[S::FR], x[S::FT];
#pragma unroll
        for (int r = 0; r < S::FR; ++r) w[r] = *reinterpret_cast<const v4i *>(from + (wr * S::FR + r) * 32 * kStep);
#pragma unroll
        for (int t = 0; t < S::FT; ++t) {
            x[t] = *reinterpret_cast<const v4i *>(from + S::ROWS * kStep + (wt * S::FT + t) * 32 * kStep);
            if (!there) x[t] = v4i{0, 0, 0, 0};
        }
#pragma unroll
        for (int r = 0; r < S::FR; ++r)
#pragma unroll
            for (int t = 0; t < S::FT; ++t) acc[r][t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[r], x[t], acc[r][t], 0, 0, 0);
    };

    const int steps = (int)(a.n / kStep), tail = (int)(a.n % kStep);
    const int stages = steps + (tail ? 1 : 0);
    stage(0, 0);
    for (int s = 0; s < steps; ++s) {
        // this step's tiles have landed, and nobody reads the other buffer any more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < stages) stage((s + 1) & 1, (uint32_t)(s + 1) * kStep);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) multiply(s & 1, kk, true);
    }
    if (tail) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        for (int kk = 0; kk * 32 < tail; ++kk) multiply(steps & 1, kk, kk * 32 + half * 16 < tail);
    }
    __syncthreads();

    // the channels' and tokens' scales, and in the backward pass the tile of dy
    float *scales = reinterpret_cast<float *>(lds + L::SCALES);
    for (int i = threadIdx.x; i < MATS * CHANNELS; i += S::WAVES * 64) {
        const uint32_t ch = i % CHANNELS;
        scales[i] = ch < chs ? a.channel_scales[i / CHANNELS][ch0 + ch] : 0.f;
    }
    float *token_scales = reinterpret_cast<float *>(lds + L::TOKEN_SCALES);
    [[maybe_unused]] float *norms = token_scales + S::TOKS;
    for (uint32_t i = threadIdx.x; i < S::TOKS; i += S::WAVES * 64) {
        token_scales[i] = a.token_scales[t0 + min(i, toks - 1)];
        if constexpr (BACKWARD) norms[i] = a.norms[t0 + min(i, toks - 1)];
    }
    constexpr int PIECES = CHANNELS / 8;                    // 16-byte pieces of a tile's row
    if constexpr (BACKWARD) {
        if (a.whole) {
            for (int i = threadIdx.x; i < S::TOKS * PIECES; i += S::WAVES * 64) {
                const uint32_t tok = i / PIECES, piece = i % PIECES;
                u32x4 v = {0, 0, 0, 0};
                if (tok < toks && piece * 8 < chs) v = *reinterpret_cast<const u32x4 *>(a.dy + (int64_t)(t0 + tok) * a.m + ch0 + piece * 8);
                *reinterpret_cast<u32x4 *>(lds + tok * L::OUT_ROW + piece * 16) = v;
            }
        } else {
            for (int i = threadIdx.x; i < S::TOKS * CHANNELS; i += S::WAVES * 64) {
                const uint32_t tok = i / CHANNELS, ch = i % CHANNELS;
                *reinterpret_cast<uint16_t *>(lds + tok * L::OUT_ROW + ch * 2) =
                    tok < toks && ch < chs ? a.dy[(int64_t)(t0 + tok) * a.m + ch0 + ch] : (uint16_t)0;
            }
        }
    }
    __syncthreads();

    [[maybe_unused]] float inv_top = 0.f;
    if constexpr (BACKWARD) inv_top = 1.f / *a.scale_top;   // (a power of two)
    // 32 sums over this wave's tokens at a time: a tile of channels of each matrix, or two tiles of the one
    constexpr int TOGETHER = BACKWARD && MATS == 1 ? 2 : 1;
    static_assert(FRC % TOGETHER == 0, "whole exchanges");
#pragma unroll
    for (int r0 = 0; r0 < FRC; r0 += TOGETHER) {
        [[maybe_unused]] float sums[32];
        if constexpr (BACKWARD)
#pragma unroll
            for (int i = 0; i < 32; ++i) sums[i] = 0.f;
#pragma unroll
        for (int r = r0; r < r0 + TOGETHER; ++r)
#pragma unroll
            for (int t = 0; t < S::FT; ++t) {
                const uint32_t tok = (wt * S::FT + t) * 32 + r32;
                const float ts = token_scales[tok];
                [[maybe_unused]] float norm = 0.f;
                if constexpr (BACKWARD) norm = norms[tok];
                const bool here = tok < toks;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int ch = (wr * FRC + r) * 32 + 8 * e + 4 * half;     // element 4 e + i: channel ch + i
                    unsigned char *at = lds + tok * L::OUT_ROW + ch * 2;
                    const v4f c0 = *reinterpret_cast<const v4f *>(scales + ch);
                    const v4f c1 = *reinterpret_cast<const v4f *>(scales + (MATS - 1) * CHANNELS + ch);
                    [[maybe_unused]] u32x2 dy = {0, 0};
                    if constexpr (BACKWARD) dy = *reinterpret_cast<const u32x2 *>(at);
                    uint32_t out[4], out2[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = (float)acc[r][t][4 * e + i] * ts;
                        [[maybe_unused]] float p2 = 0.f, slope = 0.f;
                        if constexpr (MATS == 2) p2 = (float)acc[FRC + r][t][4 * e + i] * ts;
                        if constexpr (!BACKWARD) {
                            float v = p * c0[i];
                            if constexpr (MATS == 2) v = activate<false>(v, a.activation, slope) * (p2 * c1[i]);
                            out[i] = to_16(v, a.bf16);
                        } else {
                            const float d = from_16((i & 1) ? dy[i >> 1] >> 16 : dy[i >> 1] & 0xffffu, a.bf16);
                            const bool inside = here && (uint32_t)(ch + i) < chs;
                            // The gradients that the second half multiplies are held in binary16 (11 bits): a token's by the power of two
                            // that brings its largest dy to about 1/32, times its channel's scale over the power of two above all
                            // scales, so that neither the type's range nor the scales' sizes matter.  A value is off by 2^-12 of
                            // itself, as much as by a result's last rounding.
                            const float k0 = norm * (c0[i] * inv_top);
                            if constexpr (MATS == 1) {
                                out[i] = inside ? to_16(d * k0, false) : 0u;
                                sums[(r - r0) * 16 + 4 * e + i] += inside ? d * p : 0.f;
                            } else {
                                const float act = activate<true>(p * c0[i], a.activation, slope);
                                const float dg = d * (p2 * c1[i]) * slope, du = d * act;
                                out[i] = inside ? to_16(dg * k0, false) : 0u;
                                out2[i] = inside ? to_16(du * (norm * (c1[i] * inv_top)), false) : 0u;
                                sums[4 * e + i] += inside ? dg * p : 0.f;
                                sums[16 + 4 * e + i] += inside ? du * p2 : 0.f;
                            }
                        }
                    }
                    *reinterpret_cast<u32x2 *>(at) = u32x2{out[0] | out[1] << 16, out[2] | out[3] << 16};
                    if constexpr (BACKWARD && MATS == 2)
                        *reinterpret_cast<u32x2 *>(at + L::OUT) = u32x2{out2[0] | out2[1] << 16, out2[2] | out2[3] << 16};
                }
            }
        if constexpr (BACKWARD) {
            // lane l of a half gets value l: element l % 16 of the first or second sixteen
            const float sum = sums_of_32(sums, lane);
            const int second = r32 >> 4, e = (r32 >> 2) & 3, i = r32 & 3;
            const uint32_t ch = (wr * FRC + r0 + (MATS == 1 ? second : 0)) * 32 + 8 * e + 4 * half + i;
            float *parts = a.parts + (int64_t)(token_tile * S::WT + wt) * MATS * a.m;
            if (ch < chs) parts[(int64_t)(MATS == 1 ? 0 : second) * a.m + ch0 + ch] = sum;
        }
    }
    __syncthreads();

    if constexpr (!BACKWARD) {
        if (a.whole) {
            for (int i = threadIdx.x; i < S::TOKS * PIECES; i += S::WAVES * 64) {
                const uint32_t tok = i / PIECES, piece = i % PIECES;
                if (tok < toks && piece * 8 < chs)
                    *reinterpret_cast<u32x4 *>(a.y + (int64_t)(t0 + tok) * a.m + ch0 + piece * 8) =
                        *reinterpret_cast<const u32x4 *>(lds + tok * L::OUT_ROW + piece * 16);
            }
        } else {
            for (int i = threadIdx.x; i < S::TOKS * CHANNELS; i += S::WAVES * 64) {
                const uint32_t tok = i / CHANNELS, ch = i % CHANNELS;
                if (tok < toks && ch < chs) a.y[(int64_t)(t0 + tok) * a.m + ch0 + ch] = *reinterpret_cast<const uint16_t *>(lds + tok * L::OUT_ROW + ch * 2);
            }
        }
    } else {
        // (zeros up to m_padded, which is a multiple of 64)
        for (int i = threadIdx.x; i < MATS * S::TOKS * PIECES; i += S::WAVES * 64) {
            const uint32_t piece = i % PIECES, tok = i / PIECES % S::TOKS, k = i / (PIECES * S::TOKS);
            if (tok < toks && ch0 + piece * 8 < a.m_padded)
                *reinterpret_cast<u32x4 *>(a.grad + (int64_t)(t0 + tok) * a.grad_stride + k * a.m_padded + ch0 + piece * 8) =
                    *reinterpret_cast<const u32x4 *>(lds + k * L::OUT + tok * L::OUT_ROW + piece * 16);
        }
    }
}

template <typename S, int MATS, bool BACKWARD>
hipError_t go(TileParams p, hipStream_t stream, int64_t *part_count)
{
    using L = TileLds<S, MATS, BACKWARD>;
    p.row_tiles = (p.m + L::CHANNELS - 1) / L::CHANNELS;
    p.token_tiles = (p.tokens + S::TOKS - 1) / S::TOKS;
    if (part_count) *part_count = (int64_t)p.token_tiles * S::WT;
    const auto kernel = int8_tile_kernel<S, MATS, BACKWARD>;
    if (hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), L::BYTES)) return e;
    hipLaunchKernelGGL(kernel, dim3(p.row_tiles * p.token_tiles), dim3(S::WAVES * 64), L::BYTES, stream, p);
    return hipGetLastError();
}

using Large = TileShape<2, 4, 4, 2>;        // 256 x 256
using Medium = TileShape<2, 2, 2, 2>;       // 128 x 128
// 64 x 64; in the gated backward pass 128 x 64, so that its channels are a multiple of 64 as the gradients' rows are
template <int MATS, bool BACKWARD> using Small = TileShape<BACKWARD && MATS == 2 ? 2 : 1, 2, 2, 1>;

// The largest tile that leaves no CU without one.
template <int MATS, bool BACKWARD>
hipError_t pick(const TileParams &p, hipStream_t stream, int64_t *part_count = nullptr)
{
    auto tiles = [&](int rows, int toks) { return (int64_t)((p.m * MATS + rows - 1) / rows) * ((p.tokens + toks - 1) / toks); };
    if (tiles(256, 256) >= 256) return go<Large, MATS, BACKWARD>(p, stream, part_count);
    if (tiles(128, 128) >= 256) return go<Medium, MATS, BACKWARD>(p, stream, part_count);
    return go<Small<MATS, BACKWARD>, MATS, BACKWARD>(p, stream, part_count);
}

TileParams params(const Int8Args &a)
{
    TileParams p{};
    p.q = a.q;
    for (int k = 0; k < 2; ++k) {
        p.w[k] = a.w[k];
        p.channel_scales[k] = a.channel_scales[k];
    }
    p.token_scales = a.token_scales;
    p.y = a.y;
    p.dy = a.dy;
    p.m = (uint32_t)a.m;
    p.n = (uint32_t)a.n;
    p.tokens = (uint32_t)a.tokens;
    p.activation = a.activation;
    p.bf16 = a.bf16;
    const void *rows = a.dy ? (const void *)a.dy : a.y;
    p.whole = a.m % 8 == 0 && (reinterpret_cast<uintptr_t>(rows) & 15) == 0;
    return p;
}

}  // namespace

hipError_t int8_tile_launch(const Int8Args &a, hipStream_t stream)
{
    const TileParams p = params(a);
    return a.matrices == 2 ? pick<2, false>(p, stream) : pick<1, false>(p, stream);
}

hipError_t int8_tile_backward_launch(const Int8Args &a, const Int8Workspace &ws, hipStream_t stream, int64_t &part_count)
{
    TileParams p = params(a);
    unsigned char *base = static_cast<unsigned char *>(a.workspace);
    p.grad = reinterpret_cast<_Float16 *>(base + ws.grad);
    p.norms = reinterpret_cast<const float *>(base + ws.norms);
    p.scale_top = reinterpret_cast<const float *>(base + ws.scale_top);
    p.parts = reinterpret_cast<float *>(base + ws.parts);
    p.grad_stride = (uint32_t)ws.grad_stride;
    p.m_padded = (uint32_t)(ws.grad_stride / a.matrices);
    return a.matrices == 2 ? pick<2, true>(p, stream, &part_count) : pick<1, true>(p, stream, &part_count);
}

}  // namespace bcq
