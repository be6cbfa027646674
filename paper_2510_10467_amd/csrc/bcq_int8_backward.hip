// The backward passes of the 8-bit products, codes fixed: gradients of the activations and of the channel scales.
//
//   powers    per token the power of two, f_t, that brings its gradients to where binary16 holds them best, as far as that is known beforehand
//   first     (bcq_int8_tile.hip) G = binary16 of f_t dg c for every channel of every matrix, the largest of each token, and partial sums of dc
//   again     two matrices: G once more, by the largest, of tiles with tokens whose f_t did not fit; hardly ever more than a look
//   second    dx = (1 / f_t) sum over channels of G w: a product over the weights' ROWS
//   finish    dc: the partial sums of a channel, in order; dx where the channels were taken in several runs: the runs' sums, in order
//
// The second product runs on v_mfma_f32_32x32x16_f16.  Both operands go into LDS by loads that write there, the weights as they are stored: 64
// rows of 8-bit codes by a tile's columns.  A lane needs eight codes of one column, which is what the transposing LDS read of
// 8-bit values delivers (16 lanes take eight rows of 16 columns), and turns them into binary16, exactly: a code's byte
// with its sign bit turned under the byte 0x64 is the number 1024 + 128 + code.
//
// What bounds it: the power of the matrix pipe on random operands (2048 tokens, 4096 columns, 2 x 14336 channels: 437 to 459 us = 1100 to 1050 TFLOP/s,
// with gradients of zero 330; the library's plain binary16 product of 8192^3 1300), the codes' conversion beside it, and with few tokens
// the weights' bytes (17920 x 5120, gated, 48 tokens: 47 us = 3.9 TB/s).  The whole gated backward pass of 2048 tokens: 713 to 745 us; the
// profiler, which counts the time that two launches overlap twice, has 18 for the powers, 295 for the first half, 5 for the second look with the sums, 447
// for the second half.
#include <math.h>

#include "bcq_int8.hpp"
#include "bcq_internal.hpp"

namespace bcq {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v2i __attribute__((ext_vector_type(2)));

// A token's power of two from the largest |dy c| of its channels, or, where there are two matrices, |dh c_gate c_up| and its codes' length.  A workgroup takes TOKENS of
// them, which share the channels' scales on their way (2048 tokens, 14336 channels: one each 24 us, four 18).
template <int TOKENS, int MATS>
__global__ __launch_bounds__(256) void int8_powers_kernel(const uint16_t *__restrict__ dy, const float *__restrict__ c0, const float *__restrict__ c1,
                                                          const int8_t *__restrict__ q, const float *__restrict__ token_scales,
                                                          float *__restrict__ powers, const TokenFit fit, int64_t m, int64_t n, int64_t tokens, bool bf16,
                                                          bool whole)
{
    __shared__ float tops[TOKENS][4];
    __shared__ int squares[TOKENS][4];
    const int64_t token0 = (int64_t)blockIdx.x * TOKENS;
    const int last = (int)m - 1;                        // what lies past the end counts the last value again
    const uint16_t *row[TOKENS];
    float top[TOKENS];                                  // (a NaN leaves it as it is: such a token's results are NaN whatever its power)
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        row[t] = dy + min(token0 + t, tokens - 1) * m;
        top[t] = 0.f;
    }
    auto take = [&](int t, uint32_t bits, float a, float b) {
        float v = fabsf(from_16(bits, bf16)) * fabsf(a);
        if constexpr (MATS == 2) v *= fabsf(b);
        top[t] = fmaxf(top[t], v);
    };
    v4i code[TOKENS];                                   // (asked for before what follows)
    if constexpr (MATS == 2)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) code[t] = reinterpret_cast<const v4i *>(q + min(token0 + t, tokens - 1) * n)[min((int)threadIdx.x, (int)(n / 16) - 1)];
    constexpr int AT_ONCE = TOKENS == 1 ? 2 : 1;
    if (whole) {
        const int last_piece = (int)(m / 8) - 1;
        for (int j = threadIdx.x; j <= last_piece; j += AT_ONCE * 256) {
            u32x4 v[AT_ONCE][TOKENS];
            v4f a[AT_ONCE][2], b[AT_ONCE][2];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int piece = min(j + k * 256, last_piece);
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) v[k][t] = reinterpret_cast<const u32x4 *>(row[t])[piece];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    a[k][h] = reinterpret_cast<const v4f *>(c0)[2 * piece + h];
                    b[k][h] = MATS == 2 ? reinterpret_cast<const v4f *>(c1)[2 * piece + h] : a[k][h];
                }
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                for (int t = 0; t < TOKENS; ++t)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        take(t, (i & 1) ? v[k][t][i >> 1] >> 16 : v[k][t][i >> 1] & 0xffffu, a[k][i >> 2][i & 3], b[k][i >> 2][i & 3]);
        }
    } else {
        for (int j = threadIdx.x; j <= last; j += 1024) {
            uint32_t v[4][TOKENS];
            float a[4], b[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = min(j + k * 256, last);
                a[k] = c0[at];
                b[k] = MATS == 2 ? c1[at] : 0.f;
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) v[k][t] = row[t][at];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) take(t, v[k][t], a[k], b[k]);
        }
    }
    int square[TOKENS];                                 // (131056 squares of 128 stay below 2^31)
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) square[t] = 0;
    if constexpr (MATS == 2)
        for (int j = threadIdx.x; j < (int)(n / 16); j += 256)
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) square[t] = __builtin_amdgcn_sdot4(code[t][i], code[t][i], square[t], false);
                if (j + 256 < (int)(n / 16)) code[t] = reinterpret_cast<const v4i *>(q + min(token0 + t, tokens - 1) * n)[j + 256];
            }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            top[t] = fmaxf(top[t], __shfl_xor(top[t], d, 64));
            if constexpr (MATS == 2) square[t] += __shfl_xor(square[t], d, 64);
        }
        if ((threadIdx.x & 63) == 0) {
            tops[t][threadIdx.x >> 6] = top[t];
            squares[t][threadIdx.x >> 6] = square[t];
        }
    }
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= TOKENS || token0 + t >= tokens) return;
    auto usable = [](float v) { return v > 0.f && v < __builtin_inff(); };
    const float most = fmaxf(fmaxf(tops[t][0], tops[t][1]), fmaxf(tops[t][2], tops[t][3]));
    int e = usable(most) ? (MATS == 2 ? kGatedTop : kTop) - ilogbf(most) : 0;
    if constexpr (MATS == 2) {
        const float length = sqrtf((float)(squares[t][0] + squares[t][1] + squares[t][2] + squares[t][3]));
        const float sums = fabsf(token_scales[token0 + t]) * (1.13f * 128.f * sqrtf((float)n) * length);
        // (with either beyond fp32 the gradients' size is anywhere: as they are at first)
        e = usable(most) && usable(sums) ? e - ilogbf(sums) : 0;
        fit.some[token0 + t] = fit.other[token0 + t] = 0;
    }
    powers[token0 + t] = ldexpf(1.f, min(max(e, -kMostPower), kMostPower));
}

constexpr uint32_t kTokenGroup = 4;       // token tiles whose workgroups run beside each other for a column tile

struct SecondParams {
    const _Float16 *grad;
    const int8_t *w[2];
    const float *powers;
    TokenFit fit;
    uint16_t *dx;
    uint32_t m, m_padded, n, tokens, grad_stride;
    uint32_t column_tiles, token_tiles;
    int matrices;
    bool bf16;
    // the steps in `splits` runs, each its own grid row, whose sums go to split_sums [splits][tokens][n] (one run: straight to dx)
    int splits;
    float *split_sums;
};

// FC x FT tiles of 32 columns x 32 tokens in a wave, WC x WT waves in a team, RING buffers of each team, STEP rows of the weights at a time
template <int WC_, int WT_, int FC_, int FT_, int RING_, int TEAMS_ = 1, int STEP_ = 64, bool ACROSS_ = (RING_ >= 4)>
struct SecondShape {
    static constexpr int WC = WC_, WT = WT_, FC = FC_, FT = FT_, RING = RING_, TEAMS = TEAMS_, STEP = STEP_;
    static constexpr bool ACROSS = ACROSS_;
    static constexpr int COLS = WC * FC * 32, TOKS = WT * FT * 32, TEAM_WAVES = WC * WT, WAVES = TEAMS * TEAM_WAVES;
    static constexpr int G_ROW = STEP * 2, W_BYTES = STEP * COLS, STAGE = W_BYTES + TOKS * G_ROW;
    static constexpr int PLACES = G_ROW / 16, LOAD_TOKS = 64 / PLACES;          // 16-byte parts of a token's row in LDS, tokens of a load
    static constexpr __device__ __host__ uint32_t swizzle(uint32_t tok) { return tok * PLACES / 16 % PLACES; }
    static constexpr int OUT_ROW = COLS * 2 + 16, OUT = TOKS * OUT_ROW;
    static constexpr int RINGS = TEAMS * RING * STAGE, EXCHANGE = (TEAMS - 1) * COLS * TOKS * 4;
    static constexpr int BYTES = RINGS > OUT ? (RINGS > EXCHANGE ? RINGS : EXCHANGE) : (OUT > EXCHANGE ? OUT : EXCHANGE);
};

// Eight codes to binary16: 1024 + (code + 128), less 1152.
__device__ __forceinline__ v8h halves_of(v2i codes)
{
    u32x4 out;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t c = (uint32_t)codes[k] ^ 0x80808080u;
        const v2h bias = {(_Float16)1152.f, (_Float16)1152.f};
        out[2 * k] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, c, 0x04010400u)) - bias);
        out[2 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, c, 0x04030402u)) - bias);
    }
    return __builtin_bit_cast(v8h, out);
}

// A step is STEP rows of the weights: an LDS row holds COLS codes, its 16-byte parts XOR-permuted by the row's number; a token's STEP
// gradients are a row too, permuted as in the first half.
template <typename S>
__global__ __launch_bounds__(S::WAVES * 64, 2) void int8_second_kernel(const SecondParams a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int team = wave / S::TEAM_WAVES, tw = wave % S::TEAM_WAVES;
    const int wc = tw / S::WT, wt = tw % S::WT;
    const int r32 = lane & 31, half = lane >> 5;

    const uint32_t total = gridDim.x, xcd = blockIdx.x & 7;
    const uint32_t id = xcd * (total >> 3) + min(xcd, total & 7) + (blockIdx.x >> 3);
    const uint32_t group = id / (kTokenGroup * a.column_tiles);
    const uint32_t in_group = min(kTokenGroup, a.token_tiles - group * kTokenGroup);
    const uint32_t rest = id - group * kTokenGroup * a.column_tiles;
    const uint32_t c0 = rest / in_group * S::COLS, t0 = (group * kTokenGroup + rest % in_group) * S::TOKS;
    const uint32_t cols = min((uint32_t)S::COLS, a.n - c0), toks = min((uint32_t)S::TOKS, a.tokens - t0);

    constexpr int W_LOADS = S::W_BYTES / 1024 / S::TEAM_WAVES, G_LOADS = S::TOKS / S::LOAD_TOKS / S::TEAM_WAVES;
    constexpr int PARTS = S::COLS / 16, ROWS_PER = 64 / PARTS;          // parts of an LDS row, rows of a load
    static_assert(W_LOADS * 1024 * S::TEAM_WAVES == S::W_BYTES && G_LOADS * S::LOAD_TOKS * S::TEAM_WAVES == S::TOKS, "whole loads per wave");
    uint32_t g_src[G_LOADS];
#pragma unroll
    for (int k = 0; k < G_LOADS; ++k) {
        const uint32_t tok = S::LOAD_TOKS * (tw * G_LOADS + k) + lane / S::PLACES;
        g_src[k] = min(tok, toks - 1) * a.grad_stride * 2 + (lane % S::PLACES ^ S::swizzle(tok)) * 16;
    }
    // load k of the weights: rows ROWS_PER * unit .. of the step, place lane % PARTS (columns past the end bring the last part)
    uint32_t w_row[W_LOADS], w_col[W_LOADS];
#pragma unroll
    for (int k = 0; k < W_LOADS; ++k) {
        w_row[k] = (tw * W_LOADS + k) * ROWS_PER + lane / PARTS;
        w_col[k] = min((uint32_t)((lane % PARTS) ^ (w_row[k] & (PARTS - 1))) * 16, cols - 16);
    }
    const _Float16 *const g_base = a.grad + (int64_t)t0 * a.grad_stride;
    const uint32_t per_matrix = a.m_padded / S::STEP;
    const int all_steps = (int)(per_matrix * a.matrices), run = (all_steps + a.splits - 1) / a.splits;
    const int first_step = (int)blockIdx.y * run, steps = max(0, min(run, all_steps - first_step));
    unsigned char *const mine = lds + team * S::RING * S::STAGE;        // the team's ring
    // Rows past a matrix's end repeat its last one: the gradients there are zeros.
    auto stage = [&](int buffer, uint32_t of_run) {
        unsigned char *to = mine + buffer * S::STAGE;
        const uint32_t s = first_step + of_run;
        const uint32_t k = s >= per_matrix ? 1 : 0, row0 = min((s - k * per_matrix) * S::STEP, a.m - 1);
        const uint32_t rows = min((uint32_t)S::STEP, a.m - row0);
        const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>((k ? a.w[1] : a.w[0]) + (int64_t)row0 * a.n + c0), 0,
                                                              (int)((rows - 1) * a.n + cols), 0x00020000);
        const auto g_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<_Float16 *>(g_base), 0, (int)(toks * a.grad_stride * 2), 0x00020000);
#pragma unroll
        for (int j = 0; j < W_LOADS; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (__attribute__((address_space(3))) void *)(to + (tw * W_LOADS + j) * 1024), 16,
                                                     (int)(min(w_row[j], rows - 1) * a.n + w_col[j]), 0, 0, 0);
#pragma unroll
        for (int j = 0; j < G_LOADS; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(g_rsrc, (__attribute__((address_space(3))) void *)(to + S::W_BYTES + (tw * G_LOADS + j) * 1024), 16,
                                                     (int)g_src[j], (int)(s * S::G_ROW), 0, 0);
    };

    v16f acc[S::FC][S::FT];
#pragma unroll
    for (int c = 0; c < S::FC; ++c)
#pragma unroll
        for (int t = 0; t < S::FT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c][t][i] = 0.f;

    const uint32_t swz = S::swizzle(r32);
    // the transposing read: lanes 2 r and 2 r + 1 of sixteen point at the halves of row r's 16 columns; lanes 0-31 take rows 0-7 of a
    // step of 16, lanes 32-63 rows 8-15, of which every second sixteen the next 16 columns
    const int tr_row = half * 8 + ((lane & 15) >> 1);
    struct Operands {
        v8h w[S::FC], g[S::FT];
    };
    auto operands = [&](int buffer, int kk) {
        const unsigned char *from = mine + buffer * S::STAGE;
        v2i raw[S::FC];
        Operands o;
#pragma unroll
        for (int c = 0; c < S::FC; ++c) {
            const int row = kk * 16 + tr_row;
            const int part = (wc * S::FC + c) * 2 + ((lane >> 4) & 1);
            const unsigned char *at = from + row * S::COLS + ((part ^ (row & (PARTS - 1))) << 4) + (lane & 1) * 8;
            raw[c] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i *)at);
        }
#pragma unroll
        for (int t = 0; t < S::FT; ++t)
            o.g[t] = *reinterpret_cast<const v8h *>(from + S::W_BYTES + ((wt * S::FT + t) * 32 + r32) * S::G_ROW + (((2 * kk + half) ^ swz) << 4));
#pragma unroll
        for (int c = 0; c < S::FC; ++c) o.w[c] = halves_of(raw[c]);
        return o;
    };
    auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int c = 0; c < S::FC; ++c)
#pragma unroll
            for (int t = 0; t < S::FT; ++t) acc[c][t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o.w[c], o.g[t], acc[c][t], 0, 0, 0);
    };
    // (as in the first half; between the matrix instructions first the reads, then the codes' conversion)
    [[maybe_unused]] Operands now;
    auto whole_step = [&](int buffer, int after) {
#pragma unroll
        for (int kk = 0; kk < S::STEP / 16; ++kk) {
            if constexpr (S::ACROSS) {
                const Operands later = kk + 1 < S::STEP / 16 ? operands(buffer, kk + 1) : operands(after, 0);
                multiply(now);
                now = later;
                constexpr int PRODUCTS = S::FC * S::FT, BETWEEN = PRODUCTS > 1 ? (10 * S::FC + PRODUCTS - 2) / (PRODUCTS - 1) : 1;
                __builtin_amdgcn_sched_group_barrier(0x100, S::FC, 0);
#pragma unroll
                for (int i = 0; i < PRODUCTS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    if (i < S::FT) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    if (i > 0) __builtin_amdgcn_sched_group_barrier(0x002, BETWEEN, 0);
                }
            } else {
                multiply(operands(buffer, kk));
            }
        }
    };

    constexpr int AHEAD = S::RING - 1, LOADS = W_LOADS + G_LOADS;
    static_assert(S::RING >= 3 || !S::ACROSS, "a step reads the next one's first operands");
    const int rounds = (steps + S::TEAMS - 1) / S::TEAMS;
    auto step = [&](int i) { return i * S::TEAMS + team; };
    for (int i = 0; i < min(AHEAD, rounds); ++i)
        if (step(i) < steps) stage(i, (uint32_t)step(i));
    if (rounds > AHEAD) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((AHEAD - 1) * LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    if (S::ACROSS) now = operands(0, 0);
    int buffer = 0, into = AHEAD, i = 0;
    auto next = [](int b) { return b + 1 == S::RING ? 0 : b + 1; };
    for (; i + AHEAD < rounds; ++i) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - (S::ACROSS ? 2 : 1)) * LOADS) : "memory");
        if (S::TEAMS == 1 || step(i + AHEAD) < steps) stage(into, (uint32_t)step(i + AHEAD));
        whole_step(buffer, next(buffer));
        buffer = next(buffer);
        into = next(into);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    for (; step(i) < steps; ++i) {
        whole_step(buffer, next(buffer));
        buffer = next(buffer);
    }
    __syncthreads();
    if constexpr (S::TEAMS > 1) {
        v4f *const exchange = reinterpret_cast<v4f *>(lds) + tw * (S::FC * S::FT * 4 * 64) + lane;
        constexpr int BETWEEN = S::TEAM_WAVES * S::FC * S::FT * 4 * 64;
        if (team > 0) {
#pragma unroll
            for (int c = 0; c < S::FC; ++c)
#pragma unroll
                for (int t = 0; t < S::FT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        exchange[(team - 1) * BETWEEN + ((c * S::FT + t) * 4 + e) * 64] =
                            v4f{acc[c][t][4 * e], acc[c][t][4 * e + 1], acc[c][t][4 * e + 2], acc[c][t][4 * e + 3]};
        }
        __syncthreads();
        if (team == 0) {
#pragma unroll
            for (int k = 0; k < S::TEAMS - 1; ++k)
#pragma unroll
                for (int c = 0; c < S::FC; ++c)
#pragma unroll
                    for (int t = 0; t < S::FT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const v4f v = exchange[k * BETWEEN + ((c * S::FT + t) * 4 + e) * 64];
#pragma unroll
                            for (int x = 0; x < 4; ++x) acc[c][t][4 * e + x] += v[x];
                        }
        }
        __syncthreads();
    }

    if (a.splits > 1) {
        if (team > 0) return;
#pragma unroll
        for (int t = 0; t < S::FT; ++t) {
            const uint32_t tok = (wt * S::FT + t) * 32 + r32;
#pragma unroll
            for (int c = 0; c < S::FC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t col = (wc * S::FC + c) * 32 + 8 * e + 4 * half;
                    if (tok < toks && col < cols)           // (columns come in sixteens)
                        *reinterpret_cast<v4f *>(a.split_sums + ((int64_t)blockIdx.y * a.tokens + t0 + tok) * a.n + c0 + col) =
                            v4f{acc[c][t][4 * e], acc[c][t][4 * e + 1], acc[c][t][4 * e + 2], acc[c][t][4 * e + 3]};
                }
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < (team == 0 ? S::FT : 0); ++t) {
        const uint32_t tok = (wt * S::FT + t) * 32 + r32;
        const uint32_t at = t0 + min(tok, toks - 1);
        const float back = 1.f / (a.matrices == 2 ? token_power(a.powers, a.fit, at) : a.powers[at]);     // (powers of two)
#pragma unroll
        for (int c = 0; c < S::FC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = (wc * S::FC + c) * 32 + 8 * e + 4 * half;
                uint32_t out[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = to_16(acc[c][t][4 * e + i] * back, a.bf16);
                *reinterpret_cast<u32x2 *>(lds + tok * S::OUT_ROW + col * 2) = u32x2{out[0] | out[1] << 16, out[2] | out[3] << 16};
            }
    }
    __syncthreads();
    constexpr int PIECES = S::COLS / 8;
    for (int i = threadIdx.x; i < S::TOKS * PIECES; i += S::WAVES * 64) {
        const uint32_t tok = i / PIECES, piece = i % PIECES;
        if (tok < toks && piece * 8 < cols)
            *reinterpret_cast<u32x4 *>(a.dx + (int64_t)(t0 + tok) * a.n + c0 + piece * 8) = *reinterpret_cast<const u32x4 *>(lds + tok * S::OUT_ROW + piece * 16);
    }
}

// What is left, in one launch: the first sums_blocks workgroups add up the partial sums of the scales' gradients, a channel a thread; the
// others the runs' sums of dx, four columns a thread.
struct FinishParams {
    const float *parts, *split_sums, *powers;
    TokenFit fit;
    float *dscales[2];
    uint16_t *dx;
    int64_t m, part_count, tokens;
    uint32_t n, sums_blocks;
    int matrices, splits;
    bool bf16;
};

__global__ __launch_bounds__(64) void int8_finish_kernel(const FinishParams a)
{
    if (blockIdx.x < a.sums_blocks) {
        const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x, channels = a.m * a.matrices;
        if (i >= channels) return;
        const float sum = sum_of_parts(a.parts, a.part_count, channels, i);
        if (i < a.m) a.dscales[0][i] = sum;
        else a.dscales[1][i - a.m] = sum;
        return;
    }
    const int64_t i = (int64_t)(blockIdx.x - a.sums_blocks) * 64 + threadIdx.x, count = a.tokens * a.n / 4;
    if (i >= count) return;
    v4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) sum += reinterpret_cast<const v4f *>(a.split_sums)[s * count + i];
    const int64_t token = i * 4 / a.n;
    const float back = 1.f / (a.matrices == 2 ? token_power(a.powers, a.fit, token) : a.powers[token]);     // (powers of two)
    uint32_t out[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = to_16(sum[k] * back, a.bf16);
    reinterpret_cast<u32x2 *>(a.dx)[i] = u32x2{out[0] | out[1] << 16, out[2] | out[3] << 16};
}

template <typename S>
hipError_t go(SecondParams p, hipStream_t stream)
{
    p.column_tiles = (p.n + S::COLS - 1) / S::COLS;
    p.token_tiles = (p.tokens + S::TOKS - 1) / S::TOKS;
    const auto kernel = int8_second_kernel<S>;
    if (hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), S::BYTES)) return e;
    hipLaunchKernelGGL(kernel, dim3(p.column_tiles * p.token_tiles, (unsigned)p.splits), dim3(S::WAVES * 64), S::BYTES, stream, p);
    return hipGetLastError();
}

// What a workgroup takes per step of 64 channels, alone on its CU and as one of two or more, each (microseconds, measured: gemm, 14336 x 4096 with 32 to
// 128 tokens, 4096 x 14336 with 512).  A wave turns a code into binary16 for all of its tile's tokens: with 32 columns of it in a wave instead of 64, twice, the
// second half of 4096 x 14336 with 512 tokens went from 70 to 65 us.
template <typename F>
void for_shapes(F f)
{
    f(SecondShape<8, 1, 1, 4, 2, 2>{}, 0.85f, 1.02f);       // 256 columns x 128 tokens, two teams
    f(SecondShape<4, 1, 1, 4, 3>{}, 0.50f, 0.56f);          // 128 x 128: two share a CU
    f(SecondShape<4, 1, 1, 2, 2, 2>{}, 0.50f, 0.40f);       // 128 x 64, two teams: two share a CU
    f(SecondShape<2, 2, 1, 1, 4, 2>{}, 0.40f, 0.40f);       // 64 x 64, two teams
}

// The shape, and in how many runs the channels are taken where few columns and tokens leave CUs without work: what is expected to be done first, with
// four steps for a workgroup's start and end, and the runs' sums, written and read, at 8 TB/s.  (4096 columns, 48 tokens, 2 x 14336 channels, the
// whole pass: 161 us in two runs, 101 in four, 74 in eight, 70 in 16.)
struct SecondPlan {
    int shape, splits;
};
SecondPlan second_plan(int matrices, int64_t m, int64_t n, int64_t tokens)
{
    const int64_t steps = matrices * ((m + 63) / 64);
    SecondPlan plan{0, 1};
    float best = 0.f;
    int index = 0;
    for_shapes([&](auto shape, float alone, float shared) {
        using S = decltype(shape);
        const int64_t tiles = ((n + S::COLS - 1) / S::COLS) * ((tokens + S::TOKS - 1) / S::TOKS);
        for (int splits = 1; splits <= 16; ++splits) {
            const int64_t run = (steps + splits - 1) / splits, each = (tiles * splits + 255) / 256;
            if (splits > 1 && (run < 4 || tokens * n > int64_t(1) << 32)) break;        // (the finish counts its threads in 32 bits)
            const float us = (float)(run + 4) * (each <= 1 ? alone : (float)each * shared) +
                             (splits > 1 ? 1.f + (float)splits * (float)tokens * (float)n * (8.f / 8e6f) : 0.f);
            if (best == 0.f || us < best) {
                best = us;
                plan = {index, splits};
            }
        }
        ++index;
    });
    return plan;
}

template <int TOKENS, int MATS>
hipError_t powers_go(const Int8Args &a, float *powers, const TokenFit &fit, hipStream_t stream)
{
    const float *c0 = a.channel_scales[0], *c1 = a.channel_scales[MATS - 1];
    const bool whole = a.m % 8 == 0 && ((reinterpret_cast<uintptr_t>(a.dy) | reinterpret_cast<uintptr_t>(c0) | reinterpret_cast<uintptr_t>(c1)) & 15) == 0;
    hipLaunchKernelGGL((int8_powers_kernel<TOKENS, MATS>), dim3((unsigned)((a.tokens + TOKENS - 1) / TOKENS)), dim3(256), 0, stream, a.dy, c0, c1, a.q,
                       a.token_scales, powers, fit, a.m, a.n, a.tokens, a.bf16, whole);
    return hipGetLastError();
}

hipError_t powers_launch(const Int8Args &a, float *powers, const TokenFit &fit, hipStream_t stream)
{
    if (a.tokens >= 1024) return a.matrices == 2 ? powers_go<4, 2>(a, powers, fit, stream) : powers_go<4, 1>(a, powers, fit, stream);
    return a.matrices == 2 ? powers_go<1, 2>(a, powers, fit, stream) : powers_go<1, 1>(a, powers, fit, stream);
}

}  // namespace

Int8Workspace int8_workspace(int matrices, int64_t m, int64_t n, int64_t tokens)
{
    Int8Workspace ws;
    auto up = [](int64_t bytes) { return (bytes + 255) / 256 * 256; };
    ws.grad_stride = matrices * ((m + 63) / 64 * 64);
    ws.part_count = (tokens + 63) / 64 * 2 + 2;             // at most: a wave's tokens are 64, or 32 in tiles of 64 and 32
    const SecondPlan plan = second_plan(matrices, m, n, tokens);
    ws.second_shape = plan.shape;
    ws.splits = plan.splits;
    ws.grad = 0;
    ws.powers = up(tokens * ws.grad_stride * 2);
    ws.some = ws.powers + up(tokens * 4);
    ws.other = ws.some + (matrices == 2 ? up(tokens * 4) : 0);
    ws.parts = ws.other + (matrices == 2 ? up(tokens * 4) : 0);
    ws.split_sums = ws.parts + up(ws.part_count * matrices * m * 4);
    ws.bytes = ws.split_sums + (ws.splits > 1 ? up(ws.splits * tokens * n * 4) : 0);
    return ws;
}

Int8Layout int8_second_layout(const Int8Args &a, int &runs)
{
    const SecondPlan plan = second_plan(a.matrices, a.m, a.n, a.tokens);
    runs = plan.splits;
    Int8Layout layout{};
    int index = 0;
    for_shapes([&](auto shape, float, float) {
        using S = decltype(shape);
        if (index++ != plan.shape) return;
        const int64_t steps = a.matrices * ((a.m + 63) / 64), run = (steps + runs - 1) / runs;
        layout = {S::COLS, S::TOKS, S::STEP, S::TEAMS, S::RING, (int)((run + S::TEAMS - 1) / S::TEAMS), S::BYTES};
    });
    return layout;
}

hipError_t int8_backward_launch(const Int8Args &a, hipStream_t stream)
{
    const Int8Workspace ws = int8_workspace(a.matrices, a.m, a.n, a.tokens);
    unsigned char *base = static_cast<unsigned char *>(a.workspace);
    float *powers = reinterpret_cast<float *>(base + ws.powers), *split_sums = reinterpret_cast<float *>(base + ws.split_sums);
    const TokenFit fit = {reinterpret_cast<uint32_t *>(base + ws.some), reinterpret_cast<uint32_t *>(base + ws.other)};
    // The scales' gradients are added up in the launch that adds up the runs of dx, or, where there is none and two matrices, in the second look at the gradients.
    const bool runs = ws.splits > 1 && a.tokens > 0, finish = runs || a.matrices == 1 || a.tokens == 0;
    int64_t part_count = 0;
    if (a.tokens > 0) {
        if (hipError_t e = powers_launch(a, powers, fit, stream)) return e;
        if (hipError_t e = int8_tile_backward_launch(a, ws, false, false, stream, part_count)) return e;
        if (a.matrices == 2)
            if (hipError_t e = int8_tile_backward_launch(a, ws, true, !finish, stream, part_count)) return e;
        SecondParams p{};
        p.grad = reinterpret_cast<const _Float16 *>(base + ws.grad);
        p.w[0] = a.w[0];
        p.w[1] = a.w[a.matrices - 1];
        p.powers = powers;
        p.fit = fit;
        p.dx = a.dx;
        p.m = (uint32_t)a.m;
        p.m_padded = (uint32_t)(ws.grad_stride / a.matrices);
        p.n = (uint32_t)a.n;
        p.tokens = (uint32_t)a.tokens;
        p.grad_stride = (uint32_t)ws.grad_stride;
        p.matrices = a.matrices;
        p.bf16 = a.bf16;
        p.splits = ws.splits;
        p.split_sums = split_sums;
        hipError_t result = hipErrorInvalidValue;
        int index = 0;
        for_shapes([&](auto shape, float, float) {
            if (index++ == ws.second_shape) result = go<decltype(shape)>(p, stream);
        });
        if (result) return result;
    }
    if (!finish) return hipSuccess;
    FinishParams f{};
    f.parts = reinterpret_cast<const float *>(base + ws.parts);
    f.split_sums = split_sums;
    f.powers = powers;
    f.fit = fit;
    f.dscales[0] = a.dscales[0];
    f.dscales[1] = a.dscales[a.matrices - 1];
    f.dx = a.dx;
    f.m = a.m;
    f.part_count = part_count;
    f.tokens = a.tokens;
    f.n = (uint32_t)a.n;
    f.sums_blocks = (uint32_t)((a.m * a.matrices + 63) / 64);
    f.matrices = a.matrices;
    f.splits = ws.splits;
    f.bf16 = a.bf16;
    const int64_t split_blocks = runs ? (a.tokens * a.n / 4 + 63) / 64 : 0;
    hipLaunchKernelGGL(int8_finish_kernel, dim3((unsigned)(f.sums_blocks + split_blocks)), dim3(64), 0, stream, f);
    return hipGetLastError();
}

}  // namespace bcq
