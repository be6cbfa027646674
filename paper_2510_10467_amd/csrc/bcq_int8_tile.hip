// 8-bit products on tiles in LDS, plain and gated, forward and the first half of the backward pass.
//
//   forward    y = s_t c_r sum q w;   gated: act(g) u of two such products, which one wave holds lane by lane
//   backward   the sums again (they are cheaper to make than to keep), and with dy the gradients of the projections,
//              dg = dh u act'(g), du = dh act(g), which the second half multiplies by the weights, and the sums over tokens
//              dc_r = sum_t dg s_t (sum_j q w)
//
// v_mfma_i32_32x32x32_i8, weights as rows and tokens as columns, so that a lane holds four neighbouring channels of one token.  A
// workgroup's tile is ROWS weight rows by TOKS tokens; a step of 64 or 128 columns of both goes from memory into LDS by loads that write there, into a
// ring of steps.  The 16-byte parts of an LDS row sit XOR-permuted by the row's number, so that sixteen rows' operand reads use all banks.  A
// gated tile holds as many rows of gate as of up, by turns of half a wave's rows.  Results go through LDS, to be stored in whole rows.
//
// Neighbouring workgroups' numbers go to different XCDs, each with a cache of its own: they are renumbered so that one XCD works on
// the token tiles of the same weights.
//
// What bounds it: with every CU at work on large tiles the clock that the matrix pipe's power leaves (28672 x 8192 with 2048 tokens 445 to 465 us = 2160 to 2070 TOP/s;
// the library's own 8-bit product of 8192^3 2100; with codes of zero a tenth less time).  With fewer tiles what LDS takes and gives: a KiB written
// by a load takes it 16 cycles, a KiB of operands read 8.  With few tiles the latency of a step, about 0.3 us where three steps of
// 64 x 64 are under way.  Tall matrices with 33 to 128 tokens: the CUs that the last round leaves without work, and the weights' share of
// the bytes under way (17920 x 5120 gated with 48 tokens 42 us = 4.4 TB/s, 28672 x 8192 80 us = 5.9).
#include <type_traits>

#include "bcq_int8.hpp"
#include "bcq_internal.hpp"

namespace bcq {
namespace {

// Channels from first_channel on, in row_tiles times token_tiles tiles
struct TilePart {
    uint32_t first_channel, row_tiles, token_tiles;
};

struct TileParams {
    const int8_t *q, *w[2];
    const float *token_scales, *channel_scales[2];
    uint16_t *y;
    uint32_t m, n, tokens;
    TilePart part[2];               // a launch's first workgroups, and in mixed launches those behind them
    int activation;
    bool bf16, whole;               // whole: rows of y and dy are in pieces of 16 bytes
    // backward
    const uint16_t *dy;
    const float *powers;
    TokenFit fit;                   // two matrices
    bool again, add_up;             // ... only tiles with tokens whose power does not fit; and the sums of `parts`
    float *dscales[2];
    uint32_t part_count, sums_blocks;
    _Float16 *grad;                 // [tokens][grad_stride]: matrix k from k * m_padded on
    uint32_t grad_stride, m_padded;
    float *parts;                   // [a wave's tokens, from the first on][matrices][m]
};

// FR x FT tiles of 32 x 32 in a wave, WR x WT waves in a team, RING buffers of each team
template <int WR_, int WT_, int FR_, int FT_, int RING_, int TEAMS_ = 1, int STEP_ = 128, bool ACROSS_ = (RING_ >= 4)>
struct TileShape {
    static constexpr bool ACROSS = ACROSS_;
    static constexpr int WR = WR_, WT = WT_, FR = FR_, FT = FT_, RING = RING_, TEAMS = TEAMS_;
    static constexpr int STEP = STEP_;                      // columns of a step, and bytes of an LDS row
    static constexpr int PLACES = STEP / 16, LOAD_ROWS = 64 / PLACES;          // 16-byte parts of an LDS row, rows of a load
    // what a part's number is XORed with in a row: sixteen rows' reads of a part use all banks
    static constexpr __device__ __host__ uint32_t swizzle(uint32_t row) { return row * PLACES / 16 % PLACES; }
    static constexpr int ROWS = WR * FR * 32, TOKS = WT * FT * 32, TEAM_WAVES = WR * WT, WAVES = TEAMS * TEAM_WAVES;
};

template <typename S, int MATS, bool BACKWARD>
struct TileLds {
    static constexpr int STAGE = (S::ROWS + S::TOKS) * S::STEP;
    static constexpr int CHANNELS = S::ROWS / MATS;
    static constexpr int OUT_ROW = CHANNELS * 2 + 16;
    static constexpr int OUT = S::TOKS * OUT_ROW;           // one 16-bit result tile
    static constexpr int DY_EACH = (S::TOKS * CHANNELS / 8 + S::WAVES * 64 - 1) / (S::WAVES * 64);     // pieces of dy's tile for each thread, at most
    static constexpr int OUTS = BACKWARD ? MATS : 1;
    static constexpr int SCALES = OUTS * OUT;               // the channels' scales behind them
    static constexpr int TOKEN_SCALES = SCALES + MATS * CHANNELS * 4;       // the tokens' scales, and their powers of two
    static constexpr int EPILOGUE = TOKEN_SCALES + 2 * S::TOKS * 4;
    static constexpr int EXCHANGE = (S::TEAMS - 1) * S::ROWS * S::TOKS * 4;
    static constexpr int RINGS = S::TEAMS * S::RING * STAGE;
    static constexpr int BYTES = RINGS > EPILOGUE ? (RINGS > EXCHANGE ? RINGS : EXCHANGE) : (EPILOGUE > EXCHANGE ? EPILOGUE : EXCHANGE);
};

// Sums over a half wave's 32 lanes of 32 values each: lane l ends with the sum of value l.  A step halves the values a lane holds: it keeps those
// with its own bit of the number and gives the others to a lane whose bit is the other one.  Lanes 16 apart change places in one
// instruction; the others read across a row of 16 in the addition itself: 8 apart, 7 - l, 2 apart, 1 apart, which together reach all lanes.
// (Through LDS, 31 exchanges, the sums took 70 of the 380 us of a first half of 2048 tokens and 2 x 14336 channels.)
template <int CONTROL>
__device__ __forceinline__ float across(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
}
template <int D, int CONTROL>
__device__ __forceinline__ void halve(float (&v)[32], int lane)
{
    const bool upper = lane & D;
#pragma unroll
    for (int i = 0; i < D; ++i) {
        const float keep = upper ? v[i + D] : v[i], give = upper ? v[i] : v[i + D];
        v[i] = keep + across<CONTROL>(give);
    }
}
__device__ __forceinline__ float sums_of_32(float (&v)[32], int lane)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        // rows 1 and 3 of the first change places with rows 0 and 2 of the second
        const auto swapped = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v[i]), __builtin_bit_cast(uint32_t, v[i + 16]), false, false);
        const uint32_t own = swapped[0], other = swapped[1];
        v[i] = __builtin_bit_cast(float, own) + __builtin_bit_cast(float, other);
    }
    halve<8, 0x128>(v, lane);           // row_ror:8
    halve<4, 0x141>(v, lane);           // row_half_mirror
    halve<2, 0x4e>(v, lane);            // quad_perm 2 3 0 1
    halve<1, 0xb1>(v, lane);            // quad_perm 1 0 3 2
    return v[0];
}

// Workgroup `block` of a part.
template <typename S, int MATS, bool BACKWARD, int ACT>
__device__ __forceinline__ void tile(const TileParams &a, const TilePart &part, uint32_t block)
{
    using L = TileLds<S, MATS, BACKWARD>;
    constexpr int FRC = S::FR / MATS;                       // tiles of 32 channels in a wave
    constexpr int CHANNELS = L::CHANNELS;
    static_assert(!BACKWARD || CHANNELS % 32 == 0, "the last tile writes the gradients' rows, of a multiple of 64, to their end");
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int team = wave / S::TEAM_WAVES, tw = wave % S::TEAM_WAVES;
    const int wr = tw / S::WT, wt = tw % S::WT;
    const int r32 = lane & 31, half = lane >> 5;

    // the tile: first by XCD, then in groups of up to eight token tiles, the tokens of a group running fastest
    const uint32_t total = part.row_tiles * part.token_tiles, xcd = block & 7;
    const uint32_t id = xcd * (total >> 3) + min(xcd, total & 7) + (block >> 3);
    const uint32_t group = id / (8 * part.row_tiles);
    const uint32_t in_group = min(8u, part.token_tiles - group * 8);
    const uint32_t rest = id - group * 8 * part.row_tiles;
    const uint32_t row_tile = rest / in_group, token_tile = group * 8 + rest % in_group;
    const uint32_t ch0 = part.first_channel + row_tile * CHANNELS, t0 = token_tile * S::TOKS;

    const uint32_t chs = min((uint32_t)CHANNELS, a.m - ch0), toks = min((uint32_t)S::TOKS, a.tokens - t0);
    if constexpr (BACKWARD && MATS == 2) {
        if (a.again) {                                      // (every wave looks at all of them and comes to the same answer)
            bool all_fit = true;
#pragma unroll
            for (int k = 0; k < S::TOKS; k += 64) all_fit &= power_fits(a.fit, t0 + min((uint32_t)(k + lane), toks - 1));
            if (__all(all_fit)) return;
        }
    }
    const int8_t *const q_base = a.q + (int64_t)t0 * a.n;
    const int8_t *const w_base = a.w[0] + (int64_t)ch0 * a.n, *const u_base = a.w[MATS - 1] + (int64_t)ch0 * a.n;

    // A load brings 1 KiB: LOAD_ROWS rows; lane l delivers the part that belongs at place l % PLACES of row l / PLACES of them.
    // Rows and tokens past the end repeat the last one (their results are not stored).
    constexpr int W_LOADS = S::ROWS / S::LOAD_ROWS / S::TEAM_WAVES, Q_UNITS = S::TOKS / S::LOAD_ROWS,
                  Q_LOADS = (Q_UNITS + S::TEAM_WAVES - 1) / S::TEAM_WAVES;
    static_assert(W_LOADS * S::LOAD_ROWS * S::TEAM_WAVES == S::ROWS && Q_UNITS * S::LOAD_ROWS == S::TOKS, "whole loads");
    // (six waves bring eight loads of tokens: twelve, the last ones the same)
    auto q_unit = [&](int k) { return Q_UNITS % S::TEAM_WAVES == 0 ? tw * Q_LOADS + k : min(tw * Q_LOADS + k, Q_UNITS - 1); };
    uint32_t w_src[W_LOADS], q_src[Q_LOADS], w_part[W_LOADS], q_part[Q_LOADS];
#pragma unroll
    for (int k = 0; k < W_LOADS; ++k) {
        const uint32_t row = S::LOAD_ROWS * (tw * W_LOADS + k) + lane / S::PLACES;
        w_part[k] = (lane % S::PLACES ^ S::swizzle(row)) * 16;
        const uint32_t in_wave = row % (S::FR * 32);
        const uint32_t ch = MATS == 1 ? row : row / (S::FR * 32) * (FRC * 32) + in_wave % (FRC * 32);
        w_src[k] = min(ch, chs - 1) * a.n;
    }
#pragma unroll
    for (int k = 0; k < Q_LOADS; ++k) {
        const uint32_t tok = S::LOAD_ROWS * q_unit(k) + lane / S::PLACES;
        q_part[k] = (lane % S::PLACES ^ S::swizzle(tok)) * 16;
        q_src[k] = min(tok, toks - 1) * a.n;
    }
    // The backward pass's tile of dy, asked for before everything else (at the end nothing would hide its way).
    constexpr int PIECES = CHANNELS / 8, THREADS = S::WAVES * 64;           // 16-byte pieces of a tile's row
    [[maybe_unused]] u32x4 dy_early[BACKWARD ? L::DY_EACH : 1];
    if constexpr (BACKWARD) {
        if (a.whole) {
#pragma unroll
            for (int k = 0; k < L::DY_EACH; ++k) {
                const uint32_t tok = (threadIdx.x + k * THREADS) / PIECES, piece = (threadIdx.x + k * THREADS) % PIECES;
                dy_early[k] = tok < toks && piece * 8 < chs ? *reinterpret_cast<const u32x4 *>(a.dy + (int64_t)(t0 + tok) * a.m + ch0 + piece * 8) : u32x4{0, 0, 0, 0};
            }
        }
    }

    unsigned char *const mine = lds + team * S::RING * L::STAGE;        // the team's ring
    // Columns k0 .. k0 + STEP - 1 into a buffer.  In the last step parts past the row's end bring the row's first part instead: what is
    // multiplied with them is set to zero.
    auto stage = [&](int buffer, uint32_t k0) {
        unsigned char *to = mine + buffer * L::STAGE;
        const bool last = k0 + S::STEP > a.n;
        const auto q_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(q_base), 0, (int)(toks * a.n), 0x00020000);
        auto column = [&](uint32_t part) { return last && k0 + part >= a.n ? 0u : k0 + part; };
#pragma unroll
        for (int k = 0; k < W_LOADS; ++k) {
            const int unit = tw * W_LOADS + k;
            const bool up = MATS == 2 && (unit * S::LOAD_ROWS) % (S::FR * 32) >= FRC * 32;
            const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(up ? u_base : w_base), 0, (int)(chs * a.n), 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (__attribute__((address_space(3))) void *)(to + unit * 1024), 16,
                                                     (int)(w_src[k] + column(w_part[k])), 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < Q_LOADS; ++k) {
            const int unit = q_unit(k);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(q_rsrc, (__attribute__((address_space(3))) void *)(to + S::ROWS * S::STEP + unit * 1024), 16,
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

    const uint32_t swz = S::swizzle(r32);
    struct Operands {
        v4i w[S::FR], x[S::FT];
    };
    auto operands = [&](int buffer, int kk) {
        const unsigned char *from = mine + buffer * L::STAGE + r32 * S::STEP + (((2 * kk + half) ^ swz) << 4);
        Operands o;
#pragma unroll
        for (int r = 0; r < S::FR; ++r) o.w[r] = *reinterpret_cast<const v4i *>(from + (wr * S::FR + r) * 32 * S::STEP);
#pragma unroll
        for (int t = 0; t < S::FT; ++t) o.x[t] = *reinterpret_cast<const v4i *>(from + S::ROWS * S::STEP + (wt * S::FT + t) * 32 * S::STEP);
        return o;
    };
    auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int r = 0; r < S::FR; ++r)
#pragma unroll
            for (int t = 0; t < S::FT; ++t) acc[r][t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(o.w[r], o.x[t], acc[r][t], 0, 0, 0);
    };
    // One step.  ACROSS: its first operands are there, and each time the next operands are read between the matrix instructions, at the end those of
    // the step in buffer `after`.
    [[maybe_unused]] Operands now;
    auto whole_step = [&](int buffer, int after) {
#pragma unroll
        for (int kk = 0; kk < S::STEP / 32; ++kk) {
            if constexpr (S::ACROSS) {
                const Operands later = kk + 1 < S::STEP / 32 ? operands(buffer, kk + 1) : operands(after, 0);
                multiply(now);
                now = later;
                constexpr int READS = S::FR + S::FT, PRODUCTS = S::FR * S::FT;
#pragma unroll
                for (int i = 0; i < (READS > PRODUCTS ? READS : PRODUCTS); ++i) {
                    if (i < READS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    if (i < PRODUCTS) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                }
            } else {
                multiply(operands(buffer, kk));
            }
        }
    };

    const int steps = (int)(a.n / S::STEP), tail = (int)(a.n % S::STEP);
    const int stages = steps + (tail ? 1 : 0);
    // The teams take the steps by turns: round i is step i TEAMS + team, in buffer i % RING.  At the top of a round its tiles and the next
    // one's have landed, what later rounds asked for is still under way, and nobody reads the buffer of the round before any more, into which the
    // round RING - 1 ahead then goes.  (A team may have no step in the last round, and nothing else is missing.)
    constexpr int AHEAD = S::RING - 1, LOADS = W_LOADS + Q_LOADS;
    static_assert(S::RING >= 3 || !S::ACROSS, "a step reads the next one's first operands");
    const int rounds = (stages + S::TEAMS - 1) / S::TEAMS;
    auto step = [&](int i) { return i * S::TEAMS + team; };
    // Row tiles begin 128 columns apart and come back to the first columns at the end (sums of integers are the same in any order): all at the same
    // column would ask for addresses whole rows apart, which are few of memory's channels where a row is a power of two or
    // nearly (28672 x 8192 with 48 tokens 55 -> 43 us, gated with 40 tokens 99 -> 80).
    constexpr int LINE = 128 / S::STEP;                     // steps of 128 columns
    const int turned = steps ? (int)(row_tile * LINE % steps / LINE * LINE) : 0;
    auto columns = [&](int s) {
        if (s >= steps) return (uint32_t)s * S::STEP;       // (the part of a step at the row's end stays last)
        return (uint32_t)(s + turned < steps ? s + turned : s + turned - steps) * S::STEP;
    };
    for (int i = 0; i < min(AHEAD, rounds); ++i)
        if (step(i) < stages) stage(i, columns(step(i)));
    if (rounds > AHEAD) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((AHEAD - 1) * LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    if (S::ACROSS) now = operands(0, 0);
    int buffer = 0, into = AHEAD, i = 0;
    auto next = [](int b) { return b + 1 == S::RING ? 0 : b + 1; };
    for (; i + AHEAD < rounds; ++i) {                       // (whole steps: the last one is still to come)
        constexpr int UNDER_WAY = (AHEAD - (S::ACROSS ? 2 : 1)) * LOADS;
        if constexpr (S::TEAM_WAVES == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(UNDER_WAY) : "memory");     // (a ring of its own)
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(UNDER_WAY) : "memory");
        if (S::TEAMS == 1 || step(i + AHEAD) < stages) stage(into, columns(step(i + AHEAD)));
        whole_step(buffer, next(buffer));
        buffer = next(buffer);
        into = next(into);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    for (; step(i) < steps; ++i) {                          // (behind the last step, what is read for the next one is nothing)
        whole_step(buffer, next(buffer));
        buffer = next(buffer);
    }
    if (step(i) < stages)
        for (int kk = 0; kk * 32 < tail; ++kk) {
            Operands o = operands(buffer, kk);
#pragma unroll
            for (int t = 0; t < S::FT; ++t)
                if (kk * 32 + half * 16 >= tail) o.x[t] = v4i{0, 0, 0, 0};
            multiply(o);
        }
    __syncthreads();
    // The teams add up: of each tile's four groups of four channels a team ends with GROUPS, its own sums and what the others left it.
    constexpr int GROUPS = 4 / S::TEAMS;
    v4i sums_of[S::FR][S::FT][GROUPS];
#pragma unroll
    for (int k = 0; k < S::TEAMS; ++k) {
        if (team != k) continue;
        v4i *const exchange = reinterpret_cast<v4i *>(lds) + tw * (S::FR * S::FT * 4 * 64) + lane;
        constexpr int BETWEEN = S::TEAM_WAVES * S::FR * S::FT * 4 * 64;
#pragma unroll
        for (int r = 0; r < S::FR; ++r)
#pragma unroll
            for (int t = 0; t < S::FT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const v4i v = {acc[r][t][4 * e], acc[r][t][4 * e + 1], acc[r][t][4 * e + 2], acc[r][t][4 * e + 3]};
                    const int whose = e / GROUPS;                   // its place among those that leave something for that team: all but itself
                    if (whose == k) sums_of[r][t][e % GROUPS] = v;
                    else exchange[(k - (k > whose ? 1 : 0)) * BETWEEN + ((r * S::FT + t) * 4 + e) * 64] = v;
                }
    }
    if constexpr (S::TEAMS > 1) {
        __syncthreads();
        const v4i *const exchange = reinterpret_cast<const v4i *>(lds) + tw * (S::FR * S::FT * 4 * 64) + team * GROUPS * 64 + lane;
        constexpr int BETWEEN = S::TEAM_WAVES * S::FR * S::FT * 4 * 64;
#pragma unroll
        for (int k = 0; k < S::TEAMS - 1; ++k)
#pragma unroll
            for (int r = 0; r < S::FR; ++r)
#pragma unroll
                for (int t = 0; t < S::FT; ++t)
#pragma unroll
                    for (int e = 0; e < GROUPS; ++e) sums_of[r][t][e] += exchange[k * BETWEEN + ((r * S::FT + t) * 4 + e) * 64];
        __syncthreads();
    }

    // the channels' and tokens' scales, and in the backward pass the tile of dy
    float *scales = reinterpret_cast<float *>(lds + L::SCALES);
    for (int i = threadIdx.x; i < MATS * CHANNELS; i += S::WAVES * 64) {
        const uint32_t ch = i % CHANNELS;
        scales[i] = ch < chs ? a.channel_scales[i / CHANNELS][ch0 + ch] : 0.f;
    }
    float *token_scales = reinterpret_cast<float *>(lds + L::TOKEN_SCALES);
    [[maybe_unused]] float *powers = token_scales + S::TOKS;
    for (uint32_t i = threadIdx.x; i < S::TOKS; i += S::WAVES * 64) {
        token_scales[i] = i < toks ? a.token_scales[t0 + i] : 0.f;
        if constexpr (BACKWARD) powers[i] = i >= toks ? 1.f : MATS == 2 && a.again ? token_power(a.powers, a.fit, t0 + i) : a.powers[t0 + i];
    }
    if constexpr (BACKWARD) {
        if (a.whole) {
#pragma unroll
            for (int k = 0; k < L::DY_EACH; ++k) {
                const uint32_t i = threadIdx.x + k * THREADS;
                if (i < S::TOKS * PIECES) *reinterpret_cast<u32x4 *>(lds + i / PIECES * L::OUT_ROW + i % PIECES * 16) = dy_early[k];
            }
        } else {
            for (int i = threadIdx.x; i < S::TOKS * CHANNELS; i += 8 * THREADS) {
                uint16_t v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t tok = (i + k * THREADS) / CHANNELS, ch = (i + k * THREADS) % CHANNELS;
                    v[k] = tok < toks && ch < chs ? a.dy[(int64_t)(t0 + tok) * a.m + ch0 + ch] : (uint16_t)0;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (i + k * THREADS < S::TOKS * CHANNELS)
                        *reinterpret_cast<uint16_t *>(lds + (i + k * THREADS) / CHANNELS * L::OUT_ROW + (i + k * THREADS) % CHANNELS * 2) = v[k];
            }
        }
    }
    __syncthreads();

    [[maybe_unused]] float largest[S::FT];
#pragma unroll
    for (int t = 0; t < S::FT; ++t) largest[t] = 0.f;
    // 32 sums over this wave's tokens at a time: a tile of channels of each matrix, or two tiles of the one
    constexpr int TOGETHER = BACKWARD && MATS == 1 ? 2 : 1;
    static_assert(FRC % TOGETHER == 0, "whole exchanges");
    auto results = [&] {
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
                    [[maybe_unused]] float power = 0.f;
                    if constexpr (BACKWARD) power = powers[tok];
#pragma unroll
                    for (int e = 0; e < GROUPS; ++e) {
                        const int ch = (wr * FRC + r) * 32 + 8 * (team * GROUPS + e) + 4 * half;    // element i: channel ch + i
                        unsigned char *at = lds + tok * L::OUT_ROW + ch * 2;
                        const v4f c0 = *reinterpret_cast<const v4f *>(scales + ch);
                        const v4f c1 = *reinterpret_cast<const v4f *>(scales + (MATS - 1) * CHANNELS + ch);
                        [[maybe_unused]] u32x2 dy = {0, 0};
                        if constexpr (BACKWARD) dy = *reinterpret_cast<const u32x2 *>(at);
                        uint32_t out[4], out2[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float p = (float)sums_of[r][t][e][i] * ts;
                            [[maybe_unused]] float p2 = 0.f, slope = 0.f;
                            if constexpr (MATS == 2) p2 = (float)sums_of[FRC + r][t][e][i] * ts;
                            if constexpr (!BACKWARD) {
                                float v = p * c0[i];
                                if constexpr (MATS == 2) v = activate<false>(v, ACT, slope) * (p2 * c1[i]);
                                out[i] = to_16(v, a.bf16);
                            } else {
                                // (channels and tokens past the end have a gradient and a scale of 0)
                                const float d = from_16((i & 1) ? dy[i >> 1] >> 16 : dy[i >> 1] & 0xffffu, a.bf16);
                                // What the second half multiplies is held in binary16, times the token's power of two: off by up to
                                // 2^-11 of itself, as much as by a binary16 result's last rounding, or by 2^-25 of the token's largest.
                                if constexpr (MATS == 1) {
                                    out[i] = to_16(d * c0[i] * power, false);
                                    sums[(r - r0) * 16 + 4 * e + i] += d * p;
                                } else {
                                    const float act = activate<true>(p * c0[i], ACT, slope);
                                    const float dg = d * (p2 * c1[i]) * slope, du = d * act;
                                    const float held = dg * c0[i] * power, held2 = du * c1[i] * power;
                                    out[i] = to_16(held, false);
                                    out2[i] = to_16(held2, false);
                                    largest[t] = fmaxf(largest[t], fmaxf(fabsf(held), fabsf(held2)));      // (a NaN leaves it as it is)
                                    sums[4 * e + i] += dg * p;
                                    sums[16 + 4 * e + i] += du * p2;
                                }
                            }
                        }
                        *reinterpret_cast<u32x2 *>(at) = u32x2{out[0] | out[1] << 16, out[2] | out[3] << 16};
                        if constexpr (BACKWARD && MATS == 2)
                            *reinterpret_cast<u32x2 *>(at + L::OUT) = u32x2{out2[0] | out2[1] << 16, out2[2] | out2[3] << 16};
                        // (four elements at a time: registers.  A maximum put off would hold all that it is taken of.)
                        if constexpr (BACKWARD && MATS == 2) asm volatile("" : "+v"(largest[t]));
                        if constexpr (BACKWARD) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            if constexpr (BACKWARD) {
                // lane l of a half gets value l: element l % 16 of the first or second sixteen, of which the team has 4 GROUPS
                const float sum = sums_of_32(sums, lane);
                const int second = r32 >> 4, e = (r32 >> 2) & 3, i = r32 & 3;
                const uint32_t ch = (wr * FRC + r0 + (MATS == 1 ? second : 0)) * 32 + 8 * (team * GROUPS + e) + 4 * half + i;
                float *parts = a.parts + (int64_t)(token_tile * S::WT + wt) * MATS * a.m;
                if (e < GROUPS && ch < chs && !(MATS == 2 && a.again)) parts[(int64_t)(MATS == 1 ? 0 : second) * a.m + ch0 + ch] = sum;
            }
        }
    };
    results();
    if constexpr (BACKWARD && MATS == 2) {
        if (!a.again) {
#pragma unroll
            for (int t = 0; t < S::FT; ++t) {
                const float v = fmaxf(largest[t], __shfl_xor(largest[t], 32, 64));
                const uint32_t tok = (wt * S::FT + t) * 32 + r32;
                if (half == 1 || tok >= toks) continue;
                // (mostly a store, of the same value by all; maxima of all tiles at once took 14336 channels with 64 tokens 12 us.  They are the
                // same in any order.)
                if (v >= kFitsFrom && v <= kFitsTo) a.fit.some[t0 + tok] = 1;
                else if (v > 0.f) atomicMax(a.fit.other + t0 + tok, __builtin_bit_cast(uint32_t, v));
            }
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
            if constexpr (CHANNELS % 64 != 0)               // (the last tile may end 32 channels short of it)
                if (piece < 4 && tok < toks && ch0 + CHANNELS >= a.m && ch0 + CHANNELS < a.m_padded)
                    *reinterpret_cast<u32x4 *>(a.grad + (int64_t)(t0 + tok) * a.grad_stride + k * a.m_padded + ch0 + CHANNELS + piece * 8) = u32x4{0, 0, 0, 0};
        }
    }
}

// A launch's first workgroups may add up the partial sums, a channel a thread.  Returns which of the tiles' workgroups this one is, or
// none of them (negative).
template <typename S, int MATS, bool BACKWARD>
__device__ __forceinline__ int tile_of_launch(const TileParams &a)
{
    if constexpr (BACKWARD && MATS == 2) {
        if (blockIdx.x < a.sums_blocks) {
            const uint32_t i = blockIdx.x * (S::WAVES * 64) + threadIdx.x, channels = 2 * a.m;
            if (i >= channels) return -1;
            const float sum = sum_of_parts(a.parts, a.part_count, channels, i);
            if (i < a.m) a.dscales[0][i] = sum;
            else a.dscales[1][i - a.m] = sum;
            return -1;
        }
        return (int)(blockIdx.x - a.sums_blocks);
    }
    return (int)blockIdx.x;
}

template <typename S, int MATS, bool BACKWARD, int ACT>
__global__ __launch_bounds__(S::WAVES * 64, 2) void int8_tile_kernel(const TileParams a)
{
    const int block = tile_of_launch<S, MATS, BACKWARD>(a);
    if (block < 0) return;
    tile<S, MATS, BACKWARD, ACT>(a, a.part[0], (uint32_t)block);
}

// Two shapes in one launch: the second's workgroups are behind the first's.
template <typename S, typename S2, int MATS, bool BACKWARD, int ACT>
__global__ __launch_bounds__(S::WAVES * 64, 2) void int8_tiles_kernel(const TileParams a)
{
    static_assert(S::WAVES == S2::WAVES, "one size of workgroup");
    const int first = (int)(a.part[0].row_tiles * a.part[0].token_tiles), block = tile_of_launch<S, MATS, BACKWARD>(a);
    if (block < 0) return;
    if (block < first) tile<S, MATS, BACKWARD, ACT>(a, a.part[0], (uint32_t)block);
    else tile<S2, MATS, BACKWARD, ACT>(a, a.part[1], (uint32_t)(block - first));
}

hipError_t launch(void (*kernel)(const TileParams), int lds_bytes, int waves, TileParams p, hipStream_t stream)
{
    if (hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), lds_bytes)) return e;
    const uint32_t tiles = p.part[0].row_tiles * p.part[0].token_tiles + p.part[1].row_tiles * p.part[1].token_tiles;
    p.sums_blocks = p.add_up ? (2 * p.m + waves * 64 - 1) / (waves * 64) : 0;
    hipLaunchKernelGGL(kernel, dim3(p.sums_blocks + tiles), dim3(waves * 64), lds_bytes, stream, p);
    return hipGetLastError();
}

template <typename S, int MATS>
TilePart part_of(uint32_t first_channel, uint32_t channels, uint32_t tokens)
{
    constexpr uint32_t CHANNELS = S::ROWS / MATS;
    return {first_channel, (channels + CHANNELS - 1) / CHANNELS, (tokens + S::TOKS - 1) / S::TOKS};
}

template <typename S, int MATS, bool BACKWARD, int ACT>
hipError_t go(TileParams p, hipStream_t stream, int64_t &part_count)
{
    part_count = p.part_count = (p.tokens + S::FT * 32 - 1) / (S::FT * 32);
    p.part[0] = part_of<S, MATS>(0, p.m, p.tokens);
    return launch(int8_tile_kernel<S, MATS, BACKWARD, ACT>, TileLds<S, MATS, BACKWARD>::BYTES, S::WAVES, p, stream);
}

// Full rounds of 256 workgroups of the first shape, for what is left the second.
template <typename S, typename S2, int MATS, bool BACKWARD, int ACT>
hipError_t go_mixed(TileParams p, uint32_t first_row_tiles, hipStream_t stream, int64_t &part_count)
{
    static_assert(S::FT == S2::FT, "partial sums over as many tokens");
    part_count = p.part_count = (p.tokens + S::FT * 32 - 1) / (S::FT * 32);
    constexpr uint32_t CHANNELS = S::ROWS / MATS;
    constexpr int BYTES = TileLds<S, MATS, BACKWARD>::BYTES, BYTES2 = TileLds<S2, MATS, BACKWARD>::BYTES;
    p.part[0] = part_of<S, MATS>(0, first_row_tiles * CHANNELS, p.tokens);
    p.part[1] = part_of<S2, MATS>(first_row_tiles * CHANNELS, p.m - first_row_tiles * CHANNELS, p.tokens);
    return launch(int8_tiles_kernel<S, S2, MATS, BACKWARD, ACT>, BYTES > BYTES2 ? BYTES : BYTES2, S::WAVES, p, stream);
}

// What a workgroup takes per 128 columns, alone on its CU and as one of several in turn (microseconds, measured): the shape that is expected to be done
// first is taken.  Large tiles read each operand from the caches the fewest times; small ones, with teams or a deep ring, give every CU work and
// keep enough bytes under way where there are few.
//                                       256 x 256  256 x 128  128 x 128  256 x 64  128 x 64  64 x 64  64 x 32
//   4096 x 4096, 256 tokens                    52         31         20        22        15       11       15  us
//   4096 x 4096, 100 tokens                    51         31         20        22        15     10.4      8.1
//   14336 x 4096 gated, 512 tokens             65         75         90       106       131      162
//   17920 x 5120 gated, 48 tokens              78         53         61        46        64       51       61
using Largest = TileShape<2, 4, 4, 2, 2>;
using Large = TileShape<4, 2, 2, 2, 3>;
constexpr float kLargestUs = 1.70f, kLargeUs = 1.08f;
template <typename F>
void for_shapes(F f)
{
    f(Largest{}, kLargestUs, kLargestUs);                   // 256 x 256
    f(Large{}, kLargeUs, 1.10f);                            // 256 x 128
    f(TileShape<2, 2, 2, 2, 4>{}, 0.60f, 0.62f);            // 128 x 128
    f(TileShape<4, 1, 2, 2, 4>{}, 0.69f, 0.70f);            // 256 x 64
    // 192 x 128 and 192 x 64: more workgroups, with more bytes under way, for heights between (17920 x 5120 gated with 100 tokens 54.5 -> 49.5 us, with 48
    // 46.2 -> 42.0; 8192 x 8192 with 600 tokens 59.9 -> 56.3)
    f(TileShape<3, 2, 2, 2, 4>{}, 0.97f, 1.05f);
    f(TileShape<3, 2, 2, 1, 5>{}, 0.62f, 0.66f);
    f(TileShape<2, 1, 2, 2, 6, 2, 64>{}, 0.34f, 0.50f);     // 128 x 64, two teams
    // ... where rows are no whole lines: a piece of 64 bytes is then a line's half with one round and the other with the next (25065 x 6800 with 34
    // tokens 50.7 -> 42.7 us, 8448 x 11680 gated with 17 65 -> 57).  On whole lines it depends on where the weights are: 4096 x 14336 with 512 tokens 42
    // against 47 us where they are in the last cache, 57 against 51 where they come from memory.
    f(TileShape<2, 1, 2, 2, 3, 2>{}, 0.34f, 0.50f);
    f(TileShape<1, 2, 2, 1, 4, 2>{}, 0.28f, 0.30f);         // 64 x 64, two teams
    f(TileShape<1, 1, 2, 1, 3, 4>{}, 0.20f, 0.20f);         // 64 x 32, four teams
}

// The shape, by its place among for_shapes, or the largest tiles in so many tiles of rows and Large behind them.
struct TileChoice {
    int shape;
    uint32_t first_row_tiles;
};
template <int MATS>
TileChoice choose(uint32_t m, uint32_t n, uint32_t tokens, bool aligned)
{
    const bool lines = n % 128 == 0 && aligned;
    float best = 0.f;
    int index = 0, chosen = -1;
    for_shapes([&](auto shape, float alone, float in_turn) {
        using S = decltype(shape);
        if (S::STEP < 128 && !lines) alone = in_turn = 1e9f;
        // Two matrices with rows 8 KiB apart: 192 x 64 are behind 256 x 64 (24576 rows of each with 64 tokens 78 against 70 us; 8064 columns 71 against
        // 85, 8320 columns 72 against 86, one matrix of 49152 rows 72 against 73).
        if (MATS == 2 && S::ROWS == 192 && S::TOKS == 64 && n == 8192) alone = 0.70f;
        const int64_t tiles = (int64_t)((m * MATS + S::ROWS - 1) / S::ROWS) * ((tokens + S::TOKS - 1) / S::TOKS);
        const int64_t each = (tiles + 255) / 256;                   // tiles of the busiest CU
        const float us = each == 1 ? alone : (float)each * in_turn;
        if (chosen < 0 || us < best) {
            best = us;
            chosen = index;
        }
        ++index;
    });
    // The largest tiles as far as they fill rounds, and where one round of those of half the tokens takes what is left, that (2048 tokens, 4096
    // columns, gated, 14336 rows, 3.5 rounds: 247 -> 231 us; 12288 rows, three rounds: 189).
    const TilePart all = part_of<Largest, MATS>(0, m, tokens);
    const int64_t rounds = (int64_t)all.row_tiles * all.token_tiles / 256;
    const uint32_t first = (uint32_t)(rounds * 256 / all.token_tiles);
    if (rounds > 0 && first < all.row_tiles) {
        const TilePart left = part_of<Large, MATS>(0, (all.row_tiles - first) * (Largest::ROWS / MATS), tokens);
        if ((int64_t)left.row_tiles * left.token_tiles <= 256 && (float)rounds * kLargestUs + kLargeUs < best) return {0, first};
    }
    return {chosen, 0};
}

template <int MATS, bool BACKWARD, int ACT>
hipError_t pick(const TileParams &p, hipStream_t stream, int64_t &part_count)
{
    const bool aligned = ((reinterpret_cast<uintptr_t>(p.w[0]) | reinterpret_cast<uintptr_t>(p.w[MATS - 1])) & 127) == 0;
    const TileChoice choice = choose<MATS>(p.m, p.n, p.tokens, aligned);
    if (choice.first_row_tiles) return go_mixed<Largest, Large, MATS, BACKWARD, ACT>(p, choice.first_row_tiles, stream, part_count);
    hipError_t result = hipErrorInvalidValue;
    int index = 0;
    for_shapes([&](auto shape, float, float) {
        if (index++ == choice.shape) result = go<decltype(shape), MATS, BACKWARD, ACT>(p, stream, part_count);
    });
    return result;
}

template <bool BACKWARD>
hipError_t pick(const TileParams &p, int matrices, hipStream_t stream, int64_t &part_count)
{
    if (matrices == 1) return pick<1, BACKWARD, BCQ_ACT_SILU>(p, stream, part_count);
    return p.activation == BCQ_ACT_GELU ? pick<2, BACKWARD, BCQ_ACT_GELU>(p, stream, part_count) : pick<2, BACKWARD, BCQ_ACT_SILU>(p, stream, part_count);
}

template <int MATS, bool BACKWARD>
Int8Layout layout_of(const TileChoice &choice, uint32_t n)
{
    Int8Layout layout{};
    int index = 0;
    for_shapes([&](auto shape, float, float) {
        using S = decltype(shape);
        if (index++ != choice.shape) return;
        const int steps = (int)((n + S::STEP - 1) / S::STEP);
        layout = {S::ROWS, S::TOKS, S::STEP, S::TEAMS, S::RING, (steps + S::TEAMS - 1) / S::TEAMS, TileLds<S, MATS, BACKWARD>::BYTES};
    });
    return layout;
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
    int64_t part_count;
    return pick<false>(params(a), a.matrices, stream, part_count);
}

Int8Layout int8_tile_layout(const Int8Args &a, bool backward, bool &mixed)
{
    const uint32_t m = (uint32_t)a.m, n = (uint32_t)a.n, tokens = (uint32_t)a.tokens;
    const TileChoice choice = a.matrices == 2 ? choose<2>(m, n, tokens, true) : choose<1>(m, n, tokens, true);
    mixed = choice.first_row_tiles > 0;
    if (a.matrices == 2) return backward ? layout_of<2, true>(choice, n) : layout_of<2, false>(choice, n);
    return backward ? layout_of<1, true>(choice, n) : layout_of<1, false>(choice, n);
}

hipError_t int8_tile_backward_launch(const Int8Args &a, const Int8Workspace &ws, bool again, bool add_up, hipStream_t stream, int64_t &part_count)
{
    TileParams p = params(a);
    unsigned char *base = static_cast<unsigned char *>(a.workspace);
    p.grad = reinterpret_cast<_Float16 *>(base + ws.grad);
    p.powers = reinterpret_cast<const float *>(base + ws.powers);
    p.fit = {reinterpret_cast<uint32_t *>(base + ws.some), reinterpret_cast<uint32_t *>(base + ws.other)};
    p.again = again;
    p.add_up = add_up;
    for (int k = 0; k < 2; ++k) p.dscales[k] = a.dscales[k];
    p.parts = reinterpret_cast<float *>(base + ws.parts);
    p.grad_stride = (uint32_t)ws.grad_stride;
    p.m_padded = (uint32_t)(ws.grad_stride / a.matrices);
    return pick<true>(p, a.matrices, stream, part_count);
}

}  // namespace bcq
