// 8-bit products for few tokens.  The weights are read once, straight into the operand registers of
// v_mfma_i32_16x16x64_i8 (a lane holds 16 bytes of row lane % 16), and the matrix instruction does the sum over columns: there is no
// reduction across lanes, and the 16 columns of its result are 16 tokens, of which one costs no more than sixteen.
//
// A workgroup owns 16 BLOCKS rows (of gate and of up, where there are two) and all tokens; its waves take equal runs of 64-column steps, so
// that a row's bytes are under way at once, and meet in LDS: sums of integers, in any order the same.  The codes of the
// tokens come from the cache into registers beside the weights.
//
// Bound by the weights' bytes.
#include "bcq_int8.hpp"

namespace bcq {
namespace {

struct RowsParams {
    const int8_t *q, *w[2];
    const float *token_scales, *channel_scales[2];
    uint16_t *y;
    int64_t m;
    int n, tokens, activation;
    bool bf16;
};

// TT: tiles of 16 tokens; MATS: matrices; BLOCKS: blocks of 16 rows of each; WAVES per workgroup
template <int TT, int MATS, int BLOCKS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void int8_rows_kernel(const RowsParams a)
{
    constexpr int FRAGS = MATS * BLOCKS * TT;
    constexpr int UNROLL = TT + MATS * BLOCKS <= 2 ? 8 : TT + MATS * BLOCKS <= 4 ? 4 : 2;     // steps whose operands are under way together
    __shared__ v4i parts[WAVES][FRAGS][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, part = lane >> 4;
    const int64_t row0 = (int64_t)blockIdx.x * (16 * BLOCKS);

    // rows and tokens past the end repeat the last one (their results are not stored)
    const int8_t *w_at[MATS * BLOCKS], *q_at[TT];
#pragma unroll
    for (int f = 0; f < MATS * BLOCKS; ++f) {
        const int64_t row = min(row0 + (f % BLOCKS) * 16 + r16, a.m - 1);
        w_at[f] = a.w[f / BLOCKS] + row * a.n + part * 16;
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) q_at[t] = a.q + (int64_t)min(t * 16 + r16, a.tokens - 1) * a.n + part * 16;

    v4i acc[FRAGS];
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) acc[f] = v4i{0, 0, 0, 0};

    const int steps = a.n >> 6;                         // whole steps of 64 columns
    const int each = (steps + WAVES - 1) / WAVES;
    const int first = min(wave * each, steps), end = min(first + each, steps);
    auto products = [&](const v4i *w, const v4i *x) {
#pragma unroll
        for (int f = 0; f < MATS * BLOCKS; ++f)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[f * TT + t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[f], x[t], acc[f * TT + t], 0, 0, 0);
    };
    int s = first;
    for (; s + UNROLL <= end; s += UNROLL) {
        v4i w[UNROLL][MATS * BLOCKS], x[UNROLL][TT];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
            for (int f = 0; f < MATS * BLOCKS; ++f) w[u][f] = *reinterpret_cast<const v4i *>(w_at[f] + (s + u) * 64);
#pragma unroll
            for (int t = 0; t < TT; ++t) x[u][t] = *reinterpret_cast<const v4i *>(q_at[t] + (s + u) * 64);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) products(w[u], x[u]);
    }
    for (; s < end; ++s) {
        v4i w[MATS * BLOCKS], x[TT];
#pragma unroll
        for (int f = 0; f < MATS * BLOCKS; ++f) w[f] = *reinterpret_cast<const v4i *>(w_at[f] + s * 64);
#pragma unroll
        for (int t = 0; t < TT; ++t) x[t] = *reinterpret_cast<const v4i *>(q_at[t] + s * 64);
        products(w, x);
    }
    const int rest = a.n & 63;                          // 0, 16, 32 or 48 columns more: the last wave's, parts past the end are zeros
    if (rest && wave == WAVES - 1) {
        const bool there = part * 16 < rest;
        v4i w[MATS * BLOCKS], x[TT];
#pragma unroll
        for (int f = 0; f < MATS * BLOCKS; ++f) w[f] = there ? *reinterpret_cast<const v4i *>(w_at[f] + steps * 64) : v4i{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < TT; ++t) x[t] = there ? *reinterpret_cast<const v4i *>(q_at[t] + steps * 64) : v4i{0, 0, 0, 0};
        products(w, x);
    }

#pragma unroll
    for (int f = 0; f < FRAGS; ++f) parts[wave][f][lane] = acc[f];
    __syncthreads();
    // element i of lane l: row 4 (l / 16) + i of its block, token l % 16 of its tile; here neighbouring threads take neighbouring rows
    const int *sums = reinterpret_cast<const int *>(parts);
    for (int e = threadIdx.x; e < BLOCKS * TT * 256; e += WAVES * 64) {
        const int r = e % (16 * BLOCKS), tok = e / (16 * BLOCKS);
        const int64_t row = row0 + r;
        if (row >= a.m || tok >= a.tokens) continue;
        float v[MATS];
#pragma unroll
        for (int k = 0; k < MATS; ++k) {
            const int frag = (k * BLOCKS + r / 16) * TT + tok / 16;
            const int at = (frag * 64 + (tok % 16) + 16 * ((r % 16) >> 2)) * 4 + (r & 3);
            int sum = 0;
#pragma unroll
            for (int p = 0; p < WAVES; ++p) sum += sums[p * FRAGS * 256 + at];
            v[k] = (float)sum * a.token_scales[tok] * a.channel_scales[k][row];
        }
        float out = v[0], slope;
        if constexpr (MATS == 2) out = activate<false>(v[0], a.activation, slope) * v[MATS - 1];
        a.y[(int64_t)tok * a.m + row] = (uint16_t)to_16(out, a.bf16);
    }
}

template <int TT, int MATS, int BLOCKS, int WAVES>
hipError_t go(const RowsParams &p, hipStream_t stream)
{
    const int64_t blocks = (p.m + 16 * BLOCKS - 1) / (16 * BLOCKS);
    hipLaunchKernelGGL((int8_rows_kernel<TT, MATS, BLOCKS, WAVES>), dim3((unsigned)blocks), dim3(WAVES * 64), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

bool int8_rows_supports(const Int8Args &a) { return a.tokens <= 16; }

hipError_t int8_rows_launch(const Int8Args &a, hipStream_t stream)
{
    RowsParams p{a.q, {a.w[0], a.w[1]}, a.token_scales, {a.channel_scales[0], a.channel_scales[1]}, a.y, a.m, (int)a.n, (int)a.tokens, a.activation, a.bf16};
    if (a.matrices == 2) return go<1, 2, 1, 8>(p, stream);
    return go<1, 1, 1, 8>(p, stream);
}

}  // namespace bcq
