// 8-bit products for few tokens: every wave streams rows of weights of its own through LDS of its own.
//
// A workgroup owns 16 BLOCKS rows (of gate and of up, where there are two) and up to 16 TT tokens, mostly all; its waves take equal runs of 128-column steps and meet at
// the end in LDS, with sums of integers, which are the same in any order.  In between they share nothing and wait for nothing but their own loads.
//
// v_mfma_i32_16x16x64_i8 wants 16 bytes of row lane % 16 in a lane.  Loaded like that, straight into registers, neighbouring lanes
// lie in different rows and the memory pipe takes one lane a cycle: 64 cycles per KiB, which bounded 4096 x 14336 at 16 tokens by the loads of both
// operands (14.6 us, 10.6 with one token, whose codes all lanes share; a plain read of the weights 10.1).  So both go into LDS by loads that
// write there, 128 neighbouring bytes of a row at a time, RING steps at once, and come back as operands; the eight 16-byte
// parts of a row sit XOR-permuted by half the row's number, so that sixteen rows' reads use all banks.
//
// Bound by the weights' bytes.
#include <type_traits>

#include "bcq_int8.hpp"
#include "bcq_internal.hpp"

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

constexpr int kStep = 128;

// TT: tiles of 16 tokens, or 0 for one of eight; MATS: matrices; BLOCKS: blocks of 16 rows of each; WAVES per workgroup; RING steps in LDS
template <int TT_, int MATS_, int BLOCKS_, int WAVES_, int RING_>
struct RowsShape {
    static constexpr int TT = TT_ ? TT_ : 1, MATS = MATS_, BLOCKS = BLOCKS_, WAVES = WAVES_, RING = RING_;
    static constexpr int WF = MATS * BLOCKS, FRAGS = WF * TT;
    static constexpr int Q_LOADS = TT_ ? 2 * TT_ : 1, LOADS = 2 * WF + Q_LOADS;    // of 1 KiB: eight rows of 128 bytes
    static constexpr int TOKEN_ROWS = 8 * Q_LOADS;
    static constexpr int STAGE = LOADS * 1024;
    static constexpr int PARTS = WAVES * FRAGS * 1024;                  // the waves' sums
    static constexpr int BYTES = WAVES * RING * STAGE > PARTS ? WAVES * RING * STAGE : PARTS;
};

template <typename S>
__global__ __launch_bounds__(S::WAVES * 64) void int8_rows_kernel(const RowsParams whole_call)
{
    RowsParams a = whole_call;                          // from here on this workgroup's tokens
    const int t0 = (int)blockIdx.y * (S::TT * 16);
    a.q += (int64_t)t0 * a.n;
    a.token_scales += t0;
    a.y += (int64_t)t0 * a.m;
    a.tokens = min(a.tokens - t0, S::TT * 16);
    constexpr int TT = S::TT, MATS = S::MATS, BLOCKS = S::BLOCKS, WAVES = S::WAVES, RING = S::RING, WF = S::WF, FRAGS = S::FRAGS;
    constexpr int RESULTS = BLOCKS * TT * 256, EACH = (RESULTS + WAVES * 64 - 1) / (WAVES * 64);
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row0 = (int64_t)blockIdx.x * (16 * BLOCKS);
    const uint32_t rows = (uint32_t)min((int64_t)(16 * BLOCKS), a.m - row0), n = (uint32_t)a.n;

    // Load k of a matrix brings rows 8k .. 8k+7; lane l delivers the part that belongs at place l % 8 of row 8k + l / 8.  Rows and tokens past the
    // end repeat the last one (their results are not stored).
    uint32_t w_src[2 * BLOCKS], q_src[S::Q_LOADS], part[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) part[k] = ((lane & 7) ^ (((8 * k + (lane >> 3)) >> 1) & 7)) * 16;
#pragma unroll
    for (int k = 0; k < 2 * BLOCKS; ++k) w_src[k] = min((uint32_t)(8 * k + (lane >> 3)), rows - 1) * n;
#pragma unroll
    for (int k = 0; k < S::Q_LOADS; ++k) q_src[k] = min((uint32_t)(8 * k + (lane >> 3)), (uint32_t)a.tokens - 1) * n;

    const int stages = (int)((n + kStep - 1) / kStep);
    const int each = (stages + WAVES - 1) / WAVES;
    const int first = min(wave * each, stages), end = min(first + each, stages);
    // Workgroups begin 128 columns apart, each wave's steps by turns (a part of a step at the row's end stays last): at the same column they would ask
    // for few of memory's channels where a row is a power of two or nearly (28672 x 8192 with one token 43.5 -> 39.2 us; 8192 x 8192 with 8 tokens the other way, 11.7 against 12.2).
    const int whole = end < stages || n % kStep == 0 ? end - first : end - first - 1;
    const int turned = whole > 0 ? (int)(blockIdx.x % (uint32_t)whole) : 0;
    auto turn = [&](int s) { return s >= first + whole ? s : s + turned < first + whole ? s + turned : s + turned - whole; };
    unsigned char *const mine = lds + wave * RING * S::STAGE;
    // Columns of step s into a buffer; in a last step parts past the row's end bring the row's first part instead: what is multiplied with them is
    // set to zero.
    auto stage = [&](int buffer, int s) {
        unsigned char *to = mine + buffer * S::STAGE;
        const uint32_t k0 = (uint32_t)s * kStep;
        uint32_t column[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) column[k] = k0 + part[k] >= n ? 0u : k0 + part[k];
#pragma unroll
        for (int f = 0; f < MATS; ++f) {
            const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.w[f] + row0 * n), 0, (int)(rows * n), 0x00020000);
#pragma unroll
            for (int k = 0; k < 2 * BLOCKS; ++k)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(w_rsrc, (__attribute__((address_space(3))) void *)(to + (f * 2 * BLOCKS + k) * 1024), 16,
                                                         (int)(w_src[k] + column[k & 1]), 0, 0, 0);
        }
        const auto q_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.q), 0, (int)((uint32_t)a.tokens * n), 0x00020000);
#pragma unroll
        for (int k = 0; k < S::Q_LOADS; ++k)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(q_rsrc, (__attribute__((address_space(3))) void *)(to + (2 * WF + k) * 1024), 16,
                                                     (int)(q_src[k] + column[k & 1]), 0, 0, 0);
    };

    v4i acc[FRAGS];
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) acc[f] = v4i{0, 0, 0, 0};
    const uint32_t r16 = lane & 15, quarter = lane >> 4;
    const uint32_t w_row = r16 * kStep, q_row = min(r16, (uint32_t)S::TOKEN_ROWS - 1) * kStep;
    const uint32_t w_swz = (r16 >> 1) & 7, q_swz = (min(r16, (uint32_t)S::TOKEN_ROWS - 1) >> 1) & 7;
    auto multiply = [&](int buffer, auto whole, int s) {
        const unsigned char *from = mine + buffer * S::STAGE;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint32_t p = 4 * kk + quarter;
            v4i w[WF], x[TT];
#pragma unroll
            for (int f = 0; f < WF; ++f) w[f] = *reinterpret_cast<const v4i *>(from + f * 2048 + w_row + ((p ^ w_swz) << 4));
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                x[t] = *reinterpret_cast<const v4i *>(from + WF * 2048 + t * 2048 + q_row + ((p ^ q_swz) << 4));
                if (!decltype(whole)::value && (uint32_t)s * kStep + p * 16 >= n) x[t] = v4i{0, 0, 0, 0};
            }
#pragma unroll
            for (int f = 0; f < WF; ++f)
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[f * TT + t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[f], x[t], acc[f * TT + t], 0, 0, 0);
        }
    };

    constexpr int AHEAD = RING - 1, UNDER_WAY = (AHEAD - 1) * S::LOADS;
    for (int b = 0; b < min(AHEAD, end - first); ++b) stage(b, turn(first + b));
    int buffer = 0, into = AHEAD, s = first;
    auto next = [](int b) { return b + 1 == RING ? 0 : b + 1; };
    // (a step that may be the last and end in the middle is never among these: there is at least one behind it)
    for (; s + AHEAD < end; ++s) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(UNDER_WAY) : "memory");
        stage(into, turn(s + AHEAD));
        multiply(buffer, std::true_type{}, s);
        buffer = next(buffer);
        into = next(into);
    }
    // the scales of this thread's results, beside the last operands: neighbouring threads take neighbouring rows
    float ts[EACH], cs[EACH][MATS];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int e = k * WAVES * 64 + threadIdx.x;
        ts[k] = a.token_scales[min(e / (16 * BLOCKS), a.tokens - 1)];
#pragma unroll
        for (int i = 0; i < MATS; ++i) cs[k][i] = a.channel_scales[i][min(row0 + e % (16 * BLOCKS), a.m - 1)];
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    for (; s < end; ++s) {
        multiply(buffer, std::false_type{}, turn(s));
        buffer = next(buffer);
    }

    __syncthreads();                                    // (the rings are read out: their place is the sums')
    v4i *const parts = reinterpret_cast<v4i *>(lds);
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) parts[(wave * FRAGS + f) * 64 + lane] = acc[f];
    __syncthreads();
    // element i of lane l: row 4 (l / 16) + i of its block, token l % 16 of its tile
    const int *sums = reinterpret_cast<const int *>(lds);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int e = k * WAVES * 64 + threadIdx.x;
        const int r = e % (16 * BLOCKS), tok = e / (16 * BLOCKS);
        const int64_t row = row0 + r;
        if (row >= a.m || tok >= a.tokens) continue;
        float v[MATS];
#pragma unroll
        for (int i = 0; i < MATS; ++i) {
            const int frag = (i * BLOCKS + r / 16) * TT + tok / 16;
            const int at = (frag * 64 + (tok % 16) + 16 * ((r % 16) >> 2)) * 4 + (r & 3);
            int sum = 0;
#pragma unroll
            for (int p = 0; p < WAVES; ++p) sum += sums[p * FRAGS * 256 + at];
            v[i] = (float)sum * ts[k] * cs[k][i];
        }
        float out = v[0], slope;
        if constexpr (MATS == 2) out = activate<false>(v[0], a.activation, slope) * v[MATS - 1];
        a.y[(int64_t)tok * a.m + row] = (uint16_t)to_16(out, a.bf16);
    }
}

template <typename S>
hipError_t go(const RowsParams &p, hipStream_t stream)
{
    static_assert(S::BYTES <= 160 * 1024, "LDS of a CU");
    const int64_t blocks = (p.m + 16 * S::BLOCKS - 1) / (16 * S::BLOCKS);
    const auto kernel = int8_rows_kernel<S>;
    if (hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), S::BYTES)) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks, (unsigned)((p.tokens + S::TT * 16 - 1) / (S::TT * 16))), dim3(S::WAVES * 64), S::BYTES, stream, p);
    return hipGetLastError();
}

// The tokens of a workgroup, 0 for none: up to 16 tokens all of them.  Beyond that as few as leave every workgroup of 16 rows a CU of its own: short matrices
// (1024 x 4096 with 100 tokens: of 16, 32, 64 tokens 4.6, 4.6, 5.8 us, tiles 6.9; 255 x 28672 with 85: 12, 16, 25, tiles 31; 4096 x 14336 with 48:
// of 64 13.6, tiles 16.2), though with many tokens they all bring the codes again (200 x 4096 with 1000: of 64 8.4, tiles 7.3), and with
// two matrices those of 64 only where that is all (gated 860 x 9680 with 222: 22.6, tiles 18.6).  And up to 32 tokens one matrix of at most 16384 rows
// (14336 x 4096 with 24 tokens 10.7, tiles 11.4).  Else a workgroup moves more bytes of codes than of weights, and tiles are ahead (28672 x 8192 with
// 24 tokens 47.1 against 42.4, with 8 tokens 40.1 against 41.9; 7000 x 4096 with 48 tokens 10.5 against 8.1).
int tokens_of(int64_t m, int64_t tokens, int matrices)
{
    if (tokens <= 16) return 16;
    if (tokens <= 256)
        for (int some = 16; some <= 64; some *= 2)
            if ((m + 15) / 16 * ((tokens + some - 1) / some) <= 256 && (matrices == 1 || some < 64 || tokens <= 64)) return some;
    return tokens <= 32 && matrices == 1 && m <= 16384 ? 32 : 0;
}

template <int MATS, typename F>
auto with_shape(int64_t m, int64_t tokens, F f)
{
    // More tokens' codes are worth two blocks of rows, where those still give every CU a workgroup: 14336 x 4096 with 32 tokens 13.6 -> 11.0 us
    // (4096 x 14336 the other way, 11.0 against 15.7); 35840 x 5120 with 16 tokens 41.4 -> 36.5 (with 8 tokens 34.0 both, gated
    // 17920 x 5120 with 16 tokens the other way, 37.2 against 41.5).
    const int some = tokens_of(m, tokens, MATS);
    if (tokens <= 8) return f(RowsShape<0, MATS, 1, 4, 3>{});
    if (some == 16) {
        if constexpr (MATS == 1)
            if (m >= 16384) return f(RowsShape<1, 1, 2, 4, 3>{});
        return f(RowsShape<1, MATS, 1, 4, 3>{});
    }
    if (some == 32) {
        if constexpr (MATS == 1)
            if (m >= 8192) return f(RowsShape<2, 1, 2, 4, 2>{});
        return f(RowsShape<2, MATS, 1, 4, 3>{});
    }
    return f(RowsShape<4, MATS, 1, 4, 3>{});
}

}  // namespace

bool int8_rows_supports(const Int8Args &a) { return tokens_of(a.m, a.tokens, a.matrices) > 0; }

hipError_t int8_rows_launch(const Int8Args &a, hipStream_t stream)
{
    const RowsParams p{a.q, {a.w[0], a.w[1]}, a.token_scales, {a.channel_scales[0], a.channel_scales[1]}, a.y, a.m, (int)a.n, (int)a.tokens,
                       a.activation, a.bf16};
    auto run = [&](auto shape) { return go<decltype(shape)>(p, stream); };
    return a.matrices == 2 ? with_shape<2>(a.m, a.tokens, run) : with_shape<1>(a.m, a.tokens, run);
}

Int8Layout int8_rows_layout(const Int8Args &a)
{
    auto layout = [&](auto shape) {
        using S = decltype(shape);
        const int steps = (int)((a.n + kStep - 1) / kStep);
        return Int8Layout{16 * S::WF, S::Q_LOADS == 1 ? 8 : 16 * S::TT, kStep, S::WAVES, S::RING, (steps + S::WAVES - 1) / S::WAVES, S::BYTES};
    };
    return a.matrices == 2 ? with_shape<2>(a.m, a.tokens, layout) : with_shape<1>(a.m, a.tokens, layout);
}

}  // namespace bcq
