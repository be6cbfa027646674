// Rows of 16-bit values to 8-bit codes and one scale per row:  s = max |x| / 127,  q = rint(127 x / max |x|).
//
// The codes are those of exact arithmetic, ties to even.  127 x has 18 bits and is exact in fp32; a ratio 127 x / a of 16-bit
// numbers that is not half an odd number is at least 2^-19 of its size away from one (the difference of 254 x and (2k + 1) a is a
// whole number of units of the smaller one), so a quotient good to fp32's last bit rounds the same way, and the ties themselves
// (x = a / 2 makes 63.5) are numbers that the corrected quotient hits exactly: y = t r, y += (t - y a) r with r close to 1 / a.
// Both x and a are scaled by the power of two that brings a to [1, 2) first, so that nothing on the way overflows or is
// subnormal, whatever the type's range.
//
// Bound by memory: 2 bytes read and 1 written per value, each row held in registers between its two uses.  A row belongs to one
// wave, or to a workgroup of 256 or 1024 threads where it is longer or where there are few rows.
#include "bcq_int8.hpp"

namespace bcq {
namespace {

__device__ __forceinline__ float value_at(const u32x4 &v, int i, bool bf16)
{
    return from_16((i & 1) ? v[i >> 1] >> 16 : v[i >> 1] & 0xffffu, bf16);
}

// THREADS per row, up to CHUNKS pieces of 8 values for each
template <int THREADS, int CHUNKS, bool BF16>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void int8_codes_kernel(const uint16_t *__restrict__ x, int8_t *__restrict__ q,
                                                                                     float *__restrict__ scales, int64_t rows, int n)
{
    constexpr int ROWS = THREADS == 64 ? 4 : 1;
    const int t = threadIdx.x % THREADS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
    if (THREADS == 64 && row >= rows) return;               // (whole waves, and no barrier below)
    const uint16_t *src = x + row * n;
    const int pieces = n >> 3;
    u32x4 v[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = c * THREADS + t;
        v[c] = at < pieces ? *reinterpret_cast<const u32x4 *>(src + (int64_t)at * 8) : u32x4{0, 0, 0, 0};
    }
    // The largest magnitude: as bit patterns without the sign, which order like the values, and above the infinity's if there is a NaN.
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max(v[c][i] & 0x7fffu, (v[c][i] >> 16) & 0x7fffu));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
    if constexpr (THREADS > 64) {
        __shared__ uint32_t tops[THREADS / 64];
        if ((t & 63) == 0) tops[t >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) top = max(top, tops[i]);
    }
    const bool finite = top < (BF16 ? 0x7f80u : 0x7c00u);
    const float a = from_16(top, BF16);
    if (t == 0) scales[row] = finite ? a / 127.f : __builtin_nanf("");
    const bool zero = top == 0 || !finite;
    const int e = zero ? 0 : ilogbf(a);
    const float a1 = zero ? 1.f : ldexpf(a, -e);            // [1, 2)
    const float r = __builtin_amdgcn_rcpf(a1);
    const float k = zero ? 0.f : 127.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = c * THREADS + t;
        uint32_t out[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float num = finite ? ldexpf(value_at(v[c], i, BF16), -e) * k : 0.f;
            float y = num * r;
            y = __builtin_fmaf(__builtin_fmaf(-y, a1, num), r, y);
            const int code = (int)__builtin_rintf(y);
            out[i >> 2] |= ((uint32_t)code & 0xffu) << (8 * (i & 3));
        }
        if (at < pieces) *reinterpret_cast<u32x2 *>(q + row * n + (int64_t)at * 8) = u32x2{out[0], out[1]};
    }
}

template <int THREADS, int CHUNKS>
hipError_t go(const uint16_t *x, bool bf16, int8_t *q, float *scales, int64_t rows, int64_t n, hipStream_t stream)
{
    constexpr int64_t MOST = int64_t(1) << 20;              // rows of a launch, whose threads are counted in 32 bits
    for (int64_t r = 0; r < rows; r += MOST) {
        const int64_t some = rows - r < MOST ? rows - r : MOST, blocks = THREADS == 64 ? (some + 3) / 4 : some;
        const dim3 grid((unsigned)blocks), block(THREADS == 64 ? 256 : THREADS);
        const auto kernel = bf16 ? int8_codes_kernel<THREADS, CHUNKS, true> : int8_codes_kernel<THREADS, CHUNKS, false>;
        hipLaunchKernelGGL(kernel, grid, block, 0, stream, x + r * n, q + r * n, scales + r, some, (int)n);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t int8_quantize_launch(const uint16_t *x, bool bf16, int8_t *q, float *scales, int64_t rows, int64_t n, hipStream_t stream)
{
    if (n <= 4096 && rows >= 1024) return go<64, 8>(x, bf16, q, scales, rows, n, stream);
    if (n <= 4096) return go<256, 2>(x, bf16, q, scales, rows, n, stream);
    if (n <= 16384 && rows >= 256) return go<256, 8>(x, bf16, q, scales, rows, n, stream);
    if (n <= 32768) return go<1024, 4>(x, bf16, q, scales, rows, n, stream);
    return go<1024, 16>(x, bf16, q, scales, rows, n, stream);       // n <= 131072
}

}  // namespace bcq
