// Microscaled 4-bit floating point: values to codes and scales, and back.
//
// Four lanes take a block of 32 values, eight neighbouring ones each: the largest magnitude by two exchanges of neighbours, its exponent less two
// is the scale's, and the hardware's conversion rounds v / scale to the nearest code, ties to the even one, what is past 6 to 6 (checked on
// every border between codes, at scales from 2^-127 to 2^125).  A lane writes its eight codes as one word, so a wave reads 1 KB (bfloat16) and
// writes 256 bytes in a row.
// Bound: HBM.
#include <hip/hip_runtime.h>
#include <math.h>
#include "block.hpp"
#include "blocks.hpp"
#include "internal.hpp"
#include "lanes.hpp"
#include "values.hpp"

namespace polydl {

// the largest over four neighbouring lanes (quad_perm 1 0 3 2 and 2 3 0 1)
__device__ __forceinline__ uint32_t four_max(uint32_t x)
{
    uint32_t o = (uint32_t)dpp_of<0xb1, 0xf>(0, (int)x);
    x = o > x ? o : x;
    o = (uint32_t)dpp_of<0x4e, 0xf>(0, (int)x);
    return o > x ? o : x;
}

// the codes of v[0 .. 7] / scale, the first in the lowest bits
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[8], float scale)
{
    uint32_t w = 0u;
#if defined(__HIP_DEVICE_COMPILE__)
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
#endif
    return w;
}

constexpr int kMx4Threads = 256;

// `units` words of eight codes a row
template <bool X32>
__global__ __launch_bounds__(kMx4Threads) void mx4_quantise_kernel(int64_t rows, int K, int units, const void *x, int64_t ldx, uint8_t *q, uint8_t *scales)
{
    const int64_t id = (int64_t)block_number() * kMx4Threads + threadIdx.x, r = id / units;
    if (r >= rows) return;                              // (units are whole fours of lanes)
    const int u = (int)(id - r * units), col = u * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (col < K) Values<X32>::load(static_cast<const typename Values<X32>::T *>(x) + r * ldx, col, K, v);
    uint32_t top = 0u;                                  // magnitudes as integers keep their order, infinities and NaN last
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t m = __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu;
        top = m > top ? m : top;
    }
    top = four_max(top) >> 23;
    const uint32_t b = top == 255u ? 255u : top > 2u ? top - 2u : 0u;
    // (a scale of 2^-127 is a float below the normal ones, whose exponent bits are all that the conversion looks at)
    const uint32_t word = mx4_codes(v, __builtin_bit_cast(float, b ? b << 23 : 0x00400000u));
    reinterpret_cast<uint32_t *>(q)[id] = b == 255u ? 0u : word;
    if ((u & 3) == 0) scales[id >> 2] = (uint8_t)b;
}

hipError_t mx4_quantise_launch(int64_t rows, int K, const void *x, int64_t ldx, bool x_f32, uint8_t *q, uint8_t *scales, hipStream_t st)
{
    const int units = mx4_blocks(K) * 4;
    const int64_t blocks = (rows * units + kMx4Threads - 1) / kMx4Threads;
    if (blocks > kMaxBlocks) return hipErrorInvalidValue;
    if (x_f32) return launch_kernel(mx4_quantise_kernel<true>, many_blocks(blocks, kMx4Threads), dim3(kMx4Threads), 0, st, rows, K, units, x, ldx, q, scales);
    return launch_kernel(mx4_quantise_kernel<false>, many_blocks(blocks, kMx4Threads), dim3(kMx4Threads), 0, st, rows, K, units, x, ldx, q, scales);
}

// A code's value, from its bits: two of exponent, one of mantissa; below 1 the mantissa counts halves.
__device__ __forceinline__ float mx4_value(uint32_t code)
{
    const uint32_t m = code & 7u;
    const float v = m < 2u ? 0.5f * (float)m : __builtin_bit_cast(float, (126u << 23) + (m << 22));
    return code & 8u ? -v : v;
}

template <bool Y32>
__global__ __launch_bounds__(kMx4Threads) void mx4_dequantise_kernel(int64_t rows, int K, int units, const uint8_t *q, const uint8_t *scales, void *y,
                                                                     int64_t ldy)
{
    const int64_t id = (int64_t)block_number() * kMx4Threads + threadIdx.x, r = id / units;
    if (r >= rows) return;
    const int col = (int)(id - r * units) * 8;
    if (col >= K) return;
    const uint32_t word = reinterpret_cast<const uint32_t *>(q)[id];
    const int b = scales[id >> 2];
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = b == 255 ? __builtin_nanf("") : ldexpf(mx4_value(word >> (4 * i)), b - 127);
    }
    Values<Y32>::store(static_cast<typename Values<Y32>::T *>(y) + r * ldy, col, K, v);
}

hipError_t mx4_dequantise_launch(int64_t rows, int K, const uint8_t *q, const uint8_t *scales, void *y, int64_t ldy, bool y_f32, hipStream_t st)
{
    const int units = mx4_blocks(K) * 4;
    const int64_t blocks = (rows * units + kMx4Threads - 1) / kMx4Threads;
    if (blocks > kMaxBlocks) return hipErrorInvalidValue;
    if (y_f32) return launch_kernel(mx4_dequantise_kernel<true>, many_blocks(blocks, kMx4Threads), dim3(kMx4Threads), 0, st, rows, K, units, q, scales, y, ldy);
    return launch_kernel(mx4_dequantise_kernel<false>, many_blocks(blocks, kMx4Threads), dim3(kMx4Threads), 0, st, rows, K, units, q, scales, y, ldy);
}

}  // namespace polydl
