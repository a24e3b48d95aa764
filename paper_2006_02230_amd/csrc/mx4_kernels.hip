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

// A thread takes kMx4Held words of eight codes, a workgroup's threads side by side.  Where a word lies in its row takes a division; rows that are whole and follow
// one another without gaps (FLAT) need none, and fewer than 2^32 words one of 32 bits (131072 x 1024 values and back: 74 + 86 us with 64-bit divisions and one word a
// thread).
constexpr int kMx4Threads = 256, kMx4Held = 4;
enum { MX4_FLAT = 0, MX4_SHORT = 1, MX4_LONG = 2 };
struct Mx4Place { int64_t row; int col; };
template <int KIND>
__device__ __forceinline__ Mx4Place mx4_place(int64_t id, int units)
{
    if constexpr (KIND == MX4_FLAT) return {0, 0};
    if constexpr (KIND == MX4_SHORT) {
        const uint32_t r = (uint32_t)id / (uint32_t)units;
        return {r, (int)((uint32_t)id - r * (uint32_t)units) * 8};
    }
    const int64_t r = id / units;
    return {r, (int)(id - r * units) * 8};
}
inline int mx4_kind(int64_t rows, int K, int64_t ld)
{
    return ld == K && K % 128 == 0 ? MX4_FLAT : rows * mx4_blocks(K) * 4 < 1ll << 32 ? MX4_SHORT : MX4_LONG;
}

// `words` words of eight codes in all, `units` a row
template <bool X32, int KIND>
__global__ __launch_bounds__(kMx4Threads) void mx4_quantise_kernel(int64_t words, int K, int units, const void *x, int64_t ldx, uint8_t *q, uint8_t *scales)
{
    using V = Values<X32>;
    const int64_t id0 = (int64_t)block_number() * (kMx4Threads * kMx4Held) + threadIdx.x;
    typename V::Raw raw[kMx4Held];
#pragma unroll
    for (int i = 0; i < kMx4Held; ++i) {
        const int64_t id = id0 + i * kMx4Threads;
        raw[i] = {};
        if (id >= words) continue;                      // (words are whole fours of lanes)
        if constexpr (KIND == MX4_FLAT) {
            raw[i] = V::load_raw(static_cast<const typename V::T *>(x) + id * 8, 0, 8);
        } else {
            const Mx4Place at = mx4_place<KIND>(id, units);
            if (at.col < K) raw[i] = V::load_raw(static_cast<const typename V::T *>(x) + at.row * ldx, at.col, K);
        }
    }
#pragma unroll
    for (int i = 0; i < kMx4Held; ++i) {
        const int64_t id = id0 + i * kMx4Threads;
        float v[8];
        V::convert(raw[i], v);
        uint32_t top = 0u;                              // magnitudes as integers keep their order, infinities and NaN last
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t m = __builtin_bit_cast(uint32_t, v[j]) & 0x7fffffffu;
            top = m > top ? m : top;
        }
        top = four_max(top) >> 23;
        const uint32_t b = top == 255u ? 255u : top > 2u ? top - 2u : 0u;
        // (a scale of 2^-127 is a float below the normal ones, whose exponent bits are all that the conversion looks at)
        const uint32_t word = mx4_codes(v, __builtin_bit_cast(float, b ? b << 23 : 0x00400000u));
        if (id >= words) continue;
        reinterpret_cast<uint32_t *>(q)[id] = b == 255u ? 0u : word;
        if ((id & 3) == 0) scales[id >> 2] = (uint8_t)b;
    }
}

template <bool X32, int KIND>
static hipError_t mx4_quantise_run(int64_t words, int K, int units, const void *x, int64_t ldx, uint8_t *q, uint8_t *scales, hipStream_t st)
{
    const int64_t blocks = (words + kMx4Threads * kMx4Held - 1) / (kMx4Threads * kMx4Held);
    if (blocks > kMaxBlocks) return hipErrorInvalidValue;
    return launch_kernel((mx4_quantise_kernel<X32, KIND>), many_blocks(blocks, kMx4Threads), dim3(kMx4Threads), 0, st, words, K, units, x, ldx, q, scales);
}

hipError_t mx4_quantise_launch(int64_t rows, int K, const void *x, int64_t ldx, bool x_f32, uint8_t *q, uint8_t *scales, hipStream_t st)
{
    const int units = mx4_blocks(K) * 4, kind = mx4_kind(rows, K, rows == 1 ? K : ldx);
    auto *f = kind == MX4_FLAT    ? (x_f32 ? mx4_quantise_run<true, MX4_FLAT> : mx4_quantise_run<false, MX4_FLAT>)
              : kind == MX4_SHORT ? (x_f32 ? mx4_quantise_run<true, MX4_SHORT> : mx4_quantise_run<false, MX4_SHORT>)
                                  : (x_f32 ? mx4_quantise_run<true, MX4_LONG> : mx4_quantise_run<false, MX4_LONG>);
    return f(rows * units, K, units, x, ldx, q, scales, st);
}

// A code's value, from its bits: two of exponent, one of mantissa; below 1 the mantissa counts halves.
__device__ __forceinline__ float mx4_value(uint32_t code)
{
    const uint32_t m = code & 7u;
    const float v = m < 2u ? 0.5f * (float)m : __builtin_bit_cast(float, (126u << 23) + (m << 22));
    return code & 8u ? -v : v;
}

template <bool Y32, int KIND>
__global__ __launch_bounds__(kMx4Threads) void mx4_dequantise_kernel(int64_t words, int K, int units, const uint8_t *q, const uint8_t *scales, void *y,
                                                                     int64_t ldy)
{
    using V = Values<Y32>;
    const int64_t id0 = (int64_t)block_number() * (kMx4Threads * kMx4Held) + threadIdx.x;
    uint32_t word[kMx4Held];
    int b[kMx4Held];
#pragma unroll
    for (int i = 0; i < kMx4Held; ++i) {
        const int64_t id = min(id0 + i * kMx4Threads, words - 1);
        word[i] = reinterpret_cast<const uint32_t *>(q)[id];
        b[i] = scales[id >> 2];
    }
#pragma unroll
    for (int i = 0; i < kMx4Held; ++i) {
        const int64_t id = id0 + i * kMx4Threads;
        if (id >= words) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = b[i] == 255 ? __builtin_nanf("") : ldexpf(mx4_value(word[i] >> (4 * j)), b[i] - 127);
        if constexpr (KIND == MX4_FLAT) {
            V::store(static_cast<typename V::T *>(y) + id * 8, 0, 8, v);
        } else {
            const Mx4Place at = mx4_place<KIND>(id, units);
            if (at.col < K) V::store(static_cast<typename V::T *>(y) + at.row * ldy, at.col, K, v);
        }
    }
}

template <bool Y32, int KIND>
static hipError_t mx4_dequantise_run(int64_t words, int K, int units, const uint8_t *q, const uint8_t *scales, void *y, int64_t ldy, hipStream_t st)
{
    const int64_t blocks = (words + kMx4Threads * kMx4Held - 1) / (kMx4Threads * kMx4Held);
    if (blocks > kMaxBlocks) return hipErrorInvalidValue;
    return launch_kernel((mx4_dequantise_kernel<Y32, KIND>), many_blocks(blocks, kMx4Threads), dim3(kMx4Threads), 0, st, words, K, units, q, scales, y, ldy);
}

hipError_t mx4_dequantise_launch(int64_t rows, int K, const uint8_t *q, const uint8_t *scales, void *y, int64_t ldy, bool y_f32, hipStream_t st)
{
    const int units = mx4_blocks(K) * 4, kind = mx4_kind(rows, K, rows == 1 ? K : ldy);
    auto *f = kind == MX4_FLAT    ? (y_f32 ? mx4_dequantise_run<true, MX4_FLAT> : mx4_dequantise_run<false, MX4_FLAT>)
              : kind == MX4_SHORT ? (y_f32 ? mx4_dequantise_run<true, MX4_SHORT> : mx4_dequantise_run<false, MX4_SHORT>)
                                  : (y_f32 ? mx4_dequantise_run<true, MX4_LONG> : mx4_dequantise_run<false, MX4_LONG>);
    return f(rows * units, K, units, q, scales, y, ldy, st);
}

}  // namespace polydl
