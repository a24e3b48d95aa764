// The packing of weights into 4-bit codes, scales and zero points (few_rows.hip multiplies with them).
#include <hip/hip_runtime.h>
#include <math.h>
#include "blocks.hpp"
#include "experts.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace polydl {

// One wave a tile of 16 outputs and 128 inputs.  Without zero points: scale = max |w| / 7, q = round(w / scale) + 8, so
// codes 1 to 15.  With: scale = (max(w, 0) - min(w, 0)) / 15, zero = round(-min / scale).  Scales are rounded to bfloat16
// first and the codes found with the rounded scale.  Outputs past N have scale 0, inputs past K the code of a zero.  A NaN goes through
// the extremes, an infinity becomes one: no code holds either, so the group's scale is NaN.
__global__ __launch_bounds__(64) void w4_pack_kernel(int E, int N, int K, int group, int tiles, int steps, const uint16_t *w, uint8_t *q,
                                                     uint16_t *scales, uint8_t *zeros)
{
    const int lane = threadIdx.x, row = lane & 15, quad = lane >> 4;
    const int64_t id = block_number(), tile = id / steps;
    const int s = (int)(id - tile * steps);
    const int64_t e = tile / tiles;
    if (e >= E) return;
    const int n = (int)(tile - e * tiles) * 16 + row;
    const int words = group / 32;
    float v[4][8], lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = s * 128 + i * 32 + quad * 8;
        lanes_u32x4 u = {0u, 0u, 0u, 0u};
        if (n < N && k < K) u = load_unit8(w + (e * N + n) * K + k, K - k, K);
        lo[i] = hi[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[i][j] = j & 1 ? bf16_hi(u[j >> 1]) : bf16_lo(u[j >> 1]);
            lo[i] = __builtin_elementwise_minimum(lo[i], v[i][j]);
            hi[i] = __builtin_elementwise_maximum(hi[i], v[i][j]);
        }
#pragma unroll
        for (int x = 16; x < 64; x += 16) {
            if (x == 48) continue;
            lo[i] = __builtin_elementwise_minimum(lo[i], __shfl_xor(lo[i], x));
            hi[i] = __builtin_elementwise_maximum(hi[i], __shfl_xor(hi[i], x));
        }
    }
    if (words >= 2) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            lo[i] = lo[i + 1] = __builtin_elementwise_minimum(lo[i], lo[i + 1]);
            hi[i] = hi[i + 1] = __builtin_elementwise_maximum(hi[i], hi[i + 1]);
        }
    }
    if (words == 4) {
        lo[0] = lo[1] = lo[2] = lo[3] = __builtin_elementwise_minimum(lo[0], lo[2]);
        hi[0] = hi[1] = hi[2] = hi[3] = __builtin_elementwise_maximum(hi[0], hi[2]);
    }
    lanes_u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool finite = hi[i] < INFINITY && lo[i] > -INFINITY;
        // (halves: the range may pass the largest float; halving is exact, so the quotient is the same)
        const float top = zeros ? (0.5f * hi[i] - 0.5f * lo[i]) / 7.5f : fmaxf(hi[i], -lo[i]) / 7.f;
        const uint16_t bits = bf16_one(finite ? top : __builtin_nanf(""));
        const float scale = bf16_lo(bits), some = scale > 0.f ? scale : 1.f;
        const float zero = zeros ? fminf(fmaxf(rintf(-lo[i] / some), 0.f), 15.f) : 8.f;
        uint32_t word = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t code = (uint32_t)fminf(fmaxf(rintf(v[i][j] / some) + zero, 0.f), 15.f);
            word |= code << (4 * (j / 2 + 4 * (j % 2)));
        }
        out[i] = word;
        if (i % words == 0 && quad == 0) {
            const int64_t at = (tile * steps * (4 / words) + s * (4 / words) + i / words) * 16 + row;
            scales[at] = bits;
            if (zeros) zeros[at] = (uint8_t)zero;
        }
    }
    *reinterpret_cast<lanes_u32x4 *>(q + (id * 64 + lane) * 16) = out;
}

hipError_t w4_pack_launch(int E, int N, int K, int group, const uint16_t *w, uint8_t *q, uint16_t *scales, uint8_t *zeros, hipStream_t st)
{
    const int tiles = (N + 15) / 16, steps = (K + 127) / 128;
    const int64_t all = (int64_t)E * tiles * steps;
    if (all > kMaxBlocks) return hipErrorInvalidValue;
    return launch_kernel(w4_pack_kernel, many_blocks(all, 64), dim3(64), 0, st, E, N, K, group, tiles, steps, w, q, scales, zeros);
}

}  // namespace polydl
