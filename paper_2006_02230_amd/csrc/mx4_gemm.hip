// Products of matrices in microscaled 4 bits, grouped by expert: y[s] = act(x[r(s)] w_e^T).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 rows of two blocks from each operand, a block and its scale a lane, forms the products of the
// codes exactly, scales them and adds them up in float32.
#include <hip/hip_runtime.h>
#include "block.hpp"
#include "blocks.hpp"
#include "group_tiles.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace polydl {

typedef int mx4_i32x8 __attribute__((ext_vector_type(8)));
typedef float mx4_f32x16 __attribute__((ext_vector_type(16)));

// 16 bytes of codes in the eight words that the instruction's widest operands take; the upper four are not read for 4-bit ones
__device__ __forceinline__ mx4_i32x8 mx4_operand(lanes_u32x4 v)
{
    return mx4_i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}
// BYTE: which byte of the scales' words
template <int BYTE>
__device__ __forceinline__ mx4_f32x16 mx4_mfma(lanes_u32x4 a, lanes_u32x4 b, mx4_f32x16 c, uint32_t a_scale, uint32_t b_scale)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(a), mx4_operand(b), c, 4, 4, BYTE, (int)a_scale, BYTE, (int)b_scale);
#else
    (void)a; (void)b; (void)a_scale; (void)b_scale;
    return c;
#endif
}
// comparisons that let NaN through, as the formula does
__device__ __forceinline__ float mx4_act(float v, int act)
{
    if (act != POLYDL_ACT_NONE) v = v < 0.f ? 0.f : v;
    if (act == POLYDL_ACT_RELU6) v = v > 6.f ? 6.f : v;
    return v;
}

// A wave a tile of 32 x 32, straight from memory.
template <bool OUT_F32>
__global__ __launch_bounds__(64) void mx4_wave_kernel(Mx4Problem p, int col_tiles)
{
    const int lane = threadIdx.x, l = lane & 31, half = lane >> 5;
    GroupTile t;
    GroupTiles all;
    all.init(p.offsets, p.E, p.M, 32, col_tiles);
    if (!all.find((int)block_number(), &t)) return;
    const int m0 = t.lo + t.m * 32, rows = min(32, t.hi - m0), n0 = t.n * 32;
    const int steps = t.e < p.E ? p.KB / 2 : 0;             // slots behind the last group: zeros
    int src = -1;
    if (l < rows) {
        src = p.rows ? p.rows[m0 + l] : m0 + l;
        if ((unsigned)src >= (unsigned)p.x_rows) src = -1;
    }
    const int64_t row = src, col = (int64_t)min(t.e, p.E - 1) * p.N + min(n0 + l, p.N - 1);
    mx4_f32x16 acc = {0.f};
    for (int s = 0; s < steps; ++s) {
        lanes_u32x4 x = {0u, 0u, 0u, 0u};
        uint32_t xs = 0u;
        if (src >= 0) {
            x = reinterpret_cast<const lanes_u32x4 *>(p.xq)[row * p.KB + s * 2 + half];
            xs = p.xs[row * p.KB + s * 2 + half];
        }
        const lanes_u32x4 w = reinterpret_cast<const lanes_u32x4 *>(p.wq)[col * p.KB + s * 2 + half];
        acc = mx4_mfma<0>(w, x, acc, p.ws[col * p.KB + s * 2 + half], xs);
    }
    // a lane's results: row l of the tile, columns 8 (i / 4) + 4 half + i % 4
    if (l >= rows) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int n = n0 + 8 * (i / 4) + 4 * half + i % 4;
        if (n >= p.N) continue;
        const int64_t at = (int64_t)(m0 + l) * p.ldy + n;
        const float v = mx4_act(acc[i], p.act);
        if constexpr (OUT_F32) static_cast<float *>(p.y)[at] = v;
        else static_cast<uint16_t *>(p.y)[at] = bf16_one(v);
    }
}

hipError_t mx4_gemm_launch(const Mx4Problem &p, hipStream_t st)
{
    const int64_t groups = p.M < p.E + 1 ? p.M : p.E + 1, col_tiles = (p.N + 31) / 32;
    const int64_t tiles = (p.M + groups * 31) / 32 * col_tiles;
    if (tiles > kMaxBlocks) return hipErrorInvalidValue;
    if (p.out_f32) return launch_kernel(mx4_wave_kernel<true>, many_blocks(tiles, 64), dim3(64), 0, st, p, (int)col_tiles);
    return launch_kernel(mx4_wave_kernel<false>, many_blocks(tiles, 64), dim3(64), 0, st, p, (int)col_tiles);
}

}  // namespace polydl
