// Products of few rows with 4-bit weights, y[row][n] = act(sum over groups g of scale[n][g] * sum over k in g of
// (q[n][k] - zero[n][g]) * x[row][k]), dense or by expert, and the packing of the weights.
//
// Bound: the weights' bytes.  They are packed in the order the matrix instruction takes them: 16 outputs and 128 inputs are 64
// lanes of 16 bytes, so a wave reads 1 KB in one load, and a 32-bit word of a lane is its operand of one
// v_mfma_f32_16x16x32_bf16 whose 32 inputs lie in one group.  Rows are the instruction's columns (16, or several sixteens);
// one row costs as much as 16.
// A code becomes a bfloat16 by placing it in the mantissa of 16: 16 + q, exact, two codes a shift and an and-or.  The 16
// and the zero point leave again a group at a time, scale * (sum of (16 + q) x - sum of (16 + zero) x), the second sum from matrix
// instructions of its own.  Products are exact and the sums float32, taken in the same order, so a group of codes that equal the zero
// point gives exactly zero; otherwise both are rounded as sums of terms of up to 31 |x| are.
// The waves of a workgroup take the steps of 128 inputs in turn and meet in LDS, in the order of the waves.
#include <hip/hip_runtime.h>
#include "experts.hpp"
#include "group_tiles.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace polydl {

typedef __bf16 w4_bf16x8 __attribute__((ext_vector_type(8)));
typedef float w4_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w4_u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ w4_f32x4 w4_mfma(lanes_u32x4 a, lanes_u32x4 b, w4_f32x4 c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(w4_bf16x8, a), __builtin_bit_cast(w4_bf16x8, b), c, 0, 0, 0);
#else
    (void)a; (void)b;
    return c;
#endif
}
// eight codes as 16 + q, in the order of the inputs
__device__ __forceinline__ lanes_u32x4 w4_codes(uint32_t w)
{
    constexpr uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
    return lanes_u32x4{((w << 3) & mask) | sixteen, ((w >> 1) & mask) | sixteen, ((w >> 5) & mask) | sixteen, ((w >> 9) & mask) | sixteen};
}

// WAVES waves share a tile of 16 outputs * RT by 16 rows * CT; STEPS steps of a wave are under way at a time.
template <int RT, int CT, int WAVES, int STEPS, bool OUT_F32>
__global__ __launch_bounds__(WAVES * 64) void w4_kernel(W4Problem p, int col_tiles)
{
    __shared__ w4_f32x4 sums[WAVES][RT * CT][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quad = lane >> 4;
    GroupTile t;
    GroupTiles all;
    all.init(p.offsets, p.E, p.M, 16 * CT, col_tiles);
    if (!all.find((int)blockIdx.x, &t)) return;
    const int m0 = t.lo + t.m * 16 * CT, rows = min(16 * CT, t.hi - m0), n0 = t.n * RT;     // n0: in sixteens
    const int tiles = (p.N + 15) / 16, steps = (p.K + 127) / 128, per_step = 128 / p.group, groups = steps * per_step;
    const int words = p.group / 32;                    // matrix instructions of a group

    const uint16_t *x[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int r = c * 16 + col;
        int src = -1;
        if (r < rows) {
            src = p.rows ? p.rows[m0 + r] : m0 + r;
            if ((unsigned)src >= (unsigned)p.src_rows) src = -1;
        }
        x[c] = src < 0 ? nullptr : p.x + src * p.ldx + quad * 8;
    }
    const int64_t tile0 = (int64_t)t.e * tiles + n0;
    w4_f32x4 total[RT][CT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) total[r][c] = w4_f32x4{0.f, 0.f, 0.f, 0.f};

    if (t.e < p.E)                                     // slots behind the last group: a result of zeros
    for (int s0 = wave; s0 < steps; s0 += WAVES * STEPS) {
        lanes_u32x4 w[STEPS][RT], xv[STEPS][CT][4];
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int s = s0 + u * WAVES;
            if (s >= steps) continue;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int tile = min(n0 + r, tiles - 1) - n0;
                w[u][r] = *reinterpret_cast<const lanes_u32x4 *>(p.q + (((tile0 + tile) * steps + s) * 64 + lane) * 16);
            }
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = s * 128 + i * 32 + quad * 8;
                    xv[u][c][i] = lanes_u32x4{0u, 0u, 0u, 0u};
                    if (x[c] && k < p.K) xv[u][c][i] = load_unit8(x[c] + (s * 128 + i * 32), p.K - k);
                }
        }
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int s = s0 + u * WAVES;
            if (s >= steps) continue;
            w4_f32x4 acc[RT][CT], off[RT][CT];
            lanes_u32x4 zero[RT];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t group = s * per_step + i / words;
                if (i % words == 0) {
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const int64_t at = ((tile0 + min(n0 + r, tiles - 1) - n0) * groups + group) * 16;
                        const uint32_t z = p.zeros ? p.zeros[at + col] : 8u, both = 0x41804180u | z << 3 | z << 19;
                        zero[r] = lanes_u32x4{both, both, both, both};
#pragma unroll
                        for (int c = 0; c < CT; ++c) acc[r][c] = off[r][c] = w4_f32x4{0.f, 0.f, 0.f, 0.f};
                    }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const lanes_u32x4 codes = w4_codes(w[u][r][i]);
#pragma unroll
                    for (int c = 0; c < CT; ++c) {
                        acc[r][c] = w4_mfma(codes, xv[u][c][i], acc[r][c]);
                        off[r][c] = w4_mfma(zero[r], xv[u][c][i], off[r][c]);
                    }
                }
                if ((i + 1) % words != 0) continue;
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const int64_t at = ((tile0 + min(n0 + r, tiles - 1) - n0) * groups + group) * 16 + quad * 4;
                    const w4_u32x2 sc = *reinterpret_cast<const w4_u32x2 *>(p.scales + at);
                    const float scale[4] = {bf16_lo(sc[0]), bf16_hi(sc[0]), bf16_lo(sc[1]), bf16_hi(sc[1])};
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int c = 0; c < CT; ++c) total[r][c][q] += scale[q] * (acc[r][c][q] - off[r][c][q]);
                }
            }
        }
    }

#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) sums[wave][r * CT + c][lane] = total[r][c];
    __syncthreads();
    const bool whole = (p.ldy & 3) == 0 && ((uintptr_t)p.y & 15) == 0;
    for (int i = wave; i < RT * CT; i += WAVES) {
        w4_f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int o = 1; o < WAVES; ++o) v += sums[o][i][lane];
        const int r = i / CT, row = (i - r * CT) * 16 + col, n = (n0 + r) * 16 + quad * 4, left = p.N - n;
        if (row >= rows || left <= 0) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (p.act != POLYDL_ACT_NONE) v[q] = v[q] < 0.f ? 0.f : v[q];
            if (p.act == POLYDL_ACT_RELU6) v[q] = v[q] > 6.f ? 6.f : v[q];
        }
        const int64_t at = (m0 + row) * p.ldy + n;
        if constexpr (OUT_F32) {
            float *y = static_cast<float *>(p.y) + at;
            if (whole && left >= 4) {
                *reinterpret_cast<w4_f32x4 *>(y) = v;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < left) y[q] = v[q];
            }
        } else {
            uint16_t *y = static_cast<uint16_t *>(p.y) + at;
            if (whole && left >= 4) {
                *reinterpret_cast<w4_u32x2 *>(y) = w4_u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < left) y[q] = bf16_one(v[q]);
            }
        }
    }
}

template <int RT, int CT, int WAVES, int STEPS>
static hipError_t w4_run(const W4Problem &p, hipStream_t st)
{
    const int64_t groups = p.M < p.E + 1 ? p.M : p.E + 1, col_tiles = ((p.N + 15) / 16 + RT - 1) / RT;
    const int64_t tiles = (p.M + groups * (16 * CT - 1)) / (16 * CT) * col_tiles;
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;
    if (p.out_f32) return launch_kernel((w4_kernel<RT, CT, WAVES, STEPS, true>), dim3((unsigned)tiles), dim3(WAVES * 64), 0, st, p, (int)col_tiles);
    return launch_kernel((w4_kernel<RT, CT, WAVES, STEPS, false>), dim3((unsigned)tiles), dim3(WAVES * 64), 0, st, p, (int)col_tiles);
}

hipError_t w4_launch(const W4Problem &p, hipStream_t st)
{
    const int rows = (p.M + p.E - 1) / p.E;            // of a group, in the mean
    if (rows <= 16) return w4_run<1, 1, 8, 4>(p, st);
    if (rows <= 32) return w4_run<2, 2, 8, 1>(p, st);
    return w4_run<2, 4, 8, 1>(p, st);
}

// ---- packing ------------------------------------------------------------------------------------------------------
// One wave a tile of 16 outputs and 128 inputs.  Without zero points: scale = max |w| / 7, q = round(w / scale) + 8, so
// codes 1 to 15.  With: scale = (max(w, 0) - min(w, 0)) / 15, zero = round(-min / scale).  Scales are rounded to bfloat16
// first and the codes found with the rounded scale.  Outputs past N have scale 0, inputs past K the code of a zero.
__global__ __launch_bounds__(64) void w4_pack_kernel(int N, int K, int group, int tiles, int steps, const uint16_t *w, uint8_t *q,
                                                     uint16_t *scales, uint8_t *zeros)
{
    const int lane = threadIdx.x, row = lane & 15, quad = lane >> 4;
    const int64_t id = blockIdx.x;
    const int64_t tile = id / steps;
    const int s = (int)(id - tile * steps);
    const int64_t e = tile / tiles;
    const int n = (int)(tile - e * tiles) * 16 + row;
    const int words = group / 32;
    float v[4][8], lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = s * 128 + i * 32 + quad * 8;
        lanes_u32x4 u = {0u, 0u, 0u, 0u};
        if (n < N && k < K) u = load_unit8(w + (e * N + n) * K + k, K - k);
        lo[i] = hi[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[i][j] = j & 1 ? bf16_hi(u[j >> 1]) : bf16_lo(u[j >> 1]);
            lo[i] = fminf(lo[i], v[i][j]);
            hi[i] = fmaxf(hi[i], v[i][j]);
        }
#pragma unroll
        for (int x = 16; x < 64; x += 16) {
            if (x == 48) continue;
            lo[i] = fminf(lo[i], __shfl_xor(lo[i], x));
            hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], x));
        }
    }
    if (words >= 2) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            lo[i] = lo[i + 1] = fminf(lo[i], lo[i + 1]);
            hi[i] = hi[i + 1] = fmaxf(hi[i], hi[i + 1]);
        }
    }
    if (words == 4) {
        lo[0] = lo[1] = lo[2] = lo[3] = fminf(lo[0], lo[2]);
        hi[0] = hi[1] = hi[2] = hi[3] = fmaxf(hi[0], hi[2]);
    }
    lanes_u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float top = zeros ? (hi[i] - lo[i]) / 15.f : fmaxf(hi[i], -lo[i]) / 7.f;
        const uint16_t bits = bf16_one(top);
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
    if (all > 0x7fffffff) return hipErrorInvalidValue;
    return launch_kernel(w4_pack_kernel, dim3((unsigned)all), dim3(64), 0, st, N, K, group, tiles, steps, w, q, scales, zeros);
}

}  // namespace polydl
