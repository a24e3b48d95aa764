// Products of few rows, y[row][n] = act(sum over k of w[n][k] x[row][k]), dense or by expert, with bfloat16 weights or
// with weights in 4 bits: sum over groups g of scale[n][g] * sum over k in g of (q[n][k] - zero[n][g]) * x[row][k].
//
// Bound: the weights' bytes.  No LDS on their way: a wave loads them as operands of v_mfma_f32_16x16x32_bf16, 16 outputs a tile, and
// the rows are the instruction's columns (16, or several sixteens); one row costs as much as 16.  The waves of a workgroup take the
// steps of the reduction in turn, with several steps' loads under way, and meet in LDS, in the order of the waves.
//
// bfloat16 weights [N][K]: a step is 64 inputs, a cache line of each of 16 outputs; a lane loads 16 neighbouring inputs of its
// output, which two instructions take.
//
// 4-bit weights are packed in the order the instruction takes them: 16 outputs and 128 inputs are 64 lanes of 16 bytes, a wave
// reads 1 KB in one load, and a 32-bit word of a lane is its operand of one instruction, whose 32 inputs lie in one group.
// A code becomes a bfloat16 by placing it in the mantissa of 16: 16 + q, exact, two codes a shift and an and-or.  The 16
// and the zero point leave again a group at a time, scale * (sum of (16 + q) x - sum of (16 + zero) x), the second sum from matrix
// instructions of its own.  Products are exact and the sums float32, taken in the same order, so a group of codes that equal the zero
// point gives exactly zero; otherwise both are rounded as sums of terms of up to 31 |x| are.
#include <hip/hip_runtime.h>
#include <type_traits>
#include "blocks.hpp"
#include "experts.hpp"
#include "group_tiles.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace polydl {

typedef __bf16 few_bf16x8 __attribute__((ext_vector_type(8)));
typedef float few_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t few_u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ few_f32x4 few_mfma(lanes_u32x4 a, lanes_u32x4 b, few_f32x4 c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(few_bf16x8, a), __builtin_bit_cast(few_bf16x8, b), c, 0, 0, 0);
#else
    (void)a; (void)b;
    return c;
#endif
}
// Eight values at k of a row of K, zeros past its end.  WHOLE: the step that k lies in ends inside the row, which is the wave's
// to know and costs its lanes nothing.
template <bool WHOLE>
__device__ __forceinline__ lanes_u32x4 few_row(const uint16_t *row, int k, int K)
{
    if constexpr (WHOLE) return load_unit8(row + k);
    return k < K ? load_unit8(row + k, K - k, K) : lanes_u32x4{0u, 0u, 0u, 0u};
}

// Weights<>: what a wave holds of a step of kStep inputs of 16 outputs, kOps instructions' worth.
struct WholeWeights {
    static constexpr int kStep = 64, kOps = 2;
    struct Held { lanes_u32x4 v[kOps]; };
    static __device__ __forceinline__ int input(int i, int quad) { return quad * 16 + i * 8; }
    const uint16_t *row;           // of the lane's output, its inputs of step 0

    __device__ __forceinline__ void init(const FewRowsProblem &p, int e, int tile, int lane)
    {
        row = p.w + ((int64_t)e * p.N + min(tile * 16 + (lane & 15), p.N - 1)) * p.K;
    }
    template <bool WHOLE>
    __device__ __forceinline__ Held load(int s, int K, int lane) const
    {
        Held h;
#pragma unroll
        for (int i = 0; i < kOps; ++i) h.v[i] = few_row<WHOLE>(row, s * kStep + input(i, lane >> 4), K);
        return h;
    }
    template <int CT>
    __device__ __forceinline__ void multiply(const Held &h, const lanes_u32x4 (&x)[CT][kOps], few_f32x4 (&total)[CT]) const
    {
#pragma unroll
        for (int i = 0; i < kOps; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) total[c] = few_mfma(h.v[i], x[c][i], total[c]);
    }
};

// GROUP: inputs of a scale.  ZEROS: there are zero points (a test at run time would make the wave wait for each as it is loaded:
// 32 rows of 64 experts, 2048 x 4096, 48 us against 34).
template <int GROUP, bool ZEROS>
struct CodedWeights {
    static constexpr int kStep = 128, kOps = 4, kGroups = kStep / GROUP, kOpsGroup = kOps / kGroups;
    struct Held { lanes_u32x4 q; few_u32x2 scale[kGroups]; uint32_t zero[kGroups]; };
    static __device__ __forceinline__ int input(int i, int quad) { return i * 32 + quad * 8; }
    // of the tile, step 0 (the same for the wave, so that only 32-bit offsets are the lanes'); no zeros: 8
    const uint8_t *q, *zeros;
    const uint16_t *scales;

    __device__ __forceinline__ void init(const FewRowsProblem &p, int e, int tile, int)
    {
        const int tiles = (p.N + 15) / 16, steps = (p.K + kStep - 1) / kStep;
        const int64_t at = ((int64_t)e * tiles + min(tile, tiles - 1)) * steps;
        q = p.q + at * 1024;
        scales = p.scales + at * (kGroups * 16);
        zeros = ZEROS ? p.zeros + at * (kGroups * 16) : nullptr;
    }
    template <bool WHOLE>
    __device__ __forceinline__ Held load(int s, int, int lane) const
    {
        Held h;
        h.q = *reinterpret_cast<const lanes_u32x4 *>(q + (int64_t)s * 1024 + (uint32_t)lane * 16u);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int64_t at = ((int64_t)s * kGroups + g) * 16;
            h.scale[g] = *reinterpret_cast<const few_u32x2 *>(scales + at + (uint32_t)(lane >> 4) * 4u);   // of four outputs of the result
            h.zero[g] = ZEROS ? zeros[at + (uint32_t)(lane & 15)] : 8u;                                    // of an output among the operands
        }
        return h;
    }
    // eight codes as 16 + q, in the order of the inputs
    static __device__ __forceinline__ lanes_u32x4 codes(uint32_t w)
    {
        // in registers: the and-or has no room for constants, and as constants they are two instructions
        uint32_t mask = 0x00780078u, sixteen = 0x41804180u;
        asm("" : "+v"(mask), "+v"(sixteen));
        return lanes_u32x4{((w << 3) & mask) | sixteen, ((w >> 1) & mask) | sixteen, ((w >> 5) & mask) | sixteen, ((w >> 9) & mask) | sixteen};
    }
    template <int CT>
    __device__ __forceinline__ void multiply(const Held &h, const lanes_u32x4 (&x)[CT][kOps], few_f32x4 (&total)[CT]) const
    {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const uint32_t z = 0x41804180u | h.zero[g] << 3 | h.zero[g] << 19;
            const lanes_u32x4 zero = {z, z, z, z};
            few_f32x4 acc[CT], off[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[c] = off[c] = few_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = g * kOpsGroup; i < (g + 1) * kOpsGroup; ++i) {
                const lanes_u32x4 w = codes(h.q[i]);
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    acc[c] = few_mfma(w, x[c][i], acc[c]);
                    off[c] = few_mfma(zero, x[c][i], off[c]);
                }
            }
            const float scale[4] = {bf16_lo(h.scale[g][0]), bf16_hi(h.scale[g][0]), bf16_lo(h.scale[g][1]), bf16_hi(h.scale[g][1])};
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int c = 0; c < CT; ++c) total[c][n] += scale[n] * (acc[c][n] - off[c][n]);
        }
    }
};

// WAVES waves share a tile of 16 outputs * RT by 16 rows * CT.
template <class W, int RT, int CT, int WAVES, bool OUT_F32>
__global__ __launch_bounds__(WAVES * 64) void few_rows_kernel(FewRowsProblem p, int col_tiles)
{
    __shared__ few_f32x4 sums[WAVES][RT * CT][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quad = lane >> 4;
    GroupTile t;
    GroupTiles all;
    all.init(p.offsets, p.E, p.M, 16 * CT, col_tiles);
    if (!all.find((int)block_number(), &t)) return;
    const int m0 = t.lo + t.m * 16 * CT, rows = min(16 * CT, t.hi - m0), n0 = t.n * RT;     // n0: in sixteens
    const int steps = t.e < p.E ? (p.K + W::kStep - 1) / W::kStep : 0;                      // slots behind the last group: zeros

    const uint16_t *x[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int r = c * 16 + col;
        int src = -1;
        if (r < rows) {
            src = p.rows ? p.rows[m0 + r] : m0 + r;
            if ((unsigned)src >= (unsigned)p.src_rows) src = -1;
        }
        x[c] = src < 0 ? nullptr : p.x + src * p.ldx;
    }
    few_f32x4 total[RT][CT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) total[r][c] = few_f32x4{0.f, 0.f, 0.f, 0.f};

    W weights[RT];
    if (steps > 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r) weights[r].init(p, t.e, n0 + r, lane);
    }
    const auto step = [&](int s, auto whole) {
        typename W::Held w[RT];
        lanes_u32x4 xv[CT][W::kOps];
#pragma unroll
        for (int r = 0; r < RT; ++r) w[r] = weights[r].template load<decltype(whole)::value>(s, p.K, lane);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
#pragma unroll
            for (int i = 0; i < W::kOps; ++i) xv[c][i] = lanes_u32x4{0u, 0u, 0u, 0u};
            if (x[c]) {
#pragma unroll
                for (int i = 0; i < W::kOps; ++i) xv[c][i] = few_row<decltype(whole)::value>(x[c], s * W::kStep + W::input(i, quad), p.K);
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) weights[r].template multiply<CT>(w[r], xv, total[r]);
    };
    const int whole_steps = min(steps, p.K / W::kStep);
    int s = wave;
    for (; s < whole_steps; s += WAVES) step(s, std::true_type{});
    if (s < steps) step(s, std::false_type{});

#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) sums[wave][r * CT + c][lane] = total[r][c];
    __syncthreads();
    const bool whole = (p.ldy & 3) == 0 && ((uintptr_t)p.y & 15) == 0;
    for (int i = wave; i < RT * CT; i += WAVES) {
        few_f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int o = 1; o < WAVES; ++o) v += sums[o][i][lane];
        const int r = i / CT, row = (i - r * CT) * 16 + col, n = (n0 + r) * 16 + quad * 4, left = p.N - n;
        if (row >= rows || left <= 0) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // comparisons that let NaN through, as the formula does
            if (p.act != POLYDL_ACT_NONE) v[q] = v[q] < 0.f ? 0.f : v[q];
            if (p.act == POLYDL_ACT_RELU6) v[q] = v[q] > 6.f ? 6.f : v[q];
        }
        const int64_t at = (m0 + row) * p.ldy + n;
        if constexpr (OUT_F32) {
            float *y = static_cast<float *>(p.y) + at;
            if (whole && left >= 4) {
                *reinterpret_cast<few_f32x4 *>(y) = v;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < left) y[q] = v[q];
            }
        } else {
            uint16_t *y = static_cast<uint16_t *>(p.y) + at;
            if (whole && left >= 4) {
                *reinterpret_cast<few_u32x2 *>(y) = few_u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < left) y[q] = bf16_one(v[q]);
            }
        }
    }
}

template <class W, int RT, int CT, int WAVES>
static hipError_t few_rows_run(const FewRowsProblem &p, hipStream_t st)
{
    const int64_t groups = p.M < p.E + 1 ? p.M : p.E + 1, col_tiles = ((p.N + 15) / 16 + RT - 1) / RT;
    const int64_t tiles = (p.M + groups * (16 * CT - 1)) / (16 * CT) * col_tiles;
    if (tiles > kMaxBlocks) return hipErrorInvalidValue;
    if (p.out_f32)
        return launch_kernel((few_rows_kernel<W, RT, CT, WAVES, true>), many_blocks(tiles, WAVES * 64), dim3(WAVES * 64), 0, st, p, (int)col_tiles);
    return launch_kernel((few_rows_kernel<W, RT, CT, WAVES, false>), many_blocks(tiles, WAVES * 64), dim3(WAVES * 64), 0, st, p, (int)col_tiles);
}

template <class W>
static hipError_t few_rows_pick(const FewRowsProblem &p, hipStream_t st)
{
    const int64_t rows = ((int64_t)p.M + p.E - 1) / p.E;     // of a group, in the mean
    if (rows <= 16) {
        // Two tiles of outputs share the rows' loads; with fewer workgroups than compute units that costs more than it saves (one row, 4096 x
        // 4096 in 4 bits: 4.6 us with one tile, 5.5 with two; 32 rows of 64 experts, 2048 x 4096: 38 and 34).  Four waves take longer over a
        // tile than eight, and more workgroups fit at a time (those 32 rows: 31 us; 16 rows, 8192 x 8192: 13.4 against 13.1).
        const int64_t chunks = p.M < p.E ? p.M : p.E, tiles = chunks * ((p.N + 31) / 32), cus = compute_units();
        return tiles < cus ? few_rows_run<W, 1, 1, 8>(p, st) : tiles < 4 * cus ? few_rows_run<W, 2, 1, 8>(p, st) : few_rows_run<W, 2, 1, 4>(p, st);
    }
    // (bfloat16 weights of more rows are the tiles')
    if constexpr (std::is_same_v<W, WholeWeights>) return hipErrorInvalidValue;
    else return rows <= 32 ? few_rows_run<W, 2, 2, 8>(p, st) : few_rows_run<W, 2, 4, 8>(p, st);
}

template <int GROUP>
static hipError_t few_rows_coded(const FewRowsProblem &p, hipStream_t st)
{
    return p.zeros ? few_rows_pick<CodedWeights<GROUP, true>>(p, st) : few_rows_pick<CodedWeights<GROUP, false>>(p, st);
}

hipError_t few_rows_launch(const FewRowsProblem &p, hipStream_t st)
{
    if (p.w) return few_rows_pick<WholeWeights>(p, st);
    return p.group == 32 ? few_rows_coded<32>(p, st) : p.group == 64 ? few_rows_coded<64>(p, st) : few_rows_coded<128>(p, st);
}

}  // namespace polydl
