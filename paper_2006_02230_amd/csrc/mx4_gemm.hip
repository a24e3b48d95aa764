// Products of matrices in microscaled 4 bits, grouped by expert: y[s] = act(x[r(s)] w_e^T).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 rows of two blocks from each operand, a block and its scale a lane, forms the products of the
// codes exactly, scales them and adds them up in float32.
#include <hip/hip_runtime.h>
#include <type_traits>
#include "block.hpp"
#include "blocks.hpp"
#include "group_tiles.hpp"
#include "internal.hpp"
#include "lanes.hpp"
#include "lds_loads.hpp"

namespace polydl {

typedef int mx4_i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t mx4_u32x2 __attribute__((ext_vector_type(2)));
typedef float mx4_f32x4 __attribute__((ext_vector_type(4)));
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

// A wave a tile of 32 x 32, straight from memory: where the tiles' 32-bit offsets do not reach.
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

// ---- few rows ---------------------------------------------------------------------------------------------------
// Bound: the weights' bytes.  No LDS on their way: a wave loads them as operands of v_mfma_scale_f32_16x16x128_f8f6f4, 16 outputs a tile, and
// the rows are the instruction's columns; one row costs as much as 16.  A step is 256 inputs, a cache line of each of 16 outputs: a lane loads two
// neighbouring blocks of its output and their scales, which two instructions take.  The waves of a workgroup take the steps in turn
// and meet in LDS, in the order of the waves.
struct Mx4Held { lanes_u32x4 v[2]; uint32_t scale; };
// blocks 8 s + 2 quad and the next of a row (NULL: zeros)
__device__ __forceinline__ Mx4Held mx4_pair(const uint8_t *q, const uint8_t *scales, int s, int quad, int KB)
{
    Mx4Held h = {{lanes_u32x4{0u, 0u, 0u, 0u}, lanes_u32x4{0u, 0u, 0u, 0u}}, 0u};
    const int b = s * 8 + quad * 2;
    if (q && b < KB) {
        h.v[0] = reinterpret_cast<const lanes_u32x4 *>(q)[b];
        h.v[1] = reinterpret_cast<const lanes_u32x4 *>(q)[b + 1];
        h.scale = *reinterpret_cast<const uint16_t *>(scales + b);
    }
    return h;
}
template <int BYTE>
__device__ __forceinline__ mx4_f32x4 mx4_few_mfma(const Mx4Held &a, const Mx4Held &b, mx4_f32x4 c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(a.v[BYTE]), mx4_operand(b.v[BYTE]), c, 4, 4, BYTE, (int)a.scale, BYTE, (int)b.scale);
#else
    (void)a; (void)b;
    return c;
#endif
}

// WAVES waves share a tile of 16 outputs * RT by 16 rows.
template <int RT, int WAVES, bool OUT_F32>
__global__ __launch_bounds__(WAVES * 64) void mx4_few_kernel(Mx4Problem p, int col_tiles)
{
    __shared__ mx4_f32x4 sums[WAVES][RT][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_value(tid >> 6), col = lane & 15, quad = lane >> 4;
    GroupTile t;
    GroupTiles all;
    all.init(p.offsets, p.E, p.M, 16, col_tiles);
    if (!all.find((int)block_number(), &t)) return;
    const int m0 = t.lo + t.m * 16, rows = min(16, t.hi - m0), n0 = t.n * RT * 16;
    const int steps = t.e < p.E ? (p.KB + 7) / 8 : 0;                                       // slots behind the last group: zeros
    const uint8_t *w[RT], *ws[RT];
    int src = -1;
    if (col < rows) {
        src = p.rows ? p.rows[m0 + col] : m0 + col;
        if ((unsigned)src >= (unsigned)p.x_rows) src = -1;
    }
    const uint8_t *x = nullptr, *xs = nullptr;
    if (src >= 0) {
        x = p.xq + (int64_t)src * p.KB * 16;
        xs = p.xs + (int64_t)src * p.KB;
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int64_t n = (int64_t)min(t.e, p.E - 1) * p.N + min(n0 + r * 16 + col, p.N - 1);
        w[r] = p.wq + n * p.KB * 16;
        ws[r] = p.ws + n * p.KB;
    }
    mx4_f32x4 total[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) total[r] = mx4_f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = wave; s < steps; s += WAVES) {
        Mx4Held a[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) a[r] = mx4_pair(w[r], ws[r], s, quad, p.KB);
        const Mx4Held b = mx4_pair(x, xs, s, quad, p.KB);
#pragma unroll
        for (int r = 0; r < RT; ++r) total[r] = mx4_few_mfma<1>(a[r], b, mx4_few_mfma<0>(a[r], b, total[r]));
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) sums[wave][r][lane] = total[r];
    __syncthreads();
    const bool whole = (p.ldy & 3) == 0 && ((uintptr_t)p.y & 15) == 0;
    for (int r = wave; r < RT; r += WAVES) {
        mx4_f32x4 v = sums[0][r][lane];
#pragma unroll
        for (int o = 1; o < WAVES; ++o) v += sums[o][r][lane];
        const int n = n0 + r * 16 + quad * 4, left = p.N - n;
        if (col >= rows || left <= 0) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = mx4_act(v[q], p.act);
        const int64_t at = (m0 + col) * p.ldy + n;
        if constexpr (OUT_F32) {
            float *y = static_cast<float *>(p.y) + at;
            if (whole && left >= 4) {
                *reinterpret_cast<mx4_f32x4 *>(y) = v;
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < left) y[q] = v[q];
            }
        } else {
            uint16_t *y = static_cast<uint16_t *>(p.y) + at;
            if (whole && left >= 4) {
                *reinterpret_cast<mx4_u32x2 *>(y) = mx4_u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < left) y[q] = bf16_one(v[q]);
            }
        }
    }
}

template <int RT, int WAVES>
static hipError_t mx4_few_run(const Mx4Problem &p, hipStream_t st)
{
    const int64_t groups = p.M < p.E + 1 ? p.M : p.E + 1, col_tiles = ((p.N + 15) / 16 + RT - 1) / RT;
    const int64_t tiles = (p.M + groups * 15) / 16 * col_tiles;
    if (tiles > kMaxBlocks) return hipErrorInvalidValue;
    if (p.out_f32) return launch_kernel((mx4_few_kernel<RT, WAVES, true>), many_blocks(tiles, WAVES * 64), dim3(WAVES * 64), 0, st, p, (int)col_tiles);
    return launch_kernel((mx4_few_kernel<RT, WAVES, false>), many_blocks(tiles, WAVES * 64), dim3(WAVES * 64), 0, st, p, (int)col_tiles);
}

// ---- tiles ------------------------------------------------------------------------------------------------------
// A workgroup owns tiles of BM rows by BN columns, one after another, and walks the reduction in stages of 256 inputs, 128 bytes of codes a row,
// BUFFERS of them in LDS; a wave keeps a tile WM x WN in registers.  Codes lie in LDS as they lie in memory, the unit (block) c of a row in
// place c ^ ((row >> 1) & 7), so that 16 neighbouring rows' units fall on different banks (row & 7: nearly twice the conflicts).  An instruction j of the stage's four takes the blocks j and
// 4 + j, one a half wave: a lane's four scales of a stage are then one word, of which the instruction picks byte j.
// Loads go from memory into LDS without registers; lanes without a row, or past the end of theirs, use an offset out of the
// descriptor's range, which reads as zero.  Scales come 16 bytes a row, for two stages: a load of 4 bytes fetches as many cache lines (8192 x 8192 x
// 8192, loads of 4 bytes for every stage 257 us, without scales 219).
// The stages follow one another from tile to tile: while the last ones of a tile are multiplied, the first ones of the next are on their way.
constexpr int kMx4Stage = 8;                                 // blocks

template <int BM, int BN, int WM, int WN, int BUFFERS>
struct Mx4Tile {
    static constexpr int kThreads = (BM / WM) * (BN / WN) * 64, kBuffers = BUFFERS;
    static constexpr int kStageBytes = (BM + BN) * 128;
    static constexpr int kSlots = BUFFERS / 2 + 1, kSlotBytes = (BM + BN) * 16;                 // scales of two stages
    static constexpr int kScalesAt = BUFFERS * kStageBytes, kOutAt = kScalesAt + kSlots * kSlotBytes;
    static constexpr int kOut = 2048;                        // of a wave: its results' way out
    static constexpr int kLds = kOutAt + kThreads / 64 * kOut;
    static constexpr int kUnitsA = BM * 8 / kThreads, kUnitsB = BN * 8 / kThreads, kLoads = kUnitsA + kUnitsB;
    static_assert(BM * 8 % kThreads == 0 && BN * 8 % kThreads == 0 && BM % 64 == 0 && BN % 64 == 0 && BM + BN <= kThreads, "whole loads of waves");
    static_assert(BUFFERS == 2 || BUFFERS == 4, "stages come in pairs");
};

typedef lanes_u32x4 __attribute__((aligned(2))) Mx4Halves8;

template <class T, int BM, int BN, int WM, int WN, bool GATHER, bool OUT_F32, bool PAST>
__global__ __launch_bounds__(T::kThreads) void mx4_tile_kernel(Mx4Problem p, int col_tiles)
{
    extern __shared__ __align__(1024) char mx4_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_value(tid >> 6), l32 = lane & 31, half = lane >> 5;
    constexpr int kAcross = BN / WN, MI = WM / 32, NI = WN / 32, kBuffers = T::kBuffers;
    const int wm = wave / kAcross * WM, wn = wave % kAcross * WN;
    const uint32_t row_bytes = (uint32_t)p.KB * 16u;
    const int stages = (p.KB + kMx4Stage - 1) / kMx4Stage, padded = max((stages + 1) & ~1, kBuffers);   // with stages of zeros
    GroupTiles tiles;
    tiles.init(p.offsets, p.E, p.M, BM, col_tiles);

    // Of the tile that is being loaded: the offsets of the thread's units from the bases, which move along with the stages.
    uint32_t off_a[T::kUnitsA], off_b[T::kUnitsB], off_s = 0;
    uint64_t base_a = 0, base_b = 0, base_s = 0;
    struct Out { int rows, cols; int64_t at; };
    const auto turn = [](int r) { return (r >> 1) & 7; };

    // Sets up tile `id` for loading; where there is none its loads are of zeros.  Returns whether there is one.
    const auto find = [&](int id, Out &out) {
        GroupTile t;
        const bool there = tiles.find(id, &t);
        const bool zeros = !there || t.e >= p.E;             // slots behind the last group: a result of zeros
        const int m0 = zeros ? 0 : t.lo + t.m * BM, n0 = zeros ? 0 : t.n * BN, e = zeros ? 0 : t.e;
        out.rows = there ? min(BM, t.hi - (t.lo + t.m * BM)) : 0;
        out.cols = there ? min(BN, p.N - t.n * BN) : 0;
        out.at = there ? (int64_t)(t.lo + t.m * BM) * p.ldy + t.n * BN : 0;
        const int rows = zeros ? 0 : out.rows, cols = zeros ? 0 : out.cols;
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                        // (what depends on it is formed anew for each tile, not kept through the products)
        const auto row_of = [&](int r) {
            int from = r < rows ? r : -1;
            if (GATHER && from >= 0) {
                from = p.rows[m0 + r];
                if ((unsigned)from >= (unsigned)p.x_rows) from = -1;
            }
            return from;
        };
#pragma unroll
        for (int i = 0; i < T::kUnitsA; ++i) {
            const int at = i * T::kThreads + tid, r = at >> 3, from = row_of(r);
            off_a[i] = from < 0 ? kFarOffset : (uint32_t)from * row_bytes + (uint32_t)((at & 7) ^ turn(r)) * 16u;
        }
#pragma unroll
        for (int i = 0; i < T::kUnitsB; ++i) {
            const int at = i * T::kThreads + tid, r = at >> 3;
            off_b[i] = r >= cols ? kFarOffset : (uint32_t)r * row_bytes + (uint32_t)((at & 7) ^ turn(r)) * 16u;
        }
        const int from = tid < BM ? row_of(tid) : tid - BM < cols ? tid - BM : -1;               // a row's scales each thread
        off_s = from < 0 ? kFarOffset : (uint32_t)from * (uint32_t)p.KB;
        const uint64_t a0 = GATHER ? 0 : (uint64_t)m0, b0 = (uint64_t)e * p.N + n0;
        base_a = wave_value((uint64_t)p.xq + a0 * row_bytes);
        base_b = wave_value((uint64_t)p.wq + b0 * row_bytes);
        base_s = wave_value(wave * 64 < BM ? (uint64_t)p.xs + a0 * (uint64_t)p.KB : (uint64_t)p.ws + b0 * (uint64_t)p.KB);
        return there;
    };
    const uint32_t lds0 = gg_lds_offset(mx4_lds);
    // The scales of the stages s and s+1 (s even) of the tile that is being loaded.  Rows of less than 16 scales come word by word, the last 16 of longer ones
    // whole: then the row's words lie later_words(s) words further on in LDS.
    const auto first_scale = [&](int s) { return min(s * kMx4Stage, max(p.KB - 16, 0)); };
    const auto later_words = [&](int s) { return (s * kMx4Stage - first_scale(s)) >> 2; };
    const auto load_scales = [&](int s, int slot) {
        if (wave * 64 >= BM + BN) return;
        const uint32_t at = lds0 + T::kScalesAt + (uint32_t)slot * T::kSlotBytes;
        const int from = first_scale(s);
        if (p.KB >= 16) {
            gg_dma(gg_rsrc(base_s + (uint32_t)from, (int64_t)kFarRecords), at + (uint32_t)wave * 1024u, s < stages ? off_s : kFarOffset);
        } else {
            // a wave's 64 rows, 16 of them at a time; the offsets are in the lanes of the rows
            int lane = threadIdx.x & 63;
            asm volatile("" : "+v"(lane));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t o = (uint32_t)__shfl((int)off_s, i * 16 + (lane >> 2));
                gg_dma_word(gg_rsrc(base_s, (int64_t)kFarRecords), at + (uint32_t)(wave * 64 + i * 16) * 16u,
                            o == kFarOffset || s > 0 || (lane & 3) * 4 >= p.KB ? kFarOffset : o + (uint32_t)(lane & 3) * 4u);
            }
        }
    };
    // A stage is fetched in kLoads loads after begin().  A thread's units lie in the same place of their rows, so they all are behind the rows' end or none is.
    const int unit_of = (tid & 7) ^ turn(tid >> 3);
    static_assert(T::kThreads / 8 % 16 == 0, "turn()");
    gg_i32x4 rsrc_a, rsrc_b;
    uint32_t far = 0;
    const auto begin = [&](int s) {
        rsrc_a = gg_rsrc(base_a, (int64_t)kFarRecords);
        rsrc_b = gg_rsrc(base_b, (int64_t)kFarRecords);
        base_a += kMx4Stage * 16;
        base_b += kMx4Stage * 16;
        far = s * kMx4Stage + unit_of < p.KB ? 0u : kFarOffset;
    };
    // g counts the stages from the first tile on
    const auto load = [&](uint32_t g, int i) {
        const uint32_t at = lds0 + g % kBuffers * T::kStageBytes;
        if (i < T::kUnitsA) gg_dma(rsrc_a, at + (uint32_t)(i * T::kThreads + wave * 64) * 16u, off_a[i] | far);
        else gg_dma(rsrc_b, at + BM * 128u + (uint32_t)((i - T::kUnitsA) * T::kThreads + wave * 64) * 16u, off_b[i - T::kUnitsA] | far);
    };
    const auto load_all = [&](uint32_t g) {
#pragma unroll
        for (int i = 0; i < T::kLoads; ++i) load(g, i);
    };
    // Waits until this wave's loads are down to those of BEHIND stages (scales not counted: they come before their stage) and what it has stored since, then
    // for the other waves.  Loads and global (not flat) stores are counted and end in their order, as the compiler's own waits take them to.
    const auto land = [&](auto behind, auto stores) {
        asm volatile("" ::: "memory");
        gg_wait<decltype(behind)::value * T::kLoads + decltype(stores)::value>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const uint32_t read_a = (uint32_t)((wm + l32) * 128 + (half * 4 ^ turn(l32)) * 16), read_b = read_a + (uint32_t)((BM + wn - wm) * 128);
    // the n-th operand of instruction j of a stage: the columns', then the rows'
    const auto read = [&](uint32_t g, int j, int n, lanes_u32x4 (&a)[MI], lanes_u32x4 (&b)[NI]) {
        // (the stages and rows begin at multiples of 128, so the units' places can be turned last)
        const uint32_t at = (n < NI ? read_b : read_a) + g % kBuffers * T::kStageBytes;
        const char *from = mx4_lds + (at ^ (uint32_t)(j * 16));
        if (n < NI) b[n] = *reinterpret_cast<const lanes_u32x4 *>(from + n * 32 * 128);
        else a[n - NI] = *reinterpret_cast<const lanes_u32x4 *>(from + (n - NI) * 32 * 128);
    };
    // the n-th operand's scales of the g-th stage, stage s of its tile; behind the rows' end they are zero (`there`: all ones, or zero for the half wave)
    const uint32_t read_as = (uint32_t)(T::kScalesAt + (wm + l32) * 16 + half * 4), read_bs = read_as + (uint32_t)((BM + wn - wm) * 16);
    const auto scales_at = [&](uint32_t g, int s) { return (g >> 1) % T::kSlots * T::kSlotBytes + (uint32_t)((s & 1) * 2 + later_words(s & ~1)) * 4u; };
    const auto read_scale = [&](uint32_t at, int n, uint32_t (&a)[MI], uint32_t (&b)[NI]) {
        if (n < NI) b[n] = *reinterpret_cast<const uint32_t *>(mx4_lds + read_bs + at + n * 32 * 16);
        else a[n - NI] = *reinterpret_cast<const uint32_t *>(mx4_lds + read_as + at + (n - NI) * 32 * 16);
    };
    const auto mask_scales = [&](uint32_t there, uint32_t (&a)[MI], uint32_t (&b)[NI]) {
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] &= there;
#pragma unroll
        for (int n = 0; n < NI; ++n) b[n] &= there;
    };
    const auto there_of = [&](int s) { return s * kMx4Stage + half * 4 < p.KB ? 0xffffffffu : 0u; };

    mx4_f32x16 acc[MI][NI];
    lanes_u32x4 a0[MI], b0[NI], a1[MI], b1[NI];              // operands of an instruction and of the next one
    uint32_t as[2][MI], bs[2][NI];                           // scales of a stage and of the next one
    // Instruction j of stage g, and meanwhile the reads for the one after it; the last of a stage also asks for the stage that takes its buffer, between all
    // its products (between the first two of them: 2 % slower).
    // next: the number of stage g+1 in its tile.
    const auto step = [&](uint32_t g, int next, auto which, auto odd, auto first, auto stores, const lanes_u32x4 (&a)[MI], const lanes_u32x4 (&b)[NI],
                          lanes_u32x4 (&a_next)[MI], lanes_u32x4 (&b_next)[NI]) {
        constexpr int J = decltype(which)::value, kOdd = decltype(odd)::value;
        constexpr bool kLast = J == 3;
        if constexpr (kLast) land(std::integral_constant<int, kBuffers - 2>{}, stores);      // stage g+1; and this wave has what it read of stage g
        constexpr int kReads = MI + NI, kAll = MI * NI;
        const uint32_t scales = kLast ? scales_at(g + 1, next) : 0u, there = kLast ? there_of(next) : 0u;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int at = i * NI + n;
                acc[i][n] = mx4_mfma<J>(b[n], a[i], decltype(first)::value ? mx4_f32x16{0.f} : acc[i][n], bs[kOdd][n], as[kOdd][i]);
#pragma unroll
                for (int r = at * kReads / kAll; r < (at + 1) * kReads / kAll; ++r) {
                    read(g + kLast, (J + 1) & 3, r, a_next, b_next);
                    if constexpr (kLast) read_scale(scales, r, as[1 - kOdd], bs[1 - kOdd]);
                }
                if constexpr (kLast) {
#pragma unroll
                    for (int r = at * T::kLoads / kAll; r < (at + 1) * T::kLoads / kAll; ++r) load(g + kBuffers, r);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        if constexpr (kLast) mask_scales(there, as[1 - kOdd], bs[1 - kOdd]);       // (one by one each would be waited for)
    };
    constexpr std::true_type yes;
    constexpr std::false_type no;
    constexpr std::integral_constant<int, 0> none;
    const auto first_reads = [&](uint32_t g, int s, auto odd) {
        constexpr int kOdd = decltype(odd)::value;
        const uint32_t scales = scales_at(g, s), there = there_of(s);
#pragma unroll
        for (int n = 0; n < MI + NI; ++n) {
            read(g, 0, n, a0, b0);
            read_scale(scales, n, as[kOdd], bs[kOdd]);
        }
        mask_scales(there, as[kOdd], bs[kOdd]);
    };

    // Out through LDS, each wave through a part of its own: a lane then stores 16 bytes and the lanes of a row follow one another.
    constexpr int kUnit = OUT_F32 ? 4 : 8, kCols = OUT_F32 || WN < 64 ? 32 : 64, kUnits = kCols / kUnit;      // values of a unit, columns and units of a part
    constexpr int kRows = T::kOut / (kUnits * 16), kTwist = kUnits - 1;
    constexpr int kStores = WM * WN * (OUT_F32 ? 4 : 2) / 1024;                                              // of a wave whose part is whole
    static_assert(kRows == 16 || kRows == 32, "half a result or a whole one");
    char *const mine = mx4_lds + T::kOutAt + wave * T::kOut;
    const auto leave = [&](const Out &out) {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));
        const int l32 = lane & 31, half = lane >> 5;
        if (p.act != POLYDL_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int n = 0; n < NI; ++n)
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        acc[i][n][q] = __builtin_elementwise_maximum(acc[i][n][q], 0.f);         // (lets NaN through, as the formula does)
                        if (p.act == POLYDL_ACT_RELU6) acc[i][n][q] = __builtin_elementwise_minimum(acc[i][n][q], 6.f);
                    }
        }
        const bool whole = wave_value((int)(out.rows >= wm + WM && out.cols >= wn + WN && p.ldy < (1 << 24)));
        constexpr int kSize = OUT_F32 ? 4 : 2;
        char *const y0 = static_cast<char *>(p.y) + (out.at + (int64_t)wm * p.ldy + wn) * kSize;
        const uint32_t y_off = (uint32_t)(lane / kUnits) * (uint32_t)(p.ldy * kSize) + (uint32_t)(lane % kUnits) * 16u;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += kRows)
#pragma unroll
                for (int c0 = 0; c0 < WN; c0 += kCols) {
                    // A wave's LDS accesses are in order, but lanes read here what others wrote: without the statements around the writes the
                    // compiler may keep what a lane has read where that lane itself wrote nothing since.
                    asm volatile("" ::: "memory");
                    if (kRows == 32 || (l32 & 16) == r0) {
                        const int r = l32 & (kRows - 1);
#pragma unroll
                        for (int n = 0; n < kCols / 32; ++n)
#pragma unroll
                            for (int g = 0; g < 4; ++g) {
                                const mx4_f32x16 &v = acc[i][c0 / 32 + n];
                                const int col = n * 32 + g * 8 + half * 4;
                                char *at = mine + (r * kUnits + ((col / kUnit) ^ (r & kTwist))) * 16;
                                if constexpr (OUT_F32) *reinterpret_cast<mx4_f32x4 *>(at) = mx4_f32x4{v[g * 4], v[g * 4 + 1], v[g * 4 + 2], v[g * 4 + 3]};
                                else
                                    *reinterpret_cast<mx4_u32x2 *>(at + half * 8) = mx4_u32x2{bf16_pair(v[g * 4], v[g * 4 + 1]), bf16_pair(v[g * 4 + 2], v[g * 4 + 3])};
                            }
                    }
                    asm volatile("" ::: "memory");
#pragma unroll
                    for (int k = 0; k < kRows * kUnits / 64; ++k) {
                        const int r = k * (64 / kUnits) + lane / kUnits, u = lane % kUnits;
                        const lanes_u32x4 v = *reinterpret_cast<const lanes_u32x4 *>(mine + (r * kUnits + (u ^ (r & kTwist))) * 16);
                        if (whole) {
                            Mx4Halves8 *at = reinterpret_cast<Mx4Halves8 *>(y0 + (uint64_t)(i * 32 + r0 + k * (64 / kUnits)) * (uint64_t)(p.ldy * kSize) + c0 * kSize + y_off);
                            if constexpr (PAST) __builtin_nontemporal_store(v, at);
                            else *at = v;
                            continue;
                        }
                        const int row = wm + i * 32 + r0 + r, n = wn + c0 + u * kUnit, left = out.cols - n;
                        if (row >= out.rows || left <= 0) continue;
                        const int64_t at = out.at + (int64_t)row * p.ldy + n;
                        if constexpr (OUT_F32) {
                            float *y = static_cast<float *>(p.y) + at;
                            const mx4_f32x4 f = __builtin_bit_cast(mx4_f32x4, v);
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                if (q < left) y[q] = f[q];
                        } else {
                            store_unit8(static_cast<uint16_t *>(p.y) + at, v, left);
                        }
                    }
                }
        // the next tile's first wait counts the stores of a whole part
        if (!whole) gg_wait<0>();
    };

    int id = (int)block_number();
    Out now, next;
    if (!find(id, now)) return;
    next = now;
    bool more = true;                                        // there is a next tile (or it is not known yet)
    int at = 0;                                              // the stage that is fetched next, of the tile that is being loaded
    // Sets a stage up for loading, an even one with its scales and those of the stage after it.
    const auto advance = [&](uint32_t g, auto even) {
        if constexpr (decltype(even)::value) load_scales(at, (int)((g >> 1) % T::kSlots));
        begin(at);
        ++at;
    };
#pragma unroll
    for (int g = 0; g < kBuffers; ++g) {
        if (g & 1) advance((uint32_t)g, no);
        else advance((uint32_t)g, yes);
        load_all((uint32_t)g);
    }
    land(none, none);
    first_reads(0u, 0, none);
    uint32_t g = 0;
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    const auto stage = [&](int next_stage, auto odd, auto first, auto stores) {
        step(g, next_stage, std::integral_constant<int, 0>{}, odd, first, none, a0, b0, a1, b1);
        step(g, next_stage, std::integral_constant<int, 1>{}, odd, no, none, a1, b1, a0, b0);
        step(g, next_stage, std::integral_constant<int, 2>{}, odd, no, none, a0, b0, a1, b1);
        step(g, next_stage, std::integral_constant<int, 3>{}, odd, no, stores, a1, b1, a0, b0);
    };
    // a stage without products: a wave whose part of the tile does not exist takes part in the loads, and so does every wave in a stage of zeros
    const auto pass = [&](int next_stage, auto next_odd) {
        land(std::integral_constant<int, kBuffers - 2>{}, none);
        load_all(g + kBuffers);
        first_reads(g + 1, next_stage, next_odd);
    };
    while (true) {
        const bool busy = wave_value((int)(wm < now.rows && wn < now.cols));
        for (int s = 0; s < padded; s += 2) {
            // (Here, where the loop branches anyway: at a branch between them the compiler gathers the matrix instructions on one side of it.)
            if (at == padded) {                              // the tile is loaded: on to the next one
                at = 0;
                id += (int)gridDim.x;
                more = find(id, next);
            }
            advance(g + kBuffers, yes);
            if (!busy || s >= stages) pass(s + 1, odd);
            else if (s == 0) stage(1, even, yes, std::integral_constant<int, kStores>{});
            else stage(s + 1, even, no, none);
            ++g;
            advance(g + kBuffers, no);
            const int after = s + 2 == padded ? 0 : s + 2;
            if (!busy || s + 1 >= stages) pass(after, even);
            else stage(after, odd, no, none);
            ++g;
        }
        leave(now);
        if (!more) break;
        now = next;
    }
    gg_wait<0>();                                            // no load into LDS is under way when the workgroup gives it back
}

template <int BM, int BN, int WM, int WN, int BUFFERS, bool GATHER, bool OUT_F32, bool PAST>
static hipError_t mx4_tile_launch(const Mx4Problem &p, hipStream_t st)
{
    using T = Mx4Tile<BM, BN, WM, WN, BUFFERS>;
    constexpr auto kernel = mx4_tile_kernel<T, BM, BN, WM, WN, GATHER, OUT_F32, PAST>;
    // each group, and the slots behind the last, may end in a partial tile
    const int64_t groups = p.M < p.E + 1 ? p.M : p.E + 1, col_tiles = (p.N + BN - 1) / BN;
    int64_t tiles = (p.M + groups * (BM - 1)) / BM * col_tiles;
    if (tiles > kMaxBlocks) return hipErrorInvalidValue;       // (a tile's number plus the workgroups is an int too)
    const int64_t fit = (int64_t)compute_units() * (160 * 1024 / T::kLds);
    if (tiles > fit) tiles = fit;
    if (T::kLds > 64 * 1024) {
        const hipError_t e = ask_lds<kernel>(T::kLds);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(kernel, dim3((unsigned)tiles), dim3(T::kThreads), T::kLds, st, p, (int)col_tiles);
}

template <int BM, int BN, int WM, int WN, int BUFFERS>
static hipError_t mx4_tile_pick(const Mx4Problem &p, hipStream_t st)
{
    // results that no cache would hold until they are read go past the L2, which keeps the operands
    const bool past = BM == 256 && (int64_t)p.M * p.N * (p.out_f32 ? 4 : 2) > 192ll << 20;
    if constexpr (BM == 256) {
        if (past && p.rows) return p.out_f32 ? mx4_tile_launch<BM, BN, WM, WN, BUFFERS, true, true, true>(p, st) : mx4_tile_launch<BM, BN, WM, WN, BUFFERS, true, false, true>(p, st);
        if (past) return p.out_f32 ? mx4_tile_launch<BM, BN, WM, WN, BUFFERS, false, true, true>(p, st) : mx4_tile_launch<BM, BN, WM, WN, BUFFERS, false, false, true>(p, st);
    }
    if (p.rows) return p.out_f32 ? mx4_tile_launch<BM, BN, WM, WN, BUFFERS, true, true, false>(p, st) : mx4_tile_launch<BM, BN, WM, WN, BUFFERS, true, false, false>(p, st);
    return p.out_f32 ? mx4_tile_launch<BM, BN, WM, WN, BUFFERS, false, true, false>(p, st) : mx4_tile_launch<BM, BN, WM, WN, BUFFERS, false, false, false>(p, st);
}

template <bool OUT_F32>
static hipError_t mx4_wave_launch(const Mx4Problem &p, hipStream_t st)
{
    const int64_t groups = p.M < p.E + 1 ? p.M : p.E + 1, col_tiles = (p.N + 31) / 32;
    const int64_t tiles = (p.M + groups * 31) / 32 * col_tiles;
    if (tiles > kMaxBlocks) return hipErrorInvalidValue;
    return launch_kernel(mx4_wave_kernel<OUT_F32>, many_blocks(tiles, 64), dim3(64), 0, st, p, (int)col_tiles);
}

// Rounds of `at_a_time` workgroups that tiles of `tile` squared take, groups of the mean length taken to end in half a tile each.
static int64_t mx4_rounds(const Mx4Problem &p, int64_t tile, int64_t at_a_time)
{
    const int64_t across = (p.N + tile - 1) / tile, down = p.E == 1 ? (p.M + tile - 1) / tile : (p.M + p.E * (tile / 2) + tile - 1) / tile;
    return (across * down + at_a_time - 1) / at_a_time;
}

hipError_t mx4_gemm_launch(const Mx4Problem &p, hipStream_t st)
{
    const int64_t rows = ((int64_t)p.M + p.E - 1) / p.E, cus = compute_units();           // rows of a group, in the mean
    // One matrix and up to 16 rows (16 rows, 8192 x 8192: 12.4 us, in tiles of 64 17.4), or up to 8 rows a group, where tiles are as fast for many
    // weights but slower for few (64 groups of 4 rows, 2048 x 4096: 67 / 64 us, 16 of 4 rows, 1024 x 1024: 4.9 / 5.9; but 64 of 16 rows: 97 / 73).
    if (rows <= (p.E == 1 ? 16 : 8)) {
        // two tiles of outputs share the rows' loads; with fewer workgroups than compute units that costs more than it saves (one row, 4096 x 4096: 5.6
        // us with one tile and eight waves, 6.8 with two; 32 rows of 64 experts, 2048 x 4096: 32 with one, 27 with two and four waves)
        const int64_t chunks = p.M < p.E ? p.M : p.E, tiles = chunks * ((p.N + 31) / 32);
        return tiles < cus ? mx4_few_run<1, 8>(p, st) : mx4_few_run<2, 4>(p, st);
    }
    // offsets inside a tile (rows by index: inside the tensor) below 2^32
    if ((p.rows && p.x_rows > 256 ? (int64_t)p.x_rows : 256ll) * p.KB * 16 < 0xf0000000ll) {
        // Tiles of 256 (one workgroup on a compute unit), of 128 or of 64 (two).  A round of 128 takes 0.62 of a round of 256 and does half the work, one of 64
        // takes a third for an eighth.  64 / 128 / 256, us (three sets of random operands in turn, in a graph): one group of 4096 rows, 4096 x 4096, 85 / 47 / 40; 16
        // uneven ones of 2048 in the mean, 4096 x 2048, 363 / 214 / 169 (3.2 PFLOP/s); of 256, 2048 x 2048, 28 / 20 / 22; of 128 17 / 14 / 18; of 32 11 / 13 / 17; 7
        // of 286, 777 x 531, 7.5 / 9.6 / 15.
        const double of256 = (double)mx4_rounds(p, 256, cus), of128 = 0.62 * (double)mx4_rounds(p, 128, 2 * cus), of64 = 0.33 * (double)mx4_rounds(p, 64, 2 * cus);
        if (of256 <= of128 && of256 <= of64) return mx4_tile_pick<256, 256, 128, 64, 2>(p, st);
        return of128 <= of64 ? mx4_tile_pick<128, 128, 64, 64, 2>(p, st) : mx4_tile_pick<64, 64, 32, 32, 4>(p, st);
    }
    return p.out_f32 ? mx4_wave_launch<true>(p, st) : mx4_wave_launch<false>(p, st);
}

}  // namespace polydl
