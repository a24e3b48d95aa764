// Matrix products grouped by expert, bfloat16 operands, float32 sums: the forward product of the rows of each group with
// the group's weights, and the gradients of the rows and of the weights.
//
// One kernel in three forms.  A workgroup owns a tile BM x BN of one group's result and walks the reduction in stages of 64,
// two or four of them in LDS; a wave keeps a tile WM x WN in registers as 16x16 results of v_mfma_f32_16x16x32_bf16.
// An operand lies in LDS as it lies in memory, in units of eight values (16 bytes):
//   * reduction innermost (both operands of the forward product, the rows of the gradient of the rows): [row][64]; a lane
//     reads the eight values of its row that one instruction takes.  The unit c of a row is stored in place c ^ (row & 7), so
//     that the lanes of one read fall on different banks (counted for whole kernels, results' way out included: 0.16 conflict cycles an LDS
//     instruction in the forward product, 0.12 in dX, none in dW).
//   * reduction outermost (weights in the gradient of the rows, both operands in that of the weights): [64][columns]; the
//     transposing LDS read gives a lane four values of its column from four rows.  Blocks of 16 columns are stored in the
//     block's place ^ a number of the row that differs for the eight rows that half a wave reads at a time.
// Loads go from memory into LDS without registers; the permutation is applied to the address a lane loads from.  Lanes past an
// edge use an offset out of the descriptor's range, which reads as zero: rows that the plan does not have, columns past the
// last, the reduction's tail.  The kernel reads the group of its tile from the offsets in device memory, so nothing waits for
// the host.
#include <hip/hip_runtime.h>
#include <type_traits>
#include "blocks.hpp"
#include "experts.hpp"
#include "gemm_core.hpp"
#include "group_tiles.hpp"
#include "internal.hpp"
#include "lds_loads.hpp"

namespace polydl {

typedef __bf16 gg_bf16x8 __attribute__((ext_vector_type(8)));
typedef float gg_f32x4 __attribute__((ext_vector_type(4)));
typedef short gg_i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t gg_u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStage = 64;                          // reduction of a stage: two matrix instructions' of 32
constexpr int kIndices = 4096;                      // row indices of the reduction kept in LDS at a time

struct GroupedArgs {
    int E, M, out_rows, cols, red;
    const int32_t *offsets, *rows;
    int src_rows;
    const char *a, *b;
    int64_t lda, ldb;              // bytes
    void *c;
    int64_t ldc;                   // elements
    int accumulate, act;
    const uint16_t *h;
    int64_t ldh;
    int row_tiles, col_tiles;      // of one C_e (GROUPED_DW); columns (others)
};

__device__ __forceinline__ gg_u32x2 gg_read_tr(const char *lds)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((address_space(3))) gg_i16x4 *at;
    return __builtin_bit_cast(gg_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)lds));
#else
    (void)lds;
    return gg_u32x2{0u, 0u};
#endif
}
__device__ __forceinline__ gg_f32x4 gg_mfma(lanes_u32x4 a, lanes_u32x4 b, gg_f32x4 c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(gg_bf16x8, a), __builtin_bit_cast(gg_bf16x8, b), c, 0, 0, 0);
#else
    (void)a; (void)b;
    return c;
#endif
}

// One operand of a workgroup's tile: R rows of the result's side, RED_OUTER as in the head comment.  DMA: whole units at 32-bit
// offsets, straight into LDS; else any address and row length, through registers.
template <int R, int THREADS, bool RED_OUTER, bool DMA, bool GATHER>
struct Operand {
    static constexpr int kAll = R * kStage / 8;                              // units of a stage
    static constexpr int kUnits = kAll / THREADS;                            // of a thread
    static constexpr int kRow = RED_OUTER ? R / 8 : kStage / 8;              // units of a row in LDS
    static constexpr int kBytes = kAll * 16;
    static_assert(kAll % THREADS == 0 && THREADS % kRow == 0, "whole units");
    static_assert(!RED_OUTER || R == 64 || R % 128 == 0, "the block permutation");

    static constexpr bool kIndexed = GATHER && RED_OUTER;        // the reduction's rows are read by index
    const char *base;                 // of the tile; GATHER: of the tensor (RED_OUTER: of the tile's columns in it)
    int64_t ld, bytes;                // from row to row; from base to the end of what may be read (RED_OUTER without GATHER: else offsets say it)
    int red, count;                   // length of the reduction; rows or columns of the tile that exist
    int length;                       // RED_OUTER: of a row in memory, columns of other tiles included
    const int32_t *rows;              // GATHER: of the tile's rows (innermost), of the reduction's (outermost)
    int src_rows;
    const int *index;                 // kIndexed: in LDS, entry k % kIndices is row k's, -1: none
    uint32_t off[DMA ? kUnits : 1];
    int32_t src[kIndexed ? kUnits : 1];                          // rows of the stage to be fetched
    const char *at[!DMA && !RED_OUTER ? kUnits : 1];             // of the unit's row, NULL: none
    lanes_u32x4 held[DMA ? 1 : kUnits];
    uint32_t wave_at;                 // DMA: where the wave's units lie in a stage
    // DMA: the descriptor of the stage to be fetched, kept from stage to stage: its base, what it may read from there on, and how far both
    // move a stage.  Reduction innermost and rows by index: lanes out of range are known by their offsets alone, and it may read on.
    uint64_t at_base;
    int64_t may_read;
    uint32_t stage_bytes;
    gg_i32x4 rsrc;

    // the permutation: of the blocks of 16 columns in reduction row kr, of the units of row r
    static __device__ __forceinline__ int spread(int kr)
    {
        return R == 64 ? ((kr >> 1) & 1) | ((kr >> 3) & 1) << 1 : (kr & 3) | ((kr >> 3) & 1) << 2;
    }
    static __device__ __forceinline__ int turn(int r) { return r & 7; }
    static __device__ __forceinline__ int lds_row(int tid, int i) { return tid / kRow + i * (THREADS / kRow); }
    // which unit of its row the thread's unit i holds
    static __device__ __forceinline__ int unit_of(int tid, int i)
    {
        const int r = lds_row(tid, i), u = tid % kRow;
        return RED_OUTER ? u ^ (spread(r) << 1) : u ^ turn(r);
    }

    __device__ __forceinline__ void init(int tid)
    {
        wave_at = (uint32_t)__builtin_amdgcn_readfirstlane(tid >> 6) * 1024u;
        at_base = wave_value((uint64_t)base);
        may_read = RED_OUTER && !GATHER ? (int64_t)wave_value((uint64_t)bytes) : (int64_t)kFarRecords;
        stage_bytes = !RED_OUTER ? kStage * 2 : GATHER ? 0u : (uint32_t)wave_value((int)((uint32_t)ld * kStage));
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int r = lds_row(tid, i), u = unit_of(tid, i);
            if constexpr (!RED_OUTER) {
                int from = r < count ? r : -1;
                if (GATHER && from >= 0) {
                    from = rows[r];
                    if ((unsigned)from >= (unsigned)src_rows) from = -1;
                }
                if constexpr (DMA) off[i] = from < 0 ? kFarOffset : (uint32_t)from * (uint32_t)ld + (uint32_t)u * 16u;
                else at[i] = from < 0 ? nullptr : base + from * ld;
            } else if constexpr (DMA) {
                off[i] = u * 8 < count ? (GATHER ? 0u : (uint32_t)r * (uint32_t)ld) + (uint32_t)u * 16u : kFarOffset;
            }
        }
    }
    // kIndexed: the indices of rows k0 .. k0 + kIndices - 1 of the reduction into LDS
    __device__ __forceinline__ void load_indices(int *to, int k0, int tid) const
    {
        for (int i = tid; i < kIndices && k0 + i < red; i += THREADS) {
            const int r = rows[k0 + i];
            to[i] = (unsigned)r < (unsigned)src_rows ? r : -1;
        }
    }

    // A stage is fetched in three steps: begin() once, unit() for each unit, commit() when registers held it; stage after stage.
    __device__ __forceinline__ void begin(int s, int tid)
    {
        const int k0 = s * kStage;
        if constexpr (DMA) {
            rsrc = gg_rsrc(at_base, may_read);
            at_base += stage_bytes;
            if (RED_OUTER && !GATHER) may_read -= (int64_t)stage_bytes;
            if constexpr (!RED_OUTER) {
                // the reduction's end, and stages past it: from here on these lanes have nothing to load
                if (k0 + kStage > red) {
#pragma unroll
                    for (int i = 0; i < kUnits; ++i)
                        if (k0 + unit_of(tid, i) * 8 >= red) off[i] = kFarOffset;
                }
            }
        }
        if constexpr (kIndexed) {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int k = k0 + lds_row(tid, i);
                src[i] = k < red ? index[k % kIndices] : -1;
            }
        }
    }
    __device__ __forceinline__ void unit(int s, int i, char *lds, int tid)
    {
        const int k0 = s * kStage;
        if constexpr (DMA) {
            uint32_t o = off[i];
            if constexpr (kIndexed) o = src[i] < 0 || o == kFarOffset ? kFarOffset : (uint32_t)src[i] * (uint32_t)ld + o;
            gg_dma(rsrc, gg_lds_offset(lds) + wave_at + (uint32_t)(i * THREADS) * 16u, o);
        } else {
            held[i] = lanes_u32x4{0u, 0u, 0u, 0u};
            const int u = unit_of(tid, i) * 8;
            if constexpr (!RED_OUTER) {
                if (at[i] && k0 + u < red) held[i] = load_unit8(reinterpret_cast<const uint16_t *>(at[i]) + k0 + u, red - k0 - u, red);
            } else {
                const int k = k0 + lds_row(tid, i), from = k < red && u < count ? (kIndexed ? src[i] : k) : -1;
                if (from >= 0) held[i] = load_unit8(reinterpret_cast<const uint16_t *>(base + from * ld) + u, count - u, length);
            }
        }
    }
    __device__ __forceinline__ void commit(char *lds, int tid)
    {
        if constexpr (!DMA) {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) *reinterpret_cast<lanes_u32x4 *>(lds + (i * THREADS + tid) * 16) = held[i];
        }
    }

    // What one instruction takes of rows r0 + 16 i .. r0 + 16 i + 15, half kk of the stage; r0 a multiple of 64.  Only i and kk are known to the
    // compiler, so what they add is kept out of the lane's part: it goes into the instruction.
    static __device__ __forceinline__ lanes_u32x4 operand(const char *lds, int r0, int i, int kk, int lane)
    {
        if constexpr (!RED_OUTER) {
            const char *at = lds + (r0 + (lane & 15)) * (kStage * 2) + (((lane >> 4) ^ turn(lane & 15)) * 16 ^ kk * 64);
            return *reinterpret_cast<const lanes_u32x4 *>(at + i * (16 * kStage * 2));
        } else {
            const int kr = (lane >> 4) * 8 + ((lane & 15) >> 2);
            const char *at = lds + kr * (R * 2) + ((r0 >> 4) + i ^ spread(kr)) * 32 + (lane & 3) * 8 + kk * (32 * R * 2);
            const gg_u32x2 lo = gg_read_tr(at), hi = gg_read_tr(at + 4 * R * 2);   // spread(kr + 4) == spread(kr + 32) == spread(kr) here
            return lanes_u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

// four floats at any of their addresses
typedef gg_f32x4 __attribute__((aligned(4))) Floats4;
// eight 16-bit values at any of theirs
typedef lanes_u32x4 __attribute__((aligned(2))) Halves8;

template <int FORM, int BM, int BN, int WM, int WN, int BUFFERS, bool DMA, bool GATHER, bool OUT_F32>
struct GroupedTile {
    static constexpr int kBuffers = BUFFERS;                                 // stages in LDS
    static constexpr int kThreads = (BM / WM) * (BN / WN) * 64;
    using A = Operand<BM, kThreads, FORM == GROUPED_DW, DMA, GATHER && FORM == GROUPED_FWD>;
    using B = Operand<BN, kThreads, FORM != GROUPED_FWD, DMA, GATHER && FORM == GROUPED_DW>;
    static constexpr int kStageBytes = A::kBytes + B::kBytes, kIndexBytes = B::kIndexed ? kIndices * 4 : 0;
    static constexpr bool kDma = DMA;
    // The workgroups of the forward product and of the gradient of the rows, whose tiles are alike, take tile after tile; those of the gradient of
    // the weights take one each, as the groups' lengths come, and their results leave through the stages' LDS.
    static constexpr bool kLoops = FORM != GROUPED_DW;
    static constexpr int kOutAt = kLoops ? kBuffers * kStageBytes : 0, kOutBytes = kThreads / 64 * 4096;
    static constexpr int kLds = kLoops ? kOutAt + kOutBytes : kBuffers * kStageBytes + kIndexBytes;
};

// What a finished tile leaves by: its rows and columns that exist, its first result, that of `h`.
struct GroupedOut { int rows, cols; int64_t c0, h0; };

// PAST: results go past the L2 (a choice at run time, between the stores, costs dX of 32768 x 2048 by 512 6 us of 74)
template <class T, int FORM, int BM, int BN, int WM, int WN, bool OUT_F32, bool PAST>
__global__ __launch_bounds__(T::kThreads) void grouped_kernel(GroupedArgs p)
{
    extern __shared__ __align__(1024) char grouped_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_value(tid >> 6);
    constexpr int kAcross = BN / WN, MI = WM / 16, NI = WN / 16;
    const int wm = wave / kAcross * WM, wn = wave % kAcross * WN;

    typename T::A A;
    typename T::B B;
    A.ld = p.lda;
    B.ld = p.ldb;
    A.src_rows = B.src_rows = p.src_rows;
    A.rows = B.rows = nullptr;
    A.length = p.out_rows;
    B.length = p.cols;
    GroupTiles tiles;
    if constexpr (FORM != GROUPED_DW) tiles.init(p.offsets, p.E, p.M, BM, p.col_tiles);

    // The operands and the result of tile `id`, and its stages; -1: there is no such tile.
    const auto find = [&](int id, GroupedOut &out) {
        if constexpr (FORM != GROUPED_DW) {
            GroupTile t;
            if (!tiles.find(id, &t)) return -1;
            const int m0 = t.lo + t.m * BM, n0 = t.n * BN, e = min(t.e, p.E - 1);
            out.rows = min(BM, t.hi - m0);
            out.cols = min(BN, p.cols - n0);
            const bool gathered = FORM == GROUPED_FWD && p.rows;
            A.rows = gathered ? p.rows + m0 : nullptr;
            A.base = gathered ? p.a : p.a + m0 * p.lda;
            if constexpr (FORM == GROUPED_FWD) {
                B.base = p.b + ((int64_t)e * p.cols + n0) * p.ldb;
            } else {
                B.base = p.b + (int64_t)e * p.red * p.ldb + (int64_t)n0 * 2;
                B.bytes = (int64_t)(p.red - 1) * p.ldb + (int64_t)out.cols * 2;
            }
            A.red = B.red = p.red;
            out.c0 = (int64_t)m0 * p.ldc + n0;
            out.h0 = (int64_t)m0 * p.ldh + n0;
            A.count = out.rows;
            B.count = out.cols;
            return t.e < p.E ? (p.red + kStage - 1) / kStage : 0;   // slots behind the last group: a result of zeros
        } else {
            // groups differ in length, so every die takes an eighth of each one's tiles, another eighth from group to group; long groups come in
            // the order of their lengths, the longest first (dW to bfloat16, groups' order / lengths' order: 16384 x 4096 x 2048 in 8 uneven groups 237 us /
            // 218, 32768 x 2048 x 2048 in 16 262 / 242; but 8192 x 1024 x 1024 in 32, where the order takes longer to find than it saves, 47 / 52)
            const int per = p.row_tiles * p.col_tiles, eighth = (per + 7) >> 3, at = id >> 3, turn = wave_value(at / eighth);
            const int in = (((id & 7) + (turn & 7)) & 7) * eighth + at - turn * eighth;
            if (in >= per || turn >= p.E) return -1;
            const int e = p.E <= kSorted && p.M >= 1024ll * p.E ? by_length(p.offsets, turn, p.E, p.M) : turn;
            const int m = wave_value(in / p.col_tiles), n = in - m * p.col_tiles;
            GroupRows g = group_rows(p.offsets, e, p.E, p.M);
            g.lo = wave_value(g.lo);
            g.hi = wave_value(g.hi);
            const int red = g.hi - g.lo;
            out.rows = min(BM, p.out_rows - m * BM);
            out.cols = min(BN, p.cols - n * BN);
            A.base = p.a + g.lo * p.lda + (int64_t)m * BM * 2;
            A.bytes = (int64_t)(red - 1) * p.lda + (int64_t)out.rows * 2;
            B.rows = p.rows ? p.rows + g.lo : nullptr;
            B.base = p.b + (p.rows ? 0 : g.lo * p.ldb) + (int64_t)n * BN * 2;
            B.bytes = (int64_t)(red - 1) * p.ldb + (int64_t)out.cols * 2;
            A.red = B.red = red;
            out.c0 = ((int64_t)e * p.out_rows + (int64_t)m * BM) * p.ldc + (int64_t)n * BN;
            out.h0 = 0;
            A.count = out.rows;
            B.count = out.cols;
            return (red + kStage - 1) / kStage;
        }
    };
    // Half a stage is in registers while the matrix cores work on the other half.  In the second half of stage s the first half of
    // s+1 is read, and a stage asked for into the buffer that s has left: every wave has its last values in registers.  It is waited
    // for kBuffers - 1 stages later.  (Stages of 32 in four buffers were slower where the reduction is innermost, for the memory
    // then gives half a cache line a row: 16384 x 2048 x 4160 forward 1074 against 1160 TFLOP/s.)
    constexpr int kLoads = T::A::kUnits + T::B::kUnits;
    int *const index = reinterpret_cast<int *>(grouped_lds + T::kBuffers * T::kStageBytes);
    constexpr int kBuffers = T::kBuffers;
    const auto buffer = [&](int s) { return grouped_lds + s % kBuffers * T::kStageBytes; };
    static_assert(kBuffers == 2 || kBuffers == 4, "buffer()");
    const auto load = [&](int s, int i) {
        if (i < T::A::kUnits) A.unit(s, i, buffer(s), tid);
        else B.unit(s, i - T::A::kUnits, buffer(s) + T::A::kBytes, tid);
    };
    const auto fetch = [&](int s) {
        A.begin(s, tid);
        B.begin(s, tid);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(s, i);
    };
    const auto commit = [&](int s) {
        A.commit(buffer(s), tid);
        B.commit(buffer(s) + T::A::kBytes, tid);
    };
    // waits until this wave's loads are down to those of BEHIND stages (DMA) or to none, then for the other waves
    const auto land = [&](auto behind) {
        constexpr int kBehind = T::kDma ? decltype(behind)::value : 0;
        // (the builtins say nothing of memory: without the statements around them the compiler may move reads and writes of LDS past the barrier)
        asm volatile("" ::: "memory");
        gg_wait<kBehind * kLoads>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // the n-th operand of a stage: the columns', then the rows'
    const auto read = [&](int s, int kk, int n, lanes_u32x4 (&a)[MI], lanes_u32x4 (&b)[NI]) {
        if (n < NI) b[n] = T::B::operand(buffer(s) + T::A::kBytes, wn, n, kk, lane);
        else a[n - NI] = T::A::operand(buffer(s), wm, n - NI, kk, lane);
    };
    gg_f32x4 acc[MI][NI];
    const auto step = [&](int s, auto half, auto busy, auto first, const lanes_u32x4 (&a)[MI], const lanes_u32x4 (&b)[NI], lanes_u32x4 (&a_next)[MI],
                          lanes_u32x4 (&b_next)[NI]) {
        constexpr bool kSecond = decltype(half)::value, kBusy = decltype(busy)::value;
        if constexpr (kSecond) {
            commit(s + 1);
            land(std::integral_constant<int, kBuffers - 2>{});      // stage s+1; and this wave has what it read of stage s
            if (T::B::kIndexed && (s + kBuffers) % (kIndices / kStage) == 0) {     // the next indices, rarely
                B.load_indices(index, (s + kBuffers) * kStage, tid);
                __syncthreads();
            }
        }
        // The reads of the next half and the loads go between the products: issued in one go, they hold the matrix cores up while the LDS
        // takes them in.  The loads come early, they have the longest way.
        constexpr int kReads = MI + NI, kReadRows = MI > 2 ? MI - 1 : MI, kLoadRows = (MI + 1) / 2;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            // columns as the instruction's rows: a lane then holds four neighbouring columns of one row of the result
#pragma unroll
            for (int j = 0; j < NI; ++j)
                if constexpr (kBusy) acc[i][j] = gg_mfma(b[j], a[i], decltype(first)::value ? gg_f32x4{0.f, 0.f, 0.f, 0.f} : acc[i][j]);
            if (kSecond && i == 0) {
                A.begin(s + kBuffers, tid);
                B.begin(s + kBuffers, tid);
            }
#pragma unroll
            for (int n = i * kReads / kReadRows; n < (i + 1) * kReads / kReadRows && n < kReads && kBusy; ++n) read(s + kSecond, !kSecond, n, a_next, b_next);
            if constexpr (kSecond) {
#pragma unroll
                for (int l = i * kLoads / kLoadRows; l < (i + 1) * kLoads / kLoadRows && l < kLoads; ++l) load(s + kBuffers, l);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Out through LDS, each wave through a part of its own: a lane then stores 16 bytes and the lanes of a row follow one another.
    // Straight from the registers rows went out in pieces of 32 bytes, and the activation's results came in two at a time
    // (dX of 16384 x 4096 x 2048 with ReLU: 476 us).
    constexpr int kUnit = OUT_F32 ? 4 : 8, kAcrossUnits = WN / kUnit;                   // values and units of a row
    constexpr int kRoom = T::kOutBytes / (T::kThreads / 64) / (kAcrossUnits * 16), kRows = kRoom < WM ? kRoom : WM;
    static_assert(kRows % 16 == 0 && WM % kRows == 0 && (kAcrossUnits & 3) == 0 && 64 % kAcrossUnits == 0, "whole tiles and rows");
    constexpr int kTwist = kAcrossUnits < 8 ? 3 : 7;                                    // neighbouring rows fall on other banks
    char *const mine = grouped_lds + T::kOutAt + wave * (kRows * kAcrossUnits * 16);
    // What the activation gave is asked for kAhead chunks of rows before it is needed, the first of them before the next tile's stages, where
    // the wave's part of the tile is whole.  (Asked for unit by unit as the results leave: dX of 16384 x 2048 x 4096 in 16 uneven groups with ReLU 313 us, so
    // 301; without the activation 272.)  What is left of the difference: the addresses are made of integers, so these loads and the stores are flat
    // ones, which may be to LDS as far as the compiler knows.  It waits for all that is under way, the next tile's stages among it, before
    // each unit that is masked, and before each tile's first reads of operands.
    constexpr int kChunks = WM / kRows, kPer = kRows * kAcrossUnits / 64, kWords = OUT_F32 ? 2 : 4;
    constexpr int kAhead = FORM != GROUPED_DX ? 1 : 32 / (kPer * kWords) < kChunks ? 32 / (kPer * kWords) : kChunks;
    // The activation is a pass of its own: decided value by value, it came out as selects, six instructions a value, that ran without one too.  (With the
    // first stage's zeros and one address a lane for whole tiles: forward 32768 x 4096 x 2048 in 16 groups 489 us -> 470.)  The maximum
    // lets NaN through, as the formula does.
    const auto activate = [&]() {
        if (FORM != GROUPED_FWD || p.act == POLYDL_ACT_NONE) return;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_elementwise_maximum(acc[i][j], gg_f32x4{0.f, 0.f, 0.f, 0.f});
        if (p.act != POLYDL_ACT_RELU6) return;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_elementwise_minimum(acc[i][j], gg_f32x4{6.f, 6.f, 6.f, 6.f});
    };
    // zeros where the activation did not let through what gave x
    const auto closed = [&](lanes_u32x4 v, lanes_u32x4 x) {
        const float limit = p.act == POLYDL_ACT_RELU6 ? 6.f : __builtin_nanf("");
#pragma unroll
        for (int q = 0; q < kUnit; ++q) {
            const float y = q & 1 ? bf16_hi(x[q >> 1]) : bf16_lo(x[q >> 1]);
            const bool open = y > 0.f && !(y >= limit);
            if constexpr (OUT_F32) v[q] = open ? v[q] : 0u;
            else v[q >> 1] &= open ? 0xffffffffu : q & 1 ? 0x0000ffffu : 0xffff0000u;
        }
        return v;
    };
    // go_on() starts the next tile
    const auto leave = [&](const GroupedOut &out, auto go_on) {
        // the compiler may not know that the lane is the same for every tile: it would keep all the addresses below in registers
        // through the products, and spill
        int lane = tid & 63;
        if constexpr (T::kLoops) asm volatile("" : "+v"(lane));
        // a wave's part that is whole: one address a lane, the rest of it the same for the wave
        const bool whole = wave_value((int)(out.rows >= wm + WM && out.cols >= wn + WN && p.ldc < (1 << 24) && p.ldh < (1 << 24)));
        const bool early = FORM == GROUPED_DX && p.act != POLYDL_ACT_NONE && whole;
        constexpr int kOutSize = OUT_F32 ? 4 : 2;
        const uint64_t c_base = wave_value((uint64_t)p.c + (uint64_t)(out.c0 + (int64_t)wm * p.ldc + wn) * kOutSize);
        const uint32_t c_off = (uint32_t)(lane / kAcrossUnits) * (uint32_t)(p.ldc * kOutSize) + (uint32_t)(lane % kAcrossUnits) * 16u;
        std::conditional_t<OUT_F32, gg_u32x2, lanes_u32x4> held_h[kAhead][kPer];
        const uint64_t h_base = wave_value((uint64_t)(p.h + out.h0 + (int64_t)wm * p.ldh + wn));
        const uint32_t h_off = (uint32_t)(lane / kAcrossUnits) * (uint32_t)(p.ldh * 2) + (uint32_t)(lane % kAcrossUnits * kUnit) * 2u;
        const auto ask_h = [&](int chunk) {
            if (FORM != GROUPED_DX || !early || chunk >= kChunks) return;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const uint64_t row = (uint64_t)(chunk * kRows + i * (64 / kAcrossUnits));
                const uint16_t *at = reinterpret_cast<const uint16_t *>(h_base + row * 2 * (uint64_t)p.ldh + h_off);
                if constexpr (OUT_F32) {
                    const Unit4 u = *reinterpret_cast<const Unit4 *>(at);
                    held_h[chunk % kAhead][i] = gg_u32x2{u.v[0], u.v[1]};
                } else {
                    held_h[chunk % kAhead][i] = load_unit8(at);
                }
            }
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ask_h(i);
        go_on();
        activate();
#pragma unroll
        for (int r0 = 0; r0 < WM; r0 += kRows) {
#pragma unroll
            for (int i = 0; i < kRows / 16; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    const gg_f32x4 v = acc[r0 / 16 + i][j];
                    const int r = i * 16 + (lane & 15), n = j * 16 + (lane >> 4) * 4;
                    char *at = mine + (r * kAcrossUnits + ((n / kUnit) ^ (r & kTwist))) * 16;
                    if constexpr (OUT_F32) *reinterpret_cast<gg_f32x4 *>(at) = v;
                    else *reinterpret_cast<gg_u32x2 *>(at + (n & 4) * 2) = gg_u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
                }
            if (whole) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    constexpr int kStep = 64 / kAcrossUnits;
                    const int r = i * kStep + lane / kAcrossUnits, u = lane % kAcrossUnits;
                    lanes_u32x4 v = *reinterpret_cast<const lanes_u32x4 *>(mine + (r * kAcrossUnits + (u ^ (r & kTwist))) * 16);
                    if (early) {
                        const auto x = held_h[r0 / kRows % kAhead][i];
                        if constexpr (OUT_F32) v = closed(v, lanes_u32x4{x[0], x[1], 0u, 0u});
                        else v = closed(v, x);
                    }
                    char *c = reinterpret_cast<char *>(c_base + (uint64_t)((r0 + i * kStep) * kOutSize) * (uint64_t)p.ldc + c_off);
                    if constexpr (OUT_F32) {
                        Floats4 *at = reinterpret_cast<Floats4 *>(c);
                        gg_f32x4 f = __builtin_bit_cast(gg_f32x4, v);
                        if (FORM == GROUPED_DW && p.accumulate) f += *at;
                        if constexpr (PAST) __builtin_nontemporal_store(f, at);
                        else *at = f;
                    } else {
                        Halves8 *at = reinterpret_cast<Halves8 *>(c);
                        if constexpr (PAST) __builtin_nontemporal_store(v, at);
                        else *at = v;
                    }
                }
                ask_h(r0 / kRows + kAhead);
                continue;
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = i * (64 / kAcrossUnits) + lane / kAcrossUnits, u = lane % kAcrossUnits;
                const int row = wm + r0 + r, n = wn + u * kUnit, left = out.cols - n;
                lanes_u32x4 v = *reinterpret_cast<const lanes_u32x4 *>(mine + (r * kAcrossUnits + (u ^ (r & kTwist))) * 16);
                if (row >= out.rows || left <= 0) continue;
                const int64_t at = out.c0 + (int64_t)row * p.ldc + n;
                if (FORM == GROUPED_DX && p.act != POLYDL_ACT_NONE) {
                    const uint16_t *h = p.h + out.h0 + (int64_t)row * p.ldh + n;
                    v = closed(v, kUnit == 8 || left < 4 ? load_unit8(h, min(left, kUnit), p.cols) : load_unit4(h));
                }
                if constexpr (OUT_F32) {
                    float *c = static_cast<float *>(p.c) + at;
                    gg_f32x4 f = __builtin_bit_cast(gg_f32x4, v);
                    if (left >= 4) {
                        if (FORM == GROUPED_DW && p.accumulate) f += *reinterpret_cast<const Floats4 *>(c);
                        *reinterpret_cast<Floats4 *>(c) = f;
                    } else {
#pragma unroll
                        for (int q = 0; q < 3; ++q)
                            if (q < left) c[q] = FORM == GROUPED_DW && p.accumulate ? c[q] + f[q] : f[q];
                    }
                } else {
                    uint16_t *c = static_cast<uint16_t *>(p.c) + at;
                    store_unit8(c, v, left);
                }
            }
        }
    };
    // asks for the first stages of the tile that find() has set up
    const auto start = [&]() {
        int tid = threadIdx.x;
        if constexpr (T::kLoops) asm volatile("" : "+v"(tid));       // as in leave()
        A.init(tid);
        B.init(tid);
        if constexpr (T::B::kIndexed) {
            B.index = index;
            B.load_indices(index, 0, tid);
            __syncthreads();
        }
        if constexpr (T::kDma) {
#pragma unroll
            for (int s = 0; s < kBuffers; ++s) fetch(s);   // stages past the last read as zeros, without memory
        } else {
            fetch(0);
            commit(0);
            fetch(1);
        }
    };

    int id = (int)block_number();
    GroupedOut now;
    int stages = find(id, now);
    if (stages < 0) return;
    if (stages > 0) start();
    while (true) {
        // A wave whose part of the tile does not exist takes part in the loads and leaves the matrix cores to the others (forward 32768 x 4096
        // x 2048 in 16 uneven groups: 515 us -> 499).  The first half of the forward product's first stage adds to zeros that are in
        // no register (the other forms' registers do not suffice for a first stage of its own: dW to bfloat16 239 us -> 251).
        constexpr bool kPeeled = FORM == GROUPED_FWD;
        const auto clear = [&]() {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = gg_f32x4{0.f, 0.f, 0.f, 0.f};
        };
        if constexpr (!kPeeled) clear();
        const bool busy = stages > 0 && wave_value((int)(wm < now.rows && wn < now.cols));
        if (stages > 0) land(std::integral_constant<int, kBuffers - 1>{});
        if (busy) {
            lanes_u32x4 a0[MI], b0[NI], a1[MI], b1[NI];
            constexpr std::true_type yes;
            constexpr std::false_type no;
#pragma unroll
            for (int n = 0; n < MI + NI; ++n) read(0, 0, n, a0, b0);
            if constexpr (kPeeled) {
                step(0, no, yes, yes, a0, b0, a1, b1);
                step(0, yes, yes, no, a1, b1, a0, b0);
            }
            for (int s = kPeeled ? 1 : 0; s < stages; ++s) {
                step(s, no, yes, no, a0, b0, a1, b1);
                step(s, yes, yes, no, a1, b1, a0, b0);
            }
        } else {
            if constexpr (kPeeled) clear();
            lanes_u32x4 a[MI], b[NI];
            for (int s = 0; s < stages; ++s) step(s, std::true_type{}, std::false_type{}, std::false_type{}, a, b, a, b);
        }
        if (stages > 0) {
            land(std::integral_constant<int, 0>{});        // no wave reads the stages any more, no load is under way
        }
        if constexpr (!T::kLoops) {
            leave(now, [] {});
            return;
        } else {
            // the next tile's first stages are asked for before this one's results leave
            GroupedOut next;
            leave(now, [&] {
                id += (int)gridDim.x;
                stages = find(id, next);
                if (stages > 0) start();
            });
            if (stages < 0) return;
            now = next;
        }
    }
}

template <int FORM, int BM, int BN, int WM, int WN, int BUFFERS, bool DMA, bool GATHER, bool OUT_F32, bool PAST>
static hipError_t grouped_launch(const GroupedProblem &q, hipStream_t st)
{
    using T = GroupedTile<FORM, BM, BN, WM, WN, BUFFERS, DMA, GATHER, OUT_F32>;
    constexpr auto kernel = grouped_kernel<T, FORM, BM, BN, WM, WN, OUT_F32, PAST>;
    GroupedArgs a{q.E, q.M, q.out_rows, q.cols, q.red, q.offsets, q.rows, q.src_rows, reinterpret_cast<const char *>(q.a),
                  reinterpret_cast<const char *>(q.b), q.lda * 2, q.ldb * 2, q.c, q.ldc, q.accumulate, q.act, q.h, q.ldh, 0, 0};
    a.col_tiles = (q.cols + BN - 1) / BN;
    int64_t tiles;
    if (FORM == GROUPED_DW) {
        a.row_tiles = (q.out_rows + BM - 1) / BM;
        tiles = ((int64_t)a.row_tiles * a.col_tiles + 7) / 8 * 8 * q.E;
    } else {
        // each group, and the slots behind the last, may end in a partial tile
        const int64_t groups = q.M < q.E + 1 ? q.M : q.E + 1;
        tiles = (q.M + groups * (BM - 1)) / BM * a.col_tiles;
    }
    if (tiles > kMaxBlocks) return hipErrorInvalidValue;       // (a tile's number plus the workgroups is an int too)
    if (T::kLoops) {
        const int64_t fit = (int64_t)compute_units() * (160 * 1024 / T::kLds);
        if (tiles > fit) tiles = fit;
    }
    if (T::kLds > 64 * 1024) {
        const hipError_t e = ask_lds<kernel>(T::kLds);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(kernel, many_blocks(tiles, T::kThreads), dim3(T::kThreads), T::kLds, st, a);
}

template <int FORM, int BM, int BN, int WM, int WN, int BUFFERS, bool DMA, bool GATHER, bool OUT_F32>
static hipError_t grouped_run(const GroupedProblem &q, hipStream_t st)
{
    // Results that no cache would hold until they are read go past the L2, which keeps the operands: gradients of weights, and what would fill the 256 MB
    // of the last level.  dW of 16384 x 4096 x 2048 in 8 groups, to float32 265 us -> 246, to bfloat16 264 -> 242; forward 32768 x 4096 (268 MB) with
    // reductions of 512, 189 -> 170, of 1024, 280 -> 241, of 2048, no difference; but dX of 32768 x 2048 (134 MB) by 512 71 -> 76.
    const bool past = FORM == GROUPED_DW || (int64_t)q.M * q.cols * (OUT_F32 ? 4 : 2) > 192ll << 20;
    if constexpr (FORM == GROUPED_DW || BM == 256)
        if (past) return grouped_launch<FORM, BM, BN, WM, WN, BUFFERS, DMA, GATHER, OUT_F32, true>(q, st);
    if constexpr (FORM != GROUPED_DW) return grouped_launch<FORM, BM, BN, WM, WN, BUFFERS, DMA, GATHER, OUT_F32, false>(q, st);
    return hipErrorInvalidValue;        // not reached
}

template <int FORM, int BM, int BN, int WM, int WN, int BUFFERS, bool DMA>
static hipError_t grouped_pick_types(const GroupedProblem &q, hipStream_t st)
{
    if constexpr (FORM == GROUPED_DX)
        return q.out_f32 ? grouped_run<FORM, BM, BN, WM, WN, BUFFERS, DMA, false, true>(q, st) : grouped_run<FORM, BM, BN, WM, WN, BUFFERS, DMA, false, false>(q, st);
    else if (q.rows)
        return q.out_f32 ? grouped_run<FORM, BM, BN, WM, WN, BUFFERS, DMA, true, true>(q, st) : grouped_run<FORM, BM, BN, WM, WN, BUFFERS, DMA, true, false>(q, st);
    else
        return q.out_f32 ? grouped_run<FORM, BM, BN, WM, WN, BUFFERS, DMA, false, true>(q, st) : grouped_run<FORM, BM, BN, WM, WN, BUFFERS, DMA, false, false>(q, st);
}

// Whether both operands can go into LDS in whole units at 32-bit offsets: 16-byte rows, and offsets inside a tile (rows by
// index: inside the tensor) below 2^32.
static bool grouped_whole_units(const GroupedProblem &q, int bm, int bn)
{
    const int64_t last = 0xf0000000ll;
    if ((((uintptr_t)q.a | (uintptr_t)q.b) & 15) || (q.lda | q.ldb | q.cols) % 8) return false;
    if (q.form == GROUPED_FWD) {
        return q.red % 8 == 0 && (q.rows ? (int64_t)q.src_rows : (int64_t)bm) * q.lda * 2 < last && (int64_t)bn * q.ldb * 2 < last;
    }
    if (q.form == GROUPED_DX) return q.red % 8 == 0 && bm * q.lda * 2 < last && kStage * q.ldb * 2 < last;
    return q.out_rows % 8 == 0 && kStage * q.lda * 2 < last && (q.rows ? (int64_t)q.src_rows : (int64_t)kStage) * q.ldb * 2 < last;
}

// Rounds of `at_a_time` workgroups that tiles of `tile` squared take, groups of the mean length taken to end in half a tile each.
template <int FORM>
static int64_t grouped_rounds(const GroupedProblem &q, int64_t tile, int64_t at_a_time)
{
    const int64_t across = (q.cols + tile - 1) / tile;
    const int64_t down = FORM == GROUPED_DW ? (q.out_rows + tile - 1) / tile * q.E
                         : q.E == 1         ? (q.M + tile - 1) / tile
                                            : (q.M + q.E * (tile / 2) + tile - 1) / tile;
    return (across * down + at_a_time - 1) / at_a_time;
}

// Tiles of 256 (one workgroup on a compute unit), of 128 (two) or of 64 (two, with four stages in LDS; operands that go through registers: three,
// with two).  What is left of the last round decides: a round of 128 takes 0.65 of a round of 256 and does half the work (4096 x 4096 x
// 4096: 117 us in one round of 256, 155 in two of 128); one of 64 takes half a round of 128, for a quarter of the work, and where 64 fits one
// round it is the stages' latency that counts, of which it has more under way.  Measured both ways, forward, us:
//   256 / 128: 16 groups of 256 rows, 2048 x 2048, 66 / 80; of 400, 99 / 95; of 1024, 176 / 200; one of 4096, 57 / 42;
//   64 / 128: one group of 1024 rows, 1024 x 1024, 11 / 18; 32 of 64, 512 x 512, 10 / 13; 16 of 256, 1024 x 1024, 30 / 23;
//   through registers, 64 / 128: 7 of 143 rows, 777 x 531, 13 / 20; 8 of 256, 1001 x 777, 21 / 27; 8 of 2048, 2047 x 2047, 424 / 305.
// Up to 128 rows a group tiles of 256 are mostly empty (16 groups of 128: 62 / 52).  Weight gradients of few tiles a group need smaller ones
// to even the groups out (64 groups of 512 rows, 512 x 512: 74 / 55; 8 of 1024 rows, 1024 x 2048: 51 / 56).
template <int FORM>
static hipError_t grouped_pick(const GroupedProblem &q, hipStream_t st)
{
    const int64_t cus = compute_units();
    const double of128 = (double)grouped_rounds<FORM>(q, 128, 2 * cus);
    if (!grouped_whole_units(q, 256, 256)) {
        if (0.5 * (double)grouped_rounds<FORM>(q, 64, 3 * cus) <= of128) return grouped_pick_types<FORM, 64, 64, 32, 32, 2, false>(q, st);
        return grouped_pick_types<FORM, 128, 128, 64, 64, 2, false>(q, st);
    }
    const bool empty = FORM == GROUPED_DW ? ((int64_t)q.out_rows + 255) / 256 * ((q.cols + 255) / 256) < 8 : q.M <= 128 * (int64_t)q.E;
    if (!empty && (double)grouped_rounds<FORM>(q, 256, cus) <= 0.65 * of128) return grouped_pick_types<FORM, 256, 256, 128, 64, 2, true>(q, st);
    if (0.55 * (double)grouped_rounds<FORM>(q, 64, 2 * cus) <= of128) return grouped_pick_types<FORM, 64, 64, 32, 32, 4, true>(q, st);
    return grouped_pick_types<FORM, 128, 128, 64, 64, 2, true>(q, st);
}

hipError_t grouped_gemm_launch(const GroupedProblem &q, hipStream_t st)
{
    // up to 16 rows a group in the mean (8 groups of 4096 x 4096, few rows / tiles of 128: 20 rows 75 / 81 us, 32 rows 94 / 81)
    if (q.form == GROUPED_FWD && q.M <= 16 * (int64_t)q.E) {
        const FewRowsProblem f{q.E, q.M, q.cols, q.red, 0, q.offsets, q.rows, q.src_rows, q.a, q.lda, q.b, nullptr, nullptr, nullptr, q.c, q.ldc,
                               q.out_f32, q.act};
        return few_rows_launch(f, st);
    }
    return q.form == GROUPED_FWD ? grouped_pick<GROUPED_FWD>(q, st)
           : q.form == GROUPED_DX ? grouped_pick<GROUPED_DX>(q, st)
                                  : grouped_pick<GROUPED_DW>(q, st);
}

}  // namespace polydl
