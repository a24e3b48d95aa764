// Matrix products grouped by expert, bfloat16 operands, float32 sums: the forward product of the rows of each group with
// the group's weights, and the gradients of the rows and of the weights.
//
// One kernel in three forms.  A workgroup owns a tile BM x BN of one group's result and walks the reduction in stages of 64,
// two stage buffers in LDS; a wave keeps a tile WM x WN in registers as 16x16 results of v_mfma_f32_16x16x32_bf16.
// An operand lies in LDS as it lies in memory, in units of eight values (16 bytes):
//   * reduction innermost (both operands of the forward product, the rows of the gradient of the rows): [row][64]; a lane
//     reads the eight values of its row that one instruction takes.  The unit c of a row is stored in place c ^ (row & 7), so
//     that the lanes of one read fall on different banks.
//   * reduction outermost (weights in the gradient of the rows, both operands in that of the weights): [64][columns]; the
//     transposing LDS read gives a lane four values of its column from four rows.  Blocks of 16 columns are stored in the
//     block's place ^ a number of the row that differs for the eight rows that half a wave reads at a time.
// Loads go from memory into LDS without registers; the permutation is applied to the address a lane loads from.  Lanes past an
// edge use an offset out of the descriptor's range, which reads as zero: rows that the plan does not have, columns past the
// last, the reduction's tail.  The kernel reads the group of its tile from the offsets in device memory, so nothing waits for
// the host.
#include <hip/hip_runtime.h>
#include <atomic>
#include "experts.hpp"
#include "gemm_core.hpp"
#include "group_tiles.hpp"
#include "internal.hpp"

namespace polydl {

typedef __bf16 gg_bf16x8 __attribute__((ext_vector_type(8)));
typedef float gg_f32x4 __attribute__((ext_vector_type(4)));
typedef short gg_i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void *gg_lds_t;
typedef uint32_t gg_u32x2 __attribute__((ext_vector_type(2)));

constexpr int kStage = 64;                          // reduction of a stage
constexpr uint32_t kFarOffset = 0xfffffff0u;        // out of range of every descriptor here
constexpr uint64_t kFarRecords = 0xffffffe0ull;     // so that no sum of an offset in range and a load's width reaches 2^32

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

__device__ __forceinline__ __amdgpu_buffer_rsrc_t gg_rsrc(const char *base, int64_t bytes)
{
    const uint64_t n = bytes < 0 ? 0 : (uint64_t)bytes > kFarRecords ? kFarRecords : (uint64_t)bytes;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), (short)0, (int)(uint32_t)n, 0x00020000);
}
__device__ __forceinline__ void gg_dma(__amdgpu_buffer_rsrc_t r, void *lds, uint32_t off)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (gg_lds_t)lds, 16, (int)off, 0, 0, 0);
#else
    (void)r; (void)lds; (void)off;
#endif
}
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
    static constexpr int kUnits = kAll < THREADS ? 1 : kAll / THREADS;       // of a thread
    static constexpr int kRow = RED_OUTER ? R / 8 : kStage / 8;              // units of a row in LDS
    static constexpr int kBytes = kAll * 16;
    static_assert((kAll % THREADS == 0 || kAll < THREADS) && THREADS % kRow == 0 && kAll % 64 == 0, "whole units, whole waves");
    static_assert(!RED_OUTER || R == 64 || R % 128 == 0, "the block permutation");

    const char *base;                 // of the tile; GATHER: of the tensor (RED_OUTER: of the tile's columns in it)
    int64_t ld, bytes;                // from row to row; from base to the end of what may be read
    int red, count;                   // length of the reduction; rows or columns of the tile that exist
    const int32_t *rows;              // GATHER: of the tile's rows (innermost), of the reduction's (outermost)
    int src_rows;
    uint32_t off[DMA ? kUnits : 1];
    int32_t next[DMA && GATHER && RED_OUTER ? kUnits : 1];       // rows of the next stage
    const char *at[!DMA && !RED_OUTER ? kUnits : 1];             // of the unit's row, NULL: none
    lanes_u32x4 held[DMA ? 1 : kUnits];

    // the permutation: of the blocks of 16 columns in reduction row kr
    static __device__ __forceinline__ int spread(int kr)
    {
        return R == 64 ? ((kr >> 1) & 1) | ((kr >> 3) & 1) << 1 : (kr & 3) | ((kr >> 3) & 1) << 2;
    }
    static __device__ __forceinline__ bool mine(int tid) { return kAll >= THREADS || tid < kAll; }
    static __device__ __forceinline__ int lds_row(int tid, int i) { return tid / kRow + i * (THREADS / kRow); }
    // which unit of its row the thread's unit i holds
    static __device__ __forceinline__ int unit_of(int tid, int i)
    {
        const int r = lds_row(tid, i), u = tid % kRow;
        return RED_OUTER ? u ^ (spread(r) << 1) : u ^ (r & 7);
    }
    __device__ __forceinline__ int row_index(int r) const
    {
        if (!GATHER) return r;
        const int s = rows[r];
        return (unsigned)s < (unsigned)src_rows ? s : -1;
    }

    __device__ __forceinline__ void init(int tid)
    {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int r = lds_row(tid, i), u = unit_of(tid, i);
            if constexpr (!RED_OUTER) {
                const int src = r < count ? row_index(r) : -1;
                if constexpr (DMA) off[i] = src < 0 ? kFarOffset : (uint32_t)src * (uint32_t)ld + (uint32_t)u * 16u;
                else at[i] = src < 0 ? nullptr : base + src * ld;
            } else if constexpr (DMA) {
                off[i] = u * 8 < count ? (GATHER ? 0u : (uint32_t)r * (uint32_t)ld) + (uint32_t)u * 16u : kFarOffset;
                if constexpr (GATHER) next[i] = r < red ? row_index(r) : -1;
            }
        }
    }

    // Stage s: asked for into `lds` (DMA), or into registers.
    __device__ __forceinline__ void fetch(int s, char *lds, int tid)
    {
        if (!mine(tid)) return;
        const int k0 = s * kStage;
        if constexpr (DMA) {
            const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
            const int64_t skip = RED_OUTER ? (GATHER ? 0 : (int64_t)k0 * ld) : (int64_t)k0 * 2;
            const __amdgpu_buffer_rsrc_t r = gg_rsrc(base + skip, bytes - skip);
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                uint32_t o = off[i];
                if constexpr (!RED_OUTER) {
                    if (k0 + unit_of(tid, i) * 8 >= red) o = kFarOffset;
                } else if constexpr (GATHER) {
                    o = next[i] < 0 || o == kFarOffset ? kFarOffset : (uint32_t)next[i] * (uint32_t)ld + o;
                    const int k = k0 + kStage + lds_row(tid, i);
                    next[i] = k < red ? row_index(k) : -1;
                }
                gg_dma(r, lds + (i * THREADS + wave * 64) * 16, o);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                held[i] = lanes_u32x4{0u, 0u, 0u, 0u};
                const int u = unit_of(tid, i) * 8;
                if constexpr (!RED_OUTER) {
                    if (at[i] && k0 + u < red) held[i] = load_unit8(reinterpret_cast<const uint16_t *>(at[i]) + k0 + u, red - k0 - u);
                } else {
                    const int k = k0 + lds_row(tid, i);
                    const int src = k < red && u < count ? row_index(k) : -1;
                    if (src >= 0) held[i] = load_unit8(reinterpret_cast<const uint16_t *>(base + src * ld) + u, count - u);
                }
            }
        }
    }
    __device__ __forceinline__ void commit(char *lds, int tid)
    {
        if constexpr (!DMA) {
            if (!mine(tid)) return;
#pragma unroll
            for (int i = 0; i < kUnits; ++i) *reinterpret_cast<lanes_u32x4 *>(lds + (i * THREADS + tid) * 16) = held[i];
        }
    }

    // What one instruction takes of rows r0 .. r0+15, values kk*32 .. kk*32+31 of the stage.
    static __device__ __forceinline__ lanes_u32x4 operand(const char *lds, int r0, int kk, int lane)
    {
        if constexpr (!RED_OUTER) {
            const int r = r0 + (lane & 15);
            return *reinterpret_cast<const lanes_u32x4 *>(lds + r * (kStage * 2) + (((kk * 4 + (lane >> 4)) ^ (lane & 7)) * 16));
        } else {
            const int kr = kk * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2);
            const char *at = lds + kr * (R * 2) + ((r0 >> 4) ^ spread(kr)) * 32 + (lane & 3) * 8;
            const gg_u32x2 lo = gg_read_tr(at), hi = gg_read_tr(at + 4 * R * 2);   // spread(kr + 4) == spread(kr) here
            return lanes_u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

template <int FORM, int BM, int BN, int WM, int WN, bool DMA, bool GATHER, bool OUT_F32>
struct GroupedTile {
    static constexpr int kThreads = (BM / WM) * (BN / WN) * 64;
    using A = Operand<BM, kThreads, FORM == GROUPED_DW, DMA, GATHER && FORM == GROUPED_FWD>;
    using B = Operand<BN, kThreads, FORM != GROUPED_FWD, DMA, GATHER && FORM == GROUPED_DW>;
    static constexpr int kStageBytes = A::kBytes + B::kBytes, kLds = 2 * kStageBytes;
};

template <class T, int FORM, int BM, int BN, int WM, int WN, bool OUT_F32>
__global__ __launch_bounds__(T::kThreads) void grouped_kernel(GroupedArgs p)
{
    extern __shared__ __align__(1024) char grouped_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kAcross = BN / WN, MI = WM / 16, NI = WN / 16;
    const int wm = wave / kAcross * WM, wn = wave % kAcross * WN;

    typename T::A A;
    typename T::B B;
    int rows, cols, stages;            // of the tile that exist
    int64_t c0;                        // its first result
    int64_t h0 = 0;
    if constexpr (FORM != GROUPED_DW) {
        GroupTile t;
        if (!find_tile(p.offsets, p.E, p.M, BM, p.col_tiles, (int)blockIdx.x, &t)) return;
        const int m0 = t.lo + t.m * BM, n0 = t.n * BN;
        rows = min(BM, t.hi - m0);
        cols = min(BN, p.cols - n0);
        stages = t.e < p.E ? (p.red + kStage - 1) / kStage : 0;   // slots behind the last group: a result of zeros
        const int e = min(t.e, p.E - 1);
        A.rows = p.rows ? p.rows + m0 : nullptr;
        A.base = FORM == GROUPED_FWD && A.rows ? p.a : p.a + m0 * p.lda;
        A.bytes = (int64_t)(FORM == GROUPED_FWD && A.rows ? p.src_rows - 1 : rows - 1) * p.lda + (int64_t)p.red * 2;
        A.red = p.red;
        A.count = rows;
        if constexpr (FORM == GROUPED_FWD) {
            B.base = p.b + ((int64_t)e * p.cols + n0) * p.ldb;
            B.bytes = (int64_t)(cols - 1) * p.ldb + (int64_t)p.red * 2;
        } else {
            B.base = p.b + (int64_t)e * p.red * p.ldb + (int64_t)n0 * 2;
            B.bytes = (int64_t)(p.red - 1) * p.ldb + (int64_t)cols * 2;
        }
        B.red = p.red;
        c0 = (int64_t)m0 * p.ldc + n0;
        h0 = (int64_t)m0 * p.ldh + n0;
    } else {
        const int per = p.row_tiles * p.col_tiles, id = die_order((int)blockIdx.x, (int)gridDim.x), e = id / per;
        const int m = (id - e * per) / p.col_tiles, n = id - e * per - m * p.col_tiles;
        const GroupRows g = group_rows(p.offsets, e, p.E, p.M);
        rows = min(BM, p.out_rows - m * BM);
        cols = min(BN, p.cols - n * BN);
        const int red = g.hi - g.lo;
        stages = (red + kStage - 1) / kStage;
        A.rows = nullptr;
        A.base = p.a + g.lo * p.lda + (int64_t)m * BM * 2;
        A.bytes = (int64_t)(red - 1) * p.lda + (int64_t)rows * 2;
        A.red = red;
        A.count = rows;
        B.rows = p.rows ? p.rows + g.lo : nullptr;
        B.base = p.b + (p.rows ? 0 : g.lo * p.ldb) + (int64_t)n * BN * 2;
        B.bytes = (int64_t)((p.rows ? p.src_rows : red) - 1) * p.ldb + (int64_t)cols * 2;
        B.red = red;
        c0 = ((int64_t)e * p.out_rows + (int64_t)m * BM) * p.ldc + (int64_t)n * BN;
    }
    A.ld = p.lda;
    B.ld = p.ldb;
    B.count = cols;
    A.src_rows = B.src_rows = p.src_rows;
    if constexpr (FORM != GROUPED_DW) B.rows = nullptr;

    gg_f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = gg_f32x4{0.f, 0.f, 0.f, 0.f};

    if (stages > 0) {
        A.init(tid);
        B.init(tid);
        A.fetch(0, grouped_lds, tid);
        B.fetch(0, grouped_lds + T::A::kBytes, tid);
        A.commit(grouped_lds, tid);
        B.commit(grouped_lds + T::A::kBytes, tid);
        wait_vmcnt0();
        __syncthreads();
        for (int s = 0; s < stages; ++s) {
            char *now = grouped_lds + (s & 1) * T::kStageBytes, *then = grouped_lds + ((s & 1) ^ 1) * T::kStageBytes;
            if (s + 1 < stages) {
                A.fetch(s + 1, then, tid);
                B.fetch(s + 1, then + T::A::kBytes, tid);
            }
#pragma unroll
            for (int kk = 0; kk < kStage / 32; ++kk) {
                lanes_u32x4 a[MI], b[NI];
#pragma unroll
                for (int j = 0; j < NI; ++j) b[j] = T::B::operand(now + T::A::kBytes, wn + j * 16, kk, lane);
#pragma unroll
                for (int i = 0; i < MI; ++i) a[i] = T::A::operand(now, wm + i * 16, kk, lane);
                // columns as the instruction's rows: a lane then holds four neighbouring columns of one row of the result
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = gg_mfma(b[j], a[i], acc[i][j]);
            }
            if (s + 1 < stages) {
                A.commit(then, tid);
                B.commit(then + T::A::kBytes, tid);
            }
            wait_vmcnt0();
            __syncthreads();
        }
    }

    const bool whole = (p.ldc & 3) == 0 && ((uintptr_t)p.c & 15) == 0;       // four results at a time
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int r = wm + i * 16 + (lane & 15);
        if (r >= rows) continue;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = wn + j * 16 + (lane >> 4) * 4, left = cols - n;
            if (left <= 0) continue;
            gg_f32x4 v = acc[i][j];
            if constexpr (FORM == GROUPED_FWD) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    // comparisons that let NaN through, as the formula does
                    if (p.act != POLYDL_ACT_NONE) v[q] = v[q] < 0.f ? 0.f : v[q];
                    if (p.act == POLYDL_ACT_RELU6) v[q] = v[q] > 6.f ? 6.f : v[q];
                }
            }
            if constexpr (FORM == GROUPED_DX) {
                if (p.act != POLYDL_ACT_NONE) {
                    const uint16_t *h = p.h + h0 + (int64_t)r * p.ldh + n;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float x = q < left ? bf16_lo(h[q]) : 0.f;
                        const bool open = x > 0.f && (p.act == POLYDL_ACT_RELU || x < 6.f);
                        v[q] = open ? v[q] : 0.f;
                    }
                }
            }
            const int64_t at = c0 + (int64_t)r * p.ldc + n;
            if constexpr (OUT_F32) {
                float *c = static_cast<float *>(p.c) + at;
                if (whole && left >= 4) {
                    if (p.accumulate) v += *reinterpret_cast<gg_f32x4 *>(c);
                    *reinterpret_cast<gg_f32x4 *>(c) = v;
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q < left) c[q] = p.accumulate ? c[q] + v[q] : v[q];
                }
            } else {
                uint16_t *c = static_cast<uint16_t *>(p.c) + at;
                if (whole && left >= 4) {
                    *reinterpret_cast<gg_u32x2 *>(c) = gg_u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q < left) c[q] = bf16_one(v[q]);
                }
            }
        }
    }
}

// More LDS than the default window has to be asked for, once per kernel and device.
template <auto KERNEL>
static hipError_t ask_lds(int bytes)
{
    static std::atomic<uint64_t> asked{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (asked.load(std::memory_order_relaxed) & bit) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) asked.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <int FORM, int BM, int BN, int WM, int WN, bool DMA, bool GATHER, bool OUT_F32>
static hipError_t grouped_run(const GroupedProblem &q, hipStream_t st)
{
    using T = GroupedTile<FORM, BM, BN, WM, WN, DMA, GATHER, OUT_F32>;
    constexpr auto kernel = grouped_kernel<T, FORM, BM, BN, WM, WN, OUT_F32>;
    GroupedArgs a{q.E, q.M, q.out_rows, q.cols, q.red, q.offsets, q.rows, q.src_rows, reinterpret_cast<const char *>(q.a),
                  reinterpret_cast<const char *>(q.b), q.lda * 2, q.ldb * 2, q.c, q.ldc, q.accumulate, q.act, q.h, q.ldh, 0, 0};
    a.col_tiles = (q.cols + BN - 1) / BN;
    int64_t tiles;
    if (FORM == GROUPED_DW) {
        a.row_tiles = (q.out_rows + BM - 1) / BM;
        tiles = (int64_t)q.E * a.row_tiles * a.col_tiles;
    } else {
        // each group, and the slots behind the last, may end in a partial tile
        const int64_t groups = q.M < q.E + 1 ? q.M : q.E + 1;
        tiles = (q.M + groups * (BM - 1)) / BM * a.col_tiles;
    }
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;
    if (T::kLds > 64 * 1024) {
        const hipError_t e = ask_lds<kernel>(T::kLds);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(kernel, dim3((unsigned)tiles), dim3(T::kThreads), T::kLds, st, a);
}

template <int FORM, int BM, int BN, int WM, int WN, bool DMA>
static hipError_t grouped_pick_types(const GroupedProblem &q, hipStream_t st)
{
    if constexpr (FORM == GROUPED_DX)
        return q.out_f32 ? grouped_run<FORM, BM, BN, WM, WN, DMA, false, true>(q, st) : grouped_run<FORM, BM, BN, WM, WN, DMA, false, false>(q, st);
    else if (q.rows)
        return q.out_f32 ? grouped_run<FORM, BM, BN, WM, WN, DMA, true, true>(q, st) : grouped_run<FORM, BM, BN, WM, WN, DMA, true, false>(q, st);
    else
        return q.out_f32 ? grouped_run<FORM, BM, BN, WM, WN, DMA, false, true>(q, st) : grouped_run<FORM, BM, BN, WM, WN, DMA, false, false>(q, st);
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

template <int FORM>
static hipError_t grouped_pick(const GroupedProblem &q, hipStream_t st)
{
    if (!grouped_whole_units(q, 256, 256)) return grouped_pick_types<FORM, 128, 128, 64, 64, false>(q, st);
    const int64_t rows = FORM == GROUPED_DW ? q.out_rows : q.M / q.E;    // of a group, in the mean
    if (rows > 128) return grouped_pick_types<FORM, 256, 256, 128, 64, true>(q, st);
    return grouped_pick_types<FORM, 128, 128, 64, 64, true>(q, st);
}

hipError_t grouped_gemm_launch(const GroupedProblem &q, hipStream_t st)
{
    return q.form == GROUPED_FWD ? grouped_pick<GROUPED_FWD>(q, st)
           : q.form == GROUPED_DX ? grouped_pick<GROUPED_DX>(q, st)
                                  : grouped_pick<GROUPED_DW>(q, st);
}

}  // namespace polydl
