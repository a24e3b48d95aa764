// The norm of many tensors taken as one vector, and their scaling to a largest norm.
//
// The tensors lie along one axis of chunks of kChunk values, none of which goes past a tensor's end; a launch takes the tensors that its arguments
// have room for, so that no table has to reach the device first (a captured launch keeps it, too).  First the squares, added up in 64 bits by each
// thread and workgroup; then the sum over the workgroups, the norm and the factor, by one workgroup; then the scaling.
// Bound: HBM, every value read twice and written once; the 64-bit sums cost two instructions a value.
#include <hip/hip_runtime.h>
#include <math.h>
#include <type_traits>
#include "block.hpp"
#include "blocks.hpp"
#include "internal.hpp"
#include "lanes.hpp"
#include "values.hpp"

namespace polydl {

constexpr int kClipTensors = 120;       // of a launch: its arguments stay within 4 KB
constexpr int kClipThreads = 256, kChunk = 8192;
constexpr int kClipBlocks = 2048;       // of a launch, at most

struct ClipTable {
    const void *grad[kClipTensors];
    void *out[kClipTensors];
    int64_t count[kClipTensors];
    int32_t first[kClipTensors + 1];    // chunk that tensor i begins with
    uint32_t f32[(kClipTensors + 31) / 32];
    int n;
};
static_assert(sizeof(ClipTable) <= 4000, "kernel arguments");

// a chunk: which tensor, where it begins in it, and its length
struct ClipChunk { int tensor; bool f32; int64_t at; int length; };
__device__ __forceinline__ ClipChunk clip_chunk(const ClipTable &t, int chunk)
{
    int lo = 0, hi = t.n;               // first[lo] <= chunk < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    const int64_t at = (int64_t)(chunk - t.first[lo]) * kChunk, left = t.count[lo] - at;
    return {lo, (t.f32[lo >> 5] >> (lo & 31) & 1u) != 0u, at, (int)(left < kChunk ? left : kChunk)};
}

// A chunk's values, 16 bytes a load, the lanes of a wave side by side (eight floats a lane, in two loads 32 bytes apart: 134 M floats, squares 126 us).
// use(values, n of them, where they begin in the chunk)
template <bool F32, class USE>
__device__ __forceinline__ void clip_each(const void *grad, const ClipChunk &k, USE use)
{
    constexpr int kWide = F32 ? 4 : 8, kUnits = kChunk / (kClipThreads * kWide);
    const auto *v = static_cast<const typename Values<F32>::T *>(grad) + k.at;
    if (k.length == kChunk) {
        lanes_u32x4 raw[kUnits];
#pragma unroll
        for (int i = 0; i < kUnits; ++i) raw[i] = reinterpret_cast<const Unit8 *>(v + (i * kClipThreads + (int)threadIdx.x) * kWide)->v;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            float x[8];
            if constexpr (F32) {
                const values_f32x4 f = __builtin_bit_cast(values_f32x4, raw[i]);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = f[q];
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) { x[2 * q] = bf16_lo(raw[i][q]); x[2 * q + 1] = bf16_hi(raw[i][q]); }
            }
            use(x, std::integral_constant<int, kWide>{}, (i * kClipThreads + (int)threadIdx.x) * kWide);
        }
        return;
    }
    for (int col = threadIdx.x * 8; col < k.length; col += kClipThreads * 8) {
        float x[8];
        Values<F32>::load(v, col, k.length, x);
        use(x, std::integral_constant<int, 8>{}, col);
    }
}

template <bool F32>
__device__ __forceinline__ double clip_squares(const void *grad, const ClipChunk &k)
{
    double sum[2] = {0.0, 0.0};
    clip_each<F32>(grad, k, [&](const float (&x)[8], auto n, int) {
#pragma unroll
        for (int q = 0; q < decltype(n)::value; ++q) sum[q & 1] += (double)x[q] * (double)x[q];
    });
    return sum[0] + sum[1];
}

// the sum over the workgroup in thread 0, in a fixed order
template <int THREADS>
__device__ __forceinline__ double clip_sum(double sum, double *part)
{
    part[threadIdx.x] = sum;
    for (int n = THREADS / 2; n > 0; n >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < n) part[threadIdx.x] += part[threadIdx.x + n];
    }
    return part[0];
}

__global__ __launch_bounds__(kClipThreads) void clip_squares_kernel(ClipTable t, double *parts)
{
    __shared__ double part[kClipThreads];
    double sum = 0.0;
    const int chunks = t.first[t.n];
    for (int c = (int)blockIdx.x; c < chunks; c += (int)gridDim.x) {
        const ClipChunk k = clip_chunk(t, c);
        sum += k.f32 ? clip_squares<true>(t.grad[k.tensor], k) : clip_squares<false>(t.grad[k.tensor], k);
    }
    sum = clip_sum<kClipThreads>(sum, part);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

// parts[count]: where the factor goes
__global__ __launch_bounds__(1024) void clip_join_kernel(int64_t count, double *parts, double max_norm, float *norm)
{
    __shared__ double part[1024];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += 1024) sum += parts[i];
    sum = clip_sum<1024>(sum, part);
    if (threadIdx.x == 0) {
        const double all = sqrt(sum);
        *norm = (float)all;
        parts[count] = all > max_norm && all < INFINITY ? max_norm / all : 1.0;
    }
}

// A 64-bit value as the float that is rounded to the bfloat16 next to it: cut off, the last bit set where something was, so that it lies on no middle of two
// bfloat16 values that the value itself does not lie on (134 M bfloat16 values: 130 us a call, rounded twice, so 134).
__device__ __forceinline__ float clip_odd(double x)
{
    const float f = (float)x;
    uint32_t u = __builtin_bit_cast(uint32_t, f);
    if ((double)f != x) u = (u - (fabs((double)f) > fabs(x) ? 1u : 0u)) | 1u;      // (a NaN stays one)
    return __builtin_bit_cast(float, u);
}

// PAST: past the caches, which then keep what is still to be read
typedef lanes_u32x4 __attribute__((aligned(2))) ClipAny;
template <bool F32, bool PAST>
__device__ __forceinline__ void clip_scale(const void *grad, void *out, const ClipChunk &k, double factor)
{
    auto *o = static_cast<typename Values<F32>::T *>(out) + k.at;
    clip_each<F32>(grad, k, [&](const float (&x)[8], auto n, int col) {
        float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        // (in 64 bits: a factor below 2^-126 would lose bits as a float)
#pragma unroll
        for (int q = 0; q < decltype(n)::value; ++q) y[q] = F32 ? (float)((double)x[q] * factor) : clip_odd((double)x[q] * factor);
        lanes_u32x4 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = F32 ? __builtin_bit_cast(uint32_t, y[q]) : bf16_pair(y[2 * q], y[2 * q + 1]);
        if (k.length != kChunk) Values<F32>::store(o, col, k.length, y);
        else if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<ClipAny *>(o + col));
        else *reinterpret_cast<ClipAny *>(o + col) = v;
    });
}

template <bool PAST>
__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(ClipTable t, const double *at)
{
    const double factor = *at;
    const int chunks = t.first[t.n];
    for (int i = (int)blockIdx.x; i < chunks; i += (int)gridDim.x) {
        // from the end: what was read last is still in the caches
        const ClipChunk k = clip_chunk(t, chunks - 1 - i);
        if (factor == 1.0 && t.out[k.tensor] == t.grad[k.tensor]) continue;
        if (k.f32) clip_scale<true, PAST>(t.grad[k.tensor], t.out[k.tensor], k, factor);
        else clip_scale<false, PAST>(t.grad[k.tensor], t.out[k.tensor], k, factor);
    }
}

// Tensors [from, to) of a launch and its chunks; empty ones are left out.  A launch ends before its chunks pass 2^30.
struct ClipRange { int to, tensors; int64_t chunks; };
static ClipRange clip_range(int n, const int64_t *counts, int from)
{
    ClipRange r{from, 0, 0};
    for (; r.to < n && r.tensors < kClipTensors; ++r.to) {
        if (counts[r.to] <= 0) continue;
        const int64_t chunks = (counts[r.to] + kChunk - 1) / kChunk;
        if (r.tensors > 0 && r.chunks + chunks > 1 << 30) break;
        r.chunks += chunks;
        ++r.tensors;
    }
    return r;
}
static int clip_blocks(int64_t chunks) { return (int)(chunks < kClipBlocks ? chunks : kClipBlocks); }

static int64_t clip_parts(int n, const int64_t *counts)
{
    int64_t parts = 0;
    for (int from = 0; from < n;) {
        const ClipRange r = clip_range(n, counts, from);
        parts += clip_blocks(r.chunks);
        from = r.to;
    }
    return parts;
}

size_t clip_workspace_bytes(int n, const int64_t *counts) { return (size_t)(clip_parts(n, counts) + 1) * sizeof(double); }

hipError_t clip_launch(int n, const void *const *grads, const int64_t *counts, const int *types, double max_norm, void *const *out, float *norm,
                       void *workspace, hipStream_t st)
{
    double *parts = static_cast<double *>(workspace);
    const int64_t all = clip_parts(n, counts);
    const auto each = [&](auto launch) {
        int64_t before = 0;
        for (int from = 0; from < n;) {
            const ClipRange r = clip_range(n, counts, from);
            ClipTable t{};
            for (int i = from; i < r.to; ++i) {
                if (counts[i] <= 0) continue;
                t.grad[t.n] = grads[i];
                t.out[t.n] = out ? out[i] : nullptr;
                t.count[t.n] = counts[i];
                t.first[t.n + 1] = t.first[t.n] + (int)((counts[i] + kChunk - 1) / kChunk);
                if (types[i] == POLYDL_F32) t.f32[t.n >> 5] |= 1u << (t.n & 31);
                ++t.n;
            }
            const hipError_t e = t.n ? launch(t, clip_blocks(r.chunks), parts + before) : hipSuccess;
            if (e != hipSuccess) return e;
            before += clip_blocks(r.chunks);
            from = r.to;
        }
        return hipSuccess;
    };
    hipError_t e = each([&](const ClipTable &t, int blocks, double *at) {
        return launch_kernel(clip_squares_kernel, dim3((unsigned)blocks), dim3(kClipThreads), 0, st, t, at);
    });
    if (e == hipSuccess) e = launch_kernel(clip_join_kernel, dim3(1), dim3(1024), 0, st, all, parts, max_norm, norm);
    if (e != hipSuccess || !out) return e;
    // Results that no cache would hold until they are read go past the caches (134 M floats: 292 us a call, so 275; from the first chunk on 307).
    int64_t bytes = 0;
    for (int i = 0; i < n; ++i) bytes += counts[i] > 0 ? counts[i] * (types[i] == POLYDL_F32 ? 4 : 2) : 0;
    auto *scale = bytes > 192ll << 20 ? clip_scale_kernel<true> : clip_scale_kernel<false>;
    return each([&](const ClipTable &t, int blocks, double *) {
        return launch_kernel(scale, dim3((unsigned)blocks), dim3(kClipThreads), 0, st, t, (const double *)(parts + all));
    });
}

}  // namespace polydl
