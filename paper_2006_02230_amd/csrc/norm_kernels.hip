// Layer norm of rows and its gradient.
//
// Forward: LANES lanes take a row and hold it in registers, NV units of eight values each, so it is read once; the mean first, then the squares of what
// is left (no difference of large sums), then the result.  Longer rows are read three times, the second and third time from the L2.
// Bound: HBM, x read and y written once.
#include <hip/hip_runtime.h>
#include "block.hpp"
#include "blocks.hpp"
#include "internal.hpp"
#include "lanes.hpp"
#include "values.hpp"

namespace polydl {

// The sum over LANES neighbouring threads, in all of them.  More than a wave: the waves' sums meet in `part`, in the order of the waves.
template <int LANES>
__device__ __forceinline__ float norm_sum(float x, float *part)
{
    if constexpr (LANES <= 64) return group_sum<LANES>(x);
    x = wave_sum(x);
    __syncthreads();                       // the last sum has been read
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    float sum = part[0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) sum += part[w];
    return sum;
}

template <bool X32, bool Y32, int LANES, int NV>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_kernel(NormProblem p)
{
    constexpr int kRows = LANES >= 256 ? 1 : 256 / LANES;
    __shared__ float part[16];
    const int l = threadIdx.x % LANES;
    const int64_t t = (int64_t)block_number() * kRows + threadIdx.x / LANES;
    if (LANES >= 64 && t >= p.T) return;               // (the same for a wave)
    const bool here = t < p.T;
    const auto *x = static_cast<const typename Values<X32>::T *>(p.x) + t * p.ldx;
    float v[NV][8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * LANES + l) * 8;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[i][q] = 0.f;
        if (here && col < p.D) Values<X32>::load(x, col, p.D, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) sum += ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3])) + ((v[i][4] + v[i][5]) + (v[i][6] + v[i][7]));
    const float mean = norm_sum<LANES>(sum, part) / (float)p.D;
    float square = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            v[i][q] = (i * LANES + l) * 8 + q < p.D ? v[i][q] - mean : 0.f;
            square += v[i][q] * v[i][q];
        }
    const float rstd = 1.f / sqrtf(norm_sum<LANES>(square, part) / (float)p.D + p.eps);
    if (!here) return;
    if (l == 0) {
        if (p.mean) p.mean[t] = mean;
        if (p.rstd) p.rstd[t] = rstd;
    }
    auto *y = static_cast<typename Values<Y32>::T *>(p.y) + t * p.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * LANES + l) * 8;
        if (col >= p.D) continue;
        float g[8], b[8], o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) { g[q] = 1.f; b[q] = 0.f; }
        if (p.gamma) Values<true>::load(p.gamma, col, p.D, g);
        if (p.beta) Values<true>::load(p.beta, col, p.D, b);
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] = v[i][q] * rstd * g[q] + b[q];
        Values<Y32>::store(y, col, p.D, o);
    }
}

// rows of any length
constexpr int kNormLong = 1024;
template <bool X32, bool Y32>
__global__ __launch_bounds__(kNormLong) void norm_long_kernel(NormProblem p)
{
    __shared__ float part[16];
    const int64_t t = block_number();
    if (t >= p.T) return;
    const auto *x = static_cast<const typename Values<X32>::T *>(p.x) + t * p.ldx;
    float v[8], sum = 0.f;
    for (int col = threadIdx.x * 8; col < p.D; col += kNormLong * 8) {
        Values<X32>::load(x, col, p.D, v);
        sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    const float mean = norm_sum<kNormLong>(sum, part) / (float)p.D;
    float square = 0.f;
    for (int col = threadIdx.x * 8; col < p.D; col += kNormLong * 8) {
        Values<X32>::load(x, col, p.D, v);
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s += col + q < p.D ? (v[q] - mean) * (v[q] - mean) : 0.f;
        square += s;
    }
    const float rstd = 1.f / sqrtf(norm_sum<kNormLong>(square, part) / (float)p.D + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[t] = mean;
        if (p.rstd) p.rstd[t] = rstd;
    }
    auto *y = static_cast<typename Values<Y32>::T *>(p.y) + t * p.ldy;
    for (int col = threadIdx.x * 8; col < p.D; col += kNormLong * 8) {
        Values<X32>::load(x, col, p.D, v);
        float g[8], b[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) { g[q] = 1.f; b[q] = 0.f; }
        if (p.gamma) Values<true>::load(p.gamma, col, p.D, g);
        if (p.beta) Values<true>::load(p.beta, col, p.D, b);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = (v[q] - mean) * rstd * g[q] + b[q];
        Values<Y32>::store(y, col, p.D, v);
    }
}

template <bool X32, bool Y32, int LANES, int NV>
static hipError_t norm_run(const NormProblem &p, hipStream_t st)
{
    constexpr int rows = LANES >= 256 ? 1 : 256 / LANES, threads = LANES > 256 ? LANES : 256;
    return launch_kernel((norm_kernel<X32, Y32, LANES, NV>), many_blocks(((int64_t)p.T + rows - 1) / rows, threads), dim3(threads), 0, st, p);
}

template <bool X32, bool Y32>
static hipError_t norm_pick(const NormProblem &p, hipStream_t st)
{
    if (p.D <= 16 * 8) return norm_run<X32, Y32, 16, 1>(p, st);
    if (p.D <= 64 * 8) return norm_run<X32, Y32, 64, 1>(p, st);
    if (p.D <= 64 * 16) return norm_run<X32, Y32, 64, 2>(p, st);
    if (p.D <= 64 * 32) return norm_run<X32, Y32, 64, 4>(p, st);
    if (p.D <= 256 * 16) return norm_run<X32, Y32, 256, 2>(p, st);
    if (p.D <= 256 * 32) return norm_run<X32, Y32, 256, 4>(p, st);
    if (p.D <= 1024 * 16) return norm_run<X32, Y32, 1024, 2>(p, st);
    return launch_kernel((norm_long_kernel<X32, Y32>), many_blocks(p.T, kNormLong), dim3(kNormLong), 0, st, p);
}

hipError_t norm_launch(const NormProblem &p, hipStream_t st)
{
    if (p.x_f32) return p.y_f32 ? norm_pick<true, true>(p, st) : norm_pick<true, false>(p, st);
    return p.y_f32 ? norm_pick<false, true>(p, st) : norm_pick<false, false>(p, st);
}

// ---- gradient ---------------------------------------------------------------------------------------------------
// dx: a workgroup a row, read twice.
constexpr int kGradThreads = 256;
template <bool DY32, bool X32>
__global__ __launch_bounds__(kGradThreads) void norm_dx_kernel(NormGradProblem p)
{
    __shared__ float part[16];
    const int64_t t = block_number();
    if (t >= p.T) return;
    const auto *x = static_cast<const typename Values<X32>::T *>(p.x) + t * p.ldx;
    const auto *dy = static_cast<const typename Values<DY32>::T *>(p.dy) + t * p.lddy;
    const float mean = p.mean[t], rstd = p.rstd[t];
    float sum = 0.f, along = 0.f, g[8], h[8], w[8];
    const auto read = [&](int col) {
        Values<DY32>::load(dy, col, p.D, g);
        Values<X32>::load(x, col, p.D, h);
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = 1.f;
        if (p.gamma) Values<true>::load(p.gamma, col, p.D, w);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            g[q] *= w[q];
            h[q] = col + q < p.D ? (h[q] - mean) * rstd : 0.f;
        }
    };
    for (int col = threadIdx.x * 8; col < p.D; col += kGradThreads * 8) {
        read(col);
#pragma unroll
        for (int q = 0; q < 8; ++q) { sum += g[q]; along += g[q] * h[q]; }
    }
    sum = norm_sum<kGradThreads>(sum, part) / (float)p.D;
    along = norm_sum<kGradThreads>(along, part) / (float)p.D;
    auto *dx = static_cast<typename Values<X32>::T *>(p.dx) + t * p.lddx;
    for (int col = threadIdx.x * 8; col < p.D; col += kGradThreads * 8) {
        read(col);
#pragma unroll
        for (int q = 0; q < 8; ++q) g[q] = rstd * (g[q] - sum - h[q] * along);
        Values<X32>::store(dx, col, p.D, g);
    }
}

// dgamma and dbeta of a chunk of rows: a wave takes 512 columns and every fourth row, the waves meet in LDS in their order.
template <bool DY32, bool X32>
__global__ __launch_bounds__(256) void norm_dweights_kernel(NormGradProblem p, int per, float *parts)
{
    __shared__ float sums[2][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = ((int)blockIdx.y * 64 + lane) * 8;
    const int64_t t0 = (int64_t)blockIdx.x * per, t1 = min((int64_t)p.T, t0 + per);
    float dg[8], db[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) dg[q] = db[q] = 0.f;
    if (col < p.D) {
        for (int64_t t = t0 + wave; t < t1; t += 4) {
            float g[8], h[8];
            Values<DY32>::load(static_cast<const typename Values<DY32>::T *>(p.dy) + t * p.lddy, col, p.D, g);
            Values<X32>::load(static_cast<const typename Values<X32>::T *>(p.x) + t * p.ldx, col, p.D, h);
            const float mean = p.mean[t], rstd = p.rstd[t];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                dg[q] += g[q] * ((h[q] - mean) * rstd);
                db[q] += g[q];
            }
        }
    }
    for (int w = 0; w < 4; ++w) {
        if (wave == w) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                sums[0][q * 64 + lane] = (w ? sums[0][q * 64 + lane] : 0.f) + dg[q];
                sums[1][q * 64 + lane] = (w ? sums[1][q * 64 + lane] : 0.f) + db[q];
            }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < 512; i += 256) {
        const int c = (int)blockIdx.y * 512 + i;
        if (c >= p.D) continue;
        const int at = (i & 7) * 64 + (i >> 3);
        parts[((int64_t)blockIdx.x * 2 + 0) * p.D + c] = sums[0][at];
        parts[((int64_t)blockIdx.x * 2 + 1) * p.D + c] = sums[1][at];
    }
}

// The chunks' sums: 64 columns of dgamma or dbeta a workgroup, every sixteenth chunk a wave.
__global__ __launch_bounds__(1024) void norm_join_kernel(int D, int chunks, const float *parts, float *dgamma, float *dbeta, int accumulate)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = (int)blockIdx.y;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float *out = which ? dbeta : dgamma;
    if (!out) return;
    float sum = 0.f;
    if (col < D)
        for (int c = wave; c < chunks; c += 16) sum += parts[((int64_t)c * 2 + which) * D + col];
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave || col >= D) return;
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    out[col] = accumulate ? out[col] + sum : sum;
}

static int norm_chunks(int T) { return T <= 0 ? 0 : (int)(((int64_t)T + 63) / 64 < 256 ? ((int64_t)T + 63) / 64 : 256); }

size_t norm_bwd_workspace_bytes(int T, int D) { return (size_t)norm_chunks(T) * 2 * (size_t)D * sizeof(float); }

template <bool DY32, bool X32>
static hipError_t norm_bwd_run(const NormGradProblem &p, float *parts, hipStream_t st)
{
    hipError_t e = hipSuccess;
    if (p.dx && p.T > 0) e = launch_kernel((norm_dx_kernel<DY32, X32>), many_blocks(p.T, kGradThreads), dim3(kGradThreads), 0, st, p);
    if (e != hipSuccess || (!p.dgamma && !p.dbeta)) return e;
    const int chunks = norm_chunks(p.T), per = chunks ? (int)(((int64_t)p.T + chunks - 1) / chunks) : 0;
    if (chunks) e = launch_kernel((norm_dweights_kernel<DY32, X32>), dim3((unsigned)chunks, (unsigned)((p.D + 511) / 512)), dim3(256), 0, st, p, per, parts);
    if (e != hipSuccess) return e;
    return launch_kernel(norm_join_kernel, dim3((unsigned)((p.D + 63) / 64), 2u), dim3(1024), 0, st, p.D, chunks, parts, p.dgamma, p.dbeta, p.accumulate);
}

hipError_t norm_bwd_launch(const NormGradProblem &p, void *workspace, hipStream_t st)
{
    float *parts = static_cast<float *>(workspace);
    if (p.dy_f32) return p.x_f32 ? norm_bwd_run<true, true>(p, parts, st) : norm_bwd_run<true, false>(p, parts, st);
    return p.x_f32 ? norm_bwd_run<false, true>(p, parts, st) : norm_bwd_run<false, false>(p, parts, st);
}

}  // namespace polydl
