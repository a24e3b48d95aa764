// Layer norm of rows and its gradient.
//
// Forward: LANES lanes take a row and hold it in registers, NV units of eight values each, so it is read once; the mean first, then the squares of what
// is left (no difference of large sums), then the result.  A float32 sum's mean is off by an ulp or more of itself, which may be more than the row's
// spread; the differences from it are nearly exact, and their own mean is what it is off by: that is taken out before the squares (16384 x 2048
// bfloat16 31.0 -> 31.3 us in a graph, one row 3.7 -> 3.9).  Equal values leave zeros: their sums are off by some tens of ulps, so all differences are the same
// few ulps, whose sum over 16384 values 24 bits hold exactly.  Longer rows are read three times, the second and third time from the L2, and
// their mean is formed in 64 bits, which hold the sum of 2^24 equal floats exactly, too (1600 x 20480 bfloat16 43.6 -> 45.8 us).
// Bound: HBM, x read and y written once.
#include <hip/hip_runtime.h>
#include <math.h>
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
    constexpr int kWaves = LANES / 64;
    x = wave_sum(x);
    __syncthreads();                       // the last sum has been read
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    const float *mine = part + threadIdx.x / LANES * kWaves;
    float sum = mine[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum += mine[w];
    return sum;
}

// the sum over a workgroup of 64-bit values, in all of its threads, in a fixed order
template <int THREADS>
__device__ __forceinline__ double norm_sum(double x, double *part)
{
#pragma unroll
    for (int n = 1; n < 64; n += n) x += __shfl_xor(x, n);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    double sum = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) sum += part[w];
    return sum;
}

// a * b, rounded: what is subtracted from all values of a row and added to their mean again has to be one number, not a product fused into each
__device__ __forceinline__ float norm_product(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}
// sum / n from n's reciprocal, exact where the quotient is a float: the first quotient's remainder is formed exactly and divided, too
__device__ __forceinline__ float norm_quotient(float sum, float n, float over)
{
    const float q = norm_product(sum, over);
    return fmaf(fmaf(-q, n, sum), over, q);
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
    const float length = (float)p.D, over = 1.f / length;      // (the quotients of the sums would wait for one another)
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
    const float near = norm_product(norm_sum<LANES>(sum, part), over);
    float left = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            v[i][q] = (i * LANES + l) * 8 + q < p.D ? v[i][q] - near : 0.f;
            left += v[i][q];
        }
    left = norm_quotient(norm_sum<LANES>(left, part), length, over);
    const float mean = fabsf(left) < INFINITY ? near + left : near;      // (a row with an infinity has an infinite mean)
    float square = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            v[i][q] = (i * LANES + l) * 8 + q < p.D ? v[i][q] - left : 0.f;
            square += v[i][q] * v[i][q];
        }
    const float rstd = 1.f / sqrtf(norm_sum<LANES>(square, part) * over + p.eps);
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
    __shared__ double wide[16];
    const int64_t t = block_number();
    if (t >= p.T) return;
    const auto *x = static_cast<const typename Values<X32>::T *>(p.x) + t * p.ldx;
    float v[8];
    double sum = 0.0;
    for (int col = threadIdx.x * 8; col < p.D; col += kNormLong * 8) {
        Values<X32>::load(x, col, p.D, v);
        sum += (((double)v[0] + v[1]) + ((double)v[2] + v[3])) + (((double)v[4] + v[5]) + ((double)v[6] + v[7]));
    }
    const double mean = norm_sum<kNormLong>(sum, wide) / (double)p.D;
    float square = 0.f;
    for (int col = threadIdx.x * 8; col < p.D; col += kNormLong * 8) {
        Values<X32>::load(x, col, p.D, v);
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float c = (float)(v[q] - mean);
            s += col + q < p.D ? c * c : 0.f;
        }
        square += s;
    }
    const float rstd = 1.f / sqrtf(norm_sum<kNormLong>(square, part) / (float)p.D + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[t] = (float)mean;
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
        for (int q = 0; q < 8; ++q) v[q] = (float)(v[q] - mean) * rstd * g[q] + b[q];
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
// A workgroup goes over rows with a stride, LANES lanes a row; every lane keeps its columns' parts of dgamma and dbeta in registers from row to row, so x
// and dy are read once for all three results, the next row while this one is worked on.  At its end the workgroup's rows meet in LDS in their order, the
// workgroups' sums in the workspace.
// Bound: HBM, x and dy read and dx written once (16384 x 2048 bfloat16: 36.3 us, and 4.2 for the workgroups' sums, 201 MB at 5.0 TB/s; in kernels of their own dx
// took 41.7 us and the weights 22.4 more).
constexpr int kGradThreads = 512, kGradBlocks = 256;         // (more workgroups write more sums: 16 KB each for rows of 2048)
// Two sums over LANES neighbouring threads; more than a wave's meet in `part`, of which neighbouring rows use different halves, so that one barrier a row
// suffices.
template <int LANES>
__device__ __forceinline__ void norm_sums(float &a, float &b, float (*part)[kGradThreads / 64], int row)
{
    a = group_sum<LANES < 64 ? LANES : 64>(a);
    b = group_sum<LANES < 64 ? LANES : 64>(b);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        part += (row & 1) * 2;
        if ((threadIdx.x & 63) == 0) {
            part[0][threadIdx.x >> 6] = a;
            part[1][threadIdx.x >> 6] = b;
        }
        __syncthreads();
        const int mine = threadIdx.x / LANES * kWaves;
        a = part[0][mine];
        b = part[1][mine];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            a += part[0][mine + w];
            b += part[1][mine + w];
        }
    }
}

template <bool DY32, bool X32, int LANES, int NV, bool WEIGHTS>
__global__ __launch_bounds__(kGradThreads) void norm_bwd_kernel(NormGradProblem p, float *parts)
{
    constexpr int kRows = kGradThreads / LANES, kColumns = LANES * NV * 8, kWaves = kGradThreads / 64;
    constexpr int kTurns = LANES < 64 ? kWaves : kRows;      // groups of lanes that hold the same columns, after a wave's own have met
    __shared__ float part[4][kWaves];
    __shared__ float sums[WEIGHTS && kTurns > 1 ? kTurns / 2 * 2 * kColumns : 1];
    const int l = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int64_t step = (int64_t)gridDim.x * kRows;
    typename Values<X32>::Raw xr[NV];
    typename Values<DY32>::Raw dr[NV];
    float w[NV][8], dg[NV][8], db[NV][8], mean = 0.f, rstd = 0.f;
    const auto load = [&](int64_t t) {
        if (t >= p.T) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * LANES + l) * 8;
            if (col >= p.D) continue;
            xr[i] = Values<X32>::load_raw(static_cast<const typename Values<X32>::T *>(p.x) + t * p.ldx, col, p.D);
            dr[i] = Values<DY32>::load_raw(static_cast<const typename Values<DY32>::T *>(p.dy) + t * p.lddy, col, p.D);
        }
        mean = p.mean[t];
        rstd = p.rstd[t];
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * LANES + l) * 8;
#pragma unroll
        for (int q = 0; q < 8; ++q) { w[i][q] = 1.f; dg[i][q] = db[i][q] = 0.f; }
        xr[i] = {};
        dr[i] = {};
        if (p.gamma && col < p.D) Values<true>::load(p.gamma, col, p.D, w[i]);
    }
    // (all groups of a workgroup take the same number of turns, for its barriers)
    int64_t t = (int64_t)blockIdx.x * kRows + group;
    load(t);
    const float over = 1.f / (float)p.D;
    int row = 0;
    for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < p.T; t0 += step, t += step, ++row) {
        float h[NV][8], g[NV][8], sum = 0.f, along = 0.f;
        const float m = mean, s = rstd;
        const bool here = t < p.T;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Values<X32>::convert(xr[i], h[i]);
            Values<DY32>::convert(dr[i], g[i]);
        }
        load(t + step);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const bool there = here && (i * LANES + l) * 8 + q < p.D;
                h[i][q] = there ? (h[i][q] - m) * s : 0.f;
                if constexpr (WEIGHTS) {
                    dg[i][q] += there ? g[i][q] * h[i][q] : 0.f;
                    db[i][q] += there ? g[i][q] : 0.f;
                }
                g[i][q] = there ? g[i][q] * w[i][q] : 0.f;
                sum += g[i][q];
                along += g[i][q] * h[i][q];
            }
        if (!p.dx) continue;
        norm_sums<LANES>(sum, along, part, row);
        sum *= over;
        along *= over;
        if (!here) continue;
        auto *dx = static_cast<typename Values<X32>::T *>(p.dx) + t * p.lddx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * LANES + l) * 8;
            if (col >= p.D) continue;
#pragma unroll
            for (int q = 0; q < 8; ++q) g[i][q] = s * (g[i][q] - sum - h[i][q] * along);
            Values<X32>::store(dx, col, p.D, g[i]);
        }
    }
    if constexpr (!WEIGHTS) return;
#pragma unroll
    for (int x = LANES; x < 64; x += x)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                dg[i][q] += __shfl_xor(dg[i][q], x);
                db[i][q] += __shfl_xor(db[i][q], x);
            }
    // Half of the groups hand their sums to the other half, until one has them all (in turns, eight groups took 1 us longer).  What a lane hands over lies LANES
    // apart, so that neighbouring lanes fall on different banks.
    const int mine = LANES < 64 ? (int)threadIdx.x >> 6 : group;
    const bool speaks = LANES >= 64 || (int)(threadIdx.x & 63) < LANES;
    for (int half = kTurns / 2; half >= 1; half >>= 1) {
        if (speaks && mine >= half && mine < 2 * half) {
            float *to = sums + (mine - half) * 2 * kColumns + l;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    to[(i * 8 + q) * LANES] = dg[i][q];
                    to[kColumns + (i * 8 + q) * LANES] = db[i][q];
                }
        }
        __syncthreads();
        if (speaks && mine < half) {
            const float *from = sums + mine * 2 * kColumns + l;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    dg[i][q] += from[(i * 8 + q) * LANES];
                    db[i][q] += from[kColumns + (i * 8 + q) * LANES];
                }
        }
        __syncthreads();
    }
    if (mine != 0 || !speaks) return;
    const auto leave = [&](float (&v)[NV][8], float *out, int which) {
        if (gridDim.x > 1) out = parts + ((int64_t)blockIdx.x * 2 + which) * p.D;
        if (!out) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * LANES + l) * 8;
            if (col >= p.D) continue;
            if (gridDim.x == 1 && p.accumulate) {
                float was[8];
                Values<true>::load(out, col, p.D, was);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[i][q] += was[q];
            }
            Values<true>::store(out, col, p.D, v[i]);
        }
    };
    leave(dg, p.dgamma, 0);
    leave(db, p.dbeta, 1);
}

// The workgroups' sums: 64 columns of dgamma or dbeta a workgroup, every sixteenth part a wave, sixteen of them on their way at a time.
__global__ __launch_bounds__(1024) void norm_join_kernel(int D, int chunks, const float *parts, float *dgamma, float *dbeta, int accumulate)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, which = (int)blockIdx.y;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float *out = which ? dbeta : dgamma;
    if (!out) return;
    constexpr int kHeld = 16;
    float sum = 0.f;
    for (int c0 = wave; c0 < chunks; c0 += 16 * kHeld) {
        float v[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int c = c0 + i * 16;
            v[i] = c < chunks && col < D ? parts[((int64_t)c * 2 + which) * D + col] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) sum += v[i];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave || col >= D) return;
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    out[col] = accumulate ? out[col] + sum : sum;
}

// Rows too long for registers.  dx: a workgroup a row, read twice.
constexpr int kLongThreads = 256;
template <bool DY32, bool X32>
__global__ __launch_bounds__(kLongThreads) void norm_dx_kernel(NormGradProblem p)
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
    for (int col = threadIdx.x * 8; col < p.D; col += kLongThreads * 8) {
        read(col);
#pragma unroll
        for (int q = 0; q < 8; ++q) { sum += g[q]; along += g[q] * h[q]; }
    }
    sum = norm_sum<kLongThreads>(sum, part) / (float)p.D;
    along = norm_sum<kLongThreads>(along, part) / (float)p.D;
    auto *dx = static_cast<typename Values<X32>::T *>(p.dx) + t * p.lddx;
    for (int col = threadIdx.x * 8; col < p.D; col += kLongThreads * 8) {
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

constexpr int kGradLongest = kGradThreads * 16;              // values of a row that registers hold

// Rows that a workgroup takes at a time.
static int norm_rows(int D) { return D <= 16 * 8 ? kGradThreads / 16 : D <= 64 * 16 ? kGradThreads / 64 : D <= 128 * 16 ? kGradThreads / 128 : D <= 256 * 16 ? kGradThreads / 256 : 1; }
static int norm_chunks(int T, int D)
{
    const int64_t rows = D <= kGradLongest ? norm_rows(D) : 64, chunks = ((int64_t)T + rows - 1) / rows;
    return (int)(chunks < kGradBlocks ? chunks : kGradBlocks);
}

size_t norm_bwd_workspace_bytes(int T, int D) { return (size_t)norm_chunks(T, D) * 2 * (size_t)D * sizeof(float); }

template <bool DY32, bool X32, int LANES, int NV>
static hipError_t norm_bwd_run(const NormGradProblem &p, float *parts, hipStream_t st)
{
    // without weights nothing is kept from row to row: more workgroups even the rows out
    const int64_t rows = kGradThreads / LANES, all = ((int64_t)p.T + rows - 1) / rows;
    if (!p.dgamma && !p.dbeta)
        return launch_kernel((norm_bwd_kernel<DY32, X32, LANES, NV, false>), dim3((unsigned)(all < 2048 ? all : 2048)), dim3(kGradThreads), 0, st, p, parts);
    const int chunks = norm_chunks(p.T, p.D);
    const hipError_t e = launch_kernel((norm_bwd_kernel<DY32, X32, LANES, NV, true>), dim3((unsigned)chunks), dim3(kGradThreads), 0, st, p, parts);
    if (e != hipSuccess || chunks == 1) return e;
    return launch_kernel(norm_join_kernel, dim3((unsigned)((p.D + 63) / 64), 2u), dim3(1024), 0, st, p.D, chunks, parts, p.dgamma, p.dbeta, p.accumulate);
}

template <bool DY32, bool X32>
static hipError_t norm_bwd_long(const NormGradProblem &p, float *parts, hipStream_t st)
{
    if (p.dgamma || p.dbeta) {
        const int chunks = norm_chunks(p.T, p.D), per = (int)(((int64_t)p.T + chunks - 1) / chunks);
        hipError_t e = launch_kernel((norm_dweights_kernel<DY32, X32>), dim3((unsigned)chunks, (unsigned)((p.D + 511) / 512)), dim3(256), 0, st, p, per, parts);
        if (e == hipSuccess)
            e = launch_kernel(norm_join_kernel, dim3((unsigned)((p.D + 63) / 64), 2u), dim3(1024), 0, st, p.D, chunks, parts, p.dgamma, p.dbeta, p.accumulate);
        if (e != hipSuccess) return e;
    }
    return p.dx ? launch_kernel((norm_dx_kernel<DY32, X32>), many_blocks(p.T, kLongThreads), dim3(kLongThreads), 0, st, p) : hipSuccess;
}

template <bool DY32, bool X32>
static hipError_t norm_bwd_pick(const NormGradProblem &p, float *parts, hipStream_t st)
{
    if (p.T <= 0)                      // sums of nothing
        return launch_kernel(norm_join_kernel, dim3((unsigned)((p.D + 63) / 64), 2u), dim3(1024), 0, st, p.D, 0, parts, p.dgamma, p.dbeta, p.accumulate);
    if (p.D <= 16 * 8) return norm_bwd_run<DY32, X32, 16, 1>(p, parts, st);
    if (p.D <= 64 * 8) return norm_bwd_run<DY32, X32, 64, 1>(p, parts, st);
    if (p.D <= 64 * 16) return norm_bwd_run<DY32, X32, 64, 2>(p, parts, st);
    // (four units a lane would not fit in its registers beside their sums)
    if (p.D <= 128 * 16) return norm_bwd_run<DY32, X32, 128, 2>(p, parts, st);
    if (p.D <= 256 * 16) return norm_bwd_run<DY32, X32, 256, 2>(p, parts, st);
    if (p.D <= 512 * 16) return norm_bwd_run<DY32, X32, 512, 2>(p, parts, st);
    return norm_bwd_long<DY32, X32>(p, parts, st);
}

hipError_t norm_bwd_launch(const NormGradProblem &p, void *workspace, hipStream_t st)
{
    float *parts = static_cast<float *>(workspace);
    if (p.dy_f32) return p.x_f32 ? norm_bwd_pick<true, true>(p, parts, st) : norm_bwd_pick<true, false>(p, parts, st);
    return p.x_f32 ? norm_bwd_pick<false, true>(p, parts, st) : norm_bwd_pick<false, false>(p, parts, st);
}

}  // namespace polydl
