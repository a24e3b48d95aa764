// The balance loss of a router, its counts and its gradient.
//
// A row's probabilities take LANES lanes, as its choice does (route_kernels.hip): 16 for up to 256 experts, four rows a wave, else a wave.  A
// lane adds its experts' probabilities up over the workgroup's rows in registers; the lanes' sums meet in LDS in a fixed order, the workgroups' in
// the workspace.  Choices are counted with integer atomics in LDS, whose order does not matter.
// Bound: latency and instruction issue; the logits of 16384 rows of 128 experts are 8 MB.
#include <hip/hip_runtime.h>
#include <math.h>
#include "block.hpp"
#include "blocks.hpp"
#include "experts.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace polydl {

// order-preserving keys: 0 for -infinity, all ones for NaN
__device__ __forceinline__ uint32_t balance_key(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    return v != v ? 0xffffffffu : v == -INFINITY ? 0u : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float balance_value(uint32_t key)
{
    return __builtin_bit_cast(float, key >> 31 ? key ^ 0x80000000u : ~key);
}

// p: the lane's NV probabilities of a row (NULL: none, zeros).  False where no expert is open.
template <int LANES, int NV>
__device__ __forceinline__ bool balance_row(const float *row, int E, int l, float (&p)[NV])
{
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        p[i] = row && e < E ? row[e] : -INFINITY;
        const uint32_t key = balance_key(p[i]);
        m = key > m ? key : m;
    }
    m = group_max<LANES>(m);
    const float best = balance_value(m);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        p[i] = m ? expf(p[i] - best) : 0.f;
        sum += p[i];
    }
    sum = group_sum<LANES>(sum);
#pragma unroll
    for (int i = 0; i < NV; ++i) p[i] = m ? p[i] / sum : 0.f;
    return m != 0u;
}

constexpr int kBalanceThreads = 512, kBalanceWaves = kBalanceThreads / 64;

struct BalanceArgs {
    BalanceProblem p;
    int blocks, per;                // workgroups, rows of one
    float *part;                    // [blocks][E]: sums of probabilities
    int32_t *count;                 // [blocks][E]
    int32_t *open;                  // [blocks]
};

// loss and shares from the sums of probabilities and the counts, in LDS; the whole workgroup
template <int THREADS>
__device__ __forceinline__ void balance_finish(const BalanceProblem &p, const float *sums, const int *counts, int rows, double *part)
{
    double total = 0.0, product = 0.0;
    for (int e = threadIdx.x; e < p.E; e += THREADS) {
        const float share = rows ? sums[e] / (float)rows : 0.f;
        p.shares[e] = share;
        p.counts[e] = counts[e];
        total += (double)counts[e];
        product += (double)counts[e] * (double)share;
    }
    part[threadIdx.x] = total;
    part[THREADS + threadIdx.x] = product;
    for (int n = THREADS / 2; n > 0; n >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < n) {
            part[threadIdx.x] += part[threadIdx.x + n];
            part[THREADS + threadIdx.x] += part[THREADS + threadIdx.x + n];
        }
    }
    if (threadIdx.x == 0) {
        // NaN shares make the loss NaN without choices too
        *p.loss = (float)((double)p.E * (part[0] > 0.0 ? part[THREADS] / part[0] : part[THREADS]));
        *p.rows = rows;
    }
}

template <int LANES, int NV, bool ONE>
__global__ __launch_bounds__(kBalanceThreads) void balance_kernel(BalanceArgs a)
{
    constexpr int kExperts = LANES * NV;
    __shared__ float sums[kBalanceWaves][kExperts];
    __shared__ int counts[kExperts], open[kBalanceWaves];
    __shared__ double part[ONE ? 2 * kBalanceThreads : 1];
    const BalanceProblem &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = tid % LANES, b = (int)blockIdx.x;
    const int64_t t0 = (int64_t)b * a.per, t1 = min((int64_t)p.T, t0 + a.per);
    for (int e = tid; e < kExperts; e += kBalanceThreads) counts[e] = 0;
    __syncthreads();
    for (int64_t i = t0 * p.k + tid; i < t1 * p.k; i += kBalanceThreads) {
        const int id = p.ids[i];
        if ((unsigned)id < (unsigned)p.E) atomicAdd(&counts[id], 1);
    }
    float acc[NV];
    int rows = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) acc[i] = 0.f;
    for (int64_t t = t0; t < t1; t += kBalanceThreads / LANES) {
        const int64_t at = t + tid / LANES;
        float v[NV];
        const bool is = balance_row<LANES, NV>(at < t1 ? p.logits + at * p.E : nullptr, p.E, l, v);
        rows += is && l == 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) acc[i] += v[i];
    }
    // the rows of a wave, then the waves
#pragma unroll
    for (int x = LANES; x < 64; x += x)
#pragma unroll
        for (int i = 0; i < NV; ++i) acc[i] += __shfl_xor(acc[i], x);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (lane < LANES) sums[wave][i * LANES + l] = acc[i];
    rows = lane_of(wave_prefix(rows), 63);
    if (lane == 0) open[wave] = rows;
    __syncthreads();
    rows = 0;
    for (int w = 0; w < kBalanceWaves; ++w) rows += open[w];
    for (int e = tid; e < p.E; e += kBalanceThreads) {
        float sum = sums[0][e];
        for (int w = 1; w < kBalanceWaves; ++w) sum += sums[w][e];
        if constexpr (ONE) {
            sums[0][e] = sum;
        } else {
            a.part[(int64_t)b * p.E + e] = sum;
            a.count[(int64_t)b * p.E + e] = counts[e];
        }
    }
    if constexpr (ONE) {
        __syncthreads();
        balance_finish<kBalanceThreads>(p, sums[0], counts, rows, part);
    } else if (tid == 0) {
        a.open[b] = rows;
    }
}

// The workgroups' sums.
__global__ __launch_bounds__(1024) void balance_join_kernel(BalanceArgs a)
{
    __shared__ float sums[kRouteMaxExperts];
    __shared__ int counts[kRouteMaxExperts];
    __shared__ double part[2 * 1024];
    int rows = 0;
    for (int b = 0; b < a.blocks; ++b) rows += a.open[b];
    for (int e = threadIdx.x; e < a.p.E; e += 1024) {
        float sum = 0.f;
        int count = 0;
        for (int b = 0; b < a.blocks; ++b) {
            sum += a.part[(int64_t)b * a.p.E + e];
            count += a.count[(int64_t)b * a.p.E + e];
        }
        sums[e] = sum;
        counts[e] = count;
    }
    __syncthreads();
    balance_finish<1024>(a.p, sums, counts, rows, part);
}

// Rows of a workgroup at least, and workgroups at most.
static int balance_blocks(int T)
{
    const int64_t blocks = ((int64_t)T + 127) / 128;
    return blocks < 1 ? 1 : blocks < 64 ? (int)blocks : 64;
}

size_t balance_workspace_bytes(int T, int E)
{
    const size_t blocks = (size_t)balance_blocks(T);
    return blocks <= 1 ? 0 : blocks * ((size_t)E * 8 + 4);
}

template <int LANES, int NV>
static hipError_t balance_run(const BalanceArgs &a, hipStream_t st)
{
    if (a.blocks <= 1) return launch_kernel((balance_kernel<LANES, NV, true>), dim3(1), dim3(kBalanceThreads), 0, st, a);
    return launch_kernel((balance_kernel<LANES, NV, false>), dim3((unsigned)a.blocks), dim3(kBalanceThreads), 0, st, a);
}

hipError_t balance_launch(const BalanceProblem &p, void *workspace, hipStream_t st)
{
    BalanceArgs a{p, balance_blocks(p.T), 0, nullptr, nullptr, nullptr};
    a.per = (int)(((int64_t)p.T + a.blocks - 1) / a.blocks);
    if (a.blocks > 1) {
        a.part = static_cast<float *>(workspace);
        a.count = reinterpret_cast<int32_t *>(a.part + (size_t)a.blocks * p.E);
        a.open = a.count + (size_t)a.blocks * p.E;
    }
    auto *f = p.E <= 16    ? balance_run<16, 1>
              : p.E <= 32  ? balance_run<16, 2>
              : p.E <= 64  ? balance_run<16, 4>
              : p.E <= 128 ? balance_run<16, 8>
              : p.E <= 256 ? balance_run<16, 16>
              : p.E <= 512 ? balance_run<64, 8>
                           : balance_run<64, 16>;
    const hipError_t e = f(a, st);
    if (e != hipSuccess || a.blocks <= 1) return e;
    return launch_kernel(balance_join_kernel, dim3(1), dim3(1024), 0, st, a);
}

// ---- gradient ---------------------------------------------------------------------------------------------------
template <int LANES, int NV>
__global__ __launch_bounds__(256) void balance_bwd_kernel(int T, int E, const float *logits, const int32_t *counts, const int32_t *rows,
                                                          float coefficient, const float *dloss, float *dlogits, int accumulate)
{
    const int l = threadIdx.x % LANES;
    const int64_t t = (int64_t)block_number() * (256 / LANES) + threadIdx.x / LANES;
    const bool here = t < T;
    float f[NV], p[NV], total = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        f[i] = e < E ? (float)counts[e] : 0.f;
        total += f[i];
    }
    total = group_sum<LANES>(total);
    const int n = *rows;
    const float scale = coefficient * (dloss ? *dloss : 1.f) * (float)E / (float)max(n, 1);
    balance_row<LANES, NV>(here ? logits + t * E : nullptr, E, l, p);
    float mean = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        f[i] = total > 0.f ? f[i] / total : 0.f;
        mean += p[i] * f[i];
    }
    mean = group_sum<LANES>(mean);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        if (!here || e >= E) continue;
        const float d = scale * (p[i] * (f[i] - mean));
        float *at = dlogits + t * E + e;
        *at = accumulate ? *at + d : d;
    }
}

template <int LANES, int NV>
static hipError_t balance_bwd_run(int T, int E, const float *logits, const int32_t *counts, const int32_t *rows, float coefficient,
                                  const float *dloss, float *dlogits, bool accumulate, hipStream_t st)
{
    return launch_kernel((balance_bwd_kernel<LANES, NV>), many_blocks(((int64_t)T + 256 / LANES - 1) / (256 / LANES), 256), dim3(256), 0, st, T, E,
                         logits, counts, rows, coefficient, dloss, dlogits, accumulate);
}

hipError_t balance_bwd_launch(int T, int E, const float *logits, const int32_t *counts, const int32_t *rows, float coefficient, const float *dloss,
                              float *dlogits, bool accumulate, hipStream_t st)
{
    auto *f = E <= 16    ? balance_bwd_run<16, 1>
              : E <= 32  ? balance_bwd_run<16, 2>
              : E <= 64  ? balance_bwd_run<16, 4>
              : E <= 128 ? balance_bwd_run<16, 8>
              : E <= 256 ? balance_bwd_run<16, 16>
              : E <= 512 ? balance_bwd_run<64, 8>
                         : balance_bwd_run<64, 16>;
    return f(T, E, logits, counts, rows, coefficient, dloss, dlogits, accumulate, st);
}

}  // namespace polydl
