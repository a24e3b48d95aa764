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

// The lane's NV logits of a row (NULL: none, all masked)
template <int LANES, int NV>
__device__ __forceinline__ void balance_load(const float *row, int E, int l, float (&v)[NV])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        v[i] = row && e < E ? row[e] : -INFINITY;
    }
}
// Logits to probabilities, zeros where no expert is open: then false.
template <int LANES, int NV>
__device__ __forceinline__ bool balance_row(float (&p)[NV])
{
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
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

struct BalanceArgs {
    BalanceProblem p;
    int blocks, per;                // workgroups, rows of one
    float *part;                    // [blocks][E]: sums of probabilities
    int32_t *count;                 // [blocks][E+1]: choices, open rows
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
    // in a wave, then the waves in their order
#pragma unroll
    for (int x = 1; x < 64; x += x) {
        total += __shfl_xor(total, x);
        product += __shfl_xor(product, x);
    }
    if ((threadIdx.x & 63) == 0) {
        part[threadIdx.x >> 6] = total;
        part[THREADS / 64 + (threadIdx.x >> 6)] = product;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < THREADS / 64; ++w) {
        total += part[w];
        product += part[THREADS / 64 + w];
    }
    // (NaN shares make the loss NaN without choices too)
    *p.loss = (float)((double)p.E * (total > 0.0 ? product / total : product));
    *p.rows = rows;
}

// ONE: the workgroup is the only one, and the loss is formed here too.
template <int LANES, int NV, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void balance_kernel(BalanceArgs a)
{
    constexpr int kExperts = LANES * NV, kWaves = THREADS / 64, kRows = THREADS / LANES;
    __shared__ float sums[kWaves][kExperts];
    __shared__ int counts[kExperts], open[kWaves];
    __shared__ double part[ONE ? 2 * kWaves : 1];
    const BalanceProblem &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = tid % LANES, b = (int)blockIdx.x;
    const int64_t t0 = (int64_t)b * a.per, t1 = min((int64_t)p.T, t0 + a.per), i0 = t0 * p.k + tid, i1 = t1 * p.k;
    // the next rows are on their way while these are worked on, the first choices meanwhile, too
    const auto load = [&](int64_t t, float (&v)[NV]) {
        const int64_t at = t + tid / LANES;
        balance_load<LANES, NV>(at < t1 ? p.logits + at * p.E : nullptr, p.E, l, v);
    };
    float acc[NV], v[NV], next[NV];
    load(t0, v);
    const int first = i0 < i1 ? p.ids[i0] : -1;
    for (int e = tid; e < kExperts; e += THREADS) counts[e] = 0;
    int rows = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) acc[i] = 0.f;
    for (int64_t t = t0; t < t1; t += kRows) {
        load(t + kRows, next);
        const bool is = balance_row<LANES, NV>(v);
        rows += is && l == 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) { acc[i] += v[i]; v[i] = next[i]; }
    }
    __syncthreads();                    // counts
    if ((unsigned)first < (unsigned)p.E) atomicAdd(&counts[first], 1);
    for (int64_t i = i0 + THREADS; i < i1; i += THREADS) {
        const int id = p.ids[i];
        if ((unsigned)id < (unsigned)p.E) atomicAdd(&counts[id], 1);
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
    for (int w = 0; w < kWaves; ++w) rows += open[w];
    for (int e = tid; e < p.E; e += THREADS) {
        float sum = sums[0][e];
        for (int w = 1; w < kWaves; ++w) sum += sums[w][e];
        if constexpr (ONE) {
            sums[0][e] = sum;
        } else {
            a.part[(int64_t)b * p.E + e] = sum;
            a.count[(int64_t)b * (p.E + 1) + e] = counts[e];
        }
    }
    if constexpr (ONE) {
        __syncthreads();
        balance_finish<THREADS>(p, sums[0], counts, rows, part);
    } else if (tid == 0) {
        a.count[(int64_t)b * (p.E + 1) + p.E] = rows;
    }
}

// The workgroups' sums.  A thread takes an expert of every SLICES-th workgroup; the slices meet in LDS in their order.
template <int SLICES>
__global__ __launch_bounds__(1024) void balance_join_kernel(BalanceArgs a)
{
    constexpr int kAcross = 1024 / SLICES;
    __shared__ float sums[SLICES][kAcross + 1];
    __shared__ int counts[SLICES][kAcross + 1];
    __shared__ double part[2 * 16];
    const int e = threadIdx.x % kAcross, slice = threadIdx.x / kAcross, E = a.p.E;
    float sum = 0.f;
    int count = 0, rows = 0;
    for (int b = (int)(threadIdx.x & 63); b < a.blocks; b += 64) rows += a.count[(int64_t)b * (E + 1) + E];
    // sixteen workgroups' at a time are on their way: they come from other dies, 2 us each time (four at a time: 16384 x 128 19.6 us)
    constexpr int kHeld = 16;
    for (int b0 = slice; b0 < a.blocks; b0 += SLICES * kHeld) {
        float s[kHeld];
        int c[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int b = b0 + i * SLICES;
            const bool there = e < E && b < a.blocks;
            s[i] = there ? a.part[(int64_t)b * E + e] : 0.f;
            c[i] = there ? a.count[(int64_t)b * (E + 1) + e] : 0;
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            sum += s[i];
            count += c[i];
        }
    }
    rows = lane_of(wave_prefix(rows), 63);
    sums[slice][e] = sum;
    counts[slice][e] = count;
    __syncthreads();
    if (slice == 0) {
        for (int s = 1; s < SLICES; ++s) {
            sum += sums[s][e];
            count += counts[s][e];
        }
        sums[0][e] = sum;
        counts[0][e] = count;
    }
    __syncthreads();
    balance_finish<1024>(a.p, sums[0], counts[0], rows, part);
}

// One workgroup takes up to 256 rows (a second launch costs as much as four rounds of rows); more rows go to workgroups of one round, or of two where a wave takes a
// row, but at most 256, or 128: one workgroup adds their sums up (16384 x 128: 13.7 us with 128 or 256 workgroups, 17.7 with 64; 100000 x 128: 41, 31 and 69; 8192 x 1000: 43
// and 49 with 128 and 256; 300 x 1000 16 us, with 64 rows a workgroup 29).
constexpr int kBalanceRows = 256;
static int balance_blocks(int T, int E)
{
    const bool wide = E > 256;
    const int64_t rows = wide ? 16 : 64, blocks = T <= (wide ? 16 : kBalanceRows) ? 1 : ((int64_t)T + rows - 1) / rows;
    const int64_t most = wide ? 128 : 256;
    return (int)(blocks < most ? blocks : most);
}

size_t balance_workspace_bytes(int T, int E)
{
    const size_t blocks = (size_t)balance_blocks(T, E);
    return blocks <= 1 ? 0 : blocks * ((size_t)E * 8 + 4);
}

template <int LANES, int NV>
static hipError_t balance_run(const BalanceArgs &a, hipStream_t st)
{
    constexpr int threads = LANES == 64 ? 512 : 1024;        // (more waves' sums of up to 1024 experts would not fit in LDS)
    if (a.blocks <= 1) return launch_kernel((balance_kernel<LANES, NV, threads, true>), dim3(1), dim3(threads), 0, st, a);
    return launch_kernel((balance_kernel<LANES, NV, threads, false>), dim3((unsigned)a.blocks), dim3(threads), 0, st, a);
}

hipError_t balance_launch(const BalanceProblem &p, void *workspace, hipStream_t st)
{
    BalanceArgs a{p, balance_blocks(p.T, p.E), 0, nullptr, nullptr};
    a.per = (int)(((int64_t)p.T + a.blocks - 1) / a.blocks);
    if (a.blocks > 1) {
        a.part = static_cast<float *>(workspace);
        a.count = reinterpret_cast<int32_t *>(a.part + (size_t)a.blocks * p.E);
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
    auto *join = p.E <= 32    ? balance_join_kernel<32>
                 : p.E <= 64  ? balance_join_kernel<16>
                 : p.E <= 128 ? balance_join_kernel<8>
                 : p.E <= 256 ? balance_join_kernel<4>
                 : p.E <= 512 ? balance_join_kernel<2>
                              : balance_join_kernel<1>;
    return launch_kernel(join, dim3(1), dim3(1024), 0, st, a);
}

// ---- gradient ---------------------------------------------------------------------------------------------------
// Bound: a launch and its first loads (16384 x 64: 5.2 us, 8 MB).
template <int LANES, int NV>
__global__ __launch_bounds__(256) void balance_bwd_kernel(int T, int E, const float *logits, const int32_t *counts, const int32_t *rows,
                                                          float coefficient, const float *dloss, float *dlogits, int accumulate)
{
    const int l = threadIdx.x % LANES;
    const int64_t t = (int64_t)block_number() * (256 / LANES) + threadIdx.x / LANES;
    const bool here = t < T;
    // A share less 1/E in f's place, which changes nothing in the formula: probabilities add up to 1.  Of a router that uses its experts nearly evenly
    // little would be left of f - sum p f; and nothing but roundings of one that uses them evenly, where this is zero.
    float f[NV], p[NV];
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        total += e < E ? (double)counts[e] : 0.0;
    }
#pragma unroll
    for (int x = 1; x < LANES; x += x) total += __shfl_xor(total, x);
    const double part = total > 0.0 ? 1.0 / (total * E) : 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        f[i] = e < E ? (float)(((double)counts[e] * E - total) * part) : 0.f;
    }
    const int n = *rows;
    const float scale = coefficient * (dloss ? *dloss : 1.f) * (float)E / (float)max(n, 1);
    balance_load<LANES, NV>(here ? logits + t * E : nullptr, E, l, p);
    balance_row<LANES, NV>(p);
    float mean = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) mean += p[i] * f[i];
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
