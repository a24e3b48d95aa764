// The router of a layer of experts, its plan and its gradient, and the weighted sum over a token's experts.
//
// route: of each token's E logits the k largest (ties: the lowest index; logits of -infinity never), their softmax
// weights, and the slots sorted by expert that the grouped products work on.  16 lanes take a token of up to 256 experts, four tokens a
// wave, and a wave one of more; a lane holds E/16 or E/64 logits as ordered unsigned keys.  A round is a maximum over the lanes, the lowest
// index that has it, and that key's removal, so the order does not depend on rounding.  64 tokens make a workgroup; each
// expert's tokens there are a mask of 64 bits in LDS, set with atomic ORs: a slot's place inside its expert is the number of
// bits below its own, the same in every run.
// Bound: instruction issue and latency.  The logits of 16384 tokens and 128 experts are 8 MB, 1.5 us of HBM; a round of four tokens is 50
// instructions of which 20 wait for one another.  16384 tokens, 128 experts, 8 choices: 7.6 us (13.6 with a wave to a token).
#include <hip/hip_runtime.h>
#include <math.h>
#include "blocks.hpp"
#include "experts.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace polydl {

// A float as an unsigned key of the same order; 0 for -infinity (a masked logit is never taken), all ones for NaN (taken
// first: a broken logit shows in the weights rather than being dropped).  Adding zero makes -0 the +0 that it is equal to.
__device__ __forceinline__ uint32_t route_key(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.f);
    const uint32_t key = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
    return v != v ? 0xffffffffu : v == -INFINITY ? 0u : key;
}
__device__ __forceinline__ float route_value(uint32_t key)
{
    return __builtin_bit_cast(float, key >> 31 ? key ^ 0x80000000u : ~key);
}

// Lane l of a token's LANES: choices l and l + LANES, -1 and 0 where there is none.
template <int LANES>
struct RouteRow {
    static constexpr int kHeld = LANES < kRouteMaxChoices ? kRouteMaxChoices / LANES : 1;
    int id[kHeld];
    float w[kHeld];
};

// `row`: the token's logits, or NULL for lanes without a token.
template <int LANES, int NV>
__device__ __forceinline__ RouteRow<LANES> route_row(const float *row, int E, int k, bool renorm, int l)
{
    using Row = RouteRow<LANES>;
    float v[NV];
    uint32_t key[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        v[i] = row && e < E ? row[e] : -INFINITY;
        key[i] = route_key(v[i]);
    }
    Row r;
    float own[Row::kHeld], best = 0.f;
#pragma unroll
    for (int h = 0; h < Row::kHeld; ++h) { r.id[h] = -1; r.w[h] = own[h] = 0.f; }
    for (int j = 0; j < k; ++j) {
        uint32_t m = key[0];
#pragma unroll
        for (int i = 1; i < NV; ++i) m = key[i] > m ? key[i] : m;
        m = group_max<LANES>(m);
        if (!__any(m != 0u)) break;                      // nothing left that is not masked
        uint32_t e = 0xffffffffu;
#pragma unroll
        for (int i = NV - 1; i >= 0; --i) e = key[i] == m ? (uint32_t)(i * LANES + l) : e;
        e = group_min<LANES>(e);
#pragma unroll
        for (int i = 0; i < NV; ++i) key[i] = (uint32_t)(i * LANES + l) == e ? 0u : key[i];
        const float x = route_value(m);
        if (j == 0) best = x;
#pragma unroll
        for (int h = 0; h < Row::kHeld; ++h)
            if (h * LANES + l == j && m != 0u) { r.id[h] = (int)e; own[h] = x; }
    }
    const bool any = group_max<LANES>((uint32_t)(r.id[0] + 1)) != 0u;      // some logit is not masked
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < Row::kHeld; ++h) {
        own[h] = r.id[h] >= 0 ? expf(own[h] - best) : 0.f;
        sum += own[h];
    }
    if (!renorm) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) sum += any ? expf(v[i] - best) : 0.f;
    }
    sum = group_sum<LANES>(sum);
#pragma unroll
    for (int h = 0; h < Row::kHeld; ++h) r.w[h] = r.id[h] >= 0 ? own[h] / sum : 0.f;
    return r;
}

struct RouteArgs {
    RouteProblem p;
    uint8_t *hist;          // [E][pitch]: tokens of each workgroup that chose expert e (at most 64)
    int32_t *before;        // [E][blocks]: tokens of the workgroups before (SCANNED), and
    int32_t *total;         // [E]
    int blocks, pitch;
};

// Exclusive sums of count[0 .. E) over the workgroup, into base[0 .. E], base[E] the total.  `part` holds a word a wave.
template <int THREADS>
__device__ __forceinline__ void route_sums(const int *count, int *base, int *part, int E, int tid)
{
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += THREADS) {
        const int e = e0 + tid, c = e < E ? count[e] : 0;
        const int incl = wave_prefix(c);
        __syncthreads();
        if ((tid & 63) == 63) part[tid >> 6] = incl;
        __syncthreads();
        int at = carry, all = carry;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < (tid >> 6)) at += part[w];
            all += part[w];
        }
        if (e < E) base[e] = at + incl - c;
        carry = all;
    }
    if (tid == 0) base[E] = carry;
    __syncthreads();
}

// The workgroup's slots.  base[e]: the first slot its tokens take of expert e; masks: two words an expert.
template <int THREADS>
__device__ __forceinline__ void route_place(const RouteProblem &p, const int *ids, const int *base, const uint32_t *masks, int t0,
                                            int n, int tid)
{
    for (int i = tid; i < n; i += THREADS) {
        const int t = (int)((unsigned)i / (unsigned)p.k), id = ids[i];
        int slot = -1;
        if (id >= 0) {
            const uint32_t lo = masks[2 * id], hi = masks[2 * id + 1];
            const uint32_t below = (1u << (t & 31)) - 1u;
            slot = base[id] + (t < 32 ? __builtin_popcount(lo & below) : __builtin_popcount(lo) + __builtin_popcount(hi & below));
            p.tokens[slot] = t0 + t;
        }
        p.slots[(size_t)t0 * p.k + i] = slot;
    }
}

// Choices of 64 tokens.  ONE: they are all there are, and the plan is made here too; else the counts go to `hist`.
template <int LANES, int NV, bool ONE>
__global__ __launch_bounds__(1024) void route_choose_kernel(RouteArgs a)
{
    __shared__ uint32_t masks[2 * LANES * NV];
    __shared__ int count[ONE ? LANES * NV : 1], base[ONE ? LANES * NV + 1 : 1], part[16], ids[ONE ? kRouteTokens * kRouteMaxChoices : 1];
    const RouteProblem &p = a.p;
    const int tid = threadIdx.x, l = tid % LANES, b = (int)block_number();
    if (!ONE && b >= a.blocks) return;
    const int t0 = b * kRouteTokens, nt = min(kRouteTokens, p.T - t0);
    for (int i = tid; i < 2 * p.E; i += 1024) masks[i] = 0u;
    __syncthreads();
    for (int t = tid / LANES; t < kRouteTokens; t += 1024 / LANES) {
        const auto r = route_row<LANES, NV>(t < nt ? p.logits + (size_t)(t0 + t) * p.E : nullptr, p.E, p.k, p.renorm, l);
#pragma unroll
        for (int h = 0; h < RouteRow<LANES>::kHeld; ++h) {
            const int j = h * LANES + l;
            if (t >= nt || j >= p.k) continue;
            const size_t at = (size_t)(t0 + t) * p.k + j;
            p.ids[at] = r.id[h];
            p.weights[at] = r.w[h];
            if (ONE) ids[t * p.k + j] = r.id[h];
            if (r.id[h] >= 0) atomicOr(&masks[2 * r.id[h] + (t >> 5)], 1u << (t & 31));
        }
    }
    __syncthreads();
    if constexpr (ONE) {
        for (int e = tid; e < p.E; e += 1024) count[e] = __builtin_popcount(masks[2 * e]) + __builtin_popcount(masks[2 * e + 1]);
        __syncthreads();
        route_sums<1024>(count, base, part, p.E, tid);
        for (int e = tid; e <= p.E; e += 1024) p.offsets[e] = base[e];
        route_place<1024>(p, ids, base, masks, 0, nt * p.k, tid);
        for (int s = base[p.E] + tid; s < nt * p.k; s += 1024) p.tokens[s] = -1;
    } else {
        const int pad = b == a.blocks - 1 ? a.pitch - a.blocks : 0;   // the bytes behind a row's end are zero too
        for (int e = tid; e < p.E; e += 1024) {
            a.hist[(size_t)e * a.pitch + b] = (uint8_t)(__builtin_popcount(masks[2 * e]) + __builtin_popcount(masks[2 * e + 1]));
        }
        for (int i = tid; i < p.E * pad; i += 1024) {
            const int e = (int)((unsigned)i / (unsigned)pad);
            a.hist[(size_t)e * a.pitch + a.blocks + i - e * pad] = 0;
        }
    }
}

// One wave an expert: the sums of its counts before each workgroup.
__global__ __launch_bounds__(256) void route_scan_kernel(RouteArgs a)
{
    const int e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (e >= a.p.E) return;
    const uint8_t *h = a.hist + (size_t)e * a.pitch;
    int32_t *out = a.before + (size_t)e * a.blocks;
    int carry = 0;
    for (int b0 = 0; b0 < a.blocks; b0 += 64) {
        const int b = b0 + lane, c = b < a.blocks ? h[b] : 0;
        const int incl = wave_prefix(c);
        if (b < a.blocks) out[b] = carry + incl - c;
        carry += lane_of(incl, 63);
    }
    if (lane == 0) a.total[e] = carry;
}

// Slots of 64 tokens.  SCANNED: the sums are there; else every workgroup adds the counts of all of them up, 16 bytes a load, several experts' on
// their way (one expert a wave at a time, four bytes a load: 16384 tokens, 128 experts 6.5 us against 4.8; 4096 tokens, 1000 experts 29 against 12).
struct __attribute__((packed, aligned(4))) RouteCounts { uint32_t w[4]; };
template <bool SCANNED>
__global__ __launch_bounds__(1024) void route_place_kernel(RouteArgs a)
{
    __shared__ uint32_t masks[2 * kRouteMaxExperts];
    __shared__ int count[kRouteMaxExperts], base[kRouteMaxExperts + 1], ahead[kRouteMaxExperts], part[16];
    __shared__ int ids[kRouteTokens * kRouteMaxChoices];
    const RouteProblem &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = p.E, b = (int)block_number();
    if (b >= a.blocks) return;
    const int t0 = b * kRouteTokens, n = min(kRouteTokens, p.T - t0) * p.k;
    int held[kRouteTokens * kRouteMaxChoices / 1024];       // on their way while the counts are added up
#pragma unroll
    for (int h = 0; h < kRouteTokens * kRouteMaxChoices / 1024; ++h) held[h] = h * 1024 + tid < n ? p.ids[(size_t)t0 * p.k + h * 1024 + tid] : -1;
    for (int i = tid; i < 2 * E; i += 1024) masks[i] = 0u;
    if constexpr (SCANNED) {
        for (int e = tid; e < E; e += 1024) {
            count[e] = a.total[e];
            ahead[e] = a.before[(size_t)e * a.blocks + b];
        }
    } else {
        // 16 lanes an expert, two experts a lane at a time
        // (what is loaded behind a row's end is the next row's, or the workspace's that follows: not counted)
        const int words = a.pitch / 4, units = (words + 3) / 4, l = lane & 15;
        for (int e0 = wave * 4 + (lane >> 4); e0 < E; e0 += 128) {
            uint32_t all[2] = {0u, 0u}, less[2] = {0u, 0u};
            for (int i = l; i < units; i += 16) {
                RouteCounts w[2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    w[u] = reinterpret_cast<const RouteCounts *>(a.hist + (size_t)min(e0 + u * 64, E - 1) * a.pitch)[i];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t four = i * 4 + q < words ? w[u].w[q] : 0u;
                        all[u] = __builtin_amdgcn_sad_u8(four, 0u, all[u]);
                        const int left = b - (i * 4 + q) * 4;                       // how many of its four are before this one's
                        const uint32_t keep = left <= 0 ? 0u : left >= 4 ? 0xffffffffu : (1u << (8 * left)) - 1u;
                        less[u] = __builtin_amdgcn_sad_u8(four & keep, 0u, less[u]);
                    }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t total = row_total(all[u]), part_of = row_total(less[u]);
                if (l == 0 && e0 + u * 64 < E) { count[e0 + u * 64] = (int)total; ahead[e0 + u * 64] = (int)part_of; }
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < kRouteTokens * kRouteMaxChoices / 1024; ++h) {
        const int i = h * 1024 + tid;
        if (i >= n) continue;
        const int t = (int)((unsigned)i / (unsigned)p.k);
        ids[i] = held[h];
        if (held[h] >= 0) atomicOr(&masks[2 * held[h] + (t >> 5)], 1u << (t & 31));
    }
    __syncthreads();
    route_sums<1024>(count, base, part, E, tid);
    if (b == 0) {
        for (int e = tid; e <= E; e += 1024) p.offsets[e] = base[e];
    }
    // slots that no choice took: behind the last expert's, dealt over the workgroups
    const int64_t M = (int64_t)p.T * p.k;
    for (int64_t s = base[E] + (int64_t)b * 1024 + tid; s < M; s += (int64_t)a.blocks * 1024) p.tokens[s] = -1;
    __syncthreads();
    for (int e = tid; e < E; e += 1024) base[e] += ahead[e];
    __syncthreads();
    route_place<1024>(p, ids, base, masks, t0, n, tid);
}

static int route_blocks(int T) { return (int)(((int64_t)T + kRouteTokens - 1) / kRouteTokens); }

size_t route_workspace_bytes(int T, int E)
{
    const size_t blocks = (size_t)route_blocks(T), pitch = (blocks + 3) & ~(size_t)3;
    return blocks <= 1 ? 0 : (((size_t)E * pitch + 255) & ~(size_t)255) + ((size_t)E * blocks + E) * sizeof(int32_t);
}

// Every workgroup reading all counts saves the scan's launch; its traffic grows with the square of the workgroups.
constexpr int64_t kRouteRereadBytes = 32ll << 20;

template <int LANES, int NV>
static hipError_t route_choose(const RouteArgs &a, hipStream_t st)
{
    if (a.blocks <= 1) return launch_kernel((route_choose_kernel<LANES, NV, true>), dim3(1), dim3(1024), 0, st, a);
    return launch_kernel((route_choose_kernel<LANES, NV, false>), many_blocks(a.blocks, 1024), dim3(1024), 0, st, a);
}

hipError_t route_launch(const RouteProblem &p, void *workspace, hipStream_t st)
{
    RouteArgs a{p, nullptr, nullptr, nullptr, route_blocks(p.T), 0};
    a.pitch = (a.blocks + 3) & ~3;
    const bool one = a.blocks <= 1;      // no tokens: offsets of zeros
    if (!one) {
        a.hist = static_cast<uint8_t *>(workspace);
        a.before = reinterpret_cast<int32_t *>(a.hist + (((size_t)p.E * a.pitch + 255) & ~(size_t)255));
        a.total = a.before + (size_t)p.E * a.blocks;
    }
    auto *choose = p.E <= 16    ? route_choose<16, 1>
                   : p.E <= 32  ? route_choose<16, 2>
                   : p.E <= 64  ? route_choose<16, 4>
                   : p.E <= 128 ? route_choose<16, 8>
                   : p.E <= 256 ? route_choose<16, 16>
                   : p.E <= 512 ? route_choose<64, 8>
                                : route_choose<64, 16>;
    hipError_t e = choose(a, st);
    if (e != hipSuccess || one) return e;
    if ((int64_t)a.blocks * a.pitch * p.E <= kRouteRereadBytes)
        return launch_kernel(route_place_kernel<false>, many_blocks(a.blocks, 1024), dim3(1024), 0, st, a);
    e = launch_kernel(route_scan_kernel, dim3((unsigned)((p.E + 3) / 4)), dim3(256), 0, st, a);
    if (e != hipSuccess) return e;
    return launch_kernel(route_place_kernel<true>, many_blocks(a.blocks, 1024), dim3(1024), 0, st, a);
}

// ---- gradient ---------------------------------------------------------------------------------------------------
// Weights from the softmax over all experts: dl_e = p_e (g_e - sum_j p_j g_j), g zero where e was not chosen; renormalised:
// the same with the weights in p's place, zero elsewhere (their logits are not read).  LANES lanes a token, as in the choice.
template <int LANES, int NV, bool RENORM>
__global__ __launch_bounds__(256) void route_bwd_kernel(int T, int E, int k, const float *logits, const int32_t *ids, const float *weights,
                                                        const float *dweights, float *dlogits)
{
    constexpr int kHeld = RouteRow<LANES>::kHeld;
    const int l = threadIdx.x % LANES, first = (threadIdx.x & 63) - l;
    const int64_t t = (int64_t)block_number() * (256 / LANES) + threadIdx.x / LANES;
    const bool here = t < T;
    int id[kHeld];
    float g[kHeld], w[kHeld], p[NV], own[NV];
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        const int j = h * LANES + l;
        id[h] = here && j < k ? ids[t * k + j] : -1;
        if ((unsigned)id[h] >= (unsigned)E) id[h] = -1;
        g[h] = id[h] >= 0 ? dweights[t * k + j] : 0.f;
        w[h] = RENORM && id[h] >= 0 ? weights[t * k + j] : 0.f;
    }
    if constexpr (!RENORM) {
        const float *row = logits + t * E;
        float v[NV];
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = i * LANES + l;
            v[i] = here && e < E ? row[e] : -INFINITY;
            const uint32_t key = route_key(v[i]);
            m = key > m ? key : m;
        }
        m = group_max<LANES>(m);
        const float best = route_value(m);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            p[i] = m ? expf(v[i] - best) : 0.f;          // a row without an open expert has no probabilities
            sum += p[i];
        }
        sum = group_sum<LANES>(sum);
#pragma unroll
        for (int i = 0; i < NV; ++i) p[i] = m ? p[i] / sum : 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) p[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) own[i] = 0.f;
    for (int j = 0; j < k; ++j) {
        int e = id[0];
        float gj = g[0], wj = w[0];
        if (kHeld > 1 && j >= LANES) { e = id[kHeld - 1]; gj = g[kHeld - 1]; wj = w[kHeld - 1]; }
        const int from = first + j % LANES;
        e = __shfl(e, from);
        gj = __shfl(gj, from);
        if (RENORM) wj = __shfl(wj, from);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * LANES + l == e) {
                own[i] += gj;
                if (RENORM) p[i] = wj;
            }
    }
    float mean = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) mean += own[i] != 0.f ? p[i] * own[i] : 0.f;
    mean = group_sum<LANES>(mean);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = i * LANES + l;
        if (here && e < E) dlogits[t * E + e] = p[i] * (own[i] - mean);
    }
}

template <int LANES, int NV>
static hipError_t route_bwd(int T, int E, int k, const float *logits, const int32_t *ids, const float *weights, const float *dweights,
                            bool renorm, float *dlogits, hipStream_t st)
{
    const dim3 grid = many_blocks(((int64_t)T + 256 / LANES - 1) / (256 / LANES), 256);
    if (renorm)
        return launch_kernel((route_bwd_kernel<LANES, NV, true>), grid, dim3(256), 0, st, T, E, k, logits, ids, weights, dweights, dlogits);
    return launch_kernel((route_bwd_kernel<LANES, NV, false>), grid, dim3(256), 0, st, T, E, k, logits, ids, weights, dweights, dlogits);
}

hipError_t route_bwd_launch(int T, int E, int k, const float *logits, const int32_t *ids, const float *weights, const float *dweights,
                            bool renorm, float *dlogits, hipStream_t st)
{
    auto *f = E <= 16    ? route_bwd<16, 1>
              : E <= 32  ? route_bwd<16, 2>
              : E <= 64  ? route_bwd<16, 4>
              : E <= 128 ? route_bwd<16, 8>
              : E <= 256 ? route_bwd<16, 16>
              : E <= 512 ? route_bwd<64, 8>
                         : route_bwd<64, 16>;
    return f(T, E, k, logits, ids, weights, dweights, renorm, dlogits, st);
}

// ---- the weighted sum over a token's experts ---------------------------------------------------------------------
// out[t] = sum_j w[t][j] y[slot[t][j]], summed in float32 in the order of j, rounded once.  Bound: HBM, every row of y
// read once.  A thread holds eight columns of a token and has four rows' loads under way.
template <bool OUT_F32>
__global__ __launch_bounds__(256) void combine_kernel(int T, int k, int M, int D, int units, int per_block, const uint16_t *y,
                                                      const int32_t *slots, const float *weights, void *out)
{
    const int tl = units >= 256 ? 0 : (int)((unsigned)threadIdx.x / (unsigned)units);
    const int c = units >= 256 ? (int)(blockIdx.y * 256 + threadIdx.x) : (int)threadIdx.x - tl * units;
    const int64_t t = (int64_t)block_number() * per_block + tl;
    if (tl >= per_block || c >= units || t >= T) return;
    const int col = c * 8, n = min(8, D - col);
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < k; j0 += 4) {
        lanes_u32x4 v[4];
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int s = j0 + j < k ? slots[t * k + j0 + j] : -1;
            const bool there = (unsigned)s < (unsigned)M;
            w[j] = !there ? 0.f : weights ? weights[t * k + j0 + j] : 1.f;
            v[j] = lanes_u32x4{0u, 0u, 0u, 0u};
            if (there) v[j] = load_unit8(y + (size_t)s * D + col, n, D);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[2 * i] += w[j] * bf16_lo(v[j][i]);
                sum[2 * i + 1] += w[j] * bf16_hi(v[j][i]);
            }
    }
    if constexpr (OUT_F32) {
        float *o = static_cast<float *>(out) + t * D + col;
        if (n == 8 && (D & 3) == 0 && ((uintptr_t)out & 15) == 0) {
            reinterpret_cast<float4 *>(o)[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            reinterpret_cast<float4 *>(o)[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) o[i] = sum[i];
        }
    } else {
        lanes_u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = bf16_pair(sum[2 * i], sum[2 * i + 1]);
        store_unit8(static_cast<uint16_t *>(out) + t * D + col, v, n);
    }
}

hipError_t combine_launch(int T, int k, int M, int D, const uint16_t *y, const int32_t *slots, const float *weights, void *out,
                          bool out_f32, hipStream_t st)
{
    const int units = (D + 7) / 8, per_block = units >= 256 ? 1 : 256 / units;
    const dim3 grid = many_blocks(((int64_t)T + per_block - 1) / per_block, 256, units >= 256 ? (unsigned)((units + 255) / 256) : 1u);
    if (out_f32)
        return launch_kernel(combine_kernel<true>, grid, dim3(256), 0, st, T, k, M, D, units, per_block, y, slots, weights, out);
    return launch_kernel(combine_kernel<false>, grid, dim3(256), 0, st, T, k, M, D, units, per_block, y, slots, weights, out);
}

// dy[slot] = w dout[t], dw[t][j] = <dout[t], y[slot]>: one wave a slot; the k waves of a token read its row of dout from the
// caches.  Bound: HBM, y read and dy written once.
__global__ __launch_bounds__(256) void combine_bwd_kernel(int64_t MT, int k, int M, int D, const uint16_t *dout, const uint16_t *y,
                                                          const int32_t *slots, const float *weights, uint16_t *dy, float *dweights)
{
    const int64_t i = (int64_t)block_number() * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (i >= MT) return;
    const int s = slots[i];
    if ((unsigned)s >= (unsigned)M) {
        if (dweights && lane == 0) dweights[i] = 0.f;
        return;
    }
    const int64_t t = (int64_t)((uint32_t)i / (uint32_t)k);
    const float w = weights ? weights[i] : 1.f;
    const uint16_t *d = dout + t * D, *yr = y + (size_t)s * D;
    uint16_t *o = dy + (size_t)s * D;
    float dot[2] = {0.f, 0.f};
#pragma unroll 2
    for (int col = lane * 8; col < D; col += 512) {
        const int n = min(8, D - col);
        const lanes_u32x4 dv = load_unit8(d + col, n, D);
        lanes_u32x4 yv = {0u, 0u, 0u, 0u}, ov;
        if (dweights) yv = load_unit8(yr + col, n, D);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float lo = bf16_lo(dv[q]), hi = bf16_hi(dv[q]);
            ov[q] = bf16_pair(w * lo, w * hi);
            dot[0] += lo * bf16_lo(yv[q]);
            dot[1] += hi * bf16_hi(yv[q]);
        }
        store_unit8(o + col, ov, n);
    }
    if (dweights) {
        const float sum = wave_sum(dot[0] + dot[1]);
        if (lane == 0) dweights[i] = sum;
    }
}

hipError_t combine_bwd_launch(int T, int k, int M, int D, const uint16_t *dout, const uint16_t *y, const int32_t *slots,
                              const float *weights, uint16_t *dy, float *dweights, hipStream_t st)
{
    const int64_t MT = (int64_t)T * k;
    return launch_kernel(combine_bwd_kernel, many_blocks((MT + 3) / 4, 256), dim3(256), 0, st, MT, k, M, D, dout, y, slots, weights, dy,
                         dweights);
}

}  // namespace polydl
