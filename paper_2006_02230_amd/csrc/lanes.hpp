// Reductions over the 64 lanes of a wave in registers (data parallel primitives: six shifted operations, the result in
// lane 63), and loads of eight 16-bit values from any even address.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace polydl {

typedef uint32_t lanes_u32x4 __attribute__((ext_vector_type(4)));

// `x` of the lane CTRL names, `id` where there is none
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_of(int id, int x)
{
    return __builtin_amdgcn_update_dpp(id, x, CTRL, ROWS, 0xf, false);
}
// row_shr:1, 2, 4, 8 sum each row of 16 into its last lane, row_bcast:15 and row_bcast:31 join the rows
#define POLYDL_DPP_STEPS(STEP) STEP(0x111, 0xf) STEP(0x112, 0xf) STEP(0x114, 0xf) STEP(0x118, 0xf) STEP(0x142, 0xa) STEP(0x143, 0xc)

__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
#define STEP(C, R) { const uint32_t o = (uint32_t)dpp_of<C, R>(0, (int)x); x = o > x ? o : x; }
    POLYDL_DPP_STEPS(STEP)
#undef STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ float wave_sum(float x)
{
#define STEP(C, R) x += __builtin_bit_cast(float, dpp_of<C, R>(0, __builtin_bit_cast(int, x)));
    POLYDL_DPP_STEPS(STEP)
#undef STEP
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
// sum over this and the lower lanes (lane 63: all)
__device__ __forceinline__ int wave_prefix(int x)
{
#define STEP(C, R) x += dpp_of<C, R>(0, x);
    POLYDL_DPP_STEPS(STEP)
#undef STEP
    return x;
}
// A value that is the same for all lanes, into scalar registers: what a load or a division gives is in vector registers, and what is
// computed from it would follow.
__device__ __forceinline__ int wave_value(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t wave_value(uint64_t x)
{
    return (uint64_t)(uint32_t)wave_value((int)(uint32_t)(x >> 32)) << 32 | (uint32_t)wave_value((int)(uint32_t)x);
}
__device__ __forceinline__ int lane_of(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Over LANES neighbouring lanes, 16 (a row: four rotations) or 64, the result in all of them.
#define POLYDL_ROW_STEPS(STEP) STEP(0x128) STEP(0x124) STEP(0x122) STEP(0x121)
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t x)
{
    if constexpr (LANES == 64) return wave_max(x);
#define STEP(C) { const uint32_t o = (uint32_t)dpp_of<C, 0xf>(0, (int)x); x = o > x ? o : x; }
    POLYDL_ROW_STEPS(STEP)
#undef STEP
    return x;
}
template <int LANES>
__device__ __forceinline__ uint32_t group_min(uint32_t x) { return ~group_max<LANES>(~x); }
template <int LANES>
__device__ __forceinline__ float group_sum(float x)
{
    if constexpr (LANES == 64) return wave_sum(x);
#define STEP(C) x += __builtin_bit_cast(float, dpp_of<C, 0xf>(0, __builtin_bit_cast(int, x)));
    POLYDL_ROW_STEPS(STEP)
#undef STEP
    return x;
}
// over a row of 16
__device__ __forceinline__ uint32_t row_total(uint32_t x)
{
#define STEP(C) x += (uint32_t)dpp_of<C, 0xf>(0, (int)x);
    POLYDL_ROW_STEPS(STEP)
#undef STEP
    return x;
}

// bfloat16 bits <-> float.  To bfloat16: round to nearest, ties to even; the compiler's conversion is one instruction a pair.
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
typedef __bf16 lanes_bf16x2 __attribute__((ext_vector_type(2)));
typedef float lanes_f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    const lanes_f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, lanes_bf16x2));
}
__device__ __forceinline__ uint16_t bf16_one(float x) { return (uint16_t)bf16_pair(x, 0.f); }

// Eight 16-bit values as four words.  The address need only be even: unaligned wide loads are one instruction here, and
// cost another cache line at most.
struct __attribute__((packed, aligned(2))) Unit8 { lanes_u32x4 v; };
__device__ __forceinline__ lanes_u32x4 load_unit8(const uint16_t *p) { return reinterpret_cast<const Unit8 *>(p)->v; }
__device__ __forceinline__ void store_unit8(uint16_t *p, lanes_u32x4 v) { reinterpret_cast<Unit8 *>(p)->v = v; }
// four of them, zeros behind
struct __attribute__((packed, aligned(2))) Unit4 { uint32_t v[2]; };
__device__ __forceinline__ lanes_u32x4 load_unit4(const uint16_t *p)
{
    const Unit4 u = *reinterpret_cast<const Unit4 *>(p);
    return lanes_u32x4{u.v[0], u.v[1], 0u, 0u};
}
// The first n of them, zeros for the rest, in a row of `length` that ends n values from p on (n >= 1; more than 8: as 8).  Nothing outside
// the row is read: where n < 8 the row's last eight values are loaded and shifted.  (One by one they cost a load's latency each, for the whole
// wave.)  A wave without such a lane does not wait for the load here.
__device__ __forceinline__ lanes_u32x4 load_unit8(const uint16_t *p, int n, int length)
{
    if (n >= 8) return load_unit8(p);
    lanes_u32x4 v = {0u, 0u, 0u, 0u};
    if (length < 8) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        return v;
    }
    const int past = 8 - n;
    v = load_unit8(p - past);
    v = past & 4 ? lanes_u32x4{v[2], v[3], 0u, 0u} : v;
    v = past & 2 ? lanes_u32x4{v[1], v[2], v[3], 0u} : v;
    return past & 1 ? lanes_u32x4{__builtin_amdgcn_alignbit(v[1], v[0], 16u), __builtin_amdgcn_alignbit(v[2], v[1], 16u),
                                  __builtin_amdgcn_alignbit(v[3], v[2], 16u), v[3] >> 16}
                    : v;
}
__device__ __forceinline__ void store_unit8(uint16_t *p, lanes_u32x4 v, int n)
{
    if (n >= 8) { store_unit8(p, v); return; }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) p[i] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
}

}  // namespace polydl
