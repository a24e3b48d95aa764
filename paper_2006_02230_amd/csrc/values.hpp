// Units of eight values of a row, float32 or bfloat16 in memory, float32 in registers.  Rows may begin at any element: wide accesses at any
// even address are one instruction here.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include "lanes.hpp"

namespace polydl {

typedef float values_f32x4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(4))) Floats4Any { values_f32x4 v; };

template <bool F32>
struct Values {
    using T = std::conditional_t<F32, float, uint16_t>;

    // Values col .. col + 7 of a row of `length`, zeros behind its end (col < length)
    static __device__ __forceinline__ void load(const T *row, int col, int length, float (&v)[8])
    {
        const int n = length - col;
        if constexpr (F32) {
            const float *p = row + col;
            if (n >= 8) {
                const values_f32x4 a = reinterpret_cast<const Floats4Any *>(p)[0].v, b = reinterpret_cast<const Floats4Any *>(p)[1].v;
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
            }
        } else {
            const lanes_u32x4 u = load_unit8(row + col, n, length);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_lo(u[i]); v[2 * i + 1] = bf16_hi(u[i]); }
        }
    }
    static __device__ __forceinline__ void store(T *row, int col, int length, const float (&v)[8])
    {
        const int n = length - col;
        if constexpr (F32) {
            float *p = row + col;
            if (n >= 8) {
                reinterpret_cast<Floats4Any *>(p)[0].v = values_f32x4{v[0], v[1], v[2], v[3]};
                reinterpret_cast<Floats4Any *>(p)[1].v = values_f32x4{v[4], v[5], v[6], v[7]};
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (i < n) p[i] = v[i];
            }
        } else {
            lanes_u32x4 u;
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
            store_unit8(row + col, u, n);
        }
    }
};

}  // namespace polydl
