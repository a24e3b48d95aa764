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

    // what a load gives, before it is waited for
    struct Raw { std::conditional_t<F32, values_f32x4, lanes_u32x4> v[F32 ? 2 : 1]; };
    static __device__ __forceinline__ Raw load_raw(const T *row, int col, int length)
    {
        const int n = length - col;
        Raw r;
        if constexpr (F32) {
            const float *p = row + col;
            if (n >= 8) {
                r.v[0] = reinterpret_cast<const Floats4Any *>(p)[0].v;
                r.v[1] = reinterpret_cast<const Floats4Any *>(p)[1].v;
            } else {
                r.v[0] = r.v[1] = values_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (i < n) r.v[i >> 2][i & 3] = p[i];
            }
        } else {
            r.v[0] = load_unit8(row + col, n, length);
        }
        return r;
    }
    static __device__ __forceinline__ void convert(const Raw &r, float (&v)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (F32) {
                v[i] = r.v[0][i];
                v[4 + i] = r.v[1][i];
            } else {
                v[2 * i] = bf16_lo(r.v[0][i]);
                v[2 * i + 1] = bf16_hi(r.v[0][i]);
            }
        }
    }
    // Values col .. col + 7 of a row of `length`, zeros behind its end (col < length)
    static __device__ __forceinline__ void load(const T *row, int col, int length, float (&v)[8])
    {
        convert(load_raw(row, col, length), v);
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
