// Loads from memory straight into LDS, the waits for them, and kernels with more LDS than the default window.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <atomic>

namespace polydl {

typedef int gg_i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kFarOffset = 0xfffffff0u;        // out of range of every descriptor here
constexpr uint64_t kFarRecords = 0xffffffe0ull;     // so that no sum of an offset in range and a load's width reaches 2^32

// A raw buffer descriptor of `bytes` bytes from base (none if negative), in operations of 32 bits: there are no scalar comparisons of 64.
__device__ __forceinline__ gg_i32x4 gg_rsrc(uint64_t base, int64_t bytes)
{
    const int high = (int)(bytes >> 32);
    const uint32_t low = (uint32_t)bytes, most = (uint32_t)kFarRecords;
    const uint32_t n = high < 0 ? 0u : high > 0 ? most : low < most ? low : most;
    return gg_i32x4{(int)(uint32_t)base, (int)((uint32_t)(base >> 32) & 0xffffu), (int)n, 0x00020000};
}
// Sixteen bytes a lane into LDS at `lds` + 16 * lane; not waited for.  As assembly, because the compiler puts a wait for every such
// load before each transposing LDS read, whichever buffer it reads (measured with stages of 32 at 16384 x 4096 x 2048: dX 1112
// against 902, dW 865 against 512 TFLOP/s).  No register is written; the waits are gg_wait()'s.  m0, where the
// load's LDS address is, is an operand that the compiler sets and knows of; the wait states are those that a descriptor or m0 just written needs.
__device__ __forceinline__ void gg_dma(gg_i32x4 rsrc, uint32_t lds, uint32_t off)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(lds), "v"(off), "s"(rsrc) : "memory");
#else
    (void)rsrc; (void)lds; (void)off;
#endif
}
// four bytes a lane, into LDS at `lds` + 4 * lane
__device__ __forceinline__ void gg_dma_word(gg_i32x4 rsrc, uint32_t lds, uint32_t off)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"{m0}"(lds), "v"(off), "s"(rsrc) : "memory");
#else
    (void)rsrc; (void)lds; (void)off;
#endif
}
// where a pointer into the workgroup's LDS points
__device__ __forceinline__ uint32_t gg_lds_offset(const char *lds)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)lds;
#else
    (void)lds;
    return 0;
#endif
}
// s_waitcnt of the gfx9 encoding: vmcnt N (bits 3:0, 15:14), lgkmcnt 0 (11:8), expcnt left alone
template <int N>
__device__ __forceinline__ void gg_wait()
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4 << 14) | 0x70);
#endif
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

}  // namespace polydl
