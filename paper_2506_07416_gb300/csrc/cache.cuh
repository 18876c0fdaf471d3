// The 4-bit K/V cache on the device: e2m1 codes (sign, two exponent bits, one
// mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with one e4m3 scale for every 16
// channels of a row. A code's value times its scale has at most six significant
// bits and lies in [2^-10, 2688] (or is 0), so both fit f16 and their product is
// exact there.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "cache_index.h"
#include "internal.h"
#include "ptx.cuh"

namespace lvs {

__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 bits_h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }

// Values of the byte B of w: two codes, the low four bits first.
template <int B>
__device__ __forceinline__ __half2 e2m1x2_value(uint32_t w)
{
    return __half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(w >> (8 * B)), __NV_E2M1));
}

// Values of two e4m3 codes in the low 16 bits of w.
__device__ __forceinline__ __half2 e4m3x2_value(uint32_t w)
{
    return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3));
}

// 16 bytes from global to shared memory, asynchronously; zeros where !valid.
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, bool valid)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

}  // namespace lvs
