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

// Values of the eight codes of w, byte by byte. The bytes are named to the
// assembler, which then converts them in place: 50 pairs a clock and SM where
// shifting each byte down first made it 24, and building f16 from the bits by
// masks and shifts 20.
__device__ __forceinline__ void e2m1x8_value(uint32_t w, __half2 (&v)[4])
{
    uint32_t o[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = bits_h2(o[i]);
}

// Values of two e4m3 codes in the low 16 bits of w.
__device__ __forceinline__ __half2 e4m3x2_value(uint32_t w)
{
    return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3));
}

// Values of the four e4m3 codes of w.
__device__ __forceinline__ void e4m3x4_value(uint32_t w, __half2 (&v)[2])
{
    uint32_t o[2];
    asm("{\n\t.reg .b16 h0, h1;\n\t"
        "mov.b32 {h0, h1}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, h0;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, h1;\n\t}"
        : "=r"(o[0]), "=r"(o[1])
        : "r"(w));
    v[0] = bits_h2(o[0]), v[1] = bits_h2(o[1]);
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
