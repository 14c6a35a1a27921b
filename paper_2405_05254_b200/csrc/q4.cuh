// 4-bit codes to fp16 without conversion instructions, and fp16 pairs.
#pragma once

#include <cuda_fp16.h>

#include <cstdint>

namespace yoco {

__device__ __forceinline__ float2 h2_to_f2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
    __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b) {
    __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<uint32_t*>(&r);
}
// 1024 in both halves, in a register: AND with one constant and OR with another is one instruction only when the
// second one is not an immediate.
__device__ __forceinline__ uint32_t q4_magic() {
    uint32_t m;
    asm volatile("mov.b32 %0, 0x64006400;" : "=r"(m));
    return m;
}
// two codes at bits 0-3 and 16-19 -> (n - 8) as fp16, exact
__device__ __forceinline__ uint32_t q4_signed_lo(uint32_t w, uint32_t magic) {
    uint32_t x;
    asm("lop3.b32 %0, %1, 0x000F000F, %2, 0xEA;" : "=r"(x) : "r"(w), "r"(magic));   // 1024 + n
    const uint32_t off = 0xE408E408u;                                                // -1032
    __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&off));
    return *reinterpret_cast<uint32_t*>(&r);
}
// two codes at bits 4-7 and 20-23 -> (n - 8)
__device__ __forceinline__ uint32_t q4_signed_hi(uint32_t w, uint32_t magic) {
    uint32_t x;
    asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0xEA;" : "=r"(x) : "r"(w), "r"(magic));   // 1024 + 16 n
    const uint32_t sixteenth = 0x2C002C00u, off = 0xD480D480u;                       // 1/16, -72
    __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&sixteenth),
                        *reinterpret_cast<const __half2*>(&off));
    return *reinterpret_cast<uint32_t*>(&r);
}

}  // namespace yoco
