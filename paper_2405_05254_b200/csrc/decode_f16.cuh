// What the decode kernels over narrow caches (8-bit, 4-bit) share around their fp16 products.
#pragma once

#include <cuda_fp16.h>

#include <cstdint>

namespace yoco {

// 8 x 8 transpose of 16-bit units across the warp: lane (g, tq) gives row g, columns 2 tq and 2 tq + 1,
// and receives the same positions of the transposed matrix.
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ float ex2_fast(float x) {   // 2^x, one special-function op; 2^-inf = 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace yoco
