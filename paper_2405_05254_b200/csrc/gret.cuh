// What the gated-retention kernels share: decays, and the normalisation and gate of a head's output.
#pragma once

#include <cuda_bf16.h>

#include "kernels.h"
#include "ptx.cuh"
#include "rows.cuh"
#include "tcgen05.cuh"

namespace yoco {

__device__ __forceinline__ float read_decay(const GretParams& p, int64_t tok, int h) {
    const int64_t at = tok * p.decay_stride + h;
    return p.decay_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.decay)[at]) : static_cast<const float*>(p.decay)[at];
}
// log(1 + e) for 0 <= e <= 1, by 2 artanh(s), s = e / (2 + e) <= 1/3: the first term left out is s^14 / 15 = 1.4e-8 of the sum.  (Few
// instructions: on the way into a kernel they all come from memory.)
__device__ __forceinline__ float log1p_unit(float e) {
    const float s = __fdividef(e, 2.f + e), t = s * s;
    float p = fmaf(t, 1.f / 13.f, 1.f / 11.f);
    p = fmaf(t, p, 1.f / 9.f);
    p = fmaf(t, p, 1.f / 7.f);
    p = fmaf(t, p, 1.f / 5.f);
    p = fmaf(t, p, 1.f / 3.f);
    return 2.f * fmaf(s * t, p, s);
}
// Natural logarithm of the decay that z stands for, not below kMinLogDecay; a NaN stays one.
__device__ __forceinline__ float log_decay(const GretParams& p, float z) {
    if (p.inv_tau > 0.f) z = (fminf(z, 0.f) - log1p_unit(expf(-fabsf(z)))) * p.inv_tau;        // log sigmoid(z) / tau, without overflow on either side
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(kMinLogDecay));
    return r;
}

__device__ __forceinline__ float swish(float u) { return __fdividef(u, 1.f + __expf(-u)); }

// y * swish(u) for two at a time, swish(u) = u / (1 + 2^(-u log2 e)) first: u y may overflow where swish(u) is 0.
__device__ __forceinline__ uint64_t f2_swish_mul(uint64_t u, uint64_t y) {
    float e0, e1;
    f2_unpack(f2_mul(u, f2_pack(-1.4426950408889634f, -1.4426950408889634f)), e0, e1);
    f2_unpack(f2_add(f2_pack(ex2_approx(e0), ex2_approx(e1)), f2_pack(1.f, 1.f)), e0, e1);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e0));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e1));
    return f2_mul(f2_mul(u, f2_pack(e0, e1)), y);
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) x += __shfl_xor_sync(0xffffffffu, x, m);
    return x;
}

// calls of few sequences take a table of their size (see with_table)
template <class F>
void with_gret_table(const GretTable& tab, int B, F launch) {
    if (B > kFewSequences) return launch(tab);
    GretTableOf<kFewSequences> few;
    std::memcpy(few.from, tab.from, B * sizeof few.from[0]);
    std::memcpy(few.to, tab.to, B * sizeof few.to[0]);
    std::memcpy(few.tok0, tab.tok0, (B + 1) * sizeof few.tok0[0]);
    launch(few);
}

}  // namespace yoco
