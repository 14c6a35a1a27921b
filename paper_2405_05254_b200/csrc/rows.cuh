// What the kernels over token rows share: 16-byte pieces of bf16 rows, the rotation of a pair, and the sequence a token belongs to.
#pragma once

#include <cstring>

#include "kernels.h"
#include "ptx.cuh"

namespace yoco {

// which sequence a token belongs to
template <class Table>
__device__ __forceinline__ int find_sequence(const Table& tab, int B, int per_seq, int tok) {
    if (per_seq > 0) return tok / per_seq;
    int lo = 0, hi = B - 1;                        // last i with tok0[i] <= tok (empty sequences are passed over)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.tok0[mid] <= tok) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
    const float y1 = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
    b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
    a = y1;
}

// Calls of few sequences take a table of their size: 4 KB of parameters are written for every launch.
// (Measured, 64 sequences of one token: 20 calls after a synchronisation 8.6 -> 6.4 us each, rows of hundreds 3.9 either way; the
// kernels themselves take 1.6 us.)
constexpr int kFewSequences = 64;
template <class F>
void with_table(const SeqTable& tab, int B, F launch) {
    if (B > kFewSequences) return launch(tab);
    SeqTableOf<kFewSequences> few;
    std::memcpy(few.pos0, tab.pos0, sizeof few.pos0);
    std::memcpy(few.tok0, tab.tok0, sizeof few.tok0);
    launch(few);
}

}  // namespace yoco
