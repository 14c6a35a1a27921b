// Rows of a paged cache: storing the new tokens' keys (turned by their positions) and values, reading rows
// back into the packed head-major layout, and turning the queries by the same angles.
//
// Rotation: a pair of channels (x1, x2) of the token at position p becomes
//   (x1 cos a - x2 sin a, x2 cos a + x1 sin a),  a = the pair's angle at p,
// with the cosines and sines taken from the caller's fp32 table.  The three operations are rounded one by one
// (no fused multiply-add), so that a row is the same bits wherever it is computed from the same table.
//
// 4-bit rows: 32 channels share a scale s = fp16(min(max|x| / 7, 448)); code = 8 + round(x / s) in 1 .. 15, channel
// 2 i in the low nibble of byte i.  x is the fp32 value (a key after its rotation): there is no bf16 rounding in
// between.  Division by 7 and by s are products with the fp32 reciprocal.
//
// These kernels only move bytes: a thread reads 16-byte chunks of one (token, head) row, the page number is
// read while they are in flight, and nothing is kept in shared memory.  What bounds them at size is instructions, then
// memory: so a block works on one head (no division to find it), and rounding and conversion of 4-bit codes go through
// additions to a large constant instead of the conversion instructions, which run at a quarter of the rate.
#include "kernels.h"
#include "page_map.cuh"
#include "ptx.cuh"
#include "q4.cuh"
#include "rows.cuh"

namespace yoco {

namespace {

constexpr int kRowThreads = 128;

// The two chunks of a row that thread i of d / 16 holds: channels 8 i .. 8 i + 7 (lo) and d / 2 + 8 i .. (hi).  Their
// angles at a position: halves turn together, pair j is (lo[j], hi[j]); neighbours do, pairs 0 .. 3 lie in lo, 4 .. 7 in hi.
struct Angles {
    float c[8], s[8];
};
__device__ __forceinline__ void load_angles(Angles& a, const Rotation& rot, int d, int64_t pos, int i) {
    const float* cs = rot.cos_sin + pos * d;
    const int half = d / 2, step = rot.neighbours ? half / 2 : 4, at = rot.neighbours ? 4 * i : 8 * i;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        *reinterpret_cast<float4*>(a.c + 4 * q) = __ldg(reinterpret_cast<const float4*>(cs + at + q * step));
        *reinterpret_cast<float4*>(a.s + 4 * q) = __ldg(reinterpret_cast<const float4*>(cs + half + at + q * step));
    }
}
__device__ __forceinline__ void rotate_chunks(float (&lo)[8], float (&hi)[8], const Angles& a, bool neighbours) {
    if (neighbours) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            turn(lo[2 * j], lo[2 * j + 1], a.c[j], a.s[j]);
            turn(hi[2 * j], hi[2 * j + 1], a.c[4 + j], a.s[4 + j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) turn(lo[j], hi[j], a.c[j], a.s[j]);
    }
}

// max of two; a NaN beats everything (fmaxf passes it over)
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Largest magnitude of a 32-channel group that four neighbouring lanes hold eight channels of each.  KEEP_NAN: a NaN comes
// out as one, which is how a group that has one is noticed without an instruction more; otherwise it does not count.
template <bool KEEP_NAN>
__device__ __forceinline__ float group_max(const float (&x)[8]) {
    auto larger = [](float a, float b) { return KEEP_NAN ? max_or_nan(a, b) : fmaxf(a, b); };
    float a = larger(larger(larger(fabsf(x[0]), fabsf(x[1])), larger(fabsf(x[2]), fabsf(x[3]))),
                     larger(larger(fabsf(x[4]), fabsf(x[5])), larger(fabsf(x[6]), fabsf(x[7]))));
    a = larger(a, __shfl_xor_sync(0xffffffffu, a, 1));
    return larger(a, __shfl_xor_sync(0xffffffffu, a, 2));
}
// NaN stays NaN: see group_max
__device__ __forceinline__ float capped_seventh(float largest) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__fmul_rn(largest, 1.0f / 7.0f)), "f"(kQ4ScaleMax));
    return r;
}
// The codes of eight channels.  CLAMP = false where no channel is NaN and the scale is a normal number below the limit: it is
// then within 2^-11 of a seventh of the largest magnitude, and no quotient rounds to more than 7.  (A NaN has no place in that
// sum: its bits would run into the other channels' codes.  The clamp turns it into the code 1.)
template <bool CLAMP>
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], float scale) {
    const float inv = scale > 0.f ? __frcp_rn(scale) : 0.f;
    // rint by adding 1.5 * 2^23: the bits of the sum are those of the constant plus the integer.  They are put
    // together as they are, four bits apart; the constant's share and the offset 8 are settled once at the end.
    constexpr uint32_t carried = 0x4B400000u * 0x11111111u;      // sum of the constant's bits << 4 j, modulo 2^32
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float t = __fmul_rn(x[j], inv);
        if (CLAMP) t = fminf(fmaxf(t, -7.f), 7.f);
        w += __float_as_uint(__fadd_rn(t, 12582912.f)) << (4 * j);
    }
    return w - (carried - 0x88888888u);  // 8 << 4 j summed
}

// One thread: chunks i (lo) and i (hi) of the key row and of the value row of one token, for `heads` heads one after the
// other: the sequence, the page and the angles are looked up once.
template <int D, bool Q4, class Table>
__global__ void __launch_bounds__(kRowThreads)
paged_append_kernel(const PagedRowsParams p, const __grid_constant__ Table tab, const int heads) {
    constexpr int PER_ROW = D / 16;
    const int i = threadIdx.x % PER_ROW, head0 = blockIdx.y * heads, head1 = min(head0 + heads, p.pages.Hkv);
    int tok = blockIdx.x * (kRowThreads / PER_ROW) + threadIdx.x / PER_ROW;
    const bool live = tok < p.tokens;              // lanes behind the last row stay for the group shuffles
    if (!live) tok = 0;

    const __nv_bfloat16* ks = p.k_src + (int64_t)tok * p.src_stride + head0 * D + 8 * i;
    const __nv_bfloat16* vs = p.v_src + (int64_t)tok * p.src_stride + head0 * D + 8 * i;
    uint4 k0 = __ldg(reinterpret_cast<const uint4*>(ks)), k1 = __ldg(reinterpret_cast<const uint4*>(ks + D / 2));
    uint4 v0 = __ldg(reinterpret_cast<const uint4*>(vs)), v1 = __ldg(reinterpret_cast<const uint4*>(vs + D / 2));

    const int b = find_sequence(tab, p.B, p.tokens_per_seq, tok);
    const int first = p.tokens_per_seq > 0 ? b * p.tokens_per_seq : tab.tok0[b];
    const int pos = tab.pos0[b] + (tok - first);
    const int page = __ldg(p.pages.table + (int64_t)b * p.pages.table_stride + (pos >> p.pages.page_shift));
    const bool turned = p.rot.cos_sin != nullptr, neighbours = p.rot.neighbours != 0;
    Angles ang;
    if (turned) load_angles(ang, p.rot, D, pos, i);
    const bool page_ok = (uint32_t)page < (uint32_t)p.pages.num_pages, store = live && page_ok;
    if (live && !page_ok && i == 0 && head0 == 0) report_bad_page(p.status);
    int64_t row = (int64_t)page * p.pages.page_rows + ((int64_t)head0 << p.pages.page_shift) +
                  (pos & ((1 << p.pages.page_shift) - 1));

    for (int head = head0; head < head1; ++head, row += 1 << p.pages.page_shift) {
        uint4 nk0 = k0, nk1 = k1, nv0 = v0, nv1 = v1;          // the next head's, asked for before this one is worked off
        if (head + 1 < head1) {
            ks += D;
            vs += D;
            nk0 = __ldg(reinterpret_cast<const uint4*>(ks));
            nk1 = __ldg(reinterpret_cast<const uint4*>(ks + D / 2));
            nv0 = __ldg(reinterpret_cast<const uint4*>(vs));
            nv1 = __ldg(reinterpret_cast<const uint4*>(vs + D / 2));
        }
        float lo[8], hi[8];
        unpack8(k0, lo);
        unpack8(k1, hi);
        if (turned) rotate_chunks(lo, hi, ang, neighbours);
        if (!Q4) {
            if (store) {
                __nv_bfloat16* kd = static_cast<__nv_bfloat16*>(p.k_pool) + row * D + 8 * i;
                __nv_bfloat16* vd = static_cast<__nv_bfloat16*>(p.v_pool) + row * D + 8 * i;
                *reinterpret_cast<uint4*>(kd) = pack8(lo);
                *reinterpret_cast<uint4*>(kd + D / 2) = pack8(hi);
                *reinterpret_cast<uint4*>(vd) = v0;
                *reinterpret_cast<uint4*>(vd + D / 2) = v1;
            }
        } else {
            float vlo[8], vhi[8];
            unpack8(v0, vlo);
            unpack8(v1, vhi);
            const float largest[4] = {group_max<true>(lo), group_max<true>(hi), group_max<true>(vlo), group_max<true>(vhi)};
            __half s[4];
            float f[4];
            bool plain = true;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                s[q] = __float2half_rn(capped_seventh(largest[q]));
                f[q] = __half2float(s[q]);
                plain = plain && f[q] >= 6.103515625e-5f && f[q] < kQ4ScaleMax;         // false for a NaN
            }
            uint32_t w[4];
            if (__all_sync(0xffffffffu, plain)) {
                w[0] = quantise8<false>(lo, f[0]);
                w[1] = quantise8<false>(hi, f[1]);
                w[2] = quantise8<false>(vlo, f[2]);
                w[3] = quantise8<false>(vhi, f[3]);
            } else {
                const float finite[4] = {group_max<false>(lo), group_max<false>(hi), group_max<false>(vlo), group_max<false>(vhi)};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    s[q] = __float2half_rn(fminf(__fmul_rn(finite[q], 1.0f / 7.0f), kQ4ScaleMax));
                    f[q] = __half2float(s[q]);
                }
                w[0] = quantise8<true>(lo, f[0]);
                w[1] = quantise8<true>(hi, f[1]);
                w[2] = quantise8<true>(vlo, f[2]);
                w[3] = quantise8<true>(vhi, f[3]);
            }
            if (store) {
                constexpr int GROUPS = D / kQ4Group;
                uint8_t* kd = static_cast<uint8_t*>(p.k_pool) + row * (D / 2) + 4 * i;
                uint8_t* vd = static_cast<uint8_t*>(p.v_pool) + row * (D / 2) + 4 * i;
                *reinterpret_cast<uint32_t*>(kd) = w[0];
                *reinterpret_cast<uint32_t*>(kd + D / 4) = w[1];
                *reinterpret_cast<uint32_t*>(vd) = w[2];
                *reinterpret_cast<uint32_t*>(vd + D / 4) = w[3];
                if ((i & 3) == 0) {
                    const int g = i >> 2;
                    p.k_scale[row * GROUPS + g] = s[0];
                    p.k_scale[row * GROUPS + GROUPS / 2 + g] = s[1];
                    p.v_scale[row * GROUPS + g] = s[2];
                    p.v_scale[row * GROUPS + GROUPS / 2 + g] = s[3];
                }
            }
        }
        k0 = nk0;
        k1 = nk1;
        v0 = nv0;
        v1 = nv1;
    }
}

// eight 4-bit codes times their scale -> eight bf16 (code - 8 in fp16 and the product in fp32 are exact, one rounding)
__device__ __forceinline__ uint4 expand8(uint32_t w, float s, uint32_t magic) {
    const float2 a = h2_to_f2(q4_signed_lo(w, magic)), b = h2_to_f2(q4_signed_hi(w, magic));             // channels 0 4, 1 5
    const float2 c = h2_to_f2(q4_signed_lo(w >> 8, magic)), d = h2_to_f2(q4_signed_hi(w >> 8, magic));   // 2 6, 3 7
    return make_uint4(pack_bf16x2(a.x * s, b.x * s), pack_bf16x2(c.x * s, d.x * s), pack_bf16x2(a.y * s, b.y * s),
                      pack_bf16x2(c.y * s, d.y * s));
}

// One thread: 8 channels of the key row and of the value row of one position, for `heads` heads one after the other;
// output rows are head-major inside a sequence.
template <int D, bool Q4, class Table>
__global__ void __launch_bounds__(kRowThreads)
paged_gather_kernel(const PagedRowsParams p, const __grid_constant__ Table tab, const int heads) {
    constexpr int PER_ROW = D / 8;
    const int i = threadIdx.x % PER_ROW, H = p.pages.Hkv, head0 = blockIdx.y * heads, head1 = min(head0 + heads, H);
    const int tok = blockIdx.x * (kRowThreads / PER_ROW) + threadIdx.x / PER_ROW;
    if (tok >= p.tokens) return;
    // sequence b owns output rows [tok0[b] * H, tok0[b + 1] * H), head by head
    const int b = find_sequence(tab, p.B, p.tokens_per_seq, tok);
    const int first = p.tokens_per_seq > 0 ? b * p.tokens_per_seq : tab.tok0[b];
    const int n = p.tokens_per_seq > 0 ? p.tokens_per_seq : tab.tok0[b + 1] - first;
    const int pos = tab.pos0[b] + (tok - first);
    const int page = __ldg(p.pages.table + (int64_t)b * p.pages.table_stride + (pos >> p.pages.page_shift));
    const bool good = (uint32_t)page < (uint32_t)p.pages.num_pages;
    if (!good && i == 0 && head0 == 0) report_bad_page(p.status);
    int64_t row = (int64_t)page * p.pages.page_rows + ((int64_t)head0 << p.pages.page_shift) +
                  (pos & ((1 << p.pages.page_shift) - 1));
    int64_t at = ((int64_t)first * H + (int64_t)head0 * n + (tok - first)) * PER_ROW + i;
    uint4* k_out = reinterpret_cast<uint4*>(p.k_out) + at;
    uint4* v_out = reinterpret_cast<uint4*>(p.v_out) + at;
    const int64_t out_step = (int64_t)n * PER_ROW;
    const uint32_t magic = q4_magic();
#pragma unroll 1
    for (int head = head0; head < head1; ++head, row += 1 << p.pages.page_shift, k_out += out_step, v_out += out_step) {
        uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
        if (good) {
            if (Q4) {
                const int64_t sc = row * (D / kQ4Group) + i / (kQ4Group / 8);
                const uint32_t kw = __ldg(static_cast<const uint32_t*>(p.k_pool) + row * (D / 8) + i);
                const uint32_t vw = __ldg(static_cast<const uint32_t*>(p.v_pool) + row * (D / 8) + i);
                k = expand8(kw, __half2float(p.k_scale[sc]), magic);
                v = expand8(vw, __half2float(p.v_scale[sc]), magic);
            } else {
                k = __ldg(static_cast<const uint4*>(p.k_pool) + row * (D / 8) + i);
                v = __ldg(static_cast<const uint4*>(p.v_pool) + row * (D / 8) + i);
            }
        }
        *k_out = k;
        *v_out = v;
    }
}

template <int D, class Table>
__global__ void __launch_bounds__(kRowThreads)
rope_q_kernel(const __nv_bfloat16* Q, __nv_bfloat16* Qr, int64_t rows, int Hq, int T, const Rotation rot,
              const __grid_constant__ Table tab) {
    constexpr int PER_ROW = D / 16;
    const int64_t idx = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    const int i = (int)(idx % PER_ROW);
    const int64_t row = idx / PER_ROW;
    if (row >= rows) return;
    const int64_t bh = row / T;
    const int pos = tab.pos0[bh / Hq] + (int)(row - bh * T);
    const __nv_bfloat16* src = Q + row * D + 8 * i;
    const uint4 a = *reinterpret_cast<const uint4*>(src), c = *reinterpret_cast<const uint4*>(src + D / 2);
    float lo[8], hi[8];
    unpack8(a, lo);
    unpack8(c, hi);
    if (pos >= 0) {
        Angles ang;
        load_angles(ang, rot, D, pos, i);
        rotate_chunks(lo, hi, ang, rot.neighbours != 0);
    }
    __nv_bfloat16* dst = Qr + row * D + 8 * i;
    *reinterpret_cast<uint4*>(dst) = pack8(lo);
    *reinterpret_cast<uint4*>(dst + D / 2) = pack8(hi);
}

unsigned grid_for(int64_t threads) { return (unsigned)((threads + kRowThreads - 1) / kRowThreads); }
// `per_row` threads per token; a block works on as many heads, one after the other, as leave the GPU `blocks_per_sm` blocks
// per SM.  (Measured, 9,600 tokens of 8 heads and 4-bit rows: stored with four heads per block 14.5 us, with one or two
// 16.5; read back with one head per block 14.5 us, with eight 18.6: reading back has little to look up per token, and more
// blocks hide its loads better.)
dim3 rows_grid(const PagedRowsParams& p, int per_row, int blocks_per_sm, int* heads) {
    const unsigned blocks = grid_for((int64_t)p.tokens * per_row);
    *heads = 1;
    while (*heads < p.pages.Hkv && (int64_t)blocks * ((p.pages.Hkv + 2 * *heads - 1) / (2 * *heads)) >= 148 * blocks_per_sm) *heads *= 2;
    return dim3(blocks, (unsigned)((p.pages.Hkv + *heads - 1) / *heads));
}

}  // namespace

cudaError_t launch_paged_append(const PagedRowsParams& p, const SeqTable& tab, bool q4, cudaStream_t stream) {
    if (p.tokens <= 0) return cudaSuccess;
    int heads;
    const dim3 grid = rows_grid(p, p.d / 16, 8, &heads);
    with_table(tab, p.B, [&](const auto& t) {
        if (q4)
            paged_append_kernel<128, true><<<grid, kRowThreads, 0, stream>>>(p, t, heads);
        else if (p.d == 128)
            paged_append_kernel<128, false><<<grid, kRowThreads, 0, stream>>>(p, t, heads);
        else
            paged_append_kernel<64, false><<<grid, kRowThreads, 0, stream>>>(p, t, heads);
    });
    return cudaGetLastError();
}

cudaError_t launch_paged_gather(const PagedRowsParams& p, const SeqTable& tab, bool q4, cudaStream_t stream) {
    if (p.tokens <= 0) return cudaSuccess;
    int heads;
    const dim3 grid = rows_grid(p, p.d / 8, 64, &heads);
    with_table(tab, p.B, [&](const auto& t) {
        if (q4)
            paged_gather_kernel<128, true><<<grid, kRowThreads, 0, stream>>>(p, t, heads);
        else if (p.d == 128)
            paged_gather_kernel<128, false><<<grid, kRowThreads, 0, stream>>>(p, t, heads);
        else
            paged_gather_kernel<64, false><<<grid, kRowThreads, 0, stream>>>(p, t, heads);
    });
    return cudaGetLastError();
}

cudaError_t launch_rope_q(const __nv_bfloat16* Q, __nv_bfloat16* Qr, int32_t B, int32_t Hq, int32_t T, int32_t d,
                          const Rotation& rot, const SeqTable& tab, cudaStream_t stream) {
    const int64_t rows = (int64_t)B * Hq * T;
    if (rows <= 0) return cudaSuccess;
    const unsigned grid = grid_for(rows * (d / 16));
    with_table(tab, B, [&](const auto& t) {
        if (d == 128)
            rope_q_kernel<128><<<grid, kRowThreads, 0, stream>>>(Q, Qr, rows, Hq, T, rot, t);
        else
            rope_q_kernel<64><<<grid, kRowThreads, 0, stream>>>(Q, Qr, rows, Hq, T, rot, t);
    });
    return cudaGetLastError();
}

}  // namespace yoco
