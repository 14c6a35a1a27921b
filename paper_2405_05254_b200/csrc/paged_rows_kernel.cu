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
// read while they are in flight, and nothing is kept in shared memory.
#include "kernels.h"
#include "page_map.cuh"
#include "ptx.cuh"

namespace yoco {

namespace {

constexpr int kRowThreads = 128;

// which sequence a token belongs to, and its number inside it
__device__ __forceinline__ int find_sequence(const SeqTable& tab, int B, int per_seq, int tok) {
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
// The two chunks of a row that thread i of d / 16 holds: channels 8 i .. 8 i + 7 (lo) and d / 2 + 8 i .. (hi).
__device__ __forceinline__ void rotate_chunks(float (&lo)[8], float (&hi)[8], const Rotation& rot, int d, int64_t pos, int i) {
    if (!rot.cos_sin) return;
    const float* cs = rot.cos_sin + pos * d;
    const int half = d / 2;
    float c[8], s[8];
    if (rot.neighbours) {                          // lo: pairs 4 i .. 4 i + 3, hi: the same plus d / 4
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int at = q * (half / 2) + 4 * i;
            *reinterpret_cast<float4*>(c + 4 * q) = __ldg(reinterpret_cast<const float4*>(cs + at));
            *reinterpret_cast<float4*>(s + 4 * q) = __ldg(reinterpret_cast<const float4*>(cs + half + at));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            turn(lo[2 * j], lo[2 * j + 1], c[j], s[j]);
            turn(hi[2 * j], hi[2 * j + 1], c[4 + j], s[4 + j]);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            *reinterpret_cast<float4*>(c + 4 * q) = __ldg(reinterpret_cast<const float4*>(cs + 8 * i + 4 * q));
            *reinterpret_cast<float4*>(s + 4 * q) = __ldg(reinterpret_cast<const float4*>(cs + half + 8 * i + 4 * q));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) turn(lo[j], hi[j], c[j], s[j]);
    }
}

// Eight channels of a 32-channel group that four neighbouring lanes hold: their codes, and the group's scale.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], __half& scale) {
    float a = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) a = fmaxf(a, fabsf(x[j]));
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
    scale = __float2half_rn(fminf(__fmul_rn(a, 1.0f / 7.0f), kQ4ScaleMax));
    const float s = __half2float(scale);
    const float inv = s > 0.f ? __frcp_rn(s) : 0.f;
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int n = 8 + (int)fminf(fmaxf(rintf(__fmul_rn(x[j], inv)), -7.f), 7.f);
        w |= (uint32_t)n << (4 * j);
    }
    return w;
}

// One thread: chunks i (lo) and i (hi) of the key row and of the value row of one (token, head).
template <int D, bool Q4>
__global__ void __launch_bounds__(kRowThreads)
paged_append_kernel(const PagedRowsParams p, const __grid_constant__ SeqTable tab) {
    constexpr int PER_ROW = D / 16;
    const int64_t idx = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    const int H = p.pages.Hkv;
    const int i = (int)(idx % PER_ROW);
    const int64_t rh = idx / PER_ROW;
    const bool live = rh < (int64_t)p.tokens * H;  // lanes behind the last row stay for the group shuffles
    const int tok = live ? (int)(rh / H) : 0, head = live ? (int)(rh - (int64_t)tok * H) : 0;

    const __nv_bfloat16* ks = p.k_src + (int64_t)tok * p.src_stride + head * D + 8 * i;
    const __nv_bfloat16* vs = p.v_src + (int64_t)tok * p.src_stride + head * D + 8 * i;
    const uint4 k0 = __ldg(reinterpret_cast<const uint4*>(ks)), k1 = __ldg(reinterpret_cast<const uint4*>(ks + D / 2));
    const uint4 v0 = __ldg(reinterpret_cast<const uint4*>(vs)), v1 = __ldg(reinterpret_cast<const uint4*>(vs + D / 2));

    const int b = find_sequence(tab, p.B, p.tokens_per_seq, tok);
    const int first = p.tokens_per_seq > 0 ? b * p.tokens_per_seq : tab.tok0[b];
    const int pos = tab.pos0[b] + (tok - first);
    const int page = __ldg(p.pages.table + (int64_t)b * p.pages.table_stride + (pos >> p.pages.page_shift));
    const bool page_ok = (uint32_t)page < (uint32_t)p.pages.num_pages;
    const int64_t row = (int64_t)page * p.pages.page_rows + ((int64_t)head << p.pages.page_shift) +
                        (pos & ((1 << p.pages.page_shift) - 1));

    float lo[8], hi[8];
    unpack8(k0, lo);
    unpack8(k1, hi);
    rotate_chunks(lo, hi, p.rot, D, pos, i);
    const bool store = live && page_ok;
    if (live && !page_ok && i == 0) report_bad_page(p.status);
    if (!Q4) {
        if (store) {
            __nv_bfloat16* kd = static_cast<__nv_bfloat16*>(p.k_pool) + row * D + 8 * i;
            __nv_bfloat16* vd = static_cast<__nv_bfloat16*>(p.v_pool) + row * D + 8 * i;
            *reinterpret_cast<uint4*>(kd) = pack8(lo);
            *reinterpret_cast<uint4*>(kd + D / 2) = pack8(hi);
            *reinterpret_cast<uint4*>(vd) = v0;
            *reinterpret_cast<uint4*>(vd + D / 2) = v1;
        }
        return;
    }
    float vlo[8], vhi[8];
    unpack8(v0, vlo);
    unpack8(v1, vhi);
    __half s[4];
    const uint32_t w[4] = {quantise8(lo, s[0]), quantise8(hi, s[1]), quantise8(vlo, s[2]), quantise8(vhi, s[3])};
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

// eight 4-bit codes times their scale -> eight bf16 (the product is exact in fp32, one rounding)
__device__ __forceinline__ uint4 expand8(uint32_t w, __half scale) {
    const float s = __half2float(scale);
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)((int)((w >> (4 * j)) & 15u) - 8) * s;
    return pack8(x);
}

// One thread: 8 channels of the key row and of the value row of one (sequence, head, position); output rows
// are head-major inside a sequence.
template <int D, bool Q4>
__global__ void __launch_bounds__(kRowThreads)
paged_gather_kernel(const PagedRowsParams p, const __grid_constant__ SeqTable tab) {
    constexpr int PER_ROW = D / 8;
    const int64_t idx = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    const int i = (int)(idx % PER_ROW);
    const int64_t out_row = idx / PER_ROW;
    const int H = p.pages.Hkv;
    if (out_row >= (int64_t)p.tokens * H) return;
    // sequence b owns output rows [tok0[b] * H, tok0[b + 1] * H)
    const int b = find_sequence(tab, p.B, p.tokens_per_seq, (int)(out_row / H));
    const int first = p.tokens_per_seq > 0 ? b * p.tokens_per_seq : tab.tok0[b];
    const int n = p.tokens_per_seq > 0 ? p.tokens_per_seq : tab.tok0[b + 1] - first;
    const int local = (int)(out_row - (int64_t)first * H);
    const int head = local / n, pos = tab.pos0[b] + (local - head * n);
    const int page = __ldg(p.pages.table + (int64_t)b * p.pages.table_stride + (pos >> p.pages.page_shift));
    uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
    if ((uint32_t)page < (uint32_t)p.pages.num_pages) {
        const int64_t row = (int64_t)page * p.pages.page_rows + ((int64_t)head << p.pages.page_shift) +
                            (pos & ((1 << p.pages.page_shift) - 1));
        if (Q4) {
            const int64_t at = row * (D / 8) + i, sc = row * (D / kQ4Group) + i / (kQ4Group / 8);
            const uint32_t kw = __ldg(static_cast<const uint32_t*>(p.k_pool) + at);
            const uint32_t vw = __ldg(static_cast<const uint32_t*>(p.v_pool) + at);
            k = expand8(kw, p.k_scale[sc]);
            v = expand8(vw, p.v_scale[sc]);
        } else {
            k = __ldg(static_cast<const uint4*>(p.k_pool) + row * (D / 8) + i);
            v = __ldg(static_cast<const uint4*>(p.v_pool) + row * (D / 8) + i);
        }
    } else if (i == 0) {
        report_bad_page(p.status);
    }
    reinterpret_cast<uint4*>(p.k_out)[out_row * (D / 8) + i] = k;
    reinterpret_cast<uint4*>(p.v_out)[out_row * (D / 8) + i] = v;
}

template <int D>
__global__ void __launch_bounds__(kRowThreads)
rope_q_kernel(const __nv_bfloat16* Q, __nv_bfloat16* Qr, int64_t rows, int Hq, int T, const Rotation rot,
              const __grid_constant__ SeqTable tab) {
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
    if (pos >= 0) rotate_chunks(lo, hi, rot, D, pos, i);
    __nv_bfloat16* dst = Qr + row * D + 8 * i;
    *reinterpret_cast<uint4*>(dst) = pack8(lo);
    *reinterpret_cast<uint4*>(dst + D / 2) = pack8(hi);
}

unsigned grid_for(int64_t threads) { return (unsigned)((threads + kRowThreads - 1) / kRowThreads); }

}  // namespace

cudaError_t launch_paged_append(const PagedRowsParams& p, const SeqTable& tab, bool q4, cudaStream_t stream) {
    if (p.tokens <= 0) return cudaSuccess;
    const unsigned grid = grid_for((int64_t)p.tokens * p.pages.Hkv * (p.d / 16));
    if (q4)
        paged_append_kernel<128, true><<<grid, kRowThreads, 0, stream>>>(p, tab);
    else if (p.d == 128)
        paged_append_kernel<128, false><<<grid, kRowThreads, 0, stream>>>(p, tab);
    else
        paged_append_kernel<64, false><<<grid, kRowThreads, 0, stream>>>(p, tab);
    return cudaGetLastError();
}

cudaError_t launch_paged_gather(const PagedRowsParams& p, const SeqTable& tab, bool q4, cudaStream_t stream) {
    if (p.tokens <= 0) return cudaSuccess;
    const unsigned grid = grid_for((int64_t)p.tokens * p.pages.Hkv * (p.d / 8));
    if (q4)
        paged_gather_kernel<128, true><<<grid, kRowThreads, 0, stream>>>(p, tab);
    else if (p.d == 128)
        paged_gather_kernel<128, false><<<grid, kRowThreads, 0, stream>>>(p, tab);
    else
        paged_gather_kernel<64, false><<<grid, kRowThreads, 0, stream>>>(p, tab);
    return cudaGetLastError();
}

cudaError_t launch_rope_q(const __nv_bfloat16* Q, __nv_bfloat16* Qr, int32_t B, int32_t Hq, int32_t T, int32_t d,
                          const Rotation& rot, const SeqTable& tab, cudaStream_t stream) {
    const int64_t rows = (int64_t)B * Hq * T;
    if (rows <= 0) return cudaSuccess;
    const unsigned grid = grid_for(rows * (d / 16));
    if (d == 128)
        rope_q_kernel<128><<<grid, kRowThreads, 0, stream>>>(Q, Qr, rows, Hq, T, rot, tab);
    else
        rope_q_kernel<64><<<grid, kRowThreads, 0, stream>>>(Q, Qr, rows, Hq, T, rot, tab);
    return cudaGetLastError();
}

}  // namespace yoco
