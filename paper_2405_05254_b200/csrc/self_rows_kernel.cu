// Token-major rows of a self-decoder: rotation of queries and keys by computed angles, normalisation of the heads' outputs with a gate.
// Both move bytes: rows are read and written once in 16-byte pieces.
#include <type_traits>

#include "gret.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace yoco {

namespace {

// ---- rotation -------------------------------------------------------------------------------------------
// A block works on `tb` tokens.  Cosines and sines of a token's rot / 2 angles are the same for all its heads: the block computes them once,
// into shared memory.  The angle is a product in 64 bits, reduced to a fraction of a turn in 64 bits, and only that is rounded to
// fp32: at position 10^6 an fp32 angle would be off by 0.06.  Then a thread takes units of 16 channels of a (token, head) row: eight pairs
// (halves: channels 8 u .. and rot / 2 + 8 u ..; neighbours: 16 u ..), or 16 channels that are copied.
// Bound: bytes.  Measured: 32,768 tokens, 32 + 32 heads of 128, 174-176 us (0.94 of the copy rate; 169-171 in short bursts); five sequences, 10,800 tokens, 16 + 16 heads,
// half of each head turned, 33.7 us (0.80: two and a third rounds of blocks); one token of 64 sequences 2.6 us in a recorded graph.
constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 2;            // rows that a thread has in flight

template <class Table>
__global__ void __launch_bounds__(kRopeThreads, 4)
rope_kernel(const RopeParams p, const __grid_constant__ Table tab, const int tb) {
    extern __shared__ __align__(16) float angles[];                 // [tb][2][rot / 2]: cosines, sines
    const int half = p.rot / 2, tid = threadIdx.x, tok0 = blockIdx.x * tb, n_tok = min(tb, p.tokens - tok0);
    for (int i = tid; i < n_tok * half; i += kRopeThreads) {
        const int t = i / half, j = i - t * half, tok = tok0 + t;
        const int b = find_sequence(tab, p.B, p.tokens_per_seq, tok);
        const int first = p.tokens_per_seq > 0 ? b * p.tokens_per_seq : tab.tok0[b];
        const double turns = (double)(tab.pos0[b] + (tok - first)) * p.inv_freq[j] * 0.15915494309189535;       // / 2 pi
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        angles[t * p.rot + j] = c;
        angles[t * p.rot + half + j] = s;
    }
    __syncthreads();

    const int units = p.d / 16, H = p.Hq + p.Hk, u = tid % units, step = kRopeThreads / units, rows = n_tok * H;
    int row = tid / units;
    if (row >= step) return;                                        // (units does not divide the block)
    const bool turns = 16 * u < p.rot;
    const int a_at = !turns || p.neighbours ? 16 * u : 8 * u, b_at = !turns || p.neighbours ? 16 * u + 8 : half + 8 * u;
    const int step_tokens = step / H, step_heads = step - step_tokens * H;
    int t = row / H, head = row - t * H;
    while (row < rows) {
        uint4 x[kRopeRows][2];
        __nv_bfloat16* dst[kRopeRows];
        int tok[kRopeRows];
#pragma unroll
        for (int r = 0; r < kRopeRows; ++r, row += step) {
            tok[r] = t;
            dst[r] = nullptr;
            if (row < rows) {
                const bool is_q = head < p.Hq;
                const int64_t at = tok0 + t;
                const __nv_bfloat16* src = is_q ? p.q + at * p.q_stride + head * p.d : p.k + at * p.k_stride + (head - p.Hq) * p.d;
                dst[r] = is_q ? p.q_out + at * p.q_out_stride + head * p.d : p.k_out + at * p.k_out_stride + (head - p.Hq) * p.d;
                x[r][0] = *reinterpret_cast<const uint4*>(src + a_at);
                x[r][1] = *reinterpret_cast<const uint4*>(src + b_at);
            }
            head += step_heads;
            t += step_tokens;
            if (head >= H) {
                head -= H;
                ++t;
            }
        }
#pragma unroll
        for (int r = 0; r < kRopeRows; ++r) {
            if (!dst[r]) continue;
            if (turns) {
                float a[8], b[8], c[8], s[8];
                unpack8(x[r][0], a);
                unpack8(x[r][1], b);
                const float* cs = angles + tok[r] * p.rot + 8 * u;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    *reinterpret_cast<float4*>(c + 4 * q) = *reinterpret_cast<const float4*>(cs + 4 * q);
                    *reinterpret_cast<float4*>(s + 4 * q) = *reinterpret_cast<const float4*>(cs + half + 4 * q);
                }
                if (p.neighbours) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        turn(a[2 * j], a[2 * j + 1], c[j], s[j]);
                        turn(b[2 * j], b[2 * j + 1], c[4 + j], s[4 + j]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) turn(a[j], b[j], c[j], s[j]);
                }
                x[r][0] = pack8(a);
                x[r][1] = pack8(b);
            }
            *reinterpret_cast<uint4*>(dst[r] + a_at) = x[r][0];
            *reinterpret_cast<uint4*>(dst[r] + b_at) = x[r][1];
        }
    }
}

// ---- normalisation of a group, gain, bias, gate -------------------------------------------------------
// W neighbouring lanes hold a group's channels, 8 C each; mean first, then the sum of squares of the differences.
constexpr int kNormThreads = 128;

template <int W, int C>
__global__ void __launch_bounds__(kNormThreads)
head_norm_kernel(const HeadNormParams p) {
    const int lane = threadIdx.x % W;
    const int64_t group = (int64_t)blockIdx.x * (kNormThreads / W) + threadIdx.x / W;
    const bool live = group < p.groups;
    const int g = live ? (int)group : 0, tok = g / p.H;
    const int64_t col = (int64_t)(g - tok * p.H) * p.d;             // (rows may be longer than 2^31 channels)
    const __nv_bfloat16* src = p.x + tok * p.x_stride + col;
    const __nv_bfloat16* gate = p.norm.gate ? p.norm.gate + tok * p.norm.gate_stride + col : nullptr;
    uint4 xr[C], gr[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * W + lane) * 8;
        xr[c] = gr[c] = make_uint4(0u, 0u, 0u, 0u);
        if (at < p.d) {
            xr[c] = *reinterpret_cast<const uint4*>(src + at);
            if (gate) gr[c] = *reinterpret_cast<const uint4*>(gate + at);
        }
    }
    float x[C][8], sum = 0.f, sq = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) unpack8(xr[c], x[c]);
    if (!p.norm.rms) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += x[c][j];            // (channels behind the group are zero)
#pragma unroll
        for (int m = W / 2; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
        sum *= 1.f / (float)p.d;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const bool in = (c * W + lane) * 8 < p.d;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[c][j] = in ? x[c][j] - sum : 0.f;
            sq = fmaf(x[c][j], x[c][j], sq);
        }
    }
#pragma unroll
    for (int m = W / 2; m > 0; m >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, m);
    const float inv = 1.f / sqrtf(sq / (float)p.d + p.norm.eps);
    if (!live) return;
    __nv_bfloat16* dst = p.y + tok * p.y_stride + col;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = (c * W + lane) * 8;
        if (at >= p.d) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[c][j] *= inv;
        float w[8];
        if (p.norm.gain) {
            unpack8(__ldg(reinterpret_cast<const uint4*>(p.norm.gain + col + at)), w);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[c][j] *= w[j];
        }
        if (p.norm.bias) {
            unpack8(__ldg(reinterpret_cast<const uint4*>(p.norm.bias + col + at)), w);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[c][j] += w[j];
        }
        if (gate) {
            unpack8(gr[c], w);
#pragma unroll
            for (int j = 0; j < 8; j += 2)
                f2_unpack(f2_swish_mul(f2_pack(w[j], w[j + 1]), f2_pack(x[c][j], x[c][j + 1])), x[c][j], x[c][j + 1]);
        }
        *reinterpret_cast<uint4*>(dst + at) = pack8(x[c]);
    }
}

template <int W, int C>
cudaError_t norm_one(const HeadNormParams& p, cudaStream_t stream) {
    constexpr int per_block = kNormThreads / W;
    head_norm_kernel<W, C><<<(unsigned)(((int64_t)p.groups + per_block - 1) / per_block), kNormThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p, const SeqTable& tab, int sm_count, cudaStream_t stream) {
    if (p.tokens <= 0) return cudaSuccess;
    // tokens of a block: as many as leave the GPU four blocks per SM, at most 8
    int tb = 1;
    while (tb < 8 && (int64_t)p.tokens / (2 * tb) >= 4ll * sm_count) tb *= 2;
    const unsigned grid = (unsigned)((p.tokens + tb - 1) / tb);
    const size_t smem = (size_t)tb * p.rot * sizeof(float);
    with_table(tab, p.B, [&](const auto& t) { rope_kernel<<<grid, kRopeThreads, smem, stream>>>(p, t, tb); });
    return cudaGetLastError();
}

// Lanes of a group: the fewest (a power of two) that need no more than five pieces each, but four rather than two, and two rather than one,
// where that leaves no lane idle and at least two pieces to each: a thread then has its loads in flight side by side, with few shuffles, and
// neighbouring lanes read 64 bytes.  Small blocks, because a block goes through its loads, sums and stores in step.
// (Measured, 16,001 tokens of 3,200 channels with gain, bias and gate, 307 MB: groups of 64 over two / four / eight lanes 70 / 58 / 68 us; of 80 over
// two / four / eight 59 / 60 / 84; of 128 over four / eight / sixteen 56 / 58 / 70, and in blocks of 256 instead of 128 threads 61 over four.)
cudaError_t launch_head_norm(const HeadNormParams& p, cudaStream_t stream) {
    if (p.groups <= 0) return cudaSuccess;
    const int pieces = p.d / 8;
    auto lanes = [&](auto w) {
        constexpr int W = decltype(w)::value;
        switch ((pieces + W - 1) / W) {
            case 3: return norm_one<W, 3>(p, stream);
            case 4: return norm_one<W, 4>(p, stream);
            default: return norm_one<W, 5>(p, stream);
        }
    };
    if (pieces == 1) return norm_one<1, 1>(p, stream);
    if (pieces == 2) return norm_one<1, 2>(p, stream);
    if (pieces == 3) return norm_one<1, 3>(p, stream);
    if (pieces == 4) return norm_one<2, 2>(p, stream);
    if (pieces == 5) return norm_one<1, 5>(p, stream);
    if (pieces == 8) return norm_one<4, 2>(p, stream);
    if (pieces <= 10) return lanes(std::integral_constant<int, 2>{});
    if (pieces <= 20) return lanes(std::integral_constant<int, 4>{});
    if (pieces <= 40) return lanes(std::integral_constant<int, 8>{});
    if (pieces <= 80) return lanes(std::integral_constant<int, 16>{});
    return pieces <= 96 ? norm_one<32, 3>(p, stream) : norm_one<32, 4>(p, stream);
}

}  // namespace yoco
