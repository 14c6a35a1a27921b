// Gated retention, recurrent form: S = g S + k^T v, o = scale q S, token after token with the state in registers.
//
// One CTA per (sequence, head).  Its 256 threads hold the d x d state in fp32, each four neighbouring value channels of some key
// channels: loads and stores of the state are whole rows.  A batch of up to eight tokens is staged in shared memory in fp32; a token then
// costs a multiply and two multiply-adds per element and no barrier: partial outputs of the eight warps (each has its own key
// channels) go to shared memory, and after the batch every warp finishes one token: sum, normalisation, gate, rounding.
//
// Bound: a step reads and writes 8 d^2 bytes of state per head and little else, so the loads of the state are all issued before
// anything is waited for (64 KB in flight per CTA at d = 128, two CTAs per SM).
// Measured: one token of 64 sequences, 32 heads of 128, with gate 49.2-49.5 us (0.84 of the copy rate of 6.56 TB/s), of 128 sequences without 86 us (0.95); of 37
// sequences, 24 heads of 64, 8.2 us; of one sequence 4.3 us in a recorded graph, 6.1 us a call (the host's part).
#include "gret.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rows.cuh"
#include "tcgen05.cuh"

namespace yoco {

namespace {

constexpr int kStepThreads = 256;
constexpr int kStepWarps = kStepThreads / 32;
constexpr int kStepBatch = kStepWarps;          // a warp finishes a token

// a thread's part of the state into the slot it goes to
template <int D, int N>
__device__ __forceinline__ void store_state(const uint64_t (&s)[N][2], const GretParams& p, int to, int h, int row0, int col) {
    float* dst = p.state + ((int64_t)to * p.H + h) * (D * D) + row0 * D + col;
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<ulonglong2*>(dst + i * D) = make_ulonglong2(s[i][0], s[i][1]);
}

template <int D, class Table>
__global__ void __launch_bounds__(kStepThreads, D == 128 ? 2 : 4)
gret_tokens_kernel(const GretParams p, const __grid_constant__ Table tab) {
    constexpr int LANES = D / 4;                   // threads across a row of the state
    constexpr int N = D * LANES / kStepThreads;    // key channels of a thread: 16 (d = 128) or 4
    constexpr int V = D / 32;                      // value channels of a lane that finishes a token
    __shared__ __align__(16) float rows[kStepBatch][3][D];
    __shared__ __align__(16) float part[kStepBatch][kStepWarps][D];
    __shared__ float gamma[kStepBatch];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int b = blockIdx.x / p.H, h = blockIdx.x - b * p.H;
    const int from = tab.from[b], to = tab.to[b];
    const int64_t tok0 = tab.tok0[b];
    const int n = tab.tok0[b + 1] - tab.tok0[b];
    const int col = (tid % LANES) * 4, row0 = (tid / LANES) * N;

    uint64_t s[N][2];                              // pairs of fp32
    if (from >= 0) {
        const float* src = p.state + ((int64_t)from * p.H + h) * (D * D) + row0 * D + col;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(src + i * D);
            s[i][0] = x.x;
            s[i][1] = x.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i][0] = s[i][1] = 0ull;
    }

    for (int t0 = 0; t0 < n; t0 += kStepBatch) {
        const int m = min(kStepBatch, n - t0);
        constexpr int PIECES = D / 8;              // 16-byte pieces of a row
        for (int i = tid; i < m * 3 * PIECES; i += kStepThreads) {
            const int t = i / (3 * PIECES), r = i - t * (3 * PIECES), which = r / PIECES, c = r - which * PIECES;
            const __nv_bfloat16* src = which == 0 ? p.q + (tok0 + t0 + t) * p.q_stride
                                     : which == 1 ? p.k + (tok0 + t0 + t) * p.k_stride : p.v + (tok0 + t0 + t) * p.v_stride;
            float x[8];
            unpack8(__ldg(reinterpret_cast<const uint4*>(src + h * D) + c), x);
            float4* dst = reinterpret_cast<float4*>(&rows[t][which][c * 8]);
            dst[0] = make_float4(x[0], x[1], x[2], x[3]);
            dst[1] = make_float4(x[4], x[5], x[6], x[7]);
        }
        // The gate is wanted at the end, where nothing else would be left to do meanwhile.  (128 sequences, 32 heads of 128 / of 64: 88.4 -> 86.5 us,
        // 32.7 -> 31.0; read into shared memory here instead, 96 / 33.)
        if (p.norm.gate && tid < m * (D / 64))
            asm volatile("prefetch.global.L2 [%0];" ::"l"(p.norm.gate + (tok0 + t0 + tid / (D / 64)) * p.norm.gate_stride + h * D + tid % (D / 64) * 64));
        if (tid < m) gamma[tid] = expf(log_decay(p, read_decay(p, tok0 + t0 + tid, h)));
        __syncthreads();
        for (int t = 0; t < m; ++t) {
            const uint64_t g = f2_pack(gamma[t], gamma[t]);
            const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(&rows[t][2][col]);
            uint64_t o0 = 0ull, o1 = 0ull;
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float4 q4 = *reinterpret_cast<const float4*>(&rows[t][0][row0 + i]), k4 = *reinterpret_cast<const float4*>(&rows[t][1][row0 + i]);
                const float q[4] = {q4.x, q4.y, q4.z, q4.w}, k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint64_t k2 = f2_pack(k[j], k[j]), q2 = f2_pack(q[j], q[j]);
                    s[i + j][0] = f2_fma(s[i + j][0], g, f2_fma(k2, v.x, 0ull));
                    s[i + j][1] = f2_fma(s[i + j][1], g, f2_fma(k2, v.y, 0ull));
                    o0 = f2_fma(q2, s[i + j][0], o0);
                    o1 = f2_fma(q2, s[i + j][1], o1);
                }
            }
            float4 o;
            f2_unpack(o0, o.x, o.y);
            f2_unpack(o1, o.z, o.w);
            if (LANES == 16) {                     // two rows a warp
                o.x += __shfl_xor_sync(0xffffffffu, o.x, 16);
                o.y += __shfl_xor_sync(0xffffffffu, o.y, 16);
                o.z += __shfl_xor_sync(0xffffffffu, o.z, 16);
                o.w += __shfl_xor_sync(0xffffffffu, o.w, 16);
            }
            if (lane < LANES) *reinterpret_cast<float4*>(&part[t][warp][col]) = o;
        }
        // the state leaves while the outputs are put together (d = 128: there are no registers for both; measured 58.7 us for 49.7)
        if (D == 64 && to >= 0 && t0 + kStepBatch >= n) store_state<D>(s, p, to, h, row0, col);
        __syncthreads();
        if (warp < m) {
            const int64_t tok = tok0 + t0 + warp;
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = 0.f;
#pragma unroll
            for (int w = 0; w < kStepWarps; ++w)
#pragma unroll
                for (int j = 0; j < V; ++j) y[j] += part[warp][w][lane * V + j];
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] *= p.scale;
            if (p.norm.on) {
                const int at = h * D + lane * V;
                float mean = 0.f, sq = 0.f;
                if (!p.norm.rms) {
#pragma unroll
                    for (int j = 0; j < V; ++j) mean += y[j];
                    mean = warp_sum(mean) * (1.f / D);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    y[j] -= mean;
                    sq = fmaf(y[j], y[j], sq);
                }
                const float inv = 1.f / sqrtf(warp_sum(sq) * (1.f / D) + p.norm.eps);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    y[j] *= inv;
                    if (p.norm.gain) y[j] *= __bfloat162float(p.norm.gain[at + j]);
                    if (p.norm.bias) y[j] += __bfloat162float(p.norm.bias[at + j]);
                    if (p.norm.gate) y[j] *= swish(__bfloat162float(p.norm.gate[tok * p.norm.gate_stride + at + j]));
                }
            }
            uint32_t* dst = reinterpret_cast<uint32_t*>(p.o + tok * p.o_stride + h * D + lane * V);
#pragma unroll
            for (int j = 0; j < V; j += 2) dst[j / 2] = pack_bf16x2(y[j], y[j + 1]);
        }
    }

    if (to >= 0 && (n > 0 ? D == 128 : to != from)) store_state<D>(s, p, to, h, row0, col);
}

}  // namespace

cudaError_t launch_gret_tokens(const GretParams& p, const GretTable& tab, cudaStream_t stream) {
    if (p.B <= 0) return cudaSuccess;
    const unsigned grid = (unsigned)p.B * (unsigned)p.H;
    with_gret_table(tab, p.B, [&](const auto& t) {
        if (p.d == 128)
            gret_tokens_kernel<128><<<grid, kStepThreads, 0, stream>>>(p, t);
        else
            gret_tokens_kernel<64><<<grid, kStepThreads, 0, stream>>>(p, t);
    });
    return cudaGetLastError();
}

}  // namespace yoco
