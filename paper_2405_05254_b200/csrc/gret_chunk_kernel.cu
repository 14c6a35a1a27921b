// Gated retention, chunkwise form, on the tcgen05 tensor cores.
//
// A chunk is 128 tokens of one head.  With b_i = log2 g_1 + .. + log2 g_i inside the chunk, S the state before it and C its last token:
//     P_ij = (q_i . k_j) 2^(b_i - b_j)  (j <= i),   o_i = scale (sum_j P_ij v_j + 2^b_i q_i S),
//     S' = 2^b_C S + sum_j (2^(b_C - b_j) k_j)^T v_j.
// A CTA walks a contiguous range of chunks, of one (sequence, head) stream or of several one after the other, with the state in the
// registers of a warpgroup.  512 threads:
//   warp 0       TMA producer: K, Q, V tiles (128 tokens x d, 128-byte swizzle) through one ring
//   warp 1       issuer of all products: Q K^T -> SC;  K'^T V -> DS;  Q S -> OI;  P V -> OA    (tensor memory, fp32)
//   warp 2       decays: prefix sums of the logarithms in 64 bits, kept as integer part and rest (their differences are what
//                is used: b_i - b_j stays exact to 2^-24 however strong the decays before j were)
//   warpgroup 1  thread = token: P (bf16, over the scores' own columns: it goes to P V from tensor memory), then the chunk's output:
//                scale, normalisation, gate, rounding, store
//   warpgroup 2  thread = row of the state: S' from S and DS in fp32; S in bf16 to shared memory for the next chunk's Q S
//   warpgroup 3  K' = 2^(b_C - b_j) k_j, in pieces of 16 tokens
// Roundings: P and the copy of S that multiplies Q go to bf16 (half a step, 2^-9 of the value, like the output's own).  K' goes to
// the tensor cores as the sum of three bf16, 24 bits of it: the state is handed on in fp32, and with one bf16 it would be 1.7e-3
// off (2-norm), with two 2.7e-6.
//
// Order of the products per chunk: Q K^T (then P is computed), K'^T V (3 products), Q S, P V.  None waits for work that was not begun a
// product or more earlier: P has K'^T V and Q S to be ready, the state has all of the next Q K^T and K'^T V.  Tensor
// pipe 6 x 512 cycles a chunk (d = 128).
#include "gret.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rows.cuh"
#include "tcgen05.cuh"

namespace yoco {

namespace {

constexpr int CT = kGretChunk;                 // 128 tokens
constexpr int kThreads = 512;
constexpr int HALF_BYTES = CT * 128;           // 128 rows x 64 bf16: one swizzled half tile
constexpr int PIECE = 16;                      // tokens of a piece of K': one instruction's depth
constexpr int PIECES = CT / PIECE;
constexpr int TERM_BYTES = 2 * PIECE * 128;    // a piece of one of K's three parts: two halves of 64 channels
constexpr int PIECE_BYTES = 3 * TERM_BYTES;
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t COL_SC = 0, COL_OA = 128, COL_OI = 256, COL_DS = 384;
// Registers per thread after the split; the CTA starts with 128 each.
constexpr int kRegsIo = 56, kRegsOut = 192, kRegsState = 192, kRegsKeys = 72;
static_assert(kRegsIo + kRegsOut + kRegsState + kRegsKeys <= 4 * 128, "register pool of the CTA");

template <int D>
struct GCfg {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;
    static constexpr int STAGES = D == 128 ? 5 : 9;
    static constexpr int OFF_KP = STAGES * TILE_BYTES;
    static constexpr int OFF_S = OFF_KP + 2 * PIECE_BYTES;
    static constexpr int OFF_DEC = OFF_S + D * D * 2;          // two buffers of 128 negated integer parts and 128 negated rests
    static constexpr int OFF_BAR = OFF_DEC + 2 * 2 * CT * 4;
    static constexpr int NUM_BARS = 2 * STAGES + 17;
    static constexpr int SMEM_BYTES = OFF_BAR + NUM_BARS * 8 + 16;
    static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
};

// A place in a ring of N, and which time round.
template <int N>
struct Place {
    uint32_t slot, phase;
    __device__ __forceinline__ explicit Place(uint32_t first) : slot(first % N), phase((first / N) & 1u) {}
    __device__ __forceinline__ void advance(uint32_t by) {
        slot += by;
        if (slot >= (uint32_t)N) {
            slot -= N;
            phase ^= 1u;
        }
    }
};

// The segments of a CTA: chunks [c, c_end) of stream (b, h), in the flat space of (sequence, head, chunk).
template <class Table>
struct Walk {
    const GretChunkParams& p;
    const Table& tab;
    int64_t pos, end;
    int b, h, c, c_end, chunks;
    __device__ __forceinline__ Walk(const GretChunkParams& p_, const Table& tab_) : p(p_), tab(tab_) {
        const int64_t g = blockIdx.x;
        if (p.split) {
            pos = g * p.total / p.groups;
            end = (g + 1) * p.total / p.groups;
        } else {                                   // one CTA per stream
            const int bb = (int)(g / p.base.H), hh = (int)(g - (int64_t)bb * p.base.H), n = tab.chunk0[bb + 1] - tab.chunk0[bb];
            pos = (int64_t)tab.chunk0[bb] * p.base.H + (int64_t)hh * n;
            end = pos + n;
        }
    }
    // Enters the segment at pos; false when there is none left.
    __device__ __forceinline__ bool enter() {
        if (pos >= end) return false;
        const int64_t per = pos / p.base.H;        // tab.chunk0[b] <= per < tab.chunk0[b + 1]
        int lo = 0, hi = p.base.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tab.chunk0[mid] <= per) lo = mid; else hi = mid - 1;
        }
        b = lo;
        chunks = tab.chunk0[b + 1] - tab.chunk0[b];
        const int64_t in = pos - (int64_t)tab.chunk0[b] * p.base.H;
        h = (int)(in / chunks);
        c = (int)(in - (int64_t)h * chunks);
        const int64_t left = end - pos;
        c_end = left < chunks - c ? c + (int)left : chunks;
        pos += c_end - c;
        return true;
    }
    // State-only pass: straight to the segment that the range ends in, if its stream goes on behind it.
    __device__ __forceinline__ bool enter_open_end() {
        bool any = false;
        while (enter()) any = true;
        return any && c_end < chunks;
    }
};

__device__ __forceinline__ float exp2_parts(float whole, float rest) { return exp2f(whole) * exp2f(rest); }

template <int D, bool STATE_ONLY, class Table>
__global__ void __launch_bounds__(kThreads, 1)
gret_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const GretChunkParams p, const __grid_constant__ Table tab) {
    using C = GCfg<D>;
    constexpr int PER_CHUNK = STATE_ONLY ? 2 : 3;          // tiles a chunk brings: K (Q) V
    constexpr uint32_t V_AT = PER_CHUNK - 1;

    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
    uint64_t* ring_full = bars;                            // [STAGES]
    uint64_t* ring_empty = bars + C::STAGES;               // [STAGES]
    uint64_t* kp_full = bars + 2 * C::STAGES;              // [2]
    uint64_t* kp_empty = kp_full + 2;                      // [2]
    uint64_t* dec_full = kp_full + 4;                      // [2]
    uint64_t* dec_empty = kp_full + 6;                     // [2]
    uint64_t* sc_full = kp_full + 8;
    uint64_t* p_full = kp_full + 9;
    uint64_t* ds_full = kp_full + 10;
    uint64_t* ds_empty = kp_full + 11;
    uint64_t* s_full = kp_full + 12;
    uint64_t* s_empty = kp_full + 13;
    uint64_t* o_full = kp_full + 14;
    uint64_t* o_empty = kp_full + 15;
    uint64_t* drain_bar = kp_full + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float* dec = reinterpret_cast<float*>(smem + C::OFF_DEC);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Abort ab{abort_flag, p.status, kWaitLimitNs};
    const bool aligned_ok = (smem_u32(smem) & 1023u) == 0;

    if (threadIdx.x == 0) {
        *abort_flag = aligned_ok ? 0 : 1;
        if (!aligned_ok) atomicCAS(p.status, 0, status_word(kWaitMisaligned, linear_cta()));
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(&ring_full[i], 1);
            mbar_init(&ring_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&kp_full[i], 4);
            mbar_init(&kp_empty[i], 1);
            mbar_init(&dec_full[i], 1);
            mbar_init(&dec_empty[i], STATE_ONLY ? 8 : 12);
        }
        mbar_init(sc_full, 1);
        mbar_init(p_full, 4);
        mbar_init(ds_full, 1);
        mbar_init(ds_empty, 4);
        mbar_init(s_full, 4);
        mbar_init(s_empty, 1);
        mbar_init(o_full, 1);
        mbar_init(o_empty, 4);
        mbar_init(drain_bar, 1);
        mbar_fence_init();
    }
    if (warp == 1) {
        tmem_alloc(tmem_slot, TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const uint32_t sbase = smem_u32(smem);

    // every role walks the same segments: `enter` moves to the next one
    Walk<Table> walk(p, tab);
    bool open_end_done = false;
    auto enter = [&]() -> bool {
        if (!STATE_ONLY) return walk.enter();
        if (open_end_done) return false;
        open_end_done = true;
        return walk.enter_open_end();
    };

    if (warp < 4) {
        setmaxnreg_dec<kRegsIo>();
        if (warp == 0) {
            // ======================================= TMA producer ================================
            if (lane == 0 && aligned_ok) {
                tma_prefetch_desc(&tmK);
                tma_prefetch_desc(&tmV);
                if (!STATE_ONLY) tma_prefetch_desc(&tmQ);
                Place<C::STAGES> at(0);
                uint32_t armed = 0;
                bool ok = true;
                while (ok && enter()) {
                    for (int c = walk.c; ok && c < walk.c_end; ++c) {
                        const int row = tab.tok0[walk.b] + c * CT;
                        for (int i = 0; i < PER_CHUNK; ++i) {
                            if (!(ok = wait_or_abort(&ring_empty[at.slot], at.phase ^ 1u, ab, kWaitRingEmpty))) break;
                            const CUtensorMap* tm = i == 0 ? &tmK : i == (int)V_AT ? &tmV : &tmQ;
                            mbar_expect_tx(&ring_full[at.slot], C::TILE_BYTES);
                            for (int hf = 0; hf < C::HALVES; ++hf)
                                tma_load_2d(smem + at.slot * C::TILE_BYTES + hf * HALF_BYTES, tm, walk.h * D + hf * 64, row, &ring_full[at.slot]);
                            ++armed;
                            at.advance(1);
                        }
                    }
                }
                // no copy may land after the CTA has ended (at once when all went well)
                bool drained = true;
                for (uint32_t k = armed > (uint32_t)C::STAGES ? armed - C::STAGES : 0; drained && k < armed; ++k)
                    drained = drain_wait(&ring_full[k % C::STAGES], (k / C::STAGES) & 1u, ab);
            }
        } else if (warp == 1) {
            // ======================================= issuer of the products ======================
            if (aligned_ok) {
                constexpr uint32_t idesc_qk = make_idesc(CT, false);
                constexpr uint32_t idesc_mn = make_idesc(D, true);              // B with its columns contiguous: V, S
                constexpr uint32_t idesc_kv = idesc_mn | (1u << 15);            // and A with its rows contiguous: K'
                Place<C::STAGES> kat(0), qat(1), vat(V_AT);
                uint32_t it = 0, pc = 0;
                bool ok = true;
                while (ok && enter()) {
                    for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                        const uint32_t ph = it & 1u;
                        const uint64_t q_desc = make_desc(sbase + qat.slot * C::TILE_BYTES, 16, 1024);
                        const uint64_t v_desc = make_desc(sbase + vat.slot * C::TILE_BYTES, HALF_BYTES, 1024);
                        if (!(ok = warp_wait(&ring_full[kat.slot], kat.phase, ab, kWaitRingFull))) break;
                        if (!STATE_ONLY) {
                            if (!(ok = warp_wait(&ring_full[qat.slot], qat.phase, ab, kWaitRingFull))) break;
                            tc_fence_after();
                            const uint64_t k_desc = make_desc(sbase + kat.slot * C::TILE_BYTES, 16, 1024);
                            if (elect_one()) {
#pragma unroll
                                for (int ks = 0; ks < D / 16; ++ks) {
                                    const uint32_t off = (ks >> 2) * HALF_BYTES + (ks & 3) * 32;
                                    umma_ss(tmem_base + COL_SC, q_desc + (off >> 4), k_desc + (off >> 4), idesc_qk, ks > 0 ? 1u : 0u);
                                }
                                umma_commit(sc_full);
                            }
                            __syncwarp();
                        }
                        // ---- K'^T V
                        if (!(ok = warp_wait(&ring_full[vat.slot], vat.phase, ab, kWaitRingFull))) break;
                        if (!(ok = warp_wait(ds_empty, ph ^ 1u, ab, kWaitTensor))) break;
                        for (int e = 0; e < PIECES; ++e, ++pc) {
                            const uint32_t buf = pc & 1u;
                            if (!(ok = warp_wait(&kp_full[buf], (pc >> 1) & 1u, ab, kWaitTensor))) break;
                            tc_fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int t = 0; t < 3; ++t)
                                    umma_ss(tmem_base + COL_DS, make_desc(sbase + C::OFF_KP + buf * PIECE_BYTES + t * TERM_BYTES, PIECE * 128, 1024),
                                            v_desc + ((e * PIECE * 128) >> 4), idesc_kv, e > 0 || t > 0 ? 1u : 0u);
                                umma_commit(&kp_empty[buf]);
                                if (e == PIECES - 1) {
                                    umma_commit(ds_full);
                                    umma_commit(&ring_empty[kat.slot]);
                                    if (STATE_ONLY) umma_commit(&ring_empty[vat.slot]);
                                }
                            }
                            __syncwarp();
                        }
                        if (!ok) break;
                        if (!STATE_ONLY) {
                            // ---- Q S
                            if (!(ok = warp_wait(s_full, ph, ab, kWaitTensor))) break;
                            if (!(ok = warp_wait(o_empty, ph ^ 1u, ab, kWaitTensor))) break;
                            tc_fence_after();
                            const uint64_t s_desc = make_desc(sbase + C::OFF_S, D * 128, 1024);
                            if (elect_one()) {
#pragma unroll
                                for (int ks = 0; ks < D / 16; ++ks) {
                                    const uint32_t off = (ks >> 2) * HALF_BYTES + (ks & 3) * 32;
                                    umma_ss(tmem_base + COL_OI, q_desc + (off >> 4), s_desc + ((ks * 16 * 128) >> 4), idesc_mn, ks > 0 ? 1u : 0u);
                                }
                                umma_commit(s_empty);
                                umma_commit(&ring_empty[qat.slot]);
                            }
                            __syncwarp();
                            // ---- P V
                            if (!(ok = warp_wait(p_full, ph, ab, kWaitTensor))) break;
                            tc_fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int ks = 0; ks < CT / 16; ++ks)
                                    umma_ts(tmem_base + COL_OA, tmem_base + COL_SC + ks * 8, v_desc + ((ks * 16 * 128) >> 4), idesc_mn,
                                            ks > 0 ? 1u : 0u);
                                umma_commit(o_full);
                                umma_commit(&ring_empty[vat.slot]);
                            }
                            __syncwarp();
                        }
                        kat.advance(PER_CHUNK);
                        qat.advance(PER_CHUNK);
                        vat.advance(PER_CHUNK);
                    }
                }
                // nothing issued may still run when tensor memory is released
                if (elect_one()) {
                    umma_commit(drain_bar);
                    drain_wait(drain_bar, 0u, ab);
                }
                __syncwarp();
            }
        } else if (warp == 2) {
            // ======================================= decays ======================================
            uint32_t it = 0;
            bool ok = aligned_ok;
            while (ok && enter()) {
                const int len = tab.len[walk.b];
                const int64_t tok0 = tab.tok0[walk.b];
                auto read = [&](int c, float (&z)[4]) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = c * CT + lane * 4 + j;
                        z[j] = t < len ? log_decay(p.base, tok0 + t, walk.h) : 0.f;
                    }
                };
                float z[4];
                read(walk.c, z);
                for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                    float next[4] = {0.f, 0.f, 0.f, 0.f};
                    if (c + 1 < walk.c_end) read(c + 1, next);
                    double s[4], sum = 0.0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[j] = sum += (double)z[j] * 1.4426950408889634;
                    double before = sum;
#pragma unroll
                    for (int m = 1; m < 32; m <<= 1) {
                        const double o = __shfl_up_sync(0xffffffffu, before, m);
                        if (lane >= m) before += o;
                    }
                    before -= sum;
                    const uint32_t buf = it & 1u;
                    if (!(ok = warp_wait(&dec_empty[buf], ((it >> 1) & 1u) ^ 1u, ab, kWaitTensor))) break;
                    float whole[4], rest[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const double x = before + s[j], w = rint(x);
                        whole[j] = (float)-w;
                        rest[j] = (float)(w - x);
                        z[j] = next[j];
                    }
                    *reinterpret_cast<float4*>(dec + buf * 2 * CT + lane * 4) = make_float4(whole[0], whole[1], whole[2], whole[3]);
                    *reinterpret_cast<float4*>(dec + buf * 2 * CT + CT + lane * 4) = make_float4(rest[0], rest[1], rest[2], rest[3]);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&dec_full[buf]);
                }
            }
        }
    } else if (warp < 8) {
        // ======================================= P and the output ================================
        setmaxnreg_inc<kRegsOut>();
        const int quad = warp & 3, i = quad * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
        uint32_t it = 0;
        bool ok = aligned_ok && !STATE_ONLY;
        while (ok && enter()) {
            const int len = tab.len[walk.b];
            const int64_t tok0 = tab.tok0[walk.b];
            for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                const uint32_t buf = it & 1u, ph = it & 1u;
                if (!(ok = warp_wait(&dec_full[buf], (it >> 1) & 1u, ab, kWaitTensor))) break;
                const float* whole = dec + buf * 2 * CT;                        // negated
                const float* rest = whole + CT;
                const float wi = -whole[i], ri = -rest[i];
                if (!(ok = warp_wait(sc_full, ph, ab, kWaitTensor))) break;
                tc_fence_after();
                const uint64_t wi2 = f2_pack(wi, wi), ri2 = f2_pack(ri, ri);
#pragma unroll
                for (int blk = 0; blk < 4; ++blk) {
                    uint32_t w[16];
                    if (blk <= quad) {
                        float s[32];
                        tmem_ld32(tmem_base + COL_SC + lane_addr + blk * 32, s);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const ulonglong2 wj = *reinterpret_cast<const ulonglong2*>(whole + blk * 32 + j);
                            const ulonglong2 rj = *reinterpret_cast<const ulonglong2*>(rest + blk * 32 + j);
                            float x[4];
                            f2_unpack(f2_add(f2_add(wi2, wj.x), f2_add(ri2, rj.x)), x[0], x[1]);
                            f2_unpack(f2_add(f2_add(wi2, wj.y), f2_add(ri2, rj.y)), x[2], x[3]);
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                x[q] = s[j + q] * ex2_approx(x[q]);
                                if (blk == quad) x[q] = j + q <= lane ? x[q] : 0.f;
                            }
                            w[j / 2] = pack_bf16x2(x[0], x[1]);
                            w[j / 2 + 1] = pack_bf16x2(x[2], x[3]);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j) w[j] = 0u;
                    }
                    tmem_st16(tmem_base + COL_SC + lane_addr + blk * 16, w);
                }
                const float ei = exp2_parts(wi, ri) * p.base.scale;
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(p_full);
                    mbar_arrive(&dec_empty[buf]);
                }
                // ---- output
                if (!(ok = warp_wait(o_full, ph, ab, kWaitTensor))) break;
                tc_fence_after();
                float y[D];
#pragma unroll
                for (int blk = 0; blk < D / 32; ++blk) {
                    float x[32];
                    tmem_ld32(tmem_base + COL_OA + lane_addr + blk * 32, *reinterpret_cast<float(*)[32]>(&y[blk * 32]));
                    tmem_ld32(tmem_base + COL_OI + lane_addr + blk * 32, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) y[blk * 32 + j] = fmaf(ei, x[j], p.base.scale * y[blk * 32 + j]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_empty);
                const int t = c * CT + i;
                const int64_t tok = tok0 + t;
                if (t < len) {
                    const NormGate& nm = p.base.norm;
                    if (nm.on) {
                        float mean = 0.f, sq = 0.f;
                        if (!nm.rms) {
                            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int j = 0; j < D; ++j) part[j & 3] += y[j];
                            mean = ((part[0] + part[1]) + (part[2] + part[3])) * (1.f / D);
                        }
                        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j = 0; j < D; ++j) {
                            y[j] -= mean;
                            part[j & 3] = fmaf(y[j], y[j], part[j & 3]);
                        }
                        sq = (part[0] + part[1]) + (part[2] + part[3]);
                        const float inv = 1.f / sqrtf(sq * (1.f / D) + nm.eps);
#pragma unroll
                        for (int j = 0; j < D; ++j) y[j] *= inv;
                        const int at = walk.h * D;
                        if (nm.gain) {
#pragma unroll
                            for (int j = 0; j < D; j += 8) {
                                float g[8];
                                unpack8(__ldg(reinterpret_cast<const uint4*>(nm.gain + at + j)), g);
#pragma unroll
                                for (int q = 0; q < 8; ++q) y[j + q] *= g[q];
                            }
                        }
                        if (nm.bias) {
#pragma unroll
                            for (int j = 0; j < D; j += 8) {
                                float g[8];
                                unpack8(__ldg(reinterpret_cast<const uint4*>(nm.bias + at + j)), g);
#pragma unroll
                                for (int q = 0; q < 8; ++q) y[j + q] += g[q];
                            }
                        }
                        if (nm.gate) {
                            const uint4* src = reinterpret_cast<const uint4*>(nm.gate + tok * nm.gate_stride + at);
#pragma unroll
                            for (int j = 0; j < D; j += 8) {
                                float g[8];
                                unpack8(__ldg(src + j / 8), g);
#pragma unroll
                                for (int q = 0; q < 8; ++q) y[j + q] *= swish(g[q]);
                            }
                        }
                    }
                    uint4* dst = reinterpret_cast<uint4*>(p.base.o + tok * p.base.o_stride + walk.h * D);
#pragma unroll
                    for (int j = 0; j < D; j += 8) dst[j / 8] = pack8(*reinterpret_cast<float(*)[8]>(&y[j]));
                }
                __syncwarp();
            }
        }
    } else if (warp < 12) {
        // ======================================= state ===========================================
        setmaxnreg_inc<kRegsState>();
        constexpr int N = D == 128 ? 128 : 32;             // channels of a thread (d = 64: two threads a row)
        const int quad = warp & 3, l = quad * 32 + lane, row = l % D, col = (l / D) * N;
        const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
        uint8_t* s_row = smem + C::OFF_S + row * 128;
        uint32_t it = 0;
        bool ok = aligned_ok;
        while (ok && enter()) {
            const int b = walk.b, h = walk.h;
            const bool whole_stream = walk.c == 0 && walk.c_end == walk.chunks;
            float s[N];
            // where the segment's first state is: the stream's own, or what the merge left for this CTA
            const float* src = nullptr;
            if (!STATE_ONLY) {
                if (whole_stream)
                    src = tab.from[b] >= 0 ? p.base.state + ((int64_t)tab.from[b] * p.base.H + h) * (D * D) : nullptr;
                else
                    src = p.part + (int64_t)(walk.c > 0 ? blockIdx.x : p.groups + blockIdx.x) * (D * D);
            }
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                const float4 x = src ? *reinterpret_cast<const float4*>(src + row * D + col + j) : make_float4(0.f, 0.f, 0.f, 0.f);
                s[j] = x.x;
                s[j + 1] = x.y;
                s[j + 2] = x.z;
                s[j + 3] = x.w;
            }
            float all_whole = 0.f;                         // logarithm of the segment's decay
            double all_rest = 0.0;
            for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                const uint32_t buf = it & 1u, ph = it & 1u;
                if (!STATE_ONLY) {
                    if (!(ok = warp_wait(s_empty, ph ^ 1u, ab, kWaitTensor))) break;
#pragma unroll
                    for (int j = 0; j < N; j += 8) {
                        const int ch = (col + j) / 8;
                        *reinterpret_cast<uint4*>(s_row + (ch >> 3) * (D * 128) + (((ch & 7) ^ (row & 7)) << 4)) =
                            pack8(*reinterpret_cast<float(*)[8]>(&s[j]));
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(s_full);
                }
                if (!(ok = warp_wait(&dec_full[buf], (it >> 1) & 1u, ab, kWaitTensor))) break;
                const float whole = -dec[buf * 2 * CT + CT - 1], rest = -dec[buf * 2 * CT + 2 * CT - 1];
                __syncwarp();
                if (lane == 0) mbar_arrive(&dec_empty[buf]);
                const float keep = exp2_parts(whole, rest);
                if (STATE_ONLY) {
                    all_whole += whole;
                    all_rest += (double)rest;
                }
                if (!(ok = warp_wait(ds_full, ph, ab, kWaitTensor))) break;
                tc_fence_after();
#pragma unroll
                for (int blk = 0; blk < N / 32; ++blk) {
                    float x[32];
                    tmem_ld32(tmem_base + COL_DS + lane_addr + col + blk * 32, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) s[blk * 32 + j] = fmaf(keep, s[blk * 32 + j], x[j]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(ds_empty);
            }
            if (!ok) break;
            float* dst = nullptr;
            if (STATE_ONLY)
                dst = p.part + (int64_t)(blockIdx.x + 1) * (D * D);
            else if (walk.c_end == walk.chunks && tab.to[b] >= 0)
                dst = p.base.state + ((int64_t)tab.to[b] * p.base.H + h) * (D * D);
            if (dst) {
#pragma unroll
                for (int j = 0; j < N; j += 4)
                    *reinterpret_cast<float4*>(dst + row * D + col + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
            }
            if (STATE_ONLY && l == 0) p.part_keep[blockIdx.x + 1] = exp2f(all_whole) * (float)exp2(all_rest);
        }
    } else {
        // ======================================= K' ==============================================
        setmaxnreg_dec<kRegsKeys>();
        const int l = threadIdx.x & 127, row = l >> 3, ch = l & 7;
        const uint32_t at = row * 128 + ((ch ^ (row & 7)) << 4);       // inside a piece's half; the same in a tile's
        Place<C::STAGES> kat(0), vat(V_AT);
        uint32_t it = 0, pc = 0;
        bool ok = aligned_ok;
        while (ok && enter()) {
            const int len = tab.len[walk.b];
            for (int c = walk.c; ok && c < walk.c_end; ++c, ++it) {
                const uint32_t buf = it & 1u;
                const int valid = len - c * CT;            // tokens of the sequence from here on
                if (!(ok = warp_wait(&dec_full[buf], (it >> 1) & 1u, ab, kWaitTensor))) break;
                const float* whole = dec + buf * 2 * CT;
                const float* rest = whole + CT;
                const float w_end = whole[CT - 1], r_end = rest[CT - 1];
                if (!(ok = warp_wait(&ring_full[kat.slot], kat.phase, ab, kWaitRingFull))) break;
                if (valid < CT) {
                    // rows behind the sequence are the next one's, or none: they may hold anything, and 0 times that is not 0
                    if (!(ok = warp_wait(&ring_full[vat.slot], vat.phase, ab, kWaitRingFull))) break;
                    if (l >= valid) {
#pragma unroll
                        for (int q = 0; q < 8 * C::HALVES; ++q)
                            *reinterpret_cast<uint4*>(smem + vat.slot * C::TILE_BYTES + (q >> 3) * HALF_BYTES + l * 128 + (q & 7) * 16) =
                                make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                for (int e = 0; e < PIECES; ++e, ++pc) {
                    const uint32_t pb = pc & 1u;
                    const int j = e * PIECE + row;
                    const float w = exp2_parts(whole[j] - w_end, rest[j] - r_end);
                    if (!(ok = warp_wait(&kp_empty[pb], ((pc >> 1) & 1u) ^ 1u, ab, kWaitTensor))) break;
                    const uint8_t* src = smem + kat.slot * C::TILE_BYTES + e * (PIECE * 128) + at;
                    uint8_t* dst = smem + C::OFF_KP + pb * PIECE_BYTES + at;
#pragma unroll
                    for (int hf = 0; hf < C::HALVES; ++hf) {
                        float x[8], y[8];
                        unpack8(*reinterpret_cast<const uint4*>(src + hf * HALF_BYTES), x);
#pragma unroll
                        for (int q = 0; q < 8; ++q) x[q] = j < valid ? w * x[q] : 0.f;
#pragma unroll
                        for (int t = 0; t < 3; ++t) {
                            const uint4 part = pack8(x);
                            *reinterpret_cast<uint4*>(dst + t * TERM_BYTES + hf * (PIECE * 128)) = part;
                            // d = 64: the instruction's upper 64 rows are the same ones again (the second threads of the state's rows read them)
                            if (D == 64) *reinterpret_cast<uint4*>(dst + t * TERM_BYTES + PIECE * 128) = part;
                            if (t < 2) {
                                unpack8(part, y);
#pragma unroll
                                for (int q = 0; q < 8; ++q) x[q] -= y[q];
                            }
                        }
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&kp_full[pb]);
                }
                if (!ok) break;
                __syncwarp();
                if (lane == 0) mbar_arrive(&dec_empty[buf]);
                kat.advance(PER_CHUNK);
                vat.advance(PER_CHUNK);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// States at the cuts of a stream that several CTAs share.  A block owns some elements of one such stream: from the stream's first state on, every
// CTA's part (its local state, from zero) is added to what decays from before, in the order of the CTAs.  Slot g: the state that CTA g
// starts from (the state-only pass left CTA g - 1's part there); slot groups + g: a copy of the first state of the stream
// that begins in CTA g (the pool's may be overwritten while others still run).
constexpr int kMergeThreads = 256;
template <int D, class Table>
__global__ void __launch_bounds__(kMergeThreads)
gret_merge_kernel(const GretChunkParams p, const __grid_constant__ Table tab) {
    const int g0 = blockIdx.x + 1;                         // first CTA that starts inside the stream
    const int64_t H = p.base.H, pos = (int64_t)g0 * p.total / p.groups, per = pos / H;
    int lo = 0, hi = p.base.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.chunk0[mid] <= per) lo = mid; else hi = mid - 1;
    }
    const int64_t base = (int64_t)tab.chunk0[lo] * H, chunks = tab.chunk0[lo + 1] - tab.chunk0[lo], h = (pos - base) / chunks;
    const int64_t begin = base + h * chunks, end = begin + chunks;
    if (pos == begin || (int64_t)(g0 - 1) * p.total / p.groups > begin) return;       // no cut, or not the stream's first one
    const int at = (blockIdx.y * kMergeThreads + threadIdx.x) * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tab.from[lo] >= 0) s = *reinterpret_cast<const float4*>(p.base.state + ((int64_t)tab.from[lo] * H + h) * (D * D) + at);
    *reinterpret_cast<float4*>(p.part + (int64_t)(p.groups + g0 - 1) * (D * D) + at) = s;
    for (int g = g0; g < p.groups && (int64_t)g * p.total / p.groups < end; ++g) {
        float4* slot = reinterpret_cast<float4*>(p.part + (int64_t)g * (D * D) + at);
        const float keep = p.part_keep[g];
        const float4 x = *slot;
        s.x = fmaf(keep, s.x, x.x);
        s.y = fmaf(keep, s.y, x.y);
        s.z = fmaf(keep, s.z, x.z);
        s.w = fmaf(keep, s.w, x.w);
        *slot = s;
    }
}

template <int D, class Table>
cudaError_t launch_one(const GretChunkParams& p, const Table& tab, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                       cudaStream_t stream) {
    if (p.split) {
        gret_chunk_kernel<D, true><<<p.groups, kThreads, GCfg<D>::SMEM_BYTES, stream>>>(tmQ, tmK, tmV, p, tab);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        gret_merge_kernel<D><<<dim3(p.groups - 1, D * D / (4 * kMergeThreads)), kMergeThreads, 0, stream>>>(p, tab);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    gret_chunk_kernel<D, false><<<p.groups, kThreads, GCfg<D>::SMEM_BYTES, stream>>>(tmQ, tmK, tmV, p, tab);
    return cudaGetLastError();
}

template <int D, bool STATE_ONLY>
cudaError_t setup_one() {
    cudaError_t e = cudaFuncSetAttribute(gret_chunk_kernel<D, STATE_ONLY, GretChunkTable>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         GCfg<D>::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(gret_chunk_kernel<D, STATE_ONLY, GretChunkTableOf<kFewSequences>>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, GCfg<D>::SMEM_BYTES);
}

}  // namespace

cudaError_t gret_chunk_kernel_setup() {
    cudaError_t e = setup_one<128, false>();
    if (e != cudaSuccess) return e;
    if ((e = setup_one<128, true>()) != cudaSuccess) return e;
    if ((e = setup_one<64, false>()) != cudaSuccess) return e;
    return setup_one<64, true>();
}

cudaError_t launch_gret_chunk(const GretChunkParams& p, const GretChunkTable& tab, const CUtensorMap& tmQ, const CUtensorMap& tmK,
                              const CUtensorMap& tmV, cudaStream_t stream) {
    if (p.groups <= 0) return cudaSuccess;
    auto launch = [&](const auto& t) {
        return p.base.d == 128 ? launch_one<128>(p, t, tmQ, tmK, tmV, stream) : launch_one<64>(p, t, tmQ, tmK, tmV, stream);
    };
    if (p.base.B > kFewSequences) return launch(tab);
    GretChunkTableOf<kFewSequences> few;
    std::memcpy(few.from, tab.from, sizeof few.from);
    std::memcpy(few.to, tab.to, sizeof few.to);
    std::memcpy(few.tok0, tab.tok0, sizeof few.tok0);
    std::memcpy(few.len, tab.len, sizeof few.len);
    std::memcpy(few.chunk0, tab.chunk0, sizeof few.chunk0);
    return launch(few);
}

}  // namespace yoco
