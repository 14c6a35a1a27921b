// Multi-token chunk / full-sequence attention on the tcgen05 tensor cores, two row tiles per CTA.
//
// One CTA owns 256 of the G*T query rows of a (sequence, KV head) stream, as two 128-row tiles
// that share every K/V tile brought into shared memory, and walks a contiguous range of 128-key
// tiles.  Three warpgroups (384 threads):
//   warpgroup 0   warp 0 = TMA producer (both Q tiles once per segment; K through a three-deep and
//                 V through a two-deep ring), warps 1 and 2 = issuers of all tensor-core products of
//                 row tiles 0 and 1; gives most of its registers away
//   warpgroup 1   softmax of row tile 0 (thread = query row)
//   warpgroup 2   softmax of row tile 1
// Every 128-key tile is processed as two 64-key half steps.  Tensor memory (512 columns):
//   S_0^0 S_0^1 | S_1^0 S_1^1 | O_0 | O_1      (64 fp32 columns per S buffer, 128 per O)
// S_r^h receives the scores of row tile r against half h of the key tile, so the scores of the
// next half step are already being computed while a warpgroup works on the current one.  A softmax
// thread reads its S row, keeps the running max / sum, and writes P (bf16, two per 32-bit column)
// over the first 32 columns of the same S buffer; O_r += P_r V then takes P straight from tensor
// memory as the A operand, so P never touches shared memory.  The issuer of a row tile puts the
// next score product of a buffer right behind the P V product that reads it: the tensor pipe runs
// the products of one thread in the order issued, so the buffer needs no barrier round trip between
// the two.  O in tensor memory is rescaled only when a row max outgrew the reference by more than 2^8.
// Every wait is bounded and reports through the status word.
//
// FP8 = true reads an 8-bit cache (FP8 E4M3 bytes, one fp32 scale per KV head, head dimension 128):
// the producer brings a 128-key tile of bytes (16 KB) into the upper half of a ring stage, a fourth
// warpgroup (512 threads then; one warp per scheduler, 32 rows of every tile each)
// widens it in place to fp16 in the layout the tensor-core descriptors read (every E4M3 value is an
// fp16 value, so this is exact; row r of the bytes sits exactly where row r of the second 64-channel
// half goes, so a thread only ever overwrites its own source row), Q is converted bf16 -> fp16 in
// place once per segment, P is rounded to fp16, and all products run fp16 x fp16.  k_scale folds
// into the softmax scale, v_scale multiplies the normalised output.
//
// A paged cache (kPaged16: bf16 rows, kPaged4: 4-bit rows) differs in where the producer finds the rows of a tile
// (page_map.cuh).  4-bit rows take the way of the 8-bit cache: the 32 rows of a widening warp land, codes and scales,
// inside the part of the upper half tile that the same warp's fp16 rows will fill, so a warp has read all of its
// source (one __syncwarp) before it overwrites any of it, and no two warps meet.
// A value (code - 8) * scale has up to 14 bits, three more than fp16 holds.  V takes one rounding (half a step, 2^-11
// of the value; O leaves in bf16).  K takes none: every key tile becomes two, (code - 8) times the upper eight bits of the
// scale and times its lower three, both exact in fp16, and the scores are the sum of two products.  (Rounded once, K puts a
// score off by up to 2^-11 of the sum of its products' magnitudes.  Flat softmax rows of many keys average that out, rows that a
// few keys lead do not, whatever their length: log-sum-exp 0.035 off, O 0.032, for 6,000 keys with scores of some hundreds.)
// The second part has a place of its own, written and given back by halves of 64 keys, so that a half's part can be
// written as soon as both row tiles have scored the same half of the tile before; K's ring is two deep for it.
// The polynomial exponentials are quartic (no time lost); the log-sum-exp of a few keys is then within 1.6e-7 (2-norm, chunks of
// 11 to 41 tokens over as many keys) of 64 bits.
// Bound by the softmax warps (as over a bf16 cache, 407 us) and by 1.5 times the products.  Kernel alone at the full clock, 391
// tokens over 65,927 keys, 32 query over 8 KV heads: 570 us = 740 TFLOP/s counted once (K rounded: 470; K in two parts
// through two entries of the three-deep ring: 812); 670 us a call in a loop of seconds, where the power cap takes the clock
// down (K rounded: 556).  A whole sequence of 4,096 tokens 500 us.
// V rows that a window has left behind are zeroed where they are widened: the softmax warps, which zero the rows
// past the end, have no register left for it.
#include <cuda_fp16.h>

#include "kernels.h"
#include "page_map.cuh"
#include "ptx.cuh"
#include "q4.cuh"
#include "tcgen05.cuh"

namespace yoco {

namespace {

constexpr int BM = 128;                        // rows of one tensor-core tile
constexpr int BN = kChunkTileN;                // 128 keys per shared-memory tile
constexpr int BH = BN / 2;                     // keys per half step
enum CacheKind { kPacked16, kPacked8, kPaged16, kPaged4 };
// caches whose tiles are widened to fp16 on the way
__host__ __device__ constexpr bool widened(CacheKind kind) { return kind == kPacked8 || kind == kPaged4; }
// three warpgroups for a bf16 cache; a fourth one widens the tiles of a narrow cache
template <bool FP8>
constexpr int kThreadsOf = FP8 ? 512 : 384;
// a widening warp's share of a 4-bit tile as it arrives: 32 rows of codes, then their scales
constexpr int Q4_WARP_STRIDE = 32 * 128;       // from one warp's share to the next: its rows of the half tile
constexpr int Q4_OFF_SCALE = 32 * 64;
constexpr int Q4_ROW_BYTES = 64 + 8;
constexpr int HALF_BYTES = 128 * 128;          // 128 rows x 64 bf16: one swizzled half tile
constexpr uint32_t TMEM_COLS = 512;
constexpr float kRescaleThreshold = 8.f;       // in log2 units: P stays below 2^8
// fp16 P is kept 2^7 larger, at most 2^15: the weights of many keys behind one that leads by 16 to 23 octaves, which may be most of a
// row's sum, would otherwise fall among fp16's subnormals and lose their bits (90,000 keys 20.6 octaves behind: O 2.6 % off).
__host__ __device__ constexpr float p_shift(CacheKind kind) { return widened(kind) ? 7.f : 0.f; }
// Register split after launch.  The CTA starts with what its thread count allows (168 registers per
// thread for 384 threads, 128 for 512); warpgroup 0 (and the widening warpgroup) give back down to
// kOther / kWiden and the softmax warpgroups grow to kSoftmax.  The total must fit in what the CTA
// was launched with, or the request to grow would never be granted.
template <bool FP8>
struct Regs {
    static constexpr int kLaunch = FP8 ? 128 : 168, kSoftmax = FP8 ? 192 : 224, kOther = 56, kWiden = 64;
    static_assert(128 * kOther + 256 * kSoftmax + (FP8 ? 128 * kWiden : 0) <= kLaunch * kThreadsOf<FP8>,
                  "register pool of the CTA");
};

template <int D>
struct PCfg {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;     // one Q, K or V tile
    static constexpr int K_STAGES = 3, V_STAGES = 2;
    static constexpr int OFF_Q = 0;                            // two tiles
    static constexpr int OFF_K = OFF_Q + 2 * TILE_BYTES;
    static constexpr int OFF_V = OFF_K + K_STAGES * TILE_BYTES;
    static constexpr int OFF_BAR = OFF_V + V_STAGES * TILE_BYTES;
    static constexpr int K_STAGES_4BIT = 2;                    // the third place takes the second part of K
    static constexpr int OFF_K_LOWER = OFF_K + K_STAGES_4BIT * TILE_BYTES;
    static constexpr int NUM_BARS = 2 + 2 * K_STAGES + 2 * V_STAGES + 12 + 3 + (2 * K_STAGES_4BIT + V_STAGES + 1) + 2;
    static constexpr int SMEM_BYTES = OFF_BAR + NUM_BARS * 8 + 16;
    static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
};

// Which of the 16 score pairs of a 32-key chunk take their exponential on the FMA pipe (a cubic, see
// f2_exp2_poly) instead of the special-function unit (16 results per clock per SM), spread evenly so
// that the two instruction streams interleave.  Measured on the 32K-cache chunk case with the turns
// described below in place, 0 / 2 / 4 of 16: 974 / 1,055 / 1,125 TFLOP/s.
constexpr int kPolyPairs = 4;
__host__ __device__ constexpr bool poly_pair(int j) {
    return ((j + 1) * kPolyPairs) / 16 != (j * kPolyPairs) / 16;
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
// two E4M3 bytes (low byte first) -> two fp16 (exact)
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two_bytes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two_bytes));
    return r;
}
// two bf16 -> two fp16 (round to nearest; |x| < 65504 required of Q)
__device__ __forceinline__ uint32_t bf16x2_to_f16x2(uint32_t w) {
    return pack_f16x2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

// tmKs, tmVs: maps of the scales of 4-bit rows (otherwise not read)
template <int D, CacheKind KIND>
__global__ void __launch_bounds__(kThreadsOf<widened(KIND)>, 1)
chunk_pair_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmKs, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ CUtensorMap tmVs, const ChunkParams p,
                  const __grid_constant__ ChunkFp8Scales sc) {
    constexpr bool FP8 = widened(KIND);            // fp16 products, widening warpgroup
    static_assert(!FP8 || D == 128, "the narrow cache paths are built for head dimension 128");
    using C = PCfg<D>;
    constexpr int HALVES = C::HALVES;
    constexpr int KS = KIND == kPaged4 ? C::K_STAGES_4BIT : C::K_STAGES, VS = C::V_STAGES;
    constexpr int K_READY = KIND == kPaged4 ? 2 * KS : KS;      // 4-bit rows: a tile is ready by halves
    constexpr int KSTEPS_QK = D / 16;
    constexpr int KSTEPS_PV = BH / 16;

    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
    uint64_t* q_full = bars + 0;
    uint64_t* q_empty = bars + 1;
    uint64_t* k_full = bars + 2;             // [KS]
    uint64_t* k_empty = k_full + KS;         // [KS]
    uint64_t* v_full = k_empty + KS;         // [VS]
    uint64_t* v_empty = v_full + VS;         // [VS]
    uint64_t* s_full = v_empty + VS;         // [2][2]  S_r^h holds the scores of the current half step
    uint64_t* p_full = s_full + 4;           // [2][2]  P_r^h has been written over S_r^h
    uint64_t* pv_done = p_full + 4;          // [2][2]  O_r includes the current half step; P_r^h is dead
    uint64_t* drain_bar = pv_done + 4;       // [3]     everything issuer warp 1 + i started has finished
    uint64_t* k_ready = drain_bar + 3;       // [KS]    8-bit cache: the K tile has been widened to fp16 (4-bit: [KS][2], by halves)
    uint64_t* v_ready = k_ready + K_READY;   // [VS]    ... the V tile
    uint64_t* q_ready = v_ready + VS;        //         ... both Q tiles have been converted to fp16
    uint64_t* low_empty = q_ready + 1;       // [2]     4-bit rows: both row tiles have scored this half of K's second part
    // what the issuers and the softmax warpgroups wait on for an operand tile
    uint64_t* k_use = FP8 ? k_ready : k_full;
    uint64_t* v_use = FP8 ? v_ready : v_full;
    uint64_t* q_use = FP8 ? q_ready : q_full;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = blockIdx.x / p.m_tiles, m_tile = blockIdx.x - group * p.m_tiles;
    const int seg_lo = p.group_begin[group], seg_hi = p.group_begin[group + 1];
    const Abort ab{abort_flag, p.status, kWaitLimitNs};
    constexpr bool PAGED = KIND == kPaged16 || KIND == kPaged4;
    const bool aligned_ok = (smem_u32(smem) & 1023u) == 0;

    if (threadIdx.x == 0) {
        *abort_flag = aligned_ok ? 0 : 1;
        if (!aligned_ok) atomicCAS(p.status, 0, status_word(kWaitMisaligned, linear_cta()));
        mbar_init(q_full, 1);
        mbar_init(q_empty, 2);
        for (int b = 0; b < 3; ++b) mbar_init(&drain_bar[b], 1);
        for (int b = 0; b < K_READY; ++b) mbar_init(&k_ready[b], KIND == kPaged4 ? 2 : 4);
        for (int b = 0; b < VS + 1; ++b) mbar_init(&v_ready[b], 4);           // the four widening warps (q_ready follows)
        for (int b = 0; b < 2; ++b) mbar_init(&low_empty[b], 2);
        for (int b = 0; b < KS; ++b) {
            mbar_init(&k_full[b], 1);
            mbar_init(&k_empty[b], 2);            // released by both issuers
        }
        for (int b = 0; b < VS; ++b) {
            mbar_init(&v_full[b], 1);
            mbar_init(&v_empty[b], 2);            // released by both issuers
        }
        for (int r = 0; r < 2; ++r) {
            for (int h = 0; h < 2; ++h) {
                mbar_init(&s_full[r * 2 + h], 1);
                mbar_init(&p_full[r * 2 + h], 4);
                mbar_init(&pv_done[r * 2 + h], 1);
            }
        }
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

    if (warp < 4) {
        setmaxnreg_dec<Regs<FP8>::kOther>();
        if (warp == 0 && (PAGED || lane == 0) && aligned_ok) {
            // =================================== TMA producer ================================
            // (a whole warp when the cache is paged: the lanes keep the page numbers)
            if (lane == 0) {
                tma_prefetch_desc(&tmQ);
                tma_prefetch_desc(&tmK);
                tma_prefetch_desc(&tmV);
            }
            auto wait = [&](uint64_t* bar, uint32_t parity) {
                return PAGED ? warp_wait(bar, parity, ab, kWaitRingEmpty) : wait_or_abort(bar, parity, ab, kWaitRingEmpty);
            };
            uint32_t it = 0;
            uint32_t q_armed = 0, k_armed = 0, v_armed = 0;   // copies started, for the drain on the way out
            bool ok = true;
            for (int si = seg_lo; si < seg_hi && ok; ++si) {
                const DevSegment seg = p.segments[si];
                if (seg.k_end <= seg.k_begin) continue;
                if (!(ok = wait(q_empty, (q_armed & 1u) ^ 1u))) break;
                ++q_armed;
                if (lane == 0) {
                    mbar_expect_tx(q_full, 2 * C::TILE_BYTES);
                    for (int r = 0; r < 2; ++r)
                        for (int h = 0; h < HALVES; ++h)
                            tma_load_2d(smem + C::OFF_Q + r * C::TILE_BYTES + h * HALF_BYTES, &tmQ, h * 64,
                                        seg.q_row0 + (m_tile * 2 + r) * BM, q_full);
                }
                PageCursor<BN> pc;
                if (PAGED) pc.start(p.pages, seg.stream, seg.k_begin, seg.k_end, first_seen(seg.n_full, p.window), ab.status);
                // the boxes of one tile of a paged cache
                auto load_pages = [&](uint8_t* tile, const CUtensorMap& tm, const CUtensorMap& tmS, uint64_t* bar, int k0) {
                    const int n_box = pc.enter(k0), rows = pc.box_rows();
                    for (int j = 0; j < n_box; ++j) {
                        const int row = pc.row(k0, j);
                        if (elect_one()) {
                            if (j == 0) mbar_expect_tx(bar, n_box * rows * (KIND == kPaged4 ? Q4_ROW_BYTES : D * 2));
                            if (KIND == kPaged4) {
                                const int box = min(rows, 32);           // no box spans two widening warps' rows
                                for (int i = 0; i < rows; i += box) {
                                    const int at = j * rows + i;
                                    uint8_t* dst = tile + HALF_BYTES + (at >> 5) * Q4_WARP_STRIDE;
                                    tma_load_2d(dst + (at & 31) * 64, &tm, 0, (row + i) >> 1, bar);
                                    tma_load_2d(dst + Q4_OFF_SCALE + (at & 31) * 8, &tmS, 0, (row + i) >> 4, bar);
                                }
                            } else {
                                for (int h = 0; h < HALVES; ++h)
                                    tma_load_2d(tile + h * HALF_BYTES + j * rows * 128, &tm, h * 64, row, bar);
                            }
                        }
                        __syncwarp();
                    }
                };
                for (int k0 = seg.k_begin; k0 < seg.k_end; k0 += BN, ++it) {
                    const int row = seg.kv_row0 + (k0 - seg.k_begin);
                    const uint32_t kb = it % KS, kn = it / KS;
                    if (!(ok = wait(&k_empty[kb], (kn & 1u) ^ 1u))) break;
                    ++k_armed;
                    if (PAGED) {
                        load_pages(smem + C::OFF_K + kb * C::TILE_BYTES, tmK, tmKs, &k_full[kb], k0);
                    } else if (FP8) {      // 128 keys x 128 bytes into the upper half of the stage
                        mbar_expect_tx(&k_full[kb], HALF_BYTES);
                        tma_load_2d(smem + C::OFF_K + kb * C::TILE_BYTES + HALF_BYTES, &tmK, 0, row, &k_full[kb]);
                    } else {
                        mbar_expect_tx(&k_full[kb], C::TILE_BYTES);
                        for (int h = 0; h < HALVES; ++h)
                            tma_load_2d(smem + C::OFF_K + kb * C::TILE_BYTES + h * HALF_BYTES, &tmK, h * 64, row,
                                        &k_full[kb]);
                    }
                    const uint32_t vb = it % VS, vn = it / VS;
                    if (!(ok = wait(&v_empty[vb], (vn & 1u) ^ 1u))) break;
                    ++v_armed;
                    if (PAGED) {
                        load_pages(smem + C::OFF_V + vb * C::TILE_BYTES, tmV, tmVs, &v_full[vb], k0);
                    } else if (FP8) {
                        mbar_expect_tx(&v_full[vb], HALF_BYTES);
                        tma_load_2d(smem + C::OFF_V + vb * C::TILE_BYTES + HALF_BYTES, &tmV, 0, row, &v_full[vb]);
                    } else {
                        mbar_expect_tx(&v_full[vb], C::TILE_BYTES);
                        for (int h = 0; h < HALVES; ++h)
                            tma_load_2d(smem + C::OFF_V + vb * C::TILE_BYTES + h * HALF_BYTES, &tmV, h * 64, row,
                                        &v_full[vb]);
                    }
                }
            }
            // Every copy this thread started must have landed before the CTA may end (at once when all
            // went well: the tiles were consumed long ago).
            bool drained = lane != 0 || q_armed == 0 || drain_wait(q_full, (q_armed - 1) & 1u, ab);
            for (uint32_t k = k_armed > (uint32_t)KS ? k_armed - KS : 0; lane == 0 && drained && k < k_armed; ++k)
                drained = drain_wait(&k_full[k % KS], (k / KS) & 1u, ab);
            for (uint32_t k = v_armed > (uint32_t)VS ? v_armed - VS : 0; lane == 0 && drained && k < v_armed; ++k)
                drained = drain_wait(&v_full[k % VS], (k / VS) & 1u, ab);
        } else if ((warp == 1 || warp == 2) && aligned_ok) {
            // =================================== MMA issuers =================================
            // Warp 1 + r issues every product of row tile r, half step by half step:
            //   O_r += P_r^h V^h  (key tile j)   and right behind it   S_r^h = Q_r K^h^T  (key tile j + 1).
            // The score product overwrites the buffer P_r^h sits in; the tensor pipe runs the products
            // of one thread in the order issued, so no wait (and no hand-over between two warps) is
            // needed between the two, which takes one barrier round trip out of the cycle
            // scores -> softmax -> P V -> next scores of every buffer.  The whole warp walks the
            // schedule (addresses and descriptors stay warp-uniform) and one elected lane issues:
            // issued from a diverged lane the same instructions cost several times as much.
            const int r = warp - 1;
            constexpr uint32_t idesc_qk = make_idesc(BH, false, FP8);
            constexpr uint32_t idesc_pv = make_idesc(D, true, FP8);
            const uint32_t sbase = smem_u32(smem);
            const uint32_t q_lo = desc_lo(sbase + C::OFF_Q + r * C::TILE_BYTES, 16);
            const uint32_t tmem_o = tmem_base + 2 * BN + r * BN;
            bool ok = true;
            uint32_t it = 0, n_seg = 0;
            auto k_there = [&](uint32_t tile) {      // the whole key tile
                return warp_wait(&k_use[tile % KS], (tile / KS) & 1u, ab, kWaitRingFull);
            };
            auto k_half_there = [&](uint32_t tile, int h) {      // 4-bit rows
                return warp_wait(&k_ready[(tile % KS) * 2 + h], (tile / KS) & 1u, ab, kWaitRingFull);
            };

            // scores of half h of a key tile (it must have landed)
            auto issue_scores = [&](uint32_t tile, int h, bool last_of_segment) {
                const uint32_t kb = tile % KS;
                tc_fence_after();
                // (4-bit rows: ... plus the lower bits of the scales)
                uint32_t k_lo = desc_lo(sbase + C::OFF_K + kb * C::TILE_BYTES + h * BH * 128, 16);
                if (elect_one()) {
#pragma unroll 1
                    for (int part = 0; part < (KIND == kPaged4 ? 2 : 1); ++part) {
#pragma unroll
                        for (int ks = 0; ks < KSTEPS_QK; ++ks) {
                            const uint32_t off = ((ks >> 2) * HALF_BYTES + (ks & 3) * 32) >> 4;
                            umma_ss(tmem_base + r * BN + h * BH, desc_from_lo(q_lo + off, 1024),
                                    desc_from_lo(k_lo + off, 1024), idesc_qk, part + ks > 0 ? 1u : 0u);
                        }
                        k_lo = desc_lo(sbase + C::OFF_K_LOWER + h * BH * 128, 16);
                    }
                    umma_commit(&s_full[r * 2 + h]);
                    if (KIND == kPaged4) umma_commit(&low_empty[h]);
                    if (h == 1) {
                        umma_commit(&k_empty[kb]);
                        if (last_of_segment) umma_commit(q_empty);   // this row tile's Q may be replaced
                    }
                }
                __syncwarp();
            };

            for (int si = seg_lo; si < seg_hi && ok; ++si) {
                const int n_tiles = (p.segments[si].k_end - p.segments[si].k_begin + BN - 1) / BN;
                if (n_tiles <= 0) continue;
                // both halves of the first key tile of the segment (its Q and K have to be there)
                if (!(ok = warp_wait(q_use, n_seg & 1u, ab, kWaitRingFull))) break;
                ++n_seg;
                if (!(ok = KIND == kPaged4 ? k_half_there(it, 0) : k_there(it))) break;
                issue_scores(it, 0, n_tiles == 1);
                if (KIND == kPaged4 && !(ok = k_half_there(it, 1))) break;
                issue_scores(it, 1, n_tiles == 1);
                for (int t = 0; t < n_tiles && ok; ++t, ++it) {
                    const uint32_t vb = it % VS;
                    if (!(ok = warp_wait(&v_use[vb], (it / VS) & 1u, ab, kWaitRingFull))) break;
                    const bool more = t + 1 < n_tiles;
                    if (KIND != kPaged4 && more && !(ok = k_there(it + 1))) break;
#pragma unroll (KIND == kPaged4 ? 1 : 2)     // (4-bit rows: unrolled, the issuers spill)
                    for (int h = 0; h < 2; ++h) {
                        if (!(ok = warp_wait(&p_full[r * 2 + h], it & 1u, ab, kWaitTensor))) break;
                        tc_fence_after();
                        const uint32_t v_lo = desc_lo(sbase + C::OFF_V + vb * C::TILE_BYTES + h * BH * 128, BN * 128);
                        const uint32_t a_tmem = tmem_base + r * BN + h * BH;
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < KSTEPS_PV; ++ks)
                                umma_ts(tmem_o, a_tmem + ks * 8,
                                        desc_from_lo(v_lo + ((uint32_t)(ks * 16 * 128) >> 4), 1024), idesc_pv,
                                        (t == 0 && h == 0 && ks == 0) ? 0u : 1u);
                            umma_commit(&pv_done[r * 2 + h]);
                            if (h == 1) umma_commit(&v_empty[vb]);
                        }
                        __syncwarp();
                        if (KIND == kPaged4 && more && !(ok = k_half_there(it + 1, h))) break;
                        if (more) issue_scores(it + 1, h, t + 2 == n_tiles);
                    }
                }
            }
            // Nothing this warp issued may still be running (or still owe an arrive on one of this CTA's
            // barriers) when tensor memory is released and the CTA ends: one more commit, which
            // completes after every earlier product and commit of the issuing lane, and a wait for it.
            if (elect_one()) {
                umma_commit(&drain_bar[r]);
                drain_wait(&drain_bar[r], 0u, ab);
            }
            __syncwarp();
        }
    } else if (FP8 && warp >= 12) {
        // ======================================= widening warpgroup (8-bit cache) ============
        // Four warps, one per scheduler: the conversion instruction runs at a few lanes per clock and
        // scheduler, and one warp alone could not keep up with the tensor pipe (measured: 913 TFLOP/s on
        // the 32K-cache case with one widening warp, 1,100 with the V tiles left unwidened).  Warp w
        // handles rows 32 w .. 32 w + 31 of every tile, one row per lane.
        setmaxnreg_dec<Regs<FP8>::kWiden>();
        const int wq = warp - 12;
        if (aligned_ok) {
            // The bytes of row r were written by TMA with the 128-byte swizzle (16-byte chunk c at position
            // c ^ (r & 7)); the fp16 row goes out in the same swizzle, channels 0-63 to row r of the lower
            // half tile and 64-127 to row r of the upper one, i.e. over the bytes just read.
            // 4-bit rows: in_two, a tile of K becomes two (see the head of this file); dead, this lane's row holds anything
            // and must come out as zeros.  (Both parts are written from one unpacking: a loop of two keeps the unpacked
            // row, 64 registers, or unpacks it twice.)
            auto widen_tile = [&](uint8_t* tile, bool in_two, bool dead) {
                if (KIND == kPaged4) {
                    const int rr = wq * 32 + lane;
                    const uint8_t* src = tile + HALF_BYTES + wq * Q4_WARP_STRIDE;
                    uint4 raw[4];          // 32 channels each; two rows to a 128-byte line, 128-byte swizzle
                    const int line = lane >> 1, first = (lane & 1) << 2;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        raw[c] = *reinterpret_cast<const uint4*>(src + line * 128 + (((first | c) ^ (line & 7)) << 4));
                    const uint2 sw = dead ? make_uint2(0u, 0u) : *reinterpret_cast<const uint2*>(src + Q4_OFF_SCALE + lane * 8);
                    uint32_t s2[4] = {__byte_perm(sw.x, 0u, 0x1010), __byte_perm(sw.x, 0u, 0x3232),
                                      __byte_perm(sw.y, 0u, 0x1010), __byte_perm(sw.y, 0u, 0x3232)};
                    const uint32_t magic = q4_magic();
                    __syncwarp();          // every lane has its source before any row is written
                    // a key's scales: the upper eight bits, and the three below them
                    uint32_t lower[4];
                    if (in_two) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t upper = s2[c] & 0xFFF8FFF8u;
                            lower[c] = h2_sub(s2[c], upper);
                            s2[c] = upper;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t w[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) {                // channels 32 c + 8 q .. + 7: one 16-byte chunk
                            const uint32_t l0 = q4_signed_lo(w[q], magic), h0 = q4_signed_hi(w[q], magic);             // (0, 4), (1, 5)
                            const uint32_t l1 = q4_signed_lo(w[q] >> 8, magic), h1 = q4_signed_hi(w[q] >> 8, magic);   // (2, 6), (3, 7)
                            const uint32_t n[4] = {__byte_perm(l0, h0, 0x5410), __byte_perm(l1, h1, 0x5410), __byte_perm(l0, h0, 0x7632),
                                                   __byte_perm(l1, h1, 0x7632)};
                            const int c0 = (c & 1) * 4 + q, at = (c >> 1) * HALF_BYTES + rr * 128 + ((c0 ^ (rr & 7)) << 4);
                            *reinterpret_cast<uint4*>(tile + at) = make_uint4(h2_mul(n[0], s2[c]), h2_mul(n[1], s2[c]), h2_mul(n[2], s2[c]), h2_mul(n[3], s2[c]));
                            if (in_two)
                                *reinterpret_cast<uint4*>(smem + C::OFF_K_LOWER + at) =
                                    make_uint4(h2_mul(n[0], lower[c]), h2_mul(n[1], lower[c]), h2_mul(n[2], lower[c]), h2_mul(n[3], lower[c]));
                        }
                    }
                } else {
                    const int rr = wq * 32 + lane;
                    uint8_t* src = tile + HALF_BYTES + rr * 128;
                    uint4 raw[8];
#pragma unroll
                    for (int c = 0; c < 8; ++c) raw[c] = *reinterpret_cast<const uint4*>(src + ((c ^ (rr & 7)) << 4));
#pragma unroll
                    for (int c = 0; c < 8; ++c) {                 // 16 elements: channels 16 c .. 16 c + 15
                        const uint32_t w[4] = {raw[c].x, raw[c].y, raw[c].z, raw[c].w};
                        uint32_t f[8];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            f[2 * q] = e4m3x2_to_f16x2(w[q]);
                            f[2 * q + 1] = e4m3x2_to_f16x2(w[q] >> 16);
                        }
                        uint8_t* dst = tile + (c >> 2) * HALF_BYTES + rr * 128;
                        const int c0 = (c & 3) * 2;
                        *reinterpret_cast<uint4*>(dst + (((c0) ^ (rr & 7)) << 4)) = make_uint4(f[0], f[1], f[2], f[3]);
                        *reinterpret_cast<uint4*>(dst + (((c0 + 1) ^ (rr & 7)) << 4)) = make_uint4(f[4], f[5], f[6], f[7]);
                    }
                }
                fence_proxy_async_smem();                          // generic writes -> tensor core reads
                __syncwarp();
            };
            uint32_t it = 0, n_seg = 0;
            bool ok = true;
            for (int si = seg_lo; si < seg_hi && ok; ++si) {
                const int n_tiles = (p.segments[si].k_end - p.segments[si].k_begin + BN - 1) / BN;
                if (n_tiles <= 0) continue;
                const int k_begin = p.segments[si].k_begin;
                const int seen = first_seen(p.segments[si].n_full, p.window);
                // Q: bf16 -> fp16 in place (element by element, so the swizzle does not matter)
                if (!(ok = warp_wait(q_full, n_seg & 1u, ab, kWaitRingFull))) break;
                ++n_seg;
#pragma unroll 1
                for (int off = (wq * 32 + lane) * 16; off < 2 * C::TILE_BYTES; off += 128 * 16) {
                    uint4 v = *reinterpret_cast<const uint4*>(smem + C::OFF_Q + off);
                    v.x = bf16x2_to_f16x2(v.x); v.y = bf16x2_to_f16x2(v.y);
                    v.z = bf16x2_to_f16x2(v.z); v.w = bf16x2_to_f16x2(v.w);
                    *reinterpret_cast<uint4*>(smem + C::OFF_Q + off) = v;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_ready);
                for (int t = 0; t < n_tiles && ok; ++t, ++it) {
                    const uint32_t kb = it % KS, vb = it % VS;
                    if (!(ok = warp_wait(&k_full[kb], (it / KS) & 1u, ab, kWaitRingFull))) break;
                    if (KIND == kPaged4 && !(ok = warp_wait(&low_empty[wq >> 1], (it & 1u) ^ 1u, ab, kWaitRingEmpty))) break;
                    widen_tile(smem + C::OFF_K + kb * C::TILE_BYTES, true, false);
                    if (lane == 0) mbar_arrive(&k_ready[KIND == kPaged4 ? kb * 2 + (wq >> 1) : kb]);
                    if (!(ok = warp_wait(&v_full[vb], (it / VS) & 1u, ab, kWaitRingFull))) break;
                    const int key = k_begin + t * BN + wq * 32 + lane;
                    widen_tile(smem + C::OFF_V + vb * C::TILE_BYTES, false, KIND == kPaged4 && key < seen);
                    if (lane == 0) mbar_arrive(&v_ready[vb]);
                }
            }
        }
    } else {
        // ======================================= softmax warpgroups ==========================
        setmaxnreg_inc<Regs<FP8>::kSoftmax>();
        const int r = (warp >> 2) - 1;                 // row tile of this warpgroup
        const int quad = warp & 3;                     // TMEM lane quadrant this warp may access
        const int row = quad * 32 + lane;              // row inside the 128-row tile
        const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
        const uint32_t tmem_s = tmem_base + r * BN + lane_addr;
        const uint32_t tmem_o = tmem_base + 2 * BN + r * BN + lane_addr;
        const int r_local = (m_tile * 2 + r) * BM + row;   // row inside the stream's G*T rows
        const bool row_valid = r_local < p.rows_per_stream;
        uint32_t it = 0;
        bool ok = aligned_ok;

        // The exponentials of the two row tiles take turns.  The two softmax warps that share a
        // scheduler (same quadrant, row tiles 0 and 1) would otherwise run their exponentials at the
        // same time -- both are released by score products that complete back to back -- and then
        // share the special-function unit (4 results per clock and scheduler) while the rest of their
        // half step (fetch, row max, hand-overs) leaves it idle: measured, a 32-key group costs ~230
        // cycles alone and 430-500 next to its neighbour.  With turns (row tile 0, row tile 1, row tile 0,
        // ...) one warp's exponentials overlap the other's remaining work.  A turn is passed with a
        // named barrier of the two warps: the passer arrives without waiting, the taker waits.  Both
        // warps walk the same half steps, and a warp that has given up still takes and passes its
        // turns, so neither can be left waiting.
        const int bar_to_1 = 1 + quad, bar_to_0 = 5 + quad;     // barrier ids 1..8
        auto take_turn = [&](uint32_t u) {
            if (r == 1) named_barrier_sync(bar_to_1, 64);
            else if (u > 0) named_barrier_sync(bar_to_0, 64);
        };
        uint32_t turns = 0;
        auto pass_turn = [&]() {
            named_barrier_arrive(r == 0 ? bar_to_1 : bar_to_0, 64);
            ++turns;
        };
        auto skip_turn = [&](uint32_t u) {
            take_turn(u);
            pass_turn();
        };

        for (int si = seg_lo; si < seg_hi; ++si) {
            const DevSegment seg = p.segments[si];
            const int n_full = seg.n_full;     // keys visible to row 0 (row t sees n_full + t), see DevSegment
            const int n_edge = min(n_full, seg.n_kv);      // tiles that end at or below it need no mask
            const int vis = min(seg.n_kv, max(0, n_full + (r_local % p.T)));
            // sliding window: the row at position i keeps i - C < j; lo_max is the highest such bound
            const int lo = p.window > 0 ? max(0, n_full + (r_local % p.T) - p.window) : 0;
            const int lo_max = p.window > 0 ? n_full + p.T - 1 - p.window : 0;
            const int seen = first_seen(n_full, p.window);     // V rows below it may hold anything
            float m_ref = -INFINITY, l = 0.f;
            const uint32_t seg_first_it = it, seg_first_u = 2 * it;
            // 8-bit cache: the key scale of this KV head folds into the softmax scale, the value scale
            // multiplies the normalised output
            const int head = KIND == kPacked8 ? seg.stream % sc.Hkv : 0;
            const float scale_log2 = KIND == kPacked8 ? sc.score_scale_log2[head] : p.scale_log2;
            const float out_scale = KIND == kPacked8 ? sc.v_scale[head] : 1.f;
            for (int k0 = seg.k_begin; k0 < seg.k_end; k0 += BN, ++it) {
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    const uint32_t u = 2 * it + h;             // half step number
                    if (!ok) {
                        skip_turn(u);
                        continue;
                    }
                    const int kh = k0 + h * BH;                // first key of the half step
                    if (!(ok = warp_wait(&s_full[r * 2 + h], it & 1u, ab, kWaitTensor))) {
                        skip_turn(u);
                        continue;
                    }
                    tc_fence_after();
                    float s[BH];
#pragma unroll
                    for (int c = 0; c < BH / 32; ++c)
                        tmem_ld32(tmem_s + h * BH + c * 32, *reinterpret_cast<float(*)[32]>(&s[c * 32]));
                    tmem_wait_ld();

                    const bool masked = !(kh + BH <= n_edge && kh >= lo_max);   // causal edge, sequence end or window start
                    if (masked) {
#pragma unroll
                        for (int j = 0; j < BH; ++j) s[j] = (kh + j < vis && kh + j >= lo) ? s[j] : -INFINITY;
                    }
                    // row max of the raw scores (scale > 0, so it commutes with max)
                    float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int j = 0; j < BH; j += 2) mx4[(j >> 1) & 3] = fmax3(mx4[(j >> 1) & 3], s[j], s[j + 1]);
                    const float mx = fmax3(fmaxf(mx4[0], mx4[1]), mx4[2], mx4[3]) * scale_log2;
                    // lazy rescale: the reference max moves only when the row max outgrew it by 2^8
                    const bool grow = mx > m_ref + kRescaleThreshold || (m_ref == -INFINITY && mx > -INFINITY);
                    if (__any_sync(0xffffffffu, grow)) {
                        float alpha = 1.f;
                        if (grow) {
                            alpha = ex2_approx(m_ref - mx);               // 0 when m_ref = -inf
                            m_ref = mx;
                            l *= alpha;
                        }
                        if (u > seg_first_u) {
                            // O_r holds the sums of the earlier half steps of this segment: wait for
                            // the product of the previous one (the other buffer; it belongs to this key
                            // tile when h = 1, to the previous one when h = 0)
                            if (!(ok = warp_wait(&pv_done[r * 2 + (h ^ 1)], (it ^ (h ^ 1)) & 1u, ab, kWaitTensor))) {
                                skip_turn(u);
                                continue;
                            }
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D / 32; ++c) {
                                float o[32];
                                tmem_ld32(tmem_o + c * 32, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int j = 0; j < 32; ++j) o[j] *= alpha;
                                tmem_st32(tmem_o + c * 32, o);
                            }
                        }
                    }
                    const float neg_m = m_ref == -INFINITY ? 0.f : p_shift(KIND) - m_ref;

                    // keys past the end of the sequence (or before all windows): their V rows may hold anything; zero them so
                    // that 0 * garbage cannot make NaN.  Both warpgroups write the same zeros in
                    // the first half step, each before it releases its own first product on this tile.
                    if (h == 0 && (k0 + BN > seg.n_kv || (KIND == kPaged16 && k0 < seen))) {
                        const uint32_t vb = it % VS, vn = it / VS;
                        if (!(ok = warp_wait(&v_use[vb], vn & 1u, ab, kWaitRingFull))) {
                            skip_turn(u);
                            continue;
                        }
                        if (k0 + row >= seg.n_kv || (KIND == kPaged16 && k0 + row < seen)) {
                            uint8_t* vrow = smem + C::OFF_V + vb * C::TILE_BYTES + row * 128;
#pragma unroll 1
                            for (int q = 0; q < 8 * HALVES; ++q)
                                *reinterpret_cast<uint4*>(vrow + (q >> 3) * HALF_BYTES + (q & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        fence_proxy_async_smem();                   // generic writes -> tensor core reads
                    }

                    // P = 2^(s * scale - m_ref + p_shift), two elements per instruction where the hardware
                    // allows; a masked score (-inf) comes out as exactly 0.
                    const uint64_t scale2 = f2_pack(scale_log2, scale_log2), negm2 = f2_pack(neg_m, neg_m);
                    uint64_t ls2[4] = {0ull, 0ull, 0ull, 0ull};            // packed partial row sums
                    take_turn(u);
#pragma unroll
                    for (int c = 0; c < BH / 32; ++c) {                // 32 keys -> 16 packed columns
                        uint32_t pk[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint64_t x2 = f2_fma(f2_pack(s[c * 32 + 2 * j], s[c * 32 + 2 * j + 1]), scale2, negm2);
                            uint64_t e2;
                            if (poly_pair(j)) {
                                e2 = f2_exp2_poly<KIND == kPaged4>(x2);
                            } else {
                                float x0, x1;
                                f2_unpack(x2, x0, x1);
                                e2 = f2_pack(ex2_approx(x0), ex2_approx(x1));
                            }
                            ls2[j & 3] = f2_add(ls2[j & 3], e2);
                            float e0, e1;
                            f2_unpack(e2, e0, e1);
                            pk[j] = FP8 ? pack_f16x2(e0, e1) : pack_bf16x2(e0, e1);
                        }
                        tmem_st16(tmem_s + h * BH + c * 16, pk);
                    }
                    pass_turn();
                    // announce P (announcing it only after the next half step's scores had been fetched,
                    // to keep the wait for the stores out of line, was measured slower: the product
                    // that frees this buffer for the scores after next then starts later)
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[r * 2 + h]);
                    {
                        float a0, a1, b0, b1;
                        f2_unpack(f2_add(ls2[0], ls2[1]), a0, a1);
                        f2_unpack(f2_add(ls2[2], ls2[3]), b0, b1);
                        l += (a0 + a1) + (b0 + b1);
                    }
                }
            }
            // ---- end of segment: O_r is complete once the last PV has finished ----
            // (the products of one row tile complete in order, so the last one covers all)
            if (ok && it > seg_first_it) ok = warp_wait(&pv_done[r * 2 + 1], (it - 1) & 1u, ab, kWaitTensor);
            if (ok) {
                tc_fence_after();
                const bool has = l > 0.f;
                const float inv = has ? out_scale / l : 0.f;
                const float lse = has ? (m_ref - p_shift(KIND) + log2f(l)) * 0.6931471805599453f : -INFINITY;
                const bool final_out = seg.stream_nseg == 1 && !p.force_partial;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    float o[32];
                    tmem_ld32(tmem_o + c * 32, o);
                    tmem_wait_ld();
                    if (row_valid) {
                        if (final_out) {
                            __nv_bfloat16* dst = p.O + ((int64_t)seg.q_row0 + r_local) * D + c * 32;
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                uint4 pk;
                                pk.x = pack_bf16x2(has ? o[q * 8 + 0] * inv : 0.f, has ? o[q * 8 + 1] * inv : 0.f);
                                pk.y = pack_bf16x2(has ? o[q * 8 + 2] * inv : 0.f, has ? o[q * 8 + 3] * inv : 0.f);
                                pk.z = pack_bf16x2(has ? o[q * 8 + 4] * inv : 0.f, has ? o[q * 8 + 5] * inv : 0.f);
                                pk.w = pack_bf16x2(has ? o[q * 8 + 6] * inv : 0.f, has ? o[q * 8 + 7] * inv : 0.f);
                                *reinterpret_cast<uint4*>(dst + q * 8) = pk;
                            }
                        } else {
                            float* dst = p.part_o + ((int64_t)seg.slot * p.rows_per_stream + r_local) * D + c * 32;
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                *reinterpret_cast<float4*>(dst + q * 4) =
                                    make_float4(has ? o[q * 4 + 0] * inv : 0.f, has ? o[q * 4 + 1] * inv : 0.f,
                                                has ? o[q * 4 + 2] * inv : 0.f, has ? o[q * 4 + 3] * inv : 0.f);
                        }
                    }
                }
                if (row_valid) {
                    if (final_out) {
                        if (p.lse) p.lse[seg.q_row0 + r_local] = lse;
                    } else {
                        p.part_lse[(int64_t)seg.slot * p.rows_per_stream + r_local] = lse;
                    }
                }
                tc_fence_before();
            }
        }
        // the last turn row tile 1 passed has no taker: take it, so that no barrier is left half complete
        if (r == 0 && turns > 0) named_barrier_sync(bar_to_0, 64);

    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

template <int D, CacheKind KIND>
cudaError_t launch_one(const ChunkParams& p, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmKs,
                       const CUtensorMap& tmV, const CUtensorMap& tmVs, int num_groups, cudaStream_t stream,
                       const ChunkFp8Scales& sc) {
    chunk_pair_kernel<D, KIND><<<num_groups * p.m_tiles, kThreadsOf<widened(KIND)>, PCfg<D>::SMEM_BYTES, stream>>>(
        tmQ, tmK, tmKs, tmV, tmVs, p, sc);
    return cudaGetLastError();
}

template <int D, CacheKind KIND>
cudaError_t setup_one() {
    cudaError_t e = cudaFuncSetAttribute(chunk_pair_kernel<D, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         PCfg<D>::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    // the register split inside the kernel assumes the launch allocation it was written for
    cudaFuncAttributes attr;
    if ((e = cudaFuncGetAttributes(&attr, chunk_pair_kernel<D, KIND>)) != cudaSuccess) return e;
    return attr.numRegs >= Regs<widened(KIND)>::kLaunch ? cudaSuccess : cudaErrorLaunchOutOfResources;
}

}  // namespace

cudaError_t chunk_pair_kernel_setup() {
    cudaError_t e = setup_one<128, kPacked16>();
    if (e != cudaSuccess) return e;
    if ((e = setup_one<64, kPacked16>()) != cudaSuccess) return e;
    if ((e = setup_one<128, kPacked8>()) != cudaSuccess) return e;
    if ((e = setup_one<128, kPaged16>()) != cudaSuccess) return e;
    if ((e = setup_one<64, kPaged16>()) != cudaSuccess) return e;
    return setup_one<128, kPaged4>();
}

cudaError_t launch_chunk_pair(const ChunkParams& p, const CUtensorMap& tmQ, const CUtensorMap& tmK,
                              const CUtensorMap& tmV, int num_groups, cudaStream_t stream,
                              const ChunkFp8Scales* fp8_scales, bool paged) {
    if (num_groups <= 0) return cudaSuccess;
    if (fp8_scales) {
        if (p.d != 128) return cudaErrorInvalidValue;
        return launch_one<128, kPacked8>(p, tmQ, tmK, tmK, tmV, tmV, num_groups, stream, *fp8_scales);
    }
    const ChunkFp8Scales none{};
    if (paged)
        return p.d == 128 ? launch_one<128, kPaged16>(p, tmQ, tmK, tmK, tmV, tmV, num_groups, stream, none)
                          : launch_one<64, kPaged16>(p, tmQ, tmK, tmK, tmV, tmV, num_groups, stream, none);
    return p.d == 128 ? launch_one<128, kPacked16>(p, tmQ, tmK, tmK, tmV, tmV, num_groups, stream, none)
                      : launch_one<64, kPacked16>(p, tmQ, tmK, tmK, tmV, tmV, num_groups, stream, none);
}

cudaError_t launch_chunk_pair_q4(const ChunkParams& p, const CUtensorMap& tmQ, const PagedQ4Maps& m, int num_groups,
                                 cudaStream_t stream) {
    if (num_groups <= 0) return cudaSuccess;
    if (p.d != 128) return cudaErrorInvalidValue;
    const ChunkFp8Scales none{};
    return launch_one<128, kPaged4>(p, tmQ, m.k, m.k_scale, m.v, m.v_scale, num_groups, stream, none);
}

}  // namespace yoco
