// Split-KV decode over a paged 4-bit cache: 64 bytes of codes and four fp16 scales a row (32 channels share a
// scale, value = (code - 8) * scale), head dimension 128.  Work items, ring protocol, masks and the merge are those
// of the 8-bit kernel; a 64-key tile is 4 KB of codes and 512 bytes of scales per tensor, 9 KB in all, so at the same
// HBM bandwidth a key has to be worked off in a little over half of the 8-bit kernel's time.  What this kernel does about
// that is to spend few instructions per key:
//
//   codes    No conversion instruction.  A code n sits in the low bits of an fp16 word after one AND, where it is
//            the subnormal n 2^-24 (or 16 n 2^-24 for the nibble next to it): an exact multiple, and tensor-core
//            operands keep subnormals.  The factor 16 goes into Q (exact), 2^24 into the softmax scale.
//   K        S = sum over groups j of  s_j(key) * 2^24 * (sum_c q_c n_c 2^-24  -  8 * 2^-24 * sum_c q_c).
//            The inner sums are the two products of a group; their accumulator starts at the (per row and
//            group) constant instead of zero, so the offset 8 is free; the scales are applied to the fp32
//            result, four multiply-adds per group and 16 keys.
//   V        sum over keys of P n s_j: here the group's scale is inside the sum.  It goes into P: P^T s_j in
//            fp16, one packed product per 16 keys and group.  Subtracting the offset afterwards would cancel (the
//            sum of P n is far larger than the result when many keys share the weight), so V codes are made
//            signed first: 1024 + n by AND and OR, minus 1032 (exact).
//   order    Q is loaded in the channel order in which ldmatrix hands over the nibbles; the four channels of a
//            16-bit unit of V come out in four different products, which is one float4 per lane at the end.
//
// P is kept in [0, 2^7] (the exponential of s - max + 7) so that P times a small scale keeps its bits in fp16; a V scale
// stays below 448, and 2^7 * 448 is below the largest fp16 value.
#include "decode_f16.cuh"
#include "kernels.h"
#include "page_map.cuh"
#include "ptx.cuh"
#include "q4.cuh"

namespace yoco {

namespace {

constexpr int kConsumerWarps = 4;
constexpr int kThreads = (kConsumerWarps + 1) * 32;
constexpr int TILE_N = kDecodeTileN;          // 64 keys
constexpr int D = 128;                        // head dimension
constexpr int GROUPS = D / kQ4Group;          // scale groups of a row
constexpr int CODE_BYTES = TILE_N * D / 2;    // 4 KB: 64 rows x 64 B, 64-byte swizzle
constexpr int SCALE_BYTES = TILE_N * GROUPS * 2;
constexpr int OFF_V = CODE_BYTES, OFF_KS = 2 * CODE_BYTES, OFF_VS = OFF_KS + SCALE_BYTES;
constexpr int STAGE_BYTES = 2 * (CODE_BYTES + SCALE_BYTES);
constexpr int ROW_BYTES = STAGE_BYTES / TILE_N;
constexpr float kPShift = 7.f;                // P = 2^(s - max + kPShift)

template <int ROWS>
struct CfgQ4 {
    static constexpr int MERGE_O_BYTES = kConsumerWarps * ROWS * D * 4;
    static constexpr int MERGE_ML_BYTES = kConsumerWarps * ROWS * 2 * 4;
    static constexpr int BUDGET = 113 * 1024;     // two CTAs per SM
    static constexpr int STAGES_FIT = (BUDGET - MERGE_O_BYTES - MERGE_ML_BYTES - 256) / STAGE_BYTES;
    static constexpr int STAGES = STAGES_FIT > 10 ? 10 : STAGES_FIT;
    static_assert(STAGES >= kConsumerWarps, "every consumer warp needs a tile in flight");
    static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + MERGE_O_BYTES + MERGE_ML_BYTES + 256;
    static_assert(STAGE_BYTES % 512 == 0, "the swizzle pattern repeats every 512 bytes");
};

// D = A B + C with C kept
__device__ __forceinline__ void mma_f16_from(float (&d)[4], const float (&c)[2], uint32_t a0, uint32_t a1, uint32_t a2,
                                             uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%11,%10,%11};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]));
}
template <int ROWS>
__device__ __forceinline__ void decode_q4_body(const CUtensorMap& tmK, const CUtensorMap& tmKs, const CUtensorMap& tmV,
                                               const CUtensorMap& tmVs, const DecodeParams& p,
                                               const DevSegment* segments, const int32_t* group_begin) {
    using C = CfgQ4<ROWS>;
    constexpr int STAGES = C::STAGES;

    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* stage_mem = smem;
    float* merge_o = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES);
    float* merge_ml = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES + C::MERGE_O_BYTES);
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES + C::MERGE_O_BYTES + C::MERGE_ML_BYTES);
    uint64_t* empty_bar = full_bar + STAGES;
    volatile int* give_up = reinterpret_cast<volatile int*>(empty_bar + STAGES);   // some thread ran out of patience
    uint32_t* armed = reinterpret_cast<uint32_t*>(empty_bar + STAGES) + 1;         // tiles the producer has armed so far
    uint64_t* item_full = empty_bar + STAGES + 1;  // [2] producer -> consumers: queue entry written
    uint64_t* item_empty = item_full + 2;          // [2] consumers -> producer: entry read
    volatile int32_t* item_q = reinterpret_cast<volatile int32_t*>(item_empty + 2);   // [2] item ids
    static_assert(2 * STAGES * 8 + 8 + 32 + 8 <= 256, "barrier block");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // Work items as in the bf16 kernel: with R = p.sub_items > 1 every group's range is cut into R
    // pieces; CTA g starts with piece 0 of group g and its producer, once the last copy of an item
    // is on its way, claims the next unclaimed piece from a global counter and tells the consumers
    // through a two-entry queue, so that the ring never drains between items and a fast SM takes
    // more pieces than a slow one.  What a piece computes and where its partial result goes is
    // fixed by the plan.
    const int R = p.sub_items > 1 ? p.sub_items : 1;
    const int n_groups = gridDim.x;
    const int n_items = n_groups * R;
    asm volatile("griddepcontrol.launch_dependents;");

    if ((smem_u32(smem) & 1023u) != 0) {   // the swizzle arithmetic below needs 1 KB alignment
        if (threadIdx.x == 0) atomicCAS(p.status, 0, status_word(kWaitMisaligned, linear_cta()));
        return;
    }
    const Abort ab{give_up, p.status, p.wait_limit_ns > 0 ? p.wait_limit_ns : kWaitLimitNs};
    if (threadIdx.x == 0) {
        *give_up = 0;
        *armed = 0u;
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], 1);                 // released by the one warp that read the tile
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&item_full[s], 1);
            mbar_init(&item_empty[s], kConsumerWarps);
        }
        mbar_fence_init();
    }
    __syncthreads();

    if (warp == kConsumerWarps) {
        // ------------------------------- producer ---------------------------------------
        if (lane == 0) {
            tma_prefetch_desc(&tmK);
            tma_prefetch_desc(&tmKs);
            tma_prefetch_desc(&tmV);
            tma_prefetch_desc(&tmVs);
            uint32_t it = 0;
            bool ok = true;
            int item = blockIdx.x;
            for (uint32_t n = 0; ok; ++n) {
                // hand the item (or the end mark) to the consumers
                if (!wait_or_abort(&item_empty[n & 1u], ((n >> 1) & 1u) ^ 1u, ab, kWaitItemQueue)) break;
                item_q[n & 1u] = item;
                mbar_arrive(&item_full[n & 1u]);
                if (item >= n_items) break;
                const int grp = item % n_groups, piece = item / n_groups;
                const int seg_lo = group_begin[grp], seg_hi = group_begin[grp + 1];
                int t_lo = 0, t_hi = 0x7fffffff, t_acc = 0;     // the piece's tiles inside the group
                if (R > 1) {
                    int n_g = 0;
                    for (int si = seg_lo; si < seg_hi; ++si)
                        n_g += (segments[si].k_end - segments[si].k_begin + TILE_N - 1) / TILE_N;
                    t_lo = (int)sub_bound(n_g, R, piece);
                    t_hi = (int)sub_bound(n_g, R, piece + 1);
                }
                for (int si = seg_lo; si < seg_hi && ok; ++si) {
                    const DevSegment seg = segments[si];
                    const int seg_tiles = (seg.k_end - seg.k_begin + TILE_N - 1) / TILE_N;
                    const int s_lo = max(t_lo - t_acc, 0), s_hi = min(t_hi - t_acc, seg_tiles);
                    t_acc += seg_tiles;
                    if (s_lo >= s_hi) continue;
                    const int k_lo = seg.k_begin + s_lo * TILE_N;
                    const int k_hi = min(seg.k_begin + s_hi * TILE_N, seg.k_end);
                    PageCursor<TILE_N> pc;
                    pc.start(p.pages, seg.stream, k_lo, k_hi);
                    for (int k0 = k_lo; k0 < k_hi; k0 += TILE_N, ++it) {
                        const uint32_t stage = it % STAGES, round = it / STAGES;
                        if (!wait_or_abort(&empty_bar[stage], (round & 1u) ^ 1u, ab, kWaitRingEmpty)) {
                            ok = false;
                            break;
                        }
                        uint8_t* dst = stage_mem + stage * STAGE_BYTES;
                        mbar_expect_tx(&full_bar[stage], pc.rows() * ROW_BYTES);
                        pc.for_each_box(ab.status, [&](int dst_row, int row) {
                            tma_load_2d(dst + dst_row * (D / 2), &tmK, 0, row, &full_bar[stage]);
                            tma_load_2d(dst + OFF_KS + dst_row * (2 * GROUPS), &tmKs, 0, row >> 4, &full_bar[stage]);
                            tma_load_2d(dst + OFF_V + dst_row * (D / 2), &tmV, 0, row, &full_bar[stage]);
                            tma_load_2d(dst + OFF_VS + dst_row * (2 * GROUPS), &tmVs, 0, row >> 4, &full_bar[stage]);
                        });
                        pc.next();
                        st_release_shared(armed, it + 1);        // tiles 0 .. it have their barriers armed
                    }
                }
                // all loads of this item are on their way: claim the next one
                item = R > 1 ? n_groups + atomicAdd(p.work_counter, 1) : n_items;
            }
            // every copy this thread armed must have landed before it leaves (the CTA ends with its last
            // thread, and its shared memory then belongs to another CTA); at once when all went well
            const uint32_t in_flight = it < (uint32_t)STAGES ? it : (uint32_t)STAGES;
            for (uint32_t k = it - in_flight; k < it; ++k)
                if (!drain_wait(&full_bar[k % STAGES], (k / STAGES) & 1u, ab)) break;
        }
        return;
    }

    // ----------------------------------- consumers ---------------------------------------
    // Each consumer warp takes whole tiles, round robin; a tile is released by the one warp that read it.
    constexpr int NT = ROWS / 8;                       // 8-row groups on the narrow side of the products
    const int g = lane >> 2, tq = lane & 3;
    const int n_rows = p.rows_per_stream;
    // row address this lane supplies to ldmatrix.x4 for K: matrix (lane >> 3) = (16-byte chunk of the pair, key half)
    const int ld_key16 = ((lane >> 3) & 1) * 8 + (lane & 7);            // key row inside a 16-key group
    const int ld_chunk = lane >> 4;                                      // 0: first chunk of the pair, 1: second
    uint32_t it = 0;
    bool ok = true;

    for (uint32_t n_item = 0;; ++n_item) {
    // the next item from the producer; the four warps must take the same decision, so a warp
    // that gives up waiting says so before the barrier and all of them leave together
    const bool got_item = wait_or_abort(&item_full[n_item & 1u], (n_item >> 1) & 1u, ab, kWaitItemQueue);
    const int item = item_q[n_item & 1u];
    if (named_barrier_or(1, kConsumerWarps * 32, !got_item || !ok)) break;
    if (lane == 0) mbar_arrive(&item_empty[n_item & 1u]);
    if (item >= n_items) break;
    const int grp = item % n_groups, piece = item / n_groups;
    const int seg_lo = group_begin[grp], seg_hi = group_begin[grp + 1];
    int t_lo = 0, t_hi = 0x7fffffff, t_acc = 0;       // the piece's tiles inside the group
    if (R > 1) {
        int n_g = 0;
        for (int si = seg_lo; si < seg_hi; ++si)
            n_g += (segments[si].k_end - segments[si].k_begin + TILE_N - 1) / TILE_N;
        t_lo = (int)sub_bound(n_g, R, piece);
        t_hi = (int)sub_bound(n_g, R, piece + 1);
    }

    for (int si = seg_lo; si < seg_hi; ++si) {
        const DevSegment seg = segments[si];
        const int seg_tiles = (seg.k_end - seg.k_begin + TILE_N - 1) / TILE_N;
        const int s_lo = max(t_lo - t_acc, 0), s_hi = min(t_hi - t_acc, seg_tiles);
        t_acc += seg_tiles;
        const int slot = seg.slot * R + piece;
        if (s_lo >= s_hi) {
            // this piece holds nothing of the segment: its slot must say so to the merge
            if (R > 1 && threadIdx.x < p.rows_per_stream) p.part_lse[(int64_t)slot * p.rows_per_stream + threadIdx.x] = -INFINITY;
            continue;
        }
        const int k_lo = seg.k_begin + s_lo * TILE_N;
        const int k_hi = min(seg.k_begin + s_hi * TILE_N, seg.k_end);
        const float sscale = p.scale_log2 * 16777216.f;      // the codes of K count as n 2^-24

        // Q^T as the second operand of the score products (fp16).  The two products of group j cover its 32 channels;
        // this lane's slots (k = 2 tq, 2 tq + 1, 2 tq + 8, 2 tq + 9) of product u stand for channels
        // 32 j + 8 tq + {2 u, 2 u + 4, 2 u + 1, 2 u + 5} of query row 8 nt + g, the last two divided by 16:
        // the nibbles that one AND brings into place, and those that come out 16 times too large.
        uint32_t qb[NT][GROUPS][2][2];
        float qoff[NT][GROUPS][2];        // -8 * 2^-24 * (sum of the group's q) of rows 8 nt + 2 tq + {0, 1}
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = 8 * nt + g;
            const __nv_bfloat16* q = p.Q + ((int64_t)seg.q_row0 + row) * D + tq * 8;
#pragma unroll
            for (int j = 0; j < GROUPS; ++j) {
                const uint4 w = row < n_rows ? *reinterpret_cast<const uint4*>(q + j * 32) : make_uint4(0u, 0u, 0u, 0u);
                const float x[8] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u),
                                    __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u),
                                    __uint_as_float(w.z << 16), __uint_as_float(w.z & 0xFFFF0000u),
                                    __uint_as_float(w.w << 16), __uint_as_float(w.w & 0xFFFF0000u)};
                float sum = 0.f;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    qb[nt][j][u][0] = pack_f16x2(x[2 * u], x[2 * u + 4]);
                    qb[nt][j][u][1] = pack_f16x2(x[2 * u + 1] * 0.0625f, x[2 * u + 5] * 0.0625f);
                    const float2 a = h2_to_f2(qb[nt][j][u][0]), b = h2_to_f2(qb[nt][j][u][1]);
                    sum += (a.x + a.y) + 16.f * (b.x + b.y);
                }
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                sum *= -8.f / 16777216.f;
                qoff[nt][j][0] = __shfl_sync(0xffffffffu, sum, 8 * tq);
                qoff[nt][j][1] = __shfl_sync(0xffffffffu, sum, 8 * tq + 4);
            }
        }
        const int n_full = seg.n_full;
        const int n_edge = min(n_full, seg.n_kv);      // tiles that end at or below it need no mask
        int vis[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) vis[nt][e] = min(seg.n_kv, max(0, n_full + ((8 * nt + 2 * tq + e) % p.T)));

        // running max and (this lane's part of the) sum of rows 8 nt + 2 tq + {0, 1}
        float m[NT][2], l[NT][2];
        // O^T: acc[nt][j][u] is the product tile whose channel slots i and i + 8 (i < 8) stand for channels
        // 32 j + 4 i + 2 u and 32 j + 4 i + 2 u + 1: elements 0, 1 = (slot g, rows 2 tq, 2 tq + 1), elements 2, 3 =
        // (slot g + 8, same rows)
        float acc[NT][4][2][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) acc[nt][j][e][0] = acc[nt][j][e][1] = acc[nt][j][e][2] = acc[nt][j][e][3] = 0.f;
        }

        for (int k0 = k_lo; k0 < k_hi; k0 += TILE_N, ++it) {
            if (!ok || (int)(it % kConsumerWarps) != warp) continue;       // not this warp's tile
            // A parity wait only tells the phase of a barrier apart from the one before it.  A warp
            // that takes every fourth tile could ask for round r of a stage whose round r - 1 has not
            // landed yet (copies complete in any order, and when a kernel starts all of them queue at
            // once): it would be let through at once, read a tile that is still being written and
            // release the stage a second time.  So it first waits until the producer has armed
            // THIS tile: the producer can only have done so after the previous tile of the stage was
            // released, i.e. after its round completed, and the barrier is then in the round asked for.
            const uint32_t stage = it % STAGES, round = it / STAGES;
            if (!wait_armed(armed, it + 1, ab) || !wait_or_abort(&full_bar[stage], round & 1u, ab, kWaitRingFull)) {
                ok = false;         // this warp touches no tile any more; it still walks to the barriers below
                continue;
            }
            uint8_t* tile = stage_mem + stage * STAGE_BYTES;
            const uint32_t kbase = smem_u32(tile), vbase = kbase + OFF_V;
            // ---- S^T = K Q^T for 64 keys: four 16-key groups, four scale groups of two products each ----
            float s[NT][4][4];     // [row group][16-key group]: (key g, rows 2 tq, 2 tq + 1), (key g + 8, same rows)
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                const int key = mt * 16 + ld_key16;
                const uint2 sa = *reinterpret_cast<const uint2*>(tile + OFF_KS + (mt * 16 + g) * 8);       // scales of key g
                const uint2 sb = *reinterpret_cast<const uint2*>(tile + OFF_KS + (mt * 16 + g + 8) * 8);   // of key g + 8
                const float2 sa01 = h2_to_f2(sa.x), sa23 = h2_to_f2(sa.y), sb01 = h2_to_f2(sb.x), sb23 = h2_to_f2(sb.y);
                const float ka[4] = {sa01.x, sa01.y, sa23.x, sa23.y}, kb[4] = {sb01.x, sb01.y, sb23.x, sb23.y};
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                    const int chunk = 2 * jj + ld_chunk;
                    uint32_t r[4];   // (keys 0-7, group 2 jj) (keys 8-15, 2 jj) (keys 0-7, 2 jj + 1) (keys 8-15, 2 jj + 1)
                    ldmatrix_x4(kbase + key * 64 + (((chunk ^ (key >> 1)) & 3) << 4), r[0], r[1], r[2], r[3]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int j = 2 * jj + h;
                        const uint32_t a = r[2 * h], b = r[2 * h + 1], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float t[4];
                            mma_f16_from(t, qoff[nt][j], a & 0x000F000Fu, b & 0x000F000Fu, a & 0x00F000F0u, b & 0x00F000F0u,
                                         qb[nt][j][0][0], qb[nt][j][0][1]);
                            mma_f16_16816(t, a8 & 0x000F000Fu, b8 & 0x000F000Fu, a8 & 0x00F000F0u, b8 & 0x00F000F0u,
                                          qb[nt][j][1][0], qb[nt][j][1][1]);
                            s[nt][mt][0] = j == 0 ? t[0] * ka[j] : fmaf(t[0], ka[j], s[nt][mt][0]);
                            s[nt][mt][1] = j == 0 ? t[1] * ka[j] : fmaf(t[1], ka[j], s[nt][mt][1]);
                            s[nt][mt][2] = j == 0 ? t[2] * kb[j] : fmaf(t[2], kb[j], s[nt][mt][2]);
                            s[nt][mt][3] = j == 0 ? t[3] * kb[j] : fmaf(t[3], kb[j], s[nt][mt][3]);
                        }
                    }
                }
            }
            // ---- scale, mask (causal edge, sequence end, window start), online softmax ----
            const bool need_mask = k0 + TILE_N > n_edge || (p.window > 0 && k0 < n_full + p.T - 1 - p.window);
            float alpha[NT][2];
            bool any_alpha = false;
            uint32_t pb[NT][4][2];     // P^T (fp16) as the second operand of O^T += V^T P^T: [16-key group][keys 0-7 / 8-15]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int lo = (need_mask && p.window > 0) ? n_full + ((8 * nt + 2 * tq + e) % p.T) - p.window : -1;
                    float mx = -INFINITY;
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            float v = s[nt][mt][2 * hh + e] * sscale;
                            if (need_mask) {
                                const int jj = k0 + mt * 16 + hh * 8 + g;
                                v = (jj < vis[nt][e] && jj >= lo) ? v : -INFINITY;
                            }
                            s[nt][mt][2 * hh + e] = v;
                            mx = fmaxf(mx, v);
                        }
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    const float mn = fmaxf(m[nt][e], mx);
                    const float ms = mn == -INFINITY ? 0.f : mn, mp = ms - kPShift;
                    alpha[nt][e] = ex2_fast(m[nt][e] - ms);
                    any_alpha |= alpha[nt][e] != 1.f;
                    m[nt][e] = mn;
                    float sum = 0.f;
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            const float pv = ex2_fast(s[nt][mt][2 * hh + e] - mp);
                            s[nt][mt][2 * hh + e] = pv;
                            sum += pv;
                        }
                    l[nt][e] = l[nt][e] * alpha[nt][e] + sum;
                }
                // (key g, rows 2 tq, 2 tq + 1) -> (row g, keys 2 tq, 2 tq + 1), for the first and the second
                // eight keys of every 16-key group
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {
                    pb[nt][mt][0] = movmatrix_trans(pack_f16x2(s[nt][mt][0], s[nt][mt][1]));
                    pb[nt][mt][1] = movmatrix_trans(pack_f16x2(s[nt][mt][2], s[nt][mt][3]));
                }
            }
            if (__any_sync(0xffffffffu, any_alpha)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            acc[nt][j][e][0] *= alpha[nt][0]; acc[nt][j][e][1] *= alpha[nt][1];
                            acc[nt][j][e][2] *= alpha[nt][0]; acc[nt][j][e][3] *= alpha[nt][1];
                        }
            }
            // ---- rows past the end of the sequence may hold anything, and their boxes may not have been loaded:
            //      any code is a finite value, but a scale could be NaN, and 0 * NaN must not reach O ----
            if (k0 + TILE_N > seg.n_kv) {
                const int first_bad = max(seg.n_kv - k0, 0);          // 0..63
                for (int r = first_bad + lane; r < TILE_N; r += 32)
                    *reinterpret_cast<uint2*>(tile + OFF_VS + r * 8) = make_uint2(0u, 0u);
                __syncwarp();
            }
            // ---- O^T += V^T (P^T s).  The transposed ldmatrix hands this lane, for keys 2 tq and 2 tq + 1 of an
            //      8-key group, the 16-bit unit g of a 16-byte chunk: four channels of a group ----
#pragma unroll
            for (int kg = 0; kg < 4; ++kg) {
                const int key = kg * 16 + ld_key16;
                // scales of keys 2 tq, 2 tq + 1 (and those + 8): (s0 s1 | s2 s3) of either, regrouped per scale group
                uint32_t sv[2][4];
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const uint4 w = *reinterpret_cast<const uint4*>(tile + OFF_VS + (kg * 16 + hh * 8 + 2 * tq) * 8);
                    sv[hh][0] = __byte_perm(w.x, w.z, 0x5410);
                    sv[hh][1] = __byte_perm(w.x, w.z, 0x7632);
                    sv[hh][2] = __byte_perm(w.y, w.w, 0x5410);
                    sv[hh][3] = __byte_perm(w.y, w.w, 0x7632);
                }
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                    const int chunk = 2 * jj + ld_chunk;
                    uint32_t r[4];   // (keys 0-7, group 2 jj) (keys 8-15, 2 jj) (keys 0-7, 2 jj + 1) (keys 8-15, 2 jj + 1)
                    ldmatrix_x4_trans(vbase + key * 64 + (((chunk ^ (key >> 1)) & 3) << 4), r[0], r[1], r[2], r[3]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int j = 2 * jj + h;
                        const uint32_t a = r[2 * h], b = r[2 * h + 1], a8 = a >> 8, b8 = b >> 8;
                        const uint32_t a0 = q4_signed_lo(a), a1 = q4_signed_hi(a), a2 = q4_signed_lo(b), a3 = q4_signed_hi(b);
                        const uint32_t c0 = q4_signed_lo(a8), c1 = q4_signed_hi(a8), c2 = q4_signed_lo(b8), c3 = q4_signed_hi(b8);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint32_t p0 = h2_mul(pb[nt][kg][0], sv[0][j]), p1 = h2_mul(pb[nt][kg][1], sv[1][j]);
                            mma_f16_16816(acc[nt][j][0], a0, a1, a2, a3, p0, p1);
                            mma_f16_16816(acc[nt][j][1], c0, c1, c2, c3, p0, p1);
                        }
                    }
                }
            }
            if (k0 + TILE_N > seg.n_kv) fence_proxy_async_smem();   // generic writes before TMA reuse
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty_bar[stage]);
        }

        // ---- merge the four warps' states, write the final rows or this segment's partial ----
        {
            float* mo = merge_o + (warp * ROWS) * D;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 4);
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 8);
                    l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 16);
                    const int row = 8 * nt + 2 * tq + e;
                    // the two tiles of a group hold the four channels 4 g .. 4 g + 3 of it
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<float4*>(mo + row * D + 32 * j + 4 * g) =
                            make_float4(acc[nt][j][0][e], acc[nt][j][0][2 + e], acc[nt][j][1][e], acc[nt][j][1][2 + e]);
                    if (g == 0) {
                        merge_ml[(warp * ROWS + row) * 2] = m[nt][e];
                        merge_ml[(warp * ROWS + row) * 2 + 1] = l[nt][e];
                    }
                }
        }
        named_barrier_sync(1, kConsumerWarps * 32);
        const bool final_out = seg.stream_nseg == 1 && !p.force_partial && R == 1;
        for (int idx = threadIdx.x; idx < n_rows * D; idx += kConsumerWarps * 32) {
            const int r = idx / D, col = idx - r * D;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kConsumerWarps; ++w) M = fmaxf(M, merge_ml[(w * ROWS + r) * 2]);
            float L = 0.f, acc = 0.f;
            if (M != -INFINITY) {
#pragma unroll
                for (int w = 0; w < kConsumerWarps; ++w) {
                    const float f = exp2f(merge_ml[(w * ROWS + r) * 2] - M);
                    L += merge_ml[(w * ROWS + r) * 2 + 1] * f;
                    acc += merge_o[(w * ROWS + r) * D + col] * f;
                }
            }
            const float outv = L > 0.f ? acc / L : 0.f;
            const float lse = L > 0.f ? (M + log2f(L) - kPShift) * 0.6931471805599453f : -INFINITY;
            if (final_out) {
                p.O[((int64_t)seg.q_row0 + r) * D + col] = __float2bfloat16(outv);
                if (p.lse && col == 0) p.lse[seg.q_row0 + r] = lse;
            } else {
                p.part_o[((int64_t)slot * n_rows + r) * D + col] = outv;
                if (col == 0) p.part_lse[(int64_t)slot * n_rows + r] = lse;
            }
        }
        named_barrier_sync(1, kConsumerWarps * 32);
    }
    }
}

template <int ROWS>
__global__ void __launch_bounds__(kThreads, 2)
decode_q4_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmKs,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmVs,
                 const __grid_constant__ DecodeParams p) {
    decode_q4_body<ROWS>(tmK, tmKs, tmV, tmVs, p, p.segments, p.group_begin);
}

// work tables as kernel parameters
template <int ROWS>
__global__ void __launch_bounds__(kThreads, 2)
decode_q4_kernel_inline(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmKs,
                        const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmVs,
                        const __grid_constant__ DecodeParams p, const __grid_constant__ DecodeInlineTables tab) {
    decode_q4_body<ROWS>(tmK, tmKs, tmV, tmVs, p, tab.seg, tab.group_begin);
}

template <int ROWS>
cudaError_t launch_one(const DecodeParams& p, const PagedQ4Maps& m, int num_groups, cudaStream_t stream,
                       const DecodeInlineTables* tab) {
    if (tab)
        decode_q4_kernel_inline<ROWS><<<num_groups, kThreads, CfgQ4<ROWS>::SMEM_BYTES, stream>>>(m.k, m.k_scale, m.v, m.v_scale, p, *tab);
    else
        decode_q4_kernel<ROWS><<<num_groups, kThreads, CfgQ4<ROWS>::SMEM_BYTES, stream>>>(m.k, m.k_scale, m.v, m.v_scale, p);
    return cudaGetLastError();
}

template <int ROWS>
cudaError_t setup_one() {
    cudaError_t e = cudaFuncSetAttribute(decode_q4_kernel<ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         CfgQ4<ROWS>::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(decode_q4_kernel_inline<ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                CfgQ4<ROWS>::SMEM_BYTES);
}

}  // namespace

cudaError_t decode_q4_kernel_setup() {
    cudaError_t e = setup_one<8>();
    return e != cudaSuccess ? e : setup_one<16>();
}

cudaError_t launch_decode_q4(const DecodeParams& p, const PagedQ4Maps& maps, int num_groups, cudaStream_t stream,
                             const DecodeInlineTables* tab) {
    if (num_groups <= 0) return cudaSuccess;
    return p.rows_per_stream > 8 ? launch_one<16>(p, maps, num_groups, stream, tab)
                                 : launch_one<8>(p, maps, num_groups, stream, tab);
}

}  // namespace yoco
