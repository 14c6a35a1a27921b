// Split-KV decode over a paged 4-bit cache: 64 bytes of codes and four fp16 scales a row (32 channels share a
// scale, value = (code - 8) * scale), head dimension 128.  A CTA works off the segments of its group one after the other; its
// warps take whole tiles in turn, each loads its own into places that nobody else touches (no producer, no ring, no
// pieces handed out at run time), and their states are merged at the end of every segment.  A 64-key tile is 4 KB of codes and
// 512 bytes of scales per tensor, 9 KB in all, so at the same HBM bandwidth a key has to be worked off in a little over half
// of the 8-bit kernel's time.  What this kernel does about that is to spend few instructions per key:
//
//   codes    No conversion instruction.  A code n sits in the low bits of an fp16 word after one AND, where it is
//            the subnormal n 2^-24 (or 16 n 2^-24 for the nibble next to it): an exact multiple, and tensor-core
//            operands keep subnormals.  The factor 16 goes into Q, 2^24 into the softmax scale.  (q / 16 in fp16 is exact
//            where q is a multiple of 2^-20, as a bf16 value from 2^-13 on is; below, it is off by up to 2^-21.)
//   K        S = sum over groups j of  s_j(key) * 2^24 * (sum_c q_c n_c 2^-24  -  8 * 2^-24 * sum_c q_c).
//            The inner sums are the two products of a group; the scales are applied to their fp32 result, four
//            multiply-adds per group and 16 keys; the offsets of all groups are one small product per 16 keys, which
//            the sums start from.
//   V        sum over keys of P n s_j: here the group's scale is inside the sum.  It goes into P: P^T s_j in
//            fp16, one packed product per 16 keys and group.  The offset is subtracted tile by tile: the products of
//            64 keys start from -8 sum (P s_j), itself a product with a constant, and only then join O.  (Subtracted
//            at the end it would cancel: over many keys the sum of P n is far larger than the result.  Making
//            the codes signed first costs an addition per pair of them, 128 a tile instead of 16 products.)
//            O is rescaled by the same multiply-add.
//   order    Q is loaded in the channel order in which ldmatrix hands over the nibbles; the four channels of a
//            16-bit unit of V come out in four different products, which is one float4 per lane at the end.
//
// P is kept in [0, 2^7] (the exponential of s - max + 7) so that P times a small scale keeps its bits in fp16; a V scale
// stays below 448, and 2^7 * 448 is below the largest fp16 value.  Towards zero a P s below 2^-25 is lost to O (not to
// the log-sum-exp, which sums P in fp32): weights below 2^-32 / s of the row's largest.
//
// Bound by latency with three warps a scheduler, none of the units being full: 1M keys (32 query over 8 KV heads, pages of 64), kernel
// alone in short bursts at the full clock, take 215 us = 5,620 GB/s, 0.87 of the measured copy rate; a call in a loop of
// seconds, where the power cap takes the clock down, 239 to 257 us.  1,001 instructions a tile, of them 256 ANDs and 64 shifts
// that bring the codes into place: the ALU pipe is busy 53 % of the cycles, the tensor pipe 39 %, a warp issues in 59 %, and
// fixed latencies are the most frequent stall.  Sixteen rows (T = 4): 391 us.
// W = 12 because 168 registers a thread is the least that spills little: 8 / 12 / 16 warps 272 / 219 / 232 us.
#include "decode_f16.cuh"
#include "kernels.h"
#include "page_map.cuh"
#include "ptx.cuh"
#include "q4.cuh"
#include "tcgen05.cuh"

namespace yoco {

namespace {

constexpr int TILE_N = kDecodeTileN;          // 64 keys
constexpr int D = 128;                        // head dimension
constexpr int GROUPS = D / kQ4Group;          // scale groups of a row
constexpr int CODE_BYTES = TILE_N * D / 2;    // 4 KB: 32 lines of two keys' 64 bytes, 128-byte swizzle
constexpr int SCALE_BYTES = TILE_N * GROUPS * 2;
constexpr int ROW_BYTES = D / 2 + 2 * GROUPS; // codes and scales of a K (or V) row
// -8 and -128 times 2^-24, twice: the offset of the codes against V in place and 16 times too large
constexpr uint32_t kMinus8 = 0x80088008u, kMinus128 = 0x80808080u;
constexpr float kPShift = 7.f;                // P = 2^(s - max + kPShift)

// W warps per CTA, one CTA per SM; every warp has KH places for tiles of K and VH for tiles of V of its own.
template <int ROWS>
struct CfgQ4 {
    static constexpr int W = ROWS == 8 ? kQ4Warps8 : kQ4Warps16;
    static constexpr int KH = 2;
    static constexpr int VH = ROWS == 8 ? 1 : 2;
    static constexpr int H = KH + VH;
    static constexpr int THREADS = W * 32;
    static constexpr int OFF_SCALES = W * H * CODE_BYTES;
    static constexpr int OFF_MERGE = OFF_SCALES + W * H * SCALE_BYTES;
    static constexpr int OFF_ML = OFF_MERGE + W * ROWS * D * 4;
    static constexpr int OFF_BAR = OFF_ML + W * ROWS * 2 * 4;
    static constexpr int SMEM_BYTES = OFF_BAR + W * H * 8 + 8;
    static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
    static_assert((KH & (KH - 1)) == 0 && (VH & (VH - 1)) == 0, "places are counted with masks");
};

// D += A B; not volatile: only registers are involved, and the scheduler may move it
__device__ __forceinline__ void mma_f16_add(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D = A B + C with C kept
__device__ __forceinline__ void mma_f16_from(float (&d)[4], const float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                             uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// D(16x8) = A(16x8) B(8x8), tf32 operands, with A's columns 4 .. 7 the same as 0 .. 3
__device__ __forceinline__ void mma_tf32_twice(float (&d)[4], const float (&c)[4], float a0, float a1, float b0, float b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%4,%5}, {%6,%7}, "
        "{%8,%9,%10,%11};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(__float_as_uint(a0)), "r"(__float_as_uint(a1)), "r"(__float_as_uint(b0)), "r"(__float_as_uint(b1)), "f"(c[0]),
          "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// NB: boxes of a 64-key tile, 1 with pages of 64 keys and more, else 64 / P
template <int ROWS, int NB>
__device__ __forceinline__ void decode_q4_body(const CUtensorMap& tmK, const CUtensorMap& tmKs, const CUtensorMap& tmV,
                                               const CUtensorMap& tmVs, const DecodeParams& p,
                                               const DevSegment* segments, const int32_t* group_begin) {
    using C = CfgQ4<ROWS>;
    constexpr int W = C::W, KH = C::KH, VH = C::VH, H = C::H;

    extern __shared__ __align__(1024) uint8_t smem[];
    float* merge_o = reinterpret_cast<float*>(smem + C::OFF_MERGE);
    float2* merge_ml = reinterpret_cast<float2*>(smem + C::OFF_ML);
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);   // [W][H]: the K places, then the V places
    volatile int* give_up = reinterpret_cast<volatile int*>(full_bar + W * H);   // some thread ran out of patience

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;");

    if ((smem_u32(smem) & 1023u) != 0) {   // the swizzle arithmetic below needs 1 KB alignment
        if (threadIdx.x == 0) atomicCAS(p.status, 0, status_word(kWaitMisaligned, linear_cta()));
        return;
    }
    const Abort ab{give_up, p.status, p.wait_limit_ns > 0 ? p.wait_limit_ns : kWaitLimitNs};
    if (threadIdx.x == 0) {
        *give_up = 0;
        for (int b = 0; b < W * H; ++b) mbar_init(&full_bar[b], 1);
        mbar_fence_init();
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmKs);
        tma_prefetch_desc(&tmV);
        tma_prefetch_desc(&tmVs);
    }

    constexpr int NT = ROWS / 8;                       // 8-row groups on the narrow side of the products
    const int g = lane >> 2, tq = lane & 3;
    const int n_rows = p.rows_per_stream;
    // A tile's codes lie two keys to a 128-byte line, 128-byte swizzle: 16-byte chunk c (one scale group) of key k is chunk
    // ((k & 1) * 4 + c) ^ (line & 7) of line k / 2.  Sixteen keys further is 1024 bytes further, so two offsets,
    // for the groups 0, 1 and 2, 3, serve every ldmatrix of a tile.
    const int ld_key16 = ((lane >> 3) & 1) * 8 + (lane & 7);            // key row inside a 16-key group
    const int ld_line = ld_key16 >> 1, ld_first = ((ld_key16 & 1) << 2) | (lane >> 4);
    const uint32_t ld_off[2] = {(uint32_t)(ld_line * 128 + ((ld_first ^ ld_line) << 4)),
                                (uint32_t)(ld_line * 128 + (((ld_first | 2) ^ ld_line) << 4))};
    // four registers of zeros that the compiler does not know to be zeros: a literal would be written anew before
    // every product that starts from it
    float zero[4];
    asm volatile("mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;" : "=f"(zero[0]), "=f"(zero[1]), "=f"(zero[2]), "=f"(zero[3]));
    const float sscale = p.scale_log2 * 16777216.f;      // the codes of K count as n 2^-24

    // ---- the runs of this CTA: the segments of its group.  All warps walk them alike; tile i of a run is warp
    //      i % W's, so that sums are grouped the same in every launch ----
    int si = group_begin[blockIdx.x];
    const int seg_hi = group_begin[blockIdx.x + 1];
    DevSegment run;
    auto next_run = [&]() -> bool {
        while (si < seg_hi) {
            run = segments[si++];
            if (run.k_begin < run.k_end) return true;
        }
        return false;
    };

    // ---- the loads of this warp.  Its tiles of a run, m = 0, 1, .., are the run's tiles warp + W m.  Their K and V go to
    //      places that nobody else touches: a place has one barrier, is never waited for to become free, and the
    //      warp sees every phase of its barriers.  Lane l holds the pool row of box l % nb of the tile number l / nb of a
    //      batch (nb boxes to a tile: 1, or 64 / P for small pages) ----
    constexpr int nb_shift = NB == 1 ? 0 : NB == 2 ? 1 : 2, row_shift = 6 - nb_shift;
    const int shift = NB == 1 ? p.pages.page_shift : row_shift;
    const uint32_t codes0 = smem_u32(smem) + warp * (H * CODE_BYTES), scales0 = smem_u32(smem) + C::OFF_SCALES + warp * (H * SCALE_BYTES);
    const uint32_t bar0 = smem_u32(full_bar + warp * H);
    uint32_t done_tiles = 0;             // tiles worked off before this run
    uint32_t issued_k = 0, issued_v = 0; // halves asked for in this run
    int m_count = 0, batch = 0;          // tiles of this warp in the run; first tile of the batch whose rows are held
    int32_t box_row = 0, earlier_row = 0;   // of this batch, and of the one before: V is asked for later than K
    bool ok = true;
    auto load_batch = [&](int first) {
        batch = first;
        earlier_row = box_row;
        const int j = lane & ((1 << nb_shift) - 1);
        const int key = run.k_begin + (warp + W * (first + (lane >> nb_shift))) * TILE_N + (j << shift);
        box_row = 0;
        if ((((key >> shift) + 1) << shift) <= first_seen(run.n_full, p.window)) {
            box_row = p.pages.rows;              // nobody sees a key of it
        } else if (key < run.k_end) {
            const int b = run.stream / p.pages.Hkv, head = run.stream - b * p.pages.Hkv;
            const int page = __ldg(p.pages.table + (int64_t)b * p.pages.table_stride + (key >> shift));
            if ((uint32_t)page < (uint32_t)p.pages.num_pages) {
                box_row = page * p.pages.page_rows + (head << shift) + (shift > 6 ? key & ((1 << shift) - 1) : 0);
            } else {
                report_bad_page(p.status);
                box_row = p.pages.rows;          // behind the pool: the copy fills with zeros
            }
        }
    };
    // Asks for K (or V) of tile m into place `place` of the warp.
    // (The count of boxes is a constant of the kernel, so that one elected stretch issues them all: a turn of its own per
    // box, or a count known at run time only, cost 15 to 25 % of the bandwidth at P = 16 and 32.)
    auto issue = [&](const CUtensorMap& tm, const CUtensorMap& tms, int m, uint32_t place) {
        if (((m - batch) << nb_shift) >= 32) load_batch(m);
        const int from = (m - batch) << nb_shift;           // below 0: in the batch before
        const int32_t held = from < 0 ? earlier_row : box_row;
        const uint32_t bar = bar0 + 8 * place, codes = codes0 + place * CODE_BYTES, scales = scales0 + place * SCALE_BYTES;
        int row[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) row[j] = __shfl_sync(0xffffffffu, held, (from & 31) + j);
        const int left = NB == 1 ? TILE_N : run.k_end - (run.k_begin + (warp + W * m) * TILE_N);
        if (left >= TILE_N) {
            if (elect_one()) {
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "n"(TILE_N * ROW_BYTES) : "memory");
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    tma_load_2d(codes + j * (CODE_BYTES / NB), &tm, 0, row[j] >> 1, bar);
                    tma_load_2d(scales + j * (SCALE_BYTES / NB), &tms, 0, row[j] >> 4, bar);
                }
            }
        } else {                          // the last tile of a sequence: only the pages that hold a key of it
            const int n_box = (left + (1 << row_shift) - 1) >> row_shift;
            if (elect_one()) {
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((n_box * ROW_BYTES) << row_shift) : "memory");
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (j < n_box) {
                        tma_load_2d(codes + j * (CODE_BYTES / NB), &tm, 0, row[j] >> 1, bar);
                        tma_load_2d(scales + j * (SCALE_BYTES / NB), &tms, 0, row[j] >> 4, bar);
                    }
            }
        }
        __syncwarp();
    };
    auto issue_k = [&]() {
        if ((int)issued_k < m_count) {
            issue(tmK, tmKs, issued_k, (done_tiles + issued_k) & (KH - 1));
            ++issued_k;
        }
    };
    auto issue_v = [&]() {
        if ((int)issued_v < m_count) {
            issue(tmV, tmVs, issued_v, KH + ((done_tiles + issued_v) & (VH - 1)));
            ++issued_v;
        }
    };
    auto start_run = [&]() {              // nothing of this warp is under way
        const int n_tiles = (run.k_end - run.k_begin + TILE_N - 1) / TILE_N;
        m_count = ok && warp < n_tiles ? (n_tiles - warp + W - 1) / W : 0;
        issued_k = issued_v = p.selftest_skip_loads ? m_count : 0;
        if (m_count > 0) load_batch(0);
#pragma unroll
        for (int i = 0; i < (KH > VH ? KH : VH); ++i) {
            if (i < KH) issue_k();
            if (i < VH) issue_v();
        }
    };
    // On the way out: what this warp asked for and has not waited for must have landed before it leaves (the CTA ends
    // with its last thread, and its shared memory then belongs to another CTA).  Tiles of the run from which on.
    auto drain = [&](uint32_t k, uint32_t v) {
        if (lane != 0 || p.selftest_skip_loads) return;
        for (; k < issued_k; ++k)
            if (!drain_wait(full_bar + warp * H + ((done_tiles + k) & (KH - 1)), ((done_tiles + k) / KH) & 1u, ab)) return;
        for (; v < issued_v; ++v)
            if (!drain_wait(full_bar + warp * H + KH + ((done_tiles + v) & (VH - 1)), ((done_tiles + v) / VH) & 1u, ab)) return;
    };
    // the queries of a run, as they lie in memory: row 8 nt + g, channels 32 j + 8 tq .. + 7
    uint4 q_raw[NT][GROUPS];
    auto load_q = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = 8 * nt + g;
            const __nv_bfloat16* q = p.Q + ((int64_t)run.q_row0 + row) * D + tq * 8;
#pragma unroll
            for (int j = 0; j < GROUPS; ++j)
                q_raw[nt][j] = row < n_rows ? __ldg(reinterpret_cast<const uint4*>(q + j * 32)) : make_uint4(0u, 0u, 0u, 0u);
        }
    };

    bool more = next_run();
    if (more) load_q();
    __syncthreads();                      // the barriers are there
    if (more) start_run();
    while (more) {
        // Q^T as the second operand of the score products (fp16).  The two products of group j cover its 32 channels;
        // this lane's slots (k = 2 tq, 2 tq + 1, 2 tq + 8, 2 tq + 9) of product u stand for channels
        // 32 j + 8 tq + {2 u, 2 u + 4, 2 u + 1, 2 u + 5} of query row 8 nt + g, the last two divided by 16:
        // the nibbles that one AND brings into place, and those that come out 16 times too large.
        uint32_t qb[NT][GROUPS][2][2];
        // The offset 8 of the codes: -8 * 2^-24 * (sum of the group's q) times the scale of the key's group, summed over the
        // groups, is a product of four terms itself: [keys x groups] [groups x rows], in tf32 with the second
        // operand as the sum of two (the scales fit).  This lane's part: group tq, row 8 nt + g.
        float qoff[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float own = 0.f;
#pragma unroll
            for (int j = 0; j < GROUPS; ++j) {
                const uint4 w = q_raw[nt][j];
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
                if (j == tq) own = sum * (-8.f / 16777216.f);
            }
            qoff[nt][0] = __uint_as_float(__float_as_uint(own) & 0xFFFFE000u);       // ten bits of mantissa
            qoff[nt][1] = own - qoff[nt][0];
        }
        const int n_full = run.n_full;
        const int seen = first_seen(n_full, p.window);
        const int n_edge = min(n_full, run.n_kv);      // tiles that end at or below it need no mask
        int vis[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) vis[nt][e] = min(run.n_kv, max(0, n_full + ((8 * nt + 2 * tq + e) % p.T)));

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

        for (int m_tile = 0; m_tile < m_count; ++m_tile) {
            const int k0 = run.k_begin + (warp + W * m_tile) * TILE_N;
            const uint32_t count = done_tiles + m_tile, kp = count & (KH - 1), vp = KH + (count & (VH - 1));
            if (!warp_wait_ready(full_bar + warp * H + kp, (count / KH) & 1u, ab, kWaitRingFull)) {
                ok = false;         // this warp touches no tile any more; it still walks to the barriers below
                drain(m_tile, m_tile);
                __syncwarp();
                break;
            }
            const uint32_t kbase = codes0 + kp * CODE_BYTES;
            const uint8_t* ks_tile = smem + C::OFF_SCALES + (warp * H + kp) * SCALE_BYTES;
            // ---- S^T = K Q^T for 64 keys: four 16-key groups, four scale groups of two products each ----
            float s[NT][4][4];     // [row group][16-key group]: (key g, rows 2 tq, 2 tq + 1), (key g + 8, same rows)
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                const uint8_t* sc = ks_tile + (mt * 16 + g) * 8;
                const uint2 sa = *reinterpret_cast<const uint2*>(sc), sb = *reinterpret_cast<const uint2*>(sc + 64);   // keys g, g + 8
                const float2 sa01 = h2_to_f2(sa.x), sa23 = h2_to_f2(sa.y), sb01 = h2_to_f2(sb.x), sb23 = h2_to_f2(sb.y);
                const float ka[4] = {sa01.x, sa01.y, sa23.x, sa23.y}, kb[4] = {sb01.x, sb01.y, sb23.x, sb23.y};
                const float own_a = __half2float(*reinterpret_cast<const __half*>(sc + 2 * tq));
                const float own_b = __half2float(*reinterpret_cast<const __half*>(sc + 64 + 2 * tq));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_tf32_twice(s[nt][mt], zero, own_a, own_b, qoff[nt][0], qoff[nt][1]);
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                    uint32_t r[4];   // (keys 0-7, group 2 jj) (keys 8-15, 2 jj) (keys 0-7, 2 jj + 1) (keys 8-15, 2 jj + 1)
                    ldmatrix_x4(kbase + ld_off[jj] + mt * 1024, r[0], r[1], r[2], r[3]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int j = 2 * jj + h;
                        const uint32_t a = r[2 * h], b = r[2 * h + 1], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float t[4];
                            mma_f16_from(t, zero, a & 0x000F000Fu, b & 0x000F000Fu, a & 0x00F000F0u, b & 0x00F000F0u,
                                         qb[nt][j][0][0], qb[nt][j][0][1]);
                            mma_f16_add(t, a8 & 0x000F000Fu, b8 & 0x000F000Fu, a8 & 0x00F000F0u, b8 & 0x00F000F0u,
                                        qb[nt][j][1][0], qb[nt][j][1][1]);
                            s[nt][mt][0] = fmaf(t[0], ka[j], s[nt][mt][0]);
                            s[nt][mt][1] = fmaf(t[1], ka[j], s[nt][mt][1]);
                            s[nt][mt][2] = fmaf(t[2], kb[j], s[nt][mt][2]);
                            s[nt][mt][3] = fmaf(t[3], kb[j], s[nt][mt][3]);
                        }
                    }
                }
            }
            // ---- mask (causal edge, sequence end, window start), online softmax ----
            if (k0 + TILE_N > n_edge || (p.window > 0 && k0 < n_full + p.T - 1 - p.window)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int lo = p.window > 0 ? n_full + ((8 * nt + 2 * tq + e) % p.T) - p.window : -1;
#pragma unroll
                        for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                            for (int hh = 0; hh < 2; ++hh) {
                                const int jj = k0 + mt * 16 + hh * 8 + g;
                                if (!(jj < vis[nt][e] && jj >= lo)) s[nt][mt][2 * hh + e] = -INFINITY;
                            }
                    }
            }
            float alpha[NT][2];
            uint32_t pb[NT][4][2];     // P^T (fp16) as the second operand of O^T += V^T P^T: [16-key group][keys 0-7 / 8-15]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // the scale is positive, so the largest raw score has the largest scaled one
                    const float m01 = fmax3(s[nt][0][e], s[nt][0][2 + e], s[nt][1][e]);
                    const float m12 = fmax3(s[nt][1][2 + e], s[nt][2][e], s[nt][2][2 + e]);
                    float mx = fmax3(fmax3(m01, m12, s[nt][3][e]), s[nt][3][2 + e], -INFINITY);
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    const float mn = fmaxf(m[nt][e], mx * sscale);
                    const float ms = mn == -INFINITY ? 0.f : mn, mp = ms - kPShift;
                    alpha[nt][e] = ex2_fast(m[nt][e] - ms);
                    m[nt][e] = mn;
                    float sum = 0.f;
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            const float pv = ex2_fast(fmaf(s[nt][mt][2 * hh + e], sscale, -mp));
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
            // K has been read (the scores came out of it): its place takes the tile after next
            __syncwarp();
            issue_k();
            if (!warp_wait_ready(full_bar + warp * H + vp, (count / VH) & 1u, ab, kWaitRingFull)) {
                ok = false;
                drain(m_tile + 1, m_tile);
                __syncwarp();
                break;
            }
            const uint32_t vbase = codes0 + vp * CODE_BYTES;
            uint8_t* vs_tile = smem + C::OFF_SCALES + (warp * H + vp) * SCALE_BYTES;
            // ---- rows past the end of the sequence (or before all windows) may hold anything, and their boxes may not
            //      have been loaded: any code is a finite value, but a scale could be NaN, and 0 * NaN must not reach O ----
            const bool edge = k0 + TILE_N > run.n_kv || k0 < seen;
            if (edge) {
                for (int r = lane; r < TILE_N; r += 32)
                    if (k0 + r >= run.n_kv || k0 + r < seen) *reinterpret_cast<uint2*>(vs_tile + r * 8) = make_uint2(0u, 0u);
                __syncwarp();
            }
            // ---- O^T = alpha O^T + V^T (P^T s).  P^T s in fp16, per scale group: ----
            uint32_t ps[NT][4][GROUPS][2];     // [16-key group][scale group][keys 0-7 / 8-15]
#pragma unroll
            for (int kg = 0; kg < 4; ++kg)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    // scales of keys 2 tq and 2 tq + 1: (s0 s1 | s2 s3) of either, regrouped per scale group
                    const uint4 w = *reinterpret_cast<const uint4*>(vs_tile + (kg * 16 + hh * 8 + 2 * tq) * 8);
                    const uint32_t sv[GROUPS] = {__byte_perm(w.x, w.z, 0x5410), __byte_perm(w.x, w.z, 0x7632),
                                                 __byte_perm(w.y, w.w, 0x5410), __byte_perm(w.y, w.w, 0x7632)};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < GROUPS; ++j) ps[nt][kg][j][hh] = h2_mul(pb[nt][kg][hh], sv[j]);
                }
            // The transposed ldmatrix hands this lane, for keys 2 tq and 2 tq + 1 of an 8-key group, the 16-bit unit g of a
            // 16-byte chunk: four channels of a scale group.
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
                float t[NT][2][2][4], off[NT][2][4];          // [group 2 jj + h][product tile]
                // -8 sum of (P s): a product with a constant, the starting point of both tiles of a group
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float o[4];
#pragma unroll
                        for (int kg = 0; kg < 4; ++kg) {
                            const uint32_t p0 = ps[nt][kg][2 * jj + h][0], p1 = ps[nt][kg][2 * jj + h][1];
                            if (kg == 0) mma_f16_from(o, zero, kMinus8, kMinus128, kMinus8, kMinus128, p0, p1);
                            else mma_f16_add(o, kMinus8, kMinus128, kMinus8, kMinus128, p0, p1);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) off[nt][h][e] = o[e];
                    }
#pragma unroll
                for (int kg = 0; kg < 4; ++kg) {
                    uint32_t r[4];   // (keys 0-7, group 2 jj) (keys 8-15, 2 jj) (keys 0-7, 2 jj + 1) (keys 8-15, 2 jj + 1)
                    ldmatrix_x4_trans(vbase + ld_off[jj] + kg * 1024, r[0], r[1], r[2], r[3]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t a = r[2 * h], b = r[2 * h + 1], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint32_t p0 = ps[nt][kg][2 * jj + h][0], p1 = ps[nt][kg][2 * jj + h][1];
                            if (kg == 0) {
                                mma_f16_from(t[nt][h][0], off[nt][h], a & 0x000F000Fu, a & 0x00F000F0u, b & 0x000F000Fu, b & 0x00F000F0u, p0, p1);
                                mma_f16_from(t[nt][h][1], off[nt][h], a8 & 0x000F000Fu, a8 & 0x00F000F0u, b8 & 0x000F000Fu, b8 & 0x00F000F0u, p0, p1);
                            } else {
                                mma_f16_add(t[nt][h][0], a & 0x000F000Fu, a & 0x00F000F0u, b & 0x000F000Fu, b & 0x00F000F0u, p0, p1);
                                mma_f16_add(t[nt][h][1], a8 & 0x000F000Fu, a8 & 0x00F000F0u, b8 & 0x000F000Fu, b8 & 0x00F000F0u, p0, p1);
                            }
                        }
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc[nt][2 * jj + h][u][e] = fmaf(acc[nt][2 * jj + h][u][e], alpha[nt][e & 1], t[nt][h][u][e]);
            }
            if (edge) fence_proxy_async_smem();   // generic writes before TMA reuse
            // the products must have been issued, i.e. V read, before its place in the ring is given away
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    asm volatile("" : "+f"(acc[nt][j][0][0]), "+f"(acc[nt][j][0][1]), "+f"(acc[nt][j][0][2]), "+f"(acc[nt][j][0][3]),
                                      "+f"(acc[nt][j][1][0]), "+f"(acc[nt][j][1][1]), "+f"(acc[nt][j][1][2]), "+f"(acc[nt][j][1][3]));
            __syncwarp();
            issue_v();
        }
        done_tiles += m_count;

        // the next run's first loads are on their way while this one is merged
        const DevSegment done = run;
        const int active = min(W, (run.k_end - run.k_begin + TILE_N - 1) / TILE_N);   // warps that had a tile
        more = next_run();
        const bool mine = m_count > 0;
        if (more) start_run();

        // ---- merge the warps' states, write the final rows or this segment's partial ----
        if (mine) {
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
                            make_float4(acc[nt][j][0][e] * 16777216.f, acc[nt][j][0][2 + e] * 1048576.f,
                                        acc[nt][j][1][e] * 16777216.f, acc[nt][j][1][2 + e] * 1048576.f);
                    if (g == 0) merge_ml[warp * ROWS + row] = make_float2(m[nt][e], l[nt][e]);
                }
        }
        // one answer for all warps (a barrier that ORs): nobody may be left waiting at a later barrier
        if (named_barrier_or(1, W * 32, !ok)) {
            if (more && ok) drain(0, 0);
            break;
        }
        const bool final_out = done.stream_nseg == 1 && !p.force_partial;
        for (int idx = threadIdx.x; idx < n_rows * (D / 4); idx += W * 32) {
            const int r = idx / (D / 4), col = 4 * (idx - r * (D / 4));
            float M = -INFINITY;
            for (int w = 0; w < active; ++w) M = fmaxf(M, merge_ml[w * ROWS + r].x);
            float L = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            if (M != -INFINITY)
                for (int w = 0; w < active; ++w) {
                    const float2 ml = merge_ml[w * ROWS + r];
                    const float4 v = *reinterpret_cast<const float4*>(merge_o + (w * ROWS + r) * D + col);
                    const float f = ex2_fast(ml.x - M);
                    L = fmaf(ml.y, f, L);
                    o.x = fmaf(v.x, f, o.x);
                    o.y = fmaf(v.y, f, o.y);
                    o.z = fmaf(v.z, f, o.z);
                    o.w = fmaf(v.w, f, o.w);
                }
            const float inv = L > 0.f ? 1.f / L : 0.f;
            const float lse = L > 0.f ? (M + log2f(L) - kPShift) * 0.6931471805599453f : -INFINITY;
            if (final_out) {
                *reinterpret_cast<uint2*>(p.O + ((int64_t)done.q_row0 + r) * D + col) =
                    make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
                if (p.lse && col == 0) p.lse[done.q_row0 + r] = lse;
            } else {
                *reinterpret_cast<float4*>(p.part_o + ((int64_t)done.slot * n_rows + r) * D + col) =
                    make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
                if (col == 0) p.part_lse[(int64_t)done.slot * n_rows + r] = lse;
            }
        }
        if (more) load_q();
        named_barrier_sync(1, W * 32);
    }
}

template <int ROWS, int NB>
__global__ void __launch_bounds__(CfgQ4<ROWS>::THREADS, 1)
decode_q4_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmKs,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmVs,
                 const __grid_constant__ DecodeParams p) {
    decode_q4_body<ROWS, NB>(tmK, tmKs, tmV, tmVs, p, p.segments, p.group_begin);
}

// work tables as kernel parameters
template <int ROWS, int NB>
__global__ void __launch_bounds__(CfgQ4<ROWS>::THREADS, 1)
decode_q4_kernel_inline(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmKs,
                        const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmVs,
                        const __grid_constant__ DecodeParams p, const __grid_constant__ DecodeInlineTables tab) {
    decode_q4_body<ROWS, NB>(tmK, tmKs, tmV, tmVs, p, tab.seg, tab.group_begin);
}

template <int ROWS, int NB>
cudaError_t launch_one(const DecodeParams& p, const PagedQ4Maps& m, int num_groups, cudaStream_t stream,
                       const DecodeInlineTables* tab) {
    if (tab)
        decode_q4_kernel_inline<ROWS, NB><<<num_groups, CfgQ4<ROWS>::THREADS, CfgQ4<ROWS>::SMEM_BYTES, stream>>>(m.k, m.k_scale, m.v, m.v_scale, p, *tab);
    else
        decode_q4_kernel<ROWS, NB><<<num_groups, CfgQ4<ROWS>::THREADS, CfgQ4<ROWS>::SMEM_BYTES, stream>>>(m.k, m.k_scale, m.v, m.v_scale, p);
    return cudaGetLastError();
}

template <int ROWS, int NB>
cudaError_t setup_one() {
    cudaError_t e = cudaFuncSetAttribute(decode_q4_kernel<ROWS, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         CfgQ4<ROWS>::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(decode_q4_kernel_inline<ROWS, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                CfgQ4<ROWS>::SMEM_BYTES);
}

}  // namespace

cudaError_t decode_q4_kernel_setup() {
    cudaError_t e;
    if ((e = setup_one<8, 1>()) != cudaSuccess) return e;
    if ((e = setup_one<8, 2>()) != cudaSuccess) return e;
    if ((e = setup_one<8, 4>()) != cudaSuccess) return e;
    if ((e = setup_one<16, 1>()) != cudaSuccess) return e;
    if ((e = setup_one<16, 2>()) != cudaSuccess) return e;
    return setup_one<16, 4>();
}

namespace {
template <int ROWS>
cudaError_t launch_any(const DecodeParams& p, const PagedQ4Maps& maps, int num_groups, cudaStream_t stream,
                       const DecodeInlineTables* tab) {
    if (p.pages.page_shift == 4) return launch_one<ROWS, 4>(p, maps, num_groups, stream, tab);
    if (p.pages.page_shift == 5) return launch_one<ROWS, 2>(p, maps, num_groups, stream, tab);
    return launch_one<ROWS, 1>(p, maps, num_groups, stream, tab);
}
}  // namespace

cudaError_t launch_decode_q4(const DecodeParams& p, const PagedQ4Maps& maps, int num_groups, cudaStream_t stream,
                             const DecodeInlineTables* tab) {
    if (num_groups <= 0) return cudaSuccess;
    return p.rows_per_stream > 8 ? launch_any<16>(p, maps, num_groups, stream, tab)
                                 : launch_any<8>(p, maps, num_groups, stream, tab);
}

}  // namespace yoco
