// Gated retention, chunkwise form, on the tcgen05 tensor cores.
//
// A chunk is 128 tokens of one head.  With b_i = log2 g_1 + .. + log2 g_i inside the chunk, S the state before it and C its last token:
//     P_ij = (q_i . k_j) 2^(b_i - b_j)  (j <= i),   o_i = scale (sum_j P_ij v_j + 2^b_i q_i S),
//     S' = 2^b_C S + sum_j (2^(b_C - b_j) k_j)^T v_j.
// A CTA walks a contiguous range of chunks, of one (sequence, head) stream or of several one after the other, with the state in the
// registers of two warpgroups.  1,024 threads:
//   warp 0       TMA producer: K, Q, V tiles (128 tokens x d, 128-byte swizzle); asks for the gate's rows
//   warp 1       issuer of Q K^T -> SC, Q S -> O[n & 1], P V on top of it      (tensor memory, fp32)
//   warp 3       issuer of K'^T V -> DS
//   warp 2       decays: prefix sums of the logarithms in 64 bits, kept as integer part and rest (b_i - b_j is the difference of
//                both: exact to 2^-24 however strong the decays before j were), and the factors that depend on one token alone
//   warpgroup 1  thread = token: P (bf16, over the scores' own columns: it goes to P V from tensor memory)
//   warpgroups 2, 5  thread = token, every other chunk each: the output: scale, normalisation, gate, rounding, store
//   warpgroups 3, 4  thread = half a row of the state: S' from S and DS in fp32, S in bf16 to shared memory for Q S; 2^b_i times
//                Q S, in place
//   warpgroups 6, 7  K' = 2^(b_C - b_j) k_j, in pieces of 32 tokens
// Decays of P: in the 32 x 32 blocks on the diagonal one exponential per element; below it 2^(b_i - m) 2^(m - b_j), m the value at the
// end of j's block: both factors are at most 1, and the second is the same for all rows.
// With few streams a first pass over K and V (STATES) leaves the state of each CTA's range, a merge puts those in order, and the main
// pass starts every range from its own: all SMs work, K and V are read twice.  In that first pass warpgroups 1, 2, 6 and 7 make K', a piece each, in
// tensor memory.
// What bounds it: not the bytes (measured: 47% and 55% of the memory's rate in the two passes) nor the tensor cores (39%, 40%), but the
// roles' chain, through shared memory's data pipe: a chunk's matrix products read 320 KB of operands there, the copies write 96 KB, K' and S another
// 130 KB (the pipe: 37% of the cycles the tensor cores' operands, 61% the threads' accesses, tensor memory's among them).  What took load off
// it made it faster (output and gate past it, K' of the first pass to tensor memory), and so did fewer instructions on the chain (uniform registers).
// Measured (d = 128): one sequence of 32,719 tokens, 32 heads 430-434 us in a long row of calls (1.08 GB needed: 164 us at 6.56 TB/s), in which the SM
// clock falls, 347-366 in short bursts, with gate 410; 4,096 tokens 68 in bursts, with gate 78, 82-83 in a long row; four of 4,096 tokens, 37 heads, whole
// streams, in bursts 136-141 (0.69-0.72 of that rate), with gate 172-180; one chunk 13.
// Roundings: P and the copy of S that multiplies Q go to bf16 (half a step, up to 2^-8 of the value, like the output's own): products of
// bf16 keep fp32's range at the tensor cores' full rate.  Outputs are 2.3e-3 off (2-norm), 1.7e-3 with their own rounding alone.  A group norm that takes a common offset of V out
// leaves these roundings: 2.7e-3 with an offset of 3 deviations, 5.2e-3 to 5.6e-3 with 10.  K' goes to
// the tensor cores as a sum of bf16: where the sums leave the kernel as a state, of three (24 bits; with one it would be 1.7e-3 off (2-norm),
// with two 2e-6), where they only multiply Q inside, of two.
#include <type_traits>

#include "gret.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rows.cuh"
#include "tcgen05.cuh"

namespace yoco {

namespace {

constexpr int CT = kGretChunk;                 // 128 tokens
constexpr int kThreads = 1024;
constexpr int HALF_BYTES = CT * 128;           // Q: 128 rows x 64 bf16, one swizzled half of a tile
constexpr int HT = CT / 2;                     // K and V come by halves of a chunk: 64 tokens
constexpr int SUB_BYTES = HT * 128;            // 64 rows x 64 bf16
constexpr int PIECE = 32;                      // tokens of a piece of K'
constexpr int PIECES = CT / PIECE;
constexpr int PIECE_HALF = PIECE * 128;        // 64 channels of a piece of one of K's parts
constexpr int TERM_BYTES = 2 * PIECE_HALF;
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t COL_SC = 0, COL_O = 128, COL_DS = 384;     // two buffers of O
// The state-only pass has the first 128 columns for a second buffer of DS, and the four pieces of K' where O is otherwise.
constexpr uint32_t COL_KP = COL_O, KP_COLS = PIECE / 2;       // of each part
// Registers per thread after the split; the CTA starts with 64 each.
constexpr int kRegsIo = 56, kRegsP = 56, kRegsOut = 72, kRegsState = 88, kRegsKeys = 40;
static_assert(kRegsIo + kRegsP + 2 * kRegsOut + 2 * kRegsState + 2 * kRegsKeys <= 8 * 64, "register pool of the CTA");
static_assert(kRegsIo <= 64 && kRegsP <= 64 && kRegsKeys <= 64 && kRegsOut >= 64 && kRegsState >= 64, "which way the split goes");
constexpr int kRegsAcross = 64, kRegsIdle = 24;               // the state-only pass: four warpgroups make K', one has nothing to do
static_assert(kRegsIo + 4 * kRegsAcross + kRegsIdle + 2 * kRegsState <= 8 * 64, "register pool of the CTA");
constexpr int kTerms = 3;                      // parts of K', where a state leaves; otherwise kTermsInside
constexpr int kTermsInside = 2;

// STATES: only the states, of the segments that streams are cut into.
template <int D, bool STATES>
struct GCfg {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;     // Q
    static constexpr int KV_BYTES = HALVES * SUB_BYTES;        // 64 tokens of K or V
    // Places in shared memory: half chunks of K and V (three: one and a half chunks, so that the next one's first half is there before
    // this one's second half has gone), chunks of Q.  The state-only pass, with K' in tensor memory, has room for three chunks.
    static constexpr int KS = STATES ? 6 : D == 64 ? 4 : 3, VS = KS, QS = STATES ? 0 : D == 64 ? 2 : 1;
    // K' pieces: places of three parts each, or in the same memory (not STATES) half as many again of two.
    static constexpr int KP_WIDE = STATES ? 4 : 2, KP_NARROW = 3, KP_STAGES = STATES ? 4 : 3;
    static constexpr int OFF_K = 0;
    static constexpr int OFF_Q = OFF_K + KS * KV_BYTES;
    static constexpr int OFF_V = OFF_Q + QS * TILE_BYTES;
    static constexpr int OFF_KP = OFF_V + VS * KV_BYTES;
    static constexpr int OFF_S = OFF_KP + (STATES ? 0 : KP_WIDE * kTerms * TERM_BYTES);
    static constexpr int OFF_DEC = OFF_S + (STATES ? D * 128 : D * D * 2);    // (the state-only pass: a way through for rows of the state)
    // Of a chunk: 2^(b_C - b_j); whole part and rest of b_C; and where there is output: whole parts and rests of -b_j; 2^(m - b_j).
    static constexpr int DEC_END = CT, DEC_WHOLE = CT + 4, DEC_REST = DEC_WHOLE + CT, DEC_U = DEC_REST + CT;
    static constexpr int DEC_FLOATS = STATES ? DEC_WHOLE : DEC_U + CT;
    static constexpr int OFF_BAR = OFF_DEC + 2 * DEC_FLOATS * 4;
    static constexpr int NUM_BARS = 2 * (KS + QS + VS) + 2 * KP_STAGES + 22;
    static constexpr int SMEM_BYTES = OFF_BAR + NUM_BARS * 8 + 16;
    static_assert(SMEM_BYTES <= 227 * 1024 && OFF_DEC % 16 == 0 && OFF_BAR % 8 == 0, "shared memory");
    static_assert(KP_NARROW * kTermsInside <= KP_WIDE * kTerms, "places of K'");
};

// The bounded wait of this kernel: one answer for the warp, in few instructions; what ran out is reported at the role's end.  The roles'
// loops together have to stay in the instruction cache of the SM, which is why they are rolled up wherever registers are not indexed by
// them.  (With everything unrolled, more than twice the code, one sequence of 32,768 tokens took 583 us, as it was then, instead of 400.)
struct Wait {
    int32_t limit_ns;
    int32_t what = 0;
    __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity, int32_t wait_class) {
        uint32_t polls = 0, t0 = 0;
        while (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) {
            uint32_t t;
            asm volatile("mov.u32 %0, %globaltimer_lo;" : "=r"(t));
            if (polls == 0) t0 = t;
            if (__any_sync(0xffffffffu, (int32_t)(t - t0) > limit_ns || ++polls >= kWaitMaxPolls)) {
                what = wait_class;
                return false;
            }
        }
        return true;
    }
};

// Places of half chunks, used in turn, and the parity of the time round.
template <int N>
struct Turn {
    uint32_t at = 0, round = 0;
    __device__ __forceinline__ void next() {
        if (++at == (uint32_t)N) {
            at = 0;
            round ^= 1u;
        }
    }
};
// The place of use n in a ring of N (a power of two), and the parity of its time round.
template <int N>
__device__ __forceinline__ uint32_t place(uint32_t n) { return n & (uint32_t)(N - 1); }
template <int N>
__device__ __forceinline__ uint32_t round_of(uint32_t n) { return (n / (uint32_t)N) & 1u; }

// The sequence of a place in the flat space.
template <class Table>
__device__ __forceinline__ int sequence_at(const GretChunkParams& p, const Table& tab, int pos) {
    const int per = pos / p.base.H;                // tab.chunk0[b] <= per < tab.chunk0[b + 1]
    int lo = 0, hi = p.base.B - 1;
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.chunk0[mid] <= per) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// The segments of a CTA: chunks [c, c_end) of stream (b, h).  Split: a range of the flat space of (sequence, head, chunk); otherwise whole
// streams, every gridDim.x-th one (they are sorted by length).
template <class Table>
struct Walk {
    const GretChunkParams& p;
    const Table& tab;
    int pos, end;                                  // split: chunks of the flat space; otherwise streams
    int b, h, c, c_end, chunks;
    __device__ __forceinline__ Walk(const GretChunkParams& p_, const Table& tab_) : p(p_), tab(tab_) {
        const int g = blockIdx.x;
        pos = p.split ? p.first_of(g) : g;
        end = p.split ? p.first_of(g + 1) : p.base.B * p.base.H;
    }
    // Enters the segment at pos; false when there is none left.
    __device__ __forceinline__ bool enter() {
        if (pos >= end) return false;
        if (!p.split) {
            b = pos / p.base.H;
            h = pos - b * p.base.H;
            c = 0;
            c_end = chunks = tab.chunk0[b + 1] - tab.chunk0[b];
            pos += gridDim.x;
            return true;
        }
        b = sequence_at(p, tab, pos);
        chunks = tab.chunk0[b + 1] - tab.chunk0[b];
        const int in = pos - tab.chunk0[b] * p.base.H;
        h = in / chunks;
        c = in - h * chunks;
        c_end = min(chunks, c + (end - pos));
        pos += c_end - c;
        return true;
    }
    __device__ __forceinline__ bool whole_stream() const { return c == 0 && c_end == chunks; }
};

// 16 channels of a row, on 16 or (wide) on 32 bytes.
__device__ __forceinline__ void load_row16(const __nv_bfloat16* p, bool wide, uint32_t (&v)[8]) {
    if (wide) {
        asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
    } else {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p)), b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
}
__device__ __forceinline__ void store_row16(__nv_bfloat16* p, bool wide, const uint32_t (&v)[8]) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                     "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

__device__ __forceinline__ float exp2_parts(float whole, float rest) { return exp2f(whole) * exp2f(rest); }

template <int D, bool STATES, class Table>
__global__ void __launch_bounds__(kThreads, 1)
gret_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const GretChunkParams p, const __grid_constant__ Table tab) {
    using C = GCfg<D, STATES>;
    constexpr int QS = STATES ? 1 : C::QS;
    if (STATES) asm volatile("griddepcontrol.launch_dependents;");

    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
    uint64_t* k_full = bars;                               // [KS]
    uint64_t* k_empty = k_full + C::KS;
    uint64_t* q_full = k_empty + C::KS;                    // [QS]
    uint64_t* q_empty = q_full + C::QS;
    uint64_t* v_full = q_empty + C::QS;                    // [VS]
    uint64_t* v_empty = v_full + C::VS;
    uint64_t* kp_full = v_empty + C::VS;                   // [KP_STAGES]
    uint64_t* kp_empty = kp_full + C::KP_STAGES;
    uint64_t* dec_full = kp_empty + C::KP_STAGES;          // [2]
    uint64_t* dec_empty = dec_full + 2;                    // [2]
    uint64_t* o_full = dec_full + 4;                       // [2]
    uint64_t* o_empty = dec_full + 6;                      // [2]
    uint64_t* sc_full = dec_full + 8;
    uint64_t* qs_full = dec_full + 9;
    uint64_t* p_full = dec_full + 10;
    uint64_t* s_full = dec_full + 11;
    uint64_t* s_empty = dec_full + 12;
    uint64_t* ds_full = dec_full + 13;                     // [2], the state-only pass has two buffers of DS
    uint64_t* ds_empty = dec_full + 15;                    // [2]
    uint64_t* drain_bar = dec_full + 17;                   // [2]
    uint64_t* s_staged = dec_full + 19;
    uint64_t* v_cleared = dec_full + 20;                   // [2], by sequences' last chunks
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float* dec = reinterpret_cast<float*>(smem + C::OFF_DEC);

    // The same for all lanes, for the compiler to see, so that roles issue from uniform registers; but not where it measured worse.  (32 heads,
    // one sequence.  d = 128, 16,384 tokens: main pass 188 K cycles without it, 175 K with it, state-only pass 109 K and 118 K.  d = 64,
    // 4,096 tokens, both passes: state-only pass without / with it 53.6 / 52.1 us.)
    const int warp = STATES && D == 128 ? (int)threadIdx.x >> 5 : __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const Abort ab{abort_flag, p.status, kWaitLimitNs};
    const bool aligned_ok = (smem_u32(smem) & 1023u) == 0;

    if (threadIdx.x == 0) {
        *abort_flag = aligned_ok ? 0 : 1;
        if (!aligned_ok) atomicCAS(p.status, 0, status_word(kWaitMisaligned, linear_cta()));
        for (int i = 0; i < C::KS; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], STATES ? 8 : 9);        // the warps that make K' of it, and Q K^T
        }
        for (int i = 0; i < C::QS; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < C::VS; ++i) {
            mbar_init(&v_full[i], 1);
            mbar_init(&v_empty[i], STATES ? 1 : 2);        // K'^T V, and P V
        }
        for (int i = 0; i < C::KP_STAGES; ++i) {
            mbar_init(&kp_full[i], STATES ? 4 : 8);
            mbar_init(&kp_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&dec_full[i], 1);
            mbar_init(&dec_empty[i], STATES ? 24 : 20);
            mbar_init(&o_full[i], 1);
            mbar_init(&o_empty[i], 4);
            mbar_init(&v_cleared[i], 8);
        }
        mbar_init(sc_full, 1);
        mbar_init(qs_full, 1);
        mbar_init(p_full, 12);                             // P, and the scaled Q S
        for (int i = 0; i < 2; ++i) {
            mbar_init(&ds_full[i], 1);
            mbar_init(&ds_empty[i], 8);
        }
        mbar_init(s_full, 8);
        mbar_init(s_staged, 8);
        mbar_init(s_empty, 1);
        mbar_init(&drain_bar[0], 1);
        mbar_init(&drain_bar[1], 1);
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

    Wait wait{p.wait_limit_ns > 0 ? p.wait_limit_ns : (int32_t)kWaitLimitNs};
    // every role walks the same segments: `enter` moves to the next one
    Walk<Table> walk(p, tab);
    auto enter = [&]() -> bool {
        while (walk.enter())
            if (!STATES || !walk.whole_stream()) return true;
        return false;
    };
    // Places of K': their number and size go by the segment's number of parts; bit i of `par` is the parity of place i's uses.
    struct Pieces {
        uint32_t at = 0, par = 0, count = 0, bytes = 0;
        __device__ __forceinline__ void segment(int terms) {
            at = 0;
            count = terms == kTerms ? C::KP_WIDE : C::KP_NARROW;
            bytes = terms * TERM_BYTES;
        }
        __device__ __forceinline__ uint32_t parity(uint32_t i) const { return (par >> i) & 1u; }
        __device__ __forceinline__ uint32_t offset() const { return C::OFF_KP + at * bytes; }
        __device__ __forceinline__ void next() {
            par ^= 1u << at;
            at = at + 1 == count ? 0 : at + 1;
        }
    } pieces;
    // The makers of K' in the main pass, before a segment's first piece: all places have been given back (they may lie differently from now
    // on).  Not for the state-only pass: its places never move, and there a team fills one of them alone, so that the uses of the others may go on
    // before a slower team has looked, which would then take the phase after the one it waits for, of the same parity, for that one not yet over.
    auto all_given_back = [&]() {
#pragma unroll 1
        for (uint32_t i = 0; i < C::KP_STAGES; ++i)
            if (!wait(&kp_empty[i], pieces.parity(i) ^ 1u, kWaitTensor)) return false;
        return true;
    };
    // One thread's share of a piece of K': all of its rows at a time, eight channels a thread.
    auto make_piece = [&](int tid, uint32_t k_place, int e, const float* weight, int valid, int terms) {
        constexpr int ROWS = 256 / 8;
        const int row = tid >> 3;
        const uint32_t at = row * 128 + (((tid & 7) ^ (row & 7)) << 4);            // inside a piece's half; the same in a tile's
        const uint8_t* src = smem + C::OFF_K + k_place * C::KV_BYTES + (e & 1) * PIECE_HALF + at;
        uint8_t* dst = smem + pieces.offset() + at;
        auto put = [&](int t, int off, const uint32_t (&v)[4]) {
            *reinterpret_cast<uint4*>(dst + t * TERM_BYTES + off) = make_uint4(v[0], v[1], v[2], v[3]);
            // d = 64: the instruction's upper 64 rows are the same ones again (read by the second threads of the state's rows)
            if (D == 64) *reinterpret_cast<uint4*>(dst + t * TERM_BYTES + off + PIECE_HALF) = make_uint4(v[0], v[1], v[2], v[3]);
        };
#pragma unroll 1
        for (int r = 0; r < PIECE; r += ROWS) {
            const float w = weight[e * PIECE + r + row];
            const bool in = e * PIECE + r + row < valid;
#pragma unroll 1
            for (int hf = 0; hf < C::HALVES; ++hf) {
                uint4 raw = *reinterpret_cast<const uint4*>(src + hf * SUB_BYTES + r * 128);
                if (!in) raw = make_uint4(0u, 0u, 0u, 0u);
                const int off = hf * PIECE_HALF + r * 128;
                const uint32_t kk[4] = {raw.x, raw.y, raw.z, raw.w};
                if (!STATES && terms == kTermsInside) {
                    // w = w1 + w2 to 16 bits, and all of it in bf16 pairs: w1 k rounded, what that rounding left out (exact), w2 k on top of that
                    const uint32_t w1 = pack_bf16x2(w, w), w2 = pack_bf16x2(w - __uint_as_float(w1 << 16), w - __uint_as_float(w1 << 16));
                    uint32_t a[4], b[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        a[q] = bf2_mul(w1, kk[q]);
                        b[q] = bf2_fma(w2, kk[q], bf2_fma(w1, kk[q], a[q] ^ 0x80008000u));
                    }
                    put(0, off, a);
                    put(1, off, b);
                } else {
                    const uint64_t w2 = f2_pack(w, w);
                    uint64_t x[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) x[q] = f2_mul(w2, f2_pack(__uint_as_float(kk[q] << 16), __uint_as_float(kk[q] & 0xFFFF0000u)));
#pragma unroll
                    for (int t = 0; t < kTerms; ++t) {
                        uint32_t part[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float x0, x1;
                            f2_unpack(x[q], x0, x1);
                            part[q] = pack_bf16x2(x0, x1);
                            if (t + 1 < kTerms)
                                x[q] = f2_fma(f2_pack(__uint_as_float(part[q] << 16), __uint_as_float(part[q] & 0xFFFF0000u)), f2_pack(-1.f, -1.f), x[q]);
                        }
                        put(t, off, part);
                    }
                }
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&kp_full[pieces.at]);
    };
    // The state-only pass: a piece goes to tensor memory, where the product's first operand has a row (a channel) to a thread; it is read down
    // the columns of K.  (Shared memory's bandwidth is what bounds this pass: parts that are written to it and read from it are two thirds
    // of what goes through it.)
    auto make_piece_across = [&](uint32_t k_place, int e, const float* weight, int valid) {
        const int ch = ((warp & 3) * 32 + lane) % D;       // d = 64: the upper 64 rows are the same ones again
        uint8_t* src = smem + C::OFF_K + k_place * C::KV_BYTES + (ch >> 6) * SUB_BYTES + (e & 1) * PIECE_HALF + (ch & 7) * 2;
        auto key = [&](int t) { return reinterpret_cast<uint16_t*>(src + t * 128 + ((((ch >> 3) & 7) ^ (t & 7)) << 4)); };
        tc_fence_after();                                  // (the product that read this place before)
        const uint32_t dst = tmem_base + COL_KP + pieces.at * (kTerms * KP_COLS) + ((uint32_t)((warp & 3) * 32) << 16);
        if (e * PIECE + PIECE > valid) {                   // tokens behind the sequence: anything, and 0 times that is not 0
#pragma unroll 1
            for (int t = max(valid - e * PIECE, 0); t < PIECE; ++t) *key(t) = 0;
            fence_proxy_async_smem();                      // (before the next copy comes into this place)
        }
#pragma unroll 1
        for (int t = 0; t < PIECE; t += 16) {
            uint64_t x[8];
            const ulonglong2* w = reinterpret_cast<const ulonglong2*>(weight + e * PIECE + t);
#pragma unroll
            for (int q = 0; q < 8; q += 2) {
                const ulonglong2 w2 = w[q / 2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t k0 = *key(t + 2 * (q + i)), k1 = *key(t + 2 * (q + i) + 1);
                    x[q + i] = f2_mul(i ? w2.y : w2.x, f2_pack(__uint_as_float(k0 << 16), __uint_as_float(k1 << 16)));
                }
            }
#pragma unroll
            for (int p = 0; p < kTerms; ++p) {
                uint32_t part[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    float x0, x1;
                    f2_unpack(x[q], x0, x1);
                    part[q] = pack_bf16x2(x0, x1);
                    if (p + 1 < kTerms)
                        x[q] = f2_fma(f2_pack(__uint_as_float(part[q] << 16), __uint_as_float(part[q] & 0xFFFF0000u)), f2_pack(-1.f, -1.f), x[q]);
                }
                tmem_st8(dst + p * KP_COLS + t / 2, part);
            }
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&kp_full[pieces.at]);
    };
    // rows behind the sequence are the next one's, or none: they may hold anything, and 0 times that is not 0
    auto clear_tail = [&](int threads, int tid, Turn<C::VS> vat, int valid) {
        for (int half = 0; half < 2; ++half, vat.next()) {
            if (!wait(&v_full[vat.at], vat.round, kWaitRingFull)) return false;
#pragma unroll 1
            for (int i = tid; i < HT * 8 * C::HALVES; i += threads) {
                const int r = i & (HT - 1), q = i / HT;
                if (half * HT + r >= valid)
                    *reinterpret_cast<uint4*>(smem + C::OFF_V + vat.at * C::KV_BYTES + (q >> 3) * SUB_BYTES + r * 128 + (q & 7) * 16) =
                        make_uint4(0u, 0u, 0u, 0u);
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        return true;
    };
    // parts of K': the state of a whole stream leaves with this kernel, those of cut ones come from the state-only pass
    auto terms_of = [&]() { return STATES || walk.whole_stream() ? kTerms : kTermsInside; };

    if (warp < 4) {
        setmaxnreg_dec<kRegsIo>();
        if (warp == 0) {
            // ======================================= TMA producer ================================
            if (aligned_ok) {
                if (lane == 0) {
                    tma_prefetch_desc(&tmK);
                    tma_prefetch_desc(&tmV);
                    if (!STATES) tma_prefetch_desc(&tmQ);
                }
                Turn<C::KS> kat;
                Turn<C::VS> vat;
                uint32_t chunks = 0, k_armed = 0, v_armed = 0, q_armed = 0;
                bool ok = !p.selftest_skip_loads;
                while (ok && enter()) {
                    const int x = walk.h * D;
#pragma unroll 1
                    for (int c = walk.c; c < walk.c_end; ++c, ++chunks) {
                        const int y = tab.tok0[walk.b] + c * CT;
                        // in the order in which their places become free: V first half, K both, Q, V second half
#pragma unroll 1
                        for (int i = 0; i < (STATES ? 4 : 5); ++i) {
                            const bool is_q = !STATES && i == 3, is_k = i == 1 || i == 2;
                            const int half = i == 2 || i == (STATES ? 3 : 4);
                            const uint32_t at = is_q ? place<QS>(chunks) : is_k ? kat.at : vat.at;
                            const uint32_t round = is_q ? round_of<QS>(chunks) : is_k ? kat.round : vat.round;
                            uint64_t* full = (is_q ? q_full : is_k ? k_full : v_full) + at;
                            if (!(ok = wait((is_q ? q_empty : is_k ? k_empty : v_empty) + at, round ^ 1u, kWaitRingEmpty))) break;
                            if (lane == 0) {
                                const uint32_t off = is_q ? C::OFF_Q + at * C::TILE_BYTES : (is_k ? C::OFF_K : C::OFF_V) + at * C::KV_BYTES;
                                const CUtensorMap* tm = is_q ? &tmQ : is_k ? &tmK : &tmV;
                                mbar_expect_tx(full, is_q ? C::TILE_BYTES : C::KV_BYTES);
                                for (int hf = 0; hf < C::HALVES; ++hf)
                                    tma_load_2d(smem + off + hf * (is_q ? HALF_BYTES : SUB_BYTES), tm, x + hf * 64, y + half * HT, full);
                            }
                            __syncwarp();
                            if (is_q) ++q_armed;
                            else if (is_k) { kat.next(); ++k_armed; }
                            else { vat.next(); ++v_armed; }
                        }
                        if (!ok) break;
                        if (!STATES && p.base.norm.gate) {     // the gate's rows, into L2
                            const int len = tab.len[walk.b];
#pragma unroll 1
                            for (int r = lane; r < CT * C::HALVES; r += 32) {
                                const int t = c * CT + r / C::HALVES;
                                if (t < len)
                                    asm volatile("prefetch.global.L2 [%0];" ::"l"(p.base.norm.gate + (tab.tok0[walk.b] + (int64_t)t) * p.base.norm.gate_stride +
                                                                                  x + (r % C::HALVES) * 64));
                            }
                        }
                    }
                }
                // no copy may land after the CTA has ended (at once when all went well): the last ones into every place
                if (lane == 0) {
                    auto drain = [&](uint64_t* full, uint32_t places, uint32_t n) {
#pragma unroll 1
                        for (uint32_t k = n > places ? n - places : 0; k < n; ++k)
                            if (!drain_wait(full + k % places, (k / places) & 1u, ab)) return;
                    };
                    drain(v_full, C::VS, v_armed);
                    drain(k_full, C::KS, k_armed);
                    if (!STATES) drain(q_full, QS, q_armed);
                }
            }
        } else if (warp == 1) {
            // ======================================= issuer of Q S, Q K^T, P V ===================
            if (aligned_ok) {
                constexpr uint32_t idesc_qk = make_idesc(HT, false);
                constexpr uint32_t idesc_mn = make_idesc(D, true);              // B with its columns contiguous: V, S
                const uint64_t s_desc = make_desc(sbase + C::OFF_S, D * 128, 1024);
                Turn<C::KS> kat;
                Turn<C::VS> vat;
                uint32_t it = 0;
                bool ok = !STATES;
                while (ok && enter()) {
#pragma unroll 1
                    for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                        const uint32_t ph = it & 1u;
                        const uint32_t o_cols = tmem_base + COL_O + ph * 128;
                        const uint64_t q_desc = make_desc(sbase + C::OFF_Q + place<QS>(it) * C::TILE_BYTES, 16, 1024);
                        if (!(ok = wait(&q_full[place<QS>(it)], round_of<QS>(it), kWaitRingFull))) break;
#pragma unroll 1
                        for (int half = 0; half < 2; ++half) {
                            if (!(ok = wait(&k_full[kat.at], kat.round, kWaitRingFull))) break;
                            tc_fence_after();
                            const uint64_t k_desc = make_desc(sbase + C::OFF_K + kat.at * C::KV_BYTES, 16, 1024);
                            if (elect_one()) {
#pragma unroll
                                for (int ks = 0; ks < D / 16; ++ks)
                                    umma_ss(tmem_base + COL_SC + half * HT, q_desc + (((ks >> 2) * HALF_BYTES + (ks & 3) * 32) >> 4),
                                            k_desc + (((ks >> 2) * SUB_BYTES + (ks & 3) * 32) >> 4), idesc_qk, ks > 0 ? 1u : 0u);
                                umma_commit(&k_empty[kat.at]);
                                if (half) umma_commit(sc_full);
                            }
                            __syncwarp();
                            kat.next();
                        }
                        if (!ok) break;
                        if (!(ok = wait(s_full, ph, kWaitTensor))) break;
                        if (!(ok = wait(&o_empty[ph], ((it >> 1) & 1u) ^ 1u, kWaitTensor))) break;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks) {
                                const uint32_t off = (ks >> 2) * HALF_BYTES + (ks & 3) * 32;
                                umma_ss(o_cols, q_desc + (off >> 4), s_desc + ((ks * 16 * 128) >> 4), idesc_mn, ks > 0 ? 1u : 0u);
                            }
                            umma_commit(qs_full);
                            umma_commit(s_empty);
                            umma_commit(&q_empty[place<QS>(it)]);
                        }
                        __syncwarp();
                        // P V, on top of Q S
                        if (!(ok = wait(p_full, ph, kWaitTensor))) break;
#pragma unroll 1
                        for (int half = 0; half < 2; ++half) {
                            if (!(ok = wait(&v_full[vat.at], vat.round, kWaitRingFull))) break;
                            tc_fence_after();
                            const uint64_t v_desc = make_desc(sbase + C::OFF_V + vat.at * C::KV_BYTES, SUB_BYTES, 1024);
                            if (elect_one()) {
#pragma unroll
                                for (int ks = 0; ks < HT / 16; ++ks)
                                    umma_ts(o_cols, tmem_base + COL_SC + half * (HT / 2) + ks * 8, v_desc + ((ks * 16 * 128) >> 4), idesc_mn, 1u);
                                umma_commit(&v_empty[vat.at]);
                                if (half) umma_commit(&o_full[ph]);
                            }
                            __syncwarp();
                            vat.next();
                        }
                        if (!ok) break;
                    }
                }
                // nothing issued may still run when tensor memory is released
                if (elect_one()) {
                    umma_commit(&drain_bar[0]);
                    drain_wait(&drain_bar[0], 0u, ab);
                }
                __syncwarp();
            }
        } else if (warp == 3) {
            // ======================================= issuer of K'^T V ============================
            if (aligned_ok) {
                constexpr uint32_t idesc_kv = make_idesc(D, true) | (STATES ? 0u : 1u << 15);    // K' from shared memory: its columns are contiguous too
                Turn<C::VS> vat;
                uint32_t it = 0;
                bool ok = true;
                while (ok && enter()) {
                    const int terms = terms_of();
                    pieces.segment(terms);
#pragma unroll 1
                    for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                        const uint32_t buf = STATES ? it & 1u : 0u, round = STATES ? (it >> 1) & 1u : it & 1u;
                        const uint32_t d_cols = tmem_base + (buf ? COL_SC : COL_DS);
                        if (!(ok = wait(&ds_empty[buf], round ^ 1u, kWaitTensor))) break;
#pragma unroll 1
                        for (int e = 0; e < PIECES; ++e) {
                            if ((e & 1) == 0 && !(ok = wait(&v_full[vat.at], vat.round, kWaitRingFull))) break;
                            if (!(ok = wait(&kp_full[pieces.at], pieces.parity(pieces.at), kWaitTensor))) break;
                            tc_fence_after();
                            const uint64_t kp_desc = make_desc(sbase + pieces.offset(), PIECE_HALF, 1024);
                            const uint64_t vp_desc = make_desc(sbase + C::OFF_V + vat.at * C::KV_BYTES + (e & 1) * (PIECE * 128), SUB_BYTES, 1024);
                            if (elect_one()) {
#pragma unroll
                                for (int t = 0; t < kTerms; ++t) {
                                    if (t >= kTermsInside && t >= terms) break;
#pragma unroll
                                    for (int ks = 0; ks < PIECE / 16; ++ks) {
                                        const uint32_t more = t > 0 || ks > 0 ? 1u : e > 0 ? 1u : 0u;
                                        if (STATES)
                                            umma_ts(d_cols, tmem_base + COL_KP + (pieces.at * kTerms + t) * KP_COLS + ks * 8, vp_desc + ((ks * 2048) >> 4),
                                                    idesc_kv, more);
                                        else
                                            umma_ss(d_cols, kp_desc + ((t * TERM_BYTES + ks * 2048) >> 4), vp_desc + ((ks * 2048) >> 4), idesc_kv, more);
                                    }
                                }
                                umma_commit(&kp_empty[pieces.at]);
                                if (e & 1) umma_commit(&v_empty[vat.at]);
                                if (e == PIECES - 1) umma_commit(&ds_full[buf]);
                            }
                            __syncwarp();
                            pieces.next();
                            if (e & 1) vat.next();
                        }
                        if (!ok) break;
                    }
                }
                if (elect_one()) {
                    umma_commit(&drain_bar[1]);
                    drain_wait(&drain_bar[1], 0u, ab);
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
                // a lane has four neighbouring tokens; those of the next chunk are asked for a chunk ahead
                auto read = [&](int t0, float (&z)[4]) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) z[j] = t0 + j < len ? read_decay(p.base, tok0 + t0 + j, walk.h) : 0.f;
                };
                float z[4];
                read(walk.c * CT + lane * 4, z);
#pragma unroll 1
                for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                    const int t0 = c * CT + lane * 4;
                    double s[4], sum = 0.0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const double l = (double)log_decay(p.base, z[j]) * 1.4426950408889634;
                        s[j] = sum += t0 + j < len ? l : 0.0;
                    }
                    read(t0 + CT, z);                      // (behind the segment: read for nothing)
                    double before = sum;
#pragma unroll 1
                    for (int m = 1; m < 32; m <<= 1) {
                        const double o = __shfl_up_sync(0xffffffffu, before, m);
                        if (lane >= m) before += o;
                    }
                    const double block_end = __shfl_sync(0xffffffffu, before, lane | 7), chunk_end = __shfl_sync(0xffffffffu, before, 31);
                    before -= sum;
                    const uint32_t buf = it & 1u;
                    if (!(ok = wait(&dec_empty[buf], ((it >> 1) & 1u) ^ 1u, kWaitTensor))) break;
                    float* dst = dec + buf * C::DEC_FLOATS + lane * 4;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const double x = before + s[j];
                        dst[j] = ex2_approx((float)(chunk_end - x));
                        if (!STATES) {
                            const double r = rint(x);
                            dst[C::DEC_WHOLE + j] = (float)-r;
                            dst[C::DEC_REST + j] = (float)(r - x);
                            dst[C::DEC_U + j] = ex2_approx((float)(block_end - x));
                        }
                    }
                    if (lane == 0) {
                        const double r = rint(chunk_end);
                        dst[C::DEC_END] = (float)r;
                        dst[C::DEC_END + 1] = (float)(chunk_end - r);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&dec_full[buf]);
                }
            }
        }
    } else if (warp >= 24 || (STATES && warp < 12)) {
        // ======================================= K' ==============================================
        // 256 threads make a piece together; in the state-only pass four warpgroups make one of a chunk's pieces each, always in the same place, and
        // wait for no other's: a team has seen the use before the last one of its place given back.
        setmaxnreg_dec<STATES ? kRegsAcross : kRegsKeys>();
        constexpr int TEAM = STATES ? 128 : 256;
        constexpr uint32_t TEAMS = STATES ? 4 : 1;
        const uint32_t team = !STATES ? 0u : warp < 12 ? (uint32_t)(warp >> 2) - 1u : (uint32_t)(warp >> 2) - 4u;
        const int tid = threadIdx.x & (TEAM - 1);
        Turn<C::KS> kat;
        Turn<C::VS> vat;
        uint32_t it = 0, tails = 0;
        bool ok = aligned_ok;
        while (ok && enter()) {
            const int len = tab.len[walk.b], terms = terms_of();
            if (!STATES && !(ok = all_given_back())) break;
            pieces.segment(terms);
#pragma unroll 1
            for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                const uint32_t buf = it & 1u;
                const int valid = len - c * CT;            // tokens of the sequence from here on
                if (!(ok = wait(&dec_full[buf], (it >> 1) & 1u, kWaitTensor))) break;
                if (valid < CT && team == 0) {             // (this team makes piece 0)
                    if (!(ok = clear_tail(TEAM, tid, vat, valid))) break;
                    if (!STATES && lane == 0) mbar_arrive(&v_cleared[tails & 1u]);
                    ++tails;
                }
#pragma unroll 1
                for (int e = 0; e < PIECES; ++e) {
                    if (TEAMS == 1 || (uint32_t)e == team) {
                        if ((TEAMS > 1 || !(e & 1)) && !(ok = wait(&k_full[kat.at], kat.round, kWaitRingFull))) break;
                        if (!(ok = wait(&kp_empty[pieces.at], pieces.parity(pieces.at) ^ 1u, kWaitTensor))) break;
                        if (STATES)
                            make_piece_across(kat.at, e, dec + buf * C::DEC_FLOATS, valid);
                        else
                            make_piece(tid, kat.at, e, dec + buf * C::DEC_FLOATS, valid, terms);
                        if (lane == 0 && (TEAMS > 1 || (e & 1))) mbar_arrive(&k_empty[kat.at]);
                    }
                    pieces.next();
                    if (e & 1) {
                        kat.next();
                        vat.next();
                    }
                }
                if (!ok) break;
                __syncwarp();
                if (lane == 0) mbar_arrive(&dec_empty[buf]);
            }
        }
    } else if (warp < 8) {
        // ======================================= P ===============================================
        setmaxnreg_dec<kRegsP>();
        const int quad = warp & 3, i = quad * 32 + lane;
        const uint32_t sc = tmem_base + COL_SC + ((uint32_t)(quad * 32) << 16);
        uint32_t it = 0, tails = 0;
        bool ok = aligned_ok && !STATES;
        while (ok && enter()) {
            const int len = tab.len[walk.b];
#pragma unroll 1
            for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                const uint32_t buf = it & 1u, ph = it & 1u;
                if (!(ok = wait(&dec_full[buf], (it >> 1) & 1u, kWaitTensor))) break;
                const float* whole = dec + buf * C::DEC_FLOATS + C::DEC_WHOLE;   // negated
                const float* rest = whole + CT;
                const float wi = -whole[i], ri = -rest[i];
                if (!(ok = wait(sc_full, ph, kWaitTensor))) break;
                tc_fence_after();
                uint32_t w[8];
                float s[16];
#pragma unroll 1
                for (int blk = 0; blk < 2 * quad; ++blk) {         // 16 columns below the diagonal
                    tmem_ld16(sc + blk * 16, s);
                    const int m = blk * 16 | 31;
                    const float r = ex2_approx((wi + whole[m]) + (ri + rest[m]));
                    const uint64_t r2 = f2_pack(r, r);
                    const ulonglong2* u = reinterpret_cast<const ulonglong2*>(whole + 2 * CT + blk * 16);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const ulonglong2 uj = u[j / 4];
                        float x[4];
                        f2_unpack(f2_mul(f2_mul(f2_pack(s[j], s[j + 1]), r2), uj.x), x[0], x[1]);
                        f2_unpack(f2_mul(f2_mul(f2_pack(s[j + 2], s[j + 3]), r2), uj.y), x[2], x[3]);
                        w[j / 2] = pack_bf16x2(x[0], x[1]);
                        w[j / 2 + 1] = pack_bf16x2(x[2], x[3]);
                    }
                    tmem_st8(sc + blk * 8, w);             // (over columns that have been read)
                }
                const uint64_t wi2 = f2_pack(wi, wi), ri2 = f2_pack(ri, ri);
#pragma unroll 1
                for (int blk = 2 * quad; blk < 2 * quad + 2; ++blk) {
                    tmem_ld16(sc + blk * 16, s);
                    const int last = i - blk * 16;         // the row's last column here
                    const ulonglong2* wj = reinterpret_cast<const ulonglong2*>(whole + blk * 16);
                    const ulonglong2* rj = reinterpret_cast<const ulonglong2*>(rest + blk * 16);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const ulonglong2 wq = wj[j / 4], rq = rj[j / 4];
                        float x[4];
                        f2_unpack(f2_add(f2_add(wi2, wq.x), f2_add(ri2, rq.x)), x[0], x[1]);
                        f2_unpack(f2_add(f2_add(wi2, wq.y), f2_add(ri2, rq.y)), x[2], x[3]);
#pragma unroll
                        for (int q = 0; q < 4; ++q) x[q] = j + q <= last ? s[j + q] * ex2_approx(x[q]) : 0.f;
                        w[j / 2] = pack_bf16x2(x[0], x[1]);
                        w[j / 2 + 1] = pack_bf16x2(x[2], x[3]);
                    }
                    tmem_st8(sc + blk * 8, w);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 0u;
#pragma unroll 1
                for (int blk = 2 * quad + 2; blk < 8; ++blk) tmem_st8(sc + blk * 8, w);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&dec_empty[buf]);
                // V's rows behind the sequence have been cleared (of the two barriers' next uses the later one comes behind this chunk's P V)
                if (len - c * CT < CT) {
                    if (!(ok = wait(&v_cleared[tails & 1u], (tails >> 1) & 1u, kWaitTensor))) break;
                    ++tails;
                }
                if (lane == 0) mbar_arrive(p_full);
            }
        }
    } else if (warp < 12 || warp >= 20) {
        // ======================================= output ==========================================
        if constexpr (STATES) setmaxnreg_dec<kRegsIdle>(); else setmaxnreg_inc<kRegsOut>();
        const int quad = warp & 3;
        const uint32_t mine = warp < 12 ? 0u : 1u;             // chunks of this warpgroup: even, odd
        const uint32_t o = tmem_base + COL_O + mine * 128 + ((uint32_t)(quad * 32) << 16);
        const NormGate& nm = p.base.norm;
        const float scale = p.base.scale;
        // A thread's row comes and goes 16 channels at a time: 32 bytes, a whole sector, in one access where rows start on 32 bytes.  (Through
        // shared memory, eight rows to an access, was slower: the operands of the matrix products keep that busy.  One / four sequences
        // of 4,096 tokens, 32 / 37 heads: 76.5 / 149 us against 74.1 / 140, with gate 92.7 / 204 against 85.6 / 182.)
        const bool wide_out = (((uintptr_t)p.base.o | (uintptr_t)(p.base.o_stride * 2)) & 31) == 0;
        const bool wide_gate = (((uintptr_t)nm.gate | (uintptr_t)(nm.gate_stride * 2)) & 31) == 0;
        uint32_t it = 0;
        bool ok = aligned_ok && !STATES;
        while (ok && enter()) {
            const int len = tab.len[walk.b], at = walk.h * D;
            const int64_t tok0 = tab.tok0[walk.b];
#pragma unroll 1
            for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                if ((it & 1u) != mine) continue;
                const bool live = c * CT + quad * 32 + lane < len;
                const int64_t token = tok0 + c * CT + quad * 32 + lane;
                __nv_bfloat16* out = p.base.o + token * p.base.o_stride + at;
                const __nv_bfloat16* gate = nm.gate + token * nm.gate_stride + at;
                uint32_t g[8] = {};                            // the gate's next 16 channels
                auto ask = [&](int j) {
                    if (live) load_row16(gate + j, wide_gate, g);
                };
                if (nm.gate) ask(0);
                if (!(ok = wait(&o_full[mine], (it >> 1) & 1u, kWaitTensor))) break;
                tc_fence_after();
                // 16 channels of the row: a * x + add; the ones at `next` are on their way from then on
                float x[16];
                auto channels = [&](int next, float a, float add, uint64_t (&y)[8]) {
                    const uint64_t a2 = f2_pack(a, a), add2 = f2_pack(add, add);
                    tmem_wait_ld();
#pragma unroll
                    for (int q = 0; q < 8; ++q) y[q] = f2_fma(a2, f2_pack(x[2 * q], x[2 * q + 1]), add2);
                    if (next < D) tmem_ld16(o + next, x);
                };
                tmem_ld16(o, x);
                float of = scale, add = 0.f;
                if (nm.on) {
                    // sums of the differences from the row's first channel (rms: from zero) and of their squares: one of d values is at most
                    // sqrt(d) standard deviations from the mean, so the difference of the two loses at most d roundings
                    tmem_wait_ld();
                    const float first = nm.rms ? 0.f : x[0] * scale;
                    uint64_t s1 = 0ull, s2 = 0ull;
#pragma unroll 1
                    for (int j = 0; j < D; j += 16) {
                        uint64_t y[8];
                        channels((j + 16) % D, scale, -first, y);
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            s1 = f2_add(s1, y[q]);
                            s2 = f2_fma(y[q], y[q], s2);
                        }
                    }
                    float a0, a1, b0, b1;
                    f2_unpack(s1, a0, a1);
                    f2_unpack(s2, b0, b1);
                    const float m1 = nm.rms ? 0.f : (a0 + a1) * (1.f / D);
                    const float inv = 1.f / sqrtf(fmaxf(fmaf(-m1, m1, (b0 + b1) * (1.f / D)), 0.f) + nm.eps);
                    of = scale * inv;
                    add = -(first + m1) * inv;
                }
#pragma unroll 1
                for (int j = 0; j < D; j += 16) {
                    uint64_t y[8];
                    channels(j + 16, of, add, y);
                    if (j + 16 == D) {                     // all of it has been read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&o_empty[mine]);
                    }
                    if (nm.on) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {          // eight channels
                            uint64_t f[4];
                            auto eight = [&](const uint4& v) {
                                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                                for (int q = 0; q < 4; ++q) f[q] = f2_pack(__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xFFFF0000u));
                            };
                            if (nm.gain) {
                                eight(__ldg(reinterpret_cast<const uint4*>(nm.gain + at + j) + e));
#pragma unroll
                                for (int q = 0; q < 4; ++q) y[4 * e + q] = f2_mul(y[4 * e + q], f[q]);
                            }
                            if (nm.bias) {
                                eight(__ldg(reinterpret_cast<const uint4*>(nm.bias + at + j) + e));
#pragma unroll
                                for (int q = 0; q < 4; ++q) y[4 * e + q] = f2_add(y[4 * e + q], f[q]);
                            }
                            if (nm.gate) {
                                eight(make_uint4(g[4 * e], g[4 * e + 1], g[4 * e + 2], g[4 * e + 3]));
#pragma unroll
                                for (int q = 0; q < 4; ++q) y[4 * e + q] = f2_swish_mul(f[q], y[4 * e + q]);
                            }
                        }
                    }
                    if (nm.gate && j + 16 < D) ask(j + 16);
                    uint32_t w[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        float y0, y1;
                        f2_unpack(y[q], y0, y1);
                        w[q] = pack_bf16x2(y0, y1);
                    }
                    if (live) store_row16(out + j, wide_out, w);
                }
            }
        }
    } else {
        // ======================================= state ===========================================
        setmaxnreg_inc<kRegsState>();
        constexpr int N = D * D / 256;                     // channels of a thread: half a row of the state (d = 64: a quarter)
        const int quad = warp & 3, l = quad * 32 + lane, row = l % D, col = (warp >= 16 ? D / 2 : 0) + (l / D) * N;
        uint8_t* s_row = smem + C::OFF_S + row * 128;
        // A warp's part of the state is 32 rows of N channels, a row a lane.  On the way from and to memory it goes through the warp's share of the place
        // of S, SL channels at a time, so that an access covers whole sectors of few rows (a lane's own row: 32 lines an access).
        constexpr int SL = D == 128 ? 16 : 8, CH = SL / 4;
        uint8_t* stage = smem + C::OFF_S + (warp - 12) * (32 * SL * 4);
        const int row0 = row - lane;
        auto through_rows = [&](auto&& by_lines, auto&& by_rows, bool rows_first) {
            auto at = [&](int r, int ch) { return reinterpret_cast<uint4*>(stage + r * (SL * 4) + ((ch ^ ((CH == 4 ? r >> 1 : r >> 2) & (CH - 1))) << 4)); };
#pragma unroll
            for (int j = 0; j < N; j += SL) {
                auto rows = [&]() {
#pragma unroll
                    for (int ch = 0; ch < CH; ++ch) by_rows(j, ch, at(lane, ch));
                };
                if (rows_first) rows();
                if (rows_first) __syncwarp();
#pragma unroll
                for (int i = 0; i < CH; ++i) by_lines(col + j, row0 + (i * 32 + lane) / CH, lane % CH, at((i * 32 + lane) / CH, lane % CH));
                __syncwarp();
                if (!rows_first) rows();
                if (!rows_first) __syncwarp();
            }
        };
        uint32_t it = 0, segments = 0;
        bool ok = aligned_ok;
        if (!STATES) asm volatile("griddepcontrol.wait;" ::: "memory");       // (the merge: nothing else here reads what it wrote)
        while (ok && enter()) {
            const int b = walk.b, h = walk.h;
            const bool whole_stream = walk.whole_stream();
            float s[N];
            // where the segment's first state is: the stream's own, or what the merge left for this CTA
            const float* src = nullptr;
            if (!STATES) {
                if (whole_stream)
                    src = tab.from[b] >= 0 ? p.base.state + ((int64_t)tab.from[b] * p.base.H + h) * (D * D) : nullptr;
                else
                    src = p.part + (int64_t)(walk.c > 0 ? blockIdx.x : p.groups + blockIdx.x) * (D * D);
            }
            if (STATES || !src) {
#pragma unroll
                for (int j = 0; j < N; ++j) s[j] = 0.f;
            } else {
                through_rows([&](int j, int r, int ch, uint4* place) { *place = *reinterpret_cast<const uint4*>(src + r * D + j + ch * 4); },
                             [&](int j, int ch, uint4* place) {
                                 const float4 x = *reinterpret_cast<const float4*>(place);
                                 s[j + ch * 4] = x.x;
                                 s[j + ch * 4 + 1] = x.y;
                                 s[j + ch * 4 + 2] = x.z;
                                 s[j + ch * 4 + 3] = x.w;
                             }, false);
            }
            if (!STATES) {       // S takes the place of the rows that all eight warps have come through
                __syncwarp();
                if (lane == 0) mbar_arrive(s_staged);
                if (!(ok = wait(s_staged, segments & 1u, kWaitTensor))) break;
                ++segments;
            }
            float all_whole = 0.f, all_rest = 0.f;         // logarithm of the segment's decay
#pragma unroll 1
            for (int c = walk.c; c < walk.c_end; ++c, ++it) {
                const uint32_t buf = it & 1u, ph = it & 1u;
                if (!STATES) {
                    // ---- S in bf16
                    if (!(ok = wait(s_empty, ph ^ 1u, kWaitTensor))) break;
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
                if (!(ok = wait(&dec_full[buf], (it >> 1) & 1u, kWaitTensor))) break;
                const float whole = dec[buf * C::DEC_FLOATS + C::DEC_END], rest = dec[buf * C::DEC_FLOATS + C::DEC_END + 1];
                const float ei = STATES ? 0.f : exp2_parts(-dec[buf * C::DEC_FLOATS + C::DEC_WHOLE + l], -dec[buf * C::DEC_FLOATS + C::DEC_REST + l]);
                __syncwarp();
                if (lane == 0) mbar_arrive(&dec_empty[buf]);
                // ---- S'
                const float keep = exp2_parts(whole, rest);
                const uint64_t keep2 = f2_pack(keep, keep);
                if (STATES) {
                    all_whole += whole;
                    all_rest += rest;
                }
                if (!STATES) {
                    // ---- 2^b_i q_i S, in place: this thread's token, half of the channels
                    if (!(ok = wait(qs_full, ph, kWaitTensor))) break;
                    tc_fence_after();
                    const uint32_t o = tmem_base + COL_O + ph * 128 + ((uint32_t)(quad * 32) << 16) + (warp >= 16 ? D / 2 : 0);
                    const uint64_t ei2 = f2_pack(ei, ei);
#pragma unroll 1
                    for (int j = 0; j < D / 2; j += 16) {
                        float x[16];
                        tmem_ld16(o + j, x);
                        tmem_wait_ld();
#pragma unroll
                        for (int q = 0; q < 16; q += 2) f2_unpack(f2_mul(ei2, f2_pack(x[q], x[q + 1])), x[q], x[q + 1]);
                        tmem_st16(o + j, *reinterpret_cast<uint32_t(*)[16]>(&x));
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full);
                }
                const uint32_t ds_buf = STATES ? it & 1u : 0u;
                if (!(ok = wait(&ds_full[ds_buf], STATES ? (it >> 1) & 1u : ph, kWaitTensor))) break;
                tc_fence_after();
                const uint32_t ds = tmem_base + (ds_buf ? COL_SC : COL_DS) + ((uint32_t)(quad * 32) << 16) + col;
#pragma unroll
                for (int blk = 0; blk < N / 16; ++blk) {
                    float x[16];
                    tmem_ld16(ds + blk * 16, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; j += 2)
                        f2_unpack(f2_fma(keep2, f2_pack(s[blk * 16 + j], s[blk * 16 + j + 1]), f2_pack(x[j], x[j + 1])), s[blk * 16 + j], s[blk * 16 + j + 1]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ds_empty[ds_buf]);
            }
            if (!ok) break;
            // a state-only segment that ends inside its stream: the next CTA's start; one that ends it: the last part of the final state
            const int64_t slot = walk.c_end < walk.chunks ? blockIdx.x + 1 : 2 * (int64_t)p.groups + blockIdx.x;
            float* dst = nullptr;
            if (STATES)
                dst = p.part + slot * (D * D);
            else if (whole_stream && tab.to[b] >= 0)
                dst = p.base.state + ((int64_t)tab.to[b] * p.base.H + h) * (D * D);
            if (dst) {
                through_rows([&](int j, int r, int ch, uint4* place) { *reinterpret_cast<uint4*>(dst + r * D + j + ch * 4) = *place; },
                             [&](int j, int ch, uint4* place) {
                                 *reinterpret_cast<float4*>(place) = make_float4(s[j + ch * 4], s[j + ch * 4 + 1], s[j + ch * 4 + 2], s[j + ch * 4 + 3]);
                             }, true);
            }
            if (STATES && threadIdx.x == 12 * 32) p.part_keep[slot] = exp2_parts(all_whole, all_rest);
        }
    }

    if (wait.what != 0 && lane == 0) report_give_up(ab, wait.what);
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// States of the streams that several CTAs share.  A block owns some elements of one such stream: from the stream's first state on, every
// CTA's part (its local state, from zero) is added to what decays from before, in the order of the CTAs.  Slot g: the state that CTA g
// starts from (the state-only pass left CTA g - 1's part there); slot groups + g: a copy of the first state of the stream
// that begins in CTA g (the pool's is overwritten here, if it is the slot the stream ends in); slot 2 groups + g: CTA g's part of a stream that ends in it.
constexpr int kMergeThreads = 256;
template <int D, class Table>
__global__ void __launch_bounds__(kMergeThreads)
gret_merge_kernel(const GretChunkParams p, const __grid_constant__ Table tab) {
    asm volatile("griddepcontrol.launch_dependents;");
    const int g0 = blockIdx.x + 1;                         // first CTA that starts inside the stream
    const int H = p.base.H, pos = p.first_of(g0), b = sequence_at(p, tab, pos);
    const int base = tab.chunk0[b] * H, chunks = tab.chunk0[b + 1] - tab.chunk0[b], h = (pos - base) / chunks;
    const int begin = base + h * chunks, end = begin + chunks;
    if (pos == begin || p.first_of(g0 - 1) > begin) return;        // no cut, or not the stream's first one
    const int at = (blockIdx.y * kMergeThreads + threadIdx.x) * 4;
    auto part = [&](int64_t slot) { return reinterpret_cast<float4*>(p.part + slot * (D * D) + at); };
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tab.from[b] >= 0) s = *reinterpret_cast<const float4*>(p.base.state + ((int64_t)tab.from[b] * H + h) * (D * D) + at);
    // the parts are asked for kAhead at a time: one at a time, each behind the store of the one before, every CTA of the stream would cost a
    // way to memory and back
    constexpr int kAhead = 8;
    bool first = true;
    for (int g = g0;; g += kAhead) {
        float4 x[kAhead];
        float keep[kAhead];
        int n = 0;                                         // CTAs that start inside the stream, of these
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (n < i) continue;
            const bool inside = g + i < p.groups && p.first_of(g + i) < end;
            const int64_t slot = inside ? g + i : 2 * (int64_t)p.groups + g + i - 1;
            x[i] = *part(slot);
            keep[i] = p.part_keep[slot];
            if (inside) ++n;
        }
        if (first) *part(p.groups + g0 - 1) = s;
        first = false;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (n < i) continue;
            s = make_float4(fmaf(keep[i], s.x, x[i].x), fmaf(keep[i], s.y, x[i].y), fmaf(keep[i], s.z, x[i].z), fmaf(keep[i], s.w, x[i].w));
            if (i < n) *part(g + i) = s;
        }
        if (n < kAhead) break;
    }
    if (tab.to[b] >= 0) *reinterpret_cast<float4*>(p.base.state + ((int64_t)tab.to[b] * H + h) * (D * D) + at) = s;
}

// The three kernels of cut streams follow one another with programmatic stream serialisation: each may be launched while the one before it
// ends, and waits for it before it reads what that one wrote.
template <class... Params, class... Args>
cudaError_t launch_behind(bool early, void (*kernel)(Params...), dim3 grid, int threads, int smem, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D, class Table>
cudaError_t launch_one(const GretChunkParams& p, const Table& tab, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                       cudaStream_t stream) {
    if (p.split) {
        cudaError_t e = launch_behind(false, gret_chunk_kernel<D, true, Table>, dim3(p.groups), kThreads, GCfg<D, true>::SMEM_BYTES, stream, tmQ, tmK,
                                      tmV, p, tab);
        if (e != cudaSuccess) return e;
        e = launch_behind(true, gret_merge_kernel<D, Table>, dim3(p.groups - 1, D * D / (4 * kMergeThreads)), kMergeThreads, 0, stream, p, tab);
        if (e != cudaSuccess) return e;
    }
    return launch_behind(p.split, gret_chunk_kernel<D, false, Table>, dim3(p.groups), kThreads, GCfg<D, false>::SMEM_BYTES, stream, tmQ, tmK, tmV, p,
                         tab);
}

template <int D, bool STATES>
cudaError_t setup_pass() {
    constexpr int bytes = GCfg<D, STATES>::SMEM_BYTES;
    cudaError_t e = cudaFuncSetAttribute(gret_chunk_kernel<D, STATES, GretChunkTable>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(gret_chunk_kernel<D, STATES, GretChunkTableOf<kFewSequences>>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

}  // namespace

cudaError_t gret_chunk_kernel_setup() {
    cudaError_t e = setup_pass<128, false>();
    if (e != cudaSuccess) return e;
    if ((e = setup_pass<128, true>()) != cudaSuccess) return e;
    if ((e = setup_pass<64, false>()) != cudaSuccess) return e;
    return setup_pass<64, true>();
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
