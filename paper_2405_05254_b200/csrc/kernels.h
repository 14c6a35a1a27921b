// Launch interfaces of the kernels (device code lives in the *_kernel.cu files).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "plan.h"

namespace yoco {

constexpr int32_t kStatusOk = 0;
// Status word (first int32 of a workspace, or the append kernel's own word): 0 = ok, otherwise
//   bits 0-7   which kind of wait ran out (WaitClass)
//   bits 8-31  1 + linear index of the CTA that gave up first
// The first failure wins (compare-and-swap against 0), so the word names where the trouble began.
enum WaitClass : int32_t {
    kWaitItemQueue = 1,   // decode: next work item from the producer / queue entry read by the consumers
    kWaitRingFull = 2,    // a consumer waiting for a K/V (or Q, X, W) tile to land
    kWaitRingEmpty = 3,   // the producer waiting for a stage to be released
    kWaitTensor = 4,      // a tensor-core hand-over: scores ready, P written, product finished
    kWaitDrain = 5,       // leaving: a copy or product that had been started did not finish in time
    kWaitMisaligned = 6,  // dynamic shared memory not 1 KB aligned (no wait involved; nothing ran)
    kBadPage = 7,         // a page table entry outside the pool (no wait involved; its rows read as zeros / are not written)
};
__host__ __device__ constexpr int32_t status_word(int32_t wait_class, int32_t cta) {
    return wait_class | ((cta + 1) << 8);
}


// Work tables small enough to travel as kernel parameters (the decode call then needs no
// host-to-device copy): every benchmark shape fits; larger problems read them from the workspace.
constexpr int kInlineSegments = 448;
constexpr int kInlineGroups = 303;
constexpr int kInlineStreams = 256;
struct DecodeInlineTables {
    DevSegment seg[kInlineSegments];
    int32_t group_begin[kInlineGroups + 1];
};
struct CombineInlineTables {
    int32_t stream_base[kInlineStreams];
    int32_t stream_nseg[kInlineStreams];
};

struct CombineParams {
    int64_t rows;               // output rows (B*Hq*T, or the public `rows`)
    int32_t d;
    // public layout ([rows][S][d]) when stream_base == nullptr
    int32_t S;
    // internal slot-major layout
    int32_t Hq, Hkv, T, rows_per_stream;
    int32_t max_pieces;         // most pieces any row has (S, or the plan's max_splits): picks the launch shape
    int32_t sub_items;          // internal layout: slots per table entry (0 or 1: one)
    const int32_t* stream_base; // [B*Hkv] first slot of each stream
    const int32_t* stream_nseg; // [B*Hkv] slots of each stream
    const float* part_o;
    const float* part_lse;      // natural log, -inf = empty
    __nv_bfloat16* O;           // [rows, d] bf16 result, or null when O_f32 is given
    float* lse;                 // may be null
    float* O_f32;               // [rows, d] fp32 result instead of O (a partial result that another
                                // merge will consume: key-range sharding across GPUs)
    int32_t merge_unsplit;      // internal layout: also copy rows whose stream has a single piece
                                // (set when the attention kernel was told to write no final rows)
    int32_t piece_major;        // public layout is [S][rows][d] / [S][rows] (as an all-gather over S
                                // ranks leaves it) instead of [rows][S][d] / [rows][S]
};
// inline_tab (host, may be null): stream tables passed as kernel parameters instead of
// p.stream_base / p.stream_nseg.  after_attention: launched right behind the attention kernel of
// the same call; the launch is then allowed to overlap that kernel's tail (the merge itself still
// waits for it).  warp_per_many_rows: see kManyRows (combine_kernel.cu).
cudaError_t launch_combine(const CombineParams& p, cudaStream_t stream,
                           const CombineInlineTables* inline_tab = nullptr, bool after_attention = false,
                           bool warp_per_many_rows = false);

// Where the rows of a paged cache are: row(page, head c, slot) = page * page_rows + c * P + slot, P = 1 << page_shift.
struct PageMap {
    const int32_t* table;       // device [B, table_stride]: page that holds keys [j P, (j + 1) P) of sequence b
    int32_t table_stride;
    int32_t page_shift;
    int32_t num_pages;
    int32_t page_rows;
    int32_t Hkv;
    int32_t rows;               // rows of the pool: a row number no load can reach
};

struct DecodeParams {
    const __nv_bfloat16* Q;     // [B*Hq*T, d]
    __nv_bfloat16* O;           // [B*Hq*T, d]
    float* lse;                 // [B*Hq*T] or null
    const DevSegment* segments;
    const int32_t* group_begin; // [num_groups + 1]
    float* part_o;              // [num_segments][rows_per_stream][d]
    float* part_lse;            // [num_segments][rows_per_stream]
    int32_t* status;
    float scale_log2;           // scale * log2(e)
    int32_t T;
    int32_t rows_per_stream;    // G * T (<= 16)
    int32_t d;
    int32_t window;             // sliding window C, 0 = none
    int32_t force_partial;      // write every segment to its partial slot, even of an unsplit stream
    int32_t sub_items;          // pieces per group (plan.h: sub_bound); slot = segment slot * sub_items + piece
    int32_t* work_counter;      // zeroed before the launch; hands out the pieces beyond each CTA's first
    int64_t wait_limit_ns;      // 0 = the default limit of a bounded wait
    int32_t selftest_skip_loads;// self-test of the give-up path: the producer arms no copy, so the first
                                // consumer wait runs out (with nothing in flight) and the kernel returns
    PageMap pages;              // paged cache only
};
// tmK / tmV: 2-D tensor maps over the [rows, d] view of K and V, box {64, kDecodeTileN},
// 128-byte swizzle.
// inline_tab (host, may be null): segments and group offsets passed as kernel parameters instead
// of p.segments / p.group_begin.
// paged: rows are found through p.pages; the maps' boxes are {64, min(P, kDecodeTileN)}.
cudaError_t launch_decode(const DecodeParams& p, const CUtensorMap& tmK, const CUtensorMap& tmV,
                          int num_groups, cudaStream_t stream, const DecodeInlineTables* inline_tab = nullptr,
                          bool paged = false);
// one-time per-device kernel attribute set-up (dynamic shared memory opt-in)
cudaError_t decode_kernel_setup();


// ---- decode over an 8-bit (FP8 E4M3) cache, head dimension 128 ---------------------------------
constexpr int kFp8MaxHeads = 64;
struct DecodeFp8Params {
    DecodeParams base;                    // as for the bf16 kernel; base.scale_log2 is unused
    int32_t Hkv;
    float score_scale_log2[kFp8MaxHeads]; // per KV head: softmax scale * k_scale[c] * log2(e)
    float v_scale[kFp8MaxHeads];          // per KV head
};
// tmK / tmV: 2-D uint8 tensor maps over the [rows, 128] byte view of K and V, box {128, 64},
// 128-byte swizzle.
cudaError_t launch_decode_fp8(const DecodeFp8Params& p, const CUtensorMap& tmK, const CUtensorMap& tmV,
                              int num_groups, cudaStream_t stream, const DecodeInlineTables* inline_tab);
cudaError_t decode_fp8_kernel_setup();

// ---- decode over a paged 4-bit cache, head dimension 128 ---------------------------------------
// k / v: uint8 maps over the codes as [rows / 2, 128] bytes (two keys to a line), box {128, box / 2}, 128-byte swizzle
// (a copy moves a line of up to 128 bytes as fast as one of 64); k_scale / v_scale: uint8
// maps over the scales as [rows / 16, 128], box {128, box / 16}, no swizzle (box = min(P, the kernel's tile)).
struct PagedQ4Maps {
    CUtensorMap k, k_scale, v, v_scale;
};
cudaError_t launch_decode_q4(const DecodeParams& p, const PagedQ4Maps& maps, int num_groups, cudaStream_t stream,
                             const DecodeInlineTables* inline_tab);
cudaError_t decode_q4_kernel_setup();

struct ChunkParams {
    __nv_bfloat16* O;           // [B*Hq*T, d]
    float* lse;                 // [B*Hq*T] or null
    const DevSegment* segments;
    const int32_t* group_begin; // [num_groups + 1]
    float* part_o;              // [num_segments][rows_per_stream][d]
    float* part_lse;            // [num_segments][rows_per_stream]
    int32_t* status;
    float scale_log2;           // scale * log2(e)
    int32_t T;
    int32_t rows_per_stream;    // G * T
    int32_t m_tiles;            // ceil(rows_per_stream / 128)
    int32_t d;
    int32_t window;             // sliding window C, 0 = none
    int32_t force_partial;      // write every segment to its partial slot, even of an unsplit stream
    PageMap pages;              // paged cache only
};
// tmQ: [B*Hq*T, d] box {64, 128}; tmK / tmV: [rows, d] box {64, kChunkTileN}; 128-byte swizzle.
// Grid = num_groups * m_tiles CTAs, the row tile varying fastest so that the CTAs that walk the
// same K/V range run side by side and share it through L2.
cudaError_t launch_chunk(const ChunkParams& p, const CUtensorMap& tmQ, const CUtensorMap& tmK,
                         const CUtensorMap& tmV, int num_groups, cudaStream_t stream, bool paged = false);
cudaError_t chunk_kernel_setup();
// Same interface for streams with more than 128 rows: one CTA owns two 128-row tiles (m_tiles =
// ceil(rows_per_stream / 256)), tmQ box is still {64, 128}.
// paged: rows are found through p.pages, tmK / tmV boxes are {64, min(P, kChunkTileN)}.
// fp8_scales (host, may be null): K and V are an 8-bit cache (tmK / tmV then are uint8 maps over the
// [rows, 128] byte view, box {128, kChunkTileN}); head dimension 128 only.
struct ChunkFp8Scales {
    int32_t Hkv;
    float score_scale_log2[kFp8MaxHeads]; // per KV head: softmax scale * k_scale[c] * log2(e)
    float v_scale[kFp8MaxHeads];          // per KV head
};
cudaError_t launch_chunk_pair(const ChunkParams& p, const CUtensorMap& tmQ, const CUtensorMap& tmK,
                              const CUtensorMap& tmV, int num_groups, cudaStream_t stream,
                              const ChunkFp8Scales* fp8_scales = nullptr, bool paged = false);
// The same over 4-bit pages, maps with boxes of min(P, 32) rows.
cudaError_t launch_chunk_pair_q4(const ChunkParams& p, const CUtensorMap& tmQ, const PagedQ4Maps& maps, int num_groups,
                                 cudaStream_t stream);
cudaError_t chunk_pair_kernel_setup();

// ---- writing the cache: K^ = RMSNorm(X) W_K, V^ = RMSNorm(X) W_V appended head-major ------------
constexpr int kAppendMaxSequences = 512;
struct KvAppendParams {
    const __nv_bfloat16* X;     // [M, d_model] (the few-token kernel reads it with plain loads)
    __nv_bfloat16* K;           // packed head-major caches
    __nv_bfloat16* V;
    int32_t M;                  // B * T tokens
    int32_t T, d, d_model;
    int32_t n_half;             // Hkv * d: output columns of K^ (those of V^ follow)
    float eps;
};
struct KvAppendTables {         // per sequence, as kernel parameters
    int32_t row0[kAppendMaxSequences];       // cache row (units of d elements) of (head 0, key N_i - T)
    int32_t head_rows[kAppendMaxSequences];  // rows between two heads of the sequence
};
// tmX: [M, d_model] box {64, 128}; tmWk / tmWv: gain-folded weights [d_model, Hkv*d] box {64, 128};
// 128-byte swizzle.  Grid = (2*Hkv*d/128, ceil(M/128)); with M <= 16 tokens (a decode step) a second
// kernel streams the weights instead: clusters of CTAs split d_model and add up through
// distributed shared memory.
struct KvAppendScales {         // 8-bit cache: reciprocal of the per-head scales (value = scale * e4m3(byte))
    float inv_k[kFp8MaxHeads];
    float inv_v[kFp8MaxHeads];
};
// fp8_scales (host, may be null): store FP8 E4M3 bytes instead of bf16.
cudaError_t launch_kv_append(const KvAppendParams& p, const KvAppendTables& tab, const CUtensorMap& tmX,
                             const CUtensorMap& tmWk, const CUtensorMap& tmWv, cudaStream_t stream,
                             const KvAppendScales* fp8_scales = nullptr);
cudaError_t launch_fold_gain(const __nv_bfloat16* g, const __nv_bfloat16* W, __nv_bfloat16* Wg, int64_t d_model,
                             int64_t n_out, cudaStream_t stream);
cudaError_t read_and_clear_kv_append_status(int32_t* word, cudaStream_t stream);
cudaError_t kv_append_status_address(int32_t** word);    // on the current device
cudaError_t kv_append_kernel_setup();

// ---- rows of a paged cache: append with rotation, read back, rotation of the queries --------------
constexpr int kQ4Group = 32;            // channels of a 4-bit row that share a scale
constexpr float kQ4ScaleMax = 448.f;    // largest scale a 4-bit row is given
template <int N>
struct SeqTableOf {             // per sequence, as kernel parameters
    int32_t pos0[N];            // position of the sequence's first token of this call
    int32_t tok0[N + 1];        // its first token among all tokens of the call
};
using SeqTable = SeqTableOf<kAppendMaxSequences>;
struct Rotation {
    const float* cos_sin;       // [max_pos, d]: d/2 cosines, d/2 sines of a position; null = no rotation
    int32_t neighbours;         // 0: channels (c, c + d/2) turn together; 1: (2c, 2c + 1)
};
struct PagedRowsParams {
    PageMap pages;
    Rotation rot;
    const __nv_bfloat16* k_src; // append: new rows, src_stride elements between tokens, heads consecutive
    const __nv_bfloat16* v_src;
    int64_t src_stride;
    void* k_pool;               // bf16 rows, or 4-bit codes (d/2 bytes a row)
    void* v_pool;
    __half* k_scale;            // 4-bit rows: d/32 scales a row
    __half* v_scale;
    __nv_bfloat16* k_out;       // gather: packed head-major rows
    __nv_bfloat16* v_out;
    int32_t* status;
    int32_t B, d, tokens;
    int32_t tokens_per_seq;     // > 0: every sequence has so many; 0: see SeqTable::tok0
};
cudaError_t launch_paged_append(const PagedRowsParams& p, const SeqTable& tab, bool q4, cudaStream_t stream);
cudaError_t launch_paged_gather(const PagedRowsParams& p, const SeqTable& tab, bool q4, cudaStream_t stream);
// Qr[b, h, t] = Q[b, h, t] turned by the angles of position tab.pos0[b] + t (rows at negative positions are copied)
cudaError_t launch_rope_q(const __nv_bfloat16* Q, __nv_bfloat16* Qr, int32_t B, int32_t Hq, int32_t T, int32_t d,
                          const Rotation& rot, const SeqTable& tab, cudaStream_t stream);

// ---- token-major rows: rotation by computed angles, normalisation of the heads with a gate -----------
struct RopeParams {
    const __nv_bfloat16* q;     // rows q_stride elements apart, Hq heads of d channels
    const __nv_bfloat16* k;     // null: none
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const double* inv_freq;     // [rot / 2]
    int32_t B, Hq, Hk, d, rot, neighbours, tokens;
    int32_t tokens_per_seq;     // > 0: every sequence has so many; 0: see SeqTable::tok0
};
cudaError_t launch_rope(const RopeParams& p, const SeqTable& tab, int sm_count, cudaStream_t stream);

struct NormGate {               // y = swish(gate) * (normalised x * gain + bias); see yoco_norm_gate
    const __nv_bfloat16* gate;  // null: none; heads consecutive, gate_stride elements between tokens
    const __nv_bfloat16* gain;  // null: ones
    const __nv_bfloat16* bias;  // null: zeros
    int64_t gate_stride;
    float eps;
    int32_t rms;                // 0: mean and variance, 1: root mean square
    int32_t on;                 // 0: x as it is
};
struct HeadNormParams {
    const __nv_bfloat16* x;
    __nv_bfloat16* y;
    int64_t x_stride, y_stride;
    NormGate norm;
    int32_t groups;             // tokens * H
    int32_t H, d;
};
cudaError_t launch_head_norm(const HeadNormParams& p, cudaStream_t stream);

// ---- gated retention -----------------------------------------------------------------------------------
constexpr float kMinLogDecay = -110.f;      // e^-110 is 0 in fp32
struct GretParams {
    const __nv_bfloat16* q;     // token-major rows, heads consecutive
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const void* decay;          // [tokens, H] fp32 or bf16
    __nv_bfloat16* o;
    float* state;               // [slots, H, d, d]
    int64_t q_stride, k_stride, v_stride, o_stride, decay_stride;
    NormGate norm;
    float scale;
    float inv_tau;              // 0: decay holds natural logarithms; otherwise logits, 1 / tau
    int32_t decay_bf16;
    int32_t B, H, d;
};
template <int N>
struct GretTableOf {            // per sequence, as kernel parameters
    int32_t from[N], to[N];     // slots, -1: zero state / not kept
    int32_t tok0[N + 1];        // first token among all tokens of the call
};
using GretTable = GretTableOf<kAppendMaxSequences>;
// One CTA per (sequence, head) walks its tokens with the state in registers.
cudaError_t launch_gret_tokens(const GretParams& p, const GretTable& tab, cudaStream_t stream);

// The chunkwise form.  The flat space of (sequence, head, chunk), in that order, has `total` chunks.
constexpr int kGretChunk = 128;     // tokens of a chunk
template <int N>
struct GretChunkTableOf {       // sequences with at least one token
    int32_t from[N], to[N];
    int32_t tok0[N], len[N];
    int32_t chunk0[N + 1];      // chunks of the sequences before this one (of one head)
};
using GretChunkTable = GretChunkTableOf<kAppendMaxSequences>;
struct GretChunkParams {
    GretParams base;            // base.B: sequences of the table
    int32_t total;
    int32_t groups;             // CTAs
    int32_t split;              // 1: CTA g walks chunks [first_of(g), first_of(g + 1)); 0: every groups-th stream
    int32_t share, extra;       // total / groups, total % groups
    __host__ __device__ int32_t first_of(int32_t g) const { return g * share + (g < extra ? g : extra); }
    float* part;                // split: 3 * groups states
    float* part_keep;           // split: decays over the segments that left them, 3 * groups
    int32_t* status;
    int32_t wait_limit_ns;      // 0 = the default limit of a bounded wait
    int32_t selftest_skip_loads;// self-test of the give-up path: the producer arms no copy, so the first waits run out with nothing in flight
};
// tmQ, tmK, tmV: bf16 maps over [tokens, H * d], box {64, kGretChunk} (K and V: kGretChunk / 2), 128-byte swizzle
cudaError_t launch_gret_chunk(const GretChunkParams& p, const GretChunkTable& tab, const CUtensorMap& tmQ, const CUtensorMap& tmK,
                              const CUtensorMap& tmV, cudaStream_t stream);
cudaError_t gret_chunk_kernel_setup();

}  // namespace yoco
