// Host-side planner and the device-visible work tables shared by the kernels.
//
// The split-count / tile heuristic: all (sequence, KV head) streams are laid end to end
// in units of key tiles and the resulting flat range is cut into equal contiguous pieces,
// one per CTA group, so that every group streams the same number of K/V bytes and the
// whole grid finishes together in a single wave.
#pragma once

#include <cstddef>
#include <cstdint>
#include <vector>

#include "yoco_xattn.h"

namespace yoco {

constexpr int kDecodeTileN = 64;      // keys per shared-memory stage of the decode kernel
constexpr int kDecodeTileM = 16;      // query rows of one mma.sync tile
constexpr int kDecodeGroupsPerSm = 2; // resident decode CTAs per SM
constexpr int kChunkTileN = 128;      // keys per tcgen05 tile
constexpr int kChunkTileM = 128;      // query rows per tcgen05 tile
constexpr int kChunkPairTileM = 256;  // rows per CTA when a stream has more than 128 rows: two tiles
                                      // that share every K/V tile in shared memory
constexpr int kWorkspaceHeaderBytes = 256;
constexpr int kWorkCounterOffset = 64;  // byte offset of the decode kernel's work counter in the header

// ---- pieces of a decode group ---------------------------------------------------------------
// SMs do not all stream at the same rate (their share of the memory fabric differs with their
// place on the die), so equal static shares leave the fast ones idle at the end.  With R > 1 a
// group's tile range is cut into R pieces of decreasing size; piece 0 is taken by the group's own
// CTA, the rest are handed out in order to whichever CTA is free.  The pieces are fixed by the plan
// (integers only), so the result does not depend on who ran what.
constexpr int kMaxSubItems = 4;

#ifdef __CUDACC__
#define YOCO_HD __host__ __device__
#else
#define YOCO_HD
#endif
// First tile (inside a group of n tiles) of piece r of R, r = 0..R; R in {1, 2, 4}.
YOCO_HD inline int64_t sub_bound(int64_t n, int R, int r) {
    // cumulative shares in 64ths: a large first piece, then smaller and smaller ones
    const unsigned c4 = 0x403D362Cu;                       // 44 54 61 64
    if (r <= 0) return 0;
    if (r >= R) return n;
    const int c = R == 4 ? (int)((c4 >> (8 * (r - 1))) & 0xFF) : 52;   // R == 2: 52 | 12
    return n * c / 64;
}
#undef YOCO_HD

// Pieces per group for a decode plan whose groups hold `tiles_per_group` key tiles on average.
// (Measured on B200, 32 query heads over 8 KV heads: two pieces pay from 128K keys per sequence,
// four from 256K; eight gained nothing over four at 1M and made the merge longer.)
inline int choose_sub_items(int64_t tiles_per_group, int max_sub) {
    int R = tiles_per_group >= 96 ? 4 : tiles_per_group >= 40 ? 2 : 1;
    while (R > max_sub) R /= 2;
    return R < 1 ? 1 : R;
}

// One work segment as the kernels read it (10 x int32 = 40 bytes).
struct DevSegment {
    int32_t kv_row0;     // row of key k_begin in the [rows, d] view of the packed K/V buffers
    int32_t k_begin;     // first key of the range inside its sequence
    int32_t k_end;       // one past the last key
    int32_t q_row0;      // first row of this stream in the [B*Hq*T, d] view of Q / O
    int32_t slot;        // partial-result slot
    int32_t n_kv;        // N_i of the sequence
    int32_t stream_nseg; // segments of this stream (1: the kernel writes the final output)
    int32_t stream;      // b * Hkv + c
    int32_t n_full;      // keys (counted from key 0 of this cache) that query row 0 sees: N_i - T + 1 for a
                         // whole cache; for one shard of a key-range-sharded cache the same count minus
                         // the keys held by earlier shards (may be <= 0 or exceed n_kv).  Row t sees n_full + t.
    int32_t pad_;
};
constexpr int kSegmentWords = 10;

struct Plan {
    yoco_xattn_plan_info info{};
    std::vector<yoco_xattn_segment> segments;   // public form
    std::vector<int32_t> table;                  // device blob: segments, group offsets, stream tables
    // offsets in int32 units inside `table`
    int32_t off_segments = 0, off_group_begin = 0, off_stream_base = 0, off_stream_nseg = 0;
    // byte offsets inside the workspace
    int64_t ws_table = 0, ws_part_lse = 0, ws_part_o = 0;
    int64_t kv_rows_extent = 0;                  // rows of the [rows, d] K/V view that may be touched
    int32_t rows_per_stream = 0;                 // G * T
    int32_t sub_items = 1;                       // pieces per group (decode), see sub_bound
    int32_t coarse_segments = 0;                 // entries of the device segment table; partial slots
                                                 // = coarse_segments * sub_items
};

// Warps of the 4-bit decode kernel for up to 8 query rows per stream, and above.
constexpr int kQ4Warps8 = 12, kQ4Warps16 = 8;

// What the cache of a plan is made of.
// pair_tiles: chunk plans use the two-row-tile CTA (kChunkPairTileM) whatever G*T is (an 8-bit or 4-bit cache is
// read by that kernel only).
// piece_divisor: decode plans choose the pieces per group as for so many times fewer tiles (a tile of an 8-bit
// cache is half the bytes, and the pieces pay by bytes: measured at 55 tiles per group, one piece 51.0 us, two
// 52.9 us).
// paged: rows are found through a page table, so the plan holds no row numbers and no extent.
struct CacheForm {
    bool pair_tiles = false;
    int piece_divisor = 1;
    bool paged = false;
    int groups_per_sm = kDecodeGroupsPerSm;   // resident decode CTAs per SM
    int max_pieces = 4;                       // most pieces per decode group
    // Tiles that a CTA's warps work off side by side (whole tiles per warp), up to 8 and above 8 query rows; 0: tiles
    // are shared by the warps.  A problem so small that no CTA would need a second turn is then cut at the
    // streams' ends: as many groups per stream as it has such handfuls, each a run of its own.  (Measured, 8
    // sequences of 700 to 1,100 keys, 8 KV heads: groups of equal size, most of them in two streams, 16.1 us;
    // groups that end with their stream 12.8 us, and streams of at most 12 tiles need no merge.)
    // A merge costs more than a second turn: streams of up to two handfuls stay whole (the call of the case above 15.4 -> 14.4
    // us, 16 sequences of 1,000 keys 21.6 -> 14.4), and streams of up to three where handfuls would be too many for the
    // SMs (8 sequences of 2,200 keys 22.1 -> 18.5 us; one such sequence, whose handfuls fit, 15.4 against 17.6).
    int side_by_side8 = 0, side_by_side16 = 0;
    // What going over to another stream costs a group (the warps' unequal last turns, the merge, the first loads), in
    // tiles: shares are equal with it counted in.  (Measured with 0 / 12 / 24 / 40: 16 sequences of 4,001 to 62,000
    // keys 141 / 121 / 118 / 121 us, 64 of 1,000 to 8,000 keys 104 / 88 / 86 / 90 us, one of 1M keys 221 / 219 / 219 / 219 us.)
    int stream_tiles = 0;
    bool operator==(const CacheForm& o) const {
        return pair_tiles == o.pair_tiles && piece_divisor == o.piece_divisor && paged == o.paged && groups_per_sm == o.groups_per_sm &&
               max_pieces == o.max_pieces && side_by_side8 == o.side_by_side8 && side_by_side16 == o.side_by_side16 &&
               stream_tiles == o.stream_tiles;
    }
};
constexpr CacheForm kBf16Cache{};
constexpr CacheForm kFp8Cache{true, 2, false};
constexpr CacheForm kPagedCache{false, 1, true};
constexpr CacheForm kPagedQ4Cache{true, 1, true, 1, 1, kQ4Warps8, kQ4Warps16, 24};

// Returns YOCO_OK or an error code; fills `plan`.  cu_kv_host may be null (tight packing).
// max_sub_items: upper limit of pieces per decode group (1 = every group is one piece).
// key_offset_host / kv_total_host (both null, or both [B]): the cache described by kv_len_host is
// keys [key_offset[i], key_offset[i] + kv_len[i]) of a sequence of kv_total[i] keys; the causal and
// window masks then use the rows' positions in the whole sequence.
int32_t make_plan(const yoco_xattn_shape& s, const int32_t* cu_kv_host, const int32_t* kv_len_host,
                  int32_t sm_count, int32_t mode, Plan& plan, int32_t max_sub_items = kMaxSubItems,
                  const int32_t* key_offset_host = nullptr, const int32_t* kv_total_host = nullptr,
                  const CacheForm& form = kBf16Cache);

// Bytes that suffice for make_plan's workspace with any lengths up to those given (the rest of the shape, and no shards).
int32_t workspace_bound(const yoco_xattn_shape& s, const int32_t* kv_len_host, int32_t sm_count, int32_t mode,
                        const CacheForm& form, int64_t* bytes);

int32_t validate_shape(const yoco_xattn_shape& s, int32_t mode);
// Lengths, head stride and token offsets must describe sequences that do not overlap (pure host).
int32_t validate_layout(const yoco_xattn_shape& s, const int32_t* cu_kv_host, const int32_t* kv_len_host);

}  // namespace yoco
