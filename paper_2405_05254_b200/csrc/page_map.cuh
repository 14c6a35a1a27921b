// Walking the pages of a sequence tile by tile (device side of PageMap).
#pragma once

#include "kernels.h"

namespace yoco {

__device__ __forceinline__ void report_bad_page(int32_t* status) {
    atomicCAS(status, 0, status_word(kBadPage, (int32_t)(blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z))));
}

// Lowest key that any row of a segment sees: with a window, row 0's first one.  Keys below it in the same tile are read by
// nobody: their pages may be gone and their rows may hold anything.  (n_full is negative where the first rows see no key, and a
// window may be as long as an int holds: the difference of the two would leave 32 bits.)
__device__ __forceinline__ int first_seen(int n_full, int window) { return window > 0 ? max(0, max(n_full, 0) - window) : 0; }

// A producer warp's view of the pages of one (sequence, KV head) stream.  Every lane holds one page, 32 at a time:
// the pool row of its first slot, so that a tile costs one shuffle per box; the next 32 are already requested, so a
// table read is waited for once per run.  (A producer is one warp working through a chain of dependent
// instructions: what it does per tile has to fit in the time of a tile.  Page numbers looked up, checked and
// multiplied tile by tile, or kept in registers of one thread and shifted along, where a move waits for its load, did
// not.)  All lanes call it together; keys only grow; k_lo is a multiple of TILE.
template <int TILE>
struct PageCursor {
    // copies, not a reference to the kernel's parameters: those would be read again after every barrier wait
    int shift, num_pages, page_rows, pool_rows, head_row;
    const int32_t* entries;                        // this sequence's row of the table
    int32_t* status;
    int first, last, lane;
    int seen;                                      // first page with a key that somebody sees
    int32_t now;                                   // row of page first + lane
    int32_t later;                                 // number of page first + 32 + lane

    __device__ __forceinline__ int32_t fetch(int page) const { return page <= last ? __ldg(entries + page) : 0; }
    __device__ __forceinline__ int32_t row_of(int32_t page) const {      // `page` is the entry first + lane
        if ((uint32_t)page < (uint32_t)num_pages && first + lane >= seen) return page * page_rows + head_row;
        if (first + lane >= seen) report_bad_page(status);               // (entries behind the run were replaced by page 0)
        return pool_rows;
    }
    __device__ __forceinline__ void start(const PageMap& map, int stream, int k_lo, int k_end, int key_seen, int32_t* status_word) {
        shift = map.page_shift;
        num_pages = map.num_pages;
        page_rows = map.page_rows;
        pool_rows = map.rows;
        status = status_word;
        const int b = stream / map.Hkv;
        head_row = (stream - b * map.Hkv) << shift;
        entries = map.table + (int64_t)b * map.table_stride;
        lane = (int)(threadIdx.x & 31u);
        first = k_lo >> shift;
        last = (k_end - 1) >> shift;
        seen = key_seen >> shift;
        const int32_t page = fetch(first + lane);
        later = fetch(first + 32 + lane);
        now = row_of(page);
    }
    // To be called for every tile before row(): the 32 pages at hand cover it (a tile never straddles two batches,
    // both are multiples of the tile's pages).  Returns how many boxes the tile has: those with at least one key.
    __device__ __forceinline__ int enter(int k0) {
        const int page = k0 >> shift;
        if (page - first >= 32) {
            first += 32;
            now = row_of(later);
            later = fetch(first + 32 + lane);
        }
        return min(max(1, TILE >> shift), last + 1 - page);
    }
    // pool row that box j of the tile at key k0 starts at; it brings box_rows() rows
    __device__ __forceinline__ int row(int k0, int j) const {
        return __shfl_sync(0xffffffffu, now, (k0 >> shift) + j - first) + ((1 << shift) > TILE ? k0 & ((1 << shift) - 1) : 0);
    }
    __device__ __forceinline__ int box_rows() const { return min(TILE, 1 << shift); }
};

}  // namespace yoco
