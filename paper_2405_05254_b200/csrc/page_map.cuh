// Walking the pages of a sequence tile by tile (device side of PageMap).
#pragma once

#include "kernels.h"

namespace yoco {

__device__ __forceinline__ void report_bad_page(int32_t* status) {
    atomicCAS(status, 0, status_word(kBadPage, (int32_t)(blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z))));
}

// Row of (page, head, slot 0), or a row behind the pool (which a tensor copy fills with zeros) when the
// page table entry is not a page of the pool.
__device__ __forceinline__ int page_row(const PageMap& pm, int page, int head, int32_t* status) {
    if ((uint32_t)page < (uint32_t)pm.num_pages) return page * pm.page_rows + (head << pm.page_shift);
    report_bad_page(status);
    return pm.rows;
}

// The producer's position in a run of TILE-key tiles of one (sequence, KV head) stream.  The page numbers of
// the next AHEAD tiles are already requested when a tile's copies are issued, so that a table read is
// not waited for between two copies.
template <int TILE, int AHEAD = 2>
struct PageCursor {
    static constexpr int MAX_IDS = TILE / 16;      // pages hold at least 16 keys
    const PageMap* pm;
    const int32_t* entries;                        // this sequence's row of the table
    int head, k0, k_hi;
    int32_t id[AHEAD + 1][MAX_IDS];

    __device__ __forceinline__ void fetch(int32_t (&out)[MAX_IDS], int k) const {
        const int P = 1 << pm->page_shift;
#pragma unroll
        for (int j = 0; j < MAX_IDS; ++j) {
            const int key = k + j * P;             // one page when P >= TILE
            out[j] = (j == 0 || j * P < TILE) && key < k_hi ? __ldg(entries + (key >> pm->page_shift)) : 0;
        }
    }
    __device__ __forceinline__ void start(const PageMap& map, int stream, int k_lo, int k_end) {
        pm = &map;
        const int b = stream / map.Hkv;
        head = stream - b * map.Hkv;
        entries = map.table + (int64_t)b * map.table_stride;
        k0 = k_lo;
        k_hi = k_end;
#pragma unroll
        for (int a = 0; a <= AHEAD; ++a) fetch(id[a], k_lo + a * TILE);
    }
    // rows that the boxes of this tile bring: whole boxes, those with at least one key of the run
    __device__ __forceinline__ int rows() const {
        const int P = 1 << pm->page_shift;
        return P >= TILE ? TILE : min(TILE, ((k_hi - k0 + P - 1) >> pm->page_shift) << pm->page_shift);
    }
    // f(first row inside the tile, first row in the pool) for every box
    template <class F>
    __device__ __forceinline__ void for_each_box(int32_t* status, F f) const {
        const int P = 1 << pm->page_shift;
        if (P >= TILE) {
            const int r = page_row(*pm, id[0][0], head, status);
            f(0, r == pm->rows ? r : r + (k0 & (P - 1)));
            return;
        }
#pragma unroll
        for (int j = 0; j < MAX_IDS; ++j) {
            if (j * P < TILE && k0 + j * P < k_hi) f(j * P, page_row(*pm, id[0][j], head, status));
        }
    }
    __device__ __forceinline__ void next() {
        k0 += TILE;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
#pragma unroll
            for (int j = 0; j < MAX_IDS; ++j) id[a][j] = id[a + 1][j];
        fetch(id[AHEAD], k0 + AHEAD * TILE);
    }
};

}  // namespace yoco
