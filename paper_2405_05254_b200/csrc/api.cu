// C ABI of the library: argument checks, plan cache, tensor maps, kernel launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <list>
#include <memory>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "kernels.h"
#include "plan.h"
#include "yoco_xattn.h"

namespace yoco {
namespace {

thread_local int32_t g_last_cuda_error = 0;

// what a status word of the device means to the caller
int32_t status_code(int32_t word) {
    return word == kStatusOk ? YOCO_OK : (word & 0xFF) == kBadPage ? YOCO_ERR_BAD_PAGE : YOCO_ERR_TIMEOUT;
}

int32_t cuda_fail(cudaError_t e) {
    g_last_cuda_error = (int32_t)e;
    return YOCO_ERR_CUDA;
}
#define YOCO_CUDA_TRY(expr)                               \
    do {                                                  \
        cudaError_t e__ = (expr);                         \
        if (e__ != cudaSuccess) return cuda_fail(e__);    \
    } while (0)

// ---- per-device state ---------------------------------------------------------------------
constexpr int kMaxDevices = 64;
struct DeviceState {
    bool ready = false;
    int sm_count = 0;
    int32_t* append_status = nullptr;    // status word of the kernels that take no workspace
};
std::mutex g_mutex;
DeviceState g_dev[kMaxDevices];

int32_t device_state(DeviceState** out) {
    int dev = 0;
    YOCO_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return YOCO_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_mutex);
    DeviceState& st = g_dev[dev];
    if (!st.ready) {
        int major = 0;
        YOCO_CUDA_TRY(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
        if (major != 10) return YOCO_ERR_UNSUPPORTED;   // built for sm_100a only
        YOCO_CUDA_TRY(cudaDeviceGetAttribute(&st.sm_count, cudaDevAttrMultiProcessorCount, dev));
        YOCO_CUDA_TRY(decode_kernel_setup());
        YOCO_CUDA_TRY(chunk_kernel_setup());
        YOCO_CUDA_TRY(chunk_pair_kernel_setup());
        YOCO_CUDA_TRY(kv_append_kernel_setup());
        YOCO_CUDA_TRY(decode_fp8_kernel_setup());
        YOCO_CUDA_TRY(decode_q4_kernel_setup());
        YOCO_CUDA_TRY(gret_chunk_kernel_setup());
        YOCO_CUDA_TRY(kv_append_status_address(&st.append_status));
        st.ready = true;
    }
    *out = &st;
    return YOCO_OK;
}

// ---- plan cache ---------------------------------------------------------------------------
struct PlanKey {
    yoco_xattn_shape shape;
    int32_t sm_count, mode, max_sub;
    CacheForm form;
    std::vector<int32_t> lens, cu, key_off, totals;
    bool operator==(const PlanKey& o) const {
        return std::memcmp(&shape, &o.shape, sizeof shape) == 0 && sm_count == o.sm_count &&
               mode == o.mode && max_sub == o.max_sub && form == o.form && lens == o.lens && cu == o.cu &&
               key_off == o.key_off && totals == o.totals;
    }
};
// A cached plan with the launch-ready forms of its tables.
struct ReadyPlan {
    Plan plan;
    std::vector<int32_t> blob;           // workspace image: zeroed header + tables (upload path)
    bool fits_inline = false;            // tables small enough to travel as kernel parameters
    DecodeInlineTables decode_tab;
    CombineInlineTables combine_tab;
};
struct PlanEntry {
    PlanKey key;
    std::shared_ptr<const ReadyPlan> ready;
};
std::list<PlanEntry> g_plans;   // most recently used first
constexpr size_t kPlanCacheEntries = 16;
// Plans whose table upload was recorded into a CUDA graph: the recorded copy reads the plan's host
// image at every replay, so these are never dropped.
std::vector<std::shared_ptr<const ReadyPlan>> g_captured_plans;

// Looks the plan up (most recently used first) or makes it.  The shared pointer keeps the entry
// alive for the caller even if another thread evicts it from the cache meanwhile.
int32_t cached_plan(const yoco_xattn_shape& s, const int32_t* cu, const int32_t* lens, int32_t sm_count,
                    int32_t mode, int32_t max_sub, std::shared_ptr<const ReadyPlan>& out,
                    const int32_t* key_off = nullptr, const int32_t* totals = nullptr,
                    const CacheForm& form = kBf16Cache) {
    PlanKey key;
    std::memset(&key.shape, 0, sizeof key.shape);
    key.shape = s;
    key.sm_count = sm_count;
    key.mode = mode;
    key.max_sub = max_sub;
    key.form = form;
    if (lens) key.lens.assign(lens, lens + s.B);
    if (cu) key.cu.assign(cu, cu + s.B + 1);
    if (key_off) key.key_off.assign(key_off, key_off + s.B);
    if (totals) key.totals.assign(totals, totals + s.B);
    {
        std::lock_guard<std::mutex> lock(g_mutex);
        for (auto it = g_plans.begin(); it != g_plans.end(); ++it)
            if (it->key == key) {
                g_plans.splice(g_plans.begin(), g_plans, it);
                out = g_plans.front().ready;
                return YOCO_OK;
            }
    }
    auto ready = std::make_shared<ReadyPlan>();
    int32_t rc = make_plan(s, cu, lens, sm_count, mode, ready->plan, max_sub, key_off, totals, form);
    if (rc != YOCO_OK) return rc;
    const Plan& plan = ready->plan;
    ready->blob.assign(kWorkspaceHeaderBytes / 4 + plan.table.size(), 0);
    std::copy(plan.table.begin(), plan.table.end(), ready->blob.begin() + kWorkspaceHeaderBytes / 4);
    ready->fits_inline = mode == YOCO_MODE_DECODE && plan.coarse_segments <= kInlineSegments &&
                         plan.info.num_groups <= kInlineGroups && plan.info.num_streams <= kInlineStreams;
    if (ready->fits_inline) {
        std::memset(&ready->decode_tab, 0, sizeof ready->decode_tab);
        std::memset(&ready->combine_tab, 0, sizeof ready->combine_tab);
        std::memcpy(ready->decode_tab.seg, plan.table.data() + plan.off_segments,
                    (size_t)plan.coarse_segments * sizeof(DevSegment));
        static_assert(sizeof(DecodeInlineTables) + sizeof(DecodeFp8Params) + 2 * sizeof(CUtensorMap) < 32000,
                      "kernel parameter space");
        std::memcpy(ready->decode_tab.group_begin, plan.table.data() + plan.off_group_begin,
                    (size_t)(plan.info.num_groups + 1) * 4);
        std::memcpy(ready->combine_tab.stream_base, plan.table.data() + plan.off_stream_base,
                    (size_t)plan.info.num_streams * 4);
        std::memcpy(ready->combine_tab.stream_nseg, plan.table.data() + plan.off_stream_nseg,
                    (size_t)plan.info.num_streams * 4);
    }
    out = ready;
    std::lock_guard<std::mutex> lock(g_mutex);
    g_plans.push_front(PlanEntry{std::move(key), std::move(ready)});
    if (g_plans.size() > kPlanCacheEntries) g_plans.pop_back();
    return YOCO_OK;
}

// ---- tensor maps ----------------------------------------------------------------------------
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                   const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn g_encode = nullptr;

int32_t get_encoder(EncodeTiledFn* fn) {
    std::lock_guard<std::mutex> lock(g_mutex);
    if (!g_encode) {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        YOCO_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q));
        if (q != cudaDriverEntryPointSuccess || !sym) return cuda_fail(cudaErrorNotSupported);
        g_encode = reinterpret_cast<EncodeTiledFn>(sym);
    }
    *fn = g_encode;
    return YOCO_OK;
}

// A serving loop calls with the same cache pointers and extents step after step: the last few
// encoded maps are kept per host thread, keyed by everything that goes into the encoding.
struct MapKey {
    const void* base;
    int64_t rows, stride;
    int32_t row_bytes, box_rows, box_bytes, bf16;
    CUtensorMapSwizzle swizzle;
    bool operator==(const MapKey& o) const {
        return base == o.base && rows == o.rows && stride == o.stride && row_bytes == o.row_bytes && box_rows == o.box_rows &&
               box_bytes == o.box_bytes && bf16 == o.bf16 && swizzle == o.swizzle;
    }
};
struct MapCache {
    static constexpr int kEntries = 16;
    MapKey key[kEntries];
    CUtensorMap map[kEntries];
    int used = 0, next = 0;
    bool find(const MapKey& k, CUtensorMap* out) const {
        for (int i = 0; i < used; ++i)
            if (key[i] == k) {
                *out = map[i];
                return true;
            }
        return false;
    }
    void put(const MapKey& k, const CUtensorMap& m) {
        key[next] = k;
        map[next] = m;
        next = (next + 1) % kEntries;
        if (used < kEntries) ++used;
    }
};
thread_local MapCache g_maps;

// 2-D map over a row-major matrix of `rows` rows of row_bytes bytes, stride bytes apart (0: row_bytes), as bf16 or bytes; box
// {box_bytes, box_rows}, swizzled by the box's width (128 or 64 bytes) or not at all.
int32_t make_map(CUtensorMap* map, const void* base, int64_t rows, int32_t row_bytes, int32_t box_bytes,
                 int32_t box_rows, bool bf16, CUtensorMapSwizzle swizzle, int64_t stride = 0) {
    if (stride == 0) stride = row_bytes;
    const MapKey mk{base, rows, stride, row_bytes, box_rows, box_bytes, bf16 ? 1 : 0, swizzle};
    if (g_maps.find(mk, map)) return YOCO_OK;
    EncodeTiledFn enc;
    int32_t rc = get_encoder(&enc);
    if (rc != YOCO_OK) return rc;
    const int32_t elem = bf16 ? 2 : 1;
    cuuint64_t gdim[2] = {(cuuint64_t)(row_bytes / elem), (cuuint64_t)rows};
    cuuint64_t gstride[1] = {(cuuint64_t)stride};
    cuuint32_t box[2] = {(cuuint32_t)(box_bytes / elem), (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1u, 1u};
    CUresult r = enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2,
                     const_cast<void*>(base), gdim, gstride, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cuda_fail(cudaErrorInvalidValue);
    g_maps.put(mk, *map);
    return YOCO_OK;
}

// bf16 [rows, d], box {64 channels, box_rows}, 128-byte swizzle
int32_t make_map_2d(CUtensorMap* map, const void* base, int64_t rows, int32_t d, int32_t box_rows) {
    return make_map(map, base, rows, d * 2, 128, box_rows, true, CU_TENSOR_MAP_SWIZZLE_128B);
}

// FP8 bytes [rows, 128], box {128, box_rows}, 128-byte swizzle
int32_t make_map_2d_u8(CUtensorMap* map, const void* base, int64_t rows, int32_t box_rows) {
    return make_map(map, base, rows, 128, 128, box_rows, false, CU_TENSOR_MAP_SWIZZLE_128B);
}

// the four maps of a 4-bit pool pair, for tiles of `tile` keys
int32_t make_q4_maps(PagedQ4Maps* m, const void* K, const void* k_scale, const void* V, const void* v_scale,
                     const PageMap& pages, int32_t tile) {
    const int32_t box = std::min(1 << pages.page_shift, tile);
    int32_t rc;
    if ((rc = make_map(&m->k, K, pages.rows / 2, 128, 128, box / 2, false, CU_TENSOR_MAP_SWIZZLE_128B)) != YOCO_OK) return rc;
    if ((rc = make_map(&m->v, V, pages.rows / 2, 128, 128, box / 2, false, CU_TENSOR_MAP_SWIZZLE_128B)) != YOCO_OK) return rc;
    if ((rc = make_map(&m->k_scale, k_scale, pages.rows / 16, 128, 128, box / 16, false, CU_TENSOR_MAP_SWIZZLE_NONE)) != YOCO_OK)
        return rc;
    return make_map(&m->v_scale, v_scale, pages.rows / 16, 128, 128, box / 16, false, CU_TENSOR_MAP_SWIZZLE_NONE);
}

// per-head scales of an 8-bit cache (host pointers)
struct Fp8Scales {
    const float* k_scale;
    const float* v_scale;
};

// ---- optional per-launch timing of the attention kernel -------------------------------------
struct Profiler {
    std::vector<cudaEvent_t> events;   // pairs: before / after the attention kernel
    int32_t used = 0;                  // pairs recorded so far
} g_prof;

cudaEvent_t prof_event(bool after, bool* active) {
    std::lock_guard<std::mutex> lock(g_mutex);
    const int32_t pairs = (int32_t)g_prof.events.size() / 2;
    if (g_prof.used >= pairs) {
        *active = false;
        return nullptr;
    }
    *active = true;
    cudaEvent_t e = g_prof.events[2 * g_prof.used + (after ? 1 : 0)];
    if (after) ++g_prof.used;
    return e;
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// self-test of the give-up path of the decode kernel (yoco_xattn_selftest_wait_expiry)
struct SelfTest {
    int64_t wait_limit_ns;
};
// a paged cache: where its rows are, and the scales of 4-bit rows (null: bf16 rows)
struct PagedCall {
    PageMap pages;
    const void* k_scale;
    const void* v_scale;
    CacheForm form() const { return k_scale ? kPagedQ4Cache : kPagedCache; }
};
// where the keys of this call sit in the whole sequences (one shard of a key-range-sharded cache)
struct ShardPos {
    const int32_t* key_offset;   // host [B]
    const int32_t* kv_total;     // host [B]
};

int32_t run(const yoco_xattn_shape* shape, int32_t mode, const void* Q, const void* K, const void* V,
            const int32_t* cu_kv_host, const int32_t* kv_len_host, void* O, float* lse,
            void* workspace, size_t workspace_bytes, void* stream_v, float* part_out = nullptr,
            const Fp8Scales* fp8 = nullptr, int32_t max_sub = kMaxSubItems, const SelfTest* selftest = nullptr,
            const ShardPos* shard = nullptr, const PagedCall* paged = nullptr) {
    // part_out != null: the result is a partial one (fp32 rows + their LSE in `lse`, no bf16 O)
    if (!shape) return YOCO_ERR_INVALID_ARG;
    int32_t rc = validate_shape(*shape, mode);
    if (rc != YOCO_OK) return rc;
    if (shape->B == 0) return YOCO_OK;
    if (!Q || !K || !V || !(O || part_out) || !workspace) return YOCO_ERR_INVALID_ARG;
    if (part_out && (!lse || !aligned(part_out, 16))) return YOCO_ERR_INVALID_ARG;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(O, 16) ||
        !aligned(workspace, 256) || (lse && !aligned(lse, 4)))
        return YOCO_ERR_INVALID_ARG;
    if ((rc = validate_layout(*shape, cu_kv_host, kv_len_host)) != YOCO_OK) return rc;

    DeviceState* dev = nullptr;
    if ((rc = device_state(&dev)) != YOCO_OK) return rc;

    std::shared_ptr<const ReadyPlan> ready;
    if ((rc = cached_plan(*shape, cu_kv_host, kv_len_host, dev->sm_count, mode, max_sub, ready,
                          shard ? shard->key_offset : nullptr, shard ? shard->kv_total : nullptr,
                          paged ? paged->form() : fp8 ? kFp8Cache : kBf16Cache)) != YOCO_OK)
        return rc;
    const Plan& plan = ready->plan;
    if ((int64_t)workspace_bytes < plan.info.workspace_bytes) return YOCO_ERR_WORKSPACE_TOO_SMALL;

    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_v);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const float scale = shape->scale != 0.f ? shape->scale : 1.f / std::sqrt((float)shape->d);

    const bool inline_tables = ready->fits_inline;
    if (inline_tables) {
        // the tables travel as kernel parameters: only the status word has to be cleared
        YOCO_CUDA_TRY(cudaMemsetAsync(ws, 0, kWorkspaceHeaderBytes, stream));
    } else {
        // header (status word = 0) + work tables in one copy.  The source is pageable memory, which
        // the runtime stages before the call returns, so the cache entry may go away afterwards --
        // unless the stream is being recorded into a graph: the recorded copy reads the same host
        // memory again at every replay, so such a plan is kept for the life of the process.
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        YOCO_CUDA_TRY(cudaStreamIsCapturing(stream, &cap));
        if (cap != cudaStreamCaptureStatusNone) {
            std::lock_guard<std::mutex> lock(g_mutex);
            bool kept = false;
            for (const auto& q : g_captured_plans) kept = kept || q == ready;
            if (!kept) g_captured_plans.push_back(ready);
        }
        YOCO_CUDA_TRY(cudaMemcpyAsync(ws, ready->blob.data(), ready->blob.size() * 4, cudaMemcpyHostToDevice,
                                      stream));
    }
    const int32_t* table = reinterpret_cast<const int32_t*>(ws + plan.ws_table);
    float* part_lse = reinterpret_cast<float*>(ws + plan.ws_part_lse);
    float* part_o = reinterpret_cast<float*>(ws + plan.ws_part_o);
    int32_t* status = reinterpret_cast<int32_t*>(ws);

    bool timed = false;   // an event pair was put around the attention kernel of this call
    if (plan.info.num_segments > 0) {
        bool prof = false;
        cudaEvent_t ev = prof_event(false, &prof);
        if (prof) YOCO_CUDA_TRY(cudaEventRecord(ev, stream));
        timed = prof;
        if (mode == YOCO_MODE_DECODE) {
            CUtensorMap tmK, tmV;
            PagedQ4Maps q4;
            const bool four_bit = paged && paged->k_scale;
            if (four_bit) {
                if ((rc = make_q4_maps(&q4, K, paged->k_scale, V, paged->v_scale, paged->pages, kDecodeTileN)) != YOCO_OK)
                    return rc;
            } else if (paged) {
                const int32_t box = std::min(1 << paged->pages.page_shift, kDecodeTileN);
                if ((rc = make_map_2d(&tmK, K, paged->pages.rows, shape->d, box)) != YOCO_OK) return rc;
                if ((rc = make_map_2d(&tmV, V, paged->pages.rows, shape->d, box)) != YOCO_OK) return rc;
            } else if (fp8) {
                if ((rc = make_map_2d_u8(&tmK, K, plan.kv_rows_extent, kDecodeTileN)) != YOCO_OK) return rc;
                if ((rc = make_map_2d_u8(&tmV, V, plan.kv_rows_extent, kDecodeTileN)) != YOCO_OK) return rc;
            } else {
                if ((rc = make_map_2d(&tmK, K, plan.kv_rows_extent, shape->d, kDecodeTileN)) != YOCO_OK) return rc;
                if ((rc = make_map_2d(&tmV, V, plan.kv_rows_extent, shape->d, kDecodeTileN)) != YOCO_OK) return rc;
            }
            DecodeParams p{};
            p.Q = static_cast<const __nv_bfloat16*>(Q);
            p.O = static_cast<__nv_bfloat16*>(O);
            p.lse = lse;
            p.segments = reinterpret_cast<const DevSegment*>(table + plan.off_segments);
            p.group_begin = table + plan.off_group_begin;
            p.part_o = part_o;
            p.part_lse = part_lse;
            p.status = status;
            p.scale_log2 = scale * 1.4426950408889634f;
            p.T = shape->T;
            p.rows_per_stream = plan.rows_per_stream;
            p.d = shape->d;
            p.window = shape->window;
            p.force_partial = part_out ? 1 : 0;
            p.sub_items = plan.sub_items;
            p.work_counter = reinterpret_cast<int32_t*>(ws + kWorkCounterOffset);
            if (paged) p.pages = paged->pages;
            if (selftest) {
                p.wait_limit_ns = selftest->wait_limit_ns;
                p.selftest_skip_loads = 1;
            }
            if (four_bit) {
                YOCO_CUDA_TRY(launch_decode_q4(p, q4, plan.info.num_groups, stream,
                                               inline_tables ? &ready->decode_tab : nullptr));
            } else if (fp8) {
                DecodeFp8Params p8{};
                p8.base = p;
                p8.Hkv = shape->Hkv;
                for (int c = 0; c < shape->Hkv; ++c) {
                    p8.score_scale_log2[c] = scale * fp8->k_scale[c] * 1.4426950408889634f;
                    p8.v_scale[c] = fp8->v_scale[c];
                }
                YOCO_CUDA_TRY(launch_decode_fp8(p8, tmK, tmV, plan.info.num_groups, stream,
                                                inline_tables ? &ready->decode_tab : nullptr));
            } else {
                YOCO_CUDA_TRY(launch_decode(p, tmK, tmV, plan.info.num_groups, stream,
                                            inline_tables ? &ready->decode_tab : nullptr, paged != nullptr));
            }
        } else {
            CUtensorMap tmQ, tmK, tmV;
            PagedQ4Maps q4;
            const bool four_bit = paged && paged->k_scale;
            const int64_t q_rows = (int64_t)shape->B * shape->Hq * shape->T;
            if ((rc = make_map_2d(&tmQ, Q, q_rows, shape->d, kChunkTileM)) != YOCO_OK) return rc;
            if (four_bit) {
                if ((rc = make_q4_maps(&q4, K, paged->k_scale, V, paged->v_scale, paged->pages, 32)) != YOCO_OK) return rc;
            } else if (paged) {
                const int32_t box = std::min(1 << paged->pages.page_shift, kChunkTileN);
                if ((rc = make_map_2d(&tmK, K, paged->pages.rows, shape->d, box)) != YOCO_OK) return rc;
                if ((rc = make_map_2d(&tmV, V, paged->pages.rows, shape->d, box)) != YOCO_OK) return rc;
            } else if (fp8) {
                if ((rc = make_map_2d_u8(&tmK, K, plan.kv_rows_extent, kChunkTileN)) != YOCO_OK) return rc;
                if ((rc = make_map_2d_u8(&tmV, V, plan.kv_rows_extent, kChunkTileN)) != YOCO_OK) return rc;
            } else {
                if ((rc = make_map_2d(&tmK, K, plan.kv_rows_extent, shape->d, kChunkTileN)) != YOCO_OK) return rc;
                if ((rc = make_map_2d(&tmV, V, plan.kv_rows_extent, shape->d, kChunkTileN)) != YOCO_OK) return rc;
            }
            ChunkParams p{};
            p.O = static_cast<__nv_bfloat16*>(O);
            p.lse = lse;
            p.segments = reinterpret_cast<const DevSegment*>(table + plan.off_segments);
            p.group_begin = table + plan.off_group_begin;
            p.part_o = part_o;
            p.part_lse = part_lse;
            p.status = status;
            p.scale_log2 = scale * 1.4426950408889634f;
            p.T = shape->T;
            p.rows_per_stream = plan.rows_per_stream;
            p.m_tiles = plan.info.m_tiles;
            p.d = shape->d;
            p.window = shape->window;
            p.force_partial = part_out ? 1 : 0;
            if (paged) p.pages = paged->pages;
            if (four_bit) {
                YOCO_CUDA_TRY(launch_chunk_pair_q4(p, tmQ, q4, plan.info.num_groups, stream));
            } else if (fp8) {
                ChunkFp8Scales cs{};
                cs.Hkv = shape->Hkv;
                for (int c = 0; c < shape->Hkv; ++c) {
                    cs.score_scale_log2[c] = scale * fp8->k_scale[c] * 1.4426950408889634f;
                    cs.v_scale[c] = fp8->v_scale[c];
                }
                YOCO_CUDA_TRY(launch_chunk_pair(p, tmQ, tmK, tmV, plan.info.num_groups, stream, &cs));
            } else if (plan.info.tile_m == kChunkPairTileM)
                YOCO_CUDA_TRY(launch_chunk_pair(p, tmQ, tmK, tmV, plan.info.num_groups, stream, nullptr, paged != nullptr));
            else
                YOCO_CUDA_TRY(launch_chunk(p, tmQ, tmK, tmV, plan.info.num_groups, stream, paged != nullptr));
        }
        if (prof) {
            ev = prof_event(true, &prof);
            if (prof) YOCO_CUDA_TRY(cudaEventRecord(ev, stream));
        }
    }
    if (plan.info.needs_combine || part_out) {
        CombineParams c{};
        c.rows = (int64_t)shape->B * shape->Hq * shape->T;
        c.d = shape->d;
        c.S = 0;
        c.Hq = shape->Hq;
        c.Hkv = shape->Hkv;
        c.T = shape->T;
        c.rows_per_stream = plan.rows_per_stream;
        c.max_pieces = plan.info.max_splits;
        c.sub_items = plan.sub_items;
        c.stream_base = table + plan.off_stream_base;
        c.stream_nseg = table + plan.off_stream_nseg;
        c.part_o = part_o;
        c.part_lse = part_lse;
        c.O = part_out ? nullptr : static_cast<__nv_bfloat16*>(O);
        c.lse = lse;
        c.O_f32 = part_out;
        c.merge_unsplit = part_out ? 1 : 0;
        // directly behind the attention kernel (no event in between): its launch may overlap
        // that kernel's tail
        const bool chained = plan.info.num_segments > 0 && !timed;
        YOCO_CUDA_TRY(launch_combine(c, stream, inline_tables ? &ready->combine_tab : nullptr, chained, paged != nullptr));
    }
    return YOCO_OK;
}


// ---- built-in scratch for callers that cannot allocate -------------------------------------
// Lives in every GPU that loads this library until the process exits.  In host code the
// name below is only a handle; the device address comes from cudaGetSymbolAddress.
constexpr size_t kStaticScratchBytes = 4u << 20;
static __device__ __align__(256) unsigned char g_static_scratch[kStaticScratchBytes];
void* g_static_scratch_addr[kMaxDevices] = {};

int32_t static_scratch_address(void** out) {
    int dev = 0;
    YOCO_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return YOCO_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_mutex);
    if (!g_static_scratch_addr[dev]) {
        void* ptr = nullptr;
        YOCO_CUDA_TRY(cudaGetSymbolAddress(&ptr, g_static_scratch));   // address on the current device
        if (!ptr) return cuda_fail(cudaErrorInvalidSymbol);
        g_static_scratch_addr[dev] = ptr;
    }
    *out = g_static_scratch_addr[dev];
    return YOCO_OK;
}

// ---- paged cache ---------------------------------------------------------------------------
// Runs a call that allocates host memory (plans, tables) without letting an exception through the C boundary.
template <class F>
int32_t no_throw(F f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return YOCO_ERR_HOST_MEMORY;
    } catch (...) {
        return YOCO_ERR_INVALID_ARG;
    }
}

// Longest sequence, and most rows of one append or gather: key numbers a little past the end stay 32-bit integers.
constexpr int64_t kMaxPagedLen = 1ll << 30;

bool valid_page_size(int32_t P) { return P == 16 || P == 32 || P == 64 || P == 128 || P == 256; }

// Checks the layout against the lengths of a call (kv_len_host null: every N_i = max_kv_len) and fills the map.
int32_t page_map(const yoco_paged_layout* layout, int32_t B, int32_t Hkv, const int32_t* kv_len_host, int32_t max_kv_len,
                 const int32_t* page_table, PageMap* out) {
    if (!layout) return YOCO_ERR_INVALID_ARG;
    const yoco_paged_layout& L = *layout;
    if (L.num_pages <= 0 || L.table_stride < 0 || L.page_rows < 0 || (L.rope_pairs != 0 && L.rope_pairs != 1) || Hkv <= 0 || B < 0)
        return YOCO_ERR_INVALID_ARG;
    if (!valid_page_size(L.page_size)) return YOCO_ERR_UNSUPPORTED;
    const int64_t tight = (int64_t)Hkv * L.page_size;
    const int64_t page_rows = L.page_rows ? L.page_rows : tight;
    if (page_rows < tight) return YOCO_ERR_INVALID_ARG;
    // row numbers are 32-bit, and the scale rows of a 4-bit pool are read sixteen at a time
    if (page_rows % 16 != 0 || page_rows > (1ll << 31) / L.num_pages - 1) return YOCO_ERR_UNSUPPORTED;
    if (!page_table || !aligned(page_table, 4)) return YOCO_ERR_INVALID_ARG;
    for (int32_t i = 0; i < B; ++i) {
        const int64_t n = kv_len_host ? kv_len_host[i] : max_kv_len;
        if (n < 0 || (n + L.page_size - 1) / L.page_size > L.table_stride) return YOCO_ERR_INVALID_ARG;
        if (n > kMaxPagedLen) return YOCO_ERR_UNSUPPORTED;
    }
    int shift = 4;
    while ((1 << shift) < L.page_size) ++shift;
    *out = PageMap{page_table, L.table_stride, shift, L.num_pages, (int32_t)page_rows, Hkv,
                   (int32_t)((int64_t)(L.num_pages - 1) * page_rows + tight)};
    return YOCO_OK;
}

int32_t attend_paged(int32_t mode, const yoco_xattn_shape* shape, const yoco_paged_layout* layout, const void* Q,
                     const void* K, const void* k_scale, const void* V, const void* v_scale, bool q4,
                     const int32_t* page_table, const int32_t* kv_len_host, void* O, float* lse, void* workspace,
                     size_t workspace_bytes, void* stream, const SelfTest* selftest = nullptr) {
    return no_throw([&]() -> int32_t {
        if (!shape) return YOCO_ERR_INVALID_ARG;
        int32_t rc = validate_shape(*shape, mode);
        if (rc != YOCO_OK) return rc;
        if (shape->kv_head_stride != 0) return YOCO_ERR_INVALID_ARG;
        if (q4 && shape->d != 128) return YOCO_ERR_UNSUPPORTED;
        if (shape->B == 0) return YOCO_OK;
        PagedCall pc{};
        if ((rc = page_map(layout, shape->B, shape->Hkv, kv_len_host, shape->max_kv_len, page_table, &pc.pages)) != YOCO_OK)
            return rc;
        if (q4 && (!k_scale || !v_scale || !aligned(k_scale, 16) || !aligned(v_scale, 16))) return YOCO_ERR_INVALID_ARG;
        pc.k_scale = q4 ? k_scale : nullptr;
        pc.v_scale = q4 ? v_scale : nullptr;
        return run(shape, mode, Q, K, V, nullptr, kv_len_host, O, lse, workspace, workspace_bytes, stream, nullptr,
                   nullptr, selftest ? 1 : kMaxSubItems, selftest, nullptr, &pc);
    });
}

// What append, gather and rope_q share: first positions and tokens of every sequence.  begin/end: positions of
// sequence i are [begin(i), end(i)).
template <class Begin, class End>
int32_t sequence_table(int32_t B, Begin begin, End end, SeqTable* tab, int64_t* tokens, int32_t* per_seq) {
    if (B > kAppendMaxSequences) return YOCO_ERR_UNSUPPORTED;
    std::memset(tab, 0, sizeof *tab);
    *tokens = 0;
    *per_seq = B > 0 ? end(0) - begin(0) : 0;
    for (int32_t i = 0; i < B; ++i) {
        const int64_t lo = begin(i), hi = end(i);
        if (lo < 0 || hi < lo) return YOCO_ERR_INVALID_ARG;
        tab->pos0[i] = (int32_t)lo;
        tab->tok0[i] = (int32_t)*tokens;
        *tokens += hi - lo;
        if (*tokens > kMaxPagedLen) return YOCO_ERR_UNSUPPORTED;
        if (hi - lo != *per_seq) *per_seq = 0;
    }
    tab->tok0[B] = (int32_t)*tokens;
    return YOCO_OK;
}

int32_t check_rotation(const yoco_paged_layout& L, int64_t max_len, Rotation* rot) {
    if (L.cos_sin) {
        if (!aligned(L.cos_sin, 16) || L.max_pos < max_len) return YOCO_ERR_INVALID_ARG;
        *rot = Rotation{L.cos_sin, L.rope_pairs};
    } else {
        *rot = Rotation{nullptr, 0};
    }
    return YOCO_OK;
}

int32_t paged_rows(const yoco_paged_append_shape* shape, const yoco_paged_layout* layout, bool append, bool q4,
                   const void* k_new, const void* v_new, const void* K, const void* k_scale, const void* V,
                   const void* v_scale, const int32_t* page_table, const int32_t* begin_host, const int32_t* end_host,
                   const int32_t* new_len_host, void* k_out, void* v_out, void* stream) {
    return no_throw([&]() -> int32_t {
        if (!shape) return YOCO_ERR_INVALID_ARG;
        const yoco_paged_append_shape& s = *shape;
        if (s.B < 0 || s.Hkv <= 0 || s.d <= 0 || s.T < 0 || s.src_stride < 0) return YOCO_ERR_INVALID_ARG;
        if ((s.d != 64 && s.d != 128) || (q4 && s.d != 128) || s.B > kAppendMaxSequences) return YOCO_ERR_UNSUPPORTED;
        if (s.B == 0) return YOCO_OK;
        if (!end_host || (!append && !begin_host)) return YOCO_ERR_INVALID_ARG;
        PagedRowsParams p{};
        int32_t rc = page_map(layout, s.B, s.Hkv, end_host, 0, page_table, &p.pages);
        if (rc != YOCO_OK) return rc;
        if (!K || !V || !aligned(K, 16) || !aligned(V, 16)) return YOCO_ERR_INVALID_ARG;
        if (q4 && (!k_scale || !v_scale || !aligned(k_scale, 16) || !aligned(v_scale, 16))) return YOCO_ERR_INVALID_ARG;
        if (append) {
            if (!aligned(k_new, 16) || !aligned(v_new, 16)) return YOCO_ERR_INVALID_ARG;
            p.src_stride = s.src_stride ? s.src_stride : (int64_t)s.Hkv * s.d;
            if (p.src_stride < (int64_t)s.Hkv * s.d) return YOCO_ERR_INVALID_ARG;
            if (p.src_stride % 8 != 0) return YOCO_ERR_UNSUPPORTED;
            if (new_len_host)
                for (int32_t i = 0; i < s.B; ++i)
                    if (new_len_host[i] < 0) return YOCO_ERR_INVALID_ARG;
        } else if (!aligned(k_out, 16) || !aligned(v_out, 16)) {
            return YOCO_ERR_INVALID_ARG;
        }
        SeqTable tab;
        int64_t tokens = 0;
        rc = sequence_table(
            s.B,
            [&](int32_t i) -> int64_t {
                return append ? (int64_t)end_host[i] - (new_len_host ? new_len_host[i] : s.T) : begin_host[i];
            },
            [&](int32_t i) -> int64_t { return end_host[i]; }, &tab, &tokens, &p.tokens_per_seq);
        if (rc != YOCO_OK) return rc;
        if (s.Hkv > 65535) return YOCO_ERR_UNSUPPORTED;      // a grid dimension
        if (append) {
            int64_t max_len = 0;
            for (int32_t i = 0; i < s.B; ++i) max_len = std::max<int64_t>(max_len, end_host[i]);
            if ((rc = check_rotation(*layout, max_len, &p.rot)) != YOCO_OK) return rc;
        }
        if (tokens == 0) return YOCO_OK;             // (an empty tensor's address may be null)
        if (append ? !k_new || !v_new : !k_out || !v_out) return YOCO_ERR_INVALID_ARG;
        DeviceState* dev = nullptr;
        if ((rc = device_state(&dev)) != YOCO_OK) return rc;
        p.k_src = static_cast<const __nv_bfloat16*>(k_new);
        p.v_src = static_cast<const __nv_bfloat16*>(v_new);
        p.k_pool = const_cast<void*>(K);
        p.v_pool = const_cast<void*>(V);
        p.k_scale = static_cast<__half*>(const_cast<void*>(k_scale));
        p.v_scale = static_cast<__half*>(const_cast<void*>(v_scale));
        p.k_out = static_cast<__nv_bfloat16*>(k_out);
        p.v_out = static_cast<__nv_bfloat16*>(v_out);
        p.status = dev->append_status;
        p.B = s.B;
        p.d = s.d;
        p.tokens = (int32_t)tokens;
        cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
        YOCO_CUDA_TRY(append ? launch_paged_append(p, tab, q4, st) : launch_paged_gather(p, tab, q4, st));
        return YOCO_OK;
    });
}

// ---- self-decoder: gated retention, head norm, rotation ---------------------------------------------
// Rows of `width` elements, `stride` (0: width) apart.
int32_t check_rows(const void* ptr, int64_t* stride, int64_t width) {
    if (*stride == 0) *stride = width;
    if (*stride < width || !aligned(ptr, 16)) return YOCO_ERR_INVALID_ARG;
    return *stride % 8 == 0 ? YOCO_OK : YOCO_ERR_UNSUPPORTED;
}

// n rows of `bytes` bytes, `stride` bytes apart.
struct Rows {
    const void* ptr;
    int64_t stride, bytes, n;
    // whether any row touches the bytes [lo, hi)
    bool touch(uintptr_t lo, uintptr_t hi) const {
        const uintptr_t at = (uintptr_t)ptr;
        const int64_t first = lo >= at + bytes ? (int64_t)((lo - at - bytes) / stride) + 1 : 0;      // that ends behind lo
        return first < n && at + first * stride < hi;
    }
    uintptr_t begin() const { return (uintptr_t)ptr; }
    uintptr_t end_of_first() const { return begin() + (stride == bytes ? n : 1) * bytes; }           // rows without gaps: of all
};
// Whether two sets of rows overlap; exact for rows of one distance (an overlap recurs from row to row) and where one set has no gaps.  Slices of one
// buffer that lie beside one another do not.
bool overlap(const Rows& a, const Rows& b) {
    return a.ptr && b.ptr && a.n > 0 && b.n > 0 && (a.touch(b.begin(), b.end_of_first()) || b.touch(a.begin(), a.end_of_first()));
}

int32_t check_norm(const yoco_norm_gate* norm, int64_t width, NormGate* out) {
    *out = NormGate{};
    if (!norm) return YOCO_OK;
    if (!(norm->eps >= 0.f) || !std::isfinite(norm->eps) || (norm->rms & ~1) || norm->gate_stride < 0) return YOCO_ERR_INVALID_ARG;
    int64_t stride = norm->gate_stride;
    const int32_t rc = check_rows(norm->gate, &stride, width);
    if (rc != YOCO_OK) return rc;
    if (!aligned(norm->gain, 16) || !aligned(norm->bias, 16)) return YOCO_ERR_INVALID_ARG;
    *out = NormGate{static_cast<const __nv_bfloat16*>(norm->gate), static_cast<const __nv_bfloat16*>(norm->gain),
                    static_cast<const __nv_bfloat16*>(norm->bias), stride, norm->eps, norm->rms, 1};
    return YOCO_OK;
}

// Tokens of every sequence; *tokens: their sum.
int32_t check_lengths(int32_t B, const int32_t* len_host, int32_t T, int64_t* tokens) {
    if (!len_host && T < 0) return YOCO_ERR_INVALID_ARG;
    *tokens = 0;
    for (int32_t i = 0; i < B; ++i) {
        const int64_t n = len_host ? len_host[i] : T;
        if (n < 0) return YOCO_ERR_INVALID_ARG;
        *tokens += n;
    }
    return *tokens > kMaxPagedLen ? YOCO_ERR_UNSUPPORTED : YOCO_OK;
}

int32_t check_gret_shape(const yoco_gret_shape& s) {
    if (s.B < 0 || s.H <= 0 || s.d <= 0 || !(s.scale >= 0.f) || !std::isfinite(s.scale) || !(s.tau >= 0.f) || !std::isfinite(s.tau) || (s.tau > 0.f && !std::isfinite(1.f / s.tau)) ||
        (s.decay_bf16 & ~1) || s.q_stride < 0 || s.k_stride < 0 || s.v_stride < 0 || s.o_stride < 0 || s.decay_stride < 0)
        return YOCO_ERR_INVALID_ARG;
    return (s.d == 64 || s.d == 128) && s.H <= 65535 && s.B <= kAppendMaxSequences ? YOCO_OK : YOCO_ERR_UNSUPPORTED;
}

// Slots of the states: in range, none written twice, none written that another sequence reads.
int32_t check_slots(const yoco_gret_shape& s, const int32_t* in, const int32_t* out, GretTable* tab) {
    if (s.num_slots <= 0) return YOCO_ERR_INVALID_ARG;
    for (int32_t i = 0; i < s.B; ++i) {
        tab->from[i] = in ? in[i] : i;
        tab->to[i] = out ? out[i] : i;
        if (tab->from[i] < -1 || tab->from[i] >= s.num_slots || tab->to[i] < -1 || tab->to[i] >= s.num_slots) return YOCO_ERR_INVALID_ARG;
    }
    // One sequence may write a slot; only that one may read it then.  A bit per slot for pools of usual sizes, a sorted list beyond.
    constexpr int32_t kBits = 8192;
    uint64_t bits[kBits / 64];
    std::vector<int32_t> sorted;
    const bool few = s.num_slots <= kBits;
    if (few) {
        std::memset(bits, 0, (size_t)(s.num_slots + 63) / 64 * 8);
        for (int32_t i = 0; i < s.B; ++i) {
            if (tab->to[i] < 0) continue;
            uint64_t& w = bits[tab->to[i] / 64];
            const uint64_t bit = 1ull << (tab->to[i] % 64);
            if (w & bit) return YOCO_ERR_INVALID_ARG;
            w |= bit;
        }
    } else {
        for (int32_t i = 0; i < s.B; ++i)
            if (tab->to[i] >= 0) sorted.push_back(tab->to[i]);
        std::sort(sorted.begin(), sorted.end());
        if (std::adjacent_find(sorted.begin(), sorted.end()) != sorted.end()) return YOCO_ERR_INVALID_ARG;
    }
    for (int32_t i = 0; i < s.B; ++i) {
        const int32_t f = tab->from[i];
        if (f < 0 || f == tab->to[i]) continue;
        if (few ? (bits[f / 64] >> (f % 64) & 1) != 0 : std::binary_search(sorted.begin(), sorted.end(), f)) return YOCO_ERR_INVALID_ARG;
    }
    return YOCO_OK;
}

// Calls whose sequences all have no more tokens than this walk them one by one (one CTA per head, state in registers); longer ones in chunks.
// (Measured in recorded graphs, 32 heads, us token by token / in chunks.  Heads of 128, where the border was set: one sequence of 16, 18, 20 tokens
// 9.8 / 11.1, 11.3 / 11.1, 11.9 / 11.1; eight 16.2 / 20.1, 18.0 / 20.0, 19.0 / 20.1; 32 sequences of 12, 16, 18 tokens 48 / 60, 59 / 61, 68 / 61.  Heads of 64
// would have it higher: one sequence of 20, 24, 32 tokens 6.9 / 8.2, 7.4 / 8.2, 9.3 / 8.1; eight 8.6 / 13.5, 9.1 / 13.6, 11.5 / 13.5; 32
// sequences 20 / 35, 22 / 35, 29 / 35.)
constexpr int32_t kGretTokens = 18;
// Costs in chunks of a whole stream (heads of 128: 3.3 us; of 64: 2.8): a chunk in both passes over split streams; the extra launches with their starts
// and ends; every further segment of a CTA, whose state comes and goes.  Set by heads of 128 and used for both.  (Measured in recorded graphs, us whole / split,
// one sequence.  Heads of 128: 512 tokens, 8 / 16 / 32 heads 20.4 / 18.6, 20.8 / 18.9, 21.1 / 23.1, all taken whole; 768: 27.1 / 19.1, 27.3 / 20.6
// split, 27.6 / 28.2 whole; 896, 32 heads 31.0 / 32.9 whole; 1,024: 33.7 / 19.5, 33.8 / 22.9, 34.5 / 29.6 split.  Six sequences of 37 to 1,501 tokens, 16 heads
// 49.9 / 64.5 whole.  Heads of 64: 512 tokens 16.0 / 12.6, 16.1 / 13.6, 16.3 / 17.4 whole; 768 21.5 / 13.3, 21.6 / 14.9 split, 21.8 / 21.0 whole; 896, 32 heads
// 24.7 / 22.5 whole; 1,024 split, 26.9 / 13.7, 27.2 / 16.4, 27.5 / 22.8; the six sequences 38.3 / 42.9 whole.  So the rule keeps a few short
// streams whole where a split would take 1 to 3.5 us off: 512 tokens of 8 and 16 heads, and of 32 heads of 64 768 and 896 tokens.)
constexpr double kGretSplitChunk = 1.4, kGretSplitCost = 4.0, kGretSegmentCost = 1.0;

struct GretPlan {
    GretChunkTable tab;
    int32_t seqs;               // sequences in tab
    int64_t total;              // chunks of all heads
    int32_t groups, split;
    size_t part_bytes;          // workspace: parts' states, then their decays
    void set_groups(int32_t n, int32_t d) {
        groups = n;
        part_bytes = (size_t)3 * n * d * d * sizeof(float);
    }
    size_t bytes() const { return split ? part_bytes + (size_t)3 * groups * sizeof(float) : 0; }
};

// Whole streams, dealt out to the CTAs (longest first), or equal ranges of chunks that cut streams: the latter pay a second pass over K and V.
void plan_gret(const yoco_gret_shape& s, const int32_t* len_host, const GretTable* slots, int32_t sm_count, GretPlan* out) {
    std::memset(&out->tab, 0, sizeof out->tab);
    std::vector<std::pair<int32_t, int32_t>> order;        // (-length, sequence)
    std::vector<int32_t> tok0(s.B + 1, 0);
    for (int32_t i = 0; i < s.B; ++i) {
        const int32_t n = len_host ? len_host[i] : s.T;
        tok0[i + 1] = tok0[i] + n;
        if (n > 0) order.emplace_back(-n, i);
    }
    std::stable_sort(order.begin(), order.end());
    out->seqs = (int32_t)order.size();
    for (int32_t j = 0; j < out->seqs; ++j) {
        const int32_t i = order[j].second;
        out->tab.tok0[j] = tok0[i];
        out->tab.len[j] = -order[j].first;
        out->tab.from[j] = slots ? slots->from[i] : -1;
        out->tab.to[j] = slots ? slots->to[i] : -1;
        out->tab.chunk0[j + 1] = out->tab.chunk0[j] + (out->tab.len[j] + kGretChunk - 1) / kGretChunk;
    }
    for (int32_t j = out->seqs; j < kAppendMaxSequences; ++j) out->tab.chunk0[j + 1] = out->tab.chunk0[out->seqs];
    out->total = (int64_t)out->tab.chunk0[out->seqs] * s.H;
    const int64_t streams = (int64_t)out->seqs * s.H;
    // time of whole streams, dealt out longest first: the longest of every round
    double whole = -kGretSegmentCost;
    for (int64_t first = 0; first < streams; first += sm_count)
        whole += out->tab.chunk0[first / s.H + 1] - out->tab.chunk0[first / s.H] + kGretSegmentCost;
    // time of equal shares: the last one, of the shortest streams, has the most segments
    const int64_t cut = std::min<int64_t>(out->total, sm_count);
    const double share = cut > 0 ? (double)((out->total + cut - 1) / cut) : 0.0;
    const double segments = out->seqs > 0 ? share / (out->tab.chunk0[out->seqs] - out->tab.chunk0[out->seqs - 1]) : 0.0;
    out->split = cut > 1 && share * kGretSplitChunk + kGretSplitCost + segments * kGretSegmentCost < whole;
    out->set_groups((int32_t)(out->split ? cut : std::min<int64_t>(streams, sm_count)), s.d);
}

// Workspace bytes of calls with these lengths, or with lengths up to these: none where all sequences are walked token by token.
template <class F>
int32_t gret_workspace(const yoco_gret_shape* shape, const int32_t* len_host, int32_t sm_count, size_t* bytes, F of_chunks) {
    return no_throw([&]() -> int32_t {
        if (!shape || !bytes) return YOCO_ERR_INVALID_ARG;
        int64_t tokens = 0;
        int32_t rc = check_gret_shape(*shape);
        if (rc != YOCO_OK || (rc = check_lengths(shape->B, len_host, shape->T, &tokens)) != YOCO_OK) return rc;
        int32_t longest = 0;
        for (int32_t i = 0; i < shape->B; ++i) longest = std::max(longest, len_host ? len_host[i] : shape->T);
        *bytes = 0;
        if (longest <= kGretTokens) return YOCO_OK;
        if (sm_count <= 0) {
            DeviceState* dev = nullptr;
            if ((rc = device_state(&dev)) != YOCO_OK) return rc;
            sm_count = dev->sm_count;
        }
        *bytes = of_chunks(sm_count);
        return YOCO_OK;
    });
}

int32_t gret(const yoco_gret_shape* shape, const void* Q, const void* K, const void* V, const void* decay, const yoco_norm_gate* norm,
             float* state, const int32_t* slot_in_host, const int32_t* slot_out_host, const int32_t* len_host, bool step, void* O,
             void* workspace, size_t workspace_bytes, void* stream, const SelfTest* selftest = nullptr) {
    return no_throw([&]() -> int32_t {
        if (!shape) return YOCO_ERR_INVALID_ARG;
        const yoco_gret_shape& s = *shape;
        int32_t rc = check_gret_shape(s);
        if (rc != YOCO_OK) return rc;
        if (s.B == 0) return YOCO_OK;
        const int64_t width = (int64_t)s.H * s.d;
        GretParams p{};
        int64_t tokens = 0;
        if ((rc = check_lengths(s.B, len_host, step ? 1 : s.T, &tokens)) != YOCO_OK) return rc;
        p.q_stride = s.q_stride;
        p.k_stride = s.k_stride;
        p.v_stride = s.v_stride;
        p.o_stride = s.o_stride;
        p.decay_stride = s.decay_stride ? s.decay_stride : s.H;
        if ((rc = check_rows(Q, &p.q_stride, width)) != YOCO_OK || (rc = check_rows(K, &p.k_stride, width)) != YOCO_OK ||
            (rc = check_rows(V, &p.v_stride, width)) != YOCO_OK || (rc = check_rows(O, &p.o_stride, width)) != YOCO_OK ||
            (rc = check_norm(norm, width, &p.norm)) != YOCO_OK)
            return rc;
        if (p.decay_stride < s.H || !aligned(decay, s.decay_bf16 ? 2 : 4) || !state || !aligned(state, 16)) return YOCO_ERR_INVALID_ARG;
        if (tokens > 0 && (!Q || !K || !V || !decay || !O)) return YOCO_ERR_INVALID_ARG;   // (an empty tensor's address may be null)
        GretTable tab;                                     // (entries behind the last sequence are not read)
        tab.tok0[0] = 0;
        if ((rc = check_slots(s, slot_in_host, slot_out_host, &tab)) != YOCO_OK) return rc;
        for (int32_t i = 0; i < s.B; ++i) tab.tok0[i + 1] = tab.tok0[i] + (len_host ? len_host[i] : step ? 1 : s.T);
        DeviceState* dev = nullptr;
        if ((rc = device_state(&dev)) != YOCO_OK) return rc;
        const auto rows = [&](const void* ptr, int64_t stride) { return Rows{ptr, stride * 2, width * 2, tokens}; };
        const Rows out = rows(O, p.o_stride);
        const int64_t decay_bytes = s.decay_bf16 ? 2 : 4;
        if (overlap(out, rows(Q, p.q_stride)) || overlap(out, rows(K, p.k_stride)) || overlap(out, rows(V, p.v_stride)) ||
            overlap(out, rows(p.norm.gate, p.norm.gate_stride)) || overlap(out, Rows{decay, p.decay_stride * decay_bytes, s.H * decay_bytes, tokens}))
            return YOCO_ERR_INVALID_ARG;
        p.q = static_cast<const __nv_bfloat16*>(Q);
        p.k = static_cast<const __nv_bfloat16*>(K);
        p.v = static_cast<const __nv_bfloat16*>(V);
        p.o = static_cast<__nv_bfloat16*>(O);
        p.decay = decay;
        p.state = state;
        p.scale = s.scale > 0.f ? s.scale : 1.f / std::sqrt((float)s.d);
        p.inv_tau = s.tau > 0.f ? 1.f / s.tau : 0.f;
        p.decay_bf16 = s.decay_bf16;
        p.B = s.B;
        p.H = s.H;
        p.d = s.d;
        cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
        int32_t longest = 0;
        for (int32_t i = 0; i < s.B; ++i) longest = std::max(longest, tab.tok0[i + 1] - tab.tok0[i]);
        if (longest <= kGretTokens) {
            if (selftest) return YOCO_ERR_UNSUPPORTED;     // (no waits there)
            YOCO_CUDA_TRY(launch_gret_tokens(p, tab, st));
            return YOCO_OK;
        }
        GretPlan plan;
        plan_gret(s, len_host, &tab, dev->sm_count, &plan);
        if (plan.total > INT32_MAX) return YOCO_ERR_UNSUPPORTED;
        if (plan.bytes() > 0) {
            if (!workspace || !aligned(workspace, 16)) return YOCO_ERR_INVALID_ARG;
            if (workspace_bytes < plan.bytes()) return YOCO_ERR_WORKSPACE_TOO_SMALL;
        }
        CUtensorMap tmQ, tmK, tmV;
        auto map = [&](CUtensorMap* m, const void* base, int64_t stride, int32_t rows) {
            return make_map(m, base, tokens, (int32_t)(width * 2), 128, rows, true, CU_TENSOR_MAP_SWIZZLE_128B, stride * 2);
        };
        if ((rc = map(&tmQ, Q, p.q_stride, kGretChunk)) != YOCO_OK || (rc = map(&tmK, K, p.k_stride, kGretChunk / 2)) != YOCO_OK ||
            (rc = map(&tmV, V, p.v_stride, kGretChunk / 2)) != YOCO_OK)
            return rc;
        GretChunkParams cp{};
        cp.base = p;
        cp.base.B = plan.seqs;
        cp.total = (int32_t)plan.total;
        cp.groups = plan.groups;
        cp.split = plan.split;
        cp.share = cp.total / cp.groups;
        cp.extra = cp.total % cp.groups;
        cp.part = static_cast<float*>(workspace);
        cp.part_keep = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + plan.part_bytes);
        cp.status = dev->append_status;
        cp.wait_limit_ns = selftest ? (int32_t)selftest->wait_limit_ns : 0;
        cp.selftest_skip_loads = selftest ? 1 : 0;
        if (plan.seqs < s.B) {           // sequences without tokens hand their states on
            GretTable idle;
            std::memset(&idle, 0, sizeof idle);
            GretParams ip = p;
            ip.B = 0;
            for (int32_t i = 0; i < s.B; ++i) {
                if (tab.tok0[i + 1] > tab.tok0[i] || tab.to[i] < 0 || tab.to[i] == tab.from[i]) continue;
                idle.from[ip.B] = tab.from[i];
                idle.to[ip.B++] = tab.to[i];
            }
            YOCO_CUDA_TRY(launch_gret_tokens(ip, idle, st));
        }
        YOCO_CUDA_TRY(launch_gret_chunk(cp, plan.tab, tmQ, tmK, tmV, st));
        return YOCO_OK;
    });
}

}  // namespace
}  // namespace yoco

using namespace yoco;

extern "C" {

int32_t yoco_xattn_plan(const yoco_xattn_shape* shape, const int32_t* kv_len_host, int32_t sm_count,
                        int32_t mode, yoco_xattn_plan_info* info, yoco_xattn_segment* segments_out,
                        int32_t capacity) {
    return yoco_xattn_plan_at(shape, kv_len_host, nullptr, nullptr, sm_count, mode, info, segments_out, capacity);
}

int32_t yoco_xattn_plan_at(const yoco_xattn_shape* shape, const int32_t* kv_len_host, const int32_t* key_offset_host,
                           const int32_t* kv_total_host, int32_t sm_count, int32_t mode, yoco_xattn_plan_info* info,
                           yoco_xattn_segment* segments_out, int32_t capacity) {
    if (!shape || !info || capacity < 0 || (capacity > 0 && !segments_out)) return YOCO_ERR_INVALID_ARG;
    Plan plan;
    int32_t rc = make_plan(*shape, nullptr, kv_len_host, sm_count, mode, plan, kMaxSubItems, key_offset_host,
                           kv_total_host);
    if (rc != YOCO_OK) return rc;
    *info = plan.info;
    const int32_t n = std::min<int32_t>(capacity, (int32_t)plan.segments.size());
    for (int32_t k = 0; k < n; ++k) segments_out[k] = plan.segments[k];
    return YOCO_OK;
}

int64_t yoco_xattn_sub_bound(int64_t n_tiles, int32_t sub_items, int32_t r) {
    if (n_tiles < 0 || (sub_items != 1 && sub_items != 2 && sub_items != 4)) return -1;
    return sub_bound(n_tiles, sub_items, r);
}

int32_t yoco_xattn_workspace_size(const yoco_xattn_shape* shape, const int32_t* kv_len_host,
                                  int32_t sm_count, int32_t mode, size_t* bytes) {
    return yoco_xattn_workspace_size_at(shape, kv_len_host, nullptr, nullptr, sm_count, mode, bytes);
}

int32_t yoco_xattn_workspace_size_at(const yoco_xattn_shape* shape, const int32_t* kv_len_host,
                                     const int32_t* key_offset_host, const int32_t* kv_total_host,
                                     int32_t sm_count, int32_t mode, size_t* bytes) {
    if (!shape || !bytes || sm_count < 0) return YOCO_ERR_INVALID_ARG;
    if (sm_count == 0) {
        int32_t rc = validate_shape(*shape, mode);
        if (rc != YOCO_OK) return rc;
        DeviceState* dev = nullptr;
        if ((rc = device_state(&dev)) != YOCO_OK) return rc;
        sm_count = dev->sm_count;
    }
    Plan plan;
    int32_t rc = make_plan(*shape, nullptr, kv_len_host, sm_count, mode, plan, kMaxSubItems, key_offset_host,
                           kv_total_host);
    if (rc != YOCO_OK) return rc;
    *bytes = (size_t)plan.info.workspace_bytes;
    return YOCO_OK;
}

int32_t yoco_xattn_decode(const yoco_xattn_shape* shape, const void* Q, const void* K, const void* V,
                          const int32_t* cu_kv_host, const int32_t* kv_len_host, void* O, float* lse,
                          void* workspace, size_t workspace_bytes, void* stream) {
    return run(shape, YOCO_MODE_DECODE, Q, K, V, cu_kv_host, kv_len_host, O, lse, workspace,
               workspace_bytes, stream);
}

int32_t yoco_xattn_decode_static(const yoco_xattn_shape* shape, const void* Q, const void* K,
                                 const void* V, const int32_t* cu_kv_host, const int32_t* kv_len_host,
                                 void* O, float* lse, void* stream) {
    if (!shape) return YOCO_ERR_INVALID_ARG;
    int32_t rc = validate_shape(*shape, YOCO_MODE_DECODE);
    if (rc != YOCO_OK) return rc;
    if (shape->B == 0) return YOCO_OK;
    // size check first, on the host: nothing is enqueued for a problem that does not fit
    DeviceState* dev = nullptr;
    if ((rc = device_state(&dev)) != YOCO_OK) return rc;
    // one piece per group: the fixed buffer is sized for that
    std::shared_ptr<const ReadyPlan> ready;
    if ((rc = cached_plan(*shape, cu_kv_host, kv_len_host, dev->sm_count, YOCO_MODE_DECODE, 1, ready)) != YOCO_OK)
        return rc;
    if ((size_t)ready->plan.info.workspace_bytes > kStaticScratchBytes) return YOCO_ERR_STATIC_SCRATCH_EXCEEDED;
    void* scratch = nullptr;
    if ((rc = static_scratch_address(&scratch)) != YOCO_OK) return rc;
    return run(shape, YOCO_MODE_DECODE, Q, K, V, cu_kv_host, kv_len_host, O, lse, scratch,
               kStaticScratchBytes, stream, nullptr, nullptr, 1);
}

int32_t yoco_xattn_static_scratch_bytes(void) { return (int32_t)kStaticScratchBytes; }

int32_t yoco_xattn_chunk(const yoco_xattn_shape* shape, const void* Q, const void* K, const void* V,
                         const int32_t* cu_kv_host, const int32_t* kv_len_host, void* O, float* lse,
                         void* workspace, size_t workspace_bytes, void* stream) {
    return run(shape, YOCO_MODE_CHUNK, Q, K, V, cu_kv_host, kv_len_host, O, lse, workspace,
               workspace_bytes, stream);
}

namespace {
int32_t combine_public(int64_t rows, int32_t S, int32_t d, const float* part_o, const float* part_lse, void* O,
                       float* lse, void* stream, int32_t piece_major) {
    if (rows < 0 || S <= 0 || d <= 0) return YOCO_ERR_INVALID_ARG;
    if (d % 8 != 0 || d > 256) return YOCO_ERR_UNSUPPORTED;
    if (rows == 0) return YOCO_OK;
    if (!part_o || !part_lse || !O) return YOCO_ERR_INVALID_ARG;
    if (!aligned(part_o, 16) || !aligned(part_lse, 4) || !aligned(O, 16)) return YOCO_ERR_INVALID_ARG;
    CombineParams c{};
    c.rows = rows;
    c.d = d;
    c.S = S;
    c.max_pieces = S;
    c.stream_base = nullptr;
    c.stream_nseg = nullptr;
    c.part_o = part_o;
    c.part_lse = part_lse;
    c.O = static_cast<__nv_bfloat16*>(O);
    c.lse = lse;
    c.piece_major = piece_major;
    YOCO_CUDA_TRY(launch_combine(c, reinterpret_cast<cudaStream_t>(stream)));
    return YOCO_OK;
}
}  // namespace

int32_t yoco_xattn_combine(int64_t rows, int32_t S, int32_t d, const float* part_o,
                           const float* part_lse, void* O, float* lse, void* stream) {
    return combine_public(rows, S, d, part_o, part_lse, O, lse, stream, 0);
}

int32_t yoco_xattn_combine_gathered(int64_t rows, int32_t S, int32_t d, const float* part_o,
                                    const float* part_lse, void* O, float* lse, void* stream) {
    return combine_public(rows, S, d, part_o, part_lse, O, lse, stream, 1);
}

namespace {
int32_t partial_impl(int32_t mode, const yoco_xattn_shape* shape, const void* Q, const void* K, const void* V,
                     const int32_t* cu_kv_host, const int32_t* kv_len_host, const int32_t* key_offset_host,
                     const int32_t* kv_total_host, float* part_o, float* part_lse, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (!shape || !part_o || !part_lse) return YOCO_ERR_INVALID_ARG;
    if ((key_offset_host == nullptr) != (kv_total_host == nullptr)) return YOCO_ERR_INVALID_ARG;
    // Without the shard's place in the sequence only T = 1 without a window can be answered: then every
    // key of a shard is visible whatever follows it on other shards.
    if (!key_offset_host && (shape->T != 1 || shape->window != 0)) return YOCO_ERR_UNSUPPORTED;
    if (key_offset_host && !kv_len_host) return YOCO_ERR_INVALID_ARG;
    const ShardPos pos{key_offset_host, kv_total_host};
    return run(shape, mode, Q, K, V, cu_kv_host, kv_len_host, nullptr, part_lse, workspace, workspace_bytes, stream,
               part_o, nullptr, kMaxSubItems, nullptr, key_offset_host ? &pos : nullptr);
}
}  // namespace

int32_t yoco_xattn_decode_partial(const yoco_xattn_shape* shape, const void* Q, const void* K, const void* V,
                                  const int32_t* cu_kv_host, const int32_t* kv_len_host, float* part_o,
                                  float* part_lse, void* workspace, size_t workspace_bytes, void* stream) {
    return partial_impl(YOCO_MODE_DECODE, shape, Q, K, V, cu_kv_host, kv_len_host, nullptr, nullptr, part_o, part_lse,
                        workspace, workspace_bytes, stream);
}

int32_t yoco_xattn_decode_partial_at(const yoco_xattn_shape* shape, const void* Q, const void* K, const void* V,
                                     const int32_t* cu_kv_host, const int32_t* kv_len_host,
                                     const int32_t* key_offset_host, const int32_t* kv_total_host, float* part_o,
                                     float* part_lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!key_offset_host || !kv_total_host) return YOCO_ERR_INVALID_ARG;
    return partial_impl(YOCO_MODE_DECODE, shape, Q, K, V, cu_kv_host, kv_len_host, key_offset_host, kv_total_host,
                        part_o, part_lse, workspace, workspace_bytes, stream);
}

int32_t yoco_xattn_chunk_partial_at(const yoco_xattn_shape* shape, const void* Q, const void* K, const void* V,
                                    const int32_t* cu_kv_host, const int32_t* kv_len_host,
                                    const int32_t* key_offset_host, const int32_t* kv_total_host, float* part_o,
                                    float* part_lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!key_offset_host || !kv_total_host) return YOCO_ERR_INVALID_ARG;
    return partial_impl(YOCO_MODE_CHUNK, shape, Q, K, V, cu_kv_host, kv_len_host, key_offset_host, kv_total_host,
                        part_o, part_lse, workspace, workspace_bytes, stream);
}

int32_t yoco_xattn_decode_fp8(const yoco_xattn_shape* shape, const void* Q, const void* K8, const void* V8,
                              const float* k_scale_host, const float* v_scale_host, const int32_t* cu_kv_host,
                              const int32_t* kv_len_host, void* O, float* lse, void* workspace,
                              size_t workspace_bytes, void* stream) {
    if (!shape || !k_scale_host || !v_scale_host) return YOCO_ERR_INVALID_ARG;
    if (shape->d != 128 || shape->Hkv > kFp8MaxHeads) return YOCO_ERR_UNSUPPORTED;
    for (int c = 0; c < shape->Hkv; ++c)
        if (!(k_scale_host[c] > 0.f) || !(v_scale_host[c] > 0.f) || !std::isfinite(k_scale_host[c]) ||
            !std::isfinite(v_scale_host[c]))
            return YOCO_ERR_INVALID_ARG;
    const Fp8Scales sc{k_scale_host, v_scale_host};
    return run(shape, YOCO_MODE_DECODE, Q, K8, V8, cu_kv_host, kv_len_host, O, lse, workspace, workspace_bytes,
               stream, nullptr, &sc);
}

int32_t yoco_xattn_chunk_fp8(const yoco_xattn_shape* shape, const void* Q, const void* K8, const void* V8,
                             const float* k_scale_host, const float* v_scale_host, const int32_t* cu_kv_host,
                             const int32_t* kv_len_host, void* O, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream) {
    if (!shape || !k_scale_host || !v_scale_host) return YOCO_ERR_INVALID_ARG;
    if (shape->d != 128 || shape->Hkv > kFp8MaxHeads) return YOCO_ERR_UNSUPPORTED;
    for (int c = 0; c < shape->Hkv; ++c)
        if (!(k_scale_host[c] > 0.f) || !(v_scale_host[c] > 0.f) || !std::isfinite(k_scale_host[c]) ||
            !std::isfinite(v_scale_host[c]))
            return YOCO_ERR_INVALID_ARG;
    const Fp8Scales sc{k_scale_host, v_scale_host};
    return run(shape, YOCO_MODE_CHUNK, Q, K8, V8, cu_kv_host, kv_len_host, O, lse, workspace, workspace_bytes,
               stream, nullptr, &sc);
}

int32_t yoco_xattn_workspace_size_chunk_fp8(const yoco_xattn_shape* shape, const int32_t* kv_len_host,
                                            int32_t sm_count, size_t* bytes) {
    if (!shape || !bytes || sm_count < 0) return YOCO_ERR_INVALID_ARG;
    if (sm_count == 0) {
        int32_t rc = validate_shape(*shape, YOCO_MODE_CHUNK);
        if (rc != YOCO_OK) return rc;
        DeviceState* dev = nullptr;
        if ((rc = device_state(&dev)) != YOCO_OK) return rc;
        sm_count = dev->sm_count;
    }
    Plan plan;
    int32_t rc = make_plan(*shape, nullptr, kv_len_host, sm_count, YOCO_MODE_CHUNK, plan, kMaxSubItems, nullptr, nullptr,
                           kFp8Cache);
    if (rc != YOCO_OK) return rc;
    *bytes = (size_t)plan.info.workspace_bytes;
    return YOCO_OK;
}

int32_t yoco_kv_fold_gain(int64_t d_model, int64_t n_out, const void* g, const void* W, void* Wg, void* stream) {
    if (d_model < 0 || n_out < 0) return YOCO_ERR_INVALID_ARG;
    if (d_model == 0 || n_out == 0) return YOCO_OK;
    if (!g || !W || !Wg || W == Wg) return YOCO_ERR_INVALID_ARG;
    YOCO_CUDA_TRY(launch_fold_gain(static_cast<const __nv_bfloat16*>(g), static_cast<const __nv_bfloat16*>(W),
                                   static_cast<__nv_bfloat16*>(Wg), d_model, n_out,
                                   reinterpret_cast<cudaStream_t>(stream)));
    return YOCO_OK;
}

namespace {
int32_t kv_append_impl(const yoco_kv_append_shape* shape, const void* X, const void* Wgk, const void* Wgv, void* K,
                       void* V, const float* k_scale_host, const float* v_scale_host, bool fp8,
                       const int32_t* cu_kv_host, const int32_t* kv_len_host, void* stream) {
    if (!shape) return YOCO_ERR_INVALID_ARG;
    const yoco_kv_append_shape& s = *shape;
    if (s.B < 0 || s.Hkv <= 0 || s.d <= 0 || s.T <= 0 || s.d_model <= 0 || s.kv_head_stride < 0 || !(s.eps >= 0.f))
        return YOCO_ERR_INVALID_ARG;
    if ((s.d != 64 && s.d != 128) || s.d_model % 128 != 0 || (s.Hkv * s.d) % 128 != 0 ||
        s.kv_head_stride % s.d != 0 || s.B > kAppendMaxSequences || (int64_t)s.B * s.T >= (1ll << 31))
        return YOCO_ERR_UNSUPPORTED;
    if (s.B == 0) return YOCO_OK;
    if (!X || !Wgk || !Wgv || !K || !V || !kv_len_host) return YOCO_ERR_INVALID_ARG;
    if (!aligned(X, 16) || !aligned(Wgk, 16) || !aligned(Wgv, 16) || !aligned(K, 16) || !aligned(V, 16))
        return YOCO_ERR_INVALID_ARG;
    KvAppendTables tab;
    std::memset(&tab, 0, sizeof tab);
    int64_t tok = 0;
    for (int i = 0; i < s.B; ++i) {
        const int64_t n = kv_len_host[i];
        if (n < s.T) return YOCO_ERR_INVALID_ARG;
        const int64_t head_rows = s.kv_head_stride ? s.kv_head_stride / s.d : n;
        if (head_rows < n) return YOCO_ERR_INVALID_ARG;
        if (cu_kv_host) {
            if (cu_kv_host[i] < 0 || cu_kv_host[i + 1] < cu_kv_host[i]) return YOCO_ERR_INVALID_ARG;
            // the rows written for sequence i may not reach into the next sequence's heads
            if ((int64_t)cu_kv_host[i + 1] - cu_kv_host[i] < head_rows) return YOCO_ERR_INVALID_ARG;
            tok = cu_kv_host[i];
        }
        const int64_t row0 = tok * s.Hkv + (n - s.T);
        if (row0 + (int64_t)(s.Hkv - 1) * head_rows + s.T >= (1ll << 31)) return YOCO_ERR_UNSUPPORTED;
        tab.row0[i] = (int32_t)row0;
        tab.head_rows[i] = (int32_t)head_rows;
        if (!cu_kv_host) tok += head_rows;
    }
    DeviceState* dev = nullptr;
    int32_t rc = device_state(&dev);
    if (rc != YOCO_OK) return rc;
    KvAppendParams p{};
    p.X = static_cast<const __nv_bfloat16*>(X);
    p.K = static_cast<__nv_bfloat16*>(K);
    p.V = static_cast<__nv_bfloat16*>(V);
    p.M = s.B * s.T;
    p.T = s.T;
    p.d = s.d;
    p.d_model = s.d_model;
    p.n_half = s.Hkv * s.d;
    p.eps = s.eps;
    CUtensorMap tmX, tmWk, tmWv;
    if ((rc = make_map_2d(&tmX, X, p.M, s.d_model, 128)) != YOCO_OK) return rc;
    if ((rc = make_map_2d(&tmWk, Wgk, s.d_model, p.n_half, 128)) != YOCO_OK) return rc;
    if ((rc = make_map_2d(&tmWv, Wgv, s.d_model, p.n_half, 128)) != YOCO_OK) return rc;
    KvAppendScales sc{};
    if (fp8) {
        if (!k_scale_host || !v_scale_host) return YOCO_ERR_INVALID_ARG;
        if (s.Hkv > kFp8MaxHeads) return YOCO_ERR_UNSUPPORTED;
        for (int c = 0; c < s.Hkv; ++c) {
            if (!(k_scale_host[c] > 0.f) || !(v_scale_host[c] > 0.f) || !std::isfinite(k_scale_host[c]) ||
                !std::isfinite(v_scale_host[c]))
                return YOCO_ERR_INVALID_ARG;
            sc.inv_k[c] = 1.f / k_scale_host[c];
            sc.inv_v[c] = 1.f / v_scale_host[c];
        }
    }
    YOCO_CUDA_TRY(launch_kv_append(p, tab, tmX, tmWk, tmWv, reinterpret_cast<cudaStream_t>(stream), fp8 ? &sc : nullptr));
    return YOCO_OK;
}
}  // namespace

int32_t yoco_kv_append(const yoco_kv_append_shape* shape, const void* X, const void* Wgk, const void* Wgv,
                       void* K, void* V, const int32_t* cu_kv_host, const int32_t* kv_len_host, void* stream) {
    return kv_append_impl(shape, X, Wgk, Wgv, K, V, nullptr, nullptr, false, cu_kv_host, kv_len_host, stream);
}

int32_t yoco_kv_append_fp8(const yoco_kv_append_shape* shape, const void* X, const void* Wgk, const void* Wgv,
                           void* K8, void* V8, const float* k_scale_host, const float* v_scale_host,
                           const int32_t* cu_kv_host, const int32_t* kv_len_host, void* stream) {
    return kv_append_impl(shape, X, Wgk, Wgv, K8, V8, k_scale_host, v_scale_host, true, cu_kv_host, kv_len_host,
                          stream);
}

namespace {
// checks; a zero *sm_count becomes that of the current device
int32_t paged_workspace_args(const yoco_xattn_shape* shape, const yoco_paged_layout* layout, int32_t* sm_count, int32_t mode,
                             int32_t q4, const size_t* bytes) {
    if (!shape || !layout || !bytes || *sm_count < 0) return YOCO_ERR_INVALID_ARG;
    int32_t rc = validate_shape(*shape, mode);
    if (rc != YOCO_OK) return rc;
    if (shape->kv_head_stride != 0) return YOCO_ERR_INVALID_ARG;
    if ((q4 && shape->d != 128) || !valid_page_size(layout->page_size)) return YOCO_ERR_UNSUPPORTED;
    if (*sm_count == 0) {
        DeviceState* dev = nullptr;
        if ((rc = device_state(&dev)) != YOCO_OK) return rc;
        *sm_count = dev->sm_count;
    }
    return YOCO_OK;
}
}  // namespace

int32_t yoco_xattn_workspace_size_paged(const yoco_xattn_shape* shape, const yoco_paged_layout* layout,
                                        const int32_t* kv_len_host, int32_t sm_count, int32_t mode, int32_t q4,
                                        size_t* bytes) {
    return no_throw([&]() -> int32_t {
        int32_t rc = paged_workspace_args(shape, layout, &sm_count, mode, q4, bytes);
        if (rc != YOCO_OK) return rc;
        Plan plan;
        rc = make_plan(*shape, nullptr, kv_len_host, sm_count, mode, plan, kMaxSubItems, nullptr, nullptr,
                       q4 ? kPagedQ4Cache : kPagedCache);
        if (rc != YOCO_OK) return rc;
        *bytes = (size_t)plan.info.workspace_bytes;
        return YOCO_OK;
    });
}

int32_t yoco_xattn_workspace_bound_paged(const yoco_xattn_shape* shape, const yoco_paged_layout* layout,
                                         const int32_t* kv_len_host, int32_t sm_count, int32_t mode, int32_t q4,
                                         size_t* bytes) {
    return no_throw([&]() -> int32_t {
        int32_t rc = paged_workspace_args(shape, layout, &sm_count, mode, q4, bytes);
        if (rc != YOCO_OK) return rc;
        int64_t n = 0;
        if ((rc = workspace_bound(*shape, kv_len_host, sm_count, mode, q4 ? kPagedQ4Cache : kPagedCache, &n)) != YOCO_OK) return rc;
        *bytes = (size_t)n;
        return YOCO_OK;
    });
}

int32_t yoco_xattn_decode_paged(const yoco_xattn_shape* shape, const yoco_paged_layout* layout, const void* Q,
                                const void* K_pages, const void* V_pages, const int32_t* page_table,
                                const int32_t* kv_len_host, void* O, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
    return attend_paged(YOCO_MODE_DECODE, shape, layout, Q, K_pages, nullptr, V_pages, nullptr, false, page_table,
                        kv_len_host, O, lse, workspace, workspace_bytes, stream);
}

int32_t yoco_xattn_decode_paged_q4(const yoco_xattn_shape* shape, const yoco_paged_layout* layout, const void* Q,
                                   const void* K4, const void* K_scale, const void* V4, const void* V_scale,
                                   const int32_t* page_table, const int32_t* kv_len_host, void* O, float* lse,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    return attend_paged(YOCO_MODE_DECODE, shape, layout, Q, K4, K_scale, V4, V_scale, true, page_table, kv_len_host, O,
                        lse, workspace, workspace_bytes, stream);
}

int32_t yoco_xattn_chunk_paged(const yoco_xattn_shape* shape, const yoco_paged_layout* layout, const void* Q,
                               const void* K_pages, const void* V_pages, const int32_t* page_table,
                               const int32_t* kv_len_host, void* O, float* lse, void* workspace,
                               size_t workspace_bytes, void* stream) {
    return attend_paged(YOCO_MODE_CHUNK, shape, layout, Q, K_pages, nullptr, V_pages, nullptr, false, page_table,
                        kv_len_host, O, lse, workspace, workspace_bytes, stream);
}

int32_t yoco_xattn_chunk_paged_q4(const yoco_xattn_shape* shape, const yoco_paged_layout* layout, const void* Q,
                                  const void* K4, const void* K_scale, const void* V4, const void* V_scale,
                                  const int32_t* page_table, const int32_t* kv_len_host, void* O, float* lse,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    return attend_paged(YOCO_MODE_CHUNK, shape, layout, Q, K4, K_scale, V4, V_scale, true, page_table, kv_len_host, O,
                        lse, workspace, workspace_bytes, stream);
}

int32_t yoco_paged_append(const yoco_paged_append_shape* shape, const yoco_paged_layout* layout, const void* K_new,
                          const void* V_new, void* K_pages, void* V_pages, const int32_t* page_table,
                          const int32_t* new_len_host, const int32_t* kv_len_host, void* stream) {
    return paged_rows(shape, layout, true, false, K_new, V_new, K_pages, nullptr, V_pages, nullptr, page_table, nullptr,
                      kv_len_host, new_len_host, nullptr, nullptr, stream);
}

int32_t yoco_paged_append_q4(const yoco_paged_append_shape* shape, const yoco_paged_layout* layout, const void* K_new,
                             const void* V_new, void* K4, void* K_scale, void* V4, void* V_scale,
                             const int32_t* page_table, const int32_t* new_len_host, const int32_t* kv_len_host,
                             void* stream) {
    return paged_rows(shape, layout, true, true, K_new, V_new, K4, K_scale, V4, V_scale, page_table, nullptr,
                      kv_len_host, new_len_host, nullptr, nullptr, stream);
}

int32_t yoco_paged_gather(const yoco_paged_append_shape* shape, const yoco_paged_layout* layout, const void* K_pages,
                          const void* V_pages, const int32_t* page_table, const int32_t* begin_host,
                          const int32_t* end_host, void* K, void* V, void* stream) {
    return paged_rows(shape, layout, false, false, nullptr, nullptr, K_pages, nullptr, V_pages, nullptr, page_table,
                      begin_host, end_host, nullptr, K, V, stream);
}

int32_t yoco_paged_gather_q4(const yoco_paged_append_shape* shape, const yoco_paged_layout* layout, const void* K4,
                             const void* K_scale, const void* V4, const void* V_scale, const int32_t* page_table,
                             const int32_t* begin_host, const int32_t* end_host, void* K, void* V, void* stream) {
    return paged_rows(shape, layout, false, true, nullptr, nullptr, K4, K_scale, V4, V_scale, page_table, begin_host,
                      end_host, nullptr, K, V, stream);
}

int32_t yoco_rope_q(const yoco_xattn_shape* shape, const yoco_paged_layout* layout, const void* Q,
                    const int32_t* kv_len_host, void* Q_rot, void* stream) {
    return no_throw([&]() -> int32_t {
        if (!shape || !layout) return YOCO_ERR_INVALID_ARG;
        int32_t rc = validate_shape(*shape, YOCO_MODE_CHUNK);
        if (rc != YOCO_OK) return rc;
        if (shape->B == 0) return YOCO_OK;
        if (shape->B > kAppendMaxSequences) return YOCO_ERR_UNSUPPORTED;
        if (!Q || !Q_rot || !aligned(Q, 16) || !aligned(Q_rot, 16) || !layout->cos_sin || (layout->rope_pairs & ~1))
            return YOCO_ERR_INVALID_ARG;
        SeqTable tab;
        std::memset(&tab, 0, sizeof tab);
        int64_t max_len = 0;
        for (int32_t i = 0; i < shape->B; ++i) {
            const int32_t n = kv_len_host ? kv_len_host[i] : shape->max_kv_len;
            if (n < 0) return YOCO_ERR_INVALID_ARG;
            tab.pos0[i] = (int32_t)std::max<int64_t>((int64_t)n - shape->T, INT32_MIN);   // may be negative
            max_len = std::max<int64_t>(max_len, n);
        }
        Rotation rot;
        if ((rc = check_rotation(*layout, max_len, &rot)) != YOCO_OK) return rc;
        DeviceState* dev = nullptr;
        if ((rc = device_state(&dev)) != YOCO_OK) return rc;
        YOCO_CUDA_TRY(launch_rope_q(static_cast<const __nv_bfloat16*>(Q), static_cast<__nv_bfloat16*>(Q_rot), shape->B,
                                    shape->Hq, shape->T, shape->d, rot, tab, reinterpret_cast<cudaStream_t>(stream)));
        return YOCO_OK;
    });
}

int32_t yoco_gret_step(const yoco_gret_shape* shape, const void* Q, const void* K, const void* V, const void* decay,
                       const yoco_norm_gate* norm, float* state, const int32_t* slot_in_host, const int32_t* slot_out_host,
                       void* O, void* stream) {
    return gret(shape, Q, K, V, decay, norm, state, slot_in_host, slot_out_host, nullptr, true, O, nullptr, 0, stream);
}

int32_t yoco_gret_chunk(const yoco_gret_shape* shape, const void* Q, const void* K, const void* V, const void* decay,
                        const yoco_norm_gate* norm, float* state, const int32_t* slot_in_host, const int32_t* slot_out_host,
                        const int32_t* len_host, void* O, void* workspace, size_t workspace_bytes, void* stream) {
    return gret(shape, Q, K, V, decay, norm, state, slot_in_host, slot_out_host, len_host, false, O, workspace, workspace_bytes, stream);
}

int32_t yoco_gret_workspace_size(const yoco_gret_shape* shape, const int32_t* len_host, int32_t sm_count, size_t* bytes) {
    return gret_workspace(shape, len_host, sm_count, bytes, [&](int32_t sms) {
        GretPlan plan;
        plan_gret(*shape, len_host, nullptr, sms, &plan);
        return plan.bytes();
    });
}

int32_t yoco_gret_workspace_bound(const yoco_gret_shape* shape, const int32_t* len_host, int32_t sm_count, size_t* bytes) {
    return gret_workspace(shape, len_host, sm_count, bytes, [&](int32_t sms) {
        int64_t chunks = 0;
        for (int32_t i = 0; i < shape->B; ++i) chunks += ((int64_t)(len_host ? len_host[i] : shape->T) + kGretChunk - 1) / kGretChunk;
        GretPlan plan;                                     // streams cut over as many CTAs as there can be
        plan.split = chunks * shape->H > 1;
        plan.set_groups((int32_t)std::min<int64_t>(chunks * shape->H, sms), shape->d);
        return plan.bytes();
    });
}

int32_t yoco_head_norm(const yoco_head_norm_shape* shape, const void* X, const yoco_norm_gate* norm, void* Y, void* stream) {
    if (!shape || !norm) return YOCO_ERR_INVALID_ARG;
    const yoco_head_norm_shape& s = *shape;
    if (s.tokens < 0 || s.H <= 0 || s.d <= 0 || s.x_stride < 0 || s.y_stride < 0) return YOCO_ERR_INVALID_ARG;
    if (s.d % 8 != 0 || s.d > 1024 || s.tokens > INT32_MAX / s.H) return YOCO_ERR_UNSUPPORTED;
    const int64_t width = (int64_t)s.H * s.d;
    HeadNormParams p{};
    p.x_stride = s.x_stride;
    p.y_stride = s.y_stride;
    int32_t rc;
    if ((rc = check_rows(X, &p.x_stride, width)) != YOCO_OK || (rc = check_rows(Y, &p.y_stride, width)) != YOCO_OK ||
        (rc = check_norm(norm, width, &p.norm)) != YOCO_OK)
        return rc;
    if (s.tokens == 0) return YOCO_OK;
    if (!X || !Y || (Y == X && s.tokens > 1 && p.y_stride != p.x_stride)) return YOCO_ERR_INVALID_ARG;
    DeviceState* dev = nullptr;
    if ((rc = device_state(&dev)) != YOCO_OK) return rc;
    p.x = static_cast<const __nv_bfloat16*>(X);
    p.y = static_cast<__nv_bfloat16*>(Y);
    p.groups = (int32_t)(s.tokens * s.H);
    p.H = s.H;
    p.d = s.d;
    YOCO_CUDA_TRY(launch_head_norm(p, reinterpret_cast<cudaStream_t>(stream)));
    return YOCO_OK;
}

int32_t yoco_rope(const yoco_rope_shape* shape, const void* Q, const void* K, const double* inv_freq, const int32_t* pos_host,
                  const int32_t* len_host, void* Q_rot, void* K_rot, void* stream) {
    return no_throw([&]() -> int32_t {
        if (!shape) return YOCO_ERR_INVALID_ARG;
        const yoco_rope_shape& s = *shape;
        if (s.B < 0 || s.Hq <= 0 || s.Hk < 0 || s.d <= 0 || s.rot < 0 || s.rot > s.d || (s.rope_pairs & ~1) || s.q_stride < 0 ||
            s.k_stride < 0 || s.q_out_stride < 0 || s.k_out_stride < 0)
            return YOCO_ERR_INVALID_ARG;
        if (s.d % 16 != 0 || s.d > 512 || s.rot % 16 != 0 || s.B > kAppendMaxSequences || (int64_t)s.Hq + s.Hk > 65535)
            return YOCO_ERR_UNSUPPORTED;
        int64_t tokens = 0;
        int32_t rc = check_lengths(s.B, len_host, s.T, &tokens);
        if (rc != YOCO_OK) return rc;
        if (s.B == 0) return YOCO_OK;
        if (!pos_host || !inv_freq || !aligned(inv_freq, 8)) return YOCO_ERR_INVALID_ARG;
        for (int32_t i = 0; i < s.B; ++i)
            if (pos_host[i] < 0 || (int64_t)pos_host[i] + (len_host ? len_host[i] : s.T) > (1ll << 31)) return YOCO_ERR_INVALID_ARG;
        RopeParams p{};
        p.q_stride = s.q_stride;
        p.k_stride = s.k_stride;
        p.q_out_stride = s.q_out_stride;
        p.k_out_stride = s.k_out_stride;
        const int64_t wq = (int64_t)s.Hq * s.d, wk = (int64_t)s.Hk * s.d;
        if ((rc = check_rows(Q, &p.q_stride, wq)) != YOCO_OK || (rc = check_rows(Q_rot, &p.q_out_stride, wq)) != YOCO_OK) return rc;
        if (s.Hk > 0 && ((rc = check_rows(K, &p.k_stride, wk)) != YOCO_OK || (rc = check_rows(K_rot, &p.k_out_stride, wk)) != YOCO_OK))
            return rc;
        if (tokens == 0) return YOCO_OK;
        if (!Q || !Q_rot || (s.Hk > 0 && (!K || !K_rot))) return YOCO_ERR_INVALID_ARG;
        // in place: rows of the same distance, or one token would be written over another that is still to be read
        if (tokens > 1 && ((Q_rot == Q && p.q_out_stride != p.q_stride) || (s.Hk > 0 && K_rot == K && p.k_out_stride != p.k_stride)))
            return YOCO_ERR_INVALID_ARG;
        SeqTable tab;
        std::memset(&tab, 0, sizeof tab);
        p.tokens_per_seq = len_host ? len_host[0] : s.T;
        for (int32_t i = 0; i < s.B; ++i) {
            const int32_t n = len_host ? len_host[i] : s.T;
            tab.pos0[i] = pos_host[i];
            tab.tok0[i + 1] = tab.tok0[i] + n;
            if (n != p.tokens_per_seq) p.tokens_per_seq = 0;
        }
        DeviceState* dev = nullptr;
        if ((rc = device_state(&dev)) != YOCO_OK) return rc;
        p.q = static_cast<const __nv_bfloat16*>(Q);
        p.k = static_cast<const __nv_bfloat16*>(K);
        p.q_out = static_cast<__nv_bfloat16*>(Q_rot);
        p.k_out = static_cast<__nv_bfloat16*>(K_rot);
        p.inv_freq = inv_freq;
        p.B = s.B;
        p.Hq = s.Hq;
        p.Hk = s.Hk;
        p.d = s.d;
        p.rot = s.rot ? s.rot : s.d;
        p.neighbours = s.rope_pairs;
        p.tokens = (int32_t)tokens;
        YOCO_CUDA_TRY(launch_rope(p, tab, dev->sm_count, reinterpret_cast<cudaStream_t>(stream)));
        return YOCO_OK;
    });
}

int32_t yoco_kv_append_status(void* stream) {
    int32_t word = 0;
    YOCO_CUDA_TRY(read_and_clear_kv_append_status(&word, reinterpret_cast<cudaStream_t>(stream)));
    return status_code(word);
}

int32_t yoco_kv_append_status_detail(void* stream, int32_t* wait_class, int32_t* cta) {
    int32_t word = 0;
    YOCO_CUDA_TRY(read_and_clear_kv_append_status(&word, reinterpret_cast<cudaStream_t>(stream)));
    return yoco_xattn_decode_status_word(word, wait_class, cta);
}

namespace {
// reads the status word of `workspace`, or of the built-in buffer of the current device when null
int32_t read_status_word(const void* workspace, void* stream, int32_t* word) {
    void* builtin = nullptr;
    if (!workspace) {
        int32_t rc = static_scratch_address(&builtin);
        if (rc != YOCO_OK) return rc;
        workspace = builtin;
    }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    YOCO_CUDA_TRY(cudaMemcpyAsync(word, workspace, sizeof *word, cudaMemcpyDeviceToHost, s));
    YOCO_CUDA_TRY(cudaStreamSynchronize(s));
    return YOCO_OK;
}
}  // namespace

int32_t yoco_xattn_status(const void* workspace, void* stream) {
    int32_t word = 0;
    int32_t rc = read_status_word(workspace, stream, &word);
    if (rc != YOCO_OK) return rc;
    return status_code(word);
}

int32_t yoco_xattn_status_detail(const void* workspace, void* stream, int32_t* wait_class, int32_t* cta) {
    int32_t word = 0;
    int32_t rc = read_status_word(workspace, stream, &word);
    if (rc != YOCO_OK) return rc;
    return yoco_xattn_decode_status_word(word, wait_class, cta);
}

int32_t yoco_xattn_decode_status_word(int32_t word, int32_t* wait_class, int32_t* cta) {
    if (wait_class) *wait_class = word & 0xFF;
    if (cta) *cta = (int32_t)((uint32_t)word >> 8) - 1;
    return status_code(word);
}

int32_t yoco_xattn_selftest_wait_expiry(const yoco_xattn_shape* shape, const void* Q, const void* K, const void* V,
                                        const int32_t* cu_kv_host, const int32_t* kv_len_host, void* O,
                                        void* workspace, size_t workspace_bytes, int32_t limit_ms, void* stream) {
    if (limit_ms <= 0 || limit_ms > 1000) return YOCO_ERR_INVALID_ARG;
    const SelfTest st{(int64_t)limit_ms * 1000000ll};
    return run(shape, YOCO_MODE_DECODE, Q, K, V, cu_kv_host, kv_len_host, O, nullptr, workspace, workspace_bytes,
               stream, nullptr, nullptr, 1, &st);
}

int32_t yoco_xattn_selftest_wait_expiry_fp8(const yoco_xattn_shape* shape, const void* Q, const void* K8,
                                            const void* V8, const float* k_scale_host, const float* v_scale_host,
                                            const int32_t* cu_kv_host, const int32_t* kv_len_host, void* O,
                                            void* workspace, size_t workspace_bytes, int32_t limit_ms, void* stream) {
    if (limit_ms <= 0 || limit_ms > 1000 || !k_scale_host || !v_scale_host) return YOCO_ERR_INVALID_ARG;
    const SelfTest st{(int64_t)limit_ms * 1000000ll};
    const Fp8Scales sc{k_scale_host, v_scale_host};
    return run(shape, YOCO_MODE_DECODE, Q, K8, V8, cu_kv_host, kv_len_host, O, nullptr, workspace, workspace_bytes,
               stream, nullptr, &sc, 1, &st);
}

int32_t yoco_xattn_selftest_wait_expiry_paged(const yoco_xattn_shape* shape, const yoco_paged_layout* layout,
                                              const void* Q, const void* K, const void* K_scale, const void* V,
                                              const void* V_scale, const int32_t* page_table, const int32_t* kv_len_host,
                                              void* O, void* workspace, size_t workspace_bytes, int32_t limit_ms,
                                              void* stream) {
    if (limit_ms <= 0 || limit_ms > 1000 || (K_scale == nullptr) != (V_scale == nullptr)) return YOCO_ERR_INVALID_ARG;
    const SelfTest st{(int64_t)limit_ms * 1000000ll};
    return attend_paged(YOCO_MODE_DECODE, shape, layout, Q, K, K_scale, V, V_scale, K_scale != nullptr, page_table,
                        kv_len_host, O, nullptr, workspace, workspace_bytes, stream, &st);
}

int32_t yoco_gret_selftest_wait_expiry(const yoco_gret_shape* shape, const void* Q, const void* K, const void* V, const void* decay,
                                       const yoco_norm_gate* norm, float* state, const int32_t* slot_in_host,
                                       const int32_t* slot_out_host, const int32_t* len_host, void* O, void* workspace,
                                       size_t workspace_bytes, int32_t limit_ms, void* stream) {
    if (limit_ms <= 0 || limit_ms > 1000) return YOCO_ERR_INVALID_ARG;
    const SelfTest st{(int64_t)limit_ms * 1000000ll};
    return gret(shape, Q, K, V, decay, norm, state, slot_in_host, slot_out_host, len_host, false, O, workspace, workspace_bytes, stream, &st);
}

int32_t yoco_xattn_profile_enable(int32_t max_records) {
    if (max_records < 0) return YOCO_ERR_INVALID_ARG;
    std::lock_guard<std::mutex> lock(g_mutex);
    for (cudaEvent_t e : g_prof.events) cudaEventDestroy(e);
    g_prof.events.clear();
    g_prof.used = 0;
    for (int32_t k = 0; k < 2 * max_records; ++k) {
        cudaEvent_t e;
        cudaError_t err = cudaEventCreate(&e);
        if (err != cudaSuccess) return cuda_fail(err);
        g_prof.events.push_back(e);
    }
    return YOCO_OK;
}

int32_t yoco_xattn_profile_collect(float* kernel_ms, int32_t capacity, int32_t* count) {
    if (!count || capacity < 0 || (capacity > 0 && !kernel_ms)) return YOCO_ERR_INVALID_ARG;
    std::lock_guard<std::mutex> lock(g_mutex);
    const int32_t n = std::min(capacity, g_prof.used);
    for (int32_t k = 0; k < n; ++k) {
        YOCO_CUDA_TRY(cudaEventSynchronize(g_prof.events[2 * k + 1]));
        YOCO_CUDA_TRY(cudaEventElapsedTime(&kernel_ms[k], g_prof.events[2 * k], g_prof.events[2 * k + 1]));
    }
    *count = n;
    g_prof.used = 0;
    return YOCO_OK;
}

const char* yoco_xattn_strerror(int32_t code) {
    switch (code) {
        case YOCO_OK: return "ok";
        case YOCO_ERR_INVALID_ARG: return "invalid argument";
        case YOCO_ERR_UNSUPPORTED: return "unsupported shape or device";
        case YOCO_ERR_WORKSPACE_TOO_SMALL: return "workspace too small";
        case YOCO_ERR_CUDA: return "CUDA call failed (see yoco_xattn_last_cuda_error)";
        case YOCO_ERR_TIMEOUT: return "a bounded device-side wait expired";
        case YOCO_ERR_HOST_MEMORY: return "host memory allocation failed";
        case YOCO_ERR_BAD_PAGE: return "a page table entry is not a page of the pool";
        case YOCO_ERR_STATIC_SCRATCH_EXCEEDED:
            return "problem needs more scratch than the built-in static buffer holds; "
                   "use yoco_xattn_decode with a caller-provided workspace";
        default: return "unknown error code";
    }
}

int32_t yoco_xattn_last_cuda_error(void) { return g_last_cuda_error; }

}  // extern "C"
