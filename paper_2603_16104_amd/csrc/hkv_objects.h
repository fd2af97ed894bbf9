// The library's opaque objects and what its host files share.  Not part of the C ABI.
#pragma once

#include <algorithm>
#include <deque>
#include <vector>

#include "../../include/heliumkv.h"
#include "hkv_internal.h"

using namespace hkv;

struct hkv_decode_plan {
    hkv_pool *pool = nullptr;
    int32_t n_req = 0, num_q_heads = 0, group = 0, n_parts = 0, max_parts = 1;
    std::vector<hkv_node> key_nodes;        // the caller's forest: key of the one-shot cache
    std::vector<int32_t> key_pages, req_leaf;
    std::vector<hkv_node> nodes;            // the same forest in 16-token blocks (page_begin, n_pages into node_pages)
    std::vector<int32_t> node_pages;
    std::vector<DecodeItem> items;
    // Items shared by kMinTileItemRows query rows or more (up to 256 / G requests each): run by the 256-row
    // tile kernel on tile_workgroups persistent workgroups, on a stream of the plan's own next to the kernel
    // that runs `items` (or in front of it on the caller's stream when concurrent is false).
    std::vector<DecodeItem> tile_items;
    int32_t tile_workgroups = 0;
    // Small steps: whole paths instead of items, one launch (path_waves wavefronts per workgroup; 0: items)
    std::vector<int32_t> paths;
    int32_t path_stride = 0, n_paths = 0, path_waves = 0;
    double paths_us = 0, items_us = 0;  // estimates of a step; paths_us = 0: paths are out of the question, items_us is not asked for
    int32_t *d_paths = nullptr;
    int32_t restart_tokens = kMaxSharedItemTokens;  // a stretch of a shared node's item with one reference per row
    bool row_visibility = false;  // several query tokens per request: rows see their last node in part
    bool concurrent = true;
    bool fused = false;  // both kinds of items go out as one launch (no item of `items` has more than 16 rows)
    hipStream_t side = nullptr;
    hipEvent_t ev_fork = nullptr, ev_join = nullptr;
    hipEvent_t ev_tile[2] = {nullptr, nullptr};  // profiling: begin/end of the tile kernel
    std::vector<int32_t> node_req_indptr, node_req_idx, part_count;
    // one device allocation holding items | pages | node_req_idx | part_count | tile_items
    void *dev = nullptr;
    DecodeItem *d_items = nullptr, *d_tile_items = nullptr;
    int32_t n_single = 0;  // items [0, n_single) run one per workgroup, the rest four per workgroup
    std::vector<int32_t> order;  // fp4 pools: DecodeLaunch::order
    int32_t *d_order = nullptr;
    int32_t n_stages = 3;  // LDS stages of 16 KiB per workgroup of the per-node kernel
    bool has_shared = false;  // items of `items` shared by more than 16 query rows are run by shared::body
    int tile_form = 0;  // bf16 pools: -1 never, 1 always shared::body, 2 with tall tiles (HKV_PLAN_NARROW_TILES, _WIDE_TILES, _TALL_TILES)
    bool fp8_matrix = false;  // fp8 pools: both products on the fp8 matrix instruction (HKV_PLAN_FP8_MATRIX)
    hkv_decode_plan_params opt{};  // the planner's settings (0 = the library's choice)
    int32_t *d_pages = nullptr, *d_node_req_idx = nullptr, *d_part_count = nullptr;
    std::vector<int32_t> q_rows;  // row of q / out / lse of every row of the plan (empty: row r is row r)
    int32_t *d_q_rows = nullptr;
    bool profiling = false, profiled_run = false;
    hipEvent_t ev[4] = {nullptr, nullptr, nullptr, nullptr};  // begin/end of the node kernel, begin/end of the merge
    // several query tokens per request: n_req above counts query rows (requests x tokens_per_req)
    int32_t tokens_per_req = 1;
    std::vector<StoreRequest> store;         // per request: where its newest tokens go (hkv_decode_plan_store)
    StoreRequest *d_store = nullptr;         // (inside dev, or behind d_bt)
    int store_blocks = 0;                    // plans that do not grow: 1 the newest tokens' blocks are all different, -1 they are not, 0 not looked at
    std::vector<KeyWeightItem> weight_items;  // hkv_decode_plan_track_weights
    KeyWeightItem *d_weight_items = nullptr;
    bool tracks_weights = false;
    // one allocation (d_row_mask), null when tokens_per_req == 1
    unsigned long long *d_row_mask = nullptr;
    int32_t *d_row_leaf = nullptr, *d_row_limit = nullptr;
    // fp32 pools: no work items; every query row walks its own block table (one allocation: d_bt)
    std::vector<int32_t> row_len;
    int32_t max_pages = 0;
    int32_t *d_bt = nullptr, *d_rows_req = nullptr, *d_rows_len = nullptr;
    int32_t row_parts = 1;  // shares that a row's keys are cut into where the caller's workspace has room for their results
    // growing plans (hkv_decode_plan_create_growing): every request's leaf has block slots in node_pages
    // for reserve_tokens more tokens; grow_items holds, per request, the num_kv_heads items of the leaf's
    // last chunk.  Items and block list are re-sent after every append through a ring of pinned buffers.
    int32_t reserve_tokens = 0, appended = 0;
    std::vector<int32_t> grow_items;
    static constexpr int kGrowSlots = 4;
    char *h_grow = nullptr;  // pinned, kGrowSlots x grow_bytes
    char *d_grow = nullptr;  // the same memory as the device addresses it
    int32_t *d_grow_items = nullptr;  // device copy of grow_items (up to 256 requests: updates by a small kernel)
    size_t grow_bytes = 0;   // items + block list as laid out on the device, a multiple of 16
    hipEvent_t grow_free[kGrowSlots] = {};
    bool grow_in_flight[kGrowSlots] = {};
    int grow_next = 0;
};

struct hkv_prefill_plan {
    hkv_pool *pool = nullptr;
    int32_t n_req = 0, num_q_heads = 0, total_q = 0;
    int32_t key_max_pages = 0;   // row length of the caller's block table (pages)
    int32_t max_pages = 0;       // row length of the device table (16-token blocks)
    std::vector<int32_t> cu_q, block_table, kv_len;   // key of the one-shot cache
    std::vector<int32_t> q_row_begin;                 // a request's first row of q / out where it is not cu_q (empty: it is)
    int store_blocks = 0;                             // 1: no two requests' new tokens share a 16-token block, -1: they do, 0: not looked at
    std::vector<PrefillTile> tiles;
    std::vector<PrefillTile> pieces;  // small batches: the tiles in pieces of fewer rows, a workgroup each (empty: the tiles)
    void *dev = nullptr;
    PrefillTile *d_tiles = nullptr;
    int32_t *d_block_table = nullptr;
    int32_t *d_rows_req = nullptr, *d_rows_len = nullptr;  // fp32 pools: per new token (one allocation: d_rows_req)
    // fp8 and fp4 pools: the pages the batch reads are first dequantised into a bf16 scratch pool in the caller's
    // workspace (page i of the scratch = src_pages[i]); the device block table then holds scratch indices.
    std::vector<int32_t> src_pages;
    int32_t *d_src_pages = nullptr;
    unsigned int *d_fallback = nullptr;  // tiles that repeated with a running maximum, over all runs of the plan
    // tiles split along their keys (empty: a workgroup per tile); the partials go to the caller's workspace
    std::vector<PrefillSegment> segments;
    std::vector<int32_t> seg_begin, seg_tile;  // first segment of every worker; the tile a segment was cut from
    std::vector<PrefillSplitTile> split;
    int32_t n_parts = 0;
    PrefillSegment *d_segments = nullptr;
    int32_t *d_seg_begin = nullptr;
    PrefillSplitTile *d_split = nullptr;
};

struct hkv_pool {
    hkv_pool_desc d{};
    // A page of page_size = 16 * S tokens is S consecutive 16-token blocks of the buffers: block
    // page * S + j holds tokens 16 j .. 16 j + 15 of the page.  Everything behind the entry points
    // (work lists, kernels) deals in 16-token blocks; page ids are translated where they come in.
    int32_t blocks_per_page = 1;
    std::vector<int32_t> refcnt;
    std::deque<int32_t> free_list;
    // Staging of page ids for kv_pool_write: a ring of slots (pinned host + device, one allocation
    // each), so that back-to-back writes on a stream do not wait for one another; a slot is reused
    // only after the event recorded behind its last write has completed.
    static constexpr int kMaxWritePages = 65536;
    static constexpr int kWriteSlots = 8;
    int32_t *h_ids = nullptr;  // pinned host, kWriteSlots x kMaxWritePages
    int32_t *hd_ids = nullptr; // the same memory as the device addresses it (source of the copy kernel)
    int32_t *d_ids = nullptr;  // device, same shape
    hipEvent_t slot_free[kWriteSlots] = {};
    bool slot_in_flight[kWriteSlots] = {};
    int next_slot = 0;
    // What else holds page ids of the pool (prefix caches).  It follows kv_pool_compact: prepare may throw, commit does not; is told when the pool goes; and says
    // how many of a page's references are its own.
    struct Follower {
        void *object;
        void (*prepare)(void *object, const int32_t *new_ids);
        void (*commit)(void *object);
        void (*pool_goes)(void *object);
        int32_t (*holds)(const void *object, int32_t page);
    };
    std::vector<Follower> followers;
    std::vector<uint32_t> mark;  // kv_pool_evict, kv_pool_copy_pages: pages marked in the present call (mark[id] == mark_now)
    uint32_t mark_now = 0;
    void mark_anew() {
        if (mark.empty()) mark.assign(d.num_pages, 0);
        if (++mark_now == 0) {
            std::fill(mark.begin(), mark.end(), 0u);
            mark_now = 1;
        }
    }
    hkv_decode_plan *cached_decode = nullptr;
    hkv_prefill_plan *cached_prefill = nullptr;
};


namespace hkv {

// records the thread-local message and returns the code
int fail(int code, const char *fmt, ...);

inline int fail_hip(hipError_t e, const char *what) {
    return fail(HKV_EHIP, "%s: %s", what, hipGetErrorString(e));
}

#define HKV_HIP(call)                                  \
    do {                                               \
        hipError_t e_ = (call);                        \
        if (e_ != hipSuccess) return fail_hip(e_, #call); \
    } while (0)

inline bool is_capturing(hipStream_t s) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    return hipStreamIsCapturing(s, &capture) == hipSuccess && capture != hipStreamCaptureStatusNone;
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline PoolView view_of(const hkv_pool *p) {
    return PoolView{p->d.k_pages, p->d.v_pages, p->d.k_scale, p->d.v_scale, p->d.num_kv_heads, p->d.dtype};
}

// A slot of the pool's staging ring (kv_pool_write): `take` waits until the next one is free, `leave` marks it as used by what is queued on the stream.  One that a
// call gives up on its way is left all the same, since the upload of its list may be queued already.
class Staging {
   public:
    Staging(hkv_pool *pool, hipStream_t s) : pool_(pool), stream_(s) {}
    Staging(const Staging &) = delete;
    Staging &operator=(const Staging &) = delete;
    ~Staging() { (void)leave(); }
    int take();
    int leave();
    int32_t *host = nullptr, *host_on_device = nullptr, *device = nullptr;

   private:
    hkv_pool *pool_;
    hipStream_t stream_;
    int32_t slot_ = -1;
};

// hkv_decode_plan_append with what happens to the new tokens: neither k_src nor hook: nothing; k_src / v_src: they are stored
// as hkv_decode_plan_append_tokens says; hook: called in place of the kernel that applies the update `g`, where that travels in arguments
// (up to 256 requests); `launched` then says so.
struct AppendHook {
    hipError_t (*launch)(void *ctx, const PlanGrowInline &g, hipStream_t s);
    void *ctx;
    bool launched;
};
int plan_append(hkv_decode_plan *plan, const int32_t *new_page_ids, const void *k_src, const void *v_src, AppendHook *hook, void *stream);

}  // namespace hkv
