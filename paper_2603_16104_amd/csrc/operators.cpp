// Host side of what stands around a step's attention: projections into the pool (hkv_*_store), weights of cached keys
// (attn_decode_plan_weights) and eviction (kv_pool_evict).  Checks and launches; all arithmetic lives in the kernels.
#include "hkv_objects.h"

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <exception>
#include <numeric>

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool is_capturing(hipStream_t s) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    return hipStreamIsCapturing(s, &capture) == hipSuccess && capture != hipStreamCaptureStatusNone;
}

// The call's rows, checked, as the kernels take them.
int projection_of(const hkv_pool *pool, int num_q_heads, const hkv_qkv *x, ProjectionLaunch &a, const char *who) {
    if (!x) return fail(HKV_EINVAL, "%s: null rows", who);
    if (!x->q || !x->k || !x->v || !x->q_out) return fail(HKV_EINVAL, "%s: null q, k, v or q_out", who);
    if (!aligned16(x->q) || !aligned16(x->k) || !aligned16(x->v) || !aligned16(x->q_out) || !aligned16(x->q_norm) || !aligned16(x->k_norm))
        return fail(HKV_EINVAL, "%s: q, k, v, q_out and the norms' weights must be 16-byte aligned", who);
    const int Hkv = pool->d.num_kv_heads, per16 = pool->d.dtype == HKV_FP32 ? 4 : 8;
    const int64_t wide = (int64_t)num_q_heads * HKV_HEAD_DIM, narrow = (int64_t)Hkv * HKV_HEAD_DIM;
    a.q_stride = x->q_stride ? x->q_stride : wide;
    a.k_stride = x->k_stride ? x->k_stride : narrow;
    a.v_stride = x->v_stride ? x->v_stride : narrow;
    if (a.q_stride < wide || a.k_stride < narrow || a.v_stride < narrow || a.q_stride % per16 || a.k_stride % per16 || a.v_stride % per16)
        return fail(HKV_EINVAL, "%s: row strides %lld, %lld, %lld (at least a row each, whole 16-byte pieces)", who, (long long)a.q_stride,
                    (long long)a.k_stride, (long long)a.v_stride);
    if (x->q_out == x->q && a.q_stride != wide) return fail(HKV_EINVAL, "%s: queries in place need rows without gaps", who);
    if ((x->q_norm || x->k_norm) && !(x->eps >= 0.f && std::isfinite(x->eps))) return fail(HKV_EINVAL, "%s: eps %g", who, (double)x->eps);
    if (x->rotary_dim < 0 || x->rotary_dim > HKV_HEAD_DIM || x->rotary_dim % 16)
        return fail(HKV_ESHAPE, "%s: rotary_dim %d (a multiple of 16, up to 128)", who, x->rotary_dim);
    const int n_axes = x->n_axes ? x->n_axes : 1;
    if (n_axes < 1 || n_axes > 4) return fail(HKV_EINVAL, "%s: %d position axes (1..4)", who, n_axes);
    if (x->rotary_dim > 0 && (!x->inv_freq || (reinterpret_cast<uintptr_t>(x->inv_freq) & 7)))
        return fail(HKV_EINVAL, "%s: inv_freq must be non-null and 8-byte aligned", who);
    if (x->positions && (reinterpret_cast<uintptr_t>(x->positions) & 3)) return fail(HKV_EINVAL, "%s: positions must be 4-byte aligned", who);
    if (n_axes > 1 && (!x->positions || !x->axis)) return fail(HKV_EINVAL, "%s: several axes need positions and the axis of every pair", who);
    if (x->position_stride < (n_axes > 1)) return fail(HKV_EINVAL, "%s: position_stride %lld of %d axes", who, (long long)x->position_stride, n_axes);
    if (x->axis)
        for (int p = 0; p < x->rotary_dim / 2; ++p) {
            if (x->axis[p] < 0 || x->axis[p] >= n_axes) return fail(HKV_EINVAL, "%s: pair %d has axis %d of %d", who, p, x->axis[p], n_axes);
            a.axis[p / 16] |= (uint32_t)x->axis[p] << (2 * (p % 16));
        }
    a.pool = PoolWriteLaunch{pool->d.k_pages, pool->d.v_pages, pool->d.k_scale, pool->d.v_scale, Hkv, pool->d.dtype, nullptr, 0, 0, 0, nullptr, nullptr, nullptr, nullptr};
    a.q = x->q;
    a.k = x->k;
    a.v = x->v;
    a.q_out = x->q_out;
    a.q_norm = x->q_norm;
    a.k_norm = x->k_norm;
    a.eps = x->eps;
    a.rotary_dim = x->rotary_dim;
    a.interleaved = x->interleaved != 0;
    a.inv_freq = x->inv_freq;
    a.positions = x->rotary_dim > 0 ? x->positions : nullptr;
    a.position_stride = x->position_stride;
    a.n_axes = n_axes;
    a.group = num_q_heads / Hkv;
    return HKV_OK;
}

// 1: no value (not negative) occurs twice, -1: one does.  By a table of twice the size: a step of 512 requests asks every time.
int all_different(const std::vector<int32_t> &v) {
    size_t size = 16;
    while (size < 2 * v.size()) size *= 2;
    std::vector<int32_t> table(size, -1);
    for (const int32_t x : v) {
        size_t i = ((uint32_t)x * 0x9E3779B1u) >> 7 & (size - 1);
        for (; table[i] >= 0; i = (i + 1) & (size - 1))
            if (table[i] == x) return -1;
        table[i] = x;
    }
    return 1;
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// projections
extern "C" int hkv_prefill_plan_store(hkv_prefill_plan *plan, const hkv_qkv *rows, void *stream) try {
    const char *who = "hkv_prefill_plan_store";
    if (!plan) return fail(HKV_EINVAL, "%s: null plan", who);
    if (plan->tiles.empty()) return HKV_OK;
    ProjectionPrefill p{};
    if (int rc = projection_of(plan->pool, plan->num_q_heads, rows, p.base, who)) return rc;
    if (!plan->dev) return fail(HKV_EINVAL, "%s: plan was built host-only", who);
    const hkv_pool *pool = plan->pool;
    const int S = pool->blocks_per_page, P = pool->d.page_size;
    auto tokens_of = [&](int r) { return plan->cu_q[r + 1] - plan->cu_q[r]; };
    auto units_of = [&](int r) {
        const int n = tokens_of(r), first = plan->kv_len[r] - n;
        return n > 0 ? (plan->kv_len[r] - 1) / HKV_PAGE_SIZE - first / HKV_PAGE_SIZE + 1 : 0;
    };
    if (plan->store_blocks == 0) {
        std::vector<int32_t> blocks;
        for (int r = 0; r < plan->n_req; ++r)
            if (units_of(r) > INT_MAX / 256) return fail(HKV_EINVAL, "%s: request %d brings too many tokens", who, r);  // (a launch keeps below 2^31 threads)
        for (int r = 0; r < plan->n_req; ++r)
            for (int b = (plan->kv_len[r] - tokens_of(r)) / HKV_PAGE_SIZE, e = b + units_of(r); b < e; ++b)
                blocks.push_back(plan->block_table[(size_t)r * plan->key_max_pages + (size_t)b * HKV_PAGE_SIZE / P] * S + b % S);
        plan->store_blocks = all_different(blocks);
    }
    if (plan->store_blocks < 0) return fail(HKV_EINVAL, "%s: new tokens of two requests go to the same 16-token block", who);
    for (int r = 0; r < plan->n_req; ++r) {  // (in every call: owners come and go)
        const int prefix = plan->kv_len[r] - tokens_of(r);
        if (tokens_of(r) == 0 || prefix % P == 0) continue;
        const int32_t page = plan->block_table[(size_t)r * plan->key_max_pages + prefix / P];
        if (pool->refcnt[page] > 1)
            return fail(HKV_EINVAL, "%s: page %d, which request %d continues, has %d owners: kv_pool_copy_on_write first", who, page, r, pool->refcnt[page]);
    }
    p.base.blocks = plan->d_block_table;
    p.base.src_pages = pool->d.dtype == HKV_FP8_E4M3 ? plan->d_src_pages : nullptr;
    p.table_stride = plan->max_pages;
    for (int r = 0; r < plan->n_req;) {  // the requests' places travel in the arguments, kMaxInlineRequests a launch
        p.n_units = 0;
        p.table = (int64_t)r * plan->max_pages;
        int i = 0;
        for (; i < kMaxInlineRequests && r < plan->n_req; ++i, ++r) {
            const int64_t units = units_of(r);
            if (p.n_units + units > INT_MAX / 256) break;
            p.begin[i] = p.n_units;
            p.row0[i] = plan->q_row_begin.empty() ? plan->cu_q[r] : plan->q_row_begin[r];
            p.tokens[i] = tokens_of(r);
            p.prefix[i] = plan->kv_len[r] - p.tokens[i];
            p.n_units += (int32_t)units;
        }
        std::fill(p.begin + i, p.begin + kMaxInlineRequests, INT_MAX);
        HKV_HIP(launch_projection_store(p, static_cast<hipStream_t>(stream)));
    }
    return HKV_OK;
} catch (const std::exception &) {  // (no memory for a list)
    return fail(HKV_ENOMEM, "hkv_prefill_plan_store: out of host memory");
}

static bool on_device(const hkv_decode_plan *plan) { return plan->pool->d.dtype == HKV_FP32 ? plan->d_bt != nullptr : plan->dev != nullptr; }

static void decode_places(const hkv_decode_plan *plan, ProjectionLaunch &a) {
    a.blocks = plan->pool->d.dtype == HKV_FP32 ? plan->d_bt : plan->d_pages;
    a.row_map = plan->d_q_rows;
    a.requests = plan->d_store;
    a.items = plan->d_items;
    a.tokens = plan->tokens_per_req;
    a.n_requests = plan->n_req / plan->tokens_per_req;
}

// The 16-token blocks that the newest tokens of request r lie in: b .. e - 1 of its leaf's.
static void newest_blocks(const hkv_decode_plan *plan, int r, int *b, int *e) {
    const hkv_node &leaf = plan->nodes[plan->req_leaf[(size_t)r * plan->tokens_per_req]];
    *b = (leaf.n_tokens - plan->tokens_per_req) / HKV_PAGE_SIZE;
    *e = (leaf.n_tokens + HKV_PAGE_SIZE - 1) / HKV_PAGE_SIZE;
}

extern "C" int hkv_decode_plan_store(hkv_decode_plan *plan, const hkv_qkv *rows, void *stream) try {
    const char *who = "hkv_decode_plan_store";
    if (!plan) return fail(HKV_EINVAL, "%s: null plan", who);
    if (plan->n_req == 0) return HKV_OK;
    ProjectionLaunch a{};
    if (int rc = projection_of(plan->pool, plan->num_q_heads, rows, a, who)) return rc;
    if (!on_device(plan)) return fail(HKV_EINVAL, "%s: plan was built host-only", who);
    const hkv_pool *pool = plan->pool;
    const int n = plan->n_req / plan->tokens_per_req, S = pool->blocks_per_page;
    const bool look = plan->store_blocks == 0 || plan->reserve_tokens > 0;
    std::vector<int32_t> blocks;
    for (int r = 0; r < n; ++r) {
        const hkv_node &leaf = plan->nodes[plan->req_leaf[(size_t)r * plan->tokens_per_req]];
        if (leaf.n_tokens < plan->tokens_per_req) return fail(HKV_EINVAL, "%s: the last node of request %d holds no token", who, r);
        int b, e;
        newest_blocks(plan, r, &b, &e);
        for (; b < e; ++b) {
            const int32_t block = plan->node_pages[leaf.page_begin + b];
            if (pool->refcnt[block / S] > 1)
                return fail(HKV_EINVAL, "%s: page %d (request %d) has %d owners: kv_pool_copy_on_write first", who, block / S, r, pool->refcnt[block / S]);
            if (look) blocks.push_back(block);
        }
    }
    if (look) plan->store_blocks = all_different(blocks);
    if (plan->store_blocks < 0) return fail(HKV_EINVAL, "%s: newest tokens of two requests go to the same 16-token block", who);
    const int64_t T = plan->tokens_per_req, Hkv = pool->d.num_kv_heads;  // (a launch keeps below 2^31 threads, whatever it goes by)
    if (n * ((T / HKV_PAGE_SIZE + 2) * Hkv + T * ((plan->num_q_heads + Hkv) / 16 + 1)) > INT_MAX / 256) return fail(HKV_EINVAL, "%s: too many requests", who);
    decode_places(plan, a);
    HKV_HIP(launch_projection_store(a, static_cast<hipStream_t>(stream)));
    return HKV_OK;
} catch (const std::exception &) {  // (no memory for a list)
    return fail(HKV_ENOMEM, "hkv_decode_plan_store: out of host memory");
}

extern "C" int hkv_decode_plan_append_qkv(hkv_decode_plan *plan, const int32_t *new_page_ids, const hkv_qkv *rows, void *stream) try {
    const char *who = "hkv_decode_plan_append_qkv";
    if (!plan) return fail(HKV_EINVAL, "%s: null plan", who);
    if (plan->reserve_tokens <= 0) return fail(HKV_EINVAL, "%s: not a growing plan", who);
    ProjectionAppend p{};
    ProjectionLaunch &a = p.base;
    if (plan->n_req > 0) {
        if (int rc = projection_of(plan->pool, plan->num_q_heads, rows, a, who)) return rc;
        if (!plan->dev) return fail(HKV_EINVAL, "%s: plan was built host-only", who);
        // a replay would store to the same slots and lengthen the items again, of which the host's lengths know nothing
        if (is_capturing(static_cast<hipStream_t>(stream))) return fail(HKV_EINVAL, "%s: not for capture into a graph", who);
    }
    // the places of the new tokens: blocks of their own, in pages of one owner (what plan_append refuses is refused there, before anything changes)
    const hkv_pool *pool = plan->pool;
    const int P = pool->d.page_size, S = pool->blocks_per_page;
    std::vector<int32_t> blocks(plan->n_req);
    for (int r = 0; r < plan->n_req; ++r) {
        const hkv_node &leaf = plan->nodes[plan->req_leaf[r]];
        int32_t page;
        if (leaf.n_tokens % P == 0) {
            if (!new_page_ids || new_page_ids[r] < 0 || new_page_ids[r] >= pool->d.num_pages) return plan_append(plan, new_page_ids, nullptr, nullptr, nullptr, stream);
            page = new_page_ids[r];
        } else {
            page = plan->node_pages[leaf.page_begin + leaf.n_pages - 1] / S;
        }
        if (pool->refcnt[page] > 1) return fail(HKV_EINVAL, "%s: page %d (request %d) has %d owners: kv_pool_copy_on_write first", who, page, r, pool->refcnt[page]);
        if (r < kMaxInlineAppend) p.length[r] = leaf.n_tokens;
        blocks[r] = page * S + leaf.n_tokens % P / HKV_PAGE_SIZE;
    }
    // (looked at in every call: what an earlier one found says nothing of leaves that other calls have lengthened, or that have reached the next block of their page)
    if (all_different(blocks) < 0) return fail(HKV_EINVAL, "%s: new tokens of two requests go to the same 16-token block", who);
    decode_places(plan, a);
    AppendHook hook{[](void *ctx, const PlanGrowInline &g, hipStream_t s) { return launch_projection_append(*static_cast<ProjectionAppend *>(ctx), g, s); }, &p, false};
    if (int rc = plan_append(plan, new_page_ids, nullptr, nullptr, &hook, stream)) return rc;
    if (!hook.launched) HKV_HIP(launch_projection_store(a, static_cast<hipStream_t>(stream)));  // behind the update of the plan's lists
    return HKV_OK;
} catch (const std::exception &) {  // (no memory for a list)
    return fail(HKV_ENOMEM, "hkv_decode_plan_append_qkv: out of host memory");
}

// ---------------------------------------------------------------------------------------------
// weights of cached keys
// fp32 pools: the work list, and the lists that the kernel reads beside it, which plans over them do not have on the device.
static int track_fp32(hkv_decode_plan *plan) {
    const char *who = "hkv_decode_plan_track_weights";
    const int Hkv = plan->pool->d.num_kv_heads, n_nodes = (int)plan->nodes.size(), T = plan->tokens_per_req, n = plan->n_req;
    std::vector<char> last(n_nodes, 0);
    for (int r = 0; r < n; ++r) last[plan->req_leaf[r]] = 1;
    auto requests = [&](int v) { return plan->node_req_indptr[v + 1] - plan->node_req_indptr[v]; };
    // nodes of a single tile of rows: as many tokens as make 1024 workgroups, which load their rows once; others: a step of 128, since it loads all rows
    int64_t keys = 0;
    for (int v = 0; v < n_nodes; ++v)
        if (requests(v) > 0) keys += (int64_t)plan->nodes[v].n_tokens * Hkv;
    const int alone = (int)std::clamp<int64_t>(keys / 1024 / 128 * 128, 128, kMaxWeightTokens);
    std::vector<KeyWeightItem> items;
    for (int v = 0; v < n_nodes; ++v) {
        const hkv_node &nd = plan->nodes[v];
        const int length = (int64_t)requests(v) * plan->group > 16 ? 128 : alone;
        for (int64_t t = 0; requests(v) > 0 && t < nd.n_tokens; t += length)
            for (int h = 0; h < Hkv; ++h)
                items.push_back(KeyWeightItem{nd.page_begin + (int32_t)(t / HKV_PAGE_SIZE), (int32_t)t, length, h, plan->node_req_indptr[v], requests(v), last[v] ? v : ~v,
                                              nd.n_tokens, -1});
    }
    if (items.size() > INT_MAX / (64 * kFp32Waves)) return fail(HKV_EINVAL, "%s: too many keys", who);
    if (plan->d_bt && !items.empty()) {
        std::vector<int32_t> lists(plan->node_pages);
        lists.insert(lists.end(), plan->node_req_idx.begin(), plan->node_req_idx.end());
        const size_t bytes = sizeof(KeyWeightItem) * items.size();
        std::vector<unsigned long long> masks;  // then the rows' last nodes and limits: query token t of a request sees all but the T - 1 - t newest keys
        std::vector<int32_t> rows;
        for (int r = 0; T > 1 && r < n; ++r) {
            masks.push_back((2ull << (r % T)) - 1);
            rows.push_back(plan->req_leaf[r]);
        }
        for (int r = 0; T > 1 && r < n; ++r) rows.push_back(plan->nodes[plan->req_leaf[r]].n_tokens - T);
        char *d = nullptr;
        void *visible = nullptr;
        hipError_t e = hipMalloc((void **)&d, bytes + sizeof(int32_t) * lists.size());
        if (e == hipSuccess) e = hipMemcpy(d, items.data(), bytes, hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipMemcpy(d + bytes, lists.data(), sizeof(int32_t) * lists.size(), hipMemcpyHostToDevice);
        if (T > 1) {
            if (e == hipSuccess) e = hipMalloc(&visible, n * (sizeof(unsigned long long) + 2 * sizeof(int32_t)));
            if (e == hipSuccess) e = hipMemcpy(visible, masks.data(), sizeof(unsigned long long) * n, hipMemcpyHostToDevice);
            if (e == hipSuccess) e = hipMemcpy(static_cast<unsigned long long *>(visible) + n, rows.data(), 2 * sizeof(int32_t) * n, hipMemcpyHostToDevice);
        }
        if (e != hipSuccess) {
            if (d) (void)hipFree(d);
            if (visible) (void)hipFree(visible);
            return fail_hip(e, who);
        }
        plan->d_weight_items = reinterpret_cast<KeyWeightItem *>(d);
        plan->d_pages = reinterpret_cast<int32_t *>(d + bytes);
        plan->d_node_req_idx = plan->d_pages + plan->node_pages.size();
        if (T > 1) {
            plan->d_row_mask = static_cast<unsigned long long *>(visible);
            plan->d_row_leaf = reinterpret_cast<int32_t *>(plan->d_row_mask + n);
            plan->d_row_limit = plan->d_row_leaf + n;
        }
    }
    plan->weight_items.swap(items);
    plan->tracks_weights = true;
    return HKV_OK;
}

extern "C" int hkv_decode_plan_track_weights(hkv_decode_plan *plan) try {
    const char *who = "hkv_decode_plan_track_weights";
    if (!plan) return fail(HKV_EINVAL, "%s: null plan", who);
    if (plan->tracks_weights) return HKV_OK;
    const int Hkv = plan->pool->d.num_kv_heads, n_nodes = (int)plan->nodes.size();
    std::vector<int32_t> blocks;
    for (int v = 0; v < n_nodes; ++v)
        if (plan->node_req_indptr[v + 1] > plan->node_req_indptr[v])
            blocks.insert(blocks.end(), plan->node_pages.begin() + plan->nodes[v].page_begin, plan->node_pages.begin() + plan->nodes[v].page_begin + plan->nodes[v].n_pages);
    if (all_different(blocks) < 0) return fail(HKV_EINVAL, "%s: a 16-token block is in the forest twice", who);
    if (plan->pool->d.dtype == HKV_FP32) return track_fp32(plan);
    std::vector<char> last(n_nodes, 0);
    std::vector<int32_t> grows(n_nodes, -1);
    for (int r = 0; r < plan->n_req; ++r) {
        last[plan->req_leaf[r]] = 1;
        if (plan->reserve_tokens > 0) grows[plan->req_leaf[r]] = r;
    }
    auto rows = [&](int v) { return (int64_t)(plan->node_req_indptr[v + 1] - plan->node_req_indptr[v]) * plan->group; };
    auto room = [&](int v) { return (int64_t)plan->nodes[v].n_tokens + (grows[v] >= 0 ? plan->reserve_tokens - plan->appended : 0); };
    // Tokens of an item: for nodes of up to 16 rows as many as make 4096 items, a wavefront each (what the chip holds); the others' work goes by tiles
    // of 16 rows.
    int64_t keys = 0, work = 0;
    for (int v = 0; v < n_nodes; ++v) (rows(v) > 16 ? work : keys) += room(v) * Hkv * (rows(v) > 16 ? (rows(v) + 15) / 16 : rows(v) > 0);
    const int64_t few_length = std::clamp<int64_t>((keys / 4096 + 31) / 32 * 32, 32, kMaxWeightTokens);
    // Nodes of many rows get up to 384 workgroups between them (512 are on the chip at once), fewer where the others' keys take most of the time: a
    // workgroup of theirs takes one of two places of its compute unit.  64 requests' step (2048 shared tokens, 0.7 x 512 own) 16.5 us with 64 of
    // them, 19.3 with 512; 32 queries' look back at 4 x 6400 tokens 20.8 with 384, 23.4 with 256 and 512.
    const double many_us = 0.12 / 1024 / 32 * (double)work, few_us = (double)keys * (plan->pool->d.dtype == HKV_BF16 ? 256 : 128) / 5.5e6;
    const int64_t shares = work > 0 ? std::clamp<int64_t>((int64_t)(384 * many_us / (many_us + few_us)), 64, 384) : 1;
    auto length_of = [&](int v) -> int64_t {
        if (rows(v) <= 16) return few_length;
        const int64_t tokens = work / shares / ((rows(v) + 15) / 16);
        return tokens < 64 ? 32 : tokens < 128 ? 64 : tokens < 256 ? 128 : std::min<int64_t>(tokens / 256 * 256, kMaxWeightTokens);
    };
    std::vector<KeyWeightItem> of[2];  // of nodes of up to 16 rows, of others
    std::vector<int32_t> order(n_nodes);
    std::iota(order.begin(), order.end(), 0);
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return rows(a) > rows(b); });
    for (int v : order) {
        if (rows(v) == 0) continue;
        const hkv_node &nd = plan->nodes[v];
        const int64_t length = length_of(v);
        for (int64_t t = 0; t < room(v); t += length)
            for (int h = 0; h < Hkv; ++h)
                of[rows(v) > 16].push_back(KeyWeightItem{nd.page_begin + (int32_t)(t / HKV_PAGE_SIZE), (int32_t)t, (int32_t)length, h, plan->node_req_indptr[v],
                                                         plan->node_req_indptr[v + 1] - plan->node_req_indptr[v], last[v] ? v : ~v, nd.n_tokens,
                                                         grows[v] >= 0 ? plan->grow_items[(size_t)grows[v] * Hkv + h] : -1});
    }
    // The two kinds side by side, so that one computes while the other reads; those of many rows, which take longer, in the first three quarters.
    // In groups that go round all XCDs (workgroup i runs on XCD i % 8) and all heads, so that every XCD gets its part of both; and in no regular
    // order (the multiples of the golden ratio), since an XCD deals its workgroups out to its four shader engines in turn: every fourth group
    // of many rows and they all ran on a quarter of the chip, 249 us instead of 110 for 16 prompts of 8192 tokens x 256 rows.
    const int of_wave = kWeightWaves, workgroups[2] = {((int)of[0].size() + of_wave - 1) / of_wave, (int)of[1].size()};
    of[0].resize((size_t)workgroups[0] * of_wave, KeyWeightItem{});
    const int group[2] = {8, std::lcm(8, Hkv)}, n_all = workgroups[0] + workgroups[1];
    const double share = n_all ? 4.0 / 3.0 * workgroups[1] * group[0] / (workgroups[1] * group[0] + (double)workgroups[0] * group[1]) : 0.0;
    std::vector<KeyWeightItem> items;
    items.reserve((size_t)n_all * of_wave);
    int at[2] = {0, 0};
    for (int64_t i = 1; at[0] + at[1] < n_all; ++i) {
        const double x = (double)i * 0.6180339887498949;
        int k = x - std::floor(x) < share;
        if (at[k] == workgroups[k]) k = !k;
        for (const int end = std::min(at[k] + group[k], workgroups[k]); at[k] < end; ++at[k])
            for (int w = 0; w < of_wave; ++w) items.push_back(k ? of[1][at[1]] : of[0][(size_t)at[0] * of_wave + w]);
    }
    if (items.size() > INT_MAX / 64) return fail(HKV_EINVAL, "%s: too many keys", who);
    if (plan->dev && !items.empty()) {
        KeyWeightItem *d = nullptr;
        HKV_HIP(hipMalloc((void **)&d, sizeof(KeyWeightItem) * items.size()));
        if (hipError_t e = hipMemcpy(d, items.data(), sizeof(KeyWeightItem) * items.size(), hipMemcpyHostToDevice); e != hipSuccess) {
            (void)hipFree(d);
            return fail_hip(e, who);
        }
        plan->d_weight_items = d;
    }
    plan->weight_items.swap(items);
    plan->tracks_weights = true;
    return HKV_OK;
} catch (const std::exception &) {  // (no memory for a list)
    return fail(HKV_ENOMEM, "hkv_decode_plan_track_weights: out of host memory");
}

extern "C" int attn_decode_plan_weights(hkv_decode_plan *plan, const void *q, float scale, const float *lse, float decay, int32_t n_new,
                                        float *key_weights, void *stream) {
    const char *who = "attn_decode_plan_weights";
    if (!plan) return fail(HKV_EINVAL, "%s: null plan", who);
    if (!plan->tracks_weights) return fail(HKV_EINVAL, "%s: hkv_decode_plan_track_weights has not been called", who);
    if (plan->n_req == 0) return HKV_OK;
    if (!q || !lse || !key_weights) return fail(HKV_EINVAL, "%s: null q, lse or key_weights", who);
    if (!aligned16(q) || !aligned16(key_weights) || (reinterpret_cast<uintptr_t>(lse) & 3))
        return fail(HKV_EINVAL, "%s: q and key_weights must be 16-byte aligned, lse 4-byte", who);
    if (!(decay >= 0.f && decay <= 1.f)) return fail(HKV_EINVAL, "%s: decay %g (0 to 1)", who, (double)decay);
    if (n_new < 0 || n_new > plan->tokens_per_req) return fail(HKV_EINVAL, "%s: n_new %d (0 to the %d query tokens of a request)", who, n_new, plan->tokens_per_req);
    if (!on_device(plan)) return fail(HKV_EINVAL, "%s: plan was built host-only", who);
    const KeyWeightsLaunch a{view_of(plan->pool), q, lse, plan->d_weight_items, plan->d_items, plan->d_pages, plan->d_node_req_idx, plan->d_q_rows,
                             plan->d_row_leaf, plan->d_row_limit, plan->d_row_mask, key_weights, (int32_t)plan->weight_items.size(), plan->num_q_heads,
                             plan->tokens_per_req, n_new, scale, decay};
    HKV_HIP(launch_key_weights(a, static_cast<hipStream_t>(stream)));
    return HKV_OK;
}

// ---------------------------------------------------------------------------------------------
// eviction
extern "C" int kv_pool_evict(hkv_pool *pool, int32_t n_seq, const int32_t *src_pages, const int32_t *n_tokens, const int32_t *dst_pages, const int32_t *n_keep,
                             int32_t n_first, int32_t n_recent, float *key_weights, int32_t *kept, void *stream) try {
    const char *who = "kv_pool_evict";
    if (!pool) return fail(HKV_EINVAL, "%s: null pool", who);
    if (n_seq < 0 || n_first < 0 || n_recent < 0) return fail(HKV_EINVAL, "%s: n_seq %d, n_first %d, n_recent %d", who, n_seq, n_first, n_recent);
    if (n_seq == 0) return HKV_OK;
    if (!n_tokens || !n_keep) return fail(HKV_EINVAL, "%s: null n_tokens or n_keep", who);
    if (pool->d.num_kv_heads > 1024) return fail(HKV_ESHAPE, "%s: %d KV heads (1024 at most)", who, pool->d.num_kv_heads);
    const int P = pool->d.page_size, S = pool->blocks_per_page;
    int64_t src = 0, dst = 0, total = 0;
    for (int i = 0; i < n_seq; ++i) {
        if (n_tokens[i] < 0 || n_keep[i] < 0 || n_keep[i] > n_tokens[i])
            return fail(HKV_EINVAL, "%s: sequence %d keeps %d of %d tokens", who, i, n_keep[i], n_tokens[i]);
        if (n_keep[i] < std::min<int64_t>(n_tokens[i], (int64_t)n_first + n_recent))
            return fail(HKV_EINVAL, "%s: sequence %d keeps %d tokens, fewer than the first %d and the newest %d", who, i, n_keep[i], n_first, n_recent);
        src += (n_tokens[i] + (int64_t)P - 1) / P;
        dst += (n_keep[i] + (int64_t)P - 1) / P;
        total += n_keep[i];
        if (sizeof(EvictSequence) / 4 + (n_tokens[i] + (int64_t)15) / 16 + (n_keep[i] + (int64_t)15) / 16 > hkv_pool::kMaxWritePages)
            return fail(HKV_EINVAL, "%s: sequence %d has %d tokens (about a million at most)", who, i, n_tokens[i]);
    }
    if (total == 0) return HKV_OK;
    if (!src_pages || !dst_pages || !key_weights || !kept) return fail(HKV_EINVAL, "%s: null argument", who);
    if (!aligned16(key_weights) || (reinterpret_cast<uintptr_t>(kept) & 3)) return fail(HKV_EINVAL, "%s: key_weights must be 16-byte aligned, kept 4-byte", who);
    if (total > INT_MAX) return fail(HKV_EINVAL, "%s: too many tokens", who);
    for (int64_t i = 0; i < src; ++i)
        if (src_pages[i] < 0 || src_pages[i] >= pool->d.num_pages)
            return fail(HKV_ERANGE, "%s: page id %d (entry %lld of src_pages) outside pool of %d pages", who, src_pages[i], (long long)i, pool->d.num_pages);
    // new places: pages of one owner, each once, none of those that are read
    if (pool->mark.empty()) pool->mark.assign(pool->d.num_pages, 0);
    if (++pool->mark_now == 0) {
        std::fill(pool->mark.begin(), pool->mark.end(), 0u);
        pool->mark_now = 1;
    }
    for (int64_t i = 0; i < dst; ++i) {
        const int32_t id = dst_pages[i];
        if (id < 0 || id >= pool->d.num_pages)
            return fail(HKV_ERANGE, "%s: page id %d (entry %lld of dst_pages) outside pool of %d pages", who, id, (long long)i, pool->d.num_pages);
        if (pool->refcnt[id] > 1) return fail(HKV_EINVAL, "%s: page %d of dst_pages has %d owners", who, id, pool->refcnt[id]);
        if (pool->mark[id] == pool->mark_now) return fail(HKV_EINVAL, "%s: page %d is in dst_pages twice", who, id);
        pool->mark[id] = pool->mark_now;
    }
    for (int64_t i = 0; i < src; ++i)
        if (pool->mark[src_pages[i]] == pool->mark_now) return fail(HKV_EINVAL, "%s: page %d is read and written", who, src_pages[i]);

    hipStream_t s = static_cast<hipStream_t>(stream);
    if (is_capturing(s)) return fail(HKV_EINVAL, "%s: not for capture into a graph", who);  // (a replay would need slots of the ring as they are now)
    EvictInline a{};
    a.pool = PoolWriteLaunch{pool->d.k_pages, pool->d.v_pages, pool->d.k_scale, pool->d.v_scale, pool->d.num_kv_heads, pool->d.dtype, nullptr, 0, 0, 0, nullptr, nullptr, nullptr, nullptr};
    a.weights = key_weights;
    a.kept = kept;
    a.total = total;
    a.n_first = n_first;
    a.n_recent = n_recent;
    constexpr int kRecord = sizeof(EvictSequence) / sizeof(int32_t);
    int64_t kept_at = 0, sp = 0, dp = 0;
    for (int i0 = 0; i0 < n_seq;) {  // as many sequences at once as a slot of the staging ring describes
        auto ints_of = [&](int i) { return (int64_t)kRecord + (n_tokens[i] + 15) / 16 + (n_keep[i] + 15) / 16; };
        int64_t ints = 0;
        int i1 = i0;
        while (i1 < n_seq && ints + ints_of(i1) <= hkv_pool::kMaxWritePages) ints += ints_of(i1++);
        // what the kernels index with: in their arguments where it fits (2.2 us of a call less), else through the ring
        const bool in_arguments = ints <= kMaxInlineEvict;
        int32_t slot = 0, *hm = a.list, *hdm = nullptr, *dm = nullptr;
        if (!in_arguments)
            if (int rc = take_staging(pool, &slot, &hm, &hdm, &dm)) return rc;
        int32_t at = (i1 - i0) * kRecord, unit = 0;
        for (int i = i0; i < i1; ++i) {
            const int nb = (n_tokens[i] + 15) / 16, mb = (n_keep[i] + 15) / 16;
            const EvictSequence q{at, at + nb, n_tokens[i], n_keep[i], (int32_t)kept_at, unit};
            memcpy(hm + (size_t)(i - i0) * kRecord, &q, sizeof q);
            for (int b = 0; b < nb; ++b) hm[at + b] = src_pages[sp + b / S] * S + b % S;
            for (int b = 0; b < mb; ++b) hm[at + nb + b] = dst_pages[dp + b / S] * S + b % S;
            at += nb + mb;
            unit += mb;
            sp += (nb + S - 1) / S;
            dp += (mb + S - 1) / S;
            kept_at += n_keep[i];
        }
        a.meta = dm;
        a.n_seq = i1 - i0;
        a.n_units = unit;
        a.most_tokens = *std::max_element(n_tokens + i0, n_tokens + i1);
        if (in_arguments) {
            HKV_HIP(launch_evict(a, s));
        } else {
            HKV_HIP(launch_upload(hdm, dm, align_up(sizeof(int32_t) * (size_t)at, 16), s));
            HKV_HIP(launch_evict(static_cast<const EvictLaunch &>(a), s));
            if (int rc = leave_staging(pool, slot, s)) return rc;
        }
        i0 = i1;
    }
    return HKV_OK;
} catch (const std::exception &) {  // (no memory for a list)
    return fail(HKV_ENOMEM, "kv_pool_evict: out of host memory");
}
