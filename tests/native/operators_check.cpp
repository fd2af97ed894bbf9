// Exercises the host side of the calls around a step's attention (stores of projection rows, weights of cached keys, eviction) with
// seeded random plans, for a build with AddressSanitizer and UndefinedBehaviorSanitizer.  No GPU and no HIP library: device memory is
// the host's, and the launchers are stubs that index what they are given as the kernels do and note what those would read and write, which is then
// compared with the forest.  Exit status 0 = clean.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "../../paper_2603_16104_amd/csrc/api.cpp"
#include "../../paper_2603_16104_amd/csrc/operators.cpp"

static int failures = 0;
#define CHECK(cond)                                                        \
    do {                                                                   \
        if (!(cond)) {                                                     \
            std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #cond); \
            ++failures;                                                    \
        }                                                                  \
    } while (0)

// ---- HIP, as far as the host files call it
static hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
extern "C" {
hipError_t hipMalloc(void **p, size_t n) { return (*p = std::calloc(1, n ? n : 1)) ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind) { if (n) std::memcpy(d, s, n); return hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { return hipMalloc(p, n); }
hipError_t hipHostFree(void *p) { return hipFree(p); }
hipError_t hipHostGetDevicePointer(void **d, void *p, unsigned) { *d = p; return hipSuccess; }
hipError_t hipEventCreate(hipEvent_t *e) { *e = reinterpret_cast<hipEvent_t>(8); return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { return hipEventCreate(e); }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventElapsedTime(float *ms, hipEvent_t, hipEvent_t) { *ms = 0; return hipSuccess; }
hipError_t hipStreamCreateWithFlags(hipStream_t *s, unsigned) { *s = reinterpret_cast<hipStream_t>(8); return hipSuccess; }
hipError_t hipStreamDestroy(hipStream_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = capturing; return hipSuccess; }
hipError_t hipGetDevice(int *) { return hipErrorNoDevice; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t *, int) { return hipErrorNoDevice; }
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "?"; }
}

// ---- what the kernels would do
struct Put {  // slot `slot` of block `block` (one head) gets row `row` of q, k, v, at position `pos`
    int block, slot;
    int64_t row;
    int pos;
    bool operator<(const Put &o) const { return std::make_pair(block, slot) < std::make_pair(o.block, o.slot); }
};
static std::vector<Put> stored;
static int store_launches = 0, weights_launches = 0, evict_launches = 0, inline_evicts = 0;

static void put_unit(const ProjectionLaunch &a, int block, int lo, int hi, int64_t row, int pos) {
    CHECK(0 <= lo && lo < hi && hi <= 16);
    for (int s = lo; s < hi; ++s) {
        const int64_t r = row + s - lo;
        stored.push_back(Put{block, s, a.row_map ? a.row_map[r] : r, pos + s - lo});
    }
}
static int table_block(const ProjectionLaunch &a, int64_t at) { return a.src_pages ? a.src_pages[a.blocks[at]] : a.blocks[at]; }

static std::vector<std::pair<int64_t, int>> keys_seen;  // (token of the forest as page_off * 16 + token, head), times it gets a weight
static std::vector<EvictLaunch> evictions;
static std::vector<std::vector<int32_t>> eviction_lists;

namespace hkv {
hipError_t launch_projection_store(const ProjectionLaunch &a, hipStream_t) {
    ++store_launches;
    const int spans = a.tokens == 1 ? 1 : (a.tokens + 14) / 16 + 1;
    for (int x = 0; x < a.n_requests * spans; ++x) {
        const int r = x / spans, i = x % spans;
        const StoreRequest s = a.requests[r];
        int n = s.tokens;
        if (s.item >= 0) n = a.items[s.item].tok_begin + a.items[s.item].n_tokens;
        const int first = n - a.tokens, b = first / 16 + i;
        if (b * 16 >= n) continue;
        const int lo = std::max(first - b * 16, 0);
        put_unit(a, table_block(a, s.page_off + (uint32_t)b), lo, std::min(n - b * 16, 16), (int64_t)r * a.tokens + (b * 16 + lo - first), s.pos0 + b * 16 + lo);
    }
    return hipSuccess;
}
hipError_t launch_projection_store(const ProjectionPrefill &p, hipStream_t) {
    ++store_launches;
    for (int x = 0; x < p.n_units; ++x) {
        const int i = (int)std::count_if(p.begin, p.begin + kMaxInlineRequests, [&](int32_t b) { return b <= x; }) - 1;
        CHECK(i >= 0 && i < kMaxInlineRequests);
        const int prefix = p.prefix[i], end = prefix + p.tokens[i], b = prefix / 16 + x - p.begin[i];
        const int lo = std::max(prefix - b * 16, 0), pos = b * 16 + lo;
        put_unit(p.base, table_block(p.base, p.table + (int64_t)i * p.table_stride + b), lo, std::min(end - b * 16, 16), (int64_t)p.row0[i] + pos - prefix, pos);
    }
    return hipSuccess;
}
static void grow(const PlanGrowInline &g) {
    for (int i = 0; i < g.n_grow; ++i) ++g.items[g.grow_items[i]].n_tokens;
    for (int r = 0; r < g.n_req; ++r)
        if (g.new_block[r] >= 0) g.pages[g.block_pos[r]] = g.new_block[r];
}
hipError_t launch_projection_append(const ProjectionAppend &p, const PlanGrowInline &g, hipStream_t) {
    ++store_launches;
    const ProjectionLaunch &a = p.base;
    for (int r = 0; r < a.n_requests; ++r) {
        const StoreRequest s = a.requests[r];
        const int n = p.length[r];
        for (int h = 0; h < a.pool.num_kv_heads; ++h) {
            const DecodeItem &item = g.items[g.grow_items[r * a.pool.num_kv_heads + h]];
            CHECK(item.tok_begin + item.n_tokens == n && item.kv_head == h);
        }
        put_unit(a, g.new_block[r] >= 0 ? g.new_block[r] : a.blocks[s.page_off + (uint32_t)(n / 16)], n % 16, n % 16 + 1, r, s.pos0 + n);
    }
    grow(g);
    return hipSuccess;
}
hipError_t launch_key_weights(const KeyWeightsLaunch &a, hipStream_t) {
    ++weights_launches;
    const int G = a.num_q_heads / a.pool.num_kv_heads;
    if (a.pool.dtype == HKV_FP32) {
        for (int x = 0; x < a.n_items; ++x) {
            const KeyWeightItem &it = a.items[x];
            CHECK(it.length % 128 == 0 && it.length <= kMaxWeightTokens && (it.n_req * G <= 16 || it.length == 128) && it.tok_begin < it.tokens);
            for (int j = 0; j < it.n_req; ++j) {
                const int row = a.node_req_idx[it.req_off + j];
                CHECK(row >= 0 && (!a.row_leaf || (a.row_leaf[row] >= 0 && a.row_limit[row] >= 0 && (a.row_mask[row] & 1))));
            }
            for (int t = it.tok_begin; t < std::min(it.tok_begin + it.length, it.tokens); ++t)
                keys_seen.push_back({((int64_t)a.pages[it.page_off + (t - it.tok_begin) / 16] * a.pool.num_kv_heads + it.kv_head) * 16 + t % 16, it.n_req});
        }
        return hipSuccess;
    }
    CHECK(a.n_items % kWeightWaves == 0);
    for (int x = 0; x < a.n_items; ++x) {
        const KeyWeightItem &it = a.items[x];
        const bool many = it.n_req * G > 16;
        if (x % kWeightWaves) {  // a workgroup is of one kind; of many rows, all its wavefronts have the same item
            const KeyWeightItem &before = a.items[x - 1];
            CHECK((before.n_req * G > 16) == many);
            if (many) {
                CHECK(!std::memcmp(&before, &it, sizeof it));
                continue;
            }
        }
        int n_node = it.tokens;
        if (it.item >= 0) n_node = a.plan_items[it.item].tok_begin + a.plan_items[it.item].n_tokens;
        const int n = std::min(it.length, n_node - it.tok_begin);
        if (n <= 0) continue;
        CHECK(it.length % 32 == 0 && it.length <= kMaxWeightTokens && it.tok_begin % 32 == 0 && (n + 15) / 16 <= 64);
        if (many) CHECK(it.length == 32 || it.length == 64 || it.length == 128 || it.length % 256 == 0);
        for (int j = 0; j < it.n_req; ++j) CHECK(a.node_req_idx[it.req_off + j] >= 0);
        for (int t = 0; t < n; ++t) keys_seen.push_back({((int64_t)a.pages[it.page_off + t / 16] * a.pool.num_kv_heads + it.kv_head) * 16 + t % 16, it.n_req});
    }
    return hipSuccess;
}
static void evict(const EvictLaunch &a, const int32_t *meta) {
    ++evict_launches;
    int unit = 0;
    for (int i = 0; i < a.n_seq; ++i) {
        EvictSequence q;
        std::memcpy(&q, meta + (size_t)i * sizeof q / 4, sizeof q);
        CHECK(q.unit == unit && q.tokens <= a.most_tokens && q.keep <= q.tokens);
        unit += (q.keep + 15) / 16;
        std::vector<int32_t> list{q.tokens, q.keep, q.kept};
        list.insert(list.end(), meta + q.src, meta + q.src + (q.tokens + 15) / 16);
        list.insert(list.end(), meta + q.dst, meta + q.dst + (q.keep + 15) / 16);
        eviction_lists.push_back(list);
    }
    CHECK(unit == a.n_units);
    evictions.push_back(a);
}
hipError_t launch_evict(const EvictLaunch &a, hipStream_t) { evict(a, a.meta); return hipSuccess; }
hipError_t launch_evict(const EvictInline &a, hipStream_t) { ++inline_evicts; evict(a, a.list); return hipSuccess; }

hipError_t launch_upload(const void *s, void *d, size_t n, hipStream_t) { std::memcpy(d, s, n); return hipSuccess; }
hipError_t launch_plan_grow_inline(const PlanGrowInline &g, hipStream_t) { grow(g); return hipSuccess; }
hipError_t launch_pool_write(const PoolWriteLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_pool_copy(const PoolCopyLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_pool_append_inline(const PoolAppendInline &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_step_append(const PoolAppendInline &, const PlanGrowInline &, hipStream_t) { return hipSuccess; }
hipError_t launch_pool_dequant(const PoolDequantLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode(const DecodeLaunch &, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t launch_decode_paths(const DecodePathLaunch &, int, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t prepare_decode_device(void **ws) {
    if (ws) *ws = nullptr;
    return hipSuccess;
}
hipError_t launch_rows_fp32(const RowsLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_pool_write_fp32(const PoolWriteLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_prefill(const PrefillLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_tiles(const DecodeTilesLaunch &, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t launch_decode_fused(const DecodeLaunch &, const DecodeTilesLaunch &, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t launch_lse_merge(const float *, const float *, const int32_t *, const int32_t *, int32_t, void *, int32_t, float *,
                            hipStream_t) { return hipSuccess; }
hipError_t launch_lse_merge_dense(const void *, const float *, const int32_t *, int32_t, int32_t, int32_t, void *, int32_t,
                                  float *, hipStream_t, hipEvent_t, hipEvent_t, const int32_t *, const float *) { return hipSuccess; }
hipError_t run_read_probe(const void *const *, int, size_t, int, int, float *, hipStream_t) { return hipSuccess; }
hipError_t run_mfma_probe(int, int, int, int, float *, float *, hipStream_t) { return hipSuccess; }
int prefill_tile_tokens(int group) { return 256 / group; }
}  // namespace hkv

// ---- the programs
template <class T>
static T *at(uintptr_t x) { return reinterpret_cast<T *>(x); }

static hkv_pool *make_pool(int num_pages, int page, int heads, int dtype) {
    hkv_pool_desc d{};
    d.num_pages = num_pages;
    d.page_size = page;
    d.num_kv_heads = heads;
    d.head_dim = 128;
    d.dtype = dtype;
    d.k_pages = at<void>(0x10000);  // never dereferenced
    d.v_pages = at<void>(0x20000);
    d.k_scale = at<float>(0x30000);
    d.v_scale = at<float>(0x40000);
    hkv_pool *p = nullptr;
    CHECK(kv_pool_create(&d, &p) == HKV_OK);
    return p;
}
static hkv_qkv make_rows() {
    hkv_qkv x{};
    x.q = at<void>(0x100000);
    x.k = at<void>(0x200000);
    x.v = at<void>(0x300000);
    x.q_out = at<void>(0x400000);
    return x;
}
static std::vector<Put> taken() {
    std::vector<Put> p;
    p.swap(stored);
    std::sort(p.begin(), p.end());
    return p;
}
static bool same(const std::vector<Put> &a, const std::vector<Put> &b) {
    return a.size() == b.size() && std::equal(a.begin(), a.end(), b.begin(), [](const Put &x, const Put &y) {
               return x.block == y.block && x.slot == y.slot && x.row == y.row && x.pos == y.pos;
           });
}
static int pick(std::mt19937 &rng, int n) { return (int)(rng() % (uint32_t)n); }

static void prefill_stores(std::mt19937 &rng) {
    for (int trial = 0; trial < 60; ++trial) {
        const int P = 16 << pick(rng, 4), S = P / 16, heads = 1 + pick(rng, 4), dtype = trial % 3;
        const int n = trial < 6 ? 120 + pick(rng, 150) : 1 + pick(rng, 20);
        std::vector<int32_t> cu{0}, kv(n);
        int most = 1;
        for (int r = 0; r < n; ++r) {
            const int fresh = pick(rng, 5) ? pick(rng, 60) : 0;
            kv[r] = fresh + pick(rng, 100);
            cu.push_back(cu.back() + fresh);
            most = std::max(most, (kv[r] + P - 1) / P);
        }
        hkv_pool *pool = make_pool(n * most, P, heads, dtype);
        std::vector<int32_t> table((size_t)n * most);
        for (size_t i = 0; i < table.size(); ++i) table[i] = (int32_t)i;
        std::shuffle(table.begin(), table.end(), rng);
        hkv_prefill_plan *plan = nullptr;
        CHECK(hkv_prefill_plan_create(pool, cu.data(), table.data(), most, kv.data(), n, heads * 2, 0, &plan) == HKV_OK);
        if (!plan) continue;
        std::vector<Put> want;
        for (int r = 0; r < n; ++r) {
            const int s = cu[r + 1] - cu[r];
            for (int i = 0; i < s; ++i) {
                const int t = kv[r] - s + i;
                want.push_back(Put{table[(size_t)r * most + t / P] * S + t % P / 16, t % 16, cu[r] + i, t});
            }
        }
        std::sort(want.begin(), want.end());
        const hkv_qkv x = make_rows();
        for (int again = 0; again < 2; ++again) {
            CHECK(hkv_prefill_plan_store(plan, &x, nullptr) == HKV_OK);
            CHECK(same(taken(), want));
        }
        CHECK(hkv_prefill_plan_destroy(plan) == HKV_OK);
        CHECK(kv_pool_destroy(pool) == HKV_OK);
    }
}

// A forest whose nodes have blocks of their own; the weights' work list and the stores of decode plans, growing ones among them.
static void decode_plans(std::mt19937 &rng) {
    int shared_nodes = 0;
    for (int trial = 0; trial < 120; ++trial) {
        const int dtype = trial % 5 == 4 ? HKV_FP32 : trial & 1 ? HKV_FP8_E4M3 : HKV_BF16, P = 16 << pick(rng, 4), S = P / 16, heads = 1 + pick(rng, 9), group = 1 + pick(rng, 16);
        const bool growing = dtype != HKV_FP32 && trial % 3 == 1;
        const int T = growing ? 1 : pick(rng, 3) ? 1 : 1 + pick(rng, dtype == HKV_FP32 ? 16 : 40);
        const int n = trial < 8 ? 257 + pick(rng, 60) : 1 + pick(rng, 40), reserve = growing ? 1 + pick(rng, 3 * P) : 0;
        std::vector<hkv_node> nodes;
        std::vector<int32_t> pages, leaf;
        int fresh_page = 0;
        auto add = [&](int parent, int tokens) {
            nodes.push_back(hkv_node{parent, (int32_t)pages.size(), (tokens + P - 1) / P, tokens});
            for (int j = 0; j < (tokens + P - 1) / P; ++j) pages.push_back(fresh_page++);
            return (int)nodes.size() - 1;
        };
        const int roots = 1 + pick(rng, 3);
        std::vector<int> tips;
        for (int i = 0; i < roots; ++i) {
            int v = add(-1, P * pick(rng, trial % 10 == 0 ? 300 : 9));
            if (pick(rng, 2)) v = add(v, P * (1 + pick(rng, 4)));
            tips.push_back(v);
        }
        std::vector<int32_t> len(n), pos0(n);
        for (int r = 0; r < n; ++r) {
            const int tip = tips[pick(rng, roots)];
            len[r] = T + pick(rng, pick(rng, 4) ? 80 : 700);
            leaf.push_back(add(tip, len[r]));
            for (int v = tip; v >= 0; v = nodes[v].parent) pos0[r] += nodes[v].n_tokens;
        }
        hkv_pool *pool = make_pool(fresh_page + n * (reserve / P + 2), P, heads, dtype);
        hkv_decode_plan_params params{};
        params.tokens_per_req = T;
        params.reserve_tokens = reserve;
        std::vector<uint64_t> visible;  // (a causal run, as a tree's masks)
        for (int i = 0; i < n * T; ++i) visible.push_back((2ull << (i % T)) - 1);
        if (T > 16) params.visible = visible.data();
        std::vector<int32_t> q_rows(n * T);
        for (int i = 0; i < n * T; ++i) q_rows[i] = i;
        if (dtype != HKV_FP32 && pick(rng, 2)) {
            std::shuffle(q_rows.begin(), q_rows.end(), rng);
            params.q_rows = q_rows.data();
        }
        hkv_decode_plan *plan = nullptr;
        CHECK(hkv_decode_plan_create_ex(pool, nodes.data(), (int32_t)nodes.size(), pages.data(), (int32_t)pages.size(), leaf.data(), n, heads * group, 0, &params, &plan) == HKV_OK);
        if (!plan) {
            std::fprintf(stderr, "%s\n", hkv_last_error());
            kv_pool_destroy(pool);
            continue;
        }
        std::vector<std::vector<int32_t>> own(n);  // the leaves' pages
        for (int r = 0; r < n; ++r) own[r].assign(pages.begin() + nodes[leaf[r]].page_begin, pages.begin() + nodes[leaf[r]].page_begin + nodes[leaf[r]].n_pages);
        auto newest = [&]() {
            std::vector<Put> want;
            for (int r = 0; r < n; ++r)
                for (int i = 0; i < T; ++i) {
                    const int t = len[r] - T + i;
                    want.push_back(Put{own[r][t / P] * S + t % P / 16, t % 16, q_rows[r * T + i], pos0[r] + t});
                }
            std::sort(want.begin(), want.end());
            return want;
        };
        const hkv_qkv x = make_rows();
        const int steps = growing ? std::min(reserve, 2 + pick(rng, 40)) : 0, track = pick(rng, steps + 1);
        auto weights = [&]() {
            CHECK(attn_decode_plan_weights(plan, x.q, 0.1f, at<float>(0x500000), 1.f, std::min(T, 1), at<float>(0x600000), nullptr) == HKV_OK);
            std::vector<std::pair<int64_t, int>> want;
            std::vector<int> below(nodes.size(), 0);
            for (int r = 0; r < n; ++r)
                for (int v = leaf[r]; v >= 0; v = nodes[v].parent) below[v] += T;
            for (size_t v = 0; v < nodes.size(); ++v) {
                const auto r = std::find(leaf.begin(), leaf.end(), (int32_t)v) - leaf.begin();
                const int tokens = r < n ? len[r] : nodes[v].n_tokens;
                shared_nodes += below[v] * group > 16 && tokens > 0;
                for (int t = 0; below[v] && t < tokens; ++t)
                    for (int h = 0; h < heads; ++h) {
                        const int page = r < n ? own[r][t / P] : pages[nodes[v].page_begin + t / P];
                        want.push_back({((int64_t)(page * S + t % P / 16) * heads + h) * 16 + t % 16, below[v]});
                    }
            }
            std::sort(want.begin(), want.end());
            std::sort(keys_seen.begin(), keys_seen.end());
            CHECK(keys_seen == want);
            keys_seen.clear();
        };
        for (int step = 0;; ++step) {
            CHECK(hkv_decode_plan_store(plan, &x, nullptr) == HKV_OK);
            CHECK(same(taken(), newest()));
            if (step == track) CHECK(hkv_decode_plan_track_weights(plan) == HKV_OK);
            if (step >= track && step % 4 == track % 4) weights();
            if (step == steps) break;
            std::vector<int32_t> ids(n, -1);
            for (int r = 0; r < n; ++r) {
                if (len[r] % P == 0) own[r].push_back(ids[r] = fresh_page++);
                ++len[r];
            }
            CHECK(hkv_decode_plan_append_qkv(plan, ids.data(), &x, nullptr) == HKV_OK);
            CHECK(same(taken(), newest()));
        }
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
        CHECK(kv_pool_destroy(pool) == HKV_OK);
    }
    CHECK(shared_nodes > 100);
}

// A last node without a token; and an append that is refused leaves the plan as it was.
static void refusals() {
    hkv_pool *pool = make_pool(8, 16, 2, HKV_BF16);
    const hkv_qkv x = make_rows();
    const int32_t leaf[2] = {0, 1}, pages[2] = {0, 7}, far[2] = {3, 9}, twice[2] = {3, 3}, good[2] = {3, 5}, more[2] = {1, 2};
    const hkv_node full[2] = {{-1, 0, 1, 16}, {-1, 1, 1, 16}}, part[2] = {{-1, 0, 0, 0}, {-1, 0, 1, 5}};
    hkv_decode_plan *plan = nullptr;
    CHECK(hkv_decode_plan_create(pool, part, 2, pages, 1, leaf, 2, 4, 0, &plan) == HKV_OK);
    if (plan) {
        CHECK(hkv_decode_plan_store(plan, &x, nullptr) == HKV_EINVAL && stored.empty());
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
    }
    CHECK(hkv_decode_plan_create_growing(pool, full, 2, pages, 2, leaf, 2, 4, 20, 0, &plan) == HKV_OK);
    if (plan) {
        CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_EINVAL);
        CHECK(hkv_decode_plan_append_qkv(plan, far, &x, nullptr) == HKV_ERANGE);
        CHECK(hkv_decode_plan_append_qkv(plan, twice, &x, nullptr) == HKV_EINVAL);
        CHECK(stored.empty());
        CHECK(hkv_decode_plan_append_qkv(plan, good, &x, nullptr) == HKV_OK);
        CHECK(same(taken(), {Put{3, 0, 0, 16}, Put{5, 0, 1, 16}}));
        for (int i = 1; i < 20; ++i) CHECK(hkv_decode_plan_append_qkv(plan, i == 16 ? more : nullptr, &x, nullptr) == HKV_OK);
        stored.clear();
        CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_ENOMEM && stored.empty());
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
    }
    CHECK(kv_pool_destroy(pool) == HKV_OK);
}

static void evictions_of(std::mt19937 &rng) {
    for (int trial = 0; trial < 80; ++trial) {
        const int P = 16 << pick(rng, 4), S = P / 16, heads = 1 + pick(rng, 4);
        const int n = 1 + pick(rng, trial % 8 == 0 ? 300 : 12), most = trial % 8 == 1 ? 500000 : trial & 1 ? 3000 : 200, first = pick(rng, 5), recent = pick(rng, 40);
        std::vector<int32_t> tokens(n), keep(n), src, dst;
        std::vector<std::vector<int32_t>> want;
        int fresh_page = 0, kept = 0;
        std::vector<int32_t> head;
        for (int i = 0; i < n; ++i) {
            tokens[i] = pick(rng, 6) ? pick(rng, most) : 0;
            keep[i] = std::min(tokens[i], first + recent) + (pick(rng, 3) ? pick(rng, std::max(1, tokens[i] - first - recent)) : 0);
            keep[i] = std::min(keep[i], tokens[i]);
            std::vector<int32_t> list{tokens[i], keep[i], kept};
            kept += keep[i];
            const int shared = pick(rng, 2) && !src.empty() ? 1 : 0;  // (a shared first page)
            std::vector<int32_t> s, d;
            for (int j = 0; j < (tokens[i] + P - 1) / P; ++j) s.push_back(shared && j == 0 ? src[0] : fresh_page++);
            for (int j = 0; j < (keep[i] + P - 1) / P; ++j) d.push_back(fresh_page++);
            for (int j = 0; j < (tokens[i] + 15) / 16; ++j) list.push_back(s[j / S] * S + j % S);
            for (int j = 0; j < (keep[i] + 15) / 16; ++j) list.push_back(d[j / S] * S + j % S);
            src.insert(src.end(), s.begin(), s.end());
            dst.insert(dst.end(), d.begin(), d.end());
            want.push_back(list);
        }
        hkv_pool *pool = make_pool(fresh_page + 1, P, heads, trial % 3);
        auto run = [&]() { return kv_pool_evict(pool, n, src.data(), tokens.data(), dst.data(), keep.data(), first, recent, at<float>(0x100000), at<int32_t>(0x200000), nullptr); };
        CHECK(run() == HKV_OK);
        if (kept == 0) {
            CHECK(eviction_lists.empty());
        } else {
            CHECK(eviction_lists == want);
            for (const EvictLaunch &a : evictions) CHECK(a.total == kept && a.n_first == first && a.n_recent == recent);
            eviction_lists.clear();
            capturing = hipStreamCaptureStatusActive;
            CHECK(run() == HKV_EINVAL && eviction_lists.empty());
            capturing = hipStreamCaptureStatusNone;
        }
        evictions.clear();
        CHECK(kv_pool_destroy(pool) == HKV_OK);
    }
    CHECK(inline_evicts > 10 && evict_launches > inline_evicts + 10);
}

int main() {
    std::mt19937 rng(20261206u);
    prefill_stores(rng);
    decode_plans(rng);
    refusals();
    evictions_of(rng);
    std::printf("operators_check: %d stores, %d weights, %d evictions, %d failed checks\n", store_launches, weights_launches, evict_launches, failures);
    return failures ? 1 : 0;
}
