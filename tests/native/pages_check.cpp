// Exercises the host side of the calls that move pages (copies between pools, forks, compaction) and of decode plans over 4-bit pools with seeded
// random programs, for a build with AddressSanitizer and UndefinedBehaviorSanitizer.  No GPU and no HIP library: device memory is the host's, and
// the launcher of the copies moves bytes as the kernel does, within the buffers or the sanitizers say so.  Exit status 0 = clean.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "../../paper_2603_16104_amd/csrc/api.cpp"
#include "../../paper_2603_16104_amd/csrc/pages.cpp"

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

// ---- what the copy kernel does to pools of one type
static int inline_copies = 0, listed_copies = 0;
static void move_blocks(const PageCopyLaunch &a, const int32_t *list) {
    CHECK(a.src.dtype == a.dst.dtype && a.src.num_kv_heads == a.dst.num_kv_heads && a.n > 0);
    const size_t codes = (size_t)a.src.num_kv_heads * 2048 * (a.src.dtype == HKV_BF16 ? 16 : 4) / 8, scales = a.src.dtype == HKV_BF16 ? 0 : (size_t)a.src.num_kv_heads * 64;
    auto copy = [](const void *s, const void *d, size_t bytes, int32_t from, int32_t to) {
        if (bytes) std::memcpy(static_cast<char *>(const_cast<void *>(d)) + bytes * to, static_cast<const char *>(s) + bytes * from, bytes);
    };
    std::vector<int32_t> written;
    for (int i = 0; i < a.n; ++i) {
        CHECK(list[3 * i + 2] >= 1 && list[3 * i + 2] <= 16);
        copy(a.src.k_pages, a.dst.k_pages, codes, list[3 * i], list[3 * i + 1]);
        copy(a.src.v_pages, a.dst.v_pages, codes, list[3 * i], list[3 * i + 1]);
        copy(a.src.k_scale, a.dst.k_scale, scales, list[3 * i], list[3 * i + 1]);
        copy(a.src.v_scale, a.dst.v_scale, scales, list[3 * i], list[3 * i + 1]);
        written.push_back(list[3 * i + 1]);
    }
    std::sort(written.begin(), written.end());
    CHECK(std::adjacent_find(written.begin(), written.end()) == written.end());  // (a workgroup per block, in any order)
    if (a.src.k_pages == a.dst.k_pages)
        for (int i = 0; i < a.n; ++i) CHECK(!std::binary_search(written.begin(), written.end(), list[3 * i]));
}
namespace hkv {
hipError_t launch_page_copy(const PageCopyLaunch &a, hipStream_t) {
    ++listed_copies;
    move_blocks(a, a.list);
    return hipSuccess;
}
hipError_t launch_page_copy(const PageCopyInline &a, hipStream_t) {
    ++inline_copies;
    move_blocks(a, a.entries);
    return hipSuccess;
}
hipError_t launch_upload(const void *s, void *d, size_t n, hipStream_t) { std::memcpy(d, s, n); return hipSuccess; }
hipError_t launch_plan_grow_inline(const PlanGrowInline &, hipStream_t) { return hipSuccess; }
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
struct Pool {
    int pages, page, dtype;
    size_t block;  // bytes of a block's codes
    std::vector<char> k, v;
    std::vector<uint8_t> ks, vs;
    hkv_pool *handle = nullptr;
    Pool(int n, int page_size, int type) : pages(n), page(page_size), dtype(type), block(2048u * (type == HKV_BF16 ? 16 : 4) / 8) {
        const size_t blocks = (size_t)n * page / 16;
        k.resize(blocks * block + 16);
        v.resize(blocks * block + 16);
        if (type != HKV_BF16) {
            ks.resize(blocks * 64 + 16);
            vs.resize(blocks * 64 + 16);
        }
        auto aligned = [](auto &x) -> void * { return x.empty() ? nullptr : reinterpret_cast<void *>((reinterpret_cast<uintptr_t>(x.data()) + 15) & ~uintptr_t(15)); };
        hkv_pool_desc d{};
        d.num_pages = n;
        d.page_size = page;
        d.num_kv_heads = 1;
        d.head_dim = 128;
        d.dtype = type;
        d.k_pages = aligned(k);
        d.v_pages = aligned(v);
        d.k_scale = static_cast<float *>(aligned(ks));
        d.v_scale = static_cast<float *>(aligned(vs));
        CHECK(kv_pool_create(&d, &handle) == HKV_OK);
    }
    ~Pool() { kv_pool_destroy(handle); }
    uint32_t *at(int id, int token) {  // a word of the token's own, in V's codes or scales
        const size_t b = (size_t)id * page / 16 + token / 16;
        char *base = dtype == HKV_BF16 ? static_cast<char *>(handle->d.v_pages) + b * block : reinterpret_cast<char *>(handle->d.v_scale) + b * 64;
        return reinterpret_cast<uint32_t *>(base + token % 16 * 4);
    }
};
struct Sequence {
    std::vector<int32_t> ids;
    std::vector<uint32_t> tokens;
};

static void check(Pool &p, const std::vector<Sequence> &all) {
    std::vector<int32_t> owners(p.pages, 0);
    for (const Sequence &s : all) {
        CHECK((int)s.ids.size() == ((int)s.tokens.size() + p.page - 1) / p.page);
        for (int32_t id : s.ids) ++owners[id];
        for (size_t t = 0; t < s.tokens.size(); ++t) CHECK(*p.at(s.ids[t / p.page], t % p.page) == s.tokens[t]);
    }
    int free_pages = 0;
    for (int id = 0; id < p.pages; ++id) {
        CHECK(kv_pool_refcount(p.handle, id) == owners[id]);
        free_pages += owners[id] == 0;
    }
    CHECK(kv_pool_num_free(p.handle) == free_pages);
    std::vector<int32_t> listed(p.handle->free_list.begin(), p.handle->free_list.end());
    std::sort(listed.begin(), listed.end());
    CHECK(std::adjacent_find(listed.begin(), listed.end()) == listed.end());
    for (int32_t id : listed) CHECK(owners[id] == 0);
}

// Sequences begin, grow, fork, end and move, and hold their tokens all the while.
static void pages_program(uint32_t seed) {
    std::mt19937 rng(seed);
    auto below = [&](int n) { return (int)(rng() % (uint32_t)n); };
    const int sizes[] = {16, 32, 128}, counts[] = {5, 60, 1500};
    Pool p(counts[seed % 3], sizes[seed / 3 % 3], seed % 2 ? HKV_FP4_E2M1 : HKV_BF16);
    std::vector<Sequence> all;
    uint32_t stamp = seed << 20;
    for (int step = 0; step < 60; ++step) {
        const int what = below(6);
        if (what == 0 || all.empty()) {
            Sequence s;
            const int n = below(p.page * std::max(2, p.pages / 4));
            s.ids.resize((n + p.page - 1) / p.page);
            if (kv_pool_alloc(p.handle, (int)s.ids.size(), s.ids.data()) != HKV_OK) continue;
            for (int t = 0; t < n; ++t) {
                s.tokens.push_back(++stamp);
                *p.at(s.ids[t / p.page], t % p.page) = stamp;
            }
            all.push_back(s);
        } else if (what == 1) {  // a sequence grows in its last page, which is its own
            Sequence &s = all[below((int)all.size())];
            if (s.tokens.size() % p.page == 0) {
                int32_t id;
                if (kv_pool_alloc(p.handle, 1, &id) != HKV_OK) continue;
                s.ids.push_back(id);
            }
            CHECK(kv_pool_refcount(p.handle, s.ids.back()) == 1);
            *p.at(s.ids.back(), s.tokens.size() % p.page) = ++stamp;
            s.tokens.push_back(stamp);
        } else if (what == 2) {
            const int i = below((int)all.size());
            CHECK(kv_pool_release(p.handle, (int)all[i].ids.size(), all[i].ids.data()) == HKV_OK);
            all.erase(all.begin() + i);
        } else if (what == 3) {
            std::vector<int32_t> ids(p.pages);
            const int32_t moved = kv_pool_compact(p.handle, ids.data(), nullptr);
            CHECK(moved >= 0);
            const int live = p.pages - kv_pool_num_free(p.handle);
            for (int id = 0; id < p.pages; ++id) CHECK(ids[id] < live);
            for (Sequence &s : all)
                for (int32_t &id : s.ids) id = ids[id];
        } else {
            const bool release = below(2);
            const int n = 1 + below((int)all.size());
            std::shuffle(all.begin(), all.end(), rng);
            std::vector<int32_t> ids, tokens, parent;
            for (int i = 0; i < n; ++i) {
                ids.insert(ids.end(), all[i].ids.begin(), all[i].ids.end());
                tokens.push_back((int32_t)all[i].tokens.size());
            }
            int64_t pages = 0;
            for (int j = below(2 * n + 1); j > 0; --j) {
                parent.push_back(below(n));
                pages += (int64_t)all[parent.back()].ids.size();
            }
            std::vector<int32_t> out(pages);
            const int rc = kv_pool_fork(p.handle, n, ids.data(), tokens.data(), (int)parent.size(), parent.data(), release, out.data(), nullptr);
            CHECK(rc == HKV_OK || rc == HKV_ENOMEM);
            if (rc == HKV_OK) {
                std::vector<Sequence> forks;
                size_t at = 0;
                for (int32_t i : parent) {
                    forks.push_back({{out.begin() + at, out.begin() + at + all[i].ids.size()}, all[i].tokens});
                    at += all[i].ids.size();
                }
                if (release) all.erase(all.begin(), all.begin() + n);
                all.insert(all.end(), forks.begin(), forks.end());
            }
        }
        check(p, all);
        if (step % 7 == 0) {  // refused calls change nothing
            int32_t out[4], bad = p.pages, one = 1, two = 2 * p.page, zero = 0, minus = -1;
            CHECK(kv_pool_fork(p.handle, 1, &bad, &one, 1, &zero, 0, out, nullptr) == HKV_ERANGE);
            CHECK(kv_pool_fork(p.handle, 1, &minus, &one, 1, &zero, 0, out, nullptr) == HKV_ERANGE);
            CHECK(kv_pool_fork(p.handle, 1, &zero, &minus, 1, &zero, 0, out, nullptr) == HKV_EINVAL);
            if (!p.handle->free_list.empty()) {
                const int32_t idle[2] = {p.handle->free_list.back(), p.handle->free_list.back()};
                CHECK(kv_pool_fork(p.handle, 1, idle, &one, 1, &zero, 0, out, nullptr) == HKV_EINVAL);
                CHECK(kv_pool_copy_pages(p.handle, idle, p.handle, idle, 1, nullptr, nullptr) == HKV_EINVAL);
                const int32_t from[2] = {idle[0] ? 0 : 1, idle[0] ? 0 : 1};
                CHECK(kv_pool_copy_pages(p.handle, idle, p.handle, from, 2, nullptr, nullptr) == HKV_EINVAL);
            }
            if (!all.empty() && !all[0].ids.empty()) {
                const int32_t id = all[0].ids[0], twice[2] = {id, id};
                CHECK(kv_pool_fork(p.handle, 1, &id, &one, 1, &one, 0, out, nullptr) == HKV_ERANGE);
                if (kv_pool_refcount(p.handle, id) == 1) CHECK(kv_pool_fork(p.handle, 1, twice, &two, 1, &zero, 1, out, nullptr) == HKV_EINVAL);
                capturing = hipStreamCaptureStatusActive;
                if (!p.handle->free_list.empty() && p.page > 1) CHECK(kv_pool_fork(p.handle, 1, &id, &one, 1, &zero, 0, out, nullptr) == HKV_EINVAL);
                CHECK(kv_pool_compact(p.handle, std::vector<int32_t>(p.pages).data(), nullptr) == HKV_EINVAL);
                capturing = hipStreamCaptureStatusNone;
            }
            check(p, all);
        }
    }
}

// Pages go to another pool and back.
static void copies_program(uint32_t seed) {
    std::mt19937 rng(seed);
    const int page = seed % 2 ? 16 : 64, n = seed % 3 ? 40 : 30000 / (page / 16);
    Pool a(n, page, HKV_FP4_E2M1), b(n + 7, page, HKV_FP4_E2M1);
    std::vector<int32_t> from(n), to(n + 7), tokens(n);
    for (int i = 0; i < n; ++i) from[i] = i;
    for (int i = 0; i < n + 7; ++i) to[i] = i;
    std::shuffle(from.begin(), from.end(), rng);
    std::shuffle(to.begin(), to.end(), rng);
    for (int i = 0; i < n; ++i) {
        tokens[i] = (int)(rng() % (uint32_t)(page + 1));
        for (int t = 0; t < page; ++t) *a.at(from[i], t) = (uint32_t)(i * page + t + 1);
    }
    CHECK(kv_pool_copy_pages(b.handle, to.data(), a.handle, from.data(), n, tokens.data(), nullptr) == HKV_OK);
    for (int i = 0; i < n; ++i)
        for (int t = 0; t < page; ++t) CHECK(*b.at(to[i], t) == (t < (tokens[i] + 15) / 16 * 16 ? (uint32_t)(i * page + t + 1) : 0u));
    tokens[n / 2] = page + 1;
    CHECK(kv_pool_copy_pages(b.handle, to.data(), a.handle, from.data(), n, tokens.data(), nullptr) == HKV_EINVAL);
    CHECK(kv_pool_copy_pages(b.handle, to.data(), a.handle, from.data(), -1, nullptr, nullptr) == HKV_EINVAL);
    CHECK(kv_pool_copy_pages(b.handle, nullptr, a.handle, from.data(), 1, nullptr, nullptr) == HKV_EINVAL);
    CHECK(kv_pool_copy_pages(nullptr, nullptr, a.handle, nullptr, 0, nullptr, nullptr) == HKV_EINVAL);
    CHECK(kv_pool_copy_pages(b.handle, nullptr, a.handle, nullptr, 0, nullptr, nullptr) == HKV_OK);
}

// A prefix cache over a pool that is compacted under it.
static void cache_program(uint32_t seed) {
    std::mt19937 rng(seed);
    Pool p(40, 16, HKV_BF16);
    hkv_cache *cache = nullptr, *second = nullptr;
    CHECK(kv_cache_create(p.handle, &cache) == HKV_OK && kv_cache_create(p.handle, &second) == HKV_OK);
    kv_cache_destroy(second);  // (follows no more)
    std::vector<std::vector<int32_t>> held;
    for (int step = 0; step < 80; ++step) {
        const int what = (int)(rng() % 3);
        if (what == 0) {
            const int n = 1 + (int)(rng() % 150), from = (int)(rng() % 3);
            std::vector<int32_t> prompt(n), ids((n + 15) / 16);
            for (int t = 0; t < n; ++t) prompt[t] = t < 40 ? t : t + 1000 * from;
            int32_t cached = 0;
            if (kv_cache_acquire(cache, prompt.data(), n, 0, ids.data(), &cached) >= 0) held.push_back(ids);
        } else if (what == 1 && !held.empty()) {
            const size_t i = rng() % held.size();
            CHECK(kv_cache_release(cache, held[i].data(), (int)held[i].size()) == HKV_OK);
            held.erase(held.begin() + (long)i);
        } else {
            std::vector<int32_t> ids(p.pages);
            CHECK(kv_pool_compact(p.handle, ids.data(), nullptr) >= 0);
            for (auto &list : held)
                for (int32_t &id : list) CHECK((id = ids[id]) >= 0);
        }
    }
    for (auto &list : held) CHECK(kv_cache_release(cache, list.data(), (int)list.size()) == HKV_OK);
    kv_cache_destroy(cache);
    CHECK(kv_pool_num_free(p.handle) == p.pages);
    std::vector<int32_t> ids(p.pages);
    CHECK(kv_pool_compact(p.handle, ids.data(), nullptr) == 0);
}

// Plans over 4-bit pools, made and grown.
static void plans_program(uint32_t seed) {
    std::mt19937 rng(seed);
    const int heads = 1, group = 1 + (int)(rng() % 16), n_req = 1 + (int)(rng() % 90);
    Pool p(4000, 16, HKV_FP4_E2M1);
    std::vector<hkv_node> nodes{{-1, 0, 0, 0}};
    nodes[0].n_tokens = (int)(rng() % 200) * 16;
    nodes[0].n_pages = nodes[0].n_tokens / 16;
    std::vector<int32_t> leaves;
    int at = nodes[0].n_pages;
    for (int r = 0; r < n_req; ++r) {
        const int n = 1 + (int)(rng() % 300);
        leaves.push_back((int32_t)nodes.size());
        nodes.push_back({0, at, (n + 15) / 16, n});
        at += (n + 15) / 16;
    }
    std::vector<int32_t> ids(at);
    CHECK(kv_pool_alloc(p.handle, at, ids.data()) == HKV_OK);
    hkv_decode_plan *plan = nullptr;
    CHECK(hkv_decode_plan_create_growing(p.handle, nodes.data(), (int)nodes.size(), ids.data(), at, leaves.data(), n_req, heads * group, 40, HKV_PLAN_HOST_ONLY, &plan) == HKV_OK);
    if (!plan) return;
    for (int step = 0; step < 40; ++step) {
        std::vector<int32_t> fresh(n_req, -1);
        for (int r = 0; r < n_req; ++r)
            if ((nodes[leaves[r]].n_tokens + step) % 16 == 0) CHECK(kv_pool_alloc(p.handle, 1, &fresh[r]) == HKV_OK);
        CHECK(hkv_decode_plan_append(plan, fresh.data(), nullptr) == HKV_OK);
    }
    int64_t tokens = 0, want = 0;
    for (const DecodeItem &it : plan->items) tokens += (int64_t)it.n_tokens * it.n_req;
    for (int r = 0; r < n_req; ++r) want += nodes[0].n_tokens + nodes[leaves[r]].n_tokens + 40;
    CHECK(tokens == want);
    hkv_decode_plan_destroy(plan);
}

int main() {
    for (uint32_t seed = 0; seed < 36; ++seed) pages_program(seed);
    for (uint32_t seed = 0; seed < 6; ++seed) copies_program(seed);
    for (uint32_t seed = 0; seed < 20; ++seed) cache_program(seed);
    for (uint32_t seed = 0; seed < 20; ++seed) plans_program(seed);
    CHECK(inline_copies > 0 && listed_copies > 0);
    std::printf("%d inline, %d listed copies, %d failed checks\n", inline_copies, listed_copies, failures);
    return failures != 0;
}
