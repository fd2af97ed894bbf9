// Lives of pools, caches, pages and lists that end in an unusual order, for a build with AddressSanitizer and UndefinedBehaviorSanitizer: the host
// files as they are, no GPU and no HIP library (launches do nothing unless a program says otherwise).  Argument: the program.  Exit status 0 = clean.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <numeric>
#include <vector>

#include "../../paper_2603_16104_amd/csrc/hkv_objects.h"

static int failures = 0;
#define CHECK(cond)                                                        \
    do {                                                                   \
        if (!(cond)) {                                                     \
            std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #cond); \
            ++failures;                                                    \
        }                                                                  \
    } while (0)

using namespace hkv;

// ---- HIP, as far as the host files call it
static intptr_t events = 0;
extern "C" {
hipError_t hipMalloc(void **p, size_t n) { return (*p = std::calloc(1, n ? n : 1)) ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind) { if (n) std::memcpy(d, s, n); return hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { return hipMalloc(p, n); }
hipError_t hipHostFree(void *p) { return hipFree(p); }
hipError_t hipHostGetDevicePointer(void **d, void *p, unsigned) { *d = p; return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { *e = reinterpret_cast<hipEvent_t>(++events); return hipSuccess; }
hipError_t hipEventCreate(hipEvent_t *e) { return hipEventCreateWithFlags(e, 0); }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t);
hipError_t hipEventSynchronize(hipEvent_t);
hipError_t hipEventElapsedTime(float *ms, hipEvent_t, hipEvent_t) { *ms = 0; return hipSuccess; }
hipError_t hipStreamCreateWithFlags(hipStream_t *s, unsigned) { *s = reinterpret_cast<hipStream_t>(8); return hipSuccess; }
hipError_t hipStreamDestroy(hipStream_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipGetDevice(int *) { return hipErrorNoDevice; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t *, int) { return hipErrorNoDevice; }
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "?"; }
}
// Uploads that read a list are on their way until an event recorded behind them has been waited for.
static std::map<const void *, hipEvent_t> on_their_way;  // by the list's address: the event behind it (null: none yet)
static int overtaken = 0, launches_until_failure = -1;
hipError_t hipEventRecord(hipEvent_t e, hipStream_t) {
    for (auto &u : on_their_way)
        if (!u.second) u.second = e;
    return hipSuccess;
}
hipError_t hipEventSynchronize(hipEvent_t e) {
    for (auto u = on_their_way.begin(); u != on_their_way.end();) u = u->second == e ? on_their_way.erase(u) : std::next(u);
    return hipSuccess;
}
static hipError_t launched() { return launches_until_failure-- == 0 ? hipErrorInvalidValue : hipSuccess; }

namespace hkv {
hipError_t launch_page_copy(const PageCopyLaunch &, hipStream_t) { return launched(); }
hipError_t launch_page_copy(const PageCopyInline &, hipStream_t) { return hipSuccess; }
hipError_t launch_upload(const void *s, void *d, size_t n, hipStream_t) {
    overtaken += !on_their_way.insert({s, nullptr}).second;  // (the list was written anew under an upload)
    std::memcpy(d, s, n);
    return launched();
}
hipError_t launch_evict(const EvictLaunch &, hipStream_t) { return launched(); }
hipError_t launch_evict(const EvictInline &, hipStream_t) { return launched(); }
hipError_t launch_projection_store(const ProjectionLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_projection_store(const ProjectionPrefill &, hipStream_t) { return hipSuccess; }
hipError_t launch_projection_append(const ProjectionAppend &, const PlanGrowInline &, hipStream_t) { return hipSuccess; }
hipError_t launch_key_weights(const KeyWeightsLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_plan_grow_inline(const PlanGrowInline &, hipStream_t) { return hipSuccess; }
hipError_t launch_pool_write(const PoolWriteLaunch &, hipStream_t) { return launched(); }
hipError_t launch_pool_write_fp32(const PoolWriteLaunch &, hipStream_t) { return launched(); }
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
hipError_t launch_prefill(const PrefillLaunch &, hipStream_t) { return hipSuccess; }
hipError_t launch_decode_tiles(const DecodeTilesLaunch &, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t launch_decode_fused(const DecodeLaunch &, const DecodeTilesLaunch &, hipStream_t, hipEvent_t, hipEvent_t) { return hipSuccess; }
hipError_t launch_lse_merge(const float *, const float *, const int32_t *, const int32_t *, int32_t, void *, int32_t, float *, hipStream_t) { return hipSuccess; }
hipError_t launch_lse_merge_dense(const void *, const float *, const int32_t *, int32_t, int32_t, int32_t, void *, int32_t, float *, hipStream_t, hipEvent_t, hipEvent_t,
                                  const int32_t *, const float *) { return hipSuccess; }
hipError_t run_read_probe(const void *const *, int, size_t, int, int, float *, hipStream_t) { return hipSuccess; }
hipError_t run_mfma_probe(int, int, int, int, float *, float *, hipStream_t) { return hipSuccess; }
int prefill_tile_tokens(int group) { return 256 / group; }
}  // namespace hkv

static hkv_pool *make_pool(int pages, int page_size = 16, int dtype = HKV_BF16, void *k = reinterpret_cast<void *>(0x100000), void *v = reinterpret_cast<void *>(0x40000000)) {
    hkv_pool_desc d{};
    d.num_pages = pages;
    d.page_size = page_size;
    d.num_kv_heads = 2;
    d.head_dim = 128;
    d.dtype = dtype;
    d.k_pages = k;
    d.v_pages = v;
    if (dtype == HKV_FP8_E4M3 || dtype == HKV_FP4_E2M1) {
        d.k_scale = reinterpret_cast<float *>(0x80000000);
        d.v_scale = reinterpret_cast<float *>(0xC0000000);
    }
    hkv_pool *pool = nullptr;
    CHECK(kv_pool_create(&d, &pool) == HKV_OK);
    return pool;
}
static std::vector<int32_t> acquire(hkv_cache *cache, int n, int first = 0, int want = HKV_OK) {
    std::vector<int32_t> tokens(n), ids((n + 15) / 16);
    std::iota(tokens.begin(), tokens.end(), first);
    int32_t cached = 0;
    CHECK(kv_cache_acquire(cache, tokens.data(), n, 0, ids.data(), &cached) == want);
    return ids;
}

// A cache that outlives its pool: never used, with blocks, with a sequence's pages still out; and one that does not.
static void caches_after_their_pool() {
    for (int used = 0; used < 3; ++used) {
        hkv_pool *pool = make_pool(8);
        hkv_cache *cache = nullptr, *early = nullptr;
        CHECK(kv_cache_create(pool, &early) == HKV_OK && kv_cache_create(pool, &cache) == HKV_OK);
        CHECK(kv_cache_destroy(early) == HKV_OK);
        std::vector<int32_t> ids(1, 0);
        if (used) ids = acquire(cache, 40);
        if (used == 1) CHECK(kv_cache_release(cache, ids.data(), (int)ids.size()) == HKV_OK);
        CHECK(kv_pool_destroy(pool) == HKV_OK);
        if (used) {
            acquire(cache, 10, 0, HKV_EINVAL);  // there is nothing that it could take pages from, or give them back to
            CHECK(kv_cache_unpin(cache, ids.data(), (int)ids.size()) == HKV_OK);
            CHECK(kv_cache_release(cache, ids.data(), (int)ids.size()) == (used == 1 ? HKV_ERANGE : HKV_OK));
            int64_t blocks = -1;
            CHECK(kv_cache_stats(cache, &blocks, nullptr, nullptr, nullptr) == HKV_OK && blocks == 2);
        }
        CHECK(kv_cache_destroy(cache) == HKV_OK);
    }
}

// Branches of a cached prompt go on when the cache no longer needs its blocks: their pages have another owner and go to nobody else.
static void evictions_beside_forks() {
    hkv_pool *pool = make_pool(8);
    hkv_cache *cache = nullptr;
    CHECK(kv_cache_create(pool, &cache) == HKV_OK);
    const std::vector<int32_t> old = acquire(cache, 32), young = acquire(cache, 16, 1000);
    std::vector<int32_t> fork(2);
    const int32_t n = 32, parent = 0;
    CHECK(kv_pool_fork(pool, 1, old.data(), &n, 1, &parent, 0, fork.data(), nullptr) == HKV_OK && fork == old);
    CHECK(kv_cache_release(cache, old.data(), 2) == HKV_OK && kv_cache_release(cache, young.data(), 1) == HKV_OK);
    const std::vector<int32_t> rest = acquire(cache, 80, 2000);  // the free pages
    CHECK(kv_pool_num_free(pool) == 0);
    const std::vector<int32_t> one = acquire(cache, 16, 3000);   // the oldest block is the fork's last page: the younger one's goes
    CHECK(one == young);
    acquire(cache, 16, 4000, HKV_ENOMEM);
    CHECK(kv_pool_refcount(pool, fork[0]) == 2 && kv_pool_refcount(pool, fork[1]) == 2);
    CHECK(acquire(cache, 32) == old && kv_cache_release(cache, old.data(), 2) == HKV_OK);  // still cached
    CHECK(kv_pool_release(pool, 2, fork.data()) == HKV_OK);
    const std::vector<int32_t> two = acquire(cache, 16, 4000);
    CHECK(two[0] == old[1]);
    CHECK(kv_cache_destroy(cache) == HKV_OK && kv_pool_num_free(pool) == 8);
    CHECK(kv_pool_destroy(pool) == HKV_OK);
}

// A fork that ends its sequences gives back what they hold, never a prefix cache's own references.
static void forks_that_end_cached_sequences() {
    hkv_pool *pool = make_pool(8);
    hkv_cache *cache = nullptr, *other = nullptr;
    CHECK(kv_cache_create(pool, &other) == HKV_OK && kv_cache_create(pool, &cache) == HKV_OK);
    const std::vector<int32_t> ids = acquire(cache, 40);  // two cached blocks and a private one
    const int32_t n = 40, full = 32, last = 8, parent[3] = {0, 0, 0};
    std::vector<int32_t> out(9, -5);
    auto counts = [&] { std::vector<int32_t> c; for (int i = 0; i < 8; ++i) c.push_back(kv_pool_refcount(pool, i)); return c; };
    const std::vector<int32_t> before = counts();
    for (int forks = 0; forks < 4; ++forks) {
        CHECK(kv_pool_fork(pool, 1, ids.data(), &n, forks, parent, 1, out.data(), nullptr) == HKV_EINVAL);
        CHECK(kv_pool_fork(pool, 1, ids.data(), &full, forks, parent, 1, out.data(), nullptr) == HKV_EINVAL);
        CHECK(kv_pool_fork(pool, 1, &ids[2], &last, forks, parent, 1, out.data(), nullptr) == HKV_EINVAL);
    }
    CHECK(counts() == before && kv_pool_num_free(pool) == 5 && out[0] == -5);
    // a sequence of its own over the same pages: forked, then ended by the next fork; the cache keeps its references
    CHECK(kv_pool_fork(pool, 1, ids.data(), &n, 2, parent, 0, out.data(), nullptr) == HKV_OK);
    const std::vector<int32_t> beams(out.begin(), out.begin() + 6);
    const int32_t lengths[2] = {40, 40}, both[2] = {1, 1};
    CHECK(kv_pool_fork(pool, 2, beams.data(), lengths, 2, both, 1, out.data(), nullptr) == HKV_OK);
    CHECK(kv_pool_refcount(pool, ids[0]) == 3 && kv_pool_refcount(pool, ids[2]) == 1);
    const std::vector<int32_t> now(out.begin(), out.begin() + 6);
    CHECK(kv_pool_fork(pool, 2, now.data(), lengths, 0, both, 1, out.data(), nullptr) == HKV_OK);
    CHECK(counts() == before && kv_pool_num_free(pool) == 5);
    CHECK(kv_cache_release(cache, ids.data(), 3) == HKV_OK && acquire(cache, 32) == std::vector<int32_t>(ids.begin(), ids.begin() + 2));
    CHECK(kv_cache_destroy(cache) == HKV_OK && kv_pool_num_free(pool) == 8);
    // pages that a cache held once are like any others
    std::vector<int32_t> mine(3);
    CHECK(kv_pool_alloc(pool, 3, mine.data()) == HKV_OK);
    CHECK(kv_pool_fork(pool, 1, mine.data(), &n, 1, parent, 1, out.data(), nullptr) == HKV_OK);
    CHECK(kv_cache_destroy(other) == HKV_OK && kv_pool_destroy(pool) == HKV_OK);
}

// Pools that share bytes: a page that is read is not written in the same call, whatever its ids in the two pools are.
static void copies_between_pools_that_overlap() {
    char *const k = reinterpret_cast<char *>(0x100000), *const v = reinterpret_cast<char *>(0x40000000);
    constexpr int kPageBytes = 2 * 2048 * 2;  // bf16, two heads
    auto copy = [](hkv_pool *dst, std::vector<int32_t> to, hkv_pool *src, std::vector<int32_t> from) {
        const int rc = kv_pool_copy_pages(dst, to.data(), src, from.data(), (int)to.size(), nullptr, nullptr);
        CHECK(rc == HKV_OK || !std::strncmp(hkv_last_error(), "kv_pool_copy_pages: page", 24));
        return rc;
    };
    hkv_pool *a = make_pool(8, 16, HKV_BF16, k, v);
    {  // the same type, two pages further on; K alone, V alone
        for (const int both : {0, 1, 2}) {
            hkv_pool *b = make_pool(8, 16, HKV_BF16, both == 2 ? k + 0x20000000 : k + 2 * kPageBytes, both == 1 ? v + 0x20000000 : v + 2 * kPageBytes);
            CHECK(copy(b, {3}, a, {5}) == HKV_EINVAL && copy(a, {5}, b, {3}) == HKV_EINVAL);
            CHECK(copy(b, {3}, a, {3}) == HKV_OK && copy(a, {4}, b, {3}) == HKV_OK);
            CHECK(copy(b, {0, 1, 2}, a, {0, 1, 4}) == HKV_EINVAL);  // written as b's page 2, read as a's page 4
            CHECK(copy(b, {0, 1, 7}, a, {0, 1, 4}) == HKV_OK);
            CHECK(kv_pool_destroy(b) == HKV_OK);
        }
    }
    {  // K of one pool is V of the other
        hkv_pool *b = make_pool(8, 16, HKV_BF16, v, v + 0x20000000);
        CHECK(copy(b, {3}, a, {3}) == HKV_EINVAL && copy(b, {3}, a, {4}) == HKV_OK);
        CHECK(kv_pool_destroy(b) == HKV_OK);
    }
    {  // another type over the same bytes: bf16 page 1 is fp8 pages 2 and 3, fp4 pages 4 to 7, half of fp32 page 0
        hkv_pool *eight = make_pool(16, 16, HKV_FP8_E4M3, k, v), *four = make_pool(32, 16, HKV_FP4_E2M1, k, v), *wide = make_pool(4, 16, HKV_FP32, k, v);
        CHECK(copy(eight, {1}, a, {1}) == HKV_OK && copy(eight, {2}, a, {1}) == HKV_EINVAL && copy(eight, {3}, a, {1}) == HKV_EINVAL && copy(eight, {4}, a, {1}) == HKV_OK);
        CHECK(copy(four, {1}, a, {1}) == HKV_OK && copy(four, {3}, a, {1}) == HKV_OK && copy(four, {4}, a, {1}) == HKV_EINVAL && copy(four, {7}, a, {1}) == HKV_EINVAL &&
              copy(four, {8}, a, {1}) == HKV_OK);
        CHECK(copy(wide, {0}, a, {1}) == HKV_EINVAL && copy(wide, {1}, a, {1}) == HKV_OK && copy(wide, {1}, a, {3}) == HKV_EINVAL);
        for (hkv_pool *p : {eight, four, wide}) CHECK(kv_pool_destroy(p) == HKV_OK);
    }
    {  // scales alone
        hkv_pool *b = make_pool(16, 16, HKV_FP8_E4M3, k + 0x20000000, v + 0x20000000), *c = make_pool(16, 16, HKV_FP8_E4M3, k + 0x30000000, v + 0x30000000);
        CHECK(copy(b, {3}, c, {3}) == HKV_EINVAL && copy(b, {3}, c, {4}) == HKV_OK);
        CHECK(kv_pool_destroy(b) == HKV_OK && kv_pool_destroy(c) == HKV_OK);
    }
    {  // another handle over the same pool, and buffers that only touch
        hkv_pool *b = make_pool(8, 16, HKV_BF16, k, v), *c = make_pool(8, 16, HKV_BF16, k + 8 * kPageBytes, v + 8 * kPageBytes);
        CHECK(copy(a, {3}, b, {3}) == HKV_EINVAL && copy(a, {3}, b, {4}) == HKV_OK);
        for (int i = 0; i < 8; ++i) CHECK(copy(a, {i}, c, {7 - i}) == HKV_OK && copy(c, {i}, a, {i}) == HKV_OK);
        CHECK(kv_pool_destroy(b) == HKV_OK && kv_pool_destroy(c) == HKV_OK);
    }
    CHECK(kv_pool_destroy(a) == HKV_OK);
}

// A call whose launch fails behind its list's upload: the list's place is not written anew while the upload may still read it.
static void lists_that_fail_on_their_way() {
    hkv_pool *pool = make_pool(3000), *wide = make_pool(3000, 16, HKV_FP32, reinterpret_cast<void *>(0x200000000), reinterpret_cast<void *>(0x300000000));
    std::vector<int32_t> to(1400), from(1400), slots(1400, 3), kept(1);
    std::iota(to.begin(), to.end(), 0);
    std::iota(from.begin(), from.end(), 1400);
    void *const x = reinterpret_cast<void *>(0x400000000);
    const int32_t n_tokens = 1400 * 16;
    const auto copy = [&] { return kv_pool_copy_pages(pool, to.data(), pool, from.data(), 1400, nullptr, nullptr); };
    const auto write = [&] { return kv_pool_write(pool, to.data(), 0, n_tokens, x, x, nullptr); };
    const auto write_wide = [&] { return kv_pool_write(wide, to.data(), 0, 64, x, x, nullptr); };
    const auto append = [&] { return kv_pool_append(pool, to.data(), slots.data(), 1400, x, x, nullptr); };
    const auto evict = [&] { return kv_pool_evict(pool, 1, from.data(), &n_tokens, to.data(), &n_tokens, 4, 4, static_cast<float *>(x), static_cast<int32_t *>(x), nullptr); };
    const auto each = [&](auto &&f) { f(copy); f(write); f(append); f(evict); f(write_wide); };
    each([&](auto call) {
        CHECK(call() == HKV_OK);
        for (int fails = 0; fails < 2; ++fails) {
            launches_until_failure = fails;
            CHECK(call() == HKV_EHIP);
            launches_until_failure = -1;
            for (int i = 0; i < 2 * hkv_pool::kWriteSlots; ++i) CHECK(call() == HKV_OK);
        }
        CHECK(overtaken == 0);
        overtaken = 0;
        on_their_way.clear();
    });
    CHECK(kv_pool_destroy(pool) == HKV_OK && kv_pool_destroy(wide) == HKV_OK);
}

int main(int argc, char **argv) {
    const std::pair<const char *, void (*)()> programs[] = {{"caches_after_their_pool", caches_after_their_pool}, {"evictions_beside_forks", evictions_beside_forks},
                                                           {"forks_that_end_cached_sequences", forks_that_end_cached_sequences},
                                                           {"copies_between_pools_that_overlap", copies_between_pools_that_overlap},
                                                           {"lists_that_fail_on_their_way", lists_that_fail_on_their_way}};
    int ran = 0;
    for (const auto &p : programs)
        if (argc < 2 || !std::strcmp(argv[1], p.first)) {
            p.second();
            ++ran;
        }
    std::printf("%d programs, %d failed checks\n", ran, failures);
    return failures != 0;
}
