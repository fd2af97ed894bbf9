// What the calls around a step's attention refuse in the middle of a plan's life, after other calls on it: the stubs of
// operators_check.cpp (no GPU, no HIP library), programs of its own.  Exit status 0 = clean.
#define main operators_check_main
#include "operators_check.cpp"
#undef main

static hkv_decode_plan *growing_plan(hkv_pool *pool, const std::vector<hkv_node> &nodes, const std::vector<int32_t> &pages, int reserve) {
    std::vector<int32_t> leaf(nodes.size());
    for (size_t i = 0; i < leaf.size(); ++i) leaf[i] = (int32_t)i;
    hkv_decode_plan *plan = nullptr;
    CHECK(hkv_decode_plan_create_growing(pool, nodes.data(), (int32_t)nodes.size(), pages.data(), (int32_t)pages.size(), leaf.data(), (int32_t)leaf.size(), 4, reserve,
                                         0, &plan) == HKV_OK);
    return plan;
}

// Two requests' new tokens in one block, by ways on which an earlier call has looked at the blocks already.
static void appends_to_one_block() {
    const hkv_qkv x = make_rows();
    for (int dtype : {HKV_BF16, HKV_FP8_E4M3}) {
        hkv_pool *pool = make_pool(16, 16, 2, dtype);
        // a store that is refused, then the append
        hkv_decode_plan *plan = growing_plan(pool, {{-1, 0, 1, 5}, {-1, 0, 1, 5}}, {1}, 40);
        for (int i = 0; i < 2; ++i) {
            CHECK(hkv_decode_plan_store(plan, &x, nullptr) == HKV_EINVAL && stored.empty());
            CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_EINVAL && stored.empty());
        }
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
        // appends that store, then one that only lengthens and opens one page for both, then another that stores
        plan = growing_plan(pool, {{-1, 0, 1, 15}, {-1, 1, 1, 15}}, {0, 5}, 40);
        const int32_t twice[2] = {7, 7};
        CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_OK);
        CHECK(same(taken(), {Put{0, 15, 0, 15}, Put{5, 15, 1, 15}}));
        CHECK(hkv_decode_plan_append(plan, twice, nullptr) == HKV_OK);
        CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_EINVAL && stored.empty());
        CHECK(hkv_decode_plan_store(plan, &x, nullptr) == HKV_EINVAL && stored.empty());
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
        CHECK(kv_pool_destroy(pool) == HKV_OK);
        // leaves in one page of several blocks: a leaf reaches the block of the other
        pool = make_pool(16, 64, 2, dtype);
        plan = growing_plan(pool, {{-1, 0, 1, 15}, {-1, 0, 1, 20}}, {2}, 40);
        CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_OK);
        CHECK(same(taken(), {Put{8, 15, 0, 15}, Put{9, 4, 1, 20}}));
        CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_EINVAL && stored.empty());
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
        // what is refused changes nothing: with pages of their own it goes on where it was
        plan = growing_plan(pool, {{-1, 0, 1, 64}, {-1, 1, 1, 64}}, {2, 3}, 40);
        const int32_t own[2] = {4, 5};
        for (int i = 0; i < 3; ++i) CHECK(hkv_decode_plan_append_qkv(plan, twice, &x, nullptr) == HKV_EINVAL && stored.empty());
        CHECK(hkv_decode_plan_append_qkv(plan, own, &x, nullptr) == HKV_OK);
        CHECK(same(taken(), {Put{16, 0, 0, 64}, Put{20, 0, 1, 64}}));
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
        CHECK(kv_pool_destroy(pool) == HKV_OK);
    }
}

// A prompt's new tokens behind earlier ones in a page that somebody else holds, too; pages that the call begins may have any number of holders.
static void prompts_into_shared_pages() {
    const hkv_qkv x = make_rows();
    for (int page : {16, 64})
        for (int dtype : {HKV_BF16, HKV_FP8_E4M3, HKV_FP32}) {
            hkv_pool *pool = make_pool(8, page, 2, dtype);
            int32_t ids[4];
            CHECK(kv_pool_alloc(pool, 4, ids) == HKV_OK);
            // request 0 goes on inside page ids[1], request 1 begins with it whole pages of its own
            const int inside = page == 16 ? page + 7 : page + 32;  // (of larger pages: where a block of it begins)
            const int32_t cu[3] = {0, 5, 5 + page + 3}, table[4] = {ids[0], ids[1], ids[2], ids[3]}, kv[2] = {inside + 5, page + 3};
            hkv_prefill_plan *plan = nullptr;
            CHECK(hkv_prefill_plan_create(pool, cu, table, 2, kv, 2, 4, 0, &plan) == HKV_OK);
            CHECK(hkv_prefill_plan_store(plan, &x, nullptr) == HKV_OK);
            const std::vector<Put> all = taken();
            CHECK(all.size() == (size_t)cu[2]);
            CHECK(kv_pool_retain(pool, 1, ids + 1) == HKV_OK);
            for (int again = 0; again < 2; ++again) CHECK(hkv_prefill_plan_store(plan, &x, nullptr) == HKV_EINVAL && stored.empty());
            CHECK(kv_pool_release(pool, 1, ids + 1) == HKV_OK);
            CHECK(hkv_prefill_plan_store(plan, &x, nullptr) == HKV_OK);
            CHECK(same(taken(), all));
            for (int i : {0, 2, 3}) CHECK(kv_pool_retain(pool, 1, ids + i) == HKV_OK);  // a prefix that is only read, a prompt stored once for two
            CHECK(hkv_prefill_plan_store(plan, &x, nullptr) == HKV_OK);
            CHECK(same(taken(), all));
            CHECK(hkv_prefill_plan_destroy(plan) == HKV_OK);
            CHECK(kv_pool_destroy(pool) == HKV_OK);
        }
}

// An append cannot be captured (its places travel by value, the lengths that a replay would change again are the host's): nothing changes.
static void appends_under_capture() {
    const hkv_qkv x = make_rows();
    for (int requests : {2, 300}) {  // (the update in arguments, and through the plan's buffers)
        hkv_pool *pool = make_pool(2 * requests, 16, 2, HKV_BF16);
        std::vector<hkv_node> nodes;
        std::vector<int32_t> pages, fresh;
        for (int r = 0; r < requests; ++r) {
            nodes.push_back(hkv_node{-1, r, 1, 16 - r % 2});
            pages.push_back(r);
            fresh.push_back(requests + r);
        }
        hkv_decode_plan *plan = growing_plan(pool, nodes, pages, 3);
        for (auto status : {hipStreamCaptureStatusActive, hipStreamCaptureStatusInvalidated}) {
            capturing = status;
            CHECK(hkv_decode_plan_append_qkv(plan, fresh.data(), &x, nullptr) == HKV_EINVAL && stored.empty());
            CHECK(hkv_decode_plan_append_qkv(plan, nullptr, &x, nullptr) == HKV_EINVAL && stored.empty());
        }
        CHECK(hkv_decode_plan_store(plan, &x, nullptr) == HKV_OK);  // (which may be captured)
        for (const Put &p : taken()) CHECK(p.block < requests && p.slot == 15 - p.row % 2);
        capturing = hipStreamCaptureStatusNone;
        for (int i = 0; i < 3; ++i) CHECK(hkv_decode_plan_append_qkv(plan, fresh.data(), &x, nullptr) == HKV_OK);
        stored.clear();
        CHECK(hkv_decode_plan_append_qkv(plan, fresh.data(), &x, nullptr) == HKV_ENOMEM);
        CHECK(hkv_decode_plan_destroy(plan) == HKV_OK);
        CHECK(kv_pool_destroy(pool) == HKV_OK);
    }
}

int main(int argc, char **argv) {
    const struct {
        const char *name;
        void (*run)();
    } programs[] = {{"appends_to_one_block", appends_to_one_block}, {"prompts_into_shared_pages", prompts_into_shared_pages},
                    {"appends_under_capture", appends_under_capture}};
    int ran = 0;
    for (const auto &p : programs)
        if (argc < 2 || !std::strcmp(argv[1], p.name)) {
            p.run();
            ++ran;
        }
    std::printf("operators_refusals: %d programs, %d failed checks\n", ran, failures);
    return failures || !ran ? 1 : 0;
}
