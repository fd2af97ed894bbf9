// The order in which a 4-bit plan's workgroups go out: every set of items once, as many as the launch has.  The stubs of page_lives.cpp (no GPU, no HIP library).
#define main page_lives_main
#include "page_lives.cpp"
#undef main

int main() {
    int ordered = 0, plain = 0;
    for (const int heads : {1, 2, 3, 8}) {
        for (int seed = 0; seed < 12; ++seed) {
            const int roots = 1 + seed % 8, each = 4 + 13 * (seed % 4), group = 8;
            std::vector<hkv_node> nodes;
            std::vector<int32_t> leaves;
            int at = 0;
            auto add = [&](int parent, int tokens) {
                nodes.push_back({parent, at, (tokens + 15) / 16, tokens});
                at += (tokens + 15) / 16;
            };
            for (int r = 0; r < roots; ++r) add(-1, 200 + 333 * ((seed + r) % 5));
            for (int r = 0; r < roots * each; ++r) {
                leaves.push_back((int32_t)nodes.size());
                add(r % roots, 1 + 37 * ((seed + r) % 7));
            }
            hkv_pool_desc d{};
            d.num_pages = at;
            d.page_size = 16;
            d.num_kv_heads = heads;
            d.head_dim = 128;
            d.dtype = HKV_FP4_E2M1;
            d.k_pages = d.v_pages = reinterpret_cast<void *>(0x100000);
            d.k_scale = d.v_scale = reinterpret_cast<float *>(0x200000);
            hkv_pool *pool = nullptr;
            CHECK(kv_pool_create(&d, &pool) == HKV_OK);
            std::vector<int32_t> pages(at);
            std::iota(pages.begin(), pages.end(), 0);
            hkv_decode_plan_params o{};
            o.tokens_per_req = 1;
            o.pack = 3;
            o.leaf_chunk = 64;
            o.shared_chunk = 64 << seed % 3;
            o.max_rows = 16 << seed % 4;
            hkv_decode_plan *plan = nullptr;
            CHECK(hkv_decode_plan_create_ex(pool, nodes.data(), (int32_t)nodes.size(), pages.data(), at, leaves.data(), (int32_t)leaves.size(), heads * group, HKV_PLAN_HOST_ONLY, &o,
                                            &plan) == HKV_OK);
            const int packs = ((int)plan->items.size() - plan->n_single + 3) / 4, sets[2] = {(plan->n_single + 7) / 8, (packs + 7) / 8};  // as the launch counts them
            for (size_t i = 0; i < plan->items.size(); ++i) CHECK(((int)i < plan->n_single) == (plan->items[i].n_req * group > 16));
            (plan->order.empty() ? plain : ordered) += 1;
            if (!plan->order.empty()) {
                CHECK((int)plan->order.size() == sets[0] + sets[1]);
                std::vector<int32_t> sorted(plan->order), want;
                std::sort(sorted.begin(), sorted.end());
                for (int i = sets[1]; i > 0; --i) want.push_back(-i);
                for (int i = 0; i < sets[0]; ++i) want.push_back(i);
                CHECK(sorted == want);
            }
            CHECK(hkv_decode_plan_destroy(plan) == HKV_OK && kv_pool_destroy(pool) == HKV_OK);
        }
    }
    CHECK(ordered > 10 && plain > 3);
    std::printf("%d ordered, %d plain, %d failed checks\n", ordered, plain, failures);
    return failures != 0;
}
