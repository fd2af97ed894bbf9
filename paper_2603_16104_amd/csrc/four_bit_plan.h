// Decode plans over 4-bit pools: how the forest is cut into work items (four_bit_decode.hip runs them).
#pragma once

#include <algorithm>

#include "hkv_objects.h"

// A node with T tokens that R requests pass through becomes items of up to max_rows query rows and a chunk of whole blocks each, every one of which leaves
// a partial per row; the chunks of a node take the same places in the partial lists of all requests below it (as in the other pools' plans).
static void plan_four_bit(hkv_decode_plan &pl, int n_cu) {
    const int G = pl.group, Hkv = pl.pool->d.num_kv_heads, n_nodes = (int)pl.nodes.size();
    const int max_rows = pl.opt.max_rows ? pl.opt.max_rows : 128, max_req = std::max(1, max_rows / G);
    auto requests = [&](int v) { return pl.node_req_indptr[v + 1] - pl.node_req_indptr[v]; };
    int64_t work = 0;  // blocks times row groups and heads
    for (int v = 0; v < n_nodes; ++v)
        if (requests(v) > 0) work += (int64_t)pl.nodes[v].n_pages * Hkv * ((requests(v) + max_req - 1) / max_req);
    const int chunk = (int)std::min<int64_t>(1 << 26, std::max<int64_t>(256, work * HKV_PAGE_SIZE / (4 * n_cu) / 64 * 64));
    struct Proto {
        DecodeItem it;
        int64_t cost;
    };
    std::vector<Proto> protos;
    std::vector<int32_t> node_chunks(n_nodes, 0), slot_base(n_nodes, 0);
    for (int v = 0; v < n_nodes; ++v) {
        const hkv_node &nd = pl.nodes[v];
        if (nd.parent >= 0) slot_base[v] = slot_base[nd.parent] + node_chunks[nd.parent];
        const int R = requests(v);
        if (nd.n_tokens == 0 || R == 0) continue;
        const int asked = R * G > 16 ? (pl.opt.tile_chunk ? pl.opt.tile_chunk : pl.opt.shared_chunk) : pl.opt.leaf_chunk;
        const int most = asked ? asked : chunk, cuts = (nd.n_tokens + most - 1) / most;
        const int per_chunk = std::min(nd.n_pages, ((nd.n_pages + cuts - 1) / cuts + 3) / 4 * 4);  // whole steps of four blocks
        node_chunks[v] = (nd.n_pages + per_chunk - 1) / per_chunk;
        const int groups = (R + max_req - 1) / max_req, per_group = (R + groups - 1) / groups;
        for (int r0 = 0; r0 < R; r0 += per_group)
            for (int pg = 0, ci = 0; pg < nd.n_pages; pg += per_chunk, ++ci) {
                const int nr = std::min(per_group, R - r0), nt = std::min(per_chunk * HKV_PAGE_SIZE, nd.n_tokens - pg * HKV_PAGE_SIZE);
                for (int h = 0; h < Hkv; ++h)
                    protos.push_back({DecodeItem{nd.page_begin + pg, nt, h, pl.node_req_indptr[v] + r0, nr, slot_base[v] + ci, pg * HKV_PAGE_SIZE, v},
                                      (int64_t)nt * std::max(16, (nr * G + 15) / 16 * 16)});
            }
    }
    // Heavy items first.  Many items of few rows: a wavefront each instead of a workgroup each.
    int64_t few = 0;
    for (const Proto &x : protos) few += x.it.n_req * G <= 16;
    const bool pack = pl.opt.pack == 3 || (pl.opt.pack != 1 && few > 8 * n_cu);
    auto packed = [&](const Proto &x) { return pack && x.it.n_req * G <= 16; };
    std::stable_sort(protos.begin(), protos.end(), [&](const Proto &a, const Proto &b) { return packed(a) != packed(b) ? packed(b) : a.cost > b.cost; });
    if (pl.opt.interleave >= 0) {  // items of many and of few rows with a workgroup each, side by side in whole sets of KV heads, which stay on their XCDs
        std::vector<Proto> many, others, rest;
        for (const Proto &x : protos) (packed(x) ? rest : x.it.n_req * G > 16 ? many : others).push_back(x);
        protos.clear();
        const size_t set = (8 + Hkv - 1) / Hkv * Hkv;
        for (size_t a = 0, b = 0; a < many.size() || b < others.size();) {
            const bool first = b >= others.size() || (a < many.size() && (a + set) * others.size() <= (b + set) * many.size());
            for (size_t i = 0; i < set; ++i)
                if (first && a < many.size())
                    protos.push_back(many[a++]);
                else if (!first && b < others.size())
                    protos.push_back(others[b++]);
        }
        protos.insert(protos.end(), rest.begin(), rest.end());
    }
    pl.items.clear();
    pl.n_single = 0;
    for (const Proto &x : protos) {
        pl.items.push_back(x.it);
        pl.n_single += !packed(x);
    }
    pl.concurrent = false;
    pl.part_count.assign(pl.n_req, 0);
    pl.max_parts = 1;
    for (int r = 0; r < pl.n_req; ++r) {
        const int leaf = pl.req_leaf[r];
        pl.part_count[r] = slot_base[leaf] + node_chunks[leaf];
        pl.max_parts = std::max(pl.max_parts, pl.part_count[r]);
    }
    pl.n_parts = pl.n_req * pl.num_q_heads * pl.max_parts;
}
