// Decode plans over 4-bit pools: how the forest is cut into work items (four_bit_decode.hip runs them).
#pragma once

#include <algorithm>
#include <array>
#include <functional>
#include <queue>
#include <utility>

#include "hkv_objects.h"

namespace four_plan {

// Kinds of items by query rows (up to 16, 32, 64, 128 with a workgroup each; up to 16 with a wavefront each), microseconds: what an item costs beside its
// steps of 64 tokens, a step on a full chip (two workgroups a compute unit) and on an empty one.
struct Kind {
    double fixed, full, alone;
};
constexpr Kind kKinds[5] = {{3.1, 0.47, 0.21}, {5.2, 0.61, 0.34}, {3.3, 0.85, 0.79}, {4.3, 1.04, 1.31}, {3.1, 1.78, 0.76}};
constexpr int kRowCaps[4] = {16, 32, 64, 128};
constexpr int kXcds = 8;  // (workgroups go to them in turn)
constexpr int kChunks[7] = {64, 128, 256, 512, 1024, 2048, 4096};

struct Load {  // items of one kind
    int64_t items = 0, steps = 0;
    int32_t longest = 0;
    void add(int64_t n, int32_t tokens, int64_t all_tokens) {
        items += n;
        steps += all_tokens;
        longest = std::max(longest, (tokens + 63) / 64);
    }
};

// A step's length: the items' costs over the chip's slots and part of the longest one, that one alone, or the bytes (512 sequences of 1024 to 2048 tokens:
// 143 us with a wavefront each, 160 with a workgroup each); then the merge of the partials, of
// which a row has `parts`.  Fitted to timings; of 700 random plans of 7 to 400 us (profiles/four_bit_plan_timings.csv) the cut that it prefers takes 1.02 of the time of
// the best among that one and 14 random cuts in the mean, 1.08 for one plan in ten, 1.34 at most.
inline double estimate_us(const Load (&load)[5], double bytes, int32_t parts, double partials, int n_cu) {
    double busy = 0, longest = 0;
    for (int k = 0; k < 5; ++k) {
        if (load[k].items == 0) continue;
        busy += (load[k].items * kKinds[k].fixed + load[k].steps * kKinds[k].full) * (k == 4 ? 0.25 : 1.0);
        longest = std::max(longest, kKinds[k].fixed + load[k].longest * kKinds[k].alone);
    }
    busy /= 2 * n_cu;
    return 4.7 + std::max({busy + 0.52 * longest, longest, bytes / (load[0].items ? 5.3e6 : 6.2e6)}) + 0.028 * parts + partials * 528 / 3.2e6;
}

struct Cut {
    int max_rows, shared_chunk, leaf_chunk;
    bool pack;
    double us;
};
struct Pieces {
    int count, blocks;  // chunks of a node, blocks of one (the last one shorter)
};
inline Pieces pieces_of(int blocks, int chunk) {  // evenly, in whole steps of four blocks where the chunk has room for them
    const int most = std::max(1, chunk / HKV_PAGE_SIZE), cuts = (blocks + most - 1) / most;
    const int each = std::min({blocks, most, ((blocks + cuts - 1) / cuts + 3) / 4 * 4});
    return {(blocks + each - 1) / each, each};
}

// The cut of the shortest estimated step among those whose partials fit the static workspace, or among all.  What the caller sets stays.
inline Cut choose(const hkv_decode_plan &pl, int n_cu) {
    const int G = pl.group, Hkv = pl.pool->d.num_kv_heads, n_nodes = (int)pl.nodes.size();
    Load few[7], shared[4][7][5];
    std::vector<int32_t> few_parts(n_nodes), shared_parts(n_nodes);
    int32_t most_few[7] = {}, most_shared[7] = {};  // chunks on the longest path
    double bytes = 0;
    for (int i = 0; i < 7; ++i)
        for (int v = 0; v < n_nodes; ++v) {
            const hkv_node &nd = pl.nodes[v];
            const int R = pl.node_req_indptr[v + 1] - pl.node_req_indptr[v];
            few_parts[v] = nd.parent >= 0 ? few_parts[nd.parent] : 0;
            shared_parts[v] = nd.parent >= 0 ? shared_parts[nd.parent] : 0;
            if (R == 0 || nd.n_tokens == 0) continue;
            if (i == 0) bytes += 136.0 * Hkv * nd.n_tokens;
            const bool is_few = R * G <= 16;
            const int set = is_few ? pl.opt.leaf_chunk : pl.opt.shared_chunk;
            const Pieces p = pieces_of(nd.n_pages, set ? set : kChunks[i]);
            const int tokens = std::min(nd.n_tokens, p.blocks * HKV_PAGE_SIZE);
            const int64_t steps = (int64_t)(nd.n_pages + 3) / 4 * Hkv;
            (is_few ? few_parts : shared_parts)[v] += p.count;
            most_few[i] = std::max(most_few[i], few_parts[v]);
            most_shared[i] = std::max(most_shared[i], shared_parts[v]);
            if (is_few) {
                few[i].add((int64_t)p.count * Hkv, tokens, steps);
                continue;
            }
            for (int c = 0; c < 4; ++c) {
                const int max_req = std::max(1, (pl.opt.max_rows ? pl.opt.max_rows : kRowCaps[c]) / G), groups = (R + max_req - 1) / max_req;
                const int rows = (R + groups - 1) / groups * G;
                shared[c][i][rows <= 16 ? 0 : rows <= 32 ? 1 : rows <= 64 ? 2 : 3].add((int64_t)p.count * groups * Hkv, tokens, steps * groups);
            }
        }
    Cut best{128, 2048, 4096, false, 0};
    double least = 1e300;
    bool best_fits = false;
    for (int c = 0; c < 4; ++c)
        for (int s = 0; s < 7; ++s)
            for (int f = 0; f < 7; ++f)
                for (const bool pack : {false, true}) {
                    if (pl.opt.pack == 1 ? pack : pl.opt.pack == 3 ? !pack : false) continue;
                    Load load[5];
                    for (int k = 0; k < 4; ++k) load[k] = shared[c][s][k];
                    load[0].items += few[f].items;
                    load[0].steps += few[f].steps;
                    load[0].longest = std::max(load[0].longest, few[f].longest);
                    if (pack) std::swap(load[0], load[4]);
                    const int32_t parts = most_few[f] + most_shared[s];
                    const double partials = (double)pl.n_req * pl.num_q_heads * parts;
                    const bool fits = partials * 264 + 768 <= (double)kStaticWorkspaceBytes;
                    const double us = estimate_us(load, bytes, parts, partials, n_cu);
                    if (fits == best_fits ? us >= least : !fits) continue;
                    least = us;
                    best_fits = fits;
                    best = Cut{pl.opt.max_rows ? pl.opt.max_rows : kRowCaps[c], kChunks[s], kChunks[f], pack, us};
                }
    if (pl.opt.shared_chunk) best.shared_chunk = pl.opt.shared_chunk;
    if (pl.opt.leaf_chunk) best.leaf_chunk = pl.opt.leaf_chunk;
    return best;
}

// Estimated microseconds of items in sets (of `set` items, the first ones of the longest), a wavefront or a workgroup each.
template <class Proto>
std::vector<double> lengths(const std::vector<Proto> &items, size_t set, int group, bool packed) {
    std::vector<double> us;
    for (size_t i = 0; i < items.size(); i += set) {
        const int rows = items[i].it.n_req * group;
        const Kind &k = kKinds[packed ? 4 : rows <= 16 ? 0 : rows <= 32 ? 1 : rows <= 64 ? 2 : 3];
        us.push_back(k.fixed + (items[i].it.n_tokens + 63) / 64 * k.full);
    }
    return us;
}

// The order in which sets of two kinds go out to `slots` places: set i of the first kind as i, of the second as ~i.  Whenever a place is free, the kind
// goes on whose remaining time over the places it would have, plus five times a set's, is longer: both share the chip all the while (one is bound by
// its instructions, the other by memory), and neither is left alone with long sets at the end (512 requests over
// 16 prompts of 8192 tokens: 260 us; with one set's time 267, with twenty 262).  Of those that start at once the first kind's come
// first: workgroups go to an XCD's compute units in turn, so each gets one of them before any gets two.
inline std::vector<int32_t> dispatch_order(const std::array<std::vector<double>, 2> &us, int slots) {
    std::vector<int32_t> order;
    std::priority_queue<std::pair<double, int>, std::vector<std::pair<double, int>>, std::greater<>> running;  // (end, kind)
    double left[2] = {}, now = 0;
    for (int k = 0; k < 2; ++k)
        for (const double x : us[k]) left[k] += x;
    size_t next[2] = {}, count[2] = {};
    auto urgency = [&](int k) { return next[k] < us[k].size() ? left[k] / (double)(count[k] + 1) + 5 * us[k][next[k]] : -1.0; };
    while (next[0] < us[0].size() || next[1] < us[1].size()) {
        if ((int)running.size() >= slots) {
            now = running.top().first;
            --count[running.top().second];
            running.pop();
        }
        const int k = urgency(0) >= urgency(1) ? 0 : 1;
        order.push_back(k ? ~(int32_t)next[1] : (int32_t)next[0]);
        running.push({now + us[k][next[k]], k});
        left[k] -= us[k][next[k]++];
        ++count[k];
    }
    std::stable_partition(order.begin(), order.begin() + std::min<size_t>(order.size(), (size_t)slots), [](int32_t i) { return i >= 0; });
    return order;
}

}  // namespace four_plan

// A node with T tokens that R requests pass through becomes items of up to max_rows query rows and a chunk of whole blocks each, every one of which leaves
// a partial per row; the chunks of a node take the same places in the partial lists of all requests below it (as in the other pools' plans).
static void plan_four_bit(hkv_decode_plan &pl, int n_cu) {
    const int G = pl.group, Hkv = pl.pool->d.num_kv_heads, n_nodes = (int)pl.nodes.size();
    const four_plan::Cut cut = four_plan::choose(pl, n_cu);
    pl.items_us = cut.us;
    if (pl.paths_us == 0 || pl.paths_us > 0.93 * pl.items_us) pl.n_paths = pl.path_waves = 0;  // else paths instead (estimate_paths); the items are described as ever
    const int max_req = std::max(1, cut.max_rows / G);
    struct Proto {
        DecodeItem it;
        int64_t cost;
    };
    std::vector<Proto> protos;
    std::vector<int32_t> node_chunks(n_nodes, 0), slot_base(n_nodes, 0);
    for (int v = 0; v < n_nodes; ++v) {
        const hkv_node &nd = pl.nodes[v];
        if (nd.parent >= 0) slot_base[v] = slot_base[nd.parent] + node_chunks[nd.parent];
        const int R = pl.node_req_indptr[v + 1] - pl.node_req_indptr[v];
        if (nd.n_tokens == 0 || R == 0) continue;
        const four_plan::Pieces p = four_plan::pieces_of(nd.n_pages, R * G > 16 ? cut.shared_chunk : cut.leaf_chunk);
        node_chunks[v] = p.count;
        const int groups = (R + max_req - 1) / max_req, per_group = (R + groups - 1) / groups;
        for (int r0 = 0; r0 < R; r0 += per_group)
            for (int pg = 0, ci = 0; pg < nd.n_pages; pg += p.blocks, ++ci) {
                const int nr = std::min(per_group, R - r0), nt = std::min(p.blocks * HKV_PAGE_SIZE, nd.n_tokens - pg * HKV_PAGE_SIZE);
                for (int h = 0; h < Hkv; ++h)
                    protos.push_back({DecodeItem{nd.page_begin + pg, nt, h, pl.node_req_indptr[v] + r0, nr, slot_base[v] + ci, pg * HKV_PAGE_SIZE, v},
                                      (int64_t)nt * std::max(16, (nr * G + 15) / 16 * 16)});
            }
    }
    // Heavy items first, those with a wavefront each behind the others.
    auto packed = [&](const Proto &x) { return cut.pack && x.it.n_req * G <= 16; };
    std::stable_sort(protos.begin(), protos.end(), [&](const Proto &a, const Proto &b) { return packed(a) != packed(b) ? packed(b) : a.cost > b.cost; });
    pl.order.clear();
    if (pl.opt.interleave >= 0) {  // items of many and of few rows side by side, in whole sets of KV heads, which stay on their XCDs
        std::vector<Proto> many, few;
        for (const Proto &x : protos) (x.it.n_req * G > 16 ? many : few).push_back(x);
        const int set = cut.pack ? four_plan::kXcds : (four_plan::kXcds + Hkv - 1) / Hkv * Hkv, slots = std::max(1, 2 * n_cu / set);
        const auto order = four_plan::dispatch_order({four_plan::lengths(many, set, G, false), four_plan::lengths(few, cut.pack ? 4 * set : set, G, cut.pack)}, slots);
        if (cut.pack) {
            if (!many.empty() && (int)order.size() > slots) pl.order = order;  // (what starts all at once is in order)
        } else {
            protos.clear();
            for (const int32_t i : order) {
                const std::vector<Proto> &from = i < 0 ? few : many;
                const size_t first = (size_t)(i < 0 ? ~i : i) * set;
                protos.insert(protos.end(), from.begin() + first, from.begin() + std::min(first + set, from.size()));
            }
        }
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
}
