// Host side of the calls that move pages: copies between pools (kv_pool_copy_pages), forks of sequences (kv_pool_fork) and compaction (kv_pool_compact).
// Checks, reference counts and lists of blocks; the bytes are moved by page_copy.hip.
#include "hkv_objects.h"

#include <algorithm>
#include <climits>
#include <cstring>
#include <exception>
#include <numeric>
#include <utility>

namespace {

struct PagePair {
    int32_t src, dst, tokens;  // tokens: of the page
};

// A pool's buffers and what a page has of each.
struct Buffer {
    uintptr_t base;
    size_t page, bytes;
    std::pair<uintptr_t, uintptr_t> of(int32_t id) const { return {base + page * (size_t)id, base + page * (size_t)(id + 1)}; }
};
std::vector<Buffer> buffers_of(const hkv_pool *pool) {
    const size_t heads = (size_t)pool->blocks_per_page * pool->d.num_kv_heads;
    const int dtype = pool->d.dtype;
    const size_t codes = heads * (HKV_PAGE_SIZE * HKV_HEAD_DIM / 8) * (dtype == HKV_BF16 ? 16 : dtype == HKV_FP8_E4M3 ? 8 : dtype == HKV_FP32 ? 32 : 4);
    const size_t scales = dtype == HKV_FP8_E4M3 ? heads * sizeof(float) : dtype == HKV_FP4_E2M1 ? heads * (HKV_PAGE_SIZE * HKV_HEAD_DIM / 32) : 0;
    std::vector<Buffer> out;
    auto add = [&](const void *p, size_t page) { out.push_back({reinterpret_cast<uintptr_t>(p), page, page * (size_t)pool->d.num_pages}); };
    add(pool->d.k_pages, codes);
    add(pool->d.v_pages, codes);
    if (scales > 0) {
        add(pool->d.k_scale, scales);
        add(pool->d.v_scale, scales);
    }
    return out;
}
// Of pages that go from one pool to another one whose bytes are partly the same: the first that is read where another (or it itself) is written, or -1.
int32_t read_and_written(const hkv_pool *dst, const hkv_pool *src, const std::vector<PagePair> &pages) {
    const std::vector<Buffer> to = buffers_of(dst), from = buffers_of(src);
    std::vector<std::pair<uintptr_t, uintptr_t>> written;
    for (const Buffer &w : to)
        if (std::any_of(from.begin(), from.end(), [&](const Buffer &r) { return w.base < r.base + r.bytes && r.base < w.base + w.bytes; }))
            for (const PagePair &p : pages) written.push_back(w.of(p.dst));
    if (written.empty()) return -1;  // (as good as always)
    std::sort(written.begin(), written.end());
    std::vector<uintptr_t> ends;  // the furthest end so far (the target's own buffers may overlap, too)
    for (const auto &w : written) ends.push_back(std::max(w.second, ends.empty() ? 0 : ends.back()));
    for (const PagePair &p : pages)
        for (const Buffer &r : from) {
            const auto read = r.of(p.src);
            const size_t before = (size_t)(std::lower_bound(written.begin(), written.end(), std::make_pair(read.second, (uintptr_t)0)) - written.begin());
            if (before > 0 && ends[before - 1] > read.first) return p.src;
        }
    return -1;
}

// Queues the copies of pages (blocks behind a page's last token are left): lists that fit travel in the kernel's arguments, others through the
// target pool's staging ring.
int queue_copies(hkv_pool *dst, const hkv_pool *src, const std::vector<PagePair> &pages, hipStream_t s) {
    const int S = dst->blocks_per_page;
    int64_t blocks = 0;
    for (const PagePair &p : pages) blocks += (p.tokens + HKV_PAGE_SIZE - 1) / HKV_PAGE_SIZE;
    PageCopyInline a{};
    a.src = view_of(src);
    a.dst = view_of(dst);
    const bool in_arguments = blocks <= kMaxInlineCopies;
    constexpr int kMost = hkv_pool::kMaxWritePages / 3;
    size_t page = 0;
    int block = 0;  // of the page
    while (page < pages.size()) {
        Staging staged(dst, s);
        if (!in_arguments)
            if (int rc = staged.take()) return rc;
        int32_t *const list = in_arguments ? a.entries : staged.host;
        int n = 0;
        while (page < pages.size() && n < (in_arguments ? kMaxInlineCopies : kMost)) {
            const PagePair &p = pages[page];
            if (block * HKV_PAGE_SIZE >= p.tokens) {
                ++page;
                block = 0;
                continue;
            }
            list[3 * n] = p.src * S + block;
            list[3 * n + 1] = p.dst * S + block;
            list[3 * n + 2] = std::min(HKV_PAGE_SIZE, p.tokens - block * HKV_PAGE_SIZE);
            ++n;
            ++block;
        }
        a.n = n;
        a.list = staged.device;
        if (in_arguments) {
            HKV_HIP(launch_page_copy(a, s));
        } else {
            if (n > 0) {
                HKV_HIP(launch_upload(staged.host_on_device, staged.device, align_up(sizeof(int32_t) * 3 * (size_t)n, 16), s));
                HKV_HIP(launch_page_copy(static_cast<const PageCopyLaunch &>(a), s));
            }
            if (int rc = staged.leave()) return rc;
        }
    }
    return HKV_OK;
}

}  // namespace

extern "C" int kv_pool_copy_pages(hkv_pool *dst, const int32_t *dst_ids, hkv_pool *src, const int32_t *src_ids, int32_t n, const int32_t *n_tokens,
                                  void *stream) try {
    const char *who = "kv_pool_copy_pages";
    if (!dst || !src) return fail(HKV_EINVAL, "%s: null pool", who);
    if (n < 0 || (n > 0 && (!dst_ids || !src_ids))) return fail(HKV_EINVAL, "%s: n %d, or a null list", who, n);
    if (dst->d.page_size != src->d.page_size || dst->d.num_kv_heads != src->d.num_kv_heads)
        return fail(HKV_ESHAPE, "%s: pages of %d tokens and %d KV heads into pages of %d and %d", who, src->d.page_size, src->d.num_kv_heads, dst->d.page_size,
                    dst->d.num_kv_heads);
    if (dst->d.num_kv_heads > 65535) return fail(HKV_ESHAPE, "%s: %d KV heads (65535 at most)", who, dst->d.num_kv_heads);
    dst->mark_anew();
    std::vector<PagePair> pairs;
    pairs.reserve(n);
    for (int i = 0; i < n; ++i) {
        if (dst_ids[i] < 0 || dst_ids[i] >= dst->d.num_pages)
            return fail(HKV_ERANGE, "%s: page id %d (entry %d of dst_ids) outside pool of %d pages", who, dst_ids[i], i, dst->d.num_pages);
        if (src_ids[i] < 0 || src_ids[i] >= src->d.num_pages)
            return fail(HKV_ERANGE, "%s: page id %d (entry %d of src_ids) outside pool of %d pages", who, src_ids[i], i, src->d.num_pages);
        if (dst->refcnt[dst_ids[i]] > 1) return fail(HKV_EINVAL, "%s: page %d of dst_ids has %d owners", who, dst_ids[i], dst->refcnt[dst_ids[i]]);
        if (dst->mark[dst_ids[i]] == dst->mark_now) return fail(HKV_EINVAL, "%s: page %d is in dst_ids twice", who, dst_ids[i]);
        dst->mark[dst_ids[i]] = dst->mark_now;
        const int32_t tokens = n_tokens ? n_tokens[i] : dst->d.page_size;
        if (tokens < 0 || tokens > dst->d.page_size) return fail(HKV_EINVAL, "%s: %d tokens (entry %d) of a page of %d", who, tokens, i, dst->d.page_size);
        pairs.push_back({src_ids[i], dst_ids[i], tokens});
    }
    int32_t both = -1;
    if (dst != src)
        both = read_and_written(dst, src, pairs);
    else
        for (int i = 0; i < n && both < 0; ++i)
            if (dst->mark[src_ids[i]] == dst->mark_now) both = src_ids[i];
    if (both >= 0) return fail(HKV_EINVAL, "%s: page %d is read and written", who, both);
    if (n == 0) return HKV_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (is_capturing(s)) return fail(HKV_EINVAL, "%s: not for capture into a graph", who);
    return queue_copies(dst, src, pairs, s);
} catch (const std::exception &) {  // (no memory for a list)
    return fail(HKV_ENOMEM, "kv_pool_copy_pages: out of host memory");
}

extern "C" int kv_pool_fork(hkv_pool *pool, int32_t n_seq, const int32_t *pages, const int32_t *n_tokens, int32_t n_out, const int32_t *parent, int32_t release,
                            int32_t *out_pages, void *stream) try {
    const char *who = "kv_pool_fork";
    if (!pool) return fail(HKV_EINVAL, "%s: null pool", who);
    if (n_seq < 0 || n_out < 0 || (n_seq > 0 && !n_tokens) || (n_out > 0 && !parent)) return fail(HKV_EINVAL, "%s: %d sequences, %d forks, or a null list", who, n_seq, n_out);
    if (pool->d.num_kv_heads > 65535) return fail(HKV_ESHAPE, "%s: %d KV heads (65535 at most)", who, pool->d.num_kv_heads);
    const int P = pool->d.page_size;
    std::vector<int64_t> begin(n_seq + 1, 0);
    for (int i = 0; i < n_seq; ++i) {
        if (n_tokens[i] < 0) return fail(HKV_EINVAL, "%s: sequence %d has %d tokens", who, i, n_tokens[i]);
        begin[i + 1] = begin[i] + (n_tokens[i] + (int64_t)P - 1) / P;
    }
    const int64_t total = begin[n_seq];
    if (total > 0 && !pages) return fail(HKV_EINVAL, "%s: null pages", who);
    for (int64_t i = 0; i < total; ++i) {
        if (pages[i] < 0 || pages[i] >= pool->d.num_pages)
            return fail(HKV_ERANGE, "%s: page id %d (entry %lld) outside pool of %d pages", who, pages[i], (long long)i, pool->d.num_pages);
        if (pool->refcnt[pages[i]] <= 0) return fail(HKV_EINVAL, "%s: page %d is not allocated", who, pages[i]);
    }
    if (release) {  // every listing gives a reference back, none of them a prefix cache's (counted in place, and put back)
        int64_t n = 0, bad = -1;
        for (; n < total && bad < 0; ++n) {
            int32_t cached = 0;
            for (const hkv_pool::Follower &f : pool->followers) cached += f.holds(f.object, pages[n]);
            if (--pool->refcnt[pages[n]] < cached) bad = n;
        }
        while (n-- > 0) ++pool->refcnt[pages[n]];
        if (bad >= 0) return fail(HKV_EINVAL, "%s: page %d listed more often than it is held beside prefix caches", who, pages[bad]);
    }
    std::vector<int32_t> first_fork(n_seq, -1), forks(n_seq, 0);
    int64_t out_total = 0;
    for (int j = 0; j < n_out; ++j) {
        if (parent[j] < 0 || parent[j] >= n_seq) return fail(HKV_ERANGE, "%s: fork %d of sequence %d of %d", who, j, parent[j], n_seq);
        if (first_fork[parent[j]] < 0) first_fork[parent[j]] = j;
        ++forks[parent[j]];
        out_total += begin[parent[j] + 1] - begin[parent[j]];
    }
    if (out_total > INT_MAX) return fail(HKV_EINVAL, "%s: too many pages", who);
    if (out_total > 0 && !out_pages) return fail(HKV_EINVAL, "%s: null out_pages", who);
    // a last page that is not full: the first fork takes it over where the sequence was its only owner and goes, every other fork copies it
    auto takes_over = [&](int j) {
        const int i = parent[j];
        return release && first_fork[i] == j && pool->refcnt[pages[begin[i + 1] - 1]] == 1;
    };
    std::vector<int32_t> out;
    out.reserve((size_t)out_total);
    std::vector<PagePair> copies;
    auto fresh = pool->free_list.begin();
    for (int j = 0; j < n_out; ++j) {
        const int i = parent[j];
        out.insert(out.end(), pages + begin[i], pages + begin[i + 1]);
        if (n_tokens[i] % P == 0 || takes_over(j)) continue;
        if (fresh == pool->free_list.end())
            return fail(HKV_ENOMEM, "%s: %zu pages free, fewer than the forks need for their last pages", who, pool->free_list.size());
        copies.push_back({out.back(), *fresh, n_tokens[i] % P});
        out.back() = *fresh++;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!copies.empty()) {
        if (is_capturing(s)) return fail(HKV_EINVAL, "%s: not for capture into a graph", who);  // (a replay would take the same pages again)
        if (int rc = queue_copies(pool, pool, copies, s)) return rc;
    }
    for (const PagePair &c : copies) {
        pool->free_list.pop_front();
        pool->refcnt[c.dst] = 1;
    }
    for (int j = 0; release && j < n_out; ++j)  // a last page that is taken over (given back by its sequence below)
        if (n_tokens[parent[j]] % P != 0 && takes_over(j)) ++pool->refcnt[pages[begin[parent[j] + 1] - 1]];
    for (int i = 0; i < n_seq; ++i)
        for (int64_t p = begin[i]; p < begin[i] + n_tokens[i] / P; ++p) pool->refcnt[pages[p]] += forks[i];
    if (release)
        for (int64_t i = 0; i < total; ++i)
            if (--pool->refcnt[pages[i]] == 0) pool->free_list.push_back(pages[i]);
    if (!out.empty()) memcpy(out_pages, out.data(), sizeof(int32_t) * out.size());
    return HKV_OK;
} catch (const std::exception &) {
    return fail(HKV_ENOMEM, "kv_pool_fork: out of host memory");
}

extern "C" int32_t kv_pool_compact(hkv_pool *pool, int32_t *new_ids, void *stream) try {
    const char *who = "kv_pool_compact";
    if (!pool || !new_ids) return fail(HKV_EINVAL, "%s: null argument", who);
    if (pool->d.num_kv_heads > 65535) return fail(HKV_ESHAPE, "%s: %d KV heads (65535 at most)", who, pool->d.num_kv_heads);
    const int32_t n = pool->d.num_pages;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (is_capturing(s)) return fail(HKV_EINVAL, "%s: not for capture into a graph", who);
    const int32_t live = n - (int32_t)pool->free_list.size();
    std::vector<int32_t> map(n);
    std::vector<PagePair> moves;
    moves.reserve(live);
    int32_t gap = 0;
    for (int32_t id = 0; id < n; ++id) {
        map[id] = pool->refcnt[id] > 0 ? id : -1;
        if (id < live || pool->refcnt[id] == 0) continue;
        while (pool->refcnt[gap] > 0) ++gap;
        map[id] = gap;
        moves.push_back({id, gap++, pool->d.page_size});
    }
    std::deque<int32_t> free_list(n - live);
    std::iota(free_list.begin(), free_list.end(), live);
    for (const hkv_pool::Follower &f : pool->followers) f.prepare(f.object, map.data());
    if (int rc = queue_copies(pool, pool, moves, s)) return rc;
    for (const PagePair &m : moves) {
        pool->refcnt[m.dst] = pool->refcnt[m.src];
        pool->refcnt[m.src] = 0;
    }
    pool->free_list.swap(free_list);
    for (const hkv_pool::Follower &f : pool->followers) f.commit(f.object);
    memcpy(new_ids, map.data(), sizeof(int32_t) * (size_t)n);
    return (int32_t)moves.size();
} catch (const std::exception &) {
    return fail(HKV_ENOMEM, "kv_pool_compact: out of host memory");
}
