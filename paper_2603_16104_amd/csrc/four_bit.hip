// Stores into 4-bit pools, and the pre-pass that widens their pages for prefill.  (Section 5, "Proactive Cache Management": a prefix's KV is computed
// once and kept; here in a quarter of its bytes.)  With x = 32 neighbouring dims of a token and head:
//   e = min(max(floor(log2(max |x|)) - 2, -126), 125),   code = e2m1(x / 2^e), to nearest, ties to even, saturated;
// every step is exact but that one rounding, so there is nothing to choose in how it is computed.
#include <algorithm>
#include <type_traits>

#include "four_bit.h"

namespace hkv {

namespace {

// One token of one KV head by 16 lanes, eight dims each: source row `row`, slot `slot` of block `block`.
__device__ __forceinline__ void write_token(const PoolWriteLaunch &a, int row, int block, int h, int slot, int c, bool valid) {
    u32x4 kw = {0u, 0u, 0u, 0u}, vw = {0u, 0u, 0u, 0u};
    if (valid) {
        const size_t src = (((size_t)row * a.num_kv_heads + h) * kHeadDim + 8 * c) * 2;
        kw = ld16(static_cast<const char *>(a.k_src) + src);
        vw = ld16(static_cast<const char *>(a.v_src) + src);
    }
    const size_t blk = (size_t)block * a.num_kv_heads + h;
    float x[8];
    four::unpack8(kw, x);
    four::put8(static_cast<uint8_t *>(a.k_pages), reinterpret_cast<uint8_t *>(a.k_scale), false, blk, slot, c, x, valid);
    four::unpack8(vw, x);
    four::put8(static_cast<uint8_t *>(a.v_pages), reinterpret_cast<uint8_t *>(a.v_scale), true, blk, slot, c, x, valid);
}

// A run of tokens: a workgroup per (block, head), thread (slot = tid / 16, c = tid % 16).
__device__ __forceinline__ void write_run(const PoolWriteLaunch &a, const int32_t *ids) {
    const int slot = threadIdx.x >> 4, row = (int)blockIdx.x * kPage + slot - a.first_slot;
    write_token(a, row, ids[blockIdx.x], blockIdx.y, slot, threadIdx.x & 15, row >= 0 && row < a.n_tokens);
}

__global__ __launch_bounds__(256) void four_write_kernel(PoolWriteLaunch a) {
    if (a.slots) {  // one token per block: 16 (token, head) pairs a workgroup
        const int u = blockIdx.x * 16 + (threadIdx.x >> 4), n = a.n_pages * a.num_kv_heads;
        const int i = min(u, n - 1) / a.num_kv_heads;
        write_token(a, i, a.page_ids[i], min(u, n - 1) % a.num_kv_heads, a.slots[i], threadIdx.x & 15, u < n);
    } else {
        write_run(a, a.page_ids);
    }
}

template <int N>
struct WriteInline {
    PoolWriteLaunch base;
    int32_t block[N];
};
template <int N>
__global__ __launch_bounds__(256) void four_write_inline_kernel(WriteInline<N> a) {
    write_run(a.base, a.block);
}

__global__ __launch_bounds__(256) void four_append_kernel(PoolAppendInline a) {
    const int u = blockIdx.x * 16 + (threadIdx.x >> 4), Hkv = a.base.num_kv_heads, n = a.base.n_pages * Hkv;
    const int i = min(u, n - 1) / Hkv;
    write_token(a.base, i, a.block[i], min(u, n - 1) % Hkv, a.slot[i], threadIdx.x & 15, u < n);
}

// A decode step's append with the plan's update: unit u = (request, head), as grow_items has them.
__global__ __launch_bounds__(256) void four_step_append_kernel(PoolAppendInline a, PlanGrowInline g) {
    const int u = blockIdx.x * 16 + (threadIdx.x >> 4), Hkv = a.base.num_kv_heads, n = a.base.n_pages * Hkv;
    const int i = min(u, n - 1) / Hkv, h = min(u, n - 1) % Hkv;
    write_token(a.base, i, a.block[i], h, a.slot[i], threadIdx.x & 15, u < n);
    if (u < n && (threadIdx.x & 15) == 0) {
        g.items[g.grow_items[u]].n_tokens += 1;
        if (h == 0 && g.new_block[i] >= 0) g.pages[g.block_pos[i]] = g.new_block[i];
    }
}

// 4-bit pages -> bf16 pages of a scratch pool (page i of the scratch = src_pages[i]), exact.  A workgroup per (page, head): K by all threads, a word
// (eight dims of a token) each; V by threads (c, half, b): dims 8 c + 2 b, + 1 of eight tokens, whose codes share byte b of eight words.
__global__ __launch_bounds__(256) void four_widen_kernel(PoolDequantLaunch a) {
    const int i = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    const size_t src = (size_t)a.src_pages[i] * a.pool.num_kv_heads + h, dst = ((size_t)i * a.pool.num_kv_heads + h) * kBlockElems;
    const uint8_t *kc = static_cast<const uint8_t *>(a.pool.k_pages) + src * four::kCodeBytes, *vc = static_cast<const uint8_t *>(a.pool.v_pages) + src * four::kCodeBytes;
    const uint8_t *ks = reinterpret_cast<const uint8_t *>(a.pool.k_scale) + src * four::kScaleBytes, *vs = reinterpret_cast<const uint8_t *>(a.pool.v_scale) + src * four::kScaleBytes;
    {
        const int t = tid >> 4, c = tid & 15;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(kc + (t & 3) * 256 + (t >> 2) * 64 + c * 4);
        const u32x4 out = four::widen8(w, four::scale_of(ks[(c >> 2) * 16 + t], 0));
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.k_dst) + dst + (c >> 2) * 512 + t * 32 + (c & 3) * 8) = out;
    }
    if (tid < 128) {
        const int c = tid >> 3, half = tid >> 2 & 1, b = tid & 3;
        const u32x4 w0 = ld16(vc + 2 * half * 256 + c * 16), w1 = ld16(vc + (2 * half + 1) * 256 + c * 16);
        const u32x2 sc = *reinterpret_cast<const u32x2 *>(vs + (c >> 2) * 16 + 8 * half);
        u32x4 lo, hi;
#pragma unroll
        for (int p = 0; p < 4; ++p) {  // tokens 2 p, 2 p + 1 of the eight
            const uint32_t x = p < 2 ? w0[2 * p] : w1[2 * p - 4], y = p < 2 ? w0[2 * p + 1] : w1[2 * p - 3];
            const uint32_t v0 = four::widen2<0>(x >> (8 * b), four::scale_of(sc[p >> 1], 2 * (p & 1)));
            const uint32_t v1 = four::widen2<0>(y >> (8 * b), four::scale_of(sc[p >> 1], 2 * (p & 1) + 1));
            lo[p] = __builtin_amdgcn_perm(v1, v0, 0x05040100u);
            hi[p] = __builtin_amdgcn_perm(v1, v0, 0x07060302u);
        }
        uint16_t *out = static_cast<uint16_t *>(a.v_dst) + dst + (8 * c + 2 * b) * kPage + 8 * half;
        *reinterpret_cast<u32x4 *>(out) = lo;
        *reinterpret_cast<u32x4 *>(out + kPage) = hi;
    }
}

unsigned units(const PoolWriteLaunch &a) { return (unsigned)(((int64_t)a.n_pages * a.num_kv_heads + 15) / 16); }

}  // namespace

hipError_t launch_four_write(const PoolWriteLaunch &a, hipStream_t s) {
    if (a.n_pages <= 0) return hipSuccess;
    if (a.slots) {
        hipLaunchKernelGGL(four_write_kernel, dim3(units(a)), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid(a.n_pages, a.num_kv_heads);
    if (a.host_ids) {
        auto go = [&](auto room) {
            constexpr int N = decltype(room)::value;
            WriteInline<N> w;
            w.base = a;
            w.base.host_ids = nullptr;
            std::copy(a.host_ids, a.host_ids + a.n_pages, w.block);
            std::fill(w.block + a.n_pages, w.block + N, 0);
            hipLaunchKernelGGL(four_write_inline_kernel<N>, grid, dim3(256), 0, s, w);
            return hipGetLastError();
        };
        if (a.n_pages > kMaxInlineWrite) return hipErrorInvalidValue;
        if (a.n_pages <= 64) return go(std::integral_constant<int, 64>{});
        return go(std::integral_constant<int, kMaxInlineWrite>{});
    }
    hipLaunchKernelGGL(four_write_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_four_append(const PoolAppendInline &a, hipStream_t s) {
    if (a.base.n_pages <= 0) return hipSuccess;
    hipLaunchKernelGGL(four_append_kernel, dim3(units(a.base)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_four_step_append(const PoolAppendInline &w, const PlanGrowInline &g, hipStream_t s) {
    if (w.base.n_pages <= 0) return hipSuccess;
    hipLaunchKernelGGL(four_step_append_kernel, dim3(units(w.base)), dim3(256), 0, s, w, g);
    return hipGetLastError();
}

hipError_t launch_four_widen(const PoolDequantLaunch &a, hipStream_t s) {
    if (a.n_pages <= 0) return hipSuccess;
    hipLaunchKernelGGL(four_widen_kernel, dim3(a.n_pages, a.pool.num_kv_heads), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace hkv
