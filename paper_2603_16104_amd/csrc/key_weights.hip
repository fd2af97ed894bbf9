// What the queries of a step gave to every cached key: W[t] = decay * W[t] + sum over rows r that see t of exp(scale * q_r . k_t - lse_r),
// rows being the query heads of a KV head of all requests below the key's node (attn_decode_plan_weights).
//
// The softmax is known already (lse), so one product is all there is: S = Q K^T on the matrix cores with the keys as columns: a lane
// holds one key and several rows of the result, so that the sum over rows is additions within the lane and one step across lanes, and rows
// that do not count cost nothing but their place in the tile.  A key belongs to one workgroup, which adds in a fixed order: no
// atomics, the same bits every time.  Two forms, by the rows R below the node:
// - R <= 16 (a request's own tokens): bound by reading K.  An item is a wavefront's; the rows are one 16-row operand in registers, and it walks
//   over its blocks, loading the next pair while the present one is multiplied; a block is four (fp8: two) contiguous loads.
// - more rows (shared prompts, windows of queries): an item is a workgroup's, bound by the exponentials, 8 of them a lane for a tile of 16 rows x 32 keys beside
//   eight matrix instructions.  The rows stay in LDS, up to 256 at a time, in the order in which the matrix operand is read, and
//   the wavefronts walk over the keys; more rows are taken in turns over the same keys.  Where there are few keys, a workgroup has 32, 64 or
//   128 of them and several wavefronts share the rows of a pair of blocks.
//
// fp32 pools: the same with the matrix instruction of that type, 16 times slower, so that its time is what counts beyond some 16 rows
// (64 requests over 2048 shared and 512 own tokens 44 us, their attention 92; 16 requests over 4096 own tokens 47 us; both the same inputs again and again.  A key a lane with a row's
// dimensions by scalar loads, without matrix instructions: 109 and 45.  Over three sets of inputs in turn, which no cache holds, 16 x 4096 tokens take 62 us, 4.4 TB/s).
//
// MI355X, 8 KV heads: 16 prompts x 8192 tokens x 256 rows alone 107 us (0.64 PFLOP/s; 48 vector instructions a step of 16 x 32, 8 of them exponentials); 1024 requests'
// own 2048 tokens alone (fp8) 375 to 440 us, 4.9 to 5.7 TB/s of keys beside their weights; both kinds (512 requests), 1.29 GB, 273 us.  Rows and keys the other way round (queries as
// columns, a shuffle a row for every sum) took 607 us there, tiles of 32 rows whose exponentials wait for their products 311.
#include <climits>
#include <type_traits>

#include "hkv_device.h"

namespace hkv {

namespace {

constexpr int kWaves = kWeightWaves, kThreads = 64 * kWaves, kRowsAtOnce = 256;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// A row as the kernel needs it: its place in q, and its lse in powers of two (+inf: it adds nothing, zeros are taken for its q).
struct QueryRow {
    int64_t q;
    float lse2;
    int limit;                // of the node's tokens: it sees those before `limit` and, of the 64 from there on, those whose bit of `mask` is set
    unsigned long long mask;
};
// The row's place alone, and its row of the plan (-1: there is none; the place is then the first row's) ...
__device__ __forceinline__ int64_t row_place(const KeyWeightsLaunch &a, const KeyWeightItem &it, int r, int G, int *row) {
    const bool there = r < it.n_req * G;
    r = there ? r : 0;
    const int j = (int)((uint32_t)r / (uint32_t)G), own = a.node_req_idx[it.req_off + j];
    *row = there ? own : -1;
    return ((int64_t)(a.q_rows ? a.q_rows[own] : own) * a.num_q_heads + it.kv_head * G + (r - j * G)) * kHeadDim;
}
// ... and what else there is to know.
__device__ __forceinline__ QueryRow row_at(const KeyWeightsLaunch &a, const KeyWeightItem &it, int64_t q, int row) {
    QueryRow x{q, INFINITY, INT_MAX, 0};
    if (row < 0) return x;
    const float lse = a.lse[q / kHeadDim];
    if (fabsf(lse) < INFINITY) x.lse2 = lse * kLog2e;
    if (a.row_leaf && a.row_leaf[row] == it.node) {
        x.limit = a.row_limit[row];
        x.mask = a.row_mask[row];
    }
    return x;
}
__device__ __forceinline__ bool sees(int limit, unsigned long long mask, int t) { return t < limit || (mask >> min(t - limit, 63) & 1); }

// The item's blocks: lane l holds the id of block l (of up to 64) and, fp8, its scale.  They are read from other lanes, so only where the
// whole wavefront runs.
struct Blocks {
    int id, n;
    float scale;
};
__device__ __forceinline__ int64_t place(const KeyWeightsLaunch &a, const KeyWeightItem &it, const Blocks &b, int i) {
    return (int64_t)__builtin_amdgcn_readlane(b.id, min(i, b.n - 1)) * a.pool.num_kv_heads + it.kv_head;
}
template <int DT>
__device__ __forceinline__ float factor(const KeyWeightsLaunch &a, const Blocks &b, int i) {
    const float c = a.scale * kLog2e;
    return DT == 0 ? c : c * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(b.scale), min(i, b.n - 1)));
}

// 32 keys (two blocks) of a wavefront, as loaded, and what they weighed.
template <int DT>
struct Keys {
    u32x4 w[DT == 0 ? 8 : 4];
    float old;
};
template <int DT>
__device__ __forceinline__ bf16x8 operand(const Keys<DT> &k, int i) {
    if constexpr (DT == 0) return as_bf16x8(k.w[i]);
    return fp8x8_to_bf16x8(k.w[i >> 1][2 * (i & 1)], k.w[i >> 1][2 * (i & 1) + 1]);
}
// The weight that a lane of the lower half writes for pair `tile` of blocks: block lane / 16, slot lane % 16.
__device__ __forceinline__ int64_t weight_place(const KeyWeightsLaunch &a, const KeyWeightItem &it, const Blocks &b, int tile) {
    const int lane = threadIdx.x & 63;
    const int64_t p0 = place(a, it, b, 2 * tile), p1 = place(a, it, b, 2 * tile + 1);
    return (lane & 16 ? p1 : p0) * kPage + (lane & 15);
}
// What the keys of pair `tile` get: `sum` in lanes 0 .. 31, a key each.
__device__ __forceinline__ void put_weight(const KeyWeightsLaunch &a, const KeyWeightItem &it, const Blocks &b, int tile, int n_node, bool first, float old, float sum) {
    const int lane = threadIdx.x & 63, t = it.tok_begin + 32 * tile + lane;
    const int64_t at = weight_place(a, it, b, tile);
    if (lane >= 32 || t >= min(it.tok_begin + it.length, n_node)) return;
    if (sum != sum) sum = 0.f;  // a key that is no number: rows whose lse is one gave it nothing, and those without one and those that fill the tile give NaN
    if (first && (a.decay == 0.f || (it.node >= 0 && t >= n_node - a.n_new))) old = 0.f;
    a.weights[at] = first ? __builtin_fmaf(a.decay, old, sum) : old + sum;
}

// Dims that lane group g (of 16) holds of matrix step kk (of 4): fp8: 16 codes of a load are two steps (the order of the sum is free).
template <int DT>
__device__ __forceinline__ int dim_of(int kk, int g) { return DT == 0 ? 32 * kk + 8 * g : 64 * (kk >> 1) + 16 * g + 8 * (kk & 1); }

template <int DT>
__device__ __forceinline__ void load_keys(const KeyWeightsLaunch &a, const KeyWeightItem &it, const Blocks &b, int tile, bool first, Keys<DT> &k) {
    const int lane = threadIdx.x & 63, slot = lane & 15, g = lane >> 4;
    k.old = 0.f;
    if (!first || a.decay != 0.f) k.old = a.weights[weight_place(a, it, b, tile)];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t at = place(a, it, b, 2 * tile + i) * kBlockElems;
        if constexpr (DT == 0) {
            const uint16_t *p = static_cast<const uint16_t *>(a.pool.k_pages) + at + slot * 32 + 8 * g;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) k.w[4 * i + kk] = ld16_stream(p + kk * 512);
        } else {
            const uint8_t *p = static_cast<const uint8_t *>(a.pool.k_pages) + at + slot * 64 + 16 * g;
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) k.w[2 * i + kk] = ld16_stream(p + kk * 1024);
        }
    }
}
// ---- up to 16 rows
template <int DT>
__device__ __forceinline__ void few_rows(const KeyWeightsLaunch &a, const KeyWeightItem &it, const Blocks &b, int n_node, int G) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    int row;
    const int64_t row_q = row_place(a, it, lane & 15, G, &row);
    const QueryRow r = row_at(a, it, row_q, row);
    const int n_tiles = (b.n + 1) / 2;
    constexpr int T = DT == 0 ? 1 : 2;  // pairs of blocks at a time: 8 KiB are on their way while as many are multiplied
    Keys<DT> k[T], next[T];
#pragma unroll
    for (int i = 0; i < T; ++i) load_keys<DT>(a, it, b, i, true, k[i]);  // (behind the last block: that one again)
    bf16x8 q[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) q[kk] = as_bf16x8(ld16(static_cast<const uint16_t *>(a.q) + r.q + dim_of<DT>(kk, g)));
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
        if (!(r.lse2 < INFINITY)) q[kk] = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
    float lse2[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)  // the result's rows 4 g + i
        lse2[i] = __uint_as_float(__builtin_amdgcn_ds_bpermute(4 * (4 * g + i), __float_as_uint(r.lse2)));
    for (int first = 0; first < n_tiles; first += T) {
        if (first + T < n_tiles)
#pragma unroll
            for (int i = 0; i < T; ++i) load_keys<DT>(a, it, b, first + T + i, true, next[i]);
#pragma unroll
        for (int x = 0; x < T; ++x) {
            const int tile = first + x, t0 = it.tok_begin + 32 * tile;
            const bool partial = a.row_leaf && it.node >= 0 && t0 + 32 > n_node - a.tokens_per_req;
            float sum[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float c = factor<DT>(a, b, 2 * tile + j);
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) s = mfma16(q[kk], operand<DT>(k[x], 4 * j + kk), s);
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = fast_exp2(__builtin_fmaf(s[i], c, -lse2[i]));
                if (partial) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int from = 4 * (4 * g + i);
                        const uint32_t lo = __builtin_amdgcn_ds_bpermute(from, (uint32_t)r.mask), hi = __builtin_amdgcn_ds_bpermute(from, (uint32_t)(r.mask >> 32));
                        if (!sees(__builtin_amdgcn_ds_bpermute(from, r.limit), (unsigned long long)hi << 32 | lo, t0 + 16 * j + (lane & 15))) p[i] = 0.f;
                    }
                }
                sum[j] = rows_sum((p[0] + p[1]) + (p[2] + p[3]));
            }
            put_weight(a, it, b, tile, n_node, true, k[x].old, lane & 16 ? sum[1] : sum[0]);
        }
#pragma unroll
        for (int i = 0; i < T; ++i) k[i] = next[i];
    }
}

// ---- more rows
// What many_rows keeps in LDS.
constexpr int kRowTiles = kRowsAtOnce / 16;
struct Rows {
    u32x4 q[kRowTiles][4][64];  // operands [row tile][step][lane]
    float lse2[kRowsAtOnce];
    int limit[kRowsAtOnce];
    unsigned long long mask[kRowsAtOnce];
    int64_t place[kRowsAtOnce];
    float sum[kWaves][32];
};
// The sums over the row tiles rt0, rt0 + step, ... of two blocks of keys, a quarter of them in each quarter of the wavefront.  The matrix
// instructions of a row tile run while the exponentials of the one before are taken.
template <int DT, bool PARTIAL>
__device__ __forceinline__ void sum_rows(const Rows &s, const Keys<DT> &keys, float c0, float c1, int rt0, int step, int row_tiles, int t, float (&sum)[2]) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    sum[0] = sum[1] = 0.f;
    if (rt0 >= row_tiles) return;
    bf16x8 k[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = operand<DT>(keys, i);
    u32x4 q[4];
    f32x4 x0, x1;
    auto load = [&](int rt) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) q[kk] = s.q[rt][kk][lane];
    };
    auto multiply = [&](f32x4 &a0, f32x4 &a1) {
        a0 = a1 = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            a0 = mfma16(as_bf16x8(q[kk]), k[kk], a0);
            a1 = mfma16(as_bf16x8(q[kk]), k[4 + kk], a1);
        }
    };
    load(rt0);
    multiply(x0, x1);
    load(min(rt0 + step, row_tiles - 1));
    // one row tile: x holds its products, y receives the next tile's
    auto tile = [&](int rt, f32x4 &x0, f32x4 &x1, f32x4 &y0, f32x4 &y1) {
        const float4 l = *reinterpret_cast<const float4 *>(s.lse2 + 16 * rt + 4 * g);  // rows 4 g .. + 3
        multiply(y0, y1);  // (behind the last tile: it once more, for nothing)
        load(min(rt + 2 * step, row_tiles - 1));
        float p[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float li = i == 0 ? l.x : i == 1 ? l.y : i == 2 ? l.z : l.w;
            p[i] = fast_exp2(__builtin_fmaf(x0[i], c0, -li));
            p[4 + i] = fast_exp2(__builtin_fmaf(x1[i], c1, -li));
        }
        if constexpr (PARTIAL) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 16 * rt + 4 * g + i;
                if (!sees(s.limit[r], s.mask[r], t)) p[i] = 0.f;
                if (!sees(s.limit[r], s.mask[r], t + 16)) p[4 + i] = 0.f;
            }
        }
        sum[0] += (p[0] + p[1]) + (p[2] + p[3]);
        sum[1] += (p[4] + p[5]) + (p[6] + p[7]);
    };
    f32x4 y0, y1;
    for (int rt = rt0; rt < row_tiles; rt += 2 * step) {
        tile(rt, x0, x1, y0, y1);
        if (rt + step < row_tiles) tile(rt + step, y0, y1, x0, x1);
    }
}
template <int DT>
__device__ __forceinline__ void many_rows(const KeyWeightsLaunch &a, const KeyWeightItem &it, const Blocks &b, int n_node, int G, Rows &s) {
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index(), g = lane >> 4;
    const int n_rows = it.n_req * G, n_tiles = (b.n + 1) / 2;
    const int at_once = min(it.length / 32, kWaves), step = kWaves / at_once;  // pairs of blocks at a time, wavefronts that share the rows of one
    for (int r0 = 0; r0 < n_rows; r0 += kRowsAtOnce) {
        const bool first = r0 == 0;
        const int row_tiles = min((n_rows - r0 + 15) / 16, kRowTiles);
        // rows into LDS: first their places, then what is known of them while a wavefront loads step `wave % 4` of every second row tile
        if (!first) __syncthreads();
        int row = -1;
        int64_t q = 0;
        if (tid < kRowsAtOnce) s.place[tid] = q = row_place(a, it, r0 + tid, G, &row);
        __syncthreads();
        auto bring = [&](auto count) {
            constexpr int N = decltype(count)::value;
            u32x4 w[N];
#pragma unroll
            for (int i = 0; i < N; ++i)
                w[i] = ld16(static_cast<const uint16_t *>(a.q) + s.place[16 * (2 * i + (wave >> 2)) + (lane & 15)] + dim_of<DT>(wave & 3, g));
            if (tid < kRowsAtOnce) {
                const QueryRow r = row_at(a, it, q, row);
                s.lse2[tid] = r.lse2;
                s.limit[tid] = r.limit;
                s.mask[tid] = r.mask;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int rt = 2 * i + (wave >> 2);
                s.q[rt][wave & 3][lane] = s.lse2[16 * rt + (lane & 15)] < INFINITY ? w[i] : u32x4{0u, 0u, 0u, 0u};
            }
        };
        if (row_tiles <= 4)
            bring(std::integral_constant<int, 2>{});
        else
            bring(std::integral_constant<int, kRowTiles / 2>{});
        __syncthreads();
        for (int tile0 = 0; tile0 < n_tiles; tile0 += at_once) {
            const int tile = tile0 + (wave & (at_once - 1)), rt0 = step == 1 ? 0 : wave / at_once;
            Keys<DT> k;
            load_keys<DT>(a, it, b, tile, first, k);
            const int t0 = it.tok_begin + 32 * tile;
            const float c0 = factor<DT>(a, b, 2 * tile), c1 = factor<DT>(a, b, 2 * tile + 1);
            float sums[2];
            if (a.row_leaf && it.node >= 0 && t0 + 32 > n_node - a.tokens_per_req)
                sum_rows<DT, true>(s, k, c0, c1, rt0, step, row_tiles, t0 + (lane & 15), sums);
            else
                sum_rows<DT, false>(s, k, c0, c1, rt0, step, row_tiles, 0, sums);
            sums[0] = rows_sum(sums[0]);
            sums[1] = rows_sum(sums[1]);
            float sum = lane & 16 ? sums[1] : sums[0];
            if (step > 1) {  // (one pass over the keys, then)
                if (lane < 32) s.sum[wave][lane] = sum;
                __syncthreads();
                if (rt0 > 0) break;
                for (int w = wave + at_once; w < kWaves; w += at_once) sum += s.sum[w][lane & 31];
            }
            put_weight(a, it, b, tile, n_node, first, k.old, sum);
        }
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads, 4) void key_weights_kernel(KeyWeightsLaunch a) {
    __shared__ Rows rows;
    const KeyWeightItem it = a.items[blockIdx.x * kWaves + wave_index()];  // (of many rows: the same for all)
    int n_node = it.tokens;
    if (it.item >= 0) n_node = a.plan_items[it.item].tok_begin + a.plan_items[it.item].n_tokens;
    const int n = min(it.length, n_node - it.tok_begin);
    if (n <= 0) return;
    const int G = a.num_q_heads / a.pool.num_kv_heads;
    Blocks b;
    b.n = (n + kPage - 1) / kPage;
    b.id = a.pages[it.page_off + min((int)threadIdx.x & 63, b.n - 1)];
    b.scale = DT == 0 ? 1.f : a.pool.k_scale[(int64_t)b.id * a.pool.num_kv_heads + it.kv_head];
    if (it.n_req * G <= 16)
        few_rows<DT>(a, it, b, n_node, G);
    else
        many_rows<DT>(a, it, b, n_node, G, rows);
}

// ---- fp32 pools
struct Rows32 {
    float q[16][kHeadDim + 4];
    float lse2[16];
    int limit[16];
    unsigned long long mask[16];
};
// Workgroup: an item.  A wavefront holds a pair of blocks; the rows come by in tiles of 16, through LDS, the next tile's on their way meanwhile.
__global__ __launch_bounds__(64 * kFp32Waves) void key_weights_fp32_kernel(KeyWeightsLaunch a) {
    static_assert(kFp32Waves == 4, "16 threads a row");
    __shared__ __align__(16) Rows32 s;
    const KeyWeightItem it = a.items[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_index(), g = lane >> 4, G = a.num_q_heads / a.pool.num_kv_heads;
    const int n_rows = it.n_req * G, row_tiles = (n_rows + 15) / 16;
    Blocks b;
    b.n = (min(it.length, it.tokens - it.tok_begin) + kPage - 1) / kPage;
    b.id = a.pages[it.page_off + min(lane, b.n - 1)];
    b.scale = 1.f;
    const float c = a.scale * kLog2e;
    // 16 threads bring a row: its place, two pieces of it, what is known of it
    auto row_of = [&](int rt, int *row) { return row_place(a, it, 16 * rt + (tid >> 4), G, row); };
    u32x4 w[2];
    QueryRow info;
    auto fetch = [&](int64_t q, int row) {
        const float *p = static_cast<const float *>(a.q) + q + 8 * (tid & 15);
        w[0] = ld16(p);
        w[1] = ld16(p + 4);
        info = row_at(a, it, q, row);
    };
    for (int first = 0; first < (b.n + 1) / 2; first += kFp32Waves) {
        const int tile = first + wave, t0 = it.tok_begin + 32 * tile;
        f32x4 k[2][8];  // dims 16 i + 4 g .. + 3 of a key, which are steps 4 i .. 4 i + 3 of the product
        float old = 0.f, sum[2] = {0.f, 0.f};
        if (a.decay != 0.f) old = a.weights[weight_place(a, it, b, tile)];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float *p = static_cast<const float *>(a.pool.k_pages) + place(a, it, b, 2 * tile + j) * kBlockElems + (lane & 15) * 16 + 4 * g;
#pragma unroll
            for (int i = 0; i < 8; ++i) k[j][i] = *reinterpret_cast<const f32x4 *>(p + 256 * i);
        }
        const bool staged = row_tiles == 1 && first > 0, partial = a.row_leaf && it.node >= 0 && t0 + 32 > it.tokens - a.tokens_per_req;
        int next_row;
        int64_t next_q = 0;
        if (!staged) {
            next_q = row_of(0, &next_row);
            fetch(next_q, next_row);
            next_q = row_of(1, &next_row);
        }
        for (int rt = 0; rt < row_tiles; ++rt) {
            if (!staged) {
                __syncthreads();  // the tile before has been read
                const bool counts = info.lse2 < INFINITY;
                float *p = s.q[tid >> 4] + 8 * (tid & 15);
                *reinterpret_cast<u32x4 *>(p) = counts ? w[0] : u32x4{0u, 0u, 0u, 0u};
                *reinterpret_cast<u32x4 *>(p + 4) = counts ? w[1] : u32x4{0u, 0u, 0u, 0u};
                if ((tid & 15) == 0) {
                    s.lse2[tid >> 4] = info.lse2;
                    s.limit[tid >> 4] = info.limit;
                    s.mask[tid >> 4] = info.mask;
                }
                __syncthreads();
                if (rt + 1 < row_tiles) {
                    fetch(next_q, next_row);
                    next_q = row_of(rt + 2, &next_row);
                }
            }
            f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x4 q = *reinterpret_cast<const f32x4 *>(s.q[lane & 15] + 16 * i + 4 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < 2; ++j) x[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[e], k[j][i][e], x[j], 0, 0, 0);
            }
            const float4 l = *reinterpret_cast<const float4 *>(s.lse2 + 4 * g);  // the result's rows 4 g .. 4 g + 3
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = fast_exp2(__builtin_fmaf(x[j][i], c, -(i == 0 ? l.x : i == 1 ? l.y : i == 2 ? l.z : l.w)));
                    if (partial && !sees(s.limit[4 * g + i], s.mask[4 * g + i], t0 + 16 * j + (lane & 15))) p[i] = 0.f;
                }
                sum[j] += (p[0] + p[1]) + (p[2] + p[3]);
            }
        }
        sum[0] = rows_sum(sum[0]);
        sum[1] = rows_sum(sum[1]);
        put_weight(a, it, b, tile, it.tokens, true, old, lane & 16 ? sum[1] : sum[0]);
    }
}

}  // namespace

hipError_t launch_key_weights(const KeyWeightsLaunch &a, hipStream_t s) {
    if (a.n_items <= 0) return hipSuccess;
    if (a.pool.dtype == 2)
        hipLaunchKernelGGL(key_weights_fp32_kernel, dim3(a.n_items), dim3(64 * kFp32Waves), 0, s, a);
    else if (a.pool.dtype == 0)
        hipLaunchKernelGGL(key_weights_kernel<0>, dim3(a.n_items / kWaves), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL(key_weights_kernel<1>, dim3(a.n_items / kWaves), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace hkv
