// From a step's projections to its attention in one pass: the rows of q and k are normed per head and rotated by position, queries go
// out, keys and values into the pool's blocks.
//
// A row x of a head (128 values): y = x * w / sqrt(mean(x^2) + eps); pair i of the first rotary_dim dimensions turns by the angle
// position * inv_freq[i]; one rounding at the end (bf16), or the code of the unrounded value under its block's scale (fp8).
// The angle is taken in 64 bits and reduced to a part of a turn before it is narrowed, so that it is as exact at position 10^6 as
// at 10; a table of angles would be a second input of 512 bytes a token.
//
// 16 lanes hold a row, eight dimensions each: the sum of squares is four steps across them, the other half of a split pair comes from
// the lane eight further (whole heads: one vector instruction, else through the LDS crossbar), interleaved pairs lie in one lane.
// A workgroup takes one 16-token block of one KV head: a thread row per token, K, V and then the query heads of the group, so that the
// angles are taken once for all of them, and the fp8 scale of the block is the workgroup's own.  Where a request brings a
// single token the 16 thread rows take its K / V and its query heads side by side.
#include "pool_block.h"

namespace hkv {

namespace {

struct Unit {
    int block, lo, hi;  // slots lo .. hi - 1 of this block of the pool ...
    int64_t row;        // ... are the rows from this one on (before row_map)
    int pos;            // position of slot lo
};

template <int DT>
struct Row {
    u32x4 w[DT == 2 ? 2 : 1];
};
template <int DT>
__device__ __forceinline__ Row<DT> load_row(const void *base, int64_t stride, int64_t row, int head, int c) {
    constexpr int E = DT == 2 ? 4 : 2;
    const char *p = static_cast<const char *>(base) + (row * stride + head * kHeadDim + 8 * c) * E;
    Row<DT> r;
    r.w[0] = ld16(p);
    if constexpr (DT == 2) r.w[1] = ld16(p + 16);
    return r;
}
template <int DT>
__device__ __forceinline__ void values(const Row<DT> &r, float (&x)[8]) {
    if constexpr (DT == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(r.w[j >> 2][j & 3]);
    } else {
        unpack_bf16(r.w[0], x);
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
    return u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

// What a lane's dims 8 c .. 8 c + 7 turn by: z = x * cos + (the pair's other value) * sin, sin with the sign of the place in the pair.
struct Turn {
    float cos[8], sin[8];
    bool on;
};
template <int DT>
__device__ __forceinline__ void turn_of(const ProjectionLaunch &a, int c, int64_t row, int pos, Turn &t) {
    t.on = 8 * c < a.rotary_dim;
    if (!t.on) return;
    const int half = a.rotary_dim >> 1;
    const bool second = 8 * c >= half;
    const int p0 = a.interleaved ? 4 * c : 8 * c - (second ? half : 0);
    int p[4] = {pos, pos, pos, pos};
    if (a.positions) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < a.n_axes) p[i] = a.positions[i * a.position_stride + row];
    }
    const uint32_t axes = (p0 < 32 ? (p0 < 16 ? a.axis[0] : a.axis[1]) : (p0 < 48 ? a.axis[2] : a.axis[3])) >> (2 * (p0 & 15));
    auto angle = [&](int e, float &co, float &si) {
        const uint32_t ax = axes >> (2 * e) & 3u;
        const double place = (double)(ax < 2 ? (ax == 0 ? p[0] : p[1]) : (ax == 2 ? p[2] : p[3]));
        const double turns = place * (a.inv_freq[p0 + e] * 0.15915494309189533577);
        const float part = (float)(turns - __builtin_rint(turns));
        if constexpr (DT == 2) {
            sincospif(2.0f * part, &si, &co);
        } else {  // good to 2^-19 or so of a result that keeps 8 bits and fewer
            si = __builtin_amdgcn_sinf(part);
            co = __builtin_amdgcn_cosf(part);
        }
    };
    if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float co, si;
            angle(e, co, si);
            t.cos[2 * e] = t.cos[2 * e + 1] = co;
            t.sin[2 * e] = -si;
            t.sin[2 * e + 1] = si;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            angle(e, t.cos[e], t.sin[e]);
            if (!second) t.sin[e] = -t.sin[e];
        }
    }
}

__device__ __forceinline__ float row16_sum(float v) {
    v += dpp<kQuadXor1>(v);
    v += dpp<kQuadXor2>(v);
    v += dpp<kRor4>(v);
    return v + dpp<kRor8>(v);
}

// Norm and rotation of one row.  All 16 lanes of a row take part.
__device__ __forceinline__ void norm_and_turn(const ProjectionLaunch &a, int c, bool normed, const float (&w)[8], const Turn &t, float (&x)[8]) {
    if (normed) {
        float sq = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sq = __builtin_fmaf(x[j], x[j], sq);
        const float inv = 1.0f / __builtin_sqrtf(row16_sum(sq) * (1.0f / kHeadDim) + a.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * inv * w[j];
    }
    if (a.rotary_dim == 0) return;
    float y[8];
    if (a.interleaved) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j ^ 1];
    } else if (a.rotary_dim == kHeadDim) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = dpp<kRor8>(x[j]);
    } else {
        const int step = a.rotary_dim >> 4, lane = threadIdx.x & 63;
        const int from = !t.on ? lane : c < step ? lane + step : lane - step;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __uint_as_float(__builtin_amdgcn_ds_bpermute(4 * from, __float_as_uint(x[j])));
    }
    if (t.on) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * t.cos[j] + y[j] * t.sin[j];
    }
}

template <int DT>
__device__ __forceinline__ void load_weight(const void *w, int c, float (&x)[8]) {
    if (w) values<DT>(load_row<DT>(w, 0, 0, 0, c), x);
}

template <int DT>
__device__ __forceinline__ void put_query(const ProjectionLaunch &a, int64_t row, int head, int c, const float (&x)[8]) {
    const int64_t at = (row * (a.pool.num_kv_heads * a.group) + head) * kHeadDim + 8 * c;
    if constexpr (DT == 2) {
        float4 *o = reinterpret_cast<float4 *>(static_cast<float *>(a.q_out) + at);
        o[0] = make_float4(x[0], x[1], x[2], x[3]);
        o[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.q_out) + at) = pack8(x);
    }
}

// K (normed and turned) and V of the workgroup's slots into the block.
template <int DT>
__device__ __forceinline__ void put_block(const ProjectionLaunch &a, const Unit &u, int h, bool valid, const float (&k)[8], const Row<DT> &v) {
    if constexpr (DT == 2) {
        if (!valid) return;
        const int slot = threadIdx.x >> 4, d = 8 * (threadIdx.x & 15);
        const size_t blk = ((size_t)u.block * a.pool.num_kv_heads + h) * kBlockElems;
        float *kd = static_cast<float *>(a.pool.k_pages) + blk + (d >> 4) * 256 + slot * 16 + (d & 15);
        float *vd = static_cast<float *>(a.pool.v_pages) + blk + d * kPage + slot;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            kd[j] = k[j];
            vd[j * kPage] = __uint_as_float(v.w[j >> 2][j & 3]);
        }
    } else {
        u32x4 kw = {0u, 0u, 0u, 0u};
        if (DT == 0 && valid) kw = pack8(k);
        store_block<DT>(a.pool, u.block, h, valid, kw, k, v.w[0], u.lo, u.hi);
    }
}

// One KV head of one block with up to 16 tokens: thread row = slot.
template <int DT>
__device__ __forceinline__ void store_tokens(const ProjectionLaunch &a, const Unit &u, int h) {
    const int slot = threadIdx.x >> 4, c = threadIdx.x & 15;
    const bool valid = slot >= u.lo && slot < u.hi;
    float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    Row<DT> v{};
    if (valid) {
        int64_t row = u.row + slot - u.lo;
        if (a.row_map) row = a.row_map[row];
        const Row<DT> kr = load_row<DT>(a.k, a.k_stride, row, h, c);
        v = load_row<DT>(a.v, a.v_stride, row, h, c);
        Row<DT> q = load_row<DT>(a.q, a.q_stride, row, h * a.group, c);
        float qw[8] = {}, kwt[8] = {};
        load_weight<DT>(a.q_norm, c, qw);
        load_weight<DT>(a.k_norm, c, kwt);
        Turn t;
        turn_of<DT>(a, c, row, u.pos + slot - u.lo, t);
        values<DT>(kr, k);
        norm_and_turn(a, c, a.k_norm != nullptr, kwt, t, k);
        for (int j = 0; j < a.group; ++j) {
            float x[8];
            values<DT>(q, x);
            if (j + 1 < a.group) q = load_row<DT>(a.q, a.q_stride, row, h * a.group + j + 1, c);
            norm_and_turn(a, c, a.q_norm != nullptr, qw, t, x);
            put_query<DT>(a, row, h * a.group + j, c, x);
        }
    }
    put_block<DT>(a, u, h, valid, k, v);
}

// One KV head of one token: thread row u.lo takes K and V, the others a query head each (the 16th, too, is K's row's).
template <int DT>
__device__ __forceinline__ void store_token(const ProjectionLaunch &a, const Unit &u, int h) {
    const int g = threadIdx.x >> 4, c = threadIdx.x & 15;
    const bool valid = g == u.lo;
    const int j = (g - u.lo - 1) & 15;
    const int64_t row = a.row_map ? a.row_map[u.row] : u.row;
    float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    Row<DT> v{};
    if (valid || j < a.group) {
        Row<DT> r{}, q{};
        if (valid) {
            r = load_row<DT>(a.k, a.k_stride, row, h, c);
            v = load_row<DT>(a.v, a.v_stride, row, h, c);
        }
        if (j < a.group) q = load_row<DT>(a.q, a.q_stride, row, h * a.group + j, c);
        float w[8] = {};
        Turn t;
        turn_of<DT>(a, c, row, u.pos, t);
        if (j < a.group) {
            float x[8];
            load_weight<DT>(a.q_norm, c, w);
            values<DT>(q, x);
            norm_and_turn(a, c, a.q_norm != nullptr, w, t, x);
            put_query<DT>(a, row, h * a.group + j, c, x);
        }
        if (valid) {
            load_weight<DT>(a.k_norm, c, w);
            values<DT>(r, k);
            norm_and_turn(a, c, a.k_norm != nullptr, w, t, k);
        }
    }
    put_block<DT>(a, u, h, valid, k, v);
}

// The newest tokens of a decode plan's requests.  grid: (requests x blocks that the tokens of one can span, KV heads)
template <int DT, bool ONE>
__global__ __launch_bounds__(256) void projection_decode_kernel(ProjectionLaunch a) {
    const int spans = ONE ? 1 : (a.tokens + kPage - 2) / kPage + 1;
    const int r = blockIdx.x / spans, i = blockIdx.x % spans;
    const StoreRequest s = a.requests[r];
    int n = s.tokens;
    if (s.item >= 0) n = a.items[s.item].tok_begin + a.items[s.item].n_tokens;
    const int first = n - a.tokens, b = first / kPage + i;
    if (b * kPage >= n) return;
    Unit u;
    u.block = a.blocks[s.page_off + (uint32_t)b];
    u.lo = max(first - b * kPage, 0);
    u.hi = min(n - b * kPage, kPage);
    u.row = (int64_t)r * a.tokens + (b * kPage + u.lo - first);
    u.pos = s.pos0 + b * kPage + u.lo;
    if constexpr (ONE)
        store_token<DT>(a, u, blockIdx.y);
    else
        store_tokens<DT>(a, u, blockIdx.y);
}

// The new tokens of a prefill plan's requests.  grid: (blocks they go to, KV heads)
template <int DT>
__global__ __launch_bounds__(256) void projection_prefill_kernel(ProjectionPrefill p) {
    const int x = blockIdx.x, lane = threadIdx.x & 63;
    static_assert(kMaxInlineRequests == 128, "two entries a lane");
    const int i = __popcll(__ballot(p.begin[lane] <= x)) + __popcll(__ballot(p.begin[64 + lane] <= x)) - 1;
    const int prefix = p.prefix[i], end = prefix + p.tokens[i], b = prefix / kPage + x - p.begin[i];
    Unit u;
    u.block = p.base.blocks[p.table + (int64_t)i * p.table_stride + b];
    if (p.base.src_pages) u.block = p.base.src_pages[u.block];
    u.lo = max(prefix - b * kPage, 0);
    u.hi = min(end - b * kPage, kPage);
    u.pos = b * kPage + u.lo;
    u.row = (int64_t)p.row0[i] + u.pos - prefix;
    store_tokens<DT>(p.base, u, blockIdx.y);
}

// A growing plan's step: workgroup (r, head) stores request r's new token and lengthens the item of that head in its leaf.
template <int DT>
__global__ __launch_bounds__(256) void projection_append_kernel(ProjectionLaunch a, PlanGrowInline g) {
    const int r = blockIdx.x, h = blockIdx.y;
    const StoreRequest s = a.requests[r];
    DecodeItem *item = g.items + g.grow_items[r * a.pool.num_kv_heads + h];
    const int n = item->tok_begin + item->n_tokens, fresh = g.new_block[r];  // tokens in front of the new one
    Unit u;
    u.block = fresh >= 0 ? fresh : a.blocks[s.page_off + (uint32_t)(n / kPage)];
    u.lo = n % kPage;
    u.hi = u.lo + 1;
    u.row = r;
    u.pos = s.pos0 + n;
    store_token<DT>(a, u, h);
    __syncthreads();  // every wavefront has read the item
    if (threadIdx.x == 0) item->n_tokens += 1;
    if (threadIdx.x == 1 && h == 0 && fresh >= 0) g.pages[g.block_pos[r]] = fresh;
}

}  // namespace

hipError_t launch_projection_store(const ProjectionLaunch &a, hipStream_t s) {
    const int spans = a.tokens == 1 ? 1 : (a.tokens + kPage - 2) / kPage + 1;
    const dim3 grid((unsigned)(a.n_requests * spans), a.pool.num_kv_heads), block(256);
    if (a.n_requests <= 0) return hipSuccess;
    auto go = [&](auto one, auto many) { hipLaunchKernelGGL(a.tokens == 1 ? one : many, grid, block, 0, s, a); };
    if (a.pool.dtype == 0)
        go(projection_decode_kernel<0, true>, projection_decode_kernel<0, false>);
    else if (a.pool.dtype == 1)
        go(projection_decode_kernel<1, true>, projection_decode_kernel<1, false>);
    else
        go(projection_decode_kernel<2, true>, projection_decode_kernel<2, false>);
    return hipGetLastError();
}

hipError_t launch_projection_store(const ProjectionPrefill &a, hipStream_t s) {
    if (a.n_units <= 0) return hipSuccess;
    const dim3 grid(a.n_units, a.base.pool.num_kv_heads), block(256);
    if (a.base.pool.dtype == 0)
        hipLaunchKernelGGL(projection_prefill_kernel<0>, grid, block, 0, s, a);
    else if (a.base.pool.dtype == 1)
        hipLaunchKernelGGL(projection_prefill_kernel<1>, grid, block, 0, s, a);
    else
        hipLaunchKernelGGL(projection_prefill_kernel<2>, grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_projection_append(const ProjectionLaunch &a, const PlanGrowInline &g, hipStream_t s) {
    if (a.n_requests <= 0) return hipSuccess;
    const dim3 grid(a.n_requests, a.pool.num_kv_heads), block(256);
    if (a.pool.dtype == 0)
        hipLaunchKernelGGL(projection_append_kernel<0>, grid, block, 0, s, a, g);
    else
        hipLaunchKernelGGL(projection_append_kernel<1>, grid, block, 0, s, a, g);
    return hipGetLastError();
}

}  // namespace hkv
