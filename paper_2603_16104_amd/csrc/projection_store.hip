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

// (By value: a choice between variables, or of an array's element, goes through memory, LDS whose place the wavefront then reads from the
// dispatch packet in host memory: 14 us a launch.)
__device__ __forceinline__ int choose(uint32_t i, int a, int b, int c, int d) { return i < 2 ? (i == 0 ? +a : +b) : (i == 2 ? +c : +d); }

// Cosine and sine of N pairs from p0 on (a multiple of N) of the row's angles.
template <int DT, int N>
__device__ __forceinline__ void angles(const ProjectionLaunch &a, int p0, int64_t row, int pos, float (&co)[N], float (&si)[N]) {
    double freq[N];
#pragma unroll
    for (int e = 0; e < N; ++e) freq[e] = a.inv_freq[p0 + e];
    int on0 = pos, on1 = pos, on2 = pos, on3 = pos;
    if (a.positions) {
        on0 = a.positions[row];
        if (a.n_axes > 1) on1 = a.positions[a.position_stride + row];
        if (a.n_axes > 2) on2 = a.positions[2 * a.position_stride + row];
        if (a.n_axes > 3) on3 = a.positions[3 * a.position_stride + row];
    }
    const uint32_t axes = (p0 < 32 ? (p0 < 16 ? a.axis[0] : a.axis[1]) : (p0 < 48 ? a.axis[2] : a.axis[3])) >> (2 * (p0 & 15));
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int place = a.n_axes == 1 ? on0 : choose(axes >> (2 * e) & 3u, on0, on1, on2, on3);
        const double turns = (double)place * (freq[e] * 0.15915494309189533577);
        const float part = (float)(turns - __builtin_rint(turns));
        if constexpr (DT == 2) {
            sincospif(2.0f * part, &si[e], &co[e]);
        } else {  // off by 1.25e-7 at most (2^24 parts tried): results keep 8 bits
            si[e] = __builtin_amdgcn_sinf(part);
            co[e] = __builtin_amdgcn_cosf(part);
        }
    }
}

// What a lane's dims 8 c .. 8 c + 7 turn by: z = x * cos + (the pair's other value) * sin, sin with the sign of the place in the pair.
struct Turn {
    float cos[8], sin[8];
    bool on;
};
// From a row's table of cosines and sines, [2][64] in LDS.
__device__ __forceinline__ void turn_of(const ProjectionLaunch &a, const float *table, int c, Turn &t) {
    t.on = 8 * c < a.rotary_dim;
    if (!t.on) return;
    const float4 *co = reinterpret_cast<const float4 *>(table), *si = co + 16;
    if (a.interleaved) {
        const float4 x = co[c], y = si[c];
        t.cos[0] = t.cos[1] = x.x, t.cos[2] = t.cos[3] = x.y, t.cos[4] = t.cos[5] = x.z, t.cos[6] = t.cos[7] = x.w;
        t.sin[0] = -y.x, t.sin[1] = y.x, t.sin[2] = -y.y, t.sin[3] = y.y, t.sin[4] = -y.z, t.sin[5] = y.z, t.sin[6] = -y.w, t.sin[7] = y.w;
    } else {
        const bool second = 16 * c >= a.rotary_dim;
        const int p = 2 * c - (second ? a.rotary_dim >> 3 : 0);
        const float s = second ? 1.0f : -1.0f;
        const float4 x0 = co[p], x1 = co[p + 1], y0 = si[p], y1 = si[p + 1];
        t.cos[0] = x0.x, t.cos[1] = x0.y, t.cos[2] = x0.z, t.cos[3] = x0.w, t.cos[4] = x1.x, t.cos[5] = x1.y, t.cos[6] = x1.z, t.cos[7] = x1.w;
        t.sin[0] = s * y0.x, t.sin[1] = s * y0.y, t.sin[2] = s * y0.z, t.sin[3] = s * y0.w;
        t.sin[4] = s * y1.x, t.sin[5] = s * y1.y, t.sin[6] = s * y1.z, t.sin[7] = s * y1.w;
    }
}

__device__ __forceinline__ float row16_sum(float v) {
    v += dpp<kQuadXor1>(v);
    v += dpp<kQuadXor2>(v);
    v += dpp<kRor4>(v);
    return v + dpp<kRor8>(v);
}

__device__ __forceinline__ float row16_max(float v) {
    v = fmaxf(v, dpp<kQuadXor1>(v));
    v = fmaxf(v, dpp<kQuadXor2>(v));
    v = fmaxf(v, dpp<kRor4>(v));
    return fmaxf(v, dpp<kRor8>(v));
}

// Norm and rotation of one row.  All 16 lanes of a row take part.
__device__ __forceinline__ void norm_and_turn(const ProjectionLaunch &a, int c, bool normed, const float (&w)[8], const Turn &t, float (&x)[8]) {
    if (normed) {
        float sq = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sq = __builtin_fmaf(x[j], x[j], sq);
        const float inv = __builtin_amdgcn_rsqf(row16_sum(sq) * (1.0f / kHeadDim) + a.eps);
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
    __shared__ __align__(16) float sTurn[kPage][2 * 64 + 4];
    const int slot = threadIdx.x >> 4, c = threadIdx.x & 15;
    const bool valid = slot >= u.lo && slot < u.hi;
    constexpr int kAhead = 4;  // query rows on their way
    int64_t row = u.row + max(0, min(slot, u.hi - 1) - u.lo);
    if (a.row_map) row = a.row_map[row];
    float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    Row<DT> v{};
    if (valid) {
        const Row<DT> kr = load_row<DT>(a.k, a.k_stride, row, h, c);
        v = load_row<DT>(a.v, a.v_stride, row, h, c);
        Row<DT> q[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (j < a.group) q[j] = load_row<DT>(a.q, a.q_stride, row, h * a.group + j, c);
        float qw[8] = {}, kw[8] = {};
        load_weight<DT>(a.q_norm, c, qw);
        load_weight<DT>(a.k_norm, c, kw);
        // four angles a lane; the row's lanes, of one wavefront, bring theirs together
        if (8 * c < a.rotary_dim) {
            float co[4], si[4];
            angles<DT, 4>(a, 4 * c, row, u.pos + slot - u.lo, co, si);
            *reinterpret_cast<float4 *>(&sTurn[slot][4 * c]) = make_float4(co[0], co[1], co[2], co[3]);
            *reinterpret_cast<float4 *>(&sTurn[slot][64 + 4 * c]) = make_float4(si[0], si[1], si[2], si[3]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        Turn t;
        turn_of(a, sTurn[slot], c, t);
        values<DT>(kr, k);
        norm_and_turn(a, c, a.k_norm != nullptr, kw, t, k);
        for (int j0 = 0; j0 < a.group; j0 += kAhead) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int head = j0 + j;
                if (head >= a.group) break;
                float x[8];
                values<DT>(q[j], x);
                if (head + kAhead < a.group) q[j] = load_row<DT>(a.q, a.q_stride, row, h * a.group + head + kAhead, c);
                norm_and_turn(a, c, a.q_norm != nullptr, qw, t, x);
                put_query<DT>(a, row, h * a.group + head, c, x);
            }
        }
    }
    put_block<DT>(a, u, h, valid, k, v);
}

// K and V of one token, by the 16 lanes of its thread row; all threads of the workgroup call.  fp8 blocks that are continued: as
// store_block, but the scales are found without the other wavefronts, and the workgroup comes together only to round earlier codes again.
template <int DT>
__device__ __forceinline__ void put_token(const ProjectionLaunch &a, const Unit &u, int h, bool valid, const float (&k)[8], const Row<DT> &v) {
    const int tid = threadIdx.x, c = tid & 15, d = 8 * c;
    const size_t blk = ((size_t)u.block * a.pool.num_kv_heads + h) * kBlockElems;
    if constexpr (DT == 0) {
        if (!valid) return;
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.pool.k_pages) + blk + (d >> 5) * 512 + u.lo * 32 + (d & 31)) = pack8(k);
        uint16_t *vd = static_cast<uint16_t *>(a.pool.v_pages) + blk + d * kPage + u.lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) vd[j * kPage] = (uint16_t)(v.w[0][j >> 1] >> (16 * (j & 1)));
    } else if constexpr (DT == 1) {
        __shared__ float sScales[4];  // K's and V's old scale, and new
        const size_t at = (size_t)u.block * a.pool.num_kv_heads + h;
        uint8_t *kb = static_cast<uint8_t *>(a.pool.k_pages) + blk, *vb = static_cast<uint8_t *>(a.pool.v_pages) + blk;
        if (valid) {
            float vf[8], am[2] = {0.f, 0.f}, old[2] = {0.f, 0.f}, sc[2];
            unpack_bf16(v.w[0], vf);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                am[0] = fmaxf(am[0], fabsf(k[j]));
                am[1] = fmaxf(am[1], fabsf(vf[j]));
            }
            if (u.lo > 0) {
                old[0] = a.pool.k_scale[at];
                old[1] = a.pool.v_scale[at];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float m = row16_max(am[i]);
                const float cand = m > 0.f ? m / 448.0f : 0.f;
                sc[i] = u.lo > 0 && old[i] >= cand ? old[i] : cand;  // an unset (NaN) old scale gives cand
                if (!(sc[i] > 0.f)) sc[i] = 1.0f;
            }
            if (c == 0) {
                a.pool.k_scale[at] = sc[0];
                a.pool.v_scale[at] = sc[1];
                sScales[0] = old[0];
                sScales[1] = old[1];
                sScales[2] = sc[0];
                sScales[3] = sc[1];
            }
            *reinterpret_cast<u32x2 *>(kb + (d >> 6) * 1024 + u.lo * 64 + (d & 63)) = u32x2{quant4(k[0], k[1], k[2], k[3], sc[0]), quant4(k[4], k[5], k[6], k[7], sc[0])};
            const u32x2 vc = {quant4(vf[0], vf[1], vf[2], vf[3], sc[1]), quant4(vf[4], vf[5], vf[6], vf[7], sc[1])};
#pragma unroll
            for (int j = 0; j < 8; ++j) vb[(d + j) * kPage + u.lo] = (uint8_t)(vc[j >> 2] >> (8 * (j & 3)));
        }
        if (u.lo == 0) return;
        __syncthreads();
        const float ko = sScales[0], vo = sScales[1], ks = sScales[2], vs = sScales[3];
        const int slot = tid >> 4;
        if (ks > ko && slot < u.lo) {
            u32x2 *p = reinterpret_cast<u32x2 *>(kb + (d >> 6) * 1024 + slot * 64 + (d & 63));
            const u32x2 w = *p;
            *p = u32x2{requant4(w[0], ko, ks), requant4(w[1], ko, ks)};
        }
        const int s0 = 8 * (tid & 1);
        if (vs > vo && s0 < u.lo) {  // eight slots of a dimension
            uint8_t *p = vb + (tid >> 1) * kPage + s0;
            u32x2 w = *reinterpret_cast<const u32x2 *>(p);
            w[0] = requant4(w[0], vo, vs);
            w[1] = requant4(w[1], vo, vs);
            if (s0 + 8 <= u.lo)
                *reinterpret_cast<u32x2 *>(p) = w;
            else
                for (int j = 0; s0 + j < u.lo; ++j) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
        }
    } else {
        put_block<DT>(a, u, h, valid, k, v);
    }
}

// One KV head of one token: thread row u.lo takes K and V, the others a query head each (the 16th, too, is K's row's).
template <int DT>
__device__ __forceinline__ void store_token(const ProjectionLaunch &a, const Unit &u, int h) {
    __shared__ __align__(16) float sTurn[2 * 64];
    const int g = threadIdx.x >> 4, c = threadIdx.x & 15;
    const bool valid = g == u.lo;
    const int j = (g - u.lo - 1) & 15;
    const int64_t row = a.row_map ? a.row_map[u.row] : u.row;
    float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    Row<DT> kr{}, v{}, q{};
    float w[8] = {}, kw[8] = {};
    if (valid) {
        kr = load_row<DT>(a.k, a.k_stride, row, h, c);
        v = load_row<DT>(a.v, a.v_stride, row, h, c);
        load_weight<DT>(a.k_norm, c, kw);
    }
    if (j < a.group) {
        q = load_row<DT>(a.q, a.q_stride, row, h * a.group + j, c);
        load_weight<DT>(a.q_norm, c, w);
    }
    if ((int)threadIdx.x < a.rotary_dim / 2) {  // an angle a lane, for all heads
        float co[1], si[1];
        angles<DT, 1>(a, threadIdx.x, row, u.pos, co, si);
        sTurn[threadIdx.x] = co[0];
        sTurn[64 + threadIdx.x] = si[0];
    }
    __syncthreads();
    if (valid || j < a.group) {
        Turn t;
        turn_of(a, sTurn, c, t);
        if (j < a.group) {
            float x[8];
            values<DT>(q, x);
            norm_and_turn(a, c, a.q_norm != nullptr, w, t, x);
            put_query<DT>(a, row, h * a.group + j, c, x);
        }
        if (valid) {
            values<DT>(kr, k);
            norm_and_turn(a, c, a.k_norm != nullptr, kw, t, k);
        }
    }
    put_token<DT>(a, u, h, valid, k, v);
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
