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
// angles are taken once for all of them, and the fp8 scale of the block is the workgroup's own.  Where a request brings one or two tokens, the 16 thread rows take 16
// of a token's heads (512 requests x 72 rows, fp8: 9.7 to 10.6 us; a workgroup per KV head, most of whose thread rows had nothing to do, 12.6), and up to 24 tokens, its queries
// go that way and its keys and values by blocks.
//
// Many tokens are bound by memory: 29 000 tokens of 32 + 8 heads, 708 MB, 154 us, 4.6 TB/s (fp8: 649 MB, 143; fp32, whose V leaves as single floats 64 bytes apart: 1417 MB,
// 350 us, 4.0 TB/s).  Few tokens are bound by latency: a launch, the loads of the rows
// beside those that find the block, angles, stores: 64 requests 3.9 us, four 2.6.  V's part of a block is 16 tokens wide, so that a single token
// costs a write of 32 bytes (fp8: 16) for every dimension of its V: 8 MB for the 512 requests, whose keys and values are 1 MB, beside 8 MB of queries.
#include "pool_block.h"

namespace hkv {

namespace {

// Prefill plans of up to kFewUnits blocks x KV heads: queries by workgroups of their own, kHeadsApart heads each, since there is room beside the others and a
// workgroup's chain gets shorter.  us with 1 / 2 / 4 heads / together (32 + 8 heads, bf16): 100 tokens 4.4 / 4.4 / 4.6 / 5.1, 700 6.2 / 6.2 / 6.4 / 6.9, 1500 10.2 / 9.1 / 9.3 / 9.9,
// 3000 16 / 14.6 / 15.3 / 14.4, 16000 105 / 90 / 88 / 87.
constexpr int kHeadsApart = 2, kFewUnits = 1024;

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

// What N pairs from p0 on (a multiple of N) turn by: radians per position, and the row's places on the axes (not where the caller gives none).
template <int N>
struct Angles {
    double freq[N];
    int on0, on1, on2, on3;
};
template <int N>
__device__ __forceinline__ Angles<N> load_angles(const ProjectionLaunch &a, const double *inv_freq, int p0, int64_t row) {
    Angles<N> x{};
#pragma unroll
    for (int e = 0; e < N; ++e) x.freq[e] = inv_freq[p0 + e];
    if (a.positions) {
        x.on0 = a.positions[row];
        if (a.n_axes > 1) x.on1 = a.positions[a.position_stride + row];
        if (a.n_axes > 2) x.on2 = a.positions[2 * a.position_stride + row];
        if (a.n_axes > 3) x.on3 = a.positions[3 * a.position_stride + row];
    }
    return x;
}
// Their cosines and sines; pos: the place of a row without places of its own.
template <int DT, int N>
__device__ __forceinline__ void angles(const ProjectionLaunch &a, int p0, const Angles<N> &x, int pos, float (&co)[N], float (&si)[N]) {
    const int on0 = a.positions ? x.on0 : pos;
    uint32_t axes = 0;  // (as above)
#pragma unroll
    for (int j = 0; j < 4; ++j) axes |= p0 >> 4 == j ? a.axis[j] : 0u;
    axes >>= 2 * (p0 & 15);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int place = a.n_axes == 1 ? on0 : choose(axes >> (2 * e) & 3u, on0, x.on1, x.on2, x.on3);
        const double turns = (double)place * (x.freq[e] * 0.15915494309189533577);
        const float part = (float)(turns - __builtin_rint(turns));  // (off by 2^-26 of a turn, 9.4e-8 of the radius)
        if constexpr (DT == 2) {
            sincospif(2.0f * part, &si[e], &co[e]);
        } else {  // off by 1.25e-7 at most (2^24 parts tried): bf16 results keep 8 bits, codes 4
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

// Keys and values (KV) of one KV head h of one block with up to 16 tokens, and n query heads from head q0 on (Q): thread row = slot.
template <int DT, bool KV, bool Q>
__device__ __forceinline__ void store_tokens(const ProjectionLaunch &a, const Unit &u, int h, int q0, int n) {
    __shared__ __align__(16) float sTurn[kPage][2 * 64 + 4];
    const int slot = threadIdx.x >> 4, c = threadIdx.x & 15;
    const bool valid = slot >= u.lo && slot < u.hi;
    constexpr int kAhead = 4;  // query rows on their way
    int64_t row = u.row + max(0, min(slot, u.hi - 1) - u.lo);
    if (a.row_map) row = a.row_map[row];
    // All loads at once, by all lanes and of what there is, if only a row again: a wait at the end of a branch would hold up those behind it.
    Row<DT> kr{}, vr{}, q[kAhead];
    if constexpr (KV) {
        kr = load_row<DT>(a.k, a.k_stride, row, h, c);
        vr = load_row<DT>(a.v, a.v_stride, row, h, c);
    }
    if constexpr (Q)
#pragma unroll
        for (int j = 0; j < kAhead; ++j) q[j] = load_row<DT>(a.q, a.q_stride, row, q0 + min(j, n - 1), c);
    const char *const mine = static_cast<const char *>(a.q) + row * a.q_stride * (DT == 2 ? 4 : 2);  // (for what there is none of)
    const Row<DT> qn = load_row<DT>(a.q_norm ? static_cast<const char *>(a.q_norm) + 0 : mine, 0, 0, 0, c), kn = load_row<DT>(a.k_norm ? static_cast<const char *>(a.k_norm) + 0 : mine, 0, 0, 0, c);
    const bool turns = 8 * c < a.rotary_dim;
    const int p0 = turns ? 4 * c : 0;
    const Angles<4> angle = load_angles<4>(a, a.rotary_dim > 0 ? a.inv_freq + 0 : reinterpret_cast<const double *>(mine), p0, row);
    float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    Row<DT> v{};
    if (valid) {
        v = vr;
        float qw[8], kw[8];
        values<DT>(qn, qw);
        values<DT>(kn, kw);
        // four angles a lane; the row's lanes, of one wavefront, bring theirs together
        if (turns) {
            float co[4], si[4];
            angles<DT, 4>(a, p0, angle, u.pos + slot - u.lo, co, si);
            *reinterpret_cast<float4 *>(&sTurn[slot][4 * c]) = make_float4(co[0], co[1], co[2], co[3]);
            *reinterpret_cast<float4 *>(&sTurn[slot][64 + 4 * c]) = make_float4(si[0], si[1], si[2], si[3]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        Turn t;
        turn_of(a, sTurn[slot], c, t);
        if constexpr (KV) {
            values<DT>(kr, k);
            norm_and_turn(a, c, a.k_norm != nullptr, kw, t, k);
        }
        for (int j0 = 0; Q && j0 < n; j0 += kAhead) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int i = j0 + j;
                if (i >= n) break;
                float x[8];
                values<DT>(q[j], x);
                if (i + kAhead < n) q[j] = load_row<DT>(a.q, a.q_stride, row, q0 + i + kAhead, c);
                norm_and_turn(a, c, a.q_norm != nullptr, qw, t, x);
                put_query<DT>(a, row, q0 + i, c, x);
            }
        }
    }
    if constexpr (KV) put_block<DT>(a, u, h, valid, k, v);
}

// Codes of earlier tokens (slots below lo) of an fp8 block and head under scales that have grown, by a whole wavefront; `vc`: the lanes from lane
// `at` on, sixteen, hold V's codes of the new token, which goes to slot lo with them (K's is stored apart).
__device__ __forceinline__ void round_again(const ProjectionLaunch &a, int64_t blk, int lo, int at, u32x2 vc, float ko, float ks, float vo, float vs) {
    const int lane = threadIdx.x & 63;
    if (ks > ko) {
        u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(a.pool.k_pages) + blk) + lane;  // 16 bytes of token lane / 4
        if (lane >> 2 < lo) {
            u32x4 w[2] = {p[0], p[64]};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) w[i][j] = requant4(w[i][j], ko, ks);
                p[64 * i] = w[i];
            }
        }
    }
    if (vs > vo) {
        u32x4 *p = reinterpret_cast<u32x4 *>(static_cast<uint8_t *>(a.pool.v_pages) + blk) + lane;  // dimension `lane`, all tokens
        u32x4 w[2] = {p[0], p[64]};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int from = 4 * (at + 8 * i + (lane >> 3));
            const uint32_t c0 = __builtin_amdgcn_ds_bpermute(from, vc[0]), c1 = __builtin_amdgcn_ds_bpermute(from, vc[1]);
            const uint32_t code = (lane & 4 ? c1 : c0) >> (8 * (lane & 3)) & 0xFFu;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = min(max(lo - 4 * j, 0), 4);  // earlier tokens among the word's
                const uint32_t earlier = n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1, own = lo >> 2 == j ? 0xFFu << (8 * (lo & 3)) : 0u;
                w[i][j] = (requant4(w[i][j], vo, vs) & earlier) | (code << (8 * (lo & 3)) & own) | (w[i][j] & ~(earlier | own));
            }
            p[64 * i] = w[i];
        }
    }
}

__host__ __device__ inline int token_parts(const ProjectionLaunch &a) { return (a.pool.num_kv_heads * (a.group + 1) + 15) / 16; }

// One token, row `token` of the rows: 16 of its heads' rows, from row `from` on, K's (with V's) first, then the queries'.  All threads of the workgroup call.  `place` finds the
// token's Unit, by a chain of loads that goes on beside those of the rows.
template <int DT, class Place>
__device__ __forceinline__ void store_token(const ProjectionLaunch &a, int64_t token, int from, Place &&place) {
    __shared__ __align__(16) float sTurn[2 * 64];
    const int Hkv = a.pool.num_kv_heads, Hq = Hkv * a.group, c = threadIdx.x & 15, d = 8 * c, i = from + ((int)threadIdx.x >> 4);
    const bool is_k = i < Hkv, is_q = !is_k && i - Hkv < Hq, has_angle = (int)threadIdx.x < a.rotary_dim / 2;
    const int head = is_k ? i : min(i - Hkv, Hq - 1);
    const int64_t row = a.row_map ? a.row_map[token] : token;
    // All loads at once, by all lanes and of what there is, if only the row itself again: a wait at the end of a branch would hold up those behind
    // it.  (Places, not a choice of the arguments: that would be read from memory first, by lane.)
    constexpr int E = DT == 2 ? 4 : 2;
    const char *const k_row = static_cast<const char *>(a.k) + row * a.k_stride * E, *const q_row = static_cast<const char *>(a.q) + row * a.q_stride * E;
    const char *const mine = (is_k ? k_row : q_row) + (head * kHeadDim + d) * E;
    const char *const k_norm = a.k_norm ? static_cast<const char *>(a.k_norm) + 0 : k_row, *const q_norm = a.q_norm ? static_cast<const char *>(a.q_norm) + 0 : q_row;
    const bool normed = is_k ? k_norm != k_row : q_norm != q_row;
    const Row<DT> r = load_row<DT>(mine, 0, 0, 0, 0), wr = load_row<DT>(is_k ? k_norm : q_norm, 0, 0, 0, c);
    Row<DT> v{};
    if (from < Hkv) v = load_row<DT>(a.v, a.v_stride, row, min(head, Hkv - 1), c);
    const Angles<1> angle = load_angles<1>(a, a.rotary_dim > 0 ? a.inv_freq : reinterpret_cast<const double *>(k_row), max(0, min((int)threadIdx.x, a.rotary_dim / 2 - 1)), row);
    const Unit u = place();
    const int64_t at = (int64_t)u.block * Hkv + head;
    float old[2] = {0.f, 0.f}, w[8], x[8];
    if (DT == 1 && from < Hkv && u.lo > 0) {
        const int64_t s = (int64_t)u.block * Hkv + min(head, Hkv - 1);
        old[0] = a.pool.k_scale[s];
        old[1] = a.pool.v_scale[s];
    }
    if (has_angle) {  // an angle a lane, for all heads
        float co[1], si[1];
        angles<DT, 1>(a, threadIdx.x, angle, u.pos, co, si);
        sTurn[threadIdx.x] = co[0];
        sTurn[64 + threadIdx.x] = si[0];
    }
    __syncthreads();
    if (is_k || is_q) {
        Turn t;
        turn_of(a, sTurn, c, t);
        values<DT>(r, x);
        values<DT>(wr, w);
        norm_and_turn(a, c, normed, w, t, x);
    }
    if (is_q) put_query<DT>(a, row, head, c, x);
    const int64_t blk = at * kBlockElems;
    if constexpr (DT == 0) {
        if (!is_k) return;
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.pool.k_pages) + blk + (d >> 5) * 512 + u.lo * 32 + (d & 31)) = pack8(x);
        uint16_t *vd = static_cast<uint16_t *>(a.pool.v_pages) + blk + d * kPage + u.lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) vd[j * kPage] = (uint16_t)(v.w[0][j >> 1] >> (16 * (j & 1)));
    } else if constexpr (DT == 1) {
        // the block's running scales, as store_block finds them
        float vf[8], sc[2] = {0.f, 0.f};
        u32x2 vc = {0u, 0u};
        bool grown = false;
        if (is_k) {
            float am[2] = {0.f, 0.f};
            unpack_bf16(v.w[0], vf);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                am[0] = fmaxf(am[0], fabsf(x[j]));
                am[1] = fmaxf(am[1], fabsf(vf[j]));
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const float m = row16_max(am[s]);
                const float cand = m > 0.f ? m / 448.0f : 0.f;
                sc[s] = u.lo > 0 && old[s] >= cand ? old[s] : cand;  // an unset (NaN) old scale gives cand
                if (!(sc[s] > 0.f)) sc[s] = 1.0f;
            }
            if (c == 0) {
                a.pool.k_scale[at] = sc[0];
                a.pool.v_scale[at] = sc[1];
            }
            *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.pool.k_pages) + blk + (d >> 6) * 1024 + u.lo * 64 + (d & 63)) =
                u32x2{quant4(x[0], x[1], x[2], x[3], sc[0]), quant4(x[4], x[5], x[6], x[7], sc[0])};
            vc = u32x2{quant4(vf[0], vf[1], vf[2], vf[3], sc[1]), quant4(vf[4], vf[5], vf[6], vf[7], sc[1])};
            if (!(u.lo > 0 && sc[1] > old[1])) {
                uint8_t *vd = static_cast<uint8_t *>(a.pool.v_pages) + blk + d * kPage + u.lo;
#pragma unroll
                for (int j = 0; j < 8; ++j) vd[j * kPage] = (uint8_t)(vc[j >> 2] >> (8 * (j & 3)));
            }
            grown = u.lo > 0 && (sc[0] > old[0] || sc[1] > old[1]);
        }
        // rounding again takes the whole wavefront, a head at a time
        for (uint64_t rest = __ballot(c == 0 && grown); rest; rest &= rest - 1) {
            const int l = __builtin_ctzll(rest);
            auto of = [&](float f) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), l)); };
            round_again(a, ((int64_t)u.block * Hkv + __builtin_amdgcn_readlane(head, l)) * kBlockElems, u.lo, l, vc, of(old[0]), of(sc[0]), of(old[1]), of(sc[1]));
        }
    } else {
        if (!is_k) return;
        float *kd = static_cast<float *>(a.pool.k_pages) + blk + (d >> 4) * 256 + u.lo * 16 + (d & 15);
        float *vd = static_cast<float *>(a.pool.v_pages) + blk + d * kPage + u.lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            kd[j] = x[j];
            vd[j * kPage] = __uint_as_float(v.w[j >> 2][j & 3]);
        }
    }
}

// The newest tokens of a decode plan's requests.  By tokens: a workgroup takes 16 rows of heads of one token.  By blocks: a block that the tokens of
// a request can span, and a KV head with its queries.  Both: keys and values by blocks (an fp8 block's scale is of all its new tokens), the queries by tokens.
enum class By { kTokens, kBlocks, kBoth };
__host__ __device__ inline int spans(const ProjectionLaunch &a) { return (a.tokens + kPage - 2) / kPage + 1; }
template <int DT, By BY>
__global__ __launch_bounds__(256) void projection_decode_kernel(ProjectionLaunch a) {
    const int Hkv = a.pool.num_kv_heads, n_blocks = a.n_requests * spans(a) * Hkv;  // (kBoth: workgroups that go by blocks, first)
    // position of the first of the request's newest tokens in its last node
    auto newest = [&](const StoreRequest &s) {
        int n = s.tokens;
        if (s.item >= 0) n = a.items[s.item].tok_begin + a.items[s.item].n_tokens;
        return n - a.tokens;
    };
    if (BY == By::kTokens || (BY == By::kBoth && (int)blockIdx.x >= n_blocks)) {
        const int from = BY == By::kBoth ? Hkv : 0, parts = (Hkv * (a.group + 1) - from + 15) / 16, i = blockIdx.x - (BY == By::kBoth ? n_blocks : 0);
        const int x = i / parts, part = i % parts;
        store_token<DT>(a, x, from + 16 * part, [&] {
            const int r = x / a.tokens;
            const StoreRequest s = a.requests[r];
            const int t = newest(s) + (x - r * a.tokens);
            return Unit{a.blocks[s.page_off + (uint32_t)(t / kPage)], t % kPage, t % kPage + 1, x, s.pos0 + t};
        });
    } else {
        const int unit = blockIdx.x / Hkv, h = blockIdx.x % Hkv, r = unit / spans(a), part = unit % spans(a);
        const StoreRequest s = a.requests[r];
        const int first = newest(s), b = first / kPage + part, lo = max(first - b * kPage, 0);
        if (b * kPage >= first + a.tokens) return;
        const Unit u{a.blocks[s.page_off + (uint32_t)b], lo, min(first + a.tokens - b * kPage, kPage), (int64_t)r * a.tokens + (b * kPage + lo - first), s.pos0 + b * kPage + lo};
        store_tokens<DT, true, BY != By::kBoth>(a, u, h, h * a.group, a.group);
    }
}

// The new tokens of a prefill plan's requests.  grid: (blocks they go to, KV heads), or queries APART: (blocks, KV heads and then kHeadsApart query heads each)
template <int DT, bool APART>
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
    const int h = blockIdx.y, Hkv = p.base.pool.num_kv_heads, q0 = (h - Hkv) * kHeadsApart;
    if constexpr (!APART)
        store_tokens<DT, true, true>(p.base, u, h, h * p.base.group, p.base.group);
    else if (h < Hkv)
        store_tokens<DT, true, false>(p.base, u, h, 0, 0);
    else
        store_tokens<DT, false, true>(p.base, u, 0, q0, min(kHeadsApart, Hkv * p.base.group - q0));
}

// A growing plan's step: a request's new token, and the items of its leaf get longer.  (The leaf's length comes by value: other workgroups may have
// lengthened its items already.)
template <int DT>
__global__ __launch_bounds__(256) void projection_append_kernel(ProjectionAppend p, PlanGrowInline g) {
    const ProjectionLaunch &a = p.base;
    const int parts = token_parts(a), r = blockIdx.x / parts, part = blockIdx.x % parts, Hkv = a.pool.num_kv_heads;
    const int n = p.length[r], fresh = g.new_block[r];
    store_token<DT>(a, r, 16 * part, [&] {
        const StoreRequest s = a.requests[r];
        return Unit{fresh >= 0 ? fresh : a.blocks[s.page_off + (uint32_t)(n / kPage)], n % kPage, n % kPage + 1, r, s.pos0 + n};
    });
    const int h = 16 * part + (int)threadIdx.x;
    if (threadIdx.x < 16 && h < Hkv) g.items[g.grow_items[r * Hkv + h]].n_tokens += 1;
    if (threadIdx.x == 16 && part == 0 && fresh >= 0) g.pages[g.block_pos[r]] = fresh;
}

}  // namespace

hipError_t launch_projection_store(const ProjectionLaunch &a, hipStream_t s) {
    if (a.n_requests <= 0) return hipSuccess;
    // us, 32 + 8 heads, by tokens / blocks / both.  bf16, 64 requests of 2 new tokens: 4.4 / 6.1 / 4.4, of 4: 5.9 / 6.9 / 4.8, 8: 8.5 / 7.8 / 6.0, 16: 12.6 / 9.1 / 8.3, 32: 20 / 11.7 / 11.5,
    // 64: 42 / 21.4 / 22.3; 300 requests of 2: 9.7 / 19.2 / 13.1, of 4: 16.0 / 20.3 / 15.5.  fp8, 64 requests of 2: - / 8.1 / 6.5, of 16: - / 10.0 / 9.1, of 64: - / 20.9 / 22.9.
    const By by = a.tokens == 1 || (a.tokens == 2 && a.pool.dtype != 1) ? By::kTokens : a.tokens <= 24 ? By::kBoth : By::kBlocks;
    const int heads = a.pool.num_kv_heads, blocks = a.n_requests * spans(a) * heads, tokens = a.n_requests * a.tokens;
    const dim3 grid(by == By::kTokens ? tokens * token_parts(a) : by == By::kBlocks ? blocks : blocks + tokens * ((heads * a.group + 15) / 16)), block(256);
    auto go = [&](auto tokens, auto blocks, auto both) { hipLaunchKernelGGL(by == By::kTokens ? tokens : by == By::kBlocks ? blocks : both, grid, block, 0, s, a); };
    if (a.pool.dtype == 0)
        go(projection_decode_kernel<0, By::kTokens>, projection_decode_kernel<0, By::kBlocks>, projection_decode_kernel<0, By::kBoth>);
    else if (a.pool.dtype == 1)
        go(projection_decode_kernel<1, By::kTokens>, projection_decode_kernel<1, By::kBlocks>, projection_decode_kernel<1, By::kBoth>);
    else  // (no more than 16 query tokens, so never by blocks alone)
        go(projection_decode_kernel<2, By::kTokens>, projection_decode_kernel<2, By::kBoth>, projection_decode_kernel<2, By::kBoth>);
    return hipGetLastError();
}

hipError_t launch_projection_store(const ProjectionPrefill &a, hipStream_t s) {
    if (a.n_units <= 0) return hipSuccess;
    const int Hkv = a.base.pool.num_kv_heads;
    const bool apart = (int64_t)a.n_units * Hkv <= kFewUnits;
    const dim3 grid(a.n_units, apart ? Hkv + (Hkv * a.base.group + kHeadsApart - 1) / kHeadsApart : Hkv), block(256);
    auto go = [&](auto together, auto apart_) { hipLaunchKernelGGL(apart ? apart_ : together, grid, block, 0, s, a); };
    if (a.base.pool.dtype == 0)
        go(projection_prefill_kernel<0, false>, projection_prefill_kernel<0, true>);
    else if (a.base.pool.dtype == 1)
        go(projection_prefill_kernel<1, false>, projection_prefill_kernel<1, true>);
    else
        go(projection_prefill_kernel<2, false>, projection_prefill_kernel<2, true>);
    return hipGetLastError();
}

hipError_t launch_projection_append(const ProjectionAppend &a, const PlanGrowInline &g, hipStream_t s) {
    if (a.base.n_requests <= 0) return hipSuccess;
    const dim3 grid((unsigned)(a.base.n_requests * token_parts(a.base))), block(256);
    if (a.base.pool.dtype == 0)
        hipLaunchKernelGGL(projection_append_kernel<0>, grid, block, 0, s, a, g);
    else
        hipLaunchKernelGGL(projection_append_kernel<1>, grid, block, 0, s, a, g);
    return hipGetLastError();
}

}  // namespace hkv
