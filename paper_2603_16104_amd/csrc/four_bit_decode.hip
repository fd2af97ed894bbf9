// Decode attention over 4-bit pools: one workgroup per item (a chunk of a prefix-tree node, one KV head, up to 128 query rows), partial results to
// the log-sum-exp merge.  (Section 5, "Proactive Cache Management": a node's pages are read once for all requests below it.)
//
// A wavefront takes 64 tokens (four blocks) a step, for one or two tiles of 16 query rows, or for 32 rows (run_tall has its layout):
//   S^T = K Q^T   v_mfma_scale_f32_16x16x128_f8f6f4: K's codes and scales as they lie in the pool, lane (m, g) dims 32 g .. + 31 of token 4 m + t4 in
//                 tile t4 (its four scales are one word); a query row as four e2m3 terms (split_row), whose powers of two are the other scale.  Against bf16
//                 operands widened from the codes that is the same matrix time and 68 fewer vector instructions a step.
//   O^T = V^T P^T v_mfma_f32_16x16x32_bf16: lane (m, g) brings dim 8 m + dt of eight tokens of block g.  A scale stands for one token and 32 dims, the
//                 instruction's for 32 tokens of a dim, so V is widened: two codes (neighbouring dims of a token) an instruction, then one more to
//                 bring two tokens of a dim together, 152 of a step's some 260 vector instructions; rows of more than one tile share that.
// A lane of a score tile t4 holds tokens 16 g + 4 i + t4 of its query row m: over the four tiles all 16 tokens of block g, which is what its
// share of P^T is made of, so probabilities stay where they are.  Widened values are exact (two significant bits, a power of two).
//
// What bounds it: items of few rows memory (512 sequences of 1024 to 2048 tokens, 8 KV heads: 143 us, 6.0 TB/s), items of many rows their
// instructions (16 x 8192 tokens under 256 rows of 8 KV heads: 136 us; matrix cores 53 % busy, vector units 47 %); both together, 512 requests on a
// 70B-shaped layer, 260 us at the 1.9 GHz that the card keeps under them.  Small steps wait for their loads: item, page ids and rows, queries, codes.
#include <hip/hip_ext.h>

#include <climits>
#include <type_traits>
#include <utility>

#include "four_bit.h"

namespace hkv {

namespace {

constexpr int kWaves = 4, kStep = 64;  // wavefronts; tokens of a step
constexpr int kORow = kHeadDim + 4;    // padded LDS row

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(6))) uint32_t u32x6;  // 32 e2m3 codes
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(32))) float f32x32;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
constexpr int kTerms = 4;  // of a query row
// The instruction's operands for its 6-bit and 4-bit types: the six and four registers in front count.
__device__ __forceinline__ i32x8 as_six(u32x6 q) { return i32x8{(int)q[0], (int)q[1], (int)q[2], (int)q[3], (int)q[4], (int)q[5], 0, 0}; }
__device__ __forceinline__ i32x8 as_four(u32x4 k) { return i32x8{(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0}; }
// 16 tokens (e2m1, scale byte T of k_scale) x 128 dims by 128 dims x 16 rows (e2m3, scale byte Term of q_scale).  Lane (m, g): dims 32 g .. + 31 of either.
template <int T, int Term>
__device__ __forceinline__ f32x4 mfma_four(u32x4 k, const u32x6 (&q)[kTerms], f32x4 c, uint32_t k_scale, uint32_t q_scale) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(as_four(k), as_six(q[Term]), c, 4, 2, T, k_scale, Term, q_scale);
}
// f(0), f(1), .. f(N - 1), each with its number as a constant.
template <class F, int... I>
__device__ __forceinline__ void in_turn(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void in_turn(F &&f) {
    in_turn(f, std::make_integer_sequence<int, N>{});
}

__device__ __forceinline__ int pick4(const int (&v)[4], int sel) {
    const int v0 = v[0], v1 = v[1], v2 = v[2], v3 = v[3];
    const int lo = (sel & 1) ? v1 : v0, hi = (sel & 1) ? v3 : v2;
    return (sel & 2) ? hi : lo;
}

// A step's operands of one lane as they lie in the pool.
struct Operands {
    u32x4 k[4], v[4], v_scale;
    uint32_t k_scale;
};

// What a tile of 16 query rows has: lane (m, g) row m.
struct RowTile {
    u32x6 q[kTerms];    // dims 32 g .. + 31 of the query row
    uint32_t q_scale;   // the terms' scale bytes
    f32x4 o[8];         // o[dt][i]: dim 32 g + 8 i + dt
    float m, l;         // reference (raw scores), this lane's share of the row sum
    int req;            // the plan's row of it
    int lim;            // tokens of the item that the row may see (and of those behind them the ones in row_mask)
};

// 32 dims of a query row as four e2m3 terms (three bits behind the point, at most 7.5, multiples of 1/8): the largest magnitude is brought into [4, 8) by a power of two, and
// each term is what those in front leave, under scales 2^4, 2^10 and 2^15 below the first one's.  bf16 values down to 2^-12 of the largest of the 32 are exact, of smaller ones
// 2^-20 of that is lost (2^-129 where that is more).  Products of e2m1 and e2m3 are added without loss inside the matrix instruction, and its sums are those of fp32; of products with e4m3 or e5m2 (two terms
// in the same matrix time) it cuts off what lies below 2^-13 of the largest among eight neighbouring dims: lse off by 1e-3 for rows with an outlier.
// A row that holds a NaN or an infinity gets a scale that is no number.  sign: -1 for a negative softmax scale.
__device__ __forceinline__ void split_row(u32x4 (&w)[4], float sign, u32x6 (&q)[kTerms], uint32_t &q_scale) {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    const uint32_t flip = sign < 0.f ? 0x80008000u : 0u;
    u16x2 tops = {0, 0};
    f32x16 even, odd;  // (the conversion takes the dims in this order)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t word = w[i >> 2][i & 3] ^ flip;
        tops = __builtin_elementwise_max(tops, __builtin_bit_cast(u16x2, word & 0x7FFF7FFFu));
        even[i] = __uint_as_float(word << 16);
        odd[i] = __uint_as_float(word & 0xFFFF0000u);
    }
    const int ex = max(tops[0], tops[1]) >> 7, first = min(max(ex - 2, 16), 252);  // (the last term's scale is a normal number, too)
    constexpr int kBelow[kTerms] = {0, 4, 10, 15};
    q_scale = 0;
#pragma unroll
    for (int t = 0; t < kTerms; ++t) {
        const float scale = __uint_as_float((uint32_t)(first - kBelow[t]) << 23);
        q_scale |= (uint32_t)(first - kBelow[t]) << (8 * t);
        q[t] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
        if (t + 1 == kTerms) break;
        const f32x32 term = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q[t], scale);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            even[i] -= term[2 * i];
            odd[i] -= term[2 * i + 1];
        }
    }
    if (ex == 255) q_scale = 0xFFFFFFFFu;
}

// A wavefront's lane, item and pool: where its operands lie.
struct Reader {
    const DecodeLaunch &a;
    const DecodeItem &it;
    const uint8_t *k, *v, *k_scale, *v_scale;  // with the lane's offsets inside a block
    int lane, m, g, last_page;
    __device__ __forceinline__ Reader(const DecodeLaunch &a, const DecodeItem &it) : a(a), it(it) {
        lane = (int)threadIdx.x & 63;
        m = lane & 15;
        g = lane >> 4;
        last_page = (it.n_tokens - 1) >> 4;
        k = static_cast<const uint8_t *>(a.pool.k_pages) + (m & 3) * 64 + g * 16;
        v = static_cast<const uint8_t *>(a.pool.v_pages) + m * 16;
        k_scale = reinterpret_cast<const uint8_t *>(a.pool.k_scale) + g * 16 + 4 * (m & 3);
        v_scale = reinterpret_cast<const uint8_t *>(a.pool.v_scale) + (m >> 2) * 16;
    }
    // page ids of a step, wavefront-uniform (scalar loads); clamped, so always in bounds
    __device__ __forceinline__ void ids(int (&id)[4], int b) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) id[i] = a.pages[it.page_off + min(4 * b + i, last_page)];
    }
    __device__ __forceinline__ size_t block(const int (&id)[4], int sel) const { return (size_t)pick4(id, sel) * a.pool.num_kv_heads + it.kv_head; }
    __device__ __forceinline__ void keys(Operands &x, const int (&id)[4]) const {
        const size_t blk = block(id, m >> 2);
        x.k_scale = *reinterpret_cast<const uint32_t *>(k_scale + blk * four::kScaleBytes);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.k[j] = ld16_stream(k + blk * four::kCodeBytes + 256 * j);
    }
    __device__ __forceinline__ void values(Operands &x, const int (&id)[4]) const {
        const size_t blk = block(id, g);
        x.v_scale = ld16(v_scale + blk * four::kScaleBytes);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[j] = ld16_stream(v + blk * four::kCodeBytes + 256 * j);
    }
};

// The partial that a row of the item writes.
__device__ __forceinline__ size_t part_of(const DecodeLaunch &a, const DecodeItem &it, int req, int row) {
    const int G = a.num_q_heads / a.pool.num_kv_heads;
    return (size_t)((req * a.num_q_heads + it.kv_head * G + row % G) * a.max_parts + it.part_slot);
}

// The rows' place in the plan, asked for in front of everything else: the queries' loads wait for it.
template <int RT>
__device__ __forceinline__ void find_rows(const Reader &rd, int row0, RowTile (&tile)[RT]) {
    const int G = rd.a.num_q_heads / rd.a.pool.num_kv_heads, rows = rd.it.n_req * G;
#pragma unroll
    for (int r = 0; r < RT; ++r) tile[r].req = rd.a.node_req_idx[rd.it.req_off + min(row0 + 16 * r + rd.m, rows - 1) / G];
}
// The queries, dims 32 g .. + 31 a lane.
template <int RT>
__device__ __forceinline__ void load_rows(const Reader &rd, int row0, RowTile (&tile)[RT], u32x4 (&w)[RT][4]) {
    const DecodeLaunch &a = rd.a;
    const DecodeItem &it = rd.it;
    const int G = a.num_q_heads / a.pool.num_kv_heads, rows = it.n_req * G;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int head = it.kv_head * G + min(row0 + 16 * r + rd.m, rows - 1) % G, req = tile[r].req;
        const int q_row = a.q_rows ? a.q_rows[req] : req;
        const char *qp = static_cast<const char *>(a.q) + ((size_t)q_row * a.num_q_heads + head) * (kHeadDim * 2) + 64 * rd.g;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[r][i] = ld16(qp + 16 * i);
    }
}
template <int RT>
__device__ __forceinline__ void begin_rows(const Reader &rd, RowTile (&tile)[RT], u32x4 (&w)[RT][4]) {
    const DecodeLaunch &a = rd.a;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int req = tile[r].req;
        tile[r].lim = a.row_leaf && a.row_leaf[req] == rd.it.node ? a.row_limit[req] - rd.it.tok_begin : rd.it.n_tokens;
        split_row(w[r], a.scale, tile[r].q, tile[r].q_scale);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) tile[r].o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        tile[r].m = -INFINITY;
        tile[r].l = 0.f;
    }
}

// S^T of a step.
template <int RT>
__device__ __forceinline__ void scores(const Operands &x, const RowTile (&tile)[RT], f32x4 (&acc)[RT][4]) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const RowTile &t = tile[r];
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4) acc[r][t4] = f32x4{0.f, 0.f, 0.f, 0.f};
        in_turn<4 * kTerms>([&](auto n) {
            constexpr int T = decltype(n)::value & 3, Term = decltype(n)::value >> 2;
            acc[r][T] = mfma_four<T, Term>(x.k[T], t.q, acc[r][T], x.k_scale, t.q_scale);
        });
    }
}

// Of 16 tokens those that a row sees: all in front of its limit (the first one is d0 behind that), and behind it the ones in vis.
__device__ __forceinline__ uint32_t seen_bits(int d0, unsigned long long vis) {
    return d0 < 0 ? (d0 <= -16 ? 0xFFFFu : (1u << -d0) - 1u | (uint32_t)vis << -d0) : d0 < 64 ? (uint32_t)(vis >> d0) : 0u;
}
// Scores of tokens that a row does not see are -inf, and those of tokens behind the item's end (a chunk may end inside a step, and its rows see what follows in the
// next one); of the lane's 16 tokens score j of a row is acc[j % 4][j / 4].
template <int RT>
__device__ __forceinline__ bool hide(const Reader &rd, const RowTile (&tile)[RT], f32x4 (&acc)[RT][4], int b) {
    const int tok0 = b * kStep + 16 * rd.g;
    int most = -INT_MAX;  // tokens of the step behind what a row sees at once
#pragma unroll
    for (int r = 0; r < RT; ++r) most = max(most, tok0 - min(tile[r].lim, rd.it.n_tokens));
    const bool some = __builtin_amdgcn_ballot_w64(most > -16);  // some row does not see the whole step, the item's last one among them
    if (some) {
        const uint32_t in_item = 0xFFFFu >> min(max(tok0 + 16 - rd.it.n_tokens, 0), 16);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const bool last = rd.a.row_leaf && rd.a.row_leaf[tile[r].req] == rd.it.node;  // (looked up here: this is the exception)
            const unsigned long long vis = last ? rd.a.row_mask[tile[r].req] : 0ull;
            const int d0 = tok0 - tile[r].lim;
            const uint32_t seen = seen_bits(d0, vis) & in_item;
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[r][j & 3][j >> 2] = (seen >> j & 1u) ? acc[r][j & 3][j >> 2] : -INFINITY;
        }
    }
    return some;
}
// A row's reference, of which its weights are powers: it stays until they would be large.  One that is the largest score of every step so far moves for some
// row of 32 nearly always, 66 instructions of a step's 450.
__device__ __forceinline__ void follow(RowTile &t, float top, float c) {
    const float m_new = fmaxf(t.m, rows_max(top));
    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((t.m - m_new) * c);
    t.m = m_new;
    t.l *= alpha;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) t.o[dt] *= alpha;
}
// Where the scores are at hand until all weights are made, those tell: a lane's of a step sum up to more than kMostWeight (8 instructions a row tile fewer than
// the largest score).  Elsewhere a score beyond the reference by a weight of 2^kSlack does.
constexpr float kMostWeight = 16384.f, kSlack = 8.f;
// Probabilities, rounded to bf16, half a step of 2^-8 each, as over the other pools.
template <int RT>
__device__ __forceinline__ void weigh(const RowTile (&tile)[RT], const f32x4 (&acc)[RT][4], float c, u32x4 (&pw)[RT][2], float (&sum)[RT]) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float mc = tile[r].m == -INFINITY ? 0.f : tile[r].m * c;  // (a row that has seen nothing: no inf - inf)
        float p[16];
        sum[r] = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            p[j] = fast_exp2(__builtin_fmaf(acc[r][j & 3][j >> 2], c, -mc));
            sum[r] += p[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) pw[r][j >> 2][j & 3] = pack_bf16(p[2 * j], p[2 * j + 1]);
    }
}
template <int RT>
__device__ __forceinline__ void follow_all(RowTile (&tile)[RT], const f32x4 (&acc)[RT][4], float c) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float top = acc[r][0][0];
#pragma unroll
        for (int j = 1; j < 16; ++j) top = fmaxf(top, acc[r][j & 3][j >> 2]);
        follow(tile[r], top, c);
    }
}
template <int RT>
__device__ __forceinline__ void weights(RowTile (&tile)[RT], const f32x4 (&acc)[RT][4], float c, u32x4 (&pw)[RT][2]) {
    float sum[RT];
    weigh(tile, acc, c, pw, sum);
    bool any = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) any = any || !(sum[r] <= kMostWeight) || tile[r].m == -INFINITY;  // (a NaN, too)
    if (__builtin_amdgcn_ballot_w64(any)) {
        follow_all(tile, acc, c);
        weigh(tile, acc, c, pw, sum);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) tile[r].l += sum[r];
}

// Two dims (8 m + 2 B, + 1) of tokens 0 .. 3 from their words and scales: lo, hi [tokens 0 1 | 2 3].
template <int B>
__device__ __forceinline__ void widen_pairs(const uint32_t (&w)[4], const float (&sc)[4], u32x2 &lo, u32x2 &hi) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t v0 = four::widen2<B>(w[2 * j], sc[2 * j]), v1 = four::widen2<B>(w[2 * j + 1], sc[2 * j + 1]);
        lo[j] = __builtin_amdgcn_perm(v1, v0, 0x05040100u);
        hi[j] = __builtin_amdgcn_perm(v1, v0, 0x07060302u);
    }
}

// Slots of four tokens from first_bad (of them) on may hold anything: no codes, a scale of 1.
__device__ __forceinline__ void clear_from(u32x4 &w, uint32_t &scale, int first_bad) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j >= first_bad) {
            w[j] = 0u;
            scale = (scale & ~(0xFFu << (8 * j))) | (127u << (8 * j));
        }
}

// O^T += V^T P^T of a step, V from the lane's own registers.
template <int RT>
__device__ __forceinline__ void add_values(RowTile (&tile)[RT], const Operands &x, const u32x4 (&pw)[RT][2]) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // eight tokens of every block
        float sc[2][4];
        uint32_t w[2][4];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sc[q][j] = four::scale_of(x.v_scale[2 * half + q], j);
                w[q][j] = x.v[2 * half + q][j];
            }
        auto dims = [&](auto byte) {
            constexpr int B = decltype(byte)::value;
            u32x2 lo[2], hi[2];
            widen_pairs<B>(w[0], sc[0], lo[0], hi[0]);
            widen_pairs<B>(w[1], sc[1], lo[1], hi[1]);
            const bf16x8 va = as_bf16x8(u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]}), vb = as_bf16x8(u32x4{hi[0][0], hi[0][1], hi[1][0], hi[1][1]});
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                tile[r].o[2 * B] = mfma16(va, as_bf16x8(pw[r][half]), tile[r].o[2 * B]);
                tile[r].o[2 * B + 1] = mfma16(vb, as_bf16x8(pw[r][half]), tile[r].o[2 * B + 1]);
            }
        };
        dims(std::integral_constant<int, 0>{});
        dims(std::integral_constant<int, 1>{});
        dims(std::integral_constant<int, 2>{});
        dims(std::integral_constant<int, 3>{});
    }
}

// Rows whose tokens a wavefront has seen all go out from its registers, 32 dims a lane.
template <int RT>
__device__ __forceinline__ void write_rows(const Reader &rd, int row0, float c, RowTile (&tile)[RT]) {
    const int rows = rd.it.n_req * (rd.a.num_q_heads / rd.a.pool.num_kv_heads);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        RowTile &t = tile[r];
        const float l_row = rows_sum(t.l), inv = l_row > 0.f ? 1.0f / l_row : 0.f;
        float top = 0.f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            t.o[dt] *= inv;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(t.o[dt][i]));
        }
        top = rows_max(top);
        float up, down;
        part_factors(top, up, down);
        if (row0 + 16 * r + rd.m >= rows) continue;
        const size_t part = part_of(rd.a, rd.it, t.req, row0 + 16 * r + rd.m);
        uint16_t *out = rd.a.o_parts + part * kHeadDim + 32 * rd.g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x4 w;
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = pack_f16(t.o[2 * q][i] * up, t.o[2 * q + 1][i] * up);
            *reinterpret_cast<u32x4 *>(out + 8 * i) = w;
        }
        if (rd.g == 0) {
            rd.a.down_parts[part] = down;
            rd.a.lse_parts[part] = partial_lse(l_row == l_row ? t.m * c : INFINITY, l_row);
        }
    }
}

// Of a scale of 0 the smallest number: a weight of 1 for every score, and -inf stays.
__device__ __forceinline__ float exponent_factor(float scale) {
    const float c = fabsf(scale) * kLog2e;
    return c == 0.f ? 0x1p-149f : c;
}

// What a wavefront does with a share of an item's steps, ts, ts + n_ts, ..: the operands of two steps travel while another is computed, page ids a step
// further ahead (behind the last steps once more, clamped to its last page: a condition would keep two sets of registers apart).
template <int RT>
__device__ __forceinline__ void stream(const Reader &rd, int row0, int ts, int n_ts, float c, RowTile (&tile)[RT]) {
    const int n_blk = (rd.it.n_tokens + kStep - 1) / kStep;
    int id[4], b = ts;
    find_rows(rd, row0, tile);
    rd.ids(id, b);
    Operands x;
    u32x4 w[RT][4];
    rd.keys(x, id);
    __builtin_amdgcn_sched_barrier(0);
    load_rows(rd, row0, tile, w);
    __builtin_amdgcn_sched_barrier(0);
    rd.values(x, id);
    rd.ids(id, b + n_ts);
    auto second_half = [&](Operands &v, const u32x4 (&pw)[RT][2]) {
        if ((b + 1) * kStep > rd.it.n_tokens) {
            const int first_bad = rd.it.n_tokens - (b * kStep + 16 * rd.g);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t sc = v.v_scale[q];
                clear_from(v.v[q], sc, first_bad - 4 * q);
                v.v_scale[q] = sc;
            }
        }
        add_values(tile, v, pw);
    };
    f32x4 acc[RT][4];
    u32x4 pw[RT][2];
    if constexpr (RT == 1) {
        Operands y, z;
        rd.keys(y, id);
        rd.values(y, id);
        rd.ids(id, b + 2 * n_ts);
        __builtin_amdgcn_sched_barrier(0);
        begin_rows(rd, tile, w);
        auto step = [&](Operands &now, Operands &after_next) {
            rd.keys(after_next, id);
            rd.values(after_next, id);
            rd.ids(id, b + 3 * n_ts);
            __builtin_amdgcn_sched_barrier(0);
            scores(now, tile, acc);
            hide(rd, tile, acc, b);
            weights(tile, acc, c, pw);
            second_half(now, pw);
            return (b += n_ts) < n_blk;
        };
        while (step(x, z) && step(y, x) && step(z, y)) {
        }
    } else {  // two tiles fill the registers: K of the next step is requested behind the first product, V behind the second
        begin_rows(rd, tile, w);
        for (; b < n_blk; b += n_ts) {
            scores(x, tile, acc);
            __builtin_amdgcn_sched_barrier(0);
            rd.keys(x, id);
            __builtin_amdgcn_sched_barrier(0);
            hide(rd, tile, acc, b);
            weights(tile, acc, c, pw);
            second_half(x, pw);
            __builtin_amdgcn_sched_barrier(0);
            rd.values(x, id);
            rd.ids(id, b + 2 * n_ts);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// LDS of a workgroup: partial results of wavefronts that share a row tile's tokens, or a ring of steps and two steps' V in bf16 as the second
// product's operands.
template <int W>
struct Shares {
    float o[W][16][kORow], m[W][16], l[W][16];
    int row[16];
};
static_assert(sizeof(Shares<4>) >= 3 * 64 * 4 * sizeof(u32x4), "two terms of the rows, in whole paths");
constexpr int kRing = 4;
struct Stage {  // four blocks as they lie in the pool, 16 bytes in the order of the lanes that brought them
    u32x4 k[4][64], v[4][64];
    uint32_t scale[4][64];  // K's 16 words, V's 16, and both again
};
struct Widened {
    Stage ring[kRing];
    u32x4 v[2][16][64];  // [step % 2], a matrix instruction's operand each
};
union Lds {
    Shares<kWaves> s;
    Widened w;
};

// A wavefront's share of a row tile into LDS (active: it has seen tokens).
template <int W>
__device__ __forceinline__ void leave_share(Shares<W> &s, const RowTile &t, int wave, int m, int g, bool active) {
    if (!active) {
        if (g == 0) s.m[wave][m] = -INFINITY;
        return;
    }
    const float l_row = rows_sum(t.l);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            *reinterpret_cast<f32x4 *>(&s.o[wave][m][32 * g + 8 * i + 4 * q]) = f32x4{t.o[4 * q][i], t.o[4 * q + 1][i], t.o[4 * q + 2][i], t.o[4 * q + 3][i]};
    if (g == 0) {
        s.m[wave][m] = l_row == l_row ? t.m : INFINITY;  // (a NaN or +inf among the scores: the row's sum is no number below)
        s.l[wave][m] = l_row;
    }
}
// The shares of a row brought together: eight dims, the reference and the sum.
template <int W>
__device__ __forceinline__ void join_shares(const Shares<W> &s, int row, int col, float c, f32x4 &x, f32x4 &y, float &M, float &L) {
    M = -INFINITY;
    L = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, s.m[w][row]);
    x = y = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const float mw = s.m[w][row];
        if (mw == -INFINITY) continue;  // that wavefront's tokens were all invisible to the row
        const float wgt = fast_exp2((mw - M) * c);
        L += s.l[w][row] * wgt;
        x += *reinterpret_cast<const f32x4 *>(&s.o[w][row][8 * col]) * wgt;
        y += *reinterpret_cast<const f32x4 *>(&s.o[w][row][8 * col + 4]) * wgt;
    }
    const float inv = L > 0.f ? 1.0f / L : 0.f;
    x *= inv;
    y *= inv;
}

// Items of up to 16 RT rows: the four wavefronts share the tokens, and bring their results together in LDS, a row tile at a time; then thread
// (row = tid / 16, tid % 16) has eight dims of a row, whose 16 threads are a row of lanes.
template <int RT>
__device__ __forceinline__ void run_shared_tokens(const DecodeLaunch &a, const DecodeItem &it, Shares<kWaves> &s) {
    const Reader rd(a, it);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), rows = it.n_req * (a.num_q_heads / a.pool.num_kv_heads);
    const float c = exponent_factor(a.scale);
    const bool active = wave * kStep < it.n_tokens;
    RowTile tile[RT];
    if (active) stream(rd, 0, wave, kWaves, c, tile);
    const int col = rd.lane & 15, out_row = (int)threadIdx.x >> 4;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (r > 0) __syncthreads();
        leave_share(s, tile[r], wave, rd.m, rd.g, active);
        if (wave == 0 && rd.g == 0) s.row[rd.m] = tile[r].req;  // (an item has tokens: wavefront 0 is active)
        __syncthreads();
        if (16 * r >= rows) break;  // (the same for all threads)
        f32x4 x, y;
        float M, L;
        join_shares(s, out_row, col, c, x, y, M, L);
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(x[j]), fabsf(y[j])));
        top = fmaxf(top, dpp<kQuadXor1>(top));
        top = fmaxf(top, dpp<kQuadXor2>(top));
        top = fmaxf(top, dpp<kRor4>(top));
        top = fmaxf(top, dpp<kRor8>(top));
        float up, down;
        part_factors(top, up, down);
        if (16 * r + out_row >= rows) continue;
        const size_t part = part_of(a, it, s.row[out_row], 16 * r + out_row);
        *reinterpret_cast<u32x4 *>(a.o_parts + part * kHeadDim + 8 * col) =
            u32x4{pack_f16(x[0] * up, x[1] * up), pack_f16(x[2] * up, x[3] * up), pack_f16(y[0] * up, y[1] * up), pack_f16(y[2] * up, y[3] * up)};
        if (col == 0) {
            a.down_parts[part] = down;
            a.lse_parts[part] = partial_lse(M * c, L);
        }
    }
}

// Small steps: a workgroup of W wavefronts per KV head and leaf (and up to 16 of its rows) walks the whole path and writes the result itself: no items' partials
// and no second launch (4 requests over 256 + 49 tokens 6.6 us, as items and merge 7.8).  What bounds it is the chain of record, codes and queries, and a
// step's own length.  Blocks that are not full may lie anywhere on the path, at the end of every node; `gap` is how many of a block's last slots are nobody's.
struct PathStep : Operands {
    int gap;  // of the lane's block of V, which is that of its scores too
};
template <int W>
__global__ __launch_bounds__(64 * W, W == 4 ? 3 : 2) void four_path_kernel(DecodePathLaunch a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    Shares<W> &s = *reinterpret_cast<Shares<W> *>(smem);
    const int lane = (int)threadIdx.x & 63, m = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int Hkv = a.pool.num_kv_heads, G = a.num_q_heads / Hkv, head = (int)blockIdx.x % Hkv;
    const int32_t *path = a.paths + (size_t)(blockIdx.x / Hkv) * a.path_stride;
    const int n_blocks = path[0], rows = path[1] * G, n_steps = (n_blocks + 3) / 4;
    const float c = exponent_factor(a.scale);
    const uint8_t *k = static_cast<const uint8_t *>(a.pool.k_pages) + (m & 3) * 64 + g * 16, *v = static_cast<const uint8_t *>(a.pool.v_pages) + m * 16;
    const uint8_t *k_scale = reinterpret_cast<const uint8_t *>(a.pool.k_scale) + g * 16 + 4 * (m & 3), *v_scale = reinterpret_cast<const uint8_t *>(a.pool.v_scale) + (m >> 2) * 16;
    // Clamped to the record, whose end is zeros, so always in bounds and asked for before the path's length is known; a block behind the path's last is all gap.
    auto ids = [&](int (&id)[4], int b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) id[i] = path[kPathBlocks + min(4 * b + i, a.path_stride - kPathBlocks - 1)];
    };
    auto block = [&](int id) { return (size_t)(id & kPathIdMask) * Hkv + head; };
    auto fetch_keys = [&](PathStep &x, const int (&id)[4]) {
        const size_t kb = block(pick4(id, m >> 2));
        x.k_scale = *reinterpret_cast<const uint32_t *>(k_scale + kb * four::kScaleBytes);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.k[j] = ld16(k + kb * four::kCodeBytes + 256 * j);
    };
    auto fetch_values = [&](PathStep &x, const int (&id)[4], int b) {
        const int mine = pick4(id, g) | (4 * b + g < n_blocks ? 0 : 16 << kPathIdBits);
        const size_t vb = block(mine);
        x.gap = (int)((uint32_t)mine >> kPathIdBits);
        x.v_scale = ld16(v_scale + vb * four::kScaleBytes);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[j] = ld16(v + vb * four::kCodeBytes + 256 * j);
    };
    RowTile tile[1];
    RowTile &t = tile[0];
    PathStep now, next;
    int id[4], b = wave;
    ids(id, b);
    const int q_at = path[kPathQRows + m / G] * a.num_q_heads + head * G + m % G;  // (the record has 16 requests, the last one again and again)
    t.req = path[kPathRows + m / G];
    fetch_keys(now, id);
    fetch_values(now, id, b);
    u32x4 w[4];
    const char *qp = static_cast<const char *>(a.q) + (size_t)q_at * (kHeadDim * 2) + 64 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = ld16(qp + 16 * i);
    ids(id, b + W);
    t.lim = a.row_leaf ? path[2] + a.row_limit[t.req] : INT_MAX;  // (positions count whole blocks: the leaf begins at one)
    split_row(w, a.scale, t.q, t.q_scale);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) t.o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    t.m = -INFINITY;
    t.l = 0.f;
    // With four wavefronts a workgroup (more workgroups than compute units) the third and fourth term come from LDS in every step, and V of the next step is asked for
    // behind the scores: three wavefronts a SIMD instead of two (96 requests over 200 + 60 tokens, 32 + 8 heads, 9.2 us; with all in registers 11.0). Of eight there is
    // one workgroup a compute unit, and waiting for LDS costs (4 requests over 256 + 49 tokens 6.6 us, like that 6.9).
    constexpr bool kSpare = W == 4;
    u32x4 *terms = reinterpret_cast<u32x4 *>(smem) + threadIdx.x;
    if constexpr (kSpare) {
        terms[0] = u32x4{t.q[2][0], t.q[2][1], t.q[2][2], t.q[2][3]};
        terms[64 * W] = u32x4{t.q[2][4], t.q[2][5], t.q[3][0], t.q[3][1]};
        terms[128 * W] = u32x4{t.q[3][2], t.q[3][3], t.q[3][4], t.q[3][5]};
    }
    auto step = [&](PathStep &x, PathStep &after, auto first) {
        f32x4 acc[1][4];
        u32x4 pw[1][2];
        if constexpr (kSpare) {
            asm volatile("" ::: "memory");  // (or they would stay in registers)
            const u32x4 t0 = terms[0], t1 = terms[64 * W], t2 = terms[128 * W];
            t.q[2] = u32x6{t0[0], t0[1], t0[2], t0[3], t1[0], t1[1]};
            t.q[3] = u32x6{t1[2], t1[3], t2[0], t2[1], t2[2], t2[3]};
        }
        auto fetch_rest = [&] {
            fetch_values(after, id, b + W);
            ids(id, b + 2 * W);
            __builtin_amdgcn_sched_barrier(0);
        };
        fetch_keys(after, id);
        if constexpr (!kSpare) fetch_rest();
        __builtin_amdgcn_sched_barrier(0);
        scores(x, tile, acc);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kSpare) fetch_rest();
        const int d0 = 16 * (4 * b + g) - t.lim;
        if (__builtin_amdgcn_ballot_w64(x.gap > 0 || d0 > -16)) {
            const uint32_t seen = seen_bits(d0, a.row_leaf ? a.row_mask[t.req] : 0ull) & 0xFFFFu >> x.gap;
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[0][j & 3][j >> 2] = (seen >> j & 1u) ? acc[0][j & 3][j >> 2] : -INFINITY;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t sc = x.v_scale[q];
                clear_from(x.v[q], sc, 16 - x.gap - 4 * q);
                x.v_scale[q] = sc;
            }
        }
        if constexpr (decltype(first)::value) {
            float sum[1];
            follow_all(tile, acc, c);
            weigh(tile, acc, c, pw, sum);
            t.l = sum[0];
        } else {
            weights(tile, acc, c, pw);
        }
        add_values(tile, x, pw);
        return (b += W) < n_steps;
    };
    if (step(now, next, std::true_type{}))  // (a wavefront without steps takes one of gaps: nothing waits for the path's length)
        while (step(next, now, std::false_type{}) && step(now, next, std::false_type{})) {
        }
    if constexpr (kSpare) __syncthreads();  // (the terms have been read)
    leave_share(s, t, wave, m, g, true);
    if (wave == 0 && g == 0) s.row[m] = q_at;
    __syncthreads();
    const int out_row = (int)threadIdx.x >> 4, col = lane & 15;
    if (out_row >= rows) return;
    f32x4 x, y;
    float M, L;
    join_shares(s, out_row, col, c, x, y, M, L);
    const float bad = L >= 0.f ? 0.f : __builtin_nanf("");  // a row whose scores hold a NaN or +inf
    x += bad;
    y += bad;
    const size_t to = (size_t)s.row[out_row];
    *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.out) + to * kHeadDim + 8 * col) = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    if (a.lse_out && col == 0) a.lse_out[to] = L != 0.f ? (M * c + fast_log2(L)) * kLn2 : -INFINITY;
}

// Items of more rows: a wavefront has rows of its own and sees all tokens.  Codes and scales come through a ring in LDS, a block of a step by each
// wavefront, three steps ahead: a workgroup's two steps in flight at most would be 4.4 MB on the chip, 2 TB/s.  V is widened once for all four, by
// wavefront w that of block w of the next step, 40 vector instructions instead of 152, and written where the second product's operands are read, 16 bytes a
// lane.  One barrier a step: it waits for LDS, not for what is on its way from memory.
__device__ __forceinline__ void load_to_lds4(const void *gptr, uint32_t lds_base) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(gptr), "s"(lds_base) : "memory");
}
struct RingReader {
    const DecodeItem &it;
    Widened &lds;
    const uint8_t *k, *v, *scale;  // the pool's; of a lane's words of scales
    const __attribute__((address_space(4))) int32_t *pages;  // (read by the scalar unit: a vector load would wait for the ring's loads in front of it)
    uint32_t k_at, v_at, v_word;  // a lane's bytes of a block, its word of V's scales
    int lane, wave, heads, last_page, t4;  // t4: of V it has tokens 4 t4 .. + 3, dims 8 (lane % 16) .. + 7
    int id;  // the page of the block that comes next
    u32x4 x;
    uint32_t x_scale;
    static constexpr int kLoads = 3;  // of a wavefront and step
    __device__ __forceinline__ RingReader(const DecodeLaunch &a, const DecodeItem &it, Widened &lds, uint32_t k_at, int t4) : it(it), lds(lds), k_at(k_at), t4(t4) {
        lane = (int)threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        heads = a.pool.num_kv_heads;
        last_page = (it.n_tokens - 1) >> 4;
        k = static_cast<const uint8_t *>(a.pool.k_pages);
        v = static_cast<const uint8_t *>(a.pool.v_pages);
        scale = reinterpret_cast<const uint8_t *>(lane & 16 ? a.pool.v_scale : a.pool.k_scale) + 4 * (lane & 15);
        pages = (const __attribute__((address_space(4))) int32_t *)(a.pages + it.page_off);
        v_at = t4 * 256 + (lane & 15) * 16;
        v_word = 16 + (lane >> 2 & 3) * 4 + t4;
    }
    __device__ __forceinline__ void page_of(int b) { id = pages[min(4 * b + wave, last_page)]; }  // clamped, so always in bounds
    __device__ __forceinline__ void issue(int b) {
        const size_t block = (size_t)id * heads + it.kv_head;
        const uint32_t to = lds_address(&lds.ring[b % kRing]);
        load_to_lds16(k + block * four::kCodeBytes, k_at, to + (uint32_t)offsetof(Stage, k) + 1024 * wave);
        load_to_lds16(v + block * four::kCodeBytes, v_at, to + (uint32_t)offsetof(Stage, v) + 1024 * wave);
        load_to_lds4(scale + block * four::kScaleBytes, to + (uint32_t)offsetof(Stage, scale) + 256 * wave);
        page_of(b + 1);
    }
    __device__ __forceinline__ void clean(int b) {  // V's slots behind the item's end, in this wavefront's block of step b
        if ((b + 1) * kStep <= it.n_tokens) return;
        Stage &st = lds.ring[b % kRing];
        u32x4 w = st.v[wave][lane];
        uint32_t sc = st.scale[wave][v_word];
        clear_from(w, sc, it.n_tokens - (b * kStep + 16 * wave + 4 * t4));
        st.v[wave][lane] = w;
        st.scale[wave][v_word] = sc;  // (four lanes the same)
    }
    __device__ __forceinline__ void take(int b) {
        x = lds.ring[b % kRing].v[wave][lane];
        x_scale = lds.ring[b % kRing].scale[wave][v_word];
    }
    template <int B>
    __device__ __forceinline__ void widen(char *lo_to, char *hi_to) {  // dims 2 B, 2 B + 1 of the lane's eight
        const uint32_t w[4] = {x[0], x[1], x[2], x[3]};
        const float sc[4] = {four::scale_of(x_scale, 0), four::scale_of(x_scale, 1), four::scale_of(x_scale, 2), four::scale_of(x_scale, 3)};
        u32x2 lo, hi;
        widen_pairs<B>(w, sc, lo, hi);
        *reinterpret_cast<u32x2 *>(lo_to) = lo;
        *reinterpret_cast<u32x2 *>(hi_to) = hi;
    }
    static __device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
    static __device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads * (kRing - 2)) : "memory"); }  // all but the last kRing - 2 steps requested
    static __device__ __forceinline__ void all_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }  // nothing may land in LDS that is another workgroup's by then
    // What a wavefront without rows does, from the first step's V on.
    template <class Widen>
    __device__ __forceinline__ void serve(int n_blk, Widen &&widen_all) {
        barrier();
        for (int b = 0; b < n_blk; ++b) {
            issue(b + kRing);
            clean(b + 1);
            take(b + 1);
            widen_all(b + 1);
            landed();
            barrier();
        }
        all_landed();
    }
};

// 33 to 64 rows, 16 a wavefront.
__device__ __forceinline__ void run_rows(const DecodeLaunch &a, const DecodeItem &it, Widened &lds) {
    const Reader rd(a, it);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), rows = it.n_req * (a.num_q_heads / a.pool.num_kv_heads);
    const int row0 = 16 * wave, n_blk = (it.n_tokens + kStep - 1) / kStep;
    const float c = exponent_factor(a.scale);
    // K's 16 bytes of token 4 tq + j and dims 32 dg lie at place 16 j + 4 ((block + dg) % 4) + tq, so that 16 lanes that differ in block and tq read 256 bytes of LDS
    RingReader ring(a, it, lds, (rd.lane >> 4) * 256 + (rd.lane & 3) * 64 + ((rd.lane >> 2) - wave & 3) * 16, rd.lane >> 4);
    auto widen_dims = [&](auto byte, int parity) {
        constexpr int B = decltype(byte)::value;
        char *to = reinterpret_cast<char *>(&lds.v[parity][8 * (rd.lane >> 5) + 2 * B][16 * wave + (rd.lane & 15)]) + 8 * (rd.lane >> 4 & 1);
        ring.widen<B>(to, to + 1024);
    };
    auto widen = [&](int b) {
        widen_dims(std::integral_constant<int, 0>{}, b & 1);
        widen_dims(std::integral_constant<int, 1>{}, b & 1);
        widen_dims(std::integral_constant<int, 2>{}, b & 1);
        widen_dims(std::integral_constant<int, 3>{}, b & 1);
    };
    RowTile tile[1];
    u32x4 w[1][4];
    find_rows(rd, row0, tile);
    ring.page_of(0);
    ring.issue(0);
    load_rows(rd, row0, tile, w);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 1; b < kRing; ++b) ring.issue(b);
    begin_rows(rd, tile, w);
    ring.landed();
    ring.clean(0);
    ring.take(0);
    widen(0);
    ring.barrier();
    if (row0 >= rows) return ring.serve(n_blk, widen);
    RowTile &t = tile[0];
    auto keys = [&](int b, u32x4 (&k)[4]) {
        const Stage &st = lds.ring[b % kRing];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = st.k[rd.m >> 2][16 * j + 4 * ((rd.m >> 2) + rd.g & 3) + (rd.m & 3)];
        return st.scale[rd.m >> 2][4 * rd.g + (rd.m & 3)];
    };
    // Matrix instructions and those of the softmax do not overlap between wavefronts of a SIMD by themselves (the sum of both was the kernel's time), so
    // each wavefront mixes its own: the first product of step b + 1 and the second of step b with the exponentials of step b and V's widening.
    f32x4 acc0[1][4], acc1[1][4];
    u32x4 pw[2];
    auto most = [](const f32x4 (&acc)[1][4], int j, float top) { return fmaxf(fmaxf(top, acc[0][j & 3][j >> 2]), acc[0][(j + 1) & 3][(j + 1) >> 2]); };
    auto settle = [&](f32x4 (&acc)[1][4], int b, float top) {  // scores of step b are what weights can be made of
        if (hide(rd, tile, acc, b)) {
            top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 16; j += 2) top = most(acc, j, top);
        }
        if (__builtin_amdgcn_ballot_w64((top - t.m) * c > kSlack)) follow(t, top, c);  // (-inf - -inf: no)
    };
    {
        Operands x;
        x.k_scale = keys(0, x.k);
        scores(x, tile, acc0);
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; j += 2) top = most(acc0, j, top);
        settle(acc0, 0, top);
    }
    ring.barrier();  // all are done with K of step 0
    auto step = [&](f32x4 (&now)[1][4], f32x4 (&next)[1][4], int b, auto parity) {
        constexpr int P = decltype(parity)::value;
        u32x4 k[4], va[4];
        ring.clean(b + 1);  // (behind the last step: of no use, and of no harm)
        const uint32_t k_scale = keys(b + 1, k);
        __builtin_amdgcn_sched_barrier(0);
        // every chunk up to a sched_barrier: two matrix instructions of the first product or one of the second, and about as many cycles of others
        const float mc = t.m == -INFINITY ? 0.f : t.m * c;
        float sum = 0.f, top = -INFINITY;
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4) next[0][t4] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto weigh_pair = [&](int i) {  // probabilities of two neighbouring tokens, those of the second product's first half first
            const int j = 2 * i;
            const float p0 = fast_exp2(__builtin_fmaf(now[0][j & 3][j >> 2], c, -mc)), p1 = fast_exp2(__builtin_fmaf(now[0][(j + 1) & 3][(j + 1) >> 2], c, -mc));
            sum += p0 + p1;
            pw[i >> 2][i & 3] = pack_bf16(p0, p1);
        };
        weigh_pair(0);  // while K comes from LDS
        __builtin_amdgcn_sched_barrier(0);
        constexpr int kFirst = 6;  // pairs up to the end of the first product
        in_turn<4 * kTerms>([&](auto n) {
            constexpr int i = decltype(n)::value;
            next[0][i & 3] = mfma_four<(i & 3), (i >> 2)>(k[i & 3], t.q, next[0][i & 3], k_scale, t.q_scale);
#pragma unroll
            for (int p = 1 + (kFirst - 1) * i / 16; p < 1 + (kFirst - 1) * (i + 1) / 16; ++p) weigh_pair(p);
            if constexpr (i >= 12) va[i - 12] = lds.v[P][i - 12][rd.lane];
            if constexpr (i & 1) __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            t.o[i & 7] = mfma16(as_bf16x8(va[i & 3]), as_bf16x8(pw[i >> 3]), t.o[i & 7]);
            if (i == 2) ring.take(b + 1);
            if (i + 4 < 16) va[i & 3] = lds.v[P][i + 4][rd.lane];
            if (i < 8 - kFirst) weigh_pair(kFirst + i);
            if (i == 4) ring.issue(b + kRing);  // where step b was: its keys and values left in step b - 1
            if (i >= 8) top = most(next, 2 * (i - 8), top);
            if (i == 6) widen_dims(std::integral_constant<int, 0>{}, std::integral_constant<int, 1 - P>{});
            if (i == 9) widen_dims(std::integral_constant<int, 1>{}, std::integral_constant<int, 1 - P>{});
            if (i == 11) widen_dims(std::integral_constant<int, 2>{}, std::integral_constant<int, 1 - P>{});
            if (i == 13) widen_dims(std::integral_constant<int, 3>{}, std::integral_constant<int, 1 - P>{});
            __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("" : "+v"(sum), "+v"(top));  // (found beside the product, not behind the branch that may find it anew)
        t.l += sum;
        settle(next, b + 1, top);
        ring.landed();  // the share of step b + 2; of all wavefronts behind the barrier
        ring.barrier();
    };
    for (int b = 0;;) {
        step(acc0, acc1, b, std::integral_constant<int, 0>{});
        if (++b >= n_blk) break;
        step(acc1, acc0, b, std::integral_constant<int, 1>{});
        if (++b >= n_blk) break;
    }
    ring.all_landed();
    write_rows(rd, row0, c, tile);
}

// Items of more than 64 rows: 32 a wavefront, which sees all tokens, by the 32x32 forms of both instructions.  Beside one of those another wavefront issues
// more vector instructions than beside two of the 16x16 forms (measured: three quarters of the time beside the first product's, against a half).
//   S^T  v_mfma_scale_f32_32x32x64_f8f6f4: row r of tile T is token 32 T + r of the step; lane (r, h) brings dims 64 kk + 32 h .. + 31 of it, and of query
//        row r the same.  It ends up with tokens 32 T + 8 (i / 4) + 4 h + i % 4 of its row.
//   O^T  v_mfma_f32_32x32x16_bf16: the tokens of block B that a lane has are 4 h .. + 3 and 8 + 4 h .. + 3, so those are what it brings of V for
//        dims 8 (m % 16) + 2 dt + m / 16 of tile dt.
// V is widened by wavefront w for block w, 4 tokens and 8 dims a lane.
struct TallRows {
    u32x6 q[2][kTerms];  // [kk]
    uint32_t q_scale[2];
    f32x16 o[4];
    float m, l;
    int req, lim;
};
__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int Term>
__device__ __forceinline__ f32x16 mfma_four_tall(u32x4 k, const u32x6 (&q)[kTerms], f32x16 c, uint32_t k_scale, uint32_t q_scale) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(as_four(k), as_six(q[Term]), c, 4, 2, 0, k_scale, Term, q_scale);
}
__device__ __forceinline__ void run_tall(const DecodeLaunch &a, const DecodeItem &it, Widened &lds) {
    const int lane = (int)threadIdx.x & 63, r = lane & 31, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int G = a.num_q_heads / a.pool.num_kv_heads, rows = it.n_req * G, row0 = 32 * wave, row = min(row0 + r, rows - 1), n_blk = (it.n_tokens + kStep - 1) / kStep;
    const float c = exponent_factor(a.scale);
    // K's 16 bytes of token t and dims 32 dg lie at place 16 dg + t
    RingReader ring(a, it, lds, (lane & 3) * 256 + (lane >> 2 & 3) * 64 + (lane >> 4) * 16, (lane >> 4 & 1) * 2 + h);
    auto widen_dims = [&](auto byte, int parity) {
        constexpr int B = decltype(byte)::value;
        char *to = reinterpret_cast<char *>(&lds.v[parity][4 * wave + B][32 * h + (lane & 15)]) + 8 * (lane >> 4 & 1);
        ring.widen<B>(to, to + 256);
    };
    auto widen = [&](int b) {
        widen_dims(std::integral_constant<int, 0>{}, b & 1);
        widen_dims(std::integral_constant<int, 1>{}, b & 1);
        widen_dims(std::integral_constant<int, 2>{}, b & 1);
        widen_dims(std::integral_constant<int, 3>{}, b & 1);
    };
    TallRows x;
    x.req = a.node_req_idx[it.req_off + row / G];
    ring.page_of(0);
    ring.issue(0);
    u32x4 w[2][4];  // dims 64 kk + 32 h .. + 31
    {
        const int q_row = a.q_rows ? a.q_rows[x.req] : x.req;
        const char *qp = static_cast<const char *>(a.q) + ((size_t)q_row * a.num_q_heads + it.kv_head * G + row % G) * (kHeadDim * 2) + 64 * h;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = ld16(qp + 128 * (i >> 2) + 16 * (i & 3));
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 1; b < kRing; ++b) ring.issue(b);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) split_row(w[kk], a.scale, x.q[kk], x.q_scale[kk]);
    x.lim = a.row_leaf && a.row_leaf[x.req] == it.node ? a.row_limit[x.req] - it.tok_begin : it.n_tokens;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) x.o[dt][i] = 0.f;
    x.m = -INFINITY;
    x.l = 0.f;
    ring.landed();
    ring.clean(0);
    ring.take(0);
    widen(0);
    ring.barrier();
    if (row0 >= rows) return ring.serve(n_blk, widen);
    auto most = [](const f32x16 (&acc)[2], int j, float top) { return fmaxf(fmaxf(top, acc[j >> 4][j & 15]), acc[j >> 4][(j & 15) + 1]); };
    auto settle = [&](f32x16 (&acc)[2], int b, float top) {  // scores of step b are what weights can be made of
        if (__builtin_amdgcn_ballot_w64((b + 1) * kStep > min(x.lim, it.n_tokens))) {  // some row does not see the whole step, the item's last one among them
            const bool last = a.row_leaf && a.row_leaf[x.req] == it.node;
            const unsigned long long vis = last ? a.row_mask[x.req] : 0ull;
            top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int d0 = b * kStep + 8 * j + 4 * h - x.lim;
                const uint32_t in_item = 0xFu >> min(max(b * kStep + 8 * j + 4 * h + 4 - it.n_tokens, 0), 4);
                const uint32_t seen = (d0 < 0 ? (d0 <= -4 ? 0xFu : (1u << -d0) - 1u | (uint32_t)vis << -d0) : d0 < 64 ? (uint32_t)(vis >> d0) : 0u) & in_item;
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j >> 2][4 * (j & 3) + i] = (seen >> i & 1u) ? acc[j >> 2][4 * (j & 3) + i] : -INFINITY;
                top = most(acc, 4 * j, most(acc, 4 * j + 2, top));
            }
        }
        if (__builtin_amdgcn_ballot_w64((top - x.m) * c > kSlack)) {  // (-inf - -inf: no)
            const float m_new = fmaxf(x.m, half_max(top));
            const float alpha = m_new == -INFINITY ? 1.f : fast_exp2((x.m - m_new) * c);
            x.m = m_new;
            x.l *= alpha;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) x.o[dt] *= alpha;
        }
    };
    const uint8_t *scale_at = reinterpret_cast<const uint8_t *>(&lds.ring[0].scale[0][0]) + (r >> 4) * 256 + 16 * h + (r & 15);
    auto keys = [&](int b, u32x4 (&k)[4], uint32_t (&ks)[4]) {  // [2 kk + T]
        const Stage &st = lds.ring[b % kRing];
        const uint8_t *sp = scale_at + (b % kRing) * sizeof(Stage);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            k[i] = st.k[2 * (i & 1) + (r >> 4)][16 * (2 * (i >> 1) + h) + (r & 15)];
            ks[i] = sp[512 * (i & 1) + 32 * (i >> 1)];
        }
    };
    f32x16 acc0[2], acc1[2];
    u32x4 pw[4];
    {
        u32x4 k[4];
        uint32_t ks[4];
        keys(0, k, ks);
#pragma unroll
        for (int i = 0; i < 16; ++i) acc0[0][i] = acc0[1][i] = 0.f;
        in_turn<4 * kTerms>([&](auto n) {
            constexpr int i = decltype(n)::value;
            acc0[i & 1] = mfma_four_tall<(i >> 2)>(k[i & 3], x.q[i >> 1 & 1], acc0[i & 1], ks[i & 3], x.q_scale[i >> 1 & 1]);
        });
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 32; j += 2) top = most(acc0, j, top);
        settle(acc0, 0, top);
    }
    ring.barrier();  // all are done with K of step 0
    auto step = [&](f32x16 (&now)[2], f32x16 (&next)[2], int b, auto parity) {
        constexpr int P = decltype(parity)::value;
        u32x4 k[4], va[4];
        uint32_t ks[4];
        ring.clean(b + 1);  // (behind the last step: of no use, and of no harm)
        keys(b + 1, k, ks);
        __builtin_amdgcn_sched_barrier(0);
        const float mc = x.m == -INFINITY ? 0.f : x.m * c;
        float sum = 0.f, top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) next[0][i] = next[1][i] = 0.f;
        auto weigh_pair = [&](int p) {  // probabilities of two neighbouring tokens, in the order in which the second product takes them
            const int at = 8 * (p >> 2 & 1) + 2 * (p & 3);
            const float p0 = fast_exp2(__builtin_fmaf(now[p >> 3][at], c, -mc)), p1 = fast_exp2(__builtin_fmaf(now[p >> 3][at + 1], c, -mc));
            sum += p0 + p1;
            pw[p >> 2][p & 3] = pack_bf16(p0, p1);
        };
        // every chunk up to a sched_barrier: a matrix instruction (32 cycles) and what fits beside it
        constexpr int kBefore = 2, kFirst = 12, kIssue = 5;  // pairs while K comes from LDS, and up to the end of the first product; where the ring's loads go out
#pragma unroll
        for (int p = 0; p < kBefore; ++p) weigh_pair(p);
        __builtin_amdgcn_sched_barrier(0);
        in_turn<4 * kTerms>([&](auto n) {
            constexpr int i = decltype(n)::value;
            next[i & 1] = mfma_four_tall<(i >> 2)>(k[i & 3], x.q[i >> 1 & 1], next[i & 1], ks[i & 3], x.q_scale[i >> 1 & 1]);
#pragma unroll
            for (int p = kBefore + (kFirst - kBefore) * i / 16; p < kBefore + (kFirst - kBefore) * (i + 1) / 16; ++p) weigh_pair(p);
            if constexpr (i >= 12) va[i - 12] = lds.v[P][i - 12][lane];
            __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(va[i & 3]), as_bf16x8(pw[i >> 2]), x.o[i & 3], 0, 0, 0);
            if (i == 2) ring.take(b + 1);
            if (i + 4 < 16) va[i & 3] = lds.v[P][i + 4][lane];
            if (i < 16 - kFirst) weigh_pair(kFirst + i);
            if (i == kIssue) ring.issue(b + kRing);  // where step b was: its keys and values left in step b - 1
            if (i >= 6 && i < 14) top = most(next, 4 * (i - 6), most(next, 4 * (i - 6) + 2, top));
            if (i == 8) widen_dims(std::integral_constant<int, 0>{}, std::integral_constant<int, 1 - P>{});
            if (i == 10) widen_dims(std::integral_constant<int, 1>{}, std::integral_constant<int, 1 - P>{});
            if (i == 12) widen_dims(std::integral_constant<int, 2>{}, std::integral_constant<int, 1 - P>{});
            if (i == 14) widen_dims(std::integral_constant<int, 3>{}, std::integral_constant<int, 1 - P>{});
            __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("" : "+v"(sum), "+v"(top));  // (found beside the product, not behind the branch that may find it anew)
        x.l += sum;
        settle(next, b + 1, top);
        ring.landed();  // the share of step b + 2; of all wavefronts behind the barrier
        ring.barrier();
    };
    for (int b = 0;;) {
        step(acc0, acc1, b, std::integral_constant<int, 0>{});
        if (++b >= n_blk) break;
        step(acc1, acc0, b, std::integral_constant<int, 1>{});
        if (++b >= n_blk) break;
    }
    ring.all_landed();
    const float l_row = half_sum(x.l), inv = l_row > 0.f ? 1.0f / l_row : 0.f;
    float top = 0.f;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) {
        x.o[dt] *= inv;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x.o[dt][i]));
    }
    float up, down;
    part_factors(half_max(top), up, down);
    if (row0 + r >= rows) return;
    const size_t part = part_of(a, it, x.req, row);
    uint16_t *out = a.o_parts + part * kHeadDim + 32 * h;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u32x4 word;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) word[dt] = pack_f16(x.o[dt][i] * up, x.o[dt][i + 8] * up);
        *reinterpret_cast<u32x4 *>(out + 64 * (i >> 2) + 8 * (i & 3)) = word;
    }
    if (h == 0) {
        a.down_parts[part] = down;
        a.lse_parts[part] = partial_lse(l_row == l_row ? x.m * c : INFINITY, l_row);
    }
}

// Items [0, n_single) get a workgroup each, the items behind them (at most 16 rows) one for four, a wavefront each (no LDS, no barrier), in the plan's order
// of sets of eight workgroups, one for each XCD.  Those of many rows are bound by their instructions, the others by memory, so a compute unit should hold one
// of either kind, to the end.
constexpr int kXcds = 8;
__global__ __launch_bounds__(kWaves * 64, 2) void four_decode_kernel(DecodeLaunch a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    Lds &lds = *reinterpret_cast<Lds *>(smem);
    const int G = a.num_q_heads / a.pool.num_kv_heads;
    const int set = blockIdx.x / kXcds, single_sets = (a.n_single + kXcds - 1) / kXcds;
    const int place = a.order ? a.order[set] : set < single_sets ? set : ~(set - single_sets);
    if (place < 0) {
        const int at = a.n_single + kWaves * (kXcds * ~place + (int)(blockIdx.x % kXcds)) + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        if (at >= a.n_items) return;
        const DecodeItem it = a.items[at];
        const Reader rd(a, it);
        const float c = exponent_factor(a.scale);
        RowTile tile[1];
        stream(rd, 0, 0, 1, c, tile);
        write_rows(rd, 0, c, tile);
        return;
    }
    const int at = kXcds * place + (int)(blockIdx.x % kXcds);
    if (at >= a.n_single) return;
    const DecodeItem it = a.items[at];
    const int rows = it.n_req * G;
    // Measured on both sides (16 prompts of 2048 tokens in items of 1024, 8 KV heads): 32 rows with tokens shared 17.2 us, with 16 rows a wavefront 21.5; 48
    // rows with 16 a wavefront 22.8, with 32 a wavefront, two of them idle beside it, 26.4.  More than 64 rows only the last form takes.
    if (rows <= 16)
        run_shared_tokens<1>(a, it, lds.s);
    else if (rows <= 32)
        run_shared_tokens<2>(a, it, lds.s);
    else if (rows <= 64)
        run_rows(a, it, lds.w);
    else
        run_tall(a, it, lds.w);
}

}  // namespace

hipError_t prepare_four_decode() {
    if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(four_path_kernel<8>), hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Shares<8>)); e != hipSuccess) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void *>(four_decode_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Lds));
}

hipError_t launch_four_paths(const DecodePathLaunch &a, int waves, hipStream_t s, hipEvent_t ev_begin, hipEvent_t ev_end) {
    if (a.n_paths <= 0) return hipSuccess;
    if (waves != 4 && waves != 8) return hipErrorInvalidValue;
    if (hipError_t e = prepare_decode_device(nullptr); e != hipSuccess) return e;
    const dim3 grid((unsigned)a.n_paths * (unsigned)a.pool.num_kv_heads), block(64 * waves);
    if (waves == 4)
        hipExtLaunchKernelGGL(four_path_kernel<4>, grid, block, (unsigned)sizeof(Shares<4>), s, ev_begin, ev_end, 0, a);
    else
        hipExtLaunchKernelGGL(four_path_kernel<8>, grid, block, (unsigned)sizeof(Shares<8>), s, ev_begin, ev_end, 0, a);
    return hipGetLastError();
}

hipError_t launch_four_decode(const DecodeLaunch &a, hipStream_t s, hipEvent_t ev_begin, hipEvent_t ev_end) {
    if (a.n_items <= 0) return hipSuccess;
    if (hipError_t e = prepare_decode_device(nullptr); e != hipSuccess) return e;
    const int packs = (a.n_items - a.n_single + kWaves - 1) / kWaves;
    const dim3 grid(kXcds * ((a.n_single + kXcds - 1) / kXcds + (packs + kXcds - 1) / kXcds));
    hipExtLaunchKernelGGL(four_decode_kernel, grid, dim3(kWaves * 64), (unsigned)sizeof(Lds), s, ev_begin, ev_end, 0, a);
    return hipGetLastError();
}

}  // namespace hkv
