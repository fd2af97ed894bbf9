// Decode attention over 4-bit pools: one workgroup per item (a chunk of a prefix-tree node, one KV head, up to 128 query rows), partial results to
// the log-sum-exp merge.  (Section 5, "Proactive Cache Management": a node's pages are read once for all requests below it.)
//
// A wavefront takes 64 tokens (four blocks) a step, for one or two tiles of 16 query rows:
//   S^T = K Q^T   v_mfma_scale_f32_16x16x128_f8f6f4: K's codes and scales as they lie in the pool, lane (m, g) dims 32 g .. + 31 of token 4 m + t4 in
//                 tile t4 (its four scales are one word); a query row as two e4m3 terms, x * 2^e = hi + lo, whose 2^-e is the other scale.  Against bf16
//                 operands widened from the codes that is the same matrix time and 68 fewer vector instructions a step.
//   O^T = V^T P^T v_mfma_f32_16x16x32_bf16: lane (m, g) brings dim 8 m + dt of eight tokens of block g.  A scale stands for one token and 32 dims, the
//                 instruction's for 32 tokens of a dim, so V is widened: two codes (neighbouring dims of a token) an instruction, then one more to
//                 bring two tokens of a dim together.  Two tiles share that: 160 of the 690 vector instructions (in quarters of 16
//                 lanes) of a step of two.
// A lane of a score tile t4 holds tokens 16 g + 4 i + t4 of its query row m: over the four tiles all 16 tokens of block g, which is what its
// share of P^T is made of, so probabilities stay where they are.  Widened values are exact (two significant bits, a power of two).
#include <hip/hip_ext.h>

#include <type_traits>

#include "four_bit.h"

namespace hkv {

namespace {

constexpr int kWaves = 4, kStep = 64;  // wavefronts; tokens of a step
constexpr int kORow = kHeadDim + 4;    // padded LDS row

typedef __attribute__((ext_vector_type(8))) int i32x8;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// 16 tokens (e2m1, scale byte T of k_scale) x 128 dims by 128 dims x 16 rows (e4m3, scale byte 0 of q_scale).  Lane (m, g): of the tokens dims 32 g .. + 31, of
// the rows dims 16 g .. + 15 and 64 + 16 g .. + 15.
template <int T>
__device__ __forceinline__ f32x4 mfma_four(u32x4 k, i32x8 q, f32x4 c, uint32_t k_scale, uint32_t q_scale) {
    const i32x8 a = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q, c, 4, 0, T, k_scale, 0, q_scale);
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
    i32x8 hi, lo;       // the query row
    uint32_t q_scale;
    f32x4 o[8];         // o[dt][i]: dim 32 g + 8 i + dt
    float m, l;         // reference (raw scores), this lane's share of the row sum
    uint32_t part;      // the partial that the row writes
    int lim;            // tokens of the item that the row may see, and of those behind them, the visible ones
    unsigned long long vis;
};

// Four values, |x| <= 448, as e4m3 (to nearest).
__device__ __forceinline__ int e4m3x4(float a, float b, float c, float d) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// A row as two e4m3 terms: its largest magnitude is brought into [128, 256) by a power of two, the first term holds four significant bits, the second
// what is left: exact for a bf16 value down to 2^-9 of the row's largest, from there on to 2^-17 of it.  sign: -1 for a negative softmax scale.
__device__ __forceinline__ void split_row(RowTile &x, const u32x4 (&w)[4], float sign) {
    float q[32], top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            q[8 * i + 2 * j] = __uint_as_float(w[i][j] << 16);
            q[8 * i + 2 * j + 1] = __uint_as_float(w[i][j] & 0xFFFF0000u);
        }
#pragma unroll
    for (int j = 0; j < 32; ++j) top = fmaxf(top, fabsf(q[j]));
    top = rows_max(top);
    const int ex = min(max((int)(__float_as_uint(top) >> 23), 8), 254);  // where both powers are normal numbers
    const float up = __uint_as_float((uint32_t)(261 - ex) << 23) * sign;
    x.q_scale = (uint32_t)(ex - 7);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float a = q[4 * j] * up, b = q[4 * j + 1] * up, c = q[4 * j + 2] * up, d = q[4 * j + 3] * up;
        const int h = e4m3x4(a, b, c, d);
        const auto h0 = __builtin_amdgcn_cvt_pk_f32_fp8(h, false), h1 = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
        x.hi[j] = h;
        x.lo[j] = e4m3x4(a - h0[0], b - h0[1], c - h1[0], d - h1[1]);
    }
}

// One item by the workgroup: RT row tiles a wavefront.
template <int RT>
__device__ __forceinline__ void run_item(const DecodeLaunch &a, const DecodeItem &it, float (*sO)[16][kORow], float (*sM)[16], float (*sL)[16], uint32_t (*sPart)[16]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int m = lane & 15, g = lane >> 4;
    const int Hkv = a.pool.num_kv_heads, G = a.num_q_heads / Hkv, rows = it.n_req * G;
    // wavefronts: groups of RT row tiles x shares of the steps
    const int n_rg = RT == 1 || rows <= 32 ? 1 : rows <= 64 ? 2 : 4, n_ts = kWaves / n_rg;
    const int row0 = wave % n_rg * (16 * RT), ts = wave / n_rg;
    const float c = fmaxf(fabsf(a.scale) * kLog2e, 1e-30f);  // (scores times 0: a weight of 1 each, and -inf stays)

    const int n_blk = (it.n_tokens + kStep - 1) / kStep, last_page = (it.n_tokens - 1) >> 4;
    const uint8_t *kc = static_cast<const uint8_t *>(a.pool.k_pages) + (m & 3) * 64 + g * 16, *vc = static_cast<const uint8_t *>(a.pool.v_pages) + m * 16;
    const uint8_t *ks = reinterpret_cast<const uint8_t *>(a.pool.k_scale) + g * 16 + 4 * (m & 3), *vs = reinterpret_cast<const uint8_t *>(a.pool.v_scale) + (m >> 2) * 16;
    auto load_ids = [&](int (&id)[4], int b) {  // wavefront-uniform: scalar loads; clamped, so always in bounds
#pragma unroll
        for (int i = 0; i < 4; ++i) id[i] = a.pages[it.page_off + min(4 * b + i, last_page)];
    };
    auto issue_k = [&](Operands &x, const int (&id)[4]) {
        const size_t blk = (size_t)pick4(id, m >> 2) * Hkv + it.kv_head;
        const uint8_t *p = kc + blk * four::kCodeBytes;
        x.k_scale = *reinterpret_cast<const uint32_t *>(ks + blk * four::kScaleBytes);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.k[j] = ld16(p + 256 * j);
    };
    auto issue_v = [&](Operands &x, const int (&id)[4]) {
        const size_t blk = (size_t)pick4(id, g) * Hkv + it.kv_head;
        const uint8_t *p = vc + blk * four::kCodeBytes;
        x.v_scale = ld16(vs + blk * four::kScaleBytes);
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[j] = ld16(p + 256 * j);
    };

    RowTile tile[RT];
    auto load_rows = [&]() {
        u32x4 w[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = row0 + 16 * r + m, rowc = min(row, rows - 1);
            const int req = a.node_req_idx[it.req_off + rowc / G], head = it.kv_head * G + rowc % G;
            const int q_row = a.q_rows ? a.q_rows[req] : req;
            const char *qp = static_cast<const char *>(a.q) + ((size_t)q_row * a.num_q_heads + head) * (kHeadDim * 2) + 32 * g;
            w[r][0] = ld16(qp);
            w[r][1] = ld16(qp + 16);
            w[r][2] = ld16(qp + 128);
            w[r][3] = ld16(qp + 144);
            tile[r].part = (uint32_t)((req * a.num_q_heads + head) * a.max_parts + it.part_slot);
            tile[r].lim = it.n_tokens;
            tile[r].vis = 0;
            if (a.row_leaf && a.row_leaf[req] == it.node) {
                tile[r].lim = a.row_limit[req] - it.tok_begin;
                tile[r].vis = a.row_mask[req];
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            split_row(tile[r], w[r], a.scale < 0.f ? -1.f : 1.f);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) tile[r].o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
            tile[r].m = -INFINITY;
            tile[r].l = 0.f;
        }
    };

    // The first product, softmax and second product of a step; `between` comes where K's registers are free.
    auto step = [&](Operands &x, int b, auto between) {
        const int tok0 = b * kStep + 16 * g;  // of this lane's 16 tokens the first
        f32x4 acc[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const RowTile &t = tile[r];
#pragma unroll
            for (int t4 = 0; t4 < 4; ++t4) acc[r][t4] = f32x4{0.f, 0.f, 0.f, 0.f};
            acc[r][0] = mfma_four<0>(x.k[0], t.hi, acc[r][0], x.k_scale, t.q_scale);
            acc[r][1] = mfma_four<1>(x.k[1], t.hi, acc[r][1], x.k_scale, t.q_scale);
            acc[r][2] = mfma_four<2>(x.k[2], t.hi, acc[r][2], x.k_scale, t.q_scale);
            acc[r][3] = mfma_four<3>(x.k[3], t.hi, acc[r][3], x.k_scale, t.q_scale);
            acc[r][0] = mfma_four<0>(x.k[0], t.lo, acc[r][0], x.k_scale, t.q_scale);
            acc[r][1] = mfma_four<1>(x.k[1], t.lo, acc[r][1], x.k_scale, t.q_scale);
            acc[r][2] = mfma_four<2>(x.k[2], t.lo, acc[r][2], x.k_scale, t.q_scale);
            acc[r][3] = mfma_four<3>(x.k[3], t.lo, acc[r][3], x.k_scale, t.q_scale);
        }
        between();
        u32x4 pw[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            RowTile &t = tile[r];
            float s[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) s[j] = acc[r][j & 3][j >> 2];
            const int d0 = tok0 - t.lim;
            if (__builtin_amdgcn_ballot_w64(d0 > -16)) {  // some row does not see the whole step, the item's last one among them
                const uint32_t seen = d0 < 0 ? (d0 <= -16 ? 0xFFFFu : (1u << -d0) - 1u | (uint32_t)t.vis << -d0) : d0 < 64 ? (uint32_t)(t.vis >> d0) : 0u;
#pragma unroll
                for (int j = 0; j < 16; ++j) s[j] = (seen >> j & 1u) ? s[j] : -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s[j]);
            const float m_new = fmaxf(t.m, rows_max(mx));
            const float mc = m_new == -INFINITY ? 0.f : m_new * c;  // (a row that has seen nothing: no inf - inf)
            const float alpha = fast_exp2(__builtin_fmaf(t.m, c, -mc));
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                s[j] = fast_exp2(__builtin_fmaf(s[j], c, -mc));
                sum += s[j];
            }
            t.l = t.l * alpha + sum;
            t.m = m_new;
            if (__builtin_amdgcn_ballot_w64(alpha != 1.0f)) {
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) t.o[dt] *= alpha;
            }
            // probabilities are rounded to bf16, half a step of 2^-8 each, as over the other pools
#pragma unroll
            for (int j = 0; j < 8; ++j) pw[r][j >> 2][j & 3] = pack_bf16(s[2 * j], s[2 * j + 1]);
        }
        if ((b + 1) * kStep > it.n_tokens) {  // slots behind the end may hold anything
            const int first_bad = it.n_tokens - tok0;
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j >= first_bad) {
                    x.v[j >> 2][j & 3] = 0u;
                    x.v_scale[j >> 2] = (x.v_scale[j >> 2] & ~(0xFFu << (8 * (j & 3)))) | (127u << (8 * (j & 3)));
                }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // eight tokens of every block
            float sc[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[j] = four::scale_of(x.v_scale[2 * half + (j >> 2)], j & 3);
            auto dims = [&](auto byte) {  // dims 8 m + 2 B, + 1
                constexpr int B = decltype(byte)::value;
                u32x4 lo, hi;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t v0 = four::widen2<B>(x.v[2 * half + (j >> 1)][2 * (j & 1)], sc[2 * j]);
                    const uint32_t v1 = four::widen2<B>(x.v[2 * half + (j >> 1)][2 * (j & 1) + 1], sc[2 * j + 1]);
                    lo[j] = __builtin_amdgcn_perm(v1, v0, 0x05040100u);
                    hi[j] = __builtin_amdgcn_perm(v1, v0, 0x07060302u);
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    tile[r].o[2 * B] = mfma16(as_bf16x8(lo), as_bf16x8(pw[r][half]), tile[r].o[2 * B]);
                    tile[r].o[2 * B + 1] = mfma16(as_bf16x8(hi), as_bf16x8(pw[r][half]), tile[r].o[2 * B + 1]);
                }
            };
            dims(std::integral_constant<int, 0>{});
            dims(std::integral_constant<int, 1>{});
            dims(std::integral_constant<int, 2>{});
            dims(std::integral_constant<int, 3>{});
        }
    };

    const bool active = row0 < rows && ts < n_blk;
    if (active) {
        int id[4];
        int b = ts;
        load_ids(id, b);
        Operands x;
        issue_k(x, id);
        issue_v(x, id);
        load_ids(id, b + n_ts);
        load_rows();
        if constexpr (RT == 1) {  // the operands of one step travel while another is computed, page ids a step further ahead
            Operands y;
            auto ahead = [&](Operands &next) {
                issue_k(next, id);
                issue_v(next, id);
                load_ids(id, b + 2 * n_ts);
                __builtin_amdgcn_sched_barrier(0);
            };
            for (;;) {
                if (b + n_ts < n_blk) ahead(y);
                step(x, b, [] {});
                if ((b += n_ts) >= n_blk) break;
                if (b + n_ts < n_blk) ahead(x);
                step(y, b, [] {});
                if ((b += n_ts) >= n_blk) break;
            }
        } else {  // two tiles fill the registers: K of the next step is requested behind the first product, V behind the second
            for (; b < n_blk; b += n_ts) {
                const bool more = b + n_ts < n_blk;
                step(x, b, [&] {
                    __builtin_amdgcn_sched_barrier(0);
                    if (more) issue_k(x, id);
                    __builtin_amdgcn_sched_barrier(0);
                });
                __builtin_amdgcn_sched_barrier(0);
                if (more) issue_v(x, id);
                load_ids(id, b + 2 * n_ts);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    if (n_ts == 1) {  // a wavefront has seen all tokens of its rows: they go out from its registers, 32 dims a lane
        if (!active) return;
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
            if (row0 + 16 * r + m >= rows) continue;
            uint16_t *out = a.o_parts + (size_t)t.part * kHeadDim + 32 * g;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x4 w;
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] = pack_f16(t.o[2 * q][i] * up, t.o[2 * q + 1][i] * up);
                *reinterpret_cast<u32x4 *>(out + 8 * i) = w;
            }
            if (g == 0) {
                a.down_parts[t.part] = down;
                a.lse_parts[t.part] = partial_lse(l_row == l_row ? t.m * c : INFINITY, l_row);
            }
        }
        return;
    }
    // The shares of a row tile's tokens are brought together in LDS, a tile of every wavefront at a time; then thread (row = tid / 16, tid % 16)
    // has eight dims of a row, whose 16 threads are a row of lanes.
    const int col = lane & 15, out_row = (int)threadIdx.x >> 4;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (r > 0) __syncthreads();
        if (active) {
            const RowTile &t = tile[r];
            const float l_row = rows_sum(t.l);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *reinterpret_cast<f32x4 *>(&sO[wave][m][32 * g + 8 * i + 4 * q]) = f32x4{t.o[4 * q][i], t.o[4 * q + 1][i], t.o[4 * q + 2][i], t.o[4 * q + 3][i]};
            if (g == 0) {
                sM[wave][m] = l_row == l_row ? t.m : INFINITY;  // (a NaN or +inf among the scores: the row's sum is no number below)
                sL[wave][m] = l_row;
                if (ts == 0) sPart[wave][m] = t.part;
            }
        } else if (g == 0) {
            sM[wave][m] = -INFINITY;
        }
        __syncthreads();
        for (int rg = 0; rg < n_rg; ++rg) {
            const int row = rg * (16 * RT) + 16 * r + out_row;
            if (rg * (16 * RT) + 16 * r >= rows) break;  // (the same for all threads)
            float M = -INFINITY, L = 0.f;
            for (int w = rg; w < kWaves; w += n_rg) M = fmaxf(M, sM[w][out_row]);
            f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
            for (int w = rg; w < kWaves; w += n_rg) {
                const float mw = sM[w][out_row];
                if (mw == -INFINITY) continue;  // that wavefront's tokens were all invisible to the row
                const float wgt = fast_exp2((mw - M) * c);
                L += sL[w][out_row] * wgt;
                x += *reinterpret_cast<const f32x4 *>(&sO[w][out_row][8 * col]) * wgt;
                y += *reinterpret_cast<const f32x4 *>(&sO[w][out_row][8 * col + 4]) * wgt;
            }
            const float inv = L > 0.f ? 1.0f / L : 0.f;
            x *= inv;
            y *= inv;
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(x[j]), fabsf(y[j])));
            top = fmaxf(top, dpp<kQuadXor1>(top));
            top = fmaxf(top, dpp<kQuadXor2>(top));
            top = fmaxf(top, dpp<kRor4>(top));
            top = fmaxf(top, dpp<kRor8>(top));
            float up, down;
            part_factors(top, up, down);
            if (row >= rows) continue;
            const size_t part = sPart[rg][out_row];
            *reinterpret_cast<u32x4 *>(a.o_parts + part * kHeadDim + 8 * col) =
                u32x4{pack_f16(x[0] * up, x[1] * up), pack_f16(x[2] * up, x[3] * up), pack_f16(y[0] * up, y[1] * up), pack_f16(y[2] * up, y[3] * up)};
            if (col == 0) {
                a.down_parts[part] = down;
                a.lse_parts[part] = partial_lse(M * c, L);
            }
        }
    }
}

__global__ __launch_bounds__(kWaves * 64, 2) void four_decode_kernel(DecodeLaunch a) {
    __shared__ float sO[kWaves][16][kORow];
    __shared__ float sM[kWaves][16], sL[kWaves][16];
    __shared__ uint32_t sPart[kWaves][16];
    const DecodeItem it = a.items[blockIdx.x];
    if (it.n_req * (a.num_q_heads / a.pool.num_kv_heads) <= 16)
        run_item<1>(a, it, sO, sM, sL, sPart);
    else
        run_item<2>(a, it, sO, sM, sL, sPart);
}

}  // namespace

hipError_t launch_four_decode(const DecodeLaunch &a, hipStream_t s, hipEvent_t ev_begin, hipEvent_t ev_end) {
    if (a.n_items <= 0) return hipSuccess;
    hipExtLaunchKernelGGL(four_decode_kernel, dim3(a.n_items), dim3(kWaves * 64), 0, s, ev_begin, ev_end, 0, a);
    return hipGetLastError();
}

}  // namespace hkv
