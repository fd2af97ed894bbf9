// Decode attention over 4-bit pools: one workgroup per item (a chunk of a prefix-tree node, one KV head, up to 64 query rows), partial results to
// the log-sum-exp merge.  (Section 5, "Proactive Cache Management": a node's pages are read once for all requests below it.)
//
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, four per 16 tokens: lane (m, g) brings dims 32 g + 8 j .. + 7 of token 4 m + t4 of a 64-token step
//   O^T = V^T P^T the same instruction: lane (m, g) brings dim 8 m + dt of eight tokens of block g
// Codes become bf16 exactly (two significant bits, a power of two), so the products are those of a bf16 pool that holds the same values.  A lane of
// a score tile t4 holds tokens 16 g + 4 i + t4 of its query row m: over the four tiles all 16 tokens of block g, which is what its
// share of P^T is made of, so probabilities stay where they are.
#include <hip/hip_ext.h>

#include "four_bit.h"

namespace hkv {

namespace {

constexpr int kWaves = 4, kStep = 64;  // wavefronts; tokens of a step
constexpr int kORow = kHeadDim + 4;    // padded LDS row

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

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

__global__ __launch_bounds__(kWaves * 64, 2) void four_decode_kernel(DecodeLaunch a) {
    __shared__ float sO[kWaves][16][kORow];
    __shared__ float sM[kWaves][16], sL[kWaves][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int m = lane & 15, g = lane >> 4;
    const DecodeItem it = a.items[blockIdx.x];
    const int Hkv = a.pool.num_kv_heads, G = a.num_q_heads / Hkv, rows = it.n_req * G;
    // wavefronts: row tiles of 16 x shares of the steps
    const int n_rt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4, n_ts = kWaves / n_rt;
    const int rt = wave % n_rt, ts = wave / n_rt;
    const float c = a.scale * kLog2e;
    const int row = rt * 16 + m, rowc = min(row, rows - 1);
    const bool active = rt * 16 < rows;

    const int req = a.node_req_idx[it.req_off + rowc / G], head = it.kv_head * G + rowc % G;
    bf16x8 qf[4];
    {
        const int q_row = a.q_rows ? a.q_rows[req] : req;
        const char *qp = static_cast<const char *>(a.q) + ((size_t)q_row * a.num_q_heads + head) * (kHeadDim * 2) + 64 * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4 w = ld16(qp + 16 * j);
            if (row >= rows) w = u32x4{0u, 0u, 0u, 0u};
            qf[j] = as_bf16x8(w);
        }
    }
    // tokens of the item that this lane's row may see, as in the other pools' kernels
    int lim = it.n_tokens;
    unsigned long long vis = 0;
    if (a.row_leaf && a.row_leaf[req] == it.node) {
        lim = a.row_limit[req] - it.tok_begin;
        vis = a.row_mask[req];
    }

    f32x4 o[8];  // o[dt][i]: dim 32 g + 8 i + dt of row m
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;  // reference in units of log2; this lane's share of the row sum

    const int n_blk = (it.n_tokens + kStep - 1) / kStep, last_page = (it.n_tokens - 1) >> 4;
    const uint8_t *kc = static_cast<const uint8_t *>(a.pool.k_pages), *vc = static_cast<const uint8_t *>(a.pool.v_pages);
    const uint8_t *ks = reinterpret_cast<const uint8_t *>(a.pool.k_scale), *vs = reinterpret_cast<const uint8_t *>(a.pool.v_scale);
    auto load = [&](Operands &x, int b) {
        int id[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) id[i] = a.pages[it.page_off + min(4 * b + i, last_page)];
        const size_t kblk = (size_t)pick4(id, m >> 2) * Hkv + it.kv_head, vblk = (size_t)pick4(id, g) * Hkv + it.kv_head;
        const uint8_t *kp = kc + kblk * four::kCodeBytes + (m & 3) * 64 + g * 16, *vp = vc + vblk * four::kCodeBytes + m * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x.k[j] = ld16(kp + 256 * j);
            x.v[j] = ld16(vp + 256 * j);
        }
        x.k_scale = *reinterpret_cast<const uint32_t *>(ks + kblk * four::kScaleBytes + g * 16 + 4 * (m & 3));
        x.v_scale = ld16(vs + vblk * four::kScaleBytes + (m >> 2) * 16);
    };
    auto step = [&](Operands &x, int b) {
        const int first_bad = it.n_tokens - (b * kStep + 16 * g);  // of this lane's 16 tokens, the first behind the item's end
        float s[16];
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            const float sc = four::scale_of(x.k_scale, t4);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = mfma16(as_bf16x8(four::widen8(x.k[t4][j], sc)), qf[j], acc);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[4 * i + t4] = acc[i] * c;
        }
        const bool tail = b * kStep + kStep > it.n_tokens;
        if (tail) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j >= first_bad) s[j] = -INFINITY;
        }
        const int tok0 = b * kStep + 16 * g;
        if (__builtin_amdgcn_ballot_w64(tok0 + 16 > lim)) {  // some row does not see the whole step
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int d = tok0 + j - lim;
                if (d >= 0 && !(d < 64 && ((vis >> d) & 1ull))) s[j] = -INFINITY;
            }
        }
        float mx = s[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s[j]);
        const float m_new = fmaxf(m_run, rows_max(mx));
        const float mc = m_new == -INFINITY ? 0.f : m_new;  // (a row that has seen nothing: no inf - inf)
        const float alpha = fast_exp2(m_run - mc);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            s[j] = fast_exp2(s[j] - mc);
            sum += s[j];
        }
        l_run = l_run * alpha + sum;
        m_run = m_new;
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f)) {
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[dt] *= alpha;
        }
        if (tail) {  // slots behind the end may hold anything
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j >= first_bad) {
                    x.v[j >> 2][j & 3] = 0u;
                    x.v_scale[j >> 2] = (x.v_scale[j >> 2] & ~(0xFFu << (8 * (j & 3)))) | (127u << (8 * (j & 3)));
                }
        }
        // probabilities are rounded to bf16, half a step of 2^-8 each, as over the other pools
#pragma unroll
        for (int ks2 = 0; ks2 < 2; ++ks2) {
            u32x4 pw;
#pragma unroll
            for (int j = 0; j < 4; ++j) pw[j] = pack_bf16(s[8 * ks2 + 2 * j], s[8 * ks2 + 2 * j + 1]);
            const bf16x8 pb = as_bf16x8(pw);
            float sc[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[j] = four::scale_of(x.v_scale[2 * ks2 + (j >> 2)], j & 3);
            auto dims = [&](auto byte) {  // dims 8 m + 2 B, + 1
                constexpr int B = decltype(byte)::value;
                u32x4 lo, hi;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t v0 = four::widen2<B>(x.v[2 * ks2 + (j >> 1)][2 * (j & 1)], sc[2 * j]);
                    const uint32_t v1 = four::widen2<B>(x.v[2 * ks2 + (j >> 1)][2 * (j & 1) + 1], sc[2 * j + 1]);
                    lo[j] = __builtin_amdgcn_perm(v1, v0, 0x05040100u);
                    hi[j] = __builtin_amdgcn_perm(v1, v0, 0x07060302u);
                }
                o[2 * B] = mfma16(as_bf16x8(lo), pb, o[2 * B]);
                o[2 * B + 1] = mfma16(as_bf16x8(hi), pb, o[2 * B + 1]);
            };
            dims(std::integral_constant<int, 0>{});
            dims(std::integral_constant<int, 1>{});
            dims(std::integral_constant<int, 2>{});
            dims(std::integral_constant<int, 3>{});
        }
    };

    if (active)
        for (int b = ts; b < n_blk; b += n_ts) {
            Operands x;
            load(x, b);
            step(x, b);
        }

    // the shares of a row tile's tokens are brought together, normalised and written as a partial
    const float l_row = rows_sum(l_run);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            *reinterpret_cast<f32x4 *>(&sO[wave][m][32 * g + 8 * i + 4 * q]) = f32x4{o[4 * q][i], o[4 * q + 1][i], o[4 * q + 2][i], o[4 * q + 3][i]};
    if (g == 0) {
        sM[wave][m] = l_row == l_row ? m_run : INFINITY;  // (a NaN or +inf among the scores: the row's sum is no number below)
        sL[wave][m] = l_row;
    }
    __syncthreads();
    for (int r = wave; r < rows; r += kWaves) {
        const int r_rt = r >> 4, r_m = r & 15, d = 2 * lane;
        float M = -INFINITY, L = 0.f, a0 = 0.f, a1 = 0.f;
        for (int w = r_rt; w < kWaves; w += n_rt) M = fmaxf(M, sM[w][r_m]);
        if (M != -INFINITY)
            for (int w = r_rt; w < kWaves; w += n_rt) {
                const float mw = sM[w][r_m];
                if (mw == -INFINITY) continue;
                const float wgt = fast_exp2(mw - M);
                L += sL[w][r_m] * wgt;
                a0 += sO[w][r_m][d] * wgt;
                a1 += sO[w][r_m][d + 1] * wgt;
            }
        const float inv = L > 0.f ? 1.0f / L : 0.f;
        a0 *= inv;
        a1 *= inv;
        float amax = fmaxf(fabsf(a0), fabsf(a1));
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1) amax = fmaxf(amax, __shfl_xor(amax, sh));
        float up, down;
        part_factors(amax, up, down);
        const int r_req = a.node_req_idx[it.req_off + r / G];
        const size_t part = (size_t)(r_req * a.num_q_heads + it.kv_head * G + r % G) * a.max_parts + it.part_slot;
        *reinterpret_cast<uint32_t *>(a.o_parts + part * kHeadDim + d) = pack_f16(a0 * up, a1 * up);
        if (lane == 0) {
            a.down_parts[part] = down;
            a.lse_parts[part] = partial_lse(M, L);
        }
    }
}

}  // namespace

hipError_t launch_four_decode(const DecodeLaunch &a, hipStream_t s, hipEvent_t ev_begin, hipEvent_t ev_end) {
    if (a.n_items <= 0) return hipSuccess;
    hipExtLaunchKernelGGL(four_decode_kernel, dim3(a.n_items), dim3(kWaves * 64), 0, s, ev_begin, ev_end, 0, a);
    return hipGetLastError();
}

}  // namespace hkv
