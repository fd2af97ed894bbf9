// What the queries of a step gave to every cached key: W[t] = decay * W[t] + sum over rows r that see t of exp(scale * q_r . k_t - lse_r),
// rows being the query heads of a KV head of all requests below the key's node (attn_decode_plan_weights).
//
// The softmax is known already (lse), so one product is all there is: S = K Q^T on the matrix cores, 32 keys x 32 rows a tile,
// K's operand kept in registers while the rows go by.  A lane holds one row and 16 of the keys, so the row's lse is one
// register of it, a row that does not count is a lane switched off, and the keys' sums are 16 registers that are added across lanes
// once, at the end.  A key belongs to one workgroup, which adds in a fixed order: no atomics, the same bits every time.
#include "hkv_device.h"

namespace hkv {

namespace {

// Dims that lane half h holds of matrix step kk (of 8): 32 * (kk / 2) + 16 h + 8 * (kk % 2) .. + 7, for K and Q alike (the order of the sum is
// free), so that 16 codes of an fp8 key are one load and two steps.
__device__ __forceinline__ int dim_of(int kk, int h) { return 32 * (kk >> 1) + 16 * h + 8 * (kk & 1); }

template <int DT>
__global__ __launch_bounds__(256) void key_weights_kernel(KeyWeightsLaunch a) {
    const KeyWeightItem it = a.items[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 31, h = lane >> 5;
    int n_node = it.tokens;
    if (it.item >= 0) n_node = a.plan_items[it.item].tok_begin + a.plan_items[it.item].n_tokens;
    const bool last_node = it.node >= 0;
    const int t0 = it.tok_begin + 32 * wave;  // the wavefront's 32 keys
    if (t0 >= n_node) return;
    const int Hkv = a.pool.num_kv_heads, G = a.num_q_heads / Hkv;

    // the keys: lane (m, h) holds key t0 + m; a block behind the node's last one is not looked up
    const int n_blocks = (n_node - it.tok_begin + kPage - 1) / kPage;
    const int b0 = a.pages[it.page_off + 2 * wave], b1 = a.pages[it.page_off + min(2 * wave + 1, n_blocks - 1)];
    const size_t head0 = (size_t)b0 * Hkv + it.kv_head, head1 = (size_t)b1 * Hkv + it.kv_head;
    bf16x8 k[8];
    float c0 = a.scale * kLog2e, c1 = c0;
    {
        const size_t at = (m < 16 ? head0 : head1) * kBlockElems;
        const int slot = m & 15;
        if constexpr (DT == 0) {
            const uint16_t *p = static_cast<const uint16_t *>(a.pool.k_pages) + at + slot * 32;
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) k[kk] = as_bf16x8(ld16(p + (kk >> 1) * 512 + 16 * h + 8 * (kk & 1)));
        } else {
            const uint8_t *p = static_cast<const uint8_t *>(a.pool.k_pages) + at + slot * 64;
#pragma unroll
            for (int kk = 0; kk < 8; kk += 2) {
                const u32x4 w = ld16(p + (kk >> 2) * 1024 + 32 * (kk >> 1 & 1) + 16 * h);
                k[kk] = fp8x8_to_bf16x8(w[0], w[1]);
                k[kk + 1] = fp8x8_to_bf16x8(w[2], w[3]);
            }
            c0 *= a.pool.k_scale[head0];
            c1 *= a.pool.k_scale[head1];
        }
    }

    float sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.f;
    // rows see the last tokens of their own last node in part
    const bool partial = a.row_leaf && last_node && t0 + 32 > n_node - a.tokens_per_req;
    const int n_rows = it.n_req * G;
    for (int r0 = 0; r0 < n_rows; r0 += 32) {
        const int r = r0 + m;
        bool on = r < n_rows;
        const int j = on ? r / G : 0;
        const int row = a.node_req_idx[it.req_off + j];
        const size_t qh = (size_t)(a.q_rows ? a.q_rows[row] : row) * a.num_q_heads + it.kv_head * G + (on ? r - j * G : 0);
        const float lse = a.lse[qh] * kLog2e;
        on = on && fabsf(lse) < INFINITY;
        const uint16_t *q = static_cast<const uint16_t *>(a.q) + qh * kHeadDim;
        f32x16 s = zero16();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) s = mfma32(k[kk], as_bf16x8(ld16(q + dim_of(kk, h))), s);
        if (on) {
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = fast_exp2(__builtin_fmaf(s[i], i < 8 ? c0 : c1, -lse));
            if (partial && a.row_leaf[row] == it.node) {
                const int limit = a.row_limit[row];
                const unsigned long long mask = a.row_mask[row];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int late = t0 + 8 * (i >> 2) + 4 * h + (i & 3) - limit;  // (below 64: such tokens end the node)
                    if (late >= 0 && !(mask >> min(late, 63) & 1)) p[i] = 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] += p[i];
        }
    }
    // over the 32 lanes of a half; lane i of it keeps key i
    float w = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float v = sum[i];
        v += dpp<kQuadXor1>(v);
        v += dpp<kQuadXor2>(v);
        v += dpp<kRor4>(v);
        v += dpp<kRor8>(v);
        const uint32_t x = __float_as_uint(v);
        const auto b = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
        if ((lane & 15) == i) w = v;
    }
    if (lane & 16) return;
    const int i = lane & 15, mk = 8 * (i >> 2) + 4 * h + (i & 3), t = t0 + mk;
    if (t >= n_node) return;
    float *out = a.weights + (mk < 16 ? head0 : head1) * kPage + (mk & 15);
    const bool fresh = last_node && t >= n_node - a.n_new;
    if (a.decay != 0.f && !fresh) w = __builtin_fmaf(a.decay, *out, w);
    *out = w;
}

}  // namespace

hipError_t launch_key_weights(const KeyWeightsLaunch &a, hipStream_t s) {
    if (a.n_items <= 0) return hipSuccess;
    if (a.pool.dtype == 0)
        hipLaunchKernelGGL(key_weights_kernel<0>, dim3(a.n_items), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL(key_weights_kernel<1>, dim3(a.n_items), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace hkv
