// Eviction: per sequence and KV head the heaviest tokens are chosen and moved, in order, to other blocks (kv_pool_evict).
//
// Choosing: the weights as integers in the order of the numbers, the k-th largest by its bits from the top (four histograms of 256
// bins), then the tokens above it and as many of its equals as are left, lowest index first, written in order by counts over wavefronts.
// One workgroup per (sequence, head); bound by the chain of its passes.
// Moving: one workgroup per (new block, head); 16 tokens come from 16 places.  K's dimensions lie in runs of 64 bytes a token, V's are
// 16 tokens wide, so that V is read in whole blocks however few of their tokens are kept.  fp8 blocks get the scale of what they
// hold now and are rounded again, as a block written anew.
#include "pool_block.h"

namespace hkv {

namespace {

constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;

// Order of the weights as integers: NaN below every number, both zeros equal.
__device__ __forceinline__ uint32_t key_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.0f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;
    return u >> 31 ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kChooseThreads) void evict_choose_kernel(EvictLaunch a) {
    const EvictSequence q = reinterpret_cast<const EvictSequence *>(a.meta)[blockIdx.x];
    const int h = blockIdx.y, Hkv = a.pool.num_kv_heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t *kept = a.kept + (size_t)h * a.total + q.kept;
    if (q.keep >= q.tokens) {
        for (int t = tid; t < q.tokens; t += kChooseThreads) kept[t] = t;
        return;
    }
    __shared__ int sBins[kChooseWaves][256];
    __shared__ int sCount[2][kChooseWaves];
    __shared__ uint32_t sPrefix;
    __shared__ int sLeft;
    const int begin = a.n_first, end = q.tokens - a.n_recent;  // those in between are chosen from
    auto key_at = [&](int t) { return key_of(a.weights[((size_t)a.meta[q.src + (t >> 4)] * Hkv + h) * kPage + (t & 15)]); };

    // the key of the last one chosen, and how many of its equals are chosen
    uint32_t prefix = 0;
    int left = q.keep - a.n_first - a.n_recent;
    if (left > 0)
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < kChooseWaves * 256; i += kChooseThreads) (&sBins[0][0])[i] = 0;
            __syncthreads();
            for (int t = begin + tid; t < end; t += kChooseThreads) {
                const uint32_t k = key_at(t);
                if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&sBins[wave][k >> shift & 255], 1);
            }
            __syncthreads();
            if (tid < 256) {
                int n = 0;
                for (int w = 0; w < kChooseWaves; ++w) n += sBins[w][tid];
                sBins[0][tid] = n;
            }
            __syncthreads();
            if (wave == 0) {  // lane l: bins 255 - 4 l .. 252 - 4 l
                int n[4], total = 0;
                for (int i = 0; i < 4; ++i) total += n[i] = sBins[0][255 - 4 * lane - i];
                int above = total;
                for (int d = 1; d < 64; d <<= 1) {
                    const int x = __shfl_up(above, d);
                    if (lane >= d) above += x;
                }
                above -= total;
                for (int i = 0; i < 4; ++i) {
                    if (above < left && left <= above + n[i]) {
                        sPrefix = prefix | (uint32_t)(255 - 4 * lane - i) << shift;
                        sLeft = left - above;
                    }
                    above += n[i];
                }
            }
            __syncthreads();
            prefix = sPrefix;
            left = sLeft;
            __syncthreads();
        }

    int base = 0, equal_base = 0;
    for (int t0 = 0; t0 < q.tokens; t0 += kChooseThreads) {
        const int t = t0 + tid;
        const bool free = t >= begin && t < end;
        const uint32_t k = free && q.keep > a.n_first + a.n_recent ? key_at(t) : 0u;
        const bool same = free && left > 0 && k == prefix;
        const uint64_t equals = __ballot(same);
        if (lane == 0) sCount[0][wave] = __popcll(equals);
        __syncthreads();
        int rank = equal_base + __popcll(equals & ((1ull << lane) - 1)), all = 0;
        for (int w = 0; w < kChooseWaves; ++w) {
            if (w < wave) rank += sCount[0][w];
            all += sCount[0][w];
        }
        equal_base += all;
        const bool keep = t < q.tokens && (!free || (left > 0 && (k > prefix || (same && rank < left))));
        const uint64_t keeps = __ballot(keep);
        if (lane == 0) sCount[1][wave] = __popcll(keeps);
        __syncthreads();
        int at = base + __popcll(keeps & ((1ull << lane) - 1));
        all = 0;
        for (int w = 0; w < kChooseWaves; ++w) {
            if (w < wave) at += sCount[1][w];
            all += sCount[1][w];
        }
        base += all;
        if (keep && at < q.keep) kept[at] = t;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictLaunch a) {
    const int x = blockIdx.x, h = blockIdx.y, Hkv = a.pool.num_kv_heads, tid = threadIdx.x, lane = tid & 63;
    const EvictSequence *seq = reinterpret_cast<const EvictSequence *>(a.meta);
    int i = -1;  // the last sequence that begins at or before the block
    for (int s = 0; s < a.n_seq; s += 64) i += __popcll(__ballot(s + lane < a.n_seq && seq[min(s + lane, a.n_seq - 1)].unit <= x));
    const EvictSequence q = seq[i];
    const int j0 = (x - q.unit) * kPage, n = min(kPage, q.keep - j0), to = a.meta[q.dst + (x - q.unit)];
    const int slot = tid >> 4, c = tid & 15, d0 = 8 * c;
    const bool valid = slot < n;
    size_t from = 0;
    int fs = 0;
    if (valid) {
        const int t = a.kept[(size_t)h * a.total + q.kept + j0 + slot];
        from = (size_t)a.meta[q.src + (t >> 4)] * Hkv + h;
        fs = t & 15;
        if (c == 0) a.weights[((size_t)to * Hkv + h) * kPage + slot] = a.weights[from * kPage + fs];
    }
    const size_t src = from * kBlockElems, blk = ((size_t)to * Hkv + h) * kBlockElems;
    if constexpr (DT == 0) {
        u32x4 kw = {0u, 0u, 0u, 0u}, vw = {0u, 0u, 0u, 0u};
        if (valid) {
            kw = ld16(static_cast<const uint16_t *>(a.pool.k_pages) + src + (d0 >> 5) * 512 + fs * 32 + (d0 & 31));
            const uint16_t *v = static_cast<const uint16_t *>(a.pool.v_pages) + src + d0 * kPage + fs;
#pragma unroll
            for (int j = 0; j < 4; ++j) vw[j] = (uint32_t)v[2 * j * kPage] | (uint32_t)v[(2 * j + 1) * kPage] << 16;
        }
        const float none[8] = {};
        store_block<0>(a.pool, to, h, valid, kw, none, vw, 0, n);
    } else if constexpr (DT == 1) {
        __shared__ uint32_t sV[kPage][kHeadDim / 4 + 1];
        __shared__ float sRed[2][4];
        float kf[8] = {}, vf[8] = {}, ka = 0.f, va = 0.f;
        if (valid) {
            const float ks = a.pool.k_scale[from], vs = a.pool.v_scale[from];
            const u32x2 kw = *reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(a.pool.k_pages) + src + (d0 >> 6) * 1024 + fs * 64 + (d0 & 63));
            const uint8_t *v = static_cast<const uint8_t *>(a.pool.v_pages) + src + d0 * kPage + fs;
            u32x2 vw = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 8; ++j) vw[j >> 2] |= (uint32_t)v[j * kPage] << (8 * (j & 3));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const auto k0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)kw[j], false), k1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)kw[j], true);
                const auto v0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw[j], false), v1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vw[j], true);
                kf[4 * j] = k0[0] * ks, kf[4 * j + 1] = k0[1] * ks, kf[4 * j + 2] = k1[0] * ks, kf[4 * j + 3] = k1[1] * ks;
                vf[4 * j] = v0[0] * vs, vf[4 * j + 1] = v0[1] * vs, vf[4 * j + 2] = v1[0] * vs, vf[4 * j + 3] = v1[1] * vs;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                ka = fmaxf(ka, fabsf(kf[j]));
                va = fmaxf(va, fabsf(vf[j]));
            }
        }
        ka = wave_max(ka);
        va = wave_max(va);
        if (lane == 0) {
            sRed[0][tid >> 6] = ka;
            sRed[1][tid >> 6] = va;
        }
        __syncthreads();
        ka = fmaxf(fmaxf(sRed[0][0], sRed[0][1]), fmaxf(sRed[0][2], sRed[0][3]));
        va = fmaxf(fmaxf(sRed[1][0], sRed[1][1]), fmaxf(sRed[1][2], sRed[1][3]));
        const float ks = ka > 0.f ? ka / 448.0f : 1.0f, vs = va > 0.f ? va / 448.0f : 1.0f;
        if (tid == 0) {
            a.pool.k_scale[(size_t)to * Hkv + h] = ks;
            a.pool.v_scale[(size_t)to * Hkv + h] = vs;
        }
        if (valid) {
            *reinterpret_cast<u32x2 *>(static_cast<uint8_t *>(a.pool.k_pages) + blk + (d0 >> 6) * 1024 + slot * 64 + (d0 & 63)) =
                u32x2{quant4(kf[0], kf[1], kf[2], kf[3], ks), quant4(kf[4], kf[5], kf[6], kf[7], ks)};
            sV[slot][2 * c] = quant4(vf[0], vf[1], vf[2], vf[3], vs);
            sV[slot][2 * c + 1] = quant4(vf[4], vf[5], vf[6], vf[7], vs);
        }
        __syncthreads();
        // thread (dim, half): eight slots of a dimension
        const int d = tid >> 1, s0 = 8 * (tid & 1), sh = 8 * (d & 3);
        uint8_t *vd = static_cast<uint8_t *>(a.pool.v_pages) + blk + d * kPage + s0;
        if (s0 + 8 <= n) {
            u32x2 w = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j >> 2] |= (sV[s0 + j][d >> 2] >> sh & 255u) << (8 * (j & 3));
            *reinterpret_cast<u32x2 *>(vd) = w;
        } else {
            for (int j = 0; s0 + j < n; ++j) vd[j] = (uint8_t)(sV[s0 + j][d >> 2] >> sh);
        }
    } else if (valid) {
        const float *k = static_cast<const float *>(a.pool.k_pages) + src + (d0 >> 4) * 256 + fs * 16 + (d0 & 15);
        const float *v = static_cast<const float *>(a.pool.v_pages) + src + d0 * kPage + fs;
        float *kd = static_cast<float *>(a.pool.k_pages) + blk + (d0 >> 4) * 256 + slot * 16 + (d0 & 15);
        float *vd = static_cast<float *>(a.pool.v_pages) + blk + d0 * kPage + slot;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            kd[j] = k[j];
            vd[j * kPage] = v[j * kPage];
        }
    }
}

}  // namespace

hipError_t launch_evict(const EvictLaunch &a, hipStream_t s) {
    if (a.n_units <= 0) return hipSuccess;
    hipLaunchKernelGGL(evict_choose_kernel, dim3(a.n_seq, a.pool.num_kv_heads), dim3(kChooseThreads), 0, s, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const dim3 grid(a.n_units, a.pool.num_kv_heads), block(256);
    if (a.pool.dtype == 0)
        hipLaunchKernelGGL(evict_move_kernel<0>, grid, block, 0, s, a);
    else if (a.pool.dtype == 1)
        hipLaunchKernelGGL(evict_move_kernel<1>, grid, block, 0, s, a);
    else
        hipLaunchKernelGGL(evict_move_kernel<2>, grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace hkv
