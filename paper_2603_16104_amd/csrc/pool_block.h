// Device code of the writers of pool blocks (bf16 and fp8 pools): a block's tokens, eight dimensions a thread, into the block
// format, and the fp8 scales and codes.
#pragma once

#include "hkv_device.h"

namespace hkv {

__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp<kQuadXor1>(v));
    v = fmaxf(v, dpp<kQuadXor2>(v));
    v = fmaxf(v, dpp<kRor4>(v));
    v = fmaxf(v, dpp<kRor8>(v));
    return rows_max(v);
}

__device__ __forceinline__ uint32_t quant4(float a, float b, float c, float d, float scale) {
    auto q = [scale](float x) { return fminf(fmaxf(x / scale, -448.0f), 448.0f); };
    int p = 0;
    p = __builtin_amdgcn_cvt_pk_fp8_f32(q(a), q(b), p, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(q(c), q(d), p, true);
    return (uint32_t)p;
}

// Four codes under an old scale, rounded again under a new one: value * old / scale.
__device__ __forceinline__ uint32_t requant4(uint32_t w, float old, float scale) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return quant4(lo[0] * old, lo[1] * old, hi[0] * old, hi[1] * old, scale);
}

// Codes as quant4's for bf16 values x and a scale of amax / 448 of such values, |x| <= amax, from the scale's reciprocal
// (correctly rounded): product, remainder, correction.  For every such pair with a scale in [2^-60, 2^60] (5.3e8 pairs, all
// of them tried) the quotient equals the division's bit for bit wherever it is at least 2^-11 in magnitude; below 2^-10
// both round to zero with the sign of x.  Four instructions instead of about ten, two of them slow ones.  For other values (keys before
// their rounding to bf16, codes times a scale) the quotient is the division's but for its last bit now and then, and a code another one only where the quotient
// lies between two of them to within that bit.
__device__ __forceinline__ uint32_t quant4_by(float a, float b, float c, float d, float scale, float inv) {
    auto q = [scale, inv](float x) {
        const float y = x * inv;
        const float z = __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-y, scale, x), inv, y), x);
        return fminf(fmaxf(z, -448.0f), 448.0f);
    };
    int p = 0;
    p = __builtin_amdgcn_cvt_pk_fp8_f32(q(a), q(b), p, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(q(c), q(d), p, true);
    return (uint32_t)p;
}

// Eight bf16 of a 16-byte piece.
__device__ __forceinline__ void unpack_bf16(u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
}

// Slots s_lo .. s_hi - 1 of block `page`, KV head h, by a workgroup of 256 threads: thread (slot = tid / 16, d0 = 8 * (tid % 16)) brings
// its slot's dims d0 .. d0 + 7 if the slot is one of them (valid): K as bf16 bits (kw, bf16 pools) or as floats (kf, fp8 pools), V as bf16
// bits.  Threads of other slots bring zeros.
template <int DT>
__device__ __forceinline__ void store_block(const PoolWriteLaunch &a, const int page, const int h, const bool valid, const u32x4 kw, const float (&kf)[8],
                                            const u32x4 vw, const int s_lo, const int s_hi) {
    __shared__ uint16_t sV[kPage][kHeadDim + 8];
    __shared__ float sRed[2][4];
    __shared__ float sScale[2], sOld[2], sInv[2];

    const int tid = threadIdx.x;
    const int slot = tid >> 4, d0 = (tid & 15) * 8;
    const size_t blk = ((size_t)page * a.num_kv_heads + h) * kBlockElems;
    *reinterpret_cast<u32x4 *>(&sV[slot][d0]) = vw;

    if (DT == 0) {
        if (valid) {
            uint16_t *kdst = static_cast<uint16_t *>(a.k_pages) + blk + (d0 >> 5) * (kPage * 32) + slot * 32 + (d0 & 31);
            *reinterpret_cast<u32x4 *>(kdst) = kw;
        }
        __syncthreads();
        const int d = tid >> 1, half = tid & 1;
        uint16_t *vdst = static_cast<uint16_t *>(a.v_pages) + blk + d * kPage + half * 8;
        if (s_lo <= half * 8 && s_hi >= half * 8 + 8) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = (uint32_t)sV[half * 8 + 2 * j][d] | ((uint32_t)sV[half * 8 + 2 * j + 1][d] << 16);
            *reinterpret_cast<u32x4 *>(vdst) = w;
        } else {
            for (int j = 0; j < 8; ++j) {
                const int sl = half * 8 + j;
                if (sl >= s_lo && sl < s_hi) vdst[j] = sV[sl][d];
            }
        }
    } else {
        float vf[8];
        float ka = 0.f, va = 0.f;
        unpack_bf16(vw, vf);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            ka = fmaxf(ka, fabsf(kf[j]));
            va = fmaxf(va, fabsf(vf[j]));
        }
        ka = wave_max(ka);
        va = wave_max(va);
        if ((tid & 63) == 0) {
            sRed[0][tid >> 6] = ka;
            sRed[1][tid >> 6] = va;
        }
        __syncthreads();
        const bool append = s_lo > 0;  // slots below s_lo of this block hold codes of an earlier call
        if (tid < 2) {
            const float am = fmaxf(fmaxf(sRed[tid][0], sRed[tid][1]), fmaxf(sRed[tid][2], sRed[tid][3]));
            float *scales = tid ? a.v_scale : a.k_scale;
            float sc, old = 0.f;
            if (!append) {
                sc = am > 0.f ? am / 448.0f : 1.0f;
            } else {
                old = scales[(size_t)page * a.num_kv_heads + h];
                const float cand = am > 0.f ? am / 448.0f : 0.f;
                sc = old >= cand ? old : cand;  // an unset (NaN) old scale gives cand
                if (!(sc > 0.f)) sc = 1.0f;
            }
            sScale[tid] = sc;
            sOld[tid] = old;
            sInv[tid] = !append && sc >= 0x1p-60f && sc <= 0x1p60f ? 1.0f / sc : 0.f;  // 0: divide
            scales[(size_t)page * a.num_kv_heads + h] = sc;
        }
        __syncthreads();
        const float ksc = sScale[0], vsc = sScale[1], kinv = sInv[0], vinv = sInv[1];
        auto encode = [](const float (&x)[8], float sc, float inv) {
            u32x2 c;
            if (inv != 0.f) {  // the same for the whole workgroup
                c[0] = quant4_by(x[0], x[1], x[2], x[3], sc, inv);
                c[1] = quant4_by(x[4], x[5], x[6], x[7], sc, inv);
            } else {
                c[0] = quant4(x[0], x[1], x[2], x[3], sc);
                c[1] = quant4(x[4], x[5], x[6], x[7], sc);
            }
            return c;
        };
        const bool k_grew = append && ksc > sOld[0], v_grew = append && vsc > sOld[1];
        if (k_grew && slot < s_lo) {
            uint8_t *kdst = static_cast<uint8_t *>(a.k_pages) + blk + (d0 >> 6) * (kPage * 64) + slot * 64 + (d0 & 63);
            u32x2 c = *reinterpret_cast<u32x2 *>(kdst);
            c[0] = requant4(c[0], sOld[0], ksc);
            c[1] = requant4(c[1], sOld[0], ksc);
            *reinterpret_cast<u32x2 *>(kdst) = c;
        }
        if (valid) {
            const u32x2 c = encode(kf, ksc, kinv);
            uint8_t *kdst = static_cast<uint8_t *>(a.k_pages) + blk + (d0 >> 6) * (kPage * 64) + slot * 64 + (d0 & 63);
            *reinterpret_cast<u32x2 *>(kdst) = c;
        }
        const int d = tid >> 1, half = tid & 1;
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = bf16_bits_to_float(sV[half * 8 + j][d]);
        const u32x2 c = encode(x, vsc, vinv);
        uint8_t *vdst = static_cast<uint8_t *>(a.v_pages) + blk + d * kPage + half * 8;
        if (s_lo <= half * 8 && s_hi >= half * 8 + 8) {
            *reinterpret_cast<u32x2 *>(vdst) = c;
        } else {
            u32x2 r = {0u, 0u};  // the earlier codes of these eight slots, re-encoded if the scale grew
            if (v_grew && half * 8 < s_lo) {
                r = *reinterpret_cast<u32x2 *>(vdst);
                r[0] = requant4(r[0], sOld[1], vsc);
                r[1] = requant4(r[1], sOld[1], vsc);
            }
            for (int j = 0; j < 8; ++j) {
                const int sl = half * 8 + j;
                if (sl >= s_lo && sl < s_hi)
                    vdst[j] = (uint8_t)(c[j >> 2] >> (8 * (j & 3)));
                else if (v_grew && sl < s_lo)
                    vdst[j] = (uint8_t)(r[j >> 2] >> (8 * (j & 3)));
            }
        }
    }
}

}  // namespace hkv
