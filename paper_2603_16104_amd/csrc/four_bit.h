// Device code of 4-bit pools (HKV_FP4_E2M1): e2m1 codes, and for each 32 dimensions of a token one scale, a power of two held as its
// exponent + 127 in a byte (the block format of the gfx950 matrix instructions and conversions).
//
// A (16-token block, KV head) block holds 1024 bytes of codes and 64 of scales, K and V each.  With lane = 16 g + m of a wavefront:
//   K codes   byte (t % 4) * 256 + (t / 4) * 64 + d / 2: over four blocks lane (m, g) finds dims 32 g .. 32 g + 31 of tokens 4 m .. 4 m + 3, one
//             operand of a matrix instruction (one scale) per 16-byte load;
//   V codes   byte (t / 4) * 256 + (d / 8) * 16 + (t % 4) * 4 + d % 8 / 2: lane (m, g) finds dims 8 m .. 8 m + 7 of four tokens of block g in one load,
//             eight dims of one group of 32, so that the scales of a block's 16 tokens that it needs are 16 bytes in a row;
//   scales    byte (d / 32) * 16 + t.
// The even dimension is the low half of a byte.  No byte holds two tokens, so a token's store touches nothing of the others.
#pragma once

#include "hkv_device.h"

namespace hkv {

namespace four {

constexpr int kCodeBytes = kBlockElems / 2, kScaleBytes = kPage * kHeadDim / 32;  // of a block and head

// 2^(b - 127) of scale byte `i` of a word (b is 1 .. 252 in what the writers leave).
__device__ __forceinline__ float scale_of(uint32_t w, int i) { return __uint_as_float(__builtin_amdgcn_ubfe(w, 8 * i, 8) << 23); }

// Codes 2 B, 2 B + 1 of a word times a scale, as two bf16 (exact).
template <int B>
__device__ __forceinline__ uint32_t widen2(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
__device__ __forceinline__ u32x4 widen8(uint32_t w, float scale) {
    return u32x4{widen2<0>(w, scale), widen2<1>(w, scale), widen2<2>(w, scale), widen2<3>(w, scale)};
}

// The scale's exponent for 32 values whose largest magnitude is top: floor(log2(top)) - 2, which brings it into [4, 8) (6 is the largest
// code's value), between 2^-126 and 2^125, so that code times scale is finite and normal or zero.
__device__ __forceinline__ int exponent_of(float top) { return min(max((int)(__float_as_uint(top) >> 23 & 0xFFu) - 129, -126), 125); }
// Eight values (dims of one group) as codes: x / 2^e, to nearest, ties to the even code, beyond 6 to 6; a NaN becomes 6 or -6.
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// Dims 8 c .. 8 c + 7 of one token of K or V, by the lane that holds them; the four lanes of a group of 32 are neighbours (c = lane % 16), all of
// them active.  `store`: whether this lane's token is one that goes in.
__device__ __forceinline__ void put8(uint8_t *codes, uint8_t *scales, bool v, size_t blk, int t, int c, const float (&x)[8], bool store) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[j]));
    top = fmaxf(top, dpp<kQuadXor1>(top));
    top = fmaxf(top, dpp<kQuadXor2>(top));
    const int e = exponent_of(top);
    const uint32_t w = encode8(x, __uint_as_float((uint32_t)(e + 127) << 23));
    if (!store) return;
    *reinterpret_cast<uint32_t *>(codes + blk * kCodeBytes + (v ? (t >> 2) * 256 + c * 16 + (t & 3) * 4 : (t & 3) * 256 + (t >> 2) * 64 + c * 4)) = w;
    if ((c & 3) == 0) scales[blk * kScaleBytes + (c >> 2) * 16 + t] = (uint8_t)(e + 127);
}

__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
}

}  // namespace four

}  // namespace hkv
