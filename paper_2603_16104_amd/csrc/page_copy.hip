// Copies of pool blocks, within a pool or from one pool to another of any type.  (Section 5, "Proactive Cache Management": what is kept in GPU memory is
// blocks; they go to new owners, closer together, or into fewer bytes and back.)
//
// Same type: bytes, 16 per thread and load, four loads in front of the first store, all with the streaming hint: 134 MB to other pages of a bf16
// pool 49 us, 5.5 TB/s read and written; 55 us without the hint, 67 with eight loads, 50 with two.
// Other type: a workgroup per (block, head) takes the values through fp32, sources of 8 bits and more with the streaming hint (67 MB of bf16 to 4 bits
// 29 us, without the hint 36; back 24; four heads per workgroup take the same time).  Where both formats keep V dimension-major (all but 4 bits), a thread holds
// eight tokens of a dim; into and out of 4 bits, whose V is by tokens, V passes through LDS once.
#include "four_bit.h"
#include "pool_block.h"

namespace hkv {

namespace {

// entry i of the list: source block, target block, tokens (1 .. 16)
struct Entry {
    int32_t src, dst, tokens;
};

constexpr int kPieces = 4;  // of 16 bytes, a thread's
// n16 pieces from piece `first` on, as many as a workgroup copies.
__device__ __forceinline__ void copy_pieces(const char *src, char *dst, int first, int n16) {
    u32x4 w[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const int i = first + (int)threadIdx.x + 256 * j;
        if (i < n16) w[j] = ld16_stream(src + 16 * (size_t)i);
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const int i = first + (int)threadIdx.x + 256 * j;
        if (i < n16) __builtin_nontemporal_store(w[j], reinterpret_cast<u32x4 *>(dst + 16 * (size_t)i));
    }
}

// Workgroup (entry, K or V, slice of 256 kPieces pieces of the block's heads).
__device__ __forceinline__ void copy_block(const PageCopyLaunch &a, const Entry e, const int which, const int slice) {
    const int block_bytes = a.src.num_kv_heads * (kBlockElems / 8) * a.bits;
    const char *src = static_cast<const char *>(which ? a.src.v_pages : a.src.k_pages) + (size_t)e.src * block_bytes;
    char *dst = static_cast<char *>(const_cast<void *>(which ? a.dst.v_pages : a.dst.k_pages)) + (size_t)e.dst * block_bytes;
    copy_pieces(src, dst, slice * 256 * kPieces, block_bytes / 16);
    if (a.scale_words > 0 && slice == 0) {  // of a block: fp8 a word per head, 4 bits 16
        const int n = a.scale_words * a.src.num_kv_heads;
        const uint32_t *s = reinterpret_cast<const uint32_t *>(which ? a.src.v_scale : a.src.k_scale) + (size_t)e.src * n;
        uint32_t *d = reinterpret_cast<uint32_t *>(const_cast<float *>(which ? a.dst.v_scale : a.dst.k_scale)) + (size_t)e.dst * n;
        for (int i = threadIdx.x; i < n; i += 256) d[i] = s[i];
    }
}

// ---- values of a block by thread.  By rows: dims 8 c .. 8 c + 7 of token t (c = tid % 16, t = tid / 16).  By dims: tokens 8 half .. + 7 of
// dim d (half = tid % 2, d = tid / 2), V of all types but 4 bits.
template <int DT>
__device__ __forceinline__ void load8(const void *base, size_t at, float scale, float (&x)[8]) {  // eight neighbouring elements
    if constexpr (DT == 0) {
        unpack_bf16(ld16_stream(static_cast<const uint16_t *>(base) + at), x);
    } else if constexpr (DT == 1) {
        const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(static_cast<const uint8_t *>(base) + at));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
            x[4 * j] = lo[0] * scale;
            x[4 * j + 1] = lo[1] * scale;
            x[4 * j + 2] = hi[0] * scale;
            x[4 * j + 3] = hi[1] * scale;
        }
    } else {
        const f32x4 *p = reinterpret_cast<const f32x4 *>(static_cast<const float *>(base) + at);
        const f32x4 a = __builtin_nontemporal_load(p), b = __builtin_nontemporal_load(p + 1);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = a[j];
            x[4 + j] = b[j];
        }
    }
}
// `n` of the eight (by dims, at the end of what a page holds) or all of them.
template <int DT>
__device__ __forceinline__ void store8(void *base, size_t at, float scale, const float (&x)[8], int n) {
    if (n <= 0) return;
    if constexpr (DT == 0) {
        uint16_t *p = static_cast<uint16_t *>(base) + at;
        const u32x4 w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
        if (n >= 8)
            *reinterpret_cast<u32x4 *>(p) = w;
        else
            for (int j = 0; j < n; ++j) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    } else if constexpr (DT == 1) {
        uint8_t *p = static_cast<uint8_t *>(base) + at;
        const u32x2 w = {quant4(x[0], x[1], x[2], x[3], scale), quant4(x[4], x[5], x[6], x[7], scale)};
        if (n >= 8)
            *reinterpret_cast<u32x2 *>(p) = w;
        else
            for (int j = 0; j < n; ++j) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    } else {
        float *p = static_cast<float *>(base) + at;
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = x[j];
    }
}
template <int DT>
__device__ __forceinline__ size_t k_at(int t, int c) {  // element (t, 8 c) of a K block in 64-byte chunks
    constexpr int C = DT == 0 ? 32 : DT == 1 ? 64 : 16;
    return (size_t)(8 * c / C * kPage * C + t * C + 8 * c % C);
}
__device__ __forceinline__ void load_four(const PoolView &p, bool v, size_t blk, int t, int c, float (&x)[8]) {
    const uint8_t *codes = static_cast<const uint8_t *>(v ? p.v_pages : p.k_pages) + blk * four::kCodeBytes;
    const uint8_t *scales = reinterpret_cast<const uint8_t *>(v ? p.v_scale : p.k_scale) + blk * four::kScaleBytes;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + (v ? (t >> 2) * 256 + c * 16 + (t & 3) * 4 : (t & 3) * 256 + (t >> 2) * 64 + c * 4));
    four::unpack8(four::widen8(w, four::scale_of(scales[(c >> 2) * 16 + t], 0)), x);
}

// The scale of an fp8 block from its values: the largest of 256 threads' eight over 448.
__device__ __forceinline__ float block_scale(const float (&x)[8], float *red) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[j]));
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    return top > 0.f ? top / 448.0f : 1.0f;
}

template <int SRC, int DST>
__device__ __forceinline__ void convert_block(const PageCopyLaunch &a, const Entry e, const int h) {
    constexpr bool kTurn = (SRC == kDtypeFp4) != (DST == kDtypeFp4);  // V by dims on one side, by rows on the other
    __shared__ float sV[kTurn ? kPage : 1][kHeadDim + 4];
    __shared__ float sRed[2][4];
    const int tid = threadIdx.x, t = tid >> 4, c = tid & 15, d = tid >> 1, half = tid & 1;
    const size_t sb = (size_t)e.src * a.src.num_kv_heads + h, db = (size_t)e.dst * a.src.num_kv_heads + h;
    float k[8], v[8];
    if constexpr (SRC == kDtypeFp4) {
        load_four(a.src, false, sb, t, c, k);
        load_four(a.src, true, sb, t, c, v);
    } else {
        load8<SRC>(a.src.k_pages, sb * kBlockElems + k_at<SRC>(t, c), SRC == 1 ? a.src.k_scale[sb] : 1.f, k);
        load8<SRC>(a.src.v_pages, sb * kBlockElems + d * kPage + 8 * half, SRC == 1 ? a.src.v_scale[sb] : 1.f, v);
    }
    const bool in = t < e.tokens;
    // tokens behind the last one may hold anything: they count for no scale
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (!in) k[j] = 0.f;
        if (SRC == kDtypeFp4 ? !in : 8 * half + j >= e.tokens) v[j] = 0.f;
    }
    if constexpr (kTurn) {
        if constexpr (SRC == kDtypeFp4) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) *reinterpret_cast<f32x4 *>(&sV[t][8 * c + j]) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = sV[8 * half + j][d];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) sV[8 * half + j][d] = v[j];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = sV[t][8 * c + j];
        }
    }
    if constexpr (DST == kDtypeFp4) {
        four::put8(static_cast<uint8_t *>(const_cast<void *>(a.dst.k_pages)), reinterpret_cast<uint8_t *>(const_cast<float *>(a.dst.k_scale)), false, db, t, c, k, in);
        four::put8(static_cast<uint8_t *>(const_cast<void *>(a.dst.v_pages)), reinterpret_cast<uint8_t *>(const_cast<float *>(a.dst.v_scale)), true, db, t, c, v, in);
    } else {
        float ks = 1.f, vs = 1.f;
        if constexpr (DST == 1) {
            ks = block_scale(k, sRed[0]);
            vs = block_scale(v, sRed[1]);
            if (tid == 0) {
                const_cast<float *>(a.dst.k_scale)[db] = ks;
                const_cast<float *>(a.dst.v_scale)[db] = vs;
            }
        }
        store8<DST>(const_cast<void *>(a.dst.k_pages), db * kBlockElems + k_at<DST>(t, c), ks, k, in ? 8 : 0);
        store8<DST>(const_cast<void *>(a.dst.v_pages), db * kBlockElems + d * kPage + 8 * half, vs, v, e.tokens - 8 * half);
    }
}

__device__ __forceinline__ Entry entry_of(const int32_t *list, int i) { return Entry{list[3 * i], list[3 * i + 1], list[3 * i + 2]}; }

__global__ __launch_bounds__(256) void page_copy_kernel(PageCopyLaunch a) {
    copy_block(a, entry_of(a.list, blockIdx.x), blockIdx.y & 1, blockIdx.y >> 1);
}
__global__ __launch_bounds__(256) void page_copy_inline_kernel(PageCopyInline a) {
    copy_block(a, entry_of(a.entries, blockIdx.x), blockIdx.y & 1, blockIdx.y >> 1);
}
template <int SRC, int DST>
__global__ __launch_bounds__(256) void page_convert_kernel(PageCopyLaunch a) {
    convert_block<SRC, DST>(a, entry_of(a.list, blockIdx.x), blockIdx.y);
}
template <int SRC, int DST>
__global__ __launch_bounds__(256) void page_convert_inline_kernel(PageCopyInline a) {
    convert_block<SRC, DST>(a, entry_of(a.entries, blockIdx.x), blockIdx.y);
}

template <int SRC, int DST, typename A>
void go_convert(const A &a, hipStream_t s) {
    const dim3 grid(a.n, a.src.num_kv_heads);
    if constexpr (std::is_same_v<A, PageCopyInline>)
        hipLaunchKernelGGL((page_convert_inline_kernel<SRC, DST>), grid, dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((page_convert_kernel<SRC, DST>), grid, dim3(256), 0, s, a);
}
template <int SRC, typename A>
void go_from(const A &a, hipStream_t s) {
    if constexpr (SRC != 0)
        if (a.dst.dtype == 0) go_convert<SRC, 0>(a, s);
    if constexpr (SRC != 1)
        if (a.dst.dtype == 1) go_convert<SRC, 1>(a, s);
    if constexpr (SRC != 2)
        if (a.dst.dtype == 2) go_convert<SRC, 2>(a, s);
    if constexpr (SRC != kDtypeFp4)
        if (a.dst.dtype == kDtypeFp4) go_convert<SRC, kDtypeFp4>(a, s);
}

template <typename A>
hipError_t go(const A &launch, hipStream_t s) {
    if (launch.n <= 0) return hipSuccess;
    if (launch.src.num_kv_heads != launch.dst.num_kv_heads) return hipErrorInvalidValue;
    A a = launch;
    if (a.src.dtype == a.dst.dtype) {
        a.bits = a.src.dtype == 0 ? 16 : a.src.dtype == 1 ? 8 : a.src.dtype == 2 ? 32 : 4;
        a.scale_words = a.src.dtype == 1 ? 1 : a.src.dtype == kDtypeFp4 ? four::kScaleBytes / 4 : 0;
        const int64_t bytes = (int64_t)a.src.num_kv_heads * (kBlockElems / 8) * a.bits;
        const dim3 grid(a.n, 2 * (unsigned)((bytes + 4096 * kPieces - 1) / (4096 * kPieces)));
        if constexpr (std::is_same_v<A, PageCopyInline>)
            hipLaunchKernelGGL(page_copy_inline_kernel, grid, dim3(256), 0, s, a);
        else
            hipLaunchKernelGGL(page_copy_kernel, grid, dim3(256), 0, s, a);
        return hipGetLastError();
    }
    switch (a.src.dtype) {
        case 0: go_from<0>(a, s); break;
        case 1: go_from<1>(a, s); break;
        case 2: go_from<2>(a, s); break;
        default: go_from<kDtypeFp4>(a, s); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_page_copy(const PageCopyLaunch &a, hipStream_t s) { return go(a, s); }
hipError_t launch_page_copy(const PageCopyInline &a, hipStream_t s) { return go(a, s); }

}  // namespace hkv
