// Eviction: per sequence and KV head the heaviest tokens are chosen and moved, in order, to other blocks (kv_pool_evict).
//
// Choosing: the weights as integers in the order of the numbers, kept in registers; the k-th largest is found from its highest bits down by three
// histograms of 11 bits in LDS.  Then the tokens above it and as many of its equals as are left, lowest index first, written in order
// by counts over wavefronts.  One workgroup per (sequence, head); bound by the chain of its steps.
// Moving: one wavefront per (new block, head); 16 tokens come from 16 places.  K's dimensions lie in runs of 64 bytes a token, V's are
// 16 tokens wide, so that V is read in whole blocks however few of their tokens are kept.  A lane takes all 16 tokens of two of V's dimensions: its
// loads are on their way together, neighbouring lanes read neighbouring dimensions, and what it holds goes out as it lies in the
// block.  fp8 blocks get the scale of what they hold now and are rounded again, as a block written anew.
//
// The choice is bound by the chain of its steps: 2048 of 8190 tokens, 8 heads, 11 us (loads 3, a digit 1.3, places 2; digits of two bits by ballots
// took 36).  The move is bound by memory, V's whole blocks included: 32 sequences of 4096 tokens that keep 1000 (8 heads, fp8) 52 us, 235 MB of HBM traffic
// at 4.5 TB/s; 15 of 5907 that keep 2923 57 us, in bf16 119 us, 452 MB at 3.8 TB/s.
#include <type_traits>

#include "pool_block.h"

namespace hkv {

namespace {

constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64, kMaxRounds = 32;  // a round: a token a thread

__device__ __forceinline__ const int32_t *meta_of(const EvictLaunch &a) { return a.meta; }
__device__ __forceinline__ const int32_t *meta_of(const EvictInline &a) { return a.list; }

// Order of the weights as integers: both zeros equal, NaN below every number (no number has a key of kNaN or less, or kStays).
constexpr uint32_t kOutside = 0, kNaN = 1, kStays = 0xFFFFFFFFu;  // behind the last token; no number; among the first or the newest
__device__ __forceinline__ uint32_t key_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.0f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return kNaN;
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int ones_below(uint64_t ones) {  // how many lanes below this one have a one
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(ones >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)ones, 0));
}

// N: keys a thread keeps in registers (0: more tokens than that, the weights are read again for every step).
template <int N, class Args>
__global__ __launch_bounds__(kChooseThreads) void evict_choose_kernel(Args a) {
    const int32_t *const meta = meta_of(a);
    const EvictSequence q = reinterpret_cast<const EvictSequence *>(meta)[blockIdx.x];
    const int h = blockIdx.y, Hkv = a.pool.num_kv_heads, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int32_t *kept = a.kept + (size_t)h * a.total + q.kept;
    if (q.keep >= q.tokens) {
        for (int t = tid; t < q.tokens; t += kChooseThreads) kept[t] = t;
        return;
    }
    __shared__ int sBins[2 * kChooseThreads];
    __shared__ int sWave[kChooseWaves];
    __shared__ int sPick[3];  // the digit of the last one chosen, how many there are above it with the same digits before, and how many like it
    __shared__ int sRank[2][kMaxRounds * kChooseWaves + 1];  // by round and wavefront: tokens that are sure to stay, and equals of the last one
    const int begin = a.n_first, end = q.tokens - a.n_recent;  // those in between are chosen from
    const int rounds = (q.tokens + kChooseThreads - 1) / kChooseThreads;
    auto block_at = [&](int t) { return meta[q.src + (min(t, q.tokens - 1) >> 4)]; };
    auto weight_at = [&](int t, int block) { return a.weights[((size_t)block * Hkv + h) * kPage + (min(t, q.tokens - 1) & 15)]; };
    auto key_at = [&](int t, float w) { return t >= q.tokens ? kOutside : t < begin || t >= end ? kStays : key_of(w); };
    uint32_t keys[N > 0 ? N : 1];
    if constexpr (N > 0) {  // (all loads at once)
        int block[N];
        float w[N];
#pragma unroll
        for (int i = 0; i < N; ++i) block[i] = block_at(i * kChooseThreads + tid);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = weight_at(i * kChooseThreads + tid, block[i]);
#pragma unroll
        for (int i = 0; i < N; ++i) keys[i] = key_at(i * kChooseThreads + tid, w[i]);
    }
    auto each = [&](int from, int to, auto &&f) {  // f(round, key of this thread's token), for some rounds or, in registers, all
        if constexpr (N > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < rounds) f(i, keys[i]);
        } else {
            constexpr int kAtOnce = 8;
            for (int i0 = from; i0 < to; i0 += kAtOnce) {
                int block[kAtOnce];
                float w[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) block[i] = block_at((i0 + i) * kChooseThreads + tid);
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) w[i] = weight_at((i0 + i) * kChooseThreads + tid, block[i]);
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i)
                    if (i0 + i < to) f(i0 + i, key_at((i0 + i) * kChooseThreads + tid, w[i]));
            }
        }
    };
    // `last`: the key of the last one kept; `equals`: how many tokens of that key are kept, of `alike`.
    uint32_t last = kStays;
    int above = a.n_first + a.n_recent, alike = 0;
    if (above < q.keep) {
        last = 0;
        for (int shift = 21;; shift = shift == 21 ? 10 : 0) {
            const int bits = shift > 0 ? 11 : 10, top = 2 * kChooseThreads - 1 - 2 * tid;  // this thread's bins: top, top - 1
            sBins[top] = sBins[top - 1] = 0;
            __syncthreads();
            each(0, rounds, [&](int, uint32_t k) {
                if (shift == 21 ? k != kStays : k >> (shift + bits) == last >> (shift + bits)) atomicAdd(&sBins[k >> shift & ((1u << bits) - 1)], 1);
            });
            __syncthreads();
            const int n0 = sBins[top], n1 = sBins[top - 1];
            int x = n0 + n1;
            for (int d = 1; d < 64; d <<= 1) {
                const int y = __shfl_up(x, d);
                if (lane >= d) x += y;
            }
            if (lane == 63) sWave[wave] = x;
            __syncthreads();
            x -= n0 + n1;
#pragma unroll
            for (int w = 0; w < kChooseWaves; ++w)
                if (w < wave) x += sWave[w];
            const int want = q.keep - above;  // (fewer than there are tokens)
            if (x < want && want <= x + n0) {
                sPick[0] = top;
                sPick[1] = x;
                sPick[2] = n0;
            } else if (x + n0 < want && want <= x + n0 + n1) {
                sPick[0] = top - 1;
                sPick[1] = x + n0;
                sPick[2] = n1;
            }
            __syncthreads();
            last |= (uint32_t)sPick[0] << shift;
            above += sPick[1];
            alike = sPick[2];
            if (shift == 0) break;
        }
    }
    const int equals = last == kStays ? 0 : q.keep - above;
    const bool ties = equals < alike;  // (seldom: then the lowest indexes among the equals are found too)
    const uint32_t least = ties ? last + 1 : last;  // tokens of at least this key are sure to stay

    // Places: by round, wavefront and lane.
    uint64_t stay[N > 0 ? N : 1];
    int base[2] = {0, 0};
    for (int r0 = 0; r0 < rounds; r0 += kMaxRounds) {
        const int r1 = min(rounds, r0 + kMaxRounds), n_ranks = (r1 - r0) * kChooseWaves;
        each(r0, r1, [&](int i, uint32_t k) {
            const uint64_t s = __ballot(k >= least);
            if constexpr (N > 0) stay[i] = s;
            const int e = ties ? __popcll(__ballot(k == last)) : 0;
            if (lane == 0) {
                sRank[0][(i - r0) * kChooseWaves + wave] = __popcll(s);
                sRank[1][(i - r0) * kChooseWaves + wave] = e;
            }
        });
        __syncthreads();
        if (wave < (ties ? 2 : 1)) {  // running sums: of what is sure (wavefront 0) and of equals (1)
            int run = base[wave];
            for (int j = 0; j < n_ranks; j += 64) {
                const int n = j + lane < n_ranks ? sRank[wave][j + lane] : 0;
                int x = n;
                for (int d = 1; d < 64; d <<= 1) {
                    const int y = __shfl_up(x, d);
                    if (lane >= d) x += y;
                }
                if (j + lane < n_ranks) sRank[wave][j + lane] = run + x - n;
                run += __shfl(x, 63);
            }
            if (lane == 0) sRank[wave][n_ranks] = run;
        }
        __syncthreads();
        each(r0, r1, [&](int i, uint32_t k) {
            uint64_t s;
            if constexpr (N > 0)
                s = stay[i];
            else
                s = __ballot(k >= least);
            const int j = (i - r0) * kChooseWaves + wave;
            int at = sRank[0][j] + ones_below(s);
            bool stays = k >= least;
            if (ties) {
                const int rank = sRank[1][j] + ones_below(__ballot(k == last));
                at += min(equals, rank);
                stays |= k == last && rank < equals;
            }
            if (stays) kept[at] = i * kChooseThreads + tid;
        });
        base[0] = sRank[0][n_ranks];
        base[1] = sRank[1][n_ranks];
        __syncthreads();
    }
}

// Wavefronts go by head first: the blocks that neighbouring new blocks take tokens from are the same, and with 8 heads mostly on one XCD.
template <int DT, class Args>
__global__ __launch_bounds__(256) void evict_move_kernel(Args a) {
    using Elem = std::conditional_t<DT == 0, uint16_t, std::conditional_t<DT == 1, uint8_t, float>>;
    const int32_t *const meta = meta_of(a);
    const int Hkv = a.pool.num_kv_heads, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int x = blockIdx.x / Hkv * 4 + wave, h = blockIdx.x % Hkv;
    if (x >= a.n_units) return;
    const EvictSequence *seq = reinterpret_cast<const EvictSequence *>(meta);
    int i = -1;  // the last sequence that begins at or before the block
    for (int s = 0; s < a.n_seq; s += 64) i += __popcll(__ballot(s + lane < a.n_seq && seq[min(s + lane, a.n_seq - 1)].unit <= x));
    const EvictSequence q = seq[i];
    const int j0 = (x - q.unit) * kPage, n = min(kPage, q.keep - j0), to = meta[q.dst + (x - q.unit)];
    const int64_t out = (int64_t)to * Hkv + h;
    // lane s (and s + 16, ...) knows token s: its old block and slot; behind the last token: that one again
    const int token = a.kept[(size_t)h * a.total + q.kept + j0 + min(lane & 15, n - 1)];
    const int block = meta[q.src + (token >> 4)];
    Elem *const kb = static_cast<Elem *>(a.pool.k_pages), *const vb = static_cast<Elem *>(a.pool.v_pages);
    constexpr int C = 64 / sizeof(Elem), kChunks = kHeadDim / C;  // K: dimensions of a 64-byte piece
    // K: lane (token lane / 4, 16 bytes of it) of every piece
    const int kt = lane >> 2, k_block = __builtin_amdgcn_ds_bpermute(4 * kt, block), k_slot = __builtin_amdgcn_ds_bpermute(4 * kt, token) & 15;
    const int64_t k_from = (int64_t)k_block * Hkv + h;
    const char *ks = reinterpret_cast<const char *>(kb + k_from * kBlockElems) + 64 * k_slot + 16 * (lane & 3);
    u32x4 kw[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) kw[c] = ld16(ks + 1024 * c);
    Elem v[2][kPage];   // two dimensions of the tokens
    u32x4 codes[2] = {};  // fp8: those as 16 bytes each
    float vscale = 0.f;   // fp8: of the token that this lane knows
    if constexpr (DT == 1) {
        // Whole dimensions (16 bytes) of the old blocks, each block once, and bytes picked from them: 10 loads where 16 kept tokens lie in 5 blocks, in place of
        // 32.  The lanes know by selectors of v_perm which bytes go where: lane 8 u + 2 j + p has what half p of old block u gives
        // to word j of the new one.  Four blocks at once; eight at once cost as much, with 105 registers a lane in place of 94.
        vscale = a.pool.v_scale[(int64_t)block * Hkv + h];
        const int before = __builtin_amdgcn_ds_bpermute(4 * ((lane & 15) - 1), block);
        const uint32_t first = (uint32_t)__ballot((lane & 15) == 0 || block != before) & 0xFFFFu;  // tokens that begin another old block
        const int n_old = __popc(first), place = (__popc(first & ((2u << (lane & 15)) - 1)) - 1) << 4 | (token & 15);
        uint32_t rest = first;
        for (int u0 = 0; u0 < n_old; u0 += 4) {
            u32x4 x[4][2];
            auto load = [&](int u) {
                const int64_t from = (int64_t)__builtin_amdgcn_readlane(block, __builtin_ctz(rest)) * Hkv + h;
                if (rest & (rest - 1)) rest &= rest - 1;  // (the last one again behind it)
                x[u][0] = ld16(vb + from * kBlockElems + lane * kPage);
                x[u][1] = ld16(vb + from * kBlockElems + (lane + 64) * kPage);
            };
#pragma unroll
            for (int u = 0; u < 4; ++u) load(u);
            uint32_t pick = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int from = __builtin_amdgcn_ds_bpermute(4 * (4 * (lane >> 1 & 3) + e), place), to_u = from >> 4, slot = from & 15;
                pick |= (uint32_t)(to_u == u0 + (lane >> 3 & 3) && slot >> 3 == (lane & 1) ? slot & 7 : 0x0C) << (8 * e);
            }
            auto gather = [&](int u) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t lo = __builtin_amdgcn_readlane(pick, 8 * u + 2 * j), hi = __builtin_amdgcn_readlane(pick, 8 * u + 2 * j + 1);
#pragma unroll
                    for (int d = 0; d < 2; ++d)
                        codes[d][j] |= __builtin_amdgcn_perm(x[u][d][1], x[u][d][0], lo) | __builtin_amdgcn_perm(x[u][d][3], x[u][d][2], hi);
                }
            };
#pragma unroll
            for (int u = 0; u < 4; ++u) gather(u);
        }
    } else {
#pragma unroll
        for (int s = 0; s < kPage; ++s) {
            const Elem *p = vb + ((int64_t)__builtin_amdgcn_readlane(block, s) * Hkv + h) * kBlockElems + (__builtin_amdgcn_readlane(token, s) & 15);
            v[0][s] = p[lane * kPage];
            v[1][s] = p[(lane + 64) * kPage];
        }
    }
    const float weight = a.weights[((int64_t)block * Hkv + h) * kPage + (token & 15)];
    u32x4 vw[2][kPage * sizeof(Elem) / 16];  // what goes out: two dimensions, 16 slots each
    if constexpr (DT == 1) {
        const float kscale = a.pool.k_scale[k_from];
        float kf[kChunks][16], ka = 0.f, va = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)kw[c][j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)kw[c][j], true);
                kf[c][4 * j] = lo[0] * kscale, kf[c][4 * j + 1] = lo[1] * kscale, kf[c][4 * j + 2] = hi[0] * kscale, kf[c][4 * j + 3] = hi[1] * kscale;
#pragma unroll
                for (int e = 0; e < 4; ++e) ka = fmaxf(ka, fabsf(kf[c][4 * j + e]));
            }
        float vf[2][kPage];
        float vs[kPage];
#pragma unroll
        for (int s = 0; s < kPage; ++s) vs[s] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vscale), s));
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[d][j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[d][j], true);
                const float f[4] = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    vf[d][4 * j + e] = f[e] * vs[4 * j + e];
                    va = fmaxf(va, fabsf(vf[d][4 * j + e]));
                }
            }
        ka = wave_max(ka);  // (tokens taken again behind the last one do not change it)
        va = wave_max(va);
        const float kscale1 = ka > 0.f ? ka / 448.0f : 1.0f, vscale1 = va > 0.f ? va / 448.0f : 1.0f;
        if (lane == 0) {
            a.pool.k_scale[out] = kscale1;
            a.pool.v_scale[out] = vscale1;
        }
        const float ki = 1.0f / kscale1, vi = 1.0f / vscale1;
        auto encode = [&](auto &&four) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int c = 0; c < kChunks; ++c) kw[c][j] = four(kf[c] + 4 * j, kscale1, ki);
#pragma unroll
                for (int d = 0; d < 2; ++d) vw[d][0][j] = four(vf[d] + 4 * j, vscale1, vi);
            }
        };
        const float least = fminf(kscale1, vscale1), most = fmaxf(kscale1, vscale1);
        if (__builtin_amdgcn_readfirstlane(least >= 0x1p-60f && most <= 0x1p60f)) {
            // by the reciprocal and a correction, a third of the division's instructions; the quotient is the division's but for its last bit now and then
            encode([](const float *x, float sc, float inv) { return quant4_by(x[0], x[1], x[2], x[3], sc, inv); });
        } else {
            encode([](const float *x, float sc, float) { return quant4(x[0], x[1], x[2], x[3], sc); });
        }
    } else {
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int j = 0; j < (int)(kPage * sizeof(Elem) / 4); ++j) {
                if constexpr (DT == 0)
                    vw[d][j >> 2][j & 3] = (uint32_t)v[d][2 * j] | (uint32_t)v[d][2 * j + 1] << 16;
                else
                    vw[d][j >> 2][j & 3] = __float_as_uint(v[d][j]);
            }
    }
    if (lane < n) a.weights[out * kPage + lane] = weight;
    if (kt < n) {
        char *kd = reinterpret_cast<char *>(kb + out * kBlockElems) + 64 * kt + 16 * (lane & 3);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) *reinterpret_cast<u32x4 *>(kd + 1024 * c) = kw[c];
    }
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        Elem *vd = vb + out * kBlockElems + (lane + 64 * d) * kPage;
        if (n == kPage) {
#pragma unroll
            for (int j = 0; j < (int)(kPage * sizeof(Elem) / 16); ++j) reinterpret_cast<u32x4 *>(vd)[j] = vw[d][j];
        } else {
            constexpr int E = sizeof(Elem);
#pragma unroll
            for (int s = 0; s < kPage; ++s)
                if (s < n) {
                    const uint32_t w = vw[d][s * E / 16][s * E / 4 % 4] >> (8 * (s * E % 4));
                    if constexpr (DT == 2)
                        vd[s] = __uint_as_float(w);
                    else
                        vd[s] = (Elem)w;
                }
        }
    }
}

}  // namespace

namespace {
template <class Args>
hipError_t go(const Args &a, hipStream_t s) {
    const int Hkv = a.pool.num_kv_heads, rounds = (a.most_tokens + kChooseThreads - 1) / kChooseThreads;
    auto choose = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.n_seq, Hkv), dim3(kChooseThreads), 0, s, a); };
    if (rounds <= 2)
        choose(evict_choose_kernel<2, Args>);
    else if (rounds <= 4)
        choose(evict_choose_kernel<4, Args>);
    else if (rounds <= 8)
        choose(evict_choose_kernel<8, Args>);
    else if (rounds <= 16)
        choose(evict_choose_kernel<16, Args>);
    else
        choose(evict_choose_kernel<0, Args>);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    auto move = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)((a.n_units + 3) / 4) * Hkv), dim3(256), 0, s, a); };
    if (a.pool.dtype == 0)
        move(evict_move_kernel<0, Args>);
    else if (a.pool.dtype == 1)
        move(evict_move_kernel<1, Args>);
    else
        move(evict_move_kernel<2, Args>);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_evict(const EvictLaunch &a, hipStream_t s) { return a.n_units <= 0 ? hipSuccess : go(a, s); }
hipError_t launch_evict(const EvictInline &a, hipStream_t s) { return a.n_units <= 0 ? hipSuccess : go(a, s); }

}  // namespace hkv
