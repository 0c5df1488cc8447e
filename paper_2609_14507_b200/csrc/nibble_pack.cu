// Token-major bf16 K/V -> 4-bit blocks and back (format: nibble.cuh).
//
// Per group of values (K: 64 columns of a token and head, V: all of them):
//   zero = min x, scale = bf16((max x - min x) / 15), code = min(round_half_even((x - zero) / scale), 15), in fp32.
// The quotient has to be the rounded one (ties are frequent: x, zero and scale are bf16, so (x - zero) / scale falls exactly
// between two codes once in a few hundred values), and a division per value would make the kernel arithmetic-bound.  So
// the group's reciprocal r = 1/scale is divided once and every quotient is q = d r corrected by its own residual,
// q + (d - q scale) r with fused multiply-adds: Markstein's theorem (IBM J. Res. Dev. 34, 1990) gives the rounded
// quotient from a rounded reciprocal.  Adding 1.5 * 2^23 then leaves the code in the low bits of the sum.
//
// Bound by memory (per token and head of 128 columns: 512 bytes on the bf16 side, 140 on the 4-bit side).  One tile (64 tokens of one head)
// at a time: D threads, thread (c, w, t) takes the 8 columns 8c.. of the eight tokens 32w + 8i + 2t + e, which are exactly
// the tokens that share its words of V.  All 16 loads of a thread are issued before the first is used.  Groups are reduced
// among the lanes of a token by shuffles; the tile's image is put together in shared memory and leaves in 16-byte stores.
// A tile that the span covers in part keeps the other tokens' codes: its image is loaded first.
//
// Single tokens (a decode step: one token per sequence) would move 9 KB each way for 140 bytes: they have kernels of their own, which write
// the token's K words and its nibble of every V word in place.
#include <cuda_bf16.h>

#include "launch.cuh"
#include "ops.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kThreads = 128;
constexpr float kMagic = 12582912.f;             // 1.5 * 2^23: x + kMagic holds round_half_even(x) in its low mantissa bits
constexpr uint32_t kMagicSum = 0x3f400000u;      // sum over j of the bits of kMagic shifted left by 4j, modulo 2^32

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

struct Group { float zero, scale, inverse; };

// Zero, scale and reciprocal of a group that lies in LANES neighbouring lanes, eight values each.
template <int LANES>
__device__ __forceinline__ Group group_of(const uint4& x) {
    uint32_t lo = min2(min2(x.x, x.y), min2(x.z, x.w)), hi = max2(max2(x.x, x.y), max2(x.z, x.w));
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) {
        lo = min2(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max2(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    Group g;
    g.zero = fminf(ptx::bf16_lo(lo), ptx::bf16_hi(lo));
    const float top = fmaxf(ptx::bf16_lo(hi), ptx::bf16_hi(hi));
    g.scale = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(top - g.zero, 15.f)));
    g.inverse = g.scale >= 0x1p-126f ? __frcp_rn(g.scale) : 0.f;
    return g;
}
__device__ __forceinline__ uint32_t meta_of(const Group& g) { return ptx::pack_bf16(g.scale, g.zero); }

// The code of a value in the low bits of a word whose other bits are kMagic's.
__device__ __forceinline__ uint32_t code_bits(float x, const Group& g) {
    const float d = __fsub_rn(x, g.zero);
    const float t = __fmul_rn(d, g.inverse);
    const float q = __fmaf_rn(__fmaf_rn(-t, g.scale, d), g.inverse, t);
    return __float_as_uint(__fadd_rn(fminf(q, 15.f), kMagic));
}
__device__ __forceinline__ float value_of(uint32_t code, uint32_t meta) {
    return __fmaf_rn(ptx::bf16_lo(meta), float(code), ptx::bf16_hi(meta));
}

// The span of a tile of the launch.
__device__ __forceinline__ int span_of(const NibbleMove& p, int tile) {
    int lo = 0, hi = p.n_spans - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.span[mid].tile0 <= tile) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// What a tile's threads know about it.
struct TileJob {
    char* image;                 // in the cache
    int64_t src;                 // token-major row of the tile's token 0 (may lie before the span)
    int first, end;              // tokens of the tile that the span covers: [first, end)
    int head;
    bool live;
};
template <int D>
__device__ __forceinline__ TileJob tile_job(const NibbleMove& p, int64_t unit) {
    TileJob j;
    j.live = unit < int64_t(p.n_tiles) * p.g.n_kv_heads;
    if (!j.live) { j.image = nullptr; j.src = 0; j.first = j.end = j.head = 0; return j; }
    const int tile = int(unit / p.g.n_kv_heads);
    j.head = int(unit - int64_t(tile) * p.g.n_kv_heads);
    const NibbleSpanArg& sp = p.span[span_of(p, tile)];
    const int64_t in_run = sp.first / kTileTokens + (tile - sp.tile0);
    const int64_t t0 = in_run * kTileTokens;
    j.image = sp.blocks + p.g.tile_off(in_run, j.head);
    j.src = sp.src + (t0 - sp.first);
    j.first = t0 < sp.first ? int(sp.first - t0) : 0;
    const int64_t left = sp.first + sp.n - t0;
    j.end = left < kTileTokens ? int(left) : kTileTokens;
    return j;
}

template <int D>
__global__ void __launch_bounds__(kThreads) nibble_pack_kernel(const __grid_constant__ NibbleMove p) {
    constexpr int kLanes = D / 8, kUnits = kThreads / D, kPanels = D / 64;
    constexpr int kWords = (64 * D + 256 * (kPanels + 1)) / 4, kKMeta = 8 * D, kV = kKMeta + 64 * kPanels, kVMeta = kV + 8 * D;
    __shared__ uint4 s_image[kUnits][kWords / 4];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int su = threadIdx.x / D, r = threadIdx.x % D;
    const int c = r % kLanes, wt = r / kLanes, w = wt >> 2, tt = wt & 3;
    const TileJob job = tile_job<D>(p, int64_t(blockIdx.x) * kUnits + su);
    uint32_t* image = reinterpret_cast<uint32_t*>(s_image[su]);
    const bool whole = job.live && job.first == 0 && job.end == kTileTokens;

    uint4 kx[8], vx[8];
    const int64_t at = int64_t(job.head) * D * 2 + c * 16;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int t = 32 * w + 8 * (k & 3) + 2 * tt + (k >> 2);
        const bool in = t >= job.first && t < job.end;
        kx[k] = in ? __ldcs(reinterpret_cast<const uint4*>(p.k + (job.src + t) * p.k_token + at)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int t = 32 * w + 8 * (k & 3) + 2 * tt + (k >> 2);
        const bool in = t >= job.first && t < job.end;
        vx[k] = in ? __ldcs(reinterpret_cast<const uint4*>(p.v + (job.src + t) * p.v_token + at)) : make_uint4(0, 0, 0, 0);
    }
    if (job.live && !whole)
        for (int i = r; i < kWords / 4; i += D) s_image[su][i] = reinterpret_cast<const uint4*>(job.image)[i];
    __syncthreads();

    uint32_t covered = 0;                        // bits of the nibbles of this thread's V words that the span writes
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int t = 32 * w + 8 * (k & 3) + 2 * tt + (k >> 2);
        const bool in = t >= job.first && t < job.end;
        covered |= in ? 15u << (4 * k) : 0u;
        const Group g = group_of<8>(kx[k]);
        const uint32_t x[4] = {kx[k].x, kx[k].y, kx[k].z, kx[k].w};
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            word += code_bits(ptx::bf16_lo(x[i]), g) << (8 * i);
            word += code_bits(ptx::bf16_hi(x[i]), g) << (8 * i + 4);
        }
        if (in) {
            image[nibble_k_word(kPanels, t, c)] = word - kMagicSum;
            if ((c & 7) == 0) image[kKMeta + nibble_meta_row(t) * kPanels + (c >> 3)] = meta_of(g);
        }
    }
    uint32_t words[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int t = 32 * w + 8 * (k & 3) + 2 * tt + (k >> 2);
        const Group g = group_of<kLanes>(vx[k]);
        const uint32_t x[4] = {vx[k].x, vx[k].y, vx[k].z, vx[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            words[2 * i] += code_bits(ptx::bf16_lo(x[i]), g) << (4 * k);
            words[2 * i + 1] += code_bits(ptx::bf16_hi(x[i]), g) << (4 * k);
        }
        if (c == 0 && t >= job.first && t < job.end) image[kVMeta + nibble_meta_row(t)] = meta_of(g);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t& dst = image[kV + nibble_v_word(8 * c + j, w, tt)];
        const uint32_t word = words[j] - kMagicSum;
        if (whole) dst = word;
        else if (covered) dst = (dst & ~covered) | (word & covered);
    }
    __syncthreads();
    if (job.live)
        for (int i = r; i < kWords / 4; i += D) reinterpret_cast<uint4*>(job.image)[i] = s_image[su][i];
}

template <int D>
__global__ void __launch_bounds__(kThreads) nibble_unpack_kernel(const __grid_constant__ NibbleMove p) {
    constexpr int kLanes = D / 8, kUnits = kThreads / D, kPanels = D / 64;
    constexpr int kWords = (64 * D + 256 * (kPanels + 1)) / 4, kKMeta = 8 * D, kV = kKMeta + 64 * kPanels, kVMeta = kV + 8 * D;
    __shared__ uint4 s_image[kUnits][kWords / 4];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int su = threadIdx.x / D, r = threadIdx.x % D;
    const int c = r % kLanes, wt = r / kLanes, w = wt >> 2, tt = wt & 3;
    const TileJob job = tile_job<D>(p, int64_t(blockIdx.x) * kUnits + su);
    const uint32_t* image = reinterpret_cast<const uint32_t*>(s_image[su]);
    if (job.live) {
#pragma unroll
        for (int i = 0; i < (kWords / 4 + D - 1) / D; ++i)
            if (i * D + r < kWords / 4) s_image[su][i * D + r] = reinterpret_cast<const uint4*>(job.image)[i * D + r];
    }
    __syncthreads();
    uint32_t words[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) words[j] = image[kV + nibble_v_word(8 * c + j, w, tt)];
    const int64_t at = int64_t(job.head) * D * 2 + c * 16;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int t = 32 * w + 8 * (k & 3) + 2 * tt + (k >> 2);
        if (t < job.first || t >= job.end) continue;
        const uint32_t kw = image[nibble_k_word(kPanels, t, c)], km = image[kKMeta + nibble_meta_row(t) * kPanels + (c >> 3)];
        const uint32_t vm = image[kVMeta + nibble_meta_row(t)];
        uint32_t ko[4], vo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ko[i] = ptx::pack_bf16(value_of((kw >> (8 * i)) & 15u, km), value_of((kw >> (8 * i + 4)) & 15u, km));
            vo[i] = ptx::pack_bf16(value_of((words[2 * i] >> (4 * k)) & 15u, vm), value_of((words[2 * i + 1] >> (4 * k)) & 15u, vm));
        }
        __stcs(reinterpret_cast<uint4*>(p.k + (job.src + t) * p.k_token + at), make_uint4(ko[0], ko[1], ko[2], ko[3]));
        __stcs(reinterpret_cast<uint4*>(p.v + (job.src + t) * p.v_token + at), make_uint4(vo[0], vo[1], vo[2], vo[3]));
    }
}

// Where a single token's words are: D/8 lanes per (span, head).
struct TokenJob { uint32_t* image; int64_t src; int head, t; bool live; };
template <int D>
__device__ __forceinline__ TokenJob token_job(const NibbleMove& p, int64_t unit) {
    TokenJob j;
    j.live = unit < int64_t(p.n_spans) * p.g.n_kv_heads;
    if (!j.live) { j.image = nullptr; j.src = 0; j.head = j.t = 0; return j; }
    const int i = int(unit / p.g.n_kv_heads);
    j.head = int(unit - int64_t(i) * p.g.n_kv_heads);
    const NibbleSpanArg& sp = p.span[i];
    j.image = reinterpret_cast<uint32_t*>(sp.blocks + p.g.tile_off(sp.first / kTileTokens, j.head));
    j.src = sp.src;
    j.t = int(sp.first % kTileTokens);
    return j;
}

template <int D>
__global__ void __launch_bounds__(kThreads) nibble_pack_token_kernel(const __grid_constant__ NibbleMove p) {
    constexpr int kLanes = D / 8, kPanels = D / 64, kKMeta = 8 * D, kV = kKMeta + 64 * kPanels, kVMeta = kV + 8 * D;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int c = threadIdx.x % kLanes;
    const TokenJob job = token_job<D>(p, int64_t(blockIdx.x) * (kThreads / kLanes) + threadIdx.x / kLanes);
    const int64_t at = int64_t(job.head) * D * 2 + c * 16;
    uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
    uint32_t old[8];
    if (job.live) {
        kx = *reinterpret_cast<const uint4*>(p.k + job.src * p.k_token + at);
        vx = *reinterpret_cast<const uint4*>(p.v + job.src * p.v_token + at);
#pragma unroll
        for (int j = 0; j < 8; ++j) old[j] = job.image[kV + nibble_v_word(8 * c + j, job.t >> 5, (job.t & 7) >> 1)];
    }
    const Group gk = group_of<8>(kx), gv = group_of<kLanes>(vx);
    if (!job.live) return;
    const uint32_t x[4] = {kx.x, kx.y, kx.z, kx.w}, y[4] = {vx.x, vx.y, vx.z, vx.w};
    uint32_t word = 0;
    const int shift = 4 * nibble_v_of(job.t);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        word += code_bits(ptx::bf16_lo(x[i]), gk) << (8 * i);
        word += code_bits(ptx::bf16_hi(x[i]), gk) << (8 * i + 4);
        const uint32_t a = code_bits(ptx::bf16_lo(y[i]), gv) & 15u, b = code_bits(ptx::bf16_hi(y[i]), gv) & 15u;
        old[2 * i] = (old[2 * i] & ~(15u << shift)) | (a << shift);
        old[2 * i + 1] = (old[2 * i + 1] & ~(15u << shift)) | (b << shift);
    }
    job.image[nibble_k_word(kPanels, job.t, c)] = word - kMagicSum;
    if ((c & 7) == 0) job.image[kKMeta + nibble_meta_row(job.t) * kPanels + (c >> 3)] = meta_of(gk);
    if (c == 0) job.image[kVMeta + nibble_meta_row(job.t)] = meta_of(gv);
#pragma unroll
    for (int j = 0; j < 8; ++j) job.image[kV + nibble_v_word(8 * c + j, job.t >> 5, (job.t & 7) >> 1)] = old[j];
}

template <int D>
__global__ void __launch_bounds__(kThreads) nibble_unpack_token_kernel(const __grid_constant__ NibbleMove p) {
    constexpr int kLanes = D / 8, kPanels = D / 64, kKMeta = 8 * D, kV = kKMeta + 64 * kPanels, kVMeta = kV + 8 * D;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int c = threadIdx.x % kLanes;
    const TokenJob job = token_job<D>(p, int64_t(blockIdx.x) * (kThreads / kLanes) + threadIdx.x / kLanes);
    if (!job.live) return;
    const int64_t at = int64_t(job.head) * D * 2 + c * 16;
    const uint32_t kw = job.image[nibble_k_word(kPanels, job.t, c)], km = job.image[kKMeta + nibble_meta_row(job.t) * kPanels + (c >> 3)];
    const uint32_t vm = job.image[kVMeta + nibble_meta_row(job.t)];
    uint32_t words[8], ko[4], vo[4];
#pragma unroll
    for (int j = 0; j < 8; ++j) words[j] = job.image[kV + nibble_v_word(8 * c + j, job.t >> 5, (job.t & 7) >> 1)] >> (4 * nibble_v_of(job.t));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ko[i] = ptx::pack_bf16(value_of((kw >> (8 * i)) & 15u, km), value_of((kw >> (8 * i + 4)) & 15u, km));
        vo[i] = ptx::pack_bf16(value_of(words[2 * i] & 15u, vm), value_of(words[2 * i + 1] & 15u, vm));
    }
    *reinterpret_cast<uint4*>(p.k + job.src * p.k_token + at) = make_uint4(ko[0], ko[1], ko[2], ko[3]);
    *reinterpret_cast<uint4*>(p.v + job.src * p.v_token + at) = make_uint4(vo[0], vo[1], vo[2], vo[3]);
}

cudaError_t launch(const NibbleMove& a, bool single, void (*tile64)(NibbleMove), void (*tile128)(NibbleMove), void (*token64)(NibbleMove),
                   void (*token128)(NibbleMove), cudaStream_t s) {
    const bool wide = a.g.dim == 128;
    const int64_t units = int64_t(single ? a.n_spans : a.n_tiles) * a.g.n_kv_heads;
    const int per_cta = single ? kThreads / (a.g.dim / 8) : kThreads / a.g.dim;
    const int64_t grid = (units + per_cta - 1) / per_cta;
    if (grid > INT32_MAX) return cudaErrorInvalidValue;
    auto kernel = single ? (wide ? token128 : token64) : (wide ? tile128 : tile64);
    return launch_overlapped(kernel, int(grid), kThreads, size_t(0), s, a);
}

}  // namespace

cudaError_t launch_nibble_pack(const NibbleMove& a, bool single_tokens, cudaStream_t s) {
    return launch(a, single_tokens, nibble_pack_kernel<64>, nibble_pack_kernel<128>, nibble_pack_token_kernel<64>, nibble_pack_token_kernel<128>, s);
}
cudaError_t launch_nibble_unpack(const NibbleMove& a, bool single_tokens, cudaStream_t s) {
    return launch(a, single_tokens, nibble_unpack_kernel<64>, nibble_unpack_kernel<128>, nibble_unpack_token_kernel<64>,
                  nibble_unpack_token_kernel<128>, s);
}

}  // namespace ipkvi
