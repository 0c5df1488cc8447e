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
// Bound by memory (per token and head of 128 columns: 512 bytes on the bf16 side, 140 on the 4-bit side).  K or V of one tile (64 tokens
// of one head) at a time: D threads, thread (c, w, t) takes the 8 columns 8c.. of the eight tokens 32w + 8i + 2t + e, which are
// exactly the tokens that share its words of V.  All 8 loads of a thread are issued before the first is used.  Groups are reduced
// among the lanes of a token by shuffles; the tile's image is put together in shared memory and leaves in 16-byte stores.
// A tile that the span covers in part keeps the other tokens' codes: its image is loaded first.
// 32K tokens of 4 heads of 128 columns, written and read back: 32.7 us for 171 MB, 5.2 TB/s, 0.80 of a copy's rate (issue slots 79 %
// busy in pack, 72 % in unpack), 33.8 back to back for seconds (1.89 GHz); with K and V of a tile in one CTA 36, seven ragged chunks of up to 2.5K tokens 7.9 and 15 (half as many
// CTAs, each twice as long); a scale computed by every lane, and fp32 values in unpack, 45.5.
//
// Single tokens (a decode step: one token per sequence) would move 9 KB each way for 140 bytes: they have kernels of their own, which write
// the token's K words and its nibble of every V word in place (64 tokens of 8 heads, both ways: 4.4 us, two launches).
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

// A group's smallest value and the negative of its largest, as bf16 in the low and high half of a word: one minimum serves both.
__device__ __forceinline__ uint32_t extremes(const uint4& x) {
    const uint32_t lo = min2(min2(x.x, x.y), min2(x.z, x.w)), hi = max2(max2(x.x, x.y), max2(x.z, x.w)) ^ 0x80008000u;
    return min2(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
}
// What a group's codes are made with: scale and zero as they are stored (low and high half), and 1 / (16 scale) (0: all codes are 0).
struct Group { uint32_t meta; float inverse16; };
__device__ __forceinline__ Group group_of(uint32_t ends) {
    const float zero = ptx::bf16_lo(ends), top = -ptx::bf16_hi(ends);
    Group g;
    g.meta = ptx::pack_bf16(__fdiv_rn(top - zero, 15.f), zero);
    const float scale = ptx::bf16_lo(g.meta);
    g.inverse16 = scale >= 0x1p-126f ? __frcp_rn(scale) * 0.0625f : 0.f;
    return g;
}
// Groups of eight tokens that LANES neighbouring lanes hold in parts, ends[k] of token k: lane c ends up with token (c & 7)'s whole
// extremes (each step halves the tokens a lane still carries), and computes that group's scale.  group_k() hands them out.
template <int LANES>
__device__ __forceinline__ Group own_group(uint32_t (&ends)[8], int c) {
#pragma unroll
    for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int k = 0; k < d; ++k) {
            const bool up = c & d;               // keeps tokens k + d, gives away k
            const uint32_t give = up ? ends[k] : ends[k + d], keep = up ? ends[k + d] : ends[k];
            ends[k] = min2(keep, __shfl_xor_sync(0xffffffffu, give, d));
        }
    uint32_t e = ends[0];
    if (LANES == 16) e = min2(e, __shfl_xor_sync(0xffffffffu, e, 8));
    return group_of(e);
}
__device__ __forceinline__ Group group_k(const Group& own, int lane, int k) {
    Group g;
    g.meta = __shfl_sync(0xffffffffu, own.meta, (lane & 24) | k);
    g.inverse16 = __shfl_sync(0xffffffffu, own.inverse16, (lane & 24) | k);
    return g;
}

// Two fp32 numbers as the operand of an instruction that does both.
__device__ __forceinline__ uint64_t two(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1,%2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
// What the codes of a group are made with, twice each.
struct Quotient { uint64_t minus_zero, inverse16, minus_scale16; float inverse; };
__device__ __forceinline__ Quotient quotient_of(const Group& g) {
    const float z = -ptx::bf16_hi(g.meta), s = -16.f * ptx::bf16_lo(g.meta);
    return Quotient{two(z, z), two(g.inverse16, g.inverse16), two(s, s), g.inverse16};
}
// The codes of two values in the low bits of words whose other bits are kMagic's.  Everything is done on a sixteenth of the code, so that
// the last multiply-add of the quotient can saturate to [0, 1]: a NaN becomes 0 there, and no value touches another one's code.  (All but
// that one for both values at once: 32.9 us for 32K tokens both ways, one value a time 34.0.)
__device__ __forceinline__ void two_codes(uint32_t x, const Quotient& g, uint32_t& a, uint32_t& b) {
    float r0, r1, t0, t1, q0, q1;
    asm("{.reg .b64 d, t, r; add.rn.f32x2 d, %4, %5; mul.rn.f32x2 t, d, %6; fma.rn.f32x2 r, t, %7, d; mov.b64 {%0,%1}, r; mov.b64 {%2,%3}, t;}"
        : "=f"(r0), "=f"(r1), "=f"(t0), "=f"(t1)
        : "l"(two(ptx::bf16_lo(x), ptx::bf16_hi(x))), "l"(g.minus_zero), "l"(g.inverse16), "l"(g.minus_scale16));
    asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(q0) : "f"(r0), "f"(g.inverse), "f"(t0));
    asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(q1) : "f"(r1), "f"(g.inverse), "f"(t1));
    asm("{.reg .b64 c; fma.rn.f32x2 c, %2, %3, %4; mov.b64 {%0,%1}, c;}"
        : "=r"(a), "=r"(b) : "l"(two(q0, q1)), "l"(two(16.f, 16.f)), "l"(two(kMagic, kMagic)));
}

// Two codes (bits 0..3 of either half of x) -> their two values, rounded to bf16 once: under the exponent of 128 the bits are 128 +
// code, the difference is exact, and scale * code + zero is one bf16 multiply-add.  meta2: {scale, scale}, {zero, zero}.
__device__ __forceinline__ uint32_t two_values(uint32_t x, const __nv_bfloat162& scale, const __nv_bfloat162& zero) {
    const uint32_t y = (x & 0x000f000fu) | 0x43004300u, bias = 0xc300c300u;
    const __nv_bfloat162 code = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&y), *reinterpret_cast<const __nv_bfloat162*>(&bias));
    const __nv_bfloat162 v = __hfma2(code, scale, zero);
    return *reinterpret_cast<const uint32_t*>(&v);
}
struct Meta2 { __nv_bfloat162 scale, zero; };
__device__ __forceinline__ Meta2 meta2(uint32_t meta) {
    const uint32_t s = __byte_perm(meta, meta, 0x1010), z = __byte_perm(meta, meta, 0x3232);
    return Meta2{*reinterpret_cast<const __nv_bfloat162*>(&s), *reinterpret_cast<const __nv_bfloat162*>(&z)};
}
// The eight values of a K word (nibble j is column j), in order.
__device__ __forceinline__ uint4 values_of_k(uint32_t w, uint32_t meta) {
    const Meta2 m = meta2(meta);
    const uint32_t v04 = two_values(w, m.scale, m.zero), v15 = two_values(w >> 4, m.scale, m.zero);
    const uint32_t v26 = two_values(w >> 8, m.scale, m.zero), v37 = two_values(w >> 12, m.scale, m.zero);
    return make_uint4(__byte_perm(v04, v15, 0x5410), __byte_perm(v26, v37, 0x5410), __byte_perm(v04, v15, 0x7632), __byte_perm(v26, v37, 0x7632));
}
// The values of one token in the V words of eight columns: nibble k of each.
__device__ __forceinline__ uint4 values_of_v(const uint32_t (&w)[8], int k, uint32_t meta) {
    const Meta2 m = meta2(meta);
    const uint32_t byte = k >> 1, sel = byte | (4u + byte) << 8;         // byte k/2 of either word into bytes 0 and 2 (what is in 1 and 3 is masked)
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = two_values(__byte_perm(w[2 * i], w[2 * i + 1], sel) >> (4 * (k & 1)), m.scale, m.zero);
    return make_uint4(v[0], v[1], v[2], v[3]);
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
    constexpr int kKWords = 8 * D + 64 * kPanels, kVWords = 8 * D + 64;          // of either half of a tile
    __shared__ uint4 s_image[kUnits][kKWords / 4];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int su = threadIdx.x / D, r = threadIdx.x % D, lane = threadIdx.x & 31;
    const int c = r % kLanes, wt = r / kLanes, w = wt >> 2, tt = wt & 3;
    const int64_t unit = int64_t(blockIdx.x) * kUnits + su;
    const bool is_v = unit & 1;
    const TileJob job = tile_job<D>(p, unit >> 1);
    uint32_t* image = reinterpret_cast<uint32_t*>(s_image[su]);
    uint4* const out = reinterpret_cast<uint4*>(job.image + (is_v ? 4 * kKWords : 0));
    const int n16 = (is_v ? kVWords : kKWords) / 4;
    const bool whole = job.live && job.first == 0 && job.end == kTileTokens;

    // token k = i + 4e of this thread: 32w + 8i + 2tt + e
    const int t0 = 32 * w + 2 * tt;
    auto token = [&](int k) { return t0 + 8 * (k & 3) + (k >> 2); };
    uint4 x[8];
    uint32_t in = 0;                             // which of the eight the span covers
    {
        const int64_t pitch = is_v ? p.v_token : p.k_token;
        const char* src = (is_v ? p.v : p.k) + (job.src + t0) * pitch + int64_t(job.head) * D * 2 + c * 16;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool there = token(k) >= job.first && token(k) < job.end;
            in |= there ? 1u << k : 0u;
            x[k] = there ? __ldcs(reinterpret_cast<const uint4*>(src + (8 * (k & 3) + (k >> 2)) * pitch)) : make_uint4(0, 0, 0, 0);
        }
    }
    if (job.live && !whole) {
        for (int i = r; i < n16; i += D) s_image[su][i] = out[i];
    }
    uint32_t ends[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) ends[k] = extremes(x[k]);
    const Group own = is_v ? own_group<kLanes>(ends, c) : own_group<8>(ends, c);
    __syncthreads();

    const int row0 = nibble_meta_row(t0);
    uint32_t words[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const Group g = group_k(own, lane, k);
        const Quotient quotient = quotient_of(g);
        const uint32_t xx[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
        const int row = row0 + 16 * ((k & 3) >> 1) + 2 * (k >> 2) + (k & 1);
        uint32_t bits[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) two_codes(xx[i], quotient, bits[2 * i], bits[2 * i + 1]);
        if (is_v) {
#pragma unroll
            for (int j = 0; j < 8; ++j) words[j] += bits[j] << (4 * k);
            if (c == 0 && (in >> k & 1)) image[8 * D + row] = g.meta;
        } else {
            uint32_t word = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) word += bits[j] << (4 * j);
            if (in >> k & 1) {
                image[nibble_k_word(kPanels, t0, c) + ((k & 3) >> 1) * kPanels * 128 + (k >> 2) * 16 + (k & 1) * 2] = word - kMagicSum;
                if ((c & 7) == 0) image[8 * D + row * kPanels + (c >> 3)] = g.meta;
            }
        }
    }
    if (is_v) {
        uint32_t covered = 0;                    // bits of the nibbles that the span writes
#pragma unroll
        for (int k = 0; k < 8; ++k) covered |= (in >> k & 1) ? 15u << (4 * k) : 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t& dst = image[nibble_v_word(8 * c, w, tt) + 16 * j];
            const uint32_t word = words[j] - kMagicSum;
            if (whole) dst = word;
            else if (covered) dst = (dst & ~covered) | (word & covered);
        }
    }
    __syncthreads();
    if (job.live)
        for (int i = r; i < n16; i += D) out[i] = s_image[su][i];
}

template <int D>
__global__ void __launch_bounds__(kThreads) nibble_unpack_kernel(const __grid_constant__ NibbleMove p) {
    constexpr int kLanes = D / 8, kUnits = kThreads / D, kPanels = D / 64;
    constexpr int kKWords = 8 * D + 64 * kPanels, kVWords = 8 * D + 64;
    __shared__ uint4 s_image[kUnits][kKWords / 4];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int su = threadIdx.x / D, r = threadIdx.x % D;
    const int c = r % kLanes, wt = r / kLanes, w = wt >> 2, tt = wt & 3;
    const int64_t unit = int64_t(blockIdx.x) * kUnits + su;
    const bool is_v = unit & 1;
    const TileJob job = tile_job<D>(p, unit >> 1);
    const uint32_t* image = reinterpret_cast<const uint32_t*>(s_image[su]);
    if (job.live) {
        const uint4* from = reinterpret_cast<const uint4*>(job.image + (is_v ? 4 * kKWords : 0));
        const int n16 = (is_v ? kVWords : kKWords) / 4;
#pragma unroll
        for (int i = 0; i < (kKWords / 4 + D - 1) / D; ++i)
            if (i * D + r < n16) s_image[su][i * D + r] = from[i * D + r];
    }
    __syncthreads();
    const int t0 = 32 * w + 2 * tt, row0 = nibble_meta_row(t0);
    const int64_t pitch = is_v ? p.v_token : p.k_token;
    char* dst = (is_v ? p.v : p.k) + (job.src + t0) * pitch + int64_t(job.head) * D * 2 + c * 16;
    uint32_t words[8];
    if (is_v) {
#pragma unroll
        for (int j = 0; j < 8; ++j) words[j] = image[nibble_v_word(8 * c, w, tt) + 16 * j];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int t = t0 + 8 * (k & 3) + (k >> 2), row = row0 + 16 * ((k & 3) >> 1) + 2 * (k >> 2) + (k & 1);
        if (t < job.first || t >= job.end) continue;
        const uint4 v = is_v ? values_of_v(words, k, image[8 * D + row])
                             : values_of_k(image[nibble_k_word(kPanels, t0, c) + ((k & 3) >> 1) * kPanels * 128 + (k >> 2) * 16 + (k & 1) * 2],
                                           image[8 * D + row * kPanels + (c >> 3)]);
        __stcs(reinterpret_cast<uint4*>(dst + (8 * (k & 3) + (k >> 2)) * pitch), v);
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
    uint32_t ke = extremes(kx), ve = extremes(vx);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) {
        ke = min2(ke, __shfl_xor_sync(0xffffffffu, ke, d));
        ve = min2(ve, __shfl_xor_sync(0xffffffffu, ve, d));
    }
    if (kLanes == 16) ve = min2(ve, __shfl_xor_sync(0xffffffffu, ve, 8));
    if (!job.live) return;
    const Group gk = group_of(ke), gv = group_of(ve);
    const Quotient kq = quotient_of(gk), vq = quotient_of(gv);
    const uint32_t x[4] = {kx.x, kx.y, kx.z, kx.w}, y[4] = {vx.x, vx.y, vx.z, vx.w};
    uint32_t word = 0;
    const int shift = 4 * nibble_v_of(job.t);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t a, b;
        two_codes(x[i], kq, a, b);
        word += (a << (8 * i)) + (b << (8 * i + 4));
        two_codes(y[i], vq, a, b);
        old[2 * i] = (old[2 * i] & ~(15u << shift)) | ((a & 15u) << shift);
        old[2 * i + 1] = (old[2 * i + 1] & ~(15u << shift)) | ((b & 15u) << shift);
    }
    job.image[nibble_k_word(kPanels, job.t, c)] = word - kMagicSum;
    if ((c & 7) == 0) job.image[kKMeta + nibble_meta_row(job.t) * kPanels + (c >> 3)] = gk.meta;
    if (c == 0) job.image[kVMeta + nibble_meta_row(job.t)] = gv.meta;
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
    uint32_t words[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) words[j] = job.image[kV + nibble_v_word(8 * c + j, job.t >> 5, (job.t & 7) >> 1)];
    *reinterpret_cast<uint4*>(p.k + job.src * p.k_token + at) = values_of_k(kw, km);
    *reinterpret_cast<uint4*>(p.v + job.src * p.v_token + at) = values_of_v(words, nibble_v_of(job.t), vm);
}

cudaError_t launch(const NibbleMove& a, bool single, void (*tile64)(NibbleMove), void (*tile128)(NibbleMove), void (*token64)(NibbleMove),
                   void (*token128)(NibbleMove), cudaStream_t s) {
    const bool wide = a.g.dim == 128;
    const int64_t units = int64_t(single ? a.n_spans : 2 * int64_t(a.n_tiles)) * a.g.n_kv_heads;     // K and V of a tile apart
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
