// Decode attention over a cache held in 4 bits (format: nibble.cuh): one query per row, partial output and log-sum-exp.
//
// With key = sk * code + zk per 64-column panel and value = sv * code + zv per token,
//   q . key = sum over panels of sk (q . codes) + zk sum(q),      O = sum_t (p_t sv_t) codes_t + sum_t p_t zv_t,
// so the tensor cores multiply the bare codes and the scales are applied to scores and weights, one value per token instead
// of one per element.  Codes become 16-bit operands as they lie in the word, by a mask (nibble.cuh): below the smallest normal
// number the bits of a bf16 (fp16) number are the number times 2^133 (2^24), so a code that a mask leaves in place is the code times a
// power of two, exactly, and the powers of two go into the other operand.  The zeros' share of the scores is a product of its own,
// over panels times terms of sum(q), and cheaper there than as multiply-adds.
//
// Tokens are the rows (M = 16) of the score product and columns of the head the rows of the output product; 8 query heads
// are the columns (N = 8): no row of a product is wasted on a missing head, and codes are never the operand that would have
// to be moved between lanes.  Scores come out as [token][head]; movmatrix turns the weights, two 16-bit rows at a time,
// into the [token][head] operand of the second product.
//
// Exactness.  q (bf16) times a power of two per head is exact; products are exact and sums are fp32.  A weight p sv is
// held as two fp16 numbers, head and remainder (22 bits): with at most 4 query heads per KV head they share one product (columns
// 0-3 and 4-7), otherwise there are two.  The remainder is held times 2^11: a head that is cut at fp16's smallest step, 2^-24, leaves its
// digits to a remainder that is cut at 2^-35.  (Without the factor both were cut at 2^-24: half of the tokens with weights of 2^-16 had
// lost ten digits.)  sv is brought near 1 by a power of two for each head of a warp, so that fp16's range is spent on p.  It follows the
// largest scale among tokens that count for the head (with the largest of all, one token of no weight whose values were 2^20 times the
// others' took all but seven of their digits) and leaves room for 2^4: a first token that outweighs the next by 2^12 and has no values would
// have every tile behind it look again.  So a weight p is known to 22 bits or 2^-34 of the reference's, whichever is coarser.
// The tensor cores add with two bits more than fp32 has and round towards zero, both counted from the largest exponent that
// an operand's FORMAT shows (a subnormal counts as the smallest normal number).  Two things follow.  The codes must fill the
// subnormal range: K's do in place as bf16 (7 bits of mantissa; bits 0..3 and 4..7), V's are shifted up to bits 3..6 and 7..10 of fp16,
// in place they lost up to six bits of their products.  And the sums over tokens must not be much larger than the result:
// codes are never negative, but an output is a mean of many values of either sign, so a sum of p sv code would exceed it by
// 2.5 sqrt(tokens); every other token enters complemented, code = 15 - (15 - code): the complement costs nothing in the mask, its
// weight is negative, 15 sv joins zv, and the excesses of the two halves meet in the same product (and in either half of its
// 16 tokens: with tokens 0-7 plain and 8-15 complemented the cut was one-sided, 4.2e-6 of the output at 1M tokens, now 9.5e-7).
// Remainders have sums of their own: added to the heads' they would be cut at the heads' exponent.  Without all this the output of
// 32K tokens was off by 5e-4 of itself; it is off by less than 1e-6 (a computation in fp32: 4e-7 to 1.5e-6).
//
// One warp works on one tile (64 tokens of a KV head) at a time, alone: its online softmax has its own reference maximum, raised
// only when a score exceeds it by 2^8 (then everything is rescaled), which costs one vote per tile in place of a reduction over lanes.  A
// producer warp streams tiles (one bulk copy each, they are contiguous) into a ring of stages on mbarriers; the warps of a CTA
// take them in turn.  At the end of a (row, head group) every warp writes its partial and goes on, and a second kernel joins the partials
// in a fixed order; where one CTA has the whole group (WHOLE: short sequences) it does that itself.  (Joining a CTA's warps through shared memory first made each wait for the slowest: ragged 64 192 us, now 175
// with that change alone.)  How rows and heads are shared out among CTAs: ops.h.
// More than 8 query heads per KV head: they make octets, one octet to a warp.  An even number of octets goes by twos or fours, whose warps are
// a team on one tile; other numbers of octets, and what is more than one group, read the tile once for each group (ops.h).
// Every wait is bounded; a warp whose wait ran out does no more work.
//
// Bound by instruction issue, then by the copies: a product of 16 x 8 x 16 keeps its quarter of an SM busy for eight cycles, and a tile of
// 128 columns takes 68 of them (4 query heads per KV head) or 100, beside 750 to 900 other instructions; the tiles of three
// CTAs with four such warps and 73 KB of ring each are under way on an SM (fewer or larger CTAs: 3 to 15 % slower).  Measured, 128 columns,
// back to back for seconds (in brackets: a few calls, before the board reaches its power limit and leaves 1965 MHz):
// 64 ragged rows of up to 24K tokens, 8 KV heads of 4 query heads: 190 us at 1.67 GHz (163) for 932 MB, 4.9 TB/s (5.7), 0.75 of a copy's
// rate (0.87); 16 rows of 32K, 4 KV heads of 8: 69 us at 1.75 GHz (61.5), 4.3 TB/s (4.8); one of 1M, 16 query heads on one KV head
// (every tile unpacked by two warps): 62 us, 2.3 TB/s; one of 4K: 8.4 us, two launches of which neither does much.
#include <cuda_fp16.h>

#include "kernels.h"
#include "launch.cuh"
#include "ops.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kWarps = kNibbleWarps;
constexpr int kThreads = (kWarps + 1) * 32;
constexpr int kPartRows = 8 * kWarps;            // partials of a CTA's teams: a row per head and team
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRaise = 8.f;                    // the reference maximum is raised when a score exceeds it by this (log2)
// Partials of a (row, head) above which its join is cut into slabs of 32 columns by 256 and by 512 threads.  Under 64 one CTA a head is
// better (16 rows of 32K tokens, 32 partials: 61.9 us in all, with slabs 65.4; 4 rows of 50K, 60 partials: 49 and 59), over 256 more
// threads are (one row of 1M, 888 partials: 61.2 and 66.9 with 256 threads; one of 64K, 148 partials: 21.9 and 19.2).
constexpr int kManyParts = 64, kVeryManyParts = 256;
constexpr int kRoom = 4;                         // scales this many powers of two above the largest that counted need no other factor
constexpr float kRest = 2048.f;                  // a weight's remainder is held times this
constexpr uint32_t kLowK = 0x000f000fu, kHighK = 0x00f000f0u;       // K codes as bf16 in bits 0..3 and 4..7: times 2^-133 and 2^-129
constexpr uint32_t kLow = 0x00780078u, kHigh = 0x07800780u;         // V codes as fp16 in bits 3..6 and 7..10: times 2^-21 and 2^-17

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16_k8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(b0));
}
// Two fp32 operations in one instruction, each rounded as if alone.
__device__ __forceinline__ float2 mul2(float a0, float a1, float b0, float b1) {
    float2 r;
    asm("{.reg .b64 p, q; mov.b64 p, {%2,%3}; mov.b64 q, {%4,%5}; mul.rn.f32x2 p, p, q; mov.b64 {%0,%1}, p;}"
        : "=f"(r.x), "=f"(r.y) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
    return r;
}
__device__ __forceinline__ void add2(float& a, float& b, float x, float y) {
    asm("{.reg .b64 p, q; mov.b64 p, {%0,%1}; mov.b64 q, {%2,%3}; add.rn.f32x2 p, p, q; mov.b64 {%0,%1}, p;}" : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}
__device__ __forceinline__ float2 fma2(float a0, float a1, float b0, float b1, float c0, float c1) {
    float2 r;
    asm("{.reg .b64 p, q, s; mov.b64 p, {%2,%3}; mov.b64 q, {%4,%5}; mov.b64 s, {%6,%7}; fma.rn.f32x2 p, p, q, s; mov.b64 {%0,%1}, p;}"
        : "=f"(r.x), "=f"(r.y) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
    return r;
}
// (a ^ b) & c and (a ^ ~b) & c
__device__ __forceinline__ uint32_t differ(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0x28;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t agree(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0x82;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

// All warps that compute (the one that copies has left).
__device__ __forceinline__ void consumers_meet() { asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory"); }

using Smem = NibbleSmem;

// The tables: launch parameters, or device memory when they are too large.  (Both are indexed where they are: a pointer to one or the
// other would take the address of a launch parameter.)
__device__ __forceinline__ NibbleRowArg row_at(const NibbleAttend& p, int i) { return p.rows ? p.rows[i] : p.row[i]; }
__device__ __forceinline__ NibbleRunArg run_at(const NibbleAttend& p, int i) { return p.runs ? p.runs[i] : p.run[i]; }

// A CTA's walk over (row, head group) pairs: the pair, and which of its tiles are the CTA's.
struct Pair {
    NibbleRowArg r;
    int row, kv, part;           // row, KV head, and which part of its query heads
    int tile0, n;                // the CTA's tiles of it (none where only units of its cost are in the CTA's chunk)
    int units, slot;             // units of the chunk that belong to it; where its partials go
};
__device__ __forceinline__ void set_pair(const NibbleAttend& p, Pair& x, int gh) {
    x.kv = p.groups_per_kv == 1 ? gh : gh / p.groups_per_kv;
    x.part = gh - x.kv * p.groups_per_kv;
}
// The tiles of units [first, first + x.units) of a pair: its cost comes first.
__device__ __forceinline__ void set_tiles(Pair& x, int first) {
    x.tile0 = max(first - kNibblePairCost, 0);
    x.n = max(first + x.units - kNibblePairCost, 0) - x.tile0;
}
template <bool WHOLE>
__device__ __forceinline__ Pair pair_at(const NibbleAttend& p, int u, int u1) {
    if (WHOLE) {                                 // a CTA for every pair, those without tiles too; u is the CTA
        Pair x;
        x.row = u / p.n_gh;
        x.r = row_at(p, x.row);
        set_pair(p, x, u - x.row * p.n_gh);
        x.tile0 = 0; x.n = x.r.tiles; x.units = 1; x.slot = 0;
        return x;
    }
    int lo = 0, hi = p.n_rows - 1;
    while (lo < hi) {                            // the last row that begins at or before u (rows without tiles lie in front of it)
        const int mid = (lo + hi + 1) >> 1;
        if (row_at(p, mid).first <= u) lo = mid; else hi = mid - 1;
    }
    Pair x;
    x.r = row_at(p, lo);
    x.row = lo;
    if (p.share > 0) {                           // whole CTAs to every pair, u is the CTA
        const int ctas = (x.r.tiles + p.share - 1) / p.share, gh = (u - x.r.first) / ctas, piece = u - x.r.first - gh * ctas;
        set_pair(p, x, gh);
        x.tile0 = int(int64_t(x.r.tiles) * piece / ctas);
        x.n = int(int64_t(x.r.tiles) * (piece + 1) / ctas) - x.tile0;
        x.units = 1;
        x.slot = u;
        return x;
    }
    const int all = x.r.tiles + kNibblePairCost, gh = (u - x.r.first) / all, first = u - x.r.first - gh * all;
    set_pair(p, x, gh);
    x.units = min(all - first, u1 - u);
    set_tiles(x, first);
    x.slot = int(blockIdx.x) + x.r.pair0 + gh;
    return x;
}
// The next pair of the chunk, u its first unit.
__device__ __forceinline__ void next_pair(const NibbleAttend& p, Pair& x, int u, int u1) {
    ++x.slot;
    if (++x.part == p.groups_per_kv) {
        x.part = 0;
        if (++x.kv == p.g.n_kv_heads) {
            x.kv = 0;
            do x.r = row_at(p, ++x.row); while (x.r.tiles == 0);
        }
    }
    x.units = min(x.r.tiles + kNibblePairCost, u1 - u);
    set_tiles(x, 0);
}

// HALF: at most 4 query heads per KV head.  WHOLE: one CTA to every pair, which writes the result.
template <int D, bool HALF, bool WHOLE>
__global__ void __launch_bounds__(kThreads, kNibbleCtasPerSm) nibble_attend_kernel(const __grid_constant__ NibbleAttend p) {
    constexpr int P = D / 64;
    constexpr int kTile = 64 * D + 256 * (P + 1), kKMeta = 32 * D, kV = kKMeta + 256 * P, kVMeta = kV + 32 * D;
    extern __shared__ unsigned char smem_dyn[];
    unsigned char* ring = smem_dyn + ((128u - (ptx::smem_addr(smem_dyn) & 127u)) & 127u);
    Smem& sm = *reinterpret_cast<Smem*>(ring + p.stages * kTile);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int stages = p.stages, octets = p.octets, teams = p.teams;
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) {
            ptx::mbar_init(ptx::smem_addr(&sm.full[s]), 1);
            ptx::mbar_init(ptx::smem_addr(&sm.empty[s]), octets);
        }
        ptx::mbar_fence_init();
    }
    // The tables are launch parameters, or were there before the previous kernel of the stream began: they may be read under its tail.
    const bool by_cta = WHOLE || p.share > 0;
    const int u0 = by_cta ? int(blockIdx.x) : int(int64_t(p.n_units) * blockIdx.x / p.n_ctas);
    const int u1 = by_cta ? u0 + 1 : int(int64_t(p.n_units) * (blockIdx.x + 1) / p.n_ctas);
    Pair x = pair_at<WHOLE>(p, u0, u1);
    __syncthreads();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    if (warp == kWarps) {
        // ---------------- producer ----------------
        if (lane != 0) return;
        const uint64_t pol = ptx::l2_evict_first_policy();
        int st = 0, lap = 0;
        bool ok = true;
        for (int u = u0; u < u1 && ok && x.r.tiles > 0;) {
            int k = x.r.run0, hi = (x.row + 1 < p.n_rows ? row_at(p, x.row + 1).run0 : p.n_runs) - 1;
            while (k < hi) {                     // the row's last run that begins at or before the first tile
                const int mid = (k + hi + 1) >> 1;
                if (run_at(p, mid).tile0 <= x.tile0) k = mid; else hi = mid - 1;
            }
            // the address moves from tile to tile by additions: a division per tile would make this one thread the bottleneck
            const int per = p.g.bt / kTileTokens;
            const int64_t to_next_block = p.g.block_bytes() - int64_t(per - 1) * kTile;
            NibbleRunArg run = run_at(p, k);
            int tile = x.tile0 - run.tile0, left = run.n_tokens - tile * kTileTokens, in_block = tile % per;
            const char* src = run.blocks + p.g.tile_off(tile, x.kv);
            for (int i = 0; i < x.n; ++i) {
                if (left <= 0) {
                    run = run_at(p, ++k);
                    left = run.n_tokens; in_block = 0;
                    src = run.blocks + p.g.tile_off(0, x.kv);
                }
                if (lap > 0 && !ptx::mbar_wait(ptx::smem_addr(&sm.empty[st]), (lap - 1) & 1)) { ok = false; break; }
                sm.n_valid[st] = left < kTileTokens ? left : kTileTokens;
                const uint32_t bar = ptx::smem_addr(&sm.full[st]);
                ptx::mbar_expect_tx(bar, kTile);
                const int64_t extent = kChecked && p.status ? (int64_t(run.n_tokens) + p.g.bt - 1) / p.g.bt * p.g.block_bytes() : 0;
                ptx::bulk_g2s_hint(ptx::smem_addr(ring + st * kTile), ptx::checked_src<kChecked>(src, kTile, run.blocks, extent, p.status, kStatusBadIndex),
                                   kTile, bar, pol);
                left -= kTileTokens;
                if (++in_block == per) { in_block = 0; src += to_next_block; } else src += kTile;
                if (++st == stages) { st = 0; ++lap; }
            }
            u += x.units;
            if (u < u1) next_pair(p, x, u, u1);
        }
        if (!ok && p.status) atomicOr(p.status, kStatusNoFreeStage);
        // do not leave the CTA while copies of ours may still be in flight
        for (int i = 0; i < stages; ++i) {
            const int last = i < st ? lap : lap - 1;         // the stage's last lap
            if (last >= 0 && !ptx::mbar_wait(ptx::smem_addr(&sm.full[i]), last & 1) && p.status) atomicOr(p.status, kStatusCopyNotLanded);
        }
        return;
    }

    // ---------------- consumers ----------------
    const int g = lane >> 2, t = lane & 3;
    const int team = warp / octets, octet = warp - team * octets;        // octets divide the warps: every warp has a team
    bool dead = false;
    // Which tokens enter the output product complemented: 16u + 8h + g with g + h odd.
    const uint32_t odd = p.odd_tokens;           // g odd, as the halves of a word of V (an immediate here would cost an instruction a use)
    const float k15 = (g & 1) ? 15.f : 0.f;

    int it0 = 0;                                 // tiles of this CTA before the current pair
    int st = team, phase = 0;                    // stage of the team's next tile and its parity (stages is a multiple of teams)
    for (int u = u0; u < u1;) {
        const int in_kv = x.part * p.rows_per_part;      // the head group's first head among those of its KV head
        const int n_heads = min(p.group - in_kv, p.rows_per_part), head0 = x.kv * p.group + in_kv;

        // ---- queries: operands of head g (columns 64p+16t+8w+{0,4},{1,5},{2,6},{3,7}), normalised to [2^110, 2^111) ----
        uint32_t qf[P][2][4];
        uint32_t qz;                             // 2^-133 sum(q) of each panel and head g: its t-th term of three bf16 (24 bits), 0 for t = 3
        float c[2];                              // log2 units per score, of heads 2t and 2t+1
        {
            const int hq = octet * 8 + (HALF ? (g & 3) : g);
            const bool live = hq < n_heads;
            const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t(x.row) * p.n_q_heads + head0 + hq) * (2 * D) + 32 * t);
            float v[P][16], top = 0.f;
#pragma unroll
            for (int pn = 0; pn < P; ++pn)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint4 y = live ? __ldg(src + pn * 8 + w) : make_uint4(0, 0, 0, 0);
                    const uint32_t yy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) { v[pn][8 * w + 2 * i] = ptx::bf16_lo(yy[i]); v[pn][8 * w + 2 * i + 1] = ptx::bf16_hi(yy[i]); }
                }
#pragma unroll
            for (int pn = 0; pn < P; ++pn)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(v[pn][i]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = min(max(int(__float_as_uint(top) >> 23), 110), 231);
            const float f = __uint_as_float(uint32_t(364 - e) << 23);                    // 2^110 / 2^(exponent of the largest)
            const float cg = p.scale * kLog2e * __uint_as_float(uint32_t(23 + e) << 23); // ... undone, with the codes' 2^133
            float sum[P];
#pragma unroll
            for (int pn = 0; pn < P; ++pn) {
                sum[pn] = 0.f;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    float* y = &v[pn][8 * w];
#pragma unroll
                    for (int i = 0; i < 8; ++i) { y[i] *= f; sum[pn] += y[i]; }
                    qf[pn][w][0] = ptx::pack_bf16(y[0], y[4]);
                    qf[pn][w][1] = ptx::pack_bf16(y[1] * 0.0625f, y[5] * 0.0625f);
                    qf[pn][w][2] = ptx::pack_bf16(y[2], y[6]);
                    qf[pn][w][3] = ptx::pack_bf16(y[3] * 0.0625f, y[7] * 0.0625f);
                }
                sum[pn] += __shfl_xor_sync(0xffffffffu, sum[pn], 1);
                sum[pn] += __shfl_xor_sync(0xffffffffu, sum[pn], 2);
                float rest = sum[pn] * 0x1p-100f * 0x1p-33f, term = 0.f;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    const float y = ptx::bf16_lo(ptx::pack_bf16(rest, rest));
                    if (k == t) term = y;
                    rest -= y;
                }
                sum[pn] = term;
            }
            qz = ptx::pack_bf16(sum[0], P == 2 ? sum[P - 1] : 0.f);
            c[0] = __shfl_sync(0xffffffffu, cg, 8 * t);                                  // lane 4 (2t): head 2t
            c[1] = __shfl_sync(0xffffffffu, cg, 8 * t + 4);
        }

        // ---- the warp's state over its tiles of this pair ----
        float o[D / 16][4];                      // [column g / g+8 of 16][head 2t / 2t+1], times 64 fv / 2^21
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[d][i] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, oz[2] = {0.f, 0.f};      // l and oz: this lane's tokens only
        float limit[2] = {-INFINITY, -INFINITY};                                          // scores above it raise m
        // What value scales are multiplied with, 2^(127 - x) for a head, as the operands have it: times 64, and negative where a complement's
        // weight is.  Scales from v_limit on may raise an x.
        float v_limit = -1.f, f0[2] = {0.f, 0.f};
        auto scaled_by = [&](int e) { return f0[e] == 0.f ? -1 : 260 - int(__float_as_uint(f0[e]) >> 23 & 255u); };     // x, -1: not yet

        // the tiles of team `team`: it = team modulo teams
        const int it_end = it0 + x.n;
        int first = it0 / teams * teams + team;
        if (first < it0) first += teams;
        for (int it = first; it < it_end; it += teams) {
            if (!dead && !ptx::mbar_wait(ptx::smem_addr(&sm.full[st]), phase)) {
                if (lane == 0 && p.status) atomicOr(p.status, kStatusNoTile);
                dead = true;
            }
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
            const unsigned char* tile = ring + st * kTile;
            const int nv = sm.n_valid[st];

            // scores of tokens 16u+g (0, 1) and 16u+8+g (2, 3) for heads 2t and 2t+1
            float s[4][4];
            float sv[4][2], zv[4][2];
#pragma unroll
            for (int un = 0; un < 4; ++un) {
                float acc[P][4];
#pragma unroll
                for (int pn = 0; pn < P; ++pn) {
                    acc[pn][0] = acc[pn][1] = acc[pn][2] = acc[pn][3] = 0.f;
                    const uint4 y = *reinterpret_cast<const uint4*>(tile + ((un * P + pn) * 32 + lane) * 16);
                    const uint32_t ya[2] = {y.x, y.y}, yb[2] = {y.z, y.w};
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const uint32_t a8 = ya[w] >> 8, b8 = yb[w] >> 8;
                        mma_bf16(acc[pn], ya[w] & kLowK, yb[w] & kLowK, ya[w] & kHighK, yb[w] & kHighK, qf[pn][w][0], qf[pn][w][1]);
                        mma_bf16(acc[pn], a8 & kLowK, b8 & kLowK, a8 & kHighK, b8 & kHighK, qf[pn][w][2], qf[pn][w][3]);
                    }
                }
                uint32_t km[2][P];
                if (P == 2) {
                    const uint4 y = *reinterpret_cast<const uint4*>(tile + kKMeta + (un * 8 + g) * 16);
                    km[0][0] = y.x; km[0][P - 1] = y.y; km[1][0] = y.z; km[1][P - 1] = y.w;
                } else {
                    const uint2 y = *reinterpret_cast<const uint2*>(tile + kKMeta + (un * 8 + g) * 8);
                    km[0][0] = y.x; km[1][0] = y.y;
                }
                const uint2 vm = *reinterpret_cast<const uint2*>(tile + kVMeta + (un * 8 + g) * 8);
                const uint32_t vmm[2] = {vm.x, vm.y};
                // the zeros' share, sum over panels of zk sum(q): columns 2t and 2t+1 of A are both panels' zeros, rows of B the terms of qz
                float zeros[4] = {0.f, 0.f, 0.f, 0.f};
                mma_bf16_k8(zeros, __byte_perm(km[0][0], km[0][P - 1], 0x7632), __byte_perm(km[1][0], km[1][P - 1], 0x7632), qz);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        s[un][2 * h + e] = zeros[2 * h + e];
#pragma unroll
                        for (int pn = 0; pn < P; ++pn) s[un][2 * h + e] = fmaf(ptx::bf16_lo(km[h][pn]), acc[pn][2 * h + e], s[un][2 * h + e]);
                    }
                    sv[un][h] = ptx::bf16_lo(vmm[h]);
                    zv[un][h] = fmaf(ptx::bf16_lo(vmm[h]), h ? 15.f - k15 : k15, ptx::bf16_hi(vmm[h]));
                }
            }
            if (nv < kTileTokens) {              // what lies behind the last token may be anything, NaN too
#pragma unroll
                for (int un = 0; un < 4; ++un)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (un * 16 + h * 8 + g >= nv) { s[un][2 * h] = s[un][2 * h + 1] = -INFINITY; sv[un][h] = zv[un][h] = 0.f; }
            }

            // raise the references where a score or a scale has outgrown them (the first tile always does)
            float top[2] = {s[0][0], s[0][1]}, v_top = fmaxf(sv[0][0], sv[0][1]);
#pragma unroll
            for (int un = 0; un < 4; ++un) {
                top[0] = fmaxf(top[0], fmaxf(s[un][0], s[un][2]));
                top[1] = fmaxf(top[1], fmaxf(s[un][1], s[un][3]));
                v_top = fmaxf(v_top, fmaxf(sv[un][0], sv[un][1]));
            }
            const bool outgrown = top[0] > limit[0] || top[1] > limit[1];
            if (__any_sync(0xffffffffu, outgrown || v_top >= v_limit)) {
                float alpha[2] = {1.f, 1.f};
                bool rescale = __any_sync(0xffffffffu, outgrown);
#pragma unroll
                for (int d = 4; d <= 16; d <<= 1) v_top = fmaxf(v_top, __shfl_xor_sync(0xffffffffu, v_top, d));
                if (rescale) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int d = 4; d <= 16; d <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], d));
                        const float m_new = fmaxf(m[e], top[e] * c[e]);
                        alpha[e] = m[e] == -INFINITY ? 0.f : ptx::ex2(m[e] - m_new);
                        m[e] = m_new;
                        limit[e] = (m_new + kRaise) / c[e];
                        l[e] *= alpha[e]; oz[e] *= alpha[e];
                    }
                }
                if (__any_sync(0xffffffffu, v_top >= v_limit)) {
                    // scales of one order all count; otherwise a token's does in full from a weight of 2^-12 on, and less below
                    float least = v_top, most[2] = {v_top, v_top};
#pragma unroll
                    for (int un = 0; un < 4; ++un) least = fminf(least, fminf(sv[un][0], sv[un][1]));
                    if (__any_sync(0xffffffffu, least * float(1 << kRoom) < v_top)) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            most[e] = 0.f;
#pragma unroll
                            for (int un = 0; un < 4; ++un)
#pragma unroll
                                for (int h = 0; h < 2; ++h) most[e] = fmaxf(most[e], sv[un][h] * fminf(ptx::ex2(fmaf(s[un][2 * h + e], c[e], 12.f - m[e])), 1.f));
#pragma unroll
                            for (int d = 4; d <= 16; d <<= 1) most[e] = fmaxf(most[e], __shfl_xor_sync(0xffffffffu, most[e], d));
                        }
                    }
                    bool raised = false;
                    int x_low = 255;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        int x = scaled_by(e);
                        if (most[e] >= __uint_as_float(uint32_t(x + 1) << 23)) {
                            const int x_new = min(max(int(__float_as_uint(most[e]) >> 23) + kRoom, 8), 250);     // such scales lie below 2^(1 - kRoom) then
                            alpha[e] *= x < 0 ? 0.f : __uint_as_float(uint32_t(max(127 + x - x_new, 0)) << 23);
                            f0[e] = __uint_as_float(uint32_t(260 - x_new) << 23 | (g & 1) << 31);
                            x = x_new;
                            raised = true;
                        }
                        x_low = min(x_low, x);
                    }
                    v_limit = __uint_as_float(uint32_t(x_low + 1) << 23);
                    rescale = __any_sync(0xffffffffu, raised) || rescale;
                }
                if (rescale) {
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        o[d][0] *= alpha[0]; o[d][1] *= alpha[1]; o[d][2] *= alpha[0]; o[d][3] *= alpha[1];
                    }
                }
            }

            // weights, and their products with the value scales as operands [token][head]
            uint32_t hi[4][2], lo[4][2];
            float zt[2] = {0.f, 0.f};
            const float2 f1 = mul2(f0[0], f0[1], -0.0625f, -0.0625f);                    // codes of h = 1 are times 2^4, and complements where h = 0's are not
#pragma unroll
            for (int un = 0; un < 4; ++un)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float2 svf = h ? mul2(f1.x, f1.y, sv[un][h], sv[un][h]) : mul2(f0[0], f0[1], sv[un][h], sv[un][h]);
                    const float2 y = fma2(s[un][2 * h], s[un][2 * h + 1], c[0], c[1], -m[0], -m[1]);
                    const float pr[2] = {ptx::ex2(y.x), ptx::ex2(y.y)};
                    add2(l[0], l[1], pr[0], pr[1]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) zt[e] = fmaf(pr[e], zv[un][h], zt[e]);
                    float2 w = mul2(pr[0], pr[1], svf.x, svf.y);
                    const uint32_t big = pack_f16(w.x, w.y);
                    const float2 back = unpack_f16(big);
                    add2(w.x, w.y, -back.x, -back.y);
                    w = mul2(w.x, w.y, kRest, kRest);
                    const uint32_t rest = pack_f16(w.x, w.y);
                    if (HALF) hi[un][h] = transpose8x8(t < 2 ? big : rest);              // columns 4-7 repeat heads 0-3
                    else { hi[un][h] = transpose8x8(big); lo[un][h] = transpose8x8(rest); }
                }

            add2(oz[0], oz[1], zt[0], zt[1]);

            // output: 16 columns of the head a time, the tile's 64 tokens; sums per tile, added to the state in fp32 (to nearest)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const uint4 y = *reinterpret_cast<const uint4*>(tile + kV + (d * 32 + lane) * 16);
                const uint32_t ya[2] = {y.x, y.y}, yb[2] = {y.z, y.w};
                float sum[4] = {0.f, 0.f, 0.f, 0.f}, low[4] = {0.f, 0.f, 0.f, 0.f};      // of the weights' heads and remainders
#pragma unroll
                for (int un = 0; un < 4; ++un) {
                    const uint32_t va = (un & 1) ? ya[un >> 1] >> 5 : ya[un >> 1] << 3, vb = (un & 1) ? yb[un >> 1] >> 5 : yb[un >> 1] << 3;
                    const uint32_t a0 = differ(va, odd, kLow), a1 = differ(vb, odd, kLow), a2 = agree(va, odd, kHigh), a3 = agree(vb, odd, kHigh);
                    mma_f16(sum, a0, a1, a2, a3, hi[un][0], hi[un][1]);
                    if (!HALF) mma_f16(low, a0, a1, a2, a3, lo[un][0], lo[un][1]);
                }
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    if (!HALF) {
                        const float2 both = fma2(low[i], low[i + 1], 1.f / kRest, 1.f / kRest, sum[i], sum[i + 1]);
                        add2(o[d][i], o[d][i + 1], both.x, both.y);
                    } else {
                        add2(o[d][i], o[d][i + 1], sum[i], sum[i + 1]);
                    }
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&sm.empty[st]));
            st += teams;
            if (st >= stages) { st -= stages; phase ^= 1; }
        }

        if (WHOLE) consumers_meet();             // the ring is free when every warp has done its tiles
        // ---- the warp's partial: every team writes its own (nobody waits for another warp), one without a tile an empty one ----
        {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d <= 16; d <<= 1) {
                    l[e] += __shfl_xor_sync(0xffffffffu, l[e], d);
                    oz[e] += __shfl_xor_sync(0xffffffffu, oz[e], d);
                }
                f[e] = l[e] == 0.f ? 0.f : 1.f / l[e];
            }
            float undo[2];                       // 2^(x - 127), behind 2^15: 2^21 / 64
#pragma unroll
            for (int e = 0; e < 2; ++e) undo[e] = __uint_as_float(uint32_t(max(scaled_by(e), 0)) << 23);
            const int hb = octet * 8 + 2 * t;    // of the head group
            const int64_t row0 = (int64_t(x.slot) * teams + team) * p.rows_per_part + hb;      // (of the ring's memory: slot 0)
            const bool inside = !kChecked || WHOLE || (row0 >= 0 && row0 + min(2, n_heads - hb) <= p.part_rows);      // the partial must lie inside the scratch
            if (kChecked && !inside && hb < n_heads && p.status) atomicOr(p.status, kStatusBadIndex);
            const bool writes = (!HALF || t < 2) && inside;
            float* dst = (WHOLE ? reinterpret_cast<float*>(ring) : p.part_o) + row0 * D + g;
            float2* dst_ml = (WHOLE ? reinterpret_cast<float2*>(ring + kPartRows * D * 4) : p.part_ml) + row0;
            if (x.n > (team - it0 % teams + teams) % teams) {            // the team had a tile
#pragma unroll
                for (int d = 0; d < D / 16; ++d) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (HALF) o[d][i] = fmaf(__shfl_xor_sync(0xffffffffu, o[d][i], 2), 1.f / kRest, o[d][i]);
                        o[d][i] = fmaf(o[d][i] * 0x1p15f, undo[i & 1], oz[i & 1]) * f[i & 1];
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (writes && hb + e < n_heads) { dst[e * D + 16 * d] = o[d][e]; dst[e * D + 16 * d + 8] = o[d][2 + e]; }
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (g == 0 && writes && hb + e < n_heads) dst_ml[e] = make_float2(m[e], l[e]);
        }
        if (WHOLE) {                             // the teams' partials are all there are: join them here, as nibble_reduce_kernel does
            consumers_meet();
            const float4* part = reinterpret_cast<const float4*>(ring);
            const float2* ml = reinterpret_cast<const float2*>(ring + kPartRows * D * 4);
            for (int i = tid; i < n_heads * (D / 4); i += kWarps * 32) {
                const int head = i / (D / 4), col = i - head * (D / 4);
                float m_all = -INFINITY, z = 0.f;
                for (int k = 0; k < teams; ++k) m_all = fmaxf(m_all, ml[k * p.rows_per_part + head].x);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int k = 0; k < teams; ++k) {
                    const float2 y = ml[k * p.rows_per_part + head];
                    if (y.y != 0.f) {
                        const float w = ptx::ex2(y.x - m_all) * y.y;
                        const float4 v = part[(k * p.rows_per_part + head) * (D / 4) + col];
                        acc.x += w * v.x; acc.y += w * v.y; acc.z += w * v.z; acc.w += w * v.w;
                        z += w;
                    }
                }
                const float inv = z == 0.f ? 0.f : 1.f / z;
                const int64_t item = int64_t(x.row) * p.n_q_heads + head0 + head;
                reinterpret_cast<float4*>(p.out_o + item * D)[col] = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
                if (col == 0) p.out_lse[item] = z == 0.f ? -INFINITY : m_all * kLn2 + logf(z);
            }
        }
        it0 = it_end;
        u += x.units;
        if (u < u1) next_pair(p, x, u, u1);
    }
}

// Joins the partials of every (row, query head): with partial i's maximum m_i (log2), sum l_i and normalised O_i,
//   m = max m_i,  z = sum 2^(m_i - m) l_i,  O = sum 2^(m_i - m) l_i O_i / z,  LSE = m ln 2 + ln z,   in a fixed order.
// One CTA per (row, head, COLS columns): COLS/4 column groups times THREADS / (COLS/4) slices of the partials.  Bound by the latency of
// its two dependent reads (16 rows of 32K tokens, 512 heads of 32 partials: 10 us by itself, most of it under the kernel before and after);
// many partials per head (few heads, a long sequence) want many slices, see kManyParts.
template <int D, int COLS, int THREADS>
__global__ void __launch_bounds__(THREADS) nibble_reduce_kernel(const __grid_constant__ NibbleAttend p) {
    constexpr int kCols = COLS / 4, kSlices = THREADS / kCols, kSlabs = D / COLS;
    __shared__ float4 s_o[kSlices][kCols];
    __shared__ float s_z[kSlices], s_m[THREADS / 32];
    const int item = blockIdx.x / kSlabs, slab = blockIdx.x - item * kSlabs;     // item: row * n_q_heads + head
    const int row = item / p.n_q_heads, head = item - row * p.n_q_heads;
    const NibbleRowArg r = row_at(p, row);
    const int tid = threadIdx.x, col = tid % kCols, slice = tid / kCols;
    float4* out = reinterpret_cast<float4*>(p.out_o + int64_t(item) * D + slab * COLS) + col;
    const int kv = head / p.group, in_kv = head - kv * p.group, part_of = in_kv / p.rows_per_part, rin = in_kv - part_of * p.rows_per_part;
    const int gh = kv * p.groups_per_kv + part_of, teams = p.teams;
    int e0 = 0, n = 0;
    if (r.tiles > 0 && p.share > 0) {
        const int ctas = (r.tiles + p.share - 1) / p.share;
        e0 = (r.first + gh * ctas) * teams; n = ctas * teams;
    } else if (r.tiles > 0) {                    // the CTAs that hold the pair's first and last unit, hence its first and last partial
        const int64_t a = int64_t(r.first) + int64_t(gh) * (r.tiles + kNibblePairCost), b = a + r.tiles + kNibblePairCost - 1;
        const int c0 = int(((a + 1) * p.n_ctas - 1) / p.n_units), c1 = int(((b + 1) * p.n_ctas - 1) / p.n_units);
        e0 = (c0 + r.pair0 + gh) * teams; n = (c1 - c0 + 1) * teams;
    }
    const float2* ml = p.part_ml + int64_t(e0) * p.rows_per_part + rin;
    const float4* part = reinterpret_cast<const float4*>(p.part_o + (int64_t(e0) * p.rows_per_part + rin) * D + slab * COLS) + col;
    const int64_t stride = int64_t(p.rows_per_part) * (D / 4);
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (n == 0) {                                // nothing attended: (0, -inf)
        if (slice == 0) *out = make_float4(0.f, 0.f, 0.f, 0.f);
        if (tid == 0 && slab == 0) p.out_lse[item] = -INFINITY;
        return;
    }

    float m = -INFINITY;
    for (int i = tid; i < n; i += THREADS) m = fmaxf(m, ml[int64_t(i) * p.rows_per_part].x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if ((tid & 31) == 0) s_m[tid >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) m = fmaxf(m, s_m[w]);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float z = 0.f;
#pragma unroll 4
    for (int i = slice; i < n; i += kSlices) {
        const float2 x = ml[int64_t(i) * p.rows_per_part];
        const float4 v = part[int64_t(i) * stride];
        if (x.y != 0.f) {                        // an empty one's output may hold anything (a sum of NaN is not empty: it must be seen)
            const float w = ptx::ex2(x.x - m) * x.y;
            acc.x += w * v.x; acc.y += w * v.y; acc.z += w * v.z; acc.w += w * v.w;
            z += w;
        }
    }
    s_o[slice][col] = acc;
    if (col == 0) s_z[slice] = z;
    __syncthreads();
    if (slice != 0) return;
#pragma unroll
    for (int k = 1; k < kSlices; ++k) {
        const float4 v = s_o[k][col];
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
        z += s_z[k];
    }
    const float inv = z == 0.f ? 0.f : 1.f / z;
    *out = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (tid == 0 && slab == 0) p.out_lse[item] = z == 0.f ? -INFINITY : m * kLn2 + logf(z);
}

}  // namespace

cudaError_t launch_nibble_attend(NibbleAttend& a, cudaStream_t s) {
    const bool wide = a.g.dim == 128, half = a.group <= 4;
    if (a.n_ctas > 0) {
        a.stages = nibble_stages(a.g.dim, a.octets);
        if (a.stages <= 0) return cudaErrorInvalidValue;
        const size_t smem = size_t(a.stages) * a.g.tile_bytes() + nibble_fixed_smem();
#define IPKV_NIBBLE(D) (half ? (a.whole ? nibble_attend_kernel<D, true, true> : nibble_attend_kernel<D, true, false>) \
                             : (a.whole ? nibble_attend_kernel<D, false, true> : nibble_attend_kernel<D, false, false>))
        auto kernel = wide ? IPKV_NIBBLE(128) : IPKV_NIBBLE(64);
#undef IPKV_NIBBLE
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNibbleSmemPerCta);
        if (e != cudaSuccess) return e;
        e = launch_ordered(!a.plain_launch, kernel, a.n_ctas, kThreads, smem, s, a);
        if (e != cudaSuccess) return e;
    }
    if (a.whole) return cudaSuccess;
    const int items = a.n_rows * a.n_q_heads;
    if (a.max_parts > kVeryManyParts)
        return launch_ordered(true, wide ? nibble_reduce_kernel<128, 32, 512> : nibble_reduce_kernel<64, 32, 512>, items * (a.g.dim / 32), 512,
                              size_t(0), s, a);
    if (a.max_parts > kManyParts)
        return launch_ordered(true, wide ? nibble_reduce_kernel<128, 32, 256> : nibble_reduce_kernel<64, 32, 256>, items * (a.g.dim / 32), 256,
                              size_t(0), s, a);
    return launch_ordered(a.n_units > 0, wide ? nibble_reduce_kernel<128, 128, 128> : nibble_reduce_kernel<64, 64, 128>, items, 128, size_t(0), s, a);
}

}  // namespace ipkvi
