// RMS norm of every query / key head and the rotation of its columns by position, in one pass over the heads:
//   y = x * rsqrt(mean(x^2) + eps) * w,      (a, b) -> (a cos t - b sin t, b cos t + a sin t)
// for every pair (a, b) of columns of y, t = position on the pair's axis * the pair's frequency.  The values stay in fp32
// from the load to the one rounding at the store.
//
// Angles.  A product position * frequency in fp32 is off by position * 2^-25 radians (0.03 at a position of one million).
// The host hands every frequency over as a 64-bit fraction of a turn; the product with the position modulo 2^64 is then
// the exact fraction of a turn of the product, off by position * 2^-65 turns, and its top 32 bits go to sincospif.
//
// Bound by memory: every value is read once and written once, and the weights, positions and angles are shared.  A head of
// D columns belongs to D/16 lanes, each with two 16-byte chunks that hold both columns of its eight pairs, so no value
// changes lanes; only the sum of squares does.  A warp takes 512/D heads a step.  What a token's heads share is computed once per
// token: every lane takes D/64 pairs' sine and cosine and the lanes that need them fetch them by shuffles, and the weights are
// multiplied into them, so that a pair costs six fp32 operations a head: out_a = (a r)(w_a c) - (b r)(w_b s), out_b = (b r)(w_b c) + (a r)(w_a s).
// The copies of a warp's next steps are under way while it computes, across its tokens, through a ring of 16-byte slots in shared
// memory that each lane fills and reads for itself.  32K tokens of 36 heads of 128: 95.5 us in a few calls, 97 % of the measured copy rate, and
// 100 us back to back for seconds (the board at its power limit, 1.73 GHz); with loads into registers one step ahead 137 us (too few bytes
// under way), with sines by every lane for itself and the weights by themselves 141 us (bound by its instructions), in a few calls both.  With few tokens the steps of a token are divided among warps (`split`), so
// that one token of 36 heads is not one warp's nine steps in a row.
#include <cuda_bf16.h>

#include "launch.cuh"
#include "ops.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kRopeWarps = 4, kRopeCtasPerSm = 4;
constexpr int kRopeDepth = 3;                    // steps that are on their way while one is computed (4: 103 us, 3: 96 us)

__device__ __forceinline__ void copy16(uint32_t dst, const char* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A walk over the steps of a warp's tokens: which part a step belongs to, and where its heads begin.
struct Walk {
    int64_t item;                // token and share of its steps
    int64_t token;
    int step, last;              // of the token's steps this warp takes [step, last)
    int part, part_end;          // the part of `step`, and the first step behind it
    int head;                    // of the part: the lane's head
};

template <int D, bool INTERLEAVED, bool FULL>    // FULL: all columns are rotated
__global__ void __launch_bounds__(kRopeWarps * 32, kRopeCtasPerSm) norm_rope_kernel(const __grid_constant__ RopeLaunch p) {
    constexpr int kLanes = D / 16;               // lanes of a head
    constexpr int kHeads = 32 / kLanes;          // heads of a step
    constexpr int kOwn = D / 64;                 // pairs whose sine and cosine a lane computes
    __shared__ uint4 s_ring[kRopeDepth][2][kRopeWarps * 32];
    __shared__ uint64_t s_turn[D / 2];
    __shared__ uint8_t s_axis[D / 2];
    const int tid = threadIdx.x, lane = tid & 31;
    const int pairs = FULL ? D / 2 : p.rot_dim / 2;
    for (int i = tid; i < pairs; i += kRopeWarps * 32) { s_turn[i] = p.turn[i]; s_axis[i] = p.axis[i]; }
    __syncthreads();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    const int j = lane % kLanes, sub = lane / kLanes;
    const bool rotated = FULL || j < pairs / 8;
    // the lane's two chunks: both columns of its pairs, or two neighbouring chunks (adjacent pairs, and columns that stay)
    const int c0 = (rotated && !INTERLEAVED) ? 16 * j : 32 * j;                  // bytes
    const int c1 = (rotated && !INTERLEAVED) ? 2 * pairs + 16 * j : 32 * j + 16;

    const int64_t items = p.n_tokens * p.split, item_step = int64_t(gridDim.x) * kRopeWarps;
    auto enter_part = [&](Walk& w) {             // the part of w.step
        w.part = 0;
        while (w.part + 1 < p.n_parts && w.step >= p.part[w.part + 1].step0) ++w.part;
        w.part_end = min(w.last, w.part + 1 < p.n_parts ? p.part[w.part + 1].step0 : p.n_steps);
        w.head = (w.step - p.part[w.part].step0) * kHeads + sub;
    };
    auto enter_item = [&](Walk& w) {
        if (w.item >= items) return;
        w.token = w.item; w.step = 0; w.last = p.n_steps;
        if (p.split > 1) {
            const uint32_t split = uint32_t(p.split), item = uint32_t(w.item), token = item / split, share = item - token * split;   // few tokens
            w.token = token;
            w.step = int(uint64_t(p.n_steps) * share / split);       // 2^21 steps times 2^11 warps pass 32 bits
            w.last = int(uint64_t(p.n_steps) * (share + 1) / split);
        }
        enter_part(w);
    };
    // The walk of the copies runs kRopeDepth steps ahead of the arithmetic, across parts and tokens.  A lane reads only what it copied
    // itself, so the ring needs no synchronisation but the lane's own wait.
    Walk ahead;
    ahead.item = int64_t(blockIdx.x) * kRopeWarps + (tid >> 5);
    enter_item(ahead);
    Walk w = ahead;
    const char* src = nullptr;
    int64_t src_step = 0;
    auto source = [&]() {
        const RopePart& q = p.part[ahead.part];
        src = q.in + ahead.token * q.in_token + ahead.head * q.in_head;
        src_step = q.in_head * kHeads;
    };
    if (ahead.item < items) source();
    auto copy_next = [&](int slot) {
        if (ahead.item < items) {
            if (ahead.head < p.part[ahead.part].n_heads) {
                copy16(ptx::smem_addr(&s_ring[slot][0][tid]), src + c0);
                copy16(ptx::smem_addr(&s_ring[slot][1][tid]), src + c1);
            }
            ahead.head += kHeads; src += src_step;
            if (++ahead.step == ahead.part_end) {
                if (ahead.step < ahead.last) { enter_part(ahead); source(); }
                else { ahead.item += item_step; enter_item(ahead); if (ahead.item < items) source(); }
            }
        }
        copies_commit();                         // a group per step, empty at the end
    };
    int32_t pos[kOwn];                           // positions of the lane's own pairs, a token ahead
    auto fetch_positions = [&](int64_t token) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int pair = lane * kOwn + i;
            pos[i] = (FULL || pair < pairs) ? p.positions[(p.n_axes == 1 ? 0 : int64_t(s_axis[pair]) * p.n_tokens) + token] : 0;
        }
    };
    if (w.item < items && pairs > 0) fetch_positions(w.token);
#pragma unroll
    for (int i = 0; i < kRopeDepth; ++i) copy_next(i);
    int slot = 0;

    while (w.item < items) {
        // the token's sines and cosines: D/64 pairs a lane, then the eight of this lane's own pairs from the lanes that have them
        float own_c[kOwn], own_s[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            own_c[i] = 1.f; own_s[i] = 0.f;
            if (FULL || lane * kOwn + i < pairs) {
                const uint64_t turns = uint64_t(int64_t(pos[i])) * s_turn[lane * kOwn + i];
                sincospif(float(int32_t(turns >> 32)) * 0x1p-31f, &own_s[i], &own_c[i]);
            }
        }
        const int64_t next = w.item + item_step;
        if (next < items && pairs > 0) fetch_positions(p.split > 1 ? int64_t(uint32_t(next) / uint32_t(p.split)) : next);
        float co[8], si[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int from = 8 * j / kOwn + i / kOwn;
            co[i] = __shfl_sync(0xffffffffu, own_c[i % kOwn], from & 31);
            si[i] = __shfl_sync(0xffffffffu, own_s[i % kOwn], from & 31);
            if (!rotated) { co[i] = 1.f; si[i] = 0.f; }
        }

        while (w.step < w.last) {                // part by part
            const RopePart& q = p.part[w.part];
            const bool norm = q.weight != nullptr;
            // the weights times cosine and sine (the weights alone for columns that are not rotated)
            float wc[16], ws[16];                // of the first chunk's columns, then of the second's
            {
                uint4 wa = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), wb = wa;
                if (norm) { wa = __ldg(reinterpret_cast<const uint4*>(q.weight + c0)); wb = __ldg(reinterpret_cast<const uint4*>(q.weight + c1)); }
                const uint32_t wav[4] = {wa.x, wa.y, wa.z, wa.w}, wbv[4] = {wb.x, wb.y, wb.z, wb.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = (i & 1) ? ptx::bf16_hi(wav[i / 2]) : ptx::bf16_lo(wav[i / 2]);
                    const float v = (i & 1) ? ptx::bf16_hi(wbv[i / 2]) : ptx::bf16_lo(wbv[i / 2]);
                    const int pu = INTERLEAVED ? i / 2 : i, pv = INTERLEAVED ? 4 + i / 2 : i;    // the pair of either column
                    wc[i] = u * co[pu]; ws[i] = u * si[pu];
                    wc[8 + i] = v * co[pv]; ws[8 + i] = v * si[pv];
                }
            }
            char* dst = q.out + w.token * q.out_token + w.head * q.out_head;
            const int64_t dst_step = q.out_head * kHeads;
            const int n_heads = q.n_heads;
            for (; w.step < w.part_end; ++w.step) {
                copies_wait<kRopeDepth - 1>();
                const uint4 a = s_ring[slot][0][tid], b = s_ring[slot][1][tid];
                float x[16];
                const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] = ptx::bf16_lo(av[i]); x[2 * i + 1] = ptx::bf16_hi(av[i]);
                    x[8 + 2 * i] = ptx::bf16_lo(bv[i]); x[8 + 2 * i + 1] = ptx::bf16_hi(bv[i]);
                }
                if (norm) {                      // (a lane without a head sums what its slot holds, among its own head's lanes only)
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
                    for (int d = kLanes / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
                    const float r = rsqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] *= r;
                }
                float y[16];
                if (rotated) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // the two columns of pair i of this lane
                        const int ca = INTERLEAVED ? 2 * i : i, cb = INTERLEAVED ? 2 * i + 1 : 8 + i;
                        y[ca] = x[ca] * wc[ca] - x[cb] * ws[cb];
                        y[cb] = x[cb] * wc[cb] + x[ca] * ws[ca];
                    }
                } else {                         // the columns that stay must not see their neighbours (an infinity times 0)
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = x[i] * wc[i];
                }
                if (w.head < n_heads) {
                    *reinterpret_cast<uint4*>(dst + c0) = make_uint4(ptx::pack_bf16(y[0], y[1]), ptx::pack_bf16(y[2], y[3]), ptx::pack_bf16(y[4], y[5]), ptx::pack_bf16(y[6], y[7]));
                    *reinterpret_cast<uint4*>(dst + c1) = make_uint4(ptx::pack_bf16(y[8], y[9]), ptx::pack_bf16(y[10], y[11]), ptx::pack_bf16(y[12], y[13]), ptx::pack_bf16(y[14], y[15]));
                }
                w.head += kHeads; dst += dst_step;
                copy_next(slot);                 // into the slot just read
                slot = slot + 1 == kRopeDepth ? 0 : slot + 1;
            }
            if (w.step < w.last) enter_part(w);
        }
        w.item = next;
        enter_item(w);
    }
}

}  // namespace

cudaError_t launch_norm_rope(RopeLaunch& a, cudaStream_t s) {
    constexpr int kSms = 148;
    // few tokens: divide a token's steps until every SM has its warps, or every warp one step
    int64_t split = int64_t(kSms) * kRopeCtasPerSm * kRopeWarps / a.n_tokens;
    if (split > a.n_steps) split = a.n_steps;
    a.split = split < 1 ? 1 : int(split);
    int64_t grid = (a.n_tokens * a.split + kRopeWarps - 1) / kRopeWarps;
    if (grid > int64_t(kSms) * kRopeCtasPerSm) grid = int64_t(kSms) * kRopeCtasPerSm;     // one wave: its warps walk over their tokens
    const bool full = a.rot_dim == a.dim;
#define IPKV_ROPE(D) (a.interleaved ? (full ? norm_rope_kernel<D, true, true> : norm_rope_kernel<D, true, false>) \
                                    : (full ? norm_rope_kernel<D, false, true> : norm_rope_kernel<D, false, false>))
    auto kernel = a.dim == 64 ? IPKV_ROPE(64) : a.dim == 128 ? IPKV_ROPE(128) : IPKV_ROPE(256);
#undef IPKV_ROPE
    return launch_overlapped(kernel, int(grid), kRopeWarps * 32, size_t(0), s, a);
}

}  // namespace ipkvi
