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
// changes lanes; only the sum of squares does.  A warp takes 512/D heads a step and keeps the eight cosines and sines of
// every lane through all heads of its token.  With few tokens the steps of a token are divided among warps (`split`), so
// that one token of 36 heads is not one warp's nine steps in a row.
#include <cuda_bf16.h>

#include "launch.cuh"
#include "ops.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kRopeWarps = 4;

template <int D>
__global__ void __launch_bounds__(kRopeWarps * 32) norm_rope_kernel(const __grid_constant__ RopeLaunch p) {
    constexpr int kLanes = D / 16;               // lanes of a head
    constexpr int kHeads = 32 / kLanes;          // heads of a step
    __shared__ uint64_t s_turn[D / 2];
    __shared__ uint8_t s_axis[D / 2];
    const int tid = threadIdx.x, lane = tid & 31;
    const int pairs = p.rot_dim / 2;
    for (int i = tid; i < pairs; i += kRopeWarps * 32) { s_turn[i] = p.turn[i]; s_axis[i] = p.axis[i]; }
    __syncthreads();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    const int j = lane % kLanes, sub = lane / kLanes;
    const bool rotated = j < pairs / 8;
    // the lane's two chunks: both columns of its pairs, or two neighbouring chunks (adjacent pairs, and columns that stay)
    const int c0 = (rotated && !p.interleaved) ? 8 * j : 16 * j;
    const int c1 = (rotated && !p.interleaved) ? pairs + 8 * j : 16 * j + 8;

    const int64_t items = p.n_tokens * p.split;
    for (int64_t item = int64_t(blockIdx.x) * kRopeWarps + (tid >> 5); item < items; item += int64_t(gridDim.x) * kRopeWarps) {
        const int64_t token = item / p.split;
        const int part_of = int(item - token * p.split);
        const int s0 = p.n_steps * part_of / p.split, s1 = p.n_steps * (part_of + 1) / p.split;

        // the chunks of a step, null where the lane has no head
        int part = 0;
        auto locate = [&](int step, const char*& src, char*& dst, const char*& w) {
            while (part + 1 < p.n_parts && step >= p.part[part + 1].step0) ++part;
            const RopePart& q = p.part[part];
            const int head = (step - q.step0) * kHeads + sub;
            src = head < q.n_heads ? q.in + token * q.in_token + head * q.in_head : nullptr;
            dst = q.out + token * q.out_token + head * q.out_head;
            w = q.weight;
        };
        const char* src; char* dst; const char* w;
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        locate(s0, src, dst, w);
        if (src) { a = *reinterpret_cast<const uint4*>(src + 2 * c0); b = *reinterpret_cast<const uint4*>(src + 2 * c1); }

        float co[8], si[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { co[i] = 1.f; si[i] = 0.f; }
        if (rotated) {
            const int32_t pos0 = p.n_axes == 1 ? p.positions[token] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t pos = p.n_axes == 1 ? pos0 : p.positions[int64_t(s_axis[8 * j + i]) * p.n_tokens + token];
                const uint64_t turns = uint64_t(int64_t(pos)) * s_turn[8 * j + i];
                sincospif(float(int32_t(turns >> 32)) * 0x1p-31f, &si[i], &co[i]);
            }
        }

        for (int step = s0; step < s1; ++step) {
            const char *src_n = nullptr, *w_n = nullptr;
            char* dst_n = nullptr;
            uint4 an = make_uint4(0, 0, 0, 0), bn = an;
            if (step + 1 < s1) {                 // the next step's loads go out before this one's arithmetic
                locate(step + 1, src_n, dst_n, w_n);
                if (src_n) { an = *reinterpret_cast<const uint4*>(src_n + 2 * c0); bn = *reinterpret_cast<const uint4*>(src_n + 2 * c1); }
            }
            float x[8], y[8];
            const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = ptx::bf16_lo(av[i]); x[2 * i + 1] = ptx::bf16_hi(av[i]);
                y[2 * i] = ptx::bf16_lo(bv[i]); y[2 * i + 1] = ptx::bf16_hi(bv[i]);
            }
            if (w) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) { ss += x[i] * x[i]; ss += y[i] * y[i]; }
#pragma unroll
                for (int d = kLanes / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
                const float r = rsqrtf(ss * (1.f / D) + p.eps);
                const uint4 wa = __ldg(reinterpret_cast<const uint4*>(w + 2 * c0)), wb = __ldg(reinterpret_cast<const uint4*>(w + 2 * c1));
                const uint32_t wav[4] = {wa.x, wa.y, wa.z, wa.w}, wbv[4] = {wb.x, wb.y, wb.z, wb.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] *= r * ptx::bf16_lo(wav[i]); x[2 * i + 1] *= r * ptx::bf16_hi(wav[i]);
                    y[2 * i] *= r * ptx::bf16_lo(wbv[i]); y[2 * i + 1] *= r * ptx::bf16_hi(wbv[i]);
                }
            }
            if (rotated) {
                if (p.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float u = x[2 * i], v = x[2 * i + 1];
                        x[2 * i] = u * co[i] - v * si[i]; x[2 * i + 1] = v * co[i] + u * si[i];
                        const float u2 = y[2 * i], v2 = y[2 * i + 1];
                        y[2 * i] = u2 * co[4 + i] - v2 * si[4 + i]; y[2 * i + 1] = v2 * co[4 + i] + u2 * si[4 + i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = x[i], v = y[i];
                        x[i] = u * co[i] - v * si[i]; y[i] = v * co[i] + u * si[i];
                    }
                }
            }
            if (src) {
                *reinterpret_cast<uint4*>(dst + 2 * c0) = make_uint4(ptx::pack_bf16(x[0], x[1]), ptx::pack_bf16(x[2], x[3]), ptx::pack_bf16(x[4], x[5]), ptx::pack_bf16(x[6], x[7]));
                *reinterpret_cast<uint4*>(dst + 2 * c1) = make_uint4(ptx::pack_bf16(y[0], y[1]), ptx::pack_bf16(y[2], y[3]), ptx::pack_bf16(y[4], y[5]), ptx::pack_bf16(y[6], y[7]));
            }
            src = src_n; dst = dst_n; w = w_n; a = an; b = bn;
        }
    }
}

}  // namespace

cudaError_t launch_norm_rope(RopeLaunch& a, cudaStream_t s) {
    constexpr int kSms = 148, kCtasPerSm = 8;
    // few tokens: divide a token's steps until every SM has its warps, or every warp one step
    int64_t split = int64_t(kSms) * kCtasPerSm * kRopeWarps / a.n_tokens;
    if (split > a.n_steps) split = a.n_steps;
    a.split = split < 1 ? 1 : int(split);
    int64_t grid = (a.n_tokens * a.split + kRopeWarps - 1) / kRopeWarps;
    if (grid > int64_t(kSms) * 64) grid = int64_t(kSms) * 64;
    auto kernel = a.dim == 64 ? norm_rope_kernel<64> : a.dim == 128 ? norm_rope_kernel<128> : norm_rope_kernel<256>;
    return launch_overlapped(kernel, int(grid), kRopeWarps * 32, size_t(0), s, a);
}

}  // namespace ipkvi
