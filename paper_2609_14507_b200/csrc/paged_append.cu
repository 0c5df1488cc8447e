// New tokens into the pages of a paged cache.  A CTA takes some tokens, a thread one 16-byte chunk of a token's K or V rows, the same chunk of all
// its tokens: it asks for them, a thread per token finds the row, the slot and the page meanwhile (four dependent reads, and more for the
// search among the rows), then the chunks are stored.  Bound by the bytes (read once, written once) and, for a decode step, by the
// launch and that chain of reads.  Measured: nine chunks of prompts, 20743 tokens of 4 KV heads of 128 columns, 85 MB: 17.9 us, 4.8 TB/s (two or eight
// tokens a thread 18.2 and 18.0; a warp to a token, its reads one behind the other, 23.5); 64 tokens, one for each row, 8 KV heads: 2.4 us.
#include "launch.cuh"
#include "paged.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kThreads = 256, kAhead = 4;        // tokens of a thread under way
constexpr int kMostTokens = 64;                  // of a CTA

__global__ void __launch_bounds__(kThreads, 5) paged_append_kernel(const __grid_constant__ PagedAppend p, const int per_cta) {
    __shared__ int s_row[kMostTokens], s_slot[kMostTokens];
    __shared__ int64_t s_at[kMostTokens];        // the token's row in its page, from the pool on, and slot & 7 in its low bits; -1: it has no place
    const int tid = threadIdx.x;
    const int64_t token0 = int64_t(blockIdx.x) * per_cta;
    const int tokens = int(p.n_tokens - token0 < per_cta ? p.n_tokens - token0 : per_cta);
    const BlockGeom g = p.c.g;
    const int shift = g.dim_qk == 128 ? 4 : 3;   // 16-byte chunks of a head's row: 16 or 8
    const int per_plane = g.n_kv_heads << shift, per_token = 2 * per_plane;      // of a token's K; of its K and V
    const int wide = per_token < kThreads ? per_token : kThreads, at_once = int(unsigned(kThreads) / unsigned(wide));
    const int t0 = int(unsigned(tid) / unsigned(wide)), i0 = tid - t0 * wide;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    uint4 x[kAhead];
    auto load = [&](int i) {                     // chunk i of this thread's tokens
        const bool v = i >= per_plane;
        const int64_t stride = v ? p.v_token : p.k_token;
        const char* src = (v ? p.v + (i - per_plane) * 16 : p.k + i * 16) + (token0 + t0) * stride;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (t0 < at_once && t0 + k * at_once < tokens) x[k] = __ldg(reinterpret_cast<const uint4*>(src + k * (at_once * stride)));
    };
    load(i0);
    if (tid < tokens) {
        const int64_t token = token0 + tid;
        int row = int(token), n = 0;
        int64_t slot = -1, at = -1;
        if (p.row_start) {
            int lo = 0, hi = p.c.n_rows - 1;     // the last row that begins at or before the token
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (p.row_start[mid] <= token) lo = mid; else hi = mid - 1;
            }
            row = lo;
            const int begin = p.row_start[row], end = p.row_start[row + 1];
            if (token >= begin && token < end) {                 // (else behind the last row's)
                n = p.c.lengths[row];
                slot = int64_t(n) - (end - token);
            }
        } else {
            n = p.c.lengths[row];
            slot = int64_t(n) - 1;
        }
        if (n < 0 && p.status) atomicOr(p.status, kStatusBadPage);
        if (slot >= 0) {                         // (else not counted by the length)
            int page = -1;
            const int t = slot < int64_t(p.c.max_blocks) * g.bt ? int(slot) : 0, block = int(unsigned(t) / unsigned(g.bt));
            if (t == slot) page = p.c.table[row * p.c.table_stride + block];
            if (page >= 0 && page < p.c.n_blocks) at = page * g.block_bytes() + (t - block * g.bt) * 128 + (t & 7);
            else if (p.status) atomicOr(p.status, kStatusBadPage);
        }
        s_row[tid] = row; s_slot[tid] = int(slot); s_at[tid] = at;
    }
    __syncthreads();
    for (int i = i0;;) {
        const bool v = i >= per_plane;
        const int of = v ? i - per_plane : i, chunk = of & ((1 << shift) - 1);
        char* dst = p.c.pool + (of >> shift) * g.head_bytes() + (v ? g.k_plane_bytes() : 0) + int64_t(chunk >> 3) * (g.bt * 128);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (t0 < at_once && t0 + k * at_once < tokens) {
                const int64_t at = s_at[t0 + k * at_once];
                if (at >= 0) *reinterpret_cast<uint4*>(dst + (at & ~int64_t(7)) + (((chunk ^ int(at)) & 7) << 4)) = x[k];
            }
        i += wide;
        if (i >= per_token) break;
        load(i);
    }
    if (p.c.weights || p.c.positions)
        for (int c = tid; c < tokens * g.n_kv_heads; c += kThreads) {
            const int head = int(unsigned(c) / unsigned(tokens)), t = c - head * tokens;         // neighbours write neighbouring slots
            if (s_at[t] < 0) continue;
            const int64_t at = (int64_t(s_row[t]) * g.n_kv_heads + head) * p.c.slot_stride + s_slot[t];
            if (p.c.weights) p.c.weights[at] = 0.f;
            if (p.c.positions) p.c.positions[at] = p.token_positions[token0 + t];
        }
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppend& a, cudaStream_t s) {
    // as many tokens to a CTA as its threads have under way, fewer while there are SMs without work
    const int per_token = 2 * a.c.g.n_kv_heads * (a.c.g.dim_qk / 8), wide = per_token < kThreads ? per_token : kThreads, at_once = kThreads / wide;
    const int64_t spread = a.n_tokens / (4 * 148), full = kAhead * at_once < kMostTokens ? kAhead * at_once : kMostTokens;
    const int per_cta = int(spread < 1 ? 1 : spread < full ? spread : full);
    return launch_overlapped(paged_append_kernel, int((a.n_tokens + per_cta - 1) / per_cta), kThreads, size_t(0), s, a, per_cta);
}

}  // namespace ipkvi
