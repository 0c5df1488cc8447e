// New tokens into the pages of a paged cache.  A CTA takes some tokens: every thread asks for its 16-byte chunks of their K and V rows, a thread
// per token finds the row, the slot and the page meanwhile (four dependent reads, and more for the search among the rows), then
// the chunks are stored.  Bound by the bytes (read once, written once) and, for a decode step, by the launch and that chain of reads.
// Measured: nine chunks of prompts, 20743 tokens of 4 KV heads of 128 columns, 85 MB: 19.3 us, 4.4 TB/s (23.5 with one warp to a token and its reads one
// behind the other, 20.4 with 8 chunks a thread, 19.4 to 21 with other CTAs).  64 tokens, one for each row: 2.8 us.
#include "launch.cuh"
#include "paged.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kThreads = 256, kAhead = 4;        // chunks of a thread under way
constexpr int kMostTokens = 32;                  // of a CTA

__global__ void __launch_bounds__(kThreads, 5) paged_append_kernel(const __grid_constant__ PagedAppend p, const int per_cta) {
    __shared__ int s_row[kMostTokens], s_slot[kMostTokens];
    __shared__ int64_t s_at[kMostTokens];        // the token's row in its page, from the pool on; -1: it has no place
    const int tid = threadIdx.x;
    const int64_t token0 = int64_t(blockIdx.x) * per_cta;
    const int tokens = int(p.n_tokens - token0 < per_cta ? p.n_tokens - token0 : per_cta);
    const BlockGeom g = p.c.g;
    const int shift = g.dim_qk == 128 ? 4 : 3;   // 16-byte chunks of a head's row: 16 or 8
    const int per_plane = g.n_kv_heads << shift, per_token = 2 * per_plane;      // of a token's K; of its K and V
    const int step_t = kThreads / per_token, step_i = kThreads - step_t * per_token;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    // chunk i of token t, the next one of this thread kThreads further
    auto advance = [&](int& t, int& i) {
        t += step_t; i += step_i;
        if (i >= per_token) { i -= per_token; ++t; }
    };
    auto load = [&](int t, int i) {
        const char* src = i < per_plane ? p.k + (token0 + t) * p.k_token + i * 16 : p.v + (token0 + t) * p.v_token + (i - per_plane) * 16;
        return __ldg(reinterpret_cast<const uint4*>(src));
    };
    const int t0 = tid / per_token, i0 = tid - t0 * per_token;
    uint4 x[kAhead];
    int t = t0, i = i0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        if (t < tokens) x[k] = load(t, i);
        advance(t, i);
    }
    if (tid < tokens) {
        const int64_t token = token0 + tid;
        int row = int(token);
        int64_t slot = -1, at = -1;
        if (p.row_start) {
            int lo = 0, hi = p.c.n_rows - 1;     // the last row that begins at or before the token
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (p.row_start[mid] <= token) lo = mid; else hi = mid - 1;
            }
            row = lo;
            const int begin = p.row_start[row], end = p.row_start[row + 1];
            if (token >= begin && token < end) slot = int64_t(p.c.lengths[row]) - (end - token);       // (else behind the last row's)
        } else {
            slot = int64_t(p.c.lengths[row]) - 1;
        }
        if (slot >= 0) {                         // (else not counted by the length)
            int page = -1;
            if (slot < int64_t(p.c.max_blocks) * g.bt) page = p.c.table[row * p.c.table_stride + slot / g.bt];
            if (page >= 0 && page < p.c.n_blocks) at = page * g.block_bytes() + slot % g.bt * 128;
            else if (p.status) atomicOr(p.status, kStatusBadPage);
        }
        s_row[tid] = row; s_slot[tid] = int(slot); s_at[tid] = at;
    }
    __syncthreads();
    const int64_t head_bytes = g.head_bytes(), v_bytes = g.k_plane_bytes();
    const int panel = g.bt * 128;
    auto store = [&](int t, int i, const uint4& y) {
        const int64_t at = s_at[t];
        if (at < 0) return;
        const bool v = i >= per_plane;
        const int of = v ? i - per_plane : i, chunk = of & ((1 << shift) - 1);
        *reinterpret_cast<uint4*>(p.c.pool + at + (of >> shift) * head_bytes + (v ? v_bytes : 0) + int64_t(chunk >> 3) * panel + (((chunk ^ s_slot[t]) & 7) << 4)) = y;
    };
    t = t0; i = i0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
        if (t < tokens) store(t, i, x[k]);
        advance(t, i);
    }
    for (; t < tokens; advance(t, i)) store(t, i, load(t, i));
    if (p.c.weights || p.c.positions)
        for (int c = tid; c < tokens * g.n_kv_heads; c += kThreads) {
            const int t = c / g.n_kv_heads, head = c - t * g.n_kv_heads;
            if (s_at[t] < 0) continue;
            const int64_t at = (int64_t(s_row[t]) * g.n_kv_heads + head) * p.c.slot_stride + s_slot[t];
            if (p.c.weights) p.c.weights[at] = 0.f;
            if (p.c.positions) p.c.positions[at] = p.token_positions[token0 + t];
        }
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppend& a, cudaStream_t s) {
    // as many tokens to a CTA as its threads have under way, fewer while there are SMs without work
    const int64_t chunks = int64_t(a.c.g.n_kv_heads) * a.c.g.dim_qk / 4, full = kThreads * kAhead / chunks, spread = a.n_tokens / (4 * 148);
    const int per_cta = int(full < 1 || spread < 1 ? 1 : full < spread ? (full < kMostTokens ? full : kMostTokens) : (spread < kMostTokens ? spread : kMostTokens));
    return launch_overlapped(paged_append_kernel, int((a.n_tokens + per_cta - 1) / per_cta), kThreads, size_t(0), s, a, per_cta);
}

}  // namespace ipkvi
