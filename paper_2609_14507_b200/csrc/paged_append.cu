// New tokens into the pages of a paged cache: one warp per token moves the K and V rows of all its KV heads, 16 bytes a lane, and sets
// the slots' positions and weights.  Bound by the bytes (read once, written once) and, for a decode step, by the launch: the
// loads of K and V go out before the table is looked up, so that one latency covers both.
#include "launch.cuh"
#include "paged.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kAhead = 8;

__global__ void __launch_bounds__(kThreads) paged_append_kernel(const __grid_constant__ PagedAppend p) {
    const int lane = threadIdx.x & 31;
    const int64_t token = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (token >= p.n_tokens) return;
    const BlockGeom g = p.c.g;
    const int per_row = g.dim_qk / 8, per_head = 2 * per_row, chunks = g.n_kv_heads * per_head;      // 16-byte chunks: K row, V row of a head
    auto load = [&](int c) {
        const int head = c / per_head, i = c - head * per_head;
        const char* src = i < per_row ? p.k + token * p.k_token : p.v + token * p.v_token;
        return __ldg(reinterpret_cast<const uint4*>(src + (int64_t(head) * per_row + (i < per_row ? i : i - per_row)) * 16));
    };
    uint4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (lane + 32 * k < chunks) x[k] = load(lane + 32 * k);
    // the token's row, and which of its new tokens it is
    int row, behind;                             // behind: new tokens of the row from this one on
    if (p.row_start) {
        int lo = 0, hi = p.c.n_rows - 1;         // the last row that begins at or before the token
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.row_start[mid] <= token) lo = mid; else hi = mid - 1;
        }
        row = lo;
        if (token < p.row_start[row] || token >= p.row_start[row + 1]) return;       // behind the last row's
        behind = int(p.row_start[row + 1] - token);
    } else {
        row = int(token);
        behind = 1;
    }
    const int64_t slot = int64_t(p.c.lengths[row]) - behind;
    if (slot < 0) return;                        // not counted by the length
    int page = -1;
    if (slot < int64_t(p.c.max_blocks) * g.bt) page = p.c.table[row * p.c.table_stride + slot / g.bt];
    if (page < 0 || page >= p.c.n_blocks) {
        if (lane == 0 && p.status) atomicOr(p.status, kStatusBadPage);
        return;
    }
    const int t = int(slot % g.bt);
    char* block = p.c.pool + page * g.block_bytes();
    auto store = [&](int c, const uint4& y) {
        const int head = c / per_head, i = c - head * per_head;
        char* plane = block + head * g.head_bytes() + (i < per_row ? 0 : g.k_plane_bytes());
        *reinterpret_cast<uint4*>(plane + tile_chunk_offset(g.bt, t, i < per_row ? i : i - per_row)) = y;
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (lane + 32 * k < chunks) store(lane + 32 * k, x[k]);
    for (int c = lane + 32 * kAhead; c < chunks; c += 32) store(c, load(c));
    if (p.c.weights || p.c.positions)
        for (int head = lane; head < g.n_kv_heads; head += 32) {
            const int64_t at = (int64_t(row) * g.n_kv_heads + head) * p.c.slot_stride + slot;
            if (p.c.weights) p.c.weights[at] = 0.f;
            if (p.c.positions) p.c.positions[at] = p.token_positions[token];
        }
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppend& a, cudaStream_t s) {
    return launch_overlapped(paged_append_kernel, int((a.n_tokens + kWarps - 1) / kWarps), kThreads, size_t(0), s, a);
}

}  // namespace ipkvi
