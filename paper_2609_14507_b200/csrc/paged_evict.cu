// Eviction from a paged cache by the weights that the attention added up: of every row and KV head with more than `budget` slots, the
// slots with the largest keys stay, a key being the weight, above all weights for the first and the recent tokens.
//
// A thread-block cluster takes one (row, KV head), every CTA of it a contiguous part of the slots, every warp a contiguous part of that:
//   1. the newest position (a maximum), then the keys, as integers of the same order, kept in shared memory;
//   2. the budget-th largest key, eight bits at a time: a histogram in every CTA, read by all through distributed shared memory;
//   3. slots above it are kept, and of those equal to it the lowest; ballots and prefix sums number the kept slots behind the budget
//      and the evicted ones before it, and the i-th of the ones meets the i-th of the others;
//   4. the warps of the cluster move the K and V rows, an even share each, whatever parts of the slots they come from.
// Bound by its synchronisations for small caches, by the 8 bytes of a slot and the 8 dim bytes of a moved token for large ones.
#include <cooperative_groups.h>

#include <atomic>

#include "kernels.h"
#include "launch.cuh"
#include "paged.h"
#include "plan.hpp"
#include "ptx.cuh"

namespace cg = cooperative_groups;

namespace ipkvi {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kMostCtas = 8;
constexpr int kCachedKeys = 24 * 1024;           // of a CTA, in shared memory; more are computed again where they are needed

struct Smem {
    uint32_t hist[2][256];
    int32_t newest, digit, need;
    int32_t scan[kWarps];
    int32_t count[3][kWarps];                    // of every warp: ties; kept slots behind the budget, evicted ones before it
};

// Larger is kept before smaller.  A NaN is less than every number.
__device__ __forceinline__ uint32_t key_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);         // -0 is 0
    return w != w ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
constexpr uint32_t kStays = 0xffffffffu;

__global__ void __launch_bounds__(kThreads) paged_evict_kernel(const __grid_constant__ PagedEvict p, const int ctas) {
    extern __shared__ uint32_t keys[];
    __shared__ Smem sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = int(cluster.block_rank()), pair = int(blockIdx.x) / ctas, H = p.c.g.n_kv_heads, row = pair / H, head = pair - row * H;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int capacity = p.c.max_blocks * p.c.g.bt, b = p.budget;
    int n = p.c.lengths[row];
    if (n < 0 || n > capacity) {
        if (tid == 0 && rank == 0 && head == 0 && p.status) atomicOr(p.status, kStatusBadPage);
        n = n < 0 ? 0 : capacity;
    }
    const int64_t slots0 = int64_t(pair) * p.c.slot_stride;
    const float* weights = p.c.weights + slots0;
    const int32_t* positions = p.c.positions + slots0;
    float* weights_out = p.weights_out + slots0;
    int32_t* positions_out = p.positions_out + slots0;
    int32_t* kept = p.kept ? p.kept + int64_t(pair) * b : nullptr;
    // this warp's slots
    const int per_cta = ((n + ctas - 1) / ctas + 31) & ~31, per_warp = (((per_cta + kWarps - 1) / kWarps) + 31) & ~31;
    const int cta0 = min(n, rank * per_cta), cta1 = min(n, cta0 + per_cta);
    const int w0 = min(cta1, cta0 + warp * per_warp), w1 = min(cta1, w0 + per_warp);
    auto stays_put = [&](int i) {                // a slot below the budget whose token is kept
        if (weights_out != weights) weights_out[i] = weights[i];
        if (positions_out != positions) positions_out[i] = positions[i];
        if (kept) kept[i] = i;
    };
    if (n <= b) {
        for (int i = w0 + lane; i < w1; i += 32) stays_put(i);
        return;
    }

    // ---- keys ----
    if (tid == 0) sm.newest = INT32_MIN;
    for (int i = tid; i < 512; i += kThreads) (&sm.hist[0][0])[i] = 0;
    __syncthreads();
    int newest = INT32_MIN;
    for (int i = w0 + lane; i < w1; i += 32) newest = max(newest, positions[i]);
    newest = __reduce_max_sync(0xffffffffu, newest);
    if (lane == 0) atomicMax(&sm.newest, newest);
    cluster.sync();
    for (int r = 0; r < ctas; ++r) newest = max(newest, *cluster.map_shared_rank(&sm.newest, r));
    const int64_t old = int64_t(newest) - p.recent;      // positions up to here are not recent
    const bool cached = per_cta <= kCachedKeys;
    auto make_key = [&](int i) {
        const int at = positions[i];
        return at < p.first || at > old ? kStays : key_of(weights[i]);
    };
    auto key = [&](int i) { return cached ? keys[i - cta0] : make_key(i); };

    // ---- the threshold ----
    int need = b;                                // of the keys that begin with `prefix`, as many are kept
    uint32_t prefix = 0;
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        uint32_t* hist = sm.hist[pass & 1];
        for (int i = w0 + lane; i < w1; i += 32) {
            uint32_t k;
            if (pass == 0) {
                k = make_key(i);
                if (cached) keys[i - cta0] = k;
            } else {
                k = key(i);
            }
            if (pass == 0 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        cluster.sync();
        // keys with a larger digit than this thread's
        int c = 0;
        if (tid < 256) {
            for (int r = 0; r < ctas; ++r) c += int(cluster.map_shared_rank(hist, r)[255 - tid]);
        }
        int x = c;
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) sm.scan[warp] = x;
        __syncthreads();
        int before = x - c;
        for (int w = 0; w < warp; ++w) before += sm.scan[w];
        if (tid < 256 && before < need && need <= before + c) { sm.digit = 255 - tid; sm.need = need - before; }
        // the other histogram is the next pass's: every CTA has read it, or it would not have come to this pass's barrier
        if (pass < 3)
            for (int i = tid; i < 256; i += kThreads) sm.hist[(pass + 1) & 1][i] = 0;
        __syncthreads();
        prefix |= uint32_t(sm.digit) << shift;
        need = sm.need;
    }
    const uint32_t threshold = prefix;           // `need` of the keys equal to it are kept, the lowest slots'

    // ---- numbers ----
    // sums over the warps before this one, of the whole cluster
    auto before_us = [&](int which) {
        int s = 0;
        for (int r = 0; r <= rank; ++r) {
            const int32_t* c = cluster.map_shared_rank(&sm.count[which][0], r);
            for (int w = lane; w < (r < rank ? kWarps : warp); w += 32) s += c[w];
        }
        return int(__reduce_add_sync(0xffffffffu, unsigned(s)));
    };
    int ties = 0;
    for (int i = w0 + lane; i < w1; i += 32) ties += key(i) == threshold;
    ties = int(__reduce_add_sync(0xffffffffu, unsigned(ties)));
    if (lane == 0) sm.count[0][warp] = ties;
    cluster.sync();
    const int ties0 = before_us(0);
    // calls f(slot, kept) for all slots of the warp, a group of 32 at a time
    auto for_slots = [&](auto&& f) {
        int seen = ties0;
        for (int i0 = w0; i0 < w1; i0 += 32) {
            const int i = i0 + lane;
            const uint32_t k = i < w1 ? key(i) : 0u;
            const bool tie = i < w1 && k == threshold;
            const unsigned tied = __ballot_sync(0xffffffffu, tie);
            const bool keep = i < w1 && (k > threshold || (tie && seen + __popc(tied & ((1u << lane) - 1u)) < need));
            seen += __popc(tied);
            f(i, keep);
        }
    };
    int behind = 0, holes = 0;
    for_slots([&](int i, bool keep) {
        behind += __popc(__ballot_sync(0xffffffffu, keep && i >= b));
        holes += __popc(__ballot_sync(0xffffffffu, i < w1 && !keep && i < b));
    });
    if (lane == 0) { sm.count[1][warp] = behind; sm.count[2][warp] = holes; }
    cluster.sync();
    int behind0 = before_us(1), holes0 = before_us(2), moves = 0;
    for (int r = 0; r < ctas; ++r) {
        const int32_t* c = cluster.map_shared_rank(&sm.count[2][0], r);
        for (int w = lane; w < kWarps; w += 32) moves += c[w];
    }
    moves = int(__reduce_add_sync(0xffffffffu, unsigned(moves)));
    int32_t* from = p.moved + int64_t(pair) * 2 * p.most_moved;
    int32_t* into = from + p.most_moved;
    for_slots([&](int i, bool keep) {
        const bool comes = keep && i >= b, hole = i < w1 && !keep && i < b;
        const unsigned coming = __ballot_sync(0xffffffffu, comes), open = __ballot_sync(0xffffffffu, hole), lower = (1u << lane) - 1u;
        if (comes) from[behind0 + __popc(coming & lower)] = i;
        if (hole) into[holes0 + __popc(open & lower)] = i;
        behind0 += __popc(coming);
        holes0 += __popc(open);
        if (keep && i < b) stays_put(i);
    });
    cluster.sync();                              // the lists are written; nobody reads another CTA's shared memory any more

    // ---- moves ----
    const BlockGeom g = p.c.g;
    const int32_t* table = p.c.table + row * p.c.table_stride;
    const int per_row = g.dim_qk / 8, chunks = 2 * per_row, warps = ctas * kWarps;
    constexpr int kAtOnce = 4;
    for (int i0 = rank * kWarps + warp; i0 < moves; i0 += warps * kAtOnce) {
        uint4 x[kAtOnce];
        char* to[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int i = i0 + k * warps;
            to[k] = nullptr;
            if (i >= moves) continue;
            const int src = from[i], dst = into[i];
            const int src_page = table[src / g.bt], dst_page = table[dst / g.bt];
            if (lane == 0) {
                weights_out[dst] = weights[src];
                positions_out[dst] = positions[src];
                if (kept) kept[dst] = src;
            }
            if (src_page < 0 || src_page >= p.c.n_blocks || dst_page < 0 || dst_page >= p.c.n_blocks) {
                if (lane == 0 && p.status) atomicOr(p.status, kStatusBadPage);
                continue;
            }
            if (lane < chunks) {
                const int chunk = lane < per_row ? lane : lane - per_row;
                const int64_t at = head * g.head_bytes() + (lane < per_row ? 0 : g.k_plane_bytes());
                x[k] = *reinterpret_cast<const uint4*>(p.c.pool + src_page * g.block_bytes() + at + tile_chunk_offset(g.bt, src % g.bt, chunk));
                to[k] = p.c.pool + dst_page * g.block_bytes() + at + tile_chunk_offset(g.bt, dst % g.bt, chunk);
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (to[k]) *reinterpret_cast<uint4*>(to[k]) = x[k];
    }
}

}  // namespace

cudaError_t launch_paged_evict(const PagedEvict& a, cudaStream_t s) {
    const int pairs = a.c.n_rows * a.c.g.n_kv_heads, slots = a.c.max_blocks * a.c.g.bt;
    int ctas = 1;
    while (ctas < kMostCtas && int64_t(pairs) * ctas * 2 <= 2 * kSmCount && slots / (ctas * 2) >= 1024) ctas *= 2;
    const int per_cta = ((slots + ctas - 1) / ctas + 31) & ~31;
    const size_t smem = size_t(per_cta <= kCachedKeys ? per_cta : kCachedKeys) * 4;
    static std::atomic<bool> configured[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(paged_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kCachedKeys * 4);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(pairs * ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(ctas); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = overlap_launches() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, paged_evict_kernel, a, ctas);
}

}  // namespace ipkvi
