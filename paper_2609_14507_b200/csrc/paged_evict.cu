// Eviction from a paged cache by the weights that the attention added up: of every row and KV head with more than `budget` slots, the
// slots with the largest keys stay, a key being the weight, above all weights for the first and the recent tokens.
//
// A thread-block cluster takes one (row, KV head), every CTA of it a contiguous part of the slots, every warp a contiguous part of that:
//   1. weights and positions come into shared memory by two bulk copies; the newest position (a maximum), then the keys, as integers of
//      the same order;
//   2. the budget-th largest key, eight bits at a time: a histogram in every CTA, read by all through distributed shared memory;
//   3. slots above it are kept, and of those equal to it the lowest; ballots and prefix sums number the kept slots behind the budget
//      and the evicted ones before it, and the i-th of the ones meets the i-th of the others;
//   4. the warps of the cluster move the K and V rows, an even share each, whatever parts of the slots they come from.
// Where one slot goes (a full cache that makes room for the next token), it is the smallest key, of equal ones the last slot's: one
// minimum in place of 2 and 3.
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
constexpr int kHeldSlots = 24 * 1024;            // of a CTA, 8 bytes each in shared memory; of more, keys are computed again where they are needed
constexpr int kAtOnce = 8;                       // rows that a warp has under way

struct Smem {
    uint64_t landed;
    unsigned long long least;
    uint32_t hist[2][256];
    int32_t newest, digit, need, gave_up;
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
    extern __shared__ __align__(16) uint32_t held[];     // weights, then keys, of the CTA's slots; positions behind them
    __shared__ Smem sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = int(cluster.block_rank()), pair = int(blockIdx.x) / ctas, H = p.c.g.n_kv_heads, row = pair / H, head = pair - row * H;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        ptx::mbar_init(ptx::smem_addr(&sm.landed), 1);
        ptx::mbar_fence_init();
        sm.newest = INT32_MIN; sm.least = ~0ull; sm.gave_up = 0;
    }
    sm.hist[tid >> 8][tid & 255] = 0;
    static_assert(kThreads == 512, "a thread clears one word of the histograms");
    __syncthreads();
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
    const bool in_place = weights_out == weights && positions_out == positions;
    // this warp's slots
    const int per_cta = ((n + ctas - 1) / ctas + 31) & ~31, per_warp = (((per_cta + kWarps - 1) / kWarps) + 31) & ~31;
    const int cta0 = min(n, rank * per_cta), cta1 = min(n, cta0 + per_cta);
    const int w0 = min(cta1, cta0 + warp * per_warp), w1 = min(cta1, w0 + per_warp);
    if (n <= b && in_place && !kept) return;
    const bool holds = per_cta <= kHeldSlots;
    const float* w_held = reinterpret_cast<const float*>(held);
    const int32_t* p_held = reinterpret_cast<const int32_t*>(held) + p.held;
    if (holds && cta1 > cta0) {
        const uint32_t bytes = uint32_t(cta1 - cta0 + 3) / 4 * 16;      // (whole 16 bytes: the slots behind n are there, the stride is a multiple of four)
        if (tid == 0) {
            const uint32_t bar = ptx::smem_addr(&sm.landed);
            ptx::mbar_expect_tx(bar, 2 * bytes);
            ptx::bulk_g2s(ptx::smem_addr(held), weights + cta0, bytes, bar);
            ptx::bulk_g2s(ptx::smem_addr(p_held), positions + cta0, bytes, bar);
        }
        if (!ptx::mbar_wait(ptx::smem_addr(&sm.landed), 0)) sm.gave_up = 1;
    }
    const bool lost = __syncthreads_or(sm.gave_up);      // nothing is evicted then; the CTAs of the cluster hear of it below
    if (lost && tid == 0) {
        if (p.status) atomicOr(p.status, kStatusNoTile);
        if (!ptx::mbar_wait(ptx::smem_addr(&sm.landed), 0) && p.status) atomicOr(p.status, kStatusCopyNotLanded);
    }
    auto weight = [&](int i) { return holds ? w_held[i - cta0] : weights[i]; };
    auto position = [&](int i) { return holds ? p_held[i - cta0] : positions[i]; };
    if (n <= b) {
        if (lost) return;
        for (int i = w0 + lane; i < w1; i += 32) {
            if (weights_out != weights) weights_out[i] = weight(i);
            if (positions_out != positions) positions_out[i] = position(i);
            if (kept) kept[i] = i;
        }
        return;
    }

    // ---- keys ----
    int newest = INT32_MIN;
    for (int i = w0 + lane; i < w1; i += 32) newest = max(newest, position(i));
    newest = __reduce_max_sync(0xffffffffu, newest);
    if (lane == 0) atomicMax(&sm.newest, newest);
    cluster.sync();
    bool gave_up = false;
    for (int r = 0; r < ctas; ++r) {
        newest = max(newest, *cluster.map_shared_rank(&sm.newest, r));
        gave_up |= *cluster.map_shared_rank(&sm.gave_up, r) != 0;
    }
    const int64_t old = int64_t(newest) - p.recent;      // positions up to here are not recent
    auto key = [&](int i) {
        const int at = position(i);
        return at < p.first || at > old ? kStays : key_of(weight(i));
    };
    // a slot below the budget whose token stays where it is
    auto stays_put = [&](int i) {
        if (weights_out != weights) weights_out[i] = weight(i);
        if (positions_out != positions) positions_out[i] = position(i);
        if (kept) kept[i] = i;
    };
    const BlockGeom g = p.c.g;
    const int32_t* table = p.c.table + row * p.c.table_stride;
    const int per_row = g.dim_qk / 8, chunks = 2 * per_row;
    const int chunk = lane < per_row ? lane : lane - per_row;
    const int64_t in_block = head * g.head_bytes() + (lane < per_row ? 0 : g.k_plane_bytes());      // of this lane's plane
    auto page_of = [&](int slot) {
        const int page = table[slot / g.bt];
        return page >= 0 && page < p.c.n_blocks ? page : -1;
    };
    auto place = [&](int page, int slot) { return p.c.pool + page * g.block_bytes() + in_block + tile_chunk_offset(g.bt, slot % g.bt, chunk); };

    if (gave_up) {
        cluster.sync();                          // (the others read this CTA's shared memory until here)
        return;
    }

    // ---- one slot goes ----
    if (n == b + 1) {
        unsigned long long least = ~0ull;        // key, then the slot, the last one first
        for (int i = w0 + lane; i < w1; i += 32) {
            const unsigned long long x = (static_cast<unsigned long long>(key(i)) << 32) | uint32_t(~i);
            least = x < least ? x : least;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            const unsigned long long x = __shfl_xor_sync(0xffffffffu, least, d);
            least = x < least ? x : least;
        }
        if (lane == 0) atomicMin(&sm.least, least);
        cluster.sync();
        least = ~0ull;
        for (int r = 0; r < ctas; ++r) {
            const unsigned long long x = *cluster.map_shared_rank(&sm.least, r);
            least = x < least ? x : least;
        }
        const int gone = int(~uint32_t(least));
        if (!in_place || kept)
            for (int i = w0 + lane; i < w1; i += 32)
                if (i < b && i != gone) stays_put(i);
        cluster.sync();                          // nobody reads another CTA's shared memory any more
        if (gone == b || rank != 0 || warp != 0) return;
        const int src_page = page_of(b), dst_page = page_of(gone);
        if (lane == 0) {
            weights_out[gone] = weights[b];
            positions_out[gone] = positions[b];
            if (kept) kept[gone] = b;
        }
        if (src_page >= 0 && dst_page >= 0) {
            if (lane < chunks) *reinterpret_cast<uint4*>(place(dst_page, gone)) = *reinterpret_cast<const uint4*>(place(src_page, b));
        } else if (lane == 0 && p.status) {
            atomicOr(p.status, kStatusBadPage);
        }
        return;
    }

    // ---- the threshold ----
    int need = b;                                // of the keys that begin with `prefix`, as many are kept
    uint32_t prefix = 0;
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        uint32_t* hist = sm.hist[pass & 1];
        for (int i = w0 + lane; i < w1; i += 32) {
            const uint32_t k = key(i);
            if (pass == 0 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        cluster.sync();
        // keys with a larger digit than this thread's
        int c = 0;
        if (tid < 256)
            for (int r = 0; r < ctas; ++r) c += int(cluster.map_shared_rank(hist, r)[255 - tid]);
        int x = c;
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) sm.scan[warp] = x;
        // the other histogram is the next pass's: every CTA has read it, or it would not have come to this pass's barrier
        if (tid >= 256) sm.hist[(pass + 1) & 1][tid - 256] = 0;
        __syncthreads();
        int before = x - c;
        for (int w = 0; w < 8; ++w) before += w < warp ? sm.scan[w] : 0;
        if (tid < 256 && before < need && need <= before + c) { sm.digit = 255 - tid; sm.need = need - before; }
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
            if (lane < (r < rank ? kWarps : warp)) s += c[lane];
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
        if (lane < kWarps) moves += c[lane];
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

    // ---- moves: a warp looks 32 of them up at once, a lane each, then moves their rows, a 16-byte chunk of each a lane ----
    const int warps = ctas * kWarps, each = (moves + warps - 1) / warps, first = min(moves, (rank * kWarps + warp) * each), last = min(moves, first + each);
    for (int i0 = first; i0 < last; i0 += 32) {
        int src = 0, dst = 0, src_page = -1, dst_page = -1;
        if (i0 + lane < last) {
            src = from[i0 + lane]; dst = into[i0 + lane];
            src_page = page_of(src); dst_page = page_of(dst);
            weights_out[dst] = weights[src];
            positions_out[dst] = positions[src];
            if (kept) kept[dst] = src;
            if (src_page < 0 || dst_page < 0) {
                src_page = -1;
                if (p.status) atomicOr(p.status, kStatusBadPage);
            }
        }
        const int count = min(32, last - i0);
        for (int k0 = 0; k0 < count; k0 += kAtOnce) {
            uint4 x[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int page = __shfl_sync(0xffffffffu, src_page, k0 + k), slot = __shfl_sync(0xffffffffu, src, k0 + k);
                if (page >= 0 && lane < chunks) x[k] = *reinterpret_cast<const uint4*>(place(page, slot));
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int there = __shfl_sync(0xffffffffu, src_page, k0 + k), page = __shfl_sync(0xffffffffu, dst_page, k0 + k), slot = __shfl_sync(0xffffffffu, dst, k0 + k);
                if (there >= 0 && lane < chunks) *reinterpret_cast<uint4*>(place(page, slot)) = x[k];
            }
        }
    }
}

}  // namespace

cudaError_t launch_paged_evict(PagedEvict& a, cudaStream_t s) {
    const int pairs = a.c.n_rows * a.c.g.n_kv_heads, slots = a.c.max_blocks * a.c.g.bt;
    int ctas = 1;
    while (ctas < kMostCtas && int64_t(pairs) * ctas * 2 <= 2 * kSmCount && slots / (ctas * 2) >= 1024) ctas *= 2;
    const int per_cta = ((slots + ctas - 1) / ctas + 31) & ~31;
    a.held = per_cta <= kHeldSlots ? per_cta : kHeldSlots;
    static std::atomic<bool> configured[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(paged_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldSlots * 8);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(pairs * ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = size_t(a.held) * 8;
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
