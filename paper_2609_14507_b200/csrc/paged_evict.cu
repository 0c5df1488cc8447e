// Eviction from a paged cache by the weights that the attention added up: of every row and KV head with more than `budget` slots, the
// slots with the largest keys stay, a key being the weight, above all weights for the first and the recent tokens.
//
// A thread-block cluster takes one (row, KV head), every CTA of it a contiguous part of the slots, every warp a contiguous part of that:
//   1. weights and positions come into shared memory by two bulk copies; the newest position (a maximum), then the keys, as integers of
//      the same order;
//   2. the budget-th largest key, eight bits at a time: a histogram in every CTA, sent to all of the cluster;
//   3. slots above it are kept, and of those equal to it the lowest; prefix sums number the kept slots behind the budget and the evicted
//      ones before it, and the i-th of the ones meets the i-th of the others;
//   4. the warps of the cluster move the K and V rows, an even share each, whatever parts of the slots they come from.
// Where one slot goes (a full cache that makes room for the next token), it is the smallest key, of equal ones the last slot's: one
// minimum in place of 2 and 3.
// Bound by its chain of passes, 1.7 us each in a cluster of eight with 1024 threads (the sending itself takes 0.15, counting 0.6), then by the rows moved in
// pieces of 128 bytes.  Measured (a few replays of a graph, 1965 MHz): 512 pairs, one of 4096 slots goes in every one, in place 8.2 us (17 MB read), 128 such pairs 5.6,
// 8 5.1; with arrays apart 512 12.0; 512 pairs of 4000 to 4096 slots of which 32 are cut and 480 copied to arrays apart 9.6; 8 pairs of 32K to 4K 24.2 us, 7 to 9 of them
// for 29 MB of rows (all weights equal: 21.1); 8 of 3K to 1K 16.6 (equal: 13.3); 8 pairs of 261 to 243 slots 8.2 us.
#include <atomic>

#include "kernels.h"
#include "launch.cuh"
#include "paged.h"
#include "plan.hpp"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kMostCtas = 8;
constexpr int kHeldSlots = 24 * 1024;            // of a CTA, 8 bytes each in shared memory; of more, keys are computed again where they are needed
constexpr int kMeetings = 6;                     // the newest position; the smallest key, or the numbers of moves; a pass each
constexpr int kAtOnce = 8;                       // rows that a warp has under way

template <int THREADS>
struct Smem {
    static constexpr int kWarps = THREADS / 32;
    uint64_t landed;
    uint64_t told[kMeetings];                    // what the CTAs of the cluster send one another, eight bytes each or a histogram
    unsigned long long got[2][kMostCtas];
    unsigned long long least;
    alignas(16) uint32_t hist[2][256];
    int32_t newest, digit, need, ties, all, gave_up;
    int32_t scan[8];
    int32_t count[3][kWarps];                    // of every warp: ties; kept slots behind the budget, evicted ones before it
    int32_t total[2];                            // of the CTA, the latter two
};

// Larger is kept before smaller.  A NaN is less than every number.
__device__ __forceinline__ uint32_t key_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);         // -0 is 0
    return w != w ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
constexpr uint32_t kStays = 0xffffffffu;

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) paged_evict_kernel(const __grid_constant__ PagedEvict p, const int ctas) {
    constexpr int kWarps = THREADS / 32;
    extern __shared__ __align__(16) uint32_t held[];     // weights, then keys, of the CTA's slots; positions behind them
    __shared__ Smem<THREADS> sm;
    const int rank = int(blockIdx.x) % ctas, pair = int(blockIdx.x) / ctas, H = p.c.g.n_kv_heads, row = pair / H, head = pair - row * H;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint4* const hists = reinterpret_cast<uint4*>(held + 2 * p.held);      // [2][ctas][64]: the cluster's histograms, of two passes in turn
    auto meet = [&]() {                          // all CTAs of the cluster
        if (ctas == 1) { __syncthreads(); return; }
        ptx::cluster_arrive();
        ptx::cluster_wait();
    };
    // A meeting whose outcome every CTA needs: each sends its part to all, counted by a barrier that serves once, and waits for theirs.
    // One way through the cluster's network in place of the cluster's barrier and a read there and back (8 pairs of 32K to 4K 25.7 to 24.0 us).
    auto there = [&](const void* here, int cta) { return ptx::at_rank(ptx::smem_addr(here), cta); };
    auto tell = [&](int meeting, int which, unsigned long long x) {        // (warp 0)
        if (lane < ctas) ptx::st_async_b64(there(&sm.got[which][rank], lane), x, there(&sm.told[meeting], lane));
    };
    bool lost = false;                           // a wait ran out
    auto hear = [&](int meeting) { lost |= !ptx::mbar_wait_cluster(ptx::smem_addr(&sm.told[meeting]), 0); };
    // after such a wait, by all threads of the CTA: nothing moves in the cluster, and no CTA leaves before the others have sent
    auto give_up = [&]() {
        if (tid == 0 && p.status) atomicOr(p.status, kStatusNoTile);
        if (tid < ctas) asm volatile("st.shared::cluster.u32 [%0], 1;" ::"r"(there(&sm.gave_up, tid)) : "memory");
        __syncwarp();
        meet();
    };
    if (tid == 0) {
        ptx::mbar_init(ptx::smem_addr(&sm.landed), 1);
        for (int k = 0; k < kMeetings; ++k) ptx::mbar_init(ptx::smem_addr(&sm.told[k]), 1);
        ptx::mbar_fence_init();
        for (int k = 0; k < kMeetings; ++k) ptx::mbar_expect_tx(ptx::smem_addr(&sm.told[k]), uint32_t(ctas) * (k < 2 ? 8u : 1024u));
        sm.newest = INT32_MIN; sm.least = ~0ull; sm.gave_up = 0;
    }
    if (tid < 256) sm.hist[0][tid] = sm.hist[1][tid] = 0;
    __syncthreads();
    if (ctas > 1) ptx::cluster_arrive();         // the barriers are there: waited for before the first of them is used
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (tid * 32 < p.c.max_blocks) {             // the row's table comes into the L1 cache meanwhile
        int32_t unused;
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(unused) : "l"(p.c.table + row * p.c.table_stride + tid * 32));
    }
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
    // this warp's slots, in groups of 128: four a lane
    const int per_cta = ((n + ctas - 1) / ctas + 31) & ~31, per_warp = (((per_cta + kWarps - 1) / kWarps) + 127) & ~127;
    const int cta0 = min(n, rank * per_cta), cta1 = min(n, cta0 + per_cta);
    const int w0 = min(cta1, cta0 + warp * per_warp), w1 = min(cta1, w0 + per_warp);
    auto stays_put = [&](int i) {                // a slot below the budget whose token stays where it is
        if (weights_out != weights) weights_out[i] = weights[i];
        if (positions_out != positions) positions_out[i] = positions[i];
        if (kept) kept[i] = i;
    };
    if (n <= b) {                                // all stay: copied, four slots a lane, where they go to arrays of their own
        if (ctas > 1) ptx::cluster_wait();
        if (in_place && !kept) return;
        constexpr int kGroups = 4;
        for (int i0 = w0 + 4 * lane; i0 - 4 * lane < w1; i0 += 128 * kGroups) {
            float4 w[kGroups];
            int4 at[kGroups];
#pragma unroll
            for (int k = 0; k < kGroups; ++k)
                if (i0 + 128 * k + 3 < w1) {
                    w[k] = *reinterpret_cast<const float4*>(weights + i0 + 128 * k);
                    at[k] = *reinterpret_cast<const int4*>(positions + i0 + 128 * k);
                }
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                const int i = i0 + 128 * k;
                if (i + 3 < w1) {
                    if (weights_out != weights) *reinterpret_cast<float4*>(weights_out + i) = w[k];
                    if (positions_out != positions) *reinterpret_cast<int4*>(positions_out + i) = at[k];
                } else {
                    for (int e = i; e < w1; ++e) {
                        if (weights_out != weights) weights_out[e] = weights[e];
                        if (positions_out != positions) positions_out[e] = positions[e];
                    }
                }
            }
        }
        if (kept)
            for (int i = w0 + lane; i < w1; i += 32) kept[i] = i;
        return;
    }

    // ---- keys ----
    const bool holds = per_cta <= kHeldSlots;
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
    if (__syncthreads_or(sm.gave_up) && tid == 0) {      // nothing is evicted then; the CTAs of the cluster hear of it below
        if (p.status) atomicOr(p.status, kStatusNoTile);
        if (!ptx::mbar_wait(ptx::smem_addr(&sm.landed), 0) && p.status) atomicOr(p.status, kStatusCopyNotLanded);
    }
    int newest = INT32_MIN;
    for (int i = w0 + 4 * lane; i < w1; i += 128) {
        const int4 x = holds ? *reinterpret_cast<const int4*>(p_held + (i - cta0)) : *reinterpret_cast<const int4*>(positions + i);
        newest = max(newest, x.x);
        if (i + 1 < w1) newest = max(newest, x.y);
        if (i + 2 < w1) newest = max(newest, x.z);
        if (i + 3 < w1) newest = max(newest, x.w);
    }
    newest = __reduce_max_sync(0xffffffffu, newest);
    if (lane == 0) atomicMax(&sm.newest, newest);
    __syncthreads();
    newest = sm.newest;
    if (ctas > 1) {
        ptx::cluster_wait();
        if (warp == 0) tell(0, 0, static_cast<unsigned long long>(uint32_t(sm.gave_up)) << 32 | uint32_t(newest));
        hear(0);
        if (__syncthreads_or(lost)) return give_up();
        const unsigned long long x = lane < ctas ? sm.got[0][lane] : uint32_t(INT32_MIN);
        newest = __reduce_max_sync(0xffffffffu, int(uint32_t(x)));
        if (__any_sync(0xffffffffu, x >> 32 != 0)) return meet();
    } else if (sm.gave_up) {
        return;
    }
    const int64_t old = int64_t(newest) - p.recent;      // positions up to here are not recent
    // the keys of slots i .. i + 3 from weights and positions
    auto make_keys = [&](int i) {
        const float4 w = holds ? *reinterpret_cast<const float4*>(held + (i - cta0)) : *reinterpret_cast<const float4*>(weights + i);
        const int4 at = holds ? *reinterpret_cast<const int4*>(p_held + (i - cta0)) : *reinterpret_cast<const int4*>(positions + i);
        auto one = [&](float w, int at) { return at < p.first || at > old ? kStays : key_of(w); };
        return make_uint4(one(w.x, at.x), one(w.y, at.y), one(w.z, at.z), one(w.w, at.w));
    };
    // calls f(i, keys) for all groups of the warp, i the lane's first slot; keys[e] counts if i + e < w1
    auto for_groups = [&](auto&& f) {
        for (int i = w0 + 4 * lane; i - 4 * lane < w1; i += 128) {
            uint4 k = make_uint4(0u, 0u, 0u, 0u);
            if (i < w1) k = holds ? *reinterpret_cast<const uint4*>(held + (i - cta0)) : make_keys(i);
            const uint32_t keys[4] = {k.x, k.y, k.z, k.w};
            f(i, keys);
        }
    };
    if (holds && n != b + 1)
        for (int i = w0 + 4 * lane; i < w1; i += 128) *reinterpret_cast<uint4*>(held + (i - cta0)) = make_keys(i);

    const BlockGeom g = p.c.g;
    const int32_t* table = p.c.table + row * p.c.table_stride;
    const int per_row = g.dim_qk / 8, chunks = 2 * per_row;
    const int chunk = lane < per_row ? lane : lane - per_row;
    // of this lane's chunk in a block, apart from the slot's row and the swizzle
    char* const lane_at = p.c.pool + head * g.head_bytes() + (lane < per_row ? 0 : g.k_plane_bytes()) + (chunk >> 3) * int64_t(g.bt) * 128;
    // where a slot's row begins, from the pool on; -1: its page is bad
    auto row_at = [&](int slot) {
        const int j = slot / g.bt, page = table[j];
        return page >= 0 && page < p.c.n_blocks ? page * g.block_bytes() + (slot - j * g.bt) * 128 : int64_t(-1);
    };
    auto swizzle = [&](int slot) { return ((chunk & 7) ^ (slot & 7)) << 4; };

    // ---- one slot goes ----
    if (n == b + 1) {
        unsigned long long least = ~0ull;        // key, then the slot, the last one first
        for (int i = w0 + 4 * lane; i < w1; i += 128) {
            const uint4 k = make_keys(i);
            const uint32_t keys[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned long long x = (static_cast<unsigned long long>(keys[e]) << 32) | uint32_t(~(i + e));
                if (i + e < w1 && x < least) least = x;
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            const unsigned long long x = __shfl_xor_sync(0xffffffffu, least, d);
            least = x < least ? x : least;
        }
        if (lane == 0) atomicMin(&sm.least, least);
        __syncthreads();
        least = sm.least;
        if (ctas > 1) {
            if (warp == 0) tell(1, 1, least);
            hear(1);
            if (__syncthreads_or(lost)) return give_up();
            least = sm.got[1][lane & (ctas - 1)];
#pragma unroll
            for (int d = kMostCtas / 2; d > 0; d >>= 1) {
                const unsigned long long x = __shfl_xor_sync(0xffffffffu, least, d);
                least = x < least ? x : least;
            }
            ptx::cluster_arrive();               // (no CTA leaves before the others have heard it)
        }
        const int gone = int(~uint32_t(least));
        if (!in_place || kept)
            for (int i = w0 + lane; i < w1; i += 32)
                if (i < b && i != gone) {
                    if (weights_out != weights) weights_out[i] = holds ? __uint_as_float(held[i - cta0]) : weights[i];
                    if (positions_out != positions) positions_out[i] = holds ? p_held[i - cta0] : positions[i];
                    if (kept) kept[i] = i;
                }
        if (ctas > 1) ptx::cluster_wait();
        if (gone == b || rank != 0 || warp != 0) return;
        const int64_t src_at = row_at(b), dst_at = row_at(gone);
        if (lane == 0) {
            weights_out[gone] = weights[b];
            positions_out[gone] = positions[b];
            if (kept) kept[gone] = b;
        }
        if (src_at >= 0 && dst_at >= 0) {
            if (lane < chunks) *reinterpret_cast<uint4*>(lane_at + dst_at + swizzle(gone)) = *reinterpret_cast<const uint4*>(lane_at + src_at + swizzle(b));
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
        for_groups([&](int i, const uint32_t (&keys)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < w1 && (pass == 0 || (keys[e] >> (shift + 8)) == (prefix >> (shift + 8)))) atomicAdd(&hist[(keys[e] >> shift) & 255], 1u);
        });
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // (the histogram is sent by the copy engine)
        __syncthreads();
        // keys with a larger digit than this thread's
        int c = 0, lower = 0;                    // of all CTAs; of those before this one
        if (ctas > 1) {
            uint4* const to = hists + (pass & 1) * ctas * 64;
            if (tid < ctas) ptx::bulk_s2s(there(to + rank * 64, tid), ptx::smem_addr(hist), 1024, there(&sm.told[2 + pass], tid));
            hear(2 + pass);
            if (tid < 256) {
                const uint32_t* of = reinterpret_cast<const uint32_t*>(to) + 255 - tid;
#pragma unroll
                for (int r = 0; r < kMostCtas; ++r) {
                    const int x = r < ctas ? int(of[r * 256]) : 0;
                    c += x;
                    if (r < rank) lower += x;
                }
            }
        } else if (tid < 256) {
            c = int(hist[255 - tid]);
        }
        int x = c;
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31 && warp < 8) sm.scan[warp] = x;
        // the other histogram is the next pass's (a CTA that sends into the room of two passes ago has heard from all that they are past it)
        if (tid < 256) sm.hist[(pass + 1) & 1][tid] = 0;
        __syncthreads();
        int before = x - c;
#pragma unroll
        for (int w = 0; w < 8; ++w) before += w < warp ? sm.scan[w] : 0;
        if (tid < 256 && before < need && need <= before + c) { sm.digit = 255 - tid; sm.need = need - before; sm.ties = lower; sm.all = need == before + c; }
        if (__syncthreads_or(lost)) return give_up();
        prefix |= uint32_t(sm.digit) << shift;
        need = sm.need;
        if (sm.all && pass < 3) {                // all keys that begin so are kept (most often the one that does): the bits below do not matter
            --prefix;
            need = 0;
            break;
        }
    }
    const uint32_t threshold = prefix;           // `need` of the keys equal to it are kept, the lowest slots'

    // ---- numbers ----
    auto warp_scan = [&](int x) {                // sums up to and with this lane
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        return x;
    };
    // warp 0: turns counts by warp into the sums before them in the CTA; returns the CTA's
    auto scan = [&](int which) {
        const int c = lane < kWarps ? sm.count[which][lane] : 0, upto = warp_scan(c);
        if (lane < kWarps) sm.count[which][lane] = upto - c;
        return __shfl_sync(0xffffffffu, upto, 31);
    };
    int ties = 0;
    for_groups([&](int i, const uint32_t (&keys)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) ties += i + e < w1 && keys[e] == threshold;
    });
    ties = int(__reduce_add_sync(0xffffffffu, unsigned(ties)));
    if (lane == 0) sm.count[0][warp] = ties;
    __syncthreads();
    if (warp == 0) scan(0);
    __syncthreads();
    const int ties0 = sm.ties + sm.count[0][warp];       // (the last pass counted those of the CTAs before this one)
    // calls f(i, keep) for all groups, bit e of keep: slot i + e is kept
    auto for_kept = [&](auto&& f) {
        int seen = ties0;
        for_groups([&](int i, const uint32_t (&keys)[4]) {
            unsigned above = 0, tied = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < w1) {
                    above |= unsigned(keys[e] > threshold) << e;
                    tied |= unsigned(keys[e] == threshold) << e;
                }
            if (__any_sync(0xffffffffu, tied != 0)) {
                const int mine = __popc(tied), upto = warp_scan(mine);
                int left = need - (seen + upto - mine);          // ties that are still kept from this lane's first on
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if ((tied >> e) & 1u) above |= unsigned(left-- > 0) << e;
                seen += __shfl_sync(0xffffffffu, upto, 31);
            }
            f(i, above);
        });
    };
    // of the slots i .. i + 3: those below the budget, those that are there
    auto below = [&](int i) { return i >= b ? 0u : b - i >= 4 ? 15u : (1u << (b - i)) - 1u; };
    auto present = [&](int i) { return i >= w1 ? 0u : w1 - i >= 4 ? 15u : (1u << (w1 - i)) - 1u; };
    int behind = 0, holes = 0;
    for_kept([&](int i, unsigned keep) {
        behind += __popc(keep & ~below(i));
        holes += __popc(present(i) & ~keep & below(i));
    });
    behind = int(__reduce_add_sync(0xffffffffu, unsigned(behind)));
    holes = int(__reduce_add_sync(0xffffffffu, unsigned(holes)));
    if (lane == 0) { sm.count[1][warp] = behind; sm.count[2][warp] = holes; }
    __syncthreads();
    if (warp == 0) {
        const int x = scan(1), y = scan(2);
        if (lane == 0) { sm.total[0] = x; sm.total[1] = y; }
    }
    __syncthreads();
    int of0 = 0, of1 = 0;
    if (ctas > 1) {
        if (warp == 0) tell(1, 1, static_cast<unsigned long long>(uint32_t(sm.total[1])) << 32 | uint32_t(sm.total[0]));
        hear(1);
        if (__syncthreads_or(lost)) return give_up();
        if (lane < ctas) { of0 = int(uint32_t(sm.got[1][lane])); of1 = int(sm.got[1][lane] >> 32); }
    } else if (lane == 0) {
        of0 = sm.total[0]; of1 = sm.total[1];
    }
    int behind0 = sm.count[1][warp] + int(__reduce_add_sync(0xffffffffu, unsigned(lane < rank ? of0 : 0)));
    int holes0 = sm.count[2][warp] + int(__reduce_add_sync(0xffffffffu, unsigned(lane < rank ? of1 : 0)));
    const int moves = int(__reduce_add_sync(0xffffffffu, unsigned(of1)));
    // the lists: a CTA's own, if short, where its histograms were
    const bool here = ctas == 1 && moves <= 256;
    int32_t* from = here ? reinterpret_cast<int32_t*>(sm.hist[0]) : p.moved + int64_t(pair) * 2 * p.most_moved;
    int32_t* into = here ? reinterpret_cast<int32_t*>(sm.hist[1]) : from + p.most_moved;
    const bool tells = !in_place || kept;        // what stays where it is has to be written, too
    for_kept([&](int i, unsigned keep) {
        const unsigned comes = keep & ~below(i), open = present(i) & ~keep & below(i);
        const int mine = __popc(comes) | __popc(open) << 16, upto = warp_scan(mine);
        int x = behind0 + ((upto - mine) & 0xffff), y = holes0 + ((upto - mine) >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if ((comes >> e) & 1u) from[x++] = i + e;
            if ((open >> e) & 1u) into[y++] = i + e;
            if (!holds && tells && ((keep & below(i)) >> e) & 1u) stays_put(i + e);
        }
        const int all = __shfl_sync(0xffffffffu, upto, 31);
        behind0 += all & 0xffff;
        holes0 += all >> 16;
    });
    meet();                                      // the lists are written
    if (ctas > 1 && sm.gave_up) return;
    if (holds && tells)                          // (behind the barrier, which would wait for these writes; keys that are not held are gone once rows move)
        for_kept([&](int i, unsigned keep) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (((keep & below(i)) >> e) & 1u) stays_put(i + e);
        });

    // ---- moves: a warp looks 32 of them up at once, a lane each, then moves their rows, a 16-byte chunk of each a lane ----
    const int warps = ctas * kWarps, each = (moves + warps - 1) / warps, first = min(moves, (rank * kWarps + warp) * each), last = min(moves, first + each);
    for (int i0 = first; i0 < last; i0 += 32) {
        int src = 0, dst = 0, position = 0;
        float weight = 0.f;
        int64_t src_at = -1, dst_at = -1;
        if (i0 + lane < last) {
            src = from[i0 + lane]; dst = into[i0 + lane];
            src_at = row_at(src); dst_at = row_at(dst);
            weight = weights[src]; position = positions[src];
            if (kept) kept[dst] = src;
            if (src_at < 0 || dst_at < 0) {
                src_at = -1;
                if (p.status) atomicOr(p.status, kStatusBadPage);
            }
        }
        const int count = min(32, last - i0);
        for (int k0 = 0; k0 < count; k0 += kAtOnce) {
            uint4 x[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t at = __shfl_sync(0xffffffffu, src_at, k0 + k);
                const int slot = __shfl_sync(0xffffffffu, src, k0 + k);
                if (at >= 0 && lane < chunks) x[k] = *reinterpret_cast<const uint4*>(lane_at + at + swizzle(slot));
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t from_at = __shfl_sync(0xffffffffu, src_at, k0 + k), at = __shfl_sync(0xffffffffu, dst_at, k0 + k);
                const int slot = __shfl_sync(0xffffffffu, dst, k0 + k);
                if (from_at >= 0 && lane < chunks) *reinterpret_cast<uint4*>(lane_at + at + swizzle(slot)) = x[k];
            }
        }
        if (lane < count) { weights_out[dst] = weight; positions_out[dst] = position; }
    }
}

template <int THREADS>
cudaError_t launch(const PagedEvict& a, int ctas, cudaStream_t s) {
    static std::atomic<bool> configured[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(paged_evict_kernel<THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldSlots * 8 + kMostCtas * 2048);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(a.c.n_rows * a.c.g.n_kv_heads * ctas));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = size_t(a.held) * 8 + (ctas > 1 ? size_t(ctas) * 2048 : 0);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(ctas); attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = overlap_launches() ? 1 : 0;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, paged_evict_kernel<THREADS>, a, ctas);
}

}  // namespace

cudaError_t launch_paged_evict(PagedEvict& a, cudaStream_t s) {
    const int pairs = a.c.n_rows * a.c.g.n_kv_heads, slots = a.c.max_blocks * a.c.g.bt;
    int ctas = 1;
    while (ctas < kMostCtas && int64_t(pairs) * ctas * 2 <= kSmCount && slots / (ctas * 2) >= 1024) ctas *= 2;
    const int per_cta = ((slots + ctas - 1) / ctas + 31) & ~31;
    a.held = per_cta <= kHeldSlots ? per_cta : kHeldSlots;
    // Threads by the slots of a CTA, as long as it has an SM to itself: barriers cost more with more warps (8 pairs of 261 slots 11.0 us with 1024, 8.9 with
    // 256), passes and moves less (24 pairs of 15K 30.8 and 39.3; 24 of 3.5K, 1760 to a CTA, 16.9 and 14.7).
    if (int64_t(pairs) * ctas > kSmCount || per_cta <= 512) return launch<256>(a, ctas, s);
    return per_cta <= 2048 ? launch<512>(a, ctas, s) : launch<1024>(a, ctas, s);
}

}  // namespace ipkvi
