// Decode attention over a paged cache: one query per row, all slots or a window of the last ones and some first ones; partial output,
// log-sum-exp, and the slots' softmax weights added up.
//
//   s_t = scale q . k_t,   O = sum_t p_t v_t,   p_t = 2^(s_t log2 e - m) / z,   LSE = m ln 2 + ln z      (t visible)
//
// Bound by the K/V bytes (4 dim per token and KV head for 4 dim flops and query head).  A producer warp brings units of one KV head (16 KB: 32 tokens
// of 128 columns, 64 of 64) into a ring of stages; a page of a unit or less is one bulk copy, of larger ones a unit is one
// a panel.  Four warps compute, each on a unit of its own with an online softmax of its own.  The query heads of a KV head are the rows of
// the products (m16n8k16).  Page table and lengths are read here, so a captured call follows them.
//
// Exactness.  Products of bf16 are exact, sums fp32.  A softmax weight enters the second product as bf16 pieces that add up to
// it, 24 bits in three pieces: two (16 to 18 bits) would leave the output 2.4e-6 of itself off, more than a computation in fp32 does.  Up to 4
// query heads per KV head the three share the 16 rows of one product (rows 0-3, 4-7, 8-11: the queries are in
// rows 0-3 and 4-7, so that both have the weights); up to 8 two pieces share one and the third takes another; above, three.  A unit's
// sums start from zero and join the state by a rounded multiply-add: the tensor cores round towards zero, which would add up along a row.
//
// At the end of a pair the warps' states are joined in the stages of their last units, which nobody reads any more, and
// leave as the result, or as one partial for the join kernel.  Every wait is bounded.
//
// Measured (a few replays of a graph): 16 rows of 32K tokens, 4 KV heads of 8 query heads, 128 columns: 164 us for 1074 MB, 6.5 TB/s; 64 ragged rows of up
// to 16K in pages of 16, 8 KV heads of 4: 336 us for 2259 MB, 6.7 TB/s; one row of 500K, 16 heads on one: 51 us for 256 MB, 34 of them
// streaming at 7.5 TB/s; 32 rows through a window of 4096: 85 us for 507 MB, 6.0 TB/s; one of 4K tokens: 11.0 us, a chain of latencies.  More than 16 heads
// on a KV head are bound by their products, a warp's three for every 16 heads: 4 rows of 50K, 64 heads on 2: 63 us for 205 MB, 3.2 TB/s (32 on 1: 39 us for 102 MB); an odd number of
// sixteens reads K and V once for each: one row of 200K, 40 heads on one: 48 us for 102 MB.
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "launch.cuh"
#include "paged.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kWarps = kPagedWarps, kThreads = (kWarps + 1) * 32;
constexpr float kLn2 = 0.6931471805599453f;

struct Part : PagedPart {
    int32_t kv, in_kv, n_heads;                  // the KV head, the first of its query heads, how many
};
constexpr int kMostStages = 6, kRing = kMostStages * kPagedUnitBytes;

struct Smem {
    uint64_t full[kMostStages], empty[kMostStages], met;
    PagedParts parts[kWarps + 1];                // every warp's; registers are short
    Part part[kWarps + 1];
    uint32_t tag[kMostStages];                       // of a stage: which unit of the CTA's (times 16); bit i: its tokens 16 i .. 16 i + 15 are there
    float2 ml[kWarps * 16];                      // maximum and sum of every warp's rows
    int32_t where[kWarps];                       // the stage that holds a warp's sums
    int32_t scan[kThreads / 32];
    int32_t units, pairs, fit[32];
    PagedShare share;
    float2 part_ml[kPagedMostCluster][16], head_ml[16];  // cluster: maxima and sums of its CTAs' partials; the pair's maxima and 1 / sum
    alignas(16) int32_t cum[kPagedRowsPerLaunch + 1];    // (and n: a cluster's CTAs leave here what this one joins)
    int32_t n[kPagedRowsPerLaunch];
};
static_assert(16 * 128 * 4 <= sizeof(int32_t) * (2 * kPagedRowsPerLaunch + 1), "a partial of 16 heads");
// (a cluster's partial takes as much as all rows)
inline size_t smem_bytes(int n_rows) { return 1024 + kRing + sizeof(Smem) - size_t(kPagedRowsPerLaunch - n_rows) * 4; }

__device__ __forceinline__ void or_status(uint32_t* status, uint32_t bits) {
    if (status) atomicOr(status, bits);
}

// A row's length, brought inside its table.
__device__ __forceinline__ int length_of(const PagedAttend& p, int row, bool tell) {
    const int n = p.c.lengths[row], cap = p.c.max_blocks * p.c.g.bt;
    if (n >= 0 && n <= cap) return n;
    if (tell) or_status(p.status, kStatusBadPage);
    return n < 0 ? 0 : cap;
}

// A team must not take another team's older unit in a stage for its own: the stage's barrier tells a lap from the next, but not from the one after
// that, and copies land in any order.  So a computing warp first looks for its unit's number, which the producer leaves once the stage is
// free (every lap before has then been read), then waits for the copy.  Both are accesses of one SM to its shared memory, in program order; what
// the copy brought is ordered by the barrier.
__device__ __forceinline__ void leave_tag(uint32_t* tag, uint32_t x) {
    asm volatile("st.relaxed.cta.shared::cta.u32 [%0], %1;" ::"r"(ptx::smem_addr(tag)), "r"(x) : "memory");
}
__device__ __forceinline__ bool wait_tag(const uint32_t* tag, uint32_t unit, uint32_t& slices) {
    uint64_t t0 = 0;
    for (uint32_t n = 0;; ++n) {
        uint32_t x;
        asm volatile("ld.relaxed.cta.shared::cta.u32 %0, [%1];" : "=r"(x) : "r"(ptx::smem_addr(tag)) : "memory");
        slices = x & 15u;
        if ((x >> 4) == (unit & 0x0fffffffu)) return true;
        if ((n & 63u) == 0) {
            const uint64_t now = ptx::globaltimer_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > ptx::kWaitLimitNs) return false;
        }
    }
}

// To the shared memory of another CTA of the cluster.
__device__ __forceinline__ void put(uint32_t there, const float4& v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(there), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void put(uint32_t there, const float2& v) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
}

// Lengths, and from them the shares: see paged.h.  All threads of the CTA.
__device__ PagedShare share_out(const PagedAttend& p, Smem& sm, int teams) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, R = p.c.n_rows;
    PagedShare share{0, 0, 0};
    // the first of the 32 shares with which whole CTAs to every pair stay within the grid
    auto choose = [&](int mine, int parts, int units, int pairs) {
        const unsigned fits = __ballot_sync(0xffffffffu, pairs <= p.n_ctas && int64_t(parts) * p.n_gh <= p.n_ctas);
        const int share = fits == 0 ? 0 : __shfl_sync(0xffffffffu, mine, __ffs(int(fits)) - 1);
        return paged_share_wins(share, units, pairs, p.per_cta) ? share : 0;
    };
    auto scan = [&](int x) {
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        return x;
    };
    if (R <= 32) {                               // every warp for itself: all write the same
        const int n = lane < R ? length_of(p, lane, tid < 32 && blockIdx.x == 0) : 0;
        const int units = paged_seen(n, p.window, p.first, p.unit).units;
        const int sum = __reduce_add_sync(0xffffffffu, unsigned(units)), pairs = __popc(__ballot_sync(0xffffffffu, units > 0)) * p.n_gh;
        const int mine = paged_share_tried(sum * p.n_gh, p.per_cta, teams, lane);
        if (pairs <= p.n_ctas) {
            int parts = 0;
#pragma unroll 4
            for (int r = 0; r < R; ++r) parts += (unsigned(__shfl_sync(0xffffffffu, units, r)) + unsigned(mine) - 1) / unsigned(mine);
            share.share = choose(mine, parts, sum * p.n_gh, pairs);
        }
        const int cost = paged_cost(units, share), upto = scan(cost);
        if (lane < R) { sm.n[lane] = n; sm.cum[lane] = upto - cost; }
        if (lane == 31) sm.cum[R] = upto;
        __syncwarp();
        if (share.share == 0) {
            share.cost = sm.cum[R] * p.n_gh;
            share.ctas = min(p.n_ctas, share.cost);
        }
    } else {
        int units = 0, rows = 0;
        for (int r = tid; r < R; r += kThreads) {
            const int n = length_of(p, r, blockIdx.x == 0), u = paged_seen(n, p.window, p.first, p.unit).units;
            sm.n[r] = n;
            sm.cum[r] = u;
            units += u; rows += u > 0;
        }
        if (tid < 32) sm.fit[tid] = 0;
        units = int(__reduce_add_sync(0xffffffffu, unsigned(units)));
        rows = int(__reduce_add_sync(0xffffffffu, unsigned(rows)));
        if (lane == 0) { atomicAdd(&sm.units, units); atomicAdd(&sm.pairs, rows * p.n_gh); }
        __syncthreads();
        const int mine = paged_share_tried(sm.units * p.n_gh, p.per_cta, teams, lane);
        const bool few = sm.pairs <= p.n_ctas;
        if (few) {
            int parts = 0;
#pragma unroll 4
            for (int r = warp; r < R; r += kThreads / 32) parts += (unsigned(sm.cum[r]) + unsigned(mine) - 1) / unsigned(mine);
            atomicAdd(&sm.fit[lane], parts);
        }
        __syncthreads();
        share.share = choose(mine, sm.fit[lane], sm.units * p.n_gh, sm.pairs);
        int carry = 0;                           // prefix sums over the rows
        for (int r0 = 0; r0 < R; r0 += kThreads) {
            const int r = r0 + tid, cost = r < R ? paged_cost(sm.cum[r], share) : 0, upto = scan(cost);
            if (lane == 31) sm.scan[warp] = upto;
            __syncthreads();
            int before = carry;
            for (int w = 0; w < kThreads / 32; ++w) {
                if (w < warp) before += sm.scan[w];
                carry += sm.scan[w];
            }
            if (r < R) sm.cum[r] = before + upto - cost;
            __syncthreads();
        }
        if (tid == 0) sm.cum[R] = carry;
        if (share.share == 0) {
            share.cost = carry * p.n_gh;
            share.ctas = min(p.n_ctas, share.cost);
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && warp == 0) {
        for (int r = lane; r <= R; r += 32) p.header->cum[r] = sm.cum[r];
        if (lane == 0) p.header->share = share;
    }
    return share;
}

// ROWS: rows of the products that hold queries, see above.
template <int D, int ROWS>
__global__ void __launch_bounds__(kThreads, kPagedCtasPerSm) paged_attend_kernel(const __grid_constant__ PagedAttend p) {
    constexpr int U = kPagedUnitBytes / (4 * D), kSlices = U / 16;
    // 16 rows of queries are read from shared memory for every unit, each warp's in the place of a stage: with them in registers, too, some 20 others
    // were reloaded in every unit (64 heads on 2 KV heads, 4 rows of 50K tokens: 67 us against 60 when
    // this was changed).
    constexpr int kStages = ROWS == 16 ? kMostStages - 1 : kMostStages;
    extern __shared__ unsigned char smem_dyn[];
    unsigned char* ring = smem_dyn + ((1024u - (ptx::smem_addr(smem_dyn) & 1023u)) & 1023u);      // 1024: rows of a panel on distinct banks
    Smem& sm = *reinterpret_cast<Smem*>(ring + kRing);
    const uint32_t s_ring = ptx::smem_addr(ring);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int sixteens = ROWS == 16 ? p.sixteens : 1, teams = kWarps / sixteens;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(ptx::smem_addr(&sm.full[s]), 1);
            ptx::mbar_init(ptx::smem_addr(&sm.empty[s]), sixteens);
            sm.tag[s] = 0xffffffffu;
        }
        ptx::mbar_init(ptx::smem_addr(&sm.met), kWarps);
        ptx::mbar_fence_init();
        sm.units = 0; sm.pairs = 0;
    }
    // a cluster's pair and this CTA's rank in it, before the wait
    const int c_pair = int(blockIdx.x) >> p.cluster_shift, rank = int(blockIdx.x) & ((1 << p.cluster_shift) - 1);
    const int c_row = p.n_gh > 1 ? int(__umulhi(unsigned(c_pair), p.per_gh)) : c_pair, c_gh = c_pair - c_row * p.n_gh;      // (fewer pairs than CTAs: exact)
    __syncthreads();
    if (p.cluster > 1) ptx::cluster_arrive_relaxed();         // this CTA is there: the others may write to it behind their wait
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    PagedShare share{0, 0, 0};
    if (p.cluster == 0) share = share_out(p, sm, teams);
    // Where registers are short (128 columns), a warp's part is kept in shared memory, by its first lane.
    constexpr bool kLocal = D == 64;
    Part local_part;
    PagedParts local_parts;
    Part& x = kLocal ? local_part : sm.part[warp];
    PagedParts& parts = kLocal ? local_parts : sm.parts[warp];
    auto heads = [&](bool more) {                // of the part that has just been found
        const int kv = p.groups_per_kv == 1 ? x.gh : x.gh / p.groups_per_kv, in_kv = (x.gh - kv * p.groups_per_kv) * p.rows_per_part;
        x.kv = kv; x.in_kv = in_kv; x.n_heads = min(p.rows_per_part, p.group - in_kv);
        return more;
    };
    auto begin = [&]() {                         // the warp's first part (next one)
        bool more = true;
        if (kLocal || lane == 0) {
            if (p.cluster == 0) {
                parts = PagedParts{sm.cum, sm.n, share, p.c.n_rows, p.n_gh, p.window, p.first, U, int(blockIdx.x), 0, 0};
                more = parts.begin(x);
            } else {
                const PagedSeen seen = paged_seen(length_of(p, c_row, c_gh == 0 && rank == 0 && tid == 0), p.window, p.first, U);
                const int q = seen.units >> p.cluster_shift, r = seen.units - (q << p.cluster_shift);
                x.row = c_row; x.gh = c_gh; x.seen = seen;
                x.u0 = rank * q + min(rank, r); x.u1 = x.u0 + q + (rank < r ? 1 : 0);
                x.whole = p.cluster == 1; x.place = 0;
                parts.at = parts.end = 0;
            }
            more = heads(more);
        }
        __syncwarp();
        return kLocal ? more : __shfl_sync(0xffffffffu, int(more), 0) != 0;
    };
    auto next = [&]() {
        bool more = false;
        __syncwarp();
        if ((kLocal || lane == 0) && parts.at < parts.end) more = heads(parts.next(x));
        __syncwarp();
        return kLocal ? more : __shfl_sync(0xffffffffu, int(more), 0) != 0;
    };
    const int T = min(p.c.g.bt, U);              // tokens of a page that a unit takes at once

    if (warp == kWarps) {
        // ---------------- producer ----------------
        const uint64_t pol = ptx::l2_evict_first_policy();
        const int per_unit = U / T, batch = 32 / per_unit;       // pages of a unit; units whose pages the lanes look up at once
        const int64_t head_bytes = p.c.g.head_bytes(), block_bytes = p.c.g.block_bytes();
        const int64_t extent = kChecked && p.status ? p.c.n_blocks * block_bytes : 0;
        int st = 0, lap = 0, it = 0;
        bool ok = true;
        {   // a small table comes into the L1 cache while the lengths are on their way
            const int rows = p.cluster > 0 ? 1 : p.c.n_rows, first = p.cluster > 0 ? c_row : 0, lines = (p.c.max_blocks + 31) / 32;
            const int row = lane / lines;
            if (rows * lines <= 32 && row < rows) {
                int32_t unused;
                asm volatile("ld.global.b32 %0, [%1];" : "=r"(unused) : "l"(p.c.table + (first + row) * p.c.table_stride + (lane - row * lines) * 32));
            }
        }
        for (bool more = begin(); more && ok; more = next()) {
            const int32_t* table = p.c.table + int64_t(x.row) * p.c.table_stride;
            const char* head = p.c.pool + x.kv * head_bytes;
            const PagedSeen seen = x.seen;
            const int u0 = x.u0, u1 = x.u1;
            // lane l: the page of unit j + l / per_unit, its part l % per_unit; -1: nothing of it is seen, -2: a bad one
            auto page_of = [&](int j) {
                const int u = j + lane / per_unit;
                int page = -1;
                if (u < u1) {
                    const int a = seen.unit(u) * U + (lane % per_unit) * T;
                    if (seen.sees_any(a, a + T)) {
                        page = table[p.bt_shift >= 0 ? a >> p.bt_shift : a / p.c.g.bt];
                        if (page < 0 || page >= p.c.n_blocks) { or_status(p.status, kStatusBadPage); page = -2; }
                    }
                }
                return page;
            };
            int page = page_of(u0);
            for (int j0 = u0; j0 < u1 && ok; j0 += batch) {
                const int pages = page;
                if (j0 + batch < u1) page = page_of(j0 + batch);
                for (int j = j0; j < min(j0 + batch, u1); ++j) {
                    if (lap > 0) ok = ptx::mbar_wait_warp(ptx::smem_addr(&sm.empty[st]), (lap - 1) & 1);
                    if (!ok) break;
                    const int lane0 = (j - j0) * per_unit;                  // the lane that holds the unit's first page
                    const unsigned there = (__ballot_sync(0xffffffffu, pages >= 0) >> lane0) & ((1u << per_unit) - 1u);
                    const uint32_t bar = ptx::smem_addr(&sm.full[st]), dst = s_ring + st * kPagedUnitBytes;
                    if (lane == 0) {
                        int slices = 0;
#pragma unroll
                        for (int i = 0; i < kSlices; ++i) slices |= int((there >> (i * 16 / T)) & 1u) << i;
                        leave_tag(&sm.tag[st], uint32_t(it) << 4 | uint32_t(slices));
                        ptx::mbar_expect_tx(bar, uint32_t(__popc(there)) * T * D * 4);
                    }
                    __syncwarp();
                    if (p.c.g.bt <= U) {
                        const int sub = lane - lane0;
                        if (sub >= 0 && sub < per_unit && pages >= 0) {
                            const char* src = head + int64_t(pages) * block_bytes;
                            ptx::bulk_g2s_hint(dst + sub * T * D * 4, ptx::checked_src<kChecked>(src, T * D * 4, p.c.pool, extent, p.status, kStatusBadIndex),
                                               T * D * 4, bar, pol);
                        }
                    } else {
                        const int64_t at = __shfl_sync(0xffffffffu, pages, lane0);
                        if (there && lane < D / 32) {            // a panel a lane, of K, then of V
                            const char* src = head + at * block_bytes + (int64_t(lane) * p.c.g.bt + (p.bt_shift >= 0 ? seen.unit(j) * U & (p.c.g.bt - 1) : seen.unit(j) * U % p.c.g.bt)) * 128;
                            ptx::bulk_g2s_hint(dst + lane * (U * 128), ptx::checked_src<kChecked>(src, U * 128, p.c.pool, extent, p.status, kStatusBadIndex), U * 128,
                                               bar, pol);
                        }
                    }
                    ++it;
                    if (++st == kStages) { st = 0; ++lap; }
                }
            }
        }
        if (!ok && lane == 0) or_status(p.status, kStatusNoFreeStage);
        // do not leave the CTA while copies of ours may still be in flight
        if (lane == 0)
            for (int i = it > kStages ? it - kStages : 0; i < it; ++i)
                if (!ptx::mbar_wait(ptx::smem_addr(&sm.full[i % kStages]), (i / kStages) & 1)) or_status(p.status, kStatusCopyNotLanded);
        __syncwarp();
        if (p.cluster > 1) ptx::cluster_wait();
        return;
    }

    // ---------------- computing warps ----------------
    const int team = warp / sixteens, hg = warp - team * sixteens;       // whose turn it is; which sixteen of the group's heads
    const int mi = lane >> 3, r8 = lane & 7;
    const int r0 = lane >> 2, c0 = 2 * (lane & 3);
    // offsets in a stage: panels, V, slices of 16 tokens (a page's K and V lie together)
    const uint32_t panel = uint32_t(T) * 128, v_off = uint32_t(T) * D * 2, odd = T == 16 ? 16u * D * 4 : 2048u, pair = T >= 64 ? 4096u : 32u * D * 4;
    const uint32_t s_q = s_ring + kStages * kPagedUnitBytes + warp * 4096;       // ROWS == 16
    uint32_t qa[ROWS == 16 ? 1 : D / 16][2];
    float o[D / 8][4];
    int it0 = 0, meets = 0;                      // units of the parts before this one
    bool ok = true, waited = false;
    auto meet = [&]() -> bool {                  // the four warps; they may wait for units of their own first
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&sm.met));
        return ptx::mbar_wait_warp(ptx::smem_addr(&sm.met), meets++ & 1, 2 * ptx::kWaitLimitNs);
    };
    auto item_of = [&]() { return int64_t(x.row) * p.n_q_heads + x.kv * p.group + x.in_kv; };      // of the outputs

    for (bool more = begin(); more && ok; more = next()) {
        if (x.u0 == x.u1) {                      // a chunk that ends before the pair's first unit, a cluster's CTA without one, or an empty row
            if (x.whole) {
                const int n_heads = x.n_heads;
                const int64_t item0 = item_of();
                for (int i = tid; i < n_heads * D; i += kWarps * 32) {
                    p.out_o[item0 * D + i] = 0.f;
                    if (i < n_heads) {
                        p.out_lse[item0 + i] = -INFINITY;
                        if (p.head_ml) p.head_ml[item0 + i] = make_float2(0.f, 0.f);
                    }
                }
            }
            continue;
        }
        {
            const int n_heads = x.n_heads;
            const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q + x.row * p.q_row) + (x.kv * p.group + x.in_kv) * D;
            if (ROWS == 16) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const int row = (k * 32 + lane) / (D / 8), chunk = lane % (D / 8), head = hg * 16 + row;
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (head < n_heads) v = *reinterpret_cast<const uint4*>(q + head * D + chunk * 8);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                 ::"r"(s_q + row * (D * 2) + ((chunk & 8) << 4) + (((chunk ^ row) & 7) << 4)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
                }
                __syncwarp();
            } else {
                const int head = ROWS == 4 ? r0 & 3 : r0;
                const uint32_t* from = reinterpret_cast<const uint32_t*>(q + head * D + c0);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    qa[ks][0] = head < n_heads ? from[ks * 8] : 0u;
                    qa[ks][1] = head < n_heads ? from[ks * 8 + 4] : 0u;
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < D / 8; ++nt) { o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f; }
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float* scores = p.scores ? p.scores + ((int64_t(x.row) * p.n_gh + x.gh) * p.most_units + x.u0) * (U * p.rows_per_part) + hg * (ROWS * 16) : nullptr;
        const int n_units = x.u1 - x.u0;
        int held = -1;                           // the stage of this warp's last unit

        for (int i = (team - it0 % teams + teams) % teams; i < n_units; i += teams) {
            const int it = it0 + i, st = it % kStages;
            uint32_t there;
            ok = ptx::warp_agrees(wait_tag(&sm.tag[st], uint32_t(it), there) && ptx::mbar_wait(ptx::smem_addr(&sm.full[st]), (it / kStages) & 1));
            if (!ok) break;
            const int ta = x.seen.unit(x.u0 + i) * U;
            const uint32_t stage = s_ring + st * kPagedUnitBytes;
            auto slice = [&](int sl) { return stage + (sl & 1) * odd + (sl >> 1) * pair; };
            float s[2 * kSlices][4];
#pragma unroll
            for (int nt = 0; nt < 2 * kSlices; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const int chunk = ks * 2 + (mi & 1);             // K: matrices 0, 1 tokens 0-7 of a slice, 2, 3 tokens 8-15
                uint32_t q[4] = {0u, 0u, 0u, 0u};
                if (ROWS == 16) {                                // queries: matrices 0, 2 rows 0-7, 1, 3 rows 8-15
                    const int at = ks * 2 + (mi >> 1);
                    ptx::ldmatrix_x4(s_q + ((mi & 1) * 8 + r8) * (D * 2) + ((at & 8) << 4) + (((at ^ r8) & 7) << 4), q[0], q[1], q[2], q[3]);
                } else {
                    q[0] = qa[ks][0]; q[2] = qa[ks][1];
                }
#pragma unroll
                for (int sl = 0; sl < kSlices; ++sl) {
                    uint32_t b0, b1, b2, b3;
                    ptx::ldmatrix_x4(slice(sl) + ((mi >> 1) * 8 + r8) * 128 + (ks >= 4 ? panel : 0u) + (((chunk & 7) ^ r8) << 4), b0, b1, b2, b3);
                    ptx::mma_bf16(s[2 * sl], q, b0, b1);
                    ptx::mma_bf16(s[2 * sl + 1], q, b2, b3);
                }
            }
#pragma unroll
            for (int nt = 0; nt < 2 * kSlices; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[nt][e] *= p.scale_log2;
            if (!x.seen.sees_all(ta, ta + U) || there != (1u << kSlices) - 1u) {
                // Slots that are not seen, or whose page is bad, may hold anything: their scores are replaced, and their values by zeros (0 times a NaN
                // is one).
#pragma unroll
                for (int nt = 0; nt < 2 * kSlices; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!x.seen.sees(ta + nt * 8 + c0 + (e & 1)) || !((there >> (nt / 2)) & 1)) s[nt][e] = -INFINITY;
                for (int k = lane; k < U * (D / 8); k += 32) {
                    const int t = k / (D / 8), chunk = k % (D / 8);
                    if (!x.seen.sees(ta + t) || !((there >> (t / 16)) & 1))
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};"
                                     ::"r"(slice(t / 16) + v_off + (chunk >> 3) * panel + (t % 16) * 128 + (chunk & 7) * 16), "r"(0) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // before the stage goes back to the copy engine
                __syncwarp();
            }
            if (scores) {
                float* to = scores + int64_t(i) * (U * p.rows_per_part);
#pragma unroll
                for (int nt = 0; nt < 2 * kSlices; ++nt) {
                    float* at = to + (nt / 2) * (16 * p.rows_per_part) + (nt & 1) * (ROWS * 8) + r0 * 8 + c0;
                    if (ROWS > 4 || r0 < 4) *reinterpret_cast<float2*>(at) = make_float2(s[nt][0], s[nt][1]);
                    if (ROWS == 16) *reinterpret_cast<float2*>(at + 64) = make_float2(s[nt][2], s[nt][3]);
                }
            }
            // online softmax in the log2 domain; rows r0 and, with 16, r0 + 8
            float a0, a1 = 0.f;
            {
                float mx0 = s[0][0], mx1 = s[0][2];
#pragma unroll
                for (int nt = 0; nt < 2 * kSlices; ++nt) {
                    mx0 = fmaxf(mx0, fmaxf(s[nt][0], s[nt][1]));
                    if (ROWS == 16) mx1 = fmaxf(mx1, fmaxf(s[nt][2], s[nt][3]));
                }
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
                if (ROWS == 16) mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
                mx0 = fmaxf(m0, fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2)));
                const float ms0 = mx0 == -INFINITY ? 0.f : mx0;
                a0 = ptx::ex2(m0 - ms0);
                m0 = mx0;
                float ms1 = 0.f;
                if (ROWS == 16) {
                    mx1 = fmaxf(m1, fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2)));
                    ms1 = mx1 == -INFINITY ? 0.f : mx1;
                    a1 = ptx::ex2(m1 - ms1);
                    m1 = mx1;
                }
                float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
                for (int nt = 0; nt < 2 * kSlices; ++nt) {
                    s[nt][0] = ptx::ex2(s[nt][0] - ms0); s[nt][1] = ptx::ex2(s[nt][1] - ms0);
                    sum0 += s[nt][0] + s[nt][1];
                    if (ROWS == 16) {
                        s[nt][2] = ptx::ex2(s[nt][2] - ms1); s[nt][3] = ptx::ex2(s[nt][3] - ms1);
                        sum1 += s[nt][2] + s[nt][3];
                    }
                }
                l0 = fmaf(l0, a0, sum0);
                if (ROWS == 16) l1 = fmaf(l1, a1, sum1);
            }
            // the weights in three pieces, as operands: [0] and [2] are rows r0, [1] and [3] rows r0 + 8
            constexpr int kProducts = ROWS == 16 ? 3 : ROWS == 8 ? 2 : 1;
            uint32_t pa[kSlices][kProducts][4];
#pragma unroll
            for (int sl = 0; sl < kSlices; ++sl)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int h = 0; h < (ROWS == 16 ? 2 : 1); ++h) {
                        float y0 = s[2 * sl + half][2 * h], y1 = s[2 * sl + half][2 * h + 1];
                        uint32_t piece[3];
#pragma unroll
                        for (int k = 0; k < 3; ++k) {
                            piece[k] = ptx::pack_bf16(y0, y1);
                            y0 -= ptx::bf16_lo(piece[k]); y1 -= ptx::bf16_hi(piece[k]);
                        }
                        if (ROWS == 16) {
#pragma unroll
                            for (int k = 0; k < 3; ++k) pa[sl][k % kProducts][2 * half + h] = piece[k];
                        } else if (ROWS == 8) {
                            pa[sl][0][2 * half] = piece[0]; pa[sl][0][2 * half + 1] = piece[1];
                            pa[sl][1 % kProducts][2 * half] = piece[2]; pa[sl][1 % kProducts][2 * half + 1] = 0u;
                        } else {
                            pa[sl][0][2 * half] = r0 < 4 ? piece[0] : piece[1];
                            pa[sl][0][2 * half + 1] = r0 < 4 ? piece[2] : 0u;
                        }
                    }
#pragma unroll
            for (int jj = 0; jj < D / 16; ++jj) {
                const int chunk = 2 * jj + (mi >> 1);            // V: matrices 0, 2 tokens 0-7 of a slice, 1, 3 tokens 8-15
                uint32_t b[kSlices][4];
#pragma unroll
                for (int sl = 0; sl < kSlices; ++sl)
                    ptx::ldmatrix_x4_trans(slice(sl) + v_off + ((mi & 1) * 8 + r8) * 128 + (jj >= 4 ? panel : 0u) + (((chunk & 7) ^ r8) << 4), b[sl][0], b[sl][1], b[sl][2], b[sl][3]);
                float t0[4] = {0.f, 0.f, 0.f, 0.f}, t1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = kProducts - 1; k >= 0; --k)         // the small pieces first
#pragma unroll
                    for (int sl = 0; sl < kSlices; ++sl) {
                        ptx::mma_bf16(t0, pa[sl][k], b[sl][0], b[sl][1]);
                        ptx::mma_bf16(t1, pa[sl][k], b[sl][2], b[sl][3]);
                    }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = ROWS < 16 || e < 2 ? a0 : a1;
                    o[2 * jj][e] = fmaf(o[2 * jj][e], a, t0[e]);
                    o[2 * jj + 1][e] = fmaf(o[2 * jj + 1][e], a, t1[e]);
                }
            }
            __syncwarp();
            if (i + teams < n_units) {
                if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&sm.empty[st]));
            } else {
                held = st;
            }
        }
        if (!ok) break;
        it0 += n_units;

        // ---- the part's end ----
        const int n_heads = x.n_heads;
        const int64_t item0 = item_of();
        l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
        if (ROWS == 16) {
            l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
            l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
        }
        auto leave = [&](int head, float m, float z) {           // the part's maximum and sum
            if (x.whole) {
                const float2 y = make_float2(z == 0.f ? 0.f : m, z == 0.f ? 0.f : 1.f / z);
                p.out_lse[item0 + head] = z == 0.f ? -INFINITY : m * kLn2 + logf(z);
                if (p.head_ml) p.head_ml[item0 + head] = y;
                if (p.cluster == 1 && head < 16) sm.head_ml[head] = y;
            } else {
                p.part_ml[int64_t(x.place) * p.rows_per_part + head] = make_float2(m, z);
            }
        };
        if (kChecked && !x.whole && p.cluster == 0 && (x.place < 0 || x.place >= 2 * p.n_ctas)) {     // the partial must lie inside the scratch
            if (lane == 0) or_status(p.status, kStatusBadIndex);
            x.place = 0;
        }
        float* const out = x.whole ? p.out_o + item0 * D : p.part_o + int64_t(x.place) * p.rows_per_part * D;
        if (teams == 1 || (n_units == 1 && sixteens == 1 && p.cluster <= 1)) {       // no two warps have something of the same head
            if (held >= 0) {
#pragma unroll
                for (int h = 0; h < (ROWS == 16 ? 2 : 1); ++h) {
                    const int head = hg * 16 + r0 + 8 * h;
                    const bool mine = (ROWS > 4 || r0 < 4) && head < n_heads;
                    const float m = h ? m1 : m0, z = h ? l1 : l0, f = !x.whole ? 1.f : z == 0.f ? 0.f : 1.f / z;
#pragma unroll
                    for (int nt = 0; nt < D / 8; ++nt) {
                        float y0 = o[nt][2 * h], y1 = o[nt][2 * h + 1];
                        if (ROWS < 16) { y0 += o[nt][2]; y1 += o[nt][3]; }       // the pieces' sums
                        if (ROWS == 4) {
                            y0 += __shfl_xor_sync(0xffffffffu, y0, 16);
                            y1 += __shfl_xor_sync(0xffffffffu, y1, 16);
                        }
                        if (mine) *reinterpret_cast<float2*>(out + head * D + nt * 8 + c0) = make_float2(y0 * f, y1 * f);
                    }
                    if (mine && (lane & 3) == 0) leave(head, m, z);
                }
                if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&sm.empty[held]));
            }
            continue;
        }
        if (sixteens > 1 && !meet()) { ok = false; break; }      // the warps of a team have read their unit
        if ((lane & 3) == 0 && r0 < ROWS) {
            sm.ml[warp * 16 + r0] = make_float2(m0, l0);
            if (ROWS == 16) sm.ml[warp * 16 + r0 + 8] = make_float2(m1, l1);
        }
        if (held >= 0) {
            if (lane == 0) sm.where[warp] = held;
            // pairs of columns are swapped by row, so that rows lie on distinct banks
            const uint32_t to = s_ring + held * kPagedUnitBytes + (hg * ROWS + r0) * (D * 4);
#pragma unroll
            for (int nt = 0; nt < D / 8; ++nt) {
                float y0 = o[nt][0], y1 = o[nt][1];
                if (ROWS < 16) { y0 += o[nt][2]; y1 += o[nt][3]; }       // the pieces' sums
                if (ROWS == 4) {
                    y0 += __shfl_xor_sync(0xffffffffu, y0, 16);
                    y1 += __shfl_xor_sync(0xffffffffu, y1, 16);
                }
                const uint32_t at = uint32_t((nt * 4 + (lane & 3)) ^ ((r0 & 7) << 2)) * 8;
                if (ROWS > 4 || r0 < 4) ptx::sts_f2(to + at, y0, y1);
                if (ROWS == 16) ptx::sts_f2(to + 8 * (D * 4) + at, o[nt][2], o[nt][3]);
            }
        }
        if (!meet()) { ok = false; break; }
        if (p.cluster > 1) { ptx::cluster_wait(); waited = true; }
        for (int i = tid; i < n_heads * (D / 4); i += kWarps * 32) {
            const int head = i / (D / 4), col = i - head * (D / 4), g = ROWS == 16 ? head / 16 : 0, row = ROWS == 16 ? head % 16 : head;
            float2 y[kWarps];
            float4 v[kWarps];
            float m = -INFINITY, z = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                y[w] = ROWS < 16 || (w & (sixteens - 1)) == g ? sm.ml[w * 16 + row] : make_float2(-INFINITY, 0.f);
                m = fmaxf(m, y[w].x);
                if (y[w].y != 0.f) {             // (else nothing seen)
                    const uint32_t from = s_ring + sm.where[w] * kPagedUnitBytes + (g * ROWS + row) * (D * 4) + (uint32_t(2 * col) ^ ((row & 7) << 2)) * 8;
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[w].x), "=f"(v[w].y), "=f"(v[w].z), "=f"(v[w].w) : "r"(from) : "memory");
                }
            }
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
                if (y[w].y != 0.f) {
                    const float f = ptx::ex2(y[w].x - (m == -INFINITY ? 0.f : m));
                    acc.x += f * v[w].x; acc.y += f * v[w].y; acc.z += f * v[w].z; acc.w += f * v[w].w;
                    z += f * y[w].y;
                }
            if (p.cluster > 1) {                 // to the CTA that joins these columns; maximum and sum to all
                const int to = i & (p.cluster - 1);
                put(ptx::at_rank(ptx::smem_addr(sm.cum) + (rank * (n_heads * (D / 4) >> p.cluster_shift) + (i >> p.cluster_shift)) * 16, to), acc);
                if (col < p.cluster) put(ptx::at_rank(ptx::smem_addr(&sm.part_ml[rank][head]), col), make_float2(m, z));
                continue;
            }
            const float f = !x.whole ? 1.f : z == 0.f ? 0.f : 1.f / z;
            reinterpret_cast<float4*>(out + head * D)[col] = make_float4(acc.x * f, acc.y * f, acc.z * f, acc.w * f);
            if (col == 0) leave(head, m, z);
        }
        if (parts.at < parts.end) {              // the stages are needed again once all have read them
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (!meet()) { ok = false; break; }
            if (held >= 0 && lane == 0) ptx::mbar_arrive(ptx::smem_addr(&sm.empty[held]));
        }
    }
    if (!ok && lane == 0) or_status(p.status, kStatusNoTile);
    if (p.cluster == 0) return;

    // ---- a cluster: every CTA joins its share of the columns of all partials (also after a wait that ran out: the others wait for its word) ----
    const int n_heads = x.n_heads;
    const int64_t item0 = item_of();
    __syncwarp();
    if (p.cluster > 1) {
        if (!waited) {                               // no part, or a lost one
            ptx::cluster_wait();
            for (int k = tid; k < 16 * p.cluster; k += kWarps * 32) put(ptx::at_rank(ptx::smem_addr(&sm.part_ml[rank][k & 15]), k >> 4), make_float2(-INFINITY, 0.f));
        }
        ptx::cluster_arrive();
        ptx::cluster_wait();
        auto join = [&](auto most) {             // (for eight and for sixteen: what is not there costs smaller clusters 0.3 us)
            constexpr int kMost = decltype(most)::value;
            auto state_of = [&](int head, float2 (&y)[kMost], float& m, float& z) {
                m = -INFINITY; z = 0.f;
#pragma unroll
                for (int c = 0; c < kMost; ++c) {
                    y[c] = c < p.cluster ? sm.part_ml[c][head] : make_float2(-INFINITY, 0.f);
                    m = fmaxf(m, y[c].x);
                }
#pragma unroll
                for (int c = 0; c < kMost; ++c) {
                    y[c].x = ptx::ex2(y[c].x - (m == -INFINITY ? 0.f : m));
                    if (y[c].y != 0.f) z += y[c].x * y[c].y;
                }
            };
            const int per_cta = n_heads * (D / 4) >> p.cluster_shift;
            for (int k = tid; k < per_cta; k += kWarps * 32) {
                const int i = k * p.cluster + rank, head = i / (D / 4), col = i - head * (D / 4);
                float2 y[kMost];
                float m, z;
                state_of(head, y, m, z);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int c = 0; c < kMost; ++c)
                    if (c < p.cluster && y[c].y != 0.f) {
                        const float4 v = reinterpret_cast<const float4*>(sm.cum)[c * per_cta + k];
                        acc.x += y[c].x * v.x; acc.y += y[c].x * v.y; acc.z += y[c].x * v.z; acc.w += y[c].x * v.w;
                    }
                const float inv = z == 0.f ? 0.f : 1.f / z;
                reinterpret_cast<float4*>(p.out_o + item0 * D)[i] = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
                if (col == 0) p.out_lse[item0 + head] = z == 0.f ? -INFINITY : m * kLn2 + logf(z);
            }
            if (p.scores && tid < n_heads) {
                float2 y[kMost];
                float m, z;
                state_of(tid, y, m, z);
                sm.head_ml[tid] = make_float2(z == 0.f ? 0.f : m, z == 0.f ? 0.f : 1.f / z);
            }
        };
        if (p.cluster <= 8) join(std::integral_constant<int, 8>()); else join(std::integral_constant<int, kPagedMostCluster>());
    }
    if (!p.scores || p.group > 16) return;       // (more heads of a KV head are not all here: a launch of its own)
    __syncwarp();
    asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");       // (all four warps come here without another wait)
    if (!ok) return;
    // the weights of this CTA's units (all heads of the KV head are in one group here)
    const int64_t w0 = (int64_t(x.row) * p.c.g.n_kv_heads + x.kv) * p.c.slot_stride;
    const float* scores = p.scores + (int64_t(x.row) * p.n_gh + x.gh) * p.most_units * (U * ROWS);
    constexpr int kAhead = 32 / ROWS;            // slots of a thread under way
    for (int k0 = x.u0 * U + tid; k0 < x.u1 * U; k0 += kWarps * 32 * kAhead) {
        float s[kAhead][ROWS], before[kAhead];
        int t[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int k = k0 + e * (kWarps * 32);
            t[e] = k < x.u1 * U ? x.seen.unit(k / U) * U + k % U : -1;
            if (t[e] >= 0 && !x.seen.sees(t[e])) t[e] = -1;
            if (t[e] < 0) continue;
            const float* from = scores + int64_t(k >> 4) * (16 * ROWS) + ((k >> 3) & 1) * (ROWS * 8) + (k & 7);
            before[e] = p.c.weights ? p.c.weights[w0 + t[e]] : 0.f;
#pragma unroll
            for (int h = 0; h < ROWS; ++h) s[e][h] = h < n_heads ? from[h * 8] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (t[e] < 0) continue;
            float given = 0.f;
#pragma unroll
            for (int h = 0; h < ROWS; ++h)
                if (h < n_heads && sm.head_ml[h].y != 0.f) given += ptx::ex2(s[e][h] - sm.head_ml[h].x) * sm.head_ml[h].y;
            p.weights_out[w0 + t[e]] = before[e] + given;
        }
    }
}

// Joins the partials of every (row, query head) whose pair more than one CTA had: with partial i's maximum m_i (log2), sum l_i and sums o_i,
//   m = max m_i,  z = sum 2^(m_i - m) l_i,  O = sum 2^(m_i - m) o_i / z,  LSE = m ln 2 + ln z,   in a fixed order.
// One CTA per (row, head, COLS columns): COLS / 4 column groups times slices of the partials.  Bound by the latency of its reads, one behind the
// other: the shares, the partials (all of a slice at once).  295 partials of 16 heads, 2.5 MB: 4 us behind the attention.
template <int D, int COLS, int THREADS>
__global__ void __launch_bounds__(THREADS) paged_join_kernel(const __grid_constant__ PagedAttend p) {
    constexpr int kCols = COLS / 4, kSlices = THREADS / kCols, kSlabs = D / COLS;
    __shared__ float4 s_o[THREADS / 32][kCols];
    __shared__ float2 s_ml[THREADS / 32];
    static_assert(kCols <= 32, "a warp has whole slices");
    const int item = blockIdx.x / kSlabs, slab = blockIdx.x - item * kSlabs, row = item / p.n_q_heads, head = item - row * p.n_q_heads;
    const int tid = threadIdx.x, slice = tid / kCols, col = slab * kCols + tid % kCols;
    const int kv = head / p.group, in_kv = head - kv * p.group, part_of = in_kv / p.rows_per_part, rin = in_kv - part_of * p.rows_per_part;
    const int gh = kv * p.groups_per_kv + part_of;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const PagedShare share = p.header->share;
    const int u0 = p.header->cum[row], all = p.header->cum[row + 1] - u0;
    if (all == 0) {                              // nothing seen
        if (slice == 0) reinterpret_cast<float4*>(p.out_o + int64_t(item) * D)[col] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (tid == 0 && slab == 0) {
            p.out_lse[item] = -INFINITY;
            if (p.head_ml) p.head_ml[item] = make_float2(0.f, 0.f);
        }
        return;
    }
    const PagedPartials of = paged_partials(share, u0, all, p.n_gh, gh);
    const int n = of.n;
    if (n == 1) return;                          // written by its CTA
    auto at = [&](int i) { return int64_t(2 * (of.c0 + i) + (i == 0 ? of.odd : 0)) * p.rows_per_part + rin; };
    // every slice against its own maximum, then the slices
    float m = -INFINITY, z = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kAhead = 8;
    for (int i0 = slice; i0 < n; i0 += kAhead * kSlices) {
        float2 y[kAhead];
        float4 v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k * kSlices;
            y[k] = make_float2(-INFINITY, 0.f);
            if (i < n) {
                y[k] = p.part_ml[at(i)];
                v[k] = reinterpret_cast<const float4*>(p.part_o + at(i) * D)[col];
            }
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) top = fmaxf(top, y[k].x);
        const float base = top == -INFINITY ? 0.f : top, a = ptx::ex2(m - base);
        acc.x *= a; acc.y *= a; acc.z *= a; acc.w *= a; z *= a;
        m = top;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (y[k].y != 0.f) {                 // (a sum of NaN is not empty)
                const float f = ptx::ex2(y[k].x - base);
                acc.x += f * v[k].x; acc.y += f * v[k].y; acc.z += f * v[k].z; acc.w += f * v[k].w;
                z += f * y[k].y;
            }
    }
    // the slices of a warp, then the warps
#pragma unroll
    for (int d = kCols; d < 32; d <<= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, d), z2 = __shfl_xor_sync(0xffffffffu, z, d);
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top, f = ptx::ex2(m - base), f2 = ptx::ex2(m2 - base);
        acc.x = f * acc.x + f2 * __shfl_xor_sync(0xffffffffu, acc.x, d); acc.y = f * acc.y + f2 * __shfl_xor_sync(0xffffffffu, acc.y, d);
        acc.z = f * acc.z + f2 * __shfl_xor_sync(0xffffffffu, acc.z, d); acc.w = f * acc.w + f2 * __shfl_xor_sync(0xffffffffu, acc.w, d);
        z = f * z + f2 * z2;
        m = top;
    }
    const int lane = tid & 31, warp = tid >> 5;
    if (lane < kCols) s_o[warp][lane] = acc;
    if (lane == 0) s_ml[warp] = make_float2(m, z);
    __syncthreads();
    if (tid >= kCols) return;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) top = fmaxf(top, s_ml[k].x);
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    z = 0.f;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) {
        const float2 y = s_ml[k];
        const float4 v = s_o[k][tid];
        if (y.y == 0.f) continue;
        const float f = ptx::ex2(y.x - (top == -INFINITY ? 0.f : top));
        acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
        z += f * y.y;
    }
    const float inv = z == 0.f ? 0.f : 1.f / z;
    reinterpret_cast<float4*>(p.out_o + int64_t(item) * D)[col] = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (col == 0) {
        p.out_lse[item] = z == 0.f ? -INFINITY : top * kLn2 + logf(z);
        if (p.head_ml) p.head_ml[item] = make_float2(z == 0.f ? 0.f : top, inv);
    }
}

// weights_out[t] = weights[t] + sum over the KV head's query heads of 2^(s_t - m) / z, from the scores that the attention left.  32 rows of 2.5K to 4K
// tokens, 8 KV heads of 4: 10 us by itself with cold caches, 84 us all three launches.
// Bound by issue slots, so what does not change from slot to slot is done once for some: CTA (kv, split), row takes every splits-th group of a
// row's and KV head's visible slots, a thread kAhead of a group, a CTA's width apart.
constexpr int kWeighThreads = 256;
template <int ROWS>
constexpr int weigh_ahead() { return ROWS == 4 ? 4 : 2; }
template <int ROWS>
__global__ void __launch_bounds__(kWeighThreads) paged_weigh_kernel(const __grid_constant__ PagedAttend p, const int splits) {
    constexpr int kAhead = weigh_ahead<ROWS>();
    const int row = int(blockIdx.y), kv = int(blockIdx.x) / splits, split = int(blockIdx.x) - kv * splits;
    const int shift = p.unit == 64 ? 6 : 5;
    const float2* ml = p.head_ml + int64_t(row) * p.n_q_heads + kv * p.group;
    const float* scores = p.scores + (int64_t(row) * p.n_gh + kv * p.groups_per_kv) * p.most_units * (p.unit * p.rows_per_part);
    const int64_t w0 = (int64_t(row) * p.c.g.n_kv_heads + kv) * p.c.slot_stride;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const PagedSeen seen = paged_seen(length_of(p, row, false), p.window, p.first, p.unit);
    const int slots = seen.units << shift;
    float2 y[ROWS];
    auto heads_from = [&](int head0) {
#pragma unroll
        for (int h = 0; h < ROWS; ++h) y[h] = head0 + h < p.group ? ml[head0 + h] : make_float2(0.f, 0.f);
    };
    const bool few = p.group <= ROWS;
    if (few) heads_from(0);
    for (int k0 = split * (kWeighThreads * kAhead) + int(threadIdx.x); k0 < slots; k0 += splits * (kWeighThreads * kAhead)) {
        int t[kAhead];
        float before[kAhead], given[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int k = k0 + e * kWeighThreads;
            t[e] = (seen.unit(k >> shift) << shift) + (k & (p.unit - 1));
            if (k >= slots || !seen.sees(t[e])) t[e] = -1;
            given[e] = 0.f;
            before[e] = t[e] >= 0 && p.c.weights ? p.c.weights[w0 + t[e]] : 0.f;
        }
        for (int head0 = 0, part = 0; head0 < p.group; ++part)
            for (int hg = 0; hg < p.sixteens && head0 < p.group; ++hg, head0 += ROWS) {
                if (!few) heads_from(head0);
                const float* s = scores + int64_t(part) * p.most_units * (p.unit * p.rows_per_part) + hg * (ROWS * 16);
                float x[kAhead][ROWS];
#pragma unroll
                for (int e = 0; e < kAhead; ++e) {
                    const int k = k0 + e * kWeighThreads;
                    const float* from = s + int64_t(k >> 4) * (16 * p.rows_per_part) + ((k >> 3) & 1) * (ROWS * 8) + (k & 7);
#pragma unroll
                    for (int h = 0; h < ROWS; ++h) x[e][h] = t[e] >= 0 && y[h].y != 0.f ? from[h * 8] : -INFINITY;
                }
#pragma unroll
                for (int e = 0; e < kAhead; ++e)
#pragma unroll
                    for (int h = 0; h < ROWS; ++h) given[e] += ptx::ex2(x[e][h] - y[h].x) * y[h].y;
            }
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (t[e] >= 0) p.weights_out[w0 + t[e]] = before[e] + given[e];
    }
}

// Clusters of `cluster` CTAs.
cudaLaunchConfig_t in_clusters(int n_ctas, int cluster, cudaLaunchAttribute (&attr)[2], cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(n_ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes(kPagedRowsPerLaunch);
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = overlap_launches() ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(cluster); attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cfg;
}

// Sets the kernel up on the current device, once; tells the largest cluster that it places there.
template <int D, int ROWS>
cudaError_t configure(int& largest) {
    static std::atomic<int> known[64];           // 0: not yet
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool kept = dev >= 0 && dev < 64;
    largest = kept ? known[dev].load(std::memory_order_acquire) : 0;
    if (largest) return cudaSuccess;
    e = cudaFuncSetAttribute(paged_attend_kernel<D, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem_bytes(kPagedRowsPerLaunch)));
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = in_clusters(kPagedMostCluster, kPagedMostCluster, attr, nullptr);
    int clusters = 0;
    if (cudaFuncSetAttribute(paged_attend_kernel<D, ROWS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&clusters, paged_attend_kernel<D, ROWS>, &cfg) != cudaSuccess) {
        cudaGetLastError();                      // (told here, and no later call's)
        clusters = 0;
    }
    largest = clusters > 0 ? kPagedMostCluster : kPagedPortableCluster;
    if (kept) known[dev].store(largest, std::memory_order_release);
    return cudaSuccess;
}

template <int D, int ROWS>
cudaError_t launch(const PagedAttend& a, cudaStream_t s) {
    int largest = 0;
    const cudaError_t e = configure<D, ROWS>(largest);
    if (e != cudaSuccess) return e;
    if (a.cluster <= 1) return launch_overlapped(paged_attend_kernel<D, ROWS>, a.n_ctas, kThreads, smem_bytes(a.cluster ? 0 : a.c.n_rows), s, a);
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = in_clusters(a.n_ctas, a.cluster, attr, s);
    return cudaLaunchKernelEx(&cfg, paged_attend_kernel<D, ROWS>, a);
}

// Many partials for every head (few pairs): slabs of 16 columns with many slices.
constexpr int kManyPartials = 24;

template <int D>
cudaError_t launch_join(const PagedAttend& a, cudaStream_t s) {
    const int items = a.c.n_rows * a.n_q_heads, pairs = a.c.n_rows * a.n_gh;
    if (a.n_ctas > kManyPartials * pairs) return launch_overlapped(paged_join_kernel<D, 16, 256>, items * (D / 16), 256, size_t(0), s, a);
    return launch_overlapped(paged_join_kernel<D, D, 128>, items, 128, size_t(0), s, a);
}

}  // namespace

cudaError_t paged_largest_cluster(const PagedAttend& a, int& largest) {
    const bool wide = a.c.g.dim_qk == 128;
    const int rows = a.rows_per_part / a.sixteens;
    return rows == 4 ? (wide ? configure<128, 4>(largest) : configure<64, 4>(largest))
         : rows == 8 ? (wide ? configure<128, 8>(largest) : configure<64, 8>(largest))
                     : (wide ? configure<128, 16>(largest) : configure<64, 16>(largest));
}

cudaError_t launch_paged_attend(const PagedAttend& a, cudaStream_t s) {
    const bool wide = a.c.g.dim_qk == 128;
    const int rows = a.rows_per_part / a.sixteens;
    cudaError_t e = rows == 4 ? (wide ? launch<128, 4>(a, s) : launch<64, 4>(a, s))
                  : rows == 8 ? (wide ? launch<128, 8>(a, s) : launch<64, 8>(a, s))
                              : (wide ? launch<128, 16>(a, s) : launch<64, 16>(a, s));
    if (e != cudaSuccess) return e;
    if (a.cluster == 0) {
        e = wide ? launch_join<128>(a, s) : launch_join<64>(a, s);
        if (e != cudaSuccess) return e;
    }
    if (a.weights_out && (a.cluster == 0 || a.group > 16)) {
        const int64_t pairs = int64_t(a.c.n_rows) * a.c.g.n_kv_heads, group = kWeighThreads * (rows == 4 ? weigh_ahead<4>() : weigh_ahead<8>());
        const int64_t groups = (int64_t(a.most_units) * a.unit + group - 1) / group, want = (148 * 8 + pairs - 1) / pairs;       // CTAs that run at once
        const int splits = int(want < groups ? want : groups);   // (at most 148 * 8: kPagedMostSlots has room for a step of all of them)
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(unsigned(a.c.g.n_kv_heads * splits), unsigned(a.c.n_rows));
        cfg.blockDim = dim3(kWeighThreads);
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = overlap_launches() ? 1 : 0;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, rows == 4 ? paged_weigh_kernel<4> : rows == 8 ? paged_weigh_kernel<8> : paged_weigh_kernel<16>, a, splits);
    }
    return cudaSuccess;
}

}  // namespace ipkvi
