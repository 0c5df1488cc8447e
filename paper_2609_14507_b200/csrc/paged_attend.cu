// Decode attention over a paged cache: one query per row, all slots or a window of the last ones and some first ones; partial output,
// log-sum-exp, and the slots' softmax weights added up.
//
//   s_t = scale q . k_t,   O = sum_t p_t v_t,   p_t = 2^(s_t log2 e - m) / z,   LSE = m ln 2 + ln z      (t visible)
//
// Bound by the K/V bytes (4 dim per token and KV head for 4 dim flops and query head).  A producer warp brings tiles of 64 tokens of one
// KV head (32 KB for 128 columns, contiguous in a page of 64 tokens or less: one bulk copy a page) into a ring of stages; four
// warps compute, each on 16 tokens of every tile, with an online softmax of its own.  The query heads of a KV head are the rows of
// the products (m16n8k16).  Page table and lengths are read here, so a captured call follows them.
//
// Exactness.  Products of bf16 are exact, sums fp32.  A softmax weight enters the second product as bf16 pieces that add up to
// it, 24 bits in three pieces: with two (16 to 18 bits) the output was off by 2.4e-6 of itself, more than a computation in fp32 is.  Up to 4
// query heads per KV head the three share the 16 rows of one product (rows 0-3, 4-7, 8-11: the queries are in
// rows 0-3 and 4-7, so that both have the weights); up to 8 two pieces share one and the third takes another; above, three.  A tile's
// sums start from zero and join the state by a rounded multiply-add: the tensor cores round towards zero, which would add up along a row.
//
// At the end of a pair the four warps' states are joined in the stage of the pair's last tile, which nobody reads any more, and
// leave as the result, or as one partial for the join kernel.
#include <cuda_bf16.h>

#include <atomic>
#include <cstddef>

#include "kernels.h"
#include "launch.cuh"
#include "paged.h"
#include "ptx.cuh"

namespace ipkvi {

namespace {

constexpr int kWarps = 4, kThreads = (kWarps + 1) * 32;
constexpr float kLn2 = 0.6931471805599453f;

template <int D>
struct Plan {
    static constexpr int kStage = 64 * D * 4;    // K and V of 64 tokens
    static constexpr int kStages = D == 128 ? 3 : 6;
};

struct Smem {
    uint64_t full[8], empty[8];
    int32_t slices[8];                           // of a stage: bit i: tokens 16 i .. 16 i + 15 are there
    float2 ml[2][kWarps * 16];                   // maximum and sum of every warp's rows; in turn, since a warp may be a part ahead of one that still reads
    int32_t gave_up, scan[kThreads / 32 + 1];
    int32_t tiles, pairs, fit[32];
    PagedShare share;
    int32_t cum[kPagedRowsPerLaunch + 1], n[kPagedRowsPerLaunch];
};
// up to the arrays of rows
inline size_t smem_bytes(int stage_bytes, int n_rows) {
    return 1024 + size_t(stage_bytes) + offsetof(Smem, cum) + size_t(2 * kPagedRowsPerLaunch + 1) * 4 - size_t(kPagedRowsPerLaunch - n_rows) * 4;
}

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

// Lengths, and from them the shares: see paged.h.  All threads of the CTA.
__device__ void share_out(const PagedAttend& p, Smem& sm) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, R = p.c.n_rows;
    int tiles = 0, rows = 0;
    for (int r = tid; r < R; r += kThreads) {
        const int n = length_of(p, r, blockIdx.x == 0);
        const int t = paged_seen(n, p.window, p.first).tiles;
        sm.n[r] = n;
        sm.cum[r] = t;
        tiles += t; rows += t > 0;
    }
    if (tid < 32) sm.fit[tid] = 0;
    for (int d = 16; d > 0; d >>= 1) {
        tiles += __shfl_xor_sync(0xffffffffu, tiles, d);
        rows += __shfl_xor_sync(0xffffffffu, rows, d);
    }
    if (lane == 0) { atomicAdd(&sm.tiles, tiles); atomicAdd(&sm.pairs, rows * p.n_gh); }
    __syncthreads();
    // the fewest tiles a CTA with which whole CTAs to every pair stay within the grid
    const int mine = paged_share_tried(int64_t(sm.tiles) * p.n_gh, p.n_ctas, lane);
    const bool few = sm.pairs <= p.n_ctas;
    if (few) {
        int parts = 0;
        for (int r = warp; r < R; r += kThreads / 32) parts += (sm.cum[r] + mine - 1) / mine;
        atomicAdd(&sm.fit[lane], parts);
    }
    __syncthreads();
    if (warp == 0) {
        const unsigned fits = __ballot_sync(0xffffffffu, few && int64_t(sm.fit[lane]) * p.n_gh <= p.n_ctas);
        const int which = __ffs(int(fits)) - 1;
        const int best = __shfl_sync(0xffffffffu, mine, which < 0 ? 0 : which);
        if (lane == 0) {
            sm.share.share = which < 0 ? 0 : best;
            sm.share.ctas = 0; sm.share.units = 0;
        }
    }
    __syncthreads();
    // prefix sums over the rows
    int carry = 0;
    for (int r0 = 0; r0 < R; r0 += kThreads) {
        const int r = r0 + tid;
        const int u = r < R ? paged_units(sm.cum[r], sm.share) : 0;
        int x = u;
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) sm.scan[warp] = x;
        __syncthreads();
        int before = carry;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += sm.scan[w];
            carry += sm.scan[w];
        }
        if (r < R) sm.cum[r] = before + x - u;
        __syncthreads();
    }
    if (tid == 0) {
        sm.cum[R] = carry;
        if (sm.share.share == 0) {
            sm.share.units = carry * p.n_gh;
            sm.share.ctas = min(p.n_ctas, sm.share.units);
        }
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int r = tid; r <= R; r += kThreads) p.header->cum[r] = sm.cum[r];
        if (tid == 0) p.header->share = sm.share;
    }
}

// ROWS: rows of the products that hold queries, see above.
template <int D, int ROWS>
__global__ void __launch_bounds__(kThreads, kPagedCtasPerSm) paged_attend_kernel(const __grid_constant__ PagedAttend p) {
    constexpr int kStage = Plan<D>::kStage, kStages = Plan<D>::kStages;
    extern __shared__ unsigned char smem_dyn[];
    unsigned char* ring = smem_dyn + ((1024u - (ptx::smem_addr(smem_dyn) & 1023u)) & 1023u);      // 1024: rows of a panel on distinct banks
    Smem& sm = *reinterpret_cast<Smem*>(ring + kStages * kStage);
    const uint32_t s_ring = ptx::smem_addr(ring);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(ptx::smem_addr(&sm.full[s]), 1);
            ptx::mbar_init(ptx::smem_addr(&sm.empty[s]), kWarps);
        }
        ptx::mbar_fence_init();
        sm.gave_up = 0; sm.tiles = 0; sm.pairs = 0;
    }
    __syncthreads();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (p.single) {
        if (tid == 0) {
            const int row = int(blockIdx.x) / p.n_gh;
            sm.n[row] = length_of(p, row, int(blockIdx.x) == row * p.n_gh);
        }
        __syncthreads();
    } else {
        share_out(p, sm);
    }
    const int T = min(p.c.g.bt, kTileTokens);            // tokens of a page that a tile takes at once
    PagedPart x;
    PagedParts parts{sm.cum, sm.n, sm.share, p.c.n_rows, p.n_gh, p.window, p.first, int(blockIdx.x), 0, 0};
    auto begin = [&]() {
        if (!p.single) return parts.begin(x);
        x.row = int(blockIdx.x) / p.n_gh; x.gh = int(blockIdx.x) - x.row * p.n_gh;
        x.seen = paged_seen(sm.n[x.row], p.window, p.first);
        x.t0 = 0; x.t1 = x.seen.tiles; x.whole = true; x.place = 0;
        parts.u = parts.u1 = 0;
        return true;
    };

    if (warp == kWarps) {
        // ---------------- producer ----------------
        const uint64_t pol = ptx::l2_evict_first_policy();
        const int per_tile = kTileTokens / T;            // pages of a tile
        const int64_t head_bytes = p.c.g.head_bytes(), block_bytes = p.c.g.block_bytes();
        int it = 0;
        bool ok = true;
        for (bool more = begin(); more && ok; more = parts.next(x)) {
            const int32_t* table = p.c.table + int64_t(x.row) * p.c.table_stride;
            const char* head = p.c.pool + (x.gh / p.groups_per_kv) * head_bytes;
            const int batch = 32 / per_tile;
            // lane l: the page of tile l / per_tile of a batch, its part l % per_tile; -1: nothing of it is seen, -2: a bad one
            auto page_of = [&](int j) {
                const int tile = j + lane / per_tile;
                int page = -1;
                if (tile < x.t1) {
                    const int a = x.seen.tile(tile) * kTileTokens + (lane % per_tile) * T;
                    if (x.seen.sees_any(a, a + T)) {
                        page = table[a / p.c.g.bt];
                        if (page < 0 || page >= p.c.n_blocks) { or_status(p.status, kStatusBadPage); page = -2; }
                    }
                }
                return page;
            };
            int page = page_of(x.t0);
            for (int j0 = x.t0; j0 < x.t1 && ok; j0 += batch) {
                const int pages = page;
                if (j0 + batch < x.t1) page = page_of(j0 + batch);
                for (int j = j0; j < min(j0 + batch, x.t1) && ok; ++j, ++it) {
                    const int st = it % kStages;
                    if (it >= kStages) ok = ptx::mbar_wait(ptx::smem_addr(&sm.empty[st]), ((it / kStages) - 1) & 1);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    // the lanes that hold this tile's pages issue their copies
                    const int sub = lane - (j - j0) * per_tile;
                    const bool mine = sub >= 0 && sub < per_tile && pages >= 0;
                    const unsigned there = __ballot_sync(0xffffffffu, mine) >> ((j - j0) * per_tile);
                    const uint32_t bar = ptx::smem_addr(&sm.full[st]), dst = s_ring + st * kStage;
                    if (lane == 0) {
                        int slices = 0;
                        for (int i = 0; i < 4; ++i) slices |= int((there >> (i * 16 / T)) & 1u) << i;
                        sm.slices[st] = slices;
                        ptx::mbar_expect_tx(bar, uint32_t(__popc(there & ((1u << per_tile) - 1u))) * T * D * 4);
                    }
                    __syncwarp();
                    if (mine) {
                        const char* src = head + int64_t(pages) * block_bytes;
                        const int64_t extent = kChecked ? p.c.n_blocks * block_bytes : 0;
                        if (p.c.g.bt <= kTileTokens) {
                            ptx::bulk_g2s_hint(dst + sub * T * D * 4, ptx::checked_src<kChecked>(src, T * D * 4, p.c.pool, p.status ? extent : 0, p.status, kStatusBadIndex),
                                               T * D * 4, bar, pol);
                        } else {
                            const int r0 = x.seen.tile(j) * kTileTokens % p.c.g.bt;
#pragma unroll
                            for (int i = 0; i < D / 32; ++i) {           // panels of K, then of V
                                const char* from = src + (int64_t(i) * p.c.g.bt + r0) * 128;
                                ptx::bulk_g2s_hint(dst + i * 8192, ptx::checked_src<kChecked>(from, 8192, p.c.pool, p.status ? extent : 0, p.status, kStatusBadIndex), 8192,
                                                   bar, pol);
                            }
                        }
                    }
                }
            }
        }
        if (!ok && lane == 0) or_status(p.status, kStatusNoFreeStage);
        // do not leave the CTA while copies of ours may still be in flight
        if (lane == 0)
            for (int i = it > kStages ? it - kStages : 0; i < it; ++i)
                if (!ptx::mbar_wait(ptx::smem_addr(&sm.full[i % kStages]), (i / kStages) & 1)) or_status(p.status, kStatusCopyNotLanded);
        return;
    }

    // ---------------- computing warps ----------------
    const int sixteens = ROWS == 16 ? p.sixteens : 1, hg = ROWS == 16 ? warp % sixteens : 0;      // which sixteen of the group's heads
    const int mi = lane >> 3, r8 = lane & 7;
    const int r0 = lane >> 2, c0 = 2 * (lane & 3);
    // rows that lanes address for ldmatrix: K tokens (mi >> 1) * 8 + r8 of a slice of 16, V tokens (mi & 1) * 8 + r8
    const uint32_t panel = uint32_t(T) * 128, v_off = uint32_t(T) * D * 2;
    uint32_t qa[D / 16][4];
    float o[D / 8][4];
    int it = 0, turn = 0;
    bool ok = true;

    // The four warps.  The barrier has no limit of its own; the order of events bounds it: a warp comes here after a tile that the others wait
    // for as well, each with a limit that began no earlier, and one that gave up has said so before that.
    auto meet = [&]() -> bool {
        __syncwarp();
        if (*reinterpret_cast<volatile int32_t*>(&sm.gave_up)) return false;
        asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
        return true;
    };

    for (bool more = begin(); more && ok; more = parts.next(x)) {
        const int kv = x.gh / p.groups_per_kv, in_kv = (x.gh - kv * p.groups_per_kv) * p.rows_per_part;
        const int n_heads = min(p.rows_per_part, p.group - in_kv);       // of the part
        const int64_t item0 = int64_t(x.row) * p.n_q_heads + kv * p.group + in_kv;
        if (x.t0 == x.t1) {
            // an empty row (single), or a chunk that ends before the pair's first tile (nothing to leave)
            if (x.whole)
                for (int i = tid; i < n_heads * D; i += kWarps * 32) {
                    p.out_o[item0 * D + i] = 0.f;
                    if (i < n_heads) {
                        p.out_lse[item0 + i] = -INFINITY;
                        if (p.head_ml) p.head_ml[item0 + i] = make_float2(0.f, 0.f);
                    }
                }
            continue;
        }
        {
            const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q + x.row * p.q_row) + (kv * p.group + in_kv) * D;
            const int ha = hg * 16 + (ROWS == 4 ? r0 & 3 : r0), hb = hg * 16 + r0 + 8;
            const uint32_t* qa0 = reinterpret_cast<const uint32_t*>(q + ha * D + c0);
            const uint32_t* qa1 = reinterpret_cast<const uint32_t*>(q + hb * D + c0);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                qa[ks][0] = ha < n_heads ? qa0[ks * 8] : 0u;
                qa[ks][2] = ha < n_heads ? qa0[ks * 8 + 4] : 0u;
                qa[ks][1] = ROWS == 16 ? (hb < n_heads ? qa1[ks * 8] : 0u) : 0u;
                qa[ks][3] = ROWS == 16 ? (hb < n_heads ? qa1[ks * 8 + 4] : 0u) : 0u;
            }
        }
#pragma unroll
        for (int nt = 0; nt < D / 8; ++nt) { o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f; }
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float* scores = p.scores ? p.scores + (int64_t(x.row) * p.n_gh + x.gh) * p.most_tiles * (64 * p.rows_per_part) : nullptr;

        for (int j = x.t0; j < x.t1; ++j, ++it) {
            const int st = it % kStages;
            if (!ptx::mbar_wait(ptx::smem_addr(&sm.full[st]), (it / kStages) & 1)) {
                *reinterpret_cast<volatile int32_t*>(&sm.gave_up) = 1;
                ok = false;
                break;
            }
            const int slices = sm.slices[st], t_tile = x.seen.tile(j) * kTileTokens;
            const uint32_t stage = s_ring + st * kStage;
            bool wrote = false;
            for (int sl = warp / sixteens; sl < 4; sl += kWarps / sixteens) {
                const int ta = t_tile + sl * 16;
                if (!x.seen.sees_any(ta, ta + 16)) continue;
                float* to = scores ? scores + (int64_t(j) * 4 + sl) * (16 * p.rows_per_part) + hg * (ROWS * 16) : nullptr;
                if (!((slices >> sl) & 1)) {     // its page was bad: no weight
                    if (to)
                        for (int i = lane; i < 16 * ROWS; i += 32) to[i] = -INFINITY;
                    continue;
                }
                const uint32_t base = stage + uint32_t(sl * 16 / T) * (T * D * 4) + uint32_t(sl * 16 % T) * 128;
                float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
                {
                    const uint32_t kb = base + ((mi >> 1) * 8 + r8) * 128;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        const int chunk = ks * 2 + (mi & 1);
                        uint32_t b0, b1, b2, b3;
                        ptx::ldmatrix_x4(kb + (ks >= 4 ? panel : 0u) + (((chunk & 7) ^ r8) << 4), b0, b1, b2, b3);
                        ptx::mma_bf16(s[0], qa[ks], b0, b1);
                        ptx::mma_bf16(s[1], qa[ks], b2, b3);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[nt][e] *= p.scale_log2;
                if (!x.seen.sees_all(ta, ta + 16)) {
                    // invisible slots may hold anything: their scores are replaced, and their values by zeros (0 times a NaN is one)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!x.seen.sees(ta + nt * 8 + c0 + (e & 1))) s[nt][e] = -INFINITY;
                    for (int i = lane; i < 16 * (D / 8); i += 32) {
                        const int t = i / (D / 8), chunk = i % (D / 8);
                        if (!x.seen.sees(ta + t))
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + v_off + (chunk >> 3) * panel + t * 128 + (chunk & 7) * 16), "r"(0) : "memory");
                    }
                    wrote = true;
                    __syncwarp();
                }
                if (to) {
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) {
                        if (ROWS > 4 || r0 < 4) *reinterpret_cast<float2*>(to + nt * (ROWS * 8) + r0 * 8 + c0) = make_float2(s[nt][0], s[nt][1]);
                        if (ROWS == 16) *reinterpret_cast<float2*>(to + nt * (ROWS * 8) + (r0 + 8) * 8 + c0) = make_float2(s[nt][2], s[nt][3]);
                    }
                }
                // online softmax in the log2 domain; rows r0 and, with 16, r0 + 8
                float mx0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
                const float mn0 = fmaxf(m0, mx0), ms0 = mn0 == -INFINITY ? 0.f : mn0;
                const float a0 = ptx::ex2(m0 - ms0);
                m0 = mn0;
                float a1 = a0, ms1 = ms0;
                if (ROWS == 16) {
                    float mx1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
                    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
                    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
                    const float mn1 = fmaxf(m1, mx1);
                    ms1 = mn1 == -INFINITY ? 0.f : mn1;
                    a1 = ptx::ex2(m1 - ms1);
                    m1 = mn1;
                }
                float pr[2][4];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) pr[nt][e] = (ROWS == 16 || e < 2) ? ptx::ex2(s[nt][e] - (e < 2 ? ms0 : ms1)) : 0.f;
                l0 = l0 * a0 + ((pr[0][0] + pr[0][1]) + (pr[1][0] + pr[1][1]));
                if (ROWS == 16) l1 = l1 * a1 + ((pr[0][2] + pr[0][3]) + (pr[1][2] + pr[1][3]));
                // the weights in three pieces, as operands: [0] and [2] are rows r0, [1] and [3] rows r0 + 8
                uint32_t pa[3][4];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
                    for (int h = 0; h < (ROWS == 16 ? 2 : 1); ++h) {
                        float y0 = pr[nt][2 * h], y1 = pr[nt][2 * h + 1];
                        uint32_t piece[3];
#pragma unroll
                        for (int k = 0; k < 3; ++k) {
                            piece[k] = ptx::pack_bf16(y0, y1);
                            y0 -= ptx::bf16_lo(piece[k]); y1 -= ptx::bf16_hi(piece[k]);
                        }
                        if (ROWS == 16) {
#pragma unroll
                            for (int k = 0; k < 3; ++k) pa[k][2 * nt + h] = piece[k];
                        } else if (ROWS == 8) {
                            pa[0][2 * nt] = piece[0]; pa[0][2 * nt + 1] = piece[1];
                            pa[1][2 * nt] = piece[2]; pa[1][2 * nt + 1] = 0u;
                        } else {
                            pa[0][2 * nt] = r0 < 4 ? piece[0] : piece[1];
                            pa[0][2 * nt + 1] = r0 < 4 ? piece[2] : 0u;
                        }
                    }
                }
                const uint32_t vb = base + v_off + ((mi & 1) * 8 + r8) * 128;
#pragma unroll
                for (int jj = 0; jj < D / 16; ++jj) {
                    const int chunk = 2 * jj + (mi >> 1);
                    uint32_t b0, b1, b2, b3;
                    ptx::ldmatrix_x4_trans(vb + (jj >= 4 ? panel : 0u) + (((chunk & 7) ^ r8) << 4), b0, b1, b2, b3);
                    float t0[4] = {0.f, 0.f, 0.f, 0.f}, t1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int k = (ROWS == 16 ? 3 : ROWS == 8 ? 2 : 1) - 1; k >= 0; --k) {        // the small pieces first
                        ptx::mma_bf16(t0, pa[k], b0, b1);
                        ptx::mma_bf16(t1, pa[k], b2, b3);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[2 * jj][e] = fmaf(o[2 * jj][e], e < 2 ? a0 : a1, t0[e]);
                        o[2 * jj + 1][e] = fmaf(o[2 * jj + 1][e], e < 2 ? a0 : a1, t1[e]);
                    }
                }
            }
            if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // before the stage goes back to the copy engine
            __syncwarp();
            if (j + 1 < x.t1 && lane == 0) ptx::mbar_arrive(ptx::smem_addr(&sm.empty[st]));
        }
        if (!ok) break;

        // ---- the part's end: the warps' states meet in the last tile's stage ----
        const int st = (it - 1) % kStages;
        const uint32_t buf = s_ring + st * kStage;
        float2* ml = sm.ml[turn];
        turn ^= 1;
        l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
        if (ROWS == 16) {
            l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
            l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
        }
        if ((lane & 3) == 0 && r0 < ROWS) {
            ml[warp * 16 + r0] = make_float2(m0, l0);
            if (ROWS == 16) ml[warp * 16 + r0 + 8] = make_float2(m1, l1);
        }
        if (!meet()) { ok = false; break; }      // every warp is done with the tile
        {
            // pairs of columns are swapped by row, so that rows lie on distinct banks
            const uint32_t to = buf + (warp * ROWS + r0) * (D * 4);
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
        for (int i = tid; i < n_heads * (D / 4); i += kWarps * 32) {
            const int head = i / (D / 4), col = i - head * (D / 4), w0 = ROWS == 16 ? head / 16 : 0, row = ROWS == 16 ? head % 16 : head;
            float m = -INFINITY, z = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int w = w0; w < kWarps; w += sixteens) m = fmaxf(m, ml[w * 16 + row].x);
            for (int w = w0; w < kWarps; w += sixteens) {
                const float2 y = ml[w * 16 + row];
                if (y.y == 0.f) continue;        // nothing seen
                const float f = ptx::ex2(y.x - (m == -INFINITY ? 0.f : m));
                float4 v;
                const uint32_t from = buf + (w * ROWS + row) * (D * 4) + (uint32_t(2 * col) ^ ((row & 7) << 2)) * 8;
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(from) : "memory");
                acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
                z += f * y.y;
            }
            if (x.whole) {
                const float inv = z == 0.f ? 0.f : 1.f / z;
                reinterpret_cast<float4*>(p.out_o + (item0 + head) * D)[col] = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
                if (col == 0) {
                    p.out_lse[item0 + head] = z == 0.f ? -INFINITY : m * kLn2 + logf(z);
                    if (p.head_ml) p.head_ml[item0 + head] = make_float2(z == 0.f ? 0.f : m, inv);
                }
            } else {
                const int64_t at = int64_t(x.place) * p.rows_per_part + head;
                reinterpret_cast<float4*>(p.part_o + at * D)[col] = acc;
                if (col == 0) p.part_ml[at] = make_float2(m, z);
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&sm.empty[st]));
    }
    if (!ok && lane == 0) or_status(p.status, kStatusNoTile);
}

// Joins the partials of every (row, query head) whose pair more than one CTA had: with partial i's maximum m_i (log2), sum l_i and sums o_i,
//   m = max m_i,  z = sum 2^(m_i - m) l_i,  O = sum 2^(m_i - m) o_i / z,  LSE = m ln 2 + ln z,   in a fixed order.
// One CTA per (row, head): D / 4 column groups times slices of the partials.
template <int D, int THREADS>
__global__ void __launch_bounds__(THREADS) paged_join_kernel(const __grid_constant__ PagedAttend p) {
    constexpr int kCols = D / 4, kSlices = THREADS / kCols;
    __shared__ float4 s_o[kSlices][kCols];
    __shared__ float s_z[kSlices], s_m[THREADS / 32];
    const int item = blockIdx.x, row = item / p.n_q_heads, head = item - row * p.n_q_heads;
    const int tid = threadIdx.x, col = tid % kCols, slice = tid / kCols;
    const int kv = head / p.group, in_kv = head - kv * p.group, part_of = in_kv / p.rows_per_part, rin = in_kv - part_of * p.rows_per_part;
    const int gh = kv * p.groups_per_kv + part_of;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const PagedShare share = p.header->share;
    const int u0 = p.header->cum[row], all = p.header->cum[row + 1] - u0;
    if (all == 0) {                              // nothing seen
        if (slice == 0) reinterpret_cast<float4*>(p.out_o + int64_t(item) * D)[col] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (tid == 0) {
            p.out_lse[item] = -INFINITY;
            if (p.head_ml) p.head_ml[item] = make_float2(0.f, 0.f);
        }
        return;
    }
    const PagedPartials of = paged_partials(share, u0, all, p.n_gh, gh);
    const int n = of.n;
    if (n == 1) return;                          // written by its CTA
    auto at = [&](int i) { return int64_t(2 * (of.c0 + i) + (i == 0 ? of.odd : 0)) * p.rows_per_part + rin; };
    float m = -INFINITY;
    for (int i = tid; i < n; i += THREADS) m = fmaxf(m, p.part_ml[at(i)].x);
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
        const float2 y = p.part_ml[at(i)];
        const float4 v = reinterpret_cast<const float4*>(p.part_o + at(i) * D)[col];
        if (y.y != 0.f) {                        // (a sum of NaN is not empty)
            const float f = ptx::ex2(y.x - (m == -INFINITY ? 0.f : m));
            acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
            z += f * y.y;
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
    reinterpret_cast<float4*>(p.out_o + int64_t(item) * D)[col] = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (col == 0) {
        p.out_lse[item] = z == 0.f ? -INFINITY : m * kLn2 + logf(z);
        if (p.head_ml) p.head_ml[item] = make_float2(z == 0.f ? 0.f : m, inv);
    }
}

// weights_out[t] = weights[t] + sum over the KV head's query heads of 2^(s_t - m) / z, from the scores that the attention left.
// One CTA for every splits-th group of four tiles of a (row, KV head); a thread per token.
__global__ void __launch_bounds__(256) paged_weigh_kernel(const __grid_constant__ PagedAttend p, const int splits) {
    const int split = blockIdx.x % splits, pair = blockIdx.x / splits, kv = pair % p.c.g.n_kv_heads, row = pair / p.c.g.n_kv_heads;
    const int tid = threadIdx.x, tok = tid & 63;
    const int rows = p.rows_per_part / p.sixteens;       // of one product
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int n = min(max(p.c.lengths[row], 0), p.c.max_blocks * p.c.g.bt);
    const PagedSeen seen = paged_seen(n, p.window, p.first);
    const float2* ml = p.head_ml + int64_t(row) * p.n_q_heads + kv * p.group;
    const int64_t w0 = (int64_t(row) * p.c.g.n_kv_heads + kv) * p.c.slot_stride;
    for (int j = split * 4 + (tid >> 6); j < seen.tiles; j += splits * 4) {
        const int t = seen.tile(j) * kTileTokens + tok;
        if (!seen.sees(t)) continue;
        float sum = p.c.weights ? p.c.weights[w0 + t] : 0.f;
        float given = 0.f;
        for (int part = 0; part < p.groups_per_kv; ++part) {
            const float* s = p.scores + ((int64_t(row) * p.n_gh + kv * p.groups_per_kv + part) * p.most_tiles + j) * (64 * p.rows_per_part) +
                             (tok >> 4) * (16 * p.rows_per_part) + ((tok >> 3) & 1) * (rows * 8) + (tok & 7);
            const int heads = min(p.rows_per_part, p.group - part * p.rows_per_part);
#pragma unroll 8
            for (int h = 0; h < heads; ++h) {
                const float2 y = ml[part * p.rows_per_part + h];
                const float x = s[(h / rows) * (rows * 16) + (h % rows) * 8];
                if (y.y != 0.f) given += ptx::ex2(x - y.x) * y.y;
            }
        }
        p.weights_out[w0 + t] = sum + given;
    }
}

template <int D, int ROWS>
cudaError_t launch(const PagedAttend& a, cudaStream_t s) {
    static std::atomic<bool> configured[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    constexpr int kRing = Plan<D>::kStage * Plan<D>::kStages;
    if (dev < 0 || dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(paged_attend_kernel<D, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem_bytes(kRing, kPagedRowsPerLaunch)));
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    return launch_overlapped(paged_attend_kernel<D, ROWS>, a.n_ctas, kThreads, smem_bytes(kRing, a.c.n_rows), s, a);
}

}  // namespace

cudaError_t launch_paged_attend(const PagedAttend& a, cudaStream_t s) {
    const bool wide = a.c.g.dim_qk == 128;
    const int rows = a.rows_per_part / a.sixteens;
    cudaError_t e = rows == 4 ? (wide ? launch<128, 4>(a, s) : launch<64, 4>(a, s))
                  : rows == 8 ? (wide ? launch<128, 8>(a, s) : launch<64, 8>(a, s))
                              : (wide ? launch<128, 16>(a, s) : launch<64, 16>(a, s));
    if (e != cudaSuccess) return e;
    if (!a.single) {
        const int items = a.c.n_rows * a.n_q_heads;
        e = wide ? launch_overlapped(paged_join_kernel<128, 256>, items, 256, size_t(0), s, a)
                 : launch_overlapped(paged_join_kernel<64, 256>, items, 256, size_t(0), s, a);
        if (e != cudaSuccess) return e;
    }
    if (a.weights_out) {
        const int64_t pairs = int64_t(a.c.n_rows) * a.c.g.n_kv_heads, groups = (a.most_tiles + 3) / 4;
        const int64_t want = (148 * 8 + pairs - 1) / pairs;
        const int splits = int(want < groups ? want : groups);
        return launch_overlapped(paged_weigh_kernel, int(pairs * splits), 256, size_t(0), s, a, splits);
    }
    return cudaSuccess;
}

}  // namespace ipkvi
