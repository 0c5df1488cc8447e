// Launch interface of the paged cache (paged_api.cu checks the arguments and fills these), and how the attention shares its work out.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "layout.cuh"

namespace ipkvi {

constexpr uint32_t kStatusBadPage = 16u;         // a length or a table entry out of range; the tokens were left out

// Slots of a row are counted in 32 bits, and so are the threads' steps along them: the largest, of the kernel that adds the weights up, goes
// 148 * 8 CTAs of 1024 slots beyond the last one.
constexpr int32_t kPagedMostSlots = INT32_MAX - (1 << 21);

// The cache as the kernels see it.
struct PagedCache {
    BlockGeom g;
    char* pool;
    int64_t n_blocks;
    const int32_t* table;                        // [n_rows][table_stride]
    const int32_t* lengths;
    int64_t table_stride, slot_stride;
    float* weights;
    int32_t* positions;
    int32_t n_rows, max_blocks;
};

// ---- append (paged_append.cu) --------------------------------------------------------------------------------------
struct PagedAppend {
    PagedCache c;
    const char* k;
    const char* v;
    int64_t k_token, v_token;                    // bytes between tokens
    int64_t n_tokens;
    const int32_t* row_start;                    // null: one token per row
    const int32_t* token_positions;
    uint32_t* status;
};
cudaError_t launch_paged_append(const PagedAppend& a, cudaStream_t s);

// ---- attention (paged_attend.cu) -----------------------------------------------------------------------------------
// Work is counted in units: 32 tokens of one KV head for 128 columns, 64 for 64, 16 KB either way.  One warp takes a unit at a time; with fewer
// tokens to a warp (64 shared by four) the chain of a softmax step was as long and the products stood in a row behind it: 580
// instructions for 16 tokens of 16 heads of 128 columns, 500K tokens 60 us.
constexpr int kPagedUnitBytes = 16 * 1024;
IPKV_HD int32_t paged_unit(int32_t dim) { return kPagedUnitBytes / (4 * dim); }
// What a query sees of a row's n slots, in units: all of them, or the units of the first slots and those of the window.
struct PagedSeen {
    int32_t n, first, lo;                        // slot t is visible if t < n and (t >= lo or t < first)
    int32_t head, skip;                          // units of the first slots; invisible units behind them
    int32_t units;
    IPKV_HD int32_t unit(int32_t j) const { return j < head ? j : j + skip; }
    IPKV_HD bool sees(int32_t t) const { return t < n && (t >= lo || t < first); }
    // any (all) of the slots a .. b - 1
    IPKV_HD bool sees_any(int32_t a, int32_t b) const { return a < n && ((b < n ? b : n) > lo || a < first); }
    IPKV_HD bool sees_all(int32_t a, int32_t b) const { return b <= n && (a >= lo || b <= first); }
};
IPKV_HD PagedSeen paged_seen(int32_t n, int32_t window, int32_t first, int32_t unit) {
    PagedSeen s{n, 0, 0, 0, 0, (n + unit - 1) / unit};
    if (window > 0 && int64_t(window) + first < n) {
        s.first = first;
        s.lo = n - window;
        const int32_t head = (first + unit - 1) / unit, from = s.lo / unit;
        if (from > head) { s.head = head; s.skip = from - head; s.units -= s.skip; }
    }
    return s;
}
// Units that a row of at most `capacity` slots can show.
inline int64_t paged_most_units(int64_t capacity, int64_t window, int64_t first, int32_t unit) {
    const int64_t all = (capacity + unit - 1) / unit;
    const int64_t seen = (first + unit - 1) / unit + window / unit + 2;
    return window > 0 && seen < all ? seen : all;
}

// A pair is a row and a head group (a KV head and some of its query heads).  Lengths are on the device, so every CTA works the shares out
// for itself, from the same numbers.  Two ways:
//  - whole CTAs to every pair: ceil(units / share) of them, each an equal part of the pair's units, pair after pair;
//  - equal chunks: a pair costs its units and kPagedPairCost in front of them, pair after pair, and every CTA takes an equal part of all cost.
// A part that holds all units of its pair is written out as the result; of the others a CTA has two at most, the chunk's first and last, and
// leaves them at places 2 c and 2 c + 1.  All counts of a launch fit 32 bits.
constexpr int kPagedPairCost = 4;                // queries read, the pipeline drained, a result written: as long as so many units
constexpr int kPagedRowsPerLaunch = 1024;        // the shares of so many rows are held in shared memory
constexpr int kPagedCtasPerSm = 2, kPagedWarps = 4;
// Where every pair has few units, which the host sees by the table's width or the window alone, a thread-block cluster takes it, joins
// in distributed shared memory and adds the weights up: one launch in place of two or three.  (A step of 16 rows of 2K, weighed, takes 14.4 us with a table of
// 2048 slots, 15.7 with 4096, and in three launches 19.8 with 8192 and 21.5 with 32768; one row of 4K 11.1 with 4608, 12.0 with 8192 and 32768.)
// Sixteen CTAs, more than a portable cluster, for at most eight pairs: a GPC for each (1 row of 4 KV heads, 2K tokens: 8.0 us, with eight CTAs 9.5; 3K and 4K:
// 9.8 and 10.9, with CTAs over the GPU and a join 11.6 and 11.7; sixteen pairs of sixteen 14.7 against 7.7, they take turns).  At the border that the units below
// set, nine a CTA: 4600 tokens of 128 columns 12.0 and 12.6 with a join, 9000 of 64 columns 9.6 and 10.6; beyond it, 6000 of 128 columns 12.9 and 12.7, 8000 14.4 and 12.0.
// `largest`: what the device places (a part of a GPU may have no GPC with room for sixteen).
constexpr int kPagedMostCluster = 16, kPagedPortableCluster = 8;
constexpr int kPagedClusterUnits = 24, kPagedClusterMore = 5;
inline int paged_cluster(int64_t pairs, int64_t most_units, int group, int sixteens, int ctas, int largest = kPagedMostCluster) {
    if (pairs > ctas) return 0;
    int n = 1;                                           // (more heads than one product takes stay with one CTA)
    while (group <= 16 && n < largest && pairs * n * 2 <= ctas && most_units > kPagedWarps * n && (n < kPagedPortableCluster || pairs <= 8)) n *= 2;
    // Units of a CTA, against those with whole CTAs over the GPU.  The launch saved is worth five (1 row of 4 KV heads in clusters of eight, 8 and 4: 2K tokens
    // 10.3 us against 10.9; 12 and 4: 12.5 and 11.7; 4 rows of 8 heads and 6K tokens, 24 and 20: 22.7 and 23.9).  Rows may be shorter than the table is wide, and
    // clusters do not even them out: not above 24.  (Warps that share their units take as many times more.)
    const int64_t mine = (most_units + n - 1) / n * sixteens, all = pairs * most_units / ctas, others = (all > kPagedWarps / sixteens ? all : kPagedWarps / sixteens) * sixteens;
    return mine <= kPagedClusterUnits && mine <= others + kPagedClusterMore ? n : 0;
}
struct PagedShare {
    int32_t share;                               // units of a CTA at most; 0: chunks
    int32_t cost, ctas;                          // chunks: of all pairs, and the CTAs that it is shared out to
};
IPKV_HD int32_t paged_cost(int32_t units, const PagedShare& s) {
    return s.share > 0 ? (units + s.share - 1) / s.share : units > 0 ? units + kPagedPairCost : 0;
}
// Chunks: n things in `parts` equal parts, the first n % parts of them one larger (in 32 bits: the latency of a 64-bit division is half a microsecond).
IPKV_HD int32_t paged_split(int32_t n, int32_t parts, int32_t i) {
    const int32_t q = int32_t(uint32_t(n) / uint32_t(parts)), r = n - q * parts;
    return i * q + (i < r ? i : r);
}
// one part's beginning and end
IPKV_HD void paged_split(int32_t n, int32_t parts, int32_t i, int32_t& begin, int32_t& end) {
    const int32_t q = int32_t(uint32_t(n) / uint32_t(parts)), r = n - q * parts;
    begin = i * q + (i < r ? i : r);
    end = begin + q + (i < r ? 1 : 0);
}
// the part that has thing x of n >= parts
IPKV_HD int32_t paged_part_of(int32_t n, int32_t parts, int32_t x) {
    const int32_t q = int32_t(uint32_t(n) / uint32_t(parts)), r = n - q * parts, large = r * (q + 1);
    return x < large ? int32_t(uint32_t(x) / uint32_t(q + 1)) : r + int32_t(uint32_t(x - large) / uint32_t(q));
}
// The share that whole CTAs to every pair would take is looked for among 32 values, from what `ctas` CTAs have to take of all units at least
// up to twice that, in multiples of the teams that work in a CTA while it is few rounds of them.  Chunks, if none of them gives every pair
// whole CTAs within `ctas`, or if the share is much more than a chunk (rows of different lengths: 256 pairs of 80 to 129 units gave 120
// units to a CTA, 93 in chunks).  Where a chunk has the end of one pair and the beginning of the next it loses some 3 us, 8 units: 64 pairs of
// 129 units 29.5 us by shares of 36, 31.1 in chunks of 29; 264 of 94 units 67.7 by 94 and 72 in chunks of 87.
// (In fp32, by 1 / ctas: every CTA finds the same, and an integer division is a twentieth of a microsecond.)
IPKV_HD int32_t paged_share_tried(int32_t units, float per_cta, int32_t teams, int32_t i) {
    const int32_t mean = int32_t(float(units) * per_cta) + 1, least = mean >= 8 * teams ? mean : (mean + teams - 1) & -teams;
    const int32_t step = mean >= 8 * teams ? 1 : teams;          // teams is 1, 2 or 4
    return least + (((least >> 5) & -step) + step) * i;
}
IPKV_HD bool paged_share_wins(int32_t share, int32_t units, int32_t pairs, float per_cta) {
    const float mean = float(units + pairs * kPagedPairCost) * per_cta;
    return float(share) <= mean + mean * (1.f / 16.f) + 8.f;
}

// A CTA's parts of pairs, one after the other.  cum[r]: cost (with a share: parts) of a head group in the rows before r; n[r]: slots.
struct PagedPart {
    int32_t row, gh, u0, u1, place;
    bool whole;                                  // all units of the pair
    PagedSeen seen;
};
struct PagedParts {
    const int32_t *cum, *n;
    PagedShare share;
    int32_t n_rows, n_gh, window, first, unit, cta;
    int32_t at, end;
    // the row whose cost holds x
    IPKV_HD int32_t row_of(int32_t x) const {
        int32_t lo = 0, hi = n_rows - 1;
        while (lo < hi) {
            const int32_t mid = (lo + hi + 1) >> 1;
            if (cum[mid] * n_gh <= x) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
    // the part from `at` on of the pair (x.row, x.gh); `at` moves behind the pair
    IPKV_HD void set(PagedPart& x, int32_t place) {
        const int32_t all = cum[x.row + 1] - cum[x.row], p0 = cum[x.row] * n_gh + x.gh * all;
        const int32_t to = end - p0 < all ? end - p0 : all;
        x.seen = paged_seen(n[x.row], window, first, unit);
        x.u0 = at - p0 > kPagedPairCost ? at - p0 - kPagedPairCost : 0;
        x.u1 = to > kPagedPairCost ? to - kPagedPairCost : 0;
        x.whole = x.u1 - x.u0 == x.seen.units;
        x.place = place;
        at = p0 + all;
    }
    // false: no (more) part
    IPKV_HD bool begin(PagedPart& x) {
        at = 0; end = 0;
        if (share.share > 0) {
            if (cta >= cum[n_rows] * n_gh) return false;
            x.row = row_of(cta);
            const int32_t parts = cum[x.row + 1] - cum[x.row], i = cta - cum[x.row] * n_gh;
            x.gh = int32_t(uint32_t(i) / uint32_t(parts));
            const int32_t part = i - x.gh * parts;
            x.seen = paged_seen(n[x.row], window, first, unit);
            paged_split(x.seen.units, parts, part, x.u0, x.u1);
            x.whole = parts == 1;
            x.place = 2 * cta;
            return true;
        }
        if (cta >= share.ctas) return false;
        paged_split(share.cost, share.ctas, cta, at, end);
        if (at >= end) return false;
        x.row = row_of(at);
        x.gh = int32_t(uint32_t(at - cum[x.row] * n_gh) / uint32_t(cum[x.row + 1] - cum[x.row]));
        set(x, 2 * cta);
        return true;
    }
    IPKV_HD bool next(PagedPart& x) {
        if (at >= end) return false;
        if (++x.gh == n_gh) {
            x.gh = 0;
            do ++x.row; while (cum[x.row + 1] == cum[x.row]);
        }
        set(x, 2 * cta + 1);
        return true;
    }
};
// The partials of a pair that has units: partial i of n is at place 2 (c0 + i), the first one at the next if it is not its CTA's first part.
// One alone is no partial, but the result, written out.
struct PagedPartials { int32_t c0, n, odd; };
IPKV_HD PagedPartials paged_partials(const PagedShare& s, int32_t cum, int32_t all, int32_t n_gh, int32_t gh) {
    const int32_t first = cum * n_gh + gh * all;
    if (s.share > 0) return {first, all, 0};
    const int32_t c0 = paged_part_of(s.cost, s.ctas, first + kPagedPairCost);
    return {c0, paged_part_of(s.cost, s.ctas, first + all - 1) - c0 + 1, paged_split(s.cost, s.ctas, c0) < first};
}

// Head groups: a unit is read once for a head group.  Up to 16 query heads are the rows of one product (as one group of 4, 8 or 16 rows);
// more make sixteens, one to a warp: as many to a group as divide both their number and the four computing warps, which are then so
// many teams fewer.
inline int paged_rows(int group) { return group <= 4 ? 4 : group <= 8 ? 8 : 16; }
inline int paged_sixteens(int group) {
    const int n = (group + 15) / 16;
    return n % 4 == 0 ? 4 : n % 2 == 0 ? 2 : 1;
}
inline int paged_groups_per_kv(int group) { return (group + 15) / 16 / paged_sixteens(group); }
inline int paged_rows_per_part(int group) { return paged_rows(group) * paged_sixteens(group); }

struct PagedHeader {                             // in front of the scratch, written by the attention for the join
    PagedShare share;
    int32_t cum[kPagedRowsPerLaunch + 1];        // see PagedParts
};
struct PagedAttend {
    PagedCache c;
    const char* q;                               // row r at r * q_row bytes
    int64_t q_row;
    PagedHeader* header;
    float* part_o;                               // [2 n_ctas][rows_per_part][dim]: sums of weight times value, not divided
    float2* part_ml;                             // [2 n_ctas][rows_per_part]: reference maximum (log2) and sum of weights against it
    float2* head_ml;                             // [n_rows][n_q_heads]: maximum and 1 / sum, for the weights; null without
    float* scores;                               // [n_rows][n_gh][most_units][unit * rows_per_part], null without weights
    float* weights_out;
    float* out_o;
    float* out_lse;
    uint32_t* status;
    int32_t window, first, unit, most_units;
    int32_t n_q_heads, group, groups_per_kv, n_gh, rows_per_part, sixteens;
    int32_t n_ctas;
    int32_t bt_shift;                            // log2 of the tokens of a block, -1 where there is none
    float per_cta;                               // 1 / n_ctas
    uint32_t per_gh;                             // 2^32 / n_gh, rounded up
    int32_t cluster_shift;
    int32_t cluster;                             // CTAs that take a pair together and write its result; 0: shares, and a join
    float scale_log2;
};
cudaError_t launch_paged_attend(const PagedAttend& a, cudaStream_t s);
// The largest cluster of its kernel that the current device places: kPagedMostCluster or kPagedPortableCluster.
cudaError_t paged_largest_cluster(const PagedAttend& a, int& largest);

// ---- eviction (paged_evict.cu) -------------------------------------------------------------------------------------
struct PagedEvict {
    PagedCache c;
    float* weights_out;
    int32_t* positions_out;
    int32_t* kept;                               // may be null
    int32_t* moved;                              // scratch: [n_rows][n_kv_heads][2][most_moved]: kept slots behind the budget, evicted ones before it
    uint32_t* status;
    int32_t budget, first, recent;
    int32_t most_moved;                          // min(budget, slots - budget)
    int32_t held;                                // slots that a CTA has room for in shared memory
};
cudaError_t launch_paged_evict(PagedEvict& a, cudaStream_t s);

}  // namespace ipkvi
