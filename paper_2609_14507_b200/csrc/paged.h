// Launch interface of the paged cache (paged_api.cu checks the arguments and fills these), and how the attention shares its work out.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "layout.cuh"

namespace ipkvi {

constexpr uint32_t kStatusBadPage = 16u;         // a length or a table entry out of range; the tokens were left out

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
// What a query sees of a row's n slots, in tiles of 64: all of them, or the tiles of the first slots and those of the window.
struct PagedSeen {
    int32_t n, first, lo;                        // slot t is visible if t < n and (t >= lo or t < first)
    int32_t head, skip;                          // tiles of the first slots; invisible tiles behind them
    int32_t tiles;
    IPKV_HD int32_t tile(int32_t j) const { return j < head ? j : j + skip; }
    IPKV_HD bool sees(int32_t t) const { return t < n && (t >= lo || t < first); }
    // any (all) of the slots a .. b - 1
    IPKV_HD bool sees_any(int32_t a, int32_t b) const { return a < n && ((b < n ? b : n) > lo || a < first); }
    IPKV_HD bool sees_all(int32_t a, int32_t b) const { return b <= n && (a >= lo || b <= first); }
};
IPKV_HD PagedSeen paged_seen(int32_t n, int32_t window, int32_t first) {
    PagedSeen s{n, 0, 0, 0, 0, (n + kTileTokens - 1) / kTileTokens};
    if (window > 0 && int64_t(window) + first < n) {
        s.first = first;
        s.lo = n - window;
        const int32_t head = (first + kTileTokens - 1) / kTileTokens, from = s.lo / kTileTokens;
        if (from > head) { s.head = head; s.skip = from - head; s.tiles -= s.skip; }
    }
    return s;
}
// Tiles that a row of at most `capacity` slots can show.
inline int64_t paged_most_tiles(int64_t capacity, int64_t window, int64_t first) {
    const int64_t all = (capacity + kTileTokens - 1) / kTileTokens;
    const int64_t seen = (first + kTileTokens - 1) / kTileTokens + window / kTileTokens + 2;
    return window > 0 && seen < all ? seen : all;
}

// A pair is a row and a head group (a KV head and some of its query heads).  Lengths are on the device, so every CTA works the shares out
// for itself, from the same numbers.  Two ways:
//  - whole CTAs to every pair: ceil(tiles / share) of them, each an equal part of the pair's tiles, pair after pair;
//  - equal chunks: work is counted in units, a pair's tiles and kPagedPairCost in front of them, pair after pair, and CTA c of n takes
//    units [units c / n, units (c + 1) / n).
// A part that holds all tiles of its pair is written out as the result; of the others a CTA has two at most, the chunk's first and last, and
// leaves them at places 2 c and 2 c + 1.
constexpr int kPagedPairCost = 2;                // queries read, the pipeline drained, a result written: as long as so many tiles
constexpr int kPagedRowsPerLaunch = 1024;        // the shares of so many rows are held in shared memory
constexpr int kPagedCtasPerSm = 2;
constexpr int kPagedSingleTiles = 4;             // tiles of a pair up to which one CTA takes it and no join follows
struct PagedShare {
    int32_t share;                               // tiles of a CTA at most; 0: chunks
    int32_t units, ctas;                         // chunks: all units, and the CTAs that they are shared out to
};
IPKV_HD int32_t paged_units(int32_t tiles, const PagedShare& s) {
    return s.share > 0 ? (tiles + s.share - 1) / s.share : tiles > 0 ? tiles + kPagedPairCost : 0;
}
IPKV_HD int32_t paged_chunk_begin(const PagedShare& s, int32_t c) { return int32_t(int64_t(s.units) * c / s.ctas); }
// the last CTA whose chunk begins at or before a unit: the one that has it
IPKV_HD int32_t paged_cta_of(const PagedShare& s, int32_t unit) { return int32_t(((int64_t(unit) + 1) * s.ctas - 1) / s.units); }
// The share that whole CTAs to every pair would take is looked for among 32 values, from what `ctas` CTAs have to take of n_gh * tiles at least
// up to twice that; chunks, if none of them gives every pair whole CTAs within `ctas`.
IPKV_HD int32_t paged_share_tried(int64_t tiles, int32_t ctas, int32_t i) {
    const int64_t least = tiles > 0 ? (tiles + ctas - 1) / ctas : 1;
    return int32_t(least + (least * i + 30) / 31);
}

// A CTA's parts of pairs, one after the other.  cum[r]: units (with a share: parts) of a head group in the rows before r; n[r]: slots.
struct PagedPart {
    int32_t row, gh, t0, t1, place;
    bool whole;                                  // all tiles of the pair
    PagedSeen seen;
};
struct PagedParts {
    const int32_t *cum, *n;
    PagedShare share;
    int32_t n_rows, n_gh, window, first, cta;
    int32_t u, u1;
    // the row whose units hold unit u
    IPKV_HD int32_t row_of(int32_t unit) const {
        int32_t lo = 0, hi = n_rows - 1;
        while (lo < hi) {
            const int32_t mid = (lo + hi + 1) >> 1;
            if (cum[mid] * n_gh <= unit) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
    // the part from unit u on of the pair (x.row, x.gh); u moves behind the pair
    IPKV_HD void set(PagedPart& x, int32_t place) {
        const int32_t all = cum[x.row + 1] - cum[x.row], p0 = cum[x.row] * n_gh + x.gh * all;
        const int32_t end = u1 - p0 < all ? u1 - p0 : all;
        x.seen = paged_seen(n[x.row], window, first);
        x.t0 = u - p0 > kPagedPairCost ? u - p0 - kPagedPairCost : 0;
        x.t1 = end > kPagedPairCost ? end - kPagedPairCost : 0;
        x.whole = x.t1 - x.t0 == x.seen.tiles;
        x.place = place;
        u = p0 + all;
    }
    // false: no (more) part
    IPKV_HD bool begin(PagedPart& x) {
        u = 0; u1 = 0;
        if (share.share > 0) {
            if (cta >= cum[n_rows] * n_gh) return false;
            x.row = row_of(cta);
            const int32_t parts = cum[x.row + 1] - cum[x.row], at = cta - cum[x.row] * n_gh, part = at % parts;
            x.gh = at / parts;
            x.seen = paged_seen(n[x.row], window, first);
            x.t0 = int32_t(int64_t(x.seen.tiles) * part / parts);
            x.t1 = int32_t(int64_t(x.seen.tiles) * (part + 1) / parts);
            x.whole = parts == 1;
            x.place = 2 * cta;
            return true;
        }
        if (cta >= share.ctas) return false;
        u = paged_chunk_begin(share, cta);
        u1 = paged_chunk_begin(share, cta + 1);
        if (u >= u1) return false;
        x.row = row_of(u);
        x.gh = (u - cum[x.row] * n_gh) / (cum[x.row + 1] - cum[x.row]);
        set(x, 2 * cta);
        return true;
    }
    IPKV_HD bool next(PagedPart& x) {
        if (u >= u1) return false;
        if (++x.gh == n_gh) {
            x.gh = 0;
            do ++x.row; while (cum[x.row + 1] == cum[x.row]);
        }
        set(x, 2 * cta + 1);
        return true;
    }
};
// The partials of a pair that has tiles: partial i of n is at place 2 (c0 + i), the first one at the next if it is not its CTA's first part.
// One alone is no partial, but the result, written out.
struct PagedPartials { int32_t c0, n, odd; };
IPKV_HD PagedPartials paged_partials(const PagedShare& s, int32_t cum, int32_t all, int32_t n_gh, int32_t gh) {
    const int32_t first = cum * n_gh + gh * all;
    if (s.share > 0) return {first, all, 0};
    const int32_t c0 = paged_cta_of(s, first + kPagedPairCost);
    return {c0, paged_cta_of(s, first + all - 1) - c0 + 1, paged_chunk_begin(s, c0) < first};
}

// Head groups: a tile is read once for a head group.  Up to 16 query heads are the rows of one product (as one group of 4, 8 or 16 rows);
// more make sixteens, as many to a group as divide both their number and the four computing warps.
inline int paged_rows(int group) { return group <= 4 ? 4 : group <= 8 ? 8 : 16; }
inline int paged_sixteens(int group) {
    const int n = (group + 15) / 16;
    return n % 4 == 0 ? 4 : n % 2 == 0 ? 2 : 1;
}
inline int paged_groups_per_kv(int group) { return (group + 15) / 16 / paged_sixteens(group); }
inline int paged_rows_per_part(int group) { return paged_rows(group) * paged_sixteens(group); }

struct PagedHeader {                             // in front of the scratch, written by the attention for the join
    PagedShare share;
    int32_t cum[kPagedRowsPerLaunch + 1];        // units (parts) of the rows before
};
struct PagedAttend {
    PagedCache c;
    const char* q;                               // row r at r * q_row bytes
    int64_t q_row;
    PagedHeader* header;
    float* part_o;                               // [2 n_ctas][rows_per_part][dim]: sums of weight times value, not divided
    float2* part_ml;                             // [2 n_ctas][rows_per_part]: reference maximum (log2) and sum of weights against it
    float2* head_ml;                             // [n_rows][n_q_heads]: maximum and 1 / sum, for the weights; null without
    float* scores;                               // [n_rows][n_gh][most_tiles][64 rows_per_part], null without weights
    float* weights_out;
    float* out_o;
    float* out_lse;
    uint32_t* status;
    int32_t window, first, most_tiles;
    int32_t n_q_heads, group, groups_per_kv, n_gh, rows_per_part, sixteens;
    int32_t n_ctas;
    int32_t single;                              // one CTA to every pair, which writes the result: no join
    float scale_log2;
};
cudaError_t launch_paged_attend(const PagedAttend& a, cudaStream_t s);

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
};
cudaError_t launch_paged_evict(const PagedEvict& a, cudaStream_t s);

}  // namespace ipkvi
