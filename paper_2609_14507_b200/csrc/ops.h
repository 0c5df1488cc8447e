// Launch interface of the operators beside the cache (ops_api.cu checks the arguments and fills these): head norm with
// rotation, and the cache held in 4 bits.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "nibble.cuh"

namespace ipkvi {

// ---- head norm and rotation (norm_rope.cu) ------------------------------------------------------------------------
constexpr int kRopeMaxParts = 4;
constexpr int kRopeMaxPairs = 128;
struct RopePart {
    const char* in;
    char* out;
    const char* weight;                          // [dim] bf16, null: no norm
    int64_t in_token, in_head, out_token, out_head;   // strides in bytes
    int32_t n_heads;
    int32_t step0;                               // steps (groups of heads that one warp takes at once) of the parts before this one
};
struct RopeLaunch {
    uint64_t turn[kRopeMaxPairs];                // frequency of a pair as a fraction of a turn per position, times 2^64
    uint8_t axis[kRopeMaxPairs];
    RopePart part[kRopeMaxParts];
    const int32_t* positions;                    // [n_axes][n_tokens]
    int64_t n_tokens;
    int32_t n_parts, n_steps, split, dim, rot_dim, n_axes, interleaved;
    float eps;
};
// heads that one warp takes in one step, for a head width
inline int rope_heads_per_step(int dim) { return 512 / dim; }
cudaError_t launch_norm_rope(RopeLaunch& a, cudaStream_t s);

// ---- the cache in 4 bits: writing and reading back (nibble_pack.cu) --------------------------------------------------
constexpr int kNibbleSpansPerLaunch = 96;
struct NibbleSpanArg {
    char* blocks;                                // first block of the run
    int64_t first;                               // first token of the span inside the run
    int64_t src;                                 // its row among the token-major tokens
    int32_t n;                                   // tokens
    int32_t tile0;                               // tiles of the launch's spans before this one
};
struct NibbleMove {
    NibbleSpanArg span[kNibbleSpansPerLaunch];
    NibbleGeom g;
    char* k;                                     // token-major [tokens][n_kv_heads][dim] bf16
    char* v;
    int64_t k_token, v_token;                    // bytes between tokens
    int32_t n_spans, n_tiles;
};
// All spans hold one token (a decode step): one group of lanes per token and head, no tile is moved.
cudaError_t launch_nibble_pack(const NibbleMove& a, bool single_tokens, cudaStream_t s);
cudaError_t launch_nibble_unpack(const NibbleMove& a, bool single_tokens, cudaStream_t s);

// ---- the cache in 4 bits: decode attention (nibble_attend.cu) --------------------------------------------------------
// A pair is a row and a head group (a KV head and some of its query heads); its tiles of 64 tokens are work for one CTA or several,
// which leave a partial (O, maximum, sum) of every team.  Three ways to share the pairs out, see nibble_split:
//  - one CTA to every pair, those without tiles too: it joins its teams' partials itself and writes the result, in one launch;
//  - whole CTAs to every pair: ceil(tiles / share) of them, each an equal part of the pair's tiles; partials in the CTAs' order;
//  - equal chunks: work is counted in units, a pair's tiles and its cost in front of them, pair after pair, and CTA c of n takes units
//    [units c / n, units (c + 1) / n).  With j the index of the pair among those with tiles, the partials that CTA c has of
//    it go to place c + j: distinct, and consecutive for a pair.
// So neither needs tables beside the rows'.
// The cost of a pair, in tiles: queries read, a partial written, the pipeline drained.  Without it the CTA with the shortest
// sequences was the last: 64 ragged rows of up to 24K tokens 183 us, 162 with 4 (171 with 2, 163 with 12); rows of up to 2K
// tokens 48 and 29 us.
constexpr int kNibblePairCost = 4;
struct NibbleRunArg {
    const char* blocks;
    int32_t n_tokens;
    int32_t tile0;                               // tiles of the row's runs before this one
};
struct NibbleRowArg {
    int32_t first;                               // units (whole CTAs to every pair: CTAs) of the rows before this one
    int32_t tiles;                               // tiles of the row
    int32_t run0;                                // its first run (runs without tokens are left out)
    int32_t pair0;                               // (row, head group) pairs with tiles before this row's
};
constexpr int kNibbleWarps = 4, kNibbleCtasPerSm = 3;              // warps that compute, beside the one that copies
constexpr int kNibbleInlineRows = 64, kNibbleInlineRuns = 128;      // tables up to this size travel as launch parameters
// Shared memory of a CTA: the stages and this.
constexpr int kNibbleMaxStages = 16;
struct NibbleSmem {
    uint64_t full[kNibbleMaxStages], empty[kNibbleMaxStages];
    int32_t n_valid[kNibbleMaxStages];
};
constexpr int kNibbleSmemPerCta = 228 * 1024 / kNibbleCtasPerSm - 1024;
// A tile is worked on by one team of `octets` warps.
inline int nibble_teams(int octets) { return kNibbleWarps / octets; }
inline int nibble_fixed_smem() { return int(sizeof(NibbleSmem)) + 128; }         // 128: to align the stages
// Stages of the copy ring: as many as fit, in a multiple of the teams, so that every stage has one team.  A warp that waits for a lap of
// a stage can tell that lap from the one before only if it has seen the one before complete itself; with another team's
// tile in the stage before its own it could run ahead of a copy that lands late, take the old tile for the new one and release the stage.
inline int nibble_stages(int dim, int octets) {
    const int teams = nibble_teams(octets), tile = NibbleGeom{1, dim, kTileTokens}.tile_bytes();
    if (teams < 1) return 0;
    int n = (kNibbleSmemPerCta - nibble_fixed_smem()) / tile;
    if (n > kNibbleMaxStages) n = kNibbleMaxStages;
    return n / teams * teams;
}
struct NibbleAttend {
    NibbleRowArg row[kNibbleInlineRows];
    NibbleRunArg run[kNibbleInlineRuns];
    const NibbleRowArg* rows;                    // tables on the device, null: the ones above
    const NibbleRunArg* runs;
    NibbleGeom g;
    const char* q;                               // [n_rows][n_q_heads][dim] bf16
    float* part_o;                               // [partials][teams][rows_per_part][dim]
    float2* part_ml;                             // [partials][teams][rows_per_part]: reference maximum (log2) and sum of weights against it
    float* out_o;
    float* out_lse;
    uint32_t* status;                            // may be null
    int64_t part_rows;                           // partial rows that the scratch holds (bounds-checked build)
    int32_t n_rows, n_units, n_ctas, n_q_heads, group, groups_per_kv, n_gh, rows_per_part;
    int32_t teams;                               // teams of warps in a CTA
    int32_t octets;                              // groups of 8 query heads in a head group
    int32_t stages, n_runs;
    int32_t whole;                               // one CTA for every pair, which writes the result itself
    int32_t share;                               // whole CTAs to every pair: tiles that one takes at most; 0: equal chunks of all units
    int32_t max_parts;                           // partials of a (row, head group) at most
    uint32_t odd_tokens;                         // 0xffff0000, see the kernel
    int32_t plain_launch;                        // the tables were written by the kernel in front of this launch: no overlap with it
    float scale;
};
// Head groups of a KV head's `group` query heads, and heads in each.  One warp per 8 heads works on a tile, and the tile is read once for a
// group: as many octets as divide both the computing warps and the octets there are, so that no warp is idle (40 heads on one KV head, 200K
// tokens: 36 us; in two groups of 24 and 16, three warps of four busy, 51, though the tiles were read twice in place of five times).
// Sharing reads a tile once and gives a group fewer teams, so it wins where the copies bound and loses a little elsewhere.  In us, shared
// and (in brackets) one octet a group, 128 columns: 32 heads on one KV head, 200K tokens 30.9 (37.7), 20K 12.2 (11.2), 8 rows of 20K 27.9
// (26.9); 16 heads, 1M 61.8 (63.0), 200K 27.6 (24.9), 8 x 20K 19.3 (18.1), 40 x 600 9.6 (9.0), 1K 7.3 (7.7); 48 heads, 200K 39.8 (39.8).
inline int nibble_group_octets(int group) {
    const int n = (group + 7) / 8;
    return n % 4 == 0 ? 4 : n % 2 == 0 ? 2 : 1;
}
inline int nibble_groups_per_kv(int group) { return (group + 7) / 8 / nibble_group_octets(group); }
inline int nibble_rows_per_part(int group) { return nibble_groups_per_kv(group) == 1 ? group : 8 * nibble_group_octets(group); }
static_assert(kNibbleWarps == 4, "octets of a group");
// How to share out the pairs: whole (one CTA to every pair); or else share, the tiles that a CTA takes at most where every pair has
// whole CTAs, 0 for equal chunks.
// A team that works off k tiles takes about (us, 128 columns, 4 query heads per KV head; 8 take a sixth more)
//   7 + 1.3 k with one CTA to an SM,   9.3 + 1.75 k with two,   9.5 + 2.5 k with three,
// and the chunks, which fill all SMs to the same degree but meet two pairs and more, with r rounds of tiles on three CTAs,
//   11.5 + 2.4 r, 5.5 more if there are several pairs
// (fitted there, and used as they are for 64 columns and for teams of several warps).
// Whole CTAs win where there is little work for each SM (one row of 4K tokens of 4 KV heads 8.6 us against 10.6, 16 rows of 2K 12.7 against
// 18.2, 32 ragged rows of up to 2K and 8 KV heads 17.5 against 27), chunks with more (16 rows of 32K 66 us against 71, 48 ragged rows
// of up to 8K 45 against 58).  One CTA to a pair saves the join, 2.5 us, and its launch on the host: a call on one row of 768 tokens and 4 KV
// heads (three tiles a team) 8.5 us and 9.2 with the tiles spread over more CTAs, 1024 tokens 9.7 and 9.2; 32 rows of 1024 11.0 and 14.7.
struct NibbleSplit { bool whole; int share; };
constexpr int kNibbleWholeTiles = 3;             // tiles a team up to which the launch saved decides
inline NibbleSplit nibble_split(const NibbleRowArg* row, int n_rows, int n_gh, int teams, int64_t units, int64_t pairs, int64_t longest, int sms) {
    const int64_t most = int64_t(sms) * kNibbleCtasPerSm, all = int64_t(n_rows) * n_gh, whole_tiles = (longest + teams - 1) / teams;
    if (all <= most && whole_tiles <= kNibbleWholeTiles) return {true, 0};
    const float rounds = float(units) / float(most * teams);
    if (pairs == 0 || pairs > most || rounds > 24.f) return {false, 0};
    const float at0[kNibbleCtasPerSm] = {7.f, 9.3f, 9.5f}, per_tile[kNibbleCtasPerSm] = {1.3f, 1.75f, 2.5f};
    auto ctas = [&](int share) {
        int64_t n = 0;
        for (int r = 0; r < n_rows; ++r) n += (row[r].tiles + share - 1) / share;
        return n * n_gh;
    };
    float best = 11.5f + 2.4f * rounds + (pairs > 1 ? 5.5f : 0.f);
    int share = 0;
    for (int w = 0; w < kNibbleCtasPerSm; ++w) {
        const int64_t limit = int64_t(sms) * (w + 1);
        if (pairs > limit) continue;
        // the fewest tiles a team with which the CTAs stay within the limit; they only get fewer with more tiles a team
        const float most_tiles = (best - at0[w]) / per_tile[w];          // not better from here on
        if (most_tiles < 1.f) continue;
        int lo = 1, hi = int(most_tiles);
        if (ctas(hi * teams) > limit) continue;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (ctas(mid * teams) <= limit) hi = mid; else lo = mid + 1;
        }
        const float t = at0[w] + per_tile[w] * float(lo);
        if (t < best) { best = t; share = lo * teams; }
    }
    if (all <= most) {
        const int w = int((all - 1) / sms);
        if (at0[w] - 2.5f + per_tile[w] * float(whole_tiles) < best) return {true, 0};
    }
    return {false, share};
}
cudaError_t launch_nibble_attend(NibbleAttend& a, cudaStream_t s);

}  // namespace ipkvi
