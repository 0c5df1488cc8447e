// The operators' host-side rules behind a C interface (test-only).
#include "../paper_2609_14507_b200/csrc/ops.h"

using namespace ipkvi;

extern "C" {
int shim_nibble_warps() { return kNibbleWarps; }
int shim_nibble_teams(int octets) { return nibble_teams(octets); }
int shim_nibble_stages(int dim, int octets) { return nibble_stages(dim, octets); }
int shim_nibble_smem(int dim, int octets) {
    return nibble_stages(dim, octets) * NibbleGeom{1, dim, kTileTokens}.tile_bytes() + nibble_fixed_smem();
}
int shim_nibble_smem_limit() { return kNibbleSmemPerCta; }
int shim_nibble_groups(int group) { return nibble_groups_per_kv(group); }
int shim_nibble_ctas_per_sm() { return kNibbleCtasPerSm; }
// rows of `tiles` tiles -> the share (-1: one CTA to every pair), and how many CTAs it takes
int shim_nibble_share(const int* tiles, int n_rows, int n_gh, int teams, int sms, int* ctas) {
    NibbleRowArg row[4096];
    int64_t units = 0, pairs = 0, longest = 0;
    for (int i = 0; i < n_rows; ++i) {
        row[i] = NibbleRowArg{0, tiles[i], 0, 0};
        if (tiles[i] > longest) longest = tiles[i];
        if (tiles[i] > 0) { units += int64_t(tiles[i] + kNibblePairCost) * n_gh; pairs += n_gh; }
    }
    const NibbleSplit split = nibble_split(row, n_rows, n_gh, teams, units, pairs, longest, sms);
    const int share = split.share;
    *ctas = split.whole ? n_rows * n_gh : 0;
    if (split.whole) return -1;
    for (int i = 0; i < n_rows && share > 0; ++i) *ctas += (tiles[i] + share - 1) / share * n_gh;
    return share;
}
int shim_nibble_rows(int group) { return nibble_rows_per_part(group); }
}
