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
int shim_nibble_rows(int group) { return nibble_rows_per_part(group); }
}
