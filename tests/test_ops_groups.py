"""Groups of query heads of the 4-bit attention, without a GPU."""
from tests.test_ops_host import shim  # noqa: F401


def test_every_warp_of_a_cta_has_a_team_whatever_the_heads(shim):        # noqa: F811
    warps = shim.shim_nibble_warps()
    for group in range(1, 2000):
        octets = (shim.shim_nibble_rows(group) + 7) // 8                 # of a head group: the warps of a team
        assert warps % octets == 0 and shim.shim_nibble_teams(octets) * octets == warps
        groups, all_octets = shim.shim_nibble_groups(group), (group + 7) // 8
        assert groups * octets == all_octets                             # no octet of a group is empty
