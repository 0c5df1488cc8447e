"""Host-side rules of the 4-bit cache's attention, without a GPU."""
import ctypes
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("shim") / "libops_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-I/usr/local/cuda/include", "-o", out, os.path.join(HERE, "ops_shim.cpp")],
                   check=True)
    return ctypes.CDLL(out)


@pytest.mark.parametrize("dim", [64, 128])
def test_every_stage_of_the_copy_ring_has_one_team(shim, dim):
    """A stage that laps of different teams share can be released before its tile has landed: the teams divide the stages."""
    for octets in range(1, shim.shim_nibble_warps() + 1):
        teams, stages = shim.shim_nibble_teams(octets), shim.shim_nibble_stages(dim, octets)
        assert teams >= 1 and stages >= teams and stages % teams == 0
        assert stages >= 2 * teams                       # a tile under way for every team beside the one it works on
        assert shim.shim_nibble_smem(dim, octets) <= shim.shim_nibble_smem_limit()


def test_head_groups_cover_the_heads_and_fit_the_warps(shim):
    for group in range(1, 300):
        n, rows = shim.shim_nibble_groups(group), shim.shim_nibble_rows(group)
        assert n * rows >= group > (n - 1) * rows        # no group is empty
        assert (rows + 7) // 8 <= shim.shim_nibble_warps()
        assert n == 1 or rows % 8 == 0
