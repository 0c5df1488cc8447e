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


@pytest.mark.parametrize("n_gh,teams", [(1, 2), (1, 4), (4, 4), (8, 4), (8, 1), (64, 4)])
def test_a_share_fits_the_gpu_and_is_whole_rounds(shim, n_gh, teams):
    """Whole CTAs to every pair: as many as are resident at most (the partials' place is planned for no more), and every team of a
    full one has the same number of tiles."""
    import random
    rng = random.Random(n_gh * 10 + teams)
    sms, n = 148, ctypes.c_int()
    for _ in range(300):
        rows = rng.choice([1, 1, 2, 5, 16, 64, 300])
        most = rng.choice([1, 4, 60, 700, 30000])
        tiles = [rng.randint(0, most) for _ in range(rows)]
        share = shim.shim_nibble_share((ctypes.c_int * rows)(*tiles), rows, n_gh, teams, sms, ctypes.byref(n))
        assert share == -1 or (share >= 0 and share % teams == 0)
        if share == -1:
            assert n.value == rows * n_gh <= sms * shim.shim_nibble_ctas_per_sm()
        elif share:
            assert sum(t > 0 for t in tiles) * n_gh <= n.value <= sms * shim.shim_nibble_ctas_per_sm()


def test_little_work_gets_whole_ctas_and_much_work_equal_chunks(shim):
    n = ctypes.c_int()
    share = lambda tiles: shim.shim_nibble_share((ctypes.c_int * len(tiles))(*tiles), len(tiles), 4, 4, 148, ctypes.byref(n))
    assert share([0, 0]) == -1 and share([1]) == -1 and n.value == 4                 # one CTA to every pair
    assert share([0] * 200) == 0                         # ... if they fit
    assert share([65]) == 4 and n.value == 68
    assert share([32] * 16) in (8, 16) and n.value in (128, 256)
    assert share([512] * 16) == 0 and share([(1 << 31) - 300]) == 0
