"""Host-side rules of the attention over a paged cache, without a GPU: what is seen, and how the work is shared out."""
import ctypes
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("shim") / "libpaged_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-I/usr/local/cuda/include", "-o", out, os.path.join(HERE, "paged_shim.cpp")],
                   check=True)
    return ctypes.CDLL(out)


@pytest.mark.parametrize("unit", [32, 64])
def test_the_units_show_every_visible_slot_once_and_no_other(shim, unit):
    rng = random.Random(1)
    cap = 1024
    seen = (ctypes.c_ubyte * cap)()
    for _ in range(3000):
        n = rng.choice([0, 1, 63, 64, 65, cap, rng.randint(0, cap)])
        window = rng.choice([0, 1, 2, 64, 65, cap, 2 ** 31 - 1, rng.randint(1, cap)])
        first = rng.choice([0, 1, 4, 64, 65, cap, 2 ** 31 - 1, rng.randint(0, 200)])
        units = shim.shim_paged_seen(n, window, first, unit, cap, seen)
        want = [int(t < n and (window == 0 or t >= n - window or t < first)) for t in range(cap)]
        assert list(seen) == want, (n, window, first)
        assert 0 <= units <= min(shim.shim_paged_most_units(cap, window, first, unit), shim.shim_paged_most_units(max(n, 1), window, first, unit))
        if window:                                       # no unit without a visible slot
            assert units <= len({t // unit for t in range(cap) if want[t]})


def test_head_groups_cover_the_heads(shim):
    per_kv, rows, sixteens = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    for group in range(1, 300):
        product = shim.shim_paged_group(group, ctypes.byref(per_kv), ctypes.byref(rows), ctypes.byref(sixteens))
        assert product in (4, 8, 16) and sixteens.value in (1, 2, 4) and rows.value == product * sixteens.value
        assert per_kv.value * rows.value >= group > (per_kv.value - 1) * rows.value
        assert product == 16 or (per_kv.value == 1 and sixteens.value == 1)


@pytest.mark.parametrize("ctas", [296, 7, 1])
def test_every_unit_is_taken_once_and_every_partial_is_found(shim, ctas):
    """Any lengths, empty rows among them: each unit by one CTA, each pair's result written by its one CTA or joined from the places where
    its CTAs left their partials."""
    rng = random.Random(ctas)
    most, ways = ctypes.c_int(), ctypes.c_int()
    ways_seen = set()
    for i in range(1500):
        rows = rng.choice([1, 1, 2, 3, 16, 37, 64, 300, 1024])
        n_gh = rng.choice([1, 2, 4, 8, 12])
        longest = rng.choice([0, 1, 64, 65, 500, 4097, min(100000, 60000 * 32 // (rows * n_gh))])
        longest = min(longest, 60000 * 32 // (rows * n_gh) - 64)
        n = [rng.randint(0, longest) if rng.random() < 0.8 else 0 for _ in range(rows)]
        if rows * n_gh > 1 << 14:
            continue
        window, first = rng.choice([(0, 0), (0, 0), (1, 0), (100, 3), (1000, 70), (64, 64)])
        rc = shim.shim_paged_play((ctypes.c_int * rows)(*n), rows, n_gh, window, first, rng.choice([32, 64]), rng.choice([1, 2, 4]), ctas, ctypes.byref(most), ctypes.byref(ways))
        assert rc == 0, (rc, rows, n_gh, window, first)
        ways_seen.add(ways.value > 0)
    assert ways_seen == ({True, False})


def test_little_work_gets_whole_ctas_and_many_pairs_equal_chunks(shim):
    most, ways = ctypes.c_int(), ctypes.c_int()
    play = lambda n, n_gh: shim.shim_paged_play((ctypes.c_int * len(n))(*n), len(n), n_gh, 0, 0, 64, 4, 296, ctypes.byref(most), ctypes.byref(ways))  # noqa: E731
    assert play([4097], 4) == 0 and ways.value == most.value == 4        # a unit for every warp
    assert play([2048] * 16, 4) == 0 and ways.value == most.value == 8
    assert play([2048] * 64, 8) == 0 and ways.value == 0 and most.value <= 64 * 8 * 36 // 296 + 2
    assert play([4097 if r % 3 else 2500 for r in range(32)], 8) == 0 and ways.value == 0      # whole CTAs would be uneven


def test_clusters_take_small_pairs_that_fit_the_gpu(shim):
    rng = random.Random(3)
    for _ in range(2000):
        pairs, units, group = rng.choice([1, 4, 37, 38, 296, 297, rng.randint(1, 400)]), rng.randint(1, 300), rng.choice([1, 4, 8, 16, 17, 40, 64])
        n = shim.shim_paged_cluster(pairs, units, group, 296)
        assert n in (0, 1, 2, 4, 8) or (n == 16 and pairs <= 8)
        assert n == 0 or (pairs * n <= 296 and units <= 24 * n and (group <= 16 or n == 1))
    assert shim.shim_paged_cluster(64, 32, 4, 296) == 4 and shim.shim_paged_cluster(64, 4, 4, 296) == 1 and shim.shim_paged_cluster(4, 1000, 8, 296) == 0
    assert shim.shim_paged_cluster(4, 32, 8, 296) == 8 and shim.shim_paged_cluster(4, 129, 8, 296) == 16 and shim.shim_paged_cluster(9, 129, 8, 296) == 0
    assert shim.shim_paged_cluster(32, 188, 4, 296) == 8
