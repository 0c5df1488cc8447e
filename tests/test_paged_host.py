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


def test_the_tiles_show_every_visible_slot_once_and_no_other(shim):
    rng = random.Random(1)
    cap = 1024
    seen = (ctypes.c_ubyte * cap)()
    for _ in range(3000):
        n = rng.choice([0, 1, 63, 64, 65, cap, rng.randint(0, cap)])
        window = rng.choice([0, 1, 2, 64, 65, cap, 2 ** 31 - 1, rng.randint(1, cap)])
        first = rng.choice([0, 1, 4, 64, 65, cap, 2 ** 31 - 1, rng.randint(0, 200)])
        tiles = shim.shim_paged_seen(n, window, first, cap, seen)
        want = [int(t < n and (window == 0 or t >= n - window or t < first)) for t in range(cap)]
        assert list(seen) == want, (n, window, first)
        assert 0 <= tiles <= min(shim.shim_paged_most_tiles(cap, window, first), shim.shim_paged_most_tiles(max(n, 1), window, first))
        if window:                                       # no tile without a visible slot
            assert tiles <= len({t // 64 for t in range(cap) if want[t]})


def test_head_groups_cover_the_heads(shim):
    per_kv, rows, sixteens = ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
    for group in range(1, 300):
        product = shim.shim_paged_group(group, ctypes.byref(per_kv), ctypes.byref(rows), ctypes.byref(sixteens))
        assert product in (4, 8, 16) and sixteens.value in (1, 2, 4) and rows.value == product * sixteens.value
        assert per_kv.value * rows.value >= group > (per_kv.value - 1) * rows.value
        assert product == 16 or (per_kv.value == 1 and sixteens.value == 1)


@pytest.mark.parametrize("ctas", [296, 7, 1])
def test_every_tile_is_taken_once_and_every_partial_is_found(shim, ctas):
    """Any lengths, empty rows among them: each tile by one CTA, each pair's result written by its one CTA or joined from the places where
    its CTAs left their partials."""
    rng = random.Random(ctas)
    most, ways = ctypes.c_int(), ctypes.c_int()
    ways_seen = set()
    for i in range(1500):
        rows = rng.choice([1, 1, 2, 3, 16, 37, 64, 300, 1024])
        n_gh = rng.choice([1, 2, 4, 8, 12])
        longest = rng.choice([0, 1, 64, 65, 500, 4097, min(100000, 60000 * 64 // (rows * n_gh))])
        longest = min(longest, 60000 * 64 // (rows * n_gh) - 64)
        n = [rng.randint(0, longest) if rng.random() < 0.8 else 0 for _ in range(rows)]
        if rows * n_gh > 1 << 14:
            continue
        window, first = rng.choice([(0, 0), (0, 0), (1, 0), (100, 3), (1000, 70), (64, 64)])
        rc = shim.shim_paged_play((ctypes.c_int * rows)(*n), rows, n_gh, window, first, ctas, ctypes.byref(most), ctypes.byref(ways))
        assert rc == 0, (rc, rows, n_gh, window, first)
        ways_seen.add(ways.value > 0)
    assert ways_seen == ({True, False})


def test_little_work_gets_whole_ctas_and_many_pairs_equal_chunks(shim):
    most, ways = ctypes.c_int(), ctypes.c_int()
    play = lambda n, n_gh: shim.shim_paged_play((ctypes.c_int * len(n))(*n), len(n), n_gh, 0, 0, 296, ctypes.byref(most), ctypes.byref(ways))  # noqa: E731
    assert play([4097], 4) == 0 and ways.value == most.value == 1
    assert play([2048] * 16, 4) == 0 and ways.value in (7, 8) and most.value == ways.value
    assert play([2048] * 64, 8) == 0 and ways.value == 0 and most.value <= 64 * 8 * 34 // 296 + 2
