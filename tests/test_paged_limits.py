"""The paged cache at the ends of what it counts in 32 bits (host side: these calls are refused before anything is read)."""
import ctypes as C

import pytest

from paper_2609_14507_b200 import binding
from tests.test_paged import EINVAL, append_rc, attend_rc, evict_rc, shape_of, struct

MOST = 2 ** 31 - 1 - 2 ** 21                             # slots of a row


@pytest.mark.parametrize("bt", [16, 64, 4096])
def test_rows_whose_slots_leave_no_room_for_a_step_are_refused(bt):
    """A thread goes along a row in 32-bit steps of up to 148 * 8 CTAs of 1024 slots.  With fewer slots than that below 2^31 its
    counter would pass 2^31 and go on below zero, in front of the scores and the weights."""
    step = 148 * 8 * 256 * 4                             # the weights' kernel; the eviction: 32 warps of 128 slots
    assert MOST + step + 4 * 256 <= 2 ** 31 - 1 and 32 * 128 + 4 * 128 < step
    sh, n = shape_of(4, 1, 64, bt), C.c_size_t()
    for blocks in (MOST // bt + 1, (2 ** 31 - 1 - 256) // bt, 2 ** 31 // bt, 2 ** 31 - 1):
        c = struct(max_blocks=blocks, table_stride=blocks, slot_stride=2 ** 32)
        assert append_rc(sh, c) == attend_rc(sh, c) == evict_rc(sh, c) == EINVAL, blocks
        assert binding.lib().ipkv_paged_scratch_bytes(C.byref(sh), 1, blocks, 0, 0, 1, C.byref(n)) == EINVAL
        assert binding.lib().ipkv_paged_evict_scratch_bytes(C.byref(sh), 1, blocks, 100, C.byref(n)) == EINVAL
    assert binding.lib().ipkv_paged_scratch_bytes(C.byref(sh), 1, MOST // bt, 0, 0, 1, C.byref(n)) == 0
    assert binding.lib().ipkv_paged_evict_scratch_bytes(C.byref(sh), 1, MOST // bt, 100, C.byref(n)) == 0


def test_where_the_device_places_no_cluster_of_sixteen_eight_are_taken(tmp_path):
    """The same rule for clusters of sixteen and for devices without: up to eight nothing differs, and what sixteen would have taken is
    taken by eight where they would take it, or shared out and joined."""
    import os
    import random
    import subprocess
    here = os.path.dirname(os.path.abspath(__file__))
    src, so = tmp_path / "cluster.cpp", tmp_path / "libcluster.so"
    src.write_text('#include "paged.h"\nusing namespace ipkvi;\nextern "C" int cluster(int pairs, int units, int group, int ctas, int largest) {\n'
                   '    return paged_cluster(pairs, units, group, paged_sixteens(group), ctas, largest); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-I/usr/local/cuda/include", "-I", os.path.join(here, "..", "paper_2609_14507_b200", "csrc"), "-o", str(so), str(src)],
                   check=True)
    shim, rng, sixteens = C.CDLL(str(so)), random.Random(7), 0
    for _ in range(3000):
        pairs, units, group = rng.choice([1, 4, 8, 9, 37, 296, rng.randint(1, 400)]), rng.randint(1, 300), rng.choice([1, 4, 8, 16, 17, 64])
        with16, with8 = shim.cluster(pairs, units, group, 296, 16), shim.cluster(pairs, units, group, 296, 8)
        assert with8 in (0, 1, 2, 4, 8) and pairs * with8 <= 296 and units <= 24 * with8 + (with8 == 0) * 300
        sixteens += with16 == 16
        assert with16 == with8 or (pairs <= 8 and with16 in (0, 16)), (pairs, units, group)
    assert sixteens > 50
    assert shim.cluster(4, 64, 8, 296, 8) == 8 and shim.cluster(4, 64, 8, 296, 16) == 16
    assert shim.cluster(4, 129, 8, 296, 8) == 0 and shim.cluster(4, 129, 8, 296, 16) == 16


def test_weights_and_positions_without_slots_are_refused():
    """They would pass for arrays that are not there: weights silently not counted, positions silently not kept."""
    torch = pytest.importorskip("torch")
    sh = shape_of(4, 2, 64, 64)
    pool = torch.zeros((3, 2, 2, 64 * 64), dtype=torch.bfloat16)
    table, lengths = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    w, pos = torch.zeros((2, 2, 192)), torch.zeros((2, 2, 192), dtype=torch.int32)
    for a in ((w[:, :, :0],), (w[:, :, :0], pos), (None, pos[:, :, :0]), (w, pos[:, :, :0]), (w[:, :, :0], pos[:, :, :0]), (torch.tensor(1.0),), (w, torch.tensor(1, dtype=torch.int32)),
              (w[0, 0],), (w[None],)):
        with pytest.raises(ValueError):
            binding.make_paged(sh, pool, table, lengths, *a)
    c = binding.make_paged(sh, pool, table, lengths, w, pos)
    assert (c.slot_stride, binding.make_paged(sh, pool, table, lengths, None, pos).slot_stride, binding.make_paged(sh, pool, table, lengths).slot_stride) == (192, 192, 192)
    none = binding.make_paged(sh, pool, table[:0], lengths[:0], w[:0, :, :0])        # without rows nothing needs a slot
    assert none.n_rows == 0


def test_scratch_is_told_for_the_numbers_that_the_calls_take():
    """2^32 + 5 would have been answered as 5."""
    torch = pytest.importorskip("torch")
    sh = shape_of(4, 2, 64, 64)
    c = binding.make_paged(sh, torch.zeros((3, 2, 2, 64 * 64), dtype=torch.bfloat16), torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    for kw in (dict(window=2 ** 32 + 5), dict(window=2 ** 31), dict(window=5, first=2 ** 32), dict(window=-2 ** 31 - 1), dict(window=1.5)):
        with pytest.raises(ValueError):
            binding.ipkv_paged_scratch_bytes(sh, c, **kw)
    for budget in (2 ** 32 + 7, 2 ** 31, -2 ** 31 - 1, 1.5):
        with pytest.raises(ValueError):
            binding.ipkv_paged_evict_scratch_bytes(sh, c, budget)
    with pytest.raises(binding.IpkvError):
        binding.ipkv_paged_scratch_bytes(sh, c, window=-1)
    with pytest.raises(binding.IpkvError):
        binding.ipkv_paged_evict_scratch_bytes(sh, c, 0)
    assert binding.ipkv_paged_scratch_bytes(sh, c, 2 ** 31 - 1, 2 ** 31 - 1) == binding.ipkv_paged_scratch_bytes(sh, c)
    assert binding.ipkv_paged_evict_scratch_bytes(sh, c, 2 ** 31 - 1) == 0
