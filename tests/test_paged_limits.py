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
