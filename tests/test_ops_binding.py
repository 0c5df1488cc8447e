"""The binding of the operators beside the cache, on the host: first calls from several threads, and what it refuses by itself."""
import sys

import pytest

from paper_2609_14507_b200 import binding

torch = pytest.importorskip("torch")


def fresh(monkeypatch):
    """As before the first call."""
    names = [n for n in ("_torch", "_np", "_bf16", "_f32", "_i32", "_int64", "_int32", "_current_device", "_current_stream") if hasattr(binding, n)]
    for n in names:
        monkeypatch.setattr(binding, n, None)
    return names


def test_a_call_that_finds_the_modules_finds_all_of_them(monkeypatch):
    """The entry points look at one name to know whether the others are there: whichever line of the first call another thread
    interrupts, that name comes last."""
    names = fresh(monkeypatch)
    seen = []

    def trace(frame, event, arg):
        if frame.f_code is binding._modules.__code__:
            seen.append((binding._torch is not None, [n for n in names if getattr(binding, n) is None]))
        return trace

    sys.settrace(trace)
    try:
        binding._modules()
    finally:
        sys.settrace(None)
    assert seen and binding._torch is torch
    assert all(not missing for there, missing in seen if there)


def test_the_stream_is_found_without_the_names_that_torch_keeps_to_itself(monkeypatch):
    class Stream:
        cuda_stream = 77

    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream() if device == 3 else None)
    fresh(monkeypatch)
    binding._modules()
    assert binding._call_stream(None, 3) == 77
    assert binding._call_stream(5, 3) == 5 and binding._call_stream(Stream(), 3) == 77
    for dev in (-1, 0):
        with pytest.raises(ValueError):
            binding._call_stream(None, dev)


def test_positions_lie_axis_by_axis():
    """A table with one row per token has the same number of entries, and would be read as if its rows were axes."""
    rope = binding.make_rope(64, sections=[8, 12, 12])
    x = torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    for shape in ((5, 3), (3, 5, 1), (1, 15)):
        with pytest.raises(ValueError, match="positions"):
            binding.ipkv_norm_rope(rope, [(x, None, None)], torch.zeros(shape, dtype=torch.int32))
    for rope, shape in ((rope, (3, 5)), (rope, (15,)), (binding.make_rope(64), (5,)), (binding.make_rope(64), (1, 5)), (binding.make_rope(64), (5, 1))):
        with pytest.raises(ValueError, match="on device -1"):            # refused for nothing but being on the host
            binding.ipkv_norm_rope(rope, [(x, None, None)], torch.zeros(shape, dtype=torch.int32))


def test_blocks_of_another_place_and_tables_that_are_tensors_are_refused():
    """A row of a table that names a tensor means that tensor's memory: on the host, or on another device, a kernel would run into it.
    A table that is a tensor itself would name the places of its own entries."""
    class Elsewhere:                                     # a tensor of the second device, as far as the binding can see
        def data_ptr(self): return 1 << 20
        def get_device(self): return 1

    shape = binding.make_shape(binding.GQA, 4, 2, 64, 64, 64, 0.0)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    q, o, lse, scratch = torch.zeros((1, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 4, 64)), torch.zeros((1, 4)), torch.zeros(64, dtype=torch.uint8)
    start = torch.tensor([0, 1], dtype=torch.int32).numpy()
    blocks = torch.zeros(4608 * 2, dtype=torch.uint8)
    for move in (binding.ipkv_nibble_pack, binding.ipkv_nibble_unpack):
        with pytest.raises(ValueError, match="blocks"):
            move(shape, [(Elsewhere(), 0, 3)], k, k)
        with pytest.raises(ValueError, match="table"):
            move(shape, torch.tensor([[1 << 20, 0, 3]]), k, k)
        with pytest.raises(ValueError, match="on device -1"):            # blocks where K and V are: refused for being on the host
            move(shape, [(blocks, 0, 3)], k, k)
    with pytest.raises(ValueError, match="blocks"):
        binding.ipkv_nibble_attend(shape, [[(Elsewhere(), 3)]], None, q, scratch, o, lse)
    for runs, row_start in ((torch.tensor([[1 << 20, 3]]), start), (torch.tensor([[[1 << 20, 3]]]), None), ([torch.tensor([[1 << 20, 3]])], None)):
        with pytest.raises(ValueError, match="table"):
            binding.ipkv_nibble_attend(shape, runs, row_start, q, scratch, o, lse)
    with pytest.raises(ValueError, match="on device -1"):
        binding.ipkv_nibble_attend(shape, [[(blocks, 3)]], None, q, scratch, o, lse)


@pytest.mark.gpu
def test_host_blocks_are_refused_beside_device_tensors():
    shape = binding.make_shape(binding.GQA, 4, 2, 64, 64, 64, 0.0)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    blocks = torch.zeros(4608 * 2, dtype=torch.uint8)
    for move in (binding.ipkv_nibble_pack, binding.ipkv_nibble_unpack):
        with pytest.raises(ValueError, match="blocks"):
            move(shape, [(blocks, 0, 3)], k, k)
    q, o, lse = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 4, 64), device="cuda"), torch.zeros((1, 4), device="cuda")
    scratch = torch.zeros(binding.ipkv_nibble_scratch_bytes(shape, 1, 1), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="blocks"):
        binding.ipkv_nibble_attend(shape, [[(blocks, 3)]], None, q, scratch, o, lse)


def test_a_call_without_heads_is_refused():
    with pytest.raises(ValueError, match="1 to 4"):
        binding.ipkv_norm_rope(binding.make_rope(64), [], None)
