"""What the paged cache does with bad lengths and pages, all made on the host and checked by the kernels, and with infinities."""
import pytest

from paper_2609_14507_b200 import binding
from tests import paged_ref as ref
from tests.test_paged import BAD_PAGE, Case

torch = pytest.importorskip("torch")


def pool_like(c, data):
    p = ref.Pool.__new__(ref.Pool)
    p.__dict__.update(c.pool.__dict__, data=data)
    return p


# ---- append ----------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("bad", [-1, -5, -2 ** 31])
@pytest.mark.parametrize("chunks", [False, True])
def test_an_append_tells_of_a_length_below_zero(bad, chunks):
    """It takes no token, as a row of length zero does, but that one is no mistake."""
    c = Case([40, 3, 64], 4, 2, 64, 64, per_row=2)
    c.lengths[1] = bad
    new = [2, 3, 1] if chunks else [1, 1, 1]
    total = sum(new)
    k, v = (torch.randn((total, 2, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
    at = torch.arange(1000, 1000 + total, dtype=torch.int32, device="cuda")
    start = torch.tensor([0] + [sum(new[:i + 1]) for i in range(3)], dtype=torch.int32, device="cuda") if chunks else None
    want, w, pos = pool_like(c, c.pool.data.clone()), c.weights.clone(), c.positions.clone()
    for r, n in ((0, 40), (2, 64)):
        first, slots = sum(new[:r]), list(range(n - new[r], n))
        want.put(c.pages[r], slots, k[first:first + new[r]], v[first:first + new[r]])
        w[r][:, slots] = 0.0
        pos[r][:, slots] = at[first:first + new[r]]
    binding.ipkv_paged_append(c.shape, c.cache(), k, v, positions=at, row_start=start, status=c.status)
    assert int(c.status) == BAD_PAGE
    assert torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16)) and torch.equal(c.weights, w) and torch.equal(c.positions, pos)
    c.status.zero_()
    c.lengths[1] = 0
    binding.ipkv_paged_append(c.shape, c.cache(), k, v, positions=at, row_start=start, status=c.status)
    assert int(c.status) == 0 and torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16))
    binding.ipkv_paged_append(c.shape, c.cache(), k, v, positions=at, row_start=start)       # nobody asks
