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


# ---- infinities ------------------------------------------------------------------------------------------------------

INF = float("inf")
HOW = {"cluster": [500, 500, 300], "large cluster": [3000], "shares": [20000, 500], "chunks": [3000] * 200}


@pytest.mark.gpu
@pytest.mark.parametrize("how", HOW)
@pytest.mark.parametrize("hq,hkv,d,bt", [(4, 1, 128, 64), (16, 2, 64, 16), (16, 1, 128, 32), (40, 1, 64, 64)])
def test_infinite_keys_and_values(hq, hkv, d, bt, how):
    """A score of +inf makes its head NaN, one of -inf is a weight of zero, and an infinite value makes its column infinite or NaN; other heads, rows and
    columns are as they were."""
    c = Case(HOW[how], hq, hkv, d, bt)
    r, t, g = len(c.n) - 1, c.n[-1] - 77, hq // hkv
    c.q[r, :, 5] = torch.where(torch.arange(hq, device="cuda") % 2 == 0, 1.0, -1.0).to(torch.bfloat16)
    k, v = c.pool.get(c.pages[r], [t])
    for value in (INF, -INF):
        x = k.clone()
        x[0, hkv - 1, 5] = value
        c.pool.put(c.pages[r], [t], x, v)
        out = torch.full_like(c.weights, 3.0)
        o, lse = c.attend(weights_out=out)
        head = torch.arange(hq, device="cuda")
        up = (head >= (hkv - 1) * g) & ((head % 2 == 0) == (value > 0))          # the heads whose score is +inf
        assert torch.isnan(o[r][up]).all() and torch.isnan(lse[r][up]).all()
        assert torch.isfinite(o[r][~up]).all() and torch.isfinite(lse[r][~up]).all()
        assert torch.isfinite(o[:r]).all() and torch.isfinite(lse[:r]).all() and torch.isfinite(out[:r]).all()
        seen = [s for s in range(c.n[r]) if s != t]      # for the others, the slot is not there
        eo, el, ep, to, tl, tp = ref.attend(c.q[r], *c.pool.get(c.pages[r], seen), c.scale)
        down = (head >= (hkv - 1) * g) & ~up
        assert (o[r].double() - eo).abs().le(to)[down].all() and (lse[r].double() - el).abs().le(tl)[down].all()
    c.pool.put(c.pages[r], [t], k, v)
    for value in (INF, -INF):
        x = v.clone()
        x[0, hkv - 1, 5] = value
        c.pool.put(c.pages[r], [t], k, x)
        o, lse = c.attend()
        bad = torch.zeros_like(o, dtype=torch.bool)
        bad[r, (hkv - 1) * g:, 5] = True
        assert not torch.isfinite(o[bad]).any() and torch.isfinite(o[~bad]).all() and torch.isfinite(lse).all()
    c.pool.put(c.pages[r], [t], k, v)


@pytest.mark.gpu
@pytest.mark.parametrize("how", HOW)
def test_a_row_whose_scores_are_all_minus_infinity(how):
    c = Case(HOW[how], 4, 1, 64, 32)
    r = len(c.n) - 1
    k, v = c.pool.get(c.pages[r], list(range(c.n[r])))
    k[:, 0, 9] = -INF
    c.pool.put(c.pages[r], list(range(c.n[r])), k, v)
    c.q[r, :, 9] = 1.0
    out = torch.full_like(c.weights, 3.0)
    o, lse = c.attend(weights_out=out)
    assert (o[r] == 0).all() and torch.isneginf(lse[r]).all() and torch.isfinite(lse[:r]).all()
    assert torch.equal(out[r, 0, :c.n[r]], c.weights[r, 0, :c.n[r]]) and (out[r, 0, c.n[r]:] == 3.0).all()
    c.check(o, lse, rows=list(range(r)))
