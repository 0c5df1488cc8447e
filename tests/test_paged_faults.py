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


# ---- eviction --------------------------------------------------------------------------------------------------------

def evict(c, budget, first, recent, n, bad=(), in_place=False, told=None):
    """Evicts and compares everything, byte for byte: pool, weights, positions, kept.  n: the lengths that count; bad: entries (row, page of
    the row) of the table that name no block.  K and V of a move from or to such a page stay as they are, all else moves."""
    w, pos, data = c.weights.clone(), c.positions.clone(), c.pool.data.clone()
    cache = c.cache()
    scratch = torch.randint(0, 256, (max(256, binding.ipkv_paged_evict_scratch_bytes(c.shape, cache, budget)),), dtype=torch.uint8, device="cuda")
    wo, po = (None, None) if in_place else (torch.full_like(w, -9.0), torch.full_like(pos, -9))
    kept = torch.full((len(n), c.hkv, budget), -9, dtype=torch.int32, device="cuda")
    c.status.zero_()
    binding.ipkv_paged_evict(c.shape, cache, budget, first, recent, scratch, wo, po, kept, status=c.status)
    old, want = pool_like(c, data), pool_like(c, data.clone())
    ww, wp = (w.clone(), pos.clone()) if in_place else (torch.full_like(w, -9.0), torch.full_like(pos, -9))
    wk, left_out, moves = torch.full_like(kept, -9), 0, 0
    for r, m in enumerate(n):
        for h in range(c.hkv if m else 0):
            src = ref.kept(w[r, h, :m].tolist(), pos[r, h, :m].tolist(), budget, first, recent)
            at = torch.tensor(src, device="cuda")
            wk[r, h, :len(src)] = at.int()
            ww[r, h, :len(src)], wp[r, h, :len(src)] = w[r, h][at], pos[r, h][at]
            moved = [i for i, s in enumerate(src) if i != s]
            good = [i for i in moved if (r, i // c.bt) not in bad and (r, src[i] // c.bt) not in bad]
            left_out += len(moved) - len(good)
            moves += len(good)
            if good:
                k, v = want.get(c.pages[r], good)
                k0, v0 = old.get(c.pages[r], [src[i] for i in good])
                k[:, h], v[:, h] = k0[:, h], v0[:, h]
                want.put(c.pages[r], good, k, v)
    wo, po = (c.weights, c.positions) if in_place else (wo, po)
    assert torch.equal(kept, wk)
    assert torch.equal(wo.view(torch.int32), ww.view(torch.int32)) and torch.equal(po, wp)
    assert torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16))
    assert int(c.status) == (BAD_PAGE if (left_out if told is None else told) else 0)
    return left_out, moves


BAD_ENTRIES = (-1, 2 ** 31 - 1, -2 ** 31, None)          # None: one behind the pool's last


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("hkv,d,bt,lengths,budget", [(2, 64, 64, [300, 300, 180], 150), (1, 128, 16, [300, 77, 300], 100), (4, 64, 32, [2100, 2100], 700), (1, 64, 256, [30000, 700], 600)])
def test_an_eviction_leaves_bad_pages_out_and_moves_the_rest(hkv, d, bt, lengths, budget, in_place):
    for i, entry in enumerate(BAD_ENTRIES):
        for where in ("behind", "below", "both"):
            c = Case(lengths, hkv, hkv, d, bt, seed=i)
            bad = {(0, (budget + lengths[0]) // 2 // bt)} if where != "below" else set()
            bad |= {(0, 0)} if where != "behind" else set()
            for r, j in bad:
                c.table[r, j] = c.pool.data.shape[0] if entry is None else entry
            left_out, moves = evict(c, budget, 2, 20, lengths, bad, in_place)
            assert left_out and moves


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lengths", [[300, 300, 299], [5000, 5000, 1200]])
def test_one_slot_goes_from_or_to_a_bad_page(lengths, in_place):
    budget = lengths[0] - 1
    for i, entry in enumerate(BAD_ENTRIES):
        for where in ("behind", "below", "both"):
            c = Case(lengths, 2, 2, 64, 16, seed=i)
            gone = [7, lengths[0] - 5]                   # of the two heads: the slot that goes
            for h in range(2):
                c.weights[:, h, gone[h]] = -1.0
            c.positions[:] = torch.arange(c.positions.shape[-1], dtype=torch.int32, device="cuda")
            bad = {(0, budget // 16)} if where != "below" else set()
            bad |= {(0, 0)} if where != "behind" else set()
            for r, j in bad:
                c.table[r, j] = c.pool.data.shape[0] if entry is None else entry
            left_out, moves = evict(c, budget, 1, 2, lengths, bad, in_place)
            assert left_out == (1 if where == "below" else 2) and moves


@pytest.mark.gpu
def test_a_bad_page_that_no_move_needs_is_not_told():
    c = Case([300, 300], 1, 1, 64, 64)
    c.positions[:] = torch.arange(c.positions.shape[-1], dtype=torch.int32, device="cuda")
    c.weights[0, 0, :64] = 9.0                           # stay where they are
    c.weights[0, 0, 256:] = -9.0                         # go
    for j in (0, 4):
        c.table[0, j] = -1
    left_out, moves = evict(c, 128, 0, 0, [300, 300], {(0, 0), (0, 4)})
    assert not left_out and moves


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("budget", [50, 191])
def test_an_eviction_tells_of_bad_lengths(budget, in_place):
    """Below zero counts as none, above the table's slots as all of them."""
    for bad, n in ((-5, 0), (-2 ** 31, 0), (193, 192), (2 ** 31 - 1, 192)):
        c = Case([192, 100, 192], 2, 2, 64, 64)
        c.lengths[0] = bad
        evict(c, budget, 3, 9, [n, 100, 192], (), in_place, told=True)


@pytest.mark.gpu
def test_rows_longer_than_the_ctas_hold_are_cut_in_place():
    for budget in (230000, 5000):
        c = Case([230001], 1, 1, 64, 256)
        evict(c, budget, 4, 1000, [230001], in_place=True)


# ---- a pool of more than 2^32 bytes ----------------------------------------------------------------------------------

@pytest.mark.gpu
def test_an_append_and_an_eviction_beyond_32_bits_of_bytes():
    """One row whose pages lie up to 5 GB apart."""
    d, bt, hkv, n = 128, 64, 8, 700
    block = hkv * 2 * bt * d * 2
    blocks = (5 << 30) // block
    c = Case([n], hkv, hkv, d, bt, per_row=11, spare=0)
    pool = torch.empty(blocks * block, dtype=torch.uint8, device="cuda")
    at = [(blocks - 1) - j * (blocks // 11) for j in range(11)]
    assert at[0] * block > 1 << 32
    table = torch.tensor([at], dtype=torch.int32, device="cuda")
    view = pool.view(blocks, block)
    view[at] = 0
    cache = binding.make_paged(c.shape, pool, table, c.lengths, c.weights, c.positions)
    k, v = (torch.randn((n, hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    binding.ipkv_paged_append(c.shape, cache, k, v, positions=torch.arange(n, dtype=torch.int32, device="cuda"), row_start=start, status=c.status)

    def here():                                          # the pages, gathered into a small pool
        c.pool.data[c.pages[0].cuda()] = view[at].view(torch.bfloat16).view(11, hkv, 2, bt * d)
        return c.pool.get(c.pages[0], list(range(n)))
    k1, v1 = here()
    assert torch.equal(k1, k) and torch.equal(v1, v) and int(c.status) == 0
    c.weights.uniform_()
    w, budget = c.weights.clone(), 300
    scratch = torch.empty(binding.ipkv_paged_evict_scratch_bytes(c.shape, cache, budget), dtype=torch.uint8, device="cuda")
    binding.ipkv_paged_evict(c.shape, cache, budget, 4, 30, scratch, status=c.status)
    k1, v1 = here()
    assert int(c.status) == 0
    for h in range(hkv):
        src = torch.tensor(ref.kept(w[0, h, :n].tolist(), list(range(n)), budget, 4, 30), device="cuda")
        assert torch.equal(k1[:budget, h], k[src, h]) and torch.equal(v1[:budget, h], v[src, h]) and torch.equal(c.positions[0, h, :budget], src.int())
        assert torch.equal(k1[budget:, h], k[budget:, h]) and torch.equal(v1[budget:, h], v[budget:, h])


# ---- a window over rows that were cut --------------------------------------------------------------------------------

@pytest.mark.gpu
def test_a_window_counts_slots_whatever_their_tokens():
    """As the header says: after an eviction the last slots are not the last tokens."""
    c = Case([600, 90], 4, 2, 64, 32)
    c.positions[:] = torch.arange(c.positions.shape[-1], dtype=torch.int32, device="cuda")
    scratch = torch.empty(binding.ipkv_paged_evict_scratch_bytes(c.shape, c.cache(), 200), dtype=torch.uint8, device="cuda")
    binding.ipkv_paged_evict(c.shape, c.cache(), 200, 0, 50, scratch, status=c.status)
    c.lengths.clamp_(max=200)
    c.n = [200, 90]
    recent = c.positions[0, 0, :200] >= 550              # moved in order, but only into holes: tokens that stayed are among the last slots
    assert recent.sum() == 50 and not recent[150:].all()
    for window, first in ((50, 3), (0, 0)):
        o, lse = c.attend(window, first)
        c.check(o, lse, window, first)
    assert int(c.status) == 0
