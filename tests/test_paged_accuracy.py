"""How exact the paged attention is: the norm of its error per head, which tells three bf16 pieces of a softmax weight from two (a bound of every
rounding's worst case does not)."""
import math

import pytest

from paper_2609_14507_b200 import binding
from tests import paged_ref as ref
from tests.test_paged import Case

torch = pytest.importorskip("torch")

# Of random queries, keys and values, q, k, v ~ N(0, 1) and a scale of dim^-1/2, a head's output is a sum of many tokens' weights times values whose
# errors are independent, so that the norm of its error is the weights' rms error times its own norm, and the steps' add by their squares.  In
# steps of 2^-24: a score, of order 1 to 4, has dim / 16 sums cut at 2^-23 of their largest term and two roundings, 2 to 4 in all; a weight 2 for 2^x and
# 0.3 for three pieces; the second product's three to six sums some 3; joins and the division 1.  That is 4 to 6; the arithmetic played
# below gives 1 to 5.6 (without the 2 of 2^x).  Two pieces leave up to 128, 15 to 56 as played.  Ten lies between.
#
# The cuts are a share of the sums that they cut: a score's error grows with the score.  What counts is its rms under the squares of the
# weights (a token's share of the squared error).  Of scores from N(0, 1) these weigh e^(2 s): a normal distribution of mean 2, rms 5^(1/2), which the ten
# is for.  A head that one token of a score of 5 or 6 dominates has so much more.
BOUND = 10 * 2.0 ** -24


def bound_of(scores, p):
    """Of heads with these scores and softmax weights [heads, tokens]."""
    rms = ((p * scores).square().sum(-1) / p.square().sum(-1)).sqrt()
    return BOUND * (rms / 5 ** 0.5).clamp(min=1)


def bf(x):
    return x.float().to(torch.bfloat16).double()


def f32(x):
    return x.float().double()


def mma(acc, terms):
    """acc + sum(terms, -1) as the tensor cores add: all cut towards zero at 2^-23 of the largest."""
    big = torch.maximum(terms.abs().amax(-1), acc.abs())
    ulp = torch.exp2(torch.floor(torch.log2(big.clamp(min=1e-300))) - 23)

    def cut(x, u):
        return torch.trunc(x / u) * u
    return f32(cut(cut(terms, ulp[..., None]).sum(-1) + cut(acc, ulp), ulp))


def played(q, k, v, scale, pieces, warps=4):
    """The attention's arithmetic for one KV head, with softmax weights in so many pieces."""
    (hq, d), n = q.shape, k.shape[0]
    unit = 4096 // d
    s = torch.zeros((hq, n), dtype=torch.float64)
    for c in range(0, d, 16):
        s = mma(s, q[:, None, c:c + 16].double() * k[None, :, c:c + 16].double())
    s = f32(s * f32(torch.tensor(scale / math.log(2.0))))
    states = []
    for w in range(warps):
        m = torch.full((hq,), -math.inf, dtype=torch.float64)
        z, o = torch.zeros(hq, dtype=torch.float64), torch.zeros((hq, d), dtype=torch.float64)
        for u in range(w * unit, n, warps * unit):
            x = s[:, u:u + unit]
            top = torch.maximum(m, x.amax(-1))
            a, p = f32(torch.exp2(f32(m - top))), f32(torch.exp2(f32(x - top[:, None])))
            z, left, parts = f32(z * a + f32(p.sum(-1))), p, []
            for _ in range(pieces):
                parts.append(bf(left))
                left = f32(left - parts[-1])
            t = torch.zeros((hq, d), dtype=torch.float64)
            for piece in reversed(parts):
                for c in range(0, x.shape[1], 16):
                    t = mma(t, piece[:, None, c:c + 16] * v[u + c:u + c + 16][:x.shape[1] - c].double().t()[None])
            o, m = f32(o * a[:, None] + t), top
        states.append((m, z, o))
    top = torch.stack([x[0] for x in states]).amax(0)
    f = [f32(torch.exp2(f32(x[0] - top))) for x in states]
    return f32(sum(a[:, None] * x[2] for a, x in zip(f, states)) / sum(a * x[1] for a, x in zip(f, states))[:, None])


@pytest.mark.parametrize("d,n", [(64, 500), (128, 500), (128, 37), (64, 1500)])
def test_the_bound_tells_three_pieces_from_two(d, n):
    for seed in range(2):
        gen = torch.Generator().manual_seed(seed)
        q, k, v = (torch.randn(s, generator=gen).to(torch.bfloat16) for s in ((8, d), (n, d), (n, d)))
        exact = torch.softmax(q.double() @ k.double().t() * d ** -0.5, 1) @ v.double()
        off = {pieces: (played(q, k, v, d ** -0.5, pieces) - exact).norm(dim=1) / exact.norm(dim=1) for pieces in (1, 2, 3)}
        assert off[3].max() < 0.7 * BOUND and off[2].min() > 1.4 * BOUND and off[1].min() > 100 * BOUND


def test_the_bound_of_heads_that_one_token_dominates():
    """Tokens that lean on a head's query, with scores up to 7, among 64 heads."""
    d, n = 128, 300
    for seed in range(3):
        gen = torch.Generator().manual_seed(seed)
        q, k, v = (torch.randn(s, generator=gen).to(torch.bfloat16) for s in ((64, d), (n, d), (n, d)))
        k[:24:3] = (k[:24:3].float() + 0.35 * q[:8].float()).to(torch.bfloat16)
        s = q.double() @ k.double().t() * d ** -0.5
        p = torch.softmax(s, 1)
        exact = p @ v.double()
        off = {pieces: (played(q, k, v, d ** -0.5, pieces) - exact).norm(dim=1) / exact.norm(dim=1) / bound_of(s, p) for pieces in (2, 3)}
        assert off[3].max() < 0.85 and off[2].median() > 2 and bound_of(s, p).max() > 2 * BOUND


PATHS = {"cluster": [500, 37, 300], "large cluster": [3000], "shares": [20000, 777], "chunks": [3000] * 200, "window": [7000, 600]}


@pytest.mark.gpu
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d,bt", [(64, 16), (128, 64)])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (3, 3), (8, 1), (14, 2), (16, 1), (24, 1), (40, 1), (64, 1)])
def test_the_norm_of_the_error(hq, hkv, d, bt, path):
    if path == "chunks" and hq > 16:
        lengths = PATHS[path][:120]                      # several head groups, or warps that share a unit
    else:
        lengths = PATHS[path]
    window, first = (450, 5) if path == "window" else (0, 0)
    c = Case(lengths, hq, hkv, d, bt)
    cache = c.cache(weights=False)                       # weights from zero: with some there the sum's rounding would hide the addend's
    out = torch.zeros_like(c.weights)
    o, lse = c.attend(window, first, out, cache=cache)
    o2, lse2 = c.attend(window, first, cache=cache)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and int(c.status) == 0
    for r in range(len(lengths)) if len(lengths) < 10 else (0, 1, 57, len(lengths) - 1):
        seen = ref.visible(lengths[r], window, first)
        eo, el, ep, *_ = ref.attend(c.q[r], *c.pool.get(c.pages[r], seen), c.scale)
        off = (o[r].double() - eo).norm(dim=1) / eo.norm(dim=1)
        bound = bound_of(torch.log(ep) + el[:, None], ep)                # (a score is its weight's logarithm and the log-sum-exp)
        assert (off <= bound).all(), (r, float((off / bound).max()))
        # the log-sum-exp: an average of the scores' errors, and its own rounding (it is below 16)
        assert (lse[r].double() - el).abs().max() <= BOUND + 16 * 2.0 ** -24, r
        want = ep.view(hkv, hq // hkv, -1).sum(1)
        got = out[r][:, seen].double()
        off = (got - want).norm(dim=1) / want.norm(dim=1)
        assert (off <= bound.view(hkv, -1).amax(1)).all(), (r, float((off / BOUND).max()))
