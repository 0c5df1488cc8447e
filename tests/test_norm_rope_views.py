"""Which views of one buffer a head norm and rotation takes: all that share no byte, and no others; and what it writes into them."""
import random

import pytest

from paper_2609_14507_b200 import binding
from paper_2609_14507_b200.binding import Heads
from tests.test_norm_rope import reference

torch = pytest.importorskip("torch")
C = binding.C
EINVAL, ECUDA = 1, 5
BASE = 1 << 20          # an aligned address that nothing reads: without a GPU no call gets further than the launch


def rc(rope, parts, n):
    return binding.lib().ipkv_norm_rope(C.byref(rope), n, (Heads * len(parts))(*parts), len(parts), BASE, None)


def elements(at, n, heads, ts, hs, d):
    """The 16-byte chunks that a view covers."""
    return {(at + t * ts + h * hs) // 8 + c for t in range(n) for h in range(heads) for c in range(d // 8)}


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")
@pytest.mark.parametrize("n", [1, 2, 5])
def test_heads_between_one_another_are_taken_in_place(n):
    """q | k | v of every head side by side, and two query heads and a key head of every group."""
    d = 128
    rope = binding.make_rope(d)
    for members, turned in ((3, 2), (4, 3)):
        heads = 4
        row = heads * members * d
        parts = [Heads(BASE + 2 * i * d, BASE + 2 * i * d, None, heads, row, members * d, row, members * d) for i in range(turned)]
        assert rc(rope, parts, n) == ECUDA                               # refused for nothing but the missing GPU
        parts[1] = Heads(BASE + 2 * d - 16, BASE + 2 * d - 16, None, heads, row, members * d, row, members * d)
        assert rc(rope, parts, n) == EINVAL                              # eight columns shared


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")
def test_no_views_that_share_bytes_are_taken():
    """Two parts in place with the same strides, at random places of a small buffer: what is taken shares nothing, and with strides as the
    layouts of a buffer have them, what shares nothing is taken."""
    d, rng, taken = 64, random.Random(5), 0
    rope = binding.make_rope(d)
    for _ in range(4000):
        n, ha, hb = rng.choice([1, 2, 3]), rng.choice([1, 2, 3]), rng.choice([1, 2, 3])
        ts, hs = rng.choice([64, 72, 128, 192, 256, 320, 576, 768]), rng.choice([64, 72, 128, 136, 192, 256])
        most = max(ha, hb)
        if n > 1 and ts < (most - 1) * hs + d and hs < (n - 1) * ts + d:
            continue                                                     # heads outside tokens or tokens outside heads
        at = 8 * rng.randint(0, 90)
        parts = [Heads(BASE + 2 * x, BASE + 2 * x, None, h, ts, hs, ts, hs) for x, h in ((0, ha), (at, hb))]
        shared = elements(0, n, ha, ts, hs, d) & elements(at, n, hb, ts, hs, d)
        got = rc(rope, parts, n)
        assert got == (EINVAL if shared else ECUDA), (n, ha, hb, ts, hs, at)
        taken += not shared
    assert taken > 500


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")
@pytest.mark.parametrize("ts,n", [(1 << 40, 1 << 18), (1 << 48, 1 << 20), (1 << 48, (1 << 31) - 1)])
def test_views_whose_extent_passes_63_bits(ts, n):
    d = 128
    rope = binding.make_rope(d)
    part = lambda at, heads=3: Heads(BASE + at, BASE + at, None, heads, ts, 2 * d, ts, 2 * d)
    assert rc(rope, [part(0), part(2 * d)], n) == ECUDA
    assert rc(rope, [part(0), part(2 * d - 16)], n) == EINVAL
    assert rc(rope, [part(0), part(2 * ts * 5 + 2 * d)], n) == ECUDA     # a token further on, between the heads again
    assert rc(rope, [part(0), part(2 * ts * 5 + 2 * d + 16)], n) == EINVAL
    assert rc(rope, [part(0), part(2 * ts * 5 + 4 * 3 * d)], n) == ECUDA     # behind the other's heads


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 3, 300])
@pytest.mark.parametrize("inter", [False, True])
def test_heads_between_one_another(n, inter):
    d, h = 128, 5
    g = torch.Generator().manual_seed(n)
    x = torch.randn((n, h, 3, d), generator=g).bfloat16()
    pos = torch.randint(0, 1 << 20, (1, n), generator=g)
    ws = [(1 + 0.3 * torch.randn(d, generator=g)).bfloat16() for _ in range(2)]
    y = x.cuda()
    rope = binding.make_rope(d, theta=10000.0, interleaved=inter, eps=1e-5)
    binding.ipkv_norm_rope(rope, [(y[:, :, 0], ws[0].cuda(), None), (y[:, :, 1], ws[1].cuda(), None)], pos.to(torch.int32).cuda())
    got = y.cpu()
    assert torch.equal(got[:, :, 2], x[:, :, 2])
    for i in range(2):
        want = reference(x[:, :, i], ws[i], pos, dict(rot_dim=d, theta=10000.0, interleaved=inter), 1e-5)
        # one rounding to bf16 and fp32 work below 2^-18 of a head's largest value, as in test_norm_rope.py
        bound = want.abs() * 2.0 ** -8 + want.abs().amax(-1, keepdim=True) * 2 ** 0.5 * 2.0 ** -18
        assert bool(((got[:, :, i].double() - want).abs() <= bound).all())
