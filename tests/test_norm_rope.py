"""Head norm and rotation: what the call refuses (no GPU), and its outputs against the formula in 64 bits."""
import numpy as np
import pytest

from paper_2609_14507_b200 import binding
from paper_2609_14507_b200.binding import Heads, IpkvError

torch = pytest.importorskip("torch")
C = binding.C
EINVAL = 1


# ---- refusals: decided on the host, before anything touches a GPU --------------------------------------------------

BASE = 1 << 20          # an aligned address that nothing reads: the calls below are refused first


def call(rope, parts, n_tokens=4, positions=BASE, n_parts=None):
    arr = (Heads * max(1, len(parts)))(*parts)
    return binding.lib().ipkv_norm_rope(C.byref(rope), n_tokens, arr, len(parts) if n_parts is None else n_parts, positions, None)


def heads(src=BASE, dst=2 * BASE, w=None, n=4, ts=512, hs=128, ots=512, ohs=128):
    return Heads(src, dst, w, n, ts, hs, ots, ohs)


@pytest.mark.parametrize("kw", [
    dict(dim=96), dict(dim=0), dict(dim=512), dict(dim=128, rot_dim=24), dict(dim=128, rot_dim=144), dict(dim=128, rot_dim=-16),
    dict(dim=128, theta=0.0), dict(dim=128, theta=float("nan")), dict(dim=128, theta=float("inf")), dict(dim=128, eps=-1.0),
    dict(dim=128, eps=float("nan")), dict(dim=128, inv_freq=[float("nan")] * 64), dict(dim=128, inv_freq=[1e400] * 64)])
def test_bad_rotations_are_refused(kw):
    dim = kw.pop("dim")
    rot = kw.pop("rot_dim", dim)
    rope = binding.make_rope(dim, rot, **kw)
    assert call(rope, [heads()]) == EINVAL


def test_bad_axes_are_refused():
    rope = binding.make_rope(128, sections=[16, 24, 24])
    rope.n_axes = 2                                      # a pair follows an axis that is not there
    assert call(rope, [heads()]) == EINVAL
    rope.n_axes = 5
    assert call(rope, [heads()]) == EINVAL
    with pytest.raises(ValueError):
        binding.make_rope(128, sections=[16, 24])        # pairs without an axis
    with pytest.raises(ValueError):
        binding.make_rope(128, sections=[64], pair_axis=[0] * 64)
    with pytest.raises(ValueError):
        binding.make_rope(128, inv_freq=[1.0] * 63)


@pytest.mark.parametrize("part", [
    dict(n=0), dict(src=None), dict(dst=None), dict(src=BASE + 2), dict(dst=BASE * 2 + 8), dict(w=BASE + 4), dict(ts=-512), dict(ts=516),
    dict(hs=4), dict(ohs=64),                            # heads of the output on top of one another
    dict(ots=256),                                       # tokens of the output on top of one another
    dict(ots=0),
    dict(dst=BASE, ots=1024),                            # in place with other strides
    dict(dst=BASE + 256),                                # the output overlaps the input
    dict(src=BASE, dst=BASE + 768, ts=1024, ots=1024),   # ... inside every token's row
])
def test_bad_heads_are_refused(part):
    assert call(binding.make_rope(128), [heads(**part)]) == EINVAL


def test_outputs_that_collide_between_parts_are_refused():
    rope = binding.make_rope(128)
    a = heads()
    assert call(rope, [a, heads(src=3 * BASE, dst=2 * BASE + 256)]) == EINVAL           # two outputs
    assert call(rope, [a, heads(src=2 * BASE, dst=4 * BASE)]) == EINVAL                 # an output and the other's input
    assert call(rope, [a], n_parts=0) == EINVAL and call(rope, [a] * 5) == EINVAL
    assert call(rope, [a], positions=None) == EINVAL and call(rope, [a], positions=BASE + 2) == EINVAL
    assert call(rope, [a], n_tokens=-1) == EINVAL and call(rope, [a], n_tokens=1 << 31) == EINVAL
    assert call(rope, [a], n_tokens=0) == 0                                             # nothing to do


def test_strided_views_of_one_buffer_are_not_refused():
    """q | k | v of a token side by side, rotated in place or into the next buffer: refused for nothing but the missing GPU."""
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    rope = binding.make_rope(128)
    row = 8 * 128
    q = heads(src=BASE, dst=BASE, n=4, ts=row, ots=row)
    k = heads(src=BASE + 4 * 256, dst=BASE + 4 * 256, n=2, ts=row, ots=row)
    assert call(rope, [q, k]) == 5                       # IPKV_ECUDA
    head_major = heads(src=BASE, dst=2 * BASE, ts=128, hs=4 * 128, ots=128, ohs=4 * 128)
    assert call(rope, [head_major]) == 5


def test_the_binding_refuses_other_types_and_shapes():
    rope = binding.make_rope(64)
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    pos = torch.zeros((1, 3), dtype=torch.int32)
    for parts, p in [([(x.float(), None, None)], pos), ([(x[:, :, ::2], None, None)], pos), ([(x, None, x[:2])], pos),
                     ([(x, torch.zeros(64), None)], pos), ([(x, torch.zeros(32, dtype=torch.bfloat16), None)], pos),
                     ([(x, None, None)], pos.long()), ([(x, None, None)], pos[:, :2]), ([(x, None, None), (x[:2], None, None)], pos)]:
        with pytest.raises(ValueError):
            binding.ipkv_norm_rope(rope, parts, p)


# ---- outputs ---------------------------------------------------------------------------------------------------------

def reference(x, w, positions, rope_args, eps):
    """The definition in 64 bits: x [n, H, D] bf16, positions [axes, n]."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
    rot, pairs = rope_args["rot_dim"], rope_args["rot_dim"] // 2
    if not rot:
        return y
    freq = rope_args.get("inv_freq") or [rope_args["theta"] ** (-2.0 * i / rot) for i in range(pairs)]
    axis = rope_args.get("pair_axis") or [0] * pairs
    out = y.clone()
    for i in range(pairs):
        t = positions[axis[i]].double() * freq[i]
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        a, b = (2 * i, 2 * i + 1) if rope_args["interleaved"] else (i, i + pairs)
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def check(got, want, y_scale):
    """One rounding to bf16 (2^-8 relative) behind fp32 work: squares and their sum, rsqrt, two products, two products and a sum
    (about 20 roundings of 2^-24) and an angle off by 2 pi 2^-24 (times a column of the pair), together below 2^-18 of the head's largest value."""
    err = (got.double() - want).abs()
    bound = want.abs() * 2.0 ** -8 + y_scale * 2.0 ** -18
    assert bool((err <= bound).all()), float((err / bound).max())


CASES = [
    # tokens, heads of the parts, dim, rot, sections, interleaved, norm
    (1, (32, 4), 128, 128, None, False, True),
    (1, (1,), 64, 64, None, True, False),
    (3, (32, 8), 128, 64, None, False, True),
    (5, (3, 1, 2), 64, 32, [4, 6, 6], True, True),
    (7, (5,), 256, 256, [32, 48, 48], False, True),
    (37, (16, 1), 128, 128, [16, 24, 24], False, False),
    (64, (12, 4), 64, 64, [8, 24], True, True),
    (130, (9, 7), 256, 16, None, False, True),
    (33, (8,), 128, 0, None, False, True),
    (20000, (2, 1), 64, 48, None, True, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n,hs,d,rot,sections,inter,norm", CASES)
@pytest.mark.parametrize("layout", ["dense", "fused", "in place", "head-major"])
def test_matches_the_formula(n, hs, d, rot, sections, inter, norm, layout):
    g = torch.Generator().manual_seed(n * 1000 + d + rot)
    axes = len(sections) if sections else 1
    pos = torch.randint(-5, 2 ** 31 - 1, (axes, n), generator=g, dtype=torch.int64)
    pos[:, 0] = 0
    args = dict(rot_dim=rot, theta=10000.0, interleaved=inter, pair_axis=[a for a, k in enumerate(sections) for _ in range(k)] if sections else None)
    rope = binding.make_rope(d, rot, theta=10000.0, sections=sections, interleaved=inter, eps=1e-5)
    gap = 16
    if layout == "head-major":
        whole = [torch.randn((h, n, d), generator=g).bfloat16().cuda() for h in hs]
        xs = [x.transpose(0, 1) for x in whole]
        outs = [torch.full_like(x, 7.0).transpose(0, 1) for x in whole]
    elif layout == "dense":
        xs = [torch.randn((n, h, d), generator=g).bfloat16().cuda() for h in hs]
        outs = [torch.full_like(x, 7.0) for x in xs]
    else:
        buf = torch.randn((n, sum(hs) * d + gap), generator=g).bfloat16().cuda()
        before = buf.clone()
        xs, at = [], 0
        for h in hs:
            xs.append(buf[:, at:at + h * d].unflatten(1, (h, d)))
            at += h * d
        outs = [None] * len(hs) if layout == "in place" else [torch.full((n, h, d), 7.0, dtype=torch.bfloat16, device="cuda") for h in hs]
    ws = [(1 + 0.3 * torch.randn(d, generator=g)).bfloat16().cuda() if norm and i != 2 else None for i in range(len(hs))]
    want = [reference(x.cpu(), None if w is None else w.cpu(), pos, args, 1e-5) for x, w in zip(xs, ws)]
    binding.ipkv_norm_rope(rope, list(zip(xs, ws, outs)), pos.to(torch.int32).cuda() if rot else None)
    torch.cuda.synchronize()
    for x, out, y in zip(xs, outs, want):
        got = (x if out is None else out).cpu()
        check(got, y, y.abs().amax(-1, keepdim=True) * 2 ** 0.5)
        if rot < d and not norm:
            assert torch.equal(got[..., rot:], x.cpu()[..., rot:])
    if layout in ("fused", "in place"):
        assert torch.equal(buf[:, sum(hs) * d:], before[:, sum(hs) * d:])                # the columns behind the heads stay
        if layout == "fused":
            assert torch.equal(buf, before)


@pytest.mark.gpu
def test_frequencies_given_by_the_caller_zero_rows_and_large_values():
    d, n = 128, 6
    freq = [1.0 / (3.0 + 2.5 * i) for i in range(32)]
    rope = binding.make_rope(d, 64, inv_freq=freq, eps=1e-6)
    x = torch.randn((n, 3, d)).bfloat16()
    x[1] = 0                                             # a head of zeros stays one: rsqrt(eps) times nothing
    x[2] *= 1e15                                         # squares near the top of fp32
    x[3] *= 1e-20                                        # squares below eps
    w = torch.randn(d).bfloat16()
    pos = torch.tensor([0, 1, 99, 1 << 20, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32)
    want = reference(x, w, pos[None], dict(rot_dim=64, interleaved=False, inv_freq=freq), 1e-6)
    out = torch.empty((n, 3, d), dtype=torch.bfloat16, device="cuda")
    binding.ipkv_norm_rope(rope, [(x.cuda(), w.cuda(), out)], pos.cuda())
    check(out.cpu(), want, want.abs().amax(-1, keepdim=True) * 2 ** 0.5)
    assert torch.equal(out[1].cpu(), torch.zeros((3, d), dtype=torch.bfloat16))


@pytest.mark.gpu
def test_replays_from_a_graph_and_runs_on_another_stream():
    d, n = 128, 3
    rope = binding.make_rope(d, sections=[16, 24, 24])
    x = torch.randn((n, 4, d)).bfloat16().cuda()
    pos = torch.randint(0, 1000, (3, n), dtype=torch.int32).cuda()
    out, again = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        binding.ipkv_norm_rope(rope, [(x, None, out)], pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.ipkv_norm_rope(rope, [(x, None, again)], pos)
    del rope
    for _ in range(2):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, again)
    x.mul_(2)                                            # the replay reads what is there now
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal((out.float() * 2).bfloat16(), again)


@pytest.mark.gpu
def test_one_token_of_more_heads_than_32_bits_can_divide():
    """The steps of a token are divided among warps: four parts of 2^20 heads of 256, the most that a call takes."""
    d, heads = 256, 1 << 20
    x = torch.randn((1, 1000, d), device="cuda").bfloat16()
    x = x.repeat(1, heads // 1000 + 1, 1)[:, :heads].contiguous()
    parts = [x.clone() for _ in range(4)]
    pos = torch.tensor([[7]], dtype=torch.int32, device="cuda")
    rope = binding.make_rope(d, eps=1e-6)
    few = torch.empty((1, 1000, d), dtype=torch.bfloat16, device="cuda")
    binding.ipkv_norm_rope(rope, [(x[:, :1000], None, few)], pos)
    want = few.repeat(1, heads // 1000 + 1, 1)[:, :heads]
    binding.ipkv_norm_rope(rope, [(p, None, None) for p in parts], pos)
    for p in parts:
        assert torch.equal(p, want)
