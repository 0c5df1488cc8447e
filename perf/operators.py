"""Cases and plain forms of the operators around a decode cache held in 4 bits.

Three operators, reached through ``paper_2609_14507_b200.binding``:

* ``ipkv_norm_rope``      RMS norm of every query / key head and the rotation of its columns by position, in one pass;
                          positions may have several axes (time, height, width), each pair of columns follows one axis;
* ``ipkv_nibble_pack`` /  token-major bf16 K/V into 4-bit blocks (prompts, chunks of prompts, one new token per sequence)
  ``ipkv_nibble_unpack``  and back;
* ``ipkv_nibble_attend``  attention of one decode query per row over runs of such blocks: partial output and natural-log LSE.

The 4-bit format.  A group of values x (K: the 64 columns of one panel of one token and head; V: all columns of one token
and head) is held as codes 0..15, a scale and a zero, both bf16:
  zero = min x,  scale = bf16((max x - min x) / 15),  code = min(round_half_even((x - zero) / scale), 15),
each step in fp32, the code 0 where scale is below 2^-126; a code stands for scale * code + zero.
A block holds ``block`` tokens (a multiple of 64): for each KV head, block / 64 tiles of 64 tokens.  A tile is K codes, K
scales and zeros, V codes, V scales and zeros; ``tiles_of`` and ``from_tiles`` below say where each one lies.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 1e6


# ---- the cases -----------------------------------------------------------------------------------------------------

def listed():
    return [
        # one new token of one sequence, 32 query heads on 4 KV heads: a decode step where only latency counts
        dict(name="norm_rope 1 token", op="norm_rope", tokens=1, q_heads=32, kv_heads=4, dim=128, rot=128, axes=1,
             interleaved=False, norm=True, fused=True),
        # a decode step of a batch of 64, read where the fused projection left it
        dict(name="norm_rope batch 64", op="norm_rope", tokens=64, q_heads=32, kv_heads=8, dim=128, rot=128, axes=1,
             interleaved=False, norm=True, fused=True),
        # a prompt of 32K tokens
        dict(name="norm_rope prompt 32K", op="norm_rope", tokens=32768, q_heads=32, kv_heads=4, dim=128, rot=128, axes=1,
             interleaved=False, norm=True, fused=False),
        # image tokens with positions in time, height and width; adjacent pairs; half of a 64-wide head is rotated
        dict(name="norm_rope 3 axes", op="norm_rope", tokens=4099, q_heads=12, kv_heads=4, dim=64, rot=32, axes=3,
             interleaved=True, norm=False, fused=True),
        # one new token for each of 64 sequences, written and read back
        dict(name="cache 64 tokens", op="cache", rows=64, longest=1, shortest=1, first=1000, kv_heads=8, dim=128, block=64),
        # a prompt of 32K tokens, written and read back
        dict(name="cache prompt 32K", op="cache", rows=1, longest=32768, shortest=32768, first=0, kv_heads=4, dim=128, block=64),
        # chunks of seven prompts that begin and end inside tiles
        dict(name="cache ragged chunks", op="cache", rows=7, longest=2500, shortest=1, first=333, kv_heads=4, dim=64, block=128),
        # one short sequence: latency
        dict(name="attend 1 x 4K", op="attend", rows=1, longest=4097, shortest=4097, q_heads=32, kv_heads=4, dim=128, block=64),
        # a batch of 16 at 32K tokens, groups of 8 query heads
        dict(name="attend 16 x 32K", op="attend", rows=16, longest=32769, shortest=32769, q_heads=32, kv_heads=4, dim=128, block=64),
        # a ragged batch of 64, groups of 4 query heads, an empty sequence among them
        dict(name="attend ragged 64", op="attend", rows=64, longest=24577, shortest=0, q_heads=32, kv_heads=8, dim=128, block=256),
        # one very long sequence, all 16 query heads on one KV head
        dict(name="attend 1 x 1M", op="attend", rows=1, longest=1000003, shortest=1000003, q_heads=16, kv_heads=1, dim=128, block=64),
        # a whole cache step of a small model: one new token per sequence is written, attended with the rest and read back
        dict(name="step 16 x 2K", op="step", rows=16, longest=2048, shortest=1700, q_heads=12, kv_heads=4, dim=64, block=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "cache", "attend", "attend", "step"])
    dim = rng.choice([64, 128])
    q_heads, kv_heads = rng.choice([(32, 4), (32, 8), (16, 1), (12, 4), (8, 8), (40, 1)])
    if op == "norm_rope":
        return dict(op=op, tokens=_log(rng, 1, 20000), q_heads=q_heads, kv_heads=kv_heads, dim=dim, rot=rng.choice([dim, dim // 2]),
                    axes=rng.choice([1, 3]), interleaved=rng.random() < 0.5, norm=rng.random() < 0.7, fused=rng.random() < 0.5)
    block = rng.choice([64, 128, 256])
    if op == "cache":
        rows = _log(rng, 1, 64)
        longest = _log(rng, 1, max(2, 16000 // rows))
        return dict(op=op, rows=rows, longest=longest, shortest=rng.randint(1, longest), first=rng.randint(0, 700), kv_heads=kv_heads,
                    dim=dim, block=block)
    rows = _log(rng, 1, 64)
    longest = _log(rng, 1, max(2, 500000 // (rows * kv_heads)))
    low = 1 if op == "step" else 0
    return dict(op=op, rows=rows, longest=longest, shortest=rng.randint(low, longest), q_heads=q_heads, kv_heads=kv_heads, dim=dim, block=block)


def _lengths(case):
    """Tokens of every row: between shortest and longest, both among them."""
    rng = random.Random("%(rows)d rows of %(shortest)d to %(longest)d" % case)
    n = [rng.randint(case["shortest"], case["longest"]) for _ in range(case["rows"])]
    n[-1] = case["shortest"]
    n[0] = case["longest"]
    return n


def _token_bytes(case):
    """Bytes of one token and KV head in the cache."""
    d = case["dim"]
    return d + 4 * (d // 64) + 4


def work(case):
    d = case["dim"]
    if case["op"] == "norm_rope":
        rows = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": rows * d * 4 + case["tokens"] * case["axes"] * 4 + 4 * d * case["norm"], "flops": rows * d * 7}
    n = _lengths(case)
    if case["op"] == "cache":
        values = sum(n) * case["kv_heads"]
        return {"bytes": values * (8 * d + 2 * _token_bytes(case)), "flops": values * d * 10}
    new = case["rows"] * case["kv_heads"] * (8 * d + 2 * _token_bytes(case)) if case["op"] == "step" else 0    # written, read back
    rows = case["rows"] * case["q_heads"]
    return {"bytes": sum(n) * case["kv_heads"] * _token_bytes(case) + rows * (6 * d + 4) + new, "flops": 4 * sum(n) * case["q_heads"] * d}


# ---- the format ----------------------------------------------------------------------------------------------------

def quantised(x, width):
    """fp32 values [..., D] -> codes uint8 [..., D], scale and zero bf16 [..., D / width]."""
    g = x.unflatten(-1, (-1, width))
    low = g.amin(-1, keepdim=True)
    scale = ((g.amax(-1, keepdim=True) - low) / 15.0).to(torch.bfloat16).float()
    steps = torch.where(scale >= 2.0 ** -126, (g - low) / scale, torch.zeros_like(g))
    codes = torch.round(steps).clamp(0, 15).to(torch.uint8)
    return codes.flatten(-2), scale.squeeze(-1).to(torch.bfloat16), low.squeeze(-1).to(torch.bfloat16)


def values(codes, scale, zero, width, dtype=torch.float32):
    s = scale.to(dtype).repeat_interleave(width, -1)
    return codes.to(dtype) * s + zero.to(dtype).repeat_interleave(width, -1)


def _pair(scale, zero):
    return torch.stack([scale, zero], -1).contiguous().view(torch.uint8)


def tiles_of(kc, ks, kz, vc, vs, vz):
    """Tokens [T, 64, D] (codes) and [T, 64, groups] (scales, zeros) -> tile images, uint8 [T, bytes].

    Nibble j of a 4-byte word is its bits 4j..4j+3.  K codes: token 16u + 8h + g, column 64p + 16t + 8w + j is nibble j of
    word ((((u * panels + p) * 8 + g) * 4 + t) * 2 + h) * 2 + w.  V codes: column 16d + 8h + g, token 32w + 8i + 2t + e is
    nibble i + 4e of word ((((d * 8 + g) * 4 + t) * 2 + h) * 2 + w.  Scale and zero of token 16u + 8h + g: row 16u + 2g + h
    (K: one pair per panel, V: one pair)."""
    T, d = kc.shape[0], kc.shape[2]
    p = d // 64
    k = kc.view(T, 4, 2, 8, p, 4, 2, 4, 2).permute(0, 1, 4, 3, 5, 2, 6, 7, 8).reshape(T, -1, 2)
    v = vc.view(T, 2, 2, 2, 4, 2, d // 16, 2, 8).permute(0, 6, 8, 4, 7, 1, 5, 2, 3).reshape(T, -1, 2)
    km = _pair(ks, kz).view(T, 4, 2, 8, -1).transpose(2, 3).reshape(T, -1)
    vm = _pair(vs, vz).view(T, 4, 2, 8, -1).transpose(2, 3).reshape(T, -1)
    return torch.cat([k[..., 0] | (k[..., 1] << 4), km, v[..., 0] | (v[..., 1] << 4), vm], 1)


def from_tiles(tiles, d):
    """Tile images uint8 [T, bytes] -> values K, V fp32 [T, 64, D]."""
    T, p = tiles.shape[0], d // 64
    k, km, v, vm = tiles.split([32 * d, 256 * p, 32 * d, 256], 1)
    k = torch.stack([k & 15, k >> 4], -1).view(T, 4, p, 8, 4, 2, 2, 4, 2).permute(0, 1, 5, 3, 2, 4, 6, 7, 8).reshape(T, 64, d)
    v = torch.stack([v & 15, v >> 4], -1).view(T, d // 16, 8, 4, 2, 2, 2, 2, 2).permute(0, 5, 7, 8, 3, 6, 1, 4, 2).reshape(T, 64, d)
    km = km.reshape(T, 4, 8, 2, -1).transpose(2, 3).contiguous().view(torch.bfloat16).view(T, 64, p, 2)
    vm = vm.reshape(T, 4, 8, 2, -1).transpose(2, 3).contiguous().view(torch.bfloat16).view(T, 64, 1, 2)
    return values(k, km[..., 0], km[..., 1], 64), values(v, vm[..., 0], vm[..., 1], d)


def _tile_bytes(d):
    return 64 * d + 256 * (d // 64 + 1)


# ---- inputs --------------------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def _keys(gen, n, heads, d):
    """Keys have a few columns that are much larger than the rest."""
    x = _normal(gen, n, heads, d)
    x[..., 5::29] *= 5.0
    return x.to(torch.bfloat16)


def _sections(pairs, axes):
    """Which axis every pair of columns follows: contiguous sections, the later axes a little wider."""
    first = pairs // (axes + 1) if axes > 1 else pairs
    rest = [(pairs - first) // (axes - 1)] * (axes - 1) if axes > 1 else []
    if rest:
        rest[-1] += pairs - first - sum(rest)
    return [first] + rest


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    d = case["dim"]
    if case["op"] == "norm_rope":
        n, hq, hk = case["tokens"], case["q_heads"], case["kv_heads"]
        if case["fused"]:       # views of what one projection wrote: q | k | v of a token side by side
            x = _normal(gen, n, hq + 2 * hk, d).to(torch.bfloat16)
            q, k = x[:, :hq], x[:, hq:hq + hk]
        else:
            q, k = _normal(gen, n, hq, d).to(torch.bfloat16), _normal(gen, n, hk, d).to(torch.bfloat16)
        w = (1.0 + 0.2 * _normal(gen, 2, d)).to(torch.bfloat16) if case["norm"] else None
        if case["axes"] == 1:
            pos = torch.randint(0, 1000000, (1, 1), generator=gen, device=DEV) + torch.arange(n, device=DEV)
        else:                   # a picture: 64 patches a row
            t = torch.arange(n, device=DEV)
            at = int(torch.randint(0, 30000, (1,), generator=gen, device=DEV))
            pos = torch.stack([torch.full_like(t, at), at + t // 64, at + t % 64])
        return dict(case=case, q=q, k=k, wq=w[0] if w is not None else None, wk=w[1] if w is not None else None,
                    positions=pos.to(torch.int32), sections=_sections(case["rot"] // 2, case["axes"]),
                    q_out=torch.empty((n, hq, d), dtype=torch.bfloat16, device=DEV),
                    k_out=torch.empty((n, hk, d), dtype=torch.bfloat16, device=DEV))
    n, h, bt = _lengths(case), case["kv_heads"], case["block"]
    first = case.get("first", 0)
    blocks = [-(-(first + x) // bt) for x in n]                         # blocks of every row, one row behind the other
    start = np.concatenate([[0], np.cumsum(blocks)])
    total = int(start[-1])
    tb = _tile_bytes(d)
    block_bytes = h * (bt // 64) * tb
    if case["op"] == "cache":
        pool = torch.zeros((max(1, total), h, bt // 64, tb), dtype=torch.uint8, device=DEV)
        address = pool.data_ptr() + start[:-1] * block_bytes
        spans = np.stack([address, np.full(len(n), first), np.asarray(n)], 1).astype(np.int64)
        k, v = _keys(gen, sum(n), h, d), _normal(gen, sum(n), h, d).to(torch.bfloat16)
        return dict(case=case, pool=pool, spans=spans, k=k, v=v, k_out=torch.empty_like(k), v_out=torch.empty_like(v))
    tokens = max(64, total * bt)
    k, v = _keys(gen, tokens, h, d), _normal(gen, tokens, h, d).to(torch.bfloat16)
    kq, vq = quantised(k.float(), 64), quantised(v.float(), d)
    by_tile = [x.view(tokens // 64, 64, h, -1).transpose(1, 2).reshape(tokens // 64 * h, 64, -1) for x in (*kq, *vq)]
    pool = tiles_of(*by_tile).view(-1, h, tb)                           # [tile][head], then blocks: [head][tile]
    if total:
        pool = pool.view(total, bt // 64, h, tb).transpose(1, 2).contiguous()
    rows, hq = case["rows"], case["q_heads"]
    runs = np.stack([pool.data_ptr() + start[:-1] * block_bytes, np.asarray(n)], 1).astype(np.int64)
    state = dict(case=case, pool=pool, start=start, lengths=n, runs=runs, row_start=np.arange(rows + 1, dtype=np.int32),
                 q=_normal(gen, rows, hq, d).to(torch.bfloat16),
                 scratch=torch.empty(64 << 20, dtype=torch.uint8, device=DEV),
                 o=torch.empty((rows, hq, d), device=DEV), lse=torch.empty((rows, hq), device=DEV))
    if case["op"] == "step":
        state["k_new"], state["v_new"] = _keys(gen, rows, h, d), _normal(gen, rows, h, d).to(torch.bfloat16)
        state["spans"] = np.stack([state["runs"][:, 0], np.asarray(n) - 1, np.ones(rows)], 1).astype(np.int64)
        state["k_out"], state["v_out"] = torch.empty_like(state["k_new"]), torch.empty_like(state["v_new"])
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------

def _scale(case):
    return case["dim"] ** -0.5


def run(state):
    case = state["case"]
    return _own(state, case) if own else _plain(state, case)


def _own(state, case):
    from paper_2609_14507_b200 import binding as b
    if case["op"] == "norm_rope":
        rope = b.make_rope(case["dim"], case["rot"], theta=THETA, sections=state["sections"], interleaved=case["interleaved"], eps=EPS)
        b.ipkv_norm_rope(rope, [(state["q"], state["wq"], state["q_out"]), (state["k"], state["wk"], state["k_out"])], state["positions"])
        return {"q": state["q_out"], "k": state["k_out"]}
    shape = b.make_shape(b.GQA, case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["dim"], case["dim"], case["block"], _scale(case))
    if case["op"] == "cache":
        b.ipkv_nibble_pack(shape, state["spans"], state["k"], state["v"])
        b.ipkv_nibble_unpack(shape, state["spans"], state["k_out"], state["v_out"])
        return {"k": state["k_out"], "v": state["v_out"]}
    if case["op"] == "step":
        b.ipkv_nibble_pack(shape, state["spans"], state["k_new"], state["v_new"])
    b.ipkv_nibble_attend(shape, state["runs"], state["row_start"], state["q"], state["scratch"], state["o"], state["lse"])
    out = {"o": state["o"], "lse": state["lse"]}
    if case["op"] == "step":            # what the cache holds now of the new tokens
        b.ipkv_nibble_unpack(shape, state["spans"], state["k_out"], state["v_out"])
        out.update(k=state["k_out"], v=state["v_out"])
    return out


def _plain_rope(x, w, cos, sin, case):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    r, rest = x[..., :case["rot"]], x[..., case["rot"]:]
    if case["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r.chunk(2, -1)
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, rest], -1).to(torch.bfloat16)


def _plain(state, case):
    d = case["dim"]
    if case["op"] == "norm_rope":
        # angles in 64 bits: a far position times a frequency, taken modulo a turn
        pairs = case["rot"] // 2
        frequency = THETA ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / pairs)
        sizes = torch.tensor(state["sections"], device=DEV)
        axis = torch.repeat_interleave(torch.arange(len(state["sections"]), device=DEV), sizes, output_size=pairs)
        angle = state["positions"].double().t()[:, axis] * frequency
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        return {"q": _plain_rope(state["q"], state["wq"], cos, sin, case), "k": _plain_rope(state["k"], state["wk"], cos, sin, case)}
    if case["op"] == "cache":
        k = values(*quantised(state["k"].float(), 64), 64).to(torch.bfloat16)
        v = values(*quantised(state["v"].float(), d), d).to(torch.bfloat16)
        return {"k": k, "v": v}
    n, h, bt, rows, hq = state["lengths"], case["kv_heads"], case["block"], case["rows"], case["q_heads"]
    most = -(-max(max(n), 1) // bt)                                     # blocks of the longest row: the others are padded
    length = torch.tensor(n, device=DEV)
    at = torch.as_tensor(state["start"][:-1], device=DEV)[:, None] + torch.arange(most, device=DEV)
    block = state["pool"].view(-1, h, bt // 64, state["pool"].shape[-1])[at.clamp(max=state["pool"].numel() // (h * (bt // 64) * state["pool"].shape[-1]) - 1)]
    tiles = block.transpose(1, 2).flatten(2, 3).flatten(0, 2)           # [row][head][tile]
    k, v = (x.view(rows, h, most * bt, d) for x in from_tiles(tiles, d))
    if case["op"] == "step":
        last = (length - 1).view(-1, 1, 1, 1).expand(-1, h, 1, d)
        k_new, v_new = values(*quantised(state["k_new"].float(), 64), 64), values(*quantised(state["v_new"].float(), d), d)
        k, v = k.scatter(2, last, k_new[:, :, None]), v.scatter(2, last, v_new[:, :, None])
    q = state["q"].float().view(rows, h, hq // h, d)
    s = torch.matmul(q, k.transpose(2, 3)) * _scale(case)
    s = s.masked_fill(torch.arange(most * bt, device=DEV) >= length.view(-1, 1, 1, 1), float("-inf"))
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top.isinf(), torch.zeros_like(top), top))
    z = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(z > 0, z, torch.ones_like(z))
    out = {"o": o.reshape(rows, hq, d), "lse": (top + torch.log(z)).reshape(rows, hq)}
    if case["op"] == "step":
        out.update(k=k_new.to(torch.bfloat16), v=v_new.to(torch.bfloat16))
    return out


# ---- the definition, in 64 bits ------------------------------------------------------------------------------------

def _exact_group(x, width):
    """Token-major bf16 [n, heads, D] -> the values that its codes stand for, fp64."""
    g = x.double().reshape(*x.shape[:-1], -1, width)
    low, high = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    scale = ((high - low) / 15).to(torch.bfloat16).double()
    steps = torch.where(scale >= 2.0 ** -126, (g - low) / scale, 0.0).round().clamp(0, 15)
    return (steps * scale + low).reshape(x.shape)


def exact(case, seed):
    state = prepare(case, seed)
    d = case["dim"]
    if case["op"] == "norm_rope":
        out = {}
        pairs = case["rot"] // 2
        axis = [a for a, size in enumerate(state["sections"]) for _ in range(size)]
        angle = torch.stack([state["positions"][a].double() * THETA ** (-i / pairs) for i, a in enumerate(axis)], 1)
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        for name, w in (("q", state["wq"]), ("k", state["wk"])):
            x = state[name].double()
            if w is not None:
                x = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w.double()
            if case["interleaved"]:
                first, second = range(0, case["rot"], 2), range(1, case["rot"], 2)
            else:
                first, second = range(pairs), range(pairs, 2 * pairs)
            first, second = torch.tensor(first, device=DEV), torch.tensor(second, device=DEV)
            z = torch.complex(x[..., first], x[..., second]) * turn
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    if case["op"] == "cache":
        return {"k": _exact_group(state["k"], 64), "v": _exact_group(state["v"], d)}
    # the same draws as prepare's, never laid out in blocks
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    n, h, hq = state["lengths"], case["kv_heads"], case["q_heads"]
    tokens = max(64, int(state["start"][-1]) * case["block"])
    k, v = _keys(gen, tokens, h, d), _normal(gen, tokens, h, d).to(torch.bfloat16)
    o, lse = torch.zeros((case["rows"], hq, d), device=DEV, dtype=torch.float64), torch.zeros((case["rows"], hq), device=DEV, dtype=torch.float64)
    lse.fill_(float("-inf"))
    for r, length in enumerate(n):
        if not length:
            continue
        at = int(state["start"][r]) * case["block"]
        kr, vr = k[at:at + length].clone(), v[at:at + length].clone()
        if case["op"] == "step":
            kr[length - 1], vr[length - 1] = state["k_new"][r], state["v_new"][r]
        kr, vr = _exact_group(kr, 64), _exact_group(vr, d)
        for head in range(hq):
            g = head // (hq // h)
            s = kr[:, g] @ state["q"][r, head].double() * _scale(case)
            lse[r, head] = torch.logsumexp(s, 0)
            o[r, head] = torch.softmax(s, 0) @ vr[:, g]
    out = {"o": o, "lse": lse}
    if case["op"] == "step":
        out.update(k=_exact_group(state["k_new"], 64), v=_exact_group(state["v_new"], d))
    return out
