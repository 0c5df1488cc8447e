"""Cases and plain forms of the operators around a paged decode cache of bounded length.

Three operators, reached through ``paper_2609_14507_b200.binding``; pages, page table, lengths and what a slot carries are on the device:

* ``ipkv_paged_append``   token-major bf16 K/V into the pages of every row (one new token per row, or chunks of prompts), with the
                          tokens' positions, and weights that start from zero;
* ``ipkv_paged_attend``   attention of one query per row over its pages: all tokens, or a window of the last ones and a few first
                          ones; partial output and natural-log LSE, and the attention that every token got, added to its weight;
* ``ipkv_paged_evict``    down to a budget of slots per row and KV head: the first and the most recent tokens stay, of the others those
                          with the largest weights.  A kept token behind the budget moves to the slot of an evicted one before it
                          (the i-th to the i-th); nothing else moves.

A page holds ``block`` tokens: for every KV head a K plane and a V plane, a plane is dim / 64 panels of ``block`` rows of 128 bytes,
and the 16-byte chunk c of a panel's row t lies at c ^ (t & 7).
"""
import math
import random

import torch

own = False

DEV = "cuda"


# ---- the cases -----------------------------------------------------------------------------------------------------

def listed():
    return [
        # one short sequence, 32 query heads on 4 KV heads: a decode step where only latency counts
        dict(name="attend 1 x 4K", op="attend", rows=1, longest=4097, shortest=4097, q_heads=32, kv_heads=4, dim=128, block=64,
             window=0, first=0, weigh=False),
        # a batch of 16 at 32K tokens, groups of 8 query heads
        dict(name="attend 16 x 32K", op="attend", rows=16, longest=32769, shortest=32769, q_heads=32, kv_heads=4, dim=128, block=64,
             window=0, first=0, weigh=False),
        # a ragged batch of 64 in small pages, groups of 4 query heads, an empty sequence among them
        dict(name="attend ragged 64", op="attend", rows=64, longest=16385, shortest=0, q_heads=32, kv_heads=8, dim=128, block=16,
             window=0, first=0, weigh=False),
        # one very long sequence, all 16 query heads on one KV head
        dict(name="attend 1 x 500K", op="attend", rows=1, longest=500003, shortest=500003, q_heads=16, kv_heads=1, dim=128, block=256,
             window=0, first=0, weigh=False),
        # long sequences through a window with sinks: only the last 4096 tokens and four first ones are read
        dict(name="window 32 x 4096 + 4", op="attend", rows=32, longest=20000, shortest=900, q_heads=32, kv_heads=8, dim=128, block=64,
             window=4096, first=4, weigh=False),
        # a small model's window, odd sizes, head by head
        dict(name="window 5 x 1000 + 5", op="attend", rows=5, longest=7001, shortest=1, q_heads=12, kv_heads=12, dim=64, block=32,
             window=1000, first=5, weigh=False),
        # a batch of bounded caches: attention that also adds up what every token got
        dict(name="weigh 32 x 4K", op="attend", rows=32, longest=4097, shortest=2500, q_heads=32, kv_heads=8, dim=128, block=64,
             window=0, first=0, weigh=True),
        # one new token for each of 64 sequences
        dict(name="append 64 tokens", op="append", rows=64, longest=1, shortest=1, before=1500, kv_heads=8, dim=128, block=64),
        # chunks of nine prompts that begin and end inside pages
        dict(name="append ragged chunks", op="append", rows=9, longest=4000, shortest=0, before=777, kv_heads=4, dim=128, block=16),
        # a full cache makes room for the next token: one slot of every row and head
        dict(name="evict 64 x 1 of 4K", op="evict", rows=64, longest=4096, shortest=4000, kv_heads=8, dim=128, block=64, budget=4095,
             first=4, recent=256, ordered=False),
        # a prompt of 32K tokens is cut to 4K
        dict(name="evict 32K to 4K", op="evict", rows=2, longest=32768, shortest=30001, kv_heads=4, dim=128, block=64, budget=4096,
             first=4, recent=512, ordered=True),
        # a whole step of a small model: one new token per sequence is written, attended with the rest, and all are weighed
        dict(name="step 16 x 2K", op="step", rows=16, longest=2048, shortest=1700, q_heads=12, kv_heads=4, dim=64, block=64,
             window=0, first=0, weigh=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "evict", "step"])
    dim, block = rng.choice([64, 128]), rng.choice([16, 32, 64, 128, 256])
    q_heads, kv_heads = rng.choice([(32, 4), (32, 8), (16, 1), (12, 4), (8, 8), (40, 1), (28, 4), (64, 2)])
    rows = _log(rng, 1, 64)
    if op == "append":
        longest = _log(rng, 1, max(2, 32000 // rows))
        return dict(op=op, rows=rows, longest=longest, shortest=longest if longest == 1 else rng.randint(0, longest), before=rng.randint(0, 2000),
                    kv_heads=kv_heads, dim=dim, block=block)
    if op == "evict":
        longest = _log(rng, 60, max(61, 400000 // (rows * kv_heads)))
        budget = rng.choice([longest - 1, rng.randint(longest // 2, longest - 1), rng.randint(longest // 10, longest // 2)])
        first = rng.randint(0, min(8, budget))
        return dict(op=op, rows=rows, longest=longest, shortest=rng.randint(0, longest), kv_heads=kv_heads, dim=dim, block=block, budget=budget,
                    first=first, recent=rng.randint(0, (budget - first) // 2), ordered=rng.random() < 0.5)
    longest = _log(rng, 1, max(2, 800000 // (rows * kv_heads)))
    windowed = rng.random() < 0.4
    return dict(op=op, rows=rows, longest=longest, shortest=rng.randint(1 if op == "step" else 0, longest), q_heads=q_heads, kv_heads=kv_heads,
                dim=dim, block=block, window=_log(rng, 1, max(2, longest)) if windowed else 0, first=rng.randint(0, 70) if windowed else 0,
                weigh=op == "step" or rng.random() < 0.3)


def _lengths(case):
    """Tokens of every row (of an append: new ones): between shortest and longest, both among them."""
    rng = random.Random("%(rows)d rows of %(shortest)d to %(longest)d" % case)
    n = [rng.randint(case["shortest"], case["longest"]) for _ in range(case["rows"])]
    n[-1] = case["shortest"]
    n[0] = case["longest"]
    return n


def _pages(case):
    """Pages of every row's table: an append continues rows that hold `before` tokens; an eviction's rows own their whole table."""
    return -(-(case.get("before", 0) + case["longest"]) // case["block"])


def work(case):
    d, h, n = case["dim"], case["kv_heads"], _lengths(case)
    if case["op"] == "append":
        return {"bytes": sum(n) * h * (8 * d + 8), "flops": sum(n) * h * d}
    if case["op"] == "evict":
        b = case["budget"]
        kept = sum(min(x, b) for x in n)
        moved = sum(min(b, x - b) * max(b, x - b) // x for x in n if x > b)     # expected, of kept slots spread evenly
        return {"bytes": h * (8 * sum(n) + 12 * kept + 8 * d * moved), "flops": h * sum(n) * 4}
    seen = sum(min(x, case["window"] + case["first"]) if case["window"] else x for x in n)
    rows = case["rows"] * case["q_heads"]
    new = case["rows"] * h * (4 * d + 8) if case["op"] == "step" else 0
    return {"bytes": seen * h * (4 * d + 8 * case["weigh"]) + rows * (6 * d + 4) + new, "flops": 4 * seen * case["q_heads"] * d}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    d, h, bt, rows = case["dim"], case["kv_heads"], case["block"], case["rows"]
    n = _lengths(case)
    new = torch.tensor(n, device=DEV, dtype=torch.int32)
    per_row = _pages(case)
    before = torch.zeros_like(new)
    if case["op"] == "append":
        before = torch.randint(0, case["before"] + 1, (rows,), generator=gen, device=DEV, dtype=torch.int32)
    lengths = before + new
    used = (lengths + bt - 1) // bt
    owned = torch.full_like(used, per_row) if case["op"] == "evict" else used
    # pages were handed out in any order; behind a row's last page the table holds -1
    n_pages = rows * per_row
    page = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32).view(rows, per_row)
    table = torch.where(torch.arange(per_row, device=DEV) < owned[:, None], page, torch.full_like(page, -1))
    pool = torch.empty((n_pages, h, 2, d // 64, bt, 8, 8), device=DEV, dtype=torch.bfloat16)
    pool.normal_(generator=gen)                                         # slots behind a row's length hold what was there before
    slots = per_row * bt
    # what a token has been given so far: much for a few, nothing for some
    weights = torch.exp(2.0 * _normal(gen, rows, h, slots)) * (torch.rand((rows, h, slots), generator=gen, device=DEV) > 0.05)
    if case.get("ordered", True):
        positions = torch.arange(slots, device=DEV, dtype=torch.int32).expand(rows, h, slots).contiguous()
    else:                                                               # slots have been refilled many times
        positions = (torch.rand((rows, h, slots), generator=gen, device=DEV).argsort(-1) * 3 + 7).to(torch.int32)
    state = dict(case=case, pool=pool, table=table, lengths=lengths, new=new, weights=weights, positions=positions)
    if case["op"] == "evict":
        state.update(weights_out=weights.clone(), positions_out=positions.clone(),
                     kept=torch.zeros((rows, h, case["budget"]), dtype=torch.int32, device=DEV))
    else:
        tokens = sum(n) if case["op"] == "append" else rows
        state["k"], state["v"] = _normal(gen, tokens, h, d).to(torch.bfloat16), _normal(gen, tokens, h, d).to(torch.bfloat16)
        state["at"] = torch.randint(0, 1000000, (tokens,), generator=gen, device=DEV, dtype=torch.int32)
        state["row_start"] = torch.cat([new.new_zeros(1), new.cumsum(0).to(torch.int32)]) if case["longest"] > 1 and case["op"] == "append" else None
    if case["op"] in ("attend", "step"):
        hq = case["q_heads"]
        state.update(q=_normal(gen, rows, hq, d).to(torch.bfloat16), weights_out=weights.clone(), o=torch.empty((rows, hq, d), device=DEV),
                     lse=torch.empty((rows, hq), device=DEV))
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------

def _scale(case):
    return case["dim"] ** -0.5


def run(state):
    case = state["case"]
    return _own(state, case) if own else _plain(state, case)


def _handle(state, case):
    """The shape, the cache and the scratch that a program keeps."""
    from paper_2609_14507_b200 import binding as b
    shape = b.make_shape(b.GQA, case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["dim"], case["dim"], case["block"], _scale(case))
    cache = b.make_paged(shape, state["pool"], state["table"], state["lengths"], weights=state["weights"], positions=state["positions"])
    if case["op"] == "evict":
        size = b.ipkv_paged_evict_scratch_bytes(shape, cache, case["budget"])
    elif case["op"] == "append":
        size = 0
    else:
        size = b.ipkv_paged_scratch_bytes(shape, cache, window=case["window"], first=case["first"], weigh=case["weigh"])
    state["handle"] = shape, cache, torch.empty(max(256, size), dtype=torch.uint8, device=DEV)
    return state["handle"]


def _own(state, case):
    from paper_2609_14507_b200 import binding as b
    shape, cache, scratch = state.get("handle") or _handle(state, case)
    if case["op"] == "evict":
        b.ipkv_paged_evict(shape, cache, case["budget"], case["first"], case["recent"], scratch, weights_out=state["weights_out"],
                           positions_out=state["positions_out"], kept=state["kept"])
        return {"pool": state["pool"], "weights": state["weights_out"], "positions": state["positions_out"], "kept": state["kept"]}
    if case["op"] in ("append", "step"):
        b.ipkv_paged_append(shape, cache, state["k"], state["v"], positions=state["at"], row_start=state["row_start"])
        if case["op"] == "append":
            return {"pool": state["pool"], "weights": state["weights"], "positions": state["positions"]}
    b.ipkv_paged_attend(shape, cache, state["q"], scratch, state["o"], state["lse"], window=case["window"], first=case["first"],
                        weights_out=state["weights_out"] if case["weigh"] else None)
    out = {"o": state["o"], "lse": state["lse"]}
    if case["weigh"]:
        out["weights"] = state["weights_out"]
    if case["op"] == "step":
        out.update(pool=state["pool"], positions=state["positions"])
    return out


def _index(case, page, t, head=None):
    """Where tokens lie: page and t (offset in the page) [rows, n], or [rows, heads, n] with the heads' own slots.  The result indexes
    the pool and gives [rows, n, heads, 2, panels, 8, 8], or [rows, heads, n, 2, panels, 8, 8]."""
    h, panels = case["kv_heads"], case["dim"] // 64
    if head is None:
        page, t, head = page[:, :, None], t[:, :, None], torch.arange(h, device=DEV)
    else:
        head = torch.arange(h, device=DEV)[:, None]
    page, t, head = page.long()[..., None, None, None], t.long()[..., None, None, None], head[..., None, None, None]
    kv = torch.arange(2, device=DEV)[:, None, None]
    panel = torch.arange(panels, device=DEV)[:, None]
    chunk = torch.arange(8, device=DEV) ^ (t & 7)
    return page, head, kv, panel, t, chunk


def _append(state, case):
    bt, lengths, new = case["block"], state["lengths"].long(), state["new"].long()
    k = state["k"]
    if case["op"] == "step":
        row = torch.arange(case["rows"], device=DEV)
        slot = lengths - 1
    else:
        row = torch.repeat_interleave(torch.arange(case["rows"], device=DEV), new, output_size=k.shape[0])
        slot = lengths[row] - new[row] + torch.arange(k.shape[0], device=DEV) - (new.cumsum(0) - new)[row]
    page = state["table"][row, slot // bt]
    at = _index(case, page[:, None], (slot % bt)[:, None])
    kv = torch.stack([k, state["v"]], 2)                                # [tokens, heads, 2, dim]
    state["pool"][at] = kv.view(*kv.shape[:3], case["dim"] // 64, 8, 8)[:, None]
    head = torch.arange(case["kv_heads"], device=DEV)
    state["weights"][row[:, None], head, slot[:, None]] = 0.0
    state["positions"][row[:, None], head, slot[:, None]] = state["at"][:, None].expand(-1, case["kv_heads"])
    return {"pool": state["pool"], "weights": state["weights"], "positions": state["positions"]}


def _kept(state, case):
    """For every slot below the budget, the slot whose token it holds afterwards; and the selection."""
    w, pos, b = state["weights"], state["positions"], case["budget"]
    slot = torch.arange(w.shape[-1], device=DEV)
    n = state["lengths"][:, None, None].long()
    there = slot < n
    newest = torch.where(there, pos, torch.full_like(pos, -1)).amax(-1, keepdim=True)
    stays = (pos < case["first"]) | (pos > newest - case["recent"])
    key = torch.where(stays, float("inf"), w)
    key = torch.where(there, key, float("-inf"))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order))
    chosen = (rank < b) & there
    behind = chosen & (slot >= b)
    survivors = torch.sort((~behind).to(torch.uint8), dim=-1, stable=True).indices
    hole = there & ~chosen & (slot < b)
    at = (hole.cumsum(-1) - 1).clamp(min=0)
    return torch.where(hole, survivors.gather(-1, at), slot.expand_as(order))[..., :b], hole, behind


def _plain_evict(state, case):
    b, bt = case["budget"], case["block"]
    kept, hole, behind = _kept(state, case)
    slots = state["weights"].shape[-1]
    # the moves: at most as many as there are slots behind the budget; a pair that is none writes a slot behind it onto itself
    m = min(b, slots - b)
    into = torch.sort((~hole).to(torch.uint8), dim=-1, stable=True).indices[..., :m]
    real = torch.arange(m, device=DEV) < hole.sum(-1, keepdim=True)
    into = torch.where(real, into, slots - 1)
    source = torch.where(real, kept.gather(-1, into.clamp(max=b - 1)), slots - 1)
    row = torch.arange(case["rows"], device=DEV)[:, None, None]
    place = lambda s: _index(case, state["table"][row, s // bt], s % bt, head=True)  # noqa: E731
    state["pool"][place(into)] = state["pool"][place(source)]
    there = torch.arange(b, device=DEV) < state["lengths"][:, None, None]
    for_kept = lambda x: torch.cat([torch.where(there, x.gather(-1, kept), x[..., :b]), x[..., b:]], -1)  # noqa: E731
    return {"pool": state["pool"], "weights": for_kept(state["weights"]), "positions": for_kept(state["positions"]),
            "kept": torch.where(there, kept, 0).to(torch.int32)}


def _plain(state, case):
    if case["op"] == "evict":
        return _plain_evict(state, case)
    if case["op"] == "append":
        return _append(state, case)
    out = _append(state, case) if case["op"] == "step" else {}
    rows, h, hq, d, bt = case["rows"], case["kv_heads"], case["q_heads"], case["dim"], case["block"]
    n = state["lengths"].long()[:, None]
    # the visible tokens of every row, one behind the other: the first ones, then the window
    most = min(case["longest"], case["window"] + case["first"]) if case["window"] else case["longest"]
    t = torch.arange(max(most, 1), device=DEV)
    slot = torch.where((t >= case["first"]) & (n > most), n - most + t, t) if case["window"] else t.expand(rows, -1)
    there = t < n.clamp(max=most)
    page = state["table"].gather(1, (slot // bt).clamp(max=state["table"].shape[1] - 1)).clamp(min=0)
    kv = state["pool"][_index(case, page, slot % bt)]                   # [rows, n, heads, 2, panels, 8, 8]
    kv = kv.flatten(4).masked_fill(~there[:, :, None, None, None], 0.0)
    k, v = kv[:, :, :, 0].transpose(1, 2).float(), kv[:, :, :, 1].transpose(1, 2).float()
    s = torch.matmul(state["q"].float().view(rows, h, hq // h, d), k.transpose(2, 3)) * _scale(case)
    s = s.masked_fill(~there[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top.isinf(), torch.zeros_like(top), top))
    z = e.sum(-1, keepdim=True)
    p = e / torch.where(z > 0, z, torch.ones_like(z))
    result = {"o": torch.matmul(p, v).reshape(rows, hq, d), "lse": (top + torch.log(z)).reshape(rows, hq)}
    if case["weigh"]:
        at = torch.where(there, slot, state["weights"].shape[-1])[:, None].expand(-1, h, -1)         # one more column takes what is none
        wide = torch.cat([state["weights"], torch.zeros_like(state["weights"][..., :1])], -1)
        result["weights"] = wide.scatter_add(-1, at, p.sum(2))[..., :-1].contiguous()
    if case["op"] == "step":
        result.update(pool=out["pool"], positions=out["positions"])
    return result


# ---- the definition, in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    """Row by row.  What is moved and not computed has no other value than the plain form's."""
    if case["op"] in ("append", "evict"):
        return None
    state = prepare(case, seed)
    rows, h, hq, d, bt = case["rows"], case["kv_heads"], case["q_heads"], case["dim"], case["block"]
    o = torch.zeros((rows, hq, d), device=DEV, dtype=torch.float64)
    lse = torch.full((rows, hq), float("-inf"), device=DEV, dtype=torch.float64)
    weights = state["weights"].double()
    planes = state["pool"].permute(0, 4, 1, 2, 3, 5, 6)                 # [pages][t][heads][2][panels][chunk][8]
    for r, n in enumerate(_lengths(case)):
        if not n:
            continue
        if case["op"] == "step":
            weights[r, :, n - 1] = 0.0
        if case["window"] and n > case["window"] + case["first"]:
            slot = torch.cat([torch.arange(case["first"]), torch.arange(n - case["window"], n)]).to(DEV)
        else:
            slot = torch.arange(n, device=DEV)
        t = slot % bt
        x = planes[state["table"][r].long()[slot // bt], t]
        order = (torch.arange(8, device=DEV) ^ (t % 8)[:, None])[:, None, None, None, :, None]
        x = x.gather(4, order.expand(-1, h, 2, d // 64, 8, 8)).reshape(-1, h, 2, d)
        k, v = x[:, :, 0].double(), x[:, :, 1].double()
        if case["op"] == "step":
            k[-1], v[-1] = state["k"][r].double(), state["v"][r].double()
        for g in range(h):
            of_group = slice(g * (hq // h), (g + 1) * (hq // h))
            s = state["q"][r, of_group].double() @ k[:, g].t() * _scale(case)
            lse[r, of_group] = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1)
            o[r, of_group] = p @ v[:, g]
            if case["weigh"]:
                weights[r, g, slot] += p.sum(0)
    out = {"o": o, "lse": lse}
    if case["weigh"]:
        out["weights"] = weights
    if case["op"] == "step":
        out.update(pool=None, positions=None)
    return out
