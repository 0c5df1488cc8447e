"""The paged cache restated from its definition in include/ipkv.h (torch, any device): where a token lies, attention in 64 bits with
a bound that follows the kernel's arithmetic, eviction slot by slot."""
import math

import torch


def element_offsets(bt, d, t):
    """Element offsets of the d columns of token offset t inside a plane."""
    x = torch.arange(d)
    return (x // 64) * bt * 64 + t * 64 + (((x % 64) // 8) ^ (t & 7)) * 8 + x % 8


class Pool:
    """A pool of TILE blocks as bf16 elements [n_blocks, n_kv_heads, 2, bt * d] and a page table."""

    def __init__(self, n_blocks, hkv, d, bt, device, fill=None):
        self.hkv, self.d, self.bt, self.device = hkv, d, bt, device
        self.data = torch.empty((n_blocks, hkv, 2, bt * d), dtype=torch.bfloat16, device=device)
        if fill is None:
            self.data.normal_()
        else:
            self.data.fill_(fill)
        self.at = torch.stack([element_offsets(bt, d, t) for t in range(bt)]).to(device)       # [bt, d]

    def get(self, pages, slots):
        """K and V [n, hkv, d] of slots of a row with these pages."""
        pages, slots = torch.as_tensor(pages, device=self.device).long(), torch.as_tensor(slots, device=self.device).long()
        x = self.data[pages[slots // self.bt]].gather(3, self.at[slots % self.bt][:, None, None].expand(-1, self.hkv, 2, -1))
        return x[:, :, 0], x[:, :, 1]

    def put(self, pages, slots, k, v):
        pages, slots = torch.as_tensor(pages, device=self.device).long(), torch.as_tensor(slots, device=self.device).long()
        at = self.at[slots % self.bt][:, None]
        head = torch.arange(self.hkv, device=self.device)[None, :, None]
        page = pages[slots // self.bt][:, None, None]
        self.data[page, head, 0, at] = k
        self.data[page, head, 1, at] = v


def visible(n, window, first):
    return [t for t in range(n) if window == 0 or t >= n - window or t < first]


def attend(q, k, v, scale):
    """One row in 64 bits: q [Hq, D], k, v [n, Hkv, D] -> O, LSE, the softmax weights [Hq, n], and bounds for the first three.

    The bounds: a score is a sum of D exact products in fp32, the tensor cores' sum cut towards zero (D + 2 steps of 2^-23 of the sum of
    magnitudes), times a rounded constant (2 steps of 2^-24 of the score, one of them the scale's), minus a maximum (one more); 2^x is off
    by 2^-22 of itself and a weight in three pieces by 2^-24.  Sums over tokens round once per token in a tile, per tile and per
    partial: 16 + n / 16 + 300 steps of 2^-23 at most, numerator and denominator alike."""
    hq, d = q.shape
    n, hkv = k.shape[0], k.shape[1]
    dev = q.device
    if n == 0:
        return (torch.zeros((hq, d), dtype=torch.float64, device=dev), torch.full((hq,), -math.inf, dtype=torch.float64, device=dev),
                torch.zeros((hq, 0), dtype=torch.float64, device=dev), torch.zeros((hq, d), device=dev), torch.zeros(hq, device=dev),
                torch.zeros((hq, 0), device=dev))
    qd, kd, vd = q.double().view(hkv, hq // hkv, d), k.double(), v.double()
    s = torch.einsum("hgd,nhd->hgn", qd, kd) * scale
    size = torch.einsum("hgd,nhd->hgn", qd.abs(), kd.abs()) * scale
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    p = p / z
    o = torch.einsum("hgn,nhd->hgd", p, vd)
    off = (d + 2) * 2.0 ** -23 * size + 4 * 2.0 ** -24 * (s.abs() + m.abs())       # of a score
    of_p = torch.expm1(off) + 2.0 ** -21                                            # of a weight, relative
    sums = (16 + n / 16 + 300) * 2.0 ** -23
    of_z = (p * of_p).sum(-1, keepdim=True) + sums
    tol_o = torch.einsum("hgn,nhd->hgd", p * (of_p + of_z + sums), vd.abs()) + 2.0 ** -22 * o.abs()
    tol_lse = (of_z + 2.0 ** -22 * (1 + m.abs() + torch.log(z).abs())).squeeze(-1)
    tol_p = p * (of_p + of_z + 2.0 ** -22)
    flat = lambda x: x.reshape(hq, *x.shape[2:])  # noqa: E731
    return (flat(o), flat((m + torch.log(z)).squeeze(-1)), flat(p), flat(tol_o), flat(tol_lse), flat(tol_p))


def kept(weights, positions, budget, first, recent):
    """Of one row and head (lists): the slot that every slot below the budget takes its token from."""
    n = len(weights)
    if n <= budget:
        return list(range(n))
    newest = max(positions)

    def rank(t):
        if positions[t] < first or positions[t] > newest - recent:
            return (0, 0.0, t)
        w = weights[t]
        return (2, 0.0, t) if w != w else (1, -w, t)

    chosen = set(sorted(range(n), key=rank)[:budget])
    result = list(range(budget))
    holes = [t for t in range(budget) if t not in chosen]
    for hole, slot in zip(holes, sorted(t for t in chosen if t >= budget)):
        result[hole] = slot
    return result
