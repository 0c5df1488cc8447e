"""The paged cache: refusals (no GPU), append byte by byte, attention against 64 bits, eviction slot by slot, and a captured decode run."""
import math
import random

import pytest

from paper_2609_14507_b200 import binding
from tests import paged_ref as ref

torch = pytest.importorskip("torch")
C = binding.C
EINVAL, ENOMEM, ECUDA = 1, 2, 5
BASE = 1 << 30          # an aligned address that nothing reads: the calls below are refused first
BAD_PAGE = 16


def shape_of(hq, hkv, d, bt, scale=0.0, kind=binding.GQA, dv=None):
    return binding.make_shape(kind, hq, hkv, d, d if dv is None else dv, bt, scale)


# ---- refusals --------------------------------------------------------------------------------------------------------

def struct(**kw):
    c = dict(pool_dev=BASE, pool_bytes=10 << 17, table_dev=BASE, lengths_dev=BASE, n_rows=2, max_blocks=4, table_stride=4, weights_dev=BASE, positions_dev=BASE,
             slot_stride=256)
    c.update(kw)
    return binding.Paged(**c)


def append_rc(sh, c, n=2, k=BASE, v=BASE, ks=0, vs=0, start=None, at=BASE, status=None):
    return binding.lib().ipkv_paged_append(binding._APPEND_CALL.pack(C.addressof(sh), C.addressof(c), n, k or 0, v or 0, ks, vs, start or 0, at or 0, status or 0, 0))


def attend_rc(sh, c, q=BASE, qs=0, window=0, first=0, w=None, scratch=BASE, size=1 << 40, o=BASE, lse=BASE, status=None):
    return binding.lib().ipkv_paged_attend(binding._ATTEND_CALL.pack(C.addressof(sh), C.addressof(c), q or 0, qs, window, first, w or 0, scratch or 0, size, o or 0, lse or 0,
                                                                     status or 0, 0))


def evict_rc(sh, c, budget=100, first=4, recent=10, w=None, pos=None, kept=None, scratch=BASE, size=1 << 40, status=None):
    return binding.lib().ipkv_paged_evict(binding._EVICT_CALL.pack(C.addressof(sh), C.addressof(c), budget, first, recent, w or 0, pos or 0, kept or 0, scratch or 0, size,
                                                                   status or 0, 0))


def test_the_packed_arguments_are_the_structs_of_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sz.c"
    last = {"ipkv_paged": "slot_stride", "ipkv_paged_append_call": "stream", "ipkv_paged_attend_call": "stream", "ipkv_paged_evict_call": "stream"}
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ipkv.h"\nint main(void){'
                   + "".join(f'printf("%zu %zu ", sizeof({t}), offsetof({t}, {m}));' for t, m in last.items())
                   + 'printf("%zu %zu\\n", offsetof(ipkv_paged_attend_call, weights_out_dev), offsetof(ipkv_paged_evict_call, weights_out_dev));return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = [C.sizeof(binding.Paged), binding.Paged.slot_stride.offset]
    for s in (binding._APPEND_CALL, binding._ATTEND_CALL, binding._EVICT_CALL):
        want += [s.size, s.size - 8]
    assert got == want + [40, 32]
    for call in (binding.lib().ipkv_paged_append, binding.lib().ipkv_paged_attend, binding.lib().ipkv_paged_evict):
        assert call(None) == EINVAL


@pytest.mark.parametrize("sh", [shape_of(32, 5, 128, 64), shape_of(32, 4, 96, 64), shape_of(32, 4, 256, 64), shape_of(32, 4, 128, 8), shape_of(32, 4, 128, 48),
                                shape_of(32, 4, 128, 96), shape_of(32, 4, 128, 0), shape_of(0, 4, 128, 64), shape_of(32, 0, 128, 64),
                                shape_of(32, 4, 128, 64, dv=64), shape_of(16, 1, 576, 64, kind=binding.MLA, dv=512), shape_of(32, 4, 128, -64)])
def test_shapes_without_the_operators_are_refused(sh):
    n = C.c_size_t()
    L = binding.lib()
    assert append_rc(sh, struct()) == attend_rc(sh, struct()) == evict_rc(sh, struct()) == EINVAL
    assert L.ipkv_paged_scratch_bytes(C.byref(sh), 2, 4, 0, 0, 0, C.byref(n)) == EINVAL
    assert L.ipkv_paged_evict_scratch_bytes(C.byref(sh), 2, 4, 100, C.byref(n)) == EINVAL


def test_bad_caches_are_refused():
    sh = shape_of(32, 4, 128, 64)
    for kw in (dict(pool_dev=None), dict(pool_dev=BASE + 8), dict(pool_bytes=0), dict(pool_bytes=-1), dict(pool_bytes=(1 << 17) - 1), dict(pool_bytes=1 << 48), dict(table_dev=None),
               dict(table_dev=BASE + 2), dict(lengths_dev=None), dict(lengths_dev=BASE + 1), dict(n_rows=-1), dict(max_blocks=0), dict(max_blocks=-3),
               dict(max_blocks=1 << 26, table_stride=1 << 26), dict(table_stride=3), dict(weights_dev=BASE + 4), dict(positions_dev=BASE + 8),
               dict(slot_stride=255), dict(slot_stride=252), dict(slot_stride=258)):
        c = struct(**kw)
        assert append_rc(sh, c) == attend_rc(sh, c) == evict_rc(sh, c) == EINVAL, kw
    for none in (struct(n_rows=0), struct(n_rows=0, table_dev=None, lengths_dev=None, weights_dev=None, positions_dev=None)):     # nothing to do
        assert append_rc(sh, none, n=0) == attend_rc(sh, none) == attend_rc(sh, none, q=None, scratch=None, o=None, lse=None) == evict_rc(sh, none) == 0


def test_bad_calls_are_refused():
    sh, c, L = shape_of(32, 4, 128, 64), struct(), binding.lib()
    for kw in (dict(n=-1), dict(n=3), dict(n=1), dict(n=1 << 31, start=BASE), dict(k=None), dict(v=None), dict(k=BASE + 8), dict(v=BASE + 2), dict(ks=504),
               dict(vs=-512), dict(ks=516), dict(start=BASE + 2), dict(at=BASE + 2), dict(at=None), dict(status=BASE + 1)):
        assert append_rc(sh, c, **kw) == EINVAL, kw
    assert append_rc(sh, c, n=0, start=BASE) == 0
    for kw in (dict(q=None), dict(q=BASE + 8), dict(qs=4088), dict(qs=4100), dict(window=-1), dict(first=-1), dict(w=BASE + 4), dict(w=BASE + 1024), dict(scratch=None),
               dict(scratch=BASE + 128), dict(o=None), dict(o=BASE + 4), dict(lse=None), dict(lse=BASE + 2), dict(status=BASE + 2)):
        assert attend_rc(sh, c, **kw) == EINVAL, kw
    for scale in (-1.0, float("nan"), float("inf")):
        assert attend_rc(shape_of(32, 4, 128, 64, scale), c) == EINVAL
    n = C.c_size_t()
    sizes = []
    for weigh in (0, 1):
        assert L.ipkv_paged_scratch_bytes(C.byref(sh), 2, 4, 0, 0, weigh, C.byref(n)) == 0
        assert attend_rc(sh, c, w=BASE + (1 << 20) if weigh else None, size=n.value - 1) == ENOMEM
        sizes.append(n.value)
    assert sizes[1] > sizes[0]
    assert L.ipkv_paged_scratch_bytes(C.byref(sh), 2, 4, 0, 0, 0, None) == L.ipkv_paged_scratch_bytes(C.byref(sh), -1, 4, 0, 0, 0, C.byref(n)) == EINVAL
    for kw in (dict(budget=0), dict(budget=-5), dict(first=-1), dict(recent=-1), dict(first=50, recent=51), dict(first=2 ** 31 - 1, recent=2 ** 31 - 1),
               dict(w=BASE + 2), dict(w=BASE + 1024), dict(pos=BASE + 8), dict(pos=BASE + 1024), dict(kept=BASE + 2), dict(scratch=BASE + 64), dict(scratch=None), dict(status=BASE + 2)):
        assert evict_rc(sh, c, **kw) == EINVAL, kw
    assert evict_rc(sh, struct(weights_dev=None)) == evict_rc(sh, struct(positions_dev=None)) == EINVAL
    assert L.ipkv_paged_evict_scratch_bytes(C.byref(sh), 2, 4, 100, C.byref(n)) == 0 and n.value >= 2 * 4 * 2 * 100 * 4
    assert evict_rc(sh, c, size=n.value - 1) == ENOMEM
    assert L.ipkv_paged_evict_scratch_bytes(C.byref(sh), 2, 4, 256, C.byref(n)) == 0 and n.value == 0       # a budget that nothing exceeds
    if not torch.cuda.is_available():                    # what is refused for the missing GPU alone
        assert append_rc(sh, c) == attend_rc(sh, c) == attend_rc(sh, c, w=BASE) == evict_rc(sh, c) == ECUDA


def test_the_binding_refuses_other_types_and_shapes():
    sh = shape_of(4, 2, 64, 64)
    pool = torch.zeros((3, 2, 2, 64 * 64), dtype=torch.bfloat16)
    table, lengths = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    w, pos = torch.zeros((2, 2, 192)), torch.zeros((2, 2, 192), dtype=torch.int32)
    for a in ((pool[:, :1], table, lengths), (pool.flatten()[:-1], table, lengths), (pool[:0], table, lengths), (pool, table.long(), lengths), (pool, table[0], lengths),
              (pool, table.t(), lengths), (pool, table[:1].expand(2, 3), lengths), (pool, table, lengths.long()), (pool, table, lengths[:1]),
              (pool, table, lengths, w.double()), (pool, table, lengths, w[:, :, :128].contiguous()), (pool, table, lengths, w[:, :1].contiguous()),
              (pool, table, lengths, w, pos.float()), (pool, table, lengths, w, pos[:, :, :188].contiguous()), (pool, table, lengths, w.transpose(0, 1))):
        with pytest.raises(ValueError):
            binding.make_paged(sh, *a)
    c = binding.make_paged(sh, pool, table, lengths, w, pos)
    assert (c.pool_bytes, c.n_rows, c.max_blocks, c.table_stride, c.slot_stride) == (3 * 32768, 2, 3, 3, 192)
    wide = binding.make_paged(sh, pool, torch.zeros((2, 7), dtype=torch.int32)[:, 2:5], lengths)
    assert wide.table_stride == 7 and wide.slot_stride == 192
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    at, start = torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for a, kw in (((k.float(), k), dict(positions=at)), ((k, k[:1]), dict(positions=at)), ((k[:1], k[:1]), dict(positions=at[:1])), ((k, k), {}),
                  ((k, k), dict(positions=at.long())), ((k, k), dict(positions=at[:1])), ((k, k), dict(positions=at, row_start=start[:2])),
                  ((k, k), dict(positions=at, row_start=start.long())), ((k[:1].expand(2, 2, 64), k), dict(positions=at)),
                  ((k.transpose(0, 1).contiguous().transpose(0, 1), k), dict(positions=at)), ((k[..., :32], k), dict(positions=at))):
        with pytest.raises(ValueError):
            binding.ipkv_paged_append(sh, c, *a, **kw)
    q, o, lse, scratch = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 64)), torch.zeros((2, 4)), torch.zeros(64, dtype=torch.uint8)
    for a, kw in (((q.float(), scratch, o, lse), {}), ((q[:1], scratch, o, lse), {}), ((q, scratch, o.bfloat16(), lse), {}), ((q, scratch, o, lse[:1]), {}),
                  ((q[:1].expand(2, 4, 64), scratch, o, lse), {}), ((q.transpose(0, 1).contiguous().transpose(0, 1), scratch, o, lse), {}),
                  ((q, scratch[::2], o, lse), {}), ((q, scratch, o, lse), dict(weights_out=w[:, :, :188].contiguous())), ((q, scratch, o, lse), dict(weights_out=pos)),
                  ((q, scratch, o, lse), dict(status=torch.zeros(1)))):
        with pytest.raises(ValueError):
            binding.ipkv_paged_attend(sh, c, *a, **kw)
    for kw in (dict(weights_out=pos), dict(positions_out=w), dict(kept=torch.zeros((2, 2, 9), dtype=torch.int32)), dict(kept=torch.zeros((2, 2, 10)))):
        with pytest.raises(ValueError):
            binding.ipkv_paged_evict(sh, c, 10, 0, 0, scratch, **kw)
    other = shape_of(4, 4, 64, 64)                       # more KV heads than the cache has
    for call in (lambda: binding.ipkv_paged_append(other, c, k.repeat(1, 2, 1), k.repeat(1, 2, 1), positions=at), lambda: binding.ipkv_paged_attend(other, c, q, scratch, o, lse),
                 lambda: binding.ipkv_paged_evict(other, c, 10, 0, 0, scratch)):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(window=1 << 31), dict(first=1 << 31), dict(window=1.5)):
        with pytest.raises(ValueError):
            binding.ipkv_paged_attend(sh, c, q, scratch, o, lse, **kw)
    with pytest.raises(ValueError):
        binding.ipkv_paged_evict(sh, c, 1 << 40, 0, 0, scratch)
    for call in (lambda: binding.ipkv_paged_append(sh, c, k, k, positions=at), lambda: binding.ipkv_paged_attend(sh, c, q, scratch, o, lse),
                 lambda: binding.ipkv_paged_evict(sh, c, 10, 0, 0, scratch)):
        with pytest.raises(ValueError, match="on device -1"):            # refused for nothing but being on the host
            call()


# ---- what a test works on ---------------------------------------------------------------------------------------------

class Case:
    """A pool whose pages were handed out in any order, rows of the given lengths, and what a slot carries."""

    def __init__(self, lengths, hq, hkv, d, bt, scale=0.0, per_row=None, seed=0, spare=2, fill=None):
        self.hq, self.hkv, self.d, self.bt, self.n = hq, hkv, d, bt, list(lengths)
        gen = torch.Generator().manual_seed(seed)
        torch.manual_seed(seed)
        rows = len(lengths)
        self.per_row = per_row or max(1, -(-max(lengths) // bt))
        self.pool = ref.Pool(rows * self.per_row + spare, hkv, d, bt, "cuda", fill)
        pages = torch.randperm(rows * self.per_row + spare, generator=gen)[:rows * self.per_row].view(rows, self.per_row)
        self.pages = pages
        used = torch.tensor([-(-n // bt) for n in lengths])
        junk = torch.randint(-2 ** 31, 2 ** 31, pages.shape, generator=gen)              # entries behind the length are not read
        self.table = torch.where(torch.arange(self.per_row) < used[:, None], pages, junk).to(torch.int32).cuda()
        self.lengths = torch.tensor(lengths, dtype=torch.int32).cuda()
        slots = self.per_row * bt
        self.weights = torch.rand((rows, hkv, slots), generator=gen).cuda()
        self.positions = torch.rand((rows, hkv, slots), generator=gen).argsort(-1).to(torch.int32).cuda()
        self.shape = shape_of(hq, hkv, d, bt, scale)
        self.scale = scale or d ** -0.5
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.q = torch.randn((rows, hq, d), generator=gen).to(torch.bfloat16).cuda()

    def cache(self, weights=True, positions=True):
        return binding.make_paged(self.shape, self.pool.data, self.table, self.lengths, self.weights if weights else None, self.positions if positions else None)

    def attend(self, window=0, first=0, weights_out=None, cache=None, q=None, **kw):
        cache = cache or self.cache()
        rows = len(self.n)
        size = binding.ipkv_paged_scratch_bytes(self.shape, cache, window, first, weights_out is not None)
        scratch = torch.randint(0, 256, (max(256, size),), dtype=torch.uint8, device="cuda")          # whatever was there
        o, lse = torch.full((rows, self.hq, self.d), 7.0, device="cuda"), torch.full((rows, self.hq), 7.0, device="cuda")
        binding.ipkv_paged_attend(self.shape, cache, self.q if q is None else q, scratch, o, lse, window, first, weights_out, status=self.status, **kw)
        return o, lse

    def check(self, o, lse, window=0, first=0, weights_out=None, base=None, rows=None, q=None):
        """Outputs against 64 bits; slots that are not visible keep what weights_out held (`base`)."""
        for r in rows if rows is not None else range(len(self.n)):
            seen = ref.visible(self.n[r], window, first)
            k, v = self.pool.get(self.pages[r], seen) if seen else (self.pool.data.new_zeros((0, self.hkv, self.d)),) * 2
            eo, el, ep, to, tl, tp = ref.attend((self.q if q is None else q)[r], k, v, self.scale)
            assert (o[r].double() - eo).abs().le(to).all(), (r, float(((o[r].double() - eo).abs() / to.clamp(min=1e-30)).max()))
            assert (lse[r].double() - el).abs().le(tl).logical_or(lse[r].double() == el).all(), r
            if weights_out is not None:
                g = self.hq // self.hkv
                want, tol = base[r].double().clone(), torch.zeros_like(base[r], dtype=torch.float64)
                if seen:
                    add = ep.view(self.hkv, g, -1).sum(1)
                    want[:, seen] += add
                    # the sum over the heads, and with what was there
                    tol[:, seen] = tp.view(self.hkv, g, -1).sum(1) + (g + 1) * 2.0 ** -23 * want[:, seen].abs()
                assert (weights_out[r].double() - want).abs().le(tol).all(), r


# ---- attention -------------------------------------------------------------------------------------------------------

SHAPES = [(4, 1, 128, 64), (3, 1, 64, 16), (8, 8, 128, 32), (8, 1, 64, 64), (10, 2, 128, 16), (28, 4, 128, 128), (16, 1, 128, 64), (24, 2, 64, 32), (17, 1, 128, 64),
          (32, 1, 64, 128), (40, 1, 128, 16), (64, 1, 128, 256), (128, 2, 64, 64), (40, 40, 64, 16), (50, 2, 128, 192)]
LENGTHS = [[1], [0, 1, 0], [63, 64, 65, 16, 17, 15], [4097], [300, 0, 2000, 7, 129], [1000] * 40 + [0] * 3 + [5], [5000, 1, 20, 64] * 25]


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,bt", SHAPES)
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda n: f"{len(n)}x{max(n)}")
def test_attention_matches_64_bits(hq, hkv, d, bt, lengths):
    c = Case(lengths, hq, hkv, d, bt)
    out = torch.full_like(c.weights, 3.0)
    o, lse = c.attend()
    assert int(c.status) == 0
    c.check(o, lse)
    o2, lse2 = c.attend(weights_out=out)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and int(c.status) == 0
    base = c.weights.clone()
    for r, n in enumerate(lengths):
        base[r, :, n:] = 3.0
    c.check(o2, lse2, weights_out=out, base=base)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,bt", [(1, 1, 64, 64), (5, 1, 128, 16), (16, 2, 64, 256), (16, 1, 128, 64), (7, 1, 64, 32)])
@pytest.mark.parametrize("lengths", [[2100], [33 * 32, 0, 1], [2049, 31, 500, 2100], [1, 0, 0, 4000], [64, 4200, 63, 65]], ids=str)
def test_few_pairs_of_some_units_are_taken_by_large_clusters(hq, hkv, d, bt, lengths):
    c = Case(lengths, hq, hkv, d, bt)
    for window, first in ((0, 0), (2080, 33)):
        base, out = c.weights.clone(), c.weights.clone()
        o, lse = c.attend(window, first, out)
        assert int(c.status) == 0
        c.check(o, lse, window, first, out, base)
        o2, lse2 = c.attend(window, first)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,bt", [(4, 1, 128, 64), (12, 2, 64, 16), (8, 8, 128, 32), (40, 1, 64, 256), (16, 1, 128, 128)])
@pytest.mark.parametrize("window,first", [(1, 0), (1, 1), (5, 3), (64, 0), (64, 64), (100, 70), (1000, 4), (3000, 200), (2 ** 31 - 1, 2 ** 31 - 1), (7, 5000), (4096, 0)])
def test_a_window_and_first_tokens(hq, hkv, d, bt, window, first):
    c = Case([0, 1, 5, 64, 66, 130, 1005, 4097, 3100], hq, hkv, d, bt)
    out = c.weights.clone()
    # what is not visible may hold anything
    for r, n in enumerate(c.n):
        hidden = sorted(set(range(c.per_row * bt)) - set(ref.visible(n, window, first)))
        junk = torch.tensor([math.nan, math.inf, -math.inf, 3e38], dtype=torch.bfloat16, device="cuda")
        hidden = [t for t in hidden if t < -(-n // bt) * bt]
        if hidden:
            x = junk[torch.arange(len(hidden), device="cuda") % 4][:, None, None].expand(-1, hkv, d)
            c.pool.put(c.pages[r], hidden, x, x)
    base = c.weights.clone()
    o, lse = c.attend(window, first, out)
    assert int(c.status) == 0
    c.check(o, lse, window, first, out, base)


@pytest.mark.gpu
def test_pages_that_nobody_owns_are_never_read():
    """Every block but the rows' own holds NaN, and so do the rows' own behind their lengths."""
    for bt in (16, 32, 64, 192):
        c = Case([100, 1, 0, 777, 64], 8, 2, 128, bt, spare=5)
        keep = c.pool.data.clone()
        c.pool.data.fill_(math.nan)
        for r, n in enumerate(c.n):
            if n:
                clean = ref.Pool.__new__(ref.Pool)
                clean.__dict__.update(c.pool.__dict__, data=keep)
                c.pool.put(c.pages[r], list(range(n)), *clean.get(c.pages[r], list(range(n))))
        o, lse = c.attend()
        assert torch.isfinite(o).all()
        c.check(o, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("bt", [16, 64, 256])
def test_bad_pages_and_lengths_are_told_and_left_out(bt):
    c = Case([1500, 700, 900, 40], 8, 2, 128, bt, per_row=-(-1500 // bt))
    for entry in (-1, c.pool.data.shape[0], 2 ** 31 - 1, -2 ** 31):
        j = 1 if bt < 1000 else 0
        good = int(c.table[0, j])
        c.table[0, j] = entry
        out = c.weights.clone()
        o, lse = c.attend(weights_out=out)
        assert int(c.status) == BAD_PAGE
        c.status.zero_()
        c.check(o, lse, weights_out=out, base=c.weights, rows=[1, 2, 3])
        seen = [t for t in range(1500) if t // bt != j]
        eo, el, ep, to, tl, tp = ref.attend(c.q[0], *c.pool.get(c.pages[0], seen), c.scale)
        assert (o[0].double() - eo).abs().le(to).all() and (lse[0].double() - el).abs().le(tl).all()
        assert torch.equal(out[0][:, j * bt:(j + 1) * bt], c.weights[0][:, j * bt:(j + 1) * bt])
        c.table[0, j] = good
    for bad, n in ((-5, 0), (-2 ** 31, 0), (c.per_row * bt + 1, c.per_row * bt), (2 ** 31 - 1, c.per_row * bt)):
        full = Case([c.per_row * bt, 700, 900, 40], 8, 2, 128, bt)
        full.lengths[0] = bad
        full.n[0] = n
        o, lse = full.attend()
        assert int(full.status) == BAD_PAGE
        full.check(o, lse)


@pytest.mark.gpu
def test_not_a_number_is_seen_where_it_is_and_nowhere_else():
    for where in range(2):
        c = Case([500, 500, 2000], 8, 2, 128, 32)
        k, v = c.pool.get(c.pages[1], [77])
        (k, v)[where][0, 1, 5] = math.nan
        c.pool.put(c.pages[1], [77], k, v)
        o, lse = c.attend()
        bad = torch.zeros_like(o, dtype=torch.bool)
        bad[1, 4:, slice(None) if where == 0 else 5] = True
        assert torch.equal(torch.isnan(o), bad)
        assert torch.equal(torch.isnan(lse)[1], torch.tensor([False] * 4 + [where == 0] * 4, device="cuda")) and not torch.isnan(lse[[0, 2]]).any()
        c.check(o, lse, rows=[0, 2])
    c.q[2, 3, 9] = math.nan
    o, _ = c.attend()
    assert torch.isnan(o[2, 3]).all() and not torch.isnan(o[2, [0, 1, 2, 4, 5, 6, 7]]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("scale,size", [(1.0, 8.0), (0.0884, 1e-3), (3.0, 1.0)])
def test_sharp_and_flat_softmax(scale, size):
    c = Case([3000, 129, 1], 8, 1, 128, 64, scale=scale)
    c.q = (c.q.float() * size).to(torch.bfloat16)
    out = c.weights.clone()
    o, lse = c.attend(weights_out=out)
    c.check(o, lse, weights_out=out, base=c.weights)


@pytest.mark.gpu
def test_queries_lie_apart_and_the_table_is_part_of_a_wider_one():
    c = Case([200, 3, 1000, 64, 65], 12, 4, 64, 16)
    wide = torch.randn((5, 12 + 8, 64), device="cuda").to(torch.bfloat16)
    wide[:, :12] = c.q
    table = torch.full((5, c.per_row + 9), -7, dtype=torch.int32, device="cuda")
    table[:, 3:3 + c.per_row] = c.table
    cache = binding.make_paged(c.shape, c.pool.data, table[:, 3:3 + c.per_row], c.lengths)
    o, lse = c.attend(cache=cache, q=wide[:, :12])
    c.check(o, lse)
    out = torch.full((5, 4, c.per_row * 16), 5.0, device="cuda")
    o2, _ = c.attend(cache=cache, weights_out=out)                       # weights that begin from nothing
    assert torch.equal(o, o2)
    base = torch.zeros_like(out)
    for r, n in enumerate(c.n):
        base[r, :, n:] = 5.0
    c.check(o, lse, weights_out=out, base=base)


@pytest.mark.gpu
def test_more_rows_than_one_launch_takes():
    rng = random.Random(5)
    c = Case([rng.choice([0, 1, 30, 64, 100, 200]) for _ in range(2100)], 4, 2, 64, 32)
    out = c.weights.clone()
    o, lse = c.attend(weights_out=out)
    c.check(o, lse, weights_out=out, base=c.weights, rows=list(range(0, 2100, 37)) + [1023, 1024, 2047, 2048, 2099])


@pytest.mark.gpu
def test_slots_beyond_32_bits_of_bytes():
    """One row whose pages lie more than 2^32 bytes apart in the pool."""
    d, bt, hkv = 128, 64, 8
    block = hkv * 2 * bt * d * 2
    blocks = (5 << 30) // block
    c = Case([700], 8, hkv, d, bt, per_row=11, spare=0)
    pool = torch.empty(blocks * block, dtype=torch.uint8, device="cuda")
    table = c.table.clone()
    for j in range(11):
        at = (blocks - 1) - j * (blocks // 11)
        pool.view(blocks, block)[at].copy_(c.pool.data[int(c.table[0, j])].view(torch.uint8).view(-1))
        table[0, j] = at
    cache = binding.make_paged(c.shape, pool, table, c.lengths)
    o, lse = c.attend(cache=cache)
    c.check(o, lse)


@pytest.mark.gpu
def test_a_batch_without_rows():
    sh = shape_of(4, 2, 64, 64)
    pool = torch.zeros((3, 2, 2, 64 * 64), dtype=torch.bfloat16, device="cuda")
    empty = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    c = binding.make_paged(sh, pool, empty(0, 3, t=torch.int32), empty(0, t=torch.int32), empty(0, 2, 192), empty(0, 2, 192, t=torch.int32))
    scratch = empty(max(256, binding.ipkv_paged_scratch_bytes(sh, c)), t=torch.uint8)
    binding.ipkv_paged_append(sh, c, empty(0, 2, 64, t=torch.bfloat16), empty(0, 2, 64, t=torch.bfloat16), positions=empty(0, t=torch.int32))
    binding.ipkv_paged_attend(sh, c, empty(0, 4, 64, t=torch.bfloat16), scratch, empty(0, 4, 64), empty(0, 4))
    binding.ipkv_paged_evict(sh, c, 10, 0, 0, scratch)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_the_same_call_gives_the_same_bits_and_runs_on_its_stream():
    c = Case([3000, 100, 5000, 0, 64, 2048], 32, 8, 128, 16)
    first = c.attend(weights_out=c.weights.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(side):
            again = c.attend()
        side.synchronize()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    given = c.attend(stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(first[0], given[0])


@pytest.mark.gpu
def test_partials_join_with_the_other_operators():
    """The pages hold the newer part of a sequence, a run of blocks the older one; merged, they are attention over both."""
    from paper_2609_14507_b200 import synth
    c = Case([900, 300], 8, 2, 128, 64)
    o1, l1 = c.attend()
    n_old, bb = 500, binding.ipkv_block_bytes(c.shape)
    k_old, v_old = torch.randn((n_old, 2, 128), device="cuda").to(torch.bfloat16), torch.randn((n_old, 2, 128), device="cuda").to(torch.bfloat16)
    run = torch.zeros(-(-n_old // 64) * bb, dtype=torch.uint8, device="cuda")
    binding.ipkv_pack_blocks(c.shape, binding.LAYOUT_TILE, k_old, v_old, n_old, run)
    o2, l2 = torch.empty_like(o1), torch.empty_like(l1)
    scratch = torch.empty(binding.ipkv_attend_scratch_bytes(c.shape, 2, 2, 2 * n_old), dtype=torch.uint8, device="cuda")
    binding.ipkv_attend_runs(c.shape, [[(run, n_old)], [(run, n_old)]], c.q, scratch, o2, l2)
    o, lse = torch.empty((16, 128), device="cuda"), torch.empty(16, device="cuda")
    m = binding.lib().ipkv_merge(None, 16, 128, 2, (C.c_void_p * 2)(o1.data_ptr(), o2.data_ptr()), (C.c_void_p * 2)(l1.data_ptr(), l2.data_ptr()), o.data_ptr(), 0,
                                 lse.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert m == 0 and synth is not None
    for r in range(2):
        k, v = c.pool.get(c.pages[r], list(range(c.n[r])))
        eo, el, *_ = ref.attend(c.q[r], torch.cat([k_old, k]), torch.cat([v_old, v]), c.scale)
        # the other operator holds weights to 16 bits
        assert (o.view(2, 8, 128)[r] - eo).abs().max() <= 2e-3 and (lse.view(2, 8)[r] - el).abs().max() <= 1e-3


# ---- append ----------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,bt", [(1, 64, 16), (8, 128, 64), (3, 128, 32), (40, 64, 128)])
def test_append_writes_its_tokens_and_nothing_else(hkv, d, bt):
    for new, before in (([1, 1, 1, 1], [0, 5, bt - 1, 2 * bt]), ([5, 0, 3 * bt + 1, 1], [0, 7, bt - 1, bt])):
        n = [a + b for a, b in zip(new, before)]
        c = Case(n, hkv, hkv, d, bt, per_row=-(-max(n) // bt) + 1)
        decode = new == [1, 1, 1, 1]
        total, pad = sum(new), 0 if decode else 3                        # tokens behind the last row's
        k, v = torch.randn((total + pad, hkv, d), device="cuda").to(torch.bfloat16), torch.randn((total + pad, hkv, 2 * d), device="cuda").to(torch.bfloat16)
        v = v[..., :d].contiguous() if hkv == 1 else torch.cat([v[..., :d], v[..., d:]], 1)[:, :hkv]          # rows twice as far apart
        at = torch.randint(0, 1 << 30, (total + pad,), dtype=torch.int32, device="cuda")
        start = None if decode else torch.tensor([0] + [sum(new[:i + 1]) for i in range(4)], dtype=torch.int32, device="cuda")
        want, w, pos = ref.Pool.__new__(ref.Pool), c.weights.clone(), c.positions.clone()
        want.__dict__.update(c.pool.__dict__, data=c.pool.data.clone())
        i = 0
        for r in range(4):
            slots = list(range(before[r], n[r]))
            if slots:
                want.put(c.pages[r], slots, k[i:i + new[r]], v[i:i + new[r]])
                w[r][:, slots] = 0.0
                pos[r][:, slots] = at[i:i + new[r]]
            i += new[r]
        binding.ipkv_paged_append(c.shape, c.cache(), k, v, positions=at, row_start=start, status=c.status)
        assert torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16))
        assert torch.equal(c.weights, w) and torch.equal(c.positions, pos) and int(c.status) == 0
        binding.ipkv_paged_append(c.shape, c.cache(False, False), k, v, row_start=start)       # a cache without the arrays
        assert torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16)) and torch.equal(c.weights, w)


@pytest.mark.gpu
def test_append_leaves_out_what_has_no_place():
    c = Case([0, 3, 64, 65, 70], 4, 2, 64, 64, per_row=2)
    before = c.pool.data.clone()
    k = torch.randn((5, 2, 64), device="cuda").to(torch.bfloat16)
    at = torch.arange(5, dtype=torch.int32, device="cuda")
    c.table[1, 0] = -1                                                   # a page that is not there
    c.table[2, 0] = c.pool.data.shape[0]
    c.lengths[3] = 2 * 64 + 1                                            # more slots than the table has
    w = c.weights.clone()
    binding.ipkv_paged_append(c.shape, c.cache(), k, k, positions=at, status=c.status)
    assert int(c.status) == BAD_PAGE
    want = ref.Pool.__new__(ref.Pool)
    want.__dict__.update(c.pool.__dict__, data=before)
    want.put(c.pages[4], [69], k[4:], k[4:])
    w[4][:, 69] = 0.0
    assert torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16)) and torch.equal(c.weights, w)
    # an empty row takes no token and is no mistake; of three tokens a length of two counts the last two
    c.status.zero_()
    c = Case([0, 2], 4, 2, 64, 64)
    want.__dict__.update(c.pool.__dict__, data=c.pool.data.clone())
    want.put(c.pages[1], [0, 1], k[2:4], k[2:4])
    binding.ipkv_paged_append(c.shape, c.cache(), k[:4].contiguous(), k[:4].contiguous(), positions=at[:4], row_start=torch.tensor([0, 1, 4], dtype=torch.int32, device="cuda"),
                              status=c.status)
    assert int(c.status) == 0 and torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16))


# ---- eviction --------------------------------------------------------------------------------------------------------

def check_evict(c, budget, first, recent, in_place, kept_too=True):
    w, pos, data = c.weights.clone(), c.positions.clone(), c.pool.data.clone()
    cache = c.cache()
    scratch = torch.randint(0, 256, (max(256, binding.ipkv_paged_evict_scratch_bytes(c.shape, cache, budget)),), dtype=torch.uint8, device="cuda")
    wo, po = (None, None) if in_place else (torch.full_like(w, -9.0), torch.full_like(pos, -9))
    kept = torch.full((len(c.n), c.hkv, budget), -9, dtype=torch.int32, device="cuda") if kept_too else None
    binding.ipkv_paged_evict(c.shape, cache, budget, first, recent, scratch, wo, po, kept, status=c.status)
    assert int(c.status) == 0
    want = ref.Pool.__new__(ref.Pool)
    want.__dict__.update(c.pool.__dict__, data=data.clone())
    old = ref.Pool.__new__(ref.Pool)
    old.__dict__.update(c.pool.__dict__, data=data)
    ww, wp = (w.clone(), pos.clone()) if in_place else (torch.full_like(w, -9.0), torch.full_like(pos, -9))
    wk = torch.full((len(c.n), c.hkv, budget), -9, dtype=torch.int32)
    for r, n in enumerate(c.n):
        if n == 0:
            continue
        for h in range(c.hkv):
            src = ref.kept(w[r, h, :n].tolist(), pos[r, h, :n].tolist(), budget, first, recent)
            wk[r, h, :len(src)] = torch.tensor(src, dtype=torch.int32)
            at = torch.tensor(src, device="cuda")
            ww[r, h, :len(src)], wp[r, h, :len(src)] = w[r, h][at], pos[r, h][at]
            moved = [i for i, s in enumerate(src) if i != s]
            if moved:
                k, v = want.get(c.pages[r], moved)
                k0, v0 = old.get(c.pages[r], [src[i] for i in moved])
                k[:, h], v[:, h] = k0[:, h], v0[:, h]
                want.put(c.pages[r], moved, k, v)
    wo, po = (c.weights, c.positions) if in_place else (wo, po)
    assert kept is None or torch.equal(kept.cpu(), wk)
    assert torch.equal(wo.view(torch.int32), ww.view(torch.int32)) and torch.equal(po, wp)
    assert torch.equal(c.pool.data.view(torch.int16), want.data.view(torch.int16))
    if not in_place:
        assert torch.equal(c.weights.view(torch.int32), w.view(torch.int32)) and torch.equal(c.positions, pos)


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,bt", [(1, 64, 16), (4, 128, 64), (2, 64, 256)])
@pytest.mark.parametrize("lengths,budget,first,recent", [([1], 1, 0, 0), ([2, 1, 0], 1, 0, 0), ([2, 3], 1, 0, 1), ([100, 99, 101, 100], 99, 4, 10), ([65, 64, 300], 64, 0, 64),
                                                         ([3000, 500, 0, 2999], 500, 4, 200), ([3000, 2000], 2500, 100, 0), ([5000], 4999, 0, 1), ([9000], 17, 8, 9),
                                                         ([700] * 50, 100, 3, 30)])
def test_eviction_keeps_what_it_says(hkv, d, bt, lengths, budget, first, recent):
    c = Case(lengths, hkv, hkv, d, bt)
    c.weights[:] = torch.exp(4 * torch.randn_like(c.weights))
    check_evict(c, budget, first, recent, in_place=False)
    check_evict(c, budget, first, recent, in_place=True, kept_too=False)


@pytest.mark.gpu
def test_eviction_with_one_array_in_place_and_one_apart():
    for lengths, budget in (([1000, 200, 513], 200), ([201, 200, 0], 200), ([230000], 150000)):
        for which in range(2):
            c = Case(lengths, 1, 1, 64, 256)
            w, pos = c.weights.clone(), c.positions.clone()
            both = [torch.full_like(w, -9.0), torch.full_like(pos, -9)]
            kept = torch.full((len(lengths), 1, budget), -9, dtype=torch.int32, device="cuda")
            cache = c.cache()
            scratch = torch.zeros(max(256, binding.ipkv_paged_evict_scratch_bytes(c.shape, cache, budget)), dtype=torch.uint8, device="cuda")
            binding.ipkv_paged_evict(c.shape, cache, budget, 3, 50, scratch, both[0] if which == 0 else None, both[1] if which == 1 else None, kept, status=c.status)
            assert int(c.status) == 0
            for r, n in enumerate(lengths):
                if n == 0:
                    continue
                src = torch.tensor(ref.kept(w[r, 0, :n].tolist(), pos[r, 0, :n].tolist(), budget, 3, 50), device="cuda")
                assert torch.equal(kept[r, 0, :len(src)].long(), src)
                got_w, got_pos = both[0] if which == 0 else c.weights, both[1] if which == 1 else c.positions
                assert torch.equal(got_w[r, 0, :len(src)], w[r, 0][src]) and torch.equal(got_pos[r, 0, :len(src)], pos[r, 0][src])


@pytest.mark.gpu
def test_a_budget_that_nothing_exceeds_needs_no_scratch():
    c = Case([128, 5, 0], 2, 2, 64, 64)
    cache = c.cache()
    assert binding.ipkv_paged_evict_scratch_bytes(c.shape, cache, 128) == 0
    before = [x.clone() for x in (c.pool.data, c.weights, c.positions)]
    binding.ipkv_paged_evict(c.shape, cache, 128, 4, 100, torch.empty(0, dtype=torch.uint8, device="cuda"), status=c.status)
    torch.cuda.synchronize()
    for x, y in zip((c.pool.data, c.weights, c.positions), before):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.gpu
def test_eviction_by_hard_weights():
    """Ties (the lower slot stays), nothing but ties, zeros of both signs, infinities, NaN, negative and subnormal weights, twice the same position."""
    for seed, values in enumerate(([1.0], [0.0, -0.0], [1.0, 2.0], [math.nan], [math.nan, 1.0, -1.0], [math.inf, -math.inf, 0.0, math.nan], [1e-45, -1e-45, 0.0, 1e-40],
                                   [-3.0, -3.0000002, 5.0, 5.0000005])):
        c = Case([1000, 257, 40, 800], 2, 2, 64, 16, seed=seed)
        c.weights[:] = torch.tensor(values, device="cuda")[torch.randint(0, len(values), c.weights.shape, device="cuda")]
        check_evict(c, 200, 4, 16, in_place=bool(seed % 2))
    c = Case([1000, 900], 2, 2, 64, 16)
    c.positions.fill_(3)                                                 # every token is recent, and a first one
    check_evict(c, 100, 10, 10, in_place=True)
    c.positions.random_(-2 ** 31, 2 ** 31 - 1)
    check_evict(c, 100, 10, 10, in_place=False)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,hkv", [([30000, 29001], 2), ([230001], 1)])
def test_eviction_of_long_rows(lengths, hkv):
    """More keys than the CTAs of a row hold at once, too."""
    for budget in (lengths[-1] - 1, 5000):
        c = Case(lengths, hkv, hkv, 64, 256)
        check_evict(c, budget, 4, 1000, in_place=False)


@pytest.mark.gpu
def test_eviction_leaves_bad_pages_alone():
    c = Case([300, 300], 2, 2, 64, 64)
    c.table[0, 3] = c.pool.data.shape[0] + 1
    before = c.pool.data.clone()
    cache = c.cache()
    scratch = torch.zeros(binding.ipkv_paged_evict_scratch_bytes(c.shape, cache, 100), dtype=torch.uint8, device="cuda")
    binding.ipkv_paged_evict(c.shape, cache, 100, 0, 0, scratch, status=c.status)
    assert int(c.status) == BAD_PAGE
    own = set(c.pages[0, :2].tolist()) | set(c.pages[1, :2].tolist())    # the pages of slots below the budget
    for b in range(before.shape[0]):
        assert b in own or torch.equal(c.pool.data[b].view(torch.int16), before[b].view(torch.int16))


# ---- together --------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
def test_a_captured_decode_run_of_bounded_caches():
    """Prompts go in, then a step (append, attention that weighs, eviction, lengths) is captured once and replayed: rows grow to their budget and
    stay there, one ends and another begins in its place.  Every step's attention and, at the end, every slot against a cache kept as lists."""
    torch.manual_seed(11)
    hq, hkv, d, bt, budget, first, recent = 8, 2, 64, 16, 90, 2, 20
    rows, per_row = 3, -(-(budget + 1) // bt)
    c = Case([per_row * bt] * rows, hq, hkv, d, bt)
    c.lengths.zero_()
    c.weights.zero_()
    cache, g = c.cache(), hq // hkv
    prompts = [60, 89, 5]
    start = torch.tensor([0, 60, 149, 154], dtype=torch.int32, device="cuda")
    k, v = torch.randn((154, hkv, d), device="cuda").to(torch.bfloat16), torch.randn((154, hkv, d), device="cuda").to(torch.bfloat16)
    at = torch.cat([torch.arange(n, dtype=torch.int32) for n in prompts]).cuda()
    c.lengths.copy_(torch.tensor(prompts))
    binding.ipkv_paged_append(c.shape, cache, k, v, positions=at, row_start=start)
    # the cache as lists: per row and head the slots' tokens, their positions and weights
    tokens = [[[(k[i, h], v[i, h]) for i in range(int(start[r]), int(start[r + 1]))] for h in range(hkv)] for r in range(rows)]
    pos = [[list(range(n)) for _ in range(hkv)] for n in prompts]
    weight = [[[0.0] * n for _ in range(hkv)] for n in prompts]

    kn, vn, qn = (torch.zeros((rows, h, d), dtype=torch.bfloat16, device="cuda") for h in (hkv, hkv, hq))
    pn = torch.zeros(rows, dtype=torch.int32, device="cuda")
    o, lse = torch.empty((rows, hq, d), device="cuda"), torch.empty((rows, hq), device="cuda")
    s1 = torch.empty(binding.ipkv_paged_scratch_bytes(c.shape, cache, weigh=True), dtype=torch.uint8, device="cuda")
    s2 = torch.empty(binding.ipkv_paged_evict_scratch_bytes(c.shape, cache, budget), dtype=torch.uint8, device="cuda")
    active = torch.ones(rows, dtype=torch.int32, device="cuda")

    def step():
        c.lengths.add_(active)
        binding.ipkv_paged_append(c.shape, cache, kn, vn, positions=pn, status=c.status)
        binding.ipkv_paged_attend(c.shape, cache, qn, s1, o, lse, weights_out=c.weights, status=c.status)
        binding.ipkv_paged_evict(c.shape, cache, budget, first, recent, s2, status=c.status)
        c.lengths.clamp_(max=budget)

    saved = [x.clone() for x in (c.lengths, c.weights, c.positions, c.pool.data)]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((c.lengths, c.weights, c.positions, c.pool.data), saved):
        x.copy_(y)
    n_pos = list(prompts)
    for i in range(60):
        if i == 30:                                      # row 1 ends; a new sequence begins in its slots, empty
            c.lengths[1] = 0
            tokens[1], pos[1], weight[1], n_pos[1] = [[] for _ in range(hkv)], [[] for _ in range(hkv)], [[] for _ in range(hkv)], 0
        idle = i in (31, 32)
        active[2] = 0 if idle else 1                     # a row without a sequence takes no part
        if idle:
            held = c.lengths[2].clone()
            c.lengths[2] = 0
        for x in (kn, vn, qn):
            x.copy_(torch.randn(x.shape, device="cuda"))
        pn.copy_(torch.tensor(n_pos, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert int(c.status) == 0
        for r in range(rows):
            if idle and r == 2:
                assert (o[r] == 0).all() and torch.isneginf(lse[r]).all()
                continue
            for h in range(hkv):
                tokens[r][h].append((kn[r, h].clone(), vn[r, h].clone()))
                pos[r][h].append(n_pos[r])
                weight[r][h].append(0.0)
                kk, vv = (torch.stack([t[j] for t in tokens[r][h]])[:, None] for j in range(2))
                eo, el, ep, to, tl, tp = ref.attend(qn[r, h * g:(h + 1) * g], kk, vv, c.scale)
                assert (o[r, h * g:(h + 1) * g].double() - eo).abs().le(to).all() and (lse[r, h * g:(h + 1) * g].double() - el).abs().le(tl).all()
                weight[r][h] = [a + b for a, b in zip(weight[r][h], ep.sum(0).tolist())]
                # the choice hangs on the last digits of a weight only where two are that close, which random ones of this seed are not
                src = ref.kept(weight[r][h], pos[r][h], budget, first, recent)
                n = len(src)
                assert c.positions[r, h, :n].tolist() == [pos[r][h][s] for s in src]
                assert torch.allclose(c.weights[r, h, :n].double().cpu(), torch.tensor([weight[r][h][s] for s in src], dtype=torch.float64), rtol=1e-4, atol=1e-6)
                tokens[r][h], pos[r][h], weight[r][h] = ([x[s] for s in src] for x in (tokens[r][h], pos[r][h], weight[r][h]))
            n_pos[r] += 1
        if idle:
            c.lengths[2] = held
    for r in range(rows):
        assert int(c.lengths[r]) == len(tokens[r][0])
        kk, vv = c.pool.get(c.pages[r], list(range(len(tokens[r][0]))))
        for h in range(hkv):
            assert torch.equal(kk[:, h], torch.stack([t[0] for t in tokens[r][h]])) and torch.equal(vv[:, h], torch.stack([t[1] for t in tokens[r][h]]))


@pytest.mark.gpu
def test_calls_of_two_threads():
    """Two host threads, a stream, a cache and scratch of their own each."""
    import threading
    cases = [Case([3000, 64, 777], 8, 2, 128, 64, seed=1), Case([100, 5000, 9], 16, 1, 64, 32, seed=2)]
    torch.cuda.synchronize()
    outs, faults = [None, None], []

    def work(i):
        try:
            c, s = cases[i], torch.cuda.Stream()
            with torch.cuda.stream(s):
                cache = c.cache()
                scratch = torch.empty(binding.ipkv_paged_scratch_bytes(c.shape, cache), dtype=torch.uint8, device="cuda")
                o, lse = torch.empty((3, c.hq, c.d), device="cuda"), torch.empty((3, c.hq), device="cuda")
                for _ in range(200):
                    binding.ipkv_paged_attend(c.shape, cache, c.q, scratch, o, lse, status=c.status)
            s.synchronize()
            outs[i] = (o, lse)
        except Exception as e:                           # noqa: BLE001
            faults.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not faults
    for c, (o, lse) in zip(cases, outs):
        assert int(c.status) == 0
        c.check(o, lse)


@pytest.mark.gpu
def test_two_graphs_with_scratch_of_their_own_run_at_once():
    a, b = Case([3000, 64, 777], 8, 2, 128, 64, seed=1), Case([100, 5000], 8, 2, 128, 32, seed=2)
    graphs, outs = [], []
    for c in (a, b):
        cache = c.cache()
        scratch = torch.empty(binding.ipkv_paged_scratch_bytes(c.shape, cache), dtype=torch.uint8, device="cuda")
        o, lse = torch.empty((len(c.n), 8, 128), device="cuda"), torch.empty((len(c.n), 8), device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(3):
                binding.ipkv_paged_attend(c.shape, cache, c.q, scratch, o, lse)
        graphs.append((g, cache, scratch))
        outs.append((o, lse))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, (g, *_) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for c, (o, lse) in zip((a, b), outs):
        c.check(o, lse)
