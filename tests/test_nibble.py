"""The cache in 4 bits: refusals (no GPU), the format bit by bit, attention against 64 bits, and a decode run from prompt to merge."""
import numpy as np
import pytest

from paper_2609_14507_b200 import binding, synth
from tests import nibble_ref as ref

torch = pytest.importorskip("torch")
C = binding.C
EINVAL, ENOMEM, ECUDA = 1, 2, 5
BASE = 1 << 30          # an aligned address that nothing reads: the calls below are refused first


def shape_of(hq, hkv, d, bt, scale=0.0, kind=binding.GQA, dv=None):
    return binding.make_shape(kind, hq, hkv, d, d if dv is None else dv, bt, scale)


# ---- refusals --------------------------------------------------------------------------------------------------------

BAD_SHAPES = [shape_of(32, 5, 128, 64), shape_of(32, 4, 96, 64), shape_of(32, 4, 256, 64), shape_of(32, 4, 128, 32), shape_of(32, 4, 128, 96),
              shape_of(32, 4, 128, 0), shape_of(0, 4, 128, 64), shape_of(32, 0, 128, 64), shape_of(32, 4, 128, 64, dv=64),
              shape_of(16, 1, 576, 64, kind=binding.MLA, dv=512), shape_of(32, 4, 128, -64)]


@pytest.mark.parametrize("sh", BAD_SHAPES)
def test_shapes_without_the_format_are_refused(sh):
    L = binding.lib()
    assert L.ipkv_nibble_block_bytes(C.byref(sh)) == -1
    spans = (binding.Span * 1)(binding.Span(BASE, 0, 1))
    assert L.ipkv_nibble_pack(C.byref(sh), 1, spans, 1, BASE, BASE, 0, 0, None) == EINVAL
    assert L.ipkv_nibble_unpack(C.byref(sh), 1, spans, 1, BASE, BASE, 0, 0, None) == EINVAL
    n = C.c_size_t()
    assert L.ipkv_nibble_scratch_bytes(C.byref(sh), 1, 1, C.byref(n)) == EINVAL
    runs, start = (binding.Run * 1)(binding.Run(BASE, 5)), (C.c_int32 * 2)(0, 1)
    assert L.ipkv_nibble_attend(C.byref(sh), 1, runs, start, BASE, BASE, 1 << 40, BASE, BASE, None, None) == EINVAL
    with pytest.raises(binding.IpkvError):
        binding.ipkv_nibble_block_bytes(sh)


def test_block_bytes():
    assert binding.ipkv_nibble_block_bytes(shape_of(32, 4, 128, 64)) == 4 * 8960 == ref.block_bytes(4, 128, 64)
    assert binding.ipkv_nibble_block_bytes(shape_of(12, 4, 64, 256)) == 4 * 4 * 4608 == ref.block_bytes(4, 64, 256)


def move(fn, sh, spans, k=BASE, v=BASE, ks=0, vs=0, n=None, tokens=None):
    arr = (binding.Span * max(1, len(spans)))(*[binding.Span(*s) for s in spans])
    return fn(C.byref(sh), len(spans) if n is None else n, arr, sum(s[2] for s in spans) if tokens is None else tokens, k, v, ks, vs, None)


@pytest.mark.parametrize("name", ["ipkv_nibble_pack", "ipkv_nibble_unpack"])
def test_bad_spans_are_refused(name):
    fn, sh = getattr(binding.lib(), name), shape_of(32, 4, 128, 64)
    for spans in ([(None, 0, 1)], [(BASE + 8, 0, 1)], [(BASE, -1, 1)], [(BASE, 0, -1)], [(BASE, 1 << 37, 1)], [(BASE, 0, (1 << 31) - 1)]):
        assert move(fn, sh, spans) == EINVAL
    ok = [(BASE, 5, 3)]
    assert move(fn, sh, ok, k=None) == EINVAL and move(fn, sh, ok, v=None) == EINVAL
    assert move(fn, sh, ok, k=BASE + 2) == EINVAL and move(fn, sh, ok, v=BASE + 8) == EINVAL
    assert move(fn, sh, ok, ks=504) == EINVAL and move(fn, sh, ok, vs=-512) == EINVAL and move(fn, sh, ok, ks=516) == EINVAL
    assert move(fn, sh, ok, n=-1) == EINVAL
    assert move(fn, sh, ok, tokens=2) == EINVAL and move(fn, sh, ok, tokens=4) == EINVAL
    assert fn(C.byref(sh), 1, None, 1, BASE, BASE, 0, 0, None) == EINVAL
    assert move(fn, sh, []) == 0 and move(fn, sh, [(BASE, 3, 0), (None, 0, 0)], k=None, v=None) == 0      # nothing to do


def test_spans_of_a_write_that_touch_the_same_block_are_refused():
    fn = binding.lib().ipkv_nibble_pack
    sh = shape_of(32, 4, 128, 128)
    bb = binding.ipkv_nibble_block_bytes(sh)
    far = BASE + 100 * bb
    assert move(fn, sh, [(BASE, 5, 1), (BASE, 5, 1)]) == EINVAL                       # the same token twice
    assert move(fn, sh, [(BASE, 5, 1), (far, 0, 9), (BASE, 7, 1)]) == EINVAL          # two tokens of a block
    assert move(fn, sh, [(BASE, 0, 200), (BASE + bb, 100, 5)]) == EINVAL              # by way of another first block
    assert move(fn, sh, [(BASE, 0, 1), (BASE + 16, 0, 1)]) == EINVAL                  # runs that lie across one another
    if not torch.cuda.is_available():                                                 # what is refused for the missing GPU alone
        assert move(fn, sh, [(BASE, 0, 128), (BASE, 128, 1), (far, 0, 9)]) == ECUDA
        assert move(binding.lib().ipkv_nibble_unpack, sh, [(BASE, 5, 1), (BASE, 5, 1)]) == ECUDA


def attend_rc(sh, runs, start, q=BASE, scratch=BASE, nbytes=1 << 40, o=BASE, lse=BASE, status=None, rows=None):
    r = (binding.Run * max(1, len(runs)))(*[binding.Run(*x) for x in runs])
    s = (C.c_int32 * len(start))(*start)
    return binding.lib().ipkv_nibble_attend(C.byref(sh), len(start) - 1 if rows is None else rows, r, s, q, scratch, nbytes, o, lse, status, None)


def test_bad_attention_calls_are_refused():
    sh = shape_of(32, 4, 128, 64)
    good = dict(runs=[(BASE, 100), (BASE, 5)], start=[0, 1, 2])
    for kw in (dict(q=None), dict(q=BASE + 8), dict(scratch=None), dict(scratch=BASE + 128), dict(o=None), dict(o=BASE + 4), dict(lse=None),
               dict(lse=BASE + 2), dict(status=BASE + 2), dict(rows=0), dict(rows=-1), dict(start=[0, 2, 1]), dict(start=[-1, 1, 2]),
               dict(runs=[(BASE, -1), (BASE, 5)]), dict(runs=[(None, 1), (BASE, 5)]), dict(runs=[(BASE + 4, 1), (BASE, 5)]),
               dict(runs=[(BASE, (1 << 31) - 1), (BASE, 5)])):
        assert attend_rc(sh, **{**good, **kw}) == EINVAL, kw
    for scale in (-1.0, float("nan"), float("inf")):
        assert attend_rc(shape_of(32, 4, 128, 64, scale), **good) == EINVAL
    # more tiles than the kernel counts: 2^31 units
    wide = shape_of(32, 32, 128, 64)
    assert attend_rc(wide, runs=[(BASE, (1 << 31) - 129)] * 3, start=[0, 3]) == EINVAL
    n = C.c_size_t()
    L = binding.lib()
    assert L.ipkv_nibble_scratch_bytes(C.byref(sh), 2, 2, C.byref(n)) == 0
    assert attend_rc(sh, **good, nbytes=n.value - 1) == ENOMEM
    assert L.ipkv_nibble_scratch_bytes(C.byref(sh), -1, 2, C.byref(n)) == EINVAL
    assert L.ipkv_nibble_scratch_bytes(C.byref(sh), 2, 2, None) == EINVAL


def test_the_binding_refuses_other_types_and_shapes():
    sh = shape_of(4, 2, 64, 64)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    for spans, a, b in [([(BASE, 0, 2)], k, k), ([(BASE, 0, 3)], k.float(), k), ([(BASE, 0, 3)], k, k[:2]), ([(BASE, 0, 3)], k, k[..., :32]),
                        ([(BASE, 0, 3)], k.transpose(0, 1).contiguous().transpose(0, 1), k), (np.zeros((1, 3), np.int32), k, k),
                        ([(BASE, 0, 3)], k[:1].expand(3, 2, 64), k)]:
        with pytest.raises(ValueError):
            binding.ipkv_nibble_pack(sh, spans, a, b)
    q, o, lse = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 64)), torch.zeros((2, 4))
    runs, start, w = np.array([[BASE, 3], [BASE, 1]], np.int64), np.array([0, 1, 2], np.int32), torch.zeros(1 << 20, dtype=torch.uint8)
    for a in [(runs, start, q.float(), w, o, lse), (runs, start, q[:1], w, o, lse), (runs, start, q, w, o.bfloat16(), lse),
              (runs, start, q, w, o, lse.double()), (runs[:1], start, q, w, o, lse), (runs, start.astype(np.int64), q, w, o, lse),
              (runs.astype(np.int32), start, q, w, o, lse), (runs, start, q, w, o.transpose(0, 1).contiguous().transpose(0, 1), lse)]:
        with pytest.raises(ValueError):
            binding.ipkv_nibble_attend(sh, *a)


# ---- the format ------------------------------------------------------------------------------------------------------

def hard_values(rng, n, hkv, d):
    """Normal values among rows that are constant, zero, tiny, huge, of one sign, with an outlier, on a coarse grid (many ties)."""
    x = rng.standard_normal((n, hkv, d)).astype(np.float32)
    for i in range(n):
        kind = i % 9
        if kind == 1: x[i] = np.float32(1.5)
        elif kind == 2: x[i] = 0
        elif kind == 3: x[i] *= np.float32(1e-30)
        elif kind == 4: x[i] *= np.float32(1e30)
        elif kind == 5: x[i] = np.abs(x[i]) + 3
        elif kind == 6: x[i, :, 7] = 40
        elif kind == 7: x[i] = np.round(x[i] * 4) / 4
        elif kind == 8: x[i] = x[i] * np.float32(1e-38)                  # scales at and below the smallest normal number
    return synth.f32_to_bf16_bits(x)


FORMAT_CASES = [  # hkv, d, bt, (first, n) of every run
    (1, 128, 64, [(0, 1)]), (2, 64, 64, [(63, 1)]), (4, 128, 128, [(64, 64)]), (3, 64, 128, [(5, 200), (0, 0), (127, 2)]),
    (2, 128, 64, [(0, 64), (10, 1), (33, 95)]), (1, 64, 256, [(255, 1), (250, 20)]), (8, 128, 64, [(i * 7, 1) for i in range(20)]),
    (2, 64, 64, [(i, 1) for i in range(100)]), (1, 128, 64, [(i % 64, 1 + i % 3) for i in range(130)])]


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,d,bt,spans", FORMAT_CASES)
def test_pack_writes_the_format_bit_by_bit_and_unpack_reads_it(hkv, d, bt, spans):
    rng = np.random.default_rng(hkv * 1000 + d + bt)
    sh = shape_of(hkv, hkv, d, bt)
    n = sum(c for _, c in spans)
    k, v = hard_values(rng, n, hkv, d), hard_values(rng, n, hkv, d)
    bb = ref.block_bytes(hkv, d, bt)
    sizes = [-(-(f + c) // bt) * bb for f, c in spans]
    at = np.concatenate([[0], np.cumsum(sizes)])
    image = rng.integers(0, 256, int(at[-1]) + bb, dtype=np.uint8)       # other tokens' codes, and a block behind the last
    buf = torch.from_numpy(image.copy()).cuda()
    src = 0
    for i, (f, c) in enumerate(spans):
        ref.write(image[at[i]:at[i] + sizes[i]], hkv, d, bt, f, k[src:src + c], v[src:src + c])
        src += c
    table = [(buf.data_ptr() + int(at[i]), f, c) for i, (f, c) in enumerate(spans)]
    # K a view of a wider buffer, V dense
    wide = torch.zeros((n, hkv * d + 8), dtype=torch.bfloat16, device="cuda")
    kd = wide[:, :hkv * d].unflatten(1, (hkv, d))
    kd.copy_(synth.bits_to_torch(k))
    vd = synth.bits_to_torch(v, "cuda")
    binding.ipkv_nibble_pack(sh, table, kd, vd)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(buf.cpu().numpy(), image)
    ko, vo = torch.zeros_like(wide), torch.zeros_like(vd)
    binding.ipkv_nibble_unpack(sh, table, ko[:, :hkv * d].unflatten(1, (hkv, d)), vo)
    torch.cuda.synchronize()
    kv, vv = ref.quantised_values(k, v)
    assert np.array_equal(ko[:, :hkv * d].cpu().view(torch.int16).numpy().view(np.uint16).reshape(k.shape), synth.f32_to_bf16_bits(kv.astype(np.float32)))
    assert np.array_equal(synth.torch_bits(vo), synth.f32_to_bf16_bits(vv.astype(np.float32)))
    assert not ko[:, hkv * d:].any()                                     # the columns behind the heads stay
    np.testing.assert_array_equal(buf.cpu().numpy(), image)


@pytest.mark.gpu
def test_codes_are_the_rounded_quotients():
    """Ties and near-ties: every code of a million random groups equals the one that a correctly rounded division gives."""
    rng = np.random.default_rng(5)
    n, d = 8192, 64
    x = rng.standard_normal((n, 1, d)).astype(np.float32) * np.exp2(rng.integers(-30, 30, (n, 1, 1))).astype(np.float32)
    x[::2] = np.round(x[::2] / x[::2].max() * 64) / 64
    k = synth.f32_to_bf16_bits(x)
    sh = shape_of(1, 1, d, 64)
    buf = torch.zeros(n // 64 * ref.block_bytes(1, d, 64), dtype=torch.uint8, device="cuda")
    kd = synth.bits_to_torch(k, "cuda")
    binding.ipkv_nibble_pack(sh, [(buf, 0, n)], kd, kd)
    ko, vo = torch.empty_like(kd), torch.empty_like(kd)
    binding.ipkv_nibble_unpack(sh, [(buf, 0, n)], ko, vo)
    want = synth.f32_to_bf16_bits(ref.values(*ref.quantise(k, 64), 64).astype(np.float32))
    np.testing.assert_array_equal(synth.torch_bits(ko), want)
    np.testing.assert_array_equal(synth.torch_bits(vo), want)            # one group of 64 either way


# ---- attention -------------------------------------------------------------------------------------------------------

def tolerance(q_bits, kq, vq, scale, n):
    """How far (O, LSE) may be from 64 bits.  Scores: sums of exact products in fp32; a tensor-core step adds 16 terms and the sum so
    far with errors below 17 * 2^-24 of the terms' magnitudes, four steps a panel, then four fp32 products: 2^-17 of A, the largest
    sum of |terms| of a score (sk |q||code| + |zk| |q|).  A weight is off by twice that relative to the sum, ex2 and the two
    fp16 halves by 2^-21, and the sum over n tokens by 17 * 2^-24 per step of 16 tokens, twice (head and remainder):
    all of it times V, the largest sv * 15 + |zv|."""
    codes, s, z = kq
    s, z = synth.bf16_bits_to_f32(s).astype(np.float64), np.abs(synth.bf16_bits_to_f32(z).astype(np.float64))
    hq, d = q_bits.shape
    q = np.abs(synth.bf16_bits_to_f32(q_bits).astype(np.float64)).reshape(codes.shape[1], -1, d)
    terms = np.einsum("hgd,nhd->hgn", q, codes * s.repeat(64, -1) + z.repeat(64, -1)) * scale
    A = terms.max()
    vs, vz = synth.bf16_bits_to_f32(vq[1]).astype(np.float64), np.abs(synth.bf16_bits_to_f32(vq[2]).astype(np.float64))
    V = (15 * vs + vz).max()
    steps = n / 16 * 2 + 8
    o = V * (2 * A * 2.0 ** -17 + 2.0 ** -20 + steps * 17 * 2.0 ** -24)
    lse = A * 2.0 ** -17 + (n / 16 + 8) * 2.0 ** -23 + 2.0 ** -20
    return o, lse


def fill(rng, sh, rows, spread=1.0, tail_garbage=True):
    """Random tokens for rows (lists of run lengths) in one buffer whose unused bytes are garbage (0xff: codes 15, scales and zeros NaN)."""
    hkv, d, bt = sh.n_kv_heads, sh.dim_qk, sh.block_tokens
    bb = ref.block_bytes(hkv, d, bt)
    total = sum(-(-n // bt) for r in rows for n in r) + 1
    buf = torch.full((total * bb,), 255 if tail_garbage else 0, dtype=torch.uint8, device="cuda")
    at, runs, kvs = 0, [], []
    for r in rows:
        rr, ks, vs = [], [], []
        for n in r:
            k = synth.f32_to_bf16_bits(rng.standard_normal((n, hkv, d)).astype(np.float32) * np.float32(spread))
            k[..., 3::17] = synth.f32_to_bf16_bits(synth.bf16_bits_to_f32(k[..., 3::17]) * np.float32(4))
            v = synth.f32_to_bf16_bits(rng.standard_normal((n, hkv, d)).astype(np.float32) * np.exp2(rng.integers(-3, 4, (n, hkv, 1))).astype(np.float32))
            if n:
                binding.ipkv_nibble_pack(sh, [(buf.data_ptr() + at, 0, n)], synth.bits_to_torch(k, "cuda"), synth.bits_to_torch(v, "cuda"))
            rr.append((buf.data_ptr() + at, n))
            ks.append(k); vs.append(v)
            at += -(-n // bt) * bb
        runs.append(rr)
        kvs.append((np.concatenate(ks) if ks else np.zeros((0, hkv, d), np.uint16), np.concatenate(vs) if vs else np.zeros((0, hkv, d), np.uint16)))
    return buf, runs, kvs


def check(sh, q, kvs, o, lse):
    scale = float(np.float32(sh.softmax_scale if sh.softmax_scale > 0 else sh.dim_qk ** -0.5))
    for r, (k, v) in enumerate(kvs):
        if not k.shape[0]:
            assert not o[r].any() and np.all(np.isneginf(lse[r]))
            continue
        kq, vq = ref.quantise(k, 64), ref.quantise(v, v.shape[-1])
        want_o, want_lse = ref.attend(q[r], ref.values(*kq, 64), ref.values(*vq, v.shape[-1]), scale)
        to, tl = tolerance(q[r], kq, vq, scale, k.shape[0])
        assert np.isfinite(o[r]).all()
        assert np.abs(o[r] - want_o).max() <= to, (r, np.abs(o[r] - want_o).max(), to)
        assert np.all(np.abs(lse[r] - want_lse) <= tl + np.abs(want_lse) * 2.0 ** -22), (r, np.abs(lse[r] - want_lse).max(), tl)


def attend(sh, runs, q, status=None):
    n_rows, n_runs = len(runs), sum(len(r) for r in runs)
    scratch = torch.full((binding.ipkv_nibble_scratch_bytes(sh, n_rows, n_runs),), 255, dtype=torch.uint8, device="cuda")
    o = torch.full((n_rows, sh.n_q_heads, sh.dim_qk), float("nan"), device="cuda")
    lse = torch.full((n_rows, sh.n_q_heads), float("nan"), device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda") if status is None else status
    binding.ipkv_nibble_attend(sh, runs, None, q if isinstance(q, torch.Tensor) else synth.bits_to_torch(q, "cuda"), scratch, o, lse, word)
    torch.cuda.synchronize()
    assert int(word.item()) == 0
    return o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)


ATTEND_CASES = [  # hq, hkv, d, bt, run lengths of every row
    (32, 4, 128, 64, [[1]]),
    (32, 4, 128, 64, [[4097]]),
    (32, 8, 128, 64, [[700, 33], [64], [], [1000, 1, 129]]),
    (8, 8, 128, 64, [[333]]),                    # one query head per KV head
    (6, 3, 64, 128, [[63, 65], [0], [200]]),     # two
    (12, 4, 64, 64, [[1500, 77], [2]]),          # three
    (10, 2, 128, 64, [[90], [640]]),             # five: more than four share no product
    (16, 1, 128, 64, [[450, 70], [5000]]),       # two octets on a tile
    (24, 1, 64, 64, [[1000], [64]]),             # three octets
    (40, 1, 128, 64, [[450]]),                   # five octets
    (32, 1, 64, 64, [[700, 300]]),               # four octets: one team
    (64, 1, 64, 256, [[700, 300]]),              # eight
    (119, 1, 128, 64, [[300], [65]]),            # more than 64: two head groups, the last one smaller
    (32, 4, 128, 256, [[5000, 100], [256]]),
    (4, 1, 64, 64, [[1]] * 200),                 # tables too large to travel with the launch
    (8, 2, 128, 64, [[64] * 150, [1, 64, 3] * 30]),      # pages: runs of one block
    (32, 32, 128, 64, [[20], [19]]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,bt,rows", ATTEND_CASES)
def test_attention_matches_64_bits(hq, hkv, d, bt, rows):
    rng = np.random.default_rng(hq + hkv + d + bt + len(rows))
    sh = shape_of(hq, hkv, d, bt)
    buf, runs, kvs = fill(rng, sh, rows)
    q = synth.normal_bf16(rng, (len(rows), hq, d))
    o, lse = attend(sh, runs, q)
    check(sh, q, kvs, o, lse)
    again = attend(sh, runs, q)
    assert np.array_equal(o, again[0]) and np.array_equal(lse, again[1])         # bit-reproducible


def ragged(n_rows, most, seed):
    rng = np.random.default_rng(seed)
    rows = [[int(x)] for x in rng.integers(0, most, n_rows)]
    rows[0], rows[1], rows[2], rows[-2], rows[-1] = [0], [1, 0, 64], [most], [65], []
    return rows


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,bt,rows", [
    (8, 8, 64, 64, ragged(64, 300, 1)),          # more pairs than CTAs: equal chunks that meet many pairs, tables in the launch
    (32, 4, 64, 64, ragged(130, 200, 2)),        # ... and uploaded
    (16, 8, 128, 128, ragged(60, 3000, 3)),      # chunks that end inside pairs
    (16, 1, 64, 64, ragged(500, 130, 4)),        # two octets a tile
    (4, 1, 64, 64, [[40000]]),                   # one pair, hundreds of partials
    (8, 1, 128, 64, [[40000]]),
    (16, 1, 128, 64, [[40000, 7]]),
    (16, 4, 128, 64, ragged(12, 5000, 5)),       # whole CTAs to ragged pairs
    (24, 2, 64, 64, ragged(30, 1000, 6)),
    (4, 1, 64, 64, ragged(70, 6000, 7)),         # ... their tables uploaded
    (8, 2, 128, 64, ragged(90, 700, 8)),         # one CTA to every pair, tables uploaded
])
def test_attention_however_the_work_is_shared_out(hq, hkv, d, bt, rows):
    rng = np.random.default_rng(len(rows) + hq)
    sh = shape_of(hq, hkv, d, bt)
    buf, runs, kvs = fill(rng, sh, rows)
    q = synth.normal_bf16(rng, (len(rows), hq, d))
    o, lse = attend(sh, runs, q)
    check(sh, q, kvs, o, lse)
    again = attend(sh, runs, q)
    assert np.array_equal(o, again[0]) and np.array_equal(lse, again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["peaked", "rising", "tiny values", "huge values", "scales that grow", "zero queries", "large queries", "one constant"])
def test_attention_on_hard_values(what):
    rng = np.random.default_rng(11)
    hq, hkv, d, n = 16, 2, 128, 1500
    sh = shape_of(hq, hkv, d, 64, 0.125)
    k, v = rng.standard_normal((n, hkv, d)).astype(np.float32), rng.standard_normal((n, hkv, d)).astype(np.float32)
    q = rng.standard_normal((1, hq, d)).astype(np.float32)
    if what == "peaked": k[777] = 6 * np.sign(q[0].reshape(hkv, -1, d).sum(1))
    elif what == "rising": k *= np.linspace(0, 8, n, dtype=np.float32)[:, None, None]    # the reference is raised again and again
    elif what == "tiny values": v *= np.float32(1e-25)
    elif what == "huge values": v *= np.float32(1e25)
    elif what == "scales that grow": v *= np.exp2(np.linspace(-40, 40, n, dtype=np.float32))[:, None, None]
    elif what == "zero queries": q[0, ::3] = 0
    elif what == "large queries": q *= np.float32(300)
    elif what == "one constant": v[:] = np.float32(2.5); k[:] = np.float32(-1.25)
    k, v, q = (synth.f32_to_bf16_bits(x) for x in (k, v, q))
    buf = torch.full((-(-n // 64) * ref.block_bytes(hkv, d, 64),), 255, dtype=torch.uint8, device="cuda")
    binding.ipkv_nibble_pack(sh, [(buf, 0, n)], synth.bits_to_torch(k, "cuda"), synth.bits_to_torch(v, "cuda"))
    o, lse = attend(sh, [[(buf, n)]], q)
    check(sh, q, [(k, v)], o, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("hq", [8, 16, 32])              # heads that share one product, one octet and two
def test_what_is_not_a_number_is_seen_where_it_counts_and_nowhere_else(hq):
    """A NaN in a query makes that head NaN, an infinite key (its group decodes to NaN) its KV head in its row; nothing else changes."""
    hkv, d, n = 2, 128, 700
    rng = np.random.default_rng(hq)
    sh = shape_of(hq, hkv, d, 64)
    k, v = synth.normal_bf16(rng, (2 * n, hkv, d)), synth.normal_bf16(rng, (2 * n, hkv, d))
    q = synth.normal_bf16(rng, (2, hq, d))
    buf = torch.full((2, -(-n // 64) * ref.block_bytes(hkv, d, 64)), 255, dtype=torch.uint8, device="cuda")
    spans, runs = [(buf[0], 0, n), (buf[1], 0, n)], [[(buf[0], n)], [(buf[1], n)]]
    binding.ipkv_nibble_pack(sh, spans, synth.bits_to_torch(k, "cuda"), synth.bits_to_torch(v, "cuda"))
    o, lse = attend(sh, runs, q)
    q[0, 1, 5] = 0x7fc0
    k[n + 333, 1, 70] = 0x7f80
    binding.ipkv_nibble_pack(sh, spans, synth.bits_to_torch(k, "cuda"), synth.bits_to_torch(v, "cuda"))
    o2, lse2 = attend(sh, runs, q)
    hit = np.zeros((2, hq), bool)
    hit[0, 1] = hit[1, hq // 2:] = True
    assert np.isnan(o2[hit]).all() and np.isnan(lse2[hit]).all()
    assert np.array_equal(o2[~hit], o[~hit]) and np.array_equal(lse2[~hit], lse[~hit])


@pytest.mark.gpu
def test_a_run_whose_offsets_pass_32_bits():
    """More than 4 GB in one run: the first and last tokens carry all the weight."""
    hkv, d, bt, n = 8, 128, 64, 64 * 62000 + 17
    sh = shape_of(8, hkv, d, bt, 1.0)
    bb = ref.block_bytes(hkv, d, bt)
    blocks = -(-n // bt)
    assert blocks * bb > (1 << 32)
    buf = torch.zeros(blocks * bb, dtype=torch.uint8, device="cuda")              # keys and values of zero
    rng = np.random.default_rng(3)
    q = synth.normal_bf16(rng, (1, 8, d))
    qf = synth.bf16_bits_to_f32(q)[0]
    k = synth.f32_to_bf16_bits(np.stack([qf * 0.125, qf * 0.125]))
    v = synth.normal_bf16(rng, (2, hkv, d))
    spans = [(buf, 0, 1), (buf, n - 1, 1)]
    kd, vd = synth.bits_to_torch(k, "cuda"), synth.bits_to_torch(v, "cuda")
    binding.ipkv_nibble_pack(sh, spans, kd, vd)
    ko, vo = torch.zeros_like(kd), torch.zeros_like(vd)
    binding.ipkv_nibble_unpack(sh, spans, ko, vo)
    o, lse = attend(sh, [[(buf, n)]], q)
    kv, vv = ref.quantised_values(k, v)
    assert np.array_equal(synth.torch_bits(vo), synth.f32_to_bf16_bits(vv.astype(np.float32)))
    s = np.einsum("hd,nhd->hn", qf.astype(np.float64), kv)
    z = np.exp(s).sum(1) + (n - 2)
    want = np.einsum("hn,nhd->hd", np.exp(s), vv) / z[:, None]
    # scores of about 16 (A = 2^5 with room), off by 2^-12; values below 8 therefore by 2^-8, sums of ones are exact
    np.testing.assert_allclose(o[0], want, atol=2.0 ** -8)
    np.testing.assert_allclose(lse[0], np.log(z), atol=2.0 ** -11)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 100])
def test_replays_from_a_graph_and_runs_on_another_stream(rows):
    """100 rows: the tables are uploaded inside the graph."""
    rng = np.random.default_rng(21)
    sh = shape_of(8, 2, 64, 64)
    buf, runs, kvs = fill(rng, sh, [[int(x)] for x in rng.integers(0, 300, rows)])
    q = synth.bits_to_torch(synth.normal_bf16(rng, (rows, 8, 64)), "cuda")
    scratch = [torch.empty(binding.ipkv_nibble_scratch_bytes(sh, rows, rows), dtype=torch.uint8, device="cuda") for _ in range(2)]
    o, lse = torch.zeros((2, rows, 8, 64), device="cuda"), torch.zeros((2, rows, 8), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        binding.ipkv_nibble_attend(sh, runs, None, q, scratch[0], o[0], lse[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.ipkv_nibble_attend(sh, runs, None, q, scratch[1], o[1], lse[1])
    for _ in range(2):
        o[1].zero_(); scratch[1].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o[0], o[1]) and torch.equal(lse[0], lse[1])
    check(sh, synth.torch_bits(q), kvs, o[1].cpu().numpy().astype(np.float64), lse[1].cpu().numpy().astype(np.float64))


@pytest.mark.gpu
def test_a_decode_run_from_prompt_to_merge():
    """As a serving loop uses them: prompts are normalised, rotated and packed in chunks; every step rotates, packs one token per
    sequence and attends the 4-bit part; the newest tokens of one sequence stay in bf16 blocks and their partial is joined."""
    hq, hkv, d, bt, steps = 8, 2, 64, 64, 5
    rng = np.random.default_rng(31)
    sh = shape_of(hq, hkv, d, bt)
    rope = binding.make_rope(d, sections=[8, 12, 12], eps=1e-6, theta=1e4)
    lens = [130, 1, 64, 333]
    most = -(-(max(lens) + steps) // bt)
    bb = ref.block_bytes(hkv, d, bt)
    pool = torch.full((len(lens), most * bb), 255, dtype=torch.uint8, device="cuda")
    wq, wk = (synth.bits_to_torch(synth.normal_bf16(rng, (d,)), "cuda") for _ in range(2))
    kept = [([], []) for _ in lens]

    def produce(n, pos):
        x = synth.bits_to_torch(synth.normal_bf16(rng, (n, (hq + 2 * hkv) * d)), "cuda")
        q, k, v = (y.unflatten(1, (-1, d)) for y in x.split([hq * d, hkv * d, hkv * d], 1))
        p = torch.tensor(np.stack([pos, pos // 4, pos % 4]).astype(np.int32), device="cuda")
        binding.ipkv_norm_rope(rope, [(q, wq, None), (k, wk, None)], p)
        return q, k, v

    for s, n in enumerate(lens):
        for a in range(0, n, 100):
            c = min(100, n - a)
            _, k, v = produce(c, np.arange(a, a + c))
            binding.ipkv_nibble_pack(sh, [(pool[s], a, c)], k, v)
            kept[s][0].append(synth.torch_bits(k)); kept[s][1].append(synth.torch_bits(v))
    scratch = torch.empty(binding.ipkv_nibble_scratch_bytes(sh, len(lens), len(lens)), dtype=torch.uint8, device="cuda")
    window = torch.zeros(binding.ipkv_block_bytes(sh), dtype=torch.uint8, device="cuda")      # bf16 block of the last sequence's newest tokens
    wk_bits, wv_bits = [], []
    for step in range(steps):
        q, k, v = produce(len(lens), np.asarray(lens) + step)
        new = [0, 1, 2]                                                   # the last sequence's token goes to its bf16 window
        binding.ipkv_nibble_pack(sh, [(pool[s], lens[s] + step, 1) for s in new], k[:3], v[:3])
        for s in new:
            kept[s][0].append(synth.torch_bits(k[s:s + 1])); kept[s][1].append(synth.torch_bits(v[s:s + 1]))
        wk_bits.append(synth.torch_bits(k[3:])); wv_bits.append(synth.torch_bits(v[3:]))
        kw, vw = np.concatenate(wk_bits), np.concatenate(wv_bits)
        binding.ipkv_pack_blocks(sh, binding.LAYOUT_TILE, synth.bits_to_torch(kw, "cuda"), synth.bits_to_torch(vw, "cuda"), step + 1, window)
        o, lse = torch.zeros((4, hq, d), device="cuda"), torch.zeros((4, hq), device="cuda")
        qc = q.contiguous()
        binding.ipkv_nibble_attend(sh, [[(pool[s], lens[s] + (step + 1 if s < 3 else 0))] for s in range(4)], None, qc, scratch, o, lse)
        ow, lw = torch.zeros((4, hq, d), device="cuda"), torch.full((4, hq), float("-inf"), device="cuda")
        ws = torch.zeros(binding.ipkv_attend_scratch_bytes(sh, 1, 1, step + 1), dtype=torch.uint8, device="cuda")
        binding.ipkv_attend_runs(sh, [[(window, step + 1)]], qc[3:], ws, ow[3:], lw[3:])
        out, out_lse = torch.zeros((4 * hq, d), device="cuda"), torch.zeros(4 * hq, device="cuda")
        binding.ipkv_merge(4 * hq, d, [o.view(-1, d), ow.view(-1, d)], [lse.view(-1), lw.view(-1)], out, out_lse)
        torch.cuda.synchronize()
        got, got_lse = out.view(4, hq, d).cpu().numpy(), out_lse.view(4, hq).cpu().numpy()
        for s in range(4):
            kb, vb = np.concatenate(kept[s][0]), np.concatenate(kept[s][1])
            kv, vv = ref.quantised_values(kb, vb)
            to, tl = tolerance(synth.torch_bits(qc)[s], ref.quantise(kb, 64), ref.quantise(vb, d), d ** -0.5, 512)
            if s == 3:
                kv = np.concatenate([kv, synth.bf16_bits_to_f32(kw).astype(np.float64)])
                vv = np.concatenate([vv, synth.bf16_bits_to_f32(vw).astype(np.float64)])
                to, tl = to + 2e-3, tl + 1e-3                             # the bf16 kernel's documented tolerance
            want_o, want_lse = ref.attend(synth.torch_bits(qc)[s], kv, vv, d ** -0.5)
            assert np.abs(got[s] - want_o).max() <= to and np.abs(got_lse[s] - want_lse).max() <= tl + 2.0 ** -18


@pytest.mark.gpu
@pytest.mark.parametrize("n_rows", [1, 70])              # tables in the launch, tables uploaded
def test_a_batch_without_tokens_and_a_block_that_rows_share(n_rows):
    rng = np.random.default_rng(41)
    sh = shape_of(8, 2, 128, 64)
    q = synth.normal_bf16(rng, (n_rows, 8, 128))
    o, lse = attend(sh, [[] if r % 2 else [(0, 0)] for r in range(n_rows)], q)
    assert not o.any() and np.isneginf(lse).all()
    buf, runs, kvs = fill(rng, sh, [[100]])
    (k, v), = kvs
    twice = [runs[0] * 2] * n_rows                       # the same tokens twice in a row, and in every row
    o, lse = attend(sh, twice, q)
    check(sh, q, [(np.concatenate([k, k]), np.concatenate([v, v]))] * n_rows, o, lse)


@pytest.mark.gpu
def test_k_and_v_side_by_side_and_spans_that_read_a_block_twice():
    """K and V interleaved per token in one buffer, with a column of other data between tokens that has to stay."""
    rng = np.random.default_rng(43)
    hkv, d, n = 2, 64, 150
    sh = shape_of(4, hkv, d, 64)
    row = hkv * d
    x = synth.normal_bf16(rng, (n, 2 * row + 8))
    src = synth.bits_to_torch(x, "cuda")
    k, v = src[:, :row].view(n, hkv, d), src[:, row:2 * row].view(n, hkv, d)
    buf = torch.full((3 * ref.block_bytes(hkv, d, 64),), 255, dtype=torch.uint8, device="cuda")
    binding.ipkv_nibble_pack(sh, [(buf, 0, n)], k, v)
    dst = torch.full((2 * n, 2 * row + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = dst[:, :row].view(2 * n, hkv, d), dst[:, row:2 * row].view(2 * n, hkv, d)
    binding.ipkv_nibble_unpack(sh, [(buf, 0, n), (buf, 0, n)], ko, vo)
    kv, vv = ref.quantised_values(x[:, :row].reshape(n, hkv, d), x[:, row:2 * row].reshape(n, hkv, d))
    for got, want in ((ko, kv), (vo, vv)):
        want = synth.f32_to_bf16_bits(want.astype(np.float32))
        assert np.array_equal(synth.torch_bits(got[:n].contiguous()), want) and np.array_equal(synth.torch_bits(got[n:].contiguous()), want)
    assert bool((dst[:, 2 * row:] == 7).all())


@pytest.mark.gpu
def test_calls_at_once_from_two_threads_on_their_own_streams():
    import threading
    rng = np.random.default_rng(47)
    sh = shape_of(16, 2, 128, 64)
    rows = [[2000], [], [65, 700]]
    jobs = []
    for i in range(2):
        buf, runs, _ = fill(rng, sh, rows, spread=1.0 + i)
        q = synth.bits_to_torch(synth.normal_bf16(rng, (3, 16, 128)), "cuda")
        o, lse = attend(sh, runs, q)
        scratch = torch.empty(binding.ipkv_nibble_scratch_bytes(sh, 3, 4), dtype=torch.uint8, device="cuda")
        jobs.append((runs, q, scratch, torch.empty((20, 3, 16, 128), device="cuda"), torch.empty((20, 3, 16), device="cuda"), o, lse, buf))
    errors = []

    def work(job):
        try:
            runs, q, scratch, o, lse = job[:5]
            s = torch.cuda.Stream()
            for i in range(20):
                binding.ipkv_nibble_attend(sh, runs, None, q, scratch, o[i], lse[i], stream=s)
            s.synchronize()
        except Exception as e:                           # a thread's exception would be lost
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors
    for _, _, _, o, lse, want_o, want_lse, _ in jobs:
        for i in range(20):
            assert np.array_equal(o[i].cpu().numpy(), want_o.astype(np.float32)) and np.array_equal(lse[i].cpu().numpy(), want_lse.astype(np.float32))
