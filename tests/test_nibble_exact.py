"""The 4-bit cache's attention against 64 bits under bounds that follow its arithmetic, head by head: what wider bounds would let
pass (an output of zeros, a tile left out, weights of one half) fails here, which is checked on the host.

The bound on a head's output.  With p_t the softmax weights and v_t the values in 64 bits, `size` = sqrt(sum p_t^2 |v_t|^2) is how
large the output is when values are independent, and how large its error is when every token's share is off by a relative error
that is independent of the others' (an error that all tokens have in common leaves with the denominator).  The parts of the relative error:
  * a weight: fp32 products and ex2 2^-22, and its two fp16 halves 2^-22;
  * a score: a tensor-core step adds 16 products and the sum so far, cut at 2^-26 of the largest exponent, and cuts the sum at 2^-24.  For
    normal queries sums of q * code stay below 2^7 (64 columns, codes of 0..15), so a step is off by less than
    17 * 2^-19 + 2^-17 = 2^-14.7, the eight steps of 128 columns by 2^-11.7 if all erred alike and by a quarter of that with
    cuts of either sign; times a scale of key and softmax (1.2 * 0.09): 2^-16.9;
  * the output's sums: 64 tokens a tile, products of either sign (every other token is complemented), sums below 2^7 of a value's
    scale: four steps of 2^-14.7 if all erred alike, 2^-14.7 with cuts of either sign, against 24 scales (the size of the sum of 64 values
    that lie within 15 scales): 2^-19.3.
Together below 2^-16.  An absolute share comes on top: every other weight of a tile is held in steps of 2^-33 of the reference's, the rest in finer
ones.  Off by 2^-34.8 (half a step over the root of three), half of the tokens, the root of the 192 tokens that a warp has here, times a
code of 8 against values of 3 scales: 2^-30 of the values (`FLOOR`).  It counts only where one token outweighs the others by 2^14 and
more and has no values.
"""
import numpy as np
import pytest

from paper_2609_14507_b200 import binding, synth
from tests import nibble_ref as ref
from tests.test_nibble import attend, fill, shape_of

torch = pytest.importorskip("torch")

RELATIVE, FLOOR = 2.0 ** -16, 2.0 ** -30
LSE = 2.0 ** -15        # a score's error as above, common to all tokens, twice over; ln and its sum 2^-22 of the value


def exact(sh, q, k, v):
    """One row: q bits [Hq][D], K and V bits [n][Hkv][D] -> weights [Hq][n], values [n][Hkv][D], O, LSE."""
    scale = float(np.float32(sh.softmax_scale if sh.softmax_scale > 0 else sh.dim_qk ** -0.5))
    kd, vd = ref.quantised_values(k, v)
    hq, d = q.shape
    qd = synth.bf16_bits_to_f32(q).astype(np.float64).reshape(sh.n_kv_heads, -1, d)
    s = np.matmul(qd, kd.transpose(1, 2, 0)) * scale
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    z = e.sum(-1, keepdims=True)
    p = e / z
    o = np.matmul(p, vd.transpose(1, 0, 2))
    return p, vd, o.reshape(hq, d), (m + np.log(z)).reshape(hq)


def bounds(p, vd):
    """Per query head: how far its output may be from 64 bits (Euclidean norm over its columns)."""
    v2 = (vd ** 2).sum(-1).T[:, None]                                     # [Hkv][1][n]
    size = np.sqrt((p ** 2 * v2).sum(-1))
    return (size * RELATIVE + np.sqrt(v2.max(-1)) * FLOOR).reshape(-1)


def miss(o, want, bound):
    """The largest error over its bound among the heads."""
    return float((np.linalg.norm(o - want, axis=-1) / bound).max())


def check_exact(sh, q, kvs, o, lse):
    for r, (k, v) in enumerate(kvs):
        if not k.shape[0]:
            assert not o[r].any() and np.isneginf(lse[r]).all()
            continue
        p, vd, want, want_lse = exact(sh, q[r], k, v)
        assert np.isfinite(o[r]).all()
        assert miss(o[r], want, bounds(p, vd)) <= 1, (r, k.shape[0], miss(o[r], want, bounds(p, vd)))
        assert (np.abs(lse[r] - want_lse) <= LSE + np.abs(want_lse) * 2.0 ** -22).all(), (r, np.abs(lse[r] - want_lse).max())


# ---- what the bound tells apart: mistakes made in a restatement on the host ------------------------------------------

@pytest.mark.parametrize("hq,hkv,d,n", [(4, 1, 64, 40000), (8, 2, 128, 9600), (16, 1, 128, 4097), (8, 8, 128, 64)])
def test_the_bound_fails_what_is_wrong(hq, hkv, d, n):
    rng = np.random.default_rng(n)
    sh = shape_of(hq, hkv, d, 64)
    k, v = synth.normal_bf16(rng, (n, hkv, d)), synth.normal_bf16(rng, (n, hkv, d))
    q = synth.normal_bf16(rng, (hq, d))
    p, vd, want, _ = exact(sh, q, k, v)
    bound = bounds(p, vd)
    product = lambda w: np.matmul(w, vd.transpose(1, 0, 2)).reshape(hq, d)
    assert miss(product(p.astype(np.float32).astype(np.float64)), want, bound) < 0.1     # fp32 weights pass
    assert miss(np.zeros_like(want), want, bound) > 100
    left_out = p.copy()
    left_out[..., n // 2:n // 2 + 16] = 0                                                # sixteen tokens
    assert miss(product(left_out / left_out.sum(-1, keepdims=True)), want, bound) > 100
    unit = p / p.max(-1, keepdims=True)                                                  # against the reference, as the kernel holds them
    for cut in (lambda x: x.astype(np.float16).astype(np.float64), lambda x: synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(x.astype(np.float32))).astype(np.float64)):
        one_half = cut(unit)
        assert miss(product(one_half / unit.sum(-1, keepdims=True)), want, bound) > 4    # the remainder left out
    gone = vd.copy()
    gone[1::2] -= np.abs(vd).max() * 2.0 ** -8                                           # half of the tokens a little low
    assert miss(np.matmul(p, gone.transpose(1, 0, 2)).reshape(hq, d), want, bound) > 4


# ---- outputs ---------------------------------------------------------------------------------------------------------

def long_among(n_short, short, long):
    """Rows of one length with a long one among them: more pairs than CTAs are resident, so work goes out in equal chunks, and the long
    row meets so many that its join is cut into slabs."""
    rows = [[short]] * n_short
    rows[n_short // 2] = [long]
    return rows


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,bt,rows", [
    (32, 4, 128, 64, [[1]]), (32, 4, 128, 64, [[4097]]), (32, 8, 128, 64, [[700, 33], [64], [], [1000, 1, 129]]),
    (8, 8, 64, 64, [[333]]), (6, 3, 64, 128, [[63, 65], [0], [200]]), (12, 4, 64, 64, [[1500, 77], [2]]),
    (8, 2, 128, 64, [[64] * 150, [1, 64, 3] * 30]),                       # pages
    # several heads on one tile and several groups of heads, the last one smaller: two octets, and four
    (24, 1, 128, 64, [[300], [5000]]), (44, 1, 64, 64, [[300], [65], []]), (44, 1, 128, 64, [[20000]]), (57, 1, 128, 64, [[700], [64]]),
    (60, 1, 64, 128, [[500, 3], [1]]), (60, 1, 128, 64, [[9000]]), (88, 2, 64, 64, [[130], [4000]]), (119, 1, 128, 64, [[300], [65]]),
    # one pair of many partials: joins by one CTA a head, by slabs of 256 and of 512 threads
    (4, 1, 64, 64, [[3000]]), (8, 1, 128, 64, [[9000]]), (4, 1, 64, 64, [[40000]]), (8, 1, 128, 64, [[40000]]), (16, 1, 128, 64, [[40000, 7]]),
    # equal chunks with either join, tables in the launch (up to 64 rows) and uploaded
    (8, 8, 64, 64, long_among(64, 64, 5000)), (32, 8, 128, 64, long_among(60, 100, 9000)), (16, 8, 64, 64, long_among(64, 64, 20000)),
    (4, 1, 128, 64, long_among(450, 64, 10000)), (8, 1, 64, 64, long_among(450, 64, 40000)), (44, 1, 64, 64, long_among(160, 64, 12000)),
])
def test_attention_within_its_own_arithmetic(hq, hkv, d, bt, rows):
    rng = np.random.default_rng(hq * 100 + d + len(rows))
    sh = shape_of(hq, hkv, d, bt)
    buf, runs, kvs = fill(rng, sh, rows)
    q = synth.normal_bf16(rng, (len(rows), hq, d))
    o, lse = attend(sh, runs, q)
    check_exact(sh, q, kvs, o, lse)


def packed(sh, k, v):
    n = k.shape[0]
    buf = torch.full((-(-n // 64) * ref.block_bytes(sh.n_kv_heads, sh.dim_qk, 64),), 255, dtype=torch.uint8, device="cuda")
    binding.ipkv_nibble_pack(sh, [(buf, 0, n)], synth.bits_to_torch(k, "cuda"), synth.bits_to_torch(v, "cuda"))
    return buf


def controlled(rng, hq, hkv, d, n, log2_weight):
    """Queries and keys whose scores are log2_weight[t] * ln 2 and a little noise, with softmax_scale 1."""
    sign = np.where(rng.random(d) < 0.5, -1.0, 1.0)
    a = np.asarray(log2_weight) * np.log(2) / d
    k = a[:, None, None] * sign + rng.standard_normal((n, hkv, d)) * 0.02
    q = np.broadcast_to(sign, (1, hq, d))
    return synth.f32_to_bf16_bits(q.astype(np.float32)), synth.f32_to_bf16_bits(k.astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 1), (16, 1), (32, 2)])
@pytest.mark.parametrize("at", [0, 5, 300])
@pytest.mark.parametrize("gap", [12, 16, 20])
def test_many_weak_tokens_beside_one_that_dominates(hq, hkv, at, gap):
    """The token that a softmax rests on when nothing matters: nearly all the weight and no values.  The output is what the others leave."""
    d, n = 128, 700
    rng = np.random.default_rng(gap * 1000 + at)
    sh = shape_of(hq, hkv, d, 64, 1.0)
    level = np.zeros(n)
    level[at] = gap
    q, k = controlled(rng, hq, hkv, d, n, level)
    v = synth.normal_bf16(rng, (n, hkv, d))
    v[at] = 0
    o, lse = attend(sh, [[(packed(sh, k, v), n)]], q)
    check_exact(sh, q, [(k, v)], o, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 1), (32, 2)])
@pytest.mark.parametrize("at", [0, 300, 699])
@pytest.mark.parametrize("factor,gap", [(12, 24), (20, 24), (20, 80), (30, 80), (60, 80), (20, 16), (30, 8)])
def test_a_value_far_out_takes_no_digits_from_the_others(hq, hkv, at, factor, gap):
    """One token whose values are 2^factor times the others' and whose weight is 2^-gap of theirs: what it adds counts, its scale does not."""
    d, n = 128, 700
    rng = np.random.default_rng(factor * 1000 + at + gap)
    sh = shape_of(hq, hkv, d, 64, 1.0)
    level = np.zeros(n)
    level[at] = -gap
    q, k = controlled(rng, hq, hkv, d, n, level)
    v = rng.standard_normal((n, hkv, d)).astype(np.float32)
    v[at] *= np.float32(2.0) ** factor
    v = synth.f32_to_bf16_bits(v)
    o, lse = attend(sh, [[(packed(sh, k, v), n)]], q)
    p, vd, want, want_lse = exact(sh, q[0], k, v)
    rest = np.delete(vd, at, 0)                          # the floor goes by the others' values
    size = np.sqrt((p ** 2 * (vd ** 2).sum(-1).T[:, None]).sum(-1)).reshape(-1)
    assert miss(o[0], want, size * RELATIVE + np.sqrt((rest ** 2).sum(-1).max()) * FLOOR) <= 1
    assert (np.abs(lse[0] - want_lse) <= LSE + np.abs(want_lse) * 2.0 ** -22).all()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 1), (32, 2)])
@pytest.mark.parametrize("at", [0, 300, 699])
@pytest.mark.parametrize("factor", [10, 20, 30])
def test_what_one_head_looks_at_takes_no_digits_from_the_heads_beside_it(hq, hkv, at, factor):
    """The token with values far out has all of every other head's weight and nothing of the rest's."""
    d, n = 128, 700
    rng = np.random.default_rng(factor * 1000 + at)
    sh = shape_of(hq, hkv, d, 64, 1.0)
    sign = np.where(rng.random(d) < 0.5, -1.0, 1.0)
    k = rng.standard_normal((n, hkv, d)) * 0.02
    k[at, :, :64] += sign[:64] * 20 * np.log(2) / 64
    k[at, :, 64:] -= sign[64:] * 80 * np.log(2) / 64
    q = np.zeros((1, hq, d))
    q[0, ::2, :64] = sign[:64]
    q[0, 1::2, 64:] = sign[64:]
    v = rng.standard_normal((n, hkv, d)).astype(np.float32)
    v[at] *= np.float32(2.0) ** factor
    q, k, v = (synth.f32_to_bf16_bits(x.astype(np.float32)) for x in (q, k, v))
    o, lse = attend(sh, [[(packed(sh, k, v), n)]], q)
    p, vd, want, want_lse = exact(sh, q[0], k, v)
    size = np.sqrt((p ** 2 * (vd ** 2).sum(-1).T[:, None]).sum(-1)).reshape(-1)
    floor = np.sqrt((np.delete(vd, at, 0) ** 2).sum(-1).max()) * FLOOR
    assert miss(o[0], want, size * RELATIVE + floor) <= 1
    assert (np.abs(lse[0] - want_lse) <= LSE + np.abs(want_lse) * 2.0 ** -22).all()
