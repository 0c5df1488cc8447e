"""The 4-bit block format restated from its definition in include/ipkv.h (NumPy, host): codes, tiles, blocks."""
import numpy as np

from paper_2609_14507_b200 import synth


def quantise(bits, width):
    """bf16 bits [..., D] -> codes uint8 [..., D], scale bits and zero bits uint16 [..., D / width]; every step in fp32."""
    x = synth.bf16_bits_to_f32(bits)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // width, width)
    zero = g.min(-1, keepdims=True)
    scale_bits = synth.f32_to_bf16_bits((g.max(-1, keepdims=True) - zero) / np.float32(15))
    scale = synth.bf16_bits_to_f32(scale_bits)
    ok = scale >= np.float32(2.0 ** -126)
    q = np.rint((g - zero) / np.where(ok, scale, np.float32(1)))
    codes = np.where(ok, np.minimum(q, 15), 0).astype(np.uint8)
    return codes.reshape(x.shape), scale_bits[..., 0], synth.f32_to_bf16_bits(zero)[..., 0]


def values(codes, scale_bits, zero_bits, width):
    """What codes stand for, fp64 (exact: 12-bit products plus a bf16)."""
    s = synth.bf16_bits_to_f32(scale_bits).astype(np.float64).repeat(width, -1)
    z = synth.bf16_bits_to_f32(zero_bits).astype(np.float64).repeat(width, -1)
    return codes * s + z


def quantised_values(k_bits, v_bits):
    return values(*quantise(k_bits, 64), 64), values(*quantise(v_bits, v_bits.shape[-1]), v_bits.shape[-1])


def tile_bytes(d):
    return 64 * d + 256 * (d // 64 + 1)


def block_bytes(hkv, d, bt):
    return hkv * (bt // 64) * tile_bytes(d)


def write(buf, hkv, d, bt, first, k_bits, v_bits):
    """Put tokens first.. (k, v bits [n][hkv][d]) into the byte image `buf` of a run of blocks, bit by bit as defined."""
    P, per = d // 64, bt // 64
    kq, ks, kz = quantise(k_bits, 64)
    vq, vs, vz = quantise(v_bits, d)
    cols = np.arange(d)
    for i in range(k_bits.shape[0]):
        tok = first + i
        tile, tl = divmod(tok, 64)
        u, h, g = tl // 16, (tl // 8) % 2, tl % 8
        for head in range(hkv):
            at = (tile // per) * block_bytes(hkv, d, bt) + head * per * tile_bytes(d) + (tile % per) * tile_bytes(d)
            img = buf[at:at + tile_bytes(d)].view("<u4")
            p, t, w, j = cols // 64, (cols % 64) // 16, (cols % 16) // 8, cols % 8
            word = ((((u * P + p) * 8 + g) * 4 + t) * 2 + h) * 2 + w
            for c in range(d):
                img[word[c]] = (img[word[c]] & ~np.uint32(15 << (4 * j[c]))) | np.uint32(int(kq[i, head, c]) << (4 * j[c]))
            w32, i8, tt, e = tl // 32, (tl % 32) // 8, (tl % 8) // 2, tl % 2
            dd, hh, gg = cols // 16, (cols // 8) % 2, cols % 8
            word = 8 * d + 64 * P + (((dd * 8 + gg) * 4 + tt) * 2 + hh) * 2 + w32
            n = i8 + 4 * e
            img[word] = (img[word] & ~np.uint32(15 << (4 * n))) | (vq[i, head].astype(np.uint32) << np.uint32(4 * n))
            row = 16 * u + 2 * g + h
            for pn in range(P):
                img[8 * d + row * P + pn] = np.uint32(ks[i, head, pn]) | (np.uint32(kz[i, head, pn]) << np.uint32(16))
            img[16 * d + 64 * P + row] = np.uint32(vs[i, head, 0]) | (np.uint32(vz[i, head, 0]) << np.uint32(16))


def attend(q_bits, k, v, scale):
    """One row in 64 bits: q bits [Hq][D], k, v fp64 [n][Hkv][D] -> O [Hq][D], LSE [Hq], and the largest sum of |terms| of a score."""
    hq, d = q_bits.shape
    hkv = k.shape[1]
    q = synth.bf16_bits_to_f32(q_bits).astype(np.float64).reshape(hkv, hq // hkv, d)
    if k.shape[0] == 0:
        return np.zeros((hq, d)), np.full(hq, -np.inf)
    s = np.einsum("hgd,nhd->hgn", q, k) * scale
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    z = e.sum(-1, keepdims=True)
    o = np.einsum("hgn,nhd->hgd", e / z, v)
    return o.reshape(hq, d), (m + np.log(z)).reshape(hq)
