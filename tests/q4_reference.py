"""The 4-bit format in numpy and 64 bits, for the tests: written from its definition, one value at a time where
that is clearer, and sharing nothing with the library."""
import numpy as np


def quantise(x, group):
    """x float64 [..., n] holding bf16 values -> (codes int, scales float64 [..., ceil(n / group)])"""
    n = x.shape[-1]
    pad = [(0, 0)] * (x.ndim - 1) + [(0, -n % group)]
    y = np.pad(x, pad).reshape(*x.shape[:-1], -1, group)
    bad = ~np.isfinite(y).all(-1)
    a = np.abs(np.where(np.isfinite(y), y, 0.0)).max(-1)
    m, e = np.frexp(a / 7.0)
    s = np.ldexp(np.ceil(m * 32.0), e - 5)
    s = np.where(a > 0, np.clip(s, 2.0 ** -126, 1.125 * 2.0 ** 125), 0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        c = np.rint(np.where(np.isfinite(y), y, 0.0) / np.where(s > 0, s, 1.0)[..., None])
    c = np.clip(c, -7, 7)
    c[bad] = 0
    s = np.where(bad, np.nan, s)
    return c.reshape(*x.shape[:-1], -1)[..., :n].astype(np.int64), s


def values(codes, scales, group):
    n = codes.shape[-1]
    return codes * np.repeat(scales, group, -1)[..., :n]


def row_place(col, C):
    """(byte, nibble) of column col in a row of C = 64 or 128 columns"""
    j, t, e = col // 32, col % 32 // 8, col % 8
    nib = e // 2 + 4 * (e % 2)
    return 4 * (t * (C // 32) + j) + nib // 2, nib % 2


def v_place(i, ch, hd):
    """(byte, nibble) of token i, channel ch among a tile's V codes"""
    g, r = ch // (hd // 8), ch % (hd // 8)
    return (((i // 8 * 8 + g) * 4 + i // 2 % 4) * 2 + i % 2) * (hd // 16) + r // 2, r % 2


def bf16_bytes(s):
    """float64 array of bf16 values (NaN: 0x7fff) -> bytes"""
    u = (np.asarray(s, np.float32).view(np.uint32) >> 16).astype(np.uint16)
    return np.where(np.isnan(s), np.uint16(0x7FFF), u).astype("<u2").tobytes()


def put(buf, byte, nibble, code):
    u = int(code) + 8
    buf[byte] = (int(buf[byte]) & (0x0F if nibble else 0xF0)) | (u << 4 if nibble else u)


def pack_weight(w, group):
    """float64 [N, K] -> packed bytes (uint8)"""
    N, K = w.shape
    n16, kb, ng = -(-N // 16), -(-K // 128), 128 // group
    codes, scales = quantise(w, group)
    C = np.zeros((n16 * 16, kb * 128), np.int64)
    C[:N, :K] = codes
    S = np.zeros((n16 * 16, kb * ng))
    S[:N, :scales.shape[1]] = scales
    place = [row_place(c, 128) for c in range(128)]
    out = []
    for a in range(n16):
        for b in range(kb):
            blk = np.zeros((16, 64), np.uint8)
            part = (C[16 * a:16 * a + 16, 128 * b:128 * b + 128] + 8).astype(np.uint8)
            for c, (byte, nib) in enumerate(place):
                blk[:, byte] |= part[:, c] << (4 * nib)
            out.append(blk.tobytes())
            out.append(bf16_bytes(S[16 * a:16 * a + 16, ng * b:ng * b + ng]))
    return np.frombuffer(b"".join(out), np.uint8)


def tile_bytes(hd):
    return 16 * (hd + hd // 8)


def put_token(tile, i, k, v, hd):
    """writes token i of a tile (uint8 array): k, v float64 [hd]"""
    kc, ks = quantise(k, 32)
    vc, vs = quantise(v, 32)
    for ch in range(hd):
        byte, nib = row_place(ch, hd)
        put(tile, i * hd // 2 + byte, nib, kc[ch])
        byte, nib = v_place(i, ch, hd)
        put(tile, 9 * hd + byte, nib, vc[ch])
    G = hd // 32
    tile[8 * hd + 2 * G * i:8 * hd + 2 * G * (i + 1)] = np.frombuffer(bf16_bytes(ks), np.uint8)
    for j in range(G):
        at = 17 * hd + 2 * (16 * j + i)
        tile[at:at + 2] = np.frombuffer(bf16_bytes(vs[j:j + 1]), np.uint8)


def attention(q, k, v, limit, G):
    """q [Hq, hd], k, v [T, Hkv, hd] float64, positions 0..limit visible -> ([Hq, hd], the same with |v|)"""
    Hq, hd = q.shape
    out, spread = np.zeros((Hq, hd)), np.zeros((Hq, hd))
    if limit < 0:
        return out, spread
    for h in range(Hq):
        s = k[:limit + 1, h // G] @ q[h] / np.sqrt(hd)
        p = np.exp(s - s.max())
        p /= p.sum()
        out[h] = p @ v[:limit + 1, h // G]
        spread[h] = p @ np.abs(v[:limit + 1, h // G])
    return out, spread
