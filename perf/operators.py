"""Decoding from 4-bit weights and a 4-bit cache: the cases that are measured, and the operators' plain forms.

One number format serves both.  A group of values x shares a scale s, the largest |x| / 7 rounded up to 5
significant bits and kept as bf16; a value stands for c * s with an integer code c = rint(x / s) in -7..7, which
is exactly a bf16 number (5 + 3 bits).  A code is stored as the nibble c + 8.

Weights [N, K], groups of 32, 64 or 128 along K, are packed in blocks of 16 rows by 128 columns, all blocks of 16
rows one after the other; N and K are padded with zeros.  A block is 16 rows of 64 bytes of codes, then the scales
[16 rows][128 / group].  In a row, the 32-bit word 4 t + j holds columns 32 j + 8 t .. + 7, column e of the eight at
nibble e / 2 + 4 (e % 2).

The cache is a pool of pages [n_pages][Hkv][page_size / 16 tiles].  A tile is 16 tokens of one head, groups of 32:
  K codes   16 rows of head_dim / 2 bytes; word t (head_dim / 32) + j of a row holds channels 32 j + 8 t .. + 7, as above
  K scales  [16 tokens][head_dim / 32]
  V codes   [token / 8][piece g = 0..7][(token / 2) % 4][token % 2] pieces of head_dim / 8 channels, lowest nibble first
  V scales  [head_dim / 32][16 tokens]
"""
import math

import torch

own = False

BF16 = torch.bfloat16


# ---------------------------------------------------------------- cases
def listed():
    return [
        # a checkpoint's projection is laid out once: the square one, and a feed-forward matrix with wide groups
        {"name": "pack 4096x4096 g32", "op": "pack", "N": 4096, "K": 4096, "group": 32},
        {"name": "pack 11008x4096 g128", "op": "pack", "N": 11008, "K": 4096, "group": 128},
        # one token through the smallest model's projection: latency alone
        {"name": "linear 256x256 M1", "op": "linear", "N": 256, "K": 256, "group": 32, "M": 1},
        # one token through an output projection
        {"name": "linear 4096x4096 M1", "op": "linear", "N": 4096, "K": 4096, "group": 128, "M": 1},
        # a verify pass of 7 rows through the down projection, whose length is no power of two
        {"name": "linear 4096x11008 M7", "op": "linear", "N": 4096, "K": 11008, "group": 32, "M": 7},
        # a large vocabulary's head for 16 rows (8 sequences of two)
        {"name": "linear 128256x4096 M16", "op": "linear", "N": 128256, "K": 4096, "group": 64, "M": 16},
        # a decode step of 8 sequences appends a row each
        {"name": "append 8 rows", "op": "append", "n_seq": 8, "M": 1, "ctx": 1024, "Hkv": 32, "hd": 128, "page": 64},
        # a prompt appends all its rows, and reads them back for the prompt pass
        {"name": "append prompt 4096", "op": "append", "n_seq": 1, "M": 4096, "ctx": 4096, "Hkv": 8, "hd": 128, "page": 64},
        # a draft token over a prompt of a thousand tokens
        {"name": "attention 1030 M1", "op": "attention", "n_seq": 1, "M": 1, "ctx": 1030, "Hkv": 32, "G": 1, "hd": 128, "page": 64},
        # a verify pass of seven rows over a prompt of four thousand
        {"name": "attention 4103 M7", "op": "attention", "n_seq": 1, "M": 7, "ctx": 4103, "Hkv": 32, "G": 1, "hd": 128, "page": 64},
        # 16 sequences of ragged lengths, two rows each, small pages, one sequence with nothing to see
        {"name": "attention 16 seqs", "op": "attention", "n_seq": 16, "M": 2, "ctx": 5000, "Hkv": 8, "G": 4, "hd": 128, "page": 16},
        # one token at the end of a long context
        {"name": "attention 131072 M1", "op": "attention", "n_seq": 1, "M": 1, "ctx": 131072, "Hkv": 8, "G": 4, "hd": 128, "page": 64},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("pack", "linear", "linear", "append", "attention", "attention"))
    if op in ("pack", "linear"):
        K = 8 * _log(rng, 8, 1792)
        N = _log(rng, 16, min(128256, (1 << (29 if op == "linear" else 26)) // K))
        c = {"op": op, "N": N, "K": K, "group": rng.choice((32, 64, 128))}
        return dict(c, M=rng.randint(1, 16)) if op == "linear" else c
    hd, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128, 256))
    Hkv = rng.choice((1, 2, 4, 8, 16, 32, 40))
    n_seq = _log(rng, 1, 32)
    if op == "append":
        M = _log(rng, 1, max(1, min(8192, (1 << 23) // (n_seq * Hkv * hd))))
        return {"op": op, "n_seq": n_seq, "M": M, "ctx": M + _log(rng, 1, 4096), "Hkv": Hkv, "hd": hd, "page": page}
    G, M = rng.choice((1, 2, 4, 8)), rng.randint(1, 16)
    top = (1 << 27) // (n_seq * Hkv * hd * max(1, M * G // 8))
    return {"op": op, "n_seq": n_seq, "M": M, "ctx": _log(rng, M, max(M, min(131072, top))), "Hkv": Hkv, "G": G, "hd": hd, "page": page}


def _tile_bytes(hd):
    return 16 * (hd + hd // 8)


def _weight_bytes(c):
    return -(-c["N"] // 16) * -(-c["K"] // 128) * (1024 + 32 * (128 // c["group"]))


def work(c):
    if c["op"] == "pack":
        n = c["N"] * c["K"]
        return {"bytes": 4 * n + _weight_bytes(c), "flops": 4 * n}
    if c["op"] == "linear":
        return {"bytes": _weight_bytes(c) + c["M"] * (2 * c["K"] + 4 * c["N"]), "flops": 2 * c["M"] * c["N"] * c["K"]}
    if c["op"] == "append":
        n = c["n_seq"] * c["M"] * c["Hkv"]
        return {"bytes": n * (8 * c["hd"] + _tile_bytes(c["hd"]) // 16), "flops": 8 * n * c["hd"]}
    seen = sum(_lengths(c))
    rows = c["n_seq"] * c["M"] * c["Hkv"] * c["G"] * c["hd"]
    return {"bytes": seen * c["Hkv"] * _tile_bytes(c["hd"]) // 16 + 4 * rows, "flops": 4 * seen * c["M"] * c["Hkv"] * c["G"] * c["hd"]}


def _lengths(c):
    """Tokens that the last row of each sequence sees: spread over half to all of the context; with many sequences
    one of them is idle."""
    n, ctx, M = c["n_seq"], c["ctx"], c["M"]
    lens = [max(M, ctx - (ctx // 2) * ((7 * b) % n) // n) for b in range(n)]
    if n >= 8:
        lens[n // 2] = 0
    return lens


# ---------------------------------------------------------------- inputs
def _quantised(x, group):
    """codes (int, -7..7) and scales of x's groups along the last axis, of the format's definition"""
    x = x.float().unflatten(-1, (-1, group))
    a = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a.double() / torch.full_like(a, 7, dtype=torch.float64))  # a true division: / 7 multiplies by 1 / 7
    s = torch.where(a > 0, torch.ldexp(torch.ceil(m * 32), e - 5), torch.zeros_like(m))
    c = torch.round(x.double() / torch.where(s > 0, s, torch.ones_like(s))).clamp(-7, 7)
    return c.flatten(-2).to(torch.int32), s.squeeze(-1).to(BF16)


def _bytes_of(t):
    return t.contiguous().view(torch.uint8)


def _nibbles(u):
    """bytes from nibbles (last axis, lowest first)"""
    u = u.to(torch.uint8)
    return u[..., 0::2] | (u[..., 1::2] << 4)


def _k_rows(codes):
    """[..., C] codes of rows -> [..., C / 2] bytes, in blocks of 128 columns (64 if there are only 64)"""
    C = min(128, codes.shape[-1])
    u = (codes + 8).unflatten(-1, (-1, C // 32, 4, 4, 2))  # block, j, t, lo, hi
    d = u.dim()
    u = u.permute(*range(d - 4), d - 3, d - 4, d - 1, d - 2)  # block, t, j, hi, lo
    return _nibbles(u.flatten(-5))


def _packed_weight(codes, scales, group):
    """codes [N, K] and scales [N, ceil(K / group)] as blocks of 16 rows by 128 columns"""
    N, K = codes.shape
    n16, kb, ng = -(-N // 16), -(-K // 128), 128 // group
    c = torch.nn.functional.pad(codes, (0, kb * 128 - K, 0, n16 * 16 - N))
    s = torch.nn.functional.pad(scales, (0, kb * ng - scales.shape[1], 0, n16 * 16 - N))
    cb = _k_rows(c).view(n16, 16, kb, 64).permute(0, 2, 1, 3).reshape(n16, kb, 1024)
    sb = _bytes_of(s.view(n16, 16, kb, ng).permute(0, 2, 1, 3).reshape(n16, kb, 16 * ng))
    return torch.cat([cb, sb], -1).reshape(-1)


def _cache_tiles(k, v):
    """k, v [..., 16 tokens, hd] -> tile bytes [..., 16 * (hd + hd / 8)]"""
    kc, ks = _quantised(k, 32)
    vc, vs = _quantised(v, 32)
    hd = k.shape[-1]
    vb = _nibbles((vc + 8).unflatten(-1, (8, hd // 8)))  # token, piece, bytes
    vb = vb.unflatten(-3, (2, 4, 2))  # half, t, which, piece, bytes
    d = vb.dim()
    vb = vb.permute(*range(d - 4), d - 2, d - 4, d - 3, d - 1)  # half, piece, t, which, bytes
    return torch.cat([_k_rows(kc).flatten(-2), _bytes_of(ks.flatten(-2)), vb.flatten(-5), _bytes_of(vs.transpose(-1, -2).flatten(-2))], -1)


def _kv(shape, g):
    """keys with a few loud channels, values without"""
    k = torch.randn(shape, generator=g, device="cuda")
    loud = torch.ones(shape[-1], device="cuda")
    loud[5::29] = 6.0
    return (k * loud).to(BF16), torch.randn(shape, generator=g, device="cuda").to(BF16)


def _tables(c, n_tab, extra, g):
    n_pages = c["n_seq"] * n_tab + extra
    order = torch.randperm(n_pages, generator=g, device="cuda")[: c["n_seq"] * n_tab]
    return order.to(torch.int32).view(c["n_seq"], n_tab), n_pages


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(c)
    if c["op"] in ("pack", "linear"):
        w = (torch.randn((c["N"], c["K"]), generator=g, device="cuda") * 0.02).to(BF16)
        if c["op"] == "pack":
            st["w"] = w
            st["packed"] = torch.zeros(_weight_bytes(c), dtype=torch.uint8, device="cuda")
            st["out"] = torch.zeros_like(w)
        else:
            pad = torch.nn.functional.pad(w, (0, -c["K"] % c["group"]))
            codes, scales = zip(*[_quantised(p, c["group"]) for p in pad.split(16384)])
            st["packed"] = _packed_weight(torch.cat(codes)[:, : c["K"]], torch.cat(scales), c["group"])
            st["h"] = torch.randn((c["M"], c["K"]), generator=g, device="cuda").to(BF16)
            st["out"] = torch.empty((c["M"], c["N"]), dtype=torch.float32, device="cuda")
        return st
    n_seq, M, Hkv, hd, page = c["n_seq"], c["M"], c["Hkv"], c["hd"], c["page"]
    n_tab = -(-c["ctx"] // page)
    st["max_seq"] = n_tab * page
    st["table"], n_pages = _tables(c, n_tab, 2, g)
    st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if c["op"] == "append":
        st["k"], st["v"] = _kv((n_seq, M, Hkv, hd), g)
        st["pos0"] = torch.tensor([c["ctx"] - M - (b % (c["ctx"] - M + 1)) // 2 for b in range(n_seq)], dtype=torch.int32, device="cuda")
        st["pages"] = torch.zeros((n_pages, Hkv * page // 16 * _tile_bytes(hd)), dtype=torch.uint8, device="cuda")
        st["k_pages"] = torch.zeros((n_pages, Hkv, page, hd), dtype=BF16, device="cuda")
        st["v_pages"] = torch.zeros_like(st["k_pages"])
        return st
    # slots behind a sequence's last token hold whatever was there: random bytes, NaN scales among them
    T = n_tab * page
    lens = torch.tensor(_lengths(c), device="cuda")
    pool = torch.randint(0, 256, (n_pages, Hkv, page // 16, _tile_bytes(hd)), generator=g, device="cuda", dtype=torch.uint8)
    tokens = n_seq * T * Hkv
    parts = max(1, tokens * hd // (1 << 26))
    for tab in st["table"].tensor_split(min(parts, n_tab), 1):
        k, v = _kv((n_seq, tab.shape[1], Hkv, page // 16, 16, hd), g)
        pool[tab.long().flatten()] = _cache_tiles(k, v).flatten(0, 1)
    last = (lens.clamp(min=1) - 1) // 16  # the tile with a sequence's last token gets NaN scales behind it
    phys = st["table"].gather(1, (last * 16 // page).view(-1, 1).to(torch.int64)).squeeze(1).long()
    tile = pool[phys, :, last % (page // 16)]
    ks, vs = 8 * hd, 8 * hd + hd + 8 * hd
    behind = torch.arange(16, device="cuda") >= (lens - last * 16).view(-1, 1)
    kv = tile[..., ks : ks + hd].unflatten(-1, (16, -1))
    vv = tile[..., vs : vs + hd].unflatten(-1, (hd // 32, 16, 2))
    tile[..., ks : ks + hd] = torch.where(behind[:, None, :, None], torch.full_like(kv, 255), kv).flatten(-2)
    tile[..., vs : vs + hd] = torch.where(behind[:, None, None, :, None], torch.full_like(vv, 255), vv).flatten(-3)
    pool[phys, :, last % (page // 16)] = tile
    st["pages"] = pool.view(n_pages, -1)
    st["pos0"] = (lens - M).to(torch.int32)
    st["q"] = torch.randn((n_seq, M, Hkv * c["G"] * hd), generator=g, device="cuda").to(BF16)
    st["out"] = torch.empty_like(st["q"])
    return st


# ---------------------------------------------------------------- plain forms
def _codes(b):
    """bytes -> codes, lowest nibble first, as floats"""
    return torch.stack([b & 15, b >> 4], -1).flatten(-2).float() - 8


def _k_codes(b):
    """[..., C / 2] bytes of rows -> [..., C] codes, the columns in order"""
    C = min(128, 2 * b.shape[-1])
    u = _codes(b).unflatten(-1, (-1, 4, C // 32, 2, 4))  # block, t, j, hi, lo
    d = u.dim()
    return u.permute(*range(d - 4), d - 3, d - 4, d - 1, d - 2).flatten(-5)


def _scaled(codes, s, group):
    """codes times the scales of their groups"""
    return (codes.unflatten(-1, (-1, group)) * s.unsqueeze(-1)).flatten(-2)


def _bf16_at(b):
    return b.contiguous().view(BF16).float()


def _weight_values(packed, N, K, group):
    """fp32 [N, K] of packed weights"""
    kb, ng = -(-K // 128), 128 // group
    b = packed.view(-1, kb, 1024 + 32 * ng)
    codes = _k_codes(b[..., :1024].unflatten(-1, (16, 64)))
    s = _bf16_at(b[..., 1024:]).unflatten(-1, (16, ng))
    return _scaled(codes, s, group).transpose(1, 2).reshape(-1, kb * 128)[:N, :K]


def _tile_values(tiles, hd):
    """fp32 K and V [..., 16 tokens, hd] of tiles"""
    at = (0, 8 * hd, 9 * hd, 17 * hd)
    k = _k_codes(tiles[..., : at[1]].unflatten(-1, (16, hd // 2)))
    ks = _bf16_at(tiles[..., at[1] : at[2]]).unflatten(-1, (16, hd // 32))
    v = _codes(tiles[..., at[2] : at[3]].unflatten(-1, (2, 8, 4, 2, hd // 16)))  # half, piece, t, which, channels
    d = v.dim()
    v = v.permute(*range(d - 5), d - 5, d - 3, d - 2, d - 4, d - 1).flatten(-2).flatten(-4, -2)
    vs = _bf16_at(tiles[..., at[3] :]).unflatten(-1, (hd // 32, 16)).transpose(-1, -2)
    return _scaled(k, ks, 32), _scaled(v, vs, 32)


def _rounded_to_format(x, group):
    """values that the groups of x (last axis) stand for in 4 bits; in 64 bits, as a code next to a border is decided there"""
    n = x.shape[-1]
    x = torch.nn.functional.pad(x.double(), (0, -n % group)).unflatten(-1, (-1, group))
    a = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a / torch.full_like(a, 7))
    s = torch.ldexp(torch.ceil(m * 32), e - 5)
    c = torch.round(x / torch.where(s > 0, s, torch.ones_like(s))).clamp(-7, 7)
    return (c * s).flatten(-2)[..., :n]


def _plain_append(st):
    n_seq, M, page = st["n_seq"], st["M"], st["page"]
    pos = st["pos0"].view(-1, 1).long() + torch.arange(M, device="cuda")
    phys, slot = st["table"].gather(1, pos // page).long(), pos % page
    st["k_pages"][phys, :, slot] = _rounded_to_format(st["k"], 32).to(BF16)
    st["v_pages"][phys, :, slot] = _rounded_to_format(st["v"], 32).to(BF16)
    return st["k_pages"], st["v_pages"]


def _plain_attention(st):
    n_seq, M, Hkv, G, hd, page = (st[n] for n in ("n_seq", "M", "Hkv", "G", "hd", "page"))
    tiles = st["pages"].view(-1, Hkv, page // 16, _tile_bytes(hd))[st["table"].long()]
    k, v = (t.transpose(1, 2).reshape(n_seq, Hkv, 1, -1, hd) for t in _tile_values(tiles, hd))
    q = st["q"].float().view(n_seq, M, Hkv, G, hd).permute(0, 2, 3, 1, 4)
    pos = st["pos0"].view(-1, 1).long() + torch.arange(M, device="cuda")
    sees = (torch.arange(k.shape[3], device="cuda") <= pos.unsqueeze(-1)).view(n_seq, 1, 1, M, -1)
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(hd)
    s = torch.where(sees, s, torch.full_like(s, -math.inf))
    top = s.amax(-1, keepdim=True)
    p = torch.where(sees, torch.exp(s - top), torch.zeros_like(s))
    v = torch.where(sees.any(3).view(n_seq, 1, 1, -1, 1), v, torch.zeros_like(v))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    o = torch.where(pos.view(n_seq, 1, 1, M, 1) >= 0, o, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(n_seq, M, -1).to(BF16)


def _plain(st):
    if st["op"] == "pack":
        return _rounded_to_format(st["w"], st["group"]).to(BF16)
    if st["op"] == "linear":
        return torch.matmul(st["h"].float(), _weight_values(st["packed"], st["N"], st["K"], st["group"]).t())
    return _plain_append(st) if st["op"] == "append" else _plain_attention(st)


# ---------------------------------------------------------------- the framework's calls
def _own(st):
    from paper_2404_16710_b200 import binding as B

    if st["op"] == "pack":
        B.ls_op_quantize_w4(st["w"], st["group"], st["packed"])
        B.ls_op_expand_w4(st["packed"], st["group"], st["out"])
        return st["out"]
    if st["op"] == "linear":
        B.ls_op_linear_w4(st["packed"], st["group"], st["h"], st["out"])
        return st["out"]
    if st["op"] == "append":
        B.ls_op_append_kv4(st["k"], st["v"], st["pos0"], st["page"], st["table"], st["max_seq"], st["pages"], st["status"])
        B.ls_op_expand_kv4(st["pages"], st["pos0"], st["M"], st["page"], st["table"], st["max_seq"], st["table"], st["k_pages"], st["v_pages"], st["status"])
        return st["k_pages"], st["v_pages"]
    B.ls_op_attention_kv4(st["q"], st["pos0"], st["Hkv"], st["hd"], st["page"], st["table"], st["max_seq"], st["pages"], st["out"], st["status"])
    return st["out"]


def run(st):
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------- 64 bits
def _value64(x, group):
    """What x's groups stand for, in 64 bits: the scale found by counting its binary places, the code by a search."""
    n = x.shape[-1]
    out = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    steps = torch.arange(0, 8, device=x.device, dtype=torch.float64)
    for g0 in range(0, n, group):
        part = x[..., g0 : g0 + group].double()
        a = part.abs().max(-1, keepdim=True).values
        unit = torch.exp2(torch.floor(torch.log2(a.clamp(min=1e-300) / 7)) - 4)
        s = torch.round(a / (7 * unit))
        s = (s + (7 * s * unit < a).double()) * unit  # the smallest multiple with 7 s >= a
        s = torch.where(7 * (s - unit) >= a, s - unit, s)
        size = part.abs()
        # the code is the number of midpoints (k + 1/2) s below |x|; one that |x| meets goes to the even code
        code = torch.zeros_like(size)
        for k in range(7):
            mid = (steps[k] + 0.5) * s
            code += (size > mid) | ((size == mid) & (k % 2 == 1) & (a > 0))
        out[..., g0 : g0 + group] = torch.sign(part) * code * s
    return out


def _column_place(C):
    """byte and nibble of every column of a row of codes"""
    C = min(C, 128)
    byte, high = [], []
    for col in range(C):
        j, t, e = col // 32, col % 32 // 8, col % 8
        nib = e // 2 + 4 * (e % 2)
        byte.append(4 * (t * (C // 32) + j) + nib // 2)
        high.append(nib % 2)
    return torch.tensor(byte, device="cuda"), torch.tensor(high, device="cuda")


def _exact_linear(c, st):
    byte, high = _column_place(128)
    kb, ng = -(-c["K"] // 128), 128 // c["group"]
    blocks = st["packed"].view(-1, kb, 1024 + 32 * ng)
    h = torch.nn.functional.pad(st["h"].double(), (0, kb * 128 - c["K"]))
    out = torch.zeros((c["M"], blocks.shape[0], 16), dtype=torch.float64, device="cuda")
    of = torch.arange(128, device="cuda") // c["group"]
    for b in range(kb):
        blk = blocks[:, b]
        codes = ((blk[:, :1024].reshape(-1, 16, 64)[..., byte] >> (4 * high).to(torch.uint8)) & 15).double() - 8
        s = blk[:, 1024:].contiguous().view(BF16).view(-1, 16, ng).double()
        out += torch.einsum("mk,nrk->mnr", h[:, 128 * b : 128 * b + 128], codes * s[..., of])
    return out.reshape(c["M"], -1)[:, : c["N"]]


def _exact_attention(c, st):
    n_seq, M, Hkv, G, hd, page = (c[n] for n in ("n_seq", "M", "Hkv", "G", "hd", "page"))
    byte, high = _column_place(hd)
    of = torch.arange(hd, device="cuda") // 32
    ch = torch.arange(hd, device="cuda")
    tok = torch.arange(16, device="cuda").view(16, 1)
    piece, inside = ch // (hd // 8), ch % (hd // 8)
    vbyte = ((((tok // 8) * 8 + piece) * 4 + (tok // 2) % 4) * 2 + tok % 2) * (hd // 16) + inside // 2
    out = torch.zeros((n_seq, M, Hkv, G, hd), dtype=torch.float64, device="cuda")
    pool = st["pages"].view(-1, Hkv, page // 16, _tile_bytes(hd))
    for b, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        for head in range(Hkv):
            t = pool[st["table"][b, : -(-n // page)].long(), head].reshape(-1, _tile_bytes(hd))
            kc = ((t[:, : 8 * hd].reshape(-1, 16, hd // 2)[..., byte] >> (4 * high).to(torch.uint8)) & 15).double() - 8
            ks = t[:, 8 * hd : 9 * hd].contiguous().view(BF16).view(-1, 16, hd // 32).double()
            k = (kc * ks[..., of]).reshape(-1, hd)[:n]
            vc = ((t[:, 9 * hd : 17 * hd][:, vbyte] >> (4 * (inside % 2)).to(torch.uint8)) & 15).double() - 8
            vs = t[:, 17 * hd :].contiguous().view(BF16).view(-1, hd // 32, 16).double()
            v = (vc * vs[:, of].transpose(1, 2)).reshape(-1, hd)[:n]
            q = st["q"][b].view(M, Hkv, G, hd)[:, head].double()
            for m in range(M):
                see = n - M + m + 1
                w = torch.softmax(q[m] @ k[:see].t() / math.sqrt(hd), -1)
                out[b, m, head] = w @ v[:see]
    return out.view(n_seq, M, -1)


def exact(c, seed):
    st = prepare(c, seed)
    if c["op"] == "pack":
        return _value64(st["w"], c["group"])
    if c["op"] == "linear":
        return _exact_linear(c, st)
    if c["op"] == "attention":
        return _exact_attention(c, st)
    pages = [t.double() for t in (st["k_pages"], st["v_pages"])]
    for out, x in zip(pages, (st["k"], st["v"])):
        y = _value64(x, 32)
        for b in range(c["n_seq"]):
            pos = int(st["pos0"][b]) + torch.arange(c["M"], device="cuda")
            out[st["table"][b, pos // c["page"]].long(), :, pos % c["page"]] = y[b]
    return tuple(pages)
