"""A layer's 8-bit path: the cases that are measured, and the operators' plain forms.

Values are held as a code c (e4m3: finite, at most 448) times a scale that a block shares, a power of two 2^(e - 127)
with e one byte.  A block is 128 columns of one row (activations) or 128 rows by 128 columns (weights).  Its scale is
the smallest power of two s, from 2^-117 on, with max |x| <= 448 s; c is x / s rounded to the nearest code, ties to the
even one.  c * s is exactly a bf16 number.  Codes are [rows, K], scale bytes [rows / block rows, 4 * ceil(K / 512)]: the
bytes of a row's ceil(K / 128) blocks, padded to whole 32-bit words.
"""
import math

import torch

own = False

BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "f32": F32}
EPS = 1e-5


# ---------------------------------------------------------------- cases
def listed():
    return [
        # a checkpoint's feed-forward matrix is laid out once, and read back for an operation in 16 bits
        {"name": "weights 11008x4096", "op": "quantize", "M": 11008, "K": 4096, "rows": 128, "x": "bf16"},
        # attention's output of a ragged prompt, input of the output projection
        {"name": "rows 1030x4096", "op": "quantize", "M": 1030, "K": 4096, "rows": 1, "x": "bf16"},
        # one token's residual stream before a projection: latency alone
        {"name": "norm 1x4096", "op": "norm", "M": 1, "K": 4096, "x": "f32", "d": "bf16"},
        # the residual stream of a block of a prompt, an attention's projection added to it
        {"name": "norm 4096x4096", "op": "norm", "M": 4096, "K": 4096, "x": "f32", "d": "bf16"},
        # a verify pass of seven rows through a feed-forward layer whose width is no power of two
        {"name": "swiglu 7x11008", "op": "swiglu", "M": 7, "K": 11008, "x": "f32"},
        # the same for a block of a prompt
        {"name": "swiglu 4096x11008", "op": "swiglu", "M": 4096, "K": 11008, "x": "bf16"},
        # one token through an output projection
        {"name": "linear 4096x4096 M1", "op": "linear", "M": 1, "N": 4096, "K": 4096, "out": "bf16", "add": False},
        # a verify pass of seven rows through the down projection, added to the residual stream
        {"name": "linear 4096x11008 M7", "op": "linear", "M": 7, "N": 4096, "K": 11008, "out": "f32", "add": True},
        # a large vocabulary's logits for 16 rows (8 sequences of two)
        {"name": "linear 128256x4096 M16", "op": "linear", "M": 16, "N": 128256, "K": 4096, "out": "f32", "add": False},
        # the q|k|v projection of a prompt of a thousand tokens, which leaves a ragged tile
        {"name": "linear 12288x4096 M1030", "op": "linear", "M": 1030, "N": 12288, "K": 4096, "out": "bf16", "add": False},
        # gate and up of a block of a long prompt
        {"name": "linear 22016x4096 M4096", "op": "linear", "M": 4096, "N": 22016, "K": 4096, "out": "bf16", "add": False},
        # the down projection of the same block, added to the residual stream
        {"name": "linear 4096x11008 M4096", "op": "linear", "M": 4096, "N": 4096, "K": 11008, "out": "f32", "add": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("quantize", "norm", "swiglu", "linear", "linear", "linear", "linear"))
    K = 16 * _log(rng, 8, 896)
    x = rng.choice(("bf16", "f32"))
    if op == "quantize":
        rows = rng.choice((1, 128))
        return {"op": op, "M": _log(rng, 1, (1 << 25) // K), "K": K, "rows": rows, "x": x}
    if op == "norm":
        return {"op": op, "M": _log(rng, 1, (1 << 24) // K), "K": K, "x": x, "d": rng.choice(("bf16", "f32", "none"))}
    if op == "swiglu":
        return {"op": op, "M": _log(rng, 1, (1 << 24) // K), "K": K, "x": x}
    M = rng.choice((_log(rng, 1, 16), _log(rng, 1, 4096)))
    top = min(128256, (1 << 38) // (M * K), (1 << 29) // K, (1 << 27) // M)
    return {"op": op, "M": M, "N": _log(rng, min(16, top), top), "K": K, "out": x, "add": rng.choice((False, True))}


def _size(name):
    return {"bf16": 2, "f32": 4, "none": 0}[name]


def _scale_width(K):
    return 4 * -(-K // 512)


def work(c):
    M, K = c["M"], c["K"]
    if c["op"] == "linear":
        N = c["N"]
        moved = N * K + -(-N // 128) * _scale_width(K) + M * (K + _scale_width(K)) + M * N * _size(c["out"]) * (1 + c["add"])
        return {"bytes": moved, "flops": 2 * M * N * K}
    held = M * K + -(-M // c.get("rows", 1)) * _scale_width(K)  # codes and scales
    if c["op"] == "quantize":
        return {"bytes": M * K * (_size(c["x"]) + 2) + held, "flops": 3 * M * K}
    if c["op"] == "norm":
        return {"bytes": M * K * (2 * _size(c["x"]) + _size(c["d"]) + 2) + 2 * K + held, "flops": 7 * M * K}
    return {"bytes": M * K * (2 * _size(c["x"]) + 2) + held, "flops": 8 * M * K}


# ---------------------------------------------------------------- the format
def _blocked(x, rows):
    """[R, rows, C, 128] blocks of x [M, K], padded with zeros"""
    M, K = x.shape
    x = torch.nn.functional.pad(x, (0, -K % 128, 0, -M % rows))
    return x.view(x.shape[0] // rows, rows, x.shape[1] // 128, 128)


def _quantised(x, rows):
    """codes [M, K] and scale exponents [R, C] (scale = 2^e) of x"""
    M, K = x.shape
    b = _blocked(x.float(), rows)
    m, e = torch.frexp(b.abs().amax((1, 3)))
    e = torch.clamp(e - 8 - (m <= 0.875).to(e.dtype), -117, 119)  # 448 = 0.875 * 2^9
    c = torch.ldexp(b, -e[:, None, :, None]).clamp(-448, 448).to(F8)
    return c.flatten(2).flatten(0, 1)[:M, :K].contiguous(), e


def _values(c, e, rows):
    """fp32 [M, K] of codes and exponents"""
    M, K = c.shape
    return torch.ldexp(_blocked(c.float(), rows), e[:, None, :, None]).flatten(2).flatten(0, 1)[:M, :K]


def _bytes(e, K):
    """scale bytes, rows padded to whole words"""
    return torch.nn.functional.pad((e + 127).to(torch.uint8), (0, _scale_width(K) - e.shape[1]))


# ---------------------------------------------------------------- inputs
def _loud(shape, g):
    """activations with a few loud channels, rows of different size"""
    x = torch.randn(shape, generator=g, device="cuda")
    x[:, 5::173] *= 20.0
    return x * torch.exp(torch.randn((shape[0], 1), generator=g, device="cuda"))


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st, M, K = dict(c), c["M"], c["K"]
    if c["op"] == "linear":
        N = c["N"]
        w = torch.randn((N, K), generator=g, device="cuda") * 0.02
        st["wc"], we = _quantised(w, 128)
        del w
        st["hc"], he = _quantised(_loud((M, K), g), 1)
        st["ws"], st["hs"] = _bytes(we, K), _bytes(he, K)
        st["out_t"] = torch.empty((M, N), dtype=TYPES[c["out"]], device="cuda")
        st["add_t"] = torch.randn((M, N), generator=g, device="cuda").to(TYPES[c["out"]]) if c["add"] else None
        return st
    rows = c.get("rows", 1)
    st["codes"] = torch.empty((M, K), dtype=F8, device="cuda")
    st["scales"] = torch.empty((-(-M // rows), _scale_width(K)), dtype=torch.uint8, device="cuda")
    st["values"] = torch.empty((M, K), dtype=BF16, device="cuda")
    t = TYPES[c["x"]]
    if c["op"] == "quantize":
        st["xt"] = (torch.randn((M, K), generator=g, device="cuda") * 0.02).to(t) if rows == 128 else _loud((M, K), g).to(t)
    elif c["op"] == "norm":
        st["xt"] = _loud((M, K), g).to(t)
        st["dt"] = None if c["d"] == "none" else torch.randn((M, K), generator=g, device="cuda").to(TYPES[c["d"]])
        st["gain"] = (1 + 0.1 * torch.randn((K,), generator=g, device="cuda")).to(BF16)
        st["x_out"] = torch.empty_like(st["xt"])
    else:
        st["gu"] = torch.randn((M, 2 * K), generator=g, device="cuda").to(t)  # gate | up, as one projection leaves them
    return st


# ---------------------------------------------------------------- plain forms
def _held(y, rows):
    """what y stands for in 8 bits, in bf16"""
    return _values(*_quantised(y, rows), rows).to(BF16)


def _exponents(s, K):
    return s[:, : -(-K // 128)].to(torch.int32) - 127


def _plain(st):
    K = st["K"]
    if st["op"] == "quantize":
        return _held(st["xt"], st["rows"])
    if st["op"] == "norm":
        x = st["xt"].float()
        if st["dt"] is not None:
            x = x + st["dt"].float()
        x_out = x.to(st["xt"].dtype)
        x = x_out.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * st["gain"].float()
        return x_out, _held(y, 1)
    if st["op"] == "swiglu":
        gate, up = st["gu"].float().split(K, 1)
        return _held(gate / (1 + torch.exp(-gate)) * up, 1)
    h = _values(st["hc"], _exponents(st["hs"], K), 1)
    w = _values(st["wc"], _exponents(st["ws"], K), 128)
    y = torch.matmul(h, w.t())
    if st["add_t"] is not None:
        y = y + st["add_t"].float()
    return y.to(st["out_t"].dtype)


# ---------------------------------------------------------------- the framework's calls
def _own(st):
    from paper_2404_16710_b200 import binding as B

    if st["op"] == "linear":
        B.ls_op_linear_f8(st["wc"], st["ws"], st["hc"], st["hs"], st["out_t"], add=st["add_t"])
        return st["out_t"]
    rows = 1
    if st["op"] == "quantize":
        rows = st["rows"]
        B.ls_op_quantize_f8(st["xt"], st["codes"], st["scales"], rows)
    elif st["op"] == "norm":
        B.ls_op_rmsnorm_f8(st["xt"], st["gain"], EPS, st["codes"], st["scales"], delta=st["dt"], x_out=st["x_out"])
    else:
        K = st["K"]
        B.ls_op_swiglu_f8(st["gu"][:, :K], st["gu"][:, K:], st["codes"], st["scales"])
    B.ls_op_expand_f8(st["codes"], st["scales"], st["values"], rows)
    return (st["x_out"], st["values"]) if st["op"] == "norm" else st["values"]


def run(st):
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------- 64 bits
def _held64(y, rows):
    """What y (64 bits) stands for in 8 bits: block by block of columns, the scale found by its logarithm and set right,
    the code by rounding to the spacing of its binade."""
    M, K = y.shape
    out = torch.empty_like(y)
    for k in range(0, K, 128):
        part = y[:, k : k + 128]
        a = part.abs().amax(1)
        if rows > 1:
            a = torch.cat([p.amax().expand(len(p)) for p in a.split(rows)])
        s = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0**-200))) - 10)
        for _ in range(4):
            s = torch.where(a > 448 * s, 2 * s, s)
        s = s.clamp(min=2.0**-117)[:, None]
        v = part / s
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0**-6))) - 3)
        out[:, k : k + 128] = (torch.round(v / step) * step).clamp(-448, 448) * s
    return out


def _codes64(c, s, rows):
    """64 bits [M, K] of codes and scale bytes, the codes taken apart by their fields"""
    M, K = c.shape
    u = c.view(torch.uint8).to(torch.int16)
    field, m = (u >> 3) & 15, (u & 7).double()
    v = torch.where(field > 0, (8 + m) * torch.exp2(field.double() - 10), m * 2.0**-9)
    v = torch.where(u > 127, -v, v)
    at = torch.arange(M, device="cuda") // rows
    for k in range(0, K, 128):
        v[:, k : k + 128] *= torch.exp2(s[at, k // 128].double() - 127)[:, None]
    return v


def exact(c, seed):
    st, M, K = prepare(c, seed), c["M"], c["K"]
    if c["op"] == "quantize":
        return _held64(st["xt"].double(), c["rows"])
    if c["op"] == "norm":
        x = st["xt"].double()
        if st["dt"] is not None:
            x = x + st["dt"].double()
        x_out = x
        x = x.to(st["xt"].dtype).double()  # the norm is of what is kept
        rms = torch.sqrt(torch.linalg.vector_norm(x, dim=1, keepdim=True) ** 2 / K + EPS)
        return x_out, _held64(x / rms * st["gain"].double(), 1)
    if c["op"] == "swiglu":
        gate, up = st["gu"][:, :K].double(), st["gu"][:, K:].double()
        return _held64(gate * torch.sigmoid(gate) * up, 1)
    h = _codes64(st["hc"], st["hs"], 1)
    out = torch.empty((M, c["N"]), dtype=torch.float64, device="cuda")
    for n in range(0, c["N"], 8192):  # whole blocks of rows
        w = _codes64(st["wc"][n : n + 8192], st["ws"][n // 128 : n // 128 + 64], 128)
        out[:, n : n + 8192] = h @ w.t()
    return out if st["add_t"] is None else out + st["add_t"].double()
