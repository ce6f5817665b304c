"""The 8-bit path of a layer against the format's definition and 64-bit arithmetic (tests/f8_reference.py).

Conversions are exact: bytes have to be equal.  Tolerances of the computed results, derived:
* linear: products of two codes are exact (4 by 4 significant bits).  Every one of the K / 32 tensor-core sums, the
  K / 128 scaled additions and the 8 that join parts is off by at most one unit of its result's last place (the tensor
  cores may truncate), 2^-23, of a partial sum that is at most sum |h w|; sums that begin with `add` are rounded when a part of 2048
  columns is added and when up to four parts are joined, K / 2048 + 4 times by 2^-24 of at most |add| + sum |h w|; a bf16 result is rounded once, 2^-8 of its value.
* rmsnorm, swiglu: y is off by at most delta before it is rounded to a code, so the scale byte is that of y (1 - delta) or
  of y (1 + delta), and the code lies between those of y (1 - delta) and y (1 + delta) under that scale.
  rmsnorm: a sum of D squares of which no more than D / 64 + 32 are added in a chain, half of that (the root), the
  division, root and two products: delta = (D / 128 + 24) 2^-24.  swiglu: an exponential off by 2^-22 and a rounding of its
  correction (2^-24), a sum (2^-24), a reciprocal to a unit of its last place (2^-23) and two products (2^-24 each): 10 2^-24 in all,
  delta = 2^-20.
"""
import numpy as np
import pytest
import torch

from paper_2404_16710_b200 import binding as B
from tests import f8_reference as R
from tests.helpers import vals

pytestmark = pytest.mark.gpu
F8, BF16, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32
SWIGLU_DELTA = 2.0 ** -20


def rnd(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda") * scale


def bits(codes):
    return codes.view(torch.uint8).cpu().numpy()


def empty_held(M, K, rows=1):
    codes = torch.full((M, K), 0x55, dtype=torch.uint8, device="cuda").view(F8)
    return codes, torch.full((-(-M // rows), R.scale_width(K)), 0xEE, dtype=torch.uint8, device="cuda")


def quantised(x, rows=1):
    codes, scales = empty_held(*x.shape, rows)
    B.ls_op_quantize_f8(x, codes, scales, rows)
    return codes, scales


def held_values(codes, scales, rows=1):
    return R.values(bits(codes), scales.cpu().numpy(), rows)


def f64(t):
    return t.cpu().double().numpy()


def awkward(M, K, seed):
    """fp32 values over the whole range: rows of very different size, zeros, subnormal and the largest numbers, borders
    between codes (exact ties among them), NaN and infinities"""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((M, K)) * np.exp2(rng.integers(-149, 126, (M, 1)).astype(np.float64))).astype(np.float32)
    x[1] = 0
    x[2, ::2] = -0.0
    x[3] = np.float32(2.0 ** -149)
    x[4] = np.finfo(np.float32).max * np.where(rng.random(K) < 0.5, 1, -1)
    mid = (R.CODE_VALUES[:126] + R.CODE_VALUES[1:127]) / 2  # every tie, and its neighbours
    ties = np.concatenate([mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(1e9))])
    for r, e in ((5, 0), (6, -60), (7, 100), (8, -117)):
        t = np.resize(ties, K)
        t[:: 128] = 448.0  # fixes every block's scale
        x[r] = (t * 2.0 ** e * np.where(rng.random(K) < 0.5, 1, -1)).astype(np.float32)
    x[9, ::128] = np.float32(448 * 2.0 ** 3)
    x[10, ::128] = np.nextafter(np.float32(448 * 2.0 ** 3), np.float32(1e9))
    x[11, 5], x[11, K - 1] = np.nan, np.inf
    x[12, 130 % K] = -np.inf
    x[13, 7] = np.float32(2.0 ** -118) * 448
    return x


# ------------------------------------------------------------------ conversion
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K", [(1, 16), (1, 4096), (3, 144), (17, 528), (128, 128), (129, 1040), (300, 2064)])
def test_quantize_and_expand(M, K, rows, dtype):
    x = (rnd((M, K), M + K) * torch.exp(2 * rnd((M, 1), 5))).to(dtype)
    codes, scales = quantised(x, rows)
    assert np.array_equal(scales.cpu().numpy(), R.scale_bytes(f64(x), rows))
    assert np.array_equal(bits(codes), R.codes(f64(x), rows))
    out = torch.full((M, K), 7.0, dtype=BF16, device="cuda")
    B.ls_op_expand_f8(codes, scales, out, rows)
    assert np.array_equal(vals(out), held_values(codes, scales, rows))


@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_at_the_ends_of_the_range(rows):
    x = awkward(40, 1040, 3)
    if rows == 128:  # each kind of row fills a block of its own
        x = np.repeat(x, 128, 0)
    codes, scales = quantised(torch.from_numpy(x).cuda(), rows)
    assert np.array_equal(scales.cpu().numpy(), R.scale_bytes(x.astype(np.float64), rows))
    assert np.array_equal(bits(codes), R.codes(x.astype(np.float64), rows))
    xb = torch.from_numpy(x).cuda().to(BF16)
    codes, scales = quantised(xb, rows)
    assert np.array_equal(scales.cpu().numpy(), R.scale_bytes(f64(xb), rows))
    assert np.array_equal(bits(codes), R.codes(f64(xb), rows))
    out = torch.empty(xb.shape, dtype=BF16, device="cuda")
    B.ls_op_expand_f8(codes, scales, out, rows)
    assert np.array_equal(vals(out), held_values(codes, scales, rows), equal_nan=True)


def test_expand_every_code_under_every_scale():
    codes = torch.arange(256, dtype=torch.int16).to(torch.uint8).repeat(256, 2).cuda().view(F8)
    scales = torch.zeros((256, 4), dtype=torch.uint8)
    scales[:, :] = torch.arange(256).to(torch.uint8)[:, None]
    out = torch.empty((256, 512), dtype=BF16, device="cuda")
    B.ls_op_expand_f8(codes, scales.cuda(), out)
    want = R.values(bits(codes), scales.numpy(), 1)
    inside = scales.numpy()[:, 0]  # what the quantiser writes; beyond, bf16 rounds or overflows
    with np.errstate(over="ignore"):
        rounded = torch.from_numpy(want.astype(np.float32)).to(BF16).double().numpy()
    assert np.array_equal(vals(out), rounded, equal_nan=True)
    keep = (inside >= 10) & (inside <= 246)
    exact = keep[:, None] & ~((inside == 246)[:, None] & (np.abs(want) > 448 * 2.0 ** 119))
    assert np.array_equal(rounded[exact], want[exact], equal_nan=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantize_rows_with_a_stride_and_nothing_beside_them(dtype):
    base = rnd((9, 2 * 272), 8).to(dtype)
    part = base[:, 272:]
    codes = torch.full((11, 272), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((11, 4), 0xEE, dtype=torch.uint8, device="cuda")
    for rows, n in ((1, 9), (128, 1)):
        codes.fill_(0x55), scales.fill_(0xEE)
        B.ls_op_quantize_f8(part, codes[1:10].view(F8), scales[1:1 + n], rows)
        assert np.array_equal(codes[1:10].cpu().numpy(), R.codes(f64(part), rows))
        assert (codes[[0, 10]] == 0x55).all() and (scales[0] == 0xEE).all() and (scales[1 + n:] == 0xEE).all()


def test_offsets_beyond_32_bits():
    M, K = 70000, 32768  # 2.3e9 codes
    x = torch.zeros((M, K), dtype=BF16, device="cuda")
    at = [0, 65535, 65536, M - 1]
    x[at] = rnd((len(at), K), 1).to(BF16)
    for rows in (1, 128):
        codes, scales = quantised(x, rows)
        pick = at if rows == 1 else [0, M - 1]
        s = scales[[r // rows for r in pick]].cpu().numpy()
        if rows == 1:
            assert np.array_equal(s, R.scale_bytes(f64(x[pick]), 1))
        got = R.values(bits(codes[pick]), s, 1)
        assert (np.abs(got - f64(x[pick])) <= 2.0 ** -4 * np.abs(f64(x[pick])) + 2.0 ** -10 * 2.0 ** (s.max().astype(float) - 127)).all()
        out = x
        B.ls_op_expand_f8(codes, scales, out, rows)
        assert np.array_equal(vals(out[pick]), got)
        assert not out[1:65535].any()


# ------------------------------------------------------------------ rmsnorm, swiglu
def check_rounded(codes, scales, y, delta):
    """codes and scale bytes are those of something within delta of y (64 bits)"""
    b = scales.cpu().numpy()
    lo_b, hi_b = R.scale_bytes(y * (1 - delta), 1), R.scale_bytes(y * (1 + delta), 1)
    assert ((b == lo_b) | (b == hi_b)).all()
    s = R.scales(b, *y.shape, 1)
    got = R.values(bits(codes), b, 1)
    fine = ~np.isnan(s)
    assert np.array_equal(np.isnan(got), ~fine)

    def rounded(v):  # to the codes' spacing under the scale that was written
        v = np.where(fine, v, 0) / np.where(fine, s, 1)
        step = np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
        return np.clip(np.round(v / step) * step, -448, 448)
    a, c = rounded(y * (1 - delta)), rounded(y * (1 + delta))
    v = np.where(fine, got / np.where(fine, s, 1), 0)
    assert ((v >= np.minimum(a, c)) & (v <= np.maximum(a, c))).all()
    assert (v != rounded(y)).mean() <= 1e-3


def added(x, d):
    """x + d in fp32, rounded to x's type (as a tensor)"""
    return x if d is None else (x.float() + d.float()).to(x.dtype)


def normed(x, gain, eps):
    v = f64(x)
    return v / np.sqrt((v * v).mean(1, keepdims=True) + eps) * f64(gain)


def norm_delta(D):
    return (D / 128 + 24) * 2.0 ** -24


@pytest.mark.parametrize("x_type,d_type", [(F32, BF16), (F32, F32), (BF16, BF16), (BF16, F32), (F32, None), (BF16, None)])
@pytest.mark.parametrize("M,D", [(1, 16), (1, 4096), (5, 272), (7, 5120), (300, 1040), (301, 4096), (297, 8192), (2, 16384),
                                 (300, 16400), (3, 40000), (299, 33008)])
def test_rmsnorm(M, D, x_type, d_type):
    x = (rnd((M, D), M + D) * torch.exp(rnd((M, 1), 1))).to(x_type)
    d = None if d_type is None else rnd((M, D), 2).to(d_type)
    gain = (1 + 0.1 * rnd((D,), 3)).to(BF16)
    want = added(x, d)
    codes, scales = empty_held(M, D)
    x_out = torch.full_like(x, float("nan"))
    B.ls_op_rmsnorm_f8(x, gain, 1e-5, codes, scales, delta=d, x_out=x_out)
    assert torch.equal(x_out, want)
    check_rounded(codes, scales, normed(want, gain, 1e-5), norm_delta(D))
    again = empty_held(M, D)  # the sum not kept, then in place: the same bytes
    B.ls_op_rmsnorm_f8(x, gain, 1e-5, *again, delta=d)
    assert torch.equal(again[0].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(again[1], scales)
    for target in (x, d) if d is not None and d.dtype is x.dtype else (x,):
        xs, ds = x.clone(), None if d is None else d.clone()
        again = empty_held(M, D)
        B.ls_op_rmsnorm_f8(xs, gain, 1e-5, *again, delta=ds, x_out=xs if target is x else ds)
        assert torch.equal(xs if target is x else ds, want)
        assert torch.equal(again[0].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(again[1], scales)


def test_rmsnorm_strided_rows_and_nothing_beside_them():
    M, D = 6, 400
    x, d = rnd((M, 2 * D), 1), rnd((M, D + 8), 2).to(BF16)
    gain = torch.ones(D, dtype=BF16, device="cuda")
    keep = x.clone()
    codes, scales = empty_held(M, D)
    B.ls_op_rmsnorm_f8(x[:, D:], gain, 1e-5, codes, scales, delta=d[:, :D], x_out=x[:, :D])
    want = keep[:, D:] + d[:, :D].float()
    assert torch.equal(x[:, :D], want) and torch.equal(x[:, D:], keep[:, D:])
    check_rounded(codes, scales, normed(want, gain, 1e-5), norm_delta(D))


def test_rmsnorm_rows_of_zeros_and_rows_that_are_not_finite():
    x = rnd((6, 512), 4)
    x[1] = 0
    x[2, 300] = float("nan")
    x[3, 5] = float("inf")
    x[4] *= 1e-25
    gain = torch.ones(512, dtype=BF16, device="cuda")
    codes, scales = empty_held(6, 512)
    B.ls_op_rmsnorm_f8(x, gain, 1e-5, codes, scales)
    assert (held_values(codes[1:2], scales[1:2]) == 0).all()
    assert (scales[2] == 255).all() and not codes[2].view(torch.uint8).any()
    got = held_values(codes[3:4], scales[3:4])[0]  # inf / inf, and the rest by an infinite norm
    assert np.isnan(got[:128]).all() and (got[128:] == 0).all()
    for r in (0, 4, 5):
        check_rounded(codes[r:r + 1], scales[r:r + 1], normed(x[r:r + 1], gain, 1e-5), norm_delta(512))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,F", [(1, 16), (1, 11008), (7, 11008), (3, 272), (130, 1376), (1025, 528)])
def test_swiglu(M, F, dtype):
    gu = (2 * rnd((M, 2 * F), M + F)).to(dtype)
    codes, scales = empty_held(M, F)
    B.ls_op_swiglu_f8(gu[:, :F], gu[:, F:], codes, scales)
    g, u = f64(gu[:, :F]), f64(gu[:, F:])
    check_rounded(codes, scales, g / (1 + np.exp(-g)) * u, SWIGLU_DELTA)
    again = empty_held(M, F)  # two tensors instead of two halves
    B.ls_op_swiglu_f8(gu[:, :F].contiguous(), gu[:, F:].contiguous(), *again)
    assert torch.equal(again[0].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(again[1], scales)


def test_swiglu_far_gates_and_values_that_are_not_finite():
    g = torch.zeros((4, 256), device="cuda")
    g[0] = torch.linspace(-200, 200, 256)
    g[1, 3], g[2, 200], g[3] = float("nan"), float("inf"), -1e30
    u = torch.ones_like(g)
    codes, scales = empty_held(4, 256)
    B.ls_op_swiglu_f8(g, u, codes, scales)
    x = f64(g[0:1])
    with np.errstate(over="ignore"):
        check_rounded(codes[0:1], scales[0:1], x / (1 + np.exp(-x)), SWIGLU_DELTA)
    got = held_values(codes, scales)
    assert np.isnan(got[1, :128]).all() and (got[1, 128:] == 0).all()
    assert (got[2, :128] == 0).all() and np.isnan(got[2, 128:]).all()
    assert (got[3] == 0).all()


# ------------------------------------------------------------------ linear
def reference(w, h):
    """(out, sum of magnitudes) in 64 bits of (codes, scales) pairs, on the GPU for size"""
    def value(pair, rows):
        codes, s = pair
        M, K = codes.shape
        e = s[:, : -(-K // 128)].double()
        e = torch.where(e == 255, torch.full_like(e, float("nan")), torch.exp2(e - 127))
        return codes.double() * e.repeat_interleave(rows, 0)[:M].repeat_interleave(128, 1)[:, :K]
    wv, hv = value(w, 128), value(h, 1)
    return hv @ wv.t(), hv.abs() @ wv.abs().t()


def linear_tol(K, spread, out_type, ref, base=None):
    tol = (K / 32 + K / 128 + 12) * 2.0 ** -23 * spread
    total = ref if base is None else ref + base
    if base is not None:
        tol = tol + (K / 2048 + 4) * 2.0 ** -24 * (base.abs() + spread)
    return tol + (2.0 ** -8 * total.abs() if out_type is BF16 else 0.0)


def loud(M, K, seed):
    x = rnd((M, K), seed) * torch.exp(rnd((M, 1), seed + 1))
    x[:, 3::97] *= 30
    return x


def pair_of(M, N, K, seed=1):
    return quantised((rnd((N, K), seed, 0.02)), 128), quantised(loud(M, K, seed + 1))


SHAPES = [(1, 1, 16), (1, 128, 128), (1, 4096, 4096), (2, 200, 144), (7, 333, 1040), (8, 64, 11008), (9, 130, 2064), (16, 4100, 4096),
          (16, 1000, 14336), (5, 32000, 528), (17, 300, 1040), (32, 129, 4096), (33, 4096, 656), (64, 257, 2048), (65, 500, 400),
          (100, 1000, 4096), (128, 4096, 1040), (129, 384, 1040), (255, 256, 528), (256, 512, 4096), (257, 1030, 1040), (300, 129, 4112),
          (1030, 770, 2064), (1025, 2600, 400), (2050, 300, 144), (700, 4096, 4096),
          (130, 300, 8208), (512, 512, 4112), (300, 129, 14336), (241, 1000, 4096), (777, 1030, 9232), (1919, 134, 2448), (2050, 250, 4624),
          (3, 70, 262160), (150, 70, 262160)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("out_type,add", [(F32, False), (F32, True), (BF16, False), (BF16, True)])
def test_linear(M, N, K, out_type, add):
    w, h = pair_of(M, N, K)
    ref, spread = reference(w, h)
    out = torch.full((M, N), float("nan"), dtype=out_type, device="cuda")
    base = rnd((M, N), 5).to(out_type) if add else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ls_op_linear_f8(*w, *h, out, add=base, status=status)
    want = ref if base is None else ref + base.double()
    far = (out.double() - want).abs()
    assert (far <= linear_tol(K, spread, out_type, ref, None if base is None else base.double())).all(), far.max().item()
    if out_type is F32 and not add:
        assert (out.double() - want).norm() <= 1e-6 * want.norm()
    if add:  # onto itself: the same bits
        B.ls_op_linear_f8(*w, *h, base, add=base)
        assert torch.equal(base, out)
    assert status.item() == 0


@pytest.mark.parametrize("out_type", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [(3, 333, 528), (70, 333, 528), (300, 517, 528), (520, 260, 1040)])
def test_linear_odd_addresses_and_strides_and_nothing_beside_them(M, N, K, out_type):
    w, h = pair_of(M, N, K, 7)
    ref, spread = reference(w, h)
    for off, ld in ((1, N + 5), (3, N + 3), (0, N + 8)):
        buf = torch.full((M + 1, ld), -7.0, dtype=out_type, device="cuda")
        out = buf.view(-1)[off: off + M * ld].view(M, ld)[:, :N]
        B.ls_op_linear_f8(*w, *h, out)
        assert ((out.double() - ref).abs() <= linear_tol(K, spread, out_type, ref)).all()
        rest = buf.clone()
        rest.view(-1)[off: off + M * ld].view(M, ld)[:, :N] = -7.0
        assert (rest == -7.0).all()
        base = rnd((M + 1, ld + 2), 3).to(out_type).view(-1)[off: off + M * (ld + 2)].view(M, ld + 2)[:, :N]
        B.ls_op_linear_f8(*w, *h, out, add=base)
        assert ((out.double() - ref - base.double()).abs() <= linear_tol(K, spread, out_type, ref, base.double())).all()


@pytest.mark.parametrize("N,K", [(304, 1040), (4096, 4096), (4096, 11008), (128, 14336), (18944, 528), (33000, 272)])
def test_linear_rows_do_not_depend_on_pass_size(N, K):
    w, h = pair_of(16, N, K, 11)
    full = torch.empty((16, N), device="cuda")
    B.ls_op_linear_f8(*w, *h, full)
    for m0, M in ((0, 1), (3, 2), (0, 4), (5, 7), (8, 8), (2, 9), (0, 15)):
        out = torch.full((M, N), float("nan"), device="cuda")
        B.ls_op_linear_f8(*w, h[0][m0:m0 + M], h[1][m0:m0 + M], out)
        assert torch.equal(out, full[m0:m0 + M]), M


@pytest.mark.parametrize("M", [1, 16, 30, 64, 100, 300])
def test_linear_chained_gives_the_same_bits(M):
    """chained operations run beside one another, on shorter rings of stages: the sums are the same"""
    N, K = 1000, 4112
    w, h = pair_of(M, N, K, 17)
    alone, chained = (torch.full((M, N), float("nan"), device="cuda") for _ in range(2))
    B.ls_op_linear_f8(*w, *h, alone)
    torch.cuda.synchronize()
    B.ls_op_chain(True)
    try:
        for _ in range(3):
            B.ls_op_linear_f8(*w, *h, chained)
    finally:
        B.ls_op_chain(False)
    assert torch.equal(alone, chained)


@pytest.mark.parametrize("M,N,K", [(5, 300, 1040), (90, 300, 1040), (300, 700, 1040)])
def test_linear_any_scales_and_blocks_that_are_not_finite(M, N, K):
    """bytes of other quantisers, rubbish behind the last block's byte, NaN blocks on either side"""
    w, h = pair_of(M, N, K, 13)
    g = torch.Generator(device="cuda").manual_seed(1)
    w[1][:, :9] = torch.randint(60, 140, (w[1].shape[0], 9), generator=g, device="cuda").to(torch.uint8)
    h[1][:, :9] = torch.randint(60, 140, (M, 9), generator=g, device="cuda").to(torch.uint8)
    h[1][0, :9] = 0  # 2^-127
    w[1][:, 9:], h[1][:, 9:] = 255, 255
    ref, spread = reference(w, h)
    out = torch.empty((M, N), device="cuda")
    B.ls_op_linear_f8(*w, *h, out)
    tiny = 2.0 ** -126  # products below the normal numbers may be lost
    assert ((out.double() - ref).abs() <= linear_tol(K, spread, F32, ref) + tiny).all()
    h[1][2, 8], w[1][1, 0] = 255, 255
    B.ls_op_linear_f8(*w, *h, out)
    bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    bad[2], bad[:, 128:256] = True, True
    assert torch.equal(out.isnan(), bad)
    assert ((out.double() - ref).abs() <= linear_tol(K, spread, F32, ref) + tiny)[~bad].all()
    h[1][2, 8], w[1][1, 0] = 127, 127
    h[0].view(torch.uint8)[1, 4] = 0x7F  # a NaN code of another quantiser
    B.ls_op_linear_f8(*w, *h, out)
    bad.fill_(False)
    bad[1] = True
    assert torch.equal(out.isnan(), bad)


@pytest.mark.parametrize("M", [3, 40])
def test_linear_weights_beyond_32_bits(M):
    N, K = 131072, 17408  # 2.3e9 codes
    codes, scales = empty_held(N, K, 128)
    codes.view(torch.uint8).zero_(), scales.fill_(120)
    rows = [0, 5, 65536, 123456, N - 1]
    some = torch.randint(0, 126, (len(rows), K), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.uint8)
    codes.view(torch.uint8)[rows] = some
    h = quantised(loud(M, K, 2))
    out = torch.empty((M, N), device="cuda")
    B.ls_op_linear_f8(codes, scales, *h, out)
    wv = torch.from_numpy(R.CODE_VALUES[some.cpu().numpy()] * 2.0 ** -7).cuda()
    hv = torch.from_numpy(held_values(*h)).cuda()
    ref, spread = hv @ wv.t(), hv.abs() @ wv.abs().t()
    assert ((out[:, rows].double() - ref).abs() <= linear_tol(K, spread, F32, ref)).all()
    out[:, rows] = 0
    assert not out.any()


@pytest.mark.parametrize("M", [300, 4100])
def test_linear_outputs_beyond_32_bits(M):
    N, K = (3600000, 144) if M == 300 else (530000, 144)  # 1.1e9 and 2.2e9 outputs, of 2 bytes
    w, h = quantised(rnd((N, K), 1, 0.02).to(BF16), 128), quantised(loud(M, K, 2))
    out = torch.zeros((M, N), dtype=BF16, device="cuda")
    B.ls_op_linear_f8(*w, *h, out)
    cols = [0, 130, N // 2, N - 129, N - 1]
    for c in cols:
        c0 = c // 128 * 128
        ref, spread = reference((w[0][c0:c0 + 128], w[1][c // 128:c // 128 + 1]), h)
        got = out[:, c0:c0 + 128].double()
        assert ((got - ref).abs() <= linear_tol(K, spread, BF16, ref)).all()


# ------------------------------------------------------------------ as they are used
def layer(x, delta, gain, w_gu, w_down, bufs, F):
    """the feed-forward half of a layer: x + delta, norm, gate and up, SwiGLU, down projection onto x"""
    B.ls_op_rmsnorm_f8(x, gain, 1e-5, *bufs["h"], delta=delta, x_out=x)
    B.ls_op_linear_f8(*w_gu, *bufs["h"], bufs["gu"])
    B.ls_op_swiglu_f8(bufs["gu"][:, :F], bufs["gu"][:, F:], *bufs["a"])
    B.ls_op_linear_f8(*w_down, *bufs["a"], x, add=x)


def layer_bufs(M, D, F):
    return {"h": empty_held(M, D), "gu": torch.empty((M, 2 * F), dtype=BF16, device="cuda"), "a": empty_held(M, F)}


@pytest.mark.parametrize("M", [1, 7, 40, 300])
@pytest.mark.parametrize("chained", [False, True])
def test_a_feed_forward_layer(M, chained):
    """each operation within its tolerance of 64-bit arithmetic on what the one before it left, weights packed right before"""
    D, F = 1024, 2752
    x, delta = rnd((M, D), 1), rnd((M, D), 2).to(BF16)
    gain = (1 + 0.1 * rnd((D,), 3)).to(BF16)
    wg, wd = rnd((2 * F, D), 4, 0.02).to(BF16), rnd((D, F), 5, 0.02).to(BF16)
    bufs, x0 = layer_bufs(M, D, F), x.clone()
    torch.cuda.synchronize()
    B.ls_op_chain(chained)
    try:
        w_gu, w_down = quantised(wg, 128), quantised(wd, 128)
        layer(x, delta, gain, w_gu, w_down, bufs, F)
    finally:
        B.ls_op_chain(False)
    torch.cuda.synchronize()
    x1 = x0 + delta.float()
    check_rounded(*bufs["h"], normed(x1, gain, 1e-5), norm_delta(D))
    ref, spread = reference(w_gu, bufs["h"])
    assert ((bufs["gu"].double() - ref).abs() <= linear_tol(D, spread, BF16, ref)).all()
    g, u = f64(bufs["gu"][:, :F]), f64(bufs["gu"][:, F:])
    check_rounded(*bufs["a"], g / (1 + np.exp(-g)) * u, SWIGLU_DELTA)
    ref, spread = reference(w_down, bufs["a"])
    assert ((x.double() - x1.double() - ref).abs() <= linear_tol(F, spread, F32, ref, x1.double())).all()
    # and the whole near the layer in 64 bits without any 8-bit rounding: two roundings of 2^-4 at most, of independent signs
    hv = normed(x1, gain, 1e-5) @ f64(wg).T
    want = f64(x1) + (hv[:, :F] / (1 + np.exp(-hv[:, :F])) * hv[:, F:]) @ f64(wd).T
    assert np.linalg.norm(f64(x) - want) <= 2.0 ** -3 * np.linalg.norm(want - f64(x1))


def test_captured_replayed_and_on_two_streams():
    """one graph replayed on new inputs, and another layer's eager calls on a second stream beside it, give the eager bits"""
    D, F = 512, 1408
    gain = torch.ones(D, dtype=BF16, device="cuda")
    sets = []
    for M, seed in ((5, 1), (200, 2)):
        w = quantised(rnd((2 * F, D), seed, 0.02), 128), quantised(rnd((D, F), seed + 5, 0.02), 128)
        xs = [rnd((M, D), seed + 10 + i) for i in range(3)]
        eager = []
        for x in xs:
            y = x.clone()
            layer(y, None, gain, *w, layer_bufs(M, D, F), F)
            eager.append(y)
        sets.append((w, xs, eager, layer_bufs(M, D, F), torch.empty_like(xs[0])))
    torch.cuda.synchronize()
    graphs = []
    for w, xs, _, bufs, x in sets:
        g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g, stream=st):
            layer(x, None, gain, *w, bufs, F)
        graphs.append((g, st))
    for i in (2, 0, 1):
        got = []
        for (g, st), (w, xs, eager, bufs, x) in zip(graphs, sets):
            with torch.cuda.stream(st):
                x.copy_(xs[i])
                g.replay()
            with torch.cuda.stream(torch.cuda.Stream()):
                y = xs[i].clone()
                layer(y, None, gain, *w, layer_bufs(y.shape[0], D, F), F)
                got.append(y)
        torch.cuda.synchronize()
        for (_, _, eager, _, x), y in zip(sets, got):
            assert torch.equal(x, eager[i]) and torch.equal(y, eager[i])


# ------------------------------------------------------------------ borders
# A value computed in fp32 next to a border between two codes is decided in 64 bits: codes at and above 2^-6 s and all scales are those
# of the values in 64 bits.
def check_exact(codes, scales, want):
    assert np.array_equal(scales.cpu().numpy(), R.scale_bytes(want, 1))
    s = R.scales(scales.cpu().numpy(), *want.shape, 1)
    assert ((bits(codes) == R.codes(want, 1)) | (np.abs(want) < 2.0 ** -6 * (1 + 2.0 ** -20) * s)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,F", [(1000, 2064), (300, 12304), (500, 4112)])
def test_swiglu_codes_next_to_a_border(M, F, dtype):
    gu = (2 * rnd((M, 2 * F), 5)).to(dtype)
    codes, scales = empty_held(M, F)
    B.ls_op_swiglu_f8(gu[:, :F], gu[:, F:], codes, scales)
    g, u = f64(gu[:, :F]), f64(gu[:, F:])
    check_exact(codes, scales, g / (1 + np.exp(-g)) * u)


def test_swiglu_scales_next_to_a_border():
    """each block's largest value lies within a few units of 448 2^k, on either side, in every place of the block"""
    M, F = 64, 1040
    rng = np.random.default_rng(3)
    g = rng.uniform(-3, 3, (M, F)).astype(np.float32)
    u = rng.uniform(-1, 1, (M, F)).astype(np.float32)
    for m in range(M):
        for b in range(-(-F // 128)):
            k = min(128 * b + (2 * m + b) % 128, F - 1)
            g[m, k] = rng.uniform(0.5, 4)
            y = float(g[m, k]) / (1 + np.exp(-float(g[m, k])))
            v = np.float32(448 * 2.0 ** rng.integers(-4, 5) / y)
            for _ in range(m % 3):
                v = np.nextafter(v, np.float32(0 if b % 2 else 1e9))
            u[m, k] = v
    codes, scales = empty_held(M, F)
    B.ls_op_swiglu_f8(torch.from_numpy(g).cuda(), torch.from_numpy(u).cuda(), codes, scales)
    x = g.astype(np.float64)
    check_exact(codes, scales, x / (1 + np.exp(-x)) * u.astype(np.float64))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,D", [(700, 2064), (400, 4096), (300, 8208), (40, 12304), (9, 40000)])
@pytest.mark.parametrize("form", ["alone", "added", "kept"])
def test_norm_codes_next_to_a_border(M, D, dtype, form):
    """multiples of 1/4 up to 4: their squares' sums are exact, so that nothing but the borders decides"""
    g = torch.Generator(device="cuda").manual_seed(M + D)
    x = (torch.randint(-8, 9, (M, D), generator=g, device="cuda") / 4).to(dtype)
    d = None if form == "alone" else (torch.randint(-8, 9, (M, D), generator=g, device="cuda") / 4).to(BF16)
    gain = (1 + 0.1 * rnd((D,), 3)).to(BF16)
    codes, scales = empty_held(M, D)
    out = torch.empty_like(x) if form == "kept" else None
    want = normed(added(x, d), gain, 2.0 ** -17)
    B.ls_op_rmsnorm_f8(x, gain, 2.0 ** -17, codes, scales, delta=d, x_out=out)
    check_exact(codes, scales, want)


def test_swiglu_many_rows_of_one_piece():
    """more pieces than warps that are resident, one and two a row, and a last round that only some warps have"""
    for M, F in ((20011, 16), (9001, 528), (4736 * 2 + 1, 256)):
        for dtype in (BF16, F32):
            gu = rnd((M, 2 * F), F).to(dtype)
            codes, scales = empty_held(M, F)
            B.ls_op_swiglu_f8(gu[:, :F], gu[:, F:], codes, scales)
            g, u = f64(gu[:, :F]), f64(gu[:, F:])
            check_exact(codes, scales, g / (1 + np.exp(-g)) * u)


# ------------------------------------------------------------------ the ends of SwiGLU's range
LAST_GATE = 126 * np.log(2.0)  # beyond, 1 + exp(-gate) is 2^126 and more: silu is 0


def silu64(g):
    with np.errstate(over="ignore"):
        return np.where(g < -LAST_GATE, 0.0, g / (1 + np.exp(-g)))


def partners(g, rng):
    """fp32 values u for rows of one gate each: neither silu(g) u nor silu'(g) = silu(g) / g times u leaves the normal numbers"""
    e = np.frexp(g.astype(np.float64))[1][:, None]
    k = np.where(e > 8, -np.minimum(e, 100), np.where((g[:, None] < -16), rng.integers(3, 20, (len(g), 128)), np.minimum(-e, 120)))
    return (np.ldexp(rng.uniform(0.5, 1, (len(g), 128)), k) * rng.choice([-1.0, 1.0], (len(g), 128))).astype(np.float32)


def check_gates(g, dtype, seed):
    """rows of 128 columns, each of one gate, so that nothing larger hides what becomes of it"""
    u = torch.from_numpy(partners(g, np.random.default_rng(seed))).cuda().to(dtype)
    gate = torch.from_numpy(g).cuda().to(dtype)[:, None].expand(-1, 128).contiguous()
    codes, scales = empty_held(*u.shape)
    B.ls_op_swiglu_f8(gate, u, codes, scales)
    with np.errstate(invalid="ignore"):
        check_rounded(codes, scales, silu64(f64(gate)) * f64(u), SWIGLU_DELTA)


def far_from_the_last(g):
    g = g[np.isfinite(g)]
    return g[np.abs(g.astype(np.float64) + LAST_GATE) > 1e-4]


def test_swiglu_every_bf16_gate():
    g = (np.arange(65536, dtype=np.uint32) << 16).view(np.float32)
    check_gates(far_from_the_last(g), BF16, 1)


def test_swiglu_fp32_gates_of_every_binade():
    rng = np.random.default_rng(2)
    g = np.ldexp(rng.uniform(1, 2, (277, 60)), np.arange(-149, 128)[:, None])
    far = np.ldexp(rng.uniform(1, 2, 8000), rng.integers(23, 32, 8000))  # -t's last place: 1 and more
    g = np.concatenate([g.ravel(), far, [2.0 ** -149, 88, 1e30, 2.35e38, 2.36e38, 3e38, np.finfo(np.float32).max]]).astype(np.float32)
    g = np.concatenate([g, -g, rng.uniform(-88, -87, 2000).astype(np.float32)])
    check_gates(far_from_the_last(g), F32, 3)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_swiglu_gates_that_count_as_0_beside_a_scale_in_doubt(dtype):
    """a block whose largest value is 448 s is computed again in 64 bits, by the same definition: silu(-88) is 0"""
    g = torch.zeros((2, 512), device="cuda").to(dtype)
    u = torch.ones_like(g)
    g[:, 0::128], u[:, 0::128] = 448, 2.0 ** -16
    g[:, 7::9] = -88
    u[:, 7::9] = 2.0 ** 103  # exp(-88) of it: 2^-16 * 0.36
    codes, scales = empty_held(2, 512)
    B.ls_op_swiglu_f8(g, u, codes, scales)
    check_exact(codes, scales, silu64(f64(g)) * f64(u))
    assert not held_values(codes, scales)[:, 7::9].any()


# ------------------------------------------------------------------ the norm's sum
def next_to_a_border(x, gain, eps, seed):
    """x (fp32 [M, D]) with one value of each row moved until its result is one of the two fp32 neighbours of a border between codes"""
    rng = np.random.default_rng(seed)
    M, D = x.shape
    rows, at = np.arange(M), rng.integers(0, D, M)
    v = x.astype(np.float64)
    rest = (v * v).sum(1) - v[rows, at] ** 2
    y = v[rows, at] / np.sqrt((rest + v[rows, at] ** 2) / D + eps) * gain[at]
    e = np.floor(np.log2(np.abs(y)))
    border = (np.floor(np.abs(y) / np.exp2(e - 3)) + 0.5) * np.exp2(e - 3)
    t = (border / np.abs(gain[at])) ** 2  # v^2 = t (rest + v^2) / D + t eps
    ok = t < D / 2
    size = np.sqrt(np.where(ok, t * (rest / D + eps) / np.where(ok, 1 - t / D, 1), v[rows, at] ** 2))
    near = size.astype(np.float32)
    below = np.where(near <= size, near, np.nextafter(near, np.float32(0)))
    near = np.where(rng.random(M) < 0.5, below, np.nextafter(below, np.float32(np.inf)))
    x = x.copy()
    x[rows, at] = np.copysign(near, x[rows, at])
    return x


@pytest.mark.parametrize("form", ["alone", "added", "kept"])
@pytest.mark.parametrize("M,D", [(20000, 16), (4000, 272), (600, 4112), (24, 40000)])
def test_norm_codes_that_the_sum_decides(M, D, form):
    """a few loud columns and many whose squares are lost one by one in 24 bits, and a value of each row next to a border: the error
    of the sum has to be far below that of a rounding"""
    rng = np.random.default_rng(D)
    x = rng.standard_normal((M, D)) * np.where(rng.random((M, D)) < 4 / D, 1, 2.0 ** -12.5)
    x[:, :2] = rng.uniform(0.5, 1.5, (M, 2)) * rng.choice([-1, 1], (M, 2))
    x = (x * np.exp(rng.standard_normal((M, 1)))).astype(np.float32)
    gain = (1 + 0.1 * rnd((D,), 3)).to(BF16)
    eps = 2.0 ** -17
    x = torch.from_numpy(next_to_a_border(x, f64(gain), eps, 1)).cuda()
    d = None if form == "alone" else (rnd((M, D), 4) * 2.0 ** -30).to(BF16)
    if d is not None:
        x = x - d.float()
        x = torch.from_numpy(next_to_a_border(added(x, d).cpu().numpy(), f64(gain), eps, 2)).cuda() - d.float()
    want = normed(added(x, d), gain, eps)
    codes, scales = empty_held(M, D)
    B.ls_op_rmsnorm_f8(x, gain, eps, codes, scales, delta=d, x_out=x if form == "kept" else None)
    check_exact(codes, scales, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,D", [(9, 16), (300, 272), (7, 4112), (5, 40000)])
def test_norm_codes_of_ordinary_rows(M, D, dtype):
    x = (rnd((M, D), M + D) * torch.exp(rnd((M, 1), 1))).to(dtype)
    gain = (1 + 0.1 * rnd((D,), 3)).to(BF16)
    codes, scales = empty_held(M, D)
    B.ls_op_rmsnorm_f8(x, gain, 2.0 ** -17, codes, scales)
    check_exact(codes, scales, normed(x, gain, 2.0 ** -17))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [16, 528, 4096, 40000])
def test_norm_of_rows_of_any_size(D, dtype):
    """rows whose squares, or their mean, are no numbers of fp32; without eps"""
    sizes = torch.tensor([2.0 ** k for k in (-130, -100, -76, -70, -64, -60, -30, 0, 30, 60, 63, 64, 65, 90, 120, 126)], device="cuda")
    x = (rnd((len(sizes), D), D).clamp(-1.9, 1.9) * sizes[:, None]).to(dtype)
    x[:, 3] = x[:, 2] * 0.125
    gain = (1 + 0.1 * rnd((D,), 3)).to(BF16)
    codes, scales = empty_held(*x.shape)
    for eps in (0.0, 2.0 ** -17):
        x_out = torch.empty_like(x)
        B.ls_op_rmsnorm_f8(x, gain, eps, codes, scales, x_out=x_out)
        assert torch.equal(x_out, x)
        check_exact(codes, scales, normed(x, gain, eps))
    # the largest numbers throughout: every value is its gain
    x = torch.full((2, D), torch.finfo(dtype).max, dtype=dtype, device="cuda")
    codes, scales = empty_held(2, D)
    B.ls_op_rmsnorm_f8(x, torch.ones(D, dtype=BF16, device="cuda"), 1e-5, codes, scales)
    assert (held_values(codes, scales) == 1).all()


def test_norm_in_a_chain_reads_what_the_operation_ahead_wrote_in_the_64_bit_path_too():
    """rows of one number x and gains that put every result on a border: all of them are computed twice, whatever x is; x grows by one between
    chained norms, and a value of an earlier x among the new ones would be off by far more than a code"""
    M, D, steps = 100, 4096, 48
    gain = torch.full((D,), 1.0625, dtype=BF16, device="cuda")
    w = quantised(torch.full((D, 16), 0.25, device="cuda"), 128)
    h = quantised(torch.full((M, 16), 0.25, device="cuda"))
    x = torch.ones((M, D), device="cuda")
    held = [empty_held(M, D) for _ in range(steps)]
    torch.cuda.synchronize()
    B.ls_op_chain(True)
    try:
        for codes, scales in held:
            B.ls_op_rmsnorm_f8(x, gain, 0.0, codes, scales)
            B.ls_op_linear_f8(*w, *h, x, add=x)
    finally:
        B.ls_op_chain(False)
    assert (x == 1 + steps).all()
    for i, (codes, scales) in enumerate(held):  # 1.0625 is halfway between 1 and 1.125
        assert (held_values(codes, scales) == 1).all(), i


# ------------------------------------------------------------------ which form of the product runs
# both sides of the rule by which 65 to 128 rows go to CTA pairs (more than 148 tiles of 128 rows of weights), and of those at 64 and 128 rows
MANY_TILES = [(M, N, K) for M in (64, 65, 97, 128, 129) for N, K in ((18944, 272), (18945, 272), (19073, 528))] + \
    [(65, 32000, 400), (80, 22016, 1040), (112, 19200, 2064), (128, 22016, 4112)]


@pytest.mark.parametrize("M,N,K", MANY_TILES)
@pytest.mark.parametrize("out_type,add", [(F32, True), (BF16, False)])
def test_linear_many_tiles_of_weights(M, N, K, out_type, add):
    test_linear(M, N, K, out_type, add)


@pytest.mark.parametrize("M", [1, 7, 16])
@pytest.mark.parametrize("N,K", [(4096, 4112), (5504, 1040), (11008, 4096), (18944, 528), (2048, 8208)])
@pytest.mark.parametrize("add", [False, True])
def test_linear_chained_and_alone_with_and_without_a_long_ring(M, N, K, add):
    """alone, up to 16 rows on at most one CTA an SM and clusters of at most four use the whole SM for stages; chained, half of it"""
    w, h = pair_of(M, N, K, 19)
    base = rnd((M, N), 6) if add else None
    alone, chained = (torch.full((M, N), float("nan"), device="cuda") for _ in range(2))
    B.ls_op_linear_f8(*w, *h, alone, add=base)
    torch.cuda.synchronize()
    B.ls_op_chain(True)
    try:
        for _ in range(3):
            B.ls_op_linear_f8(*w, *h, chained, add=base)
    finally:
        B.ls_op_chain(False)
    assert torch.equal(alone, chained)
