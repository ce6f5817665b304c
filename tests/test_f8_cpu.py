"""The 8-bit path without a GPU: the format's own properties, sizes, and every refusal that the entry points make on the
host before anything is launched."""
import numpy as np
import pytest
import torch

from paper_2404_16710_b200 import binding as B
from tests import f8_reference as R

BAD, CAP = B.LS_ERR_INVALID_ARG, B.LS_ERR_CAPACITY
P = 4096  # a non-null, aligned address that no refused call touches


def bf16(x):
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("rows", [1, 128])
def test_every_value_of_the_format_is_a_bf16_number_and_within_half_a_step(rows):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((130, 400)) * np.exp(rng.uniform(-40, 40, (130, 1)))
    b = R.scale_bytes(x, rows)
    y, s = R.values(R.codes(x, rows), b, rows), R.scales(b, *x.shape, rows)
    assert np.array_equal(bf16(y), y)
    assert (np.abs(x - y) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s)).all()
    assert (np.abs(x) <= 448 * s).all()
    a = np.abs(x[:, :128]).max(1)
    if rows == 1:
        assert (a > 224 * s[:, 0]).all()  # no smaller power of two would do


def test_the_reference_codes_are_torchs_own_rounding():
    x = np.random.default_rng(2).standard_normal((64, 256)).astype(np.float32)
    s = R.scales(R.scale_bytes(x.astype(np.float64), 1), 64, 256, 1)
    want = torch.from_numpy((x / s).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.codes(x.astype(np.float64), 1), want)


def test_sizes():
    assert B.ls_op_f8_scale_bytes(1, 16, 1) == 4
    assert B.ls_op_f8_scale_bytes(3, 512, 1) == 12
    assert B.ls_op_f8_scale_bytes(3, 528, 1) == 24
    assert B.ls_op_f8_scale_bytes(129, 11008, 128) == 2 * 88
    assert B.ls_op_f8_scale_bytes(1 << 22, 1 << 28, 1) == (1 << 22) * (1 << 21)
    for bad in ((0, 128, 1), (1, 0, 1), (1, 8, 1), (1, 24, 1), (1, (1 << 28) + 16, 1), ((1 << 22) + 1, 128, 1), (1, 128, 2), (1, 128, 0), (-1, 128, 1)):
        assert B.ls_op_f8_scale_bytes(*bad) == 0, bad


def refused(f, good, changes):
    for at, v in changes:
        a = list(good)
        for i, x in zip(at, v) if isinstance(at, tuple) else ((at, v),):
            a[i] = x
        assert f(*a) == BAD, (at, v)


def test_conversions_refuse_bad_arguments():
    L = B.lib()
    # x, type, ldx, M, K, block_rows, codes, scales, stream
    refused(L.ls_op_quantize_f8, [P, B.LS_BF16, 256, 4, 256, 1, P, P, None], [
        (0, None), (0, P + 8), (1, 2), (1, -1), (2, 255), (2, 252), (2, 260), ((1, 2), (B.LS_F32, 258)), (3, 0), (3, (1 << 22) + 1), (4, 0),
        (4, 250), (4, 264), (4, (1 << 28) + 16), (5, 0), (5, 2), (5, 64), (6, None), (6, P + 4), (7, None), (7, P + 2)])
    # codes, scales, M, K, block_rows, out, stream
    refused(L.ls_op_expand_f8, [P, P, 4, 256, 1, P, None], [
        (0, None), (0, P + 8), (1, None), (1, P + 1), (2, 0), (2, -4), (3, 8), (3, 2 ** 31 - 16), (4, 3), (5, None), (5, P + 8)])


def test_rmsnorm_and_swiglu_refuse_bad_arguments():
    L = B.lib()
    # x, type, ldx, delta, type, ldd, x_out, ldo, gain, M, D, eps, codes, scales, stream
    refused(L.ls_op_rmsnorm_f8, [P, B.LS_F32, 256, P, B.LS_BF16, 256, P, 256, P, 4, 256, 1e-5, P, P, None], [
        (0, None), (0, P + 4), (1, 3), (2, 128), (2, 258), (3, P + 2), (4, 7), (5, 252), (5, 260), (6, P + 8), (7, 250), (7, 8), (8, None), (8, P + 2),
        (9, 0), (9, (1 << 22) + 1), (10, 0), (10, 200), (10, 260), (12, None), (12, P + 1), (13, None), (13, P + 3)])
    # gate, up, type, ld, M, F, codes, scales, stream
    refused(L.ls_op_swiglu_f8, [P, P, B.LS_BF16, 512, 4, 256, P, P, None], [
        (0, None), (0, P + 8), (1, None), (1, P + 2), (2, 2), (3, 128), (3, 516), (4, 0), (5, 0), (5, 40), (6, None), (6, P + 8), (7, None), (7, P + 1)])


def test_linear_refuses_bad_arguments():
    L = B.lib()
    # w, ws, h, hs, M, N, K, out, type, ldo, add, lda, status, stream
    refused(L.ls_op_linear_f8, [P, P, P, P, 4, 128, 256, P, B.LS_F32, 128, P, 128, None, None], [
        (0, None), (0, P + 8), (1, None), (1, P + 2), (2, None), (2, P + 4), (3, None), (3, P + 1), (4, 0), (4, -1), (4, (1 << 22) + 1), (5, 0),
        (5, (1 << 22) + 1), (6, 0), (6, 8), (6, 264), (6, (1 << 28) + 16), (7, None), (7, P + 2), (8, 2), (9, 127), (10, P + 1), (11, 64),
        ((7, 8), (P + 1, B.LS_BF16)), ((8, 10), (B.LS_BF16, P + 1))])


def f8(*shape):
    return torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def test_the_binding_refuses_what_does_not_fit(monkeypatch):
    class On:  # a tensor that says it is on the current device
        def __init__(self, t):
            self.t = t

        def __getattr__(self, name):
            return getattr(self.t, name)

        def get_device(self):
            return 0

    monkeypatch.setattr(B._torch, "device", lambda: 0)
    monkeypatch.setattr(B._torch, "stream", lambda dev: 0)
    bf = torch.bfloat16
    codes, scales, x = f8(4, 256), u8(4, 4), torch.zeros((4, 256), dtype=bf)
    wide = torch.zeros((4, 512), dtype=bf)
    w, ws, out = f8(32, 256), u8(1, 4), torch.zeros((4, 32))
    gain = torch.zeros(256, dtype=bf)
    cases = [
        (B.ls_op_quantize_f8, (x, codes, u8(4, 3))), (B.ls_op_quantize_f8, (x[:3], codes, scales)), (B.ls_op_quantize_f8, (x.half(), codes, scales)),
        (B.ls_op_quantize_f8, (wide[:, ::2], codes, scales)), (B.ls_op_quantize_f8, (x, codes.view(torch.uint8), scales)),
        (B.ls_op_quantize_f8, (x, codes, scales, 64)), (B.ls_op_quantize_f8, (wide[:, 1:257], codes, scales)),
        (B.ls_op_expand_f8, (codes, scales, x.float())), (B.ls_op_expand_f8, (codes, scales, wide)), (B.ls_op_expand_f8, (codes, scales[:2], x)),
        (B.ls_op_rmsnorm_f8, (x, gain[:128], 1e-5, codes, scales)), (B.ls_op_rmsnorm_f8, (x, gain.float(), 1e-5, codes, scales)),
        (B.ls_op_rmsnorm_f8, (x, gain, 1e-5, codes, scales, x[:2])), (B.ls_op_rmsnorm_f8, (x, gain, 1e-5, codes, scales, None, x.float())),
        (B.ls_op_swiglu_f8, (x, x.float(), codes, scales)), (B.ls_op_swiglu_f8, (x, wide[:, 256:], codes, scales)), (B.ls_op_swiglu_f8, (x, x[:3], codes, scales)),
        (B.ls_op_linear_f8, (w, ws, codes[:, :128], scales, out)), (B.ls_op_linear_f8, (w, ws, codes, scales, out[:, :31])),
        (B.ls_op_linear_f8, (w, ws, codes, scales, out, out.to(bf))), (B.ls_op_linear_f8, (w, ws[:, :2], codes, scales, out)),
        (B.ls_op_linear_f8, (w, ws, codes, scales, out.half())), (B.ls_op_linear_f8, (w, ws, codes, scales, out, None, torch.zeros(1))),
    ]
    for f, args in cases:
        with pytest.raises(B.LsError) as e:
            f(*[On(a) if isinstance(a, torch.Tensor) else a for a in args])
        assert e.value.status in (BAD, CAP), (f.__name__, e.value)


def test_the_binding_refuses_tensors_of_another_device(monkeypatch):
    class On:
        def __init__(self, t, dev):
            self.t, self.dev = t, dev

        def __getattr__(self, name):
            return getattr(self.t, name)

        def get_device(self):
            return self.dev

    monkeypatch.setattr(B._torch, "device", lambda: 0)
    codes, scales, x = f8(4, 256), u8(4, 4), torch.zeros((4, 256), dtype=torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32)
    calls = [(B.ls_op_quantize_f8, [x, codes, scales]), (B.ls_op_expand_f8, [codes, scales, x]),
             (B.ls_op_rmsnorm_f8, [x, x[0], 1e-5, codes, scales, x, x]), (B.ls_op_swiglu_f8, [x, x, codes, scales]),
             (B.ls_op_linear_f8, [f8(32, 256), u8(1, 4), codes, scales, torch.zeros((4, 32)), torch.zeros((4, 32)), status])]
    for f, args in calls:
        tensors = [i for i, a in enumerate(args) if isinstance(a, torch.Tensor)]
        for odd in (None, *tensors):  # all on device 1, or one of them on device 1 and the rest on the current one
            a = [On(v, int(odd in (None, i))) if i in tensors else v for i, v in enumerate(args)]
            with pytest.raises(B.LsError) as e:
                f(*a)
            assert e.value.status == BAD, (f.__name__, odd)


def test_sizes_beyond_32_bits_are_not_taken_for_small_ones(monkeypatch):
    """rows and columns go to the library as 32-bit integers: 2^32 + 4 rows are refused, not 4 done"""
    big = (1 << 32) + 4
    for shape in ((big, 16, 1), (4, (1 << 32) + 256, 1), (4, 256, (1 << 32) + 1), (big, 256, 128), (4 - (1 << 32), 256, 1)):
        assert B.ls_op_f8_scale_bytes(*shape) == 0, shape

    class Unreached:
        ls_op_f8_scale_bytes, ls_strerror = B.lib().ls_op_f8_scale_bytes, B.lib().ls_strerror

        def __getattr__(self, name):
            raise AssertionError(f"{name} is called")

    class On:  # a tensor of some shape on the current device
        def __init__(self, t):
            self.t = t

        def __getattr__(self, name):
            return getattr(self.t, name)

        def get_device(self):
            return 0

    monkeypatch.setattr(B._torch, "device", lambda: 0)
    monkeypatch.setattr(B._torch, "stream", lambda dev: 0)
    monkeypatch.setattr(B, "lib", Unreached)
    B.ls_op_f8_scale_bytes.cache_clear()
    bf = torch.bfloat16

    def on(*shape, dtype=torch.float8_e4m3fn):
        return On(torch.empty(shape, dtype=dtype, device="meta"))

    codes, scales, x, gain = on(big, 256), on(big, 4, dtype=torch.uint8), on(big, 256, dtype=bf), on(256, dtype=bf)
    few, fs = on(4, 256), on(4, 4, dtype=torch.uint8)
    cases = [
        (B.ls_op_quantize_f8, (x, codes, scales)), (B.ls_op_quantize_f8, (x, codes, scales, 128)), (B.ls_op_expand_f8, (codes, scales, x)),
        (B.ls_op_rmsnorm_f8, (x, gain, 1e-5, codes, scales)), (B.ls_op_swiglu_f8, (x, x, codes, scales)),
        (B.ls_op_linear_f8, (codes, scales, few, fs, on(4, big, dtype=bf))), (B.ls_op_linear_f8, (few, fs, codes, scales, on(big, 4, dtype=bf))),
    ]
    for f, args in cases:
        with pytest.raises(B.LsError) as e:
            f(*args)
        assert e.value.status == BAD, f.__name__


def test_an_output_over_an_input_of_another_stride_is_refused():
    """in place means row over row: rows that begin together and lie differently would be written before they are read"""
    L = B.lib()
    refused(L.ls_op_rmsnorm_f8, [P, B.LS_F32, 512, 2 * P, B.LS_F32, 512, P, 512, P, 4, 256, 1e-5, P, P, None], [
        (2, 256), (7, 256), ((6, 7), (2 * P, 256)), ((4, 6), (B.LS_BF16, 2 * P)), ((5, 6), (1024, 2 * P))])
    refused(L.ls_op_linear_f8, [P, P, P, P, 4, 128, 256, 2 * P, B.LS_F32, 256, 2 * P, 256, None, None], [(9, 128), (11, 128), (11, 512)])
