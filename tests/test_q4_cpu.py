"""4-bit weights and the 4-bit cache without a GPU: the format's own properties, sizes, and every refusal that the
entry points make on the host before anything is launched."""
import numpy as np
import pytest

from paper_2404_16710_b200 import binding as B
from tests import q4_reference as R

BAD, CAP = B.LS_ERR_INVALID_ARG, B.LS_ERR_CAPACITY
P = 4096  # a non-null, aligned address that no refused call touches


def bf16(x):
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_value_of_the_format_is_a_bf16_number_and_within_half_a_step(group):
    rng = np.random.default_rng(1)
    x = bf16(rng.standard_normal((64, 256)) * np.exp(rng.uniform(-20, 20, (64, 1))))
    c, s = R.quantise(x, group)
    y = R.values(c, s, group)
    assert np.array_equal(bf16(y), y)
    step = np.repeat(s, group, -1)
    assert (np.abs(x - y) <= step / 2).all()
    a = np.abs(x).reshape(64, -1, group).max(-1)
    assert (s >= a / 7).all() and (s <= a / 7 * (1 + 2.0 ** -4)).all()


def test_codes_are_decided_alike_in_32_and_64_bits():
    """x / s in fp32 lies on the same side of every border (k + 1/2) as the exact quotient, or on it"""
    rng = np.random.default_rng(2)
    x = np.abs(bf16(rng.standard_normal(1 << 18)))
    s = np.ldexp(rng.integers(16, 32, x.size).astype(np.float64), rng.integers(-12, 0, x.size))
    q64, q32 = x / s, (x.astype(np.float32) / s.astype(np.float32)).astype(np.float64)
    for k in range(8):
        assert np.array_equal(np.sign(q64 - (k + 0.5)), np.sign(q32 - (k + 0.5)))
    near = np.abs(q64 - np.floor(q64) - 0.5)
    assert (near[near > 0] > 2.0 ** -17).all()


def test_places_of_a_row_and_a_tile_are_a_permutation():
    for C in (64, 128):
        assert len({R.row_place(c, C) for c in range(C)}) == C
        places = {R.v_place(i, ch, C) for i in range(16) for ch in range(C)}
        assert len(places) == 16 * C and max(p[0] for p in places) == 8 * C - 1


def test_sizes():
    assert B.ls_op_w4_bytes(16, 128, 32) == 1024 + 16 * 4 * 2
    assert B.ls_op_w4_bytes(17, 136, 128) == 2 * 2 * (1024 + 32)
    assert B.ls_op_w4_bytes(4096, 11008, 64) == 256 * 86 * (1024 + 64)
    assert B.ls_op_w4_bytes(2 ** 31 - 1, 8, 32) == 2 ** 27 * 1152  # beyond 32 bits
    assert B.ls_op_w4_bytes(1, 1 << 28, 32) == (1 << 21) * 1152
    for bad in ((0, 128, 32), (1, (1 << 28) + 8, 32), (1, 2 ** 31 - 8, 32), (16, 0, 32), (16, 12, 32), (16, 128, 16), (16, 128, 0), (-1, 128, 32)):
        assert B.ls_op_w4_bytes(*bad) == 0, bad
    assert B.ls_op_kv4_page_bytes(8, 128, 64) == 8 * 4 * 2304
    assert B.ls_op_kv4_page_bytes(3, 64, 16) == 3 * 1152
    for bad in ((0, 128, 64), (8, 96, 64), (8, 128, 48), (8, 128, 8), (8, 128, 2048)):
        assert B.ls_op_kv4_page_bytes(*bad) == 0, bad


def test_weight_operations_refuse_bad_arguments():
    L = B.lib()
    for f in (L.ls_op_quantize_w4, L.ls_op_expand_w4):
        assert f(None, 16, 128, 32, P, None) == BAD
        assert f(P, 16, 128, 32, None, None) == BAD
        assert f(P + 8, 16, 128, 32, P, None) == BAD
        assert f(P, 16, 128, 32, P + 2, None) == BAD
        assert f(P, 0, 128, 32, P, None) == BAD
        assert f(P, 16, 132, 32, P, None) == BAD
        assert f(P, 16, 128, 48, P, None) == BAD
    # packed, h, M, N, K, group, out, residual, stream
    good = [P, P, 1, 16, 128, 32, P, 0, None]
    for at, v in ((0, None), (0, P + 4), (1, None), (1, P + 8), (2, 0), (2, 17), (2, -1), (3, 0), (4, 4), (4, 0), (4, 2 ** 31 - 8),
                  (5, 16), (6, None), (6, P + 2)):
        a = list(good)
        a[at] = v
        assert L.ls_op_linear_w4(*a) == BAD, (at, v)


def refused(f, good, changes):
    for at, v, code in changes:
        a = list(good)
        a[at] = v
        assert f(*a) == code, (at, v)


def test_cache_operations_refuse_bad_arguments():
    L = B.lib()
    # k, v, strides, n_seq, M, pos0, Hkv, hd, page_size, table, stride, max_seq, pages, n_pages, status, stream
    good = [P, P, 1024, 256, 128, 1, 4, P, 2, 128, 64, P, 4, 256, P, 4, None, None]
    refused(L.ls_op_append_kv4, good, [
        (0, None, BAD), (0, P + 8, BAD), (1, None, BAD), (3, 12, BAD), (4, 1, BAD), (5, 0, BAD), (5, 70000, CAP),
        (6, 0, BAD), (6, (1 << 20) + 1, CAP), (6, 2 ** 31 - 1, CAP), (7, None, BAD), (8, 0, BAD), (8, 5000, CAP), (9, 96, BAD), (10, 48, BAD), (10, 8, BAD), (11, None, BAD),
        (12, 3, BAD), (13, 0, CAP), (13, (1 << 20) + 1, CAP), (14, None, BAD), (14, P + 8, BAD), (15, 0, BAD)])
    refused(L.ls_op_append_kv4, good[:5] + [2] + good[6:], [(2, 4, BAD)])
    # pages, n_pages, n_seq, M, pos0, Hkv, hd, page_size, table, stride, max_seq, out_table, kp, vp, n_out, status, stream
    good = [P, 4, 1, 4, P, 2, 128, 64, P, 4, 256, P, P, P, 4, None, None]
    refused(L.ls_op_expand_kv4, good, [
        (0, None, BAD), (1, 0, BAD), (2, 0, BAD), (3, 0, BAD), (3, 2 ** 31 - 1, CAP), (4, None, BAD), (5, 0, BAD), (6, 80, BAD), (7, 24, BAD),
        (8, None, BAD), (9, 3, BAD), (10, 1 << 21, CAP), (11, None, BAD), (12, None, BAD), (12, P + 8, BAD), (13, None, BAD),
        (14, 0, BAD)])
    # q, n_seq, M, pos0, Hq, Hkv, hd, page_size, table, stride, max_seq, pages, n_pages, out, scratch, status, stream
    good = [P, 1, 1, P, 8, 2, 128, 64, P, 4, 256, P, 4, P, None, None, None]
    refused(L.ls_op_attention_kv4, good, [
        (0, None, BAD), (0, P + 8, BAD), (1, 0, BAD), (2, 0, BAD), (2, 17, BAD), (3, None, BAD), (4, 0, BAD), (4, 7, BAD),
        (4, 18, BAD), (5, 0, BAD), (6, 256, BAD), (7, 100, BAD), (8, None, BAD), (9, 3, BAD), (10, 0, CAP), (11, None, BAD),
        (12, 0, BAD), (13, None, BAD), (13, P + 4, BAD), (14, P + 8, BAD)])


def test_the_binding_refuses_what_does_not_fit():
    import torch
    w, small = torch.zeros((16, 128), dtype=torch.bfloat16), torch.zeros(100, dtype=torch.uint8)
    with pytest.raises(B.LsError) as e:
        B.ls_op_quantize_w4(w, 32, small)
    assert e.value.status == CAP
    k = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16)
    pos, table, pages = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 4), dtype=torch.int32), torch.zeros(4 * 2 * 4 * 2304 + 1, dtype=torch.uint8)
    with pytest.raises(B.LsError):
        B.ls_op_append_kv4(k, k[:, :2], pos, 64, table, 256, pages)
    with pytest.raises(B.LsError):  # not whole pages
        B.ls_op_attention_kv4(torch.zeros((1, 1, 1024), dtype=torch.bfloat16), pos, 2, 128, 64, table, 256, pages, torch.zeros((1, 1, 1024), dtype=torch.bfloat16))
    with pytest.raises(B.LsError):
        B.ls_op_expand_kv4(pages, pos, 4, 64, table, 256, table[:, :2], k.view(1, 2, 4, 128), k.view(1, 2, 4, 128))


def test_the_binding_refuses_tensors_of_another_device(monkeypatch):
    """a kernel is launched on the current device, which another device's memory need not be open to"""
    import torch

    class On:  # a tensor that says it is on some device
        def __init__(self, t, dev):
            self.t, self.dev = t, dev

        is_cuda = True

        def __getattr__(self, name):
            return getattr(self.t, name)

        def get_device(self):
            return self.dev

    monkeypatch.setattr(B._torch, "device", lambda: 0)
    w, packed = torch.zeros((16, 128), dtype=torch.bfloat16), torch.zeros(B.ls_op_w4_bytes(16, 128, 32), dtype=torch.uint8)
    h, out = w[:1], torch.zeros((1, 16))
    k, i32 = torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16), torch.zeros((1, 4), dtype=torch.int32)
    pages, kp = torch.zeros(4 * B.ls_op_kv4_page_bytes(2, 64, 16), dtype=torch.uint8), torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    q, pos = torch.zeros((1, 1, 128), dtype=torch.bfloat16), i32[0, :1]
    calls = [(B.ls_op_quantize_w4, [w, 32, packed]), (B.ls_op_expand_w4, [packed, 32, w]), (B.ls_op_linear_w4, [packed, 32, h, out]),
             (B.ls_op_append_kv4, [k, k, pos, 16, i32, 64, pages, pos]),
             (B.ls_op_expand_kv4, [pages, pos, 1, 16, i32, 64, i32, kp, kp, pos]),
             (B.ls_op_attention_kv4, [q, pos, 2, 64, 16, i32, 64, pages, q, pos])]
    for f, args in calls:
        tensors = [i for i, a in enumerate(args) if isinstance(a, torch.Tensor)]
        for odd in (None, *tensors):  # all on device 1, or one of them on device 1 and the rest on the current one
            a = [On(x, int(odd in (None, i))) if i in tensors else x for i, x in enumerate(args)]
            with pytest.raises(B.LsError) as e:
                f(*a)
            assert e.value.status == BAD, (f.__name__, odd)
