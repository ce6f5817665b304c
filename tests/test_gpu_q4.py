"""4-bit weights and the 4-bit cache against the format's definition and 64-bit arithmetic (tests/q4_reference.py).

Conversions are exact: bytes and values have to be equal.  Tolerances of the computed results, derived:
* linear: exact products (8-bit by 3-bit significands), fp32 sums. Every one of the K / 16 tensor-core sums, the
  K / group scaled additions and the 16 at the end is off by at most one unit of its result's last place (the tensor
  cores may truncate), 2^-23, of a partial sum that is at most sum |c s h|.
* attention: the weights p = exp(score - max) <= 1 enter the product in f16: off by at most half a step, 2^-11 of p, or
  2^-25 where p < 2^-14; divided by sum p >= 1 (the largest p is 1) that is at most 2^-11 of sum_i a_i |v_i| plus
  n 2^-25 max |v|.  The scores are fp32 sums as above, so the exponent is off by at most (hd / 16 + hd / 32 + 4) 2^-23 of
  sum |q k| scale, the exponential by 2^-21, the sums by 2^-23 a term: below 2^-13 of sum_i a_i |v_i| for these inputs.
  The bf16 result is rounded once (2^-8 of its value).
"""
import numpy as np
import pytest
import torch

from paper_2404_16710_b200 import binding as B
from tests import q4_reference as R
from tests.helpers import vals

pytestmark = pytest.mark.gpu


def rnd(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda") * scale


def from_bits(u):
    return torch.from_numpy(np.ascontiguousarray(u, np.uint16).view(np.int16)).cuda().view(torch.bfloat16)


def awkward(shape, seed):
    """bf16 values over the whole range, with exact borders, zeros, denormals, the largest number, NaN, infinities"""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal(shape) * np.exp2(rng.integers(-140, 120, shape[:-1] + (1,)))).astype(np.float32)
    u = (x.view(np.uint32) >> 16).astype(np.uint16)
    flat = u.reshape(-1, 16, 8)  # blocks of 128 values: the widest group
    n = flat.shape[0]
    # 7 steps of a scale with 5 significant bits, and borders (k + 1/2) of it (6.5: next to one, as 9 bits do not fit)
    s = np.float32(21 * 2.0 ** -9)
    flat[n // 3] = ((np.float32([7, 0.5, 1.5, 2.5, -3.5, 4.5, -5.5, 6.5]) * s).view(np.uint32) >> 16)
    flat[n // 2] = 0
    flat[n // 2 + 1] = [1, 0x8001, 2, 0x7F, 0x80, 0, 0x8000, 3]
    flat[(2 * n) // 3] = [0x7F7F, 0xFF7F, 0x7F00, 0x4000, 0, 1, 0x3F80, 0xBF80]
    flat[(3 * n) // 4, 5] = [0x7F80, 0x3F80, 0x3F80, 0, 0, 0, 0, 0]
    flat[(4 * n) // 5, 9] = [0x3F80, 0x7FC1, 0x3F80, 0, 0, 0, 0, 0xFF80]
    return from_bits(flat.reshape(shape))


def quantised(w, group):
    N, K = w.shape
    packed = torch.full((B.ls_op_w4_bytes(N, K, group),), 0xEE, dtype=torch.uint8, device="cuda")
    B.ls_op_quantize_w4(w, group, packed)
    return packed


# ------------------------------------------------------------------ weights
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 8), (16, 128), (17, 136), (33, 1000), (100, 72), (5, 2056)])
def test_quantize_and_expand_weights(N, K, group):
    w = rnd((N, K), N + K, 0.02).bfloat16()
    packed = quantised(w, group)
    assert np.array_equal(packed.cpu().numpy(), R.pack_weight(vals(w), group))
    out = torch.full((N, K), 7.0, dtype=torch.bfloat16, device="cuda")
    B.ls_op_expand_w4(packed, group, out)
    assert np.array_equal(vals(out), R.values(*R.quantise(vals(w), group), group))


@pytest.mark.parametrize("group", [32, 128])
def test_quantize_weights_at_the_ends_of_the_range(group):
    w = awkward((40, 1024), 3)
    packed = quantised(w, group)
    assert np.array_equal(packed.cpu().numpy(), R.pack_weight(vals(w), group))
    out = torch.empty_like(w)
    B.ls_op_expand_w4(packed, group, out)
    assert np.array_equal(vals(out), R.values(*R.quantise(vals(w), group), group), equal_nan=True)


def test_quantize_every_border_of_every_scale():
    """all 16 mantissas a scale can have, small and large exponents, and every value within two steps of bf16 of every
    border (k + 1/2) s: the codes are those of exact arithmetic, borders to the even code"""
    rows = []
    for n in range(16, 32):
        for e in (-120, -20, -3, 0, 17, 100):
            s = np.float32(n * 2.0 ** e)
            x = np.zeros((8, 32), np.float32)
            x[:, 0] = 7 * s  # the group's largest: fixes the scale
            for k in range(7):
                border = np.float32((k + 0.5) * s)
                u = int(border.view(np.uint32)) >> 16
                x[k, 1:11] = (np.arange(u - 4, u + 6, dtype=np.uint32) << 16).view(np.float32)
            x[:, 11:21] = -x[:, 1:11]
            rows.append(x)
    x = np.concatenate(rows)
    w = from_bits((x.view(np.uint32) >> 16).astype(np.uint16))
    assert np.array_equal(vals(w), x.astype(np.float64))
    assert np.array_equal(quantised(w, 32).cpu().numpy(), R.pack_weight(vals(w), 32))


def linear_reference(w, group, h):
    v = R.values(*R.quantise(vals(w), group), group)
    hv = vals(h)
    return hv @ v.T, np.abs(hv) @ np.abs(v).T


def linear_tol(K, group, spread):
    return (K / 16 + K / group + 20) * 2.0 ** -23 * spread


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 16, 128), (1, 1, 8), (2, 200, 88), (7, 333, 1000), (8, 64, 4096), (9, 48, 2000),
                                   (16, 130, 520), (5, 1000, 14336), (16, 4096, 1376), (1, 4100, 4096)])
@pytest.mark.parametrize("residual", [False, True])
def test_linear(M, N, K, group, residual):
    w, h = rnd((N, K), 1 + N, 0.02).bfloat16(), rnd((M, K), 2 + K).bfloat16()
    out = rnd((M, N), 3) if residual else torch.full((M, N), float("nan"), device="cuda")
    base = out.cpu().numpy().astype(np.float64) if residual else 0.0
    B.ls_op_linear_w4(quantised(w, group), group, h, out, residual)
    ref, spread = linear_reference(w, group, h)
    got = out.cpu().numpy().astype(np.float64)
    tol = linear_tol(K, group, spread) + (2.0 ** -23 * np.abs(base + ref) if residual else 0.0)
    assert (np.abs(got - base - ref) <= tol).all(), np.abs(got - base - ref).max()
    assert np.linalg.norm(got - base - ref) <= 1e-5 * np.linalg.norm(ref)


def test_linear_large_vocabulary_sampled_rows():
    N, K, group, M = 128256, 4096, 64, 13
    w, h = rnd((N, K), 5, 0.02).bfloat16(), rnd((M, K), 6).bfloat16()
    out = torch.empty((M, N), device="cuda")
    B.ls_op_linear_w4(quantised(w, group), group, h, out)
    rows = np.unique(np.concatenate([[0, 15, 16, N - 1], np.random.default_rng(0).integers(0, N, 40)]))
    ref, spread = linear_reference(w[torch.from_numpy(rows).cuda()], group, h)
    assert (np.abs(out.cpu().numpy()[:, rows] - ref) <= linear_tol(K, group, spread)).all()


@pytest.mark.parametrize("N,K,group", [(304, 1384, 32), (4096, 4096, 128), (5000, 264, 64), (16, 11008, 32), (16400, 520, 32),
                                       (16500, 14336, 128), (33, 30000, 64)])
def test_linear_rows_do_not_depend_on_pass_size(N, K, group):
    packed = quantised(rnd((N, K), 7, 0.05).bfloat16(), group)
    h = rnd((16, K), 8).bfloat16()
    full = torch.empty((16, N), device="cuda")
    B.ls_op_linear_w4(packed, group, h, full)
    for m0, M in ((0, 1), (3, 2), (0, 4), (5, 7), (8, 8), (2, 9), (0, 15)):
        out = torch.empty((M, N), device="cuda")
        B.ls_op_linear_w4(packed, group, h[m0:m0 + M].contiguous(), out)
        assert torch.equal(out, full[m0:m0 + M]), M


@pytest.mark.parametrize("N,K,group", [(30784, 136, 64), (30785, 136, 64), (30800, 520, 32), (31000, 8200, 128), (33000, 264, 32)])
def test_linear_rows_of_large_matrices_do_not_depend_on_pass_size(N, K, group):
    """on both sides of the number of rows from which two tiles are taken at a time, an odd last pair among them"""
    w = rnd((N, K), 220, 0.05).bfloat16()
    packed, h = quantised(w, group), rnd((16, K), 221).bfloat16()
    full = torch.empty((16, N), device="cuda")
    B.ls_op_linear_w4(packed, group, h, full)
    rows = np.unique(np.concatenate([[0, 15, 16, N - 17, N - 1], np.random.default_rng(1).integers(0, N, 40)]))
    ref, spread = linear_reference(w[torch.from_numpy(rows).cuda()], group, h)
    assert (np.abs(full.cpu().numpy()[:, rows] - ref) <= linear_tol(K, group, spread)).all()
    for m0, M in ((0, 1), (5, 7), (8, 8), (2, 9), (0, 15)):
        out = torch.full((M, N), float("nan"), device="cuda")
        B.ls_op_linear_w4(packed, group, h[m0:m0 + M].contiguous(), out)
        assert torch.equal(out, full[m0:m0 + M]), M


def test_linear_scales_of_other_packers_and_values_that_are_not_finite():
    """any bf16 scale may stand in the packed weights; a NaN group, an infinite h make NaN where the formula does"""
    N, K, group = 40, 256, 64
    w = rnd((N, K), 9, 0.02).bfloat16()
    packed = quantised(w, group).cpu().numpy().reshape(-1, 1024 + 64)
    scales = np.random.default_rng(1).integers(0x3A00, 0x3C00, (packed.shape[0], 32)).astype("<u2")
    packed[:, 1024:] = scales.view(np.uint8)
    dev = torch.from_numpy(packed.reshape(-1).copy()).cuda()
    codes, _ = R.quantise(vals(w), group)
    S = (scales.astype(np.uint32) << 16).view(np.float32).astype(np.float64).reshape(3, 2, 16, 2)
    S = S.transpose(0, 2, 1, 3).reshape(48, 4)[:N]
    h = rnd((3, K), 10).bfloat16()
    out = torch.empty((3, N), device="cuda")
    B.ls_op_linear_w4(dev, group, h, out)
    v = R.values(codes, S, group)
    assert (np.abs(out.cpu().numpy() - vals(h) @ v.T) <= linear_tol(K, group, np.abs(vals(h)) @ np.abs(v).T)).all()
    w[5, 70] = float("nan")
    w[6, 3] = float("inf")
    h[1, 9] = float("inf")
    B.ls_op_linear_w4(quantised(w, group), group, h, out)
    got = out.cpu().numpy()
    assert np.isnan(got[:, [5, 6]]).all() and not np.isfinite(got[1]).any()
    rest = [n for n in range(N) if n not in (5, 6)]
    assert np.isfinite(got[[0, 2]][:, rest]).all()


# ------------------------------------------------------------------ the cache: append, expand
def empty_pool(n_pages, Hkv, hd, page, fill=0xFF):
    return torch.full((n_pages, B.ls_op_kv4_page_bytes(Hkv, hd, page)), fill, dtype=torch.uint8, device="cuda")


def reference_append(pool, k, v, pos0, table, page, max_seq):
    """the appended pool by the definition; pool [n_pages, page bytes] uint8, k, v float64 [n_seq, M, Hkv, hd]"""
    n_seq, M, Hkv, hd = k.shape
    tiles = pool.reshape(pool.shape[0], Hkv, page // 16, R.tile_bytes(hd))
    for b in range(n_seq):
        for m in range(M):
            p = pos0[b] + m
            if 0 <= p < max_seq and 0 <= table[b, p // page] < pool.shape[0]:
                for i in range(Hkv):
                    R.put_token(tiles[table[b, p // page], i, p % page // 16], p % 16, k[b, m, i], v[b, m, i], hd)
    return pool


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_seq,M,Hkv,page,pos", [(1, 1, 2, 16, [0]), (1, 1, 1, 64, [77]), (3, 5, 2, 16, [14, 0, 40]),
                                                  (2, 70, 1, 32, [3, 25]), (4, 3, 2, 64, [-1, -3, 93, 60])])
def test_append_and_expand(n_seq, M, Hkv, page, pos, hd):
    max_seq = 96
    n_tab = -(-max_seq // page)
    table = np.random.default_rng(5).permutation(n_seq * n_tab + 3)[:n_seq * n_tab].reshape(n_seq, n_tab).astype(np.int32)
    k, v = rnd((n_seq, M, Hkv, hd), 11, 3.0).bfloat16(), rnd((n_seq, M, Hkv, hd), 12).bfloat16()
    pool = empty_pool(n_seq * n_tab + 3, Hkv, hd, page, 0x5A)
    want = reference_append(pool.cpu().numpy().copy(), vals(k), vals(v), pos, table, page, max_seq)
    td, pd = torch.from_numpy(table).cuda(), torch.tensor(pos, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ls_op_append_kv4(k, v, pd, page, td, max_seq, pool, status)
    assert np.array_equal(pool.cpu().numpy(), want) and int(status) == 0
    # back, to pages in another order; slots that no row covers stay as they were
    out_table = np.random.default_rng(6).permutation(n_seq * n_tab).reshape(n_seq, n_tab).astype(np.int32)
    kp = torch.full((n_seq * n_tab, Hkv, page, hd), 3.0, dtype=torch.bfloat16, device="cuda")
    vp = torch.full_like(kp, 5.0)
    wk, wv = vals(kp), vals(vp)
    for b in range(n_seq):
        for m in range(M):
            p = pos[b] + m
            if p >= 0:
                at = out_table[b, p // page], slice(None), p % page
                wk[at] = R.values(*R.quantise(vals(k[b, m]), 32), 32)
                wv[at] = R.values(*R.quantise(vals(v[b, m]), 32), 32)
    B.ls_op_expand_kv4(pool, pd, M, page, td, max_seq, torch.from_numpy(out_table).cuda(), kp, vp, status)
    assert np.array_equal(vals(kp), wk) and np.array_equal(vals(vp), wv) and int(status) == 0


@pytest.mark.parametrize("hd", [64, 128])
def test_append_strided_rows_and_the_ends_of_the_range(hd):
    """rows of a fused q|k|v buffer and of a bf16 cache page (heads outermost), values over the whole range"""
    Hkv, page, M = 2, 32, 20
    table, pd = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), torch.tensor([7], dtype=torch.int32, device="cuda")
    fused = awkward((M, 6 * Hkv * hd), 13)
    heads = awkward((2, Hkv, 32, hd), 14)
    for k, v in ((fused.view(1, M, 6 * Hkv, hd)[:, :, Hkv:2 * Hkv], fused.view(1, M, 6 * Hkv, hd)[:, :, 4 * Hkv:5 * Hkv]),
                 (heads[0].transpose(0, 1)[None, 4:4 + M], heads[1].transpose(0, 1)[None, 4:4 + M])):
        pool = empty_pool(2, Hkv, hd, page)
        want = reference_append(pool.cpu().numpy().copy(), vals(k), vals(v), [7], table.cpu().numpy(), page, 64)
        B.ls_op_append_kv4(k, v, pd, page, table, 64, pool)
        assert np.array_equal(pool.cpu().numpy(), want)


def test_positions_and_pages_out_of_range_are_refused():
    Hkv, hd, page, max_seq = 2, 128, 16, 64
    table = torch.tensor([[0, 1, 2, 3], [4, 9, -1, 5], [6, 7, 8, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    k, v = rnd((3, 6, Hkv, hd), 15).bfloat16(), rnd((3, 6, Hkv, hd), 16).bfloat16()
    q = rnd((3, 6, 4 * hd), 17).bfloat16()
    kp = torch.zeros((9, Hkv, page, hd), dtype=torch.bfloat16, device="cuda")
    for pos, code in (([60, 0, 2 ** 31 - 1], 2), ([0, 12, 0], 4), ([0, 30, 0], 4), ([0, 0, 46], 4)):
        pd = torch.tensor(pos, dtype=torch.int32, device="cuda")
        for which in range(3):
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            pool = empty_pool(9, Hkv, hd, page, 0x11)
            if which == 0:
                want = reference_append(pool.cpu().numpy().copy(), vals(k), vals(v), pos, table.cpu().numpy(), page, max_seq)
                B.ls_op_append_kv4(k, v, pd, page, table, max_seq, pool, status)
                assert np.array_equal(pool.cpu().numpy(), want)
            elif which == 1:
                B.ls_op_expand_kv4(pool, pd, 6, page, table, max_seq, table, kp, kp.clone(), status)
            else:
                out = torch.full_like(q, 9.0)
                B.ls_op_attention_kv4(q, pd, Hkv, hd, page, table, max_seq, pool, out, status)
                got = vals(out)
                for b in range(3):
                    for m in range(6):
                        if pos[b] + m >= max_seq:
                            assert (got[b, m] == 0).all(), (pos, b, m)
            assert int(status) == code, (pos, which)


def test_a_row_all_of_whose_pages_are_refused_is_nan():
    """softmax of nothing; the status says why.  The other sequence is as ever."""
    c = Cache([20, 20], 1, 64, 16, 70)
    q = rnd((2, 2, 128), 71).bfloat16()
    want, status = c.run(q, 2), torch.zeros(1, dtype=torch.int32, device="cuda")
    c.table[0] = -1
    got = c.run(q, 2, status)
    assert torch.isnan(got[0]).all() and torch.equal(got[1], want[1]) and int(status) == 4


# ------------------------------------------------------------------ attention
class Cache:
    """n_seq sequences of random k, v in 4 bits: appended by the library (its bytes are tested above) to pages whose
    other slots hold 0xff bytes, i.e. NaN scales"""

    def __init__(self, lens, Hkv, hd, page, seed, max_seq=None, loud=1.0):
        self.Hkv, self.hd, self.page, self.lens = Hkv, hd, page, lens
        n_seq, T = len(lens), max(max(lens), 1)
        self.max_seq = max_seq or -(-T // page) * page
        n_tab = -(-self.max_seq // page)
        order = np.random.default_rng(seed).permutation(n_seq * n_tab).astype(np.int32)
        self.table = torch.from_numpy(order.reshape(n_seq, n_tab)).cuda()
        self.pool = empty_pool(n_seq * n_tab, Hkv, hd, page)
        self.k = [rnd((max(n, 1), Hkv, hd), seed + 10 * b, loud).bfloat16() for b, n in enumerate(lens)]
        self.v = [rnd((max(n, 1), Hkv, hd), seed + 10 * b + 1).bfloat16() for b, n in enumerate(lens)]
        for b, n in enumerate(lens):
            if n:
                B.ls_op_append_kv4(self.k[b][None, :n], self.v[b][None, :n], torch.zeros(1, dtype=torch.int32, device="cuda"),
                                   page, self.table[b:b + 1], self.max_seq, self.pool)

    def values(self, b):
        return [R.values(*R.quantise(vals(x[b]), 32), 32) for x in (self.k, self.v)]

    def run(self, q, M, status=None):
        out = torch.full_like(q, float("nan"))
        pos = torch.tensor([n - M for n in self.lens], dtype=torch.int32, device="cuda")
        B.ls_op_attention_kv4(q, pos, self.Hkv, self.hd, self.page, self.table, self.max_seq, self.pool, out, status)
        return out


def attention_tol(ref, spread, v):
    return 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -13) * spread + len(v) * 2.0 ** -25 * np.abs(v).max()


def check_attention(c, q, out, M, G):
    got, qv = vals(out), vals(q)
    for b, n in enumerate(c.lens):
        k, v = c.values(b)
        for m in range(M):
            ref, spread = R.attention(qv[b, m].reshape(-1, c.hd), k, v, n - M + m, G)
            err = np.abs(got[b, m].reshape(-1, c.hd) - ref)
            assert (err <= (attention_tol(ref, spread, v) if n - M + m >= 0 else 0)).all(), (b, m, n, err.max())


@pytest.mark.parametrize("Hkv,G,hd", [(2, 1, 128), (1, 8, 128), (2, 4, 64), (3, 2, 128), (1, 7, 64)])
@pytest.mark.parametrize("M,lens,page", [(1, [1], 16), (1, [15, 16, 17], 16), (1, [31, 32, 33], 32), (3, [2, 3, 4], 16),
                                         (7, [300], 64), (16, [16, 1000], 32), (1, [0, 257, 256, 255], 64),
                                         (5, [0, 0, 4, 130], 16), (16, [1100, 7], 256), (2, [4099], 64)])
def test_attention(Hkv, G, hd, M, lens, page):
    c = Cache(lens, Hkv, hd, page, 20)
    q = rnd((len(lens), M, Hkv * G * hd), 21).bfloat16()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = c.run(q, M, status)
    check_attention(c, q, out, M, G)
    assert int(status) == 0


@pytest.mark.parametrize("n_seq", [1, 40])
def test_attention_clusters_of_every_size_and_peaked_scores(n_seq):
    """one to 8 CTAs a head (by the number of sequences and heads), scores that differ by hundreds"""
    for Hkv in (1, 2, 8):
        c = Cache([700 - 13 * b for b in range(n_seq)], Hkv, 128, 64, 30, max_seq=4096, loud=6.0)
        q = rnd((n_seq, 2, Hkv * 2 * 128), 31, 2.0).bfloat16()
        check_attention(c, q, c.run(q, 2), 2, 2)


@pytest.mark.parametrize("Hkv,n_seq,max_seq", [(20, 1, 2048), (24, 1, 2048), (30, 1, 2048), (40, 1, 2048), (5, 7, 2048),
                                               (3, 50, 2048), (150, 1, 2048), (16, 3, 10240), (8, 8, 8192), (32, 3, 6144),
                                               (64, 2, 4096), (10, 1, 8192)])
def test_attention_clusters_of_odd_sizes(Hkv, n_seq, max_seq):
    """numbers of heads and lengths of caches that take clusters of 1 to 6 and splits of any number; every row the same in a pass of one as among 8"""
    c = Cache([900 - 11 * b for b in range(n_seq)], Hkv, 64, 64, 60, max_seq=max_seq)
    q = rnd((n_seq, 8, Hkv * 64), 61, 2.0).bfloat16()
    full = c.run(q, 8)
    check_attention(c, q, full, 8, 1)
    for m in (0, 5, 7):
        out = torch.empty((n_seq, 1, Hkv * 64), dtype=torch.bfloat16, device="cuda")
        pos = torch.tensor([900 - 11 * b - 8 + m for b in range(n_seq)], dtype=torch.int32, device="cuda")
        B.ls_op_attention_kv4(q[:, m:m + 1].contiguous(), pos, Hkv, 64, 64, c.table, max_seq, c.pool, out)
        assert torch.equal(out, full[:, m:m + 1]), m


@pytest.mark.parametrize("Hkv,G,hd", [(2, 1, 128), (2, 4, 64), (4, 8, 128)])
def test_attention_rows_do_not_depend_on_pass_size(Hkv, G, hd):
    c = Cache([1000], Hkv, hd, 64, 40, max_seq=2048)
    q = rnd((1, 16, Hkv * G * hd), 41).bfloat16()
    full = c.run(q, 16)
    for m0, M in ((0, 1), (15, 1), (4, 3), (3, 5), (9, 6), (0, 8), (7, 9)):
        out = torch.empty((1, M, q.shape[2]), dtype=torch.bfloat16, device="cuda")
        B.ls_op_attention_kv4(q[:, m0:m0 + M].contiguous(), torch.tensor([984 + m0], dtype=torch.int32, device="cuda"), Hkv, hd, 64,
                              c.table, 2048, c.pool, out)
        assert torch.equal(out, full[:, m0:m0 + M]), (m0, M)


@pytest.mark.parametrize("Hkv,hd,M,G", [(8, 128, 12, 2), (5, 64, 6, 8)])
def test_attention_clusters_that_take_several_splits(Hkv, hd, M, G):
    """a cache of 65536 positions of which 9000 are used: every split has some; rows as in passes of one"""
    c = Cache([9000], Hkv, hd, 64, 80, max_seq=1 << 16)
    q = rnd((1, M, Hkv * G * hd), 81, 2.0).bfloat16()
    full = c.run(q, M)
    check_attention(c, q, full, M, G)
    for m in (0, M // 2, M - 1):
        out = torch.empty((1, 1, q.shape[2]), dtype=torch.bfloat16, device="cuda")
        B.ls_op_attention_kv4(q[:, m:m + 1].contiguous(), torch.tensor([9000 - M + m], dtype=torch.int32, device="cuda"), Hkv, hd,
                              64, c.table, 1 << 16, c.pool, out)
        assert torch.equal(out, full[:, m:m + 1]), m


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_values_that_are_not_finite_reach_only_the_rows_that_see_them(hd):
    Hkv, G, M, n = 1, 2, 4, 90
    for what in ("k", "v"):
        c = Cache([n], Hkv, hd, 32, 50)
        bad = rnd((1, 2, Hkv, hd), 51).bfloat16()
        good = rnd((1, 2, Hkv, hd), 52).bfloat16()
        bad[0, 0, 0, 40] = float("nan")
        bad[0, 1, 0, 3] = float("inf")
        pos = torch.tensor([n - 2], dtype=torch.int32, device="cuda")
        k, v = (bad, good) if what == "k" else (good, bad)
        B.ls_op_append_kv4(k, v, pos, 32, c.table, c.max_seq, c.pool)
        c.k[0][n - 2:], c.v[0][n - 2:] = k[0], v[0]
        q = rnd((1, M, G * hd), 53).bfloat16()
        out = c.run(q, M)
        got = vals(out).reshape(M, G, hd)
        kk, vv = c.values(0)
        for m in range(2):
            ref, spread = R.attention(vals(q)[0, m].reshape(G, hd), kk[:n - 2], vv[:n - 2], n - M + m, G)
            assert (np.abs(got[m] - ref) <= attention_tol(ref, spread, vv[:n - 2])).all()
        if what == "k":
            assert np.isnan(got[2:]).all()
        else:  # the groups of channels 40 and 3
            assert np.isnan(got[2, :, 32:64]).all() and np.isfinite(got[2, :, :32]).all() and np.isfinite(got[2, :, 64:]).all()
            assert np.isnan(got[3, :, :64]).all() and np.isfinite(got[3, :, 64:]).all()


def test_attention_pages_beyond_32_bits_of_offset():
    """a pool of more than 4 GB whose used pages are the last ones"""
    Hkv, hd, page, n = 8, 128, 1024, 1500
    per = B.ls_op_kv4_page_bytes(Hkv, hd, page)
    n_pages = (1 << 32) // per + 8
    small = Cache([n], Hkv, hd, page, 60, max_seq=4096)
    pool = torch.zeros((n_pages, per), dtype=torch.uint8, device="cuda")
    far = torch.tensor([[n_pages - 1, n_pages - 3, n_pages - 2, 0]], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ls_op_append_kv4(small.k[0][None], small.v[0][None], zero, page, far, 4096, pool)
    assert not bool(pool[:n_pages - 3].any())
    q = rnd((1, 1, 16 * hd), 61).bfloat16()
    a, pos = torch.empty_like(q), torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    B.ls_op_attention_kv4(q, pos, Hkv, hd, page, far, 4096, pool, a)
    assert torch.equal(a, small.run(q, 1))
    kp = torch.zeros((4, Hkv, page, hd), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    B.ls_op_expand_kv4(pool, zero, n, page, far, 4096, torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda"), kp, vp)
    k, _ = small.values(0)
    assert np.array_equal(vals(kp).transpose(0, 2, 1, 3).reshape(-1, Hkv, hd)[:n], k)


def test_captured_and_replayed_at_other_positions_on_another_stream():
    """append and attention in one CUDA graph, positions advanced on the device between replays; a second sequence
    shares the pages of the first for what both only read"""
    Hkv, G, hd, page, max_seq = 2, 2, 128, 16, 160
    c = Cache([100], Hkv, hd, page, 70, max_seq=max_seq)
    st = torch.cuda.Stream()
    table = torch.cat([c.table, c.table])
    pool = torch.cat([c.pool, empty_pool(4, Hkv, hd, page)])
    n_own = c.pool.shape[0]
    table[1, 6:10] = torch.arange(n_own, n_own + 4, device="cuda", dtype=torch.int32)
    pool[table[1, 6].long()] = pool[table[0, 6].long()]  # positions 96..99 are copied, 0..95 shared
    k, v = rnd((2, 1, Hkv, hd), 71).bfloat16(), rnd((2, 1, Hkv, hd), 72).bfloat16()
    q, out = rnd((2, 1, Hkv * G * hd), 73).bfloat16(), torch.zeros((2, 1, Hkv * G * hd), dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor([100, 100], dtype=torch.int32, device="cuda")

    def step():
        B.ls_op_append_kv4(k, v, pos, page, table, max_seq, pool)
        B.ls_op_attention_kv4(q, pos, Hkv, hd, page, table, max_seq, pool, out)
        pos.add_(1)

    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step()  # first use outside a capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
        pos.fill_(100)
        steps = []
        for i in range(20):
            k.copy_(rnd((2, 1, Hkv, hd), 200 + i))
            v.copy_(rnd((2, 1, Hkv, hd), 300 + i))
            q.copy_(rnd((2, 1, Hkv * G * hd), 400 + i))
            steps.append((vals(k), vals(v), vals(q)))
            graph.replay()
            steps[-1] += (vals(out),)
    st.synchronize()
    ck, cv = c.values(0)
    for b in range(2):
        kk, vv = ck, cv
        for ks, vs, qs, got in steps:
            kk = np.concatenate([kk, R.values(*R.quantise(ks[b], 32), 32)])
            vv = np.concatenate([vv, R.values(*R.quantise(vs[b], 32), 32)])
            ref, spread = R.attention(qs[b, 0].reshape(-1, hd), kk, vv, kk.shape[0] - 1, G)
            assert (np.abs(got[b, 0].reshape(-1, hd) - ref) <= attention_tol(ref, spread, vv)).all()


def test_attention_values_and_keys_of_very_different_sizes():
    """tokens and channel groups whose k and v differ by factors up to 2^20 and 2^24, queries too: the kernel's shared
    powers of two must lose nothing.  The loudest values sit under the smallest weights."""
    Hkv, G, hd, n, M = 2, 4, 128, 700, 3
    c = Cache([n], Hkv, hd, 64, 90)
    rng = np.random.default_rng(91)
    size = torch.from_numpy(np.exp2(rng.uniform(-12, 12, (n, Hkv, 4)))).float().cuda()
    c.v[0] = (c.v[0].float() * size.repeat_interleave(32, 2)).bfloat16()
    c.k[0] = (c.k[0].float() * torch.from_numpy(np.exp2(rng.uniform(-20, 0, (n, Hkv, 1)))).float().cuda()).bfloat16()
    q = (rnd((1, M, Hkv * G * hd), 92) * torch.from_numpy(np.exp2(rng.uniform(-30, 2, (1, M, Hkv * G, 1)))).float().cuda()
         .expand(1, M, Hkv * G, hd).reshape(1, M, -1)).bfloat16()
    loud = int(np.argmax(vals(c.v[0]).max((1, 2))))
    c.k[0][loud] = -3.0 * q[0, 0].view(Hkv, G, hd)[:, 0].sign()  # as far from the queries as can be
    B.ls_op_append_kv4(c.k[0][None], c.v[0][None], torch.zeros(1, dtype=torch.int32, device="cuda"), 64, c.table, c.max_seq, c.pool)
    check_attention(c, q, c.run(q, M), M, G)


def refill(c, b=0):
    """the cache's sequence b again from c.k, c.v"""
    B.ls_op_append_kv4(c.k[b][None], c.v[b][None], torch.zeros(1, dtype=torch.int32, device="cuda"), c.page, c.table[b:b + 1],
                       c.max_seq, c.pool)


def check_by_group(c, q, out, M, G):
    """as check_attention, but what a weight below f16's normal numbers loses counts against the largest value of the
    channel group itself, not of the head"""
    got, qv = vals(out), vals(q)
    for b, n in enumerate(c.lens):
        k, v = c.values(b)
        top = np.abs(v).reshape(n, c.Hkv, -1, 32).max((0, 3)).repeat(32, 1).repeat(G, 0)
        for m in range(M):
            ref, spread = R.attention(qv[b, m].reshape(-1, c.hd), k, v, n - M + m, G)
            err = np.abs(got[b, m].reshape(-1, c.hd) - ref)
            tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -13) * spread + n * 2.0 ** -25 * top
            assert (err <= tol).all(), (b, m, n, (err / tol).max(), np.argmax(err / tol))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("down", [20, 24, 25, 26, 40, 100])
def test_attention_channel_groups_that_are_always_quiet(hd, down):
    """one channel group 2^-down of the others in every token: as exact as they are"""
    Hkv, G, n, M = 2, 3, 333, 2
    c = Cache([n], Hkv, hd, 32, 170)
    c.v[0][:, 0, 32:64] *= 2.0 ** -down
    c.v[0][:, 1, :32] *= 2.0 ** -down
    refill(c)
    q = rnd((1, M, Hkv * G * hd), 171).bfloat16()
    check_by_group(c, q, c.run(q, M), M, G)


@pytest.mark.parametrize("Hkv,G,hd,M,n,max_seq", [(1, 1, 64, 2, 40, 64), (2, 2, 128, 4, 700, 1024), (1, 8, 128, 16, 1010, 1024),
                                                  (3, 1, 128, 16, 24, 64), (1, 4, 64, 16, 9010, 16384), (1, 8, 64, 7, 70, 128)])
@pytest.mark.parametrize("up", [1, 12, 25, 40, 110])
def test_attention_loud_values_of_later_rows(Hkv, G, hd, M, n, max_seq, up):
    """values of the last rows' own tokens that are louder and louder than what came before (whose sizes differ too): rows
    that do not see them come out bit for bit as without them"""
    c = Cache([n], Hkv, hd, 16, 180, max_seq=max_seq)
    size = np.exp2(np.random.default_rng(181).uniform(-11, 0, (n, Hkv, 1)))
    for i in range(1, M):  # the token of every row but the first
        size[n - M + i] = 2.0 ** (up * i / (M - 1))
    x = c.v[0].float() * torch.from_numpy(size).float().cuda()
    for i in range(1, M):  # less in one channel group
        x[n - M + i, :, 32 * (i % (hd // 32)):][:, :32] *= 2.0 ** -3
    c.v[0] = x.bfloat16()
    refill(c)
    q = rnd((1, M, Hkv * G * hd), 182).bfloat16()
    full = c.run(q, M)
    for m in range(M):
        out = torch.empty((1, 1, q.shape[2]), dtype=torch.bfloat16, device="cuda")
        pos = torch.tensor([n - M + m], dtype=torch.int32, device="cuda")
        B.ls_op_attention_kv4(q[:, m:m + 1].contiguous(), pos, Hkv, hd, 16, c.table, max_seq, c.pool, out)
        assert torch.equal(out, full[:, m:m + 1]), m
        k, v = (y[:n - M + m + 1] for y in c.values(0))
        ref, spread = R.attention(vals(q)[0, m].reshape(-1, hd), k, v, n - M + m, G)
        top = np.abs(v).max()
        err = np.abs(vals(out)[0, 0].reshape(-1, hd) - ref)
        assert (err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -13) * spread + n * 2.0 ** -25 * top).all(), m


@pytest.mark.parametrize("M", [1, 3])
def test_attention_small_weights_beside_a_key_that_has_nearly_all(M):
    """the first key (7 steps of 7.25, which the format holds) outweighs each of the others by 2^25.9 and has value 0: what the
    others, all alike, sum up to is as exact as any result, also in the share of the positions (a 64th: 8 CTAs of 8 warps) that
    the first key belongs to.  There a weight of 2^-25.9 is off by 2^-32 at most: 2^-6.1 of it, 2^-12.1 of the result."""
    n, hd, G = 4096, 128, 2
    c = Cache([n], 1, hd, 64, 190)
    q = torch.zeros((1, M, G * hd), device="cuda")
    q[..., 0::hd] = 4.0
    c.k[0].zero_()
    c.k[0][0, 0, 0] = 50.75
    c.v[0] = (1.0 + 0.25 * torch.rand((n, 1, hd), generator=torch.Generator(device="cuda").manual_seed(191), device="cuda")).bfloat16()
    c.v[0][0] = 0
    refill(c)
    got = vals(c.run(q.bfloat16(), M))
    k, v = c.values(0)
    for m in range(M):
        ref, spread = R.attention(vals(q)[0, m].reshape(G, hd), k, v, n - M + m, G)
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -13) * spread
        assert (np.abs(got[0, m].reshape(G, hd) - ref) <= tol).all(), m


@pytest.mark.parametrize("M", [1, 2, 3, 4, 6, 16])
def test_attention_over_a_cache_long_enough_to_be_split(M):
    """16384 positions of one KV head: several splits joined by the second kernel, with scratch of the caller's and of
    the binding's; without any, one cluster does it.  Both within the bound; rows as in a pass of 16."""
    Hkv, G, hd, page, n = 1, 4, 64, 64, 12345
    c = Cache([n], Hkv, hd, page, 95, max_seq=16384)
    q = rnd((1, 16, Hkv * G * hd), 96).bfloat16()
    need = B.ls_op_attention_kv4_scratch_bytes(1, M, Hkv * G, Hkv, hd, 16384)
    assert need > 0 and B.ls_op_attention_kv4_scratch_bytes(1, M, Hkv * G, Hkv, hd, 4096) == 0
    pos = torch.tensor([n - M], dtype=torch.int32, device="cuda")
    mine = q[:, 16 - M:].contiguous()
    outs = []
    for scratch in (None, torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")):
        out = torch.empty_like(mine)
        B.ls_op_attention_kv4(mine, pos, Hkv, hd, page, c.table, 16384, c.pool, out, None, scratch)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], c.run(q, 16)[:, 16 - M:])
    check_attention(c, mine, outs[0], M, G)
    alone = torch.empty_like(mine)
    L, p = B.lib(), lambda t: t.data_ptr()
    assert L.ls_op_attention_kv4(p(mine), 1, M, p(pos), Hkv * G, Hkv, hd, page, p(c.table), c.table.shape[1], 16384, p(c.pool),
                                 c.pool.shape[0], p(alone), None, None, B._stream()) == 0
    check_attention(c, mine, alone, M, G)
    with pytest.raises(B.LsError):
        B.ls_op_attention_kv4(mine, pos, Hkv, hd, page, c.table, 16384, c.pool, alone, None, torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


def test_attention_split_rows_without_keys_and_captured():
    """two sequences over split caches, one with nothing to see: zeros; and the same from a replayed graph, whose scratch
    the binding takes from the graph's own memory, while an eager call uses another"""
    Hkv, G, hd, page = 1, 8, 128, 64
    c = Cache([9000, 0], Hkv, hd, page, 97, max_seq=8192 + 4096)
    q = rnd((2, 2, Hkv * G * hd), 98).bfloat16()
    assert B.ls_op_attention_kv4_scratch_bytes(2, 2, Hkv * G, Hkv, hd, c.max_seq) > 0
    eager = c.run(q, 2)
    check_attention(c, q, eager, 2, G)
    pos = torch.tensor([8998, -2], dtype=torch.int32, device="cuda")
    st, out = torch.cuda.Stream(), torch.zeros_like(q)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            B.ls_op_attention_kv4(q, pos, Hkv, hd, page, c.table, c.max_seq, c.pool, out)
            B.ls_op_attention_kv4(q, pos, Hkv, hd, page, c.table, c.max_seq, c.pool, out)
        for _ in range(3):
            out.fill_(7.0)
            graph.replay()
    again = c.run(q, 2)  # at the same time as the last replay
    st.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(out, eager) and torch.equal(again, eager)


def test_attention_over_the_longest_cache():
    """LS_KV4_MAX_SEQ positions, split: against 64-bit torch arithmetic on the expanded cache"""
    n, hd, page = 1 << 20, 64, 1024
    table = torch.randperm(n // page, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()[None]
    pool = empty_pool(n // page, 1, hd, page)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = rnd((1, n, 1, hd), 110).bfloat16(), rnd((1, n, 1, hd), 111).bfloat16()
    B.ls_op_append_kv4(k, v, zero, page, table, n, pool)
    kp, vp = (torch.empty((n // page, 1, page, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ls_op_expand_kv4(pool, zero, n, page, table, n, torch.arange(n // page, dtype=torch.int32, device="cuda")[None], kp, vp)
    q = rnd((1, 2, 8 * hd), 112, 3.0).bfloat16()
    out, status = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ls_op_attention_kv4(q, torch.tensor([n - 2], dtype=torch.int32, device="cuda"), 1, hd, page, table, n, pool, out, status)
    kd, vd = kp.view(n, hd).double(), vp.view(n, hd).double()
    for m in range(2):
        a = torch.softmax(q[0, m].view(8, hd).double() @ kd[:n - 1 + m].t() / hd ** 0.5, -1)
        ref, spread = (a @ vd[:n - 1 + m]).cpu().numpy(), (a @ vd[:n - 1 + m].abs()).cpu().numpy()
        assert (np.abs(vals(out)[0, m].reshape(8, hd) - ref) <= attention_tol(ref, spread, vals(v[0, :, 0]))).all()
    assert int(status) == 0


def test_every_split_of_the_longest_cache_counts():
    """LS_KV4_MAX_SEQ positions, 64 splits, in each of which another channel's values are raised by 2: the bound is one that a
    result without any one of them misses by a factor of 4 or more.
    A weight's absolute error, 2^-32 of the largest of its warp's 512 positions (64 splits of 4 CTAs of 8 warps), adds up to
    512 * 2^-32 of max |v| at most, as the warps' largest weights add up to no more than the sum.
    Then a key that has nearly all the weight, in each split in turn: the result is its value."""
    n, hd, page, G, M = 1 << 20, 64, 1024, 8, 2
    table = torch.randperm(n // page, generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()[None]
    pool = empty_pool(n // page, 1, hd, page)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    at = torch.arange(n, device="cuda") // 32 // 8 // 4 % 64  # split of a position: chunks of 32, 8 warps, 4 CTAs
    k, v = rnd((1, n, 1, hd), 200).bfloat16(), rnd((1, n, 1, hd), 201)
    v[0, torch.arange(n, device="cuda"), 0, at] += 2
    v = v.bfloat16()
    B.ls_op_append_kv4(k, v, zero, page, table, n, pool)
    kp, vp = (torch.empty((n // page, 1, page, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ls_op_expand_kv4(pool, zero, n, page, table, n, torch.arange(n // page, dtype=torch.int32, device="cuda")[None], kp, vp)
    q = rnd((1, 1, 1, hd), 202, 2.0).expand(1, M, G, hd).reshape(1, M, G * hd).bfloat16()
    q[0, :, hd:] = rnd((M, (G - 1) * hd), 203, 2.0).bfloat16()
    splits = B.ls_op_attention_kv4_scratch_bytes(1, M, G, 1, hd, n) // (4 * 16 * (hd + 2))  # 16 queries: (hd + 2) floats each
    assert splits == 64
    pos = torch.tensor([n - M], dtype=torch.int32, device="cuda")
    kd, vd = kp.view(n, hd).double(), vp.view(n, hd).double()

    def run():
        out = torch.empty_like(q)
        B.ls_op_attention_kv4(q, pos, 1, hd, page, table, n, pool, out)
        return torch.from_numpy(vals(out)).cuda().view(M, G, hd)

    out = run()
    for m in range(M):
        w = torch.exp(q[0, m].view(G, hd).double() @ kd[:n - M + 1 + m].t() / hd ** 0.5)
        vm, am = vd[:n - M + 1 + m], at[:n - M + 1 + m]
        ref, spread = (w @ vm) / w.sum(1, True), (w @ vm.abs()) / w.sum(1, True)
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2.0 ** -13) * spread + 512 * 2.0 ** -32 * float(vm.abs().max())
        assert bool(((out[m] - ref).abs() <= tol).all())
        for i in range(splits):
            keep = (am != i).double()
            wrong = ((w * keep) @ vm) / (w * keep).sum(1, True)
            assert bool((((wrong - ref).abs() > 4 * tol).any(1)).all()), (m, i)
    rng = np.random.default_rng(204)
    for i in range(splits):
        where = int(at.eq(i).nonzero()[int(rng.integers(0, 16000))])  # of 16384
        p = torch.tensor([where], dtype=torch.int32, device="cuda")
        loud = (8 * q[0, 0, :hd]).view(1, 1, 1, hd)  # outweighs all others together by 2^100 for the first head of either row
        B.ls_op_append_kv4(loud.contiguous(), v[:, where:where + 1].contiguous(), p, page, table, n, pool)
        got = run()[:, 0]
        assert bool(((got - vd[where]).abs() <= (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -13) * vd[where].abs() + 2.0 ** -40).all()), i
        B.ls_op_append_kv4(k[:, where:where + 1].contiguous(), v[:, where:where + 1].contiguous(), p, page, table, n, pool)


def test_packing_right_before_a_chained_linear():
    """with chained operations, which read weights ahead of time, the weights that the call before packs are the ones used"""
    N, K = 4096, 2048
    h = rnd((1, K), 120).bfloat16()
    ws = [rnd((N, K), 121 + i, 0.02).bfloat16() for i in range(6)]
    packed, outs, want = torch.zeros(B.ls_op_w4_bytes(N, K, 32), dtype=torch.uint8, device="cuda"), [], []
    for chained in (False, True):
        B.ls_op_chain(chained)
        try:
            for w in ws:
                o = torch.zeros((1, N), device="cuda")
                torch.cuda.synchronize()
                B.ls_op_quantize_w4(w, 32, packed)
                B.ls_op_linear_w4(packed, 32, h, o)
                (outs if chained else want).append(o)
        finally:
            B.ls_op_chain(False)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_expanding_right_before_a_chained_bf16_linear():
    N, K = 4096, 2048
    h = rnd((1, K), 140).bfloat16()
    packs = [torch.zeros(B.ls_op_w4_bytes(N, K, 32), dtype=torch.uint8, device="cuda") for _ in range(6)]
    for i, p in enumerate(packs):
        B.ls_op_quantize_w4(rnd((N, K), 141 + i, 0.02).bfloat16(), 32, p)
    w, outs, want = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"), [], []
    for chained in (False, True):
        B.ls_op_chain(chained)
        try:
            for p in packs:
                o = torch.zeros((1, N), device="cuda")
                torch.cuda.synchronize()
                B.ls_op_expand_w4(p, 32, w)
                B.ls_op_linear(B.LS_LINEAR_MMA, w, h, o)
                (outs if chained else want).append(o)
        finally:
            B.ls_op_chain(False)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("packing", [True, False])
def test_packing_first_and_chaining_afterwards(packing):
    """weights packed (or expanded) with chaining off, which is then turned on, and a norm between them and the linear
    layer: operations that start early use the new weights"""
    N, K = 4096, 2048
    x, gain = rnd((1, K), 150), torch.ones(K, device="cuda").bfloat16()
    ws = [rnd((N, K), 151 + i, 0.02).bfloat16() for i in range(6)]
    packs = [quantised(w, 32) for w in ws]
    packed, wide, outs, want = torch.zeros_like(packs[0]), torch.zeros_like(ws[0]), [], []
    for chained in (False, True):
        for w, p in zip(ws, packs):
            h, o = torch.zeros((1, K), device="cuda").bfloat16(), torch.zeros((1, N), device="cuda")
            torch.cuda.synchronize()
            if packing:
                B.ls_op_quantize_w4(w, 32, packed)
            else:
                B.ls_op_expand_w4(p, 32, wide)
            B.ls_op_chain(chained)
            try:
                B.ls_op_rmsnorm(x, gain, 1e-5, h)
                if packing:
                    B.ls_op_linear_w4(packed, 32, h, o)
                else:
                    B.ls_op_linear(B.LS_LINEAR_MMA, wide, h, o)
            finally:
                B.ls_op_chain(False)
            (outs if chained else want).append(o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("packing", [True, False])
@pytest.mark.parametrize("chained", [False, True])
def test_no_operation_overlaps_one_that_writes_weights(packing, chained):
    """the same calls captured and not run: whatever the switch said while packing, the operation that may start early
    depends on a launch behind the packing's, and that one on the packing's end"""
    drv = pytest.importorskip("cuda.bindings.driver")
    N, K = 256, 256
    x, gain, h = rnd((1, K), 160), torch.ones(K, device="cuda").bfloat16(), torch.zeros((1, K), device="cuda").bfloat16()
    w, o = rnd((N, K), 161).bfloat16(), torch.zeros((1, N), device="cuda")
    packed = quantised(w, 32)
    B.ls_op_expand_w4(packed, 32, w)
    B.ls_op_linear_w4(packed, 32, h, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        B.ls_op_chain(chained)
        try:
            if packing:
                B.ls_op_quantize_w4(w, 32, packed)
            else:
                B.ls_op_expand_w4(packed, 32, w)
            B.ls_op_chain(True)
            B.ls_op_rmsnorm(x, gain, 1e-5, h)
            B.ls_op_linear_w4(packed, 32, h, o)
        finally:
            B.ls_op_chain(False)
    raw = drv.CUgraph(graph.raw_cuda_graph())
    err, _, _, _, n = drv.cuGraphGetEdges_v2(raw)
    assert err == drv.CUresult.CUDA_SUCCESS
    err, start, end, data, n = drv.cuGraphGetEdges_v2(raw, n)
    assert err == drv.CUresult.CUDA_SUCCESS and n == 3
    early = drv.CUgraphDependencyType.CU_GRAPH_DEPENDENCY_TYPE_PROGRAMMATIC
    after = {int(a): (int(b), int(d.type) == int(early)) for a, b, d in zip(start, end, data)}
    node = (set(after) - {b for b, _ in after.values()}).pop()  # the packing
    overlaps = []
    while node in after:
        node, overlap = after[node]
        overlaps.append(overlap)
    assert overlaps[0] is False and overlaps[2] is True  # the packing's end; rmsnorm and linear are chained as ever


def test_chained_conversions_read_what_the_one_ahead_wrote():
    """append -> expand -> append of what was expanded -> attention, and expand -> pack, over buffers used again and again:
    the same bytes with operations that start early and ones that do not (the values are the format's own: a second packing
    changes nothing)"""
    n, Hkv, hd, page, N, K = 160, 2, 128, 32, 272, 384
    table, pd = torch.arange(5, dtype=torch.int32, device="cuda")[None], torch.zeros(1, dtype=torch.int32, device="cuda")
    last = torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    ks, vs = rnd((6, 1, n, Hkv, hd), 210).bfloat16(), rnd((6, 1, n, Hkv, hd), 211).bfloat16()
    ws, q = rnd((6, N, K), 212).bfloat16(), rnd((1, 1, 2 * Hkv * hd), 213).bfloat16()
    packs = [quantised(w, 32) for w in ws]
    a, b = empty_pool(5, Hkv, hd, page), empty_pool(5, Hkv, hd, page)
    kp, vp = (torch.zeros((5, Hkv, page, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wide, again, results = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(packs[0]), []
    for chained in (False, True):
        left = []
        for i in range(6):
            out = torch.zeros_like(q)
            torch.cuda.synchronize()
            B.ls_op_chain(chained)
            try:
                B.ls_op_append_kv4(ks[i], vs[i], pd, page, table, n, a)
                B.ls_op_expand_kv4(a, pd, n, page, table, n, table, kp, vp)
                for j in range(5):  # a page of rows at a time, heads outermost
                    pj = torch.tensor([j * page], dtype=torch.int32, device="cuda")
                    B.ls_op_append_kv4(kp[j].transpose(0, 1)[None], vp[j].transpose(0, 1)[None], pj, page, table, n, b)
                B.ls_op_attention_kv4(q, last, Hkv, hd, page, table, n, b, out)
                B.ls_op_expand_w4(packs[i], 32, wide)
                B.ls_op_quantize_w4(wide, 32, again)
            finally:
                B.ls_op_chain(False)
            torch.cuda.synchronize()
            left.append((a.clone(), b.clone(), out, again.clone()))
            assert torch.equal(a, b) and torch.equal(again, packs[i])
        results.append(left)
    assert all(torch.equal(x, y) for u, v in zip(*results) for x, y in zip(u, v))


def test_rows_of_one_sequence_and_head_with_odd_strides():
    """strides of dimensions of one do not matter"""
    x = rnd((3, 5 * 64 + 8), 130).bfloat16()
    k = x.as_strided((1, 3, 1, 64), (3, 5 * 64 + 8, 7, 1))
    pool, table = empty_pool(1, 1, 64, 16), torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    want = reference_append(pool.cpu().numpy().copy(), vals(k), vals(k), [2], table.cpu().numpy(), 16, 16)
    B.ls_op_append_kv4(k, k, torch.tensor([2], dtype=torch.int32, device="cuda"), 16, table, 16, pool)
    assert np.array_equal(pool.cpu().numpy(), want)


def test_k_and_v_whose_strides_differ_where_there_is_one():
    """a row cut out of a longer tensor and one that stands alone; strides that differ elsewhere are refused"""
    v, k = rnd((1, 9, 2, 64), 131).bfloat16(), rnd((1, 1, 2, 64), 132).bfloat16()
    table, pd = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda")
    for a, b in ((k, v[:, 4:5]), (v[:, 4:5], k), (k[:, :, 1:], v[:, 4:5].transpose(1, 2)[:, 1:])):
        pool = empty_pool(1, a.shape[2], 64, 16)
        want = reference_append(pool.cpu().numpy().copy(), vals(a), vals(b), [3], table.cpu().numpy(), 16, 16)
        B.ls_op_append_kv4(a, b, pd, 16, table, 16, pool)
        assert np.array_equal(pool.cpu().numpy(), want)
    with pytest.raises(B.LsError):
        B.ls_op_append_kv4(v[:, :2], v[:, ::4][:, :2], pd, 16, table, 16, empty_pool(1, 2, 64, 16))


def test_two_streams_at_once():
    """linear and attention calls on two streams, neither waiting for the other, give what each gives alone"""
    N, K = 4096, 2048
    packed, h = quantised(rnd((N, K), 100, 0.02).bfloat16(), 32), rnd((2, 8, K), 101).bfloat16()
    c = Cache([3000, 2500], 4, 128, 64, 102)
    q = rnd((2, 4, 8 * 128), 103).bfloat16()
    want = torch.empty((2, 8, N), device="cuda")
    for i in range(2):
        B.ls_op_linear_w4(packed, 32, h[i], want[i])
    ref = c.run(q, 4)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                o = torch.empty((8, N), device="cuda")
                B.ls_op_linear_w4(packed, 32, h[i], o)
                outs.append((o, want[i], c.run(q, 4)))
    torch.cuda.synchronize()
    for o, w, a in outs:
        assert torch.equal(o, w) and torch.equal(a, ref)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("chained", [False, True])
def test_a_layer_of_draft_and_verify_passes_on_4_bit_weights_and_cache(chained):
    """A prompt and then passes of 1, 1 and 3 rows through one layer's attention block, as a decode loop runs them:
    norm, q|k|v projections, rotary embedding (into a bf16 page), append, attention, output projection with the
    residual.  The prompt's rows go through the prompt-pass operations on expanded weights and cache.  Every step is
    checked against 64-bit arithmetic on what the step before it left; chained: with the operations linked by
    programmatic dependent launch."""
    D, Hq, Hkv, hd, page, max_seq, group, theta = 256, 4, 2, 64, 16, 96, 32, 1e4
    qw, kw = Hq * hd, Hkv * hd
    wqkv, wo = rnd((qw + 2 * kw, D), 80, 0.06).bfloat16(), rnd((D, qw), 81, 0.06).bfloat16()
    pqkv, po = quantised(wqkv, group), quantised(wo, group)
    gain = (1 + 0.1 * rnd((D,), 82)).bfloat16()
    table = torch.tensor([[3, 0, 5, 1, 4, 2]], dtype=torch.int32, device="cuda")
    pool = empty_pool(6, Hkv, hd, page)
    stage = torch.zeros((2, 1, Hkv, page, hd), dtype=torch.bfloat16, device="cuda")  # one bf16 page for new k, one for v
    at_stage = torch.zeros(6, dtype=torch.int32, device="cuda")
    x = rnd((16 + 1 + 1 + 3, D), 83)
    pos, left = 0, []
    B.ls_op_chain(chained)
    try:
        for M in (16, 1, 1, 3):
            rows = x[pos:pos + M].clone()
            h = torch.empty((M, D), dtype=torch.bfloat16, device="cuda")
            qkv = torch.empty((M, qw + 2 * kw), device="cuda")
            q, o = torch.empty((1, M, qw), dtype=torch.bfloat16, device="cuda"), torch.empty((1, M, qw), dtype=torch.bfloat16, device="cuda")
            pd = torch.tensor([pos], dtype=torch.int32, device="cuda")
            before = rows.clone()
            B.ls_op_rmsnorm(rows, gain, 1e-5, h)
            B.ls_op_linear_w4(pqkv, group, h, qkv)
            B.ls_op_rope_append(qkv, pos, Hq, Hkv, hd, theta, page, at_stage, max_seq, q, stage[0], stage[1])
            s0 = pos % page  # rows of a pass stay within the staging page here: 0..15, 0, 1, 2..4
            k, v = (stage[i, 0].transpose(0, 1)[None, s0:s0 + M] for i in range(2))
            B.ls_op_append_kv4(k, v, pd, page, table, max_seq, pool)
            B.ls_op_attention_kv4(q, pd, Hkv, hd, page, table, max_seq, pool, o)
            B.ls_op_linear_w4(po, group, o[0], rows, True)
            torch.cuda.synchronize()
            left.append((pos, M, before, h, qkv, q, o, rows, k.clone(), v.clone()))
            pos += M
    finally:
        B.ls_op_chain(False)
    ks, vs = [], []
    for pos, M, before, h, qkv, q, o, rows, k, v in left:
        ref, spread = linear_reference(wqkv, group, h)
        assert (np.abs(qkv.cpu().numpy() - ref) <= linear_tol(D, group, spread)).all()
        ks.append(R.values(*R.quantise(vals(k[0]), 32), 32))
        vs.append(R.values(*R.quantise(vals(v[0]), 32), 32))
        kk, vv = np.concatenate(ks), np.concatenate(vs)
        for m in range(M):
            ref, spread = R.attention(vals(q)[0, m].reshape(Hq, hd), kk, vv, pos + m, Hq // Hkv)
            assert (np.abs(vals(o)[0, m].reshape(Hq, hd) - ref) <= attention_tol(ref, spread, vv)).all()
        ref, spread = linear_reference(wo, group, o[0])
        base = before.cpu().numpy().astype(np.float64)
        assert (np.abs(rows.cpu().numpy() - base - ref) <= linear_tol(qw, group, spread) + 2.0 ** -23 * np.abs(base + ref)).all()
    # the prompt again by the prompt-pass operations on expanded weights and an expanded cache
    _, M, _, h, qkv, q, o, *_ = left[0]
    wide = torch.empty_like(wqkv)
    B.ls_op_expand_w4(pqkv, group, wide)
    c, status = torch.empty_like(qkv), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ls_op_gemm(h, wide, c, False, status)
    _, spread = linear_reference(wqkv, group, h)
    assert (np.abs((c - qkv).cpu().numpy()) <= 2 * linear_tol(D, group, spread)).all()
    kp = torch.full((6, Hkv, page, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    vp = torch.full_like(kp, float("nan"))
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.ls_op_expand_kv4(pool, zero, 21, page, table, max_seq, table, kp, vp, status)
    a = torch.empty_like(q[0])
    B.ls_op_prefill_attention(q[0], 0, Hq, Hkv, hd, page, table[0], max_seq, kp, vp, a, status)
    for m in range(M):  # both within their bounds of the same values: bf16 weights p there (2^-9), two results rounded
        ref, spread = R.attention(vals(q)[0, m].reshape(Hq, hd), kk, vv, m, Hq // Hkv)
        assert (np.abs(vals(a)[m].reshape(Hq, hd) - ref) <= 2.0 ** -8 * np.abs(ref).max() + 2.0 ** -8 * spread).all()
    assert int(status) == 0
