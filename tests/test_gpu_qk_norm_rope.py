"""The norm and rotation of query and key rows against a plain 64-bit evaluation.

Tolerance.  With u = 2^-24: the sum of hd <= 128 squares adds 16 of them in a lane and then
over 8 lanes, at most 19 additions deep, and each square rounds once: 20 u of the sum, so 10 u of the
square root; the division by hd (exact), the addition of eps and the reciprocal root add 0.5, 0.5
and 2 u; the two products 2 u: a normalised element is off by at most 15 u of itself.  Cosine
and sine: the argument, at most 1/4 half turn, rounds by 2^-27, pi 2^-27 < 0.4 u of the angle, and
the functions to 2 u: 2.4 u.  The rotation's two products and one addition: 2 u of |p| + |q|.  Together
below 20 u (|p| + |q|).  The angle itself, in 64 bits on both sides: two roundings of the
frequency and one of the product, 2^-51 of it on each side, 2^-50.  bf16 results round once
more, 2^-8 of themselves."""
import math

import pytest
import torch

from paper_2604_09752_amd import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def norm64(x, pos, w, eps, base):
    """(result, tolerance) in 64 bits; x [rows, heads, hd]."""
    hd = x.shape[2]
    y = x.double()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w.double()
    t = pos.double()[:, None, None] * base ** (-2.0 * torch.arange(hd // 2).double() / hd)
    a, b = y[..., : hd // 2], y[..., hd // 2:]
    c, s = t.cos(), t.sin()
    out = torch.cat((a * c - b * s, b * c + a * s), -1)
    size = a.abs() + b.abs()
    tol = size * (20 * U + 2.0 ** -50 * t.abs())
    tol = torch.cat((tol, tol), -1)
    if x.dtype == BF16:
        tol = tol + 2.0 ** -8 * (out.abs() + tol)
    return out, tol


def check(got, x, pos, w, eps=1e-5, base=1e4):
    want, tol = norm64(x, pos, w, eps, base)
    err = (got.double().cpu() - want).abs()
    # (results below the smallest normal float may lose all of themselves)
    assert (err <= tol + 2.0 ** -126).all(), float((err / (tol + 1e-300)).max())


def make(n, H, Hkv, hd, dtype, far=4096, seed=1):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn((n, H + 2 * Hkv, hd), generator=g) * 1.5).to(dtype)
    pos = torch.randint(0, far, (n,), generator=g, dtype=torch.int32)
    w = [(1 + 0.1 * torch.randn(hd, generator=g)).to(BF16) for _ in range(2)]
    return qkv, pos, w


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,H,Hkv,hd", [
    (1, 1, 1, 64), (1, 16, 8, 128), (3, 4, 4, 64), (8, 32, 8, 128), (17, 16, 2, 64),
    (5, 33, 3, 128), (1000, 2, 1, 128), (1500, 4, 4, 64), (1027, 40, 8, 128), (1030, 71, 1, 64)])
def test_rows(n, H, Hkv, hd, dtype):
    """Queries and keys inside the rows that a product leaves them in, outputs apart."""
    qkv, pos, w = make(n, H, Hkv, hd, dtype)
    d = qkv.cuda()
    q, k = d[:, :H], d[:, H: H + Hkv]
    qo = torch.full(q.shape, 9.0, dtype=dtype, device="cuda")
    ko = torch.full((n, Hkv + 1, hd), 9.0, dtype=dtype, device="cuda")
    B.aio_qk_norm_rope(q, k, pos.cuda(), qo, ko[:, :Hkv], q_weight=w[0].cuda(),
                       k_weight=w[1].cuda())
    check(qo, qkv[:, :H], pos, w[0])
    check(ko[:, :Hkv], qkv[:, H: H + Hkv], pos, w[1])
    assert (ko[:, Hkv:] == 9).all() and torch.equal(d.cpu(), qkv)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 40, 1100])
def test_in_place(n, dtype):
    qkv, pos, w = make(n, 8, 2, 128, dtype)
    d = qkv.cuda()
    q, k = d[:, :8], d[:, 8:10]
    apart = torch.empty(q.shape, dtype=dtype, device="cuda"), torch.empty(k.shape, dtype=dtype,
                                                                        device="cuda")
    kw = dict(q_weight=w[0].cuda(), k_weight=w[1].cuda())
    B.aio_qk_norm_rope(q, k, pos.cuda(), *apart, **kw)
    B.aio_qk_norm_rope(q, k, pos.cuda(), q, k, **kw)
    assert torch.equal(q, apart[0]) and torch.equal(k, apart[1])
    assert torch.equal(d[:, 10:].cpu(), qkv[:, 10:])  # the values beside them
    check(q, qkv[:, :8], pos, w[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weights_eps_and_base(dtype):
    qkv, pos, w = make(9, 4, 2, 64, dtype)
    d = qkv.cuda()
    for qw, kw in ((None, None), (w[0], None), (None, w[1])):
        for eps, base in ((1e-5, 1e4), (1e-6, 5e5), (0.5, 1.5), (1e-12, 1e7)):
            qo, ko = torch.empty_like(d[:, :4]), torch.empty_like(d[:, 4:6])
            B.aio_qk_norm_rope(d[:, :4], d[:, 4:6], pos.cuda(), qo, ko,
                               q_weight=None if qw is None else qw.cuda(),
                               k_weight=None if kw is None else kw.cuda(), eps=eps, base=base)
            # (eps and base are floats in the call)
            e, b = float(torch.tensor(eps)), float(torch.tensor(base))
            check(qo, qkv[:, :4], pos, qw, e, b)
            check(ko, qkv[:, 4:6], pos, kw, e, b)


def test_positions_of_any_size():
    pos = torch.tensor([0, 1, -1, 2047, 131071, 999983, (1 << 24) + 1, -(1 << 24) - 3, (1 << 31) - 1,
                        -(1 << 31)], dtype=torch.int32)
    n = len(pos)
    for hd in (64, 128):
        qkv, _, w = make(n, 3, 2, hd, F32)
        d = qkv.cuda()
        qo, ko = torch.empty_like(d[:, :3]), torch.empty_like(d[:, 3:5])
        B.aio_qk_norm_rope(d[:, :3], d[:, 3:5], pos.cuda(), qo, ko)
        check(qo, qkv[:, :3], pos, None)
        check(ko, qkv[:, 3:5], pos, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e-30, 1e-15, 1e15, 1e25, 3e38])
def test_magnitudes(size, dtype):
    """Elements whose squares underflow or pass the largest float."""
    qkv, pos, w = make(6, 2, 1, 128, F32)
    qkv = (qkv / qkv.abs().amax(-1, keepdim=True) * size).to(dtype)
    qkv[3, 0, 5:] = 0
    qkv[4] = 0
    d = qkv.cuda()
    qo, ko = torch.empty_like(d[:, :2]), torch.empty_like(d[:, 2:3])
    B.aio_qk_norm_rope(d[:, :2], d[:, 2:3], pos.cuda(), qo, ko, q_weight=w[0].cuda())
    check(qo, qkv[:, :2], pos, w[0], float(torch.tensor(1e-5)))
    check(ko, qkv[:, 2:3], pos, None, float(torch.tensor(1e-5)))
    assert (qo[4] == 0).all()


def test_what_is_not_finite_stays_in_its_head():
    qkv, pos, w = make(4, 3, 2, 64, F32)
    bad = qkv.clone()
    bad[1, 1, 7] = float("nan")
    bad[2, 3, 40] = float("inf")
    d = bad.cuda()
    qo, ko = torch.empty_like(d[:, :3]), torch.empty_like(d[:, 3:5])
    B.aio_qk_norm_rope(d[:, :3], d[:, 3:5], pos.cuda(), qo, ko)
    assert torch.isnan(qo[1, 1]).all()
    assert not torch.isfinite(ko[2, 0, [8, 40]]).any()
    qo[1, 1], ko[2, 0] = 0, 0
    want, tol = norm64(qkv[:, :3], pos, None, 1e-5, 1e4)
    want[1, 1] = 0
    assert ((qo.double().cpu() - want).abs() <= tol).all()
    want, tol = norm64(qkv[:, 3:5], pos, None, 1e-5, 1e4)
    want[2, 0] = 0
    assert ((ko.double().cpu() - want).abs() <= tol).all()


def test_no_rows():
    z = torch.empty((0, 4, 64), device="cuda")
    B.aio_qk_norm_rope(z, z.clone(), torch.empty(0, dtype=torch.int32, device="cuda"), z, z)


def test_offsets_past_32_bits():
    """Rows more than 2^32 bytes apart."""
    n, apart = 3, (1 << 30) + 1024
    buf = torch.zeros(2 * apart + 4 * 64, device="cuda")
    wide = buf.as_strided((n, 4, 64), (apart, 64, 1))
    qkv, pos, w = make(n, 2, 2, 64, F32)
    wide.copy_(qkv[:, :4].cuda())
    B.aio_qk_norm_rope(wide[:, :2], wide[:, 2:4], pos.cuda(), wide[:, :2], wide[:, 2:4])
    check(wide[:, :2], qkv[:, :2], pos, None)
    check(wide[:, 2:4], qkv[:, 2:4], pos, None)


def test_a_side_stream_and_a_graph():
    qkv, pos, w = make(20, 8, 2, 128, BF16)
    d, p = qkv.cuda(), pos.cuda()
    qo, ko = torch.empty_like(d[:, :8]), torch.empty_like(d[:, 8:10])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        B.aio_qk_norm_rope(d[:, :8], d[:, 8:10], p, qo, ko)
    torch.cuda.current_stream().wait_stream(st)
    check(qo, qkv[:, :8], pos, None)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.aio_qk_norm_rope(d[:, :8], d[:, 8:10], p, qo, ko)
    for seed in (5, 6, 7):
        qkv, pos, _ = make(20, 8, 2, 128, BF16, far=1 << 20, seed=seed)
        d.copy_(qkv)
        p.copy_(pos)
        g.replay()
        torch.cuda.synchronize()
        check(qo, qkv[:, :8], pos, None)
        check(ko, qkv[:, 8:10], pos, None)
