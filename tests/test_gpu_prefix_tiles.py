"""Prompt rows behind a shared prefix in tiles of 256 rows, every row and head against a plain
64-bit evaluation.

Tolerances: those of paged_cases.attention64 element by element.  On average: a weight's rounding to
bf16 is off by at most 2^-8 of it, 2^-8 / sqrt(3) in the mean square, an output's too; both are
independent from one element to the next, and with values of either sign the output's own size
and its error add up alike, so that the 2-norm of all errors is at most sqrt(2 / 3) 2^-8 =
3.2e-3 of the outputs'; 4e-3 leaves a quarter more."""
import math

import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import U, cu
from tests.test_gpu_prefix_attention import BF16, Grouped, rows
from tests.test_prefix_plan import plan

# rows and keys of each sequence, the groups, the holes (sequence, page of 16 keys)
CASES = {
    "turns": ([(900, 1400), (700, 1201), (560, 1119)], [(0, 3, 490)], ()),
    # the second begins within the prefix, the third at its end; the last tile has one row
    "within": ([(1000, 1500), (500, 700), (430, 874), (127, 640)], [(0, 4, 450)], ()),
    "holes": ([(900, 1400), (700, 1201), (560, 1119)], [(0, 3, 490)], ((0, 3), (0, 29), (1, 40), (2, 69))),
    # a short prompt between two groups, an idle place
    "groups": ([(800, 1100), (300, 555), (3, 40), (0, 0), (700, 1000), (400, 712)],
               [(0, 2, 256), (4, 6, 300)], ()),
}
HEADS = [(128, 16, 64), (128, 16, 128), (180, 12, 128)]


@pytest.mark.parametrize("H,Hkv,hd", HEADS)
@pytest.mark.parametrize("name", list(CASES))
def test_the_cases_take_tiles_of_256(name, H, Hkv, hd):
    shape, groups, _ = CASES[name]
    for key_bytes in (1, 2):
        p = plan(len(shape), sum(a for a, _ in shape), max(b for _, b in shape), len(groups),
                 max(g[2] for g in groups), H, Hkv, hd, B.AIO_BF16, True, key_bytes)
        assert p[0] == 8 and p[2] >= 1 and p[4] > 0


def check_all(out, lse, q, case, ql, what):
    """Every row, in 64 bits on the GPU, a kv head at a time."""
    H, hd = q.shape[1:]
    scale = hd ** -0.5
    q64 = q.cuda().double()
    err2 = out2 = 0.0
    r0 = 0
    for i, n in enumerate(ql):
        if n == 0:
            continue
        nk = case.k_len[i]
        G = H // case.keys[i].shape[1]
        ahead = nk - n + torch.arange(n, device="cuda")
        see = torch.arange(nk, device="cuda")[None, :] <= ahead[:, None]
        see = (see & case.visible[i].cuda()[None, :]).repeat_interleave(G, 0)
        for h in range(case.keys[i].shape[1]):
            k = case.keys[i][:, h].cuda().double().t().contiguous()
            v = case.values[i][:, h].cuda().double()
            x = q64[r0: r0 + n, h * G: (h + 1) * G].reshape(n * G, hd)
            s = torch.mm(x, k) * scale
            b = torch.mm(x.abs(), k.abs()) * scale
            d = (8 * math.sqrt(3 * hd) * U * b + 1.5 * U * s.abs()).masked_fill_(~see, 0)
            d = d.amax(1) + 2.0 ** -22
            s = s.masked_fill_(~see, -math.inf)
            want_l = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1).nan_to_num_()  # (rows that see nothing: zeros)
            o, a = torch.mm(p, v), torch.mm(p, v.abs())
            tol = (2 * d[:, None] + 2.0 ** -20) * a + 2.0 ** -8 * (a + o.abs()) * (1 + 2.0 ** -7)
            got = out[r0: r0 + n, h * G: (h + 1) * G].reshape(n * G, hd).double()
            err = (got - o).abs()
            assert (err <= tol).all(), "%s: sequence %d, head %d, row %d" % (
                what, i, h, int((err > tol).any(1).nonzero()[0]) // G)
            err2 += float((got - o).square().sum())
            out2 += float(o.square().sum())
            l = lse[r0: r0 + n, h * G: (h + 1) * G].reshape(n * G).double()
            ok = ((l - want_l).abs() <= d + 2.0 ** -22 * (1 + want_l.abs())) | (l == want_l)
            assert ok.all(), "%s: log-sum-exp of sequence %d, head %d" % (what, i, h)
        r0 += n
    assert math.sqrt(err2) <= 4e-3 * math.sqrt(out2), (what, math.sqrt(err2 / out2))


@pytest.mark.gpu
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("H,Hkv,hd", HEADS)
@pytest.mark.parametrize("name", list(CASES))
def test_every_row(name, H, Hkv, hd, q8):
    shape, groups, holes = CASES[name]
    ql, kl = [a for a, _ in shape], [b for _, b in shape]
    p = Grouped(kl, groups, Hkv, hd, q8=q8, holes=holes)
    n = sum(ql)
    q = rows(n + 2, H, hd, BF16)  # two rows of no sequence
    for kw in (dict(max_len=max(kl), max_prefix=max(g[2] for g in groups)), dict()):
        out, l = p.run(q, ql, **kw)
        check_all(out, l, q, p.case, ql, "%s %s" % (name, kw))
        assert (out[n:] == 9).all() and (l[n:] == 9).all()
