"""Log probabilities, entropies and top alternatives against a 64-bit softmax."""
import math

import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import close, logprobs64

pytestmark = pytest.mark.gpu


def run(x, targets, top, ws=None):
    rows = x.shape[0]
    dev = x.device
    lp = torch.full((rows,), 9.0, device=dev) if targets is not None else None
    ent = torch.full((rows,), 9.0, device=dev)
    ids = torch.full((rows, top), -9, dtype=torch.int32, device=dev) if top else None
    tlp = torch.full((rows, top), 9.0, device=dev) if top else None
    B.aio_logprobs(x, None if targets is None else targets.to(dev), lp, ent, ids, tlp, ws=ws)
    torch.cuda.synchronize()
    return lp, ent, ids, tlp


def check(x, targets, top, device_x=None):
    lp, ent, ids, tlp = run(x.cuda() if device_x is None else device_x, targets, top)
    wlp, went, wids, wtlp, ltol, etol = logprobs64(x, targets, top)
    close(ent, went, etol + 2.0 ** -24 * went.abs())
    if targets is not None:
        close(lp, wlp, ltol + 2.0 ** -24 * wlp.abs())
    if top:
        assert torch.equal(ids.cpu().long(), wids)
        close(tlp, wtlp, ltol[:, None] + 2.0 ** -24 * wtlp.abs())


SHAPES = [(1, 1, 1), (1, 2, 2), (3, 7, 5), (2, 64, 32), (5, 255, 1), (4, 256, 32), (1, 8192, 8),
          (1, 8193, 8), (2, 32000, 5), (1, 131072, 32), (300, 1000, 3), (3, 50257, 20),
          (260, 9000, 7)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n,top", SHAPES)
def test_rows(rows, n, top, dtype):
    g = torch.Generator().manual_seed(n)
    x = (3 * torch.randn((rows, n), generator=g)).to(dtype)
    t = torch.randint(0, n, (rows,), generator=g, dtype=torch.int32)
    check(x, t, top)
    check(x, None, 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_order_of_ties_and_runs(dtype):
    """Equal values, rising, falling and blocked ones: the lower index first, and no
    arrangement loses a candidate."""
    n, top = 20000, 32
    base = torch.arange(n, dtype=torch.float32) / 64
    rows = [torch.zeros(n), base, base.flip(0), (torch.arange(n) % 256 == 255).float() * 5,
            torch.where(torch.arange(n) % 256 == 3, base, torch.zeros(n)),
            torch.where(torch.arange(n) >= n - 40, torch.ones(n), -torch.ones(n)),
            -torch.zeros(n), (torch.arange(n) % 2).float() * -0.0]
    x = torch.stack(rows).to(dtype)
    t = torch.tensor([0, 1, n - 1, 255, 3, n - 1, 5, 6], dtype=torch.int32)
    check(x, t, top)
    check(x.repeat(70, 1), t.repeat(70), 5)  # one slice per row


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n", [(1, 2049), (1, 4100), (2, 8195), (120, 9000), (1, 131072),
                                    (200, 17000), (3, 600001)])
def test_joined_slices(rows, n, dtype):
    """Rows split over workgroups: more alternatives than slices or fewer, the largest
    values all in the first slice, all in the last, one in each, or nearly nothing left
    in a slice."""
    g = torch.Generator().manual_seed(n)
    x = torch.randn((rows, n), generator=g).to(dtype)
    kinds = [x[0].clone()]
    for at in (slice(0, 40), slice(n - 40, n), slice(0, n, max(n // 40, 1))):
        y = x[0].clone()
        y[at] += 9
        kinds.append(y)
    few = torch.full((n,), -math.inf, dtype=dtype)
    few[[1, n // 2, n - 1]] = 1.0
    few[n - 3] = 2.0
    kinds.append(few)
    for y in kinds:
        x[-1] = y
        t = torch.randint(0, n, (rows,), generator=g, dtype=torch.int32)
        for top in (1, 7, 32):
            check(x, t, top)


def test_targets_outside():
    x = torch.randn((5, 100))
    t = torch.tensor([-1, 100, -100, 99, 1 << 30], dtype=torch.int32)
    check(x, t, 3)


@pytest.mark.parametrize("n", [40, 9000, 33000])
def test_forbidden_and_not_finite(n):
    inf = math.inf
    x = torch.randn((9, n))
    x[0, 5:] = -inf                 # few allowed
    x[1] = -inf                     # none
    x[2, 7] = inf
    x[3, 11] = math.nan
    x[4, n - 1] = math.nan
    x[4, 3] = inf
    x[4, 9] = math.nan
    x[5] = torch.finfo(torch.float32).min
    x[6] = torch.finfo(torch.float32).max
    x[7, :] = -inf
    x[7, n - 2] = 3.0               # one allowed
    x[8] = math.nan
    t = torch.tensor([5, 0, 7, 11, 3, 1, 2, n - 2, 0], dtype=torch.int32)
    check(x, t, 8)


@pytest.mark.parametrize("gap", [20.0, 60.0, 200.0])
def test_confident_rows(gap):
    """Probabilities next to 1: log z = log(1 + small) keeps its digits (64-bit sums):
    relative, not absolute, to what the tail holds."""
    x = torch.zeros((2, 5000))
    x[0, 17] = gap
    x[1, 4999] = gap
    t = torch.tensor([17, 4999], dtype=torch.int32)
    lp, ent, _, _ = run(x.cuda(), t, 0)
    _, went, _, _, _, _ = logprobs64(x, t, 0)
    exact = -math.log1p(4999 * math.exp(-gap))
    # a 32-bit e^-gap is off by its argument's rounding (24 bits of `gap`) and 2^-22
    rel = 2.0 ** -23 * gap + 2.0 ** -20
    assert (lp.double().cpu() - exact).abs().max() <= rel * abs(exact) + 1e-45 + 2 ** -53 * 4
    assert (ent.double().cpu() - went).abs().max() <= rel * 2 * float(went.max()) + 2 ** -50


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [2, 300])
def test_strides_and_alignment(rows, dtype):
    """Rows inside wider ones, starting at an odd element."""
    g = torch.Generator().manual_seed(9)
    wide = torch.randn((rows, 10007), generator=g).to(dtype)
    t = torch.randint(0, 9001, (rows,), generator=g, dtype=torch.int32)
    d = wide.cuda()
    for off in (0, 1, 3, 8):
        check(wide[:, off: off + 9001], t, 6, d[:, off: off + 9001])


def test_next_to_argmax():
    """The first alternative is aio_argmax's token, whatever the row holds."""
    import synth
    cfg = synth.CONFIGS["tiny"].with_(name="lp")
    dm = B.DeviceModel(cfg, synth.make_weights(cfg))
    x = torch.randn((4, cfg.vocab), device="cuda")
    x[1, 100:200] = 50.0
    x[2, 33] = math.nan
    x[3, 44], x[3, 45] = math.inf, math.inf
    torch.cuda.synchronize()
    out = torch.zeros(4, dtype=torch.int32, device="cuda")
    dm.argmax(x, 4, out)
    dm.sync()
    _, _, ids, _ = run(x, None, 1)
    assert torch.equal(ids[:, 0], out)
    dm.close()


def test_captured_and_replayed():
    x = torch.randn((2, 32000), device="cuda")
    t = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    lp, ent = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    ids = torch.empty((2, 4), dtype=torch.int32, device="cuda")
    tlp = torch.empty((2, 4), device="cuda")
    B.aio_logprobs(x, t, lp, ent, ids, tlp)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.aio_logprobs(x, t, lp, ent, ids, tlp)
    for _ in range(4):
        x.normal_()
        g.replay()
        torch.cuda.synchronize()
        got = [a.clone() for a in (lp, ent, ids, tlp)]
        B.aio_logprobs(x, t, lp, ent, ids, tlp)
        torch.cuda.synchronize()
        for a, b in zip(got, (lp, ent, ids, tlp)):
            assert torch.equal(a, b)
        assert torch.equal(got[2].cpu().long(), logprobs64(x.cpu(), t.cpu(), 4)[2])


def test_binding_refuses():
    x = torch.randn((2, 50), device="cuda")
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    f = torch.empty(2, device="cuda")
    ids = torch.empty((2, 3), dtype=torch.int32, device="cuda")
    tl = torch.empty((2, 3), device="cuda")
    ok = dict(logits=x, targets=t, logprob=f, entropy=f.clone(), top_ids=ids, top_logprobs=tl)
    for bad in (dict(logits=x.double()), dict(logits=x.t()), dict(targets=t.long()),
                dict(targets=t[:1]), dict(logprob=f.double()), dict(top_ids=ids.long()),
                dict(top_logprobs=tl[:, :2]), dict(top_ids=None), dict(logits=x.cpu())):
        with pytest.raises(ValueError):
            B.aio_logprobs(**{**ok, **bad})
    with pytest.raises(B.AioError):
        B.aio_logprobs(**{**ok, "targets": None})
