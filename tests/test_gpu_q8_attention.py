"""Attention over pages of 8-bit codes against a plain 64-bit evaluation of what the codes
stand for."""
import math

import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import PoolCase, attention64, check_attention, cu
from tests.q8_cases import Q8Pool, quantise64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rows(n, H, hd, dtype, seed=1):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, H, hd), generator=g).to(dtype)


def run(pool, q, ql=None, lse=True, fill=9.0, **kw):
    k, v, ke, ve, lens, table = pool.device()
    qd = q.cuda()
    out = torch.full_like(qd, fill)
    l = torch.full(q.shape[:2], fill, device="cuda") if lse else None
    if ql is not None:
        kw["cu_q"] = cu(ql).cuda()
    B.aio_q8_attention(qd, k, v, ke, ve, lens, table, out, lse=l, **kw)
    torch.cuda.synchronize()
    return out, l


def ref(case, q, ql, visible=None, **kw):
    return attention64(q, case.keys, case.values, ql, case.k_len, visible, **kw)


LENS = [0, 1, 2, 31, 32, 33, 64, 127, 128, 129, 257, 500]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,Hkv,hd,page,layout", [
    (4, 4, 64, 16, "plain"), (16, 8, 128, 16, "interleaved"), (6, 2, 64, 8, "plain"),
    (8, 2, 128, 32, "plain"), (16, 1, 64, 64, "interleaved"), (8, 1, 128, 256, "plain"),
    (15, 3, 128, 8, "plain")])
def test_step(H, Hkv, hd, page, layout, dtype):
    pool = Q8Pool(PoolCase(LENS, Hkv, hd, page, seed=H), layout)
    q = rows(len(LENS), H, hd, dtype)
    want = ref(pool.case, q, [1] * len(LENS))
    for max_len in (None, 500):
        out, l = run(pool, q, max_len=max_len)
        check_attention(out, l, want, "max_len %s" % max_len)
    again, _ = run(pool, q, lse=False, max_len=500)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,length,hd", [(1, 1, 64), (1, 129, 128), (1, 4096, 128), (3, 2999, 64),
                                         (2, 9001, 128)])
def test_step_split_over_the_keys(n, length, hd, dtype):
    lens = [max(length - 7 * i, 1) for i in range(n)]
    pool = Q8Pool(PoolCase(lens, 2, hd, 16, seed=length))
    q = rows(n, 8, hd, dtype)
    want = ref(pool.case, q, [1] * n)
    for max_len in (max(lens), 40000):
        out, l = run(pool, q, max_len=max_len)
        check_attention(out, l, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 90])
def test_step_ragged_batches(n, dtype):
    """Splits with keys come first for up to 64 sequences, and one after the other beyond;
    idle places among them, whatever the workspace holds."""
    lens = [(37 * i * i + 1) % 700 if i % 7 else 0 for i in range(n)]
    lens[n // 2] = 1500
    pool = Q8Pool(PoolCase(lens, 2, 64, 16, seed=n))
    q = rows(n, 4, 64, dtype)
    want = ref(pool.case, q, [1] * n)
    for max_len in (1500, 9000):
        need = B.aio_q8_workspace_bytes(n, n, max_len, 4, 2, 64)
        assert need > 0
        for fill in (0, 255):
            ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
            out, l = run(pool, q, max_len=max_len, ws=ws)
            check_attention(out, l, want, (max_len, fill))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("page,hd", [(16, 64), (8, 128), (8, 64)])
def test_step_holes(page, hd, dtype):
    lens = [100, 40, 16, 700]
    holes = [(0, 0), (0, 3), (1, 1), (2, 0), (2, 1), (3, 5), (3, 43)]  # sequence 2 has none left
    pool = Q8Pool(PoolCase(lens, 2, hd, page, holes=holes))
    q = rows(4, 4, hd, dtype)
    want = ref(pool.case, q, [1] * 4, pool.case.visible)
    for max_len in (None, 700):
        out, l = run(pool, q, max_len=max_len)
        check_attention(out, l, want)
    assert (out[2] == 0).all() and (l[2] == -math.inf).all()


PROMPTS = [  # (rows, keys) per sequence
    [(1, 1)],
    [(5, 5), (1, 1), (0, 0), (33, 33), (64, 64), (65, 65)],
    [(128, 128), (0, 9), (129, 129), (31, 31)],
    [(3, 100), (40, 300), (1, 64), (17, 17), (2, 1000)],
    [(10, 4), (3, 0), (70, 66), (1, 0)],     # rows before the first key
    [(200, 263)],
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,Hkv,hd,page", [(4, 4, 64, 16), (4, 2, 128, 8), (6, 1, 64, 64),
                                           (16, 1, 128, 32)])
@pytest.mark.parametrize("which", range(len(PROMPTS)))
def test_prompts(which, H, Hkv, hd, page, dtype):
    ql, kl = [a for a, _ in PROMPTS[which]], [b for _, b in PROMPTS[which]]
    pool = Q8Pool(PoolCase(kl, Hkv, hd, page, seed=which), "interleaved")
    n = sum(ql)
    q = rows(n + 3, H, hd, dtype, seed=which)  # three rows of no sequence
    want = ref(pool.case, q[:n], ql)
    for max_len in (None, max(kl), 30000):
        out, l = run(pool, q, ql, max_len=max_len)
        check_attention(out, l, want, "max_len %s" % max_len)
        assert (out[n:] == 9).all() and (l[n:] == 9).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompt_holes(dtype):
    ql, kl = [20, 70, 5, 16], [20, 200, 64, 16]
    holes = [(0, 0), (1, 2), (1, 7), (1, 12), (2, 3), (3, 0)]
    pool = Q8Pool(PoolCase(kl, 2, 128, 16, holes=holes))
    q = rows(sum(ql), 4, 128, dtype)
    out, l = run(pool, q, ql)
    check_attention(out, l, ref(pool.case, q, ql, pool.case.visible))
    assert (out[0:16] == 0).all() and (l[0:16] == -math.inf).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_wide_tiles(hd):
    """Enough rows and heads for the 256-row tiles of bf16 queries: as the same values in bf16
    pages, of which the products are the same."""
    ql, kl = [700, 1, 800], [700, 90, 1000]
    pool = Q8Pool(PoolCase(kl, 16, hd, 16))
    q = rows(sum(ql), 128, hd, BF16)
    out, l = run(pool, q, ql)
    k, v, ke, ve, lens, table = pool.device()
    kb, vb = (torch.where((e == 255)[..., None], 0.0,
                          torch.ldexp(c.float(), e.int()[..., None] - 127)).to(BF16)
              for c, e in ((k, ke), (v, ve)))
    want, wl = torch.empty_like(out), torch.empty_like(l)
    B.aio_paged_attention(q.cuda(), kb, vb, lens, table, want, cu_q=cu(ql).cuda(), lse=wl)
    # weights of either side rounded to 2^-8 of themselves, outputs too; sum p |v| is at most
    # the largest |v|
    top = float(torch.cat(pool.case.values).float().abs().max())
    assert (out.float() - want.float()).abs().max() <= 2.0 ** -8 * 4 * top
    assert (l - wl).abs().max() <= 2.0 ** -20 * (1 + wl.abs().max())
    at = [0, 1, 699, 700, 701, 1500]
    seen = [1, 2, 700, 90, 201, 1000]
    of = [0, 0, 0, 1, 2, 2]
    check_attention(out[at], l[at], attention64(
        q[at], [pool.case.keys[i][:n] for i, n in zip(of, seen)],
        [pool.case.values[i][:n] for i, n in zip(of, seen)], [1] * 6, seen))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale_k,scale_v", [(2.0 ** 10, 2.0 ** -100), (2.0 ** -20, 2.0 ** 100),
                                             (1.0, 2.0 ** -110)])
@pytest.mark.parametrize("ql", [None, [70, 40]])
def test_magnitudes(ql, scale_k, scale_v, dtype):
    """Rows of tiny and of large values beside one another."""
    kl = [150, 90]
    case = PoolCase(kl, 2, 64, 16)
    g = torch.Generator().manual_seed(2)
    for i in range(2):
        for t, s in ((case.keys, scale_k), (case.values, scale_v)):
            t[i] = (t[i].float() * s * torch.exp2(torch.randint(-6, 7, (kl[i], 2, 1),
                                                                generator=g).float())).to(BF16)
            pages = case.k if t is case.keys else case.v
            for j in range(-(-kl[i] // 16)):
                m = min(16, kl[i] - j * 16)
                pages[int(case.table[i, j]), :, :m] = t[i][j * 16: j * 16 + m].transpose(0, 1)
    pool = Q8Pool(case)
    n = ql or [1, 1]
    q = (rows(sum(n), 4, 64, F32) / scale_k / 64).to(dtype)
    out, l = run(pool, q, ql)
    check_attention(out, l, ref(case, q, n))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("big", [2.0 ** 120, 2.0 ** 104, 2.0 ** -104])
@pytest.mark.parametrize("ql", [None, [40]])
def test_queries_at_the_ends_of_the_range(ql, big, dtype):
    """Queries next to the largest (smallest) numbers, keys that bring their scores back; one
    query among them is of ordinary size and sees scores next to 0, or the largest keys."""
    n, hd = 150, 64
    case = PoolCase([n], 1, hd, 16)
    case.keys[0] = (case.keys[0].float() / big).to(BF16)
    for j in range(-(-n // 16)):
        m = min(16, n - j * 16)
        case.k[int(case.table[0, j]), :, :m] = case.keys[0][j * 16: j * 16 + m].transpose(0, 1)
    pool = Q8Pool(case)
    nq = ql or [1]
    q = (rows(sum(nq), 4, hd, F32).clamp(-3, 3) * big).to(dtype)
    if big > 1:
        q[:, 2] = rows(sum(nq), 1, hd, F32)[:, 0].to(dtype)
    out, l = run(pool, q, ql)
    check_attention(out, l, ref(case, q, nq))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("length,ql", [(90, 1), (700, 1), (90, 60), (300, 130)])
def test_rows_that_were_not_finite(length, ql, dtype):
    """A key or value that came with an infinity or NaN is NaN for the rows that see it and for
    no others."""
    H, Hkv, hd = 4, 2, 64
    for which in "kv":
        pool = Q8Pool(PoolCase([length], Hkv, hd, 16))
        q = rows(ql, H, hd, dtype)
        want = ref(pool.case, q, [ql])
        at = length - 1 - ql // 2
        k, v, ke, ve = pool.views(pool.buffer)
        codes, exps = (k, ke) if which == "k" else (v, ve)
        pg, slot = int(pool.case.table[0, at // 16]), at % 16
        codes[pg, 1, slot], exps[pg, 1, slot] = 0, 255
        for max_len in (length, 20000):
            out, l = run(pool, q, [ql] if ql > 1 else None, max_len=max_len)
            out, l = out.cpu(), l.cpu()
            first = max(at - (length - ql), 0)  # the first row that sees it
            assert torch.isnan(out[first:, 2:]).all()
            if which == "k":
                assert torch.isnan(l[first:, 2:]).all()
                l[first:, 2:] = want[1][first:, 2:].float()
            out[first:, 2:] = want[0][first:, 2:].to(dtype)
            check_attention(out, l, want, which)


def test_long_sums():
    """Keys of one score and values of one number: 40000 equal weights."""
    n, hd = 40000, 64
    case = PoolCase([64], 1, hd, 64)
    pages = -(-n // 64)
    codes = torch.full((pages, 1, 64, hd), 93, dtype=torch.int8, device="cuda")
    exps = torch.full((pages, 1, 64), 120, dtype=torch.uint8, device="cuda")
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = rows(1, 4, hd, F32).cuda()
    out, l = torch.empty_like(q), torch.empty((1, 4), device="cuda")
    value = 93 * 2.0 ** -7
    for kw in (dict(), dict(cu_q=cu([1]).cuda())):
        for max_len in (n, None):
            B.aio_q8_attention(q, codes, codes, exps, exps, lens, table, out, lse=l,
                               max_len=max_len, **kw)
            assert float((out - value).abs().max()) <= 4e-6 * value
            s = q.double().sum(-1) * value * hd ** -0.5
            assert float((l.double() - s - math.log(n)).abs().max()) <= 2e-6 * (
                1 + float(s.abs().max()) + math.log(n))


def test_strides_and_places():
    """Queries and outputs inside wider rows; an output in its queries' place; a table wider
    than its view."""
    lens = [70, 5, 300]
    pool = Q8Pool(PoolCase(lens, 2, 128, 16), "interleaved")
    q = rows(3, 4, 128, F32)
    want = ref(pool.case, q, [1] * 3, scale=0.3)
    k, v, ke, ve, ln, table = pool.device()
    wide = torch.zeros((3, 6, 128), device="cuda")
    wide[:, 1:5] = q.cuda()
    into = torch.full((3, 9, 128), 7.0, device="cuda")
    tab = torch.full((3, table.shape[1] + 3), -9, dtype=torch.int32, device="cuda")
    tab[:, : table.shape[1]] = table
    B.aio_q8_attention(wide[:, 1:5], k, v, ke, ve, ln, tab[:, : table.shape[1]], into[:, 2:6],
                       scale=0.3)
    check_attention(into[:, 2:6], None, want)
    assert (into[:, :2] == 7).all() and (into[:, 6:] == 7).all()
    B.aio_q8_attention(wide[:, 1:5], k, v, ke, ve, ln, table, wide[:, 1:5], scale=0.3)
    check_attention(wide[:, 1:5], None, want)


def test_lengths_are_bounded():
    pool = Q8Pool(PoolCase([64, 64, 64, 64], 2, 64, 16, width_more=0))
    case = pool.case
    case.lens = torch.tensor([1 << 30, -5, 64, 65], dtype=torch.int32)
    q = rows(4, 4, 64, F32)
    for max_len, n in ((None, 64), (50, 50)):
        want = attention64(q, [k[:n] for k in case.keys], [v[:n] for v in case.values], [1] * 4,
                           [n, 0, n, n])
        out, l = run(pool, q, max_len=max_len)
        check_attention(out, l, want)


def test_captured_and_replayed():
    """A captured step and prompts follow lengths in device memory, replay by replay, with
    eager work between the replays; two graphs share a workspace."""
    lens = [600, 1700]
    pool = Q8Pool(PoolCase(lens, 2, 64, 16))
    k, v, ke, ve, ln, table = pool.device()
    need = B.aio_q8_workspace_bytes(2, 2, 1700, 4, 2, 64)
    assert need > 0
    ws = torch.full((max(need, B.aio_q8_workspace_bytes(2, 34, 1700, 4, 2, 64, prompts=True)),),
                    255, dtype=torch.uint8, device="cuda")
    q, ql = rows(2, 4, 64, F32).cuda(), [9, 25]
    pq = rows(sum(ql), 4, 64, BF16).cuda()
    out, pout, c = torch.empty_like(q), torch.empty_like(pq), cu(ql).cuda()
    calls = [lambda: B.aio_q8_attention(q, k, v, ke, ve, ln, table, out, max_len=1700, ws=ws),
             lambda: B.aio_q8_attention(pq, k, v, ke, ve, ln, table, pout, cu_q=c, max_len=1700,
                                        ws=ws)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        for f in calls:
            f()
    torch.cuda.current_stream().wait_stream(st)
    graphs = []
    for f in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    case = pool.case
    for a, b in ((600, 1700), (599, 30), (64, 33), (0, 25), (600, 1700)):
        ln.copy_(torch.tensor([a, b], dtype=torch.int32))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [out.clone(), pout.clone()]
        kk, vv = [case.keys[0][:a], case.keys[1][:b]], [case.values[0][:a], case.values[1][:b]]
        check_attention(got[0], None, attention64(q.cpu(), kk, vv, [1, 1], [a, b]))
        check_attention(got[1], None, attention64(pq.cpu(), kk, vv, ql, [a, b]))
        ws.fill_(255)
        for f in calls:
            f()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], pout)


def test_codes_of_a_row_stand_for_bf16():
    """What the quantisation writes reads back within half a step of the row."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn((50, 3, 64), generator=g)
    c, e = quantise64(x)
    back = torch.ldexp(c.double(), e.int()[..., None] - 127)
    assert ((back - x.double()).abs() <= x.double().abs().amax(-1, keepdim=True) / 127).all()
