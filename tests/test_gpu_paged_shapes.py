"""Shapes, pages and streams of the operators over several sequences that lie past one
launch, one tile or one layout (needs an MI355X)."""
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import PoolCase, attention64, check_attention, close, cu, logprobs64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rows(n, H, hd, dtype, seed=1):
    return torch.randn((n, H, hd), generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("layout", ["plain", "interleaved"])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
def test_prompts_in_pages_of_any_size(page, layout, hd, dtype):
    """Several pages in a key tile and several tiles in a page; holes, and queries and
    outputs inside wider rows."""
    ql, kl = [70, 5, 130, 1], [200, 5, 400, 257]
    n = sum(ql)
    for holes in ((), ((0, 1), (2, 0), (3, 0))):
        holes = [(i, j) for i, j in holes if j < -(-kl[i] // page)]
        case = PoolCase(kl, 2, hd, page, seed=page, holes=holes, layout=layout)
        q = rows(n, 6, hd, dtype)
        ref = attention64(q, case.keys, case.values, ql, kl, case.visible)
        k, v, lens, table = case.device()
        wide = torch.zeros((n, 9, hd), dtype=dtype, device="cuda")
        wide[:, 2:8] = q.cuda()
        into = torch.full((n, 11, hd), 7.0, dtype=dtype, device="cuda")
        lse = torch.empty((n, 6), device="cuda")
        for max_len in (400, 20000):
            B.aio_paged_attention(wide[:, 2:8], k, v, lens, table, into[:, 3:9], lse=lse,
                                  cu_q=cu(ql).cuda(), max_len=max_len)
            check_attention(into[:, 3:9], lse, ref, (page, layout, holes, max_len))
        assert (into[:, :3] == 7).all() and (into[:, 9:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_more_logit_rows_than_one_launch(dtype):
    n, rows_, top = 37, 131072 + 5, 3
    g = torch.Generator().manual_seed(2)
    x = torch.randn((rows_, n + 4), generator=g).to(dtype)[:, :n]
    t = torch.randint(-1, n, (rows_,), generator=g, dtype=torch.int32)
    lp, ent = (torch.full((rows_,), 9.0, device="cuda") for _ in range(2))
    ids = torch.full((rows_, top), -9, dtype=torch.int32, device="cuda")
    tlp = torch.full((rows_, top), 9.0, device="cuda")
    d = torch.zeros((rows_, n + 4), dtype=dtype, device="cuda")[:, :n]
    d.copy_(x)
    B.aio_logprobs(d, t.cuda(), lp, ent, ids, tlp)
    torch.cuda.synchronize()
    # around the borders of the launches, and every 997th row
    at = sorted(set(range(0, rows_, 997)) | {r for b in (0, 65535, 131070, rows_)
                                             for r in range(b - 3, b + 4) if 0 <= r < rows_})
    wlp, went, wids, wtlp, ltol, etol = logprobs64(x[at], t[at], top)
    close(lp[at], wlp, ltol + 2.0 ** -24 * wlp.abs())
    close(ent[at], went, etol + 2.0 ** -24 * went.abs())
    assert torch.equal(ids[at].cpu().long(), wids)
    close(tlp[at], wtlp, ltol[:, None] + 2.0 ** -24 * wtlp.abs())
    assert (ids >= 0).all() and not (ent == 9).any()


def test_more_planes_than_one_launch():
    pool = torch.randn((131070 + 3, 3, 8), device="cuda").to(BF16)
    want = pool.clone()
    want[:, 2] = pool[:, 0]
    B.aio_page_copy(pool, [0], [2])
    assert torch.equal(pool.view(torch.int16), want.view(torch.int16))


def test_more_sequences_than_a_grid_row():
    """70000 sequences of one or two keys, one new token each."""
    n, page, hd = 70000, 8, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((n, 1, page, hd), generator=g, device="cuda").to(BF16) for _ in range(2))
    table = torch.randperm(n, generator=g, device="cuda").int()[:, None]
    lens = torch.randint(0, 3, (n,), generator=g, device="cuda").int()
    q = torch.randn((n, 2, hd), generator=g, device="cuda")
    out, lse = torch.full_like(q, 9.0), torch.full((n, 2), 9.0, device="cuda")
    B.aio_paged_attention(q, k, v, lens, table, out, lse=lse)
    kk, vv = (t[table[:, 0].long(), 0, :2].double() for t in (k, v))
    s = (q.double()[:, :, None] * kk[:, None]).sum(-1) * hd ** -0.5          # [n, 2 heads, 2 keys]
    s = s.masked_fill(torch.arange(2, device="cuda") >= lens[:, None, None], -float("inf"))
    p = torch.softmax(s, -1).nan_to_num(nan=0.0)
    want = (p[..., None] * vv[:, None]).sum(2)
    # (a score of 64 products is off by some 8 sqrt(192) 2^-24 of sum |q k| / 8, below 20 here)
    assert (out.double() - want).abs().max() <= 2 * 1.4e-4 * float(vv.abs().max())
    assert torch.equal(out == 0, (lens == 0)[:, None, None].expand_as(out))
    assert torch.equal(torch.isneginf(lse), (lens == 0)[:, None].expand_as(lse))
    # the rows into pages, one each
    new = torch.randn((n, 1, hd), generator=g, device="cuda")
    before = k.clone()
    B.aio_page_append(new, new, k, v, lens, table)
    has = lens > 0
    before[table[has, 0].long(), 0, (lens[has] - 1).long()] = new[has, 0].to(BF16)
    assert torch.equal(k.view(torch.int16), before.view(torch.int16))


def test_a_step_on_a_side_stream():
    """Append, attention and scores behind one another on a stream of their own, while
    the default stream is busy."""
    lens = [40, 3000, 7]
    case = PoolCase(lens, 2, 64, 16, spare=0)
    k, v, ld, table = case.device()
    new_k, new_v = rows(3, 2, 64, F32, 3), rows(3, 2, 64, F32, 4)
    q, w = rows(3, 8, 64, F32, 5), rows(1, 500, 512, F32, 6)[0].t().contiguous()
    a = torch.zeros((8192, 8192), dtype=BF16, device="cuda")
    args = [t.cuda() for t in (new_k, new_v, q, w)]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        a @ a
    with torch.cuda.stream(st):
        kr, vr, qd, wd = args
        B.aio_page_append(kr, vr, k, v, ld, table)
        out = torch.empty_like(qd)
        B.aio_paged_attention(qd, k, v, ld, table, out, max_len=3000)
        logits = out.reshape(3, 512) @ wd
        ids, tlp = torch.empty((3, 4), dtype=torch.int32, device="cuda"), torch.empty((3, 4),
                                                                                      device="cuda")
        B.aio_logprobs(logits, None, None, None, ids, tlp)
    st.synchronize()
    for i, n in enumerate(lens):
        case.keys[i][n - 1], case.values[i][n - 1] = new_k[i].to(BF16), new_v[i].to(BF16)
    check_attention(out, None, attention64(q, case.keys, case.values, [1] * 3, lens))
    want = logprobs64(logits.cpu(), None, 4)
    assert torch.equal(ids.cpu().long(), want[2])
    close(tlp, want[3], want[4][:, None] + 2.0 ** -24 * want[3].abs())
    torch.cuda.synchronize()
