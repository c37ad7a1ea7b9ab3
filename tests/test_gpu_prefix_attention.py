"""Attention of groups of sequences that share a prefix against a plain 64-bit evaluation of
each sequence by itself."""
import math

import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import attention64, check_attention, cu
from tests.q8_cases import Q8Pool, group_case

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rows(n, H, hd, dtype, seed=1):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, H, hd), generator=g).to(dtype)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Grouped:
    """A pool of either kind and its groups (first, last, prefix), in order."""

    def __init__(self, k_len, groups, Hkv, hd, page=16, q8=False, seed=0, **kw):
        self.case = group_case(k_len, groups, Hkv, hd, page, seed=seed, **kw)
        self.q8 = q8
        if q8:
            *self.kv, self.lens, self.table = Q8Pool(self.case).device()
        else:
            *self.kv, self.lens, self.table = self.case.device()
        # a group ends where the next begins: sequences between two are a group that shares nothing
        cu_seqs, lens = [], []
        for first, last, prefix in groups:
            if cu_seqs and cu_seqs[-1] != first:
                lens.append(0)
                cu_seqs.append(first)
            elif not cu_seqs:
                cu_seqs.append(first)
            lens.append(prefix)
            cu_seqs.append(last)
        self.cu_seqs, self.prefix = i32(cu_seqs or [0]), i32(lens)

    def call(self, q, out, **kw):
        f = B.aio_q8_prefix_attention if self.q8 else B.aio_prefix_attention
        f(q, *self.kv, self.lens, self.table, self.cu_seqs, self.prefix, out, **kw)

    def run(self, q, ql=None, fill=9.0, **kw):
        qd = q.cuda()
        out = torch.full_like(qd, fill)
        l = torch.full(q.shape[:2], fill, device="cuda")
        if ql is not None:
            kw["cu_q"] = cu(ql).cuda()
        self.call(qd, out, lse=l, **kw)
        torch.cuda.synchronize()
        return out, l

    def ref(self, q, ql=None, **kw):
        c = self.case
        return attention64(q, c.keys, c.values, ql or [1] * len(c.k_len), c.k_len, c.visible, **kw)


# keys of each sequence, groups
STEPS = {
    "forks": ([700, 740, 701], [(0, 3, 700)]),
    "odd": ([130, 200, 77, 300, 65, 900], [(0, 2, 129), (2, 3, 70), (3, 6, 65)]),
    "exact": ([64, 128, 128, 64, 65], [(0, 1, 64), (1, 3, 128), (3, 5, 64)]),
    "short": ([40, 41, 63, 100], [(0, 4, 40)]),                 # nothing whole to share
    "idle": ([300, 0, 310, 0, 299, 5], [(0, 6, 298)]),          # idle places, a short one
    "first idle": ([0, 300, 310], [(0, 3, 298)]),
    "outside": ([90, 400, 410, 33, 500, 505, 20], [(1, 3, 390), (4, 6, 500)]),
    "empty": ([200, 210, 220], [(0, 0, 64), (0, 2, 190), (2, 2, 500), (2, 3, 100)]),
    "many": ([500 + 7 * (i % 11) for i in range(70)], [(0, 69, 490), (69, 70, 64)]),
    "groups": ([150 + i for i in range(140)], [(2 * i, 2 * i + 2, 140 + i) for i in range(70)]),
    "none": ([30, 600], []),
    # (48 columns per group and more with 4 or 8 heads of queries per kv head)
    "wide": ([700 + 3 * i for i in range(40)] + [0, 690, 20], [(0, 43, 688)]),
    "wide groups": ([300 + i % 9 for i in range(26)], [(0, 13, 299), (13, 26, 270)]),
}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("H,Hkv,hd", [(4, 4, 64), (8, 2, 128), (6, 2, 64), (16, 1, 128), (8, 2, 64)])
@pytest.mark.parametrize("name", list(STEPS))
def test_step(name, H, Hkv, hd, q8, dtype):
    k_len, groups = STEPS[name]
    p = Grouped(k_len, groups, Hkv, hd, q8=q8)
    q = rows(len(k_len), H, hd, dtype)
    want = p.ref(q)
    for kw in (dict(), dict(max_len=max(k_len), max_prefix=max([g[2] for g in groups] + [0])),
               dict(max_len=30000, max_prefix=20000), dict(max_prefix=100)):
        out, l = p.run(q, **kw)
        check_attention(out, l, want, "%s %s" % (name, kw))


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_wide_values_that_are_not_finite(hd, q8):
    """In the prefix they reach every row of the group, in a sequence's own keys that one."""
    k_len = [400 + i for i in range(14)]
    p = Grouped(k_len, [(0, 14, 384)], 1, hd, q8=q8)
    q = rows(14, 4, hd, BF16)
    want = p.ref(q)
    page = int(p.case.table[3, 25])  # own keys of sequence 3 (24 full pages are shared)
    for at, who in (((int(p.case.table[0, 7]), 5), range(14)), ((page, 2), [3])):
        kv = [t.clone() for t in p.kv]
        if q8:
            p.kv[1][at[0], 0, at[1]] = 0
            p.kv[3][at[0], 0, at[1]] = 255
        else:
            p.kv[1][at[0], 0, at[1]] = float("nan")
        out, l = p.run(q, max_len=420, max_prefix=384)
        out = out.cpu()
        assert torch.isnan(out[list(who)]).all()
        out[list(who)] = want[0][list(who)].to(BF16)
        check_attention(out, l.cpu(), want)
        for t, old in zip(p.kv, kv):
            t.copy_(old)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("page", [8, 32, 256])
def test_pages(page, q8, dtype):
    """Prefixes that end within pages, in pages that are shared and in copies."""
    k_len, groups = [333, 340, 400, 270, 269], [(0, 3, 321), (3, 5, 269)]
    for copied in (False, True):
        p = Grouped(k_len, groups, 2, 64, page=page, q8=q8, copied=copied)
        q = rows(5, 8, 64, dtype)
        out, l = p.run(q)
        check_attention(out, l, p.ref(q))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q8", [False, True])
def test_long_prefixes(q8, dtype):
    k_len = [5003, 5100, 4990, 9000, 8801]
    p = Grouped(k_len, [(0, 3, 4985), (3, 5, 8800)], 2, 128, page=64, q8=q8)
    q = rows(5, 8, 128, dtype)
    out, l = p.run(q, max_len=9000, max_prefix=8800)
    check_attention(out, l, p.ref(q))


# rows and keys of each sequence, groups
PROMPTS = {
    "turns": ([(40, 540), (1, 501), (17, 600), (90, 590)], [(0, 4, 500)]),
    "idle": ([(0, 0), (5, 300), (0, 290), (3, 293)], [(0, 4, 290)]),
    "first has none": ([(0, 300), (5, 300), (7, 299)], [(0, 3, 292)]),
    # new rows that begin within the prefix, at its end and behind it
    "within": ([(100, 150), (22, 150), (150, 150), (21, 149), (1, 128)], [(0, 5, 128)]),
    "outside": ([(3, 90), (40, 400), (41, 420), (200, 200), (9, 309), (5, 304)],
                [(1, 3, 360), (4, 6, 299)]),
    "many rows": ([(300, 800), (70, 570), (1, 501), (129, 640)], [(0, 4, 500)]),
    "many": ([(1 + i % 5, 200 + i) for i in range(70)], [(0, 35, 190), (35, 70, 230)]),
    "one each": ([(1, 100), (1, 101), (1, 64)], [(0, 3, 64)]),
}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("H,Hkv,hd", [(4, 4, 64), (4, 2, 128), (6, 2, 64)])
@pytest.mark.parametrize("name", list(PROMPTS))
def test_prompts(name, H, Hkv, hd, q8, dtype):
    shape, groups = PROMPTS[name]
    ql, k_len = [a for a, _ in shape], [b for _, b in shape]
    p = Grouped(k_len, groups, Hkv, hd, q8=q8)
    n = sum(ql)
    q = rows(n + 2, H, hd, dtype)  # two rows of no sequence
    want = p.ref(q[:n], ql)
    for kw in (dict(), dict(max_len=max(k_len), max_prefix=max(g[2] for g in groups)),
               dict(max_len=20000, max_prefix=20000), dict(max_prefix=64)):
        out, l = p.run(q, ql, **kw)
        check_attention(out, l, want, "%s %s" % (name, kw))
        assert (out[n:] == 9).all() and (l[n:] == 9).all()


@pytest.mark.parametrize("q8", [False, True])
def test_wide_tiles(q8):
    """Enough rows and heads for 256-row tiles of bf16 queries: as without groups."""
    ql, k_len = [900, 700, 560], [1400, 1201, 1119]
    p = Grouped(k_len, [(0, 3, 490)], 16, 64, q8=q8)
    q = rows(sum(ql), 128, 64, BF16)
    out, l = p.run(q, ql, max_len=1400, max_prefix=490)
    plain, pl = torch.empty_like(out), torch.empty_like(l)
    f = B.aio_q8_attention if q8 else B.aio_paged_attention
    f(q.cuda(), *p.kv, p.lens, p.table, plain, cu_q=cu(ql).cuda(), lse=pl)
    # weights of either side rounded to 2^-8 of themselves, outputs too; sum p |v| is at most
    # the largest |v|
    top = float(torch.cat(p.case.values).float().abs().max())
    assert (out.float() - plain.float()).abs().max() <= 2.0 ** -8 * 4 * top
    assert (l - pl).abs().max() <= 2.0 ** -20 * (1 + pl.abs().max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("ql", [None, [3, 40, 9]])
def test_holes(ql, q8, dtype):
    """Evicted pages in the prefix and behind it."""
    k_len = [400, 420, 390]
    holes = [(0, 1), (0, 7), (1, 24), (2, 24)]  # (the last two behind it)
    p = Grouped(k_len, [(0, 3, 380)], 2, 64, q8=q8, holes=holes)
    q = rows(sum(ql) if ql else 3, 4, 64, dtype)
    out, l = p.run(q, ql)
    check_attention(out, l, p.ref(q, ql))


def test_a_prefix_of_nothing_but_holes():
    k_len = [128, 130]
    p = Grouped(k_len, [(0, 2, 128)], 2, 64, holes=[(0, j) for j in range(8)])
    q = rows(2, 4, 64, F32)
    out, l = p.run(q)
    check_attention(out, l, p.ref(q))
    assert (out[0] == 0).all() and (l[0] == -math.inf).all()


@pytest.mark.parametrize("q8", [False, True])
def test_same_results_whatever_the_workspace_holds(q8):
    k_len, groups = STEPS["idle"]
    p = Grouped(k_len, groups, 2, 64, q8=q8)
    q = rows(len(k_len), 8, 64, F32)
    need = B.aio_prefix_workspace_bytes(6, 6, 310, 1, 298, 8, 2, 64)
    outs = []
    for fill in (0, 255, 127):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        outs.append(p.run(q, max_len=310, max_prefix=298, ws=ws))
    for out, l in outs:
        assert torch.equal(out, outs[0][0]) and torch.equal(l, outs[0][1])
    check_attention(*outs[0], p.ref(q))
    with pytest.raises(ValueError):
        p.run(q, max_len=310, max_prefix=298, ws=ws[:-16])


@pytest.mark.parametrize("ql", [None, [4, 9, 1, 30]])
def test_groups_that_make_no_sense(ql):
    """Boundaries and lengths of any value stay inside the buffers (what comes out means nothing
    then), and a right call afterwards is right."""
    k_len = [300, 310, 290, 340]
    p = Grouped(k_len, [(0, 4, 280)], 2, 64)
    q = rows(sum(ql) if ql else 4, 4, 64, F32)
    want = p.ref(q, ql)
    right = p.cu_seqs, p.prefix
    big = (1 << 31) - 1
    for c, n in (([0, 1 << 30], [280]), ([-5, 4], [1 << 30]), ([3, 0], [280]), ([4, 4], [100]),
                 ([0, 4], [-1]), ([0, 4], [big]), ([0, 3, 1, 4], [280, 64, 200]),
                 ([2, 2, 2, 2], [64, 64, 64]), ([-1 << 31, big], [big]),
                 ([4, 3, 2, 1, 0], [64, 128, 192, 256])):
        p.cu_seqs, p.prefix = i32(c), i32(n)
        out, l = p.run(q, ql)
        assert out.shape == q.shape
        if c[0] == 0 and n == [-1]:
            check_attention(out, l, want)
    p.cu_seqs, p.prefix = right
    out, l = p.run(q, ql)
    check_attention(out, l, want)


def test_strides_and_places():
    k_len = [300, 310, 290]
    p = Grouped(k_len, [(0, 3, 280)], 2, 64, q8=True)
    q = rows(3, 4, 64, BF16)
    want = p.ref(q, scale=0.2)
    wide = torch.zeros((3, 6, 64), dtype=BF16, device="cuda")
    wide[:, 1:5] = q.cuda()
    into = torch.full((3, 9, 64), 7.0, dtype=BF16, device="cuda")
    p.call(wide[:, 1:5], into[:, 2:6], scale=0.2)
    check_attention(into[:, 2:6], None, want)
    assert (into[:, :2] == 7).all() and (into[:, 6:] == 7).all()
    p.call(wide[:, 1:5], wide[:, 1:5], scale=0.2)
    check_attention(wide[:, 1:5], None, want)


@pytest.mark.parametrize("q8", [False, True])
def test_captured_and_replayed(q8):
    """Lengths, prefixes and groups in device memory change from replay to replay; two graphs
    share a workspace."""
    k_len = [500, 520, 490, 600]
    p = Grouped(k_len, [(0, 4, 480)], 2, 64, q8=q8)
    ql = [3, 1, 30, 7]
    q, pq = rows(4, 4, 64, F32).cuda(), rows(sum(ql), 4, 64, BF16).cuda()
    out, pout, c = torch.empty_like(q), torch.empty_like(pq), cu(ql).cuda()
    kw = dict(max_len=600, max_prefix=480)
    ws = torch.full((max(B.aio_prefix_workspace_bytes(4, 4, 600, 1, 480, 4, 2, 64),
                         B.aio_prefix_workspace_bytes(4, 41, 600, 1, 480, 4, 2, 64, prompts=True)),),
                    255, dtype=torch.uint8, device="cuda")
    calls = [lambda: p.call(q, out, ws=ws, **kw), lambda: p.call(pq, pout, cu_q=c, ws=ws, **kw)]
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
    case = p.case
    for lens, prefix, cut in ((k_len, 480, 4), ([490, 481, 485, 482], 470, 4), (k_len, 100, 3),
                              ([500, 0, 490, 31], 480, 4), (k_len, 0, 4), (k_len, 480, 4)):
        p.lens.copy_(i32(lens))
        p.prefix.copy_(i32([prefix]))
        p.cu_seqs.copy_(i32([0, cut]))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [out.clone(), pout.clone()]
        kk = [k[:n] for k, n in zip(case.keys, lens)]
        vv = [v[:n] for v, n in zip(case.values, lens)]
        check_attention(got[0], None, attention64(q.cpu(), kk, vv, [1] * 4, lens))
        check_attention(got[1], None, attention64(pq.cpu(), kk, vv, ql, lens))
        ws.fill_(255)
        for f in calls:
            f()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], pout)


def test_two_streams():
    k_len = [500, 520, 490]
    p = Grouped(k_len, [(0, 3, 480)], 2, 128)
    torch.cuda.synchronize()
    qs = [rows(3, 8, 128, F32, seed=s) for s in (5, 6)]
    outs, keep = [], []
    for q in qs:
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            qd = q.cuda()
            out = torch.empty_like(qd)
            p.call(qd, out)
            outs.append(out)
            keep.append((qd, st))
    torch.cuda.synchronize()
    for q, out in zip(qs, outs):
        check_attention(out, None, p.ref(q))
