"""Rows appended to pages of 8-bit codes, code for code."""
import numpy as np
import pytest
import torch

from paper_2604_09752_amd import binding as B
from tests.paged_cases import PoolCase, cu
from tests.q8_cases import Q8Pool, quantise64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def expect(pool, kr, vr, ql, lens, max_len=1 << 30):
    """The buffer after the append, on the CPU."""
    buf, case = pool.buffer.clone(), pool.case
    k, v, ke, ve = pool.views(buf)
    rows = [quantise64(x) for x in (kr, vr)]
    r = 0
    for i, (q, n) in enumerate(zip(ql, lens)):
        for j in range(q):
            pos = n - q + j
            if 0 <= pos < min(max_len, case.table.shape[1] * case.page):
                pg, slot = int(case.table[i, pos // case.page]), pos % case.page
                if 0 <= pg < case.n_pages:
                    for (c, e), (codes, exps) in zip(((k, ke), (v, ve)), rows):
                        c[pg, :, slot] = codes[r + j]
                        e[pg, :, slot] = exps[r + j]
        r += q
    return buf


def spread(shape, g):
    """Rows of many magnitudes, within one row too."""
    x = torch.randn(shape, generator=g)
    return x * torch.exp2(torch.randint(-30, 30, (*shape[:2], 1), generator=g).float())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hkv,hd,page,layout", [
    (8, 128, 16, "plain"), (1, 64, 8, "plain"), (3, 64, 64, "interleaved"),
    (5, 128, 8, "interleaved"), (32, 128, 256, "interleaved"), (33, 64, 32, "plain")])
def test_append(Hkv, hd, page, layout, dtype):
    ql, kl = [1, 0, 7, 20, 3], [1, 30, 40, 20, 257]
    pool = Q8Pool(PoolCase(kl, Hkv, hd, page, holes=[(2, 1)]), layout)
    g = torch.Generator().manual_seed(3)
    n = sum(ql) + 2  # two rows of no sequence
    kr, vr = spread((n, Hkv, hd), g).to(dtype), spread((n, Hkv, hd), g).to(dtype)
    k, v, ke, ve, lens, table = pool.device()
    B.aio_q8_append(kr.cuda(), vr.cuda(), k, v, ke, ve, lens, table, cu_q=cu(ql).cuda())
    torch.cuda.synchronize()
    assert torch.equal(pool.on.cpu(), expect(pool, kr, vr, ql, kl))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_one_row_each_and_strides(dtype):
    """One new token of each sequence (no boundaries), rows laid out head by head and inside
    wider rows."""
    kl = [1, 0, 16, 17, 500]
    g = torch.Generator().manual_seed(4)
    kr, vr = torch.randn((2, 4, 5, 64), generator=g).to(dtype).unbind(0)  # [heads][rows][dim]
    pool = Q8Pool(PoolCase(kl, 4, 64, 16))
    k, v, ke, ve, lens, table = pool.device()
    B.aio_q8_append(kr.cuda().transpose(0, 1), vr.cuda().transpose(0, 1), k, v, ke, ve, lens, table)
    want = expect(pool, kr.transpose(0, 1).contiguous(), vr.transpose(0, 1).contiguous(), [1] * 5, kl)
    assert torch.equal(pool.on.cpu(), want)
    qkv = torch.zeros((5, 12, 64), dtype=dtype, device="cuda")  # queries, keys, values of a row
    qkv[:, 4:8], qkv[:, 8:] = kr.transpose(0, 1).cuda(), vr.transpose(0, 1).cuda()
    k, v, ke, ve, lens, table = pool.device()
    B.aio_q8_append(qkv[:, 4:8], qkv[:, 8:], k, v, ke, ve, lens, table)
    assert torch.equal(pool.on.cpu(), want)


def bits(*v):
    return torch.tensor(v, dtype=torch.int64).to(torch.int32).view(F32)


@pytest.mark.parametrize("hd", [64, 128])
def test_append_values(hd):
    """Ties, the largest and the smallest numbers, zeros, infinities and NaN, one kind per row."""
    inf, nan, top = float("inf"), float("nan"), float(torch.finfo(F32).max)
    rows = [
        [127.5, 0.5, -0.5, 1.5, -126.5],             # 127.5 would round to the even 128
        [127.49999237060547, 63.5, -63.5],           # the float below: the code 127
        [-127.5, 2.5], [255.0, -254.99998], [1.0, -1.0], [0.9921875], [0.99218744],
        [0.0], [-0.0], [top, -top / 127], [-top], [2.0 ** 127 * 1.9921875], [3e38, 1e-38],
        [1e-45], [1e-38, -1e-39], [2.0 ** -112], [127 * 2.0 ** -119], [128 * 2.0 ** -119],
        [2.0 ** -120, 2.0 ** -119], [1.5 * 2.0 ** -120], [2.0 ** -121],
        [inf], [-inf, 1.0], [nan], [nan, inf], [1e30, nan, -1e30],
    ]
    x = torch.zeros((len(rows), 2, hd))
    for i, r in enumerate(rows):
        x[i, 0, 3: 3 + len(r)] = torch.tensor(r)
        x[i, 1, hd - len(r):] = torch.tensor(r)
        x[i, 1, : hd // 2] = torch.linspace(-0.9, 0.9, hd // 2) * r[0] if np.isfinite(r[0]) else 0.25
    n = len(rows)
    pool = Q8Pool(PoolCase([n], 2, hd, 16))
    k, v, ke, ve, lens, table = pool.device()
    B.aio_q8_append(x.cuda(), -x.flip(0).cuda(), k, v, ke, ve, lens, table, cu_q=cu([n]).cuda())
    assert torch.equal(pool.on.cpu(), expect(pool, x, -x.flip(0), [n], [n]))


def test_append_stays_inside():
    """Rows before key 0, past the table, past max_len, of bad boundaries."""
    ql, kl = [12, 4, 5], [7, 64, 20]
    g = torch.Generator().manual_seed(5)
    kr, vr = torch.randn((2, 21, 2, 64), generator=g).unbind(0)
    pool = Q8Pool(PoolCase([7, 40, 20], 2, 64, 16, width_more=0))
    for lens in (kl, [7, 50, 1 << 30], [-3, 42, 20]):
        for max_len in (None, 18):
            k, v, ke, ve, _, table = pool.device()
            B.aio_q8_append(kr.cuda(), vr.cuda(), k, v, ke, ve,
                            torch.tensor(lens, dtype=torch.int32, device="cuda"), table,
                            cu_q=cu(ql).cuda(), max_len=max_len)
            want = expect(pool, kr, vr, ql, lens, max_len or 1 << 30)
            assert torch.equal(pool.on.cpu(), want)
    for bad in ([5, 0, 1 << 30, -9], [-1 << 31, 3, 2, 21], [21, 21, 21, 21]):
        k, v, ke, ve, lens, table = pool.device()
        B.aio_q8_append(kr.cuda(), vr.cuda(), k, v, ke, ve, lens, table,
                        cu_q=torch.tensor(bad, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append_many_rows(dtype):
    """Prompts of several hundred rows that begin and end within pages, more sequences than a
    wave counts at once."""
    ql = [333, 1, 0, 250] + [1 + i % 3 for i in range(90)]
    kl = [333 + 5, 70, 9, 250] + [40 + i for i in range(90)]
    g = torch.Generator().manual_seed(6)
    n = sum(ql)
    kr, vr = spread((n, 2, 128), g).to(dtype), spread((n, 2, 128), g).to(dtype)
    pool = Q8Pool(PoolCase(kl, 2, 128, 16), "interleaved")
    k, v, ke, ve, lens, table = pool.device()
    B.aio_q8_append(kr.cuda(), vr.cuda(), k, v, ke, ve, lens, table, cu_q=cu(ql).cuda())
    assert torch.equal(pool.on.cpu(), expect(pool, kr, vr, ql, kl))


def test_append_past_32_bits():
    """Offsets in codes past 2^32: the last pages of a large pool."""
    page, Hkv, hd = 256, 8, 128
    n_pages = (1 << 32) // (Hkv * page * hd) + 3
    k = torch.zeros((n_pages, Hkv, page, hd), dtype=torch.int8, device="cuda")
    v = torch.zeros_like(k)
    ke = torch.zeros((n_pages, Hkv, page), dtype=torch.uint8, device="cuda")
    ve = torch.zeros_like(ke)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([200], dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(8)
    kr, vr = torch.randn((2, 200, Hkv, hd), generator=g).unbind(0)
    B.aio_q8_append(kr.cuda(), vr.cuda(), k, v, ke, ve, lens, table, cu_q=cu([200]).cuda())
    for codes, exps, rows in ((k, ke, kr), (v, ve, vr)):
        c, e = quantise64(rows)
        assert torch.equal(codes[-1, :, :200].cpu().transpose(0, 1), c)
        assert torch.equal(exps[-1, :, :200].cpu().transpose(0, 1), e)
        assert not codes[:-1].any() and not codes[-1, :, 200:].any()
    # read back
    from tests.paged_cases import attention64, check_attention
    from tests.q8_cases import values
    q = torch.randn((3, 16, hd), generator=g)
    keys, vals = values(*quantise64(kr)), values(*quantise64(vr))
    out = torch.empty_like(q).cuda()
    B.aio_q8_attention(q.cuda(), k, v, ke, ve, lens, table, out, cu_q=cu([3]).cuda())
    check_attention(out, None, attention64(q, [keys], [vals], [3], [200]))
    B.aio_q8_attention(q[:1].cuda(), k, v, ke, ve, lens, table, out[:1])
    check_attention(out[:1], None, attention64(q[:1], [keys], [vals], [1], [200]))


def test_forked_pages_are_copied():
    """Codes and bytes of a page laid out together are planes of one copy."""
    pool = Q8Pool(PoolCase([40, 9], 3, 64, 16), "interleaved")
    k, v, ke, ve, lens, table = pool.device()
    planes = pool.on.view(1, pool.on.shape[0], -1)
    a, b = int(pool.case.table[0, 2]), int(pool.case.table[1, 0])
    B.aio_page_copy(planes, [a], [b])
    torch.cuda.synchronize()
    assert torch.equal(pool.on[b], pool.on[a])
    assert torch.equal(k[b], k[a]) and torch.equal(ve[b], ve[a])


def test_a_side_stream_and_a_graph():
    kl = [33, 5]
    pool = Q8Pool(PoolCase(kl, 2, 64, 16))
    g = torch.Generator().manual_seed(9)
    sets = [torch.randn((2, 2, 2, 64), generator=g) for _ in range(3)]
    k, v, ke, ve, lens, table = pool.device()
    rows = sets[0].cuda()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        B.aio_q8_append(rows[0], rows[1], k, v, ke, ve, lens, table)
    torch.cuda.current_stream().wait_stream(st)
    torch.cuda.synchronize()
    want = expect(pool, sets[0][0], sets[0][1], [1, 1], kl)
    assert torch.equal(pool.on.cpu(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.aio_q8_append(rows[0], rows[1], k, v, ke, ve, lens, table)
    for s, at in zip(sets[1:], ([32, 4], [17, 1])):
        rows.copy_(s)
        lens.copy_(torch.tensor(at, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        pool.buffer = want
        want = expect(pool, s[0], s[1], [1, 1], at)
        assert torch.equal(pool.on.cpu(), want)
