"""The operators over several sequences on the host: what they refuse, their
workspaces, and the page tables against a plain model of them."""
import ctypes
import random

import pytest

from paper_2604_09752_amd import binding as B

P16 = 16  # any aligned non-null pointer: nothing is enqueued by a refused call


@pytest.fixture(scope="module")
def L():
    return B.lib()


def paged(**kw):
    kv = B.aio_paged_kv(P16, P16, 8 * 16 * 64, 16 * 64, 10, 16, 8, 64)
    for f, v in kw.items():
        setattr(kv, f, v)
    return kv


def seqs(**kw):
    s = B.aio_seqs(4, 4, 100, None, P16, P16, 8, None)
    for f, v in kw.items():
        setattr(s, f, v)
    return s


def attn(**kw):
    a = B.aio_attn(P16, P16, None, 16 * 64, 16 * 64, B.AIO_F32, 16, 0.125)
    for f, v in kw.items():
        setattr(a, f, v)
    return a


R = ctypes.byref


@pytest.mark.parametrize("field,value,code", [
    ("k_dev", None, B.AIO_EINVAL), ("v_dev", 8, B.AIO_EINVAL), ("n_pages", 0, B.AIO_EINVAL),
    ("n_kv_heads", 0, B.AIO_EINVAL), ("page_stride", -8, B.AIO_EINVAL),
    ("page_stride", 4, B.AIO_EINVAL), ("head_stride", 12, B.AIO_EINVAL),
    ("page_size", 4, B.AIO_EUNSUPPORTED), ("page_size", 24, B.AIO_EUNSUPPORTED),
    ("page_size", 512, B.AIO_EUNSUPPORTED), ("head_dim", 96, B.AIO_EUNSUPPORTED),
])
def test_pool_refusals(L, field, value, code):
    kv = paged(**{field: value})
    assert L.aio_paged_attention(R(kv), R(seqs()), R(attn()), P16, 1 << 30, None) == code
    assert L.aio_page_append(R(kv), R(seqs()), P16, P16, B.AIO_F32, 512, 64, None) == code


@pytest.mark.parametrize("change,code", [
    (dict(n_seqs=-1), B.AIO_ERANGE), (dict(n_rows=-1), B.AIO_ERANGE),
    (dict(max_len=-1), B.AIO_ERANGE), (dict(n_rows=5), B.AIO_ERANGE),
    (dict(lens_dev=None), B.AIO_EINVAL), (dict(table_dev=None), B.AIO_EINVAL),
    (dict(lens_dev=2), B.AIO_EINVAL), (dict(table_dev=6), B.AIO_EINVAL),
    (dict(cu_q_dev=2), B.AIO_EINVAL), (dict(table_stride=0), B.AIO_EINVAL),
])
def test_sequence_refusals(L, change, code):
    s = seqs(**change)
    assert L.aio_paged_attention(R(paged()), R(s), R(attn()), P16, 1 << 30, None) == code
    assert L.aio_page_append(R(paged()), R(s), P16, P16, B.AIO_F32, 512, 64, None) == code


@pytest.mark.parametrize("change,code", [
    (dict(q_dev=None), B.AIO_EINVAL), (dict(out_dev=8), B.AIO_EINVAL),
    (dict(lse_dev=2), B.AIO_EINVAL), (dict(q_stride=-4), B.AIO_EINVAL),
    (dict(q_stride=1026), B.AIO_EINVAL), (dict(out_stride=3), B.AIO_EINVAL),
    (dict(dtype=2), B.AIO_EINVAL), (dict(n_heads=12), B.AIO_EINVAL),
    (dict(n_heads=0), B.AIO_EINVAL), (dict(n_heads=8 * 17), B.AIO_EUNSUPPORTED),
    (dict(scale=0.0), B.AIO_EINVAL), (dict(scale=-1.0), B.AIO_EINVAL),
    (dict(scale=float("nan")), B.AIO_EINVAL), (dict(scale=float("inf")), B.AIO_EINVAL),
])
def test_attention_refusals(L, change, code):
    a = attn(**change)
    assert L.aio_paged_attention(R(paged()), R(seqs()), R(a), P16, 1 << 30, None) == code
    kv = B.aio_packed_kv(P16, P16, 512, 64, 100, 8, 64)
    s = seqs(cu_q_dev=P16, cu_k_dev=P16)
    assert L.aio_packed_attention(R(kv), R(s), R(a), P16, 1 << 30, None) == code


def test_bf16_strides_are_16_bytes(L):
    a = attn(dtype=B.AIO_BF16, q_stride=1028)
    assert L.aio_paged_attention(R(paged()), R(seqs()), R(a), P16, 1 << 30, None) == B.AIO_EINVAL


def test_null_structs(L):
    for kv, s, a in ((None, seqs(), attn()), (paged(), None, attn()), (paged(), seqs(), None)):
        r = [None if x is None else R(x) for x in (kv, s, a)]
        assert L.aio_paged_attention(*r, P16, 1 << 30, None) == B.AIO_EINVAL
    kv = B.aio_packed_kv(P16, P16, 512, 64, 100, 8, 64)
    for change in (dict(cu_q_dev=None, cu_k_dev=P16), dict(cu_q_dev=P16, cu_k_dev=None)):
        assert L.aio_packed_attention(R(kv), R(seqs(**change)), R(attn()), P16, 1 << 30,
                                      None) == B.AIO_EINVAL
    # packed boundaries make no sense for pages
    assert L.aio_paged_attention(R(paged()), R(seqs(cu_q_dev=P16, cu_k_dev=P16)), R(attn()), P16,
                                 1 << 30, None) == B.AIO_EINVAL


@pytest.mark.parametrize("field,value,code", [
    ("k_dev", 8, B.AIO_EINVAL), ("v_dev", None, B.AIO_EINVAL), ("row_stride", 4, B.AIO_EINVAL),
    ("head_stride", -8, B.AIO_EINVAL), ("n_rows", -1, B.AIO_ERANGE),
    ("n_kv_heads", 0, B.AIO_EINVAL), ("head_dim", 80, B.AIO_EUNSUPPORTED),
])
def test_packed_refusals(L, field, value, code):
    kv = B.aio_packed_kv(P16, P16, 512, 64, 100, 8, 64)
    setattr(kv, field, value)
    s = seqs(cu_q_dev=P16, cu_k_dev=P16)
    assert L.aio_packed_attention(R(kv), R(s), R(attn()), P16, 1 << 30, None) == code


def test_nothing_to_do(L):
    """Empty batches return before any device call."""
    s = seqs(n_seqs=0, n_rows=0, lens_dev=None, table_dev=None)
    assert L.aio_paged_attention(R(paged()), R(s), R(attn(q_dev=None, out_dev=None)), None, 0,
                                 None) == B.AIO_OK
    assert L.aio_page_append(R(paged()), R(s), None, None, B.AIO_F32, 512, 64, None) == B.AIO_OK
    kv = B.aio_packed_kv(None, None, 512, 64, 0, 8, 64)
    s = seqs(n_rows=0, cu_q_dev=P16, cu_k_dev=P16)
    assert L.aio_packed_attention(R(kv), R(s), R(attn()), None, 0, None) == B.AIO_OK
    assert L.aio_page_copy(P16, 2, 4096, 4, 512, 512, None, None, 0, None) == B.AIO_OK
    assert L.aio_logprobs(None, 0, 0, 10, 10, None, 0, None, None, None, None, None, 0,
                          None) == B.AIO_OK


def test_attention_workspace(L):
    # many sequences need no split, one long one does; a workspace too small is refused
    assert B.aio_attn_workspace_bytes(2048, 2048, 128, 32, 32, 128) == 0
    need = B.aio_attn_workspace_bytes(1, 1, 32768, 32, 8, 128)
    assert need > 0
    assert B.aio_attn_workspace_bytes(1, 5, 32768, 32, 8, 128, prompts=True) > 0
    assert B.aio_attn_workspace_bytes(1, 8192, 8192, 32, 8, 128, prompts=True) == 0
    for bad in ((-1, 1, 1, 8, 8, 64), (1, 2, 1, 8, 8, 64), (1, 1, 1, 8, 3, 64),
                (1, 1, 1, 8, 8, 65)):
        assert B.aio_attn_workspace_bytes(*bad) == 0
    kv = paged(head_dim=128, page_stride=8 * 16 * 128, head_stride=16 * 128)
    s = seqs(n_seqs=1, n_rows=1, max_len=32768)
    a = attn(n_heads=32)
    for ws, n in ((P16, need - 1), (None, need), (8, need)):
        assert L.aio_paged_attention(R(kv), R(s), R(a), ws, n, None) == B.AIO_EINVAL


def test_sizes_past_32_bits_are_refused(L):
    big = 0x7fffffff
    s = seqs(n_seqs=big, n_rows=big, max_len=1)
    assert L.aio_paged_attention(R(paged()), R(s), R(attn()), P16, 1 << 62, None) == B.AIO_ERANGE
    s = seqs(n_seqs=1, n_rows=big, max_len=big, cu_q_dev=P16)
    assert L.aio_paged_attention(R(paged()), R(s), R(attn()), P16, 1 << 62, None) == B.AIO_ERANGE


def test_grids_past_32_bits_are_refused(L):
    """A grid's axis holds fewer than 2^32 threads, 2^24 workgroups of 256."""
    n = 1 << 24
    s = seqs(n_seqs=n, n_rows=n, max_len=16)
    assert L.aio_page_append(R(paged()), R(s), P16, P16, B.AIO_F32, 512, 64, None) == B.AIO_ERANGE
    s = seqs(n_seqs=n // 8, n_rows=n // 8, max_len=16)
    assert L.aio_paged_attention(R(paged()), R(s), R(attn()), P16, 1 << 62, None) == B.AIO_ERANGE
    s = seqs(n_seqs=n // 8, n_rows=n // 8, max_len=16, cu_q_dev=P16)
    assert L.aio_paged_attention(R(paged()), R(s), R(attn()), P16, 1 << 62, None) == B.AIO_ERANGE
    one = (ctypes.c_int32 * 1)(0)
    two = (ctypes.c_int32 * 1)(1)
    for size, code in ((1 << 38, B.AIO_ERANGE), (0, B.AIO_OK)):
        assert L.aio_page_copy(P16, 1, 2 << 38, 2, 1 << 38, size, ctypes.addressof(one),
                               ctypes.addressof(two), 1, None) == code


def test_outputs_that_overlap_are_refused(L):
    for a in (attn(out_stride=0), attn(out_stride=16 * 64 - 4)):
        assert L.aio_paged_attention(R(paged()), R(seqs()), R(a), P16, 1 << 30,
                                     None) == B.AIO_EINVAL
    for kv in (paged(page_stride=0), paged(head_stride=0), paged(page_stride=16 * 64 - 8),
               paged(head_stride=16 * 64 - 8)):
        assert L.aio_page_append(R(kv), R(seqs()), P16, P16, B.AIO_F32, 512, 64,
                                 None) == B.AIO_EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), B.AIO_EINVAL), (dict(row=514), B.AIO_EINVAL), (dict(head=-4), B.AIO_EINVAL),
    (dict(k=None), B.AIO_EINVAL), (dict(v=8), B.AIO_EINVAL),
])
def test_append_refusals(L, kw, code):
    d = dict(dtype=B.AIO_F32, row=512, head=64, k=P16, v=P16)
    d.update(kw)
    assert L.aio_page_append(R(paged()), R(seqs()), d["k"], d["v"], d["dtype"], d["row"],
                             d["head"], None) == code


@pytest.mark.parametrize("src,dst,code", [
    ([0], [4], B.AIO_ERANGE), ([-1], [1], B.AIO_ERANGE), ([1], [-1], B.AIO_ERANGE),
    ([0, 1], [2, 2], B.AIO_EINVAL), ([0], [0], B.AIO_EINVAL), ([0, 1], [1, 2], B.AIO_EINVAL),
])
def test_copy_refusals(L, src, dst, code):
    a, b = (ctypes.c_int32 * len(src))(*src), (ctypes.c_int32 * len(dst))(*dst)
    assert L.aio_page_copy(P16, 2, 4096, 4, 512, 512, a, b, len(src), None) == code


def test_copy_shape_refusals(L):
    a, b = (ctypes.c_int32 * 1)(0), (ctypes.c_int32 * 1)(1)

    def call(pool=P16, planes=2, plane=4096, pages=4, stride=512, size=512, src=a, n=1):
        return L.aio_page_copy(pool, planes, plane, pages, stride, size, src, b, n, None)

    for kw in (dict(pool=None), dict(pool=8), dict(plane=4088), dict(stride=256), dict(size=500),
               dict(src=None), dict(plane=-16)):
        assert call(**kw) == B.AIO_EINVAL, kw
    for kw in (dict(planes=0), dict(pages=0), dict(n=-1)):
        assert call(**kw) == B.AIO_ERANGE, kw


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), B.AIO_ERANGE), (dict(n=0), B.AIO_ERANGE),
    (dict(n=(1 << 30) + 1, stride=1 << 31), B.AIO_ERANGE), (dict(stride=99), B.AIO_ERANGE),
    (dict(top=-1), B.AIO_ERANGE), (dict(top=33), B.AIO_ERANGE),
    (dict(n=5, top=6), B.AIO_ERANGE), (dict(dtype=2), B.AIO_EINVAL), (dict(x=None), B.AIO_EINVAL),
    (dict(x=2), B.AIO_EINVAL), (dict(t=None), B.AIO_EINVAL), (dict(lp=None), B.AIO_EINVAL),
    (dict(lp=2), B.AIO_EINVAL), (dict(ent=2), B.AIO_EINVAL), (dict(ids=None), B.AIO_EINVAL),
    (dict(tlp=None), B.AIO_EINVAL),
])
def test_logprob_refusals(L, kw, code):
    d = dict(x=P16, dtype=B.AIO_F32, rows=4, n=100, stride=100, t=P16, top=5, lp=P16, ent=P16,
             ids=P16, tlp=P16)
    d.update(kw)
    assert L.aio_logprobs(d["x"], d["dtype"], d["rows"], d["n"], d["stride"], d["t"], d["top"],
                          d["lp"], d["ent"], d["ids"], d["tlp"], P16, 1 << 30, None) == code


def test_logprob_workspace(L):
    need = B.aio_logprobs_workspace_bytes(1, 32000, 5)
    assert need > 0 and B.aio_logprobs_workspace_bytes(4096, 32000, 5) == 0
    for ws, n in ((None, need), (P16, need - 1), (8, need)):
        assert L.aio_logprobs(P16, 0, 1, 32000, 32000, None, 5, None, None, P16, P16, ws, n,
                              None) == B.AIO_EINVAL


# ------------------------------------------------------------- page tables

@pytest.mark.parametrize("seed", range(6))
def test_page_tables_hold_what_was_written(L, seed):
    """Random opens, forks, extensions, truncations, closes and compactions: every
    sequence reads back what was written to it, pages are counted right, and no two
    sequences ever write the same slot."""
    rng = random.Random(seed)
    n_pages, ps, max_seqs = rng.choice([7, 40]), 8, 6
    p = B.Pages(n_pages, ps, max_seqs)
    mem = [[None] * ps for _ in range(n_pages)]
    want, stamp = {}, 0

    def pages(s):
        lens, table = p.rows([s], n_pages)
        k = -(-int(lens[0]) // ps)
        assert (table[0, k:] == -1).all() and (table[0, :k] >= 0).all()
        return int(lens[0]), table[0, :k].tolist()

    def copy(src, dst):
        assert not set(src) & set(dst) and len(set(dst)) == len(dst)
        for a, b in zip(list(src), list(dst)):
            mem[b] = list(mem[a])

    for _ in range(400):
        op = rng.choice(["open", "fork", "extend", "extend", "extend", "trunc", "close", "compact"])
        seq = rng.choice(sorted(want)) if want else None
        if op == "open":
            if len(want) == max_seqs:
                with pytest.raises(B.AioError):
                    p.open()
            else:
                s = p.open()
                assert s not in want
                want[s] = []
        elif seq is None:
            continue
        elif op == "fork":
            if len(want) < max_seqs:
                c = p.fork(seq)
                want[c] = list(want[seq])
        elif op == "extend":
            n = rng.randint(0, 3 * ps)
            before = (p.free, pages(seq))
            try:
                copy(*p.extend(seq, n))
            except B.AioError as e:
                assert e.code == B.AIO_ENOMEM and (p.free, pages(seq)) == before
                continue
            length, tab = pages(seq)
            assert length == len(want[seq]) + n
            for i in range(len(want[seq]), length):
                stamp += 1
                mem[tab[i // ps]][i % ps] = stamp
                want[seq].append(stamp)
        elif op == "trunc":
            n = rng.randint(0, len(want[seq]))
            p.truncate(seq, n)
            del want[seq][n:]
        elif op == "close":
            p.close(seq)
            del want[seq]
        else:
            copy(*map(list, p.compact()))
            used = n_pages - p.free
            assert all(g < used for s in want for g in pages(s)[1])
        held = set()
        for s, vals in want.items():
            length, tab = pages(s)
            assert length == len(vals)
            assert [mem[tab[i // ps]][i % ps] for i in range(length)] == vals
            held |= set(tab)
        assert p.free == n_pages - len(held)


def test_page_table_refusals(L):
    h = ctypes.c_void_p()
    for args in ((0, 16, 1), (1, 12, 1), (1, 4, 1), (1, 16, 0), ((1 << 30) + 1, 16, 1)):
        assert L.aio_pages_create(*args, R(h)) == B.AIO_ERANGE
    assert L.aio_pages_create(4, 16, 1, None) == B.AIO_EINVAL
    p = B.Pages(4, 16, 2)
    i, j, k = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    assert L.aio_pages_open(None, R(i)) == B.AIO_EINVAL
    assert L.aio_pages_open(p.handle, None) == B.AIO_EINVAL
    for s in (-1, 0, 5):  # none is open
        assert L.aio_pages_close(p.handle, s) == B.AIO_ERANGE
        assert L.aio_pages_fork(p.handle, s, R(i)) == B.AIO_ERANGE
        assert L.aio_pages_extend(p.handle, s, 1, R(i), R(j), R(k)) == B.AIO_ERANGE
        assert L.aio_pages_truncate(p.handle, s, 0) == B.AIO_ERANGE
        assert L.aio_pages_row(p.handle, s, None, 0, R(i)) == B.AIO_ERANGE
    s = p.open()
    assert L.aio_pages_extend(p.handle, s, -1, R(i), R(j), R(k)) == B.AIO_ERANGE
    assert L.aio_pages_extend(p.handle, s, 65, R(i), R(j), R(k)) == B.AIO_ENOMEM
    assert L.aio_pages_extend(p.handle, s, 0x7fffffff, R(i), R(j), R(k)) == B.AIO_ERANGE
    p.extend(s, 40)
    assert L.aio_pages_truncate(p.handle, s, 41) == B.AIO_ERANGE
    row = (ctypes.c_int32 * 2)()
    assert L.aio_pages_row(p.handle, s, row, 2, R(i)) == B.AIO_ERANGE
    # a compaction without room for its copies changes nothing and says how many
    t = p.open()
    p.extend(t, 16)
    p.close(s)
    before = p.rows([t], 4)[1].tolist()
    buf = (ctypes.c_int32 * 4)()
    assert L.aio_pages_compact(p.handle, buf, buf, 0, R(i)) == B.AIO_ERANGE and i.value == 1
    assert p.rows([t], 4)[1].tolist() == before
    assert L.aio_pages_free(None) == B.AIO_EINVAL
    L.aio_pages_destroy(None)


def test_paged_forward_rejects_without_a_device(L):
    i = (ctypes.c_int32 * 1)(1)
    p = B.aio_paged_pool(paged(), 64, 2)
    assert L.aio_paged_forward(None, R(p), 1, i, i, i, 1, i, i, 1, P16, 256, 1 << 30) == B.AIO_EINVAL
    assert L.aio_paged_forward_bytes(None, 1, 1, 1) == 0


@pytest.mark.parametrize("cls,pack,fields", [
    (B.aio_paged_kv, B._pack_paged, (16, 32, 1 << 40, 1 << 33, 10, 16, 8, 64)),
    (B.aio_packed_kv, B._pack_packed, (16, 32, 1 << 40, 64, 100, 8, 64)),
    (B.aio_seqs, B._pack_seqs, (4, 5, 100, 16, 32, 48, 8, 64)),
    (B.aio_attn, B._pack_attn, (16, 32, 0, 1024, 2048, 1, 16, 0.125)),
])
def test_packed_structs_are_the_structs(cls, pack, fields):
    b = pack(*fields)
    assert len(b) == ctypes.sizeof(cls)
    s = cls.from_buffer_copy(b)
    assert tuple(getattr(s, n) or 0 for n, _ in cls._fields_) == fields
    for i, (_, t) in enumerate(cls._fields_):
        if t is ctypes.c_int32:
            with pytest.raises(ValueError, match=cls.__name__):
                pack(*fields[:i], 1 << 31, *fields[i + 1:])
        elif t is ctypes.c_float:  # (a C float: infinite, which the call refuses)
            assert cls.from_buffer_copy(pack(*fields[:i], 1e300)).scale == float("inf")
