"""The 8-bit pages, the groups of shared prefixes and the norm and rotation of query and key
rows on the host: what they refuse, and their workspaces."""
import ctypes
import random

import pytest
import torch

from paper_2604_09752_amd import binding as B

P16 = 16  # any aligned non-null pointer: nothing is enqueued by a refused call
R = ctypes.byref
BIG = 1 << 30


@pytest.fixture(scope="module")
def L():
    return B.lib()


def q8(**kw):
    kv = B.aio_q8_kv(1 << 20, 1 << 30, 1 << 40, 1 << 41, 8 * 16 * 64, 16 * 64, 8 * 16, 16, 10, 16,
                     8, 64)
    for f, v in kw.items():
        setattr(kv, f, v)
    return kv


def paged():
    return B.aio_paged_kv(1 << 20, 1 << 30, 8 * 16 * 64, 16 * 64, 10, 16, 8, 64)


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


def groups(**kw):
    x = B.aio_prefixes(2, 80, P16, P16)
    for f, v in kw.items():
        setattr(x, f, v)
    return x


def every(L, kv=None, s=None, x=None, a=None, ws=P16, n=BIG):
    """What each of the attentions over 8-bit pages or with groups returns."""
    kv, s, x, a = kv or q8(), s or seqs(), x or groups(), a or attn()
    return [L.aio_q8_attention(R(kv), R(s), R(a), ws, n, None),
            L.aio_q8_prefix_attention(R(kv), R(s), R(x), R(a), ws, n, None),
            L.aio_prefix_attention(R(paged()), R(s), R(x), R(a), ws, n, None)]


def append(L, kv=None, s=None, k=P16, v=P16, dtype=B.AIO_F32, row=512, head=64):
    return L.aio_q8_append(R(kv or q8()), R(s or seqs()), k, v, dtype, row, head, None)


@pytest.mark.parametrize("field,value,code", [
    ("k_dev", None, B.AIO_EINVAL), ("v_dev", 8, B.AIO_EINVAL), ("k_exp_dev", None, B.AIO_EINVAL),
    ("v_exp_dev", 12, B.AIO_EINVAL), ("n_pages", 0, B.AIO_EINVAL), ("n_kv_heads", 0, B.AIO_EINVAL),
    ("page_stride", -16, B.AIO_EINVAL), ("page_stride", 8, B.AIO_EINVAL),
    ("head_stride", 24, B.AIO_EINVAL), ("exp_page_stride", 4, B.AIO_EINVAL),
    ("exp_head_stride", -8, B.AIO_EINVAL), ("exp_head_stride", 12, B.AIO_EINVAL),
    ("page_size", 4, B.AIO_EUNSUPPORTED), ("page_size", 24, B.AIO_EUNSUPPORTED),
    ("page_size", 512, B.AIO_EUNSUPPORTED), ("head_dim", 96, B.AIO_EUNSUPPORTED)])
def test_pool_refusals(L, field, value, code):
    kv = q8(**{field: value})
    assert every(L, kv=kv)[:2] == [code, code]
    assert append(L, kv) == code


@pytest.mark.parametrize("change,code", [
    (dict(n_seqs=-1), B.AIO_ERANGE), (dict(n_rows=-1), B.AIO_ERANGE),
    (dict(max_len=-1), B.AIO_ERANGE), (dict(n_rows=5), B.AIO_ERANGE),
    (dict(lens_dev=None), B.AIO_EINVAL), (dict(table_dev=6), B.AIO_EINVAL),
    (dict(cu_q_dev=2), B.AIO_EINVAL), (dict(table_stride=0), B.AIO_EINVAL)])
def test_sequence_refusals(L, change, code):
    assert every(L, s=seqs(**change)) == [code] * 3
    assert append(L, s=seqs(**change)) == code


@pytest.mark.parametrize("change,code", [
    (dict(q_dev=None), B.AIO_EINVAL), (dict(out_dev=8), B.AIO_EINVAL),
    (dict(lse_dev=2), B.AIO_EINVAL), (dict(q_stride=-4), B.AIO_EINVAL),
    (dict(out_stride=512), B.AIO_EINVAL), (dict(dtype=2), B.AIO_EINVAL),
    (dict(n_heads=12), B.AIO_EINVAL), (dict(n_heads=8 * 17), B.AIO_EUNSUPPORTED),
    (dict(scale=0.0), B.AIO_EINVAL), (dict(scale=float("nan")), B.AIO_EINVAL),
    (dict(scale=2.4e38), B.AIO_EINVAL)])
def test_attention_refusals(L, change, code):
    assert every(L, a=attn(**change)) == [code] * 3


@pytest.mark.parametrize("change,code", [
    (dict(n_groups=-1), B.AIO_ERANGE), (dict(n_groups=(1 << 30) + 1), B.AIO_ERANGE),
    (dict(max_prefix=-1), B.AIO_ERANGE), (dict(cu_seqs_dev=None), B.AIO_EINVAL),
    (dict(prefix_lens_dev=None), B.AIO_EINVAL), (dict(cu_seqs_dev=18), B.AIO_EINVAL),
    (dict(prefix_lens_dev=2), B.AIO_EINVAL)])
def test_group_refusals(L, change, code):
    assert every(L, x=groups(**change))[1:] == [code] * 2


def test_null_structs_and_packed_boundaries(L):
    kv, s, x, a = R(q8()), R(seqs()), R(groups()), R(attn())
    for args in ((None, s, a), (kv, None, a), (kv, s, None)):
        assert L.aio_q8_attention(*args, P16, BIG, None) == B.AIO_EINVAL
    for args in ((None, s, x, a), (kv, None, x, a), (kv, s, None, a), (kv, s, x, None)):
        assert L.aio_q8_prefix_attention(*args, P16, BIG, None) == B.AIO_EINVAL
        assert L.aio_prefix_attention(*args, P16, BIG, None) == B.AIO_EINVAL
    assert L.aio_q8_append(None, s, P16, P16, 0, 512, 64, None) == B.AIO_EINVAL
    assert L.aio_q8_append(kv, None, P16, P16, 0, 512, 64, None) == B.AIO_EINVAL
    assert every(L, s=seqs(cu_q_dev=P16, cu_k_dev=P16)) == [B.AIO_EINVAL] * 3


def test_append_refusals(L):
    for kw in (dict(k=None), dict(v=8), dict(dtype=2), dict(row=-4), dict(row=514), dict(head=2),
               dict(dtype=B.AIO_BF16, row=516)):
        assert append(L, **kw) == B.AIO_EINVAL
    # pages, heads, K and V, codes and bytes in one another's place
    for kw in (dict(page_stride=7 * 16 * 64), dict(head_stride=15 * 64), dict(head_stride=0),
               dict(exp_page_stride=7 * 16), dict(exp_head_stride=8), dict(exp_head_stride=0),
               dict(v_dev=(1 << 20) + 16), dict(v_exp_dev=(1 << 40) + 8),
               dict(v_dev=(1 << 20) + 16 * 64),
               dict(k_exp_dev=(1 << 20) + 16 * 64 - 8), dict(v_exp_dev=(1 << 30) - 8),
               dict(k_exp_dev=1 << 30)):
        assert append(L, q8(**kw)) == B.AIO_EINVAL, kw
    # K, V and their bytes within one page, as pages may be laid out
    one = 8 * 16 * 65
    ok = q8(v_dev=(1 << 20) + one, k_exp_dev=(1 << 20) + 8 * 16 * 64,
            v_exp_dev=(1 << 20) + one + 8 * 16 * 64, page_stride=2 * one, exp_page_stride=2 * one)
    assert append(L, ok, k=None) == B.AIO_EINVAL
    assert append(L, ok, s=seqs(n_seqs=0, n_rows=0, lens_dev=None, table_dev=None)) == B.AIO_OK


def test_nothing_to_do(L):
    s = seqs(n_seqs=0, n_rows=0, lens_dev=None, table_dev=None)
    a = attn(q_dev=None, out_dev=None)
    assert every(L, s=s, a=a, ws=None, n=0) == [B.AIO_OK] * 3
    assert append(L, s=s, k=None, v=None) == B.AIO_OK
    r = B.aio_qk_rows(None, None, None, None, 512, 512, 512, 512, 0, 0, 8, 8, 64)
    assert L.aio_qk_norm_rope(R(r), None, None, None, 1e-5, 1e4, None) == B.AIO_OK


def test_workspaces(L):
    def need(*a, **kw):
        return B.aio_prefix_workspace_bytes(*a, **kw)

    # no group, or none that shares a whole unit of 64 keys: as without groups
    for n, p in ((0, 5000), (3, 0), (3, 63)):
        assert need(8, 8, 5000, n, p, 32, 8, 128) == B.aio_attn_workspace_bytes(
            8, 8, 5000, 32, 8, 128)
    # shared and own keys: a place at least for both
    row = 8 * 32 * 130 * 4
    assert need(8, 8, 128, 1, 64, 32, 8, 128) == 2 * row
    big = need(8, 8, 30000, 1, 20000, 32, 8, 128)
    assert big > 2 * row and big % row == 0
    assert need(8, 40, 30000, 2, 20000, 32, 8, 128, prompts=True) % (40 * 32 * 130 * 4) == 0
    for bad in ((-1, 1, 100, 1, 64, 8, 8, 64), (1, 1, 100, -1, 64, 8, 8, 64),
                (1, 1, 100, 1, -64, 8, 8, 64), (1, 1, 100, 1, 64, 8, 3, 64),
                (1, 2, 100, 1, 64, 8, 8, 64)):
        assert need(*bad) == 0
    assert L.aio_prefix_workspace_bytes(None, R(groups()), 8, 8, 64) == 0
    assert L.aio_prefix_workspace_bytes(R(seqs()), None, 8, 8, 64) == 0
    # a workspace that is too small or none, once everything else is right
    a = attn(n_heads=8)
    for ws, n in ((None, BIG), (P16, 16), (8, BIG)):
        assert L.aio_prefix_attention(R(paged()), R(seqs()), R(groups()), R(a), ws, n,
                                      None) == B.AIO_EINVAL
    s = seqs(n_seqs=1, n_rows=1, max_len=30000)
    assert L.aio_q8_attention(R(q8()), R(s), R(a), P16, 16, None) == B.AIO_EINVAL


def test_more_than_a_launch_covers(L):
    big = 0x7fffffff
    for cu_q in (None, P16):
        s = seqs(n_seqs=big, n_rows=big, max_len=1 << 30, cu_q_dev=cu_q)
        assert every(L, s=s, x=groups(n_groups=1 << 30, max_prefix=big)) == [B.AIO_ERANGE] * 3
    s = seqs(n_seqs=1 << 22, n_rows=1 << 22, max_len=4096)
    assert B.aio_prefix_workspace_bytes(1 << 22, 1 << 22, 4096, 1 << 22, 4096, 8, 8, 64) == 0
    assert every(L, s=s, x=groups(n_groups=1 << 22, max_prefix=4096), a=attn(n_heads=8))[1:] == \
        [B.AIO_ERANGE] * 2
    assert append(L, s=seqs(n_seqs=1 << 24, n_rows=1 << 24)) == B.AIO_ERANGE


def qk(**kw):
    # queries, keys and values of a row beside one another, outputs apart
    r = B.aio_qk_rows(1 << 20, (1 << 20) + 8 * 64 * 4, 1 << 30, 1 << 40, 16 * 64, 16 * 64, 8 * 64,
                      4 * 64, B.AIO_F32, 10, 8, 4, 64)
    for f, v in kw.items():
        setattr(r, f, v)
    return r


def norm(L, r, pos=P16, qw=P16, kw=None, eps=1e-5, base=1e4):
    return L.aio_qk_norm_rope(R(r), pos, qw, kw, eps, base, None)


@pytest.mark.parametrize("change,code", [
    (dict(q_dev=None), B.AIO_EINVAL), (dict(k_dev=8), B.AIO_EINVAL),
    (dict(q_out_dev=None), B.AIO_EINVAL), (dict(k_out_dev=(1 << 40) + 4), B.AIO_EINVAL),
    (dict(q_stride=-4), B.AIO_EINVAL), (dict(k_stride=1026), B.AIO_EINVAL),
    (dict(q_out_stride=8 * 64 - 4), B.AIO_EINVAL), (dict(k_out_stride=0), B.AIO_EINVAL),
    (dict(dtype=2), B.AIO_EINVAL), (dict(dtype=B.AIO_BF16, k_stride=1028), B.AIO_EINVAL),
    (dict(n_rows=-1), B.AIO_ERANGE), (dict(n_rows=1 << 24), B.AIO_ERANGE),
    (dict(n_heads=0), B.AIO_ERANGE), (dict(n_kv_heads=0), B.AIO_ERANGE),
    (dict(n_heads=(1 << 16) + 1), B.AIO_ERANGE), (dict(head_dim=96), B.AIO_EUNSUPPORTED)])
def test_norm_refusals(L, change, code):
    assert norm(L, qk(**change)) == code


def test_norm_arguments(L):
    assert L.aio_qk_norm_rope(None, P16, None, None, 1e-5, 1e4, None) == B.AIO_EINVAL
    for kw in (dict(pos=None), dict(pos=18), dict(qw=24), dict(kw=2), dict(eps=0.0),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(base=1.0),
               dict(base=float("inf")), dict(base=float("nan"))):
        assert norm(L, qk(), **kw) == B.AIO_EINVAL, kw


def test_norm_outputs_that_overlap(L):
    """Against the bytes of every row (a refusal: EINVAL before the null positions are)."""
    rng = random.Random(5)
    row = 16 * 64
    for kw in (dict(q_out_dev=(1 << 20) + 16),                      # its input, shifted
               dict(q_out_dev=1 << 20),                             # ... of another stride
               dict(k_out_dev=1 << 20, k_out_stride=row),           # the queries
               dict(k_out_dev=(1 << 30) + 16 * 4),                  # the other output
               dict(q_out_dev=(1 << 20) + 2048 - 16, q_out_stride=row)):
        assert norm(L, qk(**kw)) == B.AIO_EINVAL, kw
    # (rows of one stride beside one another: nothing shared)
    B.lib()
    for _ in range(300):
        n, wa, wb = rng.randint(1, 4), 16 * rng.randint(1, 4), 16 * rng.randint(1, 4)
        s, at = 16 * rng.randint(4, 9), 16 * rng.randint(0, 40)
        a = {x for i in range(n) for x in range(20 * 16 + i * s, 20 * 16 + i * s + wa)}
        b = {x for i in range(n) for x in range(at + i * s, at + i * s + wb)}
        assert overlap(20 * 16, s, wa, at, s, wb, n) == bool(a & b)


def overlap(a, sa, wa, b, sb, wb, n):
    """As the host sees it: rows of wa and wb bytes."""
    f = B.lib().aio_rows_overlap_test
    f.argtypes = [ctypes.c_int64] * 7
    return bool(f(a, sa, wa, b, sb, wb, n))


# ------------------------------------------------------------------ the binding

@pytest.fixture
def anywhere(monkeypatch):
    """CPU tensors as far as the checks of shapes."""
    monkeypatch.setattr(B, "_device_of", lambda *t: 0)

    def launch(*a):
        raise AssertionError("not refused")
    monkeypatch.setattr(B, "_launch", launch)


def tensors(**kw):
    t = dict(q=torch.zeros((2, 4, 64)), k=torch.zeros((3, 2, 16, 64), dtype=torch.int8),
             k_exp=torch.zeros((3, 2, 16), dtype=torch.uint8),
             lens=torch.zeros(2, dtype=torch.int32), table=torch.zeros((2, 2), dtype=torch.int32),
             cu_seqs=torch.zeros(2, dtype=torch.int32),
             prefix_lens=torch.zeros(1, dtype=torch.int32))
    t["v"], t["v_exp"], t["out"] = t["k"].clone(), t["k_exp"].clone(), t["q"].clone()
    t.update(kw)
    return t


@pytest.mark.parametrize("bad", [
    dict(k=torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)),
    dict(v=torch.zeros((3, 2, 16, 64), dtype=torch.uint8)),
    dict(k_exp=torch.zeros((3, 2, 16), dtype=torch.int8)),
    dict(v_exp=torch.zeros((3, 2, 8), dtype=torch.uint8)),
    dict(k_exp=torch.zeros((3, 16, 2), dtype=torch.uint8).transpose(1, 2)),
    dict(v_exp=torch.zeros((3, 3, 16), dtype=torch.uint8)[:, :2]),
    dict(k=torch.zeros((3, 2, 64, 16), dtype=torch.int8).transpose(2, 3)),
    dict(q=torch.zeros((2, 4, 128)), out=torch.zeros((2, 4, 128))),
    dict(out=torch.zeros((2, 4, 64), dtype=torch.bfloat16)),
    dict(lens=torch.zeros(2, dtype=torch.int64)),
    dict(lse=torch.zeros((2, 3)))])
def test_binding_refuses_8_bit_pages(anywhere, bad):
    t = tensors(**bad)
    x = {n: t.pop(n) for n in ("cu_seqs", "prefix_lens")}
    with pytest.raises(ValueError):
        B.aio_q8_attention(**t)
    with pytest.raises(ValueError):
        B.aio_q8_prefix_attention(**t, **x)


@pytest.mark.parametrize("bad", [
    dict(cu_seqs=torch.zeros(3, dtype=torch.int32)), dict(cu_seqs=torch.zeros(2)),
    dict(prefix_lens=torch.zeros(1, dtype=torch.int64)),
    dict(prefix_lens=torch.zeros((1, 1), dtype=torch.int32)),
    dict(cu_seqs=torch.zeros((2, 2), dtype=torch.int32)[:, 0]), dict(max_prefix=1 << 32)])
def test_binding_refuses_groups(anywhere, bad):
    t = tensors(**bad)
    with pytest.raises(ValueError):
        B.aio_q8_prefix_attention(**t)
    k = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    t.update(k=k, v=k.clone())
    del t["k_exp"], t["v_exp"]
    with pytest.raises(ValueError):
        B.aio_prefix_attention(**t)


def test_binding_refuses_rows_to_norm(anywhere):
    def call(**kw):
        t = dict(q=torch.zeros((2, 4, 64)), k=torch.zeros((2, 2, 64)),
                 positions=torch.zeros(2, dtype=torch.int32), q_out=torch.zeros((2, 4, 64)),
                 k_out=torch.zeros((2, 2, 64)))
        t.update(kw)
        with pytest.raises(ValueError):
            B.aio_qk_norm_rope(**t)
    h = torch.bfloat16
    for kw in (dict(q=torch.zeros((2, 4, 64), dtype=h)), dict(k=torch.zeros((3, 2, 64))),
               dict(k=torch.zeros((2, 2, 128))), dict(q_out=torch.zeros((2, 4, 64), dtype=h)),
               dict(k_out=torch.zeros((2, 4, 64))), dict(positions=torch.zeros(2)),
               dict(positions=torch.zeros(3, dtype=torch.int32)),
               dict(positions=torch.zeros((2, 2), dtype=torch.int32)[:, 0]),
               dict(q=torch.zeros((2, 64, 4)).transpose(1, 2)),
               dict(q_weight=torch.zeros(64)), dict(k_weight=torch.zeros(128, dtype=h)),
               dict(q=torch.zeros((2, 4, 64), dtype=torch.float16),
                    k=torch.zeros((2, 2, 64), dtype=torch.float16))):
        call(**kw)


def test_binding_sizes_that_do_not_fit():
    with pytest.raises(ValueError, match="32 bits"):
        B.aio_prefix_workspace_bytes(1, 1, 100, (1 << 32) + 1, 64, 8, 8, 64)
