"""Calls of aio_paged_forward at its limits (needs an MI355X)."""
import ctypes

import numpy as np
import pytest
import torch

import synth
from paper_2604_09752_amd import binding as B
from tests.gpu_cases import LOGIT_TOL

pytestmark = pytest.mark.gpu

TINY = synth.CONFIGS["tiny"]


def model(**kw):
    cfg = TINY.with_(prompt_len=20, n_steps=8, **kw)
    return B.DeviceModel(cfg, synth.make_weights(cfg))


def idle(n):
    """One sequence of one token, and n - 1 without any."""
    one = np.zeros(n, np.int32)
    one[n // 2] = 1
    return dict(rows=one, lens=one, table=np.zeros((n, 1), np.int32), tokens=[3], out_rows=[0])


@pytest.mark.parametrize("n", [65, 5000, 1 << 20])
def test_many_idle_sequences(n):
    """One token of one sequence among up to 2^20 without any: as alone."""
    dm = model(name="many_kv", d_model=256, ffn_dim=256, n_heads=16, n_kv_heads=16)
    with torch.cuda.stream(dm.stream):
        pool, logits, want = dm.new_pool(2), dm.new_logits(1), dm.new_logits(1)
    dm.paged_forward(pool, **idle(n), logits=logits)
    dm.paged_forward(pool, [1], [1], [[1]], [3], [0], want)
    dm.sync()
    # (alone it takes the kernel of one new token each, fp32 alike: the layers behind the first
    # differ by roundings)
    assert (logits - want).abs().max() <= LOGIT_TOL
    assert torch.equal(pool[0, :, 0], pool[0, :, 1]) and pool[0, :, 0].any()
    dm.close()


def test_more_output_rows_than_32_bits_step_over():
    dm = model(name="outs")
    with torch.cuda.stream(dm.stream):
        pool, logits = dm.new_pool(2), dm.new_logits(1)
    kv = B.aio_paged_kv(pool.data_ptr(), pool[0, 1].data_ptr(), pool.stride(2), pool.stride(3), 2,
                        16, dm.c.n_kv_heads, dm.c.head_dim)
    p = B.aio_paged_pool(kv, pool.stride(0), dm.c.n_layers)
    n = B.lib().aio_paged_forward_bytes(ctypes.byref(dm.c), 1, 1, 1)
    scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
    one, zero = np.ones(1, np.int32), np.zeros(1, np.int32)
    for n_out in (0x7fff0001, 0x7fffffff):  # (refused before out_rows is read)
        assert B.lib().aio_paged_forward(
            dm.handle, ctypes.byref(p), 1, one.ctypes.data, one.ctypes.data, zero.ctypes.data, 1,
            one.ctypes.data, zero.ctypes.data, n_out, logits.data_ptr(), scratch.data_ptr(),
            n) == B.AIO_ERANGE
    dm.sync()
    assert not pool.any()
    dm.close()


@pytest.mark.parametrize("change", [
    dict(layer_stride=0), dict(layer_stride=1), dict(v=0), dict(v=1), dict(v=2),
    dict(page_stride=1), dict(head_stride=1)])
def test_pools_whose_parts_overlap(change):
    """Strides and the distance of V are given in parts: 1 is a layer's K, a page or a
    head too short."""
    dm = model(name="overlap")
    with torch.cuda.stream(dm.stream):
        pool, logits = dm.new_pool(4), dm.new_logits(1)
    c, one = dm.c, 16 * dm.c.head_dim
    v = {0: pool[0, 0], 1: pool[0, 0, 1], 2: pool[1, 0]}
    kv = B.aio_paged_kv(pool.data_ptr(), v[change["v"]].data_ptr() if "v" in change else
                        pool[0, 1].data_ptr(), pool.stride(2), pool.stride(3), 4, 16,
                        c.n_kv_heads, c.head_dim)
    if "page_stride" in change:
        kv.page_stride = one  # its second head is the next page's first
    if "head_stride" in change:
        kv.head_stride = pool.stride(2)  # the next page's first head
    p = B.aio_paged_pool(kv, change["layer_stride"] * pool.stride(1)  # (1: on the V before)
                         if "layer_stride" in change else pool.stride(0), c.n_layers)
    n = B.lib().aio_paged_forward_bytes(ctypes.byref(c), 1, 1, 1)
    scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
    one_, zero = np.ones(1, np.int32), np.zeros(1, np.int32)
    assert B.lib().aio_paged_forward(
        dm.handle, ctypes.byref(p), 1, one_.ctypes.data, one_.ctypes.data, zero.ctypes.data, 1,
        one_.ctypes.data, zero.ctypes.data, 1, logits.data_ptr(), scratch.data_ptr(),
        n) == B.AIO_EINVAL
    dm.sync()
    assert not pool.any()
    dm.close()


def test_a_captured_pass():
    """Refused: the graph would read the call's host arrays when it is replayed.  The capture
    goes on without it."""
    dm = model(name="captured")
    with torch.cuda.stream(dm.stream):
        pool, logits, seen = dm.new_pool(2), dm.new_logits(1), torch.zeros(4, device="cuda")
    call = (pool, [1], [1], [[0]], [3], [0], logits)
    dm.paged_forward(*call)  # (its scratch is there)
    dm.sync()
    want = logits.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=dm.stream):
        with pytest.raises(B.AioError) as e:
            dm.paged_forward(*call)
        seen += 1
    assert e.value.code == B.AIO_EINVAL
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        assert (seen == i + 1).all() and torch.equal(logits, want)
    logits.zero_()
    torch.cuda.synchronize()
    dm.paged_forward(*call)
    dm.sync()
    assert torch.equal(logits, want)
    dm.close()


def test_the_call_returns_before_its_work():
    """Enqueued behind 15 ms of products, which are not done when it returns."""
    dm = model(name="behind")
    with torch.cuda.stream(dm.stream):
        pool, logits = dm.new_pool(8), dm.new_logits(40)
        a = torch.zeros((8192, 8192), dtype=torch.bfloat16, device="cuda")
        a @ a
    call = (pool, [20, 20], [20, 20], [[0, 1], [2, 3]], [5] * 40, list(range(40)), logits)
    dm.paged_forward(*call)
    dm.sync()
    want = logits.clone()
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    with torch.cuda.stream(dm.stream):
        for _ in range(20):
            a @ a
        done.record()
    dm.paged_forward(*call)
    assert not done.query()
    dm.sync()
    assert torch.equal(logits, want)
    dm.close()


@pytest.mark.parametrize("vocab,rows", [(997, 2), (1001, 3), (515, 10)])
def test_rows_of_an_odd_vocabulary(vocab, rows):
    """Groups of the LM head whose logits start at any multiple of 4 bytes: every row as in
    one group, nothing behind the last."""
    outs = []
    for most in (rows, 1):
        dm = model(name="odd", vocab=vocab, max_verify=most)
        with torch.cuda.stream(dm.stream):
            pool, logits = dm.new_pool(2), torch.full((24, vocab), 7.0, device="cuda")
        dm.paged_forward(pool, [21], [21], [[0, 1]], [i % 500 for i in range(21)],
                         list(range(21)) + [4, 4], logits[:23])
        dm.sync()
        assert (logits[23] == 7).all() and torch.equal(logits[21], logits[4])
        outs.append(logits[:23].clone())
        dm.close()
    assert torch.isfinite(outs[0]).all() and (outs[0] - outs[1]).abs().max() <= LOGIT_TOL
