"""Which kernel an attention takes (host): the cases of the 256-row tiles are the ones
that they are meant to be, and both sides of each rule."""
import ctypes

import pytest

from paper_2604_09752_amd import binding as B
from tests import test_gpu_attention_wide as wide


def plan(n_seqs, n_rows, max_len, H, Hkv, hd, dtype, prompts):
    """Waves of a workgroup of prompt rows, splits, whether keys pass the caches by."""
    s = B.aio_seqs(n_seqs, n_rows, max_len, 16 if prompts else None, None, None, 0, None)
    out = (ctypes.c_int32 * 3)()
    rc = B.lib().aio_attention_plan(ctypes.byref(s), H, Hkv, hd, dtype, out)
    return tuple(out) if rc == B.AIO_OK else rc


@pytest.mark.parametrize("name", list(wide.CASES))
def test_wide_cases(name):
    H, Hkv, hd, ql, kl, _, waves = wide.CASES[name]
    n = sum(ql) + 2  # (with the rows of no sequence)
    assert plan(len(ql), n, max(kl), H, Hkv, hd, B.AIO_BF16, True)[0] == waves
    assert plan(len(ql), n, max(kl), H, Hkv, hd, B.AIO_F32, True)[0] == 4


@pytest.mark.parametrize("args,want", [
    # one new token: splits of at least 128 keys above 512, streams past 64 MB
    ((1, 1, 512, 16, 8, 128, B.AIO_F32, False), (0, 1, 0)),
    ((1, 1, 513, 16, 8, 128, B.AIO_F32, False), (0, 5, 0)),
    ((7, 7, 4096, 32, 8, 128, B.AIO_BF16, False), (0, 8, 1)),
    ((2, 2, 4096, 32, 8, 128, B.AIO_BF16, False), (0, 32, 0)),
    ((1024, 1024, 8192, 8, 1, 64, B.AIO_BF16, False), (0, 1, 1)),
    # prompt rows: splits until there are two workgroups per CU (one of fp32 queries)
    ((1, 5, 3000, 32, 32, 128, B.AIO_BF16, True), (4, 16, 0)),
    ((1, 5, 3000, 32, 32, 128, B.AIO_F32, True), (4, 8, 0)),
    ((1, 8192, 8192, 32, 32, 128, B.AIO_BF16, True), (8, 1, 0)),
])
def test_rules(args, want):
    assert plan(*args) == want


def test_rejects():
    assert plan(1, 1, 100, 16, 3, 128, B.AIO_F32, False) == B.AIO_EINVAL
    assert plan(1, 1, 100, 16, 8, 96, B.AIO_F32, False) == B.AIO_EUNSUPPORTED
    assert plan(2, 1, 100, 16, 8, 128, B.AIO_F32, False) == B.AIO_ERANGE
    out = (ctypes.c_int32 * 3)()
    assert B.lib().aio_attention_plan(None, 8, 8, 64, 0, out) == B.AIO_EINVAL
