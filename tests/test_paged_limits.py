"""Sizes at the limits of the operators over several sequences (host): what one launch
does not cover is refused before anything is enqueued."""
import ctypes

import pytest

import synth
from paper_2604_09752_amd import binding as B

R = ctypes.byref


@pytest.fixture(scope="module")
def L():
    return B.lib()


def launched(L, n_seqs, n_rows, H, Hkv, hd, dtype):
    s = B.aio_seqs(n_seqs, n_rows, 4096, 16, None, None, 0, None)
    out = (ctypes.c_int32 * 3)()
    return L.aio_attention_plan(R(s), H, Hkv, hd, dtype, out)


@pytest.mark.parametrize("dtype", [B.AIO_F32, B.AIO_BF16])
def test_sequences_without_rows_take_no_place(L, dtype):
    """Workgroups are counted by rows: 2^30 sequences with 2048 rows among them are
    answered, 2^24 tiles x kv heads (2^23 of 256 rows) are not."""
    assert launched(L, 1 << 30, 2048, 1024, 1024, 64, dtype) == B.AIO_OK
    most = 1 << (19 if dtype == B.AIO_F32 else 18)
    assert launched(L, 1 << 30, most - 4096, 32, 32, 64, dtype) == B.AIO_OK
    assert launched(L, 1 << 30, most, 32, 32, 64, dtype) == B.AIO_ERANGE


def test_a_pass_of_any_number_of_idle_sequences(L):
    c = B.make_config(synth.CONFIGS["7b"])
    assert L.aio_paged_forward_bytes(R(c), 1 << 20, 2048, 1) > 0
    assert L.aio_paged_forward_bytes(R(c), (1 << 20) + 1, 2048, 1) == 0


def test_the_largest_sizes_of_a_plan(L):
    big = 0x7fffffff
    for n_rows, H, Hkv, hd in ((big, 1 << 30, 1 << 30, 128), (big, 16, 1, 64)):
        for cu_q in (None, 16):
            s = B.aio_seqs(big, n_rows, 1 << 30, cu_q, None, None, 0, None)
            out = (ctypes.c_int32 * 3)()
            assert L.aio_attention_plan(R(s), H, Hkv, hd, B.AIO_BF16, out) == B.AIO_ERANGE
    # the largest that one launch covers
    s = B.aio_seqs((1 << 24) - 1, (1 << 24) - 1, 1 << 30, None, None, None, 0, None)
    assert L.aio_attention_plan(R(s), 1, 1, 128, B.AIO_F32, out) == B.AIO_OK and out[2] == 1
