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


def test_counts_whose_last_step_passes_32_bits(L):
    """Rows, planes and copies go out in launches of at most 65535: past 2^31 - 2^16 the
    counter would wrap and never reach the end."""
    most, p = 0x7fff0000, 16
    for rows in (most + 1, 0x7fffffff):
        assert L.aio_logprobs_workspace_bytes(rows, 8, 2) == 0
        assert L.aio_logprobs(p, B.AIO_F32, rows, 8, 8, None, 0, None, p, None, None, None, 0,
                              None) == B.AIO_ERANGE
    one, two = (ctypes.c_int32 * 1)(0), (ctypes.c_int32 * 1)(1)
    assert L.aio_page_copy(p, most + 1, 1024, 2, 512, 512, one, two, 1, None) == B.AIO_ERANGE
    assert L.aio_page_copy(p, 1, 1024, 2, 512, 512, one, two, most + 1, None) == B.AIO_ERANGE


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


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales_that_overflow_in_units_of_log2(L, scale):
    """Finite, but not times log2 e: a score of 0 would come out NaN."""
    kv = B.aio_paged_kv(1 << 20, 1 << 30, 8 * 16 * 64, 16 * 64, 10, 16, 8, 64)
    s = B.aio_seqs(4, 4, 100, None, 16, 16, 8, None)
    a = B.aio_attn(16, 16, None, 16 * 64, 16 * 64, B.AIO_F32, 16, scale)
    assert L.aio_paged_attention(R(kv), R(s), R(a), 16, 1 << 30, None) == B.AIO_EINVAL
