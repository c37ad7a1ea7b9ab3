"""Pools whose pages, heads, planes or layers take each other's place are refused where
they would be written (host)."""
import ctypes
import random

import pytest

from paper_2604_09752_amd import binding as B

R = ctypes.byref


@pytest.fixture(scope="module")
def L():
    return B.lib()


def overlaps(n1, s1, n2, s2, size):
    """By the starts of all blocks."""
    at = sorted(i * s1 + j * s2 for i in range(n1) for j in range(n2))
    return any(b - a < size for a, b in zip(at, at[1:]))


def copy(L, planes, plane, pages, stride, size):
    """AIO_EINVAL, or AIO_ERANGE for the page id alone, which is looked at last."""
    a, b = (ctypes.c_int32 * 1)(pages), (ctypes.c_int32 * 1)(0)
    return L.aio_page_copy(1 << 20, planes, plane, pages, stride, size, a, b, 1, None)


def test_planes_and_pages_of_a_copy(L):
    rng = random.Random(3)
    seen = set()
    for _ in range(4000):
        planes, pages = rng.randint(1, 9), rng.randint(2, 12)
        size = 16 * rng.randint(1, 4)
        stride = size + 16 * rng.choice([0, 0, 1, 3, rng.randint(0, 40)])
        plane = 16 * rng.choice([0, 1, rng.randint(0, 60), pages * stride // 16, size // 16])
        want = overlaps(planes, plane, pages, stride, size)
        seen.add(want)
        got = copy(L, planes, plane, pages, stride, size)
        assert got == (B.AIO_EINVAL if want else B.AIO_ERANGE), (planes, plane, pages, stride, size)
    assert seen == {True, False}
    # strides near the largest number do not wrap
    big = (1 << 63) - 16
    assert copy(L, 0x7fff0000, big, 0x7fffffff, 512, 512) == B.AIO_ERANGE
    assert copy(L, 0x7fff0000, big, 0x7fffffff, big, 512) == B.AIO_EINVAL


def append(L, k=1 << 20, v=1 << 30, k_rows=16, v_rows=16, **kw):
    kv = B.aio_paged_kv(k, v, 8 * 16 * 64, 16 * 64, 10, 16, 8, 64)
    for f, x in kw.items():
        setattr(kv, f, x)
    s = B.aio_seqs(4, 4, 100, None, 16, 16, 8, None)
    return L.aio_page_append(R(kv), R(s), k_rows, v_rows, B.AIO_F32, 512, 64, None)


@pytest.mark.parametrize("kw", [
    dict(page_stride=16 * 64),                       # a page's second head is the next page's first
    dict(page_stride=4 * 16 * 64),                   # ... its fifth
    dict(head_stride=10 * 16 * 64, page_stride=2 * 16 * 64),
    dict(v=1 << 20, v_rows=32),                      # K and V in one place, different rows
    dict(v=(1 << 20) + 16),
    dict(v=(1 << 20) + 2 * 8 * 16 * 64),             # V's first page is K's second
    dict(k=(1 << 20) + 2 * 16 * 64, v=1 << 20),
])
def test_rows_that_would_fall_on_others(L, kw):
    assert append(L, **kw) == B.AIO_EINVAL
