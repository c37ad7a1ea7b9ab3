"""8-bit pools whose codes, bytes, K or V take each other's place are refused by the append,
in whichever page and head they meet, and no others (host)."""
import ctypes
import random

import pytest

from paper_2604_09752_amd import binding as B

R = ctypes.byref
SIZE, HD = 16, 64            # positions of a page
CODES = SIZE * HD            # bytes of a head's codes in a page
BASE = 1 << 20


@pytest.fixture(scope="module")
def L():
    return B.lib()


def pool(k, v, ke, ve, page, head, exp_page, exp_head, pages, heads):
    return B.aio_q8_kv(k, v, ke, ve, page, head, exp_page, exp_head, pages, SIZE, heads, HD)


def refused(L, kv):
    """Without rows nothing is enqueued, and the pool is looked at all the same."""
    rc = L.aio_q8_append(R(kv), R(B.aio_seqs(0, 0, 100, None, None, None, 0, None)), None, None,
                         B.AIO_F32, 512, 64, None)
    assert rc in (B.AIO_OK, B.AIO_EINVAL)
    return rc != B.AIO_OK


def overlaps(kv):
    """By the starts of all blocks, in order."""
    at = []
    for base, page, head, size in ((kv.k_dev, kv.page_stride, kv.head_stride, CODES),
                                   (kv.v_dev, kv.page_stride, kv.head_stride, CODES),
                                   (kv.k_exp_dev, kv.exp_page_stride, kv.exp_head_stride, SIZE),
                                   (kv.v_exp_dev, kv.exp_page_stride, kv.exp_head_stride, SIZE)):
        at += [(base + i * page + j * head, size) for i in range(kv.n_pages)
               for j in range(kv.n_kv_heads)]
    at.sort()
    return any(a + n > b for (a, n), (b, _) in zip(at, at[1:]))


FAR = dict(v=1 << 30, ke=1 << 40, ve=1 << 41, page=8 * CODES, head=CODES, exp_page=8 * SIZE,
           exp_head=SIZE, pages=10, heads=8)


@pytest.mark.parametrize("change", [
    dict(ke=BASE + CODES),                       # the bytes in head 1's codes of the first page
    dict(ve=BASE + 8 * CODES + 64),              # ... in page 1's
    dict(ke=(1 << 30) + 5 * 8 * CODES + 3 * CODES),
    dict(ve=BASE + 80 * CODES - 16),             # ... in the last codes
    dict(ke=BASE - 80 * SIZE + 16),              # the last bytes in the first codes
    dict(v=BASE + 8 * CODES + CODES),            # V's first head is K's second of page 1
    dict(ve=(1 << 40) + 9 * SIZE),               # ... of the bytes
    dict(v=BASE + 79 * CODES), dict(ve=(1 << 40) + 79 * SIZE),
])
def test_bytes_and_values_inside_codes(L, change):
    assert not refused(L, pool(BASE, **FAR))
    kv = pool(BASE, **dict(FAR, **change))
    assert overlaps(kv) and refused(L, kv)


def test_layouts_that_do_not_overlap(L):
    P, H, one, all_ = 6, 5, CODES, 6 * 5 * CODES
    layouts = [
        # one after the other
        pool(BASE, BASE + all_, BASE + 2 * all_, BASE + 2 * all_ + P * H * SIZE, H * one, one,
             H * SIZE, SIZE, P, H),
        # a page's codes and bytes of K, then those of V
        pool(BASE, BASE + H * (one + SIZE), BASE + H * one, BASE + H * (2 * one + SIZE),
             2 * H * (one + SIZE), one, 2 * H * (one + SIZE), SIZE, P, H),
        # a head's codes and bytes beside one another, heads of K and V in turn
        pool(BASE, BASE + one + SIZE, BASE + one, BASE + 2 * one + SIZE, 2 * H * (one + SIZE),
             2 * (one + SIZE), 2 * H * (one + SIZE), 2 * (one + SIZE), P, H),
        # all pages of a head, then the next head's
        pool(BASE, BASE + P * (one + SIZE), BASE + P * one, BASE + P * (2 * one + SIZE), one,
             2 * P * (one + SIZE), SIZE, 2 * P * (one + SIZE), P, H),
        # all bytes of a page in the gap behind its first head's codes
        pool(BASE, 1 << 30, BASE + one, BASE + one + H * SIZE, 2 * H * one, 2 * one, 2 * H * one,
             SIZE, P, H),
    ]
    for i, kv in enumerate(layouts):
        assert not overlaps(kv) and not refused(L, kv), i
        for name in ("v_dev", "k_exp_dev", "v_exp_dev"):
            for by in (-64, -16, 16, 64):
                old = getattr(kv, name)
                setattr(kv, name, old + by)
                assert refused(L, kv) == overlaps(kv), (i, name, by)
                setattr(kv, name, old)


def test_any_layout(L):
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(6000):
        P, H = rng.randint(1, 5), rng.randint(1, 4)
        head = CODES + 16 * rng.choice([0, 1, 2, 8, 64, rng.randint(0, 300)])
        page = rng.choice([H * head, 2 * H * head, H * head + 16 * rng.randint(0, 200),
                           16 * rng.randint(0, 400)])
        same = rng.random()
        exp_head = head if same < 0.3 else SIZE + 8 * rng.choice([0, 0, 2, rng.randint(0, 200)])
        exp_page = page if same < 0.7 else H * exp_head + 8 * rng.choice([0, rng.randint(0, 300)])
        near = lambda: BASE + 16 * rng.randint(-40, 1000)
        far = [1 << 30, 1 << 31, 1 << 32]
        at = [near() if rng.random() < 0.5 else f for f in far]
        kv = pool(BASE, *at, page, head, exp_page, exp_head, P, H)
        want = overlaps(kv)
        seen[want] += 1
        assert refused(L, kv) == want, [(n, getattr(kv, n)) for n, _ in kv._fields_]
    assert min(seen.values()) > 500


def test_numbers_near_the_largest_do_not_wrap(L):
    big = (1 << 63) - 16
    kv = pool(BASE, 1 << 30, 1 << 40, 1 << 41, big, CODES, big, SIZE, (1 << 31) - 1, 8)
    assert not refused(L, kv)
    kv.k_exp_dev = BASE + CODES
    assert refused(L, kv)


def test_one_page_of_many_heads_is_compared_at_once(L):
    heads = 1 << 30
    kv = pool(BASE, BASE + CODES // 2, 1 << 61, 1 << 62, 0, 2 * CODES, 0, SIZE, 1, heads)
    assert refused(L, kv)
    kv.v_dev = BASE + CODES
    assert not refused(L, kv)
    kv.v_dev = BASE + 2 * CODES * (heads - 1) + 16
    assert refused(L, kv)
