"""Which kernel attention of groups takes, and how it is split (host): both sides of each
rule, and the cases that the tests of the kernels mean to reach."""
import ctypes

import pytest

from paper_2604_09752_amd import binding as B

F32, BF16 = B.AIO_F32, B.AIO_BF16


def plan(n_seqs, n_rows, max_len, groups, prefix, H, Hkv, hd, dtype, prompts, key_bytes=2):
    """(waves, wide, shared splits, own splits, workgroups of the shared part)"""
    s = B.aio_seqs(n_seqs, n_rows, max_len, 16 if prompts else None, None, None, 0, None)
    x = B.aio_prefixes(groups, prefix, None, None)
    out = (ctypes.c_int32 * 5)()
    rc = B.lib().aio_groups_attention_plan(ctypes.byref(s), ctypes.byref(x), H, Hkv, hd, dtype,
                                           key_bytes, out)
    return tuple(out) if rc == B.AIO_OK else rc


def test_one_token_each():
    # from 48 columns per group on (12 rows of 4 heads), bf16 queries take rows
    assert plan(11, 11, 8700, 1, 8192, 32, 8, 128, BF16, False)[1] == 0
    assert plan(12, 12, 8700, 1, 8192, 32, 8, 128, BF16, False)[1] == 1
    assert plan(12, 12, 8700, 2, 8192, 32, 8, 128, BF16, False)[1] == 0
    assert plan(48, 48, 8700, 1, 8192, 32, 8, 128, F32, False)[1] == 0
    assert plan(48, 48, 8685, 1, 8192, 32, 8, 128, BF16, False, 1)[1] == 1
    # a shared workgroup per CU: 2 tiles of 8 heads, 16 splits
    assert plan(48, 48, 8685, 1, 8192, 32, 8, 128, BF16, False) == (0, 1, 16, 1, 256)
    # splits of at least 128 keys, up to 1024 workgroups of either part; own keys by what lies
    # beyond the prefix, four where that is less
    assert plan(3, 3, 742, 1, 700, 16, 8, 128, F32, False) == (0, 0, 6, 4, 48)
    assert plan(4, 4, 8192, 1, 4096, 32, 8, 128, F32, False) == (0, 0, 32, 32, 512)
    assert plan(4, 4, 128, 1, 64, 32, 8, 128, F32, False)[2:4] == (1, 1)


def test_prompt_rows():
    # one round of two workgroups per CU, own tiles among them
    waves, wide, S, own, groups = plan(20, 400, 4180, 1, 4096, 16, 8, 128, BF16, True)
    assert (waves, wide, own) == (4, 0, 1) and groups == 7 * 8 * S and groups + 26 * 8 <= 512
    # fp32 queries: one per CU
    S32 = plan(20, 400, 4180, 1, 4096, 16, 8, 128, F32, True)[2]
    assert S32 < S and 7 * 8 * S32 <= 256
    # (tests of the kernels)
    for key_bytes in (1, 2):
        assert plan(3, 2160, 1400, 1, 490, 128, 16, 64, BF16, True, key_bytes)[0] == 8
    assert plan(43, 43, 826, 1, 688, 8, 2, 128, BF16, False)[1] == 1
    assert plan(26, 26, 308, 2, 299, 8, 2, 64, BF16, False)[1] == 1
    assert plan(14, 14, 420, 1, 384, 4, 1, 64, BF16, False)[1] == 1


@pytest.mark.parametrize("groups,prefix,max_len", [(0, 500, 600), (2, 63, 600), (2, 0, 600),
                                                   (2, 500, 63)])
def test_nothing_to_share(groups, prefix, max_len):
    assert plan(4, 4, max_len, groups, prefix, 8, 2, 64, F32, False)[2] == 0
    assert plan(4, 40, max_len, groups, prefix, 8, 2, 64, F32, True)[2] == 0


def test_eight_bit_prompts_in_tiles_of_256():
    def waves(n_seqs, n_rows, H, Hkv, dtype, key_bytes=1):
        return plan(n_seqs, n_rows, 4000, 0, 0, H, Hkv, 128, dtype, True, key_bytes)[0]

    # from half a tile of rows per sequence and 4096 rows x heads on
    assert waves(6, 384, 16, 8, BF16) == 8 and waves(6, 383, 16, 8, BF16) == 4
    assert waves(1, 256, 16, 8, BF16) == 8 and waves(1, 255, 16, 8, BF16) == 4
    assert waves(6, 384, 16, 8, F32) == 4 and waves(6, 384, 16, 8, BF16, 2) == 4


def test_rejects():
    assert plan(4, 4, 600, -1, 500, 8, 2, 64, F32, False) == B.AIO_ERANGE
    assert plan(4, 4, 600, 1, 500, 8, 3, 64, F32, False) == B.AIO_EINVAL
    assert plan(4, 4, 600, 1, 500, 8, 2, 96, F32, False) == B.AIO_EUNSUPPORTED
    out = (ctypes.c_int32 * 5)()
    assert B.lib().aio_groups_attention_plan(None, None, 8, 8, 64, 0, 2, out) == B.AIO_EINVAL
