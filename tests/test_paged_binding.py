"""What the Python binding of the operators over several sequences refuses before it calls
the library (host)."""
import contextlib
import types

import numpy as np
import pytest
import torch

import synth
from paper_2604_09752_amd import binding as B

TINY = synth.CONFIGS["tiny"]


def standing_in(**kw):
    """A model's fields without a device: what paged_forward looks at."""
    m = types.SimpleNamespace(c=B.make_config(TINY), kv=torch.zeros(1), handle=None, stream=None,
                              device=torch.device("cpu"))
    for f, v in kw.items():
        setattr(m, f, v)
    return m


def pool(device="cpu", pages=2):
    c = B.make_config(TINY)
    return torch.zeros((c.n_layers, 2, pages, c.n_kv_heads, 16, c.head_dim), dtype=torch.bfloat16,
                       device=device)


@pytest.fixture
def no_device(monkeypatch):
    """Device and stream contexts that need no device: the library refuses a null handle."""
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())


def forward(m, pool_, logits, rows=(1,), lens=(1,), table=((0,),), tokens=(1,), out_rows=(0,)):
    B.DeviceModel.paged_forward(m, pool_, rows, lens, table, tokens, out_rows, logits)


def test_a_pass_on_other_devices(no_device):
    """Logits (or a pool) elsewhere: their address means nothing to the model's device."""
    logits = torch.zeros((1, TINY.vocab))
    with pytest.raises(B.AioError):  # (as far as the library)
        forward(standing_in(), pool(), logits)
    for a, b in ((pool(), logits.to("meta")), (pool("meta"), logits)):
        with pytest.raises(ValueError, match="device"):
            forward(standing_in(), a, b)


def test_a_model_on_the_current_device(no_device):
    """A model made on "cuda" has its tensors on "cuda:0"."""
    with pytest.raises(B.AioError):
        forward(standing_in(device=torch.device("cuda")), pool(), torch.zeros((1, TINY.vocab)))


BIG = (1 << 32) + 1  # cut to 32 bits, 1


@pytest.mark.parametrize("kw", [
    dict(rows=np.array([BIG])), dict(lens=np.array([BIG])), dict(table=np.array([[BIG]])),
    dict(tokens=np.array([BIG])), dict(out_rows=np.array([BIG - 1])), dict(tokens=[1.5]),
    dict(tokens=torch.tensor([BIG])), dict(lens=np.array([BIG], np.uint64))])
def test_a_pass_over_integers_that_do_not_fit(no_device, kw):
    with pytest.raises(ValueError, match="32 bits"):
        forward(standing_in(), pool(), torch.zeros((1, TINY.vocab)), **kw)


def test_a_pass_over_integers_that_fit(no_device):
    """Any integer type, and no rows asked for."""
    for kind in (np.int64, np.uint8, np.int16):
        with pytest.raises(B.AioError):
            forward(standing_in(), pool(), torch.zeros((1, TINY.vocab)), rows=np.ones(1, kind),
                    lens=np.ones(1, kind), tokens=np.ones(1, kind), out_rows=[])


def test_copies_whose_pages_do_not_fit(monkeypatch):
    monkeypatch.setattr(B, "_device_of", lambda *t: 0)
    p = torch.zeros((2, 4, 16), dtype=torch.bfloat16)
    for src, dst in ((np.array([BIG]), [0]), ([1], np.array([BIG - 1])), ([0.5], [1])):
        with pytest.raises(ValueError, match="32 bits"):
            B.aio_page_copy(p, src, dst)


def test_sizes_that_do_not_fit():
    with pytest.raises(ValueError, match="32 bits"):
        B.aio_logprobs_workspace_bytes(BIG, 32000, 5)
    with pytest.raises(ValueError, match="32 bits"):
        B.aio_attn_workspace_bytes(1, BIG, 4096, 32, 32, 128, prompts=True)
    with pytest.raises(ValueError, match="32 bits"):
        B.Pages(BIG, 16, 1)
    p = B.Pages(4, 16, 2)
    s = p.open()
    for call in (lambda: p.extend(s, BIG), lambda: p.extend(BIG - 1, 1), lambda: p.truncate(s, BIG - 1),
                 lambda: p.close((1 << 32) + s), lambda: p.fork((1 << 32) + s),
                 lambda: p.length((1 << 32) + s), lambda: p.rows([(1 << 32) + s], 4),
                 lambda: p.rows([s], BIG + 3)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    assert p.length(s) == 0 and p.free == 4
