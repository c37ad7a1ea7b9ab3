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
