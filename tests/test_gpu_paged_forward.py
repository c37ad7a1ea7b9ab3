"""A whole model over a paged pool: prompts packed into one pass, decode steps
of several sequences, forks with copies of shared pages, rejected drafts taken
back, a compaction between steps, and the answers' log probabilities, each
sequence against the oracle's decode steps of its own tokens (needs an
MI355X)."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import synth
from paper_2604_09752_amd import binding as B
from tests.gpu_cases import KV_ABS, LOGIT_TOL, log
from tests.paged_cases import logprobs64

pytestmark = pytest.mark.gpu

TINY = synth.CONFIGS["tiny"]


class Server:
    """Sequences in a pool, and the oracle's cache of each."""

    def __init__(self, cfg, n_pages=40, page=16, max_seqs=8):
        self.cfg, w = cfg, synth.make_weights(cfg)
        self.dm, self.orc = B.DeviceModel(cfg, w), oracle.OracleModel(cfg, w)
        with torch.cuda.stream(self.dm.stream):
            self.pool = self.dm.new_pool(n_pages, page)
            self.pool.fill_(float("nan"))  # nothing unwritten is ever read
        self.pages, self.width, self.page = B.Pages(n_pages, page, max_seqs), n_pages, page
        self.kv, self.toks = {}, {}
        self.worst = 0.0

    def copies(self, src, dst):
        if len(src):
            with torch.cuda.stream(self.dm.stream):
                B.aio_page_copy(self.pool.view((-1,) + self.pool.shape[2:]), src, dst)

    def open(self):
        s = self.pages.open()
        self.kv[s] = np.zeros(synth.kv_shape(self.cfg), np.uint16)
        self.toks[s] = []
        return s

    def fork(self, s):
        c = self.pages.fork(s)
        self.kv[c], self.toks[c] = self.kv[s].copy(), list(self.toks[s])
        return c

    def truncate(self, s, n):
        self.pages.truncate(s, n)
        del self.toks[s][n:]

    def close(self, s):
        self.pages.close(s)
        del self.kv[s], self.toks[s]

    def step(self, new, every_row=False):
        """new: sequence -> its next tokens.  The last (or every) row's logits of
        each, checked."""
        seqs = list(new)
        rows, out_rows, want = [], [], []
        for s in seqs:
            self.copies(*self.pages.extend(s, len(new[s])))
            for j, t in enumerate(new[s]):
                ref = self.orc.decode_step(self.kv[s], int(t), len(self.toks[s]))
                self.toks[s].append(int(t))
                if every_row or j + 1 == len(new[s]):
                    out_rows.append(sum(rows) + j)
                    want.append(ref)
            rows.append(len(new[s]))
        lens, table = self.pages.rows(seqs, self.width)
        with torch.cuda.stream(self.dm.stream):
            logits = torch.full((len(out_rows), self.cfg.vocab), float("nan"), device="cuda")
        flat = [t for s in seqs for t in new[s]]
        self.dm.paged_forward(self.pool, rows, lens, table, flat, out_rows, logits)
        self.dm.sync()
        assert self.dm.status() == 0
        got = logits.cpu().numpy()
        err = float(np.abs(got - np.stack(want)).max())
        assert err <= LOGIT_TOL, (rows, err)
        self.worst = max(self.worst, err)
        # layer 0's rows in the pages: one fp32 product of identical inputs
        pool = self.pool[0].float().cpu().numpy()
        for s in seqs:
            n = len(self.toks[s])
            _, tab = self.pages.rows([s], self.width)
            for kind in (0, 1):
                g = np.concatenate([pool[kind, p] for p in tab[0, : -(-n // self.page)]], axis=1)
                r = (self.kv[s][0, kind].astype(np.uint32) << 16).view(np.float32)[:, :n]
                g = g[:, :n]
                ok = np.abs(g - r) <= np.abs(r) * 2.0 ** -7 + KV_ABS * np.abs(r).max(-1, keepdims=True)
                assert ok.all()
        return logits, np.stack(want)

    def done(self):
        log("[%s] worst max-abs %.3e" % (self.cfg.name, self.worst))
        self.dm.close()


CASES = {
    "mha": dict(),
    "gqa_hd128": dict(n_heads=4, n_kv_heads=1, head_dim=128),
    "ragged": dict(d_model=320, ffn_dim=192, vocab=1000, n_heads=5, n_kv_heads=5),
    "one_row_lm": dict(max_verify=1),
    "wide": dict(d_model=1024, ffn_dim=2048, n_heads=8, n_kv_heads=4, head_dim=128),
}


@pytest.mark.parametrize("name", list(CASES))
def test_requests_together(name):
    cfg = TINY.with_(name="paged_" + name, prompt_len=100, n_steps=60, **CASES[name])
    sv = Server(cfg)
    rng = np.random.RandomState(5)

    def toks(n):
        return [int(t) for t in rng.randint(0, cfg.vocab, n)]

    a, b, c = sv.open(), sv.open(), sv.open()
    # three prompts of ragged lengths in one pass, every row's logits
    sv.step({a: toks(37), b: toks(1), c: toks(16)}, every_row=True)
    # a decode step of all three, then one alone
    sv.step({a: toks(1), b: toks(1), c: toks(1)})
    sv.step({b: toks(1)})
    # a fork that continues with a prompt while its parent decodes: the shared, partly
    # filled page is copied before either writes
    d = sv.fork(a)
    sv.step({a: toks(1), d: toks(9), c: toks(1)})
    sv.step({d: toks(1), a: toks(1)})
    # drafts scored and taken back
    sv.step({a: toks(5), b: toks(3)}, every_row=True)
    sv.truncate(a, len(sv.toks[a]) - 4)
    sv.truncate(b, len(sv.toks[b]) - 3)
    sv.step({b: toks(1), a: toks(1), d: toks(2)})
    # a sequence ends, the rest moves to the front
    sv.close(c)
    src, dst = sv.pages.compact()
    sv.copies(src, dst)
    e = sv.open()
    logits, want = sv.step({e: toks(20), a: toks(1), d: toks(1), b: toks(1)}, every_row=True)
    # what was answered, scored
    targets = torch.from_numpy(rng.randint(0, cfg.vocab, len(want)).astype(np.int32))
    lp, ent = torch.empty(len(want), device="cuda"), torch.empty(len(want), device="cuda")
    ids = torch.empty((len(want), 3), dtype=torch.int32, device="cuda")
    tlp = torch.empty((len(want), 3), device="cuda")
    B.aio_logprobs(logits, targets.cuda(), lp, ent, ids, tlp)
    wlp = logprobs64(torch.from_numpy(want), targets, 3)[0]
    # logits within e of the oracle's move a log probability by at most 2 e
    assert (lp.double().cpu() - wlp).abs().max() <= 2 * LOGIT_TOL
    assert torch.equal(ids[:, 0].cpu(), logits.argmax(-1).int().cpu())
    sv.done()


def test_the_handles_own_cache_is_untouched():
    cfg = TINY.with_(name="paged_own", prompt_len=20, n_steps=8)
    dm = B.DeviceModel(cfg, synth.make_weights(cfg), kv_init=synth.make_kv(cfg))
    before = dm.kv_numpy().copy()
    with torch.cuda.stream(dm.stream):
        pool, logits = dm.new_pool(4), dm.new_logits(2)
    dm.paged_forward(pool, [3, 1], [3, 1], [[0, -1], [2, -1]], [1, 2, 3, 4], [2, 3], logits)
    dm.sync()
    assert np.array_equal(before, dm.kv_numpy())
    # pages that no sequence holds are untouched too
    assert not pool[:, :, [1, 3]].any() and pool[:, :, [0, 2]].any()
    dm.close()


def test_a_prompt_equals_prefill():
    """int8 weights, a prompt of 300 tokens: the same products as aio_prefill, and
    another attention kernel (fp32 level): logits within the int8 bound."""
    cfg = TINY.with_(name="paged_int8", prompt_len=300, n_steps=8, wfmt="int8")
    dm = B.DeviceModel(cfg, synth.make_weights(cfg))
    t = [int(x) for x in synth.make_prompt(cfg)]
    with torch.cuda.stream(dm.stream):
        one, two, pool = dm.new_logits(1), dm.new_logits(1), dm.new_pool(20)
    dm.prefill(t, 0, one[0])
    dm.paged_forward(pool, [300], [300], [list(range(19))], t, [299], two)
    dm.sync()
    a, b = one[0].cpu().numpy(), two[0].cpu().numpy()
    tol = max(LOGIT_TOL, 5e-3 * float(np.sqrt((a.astype(np.float64) ** 2).mean())))
    assert np.abs(a - b).max() <= tol
    dm.close()


def test_refusals():
    cfg = TINY.with_(name="paged_refuse", prompt_len=20, n_steps=8)
    dm = B.DeviceModel(cfg, synth.make_weights(cfg))
    with torch.cuda.stream(dm.stream):
        pool, logits = dm.new_pool(4), dm.new_logits(4)
    dm.sync()
    ok = dict(rows=[2, 1], lens=[2, 17], table=[[0, -1], [1, 2]], tokens=[1, 2, 3], out_rows=[1, 2])

    def code(**kw):
        with pytest.raises(B.AioError) as e:
            dm.paged_forward(pool, **{**ok, **kw}, logits=logits)
        return e.value.code

    assert code(rows=[-1, 4]) == B.AIO_ERANGE
    assert code(rows=[0, 0], tokens=[]) == B.AIO_ERANGE
    assert code(lens=[1, 17]) == B.AIO_ERANGE            # fewer keys than rows
    assert code(lens=[2, 33]) == B.AIO_ERANGE            # past the table
    assert code(lens=[2, cfg.max_ctx + 1], table=[[0] * 40, [1] * 40]) == B.AIO_ERANGE
    assert code(tokens=[1, 2, cfg.vocab]) == B.AIO_ERANGE
    assert code(tokens=[1, -2, 3]) == B.AIO_ERANGE
    assert code(out_rows=[3]) == B.AIO_ERANGE and code(out_rows=[-1]) == B.AIO_ERANGE
    assert code(table=[[4, -1], [1, 2]]) == B.AIO_ERANGE   # no such page
    assert code(table=[[-1, 0], [1, 2]]) == B.AIO_ERANGE   # a new token in a hole
    assert code(table=[[2, -1], [1, 2]]) == B.AIO_EINVAL   # both would write page 2
    assert code(rows=[1, 2], lens=[1, 17], table=[[0, -1], [1, 1]]) == B.AIO_EINVAL  # one page twice
    assert code(rows=[0, 2049], lens=[0, 2049], table=[[0] * 200] * 2,
                tokens=[0] * 2049) == B.AIO_ERANGE
    for bad in (dict(tokens=[1]), dict(table=[[0, 1]]), dict(lens=[1])):
        with pytest.raises(ValueError):
            dm.paged_forward(pool, **{**ok, **bad}, logits=logits)
    with pytest.raises(ValueError):
        dm.paged_forward(pool[:1], **ok, logits=logits)
    # and a good call after all of them: a hole before the first new token is allowed
    dm.paged_forward(pool, [1, 1], [1, 17], [[0, -1], [-1, 2]], [1, 2], [0, 1], logits)
    dm.sync()
    assert torch.isfinite(logits[:2]).all()
    # scratch: its size, its alignment
    L, P = B.lib(), ctypes.byref
    assert B.lib().aio_paged_forward_bytes(P(dm.c), 0, 1, 1) == 0
    assert B.lib().aio_paged_forward_bytes(P(dm.c), 1, 2049, 1) == 0
    kv = B.aio_paged_kv(pool.data_ptr(), pool[0, 1].data_ptr(), pool.stride(2), pool.stride(3), 4,
                        16, cfg.n_kv_heads, cfg.head_dim)
    p = B.aio_paged_pool(kv, pool.stride(0), cfg.n_layers)
    i = [np.array(x, np.int32) for x in ([1], [1], [0], [5], [0])]
    need = B.lib().aio_paged_forward_bytes(P(dm.c), 1, 1, 1)
    s = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    base = (s.data_ptr() + 255) // 256 * 256

    def raw(pool_=p, scratch=base, nbytes=need, lg=logits.data_ptr()):
        return L.aio_paged_forward(dm.handle, P(pool_), 1, i[0].ctypes.data, i[1].ctypes.data,
                                   i[2].ctypes.data, 1, i[3].ctypes.data, i[4].ctypes.data, 1, lg,
                                   scratch, nbytes)

    assert raw(nbytes=need - 256) == B.AIO_EINVAL and raw(scratch=base + 16) == B.AIO_EINVAL
    assert raw(lg=None) == B.AIO_EINVAL and raw(scratch=None) == B.AIO_EINVAL
    for change in (dict(n_layers=1), dict(layer_stride=-8), dict(layer_stride=3)):
        q = B.aio_paged_pool(kv, p.layer_stride, p.n_layers)
        for f, v in change.items():
            setattr(q, f, v)
        assert raw(pool_=q) == B.AIO_EINVAL
    kv2 = B.aio_paged_kv(kv.k_dev, kv.v_dev, kv.page_stride, kv.head_stride, 4, 16,
                         cfg.n_kv_heads + 1, cfg.head_dim)
    assert raw(pool_=B.aio_paged_pool(kv2, p.layer_stride, p.n_layers)) == B.AIO_EINVAL
    kv2 = B.aio_paged_kv(kv.k_dev, kv.v_dev, kv.page_stride, kv.head_stride, 4, 12,
                         cfg.n_kv_heads, cfg.head_dim)
    assert raw(pool_=B.aio_paged_pool(kv2, p.layer_stride, p.n_layers)) == B.AIO_EUNSUPPORTED
    assert raw() == B.AIO_OK
    dm.sync()
    dm.close()
