"""Timed cases of the operators that serve several sequences from one pool.

Five operators, each through the C ABI's Python binding:

* ``decode``: attention of one new token per sequence over a paged key-value
  cache (``aio_paged_attention``);
* ``prompt``: causal attention over the rows of several prompts, their keys
  packed behind one another (``aio_packed_attention``) or in pages behind a
  cached prefix (``aio_paged_attention`` with rows per sequence);
* ``append``: the new rows' keys and values into their pages
  (``aio_page_append``);
* ``copy``: pages copied in every layer, for a fork or a compaction
  (``aio_page_copy``);
* ``logprobs``: log probability of given tokens, entropy and the top
  alternatives of logit rows (``aio_logprobs``).

Heads are those of the repository's tiny, 1B-class and 7B-class decoders and
grouped layouts beside them; keys and values are N(0, 1) in bf16, queries
N(0, 1) in the type that the case names, pages of a sequence lie scattered.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

HEADS = {  # query heads, kv heads, head dimension
    "tiny": (4, 4, 64),
    "1b": (16, 8, 128),
    "7b": (32, 32, 128),
    "g4": (32, 8, 128),
    "g8": (16, 2, 64),
}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _decode(heads, n, lo, hi, page, dtype, spread, name=None):
    c = {"op": "decode", "heads": heads, "n": n, "lo": lo, "hi": hi, "page": page,
         "dtype": dtype, "spread": spread}
    return dict(c, name=name) if name else c


def _prompt(heads, n, lo, hi, prefix, page, dtype, spread, name=None):
    """``page`` 0: packed keys; else the rows follow up to ``prefix`` keys in pages."""
    c = {"op": "prompt", "heads": heads, "n": n, "lo": lo, "hi": hi, "prefix": prefix,
         "page": page, "dtype": dtype, "spread": spread}
    return dict(c, name=name) if name else c


def _append(heads, n, lo, hi, prefix, page, dtype, spread, name=None):
    c = {"op": "append", "heads": heads, "n": n, "lo": lo, "hi": hi, "prefix": prefix,
         "page": page, "dtype": dtype, "spread": spread}
    return dict(c, name=name) if name else c


def _copy(heads, layers, page, pages, copies, name=None):
    c = {"op": "copy", "heads": heads, "layers": layers, "page": page, "pages": pages,
         "copies": copies}
    return dict(c, name=name) if name else c


def _logprobs(rows, vocab, top, dtype, name=None):
    c = {"op": "logprobs", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: the 1B's next token of one short request, all latency
        _decode("1b", 1, 129, 129, 16, "fp32", 1, name="decode_one_129"),
        # a serving batch of ragged requests on a grouped-head backbone
        _decode("g4", 24, 37, 4096, 16, "bf16", 2, name="decode_batch_ragged"),
        # two requests at the long context that the backbone is kept for
        _decode("7b", 2, 32768, 32768, 64, "fp32", 3, name="decode_7b_32k"),
        # short turns of six conversations behind their cached prefixes
        _prompt("1b", 6, 3, 40, 700, 16, "fp32", 4, name="prompt_turns_paged"),
        # eight prompts of odd lengths packed into one pass
        _prompt("1b", 8, 17, 2048, 0, 0, "bf16", 5, name="prompt_packed_1b"),
        # one long prompt of the backbone
        _prompt("7b", 1, 8192, 8192, 0, 0, "bf16", 6, name="prompt_7b_8k"),
        # one token of each of 16 requests into its page
        _append("1b", 16, 1, 1, 3000, 16, "fp32", 7, name="append_step"),
        # the rows of a pass of prompts into pages
        _append("7b", 5, 100, 700, 0, 16, "fp32", 8, name="append_prompts"),
        # the last, partly filled pages of three forked requests, all layers of the 1B
        _copy("1b", 24, 16, 64, 3, name="copy_fork"),
        # a compaction: 200 pages move to the front of the pool
        _copy("1b", 24, 16, 512, 200, name="copy_compact"),
        # the chosen token's log probability with five alternatives
        _logprobs(1, 32000, 5, "fp32", name="logprobs_token"),
        # every token of a prompt scored
        _logprobs(2048, 32000, 8, "fp32", name="logprobs_prompt"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "prompt", "prompt", "append", "copy", "logprobs"])
    heads = rng.choice(sorted(HEADS))
    H, Hkv, hd = HEADS[heads]
    dtype = rng.choice(["fp32", "bf16"])
    page = rng.choice([8, 16, 32, 64, 128])
    spread = rng.randrange(1 << 30)
    if op == "decode":
        n = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, min(32768, (1 << 30) // (4 * n * Hkv * hd)))
        return _decode(heads, n, rng.randint(1, hi), hi, page, dtype, spread)
    if op == "prompt":
        n = _log_int(rng, 1, 16)
        # at most the long prompt's scores (32 heads x 8192^2); three terms per
        # product where the queries are 32 bits
        most = 32 * 8192 * 8192 // (4 if dtype == "fp32" else 1)
        hi = _log_int(rng, 1, int(math.sqrt(most / (n * H))) // 2)
        paged = rng.random() < 0.5
        prefix = _log_int(rng, 1, hi) if paged else 0
        return _prompt(heads, n, rng.randint(1, hi), hi, prefix, page if paged else 0, dtype,
                       spread)
    if op == "append":
        n = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, 2048 // n)
        return _append(heads, n, rng.randint(1, hi), hi, rng.randint(0, 500), page, dtype, spread)
    if op == "copy":
        layers = rng.choice([2, 24, 32])
        room = (400 << 20) // (layers * 2 * Hkv * page * hd * 2)
        copies = _log_int(rng, 1, min(200, room // 2))
        return _copy(heads, layers, page, copies * 2 + rng.randint(0, 30), copies)
    vocab = _log_int(rng, 500, 131072)
    rows = _log_int(rng, 1, min(4096, 2048 * 32000 // vocab))
    return _logprobs(rows, vocab, rng.randint(1, 20), dtype)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """(rows, keys) of each sequence, from the case alone."""
    rng = random.Random(case["spread"])
    n, lo, hi = case["n"], case["lo"], case["hi"]
    # the longest is among them
    size = [hi] + [rng.randint(lo, hi) for _ in range(n - 1)]
    rng.shuffle(size)
    if case["op"] == "decode":
        return [1] * n, size
    p = case["prefix"]
    return size, [s + (rng.randint(p // 2, p) if p else 0) for s in size]


def _ints(values, device):
    return torch.tensor(values, dtype=torch.int32, device=device)


def _cumulative(sizes):
    return [0] + [int(v) for v in np.cumsum(sizes)]


def _inputs(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, std=1.0):
        return torch.empty(shape, dtype=dtype, device=device).normal_(0.0, std, generator=gen)

    st = dict(case)
    if case["op"] == "logprobs":
        st["logits"] = normal(case["rows"], case["vocab"], dtype=TYPES[case["dtype"]], std=3.0)
        st["targets"] = torch.randint(0, case["vocab"], (case["rows"],), generator=gen,
                                      device=device, dtype=torch.int32)
        return st
    H, Hkv, hd = HEADS[case["heads"]]
    rs = np.random.RandomState(seed % (2 ** 32))
    if case["op"] == "copy":
        st["pool"] = normal(2 * case["layers"], case["pages"], Hkv, case["page"], hd)
        ids = rs.permutation(case["pages"]).astype(np.int32)
        st["src"], st["dst"] = ids[: case["copies"]], ids[case["copies"]: 2 * case["copies"]]
        return st
    q_len, k_len = _lengths(case)
    dtype = TYPES[case["dtype"]]
    st["rows"], st["max_rows"], st["max_len"] = sum(q_len), max(q_len), max(k_len)
    st["lens"], st["cu_q"] = _ints(k_len, device), _ints(_cumulative(q_len), device)
    if case["op"] == "append":
        st["k_rows"] = normal(st["rows"], Hkv, hd, dtype=dtype)
        st["v_rows"] = normal(st["rows"], Hkv, hd, dtype=dtype)
    else:
        st["q"] = normal(st["rows"], H, hd, dtype=dtype)
    if case["page"]:
        width = -(-max(k_len) // case["page"])
        pages = sum(-(-k // case["page"]) for k in k_len) + 3
        ids = rs.permutation(pages)
        table, at = np.zeros((case["n"], width), dtype=np.int32), 0
        for i, k in enumerate(k_len):
            own_pages = -(-k // case["page"])
            table[i, :own_pages] = ids[at: at + own_pages]
            at += own_pages
        st["table"] = torch.from_numpy(table).to(device)
        st["k"] = normal(pages, Hkv, case["page"], hd)
        st["v"] = normal(pages, Hkv, case["page"], hd)
    else:
        st["cu_k"] = _ints(_cumulative(k_len), device)
        st["k"] = normal(sum(k_len), Hkv, hd)
        st["v"] = normal(sum(k_len), Hkv, hd)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    device = torch.device("cuda", torch.cuda.current_device())
    if case["op"] == "logprobs":
        rows, top = case["rows"], case["top"]
        st["logprob"] = torch.empty(rows, dtype=torch.float32, device=device)
        st["entropy"] = torch.empty(rows, dtype=torch.float32, device=device)
        st["top_ids"] = torch.empty((rows, top), dtype=torch.int32, device=device)
        st["top_logprobs"] = torch.empty((rows, top), dtype=torch.float32, device=device)
    elif "q" in st:
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device=device)
    return st


# ------------------------------------------------------------- the plain form

def _padded_rows(st):
    """Row index of each (sequence, row), and which of them exist."""
    first, q_len = st["cu_q"][:-1].long(), (st["cu_q"][1:] - st["cu_q"][:-1]).long()
    j = torch.arange(st["max_rows"], device=first.device)
    live = j[None, :] < q_len[:, None]
    return (first[:, None] + j[None, :]).clamp_(max=st["rows"] - 1), live, q_len


def _padded_keys(st, x):
    """[n, Hkv, max_len, hd] in fp32 from packed or paged rows."""
    j = torch.arange(st["max_len"], device=x.device)
    if "table" in st:
        page = st["table"].long()[:, j // st["page"]]
        rows = x[page, :, j % st["page"]]
    else:
        rows = x[(st["cu_k"][:-1].long()[:, None] + j[None, :]).clamp_(max=x.shape[0] - 1)]
    return rows.float().transpose(1, 2).contiguous()


def _plain_attention(st):
    q, n = st["q"], st["n"]
    H, Hkv, hd = HEADS[st["heads"]]
    G, R, T = H // Hkv, st["max_rows"], st["max_len"]
    idx, live, q_len = _padded_rows(st)
    qp = q.float()[idx].view(n, R, Hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * R, hd)
    k, v = _padded_keys(st, st["k"]), _padded_keys(st, st["v"])
    s = torch.matmul(qp, k.transpose(2, 3).contiguous()).view(n, Hkv, G, R, T)
    s *= 1.0 / math.sqrt(hd)
    last = (st["lens"].long() - q_len)[:, None] + torch.arange(R, device=q.device)
    hidden = torch.arange(T, device=q.device) > last[:, :, None]
    s.masked_fill_(hidden[:, None, None], -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    p = s.sub_(m).exp_()
    z = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(n, Hkv, G * R, T), v).view(n, Hkv, G, R, hd) / z
    lse = m.squeeze(-1) + z.squeeze(-1).log()
    o = o.permute(0, 3, 1, 2, 4).reshape(n, R, H, hd)
    lse = lse.permute(0, 3, 1, 2).reshape(n, R, H)
    return {"out": o[live].to(q.dtype), "lse": lse[live]}


def _plain_append(st):
    idx, live, q_len = _padded_rows(st)
    pos = (st["lens"].long() - q_len)[:, None] + torch.arange(st["max_rows"], device=idx.device)
    pos = pos.clamp_(min=0, max=st["max_len"] - 1)
    page = st["table"].long().gather(1, pos // st["page"])[live]
    slot, rows = (pos % st["page"])[live], idx[live]
    st["k"][page, :, slot] = st["k_rows"][rows].to(torch.bfloat16)
    st["v"][page, :, slot] = st["v_rows"][rows].to(torch.bfloat16)
    return {"k": st["k"], "v": st["v"]}


def _plain_copy(st):
    pool = st["pool"]
    src = torch.from_numpy(st["src"]).to(pool.device).long()
    dst = torch.from_numpy(st["dst"]).to(pool.device).long()
    pool[:, dst] = pool[:, src]
    return {"pool": pool}


def _plain_logprobs(st):
    x = st["logits"].float()
    m = x.amax(dim=-1, keepdim=True)
    d = x - m
    e = d.exp()
    z = e.sum(dim=-1, dtype=torch.float64)
    logz = z.log()
    entropy = logz - (e * d).sum(dim=-1, dtype=torch.float64) / z
    at = d.gather(1, st["targets"].long()[:, None]).squeeze(1)
    val, ids = x.sort(dim=-1, descending=True, stable=True)
    top = (val[:, : st["top"]] - m).double() - logz[:, None]
    return {"logprob": (at.double() - logz).float(), "entropy": entropy.float(),
            "top_ids": ids[:, : st["top"]].to(torch.int32), "top_logprobs": top.float()}


def run(state):
    op = state["op"]
    if own:
        from paper_2604_09752_amd import binding as aio
        if op == "decode":
            aio.aio_paged_attention(state["q"], state["k"], state["v"], state["lens"],
                                    state["table"], state["out"], lse=state["lse"],
                                    max_len=state["max_len"])
            return {"out": state["out"], "lse": state["lse"]}
        if op == "prompt":
            if state["page"]:
                aio.aio_paged_attention(state["q"], state["k"], state["v"], state["lens"],
                                        state["table"], state["out"], cu_q=state["cu_q"],
                                        lse=state["lse"], max_len=state["max_len"])
            else:
                aio.aio_packed_attention(state["q"], state["k"], state["v"], state["cu_q"],
                                         state["cu_k"], state["out"], lse=state["lse"],
                                         max_len=state["max_len"])
            return {"out": state["out"], "lse": state["lse"]}
        if op == "append":
            aio.aio_page_append(state["k_rows"], state["v_rows"], state["k"], state["v"],
                                state["lens"], state["table"], cu_q=state["cu_q"])
            return {"k": state["k"], "v": state["v"]}
        if op == "copy":
            aio.aio_page_copy(state["pool"], state["src"], state["dst"])
            return {"pool": state["pool"]}
        aio.aio_logprobs(state["logits"], state["targets"], state["logprob"], state["entropy"],
                         state["top_ids"], state["top_logprobs"])
        return {f: state[f] for f in ("logprob", "entropy", "top_ids", "top_logprobs")}
    if op in ("decode", "prompt"):
        return _plain_attention(state)
    return {"append": _plain_append, "copy": _plain_copy, "logprobs": _plain_logprobs}[op](state)


# ------------------------------------------------------------ bytes and flops

def work(case):
    size = 4 if case.get("dtype") == "fp32" else 2
    if case["op"] == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * (12 + 8 * case["top"]), "flops": 6 * n}
    H, Hkv, hd = HEADS[case["heads"]]
    if case["op"] == "copy":
        moved = 2 * case["layers"] * case["copies"] * Hkv * case["page"] * hd * 2
        return {"bytes": 2 * moved + 8 * case["copies"], "flops": 0}
    q_len, k_len = _lengths(case)
    rows, keys = sum(q_len), sum(k_len)
    index = 4 * (len(q_len) * 2 + 1)
    if case["page"]:
        index += 4 * sum(-(-k // case["page"]) for k in k_len)
    if case["op"] == "append":
        # only the pages that the rows fall on are looked up
        index = 4 * (len(q_len) * 2 + 1) + 4 * sum(q // case["page"] + 1 for q in q_len)
        return {"bytes": 2 * rows * Hkv * hd * (size + 2) + index, "flops": 0}
    seen = sum(q * k - q * (q - 1) // 2 for q, k in zip(q_len, k_len))
    return {"bytes": 2 * keys * Hkv * hd * 2 + rows * H * (2 * hd * size + 4) + index,
            "flops": 4 * H * hd * seen}


# --------------------------------------------------------- 64-bit evaluation

def _exact_attention(st):
    H, Hkv, hd = HEADS[st["heads"]]
    G, f64 = H // Hkv, torch.float64
    q_len, k_len = _lengths(st)
    out = torch.empty(st["q"].shape, dtype=f64, device=st["q"].device)
    lse = torch.empty(st["q"].shape[:2], dtype=f64, device=st["q"].device)
    r0 = t0 = 0
    for i, (nq, nk) in enumerate(zip(q_len, k_len)):
        if st["page"]:
            pages = st["table"][i, : -(-nk // st["page"])].long()
            k = st["k"][pages].transpose(1, 2).reshape(-1, Hkv, hd)[:nk]
            v = st["v"][pages].transpose(1, 2).reshape(-1, Hkv, hd)[:nk]
        else:
            k, v = st["k"][t0: t0 + nk], st["v"][t0: t0 + nk]
        above = (torch.arange(nk, device=k.device)[None, :] >
                 torch.arange(nk - nq, nk, device=k.device)[:, None])
        for h in range(H):
            s = st["q"][r0: r0 + nq, h].to(f64) @ k[:, h // G].to(f64).t()
            s = (s / math.sqrt(hd)).masked_fill_(above, -math.inf)
            lse[r0: r0 + nq, h] = torch.logsumexp(s, dim=-1)
            out[r0: r0 + nq, h] = torch.softmax(s, dim=-1) @ v[:, h // G].to(f64)
        r0, t0 = r0 + nq, t0 + nk
    return {"out": out, "lse": lse}


def _exact_append(st):
    q_len, k_len = _lengths(st)
    k, v = st["k"].to(torch.float64), st["v"].to(torch.float64)
    table, row = st["table"].cpu().tolist(), 0
    where = []
    for i, (nq, nk) in enumerate(zip(q_len, k_len)):
        where += [(table[i][p // st["page"]], p % st["page"]) for p in range(nk - nq, nk)]
        row += nq
    page = torch.tensor([w[0] for w in where], device=k.device)
    slot = torch.tensor([w[1] for w in where], device=k.device)
    for h in range(k.shape[1]):
        k[page, h, slot] = st["k_rows"][:, h].to(torch.float64)
        v[page, h, slot] = st["v_rows"][:, h].to(torch.float64)
    return {"k": k, "v": v}


def _exact_copy(st):
    pool = st["pool"].to(torch.float64)
    out = pool.clone()
    for a, b in zip(st["src"].tolist(), st["dst"].tolist()):
        out[:, b] = pool[:, a]
    return {"pool": out}


def _exact_logprobs(st):
    lp, ent, ids, top = [], [], [], []
    for x, t in zip(st["logits"].split(64), st["targets"].split(64)):
        x = x.to(torch.float64)
        y = torch.log_softmax(x, dim=-1)
        lp.append(y[torch.arange(len(t), device=x.device), t.long()])
        ent.append(-(y.exp() * y).sum(dim=-1))
        # by value, then by index
        order = torch.argsort(-x, dim=-1, stable=True)[:, : st["top"]]
        ids.append(order.to(torch.int32))
        top.append(y.gather(1, order))
    return {"logprob": torch.cat(lp), "entropy": torch.cat(ent), "top_ids": torch.cat(ids),
            "top_logprobs": torch.cat(top)}


def exact(case, seed):
    st = _inputs(case, seed)
    return {"decode": _exact_attention, "prompt": _exact_attention, "append": _exact_append,
            "copy": _exact_copy, "logprobs": _exact_logprobs}[case["op"]](st)
