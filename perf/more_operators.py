"""Timed cases of the 8-bit paged cache, of attention behind shared prefixes and of the
norm and rotation of query and key rows.

Four operators, each through the C ABI's Python binding:

* ``append``: new rows' keys and values into 8-bit pages (``aio_q8_append``);
* ``attend``: attention over 8-bit pages, of one new token per sequence or of the rows of
  prompts behind what the pages hold (``aio_q8_attention``);
* ``prefix``: the same for groups of sequences that share a prefix, which is read once per
  group, over bf16 pages (``aio_prefix_attention``) or 8-bit ones
  (``aio_q8_prefix_attention``);
* ``norm``: RMS norm of each query and key head and the rotation by position
  (``aio_qk_norm_rope``).

An 8-bit page holds each head's row of a position as int8 codes and one byte b: the values
are code * 2^(b - 127), b the least for which no code passes 127 (at least 8); b = 255 stands
for a row that held something not finite.  Codes and bytes are whole numbers: where they are
equal, so are the values.

Heads are those of the repository's tiny, 1B-class and 7B-class decoders and grouped
layouts beside them; keys and values are N(0, 1), queries N(0, 1) in the type that the
case names, pages of a sequence lie scattered.
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
EPS, BASE = 1e-5, 10000.0


def _append(heads, n, lo, hi, prefix, page, dtype, spread, name=None):
    """n sequences append lo..hi rows each behind up to ``prefix`` keys."""
    c = {"op": "append", "heads": heads, "n": n, "lo": lo, "hi": hi, "prefix": prefix,
         "page": page, "dtype": dtype, "spread": spread}
    return dict(c, name=name) if name else c


def _attend(heads, n, lo, hi, rows, page, dtype, spread, name=None):
    """n sequences of lo..hi keys; ``rows`` 0: one new token each, else up to so many rows."""
    c = {"op": "attend", "heads": heads, "n": n, "lo": lo, "hi": hi, "rows": rows,
         "page": page, "dtype": dtype, "spread": spread}
    return dict(c, name=name) if name else c


def _prefix(heads, n, groups, prefix, rest, rows, page, pool, dtype, spread, name=None):
    """n sequences in groups, each group behind a prefix of up to ``prefix`` keys of its own
    (the longest is that), every sequence with 1..rest keys more; ``rows`` as above."""
    c = {"op": "prefix", "heads": heads, "n": n, "groups": groups, "prefix": prefix,
         "rest": rest, "rows": rows, "page": page, "pool": pool, "dtype": dtype,
         "spread": spread}
    return dict(c, name=name) if name else c


def _norm(heads, rows, far, dtype, name=None):
    """Positions below ``far``."""
    c = {"op": "norm", "heads": heads, "rows": rows, "far": far, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of each of 16 requests into its page
        _append("1b", 16, 1, 1, 3000, 16, "fp32", 1, name="q8_append_step"),
        # the rows of a pass of prompts into pages
        _append("7b", 5, 100, 700, 0, 16, "fp32", 2, name="q8_append_prompts"),
        # the 1B's next token of one short request, all latency
        _attend("1b", 1, 201, 201, 0, 16, "fp32", 3, name="q8_decode_one_201"),
        # a serving batch of ragged requests on a grouped-head backbone
        _attend("g4", 24, 37, 4096, 0, 16, "bf16", 4, name="q8_decode_batch_ragged"),
        # two requests at the long context that the backbone is kept for
        _attend("7b", 2, 32768, 32768, 0, 64, "fp32", 5, name="q8_decode_7b_32k"),
        # continued prompts of six conversations behind what their pages hold
        _attend("1b", 6, 700, 3900, 900, 16, "bf16", 6, name="q8_prompt_turns"),
        # three forks of a template, a few tokens in, on the 1B
        _prefix("1b", 3, 1, 700, 60, 0, 16, "bf16", "fp32", 7, name="prefix_forks"),
        # a full batch behind one long template
        _prefix("g4", 48, 1, 8192, 500, 0, 16, "bf16", "bf16", 8, name="prefix_batch"),
        # the backbone's requests behind the templates of three task categories, in 8 bits
        _prefix("7b", 24, 3, 16384, 900, 0, 32, "q8", "fp32", 9, name="prefix_categories_q8"),
        # the first rows of twenty requests behind one template
        _prefix("1b", 20, 1, 4096, 90, 40, 16, "bf16", "bf16", 10, name="prefix_turns"),
        # one token of each of 8 requests of the 1B
        _norm("1b", 8, 4096, "fp32", name="norm_step"),
        # the rows of a pass of prompts on a grouped-head backbone
        _norm("g4", 4096, 32768, "bf16", name="norm_prompts"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "prefix", "prefix", "prefix", "norm"])
    heads = rng.choice(sorted(HEADS))
    H, Hkv, hd = HEADS[heads]
    dtype = rng.choice(["fp32", "bf16"])
    page = rng.choice([8, 16, 32, 64, 128])
    spread = rng.randrange(1 << 30)
    if op == "append":
        n = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, 2048 // n)
        return _append(heads, n, rng.randint(1, hi), hi, rng.randint(0, 500), page, dtype, spread)
    if op == "attend":
        n = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, min(32768, (1 << 28) // (n * Hkv * hd)))
        rows = 0
        if rng.random() < 0.4:
            # at most 2^31 scores; three terms per product where the queries are 32 bits
            most = (1 << 31) // (n * H * hi) // (4 if dtype == "fp32" else 1)
            rows = _log_int(rng, 1, max(1, min(hi, most, 2048)))
        return _attend(heads, n, rng.randint(1, hi), hi, rows, page, dtype, spread)
    if op == "prefix":
        n = _log_int(rng, 1, 64)
        groups = rng.randint(1, min(n, 4))
        rest = _log_int(rng, 1, 1000)
        prefix = _log_int(rng, 16, min(32768, (1 << 31) // (n * Hkv * hd)))
        rows = 0
        if rng.random() < 0.3:
            most = (1 << 31) // (n * H * (prefix + rest)) // (4 if dtype == "fp32" else 1)
            rows = _log_int(rng, 1, max(1, min(rest, most, 512)))
        return _prefix(heads, n, groups, prefix, rest, rows, page, rng.choice(["bf16", "q8"]),
                       dtype, spread)
    return _norm(heads, _log_int(rng, 1, 4096), _log_int(rng, 1, 131072), dtype)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """(rows, keys, prefix, first of its group) of each sequence, from the case alone."""
    rng = random.Random(case["spread"])
    n = case["n"]
    if case["op"] == "append":
        rows = [case["hi"]] + [rng.randint(case["lo"], case["hi"]) for _ in range(n - 1)]
        rng.shuffle(rows)
        p = case["prefix"]
        return rows, [r + rng.randint(p // 2, p) for r in rows], [0] * n, list(range(n))
    if case["op"] == "attend":
        keys = [case["hi"]] + [rng.randint(case["lo"], case["hi"]) for _ in range(n - 1)]
        rng.shuffle(keys)
        prefix, first = [0] * n, list(range(n))
        most = keys
    else:
        cuts = sorted(rng.sample(range(1, n), case["groups"] - 1))
        first = [max([0] + [c for c in cuts if c <= i]) for i in range(n)]
        long = {c: rng.randint(-(-case["prefix"] // 2), case["prefix"]) for c in [0] + cuts}
        long[rng.choice(sorted(long))] = case["prefix"]
        prefix = [long[f] for f in first]
        rest = [rng.randint(1, case["rest"]) for _ in range(n)]
        keys = [p + r for p, r in zip(prefix, rest)]
        most = rest
    if case["rows"]:
        rows = [min(m, rng.randint(1, case["rows"])) for m in most]
        i = rng.randrange(n)
        rows[i] = min(most[i], case["rows"])
    else:
        rows = [1] * n
    return rows, keys, prefix, first


def _ints(values, device):
    return torch.tensor(values, dtype=torch.int32, device=device)


def _cumulative(sizes):
    return [0] + [int(v) for v in np.cumsum(sizes)]


def _quantise(x):
    """(codes, bytes) of rows [..., head_dim]."""
    x = x.float()
    amax = x.abs().amax(dim=-1)
    m, e = torch.frexp(amax)
    e = e - 7 + (torch.round(m * 128) > 127).int()
    e = torch.where(amax > 0, e, torch.full_like(e, -119)).clamp_(-119, 121)
    code = torch.round(torch.ldexp(x, -e[..., None])).clamp_(-127, 127)
    finite = torch.isfinite(amax)
    code = torch.where(finite[..., None], code, torch.zeros_like(code))
    byte = torch.where(finite, e + 127, torch.full_like(e, 255))
    return code.to(torch.int8), byte.to(torch.uint8)


def _values(code, byte):
    scale = torch.ldexp(torch.ones_like(byte, dtype=torch.float32), byte.int() - 127)
    scale = torch.where(byte == 255, torch.full_like(scale, math.nan), scale)
    return code.float() * scale[..., None]


def _inputs(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, std=1.0):
        return torch.empty(shape, dtype=dtype, device=device).normal_(0.0, std, generator=gen)

    st = dict(case)
    H, Hkv, hd = HEADS[case["heads"]]
    dtype = TYPES[case["dtype"]]
    if case["op"] == "norm":
        n = case["rows"]
        # queries, keys and values of a row lie beside one another, as a product leaves them
        qkv = normal(n, H + 2 * Hkv, hd, dtype=dtype, std=1.5)
        st["q"], st["k"] = qkv[:, :H], qkv[:, H: H + Hkv]
        st["q_weight"] = normal(hd, std=0.1) + 1
        st["k_weight"] = normal(hd, std=0.1) + 1
        st["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device=device,
                                        dtype=torch.int32)
        return st
    q_len, k_len, prefix, first = _lengths(case)
    page, n = case["page"], case["n"]
    st["n_rows"], st["max_rows"], st["max_len"] = sum(q_len), max(q_len), max(k_len)
    st["lens"], st["cu_q"] = _ints(k_len, device), _ints(_cumulative(q_len), device)
    width = -(-max(k_len) // page)
    # full pages of a prefix are shared; the one that it ends in is a copy of each sequence's
    shared = [0 if f == i else prefix[i] // page for i, f in enumerate(first)]
    owned = [-(-k // page) - s for k, s in zip(k_len, shared)]
    pages = sum(owned) + 3
    ids = np.random.RandomState(seed % (2 ** 32)).permutation(pages)
    table, at = np.zeros((n, width), dtype=np.int32), 0
    for i in range(n):
        table[i, : shared[i]] = table[first[i], : shared[i]]
        table[i, shared[i]: shared[i] + owned[i]] = ids[at: at + owned[i]]
        at += owned[i]
    st["table"] = torch.from_numpy(table).to(device)
    q8 = case["op"] != "prefix" or case["pool"] == "q8"
    for name in "kv":
        x = normal(pages, Hkv, page, hd)
        for i in range(n):
            tail = prefix[i] % page if first[i] != i else 0
            if tail:
                x[table[i, shared[i]], :, :tail] = x[table[first[i], shared[i]], :, :tail]
        if not q8:
            st[name] = x
            continue
        done = [_quantise(part) for part in x.split(max(1, (1 << 27) // (Hkv * page * hd)))]
        st[name], st[name + "_exp"] = (torch.cat(c) for c in zip(*done))
    if case["op"] == "append":
        st["k_rows"] = normal(st["n_rows"], Hkv, hd, dtype=dtype)
        st["v_rows"] = normal(st["n_rows"], Hkv, hd, dtype=dtype)
        return st
    st["q"] = normal(st["n_rows"], H, hd, dtype=dtype)
    if case["op"] == "prefix":
        starts = sorted(set(first))
        st["cu_seqs"] = _ints(starts + [n], device)
        st["prefix_lens"] = _ints([prefix[s] for s in starts], device)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "norm":
        st["q_out"] = torch.empty(st["q"].shape, dtype=st["q"].dtype, device=st["q"].device)
        st["k_out"] = torch.empty(st["k"].shape, dtype=st["k"].dtype, device=st["k"].device)
    elif "q" in st:
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device=st["q"].device)
    return st


# ------------------------------------------------------------- the plain form

def _padded_rows(st):
    """Row index of each (sequence, row), and which of them exist."""
    first, q_len = st["cu_q"][:-1].long(), (st["cu_q"][1:] - st["cu_q"][:-1]).long()
    j = torch.arange(st["max_rows"], device=first.device)
    live = j[None, :] < q_len[:, None]
    return (first[:, None] + j[None, :]).clamp_(max=st["n_rows"] - 1), live, q_len


def _padded_keys(st, name, i, j):
    """[sequences i, Hkv, max_len, hd] in fp32 from pages."""
    page = st["table"][i].long()[:, j // st["page"]]
    rows = st[name][page, :, j % st["page"]]
    if name + "_exp" in st:
        rows = _values(rows, st[name + "_exp"][page, :, j % st["page"]])
    return rows.float().transpose(1, 2).contiguous()


def _plain_attention(st):
    q, n = st["q"], st["n"]
    H, Hkv, hd = HEADS[st["heads"]]
    G, R, T = H // Hkv, st["max_rows"], st["max_len"]
    idx, live, q_len = _padded_rows(st)
    j = torch.arange(T, device=q.device)
    out = torch.empty((n, R, H, hd), dtype=torch.float32, device=q.device)
    lse = torch.empty((n, R, H), dtype=torch.float32, device=q.device)
    # a few sequences at a time: their keys in 32 bits and their scores are written out
    step = max(1, (1 << 30) // (H * T * max(R, hd)))
    for a in range(0, n, step):
        i = slice(a, min(n, a + step))
        m = i.stop - a
        qp = q.float()[idx[i]].view(m, R, Hkv, G, hd).permute(0, 2, 3, 1, 4)
        qp = qp.reshape(m, Hkv, G * R, hd)
        k = _padded_keys(st, "k", i, j)
        s = torch.matmul(qp, k.transpose(2, 3).contiguous()).view(m, Hkv, G, R, T)
        s *= 1.0 / math.sqrt(hd)
        last = (st["lens"][i].long() - q_len[i])[:, None] + torch.arange(R, device=q.device)
        s.masked_fill_((j > last[:, :, None])[:, None, None], -math.inf)
        top = s.amax(dim=-1, keepdim=True)
        p = s.sub_(top).exp_()
        z = p.sum(dim=-1, keepdim=True)
        v = _padded_keys(st, "v", i, j)
        o = torch.matmul(p.view(m, Hkv, G * R, T), v).view(m, Hkv, G, R, hd) / z
        out[i] = o.permute(0, 3, 1, 2, 4).reshape(m, R, H, hd)
        l = top.squeeze(-1) + z.squeeze(-1).log()
        lse[i] = l.permute(0, 3, 1, 2).reshape(m, R, H)
    return {"out": out[live].to(q.dtype), "lse": lse[live]}


def _plain_append(st):
    idx, live, q_len = _padded_rows(st)
    pos = (st["lens"].long() - q_len)[:, None] + torch.arange(st["max_rows"], device=idx.device)
    pos = pos.clamp_(min=0, max=st["max_len"] - 1)
    page = st["table"].long().gather(1, pos // st["page"])[live]
    slot, rows = (pos % st["page"])[live], idx[live]
    for name in "kv":
        code, byte = _quantise(st[name + "_rows"][rows])
        st[name][page, :, slot] = code
        st[name + "_exp"][page, :, slot] = byte
    return {f: st[f] for f in ("k", "v", "k_exp", "v_exp")}


def _plain_norm(st):
    hd = st["q"].shape[2]
    i = torch.arange(hd // 2, dtype=torch.float64, device=st["q"].device)
    angle = st["positions"].double()[:, None] * torch.exp(i * (-2.0 / hd * math.log(BASE)))
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = {}
    for name in "qk":
        x = st[name].float()
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
        x = x * st[name + "_weight"].float()
        a, b = x[..., : hd // 2], x[..., hd // 2:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
        out[name] = y.to(st[name].dtype)
    return out


def run(state):
    op = state["op"]
    if own:
        from paper_2604_09752_amd import binding as aio
        if op == "norm":
            aio.aio_qk_norm_rope(state["q"], state["k"], state["positions"], state["q_out"],
                                 state["k_out"], q_weight=state["q_weight"],
                                 k_weight=state["k_weight"], eps=EPS, base=BASE)
            return {"q": state["q_out"], "k": state["k_out"]}
        if op == "append":
            aio.aio_q8_append(state["k_rows"], state["v_rows"], state["k"], state["v"],
                              state["k_exp"], state["v_exp"], state["lens"], state["table"],
                              cu_q=state["cu_q"])
            return {f: state[f] for f in ("k", "v", "k_exp", "v_exp")}
        # one new token per sequence needs no row boundaries
        cu_q = state["cu_q"] if state["rows"] else None
        if op == "attend":
            aio.aio_q8_attention(state["q"], state["k"], state["v"], state["k_exp"],
                                 state["v_exp"], state["lens"], state["table"], state["out"],
                                 cu_q=cu_q, lse=state["lse"], max_len=state["max_len"])
        elif state["pool"] == "q8":
            aio.aio_q8_prefix_attention(state["q"], state["k"], state["v"], state["k_exp"],
                                        state["v_exp"], state["lens"], state["table"],
                                        state["cu_seqs"], state["prefix_lens"], state["out"],
                                        cu_q=cu_q, lse=state["lse"], max_len=state["max_len"],
                                        max_prefix=state["prefix"])
        else:
            aio.aio_prefix_attention(state["q"], state["k"], state["v"], state["lens"],
                                     state["table"], state["cu_seqs"], state["prefix_lens"],
                                     state["out"], cu_q=cu_q, lse=state["lse"],
                                     max_len=state["max_len"], max_prefix=state["prefix"])
        return {"out": state["out"], "lse": state["lse"]}
    if op in ("attend", "prefix"):
        return _plain_attention(state)
    return {"append": _plain_append, "norm": _plain_norm}[op](state)


# ------------------------------------------------------------ bytes and flops

def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    H, Hkv, hd = HEADS[case["heads"]]
    if case["op"] == "norm":
        n = case["rows"] * (H + Hkv) * hd
        return {"bytes": 2 * n * size + 4 * case["rows"] + 4 * hd, "flops": 8 * n}
    q_len, k_len, prefix, first = _lengths(case)
    rows, n, page = sum(q_len), case["n"], case["page"]
    if case["op"] == "append":
        # only the pages that the rows fall on are looked up
        index = 4 * (2 * n + 1) + 4 * sum(q // page + 1 for q in q_len)
        return {"bytes": 2 * rows * Hkv * (hd * size + hd + 1) + index, "flops": 0}
    # a prefix counts once per group
    once = [k - (p if f != i else 0) for i, (k, p, f) in enumerate(zip(k_len, prefix, first))]
    index = 4 * (2 * n + 1) + 4 * sum(-(-k // page) for k in once)
    row = hd + 1 if case.get("pool", "q8") == "q8" else 2 * hd
    seen = sum(q * k - q * (q - 1) // 2 for q, k in zip(q_len, k_len))
    return {"bytes": 2 * sum(once) * Hkv * row + rows * H * (2 * hd * size + 4) + index,
            "flops": 4 * H * hd * seen}


# --------------------------------------------------------- 64-bit evaluation

def _exact_rows(st, name, i, nk):
    """A sequence's rows [nk, Hkv, hd] as its pages hold them."""
    pages = st["table"][i, : -(-nk // st["page"])].long()
    x = st[name][pages].transpose(1, 2).flatten(0, 1)[:nk].to(torch.float64)
    if name + "_exp" in st:
        b = st[name + "_exp"][pages].transpose(1, 2).flatten(0, 1)[:nk].to(torch.float64)
        x = x * torch.where(b < 255, torch.exp2(b - 127), math.nan).unsqueeze(-1)
    return x


def _exact_attention(st):
    H, Hkv, hd = HEADS[st["heads"]]
    G, f64 = H // Hkv, torch.float64
    q_len, k_len, _, _ = _lengths(st)
    out = torch.empty(st["q"].shape, dtype=f64, device=st["q"].device)
    lse = torch.empty(st["q"].shape[:2], dtype=f64, device=st["q"].device)
    r0 = 0
    for i, (nq, nk) in enumerate(zip(q_len, k_len)):
        k, v = _exact_rows(st, "k", i, nk), _exact_rows(st, "v", i, nk)
        above = (torch.arange(nk, device=k.device)[None, :] >
                 torch.arange(nk - nq, nk, device=k.device)[:, None])
        for h in range(H):
            s = st["q"][r0: r0 + nq, h].to(f64) @ k[:, h // G].t()
            s = (s / math.sqrt(hd)).masked_fill_(above, -math.inf)
            lse[r0: r0 + nq, h] = torch.logsumexp(s, dim=-1)
            out[r0: r0 + nq, h] = torch.softmax(s, dim=-1) @ v[:, h // G]
        r0 += nq
    return {"out": out, "lse": lse}


def _exact_append(st):
    q_len, k_len, _, _ = _lengths(st)
    table = st["table"].cpu().tolist()
    where = []
    for i, (nq, nk) in enumerate(zip(q_len, k_len)):
        where += [(table[i][p // st["page"]], p % st["page"]) for p in range(nk - nq, nk)]
    page = torch.tensor([w[0] for w in where], device=st["k"].device)
    slot = torch.tensor([w[1] for w in where], device=st["k"].device)
    out = {}
    for name in "kv":
        x = st[name + "_rows"].to(torch.float64)
        top = x.abs().amax(dim=-1, keepdim=True)
        # the least power of two from 2^-119 on for which no code passes 127
        e = torch.full_like(top, -119.0)
        for t in range(-118, 122):
            e = torch.where(torch.round(top * 2.0 ** (1 - t)) > 127, float(t), e)
        out[name], out[name + "_exp"] = st[name].clone(), st[name + "_exp"].clone()
        code = torch.round(x / torch.exp2(e)).clamp(-127, 127).to(torch.int8)
        byte = (e.squeeze(-1) + 127).to(torch.uint8)
        for h in range(x.shape[1]):
            out[name][page, h, slot] = code[:, h]
            out[name + "_exp"][page, h, slot] = byte[:, h]
    return {f: out[f] for f in ("k", "v", "k_exp", "v_exp")}


def _exact_norm(st):
    f64, out = torch.float64, {}
    hd = st["q"].shape[2]
    pos = st["positions"].to(f64)
    for name in "qk":
        x = st[name].to(f64)
        x = x / torch.sqrt(x.square().sum(dim=-1, keepdim=True) / hd + EPS)
        x = x * st[name + "_weight"].to(f64)
        y = torch.empty_like(x)
        for i in range(hd // 2):
            t = pos * BASE ** (-2.0 * i / hd)
            c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
            y[:, :, i] = x[:, :, i] * c - x[:, :, i + hd // 2] * s
            y[:, :, i + hd // 2] = x[:, :, i + hd // 2] * c + x[:, :, i] * s
        out[name] = y
    return out


def exact(case, seed):
    st = _inputs(case, seed)
    return {"attend": _exact_attention, "prefix": _exact_attention, "append": _exact_append,
            "norm": _exact_norm}[case["op"]](st)
