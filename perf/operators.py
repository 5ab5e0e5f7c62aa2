"""Attention over a paged key-value cache, as cases that can be timed and compared: new tokens'
keys and values into the cache's pages, attention of one new token a sequence, causal attention of
whole prompts, and copies of pages (the fork and the compaction of a cache).

A case is a dict of plain values.  `prepare` makes what a program holds before the call from the
seed alone, `run` makes one pass: with `own` through the library's entry points, otherwise in plain
torch operations in 32 bits.  `exact` gives the same outputs in 64 bits from the definition.

The cache: K pages [page][kv head][slot][dim], V pages [page][kv head][dim][slot].  Token j of
sequence s lies in page table[s][j // page], slot j % page.  Slots that hold no token are NaN here,
and table entries that list no page are -1.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}

# (query heads, key/value heads): as many of both, grouped, one for all
HEADS = ((32, 32), (40, 40), (32, 8), (64, 8), (28, 4), (16, 16), (8, 1), (48, 1))
DIMS = (64, 96, 128, 128, 128, 256)
PAGES = (16, 32, 64, 128)


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one user's next token, a chat turn in: the smallest call, latency; 32 heads of 128 as a 4096-wide layer has
        dict(name="decode_token", kind="decode", heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=1, longest=401, spread="same", layout="tokens", lse=False, mix=1),
        # one user behind a very long document, grouped heads: one sequence has to fill the card
        dict(name="decode_long", kind="decode", heads=32, kv=8, dim=128, page=64, dtype="bf16", seqs=1, longest=130001, spread="same", layout="tokens", lse=True, mix=2),
        # a serving batch, a key/value head for every query head: the bandwidth of the card
        dict(name="decode_batch", kind="decode", heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=24, longest=4096, spread="near", layout="features", lse=False, mix=3),
        # a batch of very unlike lengths (some sequences empty), grouped heads
        dict(name="decode_ragged", kind="decode", heads=64, kv=8, dim=128, page=32, dtype="bf16", seqs=61, longest=8192, spread="ragged", layout="features", lse=True, mix=4),
        # a short question: the smallest prompt
        dict(name="prompt_short", kind="prompt", heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=1, longest=61, prefix=0, layout="tokens", lse=False, mix=5),
        # one whole context of a 4096-wide layer, as the batched product writes it (token index contiguous)
        dict(name="prompt_4096", kind="prompt", heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=1, longest=4096, prefix=0, layout="features", lse=False, mix=6),
        # prompts of several users packed into one call, grouped heads
        dict(name="prompt_packed", kind="prompt", heads=32, kv=8, dim=128, page=64, dtype="bf16", seqs=9, longest=2500, prefix=0, layout="tokens", lse=True, mix=7),
        # the next chunk of two long prompts whose earlier tokens are in the cache, heads of 64
        dict(name="prompt_chunk", kind="prompt", heads=32, kv=8, dim=64, page=32, dtype="f16", seqs=2, longest=515, prefix=12000, layout="tokens", lse=False, mix=8),
        # the step of a serving batch: one token's keys and values for each sequence
        dict(name="append_token", kind="append", heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=64, longest=1, prefix=300, layout="tokens", mix=9),
        # prompts' keys and values, as the batched product writes them
        dict(name="append_prompt", kind="append", heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=5, longest=4096, prefix=200, layout="features", mix=10),
        # a sequence forked seven times: its last page in 32 layers' caches
        dict(name="copy_fork", kind="copy", heads=32, kv=8, dim=128, page=16, dtype="bf16", layers=32, pages=64, pairs=7, mix=11),
        # a pool compacted: four hundred pages moved into holes
        dict(name="copy_compact", kind="copy", heads=32, kv=32, dim=128, page=16, dtype="f16", layers=4, pages=1024, pairs=400, mix=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    heads, kv = rng.choice(HEADS)
    c = dict(kind=rng.choice(("decode", "decode", "decode", "prompt", "prompt", "prompt", "append", "copy")), heads=heads, kv=kv,
             dim=rng.choice(DIMS), page=rng.choice(PAGES), dtype=rng.choice(tuple(DTYPES)), mix=rng.randrange(1 << 30))
    while True:
        if c["kind"] == "decode":
            c |= dict(seqs=_log(rng, 1, 128), longest=_log(rng, 1, 131072), spread=rng.choice(("same", "near", "ragged")),
                      layout=rng.choice(("tokens", "features")), lse=rng.random() < 0.5)
            w = work(c)
            if 1e5 < w["bytes"] < 1e9 and w["flops"] < 1e11 and c["seqs"] * c["longest"] * max(c["kv"] * c["dim"], c["heads"]) < 8e8:
                return c
        elif c["kind"] == "prompt":
            c |= dict(seqs=_log(rng, 1, 24), longest=_log(rng, 1, 6000), prefix=rng.choice((0, 0, _log(rng, 1, 30000))),
                      layout=rng.choice(("tokens", "features")), lse=rng.random() < 0.5)
            if work(c)["flops"] < 1.3e11 and c["seqs"] * c["heads"] * c["longest"] * (c["longest"] + c["prefix"]) < 1.5e9 \
                    and c["seqs"] * c["kv"] * c["dim"] * (c["longest"] + c["prefix"]) < 8e8:
                return c
        elif c["kind"] == "append":
            c |= dict(seqs=_log(rng, 1, 128), longest=_log(rng, 1, 4096), prefix=_log(rng, 1, 500), layout=rng.choice(("tokens", "features")))
            if work(c)["bytes"] < 2.5e8 and c["seqs"] * (c["longest"] + c["prefix"]) * c["kv"] * c["dim"] < 3e8:
                return c
        else:
            c |= dict(layers=rng.choice((1, 4, 16, 32, 40)), pages=_log(rng, 16, 2048))
            c["pairs"] = _log(rng, 1, c["pages"] // 2)
            if work(c)["bytes"] < 8e8 and c["layers"] * c["pages"] * c["kv"] * c["dim"] * c["page"] < 3e8:
                return c


def _lengths(c):
    """(new tokens, tokens in the cache with them) of every sequence."""
    rng, n = random.Random(c["mix"]), c["seqs"]
    if c["kind"] == "decode":
        if c["spread"] == "same":
            return [1] * n, [c["longest"]] * n
        if c["spread"] == "near":
            return [1] * n, [c["longest"]] + [rng.randint((c["longest"] + 1) // 2, c["longest"]) for _ in range(n - 1)]
        return [1] * n, [c["longest"]] + [0 if rng.random() < 0.05 else _log(rng, 1, c["longest"]) for _ in range(n - 1)]
    new = [c["longest"]] + [_log(rng, max(1, c["longest"] // 20), c["longest"]) for _ in range(n - 1)]
    return new, [a + (rng.randint(c["prefix"] // 2, c["prefix"]) if c["prefix"] else 0) for a in new]


def work(case):
    row = case["kv"] * case["dim"] * 2                              # bytes of one token's keys, or values
    if case["kind"] == "copy":
        return {"bytes": 2 * case["pairs"] * 2 * case["layers"] * row * case["page"], "flops": 0}
    new, lens = _lengths(case)
    if case["kind"] == "append":
        return {"bytes": 4 * sum(new) * row, "flops": 0}
    qo = 2 * sum(new) * case["heads"] * case["dim"] * 2 + (4 * sum(new) * case["heads"] if case["lse"] else 0)
    seen = sum(b * a - a * (a - 1) // 2 for a, b in zip(new, lens))  # (token, earlier token) pairs
    return {"bytes": qo + 2 * sum(lens) * row, "flops": 4 * case["heads"] * case["dim"] * seen}


# ------------------------------------------------------------------------------------- inputs
def _rows(gen, c, n, heads, scale=1.0):
    """[n, heads, dim], stored token after token, or with the token index contiguous (rows padded to 8)."""
    dt = DTYPES[c["dtype"]]
    if c["layout"] == "tokens":
        return torch.randn(n, heads, c["dim"], dtype=dt, device=DEV, generator=gen) * scale
    t = torch.randn(heads, c["dim"], (n + 7) // 8 * 8, dtype=dt, device=DEV, generator=gen) * scale
    return t.permute(2, 0, 1)[:n]


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    if c["kind"] == "copy":
        shape = (2 * c["layers"], c["pages"], c["kv"] * c["page"] * c["dim"])
        at = rng.sample(range(c["pages"]), 2 * c["pairs"])
        pairs = list(zip(at[::2], at[1::2]))                        # (from, to)
        return dict(case=c, caches=torch.randn(shape, dtype=dt, device=DEV, generator=gen), pairs=pairs)
    new, lens = _lengths(c)
    own_pages = [(n + c["page"] - 1) // c["page"] for n in lens]
    width, used = max(1, max(own_pages)), sum(own_pages)
    n_pages = used + 3                                              # a pool is seldom full
    order = list(range(n_pages))
    rng.shuffle(order)
    table, filled, at = [], [0] * n_pages, 0
    for n, w in zip(lens, own_pages):
        table.append(order[at:at + w] + [-1] * (width - w))
        for j in range(w):
            filled[order[at + j]] = min(c["page"], n - j * c["page"])
        at += w
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    total = starts[-1]
    s = dict(case=c, n_pages=n_pages, width=width, total=total, longest=max(lens), most_new=max(new),
             table=torch.tensor(table, dtype=torch.int32, device=DEV), lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
             starts=torch.tensor(starts, dtype=torch.int32, device=DEV),
             kp=torch.randn(n_pages, c["kv"], c["page"], c["dim"], dtype=dt, device=DEV, generator=gen),
             vp=torch.randn(n_pages, c["kv"], c["dim"], c["page"], dtype=dt, device=DEV, generator=gen))
    if c["kind"] == "append":
        s["k"], s["v"] = _rows(gen, c, total, c["kv"]), _rows(gen, c, total, c["kv"])
        return s
    # logits of a standard deviation of 2: some tokens matter much more than others
    s["q"] = _rows(gen, c, total, c["heads"], 2.0)
    s["scale"] = 1 / math.sqrt(c["dim"])
    stale = torch.arange(c["page"], device=DEV) >= torch.tensor(filled, device=DEV)[:, None]
    s["kp"].masked_fill_(stale[:, None, :, None], float("nan"))
    s["vp"].masked_fill_(stale[:, None, None, :], float("nan"))
    s["out"] = torch.empty_like(s["q"])                             # the same strides
    s["lse"] = torch.empty(total, c["heads"], dtype=torch.float32, device=DEV) if c["lse"] else None
    return s


# ------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _library(state)
    kind = state["case"]["kind"]
    return _plain_copy(state) if kind == "copy" else _plain_append(state) if kind == "append" else _plain_attention(state)


def _library(s):
    import paper_2402_15319_amd as vq
    c = s["case"]
    if c["kind"] == "copy":
        if "desc" not in s:                                         # what a program keeps: descriptor and buffers
            s["desc"] = vq.make_attn_desc(c["heads"], c["kv"], c["dim"], c["page"], c["pages"], vq.VQ_F16 if c["dtype"] == "f16" else vq.VQ_BF16)
            s["buffers"] = list(s["caches"].unbind(0))
        vq.vq_cache_copy(s["desc"], s["buffers"], s["pairs"])
        return s["caches"]
    if "desc" not in s:                                             # descriptor, batch and workspace
        s["desc"] = vq.make_attn_desc(c["heads"], c["kv"], c["dim"], c["page"], s["n_pages"], vq.VQ_F16 if c["dtype"] == "f16" else vq.VQ_BF16,
                                      s.get("scale"))
        s["batch"] = vq.AttnBatch(s["lens"], s["table"], n_tokens=s["total"], max_len=s["longest"],
                                  q_start=None if c["kind"] == "decode" else s["starts"])
        if c["kind"] != "append":
            s["workspace"] = vq.attn_workspace(s["desc"], s["batch"], DEV)
    if c["kind"] == "append":
        vq.vq_cache_append(s["desc"], s["batch"], s["k"], s["v"], s["kp"], s["vp"])
        return [s["kp"], s["vp"]]
    call = vq.vq_attn_decode if c["kind"] == "decode" else vq.vq_attn_prompt
    call(s["desc"], s["batch"], s["q"], s["kp"], s["vp"], s["out"], s["workspace"], lse=s["lse"])
    return [s["out"], s["lse"]] if c["lse"] else [s["out"]]


def _plain_copy(s):
    pairs = torch.tensor(s["pairs"], device=DEV)
    s["caches"][:, pairs[:, 1]] = s["caches"][:, pairs[:, 0]]
    return s["caches"]


def _owners(s):
    """Sequence and position of every new token."""
    starts, t = s["starts"].long(), torch.arange(s["total"], device=DEV)
    seq = torch.searchsorted(starts, t, right=True) - 1
    return seq, t - starts[seq + 1] + s["lens"].long()[seq]


def _plain_append(s):
    seq, pos = _owners(s)
    page, slot = s["table"].long()[seq, pos // s["case"]["page"]], pos % s["case"]["page"]
    s["kp"][page, :, slot] = s["k"]
    s["vp"][page, :, :, slot] = s["v"]
    return [s["kp"], s["vp"]]


def _plain_attention(s):
    c = s["case"]
    n, kv, dim, group, span = c["seqs"], c["kv"], c["dim"], c["heads"] // c["kv"], s["width"] * c["page"]
    seq, pos = _owners(s)
    index = torch.arange(s["total"], device=DEV) - s["starts"].long()[seq]
    table = s["table"].long().clamp(min=0)
    live = torch.arange(span, device=DEV) < s["lens"][:, None]                                  # [n, span]
    k = s["kp"][table].permute(0, 2, 4, 1, 3).reshape(n, kv, dim, span).float()
    v = s["vp"][table].permute(0, 2, 1, 4, 3).reshape(n, kv, span, dim).float()
    v = v.masked_fill_(~live[:, None, :, None], 0)
    q = torch.zeros(n, kv, group, s["most_new"], dim, device=DEV)
    q[seq, :, :, index] = s["q"].float().reshape(-1, kv, group, dim)
    at = torch.full((n, s["most_new"]), -1, dtype=torch.long, device=DEV)
    at[seq, index] = pos
    t = torch.matmul(q.reshape(n, kv, -1, dim), k).mul_(s["scale"]).reshape(n, kv, group, -1, span)
    t.masked_fill_(torch.arange(span, device=DEV) > at[:, None, None, :, None], -math.inf)
    m = t.amax(-1, keepdim=True).clamp_(min=-3e38)                                              # a row without tokens: exp(-inf)
    p = t.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n, kv, -1, span), v).reshape(n, kv, group, -1, dim)
    o = torch.where(l > 0, o / l, 0)
    out = o[seq, :, :, index].reshape(-1, c["heads"], dim).to(DTYPES[c["dtype"]])
    if not c["lse"]:
        return [out]
    lse = torch.where(l > 0, m + l.log(), -math.inf)[..., 0]
    return [out, lse[seq, :, :, index].reshape(-1, c["heads"])]


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "copy":
        caches = s["caches"].double()
        for a, b in s["pairs"]:
            caches[:, b].copy_(caches[:, a])
        return caches
    new, lens = _lengths(c)
    table = s["table"].tolist()
    if c["kind"] == "append":
        kp, vp, t = s["kp"].double(), s["vp"].double(), 0
        for i, (a, b) in enumerate(zip(new, lens)):
            for at in range(b - a, b):
                if at == b - a or at % c["page"] == 0:              # the rest of a page at once
                    m = min(c["page"] - at % c["page"], b - at)
                    to, page = slice(at % c["page"], at % c["page"] + m), table[i][at // c["page"]]
                    kp[page, :, to] = s["k"][t:t + m].double().transpose(0, 1)
                    vp[page, :, :, to] = s["v"][t:t + m].double().permute(1, 2, 0)
                    t += m
        return [kp, vp]
    group, t = c["heads"] // c["kv"], 0
    out = torch.zeros(s["total"], c["heads"], c["dim"], dtype=torch.float64, device=DEV)
    lse = torch.full((s["total"], c["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for i, (a, b) in enumerate(zip(new, lens)):
        if b:
            pages = table[i][:(b + c["page"] - 1) // c["page"]]
            late = torch.arange(b, device=DEV) > torch.arange(b - a, b, device=DEV)[:, None]
            for h in range(c["kv"]):
                k = s["kp"][pages, h].reshape(-1, c["dim"])[:b].double()
                v = s["vp"][pages, h].transpose(1, 2).reshape(-1, c["dim"])[:b].double()
                for g in range(h * group, (h + 1) * group):
                    x = (s["q"][t:t + a, g].double() @ k.T) / math.sqrt(c["dim"])
                    x = x.masked_fill(late, -math.inf)
                    lse[t:t + a, g] = torch.logsumexp(x, -1)
                    out[t:t + a, g] = torch.softmax(x, -1) @ v
        t += a
    return [out, lse] if c["lse"] else [out]
