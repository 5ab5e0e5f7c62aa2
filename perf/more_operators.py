"""A key-value cache held in 8 bits, and attention that sees a window of the last tokens and a few first ones, as cases that can
be timed and compared: new tokens' keys and values rounded into 8-bit pages, attention over such pages (one new token a sequence,
and whole prompts), and both attentions with a window and sinks over pages of 16 and of 8 bits.

A case is a dict of plain values.  `prepare` makes what a program holds before the call from the seed alone, `run` makes one pass:
with `own` through the library's entry points, otherwise in plain torch operations in 32 bits.  `exact` gives the same outputs in
64 bits from the definition.

The cache: K pages [page][kv head][slot][dim], V pages [page][kv head][dim][slot].  Token j of sequence s lies in page
table[s][j // page], slot j % page.  In 8 bits a value is an e4m3 number times the scale of its block, 16 successive slots of a
head; a buffer holds the codes of all pages and behind them the scales, float32 [page][kv head][page / 16], all powers of two.
Slots that hold no token are NaN here, the scales of blocks without one too, and table entries that list no page are -1.

The scale of a block is the smallest power of two by which its largest value comes to 448 or less, but at least 2^-15 for fp16 and
2^-117 for bf16 (every value of the cache is then one of the type); it never shrinks while earlier tokens of the sequence stay in
the block, and where it grows their codes are rounded to it.

With a window of w tokens and n sinks the token at position p attends the tokens j <= p with j > p - w or j < n.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
LEAST_SCALE = {"f16": -15, "bf16": -117}                            # exponents
MOST_VALUE = {"f16": 1.875 * 2.0 ** 15, "bf16": 1.875 * 2.0 ** 127}  # larger ones round beyond the type
BLOCK = 16

# (query heads, key/value heads): as many of both, grouped, one for all
HEADS = ((32, 32), (40, 40), (32, 8), (64, 8), (28, 4), (16, 16), (8, 1), (48, 1))
DIMS = (64, 96, 128, 128, 128, 256)
PAGES = (16, 32, 64, 128)


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the step of a serving batch: one token's keys and values for each sequence into 8-bit pages
        dict(name="append8_token", kind="append", bits=8, heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=64, longest=1, prefix=300, layout="tokens", mix=1),
        # prompts' keys and values, as the batched product writes them (token index contiguous)
        dict(name="append8_prompt", kind="append", bits=8, heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=5, longest=4096, prefix=200, layout="features", mix=2),
        # one user's next token, a chat turn in: the smallest call, latency
        dict(name="decode8_token", kind="decode", bits=8, heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=1, longest=401, spread="same", layout="tokens",
             lse=False, window=0, sinks=0, mix=3),
        # one user behind a very long document, grouped heads: one sequence has to fill the card
        dict(name="decode8_long", kind="decode", bits=8, heads=32, kv=8, dim=128, page=64, dtype="bf16", seqs=1, longest=130001, spread="same", layout="tokens",
             lse=True, window=0, sinks=0, mix=4),
        # a serving batch, a key/value head for every query head: the bandwidth of the card
        dict(name="decode8_batch", kind="decode", bits=8, heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=40, longest=4096, spread="near", layout="features",
             lse=False, window=0, sinks=0, mix=5),
        # a batch of very unlike lengths (some sequences empty) that sees its last thousand tokens, grouped heads
        dict(name="decode8_window", kind="decode", bits=8, heads=64, kv=8, dim=128, page=32, dtype="bf16", seqs=61, longest=8192, spread="ragged", layout="features",
             lse=True, window=1000, sinks=4, mix=6),
        # the same on pages of 16 bits: long conversations whose middle pages have been given back
        dict(name="decode_window", kind="decode", bits=16, heads=32, kv=8, dim=128, page=64, dtype="bf16", seqs=48, longest=12000, spread="near", layout="tokens",
             lse=False, window=2048, sinks=4, mix=7),
        # a short question over 8-bit pages: the smallest prompt
        dict(name="prompt8_short", kind="prompt", bits=8, heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=1, longest=61, prefix=0, layout="tokens",
             lse=False, window=0, sinks=0, mix=8),
        # one whole context of a 4096-wide layer
        dict(name="prompt8_4096", kind="prompt", bits=8, heads=32, kv=32, dim=128, page=16, dtype="f16", seqs=1, longest=4096, prefix=0, layout="features",
             lse=False, window=0, sinks=0, mix=9),
        # the next chunk of two long prompts whose earlier tokens are in the cache, with a window, heads of 64
        dict(name="prompt8_chunk", kind="prompt", bits=8, heads=32, kv=8, dim=64, page=32, dtype="bf16", seqs=2, longest=515, prefix=12000, layout="tokens",
             lse=True, window=4096, sinks=16, mix=10),
        # a long prompt that sees a window, pages of 16 bits: most of the triangle is left out
        dict(name="prompt_window", kind="prompt", bits=16, heads=32, kv=8, dim=128, page=16, dtype="bf16", seqs=1, longest=5000, prefix=0, layout="tokens",
             lse=False, window=1024, sinks=4, mix=11),
        # prompts of several users packed into one call, a short window of odd length
        dict(name="prompt_window_packed", kind="prompt", bits=16, heads=32, kv=32, dim=96, page=64, dtype="f16", seqs=9, longest=2500, prefix=0, layout="features",
             lse=True, window=333, sinks=0, mix=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    heads, kv = rng.choice(HEADS)
    c = dict(kind=rng.choice(("append", "decode", "decode", "decode", "prompt", "prompt", "prompt")), heads=heads, kv=kv, dim=rng.choice(DIMS),
             page=rng.choice(PAGES), dtype=rng.choice(tuple(DTYPES)), mix=rng.randrange(1 << 30))
    while True:
        if c["kind"] == "append":
            c |= dict(bits=8, seqs=_log(rng, 1, 128), longest=_log(rng, 1, 4096), prefix=_log(rng, 1, 500), layout=rng.choice(("tokens", "features")))
            if work(c)["bytes"] < 1.9e8 and c["seqs"] * (c["longest"] + c["prefix"]) * c["kv"] * c["dim"] < 3e8:
                return c
            continue
        c |= dict(bits=rng.choice((8, 8, 16)), layout=rng.choice(("tokens", "features")), lse=rng.random() < 0.5)
        seen = c["bits"] == 16 or rng.random() < 0.4                # 16 bits without a window are measured elsewhere
        c |= dict(window=_log(rng, 1, 8192) if seen else 0, sinks=rng.choice((0, 1, 4, 17, 64)) if seen else 0)
        if c["kind"] == "decode":
            c |= dict(seqs=_log(rng, 1, 128), longest=_log(rng, 1, 131072), spread=rng.choice(("same", "near", "ragged")))
            w = work(c)
            if 1e5 < w["bytes"] < 5e8 and w["flops"] < 1e11 and c["seqs"] * c["longest"] * max(c["kv"] * c["dim"], c["heads"]) < 8e8:
                return c
        else:
            c |= dict(seqs=_log(rng, 1, 24), longest=_log(rng, 1, 6000), prefix=rng.choice((0, 0, _log(rng, 1, 30000))))
            if work(c)["flops"] < 1.3e11 and c["seqs"] * c["heads"] * c["longest"] * (c["longest"] + c["prefix"]) < 1.5e9 \
                    and c["seqs"] * c["kv"] * c["dim"] * (c["longest"] + c["prefix"]) < 8e8:
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


def _behind(c, a, b):
    """Tokens sinks .. this - 1 of a sequence are seen by none of its new ones."""
    return max(0, b - a - c["window"] + 1) if c["window"] else 0


def work(case):
    c = case
    new, lens = _lengths(c)
    row = c["kv"] * c["dim"] * c["bits"] // 8                       # bytes of one token's keys, or values, in the cache
    scales = lambda tokens: c["kv"] * 4 * -(-tokens // BLOCK) if c["bits"] == 8 else 0  # noqa: E731
    if c["kind"] == "append":
        return {"bytes": sum(2 * a * (c["kv"] * c["dim"] * 2 + row) + 2 * scales(a) for a in new), "flops": 0}
    held, pairs = 0, 0
    for a, b in zip(new, lens):
        gone = max(0, _behind(c, a, b) - c["sinks"])
        held += 2 * ((b - gone) * row + scales(b - gone))
        if c["window"]:
            pairs += sum(min(p + 1, c["window"] + min(c["sinks"], max(0, p + 1 - c["window"]))) for p in range(max(0, b - a), b))
        else:
            pairs += b * a - a * (a - 1) // 2 if b else 0
    qo = 2 * sum(new) * c["heads"] * c["dim"] * 2 + (4 * sum(new) * c["heads"] if c["lse"] else 0)
    return {"bytes": qo + held, "flops": 4 * c["heads"] * c["dim"] * pairs}


# ------------------------------------------------------------------------------------- inputs
def _rows(gen, c, n, heads, scale=1.0):
    """[n, heads, dim], stored token after token, or with the token index contiguous (rows padded to 8)."""
    dt = DTYPES[c["dtype"]]
    if c["layout"] == "tokens":
        return torch.randn(n, heads, c["dim"], dtype=dt, device=DEV, generator=gen) * scale
    t = torch.randn(heads, c["dim"], (n + 7) // 8 * 8, dtype=dt, device=DEV, generator=gen) * scale
    return t.permute(2, 0, 1)[:n]


def _scale_of(largest, least):
    """The smallest power of two, 2^least or more, that brings `largest` to 448 or less."""
    m, e = torch.frexp(largest / 448)
    e = torch.where(m > 0.5, e, e - 1).masked_fill(largest == 0, least).clamp(min=least)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)    # its bits: pow and exp2 need not be exact


def _views(s):
    """Codes and scales of the K and the V buffer: [page, kv, slot, dim], [page, kv, dim, slot], 2 x [page, kv, block]."""
    c, n = s["case"], s["n_pages"]
    codes = n * c["kv"] * c["page"] * c["dim"]
    part = lambda b: (b[:codes].view(torch.float8_e4m3fn), b[codes:].view(torch.float32).view(n, c["kv"], -1))  # noqa: E731
    (k, ks), (v, vs) = part(s["kp"]), part(s["vp"])
    return k.view(n, c["kv"], c["page"], c["dim"]), ks, v.view(n, c["kv"], c["dim"], c["page"]), vs


def _into_8_bits(c, values, stale, by_slot):
    """A buffer of these pages' values ([page, kv, slot, dim] if by_slot, else [page, kv, dim, slot]); stale: [page, slot] without a token."""
    n, kv, size = values.shape[0], c["kv"], c["page"]
    x = values if by_slot else values.transpose(2, 3)
    x = x.reshape(n, kv, size // BLOCK, BLOCK, -1).float().masked_fill_(stale.view(n, 1, size // BLOCK, BLOCK, 1), 0)
    scale = _scale_of(x.abs().amax((-1, -2)), LEAST_SCALE[c["dtype"]])
    x = (x / scale[..., None, None]).masked_fill_(stale.view(n, 1, size // BLOCK, BLOCK, 1), float("nan")).view(n, kv, size, -1)
    scale.masked_fill_(stale.view(n, 1, -1, BLOCK).all(-1), float("nan"))
    x = x if by_slot else x.transpose(2, 3)
    return torch.cat([x.contiguous().to(torch.float8_e4m3fn).view(torch.uint8).reshape(-1), scale.contiguous().view(torch.uint8).reshape(-1)])


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    new, lens = _lengths(c)
    append = c["kind"] == "append"
    # the pages of every sequence: none where no new token looks any more
    gone = [(0, 0) if append or not c["window"] else (-(-c["sinks"] // c["page"]), _behind(c, a, b) // c["page"]) for a, b in zip(new, lens)]
    width = max(1, max((n + c["page"] - 1) // c["page"] for n in lens))
    listed_at = [[j for j in range((n + c["page"] - 1) // c["page"]) if not g[0] <= j < g[1]] for n, g in zip(lens, gone)]
    n_pages = sum(map(len, listed_at)) + 3                          # a pool is seldom full
    order = list(range(n_pages))
    rng.shuffle(order)
    table, filled, at = [], [0] * n_pages, 0
    for a, n, places in zip(new, lens, listed_at):
        row = [-1] * width
        for j in places:
            row[j] = order[at]
            filled[order[at]] = min(c["page"], max(0, (n - a if append else n) - j * c["page"]))
            at += 1
        table.append(row)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    total = starts[-1]
    s = dict(case=c, n_pages=n_pages, width=width, total=total, longest=max(lens), most_new=max(new), scale=1 / math.sqrt(c["dim"]),
             table=torch.tensor(table, dtype=torch.int32, device=DEV), lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
             starts=torch.tensor(starts, dtype=torch.int32, device=DEV))
    stale = torch.arange(c["page"], device=DEV) >= torch.tensor(filled, device=DEV)[:, None]
    kp = torch.randn(n_pages, c["kv"], c["page"], c["dim"], dtype=dt, device=DEV, generator=gen)
    vp = torch.randn(n_pages, c["kv"], c["dim"], c["page"], dtype=dt, device=DEV, generator=gen)
    if c["bits"] == 8:
        s["kp"], s["vp"] = _into_8_bits(c, kp, stale, True), _into_8_bits(c, vp, stale, False)
    else:
        s["kp"], s["vp"] = kp.masked_fill_(stale[:, None, :, None], float("nan")), vp.masked_fill_(stale[:, None, None, :], float("nan"))
    if append:
        s["k"], s["v"] = _rows(gen, c, total, c["kv"]), _rows(gen, c, total, c["kv"])
        blocks = [(i, j) for i, (a, n) in enumerate(zip(new, lens)) for j in range((n - a) // BLOCK, (n + BLOCK - 1) // BLOCK)]
        s["blocks"] = torch.tensor(blocks, device=DEV).T.contiguous()   # (sequence, number in it) of every block that gets a token
        return s
    # logits of a standard deviation of 2: some tokens matter much more than others
    s["q"] = _rows(gen, c, total, c["heads"], 2.0)
    s["first_seen"] = torch.tensor([_behind(c, a, b) for a, b in zip(new, lens)], device=DEV)
    s["out"] = torch.empty_like(s["q"])                             # the same strides
    s["lse"] = torch.empty(total, c["heads"], dtype=torch.float32, device=DEV) if c["lse"] else None
    return s


# ------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _library(state)
    return _plain_append(state) if state["case"]["kind"] == "append" else _plain_attention(state)


def _library(s):
    import paper_2402_15319_amd as vq
    c = s["case"]
    if "desc" not in s:                                             # what a program keeps: descriptor, batch and workspace
        s["desc"] = vq.make_attn_desc(c["heads"], c["kv"], c["dim"], c["page"], s["n_pages"], vq.VQ_F16 if c["dtype"] == "f16" else vq.VQ_BF16,
                                      s["scale"], cache_dtype=vq.VQ_E4M3 if c["bits"] == 8 else None)
        s["batch"] = vq.AttnBatch(s["lens"], s["table"], n_tokens=s["total"], max_len=s["longest"],
                                  q_start=None if c["kind"] == "decode" else s["starts"])
        if c["kind"] != "append":
            s["workspace"] = vq.attn_workspace(s["desc"], s["batch"], DEV)
            s["window"] = vq.VQAttnWindow(c["window"], c["sinks"]) if c["window"] else None
    if c["kind"] == "append":
        vq.vq_cache_append(s["desc"], s["batch"], s["k"], s["v"], s["kp"], s["vp"])
        return list(_views(s))
    if c["window"]:
        call = vq.vq_attn_decode_window if c["kind"] == "decode" else vq.vq_attn_prompt_window
        call(s["desc"], s["batch"], s["window"], s["q"], s["kp"], s["vp"], s["out"], s["workspace"], lse=s["lse"])
    else:
        call = vq.vq_attn_decode if c["kind"] == "decode" else vq.vq_attn_prompt
        call(s["desc"], s["batch"], s["q"], s["kp"], s["vp"], s["out"], s["workspace"], lse=s["lse"])
    return [s["out"], s["lse"]] if c["lse"] else [s["out"]]


def _owners(s):
    """Sequence and position of every new token."""
    starts, t = s["starts"].long(), torch.arange(s["total"], device=DEV)
    seq = torch.searchsorted(starts, t, right=True) - 1
    return seq, t - starts[seq + 1] + s["lens"].long()[seq]


def _plain_append(s):
    c = s["case"]
    seq, number = s["blocks"]
    starts, lens = s["starts"].long(), s["lens"].long()
    first = (lens - (starts[1:] - starts[:-1]))[seq]                # position of the sequence's first new token
    pos = number[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    fresh = (pos >= first[:, None]) & (pos < lens[seq, None])       # [blocks, 16]
    kept = pos < first[:, None]
    token = (starts[seq, None] + pos - first[:, None]).clamp(0, s["total"] - 1)
    page, at = s["table"].long()[seq, number * BLOCK // c["page"]], number % (c["page"] // BLOCK)
    k, ks, v, vs = _views(s)
    n = s["n_pages"]
    for codes, scales, x in ((k.view(n, c["kv"], -1, BLOCK, c["dim"]).permute(0, 2, 1, 3, 4), ks, s["k"]),
                             (v.view(n, c["kv"], c["dim"], -1, BLOCK).permute(0, 3, 1, 4, 2), vs, s["v"])):
        x = x[token].transpose(1, 2).float()                        # [blocks, kv, 16, dim]
        largest = x.abs().masked_fill_(~fresh[:, None, :, None], 0).amax((-1, -2)).clamp_(max=MOST_VALUE[c["dtype"]])
        old = scales[page, :, at]
        some = kept.any(-1)[:, None]
        scale = torch.maximum(_scale_of(largest, LEAST_SCALE[c["dtype"]]), torch.where(some, old, 0))
        x = x.clamp_(-MOST_VALUE[c["dtype"]], MOST_VALUE[c["dtype"]]).div_(scale[..., None, None]).to(torch.float8_e4m3fn)
        was = codes.view(torch.uint8)[page, at]                     # [blocks, kv, 16, dim]
        moved = (was.view(torch.float8_e4m3fn).float() * torch.where(some, old / scale, 1)[..., None, None]).to(torch.float8_e4m3fn)
        x = torch.where(kept[:, None, :, None], moved.view(torch.uint8), torch.where(fresh[:, None, :, None], x.view(torch.uint8), was))
        codes.view(torch.uint8)[page, at] = x
        scales[page, :, at] = scale
    return [k, ks, v, vs]


def _plain_attention(s):
    c = s["case"]
    n, kv, dim, group, span = c["seqs"], c["kv"], c["dim"], c["heads"] // c["kv"], s["width"] * c["page"]
    seq, pos = _owners(s)
    index = torch.arange(s["total"], device=DEV) - s["starts"].long()[seq]
    table = s["table"].long().clamp(min=0)
    j = torch.arange(span, device=DEV)
    live = (j < s["lens"][:, None]) & ((j >= s["first_seen"][:, None]) | (j < c["sinks"]))      # [n, span]
    if c["bits"] == 8:
        k, ks, v, vs = _views(s)
        k = k.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * ks[table].repeat_interleave(BLOCK, -1)[..., None]
        v = v.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * vs[table].repeat_interleave(BLOCK, -1)[..., None, :]
    else:
        k, v = s["kp"][table].float(), s["vp"][table].float()
    k = k.permute(0, 2, 4, 1, 3).reshape(n, kv, dim, span)
    v = v.permute(0, 2, 1, 4, 3).reshape(n, kv, span, dim)
    v = v.masked_fill_(~live[:, None, :, None], 0)
    q = torch.zeros(n, kv, group, s["most_new"], dim, device=DEV)
    q[seq, :, :, index] = s["q"].float().reshape(-1, kv, group, dim)
    at = torch.full((n, s["most_new"]), -1, dtype=torch.long, device=DEV)
    at[seq, index] = pos
    t = torch.matmul(q.reshape(n, kv, -1, dim), k).mul_(s["scale"]).reshape(n, kv, group, -1, span)
    unseen = j > at[:, :, None]                                                                 # [n, new, span]
    if c["window"]:
        unseen |= (j <= at[:, :, None] - c["window"]) & (j >= c["sinks"])
    t.masked_fill_(unseen[:, None, None], -math.inf)
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
def _nearest_e4m3(x):
    """The nearest multiple of a number's last place in e4m3, ties to the even one."""
    _, e = torch.frexp(x)
    place = _power(e.clamp(min=-5) - 4)
    return torch.round(x / place) * place


def _power(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exact(case, seed):
    s, c = prepare(case, seed), case
    new, lens = _lengths(c)
    table = s["table"].tolist()
    if c["kind"] == "append":
        kc, ks, vc, vs = [t.double() for t in _views(s)]
        for x, codes, scales in ((s["k"], kc, ks), (s["v"], vc.transpose(2, 3), vs)):
            for i, (a, b) in enumerate(zip(new, lens)):
                for at in range((b - a) // BLOCK * BLOCK, b, BLOCK):
                    lo, hi = max(at, b - a), min(at + BLOCK, b)
                    page, slot = table[i][at // c["page"]], at % c["page"]
                    t = lo - b + int(s["starts"][i + 1])
                    fresh = x[t:t + hi - lo].double().transpose(0, 1)                           # [kv, tokens, dim]
                    fresh = fresh.clamp(-MOST_VALUE[c["dtype"]], MOST_VALUE[c["dtype"]])
                    largest = fresh.abs().amax((1, 2)).clamp(min=448 * 2.0 ** LEAST_SCALE[c["dtype"]])
                    e = torch.floor(torch.log2(largest)).long() - 9                             # too small by 0 or 1 and a slip of log2
                    e = torch.where(448 * _power(e) < largest, e + 1, e)
                    e = torch.where(448 * _power(e) < largest, e + 1, e)
                    scale = _power(torch.where(448 * _power(e) < largest, e + 1, e))
                    if lo > at:
                        was = scales[page, :, slot // BLOCK]
                        scale = torch.maximum(scale, was)
                        codes[page, :, slot:slot + lo - at] = _nearest_e4m3(codes[page, :, slot:slot + lo - at] * (was / scale)[:, None, None])
                    codes[page, :, slot + lo - at:slot + hi - at] = _nearest_e4m3(fresh / scale[:, None, None])
                    scales[page, :, slot // BLOCK] = scale
        return [kc, ks, vc, vs]
    if c["bits"] == 8:
        k8, ks, v8, vs = _views(s)
    group, t = c["heads"] // c["kv"], 0
    out = torch.zeros(s["total"], c["heads"], c["dim"], dtype=torch.float64, device=DEV)
    lse = torch.full((s["total"], c["heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for i, (a, b) in enumerate(zip(new, lens)):
        if b:
            j, p = torch.arange(b, device=DEV), torch.arange(b - a, b, device=DEV)[:, None]
            seen = j <= p
            if c["window"]:
                seen &= (j > p - c["window"]) | (j < c["sinks"])
            used = seen.any(0)
            at = j[used]                                                                        # tokens that some row sees
            seen = seen[:, used]
            page, slot = s["table"][i].long()[at // c["page"]], at % c["page"]
            for h in range(c["kv"]):
                if c["bits"] == 8:
                    k = k8.view(torch.uint8)[page, h, slot].view(torch.float8_e4m3fn).double() * ks[page, h, slot // BLOCK].double()[:, None]
                    v = v8.view(torch.uint8)[page, h, :, slot].view(torch.float8_e4m3fn).double() * vs[page, h, slot // BLOCK].double()[:, None]
                else:
                    k, v = s["kp"][page, h, slot].double(), s["vp"][page, h, :, slot].double()
                for g in range(h * group, (h + 1) * group):
                    x = (s["q"][t:t + a, g].double() @ k.T) / math.sqrt(c["dim"])
                    x = x.masked_fill(~seen, -math.inf)
                    lse[t:t + a, g] = torch.logsumexp(x, -1)
                    out[t:t + a, g] = torch.softmax(x, -1) @ v
        t += a
    return [out, lse] if c["lse"] else [out]
