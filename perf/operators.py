"""Timing cases of the cache's operators: K/V rows held in 4 bits, and eviction by accumulated weight.

Four kinds of work, each a thing a serving program does between two steps of the model:

  append      new K/V rows go into a paged 4-bit cache (``kv4_append``), and the same rows are read back
              (``kv4_read``): a prompt, or the few tokens of a step
  verify      attention of one layer's queries over a paged 4-bit cache (``kv4_verify``): over index
              lists or over everything, for one token or the speculated ones, with or without the
              in-flight tokens behind the context
  accumulate  the draft model's attention maps are added to every position's weight
              (``accumulate_attention``)
  evict       the positions of the lowest weight are given up (``evict``) and the rows that stay are moved
              into the holes (``move_rows``), for the pools of several layers, in 16 or in 4 bits

A row of the 4-bit cache is the 128 values of one position, KV head and side (K or V): with z the smallest
and x the largest of them, the scale is s = (x - z) / 15 rounded to 16 bits, a value's code is
min(15, rint((value - z) / s)), and a code c stands for s c + z.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
HEAD_DIM = 128
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- the cases ---------------------------------------------------------------------------------
def _append(name, **kw):
    c = {"name": name, "kind": "append", "batch": 8, "tokens": 6, "ragged": False, "start": 32768, "kv_heads": 8, "page": 16,
         "dtype": "bf16", "layout": "head"}
    c.update(kw)
    return c


def _verify(name, **kw):
    c = {"name": name, "kind": "verify", "batch": 8, "ctx": 32768, "ctx_min": 0, "n_q": 6, "q_heads": 32, "kv_heads": 8, "page": 16,
         "paged": True, "dense": False, "kept": 1228, "groups": 1, "empty": False, "tail": 0, "dtype": "bf16", "layout": "head"}
    c.update(kw)
    return c


def _accumulate(name, **kw):
    c = {"name": name, "kind": "accumulate", "draft_layers": 4, "batch": 8, "ctx": 32768, "ctx_min": 0, "heads": 12, "gamma": 5,
         "groups": 1, "decay": 1.0}
    c.update(kw)
    return c


def _evict(name, **kw):
    c = {"name": name, "kind": "evict", "batch": 8, "ctx": 32768, "ctx_min": 0, "budget": 16384, "sink": 4, "recent": 512, "groups": 1,
         "positions": False, "ties": False, "layers": 2, "kv_heads": 8, "page": 16, "bits": 16}
    c.update(kw)
    return c


def listed():
    return [
        # one token of one short conversation over the positions that the draft model kept: latency
        _verify("verify_b1_4k_token", batch=1, ctx=4096, n_q=1, kept=796, paged=False),
        # the serving workload, one layer: batch 8, 32k context, five speculated tokens and one more
        _verify("verify_b8_32k"),
        # a ragged batch as a continuous-batching server has it, one list per KV head
        _verify("verify_ragged_b32", batch=32, ctx=62699, ctx_min=2474, n_q=5, kept=16000, groups=8),
        # plain decoding over whole contexts of odd lengths, the token itself in the cache already
        _verify("verify_decode_b16", batch=16, ctx=16381, ctx_min=5003, n_q=1, dense=True, tail=1, page=32, dtype="fp16", layout="slot"),
        # a layer that keeps every position of long contexts, 40 query rows to a KV head
        _verify("verify_dense_128k", batch=4, ctx=131072, n_q=5, q_heads=64, dense=True, tail=5),
        # the tokens of one step
        _append("append_step_b8"),
        # two prompts of different lengths
        _append("append_prompts", batch=2, tokens=16384, ragged=True, start=0, dtype="fp16"),
        # one draft layer of one conversation
        _accumulate("accumulate_b1_4k", draft_layers=1, batch=1, ctx=4096, gamma=4),
        # the serving workload's draft maps, old weight fading
        _accumulate("accumulate_b8_32k", decay=0.95),
        # a conversation that has outgrown its room by a few pages: one layer in 4 bits
        _evict("evict_b1_4k", batch=1, ctx=4096, budget=3968, recent=128, layers=1, bits=4),
        # half of a 32k context goes, in the bf16 pools of two layers
        _evict("evict_b8_32k"),
        # long ragged contexts that were thinned before, a decision per KV head, four layers in 4 bits
        _evict("evict_b4_128k_heads", batch=4, ctx=131072, ctx_min=40009, budget=65536, recent=4096, groups=8, positions=True,
               layers=4, bits=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges that the listed ones stand for; never larger than the largest of them."""
    kind = rng.choice(["verify", "verify", "append", "accumulate", "evict", "evict"])
    batch, ctx = _log_int(rng, 1, 32), _log_int(rng, 500, 131072)
    while batch * ctx > 4 * 131072:
        batch = (batch + 1) // 2
    ctx_min = max(100, ctx // rng.randint(2, 12)) if batch > 1 and rng.random() < 0.5 else 0
    page, layout, dtype = rng.choice([16, 16, 32, 64, 24]), rng.choice(["head", "slot"]), rng.choice(["bf16", "fp16"])
    if kind == "verify":
        q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (64, 8), (16, 2), (8, 8), (12, 4)])
        n_q = rng.choice([1, 1, rng.randint(2, 8)])
        while n_q * (q_heads // kv_heads) > 64 or (n_q > 1 and batch * ctx * n_q * (q_heads // kv_heads) > 40 * 4 * 131072):
            n_q -= 1
        dense, tail = rng.random() < 0.4, rng.choice([0, 0, n_q, n_q + 3])
        c = _verify("", batch=batch, ctx=ctx, ctx_min=ctx_min, n_q=n_q, q_heads=q_heads, kv_heads=kv_heads, page=page,
                    paged=rng.random() < 0.8, dense=dense, kept=_log_int(rng, min(64, ctx), ctx), groups=rng.choice([1, kv_heads]),
                    empty=rng.random() < 0.3, tail=tail, dtype=dtype, layout=layout)
    elif kind == "append":
        tokens = rng.choice([1, rng.randint(2, 9), _log_int(rng, 16, 16384)])
        while batch * tokens > 32768:
            batch = (batch + 1) // 2
            tokens = min(tokens, 32768)
        c = _append("", batch=batch, tokens=tokens, ragged=rng.random() < 0.5, start=rng.randint(0, 4000),
                    kv_heads=rng.choice([1, 2, 4, 8]), page=page, dtype=dtype, layout=layout)
    elif kind == "accumulate":
        heads, groups = rng.choice([(12, 1), (16, 1), (16, 8), (12, 4)])
        gamma = rng.randint(1, 7)
        layers = max(1, min(rng.randint(1, 4), (60 << 20) // (batch * ctx * heads * gamma)))
        while batch * ctx * heads * gamma > (60 << 20):
            gamma -= 1
        c = _accumulate("", draft_layers=layers, batch=batch, ctx=ctx, ctx_min=ctx_min, heads=heads, gamma=gamma, groups=groups,
                        decay=rng.choice([1.0, 0.9]))
    else:
        bits, layers = rng.choice([16, 4]), rng.randint(1, 4)
        while layers * batch * ctx > (16 // bits) * 400000:
            layers = (layers + 1) // 2 if layers > 1 else 1
            batch = (batch + 1) // 2 if layers == 1 else batch
        budget = max(16, int(ctx * rng.uniform(0.2, 1.1)))
        c = _evict("", batch=batch, ctx=ctx, ctx_min=ctx_min if batch > 1 else 0, budget=budget, sink=rng.randint(0, 4),
                   recent=rng.randint(0, budget // 4), groups=rng.choice([1, 8]), positions=rng.random() < 0.5,
                   ties=rng.random() < 0.5, layers=layers, page=page, bits=bits)
    return {k: v for k, v in c.items() if k != "name"}


# ---- what a case's numbers say, the same for every seed -------------------------------------------
def _lens(case):
    """Context lengths: all `ctx`, or spread over [ctx_min, ctx] on a logarithmic scale, the longest somewhere inside."""
    b, hi, lo = case["batch"], case["ctx"], case["ctx_min"]
    if not lo or b == 1:
        return [hi] * b
    at = [((i * 5 + 3) % b) / (b - 1) if math.gcd(5, b) == 1 else ((i * 7 + 3) % b) / (b - 1) for i in range(b)]
    return [min(hi, max(lo, int(round(lo * (hi / lo) ** x)))) for x in at]


def _kept(case):
    """Lengths of the index lists, [batch][groups]: in proportion to the contexts, up to a quarter apart between heads."""
    got = []
    for i, n in enumerate(_lens(case)):
        row = [max(1, min(n, int(case["kept"] * n / case["ctx"] * (1 - (3 * g + i) % 8 / 32)))) for g in range(case["groups"])]
        got.append([0 if case["empty"] and (i + g) % 5 == 2 else k for g, k in enumerate(row)])
    return got


def _new_tokens(case):
    t = case["tokens"]
    return [max(0, t - (i * (t // 3) + i) % t) if case["ragged"] else t for i in range(case["batch"])]


def _pages_per_seq(case):
    longest = case["start"] + case["tokens"] if case["kind"] == "append" else case["ctx"] + case.get("tail", 0)
    return -(-longest // case["page"])


def _move_stride(case):
    return max(1, min(case["budget"], case["ctx"] - case["budget"]))


def work(case):
    kind, h = case["kind"], case.get("kv_heads", 0)
    if kind == "append":
        rows = sum(_new_tokens(case)) * h * 2
        # in as 16-bit values, out as codes and scales; these in again, out as 16-bit values
        return {"bytes": rows * 2 * (2 * HEAD_DIM + HEAD_DIM // 2 + 4), "flops": rows * HEAD_DIM * 6}
    if kind == "verify":
        b, t, hq = case["batch"], case["n_q"], case["q_heads"]
        if case["dense"]:
            n, listed_ids = sum(_lens(case)) * h, 0
        else:
            n, listed_ids = sum(map(sum, _kept(case))) * (h // case["groups"]), sum(map(sum, _kept(case)))
        n += case["tail"] * b * h
        return {"bytes": n * (HEAD_DIM + 8) + 4 * listed_ids + b * t * hq * (4 * HEAD_DIM + 4), "flops": 4 * HEAD_DIM * n * t * (hq // h)}
    if kind == "accumulate":
        n = sum(_lens(case)) * case["draft_layers"]
        return {"bytes": n * 4 * (case["heads"] * case["gamma"] + 2 * case["groups"]), "flops": n * case["heads"] * case["gamma"]}
    # a weight that stays moves if it lies behind the budget: about a share (ctx - budget) / ctx of those that stay
    moves = sum((n - case["budget"]) * case["budget"] / n for n in _lens(case) if n > case["budget"])
    row = 2 * HEAD_DIM if case["bits"] == 16 else HEAD_DIM // 2 + 4
    weights = sum(_lens(case)) * case["groups"] * 4 * (4 if case["positions"] else 2)
    return {"bytes": int(moves) * h * 2 * case["layers"] * 2 * row + weights + int(moves) * case["groups"] * 8, "flops": sum(_lens(case)) * case["groups"]}


# ---- inputs --------------------------------------------------------------------------------------
def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _pack(x):
    """Codes and (scale, zero) of rows of 128 16-bit values."""
    f = x.float()
    lo, hi = f.amin(-1, keepdim=True), f.amax(-1, keepdim=True)
    s, z = ((hi - lo) / 15).to(x.dtype), lo.to(x.dtype)
    fine = torch.isfinite(hi - lo) & torch.isfinite(f).all(-1, keepdim=True)
    usable = fine & (s.float() >= 2.0 ** -126)
    c = torch.where(usable, ((f - z.float()) / torch.where(usable, s.float(), 1.0)).round().clamp(0, 15), 0.0).to(torch.uint8)
    nan = torch.full_like(s, float("nan"))
    return c[..., 0::2] | (c[..., 1::2] << 4), torch.cat([torch.where(fine, torch.where(usable, s, torch.zeros_like(s)), nan), torch.where(fine, z, nan)], -1)


def _values(codes, params):
    """What codes and (scale, zero) stand for, in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    return params[..., 0:1].float() * c + params[..., 1:2].float()


def _pool(gen, n_pages, page, h, dtype, layout, fill=True):
    """An empty or a filled 4-bit pool: codes [pages, 2, page, heads, 64], (scale, zero) [pages, 2, page, heads, 2]."""
    shape = (n_pages, 2, h, page) if layout == "head" else (n_pages, 2, page, h)
    codes = torch.zeros(*shape, HEAD_DIM // 2, dtype=torch.uint8, device=DEV)
    params = torch.zeros(*shape, 2, dtype=dtype, device=DEV)
    if fill:
        offset = torch.randn(HEAD_DIM, generator=gen, device=DEV)  # keys have channels of their own level, values are smaller
        x = torch.randn(*shape, HEAD_DIM, generator=gen, device=DEV)
        x[:, 0] += offset
        x[:, 1] *= 0.5
        codes, params = _pack(x.to(dtype))
    return (codes.transpose(2, 3), params.transpose(2, 3)) if layout == "head" else (codes, params)


def _table(gen, case):
    pps = _pages_per_seq(case)
    return torch.randperm(case["batch"] * pps, generator=gen, device=DEV).to(torch.int32).view(case["batch"], pps)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    kind, b, pps = case["kind"], case["batch"], 0
    s = {"case": case}
    if kind in ("append", "verify", "evict"):
        pps = _pages_per_seq(case)
        s["pages_per_seq"] = pps
    if kind == "append":
        h, t, dt = case["kv_heads"], case["tokens"], DTYPES[case["dtype"]]
        # K and V lie beside the queries in the output of one projection
        x = torch.randn(b, t, 2 + 2, h, HEAD_DIM, generator=gen, device=DEV).to(dt)
        s["k"], s["v"] = x[:, :, 2], x[:, :, 3]
        s["codes"], s["params"] = _pool(gen, b * pps, case["page"], h, dt, case["layout"], fill=False)
        s["table"] = _table(gen, case)
        s["start"], s["n_new"] = _ints([case["start"]] * b), _ints(_new_tokens(case))
        s["k_back"], s["v_back"] = torch.zeros(b, t, h, HEAD_DIM, dtype=dt, device=DEV), torch.zeros(b, t, h, HEAD_DIM, dtype=dt, device=DEV)
    elif kind == "verify":
        dt = DTYPES[case["dtype"]]
        s["codes"], s["params"] = _pool(gen, b * pps, case["page"], case["kv_heads"], dt, case["layout"])
        s["table"] = _table(gen, case) if case["paged"] else None
        s["q"] = (1.5 * torch.randn(b, case["n_q"], case["q_heads"], HEAD_DIM, generator=gen, device=DEV)).to(dt)
        s["kv_len"] = _ints(_lens(case))
        s["idx"] = s["counts"] = None
        if not case["dense"]:
            g, n = case["groups"], case["ctx"]
            counts, inside = _ints(_kept(case)), torch.arange(n, device=DEV) < s["kv_len"][:, None, None]
            # any `count` positions of the context, ascending
            r = torch.where(inside, torch.rand(b, g, n, generator=gen, device=DEV), 2.0).argsort(-1)
            r = torch.where(torch.arange(n, device=DEV) < counts[..., None], r, n).sort(-1).values
            s["idx"], s["counts"] = torch.where(r < n, r, 0).to(torch.int32).contiguous(), counts
    elif kind == "accumulate":
        d, g, n = case["draft_layers"], case["groups"], case["ctx"]
        s["kv_len"] = _ints(_lens(case))
        x = 3.0 * torch.randn(d, b, case["heads"], case["gamma"], -(-n // 4) * 4, generator=gen, device=DEV)
        x = torch.where(torch.arange(x.shape[-1], device=DEV) < s["kv_len"][:, None, None, None], x, float("-inf"))
        s["probs"] = torch.softmax(x, -1)
        s["maps"] = list(s["probs"].unbind(0))
        s["old"] = torch.rand(d, b, g, x.shape[-1], generator=gen, device=DEV) * (case["heads"] / g / n)
        s["new"] = torch.zeros_like(s["old"])
        s["head_group"] = [i * g // case["heads"] for i in range(case["heads"])] if g > 1 else None
    else:
        g, n, h, m = case["groups"], case["ctx"], case["kv_heads"], _move_stride(case)
        s["kv_len"] = _ints(_lens(case))
        s["table"] = _table(gen, case)
        w = torch.exp(2.5 * torch.randn(1, b, g, n, generator=gen, device=DEV))
        s["scores"] = torch.floor(w * 8) / 8 if case["ties"] else w
        s["scores_out"] = torch.zeros_like(w)
        s["positions"] = s["positions_out"] = s["seq_len"] = None
        if case["positions"]:
            # half of what there was is gone already, and rows have been moved
            r = torch.rand(1, b, g, 2 * n, generator=gen, device=DEV)
            r = torch.where(torch.arange(2 * n, device=DEV) < 2 * s["kv_len"][:, None, None], r, 2.0).argsort(-1)
            s["positions"], s["seq_len"] = r[..., :n].to(torch.int32).contiguous(), 2 * s["kv_len"]
            s["positions_out"] = torch.zeros_like(s["positions"])
        s["src"], s["dst"] = (torch.full((1, b, g, m), -1, dtype=torch.int32, device=DEV) for _ in range(2))
        if case["bits"] == 16:
            x = torch.randint(-30000, 30000, (case["layers"], b * pps, 2, case["page"], h, HEAD_DIM), generator=gen, device=DEV, dtype=torch.int16)
            s["pools"], s["params"] = x.bfloat16(), None
        else:
            x = torch.randint(0, 256, (case["layers"], b * pps, 2, h, case["page"], HEAD_DIM // 2), generator=gen, device=DEV, dtype=torch.uint8)
            s["pools"] = x.transpose(3, 4)
            s["params"] = torch.randn(case["layers"], b * pps, 2, h, case["page"], 2, generator=gen, device=DEV).bfloat16().transpose(3, 4)
        s["pool_list"] = list(s["pools"].unbind(0))
        s["params_list"] = None if s["params"] is None else list(s["params"].unbind(0))
    return s


# ---- plain forms -----------------------------------------------------------------------------------
def _place(s, pos):
    """(page, slot) of positions [batch, ...]."""
    page = s["case"]["page"]
    at = torch.div(pos, page, rounding_mode="floor").long()
    if s["table"] is None:
        first = torch.arange(pos.shape[0], device=pos.device).view(-1, *[1] * (pos.dim() - 1)) * s["pages_per_seq"]
        return first + at, (pos % page).long()
    return torch.gather(s["table"].long(), 1, at.flatten(1)).view(pos.shape), (pos % page).long()


def _plain_append(s):
    t = s["k"].shape[1]
    real = torch.arange(t, device=DEV) < s["n_new"][:, None]
    codes, params = _pack(torch.stack([s["k"], s["v"]], 2))  # [batch, token, 2, head, ...]
    page, slot = _place(s, s["start"][:, None] + torch.arange(t, device=DEV))
    c, p = s["codes"].permute(0, 2, 1, 3, 4), s["params"].permute(0, 2, 1, 3, 4)
    # the padding's places keep what they hold
    c[page, slot] = torch.where(real[:, :, None, None, None], codes, c[page, slot])
    p[page, slot] = torch.where(real[:, :, None, None, None], params, p[page, slot])
    back = _values(c[page, slot], p[page, slot]).to(s["k"].dtype)
    keep = real[:, :, None, None]
    return {"k": torch.where(keep, back[:, :, 0], s["k_back"]), "v": torch.where(keep, back[:, :, 1], s["v_back"])}


def _plain_verify(s):
    case, q = s["case"], s["q"]
    b, t, hq, d = q.shape
    h, g = case["kv_heads"], 1 if case["dense"] else case["groups"]
    tail, lens = case["tail"], s["kv_len"]
    if case["dense"]:
        pos = torch.arange(case["ctx"], device=DEV).expand(b, 1, -1)
        live = pos < lens[:, None, None]
    else:
        longest = max(map(max, _kept(case)))
        pos = s["idx"][..., :longest].long()
        live = torch.arange(longest, device=DEV) < s["counts"][..., None]
    j = torch.arange(tail, device=DEV)
    pos = torch.cat([torch.where(live, pos, 0), (lens[:, None, None] + j).expand(b, g, -1)], -1)
    live = torch.cat([live, torch.ones(b, g, tail, dtype=torch.bool, device=DEV)], -1)
    page, slot = _place(s, pos)
    if g == 1:
        page, slot = page.expand(b, h, -1), slot.expand(b, h, -1)
        live = live.expand(b, h, -1)
    head = torch.arange(h, device=DEV)[None, :, None]
    rows = q.float().view(b, t, h, hq // h, d).permute(0, 2, 1, 3, 4).reshape(b, h, -1, d)
    k = _values(s["codes"][page, 0, slot, head], s["params"][page, 0, slot, head])  # [batch, head, position, 128]
    score = torch.matmul(rows, k.transpose(-1, -2)) / math.sqrt(d)
    del k
    # a query sees the in-flight tokens up to itself
    seen = torch.cat([torch.ones(t, pos.shape[-1] - tail, dtype=torch.bool, device=DEV), j <= torch.arange(t, device=DEV)[:, None] + (tail - t)], -1)
    score = score.masked_fill(~(live[:, :, None] & seen.repeat_interleave(hq // h, 0)), float("-inf"))
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - torch.where(torch.isinf(top), 0.0, top))
    del score
    total = e.sum(-1, keepdim=True)
    v = _values(s["codes"][page, 1, slot, head], s["params"][page, 1, slot, head])
    out = torch.matmul(e, v) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(-1)

    def back(x):
        return x.view(b, h, t, hq // h, *x.shape[3:]).transpose(1, 2).reshape(b, t, hq, *x.shape[3:])

    return {"out": back(out).to(q.dtype), "lse": back(lse)}


def _plain_accumulate(s):
    case = s["case"]
    total = s["probs"].sum(3, dtype=torch.float64)
    if s["head_group"] is not None:
        feeds = torch.tensor(s["head_group"], device=DEV) == torch.arange(case["groups"], device=DEV)[:, None]
        total = torch.matmul(feeds.double(), total)
    else:
        total = total.sum(2, keepdim=True)
    new = (case["decay"] * s["old"].double() + total).float()
    inside = torch.arange(new.shape[-1], device=DEV) < s["kv_len"][:, None, None]
    return {"weight": torch.where(inside, new, s["new"])}


def _ascending(mask, room):
    """The places where `mask` holds, ascending, and -1 behind them."""
    n = mask.shape[-1]
    to = torch.where(mask, mask.cumsum(-1) - 1, room)
    got = torch.full((*mask.shape[:-1], room + 1), -1, dtype=torch.int32, device=DEV)
    return got.scatter_(-1, to, torch.arange(n, device=DEV, dtype=torch.int32).expand(mask.shape))[..., :room].contiguous()


def _plain_evict(s):
    case, w, lens = s["case"], s["scores"], s["kv_len"][:, None, None]
    n, room = w.shape[-1], s["src"].shape[-1]
    slot = torch.arange(n, device=DEV)
    pos = slot.expand(w.shape) if s["positions"] is None else s["positions"]
    end = lens if s["seq_len"] is None else s["seq_len"][:, None, None]
    inside, new_len = slot < lens, torch.clamp(lens, max=case["budget"])
    # the sinks and the newest first, then by weight, lower slots first among equals
    rank = torch.where((pos < case["sink"]) | (pos >= end - case["recent"]), 2, 1)
    rank = torch.where(inside, rank, 0)
    by_weight = torch.sort(w, dim=-1, descending=True, stable=True).indices
    order = by_weight.gather(-1, torch.sort(rank.gather(-1, by_weight), dim=-1, descending=True, stable=True).indices)
    stays = torch.zeros(w.shape, dtype=torch.bool, device=DEV).scatter_(-1, order, (slot < new_len).expand(w.shape).contiguous())
    from_, into = stays & (slot >= new_len), ~stays & (slot < new_len)
    src, dst, moves = _ascending(from_, room), _ascending(into, room), from_.sum(-1, dtype=torch.int32)
    # a place in the lists that no move uses copies the last row, which nothing is moved into, onto itself
    live = torch.arange(room, device=DEV) < moves[..., None]
    idle = torch.clamp(lens - 1, min=0)
    a, z = torch.where(live, src, idle), torch.where(live, dst, idle)
    compact = w.scatter(-1, z.long(), w.gather(-1, a.long()))
    found = {"src": src, "dst": dst, "moves": moves, "new_len": new_len.view(-1).to(torch.int32),
             "weight": torch.where(slot < new_len, compact, 0.0)}
    if s["positions"] is not None:
        found["positions"] = torch.where(slot < new_len, pos.scatter(-1, z.long(), pos.gather(-1, a.long())), s["positions_out"])
    (ap, asl), (zp, zsl) = _place(s, a[0]), _place(s, z[0])  # [batch, group, move]
    head = torch.arange(case["groups"], device=DEV)[None, :, None]
    for name in ("pools", "params"):
        if s[name] is not None:
            if case["groups"] == 1:
                rows = s[name].permute(1, 3, 0, 2, 4, 5)
                rows[zp[:, 0], zsl[:, 0]] = rows[ap[:, 0], asl[:, 0]]
            else:
                rows = s[name].permute(1, 3, 4, 0, 2, 5)
                rows[zp, zsl, head] = rows[ap, asl, head]
            found[name] = s[name]
    return found


# ---- one pass ----------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"append": _plain_append, "verify": _plain_verify, "accumulate": _plain_accumulate, "evict": _plain_evict}[kind](s)
    import paper_2510_27641_b200 as sa
    if kind == "append":
        sa.kv4_append(s["k"], s["v"], s["codes"], s["params"], s["start"], n_new=s["n_new"], block_table=s["table"])
        k, v, _ = sa.kv4_read(s["codes"], s["params"], s["start"], n=s["n_new"], block_table=s["table"], k=s["k_back"], v=s["v_back"])
        return {"k": k, "v": v}
    if kind == "verify":
        out, lse, _ = sa.kv4_verify(s["q"], s["codes"], s["params"], s["kv_len"], block_table=s["table"], pages_per_seq=s["pages_per_seq"],
                                    idx=s["idx"], counts=s["counts"], n_groups=case["groups"], dense=case["dense"], tail_len=case["tail"])
        return {"out": out, "lse": lse}
    if kind == "accumulate":
        new, _ = sa.accumulate_attention(s["maps"], s["kv_len"], s["old"], n_groups=case["groups"],
                                         head_group=s["head_group"], decay=case["decay"], out=s["new"])
        return {"weight": new}
    src, dst, moves, new_len = sa.evict(s["scores"], s["kv_len"], case["budget"], n_sink=case["sink"], n_recent=case["recent"],
                                        positions=s["positions"], seq_len=s["seq_len"], src=s["src"], dst=s["dst"],
                                        scores_out=s["scores_out"], positions_out=s["positions_out"])
    sa.move_rows(s["pool_list"], src[0], dst[0], moves[0], params=s["params_list"], block_table=s["table"])
    found = {"src": src, "dst": dst, "moves": moves, "new_len": new_len, "weight": s["scores_out"], "pools": s["pools"]}
    if s["params"] is not None:
        found["params"] = s["params"]
    if s["positions"] is not None:
        found["positions"] = s["positions_out"]
    return found


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------
def _row64(s, b, side, pos, head):
    """Rows of a 4-bit pool, one position after the other, in 64 bits."""
    page = s["case"]["page"]
    of = s["table"][b].long()[pos // page] if s["table"] is not None else b * s["pages_per_seq"] + pos // page
    raw, p = s["codes"][of, side, pos % page, head].to(torch.int64), s["params"][of, side, pos % page, head].double()
    got = torch.empty(len(pos), HEAD_DIM, dtype=torch.float64, device=DEV)
    got[:, 0::2], got[:, 1::2] = (raw % 16).double(), (raw // 16).double()
    return got * p[:, :1] + p[:, 1:]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        found = {}
        for name in ("k", "v"):
            x = s[name].double()
            low = x.min(-1, keepdim=True).values
            scale = ((x.max(-1, keepdim=True).values - low) / 15).to(s[name].dtype).double()
            y = low + scale * torch.clamp(torch.round((x - low) / scale), max=15)
            for i, n in enumerate(_new_tokens(case)):
                y[i, n:] = 0
            found[name] = y
        return found
    if case["kind"] == "verify":
        b, t, hq, d = s["q"].shape
        h, lens = case["kv_heads"], _lens(case)
        out, lse = torch.zeros(b, t, hq, d, dtype=torch.float64, device=DEV), torch.full((b, t, hq), float("-inf"), dtype=torch.float64, device=DEV)
        kept = None if case["dense"] else _kept(case)
        for i in range(b):
            for head in range(h):
                g = head if case["groups"] > 1 else 0
                ctx = torch.arange(lens[i], device=DEV) if case["dense"] else s["idx"][i, g, :kept[i][g]].long()
                pos = torch.cat([ctx, lens[i] + torch.arange(case["tail"], device=DEV)])
                keys, values = _row64(s, i, 0, pos, head), _row64(s, i, 1, pos, head)
                mine = slice(head * (hq // h), (head + 1) * (hq // h))
                for row in range(t):
                    n = len(ctx) + max(0, min(case["tail"], row + case["tail"] - t + 1))
                    if n:
                        x = s["q"][i, row, mine].double() @ keys[:n].T / math.sqrt(d)
                        lse[i, row, mine] = torch.logsumexp(x, -1)
                        out[i, row, mine] = torch.softmax(x, -1) @ values[:n]
        return {"out": out, "lse": lse}
    if case["kind"] == "accumulate":
        new = torch.zeros(s["old"].shape, dtype=torch.float64, device=DEV)
        for i, n in enumerate(_lens(case)):
            new[:, i, :, :n] = case["decay"] * s["old"][:, i, :, :n].double()
            for head in range(case["heads"]):
                g = s["head_group"][head] if s["head_group"] is not None else slice(None)
                new[:, i, g, :n] += s["probs"][:, i, head, :, :n].double().sum(1) if s["head_group"] is not None else s["probs"][:, i, head, :, :n].double().sum(1)[:, None]
        return {"weight": new}
    # rows are copied as they are; what is left of the weights, one list after the other
    left = torch.zeros(s["scores"].shape, dtype=torch.float64, device=DEV)
    for i, n in enumerate(_lens(case)):
        for g in range(case["groups"]):
            w = s["scores"][0, i, g, :n].double().cpu().numpy()
            pos, end = (np.arange(n), n) if s["positions"] is None else (s["positions"][0, i, g, :n].cpu().numpy(), 2 * n)
            safe = (pos < case["sink"]) | (pos >= end - case["recent"])
            m = min(n, case["budget"])
            stays = np.zeros(n, bool)
            stays[np.lexsort((np.arange(n), -w, ~safe))[:m]] = True
            w[np.flatnonzero(~stays[:m])] = w[m + np.flatnonzero(stays[m:])]
            left[0, i, g, :m] = torch.from_numpy(w[:m]).to(DEV)
    return {"weight": left}
