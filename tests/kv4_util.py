"""References of the 4-bit cache's operators in 64 bits, and inputs, for the tests."""
from __future__ import annotations

import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def quantise(x: torch.Tensor):
    """(codes, params) of rows x [..., 128] in bf16 / fp16, as include/specattn.h defines them (CPU)."""
    f = x.float()
    lo, hi = f.amin(-1), f.amax(-1)
    span = hi - lo
    fine = torch.isfinite(f).all(-1) & torch.isfinite(span)
    s = (span / torch.tensor(15.0)).to(x.dtype)
    s = torch.where(s.float() < 2.0 ** -126, torch.zeros_like(s), s)
    c = torch.zeros(x.shape, dtype=torch.int64)
    ok = fine & (s.float() > 0)
    c[ok] = ((f - lo[..., None])[ok] / s.float()[..., None][ok]).round().clamp(max=15).to(torch.int64)
    nan = torch.full_like(s, float("nan"))
    params = torch.stack([torch.where(fine, s, nan), torch.where(fine, lo.to(x.dtype), nan)], -1)
    return (c[..., 0::2] + 16 * c[..., 1::2]).to(torch.uint8), params


def values(codes: torch.Tensor, params: torch.Tensor) -> torch.Tensor:
    """What rows of a 4-bit cache stand for, in 64 bits (CPU)."""
    c = torch.empty(*codes.shape[:-1], 128, dtype=torch.float64)
    c[..., 0::2], c[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    return c * params[..., 0:1].double() + params[..., 1:2].double()


def make_pool(gen, n_pages, page, heads, dtype, layout="head", spread=1.0):
    """A filled pool on the CPU: (codes, params) in the given memory order, and its values in 64 bits."""
    shape = (n_pages, 2, heads, page, 128) if layout == "head" else (n_pages, 2, page, heads, 128)
    codes, params = quantise((torch.randn(*shape, generator=gen) * spread).to(dtype))
    if layout == "head":
        codes, params = codes.transpose(2, 3), params.transpose(2, 3)
    return codes, params


def row_at(table, pages_per_seq, page, b, pos):
    at = pos // page
    return (int(table[b, at]) if table is not None else b * pages_per_seq + at), pos % page


def verify64(q, codes, params, lists, lens, tail, page, table, pages_per_seq, sm_scale=0.0):
    """(out, lse, tolerance of out, tolerance of lse): attention in 64 bits, position lists [b][head], over CPU tensors.

    The tolerances are those of the operation's roundings, with u = 2^-24 and the largest scale t of the
    rows attended: a weight is rounded to 11 bits (half a step of 2^-11 relative; 2^-30 t of its unit absolutely where
    it is subnormal) and multiplies a code at most 8 from the middle; a score's product runs over 128 terms of at
    most |q| (15 s + |z|) in binary32 (at most 16 roundings of u, truncated ones counted twice); an error d of all scores
    changes an output by at most 2 d max |v| and the logarithm by d."""
    b, t, hq, d = q.shape
    h = codes.shape[3]
    grp, val = hq // h, values(codes, params)
    out, lse = torch.zeros(b, t, hq, d, dtype=torch.float64), torch.full((b, t, hq), float("-inf"), dtype=torch.float64)
    tol_out, tol_lse = torch.zeros(b, t, hq, 1, dtype=torch.float64), torch.zeros(b, t, hq, dtype=torch.float64)
    scale = sm_scale or 1 / math.sqrt(d)
    half = HALF_STEP[q.dtype]
    for i in range(b):
        for head in range(h):
            mine = slice(head * grp, (head + 1) * grp)
            for row in range(t):
                n_tail = max(0, min(tail, row + tail - t + 1))
                pos = [int(x) for x in lists[i][head]] + [lens[i] + j for j in range(n_tail)]
                if not pos:
                    continue
                at = torch.tensor([row_at(table, pages_per_seq, page, i, x) for x in pos])
                k, v = val[at[:, 0], 0, at[:, 1], head], val[at[:, 0], 1, at[:, 1], head]
                x = q[i, row, mine].double() @ k.T * scale
                out[i, row, mine], lse[i, row, mine] = torch.softmax(x, -1) @ v, torch.logsumexp(x, -1)
                step = params[at[:, 0], 1, at[:, 1], head, 0].double().abs().max()
                kp = params[at[:, 0], 0, at[:, 1], head].double().abs()
                off = scale * q[i, row, mine].double().abs().sum(-1) * (15 * kp[:, 0] + kp[:, 1]).max() * 2.0 ** -20
                tol_lse[i, row, mine] = off + 2.0 ** -20 * (1 + lse[i, row, mine].abs())
                tol_out[i, row, mine, 0] = (8 * step * (2.0 ** -11 + len(pos) * 2.0 ** -30) + (2 * off + 2.0 ** -20) * v.abs().max()
                                            + half * out[i, row, mine].abs().amax(-1))
    return out, lse, tol_out, tol_lse
