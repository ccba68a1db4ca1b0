"""Attention over the 4-bit cache where scores and scales are far from one: the references are those of the other tests."""
import pytest
import torch

from kv4_util import quantise
from test_gpu_kv4 import DEV, _case, _check, _gen, _more, _run

pytestmark = pytest.mark.gpu


def _liked(c, gen, like, of_positions=None):
    """K rows that every query scores near `like` (natural units), V rows around zero; of_positions: a factor for each."""
    b, t, hq, _ = c["q"].shape
    heads, pages = c["codes"].shape[3], c["codes"].shape[0]
    u = torch.randn(128, generator=gen).sign()
    c["q"] = (u + 0.3 * torch.randn(b, t, hq, 128, generator=gen)).to(c["q"].dtype)
    x = torch.randn(pages, 2, c["page"], heads, 128, generator=gen)
    if of_positions is None:
        x[:, 0] += like / 128 ** 0.5 * u
    else:
        for i in range(b):
            for at in range(c["table"].shape[1]):
                pos = torch.arange(c["page"]) + at * c["page"]
                x[int(c["table"][i, at]), 0] += like / 128 ** 0.5 * of_positions(pos)[:, None, None] * u
    c["codes"], c["params"] = quantise(x.to(c["q"].dtype))


@pytest.mark.parametrize("like", [-150.0, -1000.0])
@pytest.mark.parametrize("lens,counts,tail", [
    ([1], [1], 0),
    ([40, 7], [0, 0], 5),            # the tail alone: the first query sees one row of it
    ([70, 64], [33, 32], 5),         # a row behind a chunk's end, and the tail behind that
    ([9000, 300], [8000, 250], 0),   # cut into many parts
])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_scores_far_below_zero(engine, dtype, lens, counts, tail, like):
    """The first maximum that a warp meets is far below zero; there is nothing yet that it could scale."""
    c = _case(101, len(lens), 5, _more(engine, 16, 32), 4, lens, counts, tail=tail, dtype=dtype)
    _liked(c, _gen(102), like)
    out, lse, _ = _run(c, engine=engine)
    assert torch.all(lse < like / 2)
    _check(c, out, lse)


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 8, 8), (1, 32, 8), (9, 1, 1), (8, 8, 1)])
def test_scores_far_below_zero_at_other_widths(T, Hq, Hkv):
    c = _case(103, 2, T, Hq, Hkv, [700, 3], [500, 2], tail=T)
    _liked(c, _gen(104), -200.0)
    out, lse, _ = _run(c)
    _check(c, out, lse)


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_scores_that_fall_along_the_list(engine):
    """From zero to -400: what comes first outweighs all that follows."""
    c = _case(105, 1, 5, _more(engine, 8, 16), 2, [2000], None, dense=True)
    _liked(c, _gen(106), -400.0, lambda pos: pos / 2000.0)
    out, lse, _ = _run(c, engine=engine)
    _check(c, out, lse)
