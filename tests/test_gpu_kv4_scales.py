"""V rows of the smallest scales, and scores and scales that fall along the list."""
import pytest
import torch

from kv4_util import quantise
from test_gpu_kv4 import DEV, _case, _check, _gen, _more, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("small", [-100, -112, -118, -124])
@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_rows_of_the_smallest_scales(engine, small):
    """V rows whose scales reach down to 2^-126, the least that a row is stored with."""
    c = _case(113, 2, 5, _more(engine, 16, 32), 4, [300, 50], [200, 33], tail=5)
    x = torch.randn(c["codes"].shape[0], 2, 16, 4, 128, generator=_gen(114))
    x[:, 1] *= 2.0 ** small
    c["codes"], c["params"] = quantise(x.to(torch.bfloat16))
    scales = c["params"][:, 1, ..., 0].float()
    assert torch.all((scales == 0) | (scales >= 2.0 ** -126)) and scales.any()
    out = torch.full(c["q"].shape, float("nan"), device=DEV)
    _, lse, _ = _run(c, engine=engine, out=out)
    _check(c, out, lse)


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_scores_and_scales_that_fall(engine):
    """The largest scores and the largest scales come first, by a factor of 2^30 from one end of the list to the other."""
    n = 2000
    c = _case(115, 1, 5, _more(engine, 8, 16), 2, [n], None, dense=True)
    x = torch.randn(c["codes"].shape[0], 2, 16, 2, 128, generator=_gen(115))
    for b in range(c["table"].shape[1]):
        page, pos = int(c["table"][0, b]), n - torch.arange(16) - 16 * b
        x[page, 0] += (pos / 400.0)[:, None, None] * c["q"][0, 0, 0].float().sign()
        x[page, 1] *= (2.0 ** (30.0 * pos / n - 20))[:, None, None]
    c["codes"], c["params"] = quantise(x.to(torch.bfloat16))
    out, lse, _ = _run(c, engine=engine)
    _check(c, out, lse)
