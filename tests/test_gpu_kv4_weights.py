"""How well kv4_verify holds the weights of its second product, the probabilities times the scales of V rows."""
import pytest
import torch

from kv4_util import verify64
from test_gpu_kv4 import DEV, _case, _run

pytestmark = pytest.mark.gpu
WIDTHS = [("auto", 1, 4), ("auto", 1, 16), ("auto", 2, 8), ("auto", 5, 4), ("auto", 2, 16), ("auto", 4, 16), ("mma.sync", 6, 16), ("auto", 8, 16),
          ("mma.sync", 6, 24), ("tcgen05", 6, 24), ("tcgen05", 5, 32), ("auto", 8, 32)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("engine,T,Hq", WIDTHS)
def test_weights_keep_the_bits_of_binary32_outputs(engine, T, Hq, dtype):
    """Short lists and queries so small that the scores' own rounding is out of the way.

    The tolerance, with t the largest scale of the rows attended: a weight in two parts of 11 bits is off by 2^-21 of it or by
    2^-29 t; it multiplies a code of at most 15.  The matrix units add 16 positions at a time and cut off what lies
    below 2^-23 of a sum that is at most 15 t: for up to 128 positions, two parts and the joins behind them, 32 times.
    The scores' part is that of verify64, whose terms for weights of 11 bits, and for outputs of 16, are taken out."""
    c = _case(111, 3, T, Hq, 4, [90, 40, 200], [40, 17, 64], dtype=dtype, q_scale=2.0 ** -6)
    out = torch.full(c["q"].shape, float("nan"), device=DEV)
    _run(c, engine=engine, out=out)
    want, _, tol, _ = verify64(c["q"], c["codes"], c["params"], c["lists"], c["lens"], 0, c["page"], c["table"], c["pps"])
    half = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    grp = Hq // 4
    for b in range(3):
        for head in range(4):
            mine = slice(head * grp, (head + 1) * grp)
            pos = c["lists"][b][head]
            n, t = len(pos), max(float(c["params"][int(c["table"][b, p // 16]), 1, p % 16, head, 0].double().abs()) for p in pos)
            near = tol[b, :, mine] - half * want[b, :, mine].abs().amax(-1, keepdim=True) - 8 * t * (2.0 ** -11 + n * 2.0 ** -30)
            near = near + 15 * t * (2.0 ** -21 + n * 2.0 ** -29 + 32 * 2.0 ** -23)
            off = (out[b, :, mine].cpu().double() - want[b, :, mine]).abs()
            assert torch.all(off <= near), float((off / near).max())


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 16, 4), (3, 1, 1), (5, 4, 4)])
def test_a_query_of_nan_or_infinity_spoils_no_other_of_a_few(T, Hq, Hkv):
    """Up to four rows to a KV head: the columns of the rows that there are not hold sums of their own."""
    c = _case(117, 2, T, Hq, Hkv, [200, 40], [150, 33])
    out, lse, _ = _run(c)
    for bad in (float("nan"), float("inf")):
        q = c["q"].clone()
        q[0, 0, 0, 17] = bad
        out2, lse2, _ = _run(dict(c, q=q))
        assert torch.all(torch.isnan(out2[0, 0, 0]))
        out2[0, 0, 0], lse2[0, 0, 0] = out[0, 0, 0], lse[0, 0, 0]
        assert torch.equal(out2, out) and torch.equal(lse2, lse)
