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


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_long_sums_are_held_as_well_as_the_16_bit_operators(engine):
    """131072 positions, outputs in binary32, on the same engine of both operators and values of the same distribution.

    Both add up the same number of products in the same units, which cut off towards zero; a sum whose terms have a mean
    loses a part of it each time, one around zero gains as often as it loses.  Errors are root mean squares of the
    output's; a code lies up to 15 steps from where its tile counts from and a weight comes in two parts: three times
    the 16-bit operator's error."""
    import paper_2510_27641_b200 as sa
    gen = torch.Generator(device=DEV).manual_seed(119)
    n, page, T, Hq, Hkv = 131072, 16, 5, 64, 8
    grp = Hq // Hkv
    x = torch.randn(2, n, Hkv, 128, generator=gen, device=DEV)
    x[0] += torch.randn(128, generator=gen, device=DEV)
    x[1] *= 0.5
    x = x.to(torch.bfloat16)
    codes, params = sa.kv4_cache(n // page, page, Hkv)
    start, lens = torch.zeros(1, dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV)
    sa.kv4_append(x[0][None], x[1][None], codes, params, start, pages_per_seq=n // page)
    pool = torch.stack(list(x), 0).view(2, n // page, page, Hkv, 128).transpose(0, 1).contiguous()
    q = (1.5 * torch.randn(1, T, Hq, 128, generator=gen, device=DEV)).to(torch.bfloat16)
    flags = {"mma.sync": sa.VERIFY_ENGINE_MMA_SYNC, "tcgen05": sa.VERIFY_ENGINE_TCGEN05}[engine]
    kw = dict(pages_per_seq=n // page, dense=True, flags=flags)
    out4, out16 = (torch.empty(1, T, Hq, 128, device=DEV) for _ in range(2))
    sa.kv4_verify(q, codes, params, lens, out=out4, **kw)
    sa.sparse_verify(q, pool, lens, out=out16, **kw)

    def error(out, k, v):
        want = torch.softmax(q[0, :, :grp].double() @ k.T / 128 ** 0.5, -1) @ v
        return float((out[0, :, :grp].double() - want).norm() / want.norm())

    def stands_for(side):   # of head 0
        c, p = codes[:, side, :, 0].reshape(n, 64), params[:, side, :, 0].reshape(n, 2).double()
        return torch.stack([c % 16, c // 16], -1).flatten(-2).double() * p[:, :1] + p[:, 1:]

    e4, e16 = error(out4, stands_for(0), stands_for(1)), error(out16, x[0, :, 0].double(), x[1, :, 0].double())
    assert e4 <= 3 * e16, (e4, e16)
