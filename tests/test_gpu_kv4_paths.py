"""Which of its two implementations kv4_verify takes by itself, and tcgen05 at all the widths that it runs."""
import pytest
import torch

from test_gpu_kv4 import LENGTHS, _case, _check, _run

pytestmark = pytest.mark.gpu
WIDTHS = [(5, 10, 2), (7, 16, 4), (8, 32, 8), (33, 1, 1), (41, 1, 1), (6, 32, 4)]   # rows: 25, 28, 32, 33, 41, 48


@pytest.mark.parametrize("T,Hq,Hkv", WIDTHS)
@pytest.mark.parametrize("lens,counts", LENGTHS)
def test_lists_on_tcgen05(lens, counts, T, Hq, Hkv):
    c = _case(141, len(lens), T, Hq, Hkv, lens, counts, dtype=torch.float16 if T % 2 else torch.bfloat16)
    out, lse, _ = _run(c, "tcgen05")
    _check(c, out, lse)


@pytest.mark.parametrize("T,Hq,Hkv", WIDTHS)
@pytest.mark.parametrize("lens,tail,page,layout", [([700, 0, 333], 1, 24, "slot"), ([257, 31], 60, 16, "head"), ([9000, 1], 5, 32, "head")])
def test_everything_and_a_tail_on_tcgen05(lens, tail, page, layout, T, Hq, Hkv):
    c = _case(142, len(lens), T, Hq, Hkv, lens, None, dense=True, tail=tail, page=page, layout=layout)
    out, lse, _ = _run(c, "tcgen05")
    _check(c, out, lse)


@pytest.mark.parametrize("T,Hq", [(14, 4), (16, 4), (20, 4), (24, 4)])   # 28, 32, 40, 48 rows
def test_lists_take_mma_sync_whatever_their_room(T, Hq):
    """A selection's lists have room for the whole context and hold a few per cent of it."""
    c = _case(143, 4, T, Hq, 2, [30000, 90000, 100, 70000], [300, 900, 50, 700])
    out, lse, _ = _run(c)
    mma, tc = _run(c, "mma.sync"), _run(c, "tcgen05")
    assert torch.equal(out, mma[0]) and torch.equal(lse, mma[1]) and not torch.equal(lse, tc[1])
    few = dict(c, q=c["q"][:, :2].contiguous())
    _check(few, out[:, :2], lse[:, :2])
    _check(few, tc[0][:, :2], tc[1][:, :2])


@pytest.mark.parametrize("T,Hq,least", [(14, 4, False), (14, 4, True), (20, 4, False), (20, 4, True), (24, 4, False), (24, 4, True), (12, 4, False)])
def test_long_tables_take_tcgen05(T, Hq, least):
    """28, 40, 48 and 24 rows, at either side of the limit of 64 (40 rows: 32) chunks to an SM."""
    limit = (32 if T == 20 else 64) * torch.cuda.get_device_properties(0).multi_processor_count
    page = 32
    per_seq = limit // (2 * 2) + (1 if least else -2 if T != 12 else 5000)   # of two sequences' two heads; a chunk to a page
    c = _case(144, 2, T, Hq, 2, [40, 33], None, dense=True, page=page)
    c["pps"], c["table"] = per_seq, torch.cat([c["table"], torch.zeros(2, per_seq - c["table"].shape[1], dtype=torch.int32)], 1).contiguous()
    out, lse, _ = _run(c)
    engine = "tcgen05" if least else "mma.sync"
    if T != 12:
        forced, other = _run(c, engine), _run(c, "mma.sync" if least else "tcgen05")
        assert torch.equal(lse, forced[1]) and not torch.equal(lse, other[1])
    _check(c, out, lse)


@pytest.mark.parametrize("T,Hq", [(24, 1), (7, 7), (8, 8), (1, 1)])
def test_tcgen05_refuses_what_it_does_not_run(T, Hq):
    """24, 49, 64 rows and one."""
    import paper_2510_27641_b200 as sa
    c = _case(145, 1, T, Hq, 1, [40], [20])
    with pytest.raises(sa.SpecAttnError):
        _run(c, "tcgen05")
