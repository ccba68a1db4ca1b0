"""The 4-bit cache on the GPU, through the package's entry points, against references in 64 bits."""
import math

import pytest
import torch

from kv4_util import make_pool, quantise, values, verify64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _sa():
    import paper_2510_27641_b200 as sa
    return sa


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _table(gen, b, pps):
    return torch.randperm(b * pps, generator=gen).to(torch.int32).view(b, pps)


def _to_gpu(t):
    """The same strides on the GPU."""
    if t.is_contiguous():
        return t.to(DEV)
    return t.transpose(2, 3).contiguous().to(DEV).transpose(2, 3)


# ---- append, read ----------------------------------------------------------------------------------
ROW_CASES = [
    # batch, tokens, heads, page, start, n_new
    (1, 1, 1, 16, [0], None),
    (3, 6, 8, 16, [0, 13, 31], [6, 0, 5]),
    (2, 100, 2, 24, [5, 40], [100, 77]),
    (2, 33, 5, 1, [3, 0], [40, -2]),          # counts beyond the room are clamped
    (1, 700, 8, 64, [60], None),
    (5, 3, 40, 16, [1, 2, 3, 4, 5], None),
]


@pytest.mark.parametrize("layout", ["head", "slot"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch,tokens,heads,page,start,n_new", ROW_CASES)
def test_rows_go_in_and_come_back(batch, tokens, heads, page, start, n_new, dtype, layout):
    sa, gen = _sa(), _gen(7)
    pps = -(-(max(start) + tokens) // page)
    n_pages = batch * pps + 1
    table = _table(gen, batch, pps)
    x = torch.randn(batch, tokens, 3, heads, 128, generator=gen).to(dtype)    # K and V beside something else
    x[0, 0, 1, 0, :] = 1.5                                                    # a constant row
    x[0, 0, 2, 0] = torch.arange(128).to(dtype) / 8                           # values on the borders between codes
    gx = x.to(DEV)
    before_c, before_p = make_pool(gen, n_pages, page, heads, dtype, layout)
    codes, params = _to_gpu(before_c), _to_gpu(before_p)
    assert codes.stride() == before_c.stride() or heads == 1 or page == 1
    counts = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device=DEV)
    status = torch.full((batch,), 77, dtype=torch.int32, device=DEV)
    st = torch.tensor(start, dtype=torch.int32, device=DEV)
    kw = dict(block_table=table.to(DEV), status=status)
    sa.kv4_append(gx[:, :, 1], gx[:, :, 2], codes, params, st, n_new=counts, **kw)
    assert status.tolist() == [0] * batch
    want_c, want_p = before_c.clone(), before_p.clone()
    real = [tokens] * batch if n_new is None else [max(0, min(tokens, n)) for n in n_new]
    for b in range(batch):
        for t in range(real[b]):
            pos = start[b] + t
            at = int(table[b, pos // page]), pos % page
            want_c[at[0], :, at[1]], want_p[at[0], :, at[1]] = quantise(x[b, t, 1:3])
    assert torch.equal(codes.cpu(), want_c)
    assert torch.equal(params.cpu(), want_p)
    # back, into buffers whose rows of the padding stay as they are
    k, v = (torch.full((batch, tokens, heads, 128), 9.0, dtype=dtype, device=DEV) for _ in range(2))
    sa.kv4_read(codes, params, st, n=counts, k=k, v=v, **kw)
    assert status.tolist() == [0] * batch
    for b in range(batch):
        for side, got in ((0, k), (1, v)):
            assert torch.all(got[b, real[b]:] == 9)
            for t in range(real[b]):
                pos = start[b] + t
                at = int(table[b, pos // page]), pos % page
                c = torch.stack([want_c[at[0], side, at[1]] % 16, want_c[at[0], side, at[1]] // 16], -1).flatten(-2).float()
                p = want_p[at[0], side, at[1]].float()
                assert torch.equal(got[b, t].cpu(), (c * p[:, :1] + p[:, 1:]).to(dtype))
    made = sa.kv4_read(codes, params, st, n=counts, n_tokens=tokens, block_table=table.to(DEV))
    for b in range(batch):
        assert torch.equal(made[0][b, :real[b]], k[b, :real[b]]) and torch.equal(made[1][b, :real[b]], v[b, :real[b]])
        assert not made[0][b, real[b]:].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_values_at_the_ends_of_the_type(dtype):
    """Rows of NaN, infinities, the largest and the smallest values, zeros of both signs."""
    sa, big, small = _sa(), torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    rows = torch.zeros(1, 10, 1, 128)
    rows[0, 0, 0, 5] = float("nan")
    rows[0, 1, 0, 127] = float("inf")
    rows[0, 2, 0, 64] = -float("inf")
    rows[0, 3, 0, 0], rows[0, 3, 0, 1] = big, -big       # (bf16: the span is beyond binary32)
    rows[0, 4, 0, :64] = small
    rows[0, 5, 0, 3] = small * 2.0 ** -5
    rows[0, 6, 0, 1] = -0.0
    rows[0, 7, 0] = big
    rows[0, 8, 0] = torch.linspace(100.0, 100.5, 128)
    rows[0, 9, 0] = torch.linspace(-big / 4, big / 4, 128)
    x = rows.to(dtype)
    codes, params = sa.kv4_cache(1, 16, 1, dtype=dtype)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    sa.kv4_append(x.to(DEV), x.to(DEV), codes, params, torch.zeros(1, dtype=torch.int32, device=DEV), pages_per_seq=1, status=status)
    assert status.item() == sa.ROW_INVALID_VALUE
    want_c, want_p = quantise(x[0, :, 0])
    assert torch.equal(codes[0, 0, :10, 0].cpu(), want_c)
    got_p = params[0, 0, :10, 0].cpu()
    assert torch.equal(torch.isnan(got_p), torch.isnan(want_p))
    assert torch.equal(torch.nan_to_num(got_p), torch.nan_to_num(want_p))
    bad = torch.isnan(want_p).all(-1).tolist()
    assert bad[:3] == [True] * 3 and bad[4:] == [False] * 6 and bad[3] == (dtype is torch.bfloat16)


def test_positions_that_no_page_holds_are_skipped_and_reported():
    sa, gen = _sa(), _gen(3)
    x = torch.randn(4, 4, 2, 128, generator=gen).to(torch.bfloat16).to(DEV)
    table = torch.tensor([[0, 1], [2, 9], [3, -1], [4, 5]], dtype=torch.int32, device=DEV)   # page 9 does not exist
    start = torch.tensor([30, 14, 15, -2], dtype=torch.int32, device=DEV)                     # 32 is beyond the table
    codes, params = sa.kv4_cache(6, 16, 2)
    status = torch.zeros(4, dtype=torch.int32, device=DEV)
    sa.kv4_append(x, x, codes, params, start, block_table=table, status=status)
    assert status.tolist() == [sa.ROW_BAD_INDEX] * 4
    written = (params != 0).any(-1).any(-1).any(1).cpu()          # [page, slot]
    want = torch.zeros(6, 16, dtype=torch.bool)
    for page, slot in ((1, 14), (1, 15), (2, 14), (2, 15), (3, 15), (4, 0), (4, 1)):
        want[page, slot] = True
    assert torch.equal(written, want)
    k = torch.full((4, 4, 2, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    sa.kv4_read(codes, params, start, block_table=table, k=k, v=v, status=status)
    assert status.tolist() == [sa.ROW_BAD_INDEX] * 4
    assert torch.all(k[0, 2:] == 3) and torch.all(k[1, 2:] == 3) and torch.all(k[2, 1:] == 3) and torch.all(k[3, :2] == 3)


# ---- verify ------------------------------------------------------------------------------------------
def _case(seed, B, T, Hq, Hkv, lens, counts, *, page=16, dtype=torch.bfloat16, layout="head", G=1, tail=0, dense=False,
          paged=True, spread=1.0, q_scale=1.5):
    gen = _gen(seed)
    pps = max(1, -(-(max(lens) + tail) // page))
    codes, params = make_pool(gen, B * pps, page, Hkv, dtype, layout, spread)
    q = (q_scale * torch.randn(B, T, Hq, 128, generator=gen)).to(dtype)
    table = _table(gen, B, pps) if paged else None
    stride = max(1, max(lens))
    idx, lists = torch.zeros(B, G, stride, dtype=torch.int32), []
    if not dense:
        for b in range(B):
            for g in range(G):
                n = counts[b] if G == 1 else max(0, counts[b] - 3 * g)
                idx[b, g, :n] = torch.randperm(lens[b], generator=gen)[:n].sort().values
                lists.append(idx[b, g, :n].tolist())
    cnt = torch.tensor([len(x) for x in lists], dtype=torch.int32).view(B, G) if not dense else None
    per_head = [[list(range(lens[b])) if dense else lists[b * G + (h if G > 1 else 0)] for h in range(Hkv)] for b in range(B)]
    return dict(q=q, codes=codes, params=params, lens=lens, table=table, pps=pps, idx=None if dense else idx, counts=cnt, G=G, page=page,
                tail=tail, dense=dense, lists=per_head)


ENGINES = {"auto": 0, "mma.sync": 2, "tcgen05": 4}


def _engines(T, Hq, Hkv):
    """What may run that many query rows."""
    return ["auto", "mma.sync", "tcgen05"] if 32 < T * (Hq // Hkv) <= 40 else ["auto"]


def _more(engine, few, more):
    """Query heads for an engine: tcgen05 starts at 33 query rows per KV head."""
    return more if engine == "tcgen05" else few


def _run(c, engine="auto", **kw):
    kw.setdefault("flags", ENGINES[engine])
    up = lambda t: None if t is None else t.to(DEV)
    return _sa().kv4_verify(c["q"].to(DEV), _to_gpu(c["codes"]), _to_gpu(c["params"]), torch.tensor(c["lens"], dtype=torch.int32, device=DEV),
                            block_table=up(c["table"]), pages_per_seq=c["pps"], idx=up(c["idx"]), counts=up(c["counts"]),
                            n_groups=c["G"], dense=c["dense"], tail_len=c["tail"], **kw)


def _check(c, out, lse, **kw):
    want, want_lse, tol, tol_lse = verify64(c["q"], c["codes"], c["params"], c["lists"], c["lens"], c["tail"], c["page"], c["table"],
                                            c["pps"], **kw)
    out, lse = out.cpu().double(), lse.cpu().double()
    assert torch.all(torch.isfinite(out))
    assert torch.all((out - want).abs() <= tol), float(((out - want).abs() - tol).max())
    none = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), none) and torch.all(lse[none] < 0) and not out[none].any()
    assert torch.all((lse - want_lse)[~none].abs() <= tol_lse[~none])


LENGTHS = [([1], [1]), ([40], [0]), ([33], [31]), ([64], [32]), ([90], [33]), ([300, 2, 700], [255, 1, 257]), ([5000, 0, 17], [3111, 0, 17])]
HEADS = [(1, 8, 8), (1, 32, 8), (6, 32, 8), (5, 64, 8), (8, 8, 1), (1, 64, 1), (3, 12, 4)]   # rows: 1, 4, 24, 40, 64, 64, 9


@pytest.mark.parametrize("T,Hq,Hkv", HEADS)
@pytest.mark.parametrize("lens,counts", LENGTHS)
def test_attention_over_lists(lens, counts, T, Hq, Hkv):
    c = _case(11 + T, len(lens), T, Hq, Hkv, lens, counts, dtype=torch.float16 if T % 2 else torch.bfloat16)
    for engine in _engines(T, Hq, Hkv):
        out, lse, _ = _run(c, engine)
        assert out.dtype is c["q"].dtype
        _check(c, out, lse)


@pytest.mark.parametrize("T,Hq,Hkv,lens,tail,page,layout", [
    (1, 32, 8, [700, 1, 333], 0, 16, "head"),
    (1, 32, 8, [700, 0, 333], 1, 24, "slot"),
    (5, 32, 8, [257, 31], 5, 16, "head"),
    (4, 16, 4, [64, 0], 2, 32, "slot"),      # fewer in-flight rows than queries: the first queries see none of them
    (3, 16, 4, [31, 32], 7, 5, "head"),
    (8, 64, 8, [1000], 64, 64, "head"),
])
@pytest.mark.parametrize("paged", [True, False])
def test_attention_over_everything_with_a_tail(T, Hq, Hkv, lens, tail, page, layout, paged):
    c = _case(23, len(lens), T, Hq, Hkv, lens, None, dense=True, tail=tail, page=page, layout=layout, paged=paged)
    for engine in _engines(T, Hq, Hkv):
        out, lse, _ = _run(c, engine)
        _check(c, out, lse)


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 16, 4), (6, 32, 8), (5, 64, 8)])
def test_a_list_per_kv_head(T, Hq, Hkv):
    c = _case(31, 3, T, Hq, Hkv, [400, 60, 900], [300, 5, 611], G=Hkv, tail=T)
    for engine in _engines(T, Hq, Hkv):
        out, lse, _ = _run(c, engine)
        _check(c, out, lse)


@pytest.mark.parametrize("B,T,Hq,Hkv,count", [(64, 1, 32, 8, 40), (256, 6, 32, 8, 7), (40, 5, 64, 8, 33), (2048, 1, 1, 1, 3), (19, 1, 8, 8, 64)])
def test_many_units(B, T, Hq, Hkv, count):
    """More units than CTAs, units of less than a chunk, empty ones between them."""
    counts = [0 if b % 5 == 3 else 1 + (count * (b % 7)) // 6 for b in range(B)]
    c = _case(41, B, T, Hq, Hkv, [count + 9] * B, counts)
    if B * T * Hq > 4000:   # the reference of a few sequences says enough
        few = list(range(0, B, max(1, B // 12)))
    else:
        few = list(range(B))
    for engine in _engines(T, Hq, Hkv):
        _check_few(c, few, counts, *_run(c, engine)[:2])


def _check_few(c, few, counts, out, lse):
    pick = lambda t: t if t is None else t[few]
    sub = dict(c, q=c["q"][few], table=pick(c["table"]), lens=[c["lens"][b] for b in few], lists=[c["lists"][b] for b in few])
    _check(sub, out[few], lse[few])
    none = torch.tensor([n == 0 for n in counts])
    assert torch.all(torch.isinf(lse.cpu()[none])) and not out.cpu()[none].any() and torch.all(torch.isfinite(lse.cpu()[~none]))


@pytest.mark.parametrize("T,Hq,Hkv,lens,counts", [(6, 8, 2, [70000], [64007]), (5, 32, 4, [9000, 20000], [8999, 12345]), (17, 1, 1, [3000], [2900])])
def test_long_lists_split_over_the_gpu(T, Hq, Hkv, lens, counts):
    c = _case(43, len(lens), T, Hq, Hkv, lens, counts)
    for engine in _engines(T, Hq, Hkv):
        out, lse, _ = _run(c, engine)
        _check(c, out, lse)


@pytest.mark.parametrize("T,Hq,Hkv,G", [(1, 8, 8, 8), (5, 32, 8, 1), (5, 64, 8, 8), (8, 64, 8, 1)])
def test_many_units_of_very_different_lengths(T, Hq, Hkv, G):
    """More units than CTAs, from one position to thousands, some empty: a CTA's run may end in front of a unit's first chunk."""
    lens = [(1, 5000, 33, 700, 0, 64, 2500)[b % 7] + b % 5 for b in range(41)]
    counts = [0 if n < 2 else n - 1 - b % 2 for b, n in enumerate(lens)]
    c = _case(46, len(lens), T, Hq, Hkv, lens, counts, G=G, tail=T - 1, page=24)
    few = [0, 1, 3, 4, 5, 18, 40]
    pick = lambda t: t if t is None else t[few]
    sub = dict(c, q=c["q"][few], table=pick(c["table"]), lens=[lens[b] for b in few], lists=[c["lists"][b] for b in few])
    for engine in _engines(T, Hq, Hkv):
        status = torch.full((len(lens),), 7, dtype=torch.int32, device=DEV)
        out, lse, _ = _run(c, engine, status=status)
        assert not status.any()
        _check(sub, out[few], lse[few])


@pytest.mark.parametrize("T,Hq,Hkv", [(3, 16, 4), (5, 64, 8)])
def test_no_rows_and_lists_without_room(T, Hq, Hkv):
    """No tokens to write or read; lists of no room, so that the tail is all there is, or nothing is."""
    sa = _sa()
    c = _case(50, 2, T, Hq, Hkv, [40, 0], [0, 0], tail=T)
    codes, params, table = _to_gpu(c["codes"]), _to_gpu(c["params"]), c["table"].to(DEV)
    none = torch.empty(2, 0, Hkv, 128, dtype=torch.bfloat16, device=DEV)
    start, status = torch.zeros(2, dtype=torch.int32, device=DEV), torch.full((2,), 9, dtype=torch.int32, device=DEV)
    before = codes.clone()
    sa.kv4_append(none, none, codes, params, start, block_table=table, status=status)
    assert torch.equal(codes, before) and not status.any()
    k, v, _ = sa.kv4_read(codes, params, start, n_tokens=0, block_table=table, status=status)
    assert k.shape == v.shape == (2, 0, Hkv, 128)
    idx, counts = torch.empty(2, 1, 0, dtype=torch.int32, device=DEV), torch.zeros(2, 1, dtype=torch.int32, device=DEV)
    lens = torch.tensor(c["lens"], dtype=torch.int32, device=DEV)
    kw = dict(block_table=table, idx=idx, counts=counts, status=status)
    out, lse, _ = sa.kv4_verify(c["q"].to(DEV), codes, params, lens, tail_len=T, **kw)
    _check(c, out, lse)
    out, lse, _ = sa.kv4_verify(c["q"].to(DEV), codes, params, lens, **kw)
    assert not out.any() and torch.all(lse == float("-inf")) and not status.any()


def test_a_context_beyond_the_largest_table():
    """2^23 positions, the most that a table may hold: one more is reported."""
    sa = _sa()
    codes, params = sa.kv4_cache(1, 64, 1)
    x = torch.randn(1, 64, 1, 128, generator=_gen(48)).to(torch.bfloat16).to(DEV)
    table = torch.zeros(1, 1 << 17, dtype=torch.int32, device=DEV)
    sa.kv4_append(x, x, codes, params, torch.zeros(1, dtype=torch.int32, device=DEV), block_table=table)
    q = torch.randn(1, 1, 2, 128, generator=_gen(49)).to(torch.bfloat16).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = []
    for n in (64, 1 << 23, (1 << 23) + 1, 2 ** 31 - 1):
        out, lse, _ = sa.kv4_verify(q, codes, params, torch.tensor([n], dtype=torch.int32, device=DEV), block_table=table, dense=True, status=status)
        got.append((out.float(), lse, status.item()))
    assert [s for _, _, s in got] == [0, 0, sa.ROW_BAD_INDEX, sa.ROW_BAD_INDEX]
    # the same 64 rows 2^17 times over: the output stays (two roundings of half a step of bf16), the sum of weights grows with their
    # number (a thread adds a few hundred to a few thousand of them, 2^-24 each time: 2^-12 at worst, and the joins)
    assert float((got[1][0] - got[0][0]).abs().max()) <= 2.0 ** -7 * float(got[0][0].abs().max())
    assert float((got[1][1] - got[0][1] - 17 * math.log(2)).abs().max()) <= 1e-3


def test_memory_that_the_current_stream_still_uses_is_waited_for():
    """What a call on another stream allocates may be memory that work on the current stream has yet to write."""
    sa = _sa()
    c = _case(98, 2, 6, 32, 8, [300, 200], [250, 100])
    up = lambda t: t.to(DEV)
    q, codes, params, table, idx, counts = up(c["q"]), _to_gpu(c["codes"]), _to_gpu(c["params"]), up(c["table"]), up(c["idx"]), up(c["counts"])
    lens = torch.tensor(c["lens"], dtype=torch.int32, device=DEV)
    kw = dict(block_table=table, idx=idx, counts=counts)
    ref = sa.kv4_verify(q, codes, params, lens, **kw)
    start = torch.zeros(2, dtype=torch.int32, device=DEV)
    ref_k, ref_v, _ = sa.kv4_read(codes, params, start, n_tokens=200, block_table=table)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        late = [torch.empty_like(t) for t in (ref[0], ref[1], ref_k, ref_v)]
        torch.cuda._sleep(20_000_000)
        for t in late:
            t.fill_(float("nan"))
        del late, t
        out, lse, _ = sa.kv4_verify(q, codes, params, lens, stream=stream, **kw)
        k, v, _ = sa.kv4_read(codes, params, start, n_tokens=200, block_table=table, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1]) and torch.equal(k, ref_k) and torch.equal(v, ref_v)


def test_calls_long_enough_for_tcgen05_take_it_by_themselves():
    c = _case(44, 2, 6, 12, 2, [150000, 100000], None, dense=True)
    out, lse, _ = _run(c)
    tc, mma = _run(c, "tcgen05"), _run(c, "mma.sync")
    assert torch.equal(out, tc[0]) and torch.equal(lse, tc[1]) and not torch.equal(lse, mma[1])
    few = dict(c, q=c["q"][:, :2].contiguous())
    _check(few, out[:, :2], lse[:, :2])


def test_a_bounded_wait_that_runs_out_is_reported():
    """The first completion of CTA 0 is withheld: its waits run out, the kernel returns, the status says so, and the next call is
    right."""
    sa = _sa()
    c = _case(45, 2, 6, 48, 8, [3000, 2000], None, dense=True)
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    _run(c, status=status, flags=sa.VERIFY_ENGINE_TCGEN05 | sa.VERIFY_TEST_LOSE_ARRIVAL)
    assert status[0].item() == sa.ROW_TIMEOUT
    out, lse, _ = _run(c, "tcgen05", status=status)
    assert status.tolist() == [0, 0]
    _check(c, out, lse)


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_scores_that_grow_and_scales_that_grow(engine):
    """The running maximum and the weights' scale both move along the list: K rows that a query likes more and more,
    V rows whose range spans 2^30."""
    gen, n = _gen(47), 2000
    c = _case(47, 1, 5, _more(engine, 8, 16), 2, [n], None, dense=True)
    x = torch.randn(c["codes"].shape[0], 2, 16, 2, 128, generator=gen)
    for b in range(c["table"].shape[1]):
        page = int(c["table"][0, b])
        pos = torch.arange(16) + 16 * b
        x[page, 0] += (pos / 400.0)[:, None, None] * c["q"][0, 0, 0].float().sign()
        x[page, 1] *= (2.0 ** (30.0 * pos / n - 20))[:, None, None]
    c["codes"], c["params"] = quantise(x.to(torch.bfloat16))
    out, lse, _ = _run(c, engine=engine)
    _check(c, out, lse)
    # and the other way round
    for a in ("codes", "params"):
        c[a] = c[a].flip(0).contiguous()
    c["table"] = c["table"].flip(1).contiguous()
    out, lse, _ = _run(c, engine=engine)
    _check(c, out, lse)


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_constant_rows_and_rows_far_from_zero(engine):
    c = _case(53, 2, 6, _more(engine, 32, 48), 8, [500, 33], None, dense=True)
    gen = _gen(53)
    x = torch.randn(c["codes"].shape[0], 2, 16, 8, 128, generator=gen)
    x[::3] = x[::3, :, :, :, :1]               # constant rows: scale 0
    x[1::3, 1] = x[1::3, 1] * 2 ** -6 + 40     # far from zero, little range
    c["codes"], c["params"] = quantise(x.to(torch.bfloat16))
    out, lse, _ = _run(c, engine=engine)
    _check(c, out, lse)


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -9, 2.0 ** 40])
@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_queries_of_any_magnitude(scale, engine):
    """A power of two in the queries and its inverse in sm_scale: bf16's range, beyond fp16's."""
    c = _case(59, 2, 6, _more(engine, 32, 48), 8, [200, 100], [150, 100])
    out, lse, _ = _run(c, engine=engine)
    big = dict(c, q=c["q"] * scale)
    out2, lse2, _ = _run(big, engine, sm_scale=1 / (math.sqrt(128) * scale))
    assert torch.equal(out2, out) or float((out2.float() - out.float()).abs().max()) <= 2.0 ** -7
    _check(c, out2, lse2)


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_float32_output_and_given_buffers(engine):
    sa = _sa()
    c = _case(61, 2, 6, _more(engine, 32, 48), 8, [300, 900], [280, 700])
    out16, lse16, _ = _run(c, engine=engine)
    out = torch.full(c["q"].shape, float("nan"), device=DEV)
    lse = torch.full(c["q"].shape[:3], float("nan"), device=DEV)
    status = torch.full((2,), 5, dtype=torch.int32, device=DEV)
    ws = torch.full((sa.kv4_verify_workspace_bytes(c["q"].to(DEV), _to_gpu(c["codes"])),), 255, dtype=torch.uint8, device=DEV)
    for _ in range(2):   # the workspace needs no preparation and holds no state
        _run(c, out=out, lse=lse, status=status, workspace=ws, engine=engine)
        assert status.tolist() == [0, 0]
        assert torch.equal(out.to(torch.bfloat16), out16) and torch.equal(lse, lse16)
    _check(c, out, lse)


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_nothing_outside_the_lists_is_looked_at(engine):
    """Every row that no list names, masked tail rows and ends of pages hold NaN."""
    c = _case(67, 2, 5, _more(engine, 16, 32), 4, [333, 90], [200, 60], tail=5)
    params = torch.full_like(c["params"], float("nan"))
    for b in range(2):
        for pos in c["lists"][b][0] + [c["lens"][b] + j for j in range(5)]:
            at = int(c["table"][b, pos // 16]), pos % 16
            params[at[0], :, at[1]] = c["params"][at[0], :, at[1]]
    clean = dict(c)
    c["params"] = params
    out, lse, _ = _run(c, engine=engine)
    _check(clean, out, lse)
    # the last in-flight row is NaN: only the last query sees it
    for b in range(2):
        pos = c["lens"][b] + 4
        c["params"][int(c["table"][b, pos // 16]), :, pos % 16] = float("nan")
    out, lse, _ = _run(c, engine=engine)
    assert torch.all(torch.isfinite(out[:, :4])) and torch.all(torch.isnan(out[:, 4])) and torch.all(torch.isnan(lse[:, 4]))
    want, want_lse, tol, tol_lse = verify64(clean["q"], clean["codes"], clean["params"], clean["lists"], clean["lens"], 5, 16, clean["table"], clean["pps"])
    assert torch.all((out.cpu().double() - want)[:, :4].abs() <= tol[:, :4])


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_a_query_of_nan_or_infinity_spoils_no_other(engine):
    c = _case(71, 1, 6, _more(engine, 32, 48), 8, [200], [150])
    out, lse, _ = _run(c, engine=engine)
    for bad in (float("nan"), float("inf")):
        q = c["q"].clone()
        q[0, 2, 5, 17] = bad
        out2, lse2, _ = _run(dict(c, q=q), engine=engine)
        keep = torch.ones(6, c["q"].shape[2], dtype=torch.bool)
        keep[2, 5] = False
        assert torch.equal(out2[0][keep.to(DEV)], out[0][keep.to(DEV)]) and torch.equal(lse2[0][keep.to(DEV)], lse[0][keep.to(DEV)])
        assert torch.all(torch.isnan(out2[0, 2, 5]))


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_bad_positions_and_pages_are_reported_and_read_from_the_first(engine):
    sa = _sa()
    c = _case(73, 4, 5, _more(engine, 8, 16), 2, [100, 100, 100, 100], [50, 50, 50, 50])
    c["idx"][1, 0, 7] = 100        # beyond the context
    c["idx"][2, 0, 0] = -5
    c["table"][3, 2] = 10 ** 6     # no such page
    status = torch.zeros(4, dtype=torch.int32, device=DEV)
    out, lse, _ = _run(c, status=status, engine=engine)
    hit = any(32 <= p < 48 for p in c["lists"][3][0])
    assert hit and status.tolist() == [0] + [sa.ROW_BAD_INDEX] * 3
    assert torch.all(torch.isfinite(out))
    first = dict(c, q=c["q"][:1], table=c["table"][:1], lens=[100], lists=c["lists"][:1])
    _check(first, out[:1], lse[:1])
    # a context longer than the block table, dense
    c = _case(74, 1, 5, _more(engine, 8, 16), 2, [100], None, dense=True)
    c["lens"] = [5000]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, _, _ = _run(c, status=status, engine=engine)
    assert status.item() == sa.ROW_BAD_INDEX and torch.all(torch.isfinite(out))


def test_repeated_positions_count_each_time():
    c = _case(79, 1, 2, 8, 2, [60], [50])
    c["idx"][0, 0, :50] = torch.arange(50) // 3
    c["lists"] = [[(torch.arange(50) // 3).tolist()] * 2]
    out, lse, _ = _run(c)
    _check(c, out, lse)


def test_rows_beyond_four_gigabytes():
    """The last pages of a pool of more than 2^32 bytes of codes, reached by block table."""
    sa, gen = _sa(), _gen(83)
    n_pages, page, h = 280000, 16, 8                       # 4.6 GB of codes
    codes, params = sa.kv4_cache(n_pages, page, h)
    x = torch.randn(2, 50, h, 128, generator=gen).to(torch.bfloat16)
    table = torch.tensor([[n_pages - 1, n_pages - 5, 3, n_pages - 2], [n_pages - 7, 0, n_pages - 3, n_pages - 9]], dtype=torch.int32)
    start = torch.zeros(2, dtype=torch.int32, device=DEV)
    sa.kv4_append(x.to(DEV), x.to(DEV), codes, params, start, block_table=table.to(DEV))
    k, v, _ = sa.kv4_read(codes, params, start, n_tokens=50, block_table=table.to(DEV))
    want = values(*quantise(x)).float().to(torch.bfloat16)
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), want)
    q = torch.randn(2, 1, 32, 128, generator=gen).to(torch.bfloat16)
    lens = torch.tensor([50, 50], dtype=torch.int32, device=DEV)
    out, lse, _ = sa.kv4_verify(q.to(DEV), codes, params, lens, block_table=table.to(DEV), dense=True)
    small_c, small_p = codes[table.flatten().long()].cpu(), params[table.flatten().long()].cpu()
    _check(dict(q=q, codes=small_c, params=small_p, lists=[[list(range(50))] * h] * 2, lens=[50, 50], tail=0, page=page,
                table=torch.arange(8).view(2, 4), pps=4), out, lse)


@pytest.mark.parametrize("engine", ["mma.sync", "tcgen05"])
def test_the_same_bits_again_on_a_stream_and_in_a_graph(engine):
    sa = _sa()
    c = _case(89, 3, 6, _more(engine, 32, 48), 8, [3000, 40, 700], [2500, 40, 333], tail=6)
    ref = _run(c, engine=engine)
    up = lambda t: t.to(DEV)
    q, codes, params, table, idx, counts = up(c["q"]), _to_gpu(c["codes"]), _to_gpu(c["params"]), up(c["table"]), up(c["idx"]), up(c["counts"])
    lens = torch.tensor(c["lens"], dtype=torch.int32, device=DEV)
    kw = dict(block_table=table, idx=idx, counts=counts, tail_len=6, flags=ENGINES[engine])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(20):   # two calls at once, workspaces of their own
        for s in streams:
            got.append(sa.kv4_verify(q, codes, params, lens, stream=s, **kw))
    torch.cuda.synchronize()
    for out, lse, _ in got:
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
    out, lse, status = torch.empty_like(ref[0]), torch.empty_like(ref[1]), torch.zeros(3, dtype=torch.int32, device=DEV)
    ws = torch.empty(sa.kv4_verify_workspace_bytes(q, codes), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            sa.kv4_verify(q, codes, params, lens, out=out, lse=lse, status=status, workspace=ws, **kw)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
    # other lists, lengths and queries in the same buffers
    counts.copy_(torch.tensor([[100], [0], [1]], dtype=torch.int32))
    lens.copy_(torch.tensor([2900, 30, 800], dtype=torch.int32) - 0)
    idx.copy_(torch.sort(idx % 20, -1).values)
    graph.replay()
    fresh = sa.kv4_verify(q, codes, params, lens, **kw)
    assert torch.equal(out, fresh[0]) and torch.equal(lse, fresh[1])


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    r = torch.Generator().manual_seed(1000 + seed)
    pick = lambda *x: x[int(torch.randint(len(x), (1,), generator=r))]
    Hq, Hkv = pick((32, 8), (8, 8), (64, 8), (16, 2), (12, 4), (5, 1))
    T = int(torch.randint(1, 64 // (Hq // Hkv) + 1, (1,), generator=r)) if Hq // Hkv < 64 else 1
    T = min(T, 9)
    B, dense = pick(1, 2, 5), bool(torch.randint(2, (1,), generator=r))
    lens = [int(x) for x in torch.randint(0, 1500, (B,), generator=r)]
    counts = [int(x * float(torch.rand(1, generator=r))) for x in lens]
    c = _case(seed, B, T, Hq, Hkv, lens, counts, page=pick(16, 32, 64, 7, 1), dtype=pick(torch.bfloat16, torch.float16),
              layout=pick("head", "slot"), G=pick(1, Hkv) if not dense else 1, tail=pick(0, T, T + 2, 1), dense=dense, paged=pick(True, False))
    for engine in _engines(T, Hq, Hkv):
        out, lse, _ = _run(c, engine)
        _check(c, out, lse)
