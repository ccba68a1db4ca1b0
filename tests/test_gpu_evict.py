"""Accumulated attention weight, eviction and the moves that follow, on the GPU, against plain references."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _sa():
    import paper_2510_27641_b200 as sa
    return sa


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- accumulate ------------------------------------------------------------------------------------
def _accumulate64(probs, lens, old, groups, head_group, decay, out):
    """The definition, one layer, sequence and group after the other, in numpy binary64, rounded once."""
    want = out.copy()
    for u, p in enumerate(probs):
        if p is None:
            continue
        for b, n in enumerate(lens):
            n = max(0, min(n, p.shape[3], out.shape[3]))
            for g in range(groups):
                heads = [h for h in range(p.shape[1]) if head_group is None or head_group[h] == g]
                got = p[b, heads, :, :n].astype(np.float64).sum((0, 1)) if heads else np.zeros(n)
                before = np.zeros(n) if old is None else old[u, b, g, :n].astype(np.float64)
                want[u, b, g, :n] = (decay * before + got).astype(np.float32)
    return want


def _close(got, want):
    """Sums in binary64 differ by their order (at most 2^-40 relative here), so the rounded ones by a step at most."""
    got = got.cpu().numpy()
    assert np.all(np.abs(got.astype(np.float64) - want) <= 2.0 ** -23 * np.abs(want) + 1e-45)


@pytest.mark.parametrize("layers,B,H,gamma,lens,width,score_width,groups,decay", [
    (1, 1, 1, 1, [1], 4, 1, 1, 1.0),
    (1, 1, 12, 4, [4096], 4096, 4096, 1, 1.0),
    (2, 3, 12, 5, [1000, 0, 37], 1000, 1000, 1, 0.9),
    (1, 2, 16, 3, [515, 9], 516, 515, 8, 0.0),       # rows of scores that no 16 bytes divide
    (3, 2, 12, 7, [2000, 1999], 2000, 2048, 4, 1.0),
    (1, 9, 16, 4, [9000] * 9, 9000, 9000, 1, 0.5),
    (1, 2, 3, 200, [77, 300], 300, 100, 2, 1.0),     # scores of fewer positions than the maps
    (1, 40, 4, 2, [8192] * 40, 8192, 8192, 1, 1.0),
])
@pytest.mark.parametrize("grouped", [False, True])
def test_accumulated_weight(layers, B, H, gamma, lens, width, score_width, groups, decay, grouped):
    sa, rng = _sa(), np.random.default_rng(5)
    probs = [rng.random((B, H, gamma, width), dtype=np.float32) ** 6 if u != 1 else None for u in range(layers)]
    head_group = [int(h * groups // H) if h != 2 else groups - 1 for h in range(H)] if grouped else None
    old = rng.random((layers, B, groups, score_width), dtype=np.float32)
    maps = [None if p is None else torch.from_numpy(p).to(DEV) for p in probs]
    kw = dict(n_groups=groups, head_group=head_group, decay=decay)
    status = torch.full((layers, B, groups), 3, dtype=torch.int32, device=DEV)
    out = torch.full(old.shape, 7.0, device=DEV)
    got, st = sa.accumulate_attention(maps, _ints(lens), torch.from_numpy(old).to(DEV), out=out, row_status=status, **kw)
    assert got is out and st is status and not status.any()
    _close(out, _accumulate64(probs, lens, old, groups, head_group, decay, np.full(old.shape, 7.0, np.float32)))
    # in place, and from nothing
    scores = torch.from_numpy(old).to(DEV)
    sa.accumulate_attention(maps, _ints(lens), scores, **kw)
    _close(scores, _accumulate64(probs, lens, old, groups, head_group, decay, old))
    out.fill_(7.0)
    sa.accumulate_attention(maps, _ints(lens), out=out, **kw)
    _close(out, _accumulate64(probs, lens, None, groups, head_group, decay, np.full(old.shape, 7.0, np.float32)))


def test_invalid_probabilities_leave_the_weight_alone():
    sa = _sa()
    probs = torch.full((2, 4, 3, 64), 0.25, device=DEV)
    probs[0, 1, 2, 5], probs[0, 3, 0, 9], probs[0, 0, 0, 10] = float("nan"), float("inf"), -1e-3
    probs[1, 2, 1, 40] = float("nan")       # behind the context: not looked at
    scores = torch.ones(1, 2, 2, 64, device=DEV)
    status = torch.zeros(1, 2, 2, dtype=torch.int32, device=DEV)
    sa.accumulate_attention([probs], _ints([64, 40]), scores, n_groups=2, head_group=[0, 0, 1, 1], decay=0.5, row_status=status)
    assert status.tolist() == [[[sa.ROW_INVALID_PROB] * 2, [0, 0]]]
    want = torch.full((1, 2, 2, 64), 2.0)   # 0.5 + 6 * 0.25
    want[0, 0, 0, [5, 10]] = 1
    want[0, 0, 1, 9] = 1
    want[0, 1, :, 40:] = 1
    assert torch.equal(scores.cpu(), want)


# ---- evict -------------------------------------------------------------------------------------------
def _evict_plain(w, n, budget, n_sink, n_recent, pos, seq):
    """One list: (src, dst, what stays where, as source slots of the first m)."""
    w = np.where(np.isnan(w[:n]), -np.inf, w[:n].astype(np.float64)) + 0.0
    pos = np.arange(n) if pos is None else pos[:n]
    safe = (pos < n_sink) | (pos >= (n if seq is None else seq) - n_recent)
    m = min(n, budget)
    order = np.lexsort((np.arange(n), -w, ~safe))
    stays = np.zeros(n, bool)
    stays[order[:m]] = True
    src, dst = np.flatnonzero(stays[m:]) + m, np.flatnonzero(~stays[:m])
    after = np.arange(m)
    after[dst] = src
    return src, dst, after


def _weights(rng, kind, shape):
    if kind == "spread":
        return np.exp(2.5 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        return rng.integers(0, 5, shape).astype(np.float32)
    if kind == "equal":
        return np.zeros(shape, np.float32)
    if kind == "close":      # differ in the lowest bits alone
        return (1 + rng.integers(0, 1 << 10, shape) * 2.0 ** -23).astype(np.float32)
    x = rng.standard_normal(shape).astype(np.float32)     # "odd": of both signs, with NaN, infinities, zeros of both signs
    flat = x.reshape(-1)
    pick = rng.integers(0, 12, flat.shape)
    for v, bad in enumerate((np.nan, np.inf, -np.inf, 0.0, -0.0, -np.nan, 1e-42)):
        flat[pick == v] = bad
    return x


EVICT_CASES = [
    # layers, B, G, L, lens, budget, sink, recent
    (1, 1, 1, 1, [1], 1, 0, 0),
    (1, 3, 1, 40, [40, 33, 0], 32, 4, 8),
    (1, 2, 1, 2047, [2047, 1900], 1, 0, 1),
    (2, 2, 1, 4096, [4096, 4095], 3968, 4, 128),
    (1, 4, 3, 5001, [5001, 2500, 2600, -3], 2500, 0, 0),
    (1, 2, 8, 20000, [20000, 12345], 777, 4, 512),
    (1, 1, 1, 131072, [131072], 65536, 4, 4096),
    (1, 2, 1, 196608, [196608, 300000], 100001, 0, 64),      # a length beyond the row is clamped
    (3, 40, 3, 2100, [2100 - 7 * b for b in range(40)], 1900, 2, 30),   # more lists than CTAs at once
    (1, 310, 1, 3000, [3000] * 310, 1500, 0, 0),
    (1, 8, 1, 32768, [32768 - 5000 * b for b in range(6)] + [3, 0], 16384, 4, 64),      # eight CTAs to a list
    (1, 75, 2, 17001, [17001 - 200 * b for b in range(75)], 9000, 4, 64),               # two, of more CTAs than SMs
    (1, 20, 1, 16385, [16385, 8193] * 10, 8192, 0, 100),                                # slices of 8192 and more, 1024 threads
]


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "close", "odd"])
@pytest.mark.parametrize("layers,B,G,L,lens,budget,sink,recent", EVICT_CASES)
@pytest.mark.parametrize("moved", [False, True])
def test_what_stays_and_what_moves(layers, B, G, L, lens, budget, sink, recent, kind, moved):
    sa, rng = _sa(), np.random.default_rng(17)
    w = _weights(rng, kind, (layers, B, G, L))
    pos = seq = None
    if moved:      # tokens out of order, half of them gone
        pos = np.stack([rng.permutation(2 * L)[:L] for _ in range(layers * B * G)]).reshape(layers, B, G, L).astype(np.int32)
        seq = np.full(B, 2 * L, np.int32)
    room = max(1, min(budget, L - budget)) + 3
    src, dst = (torch.full((layers, B, G, room), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    gw = torch.from_numpy(w).to(DEV)
    gp = None if pos is None else torch.from_numpy(pos).to(DEV)
    w_out = torch.full(w.shape, -7.0, device=DEV)
    p_out = None if pos is None else torch.full(w.shape, -7, dtype=torch.int32, device=DEV)
    kw = dict(n_sink=sink, n_recent=recent, positions=gp, seq_len=None if seq is None else torch.from_numpy(seq).to(DEV))
    got = sa.evict(gw, _ints(lens), budget, src=src, dst=dst, scores_out=w_out, positions_out=p_out, **kw)
    n_moves, new_len = got[2].cpu().numpy(), got[3].cpu().numpy()
    # in place, lists made by the call
    w_in, p_in = gw.clone(), None if gp is None else gp.clone()
    again = sa.evict(w_in, _ints(lens), budget, scores_out=w_in, positions_out=p_in, **dict(kw, positions=p_in))
    assert torch.equal(again[2], got[2]) and torch.equal(again[3], got[3])
    src, dst, w_out, w_in = (t.cpu().numpy() for t in (src, dst, w_out, w_in))
    a_src, a_dst = again[0].cpu().numpy(), again[1].cpu().numpy()
    for u in range(layers):
        for b in range(B):
            n = max(0, min(lens[b], L))
            m = min(n, budget)
            assert new_len[b] == m
            for g in range(G):
                s, d, after = _evict_plain(w[u, b, g], n, budget, sink, recent, None if pos is None else pos[u, b, g], None if seq is None else seq[b])
                at = u, b, g
                assert n_moves[at] == len(s)
                assert np.array_equal(src[at][:len(s)], s) and np.array_equal(dst[at][:len(s)], d)
                assert np.array_equal(a_src[at][:len(s)], s) and np.array_equal(a_dst[at][:len(s)], d)
                assert np.all(src[at][len(s):] == -1) and np.all(dst[at][len(s):] == -1)
                want = w[at].copy()
                want[:m], want[m:n] = w[at][after], 0
                assert np.array_equal(w_in[at], want, equal_nan=True)
                assert np.array_equal(w_out[at][:n], want[:n], equal_nan=True) and np.all(w_out[at][n:] == -7)
                if pos is not None:
                    assert np.array_equal(p_in[at].cpu().numpy()[:m], pos[at][after]) and np.array_equal(p_in[at].cpu().numpy()[m:], pos[at][m:])
                    assert np.array_equal(p_out[at].cpu().numpy()[:m], pos[at][after]) and np.all(p_out[at].cpu().numpy()[m:] == -7)


def test_more_protected_slots_than_the_budget():
    """Positions that name a token twice may protect more slots than there is room for: the lowest stay."""
    sa = _sa()
    pos = torch.zeros(1, 1, 1, 100, dtype=torch.int32, device=DEV)
    src, dst, n, new_len = sa.evict(torch.ones(1, 1, 1, 100, device=DEV), _ints([100]), 30, n_sink=4, positions=pos, seq_len=_ints([100]))
    assert n.item() == 0 and new_len.item() == 30


def test_eviction_in_a_graph_and_on_streams():
    sa, rng = _sa(), np.random.default_rng(3)
    w = torch.from_numpy(_weights(rng, "ties", (1, 4, 2, 9000))).to(DEV)
    lens = _ints([9000, 8000, 4000, 1])
    ref = sa.evict(w, lens, 4500, n_sink=4, n_recent=100)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [sa.evict(w, lens, 4500, n_sink=4, n_recent=100, stream=s) for s in streams for _ in range(5)]
    torch.cuda.synchronize()
    src, dst = torch.empty_like(ref[0]), torch.empty_like(ref[1])
    n, new_len = torch.empty_like(ref[2]), torch.empty_like(ref[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.evict(w, lens, 4500, n_sink=4, n_recent=100, src=src, dst=dst, n_moves=n, new_len=new_len)
    graph.replay()
    for r in got + [(src, dst, n, new_len)]:
        assert torch.equal(r[2], ref[2]) and torch.equal(r[3], ref[3])
        for b in range(4):
            for g in range(2):
                k = int(ref[2][0, b, g])
                assert torch.equal(r[0][0, b, g, :k], ref[0][0, b, g, :k]) and torch.equal(r[1][0, b, g, :k], ref[1][0, b, g, :k])


# ---- move_rows -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_pools,B,G,heads,page,width,dtype,layout,paged", [
    (1, 1, 1, 1, 16, 128, torch.bfloat16, "slot", True),
    (3, 3, 1, 8, 16, 128, torch.bfloat16, "slot", True),
    (2, 2, 8, 8, 24, 64, torch.uint8, "head", True),
    (35, 2, 4, 4, 32, 64, torch.uint8, "slot", False),       # more pools than one launch takes
    (1, 2, 3, 3, 7, 40, torch.float16, "head", False),
])
def test_rows_are_moved(n_pools, B, G, heads, page, width, dtype, layout, paged):
    sa, gen = _sa(), torch.Generator().manual_seed(9)
    L = 1300
    pps = -(-L // page)
    table = torch.randperm(B * pps, generator=gen).to(torch.int32).view(B, pps)
    shape = (B * pps, 2, heads, page) if layout == "head" else (B * pps, 2, page, heads)
    turn = (lambda t: t.transpose(2, 3)) if layout == "head" else (lambda t: t)
    pools = [turn(torch.randint(0, 200, (*shape, width), generator=gen).to(dtype).to(DEV)) for _ in range(n_pools)]
    params = [turn(torch.randn(*shape, 2, generator=gen).to(torch.bfloat16).to(DEV)) for _ in range(n_pools)] if dtype is torch.uint8 else None
    moves = torch.randint(0, 600, (B, G), generator=gen).to(torch.int32)
    moves[0, 0] = 0 if B > 1 else 600
    src = torch.stack([torch.randperm(650, generator=gen)[:600].sort().values + 650 for _ in range(B * G)]).view(B, G, 600).to(torch.int32)
    dst = torch.stack([torch.randperm(650, generator=gen)[:600].sort().values for _ in range(B * G)]).view(B, G, 600).to(torch.int32)
    want = [p.cpu().clone() for p in pools + (params or [])]
    at = lambda b, x: ((table[b, x // page].long() if paged else b * pps + x.long() // page), x.long() % page)
    for b in range(B):
        for g in range(G):
            k = int(moves[b, g])
            (sp, ss), (dp, ds) = at(b, src[b, g, :k]), at(b, dst[b, g, :k])
            for t in want:
                if G == 1:
                    t[dp, :, ds] = t[sp, :, ss]
                else:
                    t[dp, :, ds, g] = t[sp, :, ss, g]
    status = torch.full((B,), 9, dtype=torch.int32, device=DEV)
    sa.move_rows(pools, src.to(DEV), dst.to(DEV), moves.to(DEV), params=params, block_table=table.to(DEV) if paged else None, pages_per_seq=pps,
                 status=status)
    assert not status.any()
    for got, t in zip(pools + (params or []), want):
        assert torch.equal(got.cpu(), t)


def test_moves_that_no_page_holds_are_skipped_and_reported():
    sa = _sa()
    pool = torch.arange(4 * 2 * 16, device=DEV).view(4, 2, 16, 1, 1).expand(4, 2, 16, 1, 8).to(torch.float32).contiguous()
    before = pool.clone()
    table = _ints([[0, 1], [2, 77]])
    src, dst = _ints([[[31, 32, 5]], [[3, 20, -1]]]), _ints([[[0, 1, 40]], [[2, 4, 6]]])
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    sa.move_rows([pool], src, dst, _ints([[3], [9]]), block_table=table, status=status)
    assert status.tolist() == [sa.ROW_BAD_INDEX] * 2
    before[0, :, 0] = before[1, :, 15].clone()
    before[2, :, 2] = before[2, :, 3].clone()
    assert torch.equal(pool, before)


def test_rows_beyond_four_gigabytes():
    sa = _sa()
    n_pages = 70000                                   # 9.2 GB of bf16 rows
    pool = torch.zeros(n_pages, 2, 16, 16, 128, dtype=torch.bfloat16, device=DEV)
    table = _ints([[n_pages - 1, n_pages - 2, 7]])
    pool[n_pages - 2, :, 4] = 3
    sa.move_rows([pool], _ints([[[20]]]), _ints([[[2]]]), _ints([[1]]), block_table=table)
    assert torch.all(pool[n_pages - 1, :, 2] == 3) and pool[n_pages - 1].float().sum().item() == 3 * 2 * 16 * 128


# ---- together --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("G", [1, 4])
def test_a_cache_that_is_written_read_thinned_and_written_again(G):
    """Prompt, a step's attention, weights, eviction, the moves, the next tokens: after every step the attention over
    what is left is that over the same rows in a cache that never had the others."""
    sa, gen = _sa(), torch.Generator().manual_seed(21)
    B, H, Hq, page, L, budget = 2, 4, 16, 16, 320, 160
    pps = L // page
    codes, params = sa.kv4_cache(B * pps, page, H)
    table = torch.randperm(B * pps, generator=gen).to(torch.int32).view(B, pps).to(DEV)
    lens = _ints([200, 173])
    tokens = torch.randn(B, 400, 2, H, 128, generator=gen).to(torch.bfloat16).to(DEV)      # K and V of every token to come
    sa.kv4_append(tokens[:, :200, 0], tokens[:, :200, 1], codes, params, _ints([0, 0]), n_new=lens, block_table=table)
    held = [[list(range(int(n))) for _ in range(H)] for n in lens]                          # token of every slot, per head
    positions = torch.arange(L, dtype=torch.int32, device=DEV).expand(1, B, G, L).contiguous()
    seen = lens.clone()
    scores = torch.zeros(1, B, G, L, device=DEV)
    for step in range(4):
        probs = torch.zeros(B, 8, 3, L, device=DEV)
        for b in range(B):
            n = int(lens[b])
            probs[b, :, :, :n] = torch.softmax(3 * torch.randn(8, 3, n, generator=gen), -1).to(DEV)
        sa.accumulate_attention([probs], lens, scores, n_groups=G, head_group=[h * G // 8 for h in range(8)], decay=0.9)
        src, dst, n, new_len = sa.evict(scores, lens, budget, n_sink=2, n_recent=20, positions=positions, seq_len=seen,
                                        scores_out=scores, positions_out=positions)
        sa.move_rows([codes], src[0], dst[0], n[0], params=[params], block_table=table)
        for b in range(B):
            for h in range(H):
                g = h if G > 1 else 0
                k = int(n[0, b, g])
                for s, d in zip(src[0, b, g, :k].tolist(), dst[0, b, g, :k].tolist()):
                    held[b][h][d] = held[b][h][s]
                del held[b][h][int(new_len[b]):]
                assert positions[0, b, g, :int(new_len[b])].tolist() == held[b][h]
                assert {0, 1} <= set(held[b][h]) and set(range(int(seen[b]) - 20, int(seen[b]))) <= set(held[b][h])
        lens = new_len
        new = 7 + step                                                                       # the next tokens
        at = seen.tolist()
        k = torch.stack([tokens[b, at[b]:at[b] + new, 0] for b in range(B)])
        v = torch.stack([tokens[b, at[b]:at[b] + new, 1] for b in range(B)])
        sa.kv4_append(k, v, codes, params, lens, block_table=table)
        for b in range(B):
            positions[0, b, :, int(lens[b]):int(lens[b]) + new] = torch.arange(at[b], at[b] + new, device=DEV)
            for h in range(H):
                held[b][h] += list(range(at[b], at[b] + new))
        q = torch.randn(B, new, Hq, 128, generator=gen).to(torch.bfloat16).to(DEV)
        f32 = lambda t: torch.empty(t.shape, device=DEV)
        out, lse, _ = sa.kv4_verify(q, codes, params, lens, block_table=table, dense=True, tail_len=new, out=f32(q))
        # the same rows in token order per head, one head to a cache of its own
        for h in range(H):
            c2, p2 = sa.kv4_cache(B * pps, page, 1)
            k2, v2 = (torch.stack([tokens[b, held[b][h], side, h:h + 1] if len(held[b][h]) == len(held[0][h]) else
                                   torch.cat([tokens[b, held[b][h], side, h:h + 1],
                                              tokens[b, :max(0, len(held[0][h]) - len(held[b][h])), side, h:h + 1]])
                                   for b in range(B)]) for side in (0, 1))
            sa.kv4_append(k2, v2, c2, p2, _ints([0, 0]), n_new=lens + new, block_table=table)
            mine = slice(h * 4, h * 4 + 4)
            own_q = q[:, :, mine].contiguous()
            out2, lse2, _ = sa.kv4_verify(own_q, c2, p2, lens, block_table=table, dense=True, tail_len=new, out=f32(own_q))
            # values lie within 5 of zero, so scales below 10 / 15: two outputs, each with weights of 11 bits on codes at
            # most 8 from the middle; two logarithms, each of scores with up to 128 |q| (15 s + |z|) / sqrt(128) 2^-20
            assert float((out2 - out[:, :, mine]).abs().max()) <= 2 * 8 * (10 / 15) * 2.0 ** -11
            assert float((lse2 - lse[:, :, mine]).abs().max()) <= 2 * 128 * 5 * 15 / 128 ** 0.5 * 2.0 ** -20
        lens = lens + new
        seen = seen + new
