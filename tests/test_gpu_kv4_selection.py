"""Lists as select_topp makes them, on the 4-bit cache: the two calls of a step, one behind the other."""
import pytest
import torch

from test_gpu_kv4 import DEV, _case, _check, _sa, _to_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,Hq,Hkv,groups", [(5, 32, 8, 1), (5, 64, 8, 1), (1, 16, 4, 4), (3, 16, 4, 4)])
@pytest.mark.parametrize("graph", [False, True])
def test_the_lists_of_the_selection(T, Hq, Hkv, groups, graph):
    sa, gen = _sa(), torch.Generator().manual_seed(121)
    lens, width, layers, draft_heads = [1000, 33, 700], 1024, 2, 8
    c = _case(122, 3, T, Hq, Hkv, lens, None, dense=True, tail=T)
    kv_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    x = 4.0 * torch.randn(layers, 3, draft_heads, 5, width, generator=gen)
    x[:, torch.arange(width) >= torch.tensor(lens)[:, None, None, None].expand(3, draft_heads, 5, width)] = float("-inf")
    probs = [p.contiguous().to(DEV) for p in torch.softmax(x, -1)]
    head_group = None if groups == 1 else [h * groups // draft_heads for h in range(draft_heads)]
    q, codes, params, table = c["q"].to(DEV), _to_gpu(c["codes"]), _to_gpu(c["params"]), c["table"].to(DEV)
    status = torch.full((3,), 7, dtype=torch.int32, device=DEV)
    layer_map = [0, 1, 1]
    idx = torch.empty(layers, 3, groups, width, dtype=torch.int32, device=DEV)
    counts, row_status = (torch.empty(layers, 3, groups, dtype=torch.int32, device=DEV) for _ in range(2))

    def step():
        sa.select_topp(probs, kv_len, layer_map, 0.9, n_groups=groups, head_group=head_group, idx=idx, counts=counts, row_status=row_status)
        return [sa.kv4_verify(q, codes, params, kv_len, block_table=table, idx=idx[u], counts=counts[u], n_groups=groups, tail_len=T,
                              status=status) for u in layer_map]

    outs = step()
    if graph:
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            outs = step()
        for out, lse, _ in outs:
            out.fill_(float("nan")), lse.fill_(float("nan"))
        idx.fill_(-1), counts.fill_(0)
        captured.replay()
    assert not row_status.any() and not status.any()
    for u, (out, lse, _) in zip(layer_map, outs):
        n = counts[u].tolist()
        lists = [[idx[u, b, h * groups // Hkv, :n[b][h * groups // Hkv]].tolist() for h in range(Hkv)] for b in range(3)]
        assert all(0 < len(one) < lens[b] or lens[b] < 100 for b in range(3) for one in lists[b])
        _check(dict(c, lists=lists), out, lse)
