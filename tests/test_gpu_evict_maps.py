"""A draft that keeps its whole cache beside a target that evicts per KV head: maps of tokens, gathered into the order of the slots."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("heads,groups", [(12, 8), (16, 8), (4, 1)])
def test_maps_of_tokens_are_gathered_by_positions(heads, groups):
    import paper_2510_27641_b200 as sa

    rng = np.random.default_rng(151)
    batch, n, gamma, budget, grown = 2, 200, 3, 120, 40
    head_group = [h * groups // heads for h in range(heads)] if groups > 1 else None
    width = n + grown                                      # tokens that the draft will have seen
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    by_token = np.zeros((batch, groups, width))            # what every token has got, for each decision
    scores = torch.zeros(1, batch, groups, width, device=DEV)
    positions = torch.arange(width, device=DEV).to(torch.int32).expand(1, batch, groups, width).contiguous()
    lens, seen, seq_len = ints([n] * batch), n, ints([n] * batch)
    for _ in range(2):
        maps = rng.random((batch, heads, gamma, seen)).astype(np.float32)
        token_maps = torch.zeros(batch, heads, gamma, width, device=DEV)
        token_maps[..., :seen] = torch.from_numpy(maps).to(DEV)
        at = positions[0][:, torch.tensor(head_group or [0] * heads, device=DEV)].long()      # [batch, head, slot]
        slot_maps = torch.gather(token_maps, 3, at[:, :, None].expand(batch, heads, gamma, width).clamp(max=width - 1)).contiguous()
        status = torch.zeros(1, batch, groups, dtype=torch.int32, device=DEV)
        sa.accumulate_attention([slot_maps], lens, scores, n_groups=groups, head_group=head_group, row_status=status)
        for g in range(groups):
            feed = [h for h in range(heads) if head_group is None or head_group[h] == g]
            by_token[:, g, :seen] += maps[:, feed].astype(np.float64).sum((1, 2))
        m = int(lens[0])
        held = positions[0, :, :, :m].cpu().numpy()
        want = np.take_along_axis(by_token, held, -1)
        got = scores[0, :, :, :m].cpu().numpy()
        assert np.all(np.abs(got - want) <= 2.0 ** -22 * np.abs(want)) and not status.any()   # (rounded once a step)
        # the lowest go; the tokens that come next take the slots behind the budget
        src, dst, n_moves, lens = sa.evict(scores, lens, budget, positions=positions, seq_len=seq_len, scores_out=scores, positions_out=positions)
        held = positions[0, :, :, :budget].cpu().numpy()
        assert all(len(set(held[b, g])) == budget for b in range(batch) for g in range(groups))
        positions[..., budget:budget + 20] = torch.arange(seen, seen + 20, device=DEV)
        lens, seen = lens + 20, seen + 20
        seq_len = ints([seen] * batch)
