"""Counts of moves that no eviction writes: negative ones, the smallest, more than there is room for."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_no_count_moves_more_than_the_lists_hold():
    """A block takes its share of a count by subtracting where the share begins, which must not wrap around."""
    import paper_2510_27641_b200 as sa

    counts, stride, page, pages = [-2 ** 31, -2 ** 31 + 5, -1, 0, 7, 2 ** 31 - 1], 4096, 16, 1024
    batch = len(counts)
    gen = torch.Generator().manual_seed(131)
    pool = torch.randint(-2 ** 15, 2 ** 15, (batch * pages, 2, page, 2, 128), generator=gen).to(torch.int16)
    order = torch.stack([torch.randperm(pages * page, generator=gen)[:2 * stride] for _ in range(batch)]).to(torch.int32)
    src, dst = order[:, None, :stride].contiguous(), order[:, None, stride:].contiguous()
    got, status = pool.to(DEV), torch.full((batch,), 9, dtype=torch.int32, device=DEV)
    sa.move_rows([got], src.to(DEV), dst.to(DEV), torch.tensor(counts, dtype=torch.int32, device=DEV).view(batch, 1), pages_per_seq=pages,
                 status=status)
    want = pool.clone()
    for b, n in enumerate(counts):
        n = max(0, min(n, stride))
        s, d = src[b, 0, :n].long() + b * pages * page, dst[b, 0, :n].long() + b * pages * page
        want[d // page, :, d % page] = pool[s // page, :, s % page]
    assert torch.equal(got.cpu(), want) and not status.any()
