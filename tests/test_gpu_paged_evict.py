"""Eviction from paged caches into the lengths it was given."""
import pytest
import torch

from . import paged_reference as R
from .test_gpu_paged import ffd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B,budget", [(1, 1), (5, 16), (70, 100), (70, 128), (70, 129), (3, 200)])
def test_lengths_in_place(ffd, B, budget, bits):  # noqa: F811
    """new_lens may be seq_lens itself, also where there are more (sequence, KV head) pairs than workgroups run at once: every head
    selects by the old length. Lengths of zero, below, at and above the budget, one without any page that is there."""
    Hkv, page = 8, 16
    lens = [(0, 100, 128, 129, 60)[b % 5] + (b // 5) for b in range(B)]
    extra = -(-budget // page)
    holes = [(4, i) for i in range(10)] if B > 4 else []
    batch = R.Batch(lens, [0] * B, Hkv, 1, page, bits, seed=50, holes=holes, spare=extra * B)
    gen = torch.Generator("cuda").manual_seed(50)
    weights = torch.rand(B, Hkv, batch.cap, generator=gen, device="cuda")
    new_table = R.int32([batch.free[b * extra:(b + 1) * extra] for b in range(B)])
    want = R.evicted(batch, weights, budget, 5 if budget > 5 else 0)
    apart = ffd.evict_paged(batch.cache, batch.page_table, new_table, batch.seq_lens, weights, budget, recent=5 if budget > 5 else 0)
    moved = [x.clone() for x in batch.cache]
    seq_lens = batch.seq_lens.clone()
    kept, new_lens, new_weights = ffd.evict_paged(batch.cache, batch.page_table, new_table, seq_lens, weights, budget,
                                                  recent=5 if budget > 5 else 0, new_lens=seq_lens)
    assert new_lens is seq_lens and new_lens.tolist() == [len(x[0]) for x in want]
    for b in range(B):
        for h in range(Hkv):
            assert kept[b, h].tolist() == want[b][h] + [-1] * (budget - len(want[b][h])), (b, h)
    assert torch.equal(kept, apart[0]) and torch.equal(new_lens, apart[1]) and torch.equal(new_weights, apart[2])
    for x, y in zip(batch.cache, moved):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_lengths_in_place_captured(ffd):  # noqa: F811
    """The same in a graph, replayed on lengths that were set anew."""
    B, Hkv, page, budget = 6, 8, 16, 48
    lens = [0, 30, 48, 49, 300, 500]
    batch = R.Batch(lens, [0] * B, Hkv, 1, page, seed=51, spare=3 * B)
    weights = torch.rand(B, Hkv, batch.cap, device="cuda")
    new_table = R.int32([batch.free[3 * b:3 * b + 3] for b in range(B)])
    seq_lens = batch.seq_lens.clone()
    kept, new_weights = torch.empty(B, Hkv, budget, dtype=torch.int32, device="cuda"), torch.zeros(B, Hkv, budget, device="cuda")

    def run():
        ffd.evict_paged(batch.cache, batch.page_table, new_table, seq_lens, weights, budget, recent=3, new_lens=seq_lens, kept=kept,
                        new_weights=new_weights)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for turn in range(3):
        weights.uniform_()
        batch.lens = lens[turn:] + lens[:turn]
        batch.lens = [min(L, n) for L, n in zip(batch.lens, lens)]          # the pages are those of the first lengths
        seq_lens.copy_(R.int32(batch.lens))
        graph.replay()
        torch.cuda.synchronize()
        want = R.evicted(batch, weights, budget, 3)
        assert seq_lens.tolist() == [len(x[0]) for x in want]
        assert [[x[x >= 0].tolist() for x in row] for row in kept.cpu()] == want
