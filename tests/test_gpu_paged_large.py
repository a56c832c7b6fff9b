"""Attention over paged caches by tiles of 256 query rows, which chunks of many rows over capacities of many tokens take (the
capacities here are larger than the lengths, so that small inputs take them), against 64-bit forms; long evictions."""
import math

import pytest
import torch

from . import paged_reference as R
from .kv8_reference import P_BF16
from .test_gpu_paged import RULES, _attend, _for_reference, _rules, _weights, ffd  # noqa: F401

pytestmark = pytest.mark.gpu


def _batch(lens, new, Hkv, G, page, bits, seed, **kw):
    """With a capacity that makes rows times tokens twice what the small tiles take on 256 CUs."""
    cap = 2 * 256 * (40 << 10) // (sum(new) * G * Hkv) + max(lens)
    return R.Batch(lens, new, Hkv, G, page, bits, seed=seed, width=-(-cap // page), **kw)


SHAPES = [
    # lens, new, Hkv, G, page
    ([33], [33], 1, 1, 16), ([300], [300], 2, 1, 16), ([2100], [70], 1, 8, 256), ([600], [64], 1, 4, 64), ([601], [65], 1, 4, 32),
    ([700, 129, 64], [500, 100, 64], 2, 2, 64), ([515, 3, 700, 90], [500, 1, 9, 90], 1, 8, 16), ([1000, 0, 500], [300, 0, 17], 3, 4, 128),
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("lens,new,Hkv,G,page", SHAPES)
def test_attention(ffd, lens, new, Hkv, G, page, bits):
    batch = _batch(lens, new, Hkv, G, page, bits, 30, before=1, behind=2)
    R.check_attention(batch, _attend(ffd, batch), P_BF16)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", RULES + [dict(softcap=1024.0), dict(softcap=1e6), dict(softcap=1e36), dict(softcap=0.01), dict(softcap=1e-30), dict(window=64, slopes=True), dict(window=257, softcap=30.0)],
                         ids=lambda r: "_".join(f"{k}{v if v is not True else ''}" for k, v in r.items()))
@pytest.mark.parametrize("lens,new", [([700], [700]), ([1500, 515, 90, 40], [200, 300, 90, 1])])
def test_rules(ffd, lens, new, rule, bits):
    batch = _batch(lens, new, 2, 4, 32, bits, 31)
    rules = _rules(batch, rule)
    R.check_attention(batch, _attend(ffd, batch, **rules), P_BF16, **_for_reference(batch, rules))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", [dict(), dict(window=90), dict(softcap=20.0, prefix=True)], ids=lambda r: "_".join(r) or "plain")
def test_pages_that_are_not_there(ffd, bits, rule):
    holes = [(0, 0), (0, 5), (0, 6), (0, 40), (1, 0), (1, 1), (1, 2), (1, 3), (1, 11)]
    batch = _batch([900, 190], [400, 190], 2, 4, 16, bits, 32, holes=holes)
    rules = _rules(batch, rule)
    got = _attend(ffd, batch, **rules)
    R.check_attention(batch, got, P_BF16, **_for_reference(batch, rules))
    if not rule:
        at = batch.starts[1]
        assert bool((got[1][at:at + 64] == -math.inf).all()) and bool((got[0][at:at + 64] == 0).all())


def test_lengths_out_of_range(ffd):
    batch = _batch([30, 600, 300], [90, 100, 310], 1, 4, 16, 16, 33)          # fewer tokens than new ones
    got = _attend(ffd, batch)
    R.check_attention(batch, got, P_BF16)
    assert bool((got[1][:60] == -math.inf).all()) and bool((got[1][190:200] == -math.inf).all())
    lens = R.int32([-5, 600, 300])
    out, lse = ffd.paged_attention(*batch.args[:4], lens)
    assert bool((lse[:90] == -math.inf).all()) and bool((out[:90] == 0).all()) and torch.equal(out[90:], got[0][90:])
    # Places far behind the table: every query sees all of the two pages that are there, whose last two rows are NaN.
    lens = R.int32([2 ** 31 - 1, 600, 300])
    out, lse = ffd.paged_attention(*batch.args[:4], lens)
    assert bool(lse[:90].isnan().all())
    # the others' runs are cut elsewhere: two roundings of a result, and of its probabilities, apart
    assert bool(((out - got[0]).abs()[90:] <= 2.0 ** -7 * got[0].abs()[90:] + 2.0 ** -8).all())


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(ffd, value):
    L, n, G, at = 700, 300, 4, 500
    batch = _batch([L], [n], 2, G, 16, 16, 34)
    clean = ffd.paged_attention(*batch.args)
    batch.cache[1][batch.table[0][at // 16], 1, at % 16, 5] = value
    out, lse = ffd.paged_attention(*batch.args)
    sees = torch.arange(L - n, L, device="cuda") >= at
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[:, G:, 5] = sees.view(-1, 1)
    assert bool((out[hit] == value).all() if value == value else out[hit].isnan().all())
    assert bool(out[~hit].isfinite().all()) and torch.equal(lse, clean[1])
    assert bool(((out - clean[0]).abs()[~hit] <= 2.0 ** -7 * clean[0].abs()[~hit] + 2.0 ** -8).all())
    out, _ = ffd.paged_attention(*batch.args, window=20, prefix_lens=R.int32([at - 3]))
    sees = sees & (torch.arange(L - n, L, device="cuda") - at < 20)
    assert torch.equal(out[:, G:, 5].isfinite(), ~sees.view(-1, 1).expand(-1, G))


def test_keys_that_are_not_finite(ffd):
    batch = _batch([500], [300], 1, 4, 16, 16, 35)
    batch.cache[0][batch.table[0][270 // 16], 0, 270 % 16, 3] = math.nan
    out, lse = ffd.paged_attention(*batch.args)
    nan = torch.arange(200, 500, device="cuda") >= 270
    assert torch.equal(out.isnan().all(-1).all(-1), nan) and torch.equal(out.isnan().any(-1).any(-1), nan)
    assert torch.equal(lse.isnan().any(-1), nan)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", [dict(), dict(window=5, softcap=10.0)], ids=["plain", "ruled"])
def test_rows_that_see_no_block(ffd, bits, rule):
    """Tiles of rows before the first token, the table's first entry a hole, beside one that sees tokens."""
    batch = _batch([0, 100, 10], [300, 300, 300], 1, 4, 16, bits, 43, holes=[(1, 0), (2, 0)])
    out, lse = _attend(ffd, batch, **rule)
    R.check_attention(batch, (out, lse), P_BF16, **rule)
    assert bool((lse[:500 + 16] == -math.inf).all()) and bool((lse[600:] == -math.inf).all()) and bool((out[600:] == 0).all())


@pytest.mark.parametrize("B", [3, 63, 64, 65, 130])
def test_cuts_of_several_sequences(ffd, B):
    """Tiles of several sequences cut into runs, beside ones that decode; more sequences than a wave has lanes."""
    lens, new = [(29 * b) % 90 + 1 for b in range(B)], [1] * B
    for b, L, n in ((0, 3000, 100), (B // 2, 900, 300), (B - 1, 1400, 33)):
        lens[b], new[b] = L, n
    batch = _batch(lens, new, 1, 4, 64, 16, 36)
    got = _attend(ffd, batch)
    R.check_attention(batch, got, P_BF16)
    for x, y in zip(got, _attend(ffd, batch)):
        assert torch.equal(x, y)


def test_captured(ffd):
    """A chunk beside decoding sequences in a graph: replayed with other lengths, starts, pages and a workspace full of something else."""
    batch = _batch([900, 40, 65], [300, 1, 1], 2, 4, 16, 16, 37)
    out, lse = torch.empty_like(batch.q), torch.empty(batch.q.shape[:2], device="cuda")
    ws = ffd.new_paged_workspace(batch.B, batch.T, 8, 2)
    run = lambda: ffd.paged_attention(*batch.args, workspace=ws, out=out, lse=lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for lens, new in (([900, 40, 65], [300, 1, 1]), ([500, 300, 64], [100, 200, 0]), ([1, 2, 3], [1, 2, 3]), ([0, 900, 10], [0, 0, 10]), ([700, 16, 200], [101, 1, 200])):
        other = R.Batch(lens, new, 2, 4, 16, 16, seed=38, width=batch.width, behind=batch.T - sum(new))
        k, v = (torch.zeros_like(x) for x in batch.cache)
        assert other.num_pages <= k.shape[0]
        for x, y, z in zip(batch.cache, (k, v), other.cache):
            y[:z.shape[0]] = z
            x.copy_(y)
        for x, y in ((batch.q, other.q), (batch.page_table, other.page_table), (batch.q_start, other.q_start), (batch.seq_lens, other.seq_lens)):
            x.copy_(y)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        R.check_attention(other, got, P_BF16)
        run()
        rows = slice(0, sum(new))
        assert torch.equal(got[0][rows], out[rows]) and torch.equal(got[1][rows], lse[rows])


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("cap", [2.0, 50.0, 1e4])
def test_small_scores_of_a_cap(ffd, cap, bits, large):
    """Scores far below the cap keep their relative precision: of a row that sees one token the lse is the score, of which tanh takes
    2^-24 (polynomial) and six roundings; before them its 128 products have 136, and from there it is made of powers of two and
    back, two more. Also where the other row of the wave has a score near the cap."""
    n = 300 if large else 1
    batch = _batch([n] * 2, [n] * 2, 1, 4, 16, bits, 41) if large else R.Batch([n] * 2, [n] * 2, 1, 4, 16, bits, seed=41)
    batch.q[0] *= 0.01
    batch.q[batch.starts[1]] *= 40.0
    _, lse = _attend(ffd, batch, softcap=cap)
    for b in range(2):
        z, worst, _ = batch.scores(b, 0, softcap=cap)
        got, want = lse[batch.starts[b]].double(), z[0, :, 0]
        # the first token of each sequence; far from zero of tanh's slope the roundings of the products count less
        far = 2.0 ** -22 * cap * (want.abs() > 0.45 * cap)
        assert bool(((got - want).abs() <= 136 * 2.0 ** -24 * worst[0] + 10 * 2.0 ** -24 * want.abs() + far).all()), (got, want)


@pytest.mark.parametrize("lens,last", [([3000, 600], 0), ([3000, 600], 150)])
@pytest.mark.parametrize("bits", [16, 8])
def test_weights_of_many_rows(ffd, lens, last, bits):
    """More rows than are kept in LDS at once, and a capacity that leaves most shares empty."""
    batch = R.Batch(lens, [400, 37], 2, 4, 64, bits, seed=39, width=4000)
    _, lse = ffd.paged_attention(*batch.args)
    previous = torch.rand(2, 2, batch.cap, device="cuda")
    before = previous.clone()
    got = ffd.paged_attention_weights(*batch.args, lse, last=last, previous=previous, out=previous)
    R.check_weights(batch, got, lse, last, before, before)


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "mixed"])
@pytest.mark.parametrize("L,budget,recent", [(32768, 1000, 7), (32769, 32700, 1), (40000, 20000, 7000), (33000, 33000, 10)])
def test_evict_long(ffd, kind, L, budget, recent):
    """Sequences longer than what the selection keeps in LDS."""
    page, extra = 256, -(-budget // 256)
    batch = R.Batch([L, 70], [0, 0], 1, 1, page, 8, seed=40, spare=2 * extra + 1)
    weights = _weights(kind, (2, 1, batch.cap), torch.Generator("cuda").manual_seed(40))
    new_table = R.int32([[batch.free[b * extra + i] for i in range(extra)] for b in range(2)])
    codes = batch.cache[0].clone()
    kept, new_lens, new_weights = ffd.evict_paged(batch.cache, batch.page_table, new_table, batch.seq_lens, weights, budget, recent=recent)
    for b, (want,) in enumerate(R.evicted(batch, weights, budget, recent)):
        n = len(want)
        assert int(new_lens[b]) == n and kept[b, 0, :n].tolist() == want and bool((kept[b, 0, n:] == -1).all())
        j, r = kept[b, 0, :n].long(), torch.arange(n, device="cuda")
        assert torch.equal(new_weights[b, 0, :n].view(torch.int32), weights[b, 0, j].view(torch.int32)) and bool((new_weights[b, 0, n:] == 0).all())
        assert torch.equal(batch.cache[0][new_table[b, r // page].long(), 0, r % page], codes[batch.page_table[b, j // page].long(), 0, j % page])
