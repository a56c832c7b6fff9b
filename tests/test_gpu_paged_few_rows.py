"""Attention over paged caches by tiles of 16 and 32 query rows: probabilities rounded to 2^-16, whatever a sequence's number of rows;
and what is not finite in 8 bits, by all kernels."""
import math

import pytest
import torch

from . import paged_reference as R
from .kv8_reference import P_SPLIT
from .test_gpu_paged import RULES, SHAPES, _attend, _for_reference, _rules, ffd  # noqa: F401
from .test_gpu_paged_large import _batch

pytestmark = pytest.mark.gpu


def _is_little_work(batch):
    """What these tiles take whole (on 256 CUs): up to 40K rows times tokens of the capacity for each CU."""
    return batch.T * batch.G * batch.cap * batch.Hkv <= 256 * (40 << 10)


def _takes_32_rows(batch):
    rows = batch.T * batch.G
    return rows > 16 * batch.B and (rows + 15 * min(batch.B, batch.T)) // 16 * batch.Hkv * -(-batch.cap // 256) > 256


@pytest.mark.parametrize("lens,new,Hkv,G,page,bits", SHAPES)
def test_attention(ffd, lens, new, Hkv, G, page, bits):  # noqa: F811
    batch = R.Batch(lens, new, Hkv, G, page, bits, seed=60 + page)
    assert _is_little_work(batch)
    R.check_attention(batch, _attend(ffd, batch), P_SPLIT)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", RULES, ids=lambda r: "_".join(r))
@pytest.mark.parametrize("lens,new", [([300, 515, 90], [200, 37, 90]), ([20, 700], [3, 8])])
def test_rules(ffd, lens, new, rule, bits):  # noqa: F811
    batch = R.Batch(lens, new, 2, 4, 32, bits, seed=61, before=2, behind=3)
    assert _is_little_work(batch)
    rules = _rules(batch, rule)
    R.check_attention(batch, _attend(ffd, batch, **rules), P_SPLIT, **_for_reference(batch, rules))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", [dict()] + RULES, ids=lambda r: "_".join(r) or "plain")
@pytest.mark.parametrize("new,cap", [([8] * 32, 4096), ([7, 9, 3, 1] * 8, 4096), ([1, 40, 0, 100], 8192)], ids=["eight", "odd", "mixed"])
def test_tiles_of_32_rows(ffd, new, cap, rule, bits):  # noqa: F811
    """Batches with more than 16 rows a sequence and work for every CU."""
    B = len(new)
    lens = [cap - (131 * b) % 2000 if b % 5 else 40 + b for b in range(B)]
    new = [min(n, L) for n, L in zip(new, lens)]
    batch = R.Batch(lens, new, 2, 4, 64, bits, seed=62, before=1, behind=1, width=cap // 64, holes=[(1, 3), (2, 0)])
    assert _is_little_work(batch) and _takes_32_rows(batch)
    rules = _rules(batch, rule)
    R.check_attention(batch, _attend(ffd, batch, **rules), P_SPLIT, **_for_reference(batch, rules))


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("lens,new,at", [([200], [4], 198), ([700, 90], [300, 20], 500), ([3000], [40], 100), ([2500], [300], 2300), ([2500], [300], 30)])
def test_absmaxes_that_are_not_numbers(ffd, lens, new, at, which, large):  # noqa: F811
    """A token in 8 bits that had an infinity or NaN (its absmax is NaN, its codes zero) makes the queries that see it NaN, in every dim,
    and no other; before a window it reaches nobody."""
    if large and new[0] * 4 <= 32:
        pytest.skip("few rows")
    batch = (_batch if large else R.Batch)(lens, new, 2, 4, 16, 8, seed=63)
    clean = ffd.paged_attention(*batch.args)
    page, place = batch.table[0][at // 16], at % 16
    batch.cache[1 if which == "key" else 3][page, 1, place] = math.nan
    batch.cache[0 if which == "key" else 2][page, 1, place] = 0
    for rules in (dict(), dict(window=120, prefix_lens=R.int32([at] + [0] * (len(lens) - 1)))):
        out, lse = ffd.paged_attention(*batch.args, **rules)
        L, n = lens[0], new[0]
        i = torch.arange(L - n, L, device="cuda")
        sees = (i >= at) & (i - at < rules.get("window", 1 << 30))
        hit = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
        hit[:n, 4:] = sees.view(-1, 1)
        assert torch.equal(out.isnan().all(-1), hit) and torch.equal(out.isnan().any(-1), hit)
        assert torch.equal(lse.isnan(), hit if which == "key" else torch.zeros_like(hit))
        assert bool(out[~hit].isfinite().all())
        if not rules:                           # the same runs, whose sums take the same order
            assert torch.equal(out[~hit], clean[0][~hit])
            assert torch.equal(lse[~hit], clean[1][~hit])
        got = ffd.paged_attention_weights(*batch.args, lse.nan_to_num(0), **rules)
        token = torch.zeros_like(got, dtype=torch.bool)
        token[0, 1, at] = which == "key" and bool(sees.any())
        assert torch.equal(got.isnan(), token)
