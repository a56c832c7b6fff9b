"""How exactly attention over paged caches is computed, where its kernels round or divide in ways of their own; against 64-bit
forms."""
import math

import pytest
import torch

from . import paged_reference as R
from .kv8_reference import D, P_BF16, P_SPLIT, encode
from .test_gpu_paged import _attend, _for_reference, _rules, ffd  # noqa: F401
from .test_gpu_paged_large import SHAPES as LARGE
from .test_gpu_paged_large import _batch

pytestmark = pytest.mark.gpu


def _sized(large, lens, new, Hkv, G, page, bits, seed):
    """A batch that the tiles of 256 rows take (`large`: every sequence with more than 32 rows), or those of few rows."""
    return (_batch if large else R.Batch)(lens, new, Hkv, G, page, bits, seed=seed)


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("rule", [dict(), dict(window=1400)], ids=["plain", "window"])
def test_runs_of_tokens_with_scores_of_minus_infinity(ffd, rule, large):  # noqa: F811
    """They have no weight, also where a part of the cache that is attended to by itself has no other tokens."""
    batch = _sized(large, [3000], [300], 1, 4, 64, 16, 52)
    at = torch.arange(2000, device="cuda")
    batch.cache[0][batch.page_table[0, at // 64].long(), 0, at % 64, 3] = -math.inf
    batch.q[..., 3] = batch.q[..., 3].abs() + 0.5
    R.check_attention(batch, _attend(ffd, batch, **rule), P_BF16, **rule)


# Sequences of at most 32 query rows, and 8-bit caches: probabilities are rounded to 2^-16. Chunks over bf16: to 2^-8, but a row is
# divided by the sum of the rounded ones, which cancels what is alike.

@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("ahead", [False, True])
def test_one_heavy_token(ffd, ahead, large, bits):  # noqa: F811
    """A token with nearly all of a row's weight gives its value with the output's rounding alone: the others have e^-41 of it (key
    and query in one direction: 4 * 128 / sqrt(128) = 45, against N(0, 1)). `ahead`: one before it comes 5 nats close, so that the
    maximum that the exponents are taken against may stay behind; its rounding, of a weight of e^-5, moves the row by 2 * 2^-8 *
    e^-5 = 2^-14.2 where it is to 2^-8."""
    batch = _sized(large, [900, 640], [300, 40], 2, 4, 32, bits, 54)
    u = torch.where(torch.rand(D, device="cuda") < 0.5, -1.0, 1.0)
    keys = batch.cache[0]
    for h in range(2):
        for b, near, heavy in ((0, 70, 500), (1, 5, 300)):
            for at, size in ((near, 4 - 5 * math.sqrt(D) / D), (heavy, 4.0))[0 if ahead else 1:]:
                page, place = batch.table[b][at // 32], at % 32
                key = (size * u).bfloat16()
                if bits == 8:
                    keys[page, h, place], batch.cache[1][page, h, place] = encode(key)
                else:
                    keys[page, h, place] = key
    batch.q.copy_(u)
    R.check_attention(batch, _attend(ffd, batch), P_SPLIT if not ahead else P_SPLIT + 2.0 ** -14)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("M", [1.0, 1.3, 0.011])
def test_equal_scores(ffd, M, large, bits):  # noqa: F811
    """Queries of zeros: every row is the mean of the values it sees, which all have the same largest size and mostly one sign."""
    batch = _sized(large, [900, 640], [300, 40], 2, 4, 32, bits, 55)
    v = (torch.rand(batch.num_pages, 2, 32, D, device="cuda", generator=torch.Generator("cuda").manual_seed(55)) * 0.5 + 0.45).bfloat16()
    v[..., 0] = 1.0
    v = (v * M).bfloat16()
    for x, y in zip(batch.cache[len(batch.cache) // 2:], encode(v) if bits == 8 else (v,)):
        x.copy_(y)
    batch.q.zero_()
    R.check_attention(batch, _attend(ffd, batch), P_SPLIT)


@pytest.mark.parametrize("rule", [dict(), dict(softcap=20.0), dict(window=50, slopes=True), dict(window=33, prefix=True)], ids=lambda r: "_".join(r) or "plain")
@pytest.mark.parametrize("lens,new,Hkv,G,page", LARGE)
def test_chunks_over_8_bits(ffd, lens, new, Hkv, G, page, rule):  # noqa: F811
    batch = _batch(lens, new, Hkv, G, page, 8, 56)
    rules = _rules(batch, rule)
    R.check_attention(batch, _attend(ffd, batch, **rules), P_SPLIT, **_for_reference(batch, rules))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("large", [False, True])
def test_slopes_that_leave_the_nearest_token(ffd, large, bits):  # noqa: F811
    """Distances that overflow, slopes up to the largest number: all tokens but the query's own have no weight."""
    batch = _sized(large, [3000, 50], [300, 50], 1, 4, 64, bits, 53)
    slopes = torch.tensor([1e37, torch.finfo(torch.float32).max, 1e30, 2e36], device="cuda")
    out, lse = _attend(ffd, batch, slopes=slopes)
    weights = ffd.paged_attention_weights(*batch.args, lse, slopes=slopes)
    for b in range(2):
        rows, first = slice(batch.starts[b], batch.starts[b + 1]), batch.lens[b] - batch.new[b]
        own = slice(first, batch.lens[b])
        k, v = batch.rows(0, b, 0)[own].unsqueeze(1), batch.rows(1, b, 0)[own].unsqueeze(1)
        q = batch.q[rows].double()
        z, reach = (q * k).sum(-1) / math.sqrt(D), (q * k).abs().sum(-1) / math.sqrt(D)
        # of one token: the output's rounding, and its probability's
        assert bool(((out[rows].double() - v).abs() <= (2.0 ** -8 + P_SPLIT) * v.abs()).all())
        assert bool(((lse[rows].double() - z).abs() <= R.score_error(reach, 0) + 2.0 ** -21 * z.abs()).all())
        # e^(z - lse) of the four heads, each off by its exponent's error and the exponential's
        assert bool(((weights[b, 0, own] - 4).abs() <= (R.score_error(reach, 0) + 2.0 ** -20 * (z.abs() + 1)).sum(-1)).all())
        assert bool((weights[b, 0, :first] == 0).all()) and bool((weights[b, 0, batch.lens[b]:] == 0).all())


@pytest.mark.parametrize("T", [4, 5, 64])
def test_rows_of_no_sequence_count_for_one(ffd, T):  # noqa: F811
    """One sequence with one new token, in a batch of T rows over a long table: by T it is one of few rows or of many."""
    batch = R.Batch([700], [1], 2, 8, 32, 16, seed=57, behind=T - 1, width=50000)
    R.check_attention(batch, _attend(ffd, batch), P_SPLIT if T * 8 <= 32 else P_BF16)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("large", [False, True])
def test_tokens_of_almost_no_weight(ffd, large, bits):  # noqa: F811
    """A heavy token whose value is zero in half of the dims: there the others' probabilities, of e^-45 to e^-115 of it, are all that
    counts. Below 2^-126 = e^-87 they may be zeros, so that a result is off by up to 2^-126 times the sum of the values seen, beside
    the usual bound; a weight by up to 2^-126 for each query."""
    batch = _sized(large, [900], [300], 1, 4, 32, bits, 58)
    u = torch.where(torch.rand(D, device="cuda", generator=torch.Generator("cuda").manual_seed(58)) < 0.5, -1.0, 1.0).bfloat16()
    page, place = batch.table[0][7 // 32], 7 % 32
    key, value = 4 * u, torch.where(torch.arange(D, device="cuda") < 64, 1.0, 0.0).bfloat16()
    for x, y in zip(batch.cache, (*encode(key), *encode(value)) if bits == 8 else (key, value)):
        x[page, 0, place] = y
    for head, size in enumerate((1.0, 1.5, 2.0, 2.5)):
        batch.q[:, head] = size * u
    got, lse = _attend(ffd, batch)
    weights = ffd.paged_attention_weights(*batch.args, lse)
    z, worst, _ = batch.scores(0, 0)
    v = batch.rows(1, 0, 0)
    p, seen = torch.softmax(z, -1), (z > -math.inf).double()
    true, mass, sizes = p @ v, p @ v.abs(), seen @ v.abs()
    assert bool((p[seen > 0].log().min() < -100)) and bool((true[..., 64:].abs() < 2.0 ** -30).all())
    e = R.score_error(worst, 0).unsqueeze(-1) + (900 + 4) * 2.0 ** -24 + 2.0 ** -22
    p_error = P_BF16 if large and bits == 16 else P_SPLIT
    bound = 2.0 ** -8 * true.abs() + (2 * e + p_error) * mass * (1 + 2.0 ** -8) + 2.0 ** -126 * (sizes + 1)
    assert bool(((got.double() - true).abs() <= bound).all())
    w = torch.exp(z - lse.double().unsqueeze(-1))
    error = (w * (R.score_error(worst, 0) + 2.0 ** -22 * (lse.double().abs() + 2)).unsqueeze(-1)).sum((0, 1)) + 1202 * 2.0 ** -24 * w.sum((0, 1))
    assert bool(((weights[0, 0, :900].double() - w.sum((0, 1))).abs() <= error + 1200 * 2.0 ** -126).all())
