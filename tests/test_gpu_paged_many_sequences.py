"""Paged caches of batches with more sequences than a wave finds in one look, or in two."""
import random

import pytest
import torch

from . import paged_reference as R
from .kv8_reference import D, P_SPLIT
from .test_gpu_paged import _attend, ffd  # noqa: F401

pytestmark = pytest.mark.gpu


def _lengths(B, kind):
    rng = random.Random(B)
    new = {"some": [rng.choice([0, 0, 1, 2, 5]) for _ in range(B)], "one": [1] * B, "none_but_last": [0] * (B - 1) + [3], "none_but_first": [3] + [0] * (B - 1)}[kind]
    return [n + rng.randrange(20) for n in new], new


@pytest.mark.parametrize("kind", ["some", "one", "none_but_last", "none_but_first"])
@pytest.mark.parametrize("B", [63, 64, 65, 130, 4095, 4097])
def test_write_and_attend(ffd, B, kind):  # noqa: F811
    """Each row's sequence, place and page, among sequences without rows too; then attention and its weights."""
    lens, new = _lengths(B, kind)
    batch = R.Batch(lens, new, 1, 2, 16, seed=70, before=2, behind=1)
    gen = torch.Generator("cuda").manual_seed(70)
    k, v = (torch.randn(batch.T, 1, D, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    before = [x.clone() for x in batch.cache]
    out = torch.full_like(batch.q, 7.0)
    ffd.write_paged(batch.q, k, v, batch.cache, *batch.args[2:], out=out)
    rows = slice(batch.starts[0], batch.starts[-1])
    assert torch.equal(out[rows], batch.q[rows]) and bool((out[:2] == 7).all()) and bool((out[-1:] == 7).all())
    b_of = torch.tensor([b for b in range(B) for _ in range(new[b])], device="cuda")
    places = torch.tensor([lens[b] - new[b] + t for b in range(B) for t in range(new[b])], device="cuda")
    entries, at = batch.page_table[b_of, places // 16].long(), places % 16
    for x, y, w in zip(batch.cache, before, (k, v)):
        y[entries, :, at] = w[rows]
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    if B > 200:                                 # the first, the last and some others
        keep = [0, 1, 63, 64, 65, 4031, 4032, B - 2, B - 1]
    else:
        keep = range(B)
    got, lse = _attend(ffd, batch)
    weights = ffd.paged_attention_weights(*batch.args, lse)
    for b in keep:
        z, worst, _ = batch.scores(b, 0)
        v64 = batch.rows(1, b, 0)
        mine = slice(batch.starts[b], batch.starts[b + 1])
        p = torch.softmax(z, -1)
        true, mass = (p @ v64), (p @ v64.abs())
        e = R.score_error(worst, 0).unsqueeze(-1) + 2.0 ** -18              # sums and exponentials of at most 25 tokens: 29 2^-24 + 2^-22
        assert bool(((got[mine].double() - true).abs() <= 2.0 ** -8 * true.abs() + (2 * e + P_SPLIT) * mass * (1 + 2.0 ** -8)).all()), b
        w = torch.exp(z - lse[mine].double().unsqueeze(-1)).sum((0, 1))
        bound = (w * (R.score_error(worst, 0).amax() + 2.0 ** -19)) if new[b] else 0 * w        # exponent, exponential, sum of at most 10
        assert bool(((weights[b, 0, :lens[b]].double() - w).abs() <= bound + 2.0 ** -120).all()), b
        assert bool((weights[b, 0, lens[b]:] == 0).all())
