"""Paged caches of 128K tokens and more, against 64-bit forms."""
import pytest
import torch

from . import paged_reference as R
from .kv8_reference import P_BF16, P_SPLIT
from .test_gpu_paged import _attend, _for_reference, _rules, _weights, ffd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", [dict(), dict(window=70000), dict(softcap=30.0, slopes=True), dict(window=1000, prefix=True)], ids=lambda r: "_".join(r) or "plain")
@pytest.mark.parametrize("lens,new,G", [([200001], [1], 4), ([131072, 5, 131000], [1, 5, 2], 2), ([140000], [70], 4), ([132000, 9000], [100, 1], 1)])
def test_attention_and_weights(ffd, lens, new, G, rule, bits):  # noqa: F811
    batch = R.Batch(lens, new, 1, G, 256, bits, seed=90)
    rules = _rules(batch, rule)
    reference = _for_reference(batch, rules)
    many = max(new) * G > 32
    got = _attend(ffd, batch, **rules)
    R.check_attention(batch, got, P_BF16 if many and bits == 16 else P_SPLIT, **reference)
    before = torch.rand(batch.B, 1, batch.cap, device="cuda")
    for last in (0, 30):
        weights = ffd.paged_attention_weights(*batch.args, got[1], last=last, previous=before, out=before.clone(), **rules)
        R.check_weights(batch, weights, got[1], last, before, before, **reference)


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "mixed"])
@pytest.mark.parametrize("L,budget,recent", [(131072, 8192, 256), (262144 - 3, 40000, 0), (131073, 131000, 1000)])
def test_evict(ffd, kind, L, budget, recent):  # noqa: F811
    page, Hkv = 256, 2
    extra = -(-budget // page)
    batch = R.Batch([L, 300], [0, 0], Hkv, 1, page, 8, seed=91, spare=2 * extra, holes=[(0, 100), (0, 511)])
    weights = _weights(kind, (2, Hkv, batch.cap), torch.Generator("cuda").manual_seed(91))
    new_table = R.int32([batch.free[:extra], batch.free[extra:2 * extra]])
    tokens = [x.clone() for x in batch.cache]
    kept, new_lens, new_weights = ffd.evict_paged(batch.cache, batch.page_table, new_table, batch.seq_lens, weights, budget, recent=recent, new_lens=batch.seq_lens)
    for b, heads in enumerate(R.evicted(batch, weights, budget, recent)):
        for h, want in enumerate(heads):
            n = len(want)
            assert int(new_lens[b]) == n and kept[b, h, :n].tolist() == want and bool((kept[b, h, n:] == -1).all())
            j, r = kept[b, h, :n].long(), torch.arange(n, device="cuda")
            assert torch.equal(new_weights[b, h, :n].view(torch.int32), weights[b, h, j].view(torch.int32)) and bool((new_weights[b, h, n:] == 0).all())
            for x, y in zip(batch.cache, tokens):
                assert torch.equal(x[new_table[b, r // page].long(), h, r % page].view(torch.uint8), y[batch.page_table[b, j // page].long(), h, j % page].view(torch.uint8))
