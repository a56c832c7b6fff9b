"""How exactly attention over paged caches is computed, where its kernels round or divide in ways of their own; against 64-bit
forms."""
import math

import pytest
import torch

from . import paged_reference as R
from .kv8_reference import P_BF16
from .test_gpu_paged import _attend, ffd  # noqa: F401
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
