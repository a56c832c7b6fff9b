"""ffd_evict_paged refuses each bad argument by itself: the call is otherwise valid, and as large as no launch is, so that what is
left of it after the checks of its arguments is FFD_ERR_UNSUPPORTED (no GPU needed, and nothing is launched on one)."""
import pytest

from .test_paged_checks import FAKE, _evict, _paged, so  # noqa: F401

INVALID, UNSUPPORTED = 1, 2
# 2 * B * Hkv * ceil(budget / 128) is 2^23: the last check but the overlaps', which are in the wrong for no pointer here
BIG = dict(cache=dict(max_pages=64), new_table=FAKE + 0x100, new_max_pages=32, lens=FAKE + 0x200, weights=FAKE + 0x300, B=16384, Hkv=64, D=128, budget=512, recent=4,
           new_lens=FAKE + 0x400, kept=FAKE + 0x500, new_weights=FAKE + 0x600)


def _big(so, cache=None, **kw):  # noqa: F811
    a = dict(BIG, **kw)
    a["cache"] = _paged(**dict(BIG["cache"], **(cache or {})))
    return _evict(so, **a)


def test_all_else_is_valid(so):  # noqa: F811
    assert _big(so) == UNSUPPORTED
    assert _big(so, new_weights=None) == UNSUPPORTED and _big(so, recent=0) == UNSUPPORTED and _big(so, recent=512) == UNSUPPORTED
    assert _big(so, new_lens=BIG["lens"]) == UNSUPPORTED            # lengths in place


@pytest.mark.parametrize("kw", [
    dict(new_table=None), dict(new_table=FAKE + 0x102), dict(new_max_pages=0), dict(new_max_pages=-1), dict(lens=None), dict(lens=FAKE + 0x201), dict(weights=None),
    dict(weights=FAKE + 0x304), dict(weights=FAKE + 0x308), dict(new_lens=None), dict(new_lens=FAKE + 0x402), dict(kept=None), dict(kept=FAKE + 0x502),
    dict(new_weights=FAKE + 0x602), dict(budget=0), dict(budget=-5), dict(budget=513), dict(recent=-1), dict(recent=513), dict(Hkv=0), dict(B=-1),
    dict(cache=dict(k=None)), dict(cache=dict(table=None)), dict(cache=dict(num_pages=0)),
], ids=str)
def test_each_bad_argument(so, kw):  # noqa: F811
    assert _big(so, **kw) == INVALID


@pytest.mark.parametrize("kw", [dict(D=64), dict(B=70000), dict(Hkv=65536), dict(new_max_pages=(1 << 24) + 1), dict(cache=dict(page=8)), dict(cache=dict(page=512))], ids=str)
def test_each_unsupported_argument(so, kw):  # noqa: F811
    """Found before the pointers, of which one is missing here and would be invalid."""
    late = dict(kept=None) if "Hkv" not in kw else {}
    if "cache" in kw or "new_max_pages" in kw:
        assert _big(so, **kw, **late) == UNSUPPORTED
    else:
        assert _big(so, **kw, lens=None, new_lens=None, **late) == UNSUPPORTED
