"""The paged cache's entry points reject bad arguments before any launch (no GPU needed): status codes of the library, and
the binding's own checks."""
import ctypes
import os

import pytest
import torch

FAKE = 0x1000
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def so():
    from paper_2609_00097_amd import ffd
    if not os.path.exists(ffd.LIB_PATH):
        pytest.skip("libffd.so not built (run __graft_entry__.build())")
    return ffd.lib()


def _paged(k=FAKE, k_absmax=None, v=FAKE, v_absmax=None, table=FAKE, num_pages=10, page=16, max_pages=4):
    from paper_2609_00097_amd import ffd
    return ctypes.byref(ffd.PagedCache(ffd.KvCache(k, k_absmax, v, v_absmax), table, num_pages, page, max_pages))


def _rotation(q_weight=None, k_weight=None, eps=1e-6, table=FAKE, rows=100, dims=128, interleaved=0, positions=None):
    from paper_2609_00097_amd import ffd
    return ctypes.byref(ffd.Rotation(q_weight, k_weight, eps, table, rows, dims, interleaved, positions))


def _rules(softcap=0.0, window=0, slopes=None, prefix_lens=None):
    from paper_2609_00097_amd import ffd
    return ctypes.byref(ffd.ScoreRules(softcap, window, slopes, prefix_lens))


def _write(so, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, qs=None, ks=None, vs=None, q_out=FAKE, rotation=_rotation(), cache=_paged(), q_start=FAKE, lens=FAKE,
             B=2, T=5, Hq=32, Hkv=8, D=128, stream=None)
    a.update(kw)
    for s in ("qs", "ks", "vs"):
        a[s] = None if a[s] is None else (ctypes.c_int64 * 2)(*a[s])
    return so.ffd_write_paged(*a.values())


def _attend(so, **kw):
    a = dict(q=FAKE, cache=_paged(), q_start=FAKE, lens=FAKE, rules=None, B=2, T=5, Hq=32, Hkv=8, D=128, scale=0.0, out=FAKE, lse=None,
             ws=FAKE, ws_bytes=1 << 40, stream=None)
    a.update(kw)
    return so.ffd_paged_attention(*a.values())


def _weights(so, **kw):
    a = dict(q=FAKE, cache=_paged(), q_start=FAKE, lens=FAKE, rules=None, lse=FAKE, B=2, T=5, Hq=32, Hkv=8, D=128, scale=0.0, last=0, previous=None,
             weights=FAKE, stream=None)
    a.update(kw)
    return so.ffd_paged_attention_weights(*a.values())


def _evict(so, **kw):
    a = dict(cache=_paged(), new_table=FAKE, new_max_pages=2, lens=FAKE, weights=FAKE, B=2, Hkv=8, D=128, budget=20, recent=4, new_lens=FAKE, kept=FAKE,
             new_weights=None, stream=None)
    a.update(kw)
    return so.ffd_evict_paged(*a.values())


CALLS = {"write": _write, "attend": _attend, "weights": _weights, "evict": _evict}
CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(k=FAKE + 8), 1), (dict(k_absmax=FAKE), 1), (dict(v_absmax=FAKE), 1), (dict(k_absmax=FAKE + 2, v_absmax=FAKE), 1),
          (dict(table=None), 1), (dict(table=FAKE + 2), 1), (dict(num_pages=0), 1), (dict(num_pages=-3), 1), (dict(max_pages=0), 1), (dict(page=0), 1),
          (dict(page=48), 1), (dict(page=8), 2), (dict(page=512), 2), (dict(page=256, max_pages=(1 << 20) + 1), 2)]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw,status", CACHES)
def test_cache_checks(so, call, kw, status):
    assert CALLS[call](so, cache=_paged(**kw)) == status


@pytest.mark.parametrize("call", ["write", "attend", "weights"])
@pytest.mark.parametrize("kw,status", [
    (dict(cache=None), 1), (dict(q_start=None), 1), (dict(lens=None), 1), (dict(q_start=FAKE + 2), 1), (dict(lens=FAKE + 1), 1), (dict(q=FAKE + 8), 1),
    (dict(Hq=30), 1), (dict(Hq=24), 2), (dict(Hq=128), 2), (dict(Hkv=0), 1), (dict(Hq=0), 1), (dict(D=64), 2), (dict(B=-1), 1), (dict(T=-1), 1), (dict(B=70000), 2),
    (dict(T=1 << 25), 2), (dict(T=1 << 24, Hq=64, Hkv=64), 2),
])
def test_batch_checks(so, call, kw, status):
    assert CALLS[call](so, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k=FAKE + 2), 1), (dict(v=FAKE + 8), 1), (dict(q=None), 1), (dict(q_out=None), 1), (dict(q_out=FAKE + 4), 1),
    (dict(qs=(4096, 4)), 1), (dict(ks=(-8, 128)), 1), (dict(vs=(1024, 12)), 1), (dict(rotation=_rotation), 1),
    (dict(T=0, k=None, cache=None), 0), (dict(B=0, k=None, cache=None), 0),
])
def test_write_checks(so, kw, status):
    if kw.get("rotation") is _rotation:
        for bad in (dict(eps=-1e-6), dict(eps=NAN), dict(eps=INF), dict(rows=0), dict(dims=0), dict(dims=33), dict(dims=130), dict(table=FAKE + 4),
                    dict(q_weight=FAKE + 2), dict(k_weight=FAKE + 8), dict(positions=FAKE + 2)):
            assert _write(so, rotation=_rotation(**bad)) == 1, bad
        assert _write(so, rotation=_rotation(dims=48)) == 2
        return
    assert _write(so, **kw) == status


@pytest.mark.parametrize("call", ["attend", "weights"])
@pytest.mark.parametrize("kw", [dict(softcap=-1.0), dict(softcap=NAN), dict(softcap=INF), dict(window=-1), dict(slopes=FAKE + 2), dict(prefix_lens=FAKE + 1)])
def test_rule_checks(so, call, kw):
    assert CALLS[call](so, rules=_rules(**kw)) == 1
    for scale in (-1.0, NAN, INF):
        assert CALLS[call](so, scale=scale) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(out=FAKE + 8), 1), (dict(ws=FAKE + 8), 1), (dict(lse=FAKE + 2), 1), (dict(ws_bytes=1000), 3),
    (dict(B=60000, Hq=64, Hkv=64, T=60000), 2), (dict(T=0, q=None, cache=None), 0), (dict(B=0, q=None), 0),
])
def test_attention_checks(so, kw, status):
    assert _attend(so, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(lse=None), 1), (dict(weights=None), 1), (dict(weights=FAKE + 8), 1), (dict(previous=FAKE + 4), 1), (dict(lse=FAKE + 2), 1), (dict(last=-1), 1),
    (dict(B=60000, Hq=64, Hkv=64), 2), (dict(B=0, weights=None), 0),
])
def test_weights_checks(so, kw, status):
    assert _weights(so, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(cache=None), 1), (dict(new_table=None), 1), (dict(new_table=FAKE + 2), 1), (dict(new_max_pages=0), 1), (dict(lens=None), 1), (dict(weights=None), 1),
    (dict(weights=FAKE + 8), 1), (dict(new_lens=None), 1), (dict(kept=None), 1), (dict(kept=FAKE + 2), 1), (dict(new_weights=FAKE + 2), 1), (dict(budget=0), 1),
    (dict(budget=33), 1), (dict(recent=-1), 1), (dict(recent=21), 1), (dict(Hkv=0), 1), (dict(D=64), 2), (dict(B=-1), 1), (dict(B=70000), 2),
    (dict(new_max_pages=1 << 25), 2), (dict(B=60000, Hkv=64), 2), (dict(B=0, kept=None), 0),
])
def test_evict_checks(so, kw, status):
    assert _evict(so, **kw) == status


def test_workspace(so):
    size = so.ffd_paged_workspace_bytes
    assert size(32, 32, 32, 8, 128) > 0 and size(1, 8192, 32, 8, 128) > 0
    for bad in ((0, 5, 32, 8, 128), (1, 0, 32, 8, 128), (1, 5, 30, 8, 128), (1, 5, 32, 8, 64), (1, 1 << 25, 32, 8, 128), (60000, 60000, 64, 64, 128)):
        assert size(*bad) == 0
    assert _attend(so, ws_bytes=size(2, 5, 32, 8, 128) - 1) == 3


def test_binding_checks():
    """What the binding itself refuses, by name."""
    from paper_2609_00097_amd import ffd
    cache = tuple(torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16) for _ in range(2))
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    table, q_start, lens = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="q must be a CUDA"):
        ffd.paged_attention(q, cache, table, q_start, lens)
    with pytest.raises(ValueError, match="q must be \\[T"):
        ffd.paged_attention(q[0], cache, table, q_start, lens)
    with pytest.raises(ValueError, match="cache must be"):
        ffd.write_paged(q, q[:, :2], q[:, :2], cache[:1], table, q_start, lens)
    with pytest.raises(ValueError, match="cache k must be a CUDA"):
        ffd.write_paged(q, q[:, :2], q[:, :2], cache, table, q_start, lens)
    with pytest.raises(ValueError, match="cache k must be a CUDA"):
        ffd.evict_paged(cache, table, table, lens, torch.zeros(1, 2, 32), 8)
    with pytest.raises(ValueError, match="q must be \\[T"):
        ffd.paged_attention_weights(None, cache, table, q_start, lens, torch.zeros(3, 4))


def test_evict_overlaps(so):
    """new_weights on the weights, and one table for both sides."""
    weights, new = 4 * 2 * 8 * 64, 4 * 2 * 8 * 32               # bytes
    for at in (FAKE, FAKE + weights - 4, FAKE - new + 4):
        assert _evict(so, new_table=FAKE + 64, new_weights=at) == 1
    assert _evict(so, new_table=FAKE) == 1


def test_integers_of_more_than_32_bits():
    from paper_2609_00097_amd import ffd
    for x in (1 << 31, (1 << 32) + 5, -(1 << 31) - 1):
        with pytest.raises(ValueError, match="window must fit 32 bits"):
            ffd._need_int(x, "window")
    ffd._need_int((1 << 31) - 1, "window")


def test_packed_structures():
    """What the binding packs is what ctypes lays out."""
    from paper_2609_00097_amd import ffd
    assert ffd._pack_paged(1, 2, 3, 4, 5, 6, 7, 8) == bytes(ffd.PagedCache(ffd.KvCache(1, 2, 3, 4), 5, 6, 7, 8))
    assert ffd._pack_rotation(1, 2, 0.5, 3, 4, 5, True, 6) == bytes(ffd.Rotation(1, 2, 0.5, 3, 4, 5, 1, 6))
    assert ffd._pack_rules(20.0, 3, 4, 5) == bytes(ffd.ScoreRules(20.0, 3, 4, 5))
    assert ffd._pack_strides(1 << 40, 8) == bytes((ctypes.c_int64 * 2)(1 << 40, 8))
