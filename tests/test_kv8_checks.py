"""The 8-bit cache's and the shared prefix's entry points reject bad arguments before any launch (no GPU needed):
status codes of the library, and the binding's own checks."""
import ctypes
import os

import pytest
import torch

FAKE = 0x1000


@pytest.fixture(scope="module")
def so():
    from paper_2609_00097_amd import ffd
    if not os.path.exists(ffd.LIB_PATH):
        pytest.skip("libffd.so not built (run __graft_entry__.build())")
    return ffd.lib()


def _kv(k=FAKE, k_absmax=FAKE, v=FAKE, v_absmax=FAKE):
    from paper_2609_00097_amd import ffd
    return ctypes.byref(ffd.KvCache(k, k_absmax, v, v_absmax))


def _write(so, **kw):
    a = dict(k=FAKE, v=FAKE, ks=None, vs=None, cache=_kv(), start=FAKE, counts=None, B=1, T=1, Hkv=8, Lcap=4096, D=128)
    a.update(kw)
    strides = [None if a[s] is None else (ctypes.c_int64 * 3)(*a[s]) for s in ("ks", "vs")]
    return so.ffd_write_kv8(a["k"], a["v"], *strides, a["cache"], a["start"], a["counts"], a["B"], a["T"], a["Hkv"],
                            a["Lcap"], a["D"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(start=None), 1), (dict(cache=None), 1), (dict(k=FAKE + 8), 1),
    (dict(start=FAKE + 2), 1), (dict(counts=FAKE + 1), 1), (dict(T=-1), 1), (dict(Lcap=100), 1), (dict(D=96), 2),
    (dict(Hkv=0), 1), (dict(B=-1), 1), (dict(B=70000), 2), (dict(ks=(1024, 4, 128)), 1), (dict(vs=(-1024, 128, 128)), 1),
    (dict(T=0, k=None, cache=None), 0), (dict(B=0, k=None, cache=None), 0),
])
def test_write_checks(so, kw, status):
    assert _write(so, **kw) == status


@pytest.mark.parametrize("broken", [dict(k=None), dict(v=None), dict(k_absmax=None), dict(v_absmax=None),
                                    dict(k_absmax=None, v_absmax=None), dict(k=FAKE + 4), dict(v_absmax=FAKE + 2)])
def test_an_8_bit_cache_needs_all_of_its_tensors(so, broken):
    assert _write(so, cache=_kv(**broken)) == 1
    assert so.ffd_read_kv8(_kv(**broken), None, FAKE, FAKE, 1, 8, 4096, 128, 0, 1, None) == 1
    assert so.ffd_kv8_decode_attention(FAKE, _kv(**broken), FAKE, 1, 32, 8, 4096, 128, 0, 0.0, FAKE, None, FAKE, 1 << 30,
                                       None) == 1


@pytest.mark.parametrize("t0,t1,D,status", [(5, 4, 128, 1), (-1, 4, 128, 1), (0, 4097, 128, 1), (7, 7, 128, 0), (0, 1, 64, 2)])
def test_read_checks(so, t0, t1, D, status):
    assert so.ffd_read_kv8(_kv(), None, FAKE, FAKE, 1, 8, 4096, D, t0, t1, None) == status
    if t0 < t1 <= 4096 and t0 >= 0 and D == 128:
        assert so.ffd_read_kv8(_kv(), None, None, FAKE, 1, 8, 4096, D, t0, t1, None) == 1


def test_read_outputs_and_lengths_are_checked(so):
    assert so.ffd_read_kv8(_kv(), None, None, FAKE, 1, 8, 4096, 128, 0, 1, None) == 1
    assert so.ffd_read_kv8(_kv(), None, FAKE, FAKE + 8, 1, 8, 4096, 128, 0, 1, None) == 1
    assert so.ffd_read_kv8(_kv(), FAKE + 2, FAKE, FAKE, 1, 8, 4096, 128, 0, 1, None) == 1


def _attend(so, **kw):
    a = dict(q=FAKE, cache=_kv(), lens=FAKE, B=1, Hq=32, Hkv=8, Lcap=4096, D=128, splits=0, scale=0.0, out=FAKE, lse=None,
             ws=FAKE, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return so.ffd_kv8_decode_attention(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(cache=None), 1), (dict(lens=None), 1), (dict(out=None), 1), (dict(ws=None), 1),
    (dict(q=FAKE + 2), 1), (dict(ws_bytes=16), 3), (dict(D=64), 2), (dict(Hq=30), 1), (dict(Hq=24), 2), (dict(Lcap=63), 1),
    (dict(splits=-1), 1), (dict(splits=2000), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(B=60000, Hq=64, Hkv=64), 2), (dict(B=0, q=None), 0),
])
def test_kv8_attention_checks(so, kw, status):
    assert _attend(so, **kw) == status


def _shared(so, **kw):
    a = dict(q=FAKE, prefix=_kv(), prefix_lens=FAKE, Pcap=8192, own=_kv(), lens=FAKE, B=2, Hq=32, Hkv=8, Lcap=4096, D=128,
             splits=0, scale=0.0, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return so.ffd_shared_prefix_decode_attention(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(prefix=None), 1), (dict(own=None), 1), (dict(prefix_lens=None), 1), (dict(lens=None), 1),
    (dict(prefix_lens=FAKE + 2), 1), (dict(Pcap=0), 1), (dict(Pcap=100), 1), (dict(Pcap=1 << 30 | 64), 2), (dict(Lcap=32), 1),
    (dict(ws_bytes=1 << 10), 3), (dict(D=256), 2), (dict(Hq=33), 1), (dict(Hq=48), 2), (dict(splits=1025), 1),
    (dict(scale=-0.5), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(lse=FAKE + 2), 1), (dict(B=0), 0),
    (dict(B=0, Pcap=100), 1), (dict(B=60000, Hq=64, Hkv=64), 2),
])
def test_shared_prefix_checks(so, kw, status):
    assert _shared(so, **kw) == status


def test_shared_prefix_caches_are_whole(so):
    for broken in (dict(k_absmax=None), dict(v_absmax=None), dict(k=None), dict(v=FAKE + 2)):
        assert _shared(so, prefix=_kv(**broken)) == 1
        assert _shared(so, own=_kv(**broken)) == 1
    bf16 = _kv(k_absmax=None, v_absmax=None)
    assert _shared(so, prefix=bf16, own=bf16, ws_bytes=16) == 3          # the size is the first thing that is wrong


def test_kv8_workspace(so):
    size = so.ffd_kv8_workspace_bytes
    up = lambda x: -(-x // 256) * 256
    assert size(4, 32, 8, 131072, 128, 0) == so.ffd_dense_workspace_bytes(4, 32, 8, 131072, 128, 0)
    assert size(32, 32, 8, 8192, 128, 0) == so.ffd_dense_workspace_bytes(32, 32, 8, 8192, 128, 0)
    # 512 groups of 256 blocks: 170 for each of 768 workgroups, so 2048 of them (no GPU here: 256 CUs), S = 4 - 1
    assert size(64, 32, 8, 16384, 128, 0) == up(64 * 32 * (3 + 1) * 130 * 4) + 64 * 8 * 8
    assert size(64, 32, 8, 16384, 128, 1) == up(64 * 32 * 2 * 130 * 4) + 64 * 8 * 8
    assert size(300, 8, 8, 4096, 128, 1) == up(300 * 8 * 130 * 4)
    for bad in ((0, 32, 8, 4096, 128, 0), (1, 30, 8, 4096, 128, 0), (1, 32, 8, 100, 128, 0), (1, 32, 8, 4096, 64, 0),
                (1, 32, 8, 4096, 128, 5000), (60000, 64, 64, 64, 128, 0)):
        assert size(*bad) == 0
    assert _attend(so, ws_bytes=size(1, 32, 8, 4096, 128, 0) - 1) == 3


def test_shared_prefix_workspace(so):
    size = so.ffd_shared_prefix_workspace_bytes
    dense = so.ffd_dense_workspace_bytes(2, 32, 8, 4096, 128, 0)
    need = size(2, 32, 8, 8192, 4096, 128, 0)
    assert need > dense and need % 4 == 0
    assert _shared(so, ws_bytes=need - 1) == 3
    # given splits: rows rounded up to 16 times them, and those of the dense call for the same splits
    up = lambda x: -(-x // 256) * 256
    assert size(2, 32, 8, 8192, 4096, 128, 3) == up((8 * 16 * 3 + 2 * 32 * (3 + 1)) * 130 * 4) + 2 * 8 * 8
    # two tiles of 256 rows: the sequences' places
    assert size(70, 32, 8, 16384, 4096, 128, 3) == up((8 * 2 * 256 * 3 + 70 * 32 * 4) * 130 * 4) + up(70 * 16) + 70 * 8 * 8
    # little work: nine tiles of 32 rows
    assert size(70, 32, 8, 4096, 4096, 128, 3) == up((8 * 9 * 32 * 3 + 70 * 32 * 4) * 130 * 4) + 70 * 8 * 8
    assert size(300, 32, 8, 8192, 4096, 128, 3) == up((8 * 5 * 256 * 3 + 300 * 32 * 3) * 130 * 4)
    for bad in ((0, 32, 8, 8192, 4096, 128, 0), (2, 32, 8, 100, 4096, 128, 0), (2, 32, 8, 8192, 4096, 96, 0),
                (2, 30, 8, 8192, 4096, 128, 0), (2, 32, 8, 8192, 4096, 128, 5000)):
        assert size(*bad) == 0


def test_launches_past_the_limits_are_refused(so):
    huge = dict(ws_bytes=1 << 62)
    assert so.ffd_kv8_workspace_bytes(16, 65535, 65535, 64, 128, 64) == 0        # 2^20 groups of 65 workgroups
    assert _attend(so, B=16, Hq=65535, Hkv=65535, Lcap=64, splits=64, **huge) == 2
    assert so.ffd_shared_prefix_workspace_bytes(16, 65535, 65535, 64, 64, 128, 64) == 0
    assert _shared(so, B=16, Hq=65535, Hkv=65535, Pcap=64, Lcap=64, splits=64, **huge) == 2
    # 8000 groups of 1025 workgroups pass the first limit, 8000 heads of 1024 runs of the prefix do not
    assert so.ffd_kv8_workspace_bytes(1, 8000, 8000, 64, 128, 1024) > 0
    assert so.ffd_shared_prefix_workspace_bytes(1, 8000, 8000, 64, 64, 128, 1024) == 0
    assert _shared(so, B=1, Hq=8000, Hkv=8000, Pcap=64, Lcap=64, splits=1024, **huge) == 2
    assert so.ffd_write_kv8(FAKE, FAKE, None, None, _kv(), FAKE, None, 1, (1 << 28) + 1, 8, 4096, 128, None) == 2


def test_binding_refuses_host_tensors_and_wrong_shapes():
    from paper_2609_00097_amd import ffd
    cache = ffd.empty_kv8(2, 8, 128, device="cpu")
    assert [tuple(t.shape) for t in cache] == list(ffd.kv8_shapes(2, 8, 128))
    x = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16)
    lens = torch.zeros(2, dtype=torch.int32)
    q = torch.zeros(2, 32, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        ffd.write_kv8(x, x, cache, lens)
    with pytest.raises(ValueError, match="CUDA"):
        ffd.read_kv8(cache)
    with pytest.raises(ValueError, match="CUDA"):
        ffd.kv8_decode_attention(q, cache, lens)
    with pytest.raises(ValueError, match="CUDA"):
        ffd.shared_prefix_decode_attention(q, cache, lens, cache, lens)
    with pytest.raises(ValueError, match="cache must be"):
        ffd.kv8_decode_attention(q, cache[:2], lens)
    with pytest.raises(ValueError, match="cache must be"):
        ffd.shared_prefix_decode_attention(q, cache, lens, cache[:3], lens)
    with pytest.raises(ValueError, match="keys must be"):
        ffd.read_kv8((cache[0][0], *cache[1:]))
