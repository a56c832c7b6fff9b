"""Runs of a shared prefix that hold no tokens, beside those that do."""
import pytest
import torch

from tests.kv8_reference import P_SPLIT, check_attention, random_cache
from tests.test_gpu_shared_prefix import _capture, _gen, _int32, _normal, _reference
from tests.test_gpu_shared_prefix_rounding import _large, _padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,G", [(8, 8), (16, 8), (32, 8), (70, 8)])
@pytest.mark.parametrize("bits", [16, 8])
def test_empty_runs(B, G, bits):
    """More runs than the prefix has tiles, rows whose lengths differ from wave to wave and only a few of which use the
    prefix at all: all workgroups of a tile have to agree on the longest. The same bits in every call."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B + bits)
    P = 200
    prefix_lens = [P if b == B - 1 else (b % 5) * 7 for b in range(B)]
    lens = [b % 2 for b in range(B)]
    q, prefix, cache = _normal(gen, B, G, 128), random_cache(gen, 1, 1, P, bits), random_cache(gen, B, 1, 64, 16)
    ref = _reference(q, prefix, prefix_lens, cache, lens)
    prefix = _padded(prefix, _large(B * G, 1, P))
    for splits in (40, 200):
        ws = ffd.new_shared_prefix_workspace(B, G, 1, prefix[0].shape[2], 64, splits).fill_(255)
        first = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens), num_splits=splits, workspace=ws)
        check_attention(first, ref, P + 1, P_SPLIT)
        for _ in range(10):
            again = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens), num_splits=splits, workspace=ws)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("rows,B,G", [(64, 10, 4), (128, 26, 4), (224, 25, 8), (320, 40, 8)])
@pytest.mark.parametrize("thousands", [64, 120, 128])
@pytest.mark.parametrize("bits", [16, 8])
def test_on_both_sides_of_little_work(rows, B, G, thousands, bits):
    """Capacities around those up to which the rows are cut into tiles of 32 (64K, 120K and 128K rows of these tiles times
    tokens per compute unit, by the prefix's form and the number of rows): a workspace of just the size asked for, which does not
    depend on the form, holds either plan."""
    from paper_2609_00097_amd import ffd
    gen = _gen(rows + thousands)
    Hkv, P = 2, 777
    work = thousands * 1024 * torch.cuda.get_device_properties(0).multi_processor_count
    cap = work // (64 * rows * Hkv) * 64
    prefix_lens, lens = [P - 9 * b for b in range(B)], [b % 3 for b in range(B)]
    q, prefix, cache = _normal(gen, B, Hkv * G, 128), random_cache(gen, 1, Hkv, P, bits), random_cache(gen, B, Hkv, 64, 16)
    ref = _reference(q, prefix, prefix_lens, cache, lens)
    for Pcap in (cap, cap + 64):
        ws = ffd.new_shared_prefix_workspace(B, Hkv * G, Hkv, Pcap, 64)
        assert ws.numel() == ffd.shared_prefix_workspace_bytes(B, Hkv * G, Hkv, Pcap, 64)
        got = ffd.shared_prefix_decode_attention(q, _padded(prefix, Pcap), _int32(prefix_lens), cache, _int32(lens), workspace=ws.fill_(255))
        check_attention(got, ref, P + 2, P_SPLIT)
        with pytest.raises(ffd.FfdError, match="WORKSPACE"):
            ffd.shared_prefix_decode_attention(q, _padded(prefix, Pcap), _int32(prefix_lens), cache, _int32(lens), workspace=ws[:-16])


@pytest.mark.parametrize("bits", [16, 8])
def test_a_captured_call_follows_the_lengths(bits):
    """One capture over several tiles of 256 rows, replayed with lengths that are sorted differently, all equal or all zero, on
    a workspace that eager calls use in between: the eager call's bits and the 64-bit form each time."""
    from paper_2609_00097_amd import ffd
    gen = _gen(bits)
    B, G, P = 70, 8, 900
    q, prefix, cache = _normal(gen, B, G, 128), random_cache(gen, 1, 1, P, bits), random_cache(gen, B, 1, 64, 8)
    whole = _padded(prefix, _large(B * G, 1, P))
    prefix_lens, lens = _int32([P] * B), _int32([b % 3 for b in range(B)])
    ws = ffd.new_shared_prefix_workspace(B, G, 1, whole[0].shape[2], 64)
    out, lse = torch.empty_like(q), torch.empty(B, G, device="cuda")

    def call():
        ffd.shared_prefix_decode_attention(q, whole, prefix_lens, cache, lens, workspace=ws, out=out, lse=lse)

    graph = _capture(call)
    for i, step in enumerate((397, 0, 53, None, 701)):
        now = [0] * B if step is None else [(step * b) % (P + 1) for b in range(B)] if step else [P] * B
        prefix_lens.copy_(_int32(now))
        q.copy_(_normal(gen, B, G, 128))
        out.fill_(float("nan"))
        graph.replay()
        eager = ffd.shared_prefix_decode_attention(q, whole, prefix_lens, cache, lens)
        ffd.shared_prefix_decode_attention(q.flip(0), whole, prefix_lens.flip(0).contiguous(), cache, lens, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]), f"replay {i}"
        check_attention((out, lse), _reference(q, prefix, now, cache, lens.tolist()), P + 2, P_SPLIT)
