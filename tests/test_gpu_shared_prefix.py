"""Decode attention over a shared prefix and each sequence's own tokens against a plain 64-bit form."""
import math

import pytest
import torch

from tests.kv8_reference import D, P_BF16, P_SPLIT, attention, check_attention, random_cache, values

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cap(lens):
    return max(64, -(-max(lens) // 64) * 64)


def _spoil(cache, lens):
    """NaN behind each sequence's tokens (the codes of an 8-bit cache at their limit)."""
    for t in cache:
        for b, n in enumerate(lens):
            t[b, :, max(n, 0):] = 127 if t.dtype == torch.int8 else math.nan


def _with_room(prefix, rows, room):
    """The prefix in a capacity for which more than 32 query rows are not cut into tiles of 32, NaN behind its tokens."""
    if not room or rows <= 32:
        return prefix
    Hkv, P = prefix[0].shape[1:3]
    work = 81 * 1024 * torch.cuda.get_device_properties(0).multi_processor_count
    cap = 64 * -(-work // (64 * rows * Hkv))
    if cap <= P:
        return prefix
    whole = tuple(torch.empty(1, Hkv, cap, *t.shape[3:], dtype=t.dtype, device="cuda") for t in prefix)
    _spoil(whole, [P])
    for big, t in zip(whole, prefix):
        big[:, :, :P] = t
    return whole


def _reference(q, prefix, prefix_lens, cache, lens, scale=None):
    return attention(q, [(*values(prefix), prefix_lens), (*values(cache), lens)], scale)


# query rows of a KV head (B * G) around the kernel's tiles of 16, 32 and 64 rows
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 1, 1), (1, 16, 2), (4, 8, 2), (17, 2, 2), (8, 8, 2), (33, 1, 1), (16, 4, 1), (13, 10, 2)])
@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("prefix_bits,own_bits", [(16, 16), (8, 8), (8, 16), (16, 8)])
def test_full_prefix(B, Hq, Hkv, prefix_bits, own_bits, room):
    from paper_2609_00097_amd import ffd
    if Hq // Hkv not in (1, 2, 4, 8):
        Hq = 8 * Hkv
    gen = _gen(B * Hq)
    P, lens = 300, [(37 * b + 1) % 130 for b in range(B)]
    q = _normal(gen, B, Hq, D)
    prefix, cache = random_cache(gen, 1, Hkv, _cap([P]), prefix_bits), random_cache(gen, B, Hkv, _cap(lens), own_bits)
    _spoil(prefix, [P])
    _spoil(cache, lens)
    print(f"case shared B={B} Hq={Hq} Hkv={Hkv} bits {prefix_bits} {own_bits} room {room}", flush=True)
    got = ffd.shared_prefix_decode_attention(q, _with_room(prefix, B * (Hq // Hkv), room), _int32([P] * B), cache, _int32(lens))
    torch.cuda.synchronize()
    check_attention(got, _reference(q, prefix, [P] * B, cache, lens), P + 130, P_BF16)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("prefix_lens,lens", [
    ([0, 1, 31, 32, 33, 127, 128, 129], [0, 0, 1, 64, 65, 3, 0, 0]),
    ([0] * 5, [0, 5, 0, 64, 1]),                                      # nobody uses it
    ([1000, 0, 4000, -7, 99999], [0, 0, 0, 10, -1]),                  # clamped to the capacity
    ([64], [0]),
    ([0, 0], [0, 0]),
])
def test_parts_of_the_prefix(bits, prefix_lens, lens, room):
    from paper_2609_00097_amd import ffd
    gen = _gen(len(lens) + bits)
    B, Hq, Hkv, Pcap = len(lens), 16, 2, 4032
    q = _normal(gen, B, Hq, D)
    prefix, cache = random_cache(gen, 1, Hkv, Pcap, bits), random_cache(gen, B, Hkv, 128, bits)
    if room:                                              # the longest one is not clamped then
        prefix_lens = [min(n, Pcap) for n in prefix_lens]
    clamped = [min(max(n, 0), Pcap) for n in prefix_lens]
    own = [min(max(n, 0), 128) for n in lens]
    _spoil(prefix, [max(clamped)])
    _spoil(cache, own)
    print(f"case shared parts {prefix_lens} {lens} bits {bits} room {room}", flush=True)
    got = ffd.shared_prefix_decode_attention(q, _with_room(prefix, 8 * B, room), _int32(prefix_lens), cache, _int32(lens))
    torch.cuda.synchronize()
    check_attention(got, _reference(q, prefix, clamped, cache, own), Pcap + 128, P_BF16)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("copies", [1, 9])
def test_infinities_and_nan_reach_only_the_rows_that_see_them(G, copies, room):
    """Keys and values of prefix tokens that some sequences use and others do not, within one tile of tokens and in
    tiles of their own; from 5 to 360 query rows."""
    from paper_2609_00097_amd import ffd
    gen = _gen(5)
    prefix_lens, lens = [40, 44, 60, 200, 300] * copies, [3, 0, 10, 0, 1] * copies
    B = len(lens)
    q = _normal(gen, B, G, D)
    prefix, cache = random_cache(gen, 1, 1, 320, 16), random_cache(gen, B, 1, 64, 16)
    clean = _reference(q, prefix, prefix_lens, cache, lens)
    prefix[1][0, 0, 42, 9] = math.inf
    prefix[1][0, 0, 50, 17] = math.nan
    prefix[0][0, 0, 250, 3] = math.nan
    prefix[1][0, 0, 299, 100] = -math.inf
    prefix = _with_room(prefix, B * G, room)
    out, lse = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens))
    torch.cuda.synchronize()
    used = torch.tensor(prefix_lens)
    want = torch.zeros(B, G, D, dtype=torch.bool)
    want[used > 42, :, 9] = True
    want[used > 50, :, 17] = True
    want[used > 299] = True
    assert torch.equal(~out.isfinite().cpu(), want)
    mid = (used > 42) & (used <= 299)
    assert bool((out.cpu()[mid][:, :, 9] == math.inf).all()) and out.cpu()[used > 50][:, :, 17].isnan().all()
    o, fine = out.cpu().clone(), used <= 299
    o[want] = clean[0][want].bfloat16()
    check_attention((o[fine], lse.cpu()[fine]), tuple(t[fine] for t in clean), 310, P_BF16)


@pytest.mark.parametrize("B,G,bits", [(1, 1, 16), (4, 4, 16), (4, 4, 8), (4, 8, 16), (4, 8, 8), (40, 4, 16), (33, 8, 8)])
def test_probabilities_of_small_tiles_have_two_parts(B, G, bits):
    """Tiles of 16 and 32 query rows round a probability to 2^-16, not to 2^-8."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B + G)
    P, lens = 1000, [(19 * b) % 60 for b in range(B)]
    prefix_lens = [P - 13 * b for b in range(B)]
    q = _normal(gen, B, 2 * G, D)
    prefix, cache = random_cache(gen, 1, 2, _cap([P]), bits), random_cache(gen, B, 2, 64, bits)
    _spoil(prefix, [P])
    got = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens))
    check_attention(got, _reference(q, prefix, prefix_lens, cache, lens), P + 60, P_SPLIT)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("B,G", [(2, 1), (3, 4), (4, 8), (9, 8), (20, 8), (40, 8)])
def test_infinite_values_that_every_row_sees(B, G, room):
    from paper_2609_00097_amd import ffd
    gen = _gen(B * G)
    P, special = 700, [(5, 3, math.inf), (333, 127, -math.inf), (334, 64, math.inf), (690, 0, -math.inf), (200, 50, math.nan)]
    q, prefix, cache = _normal(gen, B, G, D), random_cache(gen, 1, 1, _cap([P]), 16), random_cache(gen, B, 1, 64, 16)
    lens = [b % 3 for b in range(B)]
    clean = _reference(q, prefix, [P] * B, cache, lens)
    for t, d, x in special:
        prefix[1][0, 0, t, d] = x
    prefix = _with_room(prefix, B * G, room)
    out, lse = (t.cpu() for t in ffd.shared_prefix_decode_attention(q, prefix, _int32([P] * B), cache, _int32(lens)))
    for t, d, x in special:
        assert out[:, :, d].isnan().all() if math.isnan(x) else bool((out[:, :, d] == x).all()), f"token {t}"
        out[:, :, d] = clean[0][:, :, d].bfloat16()
    check_attention((out, lse), clean, P + 3, P_BF16)


@pytest.mark.parametrize("G", [1, 4, 8])
def test_infinities_and_nan_in_own_caches(G):
    """In tiles that end inside the sequence and in whole ones, behind them and at the last token."""
    from paper_2609_00097_amd import ffd
    gen = _gen(7)
    lens, prefix_lens = [100, 128, 1, 45, 300, 31], [0, 5, 10, 0, 64, 0]
    B = len(lens)
    q = _normal(gen, B, G, D)
    prefix, cache = random_cache(gen, 1, 1, 64, 16), random_cache(gen, B, 1, 320, 16)
    clean = _reference(q, prefix, prefix_lens, cache, lens)
    _spoil(cache, lens)
    special = [(0, 7, 3, math.inf), (0, 99, 9, -math.inf), (1, 64, 17, math.nan), (1, 127, 5, math.inf), (2, 0, 100, math.inf),
               (3, 44, 127, -math.inf), (4, 200, 64, math.inf), (4, 290, 0, -math.inf), (5, 2, 2, math.inf)]
    for b, t, d, x in special:
        cache[1][b, 0, t, d] = x
    out, lse = (t.cpu() for t in ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens)))
    for b, t, d, x in special:
        assert out[b, :, d].isnan().all() if math.isnan(x) else bool((out[b, :, d] == x).all()), f"sequence {b}, token {t}"
        out[b, :, d] = clean[0][b, :, d].bfloat16()
    check_attention((out, lse), clean, 364, P_BF16)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("G", [1, 8])
def test_a_nan_token_of_an_8_bit_prefix_reaches_only_the_rows_that_see_it(G, room):
    from paper_2609_00097_amd import ffd
    gen = _gen(6)
    prefix_lens, lens = [40, 44, 60, 200, 300] * 5, [3, 0, 10, 0, 1] * 5
    q = _normal(gen, 25, G, D)
    prefix, cache = random_cache(gen, 1, 1, 320), random_cache(gen, 25, 1, 64)
    clean = _reference(q, prefix, prefix_lens, cache, lens)
    prefix[3][0, 0, 42] = math.nan                        # a value
    prefix[1][0, 0, 250] = math.nan                       # a key
    prefix = _with_room(prefix, 25 * G, room)
    out, lse = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens))
    torch.cuda.synchronize()
    fine = torch.tensor(prefix_lens) <= 42
    assert out.cpu()[~fine].isnan().all()
    check_attention((out.cpu()[fine], lse.cpu()[fine]), tuple(t[fine] for t in clean), 310, P_BF16)


@pytest.mark.parametrize("room", [False, True])
def test_splits_scale_and_given_outputs(room):
    from paper_2609_00097_amd import ffd
    gen = _gen(7)
    B, Hq, Hkv, P, lens = (12 if room else 6), 8, 2, 2500, [700, 0, 1, 64, 333, 10] * (2 if room else 1)
    q, prefix, cache = _normal(gen, B, Hq, D), random_cache(gen, 1, Hkv, _cap([P])), random_cache(gen, B, Hkv, 704, 16)
    ref = _reference(q, prefix, [P] * B, cache, lens, 0.15)
    prefix = _with_room(prefix, 4 * B, room)
    for splits in (1, 2, 9, 40, 0):                       # 40: more runs than the prefix has rounds
        out, lse = torch.full_like(q, 7.0), torch.full((B, Hq), 7.0, device="cuda")
        ws = ffd.new_shared_prefix_workspace(B, Hq, Hkv, prefix[0].shape[2], 704, splits)
        ws.fill_(255)                                     # NaN wherever the call reads what it has not written
        got = ffd.shared_prefix_decode_attention(q, prefix, _int32([P] * B), cache, _int32(lens), num_splits=splits,
                                                 softmax_scale=0.15, workspace=ws, out=out, lse=lse)
        torch.cuda.synchronize()
        assert got[0] is out and got[1] is lse
        check_attention(got, ref, P + 700, P_BF16)
    assert ffd.shared_prefix_decode_attention(q, prefix, _int32([P] * B), cache, _int32(lens), return_lse=False)[1] is None
    with pytest.raises(ffd.FfdError, match="WORKSPACE"):
        ffd.shared_prefix_decode_attention(q, prefix, _int32([P] * B), cache, _int32(lens), workspace=ws[:4096])
    with pytest.raises(ValueError, match="prefix"):
        ffd.shared_prefix_decode_attention(q, cache, _int32([P] * B), cache, _int32(lens))
    with pytest.raises(ValueError, match="prefix_lens"):
        ffd.shared_prefix_decode_attention(q, prefix, _int32([P]), cache, _int32(lens))
    with pytest.raises(ValueError, match="cache v"):
        ffd.shared_prefix_decode_attention(q, prefix, _int32([P] * B), (cache[0], cache[1][:, :, :64]), _int32(lens))


@pytest.mark.parametrize("room", [False, True])
def test_many_sequences(room):
    """300 sequences (the own caches beyond the balanced mode) in several row tiles, the last one in part."""
    from paper_2609_00097_amd import ffd
    gen = _gen(9)
    B, Hq, Hkv, P = 301, 4, 1, 1500
    lens, prefix_lens = [(53 * b) % 200 for b in range(B)], [P if b % 3 else (7 * b) % P for b in range(B)]
    q = _normal(gen, B, Hq, D)
    for bits in (16, 8):
        prefix, cache = random_cache(gen, 1, Hkv, _cap([P]), bits), random_cache(gen, B, Hkv, 256, bits)
        got = ffd.shared_prefix_decode_attention(q, _with_room(prefix, 4 * B, room), _int32(prefix_lens), cache, _int32(lens))
        torch.cuda.synchronize()
        check_attention(got, _reference(q, prefix, prefix_lens, cache, lens), P + 200, P_BF16)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("B,G,kind", [(70, 4, "equal"), (256, 2, "ragged"), (33, 8, "ragged"), (90, 8, "none"), (65, 8, "one"),
                                      (257, 1, "one"), (256, 8, "two")])
def test_sequences_in_several_row_tiles(B, G, kind, bits, room):
    """More query rows than a tile holds: the sequences are taken in order of their lengths where these differ, and the
    tiles get workgroups by theirs, some of them none."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B)
    P = 1000
    prefix_lens = {"equal": [P] * B, "none": [0] * B, "one": [P if b == B // 2 else 0 for b in range(B)],
                   "two": [P if b % 2 else 3 for b in range(B)], "ragged": [(397 * b) % (P + 1) for b in range(B)]}[kind]
    lens = [b % 3 for b in range(B)]
    q = _normal(gen, B, 2 * G, D)
    prefix, cache = random_cache(gen, 1, 2, _cap([P]), bits), random_cache(gen, B, 2, 64, bits)
    ref = _reference(q, prefix, prefix_lens, cache, lens)
    prefix = _with_room(prefix, B * G, room)
    for splits in (0, 1, 5):
        ws = ffd.new_shared_prefix_workspace(B, 2 * G, 2, prefix[0].shape[2], 64, splits)
        ws.fill_(255)
        got = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens), num_splits=splits, workspace=ws)
        torch.cuda.synchronize()
        check_attention(got, ref, P + 3, P_BF16)


@pytest.mark.parametrize("own_bits,L", [(16, 128), (8, 960), (16, 1088)])
def test_many_groups_with_short_caches(own_bits, L):
    """2048 (sequence, KV head) pairs on both sides of the capacity up to which one workgroup takes a pair's tokens."""
    from paper_2609_00097_amd import ffd
    gen = _gen(L)
    B, Hkv, G, P = 256, 8, 2, 200
    lens, prefix_lens = [(53 * b) % (L + 1) for b in range(B)], [(31 * b) % (P + 1) for b in range(B)]
    q, prefix, cache = _normal(gen, B, Hkv * G, D), random_cache(gen, 1, Hkv, _cap([P]), 16), random_cache(gen, B, Hkv, L, own_bits)
    _spoil(cache, lens)
    ws = ffd.new_shared_prefix_workspace(B, Hkv * G, Hkv, _cap([P]), L).fill_(255)
    out, lse = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens), workspace=ws)
    some = [0, 1, 100, 211, 255]
    ref = _reference(q[some], prefix, [prefix_lens[b] for b in some], tuple(t[some] for t in cache), [lens[b] for b in some])
    check_attention((out[some], lse[some]), ref, P + L, P_SPLIT)


def test_equals_dense_attention_over_the_whole():
    """The same tokens as one bf16 cache per sequence through dense_decode_attention: the two round differently, each by
    a half step of bf16 and, here, of the probabilities."""
    from paper_2609_00097_amd import ffd
    gen = _gen(15)
    B, Hq, Hkv, P, n = 3, 8, 2, 640, 192
    q, (pk, pv), (k, v) = _normal(gen, B, Hq, D), random_cache(gen, 1, Hkv, P, 16), random_cache(gen, B, Hkv, n, 16)
    whole = [torch.cat([a.expand(B, -1, -1, -1), b], 2) for a, b in ((pk, k), (pv, v))]
    dense = ffd.dense_decode_attention(q, *whole, _int32([P + n] * B))
    got = ffd.shared_prefix_decode_attention(q, (pk, pv), _int32([P] * B), (k, v), _int32([n] * B))
    torch.cuda.synchronize()
    ref = attention(q, [(whole[0].double(), whole[1].double(), [P + n] * B)])
    check_attention(dense, ref, P + n, P_BF16)
    check_attention(got, ref, P + n, P_BF16)


@pytest.mark.parametrize("B", [40, 100])
@pytest.mark.parametrize("short", [0, 1, 5000])
def test_a_prefix_filled_to_its_capacity(B, short):
    """One token per sequence, at the starts of runs and a token before them, has nearly all of the weight: the staged
    kernel's first tiles, which are asked for as if the lengths were the capacity, with that and with shorter lengths."""
    from paper_2609_00097_amd import ffd
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    P = 64 * -(-(65 * 1024 * cus) // (64 * B))
    gen = _gen(B)
    k, v = torch.zeros(1, 1, P, D, dtype=torch.bfloat16, device="cuda"), _normal(gen, 1, 1, P, D)
    units = -(-(P - short) // 128)
    at = []
    for j in range(B):
        run = j * cus // B
        start = 128 * (units // cus * run + min(run, units % cus))
        at.append(min(max(start - (j & 1), 0), P - short - 1))
        k[0, 0, at[j], j] = 1
    k[:, :, P - short:] = math.nan
    v[:, :, P - short:] = math.nan
    q = torch.zeros(B, 1, D, dtype=torch.bfloat16, device="cuda")
    q[torch.arange(B), 0, torch.arange(B)] = 30.0
    cache = random_cache(gen, B, 1, 64, 16)
    out, _ = ffd.shared_prefix_decode_attention(q, (k, v), _int32([P - short] * B), cache, _int32([0] * B), softmax_scale=1.0)
    # the others' weight is at most P e^-30, 4e-8, of values below 6; the one's, a probability near 1, two roundings
    want = v[0, 0, at].double()
    assert bool(((out[:, 0].double() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -16).all())


@pytest.mark.parametrize("bits", [16, 8])
def test_prefix_behind_32_bit_offsets(bits):
    """Rows of the prefix beyond 4 GiB: everything zero but tokens near the end, whose weights are known."""
    from paper_2609_00097_amd import ffd
    P = (1 << (24 if bits == 16 else 25)) + 192
    dtype, one = (torch.bfloat16, 1.0) if bits == 16 else (torch.int8, 127)
    k, v = (torch.zeros(1, 1, P, D, dtype=dtype, device="cuda") for _ in range(2))
    q = torch.zeros(2, 1, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0
    for i, t in enumerate((P - 1, P - 70, P - 130)):
        k[0, 0, t, 0], v[0, 0, t, i] = one, one
    prefix = (k, v)
    if bits == 8:
        m = torch.ones(1, 1, P, dtype=torch.bfloat16, device="cuda")
        prefix = (k, m, v, m)
    cache = random_cache(_gen(1), 2, 1, 64, 16)
    out, lse = ffd.shared_prefix_decode_attention(q, prefix, _int32([P, P - 1]), cache, _int32([0, 0]), softmax_scale=10.0)
    torch.cuda.synchronize()
    for b in range(2):
        total = math.exp(20.0) * (3 - b) + (P - b - (3 - b))
        want = math.exp(20.0) / total
        assert abs(lse[b, 0].item() - math.log(total)) < 1e-3
        for i in range(3):
            w = want if i >= b else 0.0
            assert abs(out[b, 0, i].item() - w) <= (2.0 ** -7 + 4e-3) * w


def _capture(fn):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    torch.cuda.synchronize()
    return g


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("B,bits", [(3, 8), (12, 16), (40, 8), (70, 16)])
def test_workspaces_hold_anything(B, bits, room):
    """A workspace of NaN (all bits set) changes nothing, in the middle of sequences without tokens."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B)
    Hq, Hkv, P, L = 8, 2, 640, 192
    q, prefix, cache = _normal(gen, B, Hq, D), random_cache(gen, 1, Hkv, P, bits), random_cache(gen, B, Hkv, L, bits)
    prefix_lens, lens = _int32([(97 * b) % P * (b % 3 > 0) for b in range(B)]), _int32([(29 * b) % L * (b % 2) for b in range(B)])
    prefix = _with_room(prefix, 4 * B, room)
    ws = ffd.new_shared_prefix_workspace(B, Hq, Hkv, prefix[0].shape[2], L)
    want = ffd.shared_prefix_decode_attention(q, prefix, prefix_lens, cache, lens, workspace=ws.zero_())
    got = ffd.shared_prefix_decode_attention(q, prefix, prefix_lens, cache, lens, workspace=ws.fill_(255))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    if bits == 8:
        ws = ffd.new_kv8_workspace(B, Hq, Hkv, L)
        want = ffd.kv8_decode_attention(q, cache, lens, workspace=ws.zero_())
        got = ffd.kv8_decode_attention(q, cache, lens, workspace=ws.fill_(255))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("room", [False, True])
def test_two_calls_at_once(room):
    """Two streams with a workspace each, a small batch and one of two row tiles, give what one after the other does."""
    from paper_2609_00097_amd import ffd
    gen = _gen(51)
    jobs = []
    for B, P in ((4, 8192), (66, 4096)):
        lens, cache = _int32([(31 * b) % 256 for b in range(B)]), random_cache(gen, B, 2, 256, 16)
        prefix_lens = _int32([P - 50 * b for b in range(B)])
        prefix = _with_room(random_cache(gen, 1, 2, P, 8), 4 * B, room)
        jobs.append((_normal(gen, B, 8, D), prefix, prefix_lens, cache, lens))
    spaces = [ffd.new_shared_prefix_workspace(len(j[0]), 8, 2, j[1][0].shape[2], 256) for j in jobs]
    want = [ffd.shared_prefix_decode_attention(*j, workspace=w) for j, w in zip(jobs, spaces)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[] for _ in jobs]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ffd.shared_prefix_decode_attention(*jobs[i], workspace=spaces[i]))
    torch.cuda.synchronize()
    for results, (out, lse) in zip(got, want):
        assert all(torch.equal(o, out) and torch.equal(l, lse) for o, l in results)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
def test_a_served_batch(bits, room):
    """As a serving program uses them together: a prompt is written once, a captured step (write or copy the new
    token, advance, attend over prompt and own tokens) is replayed between eager work on the same workspace, and one
    sequence starts anew without the prompt. Every step equals the eager call and the 64-bit form."""
    from paper_2609_00097_amd import ffd
    gen = _gen(29)
    B, Hq, Hkv, P, L = 5, 16, 2, 700, 64
    prompt_k, prompt_v = _normal(gen, 1, P, Hkv, D), _normal(gen, 1, P, Hkv, D)
    if bits == 8:
        prefix, cache = ffd.empty_kv8(1, Hkv, _cap([P])), ffd.empty_kv8(B, Hkv, L)
        for chunk in range(0, P, 256):                   # a chunked prefill, which reads back what it attends over
            ffd.write_kv8(prompt_k[:, chunk:chunk + 256], prompt_v[:, chunk:chunk + 256], prefix, _int32([chunk]))
        read = ffd.read_kv8(prefix, 0, P)
        assert torch.equal(read[0], values(prefix)[0][:, :, :P].bfloat16())
    else:
        prefix = tuple(torch.zeros(1, Hkv, _cap([P]), D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache = tuple(torch.zeros(B, Hkv, L, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        prefix[0][:, :, :P], prefix[1][:, :, :P] = prompt_k.transpose(1, 2), prompt_v.transpose(1, 2)
    prefix = _with_room(prefix, 8 * B, room)
    prefix_lens, lens = _int32([P, P, 350, P, 0]), _int32([0, 3, 0, 17, 0])
    for t in cache:
        t.zero_()
    k_new, v_new, q = (_normal(gen, B, n, D) for n in (Hkv, Hkv, Hq))
    ws = ffd.new_shared_prefix_workspace(B, Hq, Hkv, prefix[0].shape[2], L)
    out, lse = torch.empty_like(q), torch.empty(B, Hq, device="cuda")

    def write():
        if bits == 8:
            ffd.write_kv8(k_new, v_new, cache, lens)
        else:
            at = lens.long().view(B, 1, 1, 1).expand(B, Hkv, 1, D)
            cache[0].scatter_(2, at, k_new.unsqueeze(2))
            cache[1].scatter_(2, at, v_new.unsqueeze(2))

    def step():
        write()
        lens.add_(1)
        ffd.shared_prefix_decode_attention(q, prefix, prefix_lens, cache, lens, workspace=ws, out=out, lse=lse)

    first = lens.clone()
    g = _capture(step)
    lens.copy_(first)
    for i in range(4):
        for t, n in ((k_new, Hkv), (v_new, Hkv), (q, Hq)):
            t.copy_(_normal(gen, B, n, D))
        if i == 2:                                       # another request takes sequence 1's place
            prefix_lens[1] = 0
            lens[1] = 0
        out.fill_(math.nan)
        g.replay()
        eager = ffd.shared_prefix_decode_attention(q, prefix, prefix_lens, cache, lens)
        ffd.shared_prefix_decode_attention(q.flip(0), prefix, prefix_lens, cache, lens, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]), f"replay {i}"
        ref = _reference(q, prefix, prefix_lens.tolist(), cache, lens.tolist())
        check_attention((out, lse), ref, P + L, P_BF16)
