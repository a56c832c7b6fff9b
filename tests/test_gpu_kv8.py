"""The 8-bit cache on the GPU: writing, reading back and attention against plain 64-bit forms. Codes, absmaxes and
what is read back are exact."""
import math

import pytest
import torch

from tests.kv8_reference import D, P_SPLIT, attention, check_attention, decode, encode, random_cache, values

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _filled(B, Hkv, L):
    """A cache of sentinels."""
    from paper_2609_00097_amd import ffd
    cache = ffd.empty_kv8(B, Hkv, L)
    for t, x in zip(cache, (77, 3.0, -77, 5.0)):
        t.fill_(x)
    return cache


def _same(a, b):
    """Equal, NaN being equal to NaN."""
    return torch.equal(torch.nan_to_num(a, nan=-12345.0), torch.nan_to_num(b, nan=-12345.0)) and torch.equal(a.isnan(), b.isnan())


def _check_written(cache, k, v, start, counts, L):
    """Every row of the cache: the new tokens where they belong, the sentinels elsewhere."""
    want = _filled(k.shape[0], k.shape[2], L)
    for b, (s, c) in enumerate(zip(start, counts)):
        for t in range(max(0, min(c, k.shape[1]))):
            if 0 <= s + t < L:
                for w, x in zip(want, (*encode(k[b, t]), *encode(v[b, t]))):
                    w[b, :, s + t] = x
    for name, w, x in zip(("k_codes", "k_absmax", "v_codes", "v_absmax"), want, cache):
        assert _same(x.float(), w.float()), name


@pytest.mark.parametrize("T,Hkv,L,start,counts", [
    (1, 1, 64, [0, 63], None),
    (1, 8, 128, [127, 5, 128, -1], None),                 # the last position, behind the end, before the beginning
    (1, 40, 64, [1], [1]),                                # more heads than a workgroup takes
    (3, 8, 128, [126, 0, 60], [3, 0, 2]),                 # cut off at the capacity, nothing, part of it
    (33, 2, 192, [0, 100, 180], [33, 40, 31]),            # more than T means T
    (100, 3, 256, [7, 64], [-5, 99]),
    (2, 1, 64, [2 ** 31 - 1, -2 ** 31], None),            # positions that pass 32 bits
])
def test_write_puts_exact_codes_where_they_belong(T, Hkv, L, start, counts):
    from paper_2609_00097_amd import ffd
    gen = _gen(T + Hkv)
    k, v = _normal(gen, len(start), T, Hkv, D), 3 * _normal(gen, len(start), T, Hkv, D)
    cache = _filled(len(start), Hkv, L)
    print(f"case write T={T} Hkv={Hkv} start={start} counts={counts}", flush=True)
    ffd.write_kv8(k, v, cache, _int32(start), counts=None if counts is None else _int32(counts))
    torch.cuda.synchronize()
    _check_written(cache, k, v, start, counts or [T] * len(start), L)


def test_write_takes_strided_tensors():
    """Slices of one projection's output, head-major tokens, one token without its axis, a token for every sequence."""
    from paper_2609_00097_amd import ffd
    B, T, Hkv, L = 2, 5, 4, 64
    qkv = _normal(_gen(3), B, T, 6 * Hkv, D)
    head_major = _normal(_gen(4), B, Hkv, T, D).transpose(1, 2)
    one = _normal(_gen(5), 1, T, Hkv, D).expand(B, T, Hkv, D)
    for k, v in ((qkv[:, :, 4 * Hkv:5 * Hkv], qkv[:, :, 5 * Hkv:]), (head_major, qkv[:, :, :Hkv]), (one, head_major)):
        cache = _filled(B, Hkv, L)
        ffd.write_kv8(k, v, cache, _int32([9, 30]))
        torch.cuda.synchronize()
        _check_written(cache, k, v, [9, 30], [T] * B, L)
    cache = _filled(B, Hkv, L)
    ffd.write_kv8(qkv[:, 2, :Hkv], head_major[:, 2], cache, _int32([0, 63]))
    torch.cuda.synchronize()
    _check_written(cache, qkv[:, 2:3, :Hkv], head_major[:, 2:3], [0, 63], [1, 1], L)


def test_write_of_nothing_and_refused_tensors():
    from paper_2609_00097_amd import ffd
    x = _normal(_gen(6), 2, 3, 4, 2 * D)
    cache = _filled(2, 4, 64)
    start = _int32([0, 1])
    ffd.write_kv8(x[:, :0, :, :D], x[:, :0, :, :D], cache, start)
    with pytest.raises(ValueError, match="contiguous"):
        ffd.write_kv8(x[..., ::2], x[..., :D], cache, start)
    with pytest.raises(ValueError, match="shape"):
        ffd.write_kv8(x[..., :D], x[:, :2, :, :D], cache, start)
    with pytest.raises(ValueError, match="bfloat16"):
        ffd.write_kv8(x[..., :D].float(), x[..., :D], cache, start)
    with pytest.raises(ffd.FfdError):                    # a vector that does not begin on 16 bytes
        ffd.write_kv8(x[..., 1:D + 1], x[..., :D], cache, start)
    with pytest.raises(ValueError, match="start"):
        ffd.write_kv8(x[..., :D], x[..., :D], cache, start.long())
    torch.cuda.synchronize()
    _check_written(cache, x[:, :0, :, :D], x[:, :0, :, :D], [0, 0], [0, 0], 64)


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -120, 2.0 ** 120])
def test_write_is_exact_for_every_quotient(scale):
    """For every significand of M, all bf16 values up to M of the seven octaves below it (smaller ones have code 0)
    and their negatives: ties to even, and quotients next to them."""
    from paper_2609_00097_amd import ffd
    x = torch.arange(0x3f80 - 9 * 128, 0x3f80 + 128, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda()   # up to [1, 2)
    rows = []
    for m in x[-128:]:
        part = x[x <= m]
        part = torch.nn.functional.pad(part, (0, -len(part) % 127)).view(-1, 127)
        rows.append(torch.cat([m.expand(len(part), 1), part], 1))
    k = (torch.cat(rows).double() * scale).bfloat16()[None, :, None]         # [1, T, 1, 128]
    T = k.shape[1]
    L = -(-T // 64) * 64
    cache = ffd.empty_kv8(1, 1, L)
    ffd.write_kv8(k, -k, cache, _int32([0]))
    torch.cuda.synchronize()
    codes, absmax = encode(k[0, :, 0])
    assert torch.equal(cache[0][0, 0, :T], codes) and torch.equal(cache[2][0, 0, :T], -codes)
    assert torch.equal(cache[1][0, 0, :T], absmax) and torch.equal(cache[3][0, 0, :T], absmax)


def test_write_of_zeros_subnormals_infinities_and_nan():
    from paper_2609_00097_amd import ffd
    x = _normal(_gen(8), 1, 8, 1, D)
    tiny = torch.arange(1, D + 1, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda()     # subnormals
    x[0, 0] = 0
    x[0, 1] = -0.0
    x[0, 2] = tiny
    x[0, 3, 0, 5] = math.inf
    x[0, 4, 0, 127] = -math.inf
    x[0, 5, 0, 64] = math.nan
    x[0, 6] = torch.finfo(torch.bfloat16).max
    x[0, 7] = tiny
    x[0, 7, 0, 0] = torch.finfo(torch.bfloat16).max
    cache = _filled(1, 1, 64)
    ffd.write_kv8(x, x.flip(1), cache, _int32([20]))
    torch.cuda.synchronize()
    _check_written(cache, x, x.flip(1), [20], [8], 64)
    k, _ = ffd.read_kv8(cache, 20, 28)
    assert k[0, 0, [3, 4, 5]].isnan().all() and k[0, 0, [0, 1, 2, 6, 7]].isfinite().all()
    assert torch.equal(k[0, 0, 6], x[0, 6, 0]) and bool((k[0, 0, :2] == 0).all())


@pytest.mark.parametrize("B,Hkv,L,t0,t1,lens", [
    (1, 1, 64, 0, 1, None), (2, 3, 192, 63, 130, None), (3, 2, 320, 5, 320, [320, 0, 100]), (2, 8, 128, 127, 128, [127, 128]),
    (2, 1, 128, 10, 100, [-3, 1000]), (1, 2, 64, 33, 33, None)])
def test_read_is_correctly_rounded(B, Hkv, L, t0, t1, lens):
    from paper_2609_00097_amd import ffd
    cache = random_cache(_gen(L + t1), B, Hkv, L)
    cache[1].mul_(2.0 ** -60)
    out = tuple(torch.full((B, Hkv, t1 - t0, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    print(f"case read {B}x{Hkv}x{L} [{t0}, {t1}) lens {lens}", flush=True)
    got = ffd.read_kv8(cache, t0, t1, seq_lens=None if lens is None else _int32(lens), out=out)
    torch.cuda.synchronize()
    assert got[0] is out[0] and got[1] is out[1]
    for x, want in zip(got, values(cache)):
        want = want[:, :, t0:t1].bfloat16()              # one rounding: 64 bits hold n M / 127 to far below a tie
        if lens is not None:
            for b, n in enumerate(lens):
                want[b, :, max(0, n - t0):] = 0
        assert torch.equal(x, want)


def test_read_is_exact_for_every_code_and_significand():
    from paper_2609_00097_amd import ffd
    M = torch.arange(0x3f80, 0x4000, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda()       # [1, 2)
    M = torch.cat([M, M * 2.0 ** 126, M * 2.0 ** -126, torch.arange(1, 129, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda()])
    n = torch.arange(128, dtype=torch.int8, device="cuda").expand(len(M), D).contiguous()
    cache = (n[None, None], M[None, None].contiguous(), -n[None, None], M[None, None].contiguous())
    k, v = ffd.read_kv8(cache)
    torch.cuda.synchronize()
    assert torch.equal(k[0, 0], decode(n, M).bfloat16()) and torch.equal(v[0, 0], decode(-n, M).bfloat16())


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 4), (8, 2), (16, 2)])
@pytest.mark.parametrize("lens", [(1,), (31, 32, 33), (63, 64, 65, 0), (1000, 4097)])
def test_attention(Hq, Hkv, lens):
    from paper_2609_00097_amd import ffd
    gen = _gen(Hq + sum(lens))
    L = -(-max(lens) // 64) * 64 + 64
    q, cache = _normal(gen, len(lens), Hq, D), random_cache(gen, len(lens), Hkv, L)
    for b, n in enumerate(lens):                         # behind a sequence anything may lie
        cache[0][b, :, n:] = 127
        cache[1][b, :, n:] = math.nan
        cache[2][b, :, n:] = -127
        cache[3][b, :, n:] = math.inf
    print(f"case kv8 Hq={Hq} Hkv={Hkv} lens={lens}", flush=True)
    got = ffd.kv8_decode_attention(q, cache, _int32(lens))
    torch.cuda.synchronize()
    check_attention(got, attention(q, [(*values(cache), lens)]), max(lens), P_SPLIT)


def test_attention_splits_scale_and_given_outputs():
    from paper_2609_00097_amd import ffd
    gen = _gen(11)
    lens = (3000, 0, 777)
    q, cache = 2 * _normal(gen, 3, 8, D), random_cache(gen, 3, 2, 3008)
    ref = attention(q, [(*values(cache), lens)], scale=0.2)
    for splits in (1, 2, 7, 48, 0):
        out, lse = torch.full_like(q, 7.0), torch.full((3, 8), 7.0, device="cuda")
        got = ffd.kv8_decode_attention(q, cache, _int32(lens), num_splits=splits, softmax_scale=0.2, out=out, lse=lse)
        torch.cuda.synchronize()
        assert got[0] is out and got[1] is lse
        check_attention(got, ref, max(lens), P_SPLIT)
    assert ffd.kv8_decode_attention(q, cache, _int32(lens), return_lse=False)[1] is None
    with pytest.raises(ValueError, match="out"):
        ffd.kv8_decode_attention(q, cache, _int32(lens), out=out.float())
    with pytest.raises(ValueError, match="lse"):
        ffd.kv8_decode_attention(q, cache, _int32(lens), lse=lse[:2])
    with pytest.raises(ffd.FfdError, match="WORKSPACE"):
        ffd.kv8_decode_attention(q, cache, _int32(lens), workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


def test_attention_of_more_sequences_than_the_balanced_mode_takes():
    from paper_2609_00097_amd import ffd
    gen = _gen(13)
    lens = [(53 * b) % 700 for b in range(300)]
    q, cache = _normal(gen, 300, 4, D), random_cache(gen, 300, 1, 704)
    for splits in (0, 3):
        got = ffd.kv8_decode_attention(q, cache, _int32(lens), num_splits=splits)
        torch.cuda.synchronize()
        check_attention(got, attention(q, [(*values(cache), lens)]), 700, P_SPLIT)


@pytest.mark.parametrize("B,Hkv,G,L", [(3, 2, 8, 64), (5, 2, 4, 1024), (5, 2, 1, 1088), (256, 8, 2, 1088), (300, 7, 1, 128)])
def test_attention_in_one_launch(B, Hkv, G, L):
    """Around the capacities up to which a workgroup takes all tokens of a pair and writes the result: every length class,
    NaN behind the tokens, and the same as split runs within the bounds."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B + L)
    lens = [L, 0, 1, 63, 130][:B] + [(53 * b) % (L + 1) for b in range(5, B)]
    lens = [min(n, L) for n in lens]
    q, cache = _normal(gen, B, Hkv * G, D), random_cache(gen, B, Hkv, L)
    for t in cache:
        for b, n in enumerate(lens):
            t[b, :, n:] = 127 if t.dtype == torch.int8 else math.nan
    some = list(range(min(B, 5))) + ([B // 2, B - 1] if B > 5 else [])
    ref = attention(q[some], [(*values(tuple(t[some] for t in cache)), [lens[b] for b in some])])
    for splits in (0, 1, 3):
        ws = ffd.new_kv8_workspace(B, Hkv * G, Hkv, L, splits).fill_(255)
        out, lse = torch.full_like(q, 7.0), torch.full((B, Hkv * G), 7.0, device="cuda")
        ffd.kv8_decode_attention(q, cache, _int32(lens), num_splits=splits, workspace=ws, out=out, lse=lse)
        check_attention((out[some], lse[some]), ref, L, P_SPLIT)
        assert bool((out != 7.0).any(-1).all()) and bool((lse != 7.0).all())
    got = ffd.kv8_decode_attention(q, cache, _int32(lens), return_lse=False)
    assert got[1] is None
    check_attention((got[0][some], ref[1].float()), ref, L, P_SPLIT)


def test_attention_with_many_workgroups_per_compute_unit():
    """A batch whose capacity makes its automatic splits finer, with lengths far apart."""
    from paper_2609_00097_amd import ffd
    B, Hkv, L = 64, 1, 65536
    lens = [1 + (9973 * b * b) % 2500 for b in range(B)]
    lens[5], lens[40] = 0, 20000
    assert ffd.kv8_workspace_bytes(B, Hkv, Hkv, L) > ffd.workspace_bytes(B, Hkv, Hkv, L, dense=True)
    gen = _gen(14)
    q, cache = _normal(gen, B, Hkv, D), random_cache(gen, B, Hkv, 20032)
    cache = tuple(torch.nn.functional.pad(t, (0, 0) * (t.dim() == 4) + (0, L - 20032)) for t in cache)
    got = ffd.kv8_decode_attention(q, cache, _int32(lens))
    torch.cuda.synchronize()
    k, v = values([t[:, :, :20032] for t in cache])
    check_attention(got, attention(q, [(k, v, lens)]), 20000, P_SPLIT)


def test_attention_over_nan_tokens_and_large_scores():
    """A token with a NaN among those that a sequence sees makes its rows NaN, also where there is no other; scores
    of several hundred, of both signs."""
    from paper_2609_00097_amd import ffd
    gen = _gen(17)
    lens = (200, 200, 1)
    q, cache = 30 * _normal(gen, 3, 4, D), random_cache(gen, 3, 1, 256)
    cache[1][1, 0, 150] = math.nan
    cache[1][2, 0, 0] = math.nan
    out, lse = ffd.kv8_decode_attention(q, cache, _int32(lens))
    torch.cuda.synchronize()
    assert out[1:].isnan().all()
    k, v = values(cache)
    ref = attention(q[:1], [(k[:1], v[:1], lens[:1])])
    check_attention((out[:1], lse[:1]), ref, 200, P_SPLIT)


def test_attention_behind_32_bit_offsets():
    """A cache whose rows lie beyond 4 GiB of codes: all keys and values zero but for tokens near its end, which then
    have known weights."""
    from paper_2609_00097_amd import ffd
    L = (1 << 25) + 128
    codes = [torch.zeros(1, 1, L, D, dtype=torch.int8, device="cuda") for _ in range(2)]
    absmax = [torch.ones(1, 1, L, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q = torch.zeros(1, 1, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0
    hot = [L - 1, L - 70, (1 << 25) + 1]
    for i, t in enumerate(hot):
        codes[0][0, 0, t, 0] = 127
        codes[1][0, 0, t, i] = 127
    cache = (codes[0], absmax[0], codes[1], absmax[1])
    out, lse = ffd.kv8_decode_attention(q, cache, _int32([L]), softmax_scale=10.0)
    torch.cuda.synchronize()
    total = math.exp(20.0) * 3 + (L - 3)
    assert abs(lse.item() - math.log(total)) < 1e-3      # L roundings of 2^-24 at the most, and 20's
    want = math.exp(20.0) / total
    assert all(abs(out[0, 0, i].item() - want) <= (2.0 ** -8 + 4e-3) * want for i in range(3)) and bool((out[0, 0, 3:] == 0).all())
    k, _ = ffd.read_kv8(cache, L - 2, L)
    assert k[0, 0, 1, 0].item() == 1.0 and k[0, 0, 0, 0].item() == 0.0


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


def test_captured_steps_grow_the_cache():
    """One capture of [write, advance, attend]; replays with new tokens between eager work on the same workspace
    equal the eager calls on a second cache, bit for bit, and the last one the 64-bit form."""
    from paper_2609_00097_amd import ffd
    gen = _gen(19)
    B, Hq, Hkv, L = 2, 8, 2, 1088
    ours, theirs = random_cache(gen, B, Hkv, L), None
    theirs = tuple(t.clone() for t in ours)
    start = _int32([500, 1083])
    lens_g, lens_e = start.clone(), start.clone()
    k_new, v_new = _normal(gen, B, Hkv, D), _normal(gen, B, Hkv, D)
    q = _normal(gen, B, Hq, D)
    ws = ffd.new_kv8_workspace(B, Hq, Hkv, L)
    out, lse = torch.empty_like(q), torch.empty(B, Hq, device="cuda")

    def step():
        ffd.write_kv8(k_new, v_new, ours, lens_g)
        lens_g.add_(1)
        ffd.kv8_decode_attention(q, ours, lens_g, workspace=ws, out=out, lse=lse)

    kept = [t.clone() for t in ours]
    g = _capture(step)
    lens_g.copy_(start)
    for t, x in zip(ours, kept):
        t.copy_(x)
    for i in range(4):
        k_new.copy_(_normal(gen, B, Hkv, D))
        v_new.copy_(_normal(gen, B, Hkv, D))
        q.copy_(_normal(gen, B, Hq, D))
        out.fill_(math.nan)
        g.replay()
        ffd.write_kv8(k_new, v_new, theirs, lens_e)
        lens_e.add_(1)
        o, l = ffd.kv8_decode_attention(q, theirs, lens_e)
        ffd.kv8_decode_attention(q.flip(0), theirs, lens_e, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(lse, l), f"replay {i}"
        assert all(torch.equal(a, b) for a, b in zip(ours, theirs))
    check_attention((out, lse), attention(q, [(*values(ours), lens_g.tolist())]), L, P_SPLIT)


def test_calls_go_to_the_current_stream():
    """Work queued on a side stream before the call is seen by it: a cache that arrives there late."""
    from paper_2609_00097_amd import ffd
    gen = _gen(23)
    q, source = _normal(gen, 1, 8, D), random_cache(gen, 1, 2, 4096)
    cache = _filled(1, 2, 4096)
    lens = _int32([4096])
    want = ffd.kv8_decode_attention(q, source, lens)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.zeros(1 << 28, device="cuda")
        for _ in range(8):
            big.add_(1)
        for t, x in zip(cache, source):
            t.copy_(x)
        got = ffd.kv8_decode_attention(q, cache, lens)
        read = ffd.read_kv8(cache, 5, 9)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(read[0], values(source)[0][:, :, 5:9].bfloat16())
