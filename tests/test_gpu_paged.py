"""Paged caches on the GPU: writing with norms and rotation, attention of ragged chunks, attention weights, eviction, and a
run of them together, against 64-bit forms."""
import math

import pytest
import torch

from . import paged_reference as R
from .kv8_reference import D, P_BF16, P_SPLIT, encode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ffd():
    from paper_2609_00097_amd import ffd
    assert torch.cuda.is_available()
    return ffd


# ---- attention ------------------------------------------------------------------------------------------------

ROWS = 32               # query rows of a KV head up to which probabilities are rounded to 2^-16


def _p_error(batch):
    return P_SPLIT if max(batch.new) * batch.G <= ROWS else P_BF16


def _attend(ffd, batch, **rules):
    out = torch.full_like(batch.q, 7.0)
    lse = torch.full(batch.q.shape[:2], 7.0, device="cuda")
    ws = torch.full((max(ffd.paged_workspace_bytes(batch.B, batch.T, batch.q.shape[1], batch.Hkv), 16),), 255, dtype=torch.uint8, device="cuda")
    got = ffd.paged_attention(*batch.args, out=out, lse=lse, workspace=ws, **{("softmax_scale" if k == "scale" else k): v for k, v in rules.items()})
    assert got[0] is out and got[1] is lse
    for t in got:                       # rows of no sequence
        assert bool((t[:batch.starts[0]] == 7).all()) and bool((t[batch.starts[-1]:] == 7).all())
    return got


SHAPES = [
    # lens, new, Hkv, G, page, bits
    ([1], [1], 1, 1, 16, 16),
    ([2, 1, 3], [1, 1, 1], 2, 4, 16, 16),
    ([0, 5, 0], [0, 5, 0], 1, 2, 16, 16),
    ([33, 64, 65, 1], [1, 1, 1, 1], 2, 8, 32, 8),
    ([127, 128, 129, 500], [1, 1, 1, 1], 8, 4, 64, 16),
    ([1000, 3], [1, 1], 1, 4, 256, 8),
    ([40, 41, 63], [40, 3, 17], 2, 4, 16, 16),
    ([300, 1037, 777], [20, 37, 33], 2, 4, 16, 16),
    ([300, 1037, 777], [20, 37, 33], 2, 4, 16, 8),
    ([700], [700], 1, 1, 128, 16),
    ([515, 129], [515, 129], 1, 8, 64, 16),
    ([515, 129], [500, 100], 1, 8, 64, 8),
    ([257, 1, 600, 90], [256, 1, 1, 90], 2, 2, 32, 16),
    ([2100, 30, 31], [100, 1, 0], 1, 4, 16, 16),
]


@pytest.mark.parametrize("lens,new,Hkv,G,page,bits", SHAPES)
def test_attention(ffd, lens, new, Hkv, G, page, bits):
    batch = R.Batch(lens, new, Hkv, G, page, bits, seed=len(lens) + page)
    R.check_attention(batch, _attend(ffd, batch), _p_error(batch))


RULES = [dict(softcap=20.0), dict(window=1), dict(window=50), dict(window=1 << 31 - 1), dict(slopes=True), dict(prefix=True), dict(window=33, prefix=True),
         dict(softcap=5.0, window=100, slopes=True, prefix=True), dict(scale=0.5)]


def _rules(batch, rule):
    rule = dict(rule)
    if rule.pop("slopes", False):
        H = batch.Hkv * batch.G
        rule["slopes"] = 2.0 ** (-8 * torch.arange(1, H + 1, device="cuda").float() / H)
    if rule.pop("prefix", False):
        rule["prefix_lens"] = R.int32([(37 * (b + 1)) % (L + 20) if b % 3 != 1 else 0 for b, L in enumerate(batch.lens)])
    if rule.get("window", 0) >= 1 << 30:
        rule["window"] = 2 ** 31 - 1
    return rule


def _for_reference(batch, rules):
    if "prefix_lens" in rules:
        return dict(rules, prefix_lens=[min(max(int(p), 0), L) for p, L in zip(rules["prefix_lens"], batch.lens)])
    return rules


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", RULES, ids=lambda r: "_".join(r))
@pytest.mark.parametrize("lens,new", [([300, 1, 90], [1, 1, 1]), ([300, 515, 90], [200, 37, 90]), ([20, 700], [3, 8])])
def test_rules(ffd, lens, new, rule, bits):
    batch = R.Batch(lens, new, 2, 4, 32, bits, seed=3, before=2, behind=3)
    rules = _rules(batch, rule)
    R.check_attention(batch, _attend(ffd, batch, **rules), _p_error(batch), **_for_reference(batch, rules))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("missing", [-1, 10 ** 9, -2 ** 31])
def test_pages_that_are_not_there(ffd, bits, missing):
    """Tokens of such pages are seen by nobody, also where a query has no other."""
    batch = R.Batch([40, 200, 333, 16], [40, 2, 64, 1], 2, 4, 16, bits, seed=5, holes=[(0, 0), (1, 3), (1, 12), (2, 20), (2, 19), (3, 0)], missing=missing)
    got = _attend(ffd, batch)
    R.check_attention(batch, got, _p_error(batch))
    assert bool((got[1][batch.starts[0]:batch.starts[0] + 16] == -math.inf).all())
    rules = dict(window=20, prefix_lens=R.int32([10, 100, 0, 16]))
    R.check_attention(batch, _attend(ffd, batch, **rules), _p_error(batch), **rules)


def test_lengths_out_of_range(ffd):
    """Fewer tokens than new ones: the first of those see nothing. More than the table holds: its end bounds what is seen.
    Negative lengths and starts outside the batch are clamped."""
    batch = R.Batch([3, 100, 64], [9, 5, 70], 1, 4, 16, seed=6, width=5)         # the second has 20 tokens more than the table
    got = _attend(ffd, batch)
    R.check_attention(batch, got, _p_error(batch))
    assert bool((got[1][:6] == -math.inf).all()) and bool((got[0][:6] == 0).all())
    batch.seq_lens = R.int32([-5, 100, 2 ** 31 - 1])
    batch.args = batch.args[:-1] + (batch.seq_lens,)
    out, lse = _attend(ffd, batch)
    assert bool((lse[:9] == -math.inf).all()) and bool((lse[14:].isfinite()).all())
    batch.q_start = R.int32([-7, 9, 14, 10 ** 9])
    out2, lse2 = ffd.paged_attention(*batch.args[:3], batch.q_start, batch.seq_lens)
    assert torch.equal(out2[9:14], out[9:14]) and bool((lse2[14:].isfinite()).all())


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("n,G", [(4, 4), (90, 4)])
def test_values_that_are_not_finite(ffd, value, n, G):
    """They reach the queries that see them, and no other."""
    L, at = 200, 150
    batch = R.Batch([L], [n], 2, G, 16, seed=7)
    clean = ffd.paged_attention(*batch.args)
    page = batch.table[0][at // 16]
    batch.cache[1][page, 1, at % 16, 5] = value
    out, lse = ffd.paged_attention(*batch.args)
    sees = torch.arange(L - n, L, device="cuda") >= at
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[:, G:, 5] = sees.view(-1, 1)
    if value == value:
        assert bool((out[hit] == value).all())
    else:
        assert bool(out[hit].isnan().all())
    assert bool(out[~hit].isfinite().all()) and torch.equal(lse, clean[1])
    assert bool(((out - clean[0]).abs()[~hit] <= 2.0 ** -7 * clean[0].abs()[~hit] + 2.0 ** -8).all())
    # beyond the length of a sequence, or before a window, it reaches nobody
    out, _ = ffd.paged_attention(*batch.args, window=20, prefix_lens=R.int32([at - 3]))
    sees = sees & (torch.arange(L - n, L, device="cuda") - at < 20)
    assert torch.equal(out[:, G:, 5].isfinite(), ~sees.view(-1, 1).expand(-1, G))


def test_keys_that_are_not_finite(ffd):
    """A NaN among the keys makes the rows that see it NaN, and no other; an infinite score likewise gives no number."""
    batch = R.Batch([100], [60], 1, 4, 16, seed=8)
    batch.cache[0][batch.table[0][70 // 16], 0, 70 % 16, 3] = math.nan
    out, lse = ffd.paged_attention(*batch.args)
    nan = torch.arange(40, 100, device="cuda") >= 70
    assert torch.equal(out.isnan().all(-1).all(-1), nan) and torch.equal(out.isnan().any(-1).any(-1), nan)
    assert torch.equal(lse.isnan().any(-1), nan)


def test_many_sequences(ffd):
    """More sequences than a wave has lanes, most of them short, some cut into runs."""
    lens = [(37 * b) % 200 for b in range(150)]
    new = [min(L, (b * 7) % 5) for b, L in enumerate(lens)]
    for b in (3, 64, 149):
        lens[b], new[b] = 3000 + b, 1
    new[70], lens[70] = 150, 150
    batch = R.Batch(lens, new, 1, 4, 16, seed=9)
    R.check_attention(batch, _attend(ffd, batch), P_BF16)
    again = _attend(ffd, batch)
    for x, y in zip(again, _attend(ffd, batch)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("new", [1, 16, 300])
def test_a_long_cache_is_cut(ffd, new):
    batch = R.Batch([5000], [new], 1, 4, 64, seed=10)
    R.check_attention(batch, _attend(ffd, batch), _p_error(batch))


def test_far_pages(ffd):
    """Pages beyond 2^32 bytes of their tensors."""
    num, Hkv, page = 9000, 8, 256           # 4.7 GB of keys
    cache = ffd.empty_paged(num, Hkv, page)
    entries = [num - 1, 0, num - 2]
    gen = torch.Generator("cuda").manual_seed(1)
    for x in cache:
        for e in entries:
            x[e] = torch.randn(Hkv, page, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    L, n = 700, 10
    table, q_start, lens = R.int32([entries]), R.int32([0, n]), R.int32([L])
    q, k, v = (torch.randn(n, Hkv, D, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    ffd.write_paged(None, k, v, cache, table, q_start, lens)
    near = tuple(x[entries].contiguous() for x in cache)
    assert torch.equal(near[0][2, :, L - n - 512:L - 512].transpose(0, 1), k) and torch.equal(near[1][2, :, L - n - 512:L - 512].transpose(0, 1), v)
    near_table = R.int32([[0, 1, 2]])
    got, want = ffd.paged_attention(q, cache, table, q_start, lens), ffd.paged_attention(q, near, near_table, q_start, lens)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    w = ffd.paged_attention_weights(q, cache, table, q_start, lens, got[1])
    assert torch.equal(w, ffd.paged_attention_weights(q, near, near_table, q_start, lens, got[1]))
    kept, _, _ = ffd.evict_paged(cache, table, R.int32([[num - 3]]), lens, w, 100, recent=10)
    for x in cache:
        rows = x[entries].transpose(1, 2).reshape(-1, Hkv, D)
        for h in range(Hkv):
            assert torch.equal(x[num - 3, h, :100], rows[kept[0, h].long(), h])


# ---- writing --------------------------------------------------------------------------------------------------

def _rope(rows, dims, seed=0):
    rates = 10000.0 ** (-torch.arange(dims // 2, dtype=torch.float64) / (dims // 2))
    angles = torch.arange(rows, dtype=torch.float64).unsqueeze(1) * rates
    return torch.cat([angles.cos(), angles.sin()], 1).float().cuda()


def _snapshot(cache):
    return [x.clone() for x in cache]


def _new_rows(batch, gen, layout):
    """(q, k, v) as slices of a projection, or each for itself."""
    T, Hq, Hkv = batch.T, batch.Hkv * batch.G, batch.Hkv
    if layout == "sliced":
        x = torch.randn(T, Hq + 2 * Hkv, D, generator=gen, device="cuda", dtype=torch.bfloat16)
        return x[:, :Hq], x[:, Hq:-Hkv], x[:, -Hkv:]
    if layout == "transposed":
        return tuple(torch.randn(h, T, D, generator=gen, device="cuda", dtype=torch.bfloat16).transpose(0, 1) for h in (Hq, Hkv, Hkv))
    return tuple(torch.randn(T, h, D, generator=gen, device="cuda", dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))


@pytest.mark.parametrize("layout", ["sliced", "transposed", "plain"])
@pytest.mark.parametrize("norm,dims,inter", [(True, 128, False), (False, 64, False), (True, 32, True), (True, 96, False), (False, 128, True), (True, 0, False),
                                             (False, 0, False), (False, 96, True), (True, 32, False)])
@pytest.mark.parametrize("lens,new,Hkv,G,page", [([5], [1], 1, 1, 16), ([40, 0, 33, 300], [7, 0, 33, 100], 2, 4, 16), ([100, 65], [1, 1], 8, 8, 32)])
def test_write(ffd, lens, new, Hkv, G, page, norm, dims, inter, layout):
    gen = torch.Generator("cuda").manual_seed(11)
    batch = R.Batch(lens, new, Hkv, G, page, seed=12, before=1, behind=2)
    q, k, v = _new_rows(batch, gen, layout)
    qw, kw = ((1 + 0.3 * torch.randn(D, generator=gen, device="cuda")).bfloat16() for _ in range(2)) if norm else (None, None)
    rope = _rope(400, dims) if dims else None
    before = _snapshot(batch.cache)
    out = torch.full((batch.T, Hkv * G, D), 7.0, dtype=torch.bfloat16, device="cuda")
    table = (batch.page_table, batch.q_start, batch.seq_lens)
    got = ffd.write_paged(q, k, v, batch.cache, *table, q_weight=qw, k_weight=kw, rope=rope, interleaved=inter, out=out)
    assert got is out
    assert bool((out[:1] == 7).all()) and bool((out[batch.starts[-1]:] == 7).all())
    places = torch.tensor([lens[b] - new[b] + t for b in range(batch.B) for t in range(new[b])], device="cuda")
    rows = slice(batch.starts[0], batch.starts[-1])
    true, bound = R.turned(q[rows], qw, rope, places, inter)
    assert bool(((out[rows].double() - true).abs() <= bound).all())
    true, bound = R.turned(k[rows], kw, rope, places, inter)
    b_of = torch.tensor([b for b in range(batch.B) for _ in range(new[b])], device="cuda")
    entries, at = batch.page_table[b_of, places // page].long(), places % page
    assert bool(((batch.cache[0][entries, :, at].double() - true).abs() <= bound).all())
    assert torch.equal(batch.cache[1][entries, :, at], v[rows])
    for x, y in zip(batch.cache, before):               # nothing else of the cache
        y[entries, :, at] = x[entries, :, at]
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    # in 8 bits: the codes of these keys
    eight = R.Batch(lens, new, Hkv, G, page, 8, seed=12, before=1, behind=2)
    before = _snapshot(eight.cache)
    again = ffd.write_paged(q, k, v, eight.cache, *table, q_weight=qw, k_weight=kw, rope=rope, interleaved=inter)
    assert torch.equal(again[rows], out[rows])
    want = *encode(batch.cache[0][entries, :, at]), *encode(v[rows].contiguous())
    for x, y, w in zip(eight.cache, before, want):
        assert torch.equal(x[entries, :, at], w)
        y[entries, :, at] = w
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_write_positions(ffd):
    """Positions of their own; outside of the table: NaN in the rotated dims, the others as they are."""
    batch = R.Batch([20, 9], [6, 9], 2, 2, 16, seed=13)
    gen = torch.Generator("cuda").manual_seed(13)
    q, k, v = _new_rows(batch, gen, "sliced")
    rope = _rope(50, 64)
    positions = [0, 49, 50, -1, 2 ** 31 - 1, 7] + list(range(9))
    got = ffd.write_paged(q, k, v, batch.cache, batch.page_table, batch.q_start, batch.seq_lens, rope=rope, positions=R.int32(positions))
    ok = torch.tensor([0 <= p < 50 for p in positions], device="cuda")
    at = torch.tensor([p if 0 <= p < 50 else 0 for p in positions], device="cuda")
    true, bound = R.turned(q, None, rope, at, False)
    assert bool(((got.double() - true).abs() <= bound)[ok].all())
    assert bool(got[~ok][..., :64].isnan().all()) and torch.equal(got[~ok][..., 64:], q[~ok][..., 64:])


@pytest.mark.parametrize("bits", [16, 8])
def test_write_to_places_that_are_not_there(ffd, bits):
    """A page that is not there, places before the first and behind the last token of the table: not written; queries come."""
    batch = R.Batch([40, 90, 3], [30, 20, 10], 2, 2, 16, bits, seed=14, holes=[(0, 1)], width=5)
    gen = torch.Generator("cuda").manual_seed(14)
    q, k, v = _new_rows(batch, gen, "plain")
    before = _snapshot(batch.cache)
    got = ffd.write_paged(q, k, v, batch.cache, batch.page_table, batch.q_start, batch.seq_lens)
    assert torch.equal(got, q)
    where = [(b, batch.lens[b] - batch.new[b] + t, batch.starts[b] + t) for b in range(3) for t in range(batch.new[b])]
    where = [(batch.table[b][j // 16], j % 16, row) for b, j, row in where if 0 <= j < 80 and batch.there(b, j)]
    e, at, row = (torch.tensor(x, device="cuda") for x in zip(*where))
    want = (k[row], v[row]) if bits == 16 else (*encode(k[row]), *encode(v[row]))
    for x, y, w in zip(batch.cache, before, want):
        y[e, :, at] = w
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_write_without_queries_or_tokens(ffd):
    batch = R.Batch([20], [4], 2, 2, 16, seed=15)
    gen = torch.Generator("cuda").manual_seed(15)
    _, k, v = _new_rows(batch, gen, "plain")
    table = (batch.page_table, batch.q_start, batch.seq_lens)
    kw = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    assert ffd.write_paged(None, k, v, batch.cache, *table, k_weight=kw) is None
    places = torch.arange(16, 20, device="cuda")
    true, bound = R.turned(k, kw, None, None, False)
    assert bool(((batch.cache[0][batch.page_table[0, places // 16].long(), :, places % 16].double() - true).abs() <= bound).all())
    none = torch.empty(0, 2, D, dtype=torch.bfloat16, device="cuda")
    before = _snapshot(batch.cache)
    empty = (batch.page_table, R.int32([0, 0]), batch.seq_lens)
    assert ffd.write_paged(none, none, none, batch.cache, *empty).shape == (0, 2, D)
    out, lse = ffd.paged_attention(none, batch.cache, *empty)
    assert out.shape == (0, 2, D) and lse.shape == (0, 2)
    for x, y in zip(batch.cache, before):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("value", [0.0, 2.0 ** -130, 3e38, math.inf, math.nan])
def test_write_extreme_keys(ffd, value):
    """A zero vector stays zero; huge ones overflow the mean of their squares and become zeros, as the formula says in 32 bits."""
    batch = R.Batch([1], [1], 1, 1, 16, seed=16)
    k = torch.full((1, 1, D), value, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    ffd.write_paged(None, k, k, batch.cache, batch.page_table, batch.q_start, batch.seq_lens, k_weight=w)
    page = batch.table[0][0]
    got = batch.cache[0][page, 0, 0].float()
    x = k[0, 0].float()
    want = x * (1 / (x.square().mean() + 1e-6).sqrt())
    assert bool(torch.isclose(got, want, rtol=2.0 ** -7, equal_nan=True).all())
    assert torch.equal(batch.cache[1][page, 0, 0].view(torch.int16), k[0, 0].view(torch.int16))


# ---- weights --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("last", [0, 1, 20])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rule", [dict(), dict(softcap=20.0, slopes=True), dict(window=40, prefix=True)], ids=lambda r: "_".join(r) or "plain")
@pytest.mark.parametrize("lens,new", [([300, 1, 0], [1, 1, 0]), ([300, 515, 90, 77], [200, 37, 90, 0]), ([3, 700], [8, 5])])
def test_weights(ffd, lens, new, rule, bits, last):
    batch = R.Batch(lens, new, 2, 4, 32, bits, seed=17, before=1, behind=1)
    rules = _rules(batch, rule)
    _, lse = ffd.paged_attention(*batch.args, **rules)
    gen = torch.Generator("cuda").manual_seed(17)
    previous = torch.rand(batch.B, 2, batch.cap, generator=gen, device="cuda")
    out = torch.full_like(previous, 5.0)
    got = ffd.paged_attention_weights(*batch.args, lse, last=last, previous=previous, out=out, **rules)
    assert got is out
    reference = _for_reference(batch, rules)
    R.check_weights(batch, got, lse, last, previous, torch.full_like(out, 5.0), **reference)
    fresh = ffd.paged_attention_weights(*batch.args, lse, last=last, **rules)
    R.check_weights(batch, fresh, lse, last, None, torch.zeros_like(out), **reference)
    in_place = previous.clone()
    ffd.paged_attention_weights(*batch.args, lse, last=last, previous=in_place, out=in_place, **rules)
    for b, L in enumerate(lens):
        assert torch.equal(in_place[b, :, :L], got[b, :, :L]) and torch.equal(in_place[b, :, L:], previous[b, :, L:])


def test_weights_of_pages_that_are_not_there(ffd):
    batch = R.Batch([40, 200], [40, 2], 2, 4, 16, seed=18, holes=[(0, 0), (1, 3), (1, 12)])
    _, lse = ffd.paged_attention(*batch.args)
    got = ffd.paged_attention_weights(*batch.args, lse)
    R.check_weights(batch, got, lse)
    assert bool((got[0, :, :16] == 0).all()) and bool((got[1, :, 48:64] == 0).all())


def test_weights_of_many_sequences_and_none(ffd):
    lens = [(37 * b) % 200 for b in range(150)]
    batch = R.Batch(lens, [min(1, L) for L in lens], 1, 2, 16, seed=19)
    _, lse = ffd.paged_attention(*batch.args)
    R.check_weights(batch, ffd.paged_attention_weights(*batch.args, lse), lse)
    none = torch.empty(0, 2, D, dtype=torch.bfloat16, device="cuda")
    previous = torch.rand(150, 1, batch.cap, device="cuda")
    got = ffd.paged_attention_weights(none, batch.cache, batch.page_table, R.int32([0] * 151), batch.seq_lens, none.new_empty((0, 2), dtype=torch.float32), previous=previous)
    for b, L in enumerate(lens):
        assert torch.equal(got[b, :, :L], previous[b, :, :L]) and bool((got[b, :, L:] == 0).all())


# ---- eviction -------------------------------------------------------------------------------------------------

def _weights(kind, shape, gen):
    w = torch.rand(shape, generator=gen, device="cuda")
    if kind == "ties":
        return torch.round(w * 4) / 4
    if kind == "equal":
        return torch.full_like(w, 0.25)
    if kind == "zeros":
        return torch.where(w < 0.5, 0.0, -0.0)
    if kind == "mixed":
        w = torch.randn(shape, generator=gen, device="cuda") * 10.0 ** torch.randint(-30, 30, shape, generator=gen, device="cuda")
        w = torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.02, math.inf, w)
        w = torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.02, -math.inf, w)
        return torch.where(torch.rand(shape, generator=gen, device="cuda") < 0.02, math.nan, w)
    return w


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "zeros", "mixed"])
@pytest.mark.parametrize("lens,budget,recent,holes", [
    ([1], 1, 0, []), ([40, 0, 17], 20, 5, []), ([300, 301, 15], 64, 64, []), ([5000, 4096, 4097], 1000, 10, []), ([90, 200], 50, 20, [(0, 1), (1, 12)]),
    ([200], 500, 0, []), ([1000, 30], 1, 1, [(1, 0), (1, 1)]),
])
def test_evict(ffd, lens, budget, recent, holes, kind, bits):
    page, Hkv = 16, 2
    extra = -(-budget // page)
    batch = R.Batch(lens, [0] * len(lens), Hkv, 1, page, bits, seed=20, holes=holes, spare=extra * len(lens) + 2)
    gen = torch.Generator("cuda").manual_seed(20)
    weights = _weights(kind, (batch.B, Hkv, batch.cap), gen)
    new_table = R.int32([[batch.free[b * extra + i] for i in range(extra)] + [-1] for b in range(batch.B)])
    before = _snapshot(batch.cache)
    new_weights = torch.full((batch.B, Hkv, (extra + 1) * page), 9.0, device="cuda")
    kept, new_lens, got_weights = ffd.evict_paged(batch.cache, batch.page_table, new_table, batch.seq_lens, weights, budget, recent=recent, new_weights=new_weights)
    assert got_weights is new_weights
    want = R.evicted(batch, weights, budget, recent)
    for b in range(batch.B):
        n = len(want[b][0])
        assert int(new_lens[b]) == n
        for h in range(Hkv):
            assert kept[b, h].tolist() == want[b][h] + [-1] * (budget - n)
            if n == 0:
                continue
            j, r = torch.tensor(want[b][h], device="cuda"), torch.arange(n, device="cuda")
            src, dst = batch.page_table[b, j // page].long(), new_table[b, r // page].long()
            assert torch.equal(new_weights[b, h, :n].view(torch.int32), weights[b, h, j].view(torch.int32)) and bool((new_weights[b, h, n:] == 9).all())
            for x, y in zip(batch.cache, before):
                y[dst, h, r % page] = y[src, h, j % page]
    for x, y in zip(batch.cache, before):               # all of the cache: nothing else was written
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_evict_without_some_new_pages(ffd):
    """Rows whose new page is not there are not copied; the list says all the same what was kept."""
    batch = R.Batch([100], [0], 1, 1, 16, seed=21, spare=4)
    weights = torch.rand(1, 1, batch.cap, device="cuda")
    before = _snapshot(batch.cache)
    kept, new_lens, _ = ffd.evict_paged(batch.cache, batch.page_table, R.int32([[batch.free[0], 10 ** 6, batch.free[1]]]), batch.seq_lens, weights, 40)
    assert int(new_lens[0]) == 40 and kept[0, 0].tolist() == R.evicted(batch, weights, 40, 0)[0][0]
    for x, y in zip(batch.cache, before):
        for r in list(range(16)) + list(range(32, 40)):
            j = int(kept[0, 0, r])
            y[batch.free[0 if r < 16 else 1], 0, r % 16] = y[batch.table[0][j // 16], 0, j % 16]
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


# ---- together -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 8])
def test_a_run_of_them(ffd, bits):
    """Prompts in chunks, decoding, weights, an eviction and more decoding, as a serving program runs them; each step checked."""
    B, Hkv, G, page, budget = 3, 2, 4, 16, 48
    gen = torch.Generator("cuda").manual_seed(22)
    batch = R.Batch([0] * B, [0] * B, Hkv, G, page, bits, seed=22, spare=60, width=10)
    free = list(batch.free)
    rope = _rope(300, 128)
    qw = (1 + 0.1 * torch.randn(D, generator=gen, device="cuda")).bfloat16()
    text = [0] * B                          # tokens of the text so far: the rotation's positions
    weights = torch.zeros(B, Hkv, batch.cap, device="cuda")

    def step(new):
        nonlocal weights
        batch.new, batch.T = new, sum(new)
        batch.lens = [L + n for L, n in zip(batch.lens, new)]
        batch.starts = [sum(new[:b]) for b in range(B + 1)]
        for b in range(B):
            for i in range(-(-batch.lens[b] // page)):
                if batch.table[b][i] < 0:
                    batch.table[b][i] = free.pop()
        batch.page_table, batch.q_start, batch.seq_lens = R.int32(batch.table), R.int32(batch.starts), R.int32(batch.lens)
        q, k, v = _new_rows(batch, gen, "sliced")
        positions = [text[b] + t for b in range(B) for t in range(new[b])]
        table = (batch.page_table, batch.q_start, batch.seq_lens)
        batch.q = ffd.write_paged(q, k, v, batch.cache, *table, q_weight=qw, k_weight=qw, rope=rope, positions=R.int32(positions))
        true, bound = R.turned(q, qw, rope, torch.tensor(positions, device="cuda"), False)
        assert bool(((batch.q.double() - true).abs() <= bound).all())
        out, lse = ffd.paged_attention(batch.q, batch.cache, *table)
        R.check_attention(batch, (out, lse), P_BF16)
        old = weights.clone()
        ffd.paged_attention_weights(batch.q, batch.cache, *table, lse, last=16, previous=weights, out=weights)
        R.check_weights(batch, weights, lse, 16, old, old)
        for b in range(B):
            text[b] += new[b]

    step([50, 7, 33])
    step([40, 60, 1])
    for _ in range(3):
        step([1, 1, 1])
    extra = budget // page
    new_table = [[free.pop() for _ in range(extra)] + [-1] * (10 - extra) for _ in range(B)]
    want = R.evicted(batch, weights, budget, 8)
    kept, new_lens, weights = ffd.evict_paged(batch.cache, batch.page_table, R.int32(new_table), batch.seq_lens, weights, budget, recent=8)
    assert [[x[x >= 0].tolist() for x in row] for row in kept.cpu()] == want
    for row in batch.table:
        free.extend(e for e in row if e >= 0)
    batch.table, batch.lens = new_table, new_lens.tolist()
    for _ in range(3):
        step([1, 2, 1])


def test_captured_together(ffd):
    """Write, attention and weights of a decode step in a graph, replayed as the sequences grow, beside eager work."""
    B, Hkv, G, page = 4, 2, 4, 16
    batch = R.Batch([30, 100, 1, 65], [1] * B, Hkv, G, page, seed=23, spare=40, width=12)
    free = list(batch.free)
    for b in range(B):
        for i in range(12):
            if batch.table[b][i] < 0 and free:
                batch.table[b][i] = free.pop()
    batch.page_table.copy_(R.int32(batch.table))
    gen = torch.Generator("cuda").manual_seed(23)
    q, k, v = (x.contiguous() for x in _new_rows(batch, gen, "plain"))
    q_out, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(B, Hkv * G, device="cuda")
    weights = torch.zeros(B, Hkv, batch.cap, device="cuda")
    rope = _rope(200, 128)
    ws = ffd.new_paged_workspace(B, B, Hkv * G, Hkv)
    table = (batch.page_table, batch.q_start, batch.seq_lens)

    def run():
        ffd.write_paged(q, k, v, batch.cache, *table, rope=rope, out=q_out)
        ffd.paged_attention(q_out, batch.cache, *table, workspace=ws, out=out, lse=lse)
        ffd.paged_attention_weights(q_out, batch.cache, *table, lse, previous=weights, out=weights)

    start = weights.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    cache0 = _snapshot(batch.cache)
    for turn in range(4):
        lens = batch.seq_lens.clone()
        weights.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (q_out, out, lse, weights, *batch.cache)]
        weights.copy_(start)
        for x, y in zip(batch.cache, cache0):
            x.copy_(y)
        run()
        for x, y in zip(got, (q_out, out, lse, weights, *batch.cache)):
            assert torch.equal(x.view(torch.uint8), y.contiguous().view(torch.uint8)), turn
        batch.lens = lens.tolist()
        batch.q = q_out
        R.check_attention(batch, (out, lse), P_SPLIT)
        start = weights.clone()
        cache0 = _snapshot(batch.cache)
        batch.seq_lens += 1                             # the graph reads the new lengths
        for x in (q, k, v):
            x.normal_(generator=gen)


def test_two_streams(ffd):
    """Calls at once on streams of their own, with workspaces of their own."""
    batches = [R.Batch([3000 + i], [1 + 40 * i], 2, 4, 64, seed=24 + i) for i in range(3)]
    want = [ffd.paged_attention(*b.args) for b in batches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    spaces = [ffd.new_paged_workspace(b.B, b.T, 8, 2) for b in batches]
    torch.cuda.synchronize()
    got = [[] for _ in batches]
    for _ in range(5):
        for i, (b, s) in enumerate(zip(batches, streams)):
            with torch.cuda.stream(s):
                got[i].append(ffd.paged_attention(*b.args, workspace=spaces[i]))
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        for g in got[i]:
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


@pytest.mark.parametrize("B,n,cap", [(1, 1, 128), (3, 5, 256), (40, 3, 256), (200, 3, 256), (200, 3, 128), (2, 100, 272), (3, 5, 512), (3, 5, 528),
                                     (150, 1, 1024), (150, 2, 1040), (20, 1, 1024)])
def test_short_capacities(ffd, B, n, cap):
    """Capacities around those at which no tile is cut, with few and with more tiles than workgroups."""
    batch = R.Batch([cap - (7 * b) % 90 for b in range(B)], [n] * B, 4, 4, 16, seed=42, width=cap // 16)
    R.check_attention(batch, _attend(ffd, batch), _p_error(batch))


@pytest.mark.parametrize("T", [5, 700])
def test_batches_without_rows(ffd, T):
    """Rows that belong to no sequence, and sequences without any: nothing is written."""
    batch = R.Batch([40, 0, 300], [0, 0, 0], 2, 4, 16, seed=44, behind=T, width=2000)
    _attend(ffd, batch)                         # looks at the rows around
    q, k, v = (torch.randn(T, h, D, device="cuda", dtype=torch.bfloat16) for h in (8, 2, 2))
    before, out = _snapshot(batch.cache), torch.full((T, 8, D), 3.0, device="cuda", dtype=torch.bfloat16)
    ffd.write_paged(q, k, v, batch.cache, *batch.args[2:], out=out)
    assert bool((out == 3).all())
    for x, y in zip(batch.cache, before):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    previous = torch.rand(3, 2, batch.cap, device="cuda")
    got = ffd.paged_attention_weights(q, *batch.args[1:], torch.zeros(T, 8, device="cuda"), previous=previous)
    for b, L in enumerate(batch.lens):
        assert torch.equal(got[b, :, :L], previous[b, :, :L]) and bool((got[b, :, L:] == 0).all())
