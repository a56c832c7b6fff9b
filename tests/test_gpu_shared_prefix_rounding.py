"""Rounding of the probabilities in the attention over a shared prefix: on every path as fine as two bf16 parts, held to
the half step of the very output value (not to the largest that a relative half step can be)."""
import math

import pytest
import torch

from tests.kv8_reference import D, P_SPLIT, attention, encode, random_cache, values

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cap(n):
    return max(64, -(-n // 64) * 64)


def _large(rows, Hkv, tokens):
    """A capacity of at least `tokens` for which `rows` query rows are no little work: they are taken by the kernel that
    stages tokens, in tiles of 64, 128 or 256."""
    work = 129 * 1024 * torch.cuda.get_device_properties(0).multi_processor_count
    return _cap(max(tokens, -(-work // (rows * Hkv))))


def _padded(cache, cap):
    """The cache in capacity cap, NaN (codes: 127) behind its tokens."""
    P = cache[0].shape[2]
    whole = []
    for t in cache:
        big = torch.full((*t.shape[:2], cap, *t.shape[3:]), 127 if t.dtype == torch.int8 else math.nan, dtype=t.dtype, device="cuda")
        big[:, :, :P] = t
        whole.append(big)
    return tuple(whole)


def check_rounded(out, ref, tokens, p_error, finite=None):
    """`out` is the bf16 next to the 64-bit value, or to one that is off by the error of the scores, of the sums and of the
    probabilities (e and p_error of check_attention, doubled by numerator and denominator): out lies between the two
    ends of that interval, both rounded to bf16 once."""
    want, _, mass, reach = ref
    e = (136 * reach + tokens + 4) * 2.0 ** -24 + 2.0 ** -22
    err = (2 * e + p_error).unsqueeze(-1) * mass
    o, low, high = out.cpu(), (want - err).bfloat16(), (want + err).bfloat16()
    bad = ~((o >= low) & (o <= high))
    if finite is not None:
        bad &= finite
    step = (o.double() - want).abs() / (want.abs() * 2.0 ** -8 + 1e-30)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, by up to {step[bad].max().item():.3f} half steps, at {bad.nonzero()[:4].tolist()}"


# (B, G, large capacity): tiles of 16 and 32 rows, several of 32, and staged ones of 64, 128, 256 and two of 256 rows
SHAPES = [(3, 4, False), (8, 4, False), (25, 4, False), (33, 1, True), (8, 8, True), (70, 1, True), (16, 8, True), (50, 4, True),
          (32, 8, True), (70, 8, True)]


@pytest.mark.parametrize("B,G,large", SHAPES)
@pytest.mark.parametrize("bits,own_bits", [(16, 16), (8, 8), (8, 16)])
def test_equal_scores(B, G, large, bits, own_bits):
    """One token of 32 has a score s above all others, which are equal: their probability e^-s is rounded alike, so that
    what the rounding loses is not averaged out. s differs from row to row, the values are the same for all tokens but
    those above."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B * G + bits)
    P = 1500
    k, v = torch.zeros(1, 1, P, D, dtype=torch.bfloat16, device="cuda"), _normal(gen, 1, 1, 1, D).repeat(1, 1, P, 1)
    k[:, :, ::32, 0] = 1
    v[:, :, ::32] = 0
    prefix = (k, v) if bits == 16 else (*encode(k), *encode(v))
    q = torch.zeros(B, G, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = torch.linspace(0.3, 6, B * G).view(B, G).bfloat16()
    cache, lens = random_cache(gen, B, 1, 64, own_bits), [b % 2 for b in range(B)]
    ref = attention(q, [(*values(prefix), [P] * B), (*values(cache), lens)], 1.0)
    prefix = _padded(prefix, _large(B * G, 1, P) if large else _cap(P))
    print(f"case equal B={B} G={G} large={large} bits {bits} {own_bits}", flush=True)
    for splits in (0, 1):
        out, _ = ffd.shared_prefix_decode_attention(q, prefix, _int32([P] * B), cache, _int32(lens), softmax_scale=1.0, num_splits=splits)
        check_rounded(out, ref, P + 1, P_SPLIT)


@pytest.mark.parametrize("B,G,large", SHAPES)
@pytest.mark.parametrize("bits", [16, 8])
def test_a_dominant_token_behind_the_first_tile(B, G, large, bits):
    """A token that arrives late, its score up to e^5.5 above those of a few before it, has most of the weight: also
    where the reference of the exponents still is the earlier maximum."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B * G + bits)
    P, at = 1500, 1111
    k, v = torch.zeros(1, 1, P, D, dtype=torch.bfloat16, device="cuda"), _normal(gen, 1, 1, P, D)
    k[..., 1] = -20
    k[:, :, :512:32, 1] = 0
    k[0, 0, at, 1], k[0, 0, at, 0] = 0, 1
    prefix = (k, v) if bits == 16 else (*encode(k), *encode(v))
    q = torch.zeros(B, G, D, dtype=torch.bfloat16, device="cuda")
    q[..., 1] = 1
    q[..., 0] = torch.linspace(3, 5.5, B * G).view(B, G).bfloat16()
    cache, lens = random_cache(gen, B, 1, 64, 16), [0] * B
    ref = attention(q, [(*values(prefix), [P] * B), (*values(cache), lens)], 1.0)
    prefix = _padded(prefix, _large(B * G, 1, P) if large else _cap(P))
    print(f"case dominant B={B} G={G} large={large} bits {bits}", flush=True)
    for splits in (1, 0):
        out, _ = ffd.shared_prefix_decode_attention(q, prefix, _int32([P] * B), cache, _int32(lens), softmax_scale=1.0, num_splits=splits)
        check_rounded(out, ref, P, P_SPLIT)


@pytest.mark.parametrize("B,G,large", SHAPES)
@pytest.mark.parametrize("bits,own_bits", [(16, 16), (16, 8), (8, 8), (8, 16)])
def test_random_scores(B, G, large, bits, own_bits):
    """Peaked and flat rows over parts of the prefix and own tokens."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B + G + bits)
    P, lens = 1000, [(19 * b) % 60 for b in range(B)]
    prefix_lens = [P - 11 * b for b in range(B)]
    q = _normal(gen, B, 2 * G, D)
    q[::2] *= 3
    prefix, cache = random_cache(gen, 1, 2, P, bits), random_cache(gen, B, 2, 64, own_bits)
    ref = attention(q, [(*values(prefix), prefix_lens), (*values(cache), lens)])
    prefix = _padded(prefix, _large(B * G, 2, P) if large else _cap(P))
    print(f"case random B={B} G={G} large={large} bits {bits} {own_bits}", flush=True)
    out, _ = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens))
    check_rounded(out, ref, P + 60, P_SPLIT)


@pytest.mark.parametrize("B,G,large", SHAPES)
def test_infinities_cost_the_others_no_precision(B, G, large):
    """An infinite value that most sequences see, a NaN value, and a sequence whose query is NaN: the other dims and rows are
    rounded as ever. Scores as in test_equal_scores, where a coarser rounding would not be averaged out."""
    from paper_2609_00097_amd import ffd
    gen = _gen(B * G)
    P = 1500
    k, v = torch.zeros(1, 1, P, D, dtype=torch.bfloat16, device="cuda"), _normal(gen, 1, 1, 1, D).repeat(1, 1, P, 1)
    k[:, :, ::32, 0] = 1
    v[:, :, ::32] = 0
    q = torch.zeros(B, G, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = torch.linspace(0.3, 6, B * G).view(B, G).bfloat16()
    cache, lens = random_cache(gen, B, 1, 64, 16), [0] * B
    prefix_lens = [P if b % 3 else 700 for b in range(B)]
    ref = attention(q, [(*values((k, v)), prefix_lens), (*values(cache), lens)], 1.0)
    special = [(5, 3, math.inf), (333, 127, -math.inf), (400, 64, math.nan), (900, 30, math.inf), (1499, 31, math.nan)]
    finite = torch.ones(B, G, D, dtype=torch.bool)
    for t, d, x in special:
        v[0, 0, t, d] = x
        finite[torch.tensor(prefix_lens) > t, :, d] = False
    q[B - 1, G - 1, 7] = math.nan
    finite[B - 1, G - 1] = False
    prefix = _padded((k, v), _large(B * G, 1, P) if large else _cap(P))
    print(f"case infinities B={B} G={G} large={large}", flush=True)
    out, _ = ffd.shared_prefix_decode_attention(q, prefix, _int32(prefix_lens), cache, _int32(lens), softmax_scale=1.0)
    assert torch.equal(out.isfinite().cpu(), finite)
    check_rounded(out, ref, P, P_SPLIT, finite)
