"""Plain 64-bit forms of the 8-bit cache and of attention over a shared prefix, and the error bounds that the
tests hold the kernels to."""
import math

import torch

D = 128
HALF_STEP = torch.finfo(torch.bfloat16).eps / 2          # of a rounding to bf16, relative


def encode(x):
    """(codes int8, absmax bf16) of bf16 vectors [..., 128]."""
    M = x.double().abs().amax(-1)
    safe = torch.where((M > 0) & M.isfinite(), M, torch.ones_like(M)).unsqueeze(-1)
    n = torch.where(M.isfinite().unsqueeze(-1), torch.round(127 * x.double() / safe), 0.0)
    return n.to(torch.int8), torch.where(M.isfinite(), M, math.nan).bfloat16()


def decode(codes, absmax):
    """float64 values of an 8-bit tensor."""
    return codes.double() * absmax.double().unsqueeze(-1) / 127


def values(cache):
    """float64 (k, v) of a cache: bf16 (k, v) or 8-bit."""
    if len(cache) == 2:
        return cache[0].double(), cache[1].double()
    return decode(cache[0], cache[1]), decode(cache[2], cache[3])


def random_cache(gen, B, Hkv, L, bits=8):
    """N(0, 1) keys and values in a cache of the given form, on the GPU."""
    k, v = (torch.randn(B, Hkv, L, D, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    return (k, v) if bits == 16 else (*encode(k), *encode(v))


def attention(q, parts, scale=None):
    """softmax(scale q K^T) V over parts = [(k [B or 1, Hkv, L, 128], v, lens [B]), ..] in float64; tokens behind a length
    do not exist. Returns out, lse and, per row, the sum of p |v| (the scale of an error in the probabilities) and the
    largest scale * sum_d |q_d k_d| (that of an error in the scores)."""
    B, Hq, _ = q.shape
    scale = scale or 1 / math.sqrt(D)
    out, mass = torch.zeros(B, Hq, D, dtype=torch.float64), torch.zeros(B, Hq, D, dtype=torch.float64)
    lse, reach = torch.full((B, Hq), -math.inf, dtype=torch.float64), torch.zeros(B, Hq, dtype=torch.float64)
    Hkv = parts[0][0].shape[1]
    G = Hq // Hkv
    for b in range(B):
        for h in range(Hkv):
            k = torch.cat([p[0][b % p[0].shape[0], h, :int(p[2][b])] for p in parts])
            v = torch.cat([p[1][b % p[1].shape[0], h, :int(p[2][b])] for p in parts])
            if len(k) == 0:
                continue
            rows = slice(h * G, (h + 1) * G)
            qr = q[b, rows].double()
            z = scale * (qr @ k.T)
            p = torch.softmax(z, -1)
            lse[b, rows] = torch.logsumexp(z, -1).cpu()
            out[b, rows], mass[b, rows] = (p @ v).cpu(), (p @ v.abs()).cpu()
            reach[b, rows] = scale * (qr.abs() @ k.abs().T).amax(-1).cpu()
    return out, lse, mass, reach


def check_attention(got, ref, tokens, p_error):
    """out and lse against the 64-bit ones. A score is a sum of 128 products in 32 bits, scaled, with the maximum
    subtracted in powers of two: (128 + 8) roundings of at most its reach. e^x has 2^-22, sums over `tokens` tokens
    as many roundings, p_error is that of a probability (2^-8: rounded to bf16, 2^-16: to two of them). An error
    e of the probabilities moves a row by at most 2 e * sum p |v| (numerator and denominator)."""
    out, lse, mass, reach = ref
    e = (136 * reach + tokens + 4) * 2.0 ** -24 + 2.0 ** -22
    o, l = got[0].double().cpu(), got[1].double().cpu()
    bound = HALF_STEP * out.abs() + (2 * e + p_error).unsqueeze(-1) * mass * (1 + HALF_STEP) + 2.0 ** -133
    assert o.shape == out.shape
    bad = ~((o - out).abs() <= bound)
    assert not bad.any(), f"out: {int(bad.sum())} of {bad.numel()} off, worst {((o - out).abs() / bound)[bad][:4].tolist()} at {bad.nonzero()[:4].tolist()}"
    none = lse == -math.inf
    assert torch.equal(l == -math.inf, none) and bool((o[none] == 0).all())
    bad = ~((l - lse).abs() <= e + 2.0 ** -22 * lse.abs()) & ~none
    assert not bad.any(), f"lse: {(l - lse)[bad][:4].tolist()} at {bad.nonzero()[:4].tolist()}"


P_SPLIT, P_BF16 = 2.0 ** -16, 2.0 ** -8
