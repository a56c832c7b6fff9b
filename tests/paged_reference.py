"""Plain 64-bit forms of the operators over paged caches, and the error bounds that the tests hold the kernels to."""
import math
import random

import torch

from .kv8_reference import D, HALF_STEP, decode, encode

EPS = 1e-6


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Batch:
    """A paged cache with its sequences, on the GPU: lens[b] tokens of which new[b] are new, in pages handed out in no order.
    Everything in the pages that belongs to no token is NaN, or an absmax of NaN; `holes` are page numbers (sequence, page)
    that are not there; rows of the batch begin at `before` and end `behind` rows before T."""

    def __init__(self, lens, new, Hkv, G, page=16, bits=16, seed=0, holes=(), before=0, behind=0, spare=3, width=None, missing=-1):
        rng, gen = random.Random(seed), torch.Generator("cuda").manual_seed(seed)
        self.lens, self.new, self.Hkv, self.G, self.page, self.bits, self.holes = lens, new, Hkv, G, page, bits, set(holes)
        self.B, self.T, self.before = len(lens), before + sum(new) + behind, before
        self.starts = [before + sum(new[:b]) for b in range(self.B + 1)]
        counts = [-(-L // page) for L in lens]
        self.width = width or max(counts + [1]) + 1
        self.cap = self.width * page
        self.num_pages = sum(counts) + spare
        order = rng.sample(range(self.num_pages), sum(counts))
        self.free = [i for i in range(self.num_pages) if i not in set(order)]
        self.table = [[missing] * self.width for _ in range(self.B)]
        for b in range(self.B):
            for i in range(counts[b]):
                e = order.pop()
                if (b, i) not in self.holes and i < self.width:
                    self.table[b][i] = e
        values = [torch.randn(self.num_pages, Hkv, page, D, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
        belongs = torch.zeros(self.num_pages, page, dtype=torch.bool)
        for b in range(self.B):
            for j in range(lens[b]):
                if j < self.cap and self.there(b, j):
                    belongs[self.table[b][j // page], j % page] = True
        dead = ~belongs.cuda().view(self.num_pages, 1, page).expand(-1, Hkv, -1)
        if bits == 8:
            self.cache = tuple(t for x in values for t in encode(x))
            self.cache[1][dead] = self.cache[3][dead] = math.nan
        else:
            self.cache = tuple(values)
            self.cache[0][dead] = self.cache[1][dead] = math.nan
        self.q = torch.randn(self.T, Hkv * G, D, generator=gen, device="cuda", dtype=torch.bfloat16)
        self.page_table, self.q_start, self.seq_lens = int32(self.table), int32(self.starts), int32(self.lens)
        self.args = (self.q, self.cache, self.page_table, self.q_start, self.seq_lens)

    def there(self, b, j):
        return 0 <= self.table[b][j // self.page] < self.num_pages

    def rows(self, which, b, h):
        """float64 [min(len, cap), 128] of keys (0) or values (1); tokens of pages that are not there are zeros."""
        n = min(self.lens[b], self.cap)
        pages = self.page_table[b, :-(-n // self.page)].long()
        ok = (pages >= 0) & (pages < self.num_pages)
        at = torch.where(ok, pages, 0)
        if self.bits == 8:
            x = decode(self.cache[2 * which][at, h], self.cache[2 * which + 1][at, h])
        else:
            x = self.cache[which][at, h].double()
        x = torch.where(ok.view(-1, 1, 1), x, 0)
        return x.flatten(0, 1)[:n]

    def seen(self, b, window=0, prefix=0):
        """bool [new, min(len, cap)]"""
        n, L = self.new[b], self.lens[b]
        i = torch.arange(L - n, L, device="cuda").view(-1, 1)
        j = torch.arange(min(L, self.cap), device="cuda").view(1, -1)
        s = (j <= i) & ((i - j < window) if window else (j == j))
        s = s | (j < prefix)
        for x in range(-(-s.shape[1] // self.page)):
            if not self.there(b, x * self.page):
                s[:, x * self.page:(x + 1) * self.page] = False
        return s

    def scores(self, b, h, scale=None, softcap=0.0, window=0, slopes=None, prefix_lens=None):
        """float64 z [new, G, tokens] with minus infinity where a token is not seen, and the largest sum of |q_d k_d| scale and
        the largest |slope (i - j)| of what is seen."""
        n, L, G = self.new[b], self.lens[b], self.G
        scale = scale or 1 / math.sqrt(D)
        q = self.q[self.starts[b]:self.starts[b + 1], h * G:(h + 1) * G].double()
        k = self.rows(0, b, h)
        seen = self.seen(b, window, int(prefix_lens[b]) if prefix_lens is not None else 0)
        z = (q.reshape(n * G, D) @ k.T).view(n, G, k.shape[0]) * scale
        reach = (q.abs().reshape(n * G, D) @ k.abs().T).view(n, G, k.shape[0]) * scale
        far = torch.zeros_like(z)
        if softcap:
            z = softcap * torch.tanh(z / softcap)
        if slopes is not None:
            i, j = torch.arange(L - n, L, device="cuda").view(-1, 1, 1), torch.arange(k.shape[0], device="cuda").view(1, 1, -1)
            far = slopes[h * G:(h + 1) * G].double().view(1, -1, 1) * (i - j).abs()
            z = z - far
        seen = seen.unsqueeze(1)
        worst = torch.where(seen, reach, 0).nan_to_num(0, 0, 0).amax(-1) if z.shape[-1] else torch.zeros(n, G, device="cuda")
        far = torch.where(seen, far, 0).amax(-1) if z.shape[-1] else torch.zeros(n, G, device="cuda")
        return torch.where(seen, z, -math.inf), worst, far


def score_error(worst, far, softcap=0.0):
    """How far a score may be off: 128 products summed in 32 bits, scaled, in powers of two, the reference subtracted: (128 + 8)
    roundings of at most the sum of the products' sizes. Distances: the slope in powers of two (two roundings) and the sum. With
    a cap tanh(x) = 1 - 2 / (1 + e^2x): the exponential and the quotient are 2^-21 off together, of which tanh gets at most a
    half, and two roundings."""
    return 136 * 2.0 ** -24 * worst + 2.0 ** -21 * far + (2.0 ** -20 * softcap if softcap else 0.0)


def check_attention(batch, got, p_error, **rules):
    """out and lse of a call against the 64-bit ones; rows of no sequence have to be as `out`, `lse` were filled. An error e of the
    probabilities moves a row by at most 2 e * sum p |v| (numerator and denominator); e^x has 2^-22 and sums over N tokens N roundings."""
    out, lse = got
    softcap = rules.get("softcap", 0.0)
    for b in range(batch.B):
        rows = slice(batch.starts[b], batch.starts[b + 1])
        for h in range(batch.Hkv):
            heads = slice(h * batch.G, (h + 1) * batch.G)
            z, worst, far = batch.scores(b, h, **rules)
            v = batch.rows(1, b, h)
            none = (z == -math.inf).all(-1)
            true_lse = torch.logsumexp(z, -1) if z.shape[-1] else torch.full_like(none, -math.inf, dtype=torch.float64)
            p = torch.exp(z - torch.where(none, 0, true_lse).unsqueeze(-1))
            true = (p.flatten(0, 1) @ v).view(*z.shape[:2], D)
            mass = (p.flatten(0, 1) @ v.abs()).view(*z.shape[:2], D)
            e = score_error(worst, far, softcap) + (z.shape[-1] + 4) * 2.0 ** -24 + 2.0 ** -22
            bound = HALF_STEP * true.abs() + (2 * e + p_error).unsqueeze(-1) * mass * (1 + HALF_STEP) + 2.0 ** -133
            o, l = out[rows, heads].double(), lse[rows, heads].double()
            bad = ~((o - true).abs() <= bound)
            assert not bad.any(), (f"sequence {b}, KV head {h}: {int(bad.sum())} of {bad.numel()} off, worst "
                                   f"{((o - true).abs() / bound)[bad][:4].tolist()} at {bad.nonzero()[:4].tolist()}")
            assert torch.equal(l == -math.inf, none) and bool((o[none] == 0).all()), (b, h)
            bad = ~((l - true_lse).abs() <= e + 2.0 ** -22 * true_lse.abs()) & ~none
            assert not bad.any(), f"sequence {b}, KV head {h}: lse off by {(l - true_lse)[bad][:4].tolist()} at {bad.nonzero()[:4].tolist()}"


def check_weights(batch, got, lse, last=0, previous=None, before=None, **rules):
    """weights against the 64-bit sums with the given lse; entries behind a length have to be as `before` was."""
    for b in range(batch.B):
        n, L = batch.new[b], batch.lens[b]
        for h in range(batch.Hkv):
            z, worst, far = batch.scores(b, h, **rules)
            l = lse[batch.starts[b]:batch.starts[b + 1], h * batch.G:(h + 1) * batch.G].double().unsqueeze(-1)
            p = torch.where(z == -math.inf, 0, torch.exp(z - l))
            # in powers of two: the score's and lse's roundings, and the difference's
            e = (score_error(worst, far, rules.get("softcap", 0.0)).unsqueeze(-1) + 2.0 ** -22 * (l.abs() + 1)).nan_to_num(0, 0, 0)
            if last:
                p, e = p[max(0, n - last):], e[max(0, n - last):]
            w = p.sum((0, 1))
            bound = (p * e).sum((0, 1)) + (p.shape[0] * batch.G + 2) * 2.0 ** -24 * w + 2.0 ** -22 * w + 2.0 ** -126
            N = w.numel()
            if previous is not None:
                old = torch.where(torch.arange(N, device="cuda") < L - n, previous[b, h, :N].double(), 0)
                bound, w = bound + 2.0 ** -24 * (w + old).abs(), w + old
            bad = ~((got[b, h, :N].double() - w).abs() <= bound)
            assert not bad.any(), f"sequence {b}, KV head {h}: {(got[b, h, :N] - w)[bad][:4].tolist()} at {bad.nonzero()[:4].tolist()}"
            if before is not None:
                assert torch.equal(got[b, h, N:], before[b, h, N:])


def turned(x, weight, rope, at, interleaved):
    """float64 of rows x [T, heads, 128], normalised and rotated, and the error bound of the kernel's bf16 result: the mean
    of the squares takes 128 products and sums, its root and quotient three roundings, of which the root takes a half: 70; two
    for the weight; a rotated dim is the sum of two products: two roundings of each. All relative to |a| + |b| of the pair."""
    x = x.double()
    size = x.abs()
    if weight is not None:
        f = weight.double() / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        x, size = x * f, size * f.abs()
    if rope is not None:
        half = rope.shape[1] // 2
        a = torch.arange(half, device=x.device)
        i, j = (2 * a, 2 * a + 1) if interleaved else (a, a + half)
        c, s = rope[at, :half].double().unsqueeze(1), rope[at, half:].double().unsqueeze(1)
        y, both = x.clone(), size.clone()
        y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
        both[..., i] = both[..., j] = size[..., i] + size[..., j]
        x, size = y, both
    return x, HALF_STEP * x.abs() + 76 * 2.0 ** -24 * (1 + HALF_STEP) * size + 2.0 ** -133


def evicted(batch, weights, budget, recent):
    """kept [B][Hkv] as lists, by sorting."""
    kept = []
    for b in range(batch.B):
        n = min(batch.lens[b], batch.cap)
        here = [j for j in range(n) if batch.there(b, j)]
        kept.append([])
        for h in range(batch.Hkv):
            w = weights[b, h].tolist()
            late = [j for j in here if j >= n - recent]
            order = sorted((j for j in here if j < n - recent), key=lambda j: (0 if w[j] != w[j] else 1, -w[j] if w[j] == w[j] else 0, j))
            kept[b].append(sorted(late + order[:max(0, budget - len(late))]))
    return kept
