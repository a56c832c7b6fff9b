"""Reading an 8-bit cache back with lengths: zeros behind them, without reading the cache there."""
import math
import statistics

import pytest
import torch

from tests.kv8_reference import D, random_cache, values

pytestmark = pytest.mark.gpu


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("t0,t1", [(0, 320), (1, 257), (63, 65), (64, 320), (130, 131)])
def test_lengths_around_every_border(t0, t1):
    """Lengths from none to the capacity and past it, around the tokens that a workgroup takes (64 from t0 on), with NaN and
    the largest codes behind them."""
    from paper_2609_00097_amd import ffd
    L = 320
    lens = sorted({n for x in (0, t0, t0 + 16, t0 + 64, t0 + 128, t1, L) for n in (x - 1, x, x + 1)}) + [-2 ** 31, 2 ** 31 - 1]
    gen = torch.Generator("cuda").manual_seed(t0 + t1)
    cache = random_cache(gen, len(lens), 2, L)
    want = [x[:, :, t0:t1].bfloat16() for x in values(cache)]
    for b, n in enumerate(lens):
        n = min(max(n, 0), L)
        for w in want:
            w[b, :, max(0, n - t0):] = 0
        for t in cache:
            t[b, :, n:] = 127 if t.dtype == torch.int8 else math.nan
    out = tuple(torch.full((len(lens), 2, t1 - t0, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    print(f"case ragged read [{t0}, {t1}) lens {lens}", flush=True)
    ffd.read_kv8(cache, t0, t1, seq_lens=_int32(lens), out=out)
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for x, w in zip(out, want))


def test_rows_behind_the_lengths_are_not_read():
    """A call of 256K tokens and eight KV heads moves 260 bytes in and 512 out for each; one of empty sequences only the 512.
    Two thirds of the time then, and never as much as the whole: 0.85 of it at the most. (Medians, in turn.)"""
    from paper_2609_00097_amd import ffd
    B, Hkv, L = 4, 8, 65536
    cache = random_cache(torch.Generator("cuda").manual_seed(1), 1, 1, L)
    cache = tuple(t.expand(B, Hkv, *t.shape[2:]).contiguous() for t in cache)
    out = tuple(torch.empty(B, Hkv, L, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    times = {}
    for i in range(15):
        for lens in (_int32([0] * B), None):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            ffd.read_kv8(cache, seq_lens=lens, out=out)
            b.record()
            b.synchronize()
            times.setdefault(lens is None, []).append(a.elapsed_time(b))
    none, whole = (statistics.median(times[x][3:]) for x in (False, True))
    print(f"empty sequences {1000 * none:.0f} us, whole {1000 * whole:.0f} us", flush=True)
    assert none < 0.85 * whole
