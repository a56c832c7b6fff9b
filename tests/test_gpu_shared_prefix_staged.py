"""The tests of the shared prefix again with prefixes in so large a capacity that more than 32 query rows are never cut into
tiles of 32: the kernel that stages tokens in LDS takes them, in both forms and for every number of rows."""
import inspect
import itertools

import pytest
import torch

from tests import test_gpu_shared_prefix as cases
from tests.test_gpu_shared_prefix_rounding import _large, _padded

pytestmark = pytest.mark.gpu


def _calls():
    """(test, arguments) of every parametrised test that takes room, with room."""
    for name, test in inspect.getmembers(cases, inspect.isfunction):
        if not name.startswith("test_") or "room" not in inspect.signature(test).parameters:
            continue
        axes = []
        for mark in test.pytestmark:
            if mark.name == "parametrize" and mark.args[0] != "room":
                names = mark.args[0].split(",")
                axes.append([dict(zip(names, x if len(names) > 1 else (x,))) for x in mark.args[1]])
        for point in itertools.product(*axes):
            yield pytest.param(test, {k: v for part in point for k, v in part.items()}, id=f"{name[5:]}-{len(axes)}")


@pytest.mark.parametrize("test,arguments", list(_calls()))
def test_staged(test, arguments, monkeypatch):
    def with_room(prefix, rows, room):
        return _padded(prefix, _large(rows, prefix[0].shape[1], prefix[0].shape[2])) if rows > 32 else prefix

    monkeypatch.setattr(cases, "_with_room", with_room)
    print(f"case {test.__name__} {arguments}", flush=True)
    test(**arguments, room=True)


@pytest.mark.parametrize("B", [40, 100])
@pytest.mark.parametrize("short", [0, 1, 5000])
def test_a_prefix_filled_to_a_large_capacity(B, short):
    """test_a_prefix_filled_to_its_capacity in a capacity past all limits of little work: the first tiles are asked for as if
    the lengths were the capacity, with that and with shorter lengths."""
    from paper_2609_00097_amd import ffd
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    P = 64 * -(-(129 * 1024 * cus) // (64 * B))
    gen = cases._gen(B)
    k, v = torch.zeros(1, 1, P, 128, dtype=torch.bfloat16, device="cuda"), cases._normal(gen, 1, 1, P, 128)
    units = -(-(P - short) // 128)
    at = []
    for j in range(B):
        run = j * cus // B
        start = 128 * (units // cus * run + min(run, units % cus))
        at.append(min(max(start - (j & 1), 0), P - short - 1))
        k[0, 0, at[j], j] = 1
    k[:, :, P - short:] = float("nan")
    v[:, :, P - short:] = float("nan")
    q = torch.zeros(B, 1, 128, dtype=torch.bfloat16, device="cuda")
    q[torch.arange(B), 0, torch.arange(B)] = 30.0
    cache = cases.random_cache(gen, B, 1, 64, 16)
    out, _ = ffd.shared_prefix_decode_attention(q, (k, v), cases._int32([P - short] * B), cache, cases._int32([0] * B), softmax_scale=1.0)
    # the others' weight is at most P e^-30, 8e-8, of values below 6; the one's, a probability near 1, is rounded to 2^-16
    want = v[0, 0, at].double()
    assert bool(((out[:, 0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -14).all())
