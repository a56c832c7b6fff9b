"""What the binding of the paged caches' calls refuses, by name."""
import pytest
import torch

from . import paged_reference as R
from .kv8_reference import D
from .test_gpu_paged import ffd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def batch():
    return R.Batch([40, 7], [3, 7], 2, 2, 16, seed=80)


def test_numbers_beyond_32_bits(ffd, batch):  # noqa: F811
    _, lse = ffd.paged_attention(*batch.args)
    k = torch.zeros(batch.T, 2, D, device="cuda", dtype=torch.bfloat16)
    for x in (1e39, -1e39):
        for call in (lambda: ffd.paged_attention(*batch.args, softcap=x), lambda: ffd.paged_attention(*batch.args, softmax_scale=x),
                     lambda: ffd.paged_attention_weights(*batch.args, lse, softcap=x), lambda: ffd.write_paged(None, k, k, batch.cache, *batch.args[2:], eps=x)):
            with pytest.raises(ffd.FfdError):
                call()


@pytest.mark.parametrize("kw", [dict(softcap=-1.0), dict(softcap=float("inf")), dict(softcap=float("nan")), dict(window=-1), dict(softmax_scale=float("nan"))], ids=str)
def test_rules_that_are_none(ffd, batch, kw):  # noqa: F811
    with pytest.raises(ffd.FfdError):
        ffd.paged_attention(*batch.args, **kw)


def test_tensors_of_another_form(ffd, batch):  # noqa: F811
    """A type, shape or layout other than the one asked for, one argument at a time."""
    q, cache, table, q_start, lens = batch.args
    out, lse = ffd.paged_attention(*batch.args)
    weights = ffd.paged_attention_weights(*batch.args, lse)
    attend = lambda **kw: ffd.paged_attention(*{**dict(q=q, cache=cache, table=table, q_start=q_start, lens=lens), **{k: v for k, v in kw.items() if k in ("q", "cache", "table", "q_start", "lens")}}.values(),
                                              **{k: v for k, v in kw.items() if k not in ("q", "cache", "table", "q_start", "lens")})
    for kw in (dict(q=q.float()), dict(q=q[..., :64]), dict(q=q.transpose(0, 1)), dict(q=q.cpu()), dict(cache=(cache[0], cache[1][:, :1])), dict(cache=(cache[0], cache[1].float())),
               dict(cache=(cache[0].transpose(1, 2), cache[1])), dict(table=table.long()), dict(table=table[:, 0]), dict(table=table.T), dict(q_start=q_start[:2]),
               dict(q_start=q_start.long()), dict(lens=lens.cpu()), dict(lens=lens[:1]), dict(slopes=torch.ones(2, device="cuda")), dict(slopes=torch.ones(4)),
               dict(prefix_lens=lens.long()), dict(out=out.float()), dict(out=out[:1]), dict(lse=lse.double()), dict(lse=lse.T),
               dict(workspace=torch.empty(1 << 24, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            attend(**kw)
    with pytest.raises(ffd.FfdError):
        attend(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    for kw in (dict(lse=lse[:1]), dict(lse=lse.bfloat16()), dict(previous=weights[:1]), dict(previous=weights.double()), dict(out=weights[..., :16]), dict(out=weights.cpu())):
        with pytest.raises(ValueError):
            ffd.paged_attention_weights(*batch.args, **{**dict(lse=lse), **kw})
    new = R.int32([[batch.free[0]], [batch.free[1]]])
    for kw in (dict(new_table=new[:1]), dict(new_table=new.long()), dict(new_table=table), dict(seq_lens=lens[:1]), dict(weights=weights[..., :16]), dict(weights=weights.double()),
               dict(kept=torch.empty(2, 2, 4, dtype=torch.int32, device="cuda")), dict(new_lens=torch.empty(2, device="cuda")), dict(new_weights=weights), dict(budget=1 << 31)):
        a = {**dict(new_table=new, seq_lens=lens, weights=weights, budget=5), **kw}
        with pytest.raises(ValueError):
            ffd.evict_paged(cache, table, **a)
    for kw in (dict(budget=0), dict(budget=17), dict(budget=5, recent=6), dict(budget=5, recent=-1)):
        with pytest.raises(ffd.FfdError):
            ffd.evict_paged(cache, table, new, lens, weights, **kw)


def test_rows_of_another_form(ffd, batch):  # noqa: F811
    k, q = (torch.zeros(batch.T, h, D, device="cuda", dtype=torch.bfloat16) for h in (2, 4))
    odd = torch.zeros(batch.T, 2, D + 4, device="cuda", dtype=torch.bfloat16)[..., :D]          # strides that are not multiples of 8
    rope = torch.zeros(50, 64, device="cuda")
    write = lambda q=q, k=k, v=k, **kw: ffd.write_paged(q, k, v, batch.cache, *batch.args[2:], **kw)
    for kw in (dict(k=k.float()), dict(v=k[:1]), dict(k=k.transpose(1, 2)), dict(q=q[:-1]), dict(q=q.cpu()), dict(rope=rope.double()), dict(rope=rope[0]), dict(rope=rope[:, :32]),
               dict(positions=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(q_weight=torch.ones(D, device="cuda")), dict(k_weight=torch.ones(64, device="cuda").bfloat16()),
               dict(q=None, q_weight=torch.ones(D, device="cuda").bfloat16()), dict(out=q.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            write(**kw)
    for kw in (dict(k=odd), dict(v=odd), dict(rope=rope[:, :33].contiguous()), dict(rope=rope[:, :48].contiguous()), dict(eps=-1.0)):
        with pytest.raises(ffd.FfdError):
            write(**kw)
