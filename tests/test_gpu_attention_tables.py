"""Tables of pages that are wider than the keys, and views of them: a view gives the kernels a bound of the lengths."""
import pytest
import torch

from paper_2311_09549_amd.attention import Attention

from attention_reference import assert_within, attend, cache_of

pytestmark = pytest.mark.gpu


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("columns", [21, 32, 400])
def test_views_of_a_table(dtype, columns):
    """The first `columns` of 500, as a view: a call of the same operator on a table of its own gives the same bits; a length beyond them is a wrong one."""
    gen = torch.Generator().manual_seed(columns)
    lengths = [333, 60, 1]
    keys, values = ([torch.randn(n, 2, 64, generator=gen).to(dtype) for n in lengths] for _ in range(2))
    q = torch.randn(3, 8, 64, generator=gen).to(dtype)
    kc, vc, table = cache_of(keys, values, 16, 500, gen)
    attention, view = Attention(8, 2, 64, dtype, 16), table[:, :columns]
    assert not view.is_contiguous()
    got = attention.decode(q.cuda(), kc, vc, view, int32(lengths))
    assert torch.equal(got, attention.decode(q.cuda(), kc, vc, view.contiguous(), int32(lengths)))
    rows = torch.randn(40, 8, 64, generator=gen).to(dtype)
    more = attention.prompt_paged(rows.cuda(), kc, vc, view, int32(lengths), int32([0, 30, 39, 40]))
    assert torch.equal(more, attention.prompt_paged(rows.cuda(), kc, vc, view.contiguous(), int32(lengths), int32([0, 30, 39, 40])))
    for b, n in enumerate(lengths):
        want, bound = attend(q[b:b + 1], keys[b], values[b], torch.tensor([n]), 1 / 8, dtype)
        assert_within(got[b:b + 1], want, bound, f"token of {b}")
        lo, hi = (0, 30, 39, 40)[b:b + 2]
        want, bound = attend(rows[lo:hi], keys[b], values[b], torch.arange(n - hi + lo, n) + 1, 1 / 8, dtype)
        assert_within(more[lo:hi], want, bound, f"rows of {b}")
    if columns == 21:
        wrong = attention.decode(q.cuda(), kc, vc, table[:, :20], int32(lengths)).cpu()
        assert bool(torch.isnan(wrong[0]).all()) and torch.equal(wrong[1:], got[1:].cpu())
