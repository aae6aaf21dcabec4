"""Prompts whose keys are split over the GPU, and prompts of more blocks than a grid holds, against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2311_09549_amd import binding as sc
from paper_2311_09549_amd.attention import Attention

from attention_reference import assert_within, attend, cache_of

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN, INF = float("nan"), float("inf")


def normal(gen, *shape, dtype=F32):
    return torch.randn(*shape, generator=gen).to(dtype)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return out


def some(n, most, gen):
    """Rows to look at: the first, the last, those beside borders of blocks, and others."""
    at = {0, n - 1} | {r for b in (32, 64, 128, 256) for r in (b - 1, b) if r < n} | {int(x) for x in torch.randint(0, n, (most,), generator=gen)}
    return sorted(at)


def check_rows(got, q, k, v, before, dtype, causal, gen, what):
    """Rows of one sequence, `before` keys ahead of the first."""
    at = some(len(q), 12, gen)
    sees = torch.tensor([before + r + 1 if causal else len(k) for r in at])
    want, bound = attend(q[at], k, v, sees, 1 / math.sqrt(q.shape[2]), dtype)
    assert_within(got[at], want, bound, what)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv_heads,head_dim,rows,causal", [
    (4, 2, 128, [1, 700, 0, 3, 1300, 65], True),
    (8, 1, 64, [2000], True),
    (3, 3, 128, [600, 600], False),
    (2, 1, 256, [530, 31, 700], True),
    (5, 1, 80, [900, 0, 0, 200], True),
    (1, 1, 64, [4000], True),
    (4, 2, 128, [3000, 1, 0], True),
    (5, 1, 80, [2500, 200], False),
])
def test_prompt(dtype, heads, kv_heads, head_dim, rows, causal):
    gen = torch.Generator().manual_seed(sum(rows) + head_dim)
    total = sum(rows)
    q, k, v = (normal(gen, total, h, head_dim, dtype=dtype) for h in (heads, kv_heads, kv_heads))
    attention = Attention(heads, kv_heads, head_dim, dtype, causal=causal)
    workspace = torch.full((attention.prompt_ws_bytes // 4,), NAN, device="cuda") if attention.prompt_ws_bytes else None   # its contents do not matter
    args = (q.cuda(), k.cuda(), v.cuda(), int32(starts(rows)))
    got = attention.prompt(*args, workspace=workspace)
    assert torch.equal(got, attention.prompt(*args))
    at = 0
    for n in rows:
        if n:
            check_rows(got[at:at + n].cpu(), q[at:at + n], k[at:at + n], v[at:at + n], 0, dtype, causal, gen, f"sequence of {n}")
        at += n


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv_heads,head_dim,page_rows,lengths,rows,causal", [
    (4, 1, 128, 16, [3000, 40, 0, 129, 700], [70, 1, 0, 129, 5], True),
    (2, 2, 64, 64, [5000], [33], True),
    (8, 2, 128, 32, [1500, 900], [300, 2], False),
    (2, 1, 256, 16, [800, 100], [100, 100], True),
    (1, 1, 64, 16, [1, 2, 3], [1, 1, 1], True),            # room for many more keys than there are
    (2, 1, 64, 16, [5, 600], [12, 600], True),             # rows before position 0
    (1, 1, 128, 16, [1, 2, 3], [1, 1, 1], True),
    (2, 1, 128, 16, [5, 600], [12, 600], True),
])
def test_prompt_paged(dtype, heads, kv_heads, head_dim, page_rows, lengths, rows, causal):
    gen = torch.Generator().manual_seed(sum(lengths) + head_dim)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, sum(rows), heads, head_dim, dtype=dtype)
    columns = max(-(-max(lengths) // page_rows), 1024 // page_rows) + 1
    kc, vc, table = cache_of(keys, values, page_rows, columns, gen)
    attention = Attention(heads, kv_heads, head_dim, dtype, page_rows, causal=causal)
    got = attention.prompt_paged(q.cuda(), kc, vc, table, int32(lengths), int32(starts(rows))).cpu()
    at = 0
    for b, n in enumerate(rows):
        before = lengths[b] - n
        blind = max(0, -before) if causal else 0
        assert bool((got[at:at + blind] == 0).all())
        if n > blind:
            check_rows(got[at + blind:at + n], q[at + blind:at + n], keys[b], values[b], before + blind, dtype, causal, gen, f"sequence {b}")
        at += n


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_wrong_tables(dtype, head_dim):
    """Wrong lengths and pages make NaN of rows of their sequences alone, wherever shares end; row starts out of order stay in range."""
    gen = torch.Generator().manual_seed(3)
    lengths = [900, 900, 900, 900, 900]
    keys, values = ([normal(gen, 900, 1, head_dim, dtype=dtype) for _ in lengths] for _ in range(2))
    q = normal(gen, 100 * len(lengths), 2, head_dim, dtype=dtype)
    kc, vc, table = cache_of(keys, values, 16, 64, gen)
    table[1, 2] = kc.shape[0]
    table[2, 0] = -5
    attention = Attention(2, 1, head_dim, dtype, 16)
    got = attention.prompt_paged(q.cuda(), kc, vc, table, int32([900, 900, 900, -1, 1025]), int32(starts([100] * 5))).cpu()
    check_rows(got[:100], q[:100], keys[0], values[0], 800, dtype, True, gen, "good sequence")
    assert bool(torch.isnan(got[100:]).all())
    for wrong in ([0, 30, -7, 500, 400, 500], [500, 0, 0, 0, 0, 0], [0, 0, 0, 0, 0, 0], [-9, 2 ** 31 - 1, 0, 500, 500, 500]):
        attention.prompt_paged(q.cuda(), kc, vc, table, int32([900, 0, 7, 900, 1024]), int32(wrong))
        torch.cuda.synchronize()


@pytest.mark.parametrize("bad", [NAN, INF])
def test_hidden_keys_reach_nothing(bad):
    gen = torch.Generator().manual_seed(4)
    n = 1100
    q, k, v = (normal(gen, n, 1, 128, dtype=BF16) for _ in range(3))
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[800], bad_v[800] = bad, bad
    got = Attention(1, 1, 128, BF16).prompt(q.cuda(), bad_k.cuda(), bad_v.cuda(), int32([0, n])).cpu()
    check_rows(got[:800], q[:800], k[:800], v[:800], 0, BF16, True, gen, "rows before")
    assert not bool(torch.isfinite(got[800:].float()).all(dim=-1).any())


def test_workspace_refusals():
    attention = Attention(1, 1, 64, BF16)
    x = torch.zeros(600, 1, 64, dtype=BF16, device="cuda")
    with pytest.raises(sc.ScError, match="SC_ERR_WORKSPACE_SMALL"):
        attention.prompt(x, x, x, int32([0, 600]), workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(sc.ScError, match="SC_ERR_SHAPE_MISMATCH"):
        attention.prompt(x, x, x, int32([0, 600]), workspace=torch.zeros(attention.prompt_ws_bytes + 16, dtype=torch.uint8, device="cuda")[16:])


def test_step_in_a_graph():
    """A split prompt captured once and replayed for other lengths: each replay as the eager call, bit for bit."""
    gen = torch.Generator().manual_seed(6)
    keys, values = ([normal(gen, n, 1, 128, dtype=BF16) for n in (2000, 1400)] for _ in range(2))
    q = normal(gen, 100, 4, 128, dtype=BF16).cuda()
    kc, vc, table = cache_of(keys, values, 64, 40, gen, fill=0.0)
    attention = Attention(4, 1, 128, BF16, 64)
    lengths, row_start, out = int32([2000, 1400]), int32([0, 60, 100]), torch.empty_like(q)
    choices = [([2000, 1400], [0, 60, 100]), ([70, 900], [0, 1, 100])]
    eager = []
    for n, r in choices:
        lengths.copy_(int32(n))
        row_start.copy_(int32(r))
        eager.append(attention.prompt_paged(q, kc, vc, table, lengths, row_start).clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attention.prompt_paged(q, kc, vc, table, lengths, row_start, out=out)
    for i in (0, 1, 0):
        lengths.copy_(int32(choices[i][0]))
        row_start.copy_(int32(choices[i][1]))
        out.fill_(NAN)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i])


def test_workspaces_stay_where_a_graph_has_them():
    """A captured token, then a long prompt through the same handle: replays go on as before."""
    gen = torch.Generator().manual_seed(7)
    keys, values = ([normal(gen, 1500, 1, 64, dtype=BF16)] for _ in range(2))
    kc, vc, table = cache_of(keys, values, 64, 30, gen, fill=0.0)
    attention = Attention(2, 1, 64, BF16, 64)
    q, lengths, out = normal(gen, 1, 2, 64, dtype=BF16).cuda(), int32([1500]), torch.empty(1, 2, 64, dtype=BF16, device="cuda")
    eager = attention.decode(q, kc, vc, table, lengths).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attention.decode(q, kc, vc, table, lengths, out=out)
    x = normal(gen, 2000, 2, 64, dtype=BF16).cuda()
    for _ in range(2):
        attention.prompt(x, x[:, :1], x[:, :1], int32([0, 2000]))
        others = [torch.full((1 << 22,), NAN, device="cuda") for _ in range(4)]   # would be given the memory of a workspace that is gone
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert all(bool(torch.isnan(x).all()) for x in others)


def test_more_blocks_than_a_grid_holds():
    """Sequences of one row and one key: every row is its value."""
    batch, heads = 3000, 4096
    v = torch.randn(batch, heads, 8, device="cuda").to(BF16)
    got = Attention(heads, heads, 8, BF16).prompt(v, v, v, torch.arange(batch + 1, dtype=torch.int32, device="cuda"))
    assert torch.equal(got, v)
