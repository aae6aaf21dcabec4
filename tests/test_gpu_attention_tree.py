"""Trees of drafted rows on the GPU, against the definition in 64 bits: append by depths, attention of nodes over the cache and their ancestors, and the accepted path."""
import math

import pytest
import torch

from paper_2311_09549_amd.attention import Attention

from attention_masks import attend_seen, path_of, random_tree, tree_mask
from attention_reference import assert_within, cache_of, half_step, rotated

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN, INF = float("nan"), float("inf")
DTYPES = [BF16, F16, F32]


def normal(gen, *shape, dtype=F32):
    return torch.randn(*shape, generator=gen).to(dtype)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return out


def flat(trees):
    return [p for t in trees for p in t]


SHAPES = [
    # heads, kv_heads, head_dim, page_rows, lengths, nodes, spread, heads_first
    (1, 1, 64, 16, [1], [1], 1, False),
    (4, 2, 128, 16, [100, 33, 16, 17, 1], [7, 1, 16, 5, 1], 3, False),
    (4, 1, 128, 16, [200, 40, 65], [33, 40, 64], 6, True),
    (8, 8, 64, 32, [500, 3], [20, 3], 4, True),
    (32, 4, 64, 16, [300, 77], [9, 30], 5, False),
    (5, 1, 80, 16, [200, 31], [13, 31], 31, False),
    (20, 1, 128, 64, [300, 40], [3, 2], 1, False),
    (6, 2, 256, 16, [130, 70], [21, 50], 8, False),
    (2, 2, 136, 16, [90, 400], [90, 100], 12, False),
    (2, 1, 8, 16, [140], [70], 9, False),
    (4, 1, 128, 128, [5000], [12], 4, False),            # one long sequence, split over many workgroups
    (3, 1, 64, 64, [1400, 1024], [1000, 1024], 40, False),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,head_dim,page_rows,lengths,nodes,spread,heads_first", SHAPES)
@pytest.mark.parametrize("window,sinks", [(None, 0), (19, 3)])
@pytest.mark.parametrize("more_columns", [1, 2000])      # a table with room for many more keys takes other kernels
def test_tree(dtype, heads, kv_heads, head_dim, page_rows, lengths, nodes, spread, heads_first, window, sinks, more_columns):
    gen = torch.Generator().manual_seed(sum(lengths) + head_dim)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, sum(nodes), heads, head_dim, dtype=dtype)
    trees = [random_tree(n, spread, gen) for n in nodes]
    columns = -(-max(lengths) // page_rows) + more_columns
    kc, vc, table = cache_of(keys, values, page_rows, columns, gen, heads_first)
    attention = Attention(heads, kv_heads, head_dim, dtype, page_rows, window=window, sinks=sinks)
    workspace = torch.full((attention.tree_ws_bytes // 4,), NAN, device="cuda")   # its contents do not matter
    args = (q.cuda(), kc, vc, table, int32(lengths), int32(starts(nodes)), int32(flat(trees)))
    got = attention.tree(*args, workspace=workspace)
    assert torch.equal(got, attention.tree(*args))
    got, at = got.cpu(), 0
    for b, n in enumerate(nodes):
        want, bound = attend_seen(q[at:at + n], keys[b], values[b], tree_mask(trees[b], lengths[b], window, sinks)[0], 1 / math.sqrt(head_dim), dtype)
        assert_within(got[at:at + n], want, bound, f"tree {b}")
        at += n


LONG = [
    # heads, kv_heads, head_dim, lengths, nodes, window, sinks
    (4, 2, 128, [3000, 700, 1, 513], [5, 4, 1, 6], None, 0),          # one tile of pairs
    (4, 2, 128, [3000, 700, 12, 513], [12, 9, 12, 16], None, 0),      # two
    (8, 2, 128, [3000, 700, 12, 513], [12, 9, 12, 16], None, 0),      # four
    (8, 2, 64, [3000, 700, 12, 513], [12, 9, 12, 16], None, 0),
    (4, 4, 104, [2000, 900], [40, 33], None, 0),
    (3, 1, 256, [2000, 900], [7, 30], None, 0),
    (8, 1, 128, [6000], [64], None, 0),                               # tiles through LDS, keys split
    (8, 1, 64, [6000], [70], None, 0),
    (2, 1, 256, [2500, 1000], [100, 70], None, 0),
    (16, 2, 72, [4000, 900, 50], [130, 20, 50], None, 0),
    (4, 2, 128, [3000, 700, 12, 513], [12, 9, 12, 16], 600, 40),      # a window whose edge is far from the tree
    (8, 2, 64, [3000, 700, 12, 513], [12, 9, 12, 16], 640, 0),
    (8, 1, 128, [6000], [64], 2000, 130),
    (3, 1, 256, [2000, 900], [7, 30], 555, 1),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,head_dim,lengths,nodes,window,sinks", LONG)
def test_tree_behind_many_keys(dtype, heads, kv_heads, head_dim, lengths, nodes, window, sinks):
    gen = torch.Generator().manual_seed(sum(lengths) + head_dim)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, sum(nodes), heads, head_dim, dtype=dtype)
    trees = [random_tree(n, 5, gen) for n in nodes]
    kc, vc, table = cache_of(keys, values, 32, -(-max(lengths) // 32), gen)
    for b, n in enumerate(lengths):        # pages that no node sees are given back
        for c in range(table.shape[1]):
            if window is not None and c * 32 >= sinks and (c + 1) * 32 <= n - nodes[b] - window + 1:
                table[b, c] = -1
    attention = Attention(heads, kv_heads, head_dim, dtype, 32, window=window, sinks=sinks)
    args = (q.cuda(), kc, vc, table, int32(lengths), int32(starts(nodes)), int32(flat(trees)))
    got = attention.tree(*args)
    assert torch.equal(got, attention.tree(*args))
    got, at = got.cpu(), 0
    for b, n in enumerate(nodes):
        want, bound = attend_seen(q[at:at + n], keys[b], values[b], tree_mask(trees[b], lengths[b], window, sinks)[0], 1 / math.sqrt(head_dim), dtype)
        assert_within(got[at:at + n], want, bound, f"tree {b}")
        at += n


def test_blocks_of_many_sequences():
    """More sequences than are counted to find a block, with and without rows; blocks of one sequence one behind the other."""
    gen = torch.Generator().manual_seed(6)
    lengths = [int(x) for x in torch.randint(1, 90, (1100,), generator=gen)]
    nodes = [min(n, int(x)) for n, x in zip(lengths, torch.randint(0, 60, (1100,), generator=gen))]
    for count in (1100, 130):
        keys, values = ([normal(gen, n, 1, 64, dtype=BF16) for n in lengths[:count]] for _ in range(2))
        q = normal(gen, sum(nodes[:count]), 8, 64, dtype=BF16)
        trees = [random_tree(n, 3, gen) for n in nodes[:count]]
        kc, vc, table = cache_of(keys, values, 16, 40, gen)
        got = Attention(8, 1, 64, BF16, 16).tree(q.cuda(), kc, vc, table, int32(lengths[:count]), int32(starts(nodes[:count])), int32(flat(trees))).cpu()
        at = 0
        for b, n in enumerate(nodes[:count]):
            if n and (b % 7 == 0 or n > 50):
                want, bound = attend_seen(q[at:at + n], keys[b], values[b], tree_mask(trees[b], lengths[b])[0], 1 / 8, BF16)
                assert_within(got[at:at + n], want, bound, f"tree {b}")
            at += n


@pytest.mark.parametrize("dtype", DTYPES)
def test_chains(dtype):
    """Without parents each row follows the one before; more rows than a tree may have."""
    gen = torch.Generator().manual_seed(2)
    lengths, nodes = [1500, 40, 0, 9], [1100, 40, 0, 1]
    keys, values = ([normal(gen, n, 2, 64, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, sum(nodes), 4, 64, dtype=dtype)
    kc, vc, table = cache_of(keys, values, 16, 100, gen)
    got = Attention(4, 2, 64, dtype, 16).tree(q.cuda(), kc, vc, table, int32(lengths), int32(starts(nodes))).cpu()
    at = 0
    for b, n in enumerate(nodes):
        if n:
            want, bound = attend_seen(q[at:at + n], keys[b], values[b], tree_mask(list(range(-1, n - 1)), lengths[b])[0], 1 / 8, dtype)
            assert_within(got[at:at + n], want, bound, f"chain {b}")
        at += n


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_sequences(dtype):
    """More sequences than a wavefront has lanes, some without rows, and rows of no sequence, which are not written."""
    gen = torch.Generator().manual_seed(5)
    lengths = [int(x) for x in torch.randint(1, 500, (150,), generator=gen)]
    nodes = [min(n, int(x)) for n, x in zip(lengths, torch.randint(0, 12, (150,), generator=gen))]
    keys, values = ([normal(gen, n, 2, 64, dtype=dtype) for n in lengths] for _ in range(2))
    total = sum(nodes)
    q = normal(gen, 3 + total + 4, 4, 64, dtype=dtype)
    trees = [random_tree(n, 3, gen) for n in nodes]
    kc, vc, table = cache_of(keys, values, 64, 9, gen)
    out = torch.full_like(q, 7.0).cuda()
    row_start = [3 + x for x in starts(nodes)]
    Attention(4, 2, 64, dtype, 64).tree(q.cuda(), kc, vc, table, int32(lengths), int32(row_start), int32([9] * 3 + flat(trees) + [-5] * 4), out=out)
    got = out.cpu()
    assert bool((got[:3] == 7.0).all()) and bool((got[3 + total:] == 7.0).all())
    for b, n in enumerate(nodes):
        if n:
            at = row_start[b]
            want, bound = attend_seen(q[at:at + n], keys[b], values[b], tree_mask(trees[b], lengths[b])[0], 1 / 8, dtype)
            assert_within(got[at:at + n], want, bound, f"tree {b}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128, 256])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("heads,columns", [(2, 3), (1, 100), (2, 100), (8, 100)])      # by each kind of kernel
def test_other_branches_reach_nothing(dtype, head_dim, bad, heads, columns):
    """Two branches: what one of them holds reaches its own nodes alone; rows behind the length hold the same."""
    gen = torch.Generator().manual_seed(head_dim)
    n, nodes = 75, 40
    k, v, q = normal(gen, n, 1, head_dim, dtype=dtype), normal(gen, n, 1, head_dim, dtype=dtype), normal(gen, nodes, heads, head_dim, dtype=dtype)
    tree = [-1, -1] + [i - 2 for i in range(2, nodes)]       # even nodes one branch, odd nodes the other
    seen, _ = tree_mask(tree, n)
    bad_k, bad_v = k.clone(), v.clone()
    for x in (bad_k, bad_v):
        x[n - nodes + 1::2] = bad
    kc, vc, table = cache_of([bad_k], [bad_v], 64, columns, gen, fill=bad)
    got = Attention(heads, 1, head_dim, dtype, 64).tree(q.cuda(), kc, vc, table, int32([n]), int32([0, nodes]), int32(tree)).cpu()
    want, bound = attend_seen(q, k, v, seen, 1 / math.sqrt(head_dim), dtype)
    assert_within(got[::2], want[::2], bound[::2])
    if math.isnan(bad):
        assert bool(torch.isnan(got[1::2]).all())
    else:
        assert not bool(torch.isfinite(got[1::2]).all(dim=-1).any())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,columns", [(1, 2), (1, 100), (32, 100)])
def test_lowest_scores(dtype, heads, columns):
    """Scores of the type's lowest value are scores like others; nodes whose scores are all -infinity give +0."""
    d, n = 64, 20
    q, k, v = torch.zeros(4, heads, d, dtype=dtype), torch.zeros(n, 1, d, dtype=dtype), torch.ones(n, 1, d, dtype=dtype)
    q[..., 0] = 1.0
    gen = torch.Generator().manual_seed(1)
    for low, value in ((torch.finfo(dtype).min, 1.0), (-INF, 0.0)):
        k[:, 0, 0] = low
        kc, vc, table = cache_of([k], [v], 16, columns, gen)
        got = Attention(heads, 1, d, dtype, 16, scale=1.0).tree(q.cuda(), kc, vc, table, int32([n]), int32([0, 4]), int32([-1, 0, 0, -1])).cpu()
        assert bool((got == value).all()) and not bool(torch.signbit(got).any())


@pytest.mark.parametrize("heads,columns", [(4, 7), (4, 100), (64, 100)])
def test_wrong_tables(heads, columns):
    """Wrong lengths, pages and parents make NaN of the rows that they concern and leave the others as they are."""
    gen = torch.Generator().manual_seed(7)
    n, nodes = 100, 6
    count = 9
    keys, values = ([normal(gen, n, 2, 64, dtype=BF16) for _ in range(count)] for _ in range(2))
    q = normal(gen, count * nodes, heads, 64, dtype=BF16)
    tree = [-1, 0, 0, 1, 1, 4]
    trees = [list(tree) for _ in range(count)]
    trees[5][2] = 2          # itself: node 2 alone, which nobody follows
    trees[6][1] = -2         # nodes 1, 3, 4, 5
    trees[7][4] = 5          # a later one: nodes 4 and 5
    trees[8][5] = 2 ** 31 - 1
    kc, vc, table = cache_of(keys, values, 16, columns, gen)
    table[1, 3] = -1
    table[2, 6] = kc.shape[0]
    lengths = int32([n, n, n, -1, nodes - 1, n, n, n, n])
    got = Attention(heads, 2, 64, BF16, 16).tree(q.cuda(), kc, vc, table, lengths, int32(starts([nodes] * count)), int32(flat(trees))).cpu()
    wrong = {0: [], 1: range(6), 2: range(2, 6), 3: range(6), 4: range(6), 5: [2], 6: [1, 3, 4, 5], 7: [4, 5], 8: [5]}
    for b in range(count):
        want, bound = attend_seen(q[b * nodes:(b + 1) * nodes], keys[b], values[b], tree_mask(tree, n)[0], 1 / 8, BF16)
        for i in range(nodes):
            row = got[b * nodes + i]
            if b == 2 and i < 2:
                continue         # they do not see the page, but a tile of their keys has it
            if i in wrong[b]:
                assert bool(torch.isnan(row).all()), (b, i)
            else:
                assert_within(row, want[i], bound[i], f"node {i} of {b}")


def test_too_many_nodes_are_a_wrong_length():
    gen = torch.Generator().manual_seed(8)
    k, v, q = (normal(gen, 1030, 1, 64, dtype=F16) for _ in range(3))
    kc, vc, table = cache_of([k], [v], 16, 65, gen)
    attention = Attention(1, 1, 64, F16, 16)
    parents = int32(list(range(-1, 1029)))
    assert bool(torch.isnan(attention.tree(q[:1025].cuda(), kc, vc, table, int32([1030]), int32([0, 1025]), parents[:1025])).all())
    before = kc.clone(), vc.clone()
    assert attention.accept(kc, vc, table, int32([1030]), int32([0, 1025]), parents[:1025], int32([1024])).tolist() == [-1]
    torch.cuda.synchronize()
    assert torch.equal(before[0].view(torch.int16), kc.view(torch.int16)) and torch.equal(before[1].view(torch.int16), vc.view(torch.int16))


def test_wrong_row_starts():
    """Row starts out of range and out of order: nothing outside is read or written."""
    gen = torch.Generator().manual_seed(12)
    k, v, q = normal(gen, 100, 1, 64, dtype=BF16), normal(gen, 100, 1, 64, dtype=BF16), normal(gen, 40, 1, 64, dtype=BF16)
    kc, vc, table = cache_of([k] * 3, [v] * 3, 16, 7, gen)
    tree = random_tree(40, 4, gen)
    want, bound = attend_seen(q[:10], k, v, tree_mask(tree[:10], 100)[0], 1 / 8, BF16)
    wide = torch.full((3, 200), -1, dtype=torch.int32, device="cuda")
    wide[:, :7] = table
    many = q.repeat(1, 16, 1)
    for row_start in ([0, 10, -7, 40], [0, 10, 500, 2 ** 31 - 1], [-9, 10, 10, 8], [40, 0, 0, 0]):
        for heads, pages, rows in ((1, table, q), (1, wide, q), (16, wide, many)):      # by each kind of kernel
            out = Attention(heads, 1, 64, BF16, 16).tree(rows.cuda(), kc, vc, pages, int32([100] * 3), int32(row_start), int32(tree), out=torch.zeros_like(rows).cuda()).cpu()
            if row_start[0] <= 0 and row_start[2] != -7:
                assert_within(out[:8], want[:8].expand(8, heads, 64), bound[:8].expand(8, heads, 64))


def test_cache_beyond_32_bits():
    """Pages whose offsets pass 2^32 elements (and bytes): append, attention, accept and copy."""
    gen = torch.Generator().manual_seed(8)
    pages, rows, d, n, nodes = 40_000, 64, 128, 150, 9
    kc, vc = (torch.empty(pages, rows, 16, d, dtype=BF16, device="cuda") for _ in range(2))
    keys, values, q = normal(gen, n, 16, d, dtype=BF16), normal(gen, n, 16, d, dtype=BF16), normal(gen, nodes, 16, d, dtype=BF16)
    table = int32([[pages - 1, 1, pages - 5]])
    tree = random_tree(nodes, 2, gen)
    attention = Attention(16, 16, d, BF16, rows, window=140)
    attention.append(None, keys[:n - nodes].cuda(), values[:n - nodes].cuda(), kc, vc, table, int32([n - nodes]), int32([0, n - nodes]))
    attention.append(None, keys[n - nodes:].cuda(), values[n - nodes:].cuda(), kc, vc, table, int32([n]), int32([0, nodes]), parents=int32(tree))
    want, bound = attend_seen(q, keys, values, tree_mask(tree, n, 140)[0], 1 / math.sqrt(d), BF16)
    got = attention.tree(q.cuda(), kc, vc, table, int32([n]), int32([0, nodes]), int32(tree)).cpu()
    assert_within(got, want, bound)
    path = path_of(tree, nodes - 1)
    after = attention.accept(kc, vc, table, int32([n]), int32([0, nodes]), int32(tree), int32([nodes - 1]))
    assert after.tolist() == [n - nodes + len(path)]
    attention.copy(kc, vc, int32([[pages - 5, pages - 2, rows]]))
    for cache, x in ((kc, keys), (vc, values)):
        for at, i in enumerate(path):
            place = n - nodes + at
            assert torch.equal(cache[int(table[0, place // rows]), place % rows].cpu(), x[n - nodes + i])
        assert torch.equal(cache[pages - 5], cache[pages - 2])


# -- append -------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,head_dim,rotary_dim,interleaved,page_rows,lengths,nodes,heads_first", [
    (4, 2, 64, 64, False, 16, [1], [1], False),
    (4, 2, 128, 128, False, 16, [30, 100, 17, 33], [5, 20, 1, 33], False),
    (3, 1, 128, 64, True, 32, [70], [70], True),
    (2, 2, 72, 36, False, 16, [40, 9], [3, 9], False),
    (2, 1, 40, 0, False, 64, [90], [17], True),
])
def test_append(dtype, heads, kv_heads, head_dim, rotary_dim, interleaved, page_rows, lengths, nodes, heads_first):
    gen = torch.Generator().manual_seed(sum(nodes) + rotary_dim)
    total = sum(nodes)
    q, k, v = (normal(gen, total, h, head_dim, dtype=dtype) for h in (heads, kv_heads, kv_heads))
    old = [normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths]
    trees = [random_tree(n, 4, gen) for n in nodes]
    kc, vc, table = cache_of(old, old, page_rows, -(-max(lengths) // page_rows), gen, heads_first, fill=3.0)
    expect_k, expect_v, limit = kc.double().cpu(), vc.double().cpu(), torch.zeros(kc.shape, dtype=torch.float64)
    freq = [100.0 ** (-2.0 * t / max(rotary_dim, 1)) for t in range(rotary_dim // 2)]
    attention = Attention(heads, kv_heads, head_dim, dtype, page_rows, rotary_freq=freq, interleaved=interleaved)
    got = attention.append(q.cuda(), k.cuda(), v.cuda(), kc, vc, table, int32(lengths), int32(starts(nodes)), parents=int32(flat(trees))).cpu()
    u = half_step(dtype)
    at = 0
    for b, n in enumerate(nodes):
        position = tree_mask(trees[b], lengths[b])[1]
        want, bound = rotated(q[at:at + n], position, freq, interleaved)
        assert_within(got[at:at + n], want, bound + u * (want.abs() + bound) * (rotary_dim > 0), f"queries of {b}")
        want, bound = rotated(k[at:at + n], position, freq, interleaved)
        for i in range(n):
            p = lengths[b] - n + i
            page = int(table[b, p // page_rows])
            expect_k[page, p % page_rows], expect_v[page, p % page_rows] = want[i], v[at + i].double()
            limit[page, p % page_rows] = bound[i] + u * (want[i].abs() + bound[i]) * (rotary_dim > 0)
        at += n
    assert_within(kc, expect_k, limit, "keys")
    assert torch.equal(vc.double().cpu(), expect_v)


def test_append_wrong_tables():
    """Rows with wrong parents or of wrong lengths are not stored, nor anything else written."""
    gen = torch.Generator().manual_seed(9)
    k = normal(gen, 9, 1, 64, dtype=BF16).cuda()
    caches = [torch.full((4, 16, 1, 64), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
    parents = int32([-1, 1, 1, -1, 0, -1, 7, -2, -1])      # row 1 follows itself, row 2 follows it; a length of one for two; then one row each
    Attention(1, 1, 64, BF16, 16).append(None, k, k, *caches, int32([[0], [1], [2], [3], [-1], [3]]), int32([3, 1, 1, 2, 2, 1]), int32([0, 3, 5, 6, 7, 8, 9]), parents=parents)
    expect = [torch.full((4, 16, 1, 64), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
    for x in expect:
        x[0, 0], x[2, 0], x[3, 0] = k[0], k[5], k[8]
    for cache, x in zip(caches, expect):
        assert torch.equal(cache, x)


def test_append_of_wrong_lengths():
    """More nodes than a tree may have, and a length that the table has no room for: nothing is stored, also of the rows whose places it has."""
    gen = torch.Generator().manual_seed(14)
    attention = Attention(1, 1, 64, BF16, 16)
    for nodes, length, columns in ((1025, 1030, 65), (1024, 1030, 65), (5, 33, 2), (5, 32, 2)):
        k = normal(gen, nodes, 1, 64, dtype=BF16).cuda()
        kc, vc = (torch.full((columns, 16, 1, 64), 5.0, dtype=BF16, device="cuda") for _ in range(2))
        attention.append(None, k, k, kc, vc, torch.arange(columns, dtype=torch.int32, device="cuda")[None], int32([length]), int32([0, nodes]), parents=int32(range(-1, nodes - 1)))
        expect = torch.full((columns * 16, 1, 64), 5.0, dtype=BF16, device="cuda")
        if nodes <= 1024 and length <= 16 * columns:
            expect[length - nodes:length] = k
        for cache in (kc, vc):
            assert torch.equal(cache.view(-1, 1, 64), expect), (nodes, length)


def test_no_rows():
    """Sequences without rows: nothing is stored, and paths of no nodes leave what is before them."""
    gen = torch.Generator().manual_seed(15)
    k, v = normal(gen, 20, 1, 64, dtype=BF16), normal(gen, 20, 1, 64, dtype=BF16)
    kc, vc, table = cache_of([k, k], [v, v], 16, 2, gen, fill=0.0)
    before = kc.clone(), vc.clone()
    attention, lengths, row_start, none = Attention(2, 1, 64, BF16, 16), int32([20, 11]), int32([0, 0, 0]), int32([])
    q, new = torch.empty(0, 2, 64, dtype=BF16, device="cuda"), torch.empty(0, 1, 64, dtype=BF16, device="cuda")
    assert attention.append(q, new, new, kc, vc, table, lengths, row_start, parents=none).shape == q.shape
    assert attention.tree(q, kc, vc, table, lengths, row_start, none).shape == q.shape
    assert attention.accept(kc, vc, table, lengths, row_start, none, int32([-1, -1])).tolist() == [20, 11]
    assert attention.accept(kc, vc, table, lengths, row_start, none, int32([0, -1])).tolist() == [-1, 11]
    assert torch.equal(kc, before[0]) and torch.equal(vc, before[1])


# -- the accepted path ----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("kv_heads,head_dim,page_rows,lengths,nodes,spread", [
    (1, 64, 16, [1], [1], 1),
    (2, 128, 16, [40, 33, 16, 100, 20], [9, 1, 16, 30, 7], 4),
    (8, 128, 32, [200, 77], [63, 40], 3),
    (3, 72, 16, [90, 91, 92], [50, 50, 50], 1),         # a chain: nothing moves, or all of it
    (16, 256, 64, [130], [100], 2),
    (1, 8, 16, [1100], [1024], 1),
])
def test_accept(dtype, heads_first, kv_heads, head_dim, page_rows, lengths, nodes, spread):
    gen = torch.Generator().manual_seed(sum(nodes))
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    trees = [random_tree(n, spread, gen) for n in nodes]
    for last in ([n - 1 for n in nodes], [-1] * len(nodes), [n // 2 for n in nodes], [0] * len(nodes)):
        kc, vc, table = cache_of(keys, values, page_rows, -(-max(lengths) // page_rows) + 1, gen, heads_first, fill=5.0)
        expect = kc.clone(), vc.clone()
        out = Attention(kv_heads, kv_heads, head_dim, dtype, page_rows).accept(kc, vc, table, int32(lengths), int32(starts(nodes)), int32(flat(trees)), int32(last))
        for b, n in enumerate(nodes):
            path, before = path_of(trees[b], last[b]), lengths[b] - n
            assert int(out[b]) == before + len(path)
            for x, rows in zip(expect, (keys[b], values[b])):
                for at, i in enumerate(path):
                    x[int(table[b, (before + at) // page_rows]), (before + at) % page_rows] = rows[before + i].cuda()
        assert torch.equal(kc, expect[0]) and torch.equal(vc, expect[1])


def test_accept_wrong_tables():
    """What is wrong moves nothing and gives -1; rows whose places are in no page stay."""
    gen = torch.Generator().manual_seed(3)
    count, n, nodes = 8, 40, 8
    keys, values = ([normal(gen, n, 1, 64, dtype=BF16) for _ in range(count)] for _ in range(2))
    trees = [[-1, -1, 1, -1, 2, 4, 5, 6] for _ in range(count)]     # node 7 by 1, 2, 4, 5, 6
    trees[3][4] = 4
    trees[4][2] = -7
    kc, vc, table = cache_of(keys, values, 16, 3, gen)
    lengths, last = [n, nodes - 1, n, n, n, 49, n, n], [8, 7, -2, 7, 7, 7, 7, 7]
    table[6, 2] = -1      # places 32 .. 39: all of them
    before = kc.clone(), vc.clone()
    out = Attention(1, 1, 64, BF16, 16).accept(kc, vc, table, int32(lengths), int32(starts([nodes] * count)), int32(flat(trees)), int32(last))
    assert out.tolist() == [-1, -1, -1, -1, -1, -1, 38, 38]
    expect = before[0].clone(), before[1].clone()
    for x, rows in zip(expect, (keys[7], values[7])):
        for at, i in enumerate((1, 2, 4, 5, 6, 7)):
            x[int(table[7, 2]), at] = rows[32 + i].cuda()
    for x, y in zip((kc, vc), expect):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


# -- streams, strides, captures ---------------------------------------------------------------------------------------------------------
def operands(gen, heads=8, n=1500, nodes=40, d=64):
    k, v, q = normal(gen, n, 1, d, dtype=BF16), normal(gen, n, 1, d, dtype=BF16), normal(gen, nodes, heads, d, dtype=BF16)
    tree = random_tree(nodes, 4, gen)
    kc, vc, table = cache_of([k], [v], 64, 30, gen, fill=0.0)
    return q, k, v, tree, (kc, vc, table, int32([n]), int32([0, nodes]), int32(tree))


@pytest.mark.parametrize("heads", [1, 8])
def test_strides(heads):
    """Queries and results in a wider array, and heads before rows."""
    gen = torch.Generator().manual_seed(heads)
    q, k, v, tree, args = operands(gen, heads)
    want, bound = attend_seen(q, k, v, tree_mask(tree, 1500)[0], 1 / 8, BF16)
    attention = Attention(heads, 1, 64, BF16, 64)
    wide = torch.full((2, 40, heads + 3, 80), NAN, dtype=BF16, device="cuda")
    wide[0, :, 1:-2, 8:-8] = q.cuda()
    out = wide[1, :, 1:-2, 8:-8]
    assert attention.tree(wide[0, :, 1:-2, 8:-8], *args, out=out) is out
    assert_within(out, want, bound)
    assert bool(torch.isnan(wide[1, :, 0].float()).all()) and bool(torch.isnan(wide[1, :, :, :8].float()).all()) and bool(torch.isnan(wide[1, :, :, 72:].float()).all())
    turned = q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    assert_within(attention.tree(turned, *args), want, bound)


@pytest.mark.parametrize("heads", [1, 8])
@pytest.mark.parametrize("named", [False, True])
def test_first_call_in_a_capture(heads, named):
    """A handle whose first calls are captured: replays and eager calls beside them are right."""
    gen = torch.Generator().manual_seed(5)
    q, _, _, tree, args = operands(gen, heads)
    q, last = q.cuda(), int32([-1])
    want = Attention(heads, 1, 64, BF16, 64).tree(q, *args).clone()
    holders = torch.zeros(args[0].shape[0], dtype=torch.int32, device="cuda")
    holders[args[2][0, :24].long()] = 1
    tables = args[2], args[3], holders, int32([0, 0, -1])
    expect = [x.clone() for x in Attention(heads, 1, 64, BF16, 64).fork(*tables)]
    torch.cuda.synchronize()
    attention, side, graph = Attention(heads, 1, 64, BF16, 64), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    kw = dict(stream=side.cuda_stream) if named else {}
    with torch.cuda.graph(graph, stream=side):
        got = [attention.tree(q, *args, **kw), attention.accept(*args, last, **kw), *attention.fork(*tables, **kw)]
    for _ in range(3):
        for x in got:
            x.fill_(-9)
        others = [torch.full((1 << 22,), 3.0, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want) and got[1].tolist() == [1460]
        assert all(torch.equal(x, y) for x, y in zip(got[2:], expect))
        assert torch.equal(attention.tree(q, *args), want)
        torch.cuda.synchronize()
        assert all(bool((x == 3.0).all()) for x in others)


def test_calls_on_another_stream():
    """Results and workspaces are made while the current stream still reads memory that was freed on it, of their sizes."""
    gen = torch.Generator().manual_seed(1)
    q, _, _, tree, args = operands(gen)
    q = q.cuda()
    attention = Attention(8, 1, 64, BF16, 64)
    want = Attention(8, 1, 64, BF16, 64).tree(q, *args).clone()
    gate = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    side, ready, done = torch.cuda.Stream(), torch.cuda.Event(), torch.cuda.Event()
    ready.record()
    side.wait_event(ready)
    old = [torch.full((attention.tree_ws_bytes // 4,), 3.0, device="cuda"), torch.full_like(want, 3.0)]
    for _ in range(20):
        gate = (gate @ gate).clamp_(-1.0, 1.0)
    read = [x.clone() for x in old]     # queued behind that
    del old
    got = attention.tree(q, *args, stream=side.cuda_stream)
    done.record(side)
    torch.cuda.current_stream().wait_event(done)
    kept = got.clone()
    torch.cuda.synchronize()
    assert all(bool((x == 3.0).all()) for x in read) and torch.equal(kept, want)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("head_dim", [64, 40, 128, 72, 256, 200])
def test_many_trees_in_tiles(dtype, head_dim):
    """As many sequences as give every workgroup a block of rows and all of its keys, in tiles through LDS.  Rows behind the lengths hold NaN, and one branch of a tree infinities, which
    the other one does not see."""
    gen = torch.Generator().manual_seed(head_dim)
    count, nodes, bad = 40, 20, 7
    lengths = [max(nodes, int(x)) for x in torch.randint(1, 700, (count,), generator=gen)]
    lengths[bad] = 300
    keys, values = ([normal(gen, n, 4, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, count * nodes, 8, head_dim, dtype=dtype)
    trees = [random_tree(nodes, 4, gen) for _ in range(count)]
    trees[bad] = [-1, -1] + [i - 2 for i in range(2, nodes)]       # even nodes one branch, odd nodes the other
    trees[11][5] = 9                                               # a later one
    hidden = [x.clone() for x in values]
    hidden[bad][300 - nodes + 1::2] = INF
    kc, vc, table = cache_of(keys, hidden, 16, 44, gen, fill=NAN)
    args = (q.cuda(), kc, vc, table, int32(lengths), int32(starts([nodes] * count)), int32(flat(trees)))
    attention = Attention(8, 4, head_dim, dtype, 16)
    got = attention.tree(*args)
    assert torch.equal(got.nan_to_num(7.0), attention.tree(*args).nan_to_num(7.0))
    got = got.cpu()
    for b in range(count):
        rows = got[b * nodes:(b + 1) * nodes]
        if b == 11:
            wrong = [i for i in range(nodes) if i >= 5 and (i == 5 or 5 in path_of(trees[b][:5] + [-1] + trees[b][6:], i))]
            assert bool(torch.isnan(rows[wrong]).all()) and bool(torch.isfinite(rows[[i for i in range(nodes) if i not in wrong]]).all())
            continue
        want, bound = attend_seen(q[b * nodes:(b + 1) * nodes], keys[b], values[b], tree_mask(trees[b], lengths[b])[0], 1 / math.sqrt(head_dim), dtype)
        if b == bad:
            assert_within(rows[::2], want[::2], bound[::2], "the branch without infinities")
            assert not bool(torch.isfinite(rows[1::2]).any())
        else:
            assert_within(rows, want, bound, f"tree {b}")
