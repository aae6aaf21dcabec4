"""Pages of a cache on the GPU: the next batch from the present one, pages moved to the lowest numbers, copies, and a run of them with the attention that reads the cache."""
import random

import pytest
import torch

from paper_2311_09549_amd import binding as sc
from paper_2311_09549_amd.attention import Attention

import pages_reference as reference
from attention_masks import attend_seen, random_tree, path_of, through_window, tree_mask
from attention_reference import assert_within

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def int32(x, *shape):
    return torch.tensor(x, dtype=torch.int32, device="cuda").reshape(*shape) if shape else torch.tensor(x, dtype=torch.int32, device="cuda")


def batch_of(rng, sequences, columns, page_rows, spare, share=0.5, holes=0.0, outside=0):
    """Tables of sequences that share beginnings, with entries behind their lengths that are anything; `outside`: pages that sequences of no call hold."""
    lengths = [rng.choice((0, 1, page_rows, rng.randint(0, columns * page_rows), rng.randint(0, columns * page_rows), columns * page_rows)) for _ in range(sequences)]
    pages, at = [], 0
    for b, n in enumerate(lengths):
        row = []
        for c in range(reference.columns_of(n, page_rows)):
            if b and rng.random() < share and len(row) == c and c < lengths[b - 1] // page_rows and (c + 1) * page_rows <= n and (c == 0 or row[c - 1] == pages[b - 1][c - 1]):
                row.append(pages[b - 1][c])
            else:
                row.append(at)
                at += 1
        pages.append(row + [rng.choice((-1, 7, 2 ** 31 - 1, -2 ** 31)) for _ in range(columns - len(row))])
    total = max(1, at + spare + outside)      # a cache has a page
    number = list(range(total))
    rng.shuffle(number)
    holders = [0] * total
    for row, n in zip(pages, lengths):
        for c in range(reference.columns_of(n, page_rows)):
            row[c] = -1 if rng.random() < holes else number[row[c]]
            if row[c] >= 0:
                holders[row[c]] += 1
    for p in number[at:at + outside]:
        holders[p] = rng.randint(1, 3)
    return pages, lengths, holders


def held(pages, lengths, page_rows, count):
    out = [0] * count
    for row, n in zip(pages, lengths):
        for p in row[:reference.columns_of(max(n, 0), page_rows)]:
            if p >= 0:
                out[p] += 1
    return out


CASES = [
    # sequences, new ones, columns, page_rows, spare pages, outside
    (1, 1, 1, 16, 1, 0),
    (2, 4, 3, 16, 20, 0),
    (8, 8, 10, 16, 60, 5),
    (8, 20, 10, 16, 12, 5),        # not pages enough
    (30, 30, 5, 64, 0, 0),         # none but those that are given up
    (70, 300, 40, 16, 3000, 100),  # several workgroups of sequences
    (300, 70, 300, 16, 20000, 0),  # several blocks of pages, wide tables
    (5, 0, 4, 16, 3, 0),           # all are given up
    (0, 6, 4, 32, 9, 2),           # all are new
    (40, 1500, 6, 16, 12000, 0),   # more sequences than a workgroup has threads
    (1500, 40, 6, 16, 0, 0),
]


def test_tables_of_millions_of_pages():
    """More blocks of pages than a workgroup has threads: the free ones are far behind the first, and pages in use are spread over all of it."""
    count, columns = 4_300_000, 40
    attention = Attention(2, 1, 64, BF16, 16)
    rng = random.Random(1)
    pages = [[rng.randrange(count - 4_250_000, count) for _ in range(columns)] for _ in range(5)]
    lengths = [640, 633, 0, 17, 320]
    free = sorted(rng.sample(range(4_100_000, count), 500))
    holders = [1] * count
    for p in free:
        holders[p] = 0
    for row, n in zip(pages, lengths):
        for p in row[:reference.columns_of(n, 16)]:
            holders[p] = holders[p] or 1      # never below what the table holds
    parents, wanted = [1, 1, 4, -1, 3, 0], [633, 640, 600, 500, 16, 640]
    expect = reference.fork(pages, lengths, holders, parents, wanted, 16)
    got = attention.fork(int32(pages), int32(lengths), int32(holders), int32(parents), int32(wanted))
    for x, y in zip(got, expect):
        assert torch.equal(x, int32(y))
    sparse = [0] * count
    for p in rng.sample(range(count), 70_000):
        sparse[p] = rng.randint(1, 4)
    expect = reference.compact(pages, lengths, sparse, 16)
    got = attention.compact(int32(pages), int32(lengths), int32(sparse))
    for x, y in zip(got, expect):
        assert torch.equal(x, int32(y))


@pytest.mark.parametrize("sequences,new,columns,page_rows,spare,outside", CASES)
@pytest.mark.parametrize("window,sinks", [(None, 0), (20, 17), (1, 0)])
def test_fork(sequences, new, columns, page_rows, spare, outside, window, sinks):
    attention = Attention(2, 1, 64, BF16, page_rows, window=window, sinks=sinks)
    for seed in range(3):
        rng = random.Random(seed)
        pages, lengths, holders = batch_of(rng, sequences, columns, page_rows, spare, holes=0.05 * (seed == 2), outside=outside)
        parents = [rng.choice((-1, rng.randrange(sequences), rng.randrange(sequences), rng.randrange(sequences))) if sequences else -1 for _ in range(new)]
        wanted = [max(0, min(columns * page_rows, (lengths[p] if p >= 0 else 0) + rng.choice((0, 0, 1, rng.randint(-40, 40), rng.randint(-2 * page_rows, 2 * page_rows))))) for p in parents]
        for i in range(new):
            if rng.random() < 0.1:       # wrong ones
                if rng.random() < 0.5:
                    parents[i] = rng.choice((-2, sequences, 2 ** 31 - 1))
                else:
                    wanted[i] = rng.choice((-1, columns * page_rows + 1, 2 ** 31 - 1))
        if sequences > 2 and seed:
            lengths[1] = rng.choice((-1, columns * page_rows + 1))     # a wrong one holds nothing
            holders = [h + o for h, o in zip(held(pages, [0 if b == 1 else n for b, n in enumerate(lengths)], page_rows, len(holders)),
                                             [rng.randint(0, 1) * (rng.random() < 0.05) for _ in holders])]
        for want in (wanted, None):
            expect = reference.fork(pages or [[-1] * columns], lengths, holders, parents, want, page_rows, window, sinks)
            got = attention.fork(int32(pages, sequences, columns), int32(lengths, sequences), int32(holders), int32(parents, new), None if want is None else int32(want, new))
            for name, x, y, shape in zip(("pages", "lengths", "holders", "moves"), got, expect, ((new, columns), (new,), (len(holders),), (new, 3))):
                assert x.shape == shape and x.flatten().tolist() == [v for row in y for v in (row if isinstance(row, list) else [row])], f"{name}, seed {seed}"
            if not outside and not seed:
                assert got[2].tolist() == held(expect[0], expect[1], page_rows, len(holders))


def short_of_pages(seed, sequences, new, columns, page_rows, spare, outside):
    """A batch of which every sequence goes on, most of them by pages, with fewer of those than they take."""
    rng = random.Random(seed)
    pages, lengths, holders = batch_of(rng, sequences, columns, page_rows, spare, share=0.7, outside=outside)
    parents = list(range(sequences)) + [rng.randrange(sequences) for _ in range(new - sequences)]
    rng.shuffle(parents)
    wanted = [min(columns * page_rows, lengths[p] + rng.choice((0, 0, 1, page_rows, 3 * page_rows))) for p in parents]
    wanted = [rng.randint(0, n) if rng.random() < 0.2 else n for n in wanted]
    return pages, lengths, holders, parents, wanted


SHORT = [
    # sequences, new ones, columns, page_rows, spare pages, outside
    (8, 14, 8, 16, 1, 0),
    (40, 160, 12, 32, 10, 7),            # by one workgroup
    (300, 1300, 4, 16, 700, 0),          # more sequences than a workgroup has threads
    (60, 400, 15, 16, 20, 9000),         # more pages than it has room for
]


@pytest.mark.parametrize("sequences,new,columns,page_rows,spare,outside", SHORT)
@pytest.mark.parametrize("window,sinks", [(None, 0), (90, 17)])
def test_fork_without_pages_enough(sequences, new, columns, page_rows, spare, outside, window, sinks):
    """Sequences that find no free page hold nothing: with sequences before and behind them that are served, of kinds that share whole pages and that a page would have been left to."""
    attention = Attention(2, 1, 64, BF16, page_rows, window=window, sinks=sinks)
    short, between, sharing, keeping = 0, False, False, False
    for seed in range(6):
        pages, lengths, holders, parents, wanted = short_of_pages(seed, sequences, new, columns, page_rows, spare, outside)
        expect = reference.fork(pages, lengths, holders, parents, wanted, page_rows, window, sinks)
        refused = [i for i, n in enumerate(expect[1]) if n < 0]
        short += bool(refused)
        between |= bool(refused) and any(n >= 0 for n in expect[1][:refused[0]]) and any(n >= 0 for n in expect[1][refused[0]:])
        kept = [min(lengths[p], n) for p, n in zip(parents, wanted)]
        sharing |= any(kept[i] >= page_rows and any(parents[i] == parents[j] and kept[j] >= page_rows for j in range(new) if j not in refused) for i in refused)
        keeping |= any(kept[i] % page_rows and not any(pages[parents[i]][kept[i] // page_rows] in row[:reference.columns_of(max(n, 0), page_rows)] for row, n in zip(*expect[:2])) for i in refused)
        args = int32(pages), int32(lengths), int32(holders), int32(parents), int32(wanted)
        got = attention.fork(*args)
        for name, x, y in zip(("pages", "lengths", "holders", "moves"), got, expect):
            assert torch.equal(x, int32(y)), f"{name}, seed {seed}"
        if not outside:
            assert got[2].tolist() == held(expect[0], expect[1], page_rows, len(holders))
        again = attention.fork(*args, out=(*(torch.empty_like(x) for x in got[:2]), args[2], torch.empty_like(got[3])))     # holders in place
        assert all(torch.equal(x, y) for x, y in zip(got, again))
    assert short >= 3 and between and sharing and keeping


def test_fork_in_place_on_views_and_with_a_workspace():
    """Holders changed in place, tables with rows of a wider one, a workspace of the caller's whose contents do not matter."""
    rng = random.Random(4)
    attention = Attention(2, 1, 64, BF16, 16)
    pages, lengths, holders = batch_of(rng, 6, 5, 16, 30)
    parents = [0, 0, 3, 3, 5, -1]
    expect = reference.fork(pages, lengths, holders, parents, None, 16)
    wide, result = int32([[9] * 3 + row for row in pages]), torch.full((6, 11), 77, dtype=torch.int32, device="cuda")
    count = int32(holders)
    out = result[:, 4:9], torch.empty(6, dtype=torch.int32, device="cuda"), count, torch.empty(6, 3, dtype=torch.int32, device="cuda")
    workspace = torch.full((sc.attention_pages_workspace_bytes(len(holders), 6),), 255, dtype=torch.uint8, device="cuda")
    got = attention.fork(wide[:, 3:], int32(lengths), count, int32(parents), out=out, workspace=workspace)
    assert all(x is y for x, y in zip(got, out))
    assert result[:, 4:9].tolist() == expect[0] and out[1].tolist() == expect[1] and count.tolist() == expect[2] and out[3].tolist() == expect[3]
    assert bool((result[:, :4] == 77).all()) and bool((result[:, 9:] == 77).all())


@pytest.mark.parametrize("sequences,columns,page_rows,spare", [(1, 1, 16, 0), (1, 1, 16, 5), (4, 6, 16, 0), (6, 10, 32, 77), (40, 60, 16, 9000), (9, 5, 16, 4096), (0, 3, 16, 9)])
def test_compact(sequences, columns, page_rows, spare):
    attention = Attention(2, 1, 64, BF16, page_rows)
    for seed in range(4):
        rng = random.Random(seed)
        pages, lengths, holders = batch_of(rng, sequences, columns, page_rows, spare, holes=0.1 * (seed == 3), outside=5 if spare else 0)
        if seed == 2 and sequences > 1:
            lengths[0] = columns * page_rows + 1       # a wrong one: its entries stay
        expect = reference.compact(pages, lengths, holders, page_rows)
        args = int32(pages, sequences, columns), int32(lengths, sequences), int32(holders)
        got = attention.compact(*args)
        for x, y in zip(got, expect):
            assert x.flatten().tolist() == [v for row in y for v in (row if isinstance(row, list) else [row])]
        in_place = args[0].clone(), args[2].clone()
        moves = torch.empty(len(holders) // 2, 3, dtype=torch.int32, device="cuda")
        attention.compact(in_place[0], args[1], in_place[1], out=(*in_place, moves))
        assert torch.equal(in_place[0], got[0]) and torch.equal(in_place[1], got[1]) and torch.equal(moves, got[2])


@pytest.mark.parametrize("step", [0, 1, 3, 9])
def test_tables_whose_rows_share_memory(step):
    """Rows of a table that is only read may overlap or be the same; the tables that are made of it are whole."""
    columns, batch = 5, 4
    numbers = torch.arange(40, dtype=torch.int32, device="cuda") % 30
    pages = numbers.as_strided((batch, columns), (step, 1))
    lengths = int32([80, 64, 17, 33])
    holders = torch.zeros(37, dtype=torch.int32)
    for b, n in enumerate((5, 4, 2, 3)):
        for p in pages[b, :n].tolist():
            holders[p] += 1
    attention, holders = Attention(1, 1, 64, BF16, 16), holders.cuda()
    for a, b in zip(attention.compact(pages, lengths, holders), attention.compact(pages.contiguous(), lengths, holders)):
        assert torch.equal(a, b)
    parents = int32([3, 0, 1, 2])
    for a, b in zip(attention.fork(pages, lengths, holders, parents), attention.fork(pages.contiguous(), lengths, holders, parents)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("kv_heads,head_dim,page_rows,heads_first", [(1, 64, 16, False), (8, 128, 64, True), (3, 72, 32, False), (2, 8, 16, True), (16, 256, 128, False)])
def test_copy(dtype, kv_heads, head_dim, page_rows, heads_first):
    gen = torch.Generator(device="cuda").manual_seed(1)
    shape = (40, kv_heads, page_rows, head_dim) if heads_first else (40, page_rows, kv_heads, head_dim)
    caches = [torch.randn(shape, device="cuda", generator=gen).to(dtype) for _ in range(2)]
    caches = [x.transpose(1, 2) if heads_first else x for x in caches]
    moves = [[0, 20, page_rows], [39, 1, 1], [0, 2, page_rows - 1], [-1, 5, 7], [3, -1, 7], [40, 6, 2], [7, 40, 2], [8, 9, 0], [10, 11, -3], [12, 13, 2 ** 31 - 1], [14, 14, 3],
             [2 ** 31 - 1, 15, 3], [-2 ** 31, 16, 3]]
    expect = [x.clone() for x in caches]
    for x in expect:
        x[20], x[1, :1], x[2, :page_rows - 1], x[13] = x[0].clone(), x[39, :1].clone(), x[0, :page_rows - 1].clone(), x[12].clone()
    Attention(kv_heads, kv_heads, head_dim, dtype, page_rows).copy(*caches, int32(moves))
    for x, y in zip(caches, expect):
        assert torch.equal(x, y)


# -- all of them, as a program uses them ------------------------------------------------------------------------------------------------
class Model:
    """What the cache has to hold, row by row, beside the cache: rotated keys are not needed here (no rotation), so rows are what was appended."""

    def __init__(self, dtype, window, sinks, seed):
        self.rng, self.gen = random.Random(seed), torch.Generator().manual_seed(seed)
        self.dtype, self.window, self.sinks = dtype, window, sinks
        self.attention = Attention(4, 2, 64, dtype, 16, window=window, sinks=sinks)
        self.columns, count = 20, 120
        self.caches = [torch.full((count, 16, 2, 64), float("nan"), dtype=dtype, device="cuda") for _ in range(2)]
        self.pages, self.lengths = torch.zeros(0, self.columns, dtype=torch.int32, device="cuda"), int32([], 0)
        self.holders = torch.zeros(count, dtype=torch.int32, device="cuda")
        self.rows = []     # (keys, values) of each sequence

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen).to(self.dtype)

    def fork(self, parents, grow):
        lengths = [len(self.rows[p][0]) if p >= 0 else 0 for p in parents]
        wanted = [n + g for n, g in zip(lengths, grow)]
        self.pages, self.lengths, self.holders, moves = self.attention.fork(self.pages, self.lengths, self.holders, int32(parents, len(parents)), int32(wanted))
        self.attention.copy(*self.caches, moves)
        assert self.lengths.tolist() == wanted
        self.rows = [tuple(x[:w] for x in self.rows[p]) if p >= 0 else (torch.zeros(0, 2, 64, dtype=self.dtype),) * 2 for p, w in zip(parents, wanted)]

    def append(self, counts, parents=None):
        q, k, v = self.normal(sum(counts), 4, 64), self.normal(sum(counts), 2, 64), self.normal(sum(counts), 2, 64)
        row_start = int32([sum(counts[:b]) for b in range(len(counts) + 1)])
        self.attention.append(None, k.cuda(), v.cuda(), *self.caches, self.pages, self.lengths, row_start, parents=parents)
        at = 0
        for b, n in enumerate(counts):
            self.rows[b] = tuple(torch.cat([x, y[at:at + n]]) for x, y in zip(self.rows[b], (k, v)))
            at += n
        return q, row_start

    def check(self, got, q, masks):
        at = 0
        for (k, v), seen in zip(self.rows, masks):
            want, bound = attend_seen(q[at:at + len(seen)], k, v, seen, 1 / 8, self.dtype)
            assert_within(got[at:at + len(seen)], want, bound)
            at += len(seen)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("window,sinks", [(None, 0), (37, 5)])
def test_a_search_with_drafts(dtype, window, sinks):
    """Prompts, sequences that branch and end, drafted trees of which a path is accepted, single tokens, pages compacted on the way."""
    m = Model(dtype, window, sinks, 3)
    a = m.attention
    m.fork([-1, -1, -1], [70, 16, 33])
    q, row_start = m.append([70, 16, 33])
    m.check(a.prompt_paged(q.cuda(), *m.caches, m.pages, m.lengths, row_start), q, [through_window(torch.arange(n), n, window, sinks) for n in (70, 16, 33)])
    for step in range(8):
        batch = len(m.rows)
        parents = sorted(m.rng.randrange(batch) for _ in range(m.rng.choice((3, 4, 6))))
        nodes = [m.rng.randint(1, 9) for _ in parents]
        m.fork(parents, nodes)
        trees = [random_tree(n, 3, m.gen) for n in nodes]
        numbers = int32([p for t in trees for p in t])
        q, row_start = m.append(nodes, numbers)
        m.check(a.tree(q.cuda(), *m.caches, m.pages, m.lengths, row_start, numbers), q, [tree_mask(t, len(x[0]), window, sinks)[0] for t, x in zip(trees, m.rows)])
        last = [m.rng.randrange(-1, n) for n in nodes]
        after = a.accept(*m.caches, m.pages, m.lengths, row_start, numbers, int32(last))
        for b, (tree, node) in enumerate(zip(trees, last)):
            before = len(m.rows[b][0]) - len(tree)
            keep = list(range(before)) + [before + i for i in path_of(tree, node)]
            m.rows[b] = tuple(x[keep] for x in m.rows[b])
        assert after.tolist() == [len(x[0]) for x in m.rows]
        # rows that were drafted in vain are cut off, and a place for a token is made: lengths of the table's entries are still those of before
        wanted = (after + 1).to(torch.int32)
        cut = a.fork(m.pages, m.lengths, m.holders, int32(list(range(len(nodes)))), after)
        a.copy(*m.caches, cut[3])
        m.pages, m.lengths, m.holders, moves = a.fork(*cut[:3], int32(list(range(len(nodes)))), wanted)
        a.copy(*m.caches, moves)
        q, _ = m.append([1] * len(nodes))
        got = a.decode(q.cuda(), *m.caches, m.pages, m.lengths)
        m.check(got, q, [through_window(torch.tensor([len(x[0]) - 1]), len(x[0]), window, sinks) for x in m.rows])
        if step % 3 == 1:
            m.pages, m.holders, moves = a.compact(m.pages, m.lengths, m.holders)
            a.copy(*m.caches, moves)
            used = int((m.holders != 0).sum())
            assert bool((m.holders[:used] > 0).all()) and not bool(m.holders[used:].any())
        assert m.holders.tolist() == held(m.pages.tolist(), m.lengths.tolist(), 16, len(m.holders))


@pytest.mark.parametrize("window,sinks", [(None, 0), (37, 5)])
def test_pages_of_drafts_are_free_again(window, sinks):
    """Trees of many more nodes than are accepted, in the order of calls that the module gives: every page is held by the entries that lengths reach, and by nothing else."""
    rng, gen = random.Random(2), torch.Generator().manual_seed(2)
    attention = Attention(4, 2, 64, BF16, 16, window=window, sinks=sinks)
    caches = [torch.zeros(90, 16, 2, 64, dtype=BF16, device="cuda") for _ in range(2)]
    holders = torch.zeros(90, dtype=torch.int32, device="cuda")

    def fork(pages, lengths, holders, parents, wanted):
        pages, lengths, holders, moves = attention.fork(pages, lengths, holders, parents, wanted)
        attention.copy(*caches, moves)
        assert lengths.tolist() == wanted.tolist() and holders.tolist() == held(pages.tolist(), lengths.tolist(), 16, 90)
        return pages, lengths, holders

    pages, lengths, holders = fork(int32([], 0, 20), int32([], 0), holders, int32([-1] * 3), int32([15, 40, 1]))
    for step in range(5):
        nodes = [63, rng.randint(1, 63), 17]
        pages, lengths, holders = fork(pages, lengths, holders, int32([0, 1, 2]), lengths + int32(nodes))
        parents = int32([p for n in nodes for p in random_tree(n, 3, gen)])
        row_start, last = int32([0, nodes[0], nodes[0] + nodes[1], sum(nodes)]), int32([0, rng.randrange(-1, nodes[1]), 16])
        k = torch.randn(sum(nodes), 2, 64, generator=gen).to(BF16).cuda()
        attention.append(None, k, k, *caches, pages, lengths, row_start, parents=parents)
        accepted = attention.accept(*caches, pages, lengths, row_start, parents, last)
        order = [rng.randrange(3) for _ in range(3)]
        pages, lengths, holders = fork(pages, lengths, holders, int32(order), accepted[order])
        if step % 2:
            pages, holders, moves = attention.compact(pages, lengths, holders)
            attention.copy(*caches, moves)
            used = int((holders != 0).sum())
            assert holders.tolist() == held(pages.tolist(), lengths.tolist(), 16, 90) and not bool(holders[used:].any())


def test_a_step_in_a_graph():
    """Branching, drafting, attention, acceptance, captured once and replayed on other tables: each replay as the eager calls, bit for bit."""
    gen, rng = torch.Generator().manual_seed(10), random.Random(10)
    attention = Attention(8, 2, 128, BF16, 16, window=100, sinks=4)
    count, columns, new, nodes = 200, 30, 5, 6
    caches = [torch.randn(count, 16, 2, 128, generator=gen).to(BF16).cuda() for _ in range(2)]
    start = [x.clone() for x in caches]
    q, k, v = (torch.randn(new * nodes, h, 128, generator=gen).to(BF16).cuda() for h in (8, 2, 2))
    row_start = int32([nodes * b for b in range(new + 1)])

    def inputs(seed):
        r = random.Random(seed)
        pages, lengths, holders = batch_of(r, 4, columns - 1, 16, 0)
        pages = [row + [-1] for row in pages]
        holders += [0] * (count - len(holders))
        parents = [r.randrange(4) for _ in range(new)]
        wanted = [lengths[p] + nodes for p in parents]
        trees = [random_tree(nodes, 2, torch.Generator().manual_seed(seed + b)) for b in range(new)]
        return [int32(x) for x in (pages, lengths, holders, parents, wanted, [p for t in trees for p in t], [r.randrange(-1, nodes) for _ in range(new)])]

    def step(s):
        pages, lengths, holders, moves = attention.fork(*s[:5])
        attention.copy(*caches, moves)
        turned = attention.append(q, k, v, *caches, pages, lengths, row_start, parents=s[5])
        y = attention.tree(turned, *caches, pages, lengths, row_start, s[5])
        after = attention.accept(*caches, pages, lengths, row_start, s[5], s[6])
        return pages, lengths, holders, y, after

    def begin(state, seed):
        for x, y in zip(state, inputs(seed)):
            x.copy_(y)
        for x, y in zip(caches, start):
            x.copy_(y)

    state, eager = inputs(1), {}
    for seed in (1, 2, 3):
        begin(state, seed)
        result = step(state)
        torch.cuda.synchronize()
        eager[seed] = [x.clone() for x in result] + [x.clone() for x in caches]
        assert bool(torch.isfinite(eager[seed][3].float()).all()) and min(eager[seed][1].tolist()) >= nodes
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        result = step(state)
    for seed in (1, 2, 3, 1):
        begin(state, seed)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((*result, *caches), eager[seed]):
            assert torch.equal(x, y), seed
    side.wait_stream(torch.cuda.current_stream())
    begin(state, 2)
    torch.cuda.synchronize()
    before = torch.cuda.current_stream()
    pages, lengths, holders, moves = attention.fork(*state[:5], stream=side.cuda_stream)      # named, while another one is current
    before.wait_stream(side)
    assert torch.equal(pages, eager[2][0]) and torch.equal(lengths, eager[2][1]) and torch.equal(holders, eager[2][2])
