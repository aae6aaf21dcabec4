"""Attention through a sliding window whose first keys stay visible, on the GPU against the definition in 64 bits: packed prompts, prompts behind a cache and
single rows, at the edges of windows, tiles and pages; and that what a window hides is neither needed nor reaches a row."""
import math

import pytest
import torch

from paper_2311_09549_amd.attention import Attention

from attention_masks import attend_seen, through_window
from attention_reference import assert_within, cache_of

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


def check(got, q, k, v, position, window, sinks, dtype, what):
    want, bound = attend_seen(q, k, v, through_window(position, k.shape[0], window, sinks), 1 / math.sqrt(q.shape[2]), dtype)
    assert_within(got, want, bound, what)


def give_back(table, page_rows, lengths, rows, window, sinks, number=-7):
    """Entries of pages that no row sees become no pages."""
    for b, (n, r) in enumerate(zip(lengths, rows)):
        for c in range(table.shape[1]):
            if c * page_rows >= sinks and (c + 1) * page_rows <= n - r - window + 1:
                table[b, c] = number


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,head_dim,rows,window,sinks", [
    (1, 1, 64, [1], 1, 0),
    (2, 1, 64, [200], 1, 0),                             # a row sees itself alone
    (2, 1, 64, [200], 1, 1),
    (4, 2, 128, [1, 2, 15, 16, 17, 31, 32, 33, 500], 16, 0),
    (4, 2, 128, [300, 0, 700], 128, 4),
    (4, 2, 128, [300, 900], 127, 129),                   # first keys past a tile
    (8, 1, 128, [700], 129, 128),
    (6, 2, 64, [63, 0, 641, 129], 100, 17),
    (5, 5, 80, [370, 33], 33, 3),
    (4, 1, 96, [1000], 250, 0),
    (2, 1, 256, [300, 34], 40, 5),
    (2, 2, 200, [200], 64, 1),
    (2, 2, 8, [140, 5], 20, 2),
    (2, 1, 64, [300], 300, 2),                           # as long as the sequence, and longer
    (2, 1, 64, [300], 2 ** 30, 7),
    (2, 1, 64, [300], 5, 2 ** 30),
])
def test_prompt(dtype, heads, kv_heads, head_dim, rows, window, sinks):
    gen = torch.Generator().manual_seed(heads * 1000 + head_dim + window)
    total = sum(rows)
    q, k, v = (normal(gen, total, h, head_dim, dtype=dtype) for h in (heads, kv_heads, kv_heads))
    got = Attention(heads, kv_heads, head_dim, dtype, window=window, sinks=sinks).prompt(q.cuda(), k.cuda(), v.cuda(), int32(starts(rows))).cpu()
    at = 0
    for n in rows:
        check(got[at:at + n], q[at:at + n], k[at:at + n], v[at:at + n], torch.arange(n), window, sinks, dtype, f"sequence of {n}")
        at += n


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompt_split_over_the_gpu(dtype):
    """Few long blocks: keys are split, pieces joined."""
    gen = torch.Generator().manual_seed(4)
    n = 5000
    q, k, v = (normal(gen, n, h, 128, dtype=dtype) for h in (8, 1, 1))
    attention = Attention(8, 1, 128, dtype, window=3001, sinks=200)
    got = attention.prompt(q.cuda(), k.cuda(), v.cuda(), int32([0, n])).cpu()
    again = attention.prompt(q.cuda(), k.cuda(), v.cuda(), int32([0, n])).cpu()
    assert torch.equal(got, again)
    for lo, hi in ((0, 100), (2990, 3110), (4900, 5000)):
        check(got[lo:hi], q[lo:hi], k, v, torch.arange(lo, hi), 3001, 200, dtype, f"rows from {lo}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,head_dim,page_rows,lengths,rows,window,sinks,heads_first", [
    (2, 1, 64, 16, [1], [1], 1, 0, False),
    (4, 2, 128, 16, [100, 33, 0, 16, 17, 900], [70, 1, 0, 16, 5, 300], 40, 4, True),
    (4, 2, 128, 64, [2000, 700], [20, 100], 500, 0, False),
    (8, 1, 128, 16, [1500], [20], 100, 33, False),
    (3, 3, 72, 32, [500, 129], [7, 65], 63, 1, False),
    (2, 2, 256, 16, [290], [40], 100, 20, True),
    (2, 1, 64, 16, [5, 0, 20], [12, 3, 20], 4, 2, False),    # more rows than keys: rows before position 0 see nothing
    (2, 1, 64, 128, [3000], [257], 64, 130, False),
])
def test_prompt_paged(dtype, heads, kv_heads, head_dim, page_rows, lengths, rows, window, sinks, heads_first):
    """Pages behind every row's window are given back, and hold NaN where a tile reads them."""
    gen = torch.Generator().manual_seed(sum(lengths) + head_dim)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, sum(rows), heads, head_dim, dtype=dtype)
    columns = max(1, -(-max(lengths) // page_rows)) + 1
    kc, vc, table = cache_of(keys, values, page_rows, columns, gen, heads_first)
    whole = table.clone()
    attention = Attention(heads, kv_heads, head_dim, dtype, page_rows, window=window, sinks=sinks)
    for number in (-7, 2 ** 31 - 1):
        table = whole.clone()
        give_back(table, page_rows, lengths, rows, window, sinks, number)
        got = attention.prompt_paged(q.cuda(), kc, vc, table, int32(lengths), int32(starts(rows))).cpu()
        at = 0
        for b, n in enumerate(rows):
            check(got[at:at + n], q[at:at + n], keys[b], values[b], torch.arange(lengths[b] - n, lengths[b]), window, sinks, dtype, f"sequence {b}")
            at += n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,head_dim,page_rows,lengths,window,sinks,heads_first", [
    (1, 1, 64, 16, [1], 1, 0, False),
    (4, 2, 128, 16, [1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 0, 255, 1000], 16, 0, False),
    (4, 2, 128, 16, [1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 0, 255, 1000], 33, 5, True),
    (8, 8, 64, 32, [500, 3], 100, 33, True),
    (5, 1, 80, 16, [200, 0, 0, 77], 1, 1, False),
    (20, 1, 128, 64, [300, 40], 31, 16, False),          # more heads on a key head than a tile has
    (35, 1, 64, 16, [150], 20, 17, True),
    (6, 2, 256, 16, [130, 700], 100, 15, False),
    (2, 2, 136, 16, [90, 900], 700, 0, False),
    (2, 1, 8, 16, [140], 10, 3, False),
    (4, 1, 128, 128, [9000], 4000, 4, False),            # one long sequence, split over many workgroups
    (20, 1, 64, 64, [3000, 40, 0, 1500], 1000, 100, False),
    (2, 1, 256, 16, [2000, 5], 900, 33, True),
    (4, 1, 128, 16, [9000], 2 ** 30, 2 ** 30, False),
])
def test_decode(dtype, heads, kv_heads, head_dim, page_rows, lengths, window, sinks, heads_first):
    gen = torch.Generator().manual_seed(sum(lengths) + heads)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, len(lengths), heads, head_dim, dtype=dtype)
    columns = max(1, -(-max(lengths) // page_rows)) + 1
    kc, vc, table = cache_of(keys, values, page_rows, columns, gen, heads_first)
    give_back(table, page_rows, lengths, [1] * len(lengths), window, sinks)
    attention = Attention(heads, kv_heads, head_dim, dtype, page_rows, window=window, sinks=sinks)
    workspace = torch.full((attention.ws_bytes // 4,), NAN, device="cuda")   # its contents do not matter
    args = (q.cuda(), kc, vc, table, int32(lengths))
    got = attention.decode(*args, workspace=workspace)
    assert torch.equal(got, attention.decode(*args))
    for b, n in enumerate(lengths):
        check(got[b:b + 1], q[b:b + 1], keys[b], values[b], torch.tensor([n - 1]), window, sinks, dtype, f"length {n}")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 128, 256])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_hidden_keys_reach_nothing(dtype, head_dim, bad):
    """Keys and values between the first ones and the window hold infinities or NaN, as far as the tile that the window begins in."""
    gen = torch.Generator().manual_seed(head_dim)
    n, rows, window, sinks = 400, 60, 100, 5
    q, k, v = normal(gen, n, 2, head_dim, dtype=dtype), normal(gen, n, 1, head_dim, dtype=dtype), normal(gen, n, 1, head_dim, dtype=dtype)
    bad_k, bad_v = k.clone(), v.clone()
    for x in (bad_k, bad_v):
        x[sinks:n - rows - window + 1] = bad     # the first of the last `rows` rows sees keys from there on
    attention = Attention(2, 1, head_dim, dtype, 16, window=window, sinks=sinks)
    position = torch.arange(n - rows, n)
    packed = attention.prompt(q.cuda(), bad_k.cuda(), bad_v.cuda(), int32([0, n])).cpu()[n - rows:]
    check(packed, q[n - rows:], k, v, position, window, sinks, dtype, "packed")
    kc, vc, table = cache_of([bad_k], [bad_v], 16, n // 16 + 1, gen, fill=bad)
    paged = attention.prompt_paged(q[n - rows:].cuda(), kc, vc, table, int32([n]), int32([0, rows])).cpu()
    check(paged, q[n - rows:], k, v, position, window, sinks, dtype, "paged")
    one = attention.tree(q[n - rows:].cuda(), kc, vc, table, int32([n]), int32([0, rows])).cpu()
    check(one, q[n - rows:], k, v, position, window, sinks, dtype, "as a chain")
    for x in (kc, vc):
        for j in range(n - rows - window + 1, n - window):
            x[int(table[0, j // 16]), j % 16] = bad
    last = attention.decode(q[n - 1:].cuda(), kc, vc, table, int32([n])).cpu()
    check(last, q[n - 1:], k, v, position[-1:], window, sinks, dtype, "decode")
    # a window of more keys than one workgroup takes
    n, window, sinks = 1500, 700, 50
    q, k, v = normal(gen, 9, 2, head_dim, dtype=dtype), normal(gen, n, 1, head_dim, dtype=dtype), normal(gen, n, 1, head_dim, dtype=dtype)
    bad_k, bad_v = k.clone(), v.clone()
    for x in (bad_k, bad_v):
        x[sinks:n - window] = bad
    kc, vc, table = cache_of([bad_k], [bad_v], 16, n // 16 + 1, gen, fill=bad)
    attention = Attention(2, 1, head_dim, dtype, 16, window=window, sinks=sinks)
    last = attention.decode(q[8:].cuda(), kc, vc, table, int32([n])).cpu()
    check(last, q[8:], k, v, torch.tensor([n - 1]), window, sinks, dtype, "decode of many keys")
    for x in (kc, vc):
        for j in range(n - window - 8, n - window):
            x[int(table[0, j // 16]), j % 16] = (k if x is kc else v)[j].cuda()
    chain = attention.tree(q.cuda(), kc, vc, table, int32([n]), int32([0, 9])).cpu()
    check(chain, q, k, v, torch.arange(n - 9, n), window, sinks, dtype, "chain behind many keys")


@pytest.mark.parametrize("dtype", DTYPES)
def test_seen_infinities_stay(dtype):
    """A value of +infinity in one element reaches the rows whose window has it, and no others."""
    gen = torch.Generator().manual_seed(1)
    n, window = 300, 40
    q, k, v = normal(gen, n, 1, 64, dtype=dtype), normal(gen, n, 1, 64, dtype=dtype), normal(gen, n, 1, 64, dtype=dtype)
    bad = v.clone()
    bad[150, 0, 9] = INF
    attention = Attention(1, 1, 64, dtype, 16, window=window)
    kc, vc, table = cache_of([k], [bad], 16, n // 16 + 1, gen)
    want, bound = attend_seen(q, k, v, through_window(torch.arange(n), n, window, 0), 1 / 8, dtype)
    sees = (torch.arange(n) >= 150) & (torch.arange(n) < 150 + window)
    for got in (attention.prompt(q.cuda(), k.cuda(), bad.cuda(), int32([0, n])).cpu(), attention.tree(q.cuda(), kc, vc, table, int32([n]), int32([0, n])).cpu()):
        assert bool((got[sees][:, 0, 9] == INF).all())
        others = torch.arange(64) != 9
        assert_within(got[..., others], want[..., others], bound[..., others])
        assert_within(got[~sees], want[~sees], bound[~sees])


def test_wrong_tables():
    """Wrong lengths, and wrong pages among those that are seen, make NaN of their rows and leave the others as they are."""
    gen = torch.Generator().manual_seed(7)
    n, window, sinks = 300, 64, 3
    keys, values = ([normal(gen, n, 2, 64, dtype=BF16) for _ in range(6)] for _ in range(2))
    q = normal(gen, 6, 4, 64, dtype=BF16)
    kc, vc, table = cache_of(keys, values, 16, 19, gen)
    table[1, (n - 1 - 20) // 16] = -1                 # in the window
    table[2, 0] = kc.shape[0]                         # of the first keys
    table[3, 5] = -1                                  # in the gap: not read
    lengths = int32([n, n, n, n, -3, 19 * 16 + 1])
    attention = Attention(4, 2, 64, BF16, 16, window=window, sinks=sinks)
    for got in (attention.decode(q.cuda(), kc, vc, table, lengths).cpu(), attention.prompt_paged(q.cuda(), kc, vc, table, lengths, int32(range(7))).cpu()):
        for b in (0, 3):
            check(got[b:b + 1], q[b:b + 1], keys[b], values[b], torch.tensor([n - 1]), window, sinks, BF16, f"sequence {b}")
        assert bool(torch.isnan(got[[1, 2, 4, 5]]).all())


def test_a_window_of_everything_is_none():
    """Rows whose window has the whole sequence: as without one, to rounding; and tokens one by one as the prompt at once."""
    gen = torch.Generator().manual_seed(13)
    n, window = 90, 25
    q, k, v = (normal(gen, n, h, 64, dtype=F32).cuda() for h in (4, 2, 2))
    attention = Attention(4, 2, 64, F32, 16, window=window, sinks=2)
    kc, vc = (torch.full((8, 16, 2, 64), NAN, device="cuda") for _ in range(2))
    table = int32([[7, 2, 0, 5, 1, 3]])
    parts = []
    for lo, hi in ((0, 37), (37, n - 3)):
        turned = attention.append(q[lo:hi], k[lo:hi], v[lo:hi], kc, vc, table, int32([hi]), int32([0, hi - lo]))
        parts.append(attention.prompt_paged(turned, kc, vc, table, int32([hi]), int32([0, hi - lo])))
    for i in range(n - 3, n):
        turned = attention.append(q[i:i + 1], k[i:i + 1], v[i:i + 1], kc, vc, table, int32([i + 1]))
        parts.append(attention.decode(turned, kc, vc, table, int32([i + 1])))
    check(torch.cat(parts).cpu(), q.cpu(), k.cpu(), v.cpu(), torch.arange(n), window, 2, F32, "step by step")
    plain, wide = Attention(4, 2, 64, F32, 16), Attention(4, 2, 64, F32, 16, window=n)
    got = wide.prompt(q, k, v, int32([0, n])).cpu()
    check(got, q.cpu(), k.cpu(), v.cpu(), torch.arange(n), None, 0, F32, "wide")
    check(plain.prompt(q, k, v, int32([0, n])).cpu(), q.cpu(), k.cpu(), v.cpu(), torch.arange(n), n, 0, F32, "none")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim", [64, 72, 128, 200])
def test_strides_and_rows_of_no_sequence(dtype, head_dim):
    """Rows in a wider array and heads before rows; rows before the first sequence and behind the last are not written, and what they hold does not matter."""
    gen = torch.Generator().manual_seed(head_dim)
    rows, window, sinks = [150, 0, 333], 90, 5
    total = 7 + sum(rows) + 9
    attention = Attention(4, 2, head_dim, dtype, window=window, sinks=sinks)
    q, k, v = (normal(gen, total, h, head_dim, dtype=dtype) for h in (4, 2, 2))
    for x in (q, k, v):
        x[:7], x[-9:] = NAN, NAN
    for how in ("wide", "heads"):
        if how == "wide":
            views = []
            for x in (q, k, v, torch.full_like(q, 7.0)):
                wide = torch.full((total, x.shape[1] + 3, head_dim + 16), NAN, dtype=dtype, device="cuda")
                wide[:, 1:-2, 8:-8] = x.cuda()
                views.append(wide[:, 1:-2, 8:-8])
        else:
            views = [x.cuda().transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, torch.full_like(q, 7.0))]
        got = attention.prompt(*views[:3], int32([7, 157, 157, 490]), out=views[3]).cpu()
        assert bool((got[:7] == 7.0).all()) and bool((got[490:] == 7.0).all())
        for at, n in ((7, 150), (157, 333)):
            check(got[at:at + n], q[at:at + n], k[at:at + n], v[at:at + n], torch.arange(n), window, sinks, dtype, f"{how}, sequence of {n}")


def test_shared_heads_of_stride_zero():
    """Keys and values of a head that all share, by a stride of 0."""
    gen = torch.Generator().manual_seed(3)
    q, k, v = normal(gen, 200, 4, 64, dtype=BF16), normal(gen, 200, 1, 64, dtype=BF16), normal(gen, 200, 1, 64, dtype=BF16)
    got = Attention(4, 2, 64, BF16, window=30).prompt(q.cuda(), k.cuda().expand(200, 2, 64), v.cuda().expand(200, 2, 64), int32([0, 200])).cpu()
    check(got, q, k, v, torch.arange(200), 30, 0, BF16, "shared")


def test_more_sequences_than_are_counted():
    """Packed prompts of more sequences than a block is counted among."""
    gen = torch.Generator().manual_seed(9)
    rows = [int(x) for x in torch.randint(0, 6, (1500,), generator=gen)]
    rows[700] = 300
    total = sum(rows)
    q, k, v = (normal(gen, total, h, 64, dtype=BF16) for h in (2, 1, 1))
    got = Attention(2, 1, 64, BF16, window=20, sinks=1).prompt(q.cuda(), k.cuda(), v.cuda(), int32(starts(rows))).cpu()
    at = 0
    for b, n in enumerate(rows):
        if n and (b % 50 == 0 or n > 5 or b > 1490):
            check(got[at:at + n], q[at:at + n], k[at:at + n], v[at:at + n], torch.arange(n), 20, 1, BF16, f"sequence {b}")
        at += n


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_many_sequences(dtype):
    """More sequences than a wavefront has lanes, and more units than workgroups: shares that begin and end anywhere."""
    gen = torch.Generator().manual_seed(5)
    lengths = [int(x) for x in torch.randint(0, 1500, (300,), generator=gen)]
    keys, values = ([normal(gen, n, 2, 64, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, 300, 4, 64, dtype=dtype)
    kc, vc, table = cache_of(keys, values, 64, 24, gen)
    got = Attention(4, 2, 64, dtype, 64, window=700, sinks=3).decode(q.cuda(), kc, vc, table, int32(lengths)).cpu()
    for b, n in enumerate(lengths):
        check(got[b:b + 1], q[b:b + 1], keys[b], values[b], torch.tensor([n - 1]), 700, 3, dtype, f"sequence {b} of length {n}")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,head_dim", [(8, 64), (8, 40), (4, 128), (8, 104), (4, 256), (2, 200)])
def test_prompt_in_pages_split_over_the_gpu(dtype, heads, head_dim):
    """Few rows behind many keys in pages: shares that cut blocks of rows, on both sides of the gap.  Pages behind every row's window are given back; what no row sees of the others holds
    NaN; a wrong page among those that are seen makes NaN of its sequence alone."""
    gen = torch.Generator().manual_seed(head_dim)
    lengths, rows, window, sinks = [6001, 5500, 5800], [40, 33, 7], 3000, 100
    keys, values = ([normal(gen, n, 1, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, sum(rows), heads, head_dim, dtype=dtype)
    hidden = [[x.clone() for x in side] for side in (keys, values)]
    for side in hidden:
        for x, n, r in zip(side, lengths, rows):
            x[sinks:n - r - window + 1] = NAN
    kc, vc, table = cache_of(*hidden, 16, -(-max(lengths) // 16), gen, fill=NAN)
    give_back(table, 16, lengths, rows, window, sinks)
    table[2, 5700 // 16] = -1
    attention = Attention(heads, 1, head_dim, dtype, 16, window=window, sinks=sinks)
    workspace = torch.full((attention.prompt_ws_bytes // 4,), NAN, device="cuda")   # its contents do not matter
    args = (q.cuda(), kc, vc, table, int32(lengths), int32(starts(rows)))
    got = attention.prompt_paged(*args, workspace=workspace).cpu()
    at = 0
    for b, n in enumerate(rows):
        if b == 2:
            assert bool(torch.isnan(got[at:at + n]).all())
        else:
            check(got[at:at + n], q[at:at + n], keys[b], values[b], torch.arange(lengths[b] - n, lengths[b]), window, sinks, dtype, f"sequence {b}")
        at += n
    again = attention.prompt_paged(*args).cpu()
    assert torch.equal(got[:73], again[:73]) and bool(torch.isnan(again[73:]).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,head_dim", [(4, 64), (4, 56), (4, 72), (4, 256), (2, 200)])
def test_prompts_of_other_heads_split_over_the_gpu(dtype, heads, head_dim):
    """As test_prompt_split_over_the_gpu, in tiles of other sizes; keys in the middle hold NaN, which the rows that are looked at do not see."""
    gen = torch.Generator().manual_seed(head_dim)
    n, window, sinks = 4000, 2001, 200
    q, k, v = (normal(gen, n, h, head_dim, dtype=dtype) for h in (heads, 1, 1))
    bad_k, bad_v = k.clone(), v.clone()
    for x in (bad_k, bad_v):
        x[1000:1400] = NAN
    attention = Attention(heads, 1, head_dim, dtype, window=window, sinks=sinks)
    got = attention.prompt(q.cuda(), bad_k.cuda(), bad_v.cuda(), int32([0, n])).cpu()
    for lo, hi in ((0, 100), (900, 1000), (1400 + window - 1, 3500), (3900, 4000)):
        check(got[lo:hi], q[lo:hi], k, v, torch.arange(lo, hi), window, sinks, dtype, f"rows from {lo}")
    assert bool(torch.isnan(got[1000:1400 + window - 1]).all())


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(16, 4, 64), (16, 4, 72), (16, 2, 256)])
def test_many_rows_in_fp32(heads, kv_heads, head_dim):
    """As many rows and heads as make a wavefront take 16 rows and all their keys by itself, packed and in pages; infinities where nobody looked at sees them."""
    gen = torch.Generator().manual_seed(head_dim)
    rows, window, sinks = [4050, 0, 33], 130, 5
    total = sum(rows)
    q, k, v = (normal(gen, total, h, head_dim) for h in (heads, kv_heads, kv_heads))
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[1000:1050], bad_v[1000:1050] = NAN, INF
    attention = Attention(heads, kv_heads, head_dim, F32, 32, window=window, sinks=sinks)
    places = [(0, 0, 40), (0, 960, 1000), (0, 1050 + window - 1, 1230), (0, 3990, 4050), (4050, 0, 33)]

    def look(got):
        for begin, lo, hi in places:
            n = rows[0] if begin == 0 else rows[2]
            check(got[begin + lo:begin + hi], q[begin + lo:begin + hi], k[begin:begin + n], v[begin:begin + n], torch.arange(lo, hi), window, sinks, F32, f"rows from {begin + lo}")

    look(attention.prompt(q.cuda(), bad_k.cuda(), bad_v.cuda(), int32(starts(rows))).cpu())
    caches = [[x[:4050], x[:0], x[4050:]] for x in (bad_k, bad_v)]
    kc, vc, table = cache_of(*caches, 32, 128, gen, fill=NAN)
    look(attention.prompt_paged(q.cuda(), kc, vc, table, int32(rows), int32(starts(rows))).cpu())
