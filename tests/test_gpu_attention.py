"""Attention on the GPU against the definition in 64 bits: prompts (packed and in pages), single rows over a paged cache, and the append that
fills it, at the lengths, masks, layouts and wrong tables where they can go wrong."""
import math

import pytest
import torch

from paper_2311_09549_amd import binding as sc
from paper_2311_09549_amd.attention import Attention

from attention_reference import assert_within, attend, cache_of, half_step, rotated

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN, INF = float("nan"), float("inf")


def normal(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return out


def by_strides(x, how):
    """The same values at other strides: rows in a wider array, or heads before rows."""
    if how == "wide":
        wide = torch.full((x.shape[0], x.shape[1] + 3, x.shape[2] + 16), NAN, dtype=x.dtype, device=x.device)
        wide[:, 1:-2, 8:-8] = x
        return wide[:, 1:-2, 8:-8]
    if how == "heads":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    return x


# -- prompts, packed -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv_heads,head_dim,rows,causal,how", [
    (1, 1, 64, [1], True, ""),
    (4, 2, 128, [1, 2, 15, 16, 17, 31, 32, 33], True, ""),
    (6, 2, 64, [63, 0, 65, 0, 0, 129], True, "wide"),
    (3, 1, 128, [130], False, "heads"),
    (2, 2, 8, [40, 5], True, ""),
    (5, 5, 80, [70, 33], False, ""),
    (4, 1, 96, [100], True, "wide"),
    (2, 1, 256, [67, 34], True, ""),
    (2, 2, 200, [48], True, "heads"),
    (8, 1, 128, [300], True, ""),
])
def test_prompt(dtype, heads, kv_heads, head_dim, rows, causal, how):
    gen = torch.Generator().manual_seed(heads * 1000 + head_dim + len(rows))
    total = sum(rows)
    q, k, v = (normal(gen, total, h, head_dim, dtype=dtype) for h in (heads, kv_heads, kv_heads))
    attention = Attention(heads, kv_heads, head_dim, dtype, causal=causal)
    got = attention.prompt(*(by_strides(x.cuda(), how) for x in (q, k, v)), int32(starts(rows)))
    torch.cuda.synchronize()
    at = 0
    for n in rows:
        sees = torch.arange(1, n + 1) if causal else torch.full((n,), n)
        want, bound = attend(q[at:at + n], k[at:at + n], v[at:at + n], sees, 1 / math.sqrt(head_dim), dtype)
        assert_within(got[at:at + n], want, bound, f"sequence of {n}")
        at += n


def test_prompt_scale_and_large_scores():
    gen = torch.Generator().manual_seed(3)
    q, k, v = normal(gen, 90, 2, 64, dtype=F16, scale=8.0), normal(gen, 90, 1, 64, dtype=F16, scale=8.0), normal(gen, 90, 1, 64, dtype=F16)
    got = Attention(2, 1, 64, F16, scale=0.25).prompt(q.cuda(), k.cuda(), v.cuda(), int32([0, 90]))
    want, bound = attend(q, k, v, torch.arange(1, 91), 0.25, F16)
    assert_within(got, want, bound)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_prompt_many_small_weights(dtype):
    """One key far above the others: weights that fp16 could not hold beside 1 still add up to a good part of the row."""
    n, d = 2000, 64
    q, k = torch.zeros(n, 1, d), torch.zeros(n, 1, d)
    q[..., 0] = 1.0
    k[0, 0, 0] = 16.0   # the others have e^-16 = 2^-23 of its weight each
    v = torch.ones(n, 1, d)
    v[0] = 0.0
    q, k, v = q.to(dtype), k.to(dtype), (v * 1024).to(dtype)
    got = Attention(1, 1, d, dtype, scale=1.0).prompt(q.cuda(), k.cuda(), v.cuda(), int32([0, n]))
    want, bound = attend(q[-1:], k, v, torch.tensor([n]), 1.0, dtype)
    assert float(want.abs().max()) > 0.2
    assert_within(got[-1:], want, bound)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("head_dim", [64, 128, 256])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_prompt_hidden_keys_reach_nothing(dtype, head_dim, bad):
    """What a row may not see (later keys of its sequence, rows of no sequence, rows of the next sequence) holds infinities or NaN."""
    gen = torch.Generator().manual_seed(head_dim)
    rows, total = [37, 70], 130   # sequences at rows 5..41 and 42..111; the rest belongs to none
    q, k, v = normal(gen, total, 2, head_dim, dtype=dtype), normal(gen, total, 1, head_dim, dtype=dtype), normal(gen, total, 1, head_dim, dtype=dtype)
    bad_k, bad_v = k.clone(), v.clone()
    for x in (bad_k, bad_v):
        x[:5], x[112:] = bad, bad
        x[42 + 40] = bad          # rows from 40 on of the second sequence see it
        x[42 + 69, 0, 3] = bad    # its last row alone
    out = torch.full((total, 2, head_dim), 7.0, dtype=dtype, device="cuda")
    Attention(2, 1, head_dim, dtype).prompt(q.cuda(), bad_k.cuda(), bad_v.cuda(), int32([5, 42, 112]), out=out)
    got = out.cpu()
    assert bool((got[:5] == 7.0).all()) and bool((got[112:] == 7.0).all())   # rows of no sequence are not written
    for at, n, clean in ((5, 37, 37), (42, 70, 40)):
        want, bound = attend(q[at:at + clean], k[at:at + n], v[at:at + n], torch.arange(1, clean + 1), 1 / math.sqrt(head_dim), dtype)
        assert_within(got[at:at + clean], want, bound)
    seen = got[42 + 40:112]
    if math.isnan(bad):
        assert bool(torch.isnan(seen).all())
    else:
        assert not bool(torch.isfinite(seen).all(dim=-1).any())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prompt_infinite_values_stay_infinite(dtype):
    """Keys are finite, one value is +infinity in one element: rows that see it have +infinity there and are as ever elsewhere."""
    gen = torch.Generator().manual_seed(1)
    q, k, v = normal(gen, 64, 1, 64, dtype=dtype), normal(gen, 64, 1, 64, dtype=dtype), normal(gen, 64, 1, 64, dtype=dtype)
    bad = v.clone()
    bad[50, 0, 9] = INF
    bad[60, 0, 9] = -INF
    got = Attention(1, 1, 64, dtype).prompt(q.cuda(), k.cuda(), bad.cuda(), int32([0, 64])).cpu()
    want, bound = attend(q, k, v, torch.arange(1, 65), 1 / 8, dtype)
    assert bool((got[50:60, 0, 9] == INF).all()) and bool(torch.isnan(got[60:, 0, 9]).all())
    others = torch.arange(64) != 9
    assert_within(got[..., others], want[..., others], bound[..., others])
    assert_within(got[:50], want[:50], bound[:50])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_lowest_scores(dtype):
    """Scores of the type's lowest value are scores like others; rows of -infinity alone give +0."""
    d = 64
    q, k, v = torch.zeros(20, 1, d, dtype=dtype), torch.zeros(20, 1, d, dtype=dtype), torch.ones(20, 1, d, dtype=dtype)
    q[..., 0] = 1.0
    k[:, 0, 0] = torch.finfo(dtype).min
    got = Attention(1, 1, d, dtype, scale=1.0).prompt(q.cuda(), k.cuda(), v.cuda(), int32([0, 20])).cpu()
    assert bool((got == 1.0).all())
    k[:, 0, 0] = -INF
    got = Attention(1, 1, d, dtype, scale=1.0).prompt(q.cuda(), k.cuda(), v.cuda(), int32([0, 20])).cpu()
    assert bool((got == 0.0).all()) and not bool(torch.signbit(got).any())


# -- prompts behind a cache --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv_heads,head_dim,page_rows,lengths,rows,causal,heads_first", [
    (2, 1, 64, 16, [1], [1], True, False),
    (4, 2, 128, 16, [100, 33, 0, 16, 17], [70, 1, 0, 16, 5], True, True),
    (3, 3, 72, 32, [50, 129], [7, 65], False, False),
    (8, 1, 128, 64, [300], [20], True, False),
    (2, 2, 256, 16, [90], [40], True, True),
    (2, 1, 64, 16, [5, 0, 20], [12, 3, 20], True, False),    # more rows than keys: rows before position 0 see nothing
])
def test_prompt_paged(dtype, heads, kv_heads, head_dim, page_rows, lengths, rows, causal, heads_first):
    gen = torch.Generator().manual_seed(sum(lengths) + head_dim)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, sum(rows), heads, head_dim, dtype=dtype)
    columns = max(1, -(-max(lengths) // page_rows)) + 1
    kc, vc, table = cache_of(keys, values, page_rows, columns, gen, heads_first)
    got = Attention(heads, kv_heads, head_dim, dtype, page_rows, causal=causal).prompt_paged(q.cuda(), kc, vc, table, int32(lengths), int32(starts(rows))).cpu()
    at = 0
    for b, n in enumerate(rows):
        position = torch.arange(lengths[b] - n, lengths[b])
        sees = position + 1 if causal else torch.full((n,), lengths[b])
        want, bound = attend(q[at:at + n], keys[b], values[b], sees, 1 / math.sqrt(head_dim), dtype)
        assert_within(got[at:at + n], want, bound, f"sequence {b}")
        blind = sees <= 0
        assert bool((got[at:at + n][blind] == 0).all())
        at += n


def test_prompt_paged_wrong_tables():
    """Wrong lengths and pages make NaN of the rows that they concern and leave the others as they are."""
    gen = torch.Generator().manual_seed(11)
    lengths = [60, 60, 60, 60, 60]
    keys, values = ([normal(gen, 60, 1, 64, dtype=BF16) for _ in lengths] for _ in range(2))
    q = normal(gen, 10 * len(lengths), 2, 64, dtype=BF16)
    kc, vc, table = cache_of(keys, values, 16, 4, gen)
    table[1, 2] = kc.shape[0]
    table[2, 0] = -5
    got = Attention(2, 1, 64, BF16, 16).prompt_paged(q.cuda(), kc, vc, table, int32([60, 60, 60, -1, 65]), int32(starts([10] * 5))).cpu()
    want, bound = attend(q[:10], keys[0], values[0], torch.arange(51, 61), 1 / 8, BF16)
    assert_within(got[:10], want, bound)
    assert bool(torch.isnan(got[10:]).all())


def test_prompt_wrong_row_starts():
    """Row starts out of range and out of order: nothing outside is read, rows of the good sequence are right."""
    gen = torch.Generator().manual_seed(12)
    q, k, v = (normal(gen, 100, 1, 64, dtype=BF16) for _ in range(3))
    attention = Attention(1, 1, 64, BF16)
    for table in ([0, 30, -7, 100], [0, 30, 500, 2 ** 31 - 1], [-9, 30, 30, 20], [100, 0, 0, 0]):
        out = attention.prompt(q.cuda(), k.cuda(), v.cuda(), int32(table), out=torch.zeros(100, 1, 64, dtype=BF16, device="cuda"))
        torch.cuda.synchronize()
        if table[0] <= 0 and table[1] == 30:
            want, bound = attend(q[:30], k[:30], v[:30], torch.arange(1, 31), 1 / 8, BF16)
            assert bool(torch.isfinite(out.float()).all())
            assert_within(out[:20], want[:20], bound[:20])


# -- one row per sequence ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv_heads,head_dim,page_rows,lengths,heads_first", [
    (1, 1, 64, 16, [1], False),
    (4, 2, 128, 16, [1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 0, 255], False),
    (8, 8, 64, 32, [500, 3], True),
    (5, 1, 80, 16, [200, 0, 0, 77], False),
    (20, 1, 128, 64, [300, 40], False),         # more heads on a key head than one tile has
    (35, 1, 64, 16, [150], True),
    (6, 2, 256, 16, [130, 70], False),
    (2, 2, 136, 16, [90], False),
    (2, 1, 8, 16, [140], False),
    (4, 1, 128, 128, [5000], False),            # one long sequence, split over many workgroups
])
def test_decode(dtype, heads, kv_heads, head_dim, page_rows, lengths, heads_first):
    gen = torch.Generator().manual_seed(sum(lengths) + heads)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, len(lengths), heads, head_dim, dtype=dtype)
    columns = max(1, -(-max(lengths) // page_rows)) + 1
    kc, vc, table = cache_of(keys, values, page_rows, columns, gen, heads_first)
    attention = Attention(heads, kv_heads, head_dim, dtype, page_rows)
    workspace = torch.full((attention.ws_bytes // 4,), NAN, device="cuda")   # its contents do not matter
    args = (q.cuda(), kc, vc, table, int32(lengths))
    got = attention.decode(*args, workspace=workspace)
    again = attention.decode(*args)
    assert torch.equal(got, again)
    for b, n in enumerate(lengths):
        want, bound = attend(q[b:b + 1], keys[b], values[b], torch.tensor([n]), 1 / math.sqrt(head_dim), dtype)
        assert_within(got[b:b + 1], want, bound, f"length {n}")
        if n == 0:
            assert bool((got[b] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv_heads,head_dim,lengths", [
    (1, 1, 64, [1]),
    (4, 2, 128, [1, 0, 15, 16, 17, 33, 127, 128, 129, 0, 255, 256, 257]),
    (20, 1, 128, [300, 40]),
    (35, 1, 72, [150, 0, 513]),
    (6, 2, 256, [130, 1000]),
    (2, 2, 136, [90, 640]),
])
def test_decode_with_room_for_more(dtype, heads, kv_heads, head_dim, lengths):
    """Tables with room for many more keys than there are: the line of units, shares and pieces whatever the lengths."""
    gen = torch.Generator().manual_seed(sum(lengths) + heads)
    keys, values = ([normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, len(lengths), heads, head_dim, dtype=dtype)
    kc, vc, table = cache_of(keys, values, 16, 2000, gen)
    attention = Attention(heads, kv_heads, head_dim, dtype, 16)
    workspace = torch.full((attention.ws_bytes // 4,), NAN, device="cuda")
    got = attention.decode(q.cuda(), kc, vc, table, int32(lengths), workspace=workspace).cpu()
    for b, n in enumerate(lengths):
        want, bound = attend(q[b:b + 1], keys[b], values[b], torch.tensor([n]), 1 / math.sqrt(head_dim), dtype)
        assert_within(got[b:b + 1], want, bound, f"length {n}")
    table[0, 0] = -1
    wrong = attention.decode(q.cuda(), kc, vc, table, int32([lengths[0]] + [-n - 1 for n in lengths[1:]])).cpu()
    assert bool(torch.isnan(wrong).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_many_sequences(dtype):
    """More sequences than a wavefront has lanes, and more units than workgroups: shares that begin and end anywhere."""
    gen = torch.Generator().manual_seed(5)
    lengths = [int(x) for x in torch.randint(0, 700, (300,), generator=gen)]
    keys, values = ([normal(gen, n, 2, 64, dtype=dtype) for n in lengths] for _ in range(2))
    q = normal(gen, 300, 4, 64, dtype=dtype)
    kc, vc, table = cache_of(keys, values, 64, 12, gen)
    got = Attention(4, 2, 64, dtype, 64).decode(q.cuda(), kc, vc, table, int32(lengths)).cpu()
    for b, n in enumerate(lengths):
        want, bound = attend(q[b:b + 1], keys[b], values[b], torch.tensor([n]), 1 / 8, dtype)
        assert_within(got[b:b + 1], want, bound, f"sequence {b} of length {n}")


@pytest.mark.parametrize("bad", [NAN, INF])
def test_decode_rows_beyond_the_length(bad):
    """The rest of the last page holds NaN or infinities, the table's other entries are no pages."""
    gen = torch.Generator().manual_seed(6)
    for n in (1, 16, 20, 31, 33, 130):
        keys, values = normal(gen, n, 1, 64, dtype=F16), normal(gen, n, 1, 64, dtype=F16)
        q = normal(gen, 1, 3, 64, dtype=F16)
        kc, vc, table = cache_of([keys], [values], 64, 5, gen, fill=bad)
        table[table < 0] = 2 ** 31 - 1
        got = Attention(3, 1, 64, F16, 64).decode(q.cuda(), kc, vc, table, int32([n]))
        want, bound = attend(q, keys, values, torch.tensor([n]), 1 / 8, F16)
        assert_within(got, want, bound, f"length {n}")


def test_decode_wrong_tables():
    gen = torch.Generator().manual_seed(7)
    keys, values = ([normal(gen, 200, 2, 64, dtype=BF16) for _ in range(5)] for _ in range(2))
    q = normal(gen, 5, 4, 64, dtype=BF16)
    kc, vc, table = cache_of(keys, values, 16, 13, gen)
    table[1, 5] = -1
    table[2, 12] = kc.shape[0]
    got = Attention(4, 2, 64, BF16, 16).decode(q.cuda(), kc, vc, table, int32([200, 200, 200, -3, 13 * 16 + 1])).cpu()
    want, bound = attend(q[:1], keys[0], values[0], torch.tensor([200]), 1 / 8, BF16)
    assert_within(got[:1], want, bound)
    assert bool(torch.isnan(got[1:]).all())


def test_cache_beyond_32_bits():
    """Pages whose offsets pass 2^32 elements (and bytes)."""
    gen = torch.Generator().manual_seed(8)
    pages, rows, d = 40_000, 64, 128
    kc, vc = (torch.empty(pages, rows, 16, d, dtype=BF16, device="cuda") for _ in range(2))   # 5.2 G elements each, most never touched
    n = 150
    keys, values = normal(gen, n, 16, d, dtype=BF16), normal(gen, n, 16, d, dtype=BF16)
    table = int32([[pages - 1, 1, pages - 5]])
    q = normal(gen, 1, 16, d, dtype=BF16)
    attention = Attention(16, 16, d, BF16, rows)
    rotated_q = attention.append(normal(gen, n, 16, d, dtype=BF16).cuda(), keys.cuda(), values.cuda(), kc, vc, table, int32([n]), int32([0, n]))
    assert rotated_q.shape == (n, 16, d)
    want, bound = attend(q, keys, values, torch.tensor([n]), 1 / math.sqrt(d), BF16)
    assert_within(attention.decode(q.cuda(), kc, vc, table, int32([n])), want, bound)
    assert_within(attention.prompt_paged(q.cuda(), kc, vc, table, int32([n]), int32([0, 1])), want, bound)


# -- append ------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("heads,kv_heads,head_dim,rotary_dim,interleaved,page_rows,lengths,rows,how", [
    (4, 2, 64, 64, False, 16, [1], [1], ""),
    (4, 2, 128, 128, False, 16, [5, 100, 17, 0, 33], [5, 20, 1, 0, 17], "wide"),
    (3, 1, 128, 64, True, 32, [70], [70], "heads"),
    (2, 2, 72, 36, False, 16, [40, 9], [3, 9], ""),      # half a rotation is 18 elements
    (2, 1, 72, 38, False, 16, [40], [30], "wide"),       # and 19
    (2, 1, 72, 38, True, 16, [40], [30], ""),
    (2, 1, 40, 0, False, 64, [90], [90], ""),
    (2, 2, 256, 248, False, 16, [20], [20], "heads"),
    (2, 2, 24, 24, False, 16, [20], [20], ""),
    (2, 1, 64, 64, False, 16, [3, 20], [10, 4], ""),     # rows before position 0 have no place
])
@pytest.mark.parametrize("heads_first", [False, True])
def test_append(dtype, heads, kv_heads, head_dim, rotary_dim, interleaved, page_rows, lengths, rows, how, heads_first):
    gen = torch.Generator().manual_seed(sum(rows) + rotary_dim)
    total = sum(rows)
    q, k, v = (normal(gen, total, h, head_dim, dtype=dtype) for h in (heads, kv_heads, kv_heads))
    old = [normal(gen, n, kv_heads, head_dim, dtype=dtype) for n in lengths]
    columns = max(1, -(-max(lengths) // page_rows))
    kc, vc, table = cache_of(old, old, page_rows, columns, gen, heads_first, fill=3.0)
    expect_k, expect_v, limit = kc.double().cpu(), vc.double().cpu(), torch.zeros(kc.shape, dtype=torch.float64)
    freq = [100.0 ** (-2.0 * t / max(rotary_dim, 1)) for t in range(rotary_dim // 2)]
    attention = Attention(heads, kv_heads, head_dim, dtype, page_rows, rotary_freq=freq, interleaved=interleaved)
    got = attention.append(*(by_strides(x.cuda(), how) for x in (q, k, v)), kc, vc, table, int32(lengths), int32(starts(rows)))
    u = half_step(dtype)
    at = 0
    for b, n in enumerate(rows):
        position = torch.arange(lengths[b] - n, lengths[b])
        want, bound = rotated(q[at:at + n], position, freq, interleaved)
        assert_within(got[at:at + n], want, bound + u * (want.abs() + bound) * (rotary_dim > 0), f"queries of {b}")
        want, bound = rotated(k[at:at + n], position, freq, interleaved)
        for i, p in enumerate(position.tolist()):
            if p >= 0:
                page = int(table[b, p // page_rows])
                expect_k[page, p % page_rows], expect_v[page, p % page_rows] = want[i], v[at + i].double()
                limit[page, p % page_rows] = bound[i] + u * (want[i].abs() + bound[i]) * (rotary_dim > 0)
        at += n
    assert_within(kc, expect_k, limit, "keys")
    assert torch.equal(vc.double().cpu(), expect_v)


def test_append_far_positions():
    """Positions near a million: angles are reduced in 64 bits."""
    gen = torch.Generator().manual_seed(2)
    n, d = 1_000_003, 64
    k = normal(gen, 2, 1, d)
    columns = -(-n // 4096)
    kc, vc = (torch.zeros(3, 4096, 1, d, device="cuda") for _ in range(2))
    table = torch.full((1, columns), -1, dtype=torch.int32)
    table[0, (n - 1) // 4096] = 2
    freq = [10000.0 ** (-2.0 * t / d) for t in range(d // 2)]
    attention = Attention(1, 1, d, F32, 4096, rotary_freq=freq)
    got = attention.append(k.cuda(), k.cuda(), k.cuda(), kc, vc, table.cuda(), int32([n]), int32([0, 2]))
    want, bound = rotated(k, torch.tensor([n - 2, n - 1]), freq, False)
    assert_within(got, want, bound + half_step(F32) * (want.abs() + bound))
    at = (n - 2) % 4096
    assert_within(kc[2, at:at + 2], want, bound + half_step(F32) * (want.abs() + bound))


def test_append_in_place_and_without_queries():
    gen = torch.Generator().manual_seed(4)
    q, k, v = normal(gen, 9, 2, 64, dtype=BF16).cuda(), normal(gen, 9, 1, 64, dtype=BF16).cuda(), normal(gen, 9, 1, 64, dtype=BF16).cuda()
    table, lengths, row_start = int32([[0]]), int32([9]), int32([0, 9])
    attention = Attention(2, 1, 64, BF16, 16, rotary_dim=64)
    caches = [torch.zeros(1, 16, 1, 64, dtype=BF16, device="cuda") for _ in range(4)]
    apart = attention.append(q, k, v, caches[0], caches[1], table, lengths, row_start)
    assert attention.append(None, k, v, caches[2], caches[3], table, lengths, row_start) is None
    in_place = q.clone()
    assert attention.append(in_place, k, v, caches[2], caches[3], table, lengths, row_start, out=in_place) is in_place
    assert torch.equal(apart, in_place) and torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])


def test_append_wrong_tables():
    """Rows of wrong lengths and pages are not stored, nor anything else written."""
    gen = torch.Generator().manual_seed(9)
    k = normal(gen, 6, 1, 64, dtype=BF16).cuda()
    caches = [torch.full((4, 16, 1, 64), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
    table = int32([[0, 1], [4, 1], [-1, 1], [2, 2 ** 31 - 1], [3, 3], [1, 1]])
    lengths = int32([1, 1, 1, 17, 33, 0])   # in page 0; page 4 of 4; page -1; no page; beyond the table; before position 0
    Attention(1, 1, 64, BF16, 16).append(None, k, k, *caches, table, lengths)
    for cache in caches:
        expect = torch.full((4, 16, 1, 64), 5.0, dtype=BF16, device="cuda")
        expect[0, 0] = k[0]
        assert torch.equal(cache, expect)


# -- streams, graphs, the whole of a step ---------------------------------------------------------------------------------------------
def _layer(attention, state):
    q = attention.append(state["q"], state["k"], state["v"], state["keys"], state["values"], state["table"], state["lengths"], out=state["turned"])
    return attention.decode(q, state["keys"], state["values"], state["table"], state["lengths"], out=state["out"])


def _decode_state(gen, lengths, heads=8, kv_heads=2, d=128, page_rows=16):
    keys, values = ([normal(gen, n, kv_heads, d, dtype=BF16) for n in lengths] for _ in range(2))
    kc, vc, table = cache_of(keys, values, page_rows, -(-max(lengths) // page_rows), gen, fill=0.0)
    q, k, v = (normal(gen, len(lengths), h, d, dtype=BF16).cuda() for h in (heads, kv_heads, kv_heads))
    return dict(q=q, k=k, v=v, keys=kc, values=vc, table=table, lengths=int32(lengths), turned=torch.empty_like(q), out=torch.empty_like(q))


def test_step_in_a_graph_and_on_another_stream():
    """A decoding step captured once and replayed for other lengths, pages and rows: each replay as the eager call, bit for bit."""
    gen = torch.Generator().manual_seed(10)
    attention = Attention(8, 2, 128, BF16, 16, rotary_dim=128)
    first, second = [700, 3, 64, 129], [650, 1, 0, 55]
    state = _decode_state(gen, first)
    before = state["keys"].clone(), state["values"].clone()

    def begin(lengths):   # a step writes to the cache: each begins from the same one
        state["lengths"].copy_(int32(lengths))
        state["keys"].copy_(before[0])
        state["values"].copy_(before[1])
        state["out"].fill_(NAN)

    eager = {}
    for name, lengths in (("first", first), ("second", second)):
        begin(lengths)
        _layer(attention, state)
        torch.cuda.synchronize()
        eager[name] = state["out"].clone()
        assert bool(torch.isfinite(eager[name].float()).all())
    assert not torch.equal(eager["first"], eager["second"])
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _layer(attention, state)
    for name, lengths in (("first", first), ("second", second), ("first", first)):
        begin(lengths)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(state["out"], eager[name]), name
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        begin(first)
        _layer(attention, state)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(state["out"], eager["first"])


def test_prompt_then_tokens_is_the_prompt_at_once():
    """Keys rotated and appended in chunks, attention behind the cache: the rows are those of one packed prompt of rotated keys."""
    gen = torch.Generator().manual_seed(13)
    n, chunk = 90, 37
    q, k, v = (normal(gen, n, h, 64, dtype=F32).cuda() for h in (4, 2, 2))
    attention = Attention(4, 2, 64, F32, 16, rotary_dim=32)
    kc, vc = (torch.full((8, 16, 2, 64), NAN, device="cuda") for _ in range(2))
    table = int32([[7, 2, 0, 5, 1, 3]])
    parts = []
    for lo, hi in ((0, chunk), (chunk, n - 3)):
        turned = attention.append(q[lo:hi], k[lo:hi], v[lo:hi], kc, vc, table, int32([hi]), int32([0, hi - lo]))
        parts.append(attention.prompt_paged(turned, kc, vc, table, int32([hi]), int32([0, hi - lo])))
    for i in range(n - 3, n):
        turned = attention.append(q[i:i + 1], k[i:i + 1], v[i:i + 1], kc, vc, table, int32([i + 1]))
        parts.append(attention.decode(turned, kc, vc, table, int32([i + 1])))
    freq = [10000.0 ** (-2.0 * t / 32) for t in range(16)]
    position = torch.arange(n)
    turned_q, turned_k = rotated(q, position, freq, False)[0].float(), rotated(k, position, freq, False)[0].float()
    want, bound = attend(turned_q, turned_k, v, position + 1, 1 / 8, F32)
    # the kernel's rotation is off by 2^-21 of a row's elements: scores by 64 times that
    moved = 2 * 2.0 ** -21 * float((turned_q.abs().sum(-1).max() * turned_k.abs().max())) / 8 * float(v.abs().max())
    assert_within(torch.cat(parts), want, bound + moved)


def test_refusals_of_tensors():
    attention = Attention(4, 2, 64, BF16, 16)
    rows = torch.zeros(3, 4, 64, dtype=BF16, device="cuda")
    cache = torch.zeros(2, 16, 2, 64, dtype=BF16, device="cuda")
    table, lengths = int32([[0], [1], [0]]), int32([1, 1, 1])
    with pytest.raises(TypeError):
        attention.decode(rows.float(), cache, cache, table, lengths)
    with pytest.raises(ValueError):
        attention.decode(rows[:, :2], cache, cache, table, lengths)
    with pytest.raises(ValueError):
        attention.decode(rows, cache[:, :8], cache[:, :8], table, lengths)
    with pytest.raises(ValueError):
        attention.decode(rows, cache, cache, table, lengths.long())
    with pytest.raises(ValueError):
        attention.decode(rows, cache, cache, table[:2], lengths)
    wide = torch.zeros(3, 4, 65, dtype=BF16, device="cuda")
    with pytest.raises(sc.ScError, match="SC_ERR_SHAPE_MISMATCH"):
        attention.decode(wide[..., 1:], cache, cache, table, lengths)     # rows that do not begin at multiples of 16 bytes
    with pytest.raises(sc.ScError, match="SC_ERR_SHAPE_MISMATCH"):
        attention.decode(rows, cache, cache, table, lengths, out=rows[:1].expand(3, 4, 64))
    with pytest.raises(sc.ScError, match="SC_ERR_WORKSPACE_SMALL"):
        attention.decode(rows, cache, cache, table, lengths, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
