"""Timing cases of what a serving program does beside plain causal attention over a paged cache: a sliding window whose first tokens
stay visible, trees of drafted tokens, and the pages of sequences that branch, end or move.

Operators, by the name that a case gives:
  prompt, chunk, decode   attention through a sliding window of `window` positions and `sinks` first ones: packed prompts, the next rows of
                          sequences in the cache, one row a sequence
  tree                    attention of a tree of drafted tokens behind each sequence of the cache: a node sees the cache, its ancestors and itself
  accept                  the accepted path of each tree becomes the sequence: its rows of the cache move to consecutive places
  fork                    the next batch of sequences from the present one (each continues some sequence, cut or grown): tables of pages,
                          lengths, holders of pages, and the copies of pages that two sequences would write to, made for one layer
  compact                 pages in use move to the lowest numbers, tables with them, for one layer

A case has its lengths, trees and branches from itself alone, so that its work does not depend on the seed.  `run` computes the operator from
elementary torch operations in 32 bits, or, where `own` is true, through `paper_2311_09549_amd.attention.Attention`.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NO_KEEPER = 2 ** 31 - 1


def _case(name, op, dtype, heads, kv_heads, head_dim, batch, longest, *, rows=1, page_rows=16, window=0, sinks=0, spread=0, beams=1, grow=0,
          fill=0.0, heads_first=False):
    """`longest`: the longest sequence (of keys); `rows`: the most new rows of one; `spread`: how far before a node of a tree its parent may be;
    `beams`: sequences that share their beginnings; `grow`: rows that each is to gain; `fill`: the part of the cache's pages in use;
    `heads_first`: pages laid out head by head."""
    case = dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, batch=batch, longest=longest, rows=rows, page_rows=page_rows,
                window=window, sinks=sinks, spread=spread, beams=beams, grow=grow, fill=fill, heads_first=heads_first)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # one long document, each position with the 4,096 before it and the first four
        _case("window-prompt-long", "prompt", "bf16", 16, 4, 128, 1, 16384, window=4096, sinks=4),
        # the next chunk of four prompts through a window of an odd size, pages behind it given back
        _case("window-chunk-f16", "chunk", "f16", 32, 8, 128, 4, 8191, rows=509, page_rows=64, window=1000),
        # a decoding step of a full batch, contexts far longer than the window
        _case("window-decode", "decode", "bf16", 32, 8, 128, 64, 32767, window=4096, sinks=16),
        # a few drafted tokens behind one short conversation: latency is what counts
        _case("tree-one", "tree", "bf16", 32, 8, 128, 1, 341, rows=8, spread=3),
        # trees of up to 63 nodes behind the sequences of a batch
        _case("tree-batch", "tree", "bf16", 32, 8, 128, 24, 8191, rows=63, page_rows=64, spread=12),
        # full precision, every head with keys of its own, an odd head size
        _case("tree-f32", "tree", "f32", 16, 16, 80, 12, 1500, rows=21, page_rows=32, spread=5),
        # the accepted path of one small tree
        _case("accept-one", "accept", "bf16", 32, 8, 128, 1, 342, rows=8, spread=3),
        # the accepted paths of the trees of a large batch, pages laid out head by head
        _case("accept-batch-f16", "accept", "f16", 32, 8, 128, 192, 4095, rows=63, page_rows=32, spread=8, heads_first=True),
        # one step of a search with four beams for two requests
        _case("fork-beams", "fork", "bf16", 32, 8, 128, 8, 700, beams=4, grow=1),
        # a step of a large batch of beams in small pages
        _case("fork-batch", "fork", "bf16", 16, 4, 128, 384, 8191, beams=6, grow=7),
        # the few pages of a small cache
        _case("compact-small-f16", "compact", "f16", 12, 12, 64, 5, 333, page_rows=16, fill=0.5),
        # a cache of which most sequences have ended
        _case("compact-large", "compact", "bf16", 32, 8, 128, 48, 8191, page_rows=64, fill=0.3),
    ]


# ---------------------------------------------------------------------------------------------------------------------------
# what follows from a case alone
# ---------------------------------------------------------------------------------------------------------------------------
def _rng(case, what):
    return random.Random(what + " %s" % sorted((k, v) for k, v in case.items() if k != "name"))


def _lengths(case):
    """Keys and new rows of each sequence: the longest among them, the others log-uniform below it, most within a factor of 32.  Sequences that
    share a beginning are of one length."""
    rng = _rng(case, "lengths")
    longest, groups = case["longest"], case["batch"] // case["beams"]
    keys = [longest]
    for _ in range(groups - 1):
        least = 1.0 if rng.random() < 0.125 else max(1.0, longest / 32)
        keys.append(int(math.exp(rng.uniform(math.log(least), math.log(longest + 0.5)))))
    rng.shuffle(keys)
    keys = [n for n in keys for _ in range(case["beams"])]
    if case["op"] == "prompt":
        return keys, list(keys)
    return keys, [min(n, case["rows"]) if case["rows"] == 1 else min(n, rng.randint((case["rows"] + 1) // 2, case["rows"])) for n in keys]


def _trees(case):
    """Parent of every node, as a number within its tree (-1: none), and the node up to which a tree is accepted (-1: nothing of it)."""
    rng = _rng(case, "trees")
    parents, last = [], []
    for r in _lengths(case)[1]:
        parents.append([rng.randint(max(-1, i - case["spread"]), i - 1) for i in range(r)])
        last.append(rng.randrange(r) if rng.random() < 0.9 else -1)
    return parents, last


def _depths(parents):
    depth = []
    for p in parents:
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return depth


def _path(parents, node):
    path = []
    while node >= 0:
        path.append(node)
        node = parents[node]
    return path[::-1]


def _branches(case):
    """What each sequence of the next batch continues (-1: nothing), and the rows that it is to have."""
    rng = _rng(case, "branches")
    keys, beams = _lengths(case)[0], case["beams"]
    parents = [-1 if rng.random() < 0.05 else i // beams * beams + rng.randrange(beams) for i in range(len(keys))]
    wanted = [case["grow"] if p < 0 else max(0, keys[p] - rng.randint(1, 3 * case["page_rows"])) if rng.random() < 0.1 else keys[p] + case["grow"] for p in parents]
    return parents, wanted


def _copies(case):
    """Rows of each page that `fork` copies: sequences of one parent that all keep its last page in part, but for the first."""
    keys, (parents, wanted) = _lengths(case)[0], _branches(case)
    seen, rows = set(), []
    for p, w in zip(parents, wanted):
        if p < 0:
            continue
        kept = min(keys[p], w)
        shared = _shared(case, keys[p])
        if kept % case["page_rows"]:
            # cut within what the beams share: others hold that page
            if kept < shared * case["page_rows"] or (p, kept // case["page_rows"]) in seen:
                rows.append(kept % case["page_rows"])
            seen.add((p, kept // case["page_rows"]))
    return rows


def _shared(case, n):
    """Pages at the beginning that the beams of a sequence of n rows share."""
    return int(n * 0.6) // case["page_rows"] if case["beams"] > 1 else 0


def _columns(case):
    return -(-(case["longest"] + case["grow"]) // case["page_rows"]) + 1


def _pages_in_use(case):
    keys, r, beams = _lengths(case)[0], case["page_rows"], case["beams"]
    return sum(-(-n // r) * beams - (beams - 1) * _shared(case, n) for n in keys[::beams])


def _seen_by(case, position):
    """Keys that rows at these positions see: through the window, and of the first ones."""
    window, sinks = case["window"], case["sinks"]
    if not window:
        return position + 1
    return np.minimum(position + 1, window) + np.minimum(np.maximum(position + 1 - window, 0), sinks)


def _positions(case):
    """Positions of the new rows of each sequence."""
    keys, rows = _lengths(case)
    if case["op"] != "tree":
        return [np.arange(n - r, n) for n, r in zip(keys, rows)]
    return [n - r + np.array(_depths(p), dtype=np.int64) for n, r, p in zip(keys, rows, _trees(case)[0])]


def work(case):
    op, size, r = case["op"], TYPES[case["dtype"]].itemsize, case["page_rows"]
    h, g, d, batch = case["heads"], case["kv_heads"], case["head_dim"], case["batch"]
    keys, rows = _lengths(case)
    row = 2 * g * d * size   # a row's keys and values
    if op == "accept":
        parents, last = _trees(case)
        paths = [_path(p, x) for p, x in zip(parents, last)]
        moved = sum(sum(i != at for at, i in enumerate(p)) for p in paths)
        return {"bytes": 2 * moved * row + 4 * (3 * batch + 1 + sum(len(p) for p in paths)) + 4 * batch, "flops": 0}
    if op in ("fork", "compact"):
        in_use = sum(-(-n // r) for n in keys)
        if op == "fork":
            wanted = _branches(case)[1]
            pool = _pool(case)
            return {"bytes": 4 * (in_use + batch * _columns(case) + 5 * batch + 2 * pool) + 2 * row * sum(_copies(case)), "flops": 0}
        used, pool = _pages_in_use(case), _pool(case)
        # a page is as likely to be in use as any other: of those beyond the lowest `used` that many
        return {"bytes": 4 * (2 * in_use + batch + 2 * pool) + int(2 * r * row * used * (pool - used) / pool), "flops": 0}
    pairs, least = 0, 0
    for n, p in zip(keys, _positions(case)):
        pairs += int(_seen_by(case, p).sum())
        lo = max(0, int(p[0]) + 1 - case["window"]) if case["window"] and len(p) else 0
        least += n - lo + min(lo, case["sinks"])
    pages = 0 if op == "prompt" else -(-least // r)
    nodes = sum(rows) if op == "tree" else 0
    return {"bytes": 2 * sum(rows) * h * d * size + least * row + 4 * (2 * batch + 1 + pages + nodes), "flops": 4 * pairs * h * d}


def _pool(case):
    """Pages of the cache."""
    if case["op"] == "compact":
        return int(math.ceil(_pages_in_use(case) / case["fill"])) + 1
    if case["op"] == "fork":
        more = sum(-(-w // case["page_rows"]) for w in _branches(case)[1])
        return _pages_in_use(case) + more // 4 + 2 * case["batch"] + (case["batch"] * case["grow"]) // case["page_rows"] + 3
    keys, rows = _lengths(case)
    return sum(len(_held(case, n, r)) for n, r in zip(keys, rows)) + 3


def _held(case, n, new):
    """Columns of a sequence's table that have a page: with a window, those that its new rows see."""
    r, window = case["page_rows"], case["window"]
    columns = range(-(-n // r))
    if not window:
        return columns
    lo = n - new - window + 1
    return [c for c in columns if c * r < case["sinks"] or (c + 1) * r > lo]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator and type, groups of 1 to 16 heads, head sizes of every multiple of 8 up to 256, one to 96 sequences (more where
    pages alone are concerned), one token to the longest listed lengths, windows from one position on."""
    most = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        op = rng.choice(("prompt", "chunk", "decode", "tree", "tree", "accept", "fork", "compact"))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        head_dim = rng.choice((64, 64, 128, 128, 128, 8 * rng.randint(2, 32)))
        kv_heads = rng.choice((1, 2, 3, 4, 8, 8, 16))
        heads = kv_heads * rng.choice((1, 1, 2, 4, 4, 5, 7, 8, 16))
        page_rows = rng.choice((16, 16, 32, 64, 128))
        pages_alone = op in ("accept", "fork", "compact")
        longest = _log_uniform(rng, 1, {"prompt": 16384, "tree": 65535}.get(op, 32767))
        beams = rng.choice((1, 2, 4, 5)) if op == "fork" else 1
        batch = beams * max(1, _log_uniform(rng, 1, 192 if pages_alone else 96) // beams)
        windowed = op in ("prompt", "chunk", "decode") or (op == "tree" and rng.random() < 0.25)
        case = _case(None, op, dtype, heads, kv_heads, head_dim, batch, longest, page_rows=page_rows,
                     rows=_log_uniform(rng, 1, min(longest, 2048)) if op == "chunk" else _log_uniform(rng, 1, min(longest, 128)) if op in ("tree", "accept") else 1,
                     window=_log_uniform(rng, 1, 8192) if windowed else 0, sinks=rng.choice((0, 0, 1, 4, rng.randint(1, 128))) if windowed else 0,
                     spread=rng.randint(1, 16) if op in ("tree", "accept") else 0, beams=beams, grow=rng.choice((0, 1, 1, rng.randint(1, 100))) if op == "fork" else 0,
                     fill=rng.uniform(0.1, 0.9) if op == "compact" else 0.0, heads_first=rng.random() < 0.3)
        if heads > 64 or batch * longest * kv_heads * head_dim > 64 * 32767 * 8 * 128:
            continue
        keys, rows = _lengths(case)
        # the plain form holds every score of the padded batch, and caches are outputs as a whole where rows move
        scores = 0 if pages_alone else batch * heads * max(rows) * longest
        held = 2 * _pool(case) * page_rows * kv_heads * head_dim * TYPES[dtype].itemsize if op != "prompt" else 0
        if scores > 16 * 16384 ** 2 or held > (3 if pages_alone else 8) << 30:
            continue
        w = work(case)
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops:
            return case


# ---------------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------------
def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def prepare(case, seed):
    """Projections as a layer hands them over, the cache of the sequences with its tables, and trees or branches.  Scores have a spread of about two, some
    channels are larger than the others, the first key draws attention and values have a mean."""
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    op, dtype = case["op"], TYPES[case["dtype"]]
    h, g, d, r = case["heads"], case["kv_heads"], case["head_dim"], case["page_rows"]
    keys, rows = _lengths(case)
    total = sum(rows)

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, dtype=torch.float32, generator=gen)

    channel = 1.0 + normal(d).square() * 0.25
    state = dict(case=case, longest=max(keys), most_rows=max(rows), scale=1.0 / math.sqrt(d), lengths=_int32(keys))
    if op in ("prompt", "chunk", "decode", "tree"):
        # one projection holds queries, keys and values of a row side by side
        qkv = normal(total, h + 2 * g, d) * channel
        qkv[:, :h] += 0.5 * normal(1, h, d)
        qkv[:, h + g:] += 0.25
        qkv = qkv.to(dtype)
        state["q"], state["k"], state["v"] = qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:]
    if op in ("prompt", "chunk", "tree", "accept"):
        state["row_start"] = _int32(np.cumsum([0] + rows).tolist())
    if op in ("tree", "accept"):
        parents, last = _trees(case)
        state["parents"], state["last"] = _int32([p for tree in parents for p in tree]), _int32(last)
    if op == "prompt":
        return state
    count = _pool(case)
    order = torch.randperm(count, device=DEVICE, generator=gen).to(torch.int32)
    if op in ("fork", "compact"):
        table = torch.full((case["batch"], _columns(case)), -1, dtype=torch.int64)
        at, beams = 0, case["beams"]
        for b in range(0, case["batch"], beams):
            used, shared = -(-keys[b] // r), _shared(case, keys[b])
            for n in range(beams):
                table[b + n, :shared] = torch.arange(at, at + shared)
                table[b + n, shared:used] = torch.arange(at + shared + n * (used - shared), at + shared + (n + 1) * (used - shared))
            at += shared + beams * (used - shared)
        table = table.to(DEVICE)
        there = table >= 0
        table[there] = order[table[there]].long()
        state["holders"] = torch.zeros(count, dtype=torch.int32, device=DEVICE).index_add_(0, table[there], torch.ones(int(there.sum()), dtype=torch.int32, device=DEVICE))
        state["pages"] = table.to(torch.int32)
        if op == "fork":
            parents, wanted = _branches(case)
            state["parents"], state["wanted"] = _int32(parents), _int32(wanted)
    else:
        table, at = torch.full((len(keys), max(1, -(-max(keys) // r))), -1, dtype=torch.int64), 0
        for b, (n, new) in enumerate(zip(keys, rows)):
            columns = torch.tensor(list(_held(case, n, new)), dtype=torch.int64)
            table[b, columns] = torch.arange(at, at + len(columns))
            at += len(columns)
        table = table.to(DEVICE)
        state["pages"] = torch.where(table >= 0, order[table.clamp(min=0)], -1).to(torch.int32)
    for name in ("keys", "values"):
        cache = normal(count, g, r, d) if case["heads_first"] else normal(count, r, g, d)
        cache = (cache * channel + (0.25 if name == "values" else 0.0)).to(dtype)
        state[name] = cache.transpose(1, 2) if case["heads_first"] else cache
    return state


# ---------------------------------------------------------------------------------------------------------------------------
# the operators from elementary torch operations, in 32 bits
# ---------------------------------------------------------------------------------------------------------------------------
def _attend(q, k, v, seen, scale):
    """q (batch, R, heads, d), k and v (batch, N, kv_heads, d), seen (batch, R, N), all padded."""
    batch, most, h, d = q.shape
    n, g = k.shape[1], k.shape[2]
    grouped = q.float().reshape(batch, most, g, h // g, d).permute(0, 2, 3, 1, 4).reshape(batch, g, h // g * most, d)
    scores = torch.matmul(grouped, k.float().permute(0, 2, 3, 1).contiguous()).mul_(scale)
    scores = scores.view(batch, g, h // g, most, n)
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = scores.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights.view(batch, g, h // g * most, n), v.float().permute(0, 2, 1, 3).contiguous())
    out = out.view(batch, g, h // g, most, d) / torch.where(total == 0.0, 1.0, total)
    return out.permute(0, 3, 1, 2, 4).reshape(batch, most, h, d).to(q.dtype)


def _through_window(case, j, position):
    """Whether a row at `position` sees key j."""
    seen = j <= position
    if case["window"]:
        seen = seen & ((j > position - case["window"]) | (j < case["sinks"]))
    return seen


def _paged(state):
    """Keys and values of the sequences, padded to the longest."""
    r = state["keys"].shape[1]
    j = torch.arange(state["longest"], device=DEVICE)
    page = state["pages"].long().clamp(min=0)[:, j // r]
    return state["keys"][page, j % r], state["values"][page, j % r]


def _padded(state):
    """Rows of each sequence as numbers in the packed rows, padded to the most; how many there are, and each one's sequence and place there."""
    starts = state["row_start"].long()
    total = state["q"].shape[0]
    row = torch.arange(total, device=DEVICE)
    seq = torch.searchsorted(starts, row, right=True) - 1
    return (starts[:-1, None] + torch.arange(state["most_rows"], device=DEVICE)).clamp_(max=total - 1), starts[1:] - starts[:-1], seq, row - starts[seq]


def _plain_prompt(state):
    padded, rows, seq, place = _padded(state)
    lengths = state["lengths"].long()
    k, v = (state["k"][padded], state["v"][padded]) if state["case"]["op"] == "prompt" else _paged(state)
    j = torch.arange(k.shape[1], device=DEVICE)
    position = (lengths - rows)[:, None] + torch.arange(state["most_rows"], device=DEVICE)
    seen = _through_window(state["case"], j, position[:, :, None]) & (j < lengths[:, None, None])
    return _attend(state["q"][padded], k, v, seen, state["scale"])[seq, place]


def _plain_decode(state):
    k, v = _paged(state)
    position = state["lengths"].long()[:, None, None] - 1
    seen = _through_window(state["case"], torch.arange(k.shape[1], device=DEVICE), position)
    return _attend(state["q"][:, None], k, v, seen, state["scale"])[:, 0]


def _closure(parents, most):
    """parents (batch, most): whether node j is i or one of its ancestors, (batch, i, j)."""
    node = torch.arange(most, device=DEVICE)
    reach = ((node == parents[:, :, None]) | (node == node[:, None])).float()
    for _ in range(max(1, (most - 1).bit_length())):
        reach = torch.bmm(reach, reach).clamp_(max=1.0)
    return reach > 0.5


def _plain_tree(state):
    padded, rows, seq, place = _padded(state)
    most, lengths = state["most_rows"], state["lengths"].long()
    before = (lengths - rows)[:, None]
    tree = _closure(state["parents"].long()[padded], most)
    position = before + tree.sum(-1) - 1     # of the nodes
    k, v = _paged(state)
    j = torch.arange(k.shape[1], device=DEVICE)
    node = (j - before).clamp(0, most - 1)   # key j, if it is a node
    behind = (j >= before)[:, None]
    related = tree.gather(2, node[:, None].expand(-1, most, -1))
    at = torch.where(behind, position.gather(1, node)[:, None], j)
    seen = _through_window(state["case"], at, position[:, :, None]) & (~behind | related) & (j < lengths[:, None, None])
    return _attend(state["q"][padded], k, v, seen, state["scale"])[seq, place]


def _plain_accept(state):
    most, lengths, r = state["most_rows"], state["lengths"].long(), state["keys"].shape[1]
    starts, last = state["row_start"].long(), state["last"].long()
    rows, place = starts[1:] - starts[:-1], torch.arange(most, device=DEVICE)
    parents = state["parents"].long()[(starts[:-1, None] + place).clamp_(max=state["parents"].shape[0] - 1)]
    tree = _closure(parents, most)
    path = tree.gather(1, last.clamp(min=0)[:, None, None].expand(-1, 1, most))[:, 0] & (last >= 0)[:, None]
    accepted = path.sum(1)
    # what goes to place n of a sequence: the path's n-th node, behind it what is there
    order = torch.argsort((~path).to(torch.int32), dim=1, stable=True)
    place = torch.minimum(place, rows[:, None] - 1)
    source = torch.where(place < accepted[:, None], order.gather(1, place), place)
    before = (lengths - rows)[:, None]
    table = state["pages"].long()
    of, to = before + source, before + place
    of_page, to_page = table.gather(1, of // r), table.gather(1, to // r)
    for cache in (state["keys"], state["values"]):
        cache[to_page, to % r] = cache[of_page, of % r]
    return state["keys"], state["values"], (before[:, 0] + accepted).to(torch.int32)


def _copy(state, moves):
    """Rows 0 .. moves[n, 2] - 1 of page moves[n, 0] to page moves[n, 1]; pages outside the cache: nothing."""
    source, target, rows = moves.long().unbind(1)
    row = torch.arange(state["keys"].shape[1], device=DEVICE)
    move, row = ((source >= 0)[:, None] & (row < rows[:, None])).nonzero().unbind(1)
    for cache in (state["keys"], state["values"]):
        cache[target[move], row] = cache[source[move], row]


def _plain_fork(state):
    case, table, lengths = state["case"], state["pages"].long(), state["lengths"].long()
    parents, wanted, r = state["parents"].long(), state["wanted"].long(), case["page_rows"]
    pages, (batch, columns), new = state["holders"].shape[0], table.shape, parents.shape[0]
    first = torch.arange(columns, device=DEVICE) * r
    held_before = (first < lengths[:, None]) & (table >= 0)
    continued = torch.where(parents >= 0, lengths[parents.clamp(min=0)], 0)
    kept = torch.minimum(continued, wanted)
    entry = torch.where((parents >= 0)[:, None], table[parents.clamp(min=0)], -1)
    held = (first < kept[:, None]) & (entry >= 0)
    part = held & (first + r > kept[:, None])
    whole = held & ~part
    # entries that are none count for a page behind the last one
    holders = torch.cat([state["holders"], torch.zeros(1, dtype=torch.int32, device=DEVICE)])
    holders.index_add_(0, torch.where(held_before, table, pages).flatten(), torch.full((batch * columns,), -1, dtype=torch.int32, device=DEVICE))
    holders.index_add_(0, torch.where(whole, entry, pages).flatten(), torch.ones(new * columns, dtype=torch.int32, device=DEVICE))
    last = torch.where(part, entry, -1).amax(1)       # the page of each sequence that it is going to write to
    last_or_none = torch.where(last >= 0, last, pages)
    number = torch.arange(new, device=DEVICE)
    keeper = torch.full((pages + 1,), NO_KEEPER, dtype=torch.int64, device=DEVICE).scatter_reduce_(0, last_or_none, number, "amin")
    keeps = (last >= 0) & (keeper[last_or_none] == number) & (holders[last_or_none] == 0)
    copies = (last >= 0) & ~keeps
    grown = torch.clamp((wanted + r - 1) // r - (kept + r - 1) // r, min=0)
    need = copies + grown
    offset = need.cumsum(0) - need
    free = (holders[:pages] == 0) & (keeper[:pages] == NO_KEEPER)
    rank = free.cumsum(0) - 1
    by_rank = torch.zeros(pages + 1, dtype=torch.int64, device=DEVICE)
    by_rank[torch.where(free, rank, pages)] = torch.arange(pages, device=DEVICE)
    served = (need == 0) | (offset + need <= rank[-1] + 1)
    # the columns: whole pages, the one to be written to, those that are new
    column = torch.arange(columns, device=DEVICE)
    after = column - ((kept + r - 1) // r)[:, None]
    taken = by_rank[(offset[:, None] + copies[:, None] + after).clamp(0, pages)]
    copied = by_rank[offset.clamp(max=pages)]
    result = torch.where(whole, entry, -1)
    result = torch.where(part, torch.where(copies[:, None], copied[:, None], entry), result)
    result = torch.where((after >= 0) & (after < grown[:, None]), taken, result)
    result = torch.where(served[:, None], result, -1)
    # pages that were taken or kept to be written to have one holder, those of sequences that found no room one less
    holders.index_add_(0, torch.where(whole & ~served[:, None], entry, pages).flatten(), torch.full((new * columns,), -1, dtype=torch.int32, device=DEVICE))
    alone = torch.where((~whole) & (result >= 0), result, pages)
    holders[alone.flatten()] = 1
    moves = torch.stack([last, copied, kept % r], 1)
    moves = torch.where((copies & served)[:, None], moves, torch.tensor([-1, -1, 0], device=DEVICE)).to(torch.int32)
    _copy(state, moves)
    return result.to(torch.int32), torch.where(served, wanted, -1).to(torch.int32), holders[:pages].contiguous(), moves, state["keys"], state["values"]


def _plain_compact(state):
    case, holders = state["case"], state["holders"]
    pages, r = holders.shape[0], case["page_rows"]
    used = holders != 0
    count = used.sum()
    number = torch.arange(pages, device=DEVICE)
    high, low = used & (number >= count), ~used & (number < count)
    by_rank = torch.full((pages + 1,), -1, dtype=torch.int64, device=DEVICE)
    sources, targets = by_rank.clone(), by_rank
    sources[torch.where(high, high.cumsum(0) - 1, pages)] = number
    targets[torch.where(low, low.cumsum(0) - 1, pages)] = number
    moving = number < high.sum()
    to = torch.where(high, targets[(high.cumsum(0) - 1).clamp(min=0)], number)
    after = torch.where(number < count, 1, 0).to(torch.int32) * torch.where(used, holders, holders[sources[(low.cumsum(0) - 1).clamp(min=0)].clamp(min=0)])
    table = state["pages"].long()
    in_use = (torch.arange(table.shape[1], device=DEVICE) * r < state["lengths"].long()[:, None]) & (table >= 0)
    result = torch.where(in_use, to[table.clamp(min=0)], table).to(torch.int32)
    moves = torch.stack([sources[:pages], targets[:pages], torch.full_like(number, r)], 1)
    moves = torch.where(moving[:, None], moves, torch.tensor([-1, -1, 0], device=DEVICE)).to(torch.int32)[:pages // 2]
    _copy(state, moves)
    return result, after, moves, state["keys"], state["values"]


# ---------------------------------------------------------------------------------------------------------------------------
# the same through the framework
# ---------------------------------------------------------------------------------------------------------------------------
def _handle(state):
    """The handle that a program keeps for its layers."""
    from paper_2311_09549_amd.attention import Attention

    case = state["case"]
    return Attention(case["heads"], case["kv_heads"], case["head_dim"], dtype=TYPES[case["dtype"]], page_rows=case["page_rows"],
                     window=case["window"] or None, sinks=case["sinks"], device=DEVICE)


def _own(state):
    attention = state.get("handle")
    if attention is None:
        attention = state["handle"] = _handle(state)
    op = state["case"]["op"]
    if op == "prompt":
        return attention.prompt(state["q"], state["k"], state["v"], state["row_start"])
    if op == "chunk":
        return attention.prompt_paged(state["q"], state["keys"], state["values"], state["pages"], state["lengths"], state["row_start"])
    if op == "decode":
        return attention.decode(state["q"], state["keys"], state["values"], state["pages"], state["lengths"])
    if op == "tree":
        return attention.tree(state["q"], state["keys"], state["values"], state["pages"], state["lengths"], state["row_start"], state["parents"])
    if op == "accept":
        lengths = attention.accept(state["keys"], state["values"], state["pages"], state["lengths"], state["row_start"], state["parents"], state["last"])
        return state["keys"], state["values"], lengths
    if op == "fork":
        pages, lengths, holders, moves = attention.fork(state["pages"], state["lengths"], state["holders"], state["parents"], state["wanted"])
        attention.copy(state["keys"], state["values"], moves)
        return pages, lengths, holders, moves, state["keys"], state["values"]
    pages, holders, moves = attention.compact(state["pages"], state["lengths"], state["holders"])
    attention.copy(state["keys"], state["values"], moves)
    return pages, holders, moves, state["keys"], state["values"]


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_prompt, "chunk": _plain_prompt, "decode": _plain_decode, "tree": _plain_tree, "accept": _plain_accept, "fork": _plain_fork,
            "compact": _plain_compact}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------------------------------------------------------
def _exact_attention(case, state):
    lengths, positions = state["lengths"].tolist(), _positions(case)
    starts = state["row_start"].tolist() if "row_start" in state else list(range(len(lengths) + 1))
    trees = _trees(case)[0] if case["op"] == "tree" else None
    r, window, sinks = case["page_rows"], case["window"], case["sinks"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device=DEVICE)
    group = case["heads"] // case["kv_heads"]
    for b, n in enumerate(lengths):
        lo, hi = starts[b], starts[b + 1]
        new = hi - lo
        if case["op"] == "prompt":
            k, v = state["k"][lo:hi], state["v"][lo:hi]
        else:
            used = state["pages"][b, :-(-n // r)].long().clamp(min=0)
            k, v = (state[name][used].flatten(0, 1)[:n] for name in ("keys", "values"))
        hidden = np.zeros((new, n), dtype=bool)
        at = np.arange(n)   # positions of the keys
        if trees:
            at[n - new:] = positions[b]
            hidden[:, n - new:] = True
            for i in range(new):
                hidden[i, [n - new + x for x in _path(trees[b], i)]] = False
        p = positions[b][:, None]
        hidden |= at[None, :] > p
        if window:
            hidden |= (p - at[None, :] >= window) & (at[None, :] >= sinks)
        hidden = torch.from_numpy(hidden).to(DEVICE)
        for head in range(case["heads"]):
            kh, vh = k[:, head // group].double(), v[:, head // group].double()
            logits = state["q"][lo:hi, head].double() @ kh.T * state["scale"]
            logits[hidden] = -math.inf
            logits -= logits.max(1, keepdim=True).values
            logits.exp_()
            out[lo:hi, head] = logits @ vh / logits.sum(1, keepdim=True)
    return out


def _moved(state, moves):
    """The cache in 64 bits after (page, row) -> (page, row) moves, all of them from what was there before."""
    caches = []
    for name in ("keys", "values"):
        cache = state[name].double()
        if moves:
            a, b, c, e = torch.tensor(moves, device=DEVICE).unbind(1)
            cache[c, e] = state[name][a, b].double()
        caches.append(cache)
    return caches


def exact(case, seed):
    state = prepare(case, seed)
    op, r = case["op"], case["page_rows"]
    if op in ("prompt", "chunk", "decode", "tree"):
        return _exact_attention(case, state)
    table, lengths = state["pages"].tolist(), state["lengths"].tolist()
    if op == "accept":
        moves = []
        for b, (tree, node) in enumerate(zip(*_trees(case))):
            before = lengths[b] - len(tree)
            for at, i in enumerate(_path(tree, node)):
                moves.append((table[b][(before + i) // r], (before + i) % r, table[b][(before + at) // r], (before + at) % r))
        return (*_moved(state, moves), None)
    if op == "compact":
        holders = state["holders"].tolist()
        count = sum(x != 0 for x in holders)
        pairs = zip([p for p, x in enumerate(holders) if x and p >= count], [p for p, x in enumerate(holders[:count]) if not x])
        return (None, None, None, *_moved(state, [(p, row, to, row) for p, to in pairs for row in range(r)]))
    # fork: sequence after sequence, from a list of the free pages
    held = {}
    parents, wanted = _branches(case)
    kept = [min(lengths[p], w) if p >= 0 else 0 for p, w in zip(parents, wanted)]
    for p, n in zip(parents, kept):
        for page in table[p][:n // r] if p >= 0 else []:
            held[page] = held.get(page, 0) + 1
    written = {}
    for i, (p, n) in enumerate(zip(parents, kept)):
        if n % r:
            written.setdefault(table[p][n // r], []).append(i)
    free = [p for p in range(len(state["holders"])) if p not in held and p not in written]
    moves, at = [], 0
    for i, (p, n, w) in enumerate(zip(parents, kept, wanted)):
        page = table[p][n // r] if n % r else -1
        copied = page >= 0 and (page in held or written[page][0] != i)
        if copied:
            moves += [(page, row, free[at], row) for row in range(n % r)]
        at += copied + max(0, -(-w // r) - -(-n // r))
    return (None, None, None, None, *_moved(state, moves))
