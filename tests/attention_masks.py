"""Attention in 64 bits for any mask, with the bounds of attention_reference.attend, and the masks of windows and trees from their definitions."""
import math

import torch

from attention_reference import half_step


def attend_seen(q, k, v, seen, scale, dtype):
    """q (rows, heads, d), k and v (keys, kv_heads, d), seen (rows, keys).  The output in 64 bits and the error that the operator may have in `dtype`, element by
    element; the terms of the bound are attend's: the rounding of weights u A with A = sum p |v| / sum p, of the output u |o|, scores off by ds, which
    moves weights by that fraction (2 ds A), and 2^-24 (4 n + 64) A for sums of n terms, their rescaling, powers of two and joins."""
    rows, heads, _ = q.shape
    d, n = k.shape[2], k.shape[0]
    group = heads // k.shape[1]
    q, k, v, seen = q.double().cpu(), k.double().cpu(), v.double().cpu(), seen.cpu()
    out, bound = torch.zeros(rows, heads, v.shape[2], dtype=torch.float64), torch.zeros(rows, heads, v.shape[2], dtype=torch.float64)
    u = half_step(dtype)
    weight_u = u if dtype != torch.float32 else 0.0
    blind = ~seen.any(1)
    for h in range(heads):
        kh, vh = k[:, h // group], v[:, h // group]
        s = (q[:, h] @ kh.T * scale).masked_fill(~seen, -math.inf)
        size_s = (q[:, h].abs() @ kh.abs().T).masked_fill(~seen, 0.0)
        top = s.max(1, keepdim=True).values if n else torch.full((rows, 1), -math.inf, dtype=torch.float64)
        p = torch.exp(s - torch.where(top.isinf(), 0.0, top))
        total = p.sum(1, keepdim=True)
        total = torch.where(total == 0, 1.0, total)
        o, size = p @ vh / total, p @ vh.abs() / total
        largest = s.masked_fill(~seen, 0.0).abs().max(1).values if n else torch.zeros(rows, dtype=torch.float64)
        ds = 2.0 ** -24 * ((d + 4) * scale * (size_s.max(1).values if n else 0.0) + 4 * largest / math.log(2.0))
        out[:, h] = o
        bound[:, h] = size * (weight_u * 1.01 + 2 * ds[:, None] + 2.0 ** -24 * (4 * n + 64)) + u * o.abs() * 1.01 + torch.finfo(dtype).tiny
    out[blind] = 0.0
    return out, bound


def through_window(position, keys, window, sinks):
    """Rows at positions, keys at positions 0 .. keys - 1."""
    p, j = position[:, None], torch.arange(keys)[None, :]
    seen = j <= p
    return seen if window is None else seen & ((j > p - window) | (j < sinks))


def path_of(parents, node):
    path = []
    while node >= 0:
        path.append(node)
        node = parents[node]
    return path[::-1]


def tree_mask(parents, length, window=None, sinks=0):
    """(nodes, keys) of a tree whose nodes are the last keys of a sequence of `length`, and the positions of its nodes."""
    nodes = len(parents)
    before = length - nodes
    paths = [path_of(parents, i) for i in range(nodes)]
    position = torch.tensor([before + len(p) - 1 for p in paths], dtype=torch.int64)
    at = torch.arange(length)
    at[before:] = position
    seen = torch.zeros(nodes, length, dtype=torch.bool)
    seen[:, :before] = True
    for i, p in enumerate(paths):
        seen[i, [before + a for a in p]] = True
    if window is not None:
        seen &= (at[None, :] > position[:, None] - window) | (at[None, :] < sinks)
    return seen, position


def random_tree(nodes, spread, generator):
    return [int(torch.randint(max(-1, i - spread), i, (1,), generator=generator)) for i in range(nodes)]
