"""Attention and rotation in 64 bits, row by row from the definition, and how far a kernel's result may be from it."""
import math

import torch


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def attend(q, k, v, sees, scale, dtype):
    """q (rows, heads, d), k and v (keys, kv_heads, d), sees (rows): row i sees keys [0, sees[i]).  The output in 64 bits and the error that
    the operator may have in `dtype`, element by element.

    Per element, with A = sum p |v| / sum p of its row and u half a step of the type: the weights' rounding to 16 bits gives u A, the rounding of the output u
    |o|; scores are off by ds = 2^-24 ((d + 4) scale sum |q k| + 4 |s| / ln 2) at most, which moves weights by that fraction (numerator and
    denominator: 2 ds A); sums of n terms, rescaled every 16 keys at the most often, and powers of two add 2^-24 (4 n + 64) A."""
    rows, heads, d = q.shape
    group = heads // k.shape[1]
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    out, bound = torch.zeros(rows, heads, v.shape[2], dtype=torch.float64), torch.zeros(rows, heads, v.shape[2], dtype=torch.float64)
    u = half_step(dtype)
    weight_u = u if dtype != torch.float32 else 0.0
    for i in range(rows):
        n = max(0, int(sees[i]))
        if n == 0:
            continue
        for h in range(heads):
            kh, vh = k[:n, h // group], v[:n, h // group]
            s = kh @ q[i, h] * scale
            top = s.max()
            if top == -math.inf:
                continue
            p = torch.exp(s - top)
            total = p.sum()
            out[i, h] = p @ vh / total
            size = p @ vh.abs() / total
            ds = 2.0 ** -24 * ((d + 4) * scale * float((kh.abs() @ q[i, h].abs()).max()) + 4 * float(s.abs().max()) / math.log(2.0))
            bound[i, h] = size * (weight_u * 1.01 + 2 * ds + 2.0 ** -24 * (4 * n + 64)) + u * out[i, h].abs() * 1.01 + torch.finfo(dtype).tiny
    return out, bound


def rotated(x, position, freq, interleaved):
    """x (rows, heads, d) turned by position * freq, in 64 bits, and the error that a kernel may have before its last rounding: sine and cosine in 32 bits are
    off by 2^-22 at most (2^-25 turns of angle, two steps of the functions), the sum of two products by three roundings."""
    x = x.double().cpu()
    out, bound = x.clone(), torch.zeros_like(x)
    half = len(freq)
    for t in range(half):
        a, b = (2 * t, 2 * t + 1) if interleaved else (t, t + half)
        angle = position.double().cpu() * freq[t]
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        bound[..., a] = bound[..., b] = (x[..., a].abs() + x[..., b].abs()) * (2.0 ** -22 + 3 * 2.0 ** -24)
    return out, bound


def assert_within(got, want, bound, what=""):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - want).abs() - bound
    worst = float(((got - want).abs() / bound.clamp_min(1e-300)).max()) if got.numel() else 0.0
    assert bool((over <= 0).all()), f"{what}: error is {worst:.3f} of what it may be"


def cache_of(keys, values, page_rows, pages, generator, heads_first=False, spare=2, fill=float("nan"), device="cuda"):
    """Packs per-sequence keys and values (n, kv_heads, d) into pages in random order; rows of no key hold `fill`.  Returns keys, values (pages,
    page_rows, kv_heads, d) and the table with `pages` columns, -1 where a sequence needs no page."""
    need = [-(-k.shape[0] // page_rows) for k in keys]
    total = sum(need) + spare
    kv_heads, d = keys[0].shape[1:]
    order = torch.randperm(total, generator=generator).tolist()
    shape = (total, kv_heads, page_rows, d) if heads_first else (total, page_rows, kv_heads, d)
    caches = [torch.full(shape, fill, dtype=keys[0].dtype, device=device) for _ in range(2)]
    caches = [c.transpose(1, 2) if heads_first else c for c in caches]
    table = torch.full((len(keys), pages), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        for p in range(n):
            page = order[at]
            at += 1
            table[b, p] = page
            for cache, x in ((caches[0], keys[b]), (caches[1], values[b])):
                part = x[p * page_rows:(p + 1) * page_rows]
                cache[page, :part.shape[0]] = part.to(device)
    return caches[0], caches[1], table.to(device)
