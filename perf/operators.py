"""Timing cases of the attention operators: what a serving program has the library do in one step of a decoder layer.

Three operators share a paged cache of keys and values: `append` rotates new queries and keys by their positions and stores keys
and values in the pages of their sequences, `prompt` is the causal attention of whole prompts (packed, or of a chunk behind what the
cache already holds), `decode` is the attention of one new row per sequence over the cache.

A case names an operator, a type, the head layout, the lengths and the page size; lengths are drawn from the case alone, so that the
work of a case does not depend on the seed.  `run` computes the operator from elementary torch operations in 32 bits, or, where
`own` is true, through `paper_2311_09549_amd.attention.Attention`.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
THETA = 10000.0


def _case(name, op, dtype, heads, kv_heads, head_dim, batch, longest, *, rows=1, page_rows=16, paged=False, rotary_dim=0,
          interleaved=False, causal=True, heads_first=False):
    """`longest`: the longest sequence (of keys); `rows`: the most new rows of a sequence (append, and prompt with paged keys);
    `heads_first`: pages laid out head by head."""
    case = dict(op=op, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, batch=batch, longest=longest, rows=rows,
                page_rows=page_rows, paged=paged, rotary_dim=rotary_dim, interleaved=interleaved, causal=causal, heads_first=heads_first)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # the new token of a single conversation: the smallest call there is, its latency is what counts
        _case("append-one", "append", "bf16", 32, 8, 128, 1, 1001, rotary_dim=128),
        # one decoding step of a batch in fp16
        _case("append-batch-f16", "append", "f16", 16, 4, 64, 48, 4095, page_rows=32, rotary_dim=64),
        # the prompts of seven requests at once, half of each head rotated, in adjacent pairs
        _case("append-prompt", "append", "bf16", 32, 8, 128, 7, 2047, rows=2047, rotary_dim=64, interleaved=True),
        # a short question to a small model in fp16, every head with keys of its own
        _case("prompt-short-f16", "prompt", "f16", 12, 12, 64, 1, 77),
        # twelve prompts of very different lengths, packed
        _case("prompt-ragged", "prompt", "bf16", 32, 8, 128, 12, 2048),
        # one long document
        _case("prompt-long", "prompt", "bf16", 16, 4, 128, 1, 16384),
        # a check in full precision, odd lengths, a head size between the usual ones
        _case("prompt-f32", "prompt", "f32", 8, 2, 96, 5, 777),
        # the next chunk of four prompts, behind what their pages hold already
        _case("prompt-chunk-paged", "prompt", "bf16", 32, 8, 128, 4, 8191, rows=509, page_rows=64, paged=True),
        # the next token of one short conversation
        _case("decode-one", "decode", "bf16", 32, 8, 128, 1, 333),
        # a decoding step of a full batch in fp16, lengths from short to long
        _case("decode-batch-f16", "decode", "f16", 32, 8, 128, 64, 8191),
        # the next token behind one very long document
        _case("decode-long", "decode", "bf16", 64, 8, 128, 1, 131071, page_rows=64, heads_first=True),
        # full precision, every head with keys of its own, an odd head size
        _case("decode-f32", "decode", "f32", 16, 16, 80, 24, 1500, page_rows=32),
    ]


def _lengths(case):
    """Keys and new rows of each sequence: the longest among them, the others log-uniform below it, most within a factor of 32."""
    rng = random.Random("lengths %s" % sorted((k, v) for k, v in case.items() if k != "name"))
    longest, batch = case["longest"], case["batch"]
    keys = [longest]
    for _ in range(batch - 1):
        least = 1.0 if rng.random() < 0.125 else max(1.0, longest / 32)
        keys.append(int(math.exp(rng.uniform(math.log(least), math.log(longest + 0.5)))))
    rng.shuffle(keys)
    if case["op"] == "prompt" and not case["paged"]:
        return keys, list(keys)
    return keys, [min(n, case["rows"]) if case["rows"] == 1 else min(n, rng.randint((case["rows"] + 1) // 2, case["rows"])) for n in keys]


def _pairs(case):
    """(row, key) pairs that attention visits, per head."""
    pairs = 0
    for n, r in zip(*_lengths(case)):
        pairs += r * n - (r * (r - 1) // 2 if case["causal"] else 0)
    return pairs


def work(case):
    keys, rows = _lengths(case)
    size = TYPES[case["dtype"]].itemsize
    h, g, d = case["heads"], case["kv_heads"], case["head_dim"]
    tables = 4 * (2 * case["batch"] + 1)
    if case["op"] == "append":
        return {"bytes": 2 * sum(rows) * (h + 2 * g) * d * size + tables + 4 * sum(rows),
                "flops": 6 * sum(rows) * (h + g) * case["rotary_dim"] / 2}
    pages = sum(-(-n // case["page_rows"]) for n in keys) if case["op"] == "decode" or case["paged"] else 0
    return {"bytes": 2 * sum(rows) * h * d * size + 2 * sum(keys) * g * d * size + tables + 4 * pages,
            "flops": 4 * _pairs(case) * h * d}


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator and type, groups of 1 to 16 heads, head sizes of every multiple of 8 up to 256, one to 96
    sequences, one token to the longest listed lengths."""
    most = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        op = rng.choice(("append", "prompt", "decode"))
        head_dim = rng.choice((64, 64, 128, 128, 128, 8 * rng.randint(2, 32)))
        kv_heads = rng.choice((1, 2, 3, 4, 8, 8, 16))
        heads = kv_heads * rng.choice((1, 1, 2, 4, 4, 5, 7, 8, 16))
        paged = op == "prompt" and rng.random() < 0.4
        longest = _log_uniform(rng, 1, {"append": 16384, "prompt": 16384, "decode": 131071}[op])
        case = _case(None, op, rng.choice(("bf16", "bf16", "f16", "f32")), heads, kv_heads, head_dim, _log_uniform(rng, 1, 96), longest,
                     rows=_log_uniform(rng, 1, longest) if paged or (op == "append" and rng.random() < 0.5) else 1,
                     page_rows=rng.choice((16, 16, 32, 64, 128)), paged=paged,
                     rotary_dim=rng.choice((head_dim, head_dim, head_dim // 2, 0)) if op == "append" else 0,
                     interleaved=rng.random() < 0.3, causal=op != "prompt" or rng.random() < 0.8, heads_first=rng.random() < 0.3)
        w = work(case)
        keys, rows = _lengths(case)
        # the plain form holds every score of the padded batch, and the cache of `append` is an output as a whole
        scores = case["batch"] * heads * max(rows) * longest if op != "append" else 0
        held = 2 * sum(keys) * kv_heads * head_dim * TYPES[case["dtype"]].itemsize
        if heads <= 64 and w["bytes"] <= most_bytes and w["flops"] <= most_flops and scores <= 16 * 16384 ** 2 and held <= most_bytes \
                and case["batch"] * longest * kv_heads * head_dim <= 64 * 8192 * 8 * 128:
            return case


def _pages_in_all(case):
    keys, _ = _lengths(case)
    return sum(-(-n // case["page_rows"]) for n in keys) + 3


def prepare(case, seed):
    """Projections as a layer hands them over, and the cache of the sequences.  Scores have a spread of about two, some
    channels are larger than the others, the first key draws attention and values have a mean."""
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    h, g, d, r = case["heads"], case["kv_heads"], case["head_dim"], case["page_rows"]
    keys, rows = _lengths(case)
    total = sum(rows)

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, dtype=torch.float32, generator=gen)

    channel = 1.0 + normal(d).square() * 0.25
    state = dict(case=case, heads=h, kv_heads=g, head_dim=d, longest=max(keys), most_rows=max(rows), scale=1.0 / math.sqrt(d))
    # one projection holds queries, keys and values of a row side by side
    qkv = normal(total, h + 2 * g, d) * channel
    qkv[:, :h] += 0.5 * normal(1, h, d)
    qkv[:, h + g:] += 0.25
    qkv = qkv.to(dtype)
    state["q"], state["k"], state["v"] = qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:]
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    state["row_start"] = torch.tensor(starts, dtype=torch.int32, device=DEVICE)
    state["lengths"] = torch.tensor(keys, dtype=torch.int32, device=DEVICE)
    if case["rotary_dim"]:
        half = case["rotary_dim"] // 2
        state["freq"] = [THETA ** (-t / half) for t in range(half)]
        state["freq_on_device"] = torch.tensor(state["freq"], dtype=torch.float64, device=DEVICE)
    if case["op"] != "prompt" or case["paged"]:
        count = _pages_in_all(case)
        order = torch.randperm(count, device=DEVICE, generator=gen).to(torch.int32)
        widest = -(-max(keys) // r)
        table, at = torch.zeros(len(keys), widest, dtype=torch.int32, device=DEVICE), 0
        for b, n in enumerate(keys):
            used = -(-n // r)
            table[b, :used] = order[at:at + used]
            at += used
        state["pages"] = table
        for name in ("keys", "values"):
            cache = normal(count, g, r, d) if case["heads_first"] else normal(count, r, g, d)
            cache = (cache * channel + (0.25 if name == "values" else 0.0)).to(dtype)
            state[name] = cache.transpose(1, 2) if case["heads_first"] else cache
    return state


# ---------------------------------------------------------------------------------------------------------------------------
# the operators from elementary torch operations, in 32 bits
# ---------------------------------------------------------------------------------------------------------------------------
def _rows_of(state):
    """Sequence and position of every new row."""
    starts, lengths = state["row_start"].long(), state["lengths"].long()
    row = torch.arange(state["q"].shape[0], device=DEVICE)
    seq = torch.searchsorted(starts, row, right=True) - 1
    return seq, lengths[seq] - starts[seq + 1] + row


def _rotated(x, position, freq, interleaved):
    """x (rows, heads, head_dim) rotated by position * freq in its first 2 * len(freq) channels; angles in 64 bits."""
    half = freq.shape[0]
    angle = position.double()[:, None] * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float().clone()
    first, second = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if interleaved else (y[..., :half], y[..., half:2 * half])
    one, two = first * cos - second * sin, second * cos + first * sin
    first.copy_(one)
    second.copy_(two)
    return y.to(x.dtype)


def _plain_append(state):
    seq, position = _rows_of(state)
    r = state["keys"].shape[1]
    page = state["pages"].long()[seq, position // r]
    q, k = state["q"], state["k"]
    if "freq" in state:
        q = _rotated(q, position, state["freq_on_device"], state["case"]["interleaved"])
        k = _rotated(k, position, state["freq_on_device"], state["case"]["interleaved"])
    state["keys"][page, position % r] = k
    state["values"][page, position % r] = state["v"]
    return q, state["keys"], state["values"]


def _attend(q, k, v, rows, lengths, scale, causal):
    """q (batch, R, heads, d), k and v (batch, N, kv_heads, d), all padded: the last `rows` of `lengths` positions are q's."""
    batch, most, h, d = q.shape
    n, g = k.shape[1], k.shape[2]
    grouped = q.float().reshape(batch, most, g, h // g, d).permute(0, 2, 3, 1, 4).reshape(batch, g, h // g * most, d)
    scores = torch.matmul(grouped, k.float().permute(0, 2, 3, 1).contiguous()).mul_(scale)
    scores = scores.view(batch, g, h // g, most, n)
    j = torch.arange(n, device=q.device)
    seen = (j < lengths[:, None])[:, None, :].expand(batch, most, n)
    if causal:
        position = (lengths - rows)[:, None] + torch.arange(most, device=q.device)
        seen = seen & (j <= position[:, :, None])
    hidden = ~seen[:, None, None]
    scores.masked_fill_(hidden, -math.inf)
    top = scores.amax(-1, keepdim=True)
    weights = scores.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights.view(batch, g, h // g * most, n), v.float().permute(0, 2, 1, 3).contiguous())
    out = out.view(batch, g, h // g, most, d) / torch.where(total == 0.0, 1.0, total)
    return out.permute(0, 3, 1, 2, 4).reshape(batch, most, h, d).to(q.dtype)


def _paged(state):
    """Keys and values of the sequences, padded to the longest."""
    r = state["keys"].shape[1]
    j = torch.arange(state["longest"], device=DEVICE)
    page = state["pages"].long()[:, j // r]
    return state["keys"][page, j % r], state["values"][page, j % r]


def _plain_prompt(state):
    starts, lengths = state["row_start"].long(), state["lengths"].long()
    rows = starts[1:] - starts[:-1]
    total = state["q"].shape[0]
    padded = (starts[:-1, None] + torch.arange(state["most_rows"], device=DEVICE)).clamp_(max=total - 1)
    k, v = _paged(state) if state["case"]["paged"] else (state["k"][padded], state["v"][padded])
    out = _attend(state["q"][padded], k, v, rows, lengths, state["scale"], state["case"]["causal"])
    seq, position = _rows_of(state)
    return out[seq, position - (lengths - rows)[seq]]


def _plain_decode(state):
    k, v = _paged(state)
    lengths = state["lengths"].long()
    return _attend(state["q"][:, None], k, v, torch.ones_like(lengths), lengths, state["scale"], True)[:, 0]


# ---------------------------------------------------------------------------------------------------------------------------
# the same through the framework
# ---------------------------------------------------------------------------------------------------------------------------
def _handle(state):
    """The handle that a program keeps for its layers."""
    from paper_2311_09549_amd.attention import Attention

    case = state["case"]
    return Attention(case["heads"], case["kv_heads"], case["head_dim"], dtype=state["q"].dtype, page_rows=case["page_rows"],
                     causal=case["causal"], rotary_freq=state.get("freq"), interleaved=case["interleaved"], device=DEVICE)


def _own(state):
    attention = state.get("handle")
    if attention is None:
        attention = state["handle"] = _handle(state)
    op = state["case"]["op"]
    if op == "append":
        q = attention.append(state["q"], state["k"], state["v"], state["keys"], state["values"], state["pages"], state["lengths"],
                             state["row_start"])
        return q, state["keys"], state["values"]
    if op == "decode":
        return attention.decode(state["q"], state["keys"], state["values"], state["pages"], state["lengths"])
    if state["case"]["paged"]:
        return attention.prompt_paged(state["q"], state["keys"], state["values"], state["pages"], state["lengths"], state["row_start"])
    return attention.prompt(state["q"], state["k"], state["v"], state["row_start"])


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "prompt": _plain_prompt, "decode": _plain_decode}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------------------------------------------------------
def _turned(x, position, freq, interleaved):
    """Channels taken as complex numbers and multiplied by exp(i * position * freq)."""
    x = x.double().clone()
    n = 2 * len(freq)
    turn = torch.polar(torch.ones(len(position), len(freq), dtype=torch.float64, device=DEVICE),
                       torch.outer(position.double(), torch.tensor(freq, dtype=torch.float64, device=DEVICE)))[:, None, :]
    pairs = x[..., :n].unflatten(-1, (n // 2, 2)) if interleaved else x[..., :n].unflatten(-1, (2, n // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    x[..., :n] = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return x


def exact(case, seed):
    state = prepare(case, seed)
    lengths, starts = state["lengths"].tolist(), state["row_start"].tolist()
    r = case["page_rows"]
    if case["op"] == "append":
        q, keys, values = state["q"].double(), state["keys"].double(), state["values"].double()
        for b, n in enumerate(lengths):
            lo, hi = starts[b], starts[b + 1]
            position = torch.arange(n - (hi - lo), n, device=DEVICE)
            k = state["k"][lo:hi]
            if "freq" in state:
                q[lo:hi] = _turned(state["q"][lo:hi], position, state["freq"], case["interleaved"])
                k = _turned(k, position, state["freq"], case["interleaved"])
            place = state["pages"][b].long()[torch.div(position, r, rounding_mode="floor")], position.remainder(r)
            keys[place] = k.double()
            values[place] = state["v"][lo:hi].double()
        return q, keys, values
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device=DEVICE)
    group = case["heads"] // case["kv_heads"]
    for b, n in enumerate(lengths):
        lo, hi = starts[b], starts[b + 1]
        if case["op"] == "prompt" and not case["paged"]:
            k, v = state["k"][lo:hi], state["v"][lo:hi]
        else:
            used = state["pages"][b, :-(-n // r)].long()
            k, v = (state[name][used].flatten(0, 1)[:n] for name in ("keys", "values"))
        later = torch.ones(hi - lo, n, dtype=torch.bool, device=DEVICE).triu_(n - (hi - lo) + 1) if case["causal"] else None
        for head in range(case["heads"]):
            kh, vh = k[:, head // group].double(), v[:, head // group].double()
            logits = state["q"][lo:hi, head].double() @ kh.T * state["scale"]
            if later is not None:
                logits[later] = -math.inf
            logits -= logits.max(1, keepdim=True).values
            logits.exp_()
            out[lo:hi, head] = logits @ vh / logits.sum(1, keepdim=True)
    return out
