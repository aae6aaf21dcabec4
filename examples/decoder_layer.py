"""A decoder layer's attention as a serving program runs it: prompts of different lengths packed into one call, then one token at a time for all
sequences, the step captured into a HIP graph once and replayed, with a paged cache that grows as it goes.

    python examples/decoder_layer.py [--tokens 64] [--batch 8] [--longest 1500]

Weights and inputs are random.  At the end the last token's attention is taken again in 64 bits on the host from the cache itself.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2311_09549_amd.attention import Attention  # noqa: E402

HEADS, KV_HEADS, HEAD_DIM, PAGE_ROWS = 16, 4, 64, 32


class Layer:
    """Projections around the operators, and the cache with its table of pages."""

    def __init__(self, lengths, room, dtype, device):
        width = HEADS * HEAD_DIM
        self.attention = Attention(HEADS, KV_HEADS, HEAD_DIM, dtype, PAGE_ROWS, rotary_dim=HEAD_DIM, device=device)
        self.into = (torch.randn(width, (HEADS + 2 * KV_HEADS) * HEAD_DIM, device=device) / math.sqrt(width)).to(dtype)
        self.out_of = (torch.randn(width, width, device=device) / math.sqrt(width)).to(dtype)
        columns = -(-room // PAGE_ROWS)
        pages = len(lengths) * columns
        self.keys, self.values = (torch.zeros(pages, PAGE_ROWS, KV_HEADS, HEAD_DIM, dtype=dtype, device=device) for _ in range(2))
        self.pages = torch.randperm(pages, device=device).to(torch.int32).view(len(lengths), columns)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device=device)

    def _project(self, x):
        qkv = (x @ self.into).view(len(x), HEADS + 2 * KV_HEADS, HEAD_DIM)
        return qkv.split((HEADS, KV_HEADS, KV_HEADS), dim=1)   # views of one projection

    def prompt(self, x, row_start):
        q, k, v = self._project(x)
        q = self.attention.append(q, k, v, self.keys, self.values, self.pages, self.lengths, row_start)
        y = self.attention.prompt_paged(q, self.keys, self.values, self.pages, self.lengths, row_start)
        return x + y.flatten(1) @ self.out_of

    def token(self, x):
        self.lengths += 1   # on the device: a replay counts on
        self.q, k, v = self._project(x)
        self.q = self.attention.append(self.q, k, v, self.keys, self.values, self.pages, self.lengths)
        self.y = self.attention.decode(self.q, self.keys, self.values, self.pages, self.lengths)
        return x + self.y.flatten(1) @ self.out_of


def exact(layer, b):
    """Attention of the last token of sequence b in 64 bits, from what the cache holds."""
    n = int(layer.lengths[b])
    page = layer.pages[b, :-(-n // PAGE_ROWS)].long().cpu()
    k, v = (cache.cpu()[page].flatten(0, 1)[:n].double().repeat_interleave(HEADS // KV_HEADS, dim=1) for cache in (layer.keys, layer.values))
    q = layer.q[b].double().cpu()
    weights = torch.softmax((k * q).sum(-1) / math.sqrt(HEAD_DIM), dim=0)
    return (weights[..., None] * v).sum(0), (weights[..., None] * v.abs()).sum(0)


def main(tokens=64, batch=8, longest=1500, dtype=torch.bfloat16, device="cuda:0"):
    """Returns the worst error of the last token's attention, as a part of what rounding may give."""
    torch.manual_seed(0)
    lengths = [max(1, longest * (b + 1) ** 2 // batch ** 2) for b in range(batch)]
    layer = Layer(lengths, longest + tokens + 1, dtype, device)
    starts = torch.tensor([0] + lengths, device=device).cumsum(0).to(torch.int32)
    x = torch.randn(sum(lengths), HEADS * HEAD_DIM, device=device).to(dtype)
    layer.prompt(x, starts)   # the first call makes the workspace
    torch.cuda.synchronize()
    begin = time.perf_counter()
    y = layer.prompt(x, starts)
    torch.cuda.synchronize()
    print(f"{batch} prompts, {sum(lengths)} rows: {(time.perf_counter() - begin) * 1e6:.0f} us")

    state = y[starts[1:].long() - 1].clone()   # the last row of each prompt
    layer.token(state)                         # eagerly once: it makes what a captured step may not make
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        state.copy_(torch.nn.functional.normalize(layer.token(state).float(), dim=-1) * math.sqrt(HEADS * HEAD_DIM))
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(tokens):
        graph.replay()
    torch.cuda.synchronize()
    print(f"{tokens} tokens for {batch} sequences: {(time.perf_counter() - begin) * 1e6 / tokens:.1f} us a token")
    assert layer.lengths.tolist() == [n + 1 + tokens for n in lengths]

    worst, step = 0.0, torch.finfo(dtype).eps / 2
    for b in range(batch):
        want, size = exact(layer, b)
        # half a step for each weight and for the result, and fp32 sums
        worst = max(worst, float(((layer.y[b].double().cpu() - want).abs() / (1.05 * step * (size + want.abs()) + 1e-4 * size)).max()))
    print(f"last token against 64 bits: {worst:.2f} of what rounding may give")
    return worst


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    for name, default in (("tokens", 64), ("batch", 8), ("longest", 1500)):
        parser.add_argument("--" + name, type=int, default=default)
    if not main(**vars(parser.parse_args())) <= 1.0:
        sys.exit(1)
