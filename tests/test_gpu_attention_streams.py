"""Attention queued on a stream that is not torch's current one."""
import pytest
import torch

from paper_2311_09549_amd.attention import Attention

from attention_reference import cache_of

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def operands():
    """Calls whose keys are split: of one long sequence in the cache, and of a long packed prompt."""
    gen = torch.Generator().manual_seed(1)
    k, v = (torch.randn(3000, 1, 64, generator=gen).to(BF16) for _ in range(2))
    kc, vc, table = cache_of([k], [v], 64, 50, gen, fill=0.0)
    q = torch.randn(1, 2, 64, generator=gen).to(BF16).cuda()
    rows = torch.randn(3000, 2, 64, generator=gen).to(BF16).cuda()
    return (q, kc, vc, table, int32([3000])), (rows, k.cuda(), v.cuda(), int32([0, 3000]))


def busy(gate):
    """Some milliseconds of work on the current stream."""
    for _ in range(20):
        gate = (gate @ gate).clamp_(-1.0, 1.0)
    return gate


def test_first_call_on_another_stream():
    """The workspaces are made while the current stream still reads memory that was freed on it, of their sizes."""
    token, prompt = operands()
    expected = Attention(2, 1, 64, BF16, 64)
    want = expected.decode(*token).clone(), expected.prompt(*prompt).clone()
    gate = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    side, ready = torch.cuda.Stream(), torch.cuda.Event()
    attention = Attention(2, 1, 64, BF16, 64)
    out = torch.empty_like(token[0]), torch.empty_like(prompt[0])
    ready.record()
    side.wait_event(ready)
    old = [torch.full((size // 4,), 3.0, device="cuda") for size in (attention.ws_bytes, attention.prompt_ws_bytes)]
    busy(gate)
    read = [x.clone() for x in old]     # queued behind that
    del old
    attention.decode(*token, out=out[0], stream=side.cuda_stream)
    attention.prompt(*prompt, out=out[1], stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert all(bool((x == 3.0).all()) for x in read)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_results_of_calls_on_another_stream():
    """Results are made while the current stream still reads memory that was freed on it, of their size."""
    token, prompt = operands()
    attention = Attention(2, 1, 64, BF16, 64)
    want = attention.prompt(*prompt).clone()
    gate = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    side, ready, done = torch.cuda.Stream(), torch.cuda.Event(), torch.cuda.Event()
    ready.record()
    side.wait_event(ready)
    old = torch.full_like(want, 3.0)
    busy(gate)
    read = old.clone()     # queued behind that
    del old
    got = attention.prompt(*prompt, stream=side.cuda_stream)
    done.record(side)
    torch.cuda.current_stream().wait_event(done)
    kept = got.clone()     # read on the current stream, behind its work, and freed
    del got
    for _ in range(3):
        attention.prompt(torch.zeros_like(prompt[0]), *prompt[1:], stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert bool((read == 3.0).all())
    assert torch.equal(kept, want)


@pytest.mark.parametrize("named", [False, True])
def test_first_call_in_a_capture(named):
    """A handle whose first calls are captured: its workspaces and results are the graph's memory, replays and eager calls beside them are right."""
    token, prompt = operands()
    expected = Attention(2, 1, 64, BF16, 64)
    want = expected.decode(*token).clone(), expected.prompt(*prompt).clone()
    torch.cuda.synchronize()
    attention, side, graph = Attention(2, 1, 64, BF16, 64), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    kw = dict(stream=side.cuda_stream) if named else {}
    with torch.cuda.graph(graph, stream=side):
        got = attention.decode(*token, **kw), attention.prompt(*prompt, **kw)
    for _ in range(3):
        for x in got:
            x.fill_(float("nan"))
        others = [torch.full((1 << 22,), 3.0, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(attention.decode(*token), want[0]) and torch.equal(attention.prompt(*prompt), want[1])
        torch.cuda.synchronize()
        assert all(bool((x == 3.0).all()) for x in others)
