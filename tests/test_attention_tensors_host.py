"""What attention on torch tensors hands to the library and what it refuses, without a GPU: records of tensors instead of tensors, and a recorder instead of
the library's operators."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2311_09549_amd import attention as module
from paper_2311_09549_amd.attention import Attention

BF16, F32 = torch.bfloat16, torch.float32
A = 1 << 20   # an address that is a multiple of 256; nothing is launched here, so nothing is read
STREAM = 4096   # that of a HIP stream, for a recorder


def side_by_side(shape):
    strides = [1]
    for n in reversed(shape[1:]):
        strides.insert(0, strides[0] * n)
    return tuple(strides)


class Record:
    """What is read of a tensor."""

    def __init__(self, *shape, dtype=BF16, index=0, strides=None, address=A, requires_grad=False):
        self.shape, self.dtype, self.requires_grad, self._index, self._address = torch.Size(shape), dtype, requires_grad, index, address
        self.device = torch.device("cpu") if index < 0 else torch.device("cuda", index)
        self._strides = strides or side_by_side(shape)

    def stride(self):
        return self._strides

    def get_device(self):
        return self._index

    def data_ptr(self):
        return self._address

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self._strides == side_by_side(self.shape)


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    """Torch does not know a current device where there is none."""
    monkeypatch.setattr(module, "_current_device", lambda: 0, raising=False)


class Recorder:
    """In the place of an operator of the library."""

    def __init__(self):
        self.calls = []

    def __call__(self, *args):
        self.calls.append(args)
        return 0


def recorded(heads=4, kv_heads=2, head_dim=64, dtype=BF16, **kw):
    attention, recorder = Attention(heads, kv_heads, head_dim, dtype, 16, **kw), Recorder()
    attention._append = attention._prompt = attention._prompt_paged = attention._decode = recorder
    return attention, recorder


def paged(rows, heads=4, kv_heads=2, head_dim=64, dtype=BF16, batch=None):
    """Arguments of prompt_paged and decode but for row_start."""
    batch = rows if batch is None else batch
    cache = Record(9, 16, kv_heads, head_dim, dtype=dtype)
    return Record(rows, heads, head_dim, dtype=dtype), cache, cache, Record(batch, 5, dtype=torch.int32), Record(batch, dtype=torch.int32)


def packed(rows, heads=4, kv_heads=2, head_dim=64, dtype=BF16):
    key = Record(rows, kv_heads, head_dim, dtype=dtype)
    return Record(rows, heads, head_dim, dtype=dtype), key, key, Record(2, dtype=torch.int32)


BAD_WORKSPACES = [
    (torch.empty(1 << 20, dtype=torch.uint8), TypeError),                         # host memory
    (Record(1 << 27, dtype=torch.uint8, index=-1), TypeError),
    (Record(1 << 27, dtype=torch.uint8, index=1), TypeError),                      # of another GPU
    (Record(1 << 27, dtype=torch.uint8, strides=(0,)), ValueError),                # one byte that stands for all
    (Record(1 << 14, 1 << 13, dtype=torch.uint8, strides=(1 << 14, 1)), ValueError),   # with other memory between its rows
]


@pytest.mark.parametrize("workspace,error", BAD_WORKSPACES)
def test_workspace_refusals(workspace, error):
    """Kernels write to a workspace: nothing but memory of the handle's GPU, all of it the caller's."""
    attention, recorder = recorded()
    rows, table, starts = paged(3), paged(3, batch=1), Record(2, dtype=torch.int32)
    out = Record(3, 4, 64)
    for call in (lambda: attention.decode(*rows, out=out, workspace=workspace, stream=STREAM),
                 lambda: attention.prompt_paged(*table, starts, out=out, workspace=workspace, stream=STREAM),
                 lambda: attention.prompt(*packed(3), out=out, workspace=workspace, stream=STREAM)):
        with pytest.raises(error):
            call()
    assert not recorder.calls


def test_workspace_of_the_caller():
    attention, recorder = recorded()
    workspace = Record(attention.ws_bytes // 4, dtype=F32, address=3 * A)
    attention.decode(*paged(3), out=Record(3, 4, 64), workspace=workspace, stream=STREAM)
    assert recorder.calls[0][-3:] == (3 * A, attention.ws_bytes, STREAM)


class Memory:
    """Torch's streams and memory for a recorder: which stream was current when a tensor was made, and which streams it was told of."""

    def __init__(self, monkeypatch, current):
        self.current, self.made, self.told = current, [], {}
        memory = self

        class Made(Record):
            def record_stream(self, stream):
                memory.told.setdefault(self.data_ptr(), []).append(stream)

        class On:
            def __init__(self, stream):
                self.stream = stream

            def __enter__(self):
                self.before, memory.current = memory.current, self.stream

            def __exit__(self, *error):
                memory.current = self.before

        def empty(*shape, dtype, device):
            assert torch.device(device) == torch.device("cuda", 0)
            memory.made.append((memory.current, Made(*(shape[0] if isinstance(shape[0], (tuple, torch.Size)) else shape), dtype=dtype, address=(10 + len(memory.made)) * A)))
            return memory.made[-1][1]

        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda address, device=None: address)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: memory.current)
        monkeypatch.setattr(torch.cuda, "stream", On)
        monkeypatch.setattr(torch, "empty", empty)
        monkeypatch.setattr(module, "_empty_like", lambda x: empty(x.shape, dtype=x.dtype, device=x.device))
        monkeypatch.setattr(module, "_raw_stream", lambda index: memory.current)


def test_own_workspace_belongs_to_the_stream_that_uses_it(monkeypatch):
    """Memory of torch's current stream may still be in use there, by kernels that those of another stream do not wait for."""
    attention, recorder = recorded()
    rows, long, out = paged(3), packed(2000), Record(3, 4, 64)
    memory = Memory(monkeypatch, 7)
    attention.decode(*rows, out=out, stream=STREAM)
    attention.prompt(*long, out=Record(2000, 4, 64))
    assert [on for on, _ in memory.made] == [STREAM, 7]
    attention.decode(*rows, out=out, stream=STREAM)
    assert len(memory.made) == 2 and not memory.told
    attention.decode(*rows, out=out)                    # the current one: not given away before that is done with it
    attention.decode(*rows, out=out)
    address = memory.made[0][1].data_ptr()
    assert memory.told == {address: [7]}
    assert [call[-3] for call in recorder.calls if call[-2] == attention.ws_bytes] == [address] * 4


def test_results_belong_to_the_stream_of_their_call(monkeypatch):
    """Results that are made for another stream than the current one are memory of that stream, not given away before the current one is done with them."""
    attention, recorder = recorded()
    rows, table, starts, long, cache = paged(3), paged(3, batch=1), Record(2, dtype=torch.int32), packed(3), Record(9, 16, 2, 64)
    workspace = Record(1 << 27, dtype=torch.uint8)

    def append(**kw):
        return attention.append(*long[:3], cache, cache, Record(3, 5, dtype=torch.int32), Record(3, dtype=torch.int32), **kw)

    calls = (append, lambda **kw: attention.prompt(*long, **kw), lambda **kw: attention.prompt_paged(*table, starts, workspace=workspace, **kw),
             lambda **kw: attention.decode(*rows, workspace=workspace, **kw))
    for call in calls:
        memory = Memory(monkeypatch, 7)
        made = [call(), call(stream=7), call(stream=STREAM)]
        assert [on for on, _ in memory.made] == [7, 7, STREAM] and [x for _, x in memory.made] == made
        assert memory.told == {made[2].data_ptr(): [7]} and memory.current == 7
        out = Record(3, 4, 64)
        assert call(out=out, stream=STREAM) is out and len(memory.made) == 3


class Devices:
    """Torch's current device for a recorder."""

    def __init__(self, monkeypatch, current):
        self.current, devices = current, self

        class On:
            def __init__(self, index):
                self.index = torch.device("cuda", index).index if isinstance(index, int) else index.index

            def __enter__(self):
                self.before, devices.current = devices.current, self.index

            def __exit__(self, *error):
                devices.current = self.before

        monkeypatch.setattr(torch.cuda, "device", On)
        monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.current)
        monkeypatch.setattr(module, "_current_device", lambda: self.current, raising=False)


@pytest.mark.parametrize("current", [0, 2])
def test_calls_are_made_on_the_device_of_the_handle(monkeypatch, current):
    """A kernel is queued on the current device, whatever its operands are memory of."""
    attention, _ = recorded()
    devices, at = Devices(monkeypatch, current), []
    attention._append = attention._prompt = attention._prompt_paged = attention._decode = lambda *args: at.append(devices.current) or 0
    rows, table, starts, long, out, workspace = paged(3), paged(3, batch=1), Record(2, dtype=torch.int32), packed(3), Record(3, 4, 64), Record(1 << 27, dtype=torch.uint8)
    cache = Record(9, 16, 2, 64)
    assert attention.append(*long[:3], cache, cache, Record(3, 5, dtype=torch.int32), Record(3, dtype=torch.int32), out=out, stream=STREAM) is out
    assert attention.prompt(*long, out=out, stream=STREAM) is out
    assert attention.prompt_paged(*table, starts, out=out, workspace=workspace, stream=STREAM) is out
    assert attention.decode(*rows, out=out, workspace=workspace, stream=STREAM) is out
    assert at == [0] * 4 and devices.current == current


@pytest.mark.parametrize("device,index", [("cuda:1", 1), ("cuda:0", 0), ("cuda", 2)])
def test_handle_is_made_on_its_device(monkeypatch, device, index):
    """The library reads how many compute units the current device has."""
    devices, at = Devices(monkeypatch, 2), []
    create = module.sc.attention_create
    monkeypatch.setattr(module.sc, "attention_create", lambda *args: at.append(devices.current) or create(*args))
    attention = Attention(4, 2, 64, device=device)
    assert at == [index] and devices.current == 2 and attention.device == torch.device("cuda", index)


def test_device_refusals():
    with pytest.raises(ValueError):
        Attention(4, 2, 64, device="cpu")


def operators(attention, q, k, v, keys, values, out=None):
    """Calls of every operator with these operands, where it has them."""
    rows, table, lengths, starts = q.shape[0], Record(3, 5, dtype=torch.int32), Record(3, dtype=torch.int32), Record(2, dtype=torch.int32)
    workspace, kw = Record(1 << 27, dtype=torch.uint8), dict(out=out or Record(3, 4, 64), stream=STREAM)
    return {
        "append": lambda: attention.append(q, k, v, keys, values, table, lengths, **kw),
        "prompt": lambda: attention.prompt(q, k, v, starts, **kw),
        "prompt_paged": lambda: attention.prompt_paged(q, keys, values, Record(1, 5, dtype=torch.int32), Record(1, dtype=torch.int32), starts, workspace=workspace, **kw),
        "decode": lambda: attention.decode(q, keys, values, table, lengths, workspace=workspace, **kw),
    }


TAKES = dict(q=("append", "prompt", "prompt_paged", "decode"), k=("append", "prompt"), v=("append", "prompt"), keys=("append", "prompt_paged", "decode"),
             values=("append", "prompt_paged", "decode"), out=("append", "prompt", "prompt_paged", "decode"))


@pytest.mark.parametrize("name", sorted(TAKES))
def test_operands_that_require_a_gradient(name):
    """There is no backward pass: results would be without a gradient, silently."""
    attention, recorder = recorded()
    cache = (9, 16, 2, 64)
    shapes = dict(q=(3, 4, 64), k=(3, 2, 64), v=(3, 2, 64), keys=cache, values=cache, out=(3, 4, 64))
    operands = {n: Record(*shape, requires_grad=n == name) for n, shape in shapes.items()}
    for op, call in operators(attention, **operands).items():
        if op in TAKES[name]:
            with pytest.raises(RuntimeError, match="gradient"):
                call()
    assert not recorder.calls or name in ("k", "v", "keys", "values")
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            for call in operators(attention, **operands).values():
                call()


def test_operands_with_a_tangent(monkeypatch):
    attention, recorder = recorded()
    dual, plain = Record(3, 4, 64), {n: Record(*s) for n, s in dict(k=(3, 2, 64), v=(3, 2, 64), keys=(9, 16, 2, 64), values=(9, 16, 2, 64)).items()}
    monkeypatch.setattr(forward_ad, "unpack_dual", lambda x: forward_ad.UnpackedDualTensor(x, x if x is dual else None))
    for call in operators(attention, dual, **plain).values():
        call()   # at no level there is none
    with forward_ad.dual_level():
        for call in operators(attention, dual, **plain).values():
            with pytest.raises(RuntimeError, match="tangent"):
                call()
        for call in operators(attention, Record(3, 4, 64), **plain).values():
            call()
    assert len(recorder.calls) == 8


@pytest.mark.parametrize("head_dim,rows", [(256, 129), (136, 416), (256, 512), (128, 513), (64, 2000)])
def test_prompts_that_may_be_split_have_a_workspace(monkeypatch, head_dim, rows):
    """Whether a packed prompt is split is the library's to say, from five tiles of keys on: 32 keys above a head size of 128, else 128."""
    attention, recorder = recorded(head_dim=head_dim)
    memory = Memory(monkeypatch, 7)
    attention.prompt(*packed(rows, head_dim=head_dim), out=Record(rows, 4, head_dim))
    assert recorder.calls[0][-3:] == (memory.made[0][1].data_ptr(), attention.prompt_ws_bytes, 7)


@pytest.mark.parametrize("head_dim,rows", [(256, 128), (128, 512), (8, 1)])
def test_prompts_that_are_never_split_have_none(head_dim, rows):
    attention, recorder = recorded(head_dim=head_dim)
    attention.prompt(*packed(rows, head_dim=head_dim), out=Record(rows, 4, head_dim), stream=STREAM)
    assert recorder.calls[0][-3:] == (None, 0, STREAM)


def test_append_without_queries_has_no_result():
    """A place for rotated queries without queries would be given back as it was."""
    attention, recorder = recorded()
    rows = Record(3, 2, 64), Record(3, 2, 64), Record(9, 16, 2, 64), Record(9, 16, 2, 64), Record(3, 5, dtype=torch.int32), Record(3, dtype=torch.int32)
    assert attention.append(None, *rows, stream=STREAM) is None and len(recorder.calls) == 1
    with pytest.raises(ValueError, match="queries"):
        attention.append(None, *rows, out=Record(3, 4, 64), stream=STREAM)
    assert len(recorder.calls) == 1
