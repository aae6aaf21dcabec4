"""What attention on torch tensors hands to the library and what it refuses, without a GPU: records of tensors instead of tensors, and a recorder instead of
the library's operators."""
import pytest
import torch

from paper_2311_09549_amd.attention import Attention

BF16, F32 = torch.bfloat16, torch.float32
A = 1 << 20   # an address that is a multiple of 256; nothing is launched here, so nothing is read
STREAM = 4096   # that of a HIP stream, for a recorder


class Record:
    """What is read of a tensor."""

    def __init__(self, *shape, dtype=BF16, index=0, strides=None, address=A, requires_grad=False):
        self.shape, self.dtype, self.requires_grad, self._index, self._address = torch.Size(shape), dtype, requires_grad, index, address
        self.device = torch.device("cpu") if index < 0 else torch.device("cuda", index)
        self._strides = strides or torch.empty(shape, device="meta").stride()

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
        return self._strides == torch.empty(self.shape, device="meta").stride()


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
