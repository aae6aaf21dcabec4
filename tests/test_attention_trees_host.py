"""Windows, trees and pages without a GPU: what the entry points refuse, what tensors become on the way to them, and the index arithmetic of the kernels."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2311_09549_amd import attention as module
from paper_2311_09549_amd import binding as sc
from paper_2311_09549_amd.attention import Attention

from test_attention_tensors_host import Devices, Memory, Record, Recorder, recorded

HERE = os.path.dirname(os.path.abspath(__file__))
A = 1 << 20   # an address that is a multiple of 256; nothing is launched here, so nothing is read
STREAM = 4096
I32 = torch.int32


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    monkeypatch.setattr(module, "_current_device", lambda: 0, raising=False)


def _status(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except sc.ScError as e:
        return sc.STATUS_NAMES[e.status]
    return "SC_OK"


def _ready():
    return not torch.cuda.is_available()


def _create(**kw):
    return sc.attention_create(**dict(dict(dtype=sc.SC_BF16, heads=8, kv_heads=2, head_dim=128, page_rows=16), **kw))


@pytest.mark.parametrize("window,sinks,causal,status", [
    (1, 0, True, "SC_OK"), (2 ** 30, 2 ** 30, True, "SC_OK"), (0, 0, True, "SC_ERR_BAD_DIMS"), (-1, 0, True, "SC_ERR_BAD_DIMS"), (2 ** 30 + 1, 0, True, "SC_ERR_BAD_DIMS"),
    (5, -1, True, "SC_ERR_BAD_DIMS"), (5, 2 ** 30 + 1, True, "SC_ERR_BAD_DIMS"), (5, 0, False, "SC_ERR_BAD_DIMS"),
])
def test_create_window(window, sinks, causal, status):
    assert _status(_create, window=window, sinks=sinks, causal=causal) == status


def test_create_window_null():
    d = sc.AttentionDesc()
    assert sc.lib().sc_attention_create_window(None, ctypes.byref(d), 1, 0) == 1
    assert sc.lib().sc_attention_create_window(ctypes.byref(ctypes.c_void_p()), None, 1, 0) == 1


def test_a_window_says_so():
    assert "a window of 100 and the first 4" in sc.attention_describe(_create(window=100, sinks=4))
    assert "window" not in sc.attention_describe(_create())
    plain, windowed = _create(), _create(window=100)
    assert sc.attention_workspace_bytes(windowed) > sc.attention_workspace_bytes(plain)
    assert f"{sc.attention_tree_workspace_bytes(plain)} bytes" in sc.attention_describe(plain)


@pytest.mark.parametrize("kw", [dict(sinks=3), dict(window=5, causal=False), dict(window=2 ** 31), dict(window=3, sinks=-2 ** 31 - 1)])
def test_windows_of_tensors(kw):
    with pytest.raises(ValueError):
        Attention(4, 2, 64, **kw)


@pytest.mark.parametrize("kw", [dict(window=0), dict(window=-3), dict(window=5, sinks=-1)])
def test_wrong_windows_of_tensors(kw):
    with pytest.raises(sc.ScError, match="SC_ERR_BAD_DIMS"):
        Attention(4, 2, 64, **kw)


# -- entry points ------------------------------------------------------------------------------------------------------------------
def _sequences(batch=2, rows=10, row_start=A, length=A, page=A, page_ld=8, page_count=8):
    return sc.pack_sequences(batch, rows, row_start, length, page, page_ld, page_count)


def _rows(data=A, row=1024, head=128):
    return sc.pack_rows(data, row, head)


def _cache(keys=A, values=A, pages=10, page=16 * 256, row=256, head=128):
    return sc.pack_cache(keys, values, pages, page, row, head)


BAD_SEQUENCES = [
    (dict(batch=-1), "SC_ERR_BAD_DIMS"), (dict(rows=-1), "SC_ERR_BAD_DIMS"), (dict(rows=1 << 24), "SC_ERR_BAD_DIMS"), (dict(batch=1 << 20), "SC_ERR_BAD_DIMS"),
    (dict(length=0), "SC_ERR_NULL"), (dict(page=0), "SC_ERR_NULL"), (dict(page_ld=-1), "SC_ERR_BAD_DIMS"), (dict(page_count=-1), "SC_ERR_BAD_DIMS"),
    (dict(row_start=0), "SC_ERR_SHAPE_MISMATCH"),
]


def test_tree_refusals():
    h = _create()
    ws = sc.attention_tree_workspace_bytes(h)

    def call(sequences=_sequences(), parent=A, q=_rows(), cache=_cache(), out=_rows(), workspace=A, size=ws):
        return _status(sc.attention_tree, h, sequences, parent, q, cache, out, workspace, size)

    if _ready():
        assert call() == "SC_ERR_DEVICE" and call(parent=0) == "SC_ERR_DEVICE"
    for change, status in BAD_SEQUENCES:
        assert call(sequences=_sequences(**change)) == status, change
    assert call(size=ws - 1) == "SC_ERR_WORKSPACE_SMALL" and call(workspace=0) == "SC_ERR_NULL" and call(workspace=A + 16) == "SC_ERR_SHAPE_MISMATCH"
    assert call(q=None) == "SC_ERR_NULL" and call(cache=None) == "SC_ERR_NULL" and call(out=None) == "SC_ERR_NULL" and call(sequences=None) == "SC_ERR_NULL"
    assert call(out=_rows(row=0)) == "SC_ERR_SHAPE_MISMATCH" and call(q=_rows(data=A + 2)) == "SC_ERR_SHAPE_MISMATCH" and call(q=_rows(row=-8)) == "SC_ERR_BAD_DIMS"
    assert call(cache=_cache(page=256)) == "SC_ERR_SHAPE_MISMATCH" and call(cache=_cache(pages=0)) == "SC_ERR_BAD_DIMS"
    assert call(sequences=_sequences(rows=0)) == "SC_OK" and call(sequences=_sequences(batch=0, rows=0, length=0, page=0)) == "SC_OK"
    # more pairs of rows and heads than are numbered, and more units than the arithmetic of shares takes
    many = _create(heads=4096, kv_heads=1, head_dim=8)
    rows = sc.pack_rows(A, 4096 * 8, 8)
    for sequences in (_sequences(rows=(1 << 18) + 1), _sequences(batch=(1 << 20) - 1, rows=1 << 18, page_count=2 ** 31 - 1, page_ld=2 ** 31 - 1)):
        assert _status(sc.attention_tree, many, sequences, A, rows, sc.pack_cache(A, A, 10, 16 * 8, 8, 8), rows, A, sc.attention_tree_workspace_bytes(many)) == "SC_ERR_BAD_DIMS"


def test_append_tree_refusals():
    h = _create()
    k = _rows(row=256)

    def call(sequences=_sequences(), parent=A, q=_rows(), out=_rows(), key=k, cache=_cache()):
        return _status(sc.attention_append_tree, h, sequences, parent, q, key, k, out, cache)

    if _ready():
        assert call() == "SC_ERR_DEVICE" and call(q=None, out=None) == "SC_ERR_DEVICE"
    assert call(parent=0) == "SC_ERR_NULL" and call(q=None) == "SC_ERR_NULL" and call(key=None) == "SC_ERR_NULL"
    for change, status in BAD_SEQUENCES:
        assert call(sequences=_sequences(**change)) == status, change
    assert call(sequences=_sequences(rows=0)) == "SC_OK" and call(sequences=_sequences(rows=0), parent=0) == "SC_OK"
    assert call(sequences=None, parent=0) == "SC_ERR_NULL"


def test_accept_refusals():
    h = _create()

    def call(sequences=_sequences(), parent=A, last=2 * A, cache=_cache(), out=3 * A):
        return _status(sc.attention_accept, h, sequences, parent, last, cache, out)

    if _ready():
        assert call() == "SC_ERR_DEVICE" and call(out=0) == "SC_ERR_DEVICE"
    assert call(parent=0) == "SC_ERR_NULL" and call(last=0) == "SC_ERR_NULL" and call(cache=None) == "SC_ERR_NULL" and call(sequences=None) == "SC_ERR_NULL"
    for change, status in BAD_SEQUENCES:
        assert call(sequences=_sequences(**change)) == status, change
    apart = dict(row_start=4 * A, length=5 * A, page=6 * A)
    for place in (A, 2 * A, 4 * A, 5 * A, 6 * A, 6 * A + 4 * 15, 4 * A - 4):      # where something is read
        assert call(sequences=_sequences(**apart), out=place) == "SC_ERR_SHAPE_MISMATCH", place
    assert call(sequences=_sequences(batch=0, rows=0, length=0, page=0), last=0, parent=0) == "SC_OK"


PAGES = dict(batch=3, new_batch=4, pages=100, page=A, page_ld=8, page_count=7, length=2 * A, holders=3 * A, parent=4 * A, wanted=5 * A, page_out=6 * A, page_out_ld=7,
             length_out=7 * A, holders_out=8 * A, moves=9 * A)
COMPACT = dict(PAGES, new_batch=0, parent=0, wanted=0, length_out=0)
BAD_PAGES = [
    (dict(batch=-1), "SC_ERR_BAD_DIMS"), (dict(batch=1 << 20), "SC_ERR_BAD_DIMS"), (dict(pages=0), "SC_ERR_BAD_DIMS"), (dict(pages=2 ** 30 + 1), "SC_ERR_BAD_DIMS"),
    (dict(page_count=-1), "SC_ERR_BAD_DIMS"), (dict(page_count=2 ** 26 + 1), "SC_ERR_BAD_DIMS"), (dict(page_ld=-1), "SC_ERR_BAD_DIMS"), (dict(page_out_ld=-1), "SC_ERR_BAD_DIMS"),
    (dict(page_out_ld=6), "SC_ERR_SHAPE_MISMATCH"),
    (dict(page=0), "SC_ERR_NULL"), (dict(length=0), "SC_ERR_NULL"), (dict(holders=0), "SC_ERR_NULL"), (dict(page_out=0), "SC_ERR_NULL"), (dict(holders_out=0), "SC_ERR_NULL"),
    (dict(moves=0), "SC_ERR_NULL"),
    (dict(page_out=2 * A), "SC_ERR_SHAPE_MISMATCH"), (dict(holders_out=A), "SC_ERR_SHAPE_MISMATCH"), (dict(moves=3 * A), "SC_ERR_SHAPE_MISMATCH"),
    (dict(holders_out=3 * A + 4), "SC_ERR_SHAPE_MISMATCH"), (dict(moves=8 * A + 4 * 99), "SC_ERR_SHAPE_MISMATCH"), (dict(page_out=A + 4), "SC_ERR_SHAPE_MISMATCH"),
]


def _pages_call(name, record, **kw):
    h, size = _create(), sc.attention_pages_workspace_bytes(100, 4)
    kw = dict(dict(workspace=A << 8, size=size), **kw)
    return _status(getattr(sc, "attention_" + name), h, sc.pack_pages(*record.values()), kw["workspace"], kw["size"])


@pytest.mark.parametrize("name,record", [("fork", PAGES), ("compact", COMPACT)])
def test_pages_refusals(name, record):
    if _ready():
        for change in ({}, dict(holders_out=3 * A)):
            assert _pages_call(name, dict(record, **change)) == "SC_ERR_DEVICE"
    for change, status in BAD_PAGES:
        assert _pages_call(name, dict(record, **change)) == status, change
    assert _pages_call(name, record, size=255) == "SC_ERR_WORKSPACE_SMALL" and _pages_call(name, record, workspace=0) == "SC_ERR_NULL"
    assert _pages_call(name, record, workspace=A + 8) == "SC_ERR_SHAPE_MISMATCH"


def test_refusals_of_fork():
    for change, status in ((dict(new_batch=-1), "SC_ERR_BAD_DIMS"), (dict(parent=0), "SC_ERR_NULL"), (dict(length_out=0), "SC_ERR_NULL"), (dict(length_out=2 * A), "SC_ERR_SHAPE_MISMATCH"),
                           (dict(page_out=A), "SC_ERR_SHAPE_MISMATCH"), (dict(length_out=4 * A), "SC_ERR_SHAPE_MISMATCH"), (dict(moves=5 * A), "SC_ERR_SHAPE_MISMATCH")):
        assert _pages_call("fork", dict(PAGES, **change)) == status, change
    if _ready():
        assert _pages_call("fork", dict(PAGES, wanted=0)) == "SC_ERR_DEVICE"


def test_refusals_of_compact():
    for change in (dict(new_batch=4), dict(parent=4 * A), dict(wanted=5 * A), dict(length_out=7 * A), dict(page_out=A, page_out_ld=7)):   # in place at other strides
        assert _pages_call("compact", dict(COMPACT, **change)) == "SC_ERR_SHAPE_MISMATCH", change
    if _ready():
        assert _pages_call("compact", dict(COMPACT, page_out=A, page_out_ld=8, holders_out=3 * A)) == "SC_ERR_DEVICE"


def test_pages_workspace():
    for pages, new, status in ((0, 1, "SC_ERR_BAD_DIMS"), (2 ** 30 + 1, 1, "SC_ERR_BAD_DIMS"), (5, -1, "SC_ERR_BAD_DIMS"), (5, 1 << 20, "SC_ERR_BAD_DIMS"), (2 ** 30, (1 << 20) - 1, "SC_OK")):
        assert _status(sc.attention_pages_workspace_bytes, pages, new) == status
    assert sc.attention_pages_workspace_bytes(2 ** 30, 0) > 2 ** 32
    assert sc.lib().sc_attention_pages_workspace_bytes(ctypes.c_int64(1), 1, None) == 1
    assert sc.lib().sc_attention_tree_workspace_bytes(None, ctypes.byref(ctypes.c_size_t())) == 1


def test_copy_refusals():
    h = _create()
    if _ready():
        assert _status(sc.attention_copy, h, _cache(), A, 5) == "SC_ERR_DEVICE"
    assert _status(sc.attention_copy, h, _cache(), 0, 5) == "SC_ERR_NULL" and _status(sc.attention_copy, h, None, A, 5) == "SC_ERR_NULL"
    assert _status(sc.attention_copy, h, _cache(), A, -1) == "SC_ERR_BAD_DIMS" and _status(sc.attention_copy, h, _cache(), A, 2 ** 30 + 1) == "SC_ERR_BAD_DIMS"
    assert _status(sc.attention_copy, h, _cache(row=8), A, 5) == "SC_ERR_SHAPE_MISMATCH" and _status(sc.attention_copy, h, _cache(), 0, 0) == "SC_OK"


def test_index_arithmetic(tmp_path):
    exe = str(tmp_path / "attention_span_check")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "-w", "-x", "hip", "--offload-host-only", os.path.join(HERE, "native", "attention_span_check.cpp"), "-o", exe], timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


# -- tensors -----------------------------------------------------------------------------------------------------------------------
def handle(monkeypatch=None, **kw):
    attention, recorder = recorded(**kw)
    attention._append_tree = attention._tree = attention._accept = attention._fork = attention._compact = attention._copy = recorder
    return attention, recorder


def numbers(*shape, **kw):
    return Record(*shape, dtype=kw.pop("dtype", I32), **kw)


CACHE = Record(9, 16, 2, 64)


def calls(attention, **kw):
    """Each operator with good operands, but for those of `kw`."""
    def get(name, default):
        return kw.get(name, default)

    q, k = get("q", Record(6, 4, 64)), get("k", Record(6, 2, 64))
    keys, pages, lengths, starts = get("keys", CACHE), get("pages", numbers(2, 5)), get("lengths", numbers(2)), get("row_start", numbers(3))
    parents, last, holders, moves = get("parents", numbers(6)), get("last", numbers(2)), get("holders", numbers(40)), get("moves", numbers(7, 3))
    workspace = Record(1 << 28, dtype=torch.uint8)
    new = get("new", numbers(3))
    return {
        "append": lambda **o: attention.append(q, k, k, keys, keys, pages, lengths, starts, parents=parents, **o),
        "tree": lambda **o: attention.tree(q, keys, keys, pages, lengths, starts, parents, **dict(dict(workspace=workspace), **o)),
        "accept": lambda **o: attention.accept(keys, keys, pages, lengths, starts, parents, last, **o),
        "fork": lambda **o: attention.fork(pages, lengths, holders, new, get("wanted", numbers(3)), **dict(dict(workspace=workspace), **o)),
        "compact": lambda **o: attention.compact(pages, lengths, holders, **dict(dict(workspace=workspace), **o)),
        "copy": lambda **o: attention.copy(keys, keys, moves, **o),
    }


OUT = dict(append=Record(6, 4, 64), tree=Record(6, 4, 64), accept=numbers(2, address=5 * A), fork=(numbers(3, 5, address=2 * A), numbers(3, address=3 * A), numbers(40), numbers(3, 3, address=4 * A)),
           compact=(numbers(2, 5), numbers(40), numbers(20, 3, address=4 * A)))


def test_records():
    """What the library is given."""
    attention, recorder = handle()
    for name, call in calls(attention).items():
        result = call(stream=STREAM, **({"out": OUT[name]} if name in OUT else {}))
        assert result is None if name == "copy" else result is OUT[name] or result == OUT[name]
    append, tree, accept, fork, compact, copy = recorder.calls
    sequences, cache = sc.pack_sequences(2, 6, A, A, A, 5, 5), sc.pack_cache(A, A, 9, 2048, 128, 64)
    q, k = sc.pack_rows(A, 256, 64), sc.pack_rows(A, 128, 64)
    assert append[1:] == (sequences, A, q, k, k, q, cache, STREAM)
    assert tree[1:] == (sequences, A, q, cache, q, A, 1 << 28, STREAM)
    assert accept[1:] == (sequences, A, A, cache, 5 * A, STREAM)
    assert fork[1:] == (sc.pack_pages(2, 3, 40, A, 5, 5, A, A, A, A, 2 * A, 5, 3 * A, A, 4 * A), A, 1 << 28, STREAM)
    assert compact[1:] == (sc.pack_pages(2, 0, 40, A, 5, 5, A, A, 0, 0, A, 5, 0, A, 4 * A), A, 1 << 28, STREAM)
    assert copy[1:] == (cache, A, 7, STREAM)


BAD = [
    ("parents", numbers(5), ("append", "tree")), ("parents", numbers(6, dtype=torch.int64), ("append", "tree", "accept")), ("parents", numbers(6, index=-1), ("append", "tree", "accept")),
    ("parents", numbers(6, strides=(2,)), ("append", "tree", "accept")), ("last", numbers(3), ("accept",)), ("last", numbers(2, dtype=torch.int64), ("accept",)),
    ("lengths", numbers(3), ("append", "tree", "accept", "fork", "compact")), ("lengths", numbers(2, index=1), ("append", "tree", "accept", "fork", "compact")),
    ("pages", numbers(2, 5, dtype=torch.int64), ("append", "tree", "accept", "fork", "compact")), ("pages", numbers(2, 5, strides=(1, 2)), ("append", "tree", "accept", "fork", "compact")),
    ("pages", numbers(10), ("fork", "compact")), ("holders", numbers(40, dtype=torch.int64), ("fork", "compact")), ("holders", numbers(40, strides=(2,)), ("fork", "compact")),
    ("new", numbers(3, dtype=torch.int64), ("fork",)), ("wanted", numbers(2), ("fork",)), ("wanted", numbers(3, index=1), ("fork",)),
    ("moves", numbers(7, 4), ("copy",)), ("moves", numbers(21), ("copy",)), ("moves", numbers(7, 3, dtype=torch.int64), ("copy",)), ("moves", numbers(7, 3, strides=(4, 1)), ("copy",)),
    ("row_start", numbers(4), ("append", "tree", "accept")),
]


@pytest.mark.parametrize("name,value,takes", BAD)
def test_tensor_refusals(name, value, takes):
    attention, recorder = handle()
    for op, call in calls(attention, **{name: value}).items():
        if op in takes:
            with pytest.raises(ValueError):
                call(stream=STREAM, **({"out": OUT[op]} if op in OUT else {}))
    assert not recorder.calls


def test_out_refusals():
    attention, recorder = handle()
    made = calls(attention)
    for op, out in (("accept", numbers(3)), ("accept", numbers(2, dtype=torch.int64)), ("fork", OUT["fork"][:3]), ("fork", (numbers(3, 4), *OUT["fork"][1:])),
                    ("fork", (*OUT["fork"][:3], numbers(2, 3))), ("fork", (OUT["fork"][0], numbers(3, strides=(2,)), *OUT["fork"][2:])), ("compact", OUT["compact"][:2]),
                    ("compact", (*OUT["compact"][:2], numbers(19, 3)))):
        with pytest.raises(ValueError):
            made[op](out=out, stream=STREAM)
    assert not recorder.calls


@pytest.mark.parametrize("op", ["append", "tree", "accept", "copy"])
def test_gradients_and_tangents_are_refused(op):
    attention, recorder = handle()
    cache = Record(9, 16, 2, 64, requires_grad=True)
    with pytest.raises(RuntimeError, match="gradient"):
        calls(attention, keys=cache)[op](stream=STREAM, **({"out": OUT[op]} if op in OUT else {}))
    if op in ("append", "tree"):
        with pytest.raises(RuntimeError, match="gradient"):
            calls(attention, q=Record(6, 4, 64, requires_grad=True))[op](stream=STREAM, out=OUT[op])
    assert not recorder.calls
    with torch.no_grad():
        calls(attention, keys=cache)[op](stream=STREAM, **({"out": OUT[op]} if op in OUT else {}))


def test_results_and_workspaces_belong_to_the_stream_of_their_call(monkeypatch):
    attention, recorder = handle()
    for op, results in (("append", 1), ("tree", 1), ("accept", 1), ("fork", 4), ("compact", 3)):
        for stream, on in ((None, 7), (7, 7), (STREAM, STREAM)):
            memory = Memory(monkeypatch, 7)
            calls(attention)[op](stream=stream)
            assert [x for x, _ in memory.made] == [on] * results and memory.current == 7
            assert memory.told == ({} if on == 7 else {x.data_ptr(): [7] for _, x in memory.made})
    memory = Memory(monkeypatch, 7)
    calls(attention)["tree"](stream=STREAM, out=OUT["tree"], workspace=None)       # the handle's own: it stays
    calls(attention)["tree"](stream=STREAM, out=OUT["tree"], workspace=None)
    assert [(on, x.numel()) for on, x in memory.made] == [(STREAM, attention.tree_ws_bytes)]
    for op, new in (("fork", 4), ("compact", 1)):
        memory = Memory(monkeypatch, 7)
        for _ in range(2):
            calls(attention)[op](stream=STREAM, out=OUT[op], workspace=None)
        made, = memory.made
        assert made[0] == STREAM and made[1].numel() == sc.attention_pages_workspace_bytes(40, new) and not memory.told
        assert [call[-3:] for call in recorder.calls[-2:]] == [(made[1].data_ptr(), made[1].numel(), STREAM)] * 2
        calls(attention)[op](out=OUT[op], workspace=None)          # the current stream: not given away before that is done with it
        assert len(memory.made) == 1 and memory.told == {made[1].data_ptr(): [7]}


def test_workspaces_of_many_batches(monkeypatch):
    """Batches of any sizes share a few workspaces of the handle's, which stay as long as it does; each has room for its batch."""
    attention, recorder = handle()
    memory, holders = Memory(monkeypatch, 7), numbers(5000)
    for new in (1, 2, 3, 5, 9, 17, 31, 32, 33, 100, 500, 2047, 2048, 5000, 70_000, 2 ** 17 - 1, 2 ** 17, 2 ** 20 - 1):
        out = numbers(new, 5, address=2 * A), numbers(new, address=3 * A), holders, numbers(new, 3, address=4 * A)
        attention.fork(numbers(2, 5), numbers(2), holders, numbers(new), None, out=out, stream=STREAM)
        assert recorder.calls[-1][-2] >= sc.attention_pages_workspace_bytes(5000, new)
    attention.compact(numbers(2, 5), numbers(2), holders, out=(numbers(2, 5), holders, numbers(2500, 3, address=4 * A)), stream=STREAM)
    assert recorder.calls[-1][-2] >= sc.attention_pages_workspace_bytes(5000, 0)
    assert len(memory.made) <= 5


def test_calls_are_made_on_the_device_of_the_handle(monkeypatch):
    attention, _ = handle()
    devices, at = Devices(monkeypatch, 2), []
    attention._append_tree = attention._tree = attention._accept = attention._fork = attention._compact = attention._copy = lambda *args: at.append(devices.current) or 0
    for op, call in calls(attention).items():
        call(stream=STREAM, **({"out": OUT[op]} if op in OUT else {}))
    assert at == [0] * 6 and devices.current == 2


def test_append_without_parents_is_as_it_was():
    attention, recorder = handle()
    attention._append = other = Recorder()
    attention.append(Record(6, 4, 64), Record(6, 2, 64), Record(6, 2, 64), CACHE, CACHE, numbers(2, 5), numbers(2), numbers(3), out=OUT["append"], stream=STREAM)
    assert not recorder.calls and len(other.calls) == 1
