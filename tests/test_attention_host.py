"""Host side of attention, without a GPU: what the entry points refuse, what a handle says, and the index arithmetic of the kernels."""
import ctypes
import os
import subprocess

import pytest

from paper_2311_09549_amd import binding as sc

HERE = os.path.dirname(os.path.abspath(__file__))
A = 1 << 20   # an address that is a multiple of 256; nothing is launched here, so nothing is read


def _status(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except sc.ScError as e:
        return sc.STATUS_NAMES[e.status]
    return "SC_OK"


def _create(**kw):
    args = dict(dtype=sc.SC_BF16, heads=8, kv_heads=2, head_dim=128, page_rows=16)
    args.update(kw)
    return sc.attention_create(**args)


@pytest.mark.parametrize("change,status", [
    ({}, "SC_OK"),
    (dict(dtype=sc.SC_F16), "SC_OK"), (dict(dtype=sc.SC_F32), "SC_OK"), (dict(dtype=sc.SC_F64), "SC_ERR_BAD_DTYPE"), (dict(dtype=9), "SC_ERR_BAD_DTYPE"),
    (dict(heads=0), "SC_ERR_BAD_DIMS"), (dict(kv_heads=0), "SC_ERR_BAD_DIMS"), (dict(kv_heads=3), "SC_ERR_BAD_DIMS"), (dict(heads=-8, kv_heads=-2), "SC_ERR_BAD_DIMS"),
    (dict(heads=4104, kv_heads=8), "SC_ERR_BAD_DIMS"),
    (dict(head_dim=8), "SC_OK"), (dict(head_dim=256), "SC_OK"), (dict(head_dim=0), "SC_ERR_BAD_DIMS"), (dict(head_dim=264), "SC_ERR_BAD_DIMS"), (dict(head_dim=100), "SC_ERR_BAD_DIMS"),
    (dict(page_rows=8), "SC_ERR_BAD_DIMS"), (dict(page_rows=48), "SC_ERR_BAD_DIMS"), (dict(page_rows=8192), "SC_ERR_BAD_DIMS"), (dict(page_rows=4096), "SC_OK"),
    (dict(scale=-1.0), "SC_ERR_BAD_DIMS"), (dict(scale=float("nan")), "SC_ERR_BAD_DIMS"), (dict(scale=float("inf")), "SC_ERR_BAD_DIMS"), (dict(scale=0.5), "SC_OK"),
    (dict(rotary_freq=[1.0] * 64), "SC_OK"), (dict(rotary_freq=[1.0] * 65), "SC_ERR_BAD_DIMS"), (dict(rotary_freq=[1.0, float("nan")]), "SC_ERR_BAD_DIMS"),
    (dict(rotary_freq=[1.0], rotary_dim=3), "SC_ERR_BAD_DIMS"), (dict(rotary_dim=-2), "SC_ERR_BAD_DIMS"), (dict(rotary_dim=4), "SC_ERR_NULL"),
])
def test_create(change, status):
    assert _status(_create, **change) == status


def test_null_arguments():
    lib, h, desc = sc.lib(), _create(), sc.AttentionDesc()
    out, size = ctypes.c_void_p(), ctypes.c_size_t()
    assert lib.sc_attention_create(None, ctypes.byref(desc)) == 1 and lib.sc_attention_create(ctypes.byref(out), None) == 1
    assert lib.sc_attention_workspace_bytes(None, ctypes.byref(size)) == 1 and lib.sc_attention_workspace_bytes(h.handle, None) == 1
    assert lib.sc_attention_describe(h.handle, None, ctypes.c_size_t(4)) == 1
    assert lib.sc_attention_destroy(None) == 0
    s, r, c = _sequences(), _rows(), _cache()
    for bad in range(8):
        if bad in (3, 5, 7):   # q and q_out may be NULL, but together; the stream may
            continue
        args = [h.handle, s, r, r, r, r, c, 0]
        args[bad] = None
        assert lib.sc_attention_append(*args) == 1
    assert lib.sc_attention_append(h.handle, s, None, r, r, r, c, 0) == 1 and lib.sc_attention_append(h.handle, s, r, r, r, None, c, 0) == 1
    assert lib.sc_attention_append(h.handle, s, r, None, r, r, c, 0) == 1


def test_describe_and_workspace():
    h = _create(rotary_freq=[1.0] * 16)
    text = sc.attention_describe(h)
    for part in ("attention bf16", "heads 8", "key heads 2", "pages of 16 rows", "rotates 32 of 128", "softmax"):
        assert part in text
    assert sc.attention_workspace_bytes(h) % 256 == 0 and sc.attention_workspace_bytes(h) > 0
    buf = ctypes.create_string_buffer(b"x" * 9, 9)
    assert sc.lib().sc_attention_describe(h.handle, buf, ctypes.c_size_t(5)) == 0 and buf.value == b"atte"


def _sequences(batch=3, rows=3, row_start=0, length=A, page=A, page_ld=4, page_count=4):
    return sc.pack_sequences(batch, rows, row_start, length, page, page_ld, page_count)


def _rows(data=A, row=1024, head=128):
    return sc.pack_rows(data, row, head)


def _cache(keys=A, values=A, pages=10, page=16 * 256, row=256, head=128):
    return sc.pack_cache(keys, values, pages, page, row, head)


def _ready():
    """SC_OK on a GPU is not wanted here (the addresses are none): calls that pass every check end with SC_ERR_DEVICE without one."""
    import torch
    return not torch.cuda.is_available()


BAD_SEQUENCES = [
    (dict(batch=-1), "SC_ERR_BAD_DIMS"), (dict(batch=1 << 20, rows=1 << 20), "SC_ERR_BAD_DIMS"), (dict(rows=-1, row_start=A), "SC_ERR_BAD_DIMS"),
    (dict(rows=1 << 24, row_start=A), "SC_ERR_BAD_DIMS"), (dict(rows=4), "SC_ERR_SHAPE_MISMATCH"), (dict(length=0), "SC_ERR_NULL"), (dict(page=0), "SC_ERR_NULL"),
    (dict(page_ld=-1), "SC_ERR_BAD_DIMS"), (dict(page_count=-1), "SC_ERR_BAD_DIMS"), (dict(page_count=1 << 31), "SC_ERR_BAD_DIMS"),
]
BAD_CACHES = [
    (dict(keys=0), "SC_ERR_NULL"), (dict(values=0), "SC_ERR_NULL"), (dict(pages=0), "SC_ERR_BAD_DIMS"), (dict(pages=1 << 31), "SC_ERR_BAD_DIMS"),
    (dict(page=-16), "SC_ERR_BAD_DIMS"), (dict(keys=A + 8), "SC_ERR_SHAPE_MISMATCH"), (dict(values=A + 2), "SC_ERR_SHAPE_MISMATCH"), (dict(row=260), "SC_ERR_SHAPE_MISMATCH"),
    (dict(head=64), "SC_ERR_SHAPE_MISMATCH"), (dict(row=128), "SC_ERR_SHAPE_MISMATCH"), (dict(page=256), "SC_ERR_SHAPE_MISMATCH"), (dict(page=1 << 40), "SC_ERR_BAD_DIMS"),
]
BAD_ROWS = [
    (dict(data=0), "SC_ERR_NULL"), (dict(data=A + 4), "SC_ERR_SHAPE_MISMATCH"), (dict(row=1028), "SC_ERR_SHAPE_MISMATCH"), (dict(head=-8), "SC_ERR_BAD_DIMS"), (dict(row=1 << 40), "SC_ERR_BAD_DIMS"),
]
BAD_OUTPUTS = BAD_ROWS + [(dict(row=0), "SC_ERR_SHAPE_MISMATCH"), (dict(head=0), "SC_ERR_SHAPE_MISMATCH"), (dict(row=1024, head=64), "SC_ERR_SHAPE_MISMATCH"), (dict(row=512, head=128), "SC_ERR_SHAPE_MISMATCH")]


def _calls(h, sequences=None, packed=None, q=None, k=None, v=None, out=None, cache=None):
    s, p = sequences or _sequences(), packed or _sequences(length=0, row_start=A)
    q, k, v, out, c = q or _rows(), k or _rows(), v or _rows(), out or _rows(), cache or _cache()
    ws = sc.attention_workspace_bytes(h)
    return {
        "append": lambda: sc.attention_append(h, s, q, k, v, out, c),
        "prompt": lambda: sc.attention_prompt(h, p, q, k, v, out),
        "prompt_paged": lambda: sc.attention_prompt_paged(h, s, q, c, out),
        "decode": lambda: sc.attention_decode(h, s, q, c, out, A, ws),
    }


@pytest.mark.parametrize("op", ["append", "prompt", "prompt_paged", "decode"])
def test_refusals(op):
    h = _create()
    if _ready():
        assert _status(_calls(h)[op]) == "SC_ERR_DEVICE"
    paged = op != "prompt"
    for change, status in BAD_SEQUENCES:
        if paged and not (op == "decode" and "row_start" in change):
            assert _status(_calls(h, sequences=_sequences(**change))[op]) == status, change
        if not paged and "page" not in str(change) and "length" not in change and not (change.get("rows") == 4):
            assert _status(_calls(h, packed=_sequences(**dict(dict(length=0, row_start=A), **change)))[op]) == status, change
    if not paged:
        assert _status(_calls(h, packed=_sequences(row_start=A))[op]) == "SC_ERR_SHAPE_MISMATCH"   # lengths of their own
    for change, status in BAD_CACHES if paged else []:
        assert _status(_calls(h, cache=_cache(**change))[op]) == status, change
    for change, status in BAD_ROWS:
        assert _status(_calls(h, q=_rows(**change))[op]) == status, change
        if op in ("append", "prompt"):
            assert _status(_calls(h, k=_rows(**change))[op]) == status, change
            assert _status(_calls(h, v=_rows(**change))[op]) == status, change
    for change, status in BAD_OUTPUTS:
        assert _status(_calls(h, out=_rows(**change))[op]) == status, change


def test_refusals_of_one_operator():
    h = _create()
    ws = sc.attention_workspace_bytes(h)
    assert _status(sc.attention_decode, h, _sequences(row_start=A), _rows(), _cache(), _rows(), A, ws) == "SC_ERR_SHAPE_MISMATCH"
    assert _status(sc.attention_decode, h, _sequences(), _rows(), _cache(), _rows(), A, ws - 1) == "SC_ERR_WORKSPACE_SMALL"
    assert _status(sc.attention_decode, h, _sequences(), _rows(), _cache(), _rows(), 0, ws) == "SC_ERR_NULL"
    assert _status(sc.attention_decode, h, _sequences(), _rows(), _cache(), _rows(), A + 16, ws) == "SC_ERR_SHAPE_MISMATCH"
    # in place with other strides
    assert _status(sc.attention_append, h, _sequences(), _rows(row=2048), _rows(), _rows(), _rows(), _cache()) == "SC_ERR_SHAPE_MISMATCH"


def test_calls_without_work():
    h = _create()
    none = _sequences(batch=0, rows=0, length=0, page=0, page_count=0)
    for op in ("append", "prompt", "prompt_paged", "decode"):
        assert _status(_calls(h, sequences=none, packed=none)[op]) == "SC_OK"


def test_contractions_refuse_the_types_of_attention():
    v = sc.CooView()
    for code in (sc.SC_BF16, sc.SC_F16):
        import numpy as np
        coords = [np.zeros(1, np.int32)] * 3
        v = sc.coo_view(coords, np.ones(1, np.float32), (2, 2, 2))
        v.dtype = code
        nfib = (ctypes.c_int64 * 4)()
        assert sc.STATUS_NAMES[sc.lib().sc_coo_to_csf_sizes(ctypes.byref(v), nfib)] == "SC_ERR_BAD_DTYPE"


def test_index_arithmetic(tmp_path):
    exe = str(tmp_path / "attention_index_check")
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "-w", "-x", "hip", "--offload-host-only", os.path.join(HERE, "native", "attention_index_check.cpp"), "-o", exe], timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
