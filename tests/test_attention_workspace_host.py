"""Workspaces of attention, without a GPU: their sizes, and what the prompt operators refuse."""
import ctypes

import pytest

from paper_2311_09549_amd import binding as sc

A = 1 << 20   # an address that is a multiple of 256; nothing is launched here, so nothing is read


def _status(fn, *args):
    try:
        fn(*args)
    except sc.ScError as e:
        return sc.STATUS_NAMES[e.status]
    return "SC_OK"


@pytest.mark.parametrize("dtype", [sc.SC_BF16, sc.SC_F16, sc.SC_F32])
@pytest.mark.parametrize("head_dim", [8, 64, 72, 128, 136, 256])
def test_sizes(dtype, head_dim):
    h = sc.attention_create(dtype, 4, 2, head_dim, 16)
    size = sc.attention_prompt_workspace_bytes(h)
    assert (size == 0) == (dtype == sc.SC_F32)
    # two pieces of 128 or 256 rows for each of at least 200 compute units
    rows, padded = (128, 256) if head_dim > 128 else (256, 128 if head_dim > 64 else 64)
    assert size == 0 or size >= 2 * 200 * rows * padded * 4
    assert f"{size} bytes of workspace" in sc.attention_describe(h)


def test_null_arguments():
    h, size = sc.attention_create(sc.SC_BF16, 4, 2, 64, 16), ctypes.c_size_t()
    assert sc.lib().sc_attention_prompt_workspace_bytes(None, ctypes.byref(size)) == 1
    assert sc.lib().sc_attention_prompt_workspace_bytes(h.handle, None) == 1


@pytest.mark.parametrize("dtype,size", [(sc.SC_BF16, 2), (sc.SC_F16, 2), (sc.SC_F32, 4)])
def test_prompt_refusals(dtype, size):
    h = sc.attention_create(dtype, 4, 2, 64, 16)
    rows, cache = sc.pack_rows(A, 1024, 64), sc.pack_cache(A, A, 10, 16 * 128, 128, 64)
    packed, paged = sc.pack_sequences(1, 600, A, 0, 0, 0, 0), sc.pack_sequences(1, 600, A, A, A, 64, 64)
    enough = sc.attention_prompt_workspace_bytes(h)
    for call, args in ((sc.attention_prompt, (h, packed, rows, rows, rows, rows)), (sc.attention_prompt_paged, (h, paged, rows, cache, rows))):
        if size == 2:
            assert _status(call, *args, A, enough - 1) == "SC_ERR_WORKSPACE_SMALL"
            assert _status(call, *args, A + 16, enough) == "SC_ERR_SHAPE_MISMATCH"
        import torch
        if not torch.cuda.is_available():
            for ws in (0, A):
                assert _status(call, *args, ws, enough) == "SC_ERR_DEVICE"


def test_traffic_of_contractions_does_not_depend_on_attention(monkeypatch):
    """Sources of attention are no part of what the stored traffic of contractions is tied to; the others are."""
    import os

    from paper_2311_09549_amd import traffic
    there = set(os.listdir(os.path.join(traffic.HERE, "csrc")))
    assert set(traffic.ATTENTION) <= there and len(there - set(traffic.ATTENTION)) > 10
    digest, seen = traffic.source_digest(), []
    real = open
    monkeypatch.setattr("builtins.open", lambda path, *a, **k: (seen.append(os.path.basename(str(path))), real(path, *a, **k))[1])
    assert traffic.source_digest() == digest
    assert set(seen) == there - set(traffic.ATTENTION)
