"""Attention of a decoder layer over packed rows and a paged cache, on torch tensors: checks shapes and types, hands addresses
and strides to the library and queues its kernels.  No arithmetic happens here.

    attention = Attention(heads=32, kv_heads=8, head_dim=128, dtype=torch.bfloat16, page_rows=64, rotary_dim=128)
    q = attention.append(q, k, v, keys, values, pages, lengths, row_start)     # rotate, store new rows in the cache
    y = attention.prompt_paged(q, keys, values, pages, lengths, row_start)     # many new rows per sequence
    y = attention.decode(q, keys, values, pages, lengths)                      # one new row per sequence

`q` is (rows, heads, head_dim), `k` and `v` (rows, kv_heads, head_dim), `keys` and `values` (pages, page_rows, kv_heads, head_dim); any strides
that are multiples of 16 bytes, head_dim contiguous.  `pages` (batch, columns), `lengths` (batch) and `row_start` (batch + 1) are int32.
A length counts the new rows of its sequence.  The library's header says what the kernels make of wrong lengths and page numbers.
"""
from __future__ import annotations

import torch

from . import binding as sc

_DTYPES = {torch.bfloat16: sc.SC_BF16, torch.float16: sc.SC_F16, torch.float32: sc.SC_F32}


class Attention:
    """The operators for one head layout.  Holds the workspace of `decode`: calls of one Attention are to be queued on one stream, or
    ordered by the caller; more streams at once take an Attention each."""

    def __init__(self, heads, kv_heads, head_dim, dtype=torch.bfloat16, page_rows=64, *, causal=True, scale=None, rotary_dim=0,
                 rotary_theta=10000.0, rotary_freq=None, interleaved=False, device="cuda:0"):
        """`scale`: of the scores, 1 / sqrt(head_dim) unless given.  `rotary_freq`: angles per position of the rotated pairs, or
        `rotary_dim` and `rotary_theta` for theta ** (-2 t / rotary_dim)."""
        if dtype not in _DTYPES:
            raise TypeError(f"attention takes {', '.join(str(t) for t in _DTYPES)}, not {dtype}")
        if rotary_freq is None and rotary_dim:
            rotary_freq = [rotary_theta ** (-2.0 * t / rotary_dim) for t in range(rotary_dim // 2)]
        elif rotary_freq is not None and not rotary_dim:
            rotary_dim = 2 * len(rotary_freq)
        if scale is not None and not scale > 0:
            raise ValueError("the scale of the scores has to be positive")
        if rotary_dim and 2 * len(rotary_freq) != rotary_dim and rotary_dim % 2 == 0:
            raise ValueError("rotary_freq has one angle for each pair of rotary_dim")
        self.heads, self.kv_heads, self.head_dim, self.page_rows, self.dtype = heads, kv_heads, head_dim, page_rows, dtype
        self.handle = sc.attention_create(_DTYPES[dtype], heads, kv_heads, head_dim, page_rows, causal, 0.0 if scale is None else scale,
                                          rotary_freq, interleaved, rotary_dim)
        self.ws_bytes = sc.attention_workspace_bytes(self.handle)
        self.device = torch.device(device)
        self.workspace = None   # made by the first decode

    def describe(self) -> str:
        return sc.attention_describe(self.handle)

    # -- operators ---------------------------------------------------------------------------------------------------------
    def append(self, q, k, v, keys, values, pages, lengths, row_start=None, out=None, stream=None):
        """Stores k, rotated, and v in the pages of their positions; returns q, rotated (in `out`, which may be q).  q may be None."""
        rows = k.shape[0]
        sequences, cache = self._sequences(rows, row_start, lengths, pages), self._cache(keys, values)
        if q is not None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
            query, result = self._rows(q, rows, self.heads), self._rows(out, rows, self.heads)
        else:
            query = result = None
        sc.attention_append(self.handle, sequences, query, self._rows(k, rows, self.kv_heads), self._rows(v, rows, self.kv_heads), result, cache,
                            self._stream() if stream is None else stream)
        return out

    def prompt(self, q, k, v, row_start, out=None, stream=None):
        """Attention of the rows of each sequence over the keys and values of the same rows."""
        rows = q.shape[0]
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        sc.attention_prompt(self.handle, self._sequences(rows, row_start), self._rows(q, rows, self.heads), self._rows(k, rows, self.kv_heads),
                            self._rows(v, rows, self.kv_heads), self._rows(out, rows, self.heads), self._stream() if stream is None else stream)
        return out

    def prompt_paged(self, q, keys, values, pages, lengths, row_start, out=None, stream=None):
        """Attention of the last rows of each sequence over its keys in the cache."""
        rows = q.shape[0]
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        sc.attention_prompt_paged(self.handle, self._sequences(rows, row_start, lengths, pages), self._rows(q, rows, self.heads),
                                  self._cache(keys, values), self._rows(out, rows, self.heads), self._stream() if stream is None else stream)
        return out

    def decode(self, q, keys, values, pages, lengths, out=None, workspace=None, stream=None):
        """Attention of one row per sequence over all its keys in the cache.  `workspace`: device bytes of the caller's, `ws_bytes` of them."""
        rows = q.shape[0]
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        if workspace is None:
            if self.workspace is None:
                self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
            workspace = self.workspace
        sc.attention_decode(self.handle, self._sequences(rows, None, lengths, pages), self._rows(q, rows, self.heads), self._cache(keys, values),
                            self._rows(out, rows, self.heads), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                            self._stream() if stream is None else stream)
        return out

    # -- records -----------------------------------------------------------------------------------------------------------
    def _rows(self, x, rows, heads):
        if x.dtype is not self.dtype or not x.is_cuda:
            raise TypeError(f"rows have to be {self.dtype} on the GPU, not {x.dtype} on {x.device}")
        row, head, element = x.stride()
        if x.shape != (rows, heads, self.head_dim) or element != 1:
            raise ValueError(f"rows have to be ({rows}, {heads}, {self.head_dim}) with the last dimension contiguous, not {tuple(x.shape)} with strides {x.stride()}")
        return sc.pack_rows(x.data_ptr(), row, head)

    def _cache(self, keys, values):
        if keys.dtype is not self.dtype or values.dtype is not self.dtype or not keys.is_cuda or not values.is_cuda:
            raise TypeError(f"the cache has to be {self.dtype} on the GPU, not {keys.dtype} and {values.dtype}")
        shape, (page, row, head, element) = keys.shape, keys.stride()
        if shape[1:] != (self.page_rows, self.kv_heads, self.head_dim) or element != 1 or values.shape != shape or values.stride() != keys.stride():
            raise ValueError(f"keys and values have to be (pages, {self.page_rows}, {self.kv_heads}, {self.head_dim}) alike, with the last "
                             f"dimension contiguous, not {tuple(shape)} and {tuple(values.shape)} with strides {keys.stride()} and {values.stride()}")
        return sc.pack_cache(keys.data_ptr(), values.data_ptr(), shape[0], page, row, head)

    def _sequences(self, rows, row_start=None, lengths=None, pages=None):
        batch = rows if row_start is None else row_start.shape[0] - 1
        page_ld = columns = 0
        for x, n in ((row_start, batch + 1), (lengths, batch)):
            if x is not None and (x.dtype is not torch.int32 or not x.is_cuda or x.shape != (n,) or not x.is_contiguous()):
                raise ValueError(f"row_start and lengths have to be contiguous int32 on the GPU, one length and row start per sequence ({batch}): got {x.dtype} {tuple(x.shape)}")
        if pages is not None:
            if pages.dtype is not torch.int32 or not pages.is_cuda or pages.dim() != 2 or pages.shape[0] != batch or (pages.shape[1] > 1 and pages.stride(1) != 1):
                raise ValueError(f"pages have to be int32 on the GPU, a row per sequence ({batch}): got {pages.dtype} {tuple(pages.shape)}")
            page_ld, columns = pages.stride(0), pages.shape[1]
        return sc.pack_sequences(batch, rows, 0 if row_start is None else row_start.data_ptr(), 0 if lengths is None else lengths.data_ptr(),
                                 0 if pages is None else pages.data_ptr(), page_ld, columns)

    def _stream(self):
        # torch's own accessor of the address alone: the stream object around it takes 2 us to make
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None or self.device.index is None:
            return torch.cuda.current_stream(self.device).cuda_stream
        return raw(self.device.index)
