"""Attention of a decoder layer over packed rows and a paged cache, on torch tensors: checks shapes and types, hands addresses
and strides to the library and queues its kernels.  No arithmetic happens here.

    attention = Attention(heads=32, kv_heads=8, head_dim=128, dtype=torch.bfloat16, page_rows=64, rotary_dim=128)
    q = attention.append(q, k, v, keys, values, pages, lengths, row_start)     # rotate, store new rows in the cache
    y = attention.prompt_paged(q, keys, values, pages, lengths, row_start)     # many new rows per sequence
    y = attention.decode(q, keys, values, pages, lengths)                      # one new row per sequence

Drafted tokens, nodes of a tree behind each sequence (`parents`: one number per row, within its sequence, -1 for a node that follows what is before the tree):

    q = attention.append(q, k, v, keys, values, pages, lengths, row_start, parents=parents)      # rotated by their depths
    y = attention.tree(q, keys, values, pages, lengths, row_start, parents)                      # each sees its ancestors
    accepted = attention.accept(keys, values, pages, lengths, row_start, parents, last)          # the path to node last[b] becomes the sequence

Sequences that branch, end, shrink and grow share pages (`holders`: how many entries hold each page, 0 for a free one):

    pages, lengths, holders, moves = attention.fork(pages, lengths, holders, order, wanted)      # sequence i goes on from sequence order[i]
    pages, holders, moves = attention.compact(pages, lengths, holders)                           # pages in use to the lowest numbers
    attention.copy(keys, values, moves)                                                          # in every layer's cache, after either

Both take the lengths that the table's pages were given out for.  After `accept` those are the ones of before, and its own are what is wanted, of a fork before any other call on the pages:

    pages, lengths, holders, moves = attention.fork(pages, lengths, holders, order, accepted[order])     # pages of nodes that were not accepted are free again
    attention.copy(keys, values, moves)
    pages, lengths, holders, moves = attention.fork(pages, lengths, holders, same, lengths + new)        # then room for new rows (same: 0, 1, 2, ..)
    attention.copy(keys, values, moves)

`q` is (rows, heads, head_dim), `k` and `v` (rows, kv_heads, head_dim), `keys` and `values` (pages, page_rows, kv_heads, head_dim); any strides
that are multiples of 16 bytes, head_dim contiguous.  `pages` (batch, columns), `lengths` (batch) and `row_start` (batch + 1) are int32.
A length counts the new rows of its sequence.  The library's header says what the kernels make of wrong lengths and page numbers.

Choices between kernels go by the width of `pages`, for lengths are in device memory: where a table has room for many more keys than there are,
`pages[:, :columns]` with as many columns as the longest length takes makes short calls shorter (a sequence with more keys than that becomes NaN).
"""
from __future__ import annotations

from contextlib import nullcontext

import torch
import torch.autograd.forward_ad as _forward_ad

from . import binding as sc

_DTYPES = {torch.bfloat16: sc.SC_BF16, torch.float16: sc.SC_F16, torch.float32: sc.SC_F32}

_INT32, _empty_like = torch.int32, torch.empty_like
_pack_rows, _pack_cache, _pack_sequences, _pack_pages = sc.pack_rows, sc.pack_cache, sc.pack_sequences, sc.pack_pages

# torch's own accessor of a stream's address alone: the stream object around it takes 2 us to make
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class Attention:
    """The operators for one head layout.  Holds the workspace of its calls: those of one Attention are to be queued on one stream, or
    ordered by the caller; more streams at once take an Attention each.  A graph that holds its calls needs it as long as it is replayed.
    Tensors are on `device`; calls are made there, whichever is the current one.  Inference only: operands that require a gradient are refused."""

    def __init__(self, heads, kv_heads, head_dim, dtype=torch.bfloat16, page_rows=64, *, causal=True, scale=None, rotary_dim=0,
                 rotary_theta=10000.0, rotary_freq=None, interleaved=False, device="cuda:0", window=None, sinks=0):
        """`scale`: of the scores, 1 / sqrt(head_dim) unless given.  `rotary_freq`: angles per position of the rotated pairs, or
        `rotary_dim` and `rotary_theta` for theta ** (-2 t / rotary_dim).  `window`: a row sees the last so many positions, its own
        included, and the first `sinks`; None for all of them."""
        if dtype not in _DTYPES:
            raise TypeError(f"attention takes {', '.join(str(t) for t in _DTYPES)}, not {dtype}")
        if rotary_freq is None and rotary_dim:
            rotary_freq = [rotary_theta ** (-2.0 * t / rotary_dim) for t in range(rotary_dim // 2)]
        elif rotary_freq is not None and not rotary_dim:
            rotary_dim = 2 * len(rotary_freq)
        if scale is not None and not scale > 0:
            raise ValueError("the scale of the scores has to be positive")
        if window is None and sinks:
            raise ValueError("without a window every row sees the first keys")
        if window is not None and not causal:
            raise ValueError("a window is of causal attention")
        if rotary_dim and 2 * len(rotary_freq) != rotary_dim and rotary_dim % 2 == 0:
            raise ValueError("rotary_freq has one angle for each pair of rotary_dim")
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError(f"attention runs on a GPU, not on {self.device}")
        self._index = torch.cuda.current_device() if self.device.index is None else self.device.index
        self.device = torch.device("cuda", self._index)
        self.heads, self.kv_heads, self.head_dim, self.page_rows, self.dtype = heads, kv_heads, head_dim, page_rows, dtype
        self._page = (page_rows, kv_heads, head_dim)
        with torch.cuda.device(self._index) if torch.cuda.is_available() else nullcontext():   # the library asks the current device
            self.handle = sc.attention_create(_DTYPES[dtype], heads, kv_heads, head_dim, page_rows, causal, 0.0 if scale is None else scale,
                                              rotary_freq, interleaved, rotary_dim, window, sinks)
        self.window, self.sinks = window, sinks
        self.ws_bytes = sc.attention_workspace_bytes(self.handle)
        self.tree_ws_bytes = sc.attention_tree_workspace_bytes(self.handle)
        self.prompt_ws_bytes = sc.attention_prompt_workspace_bytes(self.handle)
        self._few_rows = 4 * (32 if head_dim > 128 else 128)   # of a packed prompt: no more than four tiles of keys, which the library never splits
        self._own = {}   # workspaces, made by the first calls that need them
        self._pages_bytes = {}   # of fork and compact, by the pages of a cache and sequences
        self._h = self.handle.handle
        (self._append, self._prompt, self._prompt_paged, self._decode, self._append_tree, self._tree, self._accept, self._fork, self._compact,
         self._copy) = sc.attention_calls()

    def describe(self) -> str:
        return sc.attention_describe(self.handle)

    # -- operators ---------------------------------------------------------------------------------------------------------
    # `stream`: the address of a HIP stream, torch's current one unless given.  What is made here, results and workspaces, is memory of that
    # stream; operands are the caller's to order before the call, and to keep until the stream is done with them.  `out` is apart from the other operands,
    # but for append's.
    def append(self, q, k, v, keys, values, pages, lengths, row_start=None, out=None, stream=None, parents=None):
        """Stores k, rotated, and v in the pages of their positions; returns q, rotated (in `out`, which may be q).  q may be None, and then there is no result.
        `parents`: rows are nodes of trees, stored in their order and rotated by the positions of their depths."""
        if _current_device() != self._index:
            return self._there(self.append, q, k, v, keys, values, pages, lengths, row_start, out, stream, parents)
        shape = (k.shape[0], self.kv_heads, self.head_dim)
        sequences, cache = self._sequences(shape[0], row_start, lengths, pages), self._cache(keys, values)
        key, value, key_rows = self._rows(k, shape), self._rows(v, shape), shape[0]
        query = result = None
        if q is not None:
            shape = (shape[0], self.heads, self.head_dim)
            query = self._rows(q, shape)
            out, result = self._out(q, out, shape, stream)
        elif out is not None:
            raise ValueError("out is for rotated queries, and there are no queries")
        if stream is None:
            stream = _raw_stream(self._index)
        if parents is None:
            status = self._append(self._h, sequences, query, key, value, result, cache, stream)
        else:
            status = self._append_tree(self._h, sequences, self._numbers("parents", parents, key_rows), query, key, value, result, cache, stream)
        if status:
            raise sc.ScError(status, "sc_attention_append" if parents is None else "sc_attention_append_tree")
        return out

    def prompt(self, q, k, v, row_start, out=None, workspace=None, stream=None):
        """Attention of the rows of each sequence over the keys and values of the same rows."""
        if _current_device() != self._index:
            return self._there(self.prompt, q, k, v, row_start, out, workspace, stream)
        rows = q.shape[0]
        shape, kv_shape = (rows, self.heads, self.head_dim), (rows, self.kv_heads, self.head_dim)
        query, key, value = self._rows(q, shape), self._rows(k, kv_shape), self._rows(v, kv_shape)
        out, result = self._out(q, out, shape, stream)
        if stream is None:
            stream = _raw_stream(self._index)
        address, size = self._workspace_of(stream, workspace, "prompt_ws_bytes") if workspace is not None or (self.prompt_ws_bytes and rows > self._few_rows) else (None, 0)
        status = self._prompt(self._h, self._sequences(rows, row_start, None, None), query, key, value, result, address, size, stream)
        if status:
            raise sc.ScError(status, "sc_attention_prompt")
        return out

    def prompt_paged(self, q, keys, values, pages, lengths, row_start, out=None, workspace=None, stream=None):
        """Attention of the last rows of each sequence over its keys in the cache."""
        if _current_device() != self._index:
            return self._there(self.prompt_paged, q, keys, values, pages, lengths, row_start, out, workspace, stream)
        shape = (q.shape[0], self.heads, self.head_dim)
        query = self._rows(q, shape)
        out, result = self._out(q, out, shape, stream)
        if stream is None:
            stream = _raw_stream(self._index)
        address, size = self._workspace_of(stream, workspace, "prompt_ws_bytes") if workspace is not None or self.prompt_ws_bytes else (None, 0)
        status = self._prompt_paged(self._h, self._sequences(shape[0], row_start, lengths, pages), query, self._cache(keys, values), result, address, size, stream)
        if status:
            raise sc.ScError(status, "sc_attention_prompt_paged")
        return out

    def decode(self, q, keys, values, pages, lengths, out=None, workspace=None, stream=None):
        """Attention of one row per sequence over all its keys in the cache.  `workspace`: device bytes of the caller's, `ws_bytes` of them."""
        if _current_device() != self._index:
            return self._there(self.decode, q, keys, values, pages, lengths, out, workspace, stream)
        shape = (q.shape[0], self.heads, self.head_dim)
        query = self._rows(q, shape)
        out, result = self._out(q, out, shape, stream)
        if stream is None:
            stream = _raw_stream(self._index)
        address, size = self._workspace_of(stream, workspace, "ws_bytes")
        status = self._decode(self._h, self._sequences(shape[0], None, lengths, pages), query, self._cache(keys, values), result, address, size, stream)
        if status:
            raise sc.ScError(status, "sc_attention_decode")
        return out

    def tree(self, q, keys, values, pages, lengths, row_start, parents=None, out=None, workspace=None, stream=None):
        """Attention of the nodes of trees, the last rows of each sequence, over what is before the tree, their ancestors and themselves.  Without
        `parents` each row follows the one before it.  `workspace`: device bytes of the caller's, `tree_ws_bytes` of them."""
        if _current_device() != self._index:
            return self._there(self.tree, q, keys, values, pages, lengths, row_start, parents, out, workspace, stream)
        shape = (q.shape[0], self.heads, self.head_dim)
        query = self._rows(q, shape)
        parent = None if parents is None else self._numbers("parents", parents, shape[0])
        out, result = self._out(q, out, shape, stream)
        if stream is None:
            stream = _raw_stream(self._index)
        address, size = self._workspace_of(stream, workspace, "tree_ws_bytes")
        status = self._tree(self._h, self._sequences(shape[0], row_start, lengths, pages), parent, query, self._cache(keys, values), result, address, size, stream)
        if status:
            raise sc.ScError(status, "sc_attention_tree")
        return out

    def accept(self, keys, values, pages, lengths, row_start, parents, last, out=None, stream=None):
        """Sequence b goes on from node last[b] of its tree (-1: from what is before it): the rows of the path move to the places behind what is before the
        tree.  Returns the lengths after that (in `out`, apart from the operands), -1 where a length, a path or its end is wrong.  Every layer's
        cache takes the call, with the lengths of before, and so does the `fork` that gives up the pages of the other nodes, with the new lengths as `wanted`."""
        if _current_device() != self._index:
            return self._there(self.accept, keys, values, pages, lengths, row_start, parents, last, out, stream)
        rows = parents.shape[0]
        sequences, cache, parent = self._sequences(rows, row_start, lengths, pages), self._cache(keys, values), self._numbers("parents", parents, rows)
        batch = lengths.shape[0]
        end = self._numbers("last", last, batch)
        if out is None:
            out, = self._made(stream, lambda: (_empty_like(lengths),))
            result = out.data_ptr()
        else:
            result = self._numbers("out", out, batch)
        status = self._accept(self._h, sequences, parent, end, cache, result, _raw_stream(self._index) if stream is None else stream)
        if status:
            raise sc.ScError(status, "sc_attention_accept")
        return out

    def fork(self, pages, lengths, holders, parents, wanted=None, out=None, workspace=None, stream=None):
        """The next batch of sequences: number i has the first rows of sequence parents[i] (-1: none), up to wanted[i] of them (all unless given), and pages for
        the rest of wanted[i] rows.  `lengths`: what the pages were given out for (after `accept`, those of before it).  Returns its pages and lengths (-1 for a sequence that is wrong or finds no free page), holders, and the copies of pages that
        `copy` has to make in every layer's cache before anything is written there (rows of `moves`: page, copy, rows).  `out`: those four, apart from the
        operands, but for holders, which may stay where they are.  `workspace`: device bytes of the caller's (binding.attention_pages_workspace_bytes)."""
        if _current_device() != self._index:
            return self._there(self.fork, pages, lengths, holders, parents, wanted, out, workspace, stream)
        batch, columns, page, page_ld = self._table(pages, lengths)
        new, count = parents.shape[0], holders.shape[0]
        operands = (self._numbers("lengths", lengths, batch), self._numbers("holders", holders, count), self._numbers("parents", parents, new),
                    0 if wanted is None else self._numbers("wanted", wanted, new))
        if out is None:
            out = table, after, held, moves = self._made(stream, lambda: (_empty_like(pages) if new == batch and page_ld >= columns else self._empty(new, columns), _empty_like(parents), _empty_like(holders),
                                                                          self._empty(new, 3)))
            results = table.data_ptr(), table.stride()[0], after.data_ptr(), held.data_ptr(), moves.data_ptr()
        else:
            results = self._results(out, ((new, columns), (new,), (count,), (new, 3)))
        self._pages_call(self._fork, "sc_attention_fork", (batch, new, count, page, page_ld, columns, *operands, *results), count, new, workspace, stream)
        return tuple(out)

    def compact(self, pages, lengths, holders, out=None, workspace=None, stream=None):
        """Moves the pages in use to the lowest numbers.  `lengths`: what the pages were given out for; entries behind them stay as they are.  Returns pages, holders and the moves that `copy` has to make in every layer's cache before anything
        is written there (rows: page, where it goes, rows).  `out`: those three; the first two may be the operands themselves."""
        if _current_device() != self._index:
            return self._there(self.compact, pages, lengths, holders, out, workspace, stream)
        batch, columns, page, page_ld = self._table(pages, lengths)
        count = holders.shape[0]
        length, held = self._numbers("lengths", lengths, batch), self._numbers("holders", holders, count)
        if out is None:
            out = table, after, moves = self._made(stream, lambda: (_empty_like(pages) if page_ld >= columns else self._empty(batch, columns), _empty_like(holders), self._empty(count // 2, 3)))
            table, table_ld, after, moves = table.data_ptr(), table.stride()[0], after.data_ptr(), moves.data_ptr()
        else:
            table, table_ld, after, moves = self._results(out, ((batch, columns), (count,), (count // 2, 3)))
        self._pages_call(self._compact, "sc_attention_compact", (batch, 0, count, page, page_ld, columns, length, held, 0, 0, table, table_ld, 0, after, moves), count, 0,
                         workspace, stream)
        return tuple(out)

    def copy(self, keys, values, moves, stream=None):
        """Copies the first rows of pages to other pages, as `fork` and `compact` say."""
        if _current_device() != self._index:
            return self._there(self.copy, keys, values, moves, stream)
        shape = moves.shape
        if len(shape) != 2:
            self._refuse_table("moves", "rows of three", moves)
        count = shape[0]
        status = self._copy(self._h, self._cache(keys, values), self._numbers("moves", moves, count, 3), count, _raw_stream(self._index) if stream is None else stream)
        if status:
            raise sc.ScError(status, "sc_attention_copy")

    def _there(self, operator, *args):
        with torch.cuda.device(self._index):
            return operator(*args)

    # -- records -----------------------------------------------------------------------------------------------------------
    # The host side of a call is most of the time of a short one: each attribute of a tensor is read once, and the messages are made apart.
    def _rows(self, x, shape):
        stride = x.stride()
        if (x.dtype is not self.dtype or x.get_device() != self._index or x.shape != shape or stride[2] != 1
                or x.requires_grad or _forward_ad._current_level >= 0):
            self._refuse_rows(x, shape)
        return _pack_rows(x.data_ptr(), stride[0], stride[1])

    def _refuse_rows(self, x, shape):
        if x.dtype is not self.dtype or x.get_device() != self._index:
            raise TypeError(f"rows have to be {self.dtype} on {self.device}, not {x.dtype} on {x.device}")
        if x.shape == shape and x.stride()[2] == 1:
            return self._refuse_gradient(x)
        raise ValueError(f"rows have to be {shape} with the last dimension contiguous, not {tuple(x.shape)} with strides {x.stride()}")

    def _refuse_gradient(self, *tensors):
        """Results have none: better an error than training that goes without.  Under torch.no_grad() it is as asked for."""
        if torch.is_grad_enabled() and any(x.requires_grad for x in tensors):
            raise RuntimeError("attention has no backward pass: an operand requires a gradient (call it under torch.no_grad(), or on detached tensors)")
        if _forward_ad._current_level >= 0 and any(_forward_ad.unpack_dual(x).tangent is not None for x in tensors):
            raise RuntimeError("attention has no derivative: an operand has a tangent")

    def _out(self, q, out, shape, stream):
        if out is not None:
            return out, self._rows(out, shape)
        if stream is not None and stream != _raw_stream(self._index):
            current = torch.cuda.current_stream(self.device)
            with self._memory_of(stream):
                out, result = self._out(q, None, shape, None)
            out.record_stream(current)
            return out, result
        out = _empty_like(q)
        stride = out.stride()
        if stride[2] != 1 or 0 in stride:   # of heads that share their memory, or a single one
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            stride = out.stride()
        return out, _pack_rows(out.data_ptr(), stride[0], stride[1])

    def _cache(self, keys, values):
        shape, stride, dtype = keys.shape, keys.stride(), self.dtype
        if (keys.dtype is not dtype or values.dtype is not dtype or keys.get_device() != self._index or values.get_device() != self._index
                or shape[1:] != self._page or stride[3] != 1 or values.shape != shape or values.stride() != stride
                or keys.requires_grad or values.requires_grad or _forward_ad._current_level >= 0):
            self._refuse_cache(keys, values)
        return _pack_cache(keys.data_ptr(), values.data_ptr(), shape[0], stride[0], stride[1], stride[2])

    def _refuse_cache(self, keys, values):
        if any(x.dtype is not self.dtype or x.get_device() != self._index for x in (keys, values)):
            raise TypeError(f"the cache has to be {self.dtype} on {self.device}, not {keys.dtype} on {keys.device} and {values.dtype} on {values.device}")
        if keys.shape[1:] == self._page and keys.stride()[3] == 1 and values.shape == keys.shape and values.stride() == keys.stride():
            return self._refuse_gradient(keys, values)
        raise ValueError(f"keys and values have to be (pages, {self.page_rows}, {self.kv_heads}, {self.head_dim}) alike, with the last "
                         f"dimension contiguous, not {tuple(keys.shape)} and {tuple(values.shape)} with strides {keys.stride()} and {values.stride()}")

    def _sequences(self, rows, row_start, lengths, pages):
        batch, starts, length, page, page_ld, columns = rows, 0, 0, 0, 0, 0
        if row_start is not None:
            shape = row_start.shape
            if row_start.dtype is not _INT32 or row_start.get_device() != self._index or len(shape) != 1 or not shape[0] or not row_start.is_contiguous():
                self._refuse_table("row_start", "one number more than sequences", row_start)
            batch, starts = shape[0] - 1, row_start.data_ptr()
        if lengths is not None:
            if lengths.dtype is not _INT32 or lengths.get_device() != self._index or lengths.shape != (batch,) or not lengths.is_contiguous():
                self._refuse_table("lengths", f"one for each of {batch} sequences", lengths)
            length = lengths.data_ptr()
        if pages is not None:
            shape, stride = pages.shape, pages.stride()
            if pages.dtype is not _INT32 or pages.get_device() != self._index or len(shape) != 2 or shape[0] != batch or (shape[1] > 1 and stride[1] != 1):
                self._refuse_table("pages", f"a row for each of {batch} sequences", pages)
            page, page_ld, columns = pages.data_ptr(), stride[0], shape[1]
        return _pack_sequences(batch, rows, starts, length, page, page_ld, columns)

    def _numbers(self, name, x, *shape):
        """Address of a contiguous table of that shape."""
        if x.dtype is not _INT32 or x.get_device() != self._index or x.shape != shape or not x.is_contiguous():
            self._refuse_table(name, " x ".join(str(n) for n in shape), x)
        return x.data_ptr()

    def _table(self, pages, lengths):
        shape, stride = pages.shape, pages.stride()
        if pages.dtype is not _INT32 or pages.get_device() != self._index or len(shape) != 2 or lengths.shape != shape[:1] or (shape[1] > 1 and stride[1] != 1):
            self._refuse_table("pages", f"a row for each of {tuple(lengths.shape)} sequences", pages)
        return shape[0], shape[1], pages.data_ptr(), stride[0]

    def _results(self, out, shapes):
        """Addresses of the tables that are written, of the first one its row stride too."""
        if len(out) != len(shapes):
            raise ValueError(f"out: {len(shapes)} tables, not {len(out)}")
        first, *rest = out
        stride = first.stride()
        if first.dtype is not _INT32 or first.get_device() != self._index or first.shape != shapes[0] or (shapes[0][1] > 1 and stride[1] != 1):
            self._refuse_table("out", " x ".join(str(n) for n in shapes[0]), first)
        return (first.data_ptr(), stride[0], *(self._numbers("out", x, *shape) for x, shape in zip(rest, shapes[1:])))

    def _empty(self, *shape):
        return torch.empty(shape, dtype=_INT32, device=self.device)

    def _made(self, stream, make):
        """Tables of the results, memory of the stream of the call."""
        if stream is None or stream == _raw_stream(self._index):
            return make()
        current = torch.cuda.current_stream(self.device)
        with self._memory_of(stream):
            tables = make()
        for x in tables:
            x.record_stream(current)
        return tables

    def _pages_call(self, call, name, record, count, new, workspace, stream):
        if stream is None:
            stream = _raw_stream(self._index)
        key = None
        if workspace is None:   # the handle's own, for as many pages and the next of a few sizes of batches: all of them stay, and most of a workspace goes by the pages
            key = count, 0 if new == 0 else 31 if new <= 31 else 2047 if new <= 2047 else 2 ** 17 - 1 if new < 2 ** 17 else 2 ** 20 - 1
            if key not in self._pages_bytes:
                self._pages_bytes[key] = sc.attention_pages_workspace_bytes(*key)
        address, size = self._workspace_of(stream, workspace, key)
        status = call(self._h, _pack_pages(*record), address, size, stream)
        if status:
            raise sc.ScError(status, name)

    def _refuse_table(self, name, what, x):
        raise ValueError(f"{name}: contiguous int32 on {self.device}, {what}; got {x.dtype} {tuple(x.shape)} with strides {x.stride()} on {x.device}")

    def _memory_of(self, stream):
        """What torch makes here is memory of `stream`: that of another may still be in use there, by kernels that this stream does not wait for."""
        return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=self.device))

    def _workspace_of(self, stream, given, name):
        """Address and size of a workspace: the caller's, or the handle's own, which is made once and stays where it is (a graph may hold its address)."""
        if given is not None:
            if given.get_device() != self._index:
                raise TypeError(f"a workspace has to be on {self.device}, not on {given.device}")
            if not given.is_contiguous():
                raise ValueError(f"a workspace has to be contiguous, not {tuple(given.shape)} with strides {given.stride()}")
            return given.data_ptr(), given.numel() * given.element_size()
        own = self._own.get(name)
        if own is None:
            with self._memory_of(stream):
                size = self._pages_bytes[name] if name in self._pages_bytes else getattr(self, name)
                own = self._own[name] = (torch.empty(size, dtype=torch.uint8, device=self.device), {stream})
        tensor, streams = own
        if stream not in streams:   # not given away before this stream is done with it either
            streams.add(stream)
            tensor.record_stream(torch.cuda.ExternalStream(stream, device=self.device))
        return tensor.data_ptr(), tensor.numel()
