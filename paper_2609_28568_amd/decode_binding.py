"""ctypes binding of what answers are generated with (include/qwen3_decode.h) in
libgpt2_mi355x.so: a paged cache of keys and values, attention of new tokens
over it, and the adjustment of logits before a token is chosen.

Argument marshalling only: torch supplies the device buffers and the stream,
everything runs in the library's HIP kernels. No call synchronises, so all of
them can be captured into graphs: lengths, tables and counts are read on the
device when a graph is replayed.
"""
from __future__ import annotations

import ctypes
import struct

from .binding import i32, on_stream
from .qwen3_binding import _check, _device_rows, lib as _lib_qwen3


class Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layer", "n_kv_head", "head_dim", "page_size", "n_pages", "n_seq",
                                              "max_pages")] + [
        (n, ctypes.c_void_p) for n in ("d_pages", "d_table", "d_lens", "d_refs", "d_short", "d_scratch")]


class Tree(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_head", "n_rows", "max_new", "layer", "mask_words")]


class Logits(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "vocab", "dtype")] + [
        (n, ctypes.c_int64) for n in ("logits_stride", "out_stride")] + [
        (n, ctypes.c_int32) for n in ("n_seq", "history_stride", "path_len", "n_bias", "n_masks")] + [
        (n, ctypes.c_void_p) for n in ("d_history", "d_prompt_lens", "d_lens", "d_row_seq", "d_path", "d_repetition",
                                       "d_frequency", "d_presence", "d_bias_ids", "d_bias", "d_masks", "d_row_mask")]


# the same fields, with C's padding
_LOGITS = struct.Struct("@3i2q5i12P")
assert _LOGITS.size == ctypes.sizeof(Logits)

_lib = None


def lib():
    """The shared library with the prototypes of qwen3_decode.h declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = _lib_qwen3()
    P, I32, SIZE = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    cache, tree = ctypes.POINTER(Cache), ctypes.POINTER(Tree)
    protos = {
        "qwen3_cache_scratch": [cache, ctypes.POINTER(SIZE)],
        "qwen3_cache_fork": [cache, P, P, P],
        "qwen3_cache_append": [cache, P, I32, I32, SIZE, P, P, P, I32, P],
        "qwen3_cache_compact": [cache, P],
        "qwen3_tree_size": [cache, tree, ctypes.POINTER(SIZE)],
        "qwen3_tree_attention": [cache, tree, P, P, P, P, P, P, SIZE, P],
        "qwen3_tree_positions": [cache, tree, P, P, P, P],
        "qwen3_set_cache_size": [P, cache, I32, ctypes.POINTER(SIZE)],
        "qwen3_set_cache": [P, cache, P, P, I32, I32, P, SIZE],
        "qwen3_keep_tokens": [P, P, P, I32],
        "qwen3_logits_info": [P, ctypes.POINTER(SIZE), ctypes.POINTER(I32)],
        "qwen3_adjust_logits": [P, P, P, P],
    }
    for name, args in protos.items():
        f = getattr(L, name)
        f.restype, f.argtypes = I32, args
    _lib = L
    return L


class PagedCache:
    """Keys and values of some sequences on pages that they may share
    (qwen3_cache_*). Its calls run one after another, on the current stream,
    which the caller orders where there are several; the tensors are the
    caller's to read, and to save and restore, and are not freed before the
    streams of the calls are done with them."""

    def __init__(self, pages, table, lens, refs, short):
        """Over tensors that hold a cache: pages bf16 [n_layer, n_pages, 2,
        n_kv_head, page_size, head_dim], table int32 [n_seq, max_pages], lens
        int32 [n_seq], refs int32 [n_pages], short int32 [1] (qwen3_cache)."""
        import torch
        self.torch = torch
        _device_rows(pages, "pages", torch.bfloat16)
        if pages.dim() != 6 or pages.shape[2] != 2:
            raise ValueError("pages are [n_layer, n_pages, 2, n_kv_head, page_size, head_dim]")
        n_layer, n_pages, _, n_kv_head, page_size, head_dim = map(i32, pages.shape)
        _device_rows(table, "table", torch.int32, pages)
        if table.dim() != 2:
            raise ValueError("the table is [n_seq, max_pages]")
        n_seq, max_pages = map(i32, table.shape)
        _device_rows(lens, "lens", torch.int32, pages, (n_seq,))
        _device_rows(refs, "refs", torch.int32, pages, (n_pages,))
        _device_rows(short, "short", torch.int32, pages, (1,))
        self.pages, self.table, self.lens, self.refs, self.short = pages, table, lens, refs, short
        c = Cache(n_layer, n_kv_head, head_dim, page_size, n_pages, n_seq, max_pages)
        n = ctypes.c_size_t()
        _check(lib().qwen3_cache_scratch(ctypes.byref(c), ctypes.byref(n)))
        self.scratch = torch.empty(n.value, dtype=torch.uint8, device=pages.device)
        for name in ("pages", "table", "lens", "refs", "short", "scratch"):
            setattr(c, "d_" + name, getattr(self, name).data_ptr())
        self._c, self._ref = c, ctypes.byref(c)
        self._streams = {torch.cuda.current_stream(pages.device).cuda_stream}   # that the tensors are kept for
        self._n_seq, self._index = n_seq, pages.get_device()
        self._trees, self._heads = {}, {}

    @classmethod
    def empty(cls, n_layer, n_pages, n_kv_head, page_size, head_dim, n_seq, max_pages, device="cuda"):
        """A cache without tokens."""
        import torch
        new = lambda shape, v: torch.full(shape, v, dtype=torch.int32, device=device)   # noqa: E731
        pages = torch.empty(n_layer, n_pages, 2, n_kv_head, page_size, head_dim, dtype=torch.bfloat16, device=device)
        return cls(pages, new((n_seq, max_pages), -1), new((n_seq,), 0), new((n_pages,), 0), new((1,), 0))

    def _run(self, fn, *args):
        torch, index = self.torch, self._index
        stream = torch._C._cuda_getCurrentRawStream(index)
        if stream not in self._streams:   # memory of another stream's: it stays until this one is done with it
            for t in (self.pages, self.table, self.lens, self.refs, self.short, self.scratch):
                t.record_stream(torch.cuda.current_stream(index))
            self._streams.add(stream)
        if torch.cuda.current_device() == index:
            _check(fn(self._ref, *args, stream))
        else:
            with torch.cuda.device(index):
                _check(fn(self._ref, *args, stream))

    def _given(self, t, name, shape, dtype):
        torch = self.torch
        if not (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.get_device() == self._index
                and t.is_contiguous()):
            _device_rows(t, name, dtype, self.pages, shape)
        return t.data_ptr()

    def _ints(self, t, name, shape):
        return self._given(t, name, shape, self.torch.int32)

    def fork(self, src, keep=None):
        """Sequence s becomes the first keep[s] tokens (None: all) of what
        sequence src[s] was; src[s] -1: it is freed (qwen3_cache_fork)."""
        n = (self._n_seq,)
        self._run(lib().qwen3_cache_fork, self._ints(src, "src", n), None if keep is None else self._ints(keep, "keep", n))

    def _rows(self, qkv, layers):
        """(n_head, rows, address) of q | k | v rows, of `layers` layers or (0) of one."""
        shape = tuple(qkv.shape)
        got = self._heads.get((shape, layers))
        if got is None:
            if len(shape) != (3 if layers else 2) or (layers and shape[0] != layers):
                raise ValueError("rows of q | k | v are [rows, (n_head + 2 n_kv_head) head_dim], of every layer for append")
            n_head = shape[-1] // self._c.head_dim - 2 * self._c.n_kv_head
            if n_head < 1 or shape[-1] % self._c.head_dim:
                raise ValueError("rows of q | k | v are (n_head + 2 n_kv_head) head_dim wide")
            if len(self._heads) >= 256:
                self._heads.clear()
            got = self._heads[shape, layers] = i32(n_head), i32(shape[-2])
        return (*got, self._given(qkv, "q | k | v", qkv.shape, self.torch.bfloat16))

    def append(self, qkv, starts, max_new, counts=None, path=None):
        """Keys and values of new tokens, of all layers (qwen3_cache_append):
        qkv bf16 [n_layer, rows, (n_head + 2 n_kv_head) head_dim], sequence s's
        rows starts[s]..starts[s + 1] - 1, of which it takes the first
        counts[s] (None: all), or those that path int32 [n_seq, max_new] names.
        `short` then holds the number of pages that were missing; unless it is
        0 nothing was appended."""
        if qkv.dim() == 2:
            qkv = qkv[None]
        n_head, rows, at = self._rows(qkv, self._c.n_layer)
        max_new, n = i32(max_new), self._n_seq
        self._run(lib().qwen3_cache_append, at, n_head, rows, rows * qkv.shape[2], self._ints(starts, "starts", (n + 1,)),
                  None if counts is None else self._ints(counts, "counts", (n,)),
                  None if path is None else self._ints(path, "path", (n, max_new)), max_new)

    def compact(self):
        """Moves the pages in use to the lowest numbers (qwen3_cache_compact)."""
        self._run(lib().qwen3_cache_compact)

    def _tree(self, n_head, rows, max_new, layer, words):
        """The call's description, workspace bytes and the result's width, made once per shape."""
        key = n_head, rows, max_new, layer, words
        got = self._trees.get(key)
        if got is None:
            t, n = Tree(*key), ctypes.c_size_t()
            _check(lib().qwen3_tree_size(self._ref, ctypes.byref(t), ctypes.byref(n)))
            if len(self._trees) >= 256:
                self._trees.clear()
            got = self._trees[key] = ctypes.byref(t), n.value, n_head * self._c.head_dim
        return got

    def attention(self, qkv, starts, max_new, mask=None, layer=0, out=None, lse=None):
        """(out [rows, n_head head_dim] bf16, lse [n_head, rows] fp32) of new
        tokens' rows qkv bf16 [rows, (n_head + 2 n_kv_head) head_dim] over one
        layer of the cache and among themselves (qwen3_tree_attention): without
        a mask in order, with mask int32 [rows, words] (tree_mask) as its bits
        say. Sequence s's rows are starts[s]..starts[s + 1] - 1, max_new at
        most."""
        torch = self.torch
        n_head, rows, at = self._rows(qkv, 0)
        first = self._ints(starts, "starts", (self._n_seq + 1,))
        words = bits = 0
        if mask is not None:
            words = mask_words(mask)
            bits = self._ints(mask, "mask", (rows, words))
        tree, nbytes, width = self._tree(n_head, rows, i32(max_new), i32(layer), words)
        if out is None:
            out = torch.empty(rows, width, dtype=torch.bfloat16, device=qkv.device)
        if lse is None:
            lse = torch.empty(n_head, rows, dtype=torch.float32, device=qkv.device)
        work = torch.empty(nbytes, dtype=torch.uint8, device=qkv.device)
        self._run(lib().qwen3_tree_attention, tree, at, first, bits or None,
                  self._given(out, "out", (rows, width), torch.bfloat16),
                  self._given(lse, "lse", (n_head, rows), torch.float32), work.data_ptr(), nbytes)
        return out, lse

    def positions(self, starts, rows, mask=None, out=None):
        """int32 [1, rows]: the rows' places in their sequences, for rotary
        (qwen3_tree_positions)."""
        torch = self.torch
        words, bits = 0, None
        if mask is not None:
            words = mask_words(mask)
            bits = self._ints(mask, "mask", (rows, words))
        t = Tree(self._c.n_kv_head, i32(rows), 1, 0, words)
        if out is None:
            out = torch.empty(1, rows, dtype=torch.int32, device=self.pages.device)
        self._run(lib().qwen3_tree_positions, ctypes.byref(t), self._ints(starts, "starts", (self._n_seq + 1,)), bits,
                  self._ints(out, "out", (1, rows)))
        return out


def mask_words(mask):
    """Words of a mask's rows; 1 at least, as an empty tensor has no address."""
    if mask.dim() != 2 or mask.shape[1] < 1:
        raise ValueError("a mask is [rows, words], a word or more")
    return i32(mask.shape[1])


def tree_mask(parents, device="cuda"):
    """The mask of trees of drafted tokens for PagedCache.attention: parents, a
    list for each sequence with the place of every token's parent among the
    sequence's tokens before it, or -1."""
    import numpy as np
    import torch
    words = max([(len(p) + 31) // 32 for p in parents] + [1])
    out = np.zeros((sum(map(len, parents)), words), np.uint32)
    at = 0
    for p in parents:
        for i, up in enumerate(p):
            if not -1 <= up < i:
                raise ValueError(f"the parent of token {i} must be -1 or a token before it")
            if up >= 0:
                out[at + i] = out[at + up]
            out[at + i, i // 32] |= np.uint32(1 << (i % 32))
        at += len(p)
    return torch.from_numpy(out.view(np.int32)).to(device)


def adjust_logits(logits, history=None, prompt_lens=None, lens=None, repetition=None, frequency=None, presence=None,
                  *, row_seq=None, path=None, bias_ids=None, bias=None, masks=None, row_mask=None, out=None):
    """Penalties for repeated tokens, biases and grammar masks on logits bf16 or
    fp32 [rows, vocab], whose rows may be further apart (qwen3_adjust_logits).
    history int32 [n_seq, longest], lens and prompt_lens int32 [n_seq] (the
    tokens that count as repeated begin behind the prompt), row_seq int32 [rows]
    each row's sequence; path int32 [rows, k] a row's own further tokens, -1
    where there is none; repetition, frequency and presence fp32 [rows]; bias_ids
    int32 and bias fp32 [rows, k]; masks int32 [n_masks, ceil(vocab / 32)], a bit
    for each allowed token, and row_mask int32 [rows], -1 for no mask. On the
    current stream; out may be logits."""
    import torch
    if not (isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 2
            and logits.dtype in (torch.bfloat16, torch.float32) and (logits.stride(1) == 1 or logits.shape[1] == 1)
            and logits.shape[1] > 0):
        raise ValueError("logits are a bf16 or fp32 device tensor [rows, vocab] whose columns are contiguous")
    rows, vocab = logits.shape
    if out is None:
        out = torch.empty(rows, vocab, dtype=logits.dtype, device=logits.device)
    elif (out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device
          or (out.stride(1) != 1 and vocab > 1)):
        raise ValueError("out must have the logits' shape, type and device, its columns contiguous")

    device, index = logits.device, logits.get_device()

    def given(t, name, dtype, shape):
        if not (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.get_device() == index
                and t.is_contiguous()):
            _device_rows(t, name, dtype, logits, shape)
        return t.data_ptr()

    I, F = torch.int32, torch.float32
    per_row = (rows,)
    n_seq = stride = path_len = n_bias = n_masks = 0
    if history is not None:
        if history.dim() != 2 or lens is None:
            raise ValueError("a history is [n_seq, longest], with lens")
        n_seq, stride = history.shape
    if path is not None:
        if path.dim() != 2:
            raise ValueError("a path is [rows, k]")
        path_len = path.shape[1]
    if bias is not None or bias_ids is not None:
        if bias is None or bias_ids is None or bias.dim() != 2:
            raise ValueError("bias and bias_ids go together, [rows, k]")
        n_bias = bias.shape[1]
    if masks is not None:
        if masks.dim() != 2:
            raise ValueError("masks are [n_masks, ceil(vocab / 32)]")
        n_masks = masks.shape[0]
    i32(max(rows, vocab, n_seq, stride, path_len, n_bias, n_masks))
    # (a packed description: setting 22 fields of a structure takes 3 us)
    desc = _LOGITS.pack(rows, vocab, logits.dtype is torch.bfloat16, logits.stride(0) if rows > 1 else vocab,
                        out.stride(0) if rows > 1 else vocab, n_seq, stride, path_len, n_bias, n_masks,
                        given(history, "history", I, (n_seq, stride)) if stride else 0,
                        0 if prompt_lens is None else given(prompt_lens, "prompt_lens", I, (n_seq,)),
                        0 if lens is None else given(lens, "lens", I, (n_seq,)),
                        0 if row_seq is None else given(row_seq, "row_seq", I, per_row),
                        0 if path is None else given(path, "path", I, (rows, path_len)),
                        0 if repetition is None else given(repetition, "repetition", F, per_row),
                        0 if frequency is None else given(frequency, "frequency", F, per_row),
                        0 if presence is None else given(presence, "presence", F, per_row),
                        0 if bias_ids is None else given(bias_ids, "bias_ids", I, (rows, n_bias)),
                        0 if bias is None else given(bias, "bias", F, (rows, n_bias)),
                        0 if masks is None else given(masks, "masks", I, (n_masks, (vocab + 31) // 32)),
                        0 if row_mask is None else given(row_mask, "row_mask", I, per_row))
    _check(on_stream(device, lib().qwen3_adjust_logits, desc, logits.data_ptr(), out.data_ptr()))
    return out
