"""ctypes binding of include/evospec_decode.h: an 8-bit paged key/value cache, attention over it and sampling.
Argument marshalling only; tensors are torch tensors on the GPU, work goes to torch's current HIP stream."""
from __future__ import annotations

import ctypes

import torch

from .binding import _check, _expect, _ptr, _stream, lib

_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_KINDS = {"e4m3": 0, "int8": 1}


class _Cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p)] + [
        (n, ctypes.c_int) for n in ("pages", "page", "heads", "dim", "kind")]


_vp, _ci, _ll, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t
_szp = ctypes.POINTER(_sz)
_cachep = ctypes.POINTER(_Cache)
for _name, _args in {
        "evospec_kv_cache_bytes": [_cachep, _szp, _szp],
        "evospec_kv_write": [_cachep, _vp, _ll, _vp, _ll, _ci, _ci, _vp, _ci, _vp, _vp, _ci, _ci, _vp],
        "evospec_kv_read": [_cachep, _vp, _ci, _vp, _vp, _ci, _ci, _ci, _ci, _vp, _vp, _vp],
        "evospec_kv_attention_workspace_bytes": [_cachep, _ci, _ci, _ci, _ci, _ci, _szp],
        "evospec_kv_attention": [_cachep, _vp, _ll, _ci, _ci, _ci, _vp, _ci, _vp, _vp, _ci, _ci, _ci, _vp, ctypes.c_float,
                                 _vp, _vp, _vp, _sz, _vp],
        "evospec_sample_workspace_bytes": [_ci, _ci, _szp],
        "evospec_sample": [_vp, _ll, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]}.items():
    getattr(lib, _name).restype = _ci
    getattr(lib, _name).argtypes = _args


class KVCache:
    """A paged key/value cache of one layer in 8 bits: `pages` pages of `page` tokens (32, 64, 128, 256) for `heads` heads
    of `dim` elements (64, 96, 128, 192, 256), `kind` "e4m3" or "int8".  32 tokens of a head are a block; K and V of a block
    have a scale each.  `data` (uint8) and `scales` (float32) are the buffers in the layout of include/evospec_decode.h,
    allocated here or the caller's.

    Sequences find their tokens through a page table, int32 [S, width] on the GPU: token t of sequence s is in page
    page_table[s, t // page]."""

    def __init__(self, pages: int, page: int, heads: int, dim: int, kind: str = "e4m3", device="cuda", data=None, scales=None):
        if kind not in _KINDS:
            raise ValueError(f"kind must be one of {sorted(_KINDS)}, got {kind!r}")
        self.pages, self.page, self.heads, self.dim, self.kind = int(pages), int(page), int(heads), int(dim), kind
        self._c = _Cache(None, None, self.pages, self.page, self.heads, self.dim, _KINDS[kind])
        self._ref = ctypes.byref(self._c)
        nd, ns = _sz(0), _sz(0)
        _check(lib.evospec_kv_cache_bytes(self._ref, ctypes.byref(nd), ctypes.byref(ns)), "evospec_kv_cache_bytes")
        if data is None:
            data = torch.empty(nd.value, dtype=torch.uint8, device=device)
        if scales is None:
            scales = torch.empty(ns.value // 4, dtype=torch.float32, device=device)
        _expect(data, torch.uint8, "data")
        _expect(scales, torch.float32, "scales")
        if data.numel() < nd.value or scales.numel() * 4 < ns.value:
            raise ValueError("data or scales is smaller than evospec_kv_cache_bytes reports")
        self.data, self.scales = data, scales
        self._c.data, self._c.scales = data.data_ptr(), scales.data_ptr()


def _rows(page_table, at, name, row_off):
    """(width, S) of the index tensors of a call."""
    _expect(page_table, torch.int32, "page_table", 2)
    _expect(at, torch.int32, name, 1)
    _expect(row_off, torch.int32, "row_off", 1)
    S, width = page_table.shape
    if at.shape[0] != S or row_off.shape[0] != S + 1:
        raise ValueError(f"page_table, {name} and row_off disagree about the number of sequences")
    return width, S


def _strided(x, shape, name):
    """Row stride in elements of a GPU tensor [T, heads, dim] whose rows are contiguous in themselves."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError(f"{name} must be a GPU torch tensor")
    if x.dim() != 3 or tuple(x.shape[1:]) != shape:
        raise ValueError(f"{name} must be [rows, {shape[0]}, {shape[1]}], got {tuple(x.shape)}")
    if x.stride(2) != 1 or (x.stride(1) != shape[1] and shape[0] > 1):
        raise ValueError(f"{name}: heads and elements of a row must be contiguous")
    return x.stride(0) if x.shape[0] > 1 else shape[0] * shape[1]


def kv_write(cache: KVCache, k, v, page_table, starts, row_off, max_rows: int) -> None:
    """Quantise rows row_off[s] .. row_off[s + 1] of k and v [T, heads, dim] into the cache as the tokens starts[s],
    starts[s] + 1, ... of sequence s.  No sequence may have more than max_rows of them."""
    width, S = _rows(page_table, starts, "starts", row_off)
    shape = (cache.heads, cache.dim)
    ks, vs = _strided(k, shape, "k"), _strided(v, shape, "v")
    if k.dtype not in _TYPES or v.dtype != k.dtype:
        raise TypeError(f"k and v must share one of {list(_TYPES)}")
    if v.shape[0] != k.shape[0]:
        raise ValueError("k and v differ in length")
    _check(lib.evospec_kv_write(cache._ref, k.data_ptr(), ks, v.data_ptr(), vs, _TYPES[k.dtype], k.shape[0], page_table.data_ptr(),
                                width, starts.data_ptr(), row_off.data_ptr(), S, max_rows, _stream()), "evospec_kv_write")


def kv_read(cache: KVCache, page_table, starts, row_off, max_rows: int, rows: int, dtype=torch.bfloat16, out_k=None, out_v=None):
    """The values of the tokens starts[s], starts[s] + 1, ... of every sequence as rows row_off[s] .. row_off[s + 1]:
    (k, v), `dtype` [rows, heads, dim].  Rows that belong to no sequence are left as they are."""
    width, S = _rows(page_table, starts, "starts", row_off)
    if dtype not in _TYPES:
        raise TypeError(f"dtype must be one of {list(_TYPES)}")
    shape = (int(rows), cache.heads, cache.dim)
    out_k = torch.empty(shape, dtype=dtype, device=cache.data.device) if out_k is None else out_k
    out_v = torch.empty(shape, dtype=dtype, device=cache.data.device) if out_v is None else out_v
    for t, name in ((out_k, "out_k"), (out_v, "out_v")):
        _expect(t, dtype, name, 3)
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
    _check(lib.evospec_kv_read(cache._ref, page_table.data_ptr(), width, starts.data_ptr(), row_off.data_ptr(), S, max_rows, shape[0],
                               _TYPES[dtype], out_k.data_ptr(), out_v.data_ptr(), _stream()), "evospec_kv_read")
    return out_k, out_v


def kv_attention_workspace_bytes(cache: KVCache, group: int, S: int, T: int, max_rows: int, max_len: int) -> int:
    out = _sz(0)
    _check(lib.evospec_kv_attention_workspace_bytes(cache._ref, int(group), int(S), int(T), int(max_rows), int(max_len),
                                                    ctypes.byref(out)), "evospec_kv_attention_workspace_bytes")
    return int(out.value)


def kv_attention(q, cache: KVCache, page_table, lens, row_off, max_rows: int, max_len=None, tree=None, scale=None, out=None,
                 out_lse=None, workspace=None):
    """Attention of q [T, query heads, dim] (bf16 or fp16) over the cache: (out as q, lse fp32 [T, query heads]).  Rows
    row_off[s] .. row_off[s + 1] are the last tokens of sequence s, which has lens[s] tokens in the cache.  A row sees
    the tokens up to its own; with `tree` (int64 [T], bit j: the row sees the j-th of the sequence's rows) it sees all that
    come before the sequence's rows, and those of its bits.  `scale` is 1 / sqrt(dim) if not given; max_len (a bound of lens)
    only decides how the work is split."""
    width, S = _rows(page_table, lens, "lens", row_off)
    if q.dim() != 3 or q.shape[1] % cache.heads:
        raise ValueError("q must be [rows, a multiple of the cache's heads, dim]")
    T, heads, dim = q.shape
    qs = _strided(q, (heads, cache.dim), "q")
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"q must be bfloat16 or float16, got {q.dtype}")
    if tree is not None:
        _expect(tree, torch.int64, "tree", 1)
        if tree.shape[0] != T:
            raise ValueError("tree needs a word for every row of q")
    group = heads // cache.heads
    max_len = width * cache.page if max_len is None else int(max_len)
    if out is None:
        out = torch.empty((T, heads, dim), dtype=q.dtype, device=q.device)
    else:
        _expect(out, q.dtype, "out", 3)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    if out_lse is None:
        out_lse = torch.empty((T, heads), dtype=torch.float32, device=q.device)
    else:
        _expect(out_lse, torch.float32, "out_lse", 2)
        if tuple(out_lse.shape) != (T, heads):
            raise ValueError("out_lse must be [rows, query heads]")
    if workspace is None:
        need = kv_attention_workspace_bytes(cache, group, S, T, max_rows, max_len)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _check(lib.evospec_kv_attention(cache._ref, q.data_ptr(), qs, _TYPES[q.dtype], T, group, page_table.data_ptr(), width,
                                    lens.data_ptr(), row_off.data_ptr(), S, max_rows, max_len, _ptr(tree),
                                    dim ** -0.5 if scale is None else scale, out.data_ptr(), out_lse.data_ptr(), _ptr(workspace),
                                    0 if workspace is None else workspace.numel(), _stream()), "evospec_kv_attention")
    return out, out_lse


def sample_workspace_bytes(M: int, V: int) -> int:
    out = _sz(0)
    _check(lib.evospec_sample_workspace_bytes(int(M), int(V), ctypes.byref(out)), "evospec_sample_workspace_bytes")
    return int(out.value)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, ids=None, out_ids=None, out_logprob=None,
           workspace=None):
    """One token for each row of logits [M, V] (bf16, fp16, fp32) from u [M] in [0, 1): (ids int32 [M], logprob fp32 [M]).
    temperature, top_p, min_p are fp32 [M], top_k int32 [M], each may be None (1, all, all, all).  ids (int32 [V]) are the
    columns' token ids, as of an active vocabulary.  What is kept, and in which order u runs through it, is in
    include/evospec_decode.h; temperature 0 takes the largest logit."""
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise TypeError("logits must be a GPU torch tensor")
    if logits.dtype not in _TYPES:
        raise TypeError(f"logits must be one of {list(_TYPES)}")
    if logits.dim() != 2 or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be [rows, columns] with contiguous rows")
    M, V = logits.shape
    for t, dtype, name in ((u, torch.float32, "u"), (temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"),
                           (top_p, torch.float32, "top_p"), (min_p, torch.float32, "min_p")):
        if t is not None or name == "u":
            _expect(t, dtype, name, 1)
            if t.shape[0] != M:
                raise ValueError(f"{name} needs a value for every row")
    if ids is not None:
        _expect(ids, torch.int32, "ids", 1)
        if ids.shape[0] != V:
            raise ValueError("ids needs an id for every column")
    out_ids = torch.empty(M, dtype=torch.int32, device=logits.device) if out_ids is None else out_ids
    out_logprob = torch.empty(M, dtype=torch.float32, device=logits.device) if out_logprob is None else out_logprob
    for t, dtype, name in ((out_ids, torch.int32, "out_ids"), (out_logprob, torch.float32, "out_logprob")):
        _expect(t, dtype, name, 1)
        if t.shape[0] != M:
            raise ValueError(f"{name} needs a place for every row")
    if workspace is None:
        need = sample_workspace_bytes(M, V)
        workspace = torch.empty(need, dtype=torch.uint8, device=logits.device) if need else None
    _check(lib.evospec_sample(logits.data_ptr(), logits.stride(0) if M > 1 else V, _TYPES[logits.dtype], M, V, u.data_ptr(),
                              _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), _ptr(ids), out_ids.data_ptr(),
                              out_logprob.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream()),
           "evospec_sample")
    return out_ids, out_logprob
