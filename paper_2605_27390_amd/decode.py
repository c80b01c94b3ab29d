"""ctypes binding of include/evospec_decode.h: an 8-bit paged key/value cache, attention over it and sampling.
Argument marshalling only; tensors are torch tensors on the GPU, work goes to torch's current HIP stream."""
from __future__ import annotations

import ctypes
import functools

import torch

from .binding import _check, _expect, _get_device, _ptr, _raw_stream, lib

_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_KINDS = {"e4m3": 0, "int8": 1}
_i32, _f32 = torch.int32, torch.float32
_new = torch.empty_strided      # (strides spelled out: 0.9 us a tensor, torch.empty 1.6)


def _stream_of(device):
    """The current stream, for tensors of GPU `device`: work goes to the current GPU, which may not reach another one's memory."""
    current = _get_device()
    if device != current:
        raise ValueError(f"tensors are on GPU {device}, and the current one is {current}")
    return _raw_stream(current)


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


# The sizes that the library reports depend on few numbers, which are the same from call to call.
@functools.lru_cache(maxsize=256)
def _cache_bytes(pages, page, heads, dim, kind):
    nd, ns = _sz(0), _sz(0)
    _check(lib.evospec_kv_cache_bytes(ctypes.byref(_Cache(None, None, pages, page, heads, dim, kind)), ctypes.byref(nd),
                                      ctypes.byref(ns)), "evospec_kv_cache_bytes")
    return nd.value, ns.value


@functools.lru_cache(maxsize=256)
def _attention_bytes(pages, page, heads, dim, kind, group, S, T, max_rows, max_len):
    out = _sz(0)
    _check(lib.evospec_kv_attention_workspace_bytes(ctypes.byref(_Cache(None, None, pages, page, heads, dim, kind)), group, S, T,
                                                    max_rows, max_len, ctypes.byref(out)), "evospec_kv_attention_workspace_bytes")
    return out.value


@functools.lru_cache(maxsize=256)
def _sample_bytes(M, V):
    out = _sz(0)
    _check(lib.evospec_sample_workspace_bytes(M, V, ctypes.byref(out)), "evospec_sample_workspace_bytes")
    return out.value


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
        pages, page, heads, dim = int(pages), int(page), int(heads), int(dim)
        self.pages, self.page, self.heads, self.dim, self.kind = pages, page, heads, dim, kind
        n_data, n_scales = _cache_bytes(pages, page, heads, dim, _KINDS[kind])
        if data is None:
            data = torch.empty(n_data, dtype=torch.uint8, device=device)
        if scales is None:
            scales = torch.empty(n_scales // 4, dtype=torch.float32, device=device)
        dev = data.get_device()
        if not (data.dtype is torch.uint8 and scales.dtype is _f32 and dev >= 0 and scales.get_device() == dev and data.is_contiguous()
                and scales.is_contiguous()):
            _expect(data, torch.uint8, "data")
            _expect(scales, _f32, "scales")
            raise ValueError("data and scales are on different GPUs")
        if data.numel() < n_data or scales.numel() * 4 < n_scales:
            raise ValueError("data or scales is smaller than evospec_kv_cache_bytes reports")
        self.data, self.scales, self._device = data, scales, dev
        self._c = _Cache(data.data_ptr(), scales.data_ptr(), pages, page, heads, dim, _KINDS[kind])
        self._ref = ctypes.byref(self._c)


def _elsewhere(t, dev, name):
    if t.get_device() != dev:
        raise ValueError(f"{name} is on GPU {t.get_device()}, others are on {dev}")


def _rows(page_table, at, name, row_off, dev):
    """(width, S) of the index tensors of a call, which are on GPU `dev`.  (Checks here and below are written out: a call is about
    4 us of launch, and a function for each check cost another 3.)"""
    try:
        ok = (page_table.dtype is at.dtype is row_off.dtype is _i32
              and page_table.get_device() == at.get_device() == row_off.get_device() == dev
              and page_table.dim() == 2 and at.dim() == row_off.dim() == 1
              and page_table.is_contiguous() and at.is_contiguous() and row_off.is_contiguous())
    except AttributeError:
        ok = False
    if not ok:
        for t, n, ndim in ((page_table, "page_table", 2), (at, name, 1), (row_off, "row_off", 1)):
            _expect(t, _i32, n, ndim)
            _elsewhere(t, dev, n)
    S, width = page_table.shape
    if at.numel() != S or row_off.numel() != S + 1:
        raise ValueError(f"page_table, {name} and row_off disagree about the number of sequences")
    return width, S


def _strided(x, heads, dim, name, dev):
    """Row stride in elements of a tensor [T, heads, dim] on GPU `dev` whose rows are contiguous in themselves."""
    if not isinstance(x, torch.Tensor) or x.get_device() != dev:
        if not isinstance(x, torch.Tensor) or not x.is_cuda:
            raise TypeError(f"{name} must be a GPU torch tensor")
        _elsewhere(x, dev, name)
    if x.dim() != 3 or x.size(1) != heads or x.size(2) != dim:
        raise ValueError(f"{name} must be [rows, {heads}, {dim}], got {tuple(x.shape)}")
    s = x.stride()
    if s[2] != 1 or (s[1] != dim and heads > 1):
        raise ValueError(f"{name}: heads and elements of a row must be contiguous")
    return s[0] if x.size(0) > 1 else heads * dim


def kv_write(cache: KVCache, k, v, page_table, starts, row_off, max_rows: int) -> None:
    """Quantise rows row_off[s] .. row_off[s + 1] of k and v [T, heads, dim] into the cache as the tokens starts[s],
    starts[s] + 1, ... of sequence s.  No sequence may have more than max_rows of them."""
    width, S = _rows(page_table, starts, "starts", row_off, cache._device)
    ks, vs = _strided(k, cache.heads, cache.dim, "k", cache._device), _strided(v, cache.heads, cache.dim, "v", cache._device)
    type_ = _TYPES.get(k.dtype)
    if type_ is None or v.dtype != k.dtype:
        raise TypeError(f"k and v must share one of {list(_TYPES)}")
    T = k.size(0)
    if v.size(0) != T:
        raise ValueError("k and v differ in length")
    _check(lib.evospec_kv_write(cache._ref, k.data_ptr(), ks, v.data_ptr(), vs, type_, T, page_table.data_ptr(),
                                width, starts.data_ptr(), row_off.data_ptr(), S, max_rows, _stream_of(cache._device)), "evospec_kv_write")


def kv_read(cache: KVCache, page_table, starts, row_off, max_rows: int, rows: int, dtype=torch.bfloat16, out_k=None, out_v=None):
    """The values of the tokens starts[s], starts[s] + 1, ... of every sequence as rows row_off[s] .. row_off[s + 1]:
    (k, v), `dtype` [rows, heads, dim].  Rows that belong to no sequence are left as they are."""
    width, S = _rows(page_table, starts, "starts", row_off, cache._device)
    if dtype not in _TYPES:
        raise TypeError(f"dtype must be one of {list(_TYPES)}")
    rows = int(rows)
    shape = (rows, cache.heads, cache.dim)
    for t, name in ((out_k, "out_k"), (out_v, "out_v")):
        if t is not None:
            _expect(t, dtype, name, 3)
            _elsewhere(t, cache._device, name)
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
    if out_k is None:
        out_k = _new(shape, (cache.heads * cache.dim, cache.dim, 1), dtype=dtype, device=cache.data.device)
    if out_v is None:
        out_v = _new(shape, (cache.heads * cache.dim, cache.dim, 1), dtype=dtype, device=cache.data.device)
    _check(lib.evospec_kv_read(cache._ref, page_table.data_ptr(), width, starts.data_ptr(), row_off.data_ptr(), S, max_rows, rows,
                               _TYPES[dtype], out_k.data_ptr(), out_v.data_ptr(), _stream_of(cache._device)), "evospec_kv_read")
    return out_k, out_v


def kv_attention_workspace_bytes(cache: KVCache, group: int, S: int, T: int, max_rows: int, max_len: int) -> int:
    return _attention_bytes(cache.pages, cache.page, cache.heads, cache.dim, cache._c.kind, group, S, T, max_rows, max_len)


def kv_attention(q, cache: KVCache, page_table, lens, row_off, max_rows: int, max_len=None, tree=None, scale=None, out=None,
                 out_lse=None, workspace=None):
    """Attention of q [T, query heads, dim] (bf16 or fp16) over the cache: (out as q, lse fp32 [T, query heads]).  Rows
    row_off[s] .. row_off[s + 1] are the last tokens of sequence s, which has lens[s] tokens in the cache.  A row sees
    the tokens up to its own; with `tree` (int64 [T], bit j: the row sees the j-th of the sequence's rows) it sees all that
    come before the sequence's rows, and those of its bits.  `scale` is 1 / sqrt(dim) if not given; max_len (a bound of lens)
    only decides how the work is split.  Lengths have to lie within the page table.  No gradients: outputs do not require any."""
    width, S = _rows(page_table, lens, "lens", row_off, cache._device)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor [rows, query heads, dim]")
    T, heads, dim = q.shape
    group = heads // cache.heads
    if group * cache.heads != heads:
        raise ValueError("q must have a multiple of the cache's heads")
    qs = _strided(q, heads, cache.dim, "q", cache._device)
    type_ = _TYPES.get(q.dtype, 2)
    if type_ == 2:
        raise TypeError(f"q must be bfloat16 or float16, got {q.dtype}")
    if tree is not None:
        _expect(tree, torch.int64, "tree", 1)
        _elsewhere(tree, cache._device, "tree")
        if tree.shape[0] != T:
            raise ValueError("tree needs a word for every row of q")
    max_len = min(width * cache.page, 1 << 30) if max_len is None else int(max_len)
    if out is None:
        out = _new((T, heads, dim), (heads * dim, dim, 1), dtype=q.dtype, device=q.device)
    else:
        _expect(out, q.dtype, "out", 3)
        _elsewhere(out, cache._device, "out")
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    if out_lse is None:
        out_lse = _new((T, heads), (heads, 1), dtype=_f32, device=q.device)
    else:
        _expect(out_lse, torch.float32, "out_lse", 2)
        _elsewhere(out_lse, cache._device, "out_lse")
        if tuple(out_lse.shape) != (T, heads):
            raise ValueError("out_lse must be [rows, query heads]")
    if workspace is not None:
        _expect(workspace, torch.uint8, "workspace")
        _elsewhere(workspace, cache._device, "workspace")
    else:
        need = _attention_bytes(cache.pages, cache.page, cache.heads, cache.dim, cache._c.kind, group, S, T, max_rows, max_len)
        workspace = _new((need,), (1,), dtype=torch.uint8, device=q.device) if need else None
    _check(lib.evospec_kv_attention(cache._ref, q.data_ptr(), qs, type_, T, group, page_table.data_ptr(), width,
                                    lens.data_ptr(), row_off.data_ptr(), S, max_rows, max_len, _ptr(tree),
                                    dim ** -0.5 if scale is None else scale, out.data_ptr(), out_lse.data_ptr(), _ptr(workspace),
                                    0 if workspace is None else workspace.numel(), _stream_of(cache._device)), "evospec_kv_attention")
    return out, out_lse


def sample_workspace_bytes(M: int, V: int) -> int:
    return _sample_bytes(M, V)


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, ids=None, out_ids=None, out_logprob=None,
           workspace=None):
    """One token for each row of logits [M, V] (bf16, fp16, fp32) from u [M] in [0, 1): (ids int32 [M], logprob fp32 [M]).
    temperature, top_p, min_p are fp32 [M], top_k int32 [M], each may be None (1, all, all, all).  ids (int32 [V]) are the
    columns' token ids, as of an active vocabulary.  What is kept, and in which order u runs through it, is in
    include/evospec_decode.h; temperature 0 takes the largest logit."""
    if not isinstance(logits, torch.Tensor) or logits.get_device() < 0:
        raise TypeError("logits must be a GPU torch tensor")
    dev = logits.get_device()
    if logits.dtype not in _TYPES:
        raise TypeError(f"logits must be one of {list(_TYPES)}")
    if logits.dim() != 2 or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be [rows, columns] with contiguous rows")
    M, V = logits.shape
    for t, dtype, name in ((u, torch.float32, "u"), (temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"),
                           (top_p, torch.float32, "top_p"), (min_p, torch.float32, "min_p")):
        if t is not None or name == "u":
            if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == dev and t.dim() == 1 and t.is_contiguous()):
                _expect(t, dtype, name, 1)
                _elsewhere(t, dev, name)
            if t.numel() != M:
                raise ValueError(f"{name} needs a value for every row")
    if ids is not None:
        _expect(ids, torch.int32, "ids", 1)
        _elsewhere(ids, dev, "ids")
        if ids.shape[0] != V:
            raise ValueError("ids needs an id for every column")
    for t, dtype, name in ((out_ids, _i32, "out_ids"), (out_logprob, _f32, "out_logprob")):
        if t is not None:
            _expect(t, dtype, name, 1)
            _elsewhere(t, dev, name)
            if t.numel() != M:
                raise ValueError(f"{name} needs a place for every row")
    out_ids = _new((M,), (1,), dtype=_i32, device=logits.device) if out_ids is None else out_ids
    out_logprob = _new((M,), (1,), dtype=_f32, device=logits.device) if out_logprob is None else out_logprob
    if workspace is not None:
        _expect(workspace, torch.uint8, "workspace")
        _elsewhere(workspace, dev, "workspace")
    else:
        need = _sample_bytes(M, V)
        workspace = _new((need,), (1,), dtype=torch.uint8, device=logits.device) if need else None
    _check(lib.evospec_sample(logits.data_ptr(), logits.stride(0) if M > 1 else V, _TYPES[logits.dtype], M, V, u.data_ptr(),
                              _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), _ptr(ids), out_ids.data_ptr(),
                              out_logprob.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_of(dev)),
           "evospec_sample")
    return out_ids, out_logprob
