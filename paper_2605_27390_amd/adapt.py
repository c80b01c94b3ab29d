"""ctypes binding of include/evospec_adapt.h: low-rank adapters of many requests, the distillation loss on the retained support and
AdamW.  Argument marshalling only; tensors are torch tensors on the GPU, work goes to torch's current HIP stream.  Gradients are outputs of
the calls: nothing here takes part in autograd.  What a call changes in place is a new version to torch, so that a graph that saved the old one says so,
and y, dx or an output that requires a gradient is refused while gradients are recorded, since what the call adds would be missing from them."""
from __future__ import annotations

import ctypes
import functools

import torch
from torch.autograd.graph import increment_version as _changed

from .binding import _check, _expect, _ptr, lib
from .decode import _TYPES, _elsewhere, _new, _stream_of

_bf16, _f32, _i32 = torch.bfloat16, torch.float32, torch.int32
_MOMENTS = {"fp32": 0, "8bit": 1}
ADAMW_BLOCK = 256


class _Lora(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("a", "b", "scale")] + [(n, ctypes.c_int) for n in ("n", "r", "d_in", "d_out")]


class _Tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("n", ctypes.c_longlong)]


_vp, _ci, _ll, _sz, _d = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t, ctypes.c_double
_szp, _lorap, _tensorp = ctypes.POINTER(_sz), ctypes.POINTER(_Lora), ctypes.POINTER(_Tensor)
for _name, _args in {
        "evospec_lora_forward": [_lorap, _vp, _ll, _vp, _vp, _ci, _ci, _vp, _ll, _vp, _vp],
        "evospec_lora_backward_workspace_bytes": [_lorap, _ci, _ci, _szp],
        "evospec_lora_backward": [_lorap, _vp, _ll, _vp, _vp, _ll, _vp, _vp, _ci, _ci, _vp, _ll, _vp, _vp, _vp, _sz, _vp],
        "evospec_kd_loss_workspace_bytes": [_ci, _ci, _ci, _szp],
        "evospec_kd_loss": [_vp, _ci, _ci, _vp, _ci, _vp, _vp, _vp, _ci, ctypes.c_float, _ci, _vp, _vp, _vp, _vp, _sz, _vp],
        "evospec_adamw_blocks": [_tensorp, _ci, ctypes.POINTER(_ll)],
        "evospec_adamw_step": [_tensorp, _ci, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _d, _d, _d, _d, _d, _ll, ctypes.c_uint32, _vp, _vp, _vp],
        "evospec_adamw_moments": [_vp, _vp, _vp, _ll, _ci, _vp, _vp, _vp]}.items():
    getattr(lib, _name).restype = _ci
    getattr(lib, _name).argtypes = _args


# The sizes that the library reports depend on few numbers, which are the same from call to call.
@functools.lru_cache(maxsize=256)
def _lora_bytes(n, r, d_in, d_out, S, T):
    out = _sz(0)
    _check(lib.evospec_lora_backward_workspace_bytes(ctypes.byref(_Lora(None, None, None, n, r, d_in, d_out)), S, T, ctypes.byref(out)),
           "evospec_lora_backward_workspace_bytes")
    return out.value


@functools.lru_cache(maxsize=256)
def _kd_bytes(E, K, d):
    out = _sz(0)
    _check(lib.evospec_kd_loss_workspace_bytes(E, K, d, ctypes.byref(out)), "evospec_kd_loss_workspace_bytes")
    return out.value


def _workspace_of(workspace, need, dev, device):
    """A workspace on GPU `dev`: the caller's, or a new one."""
    if workspace is not None:
        _expect(workspace, torch.uint8, "workspace")
        _elsewhere(workspace, dev, "workspace")
        return workspace
    return _new((need,), (1,), dtype=torch.uint8, device=device) if need else None


def _recorded(t, name):
    """Refuses a tensor that is written where torch records gradients and t has one."""
    if torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and the call takes no part in autograd: detach it, or call under torch.no_grad()")


def _fixed(name):
    """A handle's tensor: its address went to the library, so another one cannot take its place."""
    return property(lambda self: getattr(self, name))


class LoraBank:
    """Adapters of one projection: a bf16 [n, r, d_in], b bf16 [n, d_out, r], scale fp32 [n] or None (1).  r is a multiple of 8 up to
    64; adapters of a smaller rank are padded with zeros.  The tensors' values are used as they are at each call; the handle keeps the tensors
    and their addresses, so that their memory must stay theirs (no `.data = ...`, no `set_`)."""
    a, b, scale = _fixed("_a"), _fixed("_b"), _fixed("_scale")

    def __init__(self, a, b, scale=None):
        _expect(a, _bf16, "a", 3)
        _expect(b, _bf16, "b", 3)
        self._device = a.get_device()
        _elsewhere(b, self._device, "b")
        self.n, self.r, self.d_in = a.shape
        self.d_out = b.shape[1]
        if tuple(b.shape) != (self.n, self.d_out, self.r):
            raise ValueError(f"b must be [{self.n}, d_out, {self.r}], got {tuple(b.shape)}")
        if scale is not None:
            _expect(scale, _f32, "scale", 1)
            _elsewhere(scale, self._device, "scale")
            if scale.numel() != self.n:
                raise ValueError("scale needs a value for every adapter")
        _lora_bytes(self.n, self.r, self.d_in, self.d_out, 0, 0)      # (refuses the sizes that no call takes)
        self._a, self._b, self._scale = a, b, scale
        self._places = tuple(_place(t, n) for t, n in ((a, "the adapters' a"), (b, "the adapters' b"), (scale, "the adapters' scale")) if t is not None)
        self._lo, self._hi = min(p[0] for p in self._places), max(p[1] for p in self._places)
        self._c = _Lora(a.data_ptr(), b.data_ptr(), _ptr(scale), self.n, self.r, self.d_in, self.d_out)
        self._ref = ctypes.byref(self._c)


def _requests(row_off, adapter, dev):
    """Number of requests of a call's index tensors, which are on GPU `dev`."""
    try:
        ok = (row_off.dtype is adapter.dtype is _i32 and row_off.get_device() == adapter.get_device() == dev
              and row_off.dim() == adapter.dim() == 1 and row_off.is_contiguous() and adapter.is_contiguous())
    except AttributeError:
        ok = False
    if not ok:
        for t, n in ((row_off, "row_off"), (adapter, "adapter")):
            _expect(t, _i32, n, 1)
            _elsewhere(t, dev, n)
    S = adapter.numel()
    if row_off.numel() != S + 1:
        raise ValueError("row_off must have one entry more than adapter")
    return S


def _rows_of(x, d, name, dev, T=None):
    """Row stride in elements of a bf16 matrix [T, d] on GPU `dev` with contiguous rows."""
    if not isinstance(x, torch.Tensor) or x.get_device() != dev:
        if not isinstance(x, torch.Tensor) or not x.is_cuda:
            raise TypeError(f"{name} must be a GPU torch tensor")
        _elsewhere(x, dev, name)
    if x.dtype is not _bf16:
        raise TypeError(f"{name} must be {_bf16}, got {x.dtype}")
    if x.dim() != 2 or x.size(1) != d or (T is not None and x.size(0) != T):
        raise ValueError(f"{name} must be [{'rows' if T is None else T}, {d}], got {tuple(x.shape)}")
    s = x.stride()
    if s[1] != 1 or (s[0] < d and x.size(0) > 1):
        raise ValueError(f"{name}: elements of a row must be contiguous, and rows apart")
    return s[0] if x.size(0) > 1 else d


# A place in memory: from, to, bytes of a row, bytes from one row to the next, name.
def _place(t, name):
    lo, n = t.data_ptr(), t.nbytes
    return lo, lo + n, n, n, name


def _meet(a, b):
    """Whether two places share a byte.  Rows of one buffer may lie between one another; with different strides they are taken to meet."""
    lo, hi, row, step, _ = a
    at, end, other, per, _ = b
    if lo >= end or at >= hi or lo == hi or at == end:
        return False
    if row == hi - lo:                                               # (one row)
        if other == end - at:
            return True
        lo, row, step, at, other = at, other, per, lo, row
    elif other != end - at and step != per:
        return True
    by = (at - lo) % step
    return by < row or by + other > step


def _refuse(out, *others):
    """No byte of an output is one of an input, or of another output."""
    lo, hi = out[0], out[1]
    for x in others:
        if x[0] < hi and lo < x[1] and _meet(out, x):
            raise ValueError(f"{out[4]} overlaps {x[4]}")


def _apart(out, rows, d, stride, name, x, dx, stride_x, other):
    """Refuses an output [rows, d] some of whose elements are those of an input [rows, dx], both in bf16.  (Strides in elements; a row's own length
    where there is one row.)"""
    _refuse(_rows_place(out, rows, d, stride, name), _rows_place(x, rows, dx, stride_x, other))


def _rows_place(x, rows, d, stride, name):
    lo = x.data_ptr()
    return lo, lo + 2 * ((rows - 1) * stride + d) if rows else lo, 2 * d, 2 * stride, name


def lora_forward(x, bank: LoraBank, row_off, adapter, y, keep: bool = False, out_h=None):
    """y[t] += scale (x[t] A^T) B^T in place, with the adapter of the request that row t belongs to: rows row_off[s] .. row_off[s + 1] have
    adapter[s] (int32, both on the GPU); rows of a request whose adapter is not in 0 .. n - 1, and rows of none, stay as they are.
    x [T, d_in], y [T, d_out] in bf16.  Returns h = x A^T, transposed, fp32 [r, T] (with keep, or as out_h; zeros for rows without an
    adapter), for lora_backward, else y."""
    dev = bank._device
    S = _requests(row_off, adapter, dev)
    xs = _rows_of(x, bank.d_in, "x", dev)
    T = x.size(0)
    ys = _rows_of(y, bank.d_out, "y", dev, T)
    if y.requires_grad:
        _recorded(y, "y")
    px, py, po, pa = x.data_ptr(), y.data_ptr(), row_off.data_ptr(), adapter.data_ptr()
    end = py + 2 * ((T - 1) * ys + bank.d_out)
    # (written out: a function for each check costs as much as all of them)
    if out_h is not None or (px < end and py < px + 2 * ((T - 1) * xs + bank.d_in)) or (bank._lo < end and py < bank._hi) or po < end and py < po + 4 * S + 4 \
            or pa < end and py < pa + 4 * S:
        mine = _rows_place(x, T, bank.d_in, xs, "x"), _place(row_off, "row_off"), _place(adapter, "adapter"), *bank._places
        out = _rows_place(y, T, bank.d_out, ys, "y")
        _refuse(out, *mine)
    if out_h is not None:
        _expect(out_h, _f32, "out_h", 2)
        _elsewhere(out_h, dev, "out_h")
        if tuple(out_h.shape) != (bank.r, T):
            raise ValueError(f"out_h must be [{bank.r}, {T}], got {tuple(out_h.shape)}")
        _refuse(_place(out_h, "out_h"), out, *mine)
        if out_h.requires_grad:
            _recorded(out_h, "out_h")
        _changed(out_h)
    elif keep:
        out_h = _new((bank.r, T), (T, 1), dtype=_f32, device=x.device)
    _check(lib.evospec_lora_forward(bank._ref, px, xs, po, pa, S, T, py, ys,
                                    _ptr(out_h), _stream_of(dev)), "evospec_lora_forward")
    _changed(y)
    return y if out_h is None else out_h


def lora_backward_workspace_bytes(bank: LoraBank, S: int, T: int) -> int:
    return _lora_bytes(bank.n, bank.r, bank.d_in, bank.d_out, S, T)


def lora_backward(x, dy, bank: LoraBank, row_off, adapter, h=None, dx=None, out_da=None, out_db=None, workspace=None):
    """The backward pass of lora_forward: (da fp32 [n, r, d_in], db fp32 [n, d_out, r]), the gradients of all adapters (zeros where one
    has no rows).  h is what the forward pass kept, or None: computed again.  dx [T, d_in] (bf16) gets the gradient of x added,
    in place; None: it is not wanted."""
    dev = bank._device
    S = _requests(row_off, adapter, dev)
    xs = _rows_of(x, bank.d_in, "x", dev)
    T = x.size(0)
    gs = _rows_of(dy, bank.d_out, "dy", dev, T)
    ds = 0
    if dx is not None:
        ds = _rows_of(dx, bank.d_in, "dx", dev, T)
        if dx.requires_grad:
            _recorded(dx, "dx")
    if h is not None:
        _expect(h, _f32, "h", 2)
        _elsewhere(h, dev, "h")
        if tuple(h.shape) != (bank.r, T):
            raise ValueError(f"h must be [{bank.r}, {T}], got {tuple(h.shape)}")
    px, pg, po, pa = x.data_ptr(), dy.data_ptr(), row_off.data_ptr(), adapter.data_ptr()
    near = out_da is not None or out_db is not None or workspace is not None
    if dx is not None and not near:
        at = dx.data_ptr()
        end = at + 2 * ((T - 1) * ds + bank.d_in)
        near = (px < end and at < px + 2 * ((T - 1) * xs + bank.d_in)) or (pg < end and at < pg + 2 * ((T - 1) * gs + bank.d_out)) or (bank._lo < end and at < bank._hi) \
            or po < end and at < po + 4 * S + 4 or pa < end and at < pa + 4 * S or h is not None and h.data_ptr() < end and at < h.data_ptr() + 4 * bank.r * T
    if near:
        mine = [_rows_place(x, T, bank.d_in, xs, "x"), _rows_place(dy, T, bank.d_out, gs, "dy"), _place(row_off, "row_off"), _place(adapter, "adapter"), *bank._places]
        if h is not None:
            mine.append(_place(h, "h"))
        if dx is not None:
            out = _rows_place(dx, T, bank.d_in, ds, "dx")
            _refuse(out, *mine)
            mine.append(out)
    if out_da is not None or out_db is not None:
        for t, shape, name in ((out_da, (bank.n, bank.r, bank.d_in), "out_da"), (out_db, (bank.n, bank.d_out, bank.r), "out_db")):
            if t is not None:
                _expect(t, _f32, name, 3)
                _elsewhere(t, dev, name)
                if tuple(t.shape) != shape:
                    raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
                out = _place(t, name)
                _refuse(out, *mine)
                mine.append(out)
                if t.requires_grad:
                    _recorded(t, name)
                _changed(t)
    if workspace is not None:
        workspace = _workspace_of(workspace, 0, dev, None)
        _refuse(_place(workspace, "workspace"), *mine)
    if out_da is None:
        out_da = _new((bank.n, bank.r, bank.d_in), (bank.r * bank.d_in, bank.d_in, 1), dtype=_f32, device=x.device)
    if out_db is None:
        out_db = _new((bank.n, bank.d_out, bank.r), (bank.r * bank.d_out, bank.r, 1), dtype=_f32, device=x.device)
    if workspace is None:
        workspace = _workspace_of(None, _lora_bytes(bank.n, bank.r, bank.d_in, bank.d_out, S, T), dev, x.device)
    _check(lib.evospec_lora_backward(bank._ref, px, xs, _ptr(h), pg, gs, po, pa, S, T,
                                     _ptr(dx), ds, out_da.data_ptr(), out_db.data_ptr(), _ptr(workspace),
                                     0 if workspace is None else workspace.numel(), _stream_of(dev)), "evospec_lora_backward")
    if dx is not None:
        _changed(dx)
    return out_da, out_db


def kd_loss_workspace_bytes(E: int, K: int, d: int) -> int:
    return _kd_bytes(E, K, d)


def kd_loss(h, W_lm, support, target, weight=None, T: float = 1.0, dtype=torch.bfloat16, out_loss=None, out_dh=None, out_draft=None,
            workspace=None):
    """Distillation on the retained support (what kl_gate returns as support and target logits): per event
    weight T^2 KL(softmax(target / T) || softmax(draft / T)), draft = h . W_lm[support].  h bf16 [E, d], W_lm bf16 [V, d], support int32
    [E, K], target fp32 [E, K], weight fp32 [E] or None (1).  Returns (loss fp32 [E], its gradient to h, `dtype` (bf16 or fp32) [E, d],
    draft fp32 [E, K]).  Ids outside 0 .. V - 1 are not in the support."""
    _expect(h, _bf16, "h", 2)
    dev = h.get_device()
    E, d = h.shape
    _expect(W_lm, _bf16, "W_lm", 2)
    _expect(support, _i32, "support", 2)
    _expect(target, _f32, "target", 2)
    for t, name in ((W_lm, "W_lm"), (support, "support"), (target, "target")):
        _elsewhere(t, dev, name)
    K = support.shape[1]
    if W_lm.shape[1] != d or support.shape[0] != E or target.shape != support.shape:
        raise ValueError("h, W_lm, support and target disagree about their sizes")
    if dtype not in (_bf16, _f32):
        raise TypeError(f"dtype must be {_bf16} or {_f32}")
    if weight is not None:
        _expect(weight, _f32, "weight", 1)
        _elsewhere(weight, dev, "weight")
        if weight.numel() != E:
            raise ValueError("weight needs a value for every event")
    if out_loss is not None or out_dh is not None or out_draft is not None or workspace is not None:
        mine = [_place(t, n) for t, n in ((h, "h"), (W_lm, "W_lm"), (support, "support"), (target, "target"), (weight, "weight")) if t is not None]
        for t, kind, shape, name in ((out_loss, _f32, (E,), "out_loss"), (out_dh, dtype, (E, d), "out_dh"), (out_draft, _f32, (E, K), "out_draft")):
            if t is not None:
                _expect(t, kind, name, len(shape))
                _elsewhere(t, dev, name)
                if tuple(t.shape) != shape:
                    raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
                out = _place(t, name)
                _refuse(out, *mine)
                mine.append(out)
                if t.requires_grad:
                    _recorded(t, name)
                _changed(t)
        if workspace is not None:
            workspace = _workspace_of(workspace, 0, dev, None)
            _refuse(_place(workspace, "workspace"), *mine)
    out_loss = _new((E,), (1,), dtype=_f32, device=h.device) if out_loss is None else out_loss
    out_dh = _new((E, d), (d, 1), dtype=dtype, device=h.device) if out_dh is None else out_dh
    out_draft = _new((E, K), (K, 1), dtype=_f32, device=h.device) if out_draft is None else out_draft
    if workspace is None:
        workspace = _workspace_of(None, _kd_bytes(E, K, d), dev, h.device)
    _check(lib.evospec_kd_loss(h.data_ptr(), E, d, W_lm.data_ptr(), W_lm.shape[0], support.data_ptr(), target.data_ptr(), _ptr(weight), K, T,
                               _TYPES[dtype], out_loss.data_ptr(), out_dh.data_ptr(), out_draft.data_ptr(), _ptr(workspace),
                               0 if workspace is None else workspace.numel(), _stream_of(dev)), "evospec_kd_loss")
    return out_loss, out_dh, out_draft


def _refuse_all(written, read):
    """No byte of what is written is another's, among many places without gaps."""
    end = last = 0                                                   # of all places so far, and of those that are written
    by = of = None
    for place, writes in sorted([(p, True) for p in written if p[2]] + [(p, False) for p in read if p[2]], key=lambda x: x[0][0]):
        if place[0] < (end if writes else last):
            raise ValueError(f"{(by if writes else of)[4]} overlaps {place[4]}")
        if place[1] > end:
            end, by = place[1], place
        if writes and place[1] > last:
            last, of = place[1], place


class AdamW:
    """What adamw_step works on: parameters (bf16, fp16 or fp32, contiguous, all of one type), their gradients (that type or fp32; the
    tensors into which every step's gradients are written) and the moments, state "fp32" or "8bit", in flat buffers in which the
    tensors follow one another, each from a multiple of 256 elements on: m and v (fp32, or uint8 codes with scales fp32 [blocks, 2]).
    master: True or a flat fp32 buffer, from which parameters of 16 bits are rounded; True takes the parameters as they are now.
    Buffers that are not given are allocated here, as zeros.  `offsets` says where each tensor begins.  The handle keeps the tensors and their
    addresses: their memory must stay theirs (no `.data = ...`, no `set_`), and what a step writes must not share any with the rest.  A state that was saved is copied
    into m, v, scales and master."""
    params, grads, m, v, scales, master = (_fixed("_" + n) for n in ("params", "grads", "m", "v", "scales", "master"))

    def __init__(self, params, grads, state: str = "fp32", m=None, v=None, scales=None, master=None):
        if state not in _MOMENTS:
            raise ValueError(f"state must be one of {sorted(_MOMENTS)}, got {state!r}")
        params, grads = list(params), list(grads)
        if len(params) != len(grads) or not params:
            raise ValueError("params and grads must be lists of the same length, of one tensor at least")
        kind, gkind, dev = params[0].dtype, grads[0].dtype, params[0].get_device()
        if kind not in _TYPES or gkind not in (kind, _f32):
            raise TypeError("params must be bfloat16, float16 or float32, grads of the same type or float32")
        self.offsets, at = [], 0
        table = (_Tensor * len(params))()
        for i, (p, g) in enumerate(zip(params, grads)):
            _expect(p, kind, f"params[{i}]")
            _expect(g, gkind, f"grads[{i}]")
            _elsewhere(p, dev, f"params[{i}]")
            _elsewhere(g, dev, f"grads[{i}]")
            if p.shape != g.shape:
                raise ValueError(f"params[{i}] and grads[{i}] differ in shape")
            table[i] = _Tensor(p.data_ptr(), g.data_ptr(), p.numel())
            self.offsets.append(at)
            at += -(-p.numel() // ADAMW_BLOCK) * ADAMW_BLOCK
        spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in params if p.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("two of params are the same memory")
        blocks = _ll(0)
        _check(lib.evospec_adamw_blocks(table, len(params), ctypes.byref(blocks)), "evospec_adamw_blocks")
        self.blocks, self.state, self._device = blocks.value, state, dev
        small = state == "8bit"
        dtype = torch.uint8 if small else _f32
        given = {"m": (m, dtype, (at,)), "v": (v, dtype, (at,)), "scales": (scales, _f32, (self.blocks, 2) if small else None),
                 "master": (None if master is True else master, _f32, (at,) if master is not None and master is not False else None)}
        for name, (t, want, shape) in given.items():
            if t is False:
                t = None
            if shape is None:
                if t is not None:
                    raise ValueError(f"{name} does not belong to state {state!r}")
            elif t is None:
                t = torch.zeros(shape, dtype=want, device=params[0].device)
            else:
                _expect(t, want, name, len(shape))
                _elsewhere(t, dev, name)
                if tuple(t.shape) != shape:
                    raise ValueError(f"{name} must be {shape}, got {tuple(t.shape)}")
            setattr(self, "_" + name, t)
        written = [_place(p, f"params[{i}]") for i, p in enumerate(params)] + [
            _place(t, n) for t, n in ((self.m, "m"), (self.v, "v"), (self.scales, "scales"), (self.master, "master")) if t is not None]
        _refuse_all(written, [_place(g, f"grads[{i}]") for i, g in enumerate(grads)])
        if master is True:
            for p, o in zip(params, self.offsets):
                self.master[o:o + p.numel()] = p.detach().reshape(-1)
        self._params, self._grads = tuple(params), tuple(grads)
        self._table, self._types = table, (_TYPES[kind], _TYPES[gkind], _MOMENTS[state])
        self._written = [*params, *(t for t in (self.m, self.v, self.scales, self.master) if t is not None)]
        self._buffers = (self.m.data_ptr(), self.v.data_ptr(), _ptr(self.scales), _ptr(self.master))


def _scalars(t, n, name, dev):
    _expect(t, _f32, name, 1)
    _elsewhere(t, dev, name)
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} elements")
    return t.data_ptr()


def adamw_step(opt: AdamW, lr: float, t: int, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, seed: int = 0,
               schedule=None, grad_scale=None) -> None:
    """Step number t (from 1 on) of AdamW with the gradients as they are in opt.grads.  grad_scale (fp32 [1] on the GPU) multiplies them, and a
    value that is infinite or NaN leaves everything as it is.  schedule (fp32 [2] on the GPU: lr, t) takes the place of the two
    arguments, for a captured graph.  eps: 2^-126 (1.2e-38) or more.  seed: moments of 8 bits are rounded at random, by a hash of seed, t and an element's place."""
    at = None if schedule is None else _scalars(schedule, 2, "schedule", opt._device)
    gs = None if grad_scale is None else _scalars(grad_scale, 1, "grad_scale", opt._device)
    _check(lib.evospec_adamw_step(opt._table, len(opt._params), *opt._types, *opt._buffers, lr, betas[0], betas[1], eps, weight_decay, t,
                                  seed & 0xffffffff, at, gs, _stream_of(opt._device)), "evospec_adamw_step")
    _changed(opt._written)


def adamw_moments(opt: AdamW, dtype=torch.bfloat16, out_m=None, out_v=None):
    """(m, v) as values, flat: of state "8bit" as `dtype` (bf16, which has them exactly, or fp32), of state "fp32" the buffers themselves."""
    if opt.state == "fp32":
        return opt.m, opt.v
    if dtype not in (_bf16, _f32):
        raise TypeError(f"dtype must be {_bf16} or {_f32}")
    n = opt.blocks * ADAMW_BLOCK
    mine = [] if out_m is None and out_v is None else [_place(t, name) for t, name in ((opt.m, "m"), (opt.v, "v"), (opt.scales, "scales"))]
    for t, name in ((out_m, "out_m"), (out_v, "out_v")):
        if t is not None:
            _expect(t, dtype, name, 1)
            _elsewhere(t, opt._device, name)
            if t.numel() != n:
                raise ValueError(f"{name} must have {n} elements")
            out = _place(t, name)
            _refuse(out, *mine)
            mine.append(out)
            if t.requires_grad:
                _recorded(t, name)
            _changed(t)
    out_m = _new((n,), (1,), dtype=dtype, device=opt.m.device) if out_m is None else out_m
    out_v = _new((n,), (1,), dtype=dtype, device=opt.m.device) if out_v is None else out_v
    _check(lib.evospec_adamw_moments(opt._buffers[0], opt._buffers[1], opt._buffers[2], opt.blocks, _TYPES[dtype], out_m.data_ptr(),
                                     out_v.data_ptr(), _stream_of(opt._device)), "evospec_adamw_moments")
    return out_m, out_v
