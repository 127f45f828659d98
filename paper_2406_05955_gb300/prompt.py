"""ctypes binding of libtsffn's operators over many tokens (routed experts, grouped products): marshalling only.

Tensors are CUDA tensors of the current device; others are refused. Outputs that are not given are allocated on
the stream of the call. A call on another stream than the current one is ordered after nothing by itself: the
caller makes that stream wait for the tensors, and keeps them alive until it is done.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import numpy as np
import torch

from .binding import TS_BF16, TS_E4M3, TS_F32, TS_KN, TS_NK, Ffn, Moe, P, _check, lib

_CODES = {torch.float32: TS_F32, torch.bfloat16: TS_BF16, torch.float8_e4m3fn: TS_E4M3}
_LAYOUTS = {"nk": TS_NK, "kn": TS_KN}
BLOCK = 128  # elements of one scale
_CUDA = torch.device("cuda")


_current_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream  # (torch.cuda.current_stream() takes 1-2 us to make its object)


def _refuse(t, what: str, dtypes, dim: int, rows_apart: bool):
    """The error for a tensor that ``_tensor`` does not take."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA tensor")
    if t.get_device() != _current_device():
        raise ValueError(f"{what} is on {t.device}, not on the current device")
    if t.dtype not in dtypes:
        raise TypeError(f"{what} must be one of {[str(d) for d in dtypes]}, got {t.dtype}")
    if t.dim() != dim:
        raise ValueError(f"{what} must have {dim} dimensions")
    raise ValueError(f"{what} must have contiguous rows" if rows_apart else f"{what} must be contiguous")


def _rows_apart(t) -> bool:
    """Whether each row of a matrix is contiguous, and the next one behind it."""
    s0, s1 = t.stride()
    n0, n1 = t.shape
    return (s1 == 1 or n1 <= 1) and (s0 >= n1 or n0 <= 1)


def _tensor(t, what: str, dtypes, dim: int, rows_apart: bool = False) -> torch.Tensor:
    """``t``, checked: on the current device, its type and dimensions, contiguous (or only each row of it)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.get_device() != _current_device() or \
            t.dtype not in dtypes or t.dim() != dim or not (t.is_contiguous() or (rows_apart and _rows_apart(t))):
        _refuse(t, what, dtypes, dim, rows_apart)
    return t


def _shaped(t, what: str, dtype, shape, dev=None) -> torch.Tensor:
    """``t``, checked: on device ``dev`` (the current one), contiguous, of this type and shape."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or \
            t.get_device() != dev:
        _tensor(t, what, (dtype,), len(shape))
        if t.shape != shape:
            raise ValueError(f"{what} must be {list(shape)}, got {list(t.shape)}")
    return t


def _ld(t: torch.Tensor) -> int:
    """Elements from a row to the next one."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _handle(stream) -> int:
    if stream is None:
        return _raw_stream(_current_device())
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else int(stream)


def _empty(stream, *shape, dtype) -> torch.Tensor:
    """An output, allocated on the stream of the call."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=_CUDA)
    with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))):
        return torch.empty(shape, dtype=dtype, device=_CUDA)


class Routing(NamedTuple):
    sel: torch.Tensor      # int32 [tokens][top_k] picked experts, -1: none
    w: torch.Tensor        # fp32 [tokens][top_k] their weights
    offsets: torch.Tensor  # int32 [experts + 1] first row of each expert
    rows: torch.Tensor     # int32 [tokens * top_k] token of each row
    slots: torch.Tensor    # int32 [tokens][top_k] row of each pick, -1: none


def route(logits: torch.Tensor, top_k: int, sel=None, w=None, offsets=None, rows=None, slots=None,
          stream=None) -> Routing:
    """``ts_route``: each token's ``top_k`` experts by fp32 ``logits [tokens][experts]``, and each expert's tokens."""
    _tensor(logits, "logits", (torch.float32,), 2)
    t, e = logits.shape
    k, i32, dev = int(top_k), torch.int32, logits.get_device()
    sel = _empty(stream, t, k, dtype=i32) if sel is None else _shaped(sel, "sel", i32, (t, k), dev)
    w = _empty(stream, t, k, dtype=torch.float32) if w is None else _shaped(w, "w", torch.float32, (t, k), dev)
    offsets = _empty(stream, e + 1, dtype=i32) if offsets is None else _shaped(offsets, "offsets", i32, (e + 1,), dev)
    rows = _empty(stream, t * k, dtype=i32) if rows is None else _shaped(rows, "rows", i32, (t * k,), dev)
    slots = _empty(stream, t, k, dtype=i32) if slots is None else _shaped(slots, "slots", i32, (t, k), dev)
    _check(lib().ts_route(logits.data_ptr(), t, e, k, sel.data_ptr(), w.data_ptr(), offsets.data_ptr(),
                          rows.data_ptr(), slots.data_ptr(), _handle(stream)), "ts_route")
    return Routing(sel, w, offsets, rows, slots)


def _row_list(x, rows, n, max_rows):
    """(pointer of the list, pointer of the count, rows of the output)."""
    rp = np_ = None
    if rows is not None:
        _tensor(rows, "rows", (torch.int32,), 1)
        rp, m = rows.data_ptr(), rows.shape[0]
    else:
        m = x.shape[0]
    if max_rows is not None and max_rows != m:
        raise ValueError(f"the output must have {m} rows")
    if n is not None:
        _tensor(n, "n", (torch.int32,), 1)
        if n.shape[0] != 1:
            raise ValueError("n must have one element")
        np_ = n.data_ptr()
    return rp, np_, m


def gather_rows(x: torch.Tensor, rows: torch.Tensor, n=None, out=None, stream=None) -> torch.Tensor:
    """``ts_gather_rows``: ``out[r] = x[rows[r]]`` for ``r < n`` (a device int32, as ``offsets[-1:]``; all rows
    without); the other rows of ``out`` are left as they were."""
    _tensor(x, "x", (torch.bfloat16, torch.float32), 2, rows_apart=True)
    rp, np_, m = _row_list(x, rows, n, None if out is None else out.shape[0])
    out = _empty(stream, m, x.shape[1], dtype=x.dtype) if out is None else \
        _shaped(out, "out", x.dtype, (m, x.shape[1]), x.get_device())
    _check(lib().ts_gather_rows(x.data_ptr(), _ld(x), _CODES[x.dtype], x.shape[0], x.shape[1], rp, np_, m,
                                out.data_ptr(), _handle(stream)), "ts_gather_rows")
    return out


def quant_rows(x: torch.Tensor, rows=None, n=None, q=None, scale=None, stream=None):
    """``ts_quant_rows``: (q e4m3 [rows][k], scale fp32 [ceil(k / 128)][rows]) of the rows of ``x`` that are listed
    (all of them without a list)."""
    _tensor(x, "x", (torch.bfloat16, torch.float32), 2, rows_apart=True)
    k = x.shape[1]
    rp, np_, m = _row_list(x, rows, n, None if q is None else q.shape[0])
    kb, dev, f8 = -(-k // BLOCK), x.get_device(), torch.float8_e4m3fn
    q = _empty(stream, m, k, dtype=f8) if q is None else _shaped(q, "q", f8, (m, k), dev)
    scale = _empty(stream, kb, m, dtype=torch.float32) if scale is None else \
        _shaped(scale, "scale", torch.float32, (kb, m), dev)
    _check(lib().ts_quant_rows(x.data_ptr(), _ld(x), _CODES[x.dtype], x.shape[0], k, rp, np_, m, q.data_ptr(),
                               scale.data_ptr(), _handle(stream)), "ts_quant_rows")
    return q, scale


def combine_rows(src: torch.Tensor, slots: torch.Tensor, w: torch.Tensor, out=None, stream=None) -> torch.Tensor:
    """``ts_combine_rows``: fp32 ``out[t] = sum_j w[t][j] src[slots[t][j]]``; a slot outside ``src`` adds nothing."""
    _tensor(src, "src", (torch.bfloat16, torch.float32), 2)
    _tensor(slots, "slots", (torch.int32,), 2)
    (t, k), dev = slots.shape, src.get_device()
    _shaped(w, "w", torch.float32, (t, k), dev)
    out = _empty(stream, t, src.shape[1], dtype=torch.float32) if out is None else \
        _shaped(out, "out", torch.float32, (t, src.shape[1]), dev)
    _check(lib().ts_combine_rows(src.data_ptr(), _CODES[src.dtype], src.shape[0], src.shape[1], slots.data_ptr(),
                                 w.data_ptr(), t, k, out.data_ptr(), _handle(stream)), "ts_combine_rows")
    return out


def _matrices(t) -> list:
    """A matrix, a list of them, or a stacked tensor, as a list."""
    if isinstance(t, torch.Tensor):
        t = [t] if t.dim() == 2 else list(t.unbind(0)) if t.dim() == 3 else []
    t = list(t)
    if not t:
        raise ValueError("weights are a matrix, a list of them, or a stacked tensor")
    return t


def _pointers(ts):
    if ts is None:
        return None
    return ctypes.cast((ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts]), ctypes.c_void_p)


class Grouped:
    """Products of ragged groups of rows, each group with its own weights (``ts_grouped_*``): ``y[r] = x[r] W_e^T``
    over borrowed ``w[e] [n][k]`` (``layout="kn"``: ``x[r] W_e`` over ``[k][n]``), bf16, or e4m3 with fp32
    ``scale[e] [ceil(n / 128)][ceil(k / 128)]``. ``w`` is a tensor (one group), a list of them, or a stacked one.
    One forward may be in flight at a time, replays of graphs that hold one included."""

    def __init__(self, w, layout: str = "nk", scale=None, max_rows: int = 1, _up=None, _scale_up=None):
        w, up, scale, scale_up = (None if t is None else _matrices(t) for t in (w, _up, scale, _scale_up))
        if layout not in _LAYOUTS:
            raise ValueError('layout must be "nk" or "kn"')
        for t in w + (up or []):
            _tensor(t, "w", (torch.bfloat16, torch.float8_e4m3fn), 2)
            if t.shape != w[0].shape or t.dtype != w[0].dtype:
                raise ValueError("the groups' weights must share one shape and type")
        if up is not None and len(up) != len(w):
            raise ValueError("as many w_up as w_gate are needed")
        self.groups, self.dtype, self.max_rows = len(w), w[0].dtype, int(max_rows)
        self.n, self.k = (int(v) for v in (w[0].shape if layout == "nk" else w[0].shape[::-1]))
        e8 = self.dtype == torch.float8_e4m3fn
        for s, of in ((scale, w), (scale_up, up)):
            if (s is not None) != (e8 and of is not None):
                raise ValueError("e4m3 weights need scales, and only they have any")
            if s is not None and len(s) != len(of):
                raise ValueError("as many scales as weights are needed")
            for t in s or []:
                _shaped(t, "scale", torch.float32, (-(-self.n // BLOCK), -(-self.k // BLOCK)))
        self._keep = (w, up, scale, scale_up)
        h = ctypes.c_void_p()
        self._h = None
        _check(lib().ts_grouped_create(ctypes.byref(h), self.groups, self.n, self.k, _CODES[self.dtype],
                                       _LAYOUTS[layout], _pointers(w), _pointers(up), _pointers(scale),
                                       _pointers(scale_up), self.max_rows), "ts_grouped_create")
        self._h = h

    @classmethod
    def gated(cls, w_gate, w_up, scale_gate=None, scale_up=None, max_rows: int = 1) -> "Grouped":
        """``y[r] = max(0, x[r] G_e^T) * max(0, x[r] U_e^T)``: the dReLU products of Eq. 2."""
        return cls(w_gate, scale=scale_gate, max_rows=max_rows, _up=w_up, _scale_up=scale_up)

    @property
    def handle(self) -> ctypes.c_void_p:
        if self._h is None:
            raise RuntimeError("handle is closed")
        return self._h

    def forward(self, x: torch.Tensor, offsets=None, x_scale=None, y=None, stream=None) -> torch.Tensor:
        """``y`` (bf16 or fp32, bf16 without one) of the groups of rows ``offsets[e] .. offsets[e + 1] - 1`` of ``x``;
        rows that no group has are left as they were. e4m3 rows come with ``x_scale``, as ``quant_rows`` gives it."""
        _tensor(x, "x", (self.dtype,), 2, rows_apart=True)
        rows = x.shape[0]
        if x.shape[1] != self.k:
            raise ValueError(f"x must be [rows][{self.k}]")
        op = sp = None
        if offsets is not None:
            op = _shaped(offsets, "offsets", torch.int32, (self.groups + 1,), x.get_device()).data_ptr()
        ld = 0
        if x_scale is not None:
            _tensor(x_scale, "x_scale", (torch.float32,), 2, rows_apart=True)
            if x_scale.shape[0] != -(-self.k // BLOCK) or x_scale.shape[1] < rows:
                raise ValueError(f"x_scale must be [{-(-self.k // BLOCK)}][rows]")
            sp, ld = x_scale.data_ptr(), _ld(x_scale)
        if y is None:
            y = _empty(stream, rows, self.n, dtype=torch.bfloat16)
        else:
            _tensor(y, "y", (torch.bfloat16, torch.float32), 2, rows_apart=True)
            if tuple(y.shape) != (rows, self.n):
                raise ValueError(f"y must be [{rows}][{self.n}]")
        _check(lib().ts_grouped_forward(self.handle, x.data_ptr(), _ld(x), sp, ld, op, rows, y.data_ptr(), _ld(y),
                                        _CODES[y.dtype], _handle(stream)), "ts_grouped_forward")
        return y

    __call__ = forward

    def get_error(self, stream=None) -> int:
        return int(lib().ts_grouped_get_error(self.handle, _handle(stream)))

    def check_scratch(self, stream=None) -> int:
        """Status of the scratch guard zones (as Ffn.check_scratch)."""
        return int(lib().ts_grouped_check_scratch(self.handle, _handle(stream)))

    def set_test_stall(self, on: bool) -> None:
        """Failure-detection test hook: the next forwards' bounded waits run out."""
        _check(lib().ts_grouped_set_test_stall(self.handle, int(bool(on))), "ts_grouped_set_test_stall")

    def close(self) -> None:
        if getattr(self, "_h", None) is not None:
            lib().ts_grouped_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Experts:
    """The weights of one layer over many tokens: ``top_k`` of the dReLU FFNs ``w_gate[e], w_up[e] [m][d]`` and
    ``w_down[e]`` (bf16: ``[m][d]``, by neuron, as in ``Ffn``; e4m3: ``[d][m]``, with three lists of scales as in
    ``Grouped``), picked by ``w_router [experts][d]`` (bf16), or a single one without it. Weights are borrowed."""

    def __init__(self, w_gate, w_up, w_down, w_router=None, top_k: int = 1, scale_gate=None, scale_up=None,
                 scale_down=None):
        ws = [_matrices(t) for t in (w_gate, w_up, w_down)]
        for t in ws[0] + ws[1] + ws[2]:
            _tensor(t, "weights", (torch.bfloat16, torch.float8_e4m3fn), 2)
        self.dtype, self.n_experts, self.top_k = ws[0][0].dtype, len(ws[0]), int(top_k)
        self.m, self.d = (int(v) for v in ws[0][0].shape)
        e8 = self.dtype == torch.float8_e4m3fn
        down = (self.d, self.m) if e8 else (self.m, self.d)
        for w, shape in zip(ws, ((self.m, self.d), (self.m, self.d), down)):
            if len(w) != self.n_experts or any(tuple(t.shape) != shape or t.dtype != self.dtype for t in w):
                raise ValueError(f"w_gate and w_up must be [{self.m}][{self.d}], w_down {list(down)}, as many of each")
        scales = [None if t is None else _matrices(t) for t in (scale_gate, scale_up, scale_down)]
        for s, w in zip(scales, ws):
            if (s is not None) != e8 or (e8 and len(s) != self.n_experts):
                raise ValueError("e4m3 weights need scales, and only they have any")
            for t in s or []:
                _shaped(t, "scale", torch.float32, tuple(-(-v // BLOCK) for v in w[0].shape))
        if w_router is not None:
            _shaped(w_router, "w_router", torch.bfloat16, (self.n_experts, self.d))
        self.routed = w_router is not None
        self._keep = (ws, scales, w_router)
        h = ctypes.c_void_p()
        self._h = None
        _check(lib().ts_experts_create(ctypes.byref(h), self.d, self.m, self.n_experts, self.top_k, _CODES[self.dtype],
                                       None if w_router is None else w_router.data_ptr(), *map(_pointers, ws),
                                       *map(_pointers, scales)), "ts_experts_create")
        self._h = h

    @classmethod
    def of(cls, layer) -> "Experts":
        """The same weights as a bf16 ``Ffn`` or ``Moe`` layer."""
        if isinstance(layer, Moe):
            ws = list(zip(*(e._keep for e in layer.experts)))
            return cls(*map(list, ws), w_router=layer._keep[0], top_k=layer.top_k)
        if isinstance(layer, Ffn):
            return cls(*layer._keep)
        raise TypeError("layer must be an Ffn or a Moe")

    @property
    def handle(self) -> ctypes.c_void_p:
        if self._h is None:
            raise RuntimeError("handle is closed")
        return self._h

    def close(self) -> None:
        if getattr(self, "_h", None) is not None:
            lib().ts_experts_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Prompt:
    """Forwards of up to ``max_tokens`` tokens through ``experts``, or through any other layer of its sizes: the scratch
    of all of them (``ts_prompt_*``). One forward may be in flight at a time, replays of graphs that hold one included."""

    def __init__(self, experts: Experts, max_tokens: int):
        self.experts, self.max_tokens, self._most = experts, int(max_tokens), int(max_tokens) * experts.top_k
        h = ctypes.c_void_p()
        self._h = None
        _check(lib().ts_prompt_create(ctypes.byref(h), experts.d, experts.m, experts.n_experts, experts.top_k,
                                      _CODES[experts.dtype], self.max_tokens), "ts_prompt_create")
        self._h = h
        self._last = None

    @property
    def handle(self) -> ctypes.c_void_p:
        if self._h is None:
            raise RuntimeError("handle is closed")
        return self._h

    def forward(self, x: torch.Tensor, experts=None, y=None, stream=None) -> torch.Tensor:
        """fp32 ``y [tokens][d]`` of bf16 ``x [tokens][d]``, as ``Moe.forward`` (or ``Ffn.forward``) of few tokens."""
        layer = self.experts if experts is None else experts
        _tensor(x, "x", (torch.bfloat16,), 2)
        if x.shape[1] != layer.d:
            raise ValueError(f"x must be [tokens][{layer.d}]")
        t = x.shape[0]
        y = _empty(stream, t, layer.d, dtype=torch.float32) if y is None else \
            _shaped(y, "y", torch.float32, (t, layer.d), x.get_device())
        _check(lib().ts_prompt_forward(self.handle, layer.handle, x.data_ptr(), t, y.data_ptr(), _handle(stream)),
               "ts_prompt_forward")
        self._last = (t, layer.top_k)
        return y

    __call__ = forward

    def get_routing(self, stream=None):
        """(sel, w) of the last forward, as numpy [tokens][top_k]; -1: no expert."""
        sel, w = np.zeros(self._most, np.int32), np.zeros(self._most, np.float32)  # room for any forward's
        _check(lib().ts_prompt_get_routing(self.handle, _handle(stream), sel.ctypes.data_as(P), w.ctypes.data_as(P)),
               "ts_prompt_get_routing")
        t, k = self._last
        return sel[:t * k].reshape(t, k), w[:t * k].reshape(t, k)

    def get_error(self, stream=None) -> int:
        return int(lib().ts_prompt_get_error(self.handle, _handle(stream)))

    def check_scratch(self, stream=None) -> int:
        """Status of the scratch guard zones (as Ffn.check_scratch)."""
        return int(lib().ts_prompt_check_scratch(self.handle, _handle(stream)))

    def close(self) -> None:
        if getattr(self, "_h", None) is not None:
            lib().ts_prompt_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
