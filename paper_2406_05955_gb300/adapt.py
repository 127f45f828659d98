"""ctypes binding of libtsffn's operators for adapted layers (low-rank adapters, the activation kept in 8 bits, balance loss,
backward passes): marshalling only. Tensors, outputs and streams as in ``prompt``.

Autograd records none of these calls: their results have no ``grad_fn``, whatever requires a gradient. A caller who wants them
in its graph puts a call and its backward pass into a ``torch.autograd.Function``. What is written over an input by default (the
rows of ``Adapters``) counts as a change in place to autograd, which then refuses a backward pass that needs what was there;
buffers that the caller gives for outputs do not."""
from __future__ import annotations

from functools import lru_cache
from typing import NamedTuple, Optional

import torch
from torch.autograd.graph import increment_version

from .binding import TS_BF16, _check, lib
from .prompt import BLOCK, _CODES, _current_device, _empty, _handle, _ld, _rows_apart, _shaped, _tensor

FEW_ROWS = 512  # rows of a call without a list
_BF16, _F32, _I32, _E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn
_ROWS, _ONLY_BF16 = (_BF16, _F32), (_BF16,)  # types of rows that are added to, and of those that are multiplied


def _like(stream, t: torch.Tensor) -> torch.Tensor:
    """An output like ``t``, which is contiguous, allocated on the stream of the call."""
    return torch.empty_like(t) if stream is None else _empty(stream, *t.shape, dtype=t.dtype)


class AdapterRows(NamedTuple):
    rows: torch.Tensor     # int32 [rows] rows by adapter, those of none behind
    offsets: torch.Tensor  # int32 [adapters + 2] first entry of each adapter


def list_rows(ids: torch.Tensor, groups: int, rows=None, offsets=None, stream=None) -> AdapterRows:
    """``ts_list_rows``: the rows of each of ``groups`` groups by int32 ``ids [rows]``; an id outside them is of none."""
    _tensor(ids, "ids", (_I32,), 1)
    t, dev, groups = ids.shape[0], ids.get_device(), int(groups)
    rows = _like(stream, ids) if rows is None else _shaped(rows, "rows", _I32, (t,), dev)
    offsets = _empty(stream, groups + 2, dtype=_I32) if offsets is None else \
        _shaped(offsets, "offsets", _I32, (groups + 2,), dev)
    _check(lib().ts_list_rows(ids.data_ptr(), t, groups, rows.data_ptr(), offsets.data_ptr(), _handle(stream)),
           "ts_list_rows")
    return AdapterRows(rows, offsets)


def _matrix(t, what: str, dtypes, shape, dev: int) -> int:
    """Elements from a row of ``t`` to the next one; ``t`` checked: on device ``dev`` (the current one), rows apart, of this
    shape (a tuple)."""
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype in dtypes and t.get_device() == dev:
        if t.is_contiguous():
            return shape[1]
        if _rows_apart(t):
            return _ld(t)
    _tensor(t, what, dtypes, 2, rows_apart=True)
    raise ValueError(f"{what} must be {list(shape)}, got {list(t.shape)}")


class Adapters:
    """Low-rank adapters of many requests beside one shared product (``ts_adapt_rows``, ``ts_adapters_backward``): bf16
    ``a [adapters][r][k]`` and ``b [adapters][r][n]`` (rows of ``b`` are what a component adds, as in ``w_down``), fp32
    ``scale [adapters]``, int32 ``ranks [adapters]`` where some have fewer than ``r``. Weights are borrowed; those of one
    adapter may be exchanged between calls. Calls keep nothing: any number may be in flight."""

    def __init__(self, a: torch.Tensor, b: torch.Tensor, scale=None, ranks=None):
        _tensor(a, "a", (_BF16,), 3)
        _tensor(b, "b", (_BF16,), 3)
        if a.shape[:2] != b.shape[:2]:
            raise ValueError("a and b must have as many adapters, of one rank")
        self.adapters, self.r, self.k = a.shape
        self.n = b.shape[2]
        if scale is not None:
            _shaped(scale, "scale", _F32, (self.adapters,), a.get_device())
        if ranks is not None:
            _shaped(ranks, "ranks", _I32, (self.adapters,), a.get_device())
        self.a, self.b, self.scale, self.ranks = a, b, scale, ranks
        self.device = a.get_device()
        self._a, self._b = a.data_ptr(), b.data_ptr()
        self._scale, self._ranks = (None if t is None else t.data_ptr() for t in (scale, ranks))

    def rows(self, ids: torch.Tensor, rows=None, offsets=None, stream=None) -> AdapterRows:
        """The list of ``ids [rows]`` (-1: no adapter) that calls of more than 512 rows and gradients go by; layers whose
        rows are the same can share it."""
        return list_rows(ids, self.adapters, rows=rows, offsets=offsets, stream=stream)

    def _here(self) -> int:
        """The device of the weights, which is the current one."""
        if _current_device() != self.device:
            raise ValueError("the adapters are on another device than the current one")
        return self.device

    def _ids(self, ids, t: int, listed: bool, stream):
        """(pointers of ids, list and offsets, what keeps them alive) for ``t`` rows."""
        if isinstance(ids, AdapterRows):
            _shaped(ids.rows, "rows", _I32, (t,), self.device)
            _shaped(ids.offsets, "offsets", _I32, (self.adapters + 2,), self.device)
        else:
            _shaped(ids, "ids", _I32, (t,), self.device)
            if not listed and t <= FEW_ROWS:
                return ids.data_ptr(), None, None, ids
            ids = self.rows(ids, stream=stream)
        return None, ids.rows.data_ptr(), ids.offsets.data_ptr(), ids

    def forward(self, x: torch.Tensor, y: torch.Tensor, ids, out=None, h=None, stream=None) -> torch.Tensor:
        """``out[t] = y[t] + scale x[t] A^T B`` of the adapter that ``ids`` (int32 ``[rows]``, or what ``rows`` gives) names
        for row ``t``; without ``out`` in ``y`` itself (bf16 or fp32 ``[rows][n]``). x is bf16 ``[rows][k]``. fp32
        ``h [rows][r]``, if given, gets ``scale x[t] A^T``, for ``backward``. What is written shares no memory with x: where y
        is x, ``out`` is needed."""
        dev = self._here()
        t = x.shape[0] if isinstance(x, torch.Tensor) and x.dim() == 2 else -1
        ldx = _matrix(x, "x", _ONLY_BF16, (t, self.k), dev)
        ldo = ldy = _matrix(y, "y", _ROWS, (t, self.n), dev)
        if out is None:
            out = y
        else:
            ldo = _matrix(out, "out", (y.dtype,), (t, self.n), dev)
        if h is not None:
            _shaped(h, "h", _F32, (t, self.r), dev)
        ids, rows, offsets, _keep = self._ids(ids, t, False, stream)
        _check(lib().ts_adapt_rows(x.data_ptr(), ldx, t, self.k, self._a, self._b, self._scale, self._ranks, self.adapters,
                                   self.r, self.n, ids, rows, offsets, y.data_ptr(), ldy, _CODES[y.dtype], out.data_ptr(),
                                   ldo, None if h is None else h.data_ptr(), _handle(stream)), "ts_adapt_rows")
        if out is y:
            increment_version(y)
        return out

    __call__ = forward

    def backward(self, dy: torch.Tensor, dx: Optional[torch.Tensor], ids, h: torch.Tensor, x: torch.Tensor, x_scale=None,
                 out=None, da=None, db=None, accumulate: bool = False, stream=None):
        """(out, da, db): ``out[t] = dx[t] + dh[t] A`` with ``dh[t] = scale dy[t] B^T`` (without ``out`` in ``dx`` itself;
        no ``dx``: None), and the gradients fp32 ``da [adapters][r][k]``, ``db [adapters][r][n]``, overwritten or added to.
        dy is bf16 ``[rows][n]``, h what ``forward`` gave, x its rows: bf16, or e4m3 with ``x_scale`` as ``quant_rows`` keeps
        them. What is written shares no memory with dy, h and x: where dx is dy, ``out`` is needed."""
        dev = self._here()
        t = dy.shape[0] if isinstance(dy, torch.Tensor) and dy.dim() == 2 else -1
        ldy = _matrix(dy, "dy", _ONLY_BF16, (t, self.n), dev)
        _shaped(h, "h", _F32, (t, self.r), dev)
        ldx = _matrix(x, "x", (_BF16, _E4M3), (t, self.k), dev)
        dp = op = None
        ldd = ldo = 0
        code = TS_BF16
        if dx is not None:
            ldo = ldd = _matrix(dx, "dx", _ROWS, (t, self.k), dev)
            op = dp = dx.data_ptr()
            code = _CODES[dx.dtype]
            if out is not None:
                ldo, op = _matrix(out, "out", (dx.dtype,), (t, self.k), dev), out.data_ptr()
        elif out is not None:
            raise ValueError("out needs a dx")
        sp, ld = None, 0
        if (x_scale is not None) != (x.dtype is _E4M3):
            raise ValueError("e4m3 rows need x_scale, and only they have any")
        if x_scale is not None:
            _tensor(x_scale, "x_scale", (_F32,), 2, rows_apart=True)
            if x_scale.shape[0] != -(-self.k // BLOCK) or x_scale.shape[1] < t:
                raise ValueError(f"x_scale must be [{-(-self.k // BLOCK)}][rows]")
            sp, ld = x_scale.data_ptr(), _ld(x_scale)
        if accumulate and (da is None or db is None):
            raise ValueError("da and db are needed to add to")
        da = _empty(stream, *self.a.shape, dtype=_F32) if da is None else _shaped(da, "da", _F32, self.a.shape, dev)
        db = _empty(stream, *self.b.shape, dtype=_F32) if db is None else _shaped(db, "db", _F32, self.b.shape, dev)
        _, rows, offsets, _keep = self._ids(ids, t, True, stream)
        dh = _like(stream, h)
        _check(lib().ts_adapters_backward(
            dy.data_ptr(), ldy, t, self.n, self._a, self._b, self._scale, self._ranks, self.adapters, self.r, self.k, rows,
            offsets, h.data_ptr(), x.data_ptr(), ldx, _CODES[x.dtype], sp, ld, dp, ldd, code, op, ldo, dh.data_ptr(),
            da.data_ptr(), db.data_ptr(), int(bool(accumulate)), _handle(stream)), "ts_adapters_backward")
        if out is None:
            if dx is not None:
                increment_version(dx)
            out = dx
        return out, da, db


def adapt_error(stream=None) -> int:
    """``ts_adapt_get_error``: the status of adapters' calls on the current device, of all streams and threads, since it was last
    asked for."""
    return int(lib().ts_adapt_get_error(_handle(stream)))


def adapt_test_stall(on: bool) -> None:
    """Failure-detection test hook: a bounded wait of the next calls over many rows runs out."""
    lib().ts_adapt_set_test_stall(int(bool(on)))


class Kept(NamedTuple):
    q_gate: torch.Tensor  # e4m3 [rows][m] gate factors, 0 where either factor is not positive
    q_up: torch.Tensor    # e4m3 [rows][m] up factors
    s_gate: torch.Tensor  # fp32 [ceil(m / 128)][rows] their scales
    s_up: torch.Tensor


def _count(n, dev):
    return None if n is None else _shaped(n, "n", _I32, (1,), dev).data_ptr()


def _kept(kept, rows: int, m: int, dev: int):
    """Pointers of what is kept of ``rows`` rows of ``m``, checked."""
    mb = -(-m // BLOCK)
    q_gate, q_up, s_gate, s_up = kept
    return (_shaped(q_gate, "q_gate", _E4M3, (rows, m), dev).data_ptr(), _shaped(q_up, "q_up", _E4M3, (rows, m), dev).data_ptr(),
            _shaped(s_gate, "s_gate", _F32, (mb, rows), dev).data_ptr(), _shaped(s_up, "s_up", _F32, (mb, rows), dev).data_ptr())


def _out(t, what: str, rows: int, m: int, dev: int, stream):
    """(``t``, or a new tensor in its place, and the elements from a row to the next one)."""
    return (_empty(stream, rows, m, dtype=_BF16), m) if t is None else (t, _matrix(t, what, _ONLY_BF16, (rows, m), dev))


def drelu_rows(g: torch.Tensor, u: torch.Tensor, n=None, c=None, keep: bool = False, kept=None, stream=None):
    """``ts_drelu_rows``: bf16 ``c = max(0, g) max(0, u)`` (0 unless both are positive) of the first ``n`` rows (a device
    int32, as ``offsets[-1:]``; all rows without); with ``keep`` (or buffers ``kept`` for it), (c, Kept): what
    ``drelu_rows_backward`` needs, in 8 bits."""
    _tensor(g, "g", _ROWS, 2, rows_apart=True)
    (rows, m), dev = g.shape, g.get_device()
    ldu = _matrix(u, "u", (g.dtype,), (rows, m), dev)
    c, ldc = _out(c, "c", rows, m, dev, stream)
    p = (None,) * 4
    if kept is not None:
        p = _kept(kept, rows, m, dev)
    elif keep:
        mb = -(-m // BLOCK)
        kept = Kept(*(_empty(stream, rows, m, dtype=_E4M3) for _ in range(2)),
                    *(_empty(stream, mb, rows, dtype=_F32) for _ in range(2)))
        p = tuple(t.data_ptr() for t in kept)
    _check(lib().ts_drelu_rows(g.data_ptr(), _ld(g), u.data_ptr(), ldu, _CODES[g.dtype], _count(n, dev), rows, m,
                               c.data_ptr(), ldc, *p, _handle(stream)), "ts_drelu_rows")
    return c if kept is None else (c, kept)


def drelu_rows_backward(dc: torch.Tensor, kept: Kept, n=None, dg=None, du=None, c=None, again: bool = True, stream=None):
    """``ts_drelu_rows_backward``: bf16 (dg, du, c) of ``dc`` and what ``drelu_rows`` kept; c, that of the factors as they
    were kept, is None if ``again`` is false."""
    _tensor(dc, "dc", _ROWS, 2, rows_apart=True)
    (rows, m), dev = dc.shape, dc.get_device()
    p = _kept(kept, rows, m, dev)
    (dg, ldg), (du, ldu) = _out(dg, "dg", rows, m, dev, stream), _out(du, "du", rows, m, dev, stream)
    c, ldc = _out(c, "c", rows, m, dev, stream) if again or c is not None else (None, 0)
    _check(lib().ts_drelu_rows_backward(dc.data_ptr(), _ld(dc), _CODES[dc.dtype], *p, _count(n, dev), rows, m, dg.data_ptr(),
                                        ldg, du.data_ptr(), ldu, None if c is None else c.data_ptr(), ldc,
                                        _handle(stream)), "ts_drelu_rows_backward")
    return dg, du, c


def _columns(t) -> int:
    return t.shape[1] if isinstance(t, torch.Tensor) and t.dim() == 2 else -1


class Balance(NamedTuple):
    loss: torch.Tensor    # fp32 [1]
    counts: torch.Tensor  # int32 [experts] picks of each expert
    share: torch.Tensor   # fp32 [experts] mean probability of each expert
    totals: torch.Tensor  # int32 [2] live tokens, picks


@lru_cache(maxsize=1024)
def _balance_work(tokens: int, experts: int) -> int:
    return lib().ts_balance_work(tokens, experts)


def balance(logits: torch.Tensor, sel: torch.Tensor, loss=None, counts=None, share=None, totals=None, stream=None) -> Balance:
    """``ts_balance``: the loss on uneven routing of fp32 ``logits [tokens][experts]`` whose picks are ``sel``."""
    _tensor(logits, "logits", (_F32,), 2)
    (t, e), dev = logits.shape, logits.get_device()
    _shaped(sel, "sel", _I32, (t, _columns(sel)), dev)
    k = sel.shape[1]
    loss = _empty(stream, 1, dtype=_F32) if loss is None else _shaped(loss, "loss", _F32, (1,), dev)
    counts = _empty(stream, e, dtype=_I32) if counts is None else _shaped(counts, "counts", _I32, (e,), dev)
    share = _empty(stream, e, dtype=_F32) if share is None else _shaped(share, "share", _F32, (e,), dev)
    totals = _empty(stream, 2, dtype=_I32) if totals is None else _shaped(totals, "totals", _I32, (2,), dev)
    size = _balance_work(t, e)
    work = _empty(stream, size, dtype=_F32) if size > 0 else None
    _check(lib().ts_balance(logits.data_ptr(), t, e, sel.data_ptr(), k, loss.data_ptr(), counts.data_ptr(), share.data_ptr(),
                            totals.data_ptr(), None if work is None else work.data_ptr(), _handle(stream)), "ts_balance")
    return Balance(loss, counts, share, totals)


def route_backward(logits: torch.Tensor, sel: torch.Tensor, w: torch.Tensor, dw=None, balance=None, dloss=None, dlogits=None,
                   stream=None) -> torch.Tensor:
    """``ts_route_backward``: fp32 gradient of ``logits`` from that of the routing weights, ``dw``, and from that of the
    balance loss, fp32 ``dloss [1]``, for ``balance`` as it was for these logits and picks."""
    _tensor(logits, "logits", (_F32,), 2)
    (t, e), dev = logits.shape, logits.get_device()
    k = _columns(sel)
    _shaped(sel, "sel", _I32, (t, k), dev)
    _shaped(w, "w", _F32, (t, k), dev)
    if (balance is None) != (dloss is None):
        raise ValueError("balance and dloss come together")
    bp = (None,) * 3
    if balance is not None:
        bp = (_shaped(balance.counts, "counts", _I32, (e,), dev).data_ptr(),
              _shaped(balance.totals, "totals", _I32, (2,), dev).data_ptr(), _shaped(dloss, "dloss", _F32, (1,), dev).data_ptr())
    elif dw is None:
        raise ValueError("dw, or balance and dloss, are needed")
    if dw is not None:
        _shaped(dw, "dw", _F32, (t, k), dev)
    dlogits = _like(stream, logits) if dlogits is None else _shaped(dlogits, "dlogits", _F32, (t, e), dev)
    _check(lib().ts_route_backward(logits.data_ptr(), t, e, sel.data_ptr(), w.data_ptr(), k,
                                   None if dw is None else dw.data_ptr(), *bp, dlogits.data_ptr(), _handle(stream)),
           "ts_route_backward")
    return dlogits


def combine_rows_backward(dy: torch.Tensor, src: torch.Tensor, slots: torch.Tensor, w: torch.Tensor, rows: torch.Tensor,
                          dsrc=None, dw=None, stream=None):
    """``ts_combine_rows_backward``: (dsrc, dw) of ``dy [tokens][n]`` for ``combine_rows(src, slots, w)`` with ``slots`` and
    ``rows`` as ``route`` gives them; rows of ``dsrc`` that no token has are left as they were."""
    _tensor(src, "src", _ROWS, 2)
    _tensor(slots, "slots", (_I32,), 2)
    (t, k), dev, (m, n) = slots.shape, src.get_device(), src.shape
    if _matrix(dy, "dy", _ROWS, (t, n), dev) != n:
        _tensor(dy, "dy", _ROWS, 2)
    _shaped(w, "w", _F32, (t, k), dev)
    _shaped(rows, "rows", _I32, (m,), dev)
    dsrc = _like(stream, src) if dsrc is None else _shaped(dsrc, "dsrc", src.dtype, (m, n), dev)
    dw = _like(stream, w) if dw is None else _shaped(dw, "dw", _F32, (t, k), dev)
    _check(lib().ts_combine_rows_backward(dy.data_ptr(), _CODES[dy.dtype], src.data_ptr(), _CODES[src.dtype], m, n,
                                          slots.data_ptr(), w.data_ptr(), rows.data_ptr(), t, k, dsrc.data_ptr(),
                                          dw.data_ptr(), _handle(stream)), "ts_combine_rows_backward")
    return dsrc, dw
