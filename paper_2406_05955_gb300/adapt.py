"""ctypes binding of libtsffn's operators for adapted layers (low-rank adapters, the activation kept in 8 bits, balance loss,
backward passes): marshalling only. Tensors, outputs and streams as in ``prompt``."""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from .binding import TS_BF16, _check, lib
from .prompt import BLOCK, _CODES, _empty, _handle, _ld, _shaped, _tensor

FEW_ROWS = 64  # rows of a call without a list
_BF16, _F32, _I32, _E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn


class AdapterRows(NamedTuple):
    rows: torch.Tensor     # int32 [rows] rows by adapter, those of none behind
    offsets: torch.Tensor  # int32 [adapters + 2] first entry of each adapter


def list_rows(ids: torch.Tensor, groups: int, rows=None, offsets=None, stream=None) -> AdapterRows:
    """``ts_list_rows``: the rows of each of ``groups`` groups by int32 ``ids [rows]``; an id outside them is of none."""
    _tensor(ids, "ids", (_I32,), 1)
    t, dev, groups = ids.shape[0], ids.get_device(), int(groups)
    rows = _empty(stream, t, dtype=_I32) if rows is None else _shaped(rows, "rows", _I32, (t,), dev)
    offsets = _empty(stream, groups + 2, dtype=_I32) if offsets is None else \
        _shaped(offsets, "offsets", _I32, (groups + 2,), dev)
    _check(lib().ts_list_rows(ids.data_ptr(), t, groups, rows.data_ptr(), offsets.data_ptr(), _handle(stream)),
           "ts_list_rows")
    return AdapterRows(rows, offsets)


def _matrix(t, what: str, dtypes, shape) -> torch.Tensor:
    """``t``, checked: rows apart, of this shape."""
    _tensor(t, what, dtypes, 2, rows_apart=True)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be {list(shape)}, got {list(t.shape)}")
    return t


class Adapters:
    """Low-rank adapters of many requests beside one shared product (``ts_adapt_rows``, ``ts_adapter_grads``): bf16
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

    def rows(self, ids: torch.Tensor, rows=None, offsets=None, stream=None) -> AdapterRows:
        """The list of ``ids [rows]`` (-1: no adapter) that calls of more than 64 rows and gradients go by; layers whose
        rows are the same can share it."""
        return list_rows(ids, self.adapters, rows=rows, offsets=offsets, stream=stream)

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

    def _apply(self, x, a, b, y, ids, out, h, stream):
        """``ts_adapt_rows`` of ``x`` through ``a`` and ``b``: (out, h)."""
        t, k, n = x.shape[0], a.shape[2], b.shape[2]
        ids, rows, offsets, _keep = ids
        if y is not None:
            out = y if out is None else _matrix(out, "out", (y.dtype,), (t, n))
        if h is not None:
            _shaped(h, "h", _F32, (t, self.r), self.device)
        _check(lib().ts_adapt_rows(
            x.data_ptr(), _ld(x), t, k, a.data_ptr(), b.data_ptr(), None if self.scale is None else self.scale.data_ptr(),
            None if self.ranks is None else self.ranks.data_ptr(), self.adapters, self.r, n, ids, rows, offsets,
            None if y is None else y.data_ptr(), 0 if y is None else _ld(y), TS_BF16 if y is None else _CODES[y.dtype],
            None if y is None else out.data_ptr(), 0 if y is None else _ld(out), None if h is None else h.data_ptr(),
            _handle(stream)), "ts_adapt_rows")
        return out

    def forward(self, x: torch.Tensor, y: torch.Tensor, ids, out=None, h=None, stream=None) -> torch.Tensor:
        """``out[t] = y[t] + scale x[t] A^T B`` of the adapter that ``ids`` (int32 ``[rows]``, or what ``rows`` gives) names
        for row ``t``; without ``out`` in ``y`` itself (bf16 or fp32 ``[rows][n]``). x is bf16 ``[rows][k]``. fp32
        ``h [rows][r]``, if given, gets ``scale x[t] A^T``, for ``backward``."""
        _tensor(x, "x", (_BF16,), 2, rows_apart=True)
        t = x.shape[0]
        _matrix(x, "x", (_BF16,), (t, self.k))
        _matrix(y, "y", (_BF16, _F32), (t, self.n))
        return self._apply(x, self.a, self.b, y, self._ids(ids, t, False, stream), out, h, stream)

    __call__ = forward

    def backward(self, dy: torch.Tensor, dx: Optional[torch.Tensor], ids, h: torch.Tensor, x: torch.Tensor, x_scale=None,
                 out=None, da=None, db=None, accumulate: bool = False, stream=None):
        """(out, da, db): ``out[t] = dx[t] + dh[t] A`` with ``dh[t] = scale dy[t] B^T`` (without ``out`` in ``dx`` itself;
        no ``dx``: None), and the gradients fp32 ``da [adapters][r][k]``, ``db [adapters][r][n]``, overwritten or added to.
        dy is bf16 ``[rows][n]``, h what ``forward`` gave, x its rows: bf16, or e4m3 with ``x_scale`` as ``quant_rows`` keeps
        them."""
        _tensor(dy, "dy", (_BF16,), 2, rows_apart=True)
        t = dy.shape[0]
        _matrix(dy, "dy", (_BF16,), (t, self.n))
        _shaped(h, "h", _F32, (t, self.r), self.device)
        _matrix(x, "x", (_BF16, _E4M3), (t, self.k))
        if dx is None:
            if out is not None:
                raise ValueError("out needs a dx")
        else:
            _matrix(dx, "dx", (_BF16, _F32), (t, self.k))
        sp, ld = None, 0
        if (x_scale is not None) != (x.dtype is _E4M3):
            raise ValueError("e4m3 rows need x_scale, and only they have any")
        if x_scale is not None:
            _tensor(x_scale, "x_scale", (_F32,), 2, rows_apart=True)
            if x_scale.shape[0] != -(-self.k // BLOCK) or x_scale.shape[1] < t:
                raise ValueError(f"x_scale must be [{-(-self.k // BLOCK)}][rows]")
            sp, ld = x_scale.data_ptr(), _ld(x_scale)
        grads = []
        for given, what, like in ((da, "da", self.a), (db, "db", self.b)):
            if given is None and accumulate:
                raise ValueError(f"{what} is needed to add to")
            grads.append(_empty(stream, *like.shape, dtype=_F32) if given is None else
                         _shaped(given, what, _F32, tuple(like.shape), self.device))
        listed = self._ids(ids, t, True, stream)
        dh = _empty(stream, t, self.r, dtype=_F32)
        out = self._apply(dy, self.b, self.a, dx, listed, out, dh, stream)
        L, s = lib(), _handle(stream)
        for of, rows, scale, grad in ((dh, x, (sp, ld), grads[0]), (h, dy, (None, 0), grads[1])):
            _check(L.ts_adapter_grads(of.data_ptr(), self.r, rows.data_ptr(), _ld(rows), _CODES[rows.dtype], *scale, t,
                                      rows.shape[1], self.adapters, listed[1], listed[2], grad.data_ptr(),
                                      int(bool(accumulate)), s), "ts_adapter_grads")
        return out, grads[0], grads[1]


def adapt_error(stream=None) -> int:
    """``ts_adapt_get_error``: the status of adapters' calls on the current device since it was last asked for."""
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


def _kept(kept, rows: int, m: int, dev) -> Kept:
    mb = -(-m // BLOCK)
    for name, t in zip(Kept._fields, kept):
        _shaped(t, name, *((_E4M3, (rows, m)) if name[0] == "q" else (_F32, (mb, rows))), dev)
    return kept


def _out(t, what: str, rows: int, m: int, stream) -> torch.Tensor:
    return _empty(stream, rows, m, dtype=_BF16) if t is None else _matrix(t, what, (_BF16,), (rows, m))


def drelu_rows(g: torch.Tensor, u: torch.Tensor, n=None, c=None, keep: bool = False, kept=None, stream=None):
    """``ts_drelu_rows``: bf16 ``c = max(0, g) max(0, u)`` (0 unless both are positive) of the first ``n`` rows (a device
    int32, as ``offsets[-1:]``; all rows without); with ``keep`` (or buffers ``kept`` for it), (c, Kept): what
    ``drelu_rows_backward`` needs, in 8 bits."""
    _tensor(g, "g", (_BF16, _F32), 2, rows_apart=True)
    rows, m = g.shape
    _matrix(u, "u", (g.dtype,), (rows, m))
    c = _out(c, "c", rows, m, stream)
    if kept is not None:
        _kept(kept, rows, m, g.get_device())
    elif keep:
        mb = -(-m // BLOCK)
        kept = Kept(*(_empty(stream, rows, m, dtype=_E4M3) for _ in range(2)),
                    *(_empty(stream, mb, rows, dtype=_F32) for _ in range(2)))
    p = (None,) * 4 if kept is None else tuple(t.data_ptr() for t in kept)
    _check(lib().ts_drelu_rows(g.data_ptr(), _ld(g), u.data_ptr(), _ld(u), _CODES[g.dtype], _count(n, g.get_device()), rows,
                               m, c.data_ptr(), _ld(c), *p, _handle(stream)), "ts_drelu_rows")
    return c if kept is None else (c, kept)


def drelu_rows_backward(dc: torch.Tensor, kept: Kept, n=None, dg=None, du=None, c=None, again: bool = True, stream=None):
    """``ts_drelu_rows_backward``: bf16 (dg, du, c) of ``dc`` and what ``drelu_rows`` kept; c, that of the factors as they
    were kept, is None if ``again`` is false."""
    _tensor(dc, "dc", (_BF16, _F32), 2, rows_apart=True)
    rows, m = dc.shape
    _kept(kept, rows, m, dc.get_device())
    dg, du = _out(dg, "dg", rows, m, stream), _out(du, "du", rows, m, stream)
    c = _out(c, "c", rows, m, stream) if again or c is not None else None
    _check(lib().ts_drelu_rows_backward(dc.data_ptr(), _ld(dc), _CODES[dc.dtype], *(t.data_ptr() for t in kept),
                                        _count(n, dc.get_device()), rows, m, dg.data_ptr(), _ld(dg), du.data_ptr(), _ld(du),
                                        None if c is None else c.data_ptr(), 0 if c is None else _ld(c), _handle(stream)),
           "ts_drelu_rows_backward")
    return dg, du, c


class Balance(NamedTuple):
    loss: torch.Tensor    # fp32 [1]
    counts: torch.Tensor  # int32 [experts] picks of each expert
    share: torch.Tensor   # fp32 [experts] mean probability of each expert
    totals: torch.Tensor  # int32 [2] live tokens, picks


def balance(logits: torch.Tensor, sel: torch.Tensor, loss=None, counts=None, share=None, totals=None, stream=None) -> Balance:
    """``ts_balance``: the loss on uneven routing of fp32 ``logits [tokens][experts]`` whose picks are ``sel``."""
    _tensor(logits, "logits", (_F32,), 2)
    (t, e), dev = logits.shape, logits.get_device()
    _tensor(sel, "sel", (_I32,), 2)
    _shaped(sel, "sel", _I32, (t, sel.shape[1]), dev)
    outs = []
    for v, what, dtype, size in ((loss, "loss", _F32, 1), (counts, "counts", _I32, e), (share, "share", _F32, e),
                                 (totals, "totals", _I32, 2)):
        outs.append(_empty(stream, size, dtype=dtype) if v is None else _shaped(v, what, dtype, (size,), dev))
    work = _empty(stream, max(1, lib().ts_balance_work(t, e)), dtype=_F32)
    _check(lib().ts_balance(logits.data_ptr(), t, e, sel.data_ptr(), sel.shape[1], *(o.data_ptr() for o in outs),
                            work.data_ptr(), _handle(stream)), "ts_balance")
    return Balance(*outs)


def route_backward(logits: torch.Tensor, sel: torch.Tensor, w: torch.Tensor, dw=None, balance=None, dloss=None, dlogits=None,
                   stream=None) -> torch.Tensor:
    """``ts_route_backward``: fp32 gradient of ``logits`` from that of the routing weights, ``dw``, and from that of the
    balance loss, fp32 ``dloss [1]``, for ``balance`` as it was for these logits and picks."""
    _tensor(logits, "logits", (_F32,), 2)
    (t, e), dev = logits.shape, logits.get_device()
    _tensor(sel, "sel", (_I32,), 2)
    k = sel.shape[1]
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
    dlogits = _empty(stream, t, e, dtype=_F32) if dlogits is None else _shaped(dlogits, "dlogits", _F32, (t, e), dev)
    _check(lib().ts_route_backward(logits.data_ptr(), t, e, sel.data_ptr(), w.data_ptr(), k,
                                   None if dw is None else dw.data_ptr(), *bp, dlogits.data_ptr(), _handle(stream)),
           "ts_route_backward")
    return dlogits


def combine_rows_backward(dy: torch.Tensor, src: torch.Tensor, slots: torch.Tensor, w: torch.Tensor, rows: torch.Tensor,
                          dsrc=None, dw=None, stream=None):
    """``ts_combine_rows_backward``: (dsrc, dw) of ``dy [tokens][n]`` for ``combine_rows(src, slots, w)`` with ``slots`` and
    ``rows`` as ``route`` gives them; rows of ``dsrc`` that no token has are left as they were."""
    _tensor(dy, "dy", (_BF16, _F32), 2)
    _tensor(src, "src", (_BF16, _F32), 2)
    _tensor(slots, "slots", (_I32,), 2)
    (t, k), dev, (m, n) = slots.shape, src.get_device(), src.shape
    _shaped(dy, "dy", dy.dtype, (t, n), dev)
    _shaped(w, "w", _F32, (t, k), dev)
    _shaped(rows, "rows", _I32, (m,), dev)
    dsrc = _empty(stream, m, n, dtype=src.dtype) if dsrc is None else _shaped(dsrc, "dsrc", src.dtype, (m, n), dev)
    dw = _empty(stream, t, k, dtype=_F32) if dw is None else _shaped(dw, "dw", _F32, (t, k), dev)
    _check(lib().ts_combine_rows_backward(dy.data_ptr(), _CODES[dy.dtype], src.data_ptr(), _CODES[src.dtype], m, n,
                                          slots.data_ptr(), w.data_ptr(), rows.data_ptr(), t, k, dsrc.data_ptr(),
                                          dw.data_ptr(), _handle(stream)), "ts_combine_rows_backward")
    return dsrc, dw
