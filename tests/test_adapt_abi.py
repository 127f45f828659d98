"""The entry points of adapted layers reject bad arguments before they touch the device (no GPU needed)."""
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2406_05955_gb300 import binding, build

    build.build()
    return binding.lib()


G = 0x10000


def call(fn, defaults, **kw):
    assert set(kw) <= set(defaults), kw
    return fn(*{**defaults, **kw}.values())


def test_list_rows(lib):
    from paper_2406_05955_gb300.binding import TS_ERR_INVALID_ARG as BAD

    good = {"ids": G, "n": 4, "groups": 8, "rows": G, "offsets": G, "stream": None}
    for kw in ({"ids": None}, {"ids": G + 2}, {"n": -1}, {"n": 1 << 30}, {"groups": 0}, {"groups": 256}, {"rows": None},
               {"rows": G + 1}, {"offsets": None}, {"offsets": G + 2}):
        assert call(lib.ts_list_rows, good, **kw) == BAD, kw


def test_adapt_rows(lib):
    from paper_2406_05955_gb300.binding import (TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD,
                                                TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32, TS_INT4, TS_OK)

    good = {"x": G, "ldx": 64, "rows": 4, "k": 64, "a": G, "b": G, "scale": G, "ranks": None, "adapters": 3, "r": 8, "n": 32,
            "ids": G, "list": None, "offsets": None, "y": G, "ldy": 32, "dt": TS_BF16, "out": G, "ldo": 32, "h": None,
            "stream": None}
    for kw in ({"x": None}, {"x": G + 8}, {"ldx": 63}, {"ldx": 68}, {"rows": -1}, {"k": 0}, {"k": 60}, {"a": None},
               {"a": G + 2}, {"b": None}, {"b": G + 8}, {"scale": G + 2}, {"ranks": G + 1}, {"adapters": 0},
               {"adapters": 256}, {"r": 0}, {"r": 129}, {"n": 0}, {"n": 36}, {"ids": None}, {"ids": G + 2},
               {"rows": 513}, {"list": G}, {"list": G + 2, "offsets": G}, {"list": G, "offsets": G + 2}, {"y": None},
               {"y": G + 4}, {"ldy": 31}, {"ldy": 36}, {"dt": TS_INT4}, {"dt": TS_E4M3}, {"dt": 9}, {"out": G + 8},
               {"ldo": 24}, {"ldo": 40}, {"out": None}, {"out": None, "y": None}, {"h": G + 2},
               {"dt": TS_F32, "y": G + 8}):
        assert call(lib.ts_adapt_rows, good, **kw) == BAD, kw
    big = 1 << 24
    for kw in ({"k": big + 8, "ldx": big + 8}, {"n": big + 8, "ldy": big + 8, "ldo": big + 8},
               {"rows": (1 << 30) + 1, "list": G, "offsets": G}):
        assert call(lib.ts_adapt_rows, good, **kw) == UNSUPPORTED, kw
    assert call(lib.ts_adapt_rows, good, rows=0, x=None, y=None, out=None, ids=None) == TS_OK


def test_adapter_grads(lib):
    from paper_2406_05955_gb300.binding import (TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD,
                                                TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32)

    good = {"h": G, "r": 8, "x": G, "ldx": 64, "dt": TS_BF16, "x_scale": None, "ld_scale": 0, "rows": 4, "k": 64,
            "adapters": 3, "list": G, "offsets": G, "grad": G, "accumulate": 0, "stream": None}
    e8 = {"dt": TS_E4M3, "x_scale": G, "ld_scale": 4}
    for kw in ({"h": None}, {"h": G + 1}, {"r": 0}, {"r": 129}, {"x": None}, {"x": G + 8}, {"ldx": 56}, {"ldx": 68},
               {"dt": TS_F32}, {"x_scale": G}, {"rows": -1}, {"k": 0}, {"k": 60}, {"adapters": 0}, {"adapters": 256},
               {"list": None}, {"offsets": None}, {"grad": None}, {"grad": G + 4}, {**e8, "x_scale": None},
               {**e8, "ld_scale": 3}, {**e8, "k": 56}, {**e8, "ldx": 72}):
        assert call(lib.ts_adapter_grads, good, **kw) == BAD, kw
    assert call(lib.ts_adapter_grads, good, k=(1 << 24) + 8, ldx=(1 << 24) + 8) == UNSUPPORTED


def test_adapters_backward(lib):
    from paper_2406_05955_gb300.binding import (TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD,
                                                TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32, TS_INT4)

    good = {"dy": G, "ldy": 32, "rows": 4, "n": 32, "a": G, "b": G, "scale": None, "ranks": None, "adapters": 3, "r": 8, "k": 64,
            "list": G, "offsets": G, "h": G, "x": G, "ldx": 64, "dt": TS_BF16, "x_scale": None, "ld_scale": 0, "dx": G,
            "lddx": 64, "ddt": TS_F32, "out": G, "ldo": 64, "dh": G, "da": G, "db": G, "accumulate": 0, "stream": None}
    e8 = {"dt": TS_E4M3, "x_scale": G, "ld_scale": 4}
    for kw in ({"dy": None}, {"dy": G + 8}, {"ldy": 24}, {"rows": -1}, {"n": 36}, {"a": None}, {"b": G + 2}, {"scale": G + 2},
               {"ranks": G + 1}, {"adapters": 256}, {"r": 129}, {"k": 60}, {"list": None}, {"offsets": None}, {"offsets": G + 2},
               {"h": None}, {"x": None}, {"x": G + 8}, {"ldx": 60}, {"dt": TS_F32}, {"x_scale": G}, {**e8, "x_scale": None},
               {**e8, "ld_scale": 3}, {"dx": None}, {"lddx": 62}, {"ddt": TS_INT4}, {"out": None}, {"ldo": 8}, {"dh": None},
               {"dh": G + 2}, {"da": None}, {"da": G + 4}, {"db": None}, {"db": G + 8}):
        assert call(lib.ts_adapters_backward, good, **kw) == BAD, kw
    assert call(lib.ts_adapters_backward, good, rows=(1 << 30) + 1) == UNSUPPORTED


X, Y, O, H, M = (i << 32 for i in range(1, 6))  # far apart


def test_list_rows_over_its_inputs(lib):
    from paper_2406_05955_gb300.binding import TS_ERR_INVALID_ARG as BAD

    good = {"ids": X, "n": 100, "groups": 8, "rows": Y, "offsets": O, "stream": None}
    for kw in ({"rows": X}, {"rows": X + 396}, {"rows": X - 396}, {"offsets": X + 396}, {"offsets": X - 36}, {"offsets": Y + 4},
               {"rows": O + 36}, {"n": 1, "rows": X},
               # not of memory that is shared
               {"ids": None}, {"ids": X + 2}, {"n": -1}, {"n": 1 << 30}, {"groups": 0}, {"groups": 256}, {"rows": None},
               {"rows": Y + 1}, {"offsets": None}, {"offsets": O + 2}):
        assert call(lib.ts_list_rows, good, **kw) == BAD, kw


def test_adapt_rows_over_its_inputs(lib):
    """out over x, out beside y, h over any of them; the other refusals again, of arguments that share no memory."""
    from paper_2406_05955_gb300.binding import TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD, TS_F32, TS_INT4

    good = {"x": X, "ldx": 64, "rows": 4, "k": 64, "a": M, "b": M, "scale": None, "ranks": None, "adapters": 3, "r": 8, "n": 64,
            "ids": M, "list": None, "offsets": None, "y": Y, "ldy": 64, "dt": TS_BF16, "out": O, "ldo": 64, "h": H,
            "stream": None}
    last = 3 * 128 + 112  # byte of the last 16 of 4 rows of 64 bf16
    wide = {"ldx": 192, "ldy": 192, "ldo": 192}  # (rows 384 bytes apart, of which 128 are used)
    for kw in ({"out": X}, {"y": X, "out": X}, {"out": X + last}, {"out": X - last}, {"out": X, "ldo": 128}, {"rows": 1, "out": X + 112},
               {"out": Y + 128}, {"out": Y - 128}, {"out": Y + 16}, {"out": Y - last}, {"out": Y, "ldo": 128, "ldy": 72},
               {"h": X}, {"h": X + last + 12}, {"h": X - 124}, {"h": Y}, {"h": O + 4}, {"y": O, "h": O},
               {"dt": TS_F32, "out": X - 1008}, {"dt": TS_F32, "out": Y + 1008},
               {**wide, "out": X + 112}, {**wide, "out": X - 112}, {**wide, "out": X + 3 * 384 + 112}, {**wide, "out": X + 384 - 112},
               {**wide, "out": Y - 384 + 112}, {**wide, "out": Y + 2 * 384}, {**wide, "out": X - 3 * 384 - 112},
               # not of memory that is shared
               {"x": None}, {"x": X + 8}, {"ldx": 63}, {"ldx": 68}, {"a": None}, {"a": M + 2}, {"b": None}, {"b": M + 8}, {"scale": M + 2},
               {"ranks": M + 1}, {"ids": None}, {"ids": M + 2}, {"rows": 513}, {"list": M}, {"list": M + 2, "offsets": M},
               {"list": M, "offsets": M + 2}, {"y": None}, {"y": Y + 4}, {"ldy": 56}, {"ldy": 68}, {"dt": TS_INT4}, {"dt": TS_E4M3},
               {"out": O + 8}, {"ldo": 56}, {"y": O, "ldo": 72}, {"out": None}, {"out": None, "y": None, "h": None}, {"h": H + 2},
               {"r": 129}, {"n": 36}, {"k": 60}, {"dt": TS_F32, "y": Y + 8}):
        assert call(lib.ts_adapt_rows, good, **kw) == BAD, kw


def test_adapter_grads_over_their_inputs(lib):
    from paper_2406_05955_gb300.binding import TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD, TS_F32

    good = {"h": H, "r": 8, "x": X, "ldx": 64, "dt": TS_BF16, "x_scale": None, "ld_scale": 0, "rows": 4, "k": 64,
            "adapters": 3, "list": M, "offsets": M, "grad": O, "accumulate": 0, "stream": None}
    e8 = {"dt": TS_E4M3, "x_scale": Y, "ld_scale": 4}
    size = 3 * 8 * 64 * 4
    for kw in ({"grad": H}, {"grad": H + 112}, {"grad": H - size + 16}, {"grad": X + 496}, {"grad": X - size + 16},
               {**e8, "grad": Y}, {**e8, "grad": Y - size + 16}, {**e8, "grad": X + 192},
               # not of memory that is shared
               {"h": None}, {"h": H + 1}, {"r": 0}, {"r": 129}, {"x": None}, {"x": X + 8}, {"ldx": 56}, {"ldx": 68}, {"dt": TS_F32},
               {"x_scale": Y}, {"rows": -1}, {"k": 0}, {"k": 60}, {"adapters": 0}, {"adapters": 256}, {"list": None},
               {"offsets": None}, {"grad": None}, {"grad": O + 4}, {**e8, "x_scale": None}, {**e8, "ld_scale": 3}, {**e8, "k": 56},
               {**e8, "ldx": 72}):
        assert call(lib.ts_adapter_grads, good, **kw) == BAD, kw


def test_adapters_backward_over_its_inputs(lib):
    from paper_2406_05955_gb300.binding import TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD, TS_F32, TS_INT4

    D, E, A, B = (i << 32 for i in range(6, 10))
    good = {"dy": Y, "ldy": 64, "rows": 4, "n": 64, "a": M, "b": M, "scale": None, "ranks": None, "adapters": 3, "r": 8, "k": 64,
            "list": M, "offsets": M, "h": H, "x": X, "ldx": 64, "dt": TS_BF16, "x_scale": None, "ld_scale": 0, "dx": D,
            "lddx": 64, "ddt": TS_BF16, "out": O, "ldo": 64, "dh": E, "da": A, "db": B, "accumulate": 0, "stream": None}
    e8 = {"dt": TS_E4M3, "x_scale": M + (1 << 20), "ld_scale": 4}
    size = 3 * 8 * 64 * 4
    for kw in ({"dx": Y, "out": Y}, {"out": Y + 496}, {"out": Y - 496}, {"out": X}, {"dx": X, "out": X}, {"out": H}, {"out": D + 128},
               {"dh": Y}, {"dh": H}, {"dh": X + 508}, {"dh": D}, {"dh": O + 4}, {"da": Y}, {"da": X - size + 16}, {"da": H + 112},
               {"da": E}, {"da": O}, {"db": Y + 496}, {"db": X}, {"db": H}, {"db": E}, {"db": O - size + 16}, {"db": A + size - 16},
               {"da": B}, {"out": A, "dx": A}, {**e8, "da": M + (1 << 20)}, {**e8, "out": M + (1 << 20)}, {**e8, "dh": M + (1 << 20)},
               {"ddt": TS_F32, "out": X - 1008},
               # not of memory that is shared
               {"dy": None}, {"dy": Y + 8}, {"ldy": 56}, {"rows": -1}, {"n": 36}, {"a": None}, {"b": M + 2}, {"scale": M + 2},
               {"ranks": M + 1}, {"adapters": 256}, {"r": 129}, {"k": 60}, {"list": None}, {"offsets": None}, {"offsets": M + 2},
               {"h": None}, {"x": None}, {"x": X + 8}, {"ldx": 60}, {"dt": TS_F32}, {"x_scale": M}, {**e8, "x_scale": None},
               {**e8, "ld_scale": 3}, {"dx": None}, {"lddx": 62}, {"ddt": TS_INT4}, {"out": None}, {"ldo": 8}, {"dh": None},
               {"dh": E + 2}, {"da": None}, {"da": A + 4}, {"db": None}, {"db": B + 8}):
        assert call(lib.ts_adapters_backward, good, **kw) == BAD, kw


def test_drelu_rows(lib):
    from paper_2406_05955_gb300.binding import (TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD,
                                                TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32, TS_OK)

    good = {"g": G, "ldg": 64, "u": G, "ldu": 64, "dt": TS_BF16, "n": None, "rows": 4, "m": 64, "c": G, "ldc": 64, "qg": G,
            "qu": G, "sg": G, "su": G, "stream": None}
    for kw in ({"g": None}, {"g": G + 8}, {"ldg": 63}, {"ldg": 68}, {"u": None}, {"u": G + 2}, {"ldu": 48}, {"dt": TS_E4M3},
               {"n": G + 2}, {"rows": -1}, {"m": 0}, {"m": 72}, {"c": None}, {"c": G + 4}, {"ldc": 60}, {"qg": None},
               {"qu": None}, {"sg": None}, {"su": None}, {"qg": G + 8}, {"su": G + 2}, {"dt": TS_F32, "g": G + 4}):
        assert call(lib.ts_drelu_rows, good, **kw) == BAD, kw
    assert call(lib.ts_drelu_rows, good, m=(1 << 24) + 16) == UNSUPPORTED
    assert call(lib.ts_drelu_rows, good, rows=0, g=None, c=None) == TS_OK

    good = {"dc": G, "ldd": 64, "dt": TS_F32, "qg": G, "qu": G, "sg": G, "su": G, "n": None, "rows": 4, "m": 64, "dg": G,
            "ldg": 64, "du": G, "ldu": 64, "c": None, "ldc": 0, "stream": None}
    for kw in ({"dc": None}, {"dc": G + 8}, {"ldd": 62}, {"dt": TS_E4M3}, {"qg": None}, {"qu": G + 8}, {"sg": None},
               {"su": G + 1}, {"n": G + 2}, {"rows": -1}, {"m": 8}, {"dg": None}, {"ldg": 60}, {"du": G + 4}, {"ldu": 63},
               {"c": G + 8, "ldc": 64}, {"c": G, "ldc": 56}):
        assert call(lib.ts_drelu_rows_backward, good, **kw) == BAD, kw
    assert call(lib.ts_drelu_rows_backward, good, rows=(1 << 30) + 1) == UNSUPPORTED


def test_balance(lib):
    from paper_2406_05955_gb300.binding import TS_ERR_INVALID_ARG as BAD, TS_OK

    good = {"logits": G, "tokens": 4, "experts": 8, "sel": G, "top_k": 2, "loss": G, "counts": G, "share": G, "totals": G,
            "work": G, "stream": None}
    for kw in ({"logits": None}, {"logits": G + 2}, {"tokens": -1}, {"tokens": 1 << 29}, {"experts": 0}, {"experts": 257},
               {"sel": None}, {"top_k": 0}, {"top_k": 9}, {"experts": 1}, {"loss": None}, {"counts": None}, {"share": None},
               {"totals": None}, {"tokens": 100000, "work": None}, {"work": G + 2}):
        assert call(lib.ts_balance, good, **kw) == BAD, kw
    assert lib.ts_balance_work(-1, 8) == -1 and lib.ts_balance_work(4, 257) == -1
    assert lib.ts_balance_work(0, 1) == 0 and lib.ts_balance_work(1 << 29, 256) > 0

    good = {"logits": G, "tokens": 4, "experts": 8, "sel": G, "w": G, "top_k": 2, "dw": G, "counts": G, "totals": G,
            "dloss": G, "dlogits": G, "stream": None}
    for kw in ({"logits": None}, {"tokens": -1}, {"experts": 300}, {"sel": None}, {"w": None}, {"top_k": 9},
               {"counts": None}, {"totals": None}, {"dloss": None}, {"dlogits": None}, {"dlogits": G + 2}, {"dw": G + 1},
               {"dw": None, "counts": None, "totals": None, "dloss": None}):
        assert call(lib.ts_route_backward, good, **kw) == BAD, kw
    assert call(lib.ts_route_backward, good, tokens=0, dlogits=None) == TS_OK


def test_combine_rows_backward(lib):
    from paper_2406_05955_gb300.binding import (TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD,
                                                TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32, TS_OK)

    good = {"dy": G, "ddt": TS_F32, "src": G, "dt": TS_BF16, "n_rows": 8, "n": 64, "slots": G, "w": G, "rows": G, "tokens": 4,
            "top_k": 2, "dsrc": 2 * G, "dw": G, "stream": None}
    for kw in ({"dy": None}, {"dy": G + 2}, {"ddt": TS_E4M3}, {"src": None}, {"src": G + 1}, {"dt": TS_E4M3}, {"n_rows": -1},
               {"n": 0}, {"slots": None}, {"w": None}, {"rows": None}, {"tokens": -1}, {"top_k": 0}, {"top_k": 9},
               {"dsrc": None}, {"dsrc": G}, {"dw": None}, {"dw": G + 2}):
        assert call(lib.ts_combine_rows_backward, good, **kw) == BAD, kw
    assert call(lib.ts_combine_rows_backward, good, n=(1 << 30) + 1) == UNSUPPORTED
    assert call(lib.ts_combine_rows_backward, good, tokens=0, dy=None, dw=None) == TS_OK


def test_drelu_rows_over_their_inputs(lib):
    from paper_2406_05955_gb300.binding import TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD, TS_F32

    QG, QU, SG, SU = (i << 32 for i in range(10, 14))
    good = {"g": X, "ldg": 256, "u": Y, "ldu": 256, "dt": TS_BF16, "n": None, "rows": 4, "m": 256, "c": O, "ldc": 256, "qg": QG,
            "qu": QU, "sg": SG, "su": SU, "stream": None}
    for kw in ({"c": X + 16}, {"c": X - 16}, {"c": X, "ldc": 512}, {"dt": TS_F32, "c": X}, {"dt": TS_F32, "c": X, "ldc": 512}, {"c": Y + 512},
               {"c": QG}, {"c": SU - 16}, {"qg": X}, {"qu": Y + 2032}, {"qg": QU + 1008}, {"sg": QG + 1020}, {"su": SG + 28}, {"sg": O},
               # not of memory that is shared
               {"g": None}, {"g": X + 8}, {"ldg": 255}, {"ldg": 260}, {"u": None}, {"u": Y + 2}, {"ldu": 240}, {"dt": TS_E4M3},
               {"n": M + 2}, {"rows": -1}, {"m": 0}, {"m": 72}, {"c": None}, {"c": O + 4}, {"ldc": 252}, {"qg": None}, {"qu": None},
               {"sg": None}, {"su": None}, {"qg": QG + 8}, {"su": SU + 2}, {"dt": TS_F32, "g": X + 4}):
        assert call(lib.ts_drelu_rows, good, **kw) == BAD, kw

    good = {"dc": X, "ldd": 256, "dt": TS_BF16, "qg": QG, "qu": QU, "sg": SG, "su": SU, "n": None, "rows": 4, "m": 256, "dg": Y,
            "ldg": 256, "du": O, "ldu": 256, "c": H, "ldc": 256, "stream": None}
    for kw in ({"dg": O}, {"du": H + 2032}, {"c": Y - 2032}, {"dg": X, "du": X}, {"dg": X + 16}, {"du": X, "ldu": 264}, {"dt": TS_F32, "c": X},
               {"dg": QG}, {"du": QU + 1008}, {"c": SG}, {"dg": SU - 2032},
               # not of memory that is shared
               {"dc": None}, {"dc": X + 8}, {"ldd": 252}, {"dt": TS_E4M3}, {"qg": None}, {"qu": QU + 8}, {"sg": None}, {"su": SU + 1},
               {"n": M + 2}, {"rows": -1}, {"m": 8}, {"dg": None}, {"ldg": 252}, {"du": O + 4}, {"ldu": 255}, {"c": H + 8}, {"ldc": 248}):
        assert call(lib.ts_drelu_rows_backward, good, **kw) == BAD, kw


def test_balance_over_its_inputs(lib):
    from paper_2406_05955_gb300.binding import TS_ERR_INVALID_ARG as BAD

    L, C, S, T = (i << 32 for i in range(10, 14))
    good = {"logits": X, "tokens": 4, "experts": 8, "sel": Y, "top_k": 2, "loss": L, "counts": C, "share": S, "totals": T,
            "work": None, "stream": None}
    for kw in ({"loss": X}, {"counts": X + 124}, {"share": X - 28}, {"totals": Y + 28}, {"loss": Y}, {"loss": C}, {"share": C + 4},
               {"totals": S + 28}, {"tokens": 100000, "work": X}, {"tokens": 100000, "work": C},
               # not of memory that is shared
               {"logits": None}, {"logits": X + 2}, {"tokens": -1}, {"tokens": 1 << 29}, {"experts": 0}, {"experts": 257}, {"sel": None},
               {"top_k": 0}, {"top_k": 9}, {"experts": 1}, {"loss": None}, {"counts": None}, {"share": None}, {"totals": None},
               {"tokens": 100000}, {"work": M + 2}):
        assert call(lib.ts_balance, good, **kw) == BAD, kw

    good = {"logits": X, "tokens": 4, "experts": 8, "sel": Y, "w": O, "top_k": 2, "dw": H, "counts": C, "totals": T,
            "dloss": L, "dlogits": S, "stream": None}
    for kw in ({"dlogits": X + 4}, {"dlogits": X - 4}, {"dlogits": Y}, {"dlogits": O + 28}, {"dlogits": H - 124}, {"dlogits": C},
               {"dlogits": T + 4}, {"dlogits": L - 124},
               # not of memory that is shared
               {"logits": None}, {"tokens": -1}, {"experts": 300}, {"sel": None}, {"w": None}, {"top_k": 9}, {"counts": None},
               {"totals": None}, {"dloss": None}, {"dlogits": None}, {"dlogits": S + 2}, {"dw": H + 1},
               {"dw": None, "counts": None, "totals": None, "dloss": None}):
        assert call(lib.ts_route_backward, good, **kw) == BAD, kw


def test_combine_rows_backward_over_its_inputs(lib):
    from paper_2406_05955_gb300.binding import TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD, TS_F32

    good = {"dy": Y, "ddt": TS_F32, "src": X, "dt": TS_BF16, "n_rows": 8, "n": 64, "slots": M, "w": M, "rows": M, "tokens": 4,
            "top_k": 2, "dsrc": O, "dw": H, "stream": None}
    size = 8 * 64 * 2
    for kw in ({"dsrc": X}, {"dsrc": X + size - 2}, {"dsrc": X - size + 2}, {"dsrc": X + 128}, {"dsrc": Y}, {"dsrc": Y + 1022},
               {"dsrc": Y - size + 2}, {"dt": TS_F32, "dsrc": Y}, {"ddt": TS_BF16, "dsrc": Y + 256},
               # not of memory that is shared
               {"dy": None}, {"dy": Y + 2}, {"ddt": TS_E4M3}, {"src": None}, {"src": X + 1}, {"dt": TS_E4M3}, {"n_rows": -1}, {"n": 0},
               {"slots": None}, {"w": None}, {"rows": None}, {"tokens": -1}, {"top_k": 0}, {"top_k": 9}, {"dsrc": None}, {"dw": None},
               {"dw": H + 2}):
        assert call(lib.ts_combine_rows_backward, good, **kw) == BAD, kw


def test_tensors_that_are_not_on_the_gpu_are_refused():
    import torch

    import paper_2406_05955_gb300 as ts

    x, i = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    f, two = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    for fn in (lambda: ts.Adapters(x[None], x[None]), lambda: ts.list_rows(i, 2), lambda: ts.drelu_rows(x, x),
               lambda: ts.drelu_rows_backward(x, ts.Kept(x, x, f, f)), lambda: ts.balance(f, two),
               lambda: ts.route_backward(f, two, f[:, :2], dw=f[:, :2]),
               lambda: ts.combine_rows_backward(f, x, two, f[:, :2], i)):
        with pytest.raises(TypeError):
            fn()
