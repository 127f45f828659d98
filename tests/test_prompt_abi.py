"""The entry points over many tokens reject bad arguments before they touch the device (no GPU needed)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2406_05955_gb300 import binding, build

    build.build()
    return binding.lib()


GOOD = 0x10000


def _array(*v):
    return ctypes.cast((ctypes.c_void_p * len(v))(*v), ctypes.c_void_p)


def test_route_arguments(lib):
    from paper_2406_05955_gb300.binding import TS_ERR_INVALID_ARG as BAD

    g = GOOD
    for args in (
        (g, -1, 8, 2, g, g, g, g, g), (g, 4, 0, 1, g, g, g, g, g), (g, 4, 257, 2, g, g, g, g, g),
        (g, 4, 8, 0, g, g, g, g, g), (g, 4, 8, 9, g, g, g, g, g), (g, 4, 2, 3, g, g, g, g, g),
        (None, 4, 8, 2, g, g, g, g, g), (g, 4, 8, 2, None, g, g, g, g), (g, 4, 8, 2, g, None, g, g, g),
        (g, 4, 8, 2, g, g, None, g, g), (g, 4, 8, 2, g, g, g, None, g), (g, 4, 8, 2, g, g, g, g, None),
        (g, 2 ** 30, 8, 2, g, g, g, g, g),
    ):
        assert lib.ts_route(*args, None) == BAD, args


def test_row_arguments(lib):
    from paper_2406_05955_gb300.binding import TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD, TS_F32, TS_INT4, TS_OK

    g = GOOD
    for call, more in ((lib.ts_gather_rows, ()), (lib.ts_quant_rows, (g,))):
        def rows(x=g, ldx=64, dt=TS_BF16, src=4, k=64, m=4, out=g):
            return call(x, ldx, dt, src, k, None, None, m, out, *more, None)

        for kw in ({"x": None}, {"x": g + 8}, {"out": None}, {"out": g + 2}, {"ldx": 63}, {"ldx": 68}, {"dt": TS_INT4},
                   {"dt": TS_E4M3}, {"dt": 9}, {"src": -1}, {"k": 0}, {"k": 60}, {"m": -1}):
            assert rows(**kw) == BAD, kw
        assert rows(m=0, x=None, out=None) == TS_OK
    assert lib.ts_quant_rows(g, 24, TS_F32, 4, 24, None, None, 4, g, g, None) == BAD  # k not a multiple of 16
    assert lib.ts_quant_rows(g, 64, TS_BF16, 4, 64, None, None, 4, g, None, None) == BAD
    for args in ((g, TS_INT4, 4, 8, g, g, 2, 2, g), (g, TS_F32, -1, 8, g, g, 2, 2, g), (g, TS_F32, 4, 0, g, g, 2, 2, g),
                 (g, TS_F32, 4, 8, g, g, 2, 0, g), (g, TS_F32, 4, 8, g, g, 2, 9, g), (g, TS_F32, 4, 8, g, g, -1, 2, g),
                 (None, TS_F32, 4, 8, g, g, 2, 2, g), (g, TS_F32, 4, 8, None, g, 2, 2, g),
                 (g, TS_F32, 4, 8, g, None, 2, 2, g), (g, TS_F32, 4, 8, g, g, 2, 2, None)):
        assert lib.ts_combine_rows(*args, None) == BAD, args
    assert lib.ts_combine_rows(None, TS_F32, 0, 8, None, None, 0, 2, None, None) == TS_OK


def test_grouped_arguments(lib):
    from paper_2406_05955_gb300.binding import (TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD,
                                                TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32, TS_INT4, TS_KN, TS_NK)

    h = ctypes.c_void_p()
    one, two, none = _array(GOOD), _array(GOOD, GOOD), _array(GOOD, None)

    def create(out=ctypes.byref(h), groups=2, n=64, k=64, dt=TS_BF16, layout=TS_NK, w=two, up=None, s=None, su=None,
               rows=8):
        return lib.ts_grouped_create(out, groups, n, k, dt, layout, w, up, s, su, rows)

    for kw in ({"out": None}, {"groups": 0}, {"groups": 257}, {"n": 0}, {"k": 0}, {"k": 60}, {"w": None}, {"w": none},
               {"up": none}, {"w": _array(GOOD, GOOD + 8)}, {"dt": 9}, {"layout": 2}, {"rows": 0}, {"s": two},
               {"dt": TS_E4M3}, {"dt": TS_E4M3, "s": none}, {"dt": TS_E4M3, "s": two, "up": two},
               {"dt": TS_E4M3, "s": two, "su": two}, {"dt": TS_E4M3, "s": two, "k": 72},
               {"layout": TS_KN, "n": 60}):
        assert create(**kw) == BAD, kw
    for kw in ({"dt": TS_F32}, {"dt": TS_INT4}, {"layout": TS_KN, "up": two}, {"dt": TS_E4M3, "layout": TS_KN, "s": two}):
        assert create(**kw) == UNSUPPORTED, kw
    assert h.value is None and one is not None
    assert lib.ts_grouped_forward(None, GOOD, 64, None, 0, GOOD, 4, GOOD, 64, TS_F32, None) == BAD
    assert lib.ts_grouped_get_error(None, None) == BAD
    assert lib.ts_grouped_check_scratch(None, None) == BAD
    lib.ts_grouped_destroy(None)


def test_other_handles_refuse_8_bit_weights(lib):
    from paper_2406_05955_gb300.binding import TS_E4M3, TS_ERR_INVALID_ARG as BAD

    h = ctypes.c_void_p()
    assert lib.ts_ffn_create(ctypes.byref(h), 256, 32, TS_E4M3, GOOD, GOOD, GOOD, 1) == BAD
    assert lib.ts_moe_create(ctypes.byref(h), 256, 8, 2, TS_E4M3, GOOD, GOOD, 1) == BAD
    assert lib.ts_predictor_create(ctypes.byref(h), 256, 256, 32, TS_E4M3, GOOD, GOOD, 1) == BAD
    assert lib.ts_ffn_forward_noalloc(256, 32, TS_E4M3, GOOD, GOOD, GOOD, GOOD, 1, GOOD, None, None, 0) == BAD


def test_binding_refuses_cpu_tensors():
    import torch

    import paper_2406_05955_gb300 as ts

    w = torch.zeros(8, 64, dtype=torch.bfloat16)
    for call in (lambda: ts.Grouped(w), lambda: ts.route(torch.zeros(4, 8), 2), lambda: ts.quant_rows(w),
                 lambda: ts.gather_rows(w, torch.zeros(2, dtype=torch.int32)),
                 lambda: ts.combine_rows(w, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))):
        with pytest.raises(TypeError):
            call()


def test_experts_and_prompt_arguments(lib):
    from paper_2406_05955_gb300.binding import (TS_BF16, TS_E4M3, TS_ERR_INVALID_ARG as BAD,
                                                TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32, TS_INT4)

    h = ctypes.c_void_p()
    two, none = _array(GOOD, GOOD), _array(GOOD, None)

    def experts(out=ctypes.byref(h), d=64, m=64, e=2, k=1, dt=TS_BF16, r=GOOD, g=two, u=two, dn=two, sg=None, su=None,
                sd=None):
        return lib.ts_experts_create(out, d, m, e, k, dt, r, g, u, dn, sg, su, sd)

    for kw in ({"out": None}, {"d": 0}, {"m": 0}, {"d": 60}, {"m": 60}, {"e": 0}, {"e": 257}, {"k": 0}, {"k": 3}, {"dt": 9},
               {"r": None}, {"r": GOOD + 2}, {"g": None}, {"u": None}, {"dn": None}, {"g": none}, {"u": none},
               {"dn": none}, {"sg": two}, {"sd": two}, {"dt": TS_E4M3}, {"dt": TS_E4M3, "sg": two, "su": two},
               {"dt": TS_E4M3, "sg": two, "su": two, "sd": two, "d": 72}):
        assert experts(**kw) == BAD, kw
    for dt in (TS_F32, TS_INT4):
        assert experts(dt=dt) == UNSUPPORTED

    def prompt(out=ctypes.byref(h), d=64, m=64, e=2, k=1, dt=TS_BF16, t=8):
        return lib.ts_prompt_create(out, d, m, e, k, dt, t)

    for kw in ({"out": None}, {"d": 0}, {"m": 60}, {"e": 0}, {"k": 3}, {"dt": 9}, {"t": 0}, {"t": 2 ** 30}):
        assert prompt(**kw) == BAD, kw
    assert prompt(dt=TS_INT4) == UNSUPPORTED
    assert h.value is None
    assert lib.ts_prompt_forward(None, None, GOOD, 4, GOOD, None) == BAD
    assert lib.ts_prompt_get_routing(None, None, None, None) == BAD
    assert lib.ts_prompt_get_error(None, None) == BAD
    assert lib.ts_prompt_check_scratch(None, None) == BAD
    lib.ts_experts_destroy(None)
    lib.ts_prompt_destroy(None)


def test_sizes_beyond_the_kernels_counts(lib):
    from paper_2406_05955_gb300.binding import TS_BF16, TS_E4M3, TS_ERR_UNSUPPORTED as UNSUPPORTED, TS_F32, TS_KN, TS_NK

    g, h, two = GOOD, ctypes.c_void_p(), _array(GOOD, GOOD)
    for k, m in ((2 ** 24 + 16, 4), (64, 2 ** 30 + 1)):
        assert lib.ts_gather_rows(g, k, TS_BF16, 4, k, None, None, m, g, None) == UNSUPPORTED
        assert lib.ts_quant_rows(g, k, TS_F32, 4, k, None, None, m, g, g, None) == UNSUPPORTED
    for n, t in ((2 ** 30 + 1, 2), (8, 2 ** 30 + 1)):
        assert lib.ts_combine_rows(g, TS_F32, 4, n, g, g, t, 2, g, None) == UNSUPPORTED
    for n, k, rows in ((64, 2 ** 28 + 16, 8), (2 ** 30 + 8, 64, 8), (64, 64, 2 ** 30 + 1)):
        for layout in (TS_NK, TS_KN):
            assert lib.ts_grouped_create(ctypes.byref(h), 2, n, k, TS_BF16, layout, two, None, None, None,
                                         rows) == UNSUPPORTED
        assert lib.ts_grouped_create(ctypes.byref(h), 2, n, k, TS_E4M3, TS_NK, two, two, two, two, rows) == UNSUPPORTED
    for d, m in ((2 ** 24 + 16, 64), (64, 2 ** 24 + 16)):
        assert lib.ts_experts_create(ctypes.byref(h), d, m, 2, 1, TS_BF16, g, two, two, two, None, None,
                                     None) == UNSUPPORTED
        assert lib.ts_prompt_create(ctypes.byref(h), d, m, 2, 1, TS_BF16, 8) == UNSUPPORTED
    assert h.value is None


def test_the_stall_hook_wants_a_handle(lib):
    from paper_2406_05955_gb300.binding import TS_ERR_INVALID_ARG as BAD

    assert lib.ts_grouped_set_test_stall(None, 1) == BAD


def test_sums_by_token_want_whole_elements(lib):
    """Rows that do not start on a boundary of their elements, which no load of an element takes."""
    from paper_2406_05955_gb300.binding import TS_BF16, TS_ERR_INVALID_ARG as BAD, TS_F32

    g = GOOD
    for src, dt in ((g + 1, TS_BF16), (g + 3, TS_BF16), (g + 1, TS_F32), (g + 2, TS_F32), (g + 6, TS_F32)):
        assert lib.ts_combine_rows(src, dt, 4, 8, g, g, 2, 2, g, None) == BAD, (src, dt)
