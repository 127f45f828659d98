"""Products of ragged groups of rows (ts_grouped_*) against their formulas in 64 bits.

Tolerance, per output, derived from the arithmetic: inputs are exact, products of two bf16 or two e4m3 numbers are
exact in fp32, and a sum of k of them in fp32 (in any order, each addition off by at most 2^-23 of the magnitude it
has reached, whether rounded or truncated) is off by at most about k 2^-23 of S = sum |x_i w_i|; blocks that the tensor
cores sum at once take one addition each, so k 2^-24 S is allowed, and 2^-20 S for the scales and short sums. A gated
output g u carries each factor's error times the other factor, and an output rounded to bf16 half a step, 2^-8 of it.
On top of it the relative 2-norm error of fp32 outputs is at most 1e-5, as for every fp32 sum of this library.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
REL_F32 = 1e-5


@pytest.fixture(scope="module")
def ts():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    import paper_2406_05955_gb300 as ts

    ts.lib()
    return ts


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def make(dtype, e, n, k, rows, gated, layout="nk", seed=0):
    """x, x_scale, weights, scales (lists per factor), and x and the weights in 64 bits."""
    g = gen(seed)
    x = randn(g, rows, k)
    two = 2 if gated else 1
    shape = (n, k) if layout == "nk" else (k, n)
    w = [[randn(g, *shape) / math.sqrt(k) for _ in range(e)] for _ in range(two)]
    if dtype == BF16:
        x = x.to(BF16)
        w = [[m.to(BF16) for m in ws] for ws in w]
        return x, None, w, [None, None], x.double(), [[m.double() for m in ws] for ws in w]
    kb, nb = -(-k // 128), -(-n // 128)
    xs = torch.exp(randn(g, kb, rows))
    ss = [[torch.exp(0.5 * randn(g, nb, kb)) for _ in range(e)] for _ in range(two)]
    x = x.to(E4M3)
    w = [[m.to(E4M3) for m in ws] for ws in w]
    xd = x.double() * xs.double().repeat_interleave(128, 0)[:k].t()
    wd = [[m.double() * s.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
           for m, s in zip(ws, sc)] for ws, sc in zip(w, ss)]
    return x, xs, w, ss + [None] * (2 - two), xd, wd


def handle(ts, w, ss, gated, layout, max_rows):
    if gated:
        return ts.Grouped.gated(w[0], w[1], scale_gate=ss[0], scale_up=ss[1], max_rows=max_rows)
    return ts.Grouped(w[0], layout=layout, scale=ss[0], max_rows=max_rows)


def check(y, before, off, xd, wd, gated, layout, k):
    """Every group's rows within the bound, every other row as it was."""
    untouched = torch.ones(y.shape[0], dtype=torch.bool, device="cuda")
    eps = k * 2.0 ** -24 + 2.0 ** -20
    num = den = 0.0
    for e in range(len(off) - 1):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        untouched[a:b] = False
        ws = [w[e] if layout == "kn" else w[e].t() for w in wd]
        p = [xd[a:b] @ w for w in ws]
        err = [eps * (xd[a:b].abs() @ w.abs()) for w in ws]
        if gated:
            want = p[0].clamp(min=0) * p[1].clamp(min=0)
            tol = err[0] * p[1].abs() + err[1] * p[0].abs() + err[0] * err[1]
        else:
            want, tol = p[0], err[0]
        if y.dtype == BF16:
            tol = tol + 2.0 ** -8 * (want.abs() + tol)
        got = y[a:b].double()
        off_by = (got - want).abs()
        assert torch.isfinite(got).all()
        assert (off_by <= tol + 1e-37).all(), f"group {e}: {float((off_by - tol).max()):.3e} over the bound"
        num += float(off_by.square().sum())
        den += float(want.square().sum())
    assert torch.equal(y[untouched], before[untouched]), "a row of no group was written"
    if y.dtype == F32 and den > 0:
        assert math.sqrt(num / den) <= REL_F32


def run(ts, dtype, sizes, n, k, gated=False, layout="nk", out=F32, extra=0, seed=0, pad_x=0, pad_y=0):
    off = [0]
    for s in sizes:
        off.append(off[-1] + s)
    rows = off[-1] + extra
    x, xs, w, ss, xd, wd = make(dtype, len(sizes), n, k, rows, gated, layout, seed)
    if pad_x:  # rows further apart than k
        wide = torch.full((rows, k + pad_x), float("nan"), device="cuda").to(x.dtype)
        wide[:, :k] = x
        x = wide[:, :k]
    y = randn(gen(seed + 1), rows, n + pad_y).to(out)
    before = y.clone()
    mm = handle(ts, w, ss, gated, layout, rows)
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    got = mm.forward(x, offsets=offsets, x_scale=xs, y=y[:, :n])
    assert mm.get_error() == 0 and mm.check_scratch() == 0
    check(got, before[:, :n], off, xd, wd, gated, layout, k)
    assert torch.equal(y[:, n:], before[:, n:])
    return mm


# a single row, sizes around the tiles' edges, empty groups at the ends and in between, rows of no group behind
RAGGED = [
    ([1], 0),
    ([0, 0, 1, 0], 3),
    ([7, 0, 16, 17], 0),
    ([15, 1, 31, 33, 64], 5),
    ([0, 127, 128, 129, 0, 2], 9),
    ([255, 256, 257], 1),
    ([520, 3, 700], 40),
]
# (dtype, gated, layout)
FORMS = [(BF16, False, "nk"), (BF16, False, "kn"), (BF16, True, "nk"), (E4M3, False, "nk"), (E4M3, True, "nk")]
IDS = ["bf16", "bf16-kn", "bf16-gated", "e4m3", "e4m3-gated"]


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("sizes,extra", RAGGED)
def test_ragged_groups(ts, form, sizes, extra):
    dtype, gated, layout = form
    run(ts, dtype, sizes, 384, 512, gated, layout, F32, extra, seed=len(sizes))


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("out", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(8, 16), (64, 64), (136, 80), (1000, 144), (200, 1040), (129 * 8, 2064)])
def test_odd_sizes(ts, form, out, n, k):
    dtype, gated, layout = form
    run(ts, dtype, [5, 0, 90], n, k, gated, layout, out, 2, seed=n + k)


@pytest.mark.parametrize("form", [f for f in FORMS if f[2] == "nk"], ids=[i for i in IDS if "kn" not in i])
@pytest.mark.parametrize("n", [1, 3, 127, 257])
def test_any_number_of_outputs(ts, form, n):
    dtype, gated, layout = form
    run(ts, dtype, [3, 20], n, 256, gated, layout, BF16, 0, seed=n)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_strided_rows(ts, form):
    dtype, gated, layout = form
    run(ts, dtype, [30, 100], 160, 192, gated, layout, F32, 1, seed=5, pad_x=16, pad_y=3)
    run(ts, dtype, [30, 100], 160, 192, gated, layout, BF16, 1, seed=6, pad_x=32, pad_y=5)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("rows", [1, 9, 40, 300])
def test_layer_sizes(ts, form, rows):
    """d = 4096, m = 14336, over two experts."""
    dtype, gated, layout = form
    n, k = (4096, 14336) if layout == "kn" else (14336, 4096)
    run(ts, dtype, [rows, rows // 2], n, k, gated, layout, F32, 0, seed=rows)


@pytest.mark.parametrize("rows", [40, 700])
@pytest.mark.parametrize("n,k", [(1024, 4096), (520, 14336)])
@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_fp32_outputs_are_as_exact_as_sums_in_fp32(ts, form, n, k, rows):
    """2-norm of the error of Gaussian sums. The tensor cores truncate at 2^-24 of the power of two below a sum: half of that
    on average, 2.15e-8 of the sum (a mantissa's mean square reciprocal is 0.72^2), at each of 16 steps of 16 of k, during which
    the sum is 0.69 of its last size on average: 2.4e-7, all toward 0. An addition of k / 256 such sums in fp32 rounds
    at random, 2^-24 / sqrt 3 times 0.74 of a sum that grows with its root: 2.5e-8 sqrt(k / 512), 1.34e-7 at the most. Together
    (2.4^2 + 1.34^2)^(1/2) = 2.8e-7. e4m3: 4 steps of 32 of k are truncated, 0.6e-7, there are k / 128 additions, 1.9e-7 at the
    most, and a rounded product of two scales each, which k / 128 of them average out. Bounded by 3.3e-7, and twice that for a
    product of two. (Accumulators of 1024 of k: 9.9e-7 and 1.8e-6.)"""
    dtype, gated, layout = form
    x, xs, w, ss, xd, wd = make(dtype, 1, n, k, rows, gated, layout, seed=n + rows)
    mm = handle(ts, w, ss, gated, layout, rows)
    y = mm.forward(x, None, xs, torch.empty(rows, n, device="cuda")).double()
    p = [xd @ (m[0] if layout == "kn" else m[0].t()) for m in wd]
    want = p[0].clamp(min=0) * p[1].clamp(min=0) if gated else p[0]
    assert float((y - want).norm() / want.norm()) <= (6.6e-7 if gated else 3.3e-7)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("sizes", [[4097, 30], [30, 9000], [4096 + 300], [8192, 1]])
def test_groups_of_several_sweeps(ts, form, sizes):
    """More than the 4096 rows of a group that one sweep over its weights serves, the last sweep narrower than the others."""
    dtype, gated, layout = form
    run(ts, dtype, sizes, 520, 144, gated, layout, F32, 3, seed=sizes[0])
    run(ts, dtype, sizes, 520, 144, gated, layout, BF16, 0, seed=sizes[0])


@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
def test_one_long_group_among_many_empty_ones(ts, gated):
    """Few rows for so many groups: the weights are the MMA's M, with several sweeps."""
    sizes = [0] * 90
    sizes[41], sizes[42], sizes[89] = 5000, 1, 20
    run(ts, E4M3, sizes, 264, 272, gated, "nk", F32, 2, seed=3)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("n,k", [(40, 32768), (32768, 64)])
def test_rows_beyond_32_bits_of_elements(ts, form, n, k):
    """x, or y, of more than 2^31 elements: the first rows, and the last ones, which are a group of their own."""
    dtype, gated, layout = form
    r, few = 65900, 60
    _, _, w, ss, _, wd = make(dtype, 2, n, k, 1, gated, layout, seed=k)
    x = torch.randn(r, k, generator=gen(3), device="cuda", dtype=BF16).to(dtype)
    xs = torch.rand(-(-k // 128), r, generator=gen(4), device="cuda") + 0.5 if dtype == E4M3 else None
    y = torch.zeros(r, n, device="cuda", dtype=BF16)
    mm = handle(ts, w, ss, gated, layout, r)
    mm.forward(x, torch.tensor([0, r - few, r], dtype=torch.int32, device="cuda"), xs, y)
    assert mm.get_error() == 0
    for at, e in ((slice(0, few), 0), (slice(r - few, r), 1)):
        xd = x[at].double()
        if xs is not None:
            xd = xd * xs[:, at].double().repeat_interleave(128, 0)[:k].t()
        check(y[at], y[at], [0, few], xd, [[ws[e]] for ws in wd], gated, layout, k)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_many_groups(ts, form):
    dtype, gated, layout = form
    sizes = [(i * 37) % 61 if i % 5 else 0 for i in range(256)]
    run(ts, dtype, sizes, 64, 128, gated, layout, F32, 0, seed=9)


def test_one_group_without_offsets(ts):
    x, xs, w, ss, xd, wd = make(BF16, 1, 320, 256, 77, False, seed=3)
    mm = ts.Grouped(w[0][0], max_rows=100)
    y = mm(x)
    assert y.dtype == BF16
    check(y, y.clone(), [0, 77], xd, wd, False, "nk", 256)
    assert mm(x[:0]).shape == (0, 320)


def test_stacked_weights(ts):
    x, xs, w, ss, xd, wd = make(E4M3, 3, 256, 256, 60, True, seed=4)
    mm = ts.Grouped.gated(torch.stack(w[0]), torch.stack(w[1]), scale_gate=torch.stack(ss[0]),
                          scale_up=torch.stack(ss[1]), max_rows=60)
    off = torch.tensor([0, 10, 10, 60], dtype=torch.int32, device="cuda")
    y = torch.zeros(60, 256, device="cuda")
    check(mm.forward(x, off, xs, y), y.clone(), [0, 10, 10, 60], xd, wd, True, "nk", 256)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("off", [[0, 30, 20, 60], [-4, 10, 30, 40], [0, 10, 30, 61], [2 ** 30, 2 ** 31 - 1, 5, 9]])
def test_bad_offsets_are_skipped_and_reported(ts, form, off):
    """Groups with usable bounds are computed, the others are skipped and recorded."""
    dtype, gated, layout = form
    x, xs, w, ss, xd, wd = make(dtype, 3, 128, 128, 60, gated, layout, seed=8)
    mm = handle(ts, w, ss, gated, layout, 60)
    y = torch.zeros(60, 128, device="cuda")
    mm.forward(x, torch.tensor(off, dtype=torch.int32, device="cuda"), xs, y)
    assert mm.get_error() == 4  # TS_ERR_BAD_INDEX
    assert mm.get_error() == 0  # cleared
    for e in range(3):
        a, b = off[e], off[e + 1]
        later = [i for j in range(3) if j != e and 0 <= off[j] <= off[j + 1] <= 60 for i in range(off[j], off[j + 1])]
        if 0 <= a <= b <= 60 and not set(later) & set(range(a, b)):
            check(y[a:b], y[a:b], [0, b - a], xd[a:b], [[ws[e]] for ws in wd], gated, layout, 128)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_non_finite_rows_keep_to_themselves(ts, form):
    """NaN or infinite rows, also of the next group and behind the last one, change no other row."""
    dtype, gated, layout = form
    sizes, n, k = [5, 20, 70], 128, 256
    off = [0, 5, 25, 95]
    x, xs, w, ss, xd, wd = make(dtype, 3, n, k, 100, gated, layout, seed=12)
    bad = [4, 5, 30, 94, 95, 99]
    x.view(torch.uint8 if dtype == E4M3 else BF16)[bad, 3] = 0x7F if dtype == E4M3 else float("nan")
    if dtype == BF16:
        x[6, 7] = float("inf")
        bad.append(6)
    mm = handle(ts, w, ss, gated, layout, 100)
    y = torch.zeros(100, n, device="cuda")
    mm.forward(x, torch.tensor(off, dtype=torch.int32, device="cuda"), xs, y)
    xd[bad] = 0.0
    keep = [r for r in range(95) if r not in bad]
    want = torch.zeros(100, n, device="cuda")
    want[bad] = y[bad]
    clean = y.clone()
    clean[bad] = 0.0
    check(clean[:95], clean[:95], off, xd[:95], wd, gated, layout, k)
    assert torch.isfinite(y[keep]).all()
    if not gated:  # a gated product of NaN is 0: neither factor is positive
        inside = [r for r in bad if r < 95]
        assert not torch.isfinite(y[inside]).any()
    assert (y[95:] == 0).all()


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_repeated_calls_give_the_same_bits(ts, form):
    """Also with calls of other sizes in between, and replayed from a graph."""
    dtype, gated, layout = form
    n, k, off = 512, 1024, [0, 9, 9, 150]
    x, xs, w, ss, xd, wd = make(dtype, 3, n, k, 150, gated, layout, seed=21)
    mm = handle(ts, w, ss, gated, layout, 150)
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    o2 = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    first = mm.forward(x, o, xs, torch.zeros(150, n, device="cuda")).clone()
    for _ in range(3):
        mm.forward(x[:3], o2, None if xs is None else xs[:, :3].contiguous(), torch.zeros(3, n, device="cuda"))
        assert torch.equal(mm.forward(x, o, xs, torch.zeros(150, n, device="cuda")), first)
    y = torch.zeros(150, n, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        mm.forward(x, o, xs, y, stream=side)
    for _ in range(2):
        y.zero_()
        graph.replay()
        assert torch.equal(y, first)
    o.copy_(torch.tensor([0, 100, 120, 150], dtype=torch.int32))  # the graph reads the offsets of its replay
    graph.replay()
    check(y, y.clone(), [0, 100, 120, 150], xd, wd, gated, layout, k)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_handles_made_and_closed_in_turn(ts, form):
    """Their scratch has one size, so that one handle's maps of weights lie where another's lay. (All weights stay.)"""
    dtype, gated, layout = form
    shapes = [(64, 128), (256, 64), (520, 256), (128, 512)]
    made = [make(dtype, 3, n, k, 50, gated, layout, seed=n + k) for n, k in shapes]
    off = [0, 20, 21, 50]
    o = torch.tensor(off, dtype=torch.int32, device="cuda")
    want = [None] * len(shapes)
    for turn in range(24):
        i = turn * 7 % 4 if turn < 12 else turn % 4
        (n, k), (x, xs, w, ss, xd, wd) = shapes[i], made[i]
        mm = handle(ts, w, ss, gated, layout, 50)
        y = torch.zeros(50, n, device="cuda")
        mm.forward(x, o, xs, y)
        assert mm.get_error() == 0
        mm.close()
        if want[i] is None:
            check(y, y.clone(), off, xd, wd, gated, layout, k)
            want[i] = y
        assert torch.equal(y, want[i])


WIDE = [f for f in FORMS if f[0] == E4M3]


@pytest.mark.parametrize("form", WIDE, ids=["plain", "gated"])
@pytest.mark.parametrize("out", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,k,pad", [(1, 16, 0), (3, 128, 0), (127, 272, 1), (257, 144, 0), (264, 1040, 4), (1000, 64, 8),
                                     (520, 2064, 0)])
def test_many_e4m3_rows(ts, form, out, n, k, pad):
    """Enough rows a group for the rows to be the MMA's M; short ones, tiles' edges, an empty group, rows behind."""
    run(ts, E4M3, [300, 0, 1, 257, 511], n, k, form[1], "nk", out, 7, seed=n + k, pad_x=16 * (pad > 0), pad_y=pad)


@pytest.mark.parametrize("form", WIDE, ids=["plain", "gated"])
def test_many_e4m3_rows_with_bad_ones(ts, form):
    """Non-finite rows of the same tile, of the next group and of no group, and bad offsets."""
    n, k, off = 200, 256, [0, 300, 290, 560, 700]
    x, xs, w, ss, xd, wd = make(E4M3, 4, n, k, 720, form[1], "nk", seed=14)
    bad = [5, 130, 299, 300, 559, 560, 700, 719]
    x.view(torch.uint8)[bad, 7] = 0x7F
    mm = handle(ts, w, ss, form[1], "nk", 720)
    y = torch.full((720, n), 7.0, device="cuda")
    mm.forward(x, torch.tensor(off, dtype=torch.int32, device="cuda"), xs, y)
    assert mm.get_error() == 4 and mm.check_scratch() == 0
    assert (y[700:] == 7.0).all()
    xd[bad] = 0.0
    got = y.clone()
    got[bad] = 0.0
    for e in (0, 2, 3):  # (rows 290 to 299 belong to two groups: either may have them)
        a, b = (off[e], 290) if e == 0 else (max(off[e], 300), off[e + 1])
        check(got[a:b], got[a:b], [0, b - a], xd[a:b], [[ws[e]] for ws in wd], form[1], "nk", k)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_a_wait_that_gives_up_last_is_reported(ts, form):
    """A summing warp's wait runs out when the CTA's loads have long ended; the context and the handle stay usable."""
    dtype, gated, layout = form
    x, xs, w, ss, xd, wd = make(dtype, 2, 256, 512, 40, gated, layout, seed=31)
    mm = handle(ts, w, ss, gated, layout, 40)
    o = torch.tensor([0, 11, 40], dtype=torch.int32, device="cuda")
    want = mm.forward(x, o, xs, torch.zeros(40, 256, device="cuda")).clone()
    assert mm.get_error() == 0
    mm.set_test_stall(True)
    mm.forward(x, o, xs, torch.zeros(40, 256, device="cuda"))
    assert mm.get_error() == 5  # TS_ERR_TIMEOUT
    mm.set_test_stall(False)
    assert torch.equal(mm.forward(x, o, xs, torch.zeros(40, 256, device="cuda")), want)
    assert mm.get_error() == 0 and mm.check_scratch() == 0


@pytest.mark.parametrize("form", [FORMS[0], FORMS[3]], ids=["bf16", "e4m3"])
def test_a_forward_on_another_stream_after_a_timeout(ts, form):
    """What get_error clears is clear when it returns."""
    dtype, gated, layout = form
    x, xs, w, ss, xd, wd = make(dtype, 1, 300, 8192, 20, gated, layout, seed=32)  # tiles in several parts
    mm = handle(ts, w, ss, gated, layout, 20)
    want = mm.forward(x, None, xs, torch.zeros(20, 300, device="cuda")).clone()
    torch.cuda.synchronize()
    mm.set_test_stall(True)
    mm.forward(x, None, xs, torch.zeros(20, 300, device="cuda"))
    torch.cuda.synchronize()
    mm.set_test_stall(False)
    assert mm.get_error() == 5
    y, side = torch.zeros(20, 300, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    mm.forward(x, None, xs, y, stream=side)
    side.synchronize()
    assert torch.equal(y, want) and mm.get_error() == 0


def test_outputs_on_a_boundary_of_their_elements(ts):
    """Others are refused by the host; these need not lie on one of 16 bytes."""
    import ctypes

    mm = ts.Grouped(torch.randn(72, 64, device="cuda").to(BF16), max_rows=4)
    x = torch.randn(4, 64, device="cuda").to(BF16)
    want = mm.forward(x, y=torch.zeros(4, 72, device="cuda"))
    raw = torch.zeros(4 * 72 * 4 + 64, dtype=torch.uint8, device="cuda")
    for size, code, bad, good in ((4, 0, (1, 2, 3, 6), (0, 4, 12)), (2, 1, (1, 3, 7), (0, 2, 6))):
        def call(at):
            return ts.lib().ts_grouped_forward(mm.handle, ctypes.c_void_p(x.data_ptr()), 64, None, 0, None, 4,
                                               ctypes.c_void_p(raw.data_ptr() + at), 72, code, None)
        for at in bad:
            assert call(at) == 1, "TS_ERR_INVALID_ARG"
        for at in good:
            assert call(at) == 0
            got = raw[at:at + 4 * 72 * size].clone().view(F32 if size == 4 else BF16).view(4, 72)
            assert torch.equal(got, want.to(got.dtype))


def test_refusals(ts):
    dev = "cuda"
    w = [torch.zeros(64, 64, dtype=BF16, device=dev) for _ in range(2)]
    mm = ts.Grouped(w, max_rows=10)
    x = torch.zeros(10, 64, dtype=BF16, device=dev)
    off = torch.zeros(3, dtype=torch.int32, device=dev)
    for call in (
        lambda: mm(x),                                             # two groups need offsets
        lambda: mm(torch.zeros(11, 64, dtype=BF16, device=dev), off),  # more rows than max_rows
        lambda: mm(x[:, :32], off),                                # another width
        lambda: mm(x, off[:2]),
        lambda: mm(x, off, x_scale=torch.ones(1, 10, device=dev)),  # scales with bf16 rows
        lambda: mm(x, off, y=torch.zeros(10, 65, device=dev)),
        lambda: ts.Grouped(w, layout="kk"),
        lambda: ts.Grouped(w, scale=[torch.ones(1, 1, device=dev)] * 2),
        lambda: ts.Grouped([]),
        lambda: ts.Grouped([w[0], w[0][:32]]),
        lambda: ts.Grouped(w[0][:, :60].contiguous()),              # k not a multiple of 8
        lambda: ts.Grouped.gated(w, w[:1]),
        lambda: ts.Grouped(w, max_rows=0),
        lambda: ts.Grouped(w[0].to(E4M3)),                          # no scales
        lambda: ts.Grouped(w[0].to(E4M3), layout="kn", scale=torch.ones(1, 1, device=dev)),
    ):
        with pytest.raises((ValueError, ts.TsError)):
            call()
    for call in (lambda: mm(x.float(), off), lambda: mm(x.cpu(), off), lambda: mm(x, off.long()),
                 lambda: ts.Grouped(w[0].float())):
        with pytest.raises(TypeError):
            call()
    shifted = torch.zeros(10 * 64 + 1, dtype=BF16, device=dev)[1:].view(10, 64)
    with pytest.raises(ts.TsError):
        mm(shifted, off)  # rows off a 16-byte boundary
    mm.close()
    with pytest.raises(RuntimeError):
        mm(x, off)
