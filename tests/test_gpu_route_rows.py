"""Routing of many tokens, rows in the experts' order, and their sums (ts_route, ts_gather_rows, ts_quant_rows,
ts_combine_rows) against plain implementations in Python and 64 bits.

Tolerances: whole numbers are equal. Routing weights: exp, a sum of at most 8 and a quotient in fp32, each off by at most
2 units in the last place (2^-22 relative): 2^-20 in all. Sums of rows: products and at most 8 sums in fp32, 16 roundings
of 2^-24 of sum |w y|. Scales: one quotient, half a unit (2^-24). An e4m3 value is within half a step (2^-4 of it, 2^-10
below 2^-6) of x / scale, whose own rounding adds 2^-23 of it."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


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


def plain_route(x, k):
    """sel, w, offsets, rows, slots of logits [t][e] (numpy, 64 bits)."""
    t, e = x.shape
    sel, slots = np.full((t, k), -1), np.full((t, k), -1)
    w = np.zeros((t, k))
    for i in range(t):
        cand = sorted((j for j in range(e) if x[i, j] > -math.inf), key=lambda j: (-x[i, j], j))[:k]
        if not cand:
            continue
        top = x[i, cand[0]]
        z = [1.0 if x[i, j] == top else math.exp(x[i, j] - top) for j in cand]
        sel[i, :len(cand)] = cand
        w[i, :len(cand)] = np.array(z) / sum(z)
    offsets, rows = [0], []
    for j in range(e):
        for i in range(t):
            at = np.nonzero(sel[i] == j)[0]
            if at.size:
                slots[i, at[0]] = len(rows)
                rows.append(i)
        offsets.append(len(rows))
    return sel, w, offsets, rows, slots


def check_route(ts, logits, k):
    t = logits.shape[0]
    rows = torch.full((t * k,), -7, dtype=torch.int32, device="cuda")
    r = ts.route(logits, k, rows=rows)
    sel, w, offsets, order, slots = plain_route(logits.double().cpu().numpy(), k)
    assert r.offsets.tolist() == offsets
    assert np.array_equal(r.sel.cpu().numpy(), sel)
    assert np.array_equal(r.slots.cpu().numpy(), slots)
    assert r.rows[:len(order)].tolist() == order
    assert (r.rows[len(order):] == -7).all(), "entries behind the last row are left as they were"
    got = r.w.double().cpu().numpy()
    assert (np.abs(got - w) <= 2.0 ** -20 * w).all()
    return r


@pytest.mark.parametrize("t", [1, 2, 31, 33, 300, 1025])
@pytest.mark.parametrize("e,k", [(1, 1), (2, 2), (8, 2), (7, 3), (16, 4), (60, 6), (64, 8), (256, 8), (129, 5)])
def test_route(ts, t, e, k):
    check_route(ts, torch.randn(t, e, generator=gen(t * 1000 + e), device="cuda"), k)


@pytest.mark.parametrize("t,e,k", [(9000, 8, 2), (20000, 4, 1), (5000, 256, 8), (40001, 16, 3)])
def test_route_many_tokens(ts, t, e, k):
    """Against sorts in torch: the plain loop is slow at this size."""
    x = torch.randn(t, e, generator=gen(t), device="cuda")
    x[::7] = -math.inf
    r = ts.route(x, k, rows=torch.full((t * k,), -1, dtype=torch.int32, device="cuda"))
    top = torch.sort(x, dim=1, descending=True, stable=True)
    sel = torch.where(top.values[:, :k] > -math.inf, top.indices[:, :k], -1)
    assert torch.equal(r.sel.long(), sel)
    flat = sel.reshape(-1)
    order = torch.sort(torch.where(flat < 0, e, flat), stable=True).indices
    n = int((flat >= 0).sum())
    assert r.offsets.tolist() == [0] + torch.bincount(flat[flat >= 0], minlength=e).cumsum(0).tolist()
    assert torch.equal(r.rows[:n].long(), order[:n] // k) and (r.rows[n:] == -1).all()
    slots = torch.full_like(flat, -1)
    slots[order[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(r.slots.reshape(-1).long(), slots)


def test_route_ties_masks_and_special_values(ts):
    inf, nan = math.inf, math.nan
    rows = [
        [0.0, 0.0, 0.0, 0.0], [1.0, 2.0, 2.0, 1.0], [-inf, -inf, -inf, -inf], [nan, nan, nan, nan],
        [-inf, 3.0, -inf, -inf], [nan, 1.0, -inf, 0.5], [inf, 0.0, inf, 1.0], [inf, -inf, nan, -inf],
        [-3.4e38, -3.4e38, -inf, 3.4e38], [0.0, -0.0, 0.0, -0.0], [-3.4028235e38] * 4, [1e-45, 0.0, -1e-45, 0.0],
    ]
    for k in (1, 2, 3, 4):
        check_route(ts, torch.tensor(rows, device="cuda"), k)


def test_route_one_expert_gets_all_and_none_gets_any(ts):
    x = torch.zeros(700, 8, device="cuda")
    x[:, 5] = 1.0
    check_route(ts, x, 1)
    check_route(ts, torch.full((700, 8), -math.inf, device="cuda"), 2)
    r = ts.route(torch.zeros(0, 8, device="cuda"), 2)
    assert r.offsets.tolist() == [0] * 9


def test_route_on_a_stream_and_in_a_graph(ts):
    x = torch.randn(3000, 8, generator=gen(1), device="cuda")
    want = ts.route(x, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ts.route(x, 2, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = ts.route(x, 2)
    y = torch.randn(3000, 8, generator=gen(2), device="cuda")
    want = ts.route(y, 2)
    x.copy_(y)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


# ---------------------------------------------------------------------------
def sources(rows, n_src, seed):
    return torch.randint(0, n_src, (rows,), generator=gen(seed), device="cuda").to(torch.int32)


@pytest.mark.parametrize("k", [8, 64, 136, 4096, 14336])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gather_rows(ts, k, dtype):
    x = torch.randn(50, k + 8, generator=gen(k), device="cuda").to(dtype)[:, :k]
    rows = sources(77, 50, 3)
    rows[5], rows[6], rows[76] = -1, 50, 2 ** 31 - 1  # out of range: left as they were
    for n in (None, 0, 1, 40, 77, 1000):
        out = torch.randn(77, k, generator=gen(9), device="cuda").to(dtype)
        want = out.clone()
        m = 77 if n is None else min(n, 77)
        live = torch.zeros(77, dtype=torch.bool, device="cuda")
        live[:m] = True
        live &= (rows >= 0) & (rows < 50)
        want[live] = x[rows[live].long()]
        nt = None if n is None else torch.tensor([n], dtype=torch.int32, device="cuda")
        assert torch.equal(ts.gather_rows(x, rows, n=nt, out=out), want)
    assert ts.gather_rows(x, rows[:0]).shape == (0, k)


def steps_off(q, v):
    """How many half steps of e4m3 the values q lie off v."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return ((q - v).abs() / (step / 2)).max()


@pytest.mark.parametrize("k", [16, 128, 144, 4096, 14336])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 33, 200])
def test_quant_rows(ts, k, dtype, rows):
    g = gen(k + rows)
    x = (torch.randn(rows, k + 16, generator=g, device="cuda") * torch.exp(4 * torch.randn(rows, 1, generator=g, device="cuda")))
    x[0, :k // 2] = 0.0
    x = x.to(dtype)[:, :k]
    order = sources(rows + 3, rows, 4)
    q, s = ts.quant_rows(x, rows=order)
    xd = x.double()[order.long()]
    kb = -(-k // 128)
    for b in range(kb):
        v = xd[:, 128 * b:128 * b + 128]
        top = v.abs().amax(1)
        want = torch.where(top > 0, (top / 448).clamp(min=2.0 ** -100), 1.0)
        sc = s[b].double()
        assert ((sc - want).abs() <= 2.0 ** -24 * want).all()
        got = q.double()[:, 128 * b:128 * b + 128]
        assert got.abs().max() <= 448
        assert steps_off(got, v / sc[:, None]) <= 1 + 2.0 ** -18
    same = ts.quant_rows(x)
    assert torch.equal(same[0].view(torch.uint8)[order.long()], q.view(torch.uint8))
    assert torch.equal(same[1][:, order.long()], s)


def test_quant_rows_special_values_and_untouched_rows(ts):
    k = 256
    x = torch.zeros(6, k, device="cuda")
    x[0, 0], x[0, 130] = 1e-38, 3e38          # far below the least scale; near the largest number
    x[1, 5], x[1, 140] = math.nan, 7.0        # NaN stays in its place
    x[1, 6] = 448.0
    x[2, 3] = math.inf
    x[2, 200] = -1.0
    x[3] = -0.0
    rows = torch.tensor([0, 1, 2, 3, -1, 6, 4, 5], dtype=torch.int32, device="cuda")
    q = torch.full((8, k), 3.0, device="cuda").to(E4M3)
    s = torch.full((2, 8), -5.0, device="cuda")
    ts.quant_rows(x, rows=rows, n=torch.tensor([7], dtype=torch.int32, device="cuda"), q=q, scale=s)
    v = q.double() * s.double().repeat_interleave(128, 0).t()
    assert float(s[0, 0]) == 2.0 ** -100 and float(q[0, 0]) == 0.0
    assert abs(float(v[0, 130]) / 3e38 - 1) <= 2.0 ** -4
    assert math.isnan(float(v[1, 5])) and float(v[1, 6]) == 448.0 and float(s[0, 1]) == 1.0
    assert torch.isfinite(v[1, 6:]).all()
    assert torch.isnan(v[2, :128]).all() and torch.isfinite(v[2, 128:]).all()
    assert (v[3] == 0).all() and (s[:, 3] == 1).all()
    for r in (4, 5, 7):  # bad entries, and the row behind the count
        assert (q[r].float() == 3.0).all() and (s[:, r] == -5.0).all()
    assert (q[6].float() == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t,k,n", [(1, 1, 1), (3, 2, 7), (70, 8, 4096), (200, 2, 1001), (33, 3, 5000)])
def test_combine_rows(ts, dtype, t, k, n):
    g = gen(t + n)
    src = torch.randn(max(1, t), n, generator=g, device="cuda").to(dtype)
    slots = torch.randint(-1, t + 1, (t, k), generator=g, device="cuda").to(torch.int32)  # -1 and t: no row
    w = torch.randn(t, k, generator=g, device="cuda")
    got = ts.combine_rows(src, slots, w).double()
    ok = ((slots >= 0) & (slots < t))[..., None]
    terms = torch.where(ok, w.double()[..., None] * src.double()[slots.clamp(0, t - 1).long()], 0.0)
    assert ((got - terms.sum(1)).abs() <= 16 * 2.0 ** -24 * terms.abs().sum(1)).all()


@pytest.mark.parametrize("t", [65535, 65536, 131071, 131073])
@pytest.mark.parametrize("dtype,n", [(BF16, 8), (F32, 5)])
def test_combine_rows_of_many_tokens(ts, t, dtype, n):
    """More tokens than one launch's grid holds."""
    g = gen(t)
    src = torch.randn(1000, n, generator=g, device="cuda").to(dtype)
    slots = torch.randint(-1, 1001, (t, 2), generator=g, device="cuda").to(torch.int32)
    w = torch.randn(t, 2, generator=g, device="cuda")
    out = torch.full((t + 1, n), 7.0, device="cuda")
    ts.combine_rows(src, slots, w, out=out[:t])
    ok = ((slots >= 0) & (slots < 1000))[..., None]
    terms = torch.where(ok, w.double()[..., None] * src.double()[slots.clamp(0, 999).long()], 0.0)
    assert ((out[:t].double() - terms.sum(1)).abs() <= 16 * 2.0 ** -24 * terms.abs().sum(1)).all()
    assert (out[t] == 7.0).all()


def test_rows_beyond_32_bits_of_elements(ts):
    """Inputs and outputs of more than 2^31 elements: what lies at their ends."""
    r, k = 65900, 32768
    x = torch.randn(r, k, generator=gen(1), device="cuda", dtype=BF16)
    order = torch.arange(r - 1, -1, -1, device="cuda").to(torch.int32)
    assert torch.equal(ts.gather_rows(x, order), x.flip(0))
    q, s = ts.quant_rows(x)
    few_q, few_s = ts.quant_rows(x[-50:])
    assert torch.equal(q[-50:].view(torch.uint8), few_q.view(torch.uint8)) and torch.equal(s[:, -50:], few_s)
    del q, s
    slots = torch.stack([order, order.flip(0)], 1).contiguous()
    w = torch.rand(r, 2, generator=gen(2), device="cuda")
    y = ts.combine_rows(x, slots, w)
    for t in (0, 7, r - 1):
        terms = w[t].double()[:, None] * x[slots[t].long()].double()
        assert ((y[t].double() - terms.sum(0)).abs() <= 16 * 2.0 ** -24 * terms.abs().sum(0)).all()


def test_combine_rows_without_rows(ts):
    src = torch.zeros(0, 64, device="cuda")
    y = ts.combine_rows(src, torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.ones(4, 2, device="cuda"))
    assert (y == 0).all()
    src = torch.full((3, 64), math.nan, device="cuda")  # rows that no slot names are not read into a sum
    y = ts.combine_rows(src, torch.full((4, 2), -1, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"))
    assert (y == 0).all()


def test_refusals(ts):
    dev, i32 = "cuda", torch.int32
    x = torch.zeros(4, 8, device=dev)
    for call in (
        lambda: ts.route(x, 0), lambda: ts.route(x, 9), lambda: ts.route(torch.zeros(4, 257, device=dev), 2),
        lambda: ts.route(x, 2, sel=torch.zeros(4, 3, dtype=i32, device=dev)), lambda: ts.route(x.t(), 2),
        lambda: ts.gather_rows(x, torch.zeros(2, 1, dtype=i32, device=dev)),
        lambda: ts.gather_rows(x[:, :3], torch.zeros(2, dtype=i32, device=dev)),
        lambda: ts.gather_rows(x, torch.zeros(2, dtype=i32, device=dev), out=torch.zeros(3, 8, device=dev)),
        lambda: ts.gather_rows(x, torch.zeros(2, dtype=i32, device=dev), n=torch.zeros(2, dtype=i32, device=dev)),
        lambda: ts.quant_rows(x), lambda: ts.quant_rows(torch.zeros(4, 24, device=dev)),
        lambda: ts.combine_rows(x, torch.zeros(2, 9, dtype=i32, device=dev), torch.zeros(2, 9, device=dev)),
        lambda: ts.combine_rows(x, torch.zeros(2, 2, dtype=i32, device=dev), torch.zeros(2, 3, device=dev)),
    ):
        with pytest.raises((ValueError, ts.TsError)):
            call()
    for call in (
        lambda: ts.route(x.double(), 2), lambda: ts.route(x.cpu(), 2),
        lambda: ts.gather_rows(x, torch.zeros(2, dtype=torch.int64, device=dev)),
        lambda: ts.quant_rows(torch.zeros(4, 16, dtype=torch.float16, device=dev)),
    ):
        with pytest.raises(TypeError):
            call()
