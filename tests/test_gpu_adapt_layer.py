"""The gated activation kept in 8 bits, balance loss, gradients of routing and of combined rows, and a whole tuning step of
an adapted layer, against plain implementations in 64 bits.

Tolerances. What is kept and its backward pass are exact up to one rounding, which is emulated: equal bits, but for outputs of
fp32 inputs, whose product is rounded to fp32 before bf16 (equal to the same in torch). Probabilities: exp and a quotient of 2
units in the last place, a sum of at most 256 in 6 levels: 16 roundings of 2^-23; the mean of them over t tokens t / 8 + 16 more at
most; the loss and the logits' gradient a few dozen more: bounds of n 2^-23 of the terms' magnitudes, n written beside. Sums over
n columns: n / 256 + 16 roundings of 2^-24 of the magnitudes' sum."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
U = 2.0 ** -23


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


# ---------------------------------------------------------------------------
# the activation
# ---------------------------------------------------------------------------
def plain_kept(v):
    """(q, scale [blocks][rows]) of factors [rows][m] that are not negative, in 64 bits of numpy."""
    r, m = v.shape
    mb = -(-m // 128)
    p = np.zeros((r, mb * 128))
    p[:, :m] = np.minimum(v, 1.875 * 2.0 ** 127)
    p = p.reshape(r, mb, 128)
    top = p.max(2)
    part, e = np.frexp(top)
    scale = np.where(top > 0, np.ldexp(1.0, np.maximum(np.where(part <= 0.875, e - 9, e - 8), -100)), 1.0)
    x = p / scale[..., None]
    step = np.ldexp(1.0, np.maximum(np.frexp(np.maximum(x, 1e-300))[1] - 1, -6) - 3)
    q = np.rint(x / step) * step
    return np.where((p > 0) & (q == 0), 2.0 ** -9, q).reshape(r, mb * 128)[:, :m], scale.T


def same(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def check_drelu(ts, g, u, dc, n=None):
    r, m = g.shape
    live = r if n is None else min(r, int(n))
    c0, dg0, du0, again0 = (torch.full((r, m), 3.0, dtype=BF16, device="cuda") for _ in range(4))
    kept = ts.Kept(*(torch.full((r, m), 2.0, device="cuda").to(E4M3) for _ in range(2)),
                   *(torch.full((-(-m // 128), r), 5.0, device="cuda") for _ in range(2)))
    c, kept = ts.drelu_rows(g, u, n=n, c=c0, kept=kept)
    dg, du, again = ts.drelu_rows_backward(dc, kept, n=n, dg=dg0, du=du0, c=again0)
    assert c is c0 and dg is dg0 and again is again0
    for v in (c, dg, du, again):
        assert (v[live:] == 3).all()
    assert (kept.q_gate[live:].float() == 2).all() and (kept.s_up[:, live:] == 5).all()
    both = (g > 0) & (u > 0)
    fg, fu = (torch.where(both, v.float(), 0.0) for v in (g, u))
    want = (fg * fu).to(BF16)
    assert torch.equal(c[:live], want[:live])
    wide = []
    for f, q, s in ((fg, kept.q_gate, kept.s_gate), (fu, kept.q_up, kept.s_up)):
        wq, ws = plain_kept(f[:live].double().cpu().numpy())
        assert np.array_equal(q[:live].double().cpu().numpy(), wq)
        assert np.array_equal(s[:, :live].double().cpu().numpy(), ws)
        wide.append(torch.from_numpy(wq * np.repeat(ws.T, 128, axis=1)[:, :m]).cuda())
    assert ((wide[0] > 0) == both[:live]).all() and ((wide[1] > 0) == both[:live]).all()
    both, d = both[:live], dc[:live].float()
    for got, v in ((dg, wide[1]), (du, wide[0])):
        assert same(got[:live], torch.where(both, d * v.float(), 0.0).to(BF16))
    assert torch.equal(again[:live], (wide[0].float() * wide[1].float()).to(BF16))
    assert torch.equal(ts.drelu_rows(g, u)[:live], c[:live])
    assert ts.drelu_rows_backward(dc, kept, n=n, again=False)[2] is None
    return c, kept


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("r,m", [(1, 16), (1, 14336), (7, 144), (8, 128), (9, 1408), (33, 1040), (300, 528), (64, 4096)])
def test_drelu(ts, r, m, dtype):
    g = gen(r + m)
    args = [(randn(g, r, m) - 0.3).to(dtype) for _ in range(2)] + [randn(g, r, m).to(dtype)]
    check_drelu(ts, *args)
    check_drelu(ts, *args, n=torch.tensor([r // 2], dtype=torch.int32, device="cuda"))
    check_drelu(ts, *args, n=torch.tensor([r + 5], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_drelu_count_below_zero(ts, dtype):
    """A negative count is of no rows: nothing is written, neither rows nor scales nor what lies behind these."""
    for r, m in ((9, 272), (8, 128), (1, 1408)):
        mb = -(-m // 128)
        g, u, dc = (1.0 + randn(gen(m + i), r, m).abs().to(dtype) for i in range(3))
        for count in (-1, -2 ** 31):
            n = torch.tensor([count], dtype=torch.int32, device="cuda")
            scales = torch.full((2, mb * r + 16), 5.0, device="cuda")  # 16 elements behind each
            kept = ts.Kept(*(torch.full((r, m), 2.0, device="cuda").to(E4M3) for _ in range(2)),
                           *(s[:mb * r].view(mb, r) for s in scales))
            outs = [torch.full((r, m), 3.0, dtype=BF16, device="cuda") for _ in range(4)]
            ts.drelu_rows(g, u, n=n, c=outs[0], kept=kept)
            ts.drelu_rows_backward(dc, kept, n=n, dg=outs[1], du=outs[2], c=outs[3])
            assert (scales == 5).all() and all((o == 3).all() for o in outs)
            assert (kept.q_gate.float() == 2).all() and (kept.q_up.float() == 2).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_drelu_values(ts, dtype):
    """Zeros, subnormal and huge numbers, infinities, NaN, values next to a scale's border and to 0 in e4m3, in every pair."""
    v = [0.0, -0.0, 1.0, -1.0, 448.0, 449.0, 450.0, 447.0, 1.75, 1.7578125, 2.0 ** -9, 2.0 ** -10, 2.0 ** -11, 1e-30, 1e-38, 1e-40, 3e38,
         3.38e38, math.inf, -math.inf, math.nan, 2.0 ** 100, 2.0 ** -100, 2.0 ** -126, 1.0625, 1.1875, 17.0, 0.3, 3.19e38]
    g = torch.tensor([[a] * len(v) for a in v], device="cuda").reshape(-1)
    u = torch.tensor(v * len(v), device="cuda")
    pad = -len(g) % 16
    g, u = torch.nn.functional.pad(g, (0, pad)), torch.nn.functional.pad(u, (0, pad))
    g, u = torch.stack([g, u, g * 0 + 2.0]).to(dtype), torch.stack([u, g, u]).to(dtype)
    dc = torch.tensor([1.0, math.nan, -3.0], device="cuda")[:, None].expand_as(g).to(dtype).contiguous()
    dc[1] = torch.where((g[1] > 0) & (u[1] > 0), 0.5, math.nan).to(dtype)  # NaN where neither has a gradient
    finite = torch.isfinite(g.float()) & torch.isfinite(u.float())
    check_drelu(ts, torch.where(finite | (g != g) | (u != u), g, 1.0), torch.where(finite | (g != g) | (u != u), u, 1.0), dc)
    c, kept = ts.drelu_rows(g, u, keep=True)
    inf = torch.isinf(g.float()) & (g > 0) & (u > 0)
    assert (c[inf].float() == math.inf).all()
    wide = kept.q_gate.float() * kept.s_gate.repeat_interleave(128, 0)[:g.shape[1]].t()
    assert (wide[inf] == 1.875 * 2.0 ** 127).all()


def test_drelu_columns_of_wider_rows(ts):
    """g and u as the halves of one product, dg and du as those of one buffer."""
    r, m = 50, 272
    g = gen(1)
    both = randn(g, r, 2 * m).to(BF16)
    dc = randn(g, r, m).to(BF16)
    c, kept = check_drelu(ts, both[:, :m].contiguous(), both[:, m:].contiguous(), dc)
    wide = torch.full((r, 2 * m + 16), 7.0, dtype=BF16, device="cuda")
    c2, kept2 = ts.drelu_rows(both[:, :m], both[:, m:], c=wide[:, 8:m + 8], keep=True)
    assert torch.equal(c, c2) and all(torch.equal(a.float(), b.float()) for a, b in zip(kept, kept2))
    assert (wide[:, :8] == 7).all() and (wide[:, m + 8:] == 7).all()
    d = torch.full((r, 2 * m + 16), 7.0, dtype=BF16, device="cuda")
    ts.drelu_rows_backward(dc, kept, dg=d[:, :m], du=d[:, m:2 * m])
    dg, du, _ = ts.drelu_rows_backward(dc, kept)
    assert torch.equal(d[:, :m], dg) and torch.equal(d[:, m:2 * m], du) and (d[:, 2 * m:] == 7).all()


def test_drelu_in_place(ts):
    """c over g or u, and one of dg, du and c over dc, of one type: as apart. Half over it is refused, and nothing is written."""
    g = gen(8)
    for r, m, wide in ((1, 2064, 0), (37, 1408, 0), (20, 272, 32)):
        gate, up, dc = (randn(g, r, m + wide).to(BF16)[:, wide // 2:wide // 2 + m] for _ in range(3))
        c, kept = ts.drelu_rows(gate, up, keep=True)
        want = ts.drelu_rows_backward(dc, kept)
        for which in range(2):
            args = [gate.clone(), up.clone()]
            got, k = ts.drelu_rows(*args, c=args[which], keep=True)
            assert got is args[which] and torch.equal(got, c) and torch.equal(args[1 - which], (up, gate)[which])
            assert all(torch.equal(p.float(), q.float()) for p, q in zip(k, kept))
        for which in ("dg", "du", "c"):
            d = torch.empty(r, m + wide, dtype=BF16, device="cuda")[:, wide // 2:wide // 2 + m].copy_(dc)
            got = ts.drelu_rows_backward(d, kept, **{which: d})
            assert all(torch.equal(p, q) for p, q in zip(got, want))
        flat = torch.ones((r + 1) * m, dtype=BF16, device="cuda")
        near, behind = flat[:r * m].view(r, m), flat[m // 2:m // 2 + r * m].view(r, m)
        for call in (lambda: ts.drelu_rows(near, up, c=behind), lambda: ts.drelu_rows(gate, near, c=behind),
                     lambda: ts.drelu_rows_backward(near, kept, du=behind), lambda: ts.drelu_rows_backward(dc, kept, dg=near, du=behind)):
            with pytest.raises(ts.TsError):
                call()
        torch.cuda.synchronize()
        assert (flat == 1).all()


def test_drelu_rows_beyond_32_bits(ts):
    r, m = 150_000, 14336  # 2.15e9 elements
    g = torch.empty(r, m, dtype=BF16, device="cuda")
    g[-9:] = randn(gen(2), 9, m).to(BF16)
    n = torch.tensor([r], dtype=torch.int32, device="cuda")
    c, kept = ts.drelu_rows(g, g, n=n, keep=True)
    want, k = ts.drelu_rows(g[-9:].contiguous(), g[-9:].contiguous(), keep=True)
    assert torch.equal(c[-9:], want) and torch.equal(kept.q_up[-9:].view(torch.uint8), k.q_up.view(torch.uint8))
    dg, du, again = ts.drelu_rows_backward(g, kept, du=c)
    small = ts.drelu_rows_backward(g[-9:].contiguous(), k)
    assert all(torch.equal(a[-9:], b) for a, b in zip((dg, du, again), small))


def test_drelu_no_rows_and_refusals(ts):
    z = torch.zeros(0, 64, dtype=BF16, device="cuda")
    c, kept = ts.drelu_rows(z, z, keep=True)
    assert c.shape == (0, 64) and ts.drelu_rows_backward(z, kept)[0].shape == (0, 64)
    x = torch.zeros(4, 64, dtype=BF16, device="cuda")
    _, kept = ts.drelu_rows(x, x, keep=True)
    n = torch.tensor([2], dtype=torch.int32, device="cuda")
    for error, call in (
        (TypeError, lambda: ts.drelu_rows(x, x.float())), (ValueError, lambda: ts.drelu_rows(x, x[:, :48])),
        (TypeError, lambda: ts.drelu_rows(x.half(), x.half())), (TypeError, lambda: ts.drelu_rows(x, x, c=x.float())),
        (ValueError, lambda: ts.drelu_rows(x, x, c=x[:3])), (TypeError, lambda: ts.drelu_rows(x, x, n=n.long())),
        (ValueError, lambda: ts.drelu_rows(x, x, kept=kept._replace(s_up=kept.s_up[:, :3]))),
        (TypeError, lambda: ts.drelu_rows(x, x, kept=kept._replace(q_up=x))),
        (ValueError, lambda: ts.drelu_rows_backward(x[:3], kept)), (TypeError, lambda: ts.drelu_rows_backward(x, kept, dg=x.float())),
        (ts.TsError, lambda: ts.drelu_rows(x[:, :40].contiguous(), x[:, :40].contiguous())),
        (ts.TsError, lambda: ts.drelu_rows(x[:, 4:52], x[:, 4:52])),
    ):
        with pytest.raises(error):
            call()


# ---------------------------------------------------------------------------
# balance
# ---------------------------------------------------------------------------
def plain_balance(x, sel, w, dw, dloss):
    """loss, counts, share, dlogits, and a bound of the terms of dlogits, in 64 bits on the host."""
    x, sel = x.double().cpu(), sel.long().cpu()
    t, e = x.shape
    x = torch.where(x.isnan(), -math.inf, x)
    top = x.amax(1, keepdim=True) if t else x.new_zeros(0, 1)
    live = top[:, 0] > -math.inf
    z = torch.where(x == top, 1.0, torch.exp(x - top)) * (x > -math.inf)
    p = torch.zeros_like(x)
    p[live] = z[live] / z[live].sum(1, keepdim=True)
    picked = (sel >= 0) & (sel < e)
    counts = torch.bincount(sel[picked], minlength=e)
    tokens, picks = int(live.sum()), int(counts.sum())
    share = p.sum(0) / max(tokens, 1)
    loss = e * float((counts * share).sum()) / picks if picks else 0.0
    d, mag = torch.zeros_like(x), torch.zeros_like(x)
    if dloss is not None and picks and tokens:
        f = float(dloss) * e / picks / tokens
        c = counts.double()
        d += f * p * (c - (p @ c)[:, None])
        mag += abs(f) * p * (c + (p @ c)[:, None])
    if dw is not None:
        w, dw = torch.where(picked, w.double().cpu(), 0.0), torch.where(picked, dw.double().cpu(), 0.0)
        for j in range(sel.shape[1]):
            at = torch.nonzero(picked[:, j])[:, 0]
            d[at, sel[at, j]] += w[at, j] * (dw[at, j] - (w * dw).sum(1)[at])
            mag[at, sel[at, j]] += w[at, j].abs() * (dw[at, j].abs() + (w * dw).abs().sum(1)[at])
    return loss, counts, share, d, mag


def check_balance(ts, x, k, sel=None):
    t, e = x.shape
    r = ts.route(x, k)
    sel = r.sel if sel is None else sel
    dw, dloss = randn(gen(t + e), t, k), torch.tensor([3.0 * max(t, 1)], device="cuda")
    b = ts.balance(x, sel)
    loss, counts, share, _, _ = plain_balance(x, sel, r.w, dw, dloss)
    assert torch.equal(b.counts.cpu().long(), counts)
    assert b.totals.tolist() == [int((x > -math.inf).any(1).sum()), int(counts.sum())]
    n = t / 8 + 40
    assert ((b.share.double().cpu() - share).abs() <= n * U * share).all()
    assert abs(float(b.loss) - loss) <= (n + 8) * U * loss
    for use_w, use_l in ((True, True), (True, False), (False, True)):
        got = ts.route_backward(x, sel, r.w, dw=dw if use_w else None, balance=b if use_l else None, dloss=dloss if use_l else None)
        _, _, _, want, mag = plain_balance(x, sel, r.w, dw if use_w else None, dloss if use_l else None)
        # p 16, f 4, the sum over the experts 16, the products 4. fp32 numbers below 2^-126 are 2^-149 apart: p, which may be
        # one, is off by 2 such steps of exp and half a one of the quotient as well (and is multiplied by f (counts + dot)), and
        # so is each product
        floor = 4 * 2.0 ** -149 * (2 + 2 * float(dloss) * e * int(counts.max()) / max(1, int(counts.sum())) / max(1, b.totals[0].item()))
        assert ((got.double().cpu() - want).abs() <= 40 * U * mag + floor).all()
    again = ts.balance(x, sel)
    assert all(torch.equal(p, q) for p, q in zip(again, b))
    return b


@pytest.mark.parametrize("t", [1, 2, 31, 300, 3000])
@pytest.mark.parametrize("e,k", [(1, 1), (2, 2), (8, 2), (7, 3), (16, 4), (60, 6), (64, 8), (256, 8), (129, 5)])
def test_balance(ts, t, e, k):
    check_balance(ts, randn(gen(t + e), t, e) + randn(gen(e), e), k)


def test_balance_many_tokens(ts):
    x = randn(gen(1), 60000, 16)
    x[::5] = -math.inf
    check_balance(ts, x, 3)


def test_balance_masks_and_special_values(ts):
    inf, nan = math.inf, math.nan
    rows = [[0.0] * 4, [-inf] * 4, [nan] * 4, [-inf, 3.0, -inf, -inf], [nan, 1.0, -inf, 0.5], [inf, 0.0, inf, 1.0],
            [inf, -inf, nan, -inf], [-3.4e38, -3.4e38, -inf, 3.4e38], [100.0, -100.0, 90.0, 0.0]]
    x = torch.tensor(rows, device="cuda")
    for k in (1, 2, 4):
        check_balance(ts, x, k)
    sel = torch.tensor([[0, 0], [1, 1], [5, -1], [-9, 2 ** 31 - 1], [3, 2], [0, 1], [2, 2], [1, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    check_balance(ts, x, 2, sel=sel)
    for t in (0, 5):
        b = check_balance(ts, torch.full((t, 8), -inf, device="cuda"), 2)
        assert float(b.loss) == 0 and b.totals.tolist() == [0, 0] and (b.share == 0).all()
    even = ts.balance(torch.zeros(8, 4, device="cuda"), torch.arange(8, device="cuda").to(torch.int32)[:, None] % 4)
    assert float(even.loss) == 1.0 and even.counts.tolist() == [2] * 4


@pytest.mark.parametrize("t,e,k", [(9, 8, 2), (70, 60, 4)])
def test_balance_of_dropped_tokens(ts, t, e, k):
    """Live tokens without a pick have the balance loss's gradient and nothing of the weights'; tokens that are not live have 0."""
    x = randn(gen(t), t, e)
    x[1::4], x[2::4, 0], x[3, 1] = -math.inf, -math.inf, math.nan
    r = ts.route(x, k)
    sel = r.sel.clone()
    sel[::2] = -1  # dropped
    sel[4], sel[6, 0] = e, -7
    b, dw, dloss = ts.balance(x, sel), randn(gen(e), t, k), torch.tensor([float(t)], device="cuda")
    both = ts.route_backward(x, sel, r.w, dw=dw, balance=b, dloss=dloss)
    loss = ts.route_backward(x, sel, r.w, balance=b, dloss=dloss)
    weights = ts.route_backward(x, sel, r.w, dw=dw)
    assert torch.equal(both[::2], loss[::2]) and (weights[::2] == 0).all() and (weights[3] != 0).sum() == k
    assert (both[1::4] == 0).all() and (both[2::4, 0] == 0).all() and both[3, 1] == 0
    live = torch.nonzero((x > -math.inf).any(1))[:, 0]
    assert (loss[live] != 0).any(1).all()
    _, _, _, want, mag = plain_balance(x, sel, r.w, dw, dloss)
    assert ((both.double().cpu() - want).abs() <= 40 * U * mag).all()


@pytest.mark.parametrize("scale", [math.inf, -math.inf, math.nan])
def test_balance_of_a_loss_that_overflowed(ts, scale):
    """Tokens that are not live, and experts of logit -infinity or NaN, have 0 whatever the loss's gradient is."""
    x = randn(gen(5), 40, 12)
    x[::3], x[1::3, 2:5], x[2::3, 11] = -math.inf, -math.inf, math.nan
    r = ts.route(x, 3)
    dloss, off = torch.tensor([scale], device="cuda"), ~(x > -math.inf)
    got = ts.route_backward(x, r.sel, r.w, balance=ts.balance(x, r.sel), dloss=dloss)
    assert (got[off] == 0).all() and not torch.isfinite(got[~off]).any()


@pytest.mark.parametrize("t,e,k", [(1, 8, 2), (700, 7, 3), (300, 256, 8), (90, 60, 4)])
def test_route_backward_in_place(ts, t, e, k):
    """The gradient over the logits themselves is as apart; partly over them it is refused, and nothing is written."""
    flat = randn(gen(t), (t + 1) * e)
    x = flat[:t * e].view(t, e)
    r = ts.route(x, k)
    b, dw, dloss = ts.balance(x, r.sel), randn(gen(e), t, k), torch.tensor([2.0], device="cuda")
    want, before = ts.route_backward(x, r.sel, r.w, dw=dw, balance=b, dloss=dloss), flat.clone()
    with pytest.raises(ts.TsError):
        ts.route_backward(x, r.sel, r.w, dw=dw, balance=b, dloss=dloss, dlogits=flat[1:1 + t * e].view(t, e))
    with pytest.raises(ts.TsError):
        ts.balance(x, r.sel, share=x[0])
    torch.cuda.synchronize()
    assert torch.equal(flat, before)
    assert torch.equal(ts.route_backward(x, r.sel, r.w, dw=dw, balance=b, dloss=dloss, dlogits=x), want) and torch.equal(x, want)


def test_balance_gradient_against_differences(ts):
    """Of loss + sum(w * weight), by central differences in 64 bits: the step's own error is of third order."""
    t, e, k = 40, 9, 3
    x = randn(gen(3), t, e)
    x[5] = -math.inf
    x[6, 2:] = -math.inf
    dw = randn(gen(4), t, k)
    r = ts.route(x, k)
    b = ts.balance(x, r.sel)
    got = ts.route_backward(x, r.sel, r.w, dw=dw, balance=b, dloss=torch.tensor([2.0], device="cuda")).double()

    def value(z):
        live = torch.isfinite(z).any(1)
        p = torch.zeros_like(z)
        p[live] = torch.softmax(z[live], 1)
        counts = torch.bincount(r.sel[r.sel >= 0].long(), minlength=e).double()
        loss = e * (counts / counts.sum() * p.sum(0) / live.sum()).sum()
        v = torch.where(r.sel >= 0, z.gather(1, r.sel.clamp(min=0).long()), -math.inf)
        w = torch.where(live[:, None], torch.softmax(torch.where(live[:, None], v, 0.0), 1), 0.0)
        return float(2.0 * loss + (w * dw.double()).sum())

    for seed in range(3):
        d = randn(gen(seed), t, e).double()
        step = 1e-4
        want = (value(x.double() + step * d) - value(x.double() - step * d)) / (2 * step)
        assert abs(float((got * d).sum()) - want) <= 1e-5 * float(got.norm() * d.norm())  # 1e-8 of the step, 2^-20 of got


def test_balance_refusals(ts):
    x, sel = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    w, b = torch.zeros(4, 2, device="cuda"), ts.balance(torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda"))
    d = torch.ones(1, device="cuda")
    for error, call in (
        (TypeError, lambda: ts.balance(x.double(), sel)), (ValueError, lambda: ts.balance(x, sel[:3])), (TypeError, lambda: ts.balance(x, sel.long())),
        (ts.TsError, lambda: ts.balance(torch.zeros(4, 257, device="cuda"), sel)), (ts.TsError, lambda: ts.balance(x[:, :1].contiguous(), sel)),
        (ValueError, lambda: ts.balance(x, sel, counts=sel[:, 0].contiguous())), (ValueError, lambda: ts.route_backward(x, sel, w)),
        (ValueError, lambda: ts.route_backward(x, sel, w, balance=b)), (ValueError, lambda: ts.route_backward(x, sel, w, dloss=d)),
        (ValueError, lambda: ts.route_backward(x, sel, w[:3], dw=w)), (TypeError, lambda: ts.route_backward(x, sel, w, dw=w.double())),
        (ValueError, lambda: ts.route_backward(x, sel, w, balance=b._replace(counts=b.counts[:4]), dloss=d)),
        (ValueError, lambda: ts.route_backward(x, sel, w, dw=w, dlogits=x[:3])),
    ):
        with pytest.raises(error):
            call()


# ---------------------------------------------------------------------------
# combined rows
# ---------------------------------------------------------------------------
def check_combine(ts, dy, src, slots, w, rows):
    t, k = slots.shape
    dsrc = torch.full_like(src, 3.0)
    got, dw = ts.combine_rows_backward(dy, src, slots, w, rows, dsrc=dsrc)
    m, n = src.shape
    want, wdw, mag = np.full((m, n), 3.0), np.zeros((t, k)), np.zeros((t, k))
    sl, rw, ww = slots.tolist(), rows.tolist(), w.double().tolist()
    d, s = dy.double().cpu().numpy(), src.double().cpu().numpy()
    for i in range(t):
        for j in range(k):
            if 0 <= sl[i][j] < m:
                wdw[i, j], mag[i, j] = d[i] @ s[sl[i][j]], np.abs(d[i]) @ np.abs(s[sl[i][j]])
    for r in range(m):
        if 0 <= rw[r] < t and r in sl[rw[r]]:
            want[r] = sum(ww[rw[r]][j] for j in range(k) if sl[rw[r]][j] == r) * d[rw[r]]
    tol = np.abs(want) * ((2.0 ** -8 if src.dtype == BF16 else 0.0) + k * 2.0 ** -23)
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    assert (np.abs(dw.double().cpu().numpy() - wdw) <= (n / 256 + 16) * 2.0 ** -24 * mag).all()
    again = ts.combine_rows_backward(dy, src, slots, w, rows, dsrc=torch.full_like(src, 3.0))
    assert torch.equal(again[0], got) and torch.equal(again[1], dw)


@pytest.mark.parametrize("ddt,dt", [(F32, BF16), (F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("t,e,k,n", [(1, 2, 1, 8), (1, 8, 2, 4096), (5, 8, 2, 7), (33, 16, 8, 264), (40, 7, 3, 2049), (64, 8, 5, 512)])
def test_combine_backward(ts, t, e, k, n, ddt, dt):
    g = gen(t + n)
    logits = randn(g, t, e)
    if t > 1:
        logits[::4] = -math.inf
    rows = torch.full((t * k,), -1, dtype=torch.int32, device="cuda")
    r = ts.route(logits, k, rows=rows)
    check_combine(ts, randn(g, t, n).to(ddt), randn(g, t * k, n).to(dt), r.slots, r.w, r.rows)


def test_combine_backward_odd_slots(ts):
    """A row twice in a token, in two tokens, slots and row numbers out of range, rows that begin off 16 bytes."""
    g = gen(5)
    slots = torch.tensor([[0, 0, 1], [2, -1, 9], [0, 3, 3], [-5, 2 ** 31 - 1, 4]], dtype=torch.int32, device="cuda")
    rows = torch.tensor([0, 0, 1, 2, 3, 7, -1], dtype=torch.int32, device="cuda")
    for n in (16, 15):
        for dt in (BF16, F32):
            check_combine(ts, randn(g, 4, n), randn(g, 7, n).to(dt), slots, randn(g, 4, 3), rows)
    flat = randn(g, 4 * 16 + 1).to(BF16)
    check_combine(ts, flat[1:].view(4, 16), randn(g, 7, 16).to(BF16), slots, randn(g, 4, 3), rows)


def test_combine_backward_no_rows_and_refusals(ts):
    i32 = torch.int32
    dy, src = torch.zeros(4, 16, device="cuda"), torch.zeros(8, 16, dtype=BF16, device="cuda")
    slots, w, rows = torch.zeros(4, 2, dtype=i32, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(8, dtype=i32, device="cuda")
    _, dw = ts.combine_rows_backward(dy, src[:0], slots, w, rows[:0])
    assert (dw == 0).all()
    assert ts.combine_rows_backward(dy[:0], src, slots[:0], w[:0], rows)[1].shape == (0, 2)
    for error, call in (
        (ValueError, lambda: ts.combine_rows_backward(dy[:3], src, slots, w, rows)), (ValueError, lambda: ts.combine_rows_backward(dy[:, :8], src, slots, w, rows)),
        (TypeError, lambda: ts.combine_rows_backward(dy, src.half(), slots, w, rows)), (ValueError, lambda: ts.combine_rows_backward(dy, src, slots, w, rows[:7])),
        (ValueError, lambda: ts.combine_rows_backward(dy, src, slots, w[:, :1], rows)), (TypeError, lambda: ts.combine_rows_backward(dy, src, slots, w, rows, dsrc=dy)),
        (ts.TsError, lambda: ts.combine_rows_backward(dy, src, slots, w, rows, dsrc=src)),
        (ts.TsError, lambda: ts.combine_rows_backward(dy, src, torch.zeros(4, 9, dtype=i32, device="cuda"), torch.zeros(4, 9, device="cuda"), rows)),
    ):
        with pytest.raises(error):
            call()


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
class Layer:
    """A layer of routed experts with an adapter for each on its gate, up and down products, tuned through the library."""

    def __init__(self, ts, d, m, experts, top_k, r, tokens, seed):
        g = gen(seed)
        self.ts, self.top_k, self.e, self.r = ts, top_k, experts, r
        self.w = {"gate": randn(g, experts, m, d) / math.sqrt(d), "up": randn(g, experts, m, d) / math.sqrt(d),
                  "down": randn(g, experts, m, d) / math.sqrt(m)}
        self.w = {v: t.to(BF16) for v, t in self.w.items()}
        self.ad = {}
        for v, (i, o) in {"gate": (d, m), "up": (d, m), "down": (m, d)}.items():
            a, b = (randn(g, experts, r, i) / math.sqrt(i)).to(BF16), (0.3 * randn(g, experts, r, o)).to(BF16)
            self.ad[v] = ts.Adapters(a, b, scale=torch.full((experts,), 0.5, device="cuda"))
        self.logits, self.x = randn(g, tokens, experts), randn(g, tokens, d).to(BF16)
        self.logits[3] = -math.inf
        self.dy, self.dloss = 0.1 * randn(g, tokens, d), torch.tensor([5.0], device="cuda")
        n = tokens * top_k
        self.fwd = {"gate": ts.Grouped(self.w["gate"], max_rows=n), "up": ts.Grouped(self.w["up"], max_rows=n),
                    "down": ts.Grouped(self.w["down"], layout="kn", max_rows=n)}
        self.bwd = {"gate": ts.Grouped(self.w["gate"], layout="kn", max_rows=n), "up": ts.Grouped(self.w["up"], layout="kn", max_rows=n),
                    "down": ts.Grouped(self.w["down"], max_rows=n)}

    def step(self):
        ts, x = self.ts, self.x
        n = x.shape[0] * self.top_k
        r = ts.route(self.logits, self.top_k, rows=torch.full((n,), -1, dtype=torch.int32, device="cuda"))
        used = r.offsets[-1:]
        rows_x = ts.gather_rows(x, r.rows, n=used, out=torch.zeros(n, x.shape[1], dtype=BF16, device="cuda"))
        q, s = ts.quant_rows(x, r.rows, n=used)  # what is kept of x
        place = torch.arange(n, dtype=torch.int32, device="cuda")
        ids = torch.bucketize(place, r.offsets[1:], right=True).to(torch.int32)  # each row's expert; behind the last: none
        rows = self.ad["gate"].rows(ids)
        h = {v: torch.empty(n, self.r, device="cuda") for v in self.ad}
        pre = {}
        for v in ("gate", "up"):
            pre[v] = self.fwd[v].forward(rows_x, offsets=r.offsets)
            self.ad[v].forward(rows_x, pre[v], rows, h=h[v])
        c, kept = ts.drelu_rows(pre["gate"], pre["up"], n=used, keep=True)
        rows_y = self.fwd["down"].forward(c, offsets=r.offsets, y=torch.zeros(n, x.shape[1], device="cuda"))
        self.ad["down"].forward(c, rows_y, rows, h=h["down"])
        y = ts.combine_rows(rows_y, r.slots, r.w)
        bal = ts.balance(self.logits, r.sel)
        # back
        d_rows, dw = ts.combine_rows_backward(self.dy, rows_y, r.slots, r.w, r.rows)
        d_rows = d_rows.to(BF16)
        dc = self.bwd["down"].forward(d_rows, offsets=r.offsets)
        grads = {}
        again = torch.empty(n, c.shape[1], dtype=BF16, device="cuda")
        dg, du = (torch.empty_like(again) for _ in range(2))
        # the adapter's share of dc comes first: the activation's gradient is of their sum
        _, grads["a_down"], grads["b_down"] = self.ad["down"].backward(d_rows, dc, rows, h["down"], c)
        ts.drelu_rows_backward(dc, kept, n=used, dg=dg, du=du, c=again)
        dx_rows = self.bwd["gate"].forward(dg, offsets=r.offsets, y=torch.zeros(n, x.shape[1], device="cuda"))
        dx_up = self.bwd["up"].forward(du, offsets=r.offsets, y=torch.zeros(n, x.shape[1], device="cuda"))
        for v, d, dx in (("gate", dg, dx_rows), ("up", du, dx_up)):
            _, grads["a_" + v], grads["b_" + v] = self.ad[v].backward(d, dx, rows, h[v], q, x_scale=s)
        dx = ts.combine_rows(dx_rows.add_(dx_up), r.slots, torch.ones_like(r.w))
        dlogits = ts.route_backward(self.logits, r.sel, r.w, dw=dw, balance=bal, dloss=self.dloss)
        return {"y": y, "loss": bal.loss, "x": dx, "logits": dlogits, **grads}

    def exact(self):
        """The same by automatic differentiation in 64 bits."""
        leaves = {"x": self.x.double(), "logits": self.logits.double()}
        for v, ad in self.ad.items():
            leaves["a_" + v], leaves["b_" + v] = ad.a.double(), ad.b.double()
        leaves = {n: t.requires_grad_() for n, t in leaves.items()}
        w = {v: t.double() for v, t in self.w.items()}
        logits, x = leaves["logits"], leaves["x"]
        live = torch.isfinite(self.logits).any(1)
        v, sel = torch.topk(logits[live], self.top_k, dim=1)
        weight = torch.softmax(v, 1)
        y = torch.zeros_like(x)
        index = torch.nonzero(live)[:, 0]
        for e in range(self.e):
            def low_rank(v, t):
                return 0.5 * t @ leaves["a_" + v][e].t() @ leaves["b_" + v][e]

            i, j = torch.nonzero(sel == e, as_tuple=True)
            t = x[index[i]]
            g, u = t @ w["gate"][e].t() + low_rank("gate", t), t @ w["up"][e].t() + low_rank("up", t)
            c = torch.relu(g) * torch.relu(u)
            out = c @ w["down"][e] + low_rank("down", c)
            y = y.index_add(0, index[i], weight[i, j][:, None] * out)
        counts = torch.bincount(sel.reshape(-1), minlength=self.e).double()
        loss = self.e * (counts / counts.sum() * torch.softmax(logits[live], 1).mean(0)).sum()
        total = (y * self.dy.double()).sum() + float(self.dloss) * loss
        grads = torch.autograd.grad(total, list(leaves.values()))
        return {"y": y.detach(), "loss": loss.detach().view(1), **dict(zip(leaves, grads))}


@pytest.mark.parametrize("d,m,experts,top_k,r,tokens", [(256, 512, 4, 2, 8, 100), (512, 1408, 8, 2, 16, 300)])
def test_a_tuning_step(ts, d, m, experts, top_k, r, tokens):
    """Relative in 2-norm. y: rounded to bf16 are g and u (after each of two sums), c, 2^-8 each of a value at most, some
    terms cancelling: 2^-6. Gradients meet those, d_rows, dc and dg in bf16 as well, and the kept factors, up to 2^-4 of each
    number (2^-4 / sqrt(3) or less of a norm, errors in turn of either sign): 2^-4. What the router gets is of y's kind."""
    layer = Layer(ts, d, m, experts, top_k, r, tokens, seed=d)
    got, want = layer.step(), layer.exact()
    for name, v in want.items():
        err = float((got[name].double() - v).norm() / v.norm())
        tol = {"y": 2.0 ** -6, "logits": 2.0 ** -6, "loss": 2.0 ** -20}.get(name, 2.0 ** -4)
        assert err <= tol, (name, err)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = layer.step()
    layer.x.copy_(layer.x.roll(1, 0))
    layer.logits.copy_(layer.logits.roll(1, 0))
    graph.replay()
    again = layer.step()
    assert all(torch.equal(out[v], again[v]) for v in out)


def test_decoding_with_adapters(ts):
    """A few tokens of requests with adapters of their own through one layer, beside its frozen weights."""
    t, d, m, r, n = 9, 512, 1408, 16, 5
    g = gen(6)
    w = [(randn(g, m, d) / math.sqrt(d)).to(BF16) for _ in range(2)] + [(randn(g, m, d) / math.sqrt(m)).to(BF16)]
    x = randn(g, t, d).to(BF16)
    ids = torch.tensor([0, 3, -1, 3, 4, 0, 0, -1, 2], dtype=torch.int32, device="cuda")
    mats = [((randn(g, n, r, i) / math.sqrt(i)).to(BF16), (0.3 * randn(g, n, r, o)).to(BF16)) for i, o in ((d, m), (d, m), (m, d))]
    ads = [ts.Adapters(a, b) for a, b in mats]
    gate, up, down = ts.Grouped(w[0], max_rows=t), ts.Grouped(w[1], max_rows=t), ts.Grouped(w[2], layout="kn", max_rows=t)
    pg, pu = gate.forward(x), up.forward(x)
    ads[0].forward(x, pg, ids)
    ads[1].forward(x, pu, ids)
    c = ts.drelu_rows(pg, pu)
    y = down.forward(c, y=torch.empty(t, d, device="cuda"))
    ads[2].forward(c, y, ids)
    base = ts.Prompt(ts.Experts(*w), t)(x)

    def low_rank(i, v):
        a, b = (p[ids.clamp(min=0).long()].double() for p in mats[i])
        return torch.where((ids >= 0)[:, None], torch.einsum("tr,trn->tn", torch.einsum("tk,trk->tr", v, a), b), 0.0)

    v = x.double()
    c64 = torch.relu(v @ w[0].double().t() + low_rank(0, v)) * torch.relu(v @ w[1].double().t() + low_rank(1, v))
    want = c64 @ w[2].double() + low_rank(2, c64)
    err = (y.double() - want).norm(dim=1) / want.norm(dim=1)
    assert (err <= 2.0 ** -6).all()  # g, u and c in bf16, as in the tuning step
    none = ids < 0
    # without an adapter, the library's own layer: the same but for g and u in bf16 before their product
    assert ((y[none] - base[none]).norm(dim=1) <= 2.0 ** -6 * base[none].norm(dim=1)).all()
