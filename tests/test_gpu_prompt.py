"""Whole layers of experts over many tokens (ts_experts_*, ts_prompt_*): against the operators called one at a time
(the same bits), against the formula in 64 bits, and against the layer's forward of a few tokens.

Tolerance of a bf16 layer, per output, by arithmetic: with S the same sum over magnitudes, a product of k terms in fp32 is
off by at most (k 2^-24 + 2^-20) S (see test_gpu_grouped.py); c = g u carries each factor's error times the other and
half a step of bf16, 2^-8 of it; the down product multiplies those errors by |W_down| and adds its own; a sum of at most
8 weighted rows, whose weights are off by at most 2^-20, adds 2^-19 of sum |w y|.
"""
import numpy as np
import pytest
import torch

from paper_2406_05955_gb300 import workload as wl

pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn


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


def quant_weights(w):
    """e4m3 values and a scale for each 128 x 128 of [n][k]."""
    n, k = w.shape
    nb, kb = -(-n // 128), -(-k // 128)
    p = torch.zeros(nb * 128, kb * 128, device=w.device)
    p[:n, :k] = w.float()
    p = p.view(nb, 128, kb, 128)
    s = p.abs().amax(dim=(1, 3)) / 448
    q = (p / s[:, None, :, None]).clamp(-448, 448).view(nb * 128, kb * 128)[:n, :k]
    return q.contiguous().to(E4M3), s


def wide(q, s):
    n, k = q.shape
    return q.double() * s.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]


class Layer:
    """Weights of `e` experts in 64 bits and an Experts handle over them."""

    def __init__(self, ts, e, d, m, k, seed, e8=False, router=True):
        ls = [wl.ffn_layer(d, m, activation=0.25, dtype=BF16, seed=wl.layer_seed(seed, 0, i)) for i in range(e)]
        self.bf16 = [[t.cuda() for t in (L.w_gate, L.w_up, L.w_down)] for L in ls]
        self.router = wl.router(e, d, seed=seed).cuda() if router else None
        self.k, self.e8 = k, e8
        if e8:
            q = [[quant_weights(g), quant_weights(u), quant_weights(dn.t())] for g, u, dn in self.bf16]
            self.q = q
            self.experts = ts.Experts([a[0][0] for a in q], [a[1][0] for a in q], [a[2][0] for a in q], self.router, k,
                                      [a[0][1] for a in q], [a[1][1] for a in q], [a[2][1] for a in q])
            self.wd = [[wide(*a[0]), wide(*a[1]), wide(*a[2]).t()] for a in q]
        else:
            self.experts = ts.Experts(*[[w[i] for w in self.bf16] for i in range(3)], w_router=self.router, top_k=k)
            self.wd = [[t.double() for t in w] for w in self.bf16]

    def chain(self, ts, x):
        """The same with the operators one at a time."""
        t, e = x.shape[0], len(self.bf16)
        n = t * (self.k if self.router is not None else 1)
        if self.router is not None:
            logits = torch.empty(t, e, device="cuda")
            r = ts.route(ts.Grouped(self.router, max_rows=t).forward(x, y=logits), self.k)
            off, rows, cnt = r.offsets, r.rows, r.offsets[-1:]
        else:
            off = rows = cnt = None
        if self.e8:
            q = self.q
            xq, xs = ts.quant_rows(x, rows=rows, n=cnt)
            gu = ts.Grouped.gated([a[0][0] for a in q], [a[1][0] for a in q], scale_gate=[a[0][1] for a in q],
                                  scale_up=[a[1][1] for a in q], max_rows=n)
            cq, cs = ts.quant_rows(gu.forward(xq, off, xs), n=cnt)
            dn = ts.Grouped([a[2][0] for a in q], scale=[a[2][1] for a in q], max_rows=n)
            y = dn.forward(cq, off, cs, torch.empty(n, x.shape[1], device="cuda"))
        else:
            xr = x if rows is None else ts.gather_rows(x, rows, n=cnt)
            gu = ts.Grouped.gated([w[0] for w in self.bf16], [w[1] for w in self.bf16], max_rows=n)
            dn = ts.Grouped([w[2] for w in self.bf16], layout="kn", max_rows=n)
            y = dn.forward(gu.forward(xr, off), off, None, torch.empty(n, x.shape[1], device="cuda"))
        return y if rows is None else ts.combine_rows(y, r.slots, r.w)

    def exact(self, x, sel=None, w=None):
        """y in 64 bits and its bound, with the given picks."""
        xd = x.double()
        t, d = x.shape
        eps = lambda k: k * 2.0 ** -24 + 2.0 ** -20  # noqa: E731
        y, tol, mag = (torch.zeros(t, d, dtype=torch.float64, device="cuda") for _ in range(3))
        for e, (wg, wu, wd) in enumerate(self.wd):
            if sel is None:
                rows, weight = torch.arange(t, device="cuda"), torch.ones(t, dtype=torch.float64, device="cuda")
            else:
                rows, j = torch.nonzero(sel == e, as_tuple=True)
                weight = w[rows, j]
            xe = xd[rows]
            g, u = xe @ wg.t(), xe @ wu.t()
            eg, eu = eps(d) * (xe.abs() @ wg.abs().t()), eps(d) * (xe.abs() @ wu.abs().t())
            c = g.clamp(min=0) * u.clamp(min=0)
            ec = eg * u.abs() + eu * g.abs() + eg * eu
            ec = ec + 2.0 ** -8 * (c + ec)
            s = (c + ec) @ wd.abs()
            y[rows] += weight[:, None] * (c @ wd)
            tol[rows] += weight[:, None] * (ec @ wd.abs() + eps(wd.shape[0]) * s)
            mag[rows] += weight[:, None] * s
        return y, tol + 2.0 ** -19 * mag


def check_routing(layer, x, sel, w):
    """The picks equal those of 64-bit logits but for near ties, their weights the softmax over them."""
    logits = x.double() @ layer.router.double().t()
    k = layer.k
    top = torch.sort(logits, dim=1, descending=True, stable=True)
    want = top.indices[:, :k]
    sel = torch.from_numpy(sel).cuda().long()
    w = torch.from_numpy(w).cuda().double()
    v = top.values
    near = ((v[:, :k] - v[:, 1:k + 1]) < 1e-4).any(1) if v.shape[1] > k else ((v[:, :k - 1] - v[:, 1:k]) < 1e-4).any(1)
    assert (sel == want)[~near].all()
    p = torch.softmax(logits.gather(1, sel), 1)
    assert ((w - p).abs() <= 1e-5 * p + 1e-7).all()
    return sel, w


@pytest.mark.parametrize("tokens", [1, 7, 64, 333])
@pytest.mark.parametrize("e,k", [(8, 2), (5, 3), (4, 1), (60, 4)])
def test_bf16_experts(ts, tokens, e, k):
    d, m = 256, 392
    layer = Layer(ts, e, d, m, k, seed=tokens + e)
    p = ts.Prompt(layer.experts, tokens + 3)
    x = wl.tokens(tokens, d, seed=tokens).cuda()
    y = p(x)
    assert torch.equal(y, layer.chain(ts, x)), "the layer is its operators in a row"
    sel, w = check_routing(layer, x, *p.get_routing())
    want, tol = layer.exact(x, sel, w)
    assert ((y.double() - want).abs() <= tol).all()
    assert p.get_error() == 0 and p.check_scratch() == 0


@pytest.mark.parametrize("tokens", [1, 100, 300])
@pytest.mark.parametrize("e,k", [(8, 2), (3, 3)])
def test_e4m3_experts(ts, tokens, e, k):
    """x and c are off by at most 2^-4 of each value: 2^-4 + 2^-4 of the 2-norm, and what the products add."""
    d, m = 384, 400
    layer = Layer(ts, e, d, m, k, seed=tokens + e, e8=True)
    p = ts.Prompt(layer.experts, tokens)
    x = wl.tokens(tokens, d, seed=tokens).cuda()
    y = p(x)
    assert torch.equal(y, layer.chain(ts, x))
    want, _ = layer.exact(x, *check_routing(layer, x, *p.get_routing()))
    assert float((y.double() - want).norm() / want.norm()) <= 2.0 ** -3 + 2.0 ** -7
    assert p.get_error() == 0 and p.check_scratch() == 0


@pytest.mark.parametrize("e8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("tokens", [1, 50, 700])
def test_single_ffn(ts, tokens, e8):
    d, m = 512, 1408
    layer = Layer(ts, 1, d, m, 1, seed=tokens, e8=e8, router=False)
    p = ts.Prompt(layer.experts, tokens)
    x = wl.tokens(tokens, d, seed=tokens).cuda()
    y = p(x)
    assert torch.equal(y, layer.chain(ts, x))
    want, tol = layer.exact(x)
    if e8:
        assert float((y.double() - want).norm() / want.norm()) <= 2.0 ** -3 + 2.0 ** -7
    else:
        assert ((y.double() - want).abs() <= tol).all()
    with pytest.raises(ts.TsError):
        p.get_routing()


def test_routing_has_the_tokens_of_the_last_forward(ts):
    """None after a forward of no tokens: nothing is written behind a caller's buffers of that size."""
    import ctypes

    layer = Layer(ts, 8, 128, 128, 2, seed=2)
    p = ts.Prompt(layer.experts, 40)
    with pytest.raises(ts.TsError):
        p.get_routing()
    x = wl.tokens(40, 128, seed=2).cuda()
    for t in (40, 0, 3, 0, 17):
        p(x[:t])
        sel, w = (torch.full((80,), -77, dtype=d) for d in (torch.int32, torch.float32))
        status = ts.lib().ts_prompt_get_routing(p.handle, None, *(ctypes.c_void_p(v.data_ptr()) for v in (sel, w)))
        assert status == 0
        assert (sel[2 * t:] == -77).all() and (w[2 * t:] == -77).all(), "written behind the last forward's tokens"
        got = p.get_routing()
        assert got[0].shape == got[1].shape == (t, 2)
        assert np.array_equal(got[0].reshape(-1), sel[:2 * t].numpy()) and (got[0] >= 0).all()
    with pytest.raises(ts.TsError):
        p(torch.cat([x, x]))                     # refused: the forward before it is still the last one
    assert p.get_routing()[0].shape == (17, 2)


def test_routing_of_captured_and_replayed_forwards(ts):
    """That of the forward that ran last, or a refusal; never a mixture of two."""
    layer = Layer(ts, 8, 128, 128, 2, seed=7)
    p = ts.Prompt(layer.experts, 300)
    x = wl.tokens(300, 128, seed=7).cuda()
    p(x[:30])
    long, _ = p.get_routing()
    few, y = x[30:34].clone(), torch.zeros(4, 128, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        p.forward(few, y=y)
    with pytest.raises(ts.TsError):
        p.get_routing()                          # not replayed yet
    graph.replay()
    got, _ = p.get_routing()
    assert got.shape == (4, 2)
    p(few)
    assert np.array_equal(p.get_routing()[0], got)
    few.copy_(x[:4])
    graph.replay()                               # as many tokens as the last call had
    assert np.array_equal(p.get_routing()[0], long[:4])
    for t in (30, 300):                          # (few and many tokens are routed by one and by two kernels)
        p(x[:t])
        assert np.array_equal(p.get_routing()[0][:30], long)
        graph.replay()
        with pytest.raises(ts.TsError):
            p.get_routing()


def test_same_as_the_layers_of_few_tokens(ts):
    """Experts.of(Moe) and Experts.of(Ffn) over the tokens that those layers take; c alone is rounded differently."""
    d, m, e = 512, 1024, 8
    layer = Layer(ts, e, d, m, 2, seed=3)
    ffns = [ts.Ffn(*w, max_batch=8) for w in layer.bf16]
    moe = ts.Moe(layer.router, ffns, top_k=2, max_batch=8)
    x = wl.tokens(8, d, seed=4).cuda()
    p = ts.Prompt(ts.Experts.of(moe), 8)
    y, few = p(x), moe.forward(x)
    sel, _ = p.get_routing()
    assert np.array_equal(sel, moe.get_routing(8)[0])
    assert float((y - few).norm() / few.norm()) <= 2.0 ** -8
    one = ts.Prompt(ts.Experts.of(ffns[0]), 8)
    y, few = one(x), ffns[0].forward(x)
    assert float((y - few).norm() / few.norm()) <= 2.0 ** -8


def test_layers_share_scratch_on_a_stream_and_in_a_graph(ts):
    d, m, t = 256, 512, 200
    layers = [Layer(ts, e, d, m, k, seed=e) for e, k in ((8, 2), (4, 2), (6, 1))]
    p = ts.Prompt(layers[0].experts, t)
    x = wl.tokens(t, d, seed=1).cuda()
    want = [layer.chain(ts, x) for layer in layers]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [p.forward(x, layer.experts, stream=side) for layer in layers]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ys = [torch.zeros(t, d, device="cuda") for _ in layers]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for layer, y in zip(layers, ys):
            p.forward(x, layer.experts, y=y)
    x.copy_(wl.tokens(t, d, seed=2).cuda())
    for _ in range(2):
        graph.replay()
    want = [layer.chain(ts, x) for layer in layers]
    assert all(torch.equal(a, b) for a, b in zip(ys, want))
    assert p.get_error() == 0 and p.check_scratch() == 0


@pytest.mark.parametrize("e8", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("t", [1, 40, 700])
def test_calls_wait_for_what_is_before_them(ts, t, e8):
    """Inputs that long work writes just before a call, overwritten just after it; also in a graph whose stream joins
    another one before the call."""
    d, m = 256, 512
    layer = Layer(ts, 8, d, m, 2, seed=5, e8=e8)
    p = ts.Prompt(layer.experts, t)
    xs = [wl.tokens(t, d, seed=s).cuda() for s in range(4)]
    want = [p.forward(x).clone() for x in xs]
    big = torch.randn(4096, 4096, device="cuda")
    side, other = torch.cuda.Stream(), torch.cuda.Stream()

    def step(x, x_in, y, out):
        a = big @ big                              # holds the next copy up
        x_in.copy_(x + (a[0, 0] * 0).to(x.dtype))
        p.forward(x_in, y=y)
        x_in.fill_(float("nan"))
        out.copy_(y)
        y.fill_(float("nan"))

    x_in, y = torch.empty_like(xs[0]), torch.empty_like(want[0])
    got = [torch.empty_like(y) for _ in xs]
    for _ in range(3):
        for x, out in zip(xs, got):
            step(x, x_in, y, out)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for x, out in zip(xs, got):
            other.wait_stream(side)
            with torch.cuda.stream(other):
                x_in.copy_(x)
            side.wait_stream(other)                # the call comes after two things
            p.forward(x_in, y=out)
            p.forward(x_in, y=y)                   # and after another call
    for out in got:
        out.zero_()
    for _ in range(3):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(y, want[-1]) and p.get_error() == 0


def test_two_forwards_at_once(ts):
    """One layer through two scratches, and a layer of few tokens, on three streams at once."""
    d, m = 256, 1024
    layer = Layer(ts, 8, d, m, 2, seed=6)
    sizes = (37, 600)
    ps = [ts.Prompt(layer.experts, t) for t in sizes]
    xs = [wl.tokens(t, d, seed=t).cuda() for t in sizes]
    g = torch.Generator(device="cuda").manual_seed(3)
    w = [(torch.randn(m, d, generator=g, device="cuda") / 16).to(torch.bfloat16) for _ in range(3)]
    few = ts.Ffn(*w)
    want = [p.forward(x).clone() for p, x in zip(ps, xs)] + [few.forward(xs[0][:1]).clone()]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    ys = [[torch.empty_like(v) for _ in range(20)] for v in want]
    for i in range(20):
        for p, x, y, st in zip(ps, xs, ys, streams):
            p.forward(x, y=y[i], stream=st)
        ys[2][i] = few.forward(xs[0][:1], stream=streams[2])
    torch.cuda.synchronize()
    for y, v in zip(ys, want):
        assert all(torch.equal(a, v) for a in y)
    assert all(p.get_error() == 0 and p.check_scratch() == 0 for p in ps)


@pytest.mark.parametrize("what", ["grouped", "experts", "prompt", "ffn"])
def test_a_handle_is_destroyed_during_a_capture(ts, what):
    """As a garbage collection may do at any time: the capture goes on."""
    w = torch.randn(64, 64, device="cuda").to(torch.bfloat16)
    experts = ts.Experts(w, w, w)
    other = {"grouped": ts.Grouped(w), "experts": ts.Experts(w, w, w), "prompt": ts.Prompt(experts, 4),
             "ffn": ts.Ffn(w, w, w)}[what]
    p, x, y = ts.Prompt(experts, 8), torch.randn(8, 64, device="cuda").to(torch.bfloat16), torch.zeros(8, 64, device="cuda")
    want = p.forward(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        p.forward(x, y=y)
        other.close()
    graph.replay()
    assert torch.equal(y, want) and p.get_error() == 0 and p.check_scratch() == 0


@pytest.mark.parametrize("e8", [False, True], ids=["bf16", "e4m3"])
def test_tokens_without_an_expert_give_zero(ts, e8):
    """Padding whose router logits are NaN: no expert, y = 0; the other tokens as without it."""
    d, m, t = 256, 256, 90
    layer = Layer(ts, 4, d, m, 2, seed=9, e8=e8)
    p = ts.Prompt(layer.experts, t)
    x = wl.tokens(t, d, seed=9).cuda()
    y = p(x).clone()
    pad = torch.arange(0, t, 3, device="cuda")
    z = x.clone()
    z[pad] = float("nan")
    got = p(z)
    keep = torch.ones(t, dtype=torch.bool, device="cuda")
    keep[pad] = False
    assert (got[pad] == 0).all()
    assert (p.get_routing()[0][pad.cpu().numpy()] == -1).all()
    assert torch.allclose(got[keep], y[keep], rtol=1e-4, atol=1e-4 * float(y.abs().max()))  # other tiles, other sums
    z[:] = float("nan")
    assert (p(z) == 0).all()
    assert p.get_error() == 0


def test_layer_sizes(ts):
    """d = 4096, m = 14336, 2 of 8 experts."""
    layer = Layer(ts, 8, 4096, 14336, 2, seed=77)
    p = ts.Prompt(layer.experts, 150)
    x = wl.tokens(150, 4096, seed=78).cuda()
    y = p(x)
    want, tol = layer.exact(x, *check_routing(layer, x, *p.get_routing()))
    assert ((y.double() - want).abs() <= tol).all()
    assert float((y.double() - want).norm() / want.norm()) <= 2.0 ** -8


def test_e4m3_layer_sizes(ts):
    """d = 4096, m = 14336, 2 of 4 experts: few rows, and enough of them to be the MMA's M. (Bound: test_e4m3_experts.)"""
    layer = Layer(ts, 4, 4096, 14336, 2, seed=78, e8=True)
    p = ts.Prompt(layer.experts, 600)
    for tokens in (3, 600):
        x = wl.tokens(tokens, 4096, seed=79).cuda()
        y = p(x)
        want, _ = layer.exact(x, *check_routing(layer, x, *p.get_routing()))
        assert float((y.double() - want).norm() / want.norm()) <= 2.0 ** -3 + 2.0 ** -7
        assert p.get_error() == 0 and p.check_scratch() == 0


def test_refusals(ts):
    layer = Layer(ts, 4, 128, 128, 2, seed=1)
    p = ts.Prompt(layer.experts, 10)
    x = wl.tokens(10, 128, seed=1).cuda()
    other = Layer(ts, 4, 128, 256, 2, seed=1)
    more = Layer(ts, 5, 128, 128, 2, seed=1)
    w = layer.bf16[0]
    for call in (
        lambda: p(torch.cat([x, x])), lambda: p(x[:, :64].contiguous()), lambda: p.forward(x, other.experts),
        lambda: p.forward(x, more.experts), lambda: p.forward(x, y=torch.zeros(9, 128, device="cuda")),
        lambda: ts.Prompt(layer.experts, 0), lambda: ts.Experts(w[0], w[1], w[2][:64]),
        lambda: ts.Experts([w[0]] * 2, [w[1]] * 2, [w[2]] * 2),             # no router
        lambda: ts.Experts([w[0]] * 2, [w[1]] * 2, [w[2]] * 2, layer.router[:2].contiguous(), top_k=3),
        lambda: ts.Experts(w[0], w[1], w[2], scale_gate=torch.ones(1, 1, device="cuda")),
        lambda: ts.Experts(w[0].to(E4M3), w[1].to(E4M3), w[2].to(E4M3)),
    ):
        with pytest.raises((ValueError, ts.TsError)):
            call()
    for call in (lambda: p(x.float()), lambda: p(x.cpu()), lambda: ts.Experts(*[t.float() for t in w]),
                 lambda: ts.Experts.of(layer)):
        with pytest.raises(TypeError):
            call()
    assert p(x[:0]).shape == (0, 128)
    p.close()
    with pytest.raises(RuntimeError):
        p(x)
