"""Operators of a layer of experts that is adapted: what serving and tuning it needs beside its frozen weights, as cases.

`adapt` adds each row's share of a low-rank adapter, one of many, to a product of shared weights; `tune` is the same
with its backward pass (gradients of the rows and of the adapters, from rows kept in bf16 or in 8 bits); `drelu` is the
gated activation of a layer whose two products are computed apart, which keeps what its backward pass needs in 8 bits,
and that pass; `balance` is the loss on uneven routing with the experts' counts, and the gradient of the router's
logits; `uncombine` is the backward pass of the sum of each token's rows.

Sizes are those of this library's layers (d = 4096, m = 14336, 2 of 8 experts; d = 512, m = 1408) and generic ones
around them.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "f32": F32}
SIZE = {"bf16": 2, "f32": 4}
BLOCK = 128      # elements of one scale
LARGEST = 448.0  # of e4m3
FEW = 64         # rows of a decoding batch: the plain form takes each row's own matrices


def listed():
    return [
        # one decoding token beside a layer's gate product: all latency
        {"name": "adapt_t1", "kind": "adapt", "rows": 1, "k": 4096, "n": 14336, "r": 16, "adapters": 8, "out": "bf16",
         "none": 0.0, "ragged": False},
        # a full decoding batch of as many requests, some of which have no adapter
        {"name": "adapt_t64", "kind": "adapt", "rows": 64, "k": 4096, "n": 4096, "r": 16, "adapters": 64, "out": "f32",
         "none": 0.1, "ragged": False},
        # a larger batch over a small layer's down product, odd sizes
        {"name": "adapt_t300", "kind": "adapt", "rows": 300, "k": 1408, "n": 512, "r": 40, "adapters": 20, "out": "f32",
         "none": 0.0, "ragged": False},
        # prompts of several requests at once, ranks of up to 64
        {"name": "adapt_t8192", "kind": "adapt", "rows": 8192, "k": 4096, "n": 14336, "r": 64, "adapters": 6,
         "out": "bf16", "none": 0.05, "ragged": True},
        # a tuning step on a small layer, odd sizes
        {"name": "tune_t1000", "kind": "tune", "rows": 1000, "k": 512, "n": 1408, "r": 12, "adapters": 3, "out": "f32",
         "none": 0.0, "ragged": False, "x8": False},
        # a tuning step of 8 experts' adapters over a long batch, its rows kept in 8 bits
        {"name": "tune_t8192", "kind": "tune", "rows": 8192, "k": 4096, "n": 4096, "r": 32, "adapters": 8,
         "out": "bf16", "none": 0.0, "ragged": False, "x8": True},
        # the activation of a decoding batch, and of a long batch of routed rows
        {"name": "drelu_t16", "kind": "drelu", "type": "bf16", "rows": 16, "m": 14336, "unused": 0, "bias": -0.662},
        {"name": "drelu_t4096", "kind": "drelu", "type": "bf16", "rows": 8192, "m": 14336, "unused": 100, "bias": -0.662},
        # routing of a few hundred tokens over few experts, and of a long batch over many, an eighth of it padding
        {"name": "balance_t512", "kind": "balance", "tokens": 512, "experts": 8, "top_k": 2, "pad": 0},
        {"name": "balance_t8192_e64", "kind": "balance", "tokens": 8192, "experts": 64, "top_k": 6, "pad": 1024},
        # gradients of a few tokens' rows, and of a long batch's
        {"name": "uncombine_t32", "kind": "uncombine", "dy": "f32", "type": "bf16", "n": 4096, "tokens": 32, "top_k": 2,
         "none": 0.0},
        {"name": "uncombine_t4096", "kind": "uncombine", "dy": "f32", "type": "bf16", "n": 4096, "tokens": 4096,
         "top_k": 2, "none": 0.05},
    ]


def _log_int(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(["adapt", "adapt", "adapt", "tune", "tune", "drelu", "balance", "uncombine"])
    if kind in ("adapt", "tune"):
        c = {"kind": kind, "rows": _log_int(rng, 1, 8192), "k": _log_int(rng, 256, 14336, 8),
             "n": _log_int(rng, 256, 14336, 8), "r": rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 64)]),
             "adapters": _log_int(rng, 1, 128), "out": rng.choice(["bf16", "f32"]), "none": rng.choice([0.0, 0.0, 0.3]),
             "ragged": rng.random() < 0.4}
        while c["rows"] * (c["k"] + c["n"] * SIZE[c["out"]]) > 8192 * (4096 + 2 * 4096):
            c["rows"] = c["rows"] * 2 // 3
        if kind == "tune":
            c["k"] = (c["k"] + 8) // 16 * 16
            c["x8"] = rng.random() < 0.5
            while c["adapters"] > 1 and c["adapters"] * c["r"] * (c["k"] + c["n"]) > 8 * 32 * 2 * 8192:
                c["adapters"] //= 2
        return c
    if kind == "drelu":
        m = _log_int(rng, 256, 14336, 16)
        rows = _log_int(rng, 1, min(16384, 8192 * 14336 // m))
        return {"kind": kind, "type": rng.choice(["bf16", "bf16", "f32"]) if rows * m < 2 ** 25 else "bf16", "rows": rows,
                "m": m, "unused": rng.choice([0, 0, rows // 9]), "bias": rng.choice([-0.999, -0.662, 0.0, 0.55])}
    if kind == "balance":
        e = rng.choice([2, 4, 8, 8, 16, 60, 64, 128, 256])
        t = _log_int(rng, 1, 8192)
        return {"kind": kind, "tokens": t, "experts": e, "top_k": min(e, rng.randint(1, 8)), "pad": rng.choice([0, 0, t // 8])}
    t = _log_int(rng, 1, 8192)
    return {"kind": kind, "dy": rng.choice(["f32", "f32", "bf16"]), "type": rng.choice(["bf16", "bf16", "f32"]),
            "n": min(_log_int(rng, 256, 8192, 8), 4096 * 4096 // t // 8 * 8), "tokens": t, "top_k": rng.randint(1, 4),
            "none": rng.choice([0.0, 0.1])}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _activations(g, *shape):
    """Gaussian values with a few channels that are much larger than the rest, as a residual stream has them."""
    x = _randn(g, *shape)
    x[..., ::97] *= 6.0
    return x


def _round8_rows(x):
    """(values in e4m3, scales [k / 128][rows]) of activations [rows][k], as they were kept earlier."""
    r, k = x.shape
    kb = -(-k // BLOCK)
    p = torch.zeros(r, kb * BLOCK, device=DEV)
    p[:, :k] = x
    p = p.view(r, kb, BLOCK)
    s = p.abs().amax(dim=2) / LARGEST
    s = torch.where(s > 0, s, torch.ones_like(s))
    q = (p / s[..., None]).clamp(-LARGEST, LARGEST).view(r, kb * BLOCK)[:, :k].contiguous().to(E4M3)
    return q, s.t().contiguous()


def _routing(logits, k):
    """Picks and weights [tokens][k] of logits; a token of no finite logit has none."""
    top = torch.sort(logits, dim=1, descending=True, stable=True)
    v, i = top.values[:, :k], top.indices[:, :k]
    ok = v > -math.inf
    z = torch.where(ok, torch.exp(v - torch.where(ok[:, :1], v[:, :1], 0.0)), 0.0)
    return torch.where(ok, i, -1).to(torch.int32), z / torch.where(ok[:, :1], z.sum(1, keepdim=True), 1.0)


def _inputs(case, seed):
    """Everything that is drawn for a case, in one order."""
    g, kind = _gen(seed), case["kind"]
    if kind in ("adapt", "tune"):
        t, k, n, r, a = case["rows"], case["k"], case["n"], case["r"], case["adapters"]
        z = {"a": (_randn(g, a, r, k) / math.sqrt(k)).to(BF16), "b": (0.3 * _randn(g, a, r, n)).to(BF16),
             "scale": 16.0 / r * (1.0 + torch.rand(a, generator=g, device=DEV))}
        # some requests are longer than others; a prompt's rows lie together, a decoding batch's or an expert's do not
        ids = torch.multinomial(torch.softmax(0.7 * _randn(g, a), 0), t, replacement=True, generator=g)
        none = torch.rand(t, generator=g, device=DEV) < case["none"]
        ids = torch.where(none, -1, ids)
        z["ids"] = (torch.sort(ids).values if case["ragged"] else ids).to(torch.int32)
        z["x"] = _activations(g, t, k).to(BF16)
        z["y"] = _randn(g, t, n).to(TYPES[case["out"]])
        if kind == "tune":
            z["dy"] = (0.1 * _randn(g, t, n)).to(BF16)
            z["dx"] = (0.1 * _randn(g, t, k)).to(TYPES[case["out"]])
            z["x8"], z["x_scale"] = _round8_rows(z["x"].float()) if case["x8"] else (None, None)
        return z
    if kind == "drelu":
        r, m = case["rows"], case["m"]
        bias = case["bias"] + 0.5 * _randn(g, m)  # some neurons are active far more often than others
        z = {v: (_randn(g, r, m) + bias).to(TYPES[case["type"]]) for v in ("g", "u")}
        z["dc"] = (0.05 * _randn(g, r, m)).to(TYPES[case["type"]])
        z["n"] = torch.tensor([r - case["unused"]], dtype=torch.int32, device=DEV)
        return z
    if kind == "balance":
        t, e = case["tokens"], case["experts"]
        logits = _randn(g, t, e) + 0.7 * _randn(g, e)  # some experts are picked more often
        if case["pad"]:
            pad = torch.randperm(t, generator=g, device=DEV)[:case["pad"]]
            logits[pad] = -math.inf
        sel, w = _routing(logits, case["top_k"])
        return {"logits": logits, "sel": sel, "w": w, "dw": _randn(g, t, case["top_k"]),
                "dloss": torch.tensor([0.01 * t], device=DEV)}
    t, k, n = case["tokens"], case["top_k"], case["n"]
    z = {"src": _randn(g, t * k, n).to(TYPES[case["type"]]), "dy": (0.1 * _randn(g, t, n)).to(TYPES[case["dy"]])}
    slots = torch.randperm(t * k, generator=g, device=DEV).view(t, k)
    w = torch.softmax(_randn(g, t, k), dim=1)
    none = torch.rand(t, generator=g, device=DEV) < case["none"]  # padding: no expert has it
    rows = torch.full((t * k,), -1, dtype=torch.int64, device=DEV)
    rows[slots] = torch.where(none, -1, torch.arange(t, device=DEV))[:, None].expand(t, k)
    z["rows"] = rows.to(torch.int32)
    z["slots"] = torch.where(none[:, None], -1, slots).to(torch.int32)
    z["w"] = torch.where(none[:, None], 0.0, w)
    return z


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind in ("adapt", "tune"):
        t = case["rows"]
        s["out"] = torch.empty(t, case["n"], dtype=TYPES[case["out"]], device=DEV)
        if own:
            import paper_2406_05955_gb300 as ts
            s["ad"] = ts.Adapters(s["a"], s["b"], scale=s["scale"])
        elif t > FEW or kind == "tune":
            ids = s["ids"].tolist()
            lists = [[] for _ in range(case["adapters"])]
            for i, a in enumerate(ids):
                if a >= 0:
                    lists[a].append(i)
            s["lists"] = [torch.tensor(v, dtype=torch.int64, device=DEV) for v in lists]
        if kind == "tune":
            s["h"] = torch.empty(t, case["r"], device=DEV)
            s["dx_out"] = torch.empty(t, case["k"], dtype=TYPES[case["out"]], device=DEV)
            s["da"], s["db"] = torch.empty_like(s["a"], dtype=F32), torch.empty_like(s["b"], dtype=F32)
    elif kind == "drelu":
        r, m = case["rows"], case["m"]
        for v in ("c", "dg", "du", "c_again"):
            s[v] = torch.zeros(r, m, dtype=BF16, device=DEV)
        for v in ("q_gate", "q_up"):
            s[v] = torch.zeros(r, m, device=DEV, dtype=torch.uint8).view(E4M3)
        for v in ("s_gate", "s_up"):
            s[v] = torch.zeros(-(-m // BLOCK), r, device=DEV)
    elif kind == "uncombine":
        s["dsrc"] = torch.zeros_like(s["src"])
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_adapt(s):
    """(y and the adapters' share, in the type of y; h)."""
    case, x, y = s["case"], s["x"], s["y"].to(F32, copy=True)
    if "lists" not in s:  # each row times its own matrices
        some = s["ids"] >= 0
        i = s["ids"].clamp(min=0).long()
        scale = torch.where(some, s["scale"][i], 0.0)
        h = (x.float()[:, None] @ s["a"][i].float().transpose(1, 2)) * scale[:, None, None]
        return (y + (h @ s["b"][i].float())[:, 0]).to(TYPES[case["out"]]), h[:, 0]
    h = torch.zeros(case["rows"], case["r"], device=DEV)
    for i, rows in enumerate(s["lists"]):
        part = x[rows].float() @ s["a"][i].float().t() * s["scale"][i]
        h[rows] = part
        y[rows] += part @ s["b"][i].float()
    return y.to(TYPES[case["out"]]), h


def _plain_tune(s):
    case = s["case"]
    y, h = _plain_adapt(s)
    dx, dy = s["dx"].to(F32, copy=True), s["dy"].float()
    x = s["x"].float() if s["x8"] is None else \
        s["x8"].float() * s["x_scale"].repeat_interleave(BLOCK, 0)[:case["k"]].t()
    for i, rows in enumerate(s["lists"]):
        part = dy[rows]
        dh = part @ s["b"][i].float().t() * s["scale"][i]
        dx[rows] += dh @ s["a"][i].float()
        s["da"][i] = dh.t() @ x[rows]
        s["db"][i] = h[rows].t() @ part
    return {"y": y, "dx": dx.to(TYPES[case["out"]]), "da": s["da"], "db": s["db"]}


def _plain_keep(p):
    """(e4m3, scales [m / 128][rows]) of values that are not negative: powers of two, and no value becomes zero."""
    r, m = p.shape
    mb = -(-m // BLOCK)
    v = torch.nn.functional.pad(p, (0, mb * BLOCK - m)).view(r, mb, BLOCK)
    top = v.amax(2)
    part, e = torch.frexp(top)  # top = part * 2^e, and 448 = 0.875 * 2^9
    e = torch.where(part <= 0.875, e - 9, e - 8).clamp(min=-100)
    e = torch.where(top > 0, e, 0)
    scale, inverse = (((x + 127) << 23).to(torch.int32).view(F32) for x in (e, -e))
    q = (v * inverse[..., None]).to(E4M3)
    q = torch.where((v > 0) & (q.float() == 0), 2.0 ** -9, q.float())
    return q.view(r, mb * BLOCK)[:, :m], scale.t()


def _plain_drelu(s):
    case = s["case"]
    n, m = case["rows"] - case["unused"], case["m"]
    g, u = s["g"][:n].float(), s["u"][:n].float()
    both = (g > 0) & (u > 0)
    g, u = torch.where(both, g, 0.0), torch.where(both, u, 0.0)
    s["c"][:n] = (g * u).to(BF16)
    kept = []
    for v, q, scale in ((g, "q_gate", "s_gate"), (u, "q_up", "s_up")):
        wide, by_block = _plain_keep(v)
        s[q][:n], s[scale][:, :n] = wide.to(E4M3), by_block
        kept.append(s[q][:n].float() * s[scale][:, :n].repeat_interleave(BLOCK, 0)[:m].t())
    dc = s["dc"][:n].float()
    both = kept[0] > 0
    s["dg"][:n] = torch.where(both, dc * kept[1], 0.0).to(BF16)
    s["du"][:n] = torch.where(both, dc * kept[0], 0.0).to(BF16)
    s["c_again"][:n] = (kept[0] * kept[1]).to(BF16)
    return {v: s[v] for v in ("c", "q_gate", "q_up", "s_gate", "s_up", "dg", "du", "c_again")}


def _plain_balance(s):
    x, sel, w, dw = s["logits"], s["sel"], s["w"], s["dw"]
    e = x.shape[1]
    top = x.amax(1, keepdim=True)
    live = top > -math.inf
    z = torch.exp(x - torch.where(live, top, 0.0))
    p = z / torch.where(live, z.sum(1, keepdim=True), 1.0)
    counts = (sel.reshape(-1)[:, None] == torch.arange(e, device=DEV)).sum(0)
    tokens, picks = live.sum().clamp(min=1), counts.sum().clamp(min=1)
    share = p.double().sum(0) / tokens
    loss = e * (counts / picks.double() * share).sum()
    c = counts.float()
    d = s["dloss"] * (e / (picks.double() * tokens)).float() * p * (c - (p * c).sum(1, keepdim=True))
    picked = w * (dw - (w * dw).sum(1, keepdim=True))
    d.scatter_add_(1, sel.clamp(min=0).long(), torch.where(sel >= 0, picked, 0.0))
    return {"loss": loss.float().view(1), "counts": counts.to(torch.int32), "share": share.float(), "dlogits": d}


def _plain_uncombine(s):
    dy, slots, w = s["dy"].float(), s["slots"].long(), s["w"]
    some = slots >= 0
    dw = torch.stack([(dy * s["src"][slots[:, j].clamp(min=0)].float()).sum(1) for j in range(slots.shape[1])], 1)
    t, j = torch.nonzero(some, as_tuple=True)
    s["dsrc"][slots[t, j]] = (w[t, j][:, None] * dy[t]).to(s["dsrc"].dtype)
    return {"dsrc": s["dsrc"], "dw": torch.where(some, dw, 0.0)}


def run(s):
    kind = s["case"]["kind"]
    if not own:
        if kind == "adapt":
            return _plain_adapt(s)[0]
        return {"tune": _plain_tune, "drelu": _plain_drelu, "balance": _plain_balance, "uncombine": _plain_uncombine}[kind](s)
    import paper_2406_05955_gb300 as ts
    if kind == "adapt":
        return s["ad"].forward(s["x"], s["y"], s["ids"], out=s["out"])
    if kind == "tune":
        rows = s["ad"].rows(s["ids"])
        y = s["ad"].forward(s["x"], s["y"], rows, out=s["out"], h=s["h"])
        x, scale = (s["x"], None) if s["x8"] is None else (s["x8"], s["x_scale"])
        dx, da, db = s["ad"].backward(s["dy"], s["dx"], rows, s["h"], x, x_scale=scale, out=s["dx_out"], da=s["da"],
                                      db=s["db"])
        return {"y": y, "dx": dx, "da": da, "db": db}
    if kind == "drelu":
        kept = ts.Kept(s["q_gate"], s["q_up"], s["s_gate"], s["s_up"])
        c, kept = ts.drelu_rows(s["g"], s["u"], n=s["n"], c=s["c"], kept=kept)
        dg, du, again = ts.drelu_rows_backward(s["dc"], kept, n=s["n"], dg=s["dg"], du=s["du"], c=s["c_again"])
        return {"c": c, **kept._asdict(), "dg": dg, "du": du, "c_again": again}
    if kind == "balance":
        b = ts.balance(s["logits"], s["sel"])
        d = ts.route_backward(s["logits"], s["sel"], s["w"], dw=s["dw"], balance=b, dloss=s["dloss"])
        return {"loss": b.loss, "counts": b.counts, "share": b.share, "dlogits": d}
    dsrc, dw = ts.combine_rows_backward(s["dy"], s["src"], s["slots"], s["w"], s["rows"], dsrc=s["dsrc"])
    return {"dsrc": dsrc, "dw": dw}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind in ("adapt", "tune"):
        t, k, n, r, a = case["rows"], case["k"], case["n"], case["r"], case["adapters"]
        size = SIZE[case["out"]]
        live = t * (1.0 - case["none"])
        hit = a * (1.0 - (1.0 - 1.0 / a) ** live)  # adapters with a row at all
        b = 2 * live * k + 2 * t * n * size + 2 * hit * r * (k + n) + 4 * t
        flops = 2.0 * live * r * (k + n)
        if kind == "tune":
            b += live * (2 * n + (k + k / 32 if case["x8"] else 0)) + 2 * t * k * size + 4 * a * r * (k + n)
            flops *= 3
        return {"bytes": b, "flops": flops}
    if kind == "drelu":
        e, size = (case["rows"] - case["unused"]) * case["m"], SIZE[case["type"]]
        return {"bytes": e * (3 * size + 2 + 4 * 2 + 2 * 4 / BLOCK), "flops": 8 * e}
    if kind == "balance":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": 8 * t * e + 12 * t * k + 8 * e, "flops": 10 * t * e}
    t, k, n = case["tokens"], case["top_k"], case["n"]
    live = t * (1.0 - case["none"])
    return {"bytes": live * n * (SIZE[case["dy"]] + 2 * k * SIZE[case["type"]]) + 12 * t * k + 4 * t * k, "flops": 3 * live * k * n}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _to_e4m3(x):
    """The nearest value with 3 fraction bits (ties to the even one), at least 2^-9 apart, at most 448, in 64 bits."""
    e = torch.floor(torch.log2(torch.clamp(x.abs(), min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-LARGEST, LARGEST)


def _exact_adapters(case, z):
    ids, y = z["ids"].cpu(), z["y"].double()
    h = torch.zeros(case["rows"], case["r"], dtype=torch.float64, device=DEV)
    step = case["kind"] == "tune"
    if step:
        dx = z["dx"].double()
        da, db = torch.zeros_like(z["a"], dtype=torch.float64), torch.zeros_like(z["b"], dtype=torch.float64)
    for i in sorted(set(ids.tolist()) - {-1}):
        rows = torch.nonzero(ids == i)[:, 0].to(DEV)
        a, b, scale = z["a"][i].double(), z["b"][i].double(), float(z["scale"][i])
        h = scale * torch.einsum("tk,rk->tr", z["x"][rows].double(), a)
        y.index_add_(0, rows, torch.einsum("tr,rn->tn", h, b))
        if not step:
            continue
        dy = z["dy"][rows].double()
        dh = scale * torch.einsum("tn,rn->tr", dy, b)
        dx.index_add_(0, rows, torch.einsum("tr,rk->tk", dh, a))
        if z["x8"] is None:
            x = z["x"][rows].double()
        else:
            block = torch.arange(case["k"], device=DEV) // BLOCK
            x = z["x8"][rows].double() * z["x_scale"].double()[block][:, rows].t()
        da[i] = torch.einsum("tr,tk->rk", dh, x)
        db[i] = torch.einsum("tr,tn->rn", h, dy)
    return {"y": y, "dx": dx, "da": da, "db": db} if step else y


def _exact_drelu(case, z):
    n, r, m = int(z["n"]), case["rows"], case["m"]
    out = {v: torch.zeros(r, m, dtype=torch.float64, device=DEV) for v in ("c", "q_gate", "q_up", "dg", "du", "c_again")}
    for v in ("s_gate", "s_up"):
        out[v] = torch.zeros(-(-m // BLOCK), r, dtype=torch.float64, device=DEV)
    for i in range(-(-m // BLOCK)):
        at = slice(i * BLOCK, min(m, (i + 1) * BLOCK))
        g, u = z["g"][:n, at].double(), z["u"][:n, at].double()
        both = torch.logical_and(g > 0, u > 0).double()
        g, u = g * both, u * both
        out["c"][:n, at] = g * u
        wide = []
        for v, name in ((g, "gate"), (u, "up")):
            top = v.max(1).values
            s = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / LARGEST)).clamp(min=-101)).float().double()
            s = torch.where(top > LARGEST * s, 2 * s, s)
            s = torch.where(top <= LARGEST / 2 * s, s / 2, s)
            s = torch.where(top > 0, s.clamp(min=2.0 ** -100), torch.ones_like(s))
            q = torch.maximum(_to_e4m3(v / s[:, None]), both * 2.0 ** -9)
            out["q_" + name][:n, at], out["s_" + name][i, :n] = q, s
            wide.append(q * s[:, None])
        dc = z["dc"][:n, at].double()
        out["dg"][:n, at], out["du"][:n, at], out["c_again"][:n, at] = dc * wide[1], dc * wide[0], wide[0] * wide[1]
    return out


def _exact_balance(case, z):
    x, e = z["logits"].double().cpu(), case["experts"]
    sel, w, dw = z["sel"].long().cpu(), z["w"].double().cpu(), z["dw"].double().cpu()
    live = torch.isfinite(x).any(1)
    p = torch.zeros_like(x)
    p[live] = torch.softmax(x[live], 1)
    counts = torch.bincount(sel[sel >= 0], minlength=e)
    tokens, picks = int(live.sum()), int(counts.sum())
    share = p.sum(0) / max(tokens, 1)
    loss = e * float((counts.double() * share).sum()) / max(picks, 1)
    f = counts.double() * e / max(picks, 1) / max(tokens, 1) * float(z["dloss"].double())
    d = p * f - p * (p @ f)[:, None]
    mean = (w * dw).sum(1)
    for j in range(sel.shape[1]):
        t = torch.nonzero(sel[:, j] >= 0)[:, 0]
        d[t, sel[t, j]] += w[t, j] * (dw[t, j] - mean[t])
    return {"loss": torch.tensor([loss], dtype=torch.float64), "counts": counts.to(torch.int32), "share": share, "dlogits": d}


def exact(case, seed):
    z, kind = _inputs(case, seed), case["kind"]
    if kind in ("adapt", "tune"):
        return _exact_adapters(case, z)
    if kind == "drelu":
        return _exact_drelu(case, z)
    if kind == "balance":
        return _exact_balance(case, z)
    dy, slots, w = z["dy"].double(), z["slots"].long().cpu(), z["w"].double()
    dsrc = torch.zeros(z["src"].shape, dtype=torch.float64, device=DEV)
    dw = torch.zeros(w.shape, dtype=torch.float64, device=DEV)
    for j in range(slots.shape[1]):
        t = torch.nonzero(slots[:, j] >= 0)[:, 0].to(DEV)
        at = slots.to(DEV)[t, j]
        dsrc[at] = w[t, j, None] * dy[t]
        dw[t, j] = torch.einsum("tn,tn->t", dy[t], z["src"].double()[at])
    return {"dsrc": dsrc, "dw": dw}
