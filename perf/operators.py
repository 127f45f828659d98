"""Operators of a layer of routed experts over many tokens at once (a prompt, a large batch), as cases.

The steps of such a layer, each an operator of its own: `route` picks each token's experts from the router's logits
and lists the tokens of every expert; `gather` copies the rows of a list, `quant` rounds them to 8-bit floating
point with a scale for each 128 values; `grouped` multiplies each expert's rows with its weights, in bf16 or in
8 bits, plain or as the gated dReLU product, where one group is an ordinary matrix product; `combine` sums each
token's rows by their routing weights.

Sizes are those of this library's layers (d = 4096, m = 14336, 2 of 8 experts) and generic ones around them.
Experts differ in how often they are picked, and some of the tokens can be padding that no expert gets.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "f32": F32}
BLOCK = 128
LARGEST = 448.0  # of e4m3


def listed():
    big = {"d": 4096, "m": 14336, "experts": 8, "top_k": 2}
    return [
        # a decoding batch picks its experts: all latency
        {"name": "route_t4", "kind": "route", "tokens": 4, "experts": 8, "top_k": 2, "pad": 0},
        # a long prompt over many small experts, an eighth of the batch padding
        {"name": "route_t8192_e64", "kind": "route", "tokens": 8192, "experts": 64, "top_k": 6, "pad": 1024},
        # the rows of a few decoding tokens rounded to 8 bits, one row for each
        {"name": "quant_t16", "kind": "quant", "type": "bf16", "k": 4096, "tokens": 16, "rows": 16, "unused": 0},
        # a prompt's rows in the experts' order, each token twice
        {"name": "quant_t4096", "kind": "quant", "type": "bf16", "k": 4096, "tokens": 4096, "rows": 8192, "unused": 0},
        # gate and up products of 8 decoding tokens: nearly every expert's weights for a handful of rows
        {"name": "gated_bf16_t8", "kind": "grouped", "type": "bf16", "gated": True, "n": 14336, "k": 4096, "experts": 8,
         "rows": 16, "unused": 0, "layout": "nk", "out": "bf16"},
        # the same for a prompt
        {"name": "gated_bf16_t4096", "kind": "grouped", "type": "bf16", "gated": True, "n": 14336, "k": 4096,
         "experts": 8, "rows": 8192, "unused": 0, "layout": "nk", "out": "bf16"},
        # down products of a short prompt, weights stored by neuron, rows left over at the end
        {"name": "down_bf16_t300", "kind": "grouped", "type": "bf16", "gated": False, "n": 4096, "k": 14336, "experts": 8,
         "rows": 600, "unused": 40, "layout": "kn", "out": "f32"},
        # one token through one 8-bit matrix
        {"name": "mm_e4m3_t1", "kind": "grouped", "type": "e4m3", "gated": False, "n": 4096, "k": 14336, "experts": 1,
         "rows": 1, "unused": 0, "layout": "nk", "out": "f32"},
        # gate and up products in 8 bits, moderate ragged groups
        {"name": "gated_e4m3_t1000", "kind": "grouped", "type": "e4m3", "gated": True, "n": 14336, "k": 4096,
         "experts": 8, "rows": 2000, "unused": 0, "layout": "nk", "out": "bf16"},
        # a prompt through one 8-bit matrix
        {"name": "mm_e4m3_t8192", "kind": "grouped", "type": "e4m3", "gated": False, "n": 4096, "k": 14336,
         "experts": 1, "rows": 8192, "unused": 0, "layout": "nk", "out": "bf16"},
        # the experts' rows summed for a decoding batch and for a prompt
        {"name": "combine_t8", "kind": "combine", "type": "f32", "n": 4096, "tokens": 8, "top_k": 2, "none": 0.0},
        {"name": "combine_t4096", "kind": "combine", "type": "f32", "n": 4096, "tokens": 4096, "top_k": 2, "none": 0.05},
    ]


def _log_int(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(["route", "quant", "gather", "grouped", "grouped", "grouped", "grouped", "combine"])
    if kind == "route":
        e = rng.choice([2, 4, 8, 8, 16, 60, 64, 128, 256])
        t = _log_int(rng, 1, 16384)
        return {"kind": kind, "tokens": t, "experts": e, "top_k": min(e, rng.randint(1, 8)),
                "pad": rng.choice([0, 0, t // 8])}
    if kind == "combine":
        return {"kind": kind, "type": rng.choice(["bf16", "f32"]), "n": _log_int(rng, 256, 8192, 8),
                "tokens": _log_int(rng, 1, 8192), "top_k": rng.randint(1, 4), "none": rng.choice([0.0, 0.1])}
    if kind in ("quant", "gather"):
        t = _log_int(rng, 1, 8192)
        r = min(8192, t * rng.choice([1, 2, 2, 4]))
        return {"kind": kind, "type": rng.choice(["bf16", "bf16", "f32"]) if kind == "quant" else "bf16",
                "k": _log_int(rng, 256, 14336, 16), "tokens": t, "rows": r, "unused": rng.choice([0, r // 10])}
    kind8 = rng.random() < 0.5
    e = rng.choice([1, 2, 8, 8, 16, 64])
    k, n = _log_int(rng, 512, 14336, 16), _log_int(rng, 512, 14336, 8)
    while e * n * k > 8 * 14336 * 4096:  # the weights of the largest listed case
        n = max(512, n // 2 // 8 * 8)
        k = max(512, k * 2 // 3 // 16 * 16)
    rows = _log_int(rng, 1, 8192)
    while rows * n * k > 2 ** 38:
        rows //= 2
    gated = rng.random() < 0.4
    return {"kind": "grouped", "type": "e4m3" if kind8 else "bf16", "gated": gated, "n": n, "k": k, "experts": e,
            "rows": rows, "unused": rng.choice([0, rows // 8]),
            "layout": "nk" if kind8 or gated else rng.choice(["nk", "kn"]), "out": rng.choice(["bf16", "f32"])}


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


def _round8(w):
    """(values in e4m3, scales) of weights [n][k]: a scale for each 128 x 128."""
    n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    p = torch.zeros(nb * BLOCK, kb * BLOCK, device=DEV)
    p[:n, :k] = w
    p = p.view(nb, BLOCK, kb, BLOCK)
    s = p.abs().amax(dim=(1, 3)) / LARGEST
    q = (p / s[:, None, :, None]).clamp(-LARGEST, LARGEST).view(nb * BLOCK, kb * BLOCK)[:n, :k].contiguous().to(E4M3)
    return q, s


def _round8_rows(x):
    """(values in e4m3, scales [k / 128][rows]) of activations [rows][k]."""
    r, k = x.shape
    kb = -(-k // BLOCK)
    p = torch.zeros(r, kb * BLOCK, device=DEV)
    p[:, :k] = x
    p = p.view(r, kb, BLOCK)
    s = p.abs().amax(dim=2) / LARGEST
    s = torch.where(s > 0, s, torch.ones_like(s))
    q = (p / s[..., None]).clamp(-LARGEST, LARGEST).view(r, kb * BLOCK)[:, :k].contiguous().to(E4M3)
    return q, s.t().contiguous()


def _inputs(case, seed):
    """Everything that is drawn for a case, in one order."""
    g, kind = _gen(seed), case["kind"]
    if kind == "route":
        t, e = case["tokens"], case["experts"]
        logits = _randn(g, t, e) + 0.7 * _randn(g, e)  # some experts are picked more often
        if case["pad"]:
            pad = torch.randperm(t, generator=g, device=DEV)[:case["pad"]]
            logits[pad] = -math.inf
        return {"logits": logits}
    if kind in ("quant", "gather"):
        t, r = case["tokens"], case["rows"]
        x = _activations(g, t, case["k"]).to(TYPES[case["type"]])
        rows = torch.arange(r, device=DEV) % t  # every token equally often, in an expert's order
        rows = rows[torch.randperm(r, generator=g, device=DEV)].to(torch.int32)
        return {"x": x, "rows": rows, "n": torch.tensor([r - case["unused"]], dtype=torch.int32, device=DEV)}
    if kind == "combine":
        t, k = case["tokens"], case["top_k"]
        y = _randn(g, t * k, case["n"]).to(TYPES[case["type"]])
        slots = torch.randperm(t * k, generator=g, device=DEV).view(t, k)
        w = torch.softmax(_randn(g, t, k), dim=1)
        none = torch.rand(t, generator=g, device=DEV) < case["none"]  # padding: no expert has it
        slots = torch.where(none[:, None], -1, slots).to(torch.int32)
        return {"y": y, "slots": slots, "w": torch.where(none[:, None], 0.0, w)}
    e, n, k, r = case["experts"], case["n"], case["k"], case["rows"]
    used = r - case["unused"]
    pick = torch.multinomial(torch.softmax(0.6 * _randn(g, e), 0), used, replacement=True, generator=g)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), torch.bincount(pick, minlength=e).cumsum(0)])
    z = {"offsets": offsets.to(torch.int32)}
    x = _activations(g, r, k)
    if k > n:  # into the down product: dReLU products, most of them zero
        x = torch.relu(x - 1.0)
    shape = (k, n) if case["layout"] == "kn" else (n, k)
    two = 2 if case["gated"] else 1
    w = [[_randn(g, *shape).mul_(1.0 / math.sqrt(k)) for _ in range(e)] for _ in range(two)]
    if case["type"] == "e4m3":
        z["x"], z["x_scale"] = _round8_rows(x)
        both = [[_round8(m) for m in ws] for ws in w]
        z["w"], z["scale"] = [[q for q, _ in ws] for ws in both], [[s for _, s in ws] for ws in both]
    else:
        z["x"], z["x_scale"], z["scale"] = x.to(BF16), None, [None, None]
        z["w"] = [[m.to(BF16) for m in ws] for ws in w]
    return z


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind == "route":
        t, k = case["tokens"], case["top_k"]
        s["sel"], s["slots"] = (torch.empty(t, k, dtype=torch.int32, device=DEV) for _ in range(2))
        s["weights"] = torch.empty(t, k, device=DEV)
        s["offsets"] = torch.empty(case["experts"] + 1, dtype=torch.int32, device=DEV)
        s["rows"] = torch.full((t * k,), -1, dtype=torch.int32, device=DEV)
    elif kind == "quant":
        s["q"] = torch.zeros(case["rows"], case["k"], device=DEV).to(E4M3)
        s["s"] = torch.zeros(-(-case["k"] // BLOCK), case["rows"], device=DEV)
    elif kind == "gather":
        s["out"] = torch.zeros(case["rows"], case["k"], dtype=BF16, device=DEV)
    elif kind == "combine":
        s["out"] = torch.empty(case["tokens"], case["n"], device=DEV)
    else:
        s["y"] = torch.zeros(case["rows"], case["n"], dtype=TYPES[case["out"]], device=DEV)
        s["host_offsets"] = s["offsets"].tolist()  # the plain form slices by them
        if own:
            import paper_2406_05955_gb300 as ts
            kw = {"max_rows": case["rows"]}
            if case["gated"]:
                s["mm"] = ts.Grouped.gated(*s["w"], scale_gate=s["scale"][0], scale_up=s["scale"][1], **kw)
            else:
                s["mm"] = ts.Grouped(s["w"][0], layout=case["layout"], scale=s["scale"][0], **kw)
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_route(s):
    x, k = s["logits"], s["case"]["top_k"]
    t, e = x.shape
    top = torch.sort(x, dim=1, descending=True, stable=True)
    v, i = top.values[:, :k], top.indices[:, :k]
    ok = v > -math.inf
    z = torch.where(ok, torch.exp(v - torch.where(ok[:, :1], v[:, :1], 0.0)), 0.0)
    w = z / torch.where(ok[:, :1], z.sum(1, keepdim=True), 1.0)
    sel = torch.where(ok, i, -1)
    flat = torch.where(ok, i, e).reshape(-1)
    counts = (flat[:, None] == torch.arange(e, device=x.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    order = torch.sort(flat, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(t * k, device=x.device)
    rows = torch.where(torch.arange(t * k, device=x.device) < offsets[-1], order // k, -1)
    slots = torch.where(ok, place.view(t, k), -1)
    i32 = torch.int32
    return {"sel": sel.to(i32), "w": w, "offsets": offsets.to(i32), "rows": rows.to(i32), "slots": slots.to(i32)}


def _plain_quant(s):
    case = s["case"]
    n, r = case["rows"] - case["unused"], case["rows"]
    x = s["x"][s["rows"][:n].long()].float()
    kb = -(-case["k"] // BLOCK)
    p = torch.nn.functional.pad(x, (0, kb * BLOCK - case["k"])).view(n, kb, BLOCK)
    top = p.abs().amax(2)
    scale = torch.where(top > 0, torch.clamp(top / LARGEST, min=2.0 ** -100), 1.0)
    q = (p / scale[..., None]).clamp(-LARGEST, LARGEST).view(n, kb * BLOCK)[:, :case["k"]].to(E4M3)
    s["q"][:n] = q
    s["s"][:, :n] = scale.t()
    return {"q": s["q"], "scale": s["s"]}


def _wide(q, scale):
    """8-bit weights [n][k] with a scale for each 128 x 128, in 32 bits."""
    full = scale.repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)[:, :q.shape[1]]
    return q.float() * full


def _plain_grouped(s):
    case, off = s["case"], s["host_offsets"]
    e8 = case["type"] == "e4m3"
    x = s["x"].float()
    if e8:
        x = x * s["x_scale"].repeat_interleave(BLOCK, 0)[:case["k"]].t()

    def product(which, i):
        w = s["w"][which][i]
        w = _wide(w, s["scale"][which][i]) if e8 else w.float()
        return x[off[i]:off[i + 1]] @ (w if case["layout"] == "kn" else w.t())

    parts = [torch.relu(product(0, i)) * torch.relu(product(1, i)) if case["gated"] else product(0, i)
             for i in range(case["experts"]) if off[i + 1] > off[i]]
    s["y"][:off[-1]] = torch.cat(parts).to(s["y"].dtype)
    return s["y"]


def _plain_combine(s):
    rows = s["y"][s["slots"].clamp(min=0).long()].float()
    return (torch.where(s["slots"] >= 0, s["w"], 0.0)[..., None] * rows).sum(1)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2406_05955_gb300 as ts
        if kind == "route":
            r = ts.route(s["logits"], case["top_k"], sel=s["sel"], w=s["weights"], offsets=s["offsets"], rows=s["rows"],
                         slots=s["slots"])
            return {"sel": r.sel, "w": r.w, "offsets": r.offsets, "rows": r.rows, "slots": r.slots}
        if kind == "quant":
            q, scale = ts.quant_rows(s["x"], rows=s["rows"], n=s["n"], q=s["q"], scale=s["s"])
            return {"q": q, "scale": scale}
        if kind == "gather":
            return ts.gather_rows(s["x"], s["rows"], n=s["n"], out=s["out"])
        if kind == "combine":
            return ts.combine_rows(s["y"], s["slots"], s["w"], out=s["out"])
        return s["mm"].forward(s["x"], offsets=s["offsets"], x_scale=s["x_scale"], y=s["y"])
    if kind == "route":
        return _plain_route(s)
    if kind == "quant":
        return _plain_quant(s)
    if kind == "gather":
        n = case["rows"] - case["unused"]
        s["out"][:n] = s["x"][s["rows"][:n].long()]
        return s["out"]
    if kind == "combine":
        return _plain_combine(s)
    return _plain_grouped(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": 4 * t * e + 16 * t * k + 4 * (e + 1), "flops": t * e * (k + 1)}
    if kind in ("quant", "gather"):
        n = case["rows"] - case["unused"]
        size = {"bf16": 2, "f32": 4}[case["type"]]
        read = min(n, case["tokens"]) * case["k"] * size + 4 * n
        if kind == "gather":
            return {"bytes": read + n * case["k"] * size, "flops": 0}
        return {"bytes": read + n * case["k"] + 4 * n * -(-case["k"] // BLOCK), "flops": 3 * n * case["k"]}
    if kind == "combine":
        t, k, n = case["tokens"], case["top_k"], case["n"]
        size = {"bf16": 2, "f32": 4}[case["type"]]
        live = t * (1.0 - case["none"])
        return {"bytes": live * k * n * size + 8 * t * k + 4 * t * n, "flops": 2 * live * k * n}
    e, n, k, used = case["experts"], case["n"], case["k"], case["rows"] - case["unused"]
    size = 1 if case["type"] == "e4m3" else 2
    two = 2 if case["gated"] else 1
    hit = e * (1.0 - (1.0 - 1.0 / e) ** used)  # groups with a row at all
    b = two * hit * n * k * size + used * k * size + used * n * {"bf16": 2, "f32": 4}[case["out"]]
    if size == 1:
        b += 4 * -(-k // BLOCK) * (used + two * hit * -(-n // BLOCK))
    return {"bytes": b, "flops": 2.0 * two * used * n * k}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _to_e4m3(x):
    """The nearest value with 3 fraction bits (ties to the even one), at least 2^-9 apart, at most 448, in 64 bits."""
    e = torch.floor(torch.log2(torch.clamp(x.abs(), min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-LARGEST, LARGEST)


def _exact_route(case, x):
    x, e, k = x.double().cpu(), case["experts"], case["top_k"]
    rank = (x[:, None, :] > x[:, :, None]).sum(2) if e <= 64 else None
    if rank is None:
        order = torch.argsort(-x, dim=1, stable=True)
    else:
        ties = (x[:, None, :] == x[:, :, None]) & (torch.arange(e)[None, :] < torch.arange(e)[:, None])
        order = torch.argsort(rank + ties.sum(2), dim=1)
    sel = order[:, :k]
    v = x.gather(1, sel)
    live = torch.isfinite(v)
    shifted = torch.where(live, v - v[:, :1], torch.full_like(v, -math.inf))
    p = torch.softmax(torch.where(live.any(1, keepdim=True), shifted, torch.zeros_like(v)), 1) * live
    sel = torch.where(live, sel, -1)
    slots = torch.full_like(sel, -1)
    rows = torch.full((x.shape[0] * k,), -1, dtype=torch.int64)
    offsets = [0]
    for expert in range(e):
        t, j = torch.nonzero(sel == expert, as_tuple=True)
        at = offsets[-1] + torch.arange(t.numel())
        slots[t, j] = at
        rows[at] = t
        offsets.append(offsets[-1] + t.numel())
    i32 = torch.int32
    return {"sel": sel.to(i32), "w": p, "offsets": torch.tensor(offsets, dtype=i32), "rows": rows.to(i32),
            "slots": slots.to(i32)}


def exact(case, seed):
    z, kind = _inputs(case, seed), case["kind"]
    if kind == "route":
        return _exact_route(case, z["logits"])
    if kind == "gather":
        out = torch.zeros(case["rows"], case["k"], dtype=torch.float64, device=DEV)
        n = int(z["n"])
        out[:n] = z["x"].double().index_select(0, z["rows"][:n].int())
        return out
    if kind == "quant":
        n, k = int(z["n"]), case["k"]
        q = torch.zeros(case["rows"], k, dtype=torch.float64, device=DEV)
        scale = torch.zeros(-(-k // BLOCK), case["rows"], dtype=torch.float64, device=DEV)
        for b in range(scale.shape[0]):
            v = z["x"][:, b * BLOCK:(b + 1) * BLOCK].double()[z["rows"][:n].long()]
            top = v.abs().max(1).values
            s = torch.where(top == 0, torch.ones_like(top), torch.maximum(top / LARGEST, torch.full_like(top, 2.0 ** -100)))
            scale[b, :n] = s
            q[:n, b * BLOCK:(b + 1) * BLOCK] = _to_e4m3(v / s[:, None])
        return {"q": q, "scale": scale}
    if kind == "combine":
        y, w = z["y"].double(), z["w"].double()
        y = torch.cat([y, y.new_zeros(1, case["n"])])  # slot -1
        out = torch.zeros(case["tokens"], case["n"], dtype=torch.float64, device=DEV)
        for j in range(case["top_k"]):
            out += w[:, j:j + 1] * y[z["slots"][:, j].long()]
        return out
    out = torch.zeros(case["rows"], case["n"], dtype=torch.float64, device=DEV)
    e8, k = case["type"] == "e4m3", case["k"]
    x = z["x"].double()
    block = torch.arange(k, device=DEV) // BLOCK
    if e8:
        x *= z["x_scale"].double()[block].t()
    off = z["offsets"].cpu()
    for i in range(case["experts"]):
        a, b = int(off[i]), int(off[i + 1])
        if a == b:
            continue
        p = []
        for ws, scales in zip(z["w"], z["scale"]):
            w = ws[i].double()
            if e8:
                w *= scales[i].double()[torch.arange(case["n"], device=DEV) // BLOCK][:, block]
            p.append(x[a:b] @ w if case["layout"] == "kn" else x[a:b] @ w.t())
        out[a:b] = p[0].clamp(min=0) * p[1].clamp(min=0) if case["gated"] else p[0]
    return out
