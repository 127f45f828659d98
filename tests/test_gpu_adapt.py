"""Low-rank adapters beside a shared product, and their gradients, against plain implementations in 64 bits.

Tolerances. A sum in fp32 whose terms meet at most n roundings on their way (of 2^-24 each; the tensor cores truncate: 2^-23)
is within n 2^-23 of the sum of the terms' magnitudes. h: at most 8 steps of 16 in a tensor core, a sum for each 128 of k,
and the warps' and the cluster's joins, 48 in all for k up to 4096, and a product with the scale. out: as many more over
the r components in up to 3 parts (at most 24 steps), y and the rounding of h to 16 bits (bf16: 2^-16) or 24 (2^-23), then
the rounding to the type of out (half a step: 2^-8 of it in bf16). A gradient over n rows: n + 16 at most, plus the 2^-23 of h
in 24 bits."""
import math
import threading

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


def case(t, k, n, r, adapters, seed=0, dtype=BF16, none=0.2):
    """x, y, a, b, scale, ids."""
    g = gen(seed)
    ids = torch.randint(0, adapters, (t,), generator=g, device="cuda")
    ids = torch.where(torch.rand(t, generator=g, device="cuda") < none, -1, ids).to(torch.int32)
    return (randn(g, t, k).to(BF16), randn(g, t, n).to(dtype), (randn(g, adapters, r, k) / math.sqrt(k)).to(BF16),
            randn(g, adapters, r, n).to(BF16), 0.5 + torch.rand(adapters, generator=g, device="cuda"), ids)


def plain(x, a, b, scale, ids, y=None, ranks=None):
    """(h, its terms' magnitudes, out, its terms' magnitudes) in 64 bits."""
    t, r = x.shape[0], a.shape[1]
    h = torch.zeros(t, r, dtype=torch.float64, device="cuda")
    hm = torch.zeros_like(h)
    out = mag = None
    if y is not None:
        out, mag = y.double(), y.double().abs()
    for i in range(a.shape[0]):
        at = torch.nonzero(ids == i)[:, 0]
        rank = r if ranks is None else min(max(int(ranks[i]), 0), r)
        if not at.numel() or not rank:
            continue
        aa, bb, s = a[i, :rank].double(), b[i, :rank].double(), 1.0 if scale is None else float(scale[i])
        v = x[at].double()
        part, pm = s * v @ aa.t(), abs(s) * v.abs() @ aa.abs().t()
        h[at, :rank], hm[at, :rank] = part, pm
        if y is not None:
            out[at] += part @ bb
            mag[at] += pm @ bb.abs()
    return h, hm, out, mag


def check(ts, x, y, a, b, scale, ids, ranks=None, list_them=False, in_place=False, stream=None):
    ad = ts.Adapters(a, b, scale=scale, ranks=ranks)
    given = ad.rows(ids) if list_them else ids
    h = torch.full((x.shape[0], a.shape[1]), 7.0, device="cuda")
    want_h, hm, want, mag = plain(x, a, b, scale, ids, y, ranks)
    if in_place:
        out = y.clone()
        assert ad.forward(x, out, given, h=h) is out
    else:
        before = y.clone()
        out = ad.forward(x, y, given, out=torch.full_like(y, 9.0), h=h)
        assert torch.equal(y, before)
    assert ((h.double() - want_h).abs() <= 48 * U * hm).all()
    tol = (76 * U + (2.0 ** -16 if y.dtype == BF16 else U)) * mag
    if y.dtype == BF16:
        tol = tol + 2.0 ** -8 * want.abs()
    err = (out.double() - want).abs()
    assert (err <= tol).all(), float((err - tol).max())
    return out, h


MANY = [(512, 64, 64, 8, 1), (2060, 64, 64, 8, 1), (2600, 1408, 512, 16, 3), (1100, 136, 1032, 33, 5), (2100, 4096, 200, 64, 2),
        (1777, 8, 4096, 20, 4), (1300, 512, 8, 40, 7), (3000, 264, 520, 32, 1), (5000, 2048, 1408, 64, 90), (1025, 256, 128, 17, 1),
        # (so many rows that tiles are of 128, or, r above 64, of 64)
        (10000, 64, 64, 8, 1), (6000, 1408, 512, 16, 3), (3300, 136, 1032, 33, 5), (5000, 8, 4096, 20, 4), (3500, 512, 8, 40, 7),
        (5000, 256, 128, 17, 1), (2500, 520, 264, 100, 3)]
SIZES = [(1, 64, 64, 1, 1), (1, 4096, 1408, 16, 3), (2, 8, 8, 4, 2), (3, 136, 72, 5, 2), (17, 512, 1408, 16, 4),
         (64, 1024, 264, 32, 64), (64, 520, 4096, 64, 3), (33, 256, 136, 128, 5), (65, 512, 512, 8, 2), (130, 1408, 512, 40, 7),
         (300, 264, 1032, 12, 20), (1000, 512, 1408, 100, 3), (257, 4096, 128, 16, 1), (500, 128, 4104, 33, 255),
         (9, 4104, 1416, 13, 9), (40, 1048, 2952, 16, 30), (700, 4096, 520, 7, 64)]  # (chunks of 1024 bytes)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t,k,n,r,adapters", SIZES + MANY)
def test_forward(ts, t, k, n, r, adapters, dtype):
    c = case(t, k, n, r, adapters, seed=t + k, dtype=dtype)
    outs = [check(ts, *c, list_them=lists, in_place=place) for lists in (False, True) for place in (False, True)]
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[2][0], outs[3][0])


@pytest.mark.parametrize("t", [5, 64, 300, 511, 512, 1200, 5000])
def test_ids(ts, t):
    """No row has an adapter, all have the same, ids out of range, sorted ids, the last adapter alone."""
    x, y, a, b, scale, _ = case(t, 264, 136, 20, 4, seed=t)
    g = gen(t)
    for ids in (torch.full((t,), -1), torch.full((t,), 4), torch.full((t,), 2), torch.full((t,), 3),
                torch.randint(-3, 9, (t,), generator=g, device="cuda"), torch.arange(t) * 4 // t,
                torch.full((t,), -2 ** 31), torch.full((t,), 2 ** 31 - 1)):
        for lists in (False, True):
            check(ts, x, y, a, b, scale, ids.to("cuda", torch.int32), list_them=lists)


@pytest.mark.parametrize("t", [16, 200, 1300, 4500])
def test_ranks_scales_and_what_is_not_read(ts, t):
    """Components behind an adapter's rank and adapters without rows are not read; a scale may be absent, 0 or negative."""
    x, y, a, b, scale, ids = case(t, 256, 264, 24, 6, seed=3, none=0.1)
    ids = torch.where(ids == 4, 5, ids)
    ranks = torch.tensor([24, 0, 1, 17, 3, 30], dtype=torch.int32, device="cuda")
    a, b = a.clone(), b.clone()
    for i, rank in enumerate(ranks.tolist()):
        a[i, rank:], b[i, rank:] = math.nan, math.nan
    a[4], b[4] = math.nan, math.nan
    scale[0], scale[2], scale[3] = 0.0, -2.0, 1e-3
    for lists in (False, True):
        check(ts, x, y, a, b, scale, ids, ranks=ranks, list_them=lists)
        check(ts, x, y, a, b, None, ids, ranks=ranks, list_them=lists)


@pytest.mark.parametrize("t", [20, 150, 2100, 6000])
def test_infinities_and_nan_stay_in_their_rows(ts, t):
    x, y, a, b, scale, ids = case(t, 512, 136, 16, 3, seed=5)
    for lists in (False, True):
        want, _ = check(ts, x, y, a, b, scale, ids, list_them=lists)
        ad = ts.Adapters(a, b, scale=scale)
        bad = x.clone()
        bad[7, 3], bad[9, 500], y2 = math.nan, math.inf, y.clone()
        y2[11, 5] = -math.inf
        ids2 = ids.clone()
        ids2[7], ids2[9] = 1, -1
        got = ad.forward(bad, y2, ad.rows(ids2) if lists else ids2, out=torch.empty_like(y))
        assert got[7].isnan().all() and torch.equal(got[9], y[9]) and got[11, 5] == -math.inf
        rest = torch.ones(t, dtype=torch.bool, device="cuda")
        rest[[7, 9, 11]] = False
        assert torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("t", [3, 40, 700, 6000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_an_adapter_keep_their_bits(ts, t, dtype):
    """Zeros of either sign, subnormal numbers, infinities and NaN of any bits, through another buffer too."""
    x, y, a, b, scale, ids = case(t, 128, 272, 16, 3, seed=t, dtype=dtype)
    ids[::3], ids[1::3] = -1, 2
    ranks = torch.tensor([16, 16, 0], dtype=torch.int32, device="cuda")
    bits, special = (torch.int16, [0x8000, 1, 0x7f80, 0x7fc5, 0xffaa]) if dtype == BF16 else \
        (torch.int32, [0x80000000, 1, 0x7f800000, 0x7fc00005, 0xff8000aa])
    width = 16 if dtype == BF16 else 32
    y.view(bits)[:, 7:12] = torch.tensor([v - (1 << width) if v >> (width - 1) else v for v in special], device="cuda").to(bits)
    ad, none = ts.Adapters(a, b, scale=scale, ranks=ranks), (ids < 0) | (ids == 2)
    for given in (ids, ad.rows(ids)):
        out = ad.forward(x, y, given, out=torch.empty_like(y))
        assert torch.equal(out.view(bits)[none], y.view(bits)[none])


@pytest.mark.parametrize("t", [30, 100, 2055, 13000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_apart(ts, t, dtype):
    """Rows of x, y and out that lie in wider ones: what is between them is left as it was."""
    x, y, a, b, scale, ids = case(t, 136, 72, 6, 3, seed=7, dtype=dtype)
    want, h = check(ts, x, y, a, b, scale, ids)
    wide_x = torch.full((t, 160), math.nan, dtype=BF16, device="cuda")
    wide_y, wide_out = (torch.full((t, 96), 5.0, dtype=dtype, device="cuda") for _ in range(2))
    wide_x[:, 8:144], wide_y[:, 8:80] = x, y
    ad = ts.Adapters(a, b, scale=scale)
    got = ad.forward(wide_x[:, 8:144], wide_y[:, 8:80], ids, out=wide_out[:, 16:88])
    assert torch.equal(got, want) and torch.equal(wide_out[:, 16:88], want)
    assert (wide_out[:, :16] == 5).all() and (wide_out[:, 88:] == 5).all()
    ad.forward(wide_x[:, 8:144], wide_y[:, 8:80], ids)
    assert torch.equal(wide_y[:, 8:80], want) and (wide_y[:, :8] == 5).all() and (wide_y[:, 80:] == 5).all()


def test_no_rows(ts):
    x, y, a, b, scale, ids = case(0, 64, 64, 4, 3)
    ad = ts.Adapters(a, b, scale=scale)
    assert ad.forward(x, y, ids).shape == (0, 64)
    rows = ad.rows(ids)
    assert rows.offsets.tolist() == [0] * 5
    da, db = torch.full_like(a, 3.0, dtype=F32), torch.full_like(b, 3.0, dtype=F32)
    h, dy = torch.empty(0, 4, device="cuda"), torch.empty(0, 64, dtype=BF16, device="cuda")
    ad.backward(dy, x.clone(), rows, h, x, da=da, db=db, accumulate=True)
    assert (da == 3).all() and (db == 3).all()
    ad.backward(dy, x.clone(), rows, h, x, da=da, db=db)
    assert (da == 0).all() and (db == 0).all()


@pytest.mark.parametrize("t", [1, 2, 33, 1000, 1025, 5000, 40000])
@pytest.mark.parametrize("groups", [1, 2, 7, 64, 255])
def test_list_rows(ts, t, groups):
    ids = torch.randint(-2, groups + 2, (t,), generator=gen(t + groups), device="cuda").to(torch.int32)
    if t == 5000:
        ids.fill_(groups - 1)
    got = ts.list_rows(ids, groups)
    of = torch.where((ids >= 0) & (ids < groups), ids, groups).long()
    assert got.rows.tolist() == torch.sort(of, stable=True).indices.tolist()
    assert got.offsets.tolist() == [0] + torch.bincount(of, minlength=groups + 1).cumsum(0).tolist()


def kept_rows(ts, x):
    q, s = ts.quant_rows(x)
    return q, s, q.double() * s.double().repeat_interleave(128, 0)[:x.shape[1]].t()


@pytest.mark.parametrize("x8", [False, True])
@pytest.mark.parametrize("t,k,n,r,adapters", [(1, 64, 64, 1, 1), (3, 144, 72, 5, 2), (64, 512, 1408, 16, 4), (130, 1408, 512, 40, 7),
                                              (700, 272, 1032, 12, 20), (1000, 512, 136, 100, 3), (2049, 128, 264, 128, 2), (3000, 512, 264, 32, 3),
                                              (90, 16, 8, 33, 255)])
def test_backward(ts, t, k, n, r, adapters, x8):
    x, _, a, b, scale, ids = case(t, k, n, r, adapters, seed=t)
    g = gen(t + 1)
    dy, dx = (0.1 * randn(g, t, n)).to(BF16), randn(g, t, k).to(F32 if t % 2 else BF16)
    h = randn(g, t, r)
    ad = ts.Adapters(a, b, scale=scale)
    h[(ids < 0)] = 0.0
    x_scale, wide = None, x.double()
    if x8:
        x, x_scale, wide = kept_rows(ts, x)
    dh, dhm, want, mag = plain(dy, b, a, scale, ids, dx)
    before = dx.clone()
    out, da, db = ad.backward(dy, dx, ids, h, x, x_scale=x_scale, out=torch.empty_like(dx))
    assert torch.equal(dx, before)
    tol = (76 * U + (2.0 ** -16 if dx.dtype == BF16 else U)) * mag + (2.0 ** -8 * want.abs() if dx.dtype == BF16 else 0.0)
    assert ((out.double() - want).abs() <= tol).all()
    for i in range(adapters):
        at = torch.nonzero(ids == i)[:, 0]
        m = at.numel()
        hi, dhi = h[at].double(), dh[at]
        assert ((db[i].double() - hi.t() @ dy[at].double()).abs() <= (m + 17) * U * (hi.abs().t() @ dy[at].double().abs())).all()
        tol = (m + 17) * U * (dhi.abs().t() @ wide[at].abs()) + 48 * U * (dhm[at].t() @ wide[at].abs())
        assert ((da[i].double() - dhi.t() @ wide[at]).abs() <= tol).all()
        if m == 0:
            assert (da[i] == 0).all() and (db[i] == 0).all()
    again = ad.backward(dy, dx, ad.rows(ids), h, x, x_scale=x_scale, out=torch.empty_like(dx))
    assert all(torch.equal(p, q) for p, q in zip(again, (out, da, db)))
    # added to: exact where what is there is a power of two far below, so only that it is not overwritten
    da2, db2 = torch.full_like(da, 2.0), torch.full_like(db, -2.0)
    ad.backward(dy, None, ids, h, x, x_scale=x_scale, da=da2, db=db2, accumulate=True)
    assert torch.equal(da2, da + 2.0) and torch.equal(db2, db - 2.0)


@pytest.mark.parametrize("t,r,adapters", [(1, 8, 3), (7, 16, 7), (200, 4, 200), (900, 17, 30), (2500, 64, 5), (1100, 128, 9),
                                          (72, 33, 9), (81, 20, 9),  # (8 and 9 rows of each)
                                          (832, 8, 2), (1000, 12, 3), (1280, 16, 2), (1500, 64, 2), (7000, 30, 40)])  # (clusters of 5, 6, 7)
def test_gradients_of_uneven_adapters(ts, t, r, adapters):
    """Nearly all rows have one adapter, each its own, few at the ends: whatever part of the list a CTA has."""
    g = gen(t)
    k, n = 136, 264
    x, dy, h = randn(g, t, k).to(BF16), randn(g, t, n).to(BF16), randn(g, t, r)
    ad = ts.Adapters(torch.zeros(adapters, r, k, dtype=BF16, device="cuda"), torch.zeros(adapters, r, n, dtype=BF16, device="cuda"))
    some = torch.randint(0, adapters, (t,), generator=g, device="cuda")
    last = torch.full_like(some, adapters - 1)
    first = torch.where(torch.arange(t, device="cuda") % 100 == 3, some, 0)
    for ids in (some, last, first, torch.arange(t, device="cuda") % adapters, torch.arange(t, device="cuda") * adapters // t,
                torch.where(some == 1, -1, 1), torch.where(torch.arange(t, device="cuda") < t // 2, 0, adapters - 1)):
        _, _, db = ad.backward(dy, None, ids.to(torch.int32), h, x)
        one = torch.nn.functional.one_hot(ids.clamp(min=0).long(), adapters).double() * (ids >= 0)[:, None]
        want = torch.einsum("ta,tr,tn->arn", one, h.double(), dy.double())
        mag = torch.einsum("ta,tr,tn->arn", one, h.double().abs(), dy.double().abs())
        assert ((db.double() - want).abs() <= (one.sum(0) + 17)[:, None, None] * U * mag).all()


def test_rows_without_an_adapter_do_not_reach_the_gradients(ts):
    x, _, a, b, scale, ids = case(200, 256, 128, 8, 3, seed=9, none=0.3)
    g = gen(10)
    dy, h = (0.1 * randn(g, 200, 128)).to(BF16), randn(g, 200, 8)
    ad = ts.Adapters(a, b, scale=scale)
    _, da, db = ad.backward(dy, None, ids, h, x)
    off = ids < 0
    x2, dy2, h2 = x.clone(), dy.clone(), h.clone()
    x2[off], dy2[off], h2[off] = math.nan, math.inf, math.nan
    _, da2, db2 = ad.backward(dy2, None, ids, h2, x2)
    assert torch.equal(da, da2) and torch.equal(db, db2)
    one = int(torch.nonzero(ids == 1)[0])
    x2[one, 5] = math.nan
    _, da3, _ = ad.backward(dy2, None, ids, h2, x2)
    assert da3[1, :, 5].isnan().all() and torch.equal(da3[[0, 2]], da[[0, 2]])
    keep = torch.ones(256, dtype=torch.bool, device="cuda")
    keep[5] = False
    assert torch.equal(da3[1][:, keep], da[1][:, keep])


@pytest.mark.parametrize("r", [16, 20, 64, 100])
def test_infinities_in_gradients(ts, r):
    """An infinity in a row times an h of few bits is that infinity, for adapters of any number of rows; 0 times it is NaN, and so
    are two of both signs. Everything else is as without it."""
    g = gen(r)
    k, n, counts = 136, 264, [8, 9, 64, 65, 700]
    ids = torch.cat([torch.full((c,), i) for i, c in enumerate(counts)]).to("cuda", torch.int32)
    t = ids.numel()
    x, dy = randn(g, t, k).to(BF16), randn(g, t, n).to(BF16)
    # h of 1, 8, 16 and 24 bits, and 0
    h = torch.stack([(randn(g, t, r) * 0.25).to(BF16).float() if j == 1 else randn(g, t, r) for j in range(4)])
    h[0], h[2] = 1.0 + (h[0] > 0), h[2].mul(2.0 ** 12).round().mul(2.0 ** -12)
    h = h.gather(0, torch.randint(0, 4, (1, t, r), generator=g, device="cuda"))[0]
    h[5], h[5, 0] = 0.0, -1.0
    first = 0
    for c in counts:  # in the first, the last and two other rows of each
        dy[first, 3], dy[first + c - 1, 7], dy[first + 5, 11] = math.inf, -math.inf, math.inf
        dy[first + 1, 200], dy[first + 4, 200] = math.inf, -math.inf
        first += c
    a, b = torch.zeros(len(counts), r, k, dtype=BF16, device="cuda"), torch.zeros(len(counts), r, n, dtype=BF16, device="cuda")
    _, _, db = ts.Adapters(a, b).backward(dy, None, ids, h, x)
    _, _, plain_db = ts.Adapters(a, b).backward(torch.where(dy.isinf(), 0.0, dy), None, ids, h, x)
    for i, c in enumerate(counts):
        at = ids == i
        terms = h[at].double()[:, :, None] * dy[at].double()[:, None, :]
        want, inf = terms.sum(0), dy[at].isinf().any(0)
        assert inf.sum() == 4
        assert torch.equal(db[i][:, inf].double().nan_to_num(nan=7.0), want[:, inf].nan_to_num(nan=7.0)), (i, c)
        assert torch.equal(db[i][:, ~inf], plain_db[i][:, ~inf])
        assert ((db[i].double() - want).abs() <= (c + 17) * U * terms.abs().sum(0))[:, ~inf].all()


def test_gradients_against_differences(ts):
    """<gradient, direction> against central differences of sum(out * weight) in 64 bits: out is linear in each of x, A
    and B, so the differences are exact but for rounding, and what is left are the kernels' own tolerances."""
    t, k, n, r, adapters = 120, 128, 72, 8, 3
    x, y, a, b, scale, ids = case(t, k, n, r, adapters, seed=11, dtype=F32)
    dy = randn(gen(12), t, n).to(BF16)
    ad = ts.Adapters(a, b, scale=scale)
    h = torch.empty(t, r, device="cuda")
    ad.forward(x, y, ids, out=torch.empty_like(y), h=h)
    dx, da, db = ad.backward(dy, torch.zeros(t, k, device="cuda"), ids, h, x)

    def value(x, a, b):
        some = ids >= 0
        i = ids.clamp(min=0).long()
        h = torch.einsum("tk,trk->tr", x, a[i]) * torch.where(some, scale[i].double(), 0.0)[:, None]
        return float((dy.double() * torch.einsum("tr,trn->tn", h, b[i])).sum())

    at = (x.double(), a.double(), b.double())
    for which, grad in enumerate((dx, da, db)):
        d = torch.randn(grad.shape, generator=gen(20 + which), device="cuda").double()
        plus, minus = list(at), list(at)
        plus[which], minus[which] = at[which] + 0.5 * d, at[which] - 0.5 * d
        want = value(*plus) - value(*minus)
        got = float((grad.double() * d).sum())
        # 200 roundings of 2^-23 on terms of random signs, whose magnitudes' sum is below 64 times the norms' product here
        assert abs(got - want) <= 200 * U * float(grad.double().norm() * d.norm()) * 64, which


@pytest.mark.parametrize("t,r,adapters", [(120, 8, 3), (700, 40, 5)])
def test_gradients_along_themselves(ts, t, r, adapters):
    """As above, along the gradient itself, where the difference is its square: within the sum of each element's own roundings times
    it, which is less than half a percent of the difference, so that a wrong scale or a row left out is found."""
    k, n = 128, 72
    x, y, a, b, scale, ids = case(t, k, n, r, adapters, seed=11, dtype=F32)
    dy = randn(gen(12), t, n).to(BF16)
    ad = ts.Adapters(a, b, scale=scale)
    h = torch.empty(t, r, device="cuda")
    ad.forward(x, y, ids, out=torch.empty_like(y), h=h)
    grads = ad.backward(dy, torch.zeros(t, k, device="cuda"), ids, h, x)
    some = torch.where(ids >= 0, scale[ids.clamp(min=0).long()].double(), 0.0)[:, None]
    i = ids.clamp(min=0).long()

    def terms(x, a, b, dy):
        """h and dh, and the sums dx, da and db."""
        h, dh = torch.einsum("tk,trk->tr", x, a[i]) * some, torch.einsum("tn,trn->tr", dy, b[i]) * some
        one = torch.nn.functional.one_hot(i, adapters).double() * (ids >= 0)[:, None]
        return (h, dh), (torch.einsum("tr,trk->tk", dh, a[i]), torch.einsum("ta,tr,tk->ark", one, dh, x), torch.einsum("ta,tr,tn->arn", one, h, dy))

    at = (x.double(), a.double(), b.double(), dy.double())
    _, mags = terms(*(v.abs() for v in at))
    # out's h and dh: 48 roundings; dx 77 with those; da and db as many as an adapter's rows and 17, and those of dh and h
    m = int(torch.bincount(i[ids >= 0]).max())
    for which, (grad, mag, roundings) in enumerate(zip(grads, mags, (77, m + 17 + 48, m + 17 + 48))):
        d = grad.double()
        plus, minus = list(at), list(at)
        plus[which], minus[which] = at[which] + 0.5 * d, at[which] - 0.5 * d

        def value(x, a, b, dy):
            (h, _), _ = terms(x, a, b, dy)
            return float((dy * torch.einsum("tr,trn->tn", h, b[i])).sum())

        want, got = value(*plus) - value(*minus), float((d * d).sum())
        tol = roundings * U * float((mag * d.abs()).sum())
        assert abs(got - want) <= tol <= 0.005 * abs(want), (which, got, want, tol)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t,k,n,r,adapters", [(1, 14336, 136, 16, 2), (70, 14336, 4096, 8, 9), (300, 14336, 264, 64, 20), (2600, 14336, 520, 32, 2),
                                              (9000, 14336, 128, 64, 3), (2500, 14336, 264, 128, 2)])
def test_long_rows(ts, t, k, n, r, adapters, dtype):
    """k of 14336. h: sums of 8 or 16 steps in the tensor cores, one for each 128 of k at most, 8 CTAs' and the scale: k / 128 + 24
    roundings at most; out 28 more, as above."""
    x, y, a, b, scale, ids = case(t, k, n, r, adapters, seed=t + r, dtype=dtype)
    ad, steps = ts.Adapters(a, b, scale=scale), k / 128 + 24
    want_h, hm, want, mag = plain(x, a, b, scale, ids, y)
    for given in (ids, ad.rows(ids)):
        h = torch.full((t, r), 7.0, device="cuda")
        out = ad.forward(x, y, given, out=torch.empty_like(y), h=h)
        assert ((h.double() - want_h).abs() <= steps * U * hm).all()
        tol = ((steps + 28) * U + (2.0 ** -16 if dtype == BF16 else U)) * mag + (2.0 ** -8 * want.abs() if dtype == BF16 else 0.0)
        assert ((out.double() - want).abs() <= tol).all()
    # gradients, of k and of n columns
    dy = (0.1 * randn(gen(t), t, n)).to(BF16)
    _, da, db = ad.backward(dy, None, ids, h, x)
    dh, dhm, _, _ = plain(dy, b, a, scale, ids)
    for i in range(adapters):
        at = torch.nonzero(ids == i)[:, 0]
        m, v, d, hi = at.numel(), x[at].double(), dy[at].double(), h[at].double()
        assert ((db[i].double() - hi.t() @ d).abs() <= (m + 17) * U * (hi.abs().t() @ d.abs())).all()
        tol = (m + 17) * U * (dh[at].abs().t() @ v.abs()) + 48 * U * (dhm[at].t() @ v.abs())
        assert ((da[i].double() - dh[at].t() @ v).abs() <= tol).all()


@pytest.mark.parametrize("t,k,n,r", [(40, 512, 264, 16), (2500, 264, 520, 64), (9000, 512, 136, 32), (2300, 136, 264, 100)])
def test_pools_of_which_few_are_hit(ts, t, k, n, r):
    """255 adapters, whose weights are NaN but for the three that rows have: as a pool of these three, within roundings, and no
    gradient of the others."""
    x, y, a, b, scale, ids = case(t, k, n, r, 3, seed=t, dtype=F32)
    where = torch.tensor([7, 100, 254], device="cuda")
    pool_a, pool_b = (torch.full((255, r, v.shape[2]), math.nan, dtype=BF16, device="cuda") for v in (a, b))
    pool_a[where], pool_b[where], pool_scale = a, b, torch.ones(255, device="cuda")
    pool_scale[where] = scale
    pool_ids = torch.where(ids >= 0, where.to(torch.int32)[ids.clamp(min=0).long()], -1)
    ad, few = ts.Adapters(pool_a, pool_b, scale=pool_scale), ts.Adapters(a, b, scale=scale)
    want_h, hm, want, mag = plain(x, a, b, scale, ids, y)
    h, dy = torch.empty(t, r, device="cuda"), randn(gen(t), t, n).to(BF16)
    for given in (pool_ids, ad.rows(pool_ids)):
        out = ad.forward(x, y, given, out=torch.empty_like(y), h=h)
        assert ((h.double() - want_h).abs() <= 48 * U * hm).all()
        assert ((out.double() - want).abs() <= 77 * U * mag).all()
    _, da, db = ad.backward(dy, None, pool_ids, h, x)
    _, few_da, few_db = few.backward(dy, None, ids, h, x)
    off = torch.ones(255, dtype=torch.bool, device="cuda")
    off[where] = False
    assert (da[off] == 0).all() and (db[off] == 0).all()
    m = int(torch.bincount(ids[ids >= 0].long()).max())
    for i in range(3):
        at = ids == i
        hi, d = h[at].double().abs(), dy[at].double().abs()
        assert ((db[where[i]].double() - few_db[i].double()).abs() <= 2 * (m + 17) * U * (hi.t() @ d)).all()
        dh, dhm, _, _ = plain(dy, b, a, scale, ids)
        tol = 2 * ((m + 17) * U * (dh[at].abs().t() @ x[at].double().abs()) + 48 * U * (dhm[at].t() @ x[at].double().abs()))
        assert ((da[where[i]].double() - few_da[i].double()).abs() <= tol).all()


@pytest.mark.parametrize("t,k,r,adapters,x8", [(5, 48, 4, 3, False), (300, 272, 7, 4, True), (2000, 520, 64, 3, False), (1500, 1408, 100, 2, True)])
def test_gradients_by_themselves(ts, t, k, r, adapters, x8):
    """``ts_adapter_grads`` of h and rows alone, overwritten and added to: against 64 bits, and the same bits as in the backward pass."""
    from paper_2406_05955_gb300 import binding

    x, _, a, b, scale, ids = case(t, k, 64, r, adapters, seed=t)
    g = gen(t)
    h, dy = randn(g, t, r), randn(g, t, 64).to(BF16)
    ad = ts.Adapters(a, b, scale=scale)
    rows, x_scale, wide = ad.rows(ids), None, x.double()
    if x8:
        x, x_scale, wide = kept_rows(ts, x)

    def grads(v, v_scale, to, add):
        code = binding.TS_E4M3 if v_scale is not None else binding.TS_BF16
        status = ts.lib().ts_adapter_grads(h.data_ptr(), r, v.data_ptr(), v.stride(0), code, None if v_scale is None else v_scale.data_ptr(),
                                           0 if v_scale is None else v_scale.stride(0), t, v.shape[1], adapters, rows.rows.data_ptr(),
                                           rows.offsets.data_ptr(), to.data_ptr(), add, torch.cuda.current_stream().cuda_stream)
        assert status == binding.TS_OK
        return to

    got = grads(x, x_scale, torch.full((adapters, r, k), 5.0, device="cuda"), 0)
    for i in range(adapters):
        at = ids == i
        want, mag = h[at].double().t() @ wide[at], h[at].double().abs().t() @ wide[at].abs()
        assert ((got[i].double() - want).abs() <= (int(at.sum()) + 17) * U * mag).all()
    assert torch.equal(grads(x, x_scale, torch.full_like(got, 3.0), 1), got + 3.0)
    _, _, db = ad.backward(dy, None, rows, h, x, x_scale=x_scale)
    assert torch.equal(grads(dy, None, torch.empty_like(db), 0), db)


@pytest.mark.parametrize("r", [16, 30, 64])
def test_many_rows_at_once(ts, r):
    """A forward of many listed rows on one stream beside backward passes on another, whose sums all lie in tensor memory: the same
    bits as one after the other."""
    x, y, a, b, scale, ids = case(7000, 520, 1032, r, 3, seed=27)
    ad, g = ts.Adapters(a, b, scale=scale), gen(28)
    dy, h, rows = randn(g, 7000, 1032).to(BF16), randn(g, 7000, r), ad.rows(ids)
    few, dx = case(900, 264, 520, 12, 4, seed=29), randn(g, 900, 264)
    ad2, dy2, h2 = ts.Adapters(few[2], few[3], scale=few[4]), randn(g, 900, 520).to(BF16), randn(g, 900, 12)
    rows2 = ad2.rows(few[5])
    want = ad.forward(x, y, rows, out=torch.empty_like(y))
    want_back = ad.backward(dy, None, rows, h, x)[1:]
    want2 = ad2.backward(dy2, dx, rows2, h2, few[0], out=torch.empty_like(dx))
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = [_like(y, streams[0]) for _ in range(10)]
    back, back2 = [], []
    for out in outs:
        ad.forward(x, y, rows, out=out, stream=streams[0])
        back.append(ad.backward(dy, None, rows, h, x, stream=streams[1])[1:])
        back2.append(ad2.backward(dy2, dx, rows2, h2, few[0], out=_like(dx, streams[2]), stream=streams[2]))
    torch.cuda.synchronize()
    assert ts.adapt_error() == 0
    assert all(torch.equal(out, want) for out in outs)
    assert all(torch.equal(p, q) for got in back for p, q in zip(got, want_back))
    assert all(torch.equal(p, q) for got in back2 for p, q in zip(got, want2))


def test_streams_graphs_and_calls_at_once(ts):
    c = case(300, 512, 264, 16, 5, seed=13)
    few = case(40, 512, 264, 16, 5, seed=14)
    x, y, a, b, scale, ids = c
    ad, ad2 = ts.Adapters(a, b, scale=scale), ts.Adapters(few[2], few[3], scale=few[4])
    want = ad.forward(x, y, ids, out=torch.empty_like(y))
    want2 = ad2.forward(few[0], few[1], few[5], out=torch.empty_like(few[1]))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (s1, s2):
        s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(20):  # in flight together
        outs.append((ad.forward(x, y, ids, out=_like(y, s1), stream=s1), ad2.forward(few[0], few[1], few[5], out=_like(few[1], s2), stream=s2)))
    torch.cuda.synchronize()
    assert all(torch.equal(p, want) and torch.equal(q, want2) for p, q in outs)
    h, dy = torch.empty(300, 16, device="cuda"), (0.1 * randn(gen(15), 300, 264)).to(BF16)
    dx, out = randn(gen(16), 300, 512), torch.empty_like(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        rows = ad.rows(ids)
        ad.forward(x, y, rows, out=out, h=h)
        got = ad.backward(dy, dx, rows, h, x, out=torch.empty_like(dx))
    other = case(300, 512, 264, 16, 5, seed=17)
    x.copy_(other[0])
    ids.copy_(other[5])
    graph.replay()
    graph.replay()
    h2 = torch.empty_like(h)
    want = ad.forward(x, y, ids, out=torch.empty_like(y), h=h2)
    back = ad.backward(dy, dx, ids, h2, x, out=torch.empty_like(dx))
    assert torch.equal(out, want) and torch.equal(h, h2)
    assert all(torch.equal(p, q) for p, q in zip(got, back))


def _like(t, stream):
    with torch.cuda.stream(stream):
        return torch.empty_like(t)


@pytest.mark.parametrize("t,r,ld", [(600, 8, 1 << 22), (1800, 64, 1 << 21)])
def test_offsets_beyond_32_bits(ts, t, r, ld):
    """Rows whose elements are more than 2^31 apart."""
    k, n = 64, 64
    x, y, a, b, scale, ids = case(t, k, n, r, 3, seed=18)
    want, h = check(ts, x, y, a, b, scale, ids)
    far = torch.empty(t * ld, dtype=BF16, device="cuda")
    fx, fy = far.view(t, ld)[:, :k], far.view(t, ld)[:, 1024:1024 + n]
    fx.copy_(x)
    fy.copy_(y)
    ad = ts.Adapters(a, b, scale=scale)
    assert torch.equal(ad.forward(fx, fy, ids, out=far.view(t, ld)[:, 2048:2048 + n]), want)
    dy = (0.1 * randn(gen(19), t, n)).to(BF16)
    far_dy = far.view(t, ld)[:, 4096:4096 + n]
    far_dy.copy_(dy)
    near = ad.backward(dy, None, ids, h, x)
    assert all(torch.equal(p, q) for p, q in zip(near[1:], ad.backward(far_dy, None, ids, h, fx)[1:]))


def test_a_wait_that_gives_up(ts):
    """The wait runs out, is reported once, and the next call is right."""
    c = case(6000, 264, 264, 16, 3, seed=21)
    want, _ = check(ts, *c, list_them=True)
    assert ts.adapt_error() == 0
    x, y, a, b, scale, ids = c
    ad = ts.Adapters(a, b, scale=scale)
    ts.adapt_test_stall(True)
    try:
        ad.forward(x, y, ids, out=torch.empty_like(y))
        torch.cuda.synchronize()
    finally:
        ts.adapt_test_stall(False)
    assert ts.adapt_error() == 5 and ts.adapt_error() == 0
    assert torch.equal(ad.forward(x, y, ids, out=torch.empty_like(y)), want)
    rows, h, dy = ad.rows(ids), torch.randn(6000, 16, device="cuda"), y.clone()
    want = ad.backward(dy, None, rows, h, x)
    ts.adapt_test_stall(True)
    try:
        ad.backward(dy, None, rows, h, x)
        torch.cuda.synchronize()
    finally:
        ts.adapt_test_stall(False)
    assert ts.adapt_error() == 5 and ts.adapt_error() == 0
    assert all(torch.equal(p, q) for p, q in zip(ad.backward(dy, None, rows, h, x)[1:], want[1:]))


def test_a_wait_that_gives_up_while_others_ask(ts):
    """Whoever asks, on another stream, while waits give up: someone is told of each call, and then nothing is left."""
    x, y, a, b, scale, ids = case(6000, 264, 264, 16, 3, seed=22)
    ad = ts.Adapters(a, b, scale=scale)
    rows, h, out = ad.rows(ids), randn(gen(23), 6000, 16), torch.empty_like(y)
    torch.cuda.synchronize()
    assert ts.adapt_error() == 0
    told, stop = [], threading.Event()

    def ask(stream):
        while not stop.is_set():
            told.append(ts.adapt_error(stream=stream))

    for call in (lambda: ad.forward(x, y, rows, out=out), lambda: ad.backward(y, None, rows, h, x)):
        told.clear()
        stop.clear()
        askers = [threading.Thread(target=ask, args=(torch.cuda.Stream(),)) for _ in range(2)]
        for t in askers:
            t.start()
        ts.adapt_test_stall(True)
        try:
            call()
            torch.cuda.synchronize()
        finally:
            ts.adapt_test_stall(False)
            stop.set()
            for t in askers:
                t.join()
        told.append(ts.adapt_error())
        assert 5 in told and set(told) <= {0, 5}
        assert ts.adapt_error() == 0


def test_autograd(ts):
    """Rows changed in place are so for autograd too: a backward pass that needs what was there is refused. In a Function of the
    caller's, gradients are those of the formula."""
    x, y, a, b, scale, ids = case(90, 128, 72, 8, 3, seed=24, dtype=F32)
    ad = ts.Adapters(a, b, scale=scale)
    dy, dx, h = randn(gen(25), 90, 72).to(BF16), randn(gen(26), 90, 128), torch.zeros(90, 8, device="cuda")
    for t, call in ((y, lambda: ad.forward(x, y, ids)), (dx, lambda: ad.backward(dy, dx, ids, h, x))):
        w = torch.ones_like(t, requires_grad=True)
        z = (t * w).sum()  # keeps t
        before = t.clone()
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()
        t.copy_(before)
        z = (t * w).sum()
        ad.forward(x, y, ids, out=torch.empty_like(y))
        ad.backward(dy, dx, ids, h, x, out=torch.empty_like(dx))
        z.backward()
        assert torch.equal(w.grad, before)
    with torch.inference_mode():
        assert torch.equal(ad.forward(x, y.clone(), ids), ad.forward(x, y, ids, out=torch.empty_like(y)))

    class Adapted(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, y, a, b):
            h, out = torch.empty(x.shape[0], a.shape[1], device="cuda"), torch.empty_like(y)
            ctx.ad = ts.Adapters(a, b, scale=scale)
            ctx.ad.forward(x, y, ids, out=out, h=h)
            ctx.save_for_backward(x, h)
            return out

        @staticmethod
        def backward(ctx, dout):
            x, h = ctx.saved_tensors
            dx, da, db = ctx.ad.backward(dout.to(BF16), torch.zeros(x.shape, device="cuda"), ids, h, x)
            return dx.to(BF16), dout, da, db

    leaves = [v.clone().requires_grad_() for v in (x, y, a, b)]
    out = Adapted.apply(*leaves)
    out.backward(dy.float())
    exact = [v.double().requires_grad_() for v in (x, y, a, b)]
    i, some = ids.clamp(min=0).long(), torch.where(ids >= 0, scale[ids.clamp(min=0).long()].double(), 0.0)
    low = torch.einsum("tk,trk->tr", exact[0], exact[2][i]) * some[:, None]
    want = exact[1] + torch.einsum("tr,trn->tn", low, exact[3][i])
    want.backward(dy.double())
    for got, v in zip(leaves, exact):
        assert (got.grad.double() - v.grad).norm() <= 2.0 ** -8 * v.grad.norm()  # (x's, a's and b's are rounded to bf16)


def test_outputs_over_inputs(ts):
    """An adapter around the identity (y is x, dx is dy): written over what others still read it is refused, and nothing is written;
    into a buffer of its own it is right. Rows between each other's, as columns of one buffer, are apart."""
    for t, r in ((1, 16), (4, 16), (300, 8), (2100, 64), (1500, 100)):
        k = 512
        x, _, a, b, scale, ids = case(t, k, k, r, 3, seed=t + r, none=0.0)
        ad, h = ts.Adapters(a, b, scale=scale), torch.empty(t, r, device="cuda")
        want = ad.forward(x, x.clone(), ids, out=torch.empty_like(x), h=h)
        before = x.clone()
        flat, step = torch.zeros((t + 1) * k, dtype=BF16, device="cuda"), k if t > 1 else k // 2
        near, behind = flat[:t * k].view(t, k), flat[step:step + t * k].view(t, k)  # a row apart (half of one)
        wide = torch.zeros(t, 3 * k, dtype=BF16, device="cuda")
        for call in (lambda: ad.forward(x, x, ids), lambda: ad.forward(x, before, ids, out=x), lambda: ad.forward(near, behind, ids),
                     lambda: ad.forward(x, near, ids, out=behind), lambda: ad.forward(x, behind, ids, out=near),
                     lambda: ad.forward(wide[:, :k], wide[:, k // 2:k // 2 + k], ids),
                     lambda: ad.forward(x, before, ids, h=x.view(-1)[:t * r * 2].view(F32).view(t, r))):
            with pytest.raises(ts.TsError):
                call()
        torch.cuda.synchronize()
        assert torch.equal(x, before) and (flat == 0).all() and (wide == 0).all()
        assert torch.equal(ad.forward(x, x, ids, out=torch.empty_like(x)), want)
        wide[:, :k], wide[:, k:2 * k] = x, x
        got = ad.forward(wide[:, :k], wide[:, k:2 * k], ids, out=wide[:, 2 * k:])
        assert torch.equal(got, want) and torch.equal(wide[:, :k], x) and torch.equal(wide[:, k:2 * k], x)
        ad.forward(wide[:, :k], wide[:, k:2 * k], ids)
        assert torch.equal(wide[:, k:2 * k], want) and torch.equal(wide[:, :k], x)
        # the backward pass
        dy = (0.1 * randn(gen(t), t, k)).to(BF16)
        want = ad.backward(dy, dy.clone(), ids, h, x, out=torch.empty_like(dy))
        before = dy.clone()
        for call in (lambda: ad.backward(dy, dy, ids, h, x), lambda: ad.backward(dy, before, ids, h, x, out=x),
                     lambda: ad.backward(dy, before, ids, h, x, out=dy)):
            with pytest.raises(ts.TsError):
                call()
        torch.cuda.synchronize()
        assert torch.equal(dy, before)
        assert all(torch.equal(p, q) for p, q in zip(ad.backward(dy, dy, ids, h, x, out=torch.empty_like(dy)), want))


def test_refusals(ts):
    x, y, a, b, scale, ids = case(70, 64, 72, 4, 3)
    ad = ts.Adapters(a, b, scale=scale)
    h, dy = torch.zeros(70, 4, device="cuda"), torch.zeros(70, 72, dtype=BF16, device="cuda")
    q, s, _ = kept_rows(ts, x)
    f8 = torch.float8_e4m3fn
    for error, call in (
        (TypeError, lambda: ts.Adapters(a.float(), b)), (ValueError, lambda: ts.Adapters(a, b[:2])),
        (ValueError, lambda: ts.Adapters(a, b[:, :3])), (ValueError, lambda: ts.Adapters(a.transpose(1, 2), b)),
        (ValueError, lambda: ts.Adapters(a, b, scale=scale[:2])), (TypeError, lambda: ts.Adapters(a, b, scale=scale.double())),
        (TypeError, lambda: ts.Adapters(a, b, ranks=scale)), (TypeError, lambda: ts.Adapters(a, b.cpu())),
        (TypeError, lambda: ad.forward(x.float(), y, ids)), (ValueError, lambda: ad.forward(x[:, :56], y, ids)),
        (ValueError, lambda: ad.forward(x, y[:, :64], ids)), (ValueError, lambda: ad.forward(x, y[:69], ids)),
        (TypeError, lambda: ad.forward(x, y.half(), ids)), (ValueError, lambda: ad.forward(x, y, ids[:69])),
        (TypeError, lambda: ad.forward(x, y, ids.long())), (TypeError, lambda: ad.forward(x, y, ids, out=y.float())),
        (ValueError, lambda: ad.forward(x, y, ids, h=h[:, :3])), (ValueError, lambda: ad.forward(x, y, ts.list_rows(ids, 2))),
        (TypeError, lambda: ad.backward(dy.float(), None, ids, h, x)), (ValueError, lambda: ad.backward(dy, None, ids, h, x[:, :32])),
        (ValueError, lambda: ad.backward(dy, None, ids, h, x, x_scale=s)), (ValueError, lambda: ad.backward(dy, None, ids, h, q)),
        (ValueError, lambda: ad.backward(dy, None, ids, h, q, x_scale=s[:, :69])),
        (ValueError, lambda: ad.backward(dy, None, ids, h, x, out=x)), (ValueError, lambda: ad.backward(dy, None, ids, h, x, accumulate=True)),
        (TypeError, lambda: ad.backward(dy, None, ids, h, x.to(torch.float16))), (ValueError, lambda: ts.list_rows(ids[None], 3)),
        (ts.TsError, lambda: ts.list_rows(ids, 256)), (ts.TsError, lambda: ts.list_rows(ids, 0)),
        (ts.TsError, lambda: ad.forward(torch.zeros(70, 72, dtype=BF16, device="cuda")[:, 4:68], y, ids)),
        (ts.TsError, lambda: ts.Adapters(a.new_zeros(3, 129, 64), b.new_zeros(3, 129, 72)).forward(x, y, ids)),
        (ts.TsError, lambda: ts.Adapters(a.new_zeros(256, 4, 64), b.new_zeros(256, 4, 72)).forward(x[:4], y[:4], ids[:4])),
        (ts.TsError, lambda: ts.Adapters(a.new_zeros(3, 4, 60), b).forward(x[:, :60].contiguous(), y, ids)),
    ):
        with pytest.raises(error):
            call()
    assert f8 is E4M3
