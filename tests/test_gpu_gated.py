"""The gated block against its definition in 64 bits.

Tolerances.  With u the unit roundoff of a type and e = 2^-24 that of fp32:
  * a product of n terms: (n + 64) e |X||W|^T; of fp32 numbers, which are three bf16 numbers each (the second at most 2^-8, the third 2^-16 of the number), six of the
    nine products are taken, 6 n terms, and less than 2^-23 |X||W|^T is left out.
  * the activation: its share of g is 1 / (1 + exp(-y)) or erfc(-g / sqrt 2) / 2.  exp(y) takes y rounded, times log2 e rounded, to 2^..: 3 e |y| relative, and 8 e for the
    operations around it; erfc(y) takes y to 2 e, which it multiplies by at most 2 y^2 + 2, and is good to 16 units.  All are below s(g) = 2^-22 (g^2 + |g|^3 / 4 + 2 |g| + 16), relative.
    Activations and their slopes change by at most 1.2 per unit of g (slopes: 1).
  * D = (dH u act', dH act) is rounded to the type.
Integers that are small enough make every operation exact: there results are equal, bit for bit, with the largest sums below 2^24.
"""
import math

import pytest
import torch

from gpu_util import ctx, say
from test_gpu_layer8 import BF16, E, F16, F32, FLOOR, TYPES, UNIT, activations, gen

pytestmark = pytest.mark.gpu

ACTS = ["silu", "gelu", "gelu_tanh", "relu"]
DEV = "cuda:0"


def act64(g, act):
    """Value and slope, and what the slope's terms add up to in magnitude."""
    if act == "relu":
        s = (g > 0).double()
        return g * s, s, s
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s)), s * (1 + g.abs() * (1 - s))
    if act == "gelu":
        s, p = torch.erfc(-g / math.sqrt(2)) / 2, torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return g * s, s + g * p, s + g.abs() * p
    r = math.sqrt(8 / math.pi)
    s = torch.sigmoid(r * g * (1 + 0.044715 * g * g))
    d = s * (1 - s) * r * (1 + 0.134145 * g * g)
    return g * s, s + g * d, s + g.abs() * d


def share(g):
    return 2.0 ** -22 * (g * g + g.abs() ** 3 / 4 + 2 * g.abs() + 16)


def product_bound(x, w):
    n, both = x.shape[1], x.double().abs() @ w.double().abs().t()
    return ((n + 64) * E if x.dtype != F32 else (6 * n + 64) * E + 2.0 ** -23) * both


def forward64(x, w, act):
    """(H, products) and their bounds before the output's rounding."""
    m = w.shape[0] // 2
    gu, bound = x.double() @ w.double().t(), product_bound(x, w)
    g, u, eg, eu = gu[:, :m], gu[:, m:], bound[:, :m], bound[:, m:]
    a, _, _ = act64(g, act)
    ea = 1.2 * eg + share(g) * (a.abs() + 1.2 * eg)
    return (a * u, gu), (ea * u.abs() + a.abs() * eu + ea * eu, bound)


def slopes64(g, u, eg, eu, dh, act):
    """D and its bound before it is rounded."""
    a, s, sm = act64(g, act)
    ea = 1.2 * eg + share(g) * (a.abs() + 1.2 * eg)
    es = eg + share(g) * (sm + 1.2 * eg) * (1 + g.abs())
    if act == "relu":
        es = (g.abs() <= eg).double()
    dh = dh.double()
    d = torch.cat([dh * u * s, dh * a], dim=1)
    bound = torch.cat([dh.abs() * (es * (u.abs() + eu) + s.abs() * eu), dh.abs() * ea], dim=1)
    return d, bound + 4 * E * d.abs()


def gradient64(dh, x, w, act, kept=None):
    m, t = w.shape[0] // 2, x.shape[0]
    if kept is None:
        (_, gu), (_, bound) = forward64(x, w, act)
    else:
        gu, bound = kept.double(), torch.zeros_like(kept, dtype=torch.float64)
    d, ed = slopes64(gu[:, :m], gu[:, m:], bound[:, :m], bound[:, m:], dh, act)
    if w.dtype != F32:
        ed = ed + UNIT[w.dtype] * (d.abs() + ed) + FLOOR[w.dtype]
    W, X = w.double(), x.double()
    parts, left = (6, 2.0 ** -23) if w.dtype == F32 else (1, 0.0)
    bx = ed @ W.abs() + ((parts * 2 * m + 64) * E + left) * ((d.abs() + ed) @ W.abs())
    bw = ed.t() @ X.abs() + ((parts * t + 64) * E + left) * ((d.abs() + ed).t() @ X.abs())
    return (d @ W, d.t() @ X), (bx, bw)


def check(got, want, bound, what):
    tol = bound + UNIT[got.dtype] * (want.abs() + bound) + FLOOR[got.dtype]
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((err / tol)[bad].max()), tuple(got.shape), bad.nonzero()[:4].tolist())


def block(g, t, n, m, dtype):
    x = activations(g, t, n, dtype, 0.5)
    w = (torch.randn(2 * m, n, device=DEV, generator=g) * (0.7 / n ** 0.5)).to(dtype)
    dh = (1e-2 * torch.randn(t, m, device=DEV, generator=g)).to(dtype)
    return x, w, dh


SIZES = [(1, 1, 1), (1, 256, 512), (3, 7, 5), (17, 130, 33), (32, 72, 100), (33, 1000, 70), (64, 96, 40), (65, 64, 64), (66, 31, 129), (200, 264, 100), (513, 1030, 350), (700, 72, 257)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t,n,m", SIZES)
def test_forward(dtype, act, t, n, m):
    say("gated", dtype, act, t, n, m)
    x, w, _ = block(gen(n + t), t, n, m, TYPES[dtype])
    h, kept = ctx().rsvd_gated_product(x, w, act, keep=True)
    (H, G), (bh, bg) = forward64(x, w, act)
    check(h, H, bh, "H")
    check(kept, G, bg, "kept")
    assert torch.equal(h, ctx().rsvd_gated_product(x, w, act))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t,n,m", SIZES)
@pytest.mark.parametrize("keep", [False, True])
def test_gradient(dtype, act, t, n, m, keep):
    say("gated gradient", dtype, act, t, n, m, keep)
    x, w, dh = block(gen(n + t), t, n, m, TYPES[dtype])
    kept = ctx().rsvd_gated_product(x, w, act, keep=True)[1] if keep else None
    dx, dw = ctx().rsvd_gated_product_grad(dh, x, w, act, kept=kept)
    (DX, DW), (bx, bw) = gradient64(dh, x, w, act, kept)
    check(dx, DX, bx, "dX")
    check(dw, DW, bw, "dW")
    # only one of them; the gradient of the weight in fp32, and added to what is there
    assert torch.equal(dx, ctx().rsvd_gated_product_grad(dh, x, w, act, kept=kept, out=(torch.empty_like(x), None))[0])
    f32 = torch.empty(2 * m, n, device=DEV)
    ctx().rsvd_gated_product_grad(dh, x, w, act, kept=kept, out=(None, f32))
    check(f32, DW, bw, "dW in fp32")
    if dtype != "f32":
        assert torch.equal(f32.to(TYPES[dtype]), dw)
    more = torch.full_like(f32, 0.5)
    ctx().rsvd_gated_product_grad(dh, x, w, act, kept=kept, out=(None, more), accumulate=True)
    assert torch.equal(more, f32 + 0.5)


def integers(g, shape, dtype, most=2, share_of=1.0):
    v = torch.randint(-most, most + 1, shape, device=DEV, generator=g).double()
    if share_of < 1.0:
        v *= torch.rand(shape, device=DEV, generator=g) < share_of
    return v.to(dtype)


def rounded(v, dtype):
    return v.to(F32).to(dtype)


# every tile and number of ranges that the choice knows, with last k-tiles of one to eight pieces, and operands that are laid out first
EXACT = [(1, 4096, 33), (9, 3, 20), (9, 4, 20), (70, 6, 33), (130, 61, 95), (77, 67, 31), (301, 999, 141), (30, 4001, 4096), (64, 100, 2100), (48, 72, 2049), (20, 5000, 64), (3, 40000, 33), (5, 20001, 50), (16, 1000, 130), (33, 40, 4000), (64, 2056, 640), (65, 8, 8), (100, 4104, 48), (129, 129, 129), (300, 1096, 1000), (1000, 136, 2048), (2048, 512, 2048),
         (4100, 200, 4000), (333, 16392, 50), (8200, 80, 1600)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,m", EXACT)
def test_integers_are_exact(dtype, t, n, m):
    """relu of integers: every product, sum and gradient is an integer that fp32 holds; results are those, rounded once."""
    say("gated integers", dtype, t, n, m)
    T, g = TYPES[dtype], gen(t + n + m)
    x, w = integers(g, (t, n), T), integers(g, (2 * m, n), T, 1, min(1.0, 24.0 / n))
    dh = integers(g, (t, m), T, 1, min(1.0, 200.0 / max(t, m)))
    gu = x.double() @ w.double().t()
    a, u, dh64 = gu[:, :m].clamp(min=0), gu[:, m:], dh.double()
    assert gu.abs().max() < 2048
    h, kept = ctx().rsvd_gated_product(x, w, "relu", keep=True)
    assert torch.equal(h, rounded(a * u, T)) and torch.equal(kept, rounded(gu, T))
    for k in (None, kept):
        if k is not None:
            a, u = k[:, :m].double().clamp(min=0), k[:, m:].double()
        d = torch.cat([dh64 * u * (a > 0), dh64 * a], dim=1)
        d = rounded(d, T).double()
        DX, DW = d @ w.double(), d.t() @ x.double()
        assert DX.abs().max() < 2 ** 24 and DW.abs().max() < 2 ** 24
        dx, dw = ctx().rsvd_gated_product_grad(dh, x, w, "relu", kept=k)
        assert torch.equal(dx, rounded(DX, T)) and torch.equal(dw, rounded(DW, T))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [5, 90])
def test_views_with_other_strides(dtype, t):
    """Columns out of wider tensors, at odd offsets; results into such; what lies around them stays."""
    T, g, n, m = TYPES[dtype], gen(t), 64, 24
    for off, more in ((0, 8), (1, 3), (8, 16), (3, 8)):
        big = [torch.full((r, c + off + more), 7.0, device=DEV, dtype=T) for r, c in ((t, n), (2 * m, n), (t, m), (t, m), (t, n), (2 * m, n), (t, 2 * m))]
        x, w, dh, h, dx, dw, kept = [b[:, off:b.shape[1] - more] for b in big]
        a, b, c = block(g, t, n, m, T)
        x.copy_(a), w.copy_(b), dh.copy_(c)
        ctx().rsvd_gated_product(x, w, "silu", out=h)
        assert torch.equal(h, ctx().rsvd_gated_product(a, b))
        kept.copy_(ctx().rsvd_gated_product(a, b, keep=True)[1])
        for k in (None, kept):
            ctx().rsvd_gated_product_grad(dh, x, w, kept=k, out=(dx, dw))
            for got, want in zip((dx, dw), ctx().rsvd_gated_product_grad(c, a, b, kept=None if k is None else k.contiguous())):
                assert torch.equal(got, want)
        for v in big:
            assert bool((v[:, :off] == 7).all()) and bool((v[:, v.shape[1] - more:] == 7).all())
    # rows that share their memory are no matrix
    from paper_2110_03423_amd import RsvdError
    with pytest.raises(RsvdError):
        ctx().rsvd_gated_product(block(g, 1, n, m, T)[0].expand(t, n), w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [4, 150])
def test_infinities_and_nan_stay_in_their_rows(dtype, t):
    g = gen(t)
    x, w, dh = block(g, t, 72, 40, TYPES[dtype])
    want, kept = ctx().rsvd_gated_product(x, w, keep=True)
    wx, _ = ctx().rsvd_gated_product_grad(dh, x, w, kept=kept)
    y = x.clone()
    y[1, 5], y[2, 71] = math.nan, math.inf
    got, other = ctx().rsvd_gated_product(y, w, keep=True)
    rest = [i for i in range(t) if i not in (1, 2)]
    assert got[1].isnan().all() and not got[2].isfinite().all() and torch.equal(got[rest], want[rest]) and other[1].isnan().all()
    d = dh.clone()
    d[1, 3] = math.nan
    dx, dw = ctx().rsvd_gated_product_grad(d, x, w, kept=kept)
    assert dx[1].isnan().all() and torch.equal(dx[[0, 2, 3]], wx[[0, 2, 3]]) and dw[3].isnan().all() and dw[43].isnan().all() and dw[4].isfinite().all()


def test_no_tokens():
    w = torch.randn(20, 12, device=DEV)
    x, dh = torch.empty(0, 12, device=DEV), torch.empty(0, 10, device=DEV)
    h, kept = ctx().rsvd_gated_product(x, w, keep=True)
    assert h.shape == (0, 10) and kept.shape == (0, 20)
    dx, dw = ctx().rsvd_gated_product_grad(dh, x, w)
    assert dx.shape == (0, 12) and torch.equal(dw, torch.zeros_like(w))
    more = torch.ones_like(w)
    ctx().rsvd_gated_product_grad(dh, x, w, out=(None, more), accumulate=True)
    assert bool((more == 1).all())
    b = ctx().rsvd_gated_product_grad(dh.bfloat16(), x.bfloat16(), w.bfloat16())[1]
    assert b.dtype == BF16 and not b.any()


@pytest.mark.parametrize("act", ACTS[:3])
def test_gradient_against_differences(act):
    """Directional differences of sum(H c) over fp32 blocks: (f(+h) - f(-h)) / 2 h, in 64 bits out of fp32 results."""
    g = gen(11)
    x, w, dh = block(g, 90, 48, 40, F32)
    dx, dw = ctx().rsvd_gated_product_grad(dh, x, w, act)
    vx, vw = torch.randn(x.shape, device=DEV, generator=g), torch.randn(w.shape, device=DEV, generator=g)
    f = lambda a, b: (ctx().rsvd_gated_product(a, b, act).double() * dh.double()).sum()
    # the step's cube over 6 times third derivatives (below 100 here), and rounding: 90 * 40 values of up to 10 e each, over the step
    h = 2.0 ** -7
    for v, z, d in ((vx, x, dx), (vw, w, dw)):
        diff = (f(x + h * v, w) - f(x - h * v, w)) / (2 * h) if z is x else (f(x, w + h * v * 0.1) - f(x, w - h * v * 0.1)) / (2 * h) * 10
        want = (d.double() * v.double()).sum()
        assert abs(float(diff - want)) <= 0.02 * float((d.double().abs() * v.double().abs()).sum().sqrt() + want.abs()), (float(diff), float(want))


def test_refusals():
    c, x, w, dh = ctx(), *block(gen(2), 9, 24, 16, BF16)
    bad = [lambda: c.rsvd_gated_product(x, w, "tanh"), lambda: c.rsvd_gated_product(x, w[:31]), lambda: c.rsvd_gated_product(x[:, :23], w),
           lambda: c.rsvd_gated_product(x.t(), w), lambda: c.rsvd_gated_product(x.cpu(), w), lambda: c.rsvd_gated_product(x, w.cpu()),
           lambda: c.rsvd_gated_product(x, w, out=torch.empty(9, 15, device=DEV, dtype=BF16)), lambda: c.rsvd_gated_product(x, w, out=torch.empty(9, 16, device=DEV)),
           lambda: c.rsvd_gated_product_grad(dh.float(), x, w), lambda: c.rsvd_gated_product_grad(dh[:8], x, w), lambda: c.rsvd_gated_product_grad(dh, x, w, accumulate=True),
           lambda: c.rsvd_gated_product_grad(dh, x, w, out=(None, torch.empty_like(w)), accumulate=True),
           lambda: c.rsvd_gated_product_grad(dh, x, w, out=(None, torch.empty(32, 24, device=DEV, dtype=F16))),
           lambda: c.rsvd_gated_product_grad(dh, x, w, kept=torch.empty(9, 31, device=DEV, dtype=BF16)),
           lambda: c.rsvd_gated_product(x, w, workspace=torch.empty(4, dtype=torch.uint8))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: c.rsvd_gated_product(x, w.half()), lambda: c.rsvd_gated_product(x.double(), w.double())):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("size", [1e-5, 1e-3, 2e3])
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("t,n,m", [(3, 70, 5), (40, 1030, 33), (65, 64, 30), (200, 264, 100), (513, 1030, 350), (2100, 300, 140), (1000, 2056, 1000)])
def test_fp16_gradients_of_any_size(t, n, m, keep, size):
    """D has to leave fp16's range on neither side: gradients that are subnormal numbers, and dH u above 65504 where dX is finite.  (Bound: D is rounded in fp16 times a power of two
    that brings what it can be at most, 1.14 max |dH| max |g, u|, to 2^15 or more, so that 2^-25 there is 2^-40 of that; of products computed again, which are known by the
    norms of rows, the most is 1.02 of those.)"""
    g = gen(t + n)
    x, w, _ = block(g, t, n, m, F16)
    x = (x * 6) if size > 1 else x
    dh = (size * torch.randn(t, m, device=DEV, generator=g)).to(F16)
    say("fp16 gradients", t, n, m, keep, size)
    kept = ctx().rsvd_gated_product(x, w, keep=True)[1] if keep else None
    dx, dw = torch.empty_like(x), torch.empty(2 * m, n, device=DEV)
    ctx().rsvd_gated_product_grad(dh, x, w, kept=kept, out=(dx, dw))
    if keep:
        gu, bound, most = kept.double(), torch.zeros(t, 2 * m, device=DEV, dtype=torch.float64), float(kept.double().abs().max())
    else:
        (_, gu), (_, bound) = forward64(x, w, "silu")
        most = 1.02 * float(x.double().norm(dim=1).max() * w.double().norm(dim=1).max())
    d, ed = slopes64(gu[:, :m], gu[:, m:], bound[:, :m], bound[:, m:], dh, "silu")
    if size > 1 and t > 3:
        assert float(d.abs().max()) > 65504
    ed = ed + UNIT[F16] * (d.abs() + ed) + 2.0 ** -40 * 1.14 * float(dh.double().abs().max()) * most
    W, X = w.double(), x.double()
    want, bx = d @ W, ed @ W.abs() + (2 * m + 64) * E * ((d.abs() + ed) @ W.abs())
    inside = (want.abs() + bx) * 1.001 < 65504
    assert float(inside.double().mean()) > 0.9
    tol = bx + UNIT[F16] * (want.abs() + bx) + FLOOR[F16]
    assert bool(((dx.double() - want).abs() <= tol)[inside].all()), float(((dx.double() - want).abs() / tol)[inside].max())
    check(dw, d.t() @ X, ed.t() @ X.abs() + (t + 64) * E * ((d.abs() + ed).t() @ X.abs()), "dW")
    if size < 1e-4 and t > 100:
        # what the rounding of D leaves of dW: as much as of larger gradients, 2^-11 at the most and 2^-11 / sqrt 3 on the whole
        assert float((dw.double() - d.t() @ X).norm() / (d.t() @ X).norm()) < 2.0 ** -11 / 3 ** 0.5


def test_fp16_gradients_of_zeros_and_of_what_is_not_finite():
    x, w, dh = block(gen(5), 70, 72, 40, F16)
    kept = ctx().rsvd_gated_product(x, w, keep=True)[1]
    for k in (None, kept):
        for z in ((torch.zeros_like(dh), x, w, k), (dh, torch.zeros_like(x), w, None), (dh, x, torch.zeros_like(w), None), (dh, x, w, torch.zeros_like(kept))):
            dx, dw = ctx().rsvd_gated_product_grad(*z[:3], kept=z[3])
            assert not dx.any() and not dw.any()
        want = ctx().rsvd_gated_product_grad(dh, x, w, kept=k)
        for bad in (math.inf, math.nan):
            d, y = dh.clone(), x.clone()
            d[4] = bad
            dx, dw = ctx().rsvd_gated_product_grad(d, x, w, kept=k)
            keep = [i for i in range(70) if i != 4]
            assert not dx[4].isfinite().any() and torch.equal(dx[keep], want[0][keep])
            y[4] = bad
            dx, dw = ctx().rsvd_gated_product_grad(dh, y, w, kept=k)
            assert torch.equal(dx[keep], want[0][keep]) and not dw[3].isfinite().any()


@pytest.mark.parametrize("t", [20, 32])
def test_few_tokens_of_a_weight_that_lies_otherwise_need_no_workspace(t):
    from paper_2110_03423_amd import Rsvd
    c, n, m = Rsvd(0), 6144, 4096
    x, w, _ = block(gen(t), t, n, m, BF16)
    wide = torch.zeros(2 * m, n + 4, device=DEV, dtype=BF16)
    wide[:, 2:n + 2] = w
    h = c.rsvd_gated_product(x, wide[:, 2:n + 2])
    assert not c._layer and c.rsvd_gated_product(x, w).shape == h.shape and c._layer
    (H, _), (bh, _) = forward64(x, w, "silu")
    check(h, H, bh, "H")
    check(c.rsvd_gated_product(x, w), H, bh, "H, in tiles")
