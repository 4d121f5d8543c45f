"""The gated block's operators at the ends of their ranges: rows far apart, more numbers than 32 bits count, gates that overflow squares, sums added to in ranges, rows that are
not finite in large tiles.  Integers that every type holds make results equal, bit for bit, however they are summed (bounds: the largest sums stay below 2^24)."""
import math

import pytest
import torch

from gpu_util import ctx, say
from test_gpu_f8 import weight_values
from test_gpu_gated import ACTS, E, FLOOR, UNIT, act64, block, integers, rounded, share, slopes64
from test_gpu_layer8 import BF16, F16, F32, TYPES, gen
from test_gpu_orthogonalize import iterated, momentum

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t", [26, 70])
def test_large_and_small_gates(dtype, act, t):
    """g as it is out of the product, up 1: values and slopes stay finite where g, its square or cube, or exp(g), leave fp32.  (Bounds: those of the activation, whose terms
    stop to matter at |g| = 200, where a share is 0 or 1; what is below 1e-30 may be lost.)"""
    T = TYPES[dtype]
    some = [0.0, 1e-4, 1.0, 10.0, 30.0, 88.0, 89.0, 200.0, 1e4, 5e4] + ([] if dtype == "f16" else [1e10, 1e19, 3e19, 1e25, 1e35, 3e38])
    v = torch.tensor([s * a for a in some for s in (1.0, -1.0)], device=DEV)
    v = v[torch.arange(t, device=DEV) % len(v)].to(T)
    x = torch.zeros(t, 8, device=DEV, dtype=T)
    x[:, 0], x[:, 1] = v, 1.0
    w = torch.zeros(2, 8, device=DEV, dtype=T)
    w[0, 0], w[1, 1] = 1.0, 1.0
    dh = torch.ones(t, 1, device=DEV, dtype=T)
    g = v.double()
    a, s, sm = act64(g, act)
    short = g.clamp(-200, 200)
    u, lost = UNIT[T], max(1e-30, 2 * FLOOR[T])
    say("gates", dtype, act, t)
    h, kept = ctx().rsvd_gated_product(x, w, act, keep=True)
    assert torch.equal(kept[:, 0], v) and bool(((h[:, 0].double() - a).abs() <= (share(short) + 4 * E + u) * 1.01 * a.abs() + lost).all())
    for k in (None, kept):
        dx, _ = ctx().rsvd_gated_product_grad(dh, x, w, act, kept=k, out=(torch.empty_like(x), None))
        e0 = (share(short) * (1 + short.abs()) + 4 * E) * sm.clamp(max=300.0) + 2 * u * s.abs()
        assert bool(((dx[:, 0].double() - s).abs() <= e0 + lost).all())
        assert bool(((dx[:, 1].double() - a).abs() <= (share(short) + 4 * E + 2 * u) * 1.01 * a.abs() + lost).all())


def far(rows, cols, ld, dtype):
    return torch.empty((rows - 1) * ld + cols, device=DEV, dtype=dtype).as_strided((rows, cols), (ld, 1))


@pytest.mark.parametrize("t", [20, 300])
def test_rows_far_apart(t):
    """The largest leading dimension of operands that are read where they lie, and one more; results and others lie further apart still."""
    say("far apart", t)
    g, n, m = gen(t), 72, 70
    a, b, c = block(g, t, n, m, BF16)
    want, kept = ctx().rsvd_gated_product(a, b, keep=True)
    grads = ctx().rsvd_gated_product_grad(c, a, b, kept=kept)
    for ld in (1 << 22, (1 << 22) + 8):
        x, w, h = far(t, n, ld, BF16), far(2 * m, n, ld, BF16), far(t, m, ld + 3, BF16)
        x.copy_(a), w.copy_(b)
        assert torch.equal(ctx().rsvd_gated_product(x, w, out=h), want)
        h.copy_(c)
        for got, expected in zip(ctx().rsvd_gated_product_grad(h, x, w, kept=kept), grads):
            assert torch.equal(got, expected)
        del w
        dw = far(2 * m, n, ld + 1, BF16)
        ctx().rsvd_gated_product_grad(h, x, b, out=(None, dw))
        assert torch.equal(dw, ctx().rsvd_gated_product_grad(c, a, b)[1])
        del dw, h
        f = ctx().rsvd_f8_weight(b)
        y = far(t, 2 * m, ld + 5, BF16)
        assert torch.equal(ctx().rsvd_f8_product(x, f, out=y), ctx().rsvd_f8_product(a, f))
        assert torch.equal(ctx().rsvd_f8_weight_grad(y, x), ctx().rsvd_f8_weight_grad(y.contiguous(), a))
        del x, y
    torch.cuda.empty_cache()


def test_more_numbers_than_32_bits_count():
    t, n, m, last = (1 << 20) + 131, 64, 4100, (1 << 20) - 128
    g, c = gen(7), ctx()
    x, w = integers(g, (t, n), BF16), integers(g, (2 * m, n), BF16, 1, 0.5)
    dh = torch.zeros(t, m, device=DEV, dtype=BF16)
    dh[last:] = integers(g, (t - last, m), BF16, 1, 0.2)
    assert dh.numel() > 1 << 32
    say("gated, past 32 bits")
    h = c.rsvd_gated_product(x, w, "relu")
    assert torch.equal(h[last:], c.rsvd_gated_product(x[last:], w, "relu")) and torch.equal(h[:300], c.rsvd_gated_product(x[:300], w, "relu"))
    del h
    dx, dw = c.rsvd_gated_product_grad(dh, x, w, "relu")
    want, dw_want = c.rsvd_gated_product_grad(dh[last:], x[last:], w, "relu")
    assert torch.equal(dx[last:], want) and not dx[:last].any() and torch.equal(dw, dw_want)
    del dx, dw, want, dw_want
    say("8-bit floats, past 32 bits")
    f = c.rsvd_f8_weight(w[:m])
    y = c.rsvd_f8_product(x, f)
    assert torch.equal(y[last:], c.rsvd_f8_product(x[last:], f)) and torch.equal(y[:300], c.rsvd_f8_product(x[:300], f))
    del y
    dx = c.rsvd_f8_product_grad(dh, f)
    assert torch.equal(dx[last:], c.rsvd_f8_product_grad(dh[last:], f)) and not dx[:last].any()
    assert torch.equal(c.rsvd_f8_weight_grad(dh, x), c.rsvd_f8_weight_grad(dh[last:], x[last:]))
    del dh, dx
    torch.cuda.empty_cache()


def test_a_batch_of_more_numbers_than_32_bits_count():
    say("orthogonalize, past 32 bits")
    batch, m, n = 2051, 16, 131072
    G = torch.zeros(batch, m, n, device=DEV, dtype=BF16)
    assert G.numel() > 1 << 32
    for i in (0, batch - 1):
        G[i] = momentum(gen(i), m, n, BF16)
    got = ctx().rsvd_orthogonalize(G)
    for i in (0, batch - 1):
        iterated(G[i], got=got[i])
    assert not got[1:-1].any()
    del G, got
    torch.cuda.empty_cache()


def test_as_many_matrices_as_a_launch_takes():
    """Small tiles would be more than a launch has workgroups."""
    say("orthogonalize, 65535 matrices")
    G = torch.zeros(65535, 1, 4100, device=DEV, dtype=BF16)
    G[:, 0, torch.arange(4)] = 0.5
    G[::2] *= -1
    got = ctx().rsvd_orthogonalize(G, 1, (1.0, 0.0, 0.0))
    assert torch.equal(got, G)


# (chosen: whole tiles, ranges of k, and both)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,m", [(65, 8, 8), (1000, 136, 2048), (4100, 200, 200), (8200, 80, 1600)])
def test_sums_are_added_to_in_whatever_tiles(dtype, t, n, m):
    T, g = TYPES[dtype], gen(t + n)
    x, w, dh = integers(g, (t, n), T), integers(g, (2 * m, n), T, 1, min(1.0, 24.0 / n)), integers(g, (t, m), T, 1, min(1.0, 200.0 / max(t, m)))
    base = torch.randint(-100, 101, (2 * m, n), device=DEV, generator=g).float()
    say("added to", dtype, t, n, m)
    once = torch.empty_like(base)
    ctx().rsvd_gated_product_grad(dh, x, w, "relu", out=(None, once))
    both = base.clone()
    ctx().rsvd_gated_product_grad(dh, x, w, "relu", out=(None, both), accumulate=True)
    assert torch.equal(both, base + once) and once.any()
    once = ctx().rsvd_f8_weight_grad(dh, x, out=torch.empty(m, n, device=DEV))
    assert torch.equal(once.double(), dh.double().t() @ x.double())
    both = base[:m].clone()
    ctx().rsvd_f8_weight_grad(dh, x, out=both, accumulate=True)
    assert torch.equal(both, base[:m] + once)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,m", [(300, 1096, 2000), (2048, 512, 2048), (2100, 264, 4100)])
def test_what_is_not_finite_stays_in_its_rows_of_large_tiles(dtype, t, n, m):
    T, g = TYPES[dtype], gen(t)
    x, w, dh = block(g, t, n, m, T)
    bad = [7, 130, t - 1]
    keep = torch.ones(t, dtype=torch.bool, device=DEV)
    keep[bad] = False
    y, d = x.clone(), dh.clone()
    y[bad, 5], d[bad, 3] = torch.tensor([math.nan, math.inf, math.nan], device=DEV, dtype=T), math.nan
    say("not finite", dtype, t, n, m)
    f = ctx().rsvd_f8_weight(w[:m])
    for run, clean, broken in ((lambda v: ctx().rsvd_gated_product(v, w), x, y), (lambda v: ctx().rsvd_gated_product_grad(v, x, w, out=(torch.empty_like(x), None))[0], dh, d),
                               (lambda v: ctx().rsvd_f8_product(v, f), x, y), (lambda v: ctx().rsvd_f8_product_grad(v, f), dh, d)):
        want, got = run(clean), run(broken)
        assert torch.equal(got[keep], want[keep]) and not got[bad].isfinite().any()


@pytest.mark.parametrize("t,n,m", [(100, 67, 20), (700, 70, 330)])
def test_large_fp32_numbers_and_infinities_stay_in_their_columns(t, n, m):
    """Numbers above 3.39e38 round to infinity in bf16: their parts are taken otherwise.  (Bound: what D is off by, times the large number - of a gate of -10 its
    activation is good to 1e-4 only -, 2^-22 of that term for its product and the output's rounding, and the others beside it.)"""
    g = gen(t)
    x, w, dh = block(g, t, n, m, F32)
    kept = ctx().rsvd_gated_product(x, w, keep=True)[1]
    dx, dw = ctx().rsvd_gated_product_grad(dh, x, w, kept=kept)
    for value in (math.inf, -math.inf, math.nan, 3.4e38):
        say("large", t, n, m, value)
        v, y = w.clone(), x.clone()
        v[3, 5], y[9, n - 1] = value, value
        other, _ = ctx().rsvd_gated_product_grad(dh, x, v, kept=kept)
        _, again = ctx().rsvd_gated_product_grad(dh, y, w, kept=kept)
        keep = [c for c in range(n) if c != 5]
        assert torch.equal(other[:, keep], dx[:, keep]) and torch.equal(again[:, :n - 1], dw[:, :n - 1])
        if not math.isfinite(value):
            assert not other[:, 5].isfinite().any() and not again[:, n - 1].isfinite().any()
            continue
        none = torch.zeros(t, m, device=DEV, dtype=torch.float64)
        d, ed = slopes64(kept[:, :m].double(), kept[:, m:].double(), none, none, dh, "silu")
        for got, one, off, rest in ((other[:, 5], d[:, 3] * v[3, 5].double(), ed[:, 3], d.abs() @ w.double().abs()[:, 5]),
                                    (again[:, n - 1], d[9] * y[9, n - 1].double(), ed[9], d.abs().t() @ x.double().abs()[:, n - 1])):
            assert bool(((got.double() - one).abs() <= 2.0 ** -22 * one.abs() + off * value + 2 * rest).all())


@pytest.mark.parametrize("keep", [False, True])
def test_the_range_of_fp16_gradients_is_found_behind_32_bits(keep):
    """The one large gradient is the last number of more than 2^32: without it D would be 2^16 times too large for fp16."""
    t, n, m = (1 << 20) + 131, 16, 4100
    g, c = gen(8), ctx()
    x, w = integers(g, (t, n), F16), integers(g, (2 * m, n), F16, 1, 0.5)
    dh = torch.zeros(t, m, device=DEV, dtype=F16)
    dh[-1], dh[5, 7] = 2.0 ** 13, 2.0 ** -8
    assert dh.numel() > 1 << 32
    say("fp16 range, past 32 bits", keep)
    kept = c.rsvd_gated_product(x, w, "relu", keep=True)[1] if keep else None
    dx, dw = torch.empty_like(x), torch.empty(2 * m, n, device=DEV)
    c.rsvd_gated_product_grad(dh, x, w, "relu", kept=kept, out=(dx, dw))
    del kept
    rows = [5, t - 1]
    gu = x[rows].double() @ w.double().t()
    a, u = gu[:, :m].clamp(min=0), gu[:, m:]
    d = torch.cat([dh[rows].double() * u * (a > 0), dh[rows].double() * a], dim=1)
    assert float(d.abs().max()) > 65504
    assert torch.equal(dw.double(), d.t() @ x[rows].double()) and torch.equal(dx[rows], rounded(d @ w.double(), F16)) and int((dx != 0).any(dim=1).sum()) <= 2
    del dh, dx, dw, x
    torch.cuda.empty_cache()
