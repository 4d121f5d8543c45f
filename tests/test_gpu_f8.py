"""Products in 8-bit floats against their definitions in 64 bits.

Codes and powers are exact: the definition names no rounding but the one to a code.  Of the products, with K the number of terms:
  * fp32 results: exact products of bf16 numbers, (K + 64) 2^-24 |X^||W^|^T.
  * 16-bit results: the matrix instruction for 8-bit floats takes eight k at a time and cuts each product off, towards zero, below 2^-13 of the power of two of the largest
    of them (found with single products: 2^3 is kept beside 2^16 and 2^2 is not; products of other eights keep their bits).  The largest one is whole, so at most
    7 x 2^-13 of it is lost: 7 x 2^-13 |X^||W^|^T in all, beside the fp32 sums.
The output rounds once more.  Integers whose products span few bits are exact in every type.
"""
import math

import pytest
import torch

from gpu_util import ctx, say
from test_gpu_gated import check, integers, rounded
from test_gpu_layer8 import BF16, E, F16, F32, TYPES, activations, gen

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
DEV = "cuda:0"


def blocks64(x, rows, cols):
    """Codes' values times their powers, the exponents' bytes, by the definition; codes as numbers."""
    x = x.double().cpu()
    t, n = x.shape
    a, b = -(-t // rows), -(-n // cols)
    p = torch.zeros(a * rows, b * cols, dtype=torch.float64)
    p[:t, :n] = x
    p = p.view(a, rows, b, cols)
    top = p.abs().amax(dim=(1, 3), keepdim=True)
    bad = ~torch.isfinite(top)
    f, e = torch.frexp(torch.where(bad, 1.0, top))
    e = torch.clamp(e - 9 + (f > 0.875), min=-126)
    e = torch.where(top == 0, -126, e)
    v = torch.where(bad, math.nan, p * torch.exp2(-e.double()))
    # to three bits behind the leading one, steps of 2^-9 at the least
    step = torch.exp2(torch.clamp(torch.frexp(v.nan_to_num())[1] - 1, min=-6).double() - 3)
    code = torch.where(bad, math.nan, torch.round(v / step) * step)
    byte = torch.where(bad, 255, e + 127)
    code = code.view(a * rows, b * cols)[:t, :n]
    value = code * torch.exp2(e.double()).expand(a, rows, b, cols).reshape(a * rows, b * cols)[:t, :n]
    return value.to(DEV), byte[:, 0, :, 0].to(torch.uint8).to(DEV), code.to(DEV)


def same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(), b.nan_to_num())


def weight_values(w):
    return w.codes.double() * torch.exp2(w.powers.double() - 127).repeat_interleave(128, 0).repeat_interleave(128, 1)[:w.m, :w.n]


def product_check(got, x, w, what):
    """got against x w^T for values x, w that are held exactly."""
    want, both = x @ w.t(), x.abs() @ w.abs().t()
    check(got, want, ((x.shape[1] + 64) * E + (0.0 if got.dtype == F32 else 7 * 2.0 ** -13)) * both, what)


def weight(g, m, n, dtype=F32):
    w = torch.randn(m, n, device=DEV, generator=g) * torch.exp(0.5 * torch.randn(m, 1, device=DEV, generator=g))
    return w.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(1, 1), (127, 129), (128, 128), (130, 70), (300, 1000), (5, 2049), (513, 3)])
def test_a_weight_in_both_orders(dtype, m, n):
    say("f8 weight", dtype, m, n)
    w = weight(gen(m + n), m, n, TYPES[dtype])
    w[0, 0] = 0.0
    if m > 2 and n > 2:
        w[1, 1] = 2.0 ** -20
        w[m - 1, n - 1] = 449.0
    h = ctx().rsvd_f8_weight(w)
    _, byte, code = blocks64(w, 128, 128)
    assert torch.equal(h.powers, byte) and torch.equal(h.codes.double(), code)
    from paper_2110_03423_amd import WeightF8
    other = WeightF8(h.codes, h.powers)
    for mine, theirs in ((h._forward, other._forward), (h._backward, other._backward)):
        assert torch.equal(mine[0], theirs[0])
        blocks = -(-(n if mine is h._forward else m) // 128)
        assert torch.equal(mine[1][:, :blocks], theirs[1][:, :blocks])
    assert ctx().rsvd_f8_weight(w, backward=False)._backward is None


@pytest.mark.parametrize("dtype", TYPES)
def test_rounding_at_the_edges(dtype):
    """Halves between codes, the largest code, subnormal codes and numbers, zeros: by way of products with the unit matrix, which return what X is held as."""
    T = TYPES[dtype]
    unit = ctx().rsvd_f8_weight(torch.eye(256, device=DEV, dtype=F32))
    g = gen(5)
    rows = [torch.zeros(256), torch.arange(256).double() / 16 + 1, 448 * torch.ones(256), torch.full((256,), 2.0 ** -14), torch.linspace(-1, 1, 256),
            torch.exp2(torch.arange(256).remainder(24).double() - 20), 1.75 + torch.arange(256) / 2.0 ** 8, 256 - torch.arange(256) / 4.0,
            (2 * torch.arange(256).remainder(8) + 17) / 16.0 * 2.0 ** (torch.arange(256) // 8 - 24).double()]
    if dtype != "f16":
        rows += [torch.full((256,), 1e-38), torch.exp2(-torch.arange(256).remainder(126).double()), torch.full((256,), 1e38)]
    for t in (len(rows), 80):
        x = torch.stack([r.double() for r in rows]).to(DEV)
        x = torch.cat([x, torch.randn(max(0, t - len(rows)), 256, device=DEV, generator=g, dtype=torch.float64)]).to(T)
        value, _, _ = blocks64(x, 1, 128)
        got = ctx().rsvd_f8_product(x, unit)
        small = value.abs() < 2.0 ** -126                 # (fp32 and bf16 sums of those may be zeros)
        assert torch.equal(got[~small], value[~small].to(T)) and float(got[small].abs().max() if small.any() else 0) < 2.0 ** -125


SIZES = [(1, 1, 1), (1, 128, 16), (2, 300, 17), (16, 1000, 200), (17, 257, 130), (32, 2200, 35), (33, 4096, 100), (64, 129, 1000), (65, 128, 128), (66, 5, 300), (200, 1000, 129), (513, 640, 384),
         (1025, 333, 777)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,m", SIZES)
def test_product_and_gradients(dtype, t, n, m):
    say("f8", dtype, t, n, m)
    T, g = TYPES[dtype], gen(t + n + m)
    x, dy, w = activations(g, t, n, T), activations(g, t, m, T, 0.3), ctx().rsvd_f8_weight(weight(g, m, n))
    W = weight_values(w)
    product_check(ctx().rsvd_f8_product(x, w), blocks64(x, 1, 128)[0], W, "Y")
    product_check(ctx().rsvd_f8_product_grad(dy, w), blocks64(dy, 1, 128)[0], W.t(), "dX")
    a, b = blocks64(dy, 128, 1)[0].t(), blocks64(x, 128, 1)[0].t()
    product_check(ctx().rsvd_f8_weight_grad(dy, x), a, b, "dW")
    f32 = torch.empty(m, n, device=DEV)
    assert ctx().rsvd_f8_weight_grad(dy, x, out=f32) is f32
    product_check(f32, a, b, "dW in fp32")
    more = torch.full_like(f32, 0.25)
    ctx().rsvd_f8_weight_grad(dy, x, out=more, accumulate=True)
    assert torch.equal(more, f32 + 0.25)


EXACT = [(1, 4096, 48), (15, 200, 4000), (25, 1500, 1000), (32, 9000, 20), (12, 8200, 8192), (6, 8200, 8192), (40, 16384, 33), (64, 640, 130), (65, 16384, 64), (129, 4097, 129), (300, 1100, 1000), (1000, 130, 2048), (2048, 512, 2048), (4100, 200, 4000),
         (8200, 129, 1600), (6000, 2000, 256)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,m", EXACT)
def test_integers_are_exact(dtype, t, n, m):
    """Integers up to 2 in every block (so up to 448 / 256 of them are codes): sums are exact in any order, whatever the tile and the ranges of k."""
    say("f8 integers", dtype, t, n, m)
    T, g = TYPES[dtype], gen(t + 2 * n + m)
    x, dy, w = integers(g, (t, n), T), integers(g, (t, m), T, 2, 0.3), integers(g, (m, n), F32, 2, 0.2)
    h = ctx().rsvd_f8_weight(w)
    X, D, W = x.double(), dy.double(), w.double()
    assert torch.equal(ctx().rsvd_f8_product(x, h), rounded(X @ W.t(), T))
    assert torch.equal(ctx().rsvd_f8_product_grad(dy, h), rounded(D @ W, T))
    assert torch.equal(ctx().rsvd_f8_weight_grad(dy, x), rounded(D.t() @ X, T))
    f32 = torch.ones(m, n, device=DEV)
    ctx().rsvd_f8_weight_grad(dy, x, out=f32, accumulate=True)
    assert torch.equal(f32, (D.t() @ X + 1).float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [3, 20, 70])
def test_powers_of_blocks_are_taken_where_they_belong(dtype, t):
    """Blocks of very different size, of tokens and of the weight: each output sees them all."""
    T, g, n, m = TYPES[dtype], gen(t), 1300, 300
    e = (torch.arange(n, device=DEV) // 128 % 5 - 2).double()
    x = (torch.randn(t, n, device=DEV, generator=g) * torch.exp2(3 * e)).to(T)
    w = torch.randn(m, n, device=DEV, generator=g) * torch.exp2(-3 * e + (torch.arange(m, device=DEV) // 128 * 2)[:, None])
    h = ctx().rsvd_f8_weight(w.float())
    assert len(h.powers.unique()) > 4
    product_check(ctx().rsvd_f8_product(x, h), blocks64(x, 1, 128)[0], weight_values(h), "Y")
    tall = torch.cat([x * 2.0 ** (k % 3) for k in range(0, 700, t)])
    dy = torch.randn(len(tall), m, device=DEV, generator=g).to(T)
    product_check(ctx().rsvd_f8_weight_grad(dy, tall), blocks64(dy, 128, 1)[0].t(), blocks64(tall, 128, 1)[0].t(), "dW")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [4, 20, 150])
def test_infinities_and_nan(dtype, t):
    T, g = TYPES[dtype], gen(t)
    x, w = activations(g, t, 200, T), weight(g, 150, 200)
    h = ctx().rsvd_f8_weight(w)
    want = ctx().rsvd_f8_product(x, h)
    x[1, 3], x[2, 199] = math.inf, math.nan
    got = ctx().rsvd_f8_product(x, h)
    rest = [i for i in range(t) if i not in (1, 2)]
    assert got[1].isnan().all() and got[2].isnan().all() and torch.equal(got[rest], want[rest])
    w[0, 0] = -math.inf                                   # its block: 128 rows
    broken = ctx().rsvd_f8_weight(w)
    _, byte, _ = blocks64(w, 128, 128)
    assert torch.equal(broken.powers, byte) and broken.codes[:128, :128].float().isnan().all() and not broken.codes[128:].float().isnan().any()
    got = ctx().rsvd_f8_product(x, broken)
    assert got[:, :128].isnan().all() and torch.equal(got[rest, 128:], want[rest, 128:])
    dy = activations(g, t, 150, T)
    dw = ctx().rsvd_f8_weight_grad(dy, x)
    assert dw[:, 3].isnan().all() and dw[:, 199].isnan().all() and dw[:, [0, 1, 2, 4, 198]].isfinite().all()
    # a power of 255 in a weight of the caller's makes its block NaN, whatever the codes
    from paper_2110_03423_amd import WeightF8
    powers = h.powers.clone()
    powers[0, 1] = 255
    got = ctx().rsvd_f8_product(x, WeightF8(h.codes, powers))
    assert got[:, :128].isnan().all() and torch.equal(got[rest, 128:], want[rest, 128:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [5, 20, 90])
def test_views_with_other_strides(dtype, t):
    T, g, n, m = TYPES[dtype], gen(t), 131, 70
    h = ctx().rsvd_f8_weight(weight(g, m, n))
    for off, more in ((0, 5), (1, 3), (8, 16)):
        big = [torch.full((r, c + off + more), 7.0, device=DEV, dtype=T) for r, c in ((t, n), (t, m), (t, m), (t, n), (m, n))]
        x, dy, y, dx, dw = [b[:, off:b.shape[1] - more] for b in big]
        a, b = activations(g, t, n, T), activations(g, t, m, T)
        x.copy_(a), dy.copy_(b)
        ctx().rsvd_f8_product(x, h, out=y), ctx().rsvd_f8_product_grad(dy, h, out=dx), ctx().rsvd_f8_weight_grad(dy, x, out=dw)
        assert torch.equal(y, ctx().rsvd_f8_product(a, h)) and torch.equal(dx, ctx().rsvd_f8_product_grad(b, h)) and torch.equal(dw, ctx().rsvd_f8_weight_grad(b, a))
        for v in big:
            assert bool((v[:, :off] == 7).all()) and bool((v[:, v.shape[1] - more:] == 7).all())
        wide = torch.full((m, n + off + more), 9.0, device=DEV)
        wide[:, off:n + off].copy_(weight_values(h))
        assert torch.equal(ctx().rsvd_f8_weight(wide[:, off:n + off]).codes.float(), h.codes.float())


def test_no_tokens():
    h = ctx().rsvd_f8_weight(torch.randn(30, 20, device=DEV))
    x, dy = torch.empty(0, 20, device=DEV, dtype=BF16), torch.empty(0, 30, device=DEV, dtype=BF16)
    assert ctx().rsvd_f8_product(x, h).shape == (0, 30) and ctx().rsvd_f8_product_grad(dy, h).shape == (0, 20)
    dw = ctx().rsvd_f8_weight_grad(dy, x)
    assert dw.shape == (30, 20) and dw.dtype == BF16 and not dw.any()


def test_refusals():
    c, g = ctx(), gen(1)
    x, dy, h = activations(g, 9, 40, BF16), activations(g, 9, 30, BF16), ctx().rsvd_f8_weight(weight(g, 30, 40))
    from paper_2110_03423_amd import WeightF8
    forward, host = c.rsvd_f8_weight(weight(g, 30, 40), backward=False), WeightF8(h.codes.cpu(), h.powers.cpu())
    for call in (lambda: c.rsvd_f8_product(x[:, :39], h), lambda: c.rsvd_f8_product(x.cpu(), h), lambda: c.rsvd_f8_product(x, host), lambda: c.rsvd_f8_product_grad(dy, forward),
                 lambda: c.rsvd_f8_product(x, h, out=torch.empty(9, 30, device=DEV)), lambda: c.rsvd_f8_weight_grad(dy[:8], x), lambda: c.rsvd_f8_weight_grad(dy.float(), x),
                 lambda: c.rsvd_f8_weight_grad(dy, x, out=torch.empty(30, 40, device=DEV, dtype=F16)), lambda: c.rsvd_f8_weight_grad(dy, x, accumulate=True),
                 lambda: c.rsvd_f8_weight_grad(dy, x, out=torch.empty(30, 40, device=DEV, dtype=BF16), accumulate=True), lambda: c.rsvd_f8_weight(x.t()[:, ::2])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        c.rsvd_f8_product(x.double(), h)


def test_results_of_a_weight_may_not_lie_on_each_other():
    c, m, n = ctx(), 300, 260
    W = weight(gen(4), m, n).to(F32)
    room = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    base = room.data_ptr()
    base += -base % 256
    # (codes, powers; the same in the other order: 384 bytes of each row of codes, three rows of three powers, 4 apart)
    places = dict(q=base, p=base + (1 << 18), qt=base + (1 << 19), pt=base + (1 << 19) + (1 << 18))

    def call(**kw):
        a = dict(places, **kw)
        return c.lib.rsvd_f8_weight(c.h, None, 2, m, n, W.data_ptr(), n, a["q"], 384, a["p"], 4, a["qt"], 384, a["pt"], 4)

    assert call() == 0
    torch.cuda.synchronize()
    assert call(p=W.data_ptr()) == -10 and call(p=places["q"]) == -10 and call(p=places["q"] + 299 * 384 + 380) == -10 and call(p=places["q"] - 8) == -10
    assert call(pt=W.data_ptr()) == -14 and call(pt=places["q"]) == -14 and call(pt=places["qt"]) == -14 and call(pt=places["p"]) == -14 and call(pt=places["p"] + 8) == -14
    assert call(p=places["qt"]) == -12
    assert call(p=places["q"] + 300 * 384) == 0 and call(pt=places["p"] + 12) == 0
    torch.cuda.synchronize()
    h = c.rsvd_f8_weight(W)
    at = places["p"] - room.data_ptr()
    assert torch.equal(room[at + 12:at + 24].view(3, 4)[:, :3], h.powers.t())
