"""Updates made orthogonal, against the definition in 64 bits.

Exact: matrices of few entries +-1 with 4^k of them in all have the norm 2^k, and one step with coefficients that are short binary fractions is a short binary fraction in every
element, so that results are equal to the rounded definition.

Tolerances of iterations.  An iterate X is held in two fp16 numbers (2^-22 of each element is left out), for bf16 results in one where the first coefficients of the steps
to come multiply to less than 16; its square A and the polynomial B in fp16 off their diagonals, which
are held in fp32, and products take the first numbers (bf16 results), or the same in two fp16 numbers (others).  Sums are in fp32, with errors below those.  The model rounds in the
same places in 64-bit arithmetic; two computations that round there and differ in the last bits of their sums are each as far from the definition, so they differ by no more
than the sum of both; twice that and the output's rounding is allowed, as a 2-norm.
"""
import math

import pytest
import torch

from gpu_util import ctx, say
from test_gpu_gated import rounded
from test_gpu_layer8 import BF16, F16, F32, TYPES, UNIT, gen

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
STEP = (3.4445, -4.7750, 2.0315)


def definition(G, steps, coef, planes=0):
    """planes: fp16 numbers of A and B (0: as they are)."""
    def held(v, n):
        w = v * 8192.0
        out = torch.zeros_like(w)
        for _ in range(n):
            out = out + (w - out).to(F32).to(F16).double()
        return out / 8192.0 if n else v

    def apart(v):
        d = torch.diag(torch.diag(v))
        return d + held(v - d, planes)

    X = G.double()
    norm = torch.linalg.matrix_norm(X)
    X = held(torch.where(norm > 0, X / norm, 0.0), 2 if planes else 0)
    wide = X.shape[0] <= X.shape[1]
    grows = [math.prod(max(1.0, abs(c[0])) for c in coef[s:steps]) for s in range(steps)]
    for s in range(steps):
        a, b, c = [float(torch.tensor(v, dtype=F32)) for v in coef[s]]
        X = held(X, 1) if planes == 1 and grows[s] < 16.0 else X
        H = held(X, planes)
        A = apart(H @ H.t() if wide else H.t() @ H)
        B = apart(b * A + c * (A @ A))
        d = torch.diag(torch.diag(B))
        X = a * X + (d @ X + (B - d) @ H if wide else X @ d + H @ (B - d))
        if s + 1 < steps:
            X = held(X, 2 if planes else 0)
    return X


def iterated(g, steps=5, coef=None, got=None):
    coef = coef or [STEP] * steps
    got = ctx().rsvd_orthogonalize(g, steps, coef) if got is None else got
    assert got.dtype == g.dtype and got.shape == g.shape
    want = definition(g, steps, coef)
    planes = 1 if g.dtype == BF16 else 2
    model = definition(g, steps, coef, planes)
    lost, norm = torch.linalg.matrix_norm(model - want), torch.linalg.matrix_norm(want)
    # (sums of up to n terms in fp32 in every product, where two fp16 numbers hold more than those)
    sums = 2.0 ** -24 * math.sqrt(max(g.shape)) * 16 * norm
    off = torch.linalg.matrix_norm(got.double() - want)
    assert float(off) <= float(4 * lost + sums + UNIT[g.dtype] * norm), (tuple(g.shape), float(off / norm), float(lost / norm))
    return got


def momentum(g, m, n, dtype):
    k = max(1, min(m, n) // 4)
    low = (torch.randn(m, k, device=DEV, generator=g) * torch.arange(1, k + 1, device=DEV) ** -0.5) @ torch.randn(k, n, device=DEV, generator=g)
    return (1e-3 * (low / low.square().mean().sqrt() + 0.5 * torch.randn(m, n, device=DEV, generator=g))).to(dtype)


SIZES = [(1, 1), (1, 40), (40, 1), (2, 3), (7, 5), (64, 64), (65, 130), (130, 65), (128, 500), (777, 333), (256, 2048), (1500, 257), (1024, 1024)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", SIZES)
def test_five_steps(dtype, m, n):
    say("orthogonalize", dtype, m, n)
    got = iterated(momentum(gen(m + n), m, n, TYPES[dtype]))
    s = torch.linalg.svdvals(got.double())
    assert float(s.max()) < 1.3


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(64, 200), (300, 70)])
def test_other_coefficients_and_steps(dtype, m, n):
    g = momentum(gen(m), m, n, TYPES[dtype])
    for coef in ([(1.5, -0.5, 0.0)], [(1.875, -1.25, 0.375)] * 8, [(3.4445, -4.775, 2.0315), (2.5, -2.0, 0.6), (1.875, -1.25, 0.375)]):
        iterated(g, len(coef), coef)
    a = ctx().rsvd_orthogonalize(g, 3, STEP)
    assert torch.equal(a, ctx().rsvd_orthogonalize(g, 3, [STEP] * 3)) and torch.equal(ctx().rsvd_orthogonalize(g), ctx().rsvd_orthogonalize(g, 5, STEP))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(200, 500), (700, 130)])
@pytest.mark.parametrize("kind", ["four large", "steep"])
def test_few_large_singular_values(dtype, m, n, kind):
    """What is lost of the large ones must not be taken for a part of the small ones: three orders of magnitude below, they grow 485 times as fast.  To within the rounding of
    the result (its unit) and half as much."""
    g, k = gen(m + n), 4 if kind == "four large" else min(m, n)
    fall = torch.ones(4, device=DEV) if kind == "four large" else torch.arange(1, k + 1, device=DEV) ** -1.5
    G = (torch.randn(m, k, device=DEV, generator=g) * fall) @ torch.randn(k, n, device=DEV, generator=g)
    G = (G + (1e-2 if kind == "four large" else 1e-3) * torch.randn(m, n, device=DEV, generator=g)).to(TYPES[dtype])
    got = iterated(G)
    want = definition(G, 5, [STEP] * 5)
    # (the rounding of a bf16 result is 1.7e-3 of its norm, what is lost of the iterates 1.6e-3)
    near = 1.5 * UNIT[BF16] / 2 if dtype == "bf16" else 1.5 * UNIT[F16] if dtype == "f16" else 2e-5
    assert float((got.double() - want).norm() / want.norm()) < near


def sparse(g, m, n, entries, dtype):
    """+-1 in 4^k places, columns and rows spread over all."""
    at = torch.randperm(m * n, device=DEV, generator=g)[:entries]
    out = torch.zeros(m * n, device=DEV)
    out[at] = torch.where(torch.rand(entries, device=DEV, generator=g) < 0.5, -1.0, 1.0)
    return out.view(m, n).to(dtype)


EXACT = [(16, 16, 64), (64, 64, 256), (65, 127, 256), (200, 90, 256), (1, 300, 256), (300, 1, 256), (513, 1000, 1024), (2000, 130, 1024), (100, 5000, 1024), (1025, 1025, 4096), (4000, 2100, 4096),
         (2048, 4096, 4096)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,entries", EXACT)
def test_one_step_is_exact(dtype, m, n, entries):
    say("orthogonalize exact", dtype, m, n)
    T = TYPES[dtype]
    G = sparse(gen(m + n), m, n, entries, T)
    for coef in ((1.5, -0.5, 0.0), (0.5, 0.0, 1.0), (1.0, 0.0, 0.0)):
        want = definition(G, 1, [coef])
        if min(m, n) == 1 and coef[2]:
            want = G.double() / G.double().norm() * 1.5
        assert torch.equal(ctx().rsvd_orthogonalize(G, 1, coef), rounded(want, T))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(50, 70), (300, 130), (128, 128), (33, 1000)])
def test_a_batch_is_its_matrices(dtype, m, n):
    T, g = TYPES[dtype], gen(m)
    G = torch.stack([momentum(g, m, n, T) * 10.0 ** (i - 1) for i in range(4)])
    G[2] = 0.0
    got = ctx().rsvd_orthogonalize(G)
    assert not got[2].any()
    for i in (0, 1, 3):
        iterated(G[i], got=got[i])
    # views: the batch inside the rows, rows of wider tensors, every other matrix; in place
    big = torch.full((m, 4, n + 5), 7.0, device=DEV, dtype=T)
    view = big.permute(1, 0, 2)[:, :, 2:n + 2]
    view.copy_(G)
    room = torch.full((8, m, n + 3), 7.0, device=DEV, dtype=T)
    out = room[::2, :, 1:n + 1]
    ctx().rsvd_orthogonalize(view, out=out)
    assert torch.equal(out, got) and bool((room[1::2] == 7).all()) and bool((room[:, :, 0] == 7).all()) and bool((room[:, :, n + 1:] == 7).all())
    assert bool((big[:, :, :2] == 7).all()) and bool((big[:, :, n + 2:] == 7).all())
    again = G.clone()
    assert ctx().rsvd_orthogonalize(again, out=again) is again and torch.equal(again, got)
    assert torch.equal(ctx().rsvd_orthogonalize(G[0].expand(3, m, n))[2], ctx().rsvd_orthogonalize(G[:1].expand(3, m, n).contiguous())[0])
    assert ctx().rsvd_orthogonalize(G[:0]).shape == (0, m, n)


@pytest.mark.parametrize("dtype", TYPES)
def test_scale_does_not_matter_and_what_is_not_finite_stays_in_its_matrix(dtype):
    T, g = TYPES[dtype], gen(3)
    G = momentum(g, 40, 90, F32) * 1e3
    for by in (2.0 ** -7, 2.0 ** 9) if dtype == "f16" else (2.0 ** -100, 2.0 ** 100):
        scaled = G.to(T) * by                             # (in fp16 some of these are subnormal numbers, rounded: what they are is what counts)
        assert torch.equal(ctx().rsvd_orthogonalize(scaled), ctx().rsvd_orthogonalize((scaled.double() / by).to(T)))
    both = torch.stack([G, G]).to(T)
    want = ctx().rsvd_orthogonalize(both)
    for bad in (math.nan, math.inf, -math.inf):
        both[0, 3, 4] = bad
        got = ctx().rsvd_orthogonalize(both)
        assert got[0].isnan().all() and torch.equal(got[1], want[1])


def test_singular_vectors_stay_and_values_come_near_one():
    """Against the library's own decomposition."""
    g = gen(8)
    G = momentum(g, 96, 300, F32)
    S, U, Vt, _ = ctx().rsvd_run(G, 96, 0, 3)
    O = ctx().rsvd_orthogonalize(G, 12, [STEP] * 4 + [(1.875, -1.25, 0.375)] * 8)
    # twelve steps take every singular value above 2e-3 of the norm to one; U and Vt are good to 1e-4 of what separates singular values here
    assert float(S.min() / G.norm()) > 2e-3
    assert float((O - U @ Vt).abs().max()) < 1e-2


def test_refusals():
    c, G = ctx(), torch.randn(3, 20, 30, device=DEV)
    for call in (lambda: c.rsvd_orthogonalize(G[0, 0]), lambda: c.rsvd_orthogonalize(G.cpu()), lambda: c.rsvd_orthogonalize(G, 0), lambda: c.rsvd_orthogonalize(G, 65),
                 lambda: c.rsvd_orthogonalize(G, 2, [STEP]), lambda: c.rsvd_orthogonalize(G, 2, (1.0, 2.0)), lambda: c.rsvd_orthogonalize(G.transpose(1, 2)),
                 lambda: c.rsvd_orthogonalize(G, out=G[:2]), lambda: c.rsvd_orthogonalize(G, out=torch.empty(3, 20, 30)), lambda: c.rsvd_orthogonalize(G[:, :0])):
        with pytest.raises(ValueError):
            call()
    from paper_2110_03423_amd import RsvdError
    for coef in ((4.0, 0.0, 0.0), (math.nan, 0.0, 0.0)):
        with pytest.raises(RsvdError):
            c.rsvd_orthogonalize(G, 3, coef)
    with pytest.raises(TypeError):
        c.rsvd_orthogonalize(G.double())
    out = torch.empty(3, 20, 30, device=DEV)[:1].expand(3, 20, 30)
    with pytest.raises(RsvdError):
        c.rsvd_orthogonalize(G, out=out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(20, 33), (64, 200), (300, 70), (1000, 520)])
def test_a_schedule_that_starts_steeply(dtype, m, n):
    """First coefficients above 4 and b x^2 + c x^4 down to -8.3.  (The first coefficients multiply to 1260, those of five equal steps to 485: of the sums' errors three times as
    much is left.)  Also of matrices of one magnitude, whose entries round alike and whose one singular value starts at the end of the range."""
    from test_dense_host import SCHEDULE
    steps = len(SCHEDULE)
    for kind in ("momentum", "one magnitude"):
        g = gen(m + n)
        G = momentum(g, m, n, TYPES[dtype])
        if kind != "momentum":
            G = (torch.where(torch.rand(m, 1, device=DEV, generator=g) < 0.5, -0.3, 0.3) * torch.where(torch.rand(1, n, device=DEV, generator=g) < 0.5, -1.0, 1.0)).to(TYPES[dtype])
        say("orthogonalize, steep", dtype, m, n, kind)
        got = ctx().rsvd_orthogonalize(G, steps, SCHEDULE)
        want, model = definition(G, steps, SCHEDULE), definition(G, steps, SCHEDULE, 1 if dtype == "bf16" else 2)
        lost, norm = torch.linalg.matrix_norm(model - want), torch.linalg.matrix_norm(want)
        off = torch.linalg.matrix_norm(got.double() - want)
        sums = 3 * 2.0 ** -24 * math.sqrt(max(m, n)) * 16 * norm
        assert float(off) <= float(4 * lost + sums + UNIT[G.dtype] * norm), (kind, float(off / norm), float(lost / norm))
        assert float(torch.linalg.svdvals(got.double()).max()) < 1.02


def test_coefficients_come_as_three_for_each_step():
    c, G = ctx(), momentum(gen(6), 40, 70, F32)
    want = c.rsvd_orthogonalize(G, 2, [STEP, (1.5, -0.5, 0.0)])
    both = torch.tensor([STEP, (1.5, -0.5, 0.0)])
    for coef in (both, both.double().numpy(), tuple(map(tuple, both.tolist())), [torch.tensor(STEP), [1.5, -0.5, 0.0]]):
        assert torch.equal(c.rsvd_orthogonalize(G, 2, coef), want)
    for coef in (torch.tensor(STEP), list(STEP), torch.tensor(STEP).numpy()):
        assert torch.equal(c.rsvd_orthogonalize(G, 2, coef), c.rsvd_orthogonalize(G, 2, STEP))
    for coef in ([(1.5, -0.5), (0.0, 1.5, -0.5, 0.0)], [(1.5, -0.5, 0.0, 1.5, -0.5, 0.0), ()], [], [STEP] * 3, (1.5, -0.5, 0.0) * 2, [STEP, 1.0, 2.0]):
        with pytest.raises(ValueError):
            c.rsvd_orthogonalize(G, 2, coef)
    for steps in (2.5, "2", None):
        with pytest.raises((ValueError, TypeError)):
            c.rsvd_orthogonalize(G, steps, STEP)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n", [(16, 131072), (131072, 16), (256, 65536)])
def test_sums_of_many_equal_numbers_stay_in_the_range(dtype, m, n):
    """One singular value, at the end of the range; the last steps make up for what the first are off by, so that the rounding of the result and 2^-10 are left."""
    from test_dense_host import SCHEDULE
    say("orthogonalize, equal numbers", dtype, m, n)
    G = torch.full((m, n), 0.3, device=DEV, dtype=TYPES[dtype])
    G[:, ::2] *= -1
    got = ctx().rsvd_orthogonalize(G, len(SCHEDULE), SCHEDULE)
    want = G.double() / G.double().norm()
    assert float((got.double() - want).norm()) < UNIT[G.dtype] + 2.0 ** -10
