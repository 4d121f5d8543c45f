"""The layer operators at sizes that reach every kernel variant, with bounds that no sum without one of its terms keeps.

Sums.  Each of K additions in fp32 rounds a partial sum of k products by at most 2^-24 of it, a random walk whose standard deviation is 0.2 eps K times the
products' root mean square (eps = 2^-23).  Allowed is twenty times that: 4 eps sqrt(K) sqrt(A^2 B^2), A^2 and B^2 the matrices of squares.
Rounded operands.  A factor that is held to 2^-17 of itself (dY times a scale, the low-rank sums; of bf16 and fp16 tokens) is off by that at the most: four times
2^-17 sqrt(A^2 B^2), ten standard deviations.  For fp32 tokens it is 2^-24.
Epilogue.  Conversion, two scales, the low-rank sums added to what is there, and a bias: 4 eps sqrt(r + 8) of the parts' magnitudes.
Output.  With d the bound of all that and |round(y) - y| the rounding of the exact result, rounding y + d is off by |round(y) - y| + 2 d at most (a
rounding to nearest is no further from y + d than round(y) is).
A result without its last k, its last token or its last rank has to leave that bound, at a fifth of the elements or more.
"""
import pytest
import torch

from gpu_util import ctx, say
from test_gpu_layer8 import BF16, DEV, F32, TYPES, activations, gen, kept_values, rows8, weight

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -23


def near(got, want, d, lost):
    own = (want.to(got.dtype).double() - want).abs()
    bound = own + 2 * d
    error = (got.double() - want).abs()
    bad = ~(error <= bound)
    assert not bad.any(), (int(bad.sum()), float((error / bound)[bad].max()), bad.nonzero()[:4].tolist())
    for what, term in lost.items():
        out = ((want - term).to(got.dtype).double() - want).abs() > bound
        assert float(out.double().mean()) >= 0.2, (what, float(out.double().mean()))


def of_sums(terms, A, B):
    return 4 * EPS * terms ** 0.5 * (A.square() @ B.square()).sqrt()


def lowrank(x, F, G, dtype):
    """(x F^T) G^T, its bound and its last rank's part."""
    x, F, G = x.double(), F.double(), G.double()
    r = len(F)
    t = x @ F.t()
    d = (of_sums(x.shape[1], x, F.t()).square() @ G.t().square()).sqrt() + of_sums(r, t, G.t())
    d += 4 * (2.0 ** -24 if dtype == F32 else 2.0 ** -17) * (t.square() @ G.t().square()).sqrt()
    return t @ G.t(), d, t[:, -1:] * G[:, -1]


def normal(g, rows, cols, dtype):
    return torch.randn(rows, cols, device=DEV, generator=g).to(dtype)


def check_product(dtype, tokens, n, m, r):
    g = gen(tokens + n + m)
    w, x = weight(g, m, n, r), normal(g, tokens, n, dtype)
    q, s = rows8(x)
    q, s, c = q.double(), s.double()[:, None], w.codes.double()
    y = (q @ c.t()) * s * w.scale.double()
    parts, d, lost = y.abs() + w.bias.double().abs(), 0.0, {"k": (q[:, -1:] * s) * (c[:, -1] * w.scale.double())}
    if r:
        low, d, lost["rank"] = lowrank(x, w.Vt, w.U, dtype)
        y, parts = y + low, parts + low.abs()
    near(ctx().rsvd_q8_product(x, w), y + w.bias.double(), d + 4 * EPS * (r + 8) ** 0.5 * parts, lost)


# More than 64 tokens, by the rule for 256 CUs (tile of the product, ranges of k; ranks and blocks of tokens a wavefront of the low-rank product).
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m,r", [
    (4033, 1000, 3970, 30),          # 256 x 256, one range; 32 ranks, one block
    (3900, 2500, 4010, 100),         # 256 x 256, one range; 128 ranks
    (2000, 16400, 2100, 40),         # 256 x 256, three ranges; 64 ranks
    (8100, 4200, 2001, 70),          # 256 x 256, one range; 128 ranks, two blocks
    (8100, 4200, 130, 20),           # 64 x 64; 32 ranks, two blocks
    (8100, 4200, 130, 50),           # 64 x 64; 64 ranks, two blocks
    (1500, 16400, 1030, 1024),       # 128 x 128, four ranges; eight times 128 ranks
    (130, 2000, 150, 1024),          # 64 x 64, four ranges; the same
    (3000, 500, 300, 200)])          # 64 x 64; twice 128 ranks
def test_product_terms(dtype, tokens, n, m, r):
    say("terms of the product", dtype, tokens, n, m, r)
    check_product(TYPES[dtype], tokens, n, m, r)


# Up to 64 tokens: sixteen, 32 and 64 of them, more and fewer than 2048 features, low-rank sums joined first (eight ranges and more than 256 ranks) or not.
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m,r", [(1, 4100, 333, 64), (7, 4100, 40, 700), (16, 1900, 70, 1024), (20, 4200, 33, 64), (30, 9000, 60, 1000), (32, 2049, 64, 300),
                                          (50, 3000, 90, 0), (40, 4500, 50, 300), (64, 5000, 70, 1024), (40, 5000, 70, 64)])
def test_product_terms_of_a_few_tokens(dtype, tokens, n, m, r):
    say("terms of the product", dtype, tokens, n, m, r)
    check_product(TYPES[dtype], tokens, n, m, r)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m,r", [
    (3970, 4033, 190, 33),           # 256 x 256, one range
    (4033, 3900, 70, 1024),          # 256 x 256, one range; eight times 128 ranks
    (2000, 2100, 8200, 20),          # 256 x 256, three ranges
    (4090, 4100, 600, 40),           # 128 x 128, one range
    (2100, 1100, 5000, 64),          # 128 x 128, three ranges
    (130, 300, 200, 1024),           # 64 x 64, codes as they are
    (700, 2100, 1500, 300),          # 64 x 64, codes as a matrix
    (1, 3000, 9000, 20), (33, 700, 9000, 0)])      # 64 x 64, ranges of k
def test_product_gradient_terms(dtype, tokens, n, m, r):
    say("terms of the product's gradient", dtype, tokens, n, m, r)
    dtype = TYPES[dtype]
    g = gen(tokens + n + m)
    w, dy = weight(g, m, n, r), normal(g, tokens, m, dtype)
    D, W = dy.double(), w.codes.double() * w.scale.double()[:, None]
    y = D @ W
    parts, lost = y.abs(), {"k": D[:, -1:] * W[-1]}
    d = of_sums(m, D, W) + 4 * (2.0 ** -24 if dtype == F32 else 2.0 ** -17) * (D.square() @ W.square()).sqrt()
    if r:
        low, more, lost["rank"] = lowrank(dy, w.U.t(), w.Vt.t(), dtype)
        y, parts, d = y + low, parts + low.abs(), d + more
    near(ctx().rsvd_q8_product_grad(dy, w), y, d + 4 * EPS * (r + 8) ** 0.5 * parts, lost)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m", [
    (190, 4033, 3970),               # 256 x 256, one range
    (5000, 2050, 2050),              # 256 x 256, three ranges
    (1000, 4100, 4090),              # 128 x 128, one range
    (20001, 130, 1030),              # 64 x 64, eight ranges, codes as a matrix
    (20001, 77, 40)])                # 64 x 64, sixteen ranges, codes as they are
def test_weight_gradient_terms(dtype, tokens, n, m):
    say("terms of the weight's gradient", dtype, tokens, n, m)
    g = gen(tokens + n + m)
    kept, dy = ctx().rsvd_keep8_save(normal(g, tokens, n, F32)), normal(g, tokens, m, TYPES[dtype])
    D, X = dy.double(), kept_values(kept.codes, kept.powers)
    w, d, lost = D.t() @ X, of_sums(tokens, D.t(), X), {"token": D[-1][:, None] * X[-1]}
    b, e, lost_b = D.sum(0), 4 * EPS * tokens ** 0.5 * D.square().sum(0).sqrt(), {"token": D[-1]}
    dW, db = ctx().rsvd_keep8_grad(dy, kept)
    near(dW, w, d, lost)
    near(db, b, e, lost_b)
    before, before_b = normal(g, m, n, F32), normal(g, 1, m, F32)[0]
    to, to_b = before.clone(), before_b.clone()
    ctx().rsvd_keep8_grad(dy, kept, out=(to, to_b), accumulate=True)
    near(to, before.double() + w, d, {**lost, "what was there": before.double()})
    near(to_b, before_b.double() + b, e, {**lost_b, "what was there": before_b.double()})


# ---------------------------------------------------------------- infinities, in every type
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m,r", [(9, 200, 70, 8), (40, 2100, 50, 40), (140, 200, 70, 8), (8100, 4200, 70, 100)])
def test_product_rows_with_infinities_in_every_type(dtype, tokens, n, m, r):
    """A row that holds an infinity or NaN is NaN, and no other row changes."""
    say("infinities", dtype, tokens, n, m, r)
    g = gen(tokens)
    w, x = weight(g, m, n, r), activations(g, tokens, n, TYPES[dtype])
    clean = ctx().rsvd_q8_product(x, w)
    rows = [1, 4, 6, tokens - 1]
    x[1, 7], x[4, n - 1], x[6, 0], x[tokens - 1, n // 2] = torch.nan, torch.inf, -torch.inf, torch.inf
    y = ctx().rsvd_q8_product(x, w)
    assert y[rows].isnan().all()
    keep = torch.ones(tokens, dtype=torch.bool, device=DEV)
    keep[rows] = False
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m", [(150, 100, 70), (300, 4033, 3970)])
def test_weight_gradient_with_an_infinity_in_every_type(dtype, tokens, n, m):
    """An infinity in dY makes its row of dW infinite, by the signs of its token's activations (NaN where one is zero); nothing else."""
    g = gen(tokens)
    x, dy = normal(g, tokens, n, F32), normal(g, tokens, m, TYPES[dtype])
    x[9, 11] = 0.0
    kept = ctx().rsvd_keep8_save(x)
    clean, clean_b = ctx().rsvd_keep8_grad(dy, kept)
    dy[9, 5], dy[tokens - 1, m - 1] = torch.inf, -torch.inf
    dW, db = ctx().rsvd_keep8_grad(dy, kept)
    X = kept_values(kept.codes, kept.powers)
    want = clean.double()
    want[5], want[m - 1] = X[9] * torch.inf, X[tokens - 1] * -torch.inf
    whole = lambda t: t.nan_to_num(nan=0.0, posinf=torch.inf, neginf=-torch.inf)
    assert torch.equal(dW.isnan(), want.isnan()) and torch.equal(whole(dW), whole(want.float()))
    assert dW[5, 11].isnan() and db[5] == torch.inf and db[m - 1] == -torch.inf
    keep = [i for i in range(m) if i not in (5, m - 1)]
    assert torch.equal(db[keep], clean_b[keep])


@pytest.mark.parametrize("tokens", [1, 3, 20, 40, 100])
@pytest.mark.parametrize("r", [1, 40, 300])
def test_low_rank_sums_beyond_fp32_are_infinite(tokens, r):
    """Finite tokens whose sum with Vt is not: infinities of its sign, times U, and not NaN."""
    from paper_2110_03423_amd import Weight8
    U, Vt = torch.ones(50, r, dtype=BF16, device=DEV), torch.ones(r, 64, dtype=BF16, device=DEV)
    U[7] = -1.0
    w = Weight8(torch.zeros(50, 64, dtype=torch.int8, device=DEV), torch.ones(50, device=DEV), U, Vt)      # (codes of 0: nothing else is infinite)
    x = torch.full((tokens, 64), 3e38, device=DEV)
    y = ctx().rsvd_q8_product(x, w)
    assert (y[:, 7] == -torch.inf).all()
    y[:, 7] = torch.inf
    assert (y == torch.inf).all()
