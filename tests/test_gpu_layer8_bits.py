"""What the layer operators may lose beside the rounding of their output, and terms that a sum may not lose.

The exact result rounded to bf16 is off by e0 (2-norm).  An error d before the rounding that has nothing to do with it makes that sqrt(e0^2 + d^2).  dY
times a scale is held to 2^-17 of itself and the low-rank sums to 2^-17 of themselves (and sums of fp32 numbers are nearer), so that d is below
2^-16 of a result of terms of random signs, 0.01 e0: allowed is 1.01 e0, which 0.14 e0 = 2.3e-4 of the result would reach.  A weight rounded to bf16 is off by
1.2e-3 of it (2^-9 at most, uniform in its binade) and gives 1.24 e0.
"""
import pytest
import torch

from gpu_util import ctx, say
from test_gpu_layer8 import BF16, DEV, activations, gen, weight

pytestmark = pytest.mark.gpu


# 64 rows and columns with codes as they are (a single token first) and as a matrix; 128; 256
@pytest.mark.parametrize("tokens,n,m,r", [(1, 4096, 1030, 20), (130, 1000, 700, 33), (300, 2100, 900, 0), (1024, 2050, 500, 64), (4090, 4100, 600, 40), (3970, 4033, 190, 33)])
def test_product_gradient_in_bf16_loses_nothing_but_its_own_rounding(tokens, n, m, r):
    say("bits of the product gradient", tokens, n, m, r)
    g = gen(tokens + m)
    w = weight(g, m, n, r)
    dy = activations(g, tokens, m, BF16)
    dx = ctx().rsvd_q8_product_grad(dy, w).double()
    want = torch.matmul(dy.double(), w.codes.double() * w.scale.double()[:, None])
    if r:
        want += (dy.double() @ w.U.double()) @ w.Vt.double()
    own = float((want.float().bfloat16().double() - want).norm())
    assert float((dx - want).norm()) <= 1.01 * own


def test_codes_next_to_ties_come_from_two_roundings():
    """codes = x (127 (1 / a)): at a tie, the two roundings of the factor decide.  (One rounded quotient 127 / a would give the other neighbour in each of these
    rows; worked out by hand from the fp32 neighbours of 1 / a and 127 / a.)"""
    ties = [(15.0, 7.5, 64), (19.0, 9.5, 64), (47.0, 23.5, 63), (51.0, 25.5, 64), (83.0, 41.5, 63), (94.0, 47.0, 63), (101.0, 50.5, 63)]
    x = torch.tensor([[a, t, -t] for a, t, _ in ties], device=DEV)
    codes, _ = ctx().rsvd_q8_rows(x)
    assert codes.tolist() == [[127, q, -q] for _, _, q in ties]
