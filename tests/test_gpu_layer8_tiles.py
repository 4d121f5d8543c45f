"""The gradients of the layer operators at sizes that reach every tile (64, 128 and 256 rows and columns), ranges of k, and codes taken as they are or
as a matrix of bf16 numbers; the tolerances are those of test_gpu_layer8.py."""
import pytest
import torch

from gpu_util import ctx, say
from test_gpu_layer8 import (DEV, F32, TYPES, activations, check, gen, grad_reference, kept_of, kept_values, weight, wgrad_reference)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m,r", [(90, 150, 300, 20), (330, 200, 700, 0), (130, 4100, 2100, 33), (200, 8200, 3000, 16), (700, 2100, 1500, 40),
                                          (128, 16000, 2048, 8), (1900, 2050, 9000, 12)])
def test_product_gradient_in_every_tile(dtype, tokens, n, m, r):
    say("product gradient", dtype, tokens, n, m, r)
    g = gen(tokens + m)
    w = weight(g, m, n, r)
    dy = activations(g, tokens, m, TYPES[dtype])
    dx = ctx().rsvd_q8_product_grad(dy, w)
    want, bound = grad_reference(dy, w)
    check(dx, want, bound, "dX")
    assert torch.equal(ctx().rsvd_q8_product_grad(dy, w), dx)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,n,m", [(700, 130, 70), (500, 130, 1100), (1500, 1500, 260), (900, 6200, 900), (3000, 2100, 1100), (400, 4100, 4100),
                                        (5000, 2050, 2050), (5000, 4100, 100)])
def test_weight_gradient_in_every_tile(dtype, tokens, n, m):
    say("weight gradient", dtype, tokens, n, m)
    g = gen(tokens + m)
    kept = kept_of(g, tokens, n)
    dy = activations(g, tokens, m, TYPES[dtype])
    dW, db = ctx().rsvd_keep8_grad(dy, kept)
    w, wt, b, bt = wgrad_reference(dy, kept)
    check(dW, w, wt, "dW")
    check(db, b, bt, "db")
    ctx().rsvd_keep8_grad(dy, kept, out=(dW, db), accumulate=True)
    check(dW, 2 * w, 2 * wt, "dW +=")
    check(db, 2 * b, 2 * bt, "db +=")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,m", [(65, 33), (129, 1100)])
def test_weight_gradient_of_kept_numbers_in_wider_rows(dtype, tokens, m):
    """Codes and powers in the middle of larger tensors: rows of an odd number of powers, garbage behind the last code."""
    from paper_2110_03423_amd import Kept8
    g = gen(5)
    n = 77
    plain = kept_of(g, tokens, n)
    codes = torch.full((tokens, 384), 99, dtype=torch.int8, device=DEV)
    powers = torch.full((tokens, 9), 255, dtype=torch.uint8, device=DEV)
    codes[:, 128:128 + n], powers[:, 3:6] = plain.codes, plain.powers
    kept = Kept8(codes[:, 128:128 + n], powers[:, 3:6], F32)
    assert kept.codes.data_ptr() == codes.data_ptr() + 128 and kept.powers.data_ptr() == powers.data_ptr() + 3
    dy = activations(g, tokens, m, TYPES[dtype])
    dW, db = ctx().rsvd_keep8_grad(dy, kept)
    dW0, db0 = ctx().rsvd_keep8_grad(dy, plain)
    assert torch.equal(dW, dW0) and torch.equal(db, db0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,m", [(65, 33), (129, 1100)])
def test_a_block_that_held_a_nan_reaches_its_columns_only(dtype, tokens, m):
    g = gen(6)
    x = activations(g, tokens, 130, F32)
    x[tokens - 1, 40] = torch.nan
    kept = ctx().rsvd_keep8_save(x)
    assert kept_values(kept.codes, kept.powers)[tokens - 1, 32:64].isnan().all()
    dy = activations(g, tokens, m, TYPES[dtype])
    dW, db = ctx().rsvd_keep8_grad(dy, kept)
    assert dW[:, 32:64].isnan().all() and torch.isfinite(dW[:, :32]).all() and torch.isfinite(dW[:, 64:]).all() and torch.isfinite(db).all()


def test_workspaces_of_two_streams_are_apart():
    """Calls of one context under way on two streams at once."""
    g = gen(8)
    w = weight(g, 600, 500, 16)
    x = [activations(g, 300, 500, F32) for _ in range(2)]
    alone = [ctx().rsvd_q8_product(t, w) for t in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ctx().rsvd_q8_product(x[i], w))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, alone[i]) for y in got[i])


def test_a_layer_does_not_exchange_its_tensors():
    w = weight(gen(9), 20, 30, 4)
    with pytest.raises(AttributeError):
        w.bias = None
