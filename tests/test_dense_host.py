"""Argument checks and workspace sizes of the gated block, of products in 8-bit floats and of orthogonalised updates, on a planning context: no GPU.  The fake device
pointers are never dereferenced."""
import ctypes as C

import pytest
import torch

from paper_2110_03423_amd import binding
from paper_2110_03423_amd.binding import ERR_NO_DEVICE, X_BF16, X_F16, X_F32

UNSUPPORTED = 4
PTR = C.c_void_p(1 << 20)
ODD = C.c_void_p((1 << 20) + 1)
HALF = C.c_void_p((1 << 20) + 2)
NULL = C.c_void_p(0)
OUT, OUT2 = C.c_void_p(1 << 44), C.c_void_p(1 << 45)


@pytest.fixture(scope="module")
def plan():
    import os
    if not os.path.exists(binding.library_path()):
        from paper_2110_03423_amd import build
        build.build_library()
    return binding.Rsvd(device=None)


def caller(plan, name, order, **base):
    order = order.split()
    return lambda **kw: getattr(plan.lib, name)(*[dict(base, **kw)[k] for k in order])


def bytes_of(plan, name, *args):
    need = C.c_size_t()
    assert getattr(plan.lib, name)(plan.h, *args, C.byref(need)) == 0
    return need.value


def test_gated_product_checks_every_argument(plan):
    call = caller(plan, "rsvd_gated_product", "ctx stream type act tokens n m X ldx W ldw H ldh kept ldk ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, act=0,
                  tokens=100, n=72, m=50, X=PTR, ldx=72, W=PTR, ldw=72, H=OUT, ldh=50, kept=OUT2, ldk=100, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE and call(tokens=0, X=NULL) == 0
    assert call(ctx=None) == -1 and call(type=3) == -3 and call(act=4) == -4 and call(act=-1) == -4 and call(tokens=-1) == -5
    assert call(n=0) == -6 and call(m=0) == -7 and call(X=NULL) == -8 and call(X=ODD) == -8 and call(type=X_F32, X=HALF) == -8
    assert call(ldx=71) == -9 and call(W=NULL) == -10 and call(W=ODD) == -10 and call(ldw=71) == -11 and call(H=NULL) == -12 and call(ldh=49) == -13
    assert call(kept=ODD) == -14 and call(ldk=99) == -15 and call(kept=NULL, ldk=0) == ERR_NO_DEVICE
    assert call(ws=NULL, bytes=0, tokens=32) == ERR_NO_DEVICE
    # a matrix that does not lie as the products read it needs room
    both, neither = (bytes_of(plan, "rsvd_gated_product_bytes", X_BF16, 100, 72, 50, lie) for lie in (3, 0))
    assert neither >= both + 2 * 72 * (100 + 100)
    assert call(bytes=both) == ERR_NO_DEVICE and (both == 0 or call(bytes=both - 1) == -17)
    assert call(X=HALF, ldx=73, W=HALF, bytes=neither) == ERR_NO_DEVICE and call(X=HALF, W=HALF, bytes=neither - 1) == -17
    assert call(X=HALF, W=HALF, ws=NULL) == -16 and call(X=HALF, W=HALF, ws=C.c_void_p((1 << 20) + 128)) == -16
    assert bytes_of(plan, "rsvd_gated_product_bytes", X_F32, 100, 72, 50, 3) >= 6 * 72 * 200
    assert call(n=131073, ldx=131073, ldw=131073) == UNSUPPORTED and call(tokens=(1 << 22) + 1) == UNSUPPORTED
    assert call(tokens=1 << 22, m=8192, ldh=8192, ldk=16384) == UNSUPPORTED


def test_the_binding_knows_how_many_tokens_need_no_workspace(plan):
    few = {"rsvd_gated_product_bytes": 0, "rsvd_f8_product_bytes": 0, "rsvd_f8_product_grad_bytes": 0}
    for xt in (X_BF16, X_F16, X_F32):
        for tokens in (1, 2, 5, 8, 15, 16, 17, 20, 21, 31, 32, 33, 63, 64, 65):
            for n in (1, 100, 3000, 4096, 6144, 6145, 8192, 12288, 49153, 131072):
                for m in (1, 100, 2047, 2048, 4096, 5000, 8191, 8192, 16384, 131072):
                    none = binding._gated_few(xt, tokens, n, m)
                    # (lie = 2: a weight that lies as it is read, tokens that do not and would have to be laid out)
                    assert none <= (bytes_of(plan, "rsvd_gated_product_bytes", xt, tokens, n, m, 0) == 0)
                    if xt == X_F32 or n % 8 == 0:
                        assert none == (bytes_of(plan, "rsvd_gated_product_bytes", xt, tokens, n, m, 2) == 0)
                    few["rsvd_gated_product_bytes"] += none
                    for name, inputs, outputs in (("rsvd_f8_product_bytes", n, m), ("rsvd_f8_product_grad_bytes", m, n)):
                        none = binding._f8_few(xt, tokens, inputs, outputs)
                        assert (bytes_of(plan, name, xt, tokens, n, m) == 0) == none
                        few[name] += none
    assert all(few.values())


def test_gated_gradient_checks_every_argument(plan):
    call = caller(plan, "rsvd_gated_product_grad", "ctx stream type act tokens n m dH lddh X ldx W ldw kept ldk dX lddx dW lddw f32 acc ws bytes", ctx=plan.h, stream=NULL,
                  type=X_F16, act=1, tokens=100, n=72, m=50, dH=PTR, lddh=50, X=PTR, ldx=72, W=PTR, ldw=72, kept=PTR, ldk=100, dX=OUT, lddx=72, dW=OUT2, lddw=72,
                  f32=0, acc=0, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE
    assert call(ctx=None) == -1 and call(type=7) == -3 and call(act=9) == -4 and call(tokens=-1) == -5 and call(n=0) == -6 and call(m=0) == -7
    assert call(dH=NULL) == -8 and call(lddh=49) == -9 and call(X=NULL) == -10 and call(X=ODD) == -10 and call(ldx=71) == -11
    assert call(W=NULL) == -12 and call(ldw=71) == -13 and call(kept=ODD) == -14 and call(ldk=99) == -15 and call(dX=ODD) == -16 and call(lddx=71) == -17
    assert call(dW=ODD) == -18 and call(dW=HALF, f32=1) == -18 and call(lddw=71) == -19 and call(acc=1) == -21 and call(acc=1, f32=1) == ERR_NO_DEVICE
    assert call(ws=NULL) == -22 and call(bytes=0) == -23
    # what is not wanted need not be there
    assert call(dW=NULL, X=NULL) == ERR_NO_DEVICE and call(dX=NULL, W=NULL) == ERR_NO_DEVICE
    assert call(dW=NULL, X=NULL, kept=NULL) == -10 and call(dX=NULL, W=NULL, kept=NULL) == -12
    assert call(tokens=0, dH=NULL, X=NULL, dX=NULL) == ERR_NO_DEVICE       # (zeros are written)
    for lie in range(8):
        need = bytes_of(plan, "rsvd_gated_product_grad_bytes", X_F16, 100, 72, 50, lie)
        args = dict(X=PTR if lie & 1 else HALF, W=PTR if lie & 2 else HALF, kept=PTR if lie & 4 else NULL)
        assert call(bytes=need, **args) == ERR_NO_DEVICE and call(bytes=need - 1, **args) == -23


def test_f8_checks_every_argument(plan):
    call = caller(plan, "rsvd_f8_weight", "ctx stream type m n W ldw q ldq p ldp qt ldqt pt ldpt", ctx=plan.h, stream=NULL, type=X_F32, m=130, n=70, W=PTR, ldw=70,
                  q=OUT, ldq=128, p=PTR, ldp=4, qt=OUT2, ldqt=256, pt=PTR, ldpt=4)
    assert call() == ERR_NO_DEVICE and call(qt=NULL, pt=NULL, ldqt=0, ldpt=0) == ERR_NO_DEVICE
    assert call(ctx=None) == -1 and call(type=3) == -3 and call(m=0) == -4 and call(n=0) == -5 and call(W=HALF) == -6 and call(ldw=69) == -7
    assert call(q=HALF) == -8 and call(ldq=112) == -9 and call(ldq=130) == -9 and call(p=HALF) == -10 and call(ldp=1) == -11 and call(ldp=6) == -11
    assert call(qt=HALF) == -12 and call(ldqt=128) == -13 and call(pt=NULL) == -14 and call(ldpt=2) == -15
    for name, n, m in (("rsvd_f8_product", 200, 50), ("rsvd_f8_product_grad", 50, 200)):
        call = caller(plan, name, "ctx stream type tokens n m X ldx q ldq p ldp Y ldy ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, tokens=100, n=n, m=m, X=PTR,
                      ldx=200, q=PTR, ldq=256, p=PTR, ldp=4, Y=OUT, ldy=50, ws=PTR, bytes=1 << 40)
        assert call() == ERR_NO_DEVICE and call(tokens=0, X=NULL) == 0
        assert call(ctx=None) == -1 and call(type=5) == -3 and call(tokens=-2) == -4 and call(n=0) == -5 and call(m=0) == -6
        assert call(X=ODD) == -7 and call(ldx=199) == -8 and call(q=HALF) == -9 and call(ldq=240) == -10 and call(ldq=264) == -10
        assert call(p=ODD) == -11 and call(ldp=1) == -12 and call(ldp=5) == -12 and call(Y=NULL) == -13 and call(ldy=49) == -14
        need = bytes_of(plan, name + "_bytes", X_BF16, 100, n, m)
        assert need > 0 and call(ws=NULL) == -15 and call(bytes=need - 1) == -16 and call(bytes=need) == ERR_NO_DEVICE
        assert bytes_of(plan, name + "_bytes", X_BF16, 16, n, m) == 0 and call(tokens=16, ws=NULL, bytes=0) == ERR_NO_DEVICE
        assert call(ldq=(1 << 23) + 16) == UNSUPPORTED and call(ldp=(1 << 20) + 4) == UNSUPPORTED and call(ldp=1 << 20) == ERR_NO_DEVICE
    call = caller(plan, "rsvd_f8_weight_grad", "ctx stream type tokens n m dY lddy X ldx dW lddw f32 acc ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, tokens=100,
                  n=70, m=50, dY=PTR, lddy=50, X=PTR, ldx=70, dW=OUT, lddw=70, f32=0, acc=0, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE and call(tokens=0, dY=NULL, X=NULL) == ERR_NO_DEVICE
    assert call(type=3) == -3 and call(tokens=-1) == -4 and call(n=0) == -5 and call(m=0) == -6 and call(dY=NULL) == -7 and call(lddy=49) == -8
    assert call(X=NULL) == -9 and call(ldx=69) == -10 and call(dW=NULL) == -11 and call(f32=1, dW=HALF) == -11 and call(lddw=69) == -12
    assert call(acc=1) == -14 and call(acc=1, f32=1) == ERR_NO_DEVICE and call(ws=NULL) == -15
    need = bytes_of(plan, "rsvd_f8_weight_grad_bytes", X_BF16, 100, 70, 50, 0)
    assert call(bytes=need) == ERR_NO_DEVICE and call(bytes=need - 1) == -16


def at(p):
    return C.c_void_p(p)


def test_results_may_not_lie_on_operands(plan):
    x = 1 << 30
    call = caller(plan, "rsvd_gated_product", "ctx stream type act tokens n m X ldx W ldw H ldh kept ldk ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, act=0,
                  tokens=100, n=50, m=50, X=at(x), ldx=50, W=at(2 * x), ldw=50, H=OUT, ldh=50, kept=OUT2, ldk=100, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE and call(H=at(x)) == -12 and call(kept=at(2 * x)) == -14 and call(kept=OUT) == -14
    # one byte, from either side
    assert call(H=at(x + 9998)) == -12 and call(H=at(x + 10000)) == ERR_NO_DEVICE and call(H=at(x - 9998)) == -12 and call(H=at(x - 10000)) == ERR_NO_DEVICE
    assert call(tokens=20, H=at(x)) == -12
    # columns beside the operand's, in one wider matrix
    wide = dict(ldx=120, ldh=120)
    assert call(H=at(x + 100), **wide) == ERR_NO_DEVICE and call(H=at(x + 140), **wide) == ERR_NO_DEVICE and call(H=at(x + 98), **wide) == -12
    assert call(H=at(x + 142), **wide) == -12 and call(H=at(x + 240 * 7 + 100), **wide) == ERR_NO_DEVICE and call(H=at(x - 240 * 7 - 100), **wide) == ERR_NO_DEVICE
    # one row, too
    one = dict(wide, tokens=1, kept=NULL, ldk=0, ldw=120)
    assert call(H=at(2 * x + 240 * 7 + 100), **one) == ERR_NO_DEVICE and call(H=at(2 * x + 240 * 7 + 98), **one) == -12 and call(H=at(2 * x + 240 * 7 + 142), **one) == -12
    assert call(H=at(2 * x - 98), **one) == -12 and call(H=at(2 * x - 100), **one) == ERR_NO_DEVICE and call(H=at(x + 98), **one) == -12
    assert call(H=at(x - 240 * 7 - 98), **wide) == -12 and call(H=at(x + 100), ldx=120, ldh=122) == -12

    call = caller(plan, "rsvd_gated_product_grad", "ctx stream type act tokens n m dH lddh X ldx W ldw kept ldk dX lddx dW lddw f32 acc ws bytes", ctx=plan.h, stream=NULL,
                  type=X_F16, act=1, tokens=100, n=50, m=50, dH=at(x), lddh=50, X=at(2 * x), ldx=50, W=at(3 * x), ldw=50, kept=at(4 * x), ldk=100, dX=OUT, lddx=50, dW=OUT2,
                  lddw=50, f32=0, acc=0, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE
    for i in range(1, 5):
        assert call(dX=at(i * x)) == -16 and call(dW=at(i * x)) == -18
    assert call(dW=OUT) == -18 and call(dW=OUT, dX=NULL) == ERR_NO_DEVICE and call(dW=at(4 * x), kept=NULL, ldk=0) == ERR_NO_DEVICE

    call = caller(plan, "rsvd_f8_weight", "ctx stream type m n W ldw q ldq p ldp qt ldqt pt ldpt", ctx=plan.h, stream=NULL, type=X_F32, m=128, n=128, W=at(x), ldw=128,
                  q=OUT, ldq=128, p=PTR, ldp=4, qt=OUT2, ldqt=128, pt=PTR, ldpt=4)
    assert call() == ERR_NO_DEVICE and call(q=at(x)) == -8 and call(qt=at(x)) == -12 and call(qt=OUT) == -12
    call = caller(plan, "rsvd_f8_product", "ctx stream type tokens n m X ldx q ldq p ldp Y ldy ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, tokens=3, n=128, m=128,
                  X=at(x), ldx=128, q=at(2 * x), ldq=128, p=PTR, ldp=4, Y=OUT, ldy=128, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE and call(Y=at(x)) == -13 and call(Y=at(2 * x)) == -13
    call = caller(plan, "rsvd_f8_weight_grad", "ctx stream type tokens n m dY lddy X ldx dW lddw f32 acc ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, tokens=100,
                  n=70, m=50, dY=at(x), lddy=50, X=at(2 * x), ldx=70, dW=OUT, lddw=70, f32=0, acc=0, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE and call(dW=at(x)) == -11 and call(dW=at(2 * x)) == -11


def test_orthogonalize_checks_every_argument(plan):
    coef = (C.c_float * 6)(3.4445, -4.775, 2.0315, 1.5, -0.5, 0.0)
    call = caller(plan, "rsvd_orthogonalize", "ctx stream type batch m n G ldg sg steps coef O ldo so ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, batch=3, m=50,
                  n=70, G=PTR, ldg=70, sg=3500, steps=2, coef=coef, O=PTR, ldo=70, so=3500, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE and call(batch=0, G=NULL) == 0 and call(sg=0) == ERR_NO_DEVICE
    assert call(ctx=None) == -1 and call(type=3) == -3 and call(batch=-1) == -4 and call(m=0) == -5 and call(n=0) == -6 and call(G=ODD) == -7
    assert call(ldg=69) == -8 and call(sg=-1) == -9 and call(steps=0) == -10 and call(steps=65) == -10 and call(coef=None) == -11 and call(O=NULL) == -12
    assert call(ldo=69) == -13 and call(so=3499) == -14 and call(ws=NULL) == -15
    need = bytes_of(plan, "rsvd_orthogonalize_bytes", X_BF16, 3, 50, 70)
    assert call(bytes=need) == ERR_NO_DEVICE and call(bytes=need - 1) == -16
    for bad in ((4.0, 0.0, 0.0), (3.4445, -4.775, 4.5), (float("nan"), 0.0, 0.0), (1.0, float("inf"), 0.0), (1.0, -9.0, 0.5)):
        assert call(steps=1, coef=(C.c_float * 3)(*bad)) == UNSUPPORTED
    big = dict(sg=1 << 30, so=1 << 30, bytes=1 << 62)
    assert call(batch=65535, m=16, n=16384, ldg=16384, ldo=16384, **big) == ERR_NO_DEVICE and call(batch=65535, m=1, n=131072, ldg=131072, ldo=131072, **big) == UNSUPPORTED
    assert call(batch=65536) == UNSUPPORTED and call(m=131073, so=1 << 40) == UNSUPPORTED


def test_a_weight_of_8_bit_floats_is_checked_and_laid_out():
    from paper_2110_03423_amd import WeightF8
    codes = torch.arange(130 * 70).remainder(126).to(torch.uint8).view(130, 70).view(torch.float8_e4m3fn)
    powers = torch.tensor([[120], [130]], dtype=torch.uint8)
    w = WeightF8(codes, powers)
    assert torch.equal(w.codes.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(w.powers, powers) and (w.m, w.n) == (130, 70)
    (q, p), (qt, pt) = w._forward, w._backward
    assert q.shape == (130, 128) and not q[:, 70:].any() and qt.shape == (70, 256) and not qt[:, 130:].any()
    assert torch.equal(qt[:, :130], codes.view(torch.uint8).t()) and p.shape == (2, 4) and pt.shape == (1, 4) and pt[0, :2].tolist() == [120, 130]
    assert WeightF8(codes, powers, backward=False)._backward is None
    for error, args in ((TypeError, (codes.view(torch.uint8), powers)), (TypeError, (codes[0], powers)), (ValueError, (codes, powers.int())), (ValueError, (codes, powers[:1])),
                        (ValueError, (codes[:0], powers[:0]))):
        with pytest.raises(error):
            WeightF8(*args)


# Each step the odd polynomial whose values on the image of [0.002, 1] under the ones before are nearest to one (a linear programme on a grid), made smaller by 1.01 for rounding.
SCHEDULE = [(8.3434, -24.2028, 17.5950), (4.0709, -2.9692, 0.5470), (3.6778, -2.6964, 0.5166), (2.7544, -2.0139, 0.4410), (1.9734, -1.3354, 0.3690), (1.8569, -1.2138, 0.3569),
            (1.875, -1.25, 0.375)]


def flat(steps):
    return (C.c_float * (3 * len(steps)))(*[v for s in steps for v in s])


def test_coefficients_are_followed_between_the_ends_of_their_range(plan):
    call = caller(plan, "rsvd_orthogonalize", "ctx stream type batch m n G ldg sg steps coef O ldo so ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, batch=1, m=50,
                  n=70, G=PTR, ldg=70, sg=3500, steps=1, coef=None, O=PTR, ldo=70, so=3500, ws=PTR, bytes=1 << 40)
    step = (3.4445, -4.775, 2.0315)
    for xt in (X_BF16, X_F16, X_F32):
        # start values near 0.9923, and few others, end behind 1e13 and 2.9
        for bad in ([(2.649, -5.722, 2.047)] * 7, [(2.779, -5.08, 1.298)] * 17):
            assert call(type=xt, steps=len(bad), coef=flat(bad)) == UNSUPPORTED
        # entries off the diagonal of b A + c A^2 are half of what its eigenvalues spread by at most: 4.2 here, though they reach -8.3
        assert call(type=xt, coef=flat(SCHEDULE[:1])) == ERR_NO_DEVICE
        for good in (SCHEDULE, [step] * 64, [(1.5, -0.5, 0.0)] * 64, [(1.875, -1.25, 0.375)] * 64, [(2.0, -1.5, 0.5)] * 64, [step, (2.5, -2.0, 0.6), (1.875, -1.25, 0.375)]):
            assert call(type=xt, steps=len(good), coef=flat(good)) == ERR_NO_DEVICE
        # the eigenvalues' spread: b x^2 of [0, 1]
        assert call(type=xt, coef=flat([(15.0, -14.9, 0.0)])) == UNSUPPORTED and call(type=xt, coef=flat([(0.0, 0.0, float("inf"))])) == UNSUPPORTED
        assert call(type=xt, coef=flat([(14.9, -14.6, 0.0)])) == UNSUPPORTED and call(type=xt, coef=flat([(0.0, 0.0, 2.6)])) == ERR_NO_DEVICE
    # without the 1.01 the ends of the range are left by what bf16 results round away, not by 2^-22
    sharp = [(a * 1.01, b * 1.01 ** 3, c * 1.01 ** 5) for a, b, c in SCHEDULE[:-1]] + SCHEDULE[-1:]
    assert [call(type=xt, steps=7, coef=flat(sharp)) for xt in (X_BF16, X_F16, X_F32)] == [UNSUPPORTED, ERR_NO_DEVICE, ERR_NO_DEVICE]


@pytest.mark.parametrize("name,n,m", [("rsvd_f8_product", 300, 200), ("rsvd_f8_product_grad", 200, 300)])
def test_results_may_not_lie_on_powers(plan, name, n, m):
    """Of a weight whose codes are 200 rows of 300: two rows of four bytes of powers, 16 apart."""
    x = 1 << 30
    call = caller(plan, name, "ctx stream type tokens n m X ldx q ldq p ldp Y ldy ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, tokens=3, n=n, m=m, X=at(x), ldx=300,
                  q=at(2 * x), ldq=384, p=at(3 * x), ldp=16, Y=OUT, ldy=200, ws=PTR, bytes=1 << 40)
    assert call() == ERR_NO_DEVICE and call(Y=at(3 * x)) == -13 and call(Y=at(3 * x + 18)) == -13 and call(Y=at(3 * x + 20)) == ERR_NO_DEVICE
    assert call(Y=at(3 * x - 1198)) == -13 and call(Y=at(3 * x - 1200)) == ERR_NO_DEVICE
    assert call(tokens=100, Y=at(3 * x)) == -13


def test_the_workspace_of_what_is_known_to_lie_is_enough_whatever_else_does(plan):
    call = caller(plan, "rsvd_gated_product", "ctx stream type act tokens n m X ldx W ldw H ldh kept ldk ws bytes", ctx=plan.h, stream=NULL, type=X_BF16, act=0,
                  tokens=32, n=64, m=64, X=PTR, ldx=64, W=PTR, ldw=64, H=OUT, ldh=64, kept=NULL, ldk=0, ws=PTR, bytes=0)
    grad = caller(plan, "rsvd_gated_product_grad", "ctx stream type act tokens n m dH lddh X ldx W ldw kept ldk dX lddx dW lddw f32 acc ws bytes", ctx=plan.h, stream=NULL,
                  type=X_F16, act=1, tokens=100, n=64, m=64, dH=PTR, lddh=64, X=PTR, ldx=64, W=PTR, ldw=64, kept=PTR, ldk=100, dX=OUT, lddx=64, dW=OUT2, lddw=64,
                  f32=0, acc=0, ws=PTR, bytes=0)
    grown = 0
    for xt in (X_BF16, X_F16, X_F32):
        for tokens in (1, 16, 17, 20, 21, 32, 33, 100):
            for n, m in ((64, 64), (2048, 4096), (4096, 4096), (8192, 4096), (8192, 8192), (6144, 8200), (1000, 12000), (3001, 4100)):
                sizes = dict(type=xt, tokens=tokens, n=n, m=m, ldx=n, ldw=n, ldh=m)
                need = [bytes_of(plan, "rsvd_gated_product_bytes", xt, tokens, n, m, lie) for lie in range(4)]
                assert need[0] >= max(need) and need[1] >= need[3] and need[2] >= need[3]
                for lie in range(4):
                    places = dict(X=PTR if lie & 1 else C.c_void_p((1 << 20) + 4), W=PTR if lie & 2 else C.c_void_p((1 << 20) + 4))
                    for known in range(4):
                        if known & ~lie == 0:
                            assert call(bytes=need[known], **sizes, **places) == ERR_NO_DEVICE
                    # what the binding takes no workspace for
                    if binding._gated_few(xt, tokens, n, m, bool(lie & 2)):
                        assert call(ws=NULL, **sizes, **places) == ERR_NO_DEVICE
                grown += need[0] > 0 and binding._gated_few(xt, tokens, n, m, False)
                need = [bytes_of(plan, "rsvd_gated_product_grad_bytes", xt, tokens, n, m, lie) for lie in range(8)]
                for lie in range(8):
                    places = dict(X=PTR if lie & 1 else C.c_void_p((1 << 20) + 4), W=PTR if lie & 2 else C.c_void_p((1 << 20) + 4), kept=PTR if lie & 4 else NULL)
                    for known in range(8):
                        if known & ~lie == 0:
                            assert grad(bytes=need[known], ldk=2 * m, lddh=m, lddx=n, lddw=n, **{k: v for k, v in sizes.items() if k != "ldh"}, **places) == ERR_NO_DEVICE
    assert grown > 0


def test_a_weight_of_8_bit_floats_keeps_its_values():
    """Both orders of the codes hold one weight: what is read off it may be written to, and is a copy."""
    import copy
    import pickle
    from paper_2110_03423_amd import WeightF8
    codes = torch.arange(130 * 70).remainder(126).to(torch.uint8).view(130, 70)
    powers = torch.tensor([[120], [130]], dtype=torch.uint8)
    w = WeightF8(codes.view(torch.float8_e4m3fn), powers)
    w.codes.view(torch.uint8).zero_()
    w.powers.fill_(1)
    codes2, powers2 = w.codes, w.powers
    assert torch.equal(codes2.view(torch.uint8), codes) and codes2.dtype == torch.float8_e4m3fn and torch.equal(powers2, powers)
    assert torch.equal(w._forward[0][:, :70], codes) and torch.equal(w._backward[0][:, :130], codes.t()) and w._forward[1][:, 0].tolist() == [120, 130]
    for name, value in (("codes", codes2), ("powers", powers2), ("m", 5), ("n", 5), ("other", 1)):
        with pytest.raises(AttributeError):
            setattr(w, name, value)
    for other in (copy.copy(w), copy.deepcopy(w), pickle.loads(pickle.dumps(w))):
        assert torch.equal(other.codes.view(torch.uint8), codes) and torch.equal(other._backward[0], w._backward[0]) and (other.m, other.n) == (130, 70)


def test_sums_of_a_long_side_move_more_of_the_range(plan):
    """An fp32 sum of equal numbers is off by 2^-24 of itself for each 32 of them that are added at once: 2^-12 of 131072."""
    call = caller(plan, "rsvd_orthogonalize", "ctx stream type batch m n G ldg sg steps coef O ldo so ws bytes", ctx=plan.h, stream=NULL, type=X_F32, batch=1, m=50,
                  n=70, G=PTR, ldg=1 << 17, sg=0, steps=7, coef=None, O=PTR, ldo=1 << 17, so=0, ws=PTR, bytes=1 << 50)
    sharp = flat([(a * 1.01, b * 1.01 ** 3, c * 1.01 ** 5) for a, b, c in SCHEDULE[:-1]] + SCHEDULE[-1:])
    for xt in (X_F16, X_F32):
        for m, n, rc in ((50, 70, ERR_NO_DEVICE), (50, 4096, ERR_NO_DEVICE), (4096, 50, ERR_NO_DEVICE), (50, 131072, UNSUPPORTED), (131072, 50, UNSUPPORTED)):
            assert call(type=xt, m=m, n=n, coef=sharp) == rc
    for xt in (X_BF16, X_F16, X_F32):
        assert call(type=xt, m=50, n=131072, coef=flat(SCHEDULE)) == ERR_NO_DEVICE
