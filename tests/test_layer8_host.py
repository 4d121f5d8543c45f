"""Argument checks and workspace sizes of the layer operators on a planning context: no GPU.  The fake device pointers are
never dereferenced."""
import ctypes as C

import pytest

from paper_2110_03423_amd import binding
from paper_2110_03423_amd.binding import ERR_NO_DEVICE, X_BF16, X_F16, X_F32

UNSUPPORTED = 4
PTR = C.c_void_p(1 << 20)
ODD = C.c_void_p((1 << 20) + 1)
HALF = C.c_void_p((1 << 20) + 2)
NULL = C.c_void_p(0)


@pytest.fixture(scope="module")
def plan():
    import os
    if not os.path.exists(binding.library_path()):
        from paper_2110_03423_amd import build
        build.build_library()
    return binding.Rsvd(device=None)


def _call(plan, name, order, base, **kw):
    a = dict(base, **kw)
    return getattr(plan.lib, name)(*[a[k] for k in order])


PRODUCT = "ctx stream type tokens n m r X ldx codes ldq scale U ldu Vt ldvt bias Y ldy ws bytes".split()
GRAD = "ctx stream type tokens n m r dY lddy codes ldq scale Ut ldut V ldv dX lddx ws bytes".split()
ROWS = "ctx stream type rows n X ldx codes ldq scale".split()
SAVE = "ctx stream type tokens n X ldx codes ldc powers ldp".split()
LOAD = "ctx stream type tokens n codes ldc powers ldp X ldx".split()
WGRAD = "ctx stream type tokens n m dY lddy codes ldc powers ldp dW lddw db accumulate ws bytes".split()


def test_product_checks_every_argument(plan):
    base = dict(ctx=plan.h, stream=NULL, type=X_BF16, tokens=100, n=70, m=50, r=9, X=PTR, ldx=70, codes=PTR, ldq=80, scale=PTR, U=PTR, ldu=9,
                Vt=PTR, ldvt=70, bias=PTR, Y=PTR, ldy=50, ws=PTR, bytes=1 << 40)
    call = lambda **kw: _call(plan, "rsvd_q8_product", PRODUCT, base, **kw)
    assert call() == ERR_NO_DEVICE
    assert call(ctx=None) == -1 and call(type=3) == -3 and call(type=-1) == -3
    assert call(tokens=-1) == -4 and call(n=0) == -5 and call(m=0) == -6 and call(r=-1) == -7
    assert call(tokens=0, X=NULL, Y=NULL, ws=NULL) == 0
    assert call(X=NULL) == -8 and call(X=ODD) == -8 and call(X=HALF) == ERR_NO_DEVICE and call(type=X_F32, X=HALF) == -8
    assert call(ldx=69) == -9 and call(codes=NULL) == -10 and call(codes=HALF) == -10
    assert call(ldq=64) == -11 and call(ldq=72) == -11 and call(scale=NULL) == -12 and call(scale=HALF) == -12
    assert call(U=NULL) == -13 and call(U=ODD) == -13 and call(ldu=8) == -14 and call(Vt=NULL) == -15 and call(ldvt=69) == -16
    assert call(r=0, U=NULL, Vt=NULL, ldu=0, ldvt=0) == ERR_NO_DEVICE
    assert call(bias=HALF) == -17 and call(bias=NULL) == ERR_NO_DEVICE
    assert call(Y=NULL) == -18 and call(Y=ODD) == -18 and call(ldy=49) == -19
    assert call(ws=NULL) == -20 and call(ws=C.c_void_p((1 << 20) + 128)) == -20
    need = C.c_size_t()
    assert plan.lib.rsvd_q8_product_bytes(plan.h, X_BF16, 100, 70, 50, 9, C.byref(need)) == 0
    assert call(bytes=need.value - 1) == -21 and call(bytes=need.value) == ERR_NO_DEVICE
    wide = binding_limit()
    assert call(n=wide, ldx=wide, ldq=wide, ldvt=wide) == ERR_NO_DEVICE
    assert call(n=wide + 1, ldx=wide + 1, ldq=wide + 16, ldvt=wide + 1) == UNSUPPORTED
    assert call(r=1025, ldu=1025) == UNSUPPORTED


def binding_limit():
    return 131072


def test_product_gradient_checks_every_argument(plan):
    base = dict(ctx=plan.h, stream=NULL, type=X_F16, tokens=100, n=70, m=50, r=9, dY=PTR, lddy=50, codes=PTR, ldq=80, scale=PTR, Ut=PTR,
                ldut=50, V=PTR, ldv=9, dX=PTR, lddx=70, ws=PTR, bytes=1 << 40)
    call = lambda **kw: _call(plan, "rsvd_q8_product_grad", GRAD, base, **kw)
    assert call() == ERR_NO_DEVICE
    assert call(ctx=None) == -1 and call(type=9) == -3 and call(tokens=-5) == -4 and call(n=0) == -5 and call(m=0) == -6 and call(r=-1) == -7
    assert call(tokens=0) == 0
    assert call(dY=NULL) == -8 and call(lddy=49) == -9 and call(codes=NULL) == -10 and call(ldq=79) == -11 and call(scale=NULL) == -12
    assert call(Ut=NULL) == -13 and call(ldut=49) == -14 and call(V=NULL) == -15 and call(ldv=8) == -16
    assert call(dX=NULL) == -17 and call(lddx=69) == -18 and call(ws=NULL) == -19
    need = C.c_size_t()
    assert plan.lib.rsvd_q8_product_grad_bytes(plan.h, X_F16, 100, 70, 50, 9, C.byref(need)) == 0
    assert call(bytes=need.value - 1) == -20 and call(bytes=need.value) == ERR_NO_DEVICE
    assert call(tokens=(1 << 22) + 1) == UNSUPPORTED


def test_rows_and_kept_activations_check_every_argument(plan):
    base = dict(ctx=plan.h, stream=NULL, type=X_F32, rows=10, n=33, X=PTR, ldx=33, codes=PTR, ldq=48, scale=PTR)
    call = lambda **kw: _call(plan, "rsvd_q8_rows", ROWS, base, **kw)
    assert call() == ERR_NO_DEVICE and call(rows=0) == 0
    assert call(ctx=None) == -1 and call(type=3) == -3 and call(rows=-1) == -4 and call(n=0) == -5 and call(X=HALF) == -6
    assert call(ldx=32) == -7 and call(codes=HALF) == -8 and call(ldq=32) == -9 and call(scale=NULL) == -10
    base = dict(ctx=plan.h, stream=NULL, type=X_F32, tokens=10, n=33, X=PTR, ldx=33, codes=PTR, ldc=48, powers=ODD, ldp=2)
    call = lambda **kw: _call(plan, "rsvd_keep8_save", SAVE, base, **kw)
    assert call() == ERR_NO_DEVICE and call(tokens=0) == 0
    assert call(type=3) == -3 and call(tokens=-1) == -4 and call(n=0) == -5 and call(X=NULL) == -6 and call(ldx=32) == -7
    assert call(codes=NULL) == -8 and call(ldc=40) == -9 and call(powers=NULL) == -10 and call(ldp=1) == -11
    call = lambda **kw: _call(plan, "rsvd_keep8_load", LOAD, base, **kw)
    assert call() == ERR_NO_DEVICE and call(tokens=0) == 0
    assert call(codes=HALF) == -6 and call(ldc=32) == -7 and call(powers=NULL) == -8 and call(ldp=1) == -9
    assert call(X=NULL) == -10 and call(ldx=32) == -11


def test_weight_gradient_checks_every_argument(plan):
    base = dict(ctx=plan.h, stream=NULL, type=X_BF16, tokens=100, n=70, m=50, dY=PTR, lddy=50, codes=PTR, ldc=80, powers=ODD, ldp=3, dW=PTR,
                lddw=70, db=PTR, accumulate=0, ws=PTR, bytes=1 << 40)
    call = lambda **kw: _call(plan, "rsvd_keep8_grad", WGRAD, base, **kw)
    assert call() == ERR_NO_DEVICE and call(db=NULL) == ERR_NO_DEVICE and call(accumulate=1) == ERR_NO_DEVICE
    assert call(ctx=None) == -1 and call(type=3) == -3 and call(tokens=-1) == -4 and call(n=0) == -5 and call(m=0) == -6
    assert call(dY=NULL) == -7 and call(lddy=49) == -8 and call(codes=NULL) == -9 and call(ldc=79) == -10 and call(powers=NULL) == -11
    assert call(ldp=2) == -12 and call(dW=NULL) == -13 and call(lddw=69) == -14 and call(db=HALF) == -15
    assert call(ws=NULL) == -17 and call(bytes=0) == -18
    assert call(tokens=0, dY=NULL, codes=NULL, ws=NULL) == ERR_NO_DEVICE          # (zeros are written)
    assert call(tokens=0, dW=NULL) == -13


def test_workspace_queries(plan):
    lib, h, out = plan.lib, plan.h, C.c_size_t()
    for fn, extra in ((lib.rsvd_q8_product_bytes, (9,)), (lib.rsvd_q8_product_grad_bytes, (9,)), (lib.rsvd_keep8_grad_bytes, ())):
        sizes = []
        for tokens in (0, 1, 64, 65, 1000, 20000):
            assert fn(h, X_F32, tokens, 512, 384, *extra, C.byref(out)) == 0
            assert out.value % 256 == 0
            sizes.append(out.value)
        assert sizes[0] == 0 and sizes[1] > 0 and sizes[-1] > sizes[1]
        assert fn(None, X_F32, 1, 1, 1, *extra, C.byref(out)) == -1
        assert fn(h, 5, 1, 1, 1, *extra, C.byref(out)) == -2
        assert fn(h, X_F32, -1, 1, 1, *extra, C.byref(out)) == -3
        assert fn(h, X_F32, 1, 0, 1, *extra, C.byref(out)) == -4
        assert fn(h, X_F32, 1, 1, 0, *extra, C.byref(out)) == -5
        assert fn(h, X_F32, 1, 1 << 20, 1, *extra, C.byref(out)) == UNSUPPORTED
        assert fn(h, X_F32, 1, 1, 1, *extra, None) == -6 - len(extra)
    assert lib.rsvd_q8_product_bytes(h, X_F32, 1, 1, 1, -1, C.byref(out)) == -6


def test_binding_refuses_what_does_not_fit_together():
    torch = pytest.importorskip("torch")
    codes, scale = torch.zeros(6, 5, dtype=torch.int8), torch.zeros(6)
    U, Vt = torch.zeros(6, 2, dtype=torch.bfloat16), torch.zeros(2, 5, dtype=torch.bfloat16)
    w = binding.Weight8(codes, scale, U, Vt, torch.zeros(6))
    assert (w.m, w.n, w.r) == (6, 5, 2) and w.codes.stride(0) % 128 == 0 and w.Ut.shape == (2, 6) and w.V.shape == (5, 2)
    assert binding.Weight8(codes, scale).r == 0 and binding.Weight8(codes, scale, U[:, :0], Vt[:0]).U is None
    for bad in ((codes.float(), scale), (codes, scale[:5]), (codes, scale.double()), (codes, scale, U), (codes, scale, U.float(), Vt),
                (codes, scale, U, Vt[:1]), (codes, scale, U[:5], Vt), (codes, scale, None, None, torch.zeros(5))):
        with pytest.raises((TypeError, ValueError)):
            binding.Weight8(*bad)
    powers = torch.zeros(6, 1, dtype=torch.uint8)
    assert binding.Kept8(codes, powers, torch.float16).n == 5
    for bad in ((codes.short(), powers, torch.float32), (codes, powers.int(), torch.float32), (codes, powers[:5], torch.float32),
                (codes, powers, torch.float64)):
        with pytest.raises((TypeError, ValueError)):
            binding.Kept8(*bad)


def test_transposed_factors_follow_the_factors():
    torch = pytest.importorskip("torch")
    for U, Vt in ((torch.zeros(6, 2, dtype=torch.bfloat16), torch.zeros(2, 5, dtype=torch.bfloat16)),
                  (torch.zeros(2, 6, dtype=torch.bfloat16).t(), torch.zeros(5, 2, dtype=torch.bfloat16).t())):
        w = binding.Weight8(torch.zeros(6, 5, dtype=torch.int8), torch.zeros(6), U, Vt)
        for value in (1.0, 2.0):
            w.U.data.fill_(value)
            w.Vt[1] = value
            assert torch.equal(w.Ut, w.U.t()) and torch.equal(w.V, w.Vt.t()) and w.Ut.is_contiguous() and w.V.is_contiguous()


def test_a_captured_call_leaves_the_kept_workspace_alone(plan):
    """A graph outlives the call that recorded it: a kept workspace is neither recorded nor exchanged while a stream is captured.  (The context has the
    parts of torch that it asks for from the CPU.)"""
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace
    capturing = [False]
    ctx = binding.Rsvd(device=None)
    ctx.device = torch.device("cpu")
    ctx.torch = SimpleNamespace(empty=torch.empty, uint8=torch.uint8, cuda=SimpleNamespace(is_current_stream_capturing=lambda: capturing[0]))
    room = lambda tokens: ctx._layer_ws(7, "rsvd_keep8_grad_bytes", (X_BF16, tokens, 512, 384))
    small = room(100)
    assert room(100) is small and room(50) is small
    capturing[0] = True
    recorded, larger = room(100), room(1000)
    assert recorded[0] != small[0] and larger[0] != small[0] and larger[1] > small[1]
    capturing[0] = False
    assert room(100) is small
    grown = room(1000)
    assert grown[0] not in (recorded[0], larger[0]) and room(100) is grown


def test_rows_of_codes_that_end_with_their_storage():
    """Of a row, whole 16-byte pieces are read: a tensor whose last row ends in the middle of one is copied, one whose rows hold them is not."""
    torch = pytest.importorskip("torch")

    def read_inside(t):
        return (t.storage_offset() + (t.shape[0] - 1) * t.stride(0) + (t.shape[1] + 15) // 16 * 16) <= t.untyped_storage().nbytes()

    short = torch.as_strided(torch.arange(3 * 128 + 100, dtype=torch.int32).to(torch.int8), (4, 100), (128, 1))
    shard = torch.zeros(4, 11008, dtype=torch.int8)[:, 8256:]
    for codes, same in ((short, False), (shard, True)):
        w = binding.Weight8(codes, torch.zeros(4))
        kept = binding.Kept8(codes, torch.zeros(4, (codes.shape[1] + 31) // 32, dtype=torch.uint8), torch.bfloat16)
        for t in (w.codes, kept.codes):
            assert torch.equal(t, codes) and read_inside(t) and (t.data_ptr() == codes.data_ptr()) == same


def test_tensors_of_a_layer_are_on_one_device(plan):
    torch = pytest.importorskip("torch")
    codes, scale, bias = torch.zeros(6, 5, dtype=torch.int8), torch.zeros(6), torch.zeros(6)
    U, Vt = torch.zeros(6, 2, dtype=torch.bfloat16), torch.zeros(2, 5, dtype=torch.bfloat16)
    powers = torch.zeros(6, 1, dtype=torch.uint8)
    assert binding.Weight8(codes, scale, U, Vt, bias).device.type == "cpu" and binding.Kept8(codes, powers, torch.float32).device.type == "cpu"
    for bad in ((codes, scale.to("meta")), (codes, scale, U.to("meta"), Vt), (codes, scale, U, Vt.to("meta")), (codes, scale, U, Vt, bias.to("meta"))):
        with pytest.raises(ValueError):
            binding.Weight8(*bad)
    with pytest.raises(ValueError):
        binding.Kept8(codes, powers.to("meta"), torch.float32)
    # a context of no device, tensors on none
    w, kept, x = binding.Weight8(codes, scale), binding.Kept8(codes, powers, torch.float32), torch.zeros(3, 5)
    for call in (lambda: plan.rsvd_q8_rows(x), lambda: plan.rsvd_q8_product(x, w), lambda: plan.rsvd_q8_product_grad(torch.zeros(3, 6), w),
                 lambda: plan.rsvd_keep8_save(x), lambda: plan.rsvd_keep8_load(kept), lambda: plan.rsvd_keep8_grad(torch.zeros(6, 4), kept)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows,n", [(1, 5), (6, 5), (6, 128), (6, 1), (3, 300)])
def test_rows_that_share_their_memory(rows, n):
    """One row for all (a stride of zero), columns apart, overlapping rows: laid out as the entry points want them."""
    torch = pytest.importorskip("torch")
    flat = (torch.arange(20000) % 251).to(torch.int8)
    blocks = (n + 31) // 32
    for codes in (flat[None, :n].expand(rows, n), flat[:rows, None].expand(rows, n), torch.as_strided(flat, (rows, n), (64, 1)), torch.as_strided(flat, (rows, n), (0, 1))):
        powers = torch.arange(blocks, dtype=torch.uint8)[None].expand(rows, blocks)
        w, kept = binding.Weight8(codes, torch.zeros(rows)), binding.Kept8(codes, powers, torch.float32)
        for t in (w.codes, kept.codes):
            assert torch.equal(t, codes) and (t.stride(1) == 1 or n == 1) and binding._ld(t) >= n and binding._ld(t) % 16 == 0 and t.data_ptr() % 16 == 0
        assert torch.equal(kept.powers, powers) and binding._ld(kept.powers) >= blocks


def test_gradients_of_more_operands_than_a_launch_has_threads(plan):
    """2^32 threads of eight or sixteen operands each."""
    most = 1 << 22
    base = dict(ctx=plan.h, stream=NULL, type=X_F16, tokens=most, n=4096, m=4096, dY=PTR, lddy=8192, codes=PTR, ldc=8192, powers=ODD, ldp=256, dW=PTR,
                lddw=8192, db=PTR, accumulate=0, ws=PTR, bytes=1 << 60)
    call = lambda **kw: _call(plan, "rsvd_keep8_grad", WGRAD, base, **kw)
    assert call() == ERR_NO_DEVICE and call(m=8192) == UNSUPPORTED and call(type=X_BF16, m=8192) == ERR_NO_DEVICE
    assert call(type=X_BF16, m=8192, n=16384, ldc=16384, ldp=512, lddw=16384) == UNSUPPORTED
    base = dict(ctx=plan.h, stream=NULL, type=X_BF16, tokens=most, n=512, m=4096, r=0, dY=PTR, lddy=8192, codes=PTR, ldq=512, scale=PTR, Ut=NULL,
                ldut=0, V=NULL, ldv=0, dX=PTR, lddx=512, ws=PTR, bytes=1 << 60)
    call = lambda **kw: _call(plan, "rsvd_q8_product_grad", GRAD, base, **kw)
    assert call() == ERR_NO_DEVICE and call(m=8192) == UNSUPPORTED
