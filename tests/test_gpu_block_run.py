"""A gated block run, trained and served as it would be: the forward pass with its products kept, the projection back in 8-bit floats, both backward passes, and updates
made orthogonal; captured, replayed, on several streams, with the workspaces that calls share."""
import pytest
import torch

from gpu_util import ctx
from test_gpu_f8 import blocks64, weight_values
from test_gpu_gated import act64, block
from test_gpu_layer8 import BF16, F32, TYPES, gen

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def parts(g, t, n, m, T):
    x, w, _ = block(g, t, n, m, T)
    down = torch.randn(n, m, device=DEV, generator=g) / m ** 0.5
    dy = (1e-2 * torch.randn(t, n, device=DEV, generator=g)).to(T)
    return x, w, down, dy


def step(c, x, w, down, dy):
    """Gradients of all, and the update of the first weight: both projections as a batch of two."""
    h, kept = c.rsvd_gated_product(x, w, "silu", keep=True)
    back = c.rsvd_f8_weight(down)
    y = c.rsvd_f8_product(h, back)
    dh = c.rsvd_f8_product_grad(dy, back)
    ddown = c.rsvd_f8_weight_grad(dy, h)
    dx, dw = c.rsvd_gated_product_grad(dh, x, w, "silu", kept=kept)
    update = c.rsvd_orthogonalize(dw.view(2, -1, dw.shape[1]))
    return [y, dx, dw, ddown, update]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,m", [(3, 64, 96), (200, 264, 520), (1000, 130, 77)])
def test_a_step_against_64_bits(dtype, t, n, m):
    """From what each call was given, by its definition; to what is lost in the types between them (a 2-norm of twice their unit, and 2^-4 / 4 where a block's rounding
    of a number near a border may go the other way)."""
    T, g = TYPES[dtype], gen(t)
    x, w, down, dy = parts(g, t, n, m, T)
    y, dx, dw, ddown, update = step(ctx(), x, w, down, dy)
    gu = x.double() @ w.double().t()
    a, s, _ = act64(gu[:, :m], "silu")
    h = a * gu[:, m:]
    back = ctx().rsvd_f8_weight(down)
    D = weight_values(back)
    dh = (blocks64(dy, 1, 128)[0] @ D)
    d = torch.cat([dh * gu[:, m:] * s, dh * a], dim=1)
    want = [blocks64(h.to(T), 1, 128)[0] @ D.t(), d @ w.double(), d.t() @ x.double(), blocks64(dy, 128, 1)[0].t() @ blocks64(h.to(T), 128, 1)[0]]
    for got, ref, near in zip((y, dx, dw, ddown), want, (2.0 ** -6, 2.0 ** -6, 2.0 ** -6, 2.0 ** -6)):
        assert float((got.double() - ref).norm() / ref.norm()) < near
    assert update.shape == (2, m, n) and float(torch.linalg.svdvals(update[0].double()).max()) < 1.3
    # the update goes against the gradient
    assert float((update.double() * dw.view(2, m, n).double()).sum()) > 0


@pytest.mark.parametrize("t", [2, 300])
def test_captured_steps_are_replayed_with_new_tensors_beside_eager_ones(t):
    g = gen(t)
    from paper_2110_03423_amd import Rsvd
    c = Rsvd(0)
    x, w, down, dy = parts(g, t, 264, 200, BF16)
    big = parts(g, 2000, 520, 900, F32)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(c, x, w, down, dy)
        stream.synchronize()
        graphs = []
        for _ in range(2):                               # two graphs, whose workspaces are their own
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = step(c, x, w, down, dy)
            graphs.append((graph, out))
        step(c, *big)                                    # the stream's workspace is replaced
    torch.cuda.synchronize()
    filled = [torch.full((1 << 20,), 7, dtype=torch.uint8, device=DEV) for _ in range(64)]
    other = torch.cuda.Stream()
    for trial in range(4):
        a, b, d, e = parts(gen(100 + trial), t, 264, 200, BF16)
        x.copy_(a), w.copy_(b), down.copy_(d), dy.copy_(e)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            graphs[0][0].replay()
        graphs[1][0].replay()
        with torch.cuda.stream(stream):
            beside = step(c, *big)
        torch.cuda.synchronize()
        want, wide = step(Rsvd(0), a, b, d, e), step(Rsvd(0), *big)
        for _, out in graphs:
            for p, q in zip(out, want):
                assert torch.equal(p, q)
        for p, q in zip(beside, wide):
            assert torch.equal(p, q)
        assert all(bool((v == 7).all()) for v in filled)


def test_two_streams_at_once():
    from paper_2110_03423_amd import Rsvd
    c, streams = Rsvd(0), [torch.cuda.Stream() for _ in range(3)]
    sets = [parts(gen(i), 150 + 100 * i, 136, 264, T) for i, T in enumerate(TYPES.values())]
    want = [step(Rsvd(0), *s) for s in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                got.append(step(c, *s))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for p, q in zip(a, b):
                assert torch.equal(p, q)


def test_a_workspace_of_the_callers_is_not_written_behind_its_bytes():
    import ctypes as C
    c = ctx()
    x, w, down, dy = parts(gen(1), 150, 130, 77, BF16)
    dh = torch.randn(150, 77, device=DEV).bfloat16()
    back = c.rsvd_f8_weight(down)
    G = torch.randn(3, 90, 200, device=DEV)
    need = C.c_size_t()

    def room(name, *args):
        assert getattr(c.lib, name)(c.h, *args, C.byref(need)) == 0
        ws = torch.full((need.value + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
        return ws, ws[:need.value]

    calls = [(lambda ws: c.rsvd_gated_product(x, w, workspace=ws), ("rsvd_gated_product_bytes", 0, 150, 130, 77, 0)),
             (lambda ws: c.rsvd_gated_product_grad(dh, x, w, workspace=ws)[1], ("rsvd_gated_product_grad_bytes", 0, 150, 130, 77, 0)),
             (lambda ws: c.rsvd_f8_product(dh, back, workspace=ws), ("rsvd_f8_product_bytes", 0, 150, 77, 130)),
             (lambda ws: c.rsvd_f8_product_grad(dy, back, workspace=ws), ("rsvd_f8_product_grad_bytes", 0, 150, 77, 130)),
             (lambda ws: c.rsvd_f8_weight_grad(dh, x, workspace=ws), ("rsvd_f8_weight_grad_bytes", 0, 150, 130, 77, 0)),
             (lambda ws: c.rsvd_orthogonalize(G, workspace=ws), ("rsvd_orthogonalize_bytes", 2, 3, 90, 200))]
    for call, size in calls:
        ws, given = room(*size)
        a = call(given)
        torch.cuda.synchronize()
        assert bool((ws[given.numel():] == 0x5a).all())
        given.fill_(0xff)                                # (what a workspace holds before does not matter: NaN in every type)
        b = call(given)
        assert torch.equal(a, b) and torch.equal(a, call(None))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t,n,m", [(3, 64, 96), (200, 264, 520), (1000, 130, 77)])
def test_a_step_to_what_its_types_lose(dtype, t, n, m):
    """2-norms, u the unit of the type.  dX and dW do not see how h is held: dh, both kept products, D and the result are rounded, each to u / sqrt 3 on the whole at the most, slopes
    change by about as much as what they are of: sqrt 5 of those, twice that is below 4 u; and sums in fp32, of n, then 2 m or t terms, are below 2^-18.  y and dW of the way back
    see h in blocks, where a number near a border goes the other way: h is off by 2^-22 of itself, or, one time in 2^10 at the most, by 2 u; borders are 2^-4 apart, so
    one number in 2^14 is off by 2^-3, 2^-10 on the whole.  The update is that of dW as it came out."""
    from test_gpu_layer8 import UNIT
    from test_gpu_orthogonalize import iterated
    T, g = TYPES[dtype], gen(t)
    x, w, down, dy = parts(g, t, n, m, T)
    y, dx, dw, ddown, update = step(ctx(), x, w, down, dy)
    gu = x.double() @ w.double().t()
    a, s, _ = act64(gu[:, :m], "silu")
    h = (a * gu[:, m:]).to(T)
    D = weight_values(ctx().rsvd_f8_weight(down))
    dh = blocks64(dy, 1, 128)[0] @ D
    d = torch.cat([dh * gu[:, m:] * s, dh * a], dim=1)
    u = UNIT[T]
    own, held = 4 * u + 2.0 ** -18, u + 2.0 ** -10
    for got, ref, near in ((y, blocks64(h, 1, 128)[0] @ D.t(), held), (dx, d @ w.double(), own), (dw, d.t() @ x.double(), own),
                           (ddown, blocks64(dy, 128, 1)[0].t() @ blocks64(h, 128, 1)[0], held)):
        assert float((got.double() - ref).norm() / ref.norm()) < near
    for i in range(2):
        iterated(dw.view(2, m, n)[i], got=update[i])


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("t", [40, 700])
def test_captured_fp16_gradients_take_the_range_of_each_replay(t, keep):
    """What D is held times follows from the data, on the device: replays with gradients of other sizes, eager calls between them."""
    from paper_2110_03423_amd import Rsvd
    c, g, n, m = Rsvd(0), gen(t), 136, 72
    x, w, dh = block(g, t, n, m, torch.float16)
    kept = c.rsvd_gated_product(x, w, keep=True)[1] if keep else None
    dw = torch.empty(2 * m, n, device=DEV)
    run = lambda ctx_, dx, dw_: ctx_.rsvd_gated_product_grad(dh, x, w, kept=kept, out=(dx, dw_))
    dx = torch.empty_like(x)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        run(c, dx, dw)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run(c, dx, dw)
    for size in (1e-5, 3e3, 1e-2, 0.0, 1e-4):
        dh.copy_(size * torch.randn(t, m, device=DEV, generator=g))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, b = torch.empty_like(x), torch.empty_like(dw)
        run(Rsvd(0), a, b)
        assert torch.equal(dx, a) and torch.equal(dw, b) and bool(b.any()) == (size > 0)
