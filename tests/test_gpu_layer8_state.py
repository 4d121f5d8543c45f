"""What a layer and a context keep between calls: a layer's tensors whose values change."""
import pytest
import torch

from gpu_util import ctx
from test_gpu_layer8 import BF16, F32, TYPES, activations, check, gen, grad_reference, product_reference, weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [3, 150])
def test_changed_tensors_are_what_the_next_calls_take(dtype, tokens):
    """Both passes against a layer made of the changed tensors, bit for bit, and against the definition with the factors of the forward pass."""
    from paper_2110_03423_amd import Weight8
    g = gen(tokens)
    w = weight(g, 90, 130, 12)
    x, dy = activations(g, tokens, 130, TYPES[dtype]), activations(g, tokens, 90, TYPES[dtype])
    ctx().rsvd_q8_product(x, w), ctx().rsvd_q8_product_grad(dy, w)
    for change in (w.U, w.Vt, w.scale, w.bias):
        change.data.mul_(-0.75)
        change[0] = 0.5
        w.codes.neg_()
        other = Weight8(w.codes.clone(), w.scale.clone(), w.U.clone(), w.Vt.clone(), w.bias.clone())
        y, dx = ctx().rsvd_q8_product(x, w), ctx().rsvd_q8_product_grad(dy, w)
        assert torch.equal(y, ctx().rsvd_q8_product(x, other)) and torch.equal(dx, ctx().rsvd_q8_product_grad(dy, other))
        check(y, *product_reference(x, w), "product")
        want = dy.double() @ (w.codes.double() * w.scale.double()[:, None] + w.U.double() @ w.Vt.double())
        check(dx, want, grad_reference(dy, other)[1], "gradient")


def test_a_captured_gradient_takes_the_factors_of_the_replay():
    g = gen(3)
    w = weight(g, 90, 130, 12)
    dy = activations(g, 100, 90, BF16)
    ctx().rsvd_q8_product_grad(dy, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dx = ctx().rsvd_q8_product_grad(dy, w)
    for trial in range(4):
        w.U.mul_(-0.5)
        w.Vt[trial] = 1.0
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx, ctx().rsvd_q8_product_grad(dy, w))
        torch.cuda.synchronize()


@pytest.mark.parametrize("tokens", [1, 200])
def test_a_graph_captured_on_the_stream_of_ordinary_calls_keeps_its_workspace(tokens):
    """Ordinary calls, the capture and a larger call on one stream, and the memory that the larger call gave up filled by others."""
    from paper_2110_03423_amd import Rsvd
    g = gen(4)
    c, stream = Rsvd(0), torch.cuda.Stream()
    w, large = weight(g, 260, 2100, 40), weight(g, 1000, 2100, 64)
    x, dy = activations(g, tokens, 2100, BF16), activations(g, tokens, 260, BF16)
    more, dmore = activations(g, 3000, 2100, F32), activations(g, 3000, 1000, F32)

    def step(c, x, dy, w):
        return [c.rsvd_q8_product(x, w), c.rsvd_q8_product_grad(dy, w), *c.rsvd_keep8_grad(dy, c.rsvd_keep8_save(x))]

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(c, x, dy, w)
        stream.synchronize()
        before = dict(c._layer)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = step(c, x, dy, w)
        assert dict(c._layer) == before
        stream.synchronize()
        kept = c._layer[stream.cuda_stream][0]
        step(c, more, dmore, large)
        assert c._layer[stream.cuda_stream][0] != kept
        filled = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    for trial in range(4):
        x.copy_(activations(g, tokens, 2100, BF16))
        dy.copy_(activations(g, tokens, 260, BF16))
        torch.cuda.synchronize()
        graph.replay()
        # ordinary calls of the same context on the stream of the capture, while the graph runs on this one
        with torch.cuda.stream(stream):
            beside = step(c, more, dmore, large)
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, step(Rsvd(0), x, dy, w)):
            assert torch.equal(a, b)
        for a, b in zip(beside, step(Rsvd(0), more, dmore, large)):
            assert torch.equal(a, b)
        assert all(bool((t == 7).all()) for t in filled)


@pytest.mark.parametrize("tokens", [1, 7, 20, 40, 100])
@pytest.mark.parametrize("rows,n,first,last", [(4, 11008, 8256, 11008), (33, 640, 16, 640), (20, 256, 16, 250)])
def test_the_last_shard_of_a_layer(tokens, rows, n, first, last):
    """Columns at the end of a larger tensor, taken as they are: nothing behind its last byte belongs to them."""
    from paper_2110_03423_amd import Weight8
    g = gen(tokens + rows)
    whole = torch.randint(-127, 128, (rows, n), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
    scale, x = torch.rand(rows, device="cuda", generator=g), activations(g, tokens, last - first, F32)
    shard = Weight8(whole[:, first:last], scale)
    assert shard.codes.data_ptr() == whole.data_ptr() + first
    y = ctx().rsvd_q8_product(x, shard)
    assert torch.equal(y, ctx().rsvd_q8_product(x, Weight8(whole[:, first:last].clone(), scale)))
    check(y, *product_reference(x, shard), "shard")


def test_tensors_in_host_memory_are_refused():
    """By the binding, before anything is launched."""
    from paper_2110_03423_amd import Kept8, Weight8
    g, c = gen(9), ctx()
    w = weight(g, 40, 64, 4)
    x, dy = activations(g, 9, 64, BF16), activations(g, 9, 40, BF16)
    kept = c.rsvd_keep8_save(x)
    on_host = Weight8(w.codes.cpu(), w.scale.cpu(), w.U.cpu(), w.Vt.cpu(), w.bias.cpu())
    kept_on_host = Kept8(kept.codes.cpu(), kept.powers.cpu(), BF16)
    room, strided = torch.empty(1 << 22, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device="cuda").expand(1 << 22)
    dW, db = torch.empty(40, 64, device="cuda"), torch.empty(40, device="cuda")
    for call in (lambda: c.rsvd_q8_rows(x.cpu()), lambda: c.rsvd_q8_product(x.cpu(), w), lambda: c.rsvd_q8_product(x, on_host),
                 lambda: c.rsvd_q8_product_grad(dy.cpu(), w), lambda: c.rsvd_q8_product_grad(dy, on_host), lambda: c.rsvd_keep8_save(x.cpu()),
                 lambda: c.rsvd_keep8_load(kept_on_host), lambda: c.rsvd_keep8_load(kept, out=torch.empty(9, 64, dtype=BF16)),
                 lambda: c.rsvd_keep8_grad(dy.cpu(), kept), lambda: c.rsvd_keep8_grad(dy, kept_on_host),
                 lambda: c.rsvd_keep8_grad(dy, kept, out=(dW.cpu(), db)), lambda: c.rsvd_keep8_grad(dy, kept, out=(dW, db.cpu())),
                 lambda: c.rsvd_q8_product(x, w, out=torch.empty(9, 40, dtype=BF16)), lambda: c.rsvd_q8_product_grad(dy, w, out=torch.empty(9, 64, dtype=BF16)),
                 *[lambda s=s: c.rsvd_q8_product(x, w, workspace=s) for s in (room, strided)],
                 *[lambda s=s: c.rsvd_q8_product_grad(dy, w, workspace=s) for s in (room, strided)],
                 *[lambda s=s: c.rsvd_keep8_grad(dy, kept, workspace=s) for s in (room, strided)]):
        with pytest.raises(ValueError):
            call()
    # a workspace of the caller's, of any type
    own = torch.empty(1 << 20, device="cuda")
    assert torch.equal(c.rsvd_q8_product(x, w, workspace=own), c.rsvd_q8_product(x, w))


def test_rows_to_codes_of_more_rows_than_a_launch_has_workgroups():
    """2^24 workgroups of 256 threads are no launch."""
    rows = (1 << 24) + 5
    x = activations(gen(1), rows, 3, BF16)
    codes, scale = ctx().rsvd_q8_rows(x)
    top = x.float().abs().amax(dim=1)
    assert scale.shape == (rows,) and torch.equal(scale, top / torch.full_like(top, 127.0))
    for at in (0, (1 << 22) - 3, 1 << 22, (1 << 23) + 1, rows - 9):
        some, s = ctx().rsvd_q8_rows(x[at:at + 9])
        assert torch.equal(codes[at:at + 9], some) and torch.equal(scale[at:at + 9], s)
