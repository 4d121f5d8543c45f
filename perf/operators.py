"""The layer operators whose speed and accuracy this repository is held to: a linear layer that came out of a decomposition.

A weight W (m x n) is the sum of a low-rank part U Vt (U m x r, Vt r x n, bf16), as the randomized SVD returns it, and of a
rest held in 8 bits with a scale for each of its rows.  Activations that the backward pass needs are kept in 8 bits, in
blocks of 32 features that share a power of two.  `op` names what a case runs:

  product      Y = X W^T + bias        rows of X to 8 bits, product of the integers, low-rank term from X itself
  product_grad dX = dY W               the gradient with respect to X (rounding X to 8 bits is passed straight through)
  keep         X^                      X to blocks of 8 bits and back
  keep_grad    dW = dY^T X^, db        gradients of a weight and a bias from kept activations

Rows to 8 bits: a = max |x|, s = a / 127, code = x (127 / a) rounded to even, each of these a single fp32 operation; a row
with a < 2^-116 has scale 0 and codes 0, a row with an infinity or NaN has scale NaN and codes 0.  Blocks of 32: a = f 2^E
with f in [1/2, 1), e = max(E - 7, -126), code = x 2^-e rounded to even and cut at +-127, held with the byte e + 127; a block
with an infinity or NaN has the byte 255, codes 0 and reads back as NaN.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
LARGEST = 16384 * 16384 * 4096          # multiply-adds of the largest case


def _case(name, op, dtype, tokens, n, m=0, r=0, bias=False):
    c = dict(op=op, dtype=dtype, tokens=tokens, n=n, m=m, r=r, bias=bias)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one step of decoding: a single token through a square layer, where launches and the stream of the weight are all
        _case("one token", "product", "bf16", 1, 4096, 4096, 64),
        # a handful of sequences decoded together through a layer of the sizes of the planted-spectrum benchmark
        _case("few tokens", "product", "bf16", 7, 2000, 10000, 64, True),
        # a short prompt in fp32, every size odd
        _case("ragged product f32", "product", "f32", 333, 2999, 1410, 51, True),
        # a prompt through the widening layer of a block
        _case("prompt", "product", "bf16", 2048, 4096, 16384, 64),
        # a training batch through the narrowing layer of a large block, fp16
        _case("large product f16", "product", "f16", 16384, 16384, 4096, 128, True),
        # backward through a small layer, fp16, few tokens for its size
        _case("ragged product gradient f16", "product_grad", "f16", 301, 2000, 1410, 10),
        # backward through the widening layer of a block
        _case("product gradient", "product_grad", "bf16", 4096, 4096, 16384, 64),
        # an odd activation in fp32, kept between the passes
        _case("ragged keep f32", "keep", "f32", 1001, 2999),
        # the input of a block over a training batch
        _case("keep", "keep", "bf16", 16384, 4096),
        # the gradient of a factor of rank 64: many tokens, few outputs
        _case("factor gradient", "keep_grad", "bf16", 8192, 4096, 64),
        # a small layer trained in fp32, every size odd but one
        _case("ragged weight gradient f32", "keep_grad", "f32", 1501, 1000, 777),
        # the weight of the widening layer over a training batch
        _case("weight gradient", "keep_grad", "bf16", 16384, 4096, 16384),
    ]


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        kind = rng.random()
        if kind < 0.4 and v >= 128:
            v = v // 64 * 64              # the sizes that layers mostly have
        elif kind < 0.6 and v > 2:
            v |= 1
        return v

    op = rng.choice(["product", "product", "product_grad", "keep", "keep_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    n = size(256, 16384)
    tokens = size(1, 16384)
    if op == "keep":
        return _case(None, op, dtype, tokens, n)
    m = size(64 if op == "keep_grad" else 256, 16384)
    # gradients of fp16 and fp32 outputs are two and three bf16 products
    parts = 1 if op == "product" else {"bf16": 1, "f16": 2, "f32": 3}[dtype]
    tokens = max(1, min(tokens, LARGEST // (parts * n * m)))
    if op == "keep_grad":
        return _case(None, op, dtype, tokens, n, m)
    r = rng.choice([0, rng.randint(1, 48), 16 * rng.randint(1, 8)])
    return _case(None, op, dtype, tokens, n, m, r, rng.random() < 0.5)


def work(case):
    t, n, m, r, es = case["tokens"], case["n"], case["m"], case["r"], SIZE[case["dtype"]]
    blocks = -(-n // 32)
    if case["op"] == "keep":
        return {"bytes": 2 * t * n * es + 2 * t * (n + blocks), "flops": 4 * t * n}
    if case["op"] == "keep_grad":
        return {"bytes": t * m * es + t * (n + blocks) + 4 * m * n + 4 * m, "flops": 2 * t * n * m + t * m}
    return {"bytes": t * (n + m) * es + m * n + 4 * m + 2 * r * (m + n) + (4 * m if case["bias"] else 0),
            "flops": 2 * t * n * m + 2 * t * r * (n + m)}


# ---------------------------------------------------------------- the numbers that are held in 8 bits

def _rows8(x):
    """Codes (fp32) and scales of the rows of x (fp32)."""
    a = x.abs().amax(dim=1, keepdim=True)
    small, bad = a < 2.0 ** -116, ~torch.isfinite(a)
    inv = 127.0 / torch.where(small | bad, 1.0, a)
    q = torch.where(small | bad, 0.0, torch.round(x * inv))
    s = torch.where(bad, math.nan, torch.where(small, 0.0, a / 127.0))
    return q, s


def _blocks8(x):
    """Codes (fp32, tokens x n) and bytes of the exponents (int32, tokens x blocks) of x (fp32)."""
    t, n = x.shape
    blocks = -(-n // 32)
    if blocks * 32 != n:
        x = torch.cat([x, x.new_zeros(t, blocks * 32 - n)], dim=1)
    x = x.view(t, blocks, 32)
    a = x.abs().amax(dim=2, keepdim=True)
    bad = ~torch.isfinite(a)
    e = torch.clamp(torch.frexp(torch.where(bad, 1.0, a))[1] - 7, min=-126)
    e = torch.where(a > 0, e, -126)
    q = torch.clamp(torch.round(x * torch.exp2(-e.float())), -127.0, 127.0)
    q = torch.where(bad, 0.0, q).reshape(t, blocks * 32)[:, :n]
    return q, torch.where(bad, 255, e + 127)[..., 0]


def _unblocks8(q, byte):
    n = q.shape[1]
    two = torch.where(byte == 255, math.nan, torch.exp2(byte.float() - 127.0))
    return q * two.repeat_interleave(32, dim=1)[:, :n]


# ---------------------------------------------------------------- inputs

def _activations(g, t, n, dtype):
    """Tokens as a layer meets them: a few channels ten times the others, tokens of different size, padding of zeros."""
    x = torch.randn(t, n, device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn(t, 1, device="cuda", generator=g))
    x[:, torch.randint(n, (max(1, n // 256),), device="cuda", generator=g)] *= 10.0
    if t > 8:
        x[97::101] = 0.0
    return x.to(TYPES[dtype])


def _gradients(g, t, m, dtype):
    dy = 1e-2 * torch.randn(t, m, device="cuda", generator=g)
    dy *= torch.exp(torch.randn(t, 1, device="cuda", generator=g).clamp(-2.0, 2.0))
    if t > 8:
        dy[97::101] = 0.0
    return dy.to(TYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, n, m, r, dtype = case["tokens"], case["n"], case["m"], case["r"], case["dtype"]
    state = {"op": case["op"], "dtype": TYPES[dtype]}
    if case["op"] in ("product", "product_grad"):
        w = torch.randn(m, n, device="cuda", generator=g) * (0.7 / math.sqrt(n))
        w *= torch.exp(0.3 * torch.randn(m, 1, device="cuda", generator=g))
        codes, scale = _rows8(w)
        codes, scale = codes.to(torch.int8), scale[:, 0].contiguous()
        del w
        u = vt = bias = None
        if r > 0:
            u = (torch.randn(m, r, device="cuda", generator=g) * (0.7 / math.sqrt(r))).bfloat16()
            vt = (torch.randn(r, n, device="cuda", generator=g) / math.sqrt(n)).bfloat16()
        if case["bias"]:
            bias = torch.randn(m, device="cuda", generator=g) * 0.1
        if case["op"] == "product":
            state["x"] = _activations(g, t, n, dtype)
        else:
            state["dy"] = _gradients(g, t, m, dtype)
        if own:
            from paper_2110_03423_amd import Weight8
            state["weight"] = Weight8(codes, scale, u, vt, bias)
        else:
            state["weight"] = (codes, scale, u, vt, bias)
    elif case["op"] == "keep":
        state["x"] = _activations(g, t, n, dtype)
    else:
        q, byte = _blocks8(_activations(g, t, n, dtype).float())
        q, byte = q.to(torch.int8), byte.to(torch.uint8)
        state["dy"] = _gradients(g, t, m, dtype)
        if own:
            from paper_2110_03423_amd import Kept8
            state["kept"] = Kept8(q, byte, TYPES[dtype])
        else:
            state["kept"] = (q, byte)
    if own:
        from paper_2110_03423_amd import Rsvd
        state["ctx"] = Rsvd(0)
    return state


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    ctx = state["ctx"]
    if state["op"] == "product":
        return ctx.rsvd_q8_product(state["x"], state["weight"])
    if state["op"] == "product_grad":
        return ctx.rsvd_q8_product_grad(state["dy"], state["weight"])
    if state["op"] == "keep":
        return ctx.rsvd_keep8_load(ctx.rsvd_keep8_save(state["x"]))
    return ctx.rsvd_keep8_grad(state["dy"], state["kept"])


def _run_plain(state):
    if state["op"] == "product":
        codes, scale, u, vt, bias = state["weight"]
        x = state["x"].float()
        q, s = _rows8(x)
        y = (q @ codes.float().t()) * s * scale
        if u is not None:
            y += (x @ vt.float().t()) @ u.float().t()
        if bias is not None:
            y += bias
        return y.to(state["dtype"])
    if state["op"] == "product_grad":
        codes, scale, u, vt, _ = state["weight"]
        dy = state["dy"].float()
        dx = (dy * scale) @ codes.float()
        if u is not None:
            dx += (dy @ u.float()) @ vt.float()
        return dx.to(state["dtype"])
    if state["op"] == "keep":
        return _unblocks8(*_blocks8(state["x"].float())).to(state["dtype"])
    q, byte = state["kept"]
    dy = state["dy"].float()
    return dy.t() @ _unblocks8(q.float(), byte), dy.sum(dim=0)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    global own
    before, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = before
    if case["op"] in ("product", "product_grad"):
        codes, scale, u, vt, bias = state["weight"]
        rest = codes.double() * scale.double()[:, None]
        if case["op"] == "product_grad":
            dy = state["dy"].double()
            return torch.matmul(dy, rest if u is None else rest.addmm_(u.double(), vt.double()))
        x = state["x"].to(torch.float32)
        top = torch.maximum(x.max(dim=1).values, -x.min(dim=1).values)
        zero = top < math.ldexp(1.0, -116)
        per = torch.full_like(top, 127.0).div_(torch.where(zero, torch.ones_like(top), top))
        held = x.mul(per[:, None]).round_().double().mul_((top / 127.0).double()[:, None])
        held[zero] = 0.0
        y = torch.matmul(held, rest.t())
        if u is not None:
            y.addmm_(state["x"].double(), torch.matmul(u.double(), vt.double()).t())
        return y if bias is None else y.add_(bias.double())
    if case["op"] == "keep":
        x = state["x"].double()
        out = torch.empty_like(x)
        for j in range(0, x.shape[1], 32):
            part = x[:, j:j + 32]
            top = part.abs().max(dim=1, keepdim=True).values
            step = torch.full_like(top, 2.0 ** -126)
            some = top >= 2.0 ** -119
            step[some] = torch.exp2(torch.floor(torch.log2(top[some])) - 6.0)
            # log2 rounds: numbers just under a power of two
            step = torch.where(some & (step * 64.0 > top), step / 2.0, step)
            out[:, j:j + 32] = torch.round(part / step).clamp_(-127.0, 127.0) * step
        return out
    q, byte = state["kept"]
    dy = state["dy"].double()
    held = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    for j in range(byte.shape[1]):
        held[:, 32 * j:32 * j + 32] = torch.ldexp(q[:, 32 * j:32 * j + 32].double(), byte[:, j:j + 1].int() - 127)
    return torch.matmul(dy.t(), held), torch.sum(dy, dim=0)
