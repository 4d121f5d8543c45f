"""Operators of training and serving a gated feed-forward block whose speed and accuracy this repository is held to.  `op` names what a case runs:

  gated         H = act(X Wg^T) * (X Wu^T)             W = (Wg; Wu), 2 m x n; `keep`: also both products, in the type of X
  gated_grad    dX = D W, dW = D^T X                   D = (dH * u * act'(g), dH * act(g)); g, u as they were kept, or computed again
  f8            Y = X^ W^^T                            X to 8-bit floats in blocks of 128 features of a token, W held in blocks of 128 x 128
  f8_grad       dX = dY^ W^                            dY to blocks of 128 outputs of a token
  f8_weight     dW = dY^^T X^                          both to blocks of 128 tokens of a feature
  orthogonal    X <- a X + (b A + c A^2) X, A = X X^T  five times from G / |G|, for every matrix of a batch

8-bit floats (e4m3): a block shares a power of two 2^e, the least with max |x| <= 448 2^e, e at least -126; a code is x 2^-e rounded to even.
Rounding to blocks is passed straight through by the gradients.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
F8 = torch.float8_e4m3fn
STEP = (3.4445, -4.7750, 2.0315)        # a, b, c
STEPS = 5
LARGEST = 2 * STEPS * 5 * 4096 ** 3      # multiply-adds of the largest plain form


def _layer(name, op, dtype, tokens, n, m, act="silu", keep=False):
    c = dict(op=op, dtype=dtype, tokens=tokens, n=n, m=m)
    if op.startswith("gated"):
        c.update(act=act, keep=keep)
    return dict(c, name=name) if name else c


def _matrices(name, dtype, batch, m, n):
    c = dict(op="orthogonal", dtype=dtype, batch=batch, m=m, n=n)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one step of decoding: a single token through a small block, where launches and the stream of the weight are all
        _layer("gated one token", "gated", "bf16", 1, 2048, 4096),
        # forward over a training batch, both products kept for the backward pass
        _layer("gated block", "gated", "bf16", 8192, 4096, 8192, keep=True),
        # backward of a small block trained in fp32, every size odd or nearly
        _layer("ragged gated gradient f32", "gated_grad", "f32", 301, 2999, 1410, "gelu", True),
        # backward over a training batch that kept its input only
        _layer("gated gradient", "gated_grad", "bf16", 8192, 4096, 8192),
        # one step of decoding through a square layer
        _layer("f8 one token", "f8", "bf16", 1, 4096, 4096),
        # a training batch through the widening layer of a block, fp16
        _layer("f8 product f16", "f8", "f16", 8192, 4096, 16384),
        # backward through a small layer, few tokens for its size, blocks that end inside
        _layer("ragged f8 gradient f32", "f8_grad", "f32", 333, 2999, 1410),
        # backward through the widening layer of a block
        _layer("f8 gradient", "f8_grad", "bf16", 8192, 4096, 16384),
        # the weight of a small layer, an odd number of tokens
        _layer("ragged f8 weight gradient f16", "f8_weight", "f16", 1501, 1000, 777),
        # the weight of the widening layer over a training batch
        _layer("f8 weight gradient", "f8_weight", "bf16", 16384, 4096, 8192),
        # the update of a small tall weight, in fp32
        _matrices("orthogonal f32", "f32", 1, 1410, 777),
        # the updates of a gated block's two projections
        _matrices("orthogonal gate and up", "bf16", 2, 8192, 4096),
    ]


def _madds(c):
    if c["op"] == "orthogonal":
        s, l = min(c["m"], c["n"]), max(c["m"], c["n"])
        return c["batch"] * STEPS * (2 * s * s * l + s ** 3)
    t = c["tokens"] * c["n"] * c["m"]
    return {"gated": 2, "gated_grad": 4 if c.get("keep") else 6}.get(c["op"], 1) * t


def draw(rng):
    def size(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        kind = rng.random()
        if kind < 0.4 and v >= 128:
            v = v // 64 * 64              # the sizes that layers mostly have
        elif kind < 0.6 and v > 2:
            v |= 1
        return v

    op = rng.choice(["gated", "gated_grad", "f8", "f8_grad", "f8_weight", "orthogonal"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    # fp32 operands of products in full precision are several numbers each
    parts = 1 if dtype != "f32" or op.startswith("f8") else 4
    while True:
        if op == "orthogonal":
            c = _matrices(None, dtype, rng.choice([1, 1, 2, 3, 8]), size(64, 8192), size(64, 8192))
        else:
            c = _layer(None, op, dtype, size(1, 16384), size(256, 16384), size(256, 16384),
                       rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), rng.random() < 0.5)
        if _madds(c) * parts <= LARGEST:
            return c


def work(case):
    m, n, es = case["m"], case["n"], SIZE[case["dtype"]]
    if case["op"] == "orthogonal":
        s, l = min(m, n), max(m, n)
        # A and the polynomial in it are symmetric: half of their products
        return {"bytes": 2 * case["batch"] * m * n * es, "flops": case["batch"] * STEPS * (3 * s * s * l + s ** 3)}
    t = case["tokens"]
    flops = 2 * _madds(case)
    if case["op"] == "gated":
        return {"bytes": es * (t * n + 2 * m * n + t * m + (2 * t * m if case["keep"] else 0)), "flops": flops}
    if case["op"] == "gated_grad":
        return {"bytes": es * (t * m + 2 * t * n + 4 * m * n + (2 * t * m if case["keep"] else 0)), "flops": flops}
    if case["op"] == "f8_weight":
        return {"bytes": es * (t * (m + n) + m * n), "flops": flops}
    return {"bytes": es * t * (m + n) + m * n + -(-m // 128) * -(-n // 128), "flops": flops}


# ---------------------------------------------------------------- 8-bit floats in blocks

def _power(a):
    """The exponents e of blocks with these largest magnitudes (fp32), as int32."""
    f, e = torch.frexp(a)
    e = torch.clamp(torch.where(f > 0.875, e - 8, e - 9), min=-126)
    return torch.where(a > 0, e, -126)


def _blocks(x, rows, cols):
    """x (fp32), its zeros behind the end included, as (row blocks, rows, column blocks, cols)."""
    t, n = x.shape
    p = x.new_zeros(-(-t // rows) * rows, -(-n // cols) * cols)
    p[:t, :n] = x
    return p.view(-(-t // rows), rows, -(-n // cols), cols)


def _round8(x, rows, cols):
    """x (fp32) rounded to 8-bit floats in blocks of rows x cols: codes, and the exponents of the blocks."""
    b = _blocks(x, rows, cols)
    e = _power(b.abs().amax(dim=(1, 3), keepdim=True))
    codes = (b * torch.exp2(-e.float())).to(F8)
    return codes.view(b.shape[0] * rows, b.shape[2] * cols)[:x.shape[0], :x.shape[1]], e[:, 0, :, 0]


def _values8(codes, e, rows, cols):
    two = torch.exp2(e.float()).repeat_interleave(rows, dim=0).repeat_interleave(cols, dim=1)
    return codes.float() * two[:codes.shape[0], :codes.shape[1]]


def _rounded8(x, rows, cols):
    return _values8(*_round8(x.float(), rows, cols), rows, cols)


# ---------------------------------------------------------------- inputs

def _activations(g, t, n, dtype):
    """Tokens as a layer meets them: a few channels ten times the others, tokens of different size, padding of zeros."""
    x = torch.randn(t, n, device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn(t, 1, device="cuda", generator=g)).clamp(max=4.0)
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


def _weight(g, m, n):
    w = torch.randn(m, n, device="cuda", generator=g) * (0.7 / math.sqrt(n))
    return w * torch.exp(0.3 * torch.randn(m, 1, device="cuda", generator=g))


def _momentum(g, m, n):
    """Averaged gradients: directions of falling weight, and noise."""
    k = max(1, min(m, n) // 4)
    fall = torch.arange(1, k + 1, device="cuda", dtype=torch.float32) ** -0.5
    signal = (torch.randn(m, k, device="cuda", generator=g) * fall) @ torch.randn(k, n, device="cuda", generator=g)
    return 1e-3 * (signal / signal.square().mean().sqrt() + 0.5 * torch.randn(m, n, device="cuda", generator=g))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, n, dtype, op = case["m"], case["n"], case["dtype"], case["op"]
    state = {"op": op, "dtype": TYPES[dtype]}
    if op == "orthogonal":
        state["G"] = torch.stack([_momentum(g, m, n) for _ in range(case["batch"])]).to(TYPES[dtype])
    else:
        t = case["tokens"]
        if op in ("gated", "gated_grad"):
            state["act"], state["keep"] = case["act"], case["keep"]
            state["w"] = _weight(g, 2 * m, n).to(TYPES[dtype])
        if op in ("f8", "f8_grad"):
            codes, e = _round8(_weight(g, m, n), 128, 128)
            codes, powers = codes.contiguous(), (e + 127).to(torch.uint8)
            if own:
                from paper_2110_03423_amd import WeightF8
                state["weight"] = WeightF8(codes, powers)
            else:
                state["weight"] = (codes, powers)
        if op != "f8_grad":
            state["x"] = _activations(g, t, n, dtype)
        if op not in ("f8", "gated"):
            state["dy"] = _gradients(g, t, m, dtype)
        if op == "gated_grad" and case["keep"]:
            state["kept"] = (state["x"].float() @ state["w"].float().t()).to(TYPES[dtype])
    if own:
        from paper_2110_03423_amd import Rsvd
        state["ctx"] = Rsvd(0)
    return state


# ---------------------------------------------------------------- one pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    ctx, op = state["ctx"], state["op"]
    if op == "gated":
        return ctx.rsvd_gated_product(state["x"], state["w"], state["act"], keep=state["keep"])
    if op == "gated_grad":
        return ctx.rsvd_gated_product_grad(state["dy"], state["x"], state["w"], state["act"], kept=state.get("kept"))
    if op == "f8":
        return ctx.rsvd_f8_product(state["x"], state["weight"])
    if op == "f8_grad":
        return ctx.rsvd_f8_product_grad(state["dy"], state["weight"])
    if op == "f8_weight":
        return ctx.rsvd_f8_weight_grad(state["dy"], state["x"])
    return ctx.rsvd_orthogonalize(state["G"], STEPS, STEP)


def _act(g, act):
    """The activation and its derivative."""
    if act == "relu":
        return torch.where(g > 0, g, 0.0), (g > 0).to(g.dtype)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if act == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * math.sqrt(0.5 / math.pi)
    k = math.sqrt(2.0 / math.pi)
    th = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * k * (1.0 + 3 * 0.044715 * g * g)


def _run_plain(state):
    op, dtype = state["op"], state["dtype"]
    if op in ("gated", "gated_grad"):
        x, w = state["x"].float(), state["w"].float()
        gu = state["kept"].float() if "kept" in state else x @ w.t()
        m = w.shape[0] // 2
        a, da = _act(gu[:, :m], state["act"])
        if op == "gated":
            h = (a * gu[:, m:]).to(dtype)
            return (h, gu.to(dtype)) if state["keep"] else h
        dh = state["dy"].float()
        d = torch.cat([dh * gu[:, m:] * da, dh * a], dim=1)
        return (d @ w).to(dtype), (d.t() @ x).to(dtype)
    if op in ("f8", "f8_grad"):
        codes, powers = state["weight"]
        w = _values8(codes, powers.int() - 127, 128, 128)
        if op == "f8":
            return (_rounded8(state["x"], 1, 128) @ w.t()).to(dtype)
        return (_rounded8(state["dy"], 1, 128) @ w).to(dtype)
    if op == "f8_weight":
        return (_rounded8(state["dy"], 128, 1).t() @ _rounded8(state["x"], 128, 1)).to(dtype)
    a, b, c = STEP
    x = state["G"].float()
    norm = x.double().square().sum(dim=(1, 2), keepdim=True).sqrt().float()
    x = torch.where(norm > 0, x / norm, 0.0)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        xx = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * xx + c * torch.matmul(xx, xx), x)
    return (x.transpose(1, 2) if tall else x).contiguous().to(dtype)


# ---------------------------------------------------------------- the definition in 64 bits

def _held(x, along):
    """x (fp64) with blocks of 128 along a dimension rounded to 8-bit floats."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[along], 128):
        part = x.narrow(along, at, min(128, x.shape[along] - at))
        top = part.abs().amax(dim=along, keepdim=True)
        some = top >= math.ldexp(1.0, -117)
        unit = torch.full_like(top, math.ldexp(1.0, -126))
        near = torch.exp2(torch.ceil(torch.log2(top[some] / 448.0)))
        near = torch.where(near * 224.0 >= top[some], near / 2.0, near)      # (log2 rounds: quotients that are powers of two)
        unit[some] = torch.where(near * 448.0 < top[some], near * 2.0, near)
        v = part / unit
        # three bits behind the leading one, and 2^-9 at the least
        two = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=1e-30))))
        two = torch.where(two > v.abs(), two / 2.0, torch.where(two * 2.0 <= v.abs(), two * 2.0, two))
        grid = torch.clamp(two / 8.0, min=2.0 ** -9)
        out.narrow(along, at, part.shape[along]).copy_(torch.round(v / grid) * grid * unit)
    return out


def _derivative(z, act):
    if act == "relu":
        return torch.relu(z), torch.heaviside(z, torch.zeros_like(z))
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    r = math.sqrt(8 / math.pi)                 # (1 + tanh y) / 2 = sigmoid(2 y)
    s = torch.sigmoid(r * z * (1 + 0.044715 * z * z))
    return z * s, s + z * s * (1 - s) * r * (1 + 0.134145 * z * z)


def exact(case, seed):
    global own
    before, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = before
    op = case["op"]
    if op in ("gated", "gated_grad"):
        x, w, m = state["x"].double(), state["w"].double(), case["m"]
        if "kept" in state:
            gate, up = state["kept"][:, :m].double(), state["kept"][:, m:].double()
        else:
            gate, up = torch.matmul(x, w[:m].t()), torch.matmul(x, w[m:].t())
        value, slope = _derivative(gate, case["act"])
        if op == "gated":
            h = value.mul_(up)
            return (h, torch.hstack([gate, up])) if case["keep"] else h
        dy = state["dy"].double()
        d_gate, d_up = slope.mul_(up).mul_(dy), value.mul_(dy)
        dx = torch.matmul(d_gate, w[:m]).addmm_(d_up, w[m:])
        return dx, torch.vstack([torch.matmul(d_gate.t(), x), torch.matmul(d_up.t(), x)])
    if op in ("f8", "f8_grad"):
        codes, powers = state["weight"]
        w = codes.to(torch.float64)
        for i in range(powers.shape[0]):
            for j in range(powers.shape[1]):
                w[128 * i:128 * i + 128, 128 * j:128 * j + 128] *= 2.0 ** (int(powers[i, j]) - 127)
        return torch.matmul(_held(state["x"].double(), 1), w.t()) if op == "f8" else torch.matmul(_held(state["dy"].double(), 1), w)
    if op == "f8_weight":
        return torch.matmul(_held(state["dy"].double(), 0).t(), _held(state["x"].double(), 0))
    out = []
    for one in state["G"].double():
        y = one / torch.linalg.matrix_norm(one)
        wide = y.shape[0] <= y.shape[1]
        for _ in range(STEPS):
            s = torch.matmul(y, y.t()) if wide else torch.matmul(y.t(), y)
            p = torch.eye(len(s), dtype=s.dtype, device=s.device).mul_(STEP[0]).add_(s, alpha=STEP[1]).addmm_(s, s, alpha=STEP[2])
            y = torch.matmul(p, y) if wide else torch.matmul(y, p)
        out.append(y)
    return torch.stack(out)
