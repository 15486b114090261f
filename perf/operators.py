"""The operators of a pipeline stage's edge whose speed is measured, as a training or serving program calls them.

A stage receives an activation, normalises it, multiplies it by its first weights in 8 bits, and on the way back
takes the gradients of both.  One case is one call (or the calls of one backward step) on tensors the program
holds: `prepare` makes them, `run` computes.  Operators:

  norm           layer norm of rows, with the statistics the backward pass keeps
  norm_backward  its input's gradient, and its weights' gradients summed over the rows
  transit        an activation to 8 bits with one power-of-two scale per 128 elements of a row, and back
  product        x W^T of two 8-bit matrices with a scale per block of 128 along the reduction
  linear_backward  gradients of x W^T in 8 bits: the output's gradient quantised along both axes, two products
"""

import math

import torch

own = False

BLOCK = 128
BYTES = {"float16": 2, "bfloat16": 2, "float32": 4}
EPS = 1e-5


def listed():
    return [
        # one decode step of a 64-sequence batch: latency
        dict(name="norm_decode64_fp16", op="norm", dtype="float16", weights="float16", rows=64, cols=5120),
        # GPT-3-width activation of 8 sequences of 2048: the largest norm
        dict(name="norm_gpt3_bf16", op="norm", dtype="bfloat16", weights="float32", rows=16384, cols=12288),
        # a small fp32 layer
        dict(name="norm_grad_small_fp32", op="norm_backward", dtype="float32", weights="float32", rows=256, cols=1024),
        # a width that vectors of 16 bytes do not divide evenly among lanes, next-token rows (2047)
        dict(name="norm_grad_uneven_bf16", op="norm_backward", dtype="bfloat16", weights="float32", rows=16376,
             cols=12300),
        # a small shard whose last block is short (390 = 3 * 128 + 6)
        dict(name="transit_small_ragged_fp16", op="transit", dtype="float16", rows=128, cols=390),
        # the GPT-3-width activation between two stages
        dict(name="transit_gpt3_bf16", op="transit", dtype="bfloat16", rows=16384, cols=12288),
        # one token against a stage's projection: the weights' bytes are the work
        dict(name="product_one_token", op="product", m=1, n=12288, k=12288, scales="e8m0", tiles=True, out="bfloat16"),
        # a decode step of 64 sequences, query, key and value at once, weights with float scales
        dict(name="product_decode64_fp32_scales", op="product", m=64, n=15360, k=5120, scales="float32", tiles=True,
             out="float16"),
        # a next-token batch, odd width, reduction with a short last block, float scales
        dict(name="product_ragged_fp32_scales", op="product", m=16376, n=8191, k=4098, scales="float32", tiles=True,
             out="bfloat16"),
        # the GPT-3-width projection of 8 sequences: the largest
        dict(name="product_gpt3", op="product", m=16384, n=12288, k=12288, scales="e8m0", tiles=True, out="bfloat16"),
        # backward on a next-token sequence (2047) of a layer of odd widths
        dict(name="linear_backward_ragged", op="linear_backward", dtype="float16", m=2047, n=4098, k=5130),
        # backward of the GPT layer's widening projection, one micro-batch of 8 x 1024 tokens
        dict(name="linear_backward_gpt", op="linear_backward", dtype="bfloat16", m=8192, n=16384, k=4096),
    ]


# ------------------------------------------------------------------ the ranges

def _extent(rng, lo, hi):
    """Log-uniform; half of them whole blocks where they are long enough, the others as drawn, odd ones among them."""
    while True:
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if v >= BLOCK and rng.random() < 0.5:
            v = v // BLOCK * BLOCK
        if v != 3072:
            return v


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "transit", "product", "product", "linear_backward"])
    while True:
        if op in ("norm", "norm_backward", "transit"):
            case = dict(op=op, dtype=rng.choice(["float16", "bfloat16", "float32"]), rows=_extent(rng, 1, 16384),
                        cols=_extent(rng, 128, 16384))
            if op != "transit":
                case["weights"] = rng.choice([case["dtype"], "float32"])
            if work(case)["bytes"] <= 1.2e9:
                return case
        elif op == "product":
            # M from one token to a batch of sequences, weights of a projection
            case = dict(op=op, m=_extent(rng, 1, 16384), n=_extent(rng, 128, 16384), k=_extent(rng, 128, 16384),
                        scales=rng.choice(["e8m0", "float32"]), tiles=rng.random() < 0.75,
                        out=rng.choice(["bfloat16", "float16", "float32"]))
            if work(case)["flops"] <= 4.9e12:
                return case
        else:
            case = dict(op=op, dtype=rng.choice(["float16", "bfloat16"]), m=_extent(rng, 256, 16384),
                        n=_extent(rng, 256, 16384), k=_extent(rng, 256, 16384))
            if work(case)["flops"] <= 2.4e12:
                return case


# ------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activation(g, rows, cols, dtype):
    """N(0,1) about an offset per channel, one channel in 256 twenty times as wide, as transformers' activations are."""
    wide = torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 256, 20.0, 1.0)
    shift = 0.2 * torch.randn(cols, generator=g, device="cuda")
    x = torch.randn(rows, cols, generator=g, device="cuda")
    return x.mul_(wide).add_(shift).to(getattr(torch, dtype))


def _gradient(g, rows, cols, dtype):
    """Small, and of another size from token to token."""
    size = torch.exp(torch.randn(rows, 1, generator=g, device="cuda")) * 1e-2
    return torch.randn(rows, cols, generator=g, device="cuda").mul_(size).to(getattr(torch, dtype))


def _up(n, unit):
    return -(-n // unit) * unit


def _blocks_amax(x, rows_per_block):
    """Largest magnitude of each block of rows_per_block rows and 128 columns."""
    r, c = x.shape
    nr, nc = -(-r // rows_per_block), -(-c // BLOCK)
    if r % rows_per_block or c % BLOCK:
        x = torch.nn.functional.pad(x, (0, nc * BLOCK - c, 0, nr * rows_per_block - r))
    return x.abs().view(nr, rows_per_block, nc, BLOCK).amax(dim=(1, 3))


def _spread(s, rows_per_block, shape):
    """A block's scale at each of its elements."""
    if rows_per_block > 1:
        s = s.repeat_interleave(rows_per_block, 0)[:shape[0]]
    return s.repeat_interleave(BLOCK, 1)[:, :shape[1]]


def _power_of_two(amax):
    """The smallest power of two s (from 2^-126) with amax / s <= 448 = 1.75 * 2^8; 1 for a block of zeros."""
    bits = (amax.view(torch.int32) + 0x1FFFFF) >> 23  # exponent of amax, one more above 1.75
    e = torch.where(amax > 0, (bits - 8).clamp(min=1), 127)
    return (e << 23).view(torch.float32)


def _quantise(x, rows_per_block=1):
    """(codes, scales as float32) of a float32 matrix."""
    s = _power_of_two(_blocks_amax(x, rows_per_block))
    return (x / _spread(s, rows_per_block, x.shape)).to(torch.float8_e4m3fn), s


def _values(q, s, rows_per_block=1):
    """The float32 values that codes and scales stand for."""
    return q.float() * _spread(s.float(), rows_per_block, q.shape)


def _held(q):
    """Codes as a program holds them: rows padded to whole blocks, so that each starts on a 16-byte boundary."""
    full = torch.zeros(q.shape[0], _up(q.shape[1], BLOCK), device=q.device, dtype=torch.uint8)
    full[:, :q.shape[1]] = q.view(torch.uint8)
    return full.view(torch.float8_e4m3fn)[:, :q.shape[1]]


def _matrix(g, x, rows_per_block, scales):
    """An 8-bit matrix in hand: (codes, scales, rows per block). Float scales take any value, as published weights' do."""
    q, s = _quantise(x, rows_per_block)
    if scales == "e8m0":
        s = s.to(torch.float8_e8m0fnu)
    else:
        s = s * (0.5 + 0.5 * torch.rand(s.shape, generator=g, device="cuda"))
    return _held(q), s, rows_per_block


# ------------------------------------------------------------------ prepare

def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    if op in ("norm", "norm_backward"):
        rows, cols = case["rows"], case["cols"]
        wt = getattr(torch, case["weights"])
        s = {"x": _activation(g, rows, cols, case["dtype"]),
             "w": (1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(wt),
             "b": (0.1 * torch.randn(cols, generator=g, device="cuda")).to(wt)}
        if op == "norm_backward":
            s["dy"] = _gradient(g, rows, cols, case["dtype"])
            s["mean"], s["rstd"] = _statistics(s["x"].float())
    elif op == "transit":
        s = {"x": _activation(g, case["rows"], case["cols"], case["dtype"])}
    elif op == "product":
        m, n, k = case["m"], case["n"], case["k"]
        s = {"a": _matrix(g, _activation(g, m, k, "float32"), 1, case["scales"]),
             "b": _matrix(g, 0.02 * torch.randn(n, k, generator=g, device="cuda"), BLOCK if case["tiles"] else 1,
                          case["scales"]),
             "out": getattr(torch, case["out"])}
    else:
        m, n, k = case["m"], case["n"], case["k"]
        # kept from the forward pass: the weights in tiles, transposed, and the input quantised along the tokens
        s = {"dy": _gradient(g, m, n, case["dtype"]),
             "wt": _matrix(g, 0.02 * torch.randn(k, n, generator=g, device="cuda"), BLOCK, "e8m0"),
             "xt": _matrix(g, _activation(g, m, k, "float32").t().contiguous(), 1, "e8m0")}
    s["op"] = op
    return s


# ------------------------------------------------------------------ run

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2211_05322_amd import binding as B

    if s["op"] == "norm":
        y, mean, rstd = B.reshard_layer_norm(s["x"], s["w"], s["b"], EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if s["op"] == "norm_backward":
        dx, dw, db = B.reshard_layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"])
        return {"dx": dx, "dw": dw, "db": db}
    if s["op"] == "transit":
        return B.reshard_dequantize(B.reshard_quantize(s["x"]), s["x"].dtype)
    if s["op"] == "product":
        return B.reshard_matmul(B.Blocked(*s["a"]), B.Blocked(*s["b"]), s["out"])
    rows, columns = B.reshard_quantize(s["dy"], transposed="both")
    dx = B.reshard_matmul(rows, B.Blocked(*s["wt"]), s["dy"].dtype)
    return {"dx": dx, "dw": B.reshard_matmul(columns, B.Blocked(*s["xt"]), torch.float32)}


def _statistics(x):
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, 1 / torch.sqrt(var + EPS)


def _run_plain(s):
    if s["op"] == "norm":
        x = s["x"].float()
        mean, rstd = _statistics(x)
        y = (x - mean[:, None]) * rstd[:, None] * s["w"].float() + s["b"].float()
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if s["op"] == "norm_backward":
        dy, x = s["dy"].float(), s["x"].float()
        xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
        dw, db = (dy * xhat).sum(0), dy.sum(0)
        dy = dy * s["w"].float()
        dx = s["rstd"][:, None] * (dy - dy.mean(1, keepdim=True) - xhat * (dy * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dw": dw, "db": db}
    if s["op"] == "transit":
        return _values(*_quantise(s["x"].float())).to(s["x"].dtype)
    if s["op"] == "product":
        return torch.matmul(_values(*s["a"]), _values(*s["b"]).t()).to(s["out"])
    dy = s["dy"].float()
    dx = torch.matmul(_values(*_quantise(dy)), _values(*s["wt"]).t())
    dw = torch.matmul(_values(*_quantise(dy.t().contiguous())), _values(*s["xt"]).t())
    return {"dx": dx.to(s["dy"].dtype), "dw": dw}


# ------------------------------------------------------------------ work

def work(case):
    op = case["op"]
    if op in ("norm", "norm_backward", "transit"):
        r, c, e = case["rows"], case["cols"], BYTES[case["dtype"]]
        if op == "norm":
            return {"bytes": 2 * r * c * e + 2 * c * BYTES[case["weights"]] + 8 * r, "flops": 8 * r * c}
        if op == "norm_backward":
            return {"bytes": 3 * r * c * e + c * BYTES[case["weights"]] + 8 * r + 8 * c, "flops": 14 * r * c}
        # to 8 bits (read, written) and back (read, written)
        return {"bytes": 2 * (r * c * e + r * c + r * -(-c // BLOCK)), "flops": 4 * r * c}
    m, n, k = case["m"], case["n"], case["k"]
    if op == "product":
        es = 1 if case["scales"] == "e8m0" else 4
        kb = -(-k // BLOCK)
        scales = es * kb * (m + (-(-n // BLOCK) if case["tiles"] else n))
        return {"bytes": m * k + n * k + scales + m * n * BYTES[case["out"]], "flops": 2 * m * n * k}
    # dy read once and written in two orders, those and both kept operands read, dx and dw written
    return {"bytes": m * n * (BYTES[case["dtype"]] + 4) + k * n + k * m + m * k * BYTES[case["dtype"]] + 4 * n * k,
            "flops": 4 * m * n * k}


# ------------------------------------------------------------------ the definition in 64 bits

def _e4m3_64(v):
    """v (|v| <= 448) to the nearest of e4m3's values, ties to even: steps of 2^(exponent - 3), 2^-9 below 2^-6."""
    _, e = torch.frexp(v)  # v = f * 2^e, f in [1/2, 1)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def _quantised_64(x):
    """x, in double, rounded in blocks of 128 along its last axis; the values that the codes stand for."""
    r, c = x.shape
    out = torch.empty_like(x)
    for lo in range(0, c, BLOCK):
        b = x[:, lo:lo + BLOCK]
        f, e = torch.frexp(b.abs().amax(1, keepdim=True) / 448)  # s = 2^e, or 2^(e-1) where that holds it exactly
        s = torch.exp2(torch.where(f == 0.5, e - 1, e).clamp(min=-126).double())
        out[:, lo:lo + BLOCK] = _e4m3_64(b / s) * s
    return out


def _values_64(q, s, rows_per_block):
    v = q.double()
    s = s.float().double()
    for j in range(s.shape[1]):
        col = s[:, j:j + 1]
        if rows_per_block > 1:
            col = col.repeat_interleave(rows_per_block, 0)[:v.shape[0]]
        v[:, j * BLOCK:(j + 1) * BLOCK] *= col
    return v


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        x.sub_(mean[:, None]).mul_(rstd[:, None]).mul_(s["w"].double()).add_(s["b"].double())
        return {"y": x, "mean": mean, "rstd": rstd}
    if op == "norm_backward":
        dy, xhat = s["dy"].double(), s["x"].double()
        xhat.sub_(s["mean"].double()[:, None]).mul_(s["rstd"].double()[:, None])
        cols = xhat.shape[1]
        db, dw = dy.sum(0), torch.linalg.vecdot(dy, xhat, dim=0)
        dy.mul_(s["w"].double())
        along = torch.linalg.vecdot(dy, xhat, dim=1)[:, None] / cols
        dx = (dy - dy.sum(1, keepdim=True) / cols - xhat * along) * s["rstd"].double()[:, None]
        return {"dx": dx, "dw": dw, "db": db}
    if op == "transit":
        return _quantised_64(s["x"].double())
    if op == "product":
        return _values_64(*s["a"]) @ _values_64(*s["b"]).t()
    dy = s["dy"].double()
    return {"dx": _quantised_64(dy) @ _values_64(*s["wt"]).t(),
            "dw": _quantised_64(dy.t().contiguous()) @ _values_64(*s["xt"]).t()}
