"""The operators at a stage's edge against plain implementations in 64 bits.

layer norm and its gradients, matrices in 8 bits with a scale per block of
128 and back, and the product of two of them.  Quantising and reading back are
compared exactly.  The others' tolerances follow from what the kernels round:
every result once to its type (half a unit in the last place, U), and float32
sums.  A float32 sum of terms t, taken in a chain of at most d additions, is
off by at most d * 2^-24 * sum|t|.

GPU tests unless marked otherwise; refusals run on the CPU, since arguments are
checked before anything is launched.
"""

import itertools
import math
import zlib

import numpy as np
import pytest
import torch

from paper_2211_05322_amd import binding as B

gpu = pytest.mark.gpu
E8M0, E4M3 = torch.float8_e8m0fnu, torch.float8_e4m3fn
HALVES = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # U, relative
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # U of subnormals
F32 = 2.0 ** -24


def _seed(*what):
    return torch.Generator().manual_seed(zlib.crc32(repr(what).encode()))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def _pitched(t, extra, fill):
    """t on the GPU with `extra` more elements from row to row, those elements `fill`; and the whole buffer."""
    rows, cols = t.shape
    whole = torch.empty((rows, cols + extra), dtype=t.dtype, device="cuda")
    whole.view(torch.uint8).fill_(fill)
    whole[:, :cols] = t.cuda()
    return whole[:, :cols], whole


def _guarded(shape, dtype, extra=5):
    """An output with room after each row and after the last, all bytes 0x5A; and a check that the room is untouched."""
    rows, cols = shape
    flat = torch.empty((rows + 1) * (cols + extra) * dtype.itemsize, dtype=torch.uint8, device="cuda").fill_(0x5A)
    whole = flat.view(dtype).view(rows + 1, cols + extra)

    def untouched():
        left = whole.view(torch.uint8).clone().view(rows + 1, -1)
        left[:rows, :cols * dtype.itemsize] = 0x5A
        return bool((left == 0x5A).all())
    return whole[:rows, :cols], untouched


def _near(got, want, bound, what):
    got, want, bound = (v.double().cpu() for v in (got, want, bound))
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    off = torch.nan_to_num((got - want).abs(), nan=0.0)
    worst = (off - bound).nan_to_num(nan=0.0).max().item() if off.numel() else 0.0
    assert worst <= 0, f"{what}: {worst:.3e} over the bound"


# ------------------------------------------------------------------ layer norm

def _norm64(x, w, b, eps):
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    return (x - mean) * rstd * w + b, mean, rstd


# additions in a chain: a thread's own elements (32 at most, or the row's
# share of 1024 threads), 6 across a wave, 16 across waves
def _chain(cols):
    return max(32, math.ceil(cols / 1024) + 8) + 22


NORM_COLS = [1, 7, 64, 65, 390, 512, 1000, 2047, 2048, 4097, 5120, 12300, 16384, 16392, 33000]


@gpu
@pytest.mark.parametrize("cols", NORM_COLS)
@pytest.mark.parametrize("dtype", list(HALVES), ids=str)
def test_layer_norm(dtype, cols, gpu_lib):
    g = _seed("norm", dtype, cols)
    rows, extra = 5, cols % 3
    x = (_randn(g, rows, cols) * torch.exp(_randn(g, rows, 1)) + 3 * _randn(g, rows, 1)).to(dtype)
    for wt in sorted({dtype, torch.float32}, key=str):
        w, b = (1 + 0.3 * _randn(g, cols)).to(wt), _randn(g, cols).to(wt)
        xd, _ = _pitched(x, extra, 0xFF)  # NaN between the rows
        out, untouched = _guarded((rows, cols), dtype)
        y, mean, rstd = B.reshard_layer_norm(xd, w.cuda(), b.cuda(), 1e-5, out=out)
        torch.cuda.synchronize()
        x64, w64, b64 = x.double(), w.double(), b.double()
        want, m64, r64 = _norm64(x64, w64, b64, 1e-5)
        d = _chain(cols)
        dm = (d + 2) * F32 * x64.abs().mean(1, keepdim=True)
        spread = (x64 - m64).abs()
        # the variance: its own chain, plus what the mean's error adds (twice dm * mean|x - m|, and dm^2)
        dv = (d + 6) * F32 * (spread ** 2).mean(1, keepdim=True) + 2 * dm * spread.mean(1, keepdim=True) + dm ** 2
        dr = r64 * (0.5 * dv * r64 ** 2 + 4 * F32)
        _near(mean[:, None], m64, dm, "mean")
        _near(rstd[:, None], r64, dr + r64 * (dv * r64 ** 2) ** 2, "rstd")
        within = w64.abs() * (spread * dr + dm * r64) * 1.01 + 6 * F32 * ((spread * r64 * w64).abs() + b64.abs())
        _near(y, want, within + HALVES[dtype] * (want.abs() + within) + TINY[dtype], f"y with {wt} weights")
        assert untouched()


@gpu
def test_layer_norm_without_weights_in_place_and_no_rows(gpu_lib):
    g = _seed("plain")
    x = _randn(g, 9, 130).float()
    want, m64, r64 = _norm64(x.double(), 1.0, 0.0, 0.0)
    xd = x.cuda()
    y, _, _ = B.reshard_layer_norm(xd, eps=0.0, out=xd)
    assert y is xd
    _near(y, want, 100 * F32 * (1 + want.abs()), "in place")
    y, mean, rstd = B.reshard_layer_norm(torch.empty(0, 130, device="cuda"))
    assert y.shape == (0, 130) and mean.shape == (0,) and rstd.shape == (0,)
    y3, m3, _ = B.reshard_layer_norm(x.cuda().view(3, 3, 130))
    assert y3.shape == (3, 3, 130) and m3.shape == (3, 3)


@gpu
@pytest.mark.parametrize("cols", [3, 130, 777, 4098])
@pytest.mark.parametrize("dtype,wt", [(torch.float32, torch.float16), (torch.float32, torch.bfloat16),
                                      (torch.bfloat16, torch.float16), (torch.float16, torch.bfloat16)], ids=str)
def test_layer_norm_weights_of_another_type(dtype, wt, cols, gpu_lib):
    """Weights of one 16-bit type equal the same weights in float32, bit for bit, in both passes; either may be left out."""
    g = _seed("types", dtype, wt, cols)
    x, dy = _randn(g, 6, cols).to(dtype).cuda(), _randn(g, 6, cols).to(dtype).cuda()
    w, b = (_randn(g, cols).to(wt).cuda() for _ in range(2))
    for weight, bias in ((w, b), (w, None), (None, b)):
        got = B.reshard_layer_norm(x, weight, bias)
        want = B.reshard_layer_norm(x, *(None if v is None else v.float() for v in (weight, bias)))
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    got = B.reshard_layer_norm_backward(dy, x, w, *got[1:])
    want = B.reshard_layer_norm_backward(dy, x, w.float(), *want[1:])
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@gpu
def test_layer_norm_special_rows(gpu_lib):
    """A constant row, the type's largest values, and rows with NaN or an infinity, beside ordinary ones."""
    cols = 777
    x = _randn(_seed("special"), 6, cols).float()
    x[1] = 4.0
    x[2] = 3e38 * torch.sign(x[2])
    x[3, 5] = float("nan")
    x[4, 776] = float("inf")
    y, mean, rstd = (t.cpu() for t in B.reshard_layer_norm(x.cuda(), eps=1e-5))
    assert (y[1] == 0).all() and mean[1] == 4.0
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    want, _, _ = _norm64(x[[0, 5]].double(), 1.0, 0.0, 1e-5)
    _near(y[[0, 5]], want, 100 * F32 * (1 + want.abs()), "ordinary rows")


def _norm_grad64(dy, x, w, mean, rstd):
    xh = (x - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), xh


@gpu
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (1, 512), (700, 65), (513, 390), (1025, 1000), (37, 2048),
                                       (9, 4097), (600, 5120), (5, 12300), (3, 16384), (530, 16392), (3, 33000)])
@pytest.mark.parametrize("dtype", list(HALVES), ids=str)
def test_layer_norm_backward(dtype, rows, cols, gpu_lib):
    g = _seed("grad", dtype, rows, cols)
    x, dy = (_randn(g, rows, cols) + 0.5).to(dtype), (_randn(g, rows, cols) * 0.1).to(dtype)
    wt = torch.float32 if rows % 2 else dtype
    w = (1 + 0.3 * _randn(g, cols)).to(wt)
    _, m64, r64 = _norm64(x.double(), 1.0, 0.0, 1e-5)
    mean, rstd = m64.float().flatten(), r64.float().flatten()
    xd, _ = _pitched(x, cols % 3, 0xFF)
    dyd, _ = _pitched(dy, (cols + 1) % 3, 0xFF)
    out, untouched = _guarded((rows, cols), dtype)
    start = _randn(g, 2, cols).float()
    held = start.cuda()
    dx, dw, db = B.reshard_layer_norm_backward(dyd, xd, w.cuda(), mean.cuda(), rstd.cuda(), dweight=held[0],
                                               dbias=held[1], accumulate=True, out=out)
    again = B.reshard_layer_norm_backward(dyd, xd, w.cuda(), mean.cuda(), rstd.cuda())
    torch.cuda.synchronize()
    dy64, x64, w64 = dy.double(), x.double(), w.double()
    mean64, rstd64 = mean.double()[:, None], rstd.double()[:, None]
    wdx, wdw, wdb, xh = _norm_grad64(dy64, x64, w64, mean64, rstd64)
    gw = dy64 * w64
    d = 2 * _chain(cols)  # a thread's elements twice over: dy w and its product with xhat
    size = gw.abs() + gw.abs().mean(1, keepdim=True) + xh.abs() * (gw * xh).abs().mean(1, keepdim=True)
    within = (d + 12) * F32 * rstd64 * size
    _near(dx, wdx, within + HALVES[dtype] * (wdx.abs() + within) + TINY[dtype], "dx")
    assert untouched()
    # rows in a chain: at most those of one group of 512, then 512 / 16 groups, 16 waves, one accumulation
    chain = math.ceil(rows / 512) + 32 + 16 + 8
    _near(again[1], wdw, chain * F32 * (dy64 * xh).abs().sum(0) + 1e-30, "dweight")
    _near(again[2], wdb, chain * F32 * dy64.abs().sum(0) + 1e-30, "dbias")
    _near(dw, wdw + start[0].double(), chain * F32 * ((dy64 * xh).abs().sum(0) + start[0].double().abs()), "dweight +=")
    _near(db, wdb + start[1].double(), chain * F32 * (dy64.abs().sum(0) + start[1].double().abs()), "dbias +=")
    assert torch.equal(again[0], dx)
    third = B.reshard_layer_norm_backward(dyd, xd, w.cuda(), mean.cuda(), rstd.cuda())
    assert all(torch.equal(p, q) for p, q in zip(again, third)), "another run, other bits"


@gpu
def test_layer_norm_backward_against_differences(gpu_lib):
    """d/dx, d/dw and d/db of sum(c * y) by central differences of the forward pass in 64 bits."""
    g = _seed("differences")
    rows, cols, h = 3, 17, 1e-5
    x, w, b, c = _randn(g, rows, cols), 1 + 0.3 * _randn(g, cols), _randn(g, cols), _randn(g, rows, cols)
    x, w, b, c = (t.float().double() for t in (x, w, b, c))

    def loss(x, w, b):
        return (c * _norm64(x, w, b, 1e-5)[0]).sum()

    def differences(at, f):
        out = torch.zeros_like(at)
        for i in itertools.product(*map(range, at.shape)):
            step = torch.zeros_like(at)
            step[i] = h
            out[i] = (f(at + step) - f(at - step)) / (2 * h)
        return out
    _, mean, rstd = B.reshard_layer_norm(x.float().cuda(), w.float().cuda(), b.float().cuda(), 1e-5)
    dx, dw, db = B.reshard_layer_norm_backward(c.float().cuda(), x.float().cuda(), w.float().cuda(), mean, rstd)
    # float32 kernels on numbers of order 1 to 10: 1e-5; the differences' own error is below 1e-8
    for got, want in ((dx, differences(x, lambda v: loss(v, w, b))), (dw, differences(w, lambda v: loss(x, v, b))),
                      (db, differences(b, lambda v: loss(x, w, v)))):
        _near(got, want, 1e-5 * (1 + want.abs()), "difference")


@gpu
def test_layer_norm_backward_in_place_and_no_rows(gpu_lib):
    g = _seed("in place")
    for cols in (130, 33000):
        x, dy = _randn(g, 4, cols).float().cuda(), _randn(g, 4, cols).float().cuda()
        _, mean, rstd = B.reshard_layer_norm(x)
        want = B.reshard_layer_norm_backward(dy, x, None, mean, rstd)
        got = B.reshard_layer_norm_backward(dy, x, None, mean, rstd, out=dy)
        assert got[0] is dy and all(torch.equal(p, q) for p, q in zip(want, got))
    none = torch.empty(0, 8, device="cuda")
    stat = torch.empty(0, device="cuda")
    _, dw, db = B.reshard_layer_norm_backward(none, none, None, stat, stat)
    assert (dw == 0).all() and (db == 0).all()
    held = torch.ones(2, 8, device="cuda")
    B.reshard_layer_norm_backward(none, none, None, stat, stat, dweight=held[0], dbias=held[1], accumulate=True)
    assert (held == 1).all()


# ------------------------------------------------------------------ 8 bits

def _e4m3_values():
    return torch.arange(256, dtype=torch.uint8).view(E4M3).double()


def _nearest_e4m3(v):
    """Nearest of the format's values to each of v (|v| <= 448), ties to the even code: by search, in 64 bits."""
    table = _e4m3_values()[:127]  # 0 to 448, ascending
    a = v.abs()
    hi = torch.searchsorted(table, a.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up = table[hi] - a
    down = a - table[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(table[code], v)


def _quantise64(x, block_rows):
    """(values the codes stand for, scales) of x in blocks of block_rows x 128."""
    rows, cols = x.shape
    x = x.double()
    scales = torch.empty(-(-rows // block_rows), -(-cols // 128), dtype=torch.float64)
    values = torch.empty_like(x)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            at = slice(i * block_rows, (i + 1) * block_rows), slice(j * 128, (j + 1) * 128)
            blk = x[at]
            fin = torch.where(torch.isfinite(blk), blk.abs(), 0.0).max().item()
            e = 0 if fin == 0 else max(-126, math.ceil(math.log2(fin / 448)))
            while fin and e > -126 and fin / 2.0 ** (e - 1) <= 448:
                e -= 1
            while fin / 2.0 ** e > 448:
                e += 1
            scales[i, j] = 2.0 ** e
            values[at] = torch.where(torch.isfinite(blk), _nearest_e4m3(torch.nan_to_num(blk, 0, 0, 0) / 2.0 ** e) * 2.0 ** e,
                                     float("nan"))
    return values, scales


def _stands_for(b):
    """What a Blocked stands for, in 64 bits on the CPU."""
    rows, cols = b.data.shape
    s = b.scales.cpu().float().double().repeat_interleave(b.block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return b.data.cpu().double() * s


def _same(got, want, what):
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want)), what


@gpu
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 390), (130, 129), (128, 256), (255, 7), (7, 1000), (257, 640)])
@pytest.mark.parametrize("dtype", list(HALVES), ids=str)
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_and_back(block_rows, dtype, rows, cols, gpu_lib):
    g = _seed("quantise", block_rows, dtype, rows, cols)
    x = (_randn(g, rows, cols) * torch.exp(3 * _randn(g, rows, cols))).to(dtype)
    x[torch.rand(rows, cols, generator=g) < 0.05] = 0
    xd, _ = _pitched(x, cols % 3, 0xFF)
    for scale_dtype in (E8M0, torch.float32):
        q = B.reshard_quantize(xd, block_rows, scale_dtype=scale_dtype)
        p, t = B.reshard_quantize(xd, block_rows, transposed="both", scale_dtype=scale_dtype)
        only = B.reshard_quantize(xd, block_rows, transposed=True, scale_dtype=scale_dtype)
        torch.cuda.synchronize()
        values, scales = _quantise64(x, block_rows)
        for b in (q, p):
            _same(b.scales.cpu().double() if scale_dtype != E8M0 else b.scales.cpu().float().double(), scales, "scales")
            _same(_stands_for(b), values, "values")
        tv, ts = _quantise64(x.t().contiguous(), block_rows)
        for b in (t, only):
            _same(b.scales.cpu().float().double(), ts, "transposed scales")
            _same(_stands_for(b), tv, "transposed values")
        for dt in HALVES:
            out, untouched = _guarded((rows, cols), dt)
            back = B.reshard_dequantize(q, dt, out=out)
            torch.cuda.synchronize()
            _same(back.cpu(), values.to(dt), f"back in {dt}")
            assert untouched()


@gpu
def test_quantize_writes_nothing_past_its_outputs(gpu_lib):
    rows, cols = 131, 261
    x = torch.randn(rows, cols, device="cuda")
    for block_rows in (1, 128):
        q, q_ok = _guarded((rows, cols), torch.uint8, 3)
        s, s_ok = _guarded((-(-rows // block_rows), 3), torch.uint8, 2)
        t, t_ok = _guarded((cols, rows), torch.uint8, 6)
        u, u_ok = _guarded((-(-cols // block_rows), 2), torch.uint8, 1)
        B._check(gpu_lib.reshard_quantize(rows, cols, x.data_ptr(), cols, 4, block_rows, 13, q.data_ptr(), q.stride(0),
                                          s.data_ptr(), s.stride(0), t.data_ptr(), t.stride(0), u.data_ptr(),
                                          u.stride(0), B._stream_handle(None)))
        torch.cuda.synchronize()
        assert q_ok() and s_ok() and t_ok() and u_ok()
        p, pt = B.reshard_quantize(x, block_rows, transposed="both")
        assert torch.equal(q, p.data.view(torch.uint8)) and torch.equal(t, pt.data.view(torch.uint8))


@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_special_values(block_rows, gpu_lib):
    """Zeros of both signs, NaN, infinities, subnormals, the largest floats, exact powers and ties."""
    x = torch.zeros(128, 128 * 8)
    x[0, :4] = torch.tensor([1.0, float("nan"), -2.5, 3.0])
    x[0, 128:132] = torch.tensor([float("inf"), -float("inf"), 1.0, -7.0])
    x[0, 256:260] = torch.tensor([1e-45, 2e-40, -3e-39, 0.0])
    x[0, 384:388] = torch.tensor([3.4e38, -1.0, 1e30, 3.3e38])
    x[0, 512:517] = torch.tensor([448.0, 449.0, 0.5, -448.0, 447.9])
    x[0, 640:648] = torch.tensor([448.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, 0.0625 * 1.0625, -17.0])
    x[0, 768:770] = torch.tensor([-0.0, 0.0])
    x[0, 896:898] = torch.tensor([float("nan"), float("inf")])
    xd = x.cuda()
    values, scales = _quantise64(x, block_rows)
    q, t = B.reshard_quantize(xd, block_rows, transposed="both")
    torch.cuda.synchronize()
    _same(q.scales.cpu().float().double(), scales, "scales")
    _same(_stands_for(q), values, "values")
    tv, ts = _quantise64(x.t().contiguous(), block_rows)
    _same(_stands_for(t), tv, "transposed values")
    _same(t.scales.cpu().float().double(), ts, "transposed scales")


@gpu
def test_dequantize_any_float_scale(gpu_lib):
    codes = torch.arange(256, dtype=torch.uint8).repeat(3, 1)
    scales = torch.tensor([[0.3, -1.7], [0.0, float("inf")], [1e-40, float("nan")]])
    got = B.reshard_dequantize(B.Blocked(codes.cuda().view(E4M3), scales.cuda()), torch.float32)
    want = codes.view(E4M3).float() * scales.repeat_interleave(128, 1)
    _same(got.cpu(), want, "float scales")
    e = torch.tensor([[0, 255], [1, 254], [127, 100]], dtype=torch.uint8)
    got = B.reshard_dequantize(B.Blocked(codes.cuda().view(E4M3), e.cuda().view(E8M0)), torch.float32)
    power = torch.where(e == 255, float("nan"), torch.exp2(e.double() - 127))
    want = (codes.view(E4M3).double() * power.repeat_interleave(128, 1)).float()
    _same(got.cpu(), want, "exponent scales")


# ------------------------------------------------------------------ product

def _operand(g, rows, cols, block_rows, scale_dtype, extra):
    """A Blocked on the GPU with NaN codes between its rows, and what it stands for."""
    codes = torch.randint(0, 256, (rows, cols), generator=g).to(torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x30  # no NaN
    data, _ = _pitched(codes, extra, 0x7F)
    shape = -(-rows // block_rows), -(-cols // 128)
    if scale_dtype == E8M0:
        s = torch.randint(118, 132, shape, generator=g).to(torch.uint8).view(E8M0)
        held, _ = _pitched(s.view(torch.uint8), 3, 0xFF)
        held = held.view(E8M0)
    else:
        s = torch.rand(shape, generator=g) + 0.1
        held, _ = _pitched(s, 3, 0xFF)
    b = B.Blocked(data.view(E4M3), held, block_rows)
    return b, _stands_for(b)


SIZES = [(1, 1, 1), (1, 128, 128), (1, 300, 1000), (3, 257, 390), (16, 64, 4098), (17, 1000, 129), (64, 384, 512),
         (65, 129, 127), (128, 128, 1024), (130, 700, 16), (200, 100, 2047), (257, 513, 640), (300, 260, 272),
         (600, 520, 384), (1025, 260, 130), (4, 5000, 2560), (33, 16, 8192), (48, 200, 2064)]


@gpu
@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("scale_dtype", [E8M0, torch.float32], ids=["e8m0", "fp32"])
@pytest.mark.parametrize("a_rows,b_rows", [(1, 128), (1, 1), (128, 128)])
def test_matmul(a_rows, b_rows, scale_dtype, m, n, k, gpu_lib):
    g = _seed("matmul", a_rows, b_rows, str(scale_dtype), m, n, k)
    for extra in ((-k) % 16, (-k) % 16 + 5):  # rows on 16-byte boundaries, and not
        a, a64 = _operand(g, m, k, a_rows, scale_dtype, extra)
        b, b64 = _operand(g, n, k, b_rows, scale_dtype, extra)
        want, size = a64 @ b64.t(), a64.abs() @ b64.abs().t()
        # a block's 128 products in any order, a scale's two roundings, one addition a block, joined parts
        within = (128 + 4 + math.ceil(k / 128) + 64) * F32 * size
        out, untouched = _guarded((m, n), torch.float32)
        got = B.reshard_matmul(a, b, torch.float32, out=out)
        torch.cuda.synchronize()
        _near(got, want, within + F32 * (want.abs() + within), f"float32, extra {extra}")
        assert untouched()
        # 16-bit results: eight neighbouring products are each cut by less than 2^-13 of the largest of them
        cut = within + 2.0 ** -10 * size
        for dt in (torch.float16, torch.bfloat16):
            out, untouched = _guarded((m, n), dt)
            got = B.reshard_matmul(a, b, dt, out=out)
            torch.cuda.synchronize()
            lim = torch.finfo(dt).max
            sure = want.abs() + cut <= lim  # past it, infinity or the largest value
            _near(got.cpu().double()[sure], want[sure], (cut + HALVES[dt] * (want.abs() + cut) + TINY[dt])[sure],
                  f"{dt} extra {extra}")
            assert untouched()
        start = _randn(g, m, n).float()
        held = start.cuda()
        B.reshard_matmul(a, b, out=held, accumulate=True)
        _near(held, want + start.double(), within + 2 * F32 * (want.abs() + within + start.double().abs()), "accumulated")
        first, second = B.reshard_matmul(a, b, torch.float32), B.reshard_matmul(a, b, torch.float32)
        assert torch.equal(first, second), "another run, other bits"


# the reduction in parts (few tiles, a long reduction: whole, odd and short blocks at the parts' ends), and tiles of 256 x 256
@gpu
@pytest.mark.parametrize("m,n,k", [(65, 130, 2048), (130, 260, 4098), (100, 70, 9000), (300, 129, 5130), (257, 1000, 8191),
                                   (3080, 4100, 390), (4097, 3300, 640)])
@pytest.mark.parametrize("scale_dtype", [E8M0, torch.float32], ids=["e8m0", "fp32"])
def test_matmul_long_and_large(scale_dtype, m, n, k, gpu_lib):
    g = _seed("long", str(scale_dtype), m, n, k)
    a, a64 = _operand(g, m, k, 1, scale_dtype, (-k) % 16)
    b, b64 = _operand(g, n, k, 128, scale_dtype, (-k) % 16 + 16)
    want, size = a64 @ b64.t(), a64.abs() @ b64.abs().t()
    within = (128 + 4 + math.ceil(k / 128) + 64) * F32 * size
    start = _randn(g, m, n).float()
    for dt, cut in ((torch.float32, within), (torch.bfloat16, within + 2.0 ** -10 * size)):
        out, untouched = _guarded((m, n), dt)
        got = B.reshard_matmul(a, b, dt, out=out)
        torch.cuda.synchronize()
        _near(got, want, cut + HALVES[dt] * (want.abs() + cut), f"{dt}")
        assert untouched()
        assert torch.equal(B.reshard_matmul(a, b, dt), got), "another run, other bits"
        held = start.to(dt).cuda()
        B.reshard_matmul(a, b, out=held, accumulate=True)
        more = start.to(dt).double()
        _near(held, want + more, cut + F32 * (want.abs() + more.abs()) + HALVES[dt] * (want.abs() + cut + more.abs()), "+=")
    need = gpu_lib.reshard_matmul_workspace(m, n, k, 13 if scale_dtype == E8M0 else 4, 4)
    assert (need > 0) == (k >= 2048), "the sizes no longer reach the path that they are for"


@gpu
def test_matmul_special_values(gpu_lib):
    """NaN codes and scales reach their rows and columns alone; without a reduction the product is zeros."""
    g = _seed("special")
    for scale_dtype in (E8M0, torch.float32):
        a, a64 = _operand(g, 70, 300, 1, scale_dtype, 4)
        b, b64 = _operand(g, 90, 300, 1, scale_dtype, 4)
        a.data.view(torch.uint8)[5, 299] = 0x7F
        b.data.view(torch.uint8)[7, 0] = 0xFF
        (a.scales.view(torch.uint8) if scale_dtype == E8M0 else a.scales)[9, 1] = 255 if scale_dtype == E8M0 else float("nan")
        got = B.reshard_matmul(a, b, torch.float32).cpu()
        nan = torch.zeros(70, 90, dtype=torch.bool)
        nan[5], nan[9], nan[:, 7] = True, True, True
        assert torch.equal(torch.isnan(got), nan)
    for accumulate, left in ((False, 0.0), (True, 1.0)):
        empty = B.Blocked(torch.empty(4, 0, device="cuda", dtype=E4M3), torch.empty(4, 0, device="cuda"))
        out = torch.ones(4, 4, device="cuda")
        B.reshard_matmul(empty, empty, out=out, accumulate=accumulate)
        assert (out == left).all()
    none = B.Blocked(torch.empty(0, 256, device="cuda", dtype=E4M3), torch.empty(0, 2, device="cuda"))
    some = B.Blocked(torch.zeros(3, 256, device="cuda", dtype=torch.uint8).view(E4M3), torch.ones(3, 2, device="cuda"))
    assert B.reshard_matmul(none, some).shape == (0, 3) and B.reshard_matmul(some, none).shape == (3, 0)


@gpu
def test_matmul_scales_of_any_exponent(gpu_lib):
    """Scales from the smallest to the largest power of two; products that leave float32's range, both ways."""
    one = torch.full((16, 128), 0x38, dtype=torch.uint8, device="cuda").view(E4M3)  # 1.0
    codes = [0, 1, 2, 64, 120, 127, 134, 190, 252, 253]
    a = B.Blocked(one, torch.tensor([codes[i % 10] for i in range(16)], dtype=torch.uint8, device="cuda").view(16, 1).view(E8M0))
    got = B.reshard_matmul(a, a, torch.float32).cpu().double()
    e = torch.tensor([codes[i % 10] for i in range(16)]).double() - 127
    want = torch.exp2(e[:, None] + e[None] + 7).float().double()
    ordinary = (want >= 2.0 ** -126) & (want < 2.0 ** 127)
    assert torch.equal(got[ordinary], want[ordinary])
    assert (got[want < 2.0 ** -126] <= 2.0 ** -126).all()


@gpu
def test_linear_backward_against_differences(gpu_lib):
    """Both gradients of sum(c * (x w^T)) from 8-bit operands, against differences of that sum in 64 bits."""
    g = _seed("linear")
    m, n, k = 130, 140, 150
    x, w, c = (torch.randint(-8, 9, s, generator=g).float() for s in ((m, k), (n, k), (m, n)))  # exact in 8 bits
    cr, ct = B.reshard_quantize(c.cuda(), transposed="both")
    wt = B.reshard_quantize(w.cuda(), 128, transposed=True)
    xt = B.reshard_quantize(x.cuda(), transposed=True)
    dx = B.reshard_matmul(cr, wt, torch.float32).cpu().double()
    dw = B.reshard_matmul(ct, xt, torch.float32).cpu().double()
    x, w, c = x.double(), w.double(), c.double()
    for got, at, f in ((dx, x, lambda v: (c * (v @ w.t())).sum()), (dw, w, lambda v: (c * (x @ v.t())).sum())):
        for i in [(0, 0), (1, 149), (127, 128), (128, 127), (129, 3), (64, 64)]:
            step = torch.zeros_like(at)
            step[i] = 1.0
            # whole numbers below 2^24 and their differences: exact
            assert got[i].item() == (f(at + step) - f(at - step)).item() / 2


# ------------------------------------------------------------------ streams, graphs, large offsets

@gpu
def test_operators_on_another_stream_and_in_a_graph(gpu_lib):
    g = _seed("graph")
    x = _randn(g, 200, 640).to(torch.bfloat16).cuda()
    w = B.reshard_quantize(_randn(g, 384, 640).float().cuda(), 128)

    def step():
        y, mean, rstd = B.reshard_layer_norm(x)
        q, t = B.reshard_quantize(y, transposed="both")
        z = B.reshard_matmul(q, w, torch.float32)
        dw = B.reshard_matmul(t, t, torch.float32)
        return [y, z, dw, *B.reshard_layer_norm_backward(y, x, None, mean, rstd)]
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, _, _ = B.reshard_layer_norm(x, stream=side)
    z = B.reshard_matmul(B.reshard_quantize(y, stream=side), w, torch.float32, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(z, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn in range(4):
        x.copy_(_randn(g, 200, 640).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(got, step()):
            assert torch.equal(p, q), f"replay {turn}"
        torch.cuda.synchronize()


@gpu
def test_offsets_past_32_bits(gpu_lib):
    """Rows so far apart that the last ones lie past 4 GiB (and 2^31 elements) from the first."""
    rows, cols, pitch = 5, 300, (1 << 30) + 12
    store = torch.empty(4 * pitch + 2 * cols, dtype=torch.uint8, device="cuda")
    g = _seed("far")
    codes = torch.randint(0, 0x7F, (rows, cols), generator=g).to(torch.uint8).cuda()
    far = store.as_strided((rows, cols), (pitch, 1))
    far.copy_(codes)
    s = torch.randint(120, 130, (rows, 3), generator=g).to(torch.uint8).cuda().view(E8M0)
    a, b = B.Blocked(far.view(E4M3), s), B.Blocked(codes.view(E4M3), s)
    assert torch.equal(B.reshard_matmul(a, b, torch.float32), B.reshard_matmul(b, b, torch.float32))
    assert torch.equal(B.reshard_matmul(b, a, torch.float32), B.reshard_matmul(b, b, torch.float32))
    assert torch.equal(B.reshard_dequantize(a, torch.float32), B.reshard_dequantize(b, torch.float32))
    half = store.view(torch.float16)
    pitch //= 2
    xs = half.as_strided((rows, cols), (pitch, 1))
    x = _randn(g, rows, cols).to(torch.float16).cuda()
    xs.copy_(x)
    assert all(torch.equal(p, q) for p, q in zip(B.reshard_layer_norm(xs), B.reshard_layer_norm(x)))
    p, q = B.reshard_quantize(xs, transposed="both"), B.reshard_quantize(x, transposed="both")
    for u, v in zip(p, q):
        assert torch.equal(u.data.view(torch.uint8), v.data.view(torch.uint8))


# ------------------------------------------------------------------ refusals (CPU)

def _answer(status):
    return status, B.reshard_last_error()


def _refused(answer, status, text):
    assert answer[0] == status and text in answer[1], answer


P = 1 << 20  # an aligned address that is never used


def test_layer_norm_refusals():
    lib = B.load()

    def fwd(rows=4, cols=8, x=P, xp=8, dt=4, w=P, b=P, wt=4, eps=1e-5, y=P, yp=8):
        return _answer(lib.reshard_layer_norm(rows, cols, x, xp, dt, w, b, wt, eps, y, yp, P, P, None))

    def bwd(rows=4, cols=8, dy=P, x=P, dt=4, mean=P, dx=P, dw=P, acc=0, work=P, nbytes=1 << 20):
        return _answer(lib.reshard_layer_norm_backward(rows, cols, dy, cols, x, cols, dt, P, 4, mean, P, dx, cols, dw, P, acc,
                                               work, nbytes, None))
    EI, EU = B.RESHARD_EINVAL, B.RESHARD_EUNSUPPORTED
    for call, status, text in (
            (fwd(rows=-1), EI, "rows"), (fwd(cols=0), EI, "cols"), (fwd(cols=(1 << 24) + 1, xp=1 << 25, yp=1 << 25), EU, "cols"),
            (fwd(x=None), EI, "x is NULL"), (fwd(y=None), EI, "y is NULL"), (fwd(xp=7), EI, "pitch"),
            (fwd(x=P + 2), EI, "aligned"), (fwd(dt=6), EI, "dtype"), (fwd(wt=0), EI, "weight_dtype"),
            (fwd(eps=-1.0), EI, "eps"), (fwd(eps=float("nan")), EI, "eps"), (fwd(rows=1 << 41), EU, "rows"),
            (bwd(rows=-2), EI, "rows"), (bwd(dy=None), EI, "dy is NULL"), (bwd(mean=None), EI, "mean is NULL"),
            (bwd(acc=2), EI, "accumulate"), (bwd(work=None), EI, "workspace"), (bwd(nbytes=16), EI, "workspace"),
            (bwd(work=P + 4), EI, "workspace"), (bwd(dt=12), EI, "dtype"), (bwd(dx=P + 1), EI, "dx is not aligned")):
        _refused(call, status, text)
    assert lib.reshard_layer_norm_backward_workspace(-1, 8) == -1
    assert lib.reshard_layer_norm_backward_workspace(4, 0) == -1


def test_quantize_refusals():
    lib = B.load()
    EI, EU = B.RESHARD_EINVAL, B.RESHARD_EUNSUPPORTED

    def quant(rows=4, cols=300, x=P, dt=3, block=1, st=13, q=P, qp=300, s=P, sp=3, qt=None, qtp=4, su=None, sup=1):
        return _answer(lib.reshard_quantize(rows, cols, x, cols, dt, block, st, q, qp, s, sp, qt, qtp, su, sup, None))

    def back(rows=4, cols=300, q=P, block=1, s=P, st=13, y=P, dt=3, sp=3):
        return _answer(lib.reshard_dequantize(rows, cols, q, cols, block, s, sp, st, y, cols, dt, None))
    for call, status, text in (
            (quant(rows=-1), EI, "rows"), (quant(cols=-1), EI, "cols"), (quant(block=64), EI, "block_rows"),
            (quant(st=3), EI, "scale_dtype"), (quant(dt=12), EI, "dtype"), (quant(q=None), EI, "both NULL"),
            (quant(x=None), EI, "x is NULL"), (quant(qp=299), EI, "q: a pitch"), (quant(sp=2), EI, "scales: a pitch"),
            (quant(s=None), EI, "scales is NULL"), (quant(qt=P, su=None), EI, "scales_t is NULL"),
            (quant(qt=P, su=P, qtp=3), EI, "qt: a pitch"), (quant(st=4, s=P + 2), EI, "scales is not aligned"),
            (quant(rows=(1 << 29) + 1, cols=1, qp=1, sp=1), EU, "2^29"), (back(block=2), EI, "block_rows"),
            (back(q=None), EI, "q is NULL"), (back(s=None), EI, "scales is NULL"), (back(y=None), EI, "y is NULL"),
            (back(dt=13), EI, "dtype"), (back(st=0), EI, "scale_dtype"), (back(sp=1), EI, "scales: a pitch")):
        _refused(call, status, text)


def test_matmul_refusals():
    lib = B.load()
    EI, EU = B.RESHARD_EINVAL, B.RESHARD_EUNSUPPORTED

    def mul(m=4, n=4, k=300, a=P, ap=300, ar=1, sa=P, sap=3, b=P, bp=300, br=128, sb=P, sbp=3, st=13, out=P, op=4, ot=3,
            acc=0):
        return _answer(lib.reshard_matmul(m, n, k, a, ap, ar, sa, sap, b, bp, br, sb, sbp, st, out, op, ot, acc, None, 0, None))
    for call, status, text in (
            (mul(m=-1), EI, "m is negative"), (mul(n=-1), EI, "n is negative"), (mul(k=-1), EI, "k is negative"),
            (mul(a=None), EI, "a is NULL"), (mul(b=None), EI, "b is NULL"), (mul(out=None), EI, "out is NULL"),
            (mul(sa=None), EI, "a_scales is NULL"), (mul(sb=None), EI, "b_scales is NULL"), (mul(ap=200), EI, "a: a pitch"),
            (mul(bp=200), EI, "b: a pitch"), (mul(op=3), EI, "out: a pitch"), (mul(sap=2), EI, "a_scales: a pitch"),
            (mul(ar=2), EI, "a_block_rows"), (mul(br=0), EI, "b_block_rows"), (mul(st=2), EI, "scale_dtype"),
            (mul(ot=6), EI, "out_dtype"), (mul(acc=-1), EI, "accumulate"), (mul(out=P + 1), EI, "aligned"),
            (mul(m=1 << 30, n=1 << 30, op=1 << 30), EU, "out")):
        _refused(call, status, text)
    assert lib.reshard_matmul_workspace(-1, 1, 1, 13, 3) == -1
    need = lib.reshard_matmul_workspace(128, 128, 8192, 13, 3)  # a reduction in parts
    assert need > 0

    def split(work, nbytes):
        return _answer(lib.reshard_matmul(128, 128, 8192, P, 8192, 1, P, 64, P, 8192, 128, P, 64, 13, P, 128, 3, 0, work, nbytes,
                                          None))
    for answer in (split(None, need), split(P, need - 1), split(P + 4, need)):
        _refused(answer, EI, "workspace")


def test_binding_refusals():
    x = torch.zeros(4, 300)
    codes, ones = torch.zeros(4, 300, dtype=torch.uint8).view(E4M3), torch.ones(4, 3)
    b = B.Blocked(codes, ones)
    for call, text in (
            (lambda: B.reshard_layer_norm(x, torch.ones(299)), "weight"),
            (lambda: B.reshard_layer_norm(x.t()), "dense"),
            (lambda: B.reshard_layer_norm(x, out=torch.empty(4, 301)), "out"),
            (lambda: B.reshard_layer_norm_backward(x.half(), x, None, ones[:, 0], ones[:, 0]), "dy"),
            (lambda: B.reshard_layer_norm_backward(x, x, None, ones[:3, 0], ones[:, 0]), "mean"),
            (lambda: B.reshard_layer_norm_backward(x, x, None, x[:, 0].clone(), x[:, 0].clone(), accumulate=True), "accumulate"),
            (lambda: B.reshard_quantize(x, 3), "block_rows"), (lambda: B.reshard_quantize(x, transposed=2), "transposed"),
            (lambda: B.reshard_dequantize(B.Blocked(x, ones), torch.float32), "float8_e4m3fn"),
            (lambda: B.reshard_dequantize(B.Blocked(codes, ones, 128), torch.float32), "scales must be"),
            (lambda: B.reshard_matmul(b, B.Blocked(codes[:, :299], ones)), "columns"),
            (lambda: B.reshard_matmul(b, B.Blocked(codes, ones.to(E8M0))), "scales"),
            (lambda: B.reshard_layer_norm(x), "on the GPU"), (lambda: B.reshard_quantize(x), "on the GPU"),
            (lambda: B.reshard_layer_norm_backward(x, x, None, x[:, 0].clone(), x[:, 0].clone()), "on the GPU"),
            (lambda: B.reshard_dequantize(b, torch.float32), "on the GPU"), (lambda: B.reshard_matmul(b, b), "on the GPU"),
            (lambda: B.reshard_matmul(b, b, accumulate=True), "accumulate"),
            (lambda: B.reshard_matmul(b, b, torch.float32, out=torch.empty(4, 5)), "out")):
        with pytest.raises(ValueError, match=text):
            call()


def test_blocked_types_reshard():
    """Codes and exponent scales are element types of a plan: a plan on each moves a Blocked."""
    codes = torch.arange(32, dtype=torch.uint8).reshape(4, 8)
    for name in ("float8_e4m3fn", "float8_e8m0fnu"):
        plan = B.reshard_plan((4, 8), name, (2,), "S^0 R", (2,), "R S^0")
        src = [codes[:2].clone().view(getattr(torch, name)), codes[2:].clone().view(getattr(torch, name))]
        dst = B.empty_shards(plan, 1, device="cpu")
        B.reshard_debug_execute_host(plan, src, dst)
        for d, want in zip(dst, (codes[:, :4], codes[:, 4:])):
            assert torch.equal(d.view(torch.uint8), want)


def test_plans_refuse_buffers_with_gaps():
    """Codes whose rows are padded are no plan's buffer: moved as if they were dense, the padding would arrive as codes."""
    x = torch.zeros(128, 390)
    padded = B._empty_blocked(x, 128, 390, 1, E8M0, False)[0].data
    dense = B._empty_blocked(x, 128, 390, 1, E8M0, True)[0].data
    assert padded.stride() == (512, 1) and dense.stride() == (390, 1)
    plan = B.reshard_plan((128, 390), E4M3, (1,), "R R", (1,), "R R")
    for src, dst in ((padded, dense), (dense, padded)):
        for move in (B.reshard_debug_execute_host, B.reshard_execute, B.reshard_execute_noalloc):
            with pytest.raises(ValueError, match="dense"):
                move(plan, [src], [dst])
    with pytest.raises(ValueError, match="dense"):
        B.reshard_debug_execute_host(plan, [padded.view(torch.uint8).numpy()], [dense])
    # elements without gaps, in another order of dimensions: a permuted plan's buffer seen as the tensor it holds
    turned = torch.zeros(3, 1, 5, 4).permute(2, 0, 3, 1)
    assert B.pointer_array([turned, padded[:1], padded[:0]])[:] == [turned.data_ptr(), padded.data_ptr(), None]


def test_dense_codes_reshard_at_an_odd_width():
    codes = torch.randint(0, 256, (128, 390), generator=_seed("move")).to(torch.uint8)
    plan = B.reshard_plan((128, 390), E4M3, (2,), "S^0 R", (3,), "R S^0")
    src = [B._empty_blocked(codes, 64, 390, 1, E8M0, True)[0].data for _ in range(2)]
    for i, t in enumerate(src):
        t.view(torch.uint8).copy_(codes[64 * i:64 * i + 64])
    dst = B.empty_shards(plan, 1, device="cpu")
    B.reshard_debug_execute_host(plan, src, dst)
    for i, t in enumerate(dst):
        assert torch.equal(t.view(torch.uint8), codes[:, 130 * i:130 * i + 130])


@gpu
@pytest.mark.parametrize("cols", [390, 512, 7])
def test_quantized_shards_through_plans(cols, gpu_lib):
    """Each sender's rows to 8 bits, codes and scales through plans, and back on every receiver: the values of the
    whole tensor's 8-bit form, bit for bit."""
    x = (_randn(_seed("through", cols), 6, 64, cols) * 3).to(torch.bfloat16).cuda()
    want = B.reshard_dequantize(B.reshard_quantize(x), x.dtype)
    blocks = -(-cols // 128)
    for scale_dtype in (E8M0, torch.float32):
        sent = [B.reshard_quantize(s, scale_dtype=scale_dtype, dense=True) for s in x.split(3)]
        arrived = []
        for part, width, dtype in ((0, cols, E4M3), (1, blocks, scale_dtype)):
            plan = B.reshard_plan((6, 64, width), dtype, (2,), "S^0 R R", (4,), "R S^0 R")
            arrived.append(B.empty_shards(plan, 1))
            B.reshard_execute(plan, [b[part] for b in sent], arrived[-1])
        for q, s, w in zip(*arrived, want.split(16, 1)):
            assert torch.equal(B.reshard_dequantize(B.Blocked(q, s), x.dtype), w)


def _whole_numbers(g, rows, cols, block_rows, scale_dtype, at_end=False):
    """A Blocked of whole numbers from -8 to 8, all scales 1, and its values: eight neighbouring products span 7 bits
    at most, so that any kernel's sums are exact.  at_end: as the last bytes of an allocation of its own."""
    x = torch.randint(-8, 9, (rows, cols), generator=g).float()
    pitch = -(-cols // 16) * 16
    whole = -(-rows * pitch // (2 << 20)) * (2 << 20) + (20 << 20)  # above what an allocator shares
    store = torch.full((whole,), 0x7F, dtype=torch.uint8, device="cuda")
    end = (rows - 1) * pitch + cols
    data = store[(whole - end) // 16 * 16 if at_end else 0:].as_strided((rows, cols), (pitch, 1))
    data.copy_(x.cuda().to(E4M3).view(torch.uint8))
    scales = torch.ones(-(-rows // block_rows), -(-cols // 128), device="cuda").to(scale_dtype)
    return B.Blocked(data.view(E4M3), scales, block_rows), x.double()


# last tiles of a few rows, where most of a tile's rows lie past the end of the matrix, in both tile sizes
@gpu
@pytest.mark.parametrize("m,n,k", [(9, 1, 256), (65, 129, 512), (130, 257, 1024), (129, 130, 4096), (3080, 4100, 512)])
@pytest.mark.parametrize("scale_dtype", [E8M0, torch.float32], ids=["e8m0", "fp32"])
def test_matmul_at_the_end_of_its_memory(scale_dtype, m, n, k, gpu_lib):
    g = _seed("end", str(scale_dtype), m, n, k)
    a, a64 = _whole_numbers(g, m, k, 1, scale_dtype, at_end=True)
    b, b64 = _whole_numbers(g, n, k, 128, scale_dtype, at_end=True)
    want = (a64.float().cuda() @ b64.float().cuda().t())  # below 2^24: exact
    for dt in HALVES:
        assert torch.equal(B.reshard_matmul(a, b, dt), want.to(dt)), dt


@pytest.mark.parametrize("m,n", [(1 << 40, 1 << 40), (1 << 40, 1 << 39), (1 << 33, 1 << 38), ((1 << 40) - 127, (1 << 38) + 1),
                                 (1 << 27, 129), (129, 1 << 27)])
def test_workspace_of_more_tiles_than_a_product_has(m, n):
    """Refused by the query as by the product, also where the tiles' number leaves 64 bits; to the limit it answers."""
    lib = B.load()
    for scales in (4, 13):
        for out in (2, 3, 4):
            assert lib.reshard_matmul_workspace(m, n, 128, scales, out) == -1
            assert lib.reshard_matmul_workspace(1 << 20, 1 << 14, 1 << 20, scales, out) == 0


def _round_once(v, dtype):
    """Doubles to the nearest of dtype's values, ties to even, from its precision and smallest exponent alone."""
    digits, least = {torch.float16: (11, -14), torch.bfloat16: (8, -126)}[dtype]
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp(min=least).double() - (digits - 1))
    r = torch.round(v / step) * step
    return torch.where(r.abs() > torch.finfo(dtype).max, torch.copysign(torch.tensor(math.inf, dtype=torch.float64), r), r)


@gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
def test_dequantize_rounds_once(dtype, gpu_lib):
    """Products that lie nearer to the midpoint of two 16-bit values than float32 tells, of every code with scales of
    every size: those of the type's subnormals, of float32's, and past the largest value."""
    g = _seed("once", dtype)
    codes = torch.arange(256, dtype=torch.uint8).repeat(4, 1).t().reshape(8, 128)  # four of each code in a row
    digits = 11 if dtype == torch.float16 else 8
    rows = []
    for e in list(range(-149, 121, 3)) + list(range(-40, 20)):
        code = codes.view(E4M3).double()[torch.randint(0, 8, (1,), generator=g), torch.randint(0, 128, (16,), generator=g)]
        code = code[torch.isfinite(code) & (code != 0)].abs()
        middle = 1 + (2 * torch.randint(0, 1 << (digits - 1), code.shape, generator=g) + 1).double() * 2.0 ** -digits
        near = (middle / code * 2.0 ** e).float()  # a scale that takes this code to a midpoint, or as near as float32 comes
        rows += [near, torch.nextafter(near, torch.tensor(math.inf))]
    scales = torch.cat(rows)
    scales = torch.cat([scales, torch.tensor([0.0, -0.0, 1e-45, -1.7, math.inf, -math.inf, math.nan, float.fromhex("0x1.3caaaap-2")])])
    x = codes.repeat_interleave(len(scales), 0)
    s = scales.repeat(8)[:, None]
    got = B.reshard_dequantize(B.Blocked(x.cuda().view(E4M3), s.cuda()), dtype).cpu()
    exact = x.view(E4M3).double() * s.double()
    want = _round_once(exact, dtype)
    want = torch.where(torch.isfinite(exact), want, exact)
    _same(got.double(), want, dtype)
    assert (want != exact.float().to(dtype).double()).nan_to_num().any(), "no product here that two roundings get wrong"
    one = B.Blocked(torch.tensor([[0x03]], dtype=torch.uint8, device="cuda").view(E4M3),
                    torch.tensor([[float.fromhex("0x1.3caaaap-2")]], device="cuda"))
    if dtype == torch.bfloat16:
        assert B.reshard_dequantize(one, dtype).item() == 0.00180816650390625


def test_matrix_of_empty_leading_dimensions():
    for shape in ((4, 0, 130), (0, 4, 130), (4, 3, 0, 5), (2, 0, 0, 7), (0, 0)):
        rows, cols, _ = B._matrix("x", torch.zeros(shape))
        assert rows == 0 and cols == shape[-1]
    assert B._matrix("x", torch.zeros(4, 3, 0))[:2] == (12, 0)
    with pytest.raises(ValueError, match="step evenly"):
        B._matrix("x", torch.zeros(4, 6, 5)[:, ::2][:, :2])


@gpu
@pytest.mark.parametrize("shape", [(4, 0, 130), (0, 3, 130), (2, 0, 0, 256)])
def test_empty_batches(shape, gpu_lib):
    """A batch without rows, as a device has that a dimension's split leaves nothing: empty results, no gradient."""
    x = torch.empty(shape, device="cuda")
    y, mean, rstd = B.reshard_layer_norm(x)
    assert y.shape == x.shape and mean.shape == rstd.shape == x.shape[:-1]
    dx, dw, db = B.reshard_layer_norm_backward(y, x, None, mean, rstd)
    assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all()
    q, t = B.reshard_quantize(x, transposed="both")
    assert q.data.shape == x.shape and t.data.shape == (shape[-1], 0)
    assert B.reshard_dequantize(q, torch.float16).shape == x.shape
    w = B.reshard_quantize(torch.randn(9, shape[-1], device="cuda"), 128)
    assert B.reshard_matmul(q, w).shape == (*shape[:-1], 9)
    assert (B.reshard_matmul(t, t, torch.float32) == 0).all()  # a reduction over no rows


@gpu
@pytest.mark.parametrize("cols", [1, 300, 512])
def test_operators_on_a_single_row(cols, gpu_lib):
    """A tensor of one dimension is one row, and so are its results."""
    x = torch.randn(cols, device="cuda")
    for block_rows in (1, 128):
        q, q2 = B.reshard_quantize(x, block_rows), B.reshard_quantize(x[None], block_rows)
        assert q.data.shape == x.shape and torch.equal(q.data.view(torch.uint8), q2.data[0].view(torch.uint8))
        assert q.scales.shape == ((-(-cols // 128),) if block_rows == 1 else q2.scales.shape)
        back = B.reshard_dequantize(q, torch.float32)
        assert back.shape == x.shape and torch.equal(back, B.reshard_dequantize(q2, torch.float32)[0])
        w = B.reshard_quantize(torch.randn(9, cols, device="cuda"))
        assert torch.equal(B.reshard_matmul(q, w), B.reshard_matmul(q2, w)[0])
        t = B.reshard_quantize(x, block_rows, transposed=True)
        assert t.data.shape == (cols, 1)
    y, mean, rstd = B.reshard_layer_norm(x)
    assert y.shape == x.shape and mean.shape == rstd.shape == ()
    dx, dw, _ = B.reshard_layer_norm_backward(y, x, None, mean, rstd)
    assert dx.shape == dw.shape == x.shape


@gpu
def test_operators_keep_leading_dimensions(gpu_lib):
    x = torch.randn(2, 3, 50, 300, device="cuda")
    flat = x.view(300, 300)
    for block_rows in (1, 128):
        q, want = B.reshard_quantize(x, block_rows), B.reshard_quantize(flat, block_rows)
        assert q.data.shape == x.shape and q.scales.shape == ((2, 3, 50, 3) if block_rows == 1 else (3, 3))
        assert torch.equal(B.reshard_dequantize(q, x.dtype).view(300, 300), B.reshard_dequantize(want, x.dtype))
        assert torch.equal(B.reshard_matmul(q, want).view(300, 300), B.reshard_matmul(want, want))


@gpu
def test_quantize_takes_truth_values_of_any_type(gpu_lib):
    x = torch.randn(5, 300, device="cuda")
    for no, yes in ((0, 1), (np.False_, np.True_)):
        assert B.reshard_quantize(x, transposed=no).data.shape == (5, 300)
        assert B.reshard_quantize(x, transposed=yes).data.shape == (300, 5)


def _check_norm(x, y, mean, rstd, w, b, what):
    """Bounds of test_layer_norm, on the GPU."""
    x64, w64, b64 = x.double(), w.double(), b.double()
    want, m64, r64 = _norm64(x64, w64, b64, 1e-5)
    d = _chain(x.shape[1])
    dm = (d + 2) * F32 * x64.abs().mean(1, keepdim=True)
    spread = (x64 - m64).abs()
    dv = (d + 6) * F32 * (spread ** 2).mean(1, keepdim=True) + 2 * dm * spread.mean(1, keepdim=True) + dm ** 2
    dr = r64 * (0.5 * dv * r64 ** 2 + 4 * F32)
    within = w64.abs() * (spread * dr + dm * r64) * 1.01 + 6 * F32 * ((spread * r64 * w64).abs() + b64.abs())
    for got, ref, bound, name in ((mean[:, None], m64, dm, "mean"), (rstd[:, None], r64, dr + r64 * (dv * r64 ** 2) ** 2, "rstd"),
                                  (y, want, within + HALVES[x.dtype] * (want.abs() + within) + TINY[x.dtype], "y")):
        assert bool(((got.double() - ref).abs() <= bound).all()), f"{what}: {name}"


# more rows than the workgroups that run at once take in one turn, by a few: 64, 256, 512 and 1024 threads a row, rows
# loaded ahead and not (32768 16-bit columns, 16384 of float32)
@gpu
@pytest.mark.parametrize("rows,cols", [(8203, 390), (2055, 2047), (1030, 8200), (520, 16384), (520, 32768), (8195, 1000)])
@pytest.mark.parametrize("dtype", list(HALVES), ids=str)
def test_layer_norm_of_many_rows(dtype, rows, cols, gpu_lib):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.randn(rows, cols, generator=g, device="cuda") + torch.randn(rows, 1, generator=g, device="cuda")).to(dtype)
    w, b = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")), torch.randn(cols, generator=g, device="cuda")
    out, untouched = _guarded((rows, cols), dtype, 3)
    y, mean, rstd = B.reshard_layer_norm(x, w, b, 1e-5, out=out)
    _check_norm(x, y, mean, rstd, w, b, (rows, cols))
    assert untouched()
    # rows are computed apart from each other: the last ones by themselves have the same bits
    tail = B.reshard_layer_norm(x[-9:], w, b, 1e-5)
    assert all(torch.equal(p[-9:], q) for p, q in zip((y, mean, rstd), tail))
    assert torch.equal(B.reshard_layer_norm(x, w, b, 1e-5, out=x)[0], y)  # in place


@gpu
@pytest.mark.parametrize("rows,cols", [(300, 16384), (300, 12000), (600, 2047), (523, 8200), (4100, 4097), (2100, 1000)])
@pytest.mark.parametrize("dtype", list(HALVES), ids=str)
def test_layer_norm_backward_of_many_rows(dtype, rows, cols, gpu_lib):
    """Bounds of test_layer_norm_backward where each group of threads takes several rows in turn."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (torch.randn(rows, cols, generator=g, device="cuda") + 0.5).to(dtype)
    dy = (torch.randn(rows, cols, generator=g, device="cuda") * 0.1).to(dtype)
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    _, mean, rstd = B.reshard_layer_norm(x)
    dx, dw, db = B.reshard_layer_norm_backward(dy, x, w, mean, rstd)
    dy64, rstd64 = dy.double(), rstd.double()[:, None]
    wdx, wdw, wdb, xh = _norm_grad64(dy64, x.double(), w.double(), mean.double()[:, None], rstd64)
    gw = dy64 * w.double()
    size = gw.abs() + gw.abs().mean(1, keepdim=True) + xh.abs() * (gw * xh).abs().mean(1, keepdim=True)
    within = (2 * _chain(cols) + 12) * F32 * rstd64 * size
    assert bool(((dx.double() - wdx).abs() <= within + HALVES[dtype] * (wdx.abs() + within) + TINY[dtype]).all())
    chain = math.ceil(rows / 256) + 32 + 16 + 8  # rows of one group of 256, and as in test_layer_norm_backward
    assert bool(((dw.double() - wdw).abs() <= chain * F32 * (dy64 * xh).abs().sum(0) + 1e-30).all())
    assert bool(((db.double() - wdb).abs() <= chain * F32 * dy64.abs().sum(0) + 1e-30).all())
    assert torch.equal(B.reshard_layer_norm_backward(dy, x, w, mean, rstd, out=dy)[0], dx)  # in place


@gpu
@pytest.mark.parametrize("dtype,rows", [(torch.bfloat16, 16400), (torch.float16, 16400), (torch.float32, 8200)], ids=str)
def test_outputs_larger_than_the_cache(dtype, rows, gpu_lib):
    """From 256 MiB on results are stored past the caches: the same bits as of a few rows at a time, none beside them."""
    cols = 8191
    assert rows * cols * dtype.itemsize >= 256 << 20
    x = torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)).to(dtype)
    w, b = torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda")
    out, untouched = _guarded((rows, cols), dtype, 3)
    y, mean, rstd = B.reshard_layer_norm(x, w, b, out=out)
    assert untouched()
    for lo in range(0, rows, 1000):
        part = B.reshard_layer_norm(x[lo:lo + 1000], w, b)
        assert all(torch.equal(p[lo:lo + 1000], q) for p, q in zip((y, mean, rstd), part))
    for scale_dtype in (E8M0, torch.float32):
        q = B.reshard_quantize(x, scale_dtype=scale_dtype)
        back = B.reshard_dequantize(q, dtype, out=out)
        assert untouched()
        for lo in range(0, rows, 1000):
            some = B.Blocked(q.data[lo:lo + 1000], q.scales[lo:lo + 1000])
            assert torch.equal(back[lo:lo + 1000], B.reshard_dequantize(some, dtype))


@gpu
@pytest.mark.parametrize("cols", [6, 130, 4096, 40000])
def test_layer_norm_beyond_float32(cols, gpu_lib):
    """Squares whose sum leaves float32's range: rstd is 0 and y the bias; elements whose sum does: NaN.  Rows beside
    them are as ever."""
    x = _randn(_seed("beyond", cols), 4, cols).float()
    x[1] = 1e30 * torch.tensor([1.0, -1.0]).repeat(cols // 2)
    x[2] = 3e38
    b = _randn(_seed("bias", cols), cols).float()
    y, mean, rstd = (t.cpu() for t in B.reshard_layer_norm(x.cuda(), None, b.cuda()))
    assert rstd[1] == 0 and torch.equal(y[1], b)
    assert torch.isinf(mean[2]) and rstd[2] == 0 and torch.isnan(y[2]).all()
    alone = B.reshard_layer_norm(x[[0, 3]].cuda(), None, b.cuda())
    assert all(torch.equal(p[[0, 3]], q.cpu()) for p, q in zip((y, mean, rstd), alone))


@gpu
@pytest.mark.parametrize("m,n,k", SIZES + [(65, 130, 2048), (130, 260, 4098), (2047, 300, 5130), (3080, 4100, 390)])
@pytest.mark.parametrize("scale_dtype", [E8M0, torch.float32], ids=["e8m0", "fp32"])
@pytest.mark.parametrize("a_rows,b_rows", [(1, 128), (1, 1), (128, 128)])
def test_matmul_of_whole_numbers(a_rows, b_rows, scale_dtype, m, n, k, gpu_lib):
    """Every product counts, into every type: codes are whole numbers from -8 to 8 and scales 1/4 to 4, so that no bit is
    cut within the 8-bit instruction's eight, and sums of a few hundred thousand sixteenths are exact."""
    g = _seed("whole", a_rows, b_rows, str(scale_dtype), m, n, k)
    for extra in ((-k) % 16, (-k) % 16 + 5):
        sides = []
        for rows, block_rows in ((m, a_rows), (n, b_rows)):
            x = torch.randint(-8, 9, (rows, k), generator=g).float()
            s = torch.exp2(torch.randint(-2, 3, (-(-rows // block_rows), -(-k // 128)), generator=g).float())
            data, _ = _pitched(x.to(E4M3).view(torch.uint8), extra, 0x7F)
            b = B.Blocked(data.view(E4M3), s.cuda().to(scale_dtype), block_rows)
            spread = s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :k]
            sides.append((b, (x * spread).double()))
        (a, a64), (b, b64) = sides
        want = (a64 @ b64.t()).float()
        for dt in HALVES:
            out, untouched = _guarded((m, n), dt)
            assert torch.equal(B.reshard_matmul(a, b, dt, out=out).cpu(), want.to(dt)), (dt, extra)
            assert untouched()
        held = torch.full((m, n), 2.0, dtype=torch.bfloat16, device="cuda")
        B.reshard_matmul(a, b, out=held, accumulate=True)
        assert torch.equal(held.cpu(), (want + 2).to(torch.bfloat16))


@gpu
@pytest.mark.parametrize("m,n", [(5, 90), (70, 90), (3080, 4100)])
@pytest.mark.parametrize("scale_dtype", [E8M0, torch.float32], ids=["e8m0", "fp32"])
@pytest.mark.parametrize("extra", [4, 9])
def test_matmul_nan_into_every_type(extra, scale_dtype, m, n, gpu_lib):
    """A NaN code or scale reaches its row or column alone, whatever the kernel; in a whole and in the short last block."""
    k = 300
    g = _seed("nan", str(scale_dtype), m, n, extra)
    a, _ = _operand(g, m, k, 1, scale_dtype, extra)
    b, _ = _operand(g, n, k, 1, scale_dtype, extra)
    nan = torch.zeros(m, n, dtype=torch.bool)
    a.data.view(torch.uint8)[1, 299] = 0x7F
    a.data.view(torch.uint8)[2, 17] = 0xFF
    b.data.view(torch.uint8)[7, 0] = 0xFF
    held = [t.view(torch.uint8) if scale_dtype == E8M0 else t for t in (a.scales, b.scales)]
    for t, at in ((held[0], (3, 2)), (held[0], (4, 0)), (held[1], (n - 1, 1))):
        t[at] = 255 if scale_dtype == E8M0 else math.nan
    nan[1:5], nan[:, 7], nan[:, n - 1] = True, True, True
    for dt in HALVES:
        assert torch.equal(torch.isnan(B.reshard_matmul(a, b, dt)).cpu(), nan), dt


@gpu
def test_errors_of_other_calls_are_not_an_operators(gpu_lib):
    """An error that a caller's own HIP call left behind is not reported as a launch's, and stays for the caller to read."""
    lib, s = gpu_lib, B._stream_handle(None)
    x, y = torch.randn(200, 256, device="cuda"), torch.empty(200, 256, device="cuda")
    mean, rstd, sums = torch.empty(200, device="cuda"), torch.empty(200, device="cuda"), torch.empty(2, 256, device="cuda")
    need = lib.reshard_layer_norm_backward_workspace(200, 256)
    work = torch.empty(max(need, lib.reshard_matmul_workspace(200, 200, 2048, 13, 3)), dtype=torch.uint8, device="cuda")
    q, big = B.reshard_quantize(x), B.reshard_quantize(torch.randn(200, 2048, device="cuda"))
    odd = B.reshard_quantize(torch.randn(200, 2047, device="cuda"), dense=True)
    z = torch.empty(200, 200, dtype=torch.bfloat16, device="cuda")
    few = torch.empty(200, 8, dtype=torch.bfloat16, device="cuda")

    def product(m, n, b, out):
        k, pitch, (sr, sc) = b.data.shape[1], b.data.stride(0), b.scales.shape
        return lib.reshard_matmul(m, n, k, b.data.data_ptr(), pitch, 1, b.scales.data_ptr(), sc, b.data.data_ptr(), pitch, 1,
                                  b.scales.data_ptr(), sc, 13, out.data_ptr(), n, 3, 0, work.data_ptr(), work.numel(), s)
    calls = {
        "norm": lambda: lib.reshard_layer_norm(200, 256, x.data_ptr(), 256, 4, None, None, 4, 1e-5, y.data_ptr(), 256,
                                               mean.data_ptr(), rstd.data_ptr(), s),
        "norm gradients": lambda: lib.reshard_layer_norm_backward(
            200, 256, x.data_ptr(), 256, x.data_ptr(), 256, 4, None, 4, mean.data_ptr(), rstd.data_ptr(), y.data_ptr(), 256,
            sums[0].data_ptr(), sums[1].data_ptr(), 0, work.data_ptr(), work.numel(), s),
        "quantise": lambda: lib.reshard_quantize(200, 256, x.data_ptr(), 256, 4, 1, 13, q.data.data_ptr(), 256,
                                                 q.scales.data_ptr(), 2, None, 0, None, 0, s),
        "dequantise": lambda: lib.reshard_dequantize(200, 256, q.data.data_ptr(), 256, 1, q.scales.data_ptr(), 2, 13,
                                                     y.data_ptr(), 256, 4, s),
        "product in tiles": lambda: product(200, 200, q, z), "product in parts": lambda: product(200, 200, big, z),
        "product of few rows": lambda: product(8, 200, q, few), "unaligned product": lambda: product(200, 200, odd, z)}
    torch.cuda.synchronize()
    for name, call in calls.items():
        assert lib.hipSetDevice(1000) != 0  # no such device
        status, message = call(), B.reshard_last_error()
        left = lib.hipGetLastError()
        torch.cuda.synchronize()
        assert status == B.RESHARD_OK, (name, message)
        assert left != 0, name
