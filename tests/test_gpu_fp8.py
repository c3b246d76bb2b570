"""GPU checks of 8-bit floating point with block scales: codes and scales bit by bit against their definition, products against 64-bit sums of the same codes.

Tolerance of a product, from arithmetic: products of two codes are exact in float; a block's 128 products are added by the matrix unit (128 roundings at most), times
the product of two scales (one rounding, one for their product), added to the blocks before (one a block), then bias and residual.  Each is 2^-24 of a partial sum that is at most the sum of the
magnitudes: (128 + 3 K / 128 + 4) 2^-24 of it, twice that for a unit that rounds a partial sum once more; and the output's own rounding, half a step.
For bf16 results the matrix unit adds codes eight at a time and drops what is below 2^-13 of the largest of those products: less than 8 * 2^-13 = 2^-10 of their magnitudes."""
import math

import pytest
import torch

from helpers import DEV

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
T = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def blocks(n):
    return -(-n // 128)


def nearest(v):
    """Doubles up to 448 in magnitude -> the nearest e4m3 value, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def in_eight(x, rows):
    """Values of x [M, K] in 8 bits and the exponents of their scales, from the definition."""
    x = x.double()
    M, K = x.shape
    m, k = -(-M // rows), blocks(K)
    pad = torch.zeros((m * rows, k * 128), dtype=torch.float64)
    pad[:M, :K] = x
    v = pad.view(m, rows, k, 128)
    top = torch.where(torch.isfinite(v), v.abs(), torch.zeros(())).amax((1, 3))
    e = torch.full((m, k), -126.0, dtype=torch.float64)
    for t in range(-125, 121):                                                 # the smallest that leaves none above 448
        e = torch.where(top > 448.0 * 2.0 ** (t - 1), torch.full_like(e, float(t)), e)
    q = torch.where(torch.isfinite(v), nearest(torch.where(torch.isfinite(v), v, torch.zeros(())) / torch.exp2(e)[:, None, :, None]), torch.full((), math.nan, dtype=torch.float64))
    return q.reshape(m * rows, k * 128)[:M, :K], e


def weights(g, N, K, loud=1.0):
    q = torch.randn((N, K), generator=g).mul_(110 * loud).clamp_(-448, 448).to(E4M3)
    s = (torch.rand((blocks(N), blocks(K)), generator=g) + 0.3) * torch.where(torch.rand((blocks(N), blocks(K)), generator=g) < 0.2, -1.0, 1.0) / (110 * math.sqrt(K))
    return q, s


def wide(q, s):
    N, K = q.shape
    return q.double() * s.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]


def check(y, want, mag, K):
    err = (y.double().cpu() - want).abs()
    tol = HALF[y.dtype] * want.abs() + (2 * (128 + 3 * K / 128 + 4) * 2.0 ** -24 + (2.0 ** -10 if y.dtype == torch.bfloat16 else 0.0)) * mag
    assert bool((err <= tol).all()), (float((err / tol).max()), int((err > tol).sum()))


@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_every_code(fb, type):
    """Every bf16 value next to one that sets the scale, and halfway points of all codes: rounded to the nearest, ties to even."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    v = bits.view(torch.bfloat16).float()
    v = v[v.abs() <= 448.0]
    codes = torch.arange(0, 0x7f, dtype=torch.uint8).view(E4M3).float()
    half = (codes[1:] + codes[:-1]) / 2
    if type == "f32":
        v = torch.cat((v, half * (1 + 2.0 ** -20), half * (1 - 2.0 ** -20)))
    v = torch.cat((v, half, -half))
    v = torch.cat((v, torch.zeros(-v.numel() % 127)))
    x = torch.cat((v.view(-1, 127), torch.full((v.numel() // 127, 1), 448.0)), 1).to(T[type])
    c, s = torch.zeros(x.shape, dtype=torch.uint8, device=DEV), torch.zeros((1, x.shape[0]), device=DEV)
    fb.fise_fp8_quantize(x.to(DEV), c, s)
    want, e = in_eight(x, 1)
    assert bool((s.cpu().t() == torch.exp2(e)).all())
    assert torch.equal(c.cpu().view(E4M3).double(), want)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 8), (3, 128), (129, 136), (128, 1280), (300, 1000), (17, 2056)])
def test_quantize(fb, M, K, type, rows):
    """Magnitudes over the whole range of float, zeros, blocks of nothing else, values that are not finite; rows with gaps on both sides."""
    g = torch.Generator().manual_seed(M * 31 + K + rows)
    x = torch.randn((M, K + 8), generator=g) * torch.exp2(torch.randint(-140, 120, (M, 1), generator=g).float())
    x[torch.rand(x.shape, generator=g) < 0.1] = 0
    x[M // 2, :] = 0
    x[torch.rand(x.shape, generator=g) < 0.01] = math.nan
    x[torch.rand(x.shape, generator=g) < 0.01] = -math.inf
    x = x.to(T[type])
    c = torch.full((M, K + 16), 0xA5, dtype=torch.uint8, device=DEV)
    s = torch.zeros((blocks(K), M + 3) if rows == 1 else (blocks(M), blocks(K) + 3), device=DEV)
    fb.fise_fp8_quantize(x.to(DEV)[:, :K], c[:, :K], s[:, :M] if rows == 1 else s[:, :blocks(K)], block_rows=rows)
    want, e = in_eight(x[:, :K], rows)
    got = s.cpu()[:, :M].t() if rows == 1 else s.cpu()[:, :blocks(K)]
    assert torch.equal(got.double(), torch.exp2(e))
    q = c.cpu()[:, :K].contiguous().view(E4M3).double()
    assert torch.equal(torch.isnan(q), torch.isnan(want)) and torch.equal(torch.nan_to_num(q), torch.nan_to_num(want))
    assert bool((c[:, K:] == 0xA5).all()) and not bool(s[:, (M if rows == 1 else blocks(K)):].any())


# M, N, K, x, y, bias, residual: one row, one output, one chunk of 16 columns, parts of tiles and of blocks on every side, each tile size
CASES = [(1, 1280, 320, "f32", "f32", True, False), (1, 1, 16, "bf16", "f32", False, False), (3, 17, 48, "bf16", "bf16", True, True), (16, 130, 144, "f32", "bf16", False, False),
         (17, 1283, 1296, "bf16", "bf16", True, True), (33, 100, 128, "bf16", "f32", True, False), (54, 1283, 5136, "bf16", "bf16", True, True), (64, 640, 2048, "e4m3", "bf16", False, False),
         (65, 257, 272, "e4m3", "f32", True, True), (129, 255, 1280, "bf16", "bf16", True, False), (256, 129, 112, "f32", "f32", False, True), (300, 513, 400, "e4m3", "bf16", True, False),
         (1000, 2000, 528, "bf16", "bf16", True, True), (5, 4000, 4096, "e4m3", "bf16", True, False), (2049, 8200, 272, "bf16", "bf16", True, True), (4100, 4099, 144, "e4m3", "f32", True, False),
         (8, 30, 16384, "bf16", "f32", False, False), (700, 5, 640, "bf16", "bf16", True, False), (4096, 3840, 656, "bf16", "f32", False, True),
         # few rows for many outputs
         (20, 8300, 400, "bf16", "bf16", True, True), (32, 10000, 144, "e4m3", "f32", True, False), (50, 9001, 272, "f32", "bf16", True, False), (64, 8208, 1040, "e4m3", "f32", False, True),
         (40, 8200, 2064, "bf16", "bf16", True, False), (12, 700, 2064, "f32", "f32", True, True), (30, 333, 4112, "e4m3", "bf16", True, False)]


@pytest.mark.parametrize("M,N,K,xt,yt,bias,res", CASES)
def test_linear(fb, M, N, K, xt, yt, bias, res):
    g = torch.Generator().manual_seed(M * 7919 + N * 31 + K)
    q, s = weights(g, N, K)
    w = wide(q, s)
    b = torch.randn((N,), generator=g).to(T[yt]) if bias else None
    r = torch.randn((M, N), generator=g).to(T[yt]) if res else None
    if xt == "e4m3":
        x, xs = weights(g, M, K)[0], (torch.rand((blocks(K), M), generator=g) + 0.5) / 64
        v = x.double() * xs.double().t().repeat_interleave(128, 1)[:, :K]
    else:
        x, xs = (torch.randn((M, K), generator=g) * (1 + 30 * (torch.rand((K,), generator=g) < 0.02))).to(T[xt]), None
        c, e = in_eight(x, 1)
        v = c * torch.exp2(e).repeat_interleave(128, 1)[:, :K]
    dw, dv = w.to(DEV), v.to(DEV)
    want, mag = (dv @ dw.t()).cpu(), (dv.abs() @ dw.abs().t()).cpu()
    for t in (b, r):
        if t is not None:
            want, mag = want + t.double(), mag + t.double().abs()
    y = torch.full((M, N + 3), 5.0, dtype=T[yt], device=DEV)                   # rows that no vector fits
    a = fb.fp8_linear_args(x.to(DEV), q.to(DEV), s.to(DEV), y[:, :N], x_scale=None if xs is None else xs.to(DEV), bias=None if b is None else b.to(DEV), residual=None if r is None else r.to(DEV))
    ws = torch.full((max(fb.fise_fp8_linear_workspace_bytes(a), 1),), 0x7f, dtype=torch.uint8, device=DEV)
    fb.fise_fp8_linear(a, ws)
    check(y[:, :N], want, mag, K)
    assert bool((y[:, N:] == 5.0).all())
    first = y.clone()
    fb.fise_fp8_linear(a, ws)
    assert torch.equal(first, y)                                               # the same sums in the same order


@pytest.mark.parametrize("M", [2, 40, 300])
def test_rows_with_gaps_and_in_place(fb, M):
    """Rows of x, of the weights and of y any (aligned) distance apart, NaN codes in what lies between them, the residual in place; N and K that end inside tiles and blocks."""
    g = torch.Generator().manual_seed(M)
    N, K = 150, 208
    q, s = weights(g, N, K)
    room = torch.full((N, K + 32), 0x7f, dtype=torch.uint8)
    room[:, :K] = q.view(torch.uint8)
    xroom = torch.full((M, K + 48), 0x7f, dtype=torch.uint8)
    x, xs = weights(g, M, K)[0], torch.rand((blocks(K), M + 5), generator=g) / 64
    xroom[:, :K] = x.view(torch.uint8)
    y = torch.randn((M, 160), generator=g).to(torch.bfloat16).to(DEV)
    v, w = x.double() * xs[:, :M].double().t().repeat_interleave(128, 1)[:, :K], wide(q, s)
    old = y[:, :N].double().cpu()
    want, mag = v @ w.t() + old, v.abs() @ w.abs().t() + old.abs()
    a = fb.fp8_linear_args(xroom.to(DEV)[:, :K], room.to(DEV)[:, :K], s.to(DEV), y[:, :N], x_scale=xs.to(DEV)[:, :M], residual=y[:, :N])
    fb.fise_fp8_linear(a)
    check(y[:, :N], want, mag, K)


@pytest.mark.parametrize("M", [3, 50, 140])
def test_values_that_are_not_finite(fb, M):
    """A NaN or an infinity in a row makes that row NaN and no other; a NaN code of the weights its output."""
    g = torch.Generator().manual_seed(9)
    N, K = 140, 272
    q, s = weights(g, N, K)
    x = torch.randn((M, K), generator=g)
    x[1, 5], x[2, 270] = math.inf, math.nan
    c = q.view(torch.uint8).clone()
    c[77, 3] = 0xff
    y = torch.zeros((M, N), device=DEV)
    a = fb.fp8_linear_args(x.to(DEV), c.to(DEV), s.to(DEV), y)
    fb.fise_fp8_linear(a, torch.zeros(fb.fise_fp8_linear_workspace_bytes(a), dtype=torch.uint8, device=DEV))
    bad = torch.zeros((M, N), dtype=torch.bool)
    bad[1:3] = True
    bad[:, 77] = True
    assert torch.equal(torch.isnan(y).cpu(), bad) and bool(torch.isfinite(y.cpu()[~bad]).all())


def test_no_rows(fb):
    g = torch.Generator().manual_seed(1)
    q, s = weights(g, 32, 64)
    y = torch.zeros((0, 32), device=DEV)
    a = fb.fp8_linear_args(torch.zeros((0, 64), device=DEV), q.to(DEV), s.to(DEV), y)
    fb.fise_fp8_linear(a, torch.zeros(256, dtype=torch.uint8, device=DEV))
    fb.fise_fp8_quantize(torch.zeros((0, 64), device=DEV), torch.zeros((0, 64), dtype=torch.uint8, device=DEV), torch.zeros((1, 0), device=DEV))


def test_weights_made_here(fb):
    """Weights into 128 x 128 blocks and the product with them: what a model that has no codes yet does."""
    g = torch.Generator().manual_seed(3)
    M, N, K = 100, 200, 264
    w = torch.randn((N, K), generator=g) / 16
    c, s = torch.zeros((N, 272), dtype=torch.uint8, device=DEV), torch.zeros((2, 3), device=DEV)
    pad = torch.zeros((N, 272))
    pad[:, :K] = w
    fb.fise_fp8_quantize(pad.to(DEV), c, s, block_rows=128)
    x = torch.zeros((M, 272))
    x[:, :K] = torch.randn((M, K), generator=g)
    y = torch.zeros((M, N), device=DEV)
    a = fb.fp8_linear_args(x.to(DEV), c, s, y)
    fb.fise_fp8_linear(a, torch.zeros(fb.fise_fp8_linear_workspace_bytes(a), dtype=torch.uint8, device=DEV))
    (xq, xe), (wq, we) = in_eight(x, 1), in_eight(pad, 128)
    v, u = xq * torch.exp2(xe).repeat_interleave(128, 1)[:, :272], wq * torch.exp2(we).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :272]
    check(y, v @ u.t(), v.abs() @ u.abs().t(), 272)


@pytest.mark.parametrize("M,yt", [(3, "f32"), (3, "bf16"), (40, "bf16"), (140, "f32"), (140, "bf16")])
@pytest.mark.parametrize("low,high", [(0, 8), (0, 128), (1, 2), (0x78, 0x7f)])
def test_codes_of_every_size(fb, M, yt, low, high):
    """The smallest codes, which have no leading one, alone; all codes; the smallest of all; the largest: sums as of the values they stand for."""
    g = torch.Generator().manual_seed(low * 7 + M)
    N, K = 70, 400

    def draw(m):
        c = torch.randint(low, high, (m, K), generator=g)
        c[c == 0x7f] = 0x7e
        return (c + 128 * torch.randint(0, 2, c.shape, generator=g)).to(torch.uint8)
    x, w = draw(M), draw(N)
    xs, ws = torch.rand((blocks(K), M), generator=g) + 0.5, torch.rand((1, blocks(K)), generator=g) + 0.5
    y = torch.zeros((M, N), dtype=T[yt], device=DEV)
    fb.fise_fp8_linear(fb.fp8_linear_args(x.to(DEV), w.to(DEV), ws.to(DEV), y, x_scale=xs.to(DEV)))
    v, u = x.view(E4M3).double() * xs.double().t().repeat_interleave(128, 1)[:, :K], wide(w.view(E4M3), ws)
    check(y, v @ u.t(), v.abs() @ u.abs().t(), K)
