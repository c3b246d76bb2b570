"""GPU checks of the products with 4-bit weights: packing against its definition code by code, products against 64-bit sums of the same codes.

Tolerance of a product, from arithmetic: the codes times x are exact in the matrix unit, so an output is off by its own rounding (half a step: 2^-8 in bf16,
2^-24 in float) and by the roundings of a float sum of K products, K / group scaled sums and a few more terms: at most (K + K / group + 8) * 2^-24
times the sum of the magnitudes, twice that for a unit that rounds a partial sum once more.  SiLU in float is within 2^-19 of its value for |x| <= 20
(the exponential's argument carries |x| log2(e) 2^-24, three more roundings of 2^-22 at most behind it)."""
import math

import numpy as np
import pytest
import torch

from helpers import DEV, host

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def weights(fb, g, N, K, group):
    """Codes of every value, positive and negative scales; packed with its scales given."""
    q = torch.randint(-8, 8, (N, K), generator=g)
    s = ((torch.rand((N, -(-K // group)), generator=g) + 0.25) * torch.where(torch.rand((N, -(-K // group)), generator=g) < 0.2, -1.0, 1.0) / math.sqrt(K)).to(torch.bfloat16)
    wide = s.float().repeat_interleave(group, 1)[:, :K]
    packed = torch.full((fb.fise_w4_bytes(N, K, group),), 0xA5, dtype=torch.uint8, device=DEV)
    fb.fise_w4_pack((q.float() * wide).to(DEV), packed, group, scale=s.to(DEV))
    return q.double() * wide.double(), packed


def reference(x, w, bias, residual, silu):
    x = x.double()
    extra = 0.0
    if silu:
        x = x * torch.sigmoid(x)
        extra = 2.0 ** -19
    y, mag = x @ w.t(), x.abs() @ w.abs().t()
    for t in (bias, residual):
        if t is not None:
            y, mag = y + t.double(), mag + t.double().abs()
    return y, mag, extra


def check(y, want, mag, extra, K, group):
    err = (y.double().cpu() - want).abs()
    tol = HALF[y.dtype] * want.abs() + (2 * (K + K / group + 8) * 2.0 ** -24 + extra) * mag
    assert bool((err <= tol).all()), (float((err / tol).max()), int((err > tol).sum()))


# M, N, K, group, x, y, silu, residual: one row to several slabs (64 rows, 21 of three pieces), one output and odd numbers of them, columns of one
# tile and of part of one, more columns than LDS takes at a time, every width of a group, chunks whose tiles the waves share unevenly
CASES = [(1, 1280, 320, 32, "f32", "f32", False, False), (2, 513, 1280, 64, "f32", "f32", True, False), (3, 1, 8, 32, "bf16", "bf16", False, False),
         (1, 17, 120, 64, "bf16", "f32", False, True), (16, 100, 136, 128, "bf16", "bf16", False, False), (17, 1283, 640, 256, "bf16", "bf16", False, True),
         (27, 129, 5120, 128, "bf16", "bf16", False, True), (64, 96, 1288, 32, "bf16", "bf16", False, False), (65, 33, 256, 64, "bf16", "f32", False, True),
         (130, 64, 520, 256, "bf16", "bf16", True, False), (5, 50, 384, 32, "f32", "bf16", True, True), (21, 40, 128, 128, "f32", "f32", False, False),
         (22, 40, 264, 64, "f32", "f32", True, False), (16, 9000, 8192, 128, "bf16", "bf16", False, False), (64, 17000, 512, 64, "bf16", "bf16", False, False),
         (48, 300, 8200, 256, "bf16", "bf16", False, False), (1, 20160, 1280, 32, "f32", "f32", True, False), (11, 31, 4104, 32, "f32", "f32", False, False),
         # more than 16 rows and many columns and outputs: x through LDS, one to four waves an output, 33 to 64 rows, pieces
         (64, 8200, 2200, 64, "bf16", "bf16", False, True), (40, 4100, 3200, 32, "bf16", "bf16", False, False), (20, 4200, 4104, 256, "bf16", "f32", False, False),
         (21, 4097, 1160, 128, "f32", "f32", True, False), (70, 2100, 1032, 64, "f32", "bf16", False, True), (25, 30000, 2056, 128, "bf16", "bf16", True, False),
         # x of two tiles of rows or of columns, or both, in a wave's registers
         (1, 40, 2200, 64, "bf16", "bf16", False, False), (7, 700, 3000, 32, "f32", "f32", True, False), (30, 2100, 640, 64, "bf16", "bf16", False, True),
         (20, 2304, 2200, 128, "bf16", "f32", False, False), (10, 4500, 1160, 256, "f32", "f32", False, False),
         # and in several rounds, x's parts behind the sums of several tiles of outputs
         (5, 300, 8328, 64, "f32", "f32", True, False), (2, 4200, 8328, 128, "f32", "f32", False, True), (9, 4200, 4200, 64, "f32", "bf16", True, False)]


@pytest.mark.parametrize("M,N,K,group,xt,yt,silu,res", CASES)
def test_linear(fb, M, N, K, group, xt, yt, silu, res):
    g = torch.Generator().manual_seed(M * 7919 + N * 31 + K)
    w, packed = weights(fb, g, N, K, group)
    x = (1.5 * torch.randn((M, K), generator=g)).clamp(-8, 8).to(T[xt])
    bias = torch.randn((N,), generator=g).to(T[yt])
    residual = torch.randn((M, N), generator=g).to(T[yt]) if res else None
    want, mag, extra = reference(x, w, bias, residual, silu)
    y = torch.full((M, N), float("nan"), dtype=T[yt], device=DEV)
    a = fb.w4_linear_args(x.to(DEV), packed, group, y, bias=bias.to(DEV), residual=None if residual is None else residual.to(DEV), silu_in=silu)
    fb.fise_w4_linear(a)
    check(y, want, mag, extra, K, group)
    first = y.clone()
    fb.fise_w4_linear(a)
    assert torch.equal(first, y)                                                # the same sums in the same order


@pytest.mark.parametrize("M,N,K,group", [(4, 37, 248, 32), (33, 50, 640, 128)])
def test_strides_bias_types_and_sum_in_place(fb, M, N, K, group):
    g = torch.Generator().manual_seed(5)
    w, packed = weights(fb, g, N, K, group)
    x = torch.randn((M, K + 24), generator=g).to(torch.bfloat16)
    y = torch.randn((M, N + 5), generator=g).to(torch.bfloat16).to(DEV)
    before = y.clone()
    bias = torch.randn((N,), generator=g)
    want, mag, extra = reference(x[:, 8:8 + K], w, bias, before[:, 1:1 + N].cpu(), False)
    a = fb.w4_linear_args(x.to(DEV)[:, 8:8 + K], packed, group, y[:, 1:1 + N], bias=bias.to(DEV), residual=y[:, 1:1 + N])
    fb.fise_w4_linear(a)
    check(y[:, 1:1 + N], want, mag, extra, K, group)
    assert torch.equal(y[:, :1], before[:, :1]) and torch.equal(y[:, 1 + N:], before[:, 1 + N:])


def test_values_that_are_not_finite_stay_in_their_row(fb):
    g = torch.Generator().manual_seed(6)
    N, K, group = 64, 256, 64
    w, packed = weights(fb, g, N, K, group)
    for xt in (torch.bfloat16, torch.float32):
        x = torch.randn((5, K), generator=g).to(xt)
        x[1, 7], x[3, 100], x[4, 0] = math.inf, math.nan, torch.finfo(xt).max
        y = torch.zeros((5, N), device=DEV)
        fb.fise_w4_linear(fb.w4_linear_args(x.to(DEV), packed, group, y))
        got, sign = y.cpu(), torch.sign(w[:, 7])
        assert torch.equal(got[1][sign > 0], torch.full_like(got[1][sign > 0], math.inf)) and torch.equal(got[1][sign < 0], torch.full_like(got[1][sign < 0], -math.inf))
        assert bool(got[1][sign == 0].isnan().all()) and bool(got[3].isnan().all())
        rows = [0, 2, 4]
        want, mag, extra = reference(x[rows], w, None, None, False)
        assert bool(got[rows].isfinite().all())
        check(got[rows], want, mag, extra, K, group)


@pytest.mark.parametrize("N,K,group", [(1, 1, 32), (17, 200, 32), (40, 1280, 64), (33, 640, 128), (16, 300, 256), (32800, 24, 32)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_pack_chooses_scales_and_nearest_codes(fb, N, K, group, dt):
    g = torch.Generator().manual_seed(N + K)
    w = torch.randn((N, K), generator=g).to(T[dt])
    w[0, :] = 0 if N > 1 else w[0, :]
    packed = torch.full((fb.fise_w4_bytes(N, K, group),), 0xFF, dtype=torch.uint8, device=DEV)
    fb.fise_w4_pack(w.to(DEV), packed, group)
    back = torch.full((N, K), float("nan"), device=DEV)
    fb.fise_w4_unpack(packed, back, group)
    back = back.cpu()
    G = -(-K // group)
    pad = torch.nn.functional.pad(w.float(), (0, G * group - K)).view(N, G, group)
    s = (pad.abs().amax(-1) / 7).to(torch.bfloat16).float()
    q = torch.where(s[..., None] != 0, torch.round(pad / s[..., None]), torch.zeros(())).clamp(-7, 7)
    assert torch.equal(back, (q * s[..., None]).view(N, -1)[:, :K])             # a quotient and its rounding are the same operations here and there
    half = s[..., None].expand(-1, -1, group).reshape(N, -1)[:, :K] / 2
    assert bool(((back - w.float()).abs() <= half * (1 + 2.0 ** -20)).all())
    bf = torch.full((N, K), float("nan"), dtype=torch.bfloat16, device=DEV)
    fb.fise_w4_unpack(packed, bf, group)
    assert torch.equal(bf.cpu(), back.to(torch.bfloat16))


def test_pack_of_values_that_are_not_finite(fb):
    w = torch.randn((4, 128), generator=torch.Generator().manual_seed(1))
    w[1, 40], w[2, 70] = math.inf, math.nan
    packed = torch.zeros((fb.fise_w4_bytes(4, 128, 32),), dtype=torch.uint8, device=DEV)
    fb.fise_w4_pack(w.to(DEV), packed, 32)
    back = torch.zeros((4, 128), device=DEV)
    fb.fise_w4_unpack(packed, back, 32)
    bad = back.cpu().isnan()
    want = torch.zeros((4, 128), dtype=torch.bool)
    want[1, 32:64] = want[2, 64:96] = True
    assert torch.equal(bad, want)


def test_captured_and_replayed_on_two_streams(fb):
    g = torch.Generator().manual_seed(9)
    N, K, group = 640, 1280, 64
    w, packed = weights(fb, g, N, K, group)
    xs = [torch.randn((m, K), generator=g).to(torch.bfloat16).to(DEV) for m in (2, 30)]
    ys = [torch.zeros((x.shape[0], N), dtype=torch.bfloat16, device=DEV) for x in xs]
    args = [fb.w4_linear_args(x, packed, group, y) for x, y in zip(xs, ys)]
    want = []
    for a, y in zip(args, ys):
        fb.fise_w4_linear(a)
        want.append(y.clone())
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for a, st in zip(args, streams):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            fb.fise_w4_linear(a, stream=st)
        graphs.append(gr)
    for rep in range(4):
        for y in ys:
            y.fill_(float("nan"))
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for y, v in zip(ys, want):
            assert torch.equal(y, v), rep
