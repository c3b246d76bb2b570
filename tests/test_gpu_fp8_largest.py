"""GPU checks of blocks whose largest value is float's largest, or next to where its scale changes: the scale's exponent goes up to 120, past that of the values that other tests draw.
Codes and scales bit by bit; a product of such rows, whose tolerance is that of the other tests of products."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_fp8 import E4M3, T, blocks, check, in_eight, weights, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def tops(type):
    """Largest values of a block: the type's, 1.75 of powers of two (448 of a scale) and the values beside them, the smallest normal and subnormal numbers."""
    big = torch.finfo(T[type]).max
    edge = torch.tensor([1.75 * 2.0 ** e for e in (127, 126, 0, -118, -119, -126)] + [1.5 * 2.0 ** 127, 2.0 ** -126, 2.0 ** -127, 2.0 ** -133]).to(T[type])
    up = torch.tensor(math.inf, dtype=T[type])
    return torch.cat((torch.tensor([big], dtype=T[type]), edge, torch.nextafter(edge, up), torch.nextafter(edge, torch.zeros_like(up))))


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_codes_and_scales(fb, type, rows):
    g = torch.Generator().manual_seed(rows)
    top = tops(type)
    K, M = 264, top.numel() * rows
    x = (torch.rand((M, K), generator=g) * 2 - 1).mul_(0.999) * top.float().repeat_interleave(rows)[:, None]
    x = x.to(T[type])
    x[torch.arange(0, M, rows), :] *= 0.5
    x[torch.arange(0, M, rows), 7], x[torch.arange(0, M, rows), 200], x[torch.arange(0, M, rows), 263] = top, -top, top
    c, s = torch.zeros((M, K), dtype=torch.uint8, device=DEV), torch.zeros((blocks(K), M) if rows == 1 else (blocks(M), blocks(K)), device=DEV)
    fb.fise_fp8_quantize(x.to(DEV), c, s, block_rows=rows)
    want, e = in_eight(x, rows)
    assert float(e.max()) == 120 and float(e.min()) == -126
    assert torch.equal((s.t() if rows == 1 else s).cpu().double(), torch.exp2(e))
    assert torch.equal(c.cpu().view(E4M3).double(), want)


@pytest.mark.parametrize("M", [1, 20, 70])
@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_product(fb, type, M):
    """Weights' scales of 2^-100 bring the results back: scales 2^120 and 2^-100 of a block have an ordinary product."""
    g = torch.Generator().manual_seed(M)
    N, K = 40, 272
    q, s = weights(g, N, K)
    s = s * 2.0 ** -100
    x = ((torch.rand((M, K), generator=g) * 2 - 1) * torch.finfo(T[type]).max).to(T[type])
    x[:, 3] = x[:, 140] = x[:, 271] = torch.finfo(T[type]).max
    c, e = in_eight(x, 1)
    assert float(e.min()) == 120
    v, w = c * torch.exp2(e).repeat_interleave(128, 1)[:, :K], wide(q, s)
    y = torch.zeros((M, N), device=DEV)
    a = fb.fp8_linear_args(x.to(DEV), q.to(DEV), s.to(DEV), y)
    fb.fise_fp8_linear(a, torch.zeros(max(fb.fise_fp8_linear_workspace_bytes(a), 256), dtype=torch.uint8, device=DEV))
    check(y, v @ w.t(), v.abs() @ w.abs().t(), K)
