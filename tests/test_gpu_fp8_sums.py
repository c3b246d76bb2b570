"""GPU checks of the sums of 8-bit products of few rows, and of every form that they have for float results: nothing is lost beside float's roundings, whatever the results' type.

Tolerance: as in the other tests of products, without the 2^-10 that the 8-bit instruction may drop.  Columns whose products cancel are 2^13 times and more as large as the others, which are
all positive: what that instruction drops would be ten times as much as the tolerance."""
import pytest
import torch

from helpers import DEV
from test_gpu_fp8 import E4M3, HALF, T, blocks, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


# rows, outputs, columns, x, y: pieces of sixteen rows, one, two, three and four, with rows missing; more outputs or rows for float results only
CASES = [(M, N, K, x, y) for M in (1, 13, 17, 32, 40, 64) for (N, K) in ((70, 400), (300, 2064)) for x in ("e4m3", "bf16", "f32") for y in ("bf16", "f32")]
CASES += [(20, 8300, 272, "e4m3", "f32"), (50, 8300, 272, "bf16", "f32"), (200, 300, 400, "bf16", "f32"), (300, 257, 272, "e4m3", "f32")]


@pytest.mark.parametrize("M,N,K,xt,yt", CASES)
def test_small_terms_beside_large_ones_that_cancel(fb, M, N, K, xt, yt):
    g = torch.Generator().manual_seed(M * 31 + N + K)
    small = lambda *s: 1 + 0.125 * torch.randint(0, 6, s, generator=g).float()                    # codes, as all values here: 1 to 1.625
    x, w = small(M, K), small(N, K)
    x[:, 0::8] = x[:, 1::8] = 256.0                                            # (rows that the call puts in 8 bits get the scale 1)
    w[:, 0::8], w[:, 1::8] = 128.0, -128.0
    s = torch.rand((blocks(N), blocks(K)), generator=g) + 0.5
    xs = torch.rand((blocks(K), M), generator=g) + 0.5 if xt == "e4m3" else None
    v = x.double() if xs is None else x.double() * xs.double().t().repeat_interleave(128, 1)[:, :K]
    if xs is None:
        x = x.to(T[xt])
    else:
        x = x.to(E4M3)
    u = wide(w.to(E4M3), s)
    want, mag = v @ u.t(), v.abs() @ u.abs().t()
    y = torch.zeros((M, N), dtype=T[yt], device=DEV)
    a = fb.fp8_linear_args(x.to(DEV), w.to(E4M3).to(DEV), s.to(DEV), y, x_scale=None if xs is None else xs.to(DEV))
    fb.fise_fp8_linear(a, torch.zeros(max(fb.fise_fp8_linear_workspace_bytes(a), 256), dtype=torch.uint8, device=DEV))
    err, tol = (y.double().cpu() - want).abs(), HALF[T[yt]] * want.abs() + 2 * (128 + 3 * K / 128 + 4) * 2.0 ** -24 * mag
    assert bool((err <= tol).all()), float((err / tol).max())
