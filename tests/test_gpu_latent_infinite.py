"""GPU checks of latent attention where a key or a value is not finite: what a query sees of it comes out as the formula says, what it does not see has no effect.

A latent vector that is not finite makes the score of its key infinite or NaN and every channel of its value infinite or NaN: with a score of +inf the softmax is NaN, with one of
-inf the probability 0 meets an infinite value.  So a query that sees it gets NaN in every channel."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_latent import ABSORBED, EXPANDED, check, fb, inputs, reference, run  # noqa: F401

pytestmark = pytest.mark.gpu

# B, M, keys, heads, d, dr, dv, r: one part a tile; parts that are cut; a workgroup for every tile; values of a head in three tiles of weights
SHAPES = [(1, 70, 100, 2, 64, 32, 64, 128), (1, 130, 2000, 3, 64, 0, 80, 136), (2, 260, 300, 90, 32, 8, 32, 64), (1, 200, 1500, 4, 128, 64, 160, 256), (1, 3, 700, 5, 40, 32, 40, 128)]


def sees(M, n, causal):
    """[M, n]: whether query m sees key j."""
    return torch.arange(n)[None, :] <= n - M + torch.arange(M)[:, None] if causal else torch.ones((M, n), dtype=torch.bool)


def places(M, n):
    return sorted({0, n // 3, n - M, n - M + M // 2, n - 2, n - 1} & set(range(n)))


@pytest.mark.parametrize("form", [ABSORBED])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_latent_vector_that_is_not_finite(fb, shape, value, causal, form):  # noqa: F811
    B, M, n, H, d, dr, dv, r = shape
    g = torch.Generator().manual_seed(22)
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    x = 2
    q[..., :d] = q[..., :d].abs() + 0.01                                        # (a score of -inf for +inf, of +inf for -inf: W_uk has one sign there)
    wk[..., x] = -0.1
    seen = sees(M, n, causal)
    for at in places(M, n):
        c[:, at, x] = 0
        want = reference(q, c, wk, wv, [n] * B, 0.1, causal, form)
        bad = c.clone()
        bad[:, at, x] = value
        got = run(fb, q, bad, wk, wv, form, 0.1, causal=causal).cpu()
        assert bool(got[:, seen[:, at]].isnan().all()), at
        got[:, seen[:, at]] = want[0][:, seen[:, at]].to(got)
        check(got, want)


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
@pytest.mark.parametrize("value", [math.inf, -math.inf])
def test_a_shared_key_that_is_not_finite(fb, value, form):  # noqa: F811
    """Its score is -inf where the query's channel has the other sign: no part in the softmax, and a value that is finite."""
    B, M, n, H, d, dr, dv, r = 1, 200, 330, 3, 64, 32, 64, 128
    g = torch.Generator().manual_seed(23)
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    x, at = r + 5, 170
    q[..., d + 5] = torch.where(torch.arange(M, device=DEV)[None, :, None] % 2 == 0, -math.copysign(1, value), math.copysign(1, value)).to(q)
    seen = sees(M, n, True)[:, at]
    left_out = (torch.arange(M) % 2 == 0) & seen
    c[:, at, x] = math.copysign(3e38, value)                                    # a score that exp takes to 0, as it does -inf
    want = reference(q, c, wk, wv, [n], 0.1, True, form)
    c[:, at, x] = value
    got = run(fb, q, c, wk, wv, form, 0.1, causal=True).cpu()
    assert bool(got[:, seen & ~left_out].isnan().all())
    got[:, seen & ~left_out] = want[0][:, seen & ~left_out].to(got)
    check(got, want)
