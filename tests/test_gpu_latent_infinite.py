"""GPU checks of latent attention where a key or a value is not finite: what a query sees of it comes out as the formula says, what it does not see has no effect.

A latent vector that is not finite makes the score of its key infinite or NaN and every channel of its value infinite or NaN: with a score of +inf the softmax is NaN, with one of
-inf the probability 0 meets an infinite value.  So a query that sees it gets NaN in every channel.
A value beyond the range of bf16 (or float) from a latent vector that is finite is infinite in the expanded form, which rounds values: each query that sees it gets that infinity in its
channel, NaN where it sees both signs, and the other channels as ever (tolerances as in the tests of finite values)."""
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


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_values_that_overflow(fb, shape, causal):  # noqa: F811
    B, M, n, H, d, dr, dv, r = shape
    g = torch.Generator().manual_seed(21)
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    x, h, up, down = r - 3, H - 1, dv - 1, 1
    c[..., x], wk[..., x], wv[..., x] = 0, 0, 0
    want = reference(q, c, wk, wv, [n] * B, 0.1, causal)
    wv[h, up, x], wv[h, down, x] = 4, -4
    seen = sees(M, n, causal)
    for first in places(M, n):
        for second in (None, n - 1):                                            # one key with 8e38 in a channel and -8e38 in another, or a later one the other way round besides
            if second == first:
                continue
            bad = c.clone()
            bad[:, first, x] = 2e38
            if second is not None:
                bad[:, second, x] = -2e38
            got = run(fb, q, bad, wk, wv, EXPANDED, 0.1, causal=causal).cpu().view(B, M, H, dv)
            one, other = seen[:, first], seen[:, second] if second is not None else torch.zeros(M, dtype=torch.bool)
            for channel, sign in ((up, 1.0), (down, -1.0)):
                is_ = got[:, :, h, channel].float()
                assert bool(is_[:, one & ~other].eq(sign * math.inf).all()), (first, second, channel)
                assert bool(is_[:, other & ~one].eq(-sign * math.inf).all()) and bool(is_[:, one & other].isnan().all()), (first, second, channel)
                keep = got[:, :, h, channel]
                keep[:, one | other] = want[0].view(B, M, H, dv)[:, one | other][:, :, h, channel].to(keep)
            check(got.reshape(B, M, -1), want)


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
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
