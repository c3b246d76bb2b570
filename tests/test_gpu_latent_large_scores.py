"""GPU checks of latent attention with scores so large that a float of their size is a multiple of hundreds: what is left of a score when the row's largest is taken off is then
beyond what exp2 takes, unless both were rounded alike.  Scores are products of two bf16 numbers, exact in float, and one key's lies far above all others: its value comes
out, rounded once or twice (2 * 2^-8 of it)."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_latent import ABSORBED, BF, EXPANDED, fb, inputs, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 12.6, 2.0 ** 14, 2.0 ** 16.3, 2.0 ** 24, 2.0 ** 40])
@pytest.mark.parametrize("B,M,n,H", [(1, 96, 96, 1), (1, 150, 900, 2), (2, 260, 200, 90)])
def test_one_key_far_above_the_rest(fb, B, M, n, H, size, sign, causal, form):  # noqa: F811
    g = torch.Generator().manual_seed(31)
    d, dr, dv, r = 32, 32, 32, 64
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    q.zero_()
    q[..., d] = (size * (1 + torch.rand((B, M, H), generator=g))).to(BF).to(DEV)
    steps = 1 + torch.arange(128) / 128                                         # all bf16 numbers of a binade: neighbouring scores differ by 2^-8 of themselves at least
    key = steps[torch.randint(0, 100, (B, n), generator=g)]
    best = torch.randint(0, n, (B,), generator=g)
    key[torch.arange(B), best] = steps[127] if sign > 0 else steps[0]
    if sign < 0:
        key = torch.where(key == steps[0], steps[1], key)
        key[torch.arange(B), best] = steps[0]
    c[..., r:] = 0
    c[..., r] = (sign * size * key).to(BF).to(DEV)
    got = run(fb, q, c, wk, wv, form, 1.0, causal=causal).float().cpu().view(B, M, H, dv)
    v = torch.einsum("bjr,hvr->bjhv", c[..., :r].double().cpu(), wv.double().cpu())
    for b in range(B):
        j = int(best[b])
        for m in range(M):
            last = n - M + m if causal else n - 1
            if last < 0:
                assert bool((got[b, m] == 0).all())
            elif j <= last:
                assert bool(((got[b, m] - v[b, j]).abs() <= 2 * 2.0 ** -8 * v[b, j].abs() + 1e-3).all()), (b, m)
            else:
                assert bool(got[b, m].isfinite().all())
