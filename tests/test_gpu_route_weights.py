"""GPU checks of the weights of routing: scores and their sums are numbers of 64 bits, rounded once.

Tolerance, from arithmetic: half a step of float, 2^-24 of the weight, and what exponentials, sums and divisions in 64 bits are off by: less than 2^-52 of the exponent's 50 at most, of
each of 1024 terms' rounding and of three more, 2^-41 of it.  Weights below float's normal numbers do not occur."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_route import T_, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("E,k", [(3, 1), (16, 2), (60, 4), (64, 6), (255, 8), (256, 16), (320, 10), (1024, 64)])
def test_weights(fb, E, k, type, score, renorm):
    for T in (5, 300):
        g = torch.Generator().manual_seed(T * 31 + E)
        l = (torch.randn((T, E), generator=g) * torch.tensor([0.5, 2.0, 5.0])[torch.randint(0, 3, (T, 1), generator=g)]).clamp(-25, 25).to(T_[type])
        l[torch.rand((T, E), generator=g) < 0.1] = -math.inf
        ids, w, _, _ = run(fb, l, None, k, score=score, renormalize=renorm, scale=2.5)
        d = l.double()
        d[d == -math.inf] = -1e5                                                # (score 0; a row without any expert: ids -1)
        s = torch.softmax(d, 1) if score == "softmax" else torch.sigmoid(d)
        want = torch.where(ids >= 0, s.gather(1, ids.long().clamp(min=0)), torch.zeros((), dtype=torch.float64))
        if renorm:
            total = want.sum(1, keepdim=True)
            want = torch.where(total > 0, want / total, torch.zeros((), dtype=torch.float64))
        want = 2.5 * want
        err = (w.double() - want).abs()
        assert bool((err <= (2.0 ** -24 + 2.0 ** -41) * want).all()), float((err / want.clamp(min=1e-30)).max() * 2.0 ** 24)
