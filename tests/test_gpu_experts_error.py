"""GPU check of how far the experts' results are from 64 bits on the whole: no further than the roundings that the definition has, whatever the number of pairs.

Bound, from arithmetic.  A rounding to the nearest is off by a step / sqrt(12) in the root mean square: of the result, and of each pair's result on its way to the sum (eleven bits: half a step is at
most 2^-11 of it, its root mean square 2^-11 / sqrt(3)).  Codes of h are those of 64 bits but where h is next to a border: sums in float leave 2^-21 of h, steps are 2^-4 to 2^-3 of it, so one
code in 2^16 moves, by 2^-3 of its value at most, 2^-11 of the result.  A tenth for chance.  (Gate and up by an instruction that drops what is far below its largest products, 2^-15 of h: one
code in a thousand moves, 2^-9 of the result.)"""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_experts import T_, Experts, call, pick
from test_gpu_fp8 import in_eight

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def squares(x, ids, weight, ex):
    """The definition in 64 bits, and the sum of the squares of all pairs' weighted results."""
    E, K, I, N = ex.dims
    eight = lambda t, n: (lambda q: (q[0] * torch.exp2(q[1]).repeat_interleave(128, 1)[:, :n]).to(DEV))(in_eight(t.cpu(), 1))
    v, y, pairs = eight(x, K), torch.zeros((x.shape[0], N), dtype=torch.float64, device=DEV), 0.0
    for e in range(E):
        t, j = (ids == e).nonzero(as_tuple=True)
        gate, up = (v[t] @ w.t() for w in ex.ins[e])
        p = weight.double().to(DEV)[t, j][:, None] * (eight(gate * torch.sigmoid(gate) * up, I) @ ex.outs[e].t())
        y.index_put_((t,), p, accumulate=True)
        pairs += float((p * p).sum())
    return y.cpu(), pairs


@pytest.mark.parametrize("T,E,K,I,N,k", [(3, 4, 1024, 512, 512, 2), (200, 8, 1024, 512, 512, 2), (600, 4, 1024, 640, 512, 2), (1200, 2, 1024, 512, 512, 1), (1100, 4, 2048, 512, 512, 2)])
@pytest.mark.parametrize("yt", ["bf16", "f32"])
def test_error_on_the_whole(fb, T, E, K, I, N, k, yt):
    g = torch.Generator().manual_seed(T + K)
    ex = Experts(g, E, K, I, N)
    x = (torch.randn((T, K), generator=g) * (1 + 19 * (torch.rand((K,), generator=g) < 0.01))).bfloat16()
    ids, w = pick(g, T, E, k, 0)
    y = call(fb, ex, x, ids, w, None, T_[yt]).double().cpu()
    want, pairs = squares(x, ids, w, ex)
    step = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=1e-30))) - (7 if yt == "bf16" else 23))
    rounding = float((step * step).sum()) / 12 + (2.0 ** -22 / 3 * pairs if yt == "bf16" else 0.0)
    error, bound = float((y - want).norm()), 1.1 * math.sqrt(rounding + 2.0 ** -22 * float((want * want).sum()))
    assert error <= bound, (error / float(want.norm()), bound / float(want.norm()))
