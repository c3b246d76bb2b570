"""GPU checks of routing where different logits have one and the same score in 64 bits: sigmoids of large logits (1), of far negative ones (0), exponentials that underflow next to a row's
largest logit, logits too small to move a score.  Keys are numbers of 64 bits, so such experts are equal and the lower index comes first, with a bias of zeros as without one.

The logits are chosen so that no rounding of a 64-bit exponential decides: scores are 0, 1 or 1 / 2 exactly, or further apart than 2^-30."""
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


def choose(logits, k, score, groups, top_groups):
    """Ids of the k largest 64-bit scores, the lowest index first among equal ones; groups by their largest score."""
    l = logits.double()
    if score == "softmax":
        p = torch.exp(l - l.amax(1, keepdim=True))
        key = p / p.sum(1, keepdim=True)
    else:
        key = 1.0 / (1.0 + torch.exp(-l))
    key = key.masked_fill(l == -math.inf, -math.inf)
    T, E = key.shape
    if groups > 1:
        best = key.view(T, groups, E // groups).amax(-1)
        kept = best.sort(dim=1, descending=True, stable=True).indices[:, :top_groups]
        keep = torch.zeros((T, groups), dtype=torch.bool).scatter_(1, kept, True)
        key = key.masked_fill(~keep.repeat_interleave(E // groups, 1), -math.inf)
    top = key.sort(dim=1, descending=True, stable=True)
    return torch.where(top.values[:, :k] > -math.inf, top.indices[:, :k], -1).to(torch.int32)


def check(fb, logits, k, score="sigmoid", groups=1, top_groups=1):
    want = choose(logits.float(), k, score, groups, top_groups)
    for bias in (None, torch.zeros(logits.shape[1])):
        got = run(fb, logits, bias, k, score=score, groups=groups, top_groups=top_groups)
        assert torch.equal(got[0], want), "a bias of zeros" if bias is not None else "no bias"


def draw(kind, T, E, type, seed):
    """Logits in steps that bf16 holds, many of them equal, and what each kind saturates."""
    g = torch.Generator().manual_seed(seed)
    few = torch.rand((T, E), generator=g) < 0.5
    steps = torch.randint(-12, 13, (T, E), generator=g).float() / 4
    if kind == "large":
        l = torch.where(few, torch.randint(40, 200, (T, E), generator=g).float(), steps)
    elif kind == "far":
        l = -torch.randint(800, 2000, (T, E), generator=g).float()
        l = torch.where(torch.rand((T, E), generator=g) < 0.02, steps, l)
    elif kind == "tiny":
        l = torch.where(few, torch.randint(-5, 6, (T, E), generator=g).float() * 2.0 ** -100, steps)
    else:
        l = torch.where(few, steps, steps * 100)
        l[:, 0] = 1000.0                                                       # what is far below this has score 0
    l[torch.rand((T, E), generator=g) < 0.1] = -math.inf
    return l.to(T_[type])


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_two_experts(fb, score, type):
    """The smallest cases: two scores of 1 (0), three of which two are equal as logits too and a third is lower as a logit only."""
    rows = [[40.0, 50.0, -5.0, 0.0], [49.0, 50.0, 50.0, 3.0], [50.0, 50.0, 49.0, 60.0], [-900.0, -800.0, -1000.0, -800.0], [0.0, 2.0 ** -90, 2.0 ** -80, -1.0], [2.0 ** -80, 2.0 ** -80, 2.0 ** -90, 0.0],
            [math.inf, 60.0, math.inf, 70.0], [3.0e38, 1.0, 2.0e38, -3.0e38], [-3.0e38, -3.0e38, -2.0e38, -1.0e38]]
    l = torch.tensor(rows if score == "sigmoid" else rows[:6] + rows[7:])
    if score == "softmax":
        l = torch.cat((l - 0.0, torch.tensor([[0.0, -900.0, -800.0, -1000.0], [-900.0, 0.0, -800.0, -800.0]])))
    for k in (1, 2, 3, 4):
        check(fb, l.to(T_[type]), k, score)


# experts, places, groups, of them: each width of the kernel, groups of whole lanes, inside a lane and none
SIZES = [(16, 2, 1, 1), (64, 8, 8, 3), (64, 4, 1, 1), (60, 4, 4, 2), (256, 8, 1, 1), (256, 8, 8, 4), (160, 6, 8, 3), (320, 10, 1, 1), (512, 5, 16, 5), (64, 33, 1, 1)]


@pytest.mark.parametrize("E,k,groups,top_groups", SIZES)
@pytest.mark.parametrize("kind,score", [("large", "sigmoid"), ("far", "sigmoid"), ("tiny", "sigmoid"), ("below", "softmax"), ("tiny", "softmax")])
@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_many_experts(fb, type, kind, score, E, k, groups, top_groups):
    for T in (5, 300):
        check(fb, draw(kind, T, E, type, T * 31 + E), k, score, groups, top_groups)
