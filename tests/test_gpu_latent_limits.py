"""GPU checks of latent attention at the largest numbers of tokens, heads and rows that it takes (tolerances as in test_gpu_latent.py)."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_latent import ABSORBED, BF, EXPANDED, check, fb, inputs, reference, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
@pytest.mark.parametrize("B,M", [(1, (1 << 20) - 1), ((1 << 20) - 1, 1), (1023, 1025)])
def test_as_many_tokens_as_there_may_be(fb, B, M, form):  # noqa: F811
    """All elements have the same few keys and the queries of a group of 48, so that the reference is one of 48 queries."""
    g = torch.Generator().manual_seed(41)
    n, d, dv, r = 40, 8, 8, 8
    q, c, wk, wv = inputs(g, 1, 48, n, 1, d, 0, dv, r)
    want, spread = reference(q, c, wk, wv, [n], 0.3, False, form)
    turn = torch.arange(B * M, device=DEV) % 48
    got = run(fb, q[0, turn].view(B, M, 1, d), c.expand(B, n, r).contiguous(), wk, wv, form, 0.3)
    turn = turn.cpu()
    check(got.view(1, B * M, dv), (want[:, turn], spread[:, turn]))


@pytest.mark.parametrize("form", [ABSORBED, EXPANDED])
def test_as_many_heads_as_there_may_be(fb, form):  # noqa: F811
    g = torch.Generator().manual_seed(42)
    B, M, n, H, d, dr, dv, r = 1, 3, 70, 65535, 8, 8, 8, 16
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r)
    check(run(fb, q, c, wk, wv, form, 0.25, causal=True), reference(q, c, wk, wv, [n], 0.25, True, form))
