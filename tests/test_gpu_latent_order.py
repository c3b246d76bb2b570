"""GPU checks of latent attention, expanded form, with a workgroup for every tile of queries and several tiles a head: causal and not, lengths that differ, as many tiles as the CUs
hold workgroups and more, heads in eights and not (tolerances as in test_gpu_latent.py)."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_latent import EXPANDED, check, fb, inputs, reference, run  # noqa: F401

pytestmark = pytest.mark.gpu

# B, M, keys, heads, d, dr, dv, r, lengths; tiles: 512 of 4 a head, 640 of 5, 516 of 4 (129 heads), 528 of 11, 320 of 5 with one workgroup a CU
CASES = [(1, 500, 520, 128, 32, 0, 32, 64, [520]), (2, 513, 600, 64, 32, 8, 32, 64, [600, 301]), (3, 385, 400, 43, 32, 0, 32, 64, [400, 390, 129]), (1, 1300, 1300, 48, 64, 32, 64, 128, [1290]),
         (2, 520, 530, 32, 160, 64, 160, 64, [530, 77])]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("B,M,n,H,d,dr,dv,r,lens", CASES)
def test_a_workgroup_for_every_tile(fb, B, M, n, H, d, dr, dv, r, lens, causal):  # noqa: F811
    g = torch.Generator().manual_seed(M + H)
    q, c, wk, wv = inputs(g, B, M, n, H, d, dr, dv, r, poison=lens)
    scale = 1 / math.sqrt(d + dr)
    got = run(fb, q, c, wk, wv, EXPANDED, scale, kv_len=torch.tensor(lens, dtype=torch.int32, device=DEV), causal=causal)
    want = reference(q, c, wk, wv, lens, scale, causal)
    check(got, want)
    assert bool((got.cpu()[(want[0] == 0).all(-1)] == 0).all())
