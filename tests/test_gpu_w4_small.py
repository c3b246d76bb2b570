"""GPU check of packing weights whose scale is among the smallest numbers of bf16, where its steps are a large part of it: a weight still comes back within half a scale.

The scale of a group is its largest magnitude / 7 to the next of those steps, 2^-133, or one more where seven and a half scales would not reach the largest: at most that
seventh and a step, half of which a weight may be off (and nothing for the rounding of s q, exact in float)."""
import pytest
import torch

from helpers import DEV
from test_gpu_w4 import fb  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_weights_near_the_end_of_the_range(fb, group, dt):  # noqa: F811
    g = torch.Generator().manual_seed(51)
    N, G = 40 * 16, 3
    K = G * group
    w = 2 * torch.rand((N, G, group), generator=g, dtype=torch.float64) - 1
    w[..., 0] = 1
    tops = 2.0 ** -torch.linspace(120, 149, N * G, dtype=torch.float64).view(N, G, 1)
    w = (w * tops).float().to(dt).view(N, K)
    packed = torch.zeros(fb.fise_w4_bytes(N, K, group), dtype=torch.uint8, device=DEV)
    back = torch.zeros((N, K), device=DEV)
    fb.fise_w4_pack(w.to(DEV), packed, group)
    fb.fise_w4_unpack(packed, back, group)
    w = w.double().view(N, G, group)
    half = (w.abs().amax(-1, keepdim=True) / 7 * (1 + 2.0 ** -8) + 2.0 ** -133) / 2
    off = (back.double().cpu().view(N, G, group) - w).abs()
    assert bool((off <= half).all()), float((off / half).max())
