"""GPU check of 4-bit products whose rows do not fill the matrix unit's tiles: what LDS holds for the rest (NaN, left there by the launch before) is in no result.  Tolerances as in
test_gpu_w4.py."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_w4 import T, check, fb, reference, weights  # noqa: F401

pytestmark = pytest.mark.gpu


# three pieces of 10, 9, 21 and 20 rows (x through LDS), of 5 and 1 (x in registers), 20 and 40 rows of one piece
@pytest.mark.parametrize("M,N,K,group,xt,silu", [(10, 4500, 4200, 256, "f32", False), (9, 4200, 4200, 64, "f32", True), (21, 4097, 1160, 128, "f32", True), (20, 4097, 1160, 32, "f32", False),
                                                 (5, 300, 8328, 64, "f32", True), (1, 1280, 320, 32, "f32", False), (20, 4200, 4104, 256, "bf16", False), (40, 4100, 3200, 32, "bf16", False)])
def test_rows_that_are_left_over(fb, M, N, K, group, xt, silu):  # noqa: F811
    g = torch.Generator().manual_seed(M + N)
    w, packed = weights(fb, g, N, K, group)
    x = (1.5 * torch.randn((M, K), generator=g)).clamp(-8, 8).to(T[xt])
    want, mag, extra = reference(x, w, None, None, silu)
    y = torch.empty((64, N), dtype=T[xt], device=DEV)
    full = fb.w4_linear_args(torch.full((64, K), math.nan, dtype=T[xt], device=DEV), packed, group, y, silu_in=silu)
    few = fb.w4_linear_args(x.to(DEV), packed, group, y[:M], silu_in=silu)
    for _ in range(3):
        y.fill_(0)
        fb.fise_w4_linear(full)
        assert bool(y.isnan().all())
        fb.fise_w4_linear(few)
        check(y[:M], want, mag, extra, K, group)
        assert bool(y[M:].isnan().all())
