"""Rows that overlap (an expanded tensor, whose rows are one and the same) reach the kernels with the distance they have: the binding gave it as a row's width, so that the
kernels read, and wrote, behind the tensor's end.  The library refuses such a distance before anything is launched.  No GPU needed: nothing is launched here either."""
import ctypes

import pytest
import torch

from paper_2305_17423_amd import binding as fb

F, BF, U8 = torch.float32, torch.bfloat16, torch.uint8
i32 = dict(dtype=torch.int32)


def refused(name, a):
    """As a shape that does not fit; strides are looked at before the workspace, which is missing here."""
    assert getattr(fb.lib(), name)(ctypes.byref(a), None, 0, None) == -2 and name in fb.fise_last_error()


@pytest.mark.parametrize("rows", [2, 70])
def test_scales_of_codes(rows):
    x, w, ws, y = torch.zeros((rows, 256), dtype=U8), torch.zeros((64, 256), dtype=U8), torch.zeros((1, 2)), torch.zeros((rows, 64))
    for scale in (torch.ones(rows).expand(2, rows), torch.ones(2 * rows - 1).as_strided((2, rows), (rows - 1, 1))):
        a = fb.fp8_linear_args(x, w, ws, y, x_scale=scale)
        assert a.x_scale_stride == scale.stride(0)
        refused("fise_fp8_linear", a)
    assert fb.fp8_linear_args(x, w, ws, y, x_scale=torch.ones((2, rows + 3))[:, :rows]).x_scale_stride == rows + 3


def test_logits():
    ids, w = torch.zeros((6, 2), **i32), torch.zeros((6, 2))
    a = fb.route_args(torch.zeros(4).expand(6, 4), ids, w)
    assert a.stride == 0
    refused("fise_route_experts", a)
    assert fb.route_args(torch.zeros((1, 4)), ids[:1], w[:1]).stride == 4 and fb.route_args(torch.zeros((0, 4)), ids[:0], w[:0]).stride >= 4
    assert fb.route_args(torch.zeros((6, 1)), ids[:, :1].contiguous(), w[:, :1].contiguous()).stride == 1


@pytest.mark.parametrize("side", ["x", "y", "residual"])
def test_rows_of_experts(side):
    ok = dict(x=torch.zeros((6, 32)), ids=torch.zeros((6, 2), **i32), weights=torch.zeros((6, 2)), offsets=torch.zeros(5, **i32), slots=torch.zeros(12, **i32), w_in=torch.zeros((4, 2, 16, 32), dtype=U8),
              w_in_scale=torch.zeros((4, 2, 1, 1)), w_out=torch.zeros((4, 8, 16), dtype=U8), w_out_scale=torch.zeros((4, 1, 1)), y=torch.zeros((6, 8)))
    n = 32 if side == "x" else 8
    for t in (torch.zeros(n).expand(6, n), torch.zeros(256).as_strided((6, n), (n // 2, 1))):
        a = fb.expert_mlp_args(**{**ok, side: t})
        assert getattr(a, side + "_stride") == t.stride(0)
        refused("fise_expert_mlp", a)
    none = {**ok, **{k: ok[k][:0] for k in ("x", "ids", "weights", "slots", "y")}}
    assert fb.expert_mlp_args(**none).x_stride >= 32 and fb.expert_mlp_args(**none).y_stride >= 8


@pytest.mark.parametrize("block_rows", [1, 128])
def test_scales_of_rows_put_in_eight_bits(block_rows, monkeypatch):
    """The call is made with the distance the scales have, and refused."""
    monkeypatch.setattr(fb, "_here", lambda *a: (None, 0))
    x, codes = torch.zeros((300, 256)), torch.zeros((300, 256), dtype=U8)
    n = (2, 300) if block_rows == 1 else (3, 2)
    with pytest.raises(fb.FiseError, match="scales 0"):
        fb.fise_fp8_quantize(x, codes, torch.zeros(n[1]).expand(*n), block_rows=block_rows, stream=0)
