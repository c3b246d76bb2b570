"""What the entry points for rotary positions, 8-bit products, routing and experts refuse, on the host, before anything is launched; and what their binding refuses.  No GPU needed."""
import ctypes

import pytest
import torch

from paper_2305_17423_amd import binding as fb

A = 0x10000          # never dereferenced: validation ends first


def set_all(s, **kw):
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def call(name, base, change, *rest):
    return getattr(fb.lib(), name)(ctypes.byref(set_all(base(), **change)), *rest)


def refused(name, base, change, code, *rest):
    assert call(name, base, change, *rest) == code
    if code:
        assert name in fb.fise_last_error()


def rotary(**kw):
    a = fb.fise_rotary_args()
    a.n_tensors, a.dtype, a.B, a.M, a.n_axes, a.T, a.H, a.W, a.tile_idx, a.n_active, a.tile = 1, 1, 2, 0, 2, 1, 8, 8, A, 0, 4
    for j in range(2):
        a.axis_dim[j], a.theta[j] = 16, 100.0
    set_all(a.t[0], x=A, y=2 * A, heads=2, d=40, start=8, x_batch=5120, x_row=80, x_head=40, y_batch=5120, y_row=80, y_head=40, **kw)
    return a


@pytest.mark.parametrize("change,code", [({}, 0), ({"n_tensors": 0}, -2), ({"n_tensors": 3}, -2), ({"n_tensors": 2}, -1), ({"dtype": 2}, -3), ({"n_axes": 0}, -2), ({"n_axes": 5}, -2),
                                         ({"pairing": 3}, -2), ({"pairing": -1}, -2), ({"B": 0}, -2), ({"M": -1}, -2), ({"M": 5}, -2), ({"T": 0}, -2), ({"H": 6}, -2), ({"tile": 3}, -2), ({"tile": -4}, -2),
                                         ({"n_active": 5, "M": 80}, -5), ({"n_active": -1}, -5), ({"n_active": 1}, -2), ({"n_active": 1, "M": 16, "tile_idx": None}, -1),
                                         ({"pos": A, "pos_B": 3}, -2), ({"pos": A + 2, "pos_B": 1}, -4), ({"T": 1 << 20, "H": 1 << 10, "W": 1 << 10}, -2), ({"T": 1 << 30, "H": 1 << 30, "W": 1 << 30}, -2)])
def test_rotary(change, code):
    refused("fise_rotary", rotary, change, code, None)


@pytest.mark.parametrize("change,code", [({"x": None}, -1), ({"y": None}, -1), ({"heads": 0}, -2), ({"d": 39}, -2), ({"start": -1}, -2), ({"start": 9}, -2), ({"x_row": -80}, -2), ({"y_head": -1}, -2),
                                         ({"x": A + 1}, -4), ({"y": A}, 0), ({"y": A, "y_row": 88}, -2), ({"y": A, "y_is_map": 1}, -2), ({"x_row": 1 << 40}, 0)])
def test_rotary_tensor(change, code):
    a = rotary()
    set_all(a.t[0], **change)
    assert fb.lib().fise_rotary(ctypes.byref(a), None) == code


@pytest.mark.parametrize("axis", [0, 1, 15, 1026, -2])
@pytest.mark.parametrize("field", ["axis_dim", "theta"])
def test_rotary_axes(axis, field):
    a = rotary()
    if field == "axis_dim":
        a.axis_dim[1] = axis
    else:
        a.theta[1] = {0: 0.0, 1: -1.0, 15: float("nan"), 1026: float("inf"), -2: -2.0}[axis]
    assert fb.lib().fise_rotary(ctypes.byref(a), None) == -2
    assert fb.lib().fise_rotary(None, None) == -1
    a = rotary()
    a.tile, a.pos, a.pos_B, a.n_axes = 0, A, 1, 4                              # four axes have positions of their own only
    a.axis_dim[0] = a.axis_dim[1] = a.axis_dim[2] = a.axis_dim[3] = 8
    a.theta[2] = a.theta[3] = 1.0
    assert fb.lib().fise_rotary(ctypes.byref(a), None) == 0
    a.pos, a.M = None, 64
    assert fb.lib().fise_rotary(ctypes.byref(a), None) == -2


def test_fp8_quantize():
    f = fb.lib().fise_fp8_quantize
    ok = [A, 1, 128, 0, 128, 1, A, 128, A, 0, None]
    assert f(*ok) == 0
    for i, v, code in ((0, None, -1), (6, None, -1), (8, None, -1), (1, 2, -3), (3, -1, -2), (4, 0, -2), (4, 1 << 21, -2), (5, 64, -2), (2, 120, -2), (7, 120, -2), (4, 124, -4), (2, 132, -4), (7, 132, -4),
                       (0, A + 8, -4), (6, A + 4, -4), (8, A + 2, -4)):
        assert f(*(ok[:i] + [v] + ok[i + 1:])) == code, (i, v)
    assert f(A, 1, 128, 4, 128, 1, A, 128, A, 3, None) == -2                   # scales of four rows, three apart
    assert f(A, 1, 256, 4, 256, 128, A, 256, A, 1, None) == -2


def fp8():
    return set_all(fb.fise_fp8_linear_args(), x=A, x_dtype=1, x_stride=256, w=A, w_stride=256, w_scale=A, M=0, N=64, K=256, y=A, y_dtype=1, y_stride=64)


CODES = {"x_dtype": 2, "x_scale": A, "x_scale_stride": 0}


@pytest.mark.parametrize("change,code", [({}, 0), (CODES, 0), ({"x": None}, -1), ({"w": None}, -1), ({"w_scale": None}, -1), ({"y": None}, -1), ({"x_dtype": 3}, -3), ({"y_dtype": 2}, -3),
                                         ({"bias": A, "bias_dtype": 2}, -3), ({"x_dtype": 2}, -1), ({"x_scale": A}, -1), ({"M": -1}, -2), ({"N": 0}, -2), ({"K": 0}, -2), ({"N": 1 << 21, "y_stride": 1 << 21}, -2),
                                         ({"x_stride": 240}, -2), ({"w_stride": 240}, -2), ({"y_stride": 63}, -2), ({"residual": A, "residual_stride": 63}, -2), ({"w_stride": (1 << 22) + 16}, -2),
                                         ({"x_stride": (1 << 22) + 16}, -2), ({**CODES, "M": 4, "x_scale_stride": 3}, -2), ({"K": 248}, -4), ({"x_stride": 260}, -4), ({**CODES, "x_stride": 264}, -4),
                                         ({"x_stride": 264}, 0), ({"w_stride": 264}, -4), ({"x": A + 8}, -4), ({"w": A + 8}, -4), ({"y": A + 1}, -4), ({"bias": A + 2, "bias_dtype": 0}, -4),
                                         ({"w_scale": A + 2}, -4), ({"M": 65}, -5), ({**CODES, "M": 1 << 20, "N": 1 << 20, "y_stride": 1 << 20, "x_scale_stride": 1 << 20}, -2)])
def test_fp8_linear(change, code):
    refused("fise_fp8_linear", fp8, change, code, None, 0, None)


def test_fp8_linear_workspace():
    L, a = fb.lib(), set_all(fp8(), M=65)
    need = L.fise_fp8_linear_workspace_bytes(ctypes.byref(a))
    assert need == 65 * 256 + 768 and L.fise_fp8_linear_workspace_bytes(ctypes.byref(set_all(fp8(), M=3))) == 0      # (few rows are put in 8 bits in registers)
    assert L.fise_fp8_linear(ctypes.byref(a), A, need - 1, None) == -5 and L.fise_fp8_linear(ctypes.byref(a), A + 64, need, None) == -4
    assert L.fise_fp8_linear_workspace_bytes(ctypes.byref(set_all(fp8(), M=65, **CODES))) == 0 and L.fise_fp8_linear_workspace_bytes(None) == 0
    assert L.fise_fp8_linear_workspace_bytes(ctypes.byref(set_all(fp8(), N=0))) == 0 and L.fise_fp8_linear(None, None, 0, None) == -1


def route():
    return set_all(fb.fise_route_args(), logits=A, dtype=0, stride=64, T=0, E=64, k=4, groups=1, top_groups=1, group_top=1, ids=A, weights=A, offsets=A, slots=A, scale=1.0)


@pytest.mark.parametrize("change,code", [({}, 0), ({"logits": None}, -1), ({"ids": None}, -1), ({"weights": None}, -1), ({"offsets": None}, -1), ({"slots": None}, -1), ({"offsets": None, "slots": None}, 0),
                                         ({"dtype": 2}, -3), ({"E": 0}, -2), ({"E": 1025, "stride": 2000}, -2), ({"k": 0}, -2), ({"k": 65}, -2), ({"E": 3}, -2), ({"T": -1}, -2), ({"T": 1 << 30}, -2), ({"stride": 63}, -2),
                                         ({"score": 2}, -2), ({"score": -1}, -2), ({"groups": 0}, -2), ({"groups": 5}, -2), ({"groups": 4, "top_groups": 5}, -2), ({"groups": 4, "top_groups": 0}, -2),
                                         ({"groups": 4, "group_top": 3}, -2), ({"groups": 4, "group_top": 0}, -2), ({"groups": 4, "top_groups": 2, "group_top": 2}, 0), ({"logits": A + 2}, -4), ({"logits": A + 2, "dtype": 1}, 0),
                                         ({"ids": A + 1}, -4), ({"bias": A + 2}, -4), ({"T": 1000}, -5), ({"T": 1 << 30, "k": 1}, -2)])
def test_route(change, code):
    refused("fise_route_experts", route, change, code, None, 0, None)


def test_route_workspace():
    L = fb.lib()
    size = lambda **kw: L.fise_route_experts_workspace_bytes(ctypes.byref(set_all(route(), **kw)))
    assert size(T=0) == 0 and size(T=256) == 0 and size(T=257) > 257 * 16 and size(T=257, offsets=None, slots=None) == 0 and size(E=0) == 0 and L.fise_route_experts_workspace_bytes(None) == 0
    a = set_all(route(), T=1000)
    assert L.fise_route_experts(ctypes.byref(a), A, size(T=1000) - 1, None) == -5 and L.fise_route_experts(ctypes.byref(a), A + 128, size(T=1000), None) == -4
    assert L.fise_route_experts(None, None, 0, None) == -1


def experts():
    return set_all(fb.fise_expert_mlp_args(), x=A, x_dtype=1, x_stride=256, T=0, K=256, ids=A, weights=A, offsets=A, slots=A, k=2, E=4, I=64, N=128, w_in=A, w_in_scale=A, w_out=A, w_out_scale=A,
                   y=A, y_dtype=1, y_stride=128)


@pytest.mark.parametrize("change,code", [({}, 0)] + [({n: None}, -1) for n in ("x", "ids", "weights", "offsets", "slots", "w_in", "w_in_scale", "w_out", "w_out_scale", "y")] +
                         [({"x_dtype": 2}, -3), ({"y_dtype": 2}, -3), ({"T": -1}, -2), ({"K": 0}, -2), ({"I": 0}, -2), ({"N": 0}, -2), ({"E": 0}, -2), ({"E": 1025}, -2), ({"k": 0}, -2), ({"k": 65}, -2),
                          ({"K": 65552, "x_stride": 65552}, -2), ({"I": 65552}, -2), ({"N": 65544, "y_stride": 65544}, -2), ({"T": 1 << 23}, -2), ({"T": 1 << 22, "k": 1}, -2), ({"K": 248}, -4), ({"I": 72}, -4),
                          ({"N": 124}, -4), ({"x_stride": 248}, -2), ({"y_stride": 120}, -2), ({"residual": A, "residual_stride": 120}, -2), ({"x_stride": 260}, -4), ({"y_stride": 132}, -4),
                          ({"residual": A, "residual_stride": 132}, -4), ({"x": A + 8}, -4), ({"y": A + 8}, -4), ({"w_in": A + 8}, -4), ({"w_out": A + 4}, -4), ({"ids": A + 2}, -4), ({"w_in_scale": A + 2}, -4), ({"T": 1}, -5), ({"T": 1 << 21, "N": 1 << 13, "y_stride": 1 << 13}, -5)])
def test_expert_mlp(change, code):
    refused("fise_expert_mlp", experts, change, code, None, 0, None)


def test_expert_mlp_workspace():
    L, a = fb.lib(), set_all(experts(), T=30)
    need = L.fise_expert_mlp_workspace_bytes(ctypes.byref(a))
    assert need > 30 * 256 + 60 * 128 + 60 * 128 * 2 and L.fise_expert_mlp_workspace_bytes(ctypes.byref(set_all(experts(), T=3))) == 6 * 64 * 4
    a.T = 30
    assert L.fise_expert_mlp(ctypes.byref(a), A, need - 1, None) == -5 and L.fise_expert_mlp(ctypes.byref(a), A + 16, need, None) == -4
    assert L.fise_expert_mlp_workspace_bytes(ctypes.byref(set_all(experts(), K=8))) == 0 and L.fise_expert_mlp_workspace_bytes(None) == 0 and L.fise_expert_mlp(None, None, 0, None) == -1


# --------------------------------------------------------------------------- the binding
F, BF, U8 = torch.float32, torch.bfloat16, torch.uint8


def test_rotary_binding():
    x = torch.zeros((2, 16, 3, 32))
    grid = dict(axes=[16, 16], theta=10.0, grid=(1, 4, 4))
    a = fb.rotary_args([fb.rotary_tensor(x, x[:, :, :1].expand(2, 16, 3, 32).clone())], **grid)
    assert (a.M, a.t[0].x_row, a.t[0].x_head) == (16, 96, 32)
    m = torch.zeros((2, 16, 1, 40))[..., 8:]
    b = fb.rotary_args([fb.rotary_tensor(torch.zeros((2, 1, 1, 32)), m, y_is_map=True)], tile_idx=torch.zeros(1, dtype=torch.int32), n_active=1, tile=1, **grid)
    assert (b.M, b.t[0].y_row, b.t[0].y_batch, b.t[0].x_row) == (1, 40, 640, 0)
    for bad in (dict(tensors=[]), dict(axes=[]), dict(theta=[1.0]), dict(offset=[1.0]), dict(grid=(1, 4, 8)), dict(pos=torch.zeros((2, 16, 3))), dict(pos=torch.zeros((2, 16, 2), dtype=torch.int64)),
                dict(pos=torch.zeros((2, 2, 16)).transpose(1, 2)), dict(tile=2, n_active=4, tile_idx=torch.zeros(3, dtype=torch.int32)), dict(tile=2, n_active=4, tile_idx=torch.zeros(8, dtype=torch.int32)[::2]),
                dict(tensors=[fb.rotary_tensor(x, x[:, :8])]), dict(tensors=[fb.rotary_tensor(x, x.bfloat16())]), dict(tensors=[fb.rotary_tensor(x, x.transpose(1, 3))]),
                dict(tensors=[fb.rotary_tensor(x, x[:, :, :1].expand(2, 16, 3, 32))]), dict(tensors=[fb.rotary_tensor(x), fb.rotary_tensor(x.bfloat16())]),
                dict(tensors=[fb.rotary_tensor(torch.zeros((2, 16, 3, 64))[..., ::2])])):
        with pytest.raises(ValueError):
            fb.rotary_args(**{"tensors": [fb.rotary_tensor(x)], **grid, **bad})


def test_fp8_binding():
    x, w, s, y = torch.zeros((3, 256)), torch.zeros((130, 256), dtype=U8), torch.zeros((2, 2)), torch.zeros((3, 130))
    assert fb.fp8_linear_args(x, w, s, y).x_stride == 256
    for bad in (dict(y=y[:2]), dict(y=torch.zeros((3, 129))), dict(w=w.float()), dict(w_scale=s[:1]), dict(w_scale=s.double()), dict(w_scale=torch.zeros((2, 4))[:, ::2]), dict(w=w[:, :128]), dict(bias=torch.zeros(129)),
                dict(residual=y.bfloat16()), dict(residual=y[:2]), dict(x_scale=torch.zeros((2, 3))), dict(x=x.to(U8), x_scale=torch.zeros((2, 4))), dict(x=x.to(U8), x_scale=torch.zeros((2, 3), dtype=BF)),
                dict(x=torch.zeros((256, 3)).t())):
        with pytest.raises(ValueError):
            fb.fp8_linear_args(**{**dict(x=x, w=w, w_scale=s, y=y), **bad})
    with pytest.raises(TypeError):
        fb.fp8_linear_args(x.to(U8), w, s, y)
    for bad in (dict(codes=w), dict(codes=torch.zeros((3, 256))), dict(scale=torch.zeros((3, 2))), dict(scale=torch.zeros((2, 3), dtype=BF)), dict(block_rows=128), dict(x=x.t())):
        with pytest.raises(ValueError):
            fb.fise_fp8_quantize(**{**dict(x=x, codes=torch.zeros((3, 256), dtype=U8), scale=torch.zeros((2, 3)), stream=0), **bad})


def test_route_and_expert_bindings():
    i32 = dict(dtype=torch.int32)
    logits, ids, w, o, sl = torch.zeros((6, 4)), torch.zeros((6, 2), **i32), torch.zeros((6, 2)), torch.zeros(5, **i32), torch.zeros(12, **i32)
    assert fb.route_args(logits, ids, w, o, sl).k == 2
    for bad in (dict(ids=ids.long()), dict(ids=ids[:5]), dict(weights=w.bfloat16()), dict(offsets=o[:4]), dict(slots=sl[:11]), dict(offsets=None), dict(bias=torch.zeros(3)), dict(bias=torch.zeros(4, dtype=BF)), dict(logits=torch.zeros((4, 6)).t())):
        with pytest.raises(ValueError):
            fb.route_args(**{**dict(logits=logits, ids=ids, weights=w, offsets=o, slots=sl), **bad})
    ok = dict(x=torch.zeros((6, 32)), ids=ids, weights=w, offsets=o, slots=sl, w_in=torch.zeros((4, 2, 16, 32), dtype=U8), w_in_scale=torch.zeros((4, 2, 1, 1)), w_out=torch.zeros((4, 8, 16), dtype=U8),
              w_out_scale=torch.zeros((4, 1, 1)), y=torch.zeros((6, 8)))
    assert fb.expert_mlp_args(**ok).I == 16
    for bad in (dict(ids=ids[:5]), dict(weights=w[:5]), dict(offsets=o[:4]), dict(slots=sl[:11]), dict(w_in=torch.zeros((4, 2, 16, 16), dtype=U8)), dict(w_in=torch.zeros((4, 3, 16, 32), dtype=U8)), dict(w_in=ok["w_in"].float()),
                dict(w_in_scale=torch.zeros((4, 1, 1, 1))), dict(w_out=torch.zeros((3, 8, 16), dtype=U8)), dict(w_out_scale=torch.zeros((4, 2, 1))), dict(y=torch.zeros((6, 16))), dict(y=torch.zeros((5, 8))),
                dict(residual=torch.zeros((6, 8), dtype=BF)), dict(x=torch.zeros((32, 6)).t())):
        with pytest.raises(ValueError):
            fb.expert_mlp_args(**{**ok, **bad})


def test_tensors_that_are_not_on_the_current_gpu():
    """Tensors in host memory, or a workspace elsewhere, would fault the GPU: the calls refuse them."""
    x, w, s, y = torch.zeros((3, 256)), torch.zeros((130, 256), dtype=U8), torch.zeros((2, 2)), torch.zeros((3, 130))
    with pytest.raises(ValueError):
        fb.fise_fp8_linear(fb.fp8_linear_args(x, w, s, y), torch.zeros(4096, dtype=U8), stream=0)
    with pytest.raises(ValueError):
        fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(torch.zeros((1, 4, 1, 8)))], [8], 10.0, grid=(1, 2, 2)), stream=0)
    with pytest.raises(ValueError):
        fb.fp8_linear_args(x, w.to("meta"), s, y)
