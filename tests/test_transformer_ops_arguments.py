"""What the entry points for transformer denoisers refuse, on the host, before anything is launched; no GPU needed."""
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


def w4():
    return set_all(fb.fise_w4_linear_args(), x=A, x_dtype=1, x_stride=256, packed=A, N=64, K=256, group=64, y=A, y_dtype=1, y_stride=64, M=0)


@pytest.mark.parametrize("change,code", [({}, 0), ({"x": None}, -1), ({"packed": None}, -1), ({"y": None}, -1), ({"x_dtype": 2}, -3), ({"y_dtype": -1}, -3),
                                         ({"bias": A, "bias_dtype": 9}, -3), ({"N": 0}, -2), ({"K": 0}, -2), ({"group": 48}, -2), ({"group": 16}, -2), ({"group": 512}, -2),
                                         ({"M": -1}, -2), ({"x_stride": 248}, -2), ({"y_stride": 63}, -2), ({"residual": A, "residual_stride": 8}, -2),
                                         ({"K": 252}, -4), ({"x_stride": 260}, -4), ({"x": A + 8}, -4), ({"packed": A + 4}, -4), ({"y": A + 1}, -4),
                                         ({"bias": A + 2, "bias_dtype": 0}, -4), ({"N": 1 << 21, "y_stride": 1 << 21}, -2)])
def test_w4_linear(change, code):
    assert call("fise_w4_linear", w4, change, None) == code
    if code:
        assert "fise_w4_linear" in fb.fise_last_error()


def test_w4_pack():
    L = fb.lib()
    assert L.fise_w4_linear(None, None) == -1
    assert L.fise_w4_bytes(64, 256, 64) == 64 * 128 + 64 * 4 * 2 and L.fise_w4_bytes(1, 1, 256) == 1024 + 256
    assert L.fise_w4_bytes(0, 256, 64) == 0 and L.fise_w4_bytes(64, 256, 33) == 0
    with pytest.raises(fb.FiseError):
        fb.fise_w4_bytes(64, 256, 100)
    assert L.fise_w4_pack(None, 0, None, 64, 256, 64, A, None) == -1
    assert L.fise_w4_pack(A, 5, None, 64, 256, 64, A, None) == -3
    assert L.fise_w4_pack(A, 0, None, 64, 256, 65, A, None) == -2
    assert L.fise_w4_pack(A, 0, A + 2, 64, 256, 64, A, None) == -4
    assert L.fise_w4_unpack(A, 64, 256, 64, None, 0, None) == -1
    assert L.fise_w4_unpack(A, 64, 0, 64, A, 0, None) == -2
    assert L.fise_w4_unpack(A, 64, 256, 64, A + 4, 0, None) == -4


def test_w4_binding_checks_its_tensors():
    packed = torch.zeros(fb.fise_w4_bytes(64, 256, 64), dtype=torch.uint8)
    x, y = torch.zeros((3, 256)), torch.zeros((3, 64))
    assert fb.w4_linear_args(x, packed, 64, y).x_stride == 256
    for bad in (dict(x=x, y=y[:2]), dict(x=x.t().contiguous().t(), y=y), dict(x=x, y=y, bias=torch.zeros(63)), dict(x=x, y=y, residual=torch.zeros((3, 64), dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            fb.w4_linear_args(bad.pop("x"), packed, 64, bad.pop("y"), **bad)
    with pytest.raises(ValueError):
        fb.w4_linear_args(x, packed[:-1], 64, y)
    with pytest.raises(TypeError):
        fb.w4_linear_args(x.half(), packed, 64, y)
    with pytest.raises(ValueError):
        fb.fise_w4_pack(torch.zeros((64, 256)), packed, 64, scale=torch.zeros((64, 3), dtype=torch.bfloat16))


def norm():
    return set_all(fb.fise_gated_norm_args(), x=A, B=2, H=8, W=8, C=320, dtype=1, h=A, post_norm=2, post_w=A, gate=A, res_scale=1.0, pre_norm=1, pre_w=A, pre_b=A,
                   mod_scale=A, mod_shift=A, mod_stride=960, eps=1e-5, tile_idx=A, n_active=0, tile=4, r=A, y=2 * A)


@pytest.mark.parametrize("change,code", [({}, 0), ({"x": None}, -1), ({"r": None, "y": None}, -1), ({"dtype": 3}, -3), ({"post_norm": 3}, -2), ({"pre_norm": -1}, -2), ({"C": 0}, -2),
                                         ({"C": 16392}, -2), ({"tile": 3}, -2), ({"tile": -1}, -2), ({"B": 0}, -2), ({"H": 0}, -2), ({"C": 324}, -4), ({"mod_stride": 312}, -2),
                                         ({"mod_stride": 961}, -4), ({"h": None}, -1), ({"y": None}, -1), ({"post_b": A}, -2), ({"pre_norm": 0}, -2), ({"r": A + 8}, -4),
                                         ({"gate": A + 4}, -4), ({"n_active": -1}, -5), ({"n_active": 5}, -5), ({"n_active": 2, "tile_idx": None}, -1), ({"y": A}, -2),
                                         ({"B": 1 << 20, "H": 64, "W": 64}, -2), ({"r": None}, 0)])
def test_gated_norm(change, code):
    assert call("fise_masked_gated_norm", norm, change, None) == code
    if code:
        assert "fise_masked_gated_norm" in fb.fise_last_error()


def test_gated_norm_binding_checks_its_tensors():
    x, mod = torch.zeros((2, 8, 8, 64)), torch.zeros((2, 192))
    idx = torch.zeros(2, dtype=torch.int32)
    a = fb.gated_norm_args(x, h=torch.zeros((2, 32, 64)), gate=mod[:, :64], mod_scale=mod[:, 64:128], tile_idx=idx, n_active=2, tile=4, r=x, y=torch.zeros((2, 32, 64)))
    assert a.mod_stride == 192 and not a.h_is_map and a.C == 64
    for bad in (dict(h=torch.zeros((2, 31, 64))), dict(h=torch.zeros((2, 32, 64), dtype=torch.bfloat16)), dict(gate=mod[:, :64].bfloat16()), dict(gate=mod[:, :60]),
                dict(gate=mod[:, :64], mod_scale=torch.zeros((2, 64))), dict(pre_w=torch.zeros(63)), dict(tile_idx=idx[:1]), dict(tile_idx=idx.long())):
        with pytest.raises(ValueError):
            fb.gated_norm_args(x, **{**dict(tile_idx=idx, n_active=2, tile=4, r=x), **bad})


def latent():
    return set_all(fb.fise_latent_attention_args(), q=A, cache=A, w_uk=A, w_uv=A, out=2 * A, B=2, M=0, n_keys=100, cache_tokens=128, heads=8, d=128, dr=64, dv=128, r=512, scale=0.1,
                   dtype=1)


@pytest.mark.parametrize("change,code", [({}, 0), ({"q": None}, -1), ({"cache": None}, -1), ({"w_uk": None}, -1), ({"w_uv": None}, -1), ({"out": None}, -1), ({"dtype": 0}, -3),
                                         ({"B": 0}, -2), ({"M": -1}, -2), ({"n_keys": -1}, -2), ({"cache_tokens": 99}, -2), ({"heads": 0}, -2), ({"d": 168}, -2), ({"dv": 0}, -2),
                                         ({"dr": 72}, -2), ({"r": 520}, -2), ({"r": 0}, -2), ({"form": 3}, -2), ({"form": -1}, -2), ({"d": 36}, -4), ({"dr": 4}, -4), ({"dv": 20}, -4),
                                         ({"r": 100}, -4), ({"q": A + 8}, -4), ({"out": A + 2}, -4), ({"scale": 0.0}, -2), ({"scale": float("nan")}, -2), ({"scale": float("inf")}, -2),
                                         ({"M": 4}, -1), ({"heads": 70000}, -2), ({"M": 1 << 28}, -2), ({"n_keys": 1 << 27, "cache_tokens": 1 << 27}, -2)])
def test_latent_attention(change, code):
    assert call("fise_latent_attention", latent, change, None, 0, None) == code
    if code:
        assert "fise_latent_attention" in fb.fise_last_error()


@pytest.mark.parametrize("form", [0, 1, 2])
def test_latent_attention_workspace(form):
    L, a = fb.lib(), set_all(latent(), M=4, form=form)
    need = fb.fise_latent_attention_workspace_bytes(a)
    assert need > 256
    assert L.fise_latent_attention(ctypes.byref(a), 256, need - 1, None) == -5
    assert L.fise_latent_attention(ctypes.byref(a), 128, need, None) == -4
    assert L.fise_latent_attention(None, 256, need, None) == -1
    a.r = 7
    assert fb.fise_latent_attention_workspace_bytes(a) == 0


def test_latent_attention_binding_checks_its_tensors():
    bf = dict(dtype=torch.bfloat16)
    q, c, wk, wv, out = (torch.zeros(s, **bf) for s in ((2, 3, 4, 48), (2, 5, 6, 80), (4, 32, 64), (4, 24, 64), (2, 3, 96)))
    a = fb.latent_attention_args(q, c, wk, wv, out, 0.2)
    assert (a.n_keys, a.cache_tokens, a.d, a.dr, a.dv, a.r) == (30, 30, 32, 16, 24, 64)
    for bad in (dict(out=out[:, :2]), dict(cache=c[..., :72]), dict(q=q.float()), dict(w_uv=wv[:3]), dict(kv_len=torch.zeros(2)), dict(kv_len=torch.zeros(3, dtype=torch.int32)),
                dict(cache=c.transpose(1, 2)), dict(w_uk=wk.transpose(1, 2))):
        with pytest.raises(ValueError):
            fb.latent_attention_args(**{**dict(q=q, cache=c, w_uk=wk, w_uv=wv, out=out, scale=0.2), **bad})


@pytest.mark.parametrize("change,code", [({"B": 1 << 10, "M": 1 << 10}, -2), ({"B": 1 << 10, "M": (1 << 10) - 1, "form": 1}, -1), ({"form": 2, "n_keys": 1 << 26, "cache_tokens": 1 << 26}, -2),
                                         ({"form": 1, "n_keys": 1 << 26, "cache_tokens": 1 << 26, "M": 1}, -1), ({"form": 2, "B": 300, "heads": 65535}, -2), ({"form": 1, "B": 300, "heads": 65535}, -1),
                                         ({"form": 2, "M": 1 << 10, "heads": 1024}, -1)])
def test_latent_attention_grids(change, code):
    """What a launch's grid holds is taken (and ends at the missing workspace), more refused."""
    assert call("fise_latent_attention", latent, {"M": 1, **change}, None, 0, None) == code
    assert (fb.fise_latent_attention_workspace_bytes(set_all(latent(), M=change.get("M", 1), **{k: v for k, v in change.items() if k != "M"})) > 0 if code == -1 else True)
