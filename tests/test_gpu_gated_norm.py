"""GPU checks of the norms around a block with its gate and modulation, element by element against 64-bit arithmetic.

Tolerance, from arithmetic: an output is off by its own rounding (2^-8 of it in bf16, 2^-24 in float), and by float arithmetic on magnitudes that the
reference adds up beside the values: a sum of C channels goes through at most 64 additions of a lane, 6 of a wave and 4 of a workgroup, and fewer than
30 roundings lie around the two sums of each of the two norms: 2 * (74 + 30) * 2^-24 of those magnitudes.  A norm multiplies what its input is off
by with w / std."""
import math

import pytest
import torch

from helpers import DEV

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
T = {"f32": torch.float32, "bf16": torch.bfloat16}
STEPS = 2 * (74 + 30) * 2.0 ** -24


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def norm(v, mag, kind, w, b, eps):
    """Value and magnitude of a norm of v, whose terms have the magnitude mag."""
    if kind == "none":
        return v, mag
    top = mag.amax(-1, keepdim=True)
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    rs = 1 / torch.sqrt((v ** 2).mean(-1, keepdim=True) + eps)
    w = 1.0 if w is None else w.double()
    out, m = v * rs * w, (v.abs() + top) * rs * (w if isinstance(w, float) else w.abs())
    # what the input is off by also moves the root: by at most that over std, times the value
    m = m + out.abs() * top * rs
    return (out, m) if b is None else (out + b.double(), m + b.double().abs())


def reference(x, h, gate, sc, sh, post, pw, pb, pre, qw, qb, a, eps):
    x = x.double()
    r, mag = a * x, (a * x).abs()
    if h is not None:
        h = h.double()
        v, m = norm(h, h.abs(), post, pw, pb, eps)
        if gate is not None:
            v, m = v * gate.double()[:, None], m * gate.double().abs()[:, None]
        r, mag = r + v, mag + m
    y, my = norm(r, mag, pre, qw, qb, eps)
    if sc is not None:
        y, my = y * (1 + sc.double()[:, None]), my * (1 + sc.double().abs()[:, None])
    if sh is not None:
        y, my = y + sh.double()[:, None], my + sh.double().abs()[:, None]
    return r, mag, y, my


def close(got, want, mag):
    err = (got.double().cpu() - want).abs()
    tol = HALF[got.dtype] * want.abs() + STEPS * mag
    assert bool((err <= tol).all()), float((err / tol).max())


def token_rows(idx, tile, H, W):
    if not tile:
        return torch.arange(H * W)
    order = torch.arange(H * W).view(H // tile, tile, W // tile, tile).transpose(1, 2).reshape(-1, tile * tile)
    return order[torch.tensor(idx)].reshape(-1)


# B, H, W, C, tile, tiles, type, post, pre, gate, modulation, forms of h and y: one wave a row and a workgroup a row with 1 to 8 pieces a lane, rows that do
# not fill the workgroup's lanes, one row
CASES = [(2, 8, 8, 320, 4, [1, 2], "bf16", "rms", "layer", True, "both", "rows", "rows"), (1, 1, 1, 8, 0, [], "bf16", "layer", "rms", True, "both", "rows", "rows"),
         (2, 4, 6, 512, 1, [0, 5, 23], "f32", "layer", "layer", True, "both", "map", "map"), (1, 5, 3, 520, 0, [], "bf16", "rms", "rms", False, "none", "rows", "map"),
         (2, 8, 8, 1280, 2, [3, 15], "bf16", "none", "layer", True, "both", "map", "rows"), (3, 4, 4, 2048, 4, [0], "f32", "none", "none", True, "scale", "rows", "rows"),
         (1, 2, 2, 2056, 0, [], "bf16", "layer", "none", False, "none", "rows", None), (2, 2, 4, 4104, 2, [1], "f32", "rms", "layer", True, "shift", "rows", "rows"),
         (1, 3, 1, 8200, 0, [], "bf16", "rms", "layer", True, "both", "rows", "rows"), (1, 1, 2, 16384, 0, [], "f32", "layer", "rms", False, "both", "rows", "rows"),
         (2, 16, 16, 640, 8, [0, 3], "bf16", "no branch", "layer", False, "both", None, "rows"), (5, 8, 8, 64, 8, [0], "bf16", "rms", "rms", True, "both", "rows", "rows")]


@pytest.mark.parametrize("B,H,W,C,tile,idx,dt,post,pre,gated,modulated,hform,yform", CASES)
def test_gated_norm(fb, B, H, W, C, tile, idx, dt, post, pre, gated, modulated, hform, yform):
    g = torch.Generator().manual_seed(C * 13 + H)
    rnd = lambda *s, m=0.0, d=1.0: m + d * torch.randn(s, generator=g)
    x, r0, y0 = rnd(B, H, W, C, d=1.5, m=0.5).to(T[dt]), rnd(B, H, W, C).to(T[dt]), rnd(B, H, W, C).to(T[dt])
    rows = token_rows(idx, tile, H, W)
    M = len(rows)
    h = None if hform is None else rnd(B, H, W, C, m=-2.0).to(T[dt]) if hform == "map" else rnd(B, M, C, m=-2.0).to(T[dt])
    w = {k: rnd(C, m=1.0, d=0.2).to(T[dt]) for k in ("post", "pre")}
    b = {k: rnd(C, d=0.2).to(T[dt]) for k in ("post", "pre")}
    mod = rnd(B, 3 * C + 4, d=0.4)
    gate = mod[:, :C] if gated else None
    sc = mod[:, C:2 * C] if modulated in ("both", "scale") else None
    sh = mod[:, 2 * C:3 * C] if modulated in ("both", "shift") else None
    kind = {"no branch": "none"}.get(post, post)
    pw, pb = (w["post"] if kind != "none" else None), (b["post"] if kind == "layer" else None)
    qw, qb = (w["pre"] if pre == "rms" or (pre == "layer" and C % 16 == 0) else None), (b["pre"] if pre == "layer" and C % 16 == 0 else None)
    hr = None if h is None else h.view(B, H * W, C)[:, rows] if hform == "map" else h
    r_, mag, y_, my = reference(x.view(B, -1, C)[:, rows], hr, gate, sc, sh, kind, pw, pb, pre, qw, qb, 0.75, 1e-5)
    d = lambda t: None if t is None else t.to(DEV)
    r = r0.to(DEV)
    y = None if yform is None else y0.to(DEV) if yform == "map" else torch.full((B, M, C), float("nan"), dtype=T[dt], device=DEV)
    md = mod.to(DEV)
    a = fb.gated_norm_args(d(x), h=d(h), post=kind, post_w=d(pw), post_b=d(pb), gate=md[:, :C] if gated else None, res_scale=0.75, pre=pre, pre_w=d(qw), pre_b=d(qb),
                           mod_scale=md[:, C:2 * C] if sc is not None else None, mod_shift=md[:, 2 * C:3 * C] if sh is not None else None, eps=1e-5,
                           tile_idx=torch.tensor(idx, dtype=torch.int32, device=DEV) if tile else None, n_active=len(idx), tile=tile, r=r, y=y)
    fb.fise_masked_gated_norm(a)
    rest = torch.ones(H * W, dtype=torch.bool)
    rest[rows] = False
    close(r.view(B, -1, C).cpu()[:, rows], r_, mag)
    assert torch.equal(r.view(B, -1, C).cpu()[:, rest], r0.view(B, -1, C)[:, rest])
    if y is not None:
        yv = y.view(B, -1, C).cpu()
        close(yv[:, rows] if yform == "map" else yv, y_, my)
        if yform == "map":
            assert torch.equal(yv[:, rest], y0.view(B, -1, C)[:, rest])


def test_in_place_and_single_outputs(fb):
    """r over x, y over h, and each output alone: the same bits."""
    g = torch.Generator().manual_seed(3)
    for C in (320, 1280):
        x, h = torch.randn((2, 8, 8, C), generator=g).to(torch.bfloat16).to(DEV), torch.randn((2, 32, C), generator=g).to(torch.bfloat16).to(DEV)
        idx = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
        gate = torch.randn((2, C), generator=g).to(DEV)
        kw = dict(post="rms", gate=gate, pre="layer", tile_idx=idx, n_active=2, tile=4)
        r, y = x.clone(), torch.empty_like(h)
        fb.fise_masked_gated_norm(fb.gated_norm_args(x, h=h, r=r, y=y, **kw))
        y2 = torch.empty_like(h)
        fb.fise_masked_gated_norm(fb.gated_norm_args(x, h=h, y=y2, **kw))
        x2, h2 = x.clone(), h.clone()
        fb.fise_masked_gated_norm(fb.gated_norm_args(x2, h=h2, r=x2, y=h2, **kw))
        assert torch.equal(y, y2) and torch.equal(x2, r) and torch.equal(h2, y)
        r3 = x.clone()
        kw["pre"] = "none"
        fb.fise_masked_gated_norm(fb.gated_norm_args(x, h=h, r=r3, **kw))
        assert torch.equal(r3, r)


def test_rows_that_are_not_finite_or_constant(fb):
    C = 320
    x = torch.ones((1, 2, 4, C), dtype=torch.float32)
    x[0, 0, 1, 5], x[0, 0, 2, 7], x[0, 1, 0] = math.inf, math.nan, 0.0
    y, r = torch.zeros((1, 8, C), device=DEV), torch.zeros((1, 2, 4, C), device=DEV)
    fb.fise_masked_gated_norm(fb.gated_norm_args(x.to(DEV), pre="layer", r=r, y=y))
    assert torch.equal(r.cpu().nan_to_num(7.0), x.nan_to_num(7.0))
    bad = y.cpu().isnan().any(-1)[0]
    assert bad.tolist() == [False, True, True, False, False, False, False, False]
    assert bool((y.cpu()[0, ~bad] == 0).all())                                  # a constant row has nothing left but eps under the root


def test_captured_and_replayed(fb):
    g = torch.Generator().manual_seed(4)
    C = 640
    x, h = torch.randn((2, 16, 16, C), generator=g).to(torch.bfloat16).to(DEV), torch.randn((2, 256, C), generator=g).to(torch.bfloat16).to(DEV)
    r, y = torch.zeros_like(x), torch.zeros_like(h)
    a = fb.gated_norm_args(x, h=h, post="layer", pre="rms", r=r, y=y)
    fb.fise_masked_gated_norm(a)
    want = r.clone(), y.clone()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=st):
        fb.fise_masked_gated_norm(a, stream=st)
    for rep in range(3):
        r.zero_(); y.zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(r, want[0]) and torch.equal(y, want[1]), rep


@pytest.mark.parametrize("H,W,C", [(8192, 4097, 8), (4096, 2049, 520)])
def test_more_rows_than_a_launch_has(fb, H, W, C):
    x = torch.zeros((1, H, W, C), dtype=torch.bfloat16, device=DEV)
    y = torch.full_like(x, float("nan"))
    g = torch.Generator().manual_seed(8)
    at = torch.tensor([0, 1, 2 ** 23 - 1, 2 ** 23, 2 ** 23 + 5, H * W // 2, 2 ** 25 - 1, 2 ** 25, H * W - 1])
    at = at[at < H * W]
    rows = torch.randn((at.numel(), C), generator=g).to(torch.bfloat16)
    x.view(-1, C)[at.to(DEV)] = rows.to(DEV)
    fb.fise_masked_gated_norm(fb.gated_norm_args(x, pre="layer", y=y))
    want, mag, wy, my = reference(rows[None], None, None, None, None, "none", None, None, "layer", None, None, 1.0, 1e-5)
    close(y.view(-1, C)[at.to(DEV)][None], wy, my)
    hit = torch.ones(H * W, dtype=torch.bool, device=DEV)
    hit[at.to(DEV)] = False
    assert bool((y.view(-1, C)[hit] == 0).all())
