"""GPU checks of rotary positions on several axes against 64-bit rotations.

Tolerance, from arithmetic: an angle's fraction of a turn is rounded to float (2^-26 turns = 2^-23.3 rad), sine and cosine are within 2^-22 of their values, the
two products and the sum add three roundings of 2^-24: (|u| + |v|) 2^-21 holds all of it.  Behind that the output's own rounding, half a step."""
import math

import pytest
import torch

from helpers import DEV

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def places(grid, axes, tokens):
    t, h, w = grid
    tokens = torch.as_tensor(tokens)
    split = [tokens // (h * w), tokens // w % h, tokens % w]
    return torch.stack([tokens] if axes == 1 else split[3 - axes:], -1).double()


def tile_tokens(idx, grid, tile):
    t, h, w = grid
    out = []
    for i in idx:
        f, y, x = i // (h // tile * (w // tile)), i // (w // tile) % (h // tile), i % (w // tile)
        out += [(f * h + y * tile + p // tile) * w + x * tile + p % tile for p in range(tile * tile)]
    return out


def turn(x, pos, start, axes, theta, pairing, shared, inverse, offset):
    """x [B, M, heads, d] double and pos [B or 1, M, axes] double -> its rotation and |u| + |v| of every channel."""
    y, mag, half, first, begin = x.clone(), torch.zeros_like(x), sum(axes) // 2, 0, 0
    for j, n in enumerate(axes):
        for i in range(n // 2):
            f = theta[0] ** (-2.0 * (first + i) / (2 * half)) if shared else theta[j] ** (-2.0 * i / n)
            angle = ((pos[..., j] + offset[j]) * f)[:, :, None]
            a, b = {"adjacent": (2 * (first + i), 2 * (first + i) + 1), "halves": (first + i, first + i + half), "axis_halves": (begin + i, begin + i + n // 2)}[pairing]
            u, v, c, s = x[..., start + a], x[..., start + b], torch.cos(angle), torch.sin(angle) * (-1 if inverse else 1)
            y[..., start + a], y[..., start + b] = u * c - v * s, u * s + v * c
            mag[..., start + a] = mag[..., start + b] = u.abs() + v.abs()
        first, begin = first + n // 2, begin + n
    return y, mag


def close(got, want, mag):
    err, tol = (got.double().cpu() - want).abs(), HALF[got.dtype] * want.abs() + 2.0 ** -21 * mag
    assert bool((err <= tol).all()), float((err / tol.clamp(min=1e-30)).max())


# grid, tile, tiles (None: all tokens), heads, d, start, axes, pairing, shared, type, inverse
CASES = [((1, 8, 8), 0, None, 2, 32, 0, [32], "adjacent", False, "bf16", False), ((1, 8, 8), 4, [1, 2], 3, 72, 40, [16, 16], "adjacent", False, "bf16", False),
         ((3, 4, 8), 2, [0, 5, 23], 5, 128, 0, [16, 56, 56], "adjacent", False, "bf16", True), ((2, 6, 4), 0, None, 1, 64, 0, [24, 20, 20], "halves", True, "f32", False),
         ((2, 6, 4), 0, None, 4, 96, 16, [16, 32, 16], "axis_halves", False, "bf16", False), ((1, 4, 4), 1, [15, 0, 7], 2, 23, 3, [6, 10], "adjacent", True, "bf16", False),
         ((1, 4, 4), 0, None, 2, 21, 1, [6, 4, 8], "halves", False, "f32", True), ((5, 2, 2), 0, None, 17, 40, 0, [6, 14, 20], "axis_halves", True, "f32", False),
         ((1, 64, 64), 0, None, 24, 128, 0, [64, 64], "adjacent", False, "bf16", False), ((1, 1, 1), 0, None, 1, 2, 0, [2], "adjacent", False, "bf16", False),
         ((1, 16, 16), 8, [3], 8, 1024, 0, [512, 512], "halves", False, "f32", False)]


@pytest.mark.parametrize("grid,tile,tiles,heads,d,start,axes,pairing,shared,type,inverse", CASES)
def test_grid(fb, grid, tile, tiles, heads, d, start, axes, pairing, shared, type, inverse):
    g = torch.Generator().manual_seed(d * 31 + heads)
    tokens = tile_tokens(tiles, grid, tile) if tile else list(range(math.prod(grid)))
    B, M, theta, offset = 2, len(tokens), [10000.0, 500.0, 20.0][:len(axes)], [0.5, -3.0, 7.0][:len(axes)]
    idx = torch.tensor(tiles, dtype=torch.int32, device=DEV) if tile else None
    x = torch.randn((B, M, heads, d), generator=g).to(T[type])
    k = torch.randn((B, math.prod(grid), 1, d), generator=g).to(T[type])
    xo, ko = torch.full_like(x, float("nan"), device=DEV), torch.full_like(k, 7.0, device=DEV)
    a = fb.rotary_args([fb.rotary_tensor(x.to(DEV), xo, start), fb.rotary_tensor(k.to(DEV), ko, start, x_is_map=True, y_is_map=True)], axes, theta, offset=offset, grid=grid, tile_idx=idx,
                       n_active=len(tiles) if tile else 0, tile=tile, pairing=pairing, shared_frequencies=shared, inverse=inverse)
    fb.fise_rotary(a)
    pos = places(grid, len(axes), tokens)[None]
    close(xo, *turn(x.double(), pos, start, axes, theta, pairing, shared, inverse, offset))
    want, mag = turn(k[:, tokens].double(), pos, start, axes, theta, pairing, shared, inverse, offset)
    close(ko[:, tokens], want, mag)
    rest = torch.ones(math.prod(grid), dtype=torch.bool)
    rest[tokens] = False
    assert bool((ko[:, rest.to(DEV)] == 7.0).all())                          # tokens that are not active keep their values


@pytest.mark.parametrize("type", ["bf16", "f32"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("M,shared_pos", [(1, True), (3, False), (257, True)])
def test_positions(fb, type, whole, M, shared_pos):
    """Given positions: far, negative, fractional; strided views in and out; an angle of 10^6 and more radians is as exact as a small one."""
    g = torch.Generator().manual_seed(M)
    B, heads, axes, theta = 2, 3, [8, 16], [10000.0, 30.0]
    pos = torch.randint(-3000000, 3000000, (1 if shared_pos else B, M, 2), generator=g).to(torch.int32)
    if not whole:
        pos = pos.float() / 8
    wide = torch.randn((B, M, heads, 56), generator=g).to(T[type]).to(DEV)
    x = wide[..., 8:48]
    cache = torch.zeros((B, M, 5, 64), dtype=T[type], device=DEV)
    y = cache[:, :, 1:4, 16:56]
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(x, y, 8)], axes, theta, pos=pos.to(DEV), pairing="halves"))
    close(y, *turn(x.double().cpu(), pos.double(), 8, axes, theta, "halves", False, False, [0, 0]))
    cache[:, :, 1:4, 16:56] = 0
    assert not bool(cache.any())                                               # nothing beside it


@pytest.mark.parametrize("type", ["bf16", "f32"])
def test_in_place_and_back(fb, type):
    """In place; the inverse is the transposed map, so <R x, g> = <x, R^T g>: the gradient of a rotation."""
    g = torch.Generator().manual_seed(5)
    x, e = (torch.randn((1, 64, 4, 64), generator=g).to(T[type]) for _ in range(2))
    kw = dict(axes=[32, 32], theta=100.0, grid=(1, 8, 8), pairing="axis_halves")
    rx, re = x.to(DEV), e.to(DEV)
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(rx)], **kw))
    pos = places((1, 8, 8), 2, list(range(64)))[None]
    want, mag = turn(x.double(), pos, 0, [32, 32], [100.0] * 2, "axis_halves", False, False, [0, 0])
    close(rx, want, mag)
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(re)], inverse=True, **kw))
    close(re, *turn(e.double(), pos, 0, [32, 32], [100.0] * 2, "axis_halves", False, True, [0, 0]))
    assert abs(float((want * e.double()).sum() - (x.double() * turn(e.double(), pos, 0, [32, 32], [100.0] * 2, "axis_halves", False, True, [0, 0])[0]).sum())) < 1e-9
    # differences: the map is linear, so f(x + h e) - f(x) = h R e, whose product with e is the gradient's with e
    step = 1.0 / 64
    up = (x.double() + step * e.double()).to(torch.float32).to(DEV)
    low = x.to(torch.float32).to(DEV)
    for t in (up, low):
        fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(t)], **kw))
    slope = ((up.double() - low.double()).cpu() / step * x.double()).sum()
    grad = x.to(torch.float32).to(DEV)
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(grad)], inverse=True, **kw))
    # each of the 16384 differences is off by 2 (2^-24 |y| + 2^-21 (|u| + |v|)) / step and the rounding of up, 2^-24 |x| / step, at most
    bound = float(((2 * 2.0 ** -24 * mag + 2 * 2.0 ** -21 * mag + 2.0 ** -24 * 4 * mag) / step * x.double().abs()).sum() + (2.0 ** -20 * mag * e.double().abs()).sum())
    assert abs(float(slope - (grad.double().cpu() * e.double()).sum())) <= bound


def test_tiles_outside_and_none(fb):
    """Ids that are not on the grid: their rows stay as they were; no active tiles: nothing is written."""
    x = torch.ones((1, 8, 1, 8), device=DEV)
    y = torch.full((1, 16, 1, 8), 3.0, device=DEV)
    idx = torch.tensor([4, 1], dtype=torch.int32, device=DEV)                  # four tiles of 2 x 2
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(x, y, y_is_map=True)], [8], 10.0, grid=(1, 4, 4), tile_idx=idx, n_active=2, tile=2))
    changed = (y != 3.0).any(-1).view(16).nonzero().view(-1).tolist()
    assert changed == [2, 3, 6, 7]
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(x[:, :0], y, y_is_map=True)], [8], 10.0, grid=(1, 4, 4), tile_idx=idx, n_active=0, tile=2))
    assert (y != 3.0).any(-1).view(16).nonzero().view(-1).tolist() == changed


def test_values_that_are_not_finite_and_another_stream(fb):
    x = torch.randn((1, 4, 1, 8), device=DEV)
    x[0, 1, 0, 2], x[0, 2, 0, 5] = float("inf"), float("nan")
    y = torch.zeros_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(x, y)], [8], 10.0, grid=(1, 2, 2)), stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert (~torch.isfinite(y)).nonzero().tolist() == [[0, 1, 0, 2], [0, 1, 0, 3], [0, 2, 0, 4], [0, 2, 0, 5]]


@pytest.mark.parametrize("pairing", ["adjacent", "halves", "axis_halves"])
@pytest.mark.parametrize("type,axes", [("bf16", [6, 4, 2, 20]), ("f32", [2, 2, 2, 2]), ("bf16", [2, 14, 8, 8]), ("f32", [16, 8, 24, 16])])
@pytest.mark.parametrize("shared", [False, True])
def test_four_axes_with_borders_inside_a_thread(fb, type, axes, pairing, shared):
    """Four axes with positions of their own; axes of one pair; borders of axes anywhere among the pairs of a thread; a row of positions for each batch element."""
    g = torch.Generator().manual_seed(sum(axes))
    theta, offset = [10000.0, 7.0, 0.5, 1.0], [1.0, 0.0, -2.5, 100.0]
    pos = 500 * torch.randn((3, 5, 4), generator=g)
    x = torch.randn((3, 5, 2, sum(axes)), generator=g).to(T[type])
    y = torch.zeros_like(x, device=DEV)
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(x.to(DEV), y)], axes, theta, pos=pos.to(DEV), offset=offset, pairing=pairing, shared_frequencies=shared))
    close(y, *turn(x.double(), pos.double(), 0, axes, theta, pairing, shared, False, offset))


def test_a_tile_listed_twice(fb):
    x = torch.randn((1, 8, 2, 16), device=DEV)
    x[:, 4:] = x[:, :4]
    y = torch.zeros((1, 16, 2, 16), device=DEV)
    idx = torch.tensor([2, 2], dtype=torch.int32, device=DEV)
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(x, y, y_is_map=True)], [8, 8], 10.0, grid=(1, 4, 4), tile_idx=idx, n_active=2, tile=2))
    close(y[:, tile_tokens([2], (1, 4, 4), 2)], *turn(x[:, :4].double().cpu(), places((1, 4, 4), 2, tile_tokens([2], (1, 4, 4), 2))[None], 0, [8, 8], [10.0] * 2, "adjacent", False, False, [0, 0]))
