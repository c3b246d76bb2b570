"""GPU checks of what the experts' sums lose: nothing but float's roundings in gate and up, for float results, and below 512 pairs an expert; products below 2^-13 of the largest of eight
in the second product, for bf16 results of more.

Tolerance: as in the other tests of the experts, but the matrix unit's 2^-10 of the magnitudes only where the 8-bit instruction is the documented one, and 2^-11 for a pair's result on
its way to a sum in bf16 (eleven bits; 2^-39 of the largest it shares a power of two with), none for float."""
import pytest
import torch

from helpers import DEV
from test_gpu_experts import CASES, HALF, T_, Experts, call, pick
from test_gpu_fp8 import blocks, in_eight, nearest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def per_block(t, I):
    """The largest of each block of 128 channels, at every channel."""
    return torch.nn.functional.pad(t, (0, blocks(I) * 128 - I)).view(t.shape[0], -1, 128).amax(-1).repeat_interleave(128, 1)[:, :I]


def want(ex, x, ids, weight, residual, y_type):
    """The definition in 64 bits and its tolerance."""
    E, K, I, N = ex.dims
    T, k = ids.shape
    drop = 2.0 ** -10 if y_type == torch.bfloat16 and T * k >= 512 * E else 0.0
    sums = lambda n: 2 * (128 + 3 * n / 128 + 4) * 2.0 ** -24
    c, e = in_eight(x, 1)
    v = (c * torch.exp2(e).repeat_interleave(128, 1)[:, :K]).to(DEV)
    y = torch.zeros((T, N), dtype=torch.float64, device=DEV) if residual is None else residual.double().to(DEV)
    mag, tol = y.abs(), torch.zeros_like(y)
    weight = weight.double().to(DEV)
    for i in range(E):
        t, j = (ids == i).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        r = v[t]
        (g, dg), (u, du) = ((r @ w.t(), sums(K) * (r.abs() @ w.abs().t())) for w in ex.ins[i])
        s = g * torch.sigmoid(g)
        h = s * u
        dh = 1.1 * dg * (u.abs() + du) + s.abs() * du + 2.0 ** -20 * h.abs()
        hc, he = in_eight(h.cpu(), 1)
        step = torch.exp2(he).repeat_interleave(128, 1)[:, :I].to(DEV)
        hq = hc.to(DEV) * step
        lo, hi = hq.clone(), hq.clone()
        top, low = per_block(h.abs() + dh, I), per_block((h.abs() - dh).clamp(min=0), I)
        for f, may in ((0.5, low <= 224 * step), (1.0, torch.ones_like(h, dtype=torch.bool)), (2.0, top > 448 * step)):      # a block's scale may be the one beside it
            a, b = (nearest(((h + d) / (step * f)).clamp(-448, 448)) * step * f for d in (-dh, dh))
            lo, hi = torch.where(may, torch.minimum(lo, a), lo), torch.where(may, torch.maximum(hi, b), hi)
        w = ex.outs[i]
        f = hq @ w.t()
        off = torch.maximum(hi - hq, hq - lo) @ w.abs().t() + (drop + sums(I)) * (hq.abs() @ w.abs().t())
        if y_type == torch.bfloat16:
            off = off + 2.0 ** -11 * (f.abs() + off) + 2.0 ** -39 * (f.abs() + off).amax(1, keepdim=True)
        p = weight[t, j][:, None]
        y.index_put_((t,), p * f, accumulate=True)
        mag.index_put_((t,), (p * f).abs(), accumulate=True)
        tol.index_put_((t,), p.abs() * off, accumulate=True)
    return y.cpu(), (tol + (k + 2) * 2.0 ** -24 * mag + HALF[y_type] * (y.abs() + tol)).cpu()


# the other tests' cases, and float results on every form: tiles of 128 rows, and where bf16 takes those of 256
MORE = [(300, 4, 272, 144, 264, 2, 2, "bf16", "f32", True), (700, 8, 400, 272, 136, 3, 4, "f32", "f32", False), (1100, 2, 400, 272, 264, 1, 1, "bf16", "f32", True), (3, 8, 272, 144, 72, 2, 0, "bf16", "f32", True)]


@pytest.mark.parametrize("T,E,K,I,N,k,skew,xt,yt,res", CASES + MORE)
def test_random(fb, T, E, K, I, N, k, skew, xt, yt, res):
    g = torch.Generator().manual_seed(T * 31 + E + K)
    ex = Experts(g, E, K, I, N)
    x = (torch.randn((T, K), generator=g) * (1 + 20 * (torch.rand((K,), generator=g) < 0.02))).to(T_[xt])
    ids, w = pick(g, T, E, k, skew)
    residual = torch.randn((T, N), generator=g).to(T_[yt]) if res else None
    y = call(fb, ex, x, ids, w, residual, T_[yt])
    ref, tol = want(ex, x, ids, w, residual, T_[yt])
    err = (y.double().cpu() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
