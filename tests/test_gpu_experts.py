"""GPU checks of the experts' feed-forward against its definition in 64 bits.

Tolerance, from arithmetic.  A sum over the columns of codes is off by d = (2^-10 + 2 (128 + 3 K / 128 + 4) 2^-24) of the magnitudes' sum at most (what the matrix unit drops of
eight products, and float roundings).  gate and up carry that into h: |dh| <= |silu(g)'|max |dg| |u| + |silu(g)| |du| with a slope of at most 1.1, and 2^-20 of h for SiLU in float.
A code of h is the nearest one, so it lies between the codes of h - dh and of h + dh; the difference of those two, times the weights' magnitudes, bounds what a result is off by, with the second
sum's own d, the rounding of an expert's result (half a step; where the output is bf16 that is no more than 2^-12 of it, held to bf16's), and the output's."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_fp8 import HALF, blocks, in_eight, nearest, weights, wide

pytestmark = pytest.mark.gpu
T_ = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


class Experts:
    def __init__(self, g, E, K, I, N):
        self.dims = (E, K, I, N)
        ins = [[weights(g, I, K) for _ in range(2)] for _ in range(E)]
        outs = [weights(g, N, I) for _ in range(E)]
        self.w_in, self.w_in_scale = torch.stack([torch.stack([p[0].view(torch.uint8) for p in e]) for e in ins]), torch.stack([torch.stack([p[1] for p in e]) for e in ins])
        self.w_out, self.w_out_scale = torch.stack([p[0].view(torch.uint8) for p in outs]), torch.stack([p[1] for p in outs])
        self.ins, self.outs = [[wide(*p).to(DEV) for p in e] for e in ins], [wide(*p).to(DEV) for p in outs]
        self.dev = [t.to(DEV) for t in (self.w_in, self.w_in_scale, self.w_out, self.w_out_scale)]

    def want(self, x, ids, weight, residual, y_type):
        """The definition in 64 bits and its tolerance."""
        E, K, I, N = self.dims
        T, k = ids.shape
        c, e = in_eight(x, 1)
        v = (c * torch.exp2(e).repeat_interleave(128, 1)[:, :K]).to(DEV)
        y = torch.zeros((T, N), dtype=torch.float64, device=DEV) if residual is None else residual.double().to(DEV)
        mag, tol = y.abs(), torch.zeros_like(y)
        weight = weight.double().to(DEV)
        half = HALF[y_type] if y_type == torch.bfloat16 else 2.0 ** -24
        for ex in range(E):
            t, j = (ids == ex).nonzero(as_tuple=True)
            if t.numel() == 0:
                continue
            r, d = v[t], 2.0 ** -10 + 2 * (128 + 3 * K / 128 + 4) * 2.0 ** -24
            (g, dg), (u, du) = ((r @ w.t(), d * (r.abs() @ w.abs().t())) for w in self.ins[ex])
            h = g * torch.sigmoid(g) * u
            dh = 1.1 * dg * (u.abs() + du) + (g * torch.sigmoid(g)).abs() * du + 2.0 ** -20 * h.abs()
            hc, he = in_eight(h.cpu(), 1)
            s = torch.exp2(he).repeat_interleave(128, 1)[:, :I].to(DEV)
            hq = hc.to(DEV) * s
            # a block whose largest value is next to a power of two may get the scale beside it: codes of either
            lo, hi = hq.clone(), hq.clone()
            for f in (0.5, 1.0, 2.0):
                a, b = nearest(((h - dh) / (s * f)).clamp(-448, 448)) * s * f, nearest(((h + dh) / (s * f)).clamp(-448, 448)) * s * f
                near = f == 1.0
                top = torch.nn.functional.pad(h.abs() + dh, (0, blocks(I) * 128 - I)).view(len(t), -1, 128).amax(-1).repeat_interleave(128, 1)[:, :I]
                low = torch.nn.functional.pad((h.abs() - dh).clamp(min=0), (0, blocks(I) * 128 - I)).view(len(t), -1, 128).amax(-1).repeat_interleave(128, 1)[:, :I]
                may = torch.full_like(h, near, dtype=torch.bool) | ((f == 2.0) & (top > 448 * s)) | ((f == 0.5) & (low <= 224 * s))
                lo, hi = torch.where(may, torch.minimum(lo, a), lo), torch.where(may, torch.maximum(hi, b), hi)
            w = self.outs[ex]
            f, m = hq @ w.t(), hq.abs() @ w.abs().t()
            d2 = 2.0 ** -10 + 2 * (128 + 3 * I / 128 + 4) * 2.0 ** -24
            off = torch.maximum(hi - hq, hq - lo) @ w.abs().t() + d2 * m
            off = off + half * (f.abs() + off)
            p = weight[t, j][:, None]
            y.index_put_((t,), p * f, accumulate=True)
            mag.index_put_((t,), (p * f).abs(), accumulate=True)
            tol.index_put_((t,), p.abs() * off, accumulate=True)
        return y.cpu(), (tol + (k + 2) * 2.0 ** -24 * mag + HALF[y_type] * (y.abs() + tol)).cpu()


def lists(ids, E):
    flat = ids.view(-1).long()
    key = torch.where(flat < 0, E, flat)
    slots = key.sort(stable=True).indices.to(torch.int32)
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64), torch.bincount(key, minlength=E + 1)[:E].cumsum(0))).to(torch.int32)
    n = int(offsets[-1])
    slots[n:] = 2 ** 30                                                        # nobody reads what is behind the last pair
    return offsets.to(DEV), slots.to(DEV)


def pick(g, T, E, k, skew):
    p = torch.randn((T, E), generator=g) + skew * torch.arange(E) / E
    top = p.topk(k, 1)
    return top.indices.to(torch.int32), torch.softmax(top.values, 1)


def call(fb, ex, x, ids, w, residual, y_type, fill=0x7f):
    E, K, I, N = ex.dims
    y = torch.full((x.shape[0], N), 3.0, dtype=y_type, device=DEV)
    o, s = lists(ids, E)
    a = fb.expert_mlp_args(x.to(DEV), ids.to(DEV), w.to(DEV), o, s, *ex.dev, y, residual=None if residual is None else residual.to(DEV))
    ws = torch.full((fb.fise_expert_mlp_workspace_bytes(a),), fill, dtype=torch.uint8, device=DEV)
    fb.fise_expert_mlp(a, ws)
    first = y.clone()
    fb.fise_expert_mlp(a, ws)
    assert torch.equal(first.view(torch.uint8), y.view(torch.uint8))           # the same sums in the same order, whatever the workspace held
    return y


# T, E, K, I, N, k, skew, x, y, residual: single tokens, one expert, experts without tokens, parts of tiles and of blocks on every side, tiles full of one expert
CASES = [(1, 16, 1280, 640, 1280, 2, 0, "bf16", "bf16", True), (1, 1, 16, 16, 8, 1, 0, "f32", "f32", False), (2, 4, 144, 48, 40, 4, 0, "bf16", "bf16", False),
         (7, 8, 320, 208, 328, 3, 8, "f32", "bf16", True), (33, 4, 640, 272, 264, 2, 0, "bf16", "f32", True), (64, 64, 512, 256, 512, 6, 3, "bf16", "bf16", True),
         (300, 3, 208, 144, 392, 2, 20, "bf16", "bf16", False), (520, 2, 128, 128, 128, 1, 100, "f32", "bf16", True), (257, 5, 400, 656, 520, 5, 0, "bf16", "bf16", True),
         (1000, 8, 256, 384, 256, 2, 4, "bf16", "bf16", True), (90, 256, 128, 64, 128, 8, 2, "bf16", "bf16", True),
         (1300, 2, 144, 272, 200, 1, 1, "bf16", "bf16", True), (2100, 4, 272, 144, 264, 2, 1, "f32", "f32", False), (4, 8, 272, 144, 72, 8, 0, "f32", "bf16", True), (3, 1024, 64, 32, 64, 64, 0, "bf16", "bf16", False)]


@pytest.mark.parametrize("T,E,K,I,N,k,skew,xt,yt,res", CASES)
def test_random(fb, T, E, K, I, N, k, skew, xt, yt, res):
    g = torch.Generator().manual_seed(T * 31 + E + K)
    ex = Experts(g, E, K, I, N)
    x = (torch.randn((T, K), generator=g) * (1 + 20 * (torch.rand((K,), generator=g) < 0.02))).to(T_[xt])
    ids, w = pick(g, T, E, k, skew)
    residual = torch.randn((T, N), generator=g).to(T_[yt]) if res else None
    y = call(fb, ex, x, ids, w, residual, T_[yt])
    want, tol = ex.want(x, ids, w, residual, T_[yt])
    err = (y.double().cpu() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    # the bound above holds every code's worst case; together the errors are as small as those of h in 8 bits with sums of that kind: 2^-7 of the result
    assert float(err.norm()) <= 2.0 ** -7 * float(want.norm())


def test_pairs_without_an_expert(fb):
    """Ids of -1 and experts without tokens; tokens with none: their residual; NaN weights of broken rows reach the output; nothing else moves."""
    g = torch.Generator().manual_seed(8)
    T, E, K, I, N, k = 70, 6, 144, 80, 136, 3
    ex = Experts(g, E, K, I, N)
    x = torch.randn((T, K), generator=g).bfloat16()
    ids, w = pick(g, T, E, k, 0)
    ids[torch.rand((T, k), generator=g) < 0.4] = -1
    ids[5], ids[6] = -1, -1
    w[6] = math.nan
    ids[ids == 2] = 3
    residual = torch.randn((T, N), generator=g).bfloat16()
    y = call(fb, ex, x, ids, w, residual, torch.bfloat16)
    assert bool(torch.isnan(y[6]).all()) and torch.equal(y[5].cpu(), residual[5])
    keep = [t for t in range(T) if t != 6]
    want, tol = ex.want(x[keep], ids[keep], w[keep], residual[keep], torch.bfloat16)
    assert bool(((y[keep].double().cpu() - want).abs() <= tol).all())


def test_rows_that_are_not_finite(fb):
    """A NaN or an infinity of a token stays in that token."""
    g = torch.Generator().manual_seed(12)
    T, E, K, I, N, k = 40, 4, 272, 144, 128, 2
    ex = Experts(g, E, K, I, N)
    x = torch.randn((T, K), generator=g)
    ids, w = pick(g, T, E, k, 0)
    clean = call(fb, ex, x, ids, w, None, torch.float32)
    x[3, 7], x[20, 271] = math.nan, math.inf
    y = call(fb, ex, x, ids, w, None, torch.float32)
    keep = [t for t in range(T) if t not in (3, 20)]
    assert bool(torch.isnan(y[[3, 20]]).all()) and torch.equal(y[keep], clean[keep])


def test_lists_that_do_not_fit(fb):
    """Offsets that do not ascend or leave the list, places out of range: skipped, nothing outside the buffers is touched and every other pair has its result."""
    g = torch.Generator().manual_seed(14)
    T, E, K, I, N, k = 50, 4, 128, 64, 64, 2
    ex = Experts(g, E, K, I, N)
    x = torch.randn((T, K), generator=g).bfloat16().to(DEV)
    ids, w = pick(g, T, E, k, 0)
    o, s = lists(ids, E)
    y = torch.zeros((T, N), dtype=torch.bfloat16, device=DEV)
    good = call(fb, ex, x.cpu(), ids, w, None, torch.bfloat16)
    s2 = s.clone()
    n1 = int(o[1])
    s2[0], s2[1] = -5, 10 ** 9                                                  # two pairs of expert 0 get lost: their tokens have no defined result
    for offsets, slots in ((o, s2), (o * 0 + 10 ** 9, s), (torch.flip(o, (0,)).contiguous(), s), (o - 10 ** 6, s)):
        a = fb.expert_mlp_args(x, ids.to(DEV), w.to(DEV), offsets, slots, *ex.dev, y)
        ws = torch.zeros(fb.fise_expert_mlp_workspace_bytes(a) + 4096, dtype=torch.uint8, device=DEV)
        ws[-4096:] = 0xA5
        fb.fise_expert_mlp(a, ws[:-4096])
        torch.cuda.synchronize()
        assert bool((ws[-4096:] == 0xA5).all())
        if slots is s2:
            lost = {int(s[0]) // k, int(s[1]) // k}
            keep = [t for t in range(T) if t not in lost]
            assert n1 >= 2 and torch.equal(y[keep], good[keep])


def test_strides_and_in_place(fb):
    g = torch.Generator().manual_seed(15)
    T, E, K, I, N, k = 30, 3, 144, 96, 72, 2
    ex = Experts(g, E, K, I, N)
    x = torch.randn((T, K + 8), generator=g).bfloat16()
    ids, w = pick(g, T, E, k, 0)
    room = torch.randn((T, N + 16), generator=g).bfloat16()
    y = room.to(DEV)
    o, s = lists(ids, E)
    a = fb.expert_mlp_args(x.to(DEV)[:, :K], ids.to(DEV), w.to(DEV), o, s, *ex.dev, y[:, :N], residual=y[:, :N])
    ws = torch.zeros(fb.fise_expert_mlp_workspace_bytes(a), dtype=torch.uint8, device=DEV)
    fb.fise_expert_mlp(a, ws)
    want, tol = ex.want(x[:, :K], ids, w, room[:, :N], torch.bfloat16)
    assert bool(((y[:, :N].double().cpu() - want).abs() <= tol).all()) and torch.equal(y[:, N:].cpu(), room[:, N:])


def test_no_tokens(fb):
    g = torch.Generator().manual_seed(16)
    ex = Experts(g, 2, 16, 16, 8)
    ids, w = torch.zeros((0, 1), dtype=torch.int32, device=DEV), torch.zeros((0, 1), device=DEV)
    a = fb.expert_mlp_args(torch.zeros((0, 16), device=DEV), ids, w, torch.zeros(3, dtype=torch.int32, device=DEV), ids.view(-1), *ex.dev, torch.zeros((0, 8), device=DEV))
    fb.fise_expert_mlp(a, torch.zeros(256, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("T,E,K,I,N,k", [(48, 16, 1024, 640, 512, 4), (400, 4, 640, 384, 264, 1), (1200, 2, 384, 256, 512, 1)])
def test_calls_between_other_kernels(fb, T, E, K, I, N, k):
    """The first call and calls behind other kernels, whose code and LDS contents are what the next one finds: all alike, and the definition's.  (Loads still under way when LDS gets its
    second use show only where a kernel's code is not in the caches yet.)"""
    g = torch.Generator().manual_seed(T)
    ex = Experts(g, E, K, I, N)
    x = torch.randn((T, K), generator=g).bfloat16()
    ids, w = pick(g, T, E, k, 0)
    o, s = lists(ids, E)
    y = [torch.full((T, N), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(6)]
    xd, idd, wd, ws = x.to(DEV), ids.to(DEV), w.to(DEV), None
    noise = torch.randn((1 << 20,), device=DEV)
    for i, out in enumerate(y):
        a = fb.expert_mlp_args(xd, idd, wd, o, s, *ex.dev, out)
        if ws is None:
            ws = torch.empty(fb.fise_expert_mlp_workspace_bytes(a), dtype=torch.uint8, device=DEV)
        ws.fill_(0xFF)
        fb.fise_expert_mlp(a, ws)
        for f in (torch.sort, torch.fft.rfft, torch.erfinv, torch.lgamma, lambda t: t.view(1024, 1024) @ t.view(1024, 1024), lambda t: t.view(-1, 16).softmax(1), lambda t: t.topk(50)):
            f(noise)
    want, tol = ex.want(x, ids, w, None, torch.bfloat16)
    assert bool(((y[0].double().cpu() - want).abs() <= tol).all())
    assert all(torch.equal(y[0], t) for t in y[1:])


@pytest.mark.parametrize("T", [2, 30, 700])
def test_an_expert_twice(fb, T):
    """A token that lists an expert twice gets it with both weights; weights of zero, negative and large ones."""
    g = torch.Generator().manual_seed(T)
    ex = Experts(g, 3, 144, 80, 72)
    x = torch.randn((T, 144), generator=g).bfloat16()
    ids = torch.randint(0, 3, (T, 1), generator=g).to(torch.int32).expand(T, 3).contiguous()
    w = torch.tensor([[0.0, -2.0, 1e4]]).expand(T, 3).contiguous()
    residual = torch.randn((T, 72), generator=g).bfloat16()
    y = call(fb, ex, x, ids, w, residual, torch.bfloat16)
    want, tol = ex.want(x, ids, w, residual, torch.bfloat16)
    assert bool(((y.double().cpu() - want).abs() <= tol).all())
