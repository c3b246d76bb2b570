"""GPU checks of offsets past 32 bits: rows, weights and results of more than 2^32 bytes, held to the definition at their far end; many rows in 8 bits."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_experts import HALF, lists
from test_gpu_fp8 import blocks, check, in_eight, weights, wide
from test_gpu_rotary import close, turn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def test_rotary_of_many_rows(fb):
    M, heads, d = 1100000, 16, 128
    x = torch.empty((1, M, heads, d), dtype=BF, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    x[:, -300:].normal_(generator=g)
    y = torch.zeros_like(x)
    pos = torch.arange(M, dtype=torch.int32, device=DEV).view(1, M, 1)
    fb.fise_rotary(fb.rotary_args([fb.rotary_tensor(x, y)], [d], 10000.0, pos=pos))
    close(y[:, -300:], *turn(x[:, -300:].double().cpu(), pos[:, -300:].double().cpu(), 0, [d], [10000.0], "adjacent", False, False, [0]))


@pytest.mark.parametrize("M,N,type", [(70000, 16400, torch.float32), (270000, 8200, BF)])
def test_product_of_many_results(fb, M, N, type):
    K = 144
    g = torch.Generator().manual_seed(2)
    q, s = weights(g, N, K)
    x = torch.zeros((M, K), device=DEV)
    x[-200:] = torch.randn((200, K), generator=g).to(DEV)
    y = torch.empty((M, N), dtype=type, device=DEV)
    a = fb.fp8_linear_args(x, q.to(DEV), s.to(DEV), y)
    fb.fise_fp8_linear(a, torch.empty(fb.fise_fp8_linear_workspace_bytes(a), dtype=torch.uint8, device=DEV))
    c, e = in_eight(x[-200:].cpu(), 1)
    v, w = c * torch.exp2(e).repeat_interleave(128, 1)[:, :K], wide(q, s)
    check(y[-200:], v @ w.t(), v.abs() @ w.abs().t(), K)
    assert not bool(y[:-200].any())


@pytest.mark.parametrize("rows", [1, 128])
def test_many_values_into_eight_bits(fb, rows):
    M, K = 1100000, 2048
    x = torch.zeros((M, K), dtype=BF, device=DEV)
    g = torch.Generator().manual_seed(3)
    x[-256:] = torch.randn((256, K), generator=g).to(BF).to(DEV)
    codes = torch.empty((M, K), dtype=torch.uint8, device=DEV)
    scale = torch.empty((blocks(K), M) if rows == 1 else (blocks(M), blocks(K)), device=DEV)
    fb.fise_fp8_quantize(x, codes, scale, block_rows=rows)
    first = M - M % 128 - 128 if rows == 128 else M - 256                      # whole blocks
    want, e = in_eight(x[first:].cpu(), rows)
    assert torch.equal(codes[first:].cpu().view(torch.float8_e4m3fn).double(), want)
    assert torch.equal((scale[:, first:].t() if rows == 1 else scale[first // 128:]).cpu().double(), torch.exp2(e))
    assert not bool(codes[:-256].any())


def test_large_experts(fb):
    """Weights of 4 GB, the last expert's behind 2^32 bytes: the definition in 64 bits for a few outputs of each token.  Tolerance as in the tests of the experts, with h's codes as they may be."""
    E, K, I, N, k = 5, 16384, 16384, 16384, 1
    g = torch.Generator(device=DEV).manual_seed(5)
    w_in, w_out = (torch.randint(0x20, 0x40, s, dtype=torch.uint8, device=DEV, generator=g) for s in ((E, 2, I, K), (E, N, I)))      # values from 1 / 8 to just under 2 ...
    for w in (w_in, w_out):
        w[..., ::2] |= 0x80                                                   # ... of both signs
    s_in, s_out = torch.full((E, 2, blocks(I), blocks(K)), 1 / 64.0, device=DEV), torch.full((E, blocks(N), blocks(I)), 1 / 64.0, device=DEV)
    for T in (3, 40):
        x = torch.randn((T, K), device=DEV, generator=g).to(BF)
        ids, wt = torch.full((T, 1), E - 1, dtype=torch.int32), torch.ones((T, 1))
        o, sl = lists(ids, E)
        y = torch.empty((T, N), device=DEV)
        a = fb.expert_mlp_args(x, ids.to(DEV), wt.to(DEV), o, sl, w_in, s_in, w_out, s_out, y)
        fb.fise_expert_mlp(a, torch.empty(fb.fise_expert_mlp_workspace_bytes(a), dtype=torch.uint8, device=DEV))
        c, e = in_eight(x.cpu(), 1)
        v = (c * torch.exp2(e).repeat_interleave(128, 1)).to(DEV)
        dec = lambda t: t.view(torch.float8_e4m3fn).float().double() / 64.0
        gate, up = (torch.cat([v @ dec(w_in[E - 1, j, i:i + 2048]).t() for i in range(0, I, 2048)], 1) for j in (0, 1))
        mag = [torch.cat([v.abs() @ dec(w_in[E - 1, j, i:i + 2048]).abs().t() for i in range(0, I, 2048)], 1) for j in (0, 1)]
        d = 2 * (128 + 3 * K / 128 + 4) * 2.0 ** -24                           # (float sums: fewer than 512 pairs an expert)
        h = gate * torch.sigmoid(gate) * up
        dh = 1.1 * d * mag[0] * (up.abs() + d * mag[1]) + (gate * torch.sigmoid(gate)).abs() * d * mag[1] + 2.0 ** -20 * h.abs()
        eight = lambda t: (lambda q: q[0] * torch.exp2(q[1]).repeat_interleave(128, 1))(in_eight(t.cpu(), 1)).to(DEV)
        hq = eight(h)
        # a code is at most one step off where h +- dh rounds elsewhere: a step is at most 2^-3 of the value, or 2^-9 of its block's scale
        scale = torch.exp2(in_eight(h.cpu(), 1)[1]).repeat_interleave(128, 1).to(DEV)
        unsure = (eight(h + dh) != hq) | (eight(h - dh) != hq)
        off = torch.where(unsure, hq.abs() / 8 + scale * 2.0 ** -8, torch.zeros((), dtype=torch.float64, device=DEV))
        cols = torch.cat((torch.arange(200), torch.arange(N - 200, N))).to(DEV)
        w = dec(w_out[E - 1][cols])
        want, tol = hq @ w.t(), off @ w.abs().t() + d * (hq.abs() @ w.abs().t())
        tol = tol + HALF[torch.float32] * want.abs()
        err = (y[:, cols].double() - want).abs()
        assert bool((err <= tol).all()), (T, float((err / tol).max()))
