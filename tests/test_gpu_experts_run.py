"""GPU check of a transformer block with experts, made of the library's operators one behind the other: norm with modulation at the active tokens, queries and latent vectors by 8-bit products,
rotary positions (the latent vectors go into their map in that call), attention over the latent vectors, output product, gated norm, routing, the experts' feed-forward, gated norm.

Each of the operators here is held, on the inputs that the ones before it left on the device, to the definition and the tolerance of its own test; the block's other
operators have theirs.  What a chain adds is how they are put together: where rows go, what stays as it was, that a captured block does the same as an eager one."""
import math

import pytest
import torch

from helpers import DEV
from test_gpu_experts import Experts
from test_gpu_fp8 import blocks, check as check_product, in_eight, weights, wide
from test_gpu_rotary import close, places, tile_tokens, turn
from test_gpu_route import define

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


class Block:
    """Weights, caches and buffers of one block; run(stream) launches it."""

    def __init__(self, fb, seed, B, size, tile, active, C, heads, d, dr, r, E, k, I):
        g = torch.Generator().manual_seed(seed)
        self.fb, self.dims = fb, (B, size, tile, C, heads, d, dr, r, E, k, I)
        rnd = lambda *s, std=1.0: (std * torch.randn(s, generator=g)).to(BF).to(DEV)
        self.tiles = torch.randperm((size // tile) ** 2, generator=g)[:active].sort().values.tolist()
        idx, M = torch.tensor(self.tiles, dtype=torch.int32, device=DEV), active * tile * tile
        where = dict(tile_idx=idx, n_active=active, tile=tile)
        self.x, self.mod = rnd(B, size, size, C), (0.3 * torch.randn((B, 6 * C), generator=g)).to(DEV)
        m = [self.mod[:, i * C:(i + 1) * C] for i in range(6)]
        self.w = {n: weights(g, *s) for n, s in dict(q=(heads * (d + dr), C), lat=(r + dr, C), o=(C, heads * d), gate=(E, C)).items()}
        w = {n: (q.to(DEV), s.to(DEV)) for n, (q, s) in self.w.items()}
        self.bias = 0.1 * torch.randn((E,), generator=g)
        self.experts = Experts(g, E, C, I, C)
        self.cache0, w_uk, w_uv, self.post_w = rnd(B, size, size, r + dr), rnd(heads, d, r, std=1 / math.sqrt(r)), rnd(heads, d, r, std=1 / math.sqrt(r)), rnd(C)
        rows = lambda *s, type=BF: torch.empty((B, M, *s), dtype=type, device=DEV)
        self.y1, self.q0, self.q, self.lat, self.att, self.o, self.y2, self.logits, self.h = (rows(C), rows(heads, d + dr), rows(heads, d + dr), rows(1, r + dr), rows(heads * d), rows(C), rows(C),
                                                                                            rows(E, type=torch.float32), rows(C))
        self.ids, self.weight = rows(k, type=torch.int32), rows(k, type=torch.float32)
        self.offsets, self.slots = torch.empty(E + 1, dtype=torch.int32, device=DEV), torch.empty(B * M * k, dtype=torch.int32, device=DEV)
        self.cache, self.r1, self.r2 = self.cache0.clone(), self.x.clone(), self.x.clone()
        flat = lambda t: t.view(B * M, -1)
        bias = self.bias.to(DEV)
        ids, weight = flat(self.ids), flat(self.weight)
        self.theta, self.axes = [100.0, 30.0], [dr // 2, dr // 2]
        self.calls = [
            (fb.fise_masked_gated_norm, fb.gated_norm_args(self.x, y=self.y1, pre="rms", mod_scale=m[1], mod_shift=m[2], **where), None),
            (fb.fise_fp8_linear, fb.fp8_linear_args(flat(self.y1), *w["q"], flat(self.q0)), fb.fise_fp8_linear_workspace_bytes),
            (fb.fise_fp8_linear, fb.fp8_linear_args(flat(self.y1), *w["lat"], flat(self.lat)), fb.fise_fp8_linear_workspace_bytes),
            (fb.fise_rotary, fb.rotary_args([fb.rotary_tensor(self.q0, self.q, d), fb.rotary_tensor(self.lat, self.cache.view(B, size * size, 1, r + dr), r, y_is_map=True)], self.axes, self.theta,
                                            grid=(1, size, size), pairing="axis_halves", **where), None),
            (fb.fise_latent_attention, fb.latent_attention_args(self.q, self.cache, w_uk, w_uv, self.att, 1 / math.sqrt(d + dr)), fb.fise_latent_attention_workspace_bytes),
            (fb.fise_fp8_linear, fb.fp8_linear_args(flat(self.att), *w["o"], flat(self.o)), fb.fise_fp8_linear_workspace_bytes),
            (fb.fise_masked_gated_norm, fb.gated_norm_args(self.x, h=self.o, post="rms", post_w=self.post_w, gate=m[0], pre="rms", mod_scale=m[4], mod_shift=m[5], r=self.r1, y=self.y2, **where), None),
            (fb.fise_fp8_linear, fb.fp8_linear_args(flat(self.y2), *w["gate"], flat(self.logits)), fb.fise_fp8_linear_workspace_bytes),
            (fb.fise_route_experts, fb.route_args(flat(self.logits), ids, weight, self.offsets, self.slots, score="sigmoid", bias=bias, groups=2, top_groups=1, group_top=2, scale=1.5),
             fb.fise_route_experts_workspace_bytes),
            (fb.fise_expert_mlp, fb.expert_mlp_args(flat(self.y2), ids, weight, self.offsets, self.slots, *self.experts.dev, flat(self.h)), fb.fise_expert_mlp_workspace_bytes),
            (fb.fise_masked_gated_norm, fb.gated_norm_args(self.r1, h=self.h, gate=m[3], r=self.r2, **where), None)]
        self.ws = [torch.empty(max(size_(a), 256), dtype=torch.uint8, device=DEV) if size_ else None for _, a, size_ in self.calls]

    def run(self, stream=None):
        for (call, a, _), ws in zip(self.calls, self.ws):
            call(a, stream=stream) if ws is None else call(a, ws, stream=stream)

    def outputs(self):
        return [self.q, self.cache, self.ids, self.weight, self.offsets, self.slots, self.h, self.r1, self.r2]

    def clear(self):
        for t in (self.y1, self.q0, self.q, self.lat, self.att, self.o, self.y2, self.logits, self.h, self.weight):
            t.fill_(float("nan"))
        for t in (self.ids, self.offsets, self.slots, *(w for w in self.ws if w is not None)):
            t.fill_(113)
        self.cache.copy_(self.cache0)
        self.r1.copy_(self.x)
        self.r2.copy_(self.x)


SIZES = [(1, 2, 16, 4, 5, 320, 8, 40, 32, 128, 16, 2, 640), (2, 1, 16, 4, 1, 640, 8, 80, 64, 256, 8, 4, 336), (3, 2, 8, 2, 16, 256, 4, 64, 32, 128, 32, 6, 128), (4, 1, 4, 1, 2, 128, 2, 32, 16, 64, 4, 2, 144)]


@pytest.mark.parametrize("args", SIZES)
def test_a_block_with_experts(fb, args):
    b = Block(fb, *args)
    b.clear()
    b.run()
    B, size, tile, C, heads, d, dr, r, E, k, I = b.dims
    tok = tile_tokens(b.tiles, (1, size, size), tile)
    host = lambda t: t.reshape(-1, t.shape[-1]).cpu()

    def product(x, name, y):
        c, e = in_eight(host(x), 1)
        v, w = c * torch.exp2(e).repeat_interleave(128, 1)[:, :x.shape[-1]], wide(*b.w[name])
        check_product(y.view(-1, w.shape[0]), v @ w.t(), v.abs() @ w.abs().t(), x.shape[-1])
    product(b.y1, "q", b.q0.view(B, -1, heads * (d + dr)))
    product(b.y1, "lat", b.lat.view(B, -1, r + dr))
    product(b.att, "o", b.o)
    product(b.y2, "gate", b.logits)
    pos = places((1, size, size), 2, tok)[None]
    close(b.q, *turn(b.q0.double().cpu(), pos, d, b.axes, b.theta, "axis_halves", False, False, [0, 0]))
    cache = b.cache.view(B, size * size, r + dr)
    want, mag = turn(b.lat.double().cpu(), pos, r, b.axes, b.theta, "axis_halves", False, False, [0, 0])
    close(cache[:, tok], want[:, :, 0], mag[:, :, 0])
    ids, weight, offsets, slots = define(host(b.logits), b.bias, k, "sigmoid", 2, 1, 2, True, 1.5)
    assert torch.equal(host(b.ids), ids) and torch.equal(b.offsets.cpu(), offsets) and torch.equal(b.slots.cpu()[:int(offsets[-1])], slots)
    want, tol = b.experts.want(host(b.y2), host(b.ids), host(b.weight), None, BF)
    assert bool(((host(b.h).double() - want).abs() <= tol).all())
    rest = torch.ones(size * size, dtype=torch.bool)
    rest[tok] = False
    for now, before, n in ((b.r2, b.x, C), (b.r1, b.x, C), (b.cache, b.cache0, r + dr)):            # rows that are not active keep their value
        assert torch.equal(now.cpu().reshape(B, -1, n)[:, rest], before.cpu().reshape(B, -1, n)[:, rest])
    assert bool(torch.isfinite(b.r2).all())


def test_blocks_captured_and_replayed_beside_eager_calls(fb):
    """Two captured blocks replayed on streams of their own, a third launched beside them, several times: the same bits as alone."""
    made = [Block(fb, *a) for a in SIZES[:3]]
    want = []
    for b in made:
        b.clear()
        b.run()
        want.append([t.clone() for t in b.outputs()])
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in made[:2]]
    for b, st in zip(made, streams):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            b.run(st)
        graphs.append(gr)
    for rep in range(3):
        for b in made:
            b.clear()
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        made[2].run()
        torch.cuda.synchronize()
        for b, w in zip(made, want):
            for now, then in zip(b.outputs(), w):
                n = int(b.offsets[-1]) if now is b.slots else now.numel()
                assert torch.equal(now.view(-1)[:n], then.view(-1)[:n]), rep
