"""GPU check of a transformer block of an edit, made of the library's operators one behind the other: conditioning through 4-bit weights, norms with gate and modulation
at the active tokens, the latent cache refreshed there by the masked 1x1 convolution, attention of the active tokens over all latent vectors, output and
feed-forward products with 4-bit weights.

Tolerance, from arithmetic: a rounding to bf16 is 1.65e-3 of the value in the mean square.  The attention's branch goes through five of them (norm, latent vectors,
queries, output, product) and the attention's own 3.8e-3: sqrt(5 * 1.65^2 + 3.8^2) * 1e-3 = 5.3e-3.  The feed-forward branch has that, mixed with the
residual's, and four more with a SiLU that enlarges what goes in by at most 1.1: below 7e-3.  The sum x + both and its two roundings: at most sqrt(5.3^2 + 7^2 +
2 * 1.65^2) * 1e-3 = 9.1e-3 were the branches as large as the sum, held to 1e-2 of it in L2."""
import math

import pytest
import torch

from helpers import DEV, host, rel_l2

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


class Block:
    """Weights, caches and buffers of one block; run(stream) launches it, want() is the same in 64 bits."""

    def __init__(self, fb, seed, B, size, tile, active, C, heads, d, dr, r, group, kind):
        g = torch.Generator().manual_seed(seed)
        self.fb, self.dims, self.kind = fb, (B, size, tile, C, heads, d, dr, r), kind
        rnd = lambda *s, k=1.0: (k * torch.randn(s, generator=g)).to(BF).to(DEV)

        def packed(N, K):                                                     # weights and what they are once packed
            w = rnd(N, K, k=1 / math.sqrt(K))
            p = torch.zeros(fb.fise_w4_bytes(N, K, group), dtype=torch.uint8, device=DEV)
            back = torch.zeros((N, K), device=DEV)
            fb.fise_w4_pack(w, p, group)
            fb.fise_w4_unpack(p, back, group)
            return p, back.double().cpu()
        self.tiles = torch.randperm((size // tile) ** 2, generator=g)[:active].sort().values
        self.idx, self.M = self.tiles.to(torch.int32).to(DEV), active * tile * tile
        self.x = rnd(B, size, size, C)
        self.temb = torch.randn((B, 4 * C), generator=g).to(DEV)
        self.w_mod, self.w_q, self.w_o, self.w_up, self.w_down = packed(6 * C, 4 * C), packed(heads * (d + dr), C), packed(C, heads * d), packed(2 * C, C), packed(C, 2 * C)
        lat = packed(r + dr, C)
        self.w_lat = torch.zeros((r + dr, C), dtype=BF, device=DEV)           # for the convolution, which has many rows
        fb.fise_w4_unpack(lat[0], self.w_lat, group)
        self.b_lat, self.b_mod = rnd(r + dr, k=0.1), (0.1 * torch.randn(6 * C, generator=g)).to(DEV)
        self.w_uk, self.w_uv = rnd(heads, d, r, k=1 / math.sqrt(r)), rnd(heads, d, r, k=1 / math.sqrt(r))
        self.post_w = rnd(C)
        self.cache0 = rnd(B, size, size, r + dr)
        rows = lambda n: torch.full((B, self.M, n), float("nan"), dtype=BF, device=DEV)
        self.y_map, self.cache, self.r1, self.r2 = torch.zeros_like(self.x), self.cache0.clone(), self.x.clone(), self.x.clone()
        self.mod = torch.full((B, 6 * C), float("nan"), device=DEV)
        self.y1, self.q, self.att, self.o, self.y2, self.up, self.down = rows(C), rows(heads * (d + dr)), rows(heads * d), rows(C), rows(C), rows(2 * C), rows(C)
        flat = lambda t: t.view(B * self.M, -1)
        where = dict(tile_idx=self.idx, n_active=active, tile=tile)
        m = [self.mod[:, i * C:(i + 1) * C] for i in range(6)]
        first = dict(pre=kind, mod_scale=m[1], mod_shift=m[2], **where)
        self.calls = [
            (fb.fise_w4_linear, fb.w4_linear_args(self.temb, self.w_mod[0], group, self.mod, bias=self.b_mod, silu_in=True), False),
            (fb.fise_masked_gated_norm, fb.gated_norm_args(self.x, y=self.y_map, **first), False),
            (fb.fise_masked_gated_norm, fb.gated_norm_args(self.x, y=self.y1, **first), False),
            (fb.fise_masked_conv, fb.conv_args(self.y_map, self.w_lat, self.b_lat, self.idx, active, tile, self.cache, ksize=1), fb.fise_masked_conv_workspace_bytes),
            (fb.fise_w4_linear, fb.w4_linear_args(flat(self.y1), self.w_q[0], group, flat(self.q)), False),
            (fb.fise_latent_attention, fb.latent_attention_args(self.q.view(B, self.M, heads, d + dr), self.cache, self.w_uk, self.w_uv, self.att, 1 / math.sqrt(d + dr)),
             fb.fise_latent_attention_workspace_bytes),
            (fb.fise_w4_linear, fb.w4_linear_args(flat(self.att), self.w_o[0], group, flat(self.o)), False),
            (fb.fise_masked_gated_norm, fb.gated_norm_args(self.x, h=self.o, post="rms", post_w=self.post_w, gate=m[0], pre=kind, mod_scale=m[4], mod_shift=m[5], r=self.r1, y=self.y2,
                                                           **where), False),
            (fb.fise_w4_linear, fb.w4_linear_args(flat(self.y2), self.w_up[0], group, flat(self.up)), False),
            (fb.fise_w4_linear, fb.w4_linear_args(flat(self.up), self.w_down[0], group, flat(self.down), silu_in=True), False),
            (fb.fise_masked_gated_norm, fb.gated_norm_args(self.r1, h=self.down, gate=m[3], r=self.r2, **where), False)]
        self.ws = [torch.empty(max(bytes_(a), 256), dtype=torch.uint8, device=DEV) if bytes_ else None for _, a, bytes_ in self.calls]

    def run(self, stream=None):
        for (call, a, _), ws in zip(self.calls, self.ws):
            call(a, stream=stream) if ws is None else call(a, ws, stream=stream)

    def clear(self):
        for t in (self.mod, self.y1, self.q, self.att, self.o, self.y2, self.up, self.down):
            t.fill_(float("nan"))
        self.cache.copy_(self.cache0)
        self.r1.copy_(self.x)
        self.r2.copy_(self.x)

    def want(self):
        B, size, tile, C, heads, d, dr, r = self.dims
        f = lambda t: t.double().cpu()
        x, temb = f(self.x).reshape(B, -1, C), f(self.temb)
        a = torch.arange(tile)
        per = size // tile
        tok = torch.cat([(((t // per) * tile + a)[:, None] * size + (t % per) * tile + a[None]).reshape(-1) for t in self.tiles])
        m = ((temb * torch.sigmoid(temb)) @ self.w_mod[1].t() + f(self.b_mod)).view(B, 6, 1, C)

        def norm(v, kind):
            if kind == "layer":
                v = v - v.mean(-1, keepdim=True)
            return v / torch.sqrt((v ** 2).mean(-1, keepdim=True) + 1e-5)
        y1 = norm(x[:, tok], self.kind) * (1 + m[:, 1]) + m[:, 2]
        cache = f(self.cache0).reshape(B, -1, r + dr).clone()
        cache[:, tok] = y1 @ f(self.w_lat).t() + f(self.b_lat)
        q = (y1 @ self.w_q[1].t()).view(B, -1, heads, d + dr)
        k, v = torch.einsum("bjr,hdr->bhjd", cache[..., :r], f(self.w_uk)), torch.einsum("bjr,hdr->bhjd", cache[..., :r], f(self.w_uv))
        s = torch.einsum("bmhd,bhjd->bhmj", q[..., :d], k) + torch.einsum("bmhd,bjd->bhmj", q[..., d:], cache[..., r:])
        att = torch.einsum("bhmj,bhjd->bmhd", torch.softmax(s / math.sqrt(d + dr), -1), v).reshape(B, -1, heads * d)
        r1 = x[:, tok] + m[:, 0] * norm(att @ self.w_o[1].t(), "rms") * f(self.post_w)
        up = (norm(r1, self.kind) * (1 + m[:, 4]) + m[:, 5]) @ self.w_up[1].t()
        out = x.clone()
        out[:, tok] = r1 + m[:, 3] * ((up * torch.sigmoid(up)) @ self.w_down[1].t())
        return tok, out.view(self.x.shape), cache.view(self.cache.shape)


SIZES = [(1, 2, 32, 4, 6, 320, 8, 40, 32, 128, 64, "layer"), (2, 1, 16, 4, 1, 640, 8, 80, 64, 256, 128, "rms"), (3, 3, 8, 2, 16, 1280, 16, 128, 64, 512, 32, "layer")]


@pytest.mark.parametrize("args", SIZES)
def test_a_block_of_an_edit(fb, args):
    b = Block(fb, *args)
    b.run()
    tok, out, cache = b.want()
    C, width = out.shape[-1], cache.shape[-1]
    active = lambda t, n: t.reshape(t.shape[0], -1, n)[:, tok]
    assert rel_l2(host(active(b.r2.cpu(), C)), active(out, C).numpy()) <= 1e-2
    assert rel_l2(host(active(b.cache.cpu(), width)), active(cache, width).numpy()) <= 1e-2
    rest = torch.ones(b.dims[1] ** 2, dtype=torch.bool)
    rest[tok] = False
    for now, before, n in ((b.r2, b.x, C), (b.r1, b.x, C), (b.cache, b.cache0, width)):            # rows that are not active keep their value
        assert torch.equal(now.cpu().reshape(now.shape[0], -1, n)[:, rest], before.cpu().reshape(now.shape[0], -1, n)[:, rest])


def test_two_blocks_captured_and_replayed_beside_eager_calls(fb):
    blocks = [Block(fb, *a) for a in SIZES[:2]]
    want = []
    for b in blocks:
        b.run()
        want.append((b.r2.clone(), b.cache.clone()))
        b.clear()
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in blocks]
    for b, st in zip(blocks, streams):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=st):
            b.run(st)
        graphs.append(gr)
    other = Block(fb, *SIZES[2])
    other.run()
    third = other.r2.clone()
    for rep in range(3):
        for b in blocks + [other]:
            b.clear()
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        other.run()
        torch.cuda.synchronize()
        for b, (r2, cache) in zip(blocks, want):
            assert torch.equal(b.r2, r2) and torch.equal(b.cache, cache), rep
        assert torch.equal(other.r2, third), rep
