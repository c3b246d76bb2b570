"""GPU check of a transformer block of an edit that changes nothing: no active tile, so rows without elements for every operator, eager and captured; and of queries over a
cache that holds no token yet."""
import pytest
import torch

from helpers import DEV

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("dtype_mod", [torch.float32, BF])
def test_a_block_without_active_tiles(fb, dtype_mod):
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(s, generator=g).to(BF).to(DEV)
    B, size, tile, C, heads, d, dr, r, group = 2, 16, 4, 320, 8, 40, 32, 128, 64
    x, temb = rnd(B, size, size, C), rnd(B, 640).to(dtype_mod)

    def packed(N, K):
        p = torch.zeros(fb.fise_w4_bytes(N, K, group), dtype=torch.uint8, device=DEV)
        fb.fise_w4_pack(rnd(N, K), p, group)
        return p
    rows = lambda n: torch.empty((B, 0, n), dtype=BF, device=DEV)
    flat = lambda t: t.view(0, t.shape[-1])
    mod, r1, y_map, cache = torch.full((B, 3 * C), float("nan"), device=DEV), x.clone(), torch.zeros_like(x), rnd(B, size, size, r + dr)
    before = cache.clone()
    y1, q, att, o, y2 = rows(C), rows(heads * (d + dr)), rows(heads * d), rows(C), rows(C)
    m = [mod[:, i * C:(i + 1) * C] for i in range(3)]
    where = dict(tile_idx=torch.zeros(0, dtype=torch.int32, device=DEV), n_active=0, tile=tile)
    conv = fb.conv_args(y_map, rnd(r + dr, C), rnd(r + dr), where["tile_idx"], 0, tile, cache, ksize=1)
    lat = fb.latent_attention_args(q.view(B, 0, heads, d + dr), cache, rnd(heads, d, r), rnd(heads, d, r), att, 0.1)
    calls = [(fb.fise_w4_linear, fb.w4_linear_args(temb, packed(3 * C, 640), group, mod, silu_in=True)),
             (fb.fise_masked_gated_norm, fb.gated_norm_args(x, pre="layer", mod_scale=m[1], mod_shift=m[2], y=y_map, **where)),
             (fb.fise_masked_gated_norm, fb.gated_norm_args(x, pre="layer", mod_scale=m[1], mod_shift=m[2], y=y1, **where)),
             (fb.fise_masked_conv, conv, torch.empty(max(fb.fise_masked_conv_workspace_bytes(conv), 256), dtype=torch.uint8, device=DEV)),
             (fb.fise_w4_linear, fb.w4_linear_args(flat(y1), packed(heads * (d + dr), C), group, flat(q))),
             (fb.fise_latent_attention, lat, torch.empty(fb.fise_latent_attention_workspace_bytes(lat), dtype=torch.uint8, device=DEV)),
             (fb.fise_w4_linear, fb.w4_linear_args(flat(att), packed(C, heads * d), group, flat(o), residual=flat(y1))),
             (fb.fise_masked_gated_norm, fb.gated_norm_args(x, h=o, post="rms", gate=m[0], pre="rms", r=r1, y=y2, **where))]

    def run(stream=None):
        for call, *a in calls:
            call(*a, stream=stream)

    def untouched():
        torch.cuda.synchronize()
        return bool(mod.isfinite().all()) and all(torch.equal(a, b) for a, b in ((r1, x), (cache, before), (y_map, torch.zeros_like(x))))
    run()
    assert untouched()                                                         # (the conditioning does not depend on the mask)
    st, gr = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr, stream=st):
        run(st)
    for _ in range(2):
        mod.fill_(float("nan"))
        torch.cuda.synchronize()
        gr.replay()
        assert untouched()


@pytest.mark.parametrize("form", [0, 1, 2])
@pytest.mark.parametrize("M", [1, 200])
def test_queries_over_a_cache_without_tokens(fb, form, M):
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g).to(BF).to(DEV)
    out = torch.full((2, M, 3 * 64), float("nan"), dtype=BF, device=DEV)
    a = fb.latent_attention_args(rnd(2, M, 3, 96), torch.zeros((2, 0, 160), dtype=BF, device=DEV), rnd(3, 64, 128), rnd(3, 64, 128), out, 0.1, form=form)
    fb.fise_latent_attention(a, torch.full((fb.fise_latent_attention_workspace_bytes(a),), 0xFF, dtype=torch.uint8, device=DEV))
    assert bool((out == 0).all())
