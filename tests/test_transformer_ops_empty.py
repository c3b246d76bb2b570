"""Empty selections through the binding: an edit that leaves no active token has tensors without elements, which have no address, and touches nothing.  No GPU needed."""
import pytest
import torch

from paper_2305_17423_amd import binding as fb

BF = torch.bfloat16


@pytest.mark.parametrize("dtype", [torch.float32, BF])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("residual", [False, True])
def test_product_of_no_rows(dtype, silu, residual):
    packed = torch.zeros(fb.fise_w4_bytes(48, 64, 32) + 256, dtype=torch.uint8)
    packed = packed[-packed.data_ptr() % 16:]
    x, y = torch.zeros((0, 64), dtype=dtype), torch.zeros((0, 48), dtype=dtype)
    fb.fise_w4_linear(fb.w4_linear_args(x, packed, 32, y, bias=torch.zeros(48), residual=torch.zeros_like(y) if residual else None, silu_in=silu), stream=0)


@pytest.mark.parametrize("kw", [dict(), dict(post="rms"), dict(post="layer", gate=True), dict(pre="layer", y=True, mod=True), dict(gate=True, pre="rms", y=True), dict(y=True, r=False)])
def test_norms_of_no_tiles(kw):
    big = torch.zeros(2 * 8 * 8 * 64 + 64)
    x = big[-big.data_ptr() % 16 // 4:][:2 * 8 * 8 * 64].view(2, 8, 8, 64)
    mod = x.view(-1)[:2 * 64].view(2, 64)
    rows = torch.full((2, 0, 64), 7.0)
    a = fb.gated_norm_args(x, h=rows, post=kw.get("post", "none"), gate=mod if kw.get("gate") else None, pre=kw.get("pre", "none"), mod_scale=mod if kw.get("mod") else None,
                           tile_idx=torch.zeros(0, dtype=torch.int32), n_active=0, tile=4, r=x if kw.get("r", True) else None, y=rows if kw.get("y") else None)
    fb.fise_masked_gated_norm(a, stream=0)


@pytest.mark.parametrize("form", [0, 1, 2])
@pytest.mark.parametrize("keys", [0, 30])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_of_no_queries(form, keys, causal):
    big = torch.zeros(65536, dtype=BF)
    at = lambda n: big[-big.data_ptr() % 16 // 2:][:n]
    q, out = torch.zeros((2, 0, 4, 48), dtype=BF), torch.zeros((2, 0, 96), dtype=BF)
    cache = at(2 * keys * 80).view(2, keys, 80) if keys else torch.zeros((2, 0, 80), dtype=BF)
    a = fb.latent_attention_args(q, cache, at(4 * 32 * 64).view(4, 32, 64), at(4 * 24 * 64).view(4, 24, 64), out, 0.2, causal=causal, form=form)
    need = fb.fise_latent_attention_workspace_bytes(a)
    assert need == 256
    fb.fise_latent_attention(a, None, stream=0)
    fb.fise_latent_attention(a, torch.zeros(need, dtype=torch.uint8), stream=0)


@pytest.mark.parametrize("form", [0, 1, 2])
def test_attention_over_an_empty_cache_is_taken(form):
    """Queries, but no token in the cache (its tensor has no address): the call needs a workspace as any other, and is not refused for the cache."""
    big = torch.zeros(65536, dtype=BF)
    at = lambda n: big[-big.data_ptr() % 16 // 2:][:n]
    a = fb.latent_attention_args(at(2 * 3 * 4 * 48).view(2, 3, 4, 48), torch.zeros((2, 0, 80), dtype=BF), at(4 * 32 * 64).view(4, 32, 64), at(4 * 24 * 64).view(4, 24, 64),
                                 at(2 * 3 * 96).view(2, 3, 96), 0.2, form=form)
    assert a.n_keys == 0 and a.cache_tokens == 0 and fb.fise_latent_attention_workspace_bytes(a) > 256
    with pytest.raises(fb.FiseError, match="null workspace"):
        fb.fise_latent_attention(a, None, stream=0)


def test_a_missing_buffer_is_still_refused():
    big = torch.zeros(65536, dtype=BF)
    at = lambda n: big[-big.data_ptr() % 16 // 2:][:n]
    q, out = torch.zeros((2, 0, 4, 48), dtype=BF), torch.zeros((2, 0, 96), dtype=BF)
    a = fb.latent_attention_args(q, at(2 * 30 * 80).view(2, 30, 80), at(4 * 32 * 64).view(4, 32, 64), at(4 * 24 * 64).view(4, 24, 64), out, 0.2)
    a.w_uk = None
    with pytest.raises(fb.FiseError, match="null pointer"):
        fb.fise_latent_attention(a, None, stream=0)
    with pytest.raises(ValueError):                                     # rows that do not fit the selection, empty or not
        fb.gated_norm_args(at(2 * 8 * 8 * 64).view(2, 8, 8, 64), h=torch.zeros((2, 0, 64), dtype=BF), n_active=1, tile=4)
