"""Tensors that would make a kernel read or write outside of them are refused by the binding; no GPU needed."""
import pytest
import torch

from paper_2305_17423_amd import binding as fb


@pytest.mark.parametrize("B", [1, 2])
@pytest.mark.parametrize("name", ["gate", "mod_scale", "mod_shift"])
@pytest.mark.parametrize("shape", [(64,), (1, 60), (1, 1), (1, 128), (2, 60), (3, 64)])
def test_modulations_of_another_shape(B, name, shape):
    """One batch element too: its row is read whole, whatever the tensor holds."""
    x, y = torch.zeros((B, 4, 4, 64)), torch.zeros((B, 16, 64))
    with pytest.raises(ValueError):
        fb.gated_norm_args(x, h=y, y=y, r=x, **{name: torch.zeros(shape)})


@pytest.mark.parametrize("B", [1, 3])
def test_modulations_with_distant_columns(B):
    x, y = torch.zeros((B, 4, 4, 64)), torch.zeros((B, 16, 64))
    for bad in (torch.zeros((B, 128))[:, ::2], torch.zeros((64, max(B, 2))).t()[:B]):
        with pytest.raises(ValueError):
            fb.gated_norm_args(x, y=y, mod_scale=bad)


def test_modulations_that_fit():
    for B in (1, 2):
        x, y, mod = torch.zeros((B, 4, 4, 64)), torch.zeros((B, 16, 64)), torch.zeros((B, 192))
        assert fb.gated_norm_args(x, y=y, mod_scale=mod[:, :64], mod_shift=mod[:, 64:128]).mod_stride == (192 if B > 1 else 0)
        assert fb.gated_norm_args(x, y=y, mod_scale=mod[:1, :64].expand(B, 64), mod_shift=mod[:1, 64:128].expand(B, 64)).mod_stride == 0


def test_packed_weights_with_gaps():
    """Bytes that are counted but do not lie side by side: the packed weights are one block of memory."""
    need = fb.fise_w4_bytes(64, 256, 64)
    for packed in (torch.zeros(2 * need, dtype=torch.uint8)[::2], torch.zeros((16, need // 8), dtype=torch.uint8)[:, :need // 16]):
        assert packed.numel() >= need
        with pytest.raises(ValueError):
            fb.w4_linear_args(torch.zeros((3, 256)), packed, 64, torch.zeros((3, 64)))
        with pytest.raises(ValueError):
            fb.fise_w4_pack(torch.zeros((64, 256)), packed, 64, stream=0)
        with pytest.raises(ValueError):
            fb.fise_w4_unpack(packed, torch.zeros((64, 256)), 64, stream=0)


def test_workspaces_with_gaps():
    bf = dict(dtype=torch.bfloat16)
    q, c, wk, wv, out = (torch.zeros(s, **bf) for s in ((2, 3, 4, 48), (2, 5, 6, 80), (4, 32, 64), (4, 24, 64), (2, 3, 96)))
    a = fb.latent_attention_args(q, c, wk, wv, out, 0.2)
    with pytest.raises(ValueError):
        fb.fise_latent_attention(a, torch.zeros(2 * fb.fise_latent_attention_workspace_bytes(a), dtype=torch.uint8)[::2], stream=0)


@pytest.mark.parametrize("kw", [dict(tile_idx=torch.zeros(4, dtype=torch.int32)[::2])])
def test_lists_with_gaps(kw):
    x = torch.zeros((2, 8, 8, 64))
    with pytest.raises(ValueError):
        fb.gated_norm_args(x, r=x, n_active=2, tile=4, **kw)
