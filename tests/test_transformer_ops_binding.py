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
