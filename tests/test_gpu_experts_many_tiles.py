"""GPU check of the experts' products with more tiles than one launch holds: 2^24 pairs of 8336 channels, rows of 139 GB in 8 bits, held to the definition at tokens of the first and the last
launch and between."""
import pytest
import torch

from helpers import DEV
from test_gpu_experts import Experts
from test_gpu_experts_sums import want

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def test_more_tiles_than_a_launch_holds(fb):
    T, E, K, I, N, k = (1 << 18) - 1, 2, 16, 8336, 8, 64
    g = torch.Generator().manual_seed(3)
    ex = Experts(g, E, K, I, N)
    x = torch.randn((T, K), generator=g).bfloat16()
    ids = torch.arange(k, dtype=torch.int32).remainder(E).expand(T, k).contiguous()                    # every token has each expert k / 2 times
    weight = torch.full((T, k), 1.0 / k)
    slots = torch.cat([torch.arange(T * k, dtype=torch.int32).view(T, k)[:, e::E].reshape(-1) for e in range(E)])
    offsets = torch.tensor([0, T * k // 2, T * k], dtype=torch.int32)
    y = torch.full((T, N), 3.0, dtype=torch.bfloat16, device=DEV)
    a = fb.expert_mlp_args(x.to(DEV), ids.to(DEV), weight.to(DEV), offsets.to(DEV), slots.to(DEV), *ex.dev, y)
    need = fb.fise_expert_mlp_workspace_bytes(a)
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip(f"{need >> 30} GiB of workspace are not free")
    assert T * k // 128 * -(-I // 128) > 1 << 23
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    fb.fise_expert_mlp(a, ws)
    assert bool(torch.isfinite(y).all())
    some = torch.cat([torch.arange(n, n + 64) for n in (0, T // 4, T // 2, T - 64)])
    # (the sums' tolerance by the pairs of the call, as documented: those of the tokens that are looked at are fewer)
    ref, tol = want(ex, x[some], ids[some], weight[some], None, torch.bfloat16)
    err = (y[some.to(DEV)].double().cpu() - ref).abs()
    assert T * k >= 512 * E and some.numel() * k >= 512 * E and bool((err <= tol).all()), float((err / tol).max())
    del ws
    torch.cuda.empty_cache()
