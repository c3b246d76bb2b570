"""GPU checks of the form for a few tokens where the chosen expert's weights lie behind 2^32 bytes: codes of 8.6 GB on both sides, of which all but that expert's are NaN."""
import pytest
import torch

from helpers import DEV
from test_gpu_experts import lists
from test_gpu_experts_sums import T_, want
from test_gpu_fp8 import blocks, weights, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


class One:
    """What the definition needs of a set of experts of which one is used."""

    def __init__(self, dims, expert, ins, outs):
        self.dims, self.ins, self.outs = dims, {expert: ins}, {expert: outs}


@pytest.mark.parametrize("xt,yt", [("bf16", "f32"), ("f32", "bf16")])
def test_last_expert_of_many(fb, xt, yt):
    E, K, I, N, k = 1024, 4096, 1024, 8192, 1
    g = torch.Generator().manual_seed(7)
    ins, out = [weights(g, I, K) for _ in range(2)], weights(g, N, I)
    w_in, w_out = (torch.full(s, 0x7f, dtype=torch.uint8, device=DEV) for s in ((E, 2, I, K), (E, N, I)))
    s_in, s_out = torch.ones((E, 2, blocks(I), blocks(K)), device=DEV), torch.ones((E, blocks(N), blocks(I)), device=DEV)
    for e in (E - 1, 600):                                                     # both behind 2^32 bytes
        for j, (q, s) in enumerate(ins):
            w_in[e, j], s_in[e, j] = q.view(torch.uint8).to(DEV), s.to(DEV)
        w_out[e], s_out[e] = out[0].view(torch.uint8).to(DEV), out[1].to(DEV)
        for T in (1, 3):
            x = torch.randn((T, K), generator=g).to(T_[xt])
            ids, w = torch.full((T, k), e, dtype=torch.int32), torch.rand((T, k), generator=g) + 0.5
            o, sl = lists(ids, E)
            y = torch.empty((T, N), dtype=T_[yt], device=DEV)
            a = fb.expert_mlp_args(x.to(DEV), ids.to(DEV), w.to(DEV), o, sl, w_in, s_in, w_out, s_out, y)
            need = fb.fise_expert_mlp_workspace_bytes(a)
            assert need == -(-T * k * I * 4 // 256) * 256                      # h in float and nothing else: the form for a few tokens
            fb.fise_expert_mlp(a, torch.empty(need, dtype=torch.uint8, device=DEV))
            used = One((E, K, I, N), e, [wide(*p).to(DEV) for p in ins], wide(*out).to(DEV))
            ref, tol = want(used, x, ids, w, None, T_[yt])
            err = (y.double().cpu() - ref).abs()
            assert bool((err <= tol).all()), (e, T, float((err / tol).max()))
