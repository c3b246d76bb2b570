"""GPU check of routing and experts of many pairs (tables for tiles of two heights, sums of all scores) in a captured graph, replayed with eager calls of the same kernels between: the bits of
the eager calls, with logits and rows that change from replay to replay."""
import pytest
import torch

from helpers import DEV
from test_gpu_experts import Experts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fb():
    from paper_2305_17423_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


class Step:
    def __init__(self, fb, ex, T, k, y_type):
        E, K, I, N = ex.dims
        self.fb, new = fb, lambda *s, type=torch.float32: torch.zeros(s, dtype=type, device=DEV)
        self.logits, self.x, self.y = new(T, E), new(T, K, type=torch.bfloat16), new(T, N, type=y_type)
        self.ids, self.weights, self.offsets, self.slots = new(T, k, type=torch.int32), new(T, k), new(E + 1, type=torch.int32), new(T * k, type=torch.int32)
        self.route = fb.route_args(self.logits, self.ids, self.weights, self.offsets, self.slots, renormalize=False, scale=2.0)
        self.experts = fb.expert_mlp_args(self.x, self.ids, self.weights, self.offsets, self.slots, *ex.dev, self.y)
        self.ws = [new(max(n, 256), type=torch.uint8) for n in (fb.fise_route_experts_workspace_bytes(self.route), fb.fise_expert_mlp_workspace_bytes(self.experts))]

    def run(self, stream=None):
        self.fb.fise_route_experts(self.route, self.ws[0], stream=stream)
        self.fb.fise_expert_mlp(self.experts, self.ws[1], stream=stream)

    def outputs(self):
        return [t.clone() for t in (self.ids, self.weights, self.offsets, self.slots, self.y)]


@pytest.mark.parametrize("T,E,k,yt", [(1200, 2, 1, torch.bfloat16), (1100, 4, 2, torch.bfloat16), (1100, 4, 2, torch.float32), (300, 4, 2, torch.bfloat16)])
def test_captured_and_replayed(fb, T, E, k, yt):
    g = torch.Generator(device=DEV).manual_seed(T)
    ex = Experts(torch.Generator().manual_seed(T), E, 272, 144, 136)
    captured, eager = Step(fb, ex, T, k, yt), Step(fb, ex, T, k, yt)
    eager.run()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        captured.run(stream)
    for i in range(5):
        logits, x = torch.randn((T, E), generator=g, device=DEV), torch.randn((T, 272), generator=g, device=DEV).bfloat16()
        for s in (captured, eager):
            s.logits.copy_(logits)
            s.x.copy_(x)
            for w in s.ws:
                w.fill_(0xFF if i % 2 else 0x7F)
        torch.cuda.synchronize()
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured.outputs(), eager.outputs())), i
        assert int(eager.offsets[-1]) == T * k and bool(torch.isfinite(eager.y).all()) and bool(eager.y.any())
