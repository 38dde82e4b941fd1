"""A captured step of group norm, replayed on other inputs, gives what the calls give."""
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kept", ["input", "codes"])
@pytest.mark.parametrize("n,hw,c,groups", [(4, 500, 96, 8), (1, 40, 64, 8), (2, 9, 4100, 4), (3, 9000, 64, 4)])
def test_other_inputs(n, hw, c, groups, kept):
    """Several samples and one; one launch and three; vectors kept and read again."""
    g = torch.Generator(device="cuda:0").manual_seed(hw)
    x = torch.randn(n, hw, c, device="cuda:0", generator=g).bfloat16()
    dy = (0.1 * torch.randn(n, hw, c, device="cuda:0", generator=g)).bfloat16()
    gamma, beta = 1 + 0.2 * torch.randn(c, device="cuda:0", generator=g), 0.2 * torch.randn(c, device="cuda:0", generator=g)
    d = eoq.gn_desc(n, hw, c, groups, eoq.EOQ_BF16, eoq.EOQ_ACT_SILU)

    def buffers():
        o = {"y": torch.empty_like(x), "dx": torch.empty_like(x), "stats": G.zeros((n, groups, 2), torch.float32), "dgamma": G.zeros(c, torch.float32),
             "dbeta": G.zeros(c, torch.float32), "ws": torch.full((eoq.eoq_gn_workspace_size(d),), 0xFF, dtype=torch.uint8, device="cuda:0")}
        if kept == "codes":
            o.update(codes=G.zeros((n, hw, c), torch.int8), exps=G.zeros((n * hw, -(-c // 32)), torch.uint8))
        return o

    def step(o):
        codes, exps = o.get("codes"), o.get("exps")
        eoq.eoq_gn_fwd(G.handle(), d, x, gamma, beta, o["y"], o["stats"], codes, exps, o["ws"])
        eoq.eoq_gn_bwd(G.handle(), d, dy, None, None if kept == "codes" else x, codes, exps, gamma, beta, o["stats"], o["dx"], o["dgamma"], o["dbeta"], o["ws"])

    captured = buffers()
    step(captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for _ in range(3):
        for t in (x, dy, gamma, beta):
            t.copy_(torch.randn(t.shape, device="cuda:0", generator=g) * 0.5 + 0.1)
        called = buffers()
        step(called)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in called:
            if k != "ws":
                assert torch.equal(captured[k], called[k]), k
