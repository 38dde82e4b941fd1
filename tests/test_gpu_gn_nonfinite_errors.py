"""Group norm backward with a NaN and infinities among the errors: they go where the formula takes them, and nowhere else."""
import numpy as np
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G

pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, eoq.EOQ_F32), "fp16": (torch.float16, eoq.EOQ_F16), "bf16": (torch.bfloat16, eoq.EOQ_BF16)}
ACTS = {"none": eoq.EOQ_ACT_NONE, "relu": eoq.EOQ_ACT_RELU, "silu": eoq.EOQ_ACT_SILU}


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("kind", sorted(ACTS))
@pytest.mark.parametrize("n,hw,c,groups,kept", [(3, 70, 64, 8, "input"), (3, 70, 64, 8, "codes"), (3, 5000, 64, 8, "codes"), (3, 70, 35, 5, "input"),
                                                (3, 70, 4100, 4, "input")])
def test_where_they_go(n, hw, c, groups, kept, kind, name):
    """Channel 1 and the last one lie under closed gates at the places that are hit, channel 2 under an open one."""
    td, ed = TYPES[name]
    rng = np.random.default_rng(c + hw)
    x = torch.from_numpy(rng.normal(size=(n, hw, c))).to(td).to("cuda:0")
    dy = torch.from_numpy(rng.normal(0, 0.1, (n, hw, c))).to(td).to("cuda:0")
    x[0, 11, 1], x[2, 69, c - 1], x[1, 5, 2] = -3.0, -3.0, 3.0
    d = eoq.gn_desc(n, hw, c, groups, ed, ACTS[kind])
    ws = G.empty(eoq.eoq_gn_workspace_size(d), torch.uint8)
    stats = G.zeros((n, groups, 2), torch.float32)
    codes = G.zeros((n, hw, c), torch.int8) if kept == "codes" else None
    exps = G.zeros((n * hw, -(-c // 32)), torch.uint8) if kept == "codes" else None
    eoq.eoq_gn_fwd(G.handle(), d, x, None, None, torch.empty_like(x), stats, codes, exps, ws)

    def backward(e):
        dx, dgamma, dbeta = torch.empty_like(x), G.zeros(c, torch.float32), G.zeros(c, torch.float32)
        eoq.eoq_gn_bwd(G.handle(), d, e, None, None if kept == "codes" else x, codes, exps, None, None, stats, dx, dgamma, dbeta, ws)
        torch.cuda.synchronize()
        return [t.double().cpu().numpy() for t in (dx, dgamma, dbeta)]

    clean = backward(dy)
    hit = dy.clone()
    hit[0, 11, 1], hit[2, 69, c - 1], hit[1, 5, 2] = float("nan"), float("inf"), float("-inf")
    dx, dgamma, dbeta = backward(hit)
    per = c // groups
    group = np.zeros((n, hw, c), bool)
    group[0, :, :per] = group[1, :, :per] = group[2, :, c - per:] = True
    assert not np.isfinite(dx[group]).any() and np.array_equal(dx[~group], clean[0][~group])
    others = [k for k in range(c) if k not in (1, 2, c - 1)]
    for got, was in ((dgamma, clean[1]), (dbeta, clean[2])):
        assert np.isnan(got[1]) and np.array_equal(got[others], was[others])
    # minus infinity with u > 0 under an open gate; under a closed one, 0 times infinity
    assert dbeta[2] == -np.inf and dgamma[2] == -np.inf
    # (the slope of SiLU at -3 is below zero, as u is)
    want = {"none": (np.inf, -np.inf), "silu": (-np.inf, np.inf)}.get(kind)
    assert (dbeta[c - 1], dgamma[c - 1]) == want if want else np.isnan([dbeta[c - 1], dgamma[c - 1]]).all()
    assert G.status_clear() == 0
