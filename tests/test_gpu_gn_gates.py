"""Group norm: both passes have the same u and stand on the same side of an activation's gate."""
import numpy as np
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G

pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, eoq.EOQ_F32), "fp16": (torch.float16, eoq.EOQ_F16), "bf16": (torch.bfloat16, eoq.EOQ_BF16)}


def both_passes(x, dy, groups, name, act, kept, gamma=None, beta=None):
    """x, dy [n, hw, c] on the GPU"""
    n, hw, c = x.shape
    d = eoq.gn_desc(n, hw, c, groups, TYPES[name][1], act)
    ws = torch.full((eoq.eoq_gn_workspace_size(d),), 0xFF, dtype=torch.uint8, device="cuda:0")
    y, dx = torch.full_like(x, 33.0), torch.full_like(x, 33.0)
    stats, dgamma, dbeta = G.zeros((n, groups, 2), torch.float32), G.zeros(c, torch.float32), G.zeros(c, torch.float32)
    codes = G.zeros((n, hw, c), torch.int8) if kept == "codes" else None
    exps = G.zeros((n * hw, -(-c // 32)), torch.uint8) if kept == "codes" else None
    eoq.eoq_gn_fwd(G.handle(), d, x, gamma, beta, y, stats, codes, exps, ws)
    eoq.eoq_gn_bwd(G.handle(), d, dy, None, None if kept == "codes" else x, codes, exps, gamma, beta, stats, dx, dgamma, dbeta, ws)
    torch.cuda.synchronize()
    return y, dx, dgamma, dbeta


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("n,hw,c,groups", [(2, 30, 32, 4), (3, 1, 64, 64), (64, 1, 8, 8), (1, 4000, 48, 3), (2, 40, 35, 5), (2, 9, 4100, 4)])
def test_a_constant_group_lets_no_error_through(n, hw, c, groups, name):
    """Groups of equal values, and groups of one element: u is 0, so is ReLU's argument without beta, its gate is closed and every gradient 0."""
    rng = np.random.default_rng(n * 17 + hw + c)
    values = torch.from_numpy(rng.normal(0, 3, (n, 1, groups))).to(TYPES[name][0]).to("cuda:0")
    x = values.repeat_interleave(c // groups, 2).expand(n, hw, c).contiguous()
    dy = torch.from_numpy(rng.normal(size=(n, hw, c))).to(TYPES[name][0]).to("cuda:0")
    for out in both_passes(x, dy, groups, name, eoq.EOQ_ACT_RELU, "input"):
        assert not out.any()
    # the same from the 8-bit form, with values that it holds exactly: up to 127 eighths
    short = torch.from_numpy(rng.integers(-127, 128, (n, 1, groups)) / 8.0).to(TYPES[name][0]).to("cuda:0")
    x = short.repeat_interleave(c // groups, 2).expand(n, hw, c).contiguous()
    for out in both_passes(x, dy, groups, name, eoq.EOQ_ACT_RELU, "codes"):
        assert not out.any()


@pytest.mark.parametrize("n,hw,c,groups", [(3, 60, 64, 8), (2, 3000, 24, 3), (2, 30, 35, 5), (2, 9, 4100, 4)])
def test_the_gate_is_the_forward_passs(n, hw, c, groups):
    """Errors that are whole numbers, whose sums over the open gates are exact: dbeta counts just those pixels whose output is above zero.
    A third of the values stand at their group's mean, or a rounding away from it."""
    rng = np.random.default_rng(hw + c)
    centre = rng.normal(0, 2, (n, 1, groups)).astype(np.float32).repeat(c // groups, 2)
    away = rng.choice(np.array([-0.5, 0.0, 0.5], np.float32), (n, hw // 2, c))
    x = centre + np.concatenate([away, -away] + [0 * away[:, :1]] * (hw % 2), 1)
    x = torch.from_numpy(x.astype(np.float32)).to("cuda:0")
    dy = torch.from_numpy(rng.integers(-8, 9, (n, hw, c)).astype(np.float32)).to("cuda:0")
    gamma = G.dev(rng.normal(1, 0.3, c).astype(np.float32))
    y, _, _, dbeta = both_passes(x, dy, groups, "fp32", eoq.EOQ_ACT_RELU, "input", gamma)
    assert torch.equal(dbeta, (dy * (y > 0)).double().sum((0, 1)).float())
