"""Group norm over many pixels, and over many samples: what one sum of fp32 numbers would lose."""
import numpy as np
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G

pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, eoq.EOQ_F32, 2.0 ** -24), "bf16": (torch.bfloat16, eoq.EOQ_BF16, 2.0 ** -8)}
EPS32 = 2.0 ** -24


@pytest.mark.parametrize("errors", [(0.1, 0.1), (0.15, 0.05)])
@pytest.mark.parametrize("name,n,hw,c,groups", [("fp32", 1, 1 << 18, 64, 1), ("fp32", 1, 1 << 20, 32, 4), ("bf16", 3, 1 << 20, 8, 8), ("bf16", 200, 4096, 2056, 1),
                                                ("fp32", 1 << 18, 4, 32, 8)])
def test_equal_errors_over_every_pixel(name, n, hw, c, groups, errors):
    """Errors as an average over all pixels leaves them, one value or two: the roundings of a sum of equal terms all go one way.  x is +-a, as
    often one as the other in every sample, so that mean 0, variance a^2 and all sums are known.

    A sum of k terms in a row is off by k / 2 roundings of itself.  A thread's vectors, 4,096 at most in these cases, go in two steps of 64 terms:
    64 roundings; a block's threads in steps of 32 and 8: 20; a cluster's eight blocks: 4; samples 16 and 9, what is more in 64 bits.  A product
    and u add 6.  Room: 128."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free device memory")
    td, ed, half = TYPES[name]
    g = torch.Generator(device="cuda:0").manual_seed(c + hw)
    signs = torch.ones(n, hw, 1, device="cuda:0")
    order = torch.rand(n, hw, device="cuda:0", generator=g).argsort(1)
    signs.view(n, hw).scatter_(1, order[:, hw // 2:], -1.0)
    a, up, down = (float(torch.tensor(v).to(td)) for v in (0.7, *errors))
    x = (a * signs).to(td).expand(n, hw, c).contiguous()
    dy = torch.where(signs > 0, up, down).to(td).expand(n, hw, c).contiguous()
    d = eoq.gn_desc(n, hw, c, groups, ed, eoq.EOQ_ACT_NONE)
    ws = G.empty(eoq.eoq_gn_workspace_size(d), torch.uint8)
    stats, dgamma, dbeta = G.zeros((n, groups, 2), torch.float32), G.zeros(c, torch.float32), G.zeros(c, torch.float32)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    eoq.eoq_gn_fwd(G.handle(), d, x, None, None, y, stats, None, None, ws)
    eoq.eoq_gn_bwd(G.handle(), d, dy, None, x, None, None, None, None, stats, dx, dgamma, dbeta, ws)
    torch.cuda.synchronize()
    rstd = 1 / np.sqrt(a * a + 1e-5)
    mean_got, rstd_got = stats.double().cpu().numpy().reshape(-1, 2).T
    assert np.abs(mean_got).max() <= 128 * EPS32 * a and np.abs(rstd_got / rstd - 1).max() <= 128 * EPS32
    s1, s2 = (up + down) / 2, (up - down) / 2 * a * rstd         # the means of dy and of dy u
    size = (abs(up) + abs(down)) / 2                             # of |dy|; |u| is at most 1
    both = float(n) * hw
    assert np.abs(dbeta.double().cpu().numpy() - both * s1).max() <= 128 * EPS32 * both * size
    # (the forward pass's rounding of mean and rstd comes on top: u is off by up to 256 steps)
    assert np.abs(dgamma.double().cpu().numpy() - both * s2).max() <= (128 + 256) * EPS32 * both * size
    for sign, e in ((1.0, up), (-1.0, down)):
        got = dx[(signs == sign).expand_as(dx)]
        want = rstd * (e - s1 - sign * a * rstd * s2)
        room = rstd * (128 + 2 * 384 + 8) * EPS32 * size
        room += half * (abs(want) + room)
        assert max(abs(float(got.max()) - want), abs(float(got.min()) - want)) <= room
