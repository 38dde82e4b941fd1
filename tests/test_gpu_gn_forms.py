"""Which form of group norm a call takes, told by its launches."""
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G
import wide_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,c", [("fp16", 1056), ("bf16", 1056), ("fp32", 544)])
def test_groups_that_fit_wide_vectors_alone(name, c):
    """Groups of 33 and 17 channels in whole blocks of the 8-bit form: 132 or 136 wide vectors to a chunk, twice as many narrow ones.  Few
    samples, so that the wide form leaves SMs without a block; it keeps its vectors and is one launch all the same."""
    td, ed = {"fp16": (torch.float16, eoq.EOQ_F16), "bf16": (torch.bfloat16, eoq.EOQ_BF16), "fp32": (torch.float32, eoq.EOQ_F32)}[name]
    n, hw, groups = 1, 50, 32
    x = torch.randn(n, hw, c, generator=torch.Generator().manual_seed(c)).to(td).to("cuda:0")
    d = eoq.gn_desc(n, hw, c, groups, ed, eoq.EOQ_ACT_SILU)
    y, stats = torch.empty_like(x), G.zeros((n, groups, 2), torch.float32)
    codes, exps = G.zeros((n, hw, c), torch.int8), G.zeros((n * hw, c // 32), torch.uint8)
    ws = G.empty(eoq.eoq_gn_workspace_size(d), torch.uint8)
    before = eoq.eoq_launch_count(G.handle())
    eoq.eoq_gn_fwd(G.handle(), d, x, None, None, y, stats, codes, exps, ws)
    assert eoq.eoq_launch_count(G.handle()) - before == 1
    xw = x.double().cpu().numpy()
    want, _, _, bound = R.gn_fwd(xw, groups, 1e-5, 1.0, 0.0, "silu")
    R.within(y.double().cpu().numpy(), want, bound, name)
    want_codes, want_exps, _ = R.block_form(xw.reshape(-1, c))
    assert (G.host(codes).reshape(-1, c) == want_codes).all() and (G.host(exps) == want_exps).all()
