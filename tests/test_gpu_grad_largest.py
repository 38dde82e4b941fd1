"""The largest norms that are fp32 numbers: written, not raised, and clipped by like any other."""
import pytest
import torch

import lin_reference as ref
from gpu_util import status_clear
from paper_2105_13890_b200 import build
from test_gpu_grad import DEV, F32, NORM, SUM, call, norm_of

build.build_lib()
pytestmark = pytest.mark.gpu
MOST = torch.finfo(torch.float32).max


# (2^115 beside the largest number: a root that is rounded to it; elements apart, so that some are added in pieces that are whole and some in those that are not)
@pytest.mark.parametrize("values,size", [([MOST], 1), ([-MOST, 1.0], 9), ([MOST, 2.0 ** 115], 5000), ([0.7 * MOST, -0.7 * MOST], 20000), ([0.999 * MOST], 64)])
@pytest.mark.parametrize("inside", [True, False])
def test_largest_norms(values, size, inside):
    t = torch.zeros(size, device=DEV)
    t[torch.linspace(0, size - 1, len(values), device=DEV).long()] = torch.tensor(values, device=DEV)
    before = t.clone()
    whole = norm_of([t])
    assert whole <= MOST * (1 + 2.0 ** -25)                         # (what is rounded to the largest number at most)
    status_clear()
    norm = float(call([t]))
    assert norm <= MOST and abs(norm - whole) <= NORM * whole and status_clear() == 0
    out = torch.full_like(t, 7.0)
    limit = 2.0 ** 100
    assert float(call([t], limit, None if inside else [out])) == norm and status_clear() == 0
    want = before.double() * (limit / whole)
    ref.near(t if inside else out, want, 1.01 * (SUM + 3 * F32) * want.abs() + 2 * ref.LEAST[torch.float32])
    assert inside or torch.equal(t, before)
