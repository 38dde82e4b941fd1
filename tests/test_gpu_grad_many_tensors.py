"""Norm and clipping of more gradients than one launch takes (960): the launches' sums together, batches without elements, in place and into other tensors."""
import pytest
import torch

import lin_reference as ref
from gpu_util import status_clear
from paper_2105_13890_b200 import build, eoq
from test_gpu_grad import DEV, F32, NORM, SUM, call, norm_of, tensors
from gpu_util import handle

build.build_lib()
pytestmark = pytest.mark.gpu
SETS = {"961": [5] * 961, "2000": [(7 * k) % 300 for k in range(2000)], "first batch empty": [0] * 960 + [3000, 1, 0, 17], "last batch empty": [9000, 33] + [0] * 958 + [0] * 40,
        "middle batch empty": [4] * 960 + [0] * 960 + [100_000, 3], "the last alone": [0] * 1920 + [1], "many": [1, 0, 2] * 7000, "large and many": [300_000, 5] * 500 + [11] * 1000}


@pytest.mark.parametrize("name", list(SETS))
def test_norm(name):
    ts = tensors(SETS[name], 3)
    status_clear()
    got, want = float(call(ts)), norm_of(ts)
    assert want > 0 and abs(got - want) <= NORM * want and status_clear() == 0


@pytest.mark.parametrize("inside", [False, True])
@pytest.mark.parametrize("name", list(SETS))
def test_clip(name, inside):
    ts = tensors(SETS[name], 5)
    before = [t.clone() for t in ts]
    whole = norm_of(ts)
    max_norm = float(torch.tensor(0.3 * whole))
    out = None if inside else [torch.full_like(t, 7.0) for t in ts]
    status_clear()
    assert abs(float(call(ts, max_norm, out)) - whole) <= NORM * whole and status_clear() == 0
    for dtype in {t.dtype for t in ts}:
        got, old = (torch.cat([t for t in l if t.dtype == dtype]) for l in (ts if inside else out, before))
        want = old.double() * (max_norm / whole)
        ref.near(got, want, 1.01 * (SUM + 2 * F32 + ref.HALF[dtype]) * want.abs() + 2 * ref.LEAST[dtype])
    assert inside or all(torch.equal(t, b) for t, b in zip(ts, before))


def test_nothing_at_all():
    ts = [torch.empty(0, device=DEV) for _ in range(1000)]
    status_clear()
    assert float(call(ts)) == 0.0 and float(call(ts, 1.0)) == 0.0 and float(call(ts, 0.0)) == 0.0 and status_clear() == 0


@pytest.mark.parametrize("at", [0, 959, 960, 1999])
def test_a_number_that_is_not_finite(at):
    """In whichever batch it is."""
    ts = [torch.ones(3, device=DEV) for _ in range(2000)]
    ts[at][1] = float("inf")
    status_clear()
    assert float(call(ts, 1.0)) == float("inf") and status_clear() == eoq.EOQ_DEV_NONFINITE
    assert all(bool((t == 1).all()) for k, t in enumerate(ts) if k != at)


def test_captured_and_replayed():
    ts = tensors([50, 3, 0, 2000] * 500, 6)
    out = [torch.empty_like(t) for t in ts]
    l = eoq.grad_list(ts, out)
    ws, norm = torch.empty(eoq.eoq_grad_workspace_size(l), dtype=torch.uint8, device=DEV), torch.empty(1, device=DEV)
    step = lambda: eoq.eoq_grad_clip(handle(), l, 1.0, norm, ws)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(2):
        for t in ts:
            t.mul_(0.7)
        graph.replay()
        torch.cuda.synchronize()
        first = [norm.clone()] + [o.clone() for o in out]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, [norm] + out))
