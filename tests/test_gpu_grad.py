"""Norm and clipping of gradients on a GPU against sums in 64 bits."""
import math
import random

import pytest
import torch

import lin_reference as ref
from gpu_util import handle, status_clear
from paper_2105_13890_b200 import build, eoq

build.build_lib()
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = (torch.float32, torch.float16, torch.bfloat16)
F32 = ref.HALF[torch.float32]
# The squares of eight elements are added in fp32: four in a row in each of two chains, then both, 5 roundings of at most F32 of the sum; these sums in 64 bits.  A
# root halves what the sum is off by, and its result is rounded to fp32: 2.5 + 1 roundings.
SUM, NORM = 1.01 * 2.5 * F32, 1.01 * 3.5 * F32


def tensors(sizes, seed=0, types=TYPES, spread=1.0):
    """Gradients at all alignments of their types."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = random.Random(seed)
    out = []
    for k, n in enumerate(sizes):
        t = types[k % len(types)]
        at = rng.randrange(9)
        flat = torch.randn(n + 16, generator=g, device=DEV) * math.exp(rng.gauss(0.0, spread))
        out.append(flat.to(t)[at:at + n])
    return out


def norm_of(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts if t.numel()))


def call(ts, max_norm=None, out=None):
    l = eoq.grad_list(ts, out)
    ws = torch.full((eoq.eoq_grad_workspace_size(l),), 255, dtype=torch.uint8, device=DEV)
    norm = torch.full((1,), -1.0, device=DEV)
    if max_norm is None:
        eoq.eoq_grad_norm(handle(), l, norm, ws)
    else:
        eoq.eoq_grad_clip(handle(), l, max_norm, norm, ws)
    return norm


SETS = [[1], [5], [0, 3, 0], [64], [1000, 1, 17], [8192], [8193, 8191, 16385], [3] * 40, [100_003, 7, 64, 512, 1_000_001], list(range(300)), [11] * 600 + [200_000], [5_000_011]]


@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%d tensors" % len(s))
def test_norm(sizes):
    ts = tensors(sizes)
    status_clear()
    got, want = float(call(ts)), norm_of(ts)
    assert abs(got - want) <= NORM * want and status_clear() == 0


@pytest.mark.parametrize("inside", [False, True])
@pytest.mark.parametrize("limit", [0.25, 4.0, 0.0])
@pytest.mark.parametrize("sizes", SETS, ids=lambda s: "%d tensors" % len(s))
def test_clip(sizes, limit, inside):
    ts = tensors(sizes, 1)
    before = [t.clone() for t in ts]
    whole = norm_of(ts)
    max_norm = float(torch.tensor(limit * whole))
    rng = random.Random(2)
    room = [torch.full((t.numel() + 32,), 7.0, dtype=t.dtype, device=DEV) for t in ts]
    ats = [rng.randrange(9) for _ in ts]
    out = None if inside else [r[a:a + t.numel()] for r, a, t in zip(room, ats, ts)]
    norm = float(call(ts, max_norm, out))
    assert abs(norm - whole) <= NORM * whole
    factor = min(1.0, max_norm / whole)
    for b, t, o in zip(before, ts, ts if inside else out):
        want = b.double() * factor
        if factor == 1.0:
            assert torch.equal(o, b)
        else:
            # the factor is an fp32 number and as far off as the norm, the product one, the output its type's
            ref.near(o, want, 1.01 * (SUM + 2 * F32 + ref.HALF[b.dtype]) * want.abs() + 2 * ref.LEAST[b.dtype])
        assert inside or torch.equal(t, b)
    if not inside:
        assert all(bool((r[:a] == 7).all() and (r[a + t.numel():] == 7).all()) for r, a, t in zip(room, ats, ts))


@pytest.mark.parametrize("size", [1e-36, 1e-30, 1e-20, 1e-12, 1e-11, 1e18, 1e19, 3e37])
def test_sizes_of_gradients(size):
    """Squares of small and large gradients are numbers too."""
    for t in (torch.float32, torch.bfloat16):
        ts = [(torch.linspace(-1, 1, 100, device=DEV) * size).to(t), torch.full((3,), size, device=DEV).to(t)]
        want = norm_of(ts)
        assert abs(float(call(ts)) - want) <= NORM * want


@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38])
def test_norms_that_no_number_holds(value):
    """Raised, written as they are, and the gradients left alone."""
    ts = [torch.ones(1000, device=DEV), torch.full((2,), value, device=DEV), torch.ones(9, device=DEV, dtype=torch.float16)]
    before = [t.clone() for t in ts]
    for clip in (None, 1.0):
        status_clear()
        n = float(call(ts, clip))
        assert (math.isnan(n) if math.isnan(value) else n == math.inf) and status_clear() == eoq.EOQ_DEV_NONFINITE
    assert all(torch.equal(t.nan_to_num(5), b.nan_to_num(5)) for t, b in zip(ts, before))


def test_same_bits_every_time_and_replayed():
    ts = tensors([70_000, 3, 1_000_000, 513], 4)
    out = [torch.empty_like(t) for t in ts]
    l = eoq.grad_list(ts, out)
    ws, norm = torch.empty(eoq.eoq_grad_workspace_size(l), dtype=torch.uint8, device=DEV), torch.empty(1, device=DEV)
    step = lambda: eoq.eoq_grad_clip(handle(), l, 1.0, norm, ws)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        for t in ts:
            t.mul_(1.0 - 0.3 * k)
        graph.replay()
        torch.cuda.synchronize()
        first = [norm.clone()] + [o.clone() for o in out]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, [norm] + out))


def test_a_step_of_two_layers():
    """Group norm between two integer layers, their gradients' norm, and the clipped step, as a program runs them."""
    from test_gpu_lin import Layer

    a, b = Layer(2 * 49, 128, 256, torch.float32, seed=1), Layer(2 * 49, 256, 64, torch.float32, seed=2)
    desc = eoq.gn_desc(2, 49, 256, 8, eoq.EOQ_F32, eoq.EOQ_ACT_SILU)
    gamma, beta, stats = torch.ones(256, device=DEV), torch.zeros(256, device=DEV), torch.empty(2, 8, 2, device=DEV)
    dgamma, dbeta, ws = torch.empty(256, device=DEV), torch.empty(256, device=DEV), torch.empty(eoq.eoq_gn_workspace_size(desc), dtype=torch.uint8, device=DEV)
    for l in (a, b):
        l.code_weights()
    a.forward()
    eoq.eoq_gn_fwd(handle(), desc, a.y, gamma, beta, b.x, stats, None, None, ws)
    b.forward()
    b.backward()
    eoq.eoq_gn_bwd(handle(), desc, b.dx, None, a.y, None, None, gamma, beta, stats, a.dy, dgamma, dbeta, ws)
    a.backward()
    for l in (a, b):
        l.check_forward()
        l.check_backward()
    grads = [a.dw, a.db, dgamma, dbeta, b.dw, b.db]
    before = [g.clone() for g in grads]
    whole = norm_of(grads)
    norm = float(call(grads, 0.5))
    assert abs(norm - whole) <= NORM * whole and whole > 0.5
    for g, p in zip(grads, before):
        ref.near(g, p.double() * (0.5 / whole), (SUM + 4 * F32) * p.double().abs() + 2.0 ** -149)
