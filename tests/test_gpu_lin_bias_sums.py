"""Sums of the bias's gradient: no error is left out or counted twice at any length, sums are as near as their order allows, and the bits are the same whatever else the
call is asked for."""
import pytest
import torch

from gpu_util import status_clear
from paper_2105_13890_b200 import build
from test_gpu_lin import DEV, Layer

build.build_lib()
pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
ASKED = [(False, False), (True, False), (False, True), (True, True)]      # dx, dw beside it
# strips put together by the second look, by a kernel of its own; one group of columns a block, two; columns that one thread or a whole block shares
SIZES = [(1, 24), (7, 40), (97, 520), (700, 1000), (1301, 333), (3000, 300), (4099, 33), (20001, 264), (100001, 17), (270001, 3), (65537, 96), (9001, 1031), (33, 70001),
         (140, 2000), (200, 600), (256, 64), (249, 4099), (500, 1900)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("beside,offset", [(0, 0), (24, 8), (3, 1)])
@pytest.mark.parametrize("rows,c_out", SIZES)
def test_every_error_once(rows, c_out, beside, offset, dtype):
    """Whole numbers, whose sums fp32 holds in any order: the sums are exact."""
    l = Layer(rows, 16, c_out, dtype, True, beside, offset)
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + c_out)
    dy = torch.randint(-60, 61, (rows, c_out), generator=g, device=DEV)
    assert 60 * rows < 1 << 24
    l.dy.copy_(dy)
    l.code_weights()
    l.forward()
    want = dy.sum(0).float()
    for dx, dw in ASKED:
        l.db.fill_(float("nan"))
        l.backward(dx, dw, True)
        assert torch.equal(l.db, want)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,c_out", SIZES)
def test_same_bits_whatever_else_is_asked_for(rows, c_out, dtype):
    l = Layer(rows, 16, c_out, dtype)
    l.code_weights()
    l.forward()
    status_clear()
    got = []
    for dx, dw in ASKED:
        l.db.fill_(float("nan"))
        l.backward(dx, dw, True)
        got.append(l.db.clone())
    assert status_clear() == 0
    assert all(torch.equal(g, got[0]) for g in got[1:])
    # A value goes through at most 512 strips' sums in a row, those of 256 threads in front of it, and a thread's own additions, two of each pair of rows: a strip's rows over
    # the threads that share them.  Strips: 1/512 of the rows, or 1/(444 / groups of columns), at least eight rows; threads of a column: at least eight.
    groups = max(1, -(-c_out // 128))
    strip = max(8, -(-rows // max(1, min(512, 444 // groups))))
    depth = 512 + 256 + -(-strip // 8) + 2
    exact = l.dy.double().sum(0)
    assert bool(((got[0].double() - exact).abs() <= depth * 2.0 ** -24 * l.dy.double().abs().sum(0)).all())
