"""Backward passes whose two products share a launch of single blocks and go out in different ways, one by tensor copies, one row by row: the same bits as each product
in a call of its own, every time."""
import pytest
import torch

from gpu_util import status_clear
from paper_2105_13890_b200 import build
from test_gpu_lin import Layer

build.build_lib()
pytestmark = pytest.mark.gpu


# Rows of dx that are not whole pieces of 16 bytes, rows of dw that are (fp32 channels in fours); tiles of 32, 64 and 128 columns, many units a block.
@pytest.mark.parametrize("rows,c_in,c_out,dtype,beside", [(4000, 68, 32, torch.bfloat16, 0), (9000, 132, 128, torch.float16, 0), (9000, 132, 128, torch.float32, 3), (20000, 100, 64, torch.float16, 0),
                                                          (30000, 196, 96, torch.bfloat16, 0), (30000, 260, 256, torch.bfloat16, 0), (105151, 540, 96, torch.float16, 24)])
def test_same_bits_as_calls_of_their_own(rows, c_in, c_out, dtype, beside):
    l = Layer(rows, c_in, c_out, dtype, True, beside)
    l.code_weights()
    l.forward()
    l.backward(dx=True, dw=False, db=False)
    l.backward(dx=False, dw=True, db=False)
    dx, dw = l.dx.clone(), l.dw.clone()
    status_clear()
    for _ in range(8):
        l.dx.fill_(float("nan"))
        l.dw.fill_(float("nan"))
        l.backward()
        assert torch.equal(l.dx, dx) and torch.equal(l.dw, dw)
    assert status_clear() == 0
    l.check_backward(db=False)
