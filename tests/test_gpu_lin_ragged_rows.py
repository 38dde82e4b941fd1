"""Rows whose ends leave some threads of a warp with less than others, at every alignment: maxima over whole rows all the same, however many rows a block has."""
import pytest
import torch

import lin_reference as ref
from gpu_util import handle, status_clear
from paper_2105_13890_b200 import build, eoq
from test_gpu_lin import DEV, TYPES, Layer, rows_in

build.build_lib()
pytestmark = pytest.mark.gpu

# Columns beside the row's own, and elements in front of it: 16-bit rows are 16-, 8-, 4- and 2-byte aligned, fp32 ones 16-, 8- and 4-byte aligned, whatever the columns are
# (`to` rounds the stride up to a multiple of elements).
ALIGN = [(8, 0), (8, 4), (8, 2), (8, 1), (4, 0), (2, 0), (1, 0)]
COLS = [1, 2, 3, 5, 7, 9, 12, 15, 17, 21, 30, 33, 50, 63, 65, 70, 100, 101, 127, 129, 131, 196, 200, 201, 255, 257, 300, 513, 978, 1001, 1031, 2047, 2805]


def beside_of(cols, to):
    return -cols % to


@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("to,offset", ALIGN)
@pytest.mark.parametrize("rows", [549, 4100, 20_003])
def test_gradients(rows, to, offset, dtype):
    for c_out in COLS:
        if rows * c_out > 1 << 23:
            continue
        l = Layer(rows, 16, c_out, dtype, True, beside_of(c_out, to), offset)
        l.code_weights()
        eoq.eoq_lin_quantize(handle(), l.x, TYPES[dtype], rows, 16, 16 + l.beside, l.x_codes, l.x_scales)
        status_clear()
        l.backward(True, False, False)
        dx = l.dx.clone()
        l.check_backward(True, False, False)
        l.dx.fill_(float("nan"))
        l.backward()
        assert status_clear() == 0
        assert torch.equal(l.dx, dx), c_out
        l.check_backward()


@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("to,offset", ALIGN)
@pytest.mark.parametrize("rows", [1, 5, 8, 31, 1000, 30_001])
def test_codes(rows, to, offset, dtype):
    """Coded by the call alone, in front of the tiles and by the kernel for a few tokens."""
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    for cols in COLS + [4099, 8195, 16_390, 20_007]:
        if rows * cols > 1 << 23:
            continue
        beside = beside_of(cols, to)
        src = rows_in(torch.randn(rows, cols, generator=g, device=DEV).to(dtype), beside, offset)
        codes, scales = torch.full((rows, eoq.lin_pitch(cols)), 77, dtype=torch.int8, device=DEV), torch.full((rows,), -7.0, device=DEV)
        status_clear()
        eoq.eoq_lin_quantize(handle(), src, TYPES[dtype], rows, cols, cols + beside, codes, scales)
        assert status_clear() == 0
        want, exact = ref.codes_of(src)
        assert torch.equal(codes[:, :cols].double(), want) and torch.equal(scales.double(), exact), cols
        if rows <= 8:
            l = Layer(rows, cols, 24, dtype, True, beside, offset)
            l.x.copy_(src)
            l.code_weights()
            l.forward(keep=False)
            l.check_forward()
            y = l.y.clone()
            l.forward()
            assert torch.equal(l.y, y), cols
