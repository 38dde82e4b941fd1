"""Forms of the integer linear layers' kernels that only larger or stranger calls take, each against the plain forms."""
import pytest
import torch

import lin_reference as ref
from gpu_util import handle, status_clear
from paper_2105_13890_b200 import build, eoq
from test_gpu_lin import DEV, TYPES, Layer, rows_in

build.build_lib()
pytestmark = pytest.mark.gpu


# Errors of more than 2^22 values in rows of more than 256 (fp32: 128) that are 16-byte aligned: the first look takes two groups of columns a block.
@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("rows,c_out,beside", [(5003, 1024, 0), (16001, 300, 4), (4201, 1031, 1), (17001, 264, 8), (9001, 520, 0), (41, 110_000, 0), (33_001, 160, 0), (70_001, 257, 7)])
def test_first_look_of_two_groups(rows, c_out, beside, dtype):
    l = Layer(rows, 16, c_out, dtype, True, beside)
    l.code_weights()
    l.forward()
    status_clear()
    for dx, dw, db in ((True, True, True), (False, True, False), (False, False, True), (True, False, True), (True, True, False)):
        for t in (l.dx, l.dw, l.db):
            t.fill_(float("nan"))
        l.backward(dx, dw, db)
        l.check_backward(dx, dw, db)
    assert status_clear() == 0


@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("rows,c_out,beside", [(5003, 1024, 0), (9001, 521, 7)])
def test_first_look_of_two_groups_without_codes(rows, c_out, beside, dtype):
    """Errors that are not finite, at the ends of groups and rows."""
    l = Layer(rows, 16, c_out, dtype, True, beside)
    l.code_weights()
    l.forward()
    for k, (t, o) in enumerate(((0, 0), (rows - 1, c_out - 1), (rows // 2, 255), (7, 256), (8, 511), (9, 512))):
        l.dy[t, o] = (float("inf"), float("nan"), float("-inf"))[k % 3]
    status_clear()
    l.backward()
    assert status_clear() == eoq.EOQ_DEV_NONFINITE
    l.check_backward(db=False)
    assert int(torch.isnan(l.dx).all(1).sum()) == 6 and int(torch.isnan(l.dw).all(1).sum()) == 6 and int((~torch.isfinite(l.db)).sum()) == 6


# Gradient of the tokens alone: errors coded by rows with the columns' scales in them, rows of one value to more than a block's threads hold.
@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("beside,offset", [(0, 0), (24, 8), (4, 4), (2, 2), (3, 1)])
@pytest.mark.parametrize("rows,c_out", [(1, 1), (3, 15), (700, 96), (65, 513), (1500, 300), (130, 2051), (9, 4100), (21, 9000), (5, 20_001), (3, 40_008)])
def test_gradient_of_tokens_alone(rows, c_out, beside, offset, dtype):
    l = Layer(rows, 48, c_out, dtype, True, beside, offset)
    l.code_weights()
    status_clear()
    l.backward(True, False, False)
    assert status_clear() == 0
    l.check_backward(True, False, False)
    l.untouched()
    l.dy[rows - 1, c_out - 1] = float("nan")
    l.backward(True, False, False)
    assert status_clear() == eoq.EOQ_DEV_NONFINITE
    l.check_backward(True, False, False)


# Tiles of two blocks, more than three for each pair, so that accumulators, stages and staging go round; outputs by tensor copies and row by row.
@pytest.mark.parametrize("dtype,rows,c_in,c_out,beside", [(torch.bfloat16, 16384, 128, 2048, 0), (torch.float16, 16384, 2048, 512, 0), (torch.float32, 16000, 500, 1999, 1), (torch.bfloat16, 16001, 1003, 2001, 0),
                                                           (torch.float16, 33_000, 300, 530, 6)])
def test_pairs_of_many_tiles(dtype, rows, c_in, c_out, beside):
    l = Layer(rows, c_in, c_out, dtype, True, beside)
    l.code_weights()
    status_clear()
    l.forward()
    l.backward()
    assert status_clear() == 0
    l.check_codes()
    l.check_forward()
    l.check_backward()
    l.untouched()
    first = [t.clone() for t in (l.y, l.dx, l.dw, l.db)]
    for _ in range(3):
        l.forward()
        l.backward()
        assert all(torch.equal(p, q) for p, q in zip(first, (l.y, l.dx, l.dw, l.db)))


@pytest.mark.parametrize("dtype", list(TYPES), ids=str)
@pytest.mark.parametrize("beside,offset", [(0, 0), (24, 8), (4, 4), (2, 2), (3, 1)])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 17), (5, 255), (40, 256), (1000, 63), (33, 1025), (2000, 520), (7, 8193), (2, 50_001), (70_000, 5)])
def test_codes_of_rows(rows, cols, beside, offset, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + cols)
    src = rows_in((torch.randn(rows, cols, generator=g, device=DEV) * torch.exp(3.0 * torch.randn(rows, 1, generator=g, device=DEV))).to(dtype), beside, offset)
    pitch = eoq.lin_pitch(cols)
    codes, scales = torch.full((rows + 1, pitch), 77, dtype=torch.int8, device=DEV), torch.full((rows + 1,), -7.0, device=DEV)
    status_clear()
    eoq.eoq_lin_quantize(handle(), src, TYPES[dtype], rows, cols, cols + beside, codes, scales)
    # (some rows of many are beyond what fp16 holds: infinite, without codes)
    assert status_clear() == (0 if bool(torch.isfinite(src).all()) else eoq.EOQ_DEV_NONFINITE)
    want, exact = ref.codes_of(src)
    assert torch.equal(codes[:rows, :cols].double(), want) and torch.equal(scales[:rows].double().nan_to_num(-1.0), exact.nan_to_num(-1.0))
    assert bool((codes[rows] == 77).all()) and float(scales[rows]) == -7.0
